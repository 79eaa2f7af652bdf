"""The gate's gradient for tokens whose -inf logits leave fewer than k selectable experts.

Routing fills such a token's last picks with the lowest available expert and the constant score 1; softmax scores are
exp(l - l_0) with l_0 the logit of the best pick.  The expected gradient is 64-bit autograd through just that, with
the selected picks found by a 64-bit selection of the test's own.

Bound: as in test_gpu_backward (a handful of fp32 operations of magnitude b_j = w_j (|g_j| + sum w |g| / c): 16 k of
2^-24 of that, and 3e-7 for sigmoid_spec); the best pick of a filled softmax token is a sum of up to k - 1 others:
their bounds added, and k roundings of at most the sum of their magnitudes (each below its b_j)."""
import numpy as np
import pytest
import torch

from paper_2602_21140_b200 import binding as B

pytestmark = pytest.mark.gpu
NEG = float("-inf")


def _select(key, k, n_group, topk_group):
    """Ids of the selected experts, best first (fewer than k where nothing is left)."""
    E = key.shape[0]
    key = key.copy()
    if n_group > 1:
        per = key.reshape(n_group, -1)
        best = -np.sort(-per, axis=1)[:, :k // topk_group]
        score = np.where(np.isinf(best[:, 0]), -np.inf, np.where(np.isinf(best), 0.0, best).sum(1))
        keep = sorted(range(n_group), key=lambda g: (-score[g], g))[:topk_group]
        for g in range(n_group):
            if g not in keep:
                per[g] = -np.inf
        key = per.reshape(E)
    order = sorted(range(E), key=lambda e: (-key[e], e))[:k]
    return [e for e in order if key[e] > -np.inf]


def _run(lg, k, score, n_group=1, topk_group=1, route_scale=1.5, failed=(), with_logits=True):
    T, E = lg.shape
    cfg = B.make_config(E, k, 32, T, E, 1, 1, score, n_group, topk_group, route_scale)
    router = B.MoeRouter(cfg, range(E), None, [1.0] * E)
    if failed:
        router.set_failed_ranks(failed)
    dev = torch.from_numpy(lg).cuda()
    g = torch.Generator(device="cuda").manual_seed(E + k)
    out = router.dispatch(dev, torch.randn(T, 32, device="cuda", generator=g).bfloat16())
    d_w = torch.randn(T, k, device="cuda", generator=g)
    d_logits = torch.full((T, E), float("nan"), device="cuda")
    router.dispatch_backward(dev if with_logits else None, out.send_buf, d_w, d_logits=d_logits)
    torch.cuda.synchronize()
    status = router.device_status()
    router.close()
    ids = out.topk_ids.cpu().numpy()
    ran_out = False
    for t in range(T):
        key = lg[t].astype(np.float64)
        if score == B.MOE_SCORE_SIGMOID:
            key = np.where(np.isneginf(key), -np.inf, 1 / (1 + np.exp(-key)))
        key[list(failed)] = -np.inf
        sel = _select(key, k, n_group, topk_group)
        r = len(sel)
        ran_out |= r < k
        assert ids[t, :r].tolist() == sel
        leaf = torch.from_numpy(lg[t].astype(np.float64)).requires_grad_()
        picked = leaf[torch.tensor(sel, dtype=torch.long)]
        u = torch.ones(k, dtype=torch.float64)
        if r:
            s = torch.sigmoid(picked) if score == B.MOE_SCORE_SIGMOID else torch.exp(picked - picked[0])
            u = torch.cat((s, torch.ones(k - r, dtype=torch.float64)))
        w = route_scale * u / u.sum()
        gt = d_w[t].double().cpu()
        want = torch.zeros(E, dtype=torch.float64)
        if r:
            (w * gt).sum().backward()
            want = leaf.grad
        w = w.detach()
        assert ((out.topk_weights[t].double().cpu() - w).abs() <= 1e-6 * w).all()
        b = w * (gt.abs() + (w * gt.abs()).sum() / route_scale)
        tol = torch.zeros(E, dtype=torch.float64)
        for j, e in enumerate(sel):
            tol[e] = b[j] * (16 * k * 2.0 ** -24 + 3e-7)
        if r < k and score == B.MOE_SCORE_SOFTMAX and r:
            tol[sel[0]] = sum(tol[e] for e in sel[1:]) + k * 2.0 ** -24 * b[1:r].sum()
        err = (d_logits[t].double().cpu() - want).abs()
        assert (err <= tol).all(), (t, r, err, tol)
    assert status == (B.MOE_ERR_INSUFFICIENT_EXPERTS if ran_out else 0)


@pytest.mark.parametrize("score", [B.MOE_SCORE_SOFTMAX, B.MOE_SCORE_SIGMOID])
@pytest.mark.parametrize("E,k", [(8, 2), (16, 4), (12, 8), (32, 1), (24, 16)])
def test_fewer_selectable_experts_than_picks(score, E, k):
    """A token for every number of selectable experts from none to k + 1, the lowest expert among them or not."""
    rng = np.random.default_rng(E * k)
    rows = []
    for r in range(k + 2):
        for low in (True, False):
            row = np.full(E, NEG, np.float32)
            pool = np.arange(1, E)
            chosen = rng.choice(pool, min(r, E - 1), replace=False)
            if low and r:
                chosen[0] = 0
            row[chosen] = rng.standard_normal(chosen.size)
            rows.append(row)
    _run(np.stack(rows), k, score)
    _run(np.stack(rows), k, score, failed=(0,))          # the fill is then another expert


@pytest.mark.parametrize("score", [B.MOE_SCORE_SOFTMAX, B.MOE_SCORE_SIGMOID])
def test_equal_logits_and_unmasked_tokens(score):
    """Ties look like fills by their weights, but are not; and an ordinary token in between."""
    lg = np.zeros((4, 8), np.float32)
    lg[1, 1:] = NEG
    lg[2] = np.linspace(-1, 1, 8)
    lg[3, [0, 3]] = NEG
    _run(lg, 2, score)
    _run(lg, 8, score)


@pytest.mark.parametrize("score", [B.MOE_SCORE_SOFTMAX, B.MOE_SCORE_SIGMOID])
def test_the_fill_is_unmasked_but_its_group_was_not_kept(score):
    """Four groups of four, two kept: the kept ones have one to four selectable experts, and the fill, expert 0, has an
    ordinary logit in a group that was dropped, kept, or empty."""
    E, k = 16, 4
    rows = []
    for n1, n2 in ((1, 1), (2, 1), (1, 2), (2, 2), (3, 0), (1, 0), (4, 1)):
        for first in ([-9.0] * 4, [NEG] * 4, [-9.0, NEG, NEG, NEG], [9.0, NEG, NEG, NEG]):
            row = np.full(E, NEG, np.float32)
            row[:4] = first
            row[8:8 + n1] = 3.0 + 0.25 * np.arange(n1)
            row[12:12 + n2] = 2.0 + 0.25 * np.arange(n2)
            rows.append(row)
    _run(np.stack(rows), k, score, n_group=4, topk_group=2)


def test_softmax_without_logits_where_no_token_ran_out():
    rng = np.random.default_rng(5)
    lg = rng.standard_normal((9, 16)).astype(np.float32)
    lg[:, 3] = NEG
    _run(lg, 4, B.MOE_SCORE_SOFTMAX, with_logits=False)
    _run(lg, 4, B.MOE_SCORE_SOFTMAX, n_group=4, topk_group=2, with_logits=False)
