"""CPU-only, read off the source: a pair of CTAs whose roles give up.  A copy that one role asked for may be on its way when
another, which waits for it, gives up, in the same CTA or in the other: both CTAs stay until it has landed."""
import re

import pytest

from test_drains import _code

PAIRS = ["expert_product.cu", "mx_product.cu"]


def _function(code, name):
    body = code[code.index(name):]
    return body[:body.index("\n}\n")]


@pytest.mark.parametrize("name", PAIRS)
def test_whoever_gives_up_tells_both_ctas(name):
    code = _code(name)
    wait = _function(code, "bool wait_for(")
    assert re.search(r"give_up<CG>\(quit\);\s*return false", wait)
    told = _function(_code("tcgen05.cuh"), "void give_up(")
    assert "*quit = 1" in told and "mapa.shared::cluster" in told and "st.shared::cluster" in told and "cluster_rank() ^ 1u" in told
    # nobody sets the flag in another way
    assert "*quit = 1" not in code and len(re.findall(r"\*quit = 0", code)) == 1


@pytest.mark.parametrize("name", PAIRS)
def test_both_ctas_stay_until_copies_have_landed(name):
    code = _code(name)
    end = code[max(code.rindex("tc_fence_before();\n    " + meet) for meet in ("cluster_sync();", "if (CG == 2) cluster_sync();") if "tc_fence_before();\n    " + meet in code):]
    end = end[:end.index("tmem_dealloc")]
    # the verdict is read behind the meeting of the pair, so it is the same in both
    m = re.search(r"(?:cluster_sync|__syncthreads)\(\);\s*if \(\*quit\) \{(.*?)\n    \}\n", end, re.S)
    assert m, end
    body = m.group(1)
    assert re.search(r"warp == kTmaWarp.*drain_wait\(&full\[", body, re.S)
    assert body.index("drain_wait") < body.index("cluster_sync();") < body.index("report_status")
    # and no role's own verdict decides about its copies
    assert not re.search(r"if \(!ok\) \{[^}]*drain_wait\(&full", code)


def test_what_one_cta_writes_for_the_others_mmas_is_ordered_by_a_barrier_that_counts_it():
    """An arrival at the other CTA announces that an accumulator has been read, and nothing that was written."""
    code = _code("expert_product.cu")
    assert set(re.findall(r"mbar_arrive_lead<CG>\(&(\w+)\[", code)) == {"acc_empty"}
    second = code[code.index("kMmaWarp && kGrad"):]
    assert "load_zero_tail(" in second and "clear_tail(" not in second.replace("load_zero_tail(", "")


def test_the_zeros_behind_a_segment_are_whole_and_only_there():
    """Boxes of 1, 2, 4 and 8 lines, as load_zero_tail takes them, for every end within a K = 16."""
    code = _code("expert_product.cu")
    assert "return 16 - (left & 15);" in code and "if (tail_lines(left) & (1 << b))" in code and "at += 1 << b;" in code
    assert "encode(&zeros.lines[b], bf16, CU_TENSOR_MAP_SWIZZLE_NONE, a.a, 2, ad, as, 64, 1 << b)" in code
    for left in (v for v in range(1, 64) if v & 15):
        at, lines = left, []
        for b in range(4):
            if (16 - (left & 15)) & (1 << b):
                assert at % (1 << b) == 0
                lines += range(at, at + (1 << b))
                at += 1 << b
        assert lines == list(range(left, (left + 15) // 16 * 16)) and len(lines) == 16 - (left & 15) and max(lines) < 64
