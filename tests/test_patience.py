"""CPU-only: the longest wait of a weights' gradient.  The second CTA of a pair passes over the tiles whose segments end with a whole K =
16 and waits for the one that does not, through all of them."""
import re

from test_drains import _code
from test_network_refusals import _printed

MOST = 1 << 24


def test_polls_grow_with_what_is_waited_for_and_stay_bounded(tmp_path):
    calls = [(0, 2000, 0), (0, 2000, 17), (5000, 2000, 17), (0, 0, 1), (0, 1 << 20, 1 << 24), (MOST, (1 << 31) - 1, 1 << 24), (MOST - 1, 0, 1), (7, (1 << 31) - 1, 0)]
    assert MOST * 4e-6 < 100                                   # seconds: a poll takes 7800 clocks at most
    got = _printed(tmp_path, "expert_product.h", [f"more_patience({a}u, {b}u, {c})" for a, b, c in calls])
    assert got == [min(MOST, a + min(b, MOST) + 64 * c) for a, b, c in calls]


def test_the_wait_for_a_segments_end_counts_the_tiles_before_it():
    code = _code("expert_product.cu")
    role = code[code.index("kMmaWarp && kGrad"):]
    loop = role[role.index("for (TileStream"):]
    assert loop.index("patience = more_patience(patience, p.spin_limit, steps)") < loop.index("has_tail(")     # of every tile
    assert re.search(r"wait_for\(&tail\[at\], [^;]*max\(p\.spin_limit, patience\)\)", loop) and "patience = 0;" in loop
