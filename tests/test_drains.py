"""CPU-only: the waits of a role that gave up.  Its copies and products in flight must land before shared memory and
TMEM are given back, however few polls a context allows its ordinary waits (MOE_TUNE_SPIN_LIMIT may be 0).  Nothing
makes a copy not arrive without a fault, so this is read off the kernels' source: every wait on a barrier is either
one that gives up (it counts polls against the context's limit and then clears a verdict) or the one drain, which
takes no limit from the context."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2602_21140_b200", "csrc")
FILES = ["scatter_kernels.cuh", "combine_kernels.cuh", "backward_kernels.cuh", "mx_product.cu"]


def _code(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


@pytest.mark.parametrize("name", FILES)
def test_every_other_wait_gives_up(name):
    code = _code(name)
    waits = list(re.finditer(r"(while|for)\s*\([^{;]*(;[^{;]*)?mbar_try_wait\(", code))
    assert len(waits) >= 1
    for m in waits:
        end = re.search(r"[;}]\s*\n\s*\n|\n\s*(?=while|for|const|auto|__)", code[m.end():])
        body = code[m.start():m.end() + (end.start() if end else 300)]
        assert re.search(r"\+\+spins > (p\.spin_limit|limit)", body), body
        assert re.search(r"ok = false|return false", body), body
    assert "drain_wait(" in code


def test_the_drain_has_a_limit_of_its_own():
    code = _code("device_utils.cuh")
    body = code[code.index("void drain_wait("):]
    body = body[:body.index("\n}\n")]
    assert "spin_limit" not in body and "kDrainPolls" in body and "globaltimer" in body
    ns = int(re.search(r"kDrainNs = (\d+)ull \* 1000 \* 1000", code).group(1)) * 10 ** 6
    polls = 1 << int(re.search(r"kDrainPolls = 1u << (\d+)", code).group(1))
    assert ns >= 10 ** 7                     # a copy takes microseconds
    assert polls * 10 >= ns                  # a poll takes 10 ns at least: the polls do not end it before the time
