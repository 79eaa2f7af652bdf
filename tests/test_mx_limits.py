"""CPU-only: the products' integer limits, compiled for the host from the header that the kernels use."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2602_21140_b200", "csrc")


def _run(tmp_path, body: str) -> list:
    """Lines that a host program prints which includes mx_product.h."""
    src, exe = tmp_path / "limits.cu", tmp_path / "limits"
    src.write_text('#include <stdio.h>\n#include "mx_product.h"\nusing namespace moe;\nint main()\n{\n' + body + "\nreturn 0;\n}\n")
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.check_call([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-I", CSRC, "-o", str(exe), str(src)])
    return subprocess.check_output([str(exe)], text=True).split()


def test_sums_of_tiles_saturate(tmp_path):
    limit = int(_run(tmp_path, 'printf("%d", kTooManyTiles);')[0])
    assert 2 * limit < 1 << 31
    cases = [(0, 0), (5, 7), (limit - 1, 0), (limit - 1, 1), (limit, 0), (0, limit), (limit, limit - 1), (limit - 1, limit), (limit, limit)]
    got = _run(tmp_path, "\n".join(f'printf("%d\\n", tiles_sum({a}, {b}));' for a, b in cases) + r'''
    // inclusive prefixes the way the kernel forms them: shuffled sums of 32 lanes, then the warps before
    int v[32], n[32];
    for (int l = 0; l < 32; ++l) v[l] = 1 << 26;
    for (int off = 1; off < 32; off <<= 1) {
        for (int l = 0; l < 32; ++l) n[l] = l >= off ? tiles_sum(v[l], v[l - off]) : v[l];
        for (int l = 0; l < 32; ++l) v[l] = n[l];
    }
    int total = 0, sorted = 1;
    for (int w = 0; w < 18; ++w) total = tiles_sum(total, v[31]);
    for (int l = 1; l < 32; ++l) sorted &= v[l] >= v[l - 1];
    printf("%d %d %d\n", v[0], total, sorted);''')
    assert [int(x) for x in got[:len(cases)]] == [min(a + b, limit) for a, b in cases]
    assert got[len(cases):] == [str(1 << 26), str(limit), "1"]


def test_sizes_that_the_kernels_numbers_cannot_hold_are_refused(tmp_path):
    """Whatever is accepted, the rounding up to a pair of tiles (2 x 128 features) and the first feature of the last
    tile stay ints, and so do rows rounded up to a tile."""
    top = 2 ** 31 - 1
    cases = [(1, 8, 32, 1, 1), (1, 1 << 30, 32, 1, 1), (1 << 30, 8, 32, 1, 1),
             (1, top - 7, 32, 1, 0), (1, top - 255, 32, 1, 0), (1, top, 32, 4, 0), (1, (1 << 30) + 8, 32, 1, 0),
             ((1 << 30) + 1, 8, 32, 1, 0), (1 << 30, 1 << 30, 32, 1, 0), (1, 1 << 30, 2048, 1, 0), (1, 1 << 25, 32, 4096, 0)]
    got = _run(tmp_path, "\n".join(f'printf("%d\\n", (int)product_fits({r}ll, {n}ll, {k}ll, {p}));' for r, n, k, p, _ in cases) + """
    printf("%d\\n", (int)((long long)kMaxFeatures + 2 * 2 * 128 < (1ll << 31) && (long long)kMaxRows + 2 * 224 < (1ll << 31)));""")
    assert [int(x) for x in got] == [c[4] for c in cases] + [1]
