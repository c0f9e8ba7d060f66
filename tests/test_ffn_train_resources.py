"""Register budget of the kernels that train a gated FFN (CPU; compiles for gfx950), and the
products' rings of stages."""
import os
from concurrent.futures import ThreadPoolExecutor

import pytest

from test_kernel_resources import HIPCC
from test_norm_q8_resources import _kernels

SOURCES = ("gated.hip", "linear_grad.hip", "residual.hip", "residual_grad.hip")


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
def test_no_spills(tmp_path):
    """No scratch memory but in the gradient of fp32 rows of 1537 to 2048 vectors, whose
    1024 threads have 128 registers each; two waves a SIMD for the largest tiles."""
    with ThreadPoolExecutor(len(SOURCES)) as ex:
        found = dict(zip(SOURCES, ex.map(lambda s: _kernels(s, tmp_path), SOURCES)))
    counts = {k: 0 for k in ("product_gated_kernel", "product_pair_kernel", "gated_few_kernel", "prepare_kernel", "finish_kernel",
                             "residual_kernel", "residual_grad_kernel", "residual_vectors_kernel")}
    for kernels in found.values():
        for name, (scratch, waves, _) in kernels.items():
            for k in counts:
                counts[k] += k in name
            if "Li1024EEE" in name and "residual_grad_kernel" in name:
                assert scratch <= 96 and waves == 4, (name, scratch, waves)
                continue
            assert scratch == 0, (name, scratch)
            if "product_" in name:
                assert waves >= 2, (name, waves)
            if "residual_kernel" in name:
                assert waves >= 2, (name, waves)
    assert all(counts.values()), counts


def _ring(down_a, down_b, loads_a, loads_b, stages, first):
    """The loads of one wave in the order that product.h issues them, and at each of its waits
    whether what is read next has landed and lies where it is read."""
    ra = (5 if down_b else 4) if down_a else (3 if down_b else 2)
    rb = (5 if down_a else 4) if down_b else (3 if down_a else 2)
    h0, h1 = 2 * first, 2 * (first + stages)
    per_stage = (0 if down_a else loads_a) + (0 if down_b else loads_b)
    per_half = (loads_a if down_a else 0) + (loads_b if down_b else 0)
    rh, rs = (ra if down_a else rb), (rb if down_a else ra)
    even = (rh - 2) * per_half + (rh - 1) // 2 * per_stage
    odd = (rh - 2) * per_half + (rh - 2) // 2 * per_stage
    stage = (rs - 2) * per_stage + (2 * rs - 2) * per_half
    odd = odd if down_a and down_b else min(odd, stage) if down_a or down_b else stage
    last = 2 * max(ra, rb)
    issued, landed, holds = 0, 0, {}

    def load(op, piece, slot, n):
        nonlocal issued
        issued += n
        holds[op, slot] = piece, issued

    def wait(n):
        nonlocal landed
        assert n < 64
        landed = max(landed, issued - n)

    def read(h, sa, sb):
        for op, down, slot in (("a", down_a, sa), ("b", down_b, sb)):
            piece, end = holds[op, slot]
            assert piece == (h if down else h >> 1) and end <= landed, (op, h, slot, piece, end, landed)
    for o in range(2 - last, 1):
        q = -(-o // 2) - 1
        for op, down, ring, n in (("a", down_a, ra, loads_a), ("b", down_b, rb, loads_b)):
            if not down and o % 2 == 0 and q + ring >= 0 and h0 + 2 * (q + ring) < h1:
                load(op, h0 // 2 + q + ring, q + ring, n)
        for op, down, ring, n in (("a", down_a, ra, loads_a), ("b", down_b, rb, loads_b)):
            if down and o - 1 + ring >= 0 and h0 + o - 1 + ring < h1:
                load(op, h0 + o - 1 + ring, o - 1 + ring, n)
    pa = pb = 0

    def fill(h, is_odd):
        for op, down, ring, n, at in (("a", down_a, ra, loads_a, pa), ("b", down_b, rb, loads_b, pb)):
            if not down and is_odd and 2 * ((h >> 1) + ring) < h1:
                load(op, (h >> 1) + ring, at, n)
        for op, down, ring, n, at in (("a", down_a, ra, loads_a, pa), ("b", down_b, rb, loads_b, pb)):
            if down and h + ring < h1:
                load(op, h + ring, at, n)
    wait(odd if h0 + last < h1 else 0)
    read(h0, 0, 0)
    for h in range(h0, h1, 2):
        qa, qb = (pa + 1) % ra if down_a else pa, (pb + 1) % rb if down_b else pb
        if down_a or down_b:
            wait(even if h + last < h1 else 0)
            fill(h, False)
        read(h + 1, qa, qb)
        pa, pb = qa, qb
        qa, qb = (pa + 1) % ra, (pb + 1) % rb
        wait(odd if h + last < h1 else 0)
        fill(h + 1, True)
        if h + 2 < h1:
            read(h + 2, qa, qb)
        pa, pb = qa, qb
    assert landed == issued  # none under way when the epilogue writes LDS


def test_a_ring_is_read_after_it_has_landed():
    for down in ((False, False), (False, True), (True, True)):
        for n in (1, 2, 4):  # loads a lane for half a stage
            for stages in range(1, 40):
                for first in (0, 1, 5):
                    _ring(*down, *(n if d else 2 * n for d in down), stages, first)
