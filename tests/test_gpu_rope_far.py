"""wino_rope_append: turns of far positions at any frequency, against angles in exact rational arithmetic.

Tolerance: the turn is position times a fraction that is off by 2^-63 turns at most, so 2^-32 turns at positions up to 2^31, and its
value in fp32 by 2^-25 turns: with pi 2^-24 and the functions' two half steps under 2^-22 in cos and sin; the rest as in
test_gpu_rope.py."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2605_16941_gb300 as wino  # noqa: E402
from kv_helpers import CAUSAL, f64, half_step, make_kv  # noqa: E402

PI = Fraction(31415926535897932384626433832795028841971693993751058209749445923078164062862, 10 ** 76)
POSITIONS = [0, 1, -1, (1 << 20) + 3, 1 << 24, (1 << 24) + 1, 123456789, -123456789, 2147483647, -2147483647]


def turned(x, positions, freq):
    """Pairs (j, j + rot / 2), x float64 [rows, heads, rot]."""
    half = len(freq)
    y = x.copy()
    for r, p in enumerate(positions):
        for j, f in enumerate(freq):
            turns = p * Fraction(float(f)) / (2 * PI)
            t = 2 * math.pi * float(turns - round(turns))
            c, s = math.cos(t), math.sin(t)
            a, b = x[r, :, j], x[r, :, j + half]
            y[r, :, j], y[r, :, j + half] = a * c - b * s, b * c + a * s
    return y


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("freqs", ["theta", "high", "tiny"])
def test_far_turns(freqs, dtype):
    rot = 32
    j = np.arange(rot // 2)
    freq = {"theta": 500000.0 ** (-2.0 * j / rot), "high": 1.0e3 * 3.7 ** j, "tiny": 1e-9 / (1.0 + j)}[freqs]
    n = len(POSITIONS)
    c = make_kv(CAUSAL, [(n, n, 0)], heads=2, kv_heads=1, dim=rot, dtype=dtype, poison=False)
    g = torch.Generator().manual_seed(3)
    q, k = (torch.randn((n, h, rot), generator=g).to(dtype).cuda() for h in (2, 1))
    rope = wino.make_rope(torch.from_numpy(freq).cuda(), rot_dim=rot,
                          positions=torch.tensor(POSITIONS, dtype=torch.int32, device="cuda"))
    out, ws = torch.empty_like(q), wino.append_workspace()
    wino.wino_rope_append(q, k, k, c.batch, rope, ws, q_out=out)
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    slots = np.arange(n)
    cached = f64(c.k_cache)[c.table[0, slots // c.page], slots % c.page]
    for x, got in ((f64(q), f64(out)), (f64(k), cached)):
        want = turned(x, POSITIONS, freq)
        size = np.abs(x) + np.abs(np.roll(x, rot // 2, -1))
        tol = 2.0 ** -20 * size + 1.001 * half_step(dtype) * np.abs(want)
        if dtype == torch.float16:
            tol = tol + 2.0 ** -25
        d = np.abs(got - want)
        assert (d <= tol).all(), f"off by {d.max()}"
