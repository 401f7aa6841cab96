"""Softmax weights far below a row's largest: many slots that share a small weight beside one slot that takes most of it.

One slot (`heavy`) has score x, all n others score 0, so that each of these weighs w = exp(-x) against the heavy one's 1.  With V = 0 in
the heavy slot and 1 in the others, out = n w / (1 + n w) in every element: what the small weights add up to, alone.

Tolerance, with u = 2^-24, h = half a step of the element type: scale x log2(e) is off by 3 half steps of fp32, the exponential by
2^-21, a sum of n terms by n u, in the numerator and in the denominator; each weight is rounded to the element type, by h w, or in fp16
by half a step of the subnormals, 2^-25, where the largest weight stands for 2^9.9: n 2^-34.9; the result is rounded once."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2605_16941_gb300 as wino  # noqa: E402
from kv_helpers import CAUSAL, FULL, U, add_rows, attend, check, half_step, make_kv  # noqa: E402

BF, FP = torch.bfloat16, torch.float16


@pytest.mark.parametrize("dtype", [FP, BF], ids=["fp16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("slots,bits,heavy", [(32768, 20.4, 0), (32768, 24.4, 0), (32768, 25.2, 100), (262144, 24.4, 0),
                                              (262144, 25.2, 0), (262144, 30.7, 5), (5000, 15.3, 4999), (5000, 18.6, 70)])
def test_many_small_weights(slots, bits, heavy, dim, dtype):
    """Rows in both row tiles of as many sequences as keep a task's slots in one part, all over the same pages."""
    n_seq, rows, page = 152, 256, 128
    pages = -(-slots // page)
    k = torch.zeros((pages, page, 1, dim), dtype=dtype, device="cuda")
    v = torch.ones_like(k)
    k[heavy // page, heavy % page, 0, 0] = 16.0
    v[heavy // page, heavy % page] = 0.0
    table = torch.arange(pages, dtype=torch.int32, device="cuda").repeat(n_seq, 1)
    ints = torch.tensor([[rows * s for s in range(n_seq)], [rows] * n_seq, [slots] * n_seq, [0] * n_seq], dtype=torch.int32,
                        device="cuda")
    b = wino.make_kv_batch(k, v, table, *ints, n_rows=n_seq * rows, n_q_heads=1, mask=FULL)
    q = torch.zeros((n_seq * rows, 1, dim), dtype=dtype, device="cuda")
    q[..., 0] = 1.0
    out = torch.empty_like(q)
    scale = float(np.float32(bits * math.log(2.0) / 16.0))
    ws = wino.attend_workspace(b)
    wino.wino_attend(q, out, b, ws, scale=scale)
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    n, w, h = slots - 1, math.exp(-16.0 * scale), half_step(dtype)
    want = n * w / (1.0 + n * w)
    tol = want * 2 * (3 * U * bits + 2.0 ** -21 + n * U) + 1.01 * h * 2 * want
    if dtype == FP:
        tol += n * 2.0 ** -34.9 / (1.0 + n * w) + 2.0 ** -25
    off = (out.double() - want).abs().max().item()
    assert off <= tol, f"{out.flatten()[0].item()} for {want}: off by {off} at tolerance {tol}"


@pytest.mark.parametrize("spread", [8.0, 30.0])
@pytest.mark.parametrize("dim", [64, 128])
def test_peaked_softmax_fp16(dim, spread):
    """Scores that move the running maximum by far from tile to tile: no weight leaves fp16's range."""
    c = add_rows(make_kv(CAUSAL, [(40, 700, 660), (300, 900, 600)], heads=4, kv_heads=2, dim=dim, dtype=FP, spread=spread),
                 spread=2.0)
    ws = attend(c)
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    check(c)


@pytest.mark.parametrize("rise", [0.5, 1.0, 3.0, 4.0, 4.5, 8.0, 9.0])
def test_maximum_that_rises_by_steps(rise):
    """The maximum grows by `rise` bits from tile to tile, around what the running maximum lets pass: the largest weights that
    may stand beside it."""
    slots, dim = 1280, 64
    c = make_kv(FULL, [(256, slots, 0)], heads=1, dim=dim, dtype=FP, page=128, poison=False)
    c.k_cache.zero_()
    for t in range(slots // 128):
        c.k_cache[int(c.table[0, t]), :, 0, 0] = rise * t / 8.0
    add_rows(c)
    c.q.zero_()
    c.q[..., 0] = 8.0
    scale = float(np.float32(math.log(2.0)))
    ws = attend(c, scale=scale)
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    check(c, scale=scale)
