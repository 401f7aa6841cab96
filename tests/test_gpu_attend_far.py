"""Scores of any finite size: the weights depend on differences, and those of far scores are exact where they matter.

Every product here is a power of two times a small integer, so that the scores are exact in fp32.  Slots below a row's maximum
lie so far below that they weigh nothing; the n slots that share it weigh the same, whose weight is rounded once to the element type
(half a step h) and cancels but for that; the result is rounded once: 2.02 h mean |V|, and 2^-20 for the sums' and the quotient's fp32."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2605_16941_gb300 as wino  # noqa: E402
from kv_helpers import FULL, half_step  # noqa: E402

BF, FP = torch.bfloat16, torch.float16


def run(score, rows, dim, dtype, scale, size, sign=1.0):
    """out [rows, dim] of rows whose scores are `score` [slots] (small integers) times `size` squared, a power of two."""
    slots, page = score.numel(), 128
    pages = -(-slots // page)
    g = torch.Generator().manual_seed(slots)
    k = torch.zeros((pages * page, 1, dim), dtype=dtype)
    k[:slots, 0, 0] = (score * size).to(dtype)
    v = torch.zeros((pages * page, 1, dim), dtype=dtype)
    v[:slots] = torch.randn((slots, 1, dim), generator=g).to(dtype)
    kc, vc = (t.view(pages, page, 1, dim).cuda() for t in (k, v))
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, -1)
    ints = torch.tensor([[0], [rows], [slots], [0]], dtype=torch.int32, device="cuda")
    b = wino.make_kv_batch(kc, vc, table, *ints, n_rows=rows, n_q_heads=1, mask=FULL)
    q = torch.zeros((rows, 1, dim), dtype=dtype, device="cuda")
    q[..., 0] = sign * size
    out = torch.empty_like(q)
    ws = wino.attend_workspace(b)
    wino.wino_attend(q, out, b, ws, scale=scale)
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    top = score == score.max() if sign > 0 else score == score.min()
    V = v[:slots, 0][top].double()
    want, tol = V.mean(0), 2.02 * half_step(dtype) * V.abs().mean(0) + 2.0 ** -20
    off = (out[:, 0].cpu().double() - want).abs()
    assert (off <= tol).all(), f"off by {off.max().item()}, {out[0, 0, :4].tolist()} for {want[:4].tolist()}"


SIZES = [(FP, 2.0 ** e) for e in (2, 5, 9, 11, 12)] + [(BF, 2.0 ** e) for e in (2, 5, 9, 12, 15, 20, 50)]


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("rows", [1, 200])
@pytest.mark.parametrize("sign", [1.0, -1.0], ids=["positive", "negative"])
@pytest.mark.parametrize("dtype,size", SIZES, ids=[f"{'fp16' if d == FP else 'bf16'}-{s:g}" for d, s in SIZES])
def test_far_scores(dtype, size, sign, rows, dim):
    """A maximum that rises and falls over the tiles and is shared by slots of several of them; scores far from zero."""
    j = torch.arange(900)
    score = 4.0 + (j // 64 % 9).float()  # 4 .. 12, equal over 64 slots at a time
    run(score, rows, dim, dtype, 37.0, size, sign)


@pytest.mark.parametrize("dtype", [FP, BF], ids=["fp16", "bf16"])
@pytest.mark.parametrize("scale", [2.0 ** 20 * 1.37, 2.0 ** 60, 2.0 ** 90 * 1.1, 2.0 ** -3 * 1.61])
def test_far_by_the_scale(scale, dtype):
    j = torch.arange(700)
    run(3.0 + (j // 100 % 5).float(), 150, 64, dtype, scale, 256.0)


@pytest.mark.parametrize("dtype", [FP, BF], ids=["fp16", "bf16"])
@pytest.mark.parametrize("size", [16.0, 256.0, 1024.0, 4096.0])
def test_maximum_shared_by_every_slot(size, dtype):
    """Equal scores far from zero: the mean of V."""
    run(torch.full((1000,), 15.0), 40, 64, dtype, 0.773, size)
