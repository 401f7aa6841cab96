"""Rows of an 8-bit cache that are held as NaN, under wino_attend_scaled for more than a few rows: the rows that see the slot
get NaN in that kv head's query heads, and all others bit for bit what they get without it."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2605_16941_gb300 as wino  # noqa: E402
from cache8_helpers import BF, FP, NAN, attend8, make_kv8  # noqa: E402
from kv_helpers import CAUSAL, FULL, SHADOW, add_rows, check_on_device, sees  # noqa: E402

CASES = {
    # name: (mask, sequences, slots of the first sequence that are held as NaN, other arguments of make_kv)
    "causal": (CAUSAL, [(60, 60, 0)], [40], {}),
    "causal_first_and_last": (CAUSAL, [(60, 60, 0)], [0, 59], {}),
    "causal_behind_a_context": (CAUSAL, [(300, 700, 400), (40, 90, 50)], [411, 415, 530, 531, 699], {}),
    "causal_long": (CAUSAL, [(200, 5000, 4800)], [4900, 4999], dict(page=64)),
    "causal_in_the_context": (CAUSAL, [(200, 5000, 4800)], [17], dict(page=64)),
    "full": (FULL, [(40, 300, 0), (20, 50, 0)], [130], {}),
    "shadow_block_slot": (SHADOW, [(64, 300, 200)], [205], {}),
    "shadow_shadow_slot": (SHADOW, [(64, 300, 200), (64, 200, 100)], [307], {}),
    "shadow_hole_and_another": (SHADOW, [(64, 300, 200)], [203, 229], {}),
    "shadow_hole_and_shadow": (SHADOW, [(64, 300, 200)], [203, 331], {}),
    "shadow_two_row_tiles": (SHADOW, [(400, 900, 600)], [650, 1000], dict(page=128)),
    "one_row_tile_in_two_halves": (SHADOW, [(64, 640, 500)], [5, 639], dict(layout="heads")),
}


def hold_as_nan(c, name, slot, head):
    """Of the first sequence, as an append writes it: codes of 0 and a scale of 255."""
    page, at = c.table[0, slot // c.page], slot % c.page
    c.extra[name + "8"].view(torch.uint8)[page, at, head] = 0
    c.extra[name + "_scale"][page, head, at] = NAN


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("of", ["k", "v", "kv"])
@pytest.mark.parametrize("name", CASES)
def test_rows_that_see_it_and_no_others(name, of, dim, dtype):
    mask, seqs, slots, kw = CASES[name]
    c = add_rows(make_kv8(mask, seqs, heads=4, kv_heads=2, dim=dim, dtype=dtype, gap=1, **kw))
    ws = attend8(c)
    check_on_device(c)
    without = c.out.clone()
    for slot in slots:
        for x in of:
            hold_as_nan(c, x, slot, 1)
    c.out.fill_(77.0)
    attend8(c, ws=ws)
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    n, kv, new = seqs[0]
    hit = np.zeros(c.n_rows, dtype=bool)
    hit[c.starts[0]:c.starts[0] + n] = [np.isin(slots, sees(mask, n, kv, new, i)).any() for i in range(n)]
    hit = torch.from_numpy(hit).cuda()
    assert torch.equal(c.out[:, :2], without[:, :2])  # the other kv head
    assert torch.equal(c.out[~hit, 2:], without[~hit, 2:])
    assert torch.isnan(c.out[hit, 2:].float()).all()


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128])
def test_more_such_rows_than_a_warp_notes(dim, dtype):
    """A run of them, in K or V or both, then none in the next call of the same workspace."""
    c = add_rows(make_kv8(CAUSAL, [(150, 400, 250)], heads=4, kv_heads=2, dim=dim, dtype=dtype, poison=False))
    ws = attend8(c)
    without = c.out.clone()
    keep = {x: c.extra[x].clone() for x in ("k8", "v8", "k_scale", "v_scale")}
    for of in ("v", "k", "kv"):
        for slot in range(300, 390):
            for x in of:
                hold_as_nan(c, x, slot, 0)
        attend8(c, ws=ws)
        assert torch.equal(c.out[:50], without[:50]) and torch.equal(c.out[:, 2:], without[:, 2:])
        assert torch.isnan(c.out[50:, :2].float()).all()
        for x, t in keep.items():
            c.extra[x].copy_(t)
        attend8(c, ws=ws)
        assert torch.equal(c.out, without) and wino.wino_read_device_status(ws) == wino.WINO_OK


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
def test_an_overflowed_value_of_a_prompt(dtype):
    """As it comes about: one infinity in a value row that wino_norm_rope_append stores, over the prompt that it belongs to."""
    c = add_rows(make_kv8(CAUSAL, [(100, 100, 0)], heads=4, kv_heads=2, dim=128, dtype=dtype, poison=False))
    g = torch.Generator().manual_seed(5)
    k, v = (torch.randn((c.n_rows, 2, 128), generator=g).to(dtype).cuda() for _ in range(2))
    ws = wino.attend_workspace(c.batch)
    rope, outs = wino.make_rope(None, rot_dim=0), []
    for bad in (False, True):
        if bad:
            v[70, 1, 9] = float("inf")
        wino.wino_norm_rope_append(None, k, v, c.batch, rope, ws)
        attend8(c, ws=ws)
        assert wino.wino_read_device_status(ws) == wino.WINO_OK
        outs.append(c.out.clone())
    assert torch.equal(outs[0][:70], outs[1][:70]) and torch.equal(outs[0][:, :2], outs[1][:, :2])
    assert torch.isnan(outs[1][70:, 2:].float()).all()
