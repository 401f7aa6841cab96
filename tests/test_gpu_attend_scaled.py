"""wino_attend_scaled against the definition in 64 bits over the values that codes and scales stand for (kv_helpers, with its
tolerances): masks, lengths around tiles and pages, head layouts, types, scales that differ from slot to slot, rows that see nothing,
poisoned slots, and what a batch's device arrays may hold."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2605_16941_gb300 as wino  # noqa: E402
from cache8_helpers import BF, FP, NAN, attend8, make_kv8, rebatch  # noqa: E402
from kv_helpers import CAUSAL, FULL, SHADOW, add_rows, check, check_on_device  # noqa: E402


def run(c, **kw):
    ws = attend8(c, **kw)
    torch.cuda.synchronize()
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    return check(c)


CASES = {
    # name: (mask, [(rows, kv_len, new_slot)], other arguments of make_kv)
    "one_slot": (CAUSAL, [(1, 1, 0)], {}),
    "one_token": (CAUSAL, [(1, 300, 299)], dict(heads=8, kv_heads=2, dim=128)),
    "no_slots": (FULL, [(3, 0, 0), (2, 5, 0)], {}),
    "empty_and_absent": (FULL, [(0, 40, 0), (2, 0, 0), (0, 0, 0), (4, 33, 0)], dict(gap=3, dim=128)),
    "causal_first_rows": (CAUSAL, [(5, 5, 0), (7, 3, 0)], {}),
    "left_padding": (CAUSAL, [(9, 5, -4), (3, 0, -3)], dict(dim=128)),
    "tile_edges": (CAUSAL, [(1, n, n - 1) for n in (127, 128, 129, 255, 256, 257, 385)], dict(gap=1)),
    "tile_edges_128": (CAUSAL, [(3, n, n - 3) for n in (127, 128, 129, 255, 256, 257, 385, 640)], dict(dim=128, heads=8, kv_heads=2)),
    "pages_of_16": (FULL, [(3, n, 0) for n in (15, 16, 17, 47, 145)], {}),
    "pages_of_32": (FULL, [(3, n, 0) for n in (31, 33, 161)], dict(page=32, layout="heads")),
    "pages_of_64": (FULL, [(3, n, 0) for n in (63, 65, 200)], dict(page=64, dim=128)),
    "pages_of_128": (FULL, [(3, n, 0) for n in (128, 129, 300)], dict(page=128, layout="heads", dim=128)),
    "pages_of_384": (FULL, [(3, n, 0) for n in (384, 385, 500)], dict(page=384)),
    "shadow_1": (SHADOW, [(2, 1, 0), (2, 9, 8), (2, 9, 0)], {}),
    "shadow_32": (SHADOW, [(64, 96, 64), (64, 64, 0), (64, 200, 100)], dict(heads=4, kv_heads=4, dim=128)),
    "shadow_tile_edge": (SHADOW, [(6, 126, 123), (6, 128, 125), (8, 127, 120)], dict(heads=4, kv_heads=2)),
    "shadow_right_context": (SHADOW, [(20, 300, 40)], dict(dim=128, layout="heads")),
    "shadow_large": (SHADOW, [(300, 700, 500)], dict(heads=2, kv_heads=1, dim=64, page=64)),
    "shadow_large_128": (SHADOW, [(300, 900, 500)], dict(heads=2, kv_heads=1, dim=128, page=32, layout="heads")),
    "full_130_rows": (FULL, [(130, 257, 0)], dict(heads=1)),
    "causal_prompt": (CAUSAL, [(300, 300, 0)], dict(heads=3, kv_heads=3, dim=128)),
    "causal_ragged": (CAUSAL, [(70, 170, 100), (1, 400, 399), (129, 129, 0), (2, 2, 0)], dict(gap=2, order=[2, 0, 3, 1])),
    "causal_ragged_128": (CAUSAL, [(70, 170, 100), (1, 400, 399), (129, 129, 0), (2, 2, 0)], dict(gap=2, order=[2, 0, 3, 1], dim=128, heads=6, kv_heads=2)),
    "group_7": (CAUSAL, [(40, 140, 100), (1, 60, 59)], dict(heads=14, kv_heads=2)),
    "group_5_dim_80": (SHADOW, [(20, 50, 30)], dict(heads=10, kv_heads=2, dim=80)),
    "group_128": (CAUSAL, [(3, 200, 197)], dict(heads=128, kv_heads=1)),
    "group_100": (CAUSAL, [(3, 200, 197)], dict(heads=100, kv_heads=1, dim=128)),
    "dim_16": (FULL, [(5, 140, 0)], dict(dim=16)),
    "dim_32": (FULL, [(5, 140, 0)], dict(dim=32, layout="heads", kv_heads=2)),
    "dim_48": (FULL, [(5, 140, 0)], dict(dim=48)),
    "dim_96": (CAUSAL, [(50, 140, 90)], dict(dim=96, heads=6, kv_heads=2)),
    "dim_112": (CAUSAL, [(5, 140, 135)], dict(dim=112, layout="heads")),
    "many_short": (CAUSAL, [(1 + i % 3, 1 + (7 * i) % 90, (7 * i) % 90 - i % 3) for i in range(500)], {}),
    "long": (CAUSAL, [(1, 5000, 4999), (2, 9000, 8998)], dict(heads=8, kv_heads=2, dim=128, page=64)),
    "long_rows": (CAUSAL, [(140, 3000, 2860)], dict(heads=4, kv_heads=2, dim=128, page=32)),
    "long_rows_64": (CAUSAL, [(140, 3000, 2860)], dict(heads=4, kv_heads=2, dim=64, page=16)),
}


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("name", CASES)
def test_against_definition(name, dtype):
    mask, seqs, kw = CASES[name]
    run(add_rows(make_kv8(mask, seqs, dtype=dtype, **kw)))


@pytest.mark.parametrize("dtype,wild", [(BF, 6), (FP, 6)], ids=["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128])
def test_scales_that_differ_from_slot_to_slot(dim, dtype, wild):
    run(add_rows(make_kv8(CAUSAL, [(40, 500, 460), (3, 77, 74)], dtype=dtype, wild=wild, heads=4, kv_heads=2, dim=dim, spread=0.05)))


@pytest.mark.parametrize("layout", ["slots", "heads"])
def test_strided_rows(layout):
    run(add_rows(make_kv8(CAUSAL, [(33, 150, 117), (1, 20, 19)], heads=6, kv_heads=2, layout=layout, gap=1), strided=True))


def test_combined_cache():
    """K and V in one allocation, [pages, 2, slots, heads, dim]: views with one set of strides."""
    c = make_kv8(SHADOW, [(32, 90, 60)], heads=4, kv_heads=2)
    both = torch.stack([c.extra["k8"].view(torch.uint8), c.extra["v8"].view(torch.uint8)], dim=1).contiguous()
    c.extra["k8"], c.extra["v8"] = both[:, 0], both[:, 1]
    run(add_rows(rebatch(c)))


@pytest.mark.parametrize("spread", [8.0, 30.0])
def test_peaked_softmax(spread):
    """Scores that move the running maximum by far from tile to tile, and rows whose weights all but one vanish."""
    run(add_rows(make_kv8(CAUSAL, [(40, 700, 660)], heads=4, kv_heads=2, dim=128, spread=spread), spread=2.0))


def test_scale():
    c = add_rows(make_kv8(CAUSAL, [(4, 50, 46)]))
    attend8(c, scale=0.37)
    torch.cuda.synchronize()
    check(c, scale=0.37)


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128])
def test_many_rows_on_the_device(dim, dtype):
    c = add_rows(make_kv8(CAUSAL, [(700, 2100, 1400), (1, 1500, 1499), (300, 300, 0)], heads=8, kv_heads=2, dim=dim, page=32, dtype=dtype))
    attend8(c)
    check_on_device(c)


def test_a_row_that_is_held_as_nan():
    """NaN where it is seen, nothing where not: causal rows in front of it and the shadow row that verifies it."""
    c = make_kv8(CAUSAL, [(60, 60, 0)], heads=2, kv_heads=2, dim=128)
    page, at = c.table[0, 40 // 16], 40 % 16
    c.extra["v_scale"][page, 1, at] = NAN
    add_rows(c)
    attend8(c)
    out = c.out[c.starts[0]:].float()
    assert torch.isfinite(out[:, 0]).all()  # the other head
    assert torch.isnan(out[40:, 1]).all()


def test_workspace_is_reused_as_it_is():
    """One workspace through calls of other shapes, calls of wino_attend among them, and twice the same call: bit for bit the same."""
    big = add_rows(make_kv8(CAUSAL, [(200, 1000, 800), (1, 3000, 2999)], heads=8, kv_heads=2, dim=128))
    ws = wino.attend_workspace(big.batch)
    run(big, ws=ws)
    first = big.out.clone()
    for mask, seqs in ((SHADOW, [(64, 500, 400)]), (FULL, [(1, 0, 0)])):
        c = add_rows(make_kv8(mask, seqs, heads=4, kv_heads=2, poison=False))
        run(c, ws=ws)
        wino.wino_attend(c.q, c.out, c.extra["plain"], ws)
    big.out.fill_(77.0)
    run(big, ws=ws)
    assert torch.equal(first, big.out)


def test_captured_call_takes_new_lengths():
    seqs = [(4, 900, 896), (1, 300, 299)]
    c = add_rows(make_kv8(CAUSAL, seqs, heads=8, kv_heads=2, dim=128, poison=False))
    ws = wino.attend_workspace(c.batch)
    run(c, ws=ws)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        attend8(c, ws=ws)
    for lens in ([(4, 500, 496), (1, 301, 300)], [(3, 17, 14), (1, 0, 0)], seqs):
        c.seqs = lens
        c.ints[1:].copy_(torch.tensor([[s[i] for s in lens] for i in range(3)], dtype=torch.int32))
        c.extra["whole"].fill_(77.0)
        g.replay()
        torch.cuda.synchronize()
        assert wino.wino_read_device_status(ws) == wino.WINO_OK
        check(c)


def test_bad_pages_are_an_error_and_others_stay_right():
    c = add_rows(make_kv8(CAUSAL, [(3, 200, 197), (2, 90, 88)], heads=4, kv_heads=2, dim=128))
    for bad in (-1, c.extra["k8"].size(0), 1 << 30):
        c.table_dev[0, 3] = bad
        ws = attend8(c)
        assert wino.wino_read_device_status(ws) == wino.WINO_ERR_ARG
        c.table_dev.copy_(torch.from_numpy(c.table))
        run(c, ws=ws)


def test_bad_lengths_are_an_error():
    c = add_rows(make_kv8(CAUSAL, [(3, 200, 197), (2, 90, 88)], heads=4, kv_heads=2, dim=64))
    for row, value in ((0, -1), (1, -2), (2, 1 << 20), (1, 1 << 24)):
        keep = c.ints.clone()
        c.ints[row, 0] = value
        ws = attend8(c)
        assert wino.wino_read_device_status(ws) == wino.WINO_ERR_ARG
        c.ints.copy_(keep)
        c.extra["whole"].fill_(77.0)
        run(c, ws=ws)


def test_an_append_error_reaches_the_attention():
    """As with the plain calls: the append leaves its error for the attention of the same workspace."""
    c = add_rows(make_kv8(CAUSAL, [(4, 40, 36)], heads=4, kv_heads=2))
    ws = wino.attend_workspace(c.batch)
    keep = c.table_dev.clone()
    c.table_dev[0, 2] = -5
    k = torch.randn((c.n_rows, 2, 64)).to(BF).cuda()
    rope = wino.make_rope(None, rot_dim=0)
    wino.wino_norm_rope_append(None, k, k, c.batch, rope, ws)
    c.table_dev.copy_(keep)
    attend8(c, ws=ws)
    assert wino.wino_read_device_status(ws) == wino.WINO_ERR_ARG
    attend8(c, ws=ws)
    assert wino.wino_read_device_status(ws) == wino.WINO_OK


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("name", ["empty_and_absent", "tile_edges_128", "shadow_32", "shadow_large", "shadow_large_128", "causal_prompt",
                                  "causal_ragged_128", "group_5_dim_80", "dim_96", "long_rows", "long_rows_64"])
def test_bit_for_bit_the_attention_over_the_values(name, dtype):
    """More than a few rows per sequence: codes become tiles of the element type without rounding, and everything behind them is the
    same as over the element type."""
    mask, seqs, kw = CASES[name]
    c = add_rows(make_kv8(mask, seqs, dtype=dtype, poison=False, **kw))
    attend8(c)
    first = c.out.clone()
    c.out.fill_(77.0)
    plain = wino.make_kv_batch(c.k_cache, c.v_cache, c.table_dev, *c.ints, n_rows=c.n_rows, n_q_heads=c.heads, mask=mask)
    wino.wino_attend(c.q, c.out, plain, wino.attend_workspace(plain))
    assert torch.equal(c.out, first)


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128])
def test_every_call_gives_the_same(dim, dtype):
    """A thousand calls behind one another: codes that a copy overwrites while they are read would show."""
    c = add_rows(make_kv8(CAUSAL, [(700, 2100, 1400), (1, 1500, 1499), (300, 300, 0)], heads=8, kv_heads=2, dim=dim, page=32, dtype=dtype))
    ws = attend8(c)
    first, off = c.out.clone(), torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(1000):
        c.out.fill_(77.0)
        attend8(c, ws=ws)
        off += (c.out != first).sum()
    assert off.item() == 0 and wino.wino_read_device_status(ws) == wino.WINO_OK
