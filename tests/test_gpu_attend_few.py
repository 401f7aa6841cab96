"""wino_attend_scaled for sequences of few rows, whose codes go straight to the tensor cores, against the definition in 64 bits
(kv_helpers, with its tolerances): groups, dims, lengths around its 32 slots and 15 warps, parts over several CTAs, scales of any
size, and rows beyond what it expects."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2605_16941_gb300 as wino  # noqa: E402
from cache8_helpers import BF, FP, NAN, attend8, in_layout, make_kv8, quantise, rebatch, values_of  # noqa: E402
from kv_helpers import CAUSAL, FULL, SHADOW, add_rows, check  # noqa: E402


def run(c, **kw):
    ws = attend8(c, **kw)
    torch.cuda.synchronize()
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    return check(c, scale=kw.get("scale"))


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 7, 8])
@pytest.mark.parametrize("dim", [64, 128])
def test_groups(dim, group, dtype):
    run(add_rows(make_kv8(CAUSAL, [(1, n, n - 1) for n in (1, 33, 700)], heads=2 * group, kv_heads=2, dim=dim, dtype=dtype)))


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("group", [9, 10, 11, 12, 14, 16, 32])
def test_groups_of_more_than_a_tile(group, dtype):
    """Heads of a kv head in two tiles where 5, 6, 7 or 8 divide them; the others beside them."""
    for mask, seqs in ((CAUSAL, [(1, n, n - 1) for n in (1, 33, 700)]), (SHADOW, [(2, 90, 89), (0, 9, 0), (0, 9, 0), (2, 33, 0)])):
        run(add_rows(make_kv8(mask, seqs, heads=3 * group, kv_heads=3, dim=128, dtype=dtype, layout="heads")))


@pytest.mark.parametrize("dim", [16, 32, 48, 80, 96, 112])
@pytest.mark.parametrize("layout", ["slots", "heads"])
def test_dims(dim, layout):
    run(add_rows(make_kv8(CAUSAL, [(1, 150, 149), (2, 75, 73)], heads=4, kv_heads=2, dim=dim, layout=layout, page=32)))


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_lengths(page):
    """Around a warp's 32 slots, rounds of 11, slot tiles and pages."""
    run(add_rows(make_kv8(CAUSAL, [(1, n, n - 1) for n in (1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 351, 352, 353, 384, 704, 705)],
                          heads=4, kv_heads=1, dim=128, page=page, gap=1)))


@pytest.mark.parametrize("dim", [64, 128])
def test_lengths_around_a_round(dim):
    """Of 15 warps: 480 slots."""
    run(add_rows(make_kv8(CAUSAL, [(1, n, n - 1) for n in (447, 448, 449, 479, 480, 481, 512, 513, 959, 960, 961, 1440)], heads=4, kv_heads=2,
                          dim=dim, page=32)))


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("group,rows", [(4, 4), (4, 3), (8, 2), (5, 2), (1, 16), (3, 4), (2, 7)])
def test_two_tiles_of_rows(group, rows, dtype):
    """Rows of a sequence and kv head in two tiles of 8, the second in part; another sequence with more, one with fewer, and some without."""
    run(add_rows(make_kv8(CAUSAL, [(rows, 700, 700 - rows), (rows + 1, 65, 64 - rows), (rows - 1, 1300, 1301 - rows)] +
                          [(0, 9, 0)] * 4, heads=2 * group, kv_heads=2, dim=128, dtype=dtype)))


@pytest.mark.parametrize("mask,seqs", [
    (CAUSAL, [(2, 90, 88), (1, 70, 69), (0, 50, 0), (2, 40, 38)]),
    (CAUSAL, [(2, 5, -1), (1, 0, 0), (1, 0, -1)]),                    # rows that see nothing
    (FULL, [(2, 90, 3), (1, 33, 0), (2, 0, 0)]),
    (SHADOW, [(2, 90, 89), (2, 33, 0), (2, 129, 64)]),                # holes at an edge, in the middle
    (CAUSAL, [(3, 300, 297), (0, 9, 0), (0, 9, 0), (0, 9, 0), (1, 2, 1)]),  # more rows in one sequence than the average
    (CAUSAL, [(20, 300, 280)] + [(0, 1, 0)] * 9),
], ids=["ragged", "nothing_seen", "full", "shadow", "uneven", "one_with_all"])
@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
def test_masks(mask, seqs, dtype):
    run(add_rows(make_kv8(mask, seqs, heads=8, kv_heads=2, dim=128, dtype=dtype)))


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("dim,heads,kv_heads", [(128, 8, 1), (64, 4, 2), (128, 32, 8)])
def test_long_contexts_in_many_parts(dim, heads, kv_heads, dtype):
    run(add_rows(make_kv8(CAUSAL, [(1, 40001, 40000), (1, 700, 699)], heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, page=64)))


def test_many_sequences():
    run(add_rows(make_kv8(CAUSAL, [(1, 1 + (37 * i) % 1500, (37 * i) % 1500) for i in range(300)], heads=8, kv_heads=2, dim=128)))


@pytest.mark.parametrize("dtype,wild", [(BF, 40), (FP, 6)], ids=["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128])
def test_scales_of_any_size(dim, dtype, wild):
    """K's scale by slot, V's by slot: weights and results over many orders of magnitude."""
    c = make_kv8(CAUSAL, [(1, 900, 899), (2, 77, 75)], dtype=dtype, wild=wild, heads=4, kv_heads=2, dim=dim, spread=1.0)
    add_rows(c, spread=1.0)
    c.q *= 2.0 ** (-wild)
    run(c)


@pytest.mark.parametrize("exponent", [-60, 0, 60, 120])
def test_queries_of_any_size(exponent):
    """Rows of q far from 1: the scale brings the scores back."""
    c = add_rows(make_kv8(CAUSAL, [(1, 300, 299), (1, 40, 39)], heads=4, kv_heads=2, dim=128))
    c.q *= 2.0 ** exponent
    c.q[0, 0] *= 2.0 ** -8
    run(c, scale=2.0 ** -exponent * 0.09)


@pytest.mark.parametrize("offset", [0.0, 1e3, 1e6])
def test_far_scores(offset):
    """A dim that adds the same large amount to all of a row's scores: the differences count."""
    c = make_kv8(CAUSAL, [(1, 400, 399)], heads=4, kv_heads=2, dim=128, poison=False)
    t = c.k_cache.double()
    t[..., 0] = 8.0
    codes, scales = quantise(t, BF)
    c.k_cache = values_of(codes, scales, BF)
    c.extra["k8"], c.extra["k_scale"] = in_layout(codes.view(torch.uint8), "slots").view(torch.float8_e4m3fn), scales
    add_rows(rebatch(c))
    c.q[..., 0] = offset
    attend8(c)
    torch.cuda.synchronize()
    # the products with the large dim are exact, the other 127 are added to them with steps of 2^-23 of the sum: kv_helpers counts that
    check(c)


def test_peaked_softmax():
    for spread in (8.0, 30.0):
        run(add_rows(make_kv8(CAUSAL, [(1, 700, 699), (2, 300, 298)], heads=4, kv_heads=2, dim=128, spread=spread), spread=2.0))


def test_nan_rows():
    """K or V held as NaN: the rows that see the slot, in that kv head, and no other."""
    for name in ("k_scale", "v_scale"):
        c = make_kv8(CAUSAL, [(2, 42, 40), (1, 42, 41)], heads=8, kv_heads=2, dim=128)
        page, at = c.table[0, 41 // 16], 41 % 16
        c.extra[name][page, 1, at] = NAN  # the last row's own slot
        add_rows(c)
        attend8(c)
        out = c.out.float()
        assert torch.isfinite(out[0]).all() and torch.isfinite(out[1, :4]).all() and torch.isnan(out[1, 4:]).all(), name
        assert torch.isfinite(out[2]).all()
    # and where it is all that a row sees
    for name in ("k_scale", "v_scale"):
        c = make_kv8(CAUSAL, [(1, 1, 0)], heads=2, kv_heads=1, dim=64)
        c.extra[name][c.table[0, 0], 0, 0] = NAN
        add_rows(c)
        attend8(c)
        assert torch.isnan(c.out.float()).all(), name


@pytest.mark.parametrize("rows", [1, 40])
def test_a_query_that_is_nan_gives_nan(rows):
    """In its row and head and no other, over few rows and over many."""
    c = add_rows(make_kv8(CAUSAL, [(rows, 500, 500 - rows)], heads=4, kv_heads=2, dim=128))
    c.q[rows - 1, 2, 7] = float("nan")
    ws = attend8(c)
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    out = torch.isnan(c.out.float())
    assert out[rows - 1, 2].all() and out.sum() == 128


def test_bad_pages_and_lengths_are_errors():
    c = add_rows(make_kv8(CAUSAL, [(1, 500, 499), (1, 90, 89)], heads=8, kv_heads=2, dim=128))
    for bad in (-1, c.extra["k8"].size(0), 1 << 30):
        c.table_dev[0, 20] = bad
        ws = attend8(c)
        assert wino.wino_read_device_status(ws) == wino.WINO_ERR_ARG
        c.table_dev.copy_(torch.from_numpy(c.table))
        run(c, ws=ws)
    for row, value in ((0, -1), (1, -2), (2, 1 << 20), (1, 1 << 24)):
        keep = c.ints.clone()
        c.ints[row, 0] = value
        ws = attend8(c)
        assert wino.wino_read_device_status(ws) == wino.WINO_ERR_ARG
        c.ints.copy_(keep)
        c.extra["whole"].fill_(77.0)
        run(c, ws=ws)


def test_captured_call_takes_new_lengths_and_other_calls_share_its_workspace():
    seqs = [(1, 900, 899), (1, 30000, 29999)]
    c = add_rows(make_kv8(CAUSAL, seqs, heads=8, kv_heads=2, dim=128, poison=False))
    big = add_rows(make_kv8(SHADOW, [(64, 500, 400)] * 3, heads=8, kv_heads=2, dim=128))
    ws = wino.attend_workspace(big.batch)
    run(c, ws=ws)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        attend8(c, ws=ws)
    for lens in ([(1, 500, 499), (1, 301, 300)], [(0, 17, 14), (1, 0, 0)], [(1, 29000, 28999), (1, 1, 0)], seqs):
        c.seqs = lens
        c.ints[1:].copy_(torch.tensor([[min(s[i], 1 << 30) for s in lens] for i in range(3)], dtype=torch.int32))
        if lens[0][1] == 29000:  # as long as the other's table
            c.seqs = lens = [lens[1], lens[0]]
            c.ints[1:].copy_(torch.tensor([[s[i] for s in lens] for i in range(3)], dtype=torch.int32))
        c.extra["whole"].fill_(77.0)
        g.replay()
        torch.cuda.synchronize()
        assert wino.wino_read_device_status(ws) == wino.WINO_OK
        check(c)
        run(big, ws=ws)


@pytest.mark.parametrize("dim", [64, 128])
def test_every_call_gives_the_same(dim):
    c = add_rows(make_kv8(CAUSAL, [(1, 20000, 19999), (1, 1500, 1499), (2, 300, 298)], heads=8, kv_heads=2, dim=dim, page=32))
    ws = attend8(c)
    first, off = c.out.clone(), torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(500):
        c.out.fill_(77.0)
        attend8(c, ws=ws)
        off += (c.out != first).sum()
    assert off.item() == 0 and wino.wino_read_device_status(ws) == wino.WINO_OK


def test_far_offsets():
    """A cache whose offsets pass 32 bits: pages 3 GiB apart."""
    stride = 3 << 30
    whole = torch.zeros(2 * stride + (1 << 20), dtype=torch.uint8, device="cuda")
    k8, v8 = (torch.as_strided(whole, (3, 16, 1, 64), (stride, 64, 64, 1), x) for x in (0, 1 << 16))
    g = torch.Generator().manual_seed(3)
    c = make_kv8(CAUSAL, [(1, 33, 32)], heads=4, kv_heads=1, dim=64, poison=False)
    for i, (name, far) in enumerate((("k", k8), ("v", v8))):
        codes, scales = quantise(torch.randn((3, 16, 1, 64), generator=g).cuda(), BF)
        far.copy_(codes.view(torch.uint8))
        c.extra[name + "8"], c.extra[name + "_scale"] = far, scales
        setattr(c, name + "_cache", values_of(codes, scales, BF))
    c.table = c.table * 0 + torch.tensor([2, 0, 1, 2][:c.table.shape[1]]).numpy()
    c.table_dev.copy_(torch.from_numpy(c.table))
    run(add_rows(rebatch(c)))
    assert whole.numel() > 1 << 32


def test_two_streams_with_workspaces_of_their_own():
    """Calls that overlap on the GPU over one cache: each as alone."""
    calls = [add_rows(make_kv8(CAUSAL, [(1, 30001 + i, 30000 + i), (1, 500, 499)], heads=8, kv_heads=2, dim=128, page=64, seed=i)) for i in range(2)]
    alone = []
    for c in calls:
        attend8(c)
        alone.append(c.out.clone())
    spaces, streams = [wino.attend_workspace(c.batch) for c in calls], [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, ws, stream in zip(calls, spaces, streams):
            wino.wino_attend_scaled(c.q, c.out, c.batch, ws, stream=stream)
    torch.cuda.synchronize()
    for c, ws, want in zip(calls, spaces, alone):
        assert wino.wino_read_device_status(ws) == wino.WINO_OK and torch.equal(c.out, want)
