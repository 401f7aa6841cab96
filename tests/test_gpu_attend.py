"""wino_attend against the definition in 64 bits (kv_helpers): masks, lengths around tiles and pages, head layouts, types,
strides, rows that see nothing, poisoned slots, and what a batch's device arrays may hold."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2605_16941_gb300 as wino  # noqa: E402
from kv_helpers import CAUSAL, FULL, SHADOW, Kv, add_rows, attend, check, check_on_device, make_kv  # noqa: E402

BF, FP = torch.bfloat16, torch.float16


def run(c, **kw):
    ws = attend(c, **kw)
    torch.cuda.synchronize()
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    return check(c)


CASES = {
    # name: (mask, [(rows, kv_len, new_slot)], other arguments of make_kv)
    "one_slot": (CAUSAL, [(1, 1, 0)], {}),
    "one_token": (CAUSAL, [(1, 300, 299)], dict(heads=8, kv_heads=2, dim=128)),
    "no_slots": (FULL, [(3, 0, 0), (2, 5, 0)], {}),
    "empty_and_absent": (FULL, [(0, 40, 0), (2, 0, 0), (0, 0, 0), (4, 33, 0)], dict(gap=3)),
    "causal_first_rows": (CAUSAL, [(5, 5, 0), (7, 3, 0)], {}),  # rows past kv_len see kv_len slots
    "left_padding": (CAUSAL, [(9, 5, -4), (3, 0, -3)], {}),  # rows before slot 0 see nothing
    "tile_edges": (CAUSAL, [(1, n, n - 1) for n in (127, 128, 129, 255, 256, 257, 385)], dict(gap=1)),
    "pages_of_16": (FULL, [(3, n, 0) for n in (15, 16, 17, 47, 145)], {}),
    "pages_of_32": (FULL, [(3, n, 0) for n in (31, 33, 161)], dict(page=32, layout="heads")),
    "pages_of_64": (FULL, [(3, n, 0) for n in (63, 65, 200)], dict(page=64)),
    "pages_of_128": (FULL, [(3, n, 0) for n in (128, 129, 300)], dict(page=128, layout="heads")),
    "pages_of_384": (FULL, [(3, n, 0) for n in (384, 385, 500)], dict(page=384)),
    "shadow_1": (SHADOW, [(2, 1, 0), (2, 9, 8), (2, 9, 0)], {}),
    "shadow_32": (SHADOW, [(64, 96, 64), (64, 64, 0), (64, 200, 100)], dict(heads=4, kv_heads=4, dim=128)),
    "shadow_tile_edge": (SHADOW, [(6, 126, 123), (6, 128, 125), (8, 127, 120)], dict(heads=4, kv_heads=2)),
    "shadow_right_context": (SHADOW, [(20, 300, 40)], dict(dim=128, layout="heads")),
    "shadow_large": (SHADOW, [(300, 700, 500)], dict(heads=2, kv_heads=1, dim=64, page=64)),
    "full_130_rows": (FULL, [(130, 257, 0)], dict(heads=1)),
    "causal_prompt": (CAUSAL, [(300, 300, 0)], dict(heads=3, kv_heads=3, dim=128)),
    "causal_ragged": (CAUSAL, [(70, 170, 100), (1, 400, 399), (129, 129, 0), (2, 2, 0)], dict(gap=2, order=[2, 0, 3, 1])),
    "group_7": (CAUSAL, [(40, 140, 100), (1, 60, 59)], dict(heads=14, kv_heads=2)),
    "group_5_dim_80": (SHADOW, [(20, 50, 30)], dict(heads=10, kv_heads=2, dim=80)),
    "group_128": (CAUSAL, [(3, 200, 197)], dict(heads=128, kv_heads=1)),
    "group_100": (CAUSAL, [(3, 200, 197)], dict(heads=100, kv_heads=1)),
    "dim_8": (FULL, [(5, 140, 0)], dict(dim=8)),
    "dim_72": (FULL, [(5, 140, 0)], dict(dim=72, layout="heads")),
    "dim_96": (CAUSAL, [(50, 140, 90)], dict(dim=96, heads=6, kv_heads=2)),
    "dim_120": (CAUSAL, [(5, 140, 135)], dict(dim=120)),
    "many_short": (CAUSAL, [(1 + i % 3, 1 + (7 * i) % 90, (7 * i) % 90 - i % 3) for i in range(500)], {}),
    "long": (CAUSAL, [(1, 5000, 4999), (2, 9000, 8998)], dict(heads=8, kv_heads=2, dim=128, page=64)),
    "long_rows": (CAUSAL, [(140, 3000, 2860)], dict(heads=4, kv_heads=2, dim=128, page=32)),
}


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("name", CASES)
def test_against_definition(name, dtype):
    mask, seqs, kw = CASES[name]
    run(add_rows(make_kv(mask, seqs, dtype=dtype, **kw)))


@pytest.mark.parametrize("layout", ["slots", "heads"])
def test_strided_rows(layout):
    run(add_rows(make_kv(CAUSAL, [(33, 150, 117), (1, 20, 19)], heads=6, kv_heads=2, layout=layout, gap=1),
                 strided=True))


def test_combined_cache():
    """K and V in one allocation, [pages, 2, slots, heads, dim]: views with one set of strides."""
    c = make_kv(SHADOW, [(32, 90, 60)], heads=4, kv_heads=2)
    both = torch.stack([c.k_cache, c.v_cache], dim=1).contiguous()
    c.k_cache, c.v_cache = both[:, 0], both[:, 1]
    c.batch = wino.make_kv_batch(c.k_cache, c.v_cache, c.table_dev, *c.ints, n_rows=c.n_rows, n_q_heads=4, mask=SHADOW)
    run(add_rows(c))


@pytest.mark.parametrize("spread", [8.0, 30.0])
def test_peaked_softmax(spread):
    """Scores that move the running maximum by far from tile to tile, and rows whose weights all but one vanish."""
    run(add_rows(make_kv(CAUSAL, [(40, 700, 660)], heads=4, kv_heads=2, dim=128, spread=spread), spread=2.0))


def test_rising_maximum():
    """Keys that grow with the slot: every tile raises the maximum."""
    c = make_kv(FULL, [(130, 640, 0)], heads=1, dim=64, dtype=FP, poison=False)
    for j in range(640):
        c.k_cache[c.table[0, j // 16], j % 16] = 0.02 * j
    add_rows(c)
    c.q.fill_(0.5)
    run(c)


def test_constant_values_come_back():
    """With every V the same, out is that value whatever the weights: off by the weights' rounding at most."""
    c = make_kv(CAUSAL, [(64, 400, 336)], heads=2, dim=128, poison=False)
    c.v_cache.fill_(1.5)
    add_rows(c)
    run(c)


def test_scale():
    c = add_rows(make_kv(CAUSAL, [(4, 50, 46)]))
    ws = attend(c, scale=0.37)
    torch.cuda.synchronize()
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    check(c, scale=0.37)


def test_workspace_is_reused_as_it_is():
    """One workspace through calls of other shapes, and twice the same call: bit for bit the same."""
    big = add_rows(make_kv(CAUSAL, [(200, 1000, 800), (1, 3000, 2999)], heads=8, kv_heads=2, dim=128))
    ws = wino.attend_workspace(big.batch)
    run(big, ws=ws)
    first = big.out.clone()
    for mask, seqs in ((SHADOW, [(64, 500, 400)]), (FULL, [(1, 0, 0)])):
        run(add_rows(make_kv(mask, seqs, heads=4, kv_heads=2)), ws=ws)
    big.out.fill_(77.0)
    run(big, ws=ws)
    assert torch.equal(first, big.out)


def test_captured_call_takes_new_lengths():
    """The lengths, slots and pages are read when the call runs."""
    seqs = [(4, 900, 896), (1, 300, 299)]
    c = add_rows(make_kv(CAUSAL, seqs, heads=8, kv_heads=2, dim=128, poison=False))
    ws = wino.attend_workspace(c.batch)
    run(c, ws=ws)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        attend(c, ws=ws)
    for lens in ([(4, 500, 496), (1, 301, 300)], [(3, 17, 14), (1, 0, 0)], seqs):
        c.seqs = lens
        c.ints[1:].copy_(torch.tensor([[s[i] for s in lens] for i in range(3)], dtype=torch.int32))
        c.extra["whole"].fill_(77.0)
        g.replay()
        torch.cuda.synchronize()
        assert wino.wino_read_device_status(ws) == wino.WINO_OK
        check(c)


def test_two_streams_with_their_own_workspaces():
    cs = [add_rows(make_kv(CAUSAL, [(100, 2000, 1900)], heads=8, kv_heads=2, dim=128, seed=i), seed=i) for i in range(2)]
    wss = [wino.attend_workspace(c.batch) for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    for _ in range(3):
        for c, ws, s in zip(cs, wss, streams):
            wino.wino_attend(c.q, c.out, c.batch, ws, stream=s)
    torch.cuda.synchronize()
    for c, ws in zip(cs, wss):
        assert wino.wino_read_device_status(ws) == wino.WINO_OK
        check(c)


def test_shared_prefix_pages():
    """Two sequences read the same pages."""
    c = make_kv(CAUSAL, [(2, 100, 98), (2, 100, 98)], poison=False)
    c.table[1, :5] = c.table[0, :5]
    c.table_dev.copy_(torch.from_numpy(c.table))
    run(add_rows(c))


@pytest.mark.parametrize("what", ["page", "negative_page", "rows", "start", "length", "kv", "odd_shadow", "shadow_table"])
def test_bad_device_values_end_in_an_error(what):
    """Values that only the device can check: an error status, the other sequences as they should be, nothing outside
    the rows written, and the next call clean."""
    mask = SHADOW if "shadow" in what else CAUSAL
    c = add_rows(make_kv(mask, [(4, 60, 50), (4, 70, 60), (2, 40, 30)], gap=1, heads=4, kv_heads=2))
    ws = wino.attend_workspace(c.batch)
    keep, table = c.ints.clone(), c.table_dev.clone()
    if what == "page":
        c.table_dev[1, 2] = c.k_cache.size(0)
    elif what == "negative_page":
        c.table_dev[1, 2] = -1
    elif what == "rows":
        c.ints[1, 1] = c.n_rows + 1
    elif what == "start":
        c.ints[0, 1] = -3
    elif what == "length":
        c.ints[1, 1] = -1
    elif what == "kv":
        c.ints[2, 1] = c.table.shape[1] * c.page + 1
    elif what == "odd_shadow":
        c.ints[1, 1] = 3
    else:
        c.ints[2, 1] = c.table.shape[1] * c.page - 1
    wino.wino_attend(c.q, c.out, c.batch, ws)
    assert wino.wino_read_device_status(ws) == wino.WINO_ERR_ARG
    saved = c.seqs
    start = c.starts[1]
    c.extra["whole"][start:start + 4] = 77.0  # undefined rows
    c.seqs = [saved[0], (0, 0, 0), saved[2]]
    check(c)
    c.seqs = saved
    c.ints.copy_(keep)
    c.table_dev.copy_(table)
    run(c, ws=ws)


def test_far_offsets():
    """A cache of more than 2^31 elements: pages at both ends."""
    kv, dim, page = 8, 128, 64
    n_pages = (1 << 31) // (kv * dim * page) + 70
    k = torch.empty((n_pages, page, kv, dim), dtype=BF, device="cuda")
    v = torch.empty_like(k)
    pages = [n_pages - 1, 0, n_pages - 2, 1]
    c = make_kv(CAUSAL, [(3, 250, 247)], heads=16, kv_heads=kv, dim=dim, page=page, poison=False)
    for i, p in enumerate(pages):
        k[p].copy_(c.k_cache[c.table[0, i]])
        v[p].copy_(c.v_cache[c.table[0, i]])
    small = c.table.copy()
    far = small.copy()
    far[0, :4] = pages
    table = torch.from_numpy(far).cuda()
    add_rows(c)
    b = wino.make_kv_batch(k, v, table, *c.ints, n_rows=c.n_rows, n_q_heads=16, mask=CAUSAL)
    ws = wino.attend_workspace(b)
    wino.wino_attend(c.q, c.out, b, ws)
    torch.cuda.synchronize()
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    check(c)


def test_large_batch_matches_the_plain_form():
    """A larger ragged batch against the definition evaluated on the device."""
    rng = np.random.default_rng(3)
    seqs = [(int(n), int(n + c), int(c)) for n, c in zip(rng.integers(1, 700, 6), rng.integers(0, 5000, 6))]
    c = add_rows(make_kv(CAUSAL, seqs, heads=8, kv_heads=2, dim=128, page=64))
    ws = attend(c)
    torch.cuda.synchronize()
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    check_on_device(c)


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 96, 128])
@pytest.mark.parametrize("mask", [FULL, CAUSAL, SHADOW], ids=["full", "causal", "shadow"])
def test_tasks_of_two_row_tiles(mask, dim, dtype):
    """More tasks than CTAs, of rows in both tiles and in one, whole and in parts."""
    rng = np.random.default_rng(dim)
    seqs = []
    for s in range(45):
        n = int(rng.integers(65, 130)) * 2 if s % 5 else int(rng.integers(1, 20)) * 2
        ctx = int(rng.integers(0, 1500))
        seqs.append((n, n + ctx, ctx) if mask == CAUSAL else (n, ctx + n // 2, ctx))
    seqs[7], seqs[20] = (0, 9, 0), (4, 0, 0)
    c = add_rows(make_kv(mask, seqs, heads=4, kv_heads=2, dim=dim, page=32, dtype=dtype, gap=1))
    ws = attend(c)
    torch.cuda.synchronize()
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    check_on_device(c)
    first = c.out.clone()
    attend(c, ws=ws)
    assert torch.equal(first, c.out)


@pytest.mark.parametrize("dim", [64, 128])
def test_one_long_task_in_many_parts(dim):
    """A few tasks over all CTAs: the tree that joins their parts, in both of its forms."""
    for rows, heads in ((1, 8), (40, 4), (300, 1)):
        c = add_rows(make_kv(CAUSAL, [(rows, 30000, 30000 - rows)], heads=heads, kv_heads=1, dim=dim, page=128))
        ws = attend(c)
        torch.cuda.synchronize()
        assert wino.wino_read_device_status(ws) == wino.WINO_OK
        check_on_device(c)
        first = c.out.clone()
        for _ in range(5):
            attend(c, ws=ws)
        assert torch.equal(first, c.out)


def test_many_short_parts_with_tails():
    """Parts of one or two slot tiles, each ending inside a tile, several in flight at once in every CTA."""
    seqs = [(1, 1 + (37 * i) % 250, (37 * i) % 250) for i in range(700)]
    run(add_rows(make_kv(CAUSAL, seqs, heads=8, kv_heads=8, dim=128)))


@pytest.mark.parametrize("dim", [64, 128])
def test_few_rows_over_large_pages(dim):
    """Most warps without rows, and slot tiles that arrive at once: no warp may run a tile ahead of the others."""
    for n in (257, 300, 385, 513, 700, 1500):
        for rows in (1, 3, 40):
            run(add_rows(make_kv(FULL, [(rows, n, 0)], dim=dim, page=128, layout="heads", seed=n)))


@pytest.mark.parametrize("kv_heads", [1, 3])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("layout", ["slots", "heads", "head_major", "odd"])
def test_cache_strides(layout, page, kv_heads):
    """Caches of 128 dims whose pages are a whole number of heads apart, and such as are not."""
    c = make_kv(CAUSAL, [(3, 300, 297), (1, 77, 76)], heads=2 * kv_heads, kv_heads=kv_heads, dim=128, page=page)
    P, S, H, D = c.k_cache.shape
    caches = []
    for t in (c.k_cache, c.v_cache):
        if layout == "heads":
            new = torch.empty((P, H, S, D), dtype=BF, device="cuda").transpose(1, 2)
        elif layout == "head_major":  # all pages of a head together
            new = torch.empty((H, P, S, D), dtype=BF, device="cuda").permute(1, 2, 0, 3)
        elif layout == "odd":  # gaps of 8 elements behind heads, of 24 behind slots, of 40 behind pages
            st = (S * (H * (D + 8) + 24) + 40, H * (D + 8) + 24, D + 8, 1)
            new = torch.empty(P * st[0], dtype=BF, device="cuda").as_strided((P, S, H, D), st)
        else:
            new = torch.empty_like(t)
        caches.append(new.copy_(t))
    c.k_cache, c.v_cache = caches
    c.batch = wino.make_kv_batch(*caches, c.table_dev, *c.ints, n_rows=c.n_rows, n_q_heads=c.heads, mask=CAUSAL)
    run(add_rows(c))


@pytest.mark.parametrize("n_seq", [3, 300])
def test_work_counted_in_64_bits(n_seq):
    """One page of 2^20 slots and tables for 2^30: with 300 sequences the work might not fit 32 bits."""
    page, width = 1 << 20, 1 << 10
    g = torch.Generator().manual_seed(2)
    k, v = (torch.full((1, page, 1, 64), float("nan"), dtype=BF, device="cuda") for _ in range(2))
    for t in (k, v):
        t[0, :1600] = torch.randn((1600, 1, 64), generator=g).to(BF).cuda()
    seqs = [(1 + i % 2, 5 + (53 * i) % 1500, 3 + (53 * i) % 1500) for i in range(n_seq)]
    for s in range(n_seq):  # a slot that no row of the sequence sees may be another's: all see the same page
        assert seqs[s][1] <= 1600
    starts = np.cumsum([0] + [s[0] for s in seqs])[:-1].tolist()
    rows = sum(s[0] for s in seqs)
    table = np.zeros((n_seq, width), dtype=np.int32)
    table[:, 1:] = -1
    ints = torch.tensor([starts] + [[s[i] for s in seqs] for i in range(3)], dtype=torch.int32, device="cuda")
    td = torch.from_numpy(table).cuda()
    b = wino.make_kv_batch(k, v, td, *ints, n_rows=rows, n_q_heads=4, mask=CAUSAL)
    c = add_rows(Kv(CAUSAL, seqs, 4, 1, 64, page, BF, starts, rows, table, k[:, :2048], v[:, :2048], ints, td, b))
    run(c)


def test_sequences_that_share_rows_end():
    """Not allowed, since the rows' results race, but the call ends, and with it an ordinary one on the same workspace."""
    c = add_rows(make_kv(CAUSAL, [(64, 200, 136)] * 40, heads=8, kv_heads=2, dim=128, poison=False))
    keep = c.ints.clone()
    ws = wino.attend_workspace(c.batch)
    c.ints[0].zero_()  # every sequence has all rows
    c.ints[1].fill_(c.n_rows)
    wino.wino_attend(c.q, c.out, c.batch, ws)
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    c.ints.copy_(keep)
    c.extra["whole"].fill_(77.0)
    run(c, ws=ws)


def test_16384_sequences():
    """The most sequences a batch may have, of which some are checked."""
    seqs = [(1 + i % 3, 1 + (29 * i) % 50, (29 * i) % 50 - i % 3) for i in range(16384)]
    c = add_rows(make_kv(CAUSAL, seqs, heads=2, kv_heads=1, dim=8))
    ws = attend(c)
    torch.cuda.synchronize()
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    check(c, only=set(range(0, 16384, 331)) | {16383})
    assert not (c.out == 77.0).all(-1).any()


def test_failure_is_reported_once_and_cleared():
    """An error recorded for a call (planted here as a CTA would record a timeout, with nodes that parts which never came
    would have left) is published, and the next call on the workspace starts clean."""
    c = add_rows(make_kv(CAUSAL, [(3, 3000, 2997)], heads=4, kv_heads=1, dim=128))
    ws = wino.attend_workspace(c.batch)
    run(c, ws=ws)
    words = ws.view(torch.int32)
    words[0] = wino.WINO_ERR_DEVICE_TIMEOUT
    words[64:64 + 160 * 64] = 1  # behind the 256 bytes of status words
    wino.wino_attend(c.q, c.out, c.batch, ws)
    assert wino.wino_read_device_status(ws) == wino.WINO_ERR_DEVICE_TIMEOUT
    assert (words[64:64 + 160 * 64] == 0).all() and words[0] == 0 and words[2] == 0
    c.extra["whole"].fill_(77.0)
    run(c, ws=ws)


def test_two_graphs_share_a_workspace():
    """Graphs of other shapes on one workspace, replayed one behind the other without a pause: as the calls by themselves."""
    a = add_rows(make_kv(CAUSAL, [(300, 5000, 4700)], heads=8, kv_heads=2, dim=128))
    b = add_rows(make_kv(SHADOW, [(16, 4000, 3990), (2, 31, 30)], heads=8, kv_heads=2, dim=64))
    ws = wino.attend_workspace(a.batch)
    want = []
    for c in (a, b):
        run(c, ws=ws)
        want.append(c.out.clone())
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g, c in zip(graphs, (a, b)):
        with torch.cuda.graph(g):
            attend(c, ws=ws)
        c.extra["whole"].fill_(77.0)
    for _ in range(20):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    assert torch.equal(a.out, want[0]) and torch.equal(b.out, want[1])


@pytest.mark.parametrize("heads,kv_heads,rows", [(80, 80, 260), (80, 40, 140)])
@pytest.mark.parametrize("mask", [CAUSAL, SHADOW], ids=["causal", "shadow"])
def test_more_tasks_than_ctas(mask, heads, kv_heads, rows):
    """Several tasks of each of many kv heads, some sequences between them without any: the order by row position."""
    seqs = [(rows, rows + 20, 30), (0, 100, 0), (rows + 30, rows - 60, 40), (2, 500, 490), (0, 0, 0)]
    run(add_rows(make_kv(mask, seqs, heads=heads, kv_heads=kv_heads, dim=16, gap=1)))
