"""wino_rope_append against the definition in 64 bits.  Tolerance: cos and sin are off by at most 2^-22 (the turn by 2^-31,
its value in fp32 by 2^-25 turns, the functions by two half steps), products and sum by half steps of fp32, so
2^-20 factor (|a| + |b|), and half a step of the element type."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2605_16941_gb300 as wino  # noqa: E402
from kv_helpers import CAUSAL, FULL, SHADOW, f64, frequencies, half_step, make_kv, rotated  # noqa: E402

BF, FP = torch.bfloat16, torch.float16


def slots_of(mask, n, kv, new):
    i = np.arange(n)
    return np.where(i < n // 2, new + i, kv + i - n // 2) if mask == SHADOW else new + i


def positions_of(mask, n, kv, new):
    i = np.arange(n)
    return new + (i % max(1, n // 2) if mask == SHADOW else i)


def close(got, x, want, rot, factor, dtype, interleaved):
    j = np.arange(rot // 2)
    a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)
    size = np.zeros_like(x)
    size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    tol = 2.0 ** -20 * abs(factor) * size + 1.001 * half_step(dtype) * np.abs(want)
    if dtype == FP:
        tol = tol + 2.0 ** -25 * (size > 0)
    d = np.abs(got - want)
    assert (d <= tol).all(), f"off by {d.max()}"


def check_append(mask, seqs, heads=4, kv_heads=2, dim=64, rot=None, interleaved=False, factor=1.0, dtype=BF, positions=None,
                 in_place=False, layout="slots", page=16, gap=0, what="qkv", base=10000.0, seed=0):
    rot = dim if rot is None else rot
    c = make_kv(mask, seqs, heads=heads, kv_heads=kv_heads, dim=dim, page=page, dtype=dtype, layout=layout, gap=gap,
                poison=False, seed=seed)
    g = torch.Generator().manual_seed(seed)
    qkv = torch.randn((c.n_rows, heads + 2 * kv_heads, dim), generator=g).to(dtype).cuda()
    q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
    freq = frequencies(rot, base)
    pos = None if positions is None else torch.tensor(positions, dtype=torch.int32, device="cuda")
    rope = wino.make_rope(torch.from_numpy(freq).cuda() if rot else None, rot_dim=rot, factor=factor,
                          interleaved=interleaved, positions=pos)
    before = [f64(t) for t in (q, k, v, c.k_cache, c.v_cache)]
    out = q if in_place else torch.full((c.n_rows, heads, dim), 7.0, dtype=dtype, device="cuda")
    ws = wino.append_workspace()
    wino.wino_rope_append(q if "q" in what else None, k if "k" in what else None, v if "k" in what else None, c.batch,
                          rope, ws, q_out=None if in_place or "q" not in what else out)
    torch.cuda.synchronize()
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    x, xk, xv, want_k, want_v = before
    got, got_k, got_v = f64(out), f64(c.k_cache), f64(c.v_cache)
    rows = np.zeros(c.n_rows, dtype=bool)
    for s, (n, kv, new) in enumerate(seqs):
        r = np.arange(n) + c.starts[s]
        rows[r] = True
        p = np.asarray(positions)[r] if positions is not None else positions_of(mask, n, kv, new)
        if "q" in what:
            close(got[r], x[r], rotated(x[r], p[:, None], freq, rot, interleaved, factor), rot, factor, dtype, interleaved)
        if "k" in what:
            slot = slots_of(mask, n, kv, new)
            live = slot >= 0
            page_at = (c.table[s, slot[live] // page], slot[live] % page)
            rk = xk[r][live]
            close(got_k[page_at], rk, rotated(rk, p[live][:, None], freq, rot, interleaved, factor), rot, factor, dtype,
                  interleaved)
            assert np.array_equal(got_v[page_at], xv[r][live])
            got_k[page_at], got_v[page_at] = want_k[page_at], want_v[page_at]  # the rest is compared below
    assert np.array_equal(got_k, want_k) and np.array_equal(got_v, want_v), "a slot of no row was written"
    assert np.array_equal(got[~rows], x[~rows] if in_place else np.full_like(got[~rows], 7.0))
    if in_place:  # the columns of k and v beside q
        assert np.array_equal(f64(k), xk) and np.array_equal(f64(v), xv)


CASES = {
    "one_row": (CAUSAL, [(1, 1, 0)], {}),
    "token_batch": (CAUSAL, [(1, 10 * i + 1, 10 * i) for i in range(40)], dict(heads=8, kv_heads=2, dim=128)),
    "shadow": (SHADOW, [(64, 96, 64), (64, 40, 0)], dict(heads=4, kv_heads=4, dim=128)),
    "shadow_gap": (SHADOW, [(6, 20, 3), (0, 0, 0), (2, 1, 0)], dict(gap=2)),
    "full": (FULL, [(30, 200, 100)], dict(page=128, layout="heads")),
    "left_padding": (CAUSAL, [(9, 5, -4)], {}),
    "part": (CAUSAL, [(20, 20, 0)], dict(dim=128, rot=64)),
    "part_odd_pairs": (CAUSAL, [(20, 20, 0)], dict(dim=80, rot=20)),
    "part_2": (CAUSAL, [(5, 5, 0)], dict(dim=8, rot=2)),
    "part_72": (CAUSAL, [(5, 5, 0)], dict(dim=96, rot=72, layout="heads")),
    "no_rotation": (CAUSAL, [(5, 5, 0)], dict(rot=0)),
    "many_rows": (CAUSAL, [(3000, 3000, 0), (1200, 1500, 300)], dict(heads=2, kv_heads=1, dim=128, gap=5)),
    "dim_8": (CAUSAL, [(33, 33, 0)], dict(dim=8)),
    "dim_72": (CAUSAL, [(33, 33, 0)], dict(dim=72)),
}


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "interleaved"])
@pytest.mark.parametrize("name", CASES)
def test_against_definition(name, interleaved, dtype):
    mask, seqs, kw = CASES[name]
    check_append(mask, seqs, interleaved=interleaved, dtype=dtype, **kw)


@pytest.mark.parametrize("interleaved", [False, True])
def test_in_place(interleaved):
    check_append(CAUSAL, [(40, 40, 0)], in_place=True, interleaved=interleaved, gap=1, heads=3, kv_heads=3, dim=128)


@pytest.mark.parametrize("what", ["q", "k"])
def test_one_side_only(what):
    check_append(SHADOW, [(8, 20, 12)], what=what)


def test_positions_and_factor():
    check_append(CAUSAL, [(6, 6, 0)], positions=[5, 0, 1, 1, 100, 7], factor=1.25)


def test_far_positions():
    """Angles of positions where x f in 32 bits would be off by radians."""
    pos = [0, 1, 262143, 1 << 20, (1 << 24) + 1, 2147483647, -1, -1000000]
    check_append(CAUSAL, [(8, 8, 0)], positions=pos, base=500000.0, dim=128)


def test_bad_slots_are_not_written():
    """A page out of range, a slot past the table: an error, that row's K and V nowhere, everything else in place."""
    c = make_kv(CAUSAL, [(4, 40, 36), (4, 40, 36)], poison=False)
    c.table_dev[0, 2] = c.k_cache.size(0) + 5
    c.ints[3, 1] = c.table.shape[1] * c.page - 2  # rows 2 and 3 of sequence 1 lie past the table
    tail = c.table_dev[1, -1].item()
    assert tail < 0  # and rows 0 and 1 on an entry that is no page
    k = torch.randn((c.n_rows, 1, 64)).to(BF).cuda()
    before = c.k_cache.clone(), c.v_cache.clone()
    ws = wino.attend_workspace(c.batch)
    rope = wino.make_rope(None, rot_dim=0)
    wino.wino_rope_append(None, k, k, c.batch, rope, ws)
    assert wino.wino_read_device_status(ws) == wino.WINO_ERR_ARG
    assert torch.equal(c.k_cache, before[0]) and torch.equal(c.v_cache, before[1])
    # it stays until a wino_attend with the workspace has reported it
    c.table_dev.copy_(torch.from_numpy(c.table))
    c.ints[3, 1] = 36
    q = torch.randn((c.n_rows, 2, 64)).to(BF).cuda()
    wino.wino_attend(q, torch.empty_like(q), c.batch, ws)
    assert wino.wino_read_device_status(ws) == wino.WINO_ERR_ARG
    wino.wino_attend(q, torch.empty_like(q), c.batch, ws)
    assert wino.wino_read_device_status(ws) == wino.WINO_OK


def test_captured_append():
    c = make_kv(CAUSAL, [(2, 10, 8)], poison=False)
    k = torch.randn((c.n_rows, 1, 64)).to(BF).cuda()
    v = torch.randn((c.n_rows, 1, 64)).to(BF).cuda()
    ws, rope = wino.append_workspace(), wino.make_rope(None, rot_dim=0)
    wino.wino_rope_append(None, k, v, c.batch, rope, ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        wino.wino_rope_append(None, k, v, c.batch, rope, ws)
    for new in (3, 0, 7):
        c.k_cache.zero_()
        c.ints[3, 0] = new
        g.replay()
        torch.cuda.synchronize()
        for i in range(2):
            j = new + i
            assert torch.equal(c.k_cache[c.table[0, j // 16], j % 16], k[i])
        assert int((c.k_cache != 0).any(-1).sum()) == 2
