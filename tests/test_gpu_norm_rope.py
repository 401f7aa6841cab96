"""wino_norm_rope_append and wino_cache_read against their definitions in 64 bits.

Tolerances, u = 2^-24.  The norm: the sum of D <= 128 squares is off by 130 u of itself at most, the root's reciprocal by 2^-22
more, half of the former and the products with it, weight and 1 / sqrt by 4 u: 2^-17 of the result.  The rotation adds
2^-20 factor (|a| + |b|) (test_gpu_rope.py).  So z, what is rounded, is off by at most d = 2^-16.8 (|a| + |b|) (|z| where nothing
turns; nothing where nothing is computed).  An element-type result adds half a step; a code adds half a step of the code at
z + d, and where max |z| is within d of a power's border the scale may be the neighbour's."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2605_16941_gb300 as wino  # noqa: E402
from cache8_helpers import BF, E_MAX, E_MIN, FP, NAN, code_values, exponents, held_values, in_layout, nearest_code, normed  # noqa: E402
from kv_helpers import CAUSAL, FULL, SHADOW, f64, frequencies, half_step, make_kv, rotated  # noqa: E402
from test_gpu_rope import positions_of, slots_of  # noqa: E402

EPS = 1e-6


def rounding_slack(z, size):
    """How far the kernel's unrounded value may be from z."""
    return 2.0 ** -16.8 * size


def check_codes(got, z, slack, dtype, exact):
    """got: values read; z what was quantised, off by slack."""
    if exact:
        assert np.array_equal(got, held_values(z, dtype))
        return
    most, off = np.abs(z).max(-1), slack.max(-1)
    lo, hi = (exponents(np.maximum(most + s * off, 0.0)[..., None], dtype) for s in (-1, 1))
    fine = np.zeros(got.shape, dtype=bool)
    for e in (lo, hi):
        s = 2.0 ** e[..., None].astype(np.float64)
        a, b = nearest_code((z - slack) / s) * s, nearest_code((z + slack) / s) * s  # rounding keeps order
        fine |= (got >= a) & (got <= b) & (nearest_code(got / s) * s == got)
    assert fine.all(), f"{(~fine).sum()} codes off"


class Call:
    """One append with everything that its check needs."""

    def __init__(self, mask, seqs, heads=4, kv_heads=2, dim=64, rot=None, interleaved=False, factor=1.0, dtype=BF, axes=0,
                 norm="qk", per_head=False, offset=0.0, eps=EPS, scaled=False, in_place=False, layout="slots", page=16, gap=0,
                 what="qkv", seed=0, sizes=None, base=10000.0):
        self.__dict__.update(locals())
        self.rot = rot = dim if rot is None else rot
        c = self.c = make_kv(mask, seqs, heads=heads, kv_heads=kv_heads, dim=dim, page=page, dtype=dtype, layout=layout, gap=gap,
                             poison=False, seed=seed)
        g = torch.Generator().manual_seed(seed)
        qkv = torch.randn((c.n_rows, heads + 2 * kv_heads, dim), generator=g)
        if sizes is not None:  # rows of very different size
            qkv *= torch.exp2((torch.rand((c.n_rows, heads + 2 * kv_heads, 1), generator=g) * 2 - 1) * sizes)
        qkv = qkv.to(dtype).cuda()
        self.q, self.k, self.v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]

        def weight(n):
            return (torch.randn((n, dim) if per_head else (dim,), generator=g) * 0.3 + 1 - offset).to(dtype).cuda()
        self.qw, self.kw = (weight(n) if x in norm else None for x, n in (("q", heads), ("k", kv_heads)))
        self.freq = frequencies(rot, base)
        self.rope = wino.make_rope(torch.from_numpy(self.freq).cuda() if rot else None, rot_dim=rot, factor=factor,
                                   interleaved=interleaved)
        self.axis = self.pos = self.wino_axes = None
        if axes:
            rng = np.random.default_rng(seed)
            self.axis = rng.integers(0, axes, rot // 2).astype(np.uint8)
            self.pos = rng.integers(-5, 3000, (axes, c.n_rows)).astype(np.int32)
            wide = torch.zeros((axes, c.n_rows + 3), dtype=torch.int32, device="cuda")
            wide[:, :c.n_rows] = torch.from_numpy(self.pos)
            self.wino_axes = wino.make_rope_axes(torch.from_numpy(self.axis).cuda(), wide[:, :c.n_rows])
        self.norm_ = wino.make_head_norm(self.qw, self.kw, eps=eps, offset=offset) if norm else None
        if scaled:
            shape = c.k_cache.shape
            self.k8, self.v8 = (in_layout(torch.full(shape, 0x55, dtype=torch.uint8, device="cuda"), layout) for _ in range(2))
            self.ks, self.vs = (torch.full((shape[0], kv_heads, page), 0x7b, dtype=torch.uint8, device="cuda") for _ in range(2))
            self.batch = wino.make_kv_batch(self.k8, self.v8, c.table_dev, *c.ints, n_rows=c.n_rows, n_q_heads=heads, mask=mask,
                                            k_scale=self.ks, v_scale=self.vs, dtype=dtype)
        else:
            self.batch = c.batch
        self.out = self.q if in_place else torch.full((c.n_rows, heads, dim), 7.0, dtype=dtype, device="cuda")
        self.ws = wino.append_workspace()
        self.before = [f64(t) for t in (self.q, self.k, self.v, c.k_cache, c.v_cache)]

    def append(self):
        q, kv = "q" in self.what, "k" in self.what
        wino.wino_norm_rope_append(self.q if q else None, self.k if kv else None, self.v if kv else None, self.batch, self.rope, self.ws,
                                   norm=self.norm_, axes=self.wino_axes, q_out=None if self.in_place or not q else self.out)
        torch.cuda.synchronize()
        assert wino.wino_read_device_status(self.ws) == wino.WINO_OK

    def turned(self, x, weight, r, pos):
        """(z, how far off) for rows r."""
        z = normed(x[r], weight, self.eps, self.offset)
        n = self.rot
        j = np.arange(n // 2)
        a, b = (2 * j, 2 * j + 1) if self.interleaved else (j, j + n // 2)
        size = np.abs(z) if weight is not None else np.zeros_like(z)
        if n:
            size[..., a] = size[..., b] = np.abs(self.factor) * (np.abs(z[..., a]) + np.abs(z[..., b]))
            p = self.pos[:, r][self.axis].T[:, None] if self.axes else pos[:, None, None]
            y = z.copy()
            t = p.astype(np.float64) * self.freq
            cs, sn = np.cos(t) * self.factor, np.sin(t) * self.factor
            y[..., a], y[..., b] = z[..., a] * cs - z[..., b] * sn, z[..., b] * cs + z[..., a] * sn
            z = y
        return z, rounding_slack(z, size)

    def check(self):
        c, dtype = self.c, self.dtype
        x, xk, xv, want_k, want_v = self.before
        got = f64(self.out)
        read = None
        if "k" in self.what:
            read = [torch.full((c.n_rows, self.kv_heads, self.dim), 5.0, dtype=dtype, device="cuda") for _ in range(2)]
            wino.wino_cache_read(*read, self.batch, self.ws)
            torch.cuda.synchronize()
            assert wino.wino_read_device_status(self.ws) == wino.WINO_OK
            read = [f64(t) for t in read]
        rows = np.zeros(c.n_rows, dtype=bool)
        stored = np.zeros(c.n_rows, dtype=bool)
        written = np.zeros(c.k_cache.shape[:2], dtype=bool)
        for s, (n, kv, new) in enumerate(self.seqs):
            r = np.arange(n) + c.starts[s]
            rows[r] = True
            pos = positions_of(self.mask, n, kv, new)

            def close(y, z, slack):
                tol = slack + 1.001 * half_step(dtype) * (np.abs(z) + slack) + (2.0 ** -25 if dtype == FP else 0.0) * (slack > 0)
                d = np.abs(y - z)
                assert (d <= tol).all(), f"off by {d.max()}"
            if "q" in self.what:
                close(got[r], *self.turned(x, self.qw, r, pos))
            if read is not None:
                slot = slots_of(self.mask, n, kv, new)
                live = slot >= 0
                stored[r[live]] = True
                at = c.table[s, slot[live] // self.page], slot[live] % self.page
                written[at] = True
                z, slack = self.turned(xk, self.kw, r, pos)
                if self.scaled:
                    check_codes(read[0][r][live], z[live], slack[live], dtype, self.rot == 0 and self.kw is None)
                    check_codes(read[1][r][live], xv[r][live], None, dtype, True)
                else:
                    close(read[0][r][live], z[live], slack[live])
                    assert np.array_equal(read[1][r][live], xv[r][live])
                    assert np.array_equal(f64(c.k_cache)[at], read[0][r][live]) and np.array_equal(f64(c.v_cache)[at], read[1][r][live])
        # nothing else is written: slots of no row, rows of no sequence or slot, rows beside q
        away = ~written
        if self.scaled:
            assert all((t.cpu().numpy()[away] == 0x55).all() for t in (self.k8, self.v8))
            assert all((t.transpose(1, 2).cpu().numpy()[away] == 0x7b).all() for t in (self.ks, self.vs))
        else:
            assert np.array_equal(f64(c.k_cache)[away], want_k[away]) and np.array_equal(f64(c.v_cache)[away], want_v[away])
        if read is not None:
            assert all((t[~stored] == 5.0).all() for t in read)
        assert np.array_equal(got[~rows], x[~rows] if self.in_place else np.full_like(got[~rows], 7.0))
        if self.in_place:
            assert np.array_equal(f64(self.k), xk) and np.array_equal(f64(self.v), xv)


def run(*args, **kw):
    call = Call(*args, **kw)
    call.append()
    call.check()
    return call


CASES = {
    "one_row": (CAUSAL, [(1, 1, 0)], {}),
    "token_batch": (CAUSAL, [(1, 10 * i + 1, 10 * i) for i in range(40)], dict(heads=8, kv_heads=2, dim=128)),
    "shadow": (SHADOW, [(64, 96, 64), (64, 40, 0)], dict(heads=4, kv_heads=4, dim=128)),
    "shadow_gap": (SHADOW, [(6, 20, 3), (0, 0, 0), (2, 1, 0)], dict(gap=2, heads=3, kv_heads=1)),
    "full": (FULL, [(30, 200, 100)], dict(page=128, layout="heads")),
    "left_padding": (CAUSAL, [(9, 5, -4)], {}),
    "part": (CAUSAL, [(20, 20, 0)], dict(dim=128, rot=64)),
    "part_odd_pairs": (CAUSAL, [(20, 20, 0)], dict(dim=80, rot=20)),
    "part_2": (CAUSAL, [(5, 5, 0)], dict(dim=16, rot=2)),
    "part_72": (CAUSAL, [(5, 5, 0)], dict(dim=96, rot=72, layout="heads")),
    "no_rotation": (CAUSAL, [(5, 5, 0)], dict(rot=0)),
    "many_rows": (CAUSAL, [(3000, 3000, 0), (1200, 1500, 300)], dict(heads=2, kv_heads=1, dim=128, gap=5)),
    "more_rows": (CAUSAL, [(600, 600, 0)], dict(heads=5, kv_heads=5, dim=112, page=32)),
    "dim_16": (CAUSAL, [(33, 33, 0)], dict(dim=16, heads=7, kv_heads=7)),
    "dim_32": (CAUSAL, [(33, 33, 0)], dict(dim=32, heads=9, kv_heads=3)),
    "dim_48": (CAUSAL, [(33, 33, 0)], dict(dim=48, heads=6, kv_heads=3)),
    "dim_80": (CAUSAL, [(33, 33, 0)], dict(dim=80, heads=6, kv_heads=3, layout="heads")),
    "dim_112": (SHADOW, [(34, 33, 0)], dict(dim=112, heads=6, kv_heads=6)),
}


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "interleaved"])
@pytest.mark.parametrize("scaled", [False, True], ids=["plain", "e4m3"])
@pytest.mark.parametrize("name", CASES)
def test_against_definition(name, scaled, interleaved, dtype):
    mask, seqs, kw = CASES[name]
    run(mask, seqs, scaled=scaled, interleaved=interleaved, dtype=dtype, **kw)


@pytest.mark.parametrize("scaled", [False, True], ids=["plain", "e4m3"])
@pytest.mark.parametrize("axes", [1, 2, 3, 4])
@pytest.mark.parametrize("kw", [{}, dict(interleaved=True, dim=128), dict(dim=80, rot=20), dict(dim=128, rot=64, factor=1.25)])
def test_axes(axes, kw, scaled):
    run(CAUSAL, [(40, 90, 50), (0, 0, 0), (7, 7, 0)], axes=axes, scaled=scaled, gap=1, **kw)


@pytest.mark.parametrize("scaled", [False, True], ids=["plain", "e4m3"])
@pytest.mark.parametrize("norm,per_head,offset", [("", False, 0.0), ("q", False, 0.0), ("k", False, 1.0), ("qk", True, 0.0),
                                                  ("qk", True, 1.0)])
@pytest.mark.parametrize("dim", [64, 128, 72])
def test_norms(dim, norm, per_head, offset, scaled):
    if scaled and dim % 16:
        pytest.skip("an 8-bit cache has heads of multiples of 16 dims")
    run(SHADOW, [(20, 50, 30)], dim=dim, norm=norm, per_head=per_head, offset=offset, scaled=scaled, heads=6, kv_heads=3)


@pytest.mark.parametrize("dim", [8, 24, 72, 120])
def test_dims_of_8(dim):
    run(CAUSAL, [(33, 33, 0)], dim=dim)


@pytest.mark.parametrize("scaled", [False, True], ids=["plain", "e4m3"])
@pytest.mark.parametrize("rows", [456, 457, 913, 7000, 14592, 14593])
def test_rows_around_full_waves(rows, scaled):
    """From one row of a CTA to as many as there can be, and to two waves of half as many; in two sequences that meet inside a CTA."""
    run(CAUSAL, [(rows - 300, rows - 300, 0), (300, 300, 0)], heads=2, kv_heads=1, dim=16, page=64, scaled=scaled)


@pytest.mark.parametrize("scaled", [False, True], ids=["plain", "e4m3"])
@pytest.mark.parametrize("dim", [128, 96])
def test_in_place(dim, scaled):
    run(CAUSAL, [(40, 40, 0)], in_place=True, gap=1, heads=3, kv_heads=3, dim=dim, scaled=scaled)


@pytest.mark.parametrize("scaled", [False, True], ids=["plain", "e4m3"])
@pytest.mark.parametrize("what", ["q", "k"])
def test_one_side_only(what, scaled):
    run(SHADOW, [(8, 20, 12)], what=what, scaled=scaled)


@pytest.mark.parametrize("dtype,sizes", [(BF, 100.0), (FP, 12.0)], ids=["bf16", "fp16"])
@pytest.mark.parametrize("dim", [128, 72])
def test_rows_of_any_size_are_normalised(dtype, sizes, dim):
    """Squares that overflow or vanish in fp32; with eps in the definition small rows come out small."""
    run(CAUSAL, [(50, 50, 0)], dtype=dtype, sizes=sizes, dim=dim)
    c = Call(CAUSAL, [(4, 4, 0)], dtype=dtype, dim=dim)
    big = torch.finfo(dtype).max
    c.q[0], c.q[1], c.q[2] = big, 0.0, torch.finfo(dtype).tiny
    c.k[0], c.k[1] = -big, 0.0
    c.before[0], c.before[1] = f64(c.q), f64(c.k)
    c.append()
    c.check()


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("dim", [128, 72])
def test_infinities_and_nan_under_the_norm(dim, dtype):
    """By the formula: an infinity's root mean square leaves zeros of the finite elements and NaN of itself, a NaN leaves NaN."""
    c = Call(CAUSAL, [(4, 4, 0)], dtype=dtype, dim=dim, rot=0, heads=2, kv_heads=2)
    for x in (c.q, c.k):
        x[0, 0, 3], x[1, 1, dim - 1], x[2, 0, 0] = float("inf"), -float("inf"), float("nan")
    x = f64(c.q), f64(c.k)
    c.append()
    got = f64(c.out), f64(c.c.k_cache)[c.c.table[0, 0], :4]
    for i, w in enumerate((c.qw, c.kw)):
        with np.errstate(invalid="ignore"):
            z = normed(x[i], w, c.eps, c.offset)
        assert np.array_equal(np.isnan(got[i]), np.isnan(z))
        assert (got[i][0, 0, [0, 1, 2, 4]] == 0).all() and np.isfinite(got[i][3]).all()


@pytest.mark.parametrize("dtype,sizes", [(BF, 30.0), (FP, 12.0)], ids=["bf16", "fp16"])
@pytest.mark.parametrize("rot", [0, 64, 20])
def test_codes_of_rows_of_any_size(dtype, sizes, rot):
    run(CAUSAL, [(300, 300, 0)], dtype=dtype, sizes=sizes, rot=rot, norm="", scaled=True)


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 112])
def test_borders_of_the_scales(dim, dtype):
    """Largest values on, above and below the powers' borders, ties between codes, what saturates, zeros, infinities and NaN: K and V
    bit for bit, the scales too."""
    rng = np.random.default_rng(3)
    tops = [448.0 * 2.0 ** e for e in range(-14, 8)]
    tops += [t * (1 + 2.0 ** -7) for t in tops[:-1]] + [t * (1 - 2.0 ** -8) for t in tops] + [0.0, 60000.0, 57344.0, 65280.0, 2.0 ** -20]
    z = np.zeros((len(tops) + 4, 1, dim))
    for i, t in enumerate(tops):
        z[i, 0] = rng.choice(code_values()[:0x7f], dim) * t / 448.0 * rng.choice([1.0, 1.0625, -1.0, 0.96875], dim)
        z[i, 0] = np.clip(z[i, 0], -t, t)
        z[i, 0, rng.integers(dim)] = t
    z[-4, 0, 3], z[-3, 0, 0], z[-2, 0, dim - 1], z[-1, 0, 5] = np.nan, np.inf, -np.inf, np.nan
    c = Call(CAUSAL, [(len(z), len(z), 0)], kv_heads=1, heads=1, dim=dim, rot=0, norm="", dtype=dtype, scaled=True)
    c.k.copy_(torch.from_numpy(z))
    c.v.copy_(torch.from_numpy(z[::-1].copy()))
    c.append()
    out = [torch.empty_like(t, memory_format=torch.contiguous_format) for t in (c.k, c.v)]
    wino.wino_cache_read(*out, c.batch, c.ws)
    slot = np.arange(len(z))
    at = c.c.table[0, slot // 16], slot % 16
    for got, x, scale in ((out[0], c.k, c.ks), (out[1], c.v, c.vs)):
        x = f64(x)
        want = held_values(x, dtype)
        assert np.array_equal(f64(got), want, equal_nan=True)
        bad = ~np.isfinite(x).all(-1)
        e = np.where(bad, NAN - 127, exponents(np.where(bad[..., None], 0.0, x), dtype)) + 127
        assert np.array_equal(scale.transpose(1, 2).cpu().numpy()[at], e)


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
def test_every_code_and_scale_is_read_exactly(dtype):
    """The 254 codes under every scale that is written; under scale 255 all are NaN."""
    lo = E_MIN[dtype] + 127
    bytes_ = list(range(lo, E_MAX + 128)) + [NAN]
    codes = np.tile(np.arange(256, dtype=np.uint8).reshape(2, 128), (len(bytes_), 1))
    codes[codes & 0x7f == 0x7f] = 0
    n = len(codes)
    pages = -(-n // 16)
    k8 = torch.zeros((pages * 16, 128), dtype=torch.uint8)
    k8[:n] = torch.from_numpy(codes)
    ks = torch.zeros(pages * 16, dtype=torch.uint8)
    ks[:n] = torch.tensor(bytes_, dtype=torch.uint8).repeat_interleave(2)
    k8, ks = k8.view(pages, 16, 1, 128).cuda(), ks.view(pages, 1, 16).cuda()
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    zero, rows = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.full((1,), n, dtype=torch.int32, device="cuda")
    b = wino.make_kv_batch(k8, k8, table, zero, rows, rows, zero, n_rows=n, n_q_heads=1, mask=FULL, k_scale=ks, v_scale=ks, dtype=dtype)
    k, v = (torch.empty((n, 1, 128), dtype=dtype, device="cuda") for _ in range(2))
    wino.wino_cache_read(k, v, b, wino.append_workspace())
    want = code_values()[codes] * 2.0 ** (np.repeat(bytes_, 2).astype(np.float64)[:, None] - 127)
    want[-2:] = np.nan
    assert np.array_equal(f64(k)[:, 0], want, equal_nan=True) and torch.equal(k.view(torch.int16), v.view(torch.int16))


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("kw", [{}, dict(rot=20, dim=80), dict(dim=72), dict(dim=128, interleaved=True, rot=64)])
def test_without_extras_it_is_the_plain_append(kw, dtype):
    a = Call(SHADOW, [(64, 300, 200), (30, 40, 0)], norm="", dtype=dtype, **kw)
    b = Call(SHADOW, [(64, 300, 200), (30, 40, 0)], norm="", dtype=dtype, **kw)
    a.append()
    wino.wino_rope_append(b.q, b.k, b.v, b.batch, b.rope, b.ws, q_out=b.out)
    torch.cuda.synchronize()
    for x, y in ((a.out, b.out), (a.c.k_cache, b.c.k_cache), (a.c.v_cache, b.c.v_cache)):
        assert torch.equal(x.contiguous().view(torch.int16), y.contiguous().view(torch.int16))


def test_axes_on_equal_positions_are_one_axis():
    a, b = (Call(CAUSAL, [(30, 90, 60)], axes=n, scaled=True, dim=128) for n in (3, 0))
    pos = torch.arange(60, 90, dtype=torch.int32, device="cuda")
    a.wino_axes.tensors[1][:] = pos
    for c in (a, b):
        c.append()
    assert torch.equal(a.out, b.out) and torch.equal(a.k8, b.k8) and torch.equal(a.ks, b.ks)


def test_a_bad_axis_is_an_error():
    c = Call(CAUSAL, [(5, 5, 0)], axes=2)
    c.wino_axes.tensors[0][3] = 2
    wino.wino_norm_rope_append(c.q, c.k, c.v, c.batch, c.rope, c.ws, axes=c.wino_axes, q_out=c.out)
    assert wino.wino_read_device_status(c.ws) == wino.WINO_ERR_ARG
    keep = np.setdiff1d(np.arange(64), [3, 35])  # its pair alone is undefined
    c.axis[3] = 0
    z, _ = c.turned(c.before[0], None, np.arange(5), None)
    tol = 2.0 ** -16 * (np.abs(c.before[0]).max(-1, keepdims=True)) + 1.001 * half_step(BF) * np.abs(z)
    assert (np.abs(f64(c.out) - z) <= tol)[..., keep].all()


@pytest.mark.parametrize("scaled", [False, True], ids=["plain", "e4m3"])
def test_bad_slots_are_neither_written_nor_read(scaled):
    c = Call(CAUSAL, [(4, 40, 36), (4, 40, 36)], scaled=scaled)
    c.c.table_dev[0, 2] = c.c.k_cache.size(0) + 5
    c.c.ints[3, 1] = c.c.table.shape[1] * c.page - 2  # rows 2 and 3 of sequence 1 lie past the table
    assert c.c.table_dev[1, -1].item() < 0  # and rows 0 and 1 on an entry that is no page
    caches = (c.k8, c.v8, c.ks, c.vs) if scaled else (c.c.k_cache, c.c.v_cache)
    before = [t.clone() for t in caches]
    wino.wino_norm_rope_append(None, c.k, c.v, c.batch, c.rope, c.ws, norm=c.norm_)
    assert wino.wino_read_device_status(c.ws) == wino.WINO_ERR_ARG
    assert all(torch.equal(t, u) for t, u in zip(caches, before))
    ws = wino.append_workspace()
    k, v = (torch.full((c.c.n_rows, 2, 64), 5.0, dtype=BF, device="cuda") for _ in range(2))
    wino.wino_cache_read(k, v, c.batch, ws)
    assert wino.wino_read_device_status(ws) == wino.WINO_ERR_ARG
    assert (k == 5.0).all() and (v == 5.0).all()


def test_read_takes_one_side_and_strided_rows():
    c = run(SHADOW, [(20, 50, 30)], scaled=True, gap=1)
    whole = [torch.full((c.c.n_rows, 2, 64), 5.0, dtype=BF, device="cuda") for _ in range(2)]
    wino.wino_cache_read(*whole, c.batch, c.ws)
    for i in range(2):
        wide = torch.full((c.c.n_rows, 5, 64), 5.0, dtype=BF, device="cuda")
        wino.wino_cache_read(*((wide[:, 1:3], None) if i == 0 else (None, wide[:, 1:3])), c.batch, c.ws)
        assert torch.equal(wide[:, 1:3], whole[i]) and (wide[:, [0, 3, 4]] == 5.0).all()


@pytest.mark.parametrize("scaled", [False, True], ids=["plain", "e4m3"])
def test_captured(scaled):
    """Append and read in one graph, replayed with other rows, slots and positions; on a stream of its own."""
    c = Call(CAUSAL, [(30, 40, 10)], axes=2, scaled=scaled, dim=128)
    read = [torch.zeros((c.c.n_rows, 2, 128), dtype=BF, device="cuda") for _ in range(2)]

    def calls():
        wino.wino_norm_rope_append(c.q, c.k, c.v, c.batch, c.rope, c.ws, norm=c.norm_, axes=c.wino_axes, q_out=c.out)
        wino.wino_cache_read(*read, c.batch, c.ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls()
    for new in (3, 0, 12):
        gen = torch.Generator().manual_seed(new)
        for t in (c.q, c.k, c.v):
            t.copy_(torch.randn(t.shape, generator=gen))
        c.wino_axes.tensors[1].copy_(torch.randint(0, 99, (2, c.c.n_rows), generator=gen))
        c.c.ints[3, 0] = new
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (c.out, *read)]
        calls()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (c.out, *read)))
        c.seqs, c.pos = [(30, 40, new)], c.wino_axes.tensors[1].cpu().numpy()
        c.before = [f64(t) for t in (c.q, c.k, c.v)] + c.before[3:]
        if scaled:
            for t, x in ((c.k8, 0x55), (c.v8, 0x55), (c.ks, 0x7b), (c.vs, 0x7b)):
                t.fill_(x)
        else:
            c.c.k_cache.copy_(torch.from_numpy(c.before[3]))
            c.c.v_cache.copy_(torch.from_numpy(c.before[4]))
        c.append()
        c.check()
    assert wino.wino_read_device_status(c.ws) == wino.WINO_OK
