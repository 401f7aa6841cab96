"""Helpers of the paged-cache tests: batches of small sequences over a cache poisoned with NaN wherever no row may look,
and the operators' definition in 64 bits on the host (numpy, without the library).

Tolerances come from arithmetic, with u = 2^-24 (fp32 half step), h = half a step of the element type, A = sum p_j |V_j|:
  - a score is a sum of D fp32 products: off by at most (D + 2) u S, S = scale * sum |q_c K_c|; twice that (numerator and
    denominator of p) is the relative error it brings into out, with 2^-21 for the exponential and n u for the sums
  - each weight is rounded to the element type: h A; fp16 weights below 2^-14 by 2^-25 at most: n 2^-25 max |V|
  - the result is rounded once: h |out| (fp16 below 2^-14: 2^-25)
"""
from __future__ import annotations

import math
from dataclasses import dataclass, field

import numpy as np
import torch

import paper_2605_16941_gb300 as wino

FULL, CAUSAL, SHADOW = 0, 1, 2
U = 2.0 ** -24


def half_step(dtype) -> float:
    return torch.finfo(dtype).eps / 2


@dataclass
class Kv:
    """A batch on the GPU with what the host needs to check it."""
    mask: int
    seqs: list  # (rows, kv_len, new_slot)
    heads: int
    kv_heads: int
    dim: int
    page: int
    dtype: torch.dtype
    starts: list
    n_rows: int
    table: np.ndarray
    k_cache: torch.Tensor
    v_cache: torch.Tensor
    ints: torch.Tensor
    table_dev: torch.Tensor
    batch: object
    q: torch.Tensor = None
    out: torch.Tensor = None
    extra: dict = field(default_factory=dict)


def held_slots(mask, n, kv, new):
    return kv + n // 2 if mask == SHADOW else kv


def make_kv(mask, seqs, heads=2, kv_heads=1, dim=64, page=16, dtype=torch.bfloat16, layout="slots", seed=0, gap=0,
            poison=True, order=None, spread=1.0, device="cuda"):
    """The cache holds random values in the slots that some row may see and NaN in every other; the sequences' rows are
    `gap` rows apart and stand in `order`."""
    rng = np.random.default_rng(seed)
    need = [max(1, -(-max(held_slots(mask, *s), s[2] + s[0]) // page)) for s in seqs]
    n_pages, width = sum(need) + 2, max(need) + 1
    perm = rng.permutation(n_pages)
    table = np.full((len(seqs), width), -7, dtype=np.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = perm[at:at + n]
        at += n
    shape = (n_pages, page, kv_heads, dim)
    k = rng.standard_normal(shape).astype(np.float32) * spread
    v = rng.standard_normal(shape).astype(np.float32)
    if poison:
        seen = np.zeros(shape[:2], dtype=bool)
        for i, s in enumerate(seqs):
            j = np.arange(held_slots(mask, *s))
            seen[table[i, j // page], j % page] = True
        bad = rng.choice([np.nan, np.inf, -np.inf], size=shape)
        k = np.where(seen[..., None, None], k, bad).astype(np.float32)
        v = np.where(seen[..., None, None], v, bad).astype(np.float32)

    def cache(x):
        t = torch.from_numpy(x).to(dtype)
        if layout == "heads":
            return t.transpose(1, 2).contiguous().to(device).transpose(1, 2)
        return t.to(device)

    starts, r = [0] * len(seqs), gap
    for i in (order or range(len(seqs))):
        starts[i] = r
        r += seqs[i][0] + gap
    n_rows = max(1, r)
    ints = torch.from_numpy(np.array([starts] + [[s[c] for s in seqs] for c in range(3)], dtype=np.int32)).to(device)
    kc, vc, td = cache(k), cache(v), torch.from_numpy(table).to(device)
    b = wino.make_kv_batch(kc, vc, td, *ints, n_rows=n_rows, n_q_heads=heads, mask=mask)
    return Kv(mask, seqs, heads, kv_heads, dim, page, dtype, starts, n_rows, table, kc, vc, ints, td, b)


def add_rows(c: Kv, seed=1, spread=1.0, strided=False):
    """Random q and a canary-filled out, `strided`: parts of wider rows."""
    g = torch.Generator().manual_seed(seed)
    wide = c.heads + (3 if strided else 0)
    q = (torch.randn((c.n_rows, wide, c.dim), generator=g) * spread).to(c.dtype).cuda()
    c.q = q[:, 1:1 + c.heads] if strided else q
    out = torch.full((c.n_rows, wide, c.dim), 77.0, dtype=c.dtype, device="cuda")
    c.extra["whole"] = out
    c.out = out[:, 2:2 + c.heads] if strided else out
    return c


def sees(mask, n, kv, new, i):
    """The slots that row i sees, as a list."""
    if mask == FULL:
        return np.arange(kv)
    if mask == CAUSAL:
        return np.arange(max(0, min(kv, new + i + 1)))
    half = n // 2
    if i < half:
        return np.arange(kv)
    j = np.arange(kv + half)
    return j[j != new + i - half]


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def expected(c: Kv, scale=None, only=None):
    """{(sequence, row)}: (out [heads, dim], tolerance) by the definition."""
    scale = c.dim ** -0.5 if scale is None else scale
    h = half_step(c.dtype)
    kc, vc, q = f64(c.k_cache), f64(c.v_cache), f64(c.q)
    group = c.heads // c.kv_heads
    for s, (n, kv, new) in enumerate(c.seqs):
        if only is not None and s not in only:
            continue
        for i in range(n):
            j = sees(c.mask, n, kv, new, i)
            if len(j) == 0:
                yield s, i, np.zeros((c.heads, c.dim)), np.zeros((c.heads, c.dim))
                continue
            page, at = c.table[s, j // c.page], j % c.page
            K, V = kc[page, at], vc[page, at]  # [slots, kv_heads, dim]
            K, V = np.repeat(K, group, 1), np.repeat(V, group, 1)
            x = q[c.starts[s] + i]
            score = np.einsum("hc,jhc->hj", x, K) * scale
            size = np.abs(x)[None] * np.abs(K)
            err = (c.dim + 2) * U * (size.sum(-1).max(0) * scale)[:, None]
            p = np.exp(score - score.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            out = np.einsum("hj,jhc->hc", p, V)
            A = np.einsum("hj,jhc->hc", p, np.abs(V))
            tol = (2 * err + 2.0 ** -21 + len(j) * U) * 2 * A + 1.01 * h * (A + np.abs(out))
            if c.dtype == torch.float16:
                tol += len(j) * 2.0 ** -25 * np.abs(V).max(0) + 2.0 ** -25
            yield s, i, out, tol


def check(c: Kv, scale=None, only=None):
    got = f64(c.out)
    worst = 0.0
    for s, i, want, tol in expected(c, scale, only):
        row = got[c.starts[s] + i]
        assert np.isfinite(row).all(), f"sequence {s} row {i}: not finite"
        d = np.abs(row - want)
        assert (d <= tol + 1e-30).all(), f"sequence {s} row {i}: off by {d.max()} at tolerance {tol[d > tol].min()}"
        worst = max(worst, float((d / (tol + 1e-30)).max()))
    # rows of no sequence, and the columns beside a strided out, are as they were
    whole = f64(c.extra["whole"]).copy()
    first = int((c.out.data_ptr() - c.extra["whole"].data_ptr()) // (2 * c.dim))
    for s, (n, _, _) in enumerate(c.seqs):
        whole[c.starts[s]:c.starts[s] + n, first:first + c.heads] = 77.0
    assert (whole == 77.0).all(), "elements outside the sequences' rows were written"
    return worst


def attend(c: Kv, ws=None, scale=None, **kw):
    ws = wino.attend_workspace(c.batch) if ws is None else ws
    wino.wino_attend(c.q, c.out, c.batch, ws, scale=scale, **kw)
    return ws


def rotated(x, pos, freq, rot, interleaved, factor):
    """The definition of the rotation, x float64 [..., dim]; pos broadcasts against x's leading dims."""
    y = x.copy()
    j = np.arange(rot // 2)
    a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)
    t = np.asarray(pos, dtype=np.float64)[..., None] * freq
    cs, sn = np.cos(t) * factor, np.sin(t) * factor
    y[..., a] = x[..., a] * cs - x[..., b] * sn
    y[..., b] = x[..., b] * cs + x[..., a] * sn
    return y


def frequencies(rot, base=10000.0):
    return np.array([base ** (-2.0 * j / rot) for j in range(rot // 2)])


def check_on_device(c: Kv, scale=None):
    """As check, the definition evaluated in 64 bits by torch on the GPU: for batches of many rows."""
    scale = c.dim ** -0.5 if scale is None else scale
    h, group = half_step(c.dtype), c.heads // c.kv_heads
    for s, (n, kv, new) in enumerate(c.seqs):
        held = held_slots(c.mask, n, kv, new)
        if n == 0:
            continue
        if held == 0:
            assert (c.out[c.starts[s]:c.starts[s] + n] == 0).all(), f"sequence {s}"
            continue
        j = torch.arange(held, device="cuda")
        i = torch.arange(n, device="cuda")[:, None]
        page = c.table_dev[s].long()[j // c.page]
        K, V = (t[page, j % c.page].double().repeat_interleave(group, 1) for t in (c.k_cache, c.v_cache))
        q = c.q[c.starts[s]:c.starts[s] + n].double()
        if c.mask == FULL:
            seen = (j < kv).expand(n, held)
        elif c.mask == CAUSAL:
            seen = (j <= new + i) & (j < kv)
        else:
            seen = torch.where(i >= n // 2, j != new + i - n // 2, j < kv)
        x = torch.einsum("rhc,jhc->hrj", q, K) * scale
        p = torch.softmax(x.masked_fill(~seen[None], -torch.inf), -1)
        p = torch.where(seen.any(-1)[None, :, None], p, 0.0)  # a row that sees nothing
        want, A = torch.einsum("hrj,jhc->rhc", p, V), torch.einsum("hrj,jhc->rhc", p, V.abs())
        size = torch.einsum("rhc,jhc->hrj", q.abs(), K.abs()).amax(-1).T[..., None] * scale
        err = (c.dim + 2) * U * size
        tol = (2 * err + 2.0 ** -21 + held * U) * 2 * A + 1.01 * h * (A + want.abs())
        if c.dtype == torch.float16:
            tol += held * 2.0 ** -25 * V.abs().max() + 2.0 ** -25
        got = c.out[c.starts[s]:c.starts[s] + n].double()
        d = (got - want).abs()
        assert (d <= tol + 1e-30).all(), f"sequence {s}: off by {d.max()}"
