"""Helpers of the 8-bit cache's tests: rows as codes and scales by the definition (numpy, 64 bits), and batches whose cache
holds NaN codes and scales wherever no row may look."""
from __future__ import annotations

import numpy as np
import torch

import paper_2605_16941_gb300 as wino
from kv_helpers import f64, held_slots, make_kv

BF, FP = torch.bfloat16, torch.float16
E_MIN, E_MAX = {BF: -110, FP: -14}, 7
NAN = 255


def code_values() -> np.ndarray:
    """The values of the 256 codes; NaN for 0x7f and 0xff."""
    c = np.arange(256)
    e, m = c >> 3 & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where(c & 128, -v, v)
    v[[0x7f, 0xff]] = np.nan
    return v


def exponents(z, dtype):
    """The least e in [e_min, 7] with max |z| <= 448 2^e, of rows z [..., dim]."""
    part, x = np.frexp(np.abs(z).max(-1))
    return np.clip(np.where(part == 0, E_MIN[dtype], x - 9 + (part > 0.875)), E_MIN[dtype], E_MAX)


def nearest_code(x):
    """x to the nearest of the format's values, ties to the even one, kept within +-448."""
    size = np.minimum(np.abs(x), 448.0)
    step = 2.0 ** (np.floor(np.log2(np.maximum(size, 2.0 ** -6))) - 3)
    return np.copysign(np.round(size / step) * step, x)  # numpy rounds halves to even


def held_values(z, dtype):
    """What rows z [..., dim] read as."""
    z = np.asarray(z, dtype=np.float64)
    bad = ~np.isfinite(z).all(-1)
    e = exponents(np.where(bad[..., None], 0.0, z), dtype)[..., None].astype(np.float64)
    return np.where(bad[..., None], np.nan, nearest_code(np.where(bad[..., None], 0.0, z) * 2.0 ** -e) * 2.0 ** e)


def quantise(t, dtype):
    """Codes (float8) and scales [pages, heads, slots] of a cache t [pages, slots, heads, dim], by torch."""
    z = t.double()
    part, x = torch.frexp(z.abs().amax(-1))
    e = torch.where(part == 0, E_MIN[dtype], x - 9 + (part > 0.875).int()).clamp(E_MIN[dtype], E_MAX)
    c = torch.ldexp(z, -e[..., None]).clamp(-448.0, 448.0).float().to(torch.float8_e4m3fn)
    return c, (e + 127).to(torch.uint8).transpose(1, 2).contiguous()


def values_of(codes, scales, dtype):
    """The values that a cache's codes and scales stand for, in the element type."""
    x = codes.float() * torch.exp2(scales.transpose(1, 2).float() - 127.0)[..., None]
    return torch.where((scales == NAN).transpose(1, 2)[..., None], torch.nan, x).to(dtype)


def in_layout(t, layout):
    """[pages, slots, heads, dim] as it is, or stored with the heads outside the slots."""
    return t.transpose(1, 2).contiguous().transpose(1, 2) if layout == "heads" else t.contiguous()


def make_kv8(mask, seqs, dtype=BF, layout="slots", poison=True, spread=1.0, wild=0, **kw):
    """A batch as make_kv's over an 8-bit cache; its k_cache and v_cache become the values that the codes stand for, and
    extra["k8"], ["v8"], ["k_scale"], ["v_scale"] the 8-bit cache.  wild: heads' and slots' sizes vary by up to 2^+-wild."""
    c = make_kv(mask, seqs, dtype=dtype, poison=False, spread=spread, **kw)
    g = torch.Generator().manual_seed(kw.get("seed", 0) + 77)
    for name in ("k", "v"):
        t = getattr(c, name + "_cache").double()
        if wild:
            t = t * torch.exp2((torch.rand(t.shape[:3], generator=g).double() * 2 - 1) * wild).to(t.device)[..., None]
        codes, scales = quantise(t, dtype)
        setattr(c, name + "_cache", values_of(codes, scales, dtype))
        if poison:
            seen = np.zeros(codes.shape[:2], dtype=bool)
            for i, s in enumerate(seqs):
                j = np.arange(held_slots(mask, *s))
                seen[c.table[i, j // c.page], j % c.page] = True
            away = torch.from_numpy(~seen).to(codes.device)
            raw = codes.view(torch.uint8).clone()
            raw[away] = 0x7f
            codes = raw.view(torch.float8_e4m3fn)
            scales.transpose(1, 2)[away] = NAN
        c.extra[name + "8"], c.extra[name + "_scale"] = in_layout(codes.view(torch.uint8), layout).view(torch.float8_e4m3fn), scales
    c.extra["plain"] = c.batch
    return rebatch(c)


def rebatch(c):
    x = c.extra
    c.batch = wino.make_kv_batch(x["k8"], x["v8"], c.table_dev, *c.ints, n_rows=c.n_rows, n_q_heads=c.heads, mask=c.mask,
                                 k_scale=x["k_scale"], v_scale=x["v_scale"], dtype=c.dtype)
    return c


def attend8(c, ws=None, scale=None, **kw):
    ws = wino.attend_workspace(c.batch) if ws is None else ws
    wino.wino_attend_scaled(c.q, c.out, c.batch, ws, scale=scale, **kw)
    return ws


def normed(x, weight, eps, offset):
    """The definition of the norm in 64 bits, x [..., heads, dim]; weight None: x."""
    if weight is None:
        return x
    return x / np.sqrt(np.square(x).mean(-1, keepdims=True) + eps) * (offset + f64(weight))
