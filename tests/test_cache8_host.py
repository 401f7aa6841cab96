"""The norms, axes and 8-bit cache without a GPU: refusals before anything is launched, what the binding refuses, the
structs' mirrors, and the tests' own quantisation against the format's 256 values."""
import ctypes as C
import math
import shutil
import subprocess
from pathlib import Path

import numpy as np
import pytest
import torch

import paper_2605_16941_gb300 as wino
from cache8_helpers import BF, FP, code_values, exponents, held_values, nearest_code, quantise, values_of
from paper_2605_16941_gb300 import _abi

FAKE = 0x10000  # aligned, never dereferenced: every call below fails its checks first
A, S, W = wino.WINO_ERR_ARG, wino.WINO_ERR_SHAPE, wino.WINO_ERR_WORKSPACE


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2605_16941_gb300 import build
    build.build()


def batch(**kw):
    a = dict(n_seq=2, n_rows=8, n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=0, mask=1, page_size=16, n_pages=10,
             table_width=4, q_start=FAKE, q_len=FAKE, kv_len=FAKE, new_slot=FAKE, page_table=FAKE, k_cache=FAKE,
             v_cache=FAKE, page_stride=2048, slot_stride=128, head_stride=64)
    a.update(kw)
    return wino.WinoKvBatch(**a)


def heads(data=FAKE, row=256, head=64):
    return wino.WinoHeads(data, row, head)


def scales(k=FAKE, v=FAKE):
    return wino.WinoKvScales(k, v)


E4M3 = wino.WINO_CACHE_E4M3
# an 8-bit batch that every check accepts ends in the check behind: a misaligned scale
BAD_BATCHES = [(dict(head_dim=72), S), (dict(head_dim=8), S), (dict(slot_stride=136), S), (dict(head_stride=72), S),
               (dict(page_stride=2056), S), (dict(dtype=E4M3 | 2), A), (dict(dtype=E4M3 * 2), A), (dict(mask=3), A),
               (dict(n_rows=0), S), (dict(page_size=24), S), (dict(q_len=None), A), (dict(k_cache=FAKE + 8), A)]


@pytest.mark.parametrize("bad,status", BAD_BATCHES)
def test_batch_refusals(bad, status):
    L = wino.lib()
    b = batch(**{"dtype": E4M3, **bad})
    rope, out = wino.WinoRope(0, 0, 1.0, None, None), C.c_size_t(0)
    assert L.wino_attend_scaled(heads(), heads(FAKE * 2), 0.125, b, scales(), FAKE, 1 << 40, None) == status
    assert L.wino_norm_rope_append(heads(), heads(), heads(), heads(), b, rope, None, None, scales(), FAKE, None) == status
    assert L.wino_cache_read(heads(), heads(FAKE * 2), b, scales(), FAKE, None) == status
    assert L.wino_attend_workspace_size(b, C.byref(out)) == status


def test_the_plain_calls_refuse_an_8_bit_cache():
    L = wino.lib()
    rope = wino.WinoRope(0, 0, 1.0, None, None)
    for dtype in (E4M3, E4M3 | 1):
        assert L.wino_attend(heads(), heads(FAKE * 2), 0.125, batch(dtype=dtype), FAKE, 1 << 40, None) == A
        assert L.wino_rope_append(heads(), heads(), heads(), heads(), batch(dtype=dtype), rope, FAKE, None) == A


@pytest.mark.parametrize("dtype,s", [(E4M3, None), (0, scales()), (E4M3, scales(k=None)), (E4M3, scales(v=None)),
                                     (E4M3 | 1, scales(k=FAKE + 8)), (E4M3, scales(v=FAKE + 1))])
def test_scales_and_type_have_to_agree(dtype, s):
    L, b, rope = wino.lib(), batch(dtype=dtype), wino.WinoRope(0, 0, 1.0, None, None)
    assert L.wino_attend_scaled(heads(), heads(FAKE * 2), 0.125, b, s, FAKE, 1 << 40, None) == A
    assert L.wino_norm_rope_append(heads(), heads(), heads(), heads(), b, rope, None, None, s, FAKE, None) == A
    assert L.wino_cache_read(heads(), heads(FAKE * 2), b, s, FAKE, None) == A


def test_attend_scaled_needs_an_8_bit_cache():
    assert wino.lib().wino_attend_scaled(heads(), heads(FAKE * 2), 0.125, batch(), None, FAKE, 1 << 40, None) == A


def test_attend_scaled_refusals():
    L = wino.lib()

    def call(q=heads(), out=heads(FAKE * 2), scale=0.125, b=batch(dtype=E4M3), ws=FAKE, n=1 << 40):
        return L.wino_attend_scaled(q, out, scale, b, scales(), ws, n, None)
    assert call(b=None) == A and call(q=None) == A and call(out=None) == A and call(ws=None) == A and call(ws=FAKE + 16) == A
    assert call(out=heads()) == A and call(q=heads(FAKE + 8)) == A
    for scale in (0.0, -1.0, 1e-45, 2.0 ** 127, math.inf, math.nan):
        assert call(scale=scale) == A, scale
    assert call(q=heads(row=260)) == S and call(n=100) == W


def test_append_refusals():
    L = wino.lib()
    rope = wino.WinoRope(64, 0, 1.0, FAKE, None)

    def axes(n=3, axis=FAKE, positions=FAKE, stride=8):
        return wino.WinoRopeAxes(n, axis, positions, stride)

    def norm(qw=FAKE, kw=FAKE, qs=0, ks=0, eps=1e-6, offset=0.0):
        return wino.WinoHeadNorm(qw, kw, qs, ks, eps, offset)

    def call(q=heads(), qo=heads(FAKE * 2), k=heads(), v=heads(), b=batch(), r=rope, x=None, n=None, ws=FAKE):
        return L.wino_norm_rope_append(q, qo, k, v, b, r, x, n, None, ws, None)
    assert call(b=None) == A and call(r=None) == A and call(ws=None) == A and call(ws=FAKE + 8) == A
    assert call(q=None) == A and call(v=None) == A and call(q=None, qo=None, k=None, v=None) == A
    assert call(qo=heads(row=512)) == A and call(r=wino.WinoRope(63, 0, 1.0, FAKE, None)) == S
    for x, status in ((axes(n=0), S), (axes(n=5), S), (axes(axis=None), A), (axes(positions=None), A),
                      (axes(positions=FAKE + 2), A), (axes(stride=7), S), (axes(stride=-8), S)):
        assert call(x=x) == status
    assert call(r=wino.WinoRope(64, 0, 1.0, FAKE, FAKE), x=axes()) == A  # positions twice
    for n in (norm(qw=FAKE + 2), norm(kw=FAKE + 8), norm(eps=0.0), norm(eps=-1.0), norm(eps=math.nan), norm(eps=2.0 ** -61),
              norm(eps=2.0 ** 61), norm(offset=math.inf), norm(offset=math.nan)):
        assert call(n=n) == A
    for n in (norm(qs=56), norm(ks=-64), norm(qs=68), norm(ks=1 << 37)):
        assert call(n=n) == S


def test_read_refusals():
    L = wino.lib()

    def call(k=heads(), v=heads(FAKE * 2), b=batch(), ws=FAKE):
        return L.wino_cache_read(k, v, b, None, ws, None)
    assert call(b=None) == A and call(k=None, v=None) == A and call(ws=None) == A and call(ws=FAKE + 8) == A
    assert call(v=heads()) == A and call(k=heads(FAKE + 2)) == A and call(v=heads(FAKE * 2, row=8)) == S


def tensors(dtype=torch.float8_e4m3fn):
    k = torch.zeros((3, 16, 2, 64), dtype=torch.uint8).view(dtype) if dtype is not torch.bfloat16 else torch.zeros((3, 16, 2, 64), dtype=dtype)
    i, t = torch.zeros(2, dtype=torch.int32), torch.zeros((2, 3), dtype=torch.int32)
    return k, i, t, torch.zeros((3, 2, 16), dtype=torch.uint8)


def test_python_checks_of_batches():
    kw = dict(n_rows=4, n_q_heads=4, mask=0)
    k, i, t, s = tensors()
    b = wino.make_kv_batch(k, k, t, i, i, i, i, k_scale=s, v_scale=s, **kw)
    assert (b.dtype, b.elements, b.page_stride, b.slot_stride, b.head_stride) == (E4M3, BF, 2048, 128, 64)
    assert b.scales.k_scale == s.data_ptr()
    assert wino.make_kv_batch(k, k, t, i, i, i, i, k_scale=s, v_scale=s, dtype=FP, **kw).dtype == E4M3 | wino.WINO_FP16
    assert wino.make_kv_batch(k.view(torch.uint8), k.view(torch.uint8), t, i, i, i, i, k_scale=s, v_scale=s, **kw).dtype == E4M3
    plain = tensors(torch.bfloat16)[0]
    assert wino.make_kv_batch(plain, plain, t, i, i, i, i, **kw).scales is None
    for args, more in (((k, k), {}), ((k, k), dict(k_scale=s)), ((k, k), dict(v_scale=s)), ((plain, plain), dict(k_scale=s, v_scale=s)),
                       ((k, k), dict(k_scale=s, v_scale=s[:2])), ((k, k), dict(k_scale=s.transpose(1, 2), v_scale=s)),
                       ((k, k), dict(k_scale=s.int(), v_scale=s)), ((k, k), dict(k_scale=s, v_scale=s, dtype=torch.float32)),
                       ((k.view(torch.int8), k.view(torch.int8)), dict(k_scale=s, v_scale=s)),
                       ((plain, plain), dict(dtype=FP)), ((k, k), dict(k_scale=s.reshape(3, 16, 2), v_scale=s.reshape(3, 16, 2)))):
        with pytest.raises(wino.WinoError):
            wino.make_kv_batch(*args, t, i, i, i, i, **more, **kw)


def test_python_checks_of_norms_and_axes():
    w = torch.zeros(64, dtype=BF)
    n = wino.make_head_norm(w, w.expand(2, 64).contiguous(), offset=1.0)
    assert (n.q_head_stride, n.k_head_stride, n.offset) == (0, 64, 1.0) and n.shapes == ((64,), (2, 64))
    assert wino.make_head_norm(None, w).q_weight is None
    for args in ((w.float(), w), (w, w.half()), (w[None, None], w), (torch.zeros(128, dtype=BF)[::2], w)):
        with pytest.raises(wino.WinoError):
            wino.make_head_norm(*args)
    axis, pos = torch.zeros(32, dtype=torch.uint8), torch.zeros((3, 10), dtype=torch.int32)
    a = wino.make_rope_axes(axis, pos[:, :4])
    assert (a.n_axes, a.axis_stride, a.n_positions, a.n_pairs) == (3, 10, 4, 32)
    for args in ((axis.int(), pos), (axis, pos.long()), (axis, pos[0]), (axis, pos.T), (axis[::2], pos)):
        with pytest.raises(wino.WinoError):
            wino.make_rope_axes(*args)


def test_python_checks_of_calls(monkeypatch):
    """Weights, axes and outputs that do not fit the batch; nothing is launched."""
    monkeypatch.setattr(_abi, "_current_device", lambda: 0)
    k, i, t, s = tensors()
    b = wino.make_kv_batch(k, k, t, i, i, i, i, k_scale=s, v_scale=s, n_rows=4, n_q_heads=4, mask=0)
    b.device, b.devices = 0, {0}
    ws = type("Ws", (), dict(numel=lambda self: 256, element_size=lambda self: 1, get_device=lambda self: 0, data_ptr=lambda self: FAKE))()
    w, axis, pos = torch.zeros(64, dtype=BF), torch.zeros(16, dtype=torch.uint8), torch.zeros((2, 4), dtype=torch.int32)
    rope = wino.make_rope(None, rot_dim=0)

    def status(**kw):
        with pytest.raises(wino.WinoError) as e:
            wino.wino_norm_rope_append(None, None, None, b, rope, ws, **kw)
        return e.value.status
    assert status(norm=wino.make_head_norm(w[:32], None)) == S and status(norm=wino.make_head_norm(w.expand(2, 64).contiguous(), None)) == S
    assert status(norm=wino.make_head_norm(None, w.expand(4, 64).contiguous())) == S
    assert status(norm=wino.make_head_norm(w, w)) == A  # on the host
    assert status(axes=wino.make_rope_axes(axis, pos)) == S  # 16 pairs for none
    assert status(axes=wino.make_rope_axes(axis[:0], pos[:, :3])) == S
    assert status(axes=wino.make_rope_axes(axis[:0], pos)) == A  # on the host
    for args in ((torch.zeros((4, 4, 64), dtype=BF), None), (None, torch.zeros((4, 2, 64), dtype=FP))):
        with pytest.raises(wino.WinoError):
            wino.wino_cache_read(*args, b, ws)


@pytest.mark.parametrize("name,mirror", [("wino_kv_scales", "WinoKvScales"), ("wino_head_norm", "WinoHeadNorm"),
                                         ("wino_rope_axes", "WinoRopeAxes")])
def test_struct_layout_matches_header(tmp_path, name, mirror):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no gcc")
    cls = getattr(wino, mirror)
    fields = [f[0] for f in cls._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "wino.h"\nint main(void) {\n'
                   f'    printf("%zu\\n%d\\n", sizeof({name}), WINO_CACHE_E4M3);\n' +
                   "".join(f'    printf("%zu\\n", offsetof({name}, {f}));\n' for f in fields) + "    return 0;\n}\n")
    exe = tmp_path / "layout"
    inc = Path(__file__).resolve().parent.parent / "include"
    subprocess.run([gcc, "-std=c11", "-I", str(inc), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [C.sizeof(cls), E4M3] + [getattr(cls, f).offset for f in fields]


def test_the_definition_itself():
    """nearest_code against a search over the format's values, exponents against the inequality, both against torch."""
    v = code_values()
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(v, codes, equal_nan=True)
    fine = np.sort(v[np.isfinite(v)])
    rng = np.random.default_rng(1)
    x = np.concatenate([fine, (fine[1:] + fine[:-1]) / 2, rng.uniform(-460, 460, 2000), rng.standard_normal(2000) * 0.02])
    got = nearest_code(x)
    assert np.isin(got, fine).all()
    assert np.allclose(np.abs(got - np.clip(x, -448, 448)), np.abs(fine[None] - np.clip(x, -448, 448)[:, None]).min(1), rtol=0, atol=1e-12)
    half = (fine[1:] + fine[:-1]) / 2  # ties: the code with the even last bit
    even = {float(f): c % 2 == 0 for c, f in enumerate(v) if np.isfinite(f)}
    assert all(even[float(r)] for r in nearest_code(half) if r != 0)
    for dtype in (BF, FP):
        z = rng.standard_normal((400, 64)) * 2.0 ** rng.uniform(-20, 22, (400, 1))
        z[0] = 0.0
        z[1, 3], z[2, 3], z[3, 3] = 448.0 * 4, 449.0 * 4, 1e30
        e = exponents(z, dtype)
        most = np.abs(z).max(-1)
        e_min = -110 if dtype is BF else -14
        assert ((most <= 448 * 2.0 ** e) | (e == 7)).all() and ((most > 448 * 2.0 ** (e - 1)) | (e == e_min)).all()
        codes, s = quantise(torch.from_numpy(z)[None, :, None], dtype)
        assert np.array_equal(values_of(codes, s, dtype)[0, :, 0].double().numpy(), held_values(z, dtype))


def test_block_cache_in_8_bits():
    from paper_2605_16941_gb300 import loop
    c = loop.BlockCache(2, 3, 50, 8, 4, 2, 64, page_size=16, device="cpu", scaled=True, dtype=FP)
    assert c.k.dtype == torch.float8_e4m3fn and c.k_scale.shape == c.k.shape[:-1] and c.k_scale.dtype == torch.uint8
    for b in (c.step(20)[1], c.context(0, 20)[1]):
        assert b.dtype == E4M3 | wino.WINO_FP16 and b.k_cache == c.k[1].data_ptr() and b.scales.v_scale == c.v_scale[1].data_ptr()
    with pytest.raises(wino.WinoError):
        loop.BlockCache(1, 1, 50, 8, 4, 2, 24, page_size=16, device="cpu", scaled=True)
