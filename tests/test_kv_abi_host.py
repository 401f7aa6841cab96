"""The paged-cache entry points without a GPU: refusals before anything is launched, the rotary frequencies, and the
ctypes mirrors of their structs."""
import ctypes as C
import math
import shutil
import subprocess
from pathlib import Path
from types import SimpleNamespace

import pytest
import torch

import paper_2605_16941_gb300 as wino
from paper_2605_16941_gb300 import _abi

FAKE = 0x10000  # aligned, never dereferenced: every call below fails its checks first


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


BAD_BATCHES = [
    (dict(q_start=None), "ARG"), (dict(q_len=None), "ARG"), (dict(kv_len=None), "ARG"), (dict(new_slot=None), "ARG"),
    (dict(page_table=None), "ARG"), (dict(k_cache=None), "ARG"), (dict(v_cache=None), "ARG"),
    (dict(q_start=FAKE + 2), "ARG"), (dict(page_table=FAKE + 1), "ARG"), (dict(k_cache=FAKE + 8), "ARG"),
    (dict(v_cache=FAKE + 2), "ARG"), (dict(dtype=2), "ARG"), (dict(mask=3), "ARG"), (dict(mask=-1), "ARG"),
    (dict(n_seq=0), "SHAPE"), (dict(n_seq=16385), "SHAPE"), (dict(n_rows=0), "SHAPE"), (dict(n_rows=(1 << 24) + 1), "SHAPE"),
    (dict(n_kv_heads=0), "SHAPE"), (dict(n_q_heads=3), "SHAPE"), (dict(n_q_heads=1), "SHAPE"),
    (dict(n_q_heads=2 * 129), "SHAPE"), (dict(n_kv_heads=1025, n_q_heads=1025), "SHAPE"),
    (dict(head_dim=0), "SHAPE"), (dict(head_dim=60), "SHAPE"), (dict(head_dim=136), "SHAPE"),
    (dict(page_size=8), "SHAPE"), (dict(page_size=48), "SHAPE"), (dict(page_size=192), "SHAPE"), (dict(page_size=0), "SHAPE"),
    (dict(n_pages=0), "SHAPE"), (dict(table_width=0), "SHAPE"), (dict(table_width=(1 << 26) + 1), "SHAPE"),
    (dict(page_stride=2044), "SHAPE"), (dict(slot_stride=56), "SHAPE"), (dict(head_stride=0), "SHAPE"),
    (dict(page_stride=1 << 37), "SHAPE"), (dict(page_stride=-2048), "SHAPE"),
]


@pytest.mark.parametrize("bad,status", BAD_BATCHES)
def test_batch_refusals(bad, status):
    L = wino.lib()
    want = getattr(wino, "WINO_ERR_" + status)
    b = batch(**bad)
    rope = wino.WinoRope(0, 0, 1.0, None, None)
    h = heads()
    out = C.c_size_t(0)
    assert L.wino_attend(h, heads(FAKE * 2), 0.125, b, FAKE, 1 << 40, None) == want
    assert L.wino_rope_append(h, h, heads(), heads(), b, rope, FAKE, None) == want
    assert L.wino_attend_workspace_size(b, C.byref(out)) == want


def test_attend_refusals():
    L = wino.lib()

    def call(q=heads(), out=heads(FAKE * 2), scale=0.125, b=batch(), ws=FAKE, n=1 << 40):
        return L.wino_attend(q, out, scale, b, ws, n, None)
    A, S, W = wino.WINO_ERR_ARG, wino.WINO_ERR_SHAPE, wino.WINO_ERR_WORKSPACE
    assert call(b=None) == A and call(q=None) == A and call(out=None) == A and call(ws=None) == A
    assert call(ws=FAKE + 16) == A
    assert call(q=heads(None)) == A and call(q=heads(FAKE + 8)) == A and call(out=heads(FAKE * 2 + 2)) == A
    assert call(out=heads()) == A  # onto q
    for scale in (0.0, -1.0, 2.0 ** 127, math.inf, math.nan):
        assert call(scale=scale) == A, scale
    for q in (heads(row=260), heads(row=56), heads(head=60), heads(head=0), heads(row=1 << 37)):
        assert call(q=q) == S and call(out=wino.WinoHeads(FAKE * 2, q.row_stride, q.head_stride)) == S
    assert call(n=100) == W


def test_attend_refuses_subnormal_scales():
    L = wino.lib()

    def call(scale):  # a workspace too small for it is found behind the scale
        return L.wino_attend(heads(), heads(FAKE * 2), scale, batch(), FAKE, 100, None)
    for scale in (1e-45, 1e-42, 2.0 ** -127):
        assert call(scale) == wino.WINO_ERR_ARG, scale
    for scale in (2.0 ** -126, 1e-30):
        assert call(scale) == wino.WINO_ERR_WORKSPACE, scale


def test_append_refusals():
    L = wino.lib()

    def rope(rot=64, factor=1.0, freq=FAKE, pos=None):
        return wino.WinoRope(rot, 0, factor, freq, pos)

    def call(q=heads(), qo=heads(FAKE * 2), k=heads(), v=heads(), b=batch(), r=rope(), ws=FAKE):
        return L.wino_rope_append(q, qo, k, v, b, r, ws, None)
    A, S = wino.WINO_ERR_ARG, wino.WINO_ERR_SHAPE
    assert call(b=None) == A and call(r=None) == A and call(ws=None) == A and call(ws=FAKE + 8) == A
    assert call(q=None) == A and call(qo=None) == A and call(k=None) == A and call(v=None) == A  # halves of a pair
    assert call(q=None, qo=None, k=None, v=None) == A
    assert call(k=heads(FAKE + 2)) == A and call(v=heads(head=12)) == S and call(qo=heads(FAKE * 2, row=8)) == S
    assert call(r=rope(rot=63)) == S and call(r=rope(rot=66)) == S and call(r=rope(rot=-2)) == S
    assert call(r=rope(freq=None)) == A and call(r=rope(freq=FAKE + 4)) == A and call(r=rope(pos=FAKE + 2)) == A
    assert call(r=rope(factor=math.inf)) == A and call(r=rope(factor=math.nan)) == A
    assert call(qo=heads(row=512)) == A  # q's memory with other strides


def test_workspace_size():
    n = wino.wino_attend_workspace_size(batch())
    assert n >= 256 and n % 256 == 0
    assert wino.wino_attend_workspace_size(batch(n_rows=1 << 20)) >= n
    assert wino.lib().wino_attend_workspace_size(batch(), None) == wino.WINO_ERR_ARG


def test_frequencies():
    f, m = wino.wino_rope_frequencies(64, 10000.0)
    assert m == 1.0 and f.dtype == torch.float64
    want = [10000.0 ** (-2 * j / 64) for j in range(32)]
    assert torch.allclose(f, torch.tensor(want, dtype=torch.float64), rtol=1e-15, atol=0)
    g, m = wino.wino_rope_frequencies(64, 10000.0, scaling="linear", factor=4.0)
    assert m == 1.0 and torch.equal(g, f / 4)
    g, m = wino.wino_rope_frequencies(64, 10000.0, scaling="parts", factor=16.0, trained_len=4096)
    assert m == pytest.approx(0.1 * math.log(16.0) + 1, rel=1e-6)
    turns = 4096 * f / (2 * math.pi)
    assert torch.equal(g[turns > 32], f[turns > 32]) and (turns > 32).any()
    assert torch.allclose(g[turns < 1], f[turns < 1] / 16, rtol=1e-15, atol=0) and (turns < 1).any()
    mid = (turns > 1) & (turns < 32)
    assert mid.any() and (g[mid] < f[mid]).all() and (g[mid] > f[mid] / 16).all()
    assert wino.wino_rope_frequencies(0, 10000.0)[0].numel() == 0


@pytest.mark.parametrize("args,kw,status", [
    ((63, 1e4), {}, "SHAPE"), ((-2, 1e4), {}, "SHAPE"), ((130, 1e4), {}, "SHAPE"), ((64, 1.0), {}, "ARG"),
    ((64, math.inf), {}, "ARG"), ((64, math.nan), {}, "ARG"), ((64, 1e4), dict(scaling="linear", factor=0.5), "ARG"),
    ((64, 1e4), dict(scaling="parts", factor=math.nan), "ARG"),
    ((64, 1e4), dict(scaling="parts", factor=2.0, trained_len=0), "ARG"),
])
def test_frequency_refusals(args, kw, status):
    with pytest.raises(wino.WinoError) as e:
        wino.wino_rope_frequencies(*args, **kw)
    assert e.value.status == getattr(wino, "WINO_ERR_" + status)


def test_python_checks():
    """What the binding itself refuses: types, shapes, layouts."""
    kw = dict(n_rows=4, n_q_heads=4, mask=0)
    k, i, t = torch.zeros((3, 16, 2, 64), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32), torch.zeros((2, 3), dtype=torch.int32)
    b = wino.make_kv_batch(k, k, t, i, i, i, i, **kw)
    assert (b.n_seq, b.n_pages, b.page_size, b.n_kv_heads, b.head_dim, b.table_width) == (2, 3, 16, 2, 64, 3)
    assert (b.page_stride, b.slot_stride, b.head_stride, b.dtype) == (2048, 128, 64, wino.WINO_BF16)
    assert wino.make_kv_batch(k.half(), k.half(), t, i, i, i, i, **kw).dtype == wino.WINO_FP16
    for args in ((k, k[:, :, :1], t, i, i, i, i), (k, k.half(), t, i, i, i, i), (k.float(), k.float(), t, i, i, i, i),
                 (k, k, t.long(), i, i, i, i), (k, k, t, i.long(), i, i, i), (k, k, t, i[:1], i, i, i),
                 (k, k, t, i, i, i, torch.zeros(4, dtype=torch.int32)[::2]), (k[..., ::2], k[..., ::2], t, i, i, i, i),
                 (k, torch.zeros((3, 2, 16, 64), dtype=torch.bfloat16).transpose(1, 2), t, i, i, i, i)):
        with pytest.raises(wino.WinoError):
            wino.make_kv_batch(*args, **kw)
    with pytest.raises(wino.WinoError):
        wino.make_rope(torch.zeros(32), rot_dim=64)
    with pytest.raises(wino.WinoError):
        wino.make_rope(torch.zeros(31, dtype=torch.float64), rot_dim=64)
    with pytest.raises(wino.WinoError):
        wino.make_rope(None, rot_dim=64)
    q = torch.zeros((4, 4, 64), dtype=torch.bfloat16)
    for bad in (q[:3], q[:, :3], q[..., :32], q.half(), q.transpose(0, 1)[..., ::2]):
        with pytest.raises(wino.WinoError):
            _abi._heads(bad, b, b.q_shape, "test")


def test_rope_on_another_device_is_refused(monkeypatch):
    """The frequencies as wino_rope_frequencies returns them, on the host, for a batch on a device; nothing is launched."""
    freq, _ = wino.wino_rope_frequencies(64, 1e4)
    launched = []
    stub = SimpleNamespace(wino_status_string=wino.lib().wino_status_string,
                           wino_rope_append=lambda *a: launched.append(a) or wino.WINO_OK)
    monkeypatch.setattr(_abi, "lib", lambda: stub)
    monkeypatch.setattr(_abi, "_current_device", lambda: 0)
    k, i, t = torch.zeros((3, 16, 2, 64), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32), torch.zeros((2, 3), dtype=torch.int32)
    b = wino.make_kv_batch(k, k, t, i, i, i, i, n_rows=4, n_q_heads=4, mask=0)
    b.device, b.devices = 0, {0}  # as over a cache on device 0
    ws = torch.zeros(256, dtype=torch.uint8)
    for rope in (wino.make_rope(freq, rot_dim=64),
                 wino.make_rope(None, rot_dim=0, positions=torch.zeros(4, dtype=torch.int32))):
        with pytest.raises(wino.WinoError) as e:
            wino.wino_rope_append(None, None, None, b, rope, ws)
        assert e.value.status == wino.WINO_ERR_ARG
    with pytest.raises(wino.WinoError) as e:
        wino.wino_rope_append(None, None, None, b, wino.make_rope(None, rot_dim=0), ws[:255])
    assert e.value.status == wino.WINO_ERR_WORKSPACE and not launched


@pytest.mark.parametrize("name,mirror", [("wino_kv_batch", "WinoKvBatch"), ("wino_rope", "WinoRope"), ("wino_heads", "WinoHeads")])
def test_struct_layout_matches_header(tmp_path, name, mirror):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no gcc")
    cls = getattr(wino, mirror)
    fields = [f[0] for f in cls._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "wino.h"\nint main(void) {\n'
                   f'    printf("%zu\\n", sizeof({name}));\n' +
                   "".join(f'    printf("%zu\\n", offsetof({name}, {f}));\n' for f in fields) + "    return 0;\n}\n")
    exe = tmp_path / "layout"
    inc = Path(__file__).resolve().parent.parent / "include"
    subprocess.run([gcc, "-std=c11", "-I", str(inc), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [C.sizeof(cls)] + [getattr(cls, f).offset for f in fields]


def test_work_that_cannot_be_counted_is_refused():
    """Beyond 2^62 units; the check needs no device."""
    b = batch(n_seq=16384, n_rows=1 << 24, n_q_heads=1024 * 128, n_kv_heads=1024, page_size=1 << 20, table_width=1 << 10,
              head_dim=8, head_stride=8, slot_stride=8192, page_stride=8192 << 20)
    assert wino.lib().wino_attend(heads(row=1 << 20, head=8), heads(FAKE * 2, row=1 << 20, head=8), 0.1, b, FAKE, 1 << 40,
                                  None) == wino.WINO_ERR_SHAPE
