"""Calls over a paged cache that the documentation allows at its borders."""
import subprocess
import sys
from pathlib import Path

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2605_16941_gb300 as wino  # noqa: E402
from kv_helpers import CAUSAL, FULL, SHADOW, add_rows, attend, check, check_on_device, make_kv  # noqa: E402

BF, FP = torch.bfloat16, torch.float16


@pytest.mark.parametrize("n_seq", [1, 3, 70])
@pytest.mark.parametrize("mask", [FULL, CAUSAL, SHADOW], ids=["full", "causal", "shadow"])
def test_every_sequence_absent(mask, n_seq):
    """q_len = 0 throughout: nothing is written, in the cache or in out, and the workspace serves the next call."""
    c = add_rows(make_kv(mask, [(0, 40, 0)] * n_seq, heads=4, kv_heads=2, gap=2))
    keep = c.k_cache.clone()
    ws = wino.attend_workspace(c.batch)
    k = torch.zeros((c.n_rows, 2, 64), dtype=BF, device="cuda")
    wino.wino_rope_append(None, k, k, c.batch, wino.make_rope(None, rot_dim=0), ws)
    attend(c, ws=ws)
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    check(c)
    assert torch.equal(keep.view(torch.int16), c.k_cache.view(torch.int16))
    d = add_rows(make_kv(CAUSAL, [(1, 900, 899)], heads=4, kv_heads=2))
    attend(d, ws=ws)
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    check(d)


FIRST = """
import sys
sys.path.insert(0, {root!r})
sys.path.insert(0, {tests!r})
import torch
import paper_2605_16941_gb300 as wino
from kv_helpers import CAUSAL, add_rows, attend, check, make_kv
c = add_rows(make_kv(CAUSAL, [(3, 300, 297)], heads=4, kv_heads=2, dim={dim}))
ws, rope = wino.attend_workspace(c.batch), wino.make_rope(None, rot_dim=0)
k = torch.randn((c.n_rows, 2, {dim})).to(torch.bfloat16).cuda()
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    wino.wino_rope_append(None, k, k, c.batch, rope, ws)
    attend(c, ws=ws)
g.replay()
assert wino.wino_read_device_status(ws) == wino.WINO_OK
check(c)
print("replayed")
"""


@pytest.mark.parametrize("dim", [64, 128])
def test_first_call_of_a_process_is_captured(dim):
    tests = Path(__file__).resolve().parent
    r = subprocess.run([sys.executable, "-c", FIRST.format(root=str(tests.parent), tests=str(tests), dim=dim)],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "replayed" in r.stdout, r.stdout[-2000:] + r.stderr[-4000:]


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("scale", [2.0 ** -126, 1e-30, 1e-6])
def test_scales_that_level_all_weights(scale, dtype):
    """Scores that vanish: every visible slot weighs the same; from the smallest scale that is allowed."""
    c = add_rows(make_kv(CAUSAL, [(40, 500, 460), (1, 300, 299)], heads=4, kv_heads=2, dtype=dtype))
    ws = attend(c, scale=scale)
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    check(c, scale=scale)


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
def test_tensors_made_on_another_stream(dtype):
    """Inputs written on one stream, the calls on another that waits for it."""
    c = add_rows(make_kv(SHADOW, [(32, 300, 284), (32, 90, 74)], heads=8, kv_heads=2, dim=128, dtype=dtype))
    ws = wino.attend_workspace(c.batch)
    q = c.q.clone()
    c.q.zero_()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(a):
        torch.cuda._sleep(2_000_000)
        c.q.copy_(q)
        e = torch.cuda.Event()
        e.record()
    with torch.cuda.stream(b):
        b.wait_event(e)
        wino.wino_attend(c.q, c.out, c.batch, ws)
    torch.cuda.synchronize()
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    check(c)


def test_the_same_rows_twice_in_one_cache():
    """Two batches over one cache, whose sequences swap their places: the page table alone says whose slots they are."""
    c = add_rows(make_kv(CAUSAL, [(5, 200, 195), (9, 90, 81)], heads=4, kv_heads=2, dim=128, poison=False))
    attend(c)
    check(c)
    c.seqs = c.seqs[::-1]
    c.starts = c.starts[::-1]
    c.table = c.table[::-1].copy()
    c.ints.copy_(torch.from_numpy(np.array([c.starts] + [[s[i] for s in c.seqs] for i in range(3)], dtype=np.int32)))
    c.table_dev.copy_(torch.from_numpy(c.table))
    c.extra["whole"].fill_(77.0)
    attend(c)
    check(c)


@pytest.mark.parametrize("rows", [1, 4, 5, 260])
def test_many_heads(rows):
    """1024 kv heads, the most; and as many query heads to one as fit."""
    c = add_rows(make_kv(CAUSAL, [(rows, rows + 150, 150)], heads=1024, kv_heads=1024, dim=16, page=32))
    ws = attend(c)
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    check_on_device(c)
    d = add_rows(make_kv(SHADOW, [(2 * rows, 300, 300 - rows)], heads=256, kv_heads=2, dim=16))
    ws = attend(d)
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    check_on_device(d)
