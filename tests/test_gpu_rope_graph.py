"""A captured wino_rope_append replayed at other offsets: K, V and the rotated queries of every replay, and nothing else written."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2605_16941_gb300 as wino  # noqa: E402
from kv_helpers import CAUSAL, SHADOW, f64, frequencies, make_kv  # noqa: E402
from test_gpu_rope import close, positions_of, rotated, slots_of  # noqa: E402


@pytest.mark.parametrize("explicit", [False, True], ids=["slots", "positions"])
@pytest.mark.parametrize("mask", [CAUSAL, SHADOW], ids=["causal", "shadow"])
@pytest.mark.parametrize("rot", [64, 20])
def test_replayed_offsets(rot, mask, explicit):
    """new_slot is read again on the device, for the slots and, without explicit positions, for the rotation."""
    heads, kv_heads, dim, n = 4, 2, 64, 4
    c = make_kv(mask, [(n, 30, 8), (n, 25, 3)], heads=heads, kv_heads=kv_heads, dim=dim, poison=False)
    qkv = torch.randn((c.n_rows, heads + 2 * kv_heads, dim)).to(torch.bfloat16).cuda()
    q, k, v = qkv.split([heads, kv_heads, kv_heads], 1)
    freq = frequencies(rot)
    pos = torch.zeros(c.n_rows, dtype=torch.int32, device="cuda") if explicit else None
    rope = wino.make_rope(torch.from_numpy(freq).cuda(), rot_dim=rot, positions=pos)
    out, ws = torch.empty((c.n_rows, heads, dim), dtype=torch.bfloat16, device="cuda"), wino.append_workspace()
    wino.wino_rope_append(q, k, v, c.batch, rope, ws, q_out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        wino.wino_rope_append(q, k, v, c.batch, rope, ws, q_out=out)
    for round_, news in enumerate(([2, 17], [0, 20], [21, 9])):
        qkv.copy_(torch.randn(qkv.shape, generator=torch.Generator().manual_seed(round_)).to(torch.bfloat16))
        c.ints[3].copy_(torch.tensor(news, dtype=torch.int32))
        where = [positions_of(mask, n, kv, new) + (1000 if explicit else 0) for (_, kv, _), new in zip(c.seqs, news)]
        if explicit:
            pos.copy_(torch.from_numpy(np.concatenate(where).astype(np.int32)))
        c.k_cache.fill_(3.0)
        c.v_cache.fill_(5.0)
        out.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        assert wino.wino_read_device_status(ws) == wino.WINO_OK
        x, xk, xv, got, got_k, got_v = (f64(t) for t in (q, k, v, out, c.k_cache, c.v_cache))
        for s, ((_, kv, _), new) in enumerate(zip(c.seqs, news)):
            r = np.arange(n) + c.starts[s]
            p = where[s][:, None]
            close(got[r], x[r], rotated(x[r], p, freq, rot, False, 1.0), rot, 1.0, torch.bfloat16, False)
            slot = slots_of(mask, n, kv, new)
            at = c.table[s, slot // c.page], slot % c.page
            close(got_k[at], xk[r], rotated(xk[r], p, freq, rot, False, 1.0), rot, 1.0, torch.bfloat16, False)
            assert np.array_equal(got_v[at], xv[r])
            got_k[at], got_v[at] = 3.0, 5.0  # the rest is as it was
        assert (got_k == 3.0).all() and (got_v == 5.0).all()
