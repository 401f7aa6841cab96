"""The paged cache, the rotation, the attention and the step together: a small model's decode, whose hidden states come from
two layers over a BlockCache, every call checked against its definition on the inputs that it got."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2605_16941_gb300 as wino  # noqa: E402
from kv_helpers import CAUSAL, FULL, SHADOW, Kv, add_rows, attend, check, expected, f64, frequencies, half_step, make_kv, rotated  # noqa: E402
from paper_2605_16941_gb300 import loop  # noqa: E402

BF = torch.bfloat16
V, D_MODEL, LAYERS, HEADS, KV_HEADS, DIM, PROMPT, L, BLOCKS, N_SEQ = 320, 64, 2, 4, 2, 32, 21, 8, 2, 3
MASK = V - 1
SEQ = PROMPT + L * BLOCKS


class Model:
    """Embedding, two attention layers, LM head; plain matrix products by torch, the rest by the library."""

    def __init__(self, no_shadow, page_size, verify=True):
        g = torch.Generator().manual_seed(5)

        def weights(*shape, scale):
            return (torch.randn(shape, generator=g) * scale).to(BF).cuda()
        self.embed = weights(V, D_MODEL, scale=1.0)
        self.qkv = [weights(D_MODEL, (HEADS + 2 * KV_HEADS) * DIM, scale=0.15) for _ in range(LAYERS)]
        self.out = [weights(HEADS * DIM, D_MODEL, scale=0.1) for _ in range(LAYERS)]
        self.head = weights(V, D_MODEL, scale=0.7)
        self.freq = frequencies(DIM)
        self.rope = wino.make_rope(torch.from_numpy(self.freq).cuda(), rot_dim=DIM)
        self.cache = loop.BlockCache(LAYERS, N_SEQ, SEQ, L, HEADS, KV_HEADS, DIM, page_size=page_size, no_shadow=no_shadow)
        self.no_shadow, self.verify, self.done = no_shadow, verify, 0
        self.calls = 0

    def layers(self, x, batches, mask, seqs, positions):
        """x [rows, D_MODEL] fp32 through the layers, in place."""
        rows = x.size(0)
        for i, b in enumerate(batches):
            qkv = (x.to(BF) @ self.qkv[i]).view(rows, HEADS + 2 * KV_HEADS, DIM)
            q, k, v = qkv.split([HEADS, KV_HEADS, KV_HEADS], 1)
            before = [f64(t) for t in (q, k, v)] if self.verify else None
            self.cache.append(q, k, v, b, self.rope)
            o = torch.full((rows, HEADS, DIM), 77.0, dtype=BF, device="cuda")
            self.cache.attend(q, o, b)
            if self.verify:
                self.check_layer(i, b, mask, seqs, positions, before, q, o)
            x += (o.view(rows, -1) @ self.out[i]).float()
            self.calls += 1
        return x

    def check_layer(self, i, b, mask, seqs, positions, before, q, o):
        torch.cuda.synchronize()
        assert wino.wino_read_device_status(self.cache.ws) == wino.WINO_OK
        kc, vc = self.cache.k[i].transpose(1, 2), self.cache.v[i].transpose(1, 2)
        table = self.cache.page_table.cpu().numpy()
        page = self.cache.k.size(3)
        starts = [s * seqs[0][0] for s in range(N_SEQ)]
        # 2^-20 (|a| + |b|) for the rotation, half a step for the rounding (test_gpu_rope.py)
        def near(got, x, pos):
            want = rotated(x, pos[:, None], self.freq, DIM, False, 1.0)
            size = np.abs(x) + np.abs(np.roll(x, DIM // 2, -1))
            assert (np.abs(got - want) <= 2.0 ** -20 * size + 1.001 * half_step(BF) * np.abs(want)).all()
        near(f64(q), before[0], positions)
        for s, (n, kv, new) in enumerate(seqs):
            r = np.arange(n)
            slot = np.where(r < n // 2, new + r, kv + r - n // 2) if mask == SHADOW else new + r
            at = table[s, slot // page], slot % page
            near(f64(kc)[at], before[1][starts[s] + r], positions[starts[s] + r])
            assert np.array_equal(f64(vc)[at], before[2][starts[s] + r])
        c = Kv(mask, seqs, HEADS, KV_HEADS, DIM, page, BF, starts, q.size(0), table, kc, vc, None, None, b, q, o,
               dict(whole=o))
        check(c)

    def hidden(self, tokens):
        def step(k, blk_start):
            if self.done < blk_start:  # the prompt, or the block before: into the cache once
                rows = tokens[:, self.done:blk_start]
                n = blk_start - self.done
                seqs = [(n, blk_start, self.done)] * N_SEQ
                pos = np.tile(np.arange(self.done, blk_start), N_SEQ)
                self.layers(self.embed[rows.reshape(-1).long()].float(), self.cache.context(self.done, blk_start), FULL,
                            seqs, pos)
                self.done = blk_start
            block = tokens[:, blk_start:blk_start + L]
            kinds = 1 if self.no_shadow else 2
            ids = block if self.no_shadow else torch.stack([block, torch.full_like(block, MASK)], 1)
            seqs = [(kinds * L, blk_start + L, blk_start)] * N_SEQ
            pos = np.tile(np.arange(blk_start, blk_start + L), N_SEQ * kinds)
            x = self.layers(self.embed[ids.reshape(-1).long()].float(), self.cache.step(blk_start),
                            FULL if self.no_shadow else SHADOW, seqs, pos)
            self.h = x.to(BF)
            return self.h
        return step


def start_state():
    g = torch.Generator().manual_seed(9)
    tokens = torch.full((N_SEQ, SEQ), MASK, dtype=torch.int32)
    tokens[:, :PROMPT] = torch.randint(0, MASK, (N_SEQ, PROMPT), generator=g)
    return tokens.cuda()


@pytest.mark.parametrize("no_shadow", [False, True], ids=["shadow", "no_shadow"])
@pytest.mark.parametrize("page_size", [16, 64])
def test_decode_over_a_block_cache(no_shadow, page_size):
    m = Model(no_shadow, page_size)
    tokens = start_state()
    stats = loop.decode(m.head, tokens, prompt_len=PROMPT, blk_len=L, n_blocks=BLOCKS, tau1=0.5, tau2=0.05, mask_id=MASK,
                        hidden=m.hidden(tokens), no_shadow=no_shadow, max_steps=200)
    assert not (tokens == MASK).any() and m.calls == LAYERS * (stats.total_steps + BLOCKS)


def test_native_decode_gives_the_same_tokens():
    """The library's own loop over the same callback; the checks of the layers left out."""
    out = []
    for run in (loop.decode, loop.decode_native):
        m = Model(False, 32, verify=False)
        tokens = start_state()
        run(m.head, tokens, prompt_len=PROMPT, blk_len=L, n_blocks=BLOCKS, tau1=0.5, tau2=0.05, mask_id=MASK,
            hidden=m.hidden(tokens), max_steps=200)
        out.append(tokens.cpu())
    assert torch.equal(out[0], out[1])


def test_captured_layer_and_step():
    """Append, attend and step in one graph, replayed on new rows: as the calls by themselves."""
    m = Model(False, 16, verify=False)
    tokens = start_state()
    step = m.hidden(tokens)
    step(0, PROMPT)  # the prompt is in the cache
    batch = m.cache.step(PROMPT)[0]
    rows = N_SEQ * 2 * L
    qkv = torch.randn((rows, HEADS + 2 * KV_HEADS, DIM)).to(BF).cuda()
    parts = qkv.split([HEADS, KV_HEADS, KV_HEADS], 1)
    q_out, o = (torch.zeros((rows, HEADS, DIM), dtype=BF, device="cuda") for _ in range(2))
    p = wino.make_params(0.5, 0.05, MASK, N_SEQ, SEQ, PROMPT, L)
    ws, kws = wino.step_workspace(p, HEADS * DIM, V), wino.attend_workspace(batch)
    head = torch.randn((V, HEADS * DIM)).to(BF).cuda()
    counts = torch.zeros((N_SEQ, 3), dtype=torch.int32, device="cuda")

    def calls():
        wino.wino_rope_append(*parts, batch, m.rope, kws, q_out=q_out)
        wino.wino_attend(q_out, o, batch, kws)
        wino.wino_step(o.view(rows, -1), head, tokens, p, counts, ws)
    keep = tokens.clone()
    calls()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls()
    for seed in range(3):
        qkv.copy_(torch.randn(qkv.shape, generator=torch.Generator().manual_seed(seed)).to(BF))
        tokens.copy_(keep)
        g.replay()
        torch.cuda.synchronize()
        got = o.clone(), tokens.clone(), counts.clone()
        tokens.copy_(keep)
        calls()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (o, tokens, counts)))
        assert wino.wino_read_device_status(kws) == wino.WINO_OK == wino.wino_read_device_status(ws)


def test_finished_sequences_keep_their_rows():
    """q_len = 0 leaves a sequence's rows, slots and outputs as they are, in both calls."""
    c = add_rows(make_kv(SHADOW, [(16, 40, 30), (0, 40, 30), (16, 25, 10)], heads=4, kv_heads=2, gap=4))
    k0 = c.k_cache.clone()
    rope = wino.make_rope(None, rot_dim=0)
    k = torch.randn((c.n_rows, 2, 64)).to(BF).cuda()
    ws = wino.attend_workspace(c.batch)
    wino.wino_rope_append(None, k, k, c.batch, rope, ws)
    attend(c, ws=ws)
    torch.cuda.synchronize()
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    check(c)
    pages = c.table[1][c.table[1] >= 0]
    assert torch.equal(c.k_cache[pages].view(torch.int16), k0[pages].view(torch.int16))


def test_block_cache_refuses_positions_outside():
    cache = loop.BlockCache(1, 2, 40, 8, 4, 2, 64, page_size=16)
    for a, b in ((-1, 4), (4, 4), (10, 41)):
        with pytest.raises(ValueError):
            cache.context(a, b)
    for s in (-1, 33):
        with pytest.raises(ValueError):
            cache.step(s)


def test_captured_step_outlives_a_larger_context():
    """The cache's workspace stays where a captured step found it, whatever rows come later."""
    cache = loop.BlockCache(1, 2, 200, 8, 4, 2, 64, page_size=16)
    cache.k.normal_()
    cache.v.normal_()
    at = cache.ws.data_ptr()
    batch = cache.step(96)[0]
    q, o, want = (torch.randn((32, 4, 64)).to(BF).cuda() for _ in range(3))
    cache.attend(q, want, batch)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cache.attend(q, o, batch)
    big = cache.context(104, 200)[0]
    x = torch.randn((192, 4, 64)).to(BF).cuda()
    y = torch.zeros_like(x)
    cache.attend(x, y, big)
    g.replay()
    torch.cuda.synchronize()
    assert cache.ws.data_ptr() == at and torch.equal(o, want) and y.abs().sum() > 0
    assert wino.wino_read_device_status(cache.ws) == wino.WINO_OK
