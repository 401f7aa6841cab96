"""BlockCache in 8 bits, with norms and rotary axes, in a small model's decode: every call of every layer checked against its
definition on the inputs that it got, through steps, contexts and the native loop (tau2 = 0: random weights would re-mask for ever)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2605_16941_gb300 as wino  # noqa: E402
from cache8_helpers import BF, FP, held_values, normed, values_of  # noqa: E402
from kv_helpers import FULL, SHADOW, Kv, check, f64, frequencies, half_step  # noqa: E402
from paper_2605_16941_gb300 import loop  # noqa: E402
from test_gpu_norm_rope import check_codes, rounding_slack  # noqa: E402

V, D_MODEL, LAYERS, HEADS, KV_HEADS, DIM, PROMPT, L, BLOCKS, N_SEQ = 320, 64, 2, 4, 2, 32, 21, 8, 2, 3
MASK, EPS, AXES = V - 1, 1e-6, 3
SEQ = PROMPT + L * BLOCKS


class Model:
    """Embedding, two layers whose queries and keys are normalised and turned by three axes, LM head."""

    def __init__(self, scaled, no_shadow=False, verify=True, dtype=BF):
        g = torch.Generator().manual_seed(5)

        def weights(*shape, scale, shift=0.0):
            return (torch.randn(shape, generator=g) * scale + shift).to(dtype).cuda()
        self.embed = weights(V, D_MODEL, scale=1.0)
        self.qkv = [weights(D_MODEL, (HEADS + 2 * KV_HEADS) * DIM, scale=0.15) for _ in range(LAYERS)]
        self.out = [weights(HEADS * DIM, D_MODEL, scale=0.1) for _ in range(LAYERS)]
        self.norm_weights = [(weights(DIM, scale=0.2, shift=1.0), weights(DIM, scale=0.2, shift=1.0)) for _ in range(LAYERS)]
        self.norms = [wino.make_head_norm(*w, eps=EPS) for w in self.norm_weights]
        self.head = weights(V, D_MODEL, scale=0.7).to(BF)
        self.freq = frequencies(DIM)
        self.rope = wino.make_rope(torch.from_numpy(self.freq).cuda(), rot_dim=DIM)
        self.axis = torch.arange(DIM // 2, dtype=torch.uint8) % AXES
        self.cache = loop.BlockCache(LAYERS, N_SEQ, SEQ, L, HEADS, KV_HEADS, DIM, page_size=16, no_shadow=no_shadow, scaled=scaled,
                                     dtype=dtype)
        self.scaled, self.no_shadow, self.verify, self.dtype, self.done, self.calls = scaled, no_shadow, verify, dtype, 0, 0

    def axes(self, positions):
        """Time by 16 tokens, height and width in squares of 4."""
        p = torch.as_tensor(positions, dtype=torch.int32)
        return torch.stack([p // 16, p // 4 % 4, p % 4])

    def layers(self, x, batches, mask, seqs, positions):
        rows = x.size(0)
        pos = self.axes(positions)
        axes = wino.make_rope_axes(self.axis.cuda(), pos.cuda())
        for i, b in enumerate(batches):
            qkv = (x.to(self.dtype) @ self.qkv[i]).view(rows, HEADS + 2 * KV_HEADS, DIM)
            q, k, v = qkv.split([HEADS, KV_HEADS, KV_HEADS], 1)
            before = [f64(t) for t in (q, k, v)] if self.verify else None
            self.cache.append(q, k, v, b, self.rope, norm=self.norms[i], axes=axes)
            o = torch.full((rows, HEADS, DIM), 77.0, dtype=self.dtype, device="cuda")
            self.cache.attend(q, o, b)
            if self.verify:
                self.check_layer(i, b, mask, seqs, pos.numpy(), before, q, o)
            x += (o.view(rows, -1) @ self.out[i]).float()
            self.calls += 1
        return x

    def turned(self, x, weight, pos):
        z = normed(x, weight, EPS, 0.0)
        t = pos[self.axis.numpy()].T[:, None].astype(np.float64) * self.freq
        a, b = z[..., :DIM // 2], z[..., DIM // 2:]
        size = np.abs(a) + np.abs(b)
        y = np.concatenate([a * np.cos(t) - b * np.sin(t), b * np.cos(t) + a * np.sin(t)], -1)
        return y, rounding_slack(y, np.concatenate([size, size], -1))

    def check_layer(self, i, b, mask, seqs, pos, before, q, o):
        torch.cuda.synchronize()
        assert wino.wino_read_device_status(self.cache.ws) == wino.WINO_OK
        read = [torch.empty((q.size(0), KV_HEADS, DIM), dtype=self.dtype, device="cuda") for _ in range(2)]
        self.cache.read(*read, b)
        for got, (z, slack) in ((q, self.turned(before[0], self.norm_weights[i][0], pos)),) + \
                (() if self.scaled else ((read[0], self.turned(before[1], self.norm_weights[i][1], pos)),)):
            tol = slack + 1.001 * half_step(self.dtype) * (np.abs(z) + slack) + (2.0 ** -25 if self.dtype == FP else 0.0)
            assert (np.abs(f64(got) - z) <= tol).all()
        if self.scaled:
            check_codes(f64(read[0]), *self.turned(before[1], self.norm_weights[i][1], pos), self.dtype, False)
            assert np.array_equal(f64(read[1]), held_values(before[2], self.dtype))
        else:
            assert np.array_equal(f64(read[1]), before[2])
        kc, vc = self.cache.k[i].transpose(1, 2), self.cache.v[i].transpose(1, 2)
        if self.scaled:
            kc, vc = values_of(kc, self.cache.k_scale[i], self.dtype), values_of(vc, self.cache.v_scale[i], self.dtype)
        c = Kv(mask, seqs, HEADS, KV_HEADS, DIM, 16, self.dtype, [s * seqs[0][0] for s in range(N_SEQ)], q.size(0),
               self.cache.page_table.cpu().numpy(), kc, vc, None, None, b, q, o, dict(whole=o))
        check(c)

    def hidden(self, tokens):
        def step(k, blk_start):
            if self.done < blk_start:
                rows, n = tokens[:, self.done:blk_start], blk_start - self.done
                pos = np.tile(np.arange(self.done, blk_start), N_SEQ)
                self.layers(self.embed[rows.reshape(-1).long()].float(), self.cache.context(self.done, blk_start), FULL,
                            [(n, blk_start, self.done)] * N_SEQ, pos)
                self.done = blk_start
            block = tokens[:, blk_start:blk_start + L]
            kinds = 1 if self.no_shadow else 2
            ids = block if self.no_shadow else torch.stack([block, torch.full_like(block, MASK)], 1)
            pos = np.tile(np.arange(blk_start, blk_start + L), N_SEQ * kinds)
            x = self.layers(self.embed[ids.reshape(-1).long()].float(), self.cache.step(blk_start), FULL if self.no_shadow else SHADOW,
                            [(kinds * L, blk_start + L, blk_start)] * N_SEQ, pos)
            self.h = x.to(BF)
            return self.h
        return step


def start_state():
    g = torch.Generator().manual_seed(9)
    tokens = torch.full((N_SEQ, SEQ), MASK, dtype=torch.int32)
    tokens[:, :PROMPT] = torch.randint(0, MASK, (N_SEQ, PROMPT), generator=g)
    return tokens.cuda()


@pytest.mark.parametrize("scaled,no_shadow,dtype", [(True, False, BF), (True, True, BF), (True, False, FP), (False, False, BF)],
                         ids=["e4m3", "e4m3_no_shadow", "e4m3_fp16", "plain"])
def test_decode_over_a_block_cache(scaled, no_shadow, dtype):
    m = Model(scaled, no_shadow, dtype=dtype)
    tokens = start_state()
    stats = loop.decode(m.head, tokens, prompt_len=PROMPT, blk_len=L, n_blocks=BLOCKS, tau1=0.5, tau2=0.0, mask_id=MASK,
                        hidden=m.hidden(tokens), no_shadow=no_shadow, max_steps=200)
    assert not (tokens == MASK).any() and m.calls == LAYERS * (stats.total_steps + BLOCKS)


def test_native_decode_gives_the_same_tokens():
    out = []
    for run in (loop.decode, loop.decode_native):
        m = Model(True, verify=False)
        tokens = start_state()
        run(m.head, tokens, prompt_len=PROMPT, blk_len=L, n_blocks=BLOCKS, tau1=0.5, tau2=0.0, mask_id=MASK, hidden=m.hidden(tokens),
            max_steps=200)
        out.append(tokens.cpu())
    assert torch.equal(out[0], out[1])


def test_captured_layer_and_step():
    """Append, attend, read and step in one graph, replayed on new rows: as the calls by themselves."""
    m = Model(True, verify=False)
    tokens = start_state()
    m.hidden(tokens)(0, PROMPT)
    batch = m.cache.step(PROMPT)[0]
    rows = N_SEQ * 2 * L
    qkv = torch.randn((rows, HEADS + 2 * KV_HEADS, DIM)).to(BF).cuda()
    parts = qkv.split([HEADS, KV_HEADS, KV_HEADS], 1)
    axes = wino.make_rope_axes(m.axis.cuda(), m.axes(np.tile(np.arange(PROMPT, PROMPT + L), 2 * N_SEQ)).cuda())
    q_out, o = (torch.zeros((rows, HEADS, DIM), dtype=BF, device="cuda") for _ in range(2))
    read = [torch.zeros((rows, KV_HEADS, DIM), dtype=BF, device="cuda") for _ in range(2)]
    p = wino.make_params(0.5, 0.05, MASK, N_SEQ, SEQ, PROMPT, L)
    ws = wino.step_workspace(p, HEADS * DIM, V)
    head = torch.randn((V, HEADS * DIM)).to(BF).cuda()
    counts = torch.zeros((N_SEQ, 3), dtype=torch.int32, device="cuda")

    def calls():
        wino.wino_norm_rope_append(*parts, batch, m.rope, m.cache.ws, norm=m.norms[0], axes=axes, q_out=q_out)
        m.cache.attend(q_out, o, batch)
        m.cache.read(*read, batch)
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
        got = [t.clone() for t in (o, tokens, counts, *read)]
        tokens.copy_(keep)
        calls()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (o, tokens, counts, *read)))
        assert wino.wino_read_device_status(m.cache.ws) == wino.WINO_OK == wino.wino_read_device_status(ws)


def test_single_tokens_behind_a_prompt():
    """The prompt's rows, then tokens one by one over the same cache, in fp16: the kernel of few rows beside that of many."""
    cache = loop.BlockCache(1, N_SEQ, 60, 1, 8, 2, 64, page_size=16, dtype=FP, no_shadow=True, scaled=True)
    rope = wino.make_rope(None, rot_dim=0)
    g = torch.Generator().manual_seed(2)
    for start, end in ((0, 50),) + tuple((i, i + 1) for i in range(50, 60)):
        n = end - start
        q, k, v = torch.randn((N_SEQ * n, 12, 64), generator=g).to(FP).cuda().split([8, 2, 2], 1)
        out = torch.full((N_SEQ * n, 8, 64), 77.0, dtype=FP, device="cuda")
        batch = cache.context(start, end)[0]
        cache.append(q, k, v, batch, rope)
        cache.attend(q, out, batch)
        assert wino.wino_read_device_status(cache.ws) == wino.WINO_OK
        kc, vc = (values_of(t[0].transpose(1, 2), s[0], FP) for t, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
        check(Kv(FULL, [(n, end, start)] * N_SEQ, 8, 2, 64, 16, FP, [s * n for s in range(N_SEQ)], N_SEQ * n,
                 cache.page_table.cpu().numpy(), kc, vc, None, None, batch, q, out, dict(whole=out)))


def test_the_plain_calls_refuse_the_cache():
    cache = loop.BlockCache(1, 2, 40, 8, 4, 2, 64, page_size=16, scaled=True)
    batch = cache.step(8)[0]
    q, k = torch.zeros((32, 4, 64), dtype=BF, device="cuda"), torch.zeros((32, 2, 64), dtype=BF, device="cuda")
    for call in (lambda: wino.wino_attend(q, torch.empty_like(q), batch, cache.ws),
                 lambda: wino.wino_rope_append(q, k, k, batch, wino.make_rope(None, rot_dim=0), cache.ws)):
        with pytest.raises(wino.WinoError) as e:
            call()
        assert e.value.status == wino.WINO_ERR_ARG
    with pytest.raises(wino.WinoError):
        loop.BlockCache(1, 2, 40, 8, 4, 2, 72, page_size=16, scaled=True)
