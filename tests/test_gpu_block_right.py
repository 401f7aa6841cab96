"""BlockCache with the right context in view: rows that see [Y_left, Y_cur, Y_right, Y_shad]."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2605_16941_gb300 as wino  # noqa: E402
from kv_helpers import FULL, SHADOW, Kv, check, f64  # noqa: E402
from paper_2605_16941_gb300 import loop  # noqa: E402

BF = torch.bfloat16
N_SEQ, SEQ, L, HEADS, KV_HEADS, DIM, START = 3, 90, 8, 4, 2, 64, 40


def rows(n, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((N_SEQ * n, HEADS + 2 * KV_HEADS, DIM), generator=g).to(BF).cuda().split([HEADS, KV_HEADS, KV_HEADS], 1)


def attended(cache, i, batch, q, mask, n, seen, new):
    """One layer's attention of a batch, checked against its definition over the cache."""
    out = torch.full((N_SEQ * n, HEADS, DIM), 77.0, dtype=BF, device="cuda")
    cache.attend(q, out, batch)
    assert wino.wino_read_device_status(cache.ws) == wino.WINO_OK
    c = Kv(mask, [(n, seen, new)] * N_SEQ, HEADS, KV_HEADS, DIM, cache.k.size(3), BF, [s * n for s in range(N_SEQ)], N_SEQ * n,
           cache.page_table.cpu().numpy(), cache.k[i].transpose(1, 2), cache.v[i].transpose(1, 2), None, None, batch, q, out,
           dict(whole=out))
    check(c)
    return out


@pytest.mark.parametrize("no_shadow", [False, True], ids=["shadow", "no_shadow"])
@pytest.mark.parametrize("page_size", [16, 64])
def test_step_sees_the_right_context(page_size, no_shadow):
    cache = loop.BlockCache(2, N_SEQ, SEQ, L, HEADS, KV_HEADS, DIM, page_size=page_size, no_shadow=no_shadow)
    rope = wino.make_rope(None, rot_dim=0)
    for i, b in enumerate(cache.context(0, SEQ)):
        cache.append(*rows(SEQ, i), b, rope)
    n = L if no_shadow else 2 * L
    for i, b in enumerate(cache.step(START, seen=SEQ)):
        keep = cache.k[i].clone()
        q, k, v = rows(n, 10 + i)
        cache.append(q, k, v, b, rope)
        out = attended(cache, i, b, q, FULL if no_shadow else SHADOW, n, SEQ, START)
        # the right side is where it was: the shadow block is stored behind everything
        now, was = (t.transpose(1, 2)[cache.page_table.long()].flatten(1, 2) for t in (cache.k[i], keep))
        assert torch.equal(now[:, START + L:SEQ], was[:, START + L:SEQ]) and torch.equal(now[:, :START], was[:, :START])
        # and seen: other values there change every row
        at = SEQ - 1
        page = cache.page_table[:, at // page_size].long()
        cache.v[i].transpose(1, 2)[page, at % page_size] += 64.0
        other = torch.empty_like(out)
        cache.attend(q, other, b)
        assert ((other.float() - out.float()).abs().amax(-1) > 0).all()


def test_one_pass_over_everything():
    """Every layer stores the rows left of the block, right of it and the step's, then all of them attend."""
    cache = loop.BlockCache(2, N_SEQ, SEQ, L, HEADS, KV_HEADS, DIM, page_size=32)
    rope = wino.make_rope(None, rot_dim=0)
    parts = [(cache.context(0, START, seen=SEQ), FULL, START, 0), (cache.context(START + L, SEQ, seen=SEQ), FULL, SEQ - START - L, START + L),
             (cache.step(START, seen=SEQ), SHADOW, 2 * L, START)]
    for i in range(2):
        xs = [rows(n, 20 + 10 * i + j) for j, (_, _, n, _) in enumerate(parts)]
        for (batches, *_), x in zip(parts, xs):
            cache.append(*x, batches[i], rope)
        for (batches, mask, n, new), x in zip(parts, xs):
            attended(cache, i, batches[i], x[0], mask, n, SEQ, new)


def test_stored_slots():
    """The shadow block's keys lie in the slots from `seen` on."""
    cache = loop.BlockCache(1, N_SEQ, SEQ, L, HEADS, KV_HEADS, DIM, page_size=16)
    _, k, v = rows(2 * L, 5)
    for seen in (START + L, 70, SEQ):
        cache.k.zero_()
        wino.wino_rope_append(None, k, v, cache.step(START, seen=seen)[0], wino.make_rope(None, rot_dim=0), cache.ws)
        held = f64(cache.k[0].transpose(1, 2))[cache.page_table.cpu().numpy()].reshape(N_SEQ, -1, KV_HEADS, DIM)
        want = np.zeros_like(held)
        x = f64(k).reshape(N_SEQ, 2, L, KV_HEADS, DIM)
        want[:, START:START + L], want[:, seen:seen + L] = x[:, 0], x[:, 1]
        assert np.array_equal(held, want)
