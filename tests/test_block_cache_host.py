"""BlockCache's batches without a GPU: rows, slots and what the rows see, and what is refused."""
import pytest
import torch

import paper_2605_16941_gb300 as wino
from paper_2605_16941_gb300 import loop

N_SEQ, SEQ, L = 3, 50, 8


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2605_16941_gb300 import build
    build.build()


def cache(**kw):
    return loop.BlockCache(2, N_SEQ, SEQ, L, 4, 2, 64, page_size=16, device="cpu", **kw)


def described(batches):
    assert len(batches) == 2
    for b in batches:
        q_start, q_len, kv_len, new_slot = (t.tolist() for t in b.tensors[3:])
        assert q_start == [s * q_len[0] for s in range(N_SEQ)] and b.n_rows == N_SEQ * q_len[0]
        assert all(len(set(x)) == 1 for x in (q_len, kv_len, new_slot))
    return q_len[0], kv_len[0], new_slot[0], b.mask


def test_what_the_rows_see():
    c, full, shadow = cache(), wino.WINO_MASK_FULL, wino.WINO_MASK_SHADOW
    assert described(c.context(0, 20)) == (20, 20, 0, full)
    assert described(c.context(5, 20, seen=SEQ)) == (15, SEQ, 5, full)
    assert described(c.step(20)) == (2 * L, 28, 20, shadow)
    assert described(c.step(20, seen=28)) == (2 * L, 28, 20, shadow)
    assert described(c.step(20, seen=SEQ)) == (2 * L, SEQ, 20, shadow)
    assert described(cache(no_shadow=True).step(20, seen=40)) == (L, 40, 20, full)
    # the shadow block has its slots behind everything
    assert c.page_table.size(1) * 16 >= SEQ + L


@pytest.mark.parametrize("seen", [-1, 0, 19, SEQ + 1])
def test_seen_outside_is_refused(seen):
    c = cache()
    with pytest.raises(ValueError):
        c.context(0, 20, seen=seen)
    with pytest.raises(ValueError):
        c.step(12, seen=seen)
