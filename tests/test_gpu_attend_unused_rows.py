"""What a call leaves in shared memory does not reach the next one's results: rows of a tile that no head uses (two of 128 with
7 heads to a kv head) hold whatever was there before."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2605_16941_gb300 as wino  # noqa: E402
from cache8_helpers import attend8, make_kv8  # noqa: E402
from kv_helpers import CAUSAL, FULL, add_rows, attend, make_kv  # noqa: E402


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("scaled", [False, True], ids=["plain", "e4m3"])
def test_unused_rows_do_not_count(scaled, dim):
    make, call = (make_kv8, attend8) if scaled else (make_kv, attend)
    c = add_rows(make(CAUSAL, [(200, 3000, 2800)] * 6, heads=14, kv_heads=2, dim=dim, poison=False))
    ws = wino.attend_workspace(c.batch)
    before = add_rows(make(FULL, [(304, 128, 0)], heads=128, kv_heads=1, dim=dim, poison=False))
    other = wino.attend_workspace(before.batch)
    results = []
    for size in (0.0, 3e4, 1.0, 3e4):
        before.q.fill_(size)  # every row of every Q tile
        call(before, ws=other)
        call(c, ws=ws)
        results.append(c.out.clone())
    assert all(torch.equal(r, results[0]) for r in results[1:])
