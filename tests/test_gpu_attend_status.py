"""What wino_read_device_status says of a workspace's paged-cache calls: the first error since it was last read, once, whatever ran
behind it."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2605_16941_gb300 as wino  # noqa: E402
from kv_helpers import CAUSAL, add_rows, attend, check, make_kv  # noqa: E402
from paper_2605_16941_gb300 import loop  # noqa: E402

OK, ARG, TIMEOUT = wino.WINO_OK, wino.WINO_ERR_ARG, wino.WINO_ERR_DEVICE_TIMEOUT


def small():
    return add_rows(make_kv(CAUSAL, [(4, 60, 50), (2, 40, 30)], heads=4, kv_heads=2, poison=False))


def bad_table(c):
    t = c.table_dev.clone()
    c.table_dev[0, 2] = c.k_cache.size(0)
    return t


def test_an_earlier_failure_is_not_overwritten():
    """Two attends, of which only the first fails."""
    c = small()
    ws = wino.attend_workspace(c.batch)
    keep = bad_table(c)
    wino.wino_attend(c.q, c.out, c.batch, ws)
    c.table_dev.copy_(keep)
    for _ in range(3):
        wino.wino_attend(c.q, c.out, c.batch, ws)
    assert wino.wino_read_device_status(ws) == ARG
    assert wino.wino_read_device_status(ws) == OK  # once
    attend(c, ws=ws)
    assert wino.wino_read_device_status(ws) == OK
    check(c)


def test_the_first_of_several_failures_is_reported():
    c = small()
    ws = wino.attend_workspace(c.batch)
    ws.view(torch.int32)[0] = TIMEOUT  # as a CTA would record it
    wino.wino_attend(c.q, c.out, c.batch, ws)
    keep = bad_table(c)
    wino.wino_attend(c.q, c.out, c.batch, ws)
    c.table_dev.copy_(keep)
    assert wino.wino_read_device_status(ws) == TIMEOUT
    assert wino.wino_read_device_status(ws) == OK


def test_a_layer_of_a_step_that_fails_is_seen_behind_it():
    """Three layers over one BlockCache; the table is wrong during the first one's attention only."""
    cache = loop.BlockCache(3, 2, 48, 8, 4, 2, 64, page_size=16)
    rope = wino.make_rope(None, rot_dim=0)
    qkv = torch.randn((32, 8, 64)).to(torch.bfloat16).cuda()
    out = torch.empty((32, 4, 64), dtype=torch.bfloat16, device="cuda")
    for bad in (True, False):
        for i, b in enumerate(cache.step(32)):
            cache.append(*qkv.split([4, 2, 2], 1), b, rope)
            if bad and i == 0:
                cache.page_table[1, 0] = -1
            cache.attend(qkv[:, :4], out, b)
            if bad and i == 0:
                cache.page_table[1, 0] = cache.page_table[1, 1] - 1
        assert wino.wino_read_device_status(cache.ws) == (ARG if bad else OK)


def test_status_on_another_stream():
    """Read and cleared on the stream that it is asked for."""
    c = small()
    ws = wino.attend_workspace(c.batch)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    keep = bad_table(c)
    torch.cuda.synchronize()
    wino.wino_attend(c.q, c.out, c.batch, ws, stream=s)
    assert wino.wino_read_device_status(ws, stream=s) == ARG
    c.table_dev.copy_(keep)
    torch.cuda.synchronize()
    wino.wino_attend(c.q, c.out, c.batch, ws, stream=s)
    assert wino.wino_read_device_status(ws, stream=s) == OK
