"""Errors of wino_rope_append: reported once by wino_read_device_status, also on a workspace that no wino_attend ever uses, and by the
next wino_attend, whose cache lacks the rows."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2605_16941_gb300 as wino  # noqa: E402
from kv_helpers import CAUSAL, make_kv  # noqa: E402

OK, ARG = wino.WINO_OK, wino.WINO_ERR_ARG


class Calls:
    def __init__(self, ws_of):
        self.c = c = make_kv(CAUSAL, [(4, 40, 36), (4, 40, 36)], poison=False)
        self.ws = ws_of(c.batch)
        self.k = torch.randn((c.n_rows, 1, 64)).to(torch.bfloat16).cuda()
        self.q = torch.randn((c.n_rows, 2, 64)).to(torch.bfloat16).cuda()
        self.rope = wino.make_rope(None, rot_dim=0)

    def append(self, good):
        c = self.c
        c.ints[3, 1] = 36 if good else c.table.shape[1] * c.page - 2  # rows past the table
        wino.wino_rope_append(None, self.k, self.k, c.batch, self.rope, self.ws)
        c.ints[3, 1] = 36

    def attend(self):
        wino.wino_attend(self.q, torch.empty_like(self.q), self.c.batch, self.ws)

    def status(self):
        return wino.wino_read_device_status(self.ws)


def test_workspace_of_appends_alone():
    x = Calls(lambda b: wino.append_workspace())
    x.append(True)
    assert x.status() == OK
    for _ in range(2):
        x.append(False)
        x.append(True)
        assert x.status() == ARG
        assert x.status() == OK
        x.append(True)
        assert x.status() == OK


def test_the_next_attend_reports_it_too():
    x = Calls(wino.attend_workspace)
    x.append(False)
    assert x.status() == ARG and x.status() == OK
    x.append(True)
    assert x.status() == OK
    x.attend()
    assert x.status() == ARG and x.status() == OK
    x.attend()
    assert x.status() == OK


def test_a_second_error_after_the_first_was_read():
    x = Calls(wino.attend_workspace)
    x.append(False)
    assert x.status() == ARG
    x.append(False)
    assert x.status() == ARG and x.status() == OK
    x.append(False)
    x.attend()
    assert x.status() == ARG and x.status() == OK


def test_an_append_behind_a_failed_attend():
    """The attend's error is read once; a correct append behind it is OK."""
    x = Calls(wino.attend_workspace)
    keep = x.c.table_dev.clone()
    x.c.table_dev[0, 0] = -1
    x.attend()
    x.c.table_dev.copy_(keep)
    assert x.status() == ARG
    x.append(True)
    assert x.status() == OK
