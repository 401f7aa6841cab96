"""wino_attend_scaled for few rows over values near the smallest that a cache holds: results are as exact relative to themselves as
any others (the tolerances of kv_helpers, with nothing added)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2605_16941_gb300 as wino  # noqa: E402
from cache8_helpers import BF, attend8, in_layout, make_kv8, quantise, rebatch, values_of  # noqa: E402
from kv_helpers import CAUSAL, add_rows, expected, f64  # noqa: E402


def set_cache(c, name, t):
    codes, scales = quantise(t, c.dtype)
    setattr(c, name + "_cache", values_of(codes, scales, c.dtype))
    c.extra[name + "8"], c.extra[name + "_scale"] = in_layout(codes.view(torch.uint8), "slots").view(torch.float8_e4m3fn), scales
    return rebatch(c)


def check_relative(c):
    ws = attend8(c)
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    got = f64(c.out)
    for s, i, want, tol in expected(c):
        d = np.abs(got[c.starts[s] + i] - want)
        assert (d <= tol).all(), f"sequence {s} row {i}: off by {(d / np.abs(want).max()).max()} of the largest"


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("exponent", [-112, -108, -104, -96, -80])
@pytest.mark.parametrize("seqs", [[(1, 900, 899), (1, 33, 32)], [(1, 30000, 29999), (1, 5, 4)]], ids=["short", "long"])
def test_small_values(seqs, exponent, dim):
    """Codes of 2^-9 2^-110 upwards; sums over few and over many slots."""
    c = make_kv8(CAUSAL, seqs, heads=4, kv_heads=2, dim=dim, poison=False, page=64)
    set_cache(c, "v", torch.ldexp(c.v_cache.double(), torch.tensor(exponent)))
    check_relative(add_rows(c, spread=0.1))


@pytest.mark.parametrize("behind", [0.5, 2.0, 4.0, 9.0])
def test_small_values_beside_slots_that_nobody_wrote(behind):
    """Such slots of a zeroed cache read as zeros, and their scores of 0 may be the largest."""
    c = make_kv8(CAUSAL, [(1, 60, 59)], heads=4, kv_heads=2, dim=128, poison=False)
    g = torch.Generator(device="cuda").manual_seed(3)
    set_cache(c, "k", torch.full_like(c.k_cache, -1.0).double())
    set_cache(c, "v", torch.ldexp(1.0 + torch.rand(c.v_cache.shape, generator=g, device="cuda").double(), torch.tensor(-102)))
    for j in range(0, 60, 3):
        page, at = c.table[0, j // c.page], j % c.page
        for x in "kv":
            getattr(c, x + "_cache")[page, at] = 0.0
            c.extra[x + "8"].view(torch.uint8)[page, at] = 0
            c.extra[x + "_scale"][page, :, at] = 0
    add_rows(c)
    c.q.fill_(behind * np.log(2.0) / 128 ** 0.5)  # scores of -behind in powers of two
    check_relative(c)
