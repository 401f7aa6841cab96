"""Norms of heads whose elements lie many orders of magnitude apart: each result is exact relative to itself.

The tolerance is test_gpu_norm_rope.py's for the norm (2^-17 of the result) and half a step of bf16."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2605_16941_gb300 as wino  # noqa: E402
from cache8_helpers import BF, normed  # noqa: E402
from kv_helpers import CAUSAL, f64, half_step, make_kv  # noqa: E402


@pytest.mark.parametrize("per_head", [False, True], ids=["shared", "per_head"])
@pytest.mark.parametrize("largest", [30, 49, 50, 51, 60, 100, 127])
@pytest.mark.parametrize("dim", [128, 80, 72, 16])
def test_small_elements_beside_a_large_one(dim, largest, per_head):
    """Down to results of 2^-125: fp32 holds them all."""
    c = make_kv(CAUSAL, [(40, 40, 0)], heads=3, kv_heads=1, dim=dim, poison=False)
    g = torch.Generator().manual_seed(largest)
    size = torch.rand((c.n_rows, 3, dim), generator=g).double() * 110 + largest - 112
    q = torch.exp2(size.clamp(min=-125.0)) * (torch.rand(size.shape, generator=g) < 0.5).double().mul(2).sub(1)
    q[:, 0, 3] = 1.5 * 2.0 ** largest
    q[:, 1, dim - 1] = -1.25 * 2.0 ** largest
    q[:, 2] = torch.randn((c.n_rows, dim), generator=g)  # beside heads that need no care
    q = q.to(BF).cuda()
    weight = (1.0 + torch.rand((3, dim) if per_head else (dim,), generator=g)).to(BF).cuda()
    out, ws = torch.zeros_like(q), wino.append_workspace()
    wino.wino_norm_rope_append(q, None, None, c.batch, wino.make_rope(None, rot_dim=0), ws,
                               norm=wino.make_head_norm(weight, None), q_out=out)
    assert wino.wino_read_device_status(ws) == wino.WINO_OK
    want, got = normed(f64(q), weight, 1e-6, 0.0), f64(out)
    live = np.abs(want) >= 2.0 ** -125  # below lie subnormal numbers
    off = np.abs(got - want)
    assert (off <= (2.0 ** -17 + 1.001 * half_step(BF)) * np.abs(want))[live].all(), f"{(off / np.abs(want))[live].max()}"
    assert (off[~live] <= 2.0 ** -125).all()
