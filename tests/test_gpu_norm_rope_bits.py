"""wino_norm_rope_append without norms, axes and an 8-bit cache gives wino_rope_append's results bit for bit, NaNs and subnormal
numbers among them."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2605_16941_gb300 as wino  # noqa: E402
from cache8_helpers import BF, FP  # noqa: E402
from kv_helpers import CAUSAL, frequencies, make_kv  # noqa: E402


def any_bits(shape, g):
    """Every pattern of 16 bits, NaNs of many kinds in one element of nine."""
    bits = torch.randint(-32768, 32768, shape, generator=g, dtype=torch.int32)
    nans = torch.randint(0x7f81, 0x8000, shape, generator=g, dtype=torch.int32) - (torch.rand(shape, generator=g) < 0.5).int() * 32768
    return torch.where(torch.rand(shape, generator=g) < 0.11, nans, bits).to(torch.int16)


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "neighbours"])
@pytest.mark.parametrize("dim,rot", [(128, 0), (128, 128), (128, 64), (128, 58), (80, 0), (80, 40), (72, 72), (72, 8), (72, 6), (64, 16),
                                     (24, 24), (24, 10), (8, 0)])
def test_bit_for_bit_without_norms_axes_and_scales(dim, rot, interleaved, dtype):
    seqs = [(33, 40, 7), (1, 12, 11), (70, 70, 0)]
    c = make_kv(CAUSAL, seqs, heads=6, kv_heads=2, dim=dim, dtype=dtype, gap=1, poison=False)
    rope = wino.make_rope(torch.from_numpy(frequencies(rot)).cuda() if rot else None, rot_dim=rot, interleaved=interleaved)
    got = []
    for call in (wino.wino_rope_append, wino.wino_norm_rope_append):
        g = torch.Generator().manual_seed(11)
        q, k, v = any_bits((c.n_rows, 10, dim), g).cuda().view(dtype).split([6, 2, 2], 1)
        c.k_cache.fill_(3.0)
        c.v_cache.fill_(4.0)
        out = torch.full((c.n_rows, 6, dim), 7.0, dtype=dtype, device="cuda")
        ws = wino.append_workspace()
        call(q, k, v, c.batch, rope, ws, q_out=out)
        assert wino.wino_read_device_status(ws) == wino.WINO_OK
        got.append([t.view(torch.int16).clone() for t in (out, c.k_cache, c.v_cache)])
    for name, a, b in zip(("q", "K", "V"), *got):
        assert torch.equal(a, b), f"{name}: {(a != b).sum().item()} elements differ"


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "neighbours"])
@pytest.mark.parametrize("dim,rot", [(128, 128), (128, 58), (80, 40), (24, 10)])
def test_many_rows_without_norms(dim, rot, interleaved, dtype):
    """Ordinary values, so many that another order of rounding would show; a norm without weights is none."""
    n = 6000
    c = make_kv(CAUSAL, [(n, n, 0)], heads=6, kv_heads=2, dim=dim, dtype=dtype, page=64, poison=False)
    rope = wino.make_rope(torch.from_numpy(frequencies(rot)).cuda(), rot_dim=rot, interleaved=interleaved)
    g = torch.Generator().manual_seed(13)
    q, k, v = torch.randn((c.n_rows, 10, dim), generator=g).to(dtype).cuda().split([6, 2, 2], 1)
    got = []
    for call, more in ((wino.wino_rope_append, {}), (wino.wino_norm_rope_append, {}),
                       (wino.wino_norm_rope_append, dict(norm=wino.make_head_norm(None, None)))):
        c.k_cache.fill_(3.0)
        c.v_cache.fill_(4.0)
        out, ws = torch.zeros((c.n_rows, 6, dim), dtype=dtype, device="cuda"), wino.append_workspace()
        call(q, k, v, c.batch, rope, ws, q_out=out, **more)
        assert wino.wino_read_device_status(ws) == wino.WINO_OK
        got.append([t.clone() for t in (out, c.k_cache, c.v_cache)])
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("dim,rot", [(128, 128), (128, 64), (80, 40), (72, 6)])
def test_values_keep_their_bits_beside_norms(dim, rot, dtype):
    """V as it came; the unturned dims of heads that are not normalised too, but for which NaN a NaN is."""
    c = make_kv(CAUSAL, [(33, 40, 7)], heads=4, kv_heads=2, dim=dim, dtype=dtype, poison=False)
    g = torch.Generator().manual_seed(12)
    q, k, v = any_bits((c.n_rows, 8, dim), g).cuda().view(dtype).split([4, 2, 2], 1)
    rope = wino.make_rope(torch.from_numpy(frequencies(rot)).cuda(), rot_dim=rot)
    weight = torch.ones(dim, dtype=dtype, device="cuda")

    def same(a, b):
        return ((a.view(torch.int16) == b.view(torch.int16)) | (torch.isnan(a) & torch.isnan(b))).all()
    for norm in (wino.make_head_norm(weight, None), wino.make_head_norm(None, weight)):
        out, ws = torch.zeros((c.n_rows, 4, dim), dtype=dtype, device="cuda"), wino.append_workspace()
        wino.wino_norm_rope_append(q, k, v, c.batch, rope, ws, norm=norm, q_out=out)
        assert wino.wino_read_device_status(ws) == wino.WINO_OK
        slots = torch.arange(7, 40)
        at = torch.from_numpy(c.table[0])[slots // c.page].long().cuda(), (slots % c.page).cuda()
        assert torch.equal(c.v_cache[at].view(torch.int16), v.view(torch.int16))
        if norm.q_shape is None:
            assert same(out[..., rot:], q[..., rot:])
        else:
            assert same(c.k_cache[at][..., rot:], k[..., rot:])
