"""Calls of residual_norm_fwd / _bwd that the documentation allows, at the edges: without rows, with rows that are not finite, with tiny deviations."""
import pytest
import torch

import norm_reference as R

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def mx():
    import paper_2502_20853_b200 as m
    m.lib()
    return m


@pytest.mark.parametrize("save", ["SAVE_8BIT", "SAVE_INPUTS"])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_no_rows(mx, save, dtype):
    x, f = torch.empty(0, 96, dtype=dtype, device="cuda"), torch.empty(0, 96, dtype=BF16, device="cuda")
    norm = mx.Norm(mx.NORM_LAYER, torch.ones(96, device="cuda"), torch.zeros(96, device="cuda"))
    x_out, h, ctx = mx.residual_norm_fwd(x, f, pre=norm, post=norm, gate=torch.ones(2, 96, device="cuda"), save=getattr(mx, save))
    g = mx.residual_norm_bwd(h, x_out, ctx)
    assert x_out.shape == h.shape == g.dx.shape == g.df.shape == (0, 96) and g.gate.shape == (2, 96)
    for t in (g.pre_weight, g.pre_bias, g.post_weight, g.post_bias, g.gate):
        assert bool((t == 0).all())
    assert mx.residual_norm_fwd(x, f, pre=norm, post=norm, save=mx.SAVE_NOTHING)[2] is None


@pytest.mark.parametrize("eps", [0.0, 1e-30])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_tiny_groups_of_tiny_rows(mx, dtype, eps):
    """Rows whose deviation is 2^-45 with groups down to the smallest normal number, and eps below both: 2^-s and 1 / deviation are finite, their
    product is not."""
    g = torch.Generator(device="cuda").manual_seed(4)
    v = torch.randn(16, 128, device="cuda", generator=g, dtype=torch.float64) * 2.0 ** -45
    for row in range(16):
        v[row, 96:] *= 2.0 ** -(8 * row // 2 + 20)       # 2^-65 to 2^-125 and what is below it
    v = v.to(dtype)
    norm = mx.Norm(mx.NORM_RMS, eps=eps)
    x0 = torch.zeros_like(v)
    ref = v.double()
    want = ref / torch.sqrt(ref.square().mean(1, keepdim=True) + eps)
    # of the branch (f, bf16) and of the residual
    _, _, ctx = mx.residual_norm_fwd(x0, v.to(BF16), post=norm) if dtype == BF16 else mx.residual_norm_fwd(v, pre=norm)
    c = ctx.f if dtype == BF16 else ctx.x
    power = torch.ldexp(torch.ones_like(c.scales, dtype=torch.float64), c.scales.to(torch.int32) - 127).repeat_interleave(32, 1)
    # half a step of the code, half the smallest step of the group, and a few roundings in FP32 (2^-18 holds a row's sums)
    far = (R.load(c.codes, c.scales) - want).abs() - (want.abs() * (2.0 ** -4 + 2.0 ** -18) + power * 2.0 ** -10)
    assert bool((far <= 0).all()), far.amax(1)
    m = want.abs().reshape(16, -1, 32).amax(2)
    assert bool((torch.ldexp(m, -(c.scales.to(torch.int32) - 127)) > 223).all())      # the scale is the group's
