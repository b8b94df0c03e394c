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


@pytest.mark.parametrize("kind", ["NORM_LAYER", "NORM_RMS"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan"), 1e25])
@pytest.mark.parametrize("where", ["x", "f"])
def test_rows_without_a_deviation_in_fp32(mx, kind, dtype, value, where):
    """NaN throughout and flagged, of an RMS norm too: not zeros, which the infinite deviation would give."""
    rows, cols, row = 40, 160, 11
    g = torch.Generator(device="cuda").manual_seed(7)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    x, f = rnd(rows, cols).to(dtype), rnd(rows, cols).to(BF16)
    (x if where == "x" else f)[row, 70] = value
    norm = mx.Norm(getattr(mx, kind), 1 + 0.2 * rnd(cols), 0.1 * rnd(cols))
    rest = torch.arange(rows, device="cuda") != row
    st, hq = mx.new_status(), mx.QMat(rows, cols)
    x_out, h, ctx = mx.residual_norm_fwd(x, f, pre=norm, post=norm, hq=hq, dev_status=st)
    assert int(st.item()) == mx.DEV_NONFINITE
    assert bool(torch.isnan(h[row]).all()) and bool(torch.isfinite(h[rest]).all())
    assert bool((ctx.x.scales[row] == 255).all()) and bool((ctx.x.codes[row] == 0).all()) and bool((ctx.x.scales[rest] != 255).all())
    assert bool(torch.isnan(ctx.stats[1, row])) and bool(torch.isfinite(ctx.stats[:, rest]).all())
    if where == "f":
        assert bool(torch.isnan(x_out[row]).all()) and bool(torch.isnan(ctx.stats[3, row])) and bool((ctx.f.scales[row] == 255).all())
    else:                               # x' itself is what the sum says
        only = torch.arange(cols, device="cuda") != 70
        assert bool(torch.isfinite(x_out[row, only]).all()) and bool(torch.isfinite(ctx.stats[2:, row]).all()) and bool((ctx.f.scales[row] != 255).all())
        big = float(x_out[row, 70])
        assert big != big if value != value else big == float(x[row, 70])
    grads = mx.residual_norm_bwd(rnd(rows, cols).to(BF16), rnd(rows, cols).to(dtype), ctx)
    assert bool(torch.isnan(grads.dx[row]).all()) and bool(torch.isfinite(grads.dx[rest]).all())
    assert bool(torch.isnan(grads.df[row]).all()) and bool(torch.isfinite(grads.df[rest]).all())
