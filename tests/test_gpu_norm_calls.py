"""Calls of residual_norm_fwd / _bwd that the documentation allows, at the edges: without rows, with rows that are not finite, with tiny deviations."""
import pytest
import torch

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
