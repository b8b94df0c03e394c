"""residual_norm_bwd without a gradient from further on: bit for bit what it gives for one of zeros, whatever the call before it has left in
shared memory."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def mx():
    import paper_2502_20853_b200 as m
    m.lib()
    return m


@pytest.mark.parametrize("cols", [32, 96, 160, 384, 768, 1024, 1056, 2048, 2080, 4128, 8192])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("gates", [0, 1, 7])
def test_as_with_zeros(mx, cols, dtype, gates):
    rows = 7 * max(1, 40000 // cols)
    g = torch.Generator(device="cuda").manual_seed(cols + gates)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    for post, bias, save in ((None, False, mx.SAVE_8BIT), (None, True, mx.SAVE_INPUTS), (mx.NORM_RMS, False, mx.SAVE_8BIT), (mx.NORM_LAYER, True, mx.SAVE_8BIT)):
        side = lambda kind: mx.Norm(kind, 1 + 0.3 * rnd(cols), 0.2 * rnd(cols) if bias else None)  # noqa: E731
        _, _, ctx = mx.residual_norm_fwd(rnd(rows, cols).to(dtype), rnd(rows, cols).to(BF16), pre=side(mx.NORM_LAYER), post=side(post) if post is not None else None,
                                         gate=rnd(gates, cols) if gates else None, save=save)
        dh, zeros = rnd(rows, cols).to(BF16), torch.zeros(rows, cols, dtype=dtype, device="cuda")
        want = mx.residual_norm_bwd(dh, zeros, ctx)
        stale = torch.full((rows, cols), float("nan"), dtype=dtype, device="cuda")
        for _ in range(3):
            mx.residual_norm_bwd(dh, stale, ctx)
            got = mx.residual_norm_bwd(dh, None, ctx, dx=torch.empty(rows, cols, dtype=dtype, device="cuda"))
            for name, a, b in zip(want._fields, got, want):
                assert (a is None and b is None) or torch.equal(a, b), name
