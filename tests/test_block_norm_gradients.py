"""The fused block's norms are trained: the gradients of LayerNorm's weight and bias arrive where the plain block leaves them.  On the CPU with the
64-bit reference in the library's place, and on the GPU beside the plain block."""
import types

import pytest
import torch

import norm_reference as R
from workloads import block_harness as H


def _library():
    """residual_norm_fwd / _bwd as far as the block calls them, by the reference."""
    m = types.SimpleNamespace(NORM_LAYER=1, QMat=lambda *a: None)
    m.Norm = lambda kind, weight, bias, eps: types.SimpleNamespace(kind=kind, weight=weight, bias=bias, eps=eps)

    def fwd(x, f=None, pre=None, hq=None, dev_status=None):
        o = R.norm_fwd(x, f, ("layer", pre.weight, pre.bias) if pre is not None else None, None, None, 1.0, 1.0, pre.eps if pre is not None else 0.0)
        ctx = types.SimpleNamespace(pre=pre, xh=o.get("xh"), rstd=o["pre"][1] if pre is not None else None, f=f)
        return (o["x_out"].to(x.dtype) if f is not None else None), (o["h"].to(x.dtype) if pre is not None else None), ctx

    def bwd(dh, dx_out, ctx, df=None):
        pre = ("layer", ctx.pre.weight, ctx.pre.bias) if ctx.pre is not None else None
        o = R.norm_bwd(dh, dx_out, ctx.xh, None, ctx.rstd, None, pre, None, None, 1.0, 1.0)
        like = dx_out if dx_out is not None else dh
        return types.SimpleNamespace(dx=o["dx"].to(like.dtype), df=o["df"].to(like.dtype) if df is None else None,
                                     pre_weight=o["pre_weight"].float() if pre else None, pre_bias=o["pre_bias"].float() if pre else None)

    m.residual_norm_fwd, m.residual_norm_bwd = fwd, bwd
    return m


@pytest.mark.parametrize("branch", [False, True])
@pytest.mark.parametrize("dtype", [torch.float64, torch.bfloat16])
def test_gradients_arrive(branch, dtype):
    g = torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64).to(dtype)  # noqa: E731
    block = H.Block.__new__(H.Block)
    block.mx, block.records, block.status = _library(), {}, None
    ln, plain = (torch.nn.LayerNorm(H.D_MODEL, dtype=dtype) for _ in range(2))
    with torch.no_grad():
        ln.weight.add_(0.2 * rnd(H.D_MODEL)), ln.bias.add_(0.1 * rnd(H.D_MODEL))
        plain.weight.copy_(ln.weight), plain.bias.copy_(ln.bias)
    x, f, dx_out, dh = (rnd(3, 5, H.D_MODEL) for _ in range(4))
    leaves = []
    for which in (ln, plain):
        xs, fs = x.clone().requires_grad_(True), f.clone().requires_grad_(True)
        if which is ln:
            x_out, h, _ = block._norm("n", xs, fs if branch else None, ln)
        else:
            x_out = xs + fs if branch else xs
            h = plain(x_out)
        torch.autograd.backward([x_out, h], [dx_out, dh])
        leaves.append((which.weight.grad, which.bias.grad, xs.grad, fs.grad if branch else xs.grad))
    for got, want in zip(*leaves):
        assert got is not None and got.dtype == want.dtype
        # bf16: the plain form's sums over 15 rows are rounded on the way (x_out, h's parts) and at the end
        tol = 1e-4 if dtype == torch.float64 else 2.0 ** -4     # the reference's FP32 sums are cut to FP32 above: 2^-24 of them
        assert float((got.double() - want.double()).norm()) <= tol * float(want.double().norm())


def test_end_of_the_block_has_no_norm():
    block = H.Block.__new__(H.Block)
    block.mx, block.records, block.status = _library(), {}, None
    x, f = (torch.randn(2, 3, H.D_MODEL, dtype=torch.float64, requires_grad=True) for _ in range(2))
    out, h, hq = block._norm("end", x, f, None)
    d = torch.randn_like(out)
    out.backward(d)
    assert h is None and hq is None and torch.equal(x.grad, d) and torch.equal(f.grad, d)


@pytest.mark.gpu
def test_beside_the_plain_block():
    import paper_2502_20853_b200 as mx
    block, plain = H.Block(mx, fused=True), H.Block(mx)
    gen = torch.Generator(device="cuda").manual_seed(5)
    with torch.no_grad():
        for ln, other in ((block.ln1, plain.ln1), (block.ln2, plain.ln2)):
            ln.weight.add_(0.2 * torch.randn(ln.weight.shape, device="cuda", generator=gen))
            ln.bias.add_(0.1 * torch.randn(ln.bias.shape, device="cuda", generator=gen))
            other.weight.copy_(ln.weight), other.bias.copy_(ln.bias)
    x, dout = H.make_block_inputs(32)     # rows a multiple of 32, which the linear layers ask for
    block.step(x, dout), plain.step(x, dout)
    for name in ("ln1", "ln2"):
        for p in ("weight", "bias"):
            a, b = getattr(getattr(block, name), p).grad, getattr(getattr(plain, name), p).grad
            assert a is not None and a.dtype == b.dtype and a.shape == b.shape
            # the FP4 operands make roundings elsewhere a matter of whole codes: the direction, as for the block's outputs.  A cosine of 0.99 of dh is
            # noise of sqrt(0.02) of its size, E4M3 codes of x^ add at most 2^-4 / sqrt(3) of theirs: 1 - (0.02 + 0.0013) / 2 = 0.989 of the sums
            assert float(torch.nn.functional.cosine_similarity(a.double(), b.double(), 0)) > 0.98, (name, p)
    # twice the gradient after a second step, as autograd adds them up
    first = block.ln2.bias.grad.clone()
    block.forward(x).backward(dout)
    assert not torch.equal(first, block.ln2.bias.grad)
