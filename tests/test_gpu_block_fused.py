"""The transformer block with its norms, residual additions and activation through the library (8-bit checkpoints, the quantized input of a
linear layer written by the norm before it): every call of one training step against the 64-bit reference, every linear layer
replayed through the oracle, and the whole against the block with PyTorch's operators."""
import numpy as np
import pytest
import torch

import norm_reference as R
from test_gpu_block import f32, replay_layer
from util import qmat_to_numpy

pytestmark = pytest.mark.gpu
K = 2.0 ** -18       # FP32 errors of a norm, relative to sums over magnitudes (see test_gpu_residual_norm)


@pytest.fixture(scope="module")
def mx():
    import paper_2502_20853_b200 as m
    m.lib()
    return m


def _close(got, want, mags, what):
    far = (got.double() - want).abs() - (want.abs() * 2.0 ** -8 * 1.001 + 8 * K * mags + 1e-37)
    assert bool((far <= 0).all()), "%s: %d outside" % (what, int((far > 0).sum()))


def _before(block):
    out = {}
    for name, layer in block.layers.items():
        p, s = qmat_to_numpy(layer.osc.wq_prev)
        out[name] = dict(ema=layer.ema.cpu().numpy().copy(), w_prev=f32(layer.osc.w_prev), p_prev=p, s_prev=s, dist_w=layer.osc.dist_w.cpu().numpy().copy(),
                         dist_q=layer.osc.dist_q.cpu().numpy().copy())
    return out


def _check_norm(r, ln):
    pre = ("layer", ln.weight.detach(), ln.bias.detach()) if ln is not None else None
    o = R.norm_fwd(r["x"], r["f"], pre, None, None, 1.0, 1.0, ln.eps if ln is not None else 0.0)
    x = o["x_out"]
    if r["x_out"] is not None:
        _close(r["x_out"], x, r["x"].double().abs() + r["f"].double().abs(), "x_out")
    g = r["grads"]
    xh = None
    if ln is not None:
        rstd = o["pre"][1]
        size = o["xh"].abs() + (x.abs() + x.abs().mean(1, keepdim=True)) * rstd
        size = size + rstd * ((r["x"].double().abs() + (r["f"].double().abs() if r["f"] is not None else 0.0)) + o["xh"].abs() * x.abs().mean(1, keepdim=True))
        _close(r["h"], o["h"], size, "h")
        c = r["ctx"].x
        xh = R.load(c.codes, c.scales)
        power = torch.ldexp(torch.ones_like(c.scales, dtype=torch.float64), c.scales.to(torch.int32) - 127).repeat_interleave(32, 1)
        assert bool(((xh - o["xh"]).abs() <= o["xh"].abs() * 2.0 ** -4 + power * 2.0 ** -10 + 2 * K * size).all())
    st = r["ctx"].stats
    want = R.norm_bwd(r["dh"], r["dx_out"], xh, None, st[1].double()[:, None] if st is not None else None, None, pre, None, None, 1.0, 1.0)
    _close(g.dx, want["dx"], want["abs_dx"], "dx")
    if g.df is not None:
        _close(g.df, want["df"], want["abs_df"], "df")
    if ln is not None:
        n = (xh.shape[0] + 80) * 2.0 ** -24
        assert bool(((g.pre_weight.double() - want["pre_weight"]).abs() <= (n + 8 * K) * want["abs_pre_weight"]).all())
        assert bool(((g.pre_bias.double() - want["pre_bias"]).abs() <= (n + 8 * K) * want["abs_pre_bias"]).all())


def test_a_step_of_the_fused_block(mx):
    from workloads.block_harness import Block, make_block_inputs
    block, plain = Block(mx, fused=True), Block(mx)
    gen = torch.Generator(device="cuda").manual_seed(3)
    with torch.no_grad():
        for ln, other in ((block.ln1, plain.ln1), (block.ln2, plain.ln2)):
            ln.weight.add_(0.2 * torch.randn(ln.weight.shape, device="cuda", generator=gen))
            ln.bias.add_(0.1 * torch.randn(ln.bias.shape, device="cuda", generator=gen))
            other.weight.copy_(ln.weight), other.bias.copy_(ln.bias)
    x, dout = make_block_inputs(32)
    before = _before(block)
    out, dx = block.step(x, dout)
    torch.cuda.synchronize()
    assert int(block.status.item()) == 0 and all(int(layer.status.item()) == 0 for layer in block.layers.values())
    for name, layer in block.layers.items():
        replay_layer(layer, before[name], full=False)
    rec = block.records
    _check_norm(rec["norm1"], block.ln1)
    _check_norm(rec["norm2"], block.ln2)
    _check_norm(rec["end"], None)
    g = rec["gelu"]
    y = g["y"].double()
    assert bool(((g["z"].double() - R.act(y, "gelu")).abs() <= 2.0 ** -8 * R.act(y, "gelu").abs() + 2.0 ** -21 * y.abs()).all())
    yr = R.load(g["ckpt"].codes, g["ckpt"].scales)
    want = R.act_bwd(g["dz"].double(), yr, "gelu")
    assert bool(((g["dy"].double() - want).abs() <= 2.0 ** -8 * want.abs() + g["dz"].double().abs() * 2.0 ** -19 + 1e-37).all())
    # what one operator gives is what the next one takes
    assert torch.equal(out.reshape(-1, 384), rec["end"]["x_out"]) and torch.equal(dx.reshape(-1, 384), rec["norm1"]["grads"].dx)
    assert torch.equal(block.layers["qkv"].record["x"], rec["norm1"]["h"]) and torch.equal(block.layers["fc2"].record["x"], g["z"])
    assert torch.equal(rec["norm2"]["x_out"], rec["end"]["x"]) and torch.equal(rec["gelu"]["dy"], block.layers["fc1"].record["dy"])
    # and the whole beside PyTorch's norms and GELU: they round elsewhere, which the FP4 operands make a matter of whole codes, so only the
    # direction is compared
    out2, dx2 = plain.step(x, dout)
    cos = lambda a, b: float(torch.nn.functional.cosine_similarity(a.double().flatten(), b.double().flatten(), 0))  # noqa: E731
    assert cos(out, out2) > 0.999 and cos(dx, dx2) > 0.99
    assert np.isfinite(cos(out, out2))
