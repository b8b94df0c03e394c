"""Matrices of more than 2^31 elements (offsets beyond 32 bits in every operand), wide and long ones: the rows at both ends as a call on them alone
gives them, bit for bit, and the gradients that are sums over rows against those sums."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def mx():
    import paper_2502_20853_b200 as m
    m.lib()
    return m


@pytest.mark.parametrize("rows,cols,several", [(270080, 8192, False), (70000128, 32, False), (2800128, 800, True)])
def test_more_elements_than_32_bits(mx, rows, cols, several):
    assert rows * cols > 1 << 31
    n = 128                                     # rows at each end
    gates = rows // n if several else 1
    g = torch.Generator(device="cuda").manual_seed(cols)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    ends = [slice(0, n), slice(rows - n, rows)]

    def matrix(scale=1.0):
        t = torch.zeros(rows, cols, dtype=BF16, device="cuda")
        for e in ends:
            t[e] = (scale * rnd(n, cols)).to(BF16)
        return t

    norm = lambda kind: mx.Norm(kind, 1 + 0.3 * rnd(cols), 0.2 * rnd(cols))  # noqa: E731
    pre, post, gate = norm(mx.NORM_RMS), norm(mx.NORM_LAYER), torch.ones(gates, cols, device="cuda")
    gate[0], gate[-1] = rnd(cols), rnd(cols)
    x, f = matrix(), matrix()
    hq = mx.QMat(rows, cols)
    x_out, h, ctx = mx.residual_norm_fwd(x, f, pre=pre, post=post, gate=gate, hq=hq)
    # with several gates the small call has two of the same: one alone is multiplied into the norm's factor and summand, f^ (g w) + (g b), several
    # into their result, (f^ w + b) g, which rounds in other places
    small = [mx.residual_norm_fwd(x[e], f[e], pre=pre, post=post, gate=gate[k].repeat(2 if several else 1, 1), hq=mx.QMat(n, cols)) for k, e in zip((0, -1), ends)]
    del x, f
    for (xs, hs, cs), e in zip(small, ends):
        assert torch.equal(x_out[e], xs) and torch.equal(h[e], hs) and torch.equal(ctx.stats[:, e], cs.stats)
        for a, b in ((ctx.x, cs.x), (ctx.f, cs.f)):
            assert torch.equal(a.codes[e], b.codes) and torch.equal(a.scales[e], b.scales)
    for e in ends:                              # rows - n is a multiple of 128: whole tiles of scales
        want = mx.quantize(h[e])
        assert torch.equal(hq.data[e], want.data)
        size, at = mx.scale_bytes(n, cols), mx.scale_bytes(e.start, cols) if e.start else 0
        assert torch.equal(hq.scales[at:at + size], want.scales[:size])
    del x_out, h, hq
    dh, dx_out = matrix(1e-2), matrix(1e-2)
    got = mx.residual_norm_bwd(dh, dx_out, ctx)
    parts = [mx.residual_norm_bwd(dh[e], dx_out[e], c[2]) for c, e in zip(small, ends)]
    for p, e in zip(parts, ends):
        assert torch.equal(got.dx[e], p.dx) and torch.equal(got.df[e], p.df)
    # dh and dx' are zeros between the ends: the sums are those of the two ends.  Both sides add terms of one set in another order: 2^-24 of the
    # largest sum on the way for each of at most 128 + 40 additions that are not of zeros
    for name in ("pre_weight", "pre_bias", "post_weight", "post_bias"):
        a, b, c = (getattr(t, name).double() for t in (got, *parts))
        size = sum(_magnitudes(mx, name, s[2], dh[e], p) for s, e, p in zip(small, ends, parts))
        assert bool(((a - b - c).abs() <= 3 * 168 * 2.0 ** -24 * size + 1e-30).all()), name
    if several:
        assert got.gate.shape == (gates, cols)
        for k, p, s in zip((0, -1), parts, small):
            assert bool(((got.gate[k].double() - p.gate.double().sum(0)).abs() <= 2 * 168 * 2.0 ** -24 * _gate_size(mx, s[2], p) + 1e-30).all())
        assert bool((got.gate[1:-1] == 0).all())


def _magnitudes(mx, name, ctx, dh, p):
    """The sum of magnitudes of one end's terms (t, the gradient of x_out in all, is dx: residual_scale is 1)."""
    if name == "pre_bias":
        return dh.double().abs().sum(0)
    if name == "pre_weight":
        return (dh.double() * mx.checkpoint_load(ctx.x, mx.OUT_FP32).double()).abs().sum(0)
    t = p.dx.double().abs() * 1.01 * ctx.gate[:1].double().abs()
    return t.sum(0) if name == "post_bias" else (t * mx.checkpoint_load(ctx.f, mx.OUT_FP32).double().abs()).sum(0)


def _gate_size(mx, ctx, p):
    u = mx.checkpoint_load(ctx.f, mx.OUT_FP32).double().abs() * ctx.post.weight.double().abs() + ctx.post.bias.double().abs()
    return (p.dx.double().abs() * 1.01 * u).sum(0)
