"""Residual addition between two norms, forward and backward, against the 64-bit reference.

Tolerances.  u = 2^-24.  A sum over a row is made of at most 16 additions in a lane, one of the lane's pair, five over the warp's lanes and
16 over warps: below 40 u of the sum of magnitudes, so with the roundings around it every mean, deviation and projection is good to
K = 2^-18 of the same expression over magnitudes, and a normalized element to K (|v^| + (|v| + mean |v|) / deviation).  bf16 results are off by
half a step, 2^-8 of their value, besides; E4M3 codes by 2^-4 of it, or half the smallest step of their group.  A sum over n rows adds
(n + 80) u of the sum of magnitudes.
"""
import itertools

import pytest
import torch

import norm_reference as R

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
K = 2.0 ** -18
EPS = 1e-6


@pytest.fixture(scope="module")
def mx():
    import paper_2502_20853_b200 as m
    m.lib()
    return m


class Case:
    """Inputs of one call, for the library and for the reference."""

    def __init__(self, mx, rows, cols, pre, post, gates, dtype=BF16, params=F32, bias=True, weight=True, a=1.0, s=1.0, extra=0, offset=0.0, with_f=True, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed + rows * 7 + cols)
        rnd = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731
        kinds = {"layer": mx.NORM_LAYER, "rms": mx.NORM_RMS}
        self.mx, self.rows, self.cols, self.a, self.s, self.dtype = mx, rows, cols, a, s, dtype

        def wide(t):
            if not extra:
                return t
            big = torch.full((t.shape[0], t.shape[1] + extra), 3.0, dtype=t.dtype, device="cuda")
            big[:, :t.shape[1]] = t
            return big[:, :t.shape[1]]

        x = rnd(rows, cols) + offset
        x[:, 3] *= 20.0
        self.x = wide(x.to(dtype))
        self.f = wide((0.5 * rnd(rows, cols) + offset).to(BF16)) if with_f else None
        self.gate = wide((0.5 * rnd(gates, cols)).to(params)) if gates else None

        def side(kind):
            if kind is None:
                return None, None
            w = (1 + 0.3 * rnd(cols)).to(params) if weight else None
            b = (0.2 * rnd(cols)).to(params) if bias else None
            return mx.Norm(kinds[kind], w, b, EPS), (kind, w, b)

        self.pre, self.r_pre = side(pre)
        self.post, self.r_post = side(post)
        self.dh = wide((1e-2 * rnd(rows, cols)).to(BF16)) if pre else None
        self.dx_out = wide((1e-2 * rnd(rows, cols)).to(dtype))
        self.eight_f = with_f and (post is not None or gates > 0)

    def fwd(self, **kw):
        return self.mx.residual_norm_fwd(self.x, self.f, pre=self.pre, post=self.post, gate=self.gate, residual_scale=self.a, branch_scale=self.s, **kw)

    def reference(self):
        return R.norm_fwd(self.x, self.f, self.r_pre, self.r_post, self.gate, self.a, self.s, EPS)

    def fwd_errors(self):
        """Bounds on the FP32 errors of x_out, x^, h and f^ (before their rounding to fewer bits)."""
        o = self.reference()
        x = self.x.double()
        ef = torch.zeros_like(x)
        if self.f is not None:
            f = self.f.double()
            if self.r_post is not None:
                rstd = o["post"][1]
                ef = K * (o["fh"].abs() + (f.abs() + f.abs().mean(1, keepdim=True)) * rstd)
                w = self.r_post[1].double().abs() if self.r_post[1] is not None else 1.0
                eu = ef * w + K * o["u"].abs() + K * (o["fh"].abs() * w)
            else:
                eu = torch.zeros_like(x)
            g = R.gate_rows(self.gate, self.rows).abs() if self.gate is not None else 1.0
            ex = abs(self.s) * g * (eu + K * o["u"].abs()) + K * (self.a * x).abs()
        else:
            ex = torch.zeros_like(x)
        e = {"x_out": ex, "fh": ef}
        if self.r_pre is not None:
            xo, (mean, rstd) = o["x_out"].abs(), o["pre"]
            own = K * (o["xh"].abs() + (xo + xo.mean(1, keepdim=True)) * rstd)
            # an error of x' shifts itself, the mean and the projection of the row
            sent = rstd * (ex + ex.mean(1, keepdim=True) + o["xh"].abs() * (ex * o["xh"].abs()).mean(1, keepdim=True))
            e["xh"] = own + sent * 1.001
            w = self.r_pre[1].double().abs() if self.r_pre[1] is not None else 1.0
            e["h"] = e["xh"] * w + K * (o["h"].abs() + o["xh"].abs() * w)
        return o, e


def _within(got, want, bound, what):
    far = (got.double() - want).abs() - bound
    assert bool((far <= 0).all()), "%s: %d of %d outside, worst by %.3g at %d" % (what, int((far > 0).sum()), far.numel(), float(far.max()), int(far.argmax()))


def _half_step(t, v):
    return v.abs() * torch.finfo(t).eps / 2


def _check_ckpt(c, v, err, what):
    back = R.load(c.codes, c.scales)
    power = torch.ldexp(torch.ones_like(c.scales, dtype=torch.float64), c.scales.to(torch.int32) - 127).repeat_interleave(32, 1)
    _within(back, v, v.abs() * 2.0 ** -4 + power * 2.0 ** -10 + err * 1.1, what)
    # the scale is that of the group's largest magnitude, give or take its error at the border of the rule
    m = v.abs().reshape(v.shape[0], -1, 32).amax(2)
    e = err.reshape(v.shape[0], -1, 32).amax(2)
    lo, hi = (R.store((m + d)[:, :, None].expand(-1, -1, 32).reshape(v.shape))[1] for d in (-e.clamp(max=m), e))
    s = c.scales.to(torch.int32) - 127
    assert bool((s >= lo).all()) and bool((s <= hi).all()), what + ": scale"


def _check_fwd(k, x_out, h, ctx=None):
    o, e = k.fwd_errors()
    if x_out is not None:
        _within(x_out, o["x_out"], e["x_out"] + _half_step(k.dtype, o["x_out"]) * (1 + 1e-3) + 1e-37, "x_out")
    if h is not None:
        _within(h, o["h"], e["h"] + _half_step(BF16, o["h"]) * (1 + 1e-3) + 1e-37, "h")
    if ctx is not None:
        if k.pre is not None:
            if isinstance(ctx.x, k.mx.Checkpoint):
                _check_ckpt(ctx.x, o["xh"], e["xh"], "x^")
            mean, rstd = o["pre"]
            xo = o["x_out"].abs().mean(1) + e["x_out"].mean(1)
            _within(ctx.stats[0], mean[:, 0], K * xo + e["x_out"].mean(1), "mean")
            _within(ctx.stats[1], rstd[:, 0], rstd[:, 0] * (K * (2 + 2 * xo * rstd[:, 0]) + 2 * (e["x_out"] * o["xh"].abs()).mean(1) * rstd[:, 0]), "rstd")
        if k.post is not None:
            mean, rstd = o["post"]
            fa = k.f.double().abs().mean(1)
            _within(ctx.stats[2], mean[:, 0], K * fa, "post mean")
            _within(ctx.stats[3], rstd[:, 0], rstd[:, 0] * K * (2 + 2 * fa * rstd[:, 0]), "post rstd")
        if isinstance(ctx.f, k.mx.Checkpoint):
            _check_ckpt(ctx.f, o["fh"], e["fh"], "f^")


def _check_bwd(k, ctx, g, dx_out=None):
    x, f = ctx.x, ctx.f
    st = ctx.stats.double()[:, :, None] if ctx.stats is not None else None
    eight = isinstance(x if x is not None else f, k.mx.Checkpoint)
    xh = fh = None
    xe = fe = 0.0      # what a normalized row that is made again from its input is off by
    if x is not None:
        xh = R.load(x.codes, x.scales) if eight else (x.double() - st[0]) * st[1]
        xe = 0.0 if eight else 3 * 2.0 ** -24 * (x.double().abs() + st[0].abs()) * st[1]
    if f is not None:
        fh = R.load(f.codes, f.scales) if eight else (f.double() - st[2]) * st[3] if k.post is not None else f.double()
        fe = 3 * 2.0 ** -24 * (f.double().abs() + st[2].abs()) * st[3] if not eight and k.post is not None else 0.0
    args = (st[1] if k.pre is not None else None, st[3] if k.post is not None else None, k.r_pre, k.r_post, k.gate, k.a, k.s)
    o = R.norm_bwd(k.dh, dx_out, xh, fh, *args)
    # the same with magnitudes that hold the normalized rows' errors
    m = R.norm_bwd(k.dh, dx_out, xh.abs() + xe / K if xh is not None else None, fh.abs() + fe / K if fh is not None else None, *args)
    n = (k.rows + 80) * 2.0 ** -24
    _within(g.dx, o["dx"], _half_step(k.dtype, o["dx"]) * 1.001 + 4 * K * m["abs_dx"] + 1e-37, "dx")
    if g.df is not None:
        _within(g.df, o["df"], _half_step(BF16, o["df"]) * 1.001 + 8 * K * m["abs_df"] + 1e-37, "df")
    for name in ("pre_weight", "pre_bias", "post_weight", "post_bias", "gate"):
        got = getattr(g, name)
        if got is not None:
            _within(got, o[name], (n + 8 * K) * m["abs_" + name] + 1e-37, name)
    if k.pre is not None:
        assert (g.pre_weight is None) == (k.r_pre[1] is None) and (g.pre_bias is None) == (k.r_pre[2] is None)
    if k.post is not None:
        assert (g.post_weight is None) == (k.r_post[1] is None) and (g.post_bias is None) == (k.r_post[2] is None)
    assert (g.gate is None) == (k.gate is None)


def _both_ways(k, save, dx_out=True):
    x_out, h, ctx = k.fwd(save=save)
    _check_fwd(k, x_out, h, ctx)
    d = k.dx_out if dx_out else None
    kw = {} if dx_out else dict(dx=torch.empty(k.rows, k.cols, dtype=k.dtype, device="cuda"))
    _check_bwd(k, ctx, k.mx.residual_norm_bwd(k.dh, d, ctx, **kw), d)


KINDS = [None, "layer", "rms"]


@pytest.mark.parametrize("pre,post,gates", [c for c in itertools.product(KINDS, KINDS, [0, 1, 3])])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("eight", [True, False])
def test_every_form(mx, pre, post, gates, dtype, eight):
    k = Case(mx, 33, 160, pre, post, gates, dtype, params=F32 if dtype == F32 else BF16, a=0.75, s=1.5)
    _both_ways(k, mx.SAVE_8BIT if eight else mx.SAVE_INPUTS)


# every number of lanes and vectors per lane, full and partly filled
@pytest.mark.parametrize("cols", [32, 64, 96, 128, 160, 192, 224, 256, 288, 352, 384, 416, 512, 768, 800, 1024, 1056, 1536, 1568, 2048, 2080, 4096, 4128, 6144, 8160, 8192])
@pytest.mark.parametrize("eight", [True, False])
def test_widths(mx, cols, eight):
    for rows in (1, 2, 37):
        k = Case(mx, rows, cols, "layer", "rms" if cols % 64 else "layer", 1, F32 if cols % 96 else BF16, seed=rows)
        _both_ways(k, mx.SAVE_8BIT if eight else mx.SAVE_INPUTS)


@pytest.mark.parametrize("rows,gates", [(1, 1), (7, 7), (12, 6), (197, 1), (394, 2), (2400, 48), (2400, 600), (2401, 7), (3000, 1), (5003, 1), (5000, 1000), (5000, 5000)])
@pytest.mark.parametrize("cols", [96, 384])
def test_runs_of_gates(mx, rows, gates, cols):
    """Gates that cover one row, less than a team's rows, many teams' rows; teams that have no rows."""
    _both_ways(Case(mx, rows, cols, "rms", "layer", gates, extra=8), mx.SAVE_8BIT)


@pytest.mark.parametrize("weight,bias", [(False, False), (False, True), (True, False)])
def test_missing_parameters(mx, weight, bias):
    k = Case(mx, 65, 96, "layer", "layer", 5, weight=weight, bias=bias)
    _both_ways(k, mx.SAVE_8BIT)
    _both_ways(Case(mx, 65, 96, "layer", "layer", 0, weight=weight, bias=bias), mx.SAVE_INPUTS)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strided(mx, dtype):
    for save in (mx.SAVE_8BIT, mx.SAVE_INPUTS):
        k = Case(mx, 129, 224, "layer", "rms", 3, dtype, extra=32)
        _both_ways(k, save)
    big = torch.full((129, 224 + 32), 9.0, dtype=dtype, device="cuda")
    hig = torch.full((129, 224 + 64), 9.0, dtype=BF16, device="cuda")
    x_out, h, ctx = k.fwd(x_out=big[:, :224], h=hig[:, :224])
    _check_fwd(k, x_out, h, ctx)
    assert bool((big[:, 224:] == 9.0).all()) and bool((hig[:, 224:] == 9.0).all())
    big.fill_(9.0), hig.fill_(9.0)
    _check_bwd(k, ctx, mx.residual_norm_bwd(k.dh, k.dx_out, ctx, dx=big[:, :224], df=hig[:, :224]), k.dx_out)
    assert bool((big[:, 224:] == 9.0).all()) and bool((hig[:, 224:] == 9.0).all())


def test_large_mean(mx):
    """A row whose mean is far larger than its deviation: the two passes keep its digits."""
    for save in (mx.SAVE_8BIT, mx.SAVE_INPUTS):
        _both_ways(Case(mx, 40, 768, "layer", "layer", 1, F32, offset=100.0), save)


def test_norm_alone(mx):
    for dtype, save in ((BF16, mx.SAVE_8BIT), (F32, mx.SAVE_INPUTS)):
        k = Case(mx, 50, 384, "layer", None, 0, dtype, with_f=False)
        x_out, h, ctx = k.fwd(save=save)
        assert x_out is None
        _check_fwd(k, None, h, ctx)
        _check_bwd(k, ctx, mx.residual_norm_bwd(k.dh, k.dx_out, ctx, df=False), k.dx_out)


def test_no_gradient_from_further_on(mx):
    for dtype in (BF16, F32):
        _both_ways(Case(mx, 50, 384, "layer", "rms", 2, dtype), mx.SAVE_8BIT, dx_out=False)


def test_nothing_saved_gives_the_same(mx):
    k = Case(mx, 77, 384, "layer", "rms", 7)
    x_out, h, ctx = k.fwd(save=mx.SAVE_NOTHING)
    x2, h2, _ = k.fwd()
    assert ctx is None and torch.equal(x_out, x2) and torch.equal(h, h2)


@pytest.mark.parametrize("rows,cols", [(1, 32), (1, 4096), (33, 96), (197, 384), (128, 160), (300, 1056)])
@pytest.mark.parametrize("floor", [0, 1])
def test_quantized_for_the_next_layer(mx, rows, cols, floor):
    k = Case(mx, rows, cols, "layer", "rms", 1)
    hq = mx.QMat(rows, cols)
    hq.scales.zero_()
    _, h, _ = k.fwd(hq=hq, scale_mode=floor)
    want = mx.quantize(h, scale_mode=floor)
    assert torch.equal(hq.data, want.data) and torch.equal(hq.scales[:mx.scale_bytes(rows, cols)], want.scales[:mx.scale_bytes(rows, cols)])
    only = mx.QMat(rows, cols)
    x_out, none, _ = k.fwd(hq=only, h=False, scale_mode=floor)
    assert none is None and torch.equal(only.data, want.data)


def test_rows_that_are_not_finite(mx):
    k = Case(mx, 40, 96, "layer", "layer", 1)
    k.x[7, 5] = float("inf")
    k.f[9, 70] = float("nan")
    st = mx.new_status()
    hq = mx.QMat(40, 96)
    x_out, h, ctx = k.fwd(dev_status=st, hq=hq)
    assert int(st.item()) == mx.DEV_NONFINITE
    bad = torch.isnan(h).any(1)
    assert bad.nonzero().flatten().tolist() == [7, 9] and bool(torch.isnan(h[bad]).all())
    assert bool((ctx.x.scales[7] == 255).all()) and bool((ctx.x.scales[9] == 255).all()) and bool((ctx.x.scales[8] != 255).all())
    g = mx.residual_norm_bwd(k.dh, k.dx_out, ctx)
    assert torch.isnan(g.dx).any(1).nonzero().flatten().tolist() == [7, 9]
    k2 = Case(mx, 40, 96, "layer", "layer", 1)
    st.zero_()
    x2, h2, _ = k2.fwd(dev_status=st)
    assert int(st.item()) == 0 and torch.equal(h2[~bad], h[~bad]) and torch.equal(x2[~bad], x_out[~bad])


def test_rows_without_deviation(mx):
    """Constant and zero rows: x^ is 0, 1 / deviation 1 / sqrt(eps), and nothing divides by zero."""
    for kind in ("layer", "rms"):
        k = Case(mx, 6, 96, kind, kind, 0)
        k.x.fill_(0.0), k.f.fill_(0.0)
        x_out, h, ctx = k.fwd()
        assert bool((x_out == k.post.bias.to(x_out.dtype)).all())
        _check_bwd(k, ctx, mx.residual_norm_bwd(k.dh, k.dx_out, ctx), k.dx_out)
        assert bool((ctx.f.codes == 0).all()) and bool((ctx.f.scales == 92).all())


@pytest.mark.parametrize("scale", [1e-30, 1e-35, 1e-38, 1e30])
def test_rows_of_extreme_size(mx, scale):
    """eps dominates the deviation of tiny rows: their x^ are tiny numbers, for which 2^-s / deviation leaves FP32; squares of large rows do."""
    k = Case(mx, 9, 160, "rms", "rms", 0, F32)
    k.x.mul_(scale)
    k.f = (k.f.float() * scale).to(BF16)
    if scale > 1:
        k.x.div_(1e13), k.f.div_(1e13)      # 1e17: the squares' sum stays finite
    k.post.weight.fill_(1.0)
    k.post.bias = k.pre.bias = None
    k.r_pre, k.r_post = ("rms", k.pre.weight, None), ("rms", k.post.weight, None)
    _both_ways(k, mx.SAVE_8BIT)


@pytest.mark.parametrize("cols,rows,gates", [(32, 400000, 1), (96, 300000, 0), (64, 250000, 1250), (128, 120000, 4), (384, 60000, 300), (768, 30000, 150), (1024, 12000, 3),
                                             (4096, 9000, 1), (8192, 2500, 25)])
def test_many_rows(mx, cols, rows, gates):
    """More blocks than are resident forward, long runs of rows backward."""
    for dtype in (BF16, F32):
        k = Case(mx, rows, cols, "layer", "layer" if gates else None, gates, dtype)
        _both_ways(k, mx.SAVE_8BIT if dtype == BF16 else mx.SAVE_INPUTS)
        del k
        torch.cuda.empty_cache()


# widths whose rows do not fill their lanes: the parts of a row's warps differ by a group, a lane's last vector is missing; with the sums of one
# norm without biases (2), with them, and of two norms with them (4)
@pytest.mark.parametrize("cols", [320, 416, 480, 544, 640, 992, 1120, 1152, 1280, 1312, 1440, 1824, 2272, 2560, 2592, 3104, 4160, 5120, 5472, 6048, 6336, 7328])
@pytest.mark.parametrize("post,bias", [(None, False), (None, True), ("layer", True)])
def test_rows_that_do_not_fill_their_lanes(mx, cols, post, bias):
    for dtype, save in ((BF16, mx.SAVE_8BIT), (F32, mx.SAVE_INPUTS), (F32, mx.SAVE_8BIT)):
        _both_ways(Case(mx, 41, cols, "layer", post, 1, dtype, bias=bias, seed=cols), save)


@pytest.mark.parametrize("rows,cols,gates", [(9000, 160, 9000), (12000, 640, 800), (12000, 1056, 40), (9000, 1024, 3), (6000, 2080, 1500), (1212, 4128, 606), (700, 8192, 7)])
@pytest.mark.parametrize("bias", [False, True])
def test_gates_of_few_and_of_many_blocks(mx, rows, cols, gates, bias):
    _both_ways(Case(mx, rows, cols, "rms", "layer", gates, BF16, bias=bias), mx.SAVE_8BIT)


def test_kept_inputs_are_not_written_over(mx):
    k = Case(mx, 8, 96, "layer", "rms", 1)
    with pytest.raises(AssertionError):
        k.fwd(save=mx.SAVE_INPUTS, h=k.f)
    with pytest.raises(AssertionError):
        k.fwd(save=mx.SAVE_INPUTS, x_out=k.f)
    with pytest.raises(AssertionError):
        mx.residual_norm_bwd(None, None, k.fwd()[2])
    for bad in (k.x.cpu(), k.x.double(), k.x[0], k.x.t()):
        with pytest.raises((AssertionError, mx.MxError, ValueError)):
            mx.residual_norm_fwd(bad, pre=k.pre)
    with pytest.raises(AssertionError):
        mx.residual_norm_fwd(k.x, pre=mx.Norm(mx.NORM_LAYER, k.pre.weight[:32], None))
    with pytest.raises(AssertionError):
        mx.residual_norm_fwd(k.x, pre=mx.Norm(mx.NORM_LAYER, k.pre.weight, k.pre.bias.to(BF16)))
    with pytest.raises(AssertionError):
        mx.residual_norm_fwd(k.x, k.f[:4], pre=k.pre)
    with pytest.raises(AssertionError):
        mx.checkpoint_load(mx.checkpoint_store(k.x), out=torch.empty(8, 64, dtype=BF16, device="cuda"))


def test_outputs_over_inputs(mx):
    k = Case(mx, 90, 384, "layer", "rms", 3)
    x_out, h, ctx = k.fwd()
    x, f = k.x.clone(), k.f.clone()
    k.x, k.f = x, f
    x2, h2, ctx2 = k.fwd(x_out=x, h=f)
    assert x2 is x and h2 is f and torch.equal(x, x_out) and torch.equal(f, h) and torch.equal(ctx.f.codes, ctx2.f.codes)
    g = mx.residual_norm_bwd(k.dh, k.dx_out, ctx)
    dh, dxo = k.dh.clone(), k.dx_out.clone()
    g2 = mx.residual_norm_bwd(dh, dxo, ctx, dx=dxo, df=dh)
    for a, b in zip(g, g2):
        assert torch.equal(a, b)


def test_same_bits_every_time(mx):
    for gates in (1, 6, 300):
        k = Case(mx, 1200, 768, "layer", "layer", gates)
        _, _, ctx = k.fwd()
        g = mx.residual_norm_bwd(k.dh, k.dx_out, ctx)
        for _ in range(3):
            assert all(torch.equal(a, b) for a, b in zip(g, mx.residual_norm_bwd(k.dh, k.dx_out, ctx)))


def test_captured_and_on_another_stream(mx):
    k = Case(mx, 333, 384, "layer", "rms", 9)
    x_out, h, ctx = k.fwd()
    g = mx.residual_norm_bwd(k.dh, k.dx_out, ctx)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        _, h1, c1 = k.fwd()
        g1 = mx.residual_norm_bwd(k.dh, k.dx_out, c1)
    torch.cuda.synchronize()
    assert torch.equal(h, h1) and all(torch.equal(a, b) for a, b in zip(g, g1))
    x, x0 = torch.zeros_like(k.x), k.x
    k.x = x
    graphs = []
    for _ in range(2):      # two graphs, each with buffers of its own
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            _, h2, c2 = k.fwd()
            g2 = mx.residual_norm_bwd(k.dh, k.dx_out, c2)
        graphs.append((graph, h2, g2))
    x.copy_(x0)
    for graph, h2, g2 in graphs + graphs[:1]:
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(h, h2) and all(torch.equal(a, b) for a, b in zip(g, g2))


def test_two_streams_at_once(mx):
    cases = [Case(mx, 3000, 384, "layer", "rms", 3, seed=k) for k in range(2)]
    want = []
    for k in cases:
        _, h, ctx = k.fwd()
        want.append((h, mx.residual_norm_bwd(k.dh, k.dx_out, ctx)))
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(4):
        for i, k in enumerate(cases):
            with torch.cuda.stream(streams[i]):
                _, h, ctx = k.fwd()
                got[i] = (h, mx.residual_norm_bwd(k.dh, k.dx_out, ctx))
    torch.cuda.synchronize()
    for (h, g), (h2, g2) in zip(want, got):
        assert torch.equal(h, h2) and all(torch.equal(a, b) for a, b in zip(g, g2))


def test_against_differences(mx):
    """x_out in FP32 is linear in x, the gate and N_post's parameters: differences of the forward pass itself against its backward pass."""
    k = Case(mx, 48, 96, None, "layer", 4, F32, a=0.5, s=2.0)
    _, _, ctx = k.fwd(save=mx.SAVE_INPUTS)
    g = mx.residual_norm_bwd(None, k.dx_out, ctx)
    loss = lambda: float((k.fwd(save=mx.SAVE_NOTHING)[0].double() * k.dx_out.double()).sum())  # noqa: E731
    at = loss()
    mags = float((k.fwd(save=mx.SAVE_NOTHING)[0].double() * k.dx_out.double()).abs().sum())
    for name, t in (("dx", k.x), ("gate", k.gate), ("post_weight", k.post.weight), ("post_bias", k.post.bias)):
        d = torch.randn(t.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
        keep = t.clone()
        t.add_(d)
        moved = loss() - at
        moved_by = (t.double() - keep.double())
        t.copy_(keep)
        want = float((getattr(g, name).double() * moved_by).sum())
        bound = 40 * K * (mags + float((getattr(g, name).double() * moved_by).abs().sum())) * 4
        assert abs(moved - want) <= bound, name


def test_no_rows(mx):
    k = Case(mx, 0, 96, "layer", "rms", 2)
    x_out, h, ctx = k.fwd()
    g = mx.residual_norm_bwd(k.dh, k.dx_out, ctx)
    assert x_out.shape == h.shape == g.dx.shape == (0, 96)
    for t in (g.pre_weight, g.pre_bias, g.post_weight, g.post_bias, g.gate):
        assert bool((t == 0).all())
    assert g.gate.shape == (2, 96)
