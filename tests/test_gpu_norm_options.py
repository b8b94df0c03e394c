"""What the C entry points of the residual norms and activations leave to their caller: outputs that are not asked for, a workspace with anything in
it, floor scaling of what is kept.  Bounds as in test_gpu_residual_norm: K = 2^-18 of the same expression over magnitudes for an element, (rows + 80) 2^-24 and
8 K for a sum over few rows; half a step for the rounding at the end."""
import ctypes as C
import itertools

import pytest
import torch

import norm_reference as R

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
K = 2.0 ** -18


@pytest.fixture(scope="module")
def mx():
    import paper_2502_20853_b200 as m
    m.lib()
    return m


def _within(got, want, bound, what):
    far = (got.double() - want).abs() - bound
    assert bool((far <= 0).all()), "%s: worst by %.3g" % (what, float(far.max()))


def _case(mx, rows, cols, gates, post, dtype=BF16):
    g = torch.Generator(device="cuda").manual_seed(rows + cols + gates)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    pre = (1 + 0.3 * rnd(cols), 0.2 * rnd(cols))
    side = (1 + 0.3 * rnd(cols), 0.2 * rnd(cols)) if post else None
    gate = rnd(gates, cols) if gates else None
    return rnd(rows, cols).to(dtype), rnd(rows, cols).to(BF16), pre, side, gate, (1e-2 * rnd(rows, cols)).to(BF16), (1e-2 * rnd(rows, cols)).to(dtype)


NAMES = ["dw_pre", "db_pre", "dw_post", "db_post", "dgate"]
REFERENCE = dict(dw_pre="pre_weight", db_pre="pre_bias", dw_post="post_weight", db_post="post_bias", dgate="gate")


@pytest.mark.parametrize("cols", [96, 768, 1056])
@pytest.mark.parametrize("gates,post", [(0, False), (0, True), (1, False), (1, True), (7, False), (7, True)])
def test_gradients_that_are_not_asked_for(mx, cols, gates, post):
    from paper_2502_20853_b200 import binding as b
    rows = 7 * 19
    x, f, pre, side, gate, dh, dx_out = _case(mx, rows, cols, gates, post)
    _, _, ctx = mx.residual_norm_fwd(x, f, pre=mx.Norm(mx.NORM_LAYER, *pre), post=mx.Norm(mx.NORM_RMS, *side) if post else None, gate=gate)
    st = ctx.stats.double()[:, :, None]
    need_f = post or gates
    xh = R.load(ctx.x.codes, ctx.x.scales)
    fh = R.load(ctx.f.codes, ctx.f.scales) if need_f else None
    want = R.norm_bwd(dh, dx_out, xh, fh, st[1], st[3] if post else None, ("layer", *pre), ("rms", *side) if post else None, gate, 1.0, 1.0)
    norm = lambda kind, p: b.CNorm(kind, 1, p[0].data_ptr(), p[1].data_ptr(), 1e-6, 0) if p else b.CNorm(0, 0, None, None, 0.0, 0)  # noqa: E731
    plan = b.CResidualNorm(rows, cols, 0, 1, 1.0, 1.0, norm(1, pre), norm(2, side), gate.data_ptr() if gates else None, gates, cols)
    size = mx.residual_norm_workspace_bytes(rows, cols, gates)
    work = torch.full((size // 4 + 64,), float("nan"), device="cuda")
    possible = NAMES[:2] + (NAMES[2:4] if post else []) + (NAMES[4:] if gates else [])
    for asked in itertools.chain.from_iterable(itertools.combinations(possible, n) for n in range(len(possible) + 1)):
        for with_df in (True, False):
            out = {n: torch.full((gates if n == "dgate" else 1, cols), float("nan"), device="cuda") for n in asked}
            dx, df = torch.empty_like(dx_out), torch.empty_like(dh)
            work.fill_(float("nan"))
            k = dict(dh=dh.data_ptr(), lddh=cols, dx_out=dx_out.data_ptr(), lddxo=cols, stats=ctx.stats.data_ptr(), x_ckpt=ctx.x.c(), f_ckpt=ctx.f.c() if need_f else b._NO_CKPT,
                     x_out=None, ldxo=0, f=None, ldf=0, dx=dx.data_ptr(), lddx=cols, df=df.data_ptr() if with_df else None, lddf=cols,
                     **{n: out[n].data_ptr() if n in asked else None for n in NAMES})
            s = b.CResidualNormBwd(*[k[n] for n, _ in b.CResidualNormBwd._fields_])
            assert mx.lib().mxfp4_residual_norm_bwd(C.byref(plan), C.byref(s), work.data_ptr(), size, torch.cuda.current_stream().cuda_stream) == 0
            assert bool(torch.isnan(work[size // 4:]).all())
            _within(dx, want["dx"], want["dx"].abs() * 2.0 ** -8 * 1.001 + 4 * K * want["abs_dx"] + 1e-37, "dx")
            if with_df:
                _within(df, want["df"], want["df"].abs() * 2.0 ** -8 * 1.001 + 8 * K * want["abs_df"] + 1e-37, "df")
            for n in asked:
                _within(out[n], want[REFERENCE[n]], ((rows + 80) * 2.0 ** -24 + 8 * K) * want["abs_" + REFERENCE[n]] + 1e-37, "%s of %s" % (n, asked))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("gates", [0, 1, 7])
def test_forward_without_the_sum(mx, dtype, gates):
    """x_out is optional where there is h, h where there is x_out or hq: the rest stays as it is, bit for bit."""
    from paper_2502_20853_b200 import binding as b
    rows, cols = 7 * 19, 416
    x, f, pre, side, gate, _, _ = _case(mx, rows, cols, gates, True, dtype)
    want = mx.residual_norm_fwd(x, f, pre=mx.Norm(mx.NORM_LAYER, *pre), post=mx.Norm(mx.NORM_RMS, *side), gate=gate)
    norm = lambda kind, p: b.CNorm(kind, 1, p[0].data_ptr(), p[1].data_ptr(), 1e-6, 0)  # noqa: E731
    plan = b.CResidualNorm(rows, cols, int(dtype == F32), 1, 1.0, 1.0, norm(1, pre), norm(2, side), gate.data_ptr() if gates else None, gates, cols)
    for with_x, with_h in ((True, True), (True, False), (False, True)):
        x_out, h, stats = torch.full_like(x, 9.0), torch.full_like(f, 9.0), torch.empty(4, rows, device="cuda")
        kx, kf = mx.Checkpoint.empty(rows, cols), mx.Checkpoint.empty(rows, cols)
        assert mx.lib().mxfp4_residual_norm_fwd(C.byref(plan), x.data_ptr(), cols, f.data_ptr(), cols, x_out.data_ptr() if with_x else None, cols, h.data_ptr() if with_h else None, cols,
                                                None, stats.data_ptr(), kx.c(), kf.c(), 0, None, torch.cuda.current_stream().cuda_stream) == 0
        assert torch.equal(x_out, want[0]) if with_x else bool((x_out == 9.0).all())
        assert torch.equal(h, want[1]) if with_h else bool((h == 9.0).all())
        assert torch.equal(stats, want[2].stats)
        for a, c in ((kx, want[2].x), (kf, want[2].f)):
            assert torch.equal(a.codes, c.codes) and torch.equal(a.scales, c.scales)


def test_checkpoint_alone(mx):
    """act_fwd without z writes the checkpoint only."""
    from paper_2502_20853_b200 import binding as b
    y = (3 * torch.randn(70, 192, device="cuda")).to(BF16)
    for act, cols in ((mx.ACT_GELU, 192), (mx.ACT_SILU, 192), (mx.ACT_GEGLU, 96), (mx.ACT_SWIGLU, 96)):
        c, want = mx.Checkpoint.empty(70, 192), mx.checkpoint_store(y)
        assert mx.lib().mxfp4_act_fwd(y.data_ptr(), 192, 70, cols, act, None, 0, c.c(), 0, None, torch.cuda.current_stream().cuda_stream) == 0
        assert torch.equal(c.codes, want.codes) and torch.equal(c.scales, want.scales)
        assert mx.lib().mxfp4_act_fwd(y.data_ptr(), 192, 70, cols, act, None, 0, b._NO_CKPT, 0, None, None) == 1


@pytest.mark.parametrize("cols", [32, 96, 768, 1056, 4096])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_floor_scaling_of_what_is_kept(mx, cols, dtype):
    """s = floor(log2 M) - 8: magnitudes beyond 448 2^s are kept as that."""
    rows = 67
    x, f, pre, side, gate, _, _ = _case(mx, rows, cols, 1, True, dtype)
    x_out, h, ctx = mx.residual_norm_fwd(x, f, pre=mx.Norm(mx.NORM_LAYER, *pre), post=mx.Norm(mx.NORM_RMS, *side), gate=gate, scale_mode=mx.SCALE_FLOOR)
    free = mx.residual_norm_fwd(x, f, pre=mx.Norm(mx.NORM_LAYER, *pre), post=mx.Norm(mx.NORM_RMS, *side), gate=gate)
    assert torch.equal(x_out, free[0]) and torch.equal(h, free[1]) and torch.equal(ctx.stats, free[2].stats)
    o = R.norm_fwd(x, f, ("layer", *pre), ("rms", *side), gate, 1.0, 1.0, 1e-6)
    for c, v in ((ctx.x, o["xh"]), (ctx.f, o["fh"])):
        power = torch.ldexp(torch.ones_like(c.scales, dtype=torch.float64), c.scales.to(torch.int32) - 127)
        m = v.abs().reshape(rows, -1, 32).amax(2)
        # FP32 errors: a few 2^-18 of the row's size, which is near 1 (the branch and its gate are of the residual's size)
        err = 64 * K * (1 + v.abs())
        e = err.reshape(rows, -1, 32).amax(2)
        assert bool((power * 256 <= m + e).all()) and bool((power * 512 > m - e).all())
        power = power.repeat_interleave(32, 1)
        kept = torch.minimum(v.abs(), 448 * power) * v.sign()
        _within(R.load(c.codes, c.scales), kept, kept.abs() * 2.0 ** -4 + power * 2.0 ** -10 + err, "floor")
    dy = mx.residual_norm_bwd(torch.ones_like(f), torch.ones_like(x), ctx)
    assert bool(torch.isfinite(dy.dx).all())
