"""The sums over rows of residual_norm_bwd on long matrices, to bounds that a lost block of rows does not pass.

Bounds.  u = 2^-24.  The rows are dealt to at least 148 blocks (or one row to each team), so a block has at most rows / 148 + 1 rows for each of its teams, of
which there are at most 64.  What lies on the way of one term into its sum: the additions of its team's rows (at most rows / 148 + 1, and one
block's gates, of which there are no more than its rows), of the teams of a block (a team leaves at most two parts: 128) and of the blocks (3 in a
lane, 4 over lanes, 8 over warps, and as many over the blocks of a gate as it has, below 300).  Each is off by u of what has been added so far, which is
at most the sum of magnitudes: (rows / 148 + 450) u of it, and 2^-15 for the terms themselves (as in test_gpu_residual_norm).
The inputs have means of their own per column, so that a sum is of the order of its magnitudes and a part of it is missed when it is lost: the test
asserts for every gradient that leaving out a 1 / 400 of the rows would be seen, in each eighth of the columns."""
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


def _inputs(rows, cols, gates, dtype, post):
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    sign = torch.where(torch.arange(cols, device="cuda") % 2 == 0, 1.0, -1.0)
    x = (1.5 * sign + 0.5 * rnd(rows, cols)).to(dtype)
    f = (1.5 * sign.flip(0) + 0.5 * rnd(rows, cols)).to(BF16)
    dh = (0.01 * (1.0 + 0.5 * rnd(rows, cols)) * sign.roll(cols // 2)).to(BF16)
    dx_out = (0.01 * (2.0 + 0.5 * rnd(rows, cols))).to(dtype)
    side = lambda: (1 + 0.3 * rnd(cols), 0.2 * rnd(cols))  # noqa: E731
    gate = (1.0 + 0.3 * rnd(gates, cols)) if gates else None
    return x, f, dh, dx_out, side(), side() if post else None, gate


# widths of every number of vectors per lane and of teams per block, one gate, few rows per gate and many
CASES = [(400000, 32, 1), (300000, 96, 0), (250000, 64, 1250), (120000, 128, 4), (60000, 384, 300), (60000, 384, 1), (30000, 768, 150), (40000, 800, 8), (12000, 1024, 3),
         (9000, 2048, 0), (9000, 4096, 1), (2500, 8192, 25), (3000, 1536, 1500)]


@pytest.mark.parametrize("rows,cols,gates", CASES)
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("eight", [True, False])
def test_no_rows_are_lost(mx, rows, cols, gates, post, eight):
    dtype = BF16 if eight else F32
    x, f, dh, dx_out, pre, side, gate = _inputs(rows, cols, gates, dtype, post)
    kinds = ("layer", "rms")
    norm = lambda kind, p: mx.Norm({"layer": mx.NORM_LAYER, "rms": mx.NORM_RMS}[kind], *p)  # noqa: E731
    _, _, ctx = mx.residual_norm_fwd(x, f, pre=norm(kinds[0], pre), post=norm(kinds[1], side) if post else None, gate=gate, save=mx.SAVE_8BIT if eight else mx.SAVE_INPUTS)
    got = mx.residual_norm_bwd(dh, dx_out, ctx)
    st = ctx.stats.double()[:, :, None]
    need_f = post or gates
    fh = None
    if eight:
        xh = R.load(ctx.x.codes, ctx.x.scales)
        if need_f:
            fh = R.load(ctx.f.codes, ctx.f.scales)
    else:
        xh = (ctx.x.double() - st[0]) * st[1]
        if need_f:
            fh = (f.double() - st[2]) * st[3] if post else f.double()
    args = (st[1], st[3] if post else None, (kinds[0], *pre), (kinds[1], *side) if post else None, gate, 1.0, 1.0)
    want = R.norm_bwd(dh, dx_out, xh, fh, *args)
    # the same rows, a 1 / 400 of them without their gradients
    cut = slice(rows // 2, rows // 2 + rows // 400)
    dh[cut], dx_out[cut] = 0.0, 0.0
    less = R.norm_bwd(dh, dx_out, xh, fh, *args)
    names = ["pre_weight", "pre_bias"] + (["post_weight", "post_bias"] if post else []) + (["gate"] if gates else [])
    for name in names:
        bound = ((rows / 148 + 450) * 2.0 ** -24 + 2.0 ** -15) * want["abs_" + name]
        far = (getattr(got, name).double() - want[name]).abs() - bound
        assert bool((far <= 0).all()), "%s: %d outside, worst by %.3g" % (name, int((far > 0).sum()), float(far.max()))
        lost = ((less[name] - want[name]).abs() > bound).reshape(-1, cols).any(0)      # (of the gates, those that have these rows)
        assert bool(lost.reshape(8, -1).any(1).all()), name + ": the bound does not see rows that are lost"
        assert bool((want[name].abs() > bound).reshape(-1, cols).any(0).reshape(8, -1).any(1).all()), name
