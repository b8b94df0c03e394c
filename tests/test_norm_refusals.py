"""What the checkpoint, activation and residual-norm entry points refuse, through the C ABI and without a GPU: every call here is refused before
anything is enqueued, so the addresses are made up."""
import ctypes as C

import pytest

import paper_2502_20853_b200 as mx
from paper_2502_20853_b200 import binding as b

INVALID, SHAPE, MISALIGNED, SMALL = 1, 2, 3, 4
AT = 1 << 40      # an address


def ckpt(rows=4, cols=64, codes=AT + (1 << 30), scales=AT + (1 << 31)):
    return b.CCkpt(codes, scales, rows, cols)


@pytest.mark.parametrize("want,kw", [
    (INVALID, dict(src=None)), (INVALID, dict(dtype=2)), (INVALID, dict(mode=2)), (INVALID, dict(c=ckpt(codes=None))), (INVALID, dict(c=ckpt(scales=None))),
    (INVALID, dict(c=ckpt(rows=-1))), (SHAPE, dict(c=ckpt(cols=48))), (SHAPE, dict(ld=63)), (MISALIGNED, dict(src=AT + 8)), (MISALIGNED, dict(ld=68)),
    (MISALIGNED, dict(c=ckpt(codes=AT + 8)))])
def test_checkpoint(want, kw):
    a = dict(src=AT, dtype=0, ld=64, c=ckpt(), mode=0)
    a.update(kw)
    L = mx.lib()
    assert L.mxfp4_checkpoint_store(a["src"], a["dtype"], a["ld"], a["c"], a["mode"], None, None) == want
    if "mode" not in kw:
        assert L.mxfp4_checkpoint_load(a["c"], a["src"], a["dtype"], a["ld"], None) == want


@pytest.mark.parametrize("want,kw", [
    (INVALID, dict(y=None)), (INVALID, dict(act=4)), (INVALID, dict(act=-1)), (INVALID, dict(z=None, c=ckpt(codes=None))), (INVALID, dict(rows=-1)), (INVALID, dict(mode=3)),
    (SHAPE, dict(cols=40)), (SHAPE, dict(ldy=32)), (SHAPE, dict(ldz=32)), (SHAPE, dict(c=ckpt(rows=5))), (SHAPE, dict(act=2)),      # gated: y has 128 columns
    (MISALIGNED, dict(y=AT + 2)), (MISALIGNED, dict(ldy=66)), (MISALIGNED, dict(ldz=65)),
    (INVALID, dict(z=AT + 16)), (INVALID, dict(z=AT, ldz=72)),                                      # over y, but not in the same place
    (INVALID, dict(act=3, ldy=128, c=ckpt(cols=128), z=AT, ldz=128))])                             # gated over y
def test_act_fwd(want, kw):
    a = dict(y=AT, ldy=64, rows=4, cols=64, act=0, z=AT + (1 << 20), ldz=64, c=ckpt(), mode=0)
    a.update(kw)
    assert mx.lib().mxfp4_act_fwd(a["y"], a["ldy"], a["rows"], a["cols"], a["act"], a["z"], a["ldz"], a["c"], a["mode"], None, None) == want


@pytest.mark.parametrize("want,kw", [
    (INVALID, dict(dz=None)), (INVALID, dict(dy=None)), (INVALID, dict(act=7)), (INVALID, dict(c=ckpt(codes=None))), (SHAPE, dict(c=ckpt(cols=40))),
    (SHAPE, dict(act=2, c=ckpt(cols=96), lddy=96)), (SHAPE, dict(lddz=32)), (SHAPE, dict(lddy=32)), (MISALIGNED, dict(dz=AT + 4)), (MISALIGNED, dict(lddy=70)),
    (INVALID, dict(dy=AT + 32))])
def test_act_bwd(want, kw):
    a = dict(dz=AT, lddz=64, c=ckpt(), act=0, dy=AT + (1 << 20), lddy=64)
    a.update(kw)
    assert mx.lib().mxfp4_act_bwd(a["dz"], a["lddz"], a["c"], a["act"], a["dy"], a["lddy"], None) == want


def test_what_lies_side_by_side_does_not_overlap():
    """Refusals of overlaps go by the bytes that each matrix has: the one argument that is wrong here is found behind them."""
    L = mx.lib()
    dz, dy = AT, AT + 4 * 32 * 2                  # gated: dz [4, 32], dy [4, 64] right behind it; the checkpoint's codes lie on 8 bytes
    late = ckpt(codes=AT + (1 << 30) + 8)
    assert L.mxfp4_act_bwd(dz, 32, late, 3, dy, 64, None) == MISALIGNED
    assert L.mxfp4_act_bwd(dz, 32, ckpt(), 3, dy - 16, 64, None) == INVALID


def norm(kind=1, dtype=1, weight=AT, bias=AT + (1 << 12), eps=1e-6):
    return b.CNorm(kind, dtype, weight, bias, eps, 0)


NONE = b.CNorm(0, 0, None, None, 0.0, 0)


def plan(rows=4, cols=64, x_dtype=0, gate_dtype=0, a=1.0, s=1.0, pre=None, post=None, gate=AT + (1 << 13), gates=2, ld_gate=64):
    return b.CResidualNorm(rows, cols, x_dtype, gate_dtype, a, s, pre or norm(), post or norm(kind=2), gate, gates, ld_gate)


PLANS = [(INVALID, dict(rows=-1)), (INVALID, dict(cols=0)), (INVALID, dict(x_dtype=2)), (INVALID, dict(gate_dtype=5)), (INVALID, dict(gate=None)), (INVALID, dict(gates=0)),
         (INVALID, dict(pre=norm(kind=3))), (INVALID, dict(post=norm(dtype=2))), (INVALID, dict(pre=norm(eps=-1.0))), (INVALID, dict(pre=norm(eps=float("nan")))),
         (SHAPE, dict(cols=48)), (SHAPE, dict(cols=8224)), (SHAPE, dict(gates=3)), (SHAPE, dict(ld_gate=32)), (SHAPE, dict(rows=1 << 31, gates=1)),
         (MISALIGNED, dict(gate=AT + 8)), (MISALIGNED, dict(ld_gate=65)), (MISALIGNED, dict(pre=norm(weight=AT + 4))), (MISALIGNED, dict(post=norm(bias=AT + 8)))]


def _fwd(p, x=AT + (1 << 20), ldx=64, f=AT + (1 << 21), ldf=64, xo=AT + (1 << 22), ldxo=64, h=AT + (1 << 23), ldh=64, hq=None, stats=AT + (1 << 24), xc=None, fc=None, mode=0):
    return mx.lib().mxfp4_residual_norm_fwd(C.byref(p) if p is not None else None, x, ldx, f, ldf, xo, ldxo, h, ldh, C.byref(hq) if hq is not None else None, stats,
                                            xc or b._NO_CKPT, fc or b._NO_CKPT, mode, None, None)


@pytest.mark.parametrize("want,kw", PLANS)
def test_plans(want, kw):
    p = plan(**kw)
    assert _fwd(p) == want
    assert _bwd(p) == want


@pytest.mark.parametrize("want,kw", [
    (INVALID, dict(p=None)), (INVALID, dict(x=None)), (INVALID, dict(f=None)), (INVALID, dict(p=plan(pre=NONE))), (INVALID, dict(xo=None, h=None)), (INVALID, dict(mode=9)),
    (INVALID, dict(f=None, xo=None, p=plan(post=NONE, gate=None, gates=0, a=2.0))), (INVALID, dict(f=None, p=plan(post=NONE, gate=None, gates=0))),
    (SHAPE, dict(ldx=32)), (SHAPE, dict(ldh=0)), (SHAPE, dict(xc=ckpt(rows=5))), (SHAPE, dict(fc=ckpt(cols=96))), (INVALID, dict(xc=ckpt(scales=None))),
    (MISALIGNED, dict(x=AT + 8)), (MISALIGNED, dict(ldf=68)), (MISALIGNED, dict(stats=AT + 2)), (MISALIGNED, dict(xc=ckpt(codes=AT + 4))),
    (SHAPE, dict(hq=b.CMat(AT, AT, 4, 96))), (INVALID, dict(hq=b.CMat(None, AT, 4, 64))), (MISALIGNED, dict(hq=b.CMat(AT, AT + 4, 4, 64))),
    (INVALID, dict(xo=AT + (1 << 20) + 16)), (INVALID, dict(h=AT + (1 << 21) + 128)), (INVALID, dict(h=AT + (1 << 22))),       # over an input elsewhere, over the other output
    (INVALID, dict(p=plan(x_dtype=1), xo=AT + (1 << 21)))])                                                                  # fp32 over bf16
def test_fwd(want, kw):
    a = dict(p=plan())
    a.update(kw)
    assert _fwd(**a) == want


def _bwd(p, ws=AT + (1 << 26), ws_bytes=1 << 20, null=False, **kw):
    m = dict(dh=AT + (1 << 20), lddh=64, dx_out=AT + (1 << 21), lddxo=64, stats=AT + (1 << 22), x_ckpt=ckpt(), f_ckpt=ckpt(codes=AT + (1 << 29)), x_out=None, ldxo=0, f=None,
             ldf=0, dx=AT + (1 << 23), lddx=64, df=AT + (1 << 24), lddf=64, dw_pre=AT + (1 << 25), db_pre=None, dw_post=None, db_post=None, dgate=None)
    m.update(kw)
    s = b.CResidualNormBwd(*[m[n] for n, _ in b.CResidualNormBwd._fields_])
    return mx.lib().mxfp4_residual_norm_bwd(C.byref(p), None if null else C.byref(s), ws, ws_bytes, None)


NO_GATE = dict(gate=None, gates=0)


@pytest.mark.parametrize("want,kw", [
    (INVALID, dict(null=True)), (INVALID, dict(dh=None)), (INVALID, dict(dx=None)), (INVALID, dict(stats=None)), (INVALID, dict(ws=None)),
    (INVALID, dict(p=plan(pre=NONE))), (INVALID, dict(p=plan(pre=NONE), dh=None)), (INVALID, dict(p=plan(pre=NONE), dh=None, dw_pre=None, dx_out=None)),
    (INVALID, dict(p=plan(post=NONE), dw_post=AT)), (INVALID, dict(p=plan(**NO_GATE), dgate=AT)), (INVALID, dict(p=plan(post=NONE, **NO_GATE), db_post=AT)),
    (INVALID, dict(f_ckpt=b._NO_CKPT)), (INVALID, dict(x_ckpt=b._NO_CKPT)), (INVALID, dict(x_ckpt=b._NO_CKPT, x_out=AT, ldxo=64)),      # one in 8 bits, one as it was
    (SHAPE, dict(lddh=32)), (SHAPE, dict(lddxo=63)), (SHAPE, dict(lddx=0)), (SHAPE, dict(lddf=8)), (SHAPE, dict(x_ckpt=ckpt(cols=96))), (SHAPE, dict(f_ckpt=ckpt(rows=3))),
    (MISALIGNED, dict(dh=AT + 2)), (MISALIGNED, dict(dw_pre=AT + 4)), (MISALIGNED, dict(ws=AT + 64)), (MISALIGNED, dict(stats=AT + 1)),
    (SMALL, dict(ws_bytes=64)),
    (INVALID, dict(df=AT + (1 << 23))), (INVALID, dict(dx=AT + (1 << 21) + 128)), (INVALID, dict(df=AT + (1 << 20) + 64)), (INVALID, dict(dx=AT + (1 << 30)))])
def test_bwd(want, kw):
    a = dict(p=plan())
    a.update(kw)
    assert _bwd(**a) == want


def test_workspace():
    assert mx.residual_norm_workspace_bytes(0, 64, 1) == 0 and mx.residual_norm_workspace_bytes(4, 0, 1) == 0 and mx.residual_norm_workspace_bytes(4, 1 << 20, 1) == 0
    assert mx.residual_norm_workspace_bytes(1000, 768, 10) > mx.residual_norm_workspace_bytes(1000, 768, 1) > 0
    assert _bwd(plan(), ws_bytes=mx.residual_norm_workspace_bytes(4, 64, 2) - 1) == SMALL
