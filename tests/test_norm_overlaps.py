"""Calls whose outputs lie over what they read, or over each other, are refused before anything is enqueued: through the C ABI with made-up addresses and
without a GPU.  Whatever lies right behind something else is not refused for that: those calls get as far as the launch."""
import ctypes as C

import pytest

import paper_2502_20853_b200 as mx
from paper_2502_20853_b200 import binding as b

INVALID, LAUNCHED = 1, 6     # (there is no GPU: the launch fails)
ROWS, COLS = 4, 64
MATRIX = ROWS * COLS * 2     # bytes of bf16
CODES, SCALES = ROWS * COLS, ROWS * COLS // 32
AT = 1 << 40


@pytest.fixture(scope="module", autouse=True)
def no_gpu():
    import torch
    if torch.cuda.is_available():
        pytest.skip("the addresses are made up: nothing may be launched")


class Arena:
    """Pieces of memory one right behind the other, each on 256 bytes."""

    def __init__(self, sizes):
        self.at, self.size, p = {}, dict(sizes), AT
        for name, n in sizes.items():
            self.at[name] = p
            p += (n + 255) // 256 * 256

    def over(self, a, name):
        """The same pieces with `a` moved: its last 16 bytes over the first of `name`, then its first over the last of it."""
        for p in (self.at[name] - max(self.size[a] - 16, 0) // 256 * 256, self.at[name] + (self.size[name] - 1) // 256 * 256):
            yield dict(self.at, **{a: p})


def pairs(written, read, allowed=()):
    return [(w, o) for k, w in enumerate(written) for o in written[:k] + read if (w, o) not in allowed]


def ckpt(m, which):
    return b.CCkpt(m[which + "_codes"], m[which + "_scales"], ROWS, COLS)


A_CKPT = Arena(dict(x=MATRIX, c_codes=CODES, c_scales=SCALES))


def store(m):
    return mx.lib().mxfp4_checkpoint_store(m["x"], 0, COLS, ckpt(m, "c"), 0, None, None)


def load(m):
    return mx.lib().mxfp4_checkpoint_load(ckpt(m, "c"), m["x"], 0, COLS, None)


@pytest.mark.parametrize("call,over", [(store, pairs(["c_codes", "c_scales"], ["x"])), (load, pairs(["x"], ["c_codes", "c_scales"]))])
def test_checkpoint(call, over):
    assert call(A_CKPT.at) == LAUNCHED
    for a, name in over:
        for m in A_CKPT.over(a, name):
            assert call(m) == INVALID, (a, name)


A_ACT = Arena(dict(y=MATRIX, z=MATRIX, c_codes=CODES, c_scales=SCALES))


def act_fwd(m, z=True):
    return mx.lib().mxfp4_act_fwd(m["y"], COLS, ROWS, COLS, 0, m["z"] if z else None, COLS, ckpt(m, "c"), 0, None, None)


def act_bwd(m):
    return mx.lib().mxfp4_act_bwd(m["y"], COLS, ckpt(m, "c"), 0, m["z"], COLS, None)


def test_activations():
    for call, over in ((act_fwd, pairs(["z", "c_codes", "c_scales"], ["y"], [("z", "y")])), (lambda m: act_fwd(m, False), pairs(["c_codes", "c_scales"], ["y"])),
                       (act_bwd, pairs(["z"], ["c_codes", "c_scales"]))):
        assert call(A_ACT.at) == LAUNCHED
        for a, name in over:
            for m in A_ACT.over(a, name):
                assert call(m) == INVALID, (a, name)
    for call in (act_fwd, act_bwd):      # in place
        assert call(dict(A_ACT.at, z=A_ACT.at["y"])) == LAUNCHED


VECTOR = COLS * 4
A_FWD = Arena(dict(x=MATRIX, f=MATRIX, xo=MATRIX, h=MATRIX, x_codes=CODES, x_scales=SCALES, f_codes=CODES, f_scales=SCALES, q=ROWS * COLS // 2, qs=512, stats=16 * ROWS,
                   pw=VECTOR, pb=VECTOR, qw=VECTOR, qb=VECTOR, gate=2 * COLS * 2))


def plan(m):
    return b.CResidualNorm(ROWS, COLS, 0, 0, 1.0, 1.0, b.CNorm(1, 1, m["pw"], m["pb"], 1e-6, 0), b.CNorm(2, 1, m["qw"], m["qb"], 1e-6, 0), m["gate"], 2, COLS)


def norm_fwd(m):
    hq = b.CMat(m["q"], m["qs"], ROWS, COLS)
    return mx.lib().mxfp4_residual_norm_fwd(C.byref(plan(m)), m["x"], COLS, m["f"], COLS, m["xo"], COLS, m["h"], COLS, C.byref(hq), m["stats"], ckpt(m, "x"), ckpt(m, "f"), 0,
                                            None, None)


def test_norm_forward():
    assert norm_fwd(A_FWD.at) == LAUNCHED
    written = ["xo", "h", "x_codes", "x_scales", "f_codes", "f_scales", "q", "qs", "stats"]
    for a, name in pairs(written, ["x", "f", "pw", "pb", "qw", "qb", "gate"], [("xo", "x"), ("xo", "f"), ("h", "x"), ("h", "f")]):
        for m in A_FWD.over(a, name):
            assert norm_fwd(m) == INVALID, (a, name)
    for over in (dict(xo="x"), dict(h="f"), dict(xo="x", h="f"), dict(xo="f", h="x")):      # in place
        assert norm_fwd(dict(A_FWD.at, **{k: A_FWD.at[v] for k, v in over.items()})) == LAUNCHED


WORK = mx.residual_norm_workspace_bytes(ROWS, COLS, 2)
A_BWD = Arena(dict(dh=MATRIX, dxo=MATRIX, dx=MATRIX, df=MATRIX, stats=16 * ROWS, x_codes=CODES, x_scales=SCALES, f_codes=CODES, f_scales=SCALES, x=MATRIX, f=MATRIX, gpw=VECTOR,
                   gpb=VECTOR, gqw=VECTOR, gqb=VECTOR, gg=2 * VECTOR, work=WORK, pw=VECTOR, pb=VECTOR, qw=VECTOR, qb=VECTOR, gate=2 * COLS * 2))


def norm_bwd(m, eight=True):
    none = b.CCkpt(None, None, 0, 0)
    k = dict(dh=m["dh"], lddh=COLS, dx_out=m["dxo"], lddxo=COLS, stats=m["stats"], x_ckpt=ckpt(m, "x") if eight else none, f_ckpt=ckpt(m, "f") if eight else none,
             x_out=None if eight else m["x"], ldxo=COLS, f=None if eight else m["f"], ldf=COLS, dx=m["dx"], lddx=COLS, df=m["df"], lddf=COLS, dw_pre=m["gpw"], db_pre=m["gpb"],
             dw_post=m["gqw"], db_post=m["gqb"], dgate=m["gg"])
    s = b.CResidualNormBwd(*[k[n] for n, _ in b.CResidualNormBwd._fields_])
    return mx.lib().mxfp4_residual_norm_bwd(C.byref(plan(m)), C.byref(s), m["work"], WORK, None)


@pytest.mark.parametrize("eight", [True, False])
def test_norm_backward(eight):
    assert norm_bwd(A_BWD.at, eight) == LAUNCHED
    kept = ["x_codes", "x_scales", "f_codes", "f_scales"] if eight else ["x", "f"]
    for a, name in pairs(["dx", "df", "gpw", "gpb", "gqw", "gqb", "gg", "work"], ["dh", "dxo", "stats", "pw", "pb", "qw", "qb", "gate"] + kept,
                         [("dx", "dh"), ("dx", "dxo"), ("df", "dh"), ("df", "dxo")]):
        for m in A_BWD.over(a, name):
            assert norm_bwd(m, eight) == INVALID, (a, name)
    for over in (dict(dx="dxo"), dict(df="dh"), dict(dx="dxo", df="dh"), dict(dx="dh", df="dxo")):      # in place
        assert norm_bwd(dict(A_BWD.at, **{k: A_BWD.at[v] for k, v in over.items()}), eight) == LAUNCHED
