"""The binding of the residual norms, activations and checkpoints on tensors of the CPU (the library refuses or returns before it touches them): what it
takes and what it refuses."""
import copy

import pytest
import torch

import paper_2502_20853_b200 as mx
from paper_2502_20853_b200 import binding, build

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def on_the_cpu(monkeypatch):
    build.build()
    monkeypatch.setattr(binding, "_device", lambda: -1)      # what a CPU tensor's get_device() says
    monkeypatch.setattr(binding, "_stream", lambda: 0)


@pytest.mark.parametrize("save", [mx.SAVE_NOTHING, mx.SAVE_8BIT, mx.SAVE_INPUTS])
@pytest.mark.parametrize("with_f", [False, True])
def test_no_rows(save, with_f):
    """Tensors without elements have no addresses of their own, which is no overlap."""
    x, f = torch.empty(0, 96, dtype=F32), torch.empty(0, 96, dtype=BF16)
    norm = mx.Norm(mx.NORM_LAYER, torch.ones(96), torch.zeros(96))
    x_out, h, ctx = mx.residual_norm_fwd(x, f if with_f else None, pre=norm, post=norm if with_f else None, gate=torch.ones(96) if with_f else None, save=save)
    assert h.shape == (0, 96) and (x_out is None) == (not with_f) and (ctx is None) == (save == mx.SAVE_NOTHING)


def _plan(rows=4):
    x, f = torch.zeros(rows, 96), torch.zeros(rows, 96, dtype=BF16)
    norm = mx.Norm(mx.NORM_LAYER, torch.ones(96), torch.zeros(96))
    return x, f, norm


@pytest.mark.parametrize("number", [0, 1, True, 1 << 40])
def test_numbers_are_not_addresses(number):
    """A number in a matrix's place is refused, not written to."""
    x, f, norm = _plan()
    for kw in (dict(x_out=number), dict(h=number)):
        with pytest.raises(AssertionError):
            mx.residual_norm_fwd(x, f, pre=norm, **kw)
    with pytest.raises((AssertionError, AttributeError, TypeError)):
        mx.residual_norm_fwd(x, number, pre=norm)
    ctx = mx.NormCtx(torch.zeros(4, 96), f, torch.zeros(4, 4), norm, norm)
    for args, kw in (((f, x), dict(df=number)), ((f, x), dict(dx=number)), ((f, number), dict(dx=x)), ((number, x), dict(df=f))):
        with pytest.raises((AssertionError, AttributeError, TypeError)):
            mx.residual_norm_bwd(*args, ctx, workspace=torch.empty(1 << 20, dtype=torch.uint8), **kw)
    for kept in ((number, f), (x, number)):
        with pytest.raises((AssertionError, AttributeError, TypeError)):
            mx.residual_norm_bwd(f, x, mx.NormCtx(*kept, torch.zeros(4, 4), norm, norm), workspace=torch.empty(1 << 20, dtype=torch.uint8))


def test_gate_without_rows():
    """[0, cols] is no gate at all, not one of 1."""
    x, f, norm = _plan()
    gate = torch.empty(0, 96)
    with pytest.raises(AssertionError, match="gate"):
        mx.residual_norm_fwd(x, f, pre=norm, gate=gate)
    ctx = mx.NormCtx(torch.zeros(4, 96), f, torch.zeros(4, 4), norm, norm, gate)
    with pytest.raises(AssertionError, match="gate"):
        mx.residual_norm_bwd(f, x, ctx, workspace=torch.empty(1 << 20, dtype=torch.uint8))
    x_out, _, _ = mx.residual_norm_fwd(x[:0], f[:0], pre=norm, gate=gate)
    assert x_out.shape == (0, 96)


class _Elsewhere:
    """A tensor that says that it is on another device than the call's."""

    def __init__(self, t):
        self.t, self.device = t, torch.device("cuda", 1)

    def get_device(self):
        return 1

    def __getattr__(self, name):
        return getattr(self.t, name)


def test_what_comes_beside_the_matrices_is_on_their_device():
    x, f, norm = _plan()
    status, work = _Elsewhere(torch.zeros(1, dtype=torch.int32)), torch.empty(1 << 20, dtype=torch.uint8)
    hq = mx.QMat(4, 96, "meta", torch.empty(4, 48, dtype=torch.uint8, device="meta"), torch.empty(512, dtype=torch.uint8, device="meta"))
    for kw in (dict(dev_status=status), dict(hq=hq)):
        with pytest.raises(AssertionError):
            mx.residual_norm_fwd(x, f, pre=norm, **kw)
    with pytest.raises(AssertionError):
        mx.act_fwd(f, dev_status=status)
    with pytest.raises(AssertionError):
        mx.checkpoint_store(x, dev_status=status)
    ctx = mx.NormCtx(torch.zeros(4, 96), f, torch.zeros(4, 4), norm, norm)
    for w in (_Elsewhere(work), work[::2]):
        with pytest.raises(AssertionError, match="workspace"):
            mx.residual_norm_bwd(f, x, ctx, workspace=w)


@pytest.mark.parametrize("rows,cols", [(1, 32), (3, 96), (257, 416), (0, 64)])
def test_checkpoint_in_one_buffer(rows, cols):
    """Codes and scales that the binding allocates: one behind the other, the same addresses whether the views have been made or not, in copies too."""
    for views in ("", "codes", "scales", "codes scales", "scales codes"):
        c = mx.Checkpoint.empty(rows, cols, "cpu")
        first = c._at((rows, cols), -1)
        for name in views.split():
            getattr(c, name)
        assert c._at((rows, cols), -1) == first and c.device == torch.device("cpu") and c.shape == (rows, cols)
        assert c.codes.shape == (rows, cols) and c.scales.shape == (rows, cols // 32) and c.codes.is_contiguous() and c.scales.is_contiguous()
        if rows:
            assert first == (c.codes.data_ptr(), c.scales.data_ptr()) and first[1] - first[0] == rows * cols
            c.codes.fill_(3), c.scales.fill_(5)
            assert bool((c._buf[:rows * cols] == 3).all()) and bool((c._buf[rows * cols:] == 5).all())
            d = copy.deepcopy(c)
            assert torch.equal(d.codes, c.codes) and torch.equal(d.scales, c.scales) and d._at((rows, cols), -1) == (d.codes.data_ptr(), d.scales.data_ptr())
            c.codes.zero_()
            assert bool((d.codes == 3).all())
        with pytest.raises(AssertionError):
            c._at((rows + 1, cols), -1)
        with pytest.raises(AssertionError):
            c._at((rows, cols), 0)


def test_gradients_in_one_buffer():
    for n in range(5):
        v = list(binding._vectors(n, 96, "cpu"))
        assert len(v) == n and all(t.shape == (96,) and t.dtype == F32 and t.is_contiguous() and t.data_ptr() % 16 == 0 for t in v)
        spans = sorted((t.data_ptr(), t.data_ptr() + 4 * 96) for t in v)
        assert all(a[1] <= b[0] for a, b in zip(spans, spans[1:]))
