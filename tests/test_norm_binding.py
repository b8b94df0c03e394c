"""The binding of the residual norms, activations and checkpoints on tensors of the CPU (the library refuses or returns before it touches them): what it
takes and what it refuses."""
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
