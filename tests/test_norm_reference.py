"""The 64-bit reference of the norms and activations: its gradients against central differences, its 8-bit rounding against torch's
conversion."""
import itertools

import pytest
import torch

import norm_reference as R


def _rand(*shape, seed=0):
    return torch.randn(*shape, dtype=torch.float64, generator=torch.Generator().manual_seed(seed))


def _difference(f, v, dv, step=1e-5):
    return (f(v + step * dv) - f(v - step * dv)) / (2 * step)


@pytest.mark.parametrize("pre,post,gates", list(itertools.product([None, "layer", "rms"], [None, "layer", "rms"], [0, 1, 3])))
def test_gradients_against_differences(pre, post, gates):
    rows, cols, a, s, eps = 6, 32, 0.7, 1.3, 1e-3
    v = {"x": _rand(rows, cols, seed=1), "f": _rand(rows, cols, seed=2), "pre_w": 1 + 0.3 * _rand(cols, seed=3), "pre_b": _rand(cols, seed=4),
         "post_w": 1 + 0.3 * _rand(cols, seed=5), "post_b": _rand(cols, seed=6), "gate": _rand(max(gates, 1), cols, seed=7)}
    dh, dxo = _rand(rows, cols, seed=8), _rand(rows, cols, seed=9)

    def run(p):
        return R.norm_fwd(p["x"], p["f"], (pre, p["pre_w"], p["pre_b"]) if pre else None, (post, p["post_w"], p["post_b"]) if post else None,
                          p["gate"] if gates else None, a, s, eps)

    def loss(p):
        o = run(p)
        return float((o["x_out"] * dxo).sum() + ((o["h"] * dh).sum() if pre else 0.0))

    o = run(v)
    g = R.norm_bwd(dh if pre else None, dxo, o.get("xh"), o["fh"], o["pre"][1] if pre else None, o["post"][1] if post else None,
                   (pre, v["pre_w"], v["pre_b"]) if pre else None, (post, v["post_w"], v["post_b"]) if post else None, v["gate"] if gates else None, a, s)
    names = {"x": "dx", "f": "df", "pre_w": "pre_weight", "pre_b": "pre_bias", "post_w": "post_weight", "post_b": "post_bias", "gate": "gate"}
    for k, name in names.items():
        if name not in g:
            continue
        dv = _rand(*v[k].shape, seed=20)
        want = _difference(lambda z, k=k: loss({**v, k: z}), v[k], dv)
        # second differences of order 1e-10 and the loss's own rounding over the step
        assert abs(float((g[name] * dv).sum()) - want) <= 1e-6 * (1 + abs(want)), name


@pytest.mark.parametrize("name", ["gelu", "silu", "geglu", "swiglu"])
def test_activation_gradients_against_differences(name):
    y, dz = 2 * _rand(5, 64, seed=1), _rand(5, 64 if name in ("gelu", "silu") else 32, seed=2)
    g = R.act_bwd(dz, y, name)
    dv = _rand(5, 64, seed=3)
    want = _difference(lambda t: float((R.act_fwd(t, name) * dz).sum()), y, dv)
    assert abs(float((g * dv).sum()) - want) <= 1e-6 * (1 + abs(want))


@pytest.mark.parametrize("floor", [False, True])
def test_8_bit_rounding_against_torch(floor):
    v = torch.randn(200, 96, generator=torch.Generator().manual_seed(5)) * torch.logspace(-30, 30, 200)[:, None]
    q, s = R.store(v, floor)
    w = torch.ldexp(v.double().reshape(200, 3, 32), -s[:, :, None]).reshape(200, 96).clamp(-448, 448)
    assert torch.equal(q, w.float().to(torch.float8_e4m3fn).double())
    m = v.double().abs().reshape(200, 3, 32).amax(2)
    top = torch.ldexp(m, -s)
    assert bool((top <= (448 if not floor else 511.9999)).all()) and bool((top > (224 if not floor else 255.9999)).all())
