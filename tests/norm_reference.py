"""Plain 64-bit forms of the operators around the linear layers (8-bit checkpoints, activations, residual addition between norms), on
torch tensors of any device.  Written from the definitions in the header; the tests hold the kernels to them."""
import math

import torch

D = torch.float64


def store(v, floor=False):
    """(codes as values, scale exponents) of an 8-bit checkpoint; groups that hold Inf / NaN: codes 0, exponent 128 (the byte 0xFF)."""
    rows, cols = v.shape
    v = v.to(D).reshape(rows, cols // 32, 32)
    bad = ~torch.isfinite(v).all(2)
    m = torch.where(bad[:, :, None], torch.zeros_like(v), v).abs().amax(2)
    m = torch.where(m == 0, torch.full_like(m, 1e-8), m)
    frac, e = torch.frexp(m)                                       # m = frac 2^e, frac in [1/2, 1)
    s = e - 1 - 8 + ((frac > 1.75 / 2).to(e.dtype) if not floor else 0)
    s = s.clamp(min=-127)
    w = torch.ldexp(torch.where(bad[:, :, None], torch.zeros_like(v), v), -s[:, :, None])
    _, we = torch.frexp(w)
    step = torch.ldexp(torch.ones_like(w), we.clamp(min=-5) - 4)   # E4M3: three bits behind the first, 2^-9 below 2^-6
    q = (torch.round(w / step) * step).clamp(-448, 448)            # torch.round: ties to even
    return q.reshape(rows, cols), torch.where(bad, torch.full_like(s, 128), s)


def load(codes, scales):
    """What codes and scale bytes (uint8 tensors) stand for."""
    rows, cols = codes.shape
    c = codes.view(torch.float8_e4m3fn).to(torch.float32).to(D).reshape(rows, cols // 32, 32)
    p = torch.ldexp(torch.ones_like(scales, dtype=D), scales.to(torch.int32) - 127)
    p = torch.where(scales == 255, torch.full_like(p, math.nan), p)
    return (c * p[:, :, None]).reshape(rows, cols)


def act(a, name):
    if name in ("gelu", "geglu"):
        return 0.5 * a * torch.special.erfc(-a / math.sqrt(2.0))
    return a / (1.0 + torch.exp(-a))


def act_slope(a, name):
    if name in ("gelu", "geglu"):
        return 0.5 * torch.special.erfc(-a / math.sqrt(2.0)) + a * torch.exp(-0.5 * a * a) / math.sqrt(2.0 * math.pi)
    p = 1.0 / (1.0 + torch.exp(-a))
    return p * (1.0 + a * torch.exp(-a) * p)


def act_fwd(y, name):
    if name in ("geglu", "swiglu"):
        a, b = y.chunk(2, 1)
        return act(a, name) * b
    return act(y, name)


def act_bwd(dz, y, name):
    if name in ("geglu", "swiglu"):
        a, b = y.chunk(2, 1)
        return torch.cat([dz * b * act_slope(a, name), dz * act(a, name)], 1)
    return dz * act_slope(y, name)


def stats(v, kind, eps):
    """mean (0 for an RMS norm) and 1 / deviation of every row, as columns"""
    mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    return mean, 1.0 / torch.sqrt((v - mean).square().mean(1, keepdim=True) + eps)


def gate_rows(gate, rows):
    return gate.to(D).repeat_interleave(rows // gate.shape[0], 0)


def norm_fwd(x, f, pre, post, gate, a, s, eps):
    """pre, post: None or (kind, weight, bias).  Returns a dict with x_out, h, x^, f^ and the statistics."""
    o = {}
    x = x.to(D)
    if f is not None:
        f = f.to(D)
        u = f
        if post is not None:
            o["post"] = mean, rstd = stats(f, post[0], eps)
            f = (f - mean) * rstd
            u = f * post[1].to(D) if post[1] is not None else f
            u = u + post[2].to(D) if post[2] is not None else u
        o["fh"], o["u"] = f, u
        x = a * x + s * (gate_rows(gate, x.shape[0]) * u if gate is not None else u)
    o["x_out"] = x
    if pre is not None:
        o["pre"] = mean, rstd = stats(x, pre[0], eps)
        x = (x - mean) * rstd
        o["xh"] = x
        h = x * pre[1].to(D) if pre[1] is not None else x
        o["h"] = h + pre[2].to(D) if pre[2] is not None else h
    return o


def norm_bwd(dh, dx_out, xh, fh, pre_rstd, post_rstd, pre, post, gate, a, s):
    """From the normalized rows (whatever they are worth) and the statistics: a dict of gradients, and under "abs_*" the same sums over
    magnitudes, which rounding errors are measured by."""
    o = {}
    given = dx_out if dx_out is not None else dh
    rows = given.shape[0]
    t = dx_out.to(D) if dx_out is not None else torch.zeros(given.shape, dtype=D, device=given.device)
    ta = t.abs()

    def back(d, da, v, rstd, kind):
        c1 = d.mean(1, keepdim=True) if kind == "layer" else 0.0
        r = rstd * (d - c1 - v * (d * v).mean(1, keepdim=True))
        ra = rstd * (da + (da.mean(1, keepdim=True) if kind == "layer" else 0.0) + v.abs() * (da * v.abs()).mean(1, keepdim=True))
        return r, ra

    if pre is not None:
        dh = dh.to(D)
        o["pre_weight"], o["abs_pre_weight"] = (dh * xh).sum(0), (dh * xh).abs().sum(0)
        o["pre_bias"], o["abs_pre_bias"] = dh.sum(0), dh.abs().sum(0)
        d = dh * pre[1].to(D) if pre[1] is not None else dh
        r, ra = back(d, d.abs(), xh, pre_rstd, pre[0])
        t, ta = t + r, ta + ra
    o["dx"], o["abs_dx"] = a * t, abs(a) * ta
    t, ta = s * t, abs(s) * ta
    if gate is not None:
        u = fh
        ua = fh.abs()
        if post is not None:
            w = post[1].to(D) if post[1] is not None else torch.ones_like(fh[0])
            b = post[2].to(D) if post[2] is not None else torch.zeros_like(fh[0])
            u, ua = fh * w + b, fh.abs() * w.abs() + b.abs()
        n = gate.shape[0]
        o["gate"], o["abs_gate"] = (t * u).reshape(n, rows // n, -1).sum(1), (ta * ua).reshape(n, rows // n, -1).sum(1)
        g = gate_rows(gate, rows)
        t, ta = t * g, ta * g.abs()
    if post is not None:
        o["post_weight"], o["abs_post_weight"] = (t * fh).sum(0), (ta * fh.abs()).sum(0)
        o["post_bias"], o["abs_post_bias"] = t.sum(0), ta.sum(0)
        if post[1] is not None:
            t, ta = t * post[1].to(D), ta * post[1].to(D).abs()
        t, ta = back(t, ta, fh, post_rstd, post[0])
    o["df"], o["abs_df"] = t, ta
    return o
