"""The operators around the quantized linear layers of a transformer block, as cases to be timed: sizes, inputs, one pass, what it cannot do
without, and what it returns by its definition in 64 bits.

  norm_fwd   the end of one branch and the start of the next: u = N_post(f), x' = a x + s g u, h = N_pre(x'), and what the backward pass
             keeps: the normalized rows as 8-bit checkpoints (or nothing but the statistics), 1 / deviation and mean of each row
  norm_bwd   the gradients of all of that: dx, df, of the norms' weights and biases, of the gate
  act_fwd    z = act(y) or act(y_a) y_b, and y as an 8-bit checkpoint
  act_bwd    dy from dz and the checkpoint
  store      a tensor into an 8-bit checkpoint: E4M3 codes and one power of two for each 32 columns
  load       and back

Where `own` is false a pass is elementary torch operations in 32 bits; where it is true it is the library's calls.
"""
import math

import torch

own = False

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
OUTLIER_CHANNELS, OUTLIER_GAIN = 4, 20.0     # activations: a few channels much larger than the rest
EPS = 1e-6
CKPT = 1.0 + 1.0 / 32.0                      # bytes of a checkpointed element: its code and its share of a scale


def _norm(name, op, rows, cols, pre, post, gates, bias=True, fp32=False, eight=True, param32=True, res=1.0, branch=1.0):
    """pre, post: "layer", "rms" or "none"; gates: 0 (none), 1 (one for all rows: a layer scale) or how many runs of rows have one each."""
    return dict(name=name, op=op, rows=rows, cols=cols, pre=pre, post=post, gates=gates, bias=bias, fp32=fp32, eight=eight, param32=param32, res=res, branch=branch)


def listed():
    return [
        # one new token of a decoder with 4096 channels: residual addition and the next block's norm, nothing kept
        _norm("norm_fwd_token", "norm_fwd", 1, 4096, "rms", "none", 0, bias=False, eight=False, param32=False),
        # DeiT-Small at batch 128 x 197 tokens, training: layer scale, residual, LayerNorm
        _norm("norm_fwd_deit_small", "norm_fwd", 25216, 384, "layer", "none", 1),
        # ViT-Large at batch 256 x 197 tokens, training: norms on both sides of the branch, a gate for each image, the residual in fp32
        _norm("norm_fwd_vit_large_both", "norm_fwd", 50432, 1024, "rms", "rms", 256, bias=False, fp32=True),
        # fine-tuning on single images of 197 tokens: a small backward pass, from the inputs themselves
        _norm("norm_bwd_image", "norm_bwd", 197, 384, "layer", "none", 1, eight=False),
        # Swin-T's last stage at batch 128 x 49 tokens with norms on both sides and a gate for each image
        _norm("norm_bwd_swin_stage4_both", "norm_bwd", 6272, 768, "layer", "layer", 128, param32=False, res=0.8, branch=1.25),
        # ViT-Large as above
        _norm("norm_bwd_vit_large_both", "norm_bwd", 50432, 1024, "rms", "rms", 256, bias=False, fp32=True),
        # one image through DeiT-Small's MLP
        dict(name="act_fwd_image", op="act_fwd", rows=197, cols=1536, act="gelu"),
        # ViT-Large's MLP at batch 256 x 197, the largest activations
        dict(name="act_fwd_vit_large", op="act_fwd", rows=50432, cols=4096, act="gelu"),
        # DeiT-Small's MLP, backward
        dict(name="act_bwd_deit_small", op="act_bwd", rows=25216, cols=1536, act="gelu"),
        # a gated MLP on a ragged batch of tokens (the feature count is a multiple of 32 and of nothing larger)
        dict(name="act_bwd_swiglu", op="act_bwd", rows=6311, cols=2336, act="swiglu"),
        # any other activation kept for the backward pass: attention's output of DeiT-Base at batch 256 x 197
        dict(name="store_deit_base", op="store", rows=50432, cols=768, fp32=False),
        # and taken out again, for a small model
        dict(name="load_deit_tiny", op="load", rows=1576, cols=192, fp32=False),
    ]


def _log(rng, lo, hi, step=1):
    """A multiple of `step` between lo and hi, spread over the logarithm."""
    return max(step, int(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step + 0.5) * step)


def draw(rng):
    op = rng.choice(["norm_fwd", "norm_bwd", "norm_fwd", "norm_bwd", "act_fwd", "act_bwd", "store", "load"])
    if op in ("norm_fwd", "norm_bwd"):
        cols = _log(rng, 64, 8192, 32)
        rows = _log(rng, 1, min(50432, 48e6 / cols))
        gates = rng.choice([0, 1, 1, 2])
        if gates == 2:      # a gate for each sequence, which are of one length
            tokens = min(rows, _log(rng, 16, 1024))
            gates, rows = rows // tokens, rows // tokens * tokens
        return dict(op=op, rows=rows, cols=cols, pre=rng.choice(["layer", "rms", "layer", "rms", "none"]), post=rng.choice(["layer", "rms", "none", "none"]), gates=gates,
                    bias=rng.random() < 0.5, fp32=rng.random() < 0.4, eight=rng.random() < 0.7, param32=rng.random() < 0.5, res=rng.choice([1.0, 1.0, 0.7]),
                    branch=rng.choice([1.0, 1.0, 0.5]))
    cols = _log(rng, 32, 8192, 32)
    rows = _log(rng, 1, min(50432, 96e6 / cols))
    if op in ("act_fwd", "act_bwd"):
        return dict(op=op, rows=rows, cols=cols, act=rng.choice(["gelu", "gelu", "silu", "geglu", "swiglu"]))
    return dict(op=op, rows=rows, cols=cols, fp32=rng.random() < 0.4)


# ---- inputs ------------------------------------------------------------------------------------------------------------------------------

def _activations(g, rows, cols, dtype=BF16, std=1.0):
    x = torch.randn(rows, cols, device="cuda", generator=g) * std
    at = torch.randperm(cols, device="cuda", generator=g)[:OUTLIER_CHANNELS]
    x[:, at] *= OUTLIER_GAIN
    return x.to(dtype)


def _gradients(g, rows, cols, dtype=BF16):
    """Heavy-tailed and small: normal over the root of a mean of three squares."""
    z = torch.randn(rows, cols, device="cuda", generator=g)
    c = torch.zeros_like(z)
    for _ in range(3):
        c += torch.randn(rows, cols, device="cuda", generator=g).square()
    return (z / torch.sqrt(c / 3.0) * 1e-3).to(dtype)


def _affine(g, case, kind):
    if kind == "none":
        return None, None
    dt = F32 if case["param32"] else BF16
    w = (1.0 + 0.2 * torch.randn(case["cols"], device="cuda", generator=g)).to(dt)
    return w, (0.1 * torch.randn(case["cols"], device="cuda", generator=g)).to(dt) if case["bias"] and kind == "layer" else None


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, rows, cols = case["op"], case["rows"], case["cols"]
    s = dict(case)
    if op in ("norm_fwd", "norm_bwd"):
        dt = F32 if case["fp32"] else BF16
        s["x"], s["f"] = _activations(g, rows, cols, dt), _activations(g, rows, cols, BF16, 0.5)
        s["pre_w"], s["pre_b"] = _affine(g, case, case["pre"])
        s["post_w"], s["post_b"] = _affine(g, case, case["post"])
        s["gate"] = None
        if case["gates"] == 1:       # a layer scale is a parameter
            s["gate"] = (0.1 + 0.05 * torch.randn(1, cols, device="cuda", generator=g)).to(F32 if case["param32"] else BF16)
        elif case["gates"]:          # one of the parts of what a small projection gave for each sequence
            s["gate"] = (0.5 * torch.randn(case["gates"], 2 * cols, device="cuda", generator=g)).to(BF16)[:, cols:]
        if op == "norm_bwd":
            # what the forward pass has kept, and the gradients that come back
            f = _norm_forward(s)
            s["dh"] = _gradients(g, rows, cols) if case["pre"] != "none" else None
            s["dx_out"] = _gradients(g, rows, cols, dt)
            s["stats"] = torch.stack([f[k].reshape(-1) if f[k] is not None else torch.zeros(rows, device="cuda") for k in ("pre_mean", "pre_rstd", "post_mean", "post_rstd")])
            for k in ("x", "f"):
                s[k + "_codes"], s[k + "_scales"] = (f[k + "_codes"], f[k + "_scales"]) if case["eight"] else (None, None)
            s["x_out"] = f["x_out"] if not case["eight"] else None
            s["x"] = None
            if case["eight"]:
                s["f"] = None
    elif op == "act_fwd":
        s["y"] = _activations(g, rows, cols * _halves(case))
    elif op == "act_bwd":
        s["dz"] = _gradients(g, rows, cols)
        s["codes"], s["scales"] = _store(_activations(g, rows, cols * _halves(case)).float())
    else:
        x = _activations(g, rows, cols, F32 if case["fp32"] else BF16)
        if op == "store":
            s["x"] = x
        else:
            s["codes"], s["scales"] = _store(x.float())
    return s


def _halves(case):
    return 2 if case["act"] in ("geglu", "swiglu") else 1


# ---- the plain form ----------------------------------------------------------------------------------------------------------------------

def _store(v):
    """Codes and scales of a checkpoint: 2^s, s = ceil(log2(M / 448)), M the largest magnitude of 32 columns (1e-8 if that is 0)."""
    rows, cols = v.shape
    v = v.reshape(rows, cols // 32, 32)
    m = v.abs().amax(2, keepdim=True)
    frac, e = torch.frexp(torch.where(m == 0, torch.full_like(m, 1e-8), m))
    s = (e - 9 + (frac > 0.875).to(torch.int32)).clamp(min=-127)
    codes = torch.ldexp(v, -s).to(torch.float8_e4m3fn)
    return codes.reshape(rows, cols), (s.reshape(rows, cols // 32) + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _load(codes, scales, dtype=F32):
    rows, cols = codes.shape
    return (codes.to(dtype).reshape(rows, cols // 32, 32) * scales.to(dtype).reshape(rows, cols // 32, 1)).reshape(rows, cols)


def _normalized(v, kind):
    mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    rstd = torch.rsqrt((v - mean).square().mean(1, keepdim=True) + EPS)
    return (v - mean) * rstd, mean, rstd


def _times(v, w, b):
    return v * w.float() + b.float() if b is not None else v * w.float()


def _rows_of_gate(s, rows):
    return s["gate"].float().repeat_interleave(rows // s["gates"], 0)


def _norm_forward(s):
    """All that the forward pass gives, in 32 bits, rounded at the end."""
    x, f = s["x"].float(), s["f"].float()
    o = dict.fromkeys(("h", "pre_mean", "pre_rstd", "post_mean", "post_rstd", "x_codes", "x_scales", "f_codes", "f_scales"))
    u = f
    if s["post"] != "none":
        f, o["post_mean"], o["post_rstd"] = _normalized(f, s["post"])
        u = _times(f, s["post_w"], s["post_b"])
    g = _rows_of_gate(s, x.shape[0]) if s["gates"] else 1.0
    x = s["res"] * x + s["branch"] * g * u
    o["x_out"] = x.to(s["x"].dtype)
    if s["eight"] and (s["post"] != "none" or s["gates"]):
        o["f_codes"], o["f_scales"] = _store(f)
    if s["pre"] != "none":
        x, o["pre_mean"], o["pre_rstd"] = _normalized(x, s["pre"])
        o["h"] = _times(x, s["pre_w"], s["pre_b"]).to(BF16)
        if s["eight"]:
            o["x_codes"], o["x_scales"] = _store(x)
    return o


def _norm_fwd(s):
    o = _norm_forward(s)
    return [o["x_out"], o["h"]] + ([o[k] for k in ("x_codes", "x_scales", "f_codes", "f_scales")] + [o["pre_rstd"], o["post_rstd"]] if s["eight"] else [])


def _norm_rows_back(dv, v, rstd, kind):
    c1 = dv.mean(1, keepdim=True) if kind == "layer" else 0.0
    return rstd * (dv - c1 - v * (dv * v).mean(1, keepdim=True))


def _norm_bwd(s):
    st = [v.reshape(-1, 1) for v in s["stats"]]
    t, rows = s["dx_out"].float(), s["dx_out"].shape[0]
    o = dict.fromkeys(("df", "pre_w", "pre_b", "post_w", "post_b", "gate"))
    if s["pre"] != "none":
        v = _load(s["x_codes"], s["x_scales"]) if s["eight"] else (s["x_out"].float() - st[0]) * st[1]
        dh = s["dh"].float()
        o["pre_w"] = (dh * v).sum(0)
        o["pre_b"] = dh.sum(0) if s["pre_b"] is not None else None
        t = t + _norm_rows_back(dh * s["pre_w"].float(), v, st[1], s["pre"])
    o["dx"] = (s["res"] * t).to(s["dx_out"].dtype)
    t = s["branch"] * t
    f = None
    if s["post"] != "none" or s["gates"]:
        f = _load(s["f_codes"], s["f_scales"]) if s["eight"] else s["f"].float()
        if s["post"] != "none" and not s["eight"]:
            f = (f - st[2]) * st[3]
    u = _times(f, s["post_w"], s["post_b"]) if s["post"] != "none" else f
    if s["gates"]:
        o["gate"] = (t * u).reshape(s["gates"], rows // s["gates"], -1).sum(1)
        t = t * _rows_of_gate(s, rows)
    if s["post"] != "none":
        o["post_w"] = (t * f).sum(0)
        o["post_b"] = t.sum(0) if s["post_b"] is not None else None
        t = _norm_rows_back(t * s["post_w"].float(), f, st[3], s["post"])
    o["df"] = t.to(BF16)
    return o


def _act(a, act):
    return 0.5 * a * torch.special.erfc(a * -math.sqrt(0.5)) if act in ("gelu", "geglu") else a * torch.sigmoid(a)


def _act_slope(a, act):
    if act in ("gelu", "geglu"):
        return 0.5 * torch.special.erfc(a * -math.sqrt(0.5)) + a * torch.exp(-0.5 * a * a) * (1.0 / math.sqrt(2.0 * math.pi))
    p = torch.sigmoid(a)
    return p * (1.0 + a * (1.0 - p))


def _act_fwd(s):
    y = s["y"].float()
    a, b = y.chunk(2, 1) if _halves(s) == 2 else (y, None)
    z = _act(a, s["act"])
    return [(z * b if b is not None else z).to(BF16), *_store(y)]


def _act_bwd(s):
    y, dz = _load(s["codes"], s["scales"]), s["dz"].float()
    if _halves(s) == 1:
        return (dz * _act_slope(y, s["act"])).to(BF16)
    a, b = y.chunk(2, 1)
    return torch.cat([dz * b * _act_slope(a, s["act"]), dz * _act(a, s["act"])], 1).to(BF16)


# ---- one pass ----------------------------------------------------------------------------------------------------------------------------

def run(state):
    op = state["op"]
    if own:
        return _own(state, op)
    if op == "norm_fwd":
        return _norm_fwd(state)
    if op == "norm_bwd":
        return _norm_bwd(state)
    if op == "act_fwd":
        return _act_fwd(state)
    if op == "act_bwd":
        return _act_bwd(state)
    if op == "store":
        return _store(state["x"].float())
    return _load(state["codes"], state["scales"]).to(F32 if state["fp32"] else BF16)


def _own(s, op):
    import paper_2502_20853_b200 as mx
    if op in ("norm_fwd", "norm_bwd"):
        kinds = {"layer": mx.NORM_LAYER, "rms": mx.NORM_RMS}
        pre = mx.Norm(kinds[s["pre"]], s["pre_w"], s["pre_b"], EPS) if s["pre"] != "none" else None
        post = mx.Norm(kinds[s["post"]], s["post_w"], s["post_b"], EPS) if s["post"] != "none" else None
        if op == "norm_fwd":
            x_out, h, ctx = mx.residual_norm_fwd(s["x"], s["f"], pre=pre, post=post, gate=s["gate"], residual_scale=s["res"], branch_scale=s["branch"],
                                                 save=mx.SAVE_8BIT if s["eight"] else mx.SAVE_NOTHING)
            if not s["eight"]:
                return [x_out, h]
            x, f = ctx.x, ctx.f
            return [x_out, h, x.codes.view(torch.float8_e4m3fn) if x is not None else None, x.scales.view(torch.float8_e8m0fnu) if x is not None else None,
                    f.codes.view(torch.float8_e4m3fn) if f is not None else None, f.scales.view(torch.float8_e8m0fnu) if f is not None else None,
                    ctx.stats[1].view(-1, 1) if pre is not None else None, ctx.stats[3].view(-1, 1) if post is not None else None]
        x = _checkpoint(mx, s["x_codes"], s["x_scales"]) if s["eight"] else s["x_out"]
        f = _checkpoint(mx, s["f_codes"], s["f_scales"]) if s["eight"] else s["f"]
        ctx = mx.NormCtx(x, f, s["stats"], pre=pre, post=post, gate=s["gate"], residual_scale=s["res"], branch_scale=s["branch"])
        g = mx.residual_norm_bwd(s["dh"], s["dx_out"], ctx)
        return dict(dx=g.dx, df=g.df, pre_w=g.pre_weight, pre_b=g.pre_bias, post_w=g.post_weight, post_b=g.post_bias, gate=g.gate)
    if op in ("act_fwd", "act_bwd"):
        act = {"gelu": mx.ACT_GELU, "silu": mx.ACT_SILU, "geglu": mx.ACT_GEGLU, "swiglu": mx.ACT_SWIGLU}[s["act"]]
        if op == "act_bwd":
            return mx.act_bwd(s["dz"], _checkpoint(mx, s["codes"], s["scales"]), act)
        z, c = mx.act_fwd(s["y"], act)
    elif op == "store":
        z, c = None, mx.checkpoint_store(s["x"])
    else:
        return mx.checkpoint_load(_checkpoint(mx, s["codes"], s["scales"]), mx.OUT_FP32 if s["fp32"] else mx.OUT_BF16)
    out = (c.codes.view(torch.float8_e4m3fn), c.scales.view(torch.float8_e8m0fnu))
    return [z, *out] if z is not None else out


def _checkpoint(mx, codes, scales):
    return mx.Checkpoint(codes.view(torch.uint8), scales.view(torch.uint8)) if codes is not None else None


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------------------------

def work(case):
    op, n = case["op"], case["rows"] * case["cols"]
    if op in ("act_fwd", "act_bwd"):
        k = _halves(case)
        # forward: y in, z and y's checkpoint out; backward: dz and the checkpoint in, dy out
        return {"bytes": n * (2 * k + 2 + CKPT * k), "flops": n * (30.0 if op == "act_fwd" else 40.0)}
    if op in ("store", "load"):
        return {"bytes": n * (CKPT + (4 if case["fp32"] else 2)), "flops": n * 3.0}
    x = 4 if case["fp32"] else 2
    pre, post, gates = case["pre"] != "none", case["post"] != "none", case["gates"]
    par = 4 if case["param32"] else 2
    once = case["cols"] * (par * (pre + post) + (par * ((case["pre"] == "layer") + (case["post"] == "layer")) if case["bias"] else 0) + (par if gates == 1 else 2 * gates))
    keeps_f = post or bool(gates)
    if op == "norm_fwd":
        per = x + 2 + x + 2 * pre + (CKPT * (pre + keeps_f) if case["eight"] else 0)
        return {"bytes": n * per + once + 4 * case["rows"] * (pre + post if case["eight"] else 0), "flops": n * (4.0 + 9 * pre + 9 * post + (4 * (pre + keeps_f) if case["eight"] else 0))}
    saved = (CKPT * (pre + keeps_f)) if case["eight"] else x * pre + 2 * keeps_f
    stats = 4 * case["rows"] * (pre + post) * (1 if case["eight"] else 2)
    grads = 4 * case["cols"] * (pre + post + (((case["pre"] == "layer") + (case["post"] == "layer")) if case["bias"] else 0) + gates)
    return {"bytes": n * (2 * pre + x + saved + x + 2) + once + stats + grads, "flops": n * (4.0 + 14 * pre + 16 * post + 4 * bool(gates))}


# ---- by definition, in 64 bits -------------------------------------------------------------------------------------------------------------

def _x_store(v):
    rows, cols = v.shape
    v = v.reshape(rows, -1, 32)
    top = v.abs().max(2).values
    top[top == 0] = 1e-8
    power = torch.ceil(torch.log2(top / 448.0))
    power = torch.where(top > 448.0 * torch.exp2(power), power + 1, power)          # the logarithm's own rounding
    power = torch.where(top <= 448.0 * torch.exp2(power - 1), power - 1, power).clamp(min=-127)
    w = v * torch.exp2(-power)[:, :, None]
    step = torch.exp2(torch.floor(torch.log2(w.abs().clamp(min=2.0 ** -6) * (1 + 1e-15))).clamp(min=-6) - 3)
    return (torch.round(w / step) * step).reshape(rows, cols), torch.exp2(power)


def _x_load(s, k):
    c, p = s[k + "codes"].to(F32).double(), s[k + "scales"].to(F32).double()
    return c * p.repeat_interleave(32, 1)


def _x_stats(v, kind):
    n = v.shape[1]
    mean = v.sum(1) / n if kind == "layer" else v.new_zeros(v.shape[0])
    var = (v * v).sum(1) / n if kind == "rms" else ((v - mean[:, None]) ** 2).sum(1) / n
    return mean, (var + EPS) ** -0.5


def _x_norm_fwd(s):
    x, f = s["x"].double(), s["f"].double()
    rows = x.shape[0]
    post_rstd = pre_rstd = h = None
    u = f
    if s["post"] != "none":
        mean, post_rstd = _x_stats(f, s["post"])
        f = (f - mean[:, None]) * post_rstd[:, None]
        u = f * s["post_w"].double()
        if s["post_b"] is not None:
            u = u + s["post_b"].double()
    if s["gates"]:
        at = torch.arange(rows, device=x.device) // (rows // s["gates"])
        u = u * s["gate"].double()[at]
    x = x * s["res"] + u * s["branch"]
    out = [x]
    n = x
    if s["pre"] != "none":
        mean, pre_rstd = _x_stats(x, s["pre"])
        n = (x - mean[:, None]) * pre_rstd[:, None]
        h = n * s["pre_w"].double()
        if s["pre_b"] is not None:
            h = h + s["pre_b"].double()
    out.append(h)
    if s["eight"]:
        out += _x_store(n) if s["pre"] != "none" else (None, None)
        out += _x_store(f) if s["post"] != "none" or s["gates"] else (None, None)
        out += [pre_rstd[:, None] if pre_rstd is not None else None, post_rstd[:, None] if post_rstd is not None else None]
    return out


def _x_norm_bwd(s):
    # dL / dv of v -> (v - mean) * rstd, written with the centred gradient and its projection on the normalized row
    def back(d, v, rstd, kind):
        if kind == "layer":
            d = d - d.sum(1, keepdim=True) / d.shape[1]
        along = torch.einsum("rc,rc->r", d, v) / d.shape[1]
        return (d - along[:, None] * v) * rstd[:, None]

    pm, pr, qm, qr = s["stats"].double()
    d = s["dx_out"].double()
    rows, cols = d.shape
    o = dict.fromkeys(("df", "pre_w", "pre_b", "post_w", "post_b", "gate"))
    if s["pre"] != "none":
        v = _x_load(s, "x_") if s["eight"] else (s["x_out"].double() - pm[:, None]) * pr[:, None]
        dh = s["dh"].double()
        o["pre_w"] = torch.einsum("rc,rc->c", dh, v)
        if s["pre_b"] is not None:
            o["pre_b"] = dh.sum(0)
        dn = dh * s["pre_w"].double()
        if s["pre"] == "rms":
            d = d + back(dn, v, pr, "rms")
        else:       # v of a checkpoint need not be centred: the two means are taken apart
            d = d + pr[:, None] * (dn - dn.mean(1, keepdim=True) - v * (dn * v).mean(1, keepdim=True))
    o["dx"] = d * s["res"]
    d = d * s["branch"]
    if s["gates"] or s["post"] != "none":
        f = _x_load(s, "f_") if s["eight"] else s["f"].double()
        if s["post"] != "none" and not s["eight"]:
            f = (f - qm[:, None]) * qr[:, None]
        u = f if s["post"] == "none" else f * s["post_w"].double() + (s["post_b"].double() if s["post_b"] is not None else 0.0)
    if s["gates"]:
        at = torch.arange(rows, device=d.device) // (rows // s["gates"])
        o["gate"] = torch.zeros(s["gates"], cols, dtype=F64, device=d.device).index_add_(0, at, d * u)
        d = d * s["gate"].double()[at]
    if s["post"] != "none":
        o["post_w"] = torch.einsum("rc,rc->c", d, f)
        if s["post_b"] is not None:
            o["post_b"] = d.sum(0)
        dn = d * s["post_w"].double()
        if s["post"] == "rms":
            d = back(dn, f, qr, "rms")
        else:
            d = qr[:, None] * (dn - dn.mean(1, keepdim=True) - f * (dn * f).mean(1, keepdim=True))
    o["df"] = d
    return o


def _x_act(a, act):
    return a * torch.special.ndtr(a) if act in ("gelu", "geglu") else a / (1.0 + torch.exp(-a))


def _x_slope(a, act):
    if act in ("gelu", "geglu"):
        return torch.special.ndtr(a) + a * torch.exp(-a * a / 2.0) / (2.0 * math.pi) ** 0.5
    e = torch.exp(-a.abs())         # the same on both sides of zero but for the sign of what is behind the 1/2
    q = 1.0 / (1.0 + e)
    p = torch.where(a >= 0, q, e * q)
    return p + a * e * q * q


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "norm_fwd":
        return _x_norm_fwd(s)
    if op == "norm_bwd":
        return _x_norm_bwd(s)
    if op == "store":
        return _x_store(s["x"].double())
    if op == "load":
        return _x_load(s, "")
    act, n = case["act"], case["cols"]
    if op == "act_fwd":
        y = s["y"].double()
        z = _x_act(y[:, :n], act)
        return [z if _halves(case) == 1 else z * y[:, n:], *_x_store(y)]
    y, dz = _x_load(s, ""), s["dz"].double()
    if _halves(case) == 1:
        return dz * _x_slope(y, act)
    return torch.cat([dz * y[:, n:] * _x_slope(y[:, :n], act), dz * _x_act(y[:, :n], act)], 1)
