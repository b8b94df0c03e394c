"""8-bit activation checkpoints and the activations that write and read them, against the 64-bit reference.

Tolerances.  Codes and scales of a checkpoint are exact.  A bf16 result is off by half a step, 2^-8 of its value, and by what its FP32
computation is off:
  GELU    1.1e-7 |y| (the fit of the tail), 2^-24 for each of the three roundings behind it: 2^-21 |y| in all
  SiLU    the exponent y log2(e) is rounded twice (2^-23 |y| of e^-y), ex2 and rcp are good to 2^-22 and 2^-23: |y| 2^-23 + 2^-20 of the value
  slopes  of GELU: the tail's 1.1e-7 and y phi(y) with phi off by 2^-23 (y^2 + 4): 2^-19 in all (y^2 |y| phi(y) stays below 0.6);
          of SiLU: p (1 + y (1 - p)), p off by (|y| 2^-23 + 2^-20) of itself or, near 1, of 1 - p and 2^-23: (1 + |y|) 2^-19
A gated form multiplies once more (2^-24 of the value, inside the margins above).
"""
import math

import pytest
import torch

import norm_reference as R

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
NAMES = ["gelu", "silu", "geglu", "swiglu"]


@pytest.fixture(scope="module")
def mx():
    import paper_2502_20853_b200 as m
    m.lib()
    return m


def _act(mx, name):
    return {"gelu": mx.ACT_GELU, "silu": mx.ACT_SILU, "geglu": mx.ACT_GEGLU, "swiglu": mx.ACT_SWIGLU}[name]


def _values(rows, cols, dtype, seed=0, wide=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, cols, device="cuda", generator=g)
    if wide:        # groups of very different sizes, zeros among them
        x = x * torch.exp2(torch.randint(-40, 40, (rows, cols // 32, 1), device="cuda", generator=g).float()).expand(-1, -1, 32).reshape(rows, cols)
        x[torch.rand(rows, cols, device="cuda", generator=g) < 0.1] = 0.0
    return x.to(dtype)


def _strided(x, extra):
    if not extra:
        return x
    wide = torch.full((x.shape[0], x.shape[1] + extra), 7.0, dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def _assert_stored(c, x, floor=False):
    q, s = R.store(x, floor)
    assert torch.equal(c.scales.to(torch.int32), (s + 127).to(torch.int32))
    assert torch.equal(c.codes.view(torch.float8_e4m3fn).float().double(), q)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols,extra", [(1, 32, 0), (1, 64, 32), (2, 96, 0), (3, 160, 8), (33, 352, 0), (197, 768, 64), (513, 1056, 0)])
@pytest.mark.parametrize("floor", [False, True])
def test_store_and_load(mx, dtype, rows, cols, extra, floor):
    x = _strided(_values(rows, cols, dtype, rows + cols), extra)
    st = mx.new_status()
    c = mx.checkpoint_store(x, scale_mode=mx.SCALE_FLOOR if floor else mx.SCALE_TRUNCATION_FREE, dev_status=st)
    assert int(st.item()) == 0
    _assert_stored(c, x, floor)
    want = R.load(c.codes, c.scales)
    assert torch.equal(mx.checkpoint_load(c, mx.OUT_FP32).double(), want)
    assert torch.equal(mx.checkpoint_load(c), want.to(BF16))
    out = torch.full((rows, cols + 32), 7.0, dtype=BF16, device="cuda")
    mx.checkpoint_load(c, out=out[:, :cols])
    assert torch.equal(out[:, :cols], want.to(BF16)) and bool((out[:, cols:] == 7.0).all())


def test_store_of_every_bf16_value(mx):
    # every finite bf16 value beside a largest one: each code of each magnitude, ties among them; subnormal groups too
    bits = torch.arange(65536, device="cuda", dtype=torch.int32).to(torch.int16).view(BF16)
    x = bits[torch.isfinite(bits)].reshape(-1, 32)       # 65280 values: neighbours have one exponent
    _assert_stored(mx.checkpoint_store(x), x)
    mixed = x.t().reshape(-1, 32).contiguous()           # and values of all exponents in one group
    _assert_stored(mx.checkpoint_store(mixed), mixed)
    for k in (1.0, 1.75, 1.7578125, 1.9921875):          # the border of the scale rule
        y = torch.linspace(0.01, 1.0, 32, device="cuda").to(BF16).repeat(4, 1)
        y[:, 5] = k
        for floor in (0, 1):
            _assert_stored(mx.checkpoint_store(y, scale_mode=floor), y, bool(floor))


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_groups_that_are_not_finite(mx, bad):
    x = _values(5, 96, BF16, 3, wide=False)
    x[2, 40] = bad
    st = mx.new_status()
    c = mx.checkpoint_store(x, dev_status=st)
    assert int(st.item()) == mx.DEV_NONFINITE
    _assert_stored(c, x)
    assert int(c.scales[2, 1]) == 255 and bool((c.codes[2, 32:64] == 0).all())
    back = mx.checkpoint_load(c)
    assert bool(torch.isnan(back[2, 32:64]).all()) and int(torch.isnan(back).sum()) == 32
    st.zero_()
    _, c = mx.act_fwd(x, dev_status=st)
    assert int(st.item()) == mx.DEV_NONFINITE and int(c.scales[2, 1]) == 255
    dy = mx.act_bwd(torch.ones_like(x), c)
    assert int(torch.isnan(dy).sum()) == 32 and bool(torch.isnan(dy[2, 32:64]).all())


def _act_error(y, name):
    a = y.chunk(2, 1)[0] if name in ("geglu", "swiglu") else y
    v = a.abs() * 2.0 ** -21 if "ge" in name else R.act(a, name).abs() * (a.abs() * 2.0 ** -23 + 2.0 ** -20) + 1e-36
    return v * y.chunk(2, 1)[1].abs() if name in ("geglu", "swiglu") else v


def _slope_error(a, name):
    return torch.full_like(a, 2.0 ** -19) if "ge" in name else (1 + a.abs()) * 2.0 ** -19


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("rows,cols,extra", [(1, 32, 0), (2, 96, 32), (33, 160, 0), (197, 1536, 0), (70, 1056, 64)])
def test_act_fwd(mx, name, rows, cols, extra):
    half = 2 if name in ("geglu", "swiglu") else 1
    g = torch.Generator(device="cuda").manual_seed(rows)
    y = _strided((torch.randn(rows, cols * half, device="cuda", generator=g) * 4).to(BF16), extra)
    y[0, :8] = torch.tensor([0.0, -0.0, 30.0, -30.0, 1e-20, -1e-20, 88.0, -12.0], device="cuda").to(BF16)
    want = R.act_fwd(y.double(), name)
    z, c = mx.act_fwd(y, _act(mx, name))
    assert bool(((z.double() - want).abs() <= 2.0 ** -8 * want.abs() + _act_error(y.double(), name)).all())
    _assert_stored(c, y)
    z2, none = mx.act_fwd(y, _act(mx, name), save=mx.SAVE_NOTHING)
    assert none is None and torch.equal(z, z2)


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("rows,cols,extra", [(1, 32, 0), (2, 96, 32), (33, 160, 0), (197, 1536, 0), (70, 1056, 64)])
def test_act_bwd(mx, name, rows, cols, extra):
    half = 2 if name in ("geglu", "swiglu") else 1
    g = torch.Generator(device="cuda").manual_seed(rows)
    y = (torch.randn(rows, cols * half, device="cuda", generator=g) * 4).to(BF16)
    y[0, :8] = torch.tensor([0.0, -0.0, 30.0, -30.0, 1e-20, -1e-20, 88.0, -12.0], device="cuda").to(BF16)
    dz = _strided(torch.randn(rows, cols, device="cuda", generator=g).to(BF16), extra)
    c = mx.checkpoint_store(y)
    yr, d = R.load(c.codes, c.scales), dz.double()
    want = R.act_bwd(d, yr, name)
    if half == 2:
        a, b = yr.chunk(2, 1)
        far = torch.cat([(d * b).abs() * _slope_error(a, name), d.abs() * _act_error(torch.cat([a, torch.ones_like(a)], 1), name)], 1)
    else:
        far = d.abs() * _slope_error(yr, name)
    got = mx.act_bwd(dz, c, _act(mx, name))
    assert bool(((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + far + 1e-37).all())


def test_act_against_differences(mx):
    """The backward pass against the forward pass itself: z(y + d) - z(y - d) over 2 d, on a grid that the checkpoint holds exactly."""
    y = (torch.arange(-96, 96, device="cuda").float() / 32).reshape(6, 32)      # multiples of 2^-5 below 3
    keep = mx.checkpoint_load(mx.checkpoint_store(y.to(BF16)), mx.OUT_FP32)
    step = 0.25
    up, _ = mx.act_fwd((keep + step).to(BF16))
    down, _ = mx.act_fwd((keep - step).to(BF16))
    assert torch.equal((keep + step).to(BF16).float() - keep, torch.full_like(y, step)) and torch.equal((keep - step).to(BF16).float() - keep, torch.full_like(y, -step))
    slope = mx.act_bwd(torch.ones_like(y).to(BF16), mx.checkpoint_store(keep)).float()
    # each z is off by 2^-8 of at most 3.25, so their difference over 0.5 by 4 * 2^-8 * 3.25; the third derivative of GELU is below 1.2: 1.2 d^2 / 6
    assert float((slope - (up.float() - down.float()) / (2 * step)).abs().max()) <= 2 * 2 * 2.0 ** -8 * 3.25 + 1.2 * step * step / 6 + 2.0 ** -7


def test_gelu_is_the_epilogues(mx):
    """Between two layers GELU may be the product's epilogue or a pass of its own: the same bits."""
    g = torch.Generator(device="cuda").manual_seed(2)
    a, b = (mx.quantize(torch.randn(n, 96, device="cuda", generator=g).to(BF16)) for n in (160, 224))
    y, z = torch.empty(160, 224, dtype=BF16, device="cuda"), torch.empty(160, 224, dtype=BF16, device="cuda")
    mx.gemm_quant(a, b, mx.Epilogue(hook=mx.HOOK_GELU, y=y, z=z))
    assert torch.equal(mx.act_fwd(y)[0], z)


def test_two_streams_at_once(mx):
    """Calls on two streams that overlap on the GPU: each has its own buffers."""
    y = [(torch.randn(4096, 1536, device="cuda") * 3).to(BF16) for _ in range(2)]
    want = [mx.act_fwd(t) for t in y]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(5):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                z, c = mx.act_fwd(y[k])
                got[k] = (z, c, mx.act_bwd(z, c))
    torch.cuda.synchronize()
    for k in range(2):
        assert torch.equal(got[k][0], want[k][0]) and torch.equal(got[k][1].codes, want[k][1].codes)
        assert torch.equal(got[k][2], mx.act_bwd(want[k][0], want[k][1]))


def test_act_over_its_input(mx):
    y = (torch.randn(65, 352, device="cuda") * 3).to(BF16)
    z, c = mx.act_fwd(y)
    w = y.clone()
    z2, c2 = mx.act_fwd(w, out=w)
    assert z2 is w and torch.equal(z, w) and torch.equal(c.codes, c2.codes) and torch.equal(c.scales, c2.scales)
    dz = torch.randn(65, 352, device="cuda").to(BF16)
    dy = mx.act_bwd(dz, c)
    mx.act_bwd(dz, c, out=dz)
    assert torch.equal(dz, dy)


@pytest.mark.parametrize("name", NAMES)
def test_side_by_side(mx, name):
    """Inputs and outputs one right behind the other in memory, in either order."""
    half = 2 if name in ("geglu", "swiglu") else 1
    rows, cols = 6, 64
    buf = torch.randn(rows * cols * (2 * half + 1), device="cuda").to(BF16)
    for first in (True, False):
        n, k = rows * cols * half, rows * cols
        y = (buf[:n] if first else buf[k:k + n]).view(rows, cols * half)
        z = (buf[n:n + k] if first else buf[:k]).view(rows, cols)
        want, c = mx.act_fwd(y.clone(), _act(mx, name))
        mx.act_fwd(y, _act(mx, name), out=z)
        assert torch.equal(z, want)
        dz, dy = z, y
        g = mx.act_bwd(dz.clone(), c, _act(mx, name))
        mx.act_bwd(dz, c, _act(mx, name), out=dy)
        assert torch.equal(dy, g)


def test_no_rows(mx):
    y = torch.empty(0, 64, dtype=BF16, device="cuda")
    z, c = mx.act_fwd(y)
    assert z.shape == (0, 64) and c.codes.shape == (0, 64) and mx.act_bwd(y, c).shape == (0, 64) and mx.checkpoint_load(mx.checkpoint_store(y)).shape == (0, 64)


def test_captured_and_on_another_stream(mx):
    y = (torch.randn(300, 384, device="cuda") * 3).to(BF16)
    dz = torch.randn(300, 384, device="cuda").to(BF16)
    z, c = mx.act_fwd(y)
    dy = mx.act_bwd(dz, c)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        z1, c1 = mx.act_fwd(y)
        dy1 = mx.act_bwd(dz, c1)
    torch.cuda.synchronize()
    assert torch.equal(z, z1) and torch.equal(dy, dy1)
    y2 = torch.zeros_like(y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        z2, c2 = mx.act_fwd(y2)
        dy2 = mx.act_bwd(dz, c2)
    for k in (1.0, 2.0):
        y2.copy_(y * k)
        graph.replay()
        z, c = mx.act_fwd(y * k)
        assert torch.equal(z2, z) and torch.equal(dy2, mx.act_bwd(dz, c))


def test_more_elements_than_32_bits_of_bytes(mx):
    rows, cols = 70000, 32768       # 2.3e9 elements: offsets beyond 2^31 in the codes, beyond 2^32 in the bytes of bf16
    y = torch.empty(rows, cols, dtype=BF16, device="cuda")
    y[:128] = 1.0
    y[-128:] = (torch.randn(128, cols, device="cuda") * 3).to(BF16)
    z, c = mx.act_fwd(y)
    last, lc = mx.act_fwd(y[-128:].contiguous())
    assert torch.equal(z[-128:], last) and torch.equal(c.codes[-128:], lc.codes) and torch.equal(c.scales[-128:], lc.scales)
    del z
    dy = mx.act_bwd(y, c)
    assert torch.equal(dy[-128:], mx.act_bwd(y[-128:].contiguous(), lc))
    del dy
    assert torch.equal(mx.checkpoint_load(c)[-128:], mx.checkpoint_load(lc))
