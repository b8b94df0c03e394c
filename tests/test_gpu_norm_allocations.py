"""The buffers that the binding allocates when nothing hooks its allocations in (several results in one, views made when they are asked for):
bit for bit what the calls give with each buffer on its own between guard bytes, as in all other GPU tests."""
import itertools

import pytest
import torch

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def mx():
    import paper_2502_20853_b200 as m
    m.lib()
    return m


class Unhooked:
    """Allocations as a user's program gets them."""

    def __enter__(self):
        from paper_2502_20853_b200 import binding
        self.binding, self.hook = binding, binding.ALLOC_HOOK
        assert self.hook is not None
        binding.ALLOC_HOOK = None

    def __exit__(self, *e):
        self.binding.ALLOC_HOOK = self.hook


def _open(ckpts, views):
    for c in ckpts:
        for name in views:
            if c is not None:
                getattr(c, name)


def _same(a, b):
    return (a is None and b is None) or torch.equal(a, b)


VIEWS = [(), ("codes",), ("scales",), ("codes", "scales")]


@pytest.mark.parametrize("rows,cols", [(1, 32), (3, 96), (257, 416), (196, 768), (37, 8192)])
@pytest.mark.parametrize("views", VIEWS)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_checkpoints_and_activations(mx, rows, cols, views, dtype):
    x = (torch.randn(rows, 2 * cols, device="cuda") * 3).to(dtype)
    y, dz = x.to(BF16), torch.randn(rows, cols, device="cuda").to(BF16)

    def calls():
        c = mx.checkpoint_store(x)
        _open([c], views)
        out = [mx.checkpoint_load(c, mx.OUT_FP32), mx.checkpoint_load(c)]
        for act, t in ((mx.ACT_GELU, y[:, :cols]), (mx.ACT_SILU, y[:, :cols].contiguous()), (mx.ACT_GEGLU, y), (mx.ACT_SWIGLU, y)):
            z, k = mx.act_fwd(t, act)
            _open([k], views)
            out += [z, mx.act_bwd(dz, k, act), k.codes, k.scales]
        return out + [c.codes, c.scales]

    want = calls()
    with Unhooked():
        got = calls()
    assert all(_same(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("rows,cols,gates", [(1, 32, 1), (3, 96, 3), (257, 416, 0), (196, 768, 7), (37, 8192, 1)])
@pytest.mark.parametrize("views", VIEWS)
def test_norms(mx, rows, cols, gates, views):
    rnd = lambda *s: torch.randn(*s, device="cuda")  # noqa: E731
    for dtype, (weight, bias), post in itertools.product((BF16, F32), ((False, False), (True, False), (True, True)), (False, True)):
        x, f, gate = rnd(rows, cols).to(dtype), rnd(rows, cols).to(BF16), rnd(gates, cols) if gates else None
        side = lambda: mx.Norm(mx.NORM_LAYER, 1 + 0.3 * rnd(cols) if weight else None, rnd(cols) if bias else None)  # noqa: E731
        pre, post_n, dh, dx_out = side(), side() if post else None, rnd(rows, cols).to(BF16), rnd(rows, cols).to(dtype)

        def calls():
            hq = mx.QMat(rows, cols)
            hq.scales.zero_()
            x_out, h, ctx = mx.residual_norm_fwd(x, f, pre=pre, post=post_n, gate=gate, hq=hq)
            _open([ctx.x, ctx.f], views)
            g = mx.residual_norm_bwd(dh, dx_out, ctx)
            out = [x_out, h, hq.data, hq.scales[:mx.scale_bytes(rows, cols)], *g]
            for c in (ctx.x, ctx.f):
                out += [c.codes, c.scales] if c is not None else [None, None]
            present = [k for k, n in ((0, pre), (1, pre), (2, post_n), (3, post_n)) if n is not None]
            return out + [ctx.stats[present]]

        want = calls()
        with Unhooked():
            got = calls()
            for _ in range(2):      # buffers that come back from the allocator used
                again = calls()
                assert all(_same(a, b) for a, b in zip(again, want))
        assert all(_same(a, b) for a, b in zip(got, want))


def test_two_streams_at_once(mx):
    """Each call has buffers of its own, on the stream that it runs on."""
    rnd = lambda *s: torch.randn(*s, device="cuda")  # noqa: E731
    cases = []
    for k in range(2):
        norm = mx.Norm(mx.NORM_LAYER, 1 + 0.3 * rnd(384), rnd(384))
        cases.append(dict(x=rnd(3000, 384).to(BF16), f=rnd(3000, 384).to(BF16), pre=norm, post=norm, gate=rnd(3, 384), dh=rnd(3000, 384).to(BF16), dx=rnd(3000, 384).to(BF16),
                          y=(3 * rnd(3000, 768)).to(BF16)))

    def calls(c):
        x_out, h, ctx = mx.residual_norm_fwd(c["x"], c["f"], pre=c["pre"], post=c["post"], gate=c["gate"])
        z, k = mx.act_fwd(c["y"], mx.ACT_SWIGLU)
        return [x_out, h, z, mx.act_bwd(z, k, mx.ACT_SWIGLU), *mx.residual_norm_bwd(c["dh"], c["dx"], ctx), ctx.x.codes, ctx.f.scales]

    want = [calls(c) for c in cases]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in cases], [None, None]
    with Unhooked():
        for _ in range(6):
            for i, c in enumerate(cases):
                with torch.cuda.stream(streams[i]):
                    got[i] = calls(c)
        torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(_same(s, t) for s, t in zip(a, b))


def test_captured(mx):
    """Two graphs, each with buffers of its own from its pool, replayed in turn on other inputs."""
    rnd = lambda *s: torch.randn(*s, device="cuda")  # noqa: E731
    norm = mx.Norm(mx.NORM_RMS, 1 + 0.3 * rnd(384))
    x, f, dh, dx_out = (rnd(500, 384).to(BF16) for _ in range(4))

    def calls():
        x_out, h, ctx = mx.residual_norm_fwd(x, f, pre=norm, post=norm)
        z, k = mx.act_fwd(h)
        return [x_out, h, z, mx.act_bwd(z, k), *mx.residual_norm_bwd(dh, dx_out, ctx)]

    with Unhooked():
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            calls()
        torch.cuda.synchronize()
        graphs = []
        for _ in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                out = calls()
            graphs.append((graph, out))
        for seed in range(3):
            g = torch.Generator(device="cuda").manual_seed(seed)
            for t in (x, f, dh, dx_out):
                t.copy_(torch.randn(t.shape, device="cuda", generator=g))
            for graph, out in graphs:
                graph.replay()
            want = calls()
            torch.cuda.synchronize()
            for _, out in graphs:
                assert all(_same(a, b) for a, b in zip(out, want))
