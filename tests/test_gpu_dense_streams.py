"""Wide layers, whose backward runs on pairs of CTAs: captured into graphs and replayed, on streams side by side with contexts of
their own, and counted by the profile.  Results are the same bits as those of a call by itself."""
import pytest

pytestmark = pytest.mark.gpu

SHAPES = [(40_003, 256, 256), (3_001, 264, 512), (20_011, 512, 264)]


def _types():
    import torch
    return {"f16": torch.float16, "bf16": torch.bfloat16}


class Call:
    def __init__(self, rows, cin, cout, dtype, act, seed):
        import torch
        from paper_2609_05255_b200 import api
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        randn = lambda *s: torch.randn(s, device="cuda", generator=gen)
        self.x, self.w, self.dy = randn(rows, cin).to(dtype), (randn(cout, cin) / cin ** 0.5).to(dtype), (randn(rows, cout) * 0.01).to(dtype)
        self.layer = api.DenseLayer(self.w, randn(cout) * 0.1, act)
        self.out = [torch.empty((rows, cout), device="cuda", dtype=dtype), torch.empty((rows, cout), device="cuda", dtype=dtype), torch.empty_like(self.x),
                    torch.empty((cout, cin), device="cuda"), torch.empty((cout,), device="cuda")]
        self.ws = torch.empty((api.gs_dense_workspace_bytes(rows, cin, cout),), device="cuda", dtype=torch.uint8)

    def run(self, ctx, stream=None):
        from paper_2609_05255_b200 import api
        y, z, dx, dw, db = self.out
        api.gs_dense_forward(ctx, self.layer, self.x, y, preact=z, stream=stream)
        api.gs_dense_backward(ctx, self.layer, self.x, self.dy, preact=z, dL_dx=dx, dL_dweight=dw, dL_dbias=db, workspace=self.ws, stream=stream)

    def alone(self, ctx):
        import torch
        self.run(ctx)
        torch.cuda.synchronize()
        want = [t.clone() for t in self.out]
        for t in self.out:
            t.fill_(0)
        return want

    def same(self, want):
        import torch
        return all(torch.equal(a, b) for a, b in zip(self.out, want))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("rows,cin,cout", SHAPES)
def test_captured(rows, cin, cout, act, dtype):
    import torch
    from paper_2609_05255_b200 import api
    ctx = api.Context(0)
    c = Call(rows, cin, cout, _types()[dtype], act, rows)
    want = c.alone(ctx)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(ctx)
        c.run(ctx)
    for _ in range(3):
        for t in c.out:
            t.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert c.same(want)
    api.gs_async_status(ctx)
    del graph
    ctx.close()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_streams_side_by_side(dtype):
    """Kernels of four streams, some on pairs of CTAs and some not, all after the same tensor memory."""
    import torch
    from paper_2609_05255_b200 import api
    ctxs, streams = [api.Context(0) for _ in range(4)], [torch.cuda.Stream() for _ in range(4)]
    kinds = [(20_011, 256, 256, "silu"), (9_001, 72, 136, "gelu"), (3_001, 512, 264, "relu"), (5_003, 264, 512, "none")]
    calls = [Call(m, k, n, _types()[dtype], act, m) for m, k, n, act in kinds]
    wants = [c.alone(ctxs[0]) for c in calls]
    torch.cuda.synchronize()
    for _ in range(10):
        for c, ctx, s in zip(calls, ctxs, streams):
            c.run(ctx, s)
    torch.cuda.synchronize()
    assert all(c.same(w) for c, w in zip(calls, wants))
    for ctx in ctxs:
        api.gs_async_status(ctx)
        ctx.close()
