"""Dense layers (gs_dense_forward, gs_dense_backward) against their formulas in 64 bits: types, activations, odd widths, row
strides, the ends of tiles and pipeline steps, and what lies around the matrices."""
import pytest

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1, 1), (1, 64, 64), (2, 3, 8), (5, 8, 3), (63, 16, 16), (64, 63, 256), (65, 65, 130), (127, 256, 8), (128, 128, 128), (129, 257, 255),
          (300, 512, 520), (1000, 40, 300), (1000, 256, 256), (513, 700, 1024), (2500, 1024, 96), (40_000, 24, 16), (20_003, 96, 200)]


@pytest.fixture(scope="module")
def ctx():
    from paper_2609_05255_b200 import api
    c = api.Context(0)
    yield c
    api.gs_async_status(c)             # no wait of any call ran out
    c.close()


def make(rows, cin, cout, dtype, seed, pad=0):
    import torch
    from layer_helpers import Guarded
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    randn = lambda *s: torch.randn(s, device="cuda", generator=gen)
    ld = lambda c: (c + 7) // 8 * 8 + pad
    x = Guarded(rows, cin, dtype, ld(cin), randn(rows, cin)).t
    w = Guarded(cout, cin, dtype, ld(cin), randn(cout, cin) / cin ** 0.5).t
    b = randn(cout) * 0.3
    r = Guarded(rows, cout, dtype, ld(cout), randn(rows, cout)).t
    z = Guarded(rows, cout, dtype, ld(cout), randn(rows, cout) * 2).t
    dy = randn(rows, cout) * 0.01 * (torch.rand((rows, 1), device="cuda", generator=gen) < 0.8)
    dy = Guarded(rows, cout, dtype, ld(cout), dy).t
    return x, w, b, r, z, dy, ld


def check_forward(ctx, rows, cin, cout, dtype, act, bias=True, residual=False, keep=False, seed=0, pad=0):
    from layer_helpers import HALF_STEP, HALF_TINY, U32, Guarded, act as act64, act_error, close
    from paper_2609_05255_b200 import api
    x, w, b, r, _, _, ld = make(rows, cin, cout, dtype, seed, pad)
    layer = api.DenseLayer(w, b if bias else None, act)
    y, z = Guarded(rows, cout, dtype, ld(cout)), Guarded(rows, cout, dtype, ld(cout))
    api.gs_dense_forward(ctx, layer, x, y.t, preact=z.t if keep else None, residual=r if residual else None)
    z64, size = x.double() @ w.double().T, x.double().abs() @ w.double().abs().T
    if bias:
        z64, size = z64 + b.double(), size + b.double().abs()
    e_z = (cin + 2) * U32 * size                          # every addition loses at most a step of what it is up to
    y64, slope = act64(act, z64)[:2]
    e_y = 1.13 * e_z + act_error(act, z64)                # |act'| <= 1.13
    if residual:
        y64 = y64 + r.double()
        e_y = e_y + U32 * (y64.abs() + r.double().abs())
    close(y.check(), y64, e_y * 1.01 + HALF_STEP[dtype] * y64.abs() * 1.01 + HALF_TINY[dtype], "y")
    if keep:
        close(z.check(), z64, e_z * 1.01 + HALF_STEP[dtype] * z64.abs() * 1.01 + HALF_TINY[dtype], "preact")


def check_backward(ctx, rows, cin, cout, dtype, act, want=("dx", "dw", "db"), seed=0, pad=0):
    import torch
    from layer_helpers import HALF_STEP, HALF_TINY, U32, Guarded, act as act64, act_grad_error, close
    from paper_2609_05255_b200 import api
    x, w, b, _, z, dy, ld = make(rows, cin, cout, dtype, seed, pad)
    layer = api.DenseLayer(w, b, act)
    dx = Guarded(rows, cin, dtype, ld(cin))
    guard = torch.full((cout * cin + cout + 12,), 7.0, device="cuda")
    dw, db = guard[4:4 + cout * cin].view(cout, cin), guard[8 + cout * cin:8 + cout * cin + cout]
    ws = torch.full((api.gs_dense_workspace_bytes(rows, cin, cout) + 256,), 77, device="cuda", dtype=torch.uint8)
    call = lambda: api.gs_dense_backward(ctx, layer, x if "dw" in want else None, dy, preact=None if act == "none" else z,
                                         dL_dx=dx.t if "dx" in want else None, dL_dweight=dw if "dw" in want else None,
                                         dL_dbias=db if "db" in want else None, workspace=ws[:-256] if "dw" in want else None)
    call()
    dz = dy.double() * (act64(act, z.double())[1] if act != "none" else 1.0)
    # dz in parts: what the last one leaves, and the derivative's error; parts of dx have 16 bits (bf16) or 22, those of dW 24 or 22
    e_dz = dy.double().abs() * act_grad_error(act, z.double()) + U32 * dz.abs() if act in ("silu", "gelu") else torch.zeros_like(dz)
    smooth = act in ("silu", "gelu")
    h = HALF_STEP[dtype]
    e_x = e_dz + smooth * (h * h * dz.abs() + HALF_TINY[dtype])
    e_w = e_dz + smooth * ((h ** 3 if dtype is torch.bfloat16 else h * h) * dz.abs() + 2.0 ** -36)
    if "dx" in want:
        wa = w.double().abs()
        want_dx = dz @ w.double()
        bound = e_x @ wa + (2 * cout + 2) * U32 * (dz.abs() @ wa)
        close(dx.check(), want_dx, bound * 1.01 + h * want_dx.abs() * 1.01 + HALF_TINY[dtype], "dx")
    if "dw" in want:
        xa = x.double().abs()
        close(dw, dz.T @ x.double(), (e_w.T @ xa + (3 * rows + 4) * U32 * (dz.abs().T @ xa)) * 1.01 + 1e-37, "dW")
    if "db" in want:
        close(db, dz.sum(0), (e_w.sum(0) + (rows + 4) * U32 * dz.abs().sum(0)) * 1.01 + 1e-37, "db")
    assert torch.all(guard[:4] == 7) and torch.all(guard[4 + cout * cin:8 + cout * cin] == 7) and torch.all(guard[8 + cout * cin + cout:] == 7)
    assert torch.all(ws[-256:] == 77)
    first = [t.clone() for t in (dx.t, dw, db)]
    call()
    assert all(torch.equal(a, c) for a, c in zip(first, (dx.t, dw, db))), "two calls differ"


def _types():
    import torch
    return {"f16": torch.float16, "bf16": torch.bfloat16}


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows,cin,cout", SHAPES)
def test_forward_shapes(ctx, rows, cin, cout, dtype):
    k = (rows + cin + cout) % 4
    check_forward(ctx, rows, cin, cout, _types()[dtype], ["none", "relu", "silu", "gelu"][k], bias=k != 1, residual=rows % 2 == 0, keep=cin % 2 == 0,
                  seed=rows)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("residual,keep", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
def test_forward_epilogues(ctx, act, residual, keep, dtype):
    check_forward(ctx, 333, 72, 136, _types()[dtype], act, residual=residual, keep=keep, seed=5, pad=16)


@pytest.mark.parametrize("residual,keep", [(False, False), (True, True)])
def test_forward_many_tiles(ctx, residual, keep):
    """More tiles than SMs: several per CTA, both accumulators in use, and weights that fit in shared memory or do not."""
    import torch
    check_forward(ctx, 148 * 128 * 3 + 17, 256, 256, torch.bfloat16, "silu", residual=residual, keep=keep, seed=6)
    check_forward(ctx, 148 * 128 + 1, 520, 264, torch.float16, "gelu", residual=residual, keep=keep, seed=7)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows,cin,cout", SHAPES)
def test_backward_shapes(ctx, rows, cin, cout, dtype):
    check_backward(ctx, rows, cin, cout, _types()[dtype], ["silu", "relu", "gelu", "none"][(rows + cin + cout) % 4], seed=rows)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
def test_backward_activations(ctx, act, dtype):
    check_backward(ctx, 1111, 72, 136, _types()[dtype], act, seed=8, pad=24)
    check_backward(ctx, 148 * 128 * 2 + 5, 136, 72, _types()[dtype], act, seed=9)


@pytest.mark.parametrize("want", [("dx",), ("dw", "db"), ("dw",), ("dx", "dw")])
def test_backward_parts(ctx, want):
    import torch
    check_backward(ctx, 777, 64, 48, torch.float16, "silu", want=want, seed=10)


@pytest.mark.parametrize("rows,cin,cout", [(5, 16384, 16), (3, 16, 16384), (300, 5000, 3001), (9_000_001, 8, 16)])
def test_the_widest_and_the_longest(ctx, rows, cin, cout):
    """Weights of hundreds of steps, hundreds of column tiles, and rows whose offsets pass 2^31 bytes when padded."""
    import torch
    check_forward(ctx, rows, cin, cout, torch.bfloat16, "silu", residual=True, keep=True, seed=14, pad=240 if rows > 1_000_000 else 0)
    if rows < 1_000_000:
        check_backward(ctx, rows, cin, cout, torch.float16, "gelu", seed=15)
        check_backward(ctx, rows, cin, cout, torch.bfloat16, "relu", seed=16)


def test_extreme_preactivations(ctx):
    """act and act' at the ends of the types: 0 or linear, never NaN; a NaN stays in its row."""
    import torch
    from paper_2609_05255_b200 import api
    for dtype, big in ((torch.float16, 6.0e4), (torch.bfloat16, 1.0e38)):
        z = torch.tensor([-big, -100.0, -20.0, 0.0, 20.0, 100.0, big, float("nan")], device="cuda").to(dtype)
        eye = torch.eye(8, device="cuda", dtype=dtype)
        for act in ("silu", "gelu"):
            layer = api.DenseLayer(eye, None, act)
            x, y = z[None, :].repeat(3, 1), torch.empty((3, 8), device="cuda", dtype=dtype)
            x[0], x[2] = 1.0, 2.0
            finite = x.clone()
            finite[1, 7] = 0.0
            api.gs_dense_forward(ctx, layer, finite, y)
            assert torch.all(y[1, :2] == 0) and torch.equal(y[1, 5:7], finite[1, 5:7])
            dx = torch.empty_like(y)
            ones = torch.ones_like(y)
            dw, ws = torch.empty((8, 8), device="cuda"), torch.empty((api.gs_dense_workspace_bytes(3, 8, 8),), device="cuda", dtype=torch.uint8)
            api.gs_dense_backward(ctx, layer, ones, ones, preact=finite, dL_dx=dx, dL_dweight=dw, workspace=ws)
            assert torch.all(dx[1, :2] == 0) and torch.all(dx[1, 5:7] == 1)
            assert torch.all(dx.isfinite()) and torch.all(dw.isfinite())
            # (a row of dx is a product with all of W: one NaN of dz is in all of the row, and in one row of dW)
            api.gs_dense_backward(ctx, layer, ones, ones, preact=x, dL_dx=dx, dL_dweight=dw, workspace=ws)
            assert torch.all(dx[1].isnan()) and torch.all(dx[[0, 2]].isfinite()) and torch.all(dw[:7].isfinite()) and torch.all(dw[7].isnan())


def test_gradient_by_differences(ctx):
    """dx, dW and db of sum(y * g) against central differences of the forward pass itself (linear in each weight: SiLU's
    curvature is what the differences miss)."""
    import torch
    from layer_helpers import act as act64
    from paper_2609_05255_b200 import api
    x, w, b, _, _, g, _ = make(37, 24, 40, torch.float16, 11)
    layer = api.DenseLayer(w, b, "silu")
    y, z = torch.empty((37, 40), device="cuda", dtype=torch.float16), torch.empty((37, 40), device="cuda", dtype=torch.float16)
    api.gs_dense_forward(ctx, layer, x, y, preact=z)
    dx = torch.empty((37, 24), device="cuda", dtype=torch.float16)
    dw, db = torch.empty((40, 24), device="cuda"), torch.empty((40,), device="cuda")
    ws = torch.empty((api.gs_dense_workspace_bytes(37, 24, 40),), device="cuda", dtype=torch.uint8)
    api.gs_dense_backward(ctx, layer, x, g, preact=z, dL_dx=dx, dL_dweight=dw, dL_dbias=db, workspace=ws)
    f = lambda xx, ww, bb: (act64("silu", xx @ ww.T + bb)[0] * g.double()).sum()
    X, W, B, h = x.double(), w.double(), b.double(), 1e-4
    # z was rounded (2^-11 relative), so act' is off by at most 2^-11 |z| |act''| <= 2^-11 * 0.6; h^2 / 6 |f'''| <= 1e-8
    for i, j in ((0, 0), (3, 23), (39, 11), (17, 5)):
        E = torch.zeros_like(W)
        E[i, j] = h
        d = (f(X, W + E, B) - f(X, W - E, B)) / (2 * h)
        assert abs(float(d) - float(dw[i, j])) <= 2.0 ** -11 * 0.6 * float((g.double()[:, i].abs() * X[:, j].abs()).sum()) + 1e-7
    for i in (0, 21, 39):
        E = torch.zeros_like(B)
        E[i] = h
        d = (f(X, W, B + E) - f(X, W, B - E)) / (2 * h)
        assert abs(float(d) - float(db[i])) <= 2.0 ** -11 * 0.6 * float(g.double()[:, i].abs().sum()) + 1e-7
    for i, j in ((0, 0), (36, 23), (20, 7)):
        E = torch.zeros_like(X)
        E[i, j] = h
        d = (f(X + E, W, B) - f(X - E, W, B)) / (2 * h)
        assert abs(float(d) - float(dx[i, j])) <= 2.0 ** -11 * (0.6 * float((g.double()[i].abs() * W[:, j].abs()).sum()) + abs(float(d))) + 1e-7


def test_residual_in_place_streams_and_graph(ctx):
    import torch
    from paper_2609_05255_b200 import api
    x, w, b, r, _, dy, _ = make(3000, 64, 64, torch.bfloat16, 12)
    layer = api.DenseLayer(w, b, "gelu")
    y, z = torch.empty_like(dy), torch.empty_like(dy)
    api.gs_dense_forward(ctx, layer, x, y, preact=z, residual=r)
    same = r.clone()
    api.gs_dense_forward(ctx, layer, x, same, residual=same)
    assert torch.equal(same, y)
    dx, dw, db = torch.empty_like(x), torch.empty((64, 64), device="cuda"), torch.empty((64,), device="cuda")
    ws = torch.empty((api.gs_dense_workspace_bytes(3000, 64, 64),), device="cuda", dtype=torch.uint8)
    api.gs_dense_backward(ctx, layer, x, dy, preact=z, dL_dx=dx, dL_dweight=dw, dL_dbias=db, workspace=ws)
    want = [t.clone() for t in (y, z, dx, dw, db)]
    torch.cuda.synchronize()
    # captured, replayed on other values and back
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        api.gs_dense_forward(ctx, layer, x, y, preact=z, residual=r)
        api.gs_dense_backward(ctx, layer, x, dy, preact=z, dL_dx=dx, dL_dweight=dw, dL_dbias=db, workspace=ws)
    keep = x.clone()
    x.mul_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    assert not torch.equal(y, want[0])
    x.copy_(keep)
    for t in (y, z, dx, dw, db):
        t.fill_(0)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip((y, z, dx, dw, db), want))
    # a stream of its own, with its own context
    other = api.Context(0)
    y2 = torch.empty_like(y)
    side.wait_stream(torch.cuda.current_stream())
    api.gs_dense_forward(other, layer, x, y2, residual=r, stream=side)
    side.synchronize()
    assert torch.equal(y2, want[0])
    other.close()


def test_a_layer_follows_its_tensors(ctx):
    """Weights and bias that got other memory between the calls, as a copy of the parameters does it."""
    import torch
    from paper_2609_05255_b200 import api
    x, w, b, _, _, _, _ = make(70, 24, 40, torch.float16, 13)
    layer = api.DenseLayer(w, b, "relu")
    y, want = torch.empty((70, 40), device="cuda", dtype=torch.float16), torch.empty((70, 40), device="cuda", dtype=torch.float16)
    api.gs_dense_forward(ctx, layer, x, y)
    v, c = (w * 0.5).contiguous(), b + 1
    api.gs_dense_forward(ctx, api.DenseLayer(v, c, "relu"), x, want)
    layer.weight.data, layer.bias.data = v.clone(), c.clone()
    api.gs_dense_forward(ctx, layer, x, y)
    assert torch.equal(y, want)
    layer.weight.data = torch.zeros((40, 32), device="cuda", dtype=torch.float16)
    with pytest.raises(api.GsError):
        api.gs_dense_forward(ctx, layer, x, y)


def test_captured_before_any_other_call():
    """The first call of a process may be one that is captured: kernels are set up without a word to the stream."""
    import subprocess
    import sys
    code = """
import torch
from paper_2609_05255_b200 import api
ctx = api.Context(0)
h = lambda *s: torch.randn(s, device="cuda").half()
x, w, dy, z = h(700, 64), h(256, 64), h(700, 256), h(700, 256)
layer = api.DenseLayer(w, None, "silu")
outs = lambda: (torch.empty_like(dy), torch.empty_like(x), torch.empty((256, 64), device="cuda"), torch.empty((256,), device="cuda"), torch.empty_like(x))
ws = torch.empty((api.gs_dense_workspace_bytes(700, 64, 256),), device="cuda", dtype=torch.uint8)
clip, gws = torch.empty((2,), device="cuda"), torch.empty((api.gs_grad_workspace_bytes(),), device="cuda", dtype=torch.uint8)
def run(y, dx, dw, db, n):
    api.gs_dense_forward(ctx, layer, x, y)
    api.gs_dense_backward(ctx, layer, x, dy, preact=z, dL_dx=dx, dL_dweight=dw, dL_dbias=db, workspace=ws)
    api.gs_layer_norm_forward(ctx, x, None, None, n)
    api.gs_clip_grads(ctx, [api.GradTensor(dw, out=dw)], 1.0, clip, gws)
a, b = outs(), outs()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    run(*a)
graph.replay()
run(*b)
torch.cuda.synchronize()
assert all(torch.equal(p, q) for p, q in zip(a, b))
del graph
ctx.close()
"""
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]


def test_no_rows(ctx):
    import torch
    from paper_2609_05255_b200 import api
    layer = api.DenseLayer(torch.randn((16, 8), device="cuda").half(), None, "relu")
    x, y = torch.empty((0, 8), device="cuda", dtype=torch.float16), torch.empty((0, 16), device="cuda", dtype=torch.float16)
    api.gs_dense_forward(ctx, layer, x, y)
    dw, db = torch.ones((16, 8), device="cuda"), torch.ones((16,), device="cuda")
    api.gs_dense_backward(ctx, layer, x, y, preact=y, dL_dx=x, dL_dweight=dw, dL_dbias=db)
    assert torch.all(dw == 0) and torch.all(db == 0)


def test_refusals(ctx):
    import torch
    from paper_2609_05255_b200 import api
    h = lambda *s: torch.zeros(s, device="cuda", dtype=torch.float16)
    layer = api.DenseLayer(h(16, 8), None, "relu")

    def refused(status, f):
        with pytest.raises(api.GsError) as e:
            f()
        assert e.value.status == status and str(e.value)
    bad = api.GS_ERR_INVALID_ARG
    refused(bad, lambda: api.gs_dense_forward(ctx, layer, h(4, 9), h(4, 16)))                     # a width that is not the layer's
    refused(bad, lambda: api.gs_dense_forward(ctx, layer, h(4, 8), h(5, 16)))
    refused(bad, lambda: api.gs_dense_forward(ctx, layer, h(4, 8).bfloat16(), h(4, 16)))          # another type
    refused(bad, lambda: api.gs_dense_forward(ctx, layer, h(4, 8).cpu(), h(4, 16)))
    refused(bad, lambda: api.gs_dense_forward(ctx, layer, h(8, 4).T, h(4, 16)))                   # columns instead of rows
    refused(bad, lambda: api.gs_dense_forward(ctx, layer, h(4, 9)[:, 1:], h(4, 16)))              # row stride 9, not aligned
    refused(bad, lambda: api.gs_dense_forward(ctx, layer, h(4, 8), h(4, 20)[:, :16]))             # row stride 20
    refused(bad, lambda: api.gs_dense_forward(ctx, layer, h(4, 8), h(4, 16), preact=h(4, 8)))
    refused(bad, lambda: api.gs_dense_forward(ctx, api.DenseLayer(h(16, 9)[:, 1:], None, "relu"), h(4, 8), h(4, 16)))
    refused(api.GS_ERR_UNSUPPORTED, lambda: api.gs_dense_forward(ctx, api.DenseLayer(h(16, 8).float()), h(4, 8).float(), h(4, 16).float()))
    refused(bad, lambda: api.DenseLayer(h(16, 8), None, "tanh"))
    refused(bad, lambda: api.DenseLayer(h(16, 8), torch.zeros(15, device="cuda")))
    refused(bad, lambda: api.DenseLayer(h(16, 8), h(16)))
    dw = torch.zeros((16, 8), device="cuda")
    ws = torch.zeros((api.gs_dense_workspace_bytes(4, 8, 16),), device="cuda", dtype=torch.uint8)
    refused(bad, lambda: api.gs_dense_backward(ctx, layer, h(4, 8), h(4, 16), dL_dx=h(4, 8)))      # preact is missing
    refused(bad, lambda: api.gs_dense_backward(ctx, layer, None, h(4, 16), preact=h(4, 16), dL_dweight=dw, workspace=ws))
    refused(bad, lambda: api.gs_dense_backward(ctx, layer, h(4, 8), h(4, 16), preact=h(4, 16), dL_dweight=dw))
    refused(bad, lambda: api.gs_dense_backward(ctx, layer, h(4, 8), h(4, 16), preact=h(4, 16), dL_dbias=torch.zeros(16, device="cuda"), workspace=ws))
    refused(api.GS_ERR_CAPACITY, lambda: api.gs_dense_backward(ctx, layer, h(4, 8), h(4, 16), preact=h(4, 16), dL_dweight=dw, workspace=ws[:-16]))
