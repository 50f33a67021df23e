"""Layer norm, forward and backward, against the formulas in 64 bits: types, every layout of a row over lanes, rows that are
not aligned, and rows without spread."""
import pytest

pytestmark = pytest.mark.gpu

COLS = [1, 2, 3, 7, 8, 16, 31, 33, 45, 64, 100, 128, 129, 256, 300, 512, 513, 768, 1024, 1025, 2048, 2049, 4100, 8192]


@pytest.fixture(scope="module")
def ctx():
    from paper_2609_05255_b200 import api
    c = api.Context(0)
    yield c
    c.close()


def _types():
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def check(ctx, rows, cols, dtype, ld=None, offset=0, affine=True, eps=1e-5, seed=0, mean_of=0.5, spread=1.0, aligned_dy=True):
    import torch
    from layer_helpers import HALF_STEP, HALF_TINY, U32, Guarded, close
    from paper_2609_05255_b200 import api
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    randn = lambda *s: torch.randn(s, device="cuda", generator=gen)
    x = Guarded(rows, cols, dtype, ld, mean_of * randn(rows, 1) + spread * randn(rows, cols), offset).t
    dy = Guarded(rows, cols, dtype, ld, randn(rows, cols) * 0.01, offset if aligned_dy else 0).t
    gamma, beta = (1 + 0.3 * randn(cols), randn(cols)) if affine else (None, None)
    y, dx = Guarded(rows, cols, dtype, ld, offset=offset), Guarded(rows, cols, dtype, ld, offset=offset)
    mean, rstd = torch.full((rows + 2,), 7.0, device="cuda"), torch.full((rows + 2,), 7.0, device="cuda")
    api.gs_layer_norm_forward(ctx, x, gamma, beta, y.t, mean=mean[1:-1], rstd=rstd[1:-1], eps=eps)
    X, G, B = x.double(), 1.0 if gamma is None else gamma.double(), 0.0 if beta is None else beta.double()
    m = X.mean(1, keepdim=True)
    var = (X - m).square().mean(1, keepdim=True)
    r = (var + eps).rsqrt()
    # a sum of at most 32 values a lane, 5 exchanges and 8 warps, then the product with 1 / cols: 48 roundings of half a step
    k = 48 * U32 / 2
    e_m = k * X.abs().mean(1, keepdim=True)
    d = (X - m).abs()
    # (x - mean'): the mean's error and a rounding; in the variance the mean's error enters squared
    e_r = r * (0.5 * (k + 3 * U32) + 0.5 * r * r * (e_m * e_m + U32 * d.mean(1, keepdim=True) * (e_m + U32 * d.mean(1, keepdim=True))) + 3 * U32)
    h = (X - m) * r
    e_h = r * (e_m + U32 * d) + d * e_r + U32 * h.abs()
    want = h * G + B
    e_y = abs(G) * e_h + U32 * ((h * G).abs() + want.abs())
    step, tiny = HALF_STEP[dtype], HALF_TINY[dtype]
    close(mean[1:-1], m[:, 0], e_m[:, 0] * 1.01 + 1e-37, "mean")
    close(rstd[1:-1], r[:, 0], e_r[:, 0] * 1.01, "rstd")
    close(y.check(), want, e_y * 1.01 + step * want.abs() * 1.01 + tiny, "y")
    assert all(float(t[i]) == 7 for t in (mean, rstd) for i in (0, -1))

    # backward, from the statistics as the forward left them
    ws = torch.full((api.gs_layer_norm_workspace_bytes(rows, cols) + 256,), 77, device="cuda", dtype=torch.uint8)
    dg, db = torch.full((cols + 2,), 7.0, device="cuda"), torch.full((cols + 2,), 7.0, device="cuda")
    mean, rstd = mean[1:-1].clone(), rstd[1:-1].clone()
    call = lambda: api.gs_layer_norm_backward(ctx, dy, x, gamma, mean, rstd, dx.t, dg[1:-1], db[1:-1], ws[:-256])
    call()
    m, r, D = mean.double()[:, None], rstd.double()[:, None], dy.double()
    h = (X - m) * r
    e_h = 2 * U32 * h.abs()
    g = D * G
    avg_g, avg_gh = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    e_g = U32 * g.abs()
    e_avg_g, e_avg_gh = (k + U32) * g.abs().mean(1, keepdim=True), (k + 4 * U32) * (g * h).abs().mean(1, keepdim=True)
    want = r * (g - avg_g - h * avg_gh)
    e_x = r * (e_g + e_avg_g + h.abs() * e_avg_gh + e_h * avg_gh.abs() + 4 * U32 * (g.abs() + avg_g.abs() + (h * avg_gh).abs()))
    close(dx.check(), want, e_x * 1.01 + step * want.abs() * 1.01 + tiny, "dx")
    n = rows + 16                                   # additions of a column
    close(dg[1:-1], (D * h).sum(0), ((D.abs() * e_h).sum(0) + n * U32 * (D * h).abs().sum(0)) * 1.01 + 1e-37, "dgamma")
    close(db[1:-1], D.sum(0), n * U32 * D.abs().sum(0) * 1.01 + 1e-37, "dbeta")
    assert all(float(t[i]) == 7 for t in (dg, db) for i in (0, -1)) and torch.all(ws[-256:] == 77)
    first = [t.clone() for t in (dx.t, dg, db)]
    call()
    assert all(torch.equal(a, b) for a, b in zip(first, (dx.t, dg, db))), "two calls differ"


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("cols", COLS)
def test_columns(ctx, cols, dtype):
    check(ctx, 37, cols, _types()[dtype], seed=cols)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("cols", [1, 5, 45, 130, 700, 3001, 8191])
def test_rows_that_are_not_aligned(ctx, cols, dtype):
    check(ctx, 29, cols, _types()[dtype], ld=cols, offset=1, seed=cols)
    check(ctx, 29, cols, _types()[dtype], ld=cols + 8, offset=8, seed=cols, aligned_dy=False)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows", [1, 2, 31, 255, 4099, 150_001])
def test_rows(ctx, rows, dtype):
    check(ctx, rows, 24, _types()[dtype], seed=rows)
    check(ctx, min(rows, 9001), 264, _types()[dtype], ld=272, seed=rows, affine=False)


def test_a_mean_far_above_the_spread(ctx):
    import torch
    check(ctx, 50, 200, torch.float32, mean_of=1000.0, spread=0.1, seed=3)


def test_rows_without_spread_and_rows_with_a_nan(ctx):
    import torch
    from paper_2609_05255_b200 import api
    x = torch.randn((70, 96), device="cuda")
    x[3], x[40], x[68, 5], x[69, 7] = 2.5, 0.0, float("nan"), float("inf")
    gamma, beta = torch.randn(96, device="cuda"), torch.randn(96, device="cuda")
    y, clean = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(70, device="cuda"), torch.empty(70, device="cuda")
    api.gs_layer_norm_forward(ctx, x, gamma, beta, y, mean=mean, rstd=rstd, eps=1e-5)
    assert torch.equal(y[3], beta) and torch.equal(y[40], beta)
    api.gs_layer_norm_forward(ctx, x.nan_to_num(0.0, 0.0), gamma, beta, clean)
    assert torch.equal(y[:68], clean[:68]) and bool(y[68:].isnan().all())
    dx = torch.empty_like(x)
    api.gs_layer_norm_backward(ctx, torch.ones_like(x), x, gamma, mean, rstd, dL_dx=dx)
    assert bool(dx[:68].isfinite().all()) and bool(dx[68:].isnan().all())


def test_in_place_missing_parts_and_no_rows(ctx):
    import torch
    from paper_2609_05255_b200 import api
    x, dy = torch.randn((300, 80), device="cuda").bfloat16(), torch.randn((300, 80), device="cuda").bfloat16()
    gamma = torch.randn(80, device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty(300, device="cuda"), torch.empty(300, device="cuda")
    api.gs_layer_norm_forward(ctx, x, gamma, None, y, mean=mean, rstd=rstd)
    same = x.clone()
    api.gs_layer_norm_forward(ctx, same, gamma, None, same)
    assert torch.equal(same, y)
    dx, dg, db = torch.empty_like(x), torch.empty(80, device="cuda"), torch.empty(80, device="cuda")
    ws = torch.empty((api.gs_layer_norm_workspace_bytes(300, 80),), device="cuda", dtype=torch.uint8)
    api.gs_layer_norm_backward(ctx, dy, x, gamma, mean, rstd, dx, dg, db, ws)
    for target in (0, 1):                                            # over dL_dy, over x
        a, b = dy.clone(), x.clone()
        api.gs_layer_norm_backward(ctx, a, b, gamma, mean, rstd, dL_dx=(a, b)[target])
        assert torch.equal((a, b)[target], dx)
    one = torch.empty(80, device="cuda")
    api.gs_layer_norm_backward(ctx, dy, x, gamma, mean, rstd, dL_dgamma=one, workspace=ws)
    assert torch.equal(one, dg)
    api.gs_layer_norm_backward(ctx, dy, x, gamma, mean, rstd, dL_dbeta=one, workspace=ws)
    assert torch.equal(one, db)
    none, stat = x[:0], mean[:0]
    api.gs_layer_norm_forward(ctx, none, gamma, None, none.clone())
    api.gs_layer_norm_backward(ctx, none, none, gamma, stat, stat, dL_dgamma=dg, dL_dbeta=db, workspace=ws)
    assert torch.all(dg == 0) and torch.all(db == 0)


def test_gradient_by_differences(ctx):
    import torch
    from paper_2609_05255_b200 import api
    x, g, gamma = torch.randn((9, 33), device="cuda"), torch.randn((9, 33), device="cuda"), torch.randn(33, device="cuda")
    y, mean, rstd, dx = torch.empty_like(x), torch.empty(9, device="cuda"), torch.empty(9, device="cuda"), torch.empty_like(x)
    api.gs_layer_norm_forward(ctx, x, gamma, None, y, mean=mean, rstd=rstd)
    api.gs_layer_norm_backward(ctx, g, x, gamma, mean, rstd, dL_dx=dx)

    def f(X):
        X = X - X.mean(1, keepdim=True)
        return (X * (X.square().mean(1, keepdim=True) + 1e-5).rsqrt() * gamma.double() * g.double()).sum()
    for i, j in ((0, 0), (4, 17), (8, 32)):
        E = torch.zeros((9, 33), device="cuda", dtype=torch.float64)
        E[i, j] = 1e-4
        d = (f(x.double() + E) - f(x.double() - E)) / 2e-4
        # h^2 / 6 times a third derivative of order rstd^3 |g gamma|, and the fp32 statistics
        assert abs(float(d) - float(dx[i, j])) <= 2e-6 * float((g[i] * gamma).abs().sum())


def test_graph(ctx):
    import torch
    from paper_2609_05255_b200 import api
    x, gamma = torch.randn((500, 48), device="cuda").half(), torch.randn(48, device="cuda")
    y, want = torch.empty_like(x), torch.empty_like(x)
    api.gs_layer_norm_forward(ctx, x, gamma, None, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.gs_layer_norm_forward(ctx, x, gamma, None, y)
    y.fill_(0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want)


def test_refusals(ctx):
    import torch
    from paper_2609_05255_b200 import api
    z = lambda *s: torch.zeros(s, device="cuda")

    def refused(status, f):
        with pytest.raises(api.GsError) as e:
            f()
        assert e.value.status == status and str(e.value)
    bad = api.GS_ERR_INVALID_ARG
    refused(bad, lambda: api.gs_layer_norm_forward(ctx, z(4, 8), None, None, z(4, 9)))
    refused(bad, lambda: api.gs_layer_norm_forward(ctx, z(4, 8), z(9), None, z(4, 8)))
    refused(bad, lambda: api.gs_layer_norm_forward(ctx, z(4, 8), z(8).half(), None, z(4, 8)))
    refused(bad, lambda: api.gs_layer_norm_forward(ctx, z(4, 8).double(), None, None, z(4, 8)))
    refused(bad, lambda: api.gs_layer_norm_forward(ctx, z(4, 8), None, None, z(4, 8).cpu()))
    refused(bad, lambda: api.gs_layer_norm_forward(ctx, z(4, 8), None, None, z(4, 8), eps=0.0))
    refused(bad, lambda: api.gs_layer_norm_forward(ctx, z(4, 8), None, None, z(4, 8), eps=float("nan")))
    refused(bad, lambda: api.gs_layer_norm_forward(ctx, z(2, 8193), None, None, z(2, 8193)))
    refused(bad, lambda: api.gs_layer_norm_forward(ctx, z(8, 4).T, None, None, z(4, 8)))
    ws = torch.zeros((api.gs_layer_norm_workspace_bytes(4, 8),), device="cuda", dtype=torch.uint8)
    refused(bad, lambda: api.gs_layer_norm_backward(ctx, z(4, 8), z(4, 8), None, None, z(4), z(4, 8)))
    refused(bad, lambda: api.gs_layer_norm_backward(ctx, z(4, 8), z(4, 8), None, z(4), z(4), z(4, 8), z(8), z(8)))
    refused(api.GS_ERR_CAPACITY, lambda: api.gs_layer_norm_backward(ctx, z(4, 8), z(4, 8), None, z(4), z(4), z(4, 8), z(8), z(8), ws[:-16]))
