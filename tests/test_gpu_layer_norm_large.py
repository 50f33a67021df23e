"""Layer norm's backward on rows whose mean, in units of the spread, leaves fp32's range: the lanes that hold no column of the row
add nothing to its sums, also where (0 - mean) rstd is infinite."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2609_05255_b200 import api
    c = api.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols,ld", [(2, 8), (5, 8), (5, 5), (45, 48), (45, 45), (100, 104), (130, 131), (700, 704), (1030, 1032), (2500, 2501), (8190, 8192)])
def test_large_rows_without_spread(ctx, cols, ld, dtype):
    import torch
    from layer_helpers import HALF_STEP, HALF_TINY, U32, Guarded, close
    from paper_2609_05255_b200 import api
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(cols)
    randn = lambda *s: torch.randn(s, device="cuda", generator=gen)
    rows = 9
    value = torch.where(torch.arange(rows, device="cuda") % 2 == 0, 2.0 ** 126, -(2.0 ** 122))[:, None]
    x = Guarded(rows, cols, dt, ld, value.expand(rows, cols)).t
    dy = Guarded(rows, cols, dt, ld, randn(rows, cols)).t
    gamma = 1 + 0.3 * randn(cols)
    # the statistics of such rows: their value, and 1 / sqrt(eps)
    mean, rstd = value[:, 0].clone(), torch.full((rows,), 316.0, device="cuda")
    dx = Guarded(rows, cols, dt, ld)
    dg, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty((api.gs_layer_norm_workspace_bytes(rows, cols),), device="cuda", dtype=torch.uint8)
    api.gs_layer_norm_backward(ctx, dy, x, gamma, mean, rstd, dx.t, dg, db, ws)
    # h = 0: dx = rstd (g - avg(g)).  g is rounded once; its sum by a lane of up to 32 values, five exchanges and eight warps, and the
    # division: 48 roundings of half a step; the difference and the product with rstd: one each
    g = dy.double() * gamma.double()
    avg = g.mean(1, keepdim=True)
    want = 316.0 * (g - avg)
    e = 316.0 * (2 * U32 * (g.abs() + avg.abs()) + 24 * U32 * g.abs().mean(1, keepdim=True))
    close(dx.check(), want, e * 1.01 + HALF_STEP[dt] * want.abs() * 1.01 + HALF_TINY[dt], "dx")
    assert torch.all(dg == 0)
    close(db, dy.double().sum(0), (rows + 16) * U32 * dy.double().abs().sum(0) * 1.01, "dbeta")
