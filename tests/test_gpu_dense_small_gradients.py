"""The dense backward in fp16 on gradients far below one: dz is carried in two parts, 22 bits of it and nothing coarser than 2^-36,
into dL_dx as into dL_dweight."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2609_05255_b200 import api
    c = api.Context(0)
    yield c
    api.gs_async_status(c)
    c.close()


# (rows, in, out): a narrow tile, tiles by pairs, weights that come with every step, several tiles per CTA of each kind, and a last tile of few
# columns beside wide ones
SHAPES = [(70, 24, 256), (1001, 64, 136), (1000, 256, 256), (700, 700, 520), (148 * 128 * 2 + 77, 40, 64), (148 * 256 + 300, 256, 72), (148 * 128 + 5, 264, 1024),
          (148 * 128 * 3 + 9, 264, 72), (148 * 128 * 2 + 1, 520, 200), (148 * 256 + 3, 264, 328)]


@pytest.mark.parametrize("size", [1e-2, 1e-5, 1e-7])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("rows,cin,cout", SHAPES)
def test_gradients_of_small_size(ctx, rows, cin, cout, act, size):
    import torch
    from layer_helpers import HALF_STEP, HALF_TINY, U32, act as act64, act_grad_error, close
    from paper_2609_05255_b200 import api
    gen = torch.Generator(device="cuda")
    gen.manual_seed(rows + cout)
    randn = lambda *s: torch.randn(s, device="cuda", generator=gen)
    half = torch.float16
    # weights of one, so that what dz has lost is larger than dx's own rounding
    padded = lambda r, c: torch.zeros((r, (c + 7) // 8 * 8), device="cuda", dtype=half)[:, :c]
    x, w, z, dy = padded(rows, cin), padded(cout, cin), padded(rows, cout), padded(rows, cout)
    for t, scale in ((x, 1), (w, 1), (z, 1), (dy, size)):
        t.copy_(randn(*t.shape) * scale)
    layer = api.DenseLayer(w, None, act)
    dx, dw, db = padded(rows, cin), torch.empty((cout, cin), device="cuda"), torch.empty((cout,), device="cuda")
    ws = torch.empty((api.gs_dense_workspace_bytes(rows, cin, cout),), device="cuda", dtype=torch.uint8)
    api.gs_dense_backward(ctx, layer, x, dy, preact=z, dL_dx=dx, dL_dweight=dw, dL_dbias=db, workspace=ws)
    h = HALF_STEP[half]
    dz = dy.double() * act64(act, z.double())[1]
    # of dz: the derivative's error and the product's rounding; the first part leaves half a step (2^-11, among the subnormals
    # 2^-25), the second half a step of that (2^-22), or 2^-25 of its own subnormals, which count 2^-11 as much
    e_dz = dy.double().abs() * act_grad_error(act, z.double()) + U32 * dz.abs() + h * h * dz.abs() + 2.0 ** -36
    # of dx: every addition on the tensor core may lose a step (U32) of the largest it has summed up to; `cout` products in each part
    # (groups of 16 are one addition or more), the parts' sum, and the rounding to fp16
    wa = w.double().abs()
    want = dz @ w.double()
    bound = e_dz @ wa + (2 * cout + 2) * U32 * (dz.abs() @ wa)
    close(dx, want, bound * 1.01 + h * want.abs() * 1.01 + HALF_TINY[half], "dx")
    xa = x.double().abs()
    close(dw, dz.T @ x.double(), (e_dz.T @ xa + (3 * rows + 4) * U32 * (dz.abs().T @ xa)) * 1.01 + 1e-37, "dW")
