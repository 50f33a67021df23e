"""The dense backward over many rows: every CTA of the weights' gradient empties its accumulator several times.

On small whole numbers every product and sum is exact, in whatever order and in however many parts it is taken, so the gradients have to be
equal to the true ones: a step, a group of steps or a split that is lost, taken twice or mixed up with another shows.  On positive numbers
the sums are as large as the sums of absolute values, so what the tensor core cuts off in a long chain of additions shows."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2609_05255_b200 import api
    c = api.Context(0)
    yield c
    api.gs_async_status(c)
    c.close()


def _types():
    import torch
    return {"f16": torch.float16, "bf16": torch.bfloat16}


def padded(rows, cols, dtype):
    import torch
    return torch.zeros((rows, (cols + 7) // 8 * 8), device="cuda", dtype=dtype)[:, :cols]


def backward(ctx, act, x, w, z, dy):
    import torch
    from paper_2609_05255_b200 import api
    (rows, cin), cout = x.shape, w.shape[0]
    dx, dw, db = padded(rows, cin, x.dtype), torch.empty((cout, cin), device="cuda"), torch.empty((cout,), device="cuda")
    ws = torch.empty((api.gs_dense_workspace_bytes(rows, cin, cout),), device="cuda", dtype=torch.uint8)
    api.gs_dense_backward(ctx, api.DenseLayer(w, None, act), x, dy, preact=None if act == "none" else z, dL_dx=dx, dL_dweight=dw, dL_dbias=db, workspace=ws)
    return dx, dw, db


# (rows, in, out), on 148 SMs steps of 64 rows per split: 64 in pairs; 79 in pairs, several column tiles; 20 alone; 43 of one narrow tile; 79 in one
# split, pairs and alone; 9, so that the last group is one step; 17 in the last of which 7 rows are left
SHAPES = [(300_007, 256, 256), (20_011, 1024, 1024), (60_001, 256, 384), (400_003, 72, 40), (5_003, 2048, 2048), (5_003, 2048, 1900), (9 * 64 * 148, 64, 128),
          (64 * 148 * 16 + 7, 130, 120)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("rows,cin,cout", SHAPES)
def test_whole_numbers(ctx, rows, cin, cout, act, dtype):
    import torch
    dt = _types()[dtype]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(rows)
    whole = lambda r, c, most: padded(r, c, dt).copy_(torch.randint(-most, most + 1, (r, c), device="cuda", generator=gen))
    x, w, dy = whole(rows, cin, 4), whole(cout, cin, 1), whole(rows, cout, 2)
    # the derivative is 1 at 100; ReLU passes the rows where z is 1 and stops those where it is -1
    z = padded(rows, cout, dt).fill_(100.0)
    passes = torch.ones((rows, 1), device="cuda", dtype=torch.float64)
    if act == "relu":
        passes = (torch.rand((rows, 1), device="cuda", generator=gen) < 0.7).double()
        z.copy_((2 * passes - 1).expand(rows, cout))
    dx, dw, db = backward(ctx, act, x, w, z, dy)
    dz = dy.double() * passes
    # (the sums stay below 2^24: at most 8 x 400 003)
    assert torch.equal(dw.double(), dz.T @ x.double())
    assert torch.equal(db.double(), dz.sum(0))
    assert torch.equal(dx, (dz @ w.double()).to(dt))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("rows,cin,cout", [(40_037, 2048, 1024), (40_037, 2048, 900), (20_011, 2048, 2048), (1_000_003, 64, 48)])
def test_positive_numbers(ctx, rows, cin, cout, act, dtype):
    """dW of 40 037 rows in two splits: 313 steps, 1252 products added up one after another, each of which may cut off a step of the sum;
    left in one accumulator sums were off by about nine tenths of that (9e-5 in 845), here 1.3e-4: more than three times what the bound allows."""
    import torch
    from layer_helpers import HALF_STEP, U32, act as act64, act_grad_error, close
    dt = _types()[dtype]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(rows + cout)
    rand = lambda r, c, lo, hi: padded(r, c, dt).copy_(lo + (hi - lo) * torch.rand((r, c), device="cuda", generator=gen))
    x, w, z, dy = rand(rows, cin, 0.5, 1.5), rand(cout, cin, 0.5, 1.5), rand(rows, cout, 0.5, 3.0), rand(rows, cout, 0.5, 1.5)
    _, dw, db = backward(ctx, act, x, w, z, dy)
    smooth = act in ("silu", "gelu")
    h = HALF_STEP[dt]
    slope = act64(act, z.double())[1]
    dz = dy.double() * slope
    want = dz.T @ x.double()
    # of dz: the derivative's error and the product's rounding, and what the last part leaves
    e_dz = dy.double() * act_grad_error(act, z.double()) + U32 * dz + ((h ** 3 if dtype == "bf16" else h * h) * dz + 2.0 ** -36) if smooth else torch.zeros_like(dz)
    # A product of 16 rows and the sum so far are 17 terms, each cut off at most half a step (U32 / 2) of the largest: 8.5 steps.  32 of them,
    # then the sum goes to a register, rounded to nearest; the splits' sums are added in 64 bits and rounded once.  The lower parts, at most
    # h of dz, stay in their accumulator for the whole split; ReLU and none have one part.
    splits = max(1, min(148 // (-(-cout // 128) * -(-cin // 256)), -(-rows // 512)))
    steps = -(-rows // 64) / splits + 1
    chain = 32 * 8.5 + steps / 8 + 3 + (smooth * 2 * 4 * steps * 8.5 * h)
    close(dw, want, (e_dz.T @ x.double() + chain * U32 * want) * 1.01, "dW")
    # db: a lane adds four rows a step, then 16 lanes, then the splits in 64 bits
    close(db, dz.sum(0), (e_dz.sum(0) + (4 * steps + 20) * U32 * dz.sum(0)) * 1.01, "db")
