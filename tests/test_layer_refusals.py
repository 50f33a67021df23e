"""What the layers and the clipping refuse, without a GPU: the C entry points check their arguments before the first CUDA call, so
a zeroed block of memory stands in for the context (only its text of the last error is written), and the addresses are never read."""
import ctypes as C
import math

import pytest

A = 1 << 20                       # an address of the right alignment
BAD, CAPACITY, UNSUPPORTED = -1, -2, -4


@pytest.fixture(scope="module")
def api():
    from paper_2609_05255_b200 import build
    build.build()
    from paper_2609_05255_b200 import api
    return api


@pytest.fixture(scope="module")
def ctx():
    return C.create_string_buffer(1 << 16)


def layer(api, **change):
    s = api.GsDenseLayer(A, 16, A, 16, 24, api.GS_TYPE_F16, api.GS_DENSE_SILU)
    for k, v in change.items():
        setattr(s, k, v)
    return s


def test_dense_forward(api, ctx):
    f = api._lib.gs_dense_forward
    call = lambda l, rows=5, x=A, lx=16, r=None, lr=0, y=A, ly=24, z=None, lz=0: f(ctx, l, rows, x, lx, r, lr, y, ly, z, lz, None)
    assert f(None, layer(api), 5, A, 16, None, 0, A, 24, None, 0, None) == BAD
    assert call(layer(api), rows=0) == 0
    for change in (dict(weight=None), dict(weight=A + 2), dict(ld_weight=15), dict(ld_weight=8), dict(ld_weight=20), dict(in_features=0), dict(out_features=0),
                   dict(in_features=16385, ld_weight=16392), dict(dtype=3), dict(dtype=-1), dict(activation=4), dict(activation=-1), dict(bias=A + 1)):
        assert call(layer(api, **change)) == BAD, change
    assert call(layer(api, dtype=api.GS_TYPE_F32)) == UNSUPPORTED
    assert call(layer(api), rows=-1) == BAD and call(layer(api), rows=1 << 31) == CAPACITY
    for change in (dict(x=None), dict(x=A + 8), dict(lx=8), dict(lx=17), dict(lx=-16), dict(y=None), dict(y=A + 4), dict(ly=16), dict(ly=25),
                   dict(r=A + 2, lr=24), dict(r=A, lr=23), dict(z=A + 2, lz=24), dict(z=A, lz=0)):
        assert call(layer(api), **change) == BAD, change


def test_dense_backward(api, ctx):
    f = api._lib.gs_dense_backward
    size = api.gs_dense_workspace_bytes(5, 16, 24)

    def call(l=None, rows=5, x=A, lx=16, z=A, lz=24, dy=A, ld=24, dx=A, ldx=16, dw=A, db=A, ws=A, n=size):
        return f(ctx, l or layer(api), rows, x, lx, z, lz, dy, ld, dx, ldx, dw, db, ws, n, None)
    for change in (dict(z=None), dict(lz=16), dict(dy=None), dict(ld=20), dict(dx=A + 2), dict(ldx=12), dict(x=None), dict(lx=9), dict(ws=None), dict(ws=A + 8),
                   dict(dw=None), dict(dw=A + 2), dict(db=A + 1), dict(rows=-1)):
        assert call(**change) == BAD, change
    assert call(n=size - 1) == CAPACITY and call(rows=1 << 31) == CAPACITY


def test_workspaces(api):
    assert api.gs_dense_workspace_bytes(-1, 8, 8) == 0 and api.gs_dense_workspace_bytes(1 << 31, 8, 8) == 0
    assert api.gs_dense_workspace_bytes(5, 0, 8) == 0 and api.gs_dense_workspace_bytes(5, 8, 16385) == 0
    assert api.gs_layer_norm_workspace_bytes(-1, 8) == 0 and api.gs_layer_norm_workspace_bytes(5, 0) == 0 and api.gs_layer_norm_workspace_bytes(5, 8193) == 0
    for k, n in ((8, 8), (63, 256), (256, 256), (1024, 1000)):
        sizes = [api.gs_dense_workspace_bytes(m, k, n) for m in [*range(0, 3000, 7), *range(3000, 3_000_000, 9973)]]
        assert all(a <= b for a, b in zip(sizes, sizes[1:])) and sizes[0] >= 4 * n * (k + 1)      # one serves every smaller scene
    sizes = [api.gs_layer_norm_workspace_bytes(m, 45) for m in range(0, 3000)]
    assert all(a <= b for a, b in zip(sizes, sizes[1:])) and sizes[0] > 0
    assert api.gs_grad_workspace_bytes() >= 8


def test_layer_norm(api, ctx):
    f = api._lib.gs_layer_norm_forward
    call = lambda t=0, rows=5, cols=9, x=A, lx=9, g=A, b=A, eps=1e-5, y=A, ly=9, m=A, r=A: f(ctx, t, rows, cols, x, lx, g, b, eps, y, ly, m, r, None)
    assert call(rows=0) == 0
    for change in (dict(t=3), dict(rows=-1), dict(cols=0), dict(cols=8193, lx=8193, ly=8193), dict(x=None), dict(x=A + 2), dict(lx=8), dict(y=None), dict(ly=-9),
                   dict(g=A + 2), dict(b=A + 1), dict(m=A + 2), dict(r=A + 3), dict(eps=0.0), dict(eps=-1.0), dict(eps=math.nan)):
        assert call(**change) == BAD, change
    assert call(rows=1 << 31) == CAPACITY
    f2 = api._lib.gs_layer_norm_backward
    size = api.gs_layer_norm_workspace_bytes(5, 9)

    def back(t=1, rows=5, cols=9, dy=A, ld=9, x=A, lx=9, g=A, m=A, r=A, dx=A, ldx=9, dg=A, db=A, ws=A, n=size):
        return f2(ctx, t, rows, cols, dy, ld, x, lx, g, m, r, dx, ldx, dg, db, ws, n, None)
    for change in (dict(t=-1), dict(dy=None), dict(dy=A + 1), dict(ld=8), dict(x=None), dict(lx=0), dict(m=None), dict(r=None), dict(m=A + 2), dict(dx=A + 1),
                   dict(ldx=7), dict(dg=A + 2), dict(db=A + 2), dict(ws=None), dict(ws=A + 8)):
        assert back(**change) == BAD, change
    assert back(n=size - 1) == CAPACITY


def test_gradient_norm(api, ctx):
    size = api.gs_grad_workspace_bytes()
    more = (C.c_void_p * 8)(*[A] * 8)

    def tensor(grad=A, out=A, count=10, dtype=0, buffers=0, pointers=more):
        return api.GsGradTensor(grad, out, count, dtype, pointers, buffers)

    def call(t=None, n=1, norm=1.0, clip=A, ws=A, bytes=size, f=api._lib.gs_clip_grads):
        return f(ctx, (api.GsGradTensor * max(1, abs(n)))(*[t or tensor()] * max(1, abs(n))), n, norm, clip, ws, bytes, None)
    for t in (tensor(grad=None), tensor(grad=A + 2), tensor(grad=A + 1, dtype=1), tensor(out=None), tensor(out=A + 2), tensor(count=-1), tensor(dtype=3),
              tensor(buffers=8), tensor(buffers=-1), tensor(buffers=1, pointers=None), tensor(buffers=1, pointers=(C.c_void_p * 1)(A + 2))):
        assert call(t) == BAD
    for change in (dict(n=-1), dict(n=513), dict(norm=0.0), dict(norm=-1.0), dict(norm=math.nan), dict(clip=None), dict(clip=A + 4), dict(ws=None), dict(ws=A + 8)):
        assert call(**change) == BAD, change
    assert call(tensor(buffers=7), n=200) == BAD                           # 1400 further buffers
    assert call(bytes=size - 1) == CAPACITY and call(tensor(count=1 << 40)) == CAPACITY
    adam = (api.GsAdamTensor * 1)(api.GsAdamTensor(A, A, A, A, None, 2, 3, (C.c_float * 3)(1, 1, 1), 0.9, 0.999, 1e-8, None, 0))
    f = api._lib.gs_adam_step_clipped
    assert f(ctx, adam, 1, 1, None, None) == BAD and f(ctx, adam, 1, 1, A + 4, None) == BAD
    assert f(ctx, adam, 1, 0, A, None) == BAD and f(ctx, adam, 9, 1, A, None) == BAD


def test_the_binding_refuses_tensors_of_another_kind(api):
    import torch
    from types import SimpleNamespace
    cpu = SimpleNamespace(device=torch.device("cpu"))
    x = torch.zeros((4, 16), dtype=torch.float16)
    assert api._matrix(cpu, x, "x", 4, 16, torch.float16)[1] == 16 and api._matrix(cpu, None, "x", 4, 16, torch.float16) == (None, 0)
    assert api._matrix(cpu, x[:, :13], "x", 4, 13, torch.float16)[1] == 16
    for t, shape, dtype in ((x, (4, 15), torch.float16), (x, (4, 16), torch.bfloat16), (x.T, (16, 4), torch.float16), (x[0], (16, 1), torch.float16),
                            (x.to("meta"), (4, 16), torch.float16)):
        with pytest.raises(api.GsError) as e:
            api._matrix(cpu, t, "x", *shape, dtype)
        assert e.value.status == BAD
    for v in (torch.zeros(5), torch.zeros(4, dtype=torch.float64), torch.zeros(8)[::2]):
        with pytest.raises(api.GsError):
            api._vector(cpu, v, "v", 4)
    with pytest.raises(api.GsError):
        api.DenseLayer(x)                                                  # not on a GPU
    with pytest.raises(api.GsError):
        api.GradList([api.GradTensor(torch.zeros(4))])
