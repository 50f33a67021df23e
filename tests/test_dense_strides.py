"""Row strides of dense layers that no tensor map can hold (2^38 elements and more) are refused as arguments, before anything is
launched.  No GPU: the calls return before the first CUDA call."""
import ctypes as C

import pytest

A, FAR = 1 << 20, 1 << 38
BAD = -1


@pytest.fixture(scope="module")
def api():
    from paper_2609_05255_b200 import build
    build.build()
    from paper_2609_05255_b200 import api
    return api


@pytest.fixture(scope="module")
def ctx():
    return C.create_string_buffer(1 << 16)


def layer(api, ld=16):
    return api.GsDenseLayer(A, ld, None, 16, 24, api.GS_TYPE_F16, api.GS_DENSE_SILU)


@pytest.mark.parametrize("far", [FAR, FAR * 4, (1 << 62)])
def test_far_rows(api, ctx, far):
    f = api._lib.gs_dense_forward
    call = lambda l, lx=16, lr=24, ly=24, lz=24: f(ctx, l, 5, A, lx, A * 2, lr, A * 3, ly, A * 4, lz, None)
    assert call(layer(api, far)) == BAD
    for change in (dict(lx=far), dict(lr=far), dict(ly=far), dict(lz=far)):
        assert call(layer(api), **change) == BAD, change
    f2 = api._lib.gs_dense_backward
    size = api.gs_dense_workspace_bytes(5, 16, 24)
    back = lambda l, lx=16, lz=24, ld=24, ldx=16: f2(ctx, l, 5, A, lx, A, lz, A, ld, A, ldx, A, A, A, size, None)
    assert back(layer(api, far)) == BAD
    for change in (dict(lx=far), dict(lz=far), dict(ld=far), dict(ldx=far)):
        assert back(layer(api), **change) == BAD, change
