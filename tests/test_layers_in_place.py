"""Outputs in the place of an input (y of the residual or of x, dL_dx of dL_dy or of x) have its row stride: with another one, rows
would be written over others that are still to be read.  No GPU: the calls are refused before the first CUDA call."""
import ctypes as C

import pytest

A, B, D = 1 << 20, 1 << 21, 1 << 22            # addresses of the right alignment, never read
BAD, CAPACITY = -1, -2


@pytest.fixture(scope="module")
def api():
    from paper_2609_05255_b200 import build
    build.build()
    from paper_2609_05255_b200 import api
    return api


@pytest.fixture(scope="module")
def ctx():
    return C.create_string_buffer(1 << 16)


def error(api, ctx):
    return api._lib.gs_last_error(ctx).decode()


def test_dense_residual(api, ctx):
    layer = api.GsDenseLayer(A, 16, None, 16, 24, api.GS_TYPE_F16, api.GS_DENSE_SILU)
    f = api._lib.gs_dense_forward
    assert f(ctx, layer, 2, A, 16, B, 32, B, 24, None, 0, None) == BAD and "residual" in error(api, ctx)


def test_layer_norm(api, ctx):
    f = api._lib.gs_layer_norm_forward
    assert f(ctx, 0, 2, 9, A, 12, None, None, 1e-5, A, 9, None, None, None) == BAD and "ld" in error(api, ctx)
    f = api._lib.gs_layer_norm_backward
    size = api.gs_layer_norm_workspace_bytes(5, 9)
    for out, ld in ((A, 10), (B, 10)):
        assert f(ctx, 0, 5, 9, A, 9, B, 9, None, D, D, out, ld, None, None, D, size, None) == BAD and "dL_dx" in error(api, ctx)
    # the place itself is accepted: the next check is reached
    for out in (A, B):
        assert f(ctx, 0, 5, 9, A, 9, B, 9, None, D, D, out, 9, D, None, D, size - 1, None) == CAPACITY
