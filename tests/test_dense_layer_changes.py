"""A DenseLayer whose tensors change between calls: the struct that a call passes on is that of the tensors as they are now.  No GPU: the
tensors stay on the CPU and no entry point is called."""
from types import SimpleNamespace

import pytest


@pytest.fixture(scope="module")
def api():
    from paper_2609_05255_b200 import build
    build.build()
    from paper_2609_05255_b200 import api
    return api


def make(api):
    import torch
    layer = object.__new__(api.DenseLayer)               # (the constructor wants CUDA tensors)
    layer.weight, layer.bias = torch.zeros((4, 16), dtype=torch.float16), torch.zeros(4)
    layer._struct = api.GsDenseLayer(None, 0, None, 16, 4, api.GS_TYPE_F16, api.GS_DENSE_RELU)
    return layer, SimpleNamespace(device=torch.device("cpu"))


def test_type_and_memory_are_those_of_the_weight_now(api):
    import torch
    layer, ctx = make(api)
    assert api._layer(ctx, layer).dtype == api.GS_TYPE_F16
    layer.weight.data = torch.zeros((4, 24), dtype=torch.bfloat16)[:, :16]
    s = api._layer(ctx, layer)
    assert (s.dtype, s.ld_weight, s.weight) == (api.GS_TYPE_BF16, 24, layer.weight.data_ptr())
    layer.weight.data = torch.zeros((4, 16))
    assert api._layer(ctx, layer).dtype == api.GS_TYPE_F32        # (which the entry points refuse)


def test_weights_that_are_refused(api):
    import torch
    layer, ctx = make(api)
    for weight in (torch.zeros((4, 32), dtype=torch.float16)[:, ::2], torch.zeros((16, 4), dtype=torch.float16).T, torch.zeros((4, 16), dtype=torch.float64),
                   torch.zeros((4, 17), dtype=torch.float16), torch.zeros((64,), dtype=torch.float16)):
        layer.weight = weight
        with pytest.raises(api.GsError) as e:
            api._layer(ctx, layer)
        assert e.value.status == api.GS_ERR_INVALID_ARG


def test_a_bias_that_comes_and_goes(api):
    import torch
    layer, ctx = make(api)
    assert api._layer(ctx, layer).bias == layer.bias.data_ptr()
    layer.bias = None
    assert api._layer(ctx, layer).bias is None
    layer.bias = torch.ones(4)
    assert api._layer(ctx, layer).bias == layer.bias.data_ptr()
    layer.bias = torch.ones(5)
    with pytest.raises(api.GsError):
        api._layer(ctx, layer)


@pytest.mark.gpu
def test_a_layer_that_became_bf16_and_lost_its_bias():
    import torch
    from paper_2609_05255_b200 import api
    ctx = api.Context(0)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    randn = lambda *s: torch.randn(s, device="cuda", generator=gen)
    w, b, x = randn(40, 24), randn(40), randn(70, 24)
    layer = api.DenseLayer(w.half(), b, "silu")
    y = torch.empty((70, 40), device="cuda", dtype=torch.float16)
    api.gs_dense_forward(ctx, layer, x.half(), y)
    layer.weight.data, layer.bias = w.bfloat16(), None
    y, want = (torch.empty((70, 40), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    api.gs_dense_forward(ctx, layer, x.bfloat16(), y)
    api.gs_dense_forward(ctx, api.DenseLayer(w.bfloat16(), None, "silu"), x.bfloat16(), want)
    assert torch.equal(y, want)
    ctx.close()
