"""The layers as they are used together: a trunk over the Gaussians (layer norm, a dense layer, a residual layer, a head) gives the
decoder its features; the decoder's backward pass goes on into the trunk; all gradients, the decoder's and the scene's among them,
are clipped by their common norm and updated."""
import math

import pytest

pytestmark = pytest.mark.gpu

N, WIDTH, HIDDEN = 3001, 32, 64


class Trunk:
    def __init__(self, ctx, seed):
        import numpy as np
        import torch
        from paper_2609_05255_b200 import api, scenes
        self.ctx = ctx
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        randn = lambda *s: torch.randn(s, device="cuda", generator=gen)
        half = lambda *s: torch.zeros(s, device="cuda", dtype=torch.float16)
        f32 = lambda *s: torch.zeros(s, device="cuda")
        # masters in fp32, and the half copies that the layers read
        self.master = dict(latent=randn(N, WIDTH), w1=randn(HIDDEN, WIDTH) / WIDTH ** 0.5, w2=randn(HIDDEN, HIDDEN) / HIDDEN ** 0.5,
                           w3=randn(8, HIDDEN) / HIDDEN ** 0.5, b1=randn(HIDDEN) * 0.1, b2=randn(HIDDEN) * 0.1, b3=randn(8) * 0.1,
                           gamma=1 + 0.1 * randn(WIDTH), beta=0.1 * randn(WIDTH))
        self.halves = {k: self.master[k].half() for k in ("latent", "w1", "w2", "w3")}
        self.l1 = api.DenseLayer(self.halves["w1"], self.master["b1"], "silu")
        self.l2 = api.DenseLayer(self.halves["w2"], self.master["b2"], "gelu")
        self.l3 = api.DenseLayer(self.halves["w3"], self.master["b3"])
        self.x0, self.z1, self.h1, self.z2, self.h2, self.features = half(N, WIDTH), half(N, HIDDEN), half(N, HIDDEN), half(N, HIDDEN), half(N, HIDDEN), half(N, 8)
        self.mean, self.rstd = f32(N), f32(N)
        self.d_features, self.d2, self.d1, self.d0, self.d_latent16 = half(N, 8), half(N, HIDDEN), half(N, HIDDEN), half(N, WIDTH), half(N, WIDTH)
        self.grad = {k: torch.zeros_like(v) for k, v in self.master.items()}
        w = scenes.config2(n=N, app=scenes.APP_NEURAL)
        self.scene = api.upload_scene(w.scene, ctx.device)
        self.scene.features = self.features
        self.weights = self.scene.mlp_weights.float()
        self.base = self.scene.base_color
        dirs = randn(N, 3)
        self.dirs = (dirs / dirs.norm(dim=1, keepdim=True)).contiguous()
        self.d_color = randn(N, 3) * 0.05
        self.color, self.d_dirs = f32(N, 3), f32(N, 3)
        self.sg = api.alloc_grads_for(self.scene, ctx.device)
        sizes = [api.gs_dense_workspace_bytes(N, a, b) for a, b in ((WIDTH, HIDDEN), (HIDDEN, HIDDEN), (HIDDEN, 8))]
        ws = max(sizes + [api.gs_layer_norm_workspace_bytes(N, WIDTH), api.gs_grad_workspace_bytes()])
        self.ws, self.clip = torch.empty((ws,), device="cuda", dtype=torch.uint8), f32(2)
        g = self.grad
        self.all = api.GradList([api.GradTensor(self.d_latent16 if k == "latent" else v) for k, v in g.items()] +
                                [api.GradTensor(self.sg.base_color), api.GradTensor(self.sg.mlp_weights)])
        zeros = lambda t: torch.zeros_like(t)
        one = lambda p, grad, h=None: api.AdamTensor(p, grad, zeros(p), zeros(p), [1e-2], half_copy=h)
        adam = [one(self.master[k], g[k], self.halves.get(k)) for k in self.master] + [one(self.base, self.sg.base_color),
                                                                                       one(self.weights, self.sg.mlp_weights, self.scene.mlp_weights)]
        self.adam = [adam[:6], adam[6:]]

    def gradients(self):
        from paper_2609_05255_b200 import api
        c, g = self.ctx, self.grad
        api.gs_layer_norm_forward(c, self.halves["latent"], self.master["gamma"], self.master["beta"], self.x0, self.mean, self.rstd)
        api.gs_dense_forward(c, self.l1, self.x0, self.h1, preact=self.z1)
        api.gs_dense_forward(c, self.l2, self.h1, self.h2, preact=self.z2, residual=self.h1)
        api.gs_dense_forward(c, self.l3, self.h2, self.features)
        api.gs_appearance_forward(c, self.scene, self.dirs, self.color)
        api.gs_appearance_backward(c, self.scene, self.dirs, self.d_color, self.sg, self.d_dirs)
        self.d_features.copy_(self.sg.features[:N])
        api.gs_dense_backward(c, self.l3, self.h2, self.d_features, dL_dx=self.d2, dL_dweight=g["w3"], dL_dbias=g["b3"], workspace=self.ws)
        api.gs_dense_backward(c, self.l2, self.h1, self.d2, preact=self.z2, dL_dx=self.d1, dL_dweight=g["w2"], dL_dbias=g["b2"], workspace=self.ws)
        self.d1.add_(self.d2)                                              # the residual's share
        api.gs_dense_backward(c, self.l1, self.x0, self.d1, preact=self.z1, dL_dx=self.d0, dL_dweight=g["w1"], dL_dbias=g["b1"], workspace=self.ws)
        api.gs_layer_norm_backward(c, self.d0, self.halves["latent"], self.master["gamma"], self.mean, self.rstd, self.d_latent16, g["gamma"], g["beta"], self.ws)
        g["latent"].copy_(self.d_latent16)

    def update(self, step, max_norm):
        from paper_2609_05255_b200 import api
        api.gs_grad_norm(self.ctx, self.all, max_norm, self.clip, self.ws)
        for tensors in self.adam:
            api.gs_adam_step_clipped(self.ctx, tensors, step, self.clip)

    def state(self):
        return [t for k in self.master for t in (self.master[k],)] + list(self.halves.values()) + [self.base, self.weights, self.scene.mlp_weights]


@pytest.fixture(scope="module")
def ctx():
    from paper_2609_05255_b200 import api
    c = api.Context(0)
    yield c
    api.gs_async_status(c)
    c.close()


def test_gradients_through_the_decoder_into_the_trunk(ctx):
    """Against automatic differentiation in 64 bits, from the features' gradient that the decoder gave.  Four roundings of the
    activations and four of the gradients to half precision lie on the way, each at most 2^-11 of a value; a layer passes an
    error on with a factor of about one, the norm and the activations' curvature with another: 8 * 2 * 2^-11, norm against norm."""
    import torch
    from layer_helpers import act
    t = Trunk(ctx, 3)
    t.gradients()
    torch.cuda.synchronize()
    D = {k: (t.halves[k] if k in t.halves else v).double().requires_grad_() for k, v in t.master.items()}
    x = D["latent"]
    x = (x - x.mean(1, keepdim=True)) * (x.var(1, correction=0, keepdim=True) + 1e-5).rsqrt() * D["gamma"] + D["beta"]
    h1 = act("silu", x @ D["w1"].T + D["b1"])[0]
    h2 = act("gelu", h1 @ D["w2"].T + D["b2"])[0] + h1
    f = h2 @ D["w3"].T + D["b3"]
    (f * t.d_features.double()).sum().backward()
    f = f.detach()
    assert float((t.features.double() - f).norm() / f.norm()) <= 2.0 ** -7
    for k, v in t.grad.items():
        off = float((v.double() - D[k].grad).norm() / D[k].grad.norm())
        assert off <= 2.0 ** -7, (k, off)


def test_update_with_the_common_norm(ctx):
    import torch
    t = Trunk(ctx, 4)
    t.gradients()
    parts = [t.d_latent16 if k == "latent" else v for k, v in t.grad.items()] + [t.sg.base_color, t.sg.mlp_weights]
    norm = math.sqrt(sum(float(p.double().square().sum()) for p in parts))
    before = {k: v.clone() for k, v in t.master.items()}
    t.update(1, norm / 3)
    torch.cuda.synchronize()
    assert abs(float(t.clip[0]) - norm) <= norm * 16 * 2.0 ** -24
    assert abs(float(t.clip[1]) - 1 / 3) <= 1e-5
    for k, v in t.master.items():                                          # the first step moves by the rate wherever there is a gradient
        moved, g = (before[k] - v).double(), t.grad[k].double()
        big = g.abs() > 1e-6
        assert bool(torch.all((moved[big] - 1e-2 * g[big].sign()).abs() <= 1e-5)), k
        if k in t.halves:
            assert torch.equal(t.halves[k], v.half())


def test_a_captured_step_is_the_eager_one(ctx):
    import torch
    from paper_2609_05255_b200 import api
    eager, other = Trunk(ctx, 5), api.Context(0)
    captured = Trunk(other, 5)
    for step in (1, 2):
        eager.gradients()
        eager.update(1, 0.5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        captured.gradients()
        captured.update(1, 0.5)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    # the decoder's weight gradient is a sum by CTAs in a fixed order as well: all of the state agrees bit for bit
    assert all(torch.equal(a, b) for a, b in zip(eager.state(), captured.state()))
    del graph
    other.close()
