"""The norm over all gradients, clipping, and the clipped Adam update: against 64 bits, and bit for bit against gs_adam_step fed
with gradients that were scaled before."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2609_05255_b200 import api
    c = api.Context(0)
    yield c
    c.close()


def make(sizes, seed, buffers=1, offset=0, scale=1.0):
    """[(buffers, out)] of the sizes, types in turn, `offset` elements behind an aligned address; outs between guards."""
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    made = []
    for i, n in enumerate(sizes):
        dt = (torch.float32, torch.float16, torch.bfloat16)[i % 3]
        bufs = [(torch.randn((n + 16,), device="cuda", generator=gen) * scale).to(dt)[offset:offset + n] for _ in range(buffers)]
        out = torch.full((n + 32,), 7.0, device="cuda", dtype=dt)
        made.append((bufs, out[8 + offset:8 + offset + n], out))
    return made


def check(ctx, made, max_norm):
    import torch
    from paper_2609_05255_b200 import api
    from layer_helpers import HALF_STEP, HALF_TINY
    ws = torch.full((api.gs_grad_workspace_bytes() + 256,), 77, device="cuda", dtype=torch.uint8)
    clip = torch.full((4,), 7.0, device="cuda")
    grads = api.GradList([api.GradTensor(b[0], more_grads=b[1:], out=o) for b, o, _ in made])
    before = [[x.clone() for x in b] for b, _, _ in made]
    api.gs_grad_norm(ctx, grads, max_norm, clip[:2], ws[:-256])
    alone = clip.clone()
    api.gs_clip_grads(ctx, grads, max_norm, clip[:2], ws[:-256])
    assert torch.equal(alone, clip) and torch.all(clip[2:] == 7) and torch.all(ws[-256:] == 77)
    sums = [sum(x.double() for x in b) for b, _, _ in made]
    size = [sum(x.double().abs() for x in b) for b, _, _ in made]
    norm = math.sqrt(sum(float((s * s).sum()) for s in sums))
    # the sums of the buffers in fp32 (half a step for each of up to seven additions), eight squares in fp32, the norm rounded
    buffers = max(len(b) for b, _, _ in made)
    e_sum = (buffers - 1) * 2.0 ** -24
    e = e_sum * math.sqrt(sum(float((s * s).sum()) for s in size)) + norm * 10 * 2.0 ** -24
    assert abs(float(clip[0]) - norm) <= e
    scale = min(1.0, max_norm / norm)
    assert abs(float(clip[1]) - scale) <= scale * (e / norm + 2.0 ** -23)
    for (b, o, whole), s, a, old in zip(made, sums, size, before):
        want, dt = s * scale, o.dtype
        bound = scale * e_sum * a + want.abs() * (e / norm + 2.0 ** -22 + HALF_STEP[dt]) + HALF_TINY[dt]
        assert bool(torch.all((o.double() - want).abs() <= bound * 1.01))
        n, at = o.numel(), o.storage_offset()
        assert torch.all(whole[:at] == 7) and torch.all(whole[at + n:] == 7)
        assert all(torch.equal(x, y) for x, y in zip(b, old))


@pytest.mark.parametrize("max_norm", [0.5, 1e9])
@pytest.mark.parametrize("offset", [0, 1, 3])
@pytest.mark.parametrize("buffers", [1, 2, 8])
@pytest.mark.parametrize("sizes", [[1], [7, 8, 9], [8191, 8192, 8193, 1, 2, 3], [100_003, 5, 70_001, 33], list(range(1, 61))])
def test_norm_and_clip(ctx, sizes, buffers, offset, max_norm):
    check(ctx, make(sizes, len(sizes) + offset, buffers, offset), max_norm)


def test_many_tensors_and_large_ones(ctx):
    check(ctx, make([(37 * i) % 501 + 1 for i in range(512)], 5, 3, 1), 1.0)
    check(ctx, make([9_000_001, 12_000_003, 11_000_007], 6, 1), 1.0)


def test_buffers_that_start_differently(ctx):
    """Boundaries of 16 bytes at other elements in every buffer: element by element."""
    made = make([1001, 20_000], 7, 3)
    shifted = [([b[0][:-3], b[1][1:-2], b[2][3:]], o[2:-1], whole) for b, o, whole in made]
    check(ctx, shifted, 0.1)


@pytest.mark.parametrize("scale", [1e-30, 1e-22, 1e19, 1e25])
def test_squares_outside_the_range_of_fp32(ctx, scale):
    made = make([5000, 1, 1, 333], 8, 1, scale=1.0)
    made = [m for m in made if m[0][0].dtype.itemsize == 4]
    for b, _, _ in made:
        b[0].mul_(scale)
    check(ctx, made, scale * 3.0)


def test_zeros_empty_tensors_and_nothing(ctx):
    import torch
    from paper_2609_05255_b200 import api
    ws, clip = torch.empty((api.gs_grad_workspace_bytes(),), device="cuda", dtype=torch.uint8), torch.empty((2,), device="cuda")
    z = torch.zeros((100,), device="cuda")
    api.gs_clip_grads(ctx, [api.GradTensor(z, out=z), api.GradTensor(z[:0], out=z[:0])], 1.0, clip, ws)
    assert clip.tolist() == [0.0, 1.0] and torch.all(z == 0)
    api.gs_grad_norm(ctx, [], 1.0, clip.fill_(5), ws)
    assert clip.tolist() == [0.0, 1.0]


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_a_gradient_that_is_not_finite(ctx, bad):
    """scale 0: the outputs are zeros, the clipped update writes nothing."""
    import torch
    from paper_2609_05255_b200 import api
    ws, clip = torch.empty((api.gs_grad_workspace_bytes(),), device="cuda", dtype=torch.uint8), torch.empty((2,), device="cuda")
    for dtype, at in ((torch.float32, 3), (torch.float16, 4097), (torch.bfloat16, 9999)):
        g = torch.randn((10_000,), device="cuda").to(dtype)
        g[at] = bad
        out = torch.ones_like(g)
        api.gs_clip_grads(ctx, [api.GradTensor(g, out=out)], 1.0, clip, ws)
        assert not math.isfinite(float(clip[0])) and float(clip[1]) == 0.0 and torch.all(out == 0)
    p, m, v = (torch.randn((10_000,), device="cuda").abs() for _ in range(3))
    h = torch.ones((10_000,), device="cuda").half()
    old = [t.clone() for t in (p, m, v, h)]
    g = torch.full((10_000,), bad, device="cuda")
    api.gs_grad_norm(ctx, [api.GradTensor(g)], 1.0, clip, ws)
    api.gs_adam_step_clipped(ctx, [api.AdamTensor(p, g, m, v, [1e-3], half_copy=h)], 3, clip)
    assert all(torch.equal(a, b) for a, b in zip(old, (p, m, v, h)))


def test_in_place(ctx):
    import torch
    from paper_2609_05255_b200 import api
    ws, clip = torch.empty((api.gs_grad_workspace_bytes(),), device="cuda", dtype=torch.uint8), torch.empty((2,), device="cuda")
    a, b = torch.randn((30_001,), device="cuda"), torch.randn((30_001,), device="cuda")
    out = torch.empty_like(a)
    api.gs_clip_grads(ctx, [api.GradTensor(a, more_grads=[b], out=out)], 2.0, clip, ws)
    want = out.clone()
    api.gs_clip_grads(ctx, [api.GradTensor(a, more_grads=[b], out=a)], 2.0, clip, ws)
    assert torch.equal(a, want)
    c = a.clone()
    api.gs_clip_grads(ctx, [api.GradTensor(a, out=a)], 1e6, clip, ws)                 # nothing to scale
    assert torch.equal(a, c) and float(clip[1]) == 1.0


@pytest.mark.parametrize("max_norm", [0.05, 1e9])
@pytest.mark.parametrize("views", [1, 3, 8])
def test_clipped_adam_is_adam_of_the_clipped_gradient(ctx, views, max_norm):
    import torch
    from paper_2609_05255_b200 import api
    ws, clip = torch.empty((api.gs_grad_workspace_bytes(),), device="cuda", dtype=torch.uint8), torch.empty((2,), device="cuda")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(9)
    randn = lambda *s: torch.randn(s, device="cuda", generator=gen)
    shapes, sets = [(5003, 3), (5003, 8), (5003, 45), (816, 1), (1, 1)], []
    for s in shapes:
        sets.append(dict(p=randn(*s), g=[randn(*s) * 1e-2 for _ in range(views)], m=randn(*s) * 1e-3, v=randn(*s).square() * 1e-5))
    copies = [dict(p=t["p"].clone(), m=t["m"].clone(), v=t["v"].clone()) for t in sets]
    halves = [torch.zeros(s, device="cuda", dtype=torch.float16) for s in shapes], [torch.zeros(s, device="cuda", dtype=torch.float16) for s in shapes]
    api.gs_grad_norm(ctx, [api.GradTensor(t["g"][0], more_grads=t["g"][1:]) for t in sets], max_norm, clip, ws)
    assert (float(clip[1]) < 1) == (max_norm < 1)
    api.gs_adam_step_clipped(ctx, [api.AdamTensor(t["p"], t["g"][0], t["m"], t["v"], [1e-3] * s[1], half_copy=h, more_grads=t["g"][1:])
                                   for t, s, h in zip(sets, shapes, halves[0])], 7, clip)
    plain = []
    for t, c, s, h in zip(sets, copies, shapes, halves[1]):
        g = t["g"][0].clone()
        for more in t["g"][1:]:
            g += more
        plain.append(api.AdamTensor(c["p"], (g * clip[1]).contiguous(), c["m"], c["v"], [1e-3] * s[1], half_copy=h))
    api.gs_adam_step(ctx, plain, 7)
    for t, c, a, b in zip(sets, copies, *halves):
        assert all(torch.equal(t[k], c[k]) for k in ("p", "m", "v")) and torch.equal(a, b)


def test_graph_and_runs_agree(ctx):
    import torch
    from paper_2609_05255_b200 import api
    made = make([50_001, 70_000, 3], 10)
    ws, clip = torch.empty((api.gs_grad_workspace_bytes(),), device="cuda", dtype=torch.uint8), torch.empty((2,), device="cuda")
    grads = api.GradList([api.GradTensor(b[0], out=o) for b, o, _ in made])
    api.gs_clip_grads(ctx, grads, 1.0, clip, ws)
    want = [clip.clone()] + [o.clone() for _, o, _ in made]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.gs_clip_grads(ctx, grads, 1.0, clip, ws)
    for t in [clip] + [o for _, o, _ in made]:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, [clip] + [o for _, o, _ in made]))


def test_refusals(ctx):
    import torch
    from paper_2609_05255_b200 import api
    ws, clip = torch.empty((api.gs_grad_workspace_bytes(),), device="cuda", dtype=torch.uint8), torch.empty((2,), device="cuda")
    z = lambda n=8: torch.zeros((n,), device="cuda")

    def refused(status, f):
        with pytest.raises(api.GsError) as e:
            f()
        assert e.value.status == status and str(e.value)
    bad = api.GS_ERR_INVALID_ARG
    ok = [api.GradTensor(z(), out=z())]
    for norm in (0.0, -1.0, float("nan")):
        refused(bad, lambda: api.gs_grad_norm(ctx, ok, norm, clip, ws))
    refused(bad, lambda: api.gs_clip_grads(ctx, [api.GradTensor(z())], 1.0, clip, ws))                 # no out
    refused(bad, lambda: api.gs_grad_norm(ctx, [api.GradTensor(z(), more_grads=[z()] * 8)], 1.0, clip, ws))
    refused(bad, lambda: api.gs_grad_norm(ctx, [api.GradTensor(z(), more_grads=[z(9)])], 1.0, clip, ws))
    refused(bad, lambda: api.gs_grad_norm(ctx, [api.GradTensor(z(), more_grads=[z().half()])], 1.0, clip, ws))
    refused(bad, lambda: api.gs_grad_norm(ctx, [api.GradTensor(z().double())], 1.0, clip, ws))
    refused(bad, lambda: api.gs_grad_norm(ctx, [api.GradTensor(z().cpu())], 1.0, clip, ws))
    refused(bad, lambda: api.gs_grad_norm(ctx, [api.GradTensor(z(16)[::2])], 1.0, clip, ws))
    refused(bad, lambda: api.gs_grad_norm(ctx, [api.GradTensor(z()) for _ in range(513)], 1.0, clip, ws))
    refused(bad, lambda: api.gs_grad_norm(ctx, [api.GradTensor(z(), more_grads=[z()] * 3) for _ in range(400)], 1.0, clip, ws))
    refused(bad, lambda: api.gs_grad_norm(ctx, ok, 1.0, z(3), ws))
    refused(bad, lambda: api.gs_grad_norm(ctx, ok, 1.0, z(3)[1:], ws))                                 # clip not on 8 bytes
    refused(bad, lambda: api.gs_grad_norm(ctx, ok, 1.0, clip, None))
    refused(api.GS_ERR_CAPACITY, lambda: api.gs_grad_norm(ctx, ok, 1.0, clip, ws[:-8]))
    t = api.AdamTensor(z(), z(), z(), z(), [1e-3])
    refused(bad, lambda: api.gs_adam_step_clipped(ctx, [t], 0, clip))
    refused(bad, lambda: api.gs_adam_step_clipped(ctx, [t], 1, z(3)))
    refused(bad, lambda: api.gs_adam_step_clipped(ctx, [t] * 9, 1, clip))
