"""Operator cases: a network's layers beside the scene, and the clipping of all gradients before the update.

A case is a dict of plain values; `prepare` makes what a program holds before the call, `run` makes one pass.  Kinds:

  dense_fwd  y = act(x W^T + b) + residual, with the pre-activation kept where a backward pass follows
  dense_bwd  its gradients with respect to x, W and b from the kept pre-activation
  ln_fwd     layer norm over the rows, with the statistics a backward pass needs
  ln_bwd     its gradients with respect to x, gamma and beta
  clip       the global norm over many gradient tensors, and all of them scaled to a largest norm
  adam       the norm over a scene's gradients (several views' buffers summed) and the Adam update with the clipped gradient

Activations and weights are fp16 or bf16 (layer norm: fp32 too), rows padded to eight elements; biases, norms' parameters,
statistics, and gradients of parameters are fp32.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
LN_EPS = 1e-5
BETA1, EPS = 0.9, 1e-15
# a neural scene's parameter tensors: columns, learning rate, beta2 (0 columns: the decoder's 816 weights)
SCENE = [("means", 3, 1.6e-4, 0.999), ("log_scales", 3, 5e-3, 0.999), ("quats", 4, 1e-3, 0.999), ("opacity_logits", 1, 5e-2, 0.999),
         ("base_color", 3, 2.5e-4, 0.999), ("features", 8, 8e-3, 0.999), ("mlp_weights", 0, 3e-3, 0.99)]
STEP = 1000


def listed():
    return [
        # one Gaussian picked and edited in a viewer: launch latency
        dict(name="dense_fwd_1x64_64", kind="dense_fwd", rows=1, cin=64, cout=64, dtype="f16", act="relu", residual=False, keep=False),
        # first layer over frequency-encoded positions (3 + 3 * 2 * 10 columns), an early scene, training
        dict(name="dense_fwd_100k_63_256", kind="dense_fwd", rows=100_003, cin=63, cout=256, dtype="f16", act="relu", residual=False, keep=True),
        # a residual block of a trunk over the 1M-Gaussian scene, training
        dict(name="dense_fwd_1M_256_256_res", kind="dense_fwd", rows=1_000_000, cin=256, cout=256, dtype="bf16", act="silu", residual=True, keep=True),
        # a wide layer over the control points of a deformation, evaluation: bound by the products
        dict(name="dense_fwd_20k_1024_1024", kind="dense_fwd", rows=20_011, cin=1024, cout=1024, dtype="bf16", act="gelu", residual=False, keep=False),
        # the head that gives the decoder its eight features
        dict(name="dense_bwd_300k_256_8", kind="dense_bwd", rows=300_007, cin=256, cout=8, dtype="f16", act="none"),
        # the residual block's backward pass
        dict(name="dense_bwd_1M_256_256", kind="dense_bwd", rows=1_000_000, cin=256, cout=256, dtype="bf16", act="silu"),
        # rows of spherical-harmonics coefficients of a small scene, normalised in single precision
        dict(name="ln_fwd_1000x45_f32", kind="ln_fwd", rows=1000, cols=45, dtype="f32"),
        # the norm in front of the residual block, and its backward pass
        dict(name="ln_fwd_1M_256", kind="ln_fwd", rows=1_000_000, cols=256, dtype="bf16"),
        dict(name="ln_bwd_1M_256", kind="ln_bwd", rows=1_000_000, cols=256, dtype="f16"),
        # a trunk's many parameter gradients in three types, ragged sizes, clipped into the optimiser's buffers
        dict(name="clip_61_tensors_3M", kind="clip", tensors=61, total=3_000_000, buffers=1),
        # an early scene of one view: norm and update
        dict(name="adam_20k_1view", kind="adam", n=20_011, views=1),
        # an iteration over eight views of the 1M-Gaussian scene, a gradient buffer for each
        dict(name="adam_1M_8views", kind="adam", n=1_000_000, views=8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["dense_fwd", "dense_bwd", "ln_fwd", "ln_bwd", "clip", "adam"], [25, 25, 15, 15, 10, 10])[0]
    if kind.startswith("dense"):
        cin, cout = _log_int(rng, 3, 1024), _log_int(rng, 3, 1024)
        most = min(1_000_000, 1_000_000 * 512 // (cin + cout), 1_000_000 * 65536 // (cin * cout))
        case = dict(kind=kind, rows=_log_int(rng, 1, most), cin=cin, cout=cout, dtype=rng.choice(["f16", "bf16"]),
                    act=rng.choice(["none", "relu", "silu", "gelu"]))
        if kind == "dense_fwd":
            case.update(residual=rng.random() < 0.5, keep=rng.random() < 0.5)
        return case
    if kind.startswith("ln"):
        cols = _log_int(rng, 3, 4096)
        return dict(kind=kind, rows=_log_int(rng, 1, min(2_000_000, 1_000_000 * 128 // cols)), cols=cols, dtype=rng.choice(["f32", "f16", "bf16"]))
    if kind == "clip":
        tensors = rng.randint(1, 300)
        return dict(kind=kind, tensors=tensors, total=max(tensors * 4, _log_int(rng, 1000, 20_000_000)), buffers=rng.randint(1, 4))
    return dict(kind=kind, n=_log_int(rng, 100, 1_000_000), views=rng.randint(1, 8))


def _padded(rows, cols, dtype):
    """[rows, cols] whose rows start every multiple of eight elements."""
    return torch.zeros((rows, (cols + 7) // 8 * 8), device="cuda", dtype=dtype)[:, :cols]


def _filled(values, dtype):
    t = _padded(*values.shape, dtype)
    t.copy_(values)
    return t


def _sizes(case):
    """Ragged sizes of the clipped tensors: a few carry most of the elements, many are vectors."""
    count, total = case["tensors"], case["total"]
    shares = [1.0 / (1 + (7 * i) % count) ** 1.5 for i in range(count)]
    scale = total / sum(shares)
    return [max(1, int(scale * s)) + i % 3 for i, s in enumerate(shares)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    randn = lambda *shape: torch.randn(shape, device="cuda", generator=gen)
    kind, s = case["kind"], dict(case=case)
    if kind.startswith("dense"):
        m, k, n, dt = case["rows"], case["cin"], case["cout"], TYPES[case["dtype"]]
        s["x"] = _filled(randn(m, k), dt)
        s["w"] = _filled(randn(n, k) / math.sqrt(k), dt)
        s["b"] = randn(n) * 0.1
        if kind == "dense_fwd":
            s["r"] = _filled(randn(m, n), dt) if case["residual"] else None
            s["y"] = _padded(m, n, dt)
            s["z"] = _padded(m, n, dt) if case["keep"] else None
        else:
            s["z"] = _filled(randn(m, n) * 1.2, dt) if case["act"] != "none" else None
            seen = torch.rand((m, 1), device="cuda", generator=gen) < 0.7     # Gaussians outside the view have no gradient
            seen[0] = True
            s["dy"] = _filled(randn(m, n) * 0.01 * seen, dt)
            s["dx"] = _padded(m, k, dt)
            s["dw"] = torch.zeros((n, k), device="cuda")
            s["db"] = torch.zeros((n,), device="cuda")
    elif kind.startswith("ln"):
        m, c, dt = case["rows"], case["cols"], TYPES[case["dtype"]]
        s["x"] = _filled(randn(m, c) * (0.5 + torch.rand((m, 1), device="cuda", generator=gen)) + 0.5 * randn(m, 1), dt)
        s["gamma"], s["beta"] = 1 + 0.2 * randn(c), 0.2 * randn(c)
        if kind == "ln_fwd":
            s["y"] = _padded(m, c, dt)
            s["mean"], s["rstd"] = torch.zeros((m,), device="cuda"), torch.zeros((m,), device="cuda")
        else:
            x = s["x"].double()
            mean = x.mean(1)
            s["mean"], s["rstd"] = mean.float(), torch.rsqrt((x - mean[:, None]).square().mean(1) + LN_EPS).float()
            s["dy"] = _filled(randn(m, c) * 0.01, dt)
            s["dx"] = _padded(m, c, dt)
            s["dgamma"], s["dbeta"] = torch.zeros((c,), device="cuda"), torch.zeros((c,), device="cuda")
    elif kind == "clip":
        # gradients one behind another in a flat buffer for each type, so most start at odd places
        sizes, types = _sizes(case), ["f32", "f16", "bf16"]
        s["flat"] = {t: [randn(sum(sizes[i::3])).mul_(0.01).to(TYPES[t]) for _ in range(case["buffers"])] for i, t in enumerate(types)}
        s["out"] = {t: torch.zeros_like(s["flat"][t][0]) for t in types}
        s["views"] = []
        for i, t in enumerate(types):
            at = 0
            for size in sizes[i::3]:
                s["views"].append(([f[at:at + size] for f in s["flat"][t]], s["out"][t][at:at + size]))
                at += size
        s["max_norm"] = 1.0
        s["clip"] = torch.zeros((2,), device="cuda")
    else:
        s["tensors"] = []
        for name, cols, lr, beta2 in SCENE:
            rows = case["n"] if cols else 816
            shape = (rows, cols or 1)
            seen = torch.rand((rows, 1), device="cuda", generator=gen) < (0.7 if cols else 2.0)
            grads = [randn(*shape) * 1e-3 * seen for _ in range(case["views"])]
            half = torch.zeros(shape, device="cuda", dtype=torch.float16) if name in ("features", "mlp_weights") else None
            s["tensors"].append(dict(p=randn(*shape), g=grads, m=randn(*shape) * 1e-4, v=torch.rand(shape, device="cuda", generator=gen) * 1e-6 + 1e-8,
                                     half=half, lr=lr, beta2=beta2))
        s["max_norm"] = 0.1
        s["clip"] = torch.zeros((2,), device="cuda")
    return s


def _act(name, z):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "gelu":
        return z / (1 + torch.exp(-1.5957691216057308 * (z + 0.044715 * z * z * z)))
    return z


def _act_grad(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p + z * p * (1 - p)
    if name == "gelu":
        p = 1 / (1 + torch.exp(-1.5957691216057308 * (z + 0.044715 * z * z * z)))
        return p + z * p * (1 - p) * 1.5957691216057308 * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _f32(beta):
    return float(torch.tensor(beta, dtype=torch.float32))


def _plain(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind == "dense_fwd":
        dt = s["x"].dtype
        z = s["x"].float() @ s["w"].float().T + s["b"]
        y = _act(case["act"], z)
        if s["r"] is not None:
            y = y + s["r"].float()
        return [y.to(dt), z.to(dt)] if case["keep"] else [y.to(dt)]
    if kind == "dense_bwd":
        dz = s["dy"].float()
        if s["z"] is not None:
            dz = dz * _act_grad(case["act"], s["z"].float())
        return [(dz @ s["w"].float()).to(s["x"].dtype), dz.T @ s["x"].float(), dz.sum(0)]
    if kind == "ln_fwd":
        x = s["x"].float()
        mean = x.mean(1, keepdim=True)
        rstd = 1 / torch.sqrt((x - mean).square().mean(1, keepdim=True) + LN_EPS)
        return [((x - mean) * rstd * s["gamma"] + s["beta"]).to(s["x"].dtype), mean[:, 0], rstd[:, 0]]
    if kind == "ln_bwd":
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        h = (s["x"].float() - s["mean"][:, None]) * rstd
        g = dy * s["gamma"]
        dx = rstd * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
        return [dx.to(s["x"].dtype), (dy * h).sum(0), dy.sum(0)]
    if kind == "clip":
        sums = {t: sum((b.float() for b in f[1:]), f[0].float()) for t, f in s["flat"].items()}
        norm = torch.sqrt(sum(g.square().sum(dtype=torch.float64) for g in sums.values())).float()
        scale = torch.clamp(s["max_norm"] / norm, max=1.0)
        return [torch.stack([norm, scale])] + [(g * scale).to(TYPES[t]) for t, g in sums.items()]
    grads = [sum(t["g"][1:], t["g"][0]) for t in s["tensors"]]
    norm = torch.sqrt(sum(g.square().sum(dtype=torch.float64) for g in grads)).float()
    scale = torch.clamp(s["max_norm"] / norm, max=1.0)
    out = [torch.stack([norm, scale])]
    for t, g in zip(s["tensors"], grads):
        b1, b2, g = _f32(BETA1), _f32(t["beta2"]), g * scale
        t["m"].mul_(b1).add_(g * (1 - b1))
        t["v"].mul_(b2).add_(g * g * (1 - b2))
        t["p"].sub_(_f32(t["lr"]) / (1 - b1 ** STEP) * t["m"] / (torch.sqrt(t["v"] / (1 - b2 ** STEP)) + EPS))
        out += [t["p"], t["m"], t["v"]]
        if t["half"] is not None:
            t["half"].copy_(t["p"])
            out.append(t["half"])
    return out


_kept = {}


def _own(s):
    from paper_2609_05255_b200 import api
    if "ctx" not in _kept:
        _kept["ctx"] = api.Context(0)
    ctx, case, kind = _kept["ctx"], s["case"], s["case"]["kind"]
    if kind == "dense_fwd":
        if "layer" not in s:
            s["layer"] = api.DenseLayer(s["w"], s["b"], case["act"])
        api.gs_dense_forward(ctx, s["layer"], s["x"], s["y"], preact=s["z"], residual=s["r"])
        return [s["y"], s["z"]] if case["keep"] else [s["y"]]
    if kind == "dense_bwd":
        if "layer" not in s:
            s["layer"] = api.DenseLayer(s["w"], s["b"], case["act"])
            s["ws"] = torch.empty((api.gs_dense_workspace_bytes(case["rows"], case["cin"], case["cout"]),), device="cuda", dtype=torch.uint8)
        api.gs_dense_backward(ctx, s["layer"], s["x"], s["dy"], preact=s["z"], dL_dx=s["dx"], dL_dweight=s["dw"], dL_dbias=s["db"], workspace=s["ws"])
        return [s["dx"], s["dw"], s["db"]]
    if kind == "ln_fwd":
        api.gs_layer_norm_forward(ctx, s["x"], s["gamma"], s["beta"], s["y"], mean=s["mean"], rstd=s["rstd"], eps=LN_EPS)
        return [s["y"], s["mean"], s["rstd"]]
    if kind == "ln_bwd":
        if "ws" not in s:
            s["ws"] = torch.empty((api.gs_layer_norm_workspace_bytes(case["rows"], case["cols"]),), device="cuda", dtype=torch.uint8)
        api.gs_layer_norm_backward(ctx, s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"], s["dx"], s["dgamma"], s["dbeta"], s["ws"])
        return [s["dx"], s["dgamma"], s["dbeta"]]
    if "ws" not in s:
        s["ws"] = torch.empty((api.gs_grad_workspace_bytes(),), device="cuda", dtype=torch.uint8)
        if kind == "clip":
            s["list"] = api.GradList([api.GradTensor(g[0], more_grads=g[1:], out=out) for g, out in s["views"]])
        else:
            s["list"] = api.GradList([api.GradTensor(t["g"][0], more_grads=t["g"][1:]) for t in s["tensors"]])
            s["adam"] = [api.AdamTensor(t["p"], t["g"][0], t["m"], t["v"], [t["lr"]] * t["p"].shape[1], BETA1, t["beta2"], EPS, half_copy=t["half"],
                                        more_grads=t["g"][1:]) for t in s["tensors"]]
    if kind == "clip":
        api.gs_clip_grads(ctx, s["list"], s["max_norm"], s["clip"], s["ws"])
        return [s["clip"]] + list(s["out"].values())
    api.gs_grad_norm(ctx, s["list"], s["max_norm"], s["clip"], s["ws"])
    api.gs_adam_step_clipped(ctx, s["adam"], STEP, s["clip"])
    out = [s["clip"]]
    for t in s["tensors"]:
        out += [t["p"], t["m"], t["v"]] + ([t["half"]] if t["half"] is not None else [])
    return out


def run(s):
    if own:
        return _own(s)
    return _plain(s)


def work(case):
    kind = case["kind"]
    if kind.startswith("dense"):
        m, k, n = case["rows"], case["cin"], case["cout"]
        if kind == "dense_fwd":
            return dict(bytes=2 * (m * k + m * n * (1 + case["residual"] + case["keep"]) + n * k) + 4 * n, flops=2 * m * k * n)
        return dict(bytes=2 * (2 * m * k + m * n * (1 + (case["act"] != "none")) + n * k) + 4 * (n * k + n), flops=4 * m * k * n)
    if kind.startswith("ln"):
        m, c = case["rows"], case["cols"]
        fwd = kind == "ln_fwd"
        return dict(bytes=(2 if fwd else 3) * m * c * SIZE[case["dtype"]] + 8 * m + (8 if fwd else 12) * c, flops=(8 if fwd else 14) * m * c)
    if kind == "clip":
        sizes = _sizes(case)
        by = sum(sum(sizes[i::3]) * SIZE[t] for i, t in enumerate(["f32", "f16", "bf16"]))
        return dict(bytes=by * (case["buffers"] + 1) + 8, flops=sum(sizes) * (case["buffers"] + 3))
    count = sum((case["n"] if cols else 816) * (cols or 1) for _, cols, _, _ in SCENE)
    return dict(bytes=count * (4 * case["views"] + 24) + 2 * (8 * case["n"] + 816), flops=count * (case["views"] + 14))


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    d = lambda t: t.double()
    if kind.startswith("dense"):
        def pieces(name, z):
            """act(z) and act'(z)."""
            if name == "relu":
                return z.clamp(min=0), (z > 0).double()
            if name == "silu":
                p = torch.sigmoid(z)
                return z * p, p * (1 + z * (1 - p))
            if name == "gelu":
                c = math.sqrt(2 / math.pi)
                t = torch.tanh(c * (z + 0.044715 * z ** 3))
                return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 0.134145 * z * z)
            return z, torch.ones_like(z)
        if kind == "dense_fwd":
            z = torch.addmm(d(s["b"]), d(s["x"]), d(s["w"]).T)
            y = pieces(case["act"], z)[0]
            if case["residual"]:
                y = y + d(s["r"])
            return [y, z] if case["keep"] else [y]
        dz = d(s["dy"])
        if s["z"] is not None:
            dz = dz * pieces(case["act"], d(s["z"]))[1]
        return [dz @ d(s["w"]), dz.T @ d(s["x"]), dz.sum(0)]
    if kind == "ln_fwd":
        x = d(s["x"])
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = (var + LN_EPS).rsqrt()
        return [(x - mean[:, None]) * rstd[:, None] * d(s["gamma"]) + d(s["beta"]), mean, rstd]
    if kind == "ln_bwd":
        dy, r = d(s["dy"]), d(s["rstd"])[:, None]
        h = (d(s["x"]) - d(s["mean"])[:, None]) * r
        g = dy * d(s["gamma"])
        c = case["cols"]
        return [r * (g - g.sum(1, keepdim=True) / c - h * ((g * h).sum(1, keepdim=True) / c)), (dy * h).sum(0), dy.sum(0)]
    if kind == "clip":
        sums = [torch.stack([d(b) for b in f]).sum(0) for f in s["flat"].values()]
        norm = torch.linalg.vector_norm(torch.cat(sums))
        scale = min(1.0, s["max_norm"] / float(norm))
        return [torch.tensor([float(norm), scale], dtype=torch.float64)] + [g * scale for g in sums]
    sums = [torch.stack([d(b) for b in t["g"]]).sum(0) for t in s["tensors"]]
    norm = math.sqrt(sum(float((g * g).sum()) for g in sums))
    scale = min(1.0, s["max_norm"] / norm)
    out = [torch.tensor([norm, scale], dtype=torch.float64)]
    for t, g in zip(s["tensors"], sums):
        b1, b2 = _f32(BETA1), _f32(t["beta2"])
        m = d(t["m"]) * b1 + (1 - b1) * scale * g
        v = d(t["v"]) * b2 + (1 - b2) * (scale * g) ** 2
        p = d(t["p"]) - _f32(t["lr"]) * (m / (1 - b1 ** STEP)) / ((v / (1 - b2 ** STEP)).sqrt() + EPS)
        out += [p, m, v] + ([p] if t["half"] is not None else [])
    return out
