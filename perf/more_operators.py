"""Performance cases of more operators of a network that is trained: layer norm over
channels with its gradients, the orthogonalised update by Newton-Schulz products, and the
Muon step that makes and applies such updates.

A case is one pass through one operator:

  layer        y = act(layer_norm(x) * gamma + beta) over the channels of each pixel or
               token, and the statistics that training keeps.
  layer_grad   its gradients for x, gamma and beta, from x, dy and the statistics.
  orthogonal   five Newton-Schulz steps of each matrix of a batch, in the matrices' type.
  muon         one Muon step over a list of matrices, in place: momentum, the
               orthogonalised update, weight decay, the working copies.

Inputs are drawn on the GPU from the seed alone.
"""
from __future__ import annotations

import math

import torch

own = False  # False: the plain forms below; True: the library's kernels

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
NORM_EPS = 1e-5
STEPS, COEFFICIENTS, EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7  # of the Newton-Schulz products
LR, MOMENTUM, DECAY = 0.02, 0.95, 0.01


def _layer(kind, n, h, w, c, layout="NHWC", dtype="bf16", act="none"):
    return dict(kind=kind, n=n, h=h, w=w, c=c, layout=layout, dtype=dtype, act=act)


def _orthogonal(batch, rows, cols, dtype="f32"):
    return dict(kind="orthogonal", batch=batch, rows=rows, cols=cols, dtype=dtype)


def _muon(shapes, param="f32", grad="f32", copy=False):
    return dict(kind="muon", shapes=shapes, param=param, grad=grad, copy=copy)


# A conditional generator's transposed convolutions as matrices: input channels by output
# channels and taps.
GENERATOR = "100x16384 1024x8192 512x4096 256x2048 128x48"


def listed():
    return [
        # One image through the generator: the norm behind its second layer (latency).
        dict(_layer("layer", 1, 8, 8, 512, act="relu"), name="layer_gen_b1"),
        # The generator's training batch in the weight gradients' layout, behind its third layer.
        dict(_layer("layer", 64, 16, 16, 256, "NCHW", act="relu"), name="layer_gen_b64_nchw"),
        # The feature map that the atrous pyramid reads: large, wide rows.
        dict(_layer("layer", 8, 64, 64, 2048), name="layer_features_b8"),
        # Training the generator: the norm behind its fourth layer, where maps are largest.
        dict(_layer("layer_grad", 64, 32, 32, 128, act="relu"), name="layer_grad_gen_b64"),
        # A decoder block on an odd crop, full precision, in the weight gradients' layout.
        dict(_layer("layer_grad", 5, 33, 41, 200, "NCHW", "f32", "silu"),
             name="layer_grad_ragged_f32"),
        # Embedded text tokens: long lists of rows.
        dict(_layer("layer_grad", 32768, 1, 1, 1024, "rows"), name="layer_grad_text"),
        # The generator's last layer alone: the smallest matrix (latency).
        dict(_orthogonal(1, 128, 48), name="orthogonal_last"),
        # A few odd matrices of one shape, taller than wide.
        dict(_orthogonal(6, 1000, 333), name="orthogonal_ragged"),
        # One large matrix in 16 bits.
        dict(_orthogonal(1, 4096, 8192, "bf16"), name="orthogonal_large"),
        # The generator's matrices: fp32 weights, bf16 gradients and working copies.
        dict(_muon(GENERATOR, grad="bf16", copy=True), name="muon_generator"),
        # Many small odd matrices in 16 bits (launches).
        dict(_muon(" ".join("%dx%d" % (33 + 13 * i, 700 - 13 * i) for i in range(48)), "bf16",
                   "bf16"), name="muon_many"),
        # The largest step: square and wide matrices of 16-bit weights.
        dict(_muon("4096x4096 4096x4096 2048x8192 8192x2048 4096x4096 1024x4096", "bf16", "bf16"),
             name="muon_large"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case that costs no more than the largest listed one of its kind."""
    while True:
        kind = rng.choice(("layer", "layer", "layer_grad", "layer_grad", "orthogonal",
                           "orthogonal", "muon", "muon"))
        dtype = rng.choice(("bf16", "f32"))
        if kind.startswith("layer"):
            c = _log_int(rng, 16, 8192)
            if rng.random() < 2 / 3:
                c = c // 8 * 8
            layout = rng.choice(("rows", "NHWC", "NCHW", "NCHW"))
            h, w = (1, 1) if layout == "rows" else (_log_int(rng, 1, 128), _log_int(rng, 1, 128))
            n = _log_int(rng, 1, 65536 if layout == "rows" else 64)
            case = _layer(kind, n, h, w, c, layout, dtype,
                          rng.choice(("none", "none", "relu", "tanh", "silu")))
            if n * h * w * c <= (1 << 26) * 2 // SIZE[dtype]:
                return case
        elif kind == "orthogonal":
            case = _orthogonal(_log_int(rng, 1, 32), _log_int(rng, 16, 8192),
                               _log_int(rng, 16, 8192), dtype)
            if work(case)["flops"] <= 2e12 * 2 // SIZE[dtype]:
                return case
        else:
            lo, hi = _log_int(rng, 16, 300), _log_int(rng, 300, 4096)
            shapes = " ".join("%dx%d" % (_log_int(rng, lo, hi), _log_int(rng, lo, 2 * hi))
                              for _ in range(_log_int(rng, 1, 40)))
            case = _muon(shapes, dtype, rng.choice(("f32", "bf16")), rng.random() < 0.5)
            case["copy"] = case["copy"] and dtype == "f32"
            if work(case)["flops"] <= 4e12 * 2 // SIZE[dtype]:
                return case


def _shapes(case):
    if case["kind"] == "orthogonal":
        return [(case["rows"], case["cols"])] * case["batch"]
    return [tuple(int(n) for n in s.split("x")) for s in case["shapes"].split()]


def _sizes(case):
    return [r * c for r, c in _shapes(case)]


def work(case):
    if case["kind"].startswith("layer"):
        pixels = case["n"] * case["h"] * case["w"]
        numel, stats = pixels * case["c"], 8 * pixels
        if case["kind"] == "layer":  # x, gamma, beta in; y, statistics out
            return {"bytes": 2 * numel * SIZE[case["dtype"]] + 8 * case["c"] + stats,
                    "flops": 10 * numel}
        # x, dy, statistics, gamma, beta in; dx, dgamma, dbeta out
        return {"bytes": 3 * numel * SIZE[case["dtype"]] + 16 * case["c"] + stats,
                "flops": 20 * numel}
    # For m rows and n >= m columns a step is A = X X^T and A A, both symmetric (half of
    # their products), and (b A + c A A) X.
    pairs = [(min(s), max(s)) for s in _shapes(case)]
    flops = STEPS * sum(3 * m * m * n + m ** 3 for m, n in pairs)
    if case["kind"] == "orthogonal":
        return {"bytes": 2 * sum(_sizes(case)) * SIZE[case["dtype"]], "flops": flops}
    each = 2 * SIZE[case["param"]] + SIZE[case["grad"]] + 8 + (2 if case["copy"] else 0)
    return {"bytes": sum(_sizes(case)) * each, "flops": flops}


# ---- inputs -----------------------------------------------------------------

def _device():
    return torch.device("cuda", torch.cuda.current_device())


def _shape(case):
    n, h, w, c = (case[k] for k in ("n", "h", "w", "c"))
    return {"rows": (n, c), "NHWC": (n, h, w, c), "NCHW": (n, c, h, w)}[case["layout"]]


def _axis(case):
    return 1 if case["layout"] == "NCHW" else -1


def _layer_inputs(case, g):
    normal = lambda *s: torch.randn(s, generator=g, device=g.device)  # noqa: E731
    c, dtype = case["c"], DTYPES[case["dtype"]]
    by_channel = (c, 1, 1) if case["layout"] == "NCHW" else (c,)
    # what a convolution with a bias leaves: channels of their own mean and scale
    scale, shift = (0.5 + normal(c).abs()).reshape(by_channel), normal(c).reshape(by_channel)
    s = {"x": (normal(*_shape(case)) * scale + shift).to(dtype),
         "gamma": 1 + 0.1 * normal(c), "beta": 0.1 * normal(c)}
    if case["kind"] == "layer_grad":
        s["dy"] = normal(*_shape(case)).to(dtype)
        mean = s["x"].mean(_axis(case), dtype=torch.float64, keepdim=True)
        var = (s["x"] - mean).square_().mean(_axis(case))
        s["stats"] = torch.stack((mean.flatten(), (var.flatten() + NORM_EPS).rsqrt()), -1).float()
    return s


def _update(rows, cols, g):
    """What a batch leaves for a matrix: some directions that many samples share, each weaker
    than the one before, and every sample's own noise."""
    rank = max(1, min(rows, cols) // 8)
    normal = lambda *s: torch.randn(s, generator=g, device=g.device)  # noqa: E731
    falling = torch.arange(1, rank + 1, device=g.device).float().rsqrt() / math.sqrt(rank)
    return (normal(rows, rank) * falling) @ normal(rank, cols) + 0.5 * normal(rows, cols)


def _muon_inputs(case, g):
    shapes, sizes = _shapes(case), _sizes(case)
    padded = [-(-n // 8) * 8 for n in sizes]  # matrices lie in buffers, 16-byte aligned
    at = [sum(padded[:i]) for i in range(len(sizes))]
    s = {"shapes": shapes, "at": at, "sizes": sizes}
    p, m = (torch.zeros(sum(padded), device=g.device) for _ in range(2))
    s["grads"] = []
    for a, n, (r, c) in zip(at, sizes, shapes):
        p[a:a + n] = torch.randn(n, generator=g, device=g.device) * 0.02
        shared = _update(r, c, g)  # a gradient resembles those before it
        m[a:a + n] = 3e-3 * shared.flatten()
        s["grads"].append((1e-2 * (0.3 * shared + _update(r, c, g))).to(DTYPES[case["grad"]]))
    s["p"], s["m"] = p.to(DTYPES[case["param"]]), m
    if case["copy"]:
        s["copy"] = p.to(torch.bfloat16)
    # a matrix with more rows than columns gets the larger step
    s["scales"] = [math.sqrt(max(1.0, r / c)) for r, c in shapes]
    return s


def _inputs(case, seed):
    g = torch.Generator(_device()).manual_seed(seed)
    if case["kind"].startswith("layer"):
        return _layer_inputs(case, g)
    if case["kind"] == "muon":
        return _muon_inputs(case, g)
    x = torch.stack([1e-2 * _update(r, c, g) for r, c in _shapes(case)])
    return {"x": x.to(DTYPES[case["dtype"]])}


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        _handle(s, case)
    return s


def _views(s, name):
    """The matrices of a buffer."""
    return [s[name][a:a + n].view(shape) for a, n, shape in zip(s["at"], s["sizes"], s["shapes"])]


def _handle(s, case):
    """The library's object for these shapes, and the output buffers a program keeps."""
    from paper_1907_11210_amd import train
    if case["kind"].startswith("layer"):
        s["norm"] = train.LayerNorm(_shape(case), DTYPES[case["dtype"]],
                                    "NCHW" if case["layout"] == "NCHW" else "NHWC", case["act"],
                                    NORM_EPS)
        s["out"] = torch.empty_like(s["x"])
        if case["kind"] == "layer":
            s["stats"] = s["norm"].new_stats()
    elif case["kind"] == "orthogonal":
        s["orthogonalize"] = train.Orthogonalize(s["x"].shape, s["x"].dtype, steps=STEPS,
                                                 coefficients=COEFFICIENTS, eps=EPS)
        s["out"] = torch.empty_like(s["x"])
    else:
        s["muon"] = train.Muon(_views(s, "p"), weight_decay=DECAY, scales=s["scales"],
                               copies=_views(s, "copy") if case["copy"] else None,
                               grad_dtypes=[g.dtype for g in s["grads"]], m=_views(s, "m"),
                               steps=STEPS, coefficients=COEFFICIENTS, eps=EPS)


# ---- one pass -----------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    if kind == "muon":
        if own:
            state["muon"].step(state["grads"], lr=LR, momentum=MOMENTUM, nesterov=True)
        else:
            _plain_muon(state)
        return {k: state[k] for k in ("p", "m", "copy") if k in state}
    if not own:
        return {"layer": _plain_layer, "layer_grad": _plain_layer_grad,
                "orthogonal": _plain_orthogonal}[kind](state)
    if kind == "layer":
        y = state["norm"](state["x"], state["gamma"], state["beta"], out=state["out"],
                          stats=state["stats"])
        return y, state["stats"]
    if kind == "layer_grad":
        return state["norm"].grad(state["x"], state["dy"], state["stats"], state["gamma"],
                                  state["beta"], out=state["out"])
    return state["orthogonalize"](state["x"], out=state["out"])


# ---- plain forms: elementary operations in 32 bits ------------------------------

def _activate(z, act):
    if act == "relu":
        return torch.where(z < 0, 0, z)
    return {"none": lambda: z, "tanh": lambda: torch.tanh(z),
            "silu": lambda: z / (1 + torch.exp(-z))}[act]()


def _params(s):
    shape = (-1, 1, 1) if s["case"]["layout"] == "NCHW" else (-1,)
    return s["gamma"].reshape(shape), s["beta"].reshape(shape)


def _plain_layer(s):
    case, axis = s["case"], _axis(s["case"])
    gamma, beta = _params(s)
    x = s["x"].float()
    mean = x.mean(axis, keepdim=True)
    xc = x - mean
    rstd = 1 / torch.sqrt((xc * xc).mean(axis, keepdim=True) + NORM_EPS)
    y = _activate(xc * rstd * gamma + beta, case["act"]).to(s["x"].dtype)
    return y, torch.stack((mean.flatten(), rstd.flatten()), -1)


def _activation_grad(dy, z, act):
    if act == "none":
        return dy
    if act == "relu":
        return torch.where(z > 0, dy, 0)
    if act == "tanh":
        th = torch.tanh(z)
        return dy * (1 - th * th)
    sig = 1 / (1 + torch.exp(-z))
    return dy * (sig * (1 + z * (1 - sig)))


def _plain_layer_grad(s):
    case, axis = s["case"], _axis(s["case"])
    gamma, beta = _params(s)
    x, dy = s["x"].float(), s["dy"].float()
    shape = list(x.shape)
    shape[axis] = 1
    mean, rstd = s["stats"][:, 0].reshape(shape), s["stats"][:, 1].reshape(shape)
    xh = (x - mean) * rstd
    dz = _activation_grad(dy, xh * gamma + beta, case["act"])
    t = dz * gamma
    dx = rstd * (t - t.mean(axis, keepdim=True) - xh * (t * xh).mean(axis, keepdim=True))
    pixels = tuple(i for i in range(x.dim()) if i != axis % x.dim())
    return dx.to(s["x"].dtype), (dz * xh).sum(pixels), dz.sum(pixels)


def _newton_schulz(x):
    """Five steps for matrices [..., rows, cols] in 32 bits, each normalised first."""
    a, b, c = COEFFICIENTS
    x = x / (torch.sqrt((x * x).sum((-2, -1), keepdim=True)) + EPS)
    tall = x.shape[-2] > x.shape[-1]
    if tall:
        x = x.mT.contiguous()
    for _ in range(STEPS):
        g = x @ x.mT
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.mT.contiguous() if tall else x


def _plain_orthogonal(s):
    return _newton_schulz(s["x"].float()).to(s["x"].dtype)


def _plain_muon(s):
    copies = _views(s, "copy") if "copy" in s else [None] * len(s["shapes"])
    for p, m, g, copy, scale in zip(_views(s, "p"), _views(s, "m"), s["grads"], copies,
                                    s["scales"]):
        g = g.float()
        m.copy_(MOMENTUM * m + (1 - MOMENTUM) * g)
        x = _newton_schulz(MOMENTUM * m + (1 - MOMENTUM) * g)
        new = p.float() * (1 - LR * DECAY) - (LR * scale) * x
        p.copy_(new)
        if copy is not None:
            copy.copy_(new)


# ---- 64-bit results from the definitions ------------------------------------------

def _exact_layer(x, gamma, beta, case):
    axis = _axis(case)
    rows = x.movedim(axis, -1)
    var, mean = torch.var_mean(rows, -1, correction=0)
    rstd = (var + NORM_EPS) ** -0.5
    z = torch.addcmul(beta, (rows - mean[..., None]) * rstd[..., None], gamma)
    y = {"none": lambda v: v, "relu": torch.relu, "tanh": torch.tanh,
         "silu": torch.nn.functional.silu}[case["act"]](z)
    return y.movedim(-1, axis), torch.stack((mean.flatten(), rstd.flatten()), 1)


def _exact_orthogonal(x):
    """p(p(...)) of the singular values, through the smaller of X X^T and X^T X."""
    a, b, c = COEFFICIENTS
    x = x / (torch.linalg.matrix_norm(x) + EPS)
    wide = x.shape[0] <= x.shape[1]
    eye = torch.eye(min(x.shape), dtype=x.dtype, device=x.device)
    for _ in range(STEPS):
        g = x @ x.mT if wide else x.mT @ x
        poly = torch.addmm(a * eye, g, b * eye + c * g)
        x = poly @ x if wide else x @ poly
    return x


def exact(case, seed):
    s, kind = _inputs(case, seed), case["kind"]
    if kind == "layer":
        y, stats = _exact_layer(s["x"].double(), s["gamma"].double(), s["beta"].double(), case)
        return y.contiguous(), stats
    if kind == "layer_grad":  # the forward's definition, differentiated
        inputs = [s[k].double().requires_grad_() for k in ("x", "gamma", "beta")]
        y, _ = _exact_layer(*inputs, case)
        dx, dgamma, dbeta = torch.autograd.grad(y, inputs, s["dy"].double())
        return dx.contiguous(), dgamma, dbeta
    if kind == "orthogonal":
        return torch.stack([_exact_orthogonal(x) for x in s["x"].double()])
    out = {"p": s["p"].double(), "m": s["m"].double()}
    for a, n, shape, g, scale in zip(s["at"], s["sizes"], s["shapes"], s["grads"], s["scales"]):
        p, m = out["p"][a:a + n], out["m"][a:a + n]
        g = g.double().flatten()
        m.lerp_(g, 1 - MOMENTUM)
        update = _exact_orthogonal(torch.lerp(m, g, 1 - MOMENTUM).view(shape)).flatten()
        p.copy_(p - LR * DECAY * p - LR * scale * update)
    if case["copy"]:
        out["copy"] = out["p"]
    return out
