"""Performance cases of the operators around a generator's convolutions: group
norm with an activation, embedding lookup, and the AdamW step, with their
gradients.

A case is one pass through one operator:

  norm        y = act(group_norm(x)), and the statistics that training keeps.
  norm_grad   its gradients for x, gamma and beta, from x, dy and the statistics.
  embed       y[t] = scale * table[id[t]]; an id outside the table reads zeros.
  embed_grad  the table's gradient, dense, in the table's type.
  adamw       one AdamW step over a list of tensors, in place, with the moments
              in 32 bits or as e4m3 numbers with a scale for 256 of them.

Inputs are drawn on the GPU from the seed alone.
"""
from __future__ import annotations

import math

import torch

own = False  # False: the plain forms below; True: the library's kernels

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
BLOCK = 256                 # values that share a scale in the 8-bit moments
CODE_MAX, CODE_MIN = 448.0, 2.0 ** -9  # largest and smallest positive e4m3 number
LR, BETAS, EPS = 2e-4, (0.9, 0.999), 1e-8
NORM_EPS = 1e-5


def _norm(kind, n, h, w, c, groups, layout="NHWC", dtype="bf16", act="relu"):
    return dict(kind=kind, n=n, h=h, w=w, c=c, groups=groups, layout=layout, dtype=dtype, act=act)


def _embed(kind, tokens, rows, dim, dtype="bf16", ids="uniform", pad=0.0):
    return dict(kind=kind, tokens=tokens, rows=rows, dim=dim, dtype=dtype, ids=ids, pad=pad)


def _adamw(tensors, lo, hi, bits=32, param="f32", grad="f32", copy=False):
    return dict(kind="adamw", tensors=tensors, lo=lo, hi=hi, bits=bits, param=param, grad=grad,
                copy=copy)


def listed():
    return [
        # One image through the generator: the norm behind its second layer (latency).
        dict(_norm("norm", 1, 8, 8, 512, 32), name="norm_gen_b1"),
        # The generator's training batch in the weight gradients' layout, behind its third layer.
        dict(_norm("norm", 64, 16, 16, 256, 32, layout="NCHW"), name="norm_gen_b64_nchw"),
        # The feature map that the atrous pyramid reads: large, few images.
        dict(_norm("norm", 8, 64, 64, 2048, 32), name="norm_features_b8"),
        # Training the generator: the norm behind its fourth layer, where maps are largest.
        dict(_norm("norm_grad", 64, 32, 32, 128, 32), name="norm_grad_gen_b64"),
        # A decoder block on an odd crop, full precision: 25 channels a group.
        dict(_norm("norm_grad", 5, 33, 41, 200, 8, dtype="f32", act="silu"),
             name="norm_grad_ragged_f32"),
        # Class labels of a conditional generator, one batch (latency).
        dict(_embed("embed", 64, 100, 100), name="embed_labels"),
        # Maps of code indices to a decoder's latents: 64 maps of 32 x 32.
        dict(_embed("embed", 65536, 8192, 256), name="embed_codes"),
        # The codes' gradient at 16 x 16: few rows, each with many tokens.
        dict(_embed("embed_grad", 16384, 1024, 256, dtype="f32"), name="embed_grad_codes_f32"),
        # Text tokens: most rows untouched, some with thousands of tokens, a tenth padding.
        dict(_embed("embed_grad", 32768, 40000, 1024, ids="skewed", pad=0.1),
             name="embed_grad_text"),
        # The generator's parameters: fp32 weights, bf16 gradients and working copies.
        dict(_adamw(13, 100, 1 << 23, grad="bf16", copy=True), name="adamw_generator"),
        # The largest step: 134 M parameters in large tensors.
        dict(_adamw(8, 1 << 24, 1 << 24), name="adamw_large"),
        # Many small odd tensors with 8-bit moments (launches), bf16 gradients.
        dict(_adamw(160, 33, 99999, bits=8, grad="bf16", copy=True), name="adamw8_small"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case that costs no more than the largest listed one of its kind."""
    while True:
        kind = rng.choice(("norm", "norm", "norm_grad", "norm_grad", "embed", "embed_grad",
                           "embed_grad", "adamw", "adamw"))
        dtype = rng.choice(("bf16", "bf16", "f32"))
        if kind.startswith("norm"):
            groups = rng.choice((1, 2, 4, 8, 16, 32, 32))
            c = _log_int(rng, 16, 2048)
            if rng.random() < 2 / 3:
                c = max(8, c // 8 * 8)
            c = max(groups, c // groups * groups)
            case = _norm(kind, _log_int(rng, 1, 64), _log_int(rng, 1, 128), _log_int(rng, 1, 128),
                         c, groups, rng.choice(("NHWC", "NHWC", "NCHW")), dtype,
                         rng.choice(("none", "relu", "tanh", "silu")))
            # (a gradient over a few values alone is rounding: it sums to zero in exact terms)
            if case["h"] * case["w"] * c >= 16 * groups and \
                    case["n"] * case["h"] * case["w"] * c <= (1 << 26) * 2 // SIZE[dtype]:
                return case
        elif kind.startswith("embed"):
            dim = _log_int(rng, 16, 2048)
            if rng.random() < 2 / 3:
                dim = max(8, dim // 8 * 8)
            case = _embed(kind, _log_int(rng, 1, 65536), _log_int(rng, 10, 60000), dim, dtype,
                          rng.choice(("uniform", "skewed", "skewed", "one")),
                          rng.choice((0.0, 0.1, 0.5)))
            if max(case["tokens"], case["rows"]) * dim <= (1 << 25):
                return case
        else:
            hi = _log_int(rng, 100, 1 << 24)
            case = _adamw(_log_int(rng, 1, 200), _log_int(rng, 1, hi), hi, rng.choice((8, 32)),
                          rng.choice(("f32", "f32", "bf16")), dtype, rng.random() < 0.5)
            case["copy"] = case["copy"] and case["param"] == "f32"
            if sum(_sizes(case)) <= 1 << 26:
                return case


def _sizes(case):
    """Element counts from lo to hi, spread over their logarithm, largest first."""
    k, lo, hi = case["tensors"], case["lo"], case["hi"]
    return [int(round(hi * (lo / hi) ** (i / max(1, k - 1)))) for i in range(k)]


def work(case):
    kind = case["kind"]
    if kind.startswith("norm"):
        numel = case["n"] * case["h"] * case["w"] * case["c"]
        stats = 8 * case["n"] * case["groups"]
        if kind == "norm":  # x, gamma, beta in; y, statistics out
            return {"bytes": 2 * numel * SIZE[case["dtype"]] + 8 * case["c"] + stats,
                    "flops": 10 * numel}
        # x, dy, statistics, gamma, beta in; dx, dgamma, dbeta out
        return {"bytes": 3 * numel * SIZE[case["dtype"]] + 16 * case["c"] + stats,
                "flops": 20 * numel}
    if kind.startswith("embed"):
        t, v, d, e = case["tokens"], case["rows"], case["dim"], SIZE[case["dtype"]]
        rows = min(t, v) if kind == "embed" else v  # rows read, or rows written
        return {"bytes": 8 * t + (t + rows) * d * e, "flops": t * d}
    state = 8 if case["bits"] == 32 else 2 + 8 / BLOCK
    each = 2 * SIZE[case["param"]] + SIZE[case["grad"]] + 2 * state + (2 if case["copy"] else 0)
    return {"bytes": sum(_sizes(case)) * each, "flops": 15 * sum(_sizes(case))}


# ---- inputs -----------------------------------------------------------------

def _device():
    return torch.device("cuda", torch.cuda.current_device())


def _shape(case):
    n, h, w, c = (case[k] for k in ("n", "h", "w", "c"))
    return (n, h, w, c) if case["layout"] == "NHWC" else (n, c, h, w)


def _split(t, case):
    """[n, groups, channels a group, pixels] of a tensor in the case's layout (a view)."""
    n, g = case["n"], case["groups"]
    if case["layout"] == "NHWC":
        return t.reshape(n, -1, g, case["c"] // g).permute(0, 2, 3, 1)
    return t.reshape(n, g, case["c"] // g, -1)


def _norm_inputs(case, g):
    normal = lambda *s: torch.randn(s, generator=g, device=g.device)  # noqa: E731
    c, dtype = case["c"], DTYPES[case["dtype"]]
    by_channel = (c,) if case["layout"] == "NHWC" else (c, 1, 1)
    # what a convolution with a bias leaves: channels of their own mean and scale
    scale, shift = (0.5 + normal(c).abs()).reshape(by_channel), normal(c).reshape(by_channel)
    s = {"x": (normal(*_shape(case)) * scale + shift).to(dtype),
         "gamma": 1 + 0.1 * normal(c), "beta": 0.1 * normal(c)}
    if case["kind"] == "norm_grad":
        s["dy"] = normal(*_shape(case)).to(dtype)
        x = _split(s["x"], case)
        mean = x.mean((2, 3), dtype=torch.float64)
        var = torch.stack([v.double().var((1, 2), correction=0) for v in x])
        s["stats"] = torch.stack((mean, (var + NORM_EPS).rsqrt()), -1).float()
    return s


def _embed_inputs(case, g):
    t, v, d = case["tokens"], case["rows"], case["dim"]
    u = torch.rand(t, generator=g, device=g.device, dtype=torch.float64)
    if case["ids"] == "uniform":
        ids = (u * v).long()
    elif case["ids"] == "skewed":  # frequency falls as one over the rank; ranks lie anywhere
        step = next(p for p in (7919, 7907, 7901, 7883, 7879) if v % p)
        ids = ((v + 1.0) ** u).long().clamp(1, v) * step % v
    else:
        ids = torch.full((t,), v // 2, device=g.device)
    ids = ids.clamp(0, v - 1)
    ids[torch.rand(t, generator=g, device=g.device) < case["pad"]] = -1
    s = {"ids": ids, "scale": math.sqrt(d)}
    name, rows = ("table", v) if case["kind"] == "embed" else ("dy", t)
    s[name] = torch.randn((rows, d), generator=g, device=g.device).to(DTYPES[case["dtype"]])
    return s


def _adamw_inputs(case, g):
    sizes = _sizes(case)
    padded = [-(-n // BLOCK) * BLOCK for n in sizes]  # tensors lie on whole blocks of a buffer
    at = [sum(padded[:i]) for i in range(len(sizes))]
    total, dev = sum(padded), g.device
    inside = torch.zeros(total, dtype=torch.bool, device=dev)
    for a, n in zip(at, sizes):
        inside[a:a + n] = True
    seen = inside & (torch.rand(total, generator=g, device=dev) > 0.1)  # never had a gradient
    normal = lambda: torch.randn(total, generator=g, device=dev)  # noqa: E731
    grad = torch.where(seen, normal() * 1e-2, 0).to(DTYPES[case["grad"]])
    m = torch.where(seen, normal() * 3e-3, 0)
    v = torch.where(seen, 1e-4 * (0.3 + normal().square()), 0)
    s = {"p": torch.where(inside, normal() * 0.02, 0).to(DTYPES[case["param"]]),
         "sizes": sizes, "at": at, "t": 10,
         # matrices decay, biases and norms (the small ones) do not
         "decay": [0.01 if n >= 1024 else 0.0 for n in sizes],
         "grads": [grad[a:a + n].clone() for a, n in zip(at, sizes)]}
    s["block_decay"] = torch.tensor([d for d, q in zip(s["decay"], padded)
                                     for _ in range(q // BLOCK)], device=dev)[:, None]
    if case["bits"] == 32:
        s["m"], s["v"] = m, v
    else:
        s["m"], s["m_scale"] = _encode(m, 0.0)
        s["v"], s["v_scale"] = _encode(v.sqrt(), CODE_MIN)
    if case["copy"]:
        s["copy"] = s["p"].to(torch.bfloat16)
    return s


def _inputs(case, seed):
    g = torch.Generator(_device()).manual_seed(seed)
    make = {"norm": _norm_inputs, "embed": _embed_inputs, "adamw": _adamw_inputs}
    return make[case["kind"].split("_")[0]](case, g)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        _handle(s, case)
    return s


def _handle(s, case):
    """The library's object for these shapes, and the output buffers a program keeps."""
    from paper_1907_11210_amd import train
    kind = case["kind"]
    if kind.startswith("norm"):
        s["norm"] = train.GroupNorm(_shape(case), case["groups"], DTYPES[case["dtype"]],
                                    case["layout"], case["act"], NORM_EPS)
        s["out"] = torch.empty_like(s["x"])
        if kind == "norm":
            s["stats"] = torch.empty((case["n"], case["groups"], 2), device=s["x"].device)
    elif kind.startswith("embed"):
        s["embedding"] = train.Embedding(case["rows"], case["dim"], DTYPES[case["dtype"]],
                                         scale=s["scale"], max_tokens=case["tokens"])
        rows = case["tokens"] if kind == "embed" else case["rows"]
        s["out"] = torch.empty((rows, case["dim"]), dtype=DTYPES[case["dtype"]],
                               device=s["ids"].device)
    else:
        def views(name, per=1):
            return [s[name][a // per:a // per + -(-n // per)] for a, n in zip(s["at"], s["sizes"])]
        more = {} if case["bits"] == 32 else {"m_scale": views("m_scale", BLOCK),
                                              "v_scale": views("v_scale", BLOCK)}
        s["adamw"] = train.AdamW(views("p"), state_bits=case["bits"], weight_decay=s["decay"],
                                 m=views("m"), v=views("v"),
                                 copies=views("copy") if case["copy"] else None,
                                 grad_dtypes=[g.dtype for g in s["grads"]], **more)


# ---- one pass -----------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    if kind == "adamw":
        state["t"] += 1
        (_run_adamw if own else _plain_adamw)(state)
        return {k: state[k] for k in ("p", "m", "v", "m_scale", "v_scale", "copy") if k in state}
    if not own:
        return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "embed": _plain_embed,
                "embed_grad": _plain_embed_grad}[kind](state)
    if kind == "norm":
        y = state["norm"](state["x"], state["gamma"], state["beta"], out=state["out"],
                          stats=state["stats"])
        return y, state["stats"]
    if kind == "norm_grad":
        return state["norm"].grad(state["x"], state["dy"], state["stats"], state["gamma"],
                                  state["beta"], out=state["out"])
    if kind == "embed":
        return state["embedding"](state["ids"], state["table"], out=state["out"])
    return state["embedding"].grad(state["ids"], state["dy"], out=state["out"])


def _run_adamw(s):
    s["adamw"].step(s["grads"], lr=LR, betas=BETAS, eps=EPS, step=s["t"])


# ---- plain forms: elementary operations in 32 bits ------------------------------

def _activate(z, act):
    if act == "relu":
        return torch.where(z < 0, 0, z)
    return {"none": lambda: z, "tanh": lambda: torch.tanh(z),
            "silu": lambda: z / (1 + torch.exp(-z))}[act]()


def _plain_norm(s):
    case = s["case"]
    x = _split(s["x"], case).float()
    mean = x.mean((2, 3), keepdim=True)
    xc = x - mean
    rstd = 1 / torch.sqrt((xc * xc).mean((2, 3), keepdim=True) + NORM_EPS)
    by_channel = (case["groups"], -1, 1)
    z = xc * rstd * s["gamma"].reshape(by_channel) + s["beta"].reshape(by_channel)
    y = _activate(z, case["act"]).to(s["x"].dtype)
    return _joined(y, case), torch.stack((mean.flatten(1), rstd.flatten(1)), -1)


def _joined(y, case):
    """_split undone: contiguous in the case's layout."""
    if case["layout"] == "NHWC":
        y = y.permute(0, 3, 1, 2)
    return y.contiguous().reshape(_shape(case))


def _plain_norm_grad(s):
    case = s["case"]
    by_channel = (case["groups"], -1, 1)
    gamma, beta = s["gamma"].reshape(by_channel), s["beta"].reshape(by_channel)
    x, dy = _split(s["x"], case).float(), _split(s["dy"], case).float()
    mean, rstd = s["stats"][..., 0, None, None], s["stats"][..., 1, None, None]
    xh = (x - mean) * rstd
    dz = _activation_grad(dy, xh * gamma + beta, case["act"])
    t = dz * gamma
    dx = rstd * (t - t.mean((2, 3), keepdim=True) - xh * (t * xh).mean((2, 3), keepdim=True))
    return (_joined(dx.to(s["x"].dtype), case), (dz * xh).sum((0, 3)).flatten(),
            dz.sum((0, 3)).flatten())


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


def _plain_embed(s):
    ids, table = s["ids"], s["table"]
    known = (ids >= 0) & (ids < table.shape[0])
    rows = table[torch.where(known, ids, 0)].float() * s["scale"]
    return torch.where(known[:, None], rows, 0).to(table.dtype)


def _plain_embed_grad(s):
    ids, dy, rows = s["ids"], s["dy"], s["case"]["rows"]
    known = (ids >= 0) & (ids < rows)
    dw = torch.zeros((rows + 1, dy.shape[1]), device=dy.device)  # the last row takes the unknown
    dw.index_add_(0, torch.where(known, ids, rows), dy.float())
    return (dw[:rows] * s["scale"]).to(dy.dtype)


def _decode(codes, scale):
    return codes.float().reshape(-1, BLOCK) * scale[:, None]


def _encode(values, least):
    """e4m3 numbers and a scale for each block, so that its largest magnitude is 448; a block
    with nothing over 2^-100 is all zeros, and no positive number is rounded below `least`."""
    blocks = values.reshape(-1, BLOCK)
    top = blocks.abs().amax(1)
    none = top < 2.0 ** -100
    codes = blocks * torch.where(none, 0, CODE_MAX / top)[:, None]
    codes = torch.where((codes > 0) & (codes < least), least, codes)
    return codes.to(torch.float8_e4m3fn).flatten(), torch.where(none, 0, top / CODE_MAX)


def _plain_adamw(s):
    case, t, (b1, b2) = s["case"], s["t"], BETAS
    zeros = s["grads"][0].new_zeros(BLOCK)
    pieces = [x for g in s["grads"] for x in (g, zeros[:-g.numel() % BLOCK])]
    g = torch.cat(pieces).float().reshape(-1, BLOCK)
    m, v, p = s["m"], s["v"], s["p"].float().reshape(-1, BLOCK)
    if case["bits"] == 8:
        m, v = _decode(m, s["m_scale"]), _decode(v, s["v_scale"])
        v = v * v
    m = b1 * m.reshape(-1, BLOCK) + (1 - b1) * g
    v = b2 * v.reshape(-1, BLOCK) + (1 - b2) * (g * g)
    step = m / (torch.sqrt(v) / math.sqrt(1 - b2 ** t) + EPS)
    p = (p * (1 - LR * s["block_decay"]) - (LR / (1 - b1 ** t)) * step).flatten()
    s["p"].copy_(p)
    if case["copy"]:
        s["copy"].copy_(p)
    if case["bits"] == 8:
        m, s["m_scale"][:] = _encode(m, 0.0)
        v, s["v_scale"][:] = _encode(torch.sqrt(v), CODE_MIN)
    s["m"].copy_(m.flatten())
    s["v"].copy_(v.flatten())


# ---- 64-bit results from the definitions ------------------------------------------

def _exact_forward(x, gamma, beta, case):
    n, g, act = case["n"], case["groups"], case["act"]
    axis = 3 if case["layout"] == "NHWC" else 1
    rows = x.movedim(axis, 1).reshape(n * g, -1)
    var, mean = torch.var_mean(rows, 1, correction=0)
    rstd = (var + NORM_EPS) ** -0.5
    rows = (rows - mean[:, None]) * rstd[:, None]
    z = rows.reshape(n, case["c"], -1) * gamma[:, None] + beta[:, None]
    y = {"none": lambda v: v, "relu": torch.relu, "tanh": torch.tanh,
         "silu": torch.nn.functional.silu}[act](z)
    y = y.reshape(n, case["c"], case["h"], case["w"]).movedim(1, axis)
    return y, torch.stack((mean, rstd), 1).reshape(n, g, 2)


def _exact_adamw(s, case):
    t, (b1, b2), out = s["t"] + 1, BETAS, {k: [] for k in ("p", "m", "v")}
    for a, n, g, decay in zip(s["at"], s["sizes"], s["grads"], s["decay"]):
        q = -(-n // BLOCK) * BLOCK
        g = torch.nn.functional.pad(g.double(), (0, q - n))
        p, m, v = (s[k][a:a + q].double() for k in ("p", "m", "v"))
        if case["bits"] == 8:
            of = slice(a // BLOCK, (a + q) // BLOCK)
            m = m * s["m_scale"][of].double().repeat_interleave(BLOCK)
            v = (v * s["v_scale"][of].double().repeat_interleave(BLOCK)) ** 2
        m.lerp_(g, 1 - b1)
        v.lerp_(g ** 2, 1 - b2)
        step = (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + EPS)
        for k, x in (("p", p - LR * decay * p - LR * step), ("m", m), ("v", v)):
            out[k].append(x)
    out = {k: torch.cat(x) for k, x in out.items()}
    if case["copy"]:
        out["copy"] = out["p"]
    if case["bits"] == 8:  # the numbers that the codes round
        out["v"] = out["v"].sqrt()
        for k in ("m", "v"):
            top = out[k].reshape(-1, BLOCK).abs().amax(1)
            out[k + "_scale"] = top / CODE_MAX
            out[k] = out[k] * torch.where(top > 0, CODE_MAX / top, 0).repeat_interleave(BLOCK)
    return out


def exact(case, seed):
    s, kind = _inputs(case, seed), case["kind"]
    if kind == "adamw":
        return _exact_adamw(s, case)
    if kind == "norm":
        y, stats = _exact_forward(s["x"].double(), s["gamma"].double(), s["beta"].double(), case)
        return y.contiguous(), stats
    if kind == "norm_grad":  # the forward's definition, differentiated
        inputs = [s[k].double().requires_grad_() for k in ("x", "gamma", "beta")]
        y, _ = _exact_forward(*inputs, case)
        dx, dgamma, dbeta = torch.autograd.grad(y, inputs, s["dy"].double())
        return dx.contiguous(), dgamma, dbeta
    ids, known = s["ids"], (s["ids"] >= 0) & (s["ids"] < case["rows"])
    if kind == "embed":
        y = torch.zeros((case["tokens"], case["dim"]), dtype=torch.float64, device=ids.device)
        y[known] = s["table"].double()[ids[known]] * s["scale"]
        return y
    dw = torch.zeros((case["rows"], case["dim"]), dtype=torch.float64, device=ids.device)
    return dw.index_put_((ids[known],), s["dy"][known].double() * s["scale"], accumulate=True)
