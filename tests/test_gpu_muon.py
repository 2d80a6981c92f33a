"""Orthogonalised matrices and the Muon step on the GPU, against the formulas in 64 bits.

Tolerances, of a result's norm: the products' operands are rounded to 11 bits, or to two parts of
11, their sums are fp32, and what that leaves depends on the matrix.  So each expectation comes
with the same steps whose operands are rounded so and whose sums are rounded to fp32 after every
8 columns of a product (a lane's share of a matrix instruction: a sum of 3 K / 8 such additions is
off by their number's root times one rounding, which steep singular values amplify 140 times as
they do the operands'): three times that error is allowed, and 2e-6 for a start where it is
nothing.  A small matrix has few roundings, whose sum may by chance be next to nothing: there the
model's error is the largest for six multiples of the matrix, which round differently and give
the same.  A single element is off by at most 12 times its share of
that.  Results in bf16 are rounded besides, by at most half
a step: bf16 numbers from 1 to 2 are 2^-7 apart, so 2^-8 of the value.
"""
import math

import pytest
import torch

from paper_1907_11210_amd import train as tr

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
QUINTIC = [tr.COEFFICIENTS] * 5


def _split(v, parts, power):
    """Parts of fp16, each the nearest to what is left, times a power of two."""
    v, of = v * 2.0 ** power, []
    for _ in range(parts):
        of.append(v.half().double())
        v = v - of[-1]
    return of


def _round(v, power):
    return sum(_split(v, 2, power)) / 2.0 ** power


def _product(p, q, parts, power):
    """p q^T from operands in parts, the sums in fp32."""
    ps, qs = _split(p, parts, power[0]), _split(q, parts, power[1])
    pairs = [(0, 0)] if parts == 1 else [(0, 0), (0, 1), (1, 0)]
    total = torch.zeros(p.shape[0], q.shape[0])
    for k in range(0, p.shape[1], 8):
        for i, j in pairs:
            total = (total.double() + ps[i][:, k:k + 8] @ qs[j][:, k:k + 8].T).float()
    return total.double() / 2.0 ** sum(power)


def _steps(u, parts=None, coefficients=QUINTIC, eps=1e-7):
    """The result in 64 bits, or with operands in so many parts."""
    x = u.double() / (u.double().norm() + eps)
    if x.shape[0] > x.shape[1]:
        return _steps(u.T, parts, coefficients, eps).T
    if parts is None:
        for a, b, c in coefficients:
            g = x @ x.T
            x = a * x + (b * g + c * (g @ g)) @ x
        return x
    x = _round(x, 14)
    for a, b, c in coefficients:
        g = _product(x, x, parts, (13, 13))
        mu = g.diagonal().mean()
        g = _round(g - mu * torch.eye(len(g), dtype=g.dtype), 13)
        poly = c * _product(g, g, parts, (13, 13)) + (b + 2 * c * mu) * g
        poly = poly.float().double()
        x = (a + b * mu + c * mu * mu) * x + _product(poly, x.T, parts, (10, 13))
        x = _round(x.float().double(), 13)
    return x


def _model_error(u, want, parts, coefficients=QUINTIC, eps=1e-7):
    """What the roundings leave, of the result's norm."""
    scales = (1.0,) if min(u.shape) > 64 or float(u.double().norm()) < 1e-3 else \
        (1.0, 1.1, 1.23, 1.41, 1.59, 1.83)
    return max(float((_steps(u.double() * s, parts, coefficients, eps) - want).norm())
               for s in scales) / float(want.norm())


def _close(got, u, dtype, parts, name, scale=1.0, coefficients=QUINTIC, eps=1e-7):
    want = _steps(u, coefficients=coefficients, eps=eps)
    size = float(want.norm())
    if size == 0:
        assert float(got.abs().max()) == 0
        return
    model = _model_error(u, want, parts, coefficients, eps)
    tol = 3 * model + 2e-6
    ulp = 2.0 ** -8 if dtype == torch.bfloat16 else U
    err = (got.double() - want)
    rms = size / math.sqrt(want.numel())
    print(name, "off by %.2e, allowed %.2e" % (float(err.norm()) / size, tol + ulp), flush=True)
    assert float(err.norm()) <= (tol + ulp) * size, name
    assert (err.abs() <= 12 * tol * rms + ulp * want.abs() * (1 + 2.0 ** -7)).all(), name


def _matrix(rows, cols, seed, kind="plain"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g)
    if kind == "plain" or min(rows, cols) < 2:
        return x
    if kind == "few":  # directions of a few samples, and bf16's roundings
        r = max(1, min(rows, cols) // 8)
        return (torch.randn(rows, r, generator=g) @ torch.randn(r, cols, generator=g)).bfloat16().float()
    m = min(rows, cols)  # singular values that fall with a power of their rank
    u = torch.linalg.qr(torch.randn(rows, m, generator=g).double())[0]
    v = torch.linalg.qr(torch.randn(cols, m, generator=g).double())[0]
    s = torch.arange(1, m + 1).double() ** (-2.0 if kind == "steep" else -0.5)
    return ((u * s) @ v.T).float()


SHAPES = [(1, 1), (1, 2), (3, 1), (2, 2), (1, 300), (5, 7), (16, 16), (33, 31), (48, 128), (64, 64),
          (65, 64), (100, 130), (128, 48), (129, 257), (256, 256), (257, 300), (320, 1000),
          (1000, 333), (64, 5000), (3000, 70), (511, 513)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("products", ["f32", "f16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_orthogonalize(shape, products, dtype):
    op = tr.Orthogonalize(shape, dtype, products)
    for kind in ("plain", "falling", "steep", "few"):
        x = _matrix(*shape, 1, kind).to(dtype)
        n = x.numel()
        whole = torch.full((n + 128,), 7, dtype=dtype, device=DEV)
        out = whole[64:64 + n].view(shape)
        print("orthogonalize", shape, products, dtype, kind, flush=True)
        assert op(x.to(DEV), out=out) is out
        torch.cuda.synchronize()
        assert bool((whole[:64] == 7).all() and (whole[-64:] == 7).all())
        _close(out.cpu(), x, dtype, 2 if products == "f32" else 1, kind)


@pytest.mark.parametrize("products", ["f32", "f16"])
@pytest.mark.parametrize("shape", [(7, 40, 56), (3, 300, 129), (2, 2, 5, 66), (300, 3, 5), (0, 4, 5)],
                         ids=lambda s: "x".join(map(str, s)))
def test_batches(shape, products):
    """Each matrix as alone, more of them than share launches among them."""
    if 0 in shape:
        with pytest.raises(tr.h2.Huge2Error):
            tr.Orthogonalize(shape, torch.float32)
        return
    g = torch.Generator().manual_seed(2)
    x = torch.randn(shape, generator=g) * 10.0 ** torch.randint(-9, 9, (*shape[:-2], 1, 1), generator=g)
    y = tr.Orthogonalize(shape, torch.float32, products)(x.to(DEV)).cpu()
    xs, ys = x.reshape(-1, *shape[-2:]), y.reshape(-1, *shape[-2:])
    for i in list(range(min(6, len(xs)))) + [len(xs) - 1]:
        _close(ys[i], xs[i], torch.float32, 2 if products == "f32" else 1, i)


@pytest.mark.parametrize("products", ["f32", "f16"])
@pytest.mark.parametrize("scale", [2.0 ** -120, 1e-20, 1e-8, 1e-3, 1e18, 2.0 ** 120])
def test_sizes_of_values(scale, products):
    """Squares of these neither vanish nor overflow; below eps a matrix shrinks with its norm."""
    x = _matrix(40, 60, 3) * scale
    y = tr.Orthogonalize(x.shape, torch.float32, products)(x.to(DEV)).cpu()
    _close(y, x, torch.float32, 2 if products == "f32" else 1, scale)


@pytest.mark.parametrize("products", ["f32", "f16"])
@pytest.mark.parametrize("coefficients,steps", [
    ((2.0, -1.5, 0.5), 3), ((1.5, -0.5, 0.0), 6), ((1.0, 0.0, 0.0), 2), ((3.4445, -4.775, 2.0315), 1),
    ([(8.28, -23.6, 17.3), (4.1, -2.95, 0.545), (3.95, -2.91, 0.55)], 3), ((0.5, 0.1, -0.05), 4)])
def test_other_polynomials(coefficients, steps, products):
    x = _matrix(70, 110, 4)
    triples = [coefficients] * steps if not isinstance(coefficients, list) else coefficients
    y = tr.Orthogonalize(x.shape, torch.float32, products, steps, coefficients)(x.to(DEV)).cpu()
    _close(y, x, torch.float32, 2 if products == "f32" else 1, coefficients, coefficients=triples)


@pytest.mark.parametrize("products", ["f32", "f16"])
@pytest.mark.parametrize("steps", [1, 2, 3])
def test_few_steps_of_a_tall_matrix(steps, products):
    """The last step is formed across, from what the step before it (or the packing) leaves."""
    x = _matrix(300, 90, 7)
    y = tr.Orthogonalize(x.shape, torch.float32, products, steps)(x.to(DEV)).cpu()
    _close(y, x, torch.float32, 2 if products == "f32" else 1, steps,
           coefficients=QUINTIC[:steps])


@pytest.mark.parametrize("products", ["f32", "f16"])
@pytest.mark.parametrize("shape", [(3, 130, 1100), (700, 300), (260, 515)],
                         ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("tile", [0, 1, 2])
def test_every_tile(tile, shape, products, monkeypatch):
    """Each size of tiles, also where the rule would take another: sums cut and joined, tiles
    over the matrices' ends and over the diagonal; and a Muon step of the same."""
    monkeypatch.setenv("HUGE2_NS_TILE", str(tile))
    parts = 2 if products == "f32" else 1
    x = torch.stack([_matrix(*shape[-2:], 8 + i) for i in range(3)])[:shape[0] if len(shape) == 3 else 1]
    op = tr.Orthogonalize(x.shape, torch.float32, products)
    print("tile", tile, shape, products, flush=True)
    y = op(x.to(DEV)).cpu()
    for a, b in zip(y, x):
        _close(a, b, torch.float32, parts, tile)
    s = _state([tuple(shape[-2:]), (33, 40)], torch.float32, torch.float32, 9)
    muon, dev = _muon(s, True, 0.1, products=products)
    muon.step(dev["g"], lr=0.02)
    torch.cuda.synchronize()
    for i in range(2):
        _check(s, dev, muon, i, 0.1, 0.02)


def test_singular_values():
    """Near 1 wherever they were, and the singular vectors stay."""
    for shape in ((200, 333), (333, 200)):
        x = _matrix(*shape, 5, "falling")
        y = tr.Orthogonalize(shape, torch.float32)(x.to(DEV)).cpu().double()
        s = torch.linalg.svdvals(y)
        assert 0.6 < float(s.min()) and float(s.max()) < 1.25
        u, _, vt = torch.linalg.svd(x.double(), full_matrices=False)
        core = u.T @ y @ vt.T
        assert float((core - torch.diag(core.diagonal())).norm()) <= 1e-4 * float(core.norm())


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("products", ["f32", "f16"])
def test_not_finite_stays_in_its_matrix(products, value):
    x = torch.stack([_matrix(70, 150, 6 + i) for i in range(3)])
    x[1, 69, 149] = value
    y = tr.Orthogonalize(x.shape, torch.float32, products)(x.to(DEV)).cpu()
    assert torch.isnan(y[1]).all()
    assert torch.isfinite(y[0]).all() and torch.isfinite(y[2]).all()
    x[1] = 0
    y = tr.Orthogonalize(x.shape, torch.float32, products)(x.to(DEV)).cpu()
    assert float(y[1].abs().max()) == 0 and torch.isfinite(y).all()


# ---- the Muon step ------------------------------------------------------------

CONV = [(24, 16, 4, 4), (16, 3, 4, 4), (10, 24), (1, 5), (7, 1), (130, 90), (90, 300)]


def _state(shapes, pdtype, gdtype, seed):
    g = torch.Generator().manual_seed(seed)
    rand = lambda s: torch.randn(s, generator=g)  # noqa: E731
    return dict(p=[rand(s).to(pdtype) for s in shapes],
                g=[(rand(s) * 10.0 ** (i % 5 - 3)).to(gdtype) for i, s in enumerate(shapes)],
                m=[rand(s) * 10.0 ** (i % 5 - 3) for i, s in enumerate(shapes)])


def _check(s, dev, muon, i, decay, lr, momentum=0.95, nesterov=True, gs=1.0):
    """Parameter i against the formulas, from the state that the step found."""
    p, g, m = (s[k][i].double() for k in ("p", "g", "m"))
    g = g * gs
    rows = p.shape[0]
    m2 = momentum * m + (1 - momentum) * g
    mag = momentum * m.abs() + (1 - momentum) * g.abs()
    got_m = dev["m"][i].cpu().double()
    assert ((got_m - m2).abs() <= 6 * U * mag).all(), i
    u = momentum * m2 + (1 - momentum) * g if nesterov else m2
    u = u.reshape(rows, -1)
    want = _steps(u)
    parts = 2 if muon.products == "f32" else 1
    # (u itself is off by 12 u of its terms, which the model's 24 bits of X stand for)
    tol = 3 * _model_error(u, want, parts) + 2e-6 + 200 * U
    p2 = p * (1 - lr * decay) - lr * muon.scales[i] * want.reshape(p.shape)
    rms = float(want.norm()) / math.sqrt(want.numel())
    off = 12 * tol * rms * lr * abs(muon.scales[i]) + 8 * U * (p.abs() + lr * abs(muon.scales[i]) *
                                                                want.abs().reshape(p.shape))
    got = dev["p"][i].cpu().double()
    if dev["p"][i].dtype == torch.bfloat16:
        lo, hi = ((p2 + d).to(torch.bfloat16).double() for d in (-off, off))
        assert ((got >= lo) & (got <= hi)).all(), i
    else:
        assert ((got - p2).abs() <= off + U * p2.abs()).all(), i
    if muon.copies[i] is not None:
        assert torch.equal(muon.copies[i], dev["p"][i].bfloat16()), i


def _muon(s, copies, decay, **kw):
    dev = {k: [t.to(DEV) for t in s[k]] for k in s}
    copy = [torch.full(p.shape, 5, dtype=torch.bfloat16, device=DEV) for p in dev["p"]] \
        if copies else None
    return tr.Muon(dev["p"], decay, copies=copy, grad_dtypes=[g.dtype for g in dev["g"]], m=dev["m"],
                   **kw), dev


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("gdtype", [torch.float32, torch.bfloat16], ids=["gf32", "gbf16"])
@pytest.mark.parametrize("pdtype", [torch.float32, torch.bfloat16], ids=["pf32", "pbf16"])
def test_step(pdtype, gdtype, nesterov):
    s = _state(CONV, pdtype, gdtype, 1)
    decay = [0.1 * (i % 3) for i in range(len(CONV))]
    muon, dev = _muon(s, pdtype == torch.float32, decay)
    print("muon", pdtype, gdtype, nesterov, flush=True)
    muon.step(dev["g"], lr=0.02, nesterov=nesterov)
    torch.cuda.synchronize()
    for i in range(len(CONV)):
        _check(s, dev, muon, i, decay[i], 0.02, nesterov=nesterov)


@pytest.mark.parametrize("products", ["f32", "f16"])
def test_many_matrices(products):
    """More than share launches, of many shapes; some without a gradient, whose parameters,
    momenta and copies stay."""
    shapes = [(1 + 7 * i % 90, 1 + 11 * i % 130) for i in range(270)]
    s = _state(shapes, torch.float32, torch.bfloat16, 2)
    muon, dev = _muon(s, True, 0.01, products=products)
    grads = [None if i % 9 == 4 else g for i, g in enumerate(dev["g"])]
    before = [t.clone() for t in muon.copies]
    muon.step(grads, lr=0.1, momentum=0.9)
    torch.cuda.synchronize()
    for i in range(270):
        if grads[i] is None:
            assert torch.equal(dev["p"][i].cpu(), s["p"][i]) and torch.equal(dev["m"][i].cpu(), s["m"][i])
            assert torch.equal(muon.copies[i], before[i])
        else:
            _check(s, dev, muon, i, 0.01, 0.1, momentum=0.9)


def test_steps_from_nothing():
    """From zero momenta, several steps with the states that the steps leave; a scale of the
    gradients on the device."""
    s = _state(CONV, torch.float32, torch.float32, 3)
    s["m"] = [torch.zeros_like(m) for m in s["m"]]
    muon, dev = _muon(s, False, 0.0, scales=[0.3] * len(CONV))
    gs = torch.tensor([0.25], device=DEV)
    for t in range(4):
        now = {k: [x.cpu() for x in dev[k]] for k in dev}
        muon.step(dev["g"], lr=0.05, grad_scale=gs)
        torch.cuda.synchronize()
        for i in range(len(CONV)):
            _check(now, dev, muon, i, 0.0, 0.05, gs=0.25)


def test_zero_gradients_decay_alone():
    s = _state(CONV, torch.float32, torch.float32, 4)
    s["m"] = [torch.zeros_like(m) for m in s["m"]]
    s["g"] = [torch.zeros_like(m) for m in s["m"]]
    muon, dev = _muon(s, False, 0.5)
    muon.step(dev["g"], lr=0.1)
    for p, was in zip(dev["p"], s["p"]):
        assert ((p.cpu().double() - was.double() * 0.95).abs() <= 4 * U * was.double().abs()).all()


def test_no_gradients_at_all():
    s = _state(CONV, torch.float32, torch.float32, 4)
    muon, dev = _muon(s, True, 0.5)
    before = [c.clone() for c in muon.copies]
    muon.step([None] * len(CONV), lr=0.1)
    torch.cuda.synchronize()
    for i in range(len(CONV)):
        assert torch.equal(dev["p"][i].cpu(), s["p"][i]) and torch.equal(dev["m"][i].cpu(), s["m"][i])
        assert torch.equal(muon.copies[i], before[i])


def test_default_momentum_and_none():
    """Momenta of its own; with no parameters nothing happens."""
    p = [torch.randn(8, 4, 3, 3, device=DEV), torch.randn(6, 6, device=DEV, dtype=torch.bfloat16)]
    muon = tr.Muon(p)
    assert [m.shape for m in muon.m] == [x.shape for x in p] and muon.products == "f32"
    muon.step([torch.randn_like(x) for x in p], lr=0.1)
    assert all(bool(torch.isfinite(x).all()) for x in p + muon.m)
    none = tr.Muon([])
    none.step([], lr=0.1)


@pytest.mark.parametrize("products", ["f32", "f16"])
def test_streams_and_graphs(products):
    """The same bits again and on a side stream; two graphs on one plan, replayed with eager work
    between."""
    shape = (3, 200, 333)
    g = torch.Generator().manual_seed(5)
    xs = [torch.randn(shape, generator=g).to(DEV) for _ in range(5)]
    op, other = (tr.Orthogonalize(shape, torch.float32, products) for _ in range(2))
    want = [other(x) for x in xs]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        again = [op(x) for x in xs]
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, again))
    x, graphs, outs = xs[0].clone(), [], [torch.empty(shape, device=DEV) for _ in range(2)]
    torch.cuda.synchronize()
    for out in outs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            op(x, out=out)
        graphs.append(graph)
    for i in (1, 2, 3, 4):
        x.copy_(xs[i])
        for graph, out in zip(graphs, outs):
            out.fill_(9)
            graph.replay()
            assert torch.equal(out, want[i])
            assert torch.equal(op(xs[i - 1]), want[i - 1])


def test_step_in_a_graph():
    """Replays go on from the state that the ones before left, as eager steps do."""
    shapes = [(40, 70), (130, 60), (5, 9)]
    s = _state(shapes, torch.float32, torch.bfloat16, 6)
    muon, dev = _muon(s, True, 0.01)
    eager, dev2 = _muon(s, True, 0.01)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        muon.step(dev["g"], lr=0.03)
    for _ in range(4):
        graph.replay()
        eager.step(dev2["g"], lr=0.03)
        torch.cuda.synchronize()
        for k in ("p", "m"):
            assert all(torch.equal(a, b) for a, b in zip(dev[k], dev2[k]))
        assert all(torch.equal(a, b) for a, b in zip(muon.copies, eager.copies))


def test_refusals():
    x = torch.zeros(4, 8, 16, device=DEV)
    op = tr.Orthogonalize(x.shape, torch.float32)
    for call in (lambda: op(x.cpu()), lambda: op(x[:2]), lambda: op(x.bfloat16()),
                 lambda: op(x.transpose(1, 2)), lambda: op(x, out=torch.empty(8, 16, device=DEV)),
                 lambda: tr.Orthogonalize((5,), torch.float32),
                 lambda: tr.Orthogonalize(x.shape, torch.float16),
                 lambda: tr.Orthogonalize(x.shape, torch.float32, "f8"),
                 lambda: tr.Orthogonalize(x.shape, torch.float32, steps=0),
                 lambda: tr.Orthogonalize(x.shape, torch.float32, steps=3, coefficients=[(1, 2, 3)] * 2),
                 lambda: tr.Orthogonalize(x.shape, torch.float32, coefficients=(1, 2)),
                 lambda: tr.Muon([x[0, 0]]), lambda: tr.Muon([x.cpu()]), lambda: tr.Muon([x.half()]),
                 lambda: tr.Muon([x], weight_decay=[0.1, 0.2]), lambda: tr.Muon([x], m=[x[0]]),
                 lambda: tr.Muon([x], copies=[x]), lambda: tr.Muon([torch.empty(0, 4, device=DEV)])):
        with pytest.raises((ValueError, TypeError)):
            call()
    muon = tr.Muon([x])
    for call in (lambda: op(x, out=x), lambda: tr.Muon([x, x]), lambda: tr.Muon([x], m=[x]),
                 lambda: tr.Orthogonalize(x.shape, torch.float32, coefficients=(3000.0, 0.0, 0.0)),
                 lambda: tr.Orthogonalize(x.shape, torch.float32, coefficients=(math.nan, 0.0, 0.0)),
                 lambda: tr.Orthogonalize(x.shape, torch.float32, eps=0.0),
                 lambda: muon.step([x], lr=0.1), lambda: muon.step([muon.m[0]], lr=0.1),
                 lambda: muon.step([x.clone()], lr=-1.0),
                 lambda: muon.step([x.clone()], lr=0.1, momentum=1.0)):
        with pytest.raises(tr.h2.Huge2Error):
            call()
    for grads in ([], [x, x], [x[0]], [x.bfloat16()]):
        with pytest.raises(ValueError):
            muon.step(grads, lr=0.1)
    muon.close()
    with pytest.raises(ValueError):
        muon.step([x.clone()], lr=0.1)


def test_errors_of_the_device(monkeypatch):
    x = torch.zeros(8, 16, device=DEV)
    op, muon = tr.Orthogonalize(x.shape, torch.float32), tr.Muon([x])
    out = torch.full_like(x, 7)
    monkeypatch.setenv("HUGE2_FAULT", "launch")
    with pytest.raises(tr.h2.Huge2Error):
        op(x, out=out)
    with pytest.raises(tr.h2.Huge2Error):
        muon.step([torch.ones_like(x)], lr=0.1)
    monkeypatch.setenv("HUGE2_FAULT", "alloc")
    with pytest.raises(tr.h2.Huge2Error):
        tr.Orthogonalize(x.shape, torch.float32)
    with pytest.raises(tr.h2.Huge2Error):
        tr.Muon([x])
    assert bool((out == 7).all()) and float(x.abs().max()) == 0
