"""Layer norm over channels and its gradients on the GPU, against the definitions in 64 bits on
the CPU.

Tolerances, from the arithmetic: u = 2^-24.  A sum of values is off by less than DEPTH * u of the
sum of their magnitudes, DEPTH the longest chain of additions: at most 96 in a thread at these
sizes (long rows and general tiles; 32 where values are held) and some 32 behind it.  The mean is
then off by DEPTH * u * max|x|, a normalised value by that times rstd and by DEPTH * u of itself
(half of the variance's share), the result by that times |gamma| (every activation's slope is at
most 1.1), and a bf16 result by half a unit in its last place.
"""
import pytest
import torch

from paper_1907_11210_amd import train as tr

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U, DEPTH = 2.0 ** -24, 128
ACTS = (None, "relu", "tanh", "silu")

# (pixels, c) of lists, (n, c, h, w) of maps
ROWS = [(1, 1), (3, 2), (5, 3), (7, 7), (6, 8), (4, 9), (9, 16), (33, 100), (300, 64), (17, 333),
        (6, 1000), (3, 2048), (3, 2049), (2, 4104), (5, 8199), (2, 16400), (3, 32771), (2, 70001),
        (4, 40000), (70001, 24)]
MAPS = [(1, 1, 1, 2), (2, 3, 1, 5), (3, 5, 2, 3), (70, 16, 2, 2), (2, 24, 3, 3), (2, 200, 9, 11),
        (1, 512, 8, 8), (5, 33, 41, 7), (4, 128, 32, 32), (1, 64, 67, 131), (300, 16, 24, 24),
        (1, 1040, 3, 5), (2, 2056, 5, 7), (1, 4104, 4, 4), (3, 8200, 2, 3), (2, 9001, 4, 4),
        (2, 17000, 1, 3), (2, 40, 1, 1)]


def _shape(shape, layout):
    if len(shape) == 2:
        return shape
    n, c, h, w = shape
    return (n, c, h, w) if layout == "NCHW" else (n, h, w, c)


def _lay(t, shape, layout):
    """[pixels, c] in the layout."""
    if layout == "NCHW":
        n, c, h, w = shape
        return t.reshape(n, h * w, c).transpose(1, 2).reshape(n, c, h, w).contiguous()
    return t.reshape(_shape(shape, layout)).contiguous()


def _unlay(t, layout):
    if layout == "NCHW":
        t = t.permute(0, 2, 3, 1)
    return t.reshape(-1, t.shape[-1])


def _inputs(shape, dtype, seed, mean=0.5, std=1.0):
    pixels, c = shape if len(shape) == 2 else (shape[0] * shape[2] * shape[3], shape[1])
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(pixels, c, generator=g) * std + mean + torch.randn(c, generator=g)).to(dtype)
    dy = torch.randn(pixels, c, generator=g).to(dtype)
    return x, dy, 1 + 0.5 * torch.randn(c, generator=g), 0.5 * torch.randn(c, generator=g)


def _act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0)
    if act == "tanh":
        return torch.tanh(z)
    return z * torch.sigmoid(z) if act == "silu" else z


def _act_slope(z, act):
    if act == "tanh":
        return 1 - torch.tanh(z) ** 2
    if act == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def _reference(x, gamma, beta, act, eps=1e-5):
    x = x.double()
    mean = x.mean(1)
    rstd = 1 / torch.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    z = (x - mean[:, None]) * rstd[:, None] * gamma.double() + beta.double()
    return _act(z, act), mean, rstd


def _within(got, ref, tol, dtype):
    """A result of `dtype` of a value that is off by at most tol: between the roundings of
    the interval's ends (rounding keeps order); fp32: its own rounding beside tol."""
    if dtype == torch.bfloat16:
        lo, hi = (v.to(dtype).double() for v in (ref - tol, ref + tol))
        return (got >= lo) & (got <= hi)
    return (got - ref).abs() <= tol + ref.abs() * U


def _guarded(shape, dtype):
    """A tensor between two runs of other values, and the whole."""
    n = 1
    for s in shape:
        n *= s
    whole = torch.full((n + 128,), 7, dtype=dtype, device=DEV)
    return whole[64:64 + n].view(shape), whole


def _kept(whole):
    return bool((whole[:64] == 7).all() and (whole[-64:] == 7).all())


def _run(shape, layout, dtype, act, seed=0, **kw):
    x, dy, gamma, beta = _inputs(shape, dtype, seed, **kw)
    xs = _lay(x, shape, layout).to(DEV)
    ln = tr.LayerNorm(xs.shape, dtype, layout, act)
    stats, around = _guarded(ln.stats_shape, torch.float32)
    out, whole = _guarded(xs.shape, dtype)
    y = ln(xs, gamma.to(DEV), beta.to(DEV), out=out, stats=stats)
    torch.cuda.synchronize()
    assert y is out and _kept(whole) and _kept(around)
    return ln, x, dy, gamma, beta, xs, y, stats


CASES = [(s, "NHWC") for s in ROWS + MAPS] + [(s, "NCHW") for s in MAPS]
IDS = ["x".join(map(str, s)) + "-" + l for s, l in CASES]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape,layout", CASES, ids=IDS)
def test_forward(shape, layout, dtype):
    for act in ACTS:
        print("layer norm", shape, layout, dtype, act, flush=True)
        ln, x, _, gamma, beta, xs, y, stats = _run(shape, layout, dtype, act)
        ref, mean, rstd = _reference(x, gamma, beta, act)
        xmax = x.double().abs().max()
        by = rstd[:, None]
        xh = (x.double().abs() + xmax) * by
        tol = U * (DEPTH * (xmax * by + xh) + 8) * gamma.double().abs() * 1.1 \
            + U * 8 * beta.double().abs()
        got = _unlay(y.cpu(), layout).double()
        assert _within(got, ref, tol, dtype).all(), float(((got - ref).abs() / tol).max())
        st = stats.cpu().double()
        assert ((st[:, 0] - mean).abs() <= DEPTH * U * xmax).all()
        assert ((st[:, 1] - rstd).abs() <= DEPTH * U * (1 + xmax * rstd) * rstd).all()
        # without statistics, the same bits
        assert torch.equal(ln(xs, gamma.to(DEV), beta.to(DEV)), y)


def _grad_reference(x, dy, gamma, beta, stats, act):
    """From the statistics that the kernel is given; a ReLU's mask is that of z rounded as the
    forward rounds it (to 24 bits after each of its four operations)."""
    mean, rstd = stats[:, :1], stats[:, 1:]
    z32 = ((x.float() - mean) * rstd) * gamma + beta
    mean, rstd, ga = mean.double(), rstd.double(), gamma.double()
    xh = (x.double() - mean) * rstd
    dz = dy.double() * _act_slope(xh * ga + beta.double(), act)
    if act == "relu":
        dz = torch.where(z32 > 0, dz, 0)
    t = dz * ga
    dx = rstd * (t - t.mean(1, keepdim=True) - xh * (t * xh).mean(1, keepdim=True))
    # magnitudes of what is added up, for the tolerances
    mag = rstd * (t.abs() + t.abs().mean(1, keepdim=True)
                  + xh.abs() * (t * xh).abs().mean(1, keepdim=True))
    near = (x.double().abs() + mean.abs()) * rstd  # what xh's own rounding is a share of
    return dx, (dz * xh).sum(0), dz.sum(0), mag, dz, xh, near


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape,layout", CASES, ids=IDS)
def test_gradients(shape, layout, dtype):
    for act in ACTS:
        print("layer norm grad", shape, layout, dtype, act, flush=True)
        ln, x, dy, gamma, beta, xs, _, stats = _run(shape, layout, dtype, act, seed=1)
        out, whole = _guarded(xs.shape, dtype)
        dx, dgamma, dbeta = ln.grad(xs, _lay(dy, shape, layout).to(DEV), stats, gamma.to(DEV),
                                    beta.to(DEV), out=out)
        torch.cuda.synchronize()
        assert dx is out and _kept(whole)
        rx, rg, rb, mag, dz, xh, near = _grad_reference(x, dy, gamma, beta, stats.cpu(), act)
        # xh is off by 2u of `near`, z by that times gamma, and the slopes' own slopes are
        # below 1: a share of `slope` in dz
        slope = 4 * U * (2 + (near * (1 + gamma.double().abs())).max())
        tol = mag * (DEPTH * U + slope) * 2
        if act in ("tanh", "silu"):
            tol = tol + dy.double().abs().max() * slope * gamma.double().abs().max() * 4 * \
                stats.cpu().double()[:, 1].max() * (1 + xh.abs().max()) ** 2
        got = _unlay(dx.cpu(), layout).double()
        assert _within(got, rx, tol, dtype).all(), float(((got - rx).abs() / tol).max())
        ady = dy.double().abs() if act in ("tanh", "silu") else dz.abs()
        tol_b = (DEPTH * U * dz.abs() + slope * ady).sum(0)
        tol_g = (DEPTH * U * (dz * xh).abs() + slope * ady * (1 + xh.abs())).sum(0)
        assert ((dbeta.cpu().double() - rb).abs() <= tol_b).all()
        assert ((dgamma.cpu().double() - rg).abs() <= tol_g).all()


FORMS = [((19, 24), "NHWC"), ((5, 2056), "NHWC"), ((2, 40001), "NHWC"), ((2, 24, 5, 7), "NCHW"),
         ((3, 9000, 2, 4), "NCHW"), ((2, 700, 1, 3), "NCHW")]
FORM_IDS = ["rows", "wide", "long", "planes", "again", "narrow"]


@pytest.mark.parametrize("shape,layout", FORMS, ids=FORM_IDS)
@pytest.mark.parametrize("act", ["tanh", "silu", None])
def test_gradients_against_differences(act, shape, layout):
    """Central differences of the 64-bit definition along random directions."""
    ln, x, dy, gamma, beta, xs, _, stats = _run(shape, layout, torch.float32, act, seed=2)
    dx, dgamma, dbeta = ln.grad(xs, _lay(dy, shape, layout).to(DEV), stats, gamma.to(DEV),
                                beta.to(DEV))
    g = torch.Generator().manual_seed(3)
    x, gamma, beta = x.double(), gamma.double(), beta.double()
    for what, grad in (("x", _unlay(dx, layout)), ("gamma", dgamma), ("beta", dbeta)):
        base = {"x": x, "gamma": gamma, "beta": beta}
        v = torch.randn(base[what].shape, generator=g, dtype=torch.float64)
        h = 1e-4

        def loss(s):
            a = dict(base, **{what: base[what] + s * v})
            return (_reference(a["x"], a["gamma"], a["beta"], act)[0] * dy.double()).sum()

        got = float((grad.cpu().double() * v).sum())
        want = float((loss(h) - loss(-h)) / (2 * h))
        # differences: h^2 times third derivatives (some 10 a value, as their sum's root); sums of
        # values of size 1 and some with 24 bits
        assert abs(got - want) <= 1e-4 * (1 + abs(want)) + 1e-5 * x.numel() ** 0.5, (what, got, want)


@pytest.mark.parametrize("shape,layout", FORMS, ids=FORM_IDS)
def test_values_far_from_zero(shape, layout):
    """A mean 1000 standard deviations from zero: sums of squares around zero would lose all."""
    ln, x, _, gamma, beta, xs, y, stats = _run(shape, layout, torch.float32, None, mean=1e3)
    ref, mean, rstd = _reference(x, gamma, beta, None)
    tol = U * DEPTH * 3 * x.double().abs().max() * rstd[:, None] * (1 + gamma.double().abs())
    assert ((_unlay(y.cpu(), layout).double() - ref).abs() <= tol).all()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("shape,layout", FORMS, ids=FORM_IDS)
def test_not_finite_stays_in_its_pixel(shape, layout, value):
    x, dy, gamma, beta = _inputs(shape, torch.float32, 5)
    x[1, x.shape[1] - 2] = value
    xs = _lay(x, shape, layout).to(DEV)
    ln = tr.LayerNorm(xs.shape, torch.float32, layout, "relu")
    stats = ln.new_stats()
    y = _unlay(ln(xs, gamma.to(DEV), beta.to(DEV), stats=stats).cpu(), layout)
    bad = torch.zeros(x.shape[0], dtype=torch.bool)
    bad[1] = True
    assert torch.isnan(y[bad]).all() and torch.isfinite(y[~bad]).all()
    dx, _, _ = ln.grad(xs, _lay(dy, shape, layout).to(DEV), stats, gamma.to(DEV), beta.to(DEV))
    dx = _unlay(dx.cpu(), layout)
    assert torch.isnan(dx[bad]).all() and torch.isfinite(dx[~bad]).all()


@pytest.mark.parametrize("shape,layout", FORMS, ids=FORM_IDS)
def test_constant_pixels_and_absent_parameters(shape, layout):
    """No variance: y is zero and dx is finite; no gamma, no beta: ones, zeros."""
    x, dy, _, _ = _inputs(shape, torch.float32, 6)
    pixels, c = x.shape
    xs, dys = _lay(x, shape, layout).to(DEV), _lay(dy, shape, layout).to(DEV)
    ln = tr.LayerNorm(xs.shape, torch.float32, layout)
    stats = ln.new_stats()
    same = torch.full_like(xs, 0.25)  # (whose sum is exact)
    assert float(ln(same, stats=stats).abs().max()) <= 2 * U * 0.25 * 1e-5 ** -0.5
    stats.copy_(torch.tensor([0.25, 1e-5 ** -0.5], device=DEV).expand_as(stats))
    dx, dgamma, dbeta = ln.grad(same, same, stats)
    assert torch.isfinite(dx).all() and float(dgamma.abs().max()) == 0
    assert torch.equal(dbeta.cpu(), torch.full((c,), 0.25 * pixels))
    ones, zeros = torch.ones(c, device=DEV), torch.zeros(c, device=DEV)
    assert torch.equal(ln(xs), ln(xs, ones, zeros, stats=stats))
    for a, b in zip(ln.grad(xs, dys, stats), ln.grad(xs, dys, stats, ones, zeros)):
        assert torch.equal(a, b)
    # without the parameters' gradients
    dx = torch.empty_like(xs)
    tr.huge2_layer_norm_grad_execute(ln._open(), xs.data_ptr(), dys.data_ptr(), stats.data_ptr(), 0,
                                     0, dx.data_ptr(), stream=torch.cuda.current_stream().cuda_stream)
    assert torch.equal(dx, ln.grad(xs, dys, stats)[0])
    dgamma = torch.empty(c, device=DEV)
    tr.huge2_layer_norm_grad_execute(ln._open(), xs.data_ptr(), dys.data_ptr(), stats.data_ptr(), 0,
                                     0, dx.data_ptr(), dgamma.data_ptr(),
                                     stream=torch.cuda.current_stream().cuda_stream)
    assert torch.equal(dgamma, ln.grad(xs, dys, stats)[1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape,layout", [((40000, 1000), "NHWC"), ((40003, 1003), "NHWC"),
                                          ((16, 32, 256, 264), "NCHW"), ((16, 32, 257, 263), "NCHW")],
                         ids=["rows", "odd rows", "planes", "odd planes"])
def test_results_past_the_caches(shape, layout, dtype):
    """Results of 64 MiB and more, and many tiles: against the same pixels in parts."""
    x, dy, gamma, beta = _inputs(shape, dtype, 11)
    xs, dys = _lay(x, shape, layout).to(DEV), _lay(dy, shape, layout).to(DEV)
    assert xs.numel() * xs.element_size() >= 64 << 20
    ga, be = gamma.to(DEV), beta.to(DEV)
    ln = tr.LayerNorm(xs.shape, dtype, layout, "relu")
    stats = ln.new_stats()
    y = ln(xs, ga, be, stats=stats)
    dx, dgamma, dbeta = ln.grad(xs, dys, stats, ga, be)
    k = shape[0] // 8 if len(shape) == 2 else 1
    part = tr.LayerNorm((k, *xs.shape[1:]), dtype, layout, "relu")
    per = stats.shape[0] // shape[0] * k
    for i in (0, 3, 7):
        st = part.new_stats()
        assert torch.equal(part(xs[i * k:(i + 1) * k], ga, be, stats=st), y[i * k:(i + 1) * k])
        assert torch.equal(st, stats[i * per:(i + 1) * per])
        assert torch.equal(part.grad(xs[i * k:(i + 1) * k], dys[i * k:(i + 1) * k], st, ga, be)[0],
                           dx[i * k:(i + 1) * k])
    _, rg, rb, _, dz, xh, _ = _grad_reference(x, dy, gamma, beta, stats.cpu(), "relu")
    # threads add up to some 200 pixels, then lanes and workgroups
    assert ((dbeta.cpu().double() - rb).abs() <= 400 * U * dz.abs().sum(0)).all()
    assert ((dgamma.cpu().double() - rg).abs() <= 400 * U * (dz * xh).abs().sum(0)).all()


@pytest.mark.parametrize("shape,layout", FORMS, ids=FORM_IDS)
def test_streams_and_graphs(shape, layout):
    """On a side stream the same bits; two captured gradients on one plan, replayed with eager
    work between."""
    ln, x, dy, gamma, beta, xs, y, stats = _run(shape, layout, torch.bfloat16, "silu")
    dys, ga, be = _lay(dy, shape, layout).to(DEV), gamma.to(DEV), beta.to(DEV)
    first = ln.grad(xs, dys, stats, ga, be)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        st2 = ln.new_stats()
        y2 = ln(xs, ga, be, stats=st2)
        again = ln.grad(xs, dys, st2, ga, be)
    s.synchronize()
    assert torch.equal(y, y2) and torch.equal(stats, st2)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    out, st = torch.empty_like(xs), ln.new_stats()
    graphs, grads = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ln(xs, ga, be, out=out, stats=st)
            grads.append(ln.grad(xs, dys, st, ga, be))
        graphs.append(graph)
    for seed in (7, 8, 9):
        x2, dy2, _, _ = _inputs(shape, torch.bfloat16, seed)
        xs.copy_(_lay(x2, shape, layout))
        dys.copy_(_lay(dy2, shape, layout))
        for graph, g in zip(graphs, grads):
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in (out, *g)]
            st2 = ln.new_stats()
            want = [ln(xs, ga, be, stats=st2), *ln.grad(xs, dys, st2, ga, be)]
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_other_shapes_of_rows():
    """Channels are the last axis, whatever axes come before."""
    x = torch.randn(2, 3, 4, 5, 24, device=DEV)
    flat = tr.LayerNorm((120, 24), torch.float32)
    for shape in ((2, 3, 4, 5, 24), (6, 20, 24), (120, 24)):
        ln = tr.LayerNorm(shape, torch.float32)
        assert torch.equal(ln(x.view(shape)).view(120, 24), flat(x.view(120, 24)))
    one = tr.LayerNorm((24,), torch.float32)
    assert torch.equal(one(x[0, 0, 0, 0]), flat(x.view(120, 24))[0])


def test_refusals():
    x = torch.zeros(2, 4, 4, 16, device=DEV)
    ln = tr.LayerNorm(x.shape, torch.float32)
    stats = ln.new_stats()
    for call in (lambda: ln(x.cpu()), lambda: ln(x.permute(0, 3, 1, 2)), lambda: ln(x[:1]),
                 lambda: ln(x.bfloat16()), lambda: ln(x, torch.ones(15, device=DEV)),
                 lambda: ln(x, out=torch.empty(2, 4, 4, 8, device=DEV)),
                 lambda: ln(x, stats=torch.empty(2, 4, device=DEV)),
                 lambda: ln.grad(x, x.bfloat16(), stats),
                 lambda: tr.LayerNorm((2, 4, 4), torch.float32, "NCHW"),
                 lambda: tr.LayerNorm((), torch.float32),
                 lambda: tr.LayerNorm((2 ** 16, 2 ** 16, 4), torch.float32),
                 lambda: tr.LayerNorm(x.shape, torch.float32, activation="gelu"),
                 lambda: tr.LayerNorm(x.shape, torch.float16)):
        with pytest.raises((ValueError, TypeError)):
            call()
    for call in (lambda: ln(x, out=x), lambda: ln.grad(x, x, stats, out=x),
                 lambda: tr.LayerNorm((0, 16), torch.float32)):
        with pytest.raises(tr.h2.Huge2Error):
            call()
    assert float(ln(x).abs().max()) == 0
    ln.close()
    with pytest.raises(ValueError):
        ln(x)


def test_errors_of_the_device(monkeypatch):
    x = torch.zeros(2, 4, 4, 16, device=DEV)
    ln = tr.LayerNorm(x.shape, torch.float32)
    out = torch.full_like(x, 7)
    monkeypatch.setenv("HUGE2_FAULT", "launch")
    with pytest.raises(tr.h2.Huge2Error):
        ln(x, out=out)
    monkeypatch.setenv("HUGE2_FAULT", "alloc")
    with pytest.raises(tr.h2.Huge2Error):
        tr.LayerNorm(x.shape, torch.float32)
    assert bool((out == 7).all())
