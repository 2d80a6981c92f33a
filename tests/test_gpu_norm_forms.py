"""Group norm by each of its forms: what a form has to keep that no other shows.  The
forms are named, so that a case does not move to another one unnoticed.

Tolerances as in test_gpu_norm, from whose formulas these are.
"""
import pytest
import torch

from paper_1907_11210_amd import train as tr
from test_gpu_norm import DEPTH, DEV, U, _inputs, _lay, _reference, _unlay

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16

# layout, type, (n, c, h, w, groups), what the names of the forward's and gradient's kernels
# begin with
FORMS = [
    ("NHWC", F32, (3, 24, 6, 6, 6), "norm_slab_nhwc", "norm_slab_grad_nhwc"),
    ("NCHW", F32, (3, 24, 6, 6, 6), "norm_slab_nchw", "norm_slab_nchw"),
    ("NHWC", BF16, (3, 24, 6, 6, 6), "norm_slab_nhwc", "norm_slab_grad_nhwc"),  # groups share vectors
    ("NHWC", F32, (2, 64, 96, 96, 4), "norm_run_nhwc", "norm_run_grad_nhwc"),   # 36 runs
    ("NHWC", BF16, (2, 24, 75, 80, 6), "norm_run_nhwc", "norm_run_grad_nhwc"),  # groups share vectors
    ("NHWC", F32, (2, 16400, 12, 12, 1), "norm_sums_nhwc", "norm_sums_nhwc"),   # 3 runs
    ("NCHW", F32, (2, 64, 96, 96, 4), "norm_sums_nchw", "norm_sums_nchw"),      # 144 entries to join
    ("NCHW", BF16, (2, 64, 96, 96, 4), "norm_sums_nchw", "norm_sums_nchw"),
    ("NCHW", F32, (2, 1100, 64, 64, 1), "norm_sums_nchw", "norm_sums_nchw"),    # too many: a merge
]


def _ids(form):
    layout, dtype, shape = form[:3]
    return "%s-%s-%s" % (layout, "f32" if dtype == F32 else "bf16", "x".join(map(str, shape)))


def _norm(form, act=None):
    """The form's object, whose kernels are what the form says."""
    layout, dtype, (n, c, h, w, groups), forward, grad = form
    gn = tr.GroupNorm((n, h, w, c) if layout == "NHWC" else (n, c, h, w), groups, dtype, layout, act)
    assert [k.startswith(name) for k, name in zip(gn.kernels, (forward, grad))] == [True, True], \
        gn.kernels
    print("norm", _ids(form), act, gn.kernels, flush=True)
    return gn


def _group(shape, group):
    n, c, _, _, groups = shape
    of = torch.zeros(n, c, dtype=torch.bool)
    per = c // groups
    of[n - 1, group * per:(group + 1) * per] = True
    return of


@pytest.mark.parametrize("form", FORMS, ids=_ids)
def test_not_finite_stays_in_its_group(form):
    """A NaN or an infinity anywhere makes its group NaN, and nothing else: a variance that is
    not a number must not become none."""
    layout, dtype, shape = form[:3]
    n, c, h, w, groups = shape
    gn = _norm(form, "relu")
    group = groups // 2
    bad = _group(shape, group)
    x, dy, gamma, beta = _inputs(shape, dtype, 5)
    ga, be, dys = gamma.to(DEV), beta.to(DEV), _lay(dy, layout).to(DEV)
    last = (group + 1) * c // groups - 1
    for value in (float("nan"), float("inf"), -float("inf")):
        for ch, row, col in ((group * c // groups, 0, 0), (last, h // 2, w // 3), (last, h - 1, w - 1)):
            xb = x.clone()
            xb[n - 1, ch, row, col] = value
            xs = _lay(xb, layout).to(DEV)
            stats = gn.new_stats()
            y = _unlay(gn(xs, ga, be, stats=stats).cpu(), layout)
            case = (value, ch, row, col)
            assert torch.isnan(y[bad]).all() and torch.isfinite(y[~bad]).all(), case
            st = stats.cpu()
            assert torch.isnan(st[n - 1, group, 1]) and not torch.isfinite(st[n - 1, group, 0]), case
            st[n - 1, group] = 0
            assert torch.isfinite(st).all(), case
            dx = _unlay(gn.grad(xs, dys, stats, ga, be)[0].cpu(), layout)
            assert torch.isnan(dx[bad]).all() and torch.isfinite(dx[~bad]).all(), case


@pytest.mark.parametrize("form", FORMS, ids=_ids)
def test_squares_that_overflow(form):
    """Values of 1e20, whose squares 32 bits do not hold: the variance is infinite, its root's
    reciprocal 0, and z is beta, in every form."""
    layout, dtype, shape = form[:3]
    n, c, h, w, groups = shape
    gn = _norm(form, "relu")
    bad = _group(shape, 0)
    x, _, gamma, beta = _inputs(shape, dtype, 6)
    for row, col in ((0, 0), (h - 1, w - 1)):
        xb = x.clone()
        xb[n - 1, 0, row, col] = 1e20
        stats = gn.new_stats()
        y = _unlay(gn(_lay(xb, layout).to(DEV), gamma.to(DEV), beta.to(DEV), stats=stats).cpu(), layout)
        assert float(stats[n - 1, 0, 1]) == 0 and torch.isfinite(stats).all()
        want = torch.relu(beta).to(dtype).expand(n, c)[bad][:, None, None]
        assert torch.equal(y[bad], want.expand_as(y[bad]))


# the longest runs: 4096 values of fp32 and 8192 of bf16 in NCHW, whole maps in NHWC
LONG = [
    ("NCHW", F32, (64, 128, 64, 64, 4), "norm_sums_nchw", "norm_sums_nchw"),
    ("NCHW", BF16, (64, 128, 64, 128, 2), "norm_sums_nchw", "norm_sums_nchw"),
    ("NHWC", F32, (32, 16400, 12, 12, 1), "norm_sums_nhwc", "norm_sums_nhwc"),
    ("NHWC", F32, (64, 128, 64, 64, 4), "norm_run_nhwc", "norm_run_grad_nhwc"),
    ("NCHW", F32, (16, 1000, 64, 64, 1), "norm_sums_nchw", "norm_sums_nchw"),  # 1000 entries
    ("NHWC", BF16, (1, 128, 512, 512, 32), "norm_run_nhwc", "norm_run_grad_nhwc"),  # 128 runs
    ("NHWC", F32, (1, 2, 2048, 2048, 1), "norm_run_nhwc", "norm_run_grad_nhwc"),  # 512 runs
]


def _statistics(form, x):
    """The kernels' and the definition's, on the GPU."""
    layout, dtype, shape = form[:3]
    gn = _norm(form)
    stats = gn.new_stats()
    gn(_lay(x, layout), stats=stats)
    ones, zeros = torch.ones(shape[1], device=DEV), torch.zeros(shape[1], device=DEV)
    _, mean, rstd = _reference(x, ones, zeros, shape[4], None, 1e-5)
    st = stats.double()
    return (st[..., 0] - mean).abs(), (st[..., 1] / rstd - 1).abs()


def _normal(shape, dtype, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    return torch.randn(shape[:4], generator=g, device=DEV).to(dtype)


@pytest.mark.parametrize("form", LONG + FORMS, ids=_ids)
def test_an_outlier_where_runs_begin(form):
    """The first pixel 1e4 standard deviations out: what comes first is no measure of the rest,
    so the squares must not be taken around it.  They are off by DEPTH u of themselves."""
    shape = form[2]
    x = _normal(shape, form[1], 4)
    x[:, :, 0, 0] += 1e4
    mean, rstd = _statistics(form, x)
    assert (rstd <= DEPTH * U).all(), float(rstd.max()) / U
    assert (mean <= DEPTH * U * 1e4).all()


@pytest.mark.parametrize("form", LONG + FORMS, ids=_ids)
def test_a_first_run_far_from_the_others(form):
    """The same where a whole channel, or the first rows of each map, are 1e4 out."""
    shape = form[2]
    for where in ("channel", "rows"):
        x = _normal(shape, form[1], 5)
        if where == "channel":
            x[:, ::shape[1] // shape[4]] += 1e4
        else:
            x[:, :, :max(1, shape[2] // 64)] += 1e4
        mean, rstd = _statistics(form, x)
        assert (rstd <= DEPTH * U).all(), (where, float(rstd.max()) / U)
        assert (mean <= DEPTH * U * 1e4).all(), where


@pytest.mark.parametrize("layout", ["NHWC", "NCHW"])
def test_a_map_of_almost_2_to_the_31(layout):
    """Every pixel of the largest map is read and written: one channel, bf16.  Sums have chains
    of up to 2^16 additions (the runs of a channel, 16 side by side)."""
    hw, part, chain = 2 ** 31 - 2, 1 << 26, 1 << 16
    shape = (1, hw, 1, 1) if layout == "NHWC" else (1, 1, hw, 1)
    gn = tr.GroupNorm(shape, 1, BF16, layout)
    print("norm", shape, layout, gn.kernels, flush=True)
    g = torch.Generator(DEV).manual_seed(7)
    x, dy, y = (torch.empty(hw, dtype=BF16, device=DEV) for _ in range(3))
    for first in range(0, hw, part):
        for t in (x, dy):
            t[first:first + part].normal_(0.5, 1.0, generator=g)
    stats = gn.new_stats()
    y.fill_(float("nan"))
    gn(x.view(shape), out=y.view(shape), stats=stats)
    parts = [slice(first, min(hw, first + part)) for first in range(0, hw, part)]
    mean = sum(float(x[p].double().sum()) for p in parts) / hw
    var = sum(float((x[p].double() - mean).square().sum()) for p in parts) / hw
    st = stats.double().flatten().tolist()
    assert abs(st[0] - mean) <= chain * U * 2 and abs(st[1] * (var + 1e-5) ** 0.5 - 1) <= chain * U
    # from the kernels' statistics: three roundings and bf16's, whose unit is 2^-8
    sums = torch.zeros(4, dtype=torch.float64, device=DEV)
    for p in parts:
        xh = (x[p].double() - st[0]) * st[1]
        assert ((y[p].double() - xh).abs() <= xh.abs() * (2.0 ** -8 + 4 * U) + 1e-6).all(), p
        d = dy[p].double()
        sums += torch.stack((d.sum(), (d * xh).sum(), d.abs().sum(), (d * xh).abs().sum()))
    y.fill_(float("nan"))
    _, dgamma, dbeta = gn.grad(x.view(shape), dy.view(shape), stats, out=y.view(shape))
    db, dg, db_mag, dg_mag = sums.tolist()
    assert abs(float(dbeta) - db) <= chain * U * db_mag
    assert abs(float(dgamma) - dg) <= chain * U * dg_mag
    # the two means are off by chain u of their magnitudes' means
    off = chain * U * (db_mag / hw)
    off_xh = chain * U * (dg_mag / hw)
    for p in parts:
        xh = (x[p].double() - st[0]) * st[1]
        dx = st[1] * (dy[p].double() - db / hw - xh * (dg / hw))
        tol = st[1] * (off + xh.abs() * off_xh) + dx.abs() * 2.0 ** -8 + 8 * U * (1 + xh.abs())
        assert ((y[p].double() - dx).abs() <= tol * (1 + 2.0 ** -7)).all(), p


@pytest.mark.parametrize("layout", ["NHWC", "NCHW"])
@pytest.mark.parametrize("act", ["tanh", "silu"])
def test_fp32_activations(act, layout):
    """All x are zeros, so that z is beta, and one pixel, so that dbeta is dy's product with the
    slope: fp32 results are off by the activation's own roundings.  The device's tanh and
    exponential are within 2 and 1 units in the last place, 4u and 2u at most of the value; SiLU
    and its slope add a sum and a quotient, u each, and products of them."""
    z = torch.cat((torch.linspace(-20, 20, 16001), torch.logspace(-6, 1, 8000),
                   -torch.logspace(-6, 1, 8000))).to(DEV)
    z = z[:z.numel() // 4 * 4]
    c = z.numel()
    shape = (1, 1, 1, c) if layout == "NHWC" else (1, c, 1, 1)
    x = torch.zeros(shape, device=DEV)
    gn = tr.GroupNorm(shape, 1, F32, layout, act)
    stats = gn.new_stats()
    y = gn(x, None, z, stats=stats).flatten().double()
    dbeta = gn.grad(x, torch.ones_like(x), stats, None, z)[2].double()
    z = z.double()
    if act == "tanh":
        want, slope = torch.tanh(z), 1 - torch.tanh(z) ** 2
        tol, tol_slope = 4 * U * want.abs(), 10 * U * want ** 2 + 2 * U * slope
    else:
        s = torch.sigmoid(z)
        want, slope = z * s, s * (1 + z * (1 - s))
        tol = (2 * (1 - s) + 3) * U * want.abs()
        # s is off by 2u (1 - s) + 2u of itself, 1 - s by that of s and u of itself
        of_s = (2 * (1 - s) + 2) * U
        tol_slope = slope.abs() * (of_s + 3 * U) + s * z.abs() * (s * of_s + (1 - s) * 3 * U)
    print("norm", act, layout, "off by", float(((y - want).abs() / tol).nan_to_num().max()),
          float(((dbeta - slope).abs() / tol_slope).nan_to_num().max()), "of the tolerance", flush=True)
    assert ((y - want).abs() <= tol).all()
    assert ((dbeta - slope).abs() <= tol_slope).all()


@pytest.mark.parametrize("form", FORMS, ids=_ids)
def test_graph_replays_and_streams(form):
    """The same bits in a graph's replays, on a side stream and through the raw entry points."""
    layout, dtype, shape = form[:3]
    gn = _norm(form, "relu")
    x, dy, gamma, beta = _inputs(shape, dtype, 8)
    xs, dys, ga, be = _lay(x, layout).to(DEV), _lay(dy, layout).to(DEV), gamma.to(DEV), beta.to(DEV)
    out, st = torch.empty_like(xs), gn.new_stats()
    gn(xs, ga, be, out=out, stats=st)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gn(xs, ga, be, out=out, stats=st)
        grads = gn.grad(xs, dys, st, ga, be)
    side = torch.cuda.Stream()
    for seed in (9, 10, 11):
        x2, dy2, _, _ = _inputs(shape, dtype, seed)
        xs.copy_(_lay(x2, layout))
        dys.copy_(_lay(dy2, layout))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, st, *grads)]
        st2 = gn.new_stats()
        want = [gn(xs, ga, be, stats=st2), st2, *gn.grad(xs, dys, st2, ga, be)]
        assert all(torch.equal(a, b) for a, b in zip(got, want)), seed
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        st3 = gn.new_stats()
        again = [gn(xs, ga, be, stats=st3), st3, *gn.grad(xs, dys, st3, ga, be)]
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(again, want))
    raw = [torch.empty_like(t) for t in want]
    y, st4, dx, dgamma, dbeta = (t.data_ptr() for t in raw)
    plan = tr.huge2_norm_plan_create(gn.desc)
    stream = torch.cuda.current_stream().cuda_stream
    tr.huge2_norm_execute(plan, xs.data_ptr(), ga.data_ptr(), be.data_ptr(), y, st4, stream)
    tr.huge2_norm_grad_execute(plan, xs.data_ptr(), dys.data_ptr(), st4, ga.data_ptr(),
                               be.data_ptr(), dx, dgamma, dbeta, stream)
    tr.huge2_norm_plan_destroy(plan)
    assert all(torch.equal(a, b) for a, b in zip(raw, want))
