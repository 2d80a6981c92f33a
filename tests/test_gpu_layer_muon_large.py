"""Layer norm, orthogonalised matrices and the Muon step over more than 2^31 elements on the GPU,
where indices and offsets pass 32 bits: every element against the definitions in 64 bits, by
parts, on the device.  Tolerances as in test_gpu_layer_norm.py and test_gpu_muon_accuracy.py.
"""
import math

import pytest
import torch

from paper_1907_11210_amd import train as tr
from test_gpu_layer_norm import DEPTH, U, _grad_reference, _guarded, _kept, _reference, _within

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(autouse=True)
def memory():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def _parts(shape, layout):
    """Slices of whole pixels, as functions of a tensor and of its statistics."""
    if layout == "NHWC":
        rows, c = shape
        step = (1 << 26) // c
        for a in range(0, rows, step):
            yield (lambda t, s=slice(a, a + step): t[s]), slice(a, min(a + step, rows))
    else:
        n, c, h, w = shape
        step = (1 << 26) // c
        for i in range(n):
            for a in range(0, h * w, step):
                b = min(a + step, h * w)
                yield (lambda t, i=i, s=slice(a, b): t[i].flatten(1)[:, s].T.contiguous()), \
                    slice(i * h * w + a, i * h * w + b)


LAYERS = [((2200001, 1000), "NHWC", torch.bfloat16, "relu", "rows"),
          ((66000, 32776), "NHWC", torch.bfloat16, None, "long"),
          ((40, 512, 331, 331), "NCHW", torch.bfloat16, None, "planes"),
          ((2, 33, 5801, 5801), "NCHW", torch.float32, "relu", "planes")]


@pytest.mark.parametrize("shape,layout,dtype,act,form", LAYERS,
                         ids=["x".join(map(str, c[0])) for c in LAYERS])
def test_layer_norm(shape, layout, dtype, act, form):
    assert math.prod(shape) > 2 ** 31
    g = torch.Generator(DEV).manual_seed(1)
    c = shape[1]
    x, dy = (torch.randn(shape, generator=g, device=DEV, dtype=dtype) for _ in range(2))
    gamma = 1 + 0.5 * torch.randn(c, generator=g, device=DEV)
    beta = 0.5 * torch.randn(c, generator=g, device=DEV)
    ln = tr.LayerNorm(shape, dtype, layout, act)
    print("layer norm", shape, layout, ln.kernels, flush=True)
    assert all(form in k for k in ln.kernels)
    stats, around = _guarded(ln.stats_shape, torch.float32)
    out, whole = _guarded(shape, dtype)
    ln(x, gamma, beta, out=out, stats=stats)
    torch.cuda.synchronize()
    assert _kept(whole) and _kept(around)
    for part, pixels in _parts(shape, layout):
        xs = part(x)
        ref, mean, rstd = _reference(xs, gamma, beta, act)
        xmax, by = xs.abs().max().double(), rstd[:, None]
        tol = U * (DEPTH * (xmax * by + (xs.double().abs() + xmax) * by) + 8) * \
            gamma.double().abs() * 1.1 + U * 8 * beta.double().abs()
        assert bool(_within(part(out).double(), ref, tol, dtype).all()), pixels
        st = stats[pixels].double()
        assert bool(((st[:, 0] - mean).abs() <= DEPTH * U * xmax).all()), pixels
        assert bool(((st[:, 1] - rstd).abs() <= DEPTH * U * (1 + xmax * rstd) * rstd).all()), pixels
        del ref, tol, xs
    out.fill_(7)
    _, dgamma, dbeta = ln.grad(x, dy, stats, gamma, beta, out=out)
    torch.cuda.synchronize()
    assert _kept(whole)
    sums = torch.zeros(4, c, dtype=torch.float64, device=DEV)
    for part, pixels in _parts(shape, layout):
        xs, ds = part(x), part(dy)
        rx, rg, rb, mag, dz, xh, near = _grad_reference(xs, ds, gamma, beta, stats[pixels], act)
        slope = 4 * U * (2 + (near * (1 + gamma.double().abs())).max())
        tol = mag * (DEPTH * U + slope) * 2
        assert bool(_within(part(out).double(), rx, tol, dtype).all()), pixels
        # (a thread's sums are some 10^3 to 10^5 additions of numbers that come to less than
        # their magnitudes' sum, each off by less than u of it: by no more than their root)
        sums[0] += rb
        sums[1] += rg
        sums[2] += ((DEPTH * U + slope) * dz.abs()).sum(0)
        sums[3] += ((DEPTH * U + slope) * (dz * xh).abs() + slope * dz.abs()).sum(0)
        del rx, rg, rb, mag, dz, xh, near, tol, xs, ds
    assert bool(((dbeta.double() - sums[0]).abs() <= sums[2]).all())
    assert bool(((dgamma.double() - sums[1]).abs() <= sums[3]).all())


def _polynomial(u):
    """Q of X = Q U / (|U| + eps) after five steps, from U U^T in 64 bits (rows are few)."""
    m = u.shape[0]
    gram = torch.zeros(m, m, dtype=torch.float64, device=DEV)
    for at in range(0, u.shape[1], 1 << 22):
        v = u[:, at:at + (1 << 22)].double().contiguous()
        for i in range(m):
            gram[i] += (v * v[i]).sum(1)
    size = float(gram.trace()) ** 0.5 + 1e-7
    a, b, c = tr.COEFFICIENTS
    eye = torch.eye(m, dtype=torch.float64, device=DEV)
    q, g = eye / size, gram / size ** 2
    for _ in range(5):
        p = a * eye + b * g + c * (g @ g)
        q, g = p @ q, p @ g @ p.T.contiguous()
    return q, float(g.trace()) ** 0.5


BOUND = 2.0 ** -12  # of products in fp32, up to 1024 rows


def test_orthogonalize_a_batch():
    """More than 2^31 elements, and operands of which a matrix takes 3.2 GB: one after the other."""
    shape = (13, 40, 4194305)
    assert math.prod(shape) > 2 ** 31
    g = torch.Generator(DEV).manual_seed(2)
    x = torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)
    out, whole = _guarded(shape, torch.bfloat16)
    print("orthogonalize", shape, flush=True)
    tr.Orthogonalize(shape, torch.bfloat16)(x, out=out)
    torch.cuda.synchronize()
    assert _kept(whole)
    for i in range(shape[0]):
        q, norm = _polynomial(x[i])
        one = 12 * BOUND * norm / math.sqrt(x[i].numel())
        for at in range(0, shape[2], 1 << 22):
            want = q @ x[i, :, at:at + (1 << 22)].double()
            err = (out[i, :, at:at + (1 << 22)].double() - want).abs()
            assert bool((err <= one + 2.0 ** -8 * want.abs()).all()), (i, at)


@pytest.mark.parametrize("shape", [(33, 65075262), (65075262, 33)], ids=["wide", "tall"])
def test_step_of_a_matrix_of_almost_2_to_the_31(shape):
    """The last elements of parameters, momenta and copies."""
    n = math.prod(shape)
    assert 2 ** 31 - 66 < n < 2 ** 31
    g = torch.Generator(DEV).manual_seed(3)
    grad = torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)
    m, m_whole = _guarded(shape, torch.float32)
    p, p_whole = _guarded(shape, torch.float32)
    copy, c_whole = _guarded(shape, torch.bfloat16)
    m.zero_()
    p.zero_()
    print("muon", shape, flush=True)
    muon = tr.Muon([p], copies=[copy], m=[m], scales=[1.0])
    muon.step([grad], lr=1.0, momentum=0.5, nesterov=False)
    torch.cuda.synchronize()
    assert _kept(m_whole) and _kept(p_whole) and _kept(c_whole)
    muon.close()
    wide = (lambda t: t) if shape[0] < shape[1] else (lambda t: t.T)
    q, norm = _polynomial(wide(grad))
    one = 12 * BOUND * norm / math.sqrt(n)
    for at in range(0, max(shape), 1 << 22):
        part = slice(at, at + (1 << 22))
        u = wide(grad)[:, part].double().contiguous()
        assert bool((wide(m)[:, part].double() == 0.5 * u).all()), at
        got, want = wide(p)[:, part], q @ u
        assert bool(((got.double() + want).abs() <= one + U * want.abs()).all()), at
        assert bool((wide(copy)[:, part] == got.bfloat16()).all()), at
