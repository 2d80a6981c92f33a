"""How far orthogonalised matrices are from the steps in 64 bits, by numbers like those that are
documented (include/huge2_train.h) and not by a model of the kernels' roundings.

The hard cases are matrices of low rank: a step takes a singular value that is nothing but
roundings up to 3.4 times as high, five steps 480 times, so that what a product leaves of them
is seen in the result.  Matrices are sums of products of whole numbers, which fp32 and bf16
hold without a rounding, so that their rank is what it says.
"""
import math

import pytest
import torch

from paper_1907_11210_amd import train as tr

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
SHAPES = [(2, 2), (3, 3), (4, 4), (5, 7), (8, 8), (16, 16), (24, 24), (32, 32), (48, 48), (64, 64),
          (2, 2000), (3, 512), (4, 512), (512, 4), (130, 16), (32, 700), (300, 48)]


def of_rank(rows, cols, rank, seed):
    """Whole numbers, of which bf16 holds all that are drawn here: those up to 256."""
    g = torch.Generator().manual_seed(seed)
    a, b = (torch.randint(-3, 4, s, generator=g).float() for s in ((rows, rank), (rank, cols)))
    a[0, 0] = b[0, 0] = 1  # (not all zeros)
    x = a @ b
    assert float(x.abs().max()) > 0
    return x


def steps(u):
    """Five steps in 64 bits."""
    x = u.double() / (u.double().norm() + 1e-7)
    if x.shape[0] > x.shape[1]:
        return steps(u.mT).mT
    a, b, c = tr.COEFFICIENTS
    for _ in range(5):
        g = x @ x.mT.contiguous()
        x = a * x + (b * g + c * (g @ g)) @ x
    return x


def ranks(shape):
    m = min(shape)
    return sorted({1, max(1, m // 4), max(1, m // 2), max(1, m - 1)})


def off(got, x):
    want = steps(x)
    return float((got.double().to(want.device) - want).norm() / want.norm())


# A result's rounding is at most half a step of every value, eps / 2 of it, and so of the norm.
ROUNDING = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def bound_f32(shape):
    """Up to 1024 the operands' 22 bits: a value's last part is off by 2^-23 of it at most, by a
    third of that on average, and five steps take what that leaves where a singular value is
    missing 3.4445^5 = 485 times as high: 2e-5 to 6e-5, and four times that is allowed.  Beyond,
    the sums of B X count.  Each is 3 m / 16 additions one after the other, off by half a last
    place of what has come together so far: on average 2^-24 sqrt(3 m / 16) / 3 of the sum, that
    is 5.5e-7 for m = 4096.  B X is |b + c| = 2.75 times X where its singular value is 1, and
    four more steps take the error 3.4445^4 = 141 times as high: 2.1e-4, for 8192 3e-4.  Values
    that are whole numbers of a few sizes have the same errors many times, so that they do not
    level out: three times that is allowed."""
    return 2.0 ** -12 if min(shape) <= 1024 else 2.0 ** -10



@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_products_are_fp32_where_nothing_else_is_asked_for(shape, dtype):
    """Tensors of 16 bits ask for results of 16 bits, not for operands of fewer."""
    op = tr.Orthogonalize(shape, dtype)
    for rank in ranks(shape):
        x = of_rank(*shape, rank, 10 + rank)
        err = off(op(x.to(DEV, dtype)), x)
        print("orthogonalize", shape, dtype, "rank", rank, "off by %.1e" % err, flush=True)
        assert err <= bound_f32(shape) + ROUNDING[dtype], rank


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_a_steps_products_are_fp32_where_nothing_else_is_asked_for(dtype):
    """The same of a Muon step: of zeros with lr 1 it leaves the update, its sign turned."""
    xs = [of_rank(*s, r, 20 + r) for s in SHAPES for r in ranks(s)]
    params = [torch.zeros(x.shape, dtype=dtype, device=DEV) for x in xs]
    muon = tr.Muon(params, scales=[1.0] * len(xs))
    assert muon.products == "f32"
    muon.step([x.to(DEV, dtype) for x in xs], lr=1.0, momentum=0.0, nesterov=False)
    for p, x in zip(params, xs):
        assert off(-p, x) <= bound_f32(x.shape) + ROUNDING[dtype], tuple(x.shape)


def test_five_steps_bring_singular_values_near_one():
    """Those of |U| / 500 and more to between 0.68 and 1.21; the polynomials' own ends, 0.6818 and
    1.2024, are among them (products in fp32 move none by more than 2^-12 sqrt(300) / 20)."""
    fine = torch.logspace(-math.log10(500), 0, 1 << 20, dtype=torch.float64)
    y = fine
    a, b, c = tr.COEFFICIENTS
    for _ in range(5):
        y = a * y + b * y ** 3 + c * y ** 5
    ends = fine[torch.stack((y.argmin(), y.argmax()))]
    s = torch.cat((ends, torch.logspace(math.log10(1 / 499), math.log10(0.04), 298,
                                        dtype=torch.float64)))
    s = torch.cat((s, (1 - (s * s).sum()).sqrt()[None]))  # |U| = 1
    g = torch.Generator().manual_seed(6)
    u, v = (torch.linalg.qr(torch.randn(n, len(s), generator=g).double())[0] for n in (320, 500))
    x = ((u * s) @ v.T).float()
    got = torch.linalg.svdvals(tr.Orthogonalize(x.shape, torch.float32)(x.to(DEV)).cpu().double())
    got = got[:len(s)]
    print("from %.4f to %.4f" % (float(got.min()), float(got.max())), flush=True)
    assert 0.68 <= float(got.min()) <= 0.684 and 1.2 <= float(got.max()) <= 1.21


# ---- products in f16 ---------------------------------


def bound_f16(shape):
    return 2.0 ** -6 if min(shape) >= 32 else 2.0 ** -3


@pytest.mark.parametrize("shape", SHAPES + [(1, 1), (2, 3), (2, 33), (33, 90), (128, 128)],
                         ids=lambda s: "x".join(map(str, s)))
def test_products_in_f16_of_low_rank(shape):
    op = tr.Orthogonalize(shape, torch.float32, "f16")
    for rank in ranks(shape):
        for seed in range(4):
            x = of_rank(*shape, rank, 100 * rank + seed)
            err = off(op(x.to(DEV)), x)
            print("f16", shape, "rank", rank, "off by %.1e" % err, flush=True)
            assert err <= bound_f16(shape), rank


@pytest.mark.parametrize("products", ["f32", "f16"])
@pytest.mark.parametrize("shape", [(3, 3), (5, 7), (16, 16), (24, 3), (32, 32), (40, 200), (256, 64)],
                         ids=lambda s: "x".join(map(str, s)))
def test_products_of_given_singular_values(shape, products):
    """One large singular value (or some) and the rest as small as |U| / 2000."""
    g, m = torch.Generator().manual_seed(5), min(shape)
    u, v = (torch.linalg.qr(torch.randn(n, m, generator=g).double())[0] for n in shape)
    op = tr.Orthogonalize(shape, torch.float32, products)
    for top in (1, max(1, m // 8), m):
        for small in (0.05, 0.02, 1 / 500, 1 / 2000):
            s = torch.full((m,), small).double()
            s[:top] = 1
            x = ((u * s) @ v.T).float()
            err = off(op(x.to(DEV)), x)
            print(products, shape, top, small, "off by %.1e" % err, flush=True)
            if products == "f32":
                assert err <= bound_f32(shape), (top, small)
            else:
                far = float(s.min() / s.norm()) >= 0.01
                assert err <= (2.0 ** -8 if far and m >= 32 else bound_f16(shape)), (top, small)


def alike(shape, kind, seed):
    """Rank 1 of few values, whose roundings are the same all over and do not level out."""
    g = torch.Generator().manual_seed(seed)
    if kind == "two":
        u, v = (torch.where(torch.rand(n, generator=g) < 0.5, 1.0, 3.0) for n in shape)
    elif kind == "blocks":
        values = torch.exp(3 * torch.rand(2, 3, generator=g) - 1.5)
        u, v = (w[torch.arange(n) * 3 // n] for w, n in zip(values, shape))
    else:  # few large ones between some of one size
        u, v = (torch.zeros(n) for n in shape)
        for w in (u, v):
            w[::7] = 1.7
            w[len(w) // 3] = 100
    return torch.outer(u, v).to(DEV)


def steps32(x):
    """The steps with fp32 products, by the device's library."""
    x = x / x.norm()
    if x.shape[0] > x.shape[1]:
        x = x.mT.contiguous()
    a, b, c = tr.COEFFICIENTS
    for _ in range(5):
        g = x @ x.mT.contiguous()
        x = a * x + (b * g + c * (g @ g)) @ x
    return x


@pytest.mark.parametrize("kind", ["two", "blocks", "few"])
@pytest.mark.parametrize("shape", [(2, 64), (8, 8), (64, 64), (256, 256), (1024, 1024), (1024, 8192),
                                   (4096, 4096), (8192, 8192)], ids=lambda s: "x".join(map(str, s)))
def test_roundings_that_are_alike(shape, kind):
    """Of rank 1, X = s u v^T, what is left beside u and v grows by a = 3.4445 a step, 141 times
    after the first.  To it come, of a product's size at most: its operands' last parts, 2^-22,
    and its sums' roundings, 2^-25 for each of their 3/16 additions a column.  B X is 2.74 times X,
    c A A 2.03, and A goes into B by |b| + 2 |c| = 8.8.  So 141 (2.74 + 2.03 + 8.8) 2^-22 = 2^-11
    and 141 * 3/16 * 2^-25 (4.8 m + 8.8 n), which is less than (m + n) 2^-17."""
    x = alike(shape, kind, 1)
    want = steps(x)
    size = float(want.norm())
    errs = [float((tr.Orthogonalize(shape, torch.float32, p)(x).double() - want).norm()) / size
            for p in ("f32", "f16")]
    fp32 = float((steps32(x).double() - want).norm()) / size
    print(shape, kind, "f32 off by %.1e, f16 %.1e, the library's fp32 %.1e" % (*errs, fp32), flush=True)
    assert errs[0] <= 2.0 ** -11 + sum(shape) * 2.0 ** -17
    assert errs[1] <= 2.0 ** -3


@pytest.mark.parametrize("products", ["f32", "f16"])
@pytest.mark.parametrize("shape", [(512, 512), (1024, 1024), (3000, 700), (4096, 4096),
                                   (8192, 8192)],
                         ids=lambda s: "x".join(map(str, s)))
def test_large_matrices_of_low_rank(shape, products):
    """(The steps in 64 bits by the device.)"""
    op = tr.Orthogonalize(shape, torch.float32, products)
    for rank in (1, 8, 64):
        x = of_rank(*shape, rank, rank).to(DEV)
        err = off(op(x), x)
        print(products, shape, "rank", rank, "off by %.1e" % err, flush=True)
        assert err <= (bound_f32 if products == "f32" else bound_f16)(shape), rank
