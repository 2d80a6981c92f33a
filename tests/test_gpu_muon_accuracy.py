"""How far orthogonalised matrices are from the steps in 64 bits, by the numbers that are
documented (include/huge2_train.h) and not by a model of the kernels' roundings.

The hard cases are matrices of low rank: a step takes a singular value that is nothing but
roundings up to 3.4 times as high, five steps 480 times, so that what a product leaves of them
is seen in the result.  Matrices are sums of products of whole numbers, which fp32 and bf16
hold without a rounding, so that their rank is what it says.
"""
import pytest
import torch

from paper_1907_11210_amd import train as tr

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
SHAPES = [(2, 2), (3, 3), (4, 4), (5, 7), (8, 8), (16, 16), (24, 24), (32, 32), (48, 48), (64, 64),
          (2, 2000), (3, 512), (4, 512), (512, 4), (130, 16), (32, 700), (300, 48)]


def of_rank(rows, cols, rank, seed):
    """Whole numbers, of which bf16 holds those up to 256."""
    g = torch.Generator().manual_seed(seed)
    a, b = (torch.randint(-3, 4, s, generator=g).float() for s in ((rows, rank), (rank, cols)))
    a[0, 0] = b[0, 0] = 1  # (not all zeros)
    x = a @ b
    assert torch.equal(x.bfloat16().float(), x) and 0 < float(x.abs().max())
    return x


def steps(u):
    """Five steps in 64 bits."""
    x = u.double() / (u.double().norm() + 1e-7)
    if x.shape[0] > x.shape[1]:
        return steps(u.mT).mT
    a, b, c = tr.COEFFICIENTS
    for _ in range(5):
        g = x @ x.mT
        x = a * x + (b * g + c * (g @ g)) @ x
    return x


def ranks(shape):
    m = min(shape)
    return sorted({1, max(1, m // 4), max(1, m // 2), max(1, m - 1)})


def off(got, x):
    want = steps(x)
    return float((got.cpu().double() - want).norm() / want.norm())


# A result's rounding: at most half a step of every value, eps / 2 of it, and so of the norm.
ROUNDING = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
F32 = 2.0 ** -12  # of matrices of low rank; others are off by some 2^-19


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_products_are_fp32_where_nothing_else_is_asked_for(shape, dtype):
    """Tensors of 16 bits ask for results of 16 bits, not for operands of fewer."""
    op = tr.Orthogonalize(shape, dtype)
    for rank in ranks(shape):
        x = of_rank(*shape, rank, 10 + rank)
        err = off(op(x.to(DEV, dtype)), x)
        print("orthogonalize", shape, dtype, "rank", rank, "off by %.1e" % err, flush=True)
        assert err <= F32 + ROUNDING[dtype], rank


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_a_steps_products_are_fp32_where_nothing_else_is_asked_for(dtype):
    """The same of a Muon step: of zeros with lr 1 it leaves the update, its sign turned."""
    xs = [of_rank(*s, r, 20 + r) for s in SHAPES for r in ranks(s)]
    params = [torch.zeros(x.shape, dtype=dtype, device=DEV) for x in xs]
    muon = tr.Muon(params, scales=[1.0] * len(xs))
    assert muon.products == "f32"
    muon.step([x.to(DEV, dtype) for x in xs], lr=1.0, momentum=0.0, nesterov=False)
    for p, x in zip(params, xs):
        assert off(-p, x) <= F32 + ROUNDING[dtype], tuple(x.shape)
