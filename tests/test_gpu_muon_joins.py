"""Orthogonalised matrices and Muon steps whose products are cut along their sums and joined,
on the GPU (test_muon_joins_plan.py asserts which: every product, every size of tiles that the
rule cuts, lists that mix whole and cut tiles), against the formulas in 64 bits.

Tolerances, of a result's norm, as in test_gpu_muon.py by the same steps with operands rounded
to 11 bits (or two parts of 11) and sums to fp32 every 8 columns, here with half as much again
instead of three times: the matrices have 10^5 elements and more, whose roundings are as many
independent ones, so that their norm stands still.  2e-6 are added for the order of fp32's sums,
which for matrices of random numbers is what fp32's products are off by.  Without the mean of
A's diagonal, which every step takes from what the joins before it leave, f16 is off by three
times as much.
"""
import math

import pytest
import torch

from paper_1907_11210_amd import train as tr
from test_gpu_muon import _model_error, _steps
from test_muon_joins_plan import JOINED

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
CASES = [(products, i) for products in JOINED for i in range(len(JOINED[products]))]


def _name(case):
    shapes, _ = JOINED[case[0]][case[1]]
    return case[0] + "-" + "-".join("%dx%d" % s for s in shapes[:2]) + "-%d" % len(shapes)


def _want(u, parts, kept={}):
    """The steps' result in 64 bits, and how far off it may be."""
    with torch.device(DEV):
        want = _steps(u)
        if (u.shape, parts) not in kept:  # (the same for other numbers of the same kind)
            kept[u.shape, parts] = 1.5 * _model_error(u, want, parts) + 2e-6
    return want, kept[u.shape, parts]


def _random(shapes, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    return [torch.randn(s, generator=g, device=DEV) for s in shapes]


@pytest.mark.parametrize("case", CASES, ids=_name)
def test_steps(case):
    """Parameters in fp32 with copies and in bf16, a matrix without a gradient."""
    products, (shapes, skipped) = case[0], JOINED[case[0]][case[1]]
    parts = 2 if products == "f32" else 1
    lr, decay, momentum = 0.25, 0.1, 0.9
    dtypes = [torch.bfloat16 if i % 2 else torch.float32 for i in range(len(shapes))]
    gs, ms = _random(shapes, 1), _random(shapes, 2)
    ps = [(0.05 * p).to(d) for p, d in zip(_random(shapes, 3), dtypes)]
    params, momenta = [p.clone() for p in ps], [m.clone() for m in ms]
    copies = [torch.full(s, 5, dtype=torch.bfloat16, device=DEV) if d == torch.float32 else None
              for s, d in zip(shapes, dtypes)]
    muon = tr.Muon(params, decay, copies=copies, grad_dtypes=[torch.float32] * len(shapes),
                   m=momenta, products=products)
    print("muon", _name(case), flush=True)
    muon.step([None if i == skipped else g for i, g in enumerate(gs)], lr=lr, momentum=momentum)
    torch.cuda.synchronize()
    for i, (p, m, g) in enumerate(zip(ps, ms, gs)):
        if i == skipped:
            assert torch.equal(params[i], p) and torch.equal(momenta[i], m)
            assert copies[i] is None or bool((copies[i] == 5).all())
            continue
        m2 = momentum * m.double() + (1 - momentum) * g.double()
        size = momentum * m.double().abs() + (1 - momentum) * g.double().abs()
        assert bool(((momenta[i].double() - m2).abs() <= 6 * U * size).all()), i
        x, tol = _want(momentum * m2 + (1 - momentum) * g.double(), parts)
        rate = lr * muon.scales[i]
        p2 = p.double() * (1 - lr * decay) - rate * x
        # a single element is off by at most 12 times its share (as in test_gpu_muon.py), the
        # parameter's own arithmetic by a few roundings of its terms
        own = 4 * U * (p.double().abs() + rate * x.abs())
        one = 12 * tol * rate * float(x.norm()) / math.sqrt(x.numel()) + own
        got = params[i].double()
        if dtypes[i] == torch.bfloat16:
            lo, hi = ((p2 + d).to(torch.bfloat16).double() for d in (-one, one))
            assert bool(((got >= lo) & (got <= hi)).all()), i
        else:
            err = got - p2
            off = float(err.norm()) / rate / float(x.norm())
            print(shapes[i], "off by %.2e, allowed %.2e" % (off, tol), flush=True)
            assert float(err.norm()) <= tol * rate * float(x.norm()) + float(own.norm()), i
            assert bool((err.abs() <= one).all()), i
            assert torch.equal(copies[i], params[i].bfloat16()), i


@pytest.mark.parametrize("case", [c for c in CASES if len(set(JOINED[c[0]][c[1]][0])) == 1],
                         ids=_name)
def test_orthogonalize(case):
    """The same of matrices of one shape, and nothing behind a result's end."""
    products, (shapes, _) = case[0], JOINED[case[0]][case[1]]
    x = torch.stack(_random(shapes, 4))
    n = x.numel()
    whole = torch.full((n + 128,), 7.0, device=DEV)
    out = whole[64:64 + n].view(x.shape)
    print("orthogonalize", _name(case), flush=True)
    op = tr.Orthogonalize(x.shape, torch.float32, products)
    op(x, out=out)
    again = op(x)
    torch.cuda.synchronize()
    assert bool((whole[:64] == 7).all()) and bool((whole[-64:] == 7).all())
    assert torch.equal(out, again)
    for a, b in zip(out, x):
        want, tol = _want(b, 2 if products == "f32" else 1)
        err = a.double() - want
        off = float(err.norm() / want.norm())
        print(tuple(b.shape), "off by %.2e, allowed %.2e" % (off, tol), flush=True)
        assert off <= tol
        assert float(err.abs().max()) <= 12 * tol * float(want.norm()) / math.sqrt(want.numel())
