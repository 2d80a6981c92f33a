"""Results and states so large that they pass the caches, by every width of a store: the
same definitions and tolerances as for small ones (test_gpu_norm, test_gpu_embedding,
test_gpu_adamw), computed on the GPU in 64 bits where the CPU would take long.
"""
import pytest
import torch

from paper_1907_11210_amd import train as tr
from test_gpu_adamw import O, _decode, _expect, _opt, _state
from test_gpu_norm import DEPTH, _grad_reference, _lay, _reference, _unlay, _within

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16

# layout, type, (n, c, h, w, groups), what the kernels' names begin with: 64 MiB and more
NORMS = [
    ("NHWC", BF16, (512, 256, 16, 16, 32), "norm_slab_nhwc_kernel v8", "norm_slab_grad_nhwc_kernel v8"),
    ("NHWC", F32, (512, 256, 16, 16, 32), "norm_slab_nhwc_kernel v4", "norm_slab_grad_nhwc_kernel v4"),
    ("NHWC", BF16, (600, 250, 16, 16, 5), "norm_slab_nhwc_kernel v2", "norm_slab_grad_nhwc_kernel v2"),
    ("NHWC", F32, (64, 128, 64, 64, 4), "norm_run_nhwc_kernel v4", "norm_run_grad_nhwc_kernel v4"),
    ("NHWC", BF16, (40, 250, 64, 64, 5), "norm_run_nhwc_kernel v2", "norm_run_grad_nhwc_kernel v2"),
    ("NHWC", F32, (40, 251, 48, 48, 1), "norm_run_nhwc_kernel v1", "norm_run_grad_nhwc_kernel v1"),
    ("NHWC", BF16, (16, 16400, 8, 16, 1), "norm_sums_nhwc_kernel v8", "norm_sums_nhwc_kernel v8"),
    ("NHWC", F32, (8, 16398, 12, 12, 1), "norm_sums_nhwc_kernel v1", "norm_sums_nhwc_kernel v1"),
    ("NCHW", BF16, (512, 256, 16, 16, 32), "norm_slab_nchw_kernel v8", "norm_slab_nchw_kernel v8"),
    ("NCHW", F32, (512, 256, 16, 16, 32), "norm_slab_nchw_kernel v4", "norm_slab_nchw_kernel v4"),
    ("NCHW", F32, (64, 128, 64, 64, 4), "norm_sums_nchw_kernel v4", "norm_sums_nchw_kernel v4"),
    ("NCHW", BF16, (32, 300, 42, 123, 4), "norm_sums_nchw_kernel v2", "norm_sums_nchw_kernel v2"),
    ("NCHW", BF16, (16, 1100, 48, 48, 1), "norm_sums_nchw_kernel v8", "norm_sums_nchw_kernel v8"),
]


@pytest.mark.parametrize("form", NORMS, ids=lambda f: "%s-%s-%s" % (
    f[0], "f32" if f[1] == F32 else "bf16", "x".join(map(str, f[2]))))
def test_norm(form):
    layout, dtype, shape, forward, backward = form
    n, c, h, w, groups = shape
    gn = tr.GroupNorm((n, h, w, c) if layout == "NHWC" else (n, c, h, w), groups, dtype, layout,
                      "relu")
    print("norm", form, gn.kernels, flush=True)
    assert gn.kernels[0].startswith(forward) and gn.kernels[1].startswith(backward)
    assert n * c * h * w * dtype.itemsize >= 64 << 20
    g = torch.Generator(DEV).manual_seed(1)
    normal = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    x, dy = ((normal(n, c, h, w) + m * normal(c, 1, 1)).to(dtype) for m in (1, 0))
    gamma, beta = 1 + 0.5 * normal(c), 0.5 * normal(c)
    stats = gn.new_stats()
    xs, out = _lay(x, layout), torch.full(gn.x_shape, float("nan"), dtype=dtype, device=DEV)
    gn(xs, gamma, beta, out=out, stats=stats)
    ref, mean, rstd = _reference(x, gamma, beta, groups, "relu", 1e-5)
    xmax = x.double().abs().max()
    by = rstd.repeat_interleave(c // groups, 1)[..., None, None]
    tol = U * (DEPTH * (xmax * by + (x.double().abs() + xmax) * by) + 8) * 1.1 \
        * gamma.double().abs()[:, None, None] + U * 8 * beta.double().abs()[:, None, None]
    assert _within(_unlay(out, layout).double(), ref, tol, dtype).all()
    del ref, tol
    out.fill_(float("nan"))
    _, dgamma, dbeta = gn.grad(xs, _lay(dy, layout), stats, gamma, beta, out=out)
    rx, rg, rb, mag, dz, xh, near = _grad_reference(x, dy, gamma, beta, stats, groups, "relu")
    slope = 4 * U * (2 + (near * (1 + gamma.double().abs()[:, None, None])).max())
    assert _within(_unlay(out, layout).double(), rx, mag * (DEPTH * U + slope) * 2, dtype).all()
    tol_b = ((DEPTH * U + slope) * dz.abs()).sum((0, 2, 3))
    tol_g = (DEPTH * U * (dz * xh).abs() + slope * dz.abs() * (1 + xh.abs())).sum((0, 2, 3))
    assert ((dbeta.double() - rb).abs() <= tol_b).all()
    assert ((dgamma.double() - rg).abs() <= tol_g).all()


@pytest.mark.parametrize("dtype,dim", [(F32, 256), (F32, 258), (F32, 257), (BF16, 256), (BF16, 260),
                                       (BF16, 258), (BF16, 257)],
                         ids=["f32-16B", "f32-8B", "f32-4B", "bf16-16B", "bf16-8B", "bf16-4B", "bf16-2B"])
def test_lookup(dtype, dim):
    """Results of 16 MiB and more, exact."""
    rows, tokens = 5000, (17 << 20) // (dim * dtype.itemsize) + 3
    g = torch.Generator(DEV).manual_seed(2)
    table = torch.randn(rows, dim, generator=g, device=DEV).to(dtype)
    ids = torch.randint(-1, rows + 1, (tokens,), generator=g, device=DEV)
    print("lookup", tokens, rows, dim, dtype, flush=True)
    y = tr.Embedding(rows, dim, dtype, scale=1.7)(ids, table, out=torch.full(
        (tokens, dim), float("nan"), dtype=dtype, device=DEV))
    assert y.numel() * dtype.itemsize >= 16 << 20
    known = (ids >= 0) & (ids < rows)
    want = (table[torch.where(known, ids, 0)].float() * torch.tensor(1.7, device=DEV)).to(dtype)
    assert torch.equal(y, torch.where(known[:, None], want, 0))


def test_adamw_codes():
    """Moments in 8 bits beside 64 MiB of fp32 parameters: numbers and scales, not parameters
    alone."""
    sizes = [17000001, 1025, 2047]
    s = _state(sizes, 8, F32, BF16, 10)
    opt, dev = _opt(s, 8, True, 0.1)
    print("adamw", sizes, flush=True)
    opt.step(dev["g"], step=3, **O)
    torch.cuda.synchronize()
    for i, n in enumerate(sizes):
        p2, m2, v2, tol, mag = _expect(s, i, 8, 3, 0.1)
        assert _within(dev["p"][i].cpu().double(), p2, tol, F32).all(), i
        for k, want, err in (("m", m2, 6 * U * mag), ("v", v2.sqrt(), 6 * U * v2.sqrt())):
            scale = dev[k + "_scale"][i].cpu()
            top = torch.nn.functional.pad(want, (0, -n % 256)).reshape(-1, 256).abs().amax(1)
            assert ((scale.double() - top / 448).abs() <= 16 * U * top / 448).all()
            per = (top / 448).repeat_interleave(256)[:n]
            tol = torch.maximum(want.abs() / 16, per * 2.0 ** -10) * (1 + 2.0 ** -10) + err \
                + 16 * U * want.abs()
            if k == "v":  # (a root that is not zero may be lifted to the smallest number)
                tol = torch.maximum(tol, per * 2.0 ** -9)
            assert ((_decode(dev[k][i].cpu(), scale) - want).abs() <= tol).all(), (k, i)
