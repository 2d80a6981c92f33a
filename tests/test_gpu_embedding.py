"""Embedding lookup and the table's gradient on the GPU.

The lookup rounds once: it equals the CPU's product bit by bit.  A row of the
gradient adds up its tokens in fp32 in some order: off by less than (tokens + 2) * u
of the sum of their magnitudes, u = 2^-24; a bf16 row is such a sum's rounding.
Gradients that are small whole numbers add up exactly.
"""
import pytest
import torch

from paper_1907_11210_amd import train as tr

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24


def _within(got, ref, tol, dtype):
    """A result of `dtype` of a value that is off by at most tol: between the roundings of
    the interval's ends (rounding keeps order); fp32: its own rounding beside tol."""
    if dtype == torch.bfloat16:
        lo, hi = (v.to(dtype).double() for v in (ref - tol, ref + tol))
        return (got >= lo) & (got <= hi)
    return (got - ref).abs() <= tol + ref.abs() * U

# tokens, rows, dim
SHAPES = [
    (1, 1, 1), (1, 1000, 64), (3, 5, 8), (64, 100, 100), (257, 255, 33), (1000, 256, 30),
    (1024, 257, 16), (1025, 70000, 24), (2000, 10, 2056), (5000, 3, 130), (33, 65536, 8),
    (4096, 1024, 256), (9000, 40, 4104),
]


def _ids(kind, tokens, rows, g):
    if kind == "one":
        return torch.full((tokens,), rows // 2, dtype=torch.int64)
    u = torch.rand(tokens, generator=g, dtype=torch.float64)
    ids = (u * rows).long() if kind == "uniform" else ((rows + 1.0) ** u).long().clamp(1, rows) - 1
    if kind == "outside":
        ids = (u * rows).long()
        ids[::3] = -1
        ids[1::7] = rows
        ids[2::11] = 2 ** 40
        ids[4::13] = -2 ** 62
    if kind == "nothing":
        ids[:] = -1
    return ids.clamp(max=2 ** 62)


KINDS = ("uniform", "skewed", "one", "outside", "nothing")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_lookup(shape, dtype):
    tokens, rows, dim = shape
    g = torch.Generator().manual_seed(1)
    table = torch.randn(rows, dim, generator=g).to(dtype)
    for kind in KINDS:
        print("lookup", shape, dtype, kind, flush=True)
        ids = _ids(kind, tokens, rows, g)
        emb = tr.Embedding(rows, dim, dtype, scale=1.7)
        y = emb(ids.to(DEV), table.to(DEV)).cpu()
        known = (ids >= 0) & (ids < rows)
        want = (table[torch.where(known, ids, 0)].float() * torch.tensor(1.7)).to(dtype)
        want[~known] = 0
        assert torch.equal(y, want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_gradient(shape, dtype):
    tokens, rows, dim = shape
    g = torch.Generator().manual_seed(2)
    dy = torch.randn(tokens, dim, generator=g).to(dtype)
    emb = tr.Embedding(rows, dim, dtype, scale=1.7, max_tokens=tokens)
    scale = float(torch.tensor(1.7))
    for kind in KINDS:
        print("gradient", shape, dtype, kind, flush=True)
        ids = _ids(kind, tokens, rows, g)
        known = (ids >= 0) & (ids < rows)
        out = torch.full((rows, dim), 9.0, dtype=dtype, device=DEV)
        emb.grad(ids.to(DEV), dy.to(DEV), out=out)
        got = out.cpu().double()
        zeros = torch.zeros(rows, dim, dtype=torch.float64)
        want = zeros.index_add(0, ids[known], dy[known].double()) * scale
        mag = zeros.index_add(0, ids[known], dy[known].double().abs()) * scale
        count = torch.zeros(rows, dtype=torch.float64).index_add(
            0, ids[known], torch.ones(int(known.sum()), dtype=torch.float64))
        assert _within(got, want, U * (count + 2)[:, None] * mag, dtype).all()
        assert (got[count == 0] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(3000, 50, 100), (1500, 700, 6), (3000, 50, 50), (500, 90, 12)],
                         ids=lambda s: "x".join(map(str, s)))
def test_rows_of_half_vectors(shape, dtype):
    """Rows that 8 bytes divide and 16 do not (and 4, in the other type)."""
    test_lookup(shape, dtype)
    test_gradient(shape, dtype)


@pytest.mark.parametrize("id_dtype", [torch.int32, torch.int64])
def test_gradient_of_whole_numbers(id_dtype):
    """Exact, over every number of tokens around the sizes at which work is cut."""
    g = torch.Generator().manual_seed(3)
    rows, dim = 300, 40
    emb = tr.Embedding(rows, dim, torch.float32, max_tokens=3000, id_dtype=id_dtype)
    for tokens in (0, 1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 255, 256, 257, 1023, 1024, 1025,
                   2047, 2048, 2049, 3000):
        for kind in ("skewed", "one", "outside"):
            ids = _ids(kind, tokens, rows, g)
            if id_dtype == torch.int32:
                ids = torch.where(ids.abs() > 2 ** 31 - 1, -5, ids)
            ids = ids.to(id_dtype)
            known = (ids >= 0) & (ids < rows)
            dy = torch.randint(-8, 9, (tokens, dim), generator=g).float()
            out = torch.full((rows, dim), 9.0, device=DEV)
            emb.grad(ids.to(DEV), dy.to(DEV), out=out)
            want = torch.zeros(rows, dim).index_add(0, ids[known].long(), dy[known])
            assert torch.equal(out.cpu(), want), (tokens, kind)


def test_long_sorts():
    """Many tiles of tokens, two and three digits of ids, one id with half of the tokens."""
    g = torch.Generator().manual_seed(4)
    for tokens, rows, dim in ((200000, 1000, 8), (150001, 70000, 4), (300000, 2 ** 24 + 5, 1)):
        ids = _ids("uniform", tokens, rows, g)
        ids[torch.rand(tokens, generator=g) < 0.5] = rows - 1
        dy = torch.randint(-3, 4, (tokens, dim), generator=g).float()
        emb = tr.Embedding(rows, dim, torch.float32, max_tokens=tokens)
        got = emb.grad(ids.to(DEV), dy.to(DEV)).cpu()
        assert torch.equal(got, torch.zeros(rows, dim).index_add(0, ids, dy)), (tokens, rows)


def test_order_is_fixed():
    """The same bits each time, also on another stream, and for shapes of ids."""
    g = torch.Generator().manual_seed(5)
    ids, dy = _ids("skewed", 6000, 500, g).to(DEV), torch.randn(6000, 72, generator=g).to(DEV)
    table = torch.randn(500, 72, generator=g).to(DEV)
    emb = tr.Embedding(500, 72, torch.float32, max_tokens=6000)
    first = emb.grad(ids, dy)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        again = emb.grad(ids.reshape(60, 100), dy.reshape(60, 100, 72))
    s.synchronize()
    assert torch.equal(first, again)
    assert torch.equal(emb(ids.reshape(60, 100), table).reshape(6000, 72), emb(ids, table))


def test_graph_replays():
    g = torch.Generator().manual_seed(6)
    tokens, rows, dim = 3000, 700, 64
    emb = tr.Embedding(rows, dim, torch.bfloat16, scale=0.5, max_tokens=tokens)
    ids = _ids("skewed", tokens, rows, g).to(DEV)
    dy = torch.randn(tokens, dim, generator=g).bfloat16().to(DEV)
    table = torch.randn(rows, dim, generator=g).bfloat16().to(DEV)
    emb.grad(ids, dy)
    emb(ids, table)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, dt = emb(ids, table), emb.grad(ids, dy)
    for kind in ("one", "outside", "uniform"):
        ids.copy_(_ids(kind, tokens, rows, g))
        dy.copy_(torch.randn(tokens, dim, generator=g))
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone(), dt.clone()
        assert torch.equal(got[0], emb(ids, table)) and torch.equal(got[1], emb.grad(ids, dy))


def test_refusals(monkeypatch):
    emb = tr.Embedding(10, 16, torch.float32, max_tokens=4)
    ids, table = torch.zeros(4, dtype=torch.int64, device=DEV), torch.zeros(10, 16, device=DEV)
    dy = torch.zeros(4, 16, device=DEV)
    for call in (lambda: emb(ids.int(), table), lambda: emb(ids.cpu(), table),
                 lambda: emb(ids, table[:9]), lambda: emb(ids, table.bfloat16()),
                 lambda: emb(ids[::2], table), lambda: emb(ids, table, out=dy[:3]),
                 lambda: emb.grad(ids, dy[:3]), lambda: emb.grad(ids, dy.bfloat16())):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        tr.Embedding(10, 16, torch.float32, id_dtype=torch.int16)
    more = torch.zeros(5, dtype=torch.int64, device=DEV)
    with pytest.raises(tr.h2.Huge2Error):
        emb.grad(more, torch.zeros(5, 16, device=DEV))
    assert emb(ids[:0], table).shape == (0, 16)
    assert float(emb.grad(ids[:0], dy[:0], out=torch.ones_like(table)).abs().max()) == 0
    monkeypatch.setenv("HUGE2_FAULT", "alloc")
    with pytest.raises(tr.h2.Huge2Error):
        tr.Embedding(10, 16, torch.float32, max_tokens=4)
    monkeypatch.setenv("HUGE2_FAULT", "launch")
    with pytest.raises(tr.h2.Huge2Error):
        emb(ids, table)


def test_lookup_of_more_than_a_launch_takes():
    """2^26 tokens of 129 channels are 2^24 workgroups of 256: two launches."""
    tokens, rows, dim = (1 << 26) + 5, 7, 129
    ids = torch.arange(tokens, device=DEV) % (rows + 1)  # the last is outside the table
    table = torch.randn(rows, dim, generator=torch.Generator().manual_seed(6)).bfloat16()
    y = tr.Embedding(rows, dim, torch.bfloat16)(ids, table.to(DEV))
    torch.cuda.synchronize()
    padded = torch.cat((table, torch.zeros(1, dim, dtype=torch.bfloat16))).to(DEV)
    for first in range(0, tokens, 1 << 22):
        part = slice(first, min(tokens, first + (1 << 22)))
        assert torch.equal(y[part], padded[ids[part]]), first


def test_embedding_kernels_and_raw_entry():
    """Which kernels a gradient takes, and the lookup through its raw entry point."""
    emb = tr.Embedding(100, 24, torch.float32, max_tokens=5000)
    assert [emb.kernel(n) for n in (1024, 1025)] == ["embedding_few_kernel v4",
                                                     "embedding_sum_kernel v4"]
    ids = torch.arange(300, device=DEV) % 101
    table = torch.randn(100, 24, device=DEV)
    y = torch.empty(300, 24, device=DEV)
    tr.huge2_embedding(emb.desc, ids.data_ptr(), 300, table.data_ptr(), y.data_ptr(),
                       torch.cuda.current_stream().cuda_stream)
    assert torch.equal(y, emb(ids, table))
