"""Layer norm's C ABI on the CPU: what is refused before any HIP call, and what plans choose (in
a process whose allocations are replaced, as in test_train_plan.py)."""
import ctypes
import math

import pytest

h2 = pytest.importorskip("paper_1907_11210_amd.huge2")
from paper_1907_11210_amd import train as tr  # noqa: E402
from test_train_plan import K, START, script  # noqa: E402, F401

FAKE, OTHER = 4096, 1 << 40


def _desc(**kw):
    d = dict(n=2, c=12, h=5, w=7, layout=h2.HUGE2_NHWC, dtype=h2.HUGE2_F32, activation=0, eps=1e-5)
    d.update(kw)
    return tr.LayerNormDesc(**d)


def _create(**kw):
    plan, d = ctypes.c_void_p(77), _desc(**kw)
    status = tr.lib().huge2_layer_norm_plan_create(ctypes.byref(plan), ctypes.byref(d))
    assert plan.value is None
    return status


@pytest.mark.parametrize("kw", [
    dict(n=0), dict(c=0), dict(h=0), dict(w=-1), dict(layout=2), dict(dtype=2), dict(dtype=-1),
    dict(activation=4), dict(activation=-1), dict(eps=0.0), dict(eps=-1e-5), dict(eps=math.nan),
    dict(eps=math.inf)])
def test_refuses_descriptors(kw):
    assert _create(**kw) == h2.HUGE2_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [
    dict(h=1 << 16, w=1 << 15), dict(h=1 << 14, w=1 << 14, c=12),
    dict(n=1 << 20, h=1 << 10, w=1 << 10),
    dict(n=(1 << 31) - 1, c=1, h=1, w=65, layout=h2.HUGE2_NCHW),
    dict(n=1, c=1 << 26, h=1, w=1), dict(n=1, c=1 << 24, h=1, w=2, layout=h2.HUGE2_NCHW)])
def test_refuses_what_is_too_large(kw):
    assert _create(**kw) == h2.HUGE2_ERR_UNSUPPORTED


def test_null_plans_and_pointers():
    L, inv, d = tr.lib(), h2.HUGE2_ERR_INVALID_ARG, _desc()
    plan = ctypes.c_void_p(77)
    assert L.huge2_layer_norm_plan_create(None, ctypes.byref(d)) == inv
    assert L.huge2_layer_norm_plan_create(ctypes.byref(plan), None) == inv
    assert L.huge2_layer_norm_execute(None, FAKE, 0, 0, OTHER, 0, 0) == inv
    assert L.huge2_layer_norm_grad_execute(None, FAKE, FAKE, FAKE, 0, 0, OTHER, 0, 0, 0) == inv
    assert L.huge2_layer_norm_plan_kernel(None, 0) == b""
    assert L.huge2_layer_norm_plan_destroy(None) == 0


CALLS = START + """
L = tr.lib()
plan = tr.huge2_layer_norm_plan_create(
    tr.LayerNormDesc(2, 12, 5, 7, h2.HUGE2_NHWC, h2.HUGE2_F32, 0, 1e-5))
json.dump([getattr(L, name)(plan, *args, 0) for name, args in json.load(sys.stdin)], sys.stdout)
"""
FORWARD, GRAD = "huge2_layer_norm_execute", "huge2_layer_norm_grad_execute"


def test_refuses_pointers_and_overlaps(script):  # noqa: F811
    """Nothing that a call writes overlaps what it reads or writes beside it.  x, dy and dx take
    3360 bytes, gamma, beta and their gradients 48, statistics 560."""
    x, ga, be, y, st, dy, dg, db = (K * i for i in range(1, 9))
    calls = [(FORWARD, [x, ga, be, to, st]) for to in (x, x + 3344, x - 3344, ga - 16, be + 32, st)]
    calls += [(FORWARD, [x, ga, be, y, to]) for to in (x + 16, y + 3344, ga, be - 48, x - 544)]
    calls += [(GRAD, [x, dy, st, ga, be, to, dg, db])
              for to in (x, x + 3344, dy, dy - 3344, st + 544, ga, be, dg, db - 16)]
    calls += [(GRAD, [x, dy, st, ga, be, y, to, db])
              for to in (x + 4, dy + 3356, y, st + 556, ga, be + 4, db, db - 44, db + 44)]
    calls += [(GRAD, [x, dy, st, ga, be, y, dg, to]) for to in (x, dy, y + 100, st, ga - 44, be)]
    calls += [(FORWARD, args) for args in ([0, ga, be, y, st], [x, ga, be, 0, st],
                                           [x + 8, ga, be, y, st], [x, ga + 4, be, y, st],
                                           [x, ga, be + 8, y, st], [x, ga, be, y + 4, st],
                                           [x, ga, be, y, st + 8])]
    calls += [(GRAD, args) for args in ([0, dy, st, ga, be, y, dg, db], [x, 0, st, ga, be, y, dg, db],
                                        [x, dy, 0, ga, be, y, dg, db], [x, dy, st, ga, be, 0, dg, db],
                                        [x, dy, st, ga, be, y, dg + 2, db],
                                        [x, dy, st, ga, be, y, dg, db + 1])]
    assert script(CALLS, calls) == [h2.HUGE2_ERR_INVALID_ARG] * len(calls)


NAMES = START + """
names = []
for n, c, h, w, layout, dtype in json.load(sys.stdin):
    plan = tr.huge2_layer_norm_plan_create(tr.LayerNormDesc(n, c, h, w, layout, dtype, 0, 1e-5))
    names.append([tr.huge2_layer_norm_plan_kernel(plan, grad) for grad in (False, True)])
    tr.huge2_layer_norm_plan_destroy(plan)
json.dump(names, sys.stdout)
"""


def test_held_values_cover_a_pixel(script):  # noqa: F811
    """Where a row's or a tile's channels are held, threads times vectors are enough for them, and
    no workgroup is larger than its kernel's registers allow."""
    shapes = [(n, c, h, w, layout, dtype)
              for n in (1, 3, 70, 100000)
              for c in (1, 2, 7, 8, 9, 63, 64, 100, 512, 513, 1000, 1024, 2047, 2048, 2049, 4095,
                        4104, 8192, 8193, 16384, 16385, 32768, 32769, 70001)
              for h, w in ((1, 1), (1, 3), (1, 8), (3, 3), (8, 8), (17, 31))
              for layout in (h2.HUGE2_NHWC, h2.HUGE2_NCHW)
              for dtype in (h2.HUGE2_F32, h2.HUGE2_BF16) if n * c * h * w < 1 << 34]
    held = 0
    for shape, names in zip(shapes, script(NAMES, shapes)):
        _, c, h, w, layout, _ = shape
        for grad, name in enumerate(names):
            kernel, *fields = name.split()
            v, t, r = (int(f[1:]) for f in fields)
            assert 64 <= t <= 1024 and t & (t - 1) == 0, (shape, name)
            if "rows" in kernel:
                held += 1
                assert v * t * r >= c and v * r <= (16 if grad or c > 2048 else 32), (shape, name)
                assert v == 1 or c >= v, (shape, name)
            elif "planes" in kernel:
                assert v == 1 or h * w >= v, (shape, name)
                if r:
                    held += 1
                    assert t * r >= c, (shape, name)
                    assert r <= (16 if not grad else 8 if t <= 512 else min(8, 16 // v)), (shape, name)
            else:
                assert c > 16384, (shape, name)
    assert held > len(shapes)


def test_sizes_that_32_bits_do_not_hold():
    for field in ("n", "c", "h", "w"):
        for value in (2 ** 32 + 2, 2 ** 31, -2 ** 31 - 1):
            with pytest.raises(ValueError, match=field):
                _desc(**{field: value})


STATUS = START + """
done = []
for n, c, h, w, layout, dtype in json.load(sys.stdin):
    plan, d = ctypes.c_void_p(), tr.LayerNormDesc(n, c, h, w, layout, dtype, 0, 1e-5)
    done.append(tr.lib().huge2_layer_norm_plan_create(ctypes.byref(plan), ctypes.byref(d)))
    tr.huge2_layer_norm_plan_destroy(plan)
json.dump(done, sys.stdout)
"""


def test_the_largest_that_fits(script):  # noqa: F811
    """The limits that the header gives, from both sides: in NCHW below 2^24 channels and 2^31
    pieces of 128 bytes of the images' planes, else below 2^26 - 16 channels; 2^40 elements."""
    nchw, nhwc, f32, bf16 = h2.HUGE2_NCHW, h2.HUGE2_NHWC, h2.HUGE2_F32, h2.HUGE2_BF16
    inside, outside = [], []
    for dtype, piece in ((f32, 32), (bf16, 64)):  # pixels of 128 bytes
        for hw in (1, 2, 3, 7, piece - 1, piece, piece + 1, 2 * piece, 2 * piece + 1, 10 * piece - 1,
                   997 * piece + 1, (1 << 20) - 1):
            pieces = -(-hw // piece)
            most = min(((1 << 31) - 1) // pieces, ((1 << 40) - 1) // hw)
            inside.append((most, 1, 1, hw, nchw, dtype))
            if most < (1 << 31) - 1:
                outside.append((most + 1, 1, 1, hw, nchw, dtype))
        inside += [(1 << 20, 1, 1 << 9, (1 << 11) - 1, nhwc, dtype),
                   ((1 << 31) - 1, 2, 1, 1, nhwc, dtype), (1, (1 << 24) - 1, 2, 63, nchw, dtype)]
        outside += [(1, 1 << 24, 1, 2, nchw, dtype), (1 << 20, 1, 1 << 10, 1 << 10, nhwc, dtype)]
        for layout in (nchw, nhwc):
            inside.append((1, (1 << 26) - 17, 1, 1, layout, dtype))
            outside.append((1, (1 << 26) - 16, 1, 1, layout, dtype))
    assert script(STATUS, inside) == [h2.HUGE2_OK] * len(inside)
    assert script(STATUS, outside) == [h2.HUGE2_ERR_UNSUPPORTED] * len(outside)
