"""Descriptors of the training operators, and what the group norm's plans choose, on the CPU:
the library in a process of its own whose allocations are replaced (allocations.c)."""
import json
import os
import re
import subprocess
import sys

import pytest

h2 = pytest.importorskip("paper_1907_11210_amd.huge2")

HERE = os.path.dirname(os.path.abspath(__file__))

START = """
import ctypes, json, sys
ctypes.CDLL(sys.argv[1], ctypes.RTLD_GLOBAL)
from paper_1907_11210_amd import huge2 as h2, train as tr
"""
PLAN = START + """
names = []
for n, c, h, w, groups, layout, dtype in json.load(sys.stdin):
    desc = tr.NormDesc(n, c, h, w, groups, layout, dtype, 0, 1e-5)
    plan = tr.huge2_norm_plan_create(desc)
    names.append([tr.huge2_norm_plan_kernel(plan, grad) for grad in (False, True)])
    tr.huge2_norm_plan_destroy(plan)
json.dump(names, sys.stdout)
"""


@pytest.fixture(scope="module")
def script(tmp_path_factory):
    """Runs a script with the replaced allocations on a JSON input; its JSON output."""
    if not os.path.exists(h2.LIB_PATH):
        from paper_1907_11210_amd import _build
        _build.build()
    lib = str(tmp_path_factory.mktemp("plan") / "allocations.so")
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", lib, os.path.join(HERE, "allocations.c")],
                   check=True)

    def run(text, data):
        done = subprocess.run([sys.executable, "-c", text, lib], input=json.dumps(data), text=True,
                              capture_output=True, cwd=os.path.dirname(HERE), timeout=120)
        assert done.returncode == 0, done.stderr
        return json.loads(done.stdout)
    return run


@pytest.fixture(scope="module")
def kernels(script):
    """Names of the kernels, forward and gradient, for shapes (n, c, h, w, groups, layout, type)."""
    return lambda shapes: script(PLAN, shapes)


def _parse(name):
    """Kernel, and its numbers by their letters."""
    kernel, *fields = name.split()
    return kernel, {f[0]: int(f[1:]) for f in fields}


@pytest.mark.parametrize("layout", [h2.HUGE2_NHWC, h2.HUGE2_NCHW], ids=["nhwc", "nchw"])
@pytest.mark.parametrize("dtype", [h2.HUGE2_F32, h2.HUGE2_BF16], ids=["f32", "bf16"])
def test_maps_of_almost_2_to_the_31(kernels, layout, dtype):
    """No rounding up of a map's pixels passes 32 bits: such a map is cut into runs."""
    sides = [(1, 1, 2 ** 31 - k) for k in (1, 2, 4, 8, 64, 512, 1022, 1024, 1025)]
    sides += [(1, 2 ** 31 - 1, 1), (2, 1, 2 ** 30 - 1), (8, 16384, 16383)]
    shapes = [(1, c, h, w, 1, layout, dtype) for c, h, w in sides]
    for shape, names in zip(shapes, kernels(shapes)):
        for name in names:
            kernel, number = _parse(name)
            assert kernel.startswith(("norm_run", "norm_sums")), (shape, name)
            assert 64 <= number["k"] < 2 ** 31, (shape, name)


def test_slabs_hold_their_maps(kernels):
    """A slab's threads and their vectors cover a group's pixels, at most 16 vectors each."""
    shapes = [(n, c, h, w, g, layout, dtype)
              for n, c, h, w, g in ((1, 1, 1, 1, 1), (3, 24, 6, 6, 6), (64, 256, 16, 16, 32),
                                    (64, 64, 64, 64, 16), (2, 32, 16, 16, 4), (1, 512, 8, 8, 32),
                                    (300, 200, 11, 9, 8), (1, 1, 1, 16384, 1), (9, 8, 1, 1025, 4))
              for layout in (h2.HUGE2_NHWC, h2.HUGE2_NCHW)
              for dtype in (h2.HUGE2_F32, h2.HUGE2_BF16)]
    slabs = 0
    for shape, names in zip(shapes, kernels(shapes)):
        for name in names:
            kernel, number = _parse(name)
            if not re.match("norm_slab", kernel):
                continue
            slabs += 1
            _, c, h, w, g, layout, _ = shape
            assert 1 <= number["r"] <= 16 and 64 <= number["t"] <= 1024, (shape, name)
            held = number["v"] * number["t"] * number["r"]
            assert held >= h * w * (c // g), (shape, name)
    assert slabs >= 40


def test_sizes_that_32_bits_do_not_hold():
    """They are refused, not cut to their low bits: a table of 2^32 + 8 rows is none of 8."""
    from paper_1907_11210_amd import train as tr
    norm = dict(n=2, c=12, h=5, w=7, groups=4, layout=h2.HUGE2_NHWC, dtype=h2.HUGE2_F32,
                activation=0, eps=1e-5)
    assert tr.NormDesc(**norm).w == 7 and tr.NormDesc(2, 12, -1).h == -1
    for field in ("n", "c", "h", "w", "groups"):
        for value in (2 ** 32 + norm[field], 2 ** 31, -2 ** 31 - 1):
            with pytest.raises(ValueError, match=field):
                tr.NormDesc(**{**norm, field: value})
    with pytest.raises(ValueError, match="n is"):
        tr.NormDesc(2 ** 32 + 2, 12, 5, 7, 4, h2.HUGE2_NHWC, h2.HUGE2_F32, 0, 1e-5)
    for rows, dim in ((2 ** 32 + 8, 16), (8, 2 ** 32 + 16)):
        with pytest.raises(ValueError):
            tr.EmbeddingDesc(rows, dim, h2.HUGE2_BF16, 64, 1.0)


# Calls on made-up addresses, which are refused before anything is enqueued; their statuses.
CALLS = START + """
L = tr.lib()
desc = tr.NormDesc(2, 12, 5, 7, 4, h2.HUGE2_NHWC, h2.HUGE2_F32, 0, 1e-5)
norm = tr.huge2_norm_plan_create(desc)
done = []
for name, args in json.load(sys.stdin):
    if name == "adamw":
        tensors, bits, grads, scale = args
        plan, o = ctypes.c_void_p(), tr.AdamWOptions(1e-3, 0.9, 0.999, 1e-8, 1)
        ts = (tr.AdamWTensor * len(tensors))(*(tr.AdamWTensor(**t) for t in tensors))
        status = L.huge2_adamw_plan_create(ctypes.byref(plan), ts, len(tensors), bits, 0)
        if grads is not None:
            assert status == 0
            g = (ctypes.c_void_p * len(grads))(*grads)
            status = L.huge2_adamw_step(plan, g, ctypes.byref(o), scale, 0)
        done.append(status)
    else:
        done.append(getattr(L, name)(norm, *args, 0))
json.dump(done, sys.stdout)
"""
K = 1 << 20  # farther apart than any of the arrays is long


def test_norm_refuses_overlaps(script):
    """Nothing that a call writes overlaps what it reads or writes beside it.  x, dy and dx take
    3360 bytes, gamma, beta and their gradients 48, statistics 64."""
    x, ga, be, y, st, dy, dg, db = (K * i for i in range(1, 9))
    forward, grad = "huge2_norm_execute", "huge2_norm_grad_execute"
    calls = [(forward, [x, ga, be, to, st]) for to in (x, x + 3344, x - 3344, ga - 16, be + 32, st)]
    calls += [(forward, [x, ga, be, y, to]) for to in (x + 16, y + 3344, ga, be - 48)]
    calls += [(grad, [x, dy, st, ga, be, to, dg, db])
              for to in (x, x + 3344, dy, dy - 3344, st + 48, ga, be, dg, db - 16)]
    calls += [(grad, [x, dy, st, ga, be, y, to, db])
              for to in (x + 4, dy + 3356, y, st + 60, ga, be + 4, db, db - 44, db + 44)]
    calls += [(grad, [x, dy, st, ga, be, y, dg, to]) for to in (x, dy, y + 100, st, ga - 44, be)]
    assert script(CALLS, calls) == [h2.HUGE2_ERR_INVALID_ARG] * len(calls)


def test_adamw_refuses_overlaps(script):
    """Parameters, states, scales and copies are each one tensor's own (a tied parameter is
    listed once), and no gradient lies in them."""
    def tensor(i, bits, **kw):
        at = K * (8 * i + 1)
        t = dict(param=at, m=at + K, v=at + 2 * K, copy=at + 3 * K, count=1000)
        if bits == 8:
            t.update(m_scale=at + 4 * K, v_scale=at + 5 * K)
        return dict(t, **kw)

    good, refused = [], []
    for bits in (32, 8):
        state = 1000 * (bits // 8)
        a, b = tensor(0, bits), tensor(1, bits)
        grads = [64 * K, 65 * K]
        good += [("adamw", [[a, b], bits, None, 0]),
                 ("adamw", [[a, tensor(1, bits, count=0, param=a["param"])], bits, None, 0]),
                 # one behind the other, to the byte (rounded up to 16)
                 ("adamw", [[tensor(0, bits, m=a["v"] - (state + 15) // 16 * 16)], bits, None, 0])]
        for kw in (dict(m=a["param"]), dict(v=a["m"]), dict(copy=a["param"] + 3984),
                   dict(copy=a["v"]), dict(param=a["m"] - 3984), dict(m=a["v"] - (state - 1) // 16 * 16)):
            refused.append(("adamw", [[dict(a, **kw)], bits, None, 0]))
        refused += [("adamw", [[a, a], bits, None, 0]), ("adamw", [[a, b, a], bits, None, 0]),
                    ("adamw", [[a, dict(b, v=a["copy"])], bits, None, 0])]
        if bits == 8:
            refused += [("adamw", [[dict(a, m_scale=a["v_scale"] + 12)], bits, None, 0]),
                        ("adamw", [[a, dict(b, v_scale=a["param"] + 4)], bits, None, 0])]
        for t in (a, b):
            for field in ("param", "m", "v", "copy") + (("m_scale", "v_scale") if bits == 8 else ()):
                refused += [("adamw", [[a, b], bits, [t[field], grads[1]], 0]),
                            ("adamw", [[a, b], bits, [grads[0], t[field] - 3984], 0]),
                            ("adamw", [[a, b], bits, grads, t[field] + 4])]
    assert script(CALLS, good) == [h2.HUGE2_OK] * len(good)
    assert script(CALLS, refused) == [h2.HUGE2_ERR_INVALID_ARG] * len(refused)
