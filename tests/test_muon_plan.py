"""The C ABI of orthogonalised matrices and the Muon step on the CPU: what is refused before any
HIP call, and what in a process whose allocations are replaced."""
import ctypes
import math

import pytest

h2 = pytest.importorskip("paper_1907_11210_amd.huge2")
from paper_1907_11210_amd import train as tr  # noqa: E402
from test_train_plan import K, START, script  # noqa: E402, F401

INV, TOO_LARGE = h2.HUGE2_ERR_INVALID_ARG, h2.HUGE2_ERR_UNSUPPORTED
FAKE, OTHER = 4096, 1 << 40


def _create(desc, ns):
    plan = ctypes.c_void_p(77)
    status = tr.lib().huge2_orthogonalize_plan_create(ctypes.byref(plan), ctypes.byref(desc),
                                                      ctypes.byref(ns), 0)
    assert plan.value is None
    return status


@pytest.mark.parametrize("kw", [dict(batch=0), dict(rows=0), dict(cols=-1), dict(dtype=2)])
def test_refuses_descriptors(kw):
    d = tr.OrthogonalizeDesc(**{**dict(batch=1, rows=4, cols=5, dtype=0), **kw})
    assert _create(d, tr.newton_schulz()) == INV


@pytest.mark.parametrize("sizes", [(1, 1 << 16, 1 << 15), (1, 1, (1 << 31) - 1), (1 << 21, 2, 2),
                                   (1, (1 << 28) + 1, 2), (1 << 20, 1 << 11, 1 << 10)])
def test_refuses_what_is_too_large(sizes):
    assert _create(tr.OrthogonalizeDesc(*sizes, 0), tr.newton_schulz()) == TOO_LARGE


@pytest.mark.parametrize("kw", [
    dict(eps=0.0), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf),
    dict(coefficients=(math.nan, 0, 0)), dict(coefficients=(1, math.inf, 0)),
    dict(coefficients=(1030.0, 0, 0)), dict(coefficients=(1, 2.0 ** 30, 0)),
    dict(coefficients=(1, 0, -2.0 ** 40)),
    # 1 goes to 2.2, that to 6.2, that to some 4000
    dict(coefficients=[(8.2, -23.0, 17.0), (4.0, -2.9, 0.55), (3.9, -2.8, 0.53)], steps=3), dict(coefficients=(11.0, 0, 0), steps=3)])
def test_refuses_polynomials(kw):
    assert _create(tr.OrthogonalizeDesc(1, 4, 5, 0), tr.newton_schulz(**kw)) == INV


@pytest.mark.parametrize("field,value", [("steps", 0), ("steps", 33), ("products", 2),
                                         ("products", -1), ("coefficients", None)])
def test_refuses_fields(field, value):
    ns = tr.newton_schulz()
    setattr(ns, field, value)
    assert _create(tr.OrthogonalizeDesc(1, 4, 5, 0), ns) == INV


def test_null_plans_and_pointers():
    L, ns = tr.lib(), tr.newton_schulz()
    d, plan = tr.OrthogonalizeDesc(1, 4, 5, 0), ctypes.c_void_p(77)
    assert L.huge2_orthogonalize_plan_create(None, ctypes.byref(d), ctypes.byref(ns), 0) == INV
    assert L.huge2_orthogonalize_plan_create(ctypes.byref(plan), None, ctypes.byref(ns), 0) == INV
    assert L.huge2_orthogonalize_plan_create(ctypes.byref(plan), ctypes.byref(d), None, 0) == INV
    assert L.huge2_orthogonalize_execute(None, FAKE, OTHER, 0) == INV
    assert L.huge2_orthogonalize_plan_destroy(None) == 0
    o = tr.MuonOptions(0.1, 0.9, 1)
    assert L.huge2_muon_plan_create(None, None, 0, ctypes.byref(ns), 0) == INV
    assert L.huge2_muon_plan_create(ctypes.byref(plan), None, 1, ctypes.byref(ns), 0) == INV
    assert L.huge2_muon_plan_create(ctypes.byref(plan), None, -1, ctypes.byref(ns), 0) == INV
    assert L.huge2_muon_plan_create(ctypes.byref(plan), None, 0, None, 0) == INV
    assert L.huge2_muon_step(None, None, ctypes.byref(o), 0, 0) == INV
    assert L.huge2_muon_plan_destroy(None) == 0
    # no matrices: a plan without device memory, whose step checks its options
    assert L.huge2_muon_plan_create(ctypes.byref(plan), None, 0, ctypes.byref(ns), 0) == 0
    assert L.huge2_muon_step(plan, None, ctypes.byref(o), 0, 0) == 0
    assert L.huge2_muon_step(plan, None, None, 0, 0) == INV
    assert L.huge2_muon_step(plan, None, ctypes.byref(o), FAKE + 2, 0) == INV
    for bad in ((-0.1, 0.9), (math.nan, 0.9), (1e300, 0.9), (0.1, 1.0), (0.1, -0.1),
                (0.1, math.nan), (0.1, 1 - 1e-12)):
        o = tr.MuonOptions(*bad, 1)
        assert L.huge2_muon_step(plan, None, ctypes.byref(o), 0, 0) == INV, bad
    assert L.huge2_muon_plan_destroy(plan) == 0


@pytest.mark.parametrize("kw", [
    dict(rows=0), dict(cols=0), dict(dtype=2), dict(grad_dtype=-1), dict(weight_decay=-0.1),
    dict(weight_decay=math.nan), dict(scale=math.inf), dict(param=None), dict(m=None),
    dict(param=FAKE + 4), dict(m=OTHER + 8), dict(copy=FAKE + 2)])
def test_muon_refuses_tensors(kw):
    f = dict(param=FAKE, m=OTHER, rows=4, cols=5, dtype=0, grad_dtype=0, scale=1.0)
    t, plan, ns = tr.MuonTensor(**{**f, **kw}), ctypes.c_void_p(77), tr.newton_schulz()
    assert tr.lib().huge2_muon_plan_create(ctypes.byref(plan), ctypes.byref(t), 1, ctypes.byref(ns),
                                           0) == INV
    assert plan.value is None


def test_muon_refuses_what_is_too_large():
    t = tr.MuonTensor(param=FAKE, m=OTHER, rows=1 << 16, cols=1 << 15, scale=1.0)
    plan, ns = ctypes.c_void_p(77), tr.newton_schulz()
    assert tr.lib().huge2_muon_plan_create(ctypes.byref(plan), ctypes.byref(t), 1, ctypes.byref(ns),
                                           0) == TOO_LARGE


CALLS = START + """
L = tr.lib()
ns = tr.newton_schulz()
plan = tr.huge2_orthogonalize_plan_create(tr.OrthogonalizeDesc(3, 10, 14, 0), ns)
done = []
for name, args in json.load(sys.stdin):
    if name == "orthogonalize":
        done.append(L.huge2_orthogonalize_execute(plan, *args, 0))
        continue
    tensors, grads, scale = args
    muon, o = ctypes.c_void_p(), tr.MuonOptions(0.1, 0.9, 1)
    ts = (tr.MuonTensor * len(tensors))(*(tr.MuonTensor(**t) for t in tensors))
    status = L.huge2_muon_plan_create(ctypes.byref(muon), ts, len(tensors), ctypes.byref(ns), 0)
    if grads is not None:
        assert status == 0
        g = (ctypes.c_void_p * len(grads))(*grads)
        status = L.huge2_muon_step(muon, g, ctypes.byref(o), scale, 0)
    done.append(status)
json.dump(done, sys.stdout)
"""


def test_refuses_overlaps(script):  # noqa: F811
    """Nothing that a call writes overlaps what it reads or writes beside it."""
    def tensor(i, **kw):
        at = K * (4 * i + 1)
        return dict(dict(param=at, m=at + K, copy=at + 2 * K, rows=25, cols=40, scale=1.0), **kw)

    a, b = tensor(0), tensor(1)
    good = [("muon", [[a, b], None, 0]), ("muon", [[dict(a, copy=a["param"] + 4000)], None, 0])]
    calls = [("orthogonalize", [K, K + d]) for d in (0, 1664, -1664)]
    calls += [("orthogonalize", p) for p in ([0, K], [K, 0], [K + 8, 3 * K], [K, 3 * K + 4])]
    for kw in (dict(m=a["param"]), dict(copy=a["m"] + 3984), dict(param=a["m"] - 3984)):
        calls.append(("muon", [[dict(a, **kw)], None, 0]))
    calls += [("muon", [[a, a], None, 0]), ("muon", [[a, dict(b, m=a["copy"])], None, 0])]
    grads = [64 * K, 65 * K]
    for t in (a, b):
        for field in ("param", "m", "copy"):
            calls += [("muon", [[a, b], [t[field], grads[1]], 0]),
                      ("muon", [[a, b], [grads[0], t[field] - 3984], 0]),
                      ("muon", [[a, b], grads, t[field] + 4])]
    calls.append(("muon", [[a, b], [grads[0] + 8, grads[1]], 0]))
    assert script(CALLS, good) == [h2.HUGE2_OK] * len(good)
    assert script(CALLS, calls) == [INV] * len(calls)


def test_sizes_that_32_bits_do_not_hold():
    for field in ("batch", "rows", "cols"):
        with pytest.raises(ValueError, match=field):
            tr.OrthogonalizeDesc(**{**dict(batch=1, rows=2, cols=3, dtype=0), field: 2 ** 32 + 2})
    with pytest.raises(ValueError, match="rows"):
        tr.MuonTensor(param=FAKE, m=OTHER, rows=2 ** 32 + 4, cols=5)
