"""The C ABI of the operators around the convolutions (huge2_train.h) on the CPU:
what is refused before any HIP call."""
import ctypes
import math
import os

import pytest

h2 = pytest.importorskip("paper_1907_11210_amd.huge2")
from paper_1907_11210_amd import train as tr  # noqa: E402

FAKE = 4096   # an aligned address that no refused call may touch
OTHER = 1 << 40


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(h2.LIB_PATH):
        from paper_1907_11210_amd import _build
        _build.build()
    return tr.lib()


def _norm(**kw):
    d = dict(n=2, c=12, h=5, w=7, groups=4, layout=h2.HUGE2_NHWC, dtype=h2.HUGE2_F32,
             activation=0, eps=1e-5)
    d.update(kw)
    return tr.NormDesc(**d)


def test_header_declares_what_is_bound(L):
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "include", "huge2_train.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    declared = set(re.findall(r"\b(huge2_\w+)\s*\(", text))
    assert declared == set(tr.EXPORTED)
    for name in declared:
        assert hasattr(L, name)


@pytest.mark.parametrize("kw", [
    dict(n=0), dict(c=0), dict(h=0), dict(w=-1), dict(groups=0), dict(groups=5), dict(groups=24),
    dict(layout=2), dict(dtype=2), dict(dtype=-1), dict(activation=4), dict(activation=-1),
    dict(eps=0.0), dict(eps=-1e-5), dict(eps=math.nan), dict(eps=math.inf)])
def test_norm_refuses_descriptors(L, kw):
    plan = ctypes.c_void_p(77)
    d = _norm(**kw)
    assert L.huge2_norm_plan_create(ctypes.byref(plan), ctypes.byref(d)) == h2.HUGE2_ERR_INVALID_ARG
    assert plan.value is None


@pytest.mark.parametrize("kw", [dict(h=1 << 16, w=1 << 15), dict(h=1 << 14, w=1 << 14, c=12),
                                dict(n=1 << 20, h=1 << 10, w=1 << 10)])
def test_norm_refuses_what_is_too_large(L, kw):
    plan = ctypes.c_void_p(77)
    d = _norm(**kw)
    assert L.huge2_norm_plan_create(ctypes.byref(plan), ctypes.byref(d)) == h2.HUGE2_ERR_UNSUPPORTED
    assert plan.value is None


def test_refuses_more_than_a_launch_takes(L):
    """2^32 threads: 64 and more for a group in NCHW, 8 for a row of a gradient's table."""
    plan = ctypes.c_void_p(77)
    d = _norm(n=1 << 21, c=64, groups=64, h=1, w=1, layout=h2.HUGE2_NCHW)
    assert L.huge2_norm_plan_create(ctypes.byref(plan), ctypes.byref(d)) == h2.HUGE2_ERR_UNSUPPORTED
    assert plan.value is None
    plan.value = 77
    d = tr.EmbeddingDesc((1 << 31) - 2, 1, h2.HUGE2_BF16, 64, 1.0)
    assert L.huge2_embedding_grad_plan_create(ctypes.byref(plan), ctypes.byref(d), 4) == \
        h2.HUGE2_ERR_UNSUPPORTED
    assert plan.value is None


def test_null_plans_and_pointers(L):
    d = _norm()
    inv = h2.HUGE2_ERR_INVALID_ARG
    plan = ctypes.c_void_p(77)
    assert L.huge2_norm_plan_create(None, ctypes.byref(d)) == inv
    assert L.huge2_norm_plan_create(ctypes.byref(plan), None) == inv
    assert L.huge2_norm_execute(None, FAKE, 0, 0, OTHER, 0, 0) == inv
    assert L.huge2_norm_grad_execute(None, FAKE, FAKE, FAKE, 0, 0, OTHER, 0, 0, 0) == inv
    assert L.huge2_norm_plan_kernel(None, 0) == b""
    assert L.huge2_embedding_grad_plan_kernel(None, 5) == b""
    assert L.huge2_norm_plan_destroy(None) == 0
    assert L.huge2_embedding_grad_plan_destroy(None) == 0
    assert L.huge2_adamw_plan_destroy(None) == 0
    assert L.huge2_embedding_grad_execute(None, FAKE, 1, FAKE, OTHER, 0) == inv
    o = tr.AdamWOptions(1e-3, 0.9, 0.999, 1e-8, 1)
    assert L.huge2_adamw_step(None, None, ctypes.byref(o), 0, 0) == inv


@pytest.mark.parametrize("kw", [dict(rows=0), dict(dim=0), dict(dtype=3), dict(id_bits=16)])
def test_embedding_refuses_descriptors(L, kw):
    f = dict(rows=10, dim=8, dtype=h2.HUGE2_F32, id_bits=64, scale=1.0)
    f.update(kw)
    d = tr.EmbeddingDesc(**f)
    assert L.huge2_embedding(ctypes.byref(d), FAKE, 4, OTHER, 2 * OTHER, 0) == \
        h2.HUGE2_ERR_INVALID_ARG
    plan = ctypes.c_void_p(77)
    assert L.huge2_embedding_grad_plan_create(ctypes.byref(plan), ctypes.byref(d), 4) == \
        h2.HUGE2_ERR_INVALID_ARG
    assert plan.value is None


def test_embedding_refuses_arguments(L):
    d = tr.EmbeddingDesc(10, 8, h2.HUGE2_F32, 64, 1.0)
    p = ctypes.byref(d)
    inv = h2.HUGE2_ERR_INVALID_ARG
    assert L.huge2_embedding(None, FAKE, 4, OTHER, 2 * OTHER, 0) == inv
    assert L.huge2_embedding(p, FAKE, -1, OTHER, 2 * OTHER, 0) == inv
    assert L.huge2_embedding(p, 0, 4, OTHER, 2 * OTHER, 0) == inv
    assert L.huge2_embedding(p, FAKE + 4, 4, OTHER, 2 * OTHER, 0) == inv   # int64 ids
    assert L.huge2_embedding(p, FAKE, 4, OTHER + 8, 2 * OTHER, 0) == inv
    assert L.huge2_embedding(p, FAKE, 4, OTHER, 2 * OTHER + 4, 0) == inv
    assert L.huge2_embedding(p, FAKE, 4, OTHER, OTHER + 64, 0) == inv      # overlaps the table
    assert L.huge2_embedding(p, FAKE, 4, OTHER, FAKE + 16, 0) == inv       # overlaps the ids
    assert L.huge2_embedding(p, FAKE, 1 << 31, OTHER, 2 * OTHER, 0) == h2.HUGE2_ERR_UNSUPPORTED
    assert L.huge2_embedding(p, 0, 0, 0, 0, 0) == 0                        # nothing to do
    plan = ctypes.c_void_p(77)
    assert L.huge2_embedding_grad_plan_create(ctypes.byref(plan), p, -1) == inv
    assert L.huge2_embedding_grad_plan_create(None, p, 4) == inv
    assert L.huge2_embedding_grad_plan_create(ctypes.byref(plan), p, 1 << 30) == \
        h2.HUGE2_ERR_UNSUPPORTED
    wide = tr.EmbeddingDesc(10, 1 << 30, h2.HUGE2_F32, 64, 1.0)
    assert L.huge2_embedding(ctypes.byref(wide), FAKE, 4, OTHER, 2 * OTHER, 0) == \
        h2.HUGE2_ERR_UNSUPPORTED


def _tensor(**kw):
    f = dict(param=FAKE, m=FAKE, v=FAKE, count=5, dtype=0, grad_dtype=0, weight_decay=0.0)
    f.update(kw)
    return tr.AdamWTensor(**f)


@pytest.mark.parametrize("bits,kw", [
    (16, {}), (32, dict(count=-1)), (32, dict(dtype=2)), (32, dict(grad_dtype=-1)),
    (32, dict(weight_decay=-0.1)), (32, dict(weight_decay=math.nan)), (32, dict(param=None)),
    (32, dict(m=None)), (32, dict(v=None)), (32, dict(param=FAKE + 4)), (32, dict(m=FAKE + 8)),
    (32, dict(copy=FAKE + 2)), (32, dict(m_scale=FAKE)), (8, {}), (8, dict(m_scale=FAKE)),
    (8, dict(m_scale=FAKE, v_scale=FAKE + 2))])
def test_adamw_refuses_tensors(L, bits, kw):
    plan = ctypes.c_void_p(77)
    t = _tensor(**kw)
    assert L.huge2_adamw_plan_create(ctypes.byref(plan), ctypes.byref(t), 1, bits, 0) == \
        h2.HUGE2_ERR_INVALID_ARG
    assert plan.value is None


def test_adamw_refuses_counts_and_options(L):
    plan = ctypes.c_void_p(77)
    t = _tensor()
    inv = h2.HUGE2_ERR_INVALID_ARG
    assert L.huge2_adamw_plan_create(ctypes.byref(plan), ctypes.byref(t), -1, 32, 0) == inv
    assert L.huge2_adamw_plan_create(ctypes.byref(plan), None, 1, 32, 0) == inv
    assert L.huge2_adamw_plan_create(None, ctypes.byref(t), 1, 32, 0) == inv
    big = _tensor(count=1 << 40)
    assert L.huge2_adamw_plan_create(ctypes.byref(plan), ctypes.byref(big), 1, 32, 0) == \
        h2.HUGE2_ERR_UNSUPPORTED
    # no tensors: a plan without device memory, whose step checks its options
    assert L.huge2_adamw_plan_create(ctypes.byref(plan), None, 0, 32, 0) == 0
    good = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
    o = tr.AdamWOptions(**good)
    assert L.huge2_adamw_step(plan, None, ctypes.byref(o), 0, 0) == 0
    assert L.huge2_adamw_step(plan, None, None, 0, 0) == inv
    assert L.huge2_adamw_step(plan, None, ctypes.byref(o), FAKE + 2, 0) == inv
    for kw in (dict(lr=-1.0), dict(lr=math.nan), dict(lr=1e300), dict(beta1=1.0),
               dict(beta1=-0.1), dict(beta2=math.nan), dict(beta2=1 - 1e-12), dict(eps=0.0),
               dict(eps=1e-60), dict(eps=math.inf), dict(step=0), dict(step=-3)):
        o = tr.AdamWOptions(**{**good, **kw})
        assert L.huge2_adamw_step(plan, None, ctypes.byref(o), 0, 0) == inv, kw
    assert L.huge2_adamw_plan_destroy(plan) == 0
