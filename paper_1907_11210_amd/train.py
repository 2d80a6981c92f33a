"""Python binding of the operators around the convolutions (the C ABI in
include/huge2_train.h): group norm and layer norm with an activation, embedding
lookup and the AdamW step, with their gradients; orthogonalised matrices and the Muon step.

Argument marshalling only, as in :mod:`paper_1907_11210_amd.huge2`: the ``huge2_*``
functions mirror the C entry points and take raw device pointers (ints);
:class:`GroupNorm`, :class:`LayerNorm`, :class:`Embedding`, :class:`AdamW`,
:class:`Orthogonalize` and :class:`Muon` take torch tensors and enqueue on the
current stream.  Objects belong to the device that was current when they were made;
one object's calls share its workspace, so make them on one stream or order them.
"""
from __future__ import annotations

import array
import ctypes
import math

from . import huge2 as h2

PRODUCTS = {"f32": 0, "f16": 1}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)  # of a Newton-Schulz step
NORM_ACTIVATIONS = {None: 0, "none": 0, "relu": 1, "tanh": 2, "silu": 3}
STATE_BLOCK = 256  # elements that share a scale in 8-bit states

EXPORTED = (
    "huge2_norm_plan_create", "huge2_norm_execute", "huge2_norm_grad_execute",
    "huge2_norm_plan_kernel", "huge2_norm_plan_destroy",
    "huge2_layer_norm_plan_create", "huge2_layer_norm_execute", "huge2_layer_norm_grad_execute",
    "huge2_layer_norm_plan_kernel", "huge2_layer_norm_plan_destroy",
    "huge2_embedding", "huge2_embedding_grad_plan_create", "huge2_embedding_grad_execute",
    "huge2_embedding_grad_plan_kernel", "huge2_embedding_grad_plan_destroy",
    "huge2_adamw_plan_create", "huge2_adamw_step", "huge2_adamw_plan_destroy",
    "huge2_orthogonalize_plan_create", "huge2_orthogonalize_execute",
    "huge2_orthogonalize_plan_destroy",
    "huge2_muon_plan_create", "huge2_muon_step", "huge2_muon_plan_destroy",
)


class _Desc(ctypes.Structure):
    """A descriptor whose whole numbers fit their fields (ctypes itself keeps the low bits)."""

    def __init__(self, *args, **kw):
        super().__init__(*args, **kw)
        given = dict(zip((f for f, _ in self._fields_), args), **kw)
        for name, kind in self._fields_:
            if kind is ctypes.c_int32 and getattr(self, name) != given.get(name, 0):
                raise ValueError("%s is %s, which 32 bits do not hold" % (name, given[name]))


class NormDesc(_Desc):
    _fields_ = [(f, ctypes.c_int32) for f in ("n", "c", "h", "w", "groups", "layout", "dtype",
                                              "activation")] + [("eps", ctypes.c_float)]


class LayerNormDesc(_Desc):
    _fields_ = [(f, ctypes.c_int32) for f in ("n", "c", "h", "w", "layout", "dtype",
                                              "activation")] + [("eps", ctypes.c_float)]


class EmbeddingDesc(_Desc):
    _fields_ = [(f, ctypes.c_int32) for f in ("rows", "dim", "dtype", "id_bits")] + \
        [("scale", ctypes.c_float)]


class AdamWTensor(ctypes.Structure):
    _fields_ = [(f, ctypes.c_void_p) for f in ("param", "m", "v", "m_scale", "v_scale", "copy")] + \
        [("count", ctypes.c_int64), ("dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32),
         ("weight_decay", ctypes.c_float)]


class AdamWOptions(ctypes.Structure):
    _fields_ = [(f, ctypes.c_double) for f in ("lr", "beta1", "beta2", "eps")] + \
        [("step", ctypes.c_int64)]


class NewtonSchulz(ctypes.Structure):
    _fields_ = [("steps", ctypes.c_int32), ("products", ctypes.c_int32),
                ("coefficients", ctypes.POINTER(ctypes.c_double)), ("eps", ctypes.c_double)]


class OrthogonalizeDesc(_Desc):
    _fields_ = [(f, ctypes.c_int32) for f in ("batch", "rows", "cols", "dtype")]


class MuonTensor(_Desc):
    _fields_ = [(f, ctypes.c_void_p) for f in ("param", "m", "copy")] + \
        [(f, ctypes.c_int32) for f in ("rows", "cols", "dtype", "grad_dtype")] + \
        [("weight_decay", ctypes.c_float), ("scale", ctypes.c_float)]


class MuonOptions(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("momentum", ctypes.c_double),
                ("nesterov", ctypes.c_int32)]


_lib = None


def lib():
    """The loaded libhuge2.so with these entry points' types; raises if it is not built."""
    global _lib
    if _lib is None:
        L = h2.lib()
        vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
        out = ctypes.POINTER(vp)
        types = {
            "huge2_norm_plan_create": [out, ctypes.POINTER(NormDesc)],
            "huge2_norm_execute": [vp] * 7,
            "huge2_norm_grad_execute": [vp] * 10,
            "huge2_norm_plan_kernel": [vp, i32],
            "huge2_norm_plan_destroy": [vp],
            "huge2_layer_norm_plan_create": [out, ctypes.POINTER(LayerNormDesc)],
            "huge2_layer_norm_execute": [vp] * 7,
            "huge2_layer_norm_grad_execute": [vp] * 10,
            "huge2_layer_norm_plan_kernel": [vp, i32],
            "huge2_layer_norm_plan_destroy": [vp],
            "huge2_embedding": [ctypes.POINTER(EmbeddingDesc), vp, i64, vp, vp, vp],
            "huge2_embedding_grad_plan_create": [out, ctypes.POINTER(EmbeddingDesc), i64],
            "huge2_embedding_grad_execute": [vp, vp, i64, vp, vp, vp],
            "huge2_embedding_grad_plan_kernel": [vp, i64],
            "huge2_embedding_grad_plan_destroy": [vp],
            "huge2_adamw_plan_create": [out, ctypes.POINTER(AdamWTensor), i32, i32, vp],
            "huge2_adamw_step": [vp, vp, ctypes.POINTER(AdamWOptions), vp, vp],
            "huge2_adamw_plan_destroy": [vp],
            "huge2_orthogonalize_plan_create": [out, ctypes.POINTER(OrthogonalizeDesc),
                                                ctypes.POINTER(NewtonSchulz), vp],
            "huge2_orthogonalize_execute": [vp] * 4,
            "huge2_orthogonalize_plan_destroy": [vp],
            "huge2_muon_plan_create": [out, ctypes.POINTER(MuonTensor), i32,
                                       ctypes.POINTER(NewtonSchulz), vp],
            "huge2_muon_step": [vp, vp, ctypes.POINTER(MuonOptions), vp, vp],
            "huge2_muon_plan_destroy": [vp],
        }
        for name in EXPORTED:
            fn = getattr(L, name)
            fn.argtypes = types[name]
            fn.restype = ctypes.c_char_p if name.endswith("_kernel") else ctypes.c_int
        _lib = L
    return _lib


# ---- the C entry points ---------------------------------------------------

def huge2_norm_plan_create(desc):
    plan = ctypes.c_void_p()
    h2._check(lib().huge2_norm_plan_create(ctypes.byref(plan), ctypes.byref(desc)),
              "huge2_norm_plan_create")
    return plan


def huge2_norm_execute(plan, x_ptr, gamma_ptr, beta_ptr, y_ptr, stats_ptr=0, stream=0):
    h2._check(lib().huge2_norm_execute(plan, x_ptr, gamma_ptr, beta_ptr, y_ptr, stats_ptr, stream),
              "huge2_norm_execute")


def huge2_norm_grad_execute(plan, x_ptr, dy_ptr, stats_ptr, gamma_ptr, beta_ptr, dx_ptr,
                            dgamma_ptr=0, dbeta_ptr=0, stream=0):
    h2._check(lib().huge2_norm_grad_execute(plan, x_ptr, dy_ptr, stats_ptr, gamma_ptr, beta_ptr,
                                            dx_ptr, dgamma_ptr, dbeta_ptr, stream),
              "huge2_norm_grad_execute")


def huge2_norm_plan_kernel(plan, grad=False):
    return lib().huge2_norm_plan_kernel(plan, int(grad)).decode()


def huge2_norm_plan_destroy(plan):
    h2._check(lib().huge2_norm_plan_destroy(plan), "huge2_norm_plan_destroy")


def huge2_layer_norm_plan_create(desc):
    plan = ctypes.c_void_p()
    h2._check(lib().huge2_layer_norm_plan_create(ctypes.byref(plan), ctypes.byref(desc)),
              "huge2_layer_norm_plan_create")
    return plan


def huge2_layer_norm_execute(plan, x_ptr, gamma_ptr, beta_ptr, y_ptr, stats_ptr=0, stream=0):
    h2._check(lib().huge2_layer_norm_execute(plan, x_ptr, gamma_ptr, beta_ptr, y_ptr, stats_ptr,
                                             stream), "huge2_layer_norm_execute")


def huge2_layer_norm_grad_execute(plan, x_ptr, dy_ptr, stats_ptr, gamma_ptr, beta_ptr, dx_ptr,
                                  dgamma_ptr=0, dbeta_ptr=0, stream=0):
    h2._check(lib().huge2_layer_norm_grad_execute(plan, x_ptr, dy_ptr, stats_ptr, gamma_ptr,
                                                  beta_ptr, dx_ptr, dgamma_ptr, dbeta_ptr, stream),
              "huge2_layer_norm_grad_execute")


def huge2_layer_norm_plan_kernel(plan, grad=False):
    return lib().huge2_layer_norm_plan_kernel(plan, int(grad)).decode()


def huge2_layer_norm_plan_destroy(plan):
    h2._check(lib().huge2_layer_norm_plan_destroy(plan), "huge2_layer_norm_plan_destroy")


def huge2_embedding(desc, ids_ptr, tokens, table_ptr, y_ptr, stream=0):
    h2._check(lib().huge2_embedding(ctypes.byref(desc), ids_ptr, tokens, table_ptr, y_ptr, stream),
              "huge2_embedding")


def huge2_embedding_grad_plan_create(desc, max_tokens):
    plan = ctypes.c_void_p()
    h2._check(lib().huge2_embedding_grad_plan_create(ctypes.byref(plan), ctypes.byref(desc),
                                                     max_tokens),
              "huge2_embedding_grad_plan_create")
    return plan


def huge2_embedding_grad_execute(plan, ids_ptr, tokens, dy_ptr, dtable_ptr, stream=0):
    h2._check(lib().huge2_embedding_grad_execute(plan, ids_ptr, tokens, dy_ptr, dtable_ptr,
                                                 stream), "huge2_embedding_grad_execute")


def huge2_embedding_grad_plan_kernel(plan, tokens):
    return lib().huge2_embedding_grad_plan_kernel(plan, tokens).decode()


def huge2_embedding_grad_plan_destroy(plan):
    h2._check(lib().huge2_embedding_grad_plan_destroy(plan), "huge2_embedding_grad_plan_destroy")


def huge2_adamw_plan_create(tensors, state_bits, stream=0):
    """tensors: a sequence of :class:`AdamWTensor`."""
    plan = ctypes.c_void_p()
    arr = (AdamWTensor * len(tensors))(*tensors)
    h2._check(lib().huge2_adamw_plan_create(ctypes.byref(plan), arr, len(tensors), state_bits,
                                            stream), "huge2_adamw_plan_create")
    return plan


def huge2_adamw_step(plan, grad_ptrs, options, grad_scale_ptr=0, stream=0):
    """grad_ptrs: the address of an array of device pointers, one a tensor."""
    h2._check(lib().huge2_adamw_step(plan, grad_ptrs, ctypes.byref(options), grad_scale_ptr,
                                     stream), "huge2_adamw_step")


def huge2_adamw_plan_destroy(plan):
    h2._check(lib().huge2_adamw_plan_destroy(plan), "huge2_adamw_plan_destroy")


def huge2_orthogonalize_plan_create(desc, ns, stream=0):
    plan = ctypes.c_void_p()
    h2._check(lib().huge2_orthogonalize_plan_create(ctypes.byref(plan), ctypes.byref(desc),
                                                    ctypes.byref(ns), stream),
              "huge2_orthogonalize_plan_create")
    return plan


def huge2_orthogonalize_execute(plan, x_ptr, y_ptr, stream=0):
    h2._check(lib().huge2_orthogonalize_execute(plan, x_ptr, y_ptr, stream),
              "huge2_orthogonalize_execute")


def huge2_orthogonalize_plan_destroy(plan):
    h2._check(lib().huge2_orthogonalize_plan_destroy(plan), "huge2_orthogonalize_plan_destroy")


def huge2_muon_plan_create(tensors, ns, stream=0):
    """tensors: a sequence of :class:`MuonTensor`."""
    plan = ctypes.c_void_p()
    arr = (MuonTensor * len(tensors))(*tensors)
    h2._check(lib().huge2_muon_plan_create(ctypes.byref(plan), arr, len(tensors),
                                           ctypes.byref(ns), stream), "huge2_muon_plan_create")
    return plan


def huge2_muon_step(plan, grad_ptrs, options, grad_scale_ptr=0, stream=0):
    """grad_ptrs: the address of an array of device pointers, one a tensor."""
    h2._check(lib().huge2_muon_step(plan, grad_ptrs, ctypes.byref(options), grad_scale_ptr,
                                    stream), "huge2_muon_step")


def huge2_muon_plan_destroy(plan):
    h2._check(lib().huge2_muon_plan_destroy(plan), "huge2_muon_plan_destroy")


def newton_schulz(steps=5, coefficients=COEFFICIENTS, products="f32", eps=1e-7):
    """:class:`NewtonSchulz` of `steps` steps, with one triple of coefficients or one for each."""
    if products not in PRODUCTS:
        raise ValueError("unknown products %r (f32, f16)" % (products,))
    if steps != int(steps) or not 1 <= steps <= 32:
        raise ValueError("steps must be 1 to 32")
    steps = int(steps)
    triples = [tuple(t) for t in coefficients] if hasattr(coefficients[0], "__len__") else \
        [tuple(coefficients)] * steps
    if len(triples) != steps or any(len(t) != 3 for t in triples):
        raise ValueError("coefficients must be one triple, or one for each of %d steps" % steps)
    values = (ctypes.c_double * (3 * steps))(*(v for t in triples for v in t))
    return NewtonSchulz(steps, PRODUCTS[products], values, eps)


# ---- torch conveniences -----------------------------------------------------

_torch = h2._torch


def _current_device():
    torch = _torch()
    return torch.device("cuda", torch.cuda.current_device())


def _raw_stream():
    """The function that gives a device's current stream as a pointer (a tenth of a
    microsecond; making a torch.cuda.Stream takes one or two, as long as the smallest
    kernels)."""
    return _torch()._C._cuda_getCurrentRawStream


def _type_code(dtype):
    torch = _torch()
    if dtype == torch.float32:
        return h2.HUGE2_F32
    if dtype == torch.bfloat16:
        return h2.HUGE2_BF16
    raise TypeError("unsupported dtype %s (float32 or bfloat16)" % dtype)


def _take(t, name, index, shape, dtype):
    """Pointer of a contiguous, aligned tensor of this device, shape and type.  (The checks
    of a call's tensors take as long as half a launch: they ask each thing once.)"""
    try:
        if t.dtype is dtype and t.shape == shape and t.get_device() == index \
                and t.is_contiguous():
            p = t.data_ptr()
            if not p & 15:
                return p
    except AttributeError:
        pass
    h2._check_tensor(t, name, _torch().device("cuda", index))  # raises, or what is left is:
    raise ValueError("%s is %s %s, expected %s %s"
                     % (name, tuple(t.shape), t.dtype, tuple(shape), dtype))


class _Owner:
    """Closes its plan once."""
    _plan = None
    _destroy = None

    def close(self):
        plan, self._plan = self._plan, None
        if plan is not None:
            type(self)._destroy(plan)

    def _open(self):
        if self._plan is None:
            raise ValueError("%s is closed" % type(self).__name__)
        return self._plan

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class _Norm(_Owner):
    """The calls of a norm with a scale, a shift and an activation for each channel."""

    def _init(self, x_shape, c, stats_shape, dtype, activation):
        torch = _torch()
        if activation not in NORM_ACTIVATIONS:
            raise ValueError("unknown activation %r (none, relu, tanh, silu)" % (activation,))
        self.x_shape, self.dtype = torch.Size(x_shape), dtype
        self.param_shape, self.stats_shape = torch.Size((c,)), torch.Size(stats_shape)
        self.device = _current_device()
        self._index, self._f32, self._stream = self.device.index, torch.float32, _raw_stream()
        self._execute, self._grad_execute = (getattr(lib(), name) for name in self._names[:2])
        # (the quickest way to a new tensor)
        self._param_like = torch.empty(c, dtype=torch.float32, device=self.device)
        self._like = torch.empty_like

    def _x(self, t, name):
        return _take(t, name, self._index, self.x_shape, self.dtype)

    def _param(self, t, name):
        return 0 if t is None else _take(t, name, self._index, self.param_shape, self._f32)

    def _out(self, out):
        if out is None:
            out = _torch().empty(self.x_shape, dtype=self.dtype, device=self.device)
            return out, out.data_ptr()
        return out, self._x(out, "out")

    def __call__(self, x, gamma=None, beta=None, out=None, stats=None):
        """y; ``stats`` (float32 of ``stats_shape``, :meth:`new_stats`) receives the mean and
        reciprocal standard deviation that :meth:`grad` reads."""
        xp = self._x(x, "x")
        y, yp = self._out(out)
        sp = 0 if stats is None else _take(stats, "stats", self._index, self.stats_shape,
                                           self._f32)
        status = self._execute(self._open(), xp, self._param(gamma, "gamma"),
                               self._param(beta, "beta"), yp, sp, self._stream(self._index))
        if status:
            h2._check(status, self._names[0])
        return y

    def new_stats(self):
        return _torch().empty(self.stats_shape, dtype=self._f32, device=self.device)

    def grad(self, x, dy, stats, gamma=None, beta=None, out=None):
        """(dx, dgamma, dbeta) for the output error dy of a call with these x, gamma and
        beta, which filled stats."""
        xp, dyp = self._x(x, "x"), self._x(dy, "dy")
        sp = _take(stats, "stats", self._index, self.stats_shape, self._f32)
        dx, dxp = self._out(out)
        dgamma, dbeta = self._like(self._param_like), self._like(self._param_like)
        status = self._grad_execute(self._open(), xp, dyp, sp, self._param(gamma, "gamma"),
                                    self._param(beta, "beta"), dxp, dgamma.data_ptr(),
                                    dbeta.data_ptr(), self._stream(self._index))
        if status:
            h2._check(status, self._names[1])
        return dx, dgamma, dbeta

    @property
    def kernels(self):
        """Names of the kernels that a call and a gradient launch."""
        return tuple(self._kernel(self._open(), g) for g in (0, 1))


class GroupNorm(_Norm):
    """y = activation(group_norm(x) * gamma + beta) for inputs of one shape
    (``layout`` "NHWC" or "NCHW"), and its gradients.  activation: None, "relu",
    "tanh" or "silu".  Statistics are [n, groups, 2]."""
    _destroy = staticmethod(huge2_norm_plan_destroy)
    _kernel = staticmethod(huge2_norm_plan_kernel)
    _names = ("huge2_norm_execute", "huge2_norm_grad_execute")

    def __init__(self, x_shape, groups, dtype, layout="NCHW", activation=None, eps=1e-5):
        lay = h2._layout_code(layout)
        if len(x_shape) != 4:
            raise ValueError("x must be 4-D")
        n, c, h, w = x_shape if lay == h2.HUGE2_NCHW else [x_shape[i] for i in (0, 3, 1, 2)]
        self._init(x_shape, c, (n, groups, 2), dtype, activation)
        self.desc = NormDesc(n, c, h, w, groups, lay, _type_code(dtype),
                             NORM_ACTIVATIONS[activation], eps)
        self._plan = huge2_norm_plan_create(self.desc)


class LayerNorm(_Norm):
    """y = activation(layer_norm(x) * gamma + beta) over the channels of each pixel, for inputs
    of one shape, and its gradients.  ``layout`` "NHWC": any shape whose last axis are the
    channels ([tokens, c], [n, h, w, c], ...); "NCHW": [n, c, h, w].  activation: None, "relu",
    "tanh" or "silu".  Statistics are [pixels, 2]."""
    _destroy = staticmethod(huge2_layer_norm_plan_destroy)
    _kernel = staticmethod(huge2_layer_norm_plan_kernel)
    _names = ("huge2_layer_norm_execute", "huge2_layer_norm_grad_execute")

    def __init__(self, x_shape, dtype, layout="NHWC", activation=None, eps=1e-5):
        lay = h2._layout_code(layout)
        if lay == h2.HUGE2_NCHW:
            if len(x_shape) != 4:
                raise ValueError("x must be 4-D in NCHW")
            n, c, h, w = x_shape
        else:
            if len(x_shape) == 0:
                raise ValueError("x must have an axis of channels")
            n, c, h, w = math.prod(x_shape[:-1]), x_shape[-1], 1, 1
        self._init(x_shape, c, (n * h * w, 2), dtype, activation)
        self.desc = LayerNormDesc(n, c, h, w, lay, _type_code(dtype),
                                  NORM_ACTIVATIONS[activation], eps)
        self._plan = huge2_layer_norm_plan_create(self.desc)


class Embedding(_Owner):
    """y[t] = scale * table[ids[t]] and the table's gradient.  Ids are int32 or int64
    tensors of any shape; an id outside the table (-1 for padding) reads zeros and has no
    gradient.  ``max_tokens``: the most that :meth:`grad` will be called with (0: none, and
    no workspace)."""
    _destroy = staticmethod(huge2_embedding_grad_plan_destroy)

    def __init__(self, rows, dim, dtype, scale=1.0, max_tokens=0, id_dtype=None):
        torch = _torch()
        id_dtype = torch.int64 if id_dtype is None else id_dtype
        if id_dtype not in (torch.int32, torch.int64):
            raise TypeError("ids must be int32 or int64")
        self.device = _current_device()
        self._index, self._stream = self.device.index, _raw_stream()
        self._lookup = lib().huge2_embedding
        self.table_shape, self.dtype, self.id_dtype = torch.Size((rows, dim)), dtype, id_dtype
        self.desc = EmbeddingDesc(rows, dim, _type_code(dtype),
                                  64 if id_dtype == torch.int64 else 32, scale)
        self._desc_ref = ctypes.byref(self.desc)
        self._plan = huge2_embedding_grad_plan_create(self.desc, max_tokens)

    def _ids(self, ids):
        """Their pointer and the shape of their rows."""
        if ids.dtype is not self.id_dtype or ids.get_device() != self._index or \
                not ids.is_contiguous():
            raise ValueError("ids must be a contiguous %s tensor on %s"
                             % (self.id_dtype, self.device))
        return ids.data_ptr(), (*ids.shape, self.table_shape[1])

    def _out(self, out, shape):
        if out is None:
            out = _torch().empty(shape, dtype=self.dtype, device=self.device)
            return out, out.data_ptr()
        return out, _take(out, "out", self._index, shape, self.dtype)

    def __call__(self, ids, table, out=None):
        """y of ids' shape and the table's rows."""
        ip, shape = self._ids(ids)
        tp = _take(table, "table", self._index, self.table_shape, self.dtype)
        y, yp = self._out(out, shape)
        status = self._lookup(self._desc_ref, ip, ids.numel(), tp, yp, self._stream(self._index))
        if status:
            h2._check(status, "huge2_embedding")
        return y

    def grad(self, ids, dy, out=None):
        """The table's gradient, every row of it, for the output error dy."""
        ip, shape = self._ids(ids)
        dp = _take(dy, "dy", self._index, shape, self.dtype)
        dtable, tp = self._out(out, self.table_shape)
        huge2_embedding_grad_execute(self._open(), ip, ids.numel(), dp, tp,
                                     self._stream(self._index))
        return dtable

    def kernel(self, tokens):
        """Name of the kernels that a gradient of so many tokens launches."""
        return huge2_embedding_grad_plan_kernel(self._open(), tokens)


class _Optimizer(_Owner):
    """The gradients of a step over a list of parameters."""

    def _gradients(self, grads, grad_scale):
        """An array of the gradients' pointers (0: None) and the scale's pointer."""
        k = len(self._sizes)
        if len(grads) != k:
            raise ValueError("%d gradients for %d parameters" % (len(grads), k))
        try:
            ptrs = self._pointers(grads, self._sizes, self.grad_dtypes)
        except TypeError:  # some are None
            kept = [i for i, g in enumerate(grads) if g is not None]
            ptrs = [0] * k
            for i, p in zip(kept, self._pointers(*([x[i] for i in kept] for x in (
                    grads, self._sizes, self.grad_dtypes)))):
                ptrs[i] = p
        sp = 0
        if grad_scale is not None:
            if grad_scale.get_device() != self._index or \
                    grad_scale.dtype != _torch().float32 or grad_scale.numel() != 1:
                raise ValueError("grad_scale must be one float32 on %s" % self.device)
            sp = grad_scale.data_ptr()
        return array.array("Q", ptrs), sp

    def _pointers(self, grads, sizes, dtypes):
        # whole lists at a time: a loop over each gradient's properties takes twice as long
        T = _torch().Tensor
        if list(map(T.numel, grads)) != sizes or [g.dtype for g in grads] != dtypes or \
                not all(map(T.is_contiguous, grads)) or \
                list(map(T.get_device, grads)) != [self._index] * len(sizes):
            raise ValueError("gradients must be contiguous tensors on %s of their parameters' "
                             "sizes and of the types %s" % (self.device, dtypes))
        return list(map(T.data_ptr, grads))


class AdamW(_Optimizer):
    """AdamW over a list of parameters, all in one call, in place.

    params        contiguous float32 or bfloat16 tensors.
    state_bits    32: float32 moments ``m`` and ``v``.  8: torch.float8_e4m3fn numbers of m
                  and of sqrt(v), with float32 ``m_scale`` and ``v_scale``, one for each 256
                  elements of a tensor.
    weight_decay  one number, or one for each parameter.
    copies        None, or for each parameter None or a bfloat16 tensor that receives the
                  updated parameter (the working weights of float32 parameters).
    grad_dtypes   None (the copies', else the parameters' own types), or one for each parameter.
    m, v, m_scale, v_scale
                  lists of states to go on from; made as zeros where not given.
    """
    _destroy = staticmethod(huge2_adamw_plan_destroy)

    def __init__(self, params, state_bits=32, weight_decay=0.01, copies=None, grad_dtypes=None,
                 m=None, v=None, m_scale=None, v_scale=None):
        torch = _torch()
        self.device = _current_device()
        self._index, self._stream = self.device.index, _raw_stream()
        self.params, self.state_bits = list(params), state_bits
        if state_bits not in (32, 8):
            raise ValueError("state_bits must be 32 or 8")
        k = len(self.params)
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else \
            [weight_decay] * k
        self.copies = list(copies) if copies is not None else [None] * k
        state = torch.float32 if state_bits == 32 else torch.float8_e4m3fn

        def states(given, sizes, dtype):
            if given is not None:
                return list(given)
            return [torch.zeros(n, dtype=dtype, device=self.device) for n in sizes]

        sizes = [p.numel() for p in self.params]
        blocks = [-(-n // STATE_BLOCK) for n in sizes]
        self.m, self.v = states(m, sizes, state), states(v, sizes, state)
        self.m_scale = self.v_scale = None
        if state_bits == 8:
            self.m_scale = states(m_scale, blocks, torch.float32)
            self.v_scale = states(v_scale, blocks, torch.float32)
        elif m_scale is not None or v_scale is not None:
            raise ValueError("32-bit states have no scales")
        if grad_dtypes is None:
            grad_dtypes = [(p if c is None else c).dtype for p, c in zip(self.params, self.copies)]
        self.grad_dtypes = list(grad_dtypes)
        lists = [decay, self.copies, self.m, self.v, self.grad_dtypes]
        if state_bits == 8:
            lists += [self.m_scale, self.v_scale]
        if any(len(x) != k for x in lists):
            raise ValueError("every list needs one entry for each of %d parameters" % k)
        tensors = []
        for i, p in enumerate(self.params):
            n = sizes[i]

            def same(t, name, dtype):
                if n == 0:
                    return None
                if t.numel() != n:
                    raise ValueError("%s has %d elements, expected %d" % (name, t.numel(), n))
                return _take(t, name, self._index, t.shape, dtype)

            t = AdamWTensor(param=same(p, "param", p.dtype), m=same(self.m[i], "m", state),
                            v=same(self.v[i], "v", state), count=n, dtype=_type_code(p.dtype),
                            weight_decay=decay[i], grad_dtype=_type_code(self.grad_dtypes[i]))
            if self.copies[i] is not None:
                t.copy = same(self.copies[i], "copy", torch.bfloat16)
            if state_bits == 8:
                for name in ("m_scale", "v_scale"):
                    s = getattr(self, name)[i]
                    if s.get_device() != self._index or s.dtype != torch.float32 or \
                            s.numel() != blocks[i] or not s.is_contiguous():
                        raise ValueError("%s must be %d contiguous float32 on %s"
                                         % (name, blocks[i], self.device))
                    setattr(t, name, s.data_ptr() if n else None)
            tensors.append(t)
        self._sizes = sizes
        self._plan = huge2_adamw_plan_create(tensors, state_bits, self._stream(self._index))

    def step(self, grads, lr, step, betas=(0.9, 0.999), eps=1e-8, grad_scale=None):
        """One step (``step`` counts from 1).  grads: for each parameter its gradient, of its
        size and gradient type, or None (the parameter stays as it is).  grad_scale: None, or
        a float32 device tensor of one element that multiplies every gradient.  A step that is
        recorded into a graph keeps its step number, lr, betas and gradients in every replay:
        enqueue the steps of a training loop outside of it."""
        ptrs, sp = self._gradients(grads, grad_scale)
        huge2_adamw_step(self._open(), ptrs.buffer_info()[0],
                         AdamWOptions(lr, betas[0], betas[1], eps, step), sp,
                         self._stream(self._index))


class Orthogonalize(_Owner):
    """Newton-Schulz steps of matrices of one shape [..., rows, cols], which bring their singular
    values near 1.  products: "f32" (results as of products in fp32, whatever the tensors' type)
    or "f16" (large matrices in 45% of the time; off by some 2^-10 of a result's norm, of low rank
    by up to 2^-6, or 2^-3 where rows or columns are fewer than 32).  coefficients: one triple
    (a, b, c), or one for each step."""
    _destroy = staticmethod(huge2_orthogonalize_plan_destroy)

    def __init__(self, shape, dtype, products="f32", steps=5, coefficients=COEFFICIENTS, eps=1e-7):
        torch = _torch()
        if len(shape) < 2:
            raise ValueError("x must have rows and columns")
        self.device = _current_device()
        self._index, self._stream = self.device.index, _raw_stream()
        self.shape, self.dtype = torch.Size(shape), dtype
        code = _type_code(dtype)
        self.products = products or "f32"
        self.desc = OrthogonalizeDesc(math.prod(shape[:-2]), *shape[-2:], code)
        self._plan = huge2_orthogonalize_plan_create(
            self.desc, newton_schulz(steps, coefficients, self.products, eps),
            self._stream(self._index))

    def __call__(self, x, out=None):
        xp = _take(x, "x", self._index, self.shape, self.dtype)
        if out is None:
            out = _torch().empty(self.shape, dtype=self.dtype, device=self.device)
        huge2_orthogonalize_execute(self._open(), xp,
                                    _take(out, "out", self._index, self.shape, self.dtype),
                                    self._stream(self._index))
        return out


class Muon(_Optimizer):
    """The Muon step over a list of matrices, all in one call, in place: momentum, whose
    Newton-Schulz steps are the update.  Other parameters (norms, biases, tables) go to
    :class:`AdamW`.

    params        contiguous float32 or bfloat16 tensors of two axes or more; the first are the
                  rows (a convolution's weights: its first channels).
    weight_decay  one number, or one for each parameter.
    scales        None (sqrt(max(1, rows / cols))), or for each parameter what its update is
                  multiplied by.
    copies        None, or for each parameter None or a bfloat16 tensor that receives the
                  updated parameter (the working weights of float32 parameters).
    grad_dtypes   None (the copies', else the parameters' own types), or one for each parameter.
    m             a list of float32 momenta to go on from; made as zeros where not given.
    products, steps, coefficients, eps
                  of the Newton-Schulz steps, as in :class:`Orthogonalize`.
    """
    _destroy = staticmethod(huge2_muon_plan_destroy)

    def __init__(self, params, weight_decay=0.0, scales=None, copies=None, grad_dtypes=None,
                 m=None, products="f32", steps=5, coefficients=COEFFICIENTS, eps=1e-7):
        torch = _torch()
        self.device = _current_device()
        self._index, self._stream = self.device.index, _raw_stream()
        self.params = list(params)
        k = len(self.params)
        if any(p.dim() < 2 or p.numel() == 0 for p in self.params):
            raise ValueError("parameters must be matrices (two axes or more, no empty one)")
        shapes = [(p.shape[0], p.numel() // p.shape[0]) for p in self.params]
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else \
            [weight_decay] * k
        self.scales = [math.sqrt(max(1.0, r / c)) for r, c in shapes] if scales is None else \
            list(scales)
        self.copies = list(copies) if copies is not None else [None] * k
        self.m = [torch.zeros(p.shape, dtype=torch.float32, device=self.device)
                  for p in self.params] if m is None else list(m)
        if grad_dtypes is None:
            grad_dtypes = [(p if c is None else c).dtype for p, c in zip(self.params, self.copies)]
        self.grad_dtypes = list(grad_dtypes)
        if any(len(x) != k for x in (decay, self.scales, self.copies, self.m, self.grad_dtypes)):
            raise ValueError("every list needs one entry for each of %d parameters" % k)
        self.products = products or "f32"
        tensors = []
        for p, mt, c, shape, gd, wd, scale in zip(self.params, self.m, self.copies, shapes,
                                                  self.grad_dtypes, decay, self.scales):

            def same(t, name, dtype):
                if t.numel() != p.numel():
                    raise ValueError("%s has %d elements, expected %d"
                                     % (name, t.numel(), p.numel()))
                return _take(t, name, self._index, t.shape, dtype)

            tensors.append(MuonTensor(
                param=same(p, "param", p.dtype), m=same(mt, "m", torch.float32),
                copy=None if c is None else same(c, "copy", torch.bfloat16), rows=shape[0],
                cols=shape[1], dtype=_type_code(p.dtype), grad_dtype=_type_code(gd),
                weight_decay=wd, scale=scale))
        self._sizes = [p.numel() for p in self.params]
        self._plan = huge2_muon_plan_create(
            tensors, newton_schulz(steps, coefficients, self.products, eps),
            self._stream(self._index))

    def step(self, grads, lr, momentum=0.95, nesterov=True, grad_scale=None):
        """One step.  grads: for each parameter its gradient, of its size and gradient type, or
        None (the parameter and its momentum stay as they are).  grad_scale: None, or a float32
        device tensor of one element that multiplies every gradient.  A step that is recorded
        into a graph keeps its lr, momentum and gradients in every replay."""
        ptrs, sp = self._gradients(grads, grad_scale)
        huge2_muon_step(self._open(), ptrs.buffer_info()[0],
                        MuonOptions(lr, momentum, int(bool(nesterov))), sp,
                        self._stream(self._index))
