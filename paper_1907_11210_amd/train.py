"""Python binding of the operators around the convolutions (the C ABI in
include/huge2_train.h): group norm with an activation, embedding lookup and the
AdamW step, with their gradients.

Argument marshalling only, as in :mod:`paper_1907_11210_amd.huge2`: the ``huge2_*``
functions mirror the C entry points and take raw device pointers (ints);
:class:`GroupNorm`, :class:`Embedding` and :class:`AdamW` take torch tensors and
enqueue on the current stream.  Objects belong to the device that was current when
they were made; one object's calls share its workspace, so make them on one stream
or order them.
"""
from __future__ import annotations

import array
import ctypes

from . import huge2 as h2

NORM_ACTIVATIONS = {None: 0, "none": 0, "relu": 1, "tanh": 2, "silu": 3}
STATE_BLOCK = 256  # elements that share a scale in 8-bit states

EXPORTED = (
    "huge2_norm_plan_create", "huge2_norm_execute", "huge2_norm_grad_execute",
    "huge2_norm_plan_kernel", "huge2_norm_plan_destroy",
    "huge2_embedding", "huge2_embedding_grad_plan_create", "huge2_embedding_grad_execute",
    "huge2_embedding_grad_plan_kernel", "huge2_embedding_grad_plan_destroy",
    "huge2_adamw_plan_create", "huge2_adamw_step", "huge2_adamw_plan_destroy",
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
            "huge2_embedding": [ctypes.POINTER(EmbeddingDesc), vp, i64, vp, vp, vp],
            "huge2_embedding_grad_plan_create": [out, ctypes.POINTER(EmbeddingDesc), i64],
            "huge2_embedding_grad_execute": [vp, vp, i64, vp, vp, vp],
            "huge2_embedding_grad_plan_kernel": [vp, i64],
            "huge2_embedding_grad_plan_destroy": [vp],
            "huge2_adamw_plan_create": [out, ctypes.POINTER(AdamWTensor), i32, i32, vp],
            "huge2_adamw_step": [vp, vp, ctypes.POINTER(AdamWOptions), vp, vp],
            "huge2_adamw_plan_destroy": [vp],
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


class GroupNorm(_Owner):
    """y = activation(group_norm(x) * gamma + beta) for inputs of one shape
    (``layout`` "NHWC" or "NCHW"), and its gradients.  activation: None, "relu",
    "tanh" or "silu"."""
    _destroy = staticmethod(huge2_norm_plan_destroy)

    def __init__(self, x_shape, groups, dtype, layout="NCHW", activation=None, eps=1e-5):
        torch = _torch()
        lay = h2._layout_code(layout)
        if len(x_shape) != 4:
            raise ValueError("x must be 4-D")
        if activation not in NORM_ACTIVATIONS:
            raise ValueError("unknown activation %r (none, relu, tanh, silu)" % (activation,))
        n, c, h, w = x_shape if lay == h2.HUGE2_NCHW else [x_shape[i] for i in (0, 3, 1, 2)]
        self.x_shape, self.dtype = torch.Size(x_shape), dtype
        self.param_shape = torch.Size((c,))
        self.stats_shape = torch.Size((n, groups, 2))
        self.device = _current_device()
        self._index, self._f32, self._stream = self.device.index, torch.float32, _raw_stream()
        self._execute, self._grad_execute = (lib().huge2_norm_execute,
                                             lib().huge2_norm_grad_execute)
        self.desc = NormDesc(n, c, h, w, groups, lay, _type_code(dtype),
                             NORM_ACTIVATIONS[activation], eps)
        self._plan = huge2_norm_plan_create(self.desc)
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
        """y; ``stats`` ([n, groups, 2] float32, :meth:`new_stats`) receives the mean and
        reciprocal standard deviation that :meth:`grad` reads."""
        xp = self._x(x, "x")
        y, yp = self._out(out)
        sp = 0 if stats is None else _take(stats, "stats", self._index, self.stats_shape,
                                           self._f32)
        status = self._execute(self._open(), xp, self._param(gamma, "gamma"),
                               self._param(beta, "beta"), yp, sp, self._stream(self._index))
        if status:
            h2._check(status, "huge2_norm_execute")
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
            h2._check(status, "huge2_norm_grad_execute")
        return dx, dgamma, dbeta

    @property
    def kernels(self):
        """Names of the kernels that a call and a gradient launch."""
        return tuple(huge2_norm_plan_kernel(self._open(), g) for g in (0, 1))


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


class AdamW(_Owner):
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
        ptrs = array.array("Q", ptrs)
        huge2_adamw_step(self._open(), ptrs.buffer_info()[0],
                         AdamWOptions(lr, betas[0], betas[1], eps, step), sp,
                         self._stream(self._index))

    def _pointers(self, grads, sizes, dtypes):
        # whole lists at a time: a loop over each gradient's properties takes twice as long
        T = _torch().Tensor
        if list(map(T.numel, grads)) != sizes or [g.dtype for g in grads] != dtypes or \
                not all(map(T.is_contiguous, grads)) or \
                list(map(T.get_device, grads)) != [self._index] * len(sizes):
            raise ValueError("gradients must be contiguous tensors on %s of their parameters' "
                             "sizes and of the types %s" % (self.device, dtypes))
        return list(map(T.data_ptr, grads))
