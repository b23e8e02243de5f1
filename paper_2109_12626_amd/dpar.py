"""Python binding of libdpar.so (include/dpar.h).

Argument marshalling only: every step of the reduction runs in the library's
HIP kernels.  The functions keep the C names.  torch is imported first so that
the library binds to the HIP runtime torch already loaded (one runtime per
process); torch serves only for device memory and streams.
"""

import ctypes
import os

import numpy as np

import torch  # noqa: F401  (must precede loading libdpar: one HIP runtime)

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("DPAR_LIB_PATH") or os.path.join(_HERE, "libdpar.so")

DPAR_SUCCESS = 0
DPAR_ERR_INVALID_ARG = -1
DPAR_ERR_UNSUPPORTED = -2
DPAR_ERR_ALIAS = -3
DPAR_ERR_NOMEM = -4
DPAR_ERR_HIP = -5
DPAR_ERR_TIMEOUT = -6

DPAR_INT32, DPAR_FLOAT32, DPAR_U32_MAT2X2, DPAR_BFLOAT16, DPAR_FLOAT16 = \
    0, 1, 2, 3, 4
DPAR_SUM, DPAR_MAX, DPAR_MATMUL = 0, 1, 2
DPAR_EXEC_AUTO, DPAR_EXEC_LAUNCH_PER_ROUND, DPAR_EXEC_GRID_BARRIER, \
    DPAR_EXEC_TICKET, DPAR_EXEC_SPLIT, DPAR_EXEC_ROUNDS, \
    DPAR_EXEC_ROUNDS_BARRIER = 0, 1, 2, 3, 4, 5, 6
DPAR_ALG_DUAL_ROOT, DPAR_ALG_SINGLE_TREE, DPAR_ALG_REDUCE_BCAST = 0, 1, 2

DPAR_ACT_NONE, DPAR_ACT_RELU, DPAR_ACT_GELU, DPAR_ACT_GELU_TANH, \
    DPAR_ACT_SILU = 0, 1, 2, 3, 4
DPAR_LINEAR, DPAR_LINEAR_BACKWARD, DPAR_GATED, DPAR_GATED_BACKWARD = 0, 1, 2, 3

DTYPES = {"int32": DPAR_INT32, "float32": DPAR_FLOAT32,
          "u32mat2x2": DPAR_U32_MAT2X2, "bfloat16": DPAR_BFLOAT16,
          "float16": DPAR_FLOAT16}
OPS = {"sum": DPAR_SUM, "max": DPAR_MAX, "matmul": DPAR_MATMUL}
EXECS = {"auto": DPAR_EXEC_AUTO, "launch": DPAR_EXEC_LAUNCH_PER_ROUND,
         "barrier": DPAR_EXEC_GRID_BARRIER, "ticket": DPAR_EXEC_TICKET,
         "split": DPAR_EXEC_SPLIT, "rounds": DPAR_EXEC_ROUNDS,
         "rounds_barrier": DPAR_EXEC_ROUNDS_BARRIER}
ALGS = {"dual": DPAR_ALG_DUAL_ROOT, "single": DPAR_ALG_SINGLE_TREE,
        "reduce_bcast": DPAR_ALG_REDUCE_BCAST}

ACTS = {"none": DPAR_ACT_NONE, "relu": DPAR_ACT_RELU, "gelu": DPAR_ACT_GELU,
        "gelu_tanh": DPAR_ACT_GELU_TANH, "silu": DPAR_ACT_SILU}
PRODUCTS = {"linear": DPAR_LINEAR, "linear_backward": DPAR_LINEAR_BACKWARD,
            "gated": DPAR_GATED, "gated_backward": DPAR_GATED_BACKWARD}


class DparError(RuntimeError):
    def __init__(self, code, msg):
        self.code = code
        super().__init__(f"dpar error {code}: {msg}")


class dpar_node_t(ctypes.Structure):
    _fields_ = [("parent", ctypes.c_int), ("child0", ctypes.c_int),
                ("child1", ctypes.c_int), ("depth", ctypes.c_int),
                ("subtree_lo", ctypes.c_int), ("dual", ctypes.c_int)]


class dpar_options_t(ctypes.Structure):
    _fields_ = [("alg", ctypes.c_int), ("exec", ctypes.c_int),
                ("round_begin", ctypes.c_int), ("round_end", ctypes.c_int)]


class dpar_schedule_t(ctypes.Structure):
    _fields_ = [("b", ctypes.c_int), ("granularity", ctypes.c_int),
                ("quantum", ctypes.c_int),
                ("nquanta", ctypes.c_size_t), ("tail_elems", ctypes.c_size_t),
                ("chunks_per_block", ctypes.c_int), ("height", ctypes.c_int),
                ("waves_per_chunk", ctypes.c_int)]


class dpar_product_t(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_size_t), ("in_", ctypes.c_size_t),
                ("out", ctypes.c_size_t), ("dtype", ctypes.c_int),
                ("out_dtype", ctypes.c_int), ("act", ctypes.c_int),
                ("ldx", ctypes.c_size_t), ("ldw", ctypes.c_size_t),
                ("ldy", ctypes.c_size_t), ("ldr", ctypes.c_size_t),
                ("ldz", ctypes.c_size_t), ("lddx", ctypes.c_size_t),
                ("lddw", ctypes.c_size_t)]


_lib = None


def lib():
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with "
            "`python -c 'import __graft_entry__ as g; g.build()'`")
    L = ctypes.CDLL(LIB_PATH)
    vp, sz, i = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
    L.dpar_allreduce.argtypes = [vp, vp, i, sz, i, i, i, vp]
    L.dpar_allreduce_ex.argtypes = [vp, vp, i, sz, i, i, i, i, vp]
    L.dpar_allreduce_noalloc.argtypes = [vp, vp, i, sz, i, i, i, vp]
    L.dpar_allreduce_opt.argtypes = [vp, vp, i, sz, i, i, i,
                                     ctypes.POINTER(dpar_options_t), vp]
    L.dpar_tree_info.argtypes = [i, i, ctypes.POINTER(dpar_node_t)]
    L.dpar_tree_info_alg.argtypes = [i, i, i, ctypes.POINTER(dpar_node_t)]
    L.dpar_schedule_rounds.argtypes = [i, i, i]
    L.dpar_block_rule.argtypes = [i, sz, ctypes.c_double, ctypes.c_double]
    L.dpar_rounds.argtypes = [i, i, i]
    L.dpar_schedule_info.argtypes = [i, sz, i, i, i,
                                     ctypes.POINTER(dpar_schedule_t)]
    L.dpar_block_bounds.argtypes = [ctypes.POINTER(dpar_schedule_t), sz, i,
                                    ctypes.POINTER(sz), ctypes.POINTER(sz)]
    L.dpar_check_status.argtypes = [vp]
    L.dpar_set_phase_event.argtypes = [vp]
    opt = ctypes.POINTER(dpar_product_t)
    tail = [i, opt, vp, sz, vp]     # p, options, workspace, bytes, stream
    L.dpar_linear.argtypes = [vp] * 6 + tail
    L.dpar_linear_backward.argtypes = [vp] * 8 + tail
    L.dpar_gated.argtypes = [vp] * 8 + tail
    L.dpar_gated_backward.argtypes = [vp] * 13 + tail
    L.dpar_product_workspace.argtypes = [i, i, opt, ctypes.POINTER(sz)]
    L.dpar_last_error.restype = ctypes.c_char_p
    L.dpar_last_error.argtypes = []
    L.dpar_finalize.argtypes = []
    for name in ("dpar_allreduce", "dpar_allreduce_ex", "dpar_allreduce_opt",
                 "dpar_allreduce_noalloc",
                 "dpar_tree_info", "dpar_tree_info_alg",
                 "dpar_schedule_rounds", "dpar_block_rule", "dpar_rounds",
                 "dpar_schedule_info", "dpar_block_bounds",
                 "dpar_check_status", "dpar_finalize",
                 "dpar_set_phase_event", "dpar_linear",
                 "dpar_linear_backward", "dpar_gated", "dpar_gated_backward",
                 "dpar_product_workspace"):
        getattr(L, name).restype = ctypes.c_int
    _lib = L
    return L


def _check(rc):
    if rc < 0:
        raise DparError(rc, lib().dpar_last_error().decode())
    return rc


def _addr(v):
    if isinstance(v, torch.Tensor):
        return v.data_ptr()
    return int(v)


def _array_of(addrs):
    """A C array of void* viewing a uint64 numpy array (kept alive by it)."""
    if addrs.size == 0:
        return (ctypes.c_void_p * 0)()
    return (ctypes.c_void_p * addrs.size).from_buffer(addrs)


def pointers(seq):
    """A reusable C array of device addresses (ints or tensors); passing it
    instead of a list saves the conversion on every call."""
    if isinstance(seq, ctypes.Array):
        return seq
    if all(type(v) is int for v in seq):
        # plain addresses: one conversion in numpy instead of one per entry
        # (p = 1152: about 40 instead of 300 us on the host)
        return _array_of(np.array(seq, dtype=np.uint64))
    return (ctypes.c_void_p * len(seq))(*[_addr(v) for v in seq])


_ptr_array = pointers


def _stream(stream):
    if stream is None:
        return None
    if isinstance(stream, torch.cuda.Stream):
        return ctypes.c_void_p(stream.cuda_stream)
    return ctypes.c_void_p(int(stream))


def _enum(table, v):
    return table[v] if isinstance(v, str) else int(v)


def rows(t):
    """Device addresses of the rows of a [p, ...] tensor, as a reusable C
    array (indexable and iterable like a list of ints)."""
    if t.dim() < 1:
        raise ValueError("need at least one dimension")
    step = t.stride(0) * t.element_size()
    if step < 0:
        raise ValueError("rows with a negative stride")
    addrs = np.arange(t.shape[0], dtype=np.uint64) * np.uint64(step)
    addrs += np.uint64(t.data_ptr())
    return _array_of(addrs)


def dpar_allreduce(x, y, p, m, dtype, op, b=0, stream=None):
    """x, y: sequences of p device addresses (ints or tensors)."""
    return _check(lib().dpar_allreduce(
        _ptr_array(x), _ptr_array(y), int(p), int(m), _enum(DTYPES, dtype),
        _enum(OPS, op), int(b), _stream(stream)))


def dpar_allreduce_noalloc(x, y, p, m, dtype, op, b=0, stream=None):
    """The allocation-free variant of dpar_allreduce (include/dpar.h)."""
    return _check(lib().dpar_allreduce_noalloc(
        _ptr_array(x), _ptr_array(y), int(p), int(m), _enum(DTYPES, dtype),
        _enum(OPS, op), int(b), _stream(stream)))


def dpar_allreduce_ex(x, y, p, m, dtype, op, b=0, exec="auto", stream=None):
    return _check(lib().dpar_allreduce_ex(
        _ptr_array(x), _ptr_array(y), int(p), int(m), _enum(DTYPES, dtype),
        _enum(OPS, op), int(b), _enum(EXECS, exec), _stream(stream)))


def dpar_allreduce_opt(x, y, p, m, dtype, op, b=0, alg="dual", exec="auto",
                       round_begin=0, round_end=-1, stream=None):
    opt = dpar_options_t(_enum(ALGS, alg), _enum(EXECS, exec),
                         int(round_begin), int(round_end))
    return _check(lib().dpar_allreduce_opt(
        _ptr_array(x), _ptr_array(y), int(p), int(m), _enum(DTYPES, dtype),
        _enum(OPS, op), int(b), ctypes.byref(opt), _stream(stream)))


def dpar_tree_info(p, rank):
    out = dpar_node_t()
    _check(lib().dpar_tree_info(int(p), int(rank), ctypes.byref(out)))
    return {f: getattr(out, f) for f, _ in dpar_node_t._fields_}


def dpar_tree_info_alg(p, alg, rank):
    out = dpar_node_t()
    _check(lib().dpar_tree_info_alg(int(p), _enum(ALGS, alg), int(rank),
                                    ctypes.byref(out)))
    return {f: getattr(out, f) for f, _ in dpar_node_t._fields_}


def dpar_schedule_rounds(p, b, alg="dual"):
    return _check(lib().dpar_schedule_rounds(int(p), int(b), _enum(ALGS, alg)))


def dpar_block_rule(p, m, alpha=0.0, beta=0.0):
    return _check(lib().dpar_block_rule(int(p), int(m), float(alpha),
                                        float(beta)))


def dpar_rounds(p, b, rank=-1):
    return _check(lib().dpar_rounds(int(p), int(b), int(rank)))


def dpar_schedule_info(p, m, dtype, b=0, aligned=True):
    out = dpar_schedule_t()
    _check(lib().dpar_schedule_info(int(p), int(m), _enum(DTYPES, dtype),
                                    int(b), int(bool(aligned)),
                                    ctypes.byref(out)))
    return out


def dpar_block_bounds(sched, m, j):
    s, e = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib().dpar_block_bounds(ctypes.byref(sched), int(m), int(j),
                                   ctypes.byref(s), ctypes.byref(e)))
    return s.value, e.value


def dpar_check_status(stream=None):
    return _check(lib().dpar_check_status(_stream(stream)))


def dpar_set_phase_event(event):
    """event: a torch.cuda.Event that has been recorded once (so that it
    exists), a raw hipEvent_t handle, or None."""
    if event is None:
        h = None
    elif isinstance(event, torch.cuda.Event):
        h = ctypes.c_void_p(event.cuda_event)
    else:
        h = ctypes.c_void_p(int(event))
    return _check(lib().dpar_set_phase_event(h))


# ---------------------------------------------------------- layer products

def product_options(rows, n_in, n_out, dtype, out_dtype=None, act="none",
                    ldx=0, ldw=0, ldy=0, ldr=0, ldz=0, lddx=0, lddw=0):
    """Sizes, types and row distances of a layer product (dpar_product_t), to
    be kept and passed to any number of calls."""
    dt = _enum(DTYPES, dtype)
    return dpar_product_t(rows, n_in, n_out, dt,
                          dt if out_dtype is None else _enum(DTYPES, out_dtype),
                          _enum(ACTS, act), ldx, ldw, ldy, ldr, ldz, lddx,
                          lddw)


def dpar_product_workspace(call, p, opt):
    out = ctypes.c_size_t()
    _check(lib().dpar_product_workspace(_enum(PRODUCTS, call), int(p),
                                        ctypes.byref(opt), ctypes.byref(out)))
    return out.value


def _product(fn, arrays, p, opt, workspace, workspace_bytes, stream):
    if isinstance(workspace, torch.Tensor):
        workspace = workspace.data_ptr()
    if isinstance(stream, torch.cuda.Stream):
        stream = stream.cuda_stream
    rc = fn(*[a if a is None or isinstance(a, ctypes.Array)
              else _ptr_array(a) for a in arrays],
            p, ctypes.byref(opt), workspace, workspace_bytes, stream)
    return rc if rc >= 0 else _check(rc)


def dpar_linear(x, w, bias, residual, y, z, p, opt, workspace=None,
                workspace_bytes=0, stream=None):
    """Sequences of p device addresses (ints or tensors; 0 where a rank has no
    bias or residual), or None where optional; opt: product_options()."""
    return _product(lib().dpar_linear, (x, w, bias, residual, y, z), p, opt,
                    workspace, workspace_bytes, stream)


def dpar_linear_backward(dy, x, w, z, dx, dw, dbias, dz, p, opt,
                         workspace=None, workspace_bytes=0, stream=None):
    return _product(lib().dpar_linear_backward,
                    (dy, x, w, z, dx, dw, dbias, dz), p, opt, workspace,
                    workspace_bytes, stream)


def dpar_gated(x, wg, wu, bg, bu, h, g, u, p, opt, workspace=None,
               workspace_bytes=0, stream=None):
    return _product(lib().dpar_gated, (x, wg, wu, bg, bu, h, g, u), p, opt,
                    workspace, workspace_bytes, stream)


def dpar_gated_backward(dh, x, wg, wu, g, u, dx, dwg, dwu, dbg, dbu, dg, du, p,
                        opt, workspace=None, workspace_bytes=0, stream=None):
    return _product(lib().dpar_gated_backward,
                    (dh, x, wg, wu, g, u, dx, dwg, dwu, dbg, dbu, dg, du), p,
                    opt, workspace, workspace_bytes, stream)


def dpar_last_error():
    return lib().dpar_last_error().decode()


def dpar_finalize():
    return _check(lib().dpar_finalize())


# ------------------------------------------------------------ convenience

_ELEM = {"int32": 4, "float32": 4, "u32mat2x2": 16}


def allreduce(x, y=None, dtype=None, op="sum", b=0, exec="auto", stream=None,
              alg="dual"):
    """Tensor front end: x is a [p, m] (or [p, m, 4] uint32 for matrices)
    device tensor, or a list of p 1-D tensors; y likewise (default: a new
    [p, ...] tensor).  Returns y.  Only marshals addresses."""
    if isinstance(x, torch.Tensor):
        p = x.shape[0]
        xs = rows(x)
        sample = x[0]
    else:
        p = len(x)
        xs = [t.data_ptr() for t in x]
        sample = x[0]
    if dtype is None:
        dtype = {torch.int32: "int32", torch.float32: "float32",
                 torch.uint32: "u32mat2x2"}[sample.dtype]
    m = sample.numel() * sample.element_size() // _ELEM[dtype]
    if y is None:
        y = torch.empty((p,) + tuple(sample.shape), dtype=sample.dtype,
                        device=sample.device)
    ys = rows(y) if isinstance(y, torch.Tensor) else [t.data_ptr() for t in y]
    if stream is None:
        stream = torch.cuda.current_stream(sample.device)
    dpar_allreduce_opt(xs, ys, p, m, dtype, op, b, alg, exec, 0, -1, stream)
    return y


# Tensor front ends of the layer products.  x, dy, dh: [p, rows, ...] or, for
# all ranks alike or one rank, [rows, ...]; weights [p, out, in] or [out, in];
# biases [p, out] or [out]; a residual like the result.  Rows may be any
# distance apart; the values of a row are consecutive.  The results are new
# tensors [p, ...] (without the first dimension if w has none).  Only marshals
# addresses: every product runs in the library's kernels.  Nothing is recorded
# for autograd: tensors that require a gradient are refused where it is on.

_NAMES = {torch.float32: "float32", torch.bfloat16: "bfloat16",
          torch.float16: "float16"}


class _Call:
    """Shapes, row distances and addresses of one call's tensors."""

    def __init__(self, w, rows_, out_dtype, act):
        self.flat = w.dim() == 2
        self.p = 1 if self.flat else w.shape[0]
        self.n_out, self.n_in = w.shape[-2:]
        self.rows = rows_
        self.dtype = w.dtype
        self.out_dtype = w.dtype if out_dtype is None else out_dtype
        if w.dtype not in _NAMES or self.out_dtype not in _NAMES:
            raise ValueError(f"types {w.dtype}, {self.out_dtype}")
        self.opt = product_options(rows_, self.n_in, self.n_out,
                                   _NAMES[w.dtype], _NAMES[self.out_dtype],
                                   act)
        self.device = w.device

    def given(self, t, name, shape, ld=None, dtype=None):
        """Addresses of an operand's ranks; sets its row distance."""
        if t is None:
            return None
        if t.device != self.device or t.dtype != (dtype or self.dtype):
            raise ValueError(f"{name}: {t.dtype} on {t.device}")
        if t.requires_grad and torch.is_grad_enabled():
            raise ValueError(f"{name} requires a gradient, and these calls "
                             "record none: call under torch.no_grad() (or "
                             "detach it) and use the backward call")
        one = t.dim() == len(shape)
        if tuple(t.shape[-len(shape):]) != shape or \
                not (one or (t.dim() == len(shape) + 1
                             and t.shape[0] == self.p)):
            raise ValueError(f"{name}: shape {tuple(t.shape)}, want "
                             f"{shape} or {(self.p,) + shape}")
        if one and self.p > 1 and name not in ("x", "dy", "dh"):
            raise ValueError(f"{name}: one matrix for {self.p} ranks")
        if shape[-1] > 1 and t.stride(-1) != 1:
            raise ValueError(f"{name}: values of a row are not consecutive")
        if ld is not None:
            far = t.stride(-2) if shape[0] > 1 else shape[1]
            if far < shape[1]:
                raise ValueError(f"{name}: rows {far} values apart overlap")
            if getattr(self.opt, ld) not in (0, far):
                raise ValueError(f"{name}: another row distance than its "
                                 "companion's")
            setattr(self.opt, ld, far)
        if one:
            return pointers([t.data_ptr()] * self.p)
        return rows(t)

    def made(self, *shape, dtype=None):
        return torch.empty((self.p,) + shape, dtype=dtype or self.out_dtype,
                           device=self.device)

    def run(self, call, fn, arrays):
        n = dpar_product_workspace(call, self.p, self.opt)
        ws = torch.empty(n, dtype=torch.uint8, device=self.device) \
            if n else None
        fn(*arrays, self.p, self.opt, ws, n,
           torch.cuda.current_stream(self.device))

    def result(self, t):
        return t[0] if self.flat and t is not None else t


def _addresses(t):
    return None if t is None else rows(t)


def linear(x, w, bias=None, residual=None, act="none", out_dtype=None,
           keep=False):
    """act(x w^T + bias) + residual, and with keep=True the value before the
    activation too."""
    c = _Call(w, x.shape[-2], out_dtype, act)
    arrays = [c.given(x, "x", (c.rows, c.n_in), "ldx"),
              c.given(w, "w", (c.n_out, c.n_in), "ldw"),
              c.given(bias, "bias", (c.n_out,)),
              c.given(residual, "residual", (c.rows, c.n_out), "ldr",
                      c.out_dtype)]
    y = c.made(c.rows, c.n_out)
    z = c.made(c.rows, c.n_out, dtype=c.dtype) if keep else None
    c.run("linear", dpar_linear, arrays + [_addresses(y), _addresses(z)])
    return (c.result(y), c.result(z)) if keep else c.result(y)


def linear_backward(dy, x, w, z=None, act="none", out_dtype=None, bias=False):
    """(dx, dw), with bias=True (dx, dw, dbias); z: what linear() kept."""
    c = _Call(w, x.shape[-2], out_dtype, act)
    arrays = [c.given(dy, "dy", (c.rows, c.n_out), "ldy"),
              c.given(x, "x", (c.rows, c.n_in), "ldx"),
              c.given(w, "w", (c.n_out, c.n_in), "ldw")]
    if act != "none":
        if z is None:
            raise ValueError("an activation's slope needs z")
        z = z.contiguous()
    else:
        z = None
    arrays.append(c.given(z, "z", (c.rows, c.n_out), "ldz"))
    dx, dw = c.made(c.rows, c.n_in), c.made(c.n_out, c.n_in)
    db = c.made(c.n_out) if bias else None
    dz = None if z is None else c.made(c.rows, c.n_out, dtype=c.dtype)
    c.run("linear_backward", dpar_linear_backward,
          arrays + [_addresses(t) for t in (dx, dw, db, dz)])
    out = (dx, dw, db) if bias else (dx, dw)
    return tuple(c.result(t) for t in out)


def gated(x, wg, wu, bg=None, bu=None, act="silu", out_dtype=None, keep=False):
    """act(x wg^T + bg) * (x wu^T + bu), and with keep=True both projections
    too."""
    c = _Call(wg, x.shape[-2], out_dtype, act)
    arrays = [c.given(x, "x", (c.rows, c.n_in), "ldx"),
              c.given(wg, "wg", (c.n_out, c.n_in), "ldw"),
              c.given(wu, "wu", (c.n_out, c.n_in), "ldw"),
              c.given(bg, "bg", (c.n_out,)), c.given(bu, "bu", (c.n_out,))]
    h = c.made(c.rows, c.n_out)
    g, u = (c.made(c.rows, c.n_out, dtype=c.dtype) if keep else None
            for _ in range(2))
    c.run("gated", dpar_gated, arrays + [_addresses(t) for t in (h, g, u)])
    out = (h, g, u) if keep else (h,)
    return tuple(c.result(t) for t in out) if keep else c.result(h)


def gated_backward(dh, x, wg, wu, g, u, act="silu", out_dtype=None,
                   bias=False):
    """(dx, dwg, dwu), with bias=True (dx, dwg, dwu, dbg, dbu); g, u: what
    gated() kept."""
    c = _Call(wg, x.shape[-2], out_dtype, act)
    g, u = g.contiguous(), u.contiguous()
    arrays = [c.given(dh, "dh", (c.rows, c.n_out), "ldy"),
              c.given(x, "x", (c.rows, c.n_in), "ldx"),
              c.given(wg, "wg", (c.n_out, c.n_in), "ldw"),
              c.given(wu, "wu", (c.n_out, c.n_in), "ldw"),
              c.given(g, "g", (c.rows, c.n_out), "ldz"),
              c.given(u, "u", (c.rows, c.n_out), "ldz")]
    dx = c.made(c.rows, c.n_in)
    dwg, dwu = c.made(c.n_out, c.n_in), c.made(c.n_out, c.n_in)
    dbg, dbu = (c.made(c.n_out) if bias else None for _ in range(2))
    dg, du = (c.made(c.rows, c.n_out, dtype=c.dtype) for _ in range(2))
    c.run("gated_backward", dpar_gated_backward,
          arrays + [_addresses(t) for t in (dx, dwg, dwu, dbg, dbu, dg, du)])
    out = (dx, dwg, dwu, dbg, dbu) if bias else (dx, dwg, dwu)
    return tuple(c.result(t) for t in out)
