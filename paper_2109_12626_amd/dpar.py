"""Python binding of libdpar.so (include/dpar.h).

Argument marshalling only: every step of the reduction runs in the library's
HIP kernels.  The functions keep the C names.  torch is imported first so that
the library binds to the HIP runtime torch already loaded (one runtime per
process); torch serves only for device memory and streams.
"""

import contextlib
import ctypes
import os

import numpy as np

import torch  # noqa: F401  (must precede loading libdpar: one HIP runtime)
from torch.autograd import forward_ad

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("DPAR_LIB_PATH") or os.path.join(_HERE, "libdpar.so")

DPAR_SUCCESS = 0
DPAR_ERR_INVALID_ARG = -1
DPAR_ERR_UNSUPPORTED = -2
DPAR_ERR_ALIAS = -3
DPAR_ERR_NOMEM = -4
DPAR_ERR_HIP = -5
DPAR_ERR_TIMEOUT = -6

DPAR_INT32, DPAR_FLOAT32, DPAR_U32_MAT2X2, DPAR_BFLOAT16, DPAR_FLOAT16, \
    DPAR_INT8 = 0, 1, 2, 3, 4, 5
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
          "float16": DPAR_FLOAT16, "int8": DPAR_INT8}
OPS = {"sum": DPAR_SUM, "max": DPAR_MAX, "matmul": DPAR_MATMUL}
EXECS = {"auto": DPAR_EXEC_AUTO, "launch": DPAR_EXEC_LAUNCH_PER_ROUND,
         "barrier": DPAR_EXEC_GRID_BARRIER, "ticket": DPAR_EXEC_TICKET,
         "split": DPAR_EXEC_SPLIT, "rounds": DPAR_EXEC_ROUNDS,
         "rounds_barrier": DPAR_EXEC_ROUNDS_BARRIER}
ALGS = {"dual": DPAR_ALG_DUAL_ROOT, "single": DPAR_ALG_SINGLE_TREE,
        "reduce_bcast": DPAR_ALG_REDUCE_BCAST}

ACTS = {"none": DPAR_ACT_NONE, "relu": DPAR_ACT_RELU, "gelu": DPAR_ACT_GELU,
        "gelu_tanh": DPAR_ACT_GELU_TANH, "silu": DPAR_ACT_SILU}
DPAR_ROUTE_SOFTMAX, DPAR_ROUTE_SIGMOID = 0, 1
ROUTES = {"softmax": DPAR_ROUTE_SOFTMAX, "sigmoid": DPAR_ROUTE_SIGMOID}
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


class dpar_quantize_t(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_size_t), ("cols", ctypes.c_size_t),
                ("dtype", ctypes.c_int), ("ldx", ctypes.c_size_t),
                ("ldq", ctypes.c_size_t)]


class dpar_moe_t(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_size_t), ("in_", ctypes.c_size_t),
                ("hidden", ctypes.c_size_t), ("experts", ctypes.c_size_t),
                ("top", ctypes.c_int), ("dtype", ctypes.c_int),
                ("weight_dtype", ctypes.c_int), ("out_dtype", ctypes.c_int),
                ("act", ctypes.c_int), ("route", ctypes.c_int),
                ("normalize", ctypes.c_int), ("weight_scale", ctypes.c_float),
                ("ldx", ctypes.c_size_t), ("ldl", ctypes.c_size_t),
                ("ldw", ctypes.c_size_t), ("ldd", ctypes.c_size_t),
                ("xw", ctypes.c_size_t), ("xd", ctypes.c_size_t),
                ("ldy", ctypes.c_size_t), ("ldr", ctypes.c_size_t)]


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
    L.dpar_quantize.argtypes = [vp] * 3 + [i, ctypes.POINTER(dpar_quantize_t),
                                           vp]
    L.dpar_linear_int8.argtypes = [vp] * 7 + tail
    L.dpar_gated_int8.argtypes = [vp] * 9 + tail
    moe = ctypes.POINTER(dpar_moe_t)
    L.dpar_moe.argtypes = [vp] * 12 + [i, moe, vp, sz, vp]
    L.dpar_moe_workspace.argtypes = [i, moe, ctypes.POINTER(sz)]
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
                 "dpar_product_workspace", "dpar_quantize",
                 "dpar_linear_int8", "dpar_gated_int8", "dpar_moe",
                 "dpar_moe_workspace"):
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


def quantize_options(rows, cols, dtype, ldx=0, ldq=0):
    """Sizes, type of x and row distances of a quantisation
    (dpar_quantize_t)."""
    return dpar_quantize_t(rows, cols, _enum(DTYPES, dtype), ldx, ldq)


def dpar_quantize(x, q, scale, p, opt, stream=None):
    """Sequences of p device addresses; opt: quantize_options()."""
    if isinstance(stream, torch.cuda.Stream):
        stream = stream.cuda_stream
    rc = lib().dpar_quantize(_ptr_array(x), _ptr_array(q), _ptr_array(scale),
                             p, ctypes.byref(opt), stream)
    return rc if rc >= 0 else _check(rc)


def dpar_linear_int8(x, sx, w, sw, bias, residual, y, p, opt, workspace=None,
                     workspace_bytes=0, stream=None):
    """As dpar_linear; opt: product_options() with dtype "int8"."""
    return _product(lib().dpar_linear_int8, (x, sx, w, sw, bias, residual, y),
                    p, opt, workspace, workspace_bytes, stream)


def dpar_gated_int8(x, sx, wg, sg, wu, su, bg, bu, h, p, opt, workspace=None,
                    workspace_bytes=0, stream=None):
    return _product(lib().dpar_gated_int8,
                    (x, sx, wg, sg, wu, su, bg, bu, h), p, opt, workspace,
                    workspace_bytes, stream)


def moe_options(tokens, n_in, hidden, experts, top, dtype, weight_dtype=None,
                out_dtype=None, act="silu", route="softmax", normalize=True,
                weight_scale=1.0, ldx=0, ldl=0, ldw=0, ldd=0, xw=0, xd=0,
                ldy=0, ldr=0):
    """Sizes, types and distances of a mixture-of-experts layer (dpar_moe_t);
    experts: of each rank."""
    dt = _enum(DTYPES, dtype)
    return dpar_moe_t(tokens, n_in, hidden, experts, top, dt,
                      dt if weight_dtype is None
                      else _enum(DTYPES, weight_dtype),
                      dt if out_dtype is None else _enum(DTYPES, out_dtype),
                      _enum(ACTS, act), _enum(ROUTES, route), int(normalize),
                      weight_scale, ldx, ldl, ldw, ldd, xw, xd, ldy, ldr)


def dpar_moe(x, logits, wg, wu, wd, sg, su, sd, residual, y, index, weight, p,
             opt, workspace=None, workspace_bytes=0, stream=None):
    """Sequences of p device addresses (0 where a rank has no residual, index
    or weight), or None where optional; opt: moe_options()."""
    return _product(lib().dpar_moe,
                    (x, logits, wg, wu, wd, sg, su, sd, residual, y, index,
                     weight), p, opt, workspace, workspace_bytes, stream)


def dpar_moe_workspace(p, opt):
    out = ctypes.c_size_t()
    _check(lib().dpar_moe_workspace(int(p), ctypes.byref(opt),
                                    ctypes.byref(out)))
    return out.value


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
# for autograd: tensors that require a gradient are refused where it is on, and
# so are those that carry a tangent of forward mode.

_NAMES = {torch.float32: "float32", torch.bfloat16: "bfloat16",
          torch.float16: "float16"}


def _on(device):
    """Work for tensors of this device: the library asks for the current
    device's properties and launches there."""
    if device.index in (None, torch.cuda.current_device()):
        return contextlib.nullcontext()
    return torch.cuda.device(device)


def _no_derivative(t, name, advice):
    """Refuses a tensor whose gradient or tangent the call would drop."""
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient, and {advice}")
    if t.is_floating_point() and torch._C._is_fwd_grad_enabled() \
            and forward_ad.unpack_dual(t).tangent is not None:
        raise ValueError(f"{name} carries a tangent of forward mode, and no "
                         "call here has one: take its primal")


class _Call:
    """Shapes, row distances and addresses of one call's tensors."""

    types = _NAMES

    def __init__(self, w, rows_, out_dtype, act):
        self.flat = w.dim() == 2
        self.p = 1 if self.flat else w.shape[0]
        self.n_out, self.n_in = w.shape[-2:]
        self.rows = rows_
        self.dtype = w.dtype
        self.out_dtype = w.dtype if out_dtype is None else out_dtype
        if w.dtype not in self.types or self.out_dtype not in _NAMES:
            raise ValueError(f"types {w.dtype}, {self.out_dtype}")
        self.opt = product_options(rows_, self.n_in, self.n_out,
                                   self.types[w.dtype],
                                   _NAMES[self.out_dtype], act)
        self.device = w.device

    def given(self, t, name, shape, ld=None, dtype=None):
        """Addresses of an operand's ranks; sets its row distance."""
        if t is None:
            return None
        if t.device != self.device or t.dtype != (dtype or self.dtype):
            raise ValueError(f"{name}: {t.dtype} on {t.device}")
        _no_derivative(t, name, "these calls record none: call under "
                       "torch.no_grad() (or detach it) and use the backward "
                       "call")
        one = t.dim() == len(shape)
        if tuple(t.shape[-len(shape):]) != shape or \
                not (one or (t.dim() == len(shape) + 1
                             and t.shape[0] == self.p)):
            raise ValueError(f"{name}: shape {tuple(t.shape)}, want "
                             f"{shape} or {(self.p,) + shape}")
        if one and self.p > 1 and name not in ("x", "sx", "dy", "dh"):
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
        with _on(self.device):
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


# The 8-bit products: x and weights int8, their scales float32 [.., rows] and
# [.., out]; the result, biases and residual have out_dtype.

class _Int8Call(_Call):
    types = {torch.int8: "int8"}


def quantize(x):
    """(q, scale): the rows of x [p, rows, cols] or [rows, cols] as whole
    numbers of 8 bits and what a step of each row is."""
    if x.dim() not in (2, 3) or x.dtype not in _NAMES:
        raise ValueError(f"x: {x.dtype}, shape {tuple(x.shape)}")
    _no_derivative(x, "x", "rounding has none: call under torch.no_grad() or "
                   "detach it")
    t = x if x.dim() == 3 else x[None]
    p, n, cols = t.shape
    if cols > 1 and t.stride(-1) != 1:
        raise ValueError("x: values of a row are not consecutive")
    far = t.stride(-2) if n > 1 else cols
    if far < cols:
        raise ValueError(f"x: rows {far} values apart overlap")
    q = torch.empty(p, n, cols, dtype=torch.int8, device=x.device)
    scale = torch.empty(p, n, dtype=torch.float32, device=x.device)
    with _on(x.device):
        dpar_quantize(rows(t), rows(q), rows(scale), p,
                      quantize_options(n, cols, _NAMES[x.dtype], far),
                      torch.cuda.current_stream(x.device))
    return (q, scale) if x.dim() == 3 else (q[0], scale[0])


def linear_int8(x, sx, w, sw, bias=None, residual=None, act="none",
                out_dtype=torch.bfloat16):
    """act(sx sw (x w^T) + bias) + residual."""
    c = _Int8Call(w, x.shape[-2], out_dtype, act)
    f32 = torch.float32
    y = c.made(c.rows, c.n_out)
    c.run("linear", dpar_linear_int8,
          [c.given(x, "x", (c.rows, c.n_in), "ldx"),
           c.given(sx, "sx", (c.rows,), dtype=f32),
           c.given(w, "w", (c.n_out, c.n_in), "ldw"),
           c.given(sw, "sw", (c.n_out,), dtype=f32),
           c.given(bias, "bias", (c.n_out,), dtype=c.out_dtype),
           c.given(residual, "residual", (c.rows, c.n_out), "ldr",
                   c.out_dtype), _addresses(y)])
    return c.result(y)


def gated_int8(x, sx, wg, sg, wu, su, bg=None, bu=None, act="silu",
               out_dtype=torch.bfloat16):
    """act(sx sg (x wg^T) + bg) * (sx su (x wu^T) + bu)."""
    c = _Int8Call(wg, x.shape[-2], out_dtype, act)
    f32 = torch.float32
    h = c.made(c.rows, c.n_out)
    c.run("gated", dpar_gated_int8,
          [c.given(x, "x", (c.rows, c.n_in), "ldx"),
           c.given(sx, "sx", (c.rows,), dtype=f32),
           c.given(wg, "wg", (c.n_out, c.n_in), "ldw"),
           c.given(sg, "sg", (c.n_out,), dtype=f32),
           c.given(wu, "wu", (c.n_out, c.n_in), "ldw"),
           c.given(su, "su", (c.n_out,), dtype=f32),
           c.given(bg, "bg", (c.n_out,), dtype=c.out_dtype),
           c.given(bu, "bu", (c.n_out,), dtype=c.out_dtype), _addresses(h)])
    return c.result(h)


def moe(x, logits, wg, wu, wd, top=None, sg=None, su=None, sd=None,
        residual=None, act="silu", route="softmax", normalize=True,
        weight_scale=1.0, out_dtype=None, index=None, weight=None):
    """A mixture-of-experts layer: (y, index, weight).  x [tokens, in]; wg, wu
    [experts, hidden, in] and wd [experts, in, hidden], or [p, experts, ...]:
    then y is [p, tokens, in], the ranks' parts; int8 weights with their scales
    sg, su [.., experts, hidden], sd [.., experts, in].  logits [tokens,
    experts of all ranks] with `top`, or logits None and the choice in index
    and weight [tokens, top] (int32, float32)."""
    flat = wg.dim() == 3
    if wg.dim() not in (3, 4) or wu.shape != wg.shape \
            or wd.dim() != wg.dim() or x.dim() != 2:
        raise ValueError("x [tokens, in], weights [(p,) experts, .., ..]")
    lead = wg.shape[:-2]
    p, experts = (1, lead[0]) if flat else lead
    hidden, n_in = wg.shape[-2:]
    tokens = x.shape[0]
    eight = wg.dtype == torch.int8
    out_dtype = x.dtype if out_dtype is None else out_dtype
    if x.dtype not in _NAMES or out_dtype not in _NAMES \
            or not (eight or wg.dtype == x.dtype):
        raise ValueError(f"types {x.dtype}, {wg.dtype}, {out_dtype}")

    def checked(t, name, shape, dtype):
        if t is None:
            raise ValueError(f"{name} is missing")
        if tuple(t.shape) != tuple(shape) or t.dtype != dtype \
                or t.device != x.device:
            raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)} on "
                             f"{t.device}, want {dtype} {tuple(shape)}")
        _no_derivative(t, name, "this call has no backward pass")
        return t

    def row_distance(t, name):
        if t.shape[-1] > 1 and t.stride(-1) != 1:
            raise ValueError(f"{name}: values of a row are not consecutive")
        far = t.stride(-2) if t.shape[-2] > 1 else t.shape[-1]
        if far < t.shape[-1]:
            raise ValueError(f"{name}: rows {far} values apart overlap")
        return far

    def each(t):                       # the same for all ranks
        return pointers([t.data_ptr()] * p)

    def split(t):
        return each(t) if flat else rows(t)

    def matrices(t, name, shape):
        far = row_distance(checked(t, name, lead + shape, wg.dtype), name)
        apart = t.stride(-3) if experts > 1 else shape[0] * far
        if apart < (shape[0] - 1) * far + shape[1]:
            raise ValueError(f"{name}: matrices {apart} values apart overlap")
        return far, apart

    checked(x, "x", (tokens, n_in), x.dtype)
    at_w, at_u = (matrices(t, k, (hidden, n_in))
                  for t, k in ((wg, "wg"), (wu, "wu")))
    if at_w != at_u:
        raise ValueError("wu: other distances than wg's")
    at_d = matrices(wd, "wd", (n_in, hidden))
    scales = []
    for t, k, n in ((sg, "sg", hidden), (su, "su", hidden), (sd, "sd", n_in)):
        if eight:
            checked(t, k, lead + (n,), torch.float32)
            if not t.is_contiguous():
                raise ValueError(f"{k}: not contiguous")
        elif t is not None:
            raise ValueError(f"{k}: scales of {wg.dtype} weights")
        scales.append(split(t) if eight else None)
    if logits is None:
        if index is None or weight is None or index.dim() != 2:
            raise ValueError("neither logits nor a choice")
        top = index.shape[1]
        index = checked(index, "index", (tokens, top), torch.int32)
        weight = checked(weight, "weight", (tokens, top), torch.float32)
        index, weight = index.contiguous(), weight.contiguous()
        choice = [each(index), each(weight)]
        ldl = 0
    else:
        if index is not None or weight is not None or top is None:
            raise ValueError("logits with `top`, or index and weight")
        checked(logits, "logits", (tokens, p * experts), torch.float32)
        ldl = row_distance(logits, "logits")
        index = torch.empty(tokens, top, dtype=torch.int32, device=x.device)
        weight = torch.empty(tokens, top, device=x.device)
        choice = [pointers([t.data_ptr()] + [0] * (p - 1))
                  for t in (index, weight)]
    ldr = 0
    if residual is not None:
        checked(residual, "residual", (tokens, n_in) if flat else
                (p, tokens, n_in), out_dtype)
        ldr = row_distance(residual, "residual")
    y = torch.empty((p, tokens, n_in), dtype=out_dtype, device=x.device)
    opt = moe_options(tokens, n_in, hidden, experts, top, _NAMES[x.dtype],
                      "int8" if eight else None, _NAMES[out_dtype], act, route,
                      normalize, weight_scale, row_distance(x, "x"), ldl,
                      at_w[0], at_d[0], at_w[1], at_d[1], n_in, ldr)
    n = dpar_moe_workspace(p, opt)
    ws = torch.empty(n, dtype=torch.uint8, device=x.device)
    with _on(x.device):
        dpar_moe(each(x), None if logits is None else each(logits), split(wg),
                 split(wu), split(wd), *scales,
                 None if residual is None else split(residual), rows(y),
                 *choice, p, opt, ws, n, torch.cuda.current_stream(x.device))
    return (y[0] if flat else y), index, weight
