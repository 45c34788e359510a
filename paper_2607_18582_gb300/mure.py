"""Thin ctypes binding of libmure.so (include/mure.h).

Argument marshalling only: every step of the method runs in the library's CUDA
kernels.  Functions carry the C names.  PyTorch supplies device memory (its caching
allocator is handed to the library) and the CUDA stream.  There is no fallback: if
the library has not been built, every call raises.
"""
from __future__ import annotations

import ctypes as C
import os
import sys

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_build", "libmure.so")

STATUS = {0: "MURE_OK", 1: "MURE_ERR_INVALID_ARG", 2: "MURE_ERR_UNSUPPORTED", 3: "MURE_ERR_OOM",
          4: "MURE_ERR_CUDA", 5: "MURE_ERR_TIMEOUT"}
KINDS = {"conv": 0, "dense": 1, "maxpool": 2, "flatten": 3, "add": 4, "gap": 5, "shortcut": 6, "dwconv": 7,
         "embed": 8, "lstm": 9}
ACTS = {"none": 0, "relu": 1, "relu6": 2}
PRECISIONS = {"fp32": 0, "tf32x3": 1, "bf16": 2, "tf32": 3}
TOKEN_DTYPES = {"f32": 0, "f16": 1, "bf16": 2}
TOKEN_FORMS = {"same": 0, "e4m3": 1}

# the exported entry points of include/mure.h
EXPORTS = ("mure_create", "mure_destroy", "mure_last_error", "mure_model_load", "mure_model_free",
           "mure_model_n_layers", "mure_model_layer_kernel", "mure_kernel_launches", "mure_build_prefix_cache", "mure_cache_free", "mure_cache_outputs",
           "mure_eval_mutants", "mure_eval_vanilla", "mure_expand_patches", "mure_expand_patches_noalloc",
           "mure_check_descriptors", "mure_set_wait_limit", "mure_tokens_create", "mure_tokens_free",
           "mure_tokens_buffers", "mure_tokens_plan_create", "mure_tokens_plan_set", "mure_tokens_plan_free",
           "mure_tokens_append", "mure_tokens_read", "mure_tokens_attend", "mure_synchronize")


class MureError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"{STATUS.get(status, status)}: {msg}")
        self.status = status


class _Node(C.Structure):
    _fields_ = [("kind", C.c_int32), ("act", C.c_int32), ("in0", C.c_int32), ("in1", C.c_int32),
                ("kh", C.c_int32), ("kw", C.c_int32), ("stride", C.c_int32), ("pad", C.c_int32),
                ("cin", C.c_int32), ("cout", C.c_int32), ("W", C.c_void_p), ("b", C.c_void_p)]


class _ModelDesc(C.Structure):
    _fields_ = [("in_h", C.c_int32), ("in_w", C.c_int32), ("in_c", C.c_int32), ("n_classes", C.c_int32),
                ("n_nodes", C.c_int32), ("precision", C.c_int32), ("nodes", C.POINTER(_Node))]


MUTANT_DTYPE = np.dtype([("layer", "<i4"), ("op", "<i4"), ("n_neurons", "<i4"), ("tagged", "<i4"),
                         ("neuron_off", "<i8"), ("param", "<f4"), ("reserved2", "<f4"), ("seed", "<u8")])

_ALLOC_FN = C.CFUNCTYPE(C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p)
_FREE_FN = C.CFUNCTYPE(None, C.c_void_p, C.c_void_p, C.c_void_p)


class _Allocator(C.Structure):
    _fields_ = [("alloc", _ALLOC_FN), ("free", _FREE_FN), ("user", C.c_void_p)]


class _Opts(C.Structure):
    _fields_ = [("outputs_on_device", C.c_int32), ("kernel_timing", C.c_int32), ("workspace_bytes", C.c_int64),
                ("logits_out", C.c_void_p), ("skip_unchanged", C.c_int32), ("reserved", C.c_int32)]


class _Stats(C.Structure):
    _fields_ = [("ms_total", C.c_double), ("ms_expand", C.c_double), ("ms_suffix", C.c_double),
                ("ms_score", C.c_double), ("n_rows", C.c_int64), ("n_near_ties", C.c_int64),
                ("n_groups", C.c_int64), ("n_batches", C.c_int64), ("kernel_launches", C.c_int64),
                ("flops", C.c_int64), ("ms_layer", C.c_double * 64), ("flops_layer", C.c_int64 * 64),
                ("launches_layer", C.c_int64 * 64), ("ms_delta", C.c_double), ("ms_delta_values", C.c_double),
                ("ms_epilogue", C.c_double), ("bytes_gather", C.c_int64), ("launches_delta", C.c_int64),
                ("bytes_rows", C.c_int64), ("n_rows_unchanged", C.c_int64), ("launches_delta_values", C.c_int64),
                ("bytes_delta_values", C.c_int64)]

    def as_dict(self):
        out = {}
        for k, _ in self._fields_:
            v = getattr(self, k)
            out[k] = list(v) if hasattr(v, "__len__") else v
        return out


class _TokensDesc(C.Structure):
    _fields_ = [("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("page_size", C.c_int32), ("dtype", C.c_int32),
                ("form", C.c_int32), ("reserved", C.c_int32), ("n_pages", C.c_int64), ("k", C.c_void_p),
                ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p)]


class _TokensBatch(C.Structure):
    _fields_ = [("n_seqs", C.c_int32), ("n_heads", C.c_int32), ("new_len", C.c_void_p), ("pos", C.c_void_p),
                ("kv_len", C.c_void_p), ("page_table", C.c_void_p), ("table_stride", C.c_int64), ("window", C.c_int32),
                ("sinks", C.c_int32), ("scale", C.c_float), ("reserved", C.c_int32)]


class _TokensRows(C.Structure):
    _fields_ = [("p", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


_lib = None
# Allocator thunks stay alive for the life of the process: a context's C object may
# still call them while Python tears objects down in arbitrary (cyclic-GC) order.
_ALLOCATOR_KEEPALIVE = []


def _finalizing():
    return sys is None or sys.is_finalizing()


def lib():
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"libmure.so is not built ({LIB_PATH}); run __graft_entry__.build() "
                               "or python paper_2607_18582_gb300/build.py")
        L = C.CDLL(LIB_PATH)
        vp, i64, i32 = C.c_void_p, C.c_int64, C.c_int32
        L.mure_create.argtypes = [C.c_int, vp, C.POINTER(_Allocator), C.POINTER(vp)]
        L.mure_destroy.argtypes = [vp]
        L.mure_destroy.restype = None
        L.mure_last_error.argtypes = [vp]
        L.mure_last_error.restype = C.c_char_p
        L.mure_model_load.argtypes = [vp, C.POINTER(_ModelDesc), C.POINTER(vp)]
        L.mure_model_free.argtypes = [vp]
        L.mure_model_free.restype = None
        L.mure_model_n_layers.argtypes = [vp]
        L.mure_model_n_layers.restype = i32
        L.mure_model_layer_kernel.argtypes = [vp, i32, C.POINTER(i32), C.POINTER(i64)]
        L.mure_kernel_launches.argtypes = [vp]
        L.mure_kernel_launches.restype = i64
        L.mure_build_prefix_cache.argtypes = [vp, vp, i64, vp, C.c_int, C.POINTER(vp)]
        L.mure_cache_free.argtypes = [vp]
        L.mure_cache_free.restype = None
        L.mure_cache_outputs.argtypes = [vp, vp, vp]
        L.mure_eval_mutants.argtypes = [vp, vp, i64, vp, i64, C.POINTER(_Opts), vp, C.POINTER(C.c_double),
                                        C.POINTER(C.c_double), C.POINTER(_Stats)]
        L.mure_eval_vanilla.argtypes = [vp, vp, i64, vp, C.c_int, vp, i64, vp, i64, C.POINTER(_Opts), vp,
                                        C.POINTER(C.c_double), C.POINTER(C.c_double), C.POINTER(_Stats)]
        L.mure_expand_patches.argtypes = [vp, vp, i64, vp, i64, vp, i64, vp]
        L.mure_expand_patches_noalloc.argtypes = [vp, vp, i64, vp, i64, vp, i64, vp]
        L.mure_check_descriptors.argtypes = [C.POINTER(_ModelDesc), vp, i64, vp, i64, C.c_char_p, C.c_size_t]
        L.mure_set_wait_limit.argtypes = [vp, i64]
        rows = C.POINTER(_TokensRows)
        L.mure_tokens_create.argtypes = [vp, C.POINTER(_TokensDesc), C.POINTER(vp)]
        L.mure_tokens_free.argtypes = [vp]
        L.mure_tokens_free.restype = None
        L.mure_tokens_buffers.argtypes = [vp, C.POINTER(_TokensDesc)]
        L.mure_tokens_plan_create.argtypes = [vp, C.POINTER(_TokensBatch), C.POINTER(vp)]
        L.mure_tokens_plan_set.argtypes = [vp, C.POINTER(_TokensBatch)]
        L.mure_tokens_plan_free.argtypes = [vp]
        L.mure_tokens_plan_free.restype = None
        L.mure_tokens_append.argtypes = [vp, vp, rows, rows]
        L.mure_tokens_read.argtypes = [vp, vp, i32, rows, rows]
        L.mure_tokens_attend.argtypes = [vp, vp, rows, rows, vp]
        L.mure_synchronize.argtypes = [vp]
        for name in EXPORTS:
            if name not in ("mure_destroy", "mure_model_free", "mure_cache_free", "mure_last_error",
                            "mure_model_n_layers", "mure_kernel_launches", "mure_tokens_free",
                            "mure_tokens_plan_free"):
                getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def _ptr(a):
    """Address of a numpy array or a torch tensor (None -> NULL)."""
    if a is None:
        return None
    if hasattr(a, "data_ptr"):
        return a.data_ptr()
    return a.ctypes.data


def _is_device(a):
    return a is not None and hasattr(a, "is_cuda") and a.is_cuda


class Context:
    """Owns a library context.  Models and caches made from it count as children; the
    C context is destroyed only once none is alive (and never during interpreter
    shutdown, when the process frees everything anyway)."""

    def __init__(self, handle, keep, device=0, stream=0):
        self.h = handle
        self.device, self.stream = device, stream   # stream: the cudaStream_t as an integer
        self._keep = keep
        self._children = 0
        self._released = False

    def check(self, status):
        if status != 0:
            msg = lib().mure_last_error(self.h)
            raise MureError(status, msg.decode() if msg else "")

    def _child_gone(self):
        self._children -= 1
        if self._released and self._children == 0:
            self._destroy()

    def _destroy(self):
        if self.h and not _finalizing():
            lib().mure_destroy(self.h)
        self.h = None

    def __del__(self):
        self._released = True
        if getattr(self, "h", None) and self._children == 0:
            self._destroy()


def mure_create(device: int = 0, stream=None, torch_allocator: bool = True) -> Context:
    """A library context on `device` queueing on `stream` (default: torch's current
    stream), allocating through torch's caching allocator."""
    import torch
    if stream is None:
        stream = torch.cuda.current_stream(device)
    handle_stream = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream or 0)
    keep = []
    alloc_p = None
    if torch_allocator:
        def _alloc(nbytes, strm, user):
            try:
                return torch.cuda.caching_allocator_alloc(int(nbytes), device, int(strm or 0))
            except Exception:  # noqa: BLE001 - reported to the library as a NULL allocation
                return None

        def _free(ptr, strm, user):
            torch.cuda.caching_allocator_delete(ptr)

        def _free_guarded(ptr, strm, user):
            if not _finalizing():
                _free(ptr, strm, user)

        a = _Allocator(_ALLOC_FN(_alloc), _FREE_FN(_free_guarded), None)
        keep += [a, a.alloc, a.free]
        _ALLOCATOR_KEEPALIVE.append(keep)
        alloc_p = C.byref(a)
    out = C.c_void_p()
    st = lib().mure_create(device, handle_stream, alloc_p, C.byref(out))
    if st != 0:
        raise MureError(st, "mure_create failed")
    return Context(out.value, keep, device, int(handle_stream or 0))


class Model:
    def __init__(self, ctx, handle, src):
        self.ctx, self.h, self.src = ctx, handle, src
        ctx._children += 1
        self._children = 0
        self._released = False

    @property
    def n_layers(self):
        return lib().mure_model_n_layers(self.h)

    KERNELS = {0: "simt_gemm", 1: "simt_small", 2: "tc_gemm", 3: "tc_window", 4: "output", 5: "tc_conv"}

    def layer_kernel(self, layer):
        """(kernel name, executed multiply-accumulates per batch row) of a layer."""
        k, macs = C.c_int32(), C.c_int64()
        self.ctx.check(lib().mure_model_layer_kernel(self.h, int(layer), C.byref(k), C.byref(macs)))
        return self.KERNELS.get(k.value, str(k.value)), macs.value

    def _child_gone(self):
        self._children -= 1
        if self._released and self._children == 0:
            self._destroy()

    def _destroy(self):
        if self.h:
            if not _finalizing():
                lib().mure_model_free(self.h)
            self.h = None
            self.ctx._child_gone()

    def __del__(self):
        self._released = True
        if getattr(self, "h", None) and self._children == 0:
            self._destroy()


def _model_desc(model, precision):
    """The C description of a network (workloads.Model fields) and the arrays it points to."""
    nodes = (_Node * len(model.nodes))()
    keep = []
    for v, n in enumerate(model.nodes):
        W = None if n.W is None else np.ascontiguousarray(n.W, np.float32)
        b = None if n.b is None else np.ascontiguousarray(n.b, np.float32)
        keep += [W, b]
        ins = list(n.inputs) + [-1] * (2 - len(n.inputs))
        nodes[v] = _Node(KINDS[n.kind], ACTS[n.act], ins[0], ins[1], n.kh, n.kw, n.stride, n.pad, n.cin, n.cout,
                         _ptr(W), _ptr(b))
    h, w, c = model.in_shape
    desc = _ModelDesc(h, w, c, model.n_classes, len(model.nodes), PRECISIONS[precision], nodes)
    return desc, (keep, nodes)


def mure_model_load(ctx: Context, model, precision: str = "fp32") -> Model:
    """Copy a network description (workloads.Model fields) to the device."""
    desc, keep = _model_desc(model, precision)
    out = C.c_void_p()
    ctx.check(lib().mure_model_load(ctx.h, C.byref(desc), C.byref(out)))
    return Model(ctx, out.value, model)


class Cache:
    def __init__(self, model, handle, n_inputs):
        self.model, self.h, self.n_inputs = model, handle, n_inputs
        model._children += 1

    def free(self):
        if getattr(self, "h", None):
            if not _finalizing():
                lib().mure_cache_free(self.h)
            self.h = None
            self.model._child_gone()

    def __del__(self):
        self.free()


def _as_input(X, labels):
    on_dev = _is_device(X)
    if not on_dev:
        X = np.ascontiguousarray(X, np.float32)
        if labels is not None:
            labels = np.ascontiguousarray(labels, np.int32)
    else:
        X = X.contiguous()
        if labels is not None:
            import torch
            labels = labels.to(device=X.device, dtype=torch.int32).contiguous()
    return X, labels, int(on_dev)


def mure_build_prefix_cache(model: Model, X, labels=None) -> Cache:
    """Prefix-activation cache of X (numpy host array or CUDA tensor, NHWC fp32)."""
    X, labels, on_dev = _as_input(X, labels)
    n = int(X.shape[0])
    out = C.c_void_p()
    model.ctx.check(lib().mure_build_prefix_cache(model.h, _ptr(X) if n else None, n, _ptr(labels), on_dev,
                                                  C.byref(out)))
    return Cache(model, out.value, n)


def mure_cache_outputs(cache: Cache):
    """(original logits [n][C], original predictions [n]) held by the cache."""
    C_ = cache.model.src.n_classes
    lg = np.zeros((cache.n_inputs, C_), np.float32)
    pr = np.zeros(cache.n_inputs, np.int32)
    cache.model.ctx.check(lib().mure_cache_outputs(cache.h, _ptr(lg), _ptr(pr)))
    return lg, pr


def table_array(table):
    """A workloads.MutantTable as the C descriptor array and the neuron pool."""
    n = len(table)
    arr = np.zeros(max(n, 1), MUTANT_DTYPE)
    arr["layer"][:n] = table.layer
    arr["op"][:n] = table.op
    arr["n_neurons"][:n] = table.n_neurons
    arr["neuron_off"][:n] = table.neuron_off
    arr["param"][:n] = table.param
    arr["seed"][:n] = table.seed
    if getattr(table, "tagged", None) is not None:
        arr["tagged"][:n] = table.tagged
    pool = np.ascontiguousarray(table.pool, np.int32)
    if pool.size == 0:
        pool = np.zeros(1, np.int32)
    return arr, pool, int(table.pool.size)


def _eval_common(n_mut, n_in, n_classes, logits, outputs_on_device, workspace_bytes, kill_out, kernel_timing=False,
                 skip_unchanged=False):
    W64 = (n_in + 63) // 64
    if outputs_on_device:
        import torch
        kill = kill_out if kill_out is not None else torch.empty((max(n_mut, 1), max(W64, 1)), dtype=torch.int64,
                                                                 device="cuda")
        lg = torch.empty((n_mut, n_in, n_classes), dtype=torch.float32, device="cuda") if logits else None
    else:
        kill = kill_out if kill_out is not None else np.zeros((max(n_mut, 1), max(W64, 1)), np.uint64)
        lg = np.zeros((n_mut, n_in, n_classes), np.float32) if logits else None
    opts = _Opts(int(bool(outputs_on_device)), int(bool(kernel_timing)), int(workspace_bytes), _ptr(lg),
                 int(bool(skip_unchanged)), 0)
    return kill, lg, opts, W64


def _eval_result(kill, lg, sa, sb, st, n_mut, W64, outputs_on_device):
    if outputs_on_device:
        kill = kill[:n_mut, :W64]
    else:
        kill = kill[:n_mut, :W64]
    return {"kill_bits": kill, "scoreA": sa.value, "scoreB": sb.value, "stats": st.as_dict(), "logits": lg}


def mure_eval_mutants(cache: Cache, table, logits: bool = False, outputs_on_device: bool = False,
                      workspace_bytes: int = 0, kill_out=None, kernel_timing: bool = False, arrays=None,
                      skip_unchanged: bool = False):
    """Memoized mutation testing of `table` on the cached inputs (skip_unchanged: the
    exact unchanged-row elimination)."""
    arr, pool, plen = arrays if arrays is not None else table_array(table)
    n = len(table)
    kill, lg, opts, W64 = _eval_common(n, cache.n_inputs, cache.model.src.n_classes, logits, outputs_on_device,
                                       workspace_bytes, kill_out, kernel_timing, skip_unchanged)
    sa, sb, st = C.c_double(), C.c_double(), _Stats()
    cache.model.ctx.check(lib().mure_eval_mutants(cache.h, _ptr(arr), n, _ptr(pool), plen, C.byref(opts), _ptr(kill),
                                                  C.byref(sa), C.byref(sb), C.byref(st)))
    return _eval_result(kill, lg, sa, sb, st, n, W64, outputs_on_device)


def mure_eval_vanilla(model: Model, X, table, labels=None, logits: bool = False, outputs_on_device: bool = False,
                      workspace_bytes: int = 0, kill_out=None, kernel_timing: bool = False):
    """Vanilla mutation testing: every mutant end to end from X."""
    X, labels, on_dev = _as_input(X, labels)
    arr, pool, plen = table_array(table)
    n = len(table)
    n_in = int(X.shape[0])
    kill, lg, opts, W64 = _eval_common(n, n_in, model.src.n_classes, logits, outputs_on_device, workspace_bytes,
                                       kill_out, kernel_timing)
    sa, sb, st = C.c_double(), C.c_double(), _Stats()
    model.ctx.check(lib().mure_eval_vanilla(model.h, _ptr(X) if n_in else None, n_in, _ptr(labels), on_dev, _ptr(arr),
                                            n, _ptr(pool), plen, C.byref(opts), _ptr(kill), C.byref(sa), C.byref(sb),
                                            C.byref(st)))
    return _eval_result(kill, lg, sa, sb, st, n, W64, outputs_on_device)


def mure_kernel_launches(ctx: Context) -> int:
    """Kernels the context has launched since it was created."""
    return int(lib().mure_kernel_launches(ctx.h))


def mure_set_wait_limit(ctx: Context, cycles: int) -> None:
    """Limit of the tensor-core kernels' device-side waits in SM cycles (0: default)."""
    ctx.check(lib().mure_set_wait_limit(ctx.h, int(cycles)))


def mure_expand_patches(model: Model, table):
    """GF noise / WS-permuted weights of every GF or WS mutant: (values, offsets)."""
    arr, pool, plen = table_array(table)
    n = len(table)
    need = 0
    for i in range(n):
        if int(table.op[i]) in (0, 4):
            layer = model.src.nodes[model.src.layers()[int(table.layer[i])]]
            fan = layer.kh * layer.kw * layer.cin if layer.kind == "conv" else layer.cin
            need += int(table.n_neurons[i]) * fan
    out = np.zeros(max(need, 1), np.float32)
    offs = np.zeros(max(n, 1), np.int64)
    model.ctx.check(lib().mure_expand_patches(model.h, _ptr(arr), n, _ptr(pool), plen, _ptr(out), need, _ptr(offs)))
    return out[:need], offs[:n]


def mure_expand_patches_noalloc(model: Model, table, out_dev):
    """mure_expand_patches into a caller-provided CUDA float32 tensor, with no device
    allocation by the library; returns the offsets (host)."""
    arr, pool, plen = table_array(table)
    n = len(table)
    offs = np.zeros(max(n, 1), np.int64)
    model.ctx.check(lib().mure_expand_patches_noalloc(model.h, _ptr(arr), n, _ptr(pool), plen, _ptr(out_dev),
                                                      int(out_dev.numel()), _ptr(offs)))
    return offs[:n]


def mure_check_descriptors(model, table=None, precision: str = "fp32"):
    """Host-side validation of a network description and (optionally) a mutant table,
    with no context and no device: (status, reason); status 0 = MURE_OK."""
    desc, keep = _model_desc(model, precision)
    arr, pool, plen = table_array(table) if table is not None else (None, None, 0)
    n = len(table) if table is not None else 0
    msg = C.create_string_buffer(512)
    st = lib().mure_check_descriptors(C.byref(desc), _ptr(arr) if n else None, n,
                                      _ptr(pool) if plen else None, plen, msg, 512)
    return int(st), msg.value.decode()


# ----------------------------------------------------------------- token caches --

class Tokens:
    """A paged cache of one attention layer's keys and values (mure_tokens)."""

    def __init__(self, ctx, handle, desc, dtype, form, keep):
        self.ctx, self.h, self.dtype, self.form = ctx, handle, dtype, form
        self.n_kv_heads, self.head_dim, self.page_size = desc.n_kv_heads, desc.head_dim, desc.page_size
        self.n_pages = desc.n_pages
        import torch
        self.torch_dtype, self.torch_device = _torch_dtype(dtype), torch.device("cuda", ctx.device)
        self._keep = keep          # the caller's pools
        ctx._children += 1

    def free(self):
        if getattr(self, "h", None):
            if not _finalizing():
                lib().mure_tokens_free(self.h)
            self.h = None
            self.ctx._child_gone()

    def __del__(self):
        self.free()


class TokensPlan:
    """One batch's sequences, laid out on the device (mure_tokens_plan)."""

    def __init__(self, ctx, handle, n_heads):
        self.ctx, self.h = ctx, handle
        ctx._children += 1

    def free(self):
        if getattr(self, "h", None):
            if not _finalizing():
                lib().mure_tokens_plan_free(self.h)
            self.h = None
            self.ctx._child_gone()

    def __del__(self):
        self.free()


def _torch_dtype(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def mure_tokens_create(ctx: Context, n_kv_heads: int, head_dim: int, page_size: int, n_pages: int, dtype: str = "bf16",
                       form: str = "same", buffers=None) -> Tokens:
    """A cache of n_pages pages.  buffers: the caller's pools as CUDA tensors, (k, v) or with form
    "e4m3" (k, v, k_scale, v_scale), [n_pages][n_kv_heads][page_size][head_dim] (scales: without the
    last dimension); by default the library allocates them, filled with zeros."""
    d = _TokensDesc(_whole(n_kv_heads, "n_kv_heads"), _whole(head_dim, "head_dim"), _whole(page_size, "page_size"),
                    TOKEN_DTYPES[dtype], TOKEN_FORMS[form], 0, _whole(n_pages, "n_pages", 64))
    if buffers is not None:
        import torch
        if len(buffers) != (4 if form == "e4m3" else 2):
            raise ValueError("buffers: (k, v), with e4m3 cells (k, v, k_scale, v_scale)")
        shape = (d.n_pages, d.n_kv_heads, d.page_size, d.head_dim)
        for i, b in enumerate(buffers):
            want = shape if i < 2 else shape[:3]
            types = ((_torch_dtype(dtype),) if form == "same" else (torch.float8_e4m3fn, torch.uint8)) if i < 2 else (torch.uint8,)
            if tuple(b.shape) != want or b.dtype not in types or not b.is_contiguous() or not b.is_cuda or b.device.index != ctx.device:
                raise ValueError(f"buffers[{i}]: a contiguous CUDA tensor {want} of {types[0]} on device {ctx.device} is wanted")
        _enter(ctx, buffers)
        d.k, d.v = buffers[0].data_ptr(), buffers[1].data_ptr()
        if form == "e4m3":
            d.k_scale, d.v_scale = buffers[2].data_ptr(), buffers[3].data_ptr()
    out = C.c_void_p()
    ctx.check(lib().mure_tokens_create(ctx.h, C.byref(d), C.byref(out)))
    return Tokens(ctx, out.value, d, dtype, form, buffers)


def _whole(x, name, bits=32):
    """A whole number that an integer of so many bits holds."""
    x = int(x)
    if not -1 << (bits - 1) <= x < 1 << (bits - 1):
        raise ValueError(f"{name}: {x} does not fit {bits} bits")
    return x


def _int32(a, name, past=None):
    """Whole numbers as a dense int32 array.  past: what stands for one that does not fit (None: refused)."""
    a = np.asarray(a)
    if a.dtype == np.int32 or a.size == 0:
        return np.ascontiguousarray(a, np.int32)
    if a.dtype.kind not in "biuf":
        raise ValueError(f"{name}: whole numbers are wanted")
    fits = (a >= -2 ** 31) & (a < 2 ** 31) if a.dtype.kind == "f" else None
    if fits is None or fits.all():
        b = np.ascontiguousarray(a).astype(np.int32)
        same = b == a
        if same.all():
            return b
    if a.dtype.kind == "f" or past is None:
        raise ValueError(f"{name}: whole numbers of 32 bits are wanted")
    b[~same] = past
    return b


def _tokens_batch(n_heads, new_len, pos, kv_len, page_table, window, sinks, scale):
    new_len, pos, kv_len = (_int32(a, name).reshape(-1)
                            for a, name in ((new_len, "new_len"), (pos, "pos"), (kv_len, "kv_len")))
    n = len(new_len)
    if len(pos) != n or len(kv_len) != n:
        raise ValueError("new_len, pos and kv_len have different lengths")
    # (an id that does not fit is none; the library refuses it where a sequence's cells need it)
    table = _int32(page_table, "page_table", past=-1)
    if table.ndim != 2 or table.shape[0] < n:
        raise ValueError("page_table: a row of page ids for every sequence")
    b = _TokensBatch(n, _whole(n_heads, "n_heads"), _ptr(new_len), _ptr(pos), _ptr(kv_len), _ptr(table), table.shape[1],
                     _whole(window, "window"), _whole(sinks, "sinks"), float(scale or 0.0), 0)
    return b, (new_len, pos, kv_len, table)


def mure_tokens_plan(tokens: Tokens, n_heads: int, new_len, pos, kv_len, page_table, window: int = 0, sinks: int = 0,
                     scale: float = 0.0, plan: TokensPlan = None) -> TokensPlan:
    """Lay out a batch for caches of `tokens`' geometry: sequence b has kv_len[b] cells in the pages
    page_table[b] and new_len[b] new tokens from position pos[b] on.  plan: an existing plan that
    takes the batch (a decoding loop's next step)."""
    b, keep = _tokens_batch(n_heads, new_len, pos, kv_len, page_table, window, sinks, scale)
    ctx = tokens.ctx
    if plan is None:
        out = C.c_void_p()
        ctx.check(lib().mure_tokens_plan_create(tokens.h, C.byref(b), C.byref(out)))
        plan = TokensPlan(ctx, out.value, int(n_heads))
    else:
        ctx.check(lib().mure_tokens_plan_set(plan.h, C.byref(b)))
    plan.n_heads = int(n_heads)
    plan.n_new, plan.n_cells = int(keep[0].sum(dtype=np.int64)), int(keep[2].sum(dtype=np.int64))
    return plan


def _raw_stream(device):
    """torch's current stream as an integer (by its own short way where it has one)."""
    global _raw_stream
    import torch
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
        lambda d: torch.cuda.current_stream(d).cuda_stream)
    return _raw_stream(device)


def _enter(ctx, tensors):
    """Where torch's current stream is not the context's: the context's stream waits for what is
    queued on it, and the tensors' memory is kept until the context's stream is done with it."""
    if _raw_stream(ctx.device) == ctx.stream:
        return None
    import torch
    cur = torch.cuda.current_stream(ctx.device)
    mine = torch.cuda.ExternalStream(ctx.stream, device=ctx.device) if ctx.stream else torch.cuda.default_stream(ctx.device)
    mine.wait_stream(cur)
    for t in tensors:
        if t is not None:
            t.record_stream(mine)
    return cur, mine


def _leave(streams):
    if streams is not None:
        streams[0].wait_stream(streams[1])


def _grad_enabled():
    import torch
    return torch.is_grad_enabled()


def _token_rows(t, tokens, n, heads, name):
    if t.requires_grad and _grad_enabled():
        raise ValueError(f"{name} requires a gradient, and token caches record none: detach it or call under torch.no_grad()")
    if t.dtype is not tokens.torch_dtype or t.device != tokens.torch_device:
        raise ValueError(f"{name}: a {tokens.torch_dtype} tensor on {tokens.torch_device} is wanted")
    s = t.stride()
    if t.shape != (n, heads, tokens.head_dim) or (n and s[2] != 1):
        raise ValueError(f"{name}: shape {(n, heads, tokens.head_dim)} with a dense last dimension is wanted, "
                         f"got {tuple(t.shape)}, strides {s}")
    return _TokensRows(t.data_ptr(), s[0], s[1])


def mure_tokens_append(tokens: Tokens, plan: TokensPlan, k, v) -> None:
    """Write the batch's new tokens' keys and values [tokens][n_kv_heads][head_dim] (any token and head
    strides) into their cells."""
    ctx = tokens.ctx
    kr = _token_rows(k, tokens, plan.n_new, tokens.n_kv_heads, "k")
    vr = _token_rows(v, tokens, plan.n_new, tokens.n_kv_heads, "v")
    st = _enter(ctx, (k, v))
    ctx.check(lib().mure_tokens_append(tokens.h, plan.h, kr, vr))
    _leave(st)


def mure_tokens_read(tokens: Tokens, plan: TokensPlan, new: bool = False, out=None):
    """(k, v) [cells][n_kv_heads][head_dim] of all the batch's cells, sequence after sequence (new: of
    its new tokens' cells)."""
    import torch
    ctx, heads, dim = tokens.ctx, tokens.n_kv_heads, tokens.head_dim
    n = plan.n_new if new else plan.n_cells
    if out is None:
        out = (torch.empty((n, heads, dim), dtype=tokens.torch_dtype, device=tokens.torch_device),
               torch.empty((n, heads, dim), dtype=tokens.torch_dtype, device=tokens.torch_device))
        kr, vr = (_TokensRows(x.data_ptr(), heads * dim, dim) for x in out)
    else:
        kr = _token_rows(out[0], tokens, n, heads, "out[0]")
        vr = _token_rows(out[1], tokens, n, heads, "out[1]")
    st = _enter(ctx, out)
    ctx.check(lib().mure_tokens_read(tokens.h, plan.h, 1 if new else 0, kr, vr))
    _leave(st)
    return out


def mure_tokens_attend(tokens: Tokens, plan: TokensPlan, q, out=None, lse: bool = False):
    """Attention of the batch's new tokens q [tokens][n_heads][head_dim] over their sequences' cells:
    out (same shape), with lse=True also the logs of the rows' sums, fp32 [tokens][n_heads].  Token caches
    record no gradients: rows that require one are refused unless under torch.no_grad()."""
    import torch
    ctx, n = tokens.ctx, plan.n_new
    qr = _token_rows(q, tokens, n, plan.n_heads, "q")
    if out is None:
        out = torch.empty((n, plan.n_heads, tokens.head_dim), dtype=tokens.torch_dtype, device=tokens.torch_device)
        orow = _TokensRows(out.data_ptr(), plan.n_heads * tokens.head_dim, tokens.head_dim)
    else:
        orow = _token_rows(out, tokens, n, plan.n_heads, "out")
    ls = torch.empty((n, plan.n_heads), dtype=torch.float32, device=tokens.torch_device) if lse else None
    st = _enter(ctx, (q, out, ls))
    ctx.check(lib().mure_tokens_attend(tokens.h, plan.h, qr, orow, ls.data_ptr() if lse else None))
    _leave(st)
    return (out, ls) if lse else out


def mure_synchronize(ctx: Context) -> None:
    """Wait for everything queued on the context's stream; raises if a device-side check failed."""
    ctx.check(lib().mure_synchronize(ctx.h))
