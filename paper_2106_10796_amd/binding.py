"""Binding of libcdsgd.so: argument marshalling only.

Every step of the path runs in the HIP kernels behind the C ABI (include/cdsgd.h).
PyTorch is used for device memory and the current stream, nothing else.  There
is no fallback: a missing library is an error.

The calls that a program makes per tensor or per step are marshalled in native code (csrc/py_calls.cpp), which
declines (-1) whatever is not plainly good; ctypes and the checks below then convert it or say what is wrong.  Where
that module is not there, or was built for another library, torch or Python, ctypes serves every call.
"""
import ctypes
import os
import sysconfig
from typing import NamedTuple

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libcdsgd.so")

MAX_WORKERS = 64
STATIC_MAX_TENSORS, STATIC_MAX_CHUNKS, STATIC_CHUNK_ELEMS = 1024, 524288, 4096   # cdsgd_step_fused_static
PASS_WARMUP, PASS_COMPRESSED, PASS_CORRECTION = 0, 1, 2
GRAD_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}   # cdsgd_grad_dtype
OK, ERR_NULL, ERR_SIZE, ERR_PARAM, ERR_ALIGN, ERR_WORKERS, ERR_DEVICE, ERR_ALIAS = range(8)


class CdsgdError(RuntimeError):
    def __init__(self, status, where):
        self.status = int(status)
        msg = lib().cdsgd_status_string(int(status)).decode()
        super().__init__("%s: status %d (%s)" % (where, self.status, msg))


class cdsgd_tensor(ctypes.Structure):
    _fields_ = [("w_global", ctypes.c_void_p), ("w_local", ctypes.c_void_p),
                ("residual", ctypes.c_void_p), ("grad", ctypes.c_void_p),
                ("packed_self", ctypes.c_void_p), ("agg_full", ctypes.c_void_p),
                ("n", ctypes.c_size_t)]


class cdsgd_cost_params(ctypes.Structure):
    _fields_ = [("tau", ctypes.c_double), ("phi", ctypes.c_double), ("psi", ctypes.c_double),
                ("delta", ctypes.c_double), ("k", ctypes.c_int)]


class cdsgd_cost(ctypes.Structure):
    _fields_ = [("t_ssgd", ctypes.c_double), ("t_loc", ctypes.c_double), ("t_bit", ctypes.c_double),
                ("phi_cd", ctypes.c_double), ("t_cd", ctypes.c_double), ("save_vs_bit", ctypes.c_double),
                ("save_vs_loc", ctypes.c_double), ("case_bit", ctypes.c_int), ("case_loc", ctypes.c_int),
                ("eq9_assumption_holds", ctypes.c_int)]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


class cdsgd_adamw_tensor(ctypes.Structure):
    _fields_ = [("weight", ctypes.c_void_p), ("weight16", ctypes.c_void_p), ("grad", ctypes.c_void_p),
                ("m", ctypes.c_void_p), ("v", ctypes.c_void_p), ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("n", ctypes.c_size_t), ("weight_decay", ctypes.c_float)]


class _Declines:
    """In the place of the native calls: every call declines."""

    def __getattr__(self, name):
        return self._decline

    @staticmethod
    def _decline(*_):
        return -1


_lib = None
_calls = _Declines()

# in the order in which _calls.bind takes them
_CALLED = ("cdsgd_quantize_pack", "cdsgd_decode_sum", "cdsgd_decode_sum_sparse", "cdsgd_update", "cdsgd_sparse_encode",
           "cdsgd_sparse_words", "cdsgd_sparse_segments", "cdsgd_step_fused", "cdsgd_step_fused_range",
           "cdsgd_step_fused_static", "cdsgd_grad_norm_compute", "cdsgd_adamw_step", "cdsgd_adamw_grad_norm",
           "cdsgd_adamw_read_states", "cdsgd_mxfp4_quantize", "cdsgd_mxfp4_dequantize", "cdsgd_mxfp4_matmul")


def _native():
    """The native calls, bound to the loaded library; loads it."""
    if _lib is None:
        lib()
    return _calls


def _load_calls(L):
    try:
        from . import _calls as native
    except ImportError:
        return _Declines()
    here = (L.cdsgd_build_id().decode(), str(torch.__version__), sysconfig.get_config_var("SOABI") or "")
    if getattr(native, "made_for", None) != here:
        return _Declines()
    native.bind(*[ctypes.cast(getattr(L, name), ctypes.c_void_p).value for name in _CALLED])
    return native


def lib():
    """The loaded C-ABI library; raises if it has not been built."""
    global _lib, _calls
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libcdsgd.so is not built (run: python -m paper_2106_10796_amd.build); "
                               "there is no fallback path")
        L = ctypes.CDLL(LIB_PATH)
        vp, sz, f, i = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float, ctypes.c_int
        L.cdsgd_packed_words.restype = sz
        L.cdsgd_packed_words.argtypes = [sz]
        L.cdsgd_status_string.restype = ctypes.c_char_p
        L.cdsgd_status_string.argtypes = [i]
        L.cdsgd_build_id.restype = ctypes.c_char_p
        L.cdsgd_build_id.argtypes = []
        L.cdsgd_quantize_pack.restype = i
        L.cdsgd_quantize_pack.argtypes = [vp, vp, vp, sz, f, vp]
        L.cdsgd_decode_sum.restype = i
        L.cdsgd_decode_sum.argtypes = [ctypes.POINTER(vp), i, vp, sz, f, vp]
        L.cdsgd_update.restype = i
        L.cdsgd_update.argtypes = [vp, vp, vp, vp, sz, f, f, i, vp]
        L.cdsgd_plan_create.restype = i
        L.cdsgd_plan_create.argtypes = [ctypes.POINTER(cdsgd_tensor), i, ctypes.POINTER(ctypes.POINTER(vp)),
                                        i, i, ctypes.POINTER(vp)]
        L.cdsgd_plan_destroy.restype = i
        L.cdsgd_plan_destroy.argtypes = [vp]
        L.cdsgd_step_fused.restype = i
        L.cdsgd_step_fused.argtypes = [vp, ctypes.c_long, i, f, f, f, vp]
        L.cdsgd_plan_create_typed.restype = i
        L.cdsgd_plan_create_typed.argtypes = [ctypes.POINTER(cdsgd_tensor), i, ctypes.POINTER(ctypes.POINTER(vp)),
                                              i, i, i, ctypes.POINTER(vp)]
        L.cdsgd_plan_set_thresholds.restype = i
        L.cdsgd_plan_set_thresholds.argtypes = [vp, ctypes.POINTER(f)]
        L.cdsgd_sparse_segments.restype = sz
        L.cdsgd_sparse_segments.argtypes = [sz]
        L.cdsgd_sparse_words.restype = sz
        L.cdsgd_sparse_words.argtypes = [sz]
        L.cdsgd_sparse_encode.restype = i
        L.cdsgd_sparse_encode.argtypes = [vp, sz, vp, vp, vp]
        L.cdsgd_decode_sum_sparse.restype = i
        L.cdsgd_decode_sum_sparse.argtypes = [ctypes.POINTER(vp), i, vp, sz, f, vp]
        L.cdsgd_plan_set_peer_format.restype = i
        L.cdsgd_plan_set_peer_format.argtypes = [vp, i]
        L.cdsgd_probe_streams.restype = i
        L.cdsgd_probe_streams.argtypes = [ctypes.POINTER(vp), i, ctypes.POINTER(vp), i, sz, vp, ctypes.c_uint, vp]
        L.cdsgd_plan_set_max_workgroups.restype = i
        L.cdsgd_plan_set_max_workgroups.argtypes = [vp, i]
        L.cdsgd_step_local.restype = i
        L.cdsgd_step_local.argtypes = [vp, f, vp]
        L.cdsgd_step_global.restype = i
        L.cdsgd_step_global.argtypes = [vp, ctypes.c_long, i, f, f, vp]
        L.cdsgd_step_fused_range.restype = i
        L.cdsgd_step_fused_range.argtypes = [vp, i, i, ctypes.c_long, i, f, f, f, vp]
        L.cdsgd_step_local_range.restype = i
        L.cdsgd_step_local_range.argtypes = [vp, i, i, f, vp]
        L.cdsgd_step_global_range.restype = i
        L.cdsgd_step_global_range.argtypes = [vp, i, i, ctypes.c_long, i, f, f, vp]
        L.cdsgd_plan_bind_full_grads.restype = i
        L.cdsgd_plan_bind_full_grads.argtypes = [vp, ctypes.POINTER(ctypes.POINTER(vp))]
        L.cdsgd_step_warmup.restype = i
        L.cdsgd_step_warmup.argtypes = [vp, ctypes.c_long, ctypes.c_long, f, f, vp]
        L.cdsgd_trainer_create.restype = i
        L.cdsgd_trainer_create.argtypes = [vp, ctypes.c_long, i, f, f, f, ctypes.POINTER(vp)]
        L.cdsgd_trainer_step.restype = i
        L.cdsgd_trainer_step.argtypes = [vp, vp, ctypes.POINTER(i)]
        L.cdsgd_trainer_iteration.restype = ctypes.c_long
        L.cdsgd_trainer_iteration.argtypes = [vp]
        L.cdsgd_trainer_destroy.restype = i
        L.cdsgd_trainer_destroy.argtypes = [vp]
        L.cdsgd_step_fused_static.restype = i
        L.cdsgd_step_fused_static.argtypes = [ctypes.POINTER(cdsgd_tensor), i, ctypes.POINTER(ctypes.POINTER(vp)),
                                              i, i, i, ctypes.c_long, i, f, f, f, vp]
        L.cdsgd_cost_iteration.restype = i
        L.cdsgd_cost_iteration.argtypes = [ctypes.POINTER(cdsgd_cost_params), ctypes.c_long,
                                           ctypes.POINTER(cdsgd_cost)]
        L.cdsgd_cost_period_mean.restype = i
        L.cdsgd_cost_period_mean.argtypes = [ctypes.POINTER(cdsgd_cost_params), ctypes.POINTER(cdsgd_cost)]
        _declare_ops(L)
        _calls = _load_calls(L)
        _lib = L                       # last: another thread that sees it finds the calls bound
    return _lib


def _declare_ops(L):
    """The entry points of include/cdsgd_ops.h."""
    vp, sz, f, i, d = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float, ctypes.c_int, ctypes.c_double
    pvp = ctypes.POINTER(vp)
    for name, restype, argtypes in (
            ("cdsgd_grad_norm_create", i, [pvp, ctypes.POINTER(sz), i, i, pvp]),
            ("cdsgd_grad_norm_compute", i, [vp, d, d, vp, vp]),
            ("cdsgd_grad_norm_destroy", i, [vp]),
            ("cdsgd_state_blocks", sz, [sz]),
            ("cdsgd_adamw_plan_create", i, [ctypes.POINTER(cdsgd_adamw_tensor), i, i, i, pvp]),
            ("cdsgd_adamw_plan_destroy", i, [vp]),
            ("cdsgd_adamw_step", i, [vp, ctypes.c_long, d, d, d, d, d, ctypes.c_uint64, vp, vp]),
            ("cdsgd_adamw_grad_norm", i, [vp, d, d, vp, vp]),
            ("cdsgd_adamw_bind_readout", i, [vp, pvp, pvp, i]),
            ("cdsgd_adamw_read_states", i, [vp, vp]),
            ("cdsgd_mxfp4_code_bytes", sz, [sz, sz]),
            ("cdsgd_mxfp4_scale_bytes", sz, [sz, sz]),
            ("cdsgd_mxfp4_quantize", i, [vp, i, sz, sz, sz, vp, vp, vp, vp, vp]),
            ("cdsgd_mxfp4_dequantize", i, [vp, vp, sz, sz, vp, i, sz, vp]),
            ("cdsgd_mxfp4_matmul_workspace", sz, [sz, sz, sz]),
            ("cdsgd_mxfp4_matmul", i, [vp, vp, vp, vp, sz, sz, sz, vp, i, sz, i, vp, sz, vp])):
        fn = getattr(L, name)
        fn.restype, fn.argtypes = restype, argtypes


def packed_words(n: int) -> int:
    return int(lib().cdsgd_packed_words(int(n)))


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream():
    """The current stream of the current device, as the integer that a stream argument takes.

    Asked for without building a torch.cuda.Stream object (0.2 us instead of 2.9, of the 7 us that a call on a
    small layer list took)."""
    if _raw_stream is not None and _current_device is not None and torch.cuda.is_initialized():
        return _raw_stream(_current_device())
    return torch.cuda.current_stream().cuda_stream


def _dev(t, dtype, n=None, name="tensor"):
    if t is None:
        return None
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise TypeError("%s must be a contiguous CUDA tensor of %s" % (name, dtype))
    if n is not None and t.numel() != n:
        raise ValueError("%s has %d elements, expected %d" % (name, t.numel(), n))
    return t.data_ptr()


def _dev_list(tensors, dtype, n, name):
    """The addresses of `tensors` as a C array (at least one entry)."""
    arr = (ctypes.c_void_p * max(len(tensors), 1))()
    for j, t in enumerate(tensors):
        # (_dev again only to say what is wrong)
        if not (isinstance(t, torch.Tensor) and t.dtype == dtype and t.is_cuda and t.numel() == n and t.is_contiguous()):
            _dev(t, dtype, n, "%s[%d]" % (name, j))
        arr[j] = t.data_ptr() if t is not None else None
    return arr


# packed streams are stored in int32 tensors (torch has no full uint32 support); the bits are what matter
PACKED_DTYPE = torch.int32


def new_packed(n: int, device="cuda") -> torch.Tensor:
    return torch.empty(packed_words(n), dtype=PACKED_DTYPE, device=device)


def _check(status, where):
    if status != OK:
        raise CdsgdError(status, where)


def cdsgd_quantize_pack(grad, residual, packed, threshold):
    st = _native().quantize_pack(grad, residual, packed, threshold, _stream)
    if st < 0:
        n = grad.numel()
        st = lib().cdsgd_quantize_pack(_dev(grad, torch.float32, None, "grad"),
                                       _dev(residual, torch.float32, n, "residual"),
                                       _dev(packed, PACKED_DTYPE, packed_words(n), "packed"),
                                       n, float(threshold), _stream())
    if st != OK:
        _check(st, "cdsgd_quantize_pack")


def cdsgd_decode_sum(packed_list, agg, threshold):
    st = _native().decode_sum(packed_list, agg, threshold, _stream)
    if st < 0:
        n = agg.numel()
        N = len(packed_list)
        arr = _dev_list(packed_list, PACKED_DTYPE, packed_words(n), "packed")
        st = lib().cdsgd_decode_sum(arr, N, _dev(agg, torch.float32, None, "agg"), n, float(threshold), _stream())
    if st != OK:
        _check(st, "cdsgd_decode_sum")


PEERS_PACKED, PEERS_SPARSE = 0, 1   # cdsgd_peer_format


def sparse_segments(n: int) -> int:
    return int(lib().cdsgd_sparse_segments(int(n)))


def sparse_words(n: int) -> int:
    return int(lib().cdsgd_sparse_words(int(n)))


def new_sparse(n: int, device="cuda") -> torch.Tensor:
    return torch.empty(sparse_words(n), dtype=PACKED_DTYPE, device=device)


def cdsgd_sparse_encode(packed, n, sparse, segment_words=None):
    st = _native().sparse_encode(packed, n, sparse, segment_words, _stream)
    if st < 0:
        st = lib().cdsgd_sparse_encode(_dev(packed, PACKED_DTYPE, packed_words(n), "packed"), int(n),
                                       _dev(sparse, PACKED_DTYPE, sparse_words(n), "sparse"),
                                       _dev(segment_words, PACKED_DTYPE, sparse_segments(n), "segment_words"), _stream())
    if st != OK:
        _check(st, "cdsgd_sparse_encode")


def cdsgd_decode_sum_sparse(sparse_list, agg, threshold):
    st = _native().decode_sum_sparse(sparse_list, agg, threshold, _stream)
    if st < 0:
        n = agg.numel()
        N = len(sparse_list)
        arr = _dev_list(sparse_list, PACKED_DTYPE, sparse_words(n), "sparse")
        st = lib().cdsgd_decode_sum_sparse(arr, N, _dev(agg, torch.float32, None, "agg"), n, float(threshold), _stream())
    if st != OK:
        _check(st, "cdsgd_decode_sum_sparse")


def cdsgd_probe_streams(reads, writes, sink=None, lds_bytes=0):
    """Bare streaming of len(reads) read and len(writes) write streams (cdsgd_probe_streams)."""
    n = (reads + writes)[0].numel()
    ra = _dev_list(reads, torch.float32, n, "reads")
    wa = _dev_list(writes, torch.float32, n, "writes")
    st = lib().cdsgd_probe_streams(ra, len(reads), wa, len(writes), n,
                                   _dev(sink, torch.float32, None, "sink"), int(lds_bytes), _stream())
    _check(st, "cdsgd_probe_streams")


def cdsgd_update(w_global, w_local, grad_local, agg, lr_local, lr_global, num_workers):
    st = _native().update(w_global, w_local, grad_local, agg, lr_local, lr_global, num_workers, _stream)
    if st < 0:
        n = w_global.numel()
        st = lib().cdsgd_update(_dev(w_global, torch.float32, None, "w_global"),
                                _dev(w_local, torch.float32, n, "w_local"),
                                _dev(grad_local, torch.float32, n, "grad_local"),
                                _dev(agg, torch.float32, n, "agg"),
                                n, float(lr_local), float(lr_global), int(num_workers), _stream())
    if st != OK:
        _check(st, "cdsgd_update")


def cdsgd_cost_iteration(tau, phi, psi, delta, k, i) -> dict:
    p = cdsgd_cost_params(float(tau), float(phi), float(psi), float(delta), int(k))
    out = cdsgd_cost()
    _check(lib().cdsgd_cost_iteration(ctypes.byref(p), int(i), ctypes.byref(out)), "cdsgd_cost_iteration")
    return out.as_dict()


def cdsgd_cost_period_mean(tau, phi, psi, delta, k) -> dict:
    p = cdsgd_cost_params(float(tau), float(phi), float(psi), float(delta), int(k))
    out = cdsgd_cost()
    _check(lib().cdsgd_cost_period_mean(ctypes.byref(p), ctypes.byref(out)), "cdsgd_cost_period_mean")
    return out.as_dict()


def _marshal_layer_list(tensors, peers, num_workers, grad_dtype, peers_sparse=False):
    """The C arrays of a layer list: (cdsgd_tensor[T], peers' row table or None, keep-alive list)."""
    peer_words = sparse_words if peers_sparse else packed_words
    T = len(tensors)
    if grad_dtype not in GRAD_DTYPES:
        raise TypeError("gradients must be float32, bfloat16 or float16")
    arr = (cdsgd_tensor * max(T, 1))()
    for i, t in enumerate(tensors):
        n = t["w_global"].numel()
        arr[i].w_global = _dev(t["w_global"], torch.float32, None, "w_global")
        arr[i].w_local = _dev(t["w_local"], torch.float32, n, "w_local")
        arr[i].residual = _dev(t["residual"], torch.float32, n, "residual")
        arr[i].grad = _dev(t["grad"], grad_dtype, n, "grad")
        arr[i].packed_self = _dev(t["packed_self"], PACKED_DTYPE, packed_words(n), "packed_self")
        af = t.get("agg_full")
        arr[i].agg_full = _dev(af, torch.float32, n, "agg_full") if af is not None else None
        arr[i].n = n
    if peers is None:
        return arr, None, []
    rows = (ctypes.POINTER(ctypes.c_void_p) * max(num_workers, 1))()
    keep = []
    for j in range(num_workers):
        if peers[j] is None:
            rows[j] = ctypes.POINTER(ctypes.c_void_p)()
            continue
        row = (ctypes.c_void_p * max(T, 1))()
        for i in range(T):
            n = tensors[i]["w_global"].numel()
            row[i] = _dev(peers[j][i], PACKED_DTYPE, peer_words(n), "peers[%d][%d]" % (j, i))
        keep.append(row)
        rows[j] = ctypes.cast(row, ctypes.POINTER(ctypes.c_void_p))
    return arr, rows, keep


def cdsgd_step_fused_static(tensors, peers, num_workers, self_rank, step, k, threshold, lr_local, lr_global,
                            grad_dtype=torch.float32):
    """One fused pass over a layer list without a plan and without any allocation in the library
    (cdsgd_step_fused_static); tensors and peers as for Plan."""
    arr, rows, _keep = _marshal_layer_list(tensors, peers, num_workers, grad_dtype)
    st = lib().cdsgd_step_fused_static(arr, len(tensors), rows, int(num_workers), int(self_rank),
                                       GRAD_DTYPES[grad_dtype], int(step), int(k), float(threshold),
                                       float(lr_local), float(lr_global), _stream())
    _check(st, "cdsgd_step_fused_static")


class StaticLayerList:
    """A layer list marshalled once for cdsgd_step_fused_static: the host arrays the call reads are built
    here, so that step() costs what the C entry point costs (the tensors are kept alive by this object)."""

    def __init__(self, tensors, peers, num_workers, grad_dtype=torch.float32):
        self._keep = (tensors, peers)
        self._n = len(tensors)
        self._num_workers = int(num_workers)
        self._grad = GRAD_DTYPES[grad_dtype]
        self._arr, self._rows, self._rows_keep = _marshal_layer_list(tensors, peers, num_workers, grad_dtype)
        self._arr_at = ctypes.addressof(self._arr)
        self._rows_at = 0 if self._rows is None else ctypes.addressof(self._rows)

    def step(self, self_rank, step, k, threshold, lr_local, lr_global):
        st = _calls.step_static(self._arr_at, self._n, self._rows_at, self._num_workers, self_rank, self._grad, step, k,
                                threshold, lr_local, lr_global, _stream)
        if st < 0:
            st = lib().cdsgd_step_fused_static(self._arr, self._n, self._rows, self._num_workers, int(self_rank),
                                               self._grad, int(step), int(k), float(threshold), float(lr_local),
                                               float(lr_global), _stream())
        if st != OK:
            _check(st, "cdsgd_step_fused_static")


class Plan:
    """A fused-step plan over a layer list (cdsgd_plan_create / cdsgd_step_fused / cdsgd_plan_destroy).

    tensors: list of dicts with keys w_global, w_local, residual, grad, packed_self and
    optionally agg_full (torch CUDA tensors).  peers: list over workers of lists over
    tensors of packed tensors (sparse buffers with peers_sparse=True); the entry for `self_rank`
    may be None.  The plan keeps
    references to every tensor so that the borrowed pointers stay valid.
    """

    def __init__(self, tensors, peers, num_workers, self_rank, grad_dtype=torch.float32, peers_sparse=False):
        T = len(tensors)
        self._grad_dtype = grad_dtype
        self._keep = (tensors, peers)
        arr, rows, self._rows = _marshal_layer_list(tensors, peers, num_workers, grad_dtype, peers_sparse)
        self._sizes = [t["w_global"].numel() for t in tensors]
        handle = ctypes.c_void_p()
        if grad_dtype == torch.float32:
            st = lib().cdsgd_plan_create(arr, T, rows, int(num_workers), int(self_rank), ctypes.byref(handle))
        else:
            st = lib().cdsgd_plan_create_typed(arr, T, rows, int(num_workers), int(self_rank),
                                               GRAD_DTYPES[grad_dtype], ctypes.byref(handle))
        _check(st, "cdsgd_plan_create")
        self._handle = handle
        self._at = handle.value        # None once the plan is destroyed
        self.num_workers = int(num_workers)
        if peers_sparse:
            self.set_peer_format(PEERS_SPARSE)

    def step(self, step, k, threshold, lr_local, lr_global):
        st = _calls.step(self._at, step, k, threshold, lr_local, lr_global, _stream)
        if st < 0:
            st = lib().cdsgd_step_fused(self._handle, int(step), int(k), float(threshold), float(lr_local),
                                        float(lr_global), _stream())
        if st != OK:
            _check(st, "cdsgd_step_fused")

    def set_thresholds(self, thresholds):
        """One threshold per tensor (list of floats), or None to go back to the call's threshold."""
        if thresholds is None:
            st = lib().cdsgd_plan_set_thresholds(self._handle, None)
        else:
            if len(thresholds) != len(self._sizes):
                raise ValueError("need one threshold per tensor")
            arr = (ctypes.c_float * len(thresholds))(*[float(x) for x in thresholds])
            st = lib().cdsgd_plan_set_thresholds(self._handle, arr)
        _check(st, "cdsgd_plan_set_thresholds")

    def set_peer_format(self, fmt):
        """PEERS_PACKED or PEERS_SPARSE: how compressed passes read the peers' streams (cdsgd_plan_set_peer_format)."""
        _check(lib().cdsgd_plan_set_peer_format(self._handle, int(fmt)), "cdsgd_plan_set_peer_format")

    def set_max_workgroups(self, max_workgroups):
        """At most this many workgroups per pass (0: one per chunk); cdsgd_plan_set_max_workgroups."""
        _check(lib().cdsgd_plan_set_max_workgroups(self._handle, int(max_workgroups)),
               "cdsgd_plan_set_max_workgroups")

    def step_local(self, lr_local):
        st = lib().cdsgd_step_local(self._handle, float(lr_local), _stream())
        _check(st, "cdsgd_step_local")

    def step_global(self, step, k, threshold, lr_global):
        st = lib().cdsgd_step_global(self._handle, int(step), int(k), float(threshold), float(lr_global), _stream())
        _check(st, "cdsgd_step_global")

    def step_range(self, first_tensor, num_tensors, step, k, threshold, lr_local, lr_global):
        """The fused pass over tensors [first_tensor, first_tensor + num_tensors) only (cdsgd_step_fused_range)."""
        st = _calls.step_range(self._at, first_tensor, num_tensors, step, k, threshold, lr_local, lr_global, _stream)
        if st < 0:
            st = lib().cdsgd_step_fused_range(self._handle, int(first_tensor), int(num_tensors), int(step), int(k),
                                              float(threshold), float(lr_local), float(lr_global), _stream())
        if st != OK:
            _check(st, "cdsgd_step_fused_range")

    def step_local_range(self, first_tensor, num_tensors, lr_local):
        st = lib().cdsgd_step_local_range(self._handle, int(first_tensor), int(num_tensors), float(lr_local), _stream())
        _check(st, "cdsgd_step_local_range")

    def step_global_range(self, first_tensor, num_tensors, step, k, threshold, lr_global):
        st = lib().cdsgd_step_global_range(self._handle, int(first_tensor), int(num_tensors), int(step), int(k),
                                           float(threshold), float(lr_global), _stream())
        _check(st, "cdsgd_step_global_range")

    def bind_full_grads(self, peer_grads):
        """peer_grads[j][i]: worker j's fp32 gradient of tensor i; entry self_rank may be None
        (cdsgd_plan_bind_full_grads).  Correction and warm-up passes then sum in the kernel."""
        T = len(self._sizes)
        rows = (ctypes.POINTER(ctypes.c_void_p) * max(self.num_workers, 1))()
        keep = []
        for j in range(self.num_workers):
            if peer_grads[j] is None:
                rows[j] = ctypes.POINTER(ctypes.c_void_p)()
                continue
            row = (ctypes.c_void_p * max(T, 1))()
            for i in range(T):
                row[i] = _dev(peer_grads[j][i], self._grad_dtype, self._sizes[i], "peer_grads[%d][%d]" % (j, i))
            keep.append(row)
            rows[j] = ctypes.cast(row, ctypes.POINTER(ctypes.c_void_p))
        st = lib().cdsgd_plan_bind_full_grads(self._handle, rows)
        _check(st, "cdsgd_plan_bind_full_grads")
        self._keep_full = peer_grads

    def step_warmup(self, i, warmup_steps, lr_local, lr_global):
        st = lib().cdsgd_step_warmup(self._handle, int(i), int(warmup_steps), float(lr_local), float(lr_global),
                                     _stream())
        _check(st, "cdsgd_step_warmup")

    def destroy(self):
        if self._handle is not None and self._handle.value:
            lib().cdsgd_plan_destroy(self._handle)
        self._handle = self._at = None
        self._keep = None
        self._keep_full = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


class Trainer:
    """Alg. 1 end to end as a counter around a plan (cdsgd_trainer_*)."""

    def __init__(self, plan: Plan, warmup_steps, k, threshold, lr_local, lr_global):
        self._plan = plan
        handle = ctypes.c_void_p()
        st = lib().cdsgd_trainer_create(plan._handle, int(warmup_steps), int(k), float(threshold),
                                        float(lr_local), float(lr_global), ctypes.byref(handle))
        _check(st, "cdsgd_trainer_create")
        self._handle = handle

    def step(self) -> int:
        """Enqueue the next iteration; returns PASS_WARMUP / PASS_COMPRESSED / PASS_CORRECTION."""
        kind = ctypes.c_int(-1)
        st = lib().cdsgd_trainer_step(self._handle, _stream(), ctypes.byref(kind))
        _check(st, "cdsgd_trainer_step")
        return kind.value

    @property
    def iteration(self) -> int:
        return int(lib().cdsgd_trainer_iteration(self._handle))

    def destroy(self):
        if self._handle is not None and self._handle.value:
            lib().cdsgd_trainer_destroy(self._handle)
        self._handle = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


# ---------------------------------------------------------------------------
# include/cdsgd_ops.h: norms of gradients, AdamW, MXFP4
# ---------------------------------------------------------------------------
STATE_BLOCK = 256   # CDSGD_STATE_BLOCK


def state_blocks(n: int) -> int:
    return int(lib().cdsgd_state_blocks(int(n)))


def _same_device(tensors):
    """A handle works on the device of its tensors, which is the current one when it is made."""
    for t in tensors:
        if t.device.index != torch.cuda.current_device():
            raise ValueError("a tensor is not on the current device")


class GradNorm:
    """The norm of a list of gradients (cdsgd_grad_norm_*): contiguous CUDA tensors of one type.  Keeps references to them."""

    def __init__(self, grads):
        self._handle = self._at = None
        dtype = grads[0].dtype if len(grads) else torch.float32
        if dtype not in GRAD_DTYPES:
            raise TypeError("gradients must be float32, bfloat16 or float16")
        arr = (ctypes.c_void_p * max(len(grads), 1))(*[_dev(g, dtype, None, "grads[%d]" % i) for i, g in enumerate(grads)])
        sizes = (ctypes.c_size_t * max(len(grads), 1))(*[g.numel() for g in grads])
        _same_device(grads)
        handle = ctypes.c_void_p()
        st = lib().cdsgd_grad_norm_create(arr, sizes, len(grads), GRAD_DTYPES[dtype], ctypes.byref(handle))
        _check(st, "cdsgd_grad_norm_create")
        self._handle, self._at, self._keep = handle, handle.value, list(grads)

    def compute(self, out, grad_scale=1.0, max_norm=float("inf")):
        """out (float32, 2 elements) receives the norm and the factor that brings it down to max_norm."""
        st = _calls.grad_norm_compute(self._at, out, grad_scale, max_norm, _stream)
        if st < 0:
            st = lib().cdsgd_grad_norm_compute(self._handle, float(grad_scale), float(max_norm), _dev(out, torch.float32, 2, "out"),
                                               _stream())
        if st != OK:
            _check(st, "cdsgd_grad_norm_compute")

    def destroy(self):
        if self._handle is not None and self._handle.value:
            lib().cdsgd_grad_norm_destroy(self._handle)
        self._handle = self._at = self._keep = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


class AdamWPlan:
    """AdamW over a list of tensors, one launch a step (cdsgd_adamw_*).

    tensors: list of dicts with keys weight (float32), grad (grad_dtype), m and v (float32, or uint8 with state_bits=8),
    m_scale and v_scale (uint8, state_blocks(n) of them, with state_bits=8), and optionally weight16 (grad_dtype, receives
    a copy of the new weights; for all tensors or none) and weight_decay (0 if absent).  Contiguous CUDA tensors of any shape, of which the
    plan keeps references.  States that are all zero bytes are the start of training.
    """

    def __init__(self, tensors, grad_dtype=torch.float32, state_bits=32):
        self._handle = self._at = None
        if grad_dtype not in GRAD_DTYPES:
            raise TypeError("gradients must be float32, bfloat16 or float16")
        state = torch.uint8 if state_bits == 8 else torch.float32
        T = len(tensors)
        arr = (cdsgd_adamw_tensor * max(T, 1))()
        for i, t in enumerate(tensors):
            n = t["weight"].numel()
            arr[i].weight = _dev(t["weight"], torch.float32, None, "weight")
            arr[i].weight16 = _dev(t.get("weight16"), grad_dtype, n, "weight16")
            arr[i].grad = _dev(t["grad"], grad_dtype, n, "grad")
            for name in ("m", "v"):
                setattr(arr[i], name, _dev(t[name], state, n, name))
                setattr(arr[i], name + "_scale", _dev(t.get(name + "_scale"), torch.uint8, state_blocks(n), name + "_scale"))
            arr[i].n = n
            arr[i].weight_decay = float(t.get("weight_decay", 0.0))
        _same_device([x for t in tensors for x in t.values() if isinstance(x, torch.Tensor)])
        handle = ctypes.c_void_p()
        st = lib().cdsgd_adamw_plan_create(arr, T, GRAD_DTYPES[grad_dtype], int(state_bits), ctypes.byref(handle))
        _check(st, "cdsgd_adamw_plan_create")
        self._handle, self._at = handle, handle.value
        self._sizes = [t["weight"].numel() for t in tensors]
        self._keep, self._keep_out = [dict(t) for t in tensors], None

    def step(self, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0, seed=0, clip=None):
        """Step number `step` (from 1 on).  clip: the out of grad_norm, or None.  seed: another one for every step with 8-bit states."""
        st = _calls.adamw_step(self._at, step, lr, beta1, beta2, eps, grad_scale, seed, clip, _stream)
        if st < 0:
            st = lib().cdsgd_adamw_step(self._handle, int(step), float(lr), float(beta1), float(beta2), float(eps), float(grad_scale),
                                        int(seed) & 0xFFFFFFFFFFFFFFFF, _dev(clip, torch.float32, 2, "clip"), _stream())
        if st != OK:
            _check(st, "cdsgd_adamw_step")

    def grad_norm(self, out, grad_scale=1.0, max_norm=float("inf")):
        """The norm of the plan's gradients and the factor for clipping, into out (float32, 2 elements)."""
        st = _calls.adamw_grad_norm(self._at, out, grad_scale, max_norm, _stream)
        if st < 0:
            st = lib().cdsgd_adamw_grad_norm(self._handle, float(grad_scale), float(max_norm), _dev(out, torch.float32, 2, "out"),
                                             _stream())
        if st != OK:
            _check(st, "cdsgd_adamw_grad_norm")

    def bind_readout(self, m_out, v_out):
        """Where read_states puts the values of 8-bit states: lists of float32 or of bfloat16 tensors, one for each tensor."""
        if len(m_out) != len(self._sizes) or len(v_out) != len(self._sizes):
            raise ValueError("need one output for each tensor")
        dtype = m_out[0].dtype
        if dtype not in (torch.float32, torch.bfloat16):
            raise TypeError("states are read out as float32 or bfloat16")
        rows = []
        for name, outs in (("m_out", m_out), ("v_out", v_out)):
            rows.append((ctypes.c_void_p * len(outs))(*[_dev(t, dtype, n, "%s[%d]" % (name, i))
                                                       for i, (t, n) in enumerate(zip(outs, self._sizes))]))
        _same_device([*m_out, *v_out])
        _check(lib().cdsgd_adamw_bind_readout(self._handle, rows[0], rows[1], GRAD_DTYPES[dtype]), "cdsgd_adamw_bind_readout")
        self._keep_out = (list(m_out), list(v_out))

    def read_states(self):
        """The values that 8-bit states stand for, into the tensors of bind_readout."""
        st = _calls.adamw_read_states(self._at, _stream)
        if st < 0:
            st = lib().cdsgd_adamw_read_states(self._handle, _stream())
        if st != OK:
            _check(st, "cdsgd_adamw_read_states")

    def destroy(self):
        if self._handle is not None and self._handle.value:
            lib().cdsgd_adamw_plan_destroy(self._handle)
        self._handle = self._at = self._keep = self._keep_out = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


class _Mxfp4(NamedTuple):
    codes: torch.Tensor
    scales: torch.Tensor
    rows: int
    cols: int


def _as_bytes(t, name):
    """t, or a copy of it as uint8 where it holds bytes in integers of another type."""
    if not (isinstance(t, torch.Tensor) and t.dtype in (torch.int16, torch.int32, torch.int64)):
        return t
    if bool(((t < 0) | (t > 255)).any()):
        raise ValueError("%s holds integers that are not bytes" % name)
    return t.to(torch.uint8).contiguous()


class Mxfp4(_Mxfp4):
    """A matrix of `rows` by `cols` in microscaled 4-bit floating point (the layout is in include/cdsgd_ops.h):
    codes uint8 [rows, 64 g] and scales uint8 [g, rows, 4] with g = ceil(cols / 128), contiguous CUDA tensors, which are
    kept as they are.  Bytes in integers of another type, as a quantiser written in torch leaves them, are looked over (on the host)
    and copied: such a matrix is an operand, but nothing can be quantised into it."""
    __slots__ = ()

    def __new__(cls, codes, scales, rows, cols):
        held = [_as_bytes(codes, "codes"), _as_bytes(scales, "scales")]
        if cls is Mxfp4 and not (held[0] is codes and held[1] is scales):
            cls = _Mxfp4Copy
        return _Mxfp4.__new__(cls, *held, int(rows), int(cols))


class _Mxfp4Copy(Mxfp4):
    """A matrix whose buffers are copies of the caller's tensors."""
    __slots__ = ()


def new_mxfp4(rows: int, cols: int, device="cuda") -> Mxfp4:
    """Room for a matrix; every byte of it is written by cdsgd_mxfp4_quantize."""
    g = -(-cols // 128)
    return Mxfp4(torch.empty(rows, 64 * g, dtype=torch.uint8, device=device),
                 torch.empty(g, rows, 4, dtype=torch.uint8, device=device), rows, cols)


def new_mxfp4_workspace(shapes, device="cuda"):
    """Workspace for products of any of the shapes (M, N, K): a uint8 tensor, or None where none of them needs one."""
    need = max((int(lib().cdsgd_mxfp4_matmul_workspace(*map(int, s))) for s in shapes), default=0)
    return torch.empty(need, dtype=torch.uint8, device=device) if need else None


def _mx(q, name, rows=None, cols=None, optional=False):
    """The addresses of a matrix: (codes, scales); (None, None) for None where it is optional."""
    if q is None and optional:
        return None, None
    if not isinstance(q, Mxfp4):
        raise TypeError("%s must be an Mxfp4" % name)
    if rows is not None and (q.rows, q.cols) != (rows, cols):
        raise ValueError("%s is a matrix of %d by %d, expected %d by %d" % (name, q.rows, q.cols, rows, cols))
    g = -(-q.cols // 128)
    return (_dev(q.codes, torch.uint8, q.rows * 64 * g, name + ".codes"), _dev(q.scales, torch.uint8, q.rows * 4 * g, name + ".scales"))


def _rows(t, name, rows=None, cols=None):
    """(address, type, rows, cols, elements between two rows) of a matrix whose rows are contiguous."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dim() == 2 and t.dtype in GRAD_DTYPES):
        raise TypeError("%s must be a CUDA matrix of float32, bfloat16 or float16" % name)
    if rows is not None and tuple(t.shape) != (rows, cols):
        raise ValueError("%s is a matrix of %d by %d, expected %d by %d" % (name, *t.shape, rows, cols))
    r, c = t.shape
    if (c > 1 and t.stride(1) != 1) or (r > 1 and t.stride(0) < c):
        raise TypeError("the rows of %s must be contiguous and not overlap" % name)
    return t.data_ptr(), GRAD_DTYPES[t.dtype], r, c, t.stride(0) if r > 1 else c


def cdsgd_mxfp4_quantize(x, row=None, col=None):
    """x [rows, cols] into `row` (blocks along its rows) and into `col`, its transpose [cols, rows] (blocks down its columns); either
    may be None."""
    st = _native().mxfp4_quantize(x, row, col, _stream)
    if st < 0:
        for q, name in ((row, "row"), (col, "col")):
            if isinstance(q, _Mxfp4Copy):
                raise TypeError("%s holds copies of tensors that are not uint8: the caller's would not receive anything" % name)
        p, dtype, r, c, ld = _rows(x, "x")
        codes, scales = _mx(row, "row", r, c, optional=True)
        codes_t, scales_t = _mx(col, "col", c, r, optional=True)
        st = lib().cdsgd_mxfp4_quantize(p, dtype, r, c, ld, codes, scales, codes_t, scales_t, _stream())
    if st != OK:
        _check(st, "cdsgd_mxfp4_quantize")


def cdsgd_mxfp4_dequantize(q, out):
    """The values that q stands for, into out [rows, cols]."""
    st = _native().mxfp4_dequantize(q, out, _stream)
    if st < 0:
        codes, scales = _mx(q, "q")
        p, dtype, r, c, ld = _rows(out, "out", q.rows, q.cols)
        st = lib().cdsgd_mxfp4_dequantize(codes, scales, r, c, p, dtype, ld, _stream())
    if st != OK:
        _check(st, "cdsgd_mxfp4_dequantize")


def cdsgd_mxfp4_matmul(a, b, out, workspace=None, accumulate=False):
    """out [M, N] = a [M, K] times the transpose of b [N, K]; accumulate adds it to what out holds.  workspace: from
    new_mxfp4_workspace, not shared by products that may overlap."""
    st = _native().mxfp4_matmul(a, b, out, workspace, accumulate, _stream)
    if st < 0:
        ac, as_ = _mx(a, "a")
        bc, bs = _mx(b, "b", getattr(b, "rows", 0), a.cols)
        p, dtype, M, N, ld = _rows(out, "out", a.rows, b.rows)
        st = lib().cdsgd_mxfp4_matmul(ac, as_, bc, bs, M, N, a.cols, p, dtype, ld, int(bool(accumulate)),
                                      _dev(workspace, torch.uint8, None, "workspace"), workspace.numel() if workspace is not None else 0,
                                      _stream())
    if st != OK:
        _check(st, "cdsgd_mxfp4_matmul")
