"""Thin ctypes binding of libsparseconv.so (argument marshalling only).

Every step of the path -- the offset-stretching pass, the LDS staging, the gather-MAC kernels, the
autotuner -- runs inside the HIP library.  PyTorch appears only as the owner of device memory and
streams: tensors are passed down as raw device pointers.  There is no CPU fallback: if the shared
library is missing, importing the symbols fails loudly.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsparseconv.so")

SC_OK = 0
STATUS_NAMES = {0: "SC_OK", 1: "SC_ERR_NULL", 2: "SC_ERR_SHAPE", 3: "SC_ERR_CSR",
                4: "SC_ERR_UNSUPPORTED", 5: "SC_ERR_RANGE", 6: "SC_ERR_OOM", 7: "SC_ERR_WORKSPACE",
                8: "SC_ERR_HIP"}
SC_F32, SC_F16, SC_I8, SC_CB4_I8, SC_CB4_F16 = 0, 1, 2, 3, 4
DTYPES = {"f32": SC_F32, "f16": SC_F16, "i8": SC_I8, "cb4": SC_CB4_I8, "cb4h": SC_CB4_F16}
SC_VARIANT_AUTO, SC_VARIANT_GATHER, SC_VARIANT_SLAB, SC_VARIANT_DENSE = 0, 1, 2, 3
SC_STATIC_WORKSPACE_BYTES = 32 << 20
SC_PATH_SPARSE, SC_PATH_DENSE, SC_PATH_LIBRARY = 0, 1, 2
SC_ELEM_F32, SC_ELEM_F16, SC_ELEM_BF16, SC_ELEM_E4M3 = 0, 1, 2, 3
ELEMS = {"f32": SC_ELEM_F32, "f16": SC_ELEM_F16, "bf16": SC_ELEM_BF16, "e4m3": SC_ELEM_E4M3}
SC_ACT_NONE, SC_ACT_RELU, SC_ACT_SILU = 0, 1, 2
ACTS = {"none": SC_ACT_NONE, "relu": SC_ACT_RELU, "silu": SC_ACT_SILU}
SC_SCORE_SOFTMAX, SC_SCORE_SIGMOID = 0, 1
SCORES = {"softmax": SC_SCORE_SOFTMAX, "sigmoid": SC_SCORE_SIGMOID}
FORMS = ["nothing", "norm lanes", "norm sample", "norm two", "rows", "64", "64 split", "128", "128 deep", "256"]   # SC_FORM_*
EXPERT_FORMS = ["sort one", "sort chunks", "adapters few", "adapters many"]      # ... of sc_expert_form_t, from len(FORMS) on
BLOCK = 128                        # elements of a row that share a scale

# every symbol include/sparse_conv.h declares
EXPORTS = [
    "sparse_conv_plan_create_csr", "sparse_conv_plan_create_ell", "sparse_conv_plan_destroy",
    "sparse_conv_plan_info", "sparse_conv_plan_debug_offsets", "sparse_conv_plan_set_tuning", "sparse_conv_plan_set_epilogue",
    "sparse_conv_plan_get_tuning", "sparse_conv_workspace_size", "sparse_conv_workspace_size_max",
    "sparse_conv_forward", "sparse_conv_forward_static", "sparse_conv_plan_autotune", "sparse_conv_autotune_workspace_size", "sparse_conv_plan_dispatch", "sparse_conv_plan_set_path",
    "sparse_conv_plan_num_candidates",
    "sparse_conv_plan_candidate", "sparse_conv_quantize_pow2", "sparse_conv_status_string",
    "sparse_conv_group_norm_workspace_size", "sparse_conv_group_norm", "sparse_conv_quantize_blocks",
    "sparse_conv_matmul_blocks_workspace_size", "sparse_conv_matmul_blocks",
    "sparse_conv_matmul_grouped_workspace_size", "sparse_conv_matmul_grouped",
    "sparse_conv_group_norm_launch", "sparse_conv_matmul_blocks_launch", "sparse_conv_matmul_grouped_launch",
    "sparse_conv_route_experts", "sparse_conv_route_experts_backward",
    "sparse_conv_sort_by_expert_workspace_size", "sparse_conv_sort_by_expert_launch", "sparse_conv_sort_by_expert",
    "sparse_conv_gather_rows", "sparse_conv_combine_rows", "sparse_conv_combine_rows_backward",
    "sparse_conv_adapters_workspace_size", "sparse_conv_adapters_launch", "sparse_conv_adapters",
]


class sc_layer_t(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in
                ("C", "D", "H", "W", "R", "S", "stride_h", "stride_w", "pad_h", "pad_w")]


class sc_tuning_t(ctypes.Structure):
    _fields_ = [("variant", ctypes.c_int32), ("wg_threads", ctypes.c_int32),
                ("sub_batch", ctypes.c_int32), ("tile_p", ctypes.c_int32),
                ("tile_q", ctypes.c_int32), ("wg_per_cu", ctypes.c_int32),
                ("wsrc", ctypes.c_int32), ("split_n", ctypes.c_int32),
                ("pipeline", ctypes.c_int32), ("producers", ctypes.c_int32),
                ("chunk_c", ctypes.c_int32), ("tile_d", ctypes.c_int32), ("ragged", ctypes.c_int32), ("pack", ctypes.c_int32),
                ("waves_m", ctypes.c_int32), ("buffers", ctypes.c_int32),
                ("stage_rows", ctypes.c_int32)]

    def as_dict(self):
        return {k: int(getattr(self, k)) for k, _ in self._fields_}


class sc_dispatch_t(ctypes.Structure):
    _fields_ = [("choice", ctypes.c_int32), ("sparse_ms", ctypes.c_float), ("dense_ms", ctypes.c_float),
                ("library_ms", ctypes.c_float), ("sparse_tuning", sc_tuning_t), ("dense_tuning", sc_tuning_t)]

    def as_dict(self):
        return {"choice": ("sparse", "dense", "library")[self.choice], "sparse_ms": self.sparse_ms,
                "dense_ms": self.dense_ms, "library_ms": self.library_ms,
                "sparse_tuning": self.sparse_tuning.as_dict(), "dense_tuning": self.dense_tuning.as_dict()}


class sc_plan_info_t(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("P", ctypes.c_int32), ("Q", ctypes.c_int32),
                ("X_size", ctypes.c_int64), ("true_nnz", ctypes.c_int64),
                ("macs_per_sample", ctypes.c_int64), ("useful_macs_per_sample", ctypes.c_int64),
                ("act_bytes_per_sample", ctypes.c_int64), ("weight_bytes", ctypes.c_int64),
                ("lds_bytes", ctypes.c_int32), ("grid_size", ctypes.c_int32),
                ("tuning", sc_tuning_t), ("out_P", ctypes.c_int32), ("out_Q", ctypes.c_int32),
                ("out_elem_bytes", ctypes.c_int32)]


class sc_epilogue_t(ctypes.Structure):
    _fields_ = [("relu", ctypes.c_int32), ("pool", ctypes.c_int32), ("requant", ctypes.c_int32)]


def _fields(i32_before, f32, i32_after, i64):
    return ([(k, ctypes.c_int32) for k in i32_before] + [(k, ctypes.c_float) for k in f32] +
            [(k, ctypes.c_int32) for k in i32_after] + [(k, ctypes.c_int64) for k in i64])


class sc_group_norm_t(ctypes.Structure):
    _fields_ = _fields(("N", "S", "C", "G", "x_type", "y_type", "act"), ("eps",), (),
                       ("x_sample", "x_row", "y_sample", "y_row", "scale_row"))


class sc_quantize_blocks_t(ctypes.Structure):
    _fields_ = _fields(("M", "K", "rows", "x_type"), (), (), ("x_row", "q_row", "scale_row"))


class sc_matmul_blocks_t(ctypes.Structure):
    _fields_ = _fields(("M", "N", "K", "y_type", "act"), (), (), ("a_row", "b_row", "y_row", "a_scale_row", "b_scale_row"))


class sc_matmul_grouped_t(ctypes.Structure):
    _fields_ = _fields(("M", "N", "K", "E", "a_type", "y_type", "act", "a_rows"), (), (),
                       ("a_row", "b_row", "b_expert", "y_row", "a_scale_row", "b_scale_row", "b_scale_expert"))


class sc_launch_t(ctypes.Structure):
    _fields_ = _fields(("form", "lanes", "held", "one_die", "past_cache"), (), (), ())


class sc_route_experts_t(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_int32) for k in ("T", "E", "top", "x_type", "score", "normalize")] + [("factor", ctypes.c_float)] +
                [(k, ctypes.c_int64) for k in ("x_row", "dx_row")])


class sc_sort_by_expert_t(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("T", "top", "E")]


class sc_gather_rows_t(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("M", "C", "rows", "x_type")] + [(k, ctypes.c_int64) for k in ("x_row", "y_row")]


class sc_combine_rows_t(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_int32) for k in ("T", "top", "C", "rows", "x_type", "y_type")] +
                [(k, ctypes.c_int64) for k in ("x_row", "y_row", "residual_row", "dx_row")])


class sc_adapters_t(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_int32) for k in ("M", "N", "K", "R", "E", "rows", "x_type", "y_type")] +
                [(k, ctypes.c_int64) for k in ("x_row", "a_row", "a_adapter", "b_row", "b_adapter", "base_row", "y_row")])


class SparseConvError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().sparse_conv_status_string(status).decode()
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)} ({msg})")


_lib = None


def lib() -> ctypes.CDLL:
    """Load libsparseconv.so; raises if it has not been built (no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: run `python -c 'import __graft_entry__ as g; g.build()'`")
    # PyTorch bundles its own HIP runtime.  Import it before the library so that both bind to the one
    # runtime already in the process; loaded the other way round the process ends up with two runtimes
    # and the second to initialise reports that it sees no GPU.
    import torch  # noqa: F401
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    P = ctypes.POINTER
    L.sparse_conv_plan_create_csr.argtypes = [P(sc_layer_t), ctypes.c_int, vp, vp, vp, vp, vp, vp, P(vp)]
    L.sparse_conv_plan_create_ell.argtypes = [P(sc_layer_t), ctypes.c_int, i32, vp, vp, vp, vp, vp, P(vp)]
    L.sparse_conv_plan_destroy.argtypes = [vp]
    L.sparse_conv_plan_destroy.restype = None
    L.sparse_conv_plan_info.argtypes = [vp, P(sc_plan_info_t)]
    L.sparse_conv_plan_debug_offsets.argtypes = [vp, vp]
    L.sparse_conv_plan_set_tuning.argtypes = [vp, P(sc_tuning_t), vp]
    L.sparse_conv_plan_get_tuning.argtypes = [vp, P(sc_tuning_t)]
    L.sparse_conv_plan_set_epilogue.argtypes = [vp, P(sc_epilogue_t), vp, vp]
    L.sparse_conv_workspace_size.argtypes = [vp, i32, P(sz)]
    L.sparse_conv_workspace_size_max.argtypes = [vp, i32, P(sz)]
    L.sparse_conv_forward.argtypes = [vp, vp, vp, i32, vp, sz, vp]
    L.sparse_conv_forward_static.argtypes = [vp, vp, vp, i32, vp]
    L.sparse_conv_plan_autotune.argtypes = [vp, vp, vp, i32, vp, sz, vp]
    L.sparse_conv_autotune_workspace_size.argtypes = [vp, i32, P(sz)]
    L.sparse_conv_plan_dispatch.argtypes = [vp, vp, vp, i32, vp, sz, vp, P(sc_dispatch_t)]
    L.sparse_conv_plan_set_path.argtypes = [vp, i32, vp]
    L.sparse_conv_plan_num_candidates.argtypes = [vp, P(i32)]
    L.sparse_conv_plan_candidate.argtypes = [vp, i32, P(sc_tuning_t)]
    L.sparse_conv_quantize_pow2.argtypes = [vp, sz, i32, ctypes.c_float, vp, P(i32)]
    L.sparse_conv_status_string.argtypes = [ctypes.c_int]
    L.sparse_conv_status_string.restype = ctypes.c_char_p
    L.sparse_conv_group_norm_workspace_size.argtypes = [P(sc_group_norm_t), P(sz)]
    L.sparse_conv_group_norm.argtypes = [vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.sparse_conv_quantize_blocks.argtypes = [vp, vp, vp, vp, vp]
    L.sparse_conv_matmul_blocks_workspace_size.argtypes = [P(sc_matmul_blocks_t), P(sz)]
    L.sparse_conv_matmul_blocks.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.sparse_conv_matmul_grouped_workspace_size.argtypes = [P(sc_matmul_grouped_t), P(sz)]
    L.sparse_conv_group_norm_launch.argtypes = [P(sc_group_norm_t), P(sc_launch_t)]
    L.sparse_conv_matmul_blocks_launch.argtypes = [P(sc_matmul_blocks_t), P(sc_launch_t)]
    L.sparse_conv_matmul_grouped_launch.argtypes = [P(sc_matmul_grouped_t), P(sc_launch_t)]
    L.sparse_conv_matmul_grouped.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.sparse_conv_route_experts.argtypes = [vp, vp, vp, vp, vp, vp]
    L.sparse_conv_route_experts_backward.argtypes = [vp, vp, vp, vp, vp, vp]
    L.sparse_conv_sort_by_expert_workspace_size.argtypes = [P(sc_sort_by_expert_t), P(sz)]
    L.sparse_conv_sort_by_expert.argtypes = [vp, vp, vp, vp, vp, vp, sz, vp]
    L.sparse_conv_gather_rows.argtypes = [vp, vp, vp, vp, vp]
    L.sparse_conv_combine_rows.argtypes = [vp, vp, vp, vp, vp, vp, vp]
    L.sparse_conv_combine_rows_backward.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp]
    L.sparse_conv_adapters_workspace_size.argtypes = [P(sc_adapters_t), P(sz)]
    L.sparse_conv_sort_by_expert_launch.argtypes = [P(sc_sort_by_expert_t), P(sc_launch_t)]
    L.sparse_conv_adapters_launch.argtypes = [P(sc_adapters_t), P(sc_launch_t)]
    L.sparse_conv_adapters.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    for name in EXPORTS:
        if name not in ("sparse_conv_plan_destroy", "sparse_conv_status_string"):
            getattr(L, name).restype = ctypes.c_int
    _lib = L
    return L


def _check(status: int, where: str):
    if status != SC_OK:
        raise SparseConvError(status, where)


def _host(a: Optional[np.ndarray], dtype) -> Optional[np.ndarray]:
    return None if a is None else np.ascontiguousarray(a, dtype=dtype)


def _hp(a: Optional[np.ndarray]):
    return None if a is None else ctypes.c_void_p(a.ctypes.data)


_VALUE_NP = {SC_F32: np.float32, SC_F16: np.float16, SC_I8: np.int8, SC_CB4_I8: np.uint8, SC_CB4_F16: np.uint8}
_CODEBOOK_NP = {SC_CB4_I8: np.int8, SC_CB4_F16: np.float16}


def quantize_pow2(x: np.ndarray, total_bits: int = 8, saturate_at: float = 1.0):
    """sparse_conv_quantize_pow2: (codes int8 with the shape of x, frac_bits)."""
    xa = np.ascontiguousarray(x, dtype=np.float32)
    codes = np.empty(xa.shape, dtype=np.int8)
    fb = ctypes.c_int32(0)
    _check(lib().sparse_conv_quantize_pow2(_hp(xa) if xa.size else None, xa.size, total_bits, saturate_at,
                                           _hp(codes) if xa.size else None, ctypes.byref(fb)),
           "sparse_conv_quantize_pow2")
    return codes, int(fb.value)


def make_layer(C, D, H, W, R, S, stride=(1, 1), pad=(0, 0)) -> sc_layer_t:
    return sc_layer_t(C, D, H, W, R, S, stride[0], stride[1], pad[0], pad[1])


_ADDRESS = (int, type(None))


class Plan:
    """Owner of one sparse_conv_plan_t.  Same calls as the C ABI, same names."""

    def __init__(self, handle: int, layer: sc_layer_t, dtype: int):
        self._h = ctypes.c_void_p(handle)
        self.layer = layer
        self.dtype = dtype

    # -- construction -------------------------------------------------------------------------
    @staticmethod
    def create_csr(layer: sc_layer_t, dtype: int, rowptr, colidx, values, scales=None,
                   codebook=None, stream: int = 0) -> "Plan":
        rp = _host(rowptr, np.int32)
        ci = _host(colidx, np.int32)
        va = _host(values, _VALUE_NP.get(dtype, np.uint8))
        sc_ = _host(scales, np.float32)
        cb = _host(codebook, _CODEBOOK_NP.get(dtype, np.int8))
        out = ctypes.c_void_p()
        st = lib().sparse_conv_plan_create_csr(ctypes.byref(layer), dtype, _hp(rp), _hp(ci), _hp(va),
                                               _hp(sc_), _hp(cb), ctypes.c_void_p(stream),
                                               ctypes.byref(out))
        _check(st, "sparse_conv_plan_create_csr")
        return Plan(out.value, layer, dtype)

    @staticmethod
    def create_ell(layer: sc_layer_t, dtype: int, n: int, colidx, values, scales=None,
                   codebook=None, stream: int = 0) -> "Plan":
        ci = _host(colidx, np.int32)
        va = _host(values, _VALUE_NP.get(dtype, np.uint8))
        sc_ = _host(scales, np.float32)
        cb = _host(codebook, _CODEBOOK_NP.get(dtype, np.int8))
        out = ctypes.c_void_p()
        st = lib().sparse_conv_plan_create_ell(ctypes.byref(layer), dtype, n, _hp(ci), _hp(va),
                                               _hp(sc_), _hp(cb), ctypes.c_void_p(stream),
                                               ctypes.byref(out))
        _check(st, "sparse_conv_plan_create_ell")
        return Plan(out.value, layer, dtype)

    def destroy(self):
        if self._h:
            lib().sparse_conv_plan_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    # -- queries ------------------------------------------------------------------------------
    def info(self) -> sc_plan_info_t:
        inf = sc_plan_info_t()
        _check(lib().sparse_conv_plan_info(self._h, ctypes.byref(inf)), "sparse_conv_plan_info")
        return inf

    def debug_offsets(self) -> np.ndarray:
        inf = self.info()
        out = np.zeros((self.layer.D, inf.n), dtype=np.int32)
        _check(lib().sparse_conv_plan_debug_offsets(self._h, _hp(out)), "sparse_conv_plan_debug_offsets")
        return out

    def get_tuning(self) -> sc_tuning_t:
        t = sc_tuning_t()
        _check(lib().sparse_conv_plan_get_tuning(self._h, ctypes.byref(t)), "sparse_conv_plan_get_tuning")
        return t

    def set_tuning(self, tuning: Optional[sc_tuning_t] = None, stream: int = 0, **fields):
        t = tuning if tuning is not None else sc_tuning_t()
        for k, v in fields.items():
            setattr(t, k, v)
        _check(lib().sparse_conv_plan_set_tuning(self._h, ctypes.byref(t), ctypes.c_void_p(stream)),
               "sparse_conv_plan_set_tuning")

    def set_epilogue(self, relu: bool = False, pool: int = 0, requant_scale=None, stream: int = 0):
        ep = sc_epilogue_t(int(bool(relu)), int(pool), int(requant_scale is not None))
        rq = _host(requant_scale, np.float32)
        _check(lib().sparse_conv_plan_set_epilogue(self._h, ctypes.byref(ep), _hp(rq), ctypes.c_void_p(stream)),
               "sparse_conv_plan_set_epilogue")

    def workspace_size(self, N: int) -> int:
        b = ctypes.c_size_t()
        _check(lib().sparse_conv_workspace_size(self._h, N, ctypes.byref(b)), "sparse_conv_workspace_size")
        return int(b.value)

    def workspace_size_max(self, N: int) -> int:
        b = ctypes.c_size_t()
        _check(lib().sparse_conv_workspace_size_max(self._h, N, ctypes.byref(b)),
               "sparse_conv_workspace_size_max")
        return int(b.value)

    def dispatch(self, x_ptr: int, y_ptr: int, N: int, ws_ptr: int = 0, ws_bytes: int = 0, stream: int = 0):
        rec = sc_dispatch_t()
        _check(lib().sparse_conv_plan_dispatch(self._h, ctypes.c_void_p(x_ptr), ctypes.c_void_p(y_ptr), N,
                                               ctypes.c_void_p(ws_ptr), ws_bytes, ctypes.c_void_p(stream),
                                               ctypes.byref(rec)),
               "sparse_conv_plan_dispatch")
        return rec

    def set_path(self, path: int, stream: int = 0):
        _check(lib().sparse_conv_plan_set_path(self._h, path, ctypes.c_void_p(stream)), "sparse_conv_plan_set_path")

    def autotune_workspace_size(self, N: int) -> int:
        b = ctypes.c_size_t()
        _check(lib().sparse_conv_autotune_workspace_size(self._h, N, ctypes.byref(b)),
               "sparse_conv_autotune_workspace_size")
        return int(b.value)

    def num_candidates(self) -> int:
        c = ctypes.c_int32()
        _check(lib().sparse_conv_plan_num_candidates(self._h, ctypes.byref(c)),
               "sparse_conv_plan_num_candidates")
        return int(c.value)

    def candidate(self, i: int) -> sc_tuning_t:
        t = sc_tuning_t()
        _check(lib().sparse_conv_plan_candidate(self._h, i, ctypes.byref(t)), "sparse_conv_plan_candidate")
        return t

    # -- execution (raw device pointers) --------------------------------------------------------
    def forward(self, x_ptr: int, y_ptr: int, N: int, ws_ptr: int = 0, ws_bytes: int = 0,
                stream: int = 0):
        # (plain integers: the declared argument types convert them, which is quicker than four pointer
        # objects -- but they would also take the address of a bytes or str object)
        if not (isinstance(x_ptr, _ADDRESS) and isinstance(y_ptr, _ADDRESS) and isinstance(ws_ptr, _ADDRESS) and
                isinstance(stream, _ADDRESS)):
            raise TypeError("device pointers and the stream are integers (or None)")
        st = lib().sparse_conv_forward(self._h, x_ptr, y_ptr, N, ws_ptr, ws_bytes, stream)
        if st:
            raise SparseConvError(st, "sparse_conv_forward")

    def forward_static(self, x_ptr: int, y_ptr: int, N: int, stream: int = 0):
        _check(lib().sparse_conv_forward_static(self._h, ctypes.c_void_p(x_ptr), ctypes.c_void_p(y_ptr), N,
                                                ctypes.c_void_p(stream)),
               "sparse_conv_forward_static")

    def autotune(self, x_ptr: int, y_ptr: int, N: int, ws_ptr: int = 0, ws_bytes: int = 0,
                 stream: int = 0):
        _check(lib().sparse_conv_plan_autotune(self._h, ctypes.c_void_p(x_ptr), ctypes.c_void_p(y_ptr),
                                               N, ctypes.c_void_p(ws_ptr), ws_bytes,
                                               ctypes.c_void_p(stream)),
               "sparse_conv_plan_autotune")


# -------------------------------------------------------------------------------------------------
# operators of channels-last blocks
# -------------------------------------------------------------------------------------------------
def _elem(t) -> int:
    """SC_ELEM_* of a name ("f16"), a torch dtype or the number itself."""
    if isinstance(t, int):
        return t
    if isinstance(t, str):
        return ELEMS[t]
    import torch
    return {torch.float32: SC_ELEM_F32, torch.float16: SC_ELEM_F16, torch.bfloat16: SC_ELEM_BF16,
            torch.float8_e4m3fn: SC_ELEM_E4M3}[t]


def _code(act) -> int:
    return ACTS[act] if isinstance(act, str) else int(act)


def _up(n: int, to: int) -> int:
    return -(-n // to) * to


class _Operator:
    """A description in the form that the library reads: same calls as the C ABI."""
    _name = ""

    def __init__(self, desc):
        self.desc = desc
        self._at = ctypes.addressof(desc)      # (the structure lives as long as this object)
        self._fn = getattr(lib(), self._name)

    def workspace_size(self) -> int:
        b = ctypes.c_size_t()
        name = self._name + "_workspace_size"
        _check(getattr(lib(), name)(ctypes.byref(self.desc), ctypes.byref(b)), name)
        return int(b.value)

    def launch(self) -> dict:
        """What a call runs: "form" (one of FORMS, EXPERT_FORMS) and, of a group norm in one launch, "lanes", "held", "one_die", "past_cache"."""
        l = sc_launch_t()
        name = self._name + "_launch"
        _check(getattr(lib(), name)(ctypes.byref(self.desc), ctypes.byref(l)), name)
        return {k: (FORMS + EXPERT_FORMS)[l.form] if k == "form" else int(getattr(l, k)) for k, _ in l._fields_}

    def _refused(self, status):
        raise SparseConvError(status, self._name)


# (In every forward: addresses, sizes and the stream are integers, 0 for none; the alternation of all of them is a TypeError for
# anything else, bytes and str among it, which ctypes would pass as their address.)


class GroupNorm(_Operator):
    """sparse_conv_group_norm: y = act(group norm of x), channels last.  Strides are (sample, position) in
    elements; left out, x and y are contiguous (codes: rows of the next multiple of 16)."""
    _name = "sparse_conv_group_norm"

    def __init__(self, N, S, C, G, eps=1e-5, act="none", x_type="f16", y_type=None, x_strides=None, y_strides=None, scale_row=None):
        xt = _elem(x_type)
        yt = xt if y_type is None else _elem(y_type)
        xs = (S * C, C) if x_strides is None else x_strides
        row = _up(C, 16) if yt == SC_ELEM_E4M3 else C
        ys = (S * row, row) if y_strides is None else y_strides
        super().__init__(sc_group_norm_t(N, S, C, G, xt, yt, _code(act), eps, xs[0], xs[1], ys[0], ys[1],
                                         -(-C // BLOCK) if scale_row is None else scale_row))

    def forward(self, x_ptr: int, gamma_ptr: int, beta_ptr: int, y_ptr: int, scale_ptr: int = 0, ws_ptr: int = 0,
                ws_bytes: int = 0, stream: int = 0):
        x_ptr | gamma_ptr | beta_ptr | y_ptr | scale_ptr | ws_ptr | ws_bytes | stream
        status = self._fn(self._at, x_ptr, gamma_ptr, beta_ptr, y_ptr, scale_ptr, ws_ptr, ws_bytes, stream)
        if status:
            self._refused(status)


class BlockQuantizer(_Operator):
    """sparse_conv_quantize_blocks: codes and scales of blocks of rows x 128."""
    _name = "sparse_conv_quantize_blocks"

    def __init__(self, M, K, rows=1, x_type="f16", x_row=None, q_row=None, scale_row=None):
        super().__init__(sc_quantize_blocks_t(M, K, rows, _elem(x_type), K if x_row is None else x_row,
                                              _up(K, 16) if q_row is None else q_row,
                                              -(-K // BLOCK) if scale_row is None else scale_row))

    def workspace_size(self) -> int:
        return 0

    def forward(self, x_ptr: int, q_ptr: int, scale_ptr: int, stream: int = 0):
        x_ptr | q_ptr | scale_ptr | stream
        status = self._fn(self._at, x_ptr, q_ptr, scale_ptr, stream)
        if status:
            self._refused(status)


class BlockMatmul(_Operator):
    """sparse_conv_matmul_blocks: y = act(a b^T + bias) of operands in e4m3 blocks."""
    _name = "sparse_conv_matmul_blocks"

    def __init__(self, M, N, K, y_type="bf16", act="none", a_row=None, b_row=None, y_row=None, a_scale_row=None, b_scale_row=None):
        row, kb = _up(K, 16), -(-K // BLOCK)
        super().__init__(sc_matmul_blocks_t(M, N, K, _elem(y_type), _code(act), row if a_row is None else a_row,
                                            row if b_row is None else b_row, N if y_row is None else y_row,
                                            kb if a_scale_row is None else a_scale_row, kb if b_scale_row is None else b_scale_row))

    def forward(self, a_ptr: int, a_scale_ptr: int, b_ptr: int, b_scale_ptr: int, bias_ptr: int, y_ptr: int, ws_ptr: int = 0,
                ws_bytes: int = 0, stream: int = 0):
        a_ptr | a_scale_ptr | b_ptr | b_scale_ptr | bias_ptr | y_ptr | ws_ptr | ws_bytes | stream
        status = self._fn(self._at, a_ptr, a_scale_ptr, b_ptr, b_scale_ptr, bias_ptr, y_ptr, ws_ptr, ws_bytes, stream)
        if status:
            self._refused(status)


class GroupedMatmul(_Operator):
    """sparse_conv_matmul_grouped: the rows of group e of y = act(a[index] b[e]^T + bias[e])."""
    _name = "sparse_conv_matmul_grouped"

    def __init__(self, M, N, K, E, a_type="bf16", y_type=None, act="none", a_rows=None, a_row=None, b_row=None, b_expert=None,
                 y_row=None, a_scale_row=None, b_scale_row=None, b_scale_expert=None):
        at = _elem(a_type)
        yt = _elem(y_type) if y_type is not None else SC_ELEM_BF16 if at == SC_ELEM_E4M3 else at
        row, kb = _up(K, 16 if at == SC_ELEM_E4M3 else 8), -(-K // BLOCK)
        b_row = row if b_row is None else b_row
        b_scale_row = kb if b_scale_row is None else b_scale_row
        super().__init__(sc_matmul_grouped_t(M, N, K, E, at, yt, _code(act), M if a_rows is None else a_rows,
                                             row if a_row is None else a_row, b_row, N * b_row if b_expert is None else b_expert,
                                             N if y_row is None else y_row, kb if a_scale_row is None else a_scale_row, b_scale_row,
                                             -(-N // BLOCK) * b_scale_row if b_scale_expert is None else b_scale_expert))

    def forward(self, a_ptr: int, a_scale_ptr: int, index_ptr: int, offsets_ptr: int, b_ptr: int, b_scale_ptr: int, bias_ptr: int,
                y_ptr: int, ws_ptr: int = 0, ws_bytes: int = 0, stream: int = 0):
        a_ptr | a_scale_ptr | index_ptr | offsets_ptr | b_ptr | b_scale_ptr | bias_ptr | y_ptr | ws_ptr | ws_bytes | stream
        status = self._fn(self._at, a_ptr, a_scale_ptr, index_ptr, offsets_ptr, b_ptr, b_scale_ptr, bias_ptr, y_ptr, ws_ptr, ws_bytes, stream)
        if status:
            self._refused(status)


class _WithGradient(_Operator):
    """An operator with a gradient: `backward` is <name>_backward of the C ABI, on the same description."""

    def __init__(self, desc):
        super().__init__(desc)
        self._back = getattr(lib(), self._name + "_backward")

    def workspace_size(self) -> int:
        return 0

    def _backward_refused(self, status):
        raise SparseConvError(status, self._name + "_backward")


class ExpertRouter(_WithGradient):
    """sparse_conv_route_experts: the `top` experts of each token and their weights from logits [T, E]."""
    _name = "sparse_conv_route_experts"

    def __init__(self, T, E, top, score="softmax", normalize=False, factor=1.0, x_type="f32", x_row=None, dx_row=None):
        super().__init__(sc_route_experts_t(T, E, top, _elem(x_type), SCORES[score] if isinstance(score, str) else int(score), int(normalize), factor,
                                            E if x_row is None else x_row, E if dx_row is None else dx_row))

    def forward(self, x_ptr: int, bias_ptr: int, ids_ptr: int, weights_ptr: int, stream: int = 0):
        x_ptr | bias_ptr | ids_ptr | weights_ptr | stream
        status = self._fn(self._at, x_ptr, bias_ptr, ids_ptr, weights_ptr, stream)
        if status:
            self._refused(status)

    def backward(self, x_ptr: int, ids_ptr: int, dweights_ptr: int, dx_ptr: int, stream: int = 0):
        x_ptr | ids_ptr | dweights_ptr | dx_ptr | stream
        status = self._back(self._at, x_ptr, ids_ptr, dweights_ptr, dx_ptr, stream)
        if status:
            self._backward_refused(status)


class ExpertSort(_Operator):
    """sparse_conv_sort_by_expert: offsets [E + 1], index [T top] and position [T, top] of ids [T, top]."""
    _name = "sparse_conv_sort_by_expert"

    def __init__(self, T, top, E):
        super().__init__(sc_sort_by_expert_t(T, top, E))

    def forward(self, ids_ptr: int, offsets_ptr: int, index_ptr: int, position_ptr: int, ws_ptr: int = 0, ws_bytes: int = 0, stream: int = 0):
        ids_ptr | offsets_ptr | index_ptr | position_ptr | ws_ptr | ws_bytes | stream
        status = self._fn(self._at, ids_ptr, offsets_ptr, index_ptr, position_ptr, ws_ptr, ws_bytes, stream)
        if status:
            self._refused(status)


class RowGather(_Operator):
    """sparse_conv_gather_rows: y[i] = x[index[i]], M rows of C elements from x with `rows` rows."""
    _name = "sparse_conv_gather_rows"

    def __init__(self, M, C, rows, x_type="f16", x_row=None, y_row=None):
        super().__init__(sc_gather_rows_t(M, C, rows, _elem(x_type), C if x_row is None else x_row, C if y_row is None else y_row))

    def workspace_size(self) -> int:
        return 0

    def forward(self, x_ptr: int, index_ptr: int, y_ptr: int, stream: int = 0):
        x_ptr | index_ptr | y_ptr | stream
        status = self._fn(self._at, x_ptr, index_ptr, y_ptr, stream)
        if status:
            self._refused(status)


class RowCombine(_WithGradient):
    """sparse_conv_combine_rows: y[t] = residual[t] + sum_j weights[t, j] x[position[t, j]]; y_row is dy's distance in a backward call."""
    _name = "sparse_conv_combine_rows"

    def __init__(self, T, top, C, rows, x_type="f16", y_type=None, x_row=None, y_row=None, residual_row=None, dx_row=None):
        xt = _elem(x_type)
        super().__init__(sc_combine_rows_t(T, top, C, rows, xt, xt if y_type is None else _elem(y_type), *(C if r is None else r for r in (x_row, y_row, residual_row, dx_row))))

    def forward(self, x_ptr: int, position_ptr: int, weights_ptr: int, residual_ptr: int, y_ptr: int, stream: int = 0):
        x_ptr | position_ptr | weights_ptr | residual_ptr | y_ptr | stream
        status = self._fn(self._at, x_ptr, position_ptr, weights_ptr, residual_ptr, y_ptr, stream)
        if status:
            self._refused(status)

    def backward(self, dy_ptr: int, x_ptr: int, position_ptr: int, weights_ptr: int, dx_ptr: int, dweights_ptr: int, stream: int = 0):
        dy_ptr | x_ptr | position_ptr | weights_ptr | dx_ptr | dweights_ptr | stream
        status = self._back(self._at, dy_ptr, x_ptr, position_ptr, weights_ptr, dx_ptr, dweights_ptr, stream)
        if status:
            self._backward_refused(status)


class Adapters(_Operator):
    """sparse_conv_adapters: y[t] = base[t] + scale[e] (x[t] a[e]^T) b[e]^T for the rows t of group e."""
    _name = "sparse_conv_adapters"

    def __init__(self, M, N, K, R, E, rows=None, x_type="bf16", y_type=None, x_row=None, a_row=None, a_adapter=None, b_row=None, b_adapter=None,
                 base_row=None, y_row=None):
        xt = _elem(x_type)
        a_row, b_row = _up(K, 8) if a_row is None else a_row, _up(R, 8) if b_row is None else b_row
        super().__init__(sc_adapters_t(M, N, K, R, E, M if rows is None else rows, xt, xt if y_type is None else _elem(y_type), _up(K, 8) if x_row is None else x_row,
                                       a_row, R * a_row if a_adapter is None else a_adapter, b_row, N * b_row if b_adapter is None else b_adapter,
                                       N if base_row is None else base_row, N if y_row is None else y_row))

    def forward(self, x_ptr: int, index_ptr: int, offsets_ptr: int, a_ptr: int, b_ptr: int, scale_ptr: int, base_ptr: int, y_ptr: int,
                ws_ptr: int = 0, ws_bytes: int = 0, stream: int = 0):
        x_ptr | index_ptr | offsets_ptr | a_ptr | b_ptr | scale_ptr | base_ptr | y_ptr | ws_ptr | ws_bytes | stream
        status = self._fn(self._at, x_ptr, index_ptr, offsets_ptr, a_ptr, b_ptr, scale_ptr, base_ptr, y_ptr, ws_ptr, ws_bytes, stream)
        if status:
            self._refused(status)


# -------------------------------------------------------------------------------------------------
# torch conveniences used by the tests and the benchmark (device memory and streams only)
# -------------------------------------------------------------------------------------------------
def torch_out_dtype(dtype: int):
    import torch
    return {SC_F32: torch.float32, SC_F16: torch.float16, SC_I8: torch.int32, SC_CB4_I8: torch.int32,
            SC_CB4_F16: torch.float16}[dtype]


def forward_torch(plan: Plan, x, y=None, workspace=None):
    """Run sparse_conv_forward on torch CUDA tensors, on their device and torch's current stream there."""
    import torch
    assert x.is_cuda and x.is_contiguous()
    N = x.shape[0]
    inf = plan.info()
    if y is None:
        y = torch.empty((N, plan.layer.D, inf.P, inf.Q), dtype=torch_out_dtype(plan.dtype), device=x.device)
    need = plan.workspace_size(N)
    if need and (workspace is None or workspace.numel() * workspace.element_size() < need):
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
    with torch.cuda.device(x.device):
        plan.forward(x.data_ptr(), y.data_ptr(), N,
                     workspace.data_ptr() if workspace is not None else 0,
                     workspace.numel() * workspace.element_size() if workspace is not None else 0,
                     torch.cuda.current_stream(x.device).cuda_stream)
    return y


# ... and of the operators of channels-last blocks: tensors in, tensors out, on their device and torch's current stream there.  Rows may lie further apart than
# their length; the last dimension is contiguous.  They have no gradient, and refuse tensors that want one.

def _call(op, like, *args):
    """op.forward on the device where `like` lies, on torch's current stream there, whatever device is the current one."""
    import torch
    with torch.cuda.device(like.device):
        op.forward(*args, torch.cuda.current_stream(like.device).cuda_stream)


def _call_backward(op, like, *args):
    import torch
    with torch.cuda.device(like.device):
        op.backward(*args, torch.cuda.current_stream(like.device).cuda_stream)


def _workspace(op, like):
    import torch
    n = op.workspace_size()
    return (torch.empty(n, dtype=torch.uint8, device=like.device), n) if n else (None, 0)


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


def _rows(t, what: str):
    if not t.is_cuda or t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError(f"{what}: a GPU tensor with a contiguous last dimension")
    return t


def _forward_only(*tensors, gradient: str = ""):
    """`gradient`: the call that takes the gradient of this one, which autograd does not make."""
    import torch
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors):
        what = f"autograd does not see this operator, whose gradient is {gradient}" if gradient else "the operators have no gradient"
        raise ValueError(f"{what}: call {'both' if gradient else 'them'} under torch.no_grad(), or on detached tensors")


def _params(t, n: int, like, what: str):
    import torch
    if t is not None and not (t.device == like.device and t.dtype == torch.float32 and t.is_contiguous() and t.numel() == n):
        raise ValueError(f"{what}: {n} contiguous 32-bit floats on the GPU, beside the operands")
    return t


def _scales(t, a, rows: int, what: str):
    """Scales of the codes `a` in blocks of rows x 128."""
    import torch
    shape = tuple(a.shape[:-2]) + (-(-a.shape[-2] // rows), -(-a.shape[-1] // BLOCK))
    if t is None or t.dtype != torch.float32 or t.device != a.device or tuple(t.shape) != shape or (t.stride(-1) != 1 and shape[-1] > 1):
        raise ValueError(f"{what}: {list(shape)} 32-bit floats beside the codes, with a contiguous last dimension")
    return t


def _integers(t, like, what: str):
    import torch
    if t.dtype != torch.int32 or t.device != like.device or t.dim() != 1 or not t.is_contiguous():
        raise ValueError(f"{what}: contiguous 32-bit integers beside the operands")
    return t


def _table(t, shape, dtype, like, what: str):
    if t.device != like.device or t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{what}: contiguous {list(shape)} of {dtype} beside the operands")
    return t


def stream_of(t) -> int:
    """torch's current stream on the device of t, as the integer that forward and backward take."""
    import torch
    return torch._C._cuda_getCurrentRawStream(t.device.index)


def empty_codes(*shape, device="cuda"):
    """A tensor for codes, its rows on 16 bytes."""
    import torch
    return torch.empty(*shape[:-1], _up(shape[-1], 16), dtype=torch.float8_e4m3fn, device=device)[..., :shape[-1]]


def group_norm_torch(x, groups: int, gamma=None, beta=None, eps: float = 1e-5, act: str = "none", codes: bool = False):
    """act(group norm) of x [N, S, C], channels last: a tensor like x, or with codes = True (e4m3 codes [N S, C], scales)."""
    import torch
    _rows(x, "x")
    _forward_only(x, gamma, beta)
    N, S, C = x.shape
    y = empty_codes(N * S, C, device=x.device) if codes else torch.empty((N, S, C), dtype=x.dtype, device=x.device)
    scale = torch.empty(N * S, -(-C // BLOCK), dtype=torch.float32, device=x.device) if codes else None
    op = GroupNorm(N, S, C, groups, eps=eps, act=act, x_type=x.dtype, y_type=y.dtype, x_strides=x.stride()[:2])
    ws, n = _workspace(op, x)
    _call(op, x, x.data_ptr(), _ptr(_params(gamma, C, x, "gamma")), _ptr(_params(beta, C, x, "beta")), y.data_ptr(), _ptr(scale), _ptr(ws), n)
    return (y, scale) if codes else y


def quantize_blocks_torch(x, rows: int = 1):
    """(e4m3 codes, scales) of a matrix [M, K] in blocks of rows x 128; a stack [E, M, K] matrix by matrix."""
    import torch
    _rows(x, "x")
    _forward_only(x)
    lead, (M, K) = x.shape[:-2], x.shape[-2:]
    q = empty_codes(*lead, M, K, device=x.device)
    scale = torch.empty(*lead, -(-M // rows), -(-K // BLOCK), dtype=torch.float32, device=x.device)
    op = BlockQuantizer(M, K, rows=rows, x_type=x.dtype, x_row=x.stride(-2), q_row=q.stride(-2))
    for i in np.ndindex(*lead):
        _call(op, x, x[i].data_ptr(), q[i].data_ptr(), scale[i].data_ptr())
    return q, scale


def matmul_blocks_torch(a, a_scale, b, b_scale, bias=None, act: str = "none", dtype=None):
    """act(a b^T + bias) of codes a [M, K] with scales of 1 x 128 and b [N, K] with scales of 128 x 128 blocks."""
    import torch
    if _rows(a, "a").dim() != 2 or _rows(b, "b").dim() != 2:
        raise ValueError(f"a and b: matrices, not {list(a.shape)} and {list(b.shape)} (a stack of weights goes to matmul_grouped_torch)")
    _forward_only(a, a_scale, b, b_scale, bias)
    (M, K), N = a.shape, b.shape[0]
    if b.shape[1] != K:
        raise ValueError(f"b has {b.shape[1]} columns, a has {K}")
    if a.dtype != torch.float8_e4m3fn or b.dtype != a.dtype or b.device != a.device:
        raise ValueError("a and b: codes on one GPU")
    _scales(a_scale, a, 1, "a_scale"), _scales(b_scale, b, BLOCK, "b_scale")
    y = torch.empty(M, N, dtype=dtype or torch.bfloat16, device=a.device)
    op = BlockMatmul(M, N, K, y_type=y.dtype, act=act, a_row=a.stride(0), b_row=b.stride(0), a_scale_row=a_scale.stride(0), b_scale_row=b_scale.stride(0))
    ws, n = _workspace(op, a)
    _call(op, a, a.data_ptr(), a_scale.data_ptr(), b.data_ptr(), b_scale.data_ptr(), _ptr(_params(bias, N, a, "bias")), y.data_ptr(), _ptr(ws), n)
    return y


def matmul_grouped_torch(a, b, offsets, a_scale=None, b_scale=None, index=None, bias=None, act: str = "none", dtype=None):
    """Rows offsets[e] .. offsets[e+1] - 1 of the result: act(a[index] b[e]^T + bias[e]); a [rows, K], b [E, N, K], f16, bf16 or
    codes with their scales; offsets and index 32-bit integers on the GPU.  Rows outside all groups are left as they were allocated."""
    import torch
    _rows(a, "a"), _rows(b, "b")
    _forward_only(a, a_scale, b, b_scale, bias)
    E, N, K = b.shape
    if a.dim() != 2 or a.shape[1] != K or a.dtype != b.dtype or a.device != b.device or offsets.numel() != E + 1:
        raise ValueError("a [rows, K] and b [E, N, K] of one type on one GPU, offsets [E + 1]")
    _integers(offsets, a, "offsets")
    if index is not None:
        _integers(index, a, "index")
    M = a.shape[0] if index is None else index.numel()
    codes = a.dtype == torch.float8_e4m3fn
    if codes:
        _scales(a_scale, a, 1, "a_scale"), _scales(b_scale, b, BLOCK, "b_scale")
    y = torch.empty(M, N, dtype=dtype or (torch.bfloat16 if codes else a.dtype), device=a.device)
    op = GroupedMatmul(M, N, K, E, a_type=a.dtype, y_type=y.dtype, act=act, a_rows=a.shape[0], a_row=a.stride(0), b_row=b.stride(1), b_expert=b.stride(0),
                       a_scale_row=a_scale.stride(0) if codes else 0, b_scale_row=b_scale.stride(1) if codes else 0, b_scale_expert=b_scale.stride(0) if codes else 0)
    ws, n = _workspace(op, a)
    _call(op, a, a.data_ptr(), _ptr(a_scale if codes else None), _ptr(index), offsets.data_ptr(), b.data_ptr(), _ptr(b_scale if codes else None),
          _ptr(_params(bias, E * N, a, "bias")), y.data_ptr(), _ptr(ws), n)
    return y


# ... and around a layer of experts.  Calls with a gradient have it as a call of its own (route_experts_backward_torch, ...): autograd does not see them.

def route_experts_torch(logits, top: int, score: str = "softmax", normalize: bool = False, factor: float = 1.0, bias=None):
    """(ids [T, top] 32-bit integers, weights [T, top] 32-bit floats) of logits [T, E]: the experts with the largest logit (with a
    bias [E]: score + bias), -1 where none is left, and factor * score of each, normalize: divided by the token's sum."""
    import torch
    if _rows(logits, "logits").dim() != 2:
        raise ValueError(f"logits: a matrix, not {list(logits.shape)}")
    _forward_only(logits, bias, gradient="route_experts_backward_torch")
    T, E = logits.shape
    ids = torch.empty(T, top, dtype=torch.int32, device=logits.device)
    weights = torch.empty(T, top, dtype=torch.float32, device=logits.device)
    op = ExpertRouter(T, E, top, score=score, normalize=normalize, factor=factor, x_type=logits.dtype, x_row=logits.stride(0))
    _call(op, logits, logits.data_ptr(), _ptr(_params(bias, E, logits, "bias")), ids.data_ptr(), weights.data_ptr())
    return ids, weights


def route_experts_backward_torch(logits, ids, dweights, score: str = "softmax", normalize: bool = False, factor: float = 1.0):
    """The gradient of the logits from that of the weights; logits, ids and the rest as in route_experts_torch."""
    import torch
    if _rows(logits, "logits").dim() != 2:
        raise ValueError(f"logits: a matrix, not {list(logits.shape)}")
    _forward_only(logits, dweights)
    T, E = logits.shape
    top = ids.shape[-1]
    _table(ids, (T, top), torch.int32, logits, "ids"), _table(dweights, (T, top), torch.float32, logits, "dweights")
    dx = torch.empty(T, E, dtype=logits.dtype, device=logits.device)
    op = ExpertRouter(T, E, top, score=score, normalize=normalize, factor=factor, x_type=logits.dtype, x_row=logits.stride(0))
    _call_backward(op, logits, logits.data_ptr(), ids.data_ptr(), dweights.data_ptr(), dx.data_ptr())
    return dx


def sort_by_expert_torch(ids, experts: int):
    """(offsets [E + 1], index [T top], position [T, top]), 32-bit integers, of ids [T, top] or [T]: the rows of expert e are offsets[e] ..
    offsets[e+1] - 1, index their tokens (-1 behind the last), position the row of each slot (-1: an id outside 0 .. E - 1)."""
    import torch
    if not ids.is_cuda or ids.dtype != torch.int32 or ids.dim() not in (1, 2) or not ids.is_contiguous():
        raise ValueError("ids: contiguous 32-bit integers [T, top] or [T] on the GPU")
    T, top = ids.shape if ids.dim() == 2 else (ids.shape[0], 1)
    made = lambda *shape: torch.empty(*shape, dtype=torch.int32, device=ids.device)  # noqa: E731
    op = ExpertSort(T, top, experts)
    offsets, index, position = made(experts + 1), made(T * top), made(*ids.shape)
    ws, n = _workspace(op, ids)
    _call(op, ids, ids.data_ptr(), offsets.data_ptr(), index.data_ptr(), position.data_ptr(), _ptr(ws), n)
    return offsets, index, position


def gather_rows_torch(x, index):
    """x[index], rows of zeros where the index lies outside x: x [rows, C] of any operator type (codes too), index 32-bit integers.  Its gradient is
    combine_rows_torch of the rows' gradients, without weights."""
    import torch
    if _rows(x, "x").dim() != 2:
        raise ValueError(f"x: a matrix, not {list(x.shape)}")
    _forward_only(x, gradient="combine_rows_torch")
    _integers(index, x, "index")
    M, (rows, C) = index.numel(), x.shape
    y = empty_codes(M, C, device=x.device) if x.dtype == torch.float8_e4m3fn else torch.empty(M, C, dtype=x.dtype, device=x.device)
    op = RowGather(M, C, rows, x_type=x.dtype, x_row=x.stride(0), y_row=y.stride(0))
    _call(op, x, x.data_ptr(), index.data_ptr(), y.data_ptr())
    return y


def combine_rows_torch(x, position, weights=None, residual=None, dtype=None):
    """residual[t] + the sum over j of weights[t, j] x[position[t, j]]: x [rows, C], position [T, top] 32-bit integers (outside x: nothing is added),
    weights [T, top] 32-bit floats, residual [T, C] of the result's type, which is that of x or torch.float32."""
    import torch
    if _rows(x, "x").dim() != 2 or position.dim() != 2:
        raise ValueError(f"x [rows, C] and position [T, top], not {list(x.shape)} and {list(position.shape)}")
    _forward_only(x, weights, residual, gradient="combine_rows_backward_torch")
    (rows, C), (T, top) = x.shape, position.shape
    _table(position, (T, top), torch.int32, x, "position")
    if weights is not None:
        _table(weights, (T, top), torch.float32, x, "weights")
    y = torch.empty(T, C, dtype=dtype or x.dtype, device=x.device)
    if residual is not None and (_rows(residual, "residual").shape != y.shape or residual.dtype != y.dtype or residual.device != y.device):
        raise ValueError(f"residual: [{T}, {C}] of {y.dtype} beside x")
    op = RowCombine(T, top, C, rows, x_type=x.dtype, y_type=y.dtype, x_row=x.stride(0), residual_row=None if residual is None else residual.stride(0))
    _call(op, x, x.data_ptr(), position.data_ptr(), _ptr(weights), _ptr(residual), y.data_ptr())
    return y


def combine_rows_backward_torch(dy, x, position, weights=None):
    """(dx, dweights) from dy [T, C], of x's type or torch.float32; x, position and weights as in combine_rows_torch.  Rows of dx that no slot has are
    zeros; no two slots may have the same row."""
    import torch
    if _rows(x, "x").dim() != 2 or position.dim() != 2 or _rows(dy, "dy").dim() != 2:
        raise ValueError(f"dy [T, C], x [rows, C] and position [T, top], not {list(dy.shape)}, {list(x.shape)} and {list(position.shape)}")
    _forward_only(dy, x, weights)
    (rows, C), (T, top) = x.shape, position.shape
    _table(position, (T, top), torch.int32, x, "position")
    if weights is not None:
        _table(weights, (T, top), torch.float32, x, "weights")
    if tuple(dy.shape) != (T, C) or dy.device != x.device:
        raise ValueError(f"dy: [{T}, {C}] beside x")
    dx = torch.zeros(rows, C, dtype=x.dtype, device=x.device)
    dweights = torch.empty(T, top, dtype=torch.float32, device=x.device)
    op = RowCombine(T, top, C, rows, x_type=x.dtype, y_type=dy.dtype, x_row=x.stride(0), y_row=dy.stride(0))
    _call_backward(op, x, dy.data_ptr(), x.data_ptr(), position.data_ptr(), _ptr(weights), dx.data_ptr(), dweights.data_ptr())
    return dx, dweights


def adapters_torch(y, x, a, b, offsets, index=None, scale=None):
    """y[t] += scale[e] (x[t] a[e]^T) b[e]^T in place for the rows t of group e, index[offsets[e]] .. index[offsets[e+1] - 1], and y: y [rows, N] is the
    projection's result, x [rows, K], a [E, R, K] and b [E, N, R] of one 16-bit type, y of that or 32-bit; their rows on 16 bytes; scale [E] 32-bit
    floats.  offsets and index come from sort_by_expert_torch of each row's adapter; rows without one keep what they hold."""
    import torch
    for t, what in ((y, "y"), (x, "x"), (a, "a"), (b, "b")):
        _rows(t, what)
    _forward_only(y, x, a, b, scale)
    if y.dim() != 2 or x.dim() != 2 or a.dim() != 3 or b.dim() != 3:
        raise ValueError("y [rows, N], x [rows, K], a [E, R, K] and b [E, N, R]")
    (rows, N), K, (E, R, _) = y.shape, x.shape[1], a.shape
    if x.shape[0] != rows or a.shape[2] != K or tuple(b.shape) != (E, N, R) or a.dtype != x.dtype or b.dtype != x.dtype or offsets.numel() != E + 1:
        raise ValueError(f"y [rows, N], x [rows, K], a [E, R, K], b [E, N, R] and offsets [E + 1], not {[list(t.shape) for t in (y, x, a, b, offsets)]}")
    if any(t.device != y.device for t in (x, a, b)):
        raise ValueError("y, x, a and b: on one GPU")
    _integers(offsets, y, "offsets")
    if index is not None:
        _integers(index, y, "index")
    M = rows if index is None else index.numel()
    op = Adapters(M, N, K, R, E, rows=rows, x_type=x.dtype, y_type=y.dtype, x_row=x.stride(0), a_row=a.stride(1), a_adapter=a.stride(0), b_row=b.stride(1),
                  b_adapter=b.stride(0), base_row=y.stride(0), y_row=y.stride(0))
    ws, n = _workspace(op, y)
    _call(op, y, x.data_ptr(), _ptr(index), offsets.data_ptr(), a.data_ptr(), b.data_ptr(), _ptr(_params(scale, E, y, "scale")), y.data_ptr(), y.data_ptr(), _ptr(ws), n)
    return y
