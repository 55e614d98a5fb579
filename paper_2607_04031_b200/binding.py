"""Thin Python binding of the tilelens C ABI (``include/tilelens.h``): argument marshalling only.

Every step of the path runs inside ``libtilelens.so``.  torch is used for device
memory and streams, nothing else.  There is no fallback: if the library has not
been built, or a call returns a non-zero status, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtilelens.so")

TL_OK = 0
TO_TILE_MAJOR, TO_ROW_MAJOR = 0, 1
LAYOUT_ROW_MAJOR, LAYOUT_COL_MAJOR, LAYOUT_TILE_MAJOR, LAYOUT_TILE_MAJOR_K = 0, 1, 2, 3

# Every symbol include/tilelens.h declares: (name, restype, argtypes)
_i64, _int, _vp, _sz = ctypes.c_int64, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t
_u64p = ctypes.POINTER(ctypes.c_uint64)
_SIGNATURES = {
    "tl_status_string": (ctypes.c_char_p, [_int]),
    "tl_last_cuda_error": (_int, []),
    "tl_set_stream": (_int, [_vp]),
    "tl_device_status": (_int, [ctypes.POINTER(ctypes.c_uint32)]),
    "tl_set_option": (_int, [_int, _i64]),
    "tl_get_option": (_i64, [_int]),
    "tl_gemm_plan": (_int, [_i64, _i64, _i64, _i64, _int, _int, _int, _int, _int, _int, _int, _vp]),
    "tl_gemm_last_plan": (_int, [_vp]),
    "tl_relayout": (_int, [_vp, _vp, _i64, _i64, _int, _i64, _int, _int, _int]),
    "tl_relayout_on": (_int, [_vp, _vp, _i64, _i64, _int, _i64, _int, _int, _int, _vp]),
    "tl_relayout_batch": (_int, [_int, _vp, _vp, _vp, _vp, _int, _i64, _int, _int, _int, _vp]),
    "tl_gemm": (_int, [_vp, _vp, _vp, _i64, _i64, _i64, _i64, _int, _int, _int, _int, _int, _vp]),
    "tl_gemm_grouped": (_int, [_vp, _vp, _vp, _vp, _int, _i64, _i64, _i64, _i64, _int, _int, _int, _int, _int, _vp]),
    "tl_gemm_bf16": (_int, [_vp, _vp, _vp, _i64, _i64, _i64, _i64, _int, _int, _int, _int, _int, _vp]),
    "tl_gemm_grouped_bf16": (_int, [_vp, _vp, _vp, _vp, _int, _i64, _i64, _i64, _i64, _int, _int, _int, _int, _int, _vp]),
    "tl_gemm_grouped_swiglu": (_int, [_vp, _vp, _vp, _vp, _int, _i64, _i64, _i64, _i64, _int, _int, _int, _int, _int,
                                      _vp]),
    "tl_moe_ffn": (_int, [_vp, _vp, _vp, _vp, _vp, _vp, _int, _i64, _i64, _i64, _i64, _int, _int, _vp]),
    "tl_gemm_kmajor": (_int, [_vp, _vp, _vp, _i64, _i64, _i64, _i64, _int, _int, _int, _int, _int, _vp]),
    "tl_gemm_grouped_kmajor": (_int, [_vp, _vp, _vp, _vp, _int, _i64, _i64, _i64, _i64, _int, _int, _int, _int, _int,
                                      _vp]),
    "tl_gemm_fp8_kmajor": (_int, [_vp, _vp, _vp, _i64, _i64, _i64, _i64, _int, _int, _int, _int, _int, _vp]),
    "tl_gemm_grouped_fp8_kmajor": (_int, [_vp, _vp, _vp, _vp, _int, _i64, _i64, _i64, _i64, _int, _int, _int, _int,
                                          _int, _vp]),
    "tl_read_amp_async": (_int, [_i64, _i64, _i64, _int, _int, _int, _int, _i64, _int, _int, _int, _vp, _vp]),
    "tl_read_amp_batch": (_int, [_vp, _int, _vp, _vp]),
    "tl_read_amp_shared": (_int, [_i64, _i64, _i64, _int, _int, _int, _i64, _int, _i64, _int, _int, _int, _vp, _vp, _vp]),
    "tl_prefetch_degree": (_i64, [ctypes.c_double, ctypes.c_double, _i64, _i64, _i64, _i64, _i64, _i64, ctypes.c_double]),
    "tl_tile_arrival_latency": (_int, [_vp, _i64, _i64, ctypes.c_double, ctypes.POINTER(ctypes.c_double),
                                       ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]),
    "tl_hw_box_offsets": (_int, [_vp, _vp, _i64, _vp, _vp]),
    "tl_hw_box_load": (_int, [_vp, _vp, ctypes.c_uint64, _vp, _i64, _vp, _vp]),
    "tl_gemm_workspace_bytes": (_sz, [_i64, _i64, _i64, _int, _int, _int]),
    "tl_set_workspace": (_int, [_vp, _sz]),
    "tl_gemm_host": (_int, [_vp, _vp, _vp, _i64, _i64, _i64, _i64, _int, _int, _int, _int, _int, _vp, _sz, _vp]),
    "tl_gemm_host_scratch_bytes": (_sz, [_i64, _i64, _i64]),
    "tl_gemm_noalloc": (_int, [_vp, _vp, _vp, _i64, _i64, _i64, _i64, _int, _int, _int, _int, _int, _vp, _vp]),
    "tl_read_amp": (_int, [_i64, _i64, _i64, _int, _int, _int, _int, _i64, _int, _int, _int, _u64p, _u64p, _u64p]),
    "tl_read_amp_grouped": (_int, [_vp, _int, _i64, _i64, _int, _int, _int, _int, _i64, _int, _int, _int,
                                   _u64p, _u64p, _u64p]),
    "tl_kv_append": (_int, [_vp, _vp, _vp, _vp, _int, _i64, _vp]),
    "tl_kv_read": (_int, [_vp, _vp, _vp, _vp, _int, _i64, _vp]),
    "tl_kv_commit": (_int, [_vp, _vp, _vp, _i64, _vp, _vp, _vp]),
    "tl_tree_mask": (_int, [_vp, _vp, _int, _int, _vp, _int, _vp]),
    "tl_tree_attention": (_int, [_vp, _vp, _vp, _i64, _int, _vp, _int, ctypes.c_float, _vp, _i64, _vp, _vp]),
    "tl_tree_attention_workspace_bytes": (_sz, [_vp, _vp, _int]),
    "tl_tree_verify": (_int, [_vp, _i64, _vp, _i64, _i64, _vp, _vp, _vp, _int, _int, _vp, _vp, _vp, _i64, _vp, _vp, _vp]),
    "tl_rope_turns": (_int, [_int, ctypes.c_double, _int, ctypes.c_double, ctypes.c_double, ctypes.c_double, ctypes.c_double, _vp]),
    "tl_rope_rows": (_int, [_vp, _vp, _i64, _vp, _i64, _int, _int, _int, _int, _vp, _int, _vp]),
    "tl_rope_append": (_int, [_vp, _vp, _vp, _vp, _vp, _i64, _int, _vp, _i64, _vp, _vp, _int, _i64, _vp]),
    "tl_tree_positions": (_int, [_vp, _vp, _vp, _int, _int, _vp, _vp]),
    "tl_page_reserve": (_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "tl_page_release": (_int, [_vp, _vp, _vp]),
    "tl_page_fork": (_int, [_vp, _vp, _vp, _vp, _int, _vp]),
    "tl_page_compact": (_int, [_vp, _vp, _int, _vp, _vp, _vp]),
    "tl_page_workspace_bytes": (_sz, [_vp, _int]),
    "tl_page_copy": (_int, [_vp, _vp, _vp, _vp, _int, _vp]),
    "tl_read_amp_per_cta": (_int, [_i64, _i64, _i64, _int, _int, _int, _int, _i64, _int, _int, _int, _vp, _vp, _vp]),
}

# tl_option
(OPT_PDL, OPT_PREFETCH_STAGES, OPT_PAIR_KERNEL, OPT_PAIR_512, OPT_BOX_PER_BLOCK, OPT_MAX_STAGES, OPT_UMMA_M128,
 OPT_RELAYOUT_TMA, OPT_LOG, OPT_WAIT_LIMIT_US, OPT_STALL_ONCE, OPT_MOE_ROW_CAP, OPT_REDUCE_SPLIT, OPT_SM_LIMIT,
 OPT_NO_SCRATCH_PLANS, OPT_FFN_ONE_LAUNCH, OPT_GENERIC_RAW, OPT_PAIR_TMA_STORE, OPT_PLAN_AS_IF_SMS) = range(19)
FLAVOUR_N_BF16, FLAVOUR_K_BF16, FLAVOUR_K_FP8 = 0, 1, 2

_lib = None


class TileLensError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().tl_status_string(status).decode()
        extra = f" (cuda error {lib().tl_last_cuda_error()})" if status == 4 else ""
        super().__init__(f"{where}: {msg}{extra}")


def lib() -> ctypes.CDLL:
    """Loads libtilelens.so; raises if it has not been built (no CPU fallback exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2607_04031_b200.build` "
                "(nvcc, sm_100a). The CUDA library is the only implementation of this path.")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(L, name)          # AttributeError if the library lacks a declared symbol
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def declared_symbols():
    return list(_SIGNATURES)


def _check(status: int, where: str):
    if status != TL_OK:
        raise TileLensError(status, where)


def _dev_ptr(t: torch.Tensor) -> int:
    if not t.is_cuda:
        raise ValueError("expected a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    return t.data_ptr()


def _stream_ptr(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def status_string(status: int) -> str:
    return lib().tl_status_string(status).decode()


def set_stream(stream=None):
    _check(lib().tl_set_stream(_stream_ptr(stream)), "tl_set_stream")


def device_status():
    """Synchronises; raises TileLensError(TL_ERR_TIMEOUT) if a kernel abandoned a bounded wait."""
    detail = ctypes.c_uint32(0)
    st = lib().tl_device_status(ctypes.byref(detail))
    if st != TL_OK:
        raise TileLensError(st, f"tl_device_status detail=0x{detail.value:x}")


def set_option(option: int, value: int):
    _check(lib().tl_set_option(option, value), "tl_set_option")


def get_option(option: int) -> int:
    return int(lib().tl_get_option(option))


class option:
    """with option(OPT_x, v): ... sets a library switch for the block and restores the previous value afterwards."""

    def __init__(self, opt: int, value: int):
        self.opt, self.value = opt, value

    def __enter__(self):
        self.old = get_option(self.opt)
        set_option(self.opt, self.value)
        return self

    def __exit__(self, *exc):
        set_option(self.opt, self.old)
        return False


class GemmPlan(ctypes.Structure):
    """tl_gemm_plan_info"""
    _fields_ = [("cta_m", ctypes.c_int32), ("cta_n", ctypes.c_int32), ("cta_k", ctypes.c_int32),
                ("pair_kernel", ctypes.c_int32), ("stream_k", ctypes.c_int32), ("grid", ctypes.c_int32),
                ("stages", ctypes.c_int32), ("weights_on_n", ctypes.c_int32), ("generic_path", ctypes.c_int32),
                ("cluster_k", ctypes.c_int32), ("pair_tiles_512", ctypes.c_int64), ("pair_tiles_256", ctypes.c_int64),
                ("chained", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("workspace_bytes", ctypes.c_uint64)]

    def as_dict(self):
        return {name: int(getattr(self, name)) for name, _ in self._fields_ if name != "reserved"}

    @property
    def cta(self):
        return (int(self.cta_m), int(self.cta_n), int(self.cta_k))


def gemm_plan(M: int, N: int, K: int, G: int = 4096, block_rows: int = 16, block_cols: int = 128, cta=(0, 0, 0),
              E: int = 0, flavour: int = FLAVOUR_N_BF16) -> GemmPlan:
    """The schedule a GEMM call with these sizes runs (host only, nothing is enqueued)."""
    out = GemmPlan()
    _check(lib().tl_gemm_plan(M, N, K, G, block_rows, block_cols, cta[0], cta[1], cta[2], E, flavour,
                              ctypes.addressof(out)), "tl_gemm_plan")
    return out


def gemm_last_plan() -> GemmPlan:
    """What this thread's most recent GEMM launch ran."""
    out = GemmPlan()
    _check(lib().tl_gemm_last_plan(ctypes.addressof(out)), "tl_gemm_last_plan")
    return out


def relayout(src: torch.Tensor, dst: torch.Tensor, rows: int, cols: int, elem_bytes: int, G: int,
             block_rows: int, block_cols: int, direction: int, stream=None):
    _check(lib().tl_relayout_on(_dev_ptr(src), _dev_ptr(dst), rows, cols, elem_bytes, G, block_rows, block_cols,
                                direction, _stream_ptr(stream)), "tl_relayout")


def relayout_batch(srcs, dsts, shapes, elem_bytes: int, G: int, block_rows: int, block_cols: int,
                   direction: int = TO_TILE_MAJOR, stream=None):
    """srcs, dsts: lists of CUDA tensors; shapes: list of (rows, cols).  One launch for the whole list where possible."""
    n = len(srcs)
    ptr_arr, i64_arr = ctypes.c_void_p * n, ctypes.c_int64 * n
    _check(lib().tl_relayout_batch(n, ptr_arr(*[_dev_ptr(t) for t in srcs]), ptr_arr(*[_dev_ptr(t) for t in dsts]),
                                   i64_arr(*[int(r) for r, _ in shapes]), i64_arr(*[int(c) for _, c in shapes]),
                                   elem_bytes, G, block_rows, block_cols, direction, _stream_ptr(stream)),
           "tl_relayout_batch")


def gemm(A: torch.Tensor, B: torch.Tensor, C: torch.Tensor, M: int, N: int, K: int, G: int = 4096,
         block_rows: int = 16, block_cols: int = 128, cta=(0, 0, 0), stream=None):
    """C (fp32 [M,N]) = A (bf16 [M,K]) x B (bf16, tile-major blocks; block_rows == 0: row-major [K,N])."""
    _check(lib().tl_gemm(_dev_ptr(A), _dev_ptr(B), _dev_ptr(C), M, N, K, G, block_rows, block_cols,
                         cta[0], cta[1], cta[2], _stream_ptr(stream)), "tl_gemm")


def gemm_grouped(A: torch.Tensor, B: torch.Tensor, C: torch.Tensor, offsets: torch.Tensor, E: int,
                 total_rows: int, N: int, K: int, G: int = 4096, block_rows: int = 16, block_cols: int = 128,
                 cta=(0, 0, 0), stream=None):
    _check(lib().tl_gemm_grouped(_dev_ptr(A), _dev_ptr(B), _dev_ptr(C), _dev_ptr(offsets), E, total_rows, N, K, G,
                                 block_rows, block_cols, cta[0], cta[1], cta[2], _stream_ptr(stream)),
           "tl_gemm_grouped")


def gemm_bf16(A: torch.Tensor, B: torch.Tensor, C_bf16: torch.Tensor, M: int, N: int, K: int, G: int = 4096,
              block_rows: int = 16, block_cols: int = 128, cta=(0, 0, 0), stream=None):
    """tl_gemm with a bf16 C."""
    _check(lib().tl_gemm_bf16(_dev_ptr(A), _dev_ptr(B), _dev_ptr(C_bf16), M, N, K, G, block_rows, block_cols,
                              cta[0], cta[1], cta[2], _stream_ptr(stream)), "tl_gemm_bf16")


def gemm_grouped_bf16(A: torch.Tensor, B: torch.Tensor, C_bf16: torch.Tensor, offsets: torch.Tensor, E: int,
                      total_rows: int, N: int, K: int, G: int = 4096, block_rows: int = 16, block_cols: int = 128,
                      cta=(0, 0, 0), stream=None):
    _check(lib().tl_gemm_grouped_bf16(_dev_ptr(A), _dev_ptr(B), _dev_ptr(C_bf16), _dev_ptr(offsets), E, total_rows, N, K,
                                      G, block_rows, block_cols, cta[0], cta[1], cta[2], _stream_ptr(stream)),
           "tl_gemm_grouped_bf16")


def gemm_grouped_swiglu(A: torch.Tensor, B_gate_up: torch.Tensor, H: torch.Tensor, offsets: torch.Tensor, E: int,
                        total_rows: int, N: int, K: int, G: int = 4096, block_rows: int = 16, block_cols: int = 128,
                        cta=(0, 0, 0), stream=None):
    """H (bf16 [rows, N/2]) = silu(gate) * up, gate/up = columns 2j / 2j+1 of A x B."""
    _check(lib().tl_gemm_grouped_swiglu(_dev_ptr(A), _dev_ptr(B_gate_up), _dev_ptr(H), _dev_ptr(offsets), E, total_rows,
                                        N, K, G, block_rows, block_cols, cta[0], cta[1], cta[2], _stream_ptr(stream)),
           "tl_gemm_grouped_swiglu")


def moe_ffn(X: torch.Tensor, W_gate_up: torch.Tensor, W_down: torch.Tensor, H: torch.Tensor, Y: torch.Tensor,
            offsets: torch.Tensor, E: int, total_rows: int, hidden: int, inter: int, G: int = 4096,
            block_rows: int = 16, block_cols: int = 128, stream=None):
    _check(lib().tl_moe_ffn(_dev_ptr(X), _dev_ptr(W_gate_up), _dev_ptr(W_down), _dev_ptr(H), _dev_ptr(Y),
                            _dev_ptr(offsets), E, total_rows, hidden, inter, G, block_rows, block_cols,
                            _stream_ptr(stream)), "tl_moe_ffn")


def gemm_kmajor(A: torch.Tensor, B_nk: torch.Tensor, C: torch.Tensor, M: int, N: int, K: int, G: int = 4096,
                tile_n: int = 32, tile_k: int = 64, cta=(0, 0, 0), stream=None):
    """Weights stored [N][K] (K contiguous), tile-major as Eq. 2 prints it; tile_n == 0: the plain [N][K] array."""
    _check(lib().tl_gemm_kmajor(_dev_ptr(A), _dev_ptr(B_nk), _dev_ptr(C), M, N, K, G, tile_n, tile_k,
                                cta[0], cta[1], cta[2], _stream_ptr(stream)), "tl_gemm_kmajor")


def gemm_grouped_kmajor(A: torch.Tensor, B_nk: torch.Tensor, C: torch.Tensor, offsets: torch.Tensor, E: int,
                        total_rows: int, N: int, K: int, G: int = 4096, tile_n: int = 32, tile_k: int = 64,
                        cta=(0, 0, 0), stream=None):
    _check(lib().tl_gemm_grouped_kmajor(_dev_ptr(A), _dev_ptr(B_nk), _dev_ptr(C), _dev_ptr(offsets), E, total_rows,
                                        N, K, G, tile_n, tile_k, cta[0], cta[1], cta[2], _stream_ptr(stream)),
           "tl_gemm_grouped_kmajor")


def gemm_fp8_kmajor(A: torch.Tensor, B_nk: torch.Tensor, C: torch.Tensor, M: int, N: int, K: int, G: int = 4096,
                    tile_n: int = 64, tile_k: int = 64, cta=(0, 0, 0), stream=None):
    """FP8 (E4M3) A [M,K] and weights [N,K] (tile-major tile_n x tile_k bytes, or plain when tile_n == 0); C fp32."""
    _check(lib().tl_gemm_fp8_kmajor(_dev_ptr(A), _dev_ptr(B_nk), _dev_ptr(C), M, N, K, G, tile_n, tile_k,
                                    cta[0], cta[1], cta[2], _stream_ptr(stream)), "tl_gemm_fp8_kmajor")


def gemm_grouped_fp8_kmajor(A: torch.Tensor, B_nk: torch.Tensor, C: torch.Tensor, offsets: torch.Tensor, E: int,
                            total_rows: int, N: int, K: int, G: int = 4096, tile_n: int = 64, tile_k: int = 64,
                            cta=(0, 0, 0), stream=None):
    _check(lib().tl_gemm_grouped_fp8_kmajor(_dev_ptr(A), _dev_ptr(B_nk), _dev_ptr(C), _dev_ptr(offsets), E, total_rows,
                                            N, K, G, tile_n, tile_k, cta[0], cta[1], cta[2], _stream_ptr(stream)),
           "tl_gemm_grouped_fp8_kmajor")


def gemm_workspace_bytes(M: int, N: int, K: int, cta=(0, 0, 0)) -> int:
    return int(lib().tl_gemm_workspace_bytes(M, N, K, cta[0], cta[1], cta[2]))


def set_workspace(buf: torch.Tensor | None):
    if buf is None:
        _check(lib().tl_set_workspace(None, 0), "tl_set_workspace")
    else:
        _check(lib().tl_set_workspace(_dev_ptr(buf), buf.numel() * buf.element_size()), "tl_set_workspace")


def gemm_host_scratch_bytes(M: int, N: int, K: int) -> int:
    return int(lib().tl_gemm_host_scratch_bytes(M, N, K))


def gemm_host(A_host: torch.Tensor, B_rowmajor_host: torch.Tensor, C_host: torch.Tensor, M: int, N: int, K: int,
              scratch: torch.Tensor, G: int = 4096, block_rows: int = 16, block_cols: int = 128, cta=(0, 0, 0),
              stream=None):
    """Host buffers in, host buffer out: H2D copies, relayout, GEMM and D2H copy all inside the call."""
    for t in (A_host, B_rowmajor_host, C_host):
        if t.is_cuda or not t.is_contiguous():
            raise ValueError("gemm_host takes contiguous host tensors")
    _check(lib().tl_gemm_host(A_host.data_ptr(), B_rowmajor_host.data_ptr(), C_host.data_ptr(), M, N, K, G,
                              block_rows, block_cols, cta[0], cta[1], cta[2], _dev_ptr(scratch),
                              scratch.numel() * scratch.element_size(), _stream_ptr(stream)), "tl_gemm_host")


def gemm_noalloc(A: torch.Tensor, B: torch.Tensor, C: torch.Tensor, M: int, N: int, K: int, G: int = 4096,
                 block_rows: int = 16, block_cols: int = 128, cta=(0, 0, 0), timeout_flag: torch.Tensor | None = None,
                 stream=None):
    """tl_gemm for processes that may not allocate device memory: split-K scratch is a fixed array
    inside the library (8 MiB per GPU).  `timeout_flag`: optional zeroed uint32/int32 CUDA tensor."""
    flag = _dev_ptr(timeout_flag) if timeout_flag is not None else None
    _check(lib().tl_gemm_noalloc(_dev_ptr(A), _dev_ptr(B), _dev_ptr(C), M, N, K, G, block_rows, block_cols,
                                 cta[0], cta[1], cta[2], flag, _stream_ptr(stream)), "tl_gemm_noalloc")


class HwDesc(ctypes.Structure):
    """tl_hw_desc: a tensor view of the column-major K x N matrix plus the memory tile (a, b) and the leading stride."""
    _fields_ = [("rank", ctypes.c_int32), ("elem_bytes", ctypes.c_int32), ("dims", ctypes.c_int64 * 5),
                ("strides", ctypes.c_int64 * 5), ("box", ctypes.c_int32 * 5), ("tile_a", ctypes.c_int32),
                ("tile_b", ctypes.c_int32), ("leading_stride", ctypes.c_int64)]


def hw_desc(dims, strides, box, elem_bytes: int, tile_a: int, tile_b: int, leading_stride: int) -> HwDesc:
    d = HwDesc()
    d.rank, d.elem_bytes, d.tile_a, d.tile_b, d.leading_stride = len(dims), elem_bytes, tile_a, tile_b, leading_stride
    for k in range(min(len(dims), 5)):
        d.dims[k], d.strides[k], d.box[k] = dims[k], strides[k], box[k]
    return d


def hw_box_offsets(desc: HwDesc, coords: torch.Tensor, offsets: torch.Tensor, stream=None):
    """coords: int32 CUDA tensor [n_boxes, rank]; offsets: uint64/int64 CUDA tensor [n_boxes * prod(box)]."""
    _check(lib().tl_hw_box_offsets(ctypes.addressof(desc), _dev_ptr(coords), coords.shape[0], _dev_ptr(offsets),
                                   _stream_ptr(stream)), "tl_hw_box_offsets")


def hw_box_load(desc: HwDesc, src: torch.Tensor, coords: torch.Tensor, dst: torch.Tensor, stream=None):
    """src: the tile-major buffer; dst: n_boxes dense boxes."""
    _check(lib().tl_hw_box_load(ctypes.addressof(desc), _dev_ptr(src), src.numel() * src.element_size(),
                                _dev_ptr(coords), coords.shape[0], _dev_ptr(dst), _stream_ptr(stream)),
           "tl_hw_box_load")


def read_amp(M: int, N: int, K: int, cta, layout: int, G: int, block_rows: int = 0, block_cols: int = 0,
             elem_bytes: int = 2):
    """Returns (bytes_fetched, bytes_used, requests), exact integers."""
    f, u, q = ctypes.c_uint64(), ctypes.c_uint64(), ctypes.c_uint64()
    _check(lib().tl_read_amp(M, N, K, cta[0], cta[1], cta[2], layout, G, block_rows, block_cols, elem_bytes,
                             ctypes.byref(f), ctypes.byref(u), ctypes.byref(q)), "tl_read_amp")
    return int(f.value), int(u.value), int(q.value)


def read_amp_async(M: int, N: int, K: int, cta, layout: int, G: int, block_rows: int, block_cols: int, elem_bytes: int,
                   totals: torch.Tensor, stream=None):
    """totals: CUDA tensor of 3 int64/uint64 that receives (bytes_fetched, bytes_used, requests); no wait."""
    _check(lib().tl_read_amp_async(M, N, K, cta[0], cta[1], cta[2], layout, G, block_rows, block_cols, elem_bytes,
                                   _dev_ptr(totals), _stream_ptr(stream)), "tl_read_amp_async")


class ReadAmpCfg(ctypes.Structure):
    """tl_read_amp_cfg"""
    _fields_ = [("M", ctypes.c_int64), ("N", ctypes.c_int64), ("K", ctypes.c_int64), ("cta_m", ctypes.c_int32),
                ("cta_n", ctypes.c_int32), ("cta_k", ctypes.c_int32), ("layout", ctypes.c_int32), ("G", ctypes.c_int64),
                ("block_rows", ctypes.c_int32), ("block_cols", ctypes.c_int32), ("elem_bytes", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


def read_amp_cfgs(cfgs):
    """cfgs: iterable of (M, N, K, cta, layout, G, block_rows, block_cols, elem_bytes) -> ctypes array for read_amp_batch."""
    cfgs = list(cfgs)
    arr = (ReadAmpCfg * len(cfgs))()
    for a, (M, N, K, cta, layout, G, br, bc, s) in zip(arr, cfgs):
        a.M, a.N, a.K, a.cta_m, a.cta_n, a.cta_k, a.layout, a.G = M, N, K, cta[0], cta[1], cta[2], layout, G
        a.block_rows, a.block_cols, a.elem_bytes = br, bc, s
    return arr


def read_amp_batch(cfg_array, totals: torch.Tensor, stream=None):
    """One launch for up to 16 configurations; totals: CUDA int64/uint64 tensor [n, 3]; no wait."""
    _check(lib().tl_read_amp_batch(ctypes.addressof(cfg_array), len(cfg_array), _dev_ptr(totals), _stream_ptr(stream)),
           "tl_read_amp_batch")


def read_amp_shared(M: int, N: int, K: int, cta, wave_ctas: int, layout: int, G: int, block_rows: int = 0,
                    block_cols: int = 0, elem_bytes: int = 2):
    """(bytes_fetched, bytes_needed, requests) when the wave_ctas co-resident CTA tiles share blocks per K step."""
    f, u, q = ctypes.c_uint64(), ctypes.c_uint64(), ctypes.c_uint64()
    _check(lib().tl_read_amp_shared(M, N, K, cta[0], cta[1], cta[2], wave_ctas, layout, G, block_rows, block_cols,
                                    elem_bytes, ctypes.byref(f), ctypes.byref(u), ctypes.byref(q)), "tl_read_amp_shared")
    return int(f.value), int(u.value), int(q.value)


def prefetch_degree(bandwidth_bytes_per_s: float, latency_s: float, G: int, n_sm: int, ctas_per_sm: int,
                    requests_per_tile: int, K: int, cta_k: int, collision_factor: float = 1.0) -> int:
    d = int(lib().tl_prefetch_degree(bandwidth_bytes_per_s, latency_s, G, n_sm, ctas_per_sm, requests_per_tile, K,
                                     cta_k, collision_factor))
    if d < 0:
        raise ValueError("tl_prefetch_degree: bad arguments")
    return d


def tile_arrival_latency(latencies, requests: int, threshold: float = 0.0):
    """(E[first arrival], E[last arrival], P(last arrival > threshold)) for `requests` requests per tile whose
    latencies are independent draws from the sample `latencies` (host arithmetic, Section 6.5)."""
    import numpy as np
    x = np.ascontiguousarray(latencies, dtype=np.float64)
    first, last, late = ctypes.c_double(), ctypes.c_double(), ctypes.c_double()
    _check(lib().tl_tile_arrival_latency(x.ctypes.data, x.size, requests, threshold, ctypes.byref(first),
                                         ctypes.byref(last), ctypes.byref(late)), "tl_tile_arrival_latency")
    return first.value, last.value, late.value


def read_amp_grouped(offsets_host, N: int, K: int, cta, layout: int, G: int, block_rows: int = 0,
                     block_cols: int = 0, elem_bytes: int = 2):
    import numpy as np
    offs = np.ascontiguousarray(offsets_host, dtype=np.int32)
    f, u, q = ctypes.c_uint64(), ctypes.c_uint64(), ctypes.c_uint64()
    _check(lib().tl_read_amp_grouped(offs.ctypes.data, offs.size - 1, N, K, cta[0], cta[1], cta[2], layout, G,
                                     block_rows, block_cols, elem_bytes, ctypes.byref(f), ctypes.byref(u),
                                     ctypes.byref(q)), "tl_read_amp_grouped")
    return int(f.value), int(u.value), int(q.value)


def read_amp_per_cta(M: int, N: int, K: int, cta, layout: int, G: int, block_rows: int, block_cols: int,
                     elem_bytes: int, fetched: torch.Tensor, used: torch.Tensor, stream=None):
    _check(lib().tl_read_amp_per_cta(M, N, K, cta[0], cta[1], cta[2], layout, G, block_rows, block_cols, elem_bytes,
                                     _dev_ptr(fetched), _dev_ptr(used), _stream_ptr(stream)), "tl_read_amp_per_cta")


# ------------------------------------------------------------------ key/value cache for drafted tokens

KV_BF16, KV_E4M3, KV_INT8, KV_E2M1 = 0, 1, 2, 4
ELEM_BF16, ELEM_F32 = 0, 1
_KV_FORMATS = {torch.bfloat16: KV_BF16, torch.float8_e4m3fn: KV_E4M3, torch.int8: KV_INT8, torch.uint8: KV_E2M1}
_ELEMS = {torch.bfloat16: ELEM_BF16, torch.float32: ELEM_F32}


# (_ref of the descriptions below is their address: a ctypes reference would refer back to the object that holds it, and device memory
# would wait for Python's cycle collector.)


class KvCache(ctypes.Structure):
    """tl_kv_cache; keeps the tensors it was made from alive."""
    _fields_ = [("k", _vp), ("v", _vp), ("k_scale", _vp), ("v_scale", _vp), ("pages", _i64), ("page_stride", _i64),
                ("head_stride", _i64), ("token_stride", _i64), ("scale_page_stride", _i64), ("scale_head_stride", _i64),
                ("format", ctypes.c_int32), ("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("page_tokens", ctypes.c_int32), ("k_group", _vp), ("v_group", _vp), ("group_page_stride", _i64),
                ("group_head_stride", _i64)]


class KvBatch(ctypes.Structure):
    """tl_kv_batch; keeps the tensors it was made from alive."""
    _fields_ = [("page_table", _vp), ("start", _vp), ("token_offsets", _vp), ("table_stride", _i64),
                ("requests", ctypes.c_int32), ("tokens", ctypes.c_int32)]
    _device = None                                           # of the tensors, where it was made from some


def _cuda(t: torch.Tensor, name: str, dtype=None, dims=None) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name}: expected a CUDA tensor")
    if dtype is not None and t.dtype is not dtype:
        raise ValueError(f"{name}: expected {dtype}, got {t.dtype}")
    if dims is not None and t.dim() != dims:
        raise ValueError(f"{name}: expected {dims} dimensions, got {t.dim()}")
    return t


def _elsewhere(t: torch.Tensor, name: str, device: int) -> ValueError:
    return ValueError(f"{name}: expected a tensor on cuda:{device}, got {'cuda:%d' % t.get_device() if t.is_cuda else 'the CPU'}")


def _int32(t: torch.Tensor, name: str, shape, device: int) -> int:
    if t.dtype is not torch.int32 or t.get_device() != device or t.shape != shape or not t.is_contiguous():
        if t.is_cuda and t.get_device() != device:
            raise _elsewhere(t, name, device)
        raise ValueError(f"{name}: expected a contiguous CUDA tensor of int32 and shape {tuple(shape)}, got {t.dtype}, {tuple(t.shape)}")
    return t.data_ptr()


def kv_cache(k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor | None = None,
             v_scale: torch.Tensor | None = None, k_group: torch.Tensor | None = None,
             v_group: torch.Tensor | None = None) -> KvCache:
    """k, v: [pages, heads, page_tokens, head_dim], bf16, float8_e4m3fn or int8, the last dimension contiguous (the other
    strides are free: a permuted [pages, page_tokens, heads, head_dim] pool serves too).  k_scale, v_scale: fp32
    [pages, heads, page_tokens], for the 8-bit and 4-bit formats.  The 4-bit one: k, v uint8 [..., head_dim / 2], two E2M1 codes
    a byte, and k_group, v_group float8_e4m3fn [pages, heads, page_tokens, head_dim / 16]."""
    _cuda(k, "k", dims=4), _cuda(v, "v", k.dtype, 4)
    if k.dtype not in _KV_FORMATS:
        raise ValueError(f"k: expected bf16, float8_e4m3fn, int8 or (4 bits) uint8, got {k.dtype}")
    if v.shape != k.shape or v.stride() != k.stride() or k.stride(3) != 1:
        raise ValueError("k and v: expected one shape and one set of strides, the last dimension contiguous")
    c = KvCache()
    c.format = _KV_FORMATS[k.dtype]
    two = 2 if c.format == KV_E2M1 else 1                    # elements to one of the tensors'
    c.pages, c.heads, c.page_tokens, c.head_dim = k.shape
    c.head_dim *= two
    c.k, c.v = k.data_ptr(), v.data_ptr()
    c.page_stride, c.head_stride, c.token_stride = (n * two for n in k.stride()[:3])
    if c.format != KV_BF16:
        for t, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            _cuda(t, name, torch.float32, 3)
            if tuple(t.shape) != tuple(k.shape[:3]) or t.stride() != k_scale.stride() or t.stride(2) != 1:
                raise ValueError(f"{name}: expected [pages, heads, page_tokens], the tokens contiguous, one set of strides")
        c.k_scale, c.v_scale = k_scale.data_ptr(), v_scale.data_ptr()
        c.scale_page_stride, c.scale_head_stride = k_scale.stride()[:2]
    elif k_scale is not None or v_scale is not None:
        raise ValueError("a bf16 cache has no scales")
    if c.format == KV_E2M1:
        n = c.head_dim // 16
        for t, name in ((k_group, "k_group"), (v_group, "v_group")):
            _cuda(t, name, torch.float8_e4m3fn, 4)
            if tuple(t.shape) != (*k.shape[:3], n) or t.stride() != k_group.stride() or t.stride()[2:] != (n, 1):
                raise ValueError(f"{name}: expected [pages, heads, page_tokens, head_dim / 16], a head's tokens contiguous, one set of strides")
        c.k_group, c.v_group = k_group.data_ptr(), v_group.data_ptr()
        c.group_page_stride, c.group_head_stride = k_group.stride()[:2]
    elif k_group is not None or v_group is not None:
        raise ValueError("only a 4-bit cache has group scales")
    c._tensors, c._ref, c._device = (k, v, k_scale, v_scale, k_group, v_group), ctypes.addressof(c), k.get_device()
    for t, name in ((v, "v"), (k_scale, "k_scale"), (v_scale, "v_scale"), (k_group, "k_group"), (v_group, "v_group")):
        if t is not None and t.get_device() != c._device:
            raise _elsewhere(t, name, c._device)
    return c


def kv_batch(page_table: torch.Tensor, start: torch.Tensor, token_offsets: torch.Tensor, tokens: int) -> KvBatch:
    """page_table: int32 [requests, n]; start: int32 [requests]; token_offsets: int32 [requests + 1]."""
    _cuda(page_table, "page_table", torch.int32, 2)
    n = page_table.shape[0]
    b = KvBatch()
    b._device = device = page_table.get_device()
    b.page_table = _int32(page_table, "page_table", page_table.shape, device)
    b.start = _int32(start, "start", (n,), device)
    b.token_offsets = _int32(token_offsets, "token_offsets", (n + 1,), device)
    b.table_stride = page_table.shape[1]
    b.requests, b.tokens = n, int(tokens)
    b._tensors, b._ref = (page_table, start, token_offsets), ctypes.addressof(b)
    return b


# The calls below run once per layer and step, next to kernels of a few microseconds: their checks read every attribute
# once and build nothing that is not needed.

_current_device, _current_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream


def _kv_raw_stream(stream, device: int) -> int:
    """The stream's handle.  The library launches on the current device, which has to be the tensors'."""
    if stream is not None:
        return stream.cuda_stream
    if _current_device() != device:
        raise ValueError(f"the tensors lie on cuda:{device}, the current device is cuda:{_current_device()}")
    return _current_stream(device)


def _apart(cache: KvCache, batch: KvBatch) -> ValueError:
    return ValueError(f"the batch lies on cuda:{batch._device}, the cache on cuda:{cache._device}")


def _kv_pair(k, v, cache, batch):
    """(pointer of k, pointer of v, element type, row stride) of a step's two [tokens, heads, head_dim] tensors."""
    shape, stride, dtype = k.shape, k.stride(), k.dtype
    if v.shape != shape or v.stride() != stride or v.dtype is not dtype:
        raise ValueError("k and v: expected one shape, one element type and one set of strides")
    if dtype not in _ELEMS:
        raise ValueError(f"k, v: expected CUDA tensors of bf16 or fp32, got {dtype}")
    device = cache._device
    if batch._device != device and batch._device is not None:
        raise _apart(cache, batch)
    if k.get_device() != device or v.get_device() != device:
        raise _elsewhere(*((v, "v") if k.get_device() == device else (k, "k")), device)
    tokens, heads, dim = batch.tokens, cache.heads, cache.head_dim
    if shape != (tokens, heads, dim) or stride[2] != 1 or (heads > 1 and stride[1] != dim):
        raise ValueError("k, v: expected [tokens, heads, head_dim] with contiguous heads")
    return k.data_ptr(), v.data_ptr(), _ELEMS[dtype], stride[0] if tokens > 1 else heads * dim


def kv_append(cache: KvCache, batch: KvBatch, k: torch.Tensor, v: torch.Tensor, stream=None):
    """Quantises k, v ([tokens, heads, head_dim], bf16 or fp32; column ranges of a fused product's output serve) into the
    cache, request b's i-th row at position start[b] + i."""
    kp, vp, elem, stride = _kv_pair(k, v, cache, batch)
    st = lib().tl_kv_append(cache._ref, batch._ref, kp, vp, elem, stride, _kv_raw_stream(stream, cache._device))
    if st:
        _check(st, "tl_kv_append")


def kv_read(cache: KvCache, batch: KvBatch, k: torch.Tensor, v: torch.Tensor, stream=None):
    """Reads the positions kv_append with the same batch writes back into k, v (bf16 or fp32)."""
    kp, vp, elem, stride = _kv_pair(k, v, cache, batch)
    st = lib().tl_kv_read(cache._ref, batch._ref, kp, vp, elem, stride, _kv_raw_stream(stream, cache._device))
    if st:
        _check(st, "tl_kv_read")


def kv_commit(cache: KvCache, batch: KvBatch, accepted: torch.Tensor, n_accepted: torch.Tensor,
              new_start: torch.Tensor | None = None, stream=None):
    """Moves the rows of accepted[b][i], i < n_accepted[b], to positions start[b] + i; new_start = start + n_accepted."""
    shape, n = accepted.shape, batch.requests
    if len(shape) != 2:
        raise ValueError("accepted: expected [requests, n]")
    device = cache._device
    if batch._device != device and batch._device is not None:
        raise _apart(cache, batch)
    a = _int32(accepted, "accepted", (n, shape[1]), device)
    st = lib().tl_kv_commit(cache._ref, batch._ref, a, shape[1], _int32(n_accepted, "n_accepted", (n,), device),
                            _int32(new_start, "new_start", (n,), device) if new_start is not None else None,
                            _kv_raw_stream(stream, device))
    if st:
        _check(st, "tl_kv_commit")


def tree_mask(parents: torch.Tensor, token_offsets: torch.Tensor, mask: torch.Tensor, stream=None):
    """mask (int32 [tokens, words]): bit j of row i is set when token i of its request sees token j."""
    _cuda(mask, "mask", torch.int32, 2)
    device = mask.get_device()
    m = _int32(mask, "mask", (parents.shape[0], mask.shape[1]), device)
    _check(lib().tl_tree_mask(_int32(parents, "parents", (mask.shape[0],), device),
                              _int32(token_offsets, "token_offsets", (token_offsets.shape[0],), device), token_offsets.shape[0] - 1,
                              mask.shape[0], m, mask.shape[1], _kv_raw_stream(stream, device)), "tl_tree_mask")


def tree_attention(cache: KvCache, batch: KvBatch, q: torch.Tensor, out: torch.Tensor, mask: torch.Tensor | None = None,
                   scale: float | None = None, lse: torch.Tensor | None = None, stream=None):
    """out (bf16 [tokens, q_heads, head_dim]) = attention of q over the cache, which holds the step's own rows already.
    mask: int32 [tokens, words] (None: causal within the step's rows); scale: 1 / sqrt(head_dim) by default; lse: fp32
    [tokens, q_heads].  Rows of q and out may be strided."""
    shape, qs, os_ = q.shape, q.stride(), out.stride()
    tokens, dim = batch.tokens, cache.head_dim
    if q.dtype is not torch.bfloat16 or out.dtype is not torch.bfloat16:
        raise ValueError("q, out: expected CUDA tensors of bf16")
    if len(shape) != 3 or out.shape != shape or shape[0] != tokens or shape[2] != dim or qs[2] != 1 or os_[2] != 1 or \
            (shape[1] > 1 and (qs[1] != dim or os_[1] != dim)):
        raise ValueError("q, out: expected [tokens, q_heads, head_dim] with contiguous heads")
    device = cache._device
    if batch._device != device and batch._device is not None:
        raise _apart(cache, batch)
    if q.get_device() != device or out.get_device() != device:
        raise _elsewhere(*((out, "out") if q.get_device() == device else (q, "q")), device)
    heads, words, m, l = shape[1], 0, None, None
    wide = heads * dim
    if mask is not None:
        words = mask.shape[1]
        m = _int32(mask, "mask", (tokens, words), device)
    if lse is not None:
        if _cuda(lse, "lse", torch.float32).shape != shape[:2] or not lse.is_contiguous():
            raise ValueError("lse: expected a contiguous [tokens, q_heads]")
        if lse.get_device() != device:
            raise _elsewhere(lse, "lse", device)
        l = lse.data_ptr()
    st = lib().tl_tree_attention(cache._ref, batch._ref, q.data_ptr(), qs[0] if tokens > 1 else wide, heads, m, words,
                                 dim ** -0.5 if scale is None else scale, out.data_ptr(), os_[0] if tokens > 1 else wide, l,
                                 _kv_raw_stream(stream, device))
    if st:
        _check(st, "tl_tree_attention")


def tree_attention_workspace_bytes(cache: KvCache, batch: KvBatch, q_heads: int) -> int:
    return int(lib().tl_tree_attention_workspace_bytes(cache._ref, batch._ref, q_heads))


def tree_verify(target: torch.Tensor, draft: torch.Tensor | None, tokens: torch.Tensor, parents: torch.Tensor,
                token_offsets: torch.Tensor, accept: torch.Tensor, sample: torch.Tensor, accepted: torch.Tensor,
                n_accepted: torch.Tensor, next_token: torch.Tensor, stream=None):
    """Which drafts the target's distribution keeps, and the token that follows them.

    target, draft: fp32 [tokens, vocab], every row in memory of its own (draft None: the drafts were chosen without chance);
    tokens, parents: int32 [tokens]; accept: fp32 [tokens] and sample: fp32 [requests], uniform in [0, 1).  Written: accepted int32 [requests, n]
    (rows kept within the request, root first, then -1), n_accepted and next_token int32 [requests].
    """
    shape, ts, f32 = target.shape, target.stride(), torch.float32
    rows, vocab = shape
    requests, most = token_offsets.shape[0] - 1, accepted.shape[1]
    if target.dtype is not f32 or not target.is_cuda or (ts[1] != 1 and vocab > 1):
        raise ValueError("target: expected a CUDA tensor of fp32 with contiguous rows")
    device = target.get_device()
    dp = ds = 0
    if draft is not None:
        ds = draft.stride()
        if draft.dtype is not f32 or draft.shape != shape or (ds[1] != 1 and vocab > 1):
            raise ValueError("draft: expected target's shape, type and contiguous rows")
        if draft.get_device() != device:
            raise _elsewhere(draft, "draft", device)
        dp, ds = draft.data_ptr(), ds[0] if rows > 1 else vocab
    for t, name, n in ((accept, "accept", rows), (sample, "sample", requests)):
        if t.dtype is not f32 or t.shape != (n,) or not t.is_contiguous():
            raise ValueError(f"{name}: expected a contiguous CUDA tensor of {n} fp32 numbers")
        if t.get_device() != device:
            raise _elsewhere(t, name, device)
    st = lib().tl_tree_verify(target.data_ptr(), ts[0] if rows > 1 else vocab, dp, ds, vocab, _int32(tokens, "tokens", (rows,), device),
                              _int32(parents, "parents", (rows,), device),
                              _int32(token_offsets, "token_offsets", (requests + 1,), device), requests, rows, accept.data_ptr(),
                              sample.data_ptr(), _int32(accepted, "accepted", (requests, most), device), most,
                              _int32(n_accepted, "n_accepted", (requests,), device),
                              _int32(next_token, "next_token", (requests,), device), _kv_raw_stream(stream, device))
    if st:
        _check(st, "tl_tree_verify")


# ------------------------------------------------------------------ rotary positions

ROPE_HALF, ROPE_INTERLEAVED = 0, 1
ROPE_PLAIN, ROPE_LINEAR, ROPE_BANDS, ROPE_RAMP = 0, 1, 2, 3


class Rope(ctypes.Structure):
    """tl_rope; keeps the tensor it was made from alive."""
    _fields_ = [("turns", _vp), ("amplitude", ctypes.c_float), ("rotary_dim", ctypes.c_int32), ("layout", ctypes.c_int32)]


def rope_turns(rotary_dim: int, base: float = 10000.0, scaling: int = ROPE_PLAIN, factor: float = 1.0, original: float = 0.0,
               low: float = 1.0, high: float = 4.0) -> torch.Tensor:
    """The frequencies of a model's rotary positions, int64 [rotary_dim / 2] on the host (2^-64 turns per position): computed once
    and copied to the device.  low and high: turns over the original context (ROPE_BANDS usually 1 and 4, ROPE_RAMP 1 and 32)."""
    out = torch.empty(max(0, rotary_dim // 2), dtype=torch.int64)
    _check(lib().tl_rope_turns(rotary_dim, base, scaling, factor, original, low, high, out.data_ptr()), "tl_rope_turns")
    return out


def rope(turns: torch.Tensor, layout: int = ROPE_HALF, amplitude: float = 1.0) -> Rope:
    """turns: what rope_turns gave, on the device."""
    _cuda(turns, "turns", torch.int64, 1)
    if not turns.is_contiguous():
        raise ValueError("turns: expected a contiguous tensor")
    r = Rope()
    r.turns, r.amplitude, r.rotary_dim, r.layout = turns.data_ptr(), amplitude, 2 * turns.shape[0], layout
    r._tensors, r._ref, r._device = (turns,), ctypes.addressof(r), turns.get_device()
    return r


def _head_rows(t: torch.Tensor, name: str, shape, device: int):
    """Stride between the tokens of a [tokens, heads, head_dim] tensor with contiguous heads."""
    stride = t.stride()
    if t.shape != shape or (shape[2] > 1 and stride[2] != 1) or (shape[1] > 1 and stride[1] != shape[2]):
        raise ValueError(f"{name}: expected {tuple(shape)} with contiguous heads, got {tuple(t.shape)}")
    if t.get_device() != device:
        raise _elsewhere(t, name, device)
    return stride[0] if shape[0] > 1 else shape[1] * shape[2]


def rope_rows(rope: Rope, x: torch.Tensor, out: torch.Tensor, positions: torch.Tensor, inverse: bool = False, stream=None):
    """out = x [tokens, heads, head_dim] (bf16 or fp32; out may be x) turned by positions (int32 [tokens]); inverse: turned back, the
    gradient of x from that of out."""
    shape, device = x.shape, rope._device
    if x.dtype not in _ELEMS or out.dtype is not x.dtype:
        raise ValueError(f"x, out: expected CUDA tensors of bf16 or of fp32, got {x.dtype} and {out.dtype}")
    if len(shape) != 3:
        raise ValueError("x: expected [tokens, heads, head_dim]")
    xs, os_ = _head_rows(x, "x", shape, device), _head_rows(out, "out", shape, device)
    st = lib().tl_rope_rows(rope._ref, x.data_ptr(), xs, out.data_ptr(), os_, _ELEMS[x.dtype], shape[0], shape[1], shape[2],
                            _int32(positions, "positions", (shape[0],), device), 1 if inverse else 0, _kv_raw_stream(stream, device))
    if st:
        _check(st, "tl_rope_rows")


def rope_append(cache: KvCache, batch: KvBatch, rope: Rope, q: torch.Tensor | None, q_out: torch.Tensor | None, k: torch.Tensor,
                v: torch.Tensor, positions: torch.Tensor | None = None, stream=None):
    """q ([tokens, q_heads, head_dim], k's type; None: keys and values alone) turned into q_out (bf16), k turned and appended, v appended.
    positions: int32 [tokens] (None: every row's position in its sequence; in a draft tree tree_positions gives them)."""
    kp, vp, elem, stride = _kv_pair(k, v, cache, batch)
    device = cache._device
    if rope._device != device:
        raise ValueError(f"the frequencies lie on cuda:{rope._device}, the cache on cuda:{device}")
    qp = op = None
    heads = qs = os_ = 0
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out: expected both or neither")
    if q is not None:
        if q.dtype is not k.dtype or q_out.dtype is not torch.bfloat16:
            raise ValueError(f"q: expected {k.dtype}, q_out: expected bf16, got {q.dtype} and {q_out.dtype}")
        if len(q.shape) != 3:
            raise ValueError("q: expected [tokens, q_heads, head_dim]")
        shape = (batch.tokens, q.shape[1], cache.head_dim)
        qs, os_ = _head_rows(q, "q", shape, device), _head_rows(q_out, "q_out", shape, device)
        heads, qp, op = shape[1], q.data_ptr(), q_out.data_ptr()
    st = lib().tl_rope_append(cache._ref, batch._ref, rope._ref,
                              None if positions is None else _int32(positions, "positions", (batch.tokens,), device),
                              qp, qs, heads, op, os_, kp, vp, elem, stride, _kv_raw_stream(stream, device))
    if st:
        _check(st, "tl_rope_append")


def tree_positions(parents: torch.Tensor, token_offsets: torch.Tensor, start: torch.Tensor, positions: torch.Tensor, stream=None):
    """positions (int32 [tokens]) = start of the row's request + the row's depth in its tree."""
    _cuda(positions, "positions", torch.int32, 1)
    device, n = positions.get_device(), positions.shape[0]
    requests = start.shape[0]
    _check(lib().tl_tree_positions(_int32(parents, "parents", (n,), device), _int32(token_offsets, "token_offsets", (requests + 1,), device),
                                   _int32(start, "start", (requests,), device), requests, n, _int32(positions, "positions", (n,), device),
                                   _kv_raw_stream(stream, device)), "tl_tree_positions")


# ------------------------------------------------------------------ pages

class PageTables(ctypes.Structure):
    """tl_page_tables; keeps the tensors it was made from alive."""
    _fields_ = [("page_table", _vp), ("held", _vp), ("holders", _vp), ("table_stride", _i64), ("requests", ctypes.c_int32),
                ("pages", ctypes.c_int32), ("page_tokens", ctypes.c_int32)]


def page_tables(page_table: torch.Tensor, held: torch.Tensor, holders: torch.Tensor, page_tokens: int) -> PageTables:
    """page_table: int32 [requests, n]; held: int32 [requests], pages of each; holders: int32 [pages], entries that name each page
    (zeros for a pool that nobody uses yet, with held zeros)."""
    _cuda(page_table, "page_table", torch.int32, 2), _cuda(holders, "holders", torch.int32, 1)
    t = PageTables()
    t._device = device = page_table.get_device()
    t.requests, t.table_stride = page_table.shape
    t.pages, t.page_tokens = holders.shape[0], int(page_tokens)
    t.page_table = _int32(page_table, "page_table", page_table.shape, device)
    t.held = _int32(held, "held", (t.requests,), device)
    t.holders = _int32(holders, "holders", holders.shape, device)
    t._tensors, t._ref = (page_table, held, holders), ctypes.addressof(t)
    return t


def page_reserve(tables: PageTables, start: torch.Tensor, tokens: torch.Tensor, moves: torch.Tensor, n_moves: torch.Tensor,
                 missing: torch.Tensor, stream=None):
    """Pages for tokens[b] positions of every request (tokens[b] < 0: left alone), those of start[b] .. tokens[b] - 1 its own.  moves
    (int32 [requests or more, 3]) and n_moves (int32 [1]): what page_copy is to do; missing (int32 [1]): free pages that lack (then
    nothing has changed).  Of a shared page that is replaced the rows in front of start[b] are copied, none from tokens[b] on."""
    n, device = tables.requests, tables._device
    if moves.shape[0] < n:
        raise ValueError(f"moves: expected at least {n} rows")
    st = lib().tl_page_reserve(tables._ref, _int32(start, "start", (n,), device), _int32(tokens, "tokens", (n,), device),
                               _int32(moves, "moves", (moves.shape[0], 3), device), _int32(n_moves, "n_moves", (1,), device),
                               _int32(missing, "missing", (1,), device), _kv_raw_stream(stream, device))
    if st:
        _check(st, "tl_page_reserve")


def page_release(tables: PageTables, tokens: torch.Tensor | None = None, stream=None):
    """Request b keeps the pages of its first tokens[b] positions (all if negative; tokens None: no request keeps any)."""
    device = tables._device
    st = lib().tl_page_release(tables._ref, None if tokens is None else _int32(tokens, "tokens", (tables.requests,), device),
                               _kv_raw_stream(stream, device))
    if st:
        _check(st, "tl_page_release")


def page_fork(tables: PageTables, from_: torch.Tensor, to: torch.Tensor, tokens: torch.Tensor, stream=None):
    """Request to[f] (which holds nothing) shares the pages of the first tokens[f] positions of from_[f]."""
    device, shape = tables._device, from_.shape
    if len(shape) != 1:
        raise ValueError("from_: expected [forks]")
    st = lib().tl_page_fork(tables._ref, _int32(from_, "from_", shape, device), _int32(to, "to", shape, device),
                            _int32(tokens, "tokens", shape, device), shape[0], _kv_raw_stream(stream, device))
    if st:
        _check(st, "tl_page_fork")


def page_compact(tables: PageTables, moves: torch.Tensor, n_moves: torch.Tensor, in_use: torch.Tensor, stream=None):
    """The pages in use move to the front of the pool, at most as many as moves (int32 [n, 3]) has rows; n_moves and in_use: int32 [1]."""
    device = tables._device
    if len(moves.shape) != 2:
        raise ValueError("moves: expected [n, 3]")
    st = lib().tl_page_compact(tables._ref, _int32(moves, "moves", (moves.shape[0], 3), device), moves.shape[0],
                               _int32(n_moves, "n_moves", (1,), device), _int32(in_use, "in_use", (1,), device), _kv_raw_stream(stream, device))
    if st:
        _check(st, "tl_page_compact")


def page_workspace_bytes(tables: PageTables, forks: int = 0) -> int:
    return int(lib().tl_page_workspace_bytes(tables._ref, forks))


def page_copy(cache: KvCache, moves: torch.Tensor, n_moves: torch.Tensor | None = None, to: KvCache | None = None, stream=None):
    """For the first n_moves (all) rows of moves (int32 [n, 3]: from, to, tokens): copies the first tokens of a page of cache to a
    page of `to` (the same cache by default)."""
    device, dst = cache._device, cache if to is None else to
    if dst._device != device:
        raise ValueError(f"the caches lie on cuda:{device} and cuda:{dst._device}")
    if len(moves.shape) != 2:
        raise ValueError("moves: expected [n, 3]")
    st = lib().tl_page_copy(cache._ref, dst._ref, _int32(moves, "moves", (moves.shape[0], 3), device),
                            None if n_moves is None else _int32(n_moves, "n_moves", (1,), device), moves.shape[0],
                            _kv_raw_stream(stream, device))
    if st:
        _check(st, "tl_page_copy")
