"""ctypes binding of libdash_attn.so: argument marshalling only, every computation runs in the CUDA library.

Function names mirror the C ABI (include/dash_attn.h).  Tensors are torch CUDA tensors used purely as
device buffers; launches go to torch's current stream.  There is no fallback: if the shared library is
missing or cannot be loaded, every call raises.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import POINTER, c_char_p, c_float, c_int32, c_int64, c_size_t, c_uint32, c_void_p

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libdash_attn.so")
DEBUG_LIB_PATH = os.path.join(_PKG, "libdash_attn_debug.so")    # same library with bounds checks compiled in

DASH_F32, DASH_BF16 = 0, 1
DASH_OK = 0
STATUS = {0: "DASH_OK", -1: "DASH_ERR_INVALID_ARG", -2: "DASH_ERR_UNSUPPORTED", -3: "DASH_ERR_WORKSPACE",
          -4: "DASH_ERR_CAPACITY", -5: "DASH_ERR_CUDA", -6: "DASH_ERR_ARCH", -7: "DASH_ERR_TIMEOUT",
          -8: "DASH_ERR_TOO_LARGE"}

EXPORTS = [
    "dash_attn_workspace_bytes", "dash_attn_list_capacity", "dash_attn_list_offset",
    "dash_attn_block_summaries", "dash_attn_select", "dash_attn_attend_prefill", "dash_attn_attend_decode",
    "dash_attn_attend_decode_static", "dash_attn_bwd_attend_prefill",
    "dash_attn_bwd_workspace_bytes", "dash_attn_bwd_attend_prefill_tc",
    "dash_attn_block_summaries_paged", "dash_attn_fwd_decode_paged",
    "dash_attn_bwd_select_prefill", "dash_attn_bwd_block_summaries",
    "dash_attn_rope", "dash_attn_append_paged", "dash_attn_paged_workspace_bytes", "dash_attn_attend_chunk_paged",
    "dash_attn_key_mass_paged", "dash_attn_evict_paged",
    "dash_attn_fwd_prefill", "dash_attn_fwd_decode", "dash_attn_reset_status", "dash_attn_last_status",
    "dash_attn_launch_count", "dash_attn_strerror", "dash_attn_test_hooks",
    "dash_attn_test_hold_loads",
]


class DashError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {STATUS.get(code, code)} ({strerror(code)})")


class DashParams(ctypes.Structure):
    _fields_ = [
        ("struct_size", c_uint32), ("batch", c_int32), ("seq_q", c_int32), ("seq_kv", c_int32),
        ("h_q", c_int32), ("h_kv", c_int32), ("head_dim", c_int32), ("block", c_int32),
        ("dtype", c_int32), ("causal", c_int32), ("alpha", c_float), ("gamma", c_float), ("sigma", c_float),
        ("local_blocks", c_int32), ("q_to_kv", POINTER(c_int32)),
        ("q_stride", c_int64 * 3), ("k_stride", c_int64 * 3), ("v_stride", c_int64 * 3), ("o_stride", c_int64 * 3),
    ]


class DashPagedParams(ctypes.Structure):
    _fields_ = [
        ("struct_size", c_uint32), ("batch", c_int32), ("rows", c_int32), ("h_q", c_int32), ("h_kv", c_int32),
        ("head_dim", c_int32), ("dtype", c_int32), ("page_size", c_int32), ("max_pages", c_int32), ("num_pages", c_int32),
        ("q_stride", c_int64 * 2), ("kn_stride", c_int64 * 2), ("vn_stride", c_int64 * 2), ("o_stride", c_int64 * 2),
        ("k_stride", c_int64 * 3), ("v_stride", c_int64 * 3),
    ]


class DashRope(ctypes.Structure):
    _fields_ = [("struct_size", c_uint32), ("pairs", c_int32), ("axes", c_int32), ("interleaved", c_int32),
                ("axis", POINTER(c_int32)), ("inv_freq", POINTER(ctypes.c_double))]


_lib = None


def lib() -> ctypes.CDLL:
    """Loads the CUDA library; raises if it has not been built (there is no other implementation)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2605_18753_b200.build`; "
                               "the DashAttention path has no CPU or PyTorch fallback")
        L = ctypes.CDLL(LIB_PATH)
        P = POINTER(DashParams)
        L.dash_attn_workspace_bytes.restype = c_size_t
        L.dash_attn_workspace_bytes.argtypes = [P]
        L.dash_attn_list_capacity.restype = c_int64
        L.dash_attn_list_capacity.argtypes = [P]
        L.dash_attn_list_offset.restype = c_int64
        L.dash_attn_list_offset.argtypes = [P, c_int32, c_int32, c_int32]
        L.dash_attn_block_summaries.restype = ctypes.c_int
        L.dash_attn_block_summaries.argtypes = [P, c_void_p, c_void_p, c_int64, c_void_p, c_int32, c_int32, c_void_p, c_void_p]
        L.dash_attn_select.restype = ctypes.c_int
        L.dash_attn_select.argtypes = [P] + [c_void_p] * 9 + [c_size_t, c_void_p]
        L.dash_attn_attend_prefill.restype = ctypes.c_int
        L.dash_attn_attend_prefill.argtypes = [P] + [c_void_p] * 7 + [c_size_t, c_void_p]
        L.dash_attn_attend_decode.restype = ctypes.c_int
        L.dash_attn_attend_decode.argtypes = [P] + [c_void_p] * 9 + [c_size_t, c_void_p]
        L.dash_attn_attend_decode_static.restype = ctypes.c_int
        L.dash_attn_attend_decode_static.argtypes = [P] + [c_void_p] * 9
        L.dash_attn_bwd_attend_prefill.restype = ctypes.c_int
        L.dash_attn_bwd_attend_prefill.argtypes = [P] + [c_void_p] * 11
        L.dash_attn_bwd_workspace_bytes.restype = c_size_t
        L.dash_attn_bwd_workspace_bytes.argtypes = [P]
        L.dash_attn_bwd_attend_prefill_tc.restype = ctypes.c_int
        L.dash_attn_bwd_attend_prefill_tc.argtypes = [P] + [c_void_p] * 11 + [c_size_t, c_void_p]
        L.dash_attn_bwd_select_prefill.restype = ctypes.c_int
        L.dash_attn_bwd_select_prefill.argtypes = [P] + [c_void_p] * 9
        L.dash_attn_bwd_block_summaries.restype = ctypes.c_int
        L.dash_attn_bwd_block_summaries.argtypes = [P, c_void_p, c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_void_p]
        L.dash_attn_fwd_prefill.restype = ctypes.c_int
        L.dash_attn_fwd_prefill.argtypes = [P, c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_void_p, c_void_p,
                                            c_void_p, c_void_p, c_size_t, c_void_p]
        L.dash_attn_fwd_decode.restype = ctypes.c_int
        L.dash_attn_fwd_decode.argtypes = [P] + [c_void_p] * 7 + [c_size_t, c_void_p]
        L.dash_attn_block_summaries_paged.restype = ctypes.c_int
        L.dash_attn_block_summaries_paged.argtypes = [P, c_void_p, c_void_p, c_int32, c_int32, c_int32, c_void_p, c_int64,
                                                      c_void_p, c_int32, c_int32, c_void_p, c_void_p]
        L.dash_attn_fwd_decode_paged.restype = ctypes.c_int
        L.dash_attn_fwd_decode_paged.argtypes = [P, c_void_p, c_void_p, c_void_p, c_void_p, c_int32, c_int32, c_int32,
                                                 c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
        G, R = POINTER(DashPagedParams), POINTER(DashRope)
        L.dash_attn_rope.restype = ctypes.c_int
        L.dash_attn_rope.argtypes = [P, R] + [c_void_p] * 5 + [c_int32, c_void_p]
        L.dash_attn_append_paged.restype = ctypes.c_int
        L.dash_attn_append_paged.argtypes = [G, R] + [c_void_p] * 11
        L.dash_attn_paged_workspace_bytes.restype = c_size_t
        L.dash_attn_paged_workspace_bytes.argtypes = [G]
        L.dash_attn_attend_chunk_paged.restype = ctypes.c_int
        L.dash_attn_attend_chunk_paged.argtypes = [G] + [c_void_p] * 9 + [c_size_t, c_void_p]
        L.dash_attn_key_mass_paged.restype = ctypes.c_int
        L.dash_attn_key_mass_paged.argtypes = [G] + [c_void_p] * 6 + [c_float] + [c_void_p] * 3 + [c_size_t, c_void_p]
        L.dash_attn_evict_paged.restype = ctypes.c_int
        L.dash_attn_evict_paged.argtypes = [G, c_int32, c_int32, c_int32] + [c_void_p] * 8 + [c_int32, c_int32] + [c_void_p] * 4
        L.dash_attn_reset_status.restype = ctypes.c_int
        L.dash_attn_reset_status.argtypes = [c_void_p, c_void_p]
        L.dash_attn_last_status.restype = ctypes.c_int
        L.dash_attn_last_status.argtypes = [c_void_p, c_void_p]
        L.dash_attn_launch_count.restype = c_int64
        L.dash_attn_launch_count.argtypes = []
        L.dash_attn_test_hooks.restype = None
        L.dash_attn_test_hooks.argtypes = [c_int64, c_int32]
        L.dash_attn_test_hold_loads.restype = None
        L.dash_attn_test_hold_loads.argtypes = [c_int64, c_int32]
        L.dash_attn_strerror.restype = c_char_p
        L.dash_attn_strerror.argtypes = [ctypes.c_int]
        _lib = L
    return _lib


class use_debug_library:
    """Context manager: inside it every binding call goes to libdash_attn_debug.so (built by
    `python -m paper_2605_18753_b200.build --debug`), whose kernels check every index they read from device memory
    and record DASH_ERR_CAPACITY instead of making a bad access.  Raises if that library has not been built."""

    def __enter__(self):
        global _lib, LIB_PATH
        if not os.path.exists(DEBUG_LIB_PATH):
            raise RuntimeError(f"{DEBUG_LIB_PATH} is missing: build it with `python -m paper_2605_18753_b200.build --debug`")
        self._saved = (_lib, LIB_PATH)
        _lib, LIB_PATH = None, DEBUG_LIB_PATH
        lib()
        return self

    def __exit__(self, *exc):
        global _lib, LIB_PATH
        _lib, LIB_PATH = self._saved
        return False


def strerror(code: int) -> str:
    return lib().dash_attn_strerror(int(code)).decode()


# A short decode step is one or two kernels of a few microseconds, so what a call costs here counts: plain integers go to
# ctypes (the declared argument types convert them), and the stream handle is read without building a torch.cuda.Stream
# object (3.4 -> 0.1 us a call; a decode step's issue 14.3 -> 10.3 us).
def _ptr(t):
    return t if t is None or isinstance(t, int) else t.data_ptr()


def _stream():
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _check(rc: int, where: str):
    if rc != DASH_OK:
        raise DashError(rc, where)


def _dtype_code(dt: torch.dtype) -> int:
    if dt == torch.float32:
        return DASH_F32
    if dt == torch.bfloat16:
        return DASH_BF16
    raise ValueError(f"unsupported dtype {dt}")


def _strides3(t: torch.Tensor, decode_q: bool = False):
    """Element strides (batch, token, head) of a [b, n, h, d] tensor, or of a decode query [b, h, d]."""
    if t.stride(-1) != 1:
        raise ValueError("head_dim axis must be contiguous")
    if decode_q:
        return (t.stride(0), 0, t.stride(1))
    return (t.stride(0), t.stride(1), t.stride(2))


def make_params(*, batch, seq_q, seq_kv, h_q, h_kv, head_dim, block, dtype, alpha, gamma=1.0, sigma=10.0,
                causal=1, local_blocks=0, q_stride=None, k_stride=None, v_stride=None, o_stride=None) -> DashParams:
    """Fills a dash_params; strides default to contiguous [b, n, h, d] (decode Q/O: [b, h, d])."""
    p = DashParams()
    p.struct_size = ctypes.sizeof(DashParams)
    p.batch, p.seq_q, p.seq_kv = batch, seq_q, seq_kv
    p.h_q, p.h_kv, p.head_dim, p.block = h_q, h_kv, head_dim, block
    p.dtype = dtype if isinstance(dtype, int) else _dtype_code(dtype)
    p.causal = causal
    p.alpha, p.gamma, p.sigma = alpha, gamma, sigma
    p.local_blocks = local_blocks
    p.q_to_kv = None
    dq = (seq_q * h_q * head_dim, h_q * head_dim, head_dim) if seq_q == seq_kv else (h_q * head_dim, 0, head_dim)
    dk = (seq_kv * h_kv * head_dim, h_kv * head_dim, head_dim)
    for name, val, dflt in (("q_stride", q_stride, dq), ("k_stride", k_stride, dk), ("v_stride", v_stride, dk),
                            ("o_stride", o_stride, dq)):
        setattr(p, name, (c_int64 * 3)(*(val if val is not None else dflt)))
    return p


def params_for_prefill(Q, K, V, O, *, block, alpha, gamma=1.0, sigma=10.0, local_blocks=0, causal=1) -> DashParams:
    b, n, h_q, d = Q.shape
    return make_params(batch=b, seq_q=n, seq_kv=K.shape[1], h_q=h_q, h_kv=K.shape[2], head_dim=d, block=block,
                       dtype=Q.dtype, alpha=alpha, gamma=gamma, sigma=sigma, local_blocks=local_blocks, causal=causal,
                       q_stride=_strides3(Q),
                       k_stride=_strides3(K), v_stride=_strides3(V), o_stride=_strides3(O))


def params_for_decode(Q, Kc, Vc, O, *, block, alpha, gamma=1.0, sigma=10.0, local_blocks=0) -> DashParams:
    b, h_q, d = Q.shape
    return make_params(batch=b, seq_q=1, seq_kv=Kc.shape[1], h_q=h_q, h_kv=Kc.shape[2], head_dim=d, block=block,
                       dtype=Q.dtype, alpha=alpha, gamma=gamma, sigma=sigma, local_blocks=local_blocks,
                       q_stride=_strides3(Q, True),
                       k_stride=_strides3(Kc), v_stride=_strides3(Vc), o_stride=_strides3(O, True))


# ---------------------------------------------------------------- sizes and buffers

def dash_attn_workspace_bytes(p: DashParams) -> int:
    return int(lib().dash_attn_workspace_bytes(ctypes.byref(p)))


def dash_attn_list_capacity(p: DashParams) -> int:
    return int(lib().dash_attn_list_capacity(ctypes.byref(p)))


def dash_attn_list_offset(p: DashParams, b: int, kv_head: int, row: int) -> int:
    return int(lib().dash_attn_list_offset(ctypes.byref(p), b, kv_head, row))


def alloc_workspace(p: DashParams, device="cuda") -> torch.Tensor:
    nbytes = dash_attn_workspace_bytes(p)
    if nbytes == 0:
        raise DashError(-1, "dash_attn_workspace_bytes")
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    assert ws.data_ptr() % 256 == 0
    dash_attn_reset_status(ws)
    return ws


def alloc_routing(p: DashParams, device="cuda", with_tau=False) -> dict:
    """Buffers for dash_attn_select's outputs."""
    T_a = (p.seq_kv + p.block - 1) // p.block
    W = (T_a + 31) // 32
    T_s = p.seq_kv // p.block
    cap = max(dash_attn_list_capacity(p), 1)
    out = {
        "mask": torch.empty(p.batch, p.h_kv, p.seq_q, W, dtype=torch.int32, device=device),
        "count": torch.empty(p.batch, p.h_kv, p.seq_q, dtype=torch.int32, device=device),
        "blk_idx": torch.empty(cap, dtype=torch.int32, device=device),
        "blk_bias": torch.empty(cap, dtype=torch.float32, device=device),
        "tau": torch.empty(p.batch, p.h_q, p.seq_q, dtype=torch.float32, device=device) if with_tau else None,
    }
    return out


def alloc_kbar(p: DashParams, device="cuda") -> torch.Tensor:
    return torch.empty(p.batch, p.h_kv, max(p.seq_kv // p.block, 0), p.head_dim, dtype=torch.float32, device=device)


# ---------------------------------------------------------------- entry points

def dash_attn_block_summaries(p, K, Kbar, qbar=None, qbar_chunk_stride=0, kv_len=None, first_block=0, num_blocks=-1):
    _check(lib().dash_attn_block_summaries(ctypes.byref(p), _ptr(K), _ptr(qbar), qbar_chunk_stride, _ptr(kv_len),
                                           first_block, num_blocks, _ptr(Kbar), _stream()), "dash_attn_block_summaries")


def dash_attn_select(p, Q, Kbar, mask, count, blk_idx, blk_bias, workspace, tau=None, kv_len=None):
    _check(lib().dash_attn_select(ctypes.byref(p), _ptr(Q), _ptr(Kbar), _ptr(kv_len), _ptr(mask), _ptr(count),
                                  _ptr(blk_idx), _ptr(blk_bias), _ptr(tau), _ptr(workspace), workspace.numel(),
                                  _stream()), "dash_attn_select")


def dash_attn_attend_prefill(p, Q, K, V, mask, blk_bias, O, workspace):
    _check(lib().dash_attn_attend_prefill(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(mask), _ptr(blk_bias),
                                          _ptr(O), _ptr(workspace), workspace.numel(), _stream()),
           "dash_attn_attend_prefill")


def dash_attn_attend_decode(p, Q, Kc, Vc, kv_len, count, blk_idx, blk_bias, O, workspace):
    _check(lib().dash_attn_attend_decode(ctypes.byref(p), _ptr(Q), _ptr(Kc), _ptr(Vc), _ptr(kv_len), _ptr(count),
                                         _ptr(blk_idx), _ptr(blk_bias), _ptr(O), _ptr(workspace), workspace.numel(),
                                         _stream()), "dash_attn_attend_decode")


def dash_attn_attend_decode_static(p, Q, Kc, Vc, kv_len, count, blk_idx, blk_bias, O):
    """Split-KV decode attention for callers that cannot allocate device memory: no workspace argument, the
    split partials use a fixed 4 MiB array inside the library.  Calls must not overlap on the GPU."""
    _check(lib().dash_attn_attend_decode_static(ctypes.byref(p), _ptr(Q), _ptr(Kc), _ptr(Vc), _ptr(kv_len),
                                                _ptr(count), _ptr(blk_idx), _ptr(blk_bias), _ptr(O), _stream()),
           "dash_attn_attend_decode_static")


def dash_attn_bwd_attend_prefill(p, Q, K, V, dO, mask, blk_bias, dQ, dK, dV, dbias):
    """Backward of Stage 2 (prefill) with the routing held fixed; dK / dV fp32 [b, n, h_kv, d], dbias like blk_bias."""
    _check(lib().dash_attn_bwd_attend_prefill(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(dO), _ptr(mask),
                                              _ptr(blk_bias), _ptr(dQ), _ptr(dK), _ptr(dV), _ptr(dbias), _stream()),
           "dash_attn_bwd_attend_prefill")


def alloc_bwd_workspace(p: DashParams, device="cuda") -> torch.Tensor:
    nbytes = int(lib().dash_attn_bwd_workspace_bytes(ctypes.byref(p)))
    if nbytes == 0:
        raise DashError(-1, "dash_attn_bwd_workspace_bytes")
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    assert ws.data_ptr() % 256 == 0
    dash_attn_reset_status(ws)
    return ws


def dash_attn_bwd_attend_prefill_tc(p, Q, K, V, dO, mask, blk_bias, dQ, dK, dV, dbias, bwd_workspace):
    """The same gradients from the tensor-core kernels (bf16, head_dim 128, chunks of 64 / 128); raises DashError with
    DASH_ERR_UNSUPPORTED for other shapes."""
    _check(lib().dash_attn_bwd_attend_prefill_tc(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(dO), _ptr(mask),
                                                 _ptr(blk_bias), _ptr(dQ), _ptr(dK), _ptr(dV), _ptr(dbias),
                                                 _ptr(bwd_workspace), bwd_workspace.numel(), _stream()),
           "dash_attn_bwd_attend_prefill_tc")


def dash_attn_bwd_select_prefill(p, Q, Kbar, count, blk_idx, tau, dbias, dQ_route, dKbar):
    """Backward of Stage 1 (prefill): dbias -> dQ_route (fp32 [b, n, h_q, d]) and dKbar (fp32 like Kbar)."""
    _check(lib().dash_attn_bwd_select_prefill(ctypes.byref(p), _ptr(Q), _ptr(Kbar), _ptr(count), _ptr(blk_idx), _ptr(tau),
                                              _ptr(dbias), _ptr(dQ_route), _ptr(dKbar), _stream()),
           "dash_attn_bwd_select_prefill")


def dash_attn_bwd_block_summaries(p, K, dKbar, dK, qbar=None, qbar_chunk_stride=0, dqbar=None):
    """Backward of Stage 0: adds the summaries' share to dK (fp32 [b, n, h_kv, d]); dqbar gets the summary query's gradient."""
    _check(lib().dash_attn_bwd_block_summaries(ctypes.byref(p), _ptr(K), _ptr(qbar), qbar_chunk_stride, _ptr(dKbar),
                                               _ptr(dK), _ptr(dqbar), _stream()), "dash_attn_bwd_block_summaries")


def dash_attn_fwd_prefill(p, Q, K, V, O, workspace, qbar=None, qbar_chunk_stride=0, Kbar=None, mask_out=None):
    _check(lib().dash_attn_fwd_prefill(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(qbar), qbar_chunk_stride,
                                       _ptr(Kbar), _ptr(O), _ptr(mask_out), _ptr(workspace), workspace.numel(),
                                       _stream()), "dash_attn_fwd_prefill")


def dash_attn_fwd_decode(p, Q, Kc, Vc, Kbar, kv_len, O, workspace):
    _check(lib().dash_attn_fwd_decode(ctypes.byref(p), _ptr(Q), _ptr(Kc), _ptr(Vc), _ptr(Kbar), _ptr(kv_len),
                                      _ptr(O), _ptr(workspace), workspace.numel(), _stream()), "dash_attn_fwd_decode")


def params_for_paged_decode(Q, Kpool, Vpool, O, *, max_pages, block, alpha, gamma=1.0, sigma=10.0, local_blocks=0):
    """Decode parameters over pools [num_pages, page_size, h_kv, d]: seq_kv is the logical capacity max_pages * page_size
    and the K / V strides are those of (page, token in page, head)."""
    b, h_q, d = Q.shape
    return make_params(batch=b, seq_q=1, seq_kv=max_pages * Kpool.shape[1], h_q=h_q, h_kv=Kpool.shape[2], head_dim=d,
                       block=block, dtype=Q.dtype, alpha=alpha, gamma=gamma, sigma=sigma, local_blocks=local_blocks,
                       q_stride=_strides3(Q, True), k_stride=_strides3(Kpool), v_stride=_strides3(Vpool),
                       o_stride=_strides3(O, True))


def dash_attn_block_summaries_paged(p, Kpool, page_table, Kbar, qbar=None, qbar_chunk_stride=0, kv_len=None,
                                    first_block=0, num_blocks=-1):
    _check(lib().dash_attn_block_summaries_paged(ctypes.byref(p), _ptr(Kpool), _ptr(page_table), Kpool.shape[1],
                                                 page_table.shape[1], Kpool.shape[0], _ptr(qbar), qbar_chunk_stride,
                                                 _ptr(kv_len), first_block, num_blocks, _ptr(Kbar), _stream()),
           "dash_attn_block_summaries_paged")


def dash_attn_fwd_decode_paged(p, Q, Kpool, Vpool, page_table, Kbar, kv_len, O, workspace):
    _check(lib().dash_attn_fwd_decode_paged(ctypes.byref(p), _ptr(Q), _ptr(Kpool), _ptr(Vpool), _ptr(page_table),
                                            Kpool.shape[1], page_table.shape[1], Kpool.shape[0], _ptr(Kbar), _ptr(kv_len),
                                            _ptr(O), _ptr(workspace), workspace.numel(), _stream()),
           "dash_attn_fwd_decode_paged")


# ---------------------------------------------------------------- operators around the paged cache

def make_rope(inv_freq, axis=None, interleaved=False) -> DashRope:
    """Rotary positions: pair i turns by positions[axis[i]] * inv_freq[i] radians (axis None: one axis for all pairs)."""
    pairs = len(inv_freq)
    axis = [0] * pairs if axis is None else [int(x) for x in axis]
    if len(axis) != pairs:
        raise ValueError("axis and inv_freq must have an entry per pair")
    r = DashRope()
    r.struct_size = ctypes.sizeof(DashRope)
    r.pairs, r.axes, r.interleaved = pairs, max(axis, default=0) + 1, int(bool(interleaved))
    r.axis = (c_int32 * pairs)(*axis)                                   # (the structure keeps the arrays alive)
    r.inv_freq = (ctypes.c_double * pairs)(*[float(f) for f in inv_freq])
    return r


def params_for_paged(Kpool, Vpool, page_table, *, h_q, rows=None, Q=None, O=None, K=None, V=None) -> DashPagedParams:
    """Parameters over pools [num_pages, page_size, h_kv, d] and packed rows Q / O [rows, h_q, d], K / V [rows, h_kv, d].
    Tensors that are absent count as contiguous; Vpool None stands for the strides of Kpool."""
    num_pages, page_size, h_kv, d = Kpool.shape
    packed = [t for t in (Q, O, K, V) if t is not None]
    if rows is None:
        rows = packed[0].shape[0] if packed else 0
    for t, h in ((Q, h_q), (O, h_q), (K, h_kv), (V, h_kv)):
        if t is not None and (tuple(t.shape) != (rows, h, d) or t.dtype != Kpool.dtype or t.stride(-1) != 1):
            raise ValueError(f"packed tensors are [rows, heads, head_dim] of the pools' dtype with a contiguous head_dim; got {tuple(t.shape)} {t.dtype}")
    if Vpool is not None and (Vpool.shape != Kpool.shape or Vpool.dtype != Kpool.dtype):
        raise ValueError("Kpool and Vpool must agree in shape and dtype")
    p = DashPagedParams()
    p.struct_size = ctypes.sizeof(DashPagedParams)
    p.batch, p.rows, p.h_q, p.h_kv, p.head_dim = page_table.shape[0], rows, h_q, h_kv, d
    p.dtype = _dtype_code(Kpool.dtype)
    p.page_size, p.max_pages, p.num_pages = page_size, page_table.shape[1], num_pages
    for name, t, h in (("q_stride", Q, h_q), ("o_stride", O, h_q), ("kn_stride", K, h_kv), ("vn_stride", V, h_kv)):
        setattr(p, name, (c_int64 * 2)(*((t.stride(0), t.stride(1)) if t is not None else (h * d, d))))
    p.k_stride = (c_int64 * 3)(*_strides3(Kpool))
    p.v_stride = (c_int64 * 3)(*_strides3(Kpool if Vpool is None else Vpool))
    return p


_I32, _F32 = torch.int32, torch.float32
_TORCH_DTYPE = (torch.float32, torch.bfloat16)        # by dash_dtype


class _Layout:
    """Sizes, shapes and strides that the parameters say, worked out once per set of values (the parameters keep them beside a copy of
    the values they come from, so a change shows)."""
    __slots__ = ("raw", "dtype", "batch", "rows", "entries", "sums", "groups", "slots", "q", "o", "kn", "vn", "k", "v")

    def __init__(self, p, raw):
        self.raw, self.dtype, d = raw, _TORCH_DTYPE[p.dtype], p.head_dim
        if isinstance(p, DashPagedParams):
            self.batch, self.rows, self.entries, self.sums = p.batch, p.rows, p.batch * p.max_pages, p.rows * p.h_q
            self.groups, self.slots = p.batch * p.h_kv, p.batch * p.h_kv * p.max_pages * p.page_size
            self.q, self.o = (((p.rows, p.h_q, d), (*s, 1)) for s in (p.q_stride, p.o_stride))
            self.kn, self.vn = (((p.rows, p.h_kv, d), (*s, 1)) for s in (p.kn_stride, p.vn_stride))
            self.k, self.v = (((p.num_pages, p.page_size, p.h_kv, d), (*s, 1)) for s in (p.k_stride, p.v_stride))
        else:
            self.q, self.k = (((p.batch, p.seq_q, h, d), (*s, 1)) for h, s in ((p.h_q, p.q_stride), (p.h_kv, p.k_stride)))


def _layout(p):
    raw, got = bytes(p), p.__dict__.get("_layout")
    if got is None or got.raw != raw:
        got = p._layout = _Layout(p, raw)
    return got


def _misfits(where, **pairs):
    """Raises for the tensors that do not have the parameters' shape and strides (the stride of a dimension of one element says
    nothing, and an empty tensor's none)."""
    for name, (t, (shape, stride)) in pairs.items():
        if t is None:
            continue
        if t.shape != shape or t.numel() > 0 and any(n > 1 and a != b for n, a, b in zip(shape, t.stride(), stride)):
            raise ValueError(f"{where}: {name} has shape {tuple(t.shape)} with strides {t.stride()}, the parameters say {shape} with strides {stride}")


def _refuse(where, dtype, ints, floats, tensors, workspace=None):
    """Says which argument the kernels would misread: they take index tensors as contiguous int32, lse and mass as contiguous fp32,
    queries, keys and values in the parameters' dtype, all on the current device, as is the workspace."""
    if workspace is not None and not (workspace.get_device() == torch._C._cuda_getDevice() and workspace.is_contiguous()):
        raise ValueError(f"{where}: expected a contiguous workspace on the current device, got one on {workspace.device} with strides {workspace.stride()}")
    for kind, want, ts in (("int32", _I32, ints), ("float32", _F32, floats), ("", dtype, tensors)):
        for t in ts:
            if t is None:
                continue
            if t.dtype is not want or (kind and not t.is_contiguous()) or t.get_device() != torch._C._cuda_getDevice():
                raise ValueError(f"{where}: expected a {'contiguous ' if kind else ''}{want} tensor on the current device, got {t.dtype} "
                                 f"{tuple(t.shape)} with strides {t.stride()} on {t.device}")


def _sizes(where, **pairs):
    bad = [f"{name} {got}, not {want}" for name, (got, want) in pairs.items() if got != want]
    raise ValueError(f"{where}: sizes that do not fit the parameters: " + ", ".join(bad))


# A short call is a kernel of a few microseconds, so what these checks cost counts: one expression on the way that is taken, the search
# for the culprit only behind it.

def dash_attn_rope(p, rope, positions, Q, K, Qout, Kout, inverse=False):
    """Q and K (either may be None) of a prefill shape rotated; inverse=True turns them back, which is the backward pass when it is
    given the gradients.  positions int32 [axes, batch, seq]; inputs and outputs have the parameters' strides, and an output may be its input."""
    dev, lay = torch._C._cuda_getDevice(), _layout(p)
    dt = lay.dtype
    if not (positions.dtype is _I32 and positions.get_device() == dev and positions.is_contiguous()):
        _refuse("dash_attn_rope", dt, (positions,), (), ())
    for x, y, (shape, stride) in ((Q, Qout, lay.q), (K, Kout, lay.k)):
        if x is None and y is None:
            continue
        if x is None or y is None:
            raise ValueError("dash_attn_rope: every input has an output")
        if not (x.dtype is dt and y.dtype is dt and x.get_device() == dev and y.get_device() == dev):
            _refuse("dash_attn_rope", dt, (), (), (x, y))
        if not (x.shape == shape and x.stride() == stride and (x is y or y.shape == shape and y.stride() == stride)):
            _misfits("dash_attn_rope", input=(x, (shape, stride)), output=(y, (shape, stride)))
    if positions.numel() != rope.axes * p.batch * p.seq_q:
        raise ValueError("positions must be [axes, batch, seq]")
    rc = (_lib or lib()).dash_attn_rope(ctypes.byref(p), ctypes.byref(rope), positions.data_ptr(), Q if Q is None else Q.data_ptr(),
                                        K if K is None else K.data_ptr(), Q if Q is None else Qout.data_ptr(),
                                        K if K is None else Kout.data_ptr(), 1 if inverse else 0, torch._C._cuda_getCurrentRawStream(dev))
    if rc:
        raise DashError(rc, "dash_attn_rope")


def dash_attn_append_paged(p, rope, positions, q_start, kv_len, page_table, Q, Qout, K, V, Kpool, Vpool):
    """Packed new tokens into their pages: K rotated, V as it is, Q rotated into Qout (Q and Qout None: keys and values only;
    rope and positions None: no rotation)."""
    dev, lay = torch._C._cuda_getDevice(), _layout(p)
    dt = lay.dtype
    if not (q_start.dtype is _I32 and kv_len.dtype is _I32 and page_table.dtype is _I32 and K.dtype is dt and V.dtype is dt
            and Kpool.dtype is dt and Vpool.dtype is dt and q_start.get_device() == dev and kv_len.get_device() == dev
            and page_table.get_device() == dev and K.get_device() == dev and V.get_device() == dev and Kpool.get_device() == dev
            and Vpool.get_device() == dev and q_start.is_contiguous() and kv_len.is_contiguous() and page_table.is_contiguous()
            and (positions is None or (positions.dtype is _I32 and positions.get_device() == dev and positions.is_contiguous()))
            and (Q is None or (Q.dtype is dt and Q.get_device() == dev)) and (Qout is None or (Qout.dtype is dt and Qout.get_device() == dev))):
        _refuse("dash_attn_append_paged", dt, (positions, q_start, kv_len, page_table), (), (Q, Qout, K, V, Kpool, Vpool))
    n, rows = lay.batch, lay.rows
    if not (q_start.numel() == n + 1 and kv_len.numel() == n and page_table.numel() == lay.entries):
        _sizes("dash_attn_append_paged", q_start=(q_start.numel(), n + 1), kv_len=(kv_len.numel(), n),
               page_table=(page_table.numel(), lay.entries))
    if not (K.shape == lay.kn[0] and K.stride() == lay.kn[1] and V.shape == lay.vn[0] and V.stride() == lay.vn[1]
            and Kpool.shape == lay.k[0] and Kpool.stride() == lay.k[1] and Vpool.shape == lay.v[0] and Vpool.stride() == lay.v[1]
            and (Q is None or (Q.shape == lay.q[0] and Q.stride() == lay.q[1]))
            and (Qout is None or (Qout.shape == lay.o[0] and Qout.stride() == lay.o[1]))):
        _misfits("dash_attn_append_paged", Q=(Q, lay.q), Qout=(Qout, lay.o), K=(K, lay.kn), V=(V, lay.vn), Kpool=(Kpool, lay.k), Vpool=(Vpool, lay.v))
    if (rope is None) != (positions is None):
        raise ValueError("dash_attn_append_paged: rope and positions come together")
    if positions is not None and positions.numel() != rope.axes * rows:
        raise ValueError("positions must be [axes, rows]")
    rc = (_lib or lib()).dash_attn_append_paged(
        ctypes.byref(p), None if rope is None else ctypes.byref(rope), None if positions is None else positions.data_ptr(),
        q_start.data_ptr(), kv_len.data_ptr(), page_table.data_ptr(), None if Q is None else Q.data_ptr(),
        None if Qout is None else Qout.data_ptr(), K.data_ptr(), V.data_ptr(), Kpool.data_ptr(), Vpool.data_ptr(),
        torch._C._cuda_getCurrentRawStream(dev))
    if rc:
        raise DashError(rc, "dash_attn_append_paged")


def dash_attn_paged_workspace_bytes(p: DashPagedParams) -> int:
    return int(lib().dash_attn_paged_workspace_bytes(ctypes.byref(p)))


def alloc_paged_workspace(p: DashPagedParams, device="cuda") -> torch.Tensor:
    nbytes = dash_attn_paged_workspace_bytes(p)
    if nbytes == 0:
        raise DashError(-1, "dash_attn_paged_workspace_bytes")
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    assert ws.data_ptr() % 256 == 0
    dash_attn_reset_status(ws)
    return ws


def dash_attn_attend_chunk_paged(p, Q, Kpool, Vpool, page_table, q_start, kv_len, O, lse, workspace):
    """Dense causal attention of packed new tokens over their sequences' pages; lse (None to skip) fp32 [rows, h_q]."""
    dev, lay = torch._C._cuda_getDevice(), _layout(p)
    dt = lay.dtype
    if not (q_start.dtype is _I32 and kv_len.dtype is _I32 and page_table.dtype is _I32 and Q.dtype is dt and O.dtype is dt
            and Kpool.dtype is dt and Vpool.dtype is dt and q_start.get_device() == dev and kv_len.get_device() == dev
            and page_table.get_device() == dev and Q.get_device() == dev and O.get_device() == dev and Kpool.get_device() == dev
            and Vpool.get_device() == dev and q_start.is_contiguous() and kv_len.is_contiguous() and page_table.is_contiguous()
            and workspace.get_device() == dev and workspace.is_contiguous()
            and (lse is None or (lse.dtype is _F32 and lse.get_device() == dev and lse.is_contiguous()))):
        _refuse("dash_attn_attend_chunk_paged", dt, (page_table, q_start, kv_len), (lse,), (Q, Kpool, Vpool, O), workspace)
    n = lay.batch
    if not (q_start.numel() == n + 1 and kv_len.numel() == n and page_table.numel() == lay.entries
            and (lse is None or lse.numel() == lay.sums)):
        _sizes("dash_attn_attend_chunk_paged", q_start=(q_start.numel(), n + 1), kv_len=(kv_len.numel(), n),
               page_table=(page_table.numel(), lay.entries), lse=(lay.sums if lse is None else lse.numel(), lay.sums))
    if not (Q.shape == lay.q[0] and Q.stride() == lay.q[1] and O.shape == lay.o[0] and O.stride() == lay.o[1]
            and Kpool.shape == lay.k[0] and Kpool.stride() == lay.k[1] and Vpool.shape == lay.v[0] and Vpool.stride() == lay.v[1]):
        _misfits("dash_attn_attend_chunk_paged", Q=(Q, lay.q), O=(O, lay.o), Kpool=(Kpool, lay.k), Vpool=(Vpool, lay.v))
    rc = (_lib or lib()).dash_attn_attend_chunk_paged(
        ctypes.byref(p), Q.data_ptr(), Kpool.data_ptr(), Vpool.data_ptr(), page_table.data_ptr(), q_start.data_ptr(), kv_len.data_ptr(),
        O.data_ptr(), None if lse is None else lse.data_ptr(), workspace.data_ptr(), workspace.numel(),
        torch._C._cuda_getCurrentRawStream(dev))
    if rc:
        raise DashError(rc, "dash_attn_attend_chunk_paged")


def dash_attn_key_mass_paged(p, Q, Kpool, page_table, q_start, kv_len, lse, mass_in, mass_out, workspace, decay=1.0):
    """Weights that the new rows give every cached token, added to decay * mass_in (None: zeros); fp32 [batch, h_kv, slots]."""
    dev, lay = torch._C._cuda_getDevice(), _layout(p)
    dt = lay.dtype
    if not (q_start.dtype is _I32 and kv_len.dtype is _I32 and page_table.dtype is _I32 and Q.dtype is dt and Kpool.dtype is dt
            and lse.dtype is _F32 and mass_out.dtype is _F32 and q_start.get_device() == dev and kv_len.get_device() == dev
            and page_table.get_device() == dev and Q.get_device() == dev and Kpool.get_device() == dev and lse.get_device() == dev
            and mass_out.get_device() == dev and q_start.is_contiguous() and kv_len.is_contiguous() and page_table.is_contiguous()
            and lse.is_contiguous() and mass_out.is_contiguous() and workspace.get_device() == dev and workspace.is_contiguous()
            and (mass_in is None or (mass_in.dtype is _F32 and mass_in.get_device() == dev and mass_in.is_contiguous()))):
        _refuse("dash_attn_key_mass_paged", dt, (page_table, q_start, kv_len), (lse, mass_in, mass_out), (Q, Kpool), workspace)
    n, slots = lay.batch, lay.slots
    if not (q_start.numel() == n + 1 and kv_len.numel() == n and page_table.numel() == lay.entries and lse.numel() == lay.sums
            and mass_out.numel() == slots and (mass_in is None or mass_in.numel() == slots)):
        _sizes("dash_attn_key_mass_paged", q_start=(q_start.numel(), n + 1), kv_len=(kv_len.numel(), n),
               page_table=(page_table.numel(), lay.entries), lse=(lse.numel(), lay.sums),
               mass_in=(slots if mass_in is None else mass_in.numel(), slots), mass_out=(mass_out.numel(), slots))
    if not (Q.shape == lay.q[0] and Q.stride() == lay.q[1] and Kpool.shape == lay.k[0] and Kpool.stride() == lay.k[1]):
        _misfits("dash_attn_key_mass_paged", Q=(Q, lay.q), Kpool=(Kpool, lay.k))
    rc = (_lib or lib()).dash_attn_key_mass_paged(
        ctypes.byref(p), Q.data_ptr(), Kpool.data_ptr(), page_table.data_ptr(), q_start.data_ptr(), kv_len.data_ptr(), lse.data_ptr(),
        decay, None if mass_in is None else mass_in.data_ptr(), mass_out.data_ptr(), workspace.data_ptr(), workspace.numel(),
        torch._C._cuda_getCurrentRawStream(dev))
    if rc:
        raise DashError(rc, "dash_attn_key_mass_paged")


def dash_attn_evict_paged(p, mass, kv_len, page_table, Kpool, Vpool, kept, new_len, dst_table, Kdst, Vdst, mass_out=None, *, keep,
                          sinks=0, recent=0):
    """Keeps `keep` tokens of every (sequence, KV head) and moves them to the front of the destination pages (page_table, Kpool,
    Vpool themselves for in place)."""
    dev, lay = torch._C._cuda_getDevice(), _layout(p)
    dt = lay.dtype
    if not (kv_len.dtype is _I32 and page_table.dtype is _I32 and kept.dtype is _I32 and new_len.dtype is _I32 and dst_table.dtype is _I32
            and mass.dtype is _F32 and Kpool.dtype is dt and Vpool.dtype is dt and Kdst.dtype is dt and Vdst.dtype is dt
            and kv_len.get_device() == dev and page_table.get_device() == dev and kept.get_device() == dev and new_len.get_device() == dev
            and dst_table.get_device() == dev and mass.get_device() == dev and Kpool.get_device() == dev and Vpool.get_device() == dev
            and Kdst.get_device() == dev and Vdst.get_device() == dev and kv_len.is_contiguous() and page_table.is_contiguous()
            and kept.is_contiguous() and new_len.is_contiguous() and dst_table.is_contiguous() and mass.is_contiguous()
            and (mass_out is None or (mass_out.dtype is _F32 and mass_out.get_device() == dev and mass_out.is_contiguous()))):
        _refuse("dash_attn_evict_paged", dt, (kv_len, page_table, kept, new_len, dst_table), (mass, mass_out), (Kpool, Vpool, Kdst, Vdst))
    n, groups, shape, page = lay.batch, lay.groups, Kdst.shape, lay.k[0][1]
    width = dst_table.size(-1)
    if not (kv_len.numel() == n and new_len.numel() == n and page_table.numel() == lay.entries and dst_table.numel() == n * width
            and kept.numel() == groups * keep and mass.numel() == lay.slots
            and (mass_out is None or mass_out.numel() == groups * width * page) and Vdst.shape == shape):
        out = groups * width * page
        _sizes("dash_attn_evict_paged", kv_len=(kv_len.numel(), n), new_len=(new_len.numel(), n),
               page_table=(page_table.numel(), lay.entries), dst_table=(dst_table.numel(), n * width), kept=(kept.numel(), groups * keep),
               mass=(mass.numel(), lay.slots), mass_out=(out if mass_out is None else mass_out.numel(), out), Vdst=(tuple(Vdst.shape), tuple(shape)))
    if not (Kpool.shape == lay.k[0] and Kpool.stride() == lay.k[1] and Vpool.shape == lay.v[0] and Vpool.stride() == lay.v[1]
            and shape[1:] == lay.k[0][1:] and Kdst.stride() == lay.k[1] and Vdst.stride() == lay.v[1]):
        to = (shape[0], *lay.k[0][1:])         # the destination's pages: as many as there are, of the pools' size, heads and strides
        _misfits("dash_attn_evict_paged", Kpool=(Kpool, lay.k), Vpool=(Vpool, lay.v), Kdst=(Kdst, (to, lay.k[1])), Vdst=(Vdst, (to, lay.v[1])))
    if not (0 <= sinks <= keep and 0 <= recent <= keep):         # (beyond 32 bits they would arrive as something else)
        raise ValueError(f"dash_attn_evict_paged: sinks {sinks} and recent {recent} are parts of keep {keep}")
    rc = (_lib or lib()).dash_attn_evict_paged(
        ctypes.byref(p), keep, sinks, recent, mass.data_ptr(), kv_len.data_ptr(), page_table.data_ptr(), Kpool.data_ptr(), Vpool.data_ptr(),
        kept.data_ptr(), new_len.data_ptr(), dst_table.data_ptr(), width, shape[0], Kdst.data_ptr(), Vdst.data_ptr(),
        None if mass_out is None else mass_out.data_ptr(), torch._C._cuda_getCurrentRawStream(dev))
    if rc:
        raise DashError(rc, "dash_attn_evict_paged")


def dash_attn_reset_status(workspace):
    _check(lib().dash_attn_reset_status(_ptr(workspace), _stream()), "dash_attn_reset_status")


def dash_attn_last_status(workspace) -> int:
    return int(lib().dash_attn_last_status(_ptr(workspace), _stream()))


def dash_attn_test_hooks(wait_limit_cycles: int = 0, skip_own_k_load: int = 0) -> None:
    """Test-suite switches (see the header); calling it without arguments restores the defaults."""
    lib().dash_attn_test_hooks(int(wait_limit_cycles), int(skip_own_k_load))


def dash_attn_test_hold_loads(cycles: int = 0, odd: bool = False) -> None:
    """Test-suite switch (see the header); calling it without arguments restores the default."""
    lib().dash_attn_test_hold_loads(int(cycles), int(bool(odd)))


def dash_attn_launch_count() -> int:
    return int(lib().dash_attn_launch_count())
