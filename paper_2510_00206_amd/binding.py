"""ctypes binding of the C ABI in include/lorafusion.h: argument marshalling only.

Every function takes torch tensors that already live on the GPU (torch is used for device
memory and the stream handle, nothing else), passes raw pointers to the library and returns
the output tensors.  There is no fallback: if the library is not built, import of the symbols
fails loudly.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblorafusion_hip.so")

EXPORTS = ("lora_fwd", "lora_bwd", "lora_bwd_noalloc", "multi_lora_fwd", "multi_lora_bwd", "multi_lora_fwd_ranked",
           "multi_lora_bwd_ranked", "lora_bwd_workspace_bytes",
           "lora_debug_mask", "lora_status_string", "lora_version", "lora_set_row_tile", "lora_set_slab_lookahead", "lora_debug_stream_panels",
           "lora_debug_da_panels", "lora_debug_bwd_plan", "lora_debug_gemm_tiles", "lora_debug_launches",
           "lora_unfused_fwd", "lora_unfused_bwd", "lora_unfused_workspace_bytes",
           "lora_requests_fwd", "lora_qk_norm_rope_fwd", "lora_qk_norm_rope_bwd", "lora_qk_norm_rope_workspace_bytes",
           "lora_kv_cache_write", "lora_kv_cache_read", "lora_paged_attn_fwd", "lora_paged_attn_workspace_bytes",
           "lora_weights_write", "lora_weights_read", "lora_requests_quantised_fwd", "lora_debug_quantised_tiles", "lora_kv_cache_append")

_lib = None


class BwdPlan(C.Structure):
    """What a backward call launches (lora_bwd_plan in the header)."""
    _fields_ = [("ds_alone", C.c_int32), ("panel_rows_db", C.c_int32), ("panel_rows_da", C.c_int32), ("added_in_strips", C.c_int32),
                ("with_dx", C.c_int32), ("bytes", C.c_int64)]


class GemmLaunch(C.Structure):
    """One kernel of operation (2) or (5) (lora_gemm_launch in the header)."""
    _fields_ = [(f, C.c_int32) for f in ("rows", "columns", "depth", "stages", "waves", "asks_ahead")] + [("workgroups", C.c_int64)]


class Launches(C.Structure):
    """What operations (1), (2) and (5) launch (lora_launches in the header)."""
    _fields_ = [(f, C.c_int32) for f in ("down_rows", "down_parts", "down_ring")] + \
               [("down_workgroups", C.c_int64), ("fwd", GemmLaunch * 2), ("dx", GemmLaunch * 2)]


class QuantisedTiles(C.Structure):
    """What lora_requests_quantised_fwd runs with (lora_quantised_tiles in the header)."""
    _fields_ = [(f, C.c_int32) for f in ("rows", "columns", "ring_blocks", "own_term")]


class CacheArrays(C.Structure):
    """A paged cache (lora_kv_cache in the header)."""
    _fields_ = [(f, C.c_void_p) for f in ("k", "v", "k_exp", "v_exp")] + [("pages", C.c_int64)] + \
               [(f, C.c_int32) for f in ("page", "heads", "dim", "fp8")]


def load_library() -> C.CDLL:
    """Loads the built HIP library; raises if it is missing (build with __graft_entry__.build())."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is not built: run `python -m paper_2510_00206_amd.build`")
    lib = C.CDLL(LIB_PATH)
    P, I64, I32, F, U64, SZ = C.c_void_p, C.c_int64, C.c_int32, C.c_float, C.c_uint64, C.c_size_t
    lib.lora_fwd.argtypes = [P, P, P, P, I64, I64, I64, I32, F, F, U64, P, P, P]
    lib.lora_bwd.argtypes = [P, P, P, P, P, P, I64, I64, I64, I32, F, F, U64, P, P, P, C.c_int, P, SZ, P]
    lib.lora_bwd_noalloc.argtypes = [P, P, P, P, P, P, I64, I64, I64, I32, F, F, U64, P, P, P, C.c_int, P]
    lib.lora_bwd_noalloc.restype = C.c_int
    lib.multi_lora_fwd.argtypes = [P, P, P, P, I64, I64, I64, I32, I32,
                                   C.POINTER(I64), C.POINTER(F), C.POINTER(F), C.POINTER(U64), P, P, P]
    lib.multi_lora_bwd.argtypes = [P, P, P, P, P, P, I64, I64, I64, I32, I32,
                                   C.POINTER(I64), C.POINTER(F), C.POINTER(F), C.POINTER(U64),
                                   P, P, P, C.c_int, P, SZ, P]
    lib.multi_lora_fwd_ranked.argtypes = [P, P, P, P, I64, I64, I64, I32, I32, C.POINTER(I64), C.POINTER(I32),
                                          C.POINTER(F), C.POINTER(F), C.POINTER(U64), P, P, P]
    lib.multi_lora_bwd_ranked.argtypes = [P, P, P, P, P, P, I64, I64, I64, I32, I32, C.POINTER(I64), C.POINTER(I32),
                                          C.POINTER(F), C.POINTER(F), C.POINTER(U64),
                                          P, P, P, C.c_int, P, SZ, P]
    lib.lora_bwd_workspace_bytes.argtypes = [I64, I64, I64, I32, I32]
    lib.lora_bwd_workspace_bytes.restype = SZ
    lib.lora_debug_mask.argtypes = [I64, I64, F, U64, P, P]
    lib.lora_status_string.argtypes = [C.c_int]
    lib.lora_status_string.restype = C.c_char_p
    lib.lora_version.restype = C.c_int
    lib.lora_unfused_workspace_bytes.argtypes = [I64, I64, I64, I32]
    lib.lora_unfused_workspace_bytes.restype = SZ
    lib.lora_unfused_fwd.argtypes = [P, P, P, P, I64, I64, I64, I32, F, F, U64, P, P, SZ, P]
    lib.lora_unfused_bwd.argtypes = [P, P, P, P, I64, I64, I64, I32, F, F, U64, P, P, P, P, SZ, P]
    lib.lora_frozen_fwd.argtypes = [P, P, I64, I64, I64, P, P]
    lib.lora_frozen_bwd.argtypes = [P, P, I64, I64, I64, P, P]
    lib.lora_frozen_fwd.restype = C.c_int
    lib.lora_frozen_bwd.restype = C.c_int
    lib.lora_unfused_fwd.restype = C.c_int
    lib.lora_unfused_bwd.restype = C.c_int
    lib.lora_debug_gemm_tiles.argtypes = [I64, I64, I64, I32, I32, C.POINTER(I64), C.POINTER(I32), C.POINTER(I32),
                                          C.POINTER(I32), C.POINTER(I64)]
    lib.lora_debug_gemm_tiles.restype = C.c_int
    for f in ("lora_debug_stream_panels", "lora_debug_da_panels"):
        getattr(lib, f).argtypes = [I64, I64, I32, C.POINTER(I64), C.POINTER(I32), C.POINTER(I64), C.POINTER(I64)]
        getattr(lib, f).restype = C.c_int
    lib.lora_debug_bwd_plan.argtypes = [I64, I64, I64, I32, I32, C.POINTER(I64), I32, SZ, C.POINTER(BwdPlan)]
    lib.lora_debug_bwd_plan.restype = C.c_int
    lib.lora_debug_launches.argtypes = [I64, I64, I64, I32, I32, C.POINTER(I64), C.POINTER(Launches)]
    lib.lora_debug_launches.restype = C.c_int
    lib.lora_profile_end.argtypes = [C.POINTER(F), C.POINTER(I32)]
    lib.lora_ceiling_mfma.argtypes = [P, P, I32, I32, I32, C.POINTER(C.c_double), P]
    lib.lora_ceiling_mfma.restype = C.c_int
    lib.lora_ceiling_hbm_read.argtypes = [P, SZ, P, I32, P]
    lib.lora_ceiling_hbm_read.restype = C.c_int
    CA = C.POINTER(CacheArrays)
    lib.lora_requests_fwd.argtypes = [P] * 7 + [I64, I64, I64, I32, I64, P, P, P]
    lib.lora_qk_norm_rope_fwd.argtypes = [P] * 7 + [I64, I32, I32, I32, I32, I64, I64, I64, I64, I64, F, C.c_int, P, P, P]
    lib.lora_qk_norm_rope_bwd.argtypes = [P] * 9 + [I64, I32, I32, I32, I32] + [I64] * 7 + [F, C.c_int, P, P, P, P, C.c_int, P, SZ, P]
    lib.lora_qk_norm_rope_workspace_bytes.argtypes = [I64, I32, I32, I32]
    lib.lora_kv_cache_write.argtypes = [CA, P, P, I64, I64, P, I64, P]
    lib.lora_kv_cache_read.argtypes = [CA, P, I64, P, P, I64, I64, P]
    lib.lora_weights_write.argtypes = [P, I64, I64, P, P, P]
    lib.lora_weights_read.argtypes = [P, P, I64, I64, P, P]
    lib.lora_requests_quantised_fwd.argtypes = [P] * 8 + [I64, I64, I64, I32, I64, P, P, P]
    lib.lora_debug_quantised_tiles.argtypes = [I64, I64, I64, I32, I64, C.POINTER(QuantisedTiles)]
    lib.lora_kv_cache_append.argtypes = [CA] + [P] * 9 + [I64, I32, I32, I64, I64, I64, I64, I64, F, C.c_int, P, P]
    lib.lora_paged_attn_fwd.argtypes = [P, CA, P, P, P, I64, I32] + [I64] * 7 + [F, I32, P, P, SZ, P]
    lib.lora_paged_attn_workspace_bytes.argtypes = [CA, I64, I32, I64, I64, I64, I32]
    for f in ("lora_qk_norm_rope_workspace_bytes", "lora_paged_attn_workspace_bytes"):
        getattr(lib, f).restype = SZ
    for f in ("lora_requests_fwd", "lora_qk_norm_rope_fwd", "lora_qk_norm_rope_bwd", "lora_kv_cache_write", "lora_kv_cache_read",
              "lora_paged_attn_fwd", "lora_weights_write", "lora_weights_read", "lora_requests_quantised_fwd", "lora_debug_quantised_tiles",
              "lora_kv_cache_append"):
        getattr(lib, f).restype = C.c_int
    for f in ("lora_fwd", "lora_bwd", "multi_lora_fwd", "multi_lora_bwd", "multi_lora_fwd_ranked",
              "multi_lora_bwd_ranked", "lora_debug_mask",
              "lora_profile_begin", "lora_profile_end"):
        getattr(lib, f).restype = C.c_int
    _lib = lib
    return lib


class LoraError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        super().__init__(f"lorafusion status {status}: {load_library().lora_status_string(status).decode()}")


def _check(status: int):
    if status != 0:
        raise LoraError(status)


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "tensors must be contiguous GPU tensors"
    return t.data_ptr()                # (the argument types make a pointer of it)


def _stream():
    # the raw handle, without a Stream object around it, as the pointers go without an object of their own: a forward and a backward
    # call are marshalled and enqueued in 23 us instead of 30, and the kernels of a small layer (256 x 1024 x 1024) run for 21
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _arr(ctype, vals):
    return (ctype * len(vals))(*vals)


def workspace_bytes(M, K, N, r, G=1) -> int:
    return int(load_library().lora_bwd_workspace_bytes(M, K, N, r, G))


def alloc_workspace(M, K, N, r, G=1, device="cuda") -> torch.Tensor:
    return torch.empty(max(workspace_bytes(M, K, N, r, G), 256), dtype=torch.uint8, device=device)


def lora_fwd(X, W, A, B, s, p, seed, Y=None, S=None):
    """Y [M,N], S_saved [M,r] = forward of one adapter.  X [M,K], W [N,K], A [r,K], B [N,r] bf16."""
    M, K = X.shape
    N, r = B.shape
    Y = torch.empty((M, N), dtype=torch.bfloat16, device=X.device) if Y is None else Y
    S = torch.empty((M, r), dtype=torch.bfloat16, device=X.device) if S is None else S
    _check(load_library().lora_fwd(_ptr(X), _ptr(W), _ptr(A), _ptr(B), M, K, N, r, s, p, seed,
                                   _ptr(Y), _ptr(S), _stream()))
    return Y, S


def lora_bwd(X, W, A, B, S, dY, s, p, seed, need_dx=True, dA=None, dB=None, accumulate=False, workspace=None,
             dX=None):
    """dX [M,K] bf16 (or None), dA [r,K] fp32, dB [N,r] fp32."""
    M, K = X.shape
    N, r = B.shape
    if need_dx and dX is None:
        dX = torch.empty((M, K), dtype=torch.bfloat16, device=X.device)
    dX = dX if need_dx else None
    dA = torch.empty((r, K), dtype=torch.float32, device=X.device) if dA is None else dA
    dB = torch.empty((N, r), dtype=torch.float32, device=X.device) if dB is None else dB
    ws = alloc_workspace(M, K, N, r, 1, X.device) if workspace is None else workspace
    _check(load_library().lora_bwd(_ptr(X), _ptr(W), _ptr(A), _ptr(B), _ptr(S), _ptr(dY), M, K, N, r, s, p, seed,
                                   _ptr(dX), _ptr(dA), _ptr(dB), int(accumulate), _ptr(ws), ws.numel(), _stream()))
    return dX, dA, dB


NOALLOC_SCRATCH_BYTES = 32 << 20


def lora_bwd_noalloc(X, W, A, B, S, dY, s, p, seed, dX, dA, dB, accumulate=False):
    """lora_bwd on the library's built-in scratch: the caller passes every output (dX may be None), nothing
    is allocated here or in the library."""
    M, K = X.shape
    N, r = B.shape
    _check(load_library().lora_bwd_noalloc(_ptr(X), _ptr(W), _ptr(A), _ptr(B), _ptr(S), _ptr(dY), M, K, N, r, s, p, seed,
                                           _ptr(dX), _ptr(dA), _ptr(dB), int(accumulate), _stream()))
    return dX, dA, dB


def multi_lora_fwd(X, W, A, B, seg_offsets: Sequence[int], s, p, seeds, Y=None, S=None, ranks=None):
    """Packed mixed-adapter forward.  A [G,r,K], B [G,N,r]; seg_offsets, s, p, seeds are host lists;
    ranks (optional host list): per-adapter rank <= r, the arrays keep r as the allocated rank."""
    M, K = X.shape
    G, N, r = B.shape
    Y = torch.empty((M, N), dtype=torch.bfloat16, device=X.device) if Y is None else Y
    S = torch.empty((M, r), dtype=torch.bfloat16, device=X.device) if S is None else S
    if ranks is not None:
        _check(load_library().multi_lora_fwd_ranked(
            _ptr(X), _ptr(W), _ptr(A), _ptr(B), M, K, N, r, G,
            _arr(C.c_int64, list(seg_offsets)), _arr(C.c_int32, list(ranks)), _arr(C.c_float, list(s)),
            _arr(C.c_float, list(p)), _arr(C.c_uint64, list(seeds)), _ptr(Y), _ptr(S), _stream()))
        return Y, S
    _check(load_library().multi_lora_fwd(
        _ptr(X), _ptr(W), _ptr(A), _ptr(B), M, K, N, r, G,
        _arr(C.c_int64, list(seg_offsets)), _arr(C.c_float, list(s)), _arr(C.c_float, list(p)),
        _arr(C.c_uint64, list(seeds)), _ptr(Y), _ptr(S), _stream()))
    return Y, S


def multi_lora_bwd(X, W, A, B, S, dY, seg_offsets, s, p, seeds, need_dx=True, dA=None, dB=None,
                   accumulate=False, workspace=None, dX=None, ranks=None):
    """dX [M,K] bf16 (or None), dA [G,r,K] fp32, dB [G,N,r] fp32."""
    M, K = X.shape
    G, N, r = B.shape
    if need_dx and dX is None:
        dX = torch.empty((M, K), dtype=torch.bfloat16, device=X.device)
    dX = dX if need_dx else None
    dA = torch.empty((G, r, K), dtype=torch.float32, device=X.device) if dA is None else dA
    dB = torch.empty((G, N, r), dtype=torch.float32, device=X.device) if dB is None else dB
    ws = alloc_workspace(M, K, N, r, G, X.device) if workspace is None else workspace
    if ranks is not None:
        _check(load_library().multi_lora_bwd_ranked(
            _ptr(X), _ptr(W), _ptr(A), _ptr(B), _ptr(S), _ptr(dY), M, K, N, r, G,
            _arr(C.c_int64, list(seg_offsets)), _arr(C.c_int32, list(ranks)), _arr(C.c_float, list(s)),
            _arr(C.c_float, list(p)), _arr(C.c_uint64, list(seeds)), _ptr(dX), _ptr(dA), _ptr(dB), int(accumulate),
            _ptr(ws), ws.numel(), _stream()))
        return dX, dA, dB
    _check(load_library().multi_lora_bwd(
        _ptr(X), _ptr(W), _ptr(A), _ptr(B), _ptr(S), _ptr(dY), M, K, N, r, G,
        _arr(C.c_int64, list(seg_offsets)), _arr(C.c_float, list(s)), _arr(C.c_float, list(p)),
        _arr(C.c_uint64, list(seeds)), _ptr(dX), _ptr(dA), _ptr(dB), int(accumulate),
        _ptr(ws), ws.numel(), _stream()))
    return dX, dA, dB


def lora_debug_mask(M, K, p, seed, device="cuda"):
    keep = torch.empty((M, K), dtype=torch.uint8, device=device)
    _check(load_library().lora_debug_mask(M, K, p, seed, _ptr(keep), _stream()))
    return keep


def lora_debug_gemm_tiles(contraction, columns, r, seg_offsets):
    """[(tile rows, tile columns, first row)] of the one or two launches of a GEMM over these segments (host only)."""
    G = len(seg_offsets) - 1
    parts, rows, cols, first = C.c_int32(), (C.c_int32 * 2)(), (C.c_int32 * 2)(), (C.c_int64 * 2)()
    _check(load_library().lora_debug_gemm_tiles(seg_offsets[-1], contraction, columns, r, G, _arr(C.c_int64, seg_offsets),
                                                C.byref(parts), rows, cols, first))
    return [(rows[i], cols[i], first[i]) for i in range(parts.value)]


def lora_debug_bwd_plan(K, N, r, seg_offsets, need_dx=True, scratch=0) -> BwdPlan:
    """What a backward over these segments would launch (host only); scratch: bytes for its partial sums, 0 = the workspace's."""
    plan = BwdPlan()
    _check(load_library().lora_debug_bwd_plan(seg_offsets[-1], K, N, r, len(seg_offsets) - 1, _arr(C.c_int64, seg_offsets), int(need_dx),
                                              scratch, C.byref(plan)))
    return plan


def lora_debug_launches(K, N, r, seg_offsets) -> Launches:
    """The kernels of (1), (2) and (5) that a forward and a backward over these segments would launch (host only)."""
    out = Launches()
    _check(load_library().lora_debug_launches(seg_offsets[-1], K, N, r, len(seg_offsets) - 1, _arr(C.c_int64, seg_offsets), C.byref(out)))
    return out


def lora_set_row_tile(rows: int):
    """0: automatic choice per launch; 128 / 256: the small / large height of the GEMM tiles and the down-projection workgroups."""
    _check(load_library().lora_set_row_tile(int(rows)))


def lora_set_slab_lookahead(slabs: int):
    """0: automatic choice per launch; 1 / 2: the GEMMs copy their operand slabs one / two slabs ahead of the matrix work."""
    _check(load_library().lora_set_slab_lookahead(int(slabs)))


PROF_KERNELS = ("down", "fwd_gemm", "ds_db", "finalize_ds_db", "da", "finalize_da", "dx_gemm")


def profile_begin():
    _check(load_library().lora_profile_begin())


def profile_end():
    """{kernel name: (total ms, launches)} of the kernels enqueued since profile_begin()."""
    n = len(PROF_KERNELS)
    ms, cnt = (C.c_float * n)(), (C.c_int32 * n)()
    _check(load_library().lora_profile_end(ms, cnt))
    return {k: (float(ms[i]), int(cnt[i])) for i, k in enumerate(PROF_KERNELS)}


def unfused_workspace(M, K, N, r, device="cuda"):
    n = int(load_library().lora_unfused_workspace_bytes(M, K, N, r))
    if n == 0:
        raise LoraError(7)
    return torch.empty(n, dtype=torch.uint8, device=device)


def lora_unfused_fwd(X, W, A, B, s, p, seed, workspace, Y=None):
    """Unfused baseline forward: Y [M,N]; the dropped input and S stay in `workspace` for the backward."""
    M, K = X.shape
    N, r = B.shape
    Y = torch.empty((M, N), dtype=torch.bfloat16, device=X.device) if Y is None else Y
    _check(load_library().lora_unfused_fwd(_ptr(X), _ptr(W), _ptr(A), _ptr(B), M, K, N, r, s, p, seed, _ptr(Y),
                                           _ptr(workspace), workspace.numel(), _stream()))
    return Y


def lora_unfused_bwd(W, A, B, dY, s, p, seed, workspace, dX=None, dA=None, dB=None):
    """Unfused baseline backward (after lora_unfused_fwd on the same workspace): dX, dA, dB."""
    M, N = dY.shape
    r, K = A.shape
    dX = torch.empty((M, K), dtype=torch.bfloat16, device=dY.device) if dX is None else dX
    dA = torch.empty((r, K), dtype=torch.float32, device=dY.device) if dA is None else dA
    dB = torch.empty((N, r), dtype=torch.float32, device=dY.device) if dB is None else dB
    _check(load_library().lora_unfused_bwd(_ptr(W), _ptr(A), _ptr(B), _ptr(dY), M, K, N, r, s, p, seed,
                                           _ptr(dX), _ptr(dA), _ptr(dB), _ptr(workspace), workspace.numel(), _stream()))
    return dX, dA, dB


def frozen_fwd(X, W, Y=None):
    """Y = X W^T (frozen linear alone, same GEMM kernel)."""
    M, K = X.shape
    N = W.shape[0]
    Y = torch.empty((M, N), dtype=torch.bfloat16, device=X.device) if Y is None else Y
    _check(load_library().lora_frozen_fwd(_ptr(X), _ptr(W), M, K, N, _ptr(Y), _stream()))
    return Y


def frozen_bwd(dY, W, dX=None):
    """dX = dY W (frozen linear alone; the frozen weight gets no gradient)."""
    M, N = dY.shape
    K = W.shape[1]
    dX = torch.empty((M, K), dtype=torch.bfloat16, device=dY.device) if dX is None else dX
    _check(load_library().lora_frozen_bwd(_ptr(dY), _ptr(W), M, K, N, _ptr(dX), _stream()))
    return dX


def ceiling_mfma(operands, sink, workgroups, iters, shape=16) -> float:
    """Enqueues the register-resident MFMA loop (shape 16: the GEMM kernels' 16x16x32 instruction, 32: 32x32x16);
    returns the floating-point operations of the launch."""
    assert operands.numel() * operands.element_size() >= 65536 and sink.numel() >= workgroups * 256
    flops = C.c_double()
    _check(load_library().lora_ceiling_mfma(_ptr(operands), _ptr(sink), workgroups, iters, shape, C.byref(flops), _stream()))
    return flops.value


def ceiling_hbm_read(src, sink, workgroups) -> int:
    """Enqueues one plain read of `src`; returns the bytes read."""
    nbytes = src.numel() * src.element_size() // 16 * 16
    assert sink.numel() >= workgroups * 256
    _check(load_library().lora_ceiling_hbm_read(_ptr(src), nbytes, _ptr(sink), workgroups, _stream()))
    return nbytes


# ---- serving adapters, and what stands behind the query and key projections -----------------------------
# (a decode step's launches run for 3 - 5 us each: the checks look at every tensor once, and pointers go as numbers)
_BF16, _F32, _I32, _FP8, _U8 = torch.bfloat16, torch.float32, torch.int32, torch.float8_e4m3fn, torch.uint8
KV_FP4 = -4                            # LORA_KV_FP4 in the header


def _at(t: torch.Tensor, dtype) -> int:
    """Pointer of a contiguous GPU tensor of this type."""
    assert t.dtype is dtype and t.is_cuda and t.is_contiguous(), f"a contiguous GPU tensor of {dtype} is wanted, not {t.dtype} on {t.device}"
    return t.data_ptr()


def _heads(t: torch.Tensor):
    """Pointer and row stride of [rows, heads, dim] whose rows may be apart (a part of a fused projection's output)."""
    n, h, d = t.shape
    s = t.stride()
    assert t.dtype is _BF16 and t.is_cuda, f"bfloat16 [rows, heads, dim] on the GPU is wanted, not {t.dtype} on {t.device}"
    assert (s[2] == 1 or d == 1) and (s[1] == d or h == 1), "the heads of a row must lie side by side"
    return t.data_ptr(), s[0] if n > 1 else h * d


def lora_requests_fwd(X, W, A, B, ids, s, ranks=None, Y=None, S=None):
    """Y [M,N], S [M,r] of a batch in which row i has adapter ids[i] (outside 0 .. P-1: none).  X [M,K], W [N,K], A [P,r,K], B [P,N,r]
    bf16; ids [M] int32, s [P] fp32 and ranks [P] int32 (optional) on the GPU."""
    M, K = X.shape
    P, N, r = B.shape
    Y = torch.empty((M, N), dtype=_BF16, device=X.device) if Y is None else Y
    S = torch.empty((M, r), dtype=_BF16, device=X.device) if S is None else S
    assert W.shape == (N, K) and A.shape == (P, r, K) and ids.numel() == M and s.numel() == P and (ranks is None or ranks.numel() == P) and \
        Y.shape == (M, N) and S.shape == (M, r), "shapes do not fit"
    _check(load_library().lora_requests_fwd(_at(X, _BF16), _at(W, _BF16), _at(A, _BF16), _at(B, _BF16), _at(ids, _I32),
                                            None if ranks is None else _at(ranks, _I32), _at(s, _F32), M, K, N, r, P, _at(Y, _BF16),
                                            _at(S, _BF16), _stream()))
    return Y, S


def lora_weights_write(W, codes=None, exps=None):
    """codes [N,K/2], exps [N,K/32] (uint8): W [N,K] bf16 in 4 bits with a power of two for every 32 entries of a row."""
    N, K = W.shape
    codes = torch.empty((N, K // 2), dtype=_U8, device=W.device) if codes is None else codes
    exps = torch.empty((N, K // 32), dtype=_U8, device=W.device) if exps is None else exps
    assert codes.shape == (N, K // 2) and exps.shape == (N, K // 32), "shapes do not fit"
    _check(load_library().lora_weights_write(_at(W, _BF16), N, K, _at(codes, _U8), _at(exps, _U8), _stream()))
    return codes, exps


def lora_weights_read(codes, exps, W=None):
    """W [N,K] bf16, exactly what codes and exps hold: for lora_fwd, lora_bwd and the like over the same frozen weights."""
    N, K = codes.shape[0], 2 * codes.shape[1]
    W = torch.empty((N, K), dtype=_BF16, device=codes.device) if W is None else W
    assert W.shape == (N, K) and exps.shape == (N, K // 32), "shapes do not fit"
    _check(load_library().lora_weights_read(_at(codes, _U8), _at(exps, _U8), N, K, _at(W, _BF16), _stream()))
    return W


def lora_requests_quantised_fwd(X, codes, exps, A=None, B=None, ids=None, s=None, ranks=None, Y=None, S=None):
    """lora_requests_fwd over weights in 4 bits (codes, exps: lora_weights_write).  Without A, B, ids and s: no adapters, and S is None."""
    M, K = X.shape
    N = codes.shape[0]
    Y = torch.empty((M, N), dtype=_BF16, device=X.device) if Y is None else Y
    assert codes.shape == (N, K // 2) and exps.shape == (N, K // 32) and Y.shape == (M, N), "shapes do not fit"
    if A is None:
        assert B is None and ids is None and s is None and ranks is None, "adapters are A, B, ids and s together"
        _check(load_library().lora_requests_quantised_fwd(_at(X, _BF16), _at(codes, _U8), _at(exps, _U8), None, None, None, None, None, M, K, N, 0, 0,
                                                          _at(Y, _BF16), None, _stream()))
        return Y, None
    P, _, r = B.shape
    S = torch.empty((M, r), dtype=_BF16, device=X.device) if S is None else S
    assert A.shape == (P, r, K) and B.shape == (P, N, r) and ids.numel() == M and s.numel() == P and (ranks is None or ranks.numel() == P) and \
        S.shape == (M, r), "shapes do not fit"
    _check(load_library().lora_requests_quantised_fwd(_at(X, _BF16), _at(codes, _U8), _at(exps, _U8), _at(A, _BF16), _at(B, _BF16), _at(ids, _I32),
                                                      None if ranks is None else _at(ranks, _I32), _at(s, _F32), M, K, N, r, P, _at(Y, _BF16),
                                                      _at(S, _BF16), _stream()))
    return Y, S


def lora_debug_quantised_tiles(M, K, N, r=0, P=0) -> QuantisedTiles:
    """What lora_requests_quantised_fwd of these sizes runs with (host only)."""
    out = QuantisedTiles()
    _check(load_library().lora_debug_quantised_tiles(M, K, N, r, P, C.byref(out)))
    return out


def _rope_sizes(q, k, gq, gk, cos, sin, pos):
    M, H, D = q.shape
    G = k.shape[1]
    positions, half = cos.shape
    assert k.shape == (M, G, D) and gq.numel() == D and gk.numel() == D and pos.numel() == M and cos.shape == sin.shape, "shapes do not fit"
    return M, H, G, D, 2 * half, positions


def lora_qk_norm_rope_fwd(q, k, gq, gk, cos, sin, pos, eps=1e-6, interleaved=False, q_out=None, k_out=None):
    """q_out [M,H,D], k_out [M,G,D]: RMS norm of every head of q [M,H,D] and k [M,G,D] (rows may be apart) with gq, gk [D], turned by row
    pos[i] (int32) of cos, sin [positions, rot/2] fp32."""
    M, H, G, D, rot, positions = _rope_sizes(q, k, gq, gk, cos, sin, pos)
    q_out = torch.empty((M, H, D), dtype=_BF16, device=q.device) if q_out is None else q_out
    k_out = torch.empty((M, G, D), dtype=_BF16, device=q.device) if k_out is None else k_out
    assert q_out.shape == q.shape and k_out.shape == k.shape, "shapes do not fit"
    qp, ldq = _heads(q)
    kp, ldk = _heads(k)
    qo, ldqo = _heads(q_out)
    ko, ldko = _heads(k_out)
    _check(load_library().lora_qk_norm_rope_fwd(qp, kp, _at(gq, _BF16), _at(gk, _BF16), _at(cos, _F32), _at(sin, _F32), _at(pos, _I32), M, H, G, D,
                                                rot, positions, ldq, ldk, ldqo, ldko, eps, interleaved, qo, ko, _stream()))
    return q_out, k_out


def alloc_qk_norm_rope_workspace(M, H, G, D, device="cuda") -> torch.Tensor:
    return torch.empty(max(int(load_library().lora_qk_norm_rope_workspace_bytes(M, H, G, D)), 256), dtype=torch.uint8, device=device)


def lora_qk_norm_rope_bwd(q, k, gq, gk, cos, sin, pos, dq_out, dk_out, eps=1e-6, interleaved=False, dq=None, dk=None, dgq=None, dgk=None,
                          accumulate=False, workspace=None):
    """dq, dk (bf16, as q and k), dgq, dgk [D] fp32 of lora_qk_norm_rope_fwd for the gradients dq_out, dk_out of its outputs."""
    M, H, G, D, rot, positions = _rope_sizes(q, k, gq, gk, cos, sin, pos)
    dq = torch.empty((M, H, D), dtype=_BF16, device=q.device) if dq is None else dq
    dk = torch.empty((M, G, D), dtype=_BF16, device=q.device) if dk is None else dk
    dgq = torch.empty(D, dtype=_F32, device=q.device) if dgq is None else dgq
    dgk = torch.empty(D, dtype=_F32, device=q.device) if dgk is None else dgk
    assert dq.shape == q.shape == dq_out.shape and dk.shape == k.shape == dk_out.shape and dgq.numel() == D and dgk.numel() == D, "shapes do not fit"
    ws = alloc_qk_norm_rope_workspace(M, H, G, D, q.device) if workspace is None else workspace
    (qp, ldq), (kp, ldk), (qo, ldqo), (ko, ldko), (dqp, lddq), (dkp, lddk) = (_heads(t) for t in (q, k, dq_out, dk_out, dq, dk))
    _check(load_library().lora_qk_norm_rope_bwd(qp, kp, _at(gq, _BF16), _at(gk, _BF16), _at(cos, _F32), _at(sin, _F32), _at(pos, _I32), qo, ko, M, H, G,
                                                D, rot, positions, ldq, ldk, ldqo, ldko, lddq, lddk, eps, interleaved, dqp, dkp, _at(dgq, _F32),
                                                _at(dgk, _F32), accumulate, _at(ws, torch.uint8), ws.numel(), _stream()))
    return dq, dk, dgq, dgk


class KVCache:
    """A paged cache over tensors that the caller holds: k, v [pages, heads, page, dim], bf16, or fp8 (torch.float8_e4m3fn) with
    the biased exponents k_exp, v_exp [pages, heads, page] (uint8) of a power of two for every token and head, or 4 bits: k, v [pages, heads, page, dim/2]
    (uint8, two codes to a byte) with k_exp, v_exp [pages, heads, page, dim/32] of a power of two for every 32 entries."""
    __slots__ = ("tensors", "pages", "heads", "page", "dim", "_c", "_ref")

    def __init__(self, k, v, k_exp=None, v_exp=None):
        shape = k.shape
        assert len(shape) == 4 and v.shape == shape, "k and v are [pages, heads, page, dim]"
        self.pages, self.heads, self.page, self.dim = pages, heads, page, dim = shape
        dtype, form, exps = k.dtype, 0, None
        if dtype is _U8:
            self.dim = 2 * dim
            form, exps = KV_FP4, (pages, heads, page, dim // 16)
        elif dtype is _FP8:
            form, exps = 1, (pages, heads, page)
        if form:
            assert k_exp is not None and v_exp is not None and k_exp.shape == v_exp.shape == exps, "exponents: one for every token and head, 4 bits for every 32 entries"
            self.tensors = (k, v, k_exp, v_exp)
            self._c = CacheArrays(_at(k, dtype), _at(v, dtype), _at(k_exp, _U8), _at(v_exp, _U8), pages, page, heads, self.dim, form)
        else:
            self.tensors = (k, v, None, None)
            self._c = CacheArrays(_at(k, _BF16), _at(v, _BF16), None, None, pages, page, heads, dim, 0)
        self._ref = C.byref(self._c)

    @classmethod
    def empty(cls, pages, page, heads, dim, fp8=False, device="cuda", fp4=False):
        assert not (fp8 and fp4), "fp8 or fp4"
        width, dtype = (dim // 2, _U8) if fp4 else (dim, _FP8 if fp8 else _BF16)
        k, v = (torch.zeros((pages, heads, page, width), dtype=dtype, device=device) for _ in range(2))
        shape = (pages, heads, page, dim // 32) if fp4 else (pages, heads, page)
        exps = (torch.zeros(shape, dtype=_U8, device=device) for _ in range(2)) if fp8 or fp4 else (None, None)
        return cls(k, v, *exps)


def lora_kv_cache_write(cache: KVCache, k, v, slots):
    """Rows of k, v [M, heads, dim] (rows may be apart) to the slots (int64: page number * page + place; outside the cache: left out; each at most
    once)."""
    M = slots.numel()
    assert k.shape == (M, cache.heads, cache.dim) and v.shape == k.shape, "shapes do not fit"
    kp, ldk = _heads(k)
    vp, ldv = _heads(v)
    _check(load_library().lora_kv_cache_write(cache._ref, kp, vp, ldk, ldv, _at(slots, torch.int64), M, _stream()))


def lora_kv_cache_read(cache: KVCache, slots, k=None, v=None):
    """k, v [M, heads, dim] bf16 of the slots (outside the cache: zeros)."""
    M = slots.numel()
    k = torch.empty((M, cache.heads, cache.dim), dtype=_BF16, device=slots.device) if k is None else k
    v = torch.empty((M, cache.heads, cache.dim), dtype=_BF16, device=slots.device) if v is None else v
    assert k.shape == (M, cache.heads, cache.dim) and v.shape == k.shape, "shapes do not fit"
    kp, ldk = _heads(k)
    vp, ldv = _heads(v)
    _check(load_library().lora_kv_cache_read(cache._ref, _at(slots, torch.int64), M, kp, vp, ldk, ldv, _stream()))
    return k, v


def lora_kv_cache_append(cache: KVCache, q, k, v, cos, sin, pos, slots, gq=None, gk=None, eps=1e-6, interleaved=False, q_out=None):
    """q_out [M,H,D]: lora_qk_norm_rope_fwd and lora_kv_cache_write in one call: queries out, keys and v [M, heads, dim] (rows may be apart) to their slots; without gq
    and gk no norm, the rotation alone."""
    M, H, D = q.shape
    positions, half = cos.shape
    q_out = torch.empty((M, H, D), dtype=_BF16, device=q.device) if q_out is None else q_out
    assert D == cache.dim and k.shape == v.shape == (M, cache.heads, D) and cos.shape == sin.shape and pos.numel() == M and slots.numel() == M and \
        q_out.shape == q.shape and (gq is None or gq.numel() == D) and (gk is None or gk.numel() == D), "shapes do not fit"
    qp, ldq = _heads(q)
    kp, ldk = _heads(k)
    vp, ldv = _heads(v)
    qo, ldqo = _heads(q_out)
    _check(load_library().lora_kv_cache_append(cache._ref, qp, kp, vp, None if gq is None else _at(gq, _BF16), None if gk is None else _at(gk, _BF16),
                                               _at(cos, _F32), _at(sin, _F32), _at(pos, _I32), _at(slots, torch.int64), M, H, 2 * half, positions, ldq,
                                               ldk, ldv, ldqo, eps, interleaved, qo, _stream()))
    return q_out


def alloc_paged_attn_workspace(cache: KVCache, T, H, seqs, max_new, max_kv, window=0, device="cuda") -> torch.Tensor:
    """For steps of at most T tokens of at most seqs sequences, max_new tokens of each and max_kv keys."""
    n = int(load_library().lora_paged_attn_workspace_bytes(cache._ref, T, H, seqs, max_new, max_kv, window))
    return torch.empty(max(n, 256), dtype=torch.uint8, device=device)


def lora_paged_attn_fwd(q, cache: KVCache, table, offsets, kv_lens, max_new, max_kv, scale=None, window=0, out=None, workspace=None):
    """out [T,H,dim]: the new tokens q [T,H,dim] of len(kv_lens) sequences (rows offsets[b] .. offsets[b+1]-1) over the kv_lens[b] tokens that the
    cache holds of each in the pages table[b] (int32 [sequences, pages], as offsets and kv_lens), the new ones among them."""
    T, H, D = q.shape
    B, max_pages = table.shape
    out = torch.empty((T, H, D), dtype=_BF16, device=q.device) if out is None else out
    assert D == cache.dim and offsets.numel() == B + 1 and kv_lens.numel() == B and out.shape == q.shape, "shapes do not fit"
    ldt, one = table.stride()
    assert table.dtype is _I32 and table.is_cuda and (one == 1 or max_pages <= 1), "int32 pages on the GPU, those of a sequence side by side, are wanted"
    ws = alloc_paged_attn_workspace(cache, T, H, B, max_new, max_kv, window, q.device) if workspace is None else workspace
    qp, ldq = _heads(q)
    op, ldo = _heads(out)
    _check(load_library().lora_paged_attn_fwd(qp, cache._ref, table.data_ptr(), _at(offsets, _I32), _at(kv_lens, _I32), T, H, B, max_pages, ldq,
                                              ldt if B > 1 else max_pages, ldo, max_new, max_kv, D ** -0.5 if scale is None else scale, window, op,
                                              _at(ws, torch.uint8), ws.numel(), _stream()))
    return out
