"""Thin ctypes binding of libsik.so (C ABI in include/sik.h).

Argument marshalling only: every step of the path runs in the HIP kernels.  torch is used for
device memory and streams; tensors are passed as raw device pointers.  There is no CPU fallback:
if the shared library is missing or a call fails, an exception is raised.
"""
import ctypes
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsik.so")

SIK_F16, SIK_BF16, SIK_F32 = 0, 1, 2
SIK_Q_FIT, SIK_Q_ENCODE = 1, 2
_TORCH2SIK = {torch.float16: SIK_F16, torch.bfloat16: SIK_BF16, torch.float32: SIK_F32}

EXPORTS = ("sik_strerror", "sik_version", "sik_plan_info", "sik_workspace_bytes", "sik_workspace_init",
           "sik_workspace_status", "sik_quantize_keys", "sik_score",
           "sik_topk", "sik_sparse_attn", "sik_decode_step", "sik_decode_step_static", "sik_decode_step_profiled", "sik_kvq_bytes",
           "sik_quantize_kv", "sik_prefill_compress", "sik_sparse_attn_q2", "sik_decode_step_q2", "sik_decode_step_ex",
           "sik_rope_append", "sik_chunk_workspace_bytes", "sik_chunk_attn", "sik_attn_mass", "sik_evict")


class SikError(RuntimeError):
    def __init__(self, status, text):
        super().__init__(f"sik status {status}: {text}")
        self.status = status


class DecodeArgs(ctypes.Structure):
    """sik_decode_args of include/sik.h."""
    _fields_ = [("q", ctypes.c_void_p), ("k_new", ctypes.c_void_p), ("v_new", ctypes.c_void_p),
                ("K", ctypes.c_void_p), ("V", ctypes.c_void_p), ("kvq", ctypes.c_void_p), ("alpha", ctypes.c_void_p),
                ("seq_len", ctypes.c_void_p), ("mu", ctypes.c_void_p), ("codebook", ctypes.c_void_p),
                ("codes", ctypes.c_void_p), ("k", ctypes.c_int32), ("k_per_mille", ctypes.c_int32),
                ("group_shared", ctypes.c_int32), ("softmax_scale", ctypes.c_float),
                ("forced_idx", ctypes.c_void_p), ("n_forced", ctypes.c_int32), ("forced_K", ctypes.c_void_p),
                ("forced_V", ctypes.c_void_p), ("out", ctypes.c_void_p), ("idx_out", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t), ("stream", ctypes.c_void_p),
                ("kernel_us", ctypes.POINTER(ctypes.c_float)), ("launches", ctypes.c_int32),
                ("spin_limit", ctypes.c_int32)]


class Layout(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("max_len", ctypes.c_int32), ("kv_dtype", ctypes.c_int32),
                ("out_dtype", ctypes.c_int32)]


class Pages(ctypes.Structure):
    """sik_pages of include/sik.h (make_pages keeps the tensor it points to alive)."""
    _fields_ = [("page_table", ctypes.c_void_p), ("pages_per_seq", ctypes.c_int32), ("page_len", ctypes.c_int32),
                ("n_pages", ctypes.c_int32)]


class Chunk(ctypes.Structure):
    """sik_chunk of include/sik.h (make_chunk keeps what it points to alive)."""
    _fields_ = [("n", ctypes.c_int32), ("n_new", ctypes.c_void_p), ("seq_len", ctypes.c_void_p),
                ("pages", ctypes.POINTER(Pages))]


class RopeArgs(ctypes.Structure):
    """sik_rope_args of include/sik.h."""
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("q_stride", ctypes.c_int64),
                ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64), ("q_weight", ctypes.c_void_p),
                ("k_weight", ctypes.c_void_p), ("eps", ctypes.c_float), ("inv_freq", ctypes.c_void_p),
                ("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("positions", ctypes.c_void_p),
                ("q_out", ctypes.c_void_p), ("k_out", ctypes.c_void_p), ("K", ctypes.c_void_p), ("V", ctypes.c_void_p),
                ("stream", ctypes.c_void_p)]


class EvictArgs(ctypes.Structure):
    """sik_evict_args of include/sik.h."""
    _fields_ = [("mass", ctypes.c_void_p), ("seq_len", ctypes.c_void_p), ("n_keep", ctypes.c_int32),
                ("n_sink", ctypes.c_int32), ("n_recent", ctypes.c_int32), ("keep", ctypes.c_void_p),
                ("new_len", ctypes.c_void_p), ("K", ctypes.c_void_p), ("V", ctypes.c_void_p),
                ("pages", ctypes.POINTER(Pages)), ("K_out", ctypes.c_void_p), ("V_out", ctypes.c_void_p),
                ("mass_out", ctypes.c_void_p), ("out_len", ctypes.c_int32), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t), ("stream", ctypes.c_void_p)]


_lib = None


def lib():
    """Load libsik.so (built in-tree by paper_2603_14224_amd/build.py); raises if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} not built: run `python -m paper_2603_14224_amd.build` "
                              "(or __graft_entry__.build()) first; there is no fallback path")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, sz, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t, ctypes.c_float
        lp = ctypes.POINTER(Layout)
        L.sik_strerror.restype = ctypes.c_char_p
        L.sik_strerror.argtypes = [ctypes.c_int]
        L.sik_version.restype = ctypes.c_int
        L.sik_plan_info.restype = ctypes.c_int
        L.sik_plan_info.argtypes = [lp, ctypes.POINTER(i32)]
        L.sik_workspace_bytes.restype = sz
        L.sik_workspace_init.restype = ctypes.c_int
        L.sik_workspace_init.argtypes = [lp, i32, vp, sz, vp]
        L.sik_workspace_status.restype = ctypes.c_int
        L.sik_workspace_status.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_uint32)]
        L.sik_workspace_bytes.argtypes = [lp, i32]
        L.sik_quantize_keys.restype = ctypes.c_int
        L.sik_quantize_keys.argtypes = [lp, vp, vp, i32, i32, ctypes.c_int, vp, vp, vp, vp, vp, sz, vp]
        L.sik_score.restype = ctypes.c_int
        L.sik_score.argtypes = [lp, vp, vp, vp, vp, vp, vp]
        L.sik_topk.restype = ctypes.c_int
        L.sik_topk.argtypes = [lp, vp, vp, i32, vp, vp, sz, vp]
        L.sik_sparse_attn.restype = ctypes.c_int
        L.sik_sparse_attn.argtypes = [lp, vp, vp, vp, vp, i32, f32, vp, vp, sz, vp]
        L.sik_decode_step.restype = ctypes.c_int
        L.sik_decode_step.argtypes = [lp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, f32, vp, vp, vp, sz, vp]
        L.sik_decode_step_static.restype = ctypes.c_int
        L.sik_decode_step_static.argtypes = [lp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, f32, vp, vp, vp]
        L.sik_decode_step_profiled.restype = ctypes.c_int
        L.sik_decode_step_profiled.argtypes = L.sik_decode_step.argtypes + [ctypes.POINTER(ctypes.c_float)]
        L.sik_kvq_bytes.restype = sz
        L.sik_kvq_bytes.argtypes = [lp]
        L.sik_quantize_kv.restype = ctypes.c_int
        L.sik_quantize_kv.argtypes = [lp, vp, vp, vp, i32, i32, ctypes.c_int, vp, vp, vp, vp]
        L.sik_prefill_compress.restype = ctypes.c_int
        L.sik_prefill_compress.argtypes = [lp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.sik_sparse_attn_q2.restype = ctypes.c_int
        L.sik_sparse_attn_q2.argtypes = [lp, vp, vp, vp, vp, i32, f32, vp, vp, sz, vp]
        L.sik_decode_step_ex.restype = ctypes.c_int
        L.sik_decode_step_ex.argtypes = [lp, ctypes.POINTER(DecodeArgs)]
        L.sik_decode_step_q2.restype = ctypes.c_int
        L.sik_decode_step_q2.argtypes = [lp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, f32, vp, vp, vp, sz, vp,
                                         ctypes.POINTER(ctypes.c_float)]
        L.sik_rope_append.restype = ctypes.c_int
        L.sik_rope_append.argtypes = [lp, ctypes.POINTER(Chunk), ctypes.POINTER(RopeArgs)]
        L.sik_chunk_workspace_bytes.restype = sz
        L.sik_chunk_workspace_bytes.argtypes = [lp, i32]
        L.sik_chunk_attn.restype = ctypes.c_int
        L.sik_chunk_attn.argtypes = [lp, ctypes.POINTER(Chunk), vp, vp, vp, f32, vp, vp, vp, sz, vp]
        L.sik_attn_mass.restype = ctypes.c_int
        L.sik_attn_mass.argtypes = [lp, ctypes.POINTER(Chunk), vp, vp, f32, vp, i32, vp, vp, vp]
        L.sik_evict.restype = ctypes.c_int
        L.sik_evict.argtypes = [lp, ctypes.POINTER(EvictArgs)]
        _lib = L
    return _lib


def _check(rc):
    if rc != 0:
        raise SikError(rc, lib().sik_strerror(rc).decode())


def _ptr(t):
    if t is None:
        return None
    assert t.is_contiguous(), "sik tensors must be contiguous"
    return ctypes.c_void_p(t.data_ptr())


def _stream():
    # Without a GPU the C side still validates arguments first; any launch then reports SIK_ERR_LAUNCH.
    if not torch.cuda.is_available():
        return None
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def make_layout(batch, n_kv_heads, n_q_heads, head_dim, max_len, kv_dtype, out_dtype=None) -> Layout:
    kd = _TORCH2SIK[kv_dtype] if isinstance(kv_dtype, torch.dtype) else int(kv_dtype)
    od = kd if out_dtype is None else (_TORCH2SIK[out_dtype] if isinstance(out_dtype, torch.dtype) else int(out_dtype))
    return Layout(batch, n_kv_heads, n_q_heads, head_dim, max_len, kd, od)


def sik_strerror(status: int) -> str:
    return lib().sik_strerror(status).decode()


def sik_plan_info(layout: Layout):
    """Launch geometry of a layout (SIK_PLAN_INFO_LEN ints, see include/sik.h); raises on a bad layout."""
    info = (ctypes.c_int32 * 8)()
    _check(lib().sik_plan_info(ctypes.byref(layout), info))
    return [int(x) for x in info]


def sik_workspace_bytes(layout: Layout, k: int) -> int:
    return int(lib().sik_workspace_bytes(ctypes.byref(layout), int(k)))


def alloc_workspace(layout: Layout, k: int, device="cuda") -> torch.Tensor:
    """Device buffer of sik_workspace_bytes, initialised with sik_workspace_init."""
    n = sik_workspace_bytes(layout, k)
    if n == 0:
        raise SikError(-2, "sik_workspace_bytes rejected the layout / k")
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    sik_workspace_init(layout, k, ws)
    return ws


def sik_workspace_init(layout: Layout, k: int, workspace):
    _check(lib().sik_workspace_init(ctypes.byref(layout), int(k), _ptr(workspace), workspace.numel(), _stream()))


def sik_workspace_status(workspace) -> int:
    """Status word of the workspace after waiting for the current stream (0 = every step completed)."""
    st = ctypes.c_uint32(0)
    _check(lib().sik_workspace_status(_ptr(workspace), _stream(), ctypes.byref(st)))
    return int(st.value)


def sik_quantize_keys(layout, K, seq_len, t0, n, mode, mu, codebook, counts, codes, workspace):
    _check(lib().sik_quantize_keys(ctypes.byref(layout), _ptr(K), _ptr(seq_len), int(t0), int(n), int(mode),
                                   _ptr(mu), _ptr(codebook), _ptr(counts), _ptr(codes), _ptr(workspace),
                                   workspace.numel() if workspace is not None else 0, _stream()))


def sik_score(layout, q, codebook, codes, seq_len, scores):
    _check(lib().sik_score(ctypes.byref(layout), _ptr(q), _ptr(codebook), _ptr(codes), _ptr(seq_len),
                           _ptr(scores), _stream()))


def sik_topk(layout, scores, seq_len, k, idx, workspace):
    _check(lib().sik_topk(ctypes.byref(layout), _ptr(scores), _ptr(seq_len), int(k), _ptr(idx),
                          _ptr(workspace), workspace.numel() if workspace is not None else 0, _stream()))


def sik_sparse_attn(layout, q, K, V, idx, k, softmax_scale, out, workspace):
    _check(lib().sik_sparse_attn(ctypes.byref(layout), _ptr(q), _ptr(K), _ptr(V), _ptr(idx), int(k),
                                 float(softmax_scale), _ptr(out), _ptr(workspace),
                                 workspace.numel() if workspace is not None else 0, _stream()))


def sik_kvq_bytes(layout: Layout) -> int:
    return int(lib().sik_kvq_bytes(ctypes.byref(layout)))


def alloc_kvq(layout: Layout, device="cuda") -> torch.Tensor:
    """Zeroed record plane [B, Hkv, max_len, 128] uint8 of the 2-bit K/V format."""
    n = sik_kvq_bytes(layout)
    if n == 0:
        raise SikError(-2, "sik_kvq_bytes rejected the layout")
    return torch.zeros(layout.batch, layout.n_kv_heads, layout.max_len, 128, dtype=torch.uint8, device=device)


def sik_quantize_kv(layout, K, V, seq_len, t0, n, mode, mu, alpha, kvq):
    _check(lib().sik_quantize_kv(ctypes.byref(layout), _ptr(K), _ptr(V), _ptr(seq_len), int(t0), int(n), int(mode),
                                 _ptr(mu), _ptr(alpha), _ptr(kvq), _stream()))


def sik_prefill_compress(layout, K, V, seq_len, mu, codebook, counts, codes, alpha, kvq, workspace):
    """mu, codes, codebook, counts, alpha and records of the fitted tokens in two passes over K and one over V."""
    _check(lib().sik_prefill_compress(ctypes.byref(layout), _ptr(K), _ptr(V), _ptr(seq_len), _ptr(mu), _ptr(codebook),
                                      _ptr(counts), _ptr(codes), _ptr(alpha), _ptr(kvq), _ptr(workspace),
                                      workspace.numel() if workspace is not None else 0, _stream()))


def sik_sparse_attn_q2(layout, q, kvq, alpha, idx, k, softmax_scale, out, workspace):
    _check(lib().sik_sparse_attn_q2(ctypes.byref(layout), _ptr(q), _ptr(kvq), _ptr(alpha), _ptr(idx), int(k),
                                    float(softmax_scale), _ptr(out), _ptr(workspace),
                                    workspace.numel() if workspace is not None else 0, _stream()))


def sik_decode_step_q2(layout, q, k_new, v_new, kvq, seq_len, mu, alpha, codebook, codes, k, softmax_scale, out,
                       idx_out, workspace, profiled=False):
    """Decode step on the 2-bit cache; with profiled=True returns the SIK_N_KERNELS + 1 event intervals (us)."""
    us = (ctypes.c_float * 5)() if profiled else None
    _check(lib().sik_decode_step_q2(ctypes.byref(layout), _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(kvq),
                                    _ptr(seq_len), _ptr(mu), _ptr(alpha), _ptr(codebook), _ptr(codes), int(k),
                                    float(softmax_scale), _ptr(out), _ptr(idx_out), _ptr(workspace),
                                    workspace.numel() if workspace is not None else 0, _stream(), us))
    return [float(x) for x in us] if profiled else None


def sik_decode_step_ex(layout, *, q, seq_len, codebook, codes, k, out, workspace, k_new=None, v_new=None, K=None,
                       V=None, kvq=None, alpha=None, mu=None, softmax_scale=0.0, forced_idx=None, forced_K=None,
                       forced_V=None, idx_out=None, k_per_mille=0, group_shared=False, profiled=False,
                       launches=0, spin_limit=0):
    """General decode step (argument block of include/sik.h): either cache format, optional forced set."""
    us = (ctypes.c_float * 5)() if profiled else None

    def vp(t):
        return None if t is None else _ptr(t).value

    st = _stream()

    a = DecodeArgs(q=vp(q), k_new=vp(k_new), v_new=vp(v_new), K=vp(K), V=vp(V), kvq=vp(kvq), alpha=vp(alpha),
                   seq_len=vp(seq_len), mu=vp(mu), codebook=vp(codebook), codes=vp(codes), k=int(k),
                   k_per_mille=int(k_per_mille), group_shared=1 if group_shared else 0, softmax_scale=float(softmax_scale), forced_idx=vp(forced_idx),
                   n_forced=0 if forced_idx is None else int(forced_idx.shape[-1]), forced_K=vp(forced_K),
                   forced_V=vp(forced_V), out=vp(out), idx_out=vp(idx_out), workspace=vp(workspace),
                   workspace_bytes=workspace.numel() if workspace is not None else 0,
                   stream=None if st is None else st.value, kernel_us=us, launches=int(launches),
                   spin_limit=int(spin_limit))
    _check(lib().sik_decode_step_ex(ctypes.byref(layout), ctypes.byref(a)))
    return [float(x) for x in us] if profiled else None


def sik_decode_step(layout, q, k_new, v_new, K, V, seq_len, mu, codebook, codes, k, softmax_scale, out, idx_out,
                    workspace):
    _check(lib().sik_decode_step(ctypes.byref(layout), _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(K), _ptr(V),
                                 _ptr(seq_len), _ptr(mu), _ptr(codebook), _ptr(codes), int(k),
                                 float(softmax_scale), _ptr(out), _ptr(idx_out), _ptr(workspace),
                                 workspace.numel() if workspace is not None else 0, _stream()))


SIK_STATIC_SCRATCH_BYTES = 32 << 20


def sik_decode_step_static(layout, q, k_new, v_new, K, V, seq_len, mu, codebook, codes, k, softmax_scale, out, idx_out):
    """sik_decode_step on the library's built-in scratch buffer (no workspace argument, nothing allocated)."""
    _check(lib().sik_decode_step_static(ctypes.byref(layout), _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(K), _ptr(V),
                                        _ptr(seq_len), _ptr(mu), _ptr(codebook), _ptr(codes), int(k),
                                        float(softmax_scale), _ptr(out), _ptr(idx_out), _stream()))


def sik_decode_step_profiled(layout, q, k_new, v_new, K, V, seq_len, mu, codebook, codes, k, softmax_scale, out,
                             idx_out, workspace):
    """Runs one decode step with per-kernel HIP events; returns the 4 event-to-event intervals and the
    empty-interval cost of an event pair, in microseconds."""
    us = (ctypes.c_float * 5)()
    _check(lib().sik_decode_step_profiled(ctypes.byref(layout), _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(K),
                                          _ptr(V), _ptr(seq_len), _ptr(mu), _ptr(codebook), _ptr(codes), int(k),
                                          float(softmax_scale), _ptr(out), _ptr(idx_out), _ptr(workspace),
                                          workspace.numel() if workspace is not None else 0, _stream(), us))
    return list(us)


# ---- the prompt side of the cache.  These calls check types, shapes and devices of the tensors here; what the C ABI can
# see (alignment, ranges, page sizes) it checks itself.

_has_gpu = None


def _device():
    """Index of the device that the calls run on (-1 without a GPU: the C side then validates and reports)."""
    global _has_gpu
    if _has_gpu is None:
        _has_gpu = torch.cuda.is_available()
    return torch.cuda.current_device() if _has_gpu else -1


def _stream_of(dev):
    return torch.cuda.current_stream(dev).cuda_stream if dev >= 0 else None


def _tensor(name, t, dtype, dev, shape=None, numel=None, optional=False):
    """Address of a tensor after its checks, None for an absent optional one."""
    if t is None:
        if optional:
            return None
        raise ValueError(f"{name} is required")
    if t.dtype is not dtype:
        raise ValueError(f"{name}: {t.dtype} given, {dtype} needed")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)} given, {shape} needed")
    if numel is not None and t.numel() != numel:
        raise ValueError(f"{name}: {t.numel()} elements given, {numel} needed")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, the call runs on device {dev}")
    return t.data_ptr()


_SIK2TORCH = {SIK_F16: torch.float16, SIK_BF16: torch.bfloat16, SIK_F32: torch.float32}


def make_pages(page_table, page_len, n_pages) -> Pages:
    """Description of a paged cache: page_table [B, pages_per_seq] int32, pools of n_pages pages of page_len tokens."""
    if page_table.dim() != 2:
        raise ValueError("page_table must be [batch, pages per sequence]")
    pages = Pages(_tensor("page_table", page_table, torch.int32, _device()), page_table.shape[1], int(page_len), int(n_pages))
    pages.tensor = page_table
    return pages


def make_chunk(n, seq_len, n_new=None, pages=None) -> Chunk:
    """A chunk of n new tokens per sequence (n_new[b] of them real) behind the seq_len[b] tokens in the cache."""
    dev = _device()
    chunk = Chunk(int(n), _tensor("n_new", n_new, torch.int32, dev, optional=True),
                  _tensor("seq_len", seq_len, torch.int32, dev), None if pages is None else ctypes.pointer(pages))
    chunk.tensors = (seq_len, n_new, pages)
    return chunk


def _check_chunk(layout, chunk, dev):
    seq_len, n_new, pages = chunk.tensors
    if seq_len.numel() != layout.batch or (n_new is not None and n_new.numel() != layout.batch):
        raise ValueError("seq_len and n_new hold one length per sequence")
    if seq_len.get_device() != dev:
        raise ValueError(f"the chunk is on {seq_len.device}, the call runs on device {dev}")
    _check_page_table(layout, pages, dev)
    return pages


def _check_page_table(layout, pages, dev):
    if pages is not None and (pages.tensor.shape[0] != layout.batch or pages.tensor.get_device() != dev):
        raise ValueError("page_table holds one row per sequence and lies on the device of the call")


def _cache_shape(layout, pages):
    """Shape of one side of a contiguous or paged cache."""
    if pages is None:
        return (layout.batch, layout.n_kv_heads, layout.max_len, layout.head_dim)
    return (pages.n_pages, layout.n_kv_heads, pages.page_len, layout.head_dim)


def _head_rows(name, t, dtype, dev, shape):
    """Address and token stride of [B, n, heads, D] head rows, which may be part of a wider projection's output."""
    if t is None:
        raise ValueError(f"{name} is required")
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)} given, {dtype} {shape} needed")
    B, n, heads, D = shape
    s0, s1, s2, s3 = t.stride()
    stride = s1 if n > 1 else s0 if B > 1 else heads * D
    if s3 != 1 or (heads > 1 and s2 != D) or (B > 1 and s0 != n * stride):
        raise ValueError(f"{name}: head rows of a token must be contiguous and tokens evenly spaced")
    if stride < heads * D:  # a broadcast row has the stride 0, which to the C side means packed rows
        raise ValueError(f"{name}: tokens overlap (one every {stride} elements, {heads * D} needed)")
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, the call runs on device {dev}")
    return t.data_ptr(), stride


def sik_rope_append(layout, chunk, q, k, q_out, *, v=None, k_out=None, K=None, V=None, q_weight=None, k_weight=None,
                    eps=1e-6, inv_freq=None, interleaved=False, positions=None):
    """Per-head norms and position rotation of q, k [B,n,heads,D]; keys (and values) into the cache, or keys to k_out."""
    B, n, Hkv, Hq, D = layout.batch, chunk.n, layout.n_kv_heads, layout.n_q_heads, layout.head_dim
    dev, kd, f32 = _device(), _SIK2TORCH[layout.kv_dtype], torch.float32
    pages = _check_chunk(layout, chunk, dev)
    q_rows, k_rows = (B, n, Hq, D), (B, n, Hkv, D)
    qp, qs = _head_rows("q", q, kd, dev, q_rows)
    kp, ks = _head_rows("k", k, kd, dev, k_rows)
    vp, vs = (None, 0) if v is None else _head_rows("v", v, kd, dev, k_rows)
    cache = _cache_shape(layout, pages)
    a = RopeArgs(qp, kp, vp, qs, ks, vs, _tensor("q_weight", q_weight, f32, dev, (D,), optional=True),
                 _tensor("k_weight", k_weight, f32, dev, (D,), optional=True), eps,
                 _tensor("inv_freq", inv_freq, f32, dev, optional=True), 0 if inv_freq is None else 2 * inv_freq.numel(),
                 1 if interleaved else 0, _tensor("positions", positions, torch.int32, dev, (B, n), optional=True),
                 _tensor("q_out", q_out, kd, dev, q_rows), _tensor("k_out", k_out, kd, dev, k_rows, optional=True),
                 _tensor("K", K, kd, dev, cache, optional=True), _tensor("V", V, kd, dev, cache, optional=True),
                 _stream_of(dev))
    _check(lib().sik_rope_append(ctypes.byref(layout), ctypes.byref(chunk), ctypes.byref(a)))


def sik_chunk_workspace_bytes(layout: Layout, n: int) -> int:
    return int(lib().sik_chunk_workspace_bytes(ctypes.byref(layout), int(n)))


def alloc_chunk_workspace(layout: Layout, n: int, device="cuda") -> torch.Tensor:
    """Scratch memory of sik_chunk_attn and sik_evict for chunks of up to n tokens (needs no initialisation)."""
    size = sik_chunk_workspace_bytes(layout, n)
    if size == 0:
        raise SikError(-2, "sik_chunk_workspace_bytes rejected the layout / n")
    return torch.empty(size, dtype=torch.uint8, device=device)


def sik_chunk_attn(layout, chunk, q, K, V, softmax_scale, out, lse, workspace):
    """Attention of the chunk's queries q [B,n,Hq,D] over the cache; lse [B,n,Hq] fp32 or None."""
    dev, kd = _device(), _SIK2TORCH[layout.kv_dtype]
    rows = (layout.batch, chunk.n, layout.n_q_heads, layout.head_dim)
    cache = _cache_shape(layout, _check_chunk(layout, chunk, dev))
    _check(lib().sik_chunk_attn(
        ctypes.byref(layout), ctypes.byref(chunk), _tensor("q", q, kd, dev, rows), _tensor("K", K, kd, dev, cache),
        _tensor("V", V, kd, dev, cache), softmax_scale, _tensor("out", out, _SIK2TORCH[layout.out_dtype], dev, rows),
        _tensor("lse", lse, torch.float32, dev, rows[:3], optional=True),
        _tensor("workspace", workspace, torch.uint8, dev, optional=True),
        workspace.numel() if workspace is not None else 0, _stream_of(dev)))


def sik_attn_mass(layout, chunk, q, K, softmax_scale, lse, n_obs, before, mass):
    """Attention weight of the cached tokens from the last n_obs queries; before [B,Hkv,max_len] fp32 or None is added."""
    dev, kd, f32 = _device(), _SIK2TORCH[layout.kv_dtype], torch.float32
    rows = (layout.batch, chunk.n, layout.n_q_heads, layout.head_dim)
    sums = (layout.batch, layout.n_kv_heads, layout.max_len)
    cache = _cache_shape(layout, _check_chunk(layout, chunk, dev))
    _check(lib().sik_attn_mass(
        ctypes.byref(layout), ctypes.byref(chunk), _tensor("q", q, kd, dev, rows), _tensor("K", K, kd, dev, cache),
        softmax_scale, _tensor("lse", lse, f32, dev, rows[:3]), int(n_obs),
        _tensor("before", before, f32, dev, sums, optional=True), _tensor("mass", mass, f32, dev, sums), _stream_of(dev)))


def sik_evict(layout, mass, seq_len, n_keep, keep, workspace, *, n_sink=0, n_recent=0, new_len=None, K=None, V=None,
              pages=None, K_out=None, V_out=None, mass_out=None):
    """The n_keep tokens per (sequence, KV head) that stay, and with K_out and V_out the cache cut down to them."""
    B, H, D = layout.batch, layout.n_kv_heads, layout.head_dim
    dev, kd, f32, i32 = _device(), _SIK2TORCH[layout.kv_dtype], torch.float32, torch.int32
    n_keep = int(n_keep)
    _check_page_table(layout, pages, dev)
    out_len = K_out.shape[2] if K_out is not None else mass_out.shape[2] if mass_out is not None else 0
    cache, cut = _cache_shape(layout, pages), (B, H, out_len, D)
    a = EvictArgs(_tensor("mass", mass, f32, dev, (B, H, layout.max_len)), _tensor("seq_len", seq_len, i32, dev, numel=B),
                  n_keep, int(n_sink), int(n_recent), _tensor("keep", keep, i32, dev, (B, H, n_keep)),
                  _tensor("new_len", new_len, i32, dev, numel=B, optional=True),
                  _tensor("K", K, kd, dev, cache, optional=True), _tensor("V", V, kd, dev, cache, optional=True),
                  None if pages is None else ctypes.pointer(pages), _tensor("K_out", K_out, kd, dev, cut, optional=True),
                  _tensor("V_out", V_out, kd, dev, cut, optional=True),
                  _tensor("mass_out", mass_out, f32, dev, cut[:3], optional=True), out_len,
                  _tensor("workspace", workspace, torch.uint8, dev, optional=True),
                  workspace.numel() if workspace is not None else 0, _stream_of(dev))
    _check(lib().sik_evict(ctypes.byref(layout), ctypes.byref(a)))
