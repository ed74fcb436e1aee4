"""ctypes binding of libsjd.so: same names as include/sjd.h, argument marshalling only.

PyTorch supplies device memory and streams; every step of the decoding path runs inside the
library's CUDA kernels.  Loading fails loudly if the library has not been built
(`python -m paper_2410_01699_b200.build`); there is no fallback of any kind.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libsjd.so")

SJD_OK = 0
SJD_ERR_BAD_ARG, SJD_ERR_CAPACITY, SJD_ERR_UNSUPPORTED = -1, -2, -3
SJD_ERR_CUDA, SJD_ERR_DEVICE_TIMEOUT, SJD_ERR_STATE = -4, -5, -6
SJD_F32, SJD_BF16 = 0, 1
SJD_INIT_RANDOM, SJD_INIT_COPY_ABOVE, SJD_INIT_COPY_LEFT, SJD_INIT_RESAMPLE_LEFT, SJD_INIT_RESAMPLE_ABOVE = 0, 1, 2, 3, 4
SJD_Q_ROW, SJD_Q_UNIFORM, SJD_Q_ONEHOT, SJD_Q_RING = 0, 1, 2, 3
SJD_NORM_RMS, SJD_NORM_LAYER = 0, 1
SJD_ACT_NONE, SJD_ACT_RELU, SJD_ACT_SILU, SJD_ACT_GELU, SJD_ACT_GELU_TANH = 0, 1, 2, 3, 4
SJD_SCHEDULE_SJD, SJD_SCHEDULE_JACOBI, SJD_SCHEDULE_NO_REFINE = 0, 1, 2
SJD_FLAG_NEAR_TIE_ACCEPT, SJD_FLAG_RESIDUAL_EMPTY, SJD_FLAG_NONFINITE, SJD_FLAG_DONE = 1, 4, 8, 16

DTYPES = {"f32": SJD_F32, "bf16": SJD_BF16}
TORCH_DTYPES = {SJD_F32: torch.float32, SJD_BF16: torch.bfloat16}

EXPORTS = ["sjd_workspace_bytes", "sjd_init", "sjd_prefill", "sjd_step", "sjd_get_window", "sjd_peek_logits",
           "sjd_verify_workspace_bytes", "sjd_verify", "sjd_last_device_status", "sjd_last_cuda_error",
           "sjd_destroy", "sjd_strerror", "sjd_launch_count", "sjd_trace", "sjd_trace_read", "sjd_verify_static",
           "sjd_gemm_workspace_bytes", "sjd_gemm", "sjd_attention_workspace_bytes", "sjd_attention", "sjd_get_info",
           "sjd_prefill_ragged", "sjd_get_tokens", "sjd_pool_append", "sjd_pool_attention_workspace_bytes",
           "sjd_pool_attention", "sjd_pool_workspace_bytes", "sjd_pool_reserve", "sjd_pool_fork", "sjd_pool_free",
           "sjd_pool_compact", "sjd_block_norm", "sjd_linear",
           "sjd_pool_attention_shared_workspace_bytes", "sjd_pool_attention_shared"]
SJD_KV_PAGE, SJD_POOL_BLOCK, SJD_POOL_MAX_LIST = 64, 16, 1024


class SJDError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().sjd_strerror(status).decode()
        if status == SJD_ERR_CUDA:
            msg += " [cudaError %d]" % lib().sjd_last_cuda_error()
        super().__init__("%s: %s (%d)" % (where, msg, status))


class sjd_model_cfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "d_model", "n_heads", "n_kv_heads", "head_dim", "ffn_hidden",
                                         "vocab")] + \
               [("rope_theta", C.c_float), ("rms_eps", C.c_float), ("dtype", C.c_int32),
                ("max_batch", C.c_int32), ("max_seq", C.c_int32), ("max_window", C.c_int32), ("max_ring", C.c_int32),
                ("kv_pages", C.c_int32)]


_PP = C.POINTER(C.c_void_p)


class sjd_weights(C.Structure):
    _fields_ = [("tok_emb", C.c_void_p), ("final_norm", C.c_void_p), ("lm_head", C.c_void_p)] + \
               [(n, _PP) for n in ("attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "w_gate", "w_up", "w_down",
                                   "q_norm", "k_norm")]


class sjd_sample_cfg(C.Structure):
    _fields_ = [("temperature", C.c_float), ("top_k", C.c_int32), ("seed", C.c_uint64), ("window", C.c_int32),
                ("init", C.c_int32), ("grid_stride", C.c_int32), ("n_generate", C.c_int32), ("seq_base", C.c_int32),
                ("guidance", C.c_float), ("schedule", C.c_int32)]


class sjd_step_out(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("n_accepted", "n_committed", "committed", "draft", "q_kind", "q_draft",
                                          "total_committed", "flags")]


class sjd_info(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("tensor_core_projections", "tensor_core_attention", "step_graph",
                                         "rows_per_step")]


class sjd_pool(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("pages", "exps", "table", "refs", "status")] + \
               [(n, C.c_int32) for n in ("n_pages", "n_seqs", "pages_per_seq", "n_layers", "n_kv_heads", "head_dim")]


class sjd_rope(C.Structure):
    _fields_ = [("n_axes", C.c_int32), ("pairs", C.c_int32 * 3), ("interleaved", C.c_int32), ("per_axis", C.c_int32),
                ("theta", C.c_double)]


_lib = None


def lib():
    """The loaded library; raises if it is missing or lacks a declared symbol."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("libsjd.so is not built: run `python -m paper_2410_01699_b200.build` "
                           "(needs nvcc with sm_100a support); there is no fallback path")
    L = C.CDLL(LIB_PATH)
    for name in EXPORTS:
        if not hasattr(L, name):
            raise RuntimeError("libsjd.so does not export %s" % name)
    L.sjd_workspace_bytes.restype = C.c_size_t
    L.sjd_workspace_bytes.argtypes = [C.POINTER(sjd_model_cfg)]
    L.sjd_init.restype = C.c_int
    L.sjd_init.argtypes = [C.POINTER(C.c_void_p), C.POINTER(sjd_model_cfg), C.POINTER(sjd_weights), C.c_void_p,
                           C.c_size_t]
    L.sjd_prefill.restype = C.c_int
    L.sjd_prefill.argtypes = [C.c_void_p, C.c_int, C.c_void_p, C.c_int, C.POINTER(sjd_sample_cfg), C.c_void_p]
    L.sjd_prefill_ragged.restype = C.c_int
    L.sjd_prefill_ragged.argtypes = [C.c_void_p, C.c_int, C.c_void_p, C.POINTER(C.c_int32), C.c_int,
                                     C.POINTER(sjd_sample_cfg), C.c_void_p]
    L.sjd_step.restype = C.c_int
    L.sjd_step.argtypes = [C.c_void_p, C.POINTER(sjd_step_out), C.c_void_p]
    L.sjd_get_tokens.restype = C.c_int
    L.sjd_get_tokens.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p]
    L.sjd_get_window.restype = C.c_int
    L.sjd_get_window.argtypes = [C.c_void_p, C.POINTER(sjd_step_out), C.c_void_p]
    L.sjd_peek_logits.restype = C.c_int
    L.sjd_peek_logits.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    L.sjd_verify_workspace_bytes.restype = C.c_size_t
    L.sjd_verify_workspace_bytes.argtypes = [C.c_int, C.c_int]
    L.sjd_verify.restype = C.c_int
    L.sjd_verify.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                             C.c_void_p, C.POINTER(sjd_sample_cfg), C.c_uint32, C.POINTER(sjd_step_out), C.c_void_p,
                             C.c_size_t, C.c_void_p]
    L.sjd_verify_static.restype = C.c_int
    L.sjd_verify_static.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                    C.c_void_p, C.POINTER(sjd_sample_cfg), C.c_uint32, C.POINTER(sjd_step_out),
                                    C.c_void_p]
    L.sjd_gemm_workspace_bytes.restype = C.c_size_t
    L.sjd_gemm_workspace_bytes.argtypes = [C.c_int, C.c_int, C.c_int]
    L.sjd_gemm.restype = C.c_int
    L.sjd_gemm.argtypes = [C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p,
                           C.c_size_t, C.c_void_p]
    L.sjd_attention_workspace_bytes.restype = C.c_size_t
    L.sjd_attention_workspace_bytes.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int]
    L.sjd_attention.restype = C.c_int
    L.sjd_attention.argtypes = [C.c_int] * 6 + [C.c_void_p] * 5 + [C.c_size_t, C.c_void_p]
    _pool, _i64 = C.POINTER(sjd_pool), C.c_int64
    L.sjd_linear.restype = C.c_int
    L.sjd_linear.argtypes = [C.c_int] * 3 + [C.c_void_p, _i64, C.c_void_p, C.c_void_p, _i64, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, _i64,
                                             C.c_void_p, _i64, C.c_void_p, C.c_void_p]
    L.sjd_block_norm.restype = C.c_int
    L.sjd_block_norm.argtypes = [C.c_int, C.c_int, C.c_int, C.c_float, C.c_int, C.c_int, C.c_void_p, _i64, C.c_void_p, _i64, C.c_void_p,
                                 C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_float, C.c_void_p, _i64, C.c_void_p, C.c_void_p,
                                 C.c_void_p, _i64, C.c_void_p]
    L.sjd_pool_append.restype = C.c_int
    L.sjd_pool_append.argtypes = [_pool] + [C.c_int] * 5 + [C.c_void_p, _i64] * 3 + \
        [C.c_void_p, C.c_void_p, C.POINTER(sjd_rope), C.c_void_p, C.c_void_p, _i64, C.c_void_p]
    L.sjd_pool_attention_workspace_bytes.restype = C.c_size_t
    L.sjd_pool_attention_workspace_bytes.argtypes = [_pool, C.c_int, C.c_int]
    L.sjd_pool_attention.restype = C.c_int
    L.sjd_pool_attention.argtypes = [_pool] + [C.c_int] * 5 + [C.c_void_p, _i64, C.c_void_p, C.c_void_p, C.c_int, C.c_int,
                                                               C.c_float, C.c_void_p, _i64, C.c_void_p, C.c_size_t, C.c_void_p]
    L.sjd_pool_attention_shared_workspace_bytes.restype = C.c_size_t
    L.sjd_pool_attention_shared_workspace_bytes.argtypes = [_pool, C.c_int, C.c_int, C.c_int]
    L.sjd_pool_attention_shared.restype = C.c_int
    L.sjd_pool_attention_shared.argtypes = [_pool] + [C.c_int] * 5 + [C.c_void_p, _i64, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_float,
                                                                      C.c_void_p, _i64, C.c_void_p, C.c_size_t, C.c_void_p]
    L.sjd_pool_workspace_bytes.restype = C.c_size_t
    L.sjd_pool_workspace_bytes.argtypes = [_pool]
    L.sjd_pool_reserve.restype = C.c_int
    L.sjd_pool_reserve.argtypes = [_pool, C.c_int] + [C.c_void_p] * 4 + [C.c_size_t, C.c_void_p]
    L.sjd_pool_fork.restype = C.c_int
    L.sjd_pool_fork.argtypes = [_pool, C.c_int] + [C.c_void_p] * 4
    L.sjd_pool_free.restype = C.c_int
    L.sjd_pool_free.argtypes = [_pool, C.c_int] + [C.c_void_p] * 3
    L.sjd_pool_compact.restype = C.c_int
    L.sjd_pool_compact.argtypes = [_pool, C.c_void_p, C.c_size_t, C.c_void_p]
    L.sjd_get_info.restype = C.c_int
    L.sjd_get_info.argtypes = [C.c_void_p, C.POINTER(sjd_info)]
    L.sjd_last_device_status.restype = C.c_int
    L.sjd_last_device_status.argtypes = [C.c_void_p]
    L.sjd_last_cuda_error.restype = C.c_int
    L.sjd_launch_count.restype = C.c_int64
    L.sjd_trace.restype = C.c_int
    L.sjd_trace.argtypes = [C.c_void_p, C.c_int]
    L.sjd_trace_read.restype = C.c_int
    L.sjd_trace_read.argtypes = [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_int64), C.POINTER(C.c_double)]
    L.sjd_destroy.restype = None
    L.sjd_destroy.argtypes = [C.c_void_p]
    L.sjd_strerror.restype = C.c_char_p
    L.sjd_strerror.argtypes = [C.c_int]
    _lib = L
    return L


def _check(status: int, where: str):
    if status != SJD_OK:
        raise SJDError(status, where)


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def make_model_cfg(wl, max_batch: int, max_seq: int, max_window: int, max_ring: int = 0,
                   kv_pages: int = 0) -> sjd_model_cfg:
    """wl: anything with the model fields of inputs.Workload."""
    return sjd_model_cfg(wl.n_layers, wl.d_model, wl.n_heads, wl.n_kv_heads, wl.head_dim, wl.ffn_hidden, wl.vocab,
                         wl.rope_theta, wl.rms_eps, DTYPES[wl.dtype], max_batch, max_seq, max_window, max_ring, kv_pages)


def make_sample_cfg(temperature=1.0, top_k=2000, seed=0, window=16, init=SJD_INIT_RANDOM, grid_stride=0,
                    n_generate=0, seq_base=0, guidance=0.0, schedule=0) -> sjd_sample_cfg:
    return sjd_sample_cfg(float(temperature), int(top_k), int(seed), int(window), int(init), int(grid_stride),
                          int(n_generate), int(seq_base), float(guidance), int(schedule))


class StepOut:
    """Caller-owned result buffers of one step (device tensors, or pinned host tensors)."""

    def __init__(self, batch: int, window: int, device="cuda", pinned: bool = False):
        kw = dict(device="cpu", pin_memory=True) if pinned else dict(device=device)
        i32 = lambda *s: torch.full(s, -7, dtype=torch.int32, **kw)
        self.n_accepted, self.n_committed = i32(batch), i32(batch)
        self.committed, self.draft, self.q_kind = i32(batch, window), i32(batch, window), i32(batch, window)
        self.q_draft = torch.zeros(batch, window, dtype=torch.float32, **kw)
        self.total_committed, self.flags = i32(batch), i32(batch)
        self.c = sjd_step_out(*[C.c_void_p(t.data_ptr()) for t in (
            self.n_accepted, self.n_committed, self.committed, self.draft, self.q_kind, self.q_draft,
            self.total_committed, self.flags)])

    def host(self):
        """dict of numpy copies (synchronises the current stream)."""
        torch.cuda.current_stream().synchronize()
        names = ("n_accepted", "n_committed", "committed", "draft", "q_kind", "q_draft", "total_committed", "flags")
        return {n: getattr(self, n).cpu().numpy().copy() for n in names}


def sjd_workspace_bytes(cfg: sjd_model_cfg) -> int:
    return int(lib().sjd_workspace_bytes(C.byref(cfg)))


def sjd_verify_workspace_bytes(batch: int, window: int) -> int:
    return int(lib().sjd_verify_workspace_bytes(batch, window))


def sjd_verify(logits_cur, logits_prev, draft, q_kind, base_pos, sample: sjd_sample_cfg, step: int, out: StepOut,
               ws=None):
    """Isolated verification (Eqs. 1-3).  logits_*: [B][W][V] cuda tensors (float32 or bfloat16)."""
    b, w, v = logits_cur.shape
    dt = {torch.float32: SJD_F32, torch.bfloat16: SJD_BF16}[logits_cur.dtype]
    if ws is None:
        ws = torch.empty(sjd_verify_workspace_bytes(b, w), dtype=torch.uint8, device=logits_cur.device)
    st = lib().sjd_verify(b, w, v, dt, _ptr(logits_cur), _ptr(logits_prev), _ptr(draft), _ptr(q_kind), _ptr(base_pos),
                          C.byref(sample), C.c_uint32(step), C.byref(out.c), _ptr(ws), ws.numel(), _stream())
    _check(st, "sjd_verify")
    return ws


SJD_VERIFY_STATIC_MAX_ROWS, SJD_VERIFY_STATIC_MAX_BATCH = 2048, 256


def sjd_verify_static(logits_cur, logits_prev, draft, q_kind, base_pos, sample: sjd_sample_cfg, step: int,
                      out: StepOut):
    """sjd_verify for callers that cannot allocate: no scratch argument, the library's built-in
    scratch array is used (batch * window <= SJD_VERIFY_STATIC_MAX_ROWS).  Calls on one device must
    not overlap; make the first call on a device outside any stream capture."""
    b, w, v = logits_cur.shape
    dt = {torch.float32: SJD_F32, torch.bfloat16: SJD_BF16}[logits_cur.dtype]
    st = lib().sjd_verify_static(b, w, v, dt, _ptr(logits_cur), _ptr(logits_prev), _ptr(draft), _ptr(q_kind),
                                 _ptr(base_pos), C.byref(sample), C.c_uint32(step), C.byref(out.c), _stream())
    _check(st, "sjd_verify_static")


def sjd_gemm(x, w, out=None, accumulate=False):
    """out[M][N] (+)= x[M][K] @ w[N][K]^T on the tensor-core weight-streaming kernel.
    x: float32 cuda, w: bfloat16 cuda.  Returns (out, status word tensor)."""
    m, k = x.shape
    n = w.shape[0]
    if out is None:
        out = (torch.zeros if accumulate else torch.empty)(m, n, dtype=torch.float32, device=x.device)
    nbytes = int(lib().sjd_gemm_workspace_bytes(m, n, k))
    if nbytes == 0:
        raise SJDError(SJD_ERR_UNSUPPORTED, "sjd_gemm_workspace_bytes")
    ws = torch.empty(nbytes, dtype=torch.uint8, device=x.device)
    _check(lib().sjd_gemm(m, n, k, _ptr(x), _ptr(w), _ptr(out), 1 if accumulate else 0, _ptr(ws), nbytes, _stream()),
           "sjd_gemm")
    return out, ws[:4].view(torch.int32)


def sjd_attention(q, kv_cache, in_pos, window, n_kv_heads, out=None, ws=None):
    """Window-causal attention on the tensor-core kernel.  q: float32 cuda [B*W][H][hd]; kv_cache:
    bfloat16 cuda [B][2][KVh][max_seq][hd]; in_pos: int32 cuda [B*W].  Returns (out, status word)."""
    m, h, hd = q.shape
    b, max_seq = kv_cache.shape[0], kv_cache.shape[3]
    if out is None:
        out = torch.empty_like(q)
    nbytes = int(lib().sjd_attention_workspace_bytes(b, window, h, hd))
    if nbytes == 0:
        raise SJDError(SJD_ERR_UNSUPPORTED, "sjd_attention_workspace_bytes")
    if ws is None:
        ws = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
    _check(lib().sjd_attention(b, window, h, n_kv_heads, hd, max_seq, _ptr(q), _ptr(kv_cache), _ptr(in_pos), _ptr(out),
                               _ptr(ws), nbytes, _stream()), "sjd_attention")
    return out, ws[:4].view(torch.int32)


class CachePool:
    """A paged cache in 8 bits (see sjd_pool in include/sjd.h) on borrowed torch tensors of one cuda device:

      pages  float8_e4m3fn [n_pages][n_layers][2][n_kv_heads][64][head_dim]    exps  int8 [n_pages][n_layers][2][n_kv_heads][4]
      table  int32 [n_seqs][pages_per_seq], -1: none                           refs  int32 [n_pages], table entries per page

    `status` (int32 [1], zero at the start) keeps the first fault that a kernel found until `clear()`; `ws` and the workspaces
    of attention() are the pool's own, so that calls on one pool follow one another (one stream, or ordered by the caller)."""

    def __init__(self, pages, exps, table, refs):
        n_pages, n_layers, two, n_kv_heads, rows, head_dim = pages.shape
        want = (n_pages, n_layers, 2, n_kv_heads, SJD_KV_PAGE // SJD_POOL_BLOCK)
        if two != 2 or rows != SJD_KV_PAGE or tuple(exps.shape) != want or tuple(refs.shape) != (n_pages,) or table.dim() != 2:
            raise ValueError("shapes of a pool do not fit together")
        for x, dt in ((pages, torch.float8_e4m3fn), (exps, torch.int8), (table, torch.int32), (refs, torch.int32)):
            if x.dtype != dt or not x.is_contiguous() or x.device != pages.device:
                raise ValueError("a pool's tensors are contiguous, on one device, of types e4m3, int8, int32 and int32")
        self.pages, self.exps, self.table, self.refs = pages, exps, table, refs
        self.device, self.index = pages.device, pages.get_device()   # (-1: on the host, where nothing can be launched)
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self.c = sjd_pool(pages.data_ptr(), exps.data_ptr(), table.data_ptr(), refs.data_ptr(), self.status.data_ptr(), n_pages,
                          table.shape[0], table.shape[1], n_layers, n_kv_heads, head_dim)
        self.n_kv_heads, self.head_dim = n_kv_heads, head_dim
        self.ref = C.byref(self.c)
        self.ws_bytes = int(lib().sjd_pool_workspace_bytes(self.ref))
        if self.ws_bytes == 0:
            raise SJDError(SJD_ERR_UNSUPPORTED, "sjd_pool_workspace_bytes")
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=self.device)
        self.ws_at = self.ws.data_ptr()
        self._attention_ws = None
        self._shared_ws, self._shared_bytes = [], {}

    @classmethod
    def empty(cls, n_pages, n_seqs, pages_per_seq, n_layers, n_kv_heads, head_dim, device="cuda"):
        """A pool of its own tensors, no page in use."""
        return cls(torch.zeros(n_pages, n_layers, 2, n_kv_heads, SJD_KV_PAGE, head_dim, dtype=torch.float8_e4m3fn, device=device),
                   torch.zeros(n_pages, n_layers, 2, n_kv_heads, SJD_KV_PAGE // SJD_POOL_BLOCK, dtype=torch.int8, device=device),
                   torch.full((n_seqs, pages_per_seq), -1, dtype=torch.int32, device=device),
                   torch.zeros(n_pages, dtype=torch.int32, device=device))

    def attention_ws(self):
        """The pool's workspace for attention calls, large enough for all of them (a captured graph keeps its address)."""
        if self._attention_ws is None:
            nbytes = int(lib().sjd_pool_attention_workspace_bytes(self.ref, 64, self.n_kv_heads))   # (tiles have at most 64 rows)
            self._attention_ws = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        return self._attention_ws

    def shared_ws(self, batch, window, heads):
        """The pool's workspace for attention over shared pages: the last of those so far if it is large enough for such a call, else another
        one (the others stay: a captured graph keeps the address that it was given).  Each is at least twice the one before, so that all of them
        are less than four times what the largest call needs."""
        nbytes = self._shared_bytes.get((batch, window, heads))
        if nbytes is None:
            nbytes = int(lib().sjd_pool_attention_shared_workspace_bytes(self.ref, batch, window, heads))
            self._shared_bytes[batch, window, heads] = nbytes
        have = self._shared_ws[-1].nbytes if self._shared_ws else 0
        if have < max(nbytes, 1):
            self._shared_ws.append(torch.empty(max(nbytes, 2 * have, 1), dtype=torch.uint8, device=self.device))
        return self._shared_ws[-1]

    def fault(self) -> int:
        """The first fault that a kernel found since the start or clear() (an SJD_ERR_* value, 0: none).  Synchronises."""
        return int(self.status.item())

    def clear(self):
        self.status.zero_()


def make_rope_cfg(pairs, theta=10000.0, interleaved=False, per_axis=False) -> sjd_rope:
    """pairs: pairs of each axis, one to three of them (they add up to head_dim / 2)."""
    pairs = [int(x) for x in pairs]
    if not 1 <= len(pairs) <= 3:
        raise ValueError("one to three axes")
    return sjd_rope(len(pairs), (C.c_int32 * 3)(*(pairs + [0] * (3 - len(pairs)))), int(bool(interleaved)), int(bool(per_axis)),
                    float(theta))


# These calls are made once or more a layer and can be shorter on the device than in here: pointers go as plain integers, the device is
# switched only where it is another one than the current, and the stream is asked for without making an object of it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _pool_call(pool, where, function, *args):
    """function(pool, *args, stream) on the pool's device and its current stream."""
    if pool.index < 0:
        raise ValueError("%s: a pool on the host" % where)
    _call_on(pool.index, where, function, pool.ref, *args)


def _call_on(index, where, function, *args):
    """function(*args, stream) on device `index` and its current stream."""
    if torch.cuda.current_device() == index:
        status = function(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            status = function(*args, _raw_stream(index))
    if status != SJD_OK:
        raise SJDError(status, where)


def _rows(x, rows, d, dtype, index, where):
    """(address, row stride) of x [rows][d] of `dtype` on device `index`; entries of a row are contiguous."""
    stride = x.stride()
    if x.dtype is not dtype or x.get_device() != index or x.shape != (rows, d) or (stride[1] != 1 and d > 1) or (stride[0] < d and rows > 1):
        raise ValueError("%s: [%d][%d] of %s on the device of the other tensors, entries of a row contiguous" % (where, rows, d, dtype))
    return x.data_ptr(), stride[0] if rows > 1 else d


def _vector(x, d, dtype, index, where):
    """Address of d contiguous entries of `dtype` on device `index`; None for None."""
    if x is None:
        return None
    if x.dtype is not dtype or x.get_device() != index or x.numel() != d or not x.is_contiguous():
        raise ValueError("%s: %d contiguous entries of %s on the device of the other tensors" % (where, d, dtype))
    return x.data_ptr()


def sjd_block_norm(h, y=None, post_gain=None, post_bias=None, gate=None, gate_tanh=False, scale=1.0, pre_gain=None, pre_bias=None,
                   kind=SJD_NORM_RMS, eps=1e-5, h_out=None, z=None):
    """(h + scale * gate * N(y), the norm of that): a block's output y [M][d], normed (post_gain) and gated, goes to the residual stream h
    [M][d], and what the next block reads is its norm (pre_gain).  What is None is left out (see sjd_block_norm in include/sjd.h); without
    y the norm of h alone.  gate [G][d], one row for each M / G rows; y, gains, biases, gate and z are of one type, h and h_out of one.
    Returns (h_out, z), new tensors unless given; None for what is not asked for."""
    index, kin = h.get_device(), y if y is not None else pre_gain
    if index < 0 or h.dim() != 2:
        raise ValueError("sjd_block_norm: h [M][d] on a cuda device")
    if kin is None or (y is None and h_out is not None) or (pre_gain is None and z is not None):
        raise ValueError("sjd_block_norm: y, pre_gain or both, and outputs of what is asked for")
    m, d = h.shape
    t, ht = kin.dtype, h.dtype
    dtype, h_dtype = _pool_dtype(kin, "sjd_block_norm"), _pool_dtype(h, "sjd_block_norm")
    h_at, h_stride = _rows(h, m, d, ht, index, "h")
    y_at, y_stride, out_at, out_stride, z_at, z_stride, gate_at, gate_rows = None, 0, None, 0, None, 0, None, 0
    if y is not None:
        y_at, y_stride = _rows(y, m, d, t, index, "y")
        if h_out is None:
            h_out = torch.empty_like(h, memory_format=torch.contiguous_format)
        out_at, out_stride = _rows(h_out, m, d, ht, index, "h_out")
    if pre_gain is not None:
        if z is None:
            z = torch.empty((m, d), dtype=t, device=h.device)
        z_at, z_stride = _rows(z, m, d, t, index, "z")
    if gate is not None:
        if gate.dim() != 2 or gate.shape[0] < 1 or m % gate.shape[0] != 0:
            raise ValueError("gate: [G][%d], G a divisor of the rows" % d)
        gate_at, gate_rows = _vector(gate, gate.shape[0] * d, t, index, "gate"), max(1, m // gate.shape[0])
    _call_on(index, "sjd_block_norm", lib().sjd_block_norm, m, d, kind, eps, dtype, h_dtype, h_at, h_stride, y_at, y_stride,
             _vector(post_gain, d, t, index, "post_gain"), _vector(post_bias, d, t, index, "post_bias"), gate_at, gate_rows, gate_tanh, scale,
             out_at, out_stride, _vector(pre_gain, d, t, index, "pre_gain"), _vector(pre_bias, d, t, index, "pre_bias"), z_at, z_stride)
    return h_out, z


def sjd_linear(x, w, w_up=None, bias=None, bias_up=None, act=SJD_ACT_NONE, residual=None, out=None, status=None):
    """residual + act(x w^T + bias) * (x w_up^T + bias_up) of bf16 cuda tensors: x [M][K], w and w_up [N][K], biases [N], residual and out
    [M][N]; what is None is left out (see sjd_linear in include/sjd.h).  Rows may be parts of longer ones; those of x, w and w_up start on
    16 bytes.  status: an int32 tensor in which a kernel leaves SJD_ERR_DEVICE_TIMEOUT if a wait ran out.  Returns out."""
    index = x.get_device()
    if index < 0 or x.dim() != 2 or w.dim() != 2:
        raise ValueError("sjd_linear: x [M][K] and w [N][K] on a cuda device")
    m, k = x.shape
    n = w.shape[0]
    bf16 = torch.bfloat16
    if x.dtype is not bf16:
        raise SJDError(SJD_ERR_UNSUPPORTED, "sjd_linear")
    x_at, x_stride = _rows(x, m, k, bf16, index, "x")
    w_at, w_stride = _rows(w, n, k, bf16, index, "w")
    up_at, r_at, r_stride = None, None, 0
    if w_up is not None:
        up_at, up_stride = _rows(w_up, n, k, bf16, index, "w_up")
        if up_stride != w_stride:
            raise ValueError("w_up: rows as far apart as those of w")
    if residual is not None:
        r_at, r_stride = _rows(residual, m, n, bf16, index, "residual")
    if out is None:
        out = torch.empty((m, n), dtype=bf16, device=x.device)
    out_at, out_stride = _rows(out, m, n, bf16, index, "out")
    if status is not None and (status.dtype is not torch.int32 or status.get_device() != index or status.numel() < 1):
        raise ValueError("status: int32 on the device of the other tensors")
    _call_on(index, "sjd_linear", lib().sjd_linear, m, n, k, x_at, x_stride, w_at, up_at, w_stride, _vector(bias, n, bf16, index, "bias"),
             _vector(bias_up, n, bf16, index, "bias_up"), act, r_at, r_stride, out_at, out_stride, None if status is None else status.data_ptr())
    return out


def _pool_rows(x, heads, pool, rows, where):
    """Row stride of x [rows][heads][head_dim], whose rows may be parts of longer ones."""
    hd, stride = pool.head_dim, x.stride()
    if x.shape != (rows, heads, hd) or stride[2] != 1 or (heads > 1 and stride[1] != hd):
        raise ValueError("%s: a tensor [%d][%d][%d] whose rows are contiguous" % (where, rows, heads, hd))
    if x.get_device() != pool.index:
        raise ValueError("%s: on another device than the pool" % where)
    return stride[0] if rows > 1 else heads * hd


def _ints(x, n, pool, where):
    """Address of n int32 entries on the pool's device; None for None."""
    if x is None:
        return None
    if x.dtype is not torch.int32 or x.numel() != n or not x.is_contiguous() or x.get_device() != pool.index:
        raise ValueError("%s: %d contiguous int32 entries on the pool's device" % (where, n))
    return x.data_ptr()


def _pool_dtype(x, where):
    if x.dtype is torch.float32:
        return SJD_F32
    if x.dtype is torch.bfloat16:
        return SJD_BF16
    raise SJDError(SJD_ERR_UNSUPPORTED, where)


def sjd_pool_append(pool: CachePool, layer: int, k, v, in_pos, window: int, q=None, q_out=None, rope: sjd_rope | None = None,
                    axis_pos=None, seqs=None):
    """Rotates q and k, appends k and v to the pool; returns the rotated q (q_out, which may be q; a new tensor if not given).
    q [B*W][H][hd], k, v [B*W][KVh][hd] of one type, float32 or bfloat16, possibly parts of one matrix; in_pos int32 [B*W];
    axis_pos int32 [B*W][n_axes]; seqs int32 [B] or None (sequence b is row b of the table)."""
    m, kvh = in_pos.numel(), pool.n_kv_heads
    dtype = _pool_dtype(k, "sjd_pool_append")
    if window < 1 or m % window != 0 or v.dtype != k.dtype or (q is not None and q.dtype != k.dtype):
        raise ValueError("sjd_pool_append: whole windows, and q, k, v of one type")
    heads, q_at, q_stride, out_at, out_stride = 0, None, 0, None, 0
    if q is not None:
        heads = q.shape[1]
        q_at, q_stride = q.data_ptr(), _pool_rows(q, heads, pool, m, "q")
        if q_out is None:
            q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
        if q_out.dtype != q.dtype:
            raise ValueError("q_out: of q's type")
        out_at, out_stride = q_out.data_ptr(), _pool_rows(q_out, heads, pool, m, "q_out")
    if axis_pos is not None and rope is None:
        raise ValueError("axis_pos without rope")
    _pool_call(pool, "sjd_pool_append", lib().sjd_pool_append, layer, m // window, window, heads, dtype, q_at, q_stride, k.data_ptr(),
               _pool_rows(k, kvh, pool, m, "k"), v.data_ptr(), _pool_rows(v, kvh, pool, m, "v"), _ints(seqs, m // window, pool, "seqs"),
               _ints(in_pos, m, pool, "in_pos"), C.byref(rope) if rope is not None else None,
               _ints(axis_pos, m * (rope.n_axes if rope is not None else 0), pool, "axis_pos"), out_at, out_stride)
    return q_out


def sjd_pool_attention(pool: CachePool, layer: int, q, in_pos, window: int, sliding=0, sinks=0, scale=0.0, out=None, ws=None, seqs=None):
    """Attention of q [B*W][H][hd] (float32 or bfloat16) at positions in_pos over the pool; out of q's type.  ws: a workspace of
    its own for calls that may run at the same time as others on the pool (default: the pool's)."""
    m, heads = in_pos.numel(), q.shape[1]
    dtype = _pool_dtype(q, "sjd_pool_attention")
    if window < 1 or m % window != 0:
        raise ValueError("sjd_pool_attention: whole windows")
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    if out.dtype != q.dtype:
        raise ValueError("out: of q's type")
    if ws is None:
        ws = pool.attention_ws()
    elif ws.get_device() != pool.index or not ws.is_contiguous():
        raise ValueError("ws: contiguous, on the pool's device")
    _pool_call(pool, "sjd_pool_attention", lib().sjd_pool_attention, layer, m // window, window, heads, dtype, q.data_ptr(),
               _pool_rows(q, heads, pool, m, "q"), _ints(seqs, m // window, pool, "seqs"), _ints(in_pos, m, pool, "in_pos"), sliding, sinks,
               scale, out.data_ptr(), _pool_rows(out, heads, pool, m, "out"), ws.data_ptr(), ws.nbytes)
    return out


def sjd_pool_attention_shared(pool: CachePool, layer: int, q, in_pos, window: int, group_begin=None, scale=0.0, out=None, ws=None, seqs=None):
    """Attention of q [B*W][H][hd] (bfloat16) at positions in_pos over the pool, where the sequences group_begin[g] .. group_begin[g + 1] - 1
    of the call (int32, rising from 0 to B; None: all are one group) may share the pages that their tables begin with: those are attended once
    for all rows of the group.  ws: as for sjd_pool_attention."""
    m, heads = in_pos.numel(), q.shape[1]
    if q.dtype is not torch.bfloat16:
        raise SJDError(SJD_ERR_UNSUPPORTED, "sjd_pool_attention_shared")
    if window < 1 or m % window != 0:
        raise ValueError("sjd_pool_attention_shared: whole windows")
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    if out.dtype != q.dtype:
        raise ValueError("out: of q's type")
    if ws is None:
        ws = pool.shared_ws(m // window, window, heads)
    elif ws.get_device() != pool.index or not ws.is_contiguous():
        raise ValueError("ws: contiguous, on the pool's device")
    groups = group_begin.numel() - 1 if group_begin is not None else 1
    if groups < 1:
        raise ValueError("group_begin: one entry more than groups")
    _pool_call(pool, "sjd_pool_attention_shared", lib().sjd_pool_attention_shared, layer, m // window, window, heads, SJD_BF16, q.data_ptr(),
               _pool_rows(q, heads, pool, m, "q"), _ints(seqs, m // window, pool, "seqs"), _ints(in_pos, m, pool, "in_pos"), groups,
               _ints(group_begin, groups + 1, pool, "group_begin"), scale, out.data_ptr(), _pool_rows(out, heads, pool, m, "out"), ws.data_ptr(),
               ws.nbytes)
    return out


def sjd_pool_reserve(pool: CachePool, seqs, begin, end):
    """Own pages for positions begin[i] .. end[i] - 1 of sequence seqs[i] (int32 cuda tensors)."""
    n = seqs.numel()
    _pool_call(pool, "sjd_pool_reserve", lib().sjd_pool_reserve, n, _ints(seqs, n, pool, "seqs"), _ints(begin, n, pool, "begin"),
               _ints(end, n, pool, "end"), pool.ws_at, pool.ws_bytes)


def sjd_pool_fork(pool: CachePool, src, dst, length):
    """The empty sequence dst[i] shares the pages of the first length[i] positions of src[i] (int32 cuda tensors)."""
    n = src.numel()
    _pool_call(pool, "sjd_pool_fork", lib().sjd_pool_fork, n, _ints(src, n, pool, "src"), _ints(dst, n, pool, "dst"),
               _ints(length, n, pool, "length"))


def sjd_pool_free(pool: CachePool, seqs, keep):
    """Sequence seqs[i] gives back the pages behind its first keep[i] positions (int32 cuda tensors)."""
    n = seqs.numel()
    _pool_call(pool, "sjd_pool_free", lib().sjd_pool_free, n, _ints(seqs, n, pool, "seqs"), _ints(keep, n, pool, "keep"))


def sjd_pool_compact(pool: CachePool):
    """Moves pages so that those in use are the first ones of the pool."""
    _pool_call(pool, "sjd_pool_compact", lib().sjd_pool_compact, pool.ws_at, pool.ws_bytes)


class Context:
    """sjd_init / sjd_prefill / sjd_step on borrowed torch tensors."""

    def __init__(self, cfg: sjd_model_cfg, weights: dict, device="cuda"):
        self.cfg = cfg
        self.device = torch.device(device)
        self.weights = weights  # keep the tensors alive: the library borrows them
        nbytes = sjd_workspace_bytes(cfg)
        if nbytes == 0:
            raise SJDError(SJD_ERR_BAD_ARG, "sjd_workspace_bytes")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        n_layers = cfg.n_layers
        self._arrays = {}
        w = sjd_weights()
        w.tok_emb, w.final_norm, w.lm_head = (weights[k].data_ptr() for k in ("tok_emb", "final_norm", "lm_head"))
        names = ["attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "w_gate", "w_up", "w_down"]
        if n_layers and "q_norm" in weights["layers"][0]:   # QK-norm variant
            names += ["q_norm", "k_norm"]
        for name in names:
            arr = (C.c_void_p * n_layers)(*[weights["layers"][l][name].data_ptr() for l in range(n_layers)])
            self._arrays[name] = arr
            setattr(w, name, C.cast(arr, _PP))
        self._w = w
        self._ctx = C.c_void_p()
        _check(lib().sjd_init(C.byref(self._ctx), C.byref(cfg), C.byref(w), _ptr(self.workspace), nbytes), "sjd_init")
        self.batch = self.window = 0
        self._guided = False

    def prefill(self, prompt, sample: sjd_sample_cfg):
        """prompt: int32 cuda tensor [B][P]."""
        assert prompt.dtype == torch.int32 and prompt.is_cuda and prompt.is_contiguous()
        _check(lib().sjd_prefill(self._ctx, int(prompt.shape[0]), _ptr(prompt), int(prompt.shape[1]), C.byref(sample),
                                 _stream()), "sjd_prefill")
        self._prefilled(prompt, sample)

    def prefill_ragged(self, prompt, prompt_lens, sample: sjd_sample_cfg):
        """prompt: int32 cuda tensor [B][row_stride]; prompt_lens: B host integers (sequence b uses the first
        prompt_lens[b] tokens of its row)."""
        assert prompt.dtype == torch.int32 and prompt.is_cuda and prompt.is_contiguous()
        batch = int(prompt.shape[0])
        lens = (C.c_int32 * batch)(*[int(x) for x in prompt_lens])
        _check(lib().sjd_prefill_ragged(self._ctx, batch, _ptr(prompt), lens, int(prompt.shape[1]), C.byref(sample),
                                        _stream()), "sjd_prefill_ragged")
        self._prefilled(prompt, sample)

    def _prefilled(self, prompt, sample):   # (a refused call changes nothing: the generation under way can go on)
        self._prompt = prompt
        self.batch, self.window = int(prompt.shape[0]), int(sample.window)
        self._guided = float(sample.guidance) != 0.0

    def step(self, out: StepOut | None = None):
        _check(lib().sjd_step(self._ctx, C.byref(out.c) if out is not None else None, _stream()), "sjd_step")

    def get_window(self, out: StepOut):
        _check(lib().sjd_get_window(self._ctx, C.byref(out.c), _stream()), "sjd_get_window")

    def get_tokens(self, row_stride: int | None = None):
        """(tokens int32 [images][row_stride], counts int32 [images]) on the device: every image's prompt and the
        tokens fixed so far; see sjd_get_tokens."""
        images = self.batch // 2 if self._guided else self.batch
        row_stride = int(row_stride or self.cfg.max_seq)
        tokens = torch.zeros(images, row_stride, dtype=torch.int32, device=self.device)
        counts = torch.zeros(images, dtype=torch.int32, device=self.device)
        _check(lib().sjd_get_tokens(self._ctx, _ptr(tokens), row_stride, _ptr(counts), _stream()), "sjd_get_tokens")
        return tokens, counts

    def peek_logits(self):
        t = torch.empty(self.batch, self.window, self.cfg.vocab, dtype=TORCH_DTYPES[self.cfg.dtype], device=self.device)
        _check(lib().sjd_peek_logits(self._ctx, _ptr(t), t.numel() * t.element_size(), _stream()), "sjd_peek_logits")
        return t

    def trace(self, enable: bool):
        _check(lib().sjd_trace(self._ctx, 1 if enable else 0), "sjd_trace")

    def trace_read(self):
        """{'ms': {class: ms}, 'launches': {class: n}, 'gemm_weight_bytes': float}"""
        ms, n, wb = (C.c_double * 4)(), (C.c_int64 * 4)(), C.c_double()
        _check(lib().sjd_trace_read(self._ctx, ms, n, C.byref(wb)), "sjd_trace_read")
        names = ("gemm", "attention", "verify", "other")
        return {"ms": dict(zip(names, list(ms))), "launches": dict(zip(names, list(n))),
                "gemm_weight_bytes": float(wb.value)}

    def info(self) -> dict:
        """Which kernels the steps of this (pre-filled) context run; see sjd_get_info."""
        i = sjd_info()
        _check(lib().sjd_get_info(self._ctx, C.byref(i)), "sjd_get_info")
        return {n: int(getattr(i, n)) for n, _ in sjd_info._fields_}

    def device_status(self) -> int:
        return int(lib().sjd_last_device_status(self._ctx))

    def close(self):
        if self._ctx:
            lib().sjd_destroy(self._ctx)
            self._ctx = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def sjd_launch_count() -> int:
    return int(lib().sjd_launch_count())


def weights_to_device(weights: dict, device="cuda") -> dict:
    out = {k: v.to(device).contiguous() for k, v in weights.items() if k != "layers"}
    out["layers"] = [{k: v.to(device).contiguous() for k, v in lw.items()} for lw in weights["layers"]]
    return out
