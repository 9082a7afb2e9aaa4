"""ctypes binding of libctx_decode_attn.so: argument marshalling only.

Every step of the attention runs in the library's HIP kernels; PyTorch only
provides device memory and the stream.  There is no fallback: if the library
is missing, loading fails with an error that says how to build it.
"""
from __future__ import annotations

import contextlib
import ctypes
import os

from .build import LIB

CTX_OK = 0
CTX_ERR_INVALID_ARG = -1
CTX_ERR_UNSUPPORTED = -2
CTX_ERR_CAPACITY = -3
CTX_ERR_ALIGNMENT = -4
CTX_ERR_HIP = -5
CTX_ERR_OOM = -6

CTX_DTYPE_BF16 = 0
CTX_DTYPE_F32 = 1

HEAD_DIM = 128
CTX_ROTARY_INTERLEAVED = 1  # ctx_rotary flag: pairs of neighbouring dimensions
CTX_PREFILL_SPLIT_P = 1  # ctx_prefill_attn_run flag: softmax weights as two bf16 terms
CTX_SCORES_SPLIT_P = 1  # ctx_attn_scores flag: the same of ctx_prefill_attn_run_paged with bf16 outputs
CTX_STATIC_SCRATCH_BYTES = 16 << 20  # static workspace of ctx_decode_attn_run_static, per device
CTX_HBM_SINK_BYTES_PER_WORKGROUP = 64
CTX_HBM_NONTEMPORAL = 1
CTX_MFMA_16X16X32 = 0
CTX_MFMA_32X32X16 = 1
MFMA_FLOPS_PER_WAVE_ROUND = {CTX_MFMA_16X16X32: 8 * 16 * 16 * 32 * 2, CTX_MFMA_32X32X16: 8 * 32 * 32 * 16 * 2}

# every function the C header declares
EXPORTS = (
    "ctx_decode_attn_create",
    "ctx_decode_attn_run",
    "ctx_decode_attn_run_static",
    "ctx_decode_attn_run_paged",
    "ctx_prefill_attn_run",
    "ctx_kv_append_run_paged",
    "ctx_prefill_attn_run_paged",
    "ctx_decode_attn_run_paged_scored",
    "ctx_tree_attn_workspace",
    "ctx_tree_attn_run_paged",
    "ctx_kv_fork_run_paged",
    "ctx_kv_resize_workspace",
    "ctx_kv_resize_run_paged",
    "ctx_kv_copy_run_paged",
    "ctx_kv_compact_run_paged",
    "ctx_opd_loss_run",
    "ctx_token_logprob_workspace",
    "ctx_token_logprob_run",
    "ctx_token_logprob_grad_run",
    "ctx_rollout_simulate",
    "ctx_rollout_simulate_engine",
    "ctx_hbm_read",
    "ctx_hbm_copy",
    "ctx_mfma_bf16",
    "ctx_decode_attn_destroy",
    "ctx_decode_attn_status_string",
    "ctx_decode_attn_last_error",
)


class CtxDesc(ctypes.Structure):
    _fields_ = [
        ("num_q_heads", ctypes.c_int32),
        ("num_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("max_batch", ctypes.c_int32),
        ("max_seq_len", ctypes.c_int32),
        ("out_dtype", ctypes.c_int),
        ("split_tokens", ctypes.c_int32),
        ("page_tokens", ctypes.c_int32),
    ]


class OpdParams(ctypes.Structure):
    """ctx_opd_loss_params; defaults are the paper's values (App. OPD Optimization)."""
    _fields_ = [
        ("log_ratio_clip", ctypes.c_float),
        ("clip_delta", ctypes.c_float),
        ("dual_clip", ctypes.c_float),
        ("eps", ctypes.c_float),
    ]

    def __init__(self, log_ratio_clip=20.0, clip_delta=0.2, dual_clip=3.0, eps=1e-8):
        super().__init__(log_ratio_clip, clip_delta, dual_clip, eps)


_OPD_DEFAULTS = OpdParams()


class CtxRotary(ctypes.Structure):
    _fields_ = [("inv_freq", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("q_norm", ctypes.c_void_p),
                ("k_norm", ctypes.c_void_p), ("norm_eps", ctypes.c_float), ("rotary_dim", ctypes.c_int32),
                ("flags", ctypes.c_uint32)]


class CtxAttnScores(ctypes.Structure):
    _fields_ = [("softcap", ctypes.c_float), ("window", ctypes.c_int32), ("slopes", ctypes.c_void_p),
                ("prefix_lens", ctypes.c_void_p), ("doc_starts", ctypes.c_void_p), ("flags", ctypes.c_uint32)]


class RolloutConfig(ctypes.Structure):
    _fields_ = [("policy", ctypes.c_int32), ("num_tasks", ctypes.c_int32), ("turns", ctypes.c_int32),
                ("max_concurrency", ctypes.c_int32)]


class RolloutEngine(ctypes.Structure):
    _fields_ = [("step_base", ctypes.c_double), ("step_per_kv_token", ctypes.c_double),
                ("prefill_per_token", ctypes.c_double), ("fast_tokens", ctypes.c_int32),
                ("full_tokens", ctypes.c_int32)]


ROLLOUT_VANILLA = 0
ROLLOUT_ACTFIRST = 1


class CtxError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"ctx_decode_attn status {status}: {message}")
        self.status = status


_lib = None


def load_library(path: str | None = None):
    """Load the HIP library (built in-tree by __graft_entry__.build())."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    path = path or LIB
    # torch ships its own libamdhip64.so.7; load it first so this library binds
    # to the same HIP runtime as the streams and memory torch hands us
    import torch  # noqa: F401

    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()')")
    lib = ctypes.CDLL(path)
    vp, i32 = ctypes.c_void_p, ctypes.c_int32
    lib.ctx_decode_attn_create.argtypes = [ctypes.POINTER(CtxDesc), ctypes.POINTER(ctypes.c_void_p)]
    lib.ctx_decode_attn_create.restype = ctypes.c_int
    lib.ctx_decode_attn_run.argtypes = [vp, vp, vp, vp, vp, vp, i32, ctypes.c_float, vp, vp]
    lib.ctx_decode_attn_run.restype = ctypes.c_int
    lib.ctx_decode_attn_run_static.argtypes = [ctypes.POINTER(CtxDesc), vp, vp, vp, vp, vp, i32, ctypes.c_float,
                                               vp, vp]
    lib.ctx_decode_attn_run_static.restype = ctypes.c_int
    lib.ctx_decode_attn_run_paged.argtypes = [vp, vp, vp, vp, vp, i32, vp, i32, vp, vp, ctypes.c_float, vp, vp]
    lib.ctx_decode_attn_run_paged.restype = ctypes.c_int
    lib.ctx_prefill_attn_run.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, ctypes.c_float, ctypes.c_uint32,
                                         vp, vp]
    lib.ctx_prefill_attn_run.restype = ctypes.c_int
    lib.ctx_kv_append_run_paged.argtypes = [vp, vp, ctypes.c_int64, vp, ctypes.c_int64, vp, ctypes.c_int64, vp, vp, i32,
                                            vp, i32, vp, vp, vp, i32, i32, ctypes.POINTER(CtxRotary), vp, vp]
    lib.ctx_kv_append_run_paged.restype = ctypes.c_int
    lib.ctx_prefill_attn_run_paged.argtypes = [vp, vp, vp, vp, i32, vp, i32, vp, vp, vp, i32, i32, i32, ctypes.c_float,
                                               ctypes.POINTER(CtxAttnScores), vp, vp]
    lib.ctx_prefill_attn_run_paged.restype = ctypes.c_int
    lib.ctx_decode_attn_run_paged_scored.argtypes = [vp, vp, vp, vp, i32, vp, i32, vp, i32, ctypes.c_float,
                                                     ctypes.POINTER(CtxAttnScores), vp, vp]
    lib.ctx_decode_attn_run_paged_scored.restype = ctypes.c_int
    lib.ctx_opd_loss_run.argtypes = [vp, ctypes.c_int64, i32, vp, vp, vp, vp, vp, i32, i32,
                                     ctypes.POINTER(OpdParams), vp, vp, vp, vp, vp, ctypes.c_int64, vp]
    lib.ctx_opd_loss_run.restype = ctypes.c_int
    size_t, i64, f32 = ctypes.c_size_t, ctypes.c_int64, ctypes.c_float
    lib.ctx_tree_attn_workspace.argtypes = [vp, i32, i32, ctypes.POINTER(size_t)]
    lib.ctx_tree_attn_workspace.restype = ctypes.c_int
    lib.ctx_tree_attn_run_paged.argtypes = [vp, vp, vp, vp, i32, vp, i32, vp, vp, vp, vp, i32, i32, i32, f32,
                                            ctypes.POINTER(CtxAttnScores), vp, vp, size_t, vp]
    lib.ctx_tree_attn_run_paged.restype = ctypes.c_int
    lib.ctx_kv_fork_run_paged.argtypes = [vp, vp, i32, vp, i32, vp, vp, i32, vp]
    lib.ctx_kv_fork_run_paged.restype = ctypes.c_int
    lib.ctx_kv_resize_workspace.argtypes = [i32, i32]
    lib.ctx_kv_resize_workspace.restype = size_t
    lib.ctx_kv_resize_run_paged.argtypes = [vp, vp, i32, vp, vp, i32, vp, i32, vp, vp, vp, size_t, vp]
    lib.ctx_kv_resize_run_paged.restype = ctypes.c_int
    lib.ctx_kv_copy_run_paged.argtypes = [vp, vp, vp, i32, vp, i32, vp]
    lib.ctx_kv_copy_run_paged.restype = ctypes.c_int
    lib.ctx_kv_compact_run_paged.argtypes = [vp, vp, vp, i32, vp, i32, vp, vp, vp, vp, vp, i32, i32, vp, vp]
    lib.ctx_kv_compact_run_paged.restype = ctypes.c_int
    lib.ctx_token_logprob_workspace.argtypes = [ctypes.c_int, i32, i32, i32, ctypes.POINTER(size_t)]
    lib.ctx_token_logprob_workspace.restype = ctypes.c_int
    lib.ctx_token_logprob_run.argtypes = [vp, ctypes.c_int, i64, i32, vp, i32, vp, i32, f32, i32, vp, vp, vp, vp, vp, vp,
                                          size_t, vp]
    lib.ctx_token_logprob_run.restype = ctypes.c_int
    lib.ctx_token_logprob_grad_run.argtypes = [vp, ctypes.c_int, i64, i32, vp, i32, vp, i32, f32, vp, vp, vp, vp, vp, i64,
                                               vp]
    lib.ctx_token_logprob_grad_run.restype = ctypes.c_int
    lib.ctx_rollout_simulate.argtypes = [ctypes.POINTER(RolloutConfig), vp, vp, vp, vp, vp, vp]
    lib.ctx_rollout_simulate.restype = ctypes.c_int
    lib.ctx_rollout_simulate_engine.argtypes = [ctypes.POINTER(RolloutConfig), ctypes.POINTER(RolloutEngine), vp, vp,
                                                vp, vp, vp, vp]
    lib.ctx_rollout_simulate_engine.restype = ctypes.c_int
    lib.ctx_hbm_read.argtypes = [vp, ctypes.c_size_t, vp, i32, ctypes.c_uint32, vp]
    lib.ctx_hbm_read.restype = ctypes.c_int
    lib.ctx_hbm_copy.argtypes = [vp, vp, ctypes.c_size_t, i32, ctypes.c_uint32, vp]
    lib.ctx_hbm_copy.restype = ctypes.c_int
    lib.ctx_mfma_bf16.argtypes = [i32, i32, i32, vp, vp]
    lib.ctx_mfma_bf16.restype = ctypes.c_int
    lib.ctx_decode_attn_destroy.argtypes = [vp]
    lib.ctx_decode_attn_destroy.restype = ctypes.c_int
    lib.ctx_decode_attn_status_string.argtypes = [ctypes.c_int]
    lib.ctx_decode_attn_status_string.restype = ctypes.c_char_p
    lib.ctx_decode_attn_last_error.argtypes = []
    lib.ctx_decode_attn_last_error.restype = ctypes.c_char_p
    if path == LIB:
        _lib = lib
    return lib


def error_for(lib, status: int) -> CtxError:
    msg = lib.ctx_decode_attn_status_string(status).decode()
    detail = lib.ctx_decode_attn_last_error().decode()
    return CtxError(status, f"{msg}: {detail}" if detail else msg)


def _dtype_code(dtype) -> int:
    import torch

    if dtype == torch.float32:
        return CTX_DTYPE_F32
    if dtype == torch.bfloat16:
        return CTX_DTYPE_BF16
    raise ValueError(f"out dtype must be float32 or bfloat16, not {dtype}")


def _check_tensors(device: int, checks) -> None:
    """Each (name, tensor, dtype): that dtype, on cuda:device, contiguous."""
    for name, t, dt in checks:
        # one short test each where nothing is wrong (get_device() is -1 on the
        # CPU): a call on a short batch takes less GPU time than these checks did
        if t.dtype is dt and t.is_cuda and t.get_device() == device and t.is_contiguous():
            continue
        if t.dtype != dt:
            raise TypeError(f"{name} must be {dt}, got {t.dtype}")
        if not t.is_cuda or t.device.index != device:
            raise ValueError(f"{name} must be on cuda:{device}")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")


def _need(name: str, t, dtype, device: int, shape) -> None:
    """One contiguous tensor of that dtype and shape on cuda:device: four tests where nothing is wrong."""
    if t.dtype is dtype and t.get_device() == device and t.is_contiguous() and t.shape == shape:
        return
    _check_tensors(device, ((name, t, dtype),))
    raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")


def _int32(name: str, x) -> int:
    """x, which ctypes would wrap round where it does not fit."""
    if not -2 ** 31 <= x < 2 ** 31:
        raise ValueError(f"{name} {x} does not fit 32 bits")
    return x


def _stream_ptr(stream, device=None) -> int:
    """hipStream_t of a torch stream (default: the current one of `device`) or a raw handle."""
    import torch

    if stream is None:
        # the handle alone, without a Stream object around it
        if device is not None and device.type != "cuda":
            raise ValueError(f"Expected a cuda device, but got: {device}")
        index = torch.cuda.current_device() if device is None or device.index is None else device.index
        return torch._C._cuda_getCurrentRawStream(index)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _allocating_on(stream, device):
    """Where a call allocates its results: on the stream that it runs on, which then orders them
    after what held their memory before and before what holds it next."""
    import torch

    if stream is None:
        return contextlib.nullcontext()
    if not isinstance(stream, torch.cuda.Stream):
        ptr = _stream_ptr(stream)  # 0, the default stream's, would make ExternalStream a stream of its own
        stream = torch.cuda.ExternalStream(ptr, device=device) if ptr else torch.cuda.default_stream(device)
    return torch.cuda.stream(stream)


class Rotary:
    """What DecodeAttention.append_paged does to queries and keys (ctx_rotary): the norm of each
    head, if weights q_norm / k_norm (bf16 [128]) are given, then the rotation of the first
    2 * len(inv_freq) dimensions by position * inv_freq (float32; None: no rotation), over the pairs
    (i, i + len(inv_freq)) or, interleaved, (2 i, 2 i + 1).  positions: int32 per packed row, or
    None: each token's position in its sequence."""

    def __init__(self, inv_freq=None, interleaved: bool = False, positions=None, q_norm=None, k_norm=None,
                 norm_eps: float = 1e-6):
        self.inv_freq, self.interleaved, self.positions = inv_freq, interleaved, positions
        self.q_norm, self.k_norm, self.norm_eps = q_norm, k_norm, norm_eps


class AttnScores:
    """Scores and masks of paged attention (ctx_attn_scores): s = scale q.k, capped by
    softcap * tanh(s / softcap), less slopes[head] * |p - t|; token t is seen from position p if
    t < prefix_lens[sequence] or max(doc_start, p - window + 1) <= t <= p.  slopes: float32 [Hq],
    prefix_lens: int32 [B], doc_starts: int32, one per packed row (prefill) or sequence (decode);
    0 and None leave a part out.  split_p: the prefill with bf16 outputs carries its softmax weights
    as two bf16 terms (CTX_SCORES_SPLIT_P) instead of one; the other calls always do, or as three."""

    def __init__(self, softcap: float = 0.0, window: int = 0, slopes=None, prefix_lens=None, doc_starts=None,
                 split_p: bool = False):
        self.softcap, self.window, self.split_p = softcap, window, split_p
        self.slopes, self.prefix_lens, self.doc_starts = slopes, prefix_lens, doc_starts


def _ptr(t):
    return None if t is None else t.data_ptr()


def _scores_struct(scores: AttnScores, device: int, num_q_heads: int, seqs: int, rows: int):
    """ctx_attn_scores of checked tensors, for a call (None: NULL)."""
    import torch

    if scores is None:
        return None
    slopes, prefix, docs = scores.slopes, scores.prefix_lens, scores.doc_starts
    if slopes is not None:
        _need("slopes", slopes, torch.float32, device, (num_q_heads,))
    if prefix is not None:
        _need("prefix_lens", prefix, torch.int32, device, (seqs,))
    if docs is not None:
        _need("doc_starts", docs, torch.int32, device, (rows,))
    s = CtxAttnScores(scores.softcap, _int32("window", scores.window), _ptr(slopes), _ptr(prefix), _ptr(docs),
                      CTX_SCORES_SPLIT_P if scores.split_p else 0)
    if s.softcap == 0.0 and scores.softcap != 0.0:  # would be no cap at all
        raise ValueError(f"softcap {scores.softcap} is below the smallest float32")
    return ctypes.byref(s)


class DecodeAttention:
    """Handle for ctx_decode_attn_run: decode-step GQA attention of one new token
    per sequence over ragged KV caches [rows, Hkv, 128] (bf16)."""

    def __init__(self, num_q_heads: int, num_kv_heads: int, max_batch: int, max_seq_len: int,
                 head_dim: int = 128, out_dtype=None, split_tokens: int = 0, page_tokens: int = 0):
        import torch

        self.lib = load_library()
        self.out_dtype = torch.float32 if out_dtype is None else out_dtype
        self.desc = CtxDesc(num_q_heads, num_kv_heads, head_dim, max_batch, max_seq_len,
                            _dtype_code(self.out_dtype), split_tokens, page_tokens)
        handle = ctypes.c_void_p()
        rc = self.lib.ctx_decode_attn_create(ctypes.byref(self.desc), ctypes.byref(handle))
        if rc != CTX_OK:
            raise error_for(self.lib, rc)
        self.handle = handle
        self.device = torch.cuda.current_device()
        self.q_heads, self.kv_heads, self.page_tokens = num_q_heads, num_kv_heads, page_tokens

    def run(self, q, k_cache, v_cache, seq_offsets, seq_lens, scale: float, out, stream=None):
        import torch

        if self.handle is None:
            raise RuntimeError("handle is closed")
        d = self.desc
        _check_tensors(self.device, (("q", q, torch.bfloat16), ("k_cache", k_cache, torch.bfloat16),
                                     ("v_cache", v_cache, torch.bfloat16), ("seq_offsets", seq_offsets, torch.int32),
                                     ("seq_lens", seq_lens, torch.int32), ("out", out, self.out_dtype)))
        b = q.shape[0]
        if q.shape != (b, d.num_q_heads, d.head_dim) or out.shape != q.shape:
            raise ValueError(f"q/out must be [{b}, {d.num_q_heads}, {d.head_dim}]")
        if k_cache.dim() != 3 or k_cache.shape[1:] != (d.num_kv_heads, d.head_dim) or v_cache.shape != k_cache.shape:
            raise ValueError(f"k_cache/v_cache must be [rows, {d.num_kv_heads}, {d.head_dim}]")
        if seq_offsets.shape != (b,) or seq_lens.shape != (b,):
            raise ValueError(f"seq_offsets/seq_lens must be [{b}]")
        sp = _stream_ptr(stream)
        rc = self.lib.ctx_decode_attn_run(self.handle, q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
                                          seq_offsets.data_ptr(), seq_lens.data_ptr(), b, float(scale),
                                          out.data_ptr(), sp)
        if rc != CTX_OK:
            raise error_for(self.lib, rc)
        return out

    def run_paged(self, q, k_pages, v_pages, block_tables, seq_lens, scale: float, out,
                  k_new=None, v_new=None, stream=None, scores: AttnScores | None = None):
        """Paged caches [num_pages, P, Hkv, D]; block_tables [B, max_pages] int32;
        optional k_new / v_new [B, Hkv, D] are appended as each sequence's
        newest token (written into its cache slot).  scores: the step with changed scores
        (ctx_decode_attn_run_paged_scored), whose newest tokens are in the pages already."""
        import torch

        if self.handle is None:
            raise RuntimeError("handle is closed")
        if (k_new is None) != (v_new is None):
            raise ValueError("k_new and v_new go together")
        if scores is not None:
            if k_new is not None:
                raise ValueError("with scores, append the new tokens first (append_paged)")
            dev, b = self.device, q.shape[0]
            _need("q", q, torch.bfloat16, dev, (b, self.q_heads, HEAD_DIM))
            _need("out", out, self.out_dtype, dev, (b, self.q_heads, HEAD_DIM))
            _need("seq_lens", seq_lens, torch.int32, dev, (b,))
            self._check_pages(k_pages, v_pages, block_tables, b)
            rc = self.lib.ctx_decode_attn_run_paged_scored(
                self.handle, q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), k_pages.shape[0],
                block_tables.data_ptr(), block_tables.shape[1], seq_lens.data_ptr(), b, scale,
                _scores_struct(scores, dev, self.q_heads, b, b), out.data_ptr(), self._stream(stream))
            if rc != CTX_OK:
                raise error_for(self.lib, rc)
            return out
        d = self.desc
        checks = [("q", q, torch.bfloat16), ("k_pages", k_pages, torch.bfloat16),
                  ("v_pages", v_pages, torch.bfloat16), ("block_tables", block_tables, torch.int32),
                  ("seq_lens", seq_lens, torch.int32), ("out", out, self.out_dtype)]
        if k_new is not None:
            checks += [("k_new", k_new, torch.bfloat16), ("v_new", v_new, torch.bfloat16)]
        _check_tensors(self.device, checks)
        b = q.shape[0]
        if q.shape != (b, d.num_q_heads, d.head_dim) or out.shape != q.shape:
            raise ValueError(f"q/out must be [{b}, {d.num_q_heads}, {d.head_dim}]")
        if k_pages.dim() != 4 or k_pages.shape[1:] != (d.page_tokens, d.num_kv_heads, d.head_dim) \
                or v_pages.shape != k_pages.shape:
            raise ValueError(f"k_pages/v_pages must be [pages, {d.page_tokens}, {d.num_kv_heads}, {d.head_dim}]")
        if block_tables.dim() != 2 or block_tables.shape[0] != b or seq_lens.shape != (b,):
            raise ValueError(f"block_tables must be [{b}, max_pages] and seq_lens [{b}]")
        if k_new is not None and (k_new.shape != (b, d.num_kv_heads, d.head_dim) or v_new.shape != k_new.shape):
            raise ValueError(f"k_new/v_new must be [{b}, {d.num_kv_heads}, {d.head_dim}]")
        sp = _stream_ptr(stream)
        rc = self.lib.ctx_decode_attn_run_paged(
            self.handle, q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), block_tables.data_ptr(),
            block_tables.shape[1], seq_lens.data_ptr(), b,
            k_new.data_ptr() if k_new is not None else None, v_new.data_ptr() if v_new is not None else None,
            float(scale), out.data_ptr(), sp)
        if rc != CTX_OK:
            raise error_for(self.lib, rc)
        return out

    def _check_pages(self, k_pages, v_pages, block_tables, seqs: int):
        import torch

        pages = (k_pages.shape[0], self.page_tokens, self.kv_heads, HEAD_DIM)
        _need("k_pages", k_pages, torch.bfloat16, self.device, pages)
        _need("v_pages", v_pages, torch.bfloat16, self.device, pages)
        _need("block_tables", block_tables, torch.int32, self.device, (seqs, block_tables.shape[-1]))

    def _stream(self, stream):
        import torch

        # of the handle's device, which the call checks to be the current one
        return torch._C._cuda_getCurrentRawStream(self.device) if stream is None else _stream_ptr(stream)

    def _row_stride(self, name: str, t, rows: int, heads: int) -> int:
        """Elements between the rows of heads that may be slices of wider rows."""
        import torch

        if t.dtype is not torch.bfloat16:
            raise TypeError(f"{name} must be torch.bfloat16, got {t.dtype}")
        if t.get_device() != self.device:
            raise ValueError(f"{name} must be on cuda:{self.device}")
        if t.shape != (rows, heads, HEAD_DIM):
            raise ValueError(f"{name} must be [{rows}, {heads}, {HEAD_DIM}]")
        row, head, dim = t.stride()
        if dim != 1 or (head != HEAD_DIM and heads > 1):
            raise ValueError(f"the heads of {name} must be contiguous within its rows")
        return row if rows > 1 else heads * HEAD_DIM  # the stride of a single row says nothing

    def append_paged(self, k, v, k_pages, v_pages, block_tables, seq_lens, q=None, q_out=None, q_starts=None,
                     q_lens=None, rotary: Rotary | None = None, stream=None):
        """Append new tokens to paged caches (ctx_kv_append_run_paged): rows k, v [rows, Hkv, D] go to the
        slots of each sequence's last q_lens[b] of seq_lens[b] tokens (rows q_starts[b] ..; without
        q_starts / q_lens row b is the newest token of sequence b), and q [rows, Hq, D], if given, to
        q_out; q and k are normed and rotated as `rotary` says.  k, v and q may be slices of wider
        rows (heads and dimensions contiguous).  Returns q_out (if None, allocated on the stream
        that the call runs on; without q None)."""
        import torch

        if self.handle is None:
            raise RuntimeError("handle is closed")
        if (q_starts is None) != (q_lens is None):
            raise ValueError("q_starts and q_lens go together")
        dev, rows, seqs = self.device, k.shape[0], seq_lens.shape[0]
        k_stride, v_stride = self._row_stride("k", k, rows, self.kv_heads), self._row_stride("v", v, rows, self.kv_heads)
        q_stride = 0
        if q is not None:
            q_stride = self._row_stride("q", q, rows, self.q_heads)
            if q_out is None:
                with _allocating_on(stream, q.device):
                    q_out = torch.empty((rows, self.q_heads, HEAD_DIM), dtype=torch.bfloat16, device=q.device)
            else:
                _need("q_out", q_out, torch.bfloat16, dev, (rows, self.q_heads, HEAD_DIM))
        elif q_out is not None:
            raise ValueError("q_out needs q")
        self._check_pages(k_pages, v_pages, block_tables, seqs)
        _need("seq_lens", seq_lens, torch.int32, dev, (seqs,))
        if q_starts is not None:
            _need("q_starts", q_starts, torch.int32, dev, (seqs,))
            _need("q_lens", q_lens, torch.int32, dev, (seqs,))
        elif seqs != rows:
            raise ValueError(f"without q_starts, seq_lens must be [{rows}]")
        r = None
        if rotary is not None:
            freqs, positions, q_norm, k_norm = rotary.inv_freq, rotary.positions, rotary.q_norm, rotary.k_norm
            if freqs is not None:
                _need("inv_freq", freqs, torch.float32, dev, (freqs.shape[0],))
            if positions is not None:
                _need("positions", positions, torch.int32, dev, (rows,))
            if q_norm is not None:
                _need("q_norm", q_norm, torch.bfloat16, dev, (HEAD_DIM,))
            if k_norm is not None:
                _need("k_norm", k_norm, torch.bfloat16, dev, (HEAD_DIM,))
            r = ctypes.byref(CtxRotary(_ptr(freqs), _ptr(positions), _ptr(q_norm), _ptr(k_norm), rotary.norm_eps,
                                       0 if freqs is None else 2 * freqs.shape[0],
                                       CTX_ROTARY_INTERLEAVED if rotary.interleaved else 0))
        rc = self.lib.ctx_kv_append_run_paged(
            self.handle, _ptr(q), q_stride, k.data_ptr(), k_stride, v.data_ptr(), v_stride, k_pages.data_ptr(),
            v_pages.data_ptr(), k_pages.shape[0], block_tables.data_ptr(), block_tables.shape[1], seq_lens.data_ptr(),
            _ptr(q_starts), _ptr(q_lens), seqs, rows, r, _ptr(q_out), self._stream(stream))
        if rc != CTX_OK:
            raise error_for(self.lib, rc)
        return q_out

    def prefill_paged(self, q, k_pages, v_pages, block_tables, seq_lens, q_starts, q_lens, max_q_len: int,
                      scale: float, out, scores: AttnScores | None = None, stream=None):
        """Causal prefill over paged caches (ctx_prefill_attn_run_paged): q / out [rows, Hq, D];
        sequence b's q_lens[b] queries (rows q_starts[b] ..) are the last of its seq_lens[b] tokens,
        whose keys and values are in the pages; scores changes scores and masks."""
        import torch

        if self.handle is None:
            raise RuntimeError("handle is closed")
        dev, b, rows = self.device, seq_lens.shape[0], q.shape[0]
        _need("q", q, torch.bfloat16, dev, (rows, self.q_heads, HEAD_DIM))
        _need("out", out, self.out_dtype, dev, (rows, self.q_heads, HEAD_DIM))
        for name, t in (("seq_lens", seq_lens), ("q_starts", q_starts), ("q_lens", q_lens)):
            _need(name, t, torch.int32, dev, (b,))
        self._check_pages(k_pages, v_pages, block_tables, b)
        rc = self.lib.ctx_prefill_attn_run_paged(
            self.handle, q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), k_pages.shape[0],
            block_tables.data_ptr(), block_tables.shape[1], seq_lens.data_ptr(), q_starts.data_ptr(),
            q_lens.data_ptr(), b, rows, _int32("max_q_len", max_q_len), scale, _scores_struct(scores, dev, self.q_heads, b, rows),
            out.data_ptr(), self._stream(stream))
        if rc != CTX_OK:
            raise error_for(self.lib, rc)
        return out

    def tree_paged(self, q, k_pages, v_pages, block_tables, seq_lens, q_starts, q_lens, parents, max_q_len: int,
                   scale: float, out, scores: AttnScores | None = None, workspace=None, stream=None):
        """Attention of drafted trees over paged caches (ctx_tree_attn_run_paged): q / out [rows, Hq, D];
        sequence b's q_lens[b] drafts (rows q_starts[b] ..) are the last of its seq_lens[b] tokens, whose
        keys and values are in the pages.  parents int32 [rows]: -1, or the index of a draft's parent
        among its sequence's drafts before it (any other value: a padding row).  A draft sees the tokens
        before the drafts, its ancestors and itself; scores (without doc_starts) changes scores and
        masks by positions, which count depths.  workspace: uint8, at least tree_workspace bytes; None:
        allocated on the stream that the call runs on.  Calls that may overlap need one each."""
        import torch

        if self.handle is None:
            raise RuntimeError("handle is closed")
        dev, b, rows = self.device, seq_lens.shape[0], q.shape[0]
        _need("q", q, torch.bfloat16, dev, (rows, self.q_heads, HEAD_DIM))
        _need("out", out, self.out_dtype, dev, (rows, self.q_heads, HEAD_DIM))
        for name, t in (("seq_lens", seq_lens), ("q_starts", q_starts), ("q_lens", q_lens)):
            _need(name, t, torch.int32, dev, (b,))
        _need("parents", parents, torch.int32, dev, (rows,))
        self._check_pages(k_pages, v_pages, block_tables, b)
        if scores is not None and scores.doc_starts is not None:
            raise ValueError("trees have no doc_starts")
        max_q_len = _int32("max_q_len", max_q_len)
        if workspace is None:
            size = self.tree_workspace(b, max_q_len)
            with _allocating_on(stream, q.device):
                workspace = torch.empty(size, dtype=torch.uint8, device=q.device)
        else:
            _need("workspace", workspace, torch.uint8, dev, (workspace.numel(),))
        rc = self.lib.ctx_tree_attn_run_paged(
            self.handle, q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), k_pages.shape[0], block_tables.data_ptr(),
            block_tables.shape[1], seq_lens.data_ptr(), q_starts.data_ptr(), q_lens.data_ptr(), parents.data_ptr(), b, rows,
            max_q_len, scale, _scores_struct(scores, dev, self.q_heads, b, rows), out.data_ptr(), workspace.data_ptr(),
            workspace.numel(), self._stream(stream))
        if rc != CTX_OK:
            raise error_for(self.lib, rc)
        return out

    def tree_workspace(self, num_seqs: int, max_q_len: int) -> int:
        """Bytes of workspace of a tree_paged call (ctx_tree_attn_workspace)."""
        if self.handle is None:
            raise RuntimeError("handle is closed")
        size = ctypes.c_size_t()
        rc = self.lib.ctx_tree_attn_workspace(self.handle, num_seqs, max_q_len, ctypes.byref(size))
        if rc != CTX_OK:
            raise error_for(self.lib, rc)
        return size.value

    def _check_rows(self, block_tables, seq_lens, page_refs) -> int:
        """Rows of a block table whose pages are counted."""
        import torch

        if self.handle is None:
            raise RuntimeError("handle is closed")
        seqs = seq_lens.shape[0]
        _need("seq_lens", seq_lens, torch.int32, self.device, (seqs,))
        _need("block_tables", block_tables, torch.int32, self.device, (seqs, block_tables.shape[-1]))
        _need("page_refs", page_refs, torch.int32, self.device, (page_refs.shape[0],))
        return seqs

    def fork_pages(self, block_tables, seq_lens, page_refs, parents, stream=None):
        """Fork rows of a block table (ctx_kv_fork_run_paged): row b and seq_lens[b] become those of
        row parents[b] (-1: row b stays as it is), whose pages both then hold; page_refs int32 [pages]
        counts the rows that hold each page.  All three are written in place."""
        import torch

        seqs = self._check_rows(block_tables, seq_lens, page_refs)
        _need("parents", parents, torch.int32, self.device, (seqs,))
        rc = self.lib.ctx_kv_fork_run_paged(
            self.handle, block_tables.data_ptr(), block_tables.shape[1], seq_lens.data_ptr(), seqs, parents.data_ptr(),
            page_refs.data_ptr(), page_refs.shape[0], self._stream(stream))
        if rc != CTX_OK:
            raise error_for(self.lib, rc)

    def resize_pages(self, block_tables, seq_lens, new_lens, page_refs, granted=None, copies=None, workspace=None,
                     stream=None):
        """Change the lengths of the rows of a block table from seq_lens to new_lens
        (ctx_kv_resize_run_paged): pages are given back, or the lowest free ones taken, in the order of
        rows, and a last page that other rows hold too is replaced where the row grows in it.  Writes
        block_tables and page_refs in place; returns granted int32 [B], the lengths from now on
        (seq_lens[b] where the free pages did not suffice; may be seq_lens itself), and copies
        int32 [B, 2], the pages that copy_pages has to copy in each layer's caches.  Those not
        given, and the workspace (uint8), are allocated on the stream that the call runs on."""
        import torch

        seqs = self._check_rows(block_tables, seq_lens, page_refs)
        pages, dev = page_refs.shape[0], seq_lens.device
        _need("new_lens", new_lens, torch.int32, self.device, (seqs,))
        if granted is not None:
            _need("granted", granted, torch.int32, self.device, (seqs,))
        if copies is not None:
            _need("copies", copies, torch.int32, self.device, (seqs, 2))
        if workspace is not None:
            _need("workspace", workspace, torch.uint8, self.device, (workspace.numel(),))
        with _allocating_on(stream, dev):
            if granted is None:
                granted = torch.empty((seqs,), dtype=torch.int32, device=dev)
            if copies is None:
                copies = torch.empty((seqs, 2), dtype=torch.int32, device=dev)
            if workspace is None:
                workspace = torch.empty(self.lib.ctx_kv_resize_workspace(seqs, pages), dtype=torch.uint8, device=dev)
        rc = self.lib.ctx_kv_resize_run_paged(
            self.handle, block_tables.data_ptr(), block_tables.shape[1], seq_lens.data_ptr(), new_lens.data_ptr(), seqs,
            page_refs.data_ptr(), pages, granted.data_ptr(), copies.data_ptr(), workspace.data_ptr(), workspace.numel(),
            self._stream(stream))
        if rc != CTX_OK:
            raise error_for(self.lib, rc)
        return granted, copies

    def _check_caches(self, k_pages, v_pages):
        import torch

        pages = (k_pages.shape[0], self.page_tokens, self.kv_heads, HEAD_DIM)
        _need("k_pages", k_pages, torch.bfloat16, self.device, pages)
        _need("v_pages", v_pages, torch.bfloat16, self.device, pages)

    def copy_pages(self, k_pages, v_pages, copies, stream=None):
        """Copy whole pages of a layer's caches (ctx_kv_copy_run_paged): page copies[i, 0] to
        copies[i, 1]; -1: nothing."""
        import torch

        if self.handle is None:
            raise RuntimeError("handle is closed")
        self._check_caches(k_pages, v_pages)
        _need("copies", copies, torch.int32, self.device, (copies.shape[0], 2))
        rc = self.lib.ctx_kv_copy_run_paged(self.handle, k_pages.data_ptr(), v_pages.data_ptr(), k_pages.shape[0],
                                            copies.data_ptr(), copies.shape[0], self._stream(stream))
        if rc != CTX_OK:
            raise error_for(self.lib, rc)

    def compact_paged(self, k_pages, v_pages, block_tables, seq_lens, q_starts, q_lens, keep, keep_lens, new_lens=None,
                      stream=None):
        """Move the kept tokens of each sequence together (ctx_kv_compact_run_paged): of its last
        q_lens[b] tokens those that keep [rows] lists, rising, in rows q_starts[b] .. q_starts[b] +
        keep_lens[b] - 1.  Returns new_lens int32 [B], the sequences' lengths without the others (if
        None, allocated on the stream that the call runs on)."""
        import torch

        if self.handle is None:
            raise RuntimeError("handle is closed")
        dev, seqs, rows = self.device, seq_lens.shape[0], keep.shape[0]
        self._check_pages(k_pages, v_pages, block_tables, seqs)
        for name, t in (("seq_lens", seq_lens), ("q_starts", q_starts), ("q_lens", q_lens), ("keep_lens", keep_lens)):
            _need(name, t, torch.int32, dev, (seqs,))
        _need("keep", keep, torch.int32, dev, (rows,))
        if new_lens is None:
            with _allocating_on(stream, seq_lens.device):
                new_lens = torch.empty((seqs,), dtype=torch.int32, device=seq_lens.device)
        else:
            _need("new_lens", new_lens, torch.int32, dev, (seqs,))
        rc = self.lib.ctx_kv_compact_run_paged(
            self.handle, k_pages.data_ptr(), v_pages.data_ptr(), k_pages.shape[0], block_tables.data_ptr(),
            block_tables.shape[1], seq_lens.data_ptr(), q_starts.data_ptr(), q_lens.data_ptr(), keep.data_ptr(),
            keep_lens.data_ptr(), seqs, rows, new_lens.data_ptr(), self._stream(stream))
        if rc != CTX_OK:
            raise error_for(self.lib, rc)
        return new_lens

    def prefill(self, q, k_cache, v_cache, seq_offsets, seq_lens, q_starts, q_lens, max_q_len: int,
                scale: float, out, stream=None, split_p: bool = False):
        """Causal prefill: q / out [total_q, Hq, D]; sequence b's q_lens[b] queries
        (rows q_starts[b] ..) are the last q_lens[b] of its seq_lens[b] cached rows.
        split_p: carry the softmax weights as two bf16 terms (CTX_PREFILL_SPLIT_P)
        instead of one."""
        import torch

        if self.handle is None:
            raise RuntimeError("handle is closed")
        d = self.desc
        _check_tensors(self.device, (("q", q, torch.bfloat16), ("k_cache", k_cache, torch.bfloat16),
                                     ("v_cache", v_cache, torch.bfloat16), ("seq_offsets", seq_offsets, torch.int32),
                                     ("seq_lens", seq_lens, torch.int32), ("q_starts", q_starts, torch.int32),
                                     ("q_lens", q_lens, torch.int32), ("out", out, self.out_dtype)))
        b = seq_lens.shape[0]
        if q.dim() != 3 or q.shape[1:] != (d.num_q_heads, d.head_dim) or out.shape != q.shape:
            raise ValueError(f"q/out must be [rows, {d.num_q_heads}, {d.head_dim}]")
        if k_cache.dim() != 3 or k_cache.shape[1:] != (d.num_kv_heads, d.head_dim) or v_cache.shape != k_cache.shape:
            raise ValueError(f"k_cache/v_cache must be [rows, {d.num_kv_heads}, {d.head_dim}]")
        if seq_offsets.shape != (b,) or q_starts.shape != (b,) or q_lens.shape != (b,):
            raise ValueError(f"seq_offsets, seq_lens, q_starts, q_lens must all be [{b}]")
        sp = _stream_ptr(stream)
        rc = self.lib.ctx_prefill_attn_run(self.handle, q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
                                           seq_offsets.data_ptr(), seq_lens.data_ptr(), q_starts.data_ptr(),
                                           q_lens.data_ptr(), b, _int32("max_q_len", int(max_q_len)), float(scale),
                                           CTX_PREFILL_SPLIT_P if split_p else 0, out.data_ptr(), sp)
        if rc != CTX_OK:
            raise error_for(self.lib, rc)
        return out

    def close(self):
        if getattr(self, "handle", None) is not None:
            rc = self.lib.ctx_decode_attn_destroy(self.handle)
            self.handle = None
            if rc != CTX_OK:
                raise error_for(self.lib, rc)

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def ctx_decode_attn_run_static(q, k_cache, v_cache, seq_offsets, seq_lens, scale: float, out, num_kv_heads: int,
                               max_batch: int | None = None, stream=None):
    """ctx_decode_attn_run_static: the decode step with no handle and no
    allocation (the split workspace is the library's static device array).
    q / out [B, Hq, 128] (out float32 or bfloat16), caches [rows, Hkv, 128] bf16,
    seq_offsets / seq_lens [B] int32; max_batch defaults to B (1 for an empty batch)."""
    import torch

    lib = load_library()
    b, hq = q.shape[0], q.shape[1]
    device = q.device.index if q.is_cuda else -1
    _check_tensors(device, (("q", q, torch.bfloat16), ("k_cache", k_cache, torch.bfloat16),
                            ("v_cache", v_cache, torch.bfloat16), ("seq_offsets", seq_offsets, torch.int32),
                            ("seq_lens", seq_lens, torch.int32), ("out", out, out.dtype)))
    if q.dim() != 3 or out.shape != q.shape:
        raise ValueError("q/out must be [B, Hq, 128] of one shape")
    if k_cache.dim() != 3 or k_cache.shape[1] != num_kv_heads or v_cache.shape != k_cache.shape:
        raise ValueError(f"k_cache/v_cache must be [rows, {num_kv_heads}, 128]")
    if seq_offsets.shape != (b,) or seq_lens.shape != (b,):
        raise ValueError(f"seq_offsets/seq_lens must be [{b}]")
    desc = CtxDesc(hq, num_kv_heads, q.shape[2], max(b, 1) if max_batch is None else max_batch, 1,
                   _dtype_code(out.dtype), 0, 0)
    rc = lib.ctx_decode_attn_run_static(ctypes.byref(desc), q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
                                        seq_offsets.data_ptr(), seq_lens.data_ptr(), b, float(scale), out.data_ptr(),
                                        _stream_ptr(stream, q.device))
    if rc != CTX_OK:
        raise error_for(lib, rc)
    return out


def opd_loss(logits, tokens, old_logp, teacher_logp, mask, seq_starts, params: OpdParams | None = None,
             grad: bool = True, out: dict | None = None, stream=None) -> dict:
    """Fused OPD token loss (ctx_opd_loss_run) over a packed batch.

    logits bf16 [N, stride] (the last dimension may be a view wider than vocab:
    pass `vocab` via logits.shape[1] unless `out["vocab"]` is given), tokens int32 [N],
    old_logp / teacher_logp float32 [N], mask uint8 [N], seq_starts int32 [B + 1].
    Returns a dict of device tensors: loss [1], token_logp, token_weight,
    token_loss [N] and, with grad=True, grad_logits bf16 [N, vocab].  Tensors
    given in `out` under those names are written in place (no allocation); the others
    are allocated on the stream that the call runs on."""
    import torch

    lib = load_library()
    params = params or _OPD_DEFAULTS
    n = tokens.shape[0]
    dev = logits.device
    for name, t, dt in (("logits", logits, torch.bfloat16), ("tokens", tokens, torch.int32),
                        ("old_logp", old_logp, torch.float32), ("teacher_logp", teacher_logp, torch.float32),
                        ("mask", mask, torch.uint8), ("seq_starts", seq_starts, torch.int32)):
        if t.dtype is dt and t.is_cuda and t.device == dev:
            continue
        if t.dtype != dt:
            raise TypeError(f"{name} must be {dt}, got {t.dtype}")
        if not t.is_cuda or t.device != dev:
            raise ValueError(f"{name} must be on {dev}")
    if logits.dim() != 2 or logits.shape[0] != n or logits.stride(1) != 1:
        raise ValueError("logits must be [N, V] with unit column stride")
    for name, t in (("tokens", tokens), ("old_logp", old_logp), ("teacher_logp", teacher_logp),
                    ("mask", mask), ("seq_starts", seq_starts)):
        if not t.is_contiguous() or t.dim() != 1:
            raise ValueError(f"{name} must be a contiguous vector")
    out = dict(out or {})
    vocab = int(out.pop("vocab", logits.shape[1]))
    if not 0 < vocab <= logits.shape[1]:
        raise ValueError(f"vocab {vocab} must be in 1..{logits.shape[1]} (the columns of logits)")

    def buf(name, shape, dtype):
        t = out.get(name)
        if t is None:
            with _allocating_on(stream, dev):
                return torch.empty(shape, dtype=dtype, device=dev)
        if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous() or t.device != dev:
            raise ValueError(f"out[{name!r}] must be a contiguous {dtype} tensor of shape {tuple(shape)}")
        return t

    res = {"loss": buf("loss", (1,), torch.float32), "token_logp": buf("token_logp", (n,), torch.float32),
           "token_weight": buf("token_weight", (n,), torch.float32),
           "token_loss": buf("token_loss", (n,), torch.float32)}
    g = None
    if grad:
        g = out.get("grad_logits")
        if g is None:  # rows padded to a multiple of 8 elements (16-byte chunks)
            with _allocating_on(stream, dev):
                g = torch.empty((n, (vocab + 7) // 8 * 8), dtype=torch.bfloat16, device=dev)
        elif (g.dtype != torch.bfloat16 or g.dim() != 2 or g.shape[0] != n or g.stride(1) != 1
              or g.shape[1] < vocab or g.device != dev):
            raise ValueError(f"out['grad_logits'] must be bf16 [N, >= {vocab}] with unit column stride on {dev}")
        res["grad_logits"] = g if out.get("grad_logits") is not None else g[:, :vocab]
    sp = _stream_ptr(stream, dev)
    rc = lib.ctx_opd_loss_run(logits.data_ptr(), logits.stride(0), vocab, tokens.data_ptr(), old_logp.data_ptr(),
                              teacher_logp.data_ptr(), mask.data_ptr(), seq_starts.data_ptr(),
                              seq_starts.shape[0] - 1, n, ctypes.byref(params), res["token_logp"].data_ptr(),
                              res["token_weight"].data_ptr(), res["token_loss"].data_ptr(), res["loss"].data_ptr(),
                              g.data_ptr() if g is not None else None, g.stride(0) if g is not None else 0, sp)
    if rc != CTX_OK:
        raise error_for(lib, rc)
    return res


def _logits_rows(logits, name: str = "logits"):
    """dtype code, rows, columns and row stride of a matrix of logits."""
    import torch

    if logits.dtype is not torch.bfloat16 and logits.dtype is not torch.float32:
        raise TypeError(f"{name} must be bfloat16 or float32, got {logits.dtype}")
    if not logits.is_cuda:
        raise ValueError(f"{name} must be on a cuda device")
    if logits.dim() != 2 or logits.stride(1) != 1:
        raise ValueError(f"{name} must be [N, V] with unit column stride")
    rows, vocab = logits.shape
    # the stride of a single row says nothing
    stride = logits.stride(0) if rows > 1 else (vocab + 7) // 8 * 8
    return _dtype_code(logits.dtype), rows, vocab, stride


def _logit_tokens(tokens, rows: int, device: int) -> int:
    """Given tokens per row."""
    import torch

    if tokens is None:
        return 0
    if tokens.dim() == 1:
        _need("tokens", tokens, torch.int32, device, (rows,))
        return 1
    _need("tokens", tokens, torch.int32, device, (rows, tokens.shape[-1]))
    return tokens.shape[1]


def _scale_of(temperature: float) -> float:
    if not temperature > 0:
        raise ValueError(f"temperature must be positive, got {temperature}")
    return 1.0 / temperature


def _on_current(device: int, what: str) -> None:
    import torch

    if torch.cuda.current_device() != device:
        raise ValueError(f"{what} on cuda:{device}, which is not the current device")


def token_logprobs(logits, tokens=None, mask=None, temperature: float = 1.0, top: int = 0, entropy: bool = True,
                   out: dict | None = None, workspace=None, stream=None) -> dict:
    """Log probabilities of given tokens under softmax(logits / temperature), its entropy and the
    `top` largest logits (ctx_token_logprob_run).

    logits bf16 or float32 [N, V] (rows may be views of wider ones, a multiple of 16 bytes apart),
    tokens int32 [N] or [N, M] (M up to 64; below 0: none), mask uint8 [N] (0: the row is not read).
    Returns a dict of device tensors: token_logp float32 like tokens (if M > 0), entropy [N] (with entropy=True),
    top_tokens int32 and top_logp [N, top] (the lowest column first among equal logits, -1 where there
    is none) and stats [N, 2], which token_logprobs_grad takes.  Tensors given in `out` under those
    names are written in place; the others, and the workspace of a call on few rows (uint8), are
    allocated on the stream that the call runs on.  Calls that may overlap need a workspace each."""
    import torch

    lib = load_library()
    code, n, vocab, stride = _logits_rows(logits)
    dev, index = logits.device, logits.get_device()
    _on_current(index, "logits")
    m = _logit_tokens(tokens, n, index)
    if mask is not None:
        _need("mask", mask, torch.uint8, index, (n,))
    out = out or {}

    def buf(name, shape, dtype):
        t = out.get(name)
        if t is None:
            return torch.empty(shape, dtype=dtype, device=dev)
        _need(f"out[{name!r}]", t, dtype, index, shape)
        return t

    nbytes = ctypes.c_size_t()
    top = _int32("top", top)
    if (rc := lib.ctx_token_logprob_workspace(code, _int32("vocab", vocab), n, top, ctypes.byref(nbytes))) != CTX_OK:
        raise error_for(lib, rc)
    with _allocating_on(stream, dev):
        res = {"stats": buf("stats", (n, 2), torch.float32)}
        if m > 0:
            res["token_logp"] = buf("token_logp", tokens.shape, torch.float32)
        if entropy:
            res["entropy"] = buf("entropy", (n,), torch.float32)
        if top > 0:
            res["top_tokens"] = buf("top_tokens", (n, top), torch.int32)
            res["top_logp"] = buf("top_logp", (n, top), torch.float32)
        size = nbytes.value
        if workspace is None:
            workspace = torch.empty(size, dtype=torch.uint8, device=dev) if size else None
        else:
            _need("workspace", workspace, torch.uint8, index, (workspace.numel(),))
    rc = lib.ctx_token_logprob_run(
        logits.data_ptr(), code, stride, vocab, _ptr(tokens) if m > 0 else None, m, _ptr(mask), n, _scale_of(temperature), top,
        _ptr(res.get("token_logp")), _ptr(res.get("entropy")), res["stats"].data_ptr(), _ptr(res.get("top_tokens")),
        _ptr(res.get("top_logp")), _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream_ptr(stream, dev))
    if rc != CTX_OK:
        raise error_for(lib, rc)
    return res


def token_logprobs_grad(logits, tokens, result: dict, grad_logp, grad_entropy=None, mask=None, temperature: float = 1.0,
                        out=None, stream=None):
    """Gradient by the logits of sum(grad_logp * token_logp) + sum(grad_entropy * entropy)
    (ctx_token_logprob_grad_run); result: what token_logprobs returned for the same logits, mask and
    temperature.  tokens may be others than that call's (its top_tokens, for instance, with grad_logp
    the gradient of top_logp); grad_logp float32 like tokens, both None without any.  Returns
    grad_logits [N, V] of the logits' type (`out`, or allocated on the stream that the call runs on,
    its rows padded to 16 bytes)."""
    import torch

    lib = load_library()
    code, n, vocab, stride = _logits_rows(logits)
    dev, index = logits.device, logits.get_device()
    _on_current(index, "logits")
    m = _logit_tokens(tokens, n, index)
    if (grad_logp is None) != (tokens is None):
        raise ValueError("tokens and grad_logp go together")
    if m > 0:
        _need("grad_logp", grad_logp, torch.float32, index, tokens.shape)
    if mask is not None:
        _need("mask", mask, torch.uint8, index, (n,))
    _need("result['stats']", result["stats"], torch.float32, index, (n, 2))
    h = None
    if grad_entropy is not None:
        h = result.get("entropy")
        if h is None:
            raise ValueError("grad_entropy needs the entropy of the forward call")
        _need("result['entropy']", h, torch.float32, index, (n,))
        _need("grad_entropy", grad_entropy, torch.float32, index, (n,))
    if out is None:
        with _allocating_on(stream, dev):
            grad = torch.empty((n, (vocab + 7) // 8 * 8), dtype=logits.dtype, device=dev)
        out = grad[:, :vocab]
    elif out.dtype != logits.dtype or out.shape != logits.shape or out.get_device() != index or out.stride(1) != 1:
        raise ValueError(f"out must be {logits.dtype} {list(logits.shape)} with unit column stride on {dev}")
    rc = lib.ctx_token_logprob_grad_run(
        logits.data_ptr(), code, stride, vocab, _ptr(tokens) if m > 0 else None, m, _ptr(mask), n, _scale_of(temperature),
        result["stats"].data_ptr(), _ptr(h), _ptr(grad_logp) if m > 0 else None, _ptr(grad_entropy), out.data_ptr(),
        _logits_rows(out, "out")[3], _stream_ptr(stream, dev))
    if rc != CTX_OK:
        raise error_for(lib, rc)
    return out


def _rollout_outputs(n, turns):
    import numpy as np

    return (np.zeros(1, np.float64), np.full(n * turns * 2, -1.0), np.full(n * turns * 2, -1.0),
            np.zeros(1, np.int32))


def rollout_simulate(policy: int, fast_latency, full_latency, max_concurrency: int) -> dict:
    """Latency model of ctx_rollout_simulate.  fast_latency, full_latency:
    [N, T] seconds (host arrays).  Returns completion, start and end [N, T, 2]
    (kind 0 = fast action, 1 = full response; -1 = not submitted) and peak."""
    import numpy as np

    lib = load_library()
    full = np.ascontiguousarray(full_latency, dtype=np.float64)
    fast = np.ascontiguousarray(fast_latency, dtype=np.float64)
    n, turns = full.shape
    cfg = RolloutConfig(policy, n, turns, max_concurrency)
    comp, st, en, pk = _rollout_outputs(n, turns)
    p = lambda a: a.ctypes.data_as(ctypes.c_void_p)  # noqa: E731
    rc = lib.ctx_rollout_simulate(ctypes.byref(cfg), p(fast), p(full), p(comp), p(st), p(en), p(pk))
    if rc != CTX_OK:
        raise error_for(lib, rc)
    return {"completion": float(comp[0]), "start": st.reshape(n, turns, 2), "end": en.reshape(n, turns, 2),
            "peak": int(pk[0])}


def rollout_simulate_engine(policy: int, context_tokens, fast_tokens: int, full_tokens: int, max_concurrency: int,
                            step_base: float, step_per_kv_token: float, prefill_per_token: float) -> dict:
    """Engine model of ctx_rollout_simulate_engine; context_tokens [N, T]."""
    import numpy as np

    lib = load_library()
    ctx = np.ascontiguousarray(context_tokens, dtype=np.int32)
    n, turns = ctx.shape
    cfg = RolloutConfig(policy, n, turns, max_concurrency)
    eng = RolloutEngine(step_base, step_per_kv_token, prefill_per_token, fast_tokens, full_tokens)
    comp, st, en, pk = _rollout_outputs(n, turns)
    steps = np.zeros(1, np.int64)
    p = lambda a: a.ctypes.data_as(ctypes.c_void_p)  # noqa: E731
    rc = lib.ctx_rollout_simulate_engine(ctypes.byref(cfg), ctypes.byref(eng), p(ctx), p(comp), p(st), p(en),
                                         p(pk), p(steps))
    if rc != CTX_OK:
        raise error_for(lib, rc)
    return {"completion": float(comp[0]), "start": st.reshape(n, turns, 2), "end": en.reshape(n, turns, 2),
            "peak": int(pk[0]), "steps": int(steps[0])}


def ctx_hbm_read(src, sink, workgroups: int, nontemporal: bool = True, stream=None):
    """Stream every byte of the contiguous CUDA tensor `src` once through the
    compute units (ctx_hbm_read); `sink` is a CUDA tensor of at least
    workgroups * 64 bytes."""
    lib = load_library()
    nbytes = src.numel() * src.element_size()
    if not src.is_contiguous() or sink.numel() * sink.element_size() < workgroups * CTX_HBM_SINK_BYTES_PER_WORKGROUP:
        raise ValueError("src must be contiguous and sink hold workgroups * 64 bytes")
    rc = lib.ctx_hbm_read(src.data_ptr(), nbytes, sink.data_ptr(), int(workgroups),
                          CTX_HBM_NONTEMPORAL if nontemporal else 0, _stream_ptr(stream, src.device))
    if rc != CTX_OK:
        raise error_for(lib, rc)


def ctx_hbm_copy(src, dst, workgroups: int, nontemporal: bool = True, stream=None):
    """dst = src (contiguous CUDA tensors of equal byte size), every byte read and written once."""
    lib = load_library()
    nbytes = src.numel() * src.element_size()
    if not (src.is_contiguous() and dst.is_contiguous()) or dst.numel() * dst.element_size() != nbytes:
        raise ValueError("src and dst must be contiguous and of equal size")
    rc = lib.ctx_hbm_copy(src.data_ptr(), dst.data_ptr(), nbytes, int(workgroups),
                          CTX_HBM_NONTEMPORAL if nontemporal else 0, _stream_ptr(stream, src.device))
    if rc != CTX_OK:
        raise error_for(lib, rc)


def ctx_mfma_bf16(shape: int, workgroups: int, iterations: int, sink, stream=None) -> int:
    """Run the matrix-core rate probe (ctx_mfma_bf16); returns the flops it performs.
    `sink` is a CUDA tensor of at least workgroups * 64 bytes."""
    lib = load_library()
    if sink.numel() * sink.element_size() < workgroups * CTX_HBM_SINK_BYTES_PER_WORKGROUP:
        raise ValueError("sink must hold workgroups * 64 bytes")
    rc = lib.ctx_mfma_bf16(int(shape), int(workgroups), int(iterations), sink.data_ptr(), _stream_ptr(stream, sink.device))
    if rc != CTX_OK:
        raise error_for(lib, rc)
    return workgroups * 4 * iterations * MFMA_FLOPS_PER_WAVE_ROUND[shape]
