"""ctypes binding of libjf (include/jf.h) -- argument marshalling only.

Every function of the C ABI is exposed under its own name on ``lib()``; the
``Model`` class is a thin owner of the device buffers the ABI asks for
(allocated with torch, which is used here only for device memory and
streams).  No step of the decoding path runs in Python: each call below is
one ABI call that enqueues HIP kernels.
"""
from __future__ import annotations

import ctypes
import functools
import os
from operator import index

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libjf.so")

JF_OK, JF_E_INVAL, JF_E_SHAPE, JF_E_CAPACITY, JF_E_DTYPE, JF_E_HIP, JF_E_STATE = 0, -1, -2, -3, -4, -5, -6
JF_F32, JF_BF16, JF_E4M3 = 0, 1, 2
JF_ROLE_RA, JF_ROLE_CAND, JF_ROLE_PSEUDO = 0, 1, 2
JF_MAX_SEGMENTS = 16
JF_MAX_ROWS = 512      # rows of one step at most
JF_STEP_COMMIT = 2     # jf_jacobi_step mode bit: commit the accepted rows in the step
JF_VIS_WORDS = 8       # u64 words of a row's in-step visibility mask
JF_PAGE = 64           # cache slots of a page
JF_FLAG_BAD_TOKEN, JF_FLAG_CAPACITY, JF_FLAG_SYNC, JF_FLAG_BAD_PAGE = 1, 2, 4, 8
JF_MAX_TOP = 32        # alternatives of jf_token_logprobs at most
JF_OPT_FUSED_ATTENTION = 1
JF_MASK_NOISY_CONTEXT, JF_MASK_CLEAN_CONTEXT = 0, 1
JF_MEAN_TOKENS, JF_MEAN_SEQS, JF_SUM = 0, 1, 2
JF_POLICY_STATS = 6    # loss, then the means of policy term, KL, entropy and clipped rows, then tokens
(JF_KERNEL_QKV, JF_KERNEL_ATTN, JF_KERNEL_O, JF_KERNEL_GATEUP, JF_KERNEL_DOWN, JF_KERNEL_LMHEAD,
 JF_KERNEL_STEP, JF_KERNEL_ATTN_BLOCK) = range(1, 9)
STATUS_NAMES = {0: "JF_OK", -1: "JF_E_INVAL", -2: "JF_E_SHAPE", -3: "JF_E_CAPACITY",
                -4: "JF_E_DTYPE", -5: "JF_E_HIP", -6: "JF_E_STATE"}


def act_layout(x):
    """[R][K] row-major -> the GEMM-input activation layout of include/jf.h.

    Rows are padded to a multiple of 16 (padding rows are zero); the result
    is flat, ceil(R/16)*16*K elements.  K must be a multiple of 128.
    """
    x = np.asarray(x)
    R, K = x.shape
    Rp = (R + 15) // 16 * 16
    xp = np.zeros((Rp, K), x.dtype)
    xp[:R] = x
    # [tile, r, kc, q, j, e] -> [tile, kc, j, q, r, e]  (lane = 16 q + r)
    return np.ascontiguousarray(
        xp.reshape(Rp // 16, 16, K // 128, 4, 4, 8).transpose(0, 2, 4, 3, 1, 5)).reshape(-1)


def act_unlayout(a, R, K):
    """Inverse of act_layout: the first R rows as an [R][K] array."""
    a = np.asarray(a)
    Rp = (R + 15) // 16 * 16
    t = a[:Rp * K].reshape(Rp // 16, K // 128, 4, 4, 16, 8).transpose(0, 4, 1, 3, 2, 5)
    return np.ascontiguousarray(t).reshape(Rp, K)[:R]


class JfConfig(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32),
                ("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("d_ffn", ctypes.c_int32),
                ("vocab", ctypes.c_int32), ("rope_base", ctypes.c_float),
                ("rms_eps", ctypes.c_float), ("dtype", ctypes.c_int32),
                ("max_rows", ctypes.c_int32), ("max_ctx", ctypes.c_int32)]


class JfSegment(ctypes.Structure):
    _fields_ = [("first_row", ctypes.c_int32), ("n_rows", ctypes.c_int32),
                ("attach_row", ctypes.c_int32), ("role", ctypes.c_int32),
                ("verify_from", ctypes.c_int32)]


class JfBatch(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("n_rows", ctypes.c_int32), ("max_rows", ctypes.c_int32),
                ("max_ctx", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("table_stride", ctypes.c_int32),
                ("d_row_start", ctypes.c_void_p), ("d_ctx", ctypes.c_void_p), ("d_page_table", ctypes.c_void_p)]


class JfPrefix(ctypes.Structure):
    _fields_ = [("n_groups", ctypes.c_int32), ("max_rows", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("d_seq_start", ctypes.c_void_p), ("d_pages", ctypes.c_void_p)]


class JfPolicy(ctypes.Structure):
    _fields_ = [("clip_low", ctypes.c_double), ("clip_high", ctypes.c_double), ("kl_weight", ctypes.c_double),
                ("entropy_weight", ctypes.c_double), ("scale", ctypes.c_double), ("mean", ctypes.c_int32),
                ("adv_rows", ctypes.c_int32)]


class JfError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


_LIB = None
P, I32, U64, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint64, ctypes.c_size_t
I64, F64, PB = ctypes.c_int64, ctypes.c_double, ctypes.POINTER(JfBatch)
PX, PY = ctypes.POINTER(JfPrefix), ctypes.POINTER(JfPolicy)
_SIGS = {
    "jf_query_sizes": (I32, [ctypes.POINTER(JfConfig), ctypes.POINTER(SZ), ctypes.POINTER(SZ), ctypes.POINTER(SZ)]),
    "jf_model_load": (I32, [ctypes.POINTER(JfConfig), ctypes.POINTER(P), I32, P, P, P, P, ctypes.POINTER(P)]),
    "jf_model_free": (I32, [P]),
    "jf_last_error": (ctypes.c_char_p, []),
    "jf_prefill": (I32, [P, P, I32, P, P]),
    "jf_jacobi_step": (I32, [P, P, I32, I32, U64, P, P, P, P, P]),
    "jf_multiblock_step": (I32, [P, P, I32, ctypes.POINTER(JfSegment), I32, P, P, P, P, P, P]),
    "jf_commit_kv": (I32, [P, P, P, I32, P]),
    "jf_kv_length": (I32, [P, ctypes.POINTER(I32), P]),
    "jf_kv_truncate": (I32, [P, I32, P]),
    "jf_kv_set_page_table": (I32, [P, ctypes.POINTER(I32), I32, P]),
    "jf_model_set_option": (I32, [P, I32, I32]),
    "jf_profile_begin": (I32, [P, I32]),
    "jf_profile_end": (I32, [P, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(I32)]),
    "jf_attention_ws_bytes": (SZ, [I32, I32, I32]),
    "jf_attention": (I32, [I32, I32, I32, I32, I32, I32, P, P, P, P, P, P, P]),
    "jf_packed_matrix_bytes": (SZ, [I32, I32, I32]),
    "jf_pack_matrix": (I32, [I32, I32, I32, P, P, P]),
    "jf_lm_head_ws_bytes": (SZ, [I32, I32]),
    "jf_lm_head_accept": (I32, [I32, I32, I32, I32, P, P, P, P, P, P, P, P]),
    "jf_lm_head_accept_noalloc": (I32, [I32, I32, I32, I32, P, P, P, P, P, P, P]),
    "jf_packed_forward": (I32, [P, P, I32, I32, I32, P, P, P]),
    "jf_trajectory_record": (I32, [P, P, I32, I32, P, P]),
    "jf_trajectory_select": (I32, [P, P, I32, I32, I32, I32, P, P, P, P]),
    "jf_kv_page_bytes": (SZ, [I32, I32, I32]),
    "jf_kv_append": (I32, [PB, I32, I32, I32, I32, I32, I32, P, I64, P, I64, P, I64, P, F64, P, P, P, P]),
    "jf_kv_read": (I32, [PB, I32, I32, I32, I32, P, P, I64, P, I64, P, P]),
    "jf_attention_kv8_ws_bytes": (SZ, [PB, I32, I32, I32]),
    "jf_attention_kv8": (I32, [PB, I32, I32, I32, I32, P, P, P, P, P, P, P]),
    "jf_token_logprobs_ws_bytes": (SZ, [I32, I32, I32]),
    "jf_token_logprobs": (I32, [I32, I32, I32, P, I64, P, I32, P, P, P, P, P, P, P]),
    "jf_token_logprobs_grad": (I32, [I32, I32, I32, P, I64, P, P, P, P, P, P, I64, P]),
    "jf_attention_causal": (I32, [I32, I32, P, I32, I32, I32, I32, P, I64, P, I64, P, I64, P, I64, P, P, P]),
    "jf_attention_causal_grad_ws_bytes": (SZ, [I32, I32, I32, I32, I32]),
    "jf_attention_causal_grad": (I32, [I32, I32, P, I32, I32, I32, I32, P, I64, P, I64, P, I64, P, I64, P, P, I64, P, I64,
                                       P, I64, P, I64, P, P, P]),
    "jf_attention_shared_ws_bytes": (SZ, [PB, PX, I32, I32, I32]),
    "jf_attention_shared": (I32, [PB, PX, I32, I32, I32, I32, P, P, P, P, P, P, P]),
    "jf_policy_loss_ws_bytes": (SZ, [I32, I32]),
    "jf_policy_loss": (I32, [PY, I32, I32, P, P, P, P, P, P, P, P, P, P, P, P, P]),
}
EXPORTS = tuple(_SIGS)


def lib():
    """The loaded libjf; raises if it has not been built (no fallback)."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2512_14681_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        _LIB = L
    return _LIB


def check(status):
    if status != JF_OK:
        raise JfError(status, lib().jf_last_error().decode())
    return status


def config(shape: dict, max_rows: int, max_ctx: int) -> JfConfig:
    return JfConfig(shape["n_layers"], shape["d_model"], shape["n_heads"], shape["n_kv_heads"],
                    shape["head_dim"], shape["d_ffn"], shape["vocab"], float(shape["rope_base"]),
                    float(shape["rms_eps"]), JF_BF16 if shape["dtype"] == "bf16" else JF_F32,
                    int(max_rows), int(max_ctx))


def query_sizes(cfg: JfConfig):
    a, b, c = SZ(), SZ(), SZ()
    check(lib().jf_query_sizes(ctypes.byref(cfg), ctypes.byref(a), ctypes.byref(b), ctypes.byref(c)))
    return a.value, b.value, c.value


def weight_names(shape: dict):
    """Weight tensors in the order jf_model_load takes them."""
    names = ["embed"]
    for l in range(shape["n_layers"]):
        names += [f"layers.{l}.{k}" for k in ("attn_norm", "wq", "wk", "wv", "wo", "ffn_norm",
                                               "w_gate", "w_up", "w_down")]
    return names + ["final_norm", "lm_head"]


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def segments(segs):
    """Host array of jf_segment from (first, n_rows, attach, role, verify_from) tuples."""
    arr = (JfSegment * len(segs))()
    for i, s in enumerate(segs):
        arr[i] = JfSegment(*[int(v) for v in s])
    return arr


class Model:
    """Device buffers of one libjf model (one sequence) and its ABI calls."""

    def __init__(self, shape: dict, weights: dict, max_rows: int, max_ctx: int, device="cuda",
                 stream=None):
        import torch
        self.torch = torch
        self.shape = dict(shape)
        self.cfg = config(shape, max_rows, max_ctx)
        self.stream = stream
        packed, kv, ws = query_sizes(self.cfg)
        self.packed = torch.empty(packed, dtype=torch.uint8, device=device)
        self.kv = torch.empty(kv, dtype=torch.uint8, device=device)
        self.ws = torch.empty(ws, dtype=torch.uint8, device=device)
        names = weight_names(shape)
        dev = []
        for n in names:
            a = np.ascontiguousarray(weights[n])
            t = torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).to(device)
            dev.append(t)
        ptrs = (ctypes.c_void_p * len(dev))(*[t.data_ptr() for t in dev])
        h = ctypes.c_void_p()
        check(lib().jf_model_load(ctypes.byref(self.cfg), ptrs, len(dev), _ptr(self.packed),
                                  _ptr(self.kv), _ptr(self.ws), _stream(stream), ctypes.byref(h)))
        self.h = h
        del dev
        self.V = shape["vocab"]

    def __del__(self):
        try:
            if getattr(self, "h", None):
                lib().jf_model_free(self.h)
                self.h = None
        except Exception:
            pass

    # ---- ABI calls (device tensors in, device tensors out) ----------------
    def jf_prefill(self, d_tokens, d_pending):
        check(lib().jf_prefill(self.h, _ptr(d_tokens), int(d_tokens.numel()), _ptr(d_pending),
                               _stream(self.stream)))

    def jf_jacobi_step(self, d_draft, n, mode, pad_seed, d_argmax, d_result, d_next, d_logits=None):
        check(lib().jf_jacobi_step(self.h, _ptr(d_draft), int(n), int(mode), int(pad_seed),
                                   _ptr(d_argmax), _ptr(d_result), _ptr(d_next), _ptr(d_logits),
                                   _stream(self.stream)))

    def jf_multiblock_step(self, d_tokens, R, segs, d_argmax, d_seg_accept, d_result, d_path,
                           d_logits=None):
        arr = segments(segs)
        check(lib().jf_multiblock_step(self.h, _ptr(d_tokens), int(R), arr, len(segs), _ptr(d_argmax),
                                       _ptr(d_seg_accept), _ptr(d_result), _ptr(d_path),
                                       _ptr(d_logits), _stream(self.stream)))

    def jf_packed_forward(self, d_tokens, n_blocks, n, mask, d_argmax, d_logits=None):
        check(lib().jf_packed_forward(self.h, _ptr(d_tokens), int(n_blocks), int(n), int(mask),
                                      _ptr(d_argmax), _ptr(d_logits), _stream(self.stream)))

    def jf_commit_kv(self, d_path, d_result, max_commit=0):
        check(lib().jf_commit_kv(self.h, _ptr(d_path), _ptr(d_result), int(max_commit),
                                 _stream(self.stream)))

    def jf_kv_length(self):
        v = ctypes.c_int32()
        check(lib().jf_kv_length(self.h, ctypes.byref(v), _stream(self.stream)))
        return v.value

    def jf_kv_truncate(self, n):
        check(lib().jf_kv_truncate(self.h, int(n), _stream(self.stream)))

    def jf_model_set_option(self, option, value):
        check(lib().jf_model_set_option(self.h, int(option), int(value)))

    def jf_profile_begin(self, kernel_class):
        check(lib().jf_profile_begin(self.h, int(kernel_class)))

    def jf_profile_end(self):
        t, n = ctypes.c_double(), ctypes.c_int32()
        check(lib().jf_profile_end(self.h, ctypes.byref(t), ctypes.byref(n)))
        return t.value, n.value

    def jf_kv_set_page_table(self, table):
        t = np.ascontiguousarray(table, dtype=np.int32)
        check(lib().jf_kv_set_page_table(self.h, t.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
                                         len(t), _stream(self.stream)))


# ---- trajectories (component calls, no model) ------------------------------------
def trajectory_record(d_prev, d_argmax, n, rows, d_out, stream=None):
    check(lib().jf_trajectory_record(_ptr(d_prev), _ptr(d_argmax), int(n), int(rows), _ptr(d_out),
                                     _stream(stream)))


def trajectory_select(d_traj, d_len, n_blocks, n, max_points, w, d_sel, d_t_num=None, d_unconv=None,
                      stream=None):
    check(lib().jf_trajectory_select(_ptr(d_traj), _ptr(d_len), int(n_blocks), int(n), int(max_points),
                                     int(w), _ptr(d_t_num), _ptr(d_sel), _ptr(d_unconv), _stream(stream)))


# ---- batches of sequences over a paged cache, log probabilities (component calls) -----
_DTYPES = {}


def _types():
    """{torch dtype: jf_dtype} of rows, and int32; torch is imported at the first use."""
    if not _DTYPES:
        import torch
        global _I32, _F32, _U8, _ACT, _current_device, _raw_stream
        _I32, _F32, _U8 = torch.int32, torch.float32, torch.uint8
        _ACT = {JF_F32: torch.float32, JF_BF16: torch.bfloat16}
        # the stream's address without a Stream object around it (2.7 us a call)
        _current_device, _raw_stream = torch.cuda.current_device, torch._C._cuda_getCurrentRawStream
        # last: who finds a type here (in another thread) finds the names above too
        _DTYPES.update({torch.float32: JF_F32, torch.bfloat16: JF_BF16})
    return _DTYPES


def _at(dev, t):
    """Address of a tensor on the current GPU; None stays None."""
    if t is None:
        return None
    if t.get_device() != dev:
        raise ValueError(f"a tensor is on {t.device}, the call runs on GPU {dev}")
    return t.data_ptr()


def _vec(dev, t, dtype, n):
    """Address of a contiguous tensor of n elements or more."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() < n or not t.is_contiguous():
        raise TypeError(f"expected a contiguous {dtype} tensor of {n} elements, got {tuple(t.shape)} of {t.dtype}")
    return _at(dev, t)


def _buf(dev, t, n):
    """Address of a contiguous tensor of n bytes or more."""
    if t is None:
        return None
    if t.nbytes < n or not t.is_contiguous():
        raise ValueError(f"expected a contiguous tensor of {n} bytes, got {tuple(t.shape)} of {t.dtype}")
    return _at(dev, t)


def _act(dev, t, act_dtype, n):
    """Address of activation planes of act_dtype in a contiguous tensor of that type (or raw bytes), n bytes or more."""
    if t is None:
        return None
    if t.dtype is not _ACT.get(act_dtype, t.dtype) and t.dtype is not _U8:
        raise TypeError(f"expected activation planes of jf_dtype {act_dtype}, got {t.dtype}")
    if t.nbytes < n or not t.is_contiguous():
        raise ValueError(f"expected a contiguous tensor of {n} bytes, got {tuple(t.shape)} of {t.dtype}")
    return _at(dev, t)


def _rows(t, least=0, width=1):
    """(jf_dtype, row stride in elements) of a [rows][columns] tensor of fp32 or bf16 whose rows are contiguous,
    `least` of them or more with `width` columns or more."""
    code = _DTYPES.get(t.dtype)
    if code is None:
        code = _types().get(t.dtype)
    if code is None or t.dim() != 2:
        raise TypeError("rows are 2-dimensional fp32 or bf16 tensors")
    (n, w), (ld, step) = t.shape, t.stride()
    if step != 1 and w > 1:
        raise TypeError("a row's elements lie side by side")
    if n < least or w < width:
        raise ValueError(f"expected {least} rows of {width} columns, got {n} of {w}")
    if n <= 1 and ld < w:   # the stride of a single row says nothing
        ld = w
    return code, ld


def _count(*counts):
    """Refuses what a 32-bit argument would take for another number."""
    for n in counts:
        if not -1 << 31 <= n < 1 << 31:
            raise JfError(JF_E_CAPACITY, f"{n} does not fit 32 bits")


def _on(dev, stream):
    return _raw_stream(dev) if stream is None else stream.cuda_stream


class Batch:
    """A jf_batch over device int32 tensors (kept alive here): row_start [n_seqs + 1], ctx [n_seqs] and
    page_table [n_seqs][stride], with the host's bounds."""

    def __init__(self, row_start, ctx, page_table, n_rows, max_rows, max_ctx, n_pages):
        _types()
        self.tensors = (row_start, ctx, page_table)
        for t in self.tensors:
            if t.dtype is not _I32 or not t.is_contiguous():
                raise TypeError("row_start, ctx and page_table are contiguous int32 tensors")
        n = ctx.numel()
        if row_start.numel() != n + 1 or page_table.dim() != 2 or page_table.shape[0] != n:
            raise ValueError(f"{n} sequences need {n + 1} row starts and {n} rows of the page table")
        if not ctx.get_device() == row_start.get_device() == page_table.get_device():
            raise ValueError("row_start, ctx and page_table are on one device")
        _count(n, int(n_rows), min(int(max_rows), int(max_ctx)), int(max_ctx), int(n_pages), page_table.shape[1])
        self.device, self.n_rows, self.n_pages = ctx.get_device(), int(n_rows), int(n_pages)
        # a looser bound on the rows than the slots allow is no other bound
        self.c = JfBatch(n, self.n_rows, min(int(max_rows), int(max_ctx)), int(max_ctx), int(n_pages), int(page_table.shape[1]),
                         row_start.data_ptr(), ctx.data_ptr(), page_table.data_ptr())
        self.ref = ctypes.byref(self.c)
        self.ws = {}    # {(n_heads, n_kv_heads, head_dim): bytes of attention_kv8's workspace}

    def on(self, dev):
        if self.device != dev:
            raise ValueError(f"the batch is on device {self.device}, the call runs on GPU {dev}")
        return self.ref


def kv_page_bytes(n_kv_heads, head_dim, kv_dtype):
    return lib().jf_kv_page_bytes(int(n_kv_heads), int(head_dim), int(kv_dtype))


def _pool_bytes(batch, n_kv_heads, head_dim, kv_dtype):
    """batch.n_pages of kv_page_bytes (without the call, half a microsecond)."""
    n = 2 * JF_PAGE * n_kv_heads * head_dim
    if kv_dtype == JF_E4M3:
        return batch.n_pages * ((n + 8 * n_kv_heads + 127) // 128 * 128)
    return batch.n_pages * n * (4 if kv_dtype == JF_F32 else 2)


def kv_append(batch, n_heads, n_kv_heads, head_dim, kv_dtype, d_kv, d_k, d_v, d_q=None, d_q_out=None,
              act_dtype=JF_BF16, d_pos=None, rope_base=0.0, d_flags=None, stream=None):
    n, w = batch.n_rows, n_kv_heads * head_dim
    x, ld_k = _rows(d_k, n, w)
    xv, ld_v = _rows(d_v, n, w)
    xq, ld_q = _rows(d_q, n, n_heads * head_dim) if d_q is not None else (x, 0)
    if not x == xv == xq:
        raise TypeError("queries, keys and values have one type")
    dev = _current_device()
    status = lib().jf_kv_append(batch.on(dev), n_heads, n_kv_heads, head_dim, kv_dtype, x, act_dtype, _at(dev, d_q),
                                ld_q, _at(dev, d_k), ld_k, _at(dev, d_v), ld_v, _vec(dev, d_pos, _I32, n), rope_base,
                                _buf(dev, d_kv, _pool_bytes(batch, n_kv_heads, head_dim, kv_dtype)),
                                _act(dev, d_q_out, act_dtype, 4 * n * n_heads * head_dim),  # fp32, or two bf16 planes
                                _vec(dev, d_flags, _I32, 1), _on(dev, stream))
    if status:
        check(status)


def kv_read(batch, n_kv_heads, head_dim, kv_dtype, d_kv, d_k, d_v, d_flags=None, stream=None):
    n, w = batch.n_rows, n_kv_heads * head_dim
    x, ld_k = _rows(d_k, n, w)
    xv, ld_v = _rows(d_v, n, w)
    if x != xv:
        raise TypeError("keys and values have one type")
    dev = _current_device()
    status = lib().jf_kv_read(batch.on(dev), n_kv_heads, head_dim, kv_dtype, x,
                              _buf(dev, d_kv, _pool_bytes(batch, n_kv_heads, head_dim, kv_dtype)), _at(dev, d_k), ld_k,
                              _at(dev, d_v), ld_v, _vec(dev, d_flags, _I32, 1), _on(dev, stream))
    if status:
        check(status)


def _kv8_ws_bytes(batch, n_heads, n_kv_heads, head_dim):
    shape = index(n_heads), index(n_kv_heads), index(head_dim)
    n = batch.ws.get(shape)
    if n is None:
        n = batch.ws[shape] = lib().jf_attention_kv8_ws_bytes(batch.ref, *shape)
    return n


def attention_kv8_ws_bytes(batch, n_heads, n_kv_heads, head_dim):
    n = _kv8_ws_bytes(batch, n_heads, n_kv_heads, head_dim)
    if n == 0:
        raise JfError(JF_E_SHAPE, "no batch or heads that jf_attention_kv8 takes")
    return n


def attention_kv8(batch, n_heads, n_kv_heads, head_dim, act_dtype, d_q, d_kv, d_out, d_ws, d_vis=None, d_flags=None,
                  stream=None):
    dev, n = _current_device(), batch.n_rows
    row = 4 * n_heads * head_dim        # bytes: fp32, or two bf16 planes
    status = lib().jf_attention_kv8(batch.on(dev), n_heads, n_kv_heads, head_dim, act_dtype,
                                    _act(dev, d_q, act_dtype, n * row),
                                    _buf(dev, d_kv, _pool_bytes(batch, n_kv_heads, head_dim, JF_E4M3)),
                                    _buf(dev, d_vis, n * 8 * JF_VIS_WORDS),
                                    _act(dev, d_out, act_dtype, (n + 15) // 16 * 16 * row),  # 16 rows a tile
                                    _buf(dev, d_ws, _kv8_ws_bytes(batch, n_heads, n_kv_heads, head_dim)),
                                    _vec(dev, d_flags, _I32, 1), _on(dev, stream))
    if status:
        check(status)


# Sizes and parameters are remembered by their numbers: a tensor that changes in place stays the same key.
@functools.lru_cache(4096)
def _logprobs_ws(R, V, k):
    _count(R, V, k)
    return lib().jf_token_logprobs_ws_bytes(R, V, k)


def token_logprobs_ws_bytes(R, V, k=0):
    return _logprobs_ws(int(R), int(V), int(k))


def token_logprobs(d_logits, d_ws, d_tokens=None, k=0, d_logprob=None, d_entropy=None, d_norm=None, d_top_ids=None,
                   d_top_logprob=None, stream=None):
    x, ld = _rows(d_logits)
    R, V = d_logits.shape
    dev = _current_device()
    status = lib().jf_token_logprobs(R, V, x, _at(dev, d_logits), ld, _vec(dev, d_tokens, _I32, R), k,
                                     _vec(dev, d_logprob, _F32, R), _vec(dev, d_entropy, _F32, R),
                                     _vec(dev, d_norm, _F32, 2 * R), _vec(dev, d_top_ids, _I32, R * k),
                                     _vec(dev, d_top_logprob, _F32, R * k),
                                     _buf(dev, d_ws, token_logprobs_ws_bytes(R, V, k)), _on(dev, stream))
    if status:
        check(status)


def token_logprobs_grad(d_logits, d_norm, d_grad, d_tokens=None, d_entropy=None, d_g_logprob=None, d_g_entropy=None,
                        stream=None):
    x, ld = _rows(d_logits)
    xg, ld_g = _rows(d_grad)
    if x != xg or d_grad.shape != d_logits.shape:
        raise TypeError("the gradient has the logits' shape and type")
    R, V = d_logits.shape
    _count(R, V)
    dev = _current_device()
    status = lib().jf_token_logprobs_grad(R, V, x, _at(dev, d_logits), ld, _vec(dev, d_tokens, _I32, R),
                                          _vec(dev, d_norm, _F32, 2 * R), _vec(dev, d_entropy, _F32, R),
                                          _vec(dev, d_g_logprob, _F32, R), _vec(dev, d_g_entropy, _F32, R),
                                          _at(dev, d_grad), ld_g, _on(dev, stream))
    if status:
        check(status)


# ---- training on sampled groups: causal attention, shared prefixes, policy loss (component calls) -----
def _starts(dev, t):
    """(address, sequences) of row starts [n_seqs + 1] on the current GPU."""
    if t.dtype is not _I32 or not t.is_contiguous() or t.numel() < 1:
        raise TypeError("row starts are a contiguous int32 tensor of one element more than there are sequences")
    return _at(dev, t), t.numel() - 1


def attention_causal(d_row_start, n_heads, n_kv_heads, head_dim, d_q, d_k, d_v, d_out, d_lse=None, d_flags=None,
                     stream=None):
    """Rows of d_q [rows][n_heads * head_dim] over those of d_k and d_v up to their own, sequence by sequence, to d_out;
    d_lse [n_heads][rows] for attention_causal_grad."""
    wide, narrow = n_heads * head_dim, n_kv_heads * head_dim
    x, ld_q = _rows(d_q, 0, wide)
    n = d_q.shape[0]
    xo, ld_out = _rows(d_out, n, wide)
    xk, ld_k = _rows(d_k, n, narrow)
    xv, ld_v = _rows(d_v, n, narrow)
    if not x == xo == xk == xv:
        raise TypeError("all rows have one type")
    dev = _current_device()
    start, n_seqs = _starts(dev, d_row_start)
    _count(n, n_seqs)
    status = lib().jf_attention_causal(n_seqs, n, start, n_heads, n_kv_heads, head_dim, x, _at(dev, d_q), ld_q,
                                       _at(dev, d_k), ld_k, _at(dev, d_v), ld_v, _at(dev, d_out), ld_out,
                                       _vec(dev, d_lse, _F32, n_heads * n), _vec(dev, d_flags, _I32, 1),
                                       _on(dev, stream))
    if status:
        check(status)


@functools.lru_cache(4096)
def _causal_grad_ws(n_seqs, n_rows, n_heads, n_kv_heads, head_dim):
    _count(n_seqs, n_rows)
    n = lib().jf_attention_causal_grad_ws_bytes(n_seqs, n_rows, n_heads, n_kv_heads, head_dim)
    if n == 0:
        raise JfError(JF_E_SHAPE, "no rows or heads that jf_attention_causal_grad takes")
    return n


def attention_causal_grad_ws_bytes(n_seqs, n_rows, n_heads, n_kv_heads, head_dim):
    return _causal_grad_ws(index(n_seqs), index(n_rows), index(n_heads), index(n_kv_heads), index(head_dim))


def attention_causal_grad(d_row_start, n_heads, n_kv_heads, head_dim, d_q, d_k, d_v, d_out, d_lse, d_g_out, d_g_q, d_g_k,
                          d_g_v, d_ws, d_flags=None, stream=None):
    """Gradient of sum(d_g_out * d_out) to queries, keys and values, from attention_causal's inputs and outputs."""
    wide, narrow = n_heads * head_dim, n_kv_heads * head_dim
    x, ld_q = _rows(d_q, 0, wide)
    n = d_q.shape[0]
    (xo, ld_out), (xg, ld_g), (x1, ld_gq) = _rows(d_out, n, wide), _rows(d_g_out, n, wide), _rows(d_g_q, n, wide)
    (xk, ld_k), (xv, ld_v) = _rows(d_k, n, narrow), _rows(d_v, n, narrow)
    (x2, ld_gk), (x3, ld_gv) = _rows(d_g_k, n, narrow), _rows(d_g_v, n, narrow)
    if not x == xo == xg == x1 == xk == xv == x2 == x3:
        raise TypeError("all rows have one type")
    dev = _current_device()
    start, n_seqs = _starts(dev, d_row_start)
    status = lib().jf_attention_causal_grad(
        n_seqs, n, start, n_heads, n_kv_heads, head_dim, x, _at(dev, d_q), ld_q, _at(dev, d_k), ld_k, _at(dev, d_v), ld_v,
        _at(dev, d_out), ld_out, _vec(dev, d_lse, _F32, n_heads * n), _at(dev, d_g_out), ld_g, _at(dev, d_g_q), ld_gq,
        _at(dev, d_g_k), ld_gk, _at(dev, d_g_v), ld_gv,
        _buf(dev, d_ws, attention_causal_grad_ws_bytes(n_seqs, n, n_heads, n_kv_heads, head_dim)),
        _vec(dev, d_flags, _I32, 1), _on(dev, stream))
    if status:
        check(status)


class Prefix:
    """A jf_prefix over device int32 tensors (kept alive here): seq_start [n_groups + 1] and pages [n_groups], with the
    host's bounds on the rows and the shared pages of a group."""

    def __init__(self, seq_start, pages, max_rows, max_pages):
        _types()
        self.tensors = (seq_start, pages)
        for t in self.tensors:
            if t.dtype is not _I32 or not t.is_contiguous():
                raise TypeError("seq_start and pages are contiguous int32 tensors")
        n = pages.numel()
        if seq_start.numel() != n + 1:
            raise ValueError(f"{n} groups need {n + 1} sequence starts")
        if pages.get_device() != seq_start.get_device():
            raise ValueError("seq_start and pages are on one device")
        _count(n, int(max_rows), int(max_pages))
        self.device = pages.get_device()
        self.c = JfPrefix(n, int(max_rows), int(max_pages), seq_start.data_ptr(), pages.data_ptr())
        self.ref = ctypes.byref(self.c)

    def on(self, dev):
        if self.device != dev:
            raise ValueError(f"the prefix is on device {self.device}, the call runs on GPU {dev}")
        return self.ref


def _shared_ws_bytes(batch, prefix, n_heads, n_kv_heads, head_dim):
    shape = "shared", index(n_heads), index(n_kv_heads), index(head_dim)
    key = shape if prefix is None else shape + (prefix.c.n_groups, prefix.c.max_rows, prefix.c.max_pages)
    n = batch.ws.get(key)
    if n is None:
        n = lib().jf_attention_shared_ws_bytes(batch.ref, None if prefix is None else prefix.ref, *shape[1:])
        batch.ws[key] = n
    return n


def attention_shared_ws_bytes(batch, prefix, n_heads, n_kv_heads, head_dim):
    n = _shared_ws_bytes(batch, prefix, n_heads, n_kv_heads, head_dim)
    if n == 0:
        raise JfError(JF_E_SHAPE, "no batch, prefix or heads that jf_attention_shared takes")
    return n


def attention_shared(batch, prefix, n_heads, n_kv_heads, head_dim, dtype, d_q, d_kv, d_out, d_ws, d_vis=None,
                     d_flags=None, stream=None):
    """Attention of a batch over a paged cache of dtype, the pages that groups of its sequences share read once for all
    rows of a group (prefix None: nothing is shared)."""
    dev, n = _current_device(), batch.n_rows
    row = 4 * n_heads * head_dim        # bytes: fp32, or two bf16 planes
    status = lib().jf_attention_shared(batch.on(dev), None if prefix is None else prefix.on(dev), n_heads, n_kv_heads,
                                       head_dim, dtype, _act(dev, d_q, dtype, n * row),
                                       _buf(dev, d_kv, _pool_bytes(batch, n_kv_heads, head_dim, dtype)),
                                       _buf(dev, d_vis, n * 8 * JF_VIS_WORDS),
                                       _act(dev, d_out, dtype, (n + 15) // 16 * 16 * row),  # 16 rows a tile
                                       _buf(dev, d_ws, _shared_ws_bytes(batch, prefix, n_heads, n_kv_heads, head_dim)),
                                       _vec(dev, d_flags, _I32, 1), _on(dev, stream))
    if status:
        check(status)


@functools.lru_cache(4096)
def _policy_ws(n_seqs, n_rows):
    _count(n_seqs, n_rows)
    n = lib().jf_policy_loss_ws_bytes(n_seqs, n_rows)
    if n == 0:
        raise JfError(JF_E_CAPACITY, "more sequences or rows than jf_policy_loss takes")
    return n


def policy_loss_ws_bytes(n_seqs, n_rows):
    return _policy_ws(index(n_seqs), index(n_rows))


@functools.lru_cache(256)
def _policy(*fields):
    return JfPolicy(*fields)


def policy_loss(d_row_start, d_tokens, d_logprob, d_old_logprob, d_advantage, d_stats, d_ws, d_ref_logprob=None,
                d_entropy=None, d_g_logprob=None, d_g_entropy=None, clip_low=0.2, clip_high=0.2, kl_weight=0.0,
                entropy_weight=0.0, scale=1.0, mean=JF_MEAN_TOKENS, adv_rows=False, d_flags=None, stream=None):
    """Clipped policy loss over the tokens of sampled sequences: d_stats [JF_POLICY_STATS] and, where given, its gradient
    to the log probabilities and entropies of token_logprobs.  d_advantage has one element a sequence, or one a row
    (adv_rows); d_tokens None: every row has a token."""
    _types()
    n = d_logprob.numel()
    dev = _current_device()
    start, n_seqs = _starts(dev, d_row_start)
    params = _policy(float(clip_low), float(clip_high), float(kl_weight), float(entropy_weight), float(scale), index(mean),
                     1 if adv_rows else 0)
    status = lib().jf_policy_loss(ctypes.byref(params), n_seqs, n, start, _vec(dev, d_tokens, _I32, n),
                                  _vec(dev, d_logprob, _F32, n), _vec(dev, d_old_logprob, _F32, n),
                                  _vec(dev, d_ref_logprob, _F32, n), _vec(dev, d_entropy, _F32, n),
                                  _vec(dev, d_advantage, _F32, n if adv_rows else n_seqs),
                                  _vec(dev, d_stats, _F32, JF_POLICY_STATS),
                                  _vec(dev, d_g_logprob, _F32, n),
                                  _vec(dev, d_g_entropy, _F32, n), _buf(dev, d_ws, policy_loss_ws_bytes(n_seqs, n)),
                                  _vec(dev, d_flags, _I32, 1), _on(dev, stream))
    if status:
        check(status)
