"""Thin ctypes binding of libtreekv.so: argument marshalling only.

Function names match include/treekv.h.  `TreeKV` is a convenience wrapper that owns the device workspace as a
torch tensor and passes torch tensors' device pointers and the current CUDA stream; every step of the path runs
in the library's kernels.  There is no CPU fallback: if the shared library cannot be loaded the import of this
module fails.
"""
from __future__ import annotations

import ctypes as C
import os
from array import array as _array

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtreekv.so")

TREEKV_OK = 0
TREEKV_F32, TREEKV_BF16 = 0, 1
RULE_SCORES, RULE_KEEP_LEFT, RULE_EVICT_LEFT, RULE_ACCUMULATED = 0, 1, 2, 3
OPT_DECODE_SPLIT, OPT_PREFILL_PATH, OPT_DECODE_PATH, OPT_PREFILL_APPEND, OPT_EVICTION_STREAM = 0, 1, 2, 3, 4
OPT_PREFILL_KEY_SPLIT = 5

# every symbol include/treekv.h declares
EXPORTS = [
    "treekv_workspace_bytes", "treekv_create", "treekv_decode_step", "treekv_prefill_chunk",
    "treekv_decode_step_host", "treekv_prefill_chunk_host", "treekv_prefill_chunk_static_scratch", "treekv_retained_positions", "treekv_scores",
    "treekv_get_stats", "treekv_tokens_seen", "treekv_set_rule", "treekv_set_option", "treekv_reset",
    "treekv_destroy", "treekv_status_string", "treekv_version",
    "treekv_state_bytes", "treekv_export_state", "treekv_import_state", "treekv_selftest_wait_giveup",
    "treekv_set_protection", "treekv_prefill_oneshot", "treekv_set_positions",
    "treekv_norm_rope", "treekv_verify_tree", "treekv_accept_path", "treekv_fork_sequences", "treekv_selftest_fork_plan",
    "treekv_paged_scratch_bytes", "treekv_paged_attend", "treekv_paged_score", "treekv_adopt_pages", "treekv_pick_path",
]


class TreeKVStats(C.Structure):
    _fields_ = [
        ("evictions", C.c_uint64),
        ("near_ties", C.c_uint64),
        ("kernel_launches", C.c_uint64),
        ("device_error", C.c_uint32),
        ("last_cuda_error", C.c_int32),
    ]


class TreeKVError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        super().__init__("%s failed: %s (status %d)" % (what, status_string(status), status))


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            "libtreekv.so is missing at %s; build it with `python -m paper_2501_04987_b200._build` "
            "(there is no CPU fallback)" % LIB_PATH
        )
    lib = C.CDLL(LIB_PATH)
    vp, i32 = C.c_void_p, C.c_int
    lib.treekv_workspace_bytes.restype = C.c_size_t
    lib.treekv_workspace_bytes.argtypes = [i32] * 7
    lib.treekv_create.restype = i32
    lib.treekv_create.argtypes = [C.POINTER(vp), i32, i32, i32, i32, i32, i32, i32, vp, C.c_size_t, vp]
    lib.treekv_decode_step.restype = i32
    lib.treekv_decode_step.argtypes = [vp, vp, vp, vp, vp, C.POINTER(C.c_uint8), vp]
    lib.treekv_decode_step_host.restype = i32
    lib.treekv_decode_step_host.argtypes = [vp, vp, vp, vp, vp, C.POINTER(C.c_uint8), vp]
    lib.treekv_prefill_chunk.restype = i32
    lib.treekv_prefill_chunk.argtypes = [vp, vp, vp, vp, vp, C.POINTER(C.c_int32), i32, vp]
    lib.treekv_prefill_chunk_host.restype = i32
    lib.treekv_prefill_chunk_host.argtypes = [vp, vp, vp, vp, vp, C.POINTER(C.c_int32), i32, vp]
    lib.treekv_prefill_chunk_static_scratch.restype = i32
    lib.treekv_prefill_chunk_static_scratch.argtypes = [vp, vp, vp, vp, vp, C.POINTER(C.c_int32), i32, vp]
    lib.treekv_retained_positions.restype = i32
    lib.treekv_retained_positions.argtypes = [vp, vp, vp, vp]
    lib.treekv_scores.restype = i32
    lib.treekv_scores.argtypes = [vp, vp, vp]
    lib.treekv_get_stats.restype = i32
    lib.treekv_get_stats.argtypes = [vp, C.POINTER(TreeKVStats), vp]
    lib.treekv_tokens_seen.restype = C.c_int64
    lib.treekv_tokens_seen.argtypes = [vp, i32]
    lib.treekv_set_rule.restype = i32
    lib.treekv_set_rule.argtypes = [vp, i32]
    lib.treekv_set_option.restype = i32
    lib.treekv_set_option.argtypes = [vp, i32, i32]
    lib.treekv_reset.restype = i32
    lib.treekv_reset.argtypes = [vp, vp]
    lib.treekv_destroy.restype = None
    lib.treekv_destroy.argtypes = [vp]
    lib.treekv_status_string.restype = C.c_char_p
    lib.treekv_status_string.argtypes = [i32]
    lib.treekv_version.restype = C.c_char_p
    lib.treekv_version.argtypes = []
    lib.treekv_state_bytes.restype = C.c_size_t
    lib.treekv_state_bytes.argtypes = [vp]
    lib.treekv_export_state.restype = i32
    lib.treekv_export_state.argtypes = [vp, vp, C.POINTER(C.c_int64), vp]
    lib.treekv_import_state.restype = i32
    lib.treekv_import_state.argtypes = [vp, vp, C.POINTER(C.c_int64), vp]
    lib.treekv_prefill_oneshot.restype = i32
    lib.treekv_prefill_oneshot.argtypes = [vp, vp, vp, vp, vp, C.POINTER(C.c_int32), i32, i32, vp]
    lib.treekv_set_positions.restype = i32
    lib.treekv_set_positions.argtypes = [vp, vp, vp, i32]
    lib.treekv_set_protection.restype = i32
    lib.treekv_set_protection.argtypes = [vp, i32, i32]
    lib.treekv_selftest_wait_giveup.restype = i32
    lib.treekv_selftest_wait_giveup.argtypes = [vp, i32, vp]
    lib.treekv_norm_rope.restype = i32
    lib.treekv_norm_rope.argtypes = [vp, vp, C.c_int64, vp, vp, C.c_float, vp, vp, i32, vp, vp, vp, vp, i32, vp]
    lib.treekv_verify_tree.restype = i32
    lib.treekv_verify_tree.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i32, vp]
    lib.treekv_accept_path.restype = i32
    lib.treekv_accept_path.argtypes = [vp, vp, vp, vp, vp, i32, vp, i32, vp, vp]
    lib.treekv_fork_sequences.restype = i32
    lib.treekv_fork_sequences.argtypes = [vp, vp, vp]
    lib.treekv_selftest_fork_plan.restype = i32
    lib.treekv_selftest_fork_plan.argtypes = [C.POINTER(C.c_int32), i32, C.POINTER(C.c_int64), C.POINTER(C.c_int32)]
    lib.treekv_paged_attend.restype = i32
    lib.treekv_paged_attend.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, vp, i32, vp, i32, vp, vp, vp, i32, vp, C.c_size_t, vp]
    lib.treekv_paged_scratch_bytes.restype = C.c_size_t
    lib.treekv_paged_scratch_bytes.argtypes = [vp, i32]
    lib.treekv_paged_score.restype = i32
    lib.treekv_paged_score.argtypes = [vp, vp, vp, vp, i32, i32, vp, i32, vp, i32, vp, C.c_int64, i32, vp, i32, vp]
    lib.treekv_adopt_pages.restype = i32
    lib.treekv_adopt_pages.argtypes = [vp, vp, vp, i32, i32, vp, i32, vp, C.c_int64, vp, vp, vp]
    lib.treekv_pick_path.restype = i32
    lib.treekv_pick_path.argtypes = [vp, vp, i32, i32, vp, vp, vp, C.c_float, vp, vp, vp, vp, vp, vp, i32, vp]
    return lib


lib = _load()


def status_string(status: int) -> str:
    return lib.treekv_status_string(status).decode()


def _check(status, what):
    if status != TREEKV_OK:
        raise TreeKVError(status, what)


# ---- the C ABI, same names, raw pointers (ints) ---------------------------------------------------------
def treekv_workspace_bytes(budget, n_heads, n_kv_heads, head_dim, dtype, batch, max_chunk) -> int:
    return lib.treekv_workspace_bytes(budget, n_heads, n_kv_heads, head_dim, dtype, batch, max_chunk)


def treekv_create(budget, n_heads, n_kv_heads, head_dim, dtype, batch, max_chunk, dev_workspace, workspace_bytes, stream=0):
    h = C.c_void_p()
    st = lib.treekv_create(C.byref(h), budget, n_heads, n_kv_heads, head_dim, dtype, batch, max_chunk,
                           dev_workspace, workspace_bytes, stream)
    return st, h


def _u8(active):
    if active is None:
        return None
    arr = (C.c_uint8 * len(active))(*[1 if a else 0 for a in active])
    return arr


def _i32(lens):
    if lens is None:
        return None
    return (C.c_int32 * len(lens))(*[int(x) for x in lens])


def treekv_decode_step(ctx, q, k, v, out, active=None, stream=0) -> int:
    return lib.treekv_decode_step(ctx, q, k, v, out, _u8(active), stream)


def treekv_decode_step_host(ctx, q, k, v, out, active=None, stream=0) -> int:
    return lib.treekv_decode_step_host(ctx, q, k, v, out, _u8(active), stream)


def treekv_prefill_chunk(ctx, q, k, v, out, chunk_lens, chunk_stride, stream=0) -> int:
    return lib.treekv_prefill_chunk(ctx, q, k, v, out, _i32(chunk_lens), chunk_stride, stream)


def treekv_prefill_oneshot(ctx, q, k, v, out, lens, stride, block, stream=0) -> int:
    return lib.treekv_prefill_oneshot(ctx, q, k, v, out, _i32(lens), stride, block, stream)


def treekv_prefill_chunk_host(ctx, q, k, v, out, chunk_lens, chunk_stride, stream=0) -> int:
    return lib.treekv_prefill_chunk_host(ctx, q, k, v, out, _i32(chunk_lens), chunk_stride, stream)


def treekv_prefill_chunk_static_scratch(ctx, q, k, v, out, chunk_lens, chunk_stride, stream=0) -> int:
    """treekv_prefill_chunk with its scratch in the library's fixed 16 MiB device area: for callers that cannot
    allocate device memory where they run.  Calls sharing a GPU must not overlap."""
    return lib.treekv_prefill_chunk_static_scratch(ctx, q, k, v, out, _i32(chunk_lens), chunk_stride, stream)


def treekv_retained_positions(ctx, dev_pos, dev_count, stream=0) -> int:
    return lib.treekv_retained_positions(ctx, dev_pos, dev_count, stream)


def treekv_scores(ctx, dev_sbar, stream=0) -> int:
    return lib.treekv_scores(ctx, dev_sbar, stream)


def treekv_get_stats(ctx, stream=0):
    s = TreeKVStats()
    st = lib.treekv_get_stats(ctx, C.byref(s), stream)
    return st, s


def treekv_tokens_seen(ctx, b) -> int:
    return lib.treekv_tokens_seen(ctx, b)


def treekv_set_rule(ctx, rule) -> int:
    return lib.treekv_set_rule(ctx, rule)


def treekv_set_protection(ctx, n_sink, n_recent) -> int:
    return lib.treekv_set_protection(ctx, n_sink, n_recent)


def treekv_set_positions(ctx, dev_cos, dev_sin, slots) -> int:
    return lib.treekv_set_positions(ctx, dev_cos, dev_sin, slots)


def treekv_set_option(ctx, opt, value) -> int:
    return lib.treekv_set_option(ctx, opt, value)


def treekv_reset(ctx, stream=0) -> int:
    return lib.treekv_reset(ctx, stream)


def treekv_state_bytes(ctx) -> int:
    return lib.treekv_state_bytes(ctx)


def treekv_export_state(ctx, dev_image, batch, stream=0):
    seen = (C.c_int64 * batch)()
    st = lib.treekv_export_state(ctx, dev_image, seen, stream)
    return st, list(seen)


def treekv_import_state(ctx, dev_image, tokens_seen, stream=0) -> int:
    seen = (C.c_int64 * len(tokens_seen))(*[int(x) for x in tokens_seen])
    return lib.treekv_import_state(ctx, dev_image, seen, stream)


def treekv_norm_rope(ctx, qkv, row_stride, q_weight, k_weight, eps, cos, sin, slots, pos, q, k, v, tokens, stream=0) -> int:
    return lib.treekv_norm_rope(ctx, qkv, row_stride, q_weight, k_weight, eps, cos, sin, slots, pos, q, k, v, tokens, stream)


def treekv_verify_tree(ctx, q, k, v, mask, out, lse, lens, stride, stream=0) -> int:
    return lib.treekv_verify_tree(ctx, q, k, v, mask, out, lse, _i32(lens), stride, stream)


def treekv_accept_path(ctx, q, k, v, lse, stride, path, path_stride, lens, stream=0) -> int:
    return lib.treekv_accept_path(ctx, q, k, v, lse, stride, path, path_stride, _i32(lens), stream)


def treekv_fork_sequences(ctx, source, stream=0) -> int:
    return lib.treekv_fork_sequences(ctx, _i32(source), stream)


def treekv_paged_scratch_bytes(ctx, stride) -> int:
    return lib.treekv_paged_scratch_bytes(ctx, stride)


def treekv_paged_attend(ctx, q, k, v, k_pages, v_pages, n_pages, page_size, table, table_stride, past, max_past, out, lse, lens, stride,
                        scratch, scratch_bytes, stream=0) -> int:
    return lib.treekv_paged_attend(ctx, q, k, v, k_pages, v_pages, n_pages, page_size, table, table_stride, past, max_past, out, lse,
                                   _i32(lens), stride, scratch, scratch_bytes, stream)


def treekv_paged_score(ctx, q, lse, k_pages, n_pages, page_size, table, table_stride, past, max_past, scores, score_stride, add, lens,
                       stride, stream=0) -> int:
    return lib.treekv_paged_score(ctx, q, lse, k_pages, n_pages, page_size, table, table_stride, past, max_past, scores, score_stride, add,
                                  _i32(lens), stride, stream)


def treekv_adopt_pages(ctx, k_pages, v_pages, n_pages, page_size, table, table_stride, scores, score_stride, lens, first, stream=0) -> int:
    return lib.treekv_adopt_pages(ctx, k_pages, v_pages, n_pages, page_size, table, table_stride, scores, score_stride, _i32(lens),
                                  _i32(first), stream)


def treekv_pick_path(ctx, logits, logits_type, vocab, tokens, mask, draft, temperature, uniform, noise, path, count, next_, lens, stride,
                     stream=0) -> int:
    return lib.treekv_pick_path(ctx, logits, logits_type, vocab, tokens, mask, draft, temperature, uniform, noise, path, count, next_,
                                _i32(lens), stride, stream)


def treekv_selftest_fork_plan(source, seen):
    """The copy operations of treekv_fork_sequences as (component, source, destination, tokens seen) rows."""
    n = len(source)
    ops = (C.c_int32 * (4 * (n + n // 2 + 1)))()
    count = lib.treekv_selftest_fork_plan(_i32(source), n, (C.c_int64 * n)(*[int(x) for x in seen]), ops)
    return None if count < 0 else [tuple(ops[4 * o:4 * o + 4]) for o in range(count)]


def treekv_selftest_wait_giveup(ctx, attempts, stream=0) -> int:
    return lib.treekv_selftest_wait_giveup(ctx, attempts, stream)


def treekv_destroy(ctx) -> None:
    lib.treekv_destroy(ctx)


def treekv_version() -> str:
    return lib.treekv_version().decode()


# ---- convenience wrapper over torch tensors --------------------------------------------------------------
class TreeKV:
    """One attention layer's TreeKV cache on the current CUDA device.  torch supplies memory and streams only."""

    def __init__(self, budget, n_heads, n_kv_heads, head_dim, dtype="bf16", batch=1, max_chunk=0, device=None):
        import torch

        self.torch = torch
        if not torch.cuda.is_available():
            raise RuntimeError("TreeKV needs a CUDA device; there is no CPU fallback")
        self.device = torch.device(device if device is not None else "cuda:%d" % torch.cuda.current_device())
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        # handle of torch's current stream, without making a Stream object for every call where torch offers that
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
        self.budget, self.n_heads, self.n_kv_heads, self.head_dim = budget, n_heads, n_kv_heads, head_dim
        self.batch, self.max_chunk = batch, max_chunk
        self.dtype_code = TREEKV_F32 if dtype in ("f32", "fp32", torch.float32) else TREEKV_BF16
        self.tdtype = torch.float32 if self.dtype_code == TREEKV_F32 else torch.bfloat16
        nbytes = treekv_workspace_bytes(budget, n_heads, n_kv_heads, head_dim, self.dtype_code, batch, max_chunk)
        if nbytes == 0:
            raise TreeKVError(4, "treekv_workspace_bytes")
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        base = (self.workspace.data_ptr() + 255) // 256 * 256
        st, h = treekv_create(budget, n_heads, n_kv_heads, head_dim, self.dtype_code, batch, max_chunk, base, nbytes,
                              self._stream())
        _check(st, "treekv_create")
        self._h = h

    def _stream(self):
        return self._raw_stream(self.device.index)

    def close(self):
        h, self._h = getattr(self, "_h", None), None
        if h and lib is not None and getattr(lib, "treekv_destroy", None) is not None:   # (names vanish at interpreter exit)
            lib.treekv_destroy(h)

    def __del__(self):
        self.close()

    def _chk(self, t, shape):
        if not (t.is_cuda and t.is_contiguous() and t.dtype == self.tdtype and tuple(t.shape) == tuple(shape)):
            raise ValueError("expected contiguous %s CUDA tensor of shape %s, got %s %s" %
                             (self.tdtype, tuple(shape), t.dtype, tuple(t.shape)))

    def decode_step(self, q, k, v, out=None, active=None):
        B, Hq, Hkv, d = self.batch, self.n_heads, self.n_kv_heads, self.head_dim
        self._chk(q, (B, Hq, d)); self._chk(k, (B, Hkv, d)); self._chk(v, (B, Hkv, d))
        if out is None:
            out = self.torch.empty_like(q)
        self._chk(out, (B, Hq, d))
        _check(treekv_decode_step(self._h, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), active,
                                  self._stream()), "treekv_decode_step")
        return out

    def prefill_chunk(self, q, k, v, out=None, chunk_lens=None):
        B, Hq, Hkv, d = self.batch, self.n_heads, self.n_kv_heads, self.head_dim
        stride = q.shape[1]
        self._chk(q, (B, stride, Hq, d)); self._chk(k, (B, stride, Hkv, d)); self._chk(v, (B, stride, Hkv, d))
        if out is None:
            out = self.torch.empty_like(q)
        self._chk(out, (B, stride, Hq, d))
        _check(treekv_prefill_chunk(self._h, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), chunk_lens,
                                    stride, self._stream()), "treekv_prefill_chunk")
        return out

    def prefill_oneshot(self, q, k, v, block, out=None, lens=None):
        B, Hq, Hkv, d = self.batch, self.n_heads, self.n_kv_heads, self.head_dim
        stride = q.shape[1]
        self._chk(q, (B, stride, Hq, d)); self._chk(k, (B, stride, Hkv, d)); self._chk(v, (B, stride, Hkv, d))
        if out is None:
            out = self.torch.empty_like(q)
        self._chk(out, (B, stride, Hq, d))
        _check(treekv_prefill_oneshot(self._h, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lens, stride,
                                      block, self._stream()), "treekv_prefill_oneshot")
        return out

    def prefill_chunk_static_scratch(self, q, k, v, out=None, chunk_lens=None):
        """prefill_chunk through the entry point whose scratch is the library's fixed device area (no allocation)."""
        B, Hq, Hkv, d = self.batch, self.n_heads, self.n_kv_heads, self.head_dim
        stride = q.shape[1]
        self._chk(q, (B, stride, Hq, d)); self._chk(k, (B, stride, Hkv, d)); self._chk(v, (B, stride, Hkv, d))
        if out is None:
            out = self.torch.empty_like(q)
        self._chk(out, (B, stride, Hq, d))
        _check(treekv_prefill_chunk_static_scratch(self._h, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                                                   chunk_lens, stride, self._stream()),
               "treekv_prefill_chunk_static_scratch")
        return out

    def decode_step_host(self, q, k, v, out, active=None):
        """q,k,v,out: CPU tensors (pinned for asynchronous copies)."""
        _check(treekv_decode_step_host(self._h, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), active,
                                       self._stream()), "treekv_decode_step_host")
        return out

    def prefill_chunk_host(self, q, k, v, out, chunk_lens=None):
        _check(treekv_prefill_chunk_host(self._h, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), chunk_lens,
                                         q.shape[1], self._stream()), "treekv_prefill_chunk_host")
        return out

    # The calls of drafted decoding are short on the device: their checks are written for few interpreter steps, and tensors
    # made here are not looked at again.
    def _lens(self, lens, what):
        """Address of the numbers as int32 (and what keeps them), None where there are none."""
        if lens is None:
            return None, None
        if len(lens) != self.batch:
            raise ValueError("expected %d %s, got %d" % (self.batch, what, len(lens)))
        kept = _array("i", lens)
        return kept.buffer_info()[0], kept

    def _want(self, x, dtype, shape, what):
        if not (x.shape == shape and x.dtype is dtype and x.device == self.device and x.is_contiguous()):
            raise ValueError("expected %s as a contiguous %s tensor of shape %s on %s, got %s %s on %s" %
                             (what, dtype, shape, self.device, x.dtype, tuple(x.shape), x.device))
        return x.data_ptr()

    def norm_rope(self, qkv, q_weight=None, k_weight=None, cos=None, sin=None, positions=None, eps=1e-6, q=None, k=None, v=None):
        """(q, k, v) of the tokens of a packed projection [tokens, (n_heads + 2 n_kv_heads) * head_dim], whose rows may lie
        in wider ones: every q and k head normalised (where its weight [head_dim] is given) and rotated to the token's
        position (where tables [slots, head_dim/2] are given)."""
        t, want, dt = self.torch, self._want, self.tdtype
        Hq, Hkv, d = self.n_heads, self.n_kv_heads, self.head_dim
        row = (Hq + 2 * Hkv) * d
        steps = qkv.stride()
        if not (len(steps) == 2 and steps[1] == 1 and qkv.shape[1] == row and qkv.dtype is dt and qkv.device == self.device):
            raise ValueError("expected a %s tensor [tokens, %d] with adjacent columns on %s, got %s %s on %s" %
                             (dt, row, self.device, qkv.dtype, tuple(qkv.shape), qkv.device))
        n = qkv.shape[0]
        wq = None if q_weight is None else want(q_weight, dt, (d,), "q_weight")
        wk = None if k_weight is None else want(k_weight, dt, (d,), "k_weight")
        pc = ps = pp = None
        slots = 0
        if cos is not None or sin is not None:
            if cos is None or sin is None or positions is None:
                raise ValueError("a rotation takes cos, sin and positions")
            slots = cos.shape[0]
            pc, ps = want(cos, t.float32, (slots, d // 2), "cos"), want(sin, t.float32, (slots, d // 2), "sin")
        if positions is not None:
            pp = want(positions, t.int32, (n,), "positions")
        if q is None:
            q = qkv.new_empty(n, Hq, d)
            pq = q.data_ptr()
        else:
            pq = want(q, dt, (n, Hq, d), "q")
        if k is None:
            k = qkv.new_empty(n, Hkv, d)
            pk = k.data_ptr()
        else:
            pk = want(k, dt, (n, Hkv, d), "k")
        if v is None:
            v = qkv.new_empty(n, Hkv, d)
            pv = v.data_ptr()
        else:
            pv = want(v, dt, (n, Hkv, d), "v")
        # (torch reports any stride for the rows of a tensor of one row)
        st = lib.treekv_norm_rope(self._h, qkv.data_ptr(), steps[0] if n > 1 else row, wq, wk, eps, pc, ps, slots, pp, pq, pk, pv,
                                  n, self._stream())
        if st:
            _check(st, "treekv_norm_rope")
        return q, k, v

    def verify_tree(self, q, k, v, mask=None, lens=None, out=None, lse=None):
        """(out, lse) of drafted tokens [batch, stride, heads, head_dim] over the cache and the drafted tokens that each
        one's mask word (int64 [batch, stride], bit j = drafted token j) names; without masks a chain."""
        want, dt = self._want, self.tdtype
        B, Hq, Hkv, d = self.batch, self.n_heads, self.n_kv_heads, self.head_dim
        n = q.shape[1]
        pq, pk, pv = want(q, dt, (B, n, Hq, d), "q"), want(k, dt, (B, n, Hkv, d), "k"), want(v, dt, (B, n, Hkv, d), "v")
        pm = None if mask is None else want(mask, self.torch.int64, (B, n), "mask")
        if out is None:
            out = q.new_empty(B, n, Hq, d)
            po = out.data_ptr()
        else:
            po = want(out, dt, (B, n, Hq, d), "out")
        if lse is None:
            lse = q.new_empty(B, n, Hq, dtype=self.torch.float32)
            pl = lse.data_ptr()
        else:
            pl = want(lse, self.torch.float32, (B, n, Hq), "lse")
        pn, kept = self._lens(lens, "draft lengths")
        st = lib.treekv_verify_tree(self._h, pq, pk, pv, pm, po, pl, pn, n, self._stream())
        if st:
            _check(st, "treekv_verify_tree")
        return out, lse

    def accept_path(self, q, k, v, lse, path, lens=None):
        """The drafted tokens path[b, :lens[b]] (int32) of every sequence enter the cache; q, k, v, lse as in verify_tree."""
        want, dt = self._want, self.tdtype
        B, Hq, Hkv, d = self.batch, self.n_heads, self.n_kv_heads, self.head_dim
        n, m = q.shape[1], path.shape[1]
        pq, pk, pv = want(q, dt, (B, n, Hq, d), "q"), want(k, dt, (B, n, Hkv, d), "k"), want(v, dt, (B, n, Hkv, d), "v")
        pl, pp = want(lse, self.torch.float32, (B, n, Hq), "lse"), want(path, self.torch.int32, (B, m), "path")
        pn, kept = self._lens(lens, "accepted lengths")
        st = lib.treekv_accept_path(self._h, pq, pk, pv, pl, n, pp, m, pn, self._stream())
        if st:
            _check(st, "treekv_accept_path")

    def fork_sequences(self, source):
        """Sequence b becomes what sequence source[b] was (b: stays, -1: emptied), all at once."""
        p, kept = self._lens(source, "sources")
        st = lib.treekv_fork_sequences(self._h, p, self._stream())
        if st:
            _check(st, "treekv_fork_sequences")

    # Prompts in pages: pools [n_pages, n_kv_heads, page_size, head_dim], table [batch, pages of a sequence] int32, past [batch]
    # int32, all on the device.
    def _pages(self, k_pages, v_pages, table):
        """(k, v, number of pages, tokens of a page, table, entries of its rows) as the library takes them."""
        want = self._want
        n, page, width = k_pages.shape[0], k_pages.shape[2] if k_pages.dim() == 4 else 0, table.shape[1] if table.dim() == 2 else 0
        shape = (n, self.n_kv_heads, page, self.head_dim)
        return (want(k_pages, self.tdtype, shape, "k_pages"), None if v_pages is None else want(v_pages, self.tdtype, shape, "v_pages"), n, page,
                want(table, self.torch.int32, (self.batch, width), "table"), width)

    def paged_attend(self, q, k, v, k_pages, v_pages, table, past, lens=None, max_past=None, out=None, lse=None):
        """(out, lse) of a chunk of new tokens [batch, stride, heads, head_dim] over the pages, which it enters behind the
        past[b] tokens there are.  max_past: no past is larger (what the table holds otherwise; a closer bound gives a better
        launch)."""
        want, dt = self._want, self.tdtype
        B, Hq, Hkv, d = self.batch, self.n_heads, self.n_kv_heads, self.head_dim
        n = q.shape[1]
        pq, pk, pv = want(q, dt, (B, n, Hq, d), "q"), want(k, dt, (B, n, Hkv, d), "k"), want(v, dt, (B, n, Hkv, d), "v")
        kp, vp, pages, page, pt, width = self._pages(k_pages, v_pages, table)
        pp = want(past, self.torch.int32, (B,), "past")
        if out is None:
            out = q.new_empty(B, n, Hq, d)
            po = out.data_ptr()
        else:
            po = want(out, dt, (B, n, Hq, d), "out")
        if lse is None:
            lse = q.new_empty(B, n, Hq, dtype=self.torch.float32)
            pl = lse.data_ptr()
        else:
            pl = want(lse, self.torch.float32, (B, n, Hq), "lse")
        pn, kept = self._lens(lens, "chunk lengths")
        nbytes = lib.treekv_paged_scratch_bytes(self._h, n)
        scratch = q.new_empty(nbytes, dtype=self.torch.uint8)   # (torch keeps it for this stream's later work)
        st = lib.treekv_paged_attend(self._h, pq, pk, pv, kp, vp, pages, page, pt, width, pp, width * page if max_past is None else max_past,
                                     po, pl, pn, n, scratch.data_ptr(), nbytes, self._stream())
        if st:
            _check(st, "treekv_paged_attend")
        return out, lse

    def paged_score(self, q, lse, k_pages, table, past, scores, lens=None, max_past=None, add=False):
        """scores [batch, n_kv_heads, tokens] float32: written, or with add=True increased by, what the rows q gave to every token
        of their sequence; past[b] is the position of the first of them, and past[b] + lens[b] at most `tokens`.  max_past: no past
        is larger (what the scores hold otherwise)."""
        want, t = self._want, self.torch
        B, Hq = self.batch, self.n_heads
        n = q.shape[1]
        pq, pl = want(q, self.tdtype, (B, n, Hq, self.head_dim), "q"), want(lse, t.float32, (B, n, Hq), "lse")
        kp, _, pages, page, pt, width = self._pages(k_pages, None, table)
        pp = want(past, t.int32, (B,), "past")
        steps = scores.shape[-1]
        ps = want(scores, t.float32, (B, self.n_kv_heads, steps), "scores")
        pn, kept = self._lens(lens, "chunk lengths")
        if max_past is None:
            max_past = max(0, min(width * page, steps - (n if lens is None else min((x for x in lens if x), default=0))))
        st = lib.treekv_paged_score(self._h, pq, pl, kp, pages, page, pt, width, pp, max_past, ps, steps, 1 if add else 0, pn, n, self._stream())
        if st:
            _check(st, "treekv_paged_score")
        return scores

    def adopt_pages(self, k_pages, v_pages, table, scores, lens, first=None):
        """The lens[b] first tokens of the pages become what sequence b has seen; beyond the budget the heaviest stay.  first[b]: the
        first token whose row is in the scores."""
        kp, vp, pages, page, pt, width = self._pages(k_pages, v_pages, table)
        steps = scores.shape[-1]
        ps = self._want(scores, self.torch.float32, (self.batch, self.n_kv_heads, steps), "scores")
        pn, kept = self._lens(lens, "prompt lengths")
        if pn is None:
            raise ValueError("adopt_pages takes the prompts' lengths")
        pf, kept2 = self._lens(first, "first counted tokens")
        st = lib.treekv_adopt_pages(self._h, kp, vp, pages, page, pt, width, ps, steps, pn, pf, self._stream())
        if st:
            _check(st, "treekv_adopt_pages")

    def pick_path(self, logits, tokens, uniform=None, noise=None, mask=None, lens=None, draft=None, temperature=1.0):
        """(path [batch, stride], count [batch], next token [batch]), int32, of drafted trees whose node 0 is given: logits [batch,
        stride, vocab] (float32 or bfloat16), tokens int32 [batch, stride], uniform float32 [batch, stride], noise float32 [batch,
        vocab] (exponential), draft float32 [batch, stride, vocab] (what each node's children were drawn from)."""
        t, want = self.torch, self._want
        B, n, V = self.batch, tokens.shape[1], logits.shape[-1]
        if logits.dtype not in (t.float32, t.bfloat16):
            raise ValueError("expected float32 or bfloat16 logits, got %s" % logits.dtype)
        pl, pt = want(logits, logits.dtype, (B, n, V), "logits"), want(tokens, t.int32, (B, n), "tokens")
        pu = None if uniform is None else want(uniform, t.float32, (B, n), "uniform")
        pe = None if noise is None else want(noise, t.float32, (B, V), "noise")
        pm = None if mask is None else want(mask, t.int64, (B, n), "mask")
        pd = None if draft is None else want(draft, t.float32, (B, n, V), "draft")
        path, count, after = tokens.new_empty(B, n), tokens.new_empty(B), tokens.new_empty(B)
        pn, kept = self._lens(lens, "draft lengths")
        st = lib.treekv_pick_path(self._h, pl, TREEKV_F32 if logits.dtype is t.float32 else TREEKV_BF16, V, pt, pm, pd, temperature, pu, pe,
                                  path.data_ptr(), count.data_ptr(), after.data_ptr(), pn, n, self._stream())
        if st:
            _check(st, "treekv_pick_path")
        return path, count, after

    def retained_positions(self):
        t = self.torch
        pos = t.empty((self.batch, self.n_kv_heads, self.budget), dtype=t.int32, device=self.device)
        cnt = t.empty((self.batch, self.n_kv_heads), dtype=t.int32, device=self.device)
        _check(treekv_retained_positions(self._h, pos.data_ptr(), cnt.data_ptr(), self._stream()),
               "treekv_retained_positions")
        return pos, cnt

    def scores(self):
        t = self.torch
        sb = t.empty((self.batch, self.n_kv_heads, self.budget), dtype=t.float32, device=self.device)
        _check(treekv_scores(self._h, sb.data_ptr(), self._stream()), "treekv_scores")
        return sb

    def stats(self, check=True):
        """Counters as a dict.  With check=False what the device recorded - a give-up (TREEKV_ERR_TIMEOUT), an index out of
        range (TREEKV_ERR_INVALID_ARG) - is reported through 'device_error' and 'status' instead of raising; a call that could
        not read it raises all the same."""
        st, s = treekv_get_stats(self._h, self._stream())
        if check or not s.device_error:
            _check(st, "treekv_get_stats")
        return {"status": st, "evictions": s.evictions, "near_ties": s.near_ties, "kernel_launches": s.kernel_launches,
                "device_error": s.device_error, "last_cuda_error": s.last_cuda_error}

    def tokens_seen(self, b=0):
        return treekv_tokens_seen(self._h, b)

    def set_rule(self, rule):
        _check(treekv_set_rule(self._h, rule), "treekv_set_rule")

    def set_protection(self, n_sink, n_recent):
        _check(treekv_set_protection(self._h, n_sink, n_recent), "treekv_set_protection")

    def set_positions(self, cos, sin):
        """cos, sin: float32 CUDA tensors [slots, head_dim/2] (kept alive by this object), or None, None."""
        if cos is None:
            _check(treekv_set_positions(self._h, None, None, 0), "treekv_set_positions")
            self._rope = None
            return
        t = self.torch
        if not (cos.is_cuda and cos.is_contiguous() and cos.dtype == t.float32 and sin.shape == cos.shape and sin.is_cuda
                and sin.is_contiguous() and sin.dtype == t.float32 and cos.shape[1] == self.head_dim // 2):
            raise ValueError("expected two contiguous float32 CUDA tensors of shape [slots, head_dim/2]")
        _check(treekv_set_positions(self._h, cos.data_ptr(), sin.data_ptr(), cos.shape[0]), "treekv_set_positions")
        self._rope = (cos, sin)

    def set_option(self, opt, value):
        _check(treekv_set_option(self._h, opt, value), "treekv_set_option")

    def reset(self):
        _check(treekv_reset(self._h, self._stream()), "treekv_reset")

    def export_state(self):
        """(image, tokens_seen): a uint8 CUDA tensor holding the state image and the per-sequence token counts."""
        n = treekv_state_bytes(self._h)
        image = self.torch.empty(n + 256, dtype=self.torch.uint8, device=self.device)
        off = (-image.data_ptr()) % 256
        image = image[off:off + n]
        st, seen = treekv_export_state(self._h, image.data_ptr(), self.batch, self._stream())
        _check(st, "treekv_export_state")
        return image, seen

    def import_state(self, image, tokens_seen):
        if not (image.is_cuda and image.dtype == self.torch.uint8 and image.numel() >= treekv_state_bytes(self._h)
                and image.data_ptr() % 16 == 0):
            raise ValueError("expected a uint8 CUDA tensor of at least treekv_state_bytes, 16-byte aligned")
        _check(treekv_import_state(self._h, image.data_ptr(), tokens_seen, self._stream()), "treekv_import_state")
