"""ctypes binding of ``libchess.so``: argument marshalling only.

Every method of :class:`Chess` maps one-to-one onto the C entry point of the same name in
``include/chess.h``; tensors are passed as raw device pointers and the launch goes onto torch's
current HIP stream.  There is no fallback: if the library has not been built, loading fails."""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import torch

PLAN_BUDGET, PLAN_RATIO, PLAN_FLAT = 0, 1, 2
PROBE_QUERY, PROBE_ANCHOR = 0, 1
CUT_COUNT, CUT_THRESHOLD = 0, 1
SUMMARY_F32, SUMMARY_BF16 = 0, 1

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libchess.so")
_lib = None

EXPORTS = ["chess_create", "chess_destroy", "chess_summary_bytes", "chess_summary_layout", "chess_workspace_bytes", "chess_workspace_init",
           "chess_summarize", "chess_summarize_tail", "chess_summarize_recent", "chess_append_kv", "chess_select", "chess_anchor", "chess_select_shared", "chess_entropy", "chess_trigger_update", "chess_monitor_step", "chess_extend_window", "chess_reuse_step", "chess_sparse_decode", "chess_sparse_decode_static", "chess_dense_decode", "chess_decode_step",
           "chess_write_rows", "chess_release_pages", "chess_map_tokens", "chess_quant_store", "chess_quant_store_bounded", "chess_quant_summarize",
           "chess_quant_sparse_decode", "chess_quant_dense_decode",
           "chess_rotate", "chess_rotate_store", "chess_attend_scratch_bytes", "chess_dense_attend", "chess_sparse_attend", "chess_verify",
           "chess_trim_pages",
           "chess_debug_force_splits", "chess_debug_force_cluster", "chess_debug_force_schedule", "chess_debug_force_general_cut", "chess_debug_set_poll_limit", "chess_workspace_error", "chess_strerror", "chess_version"]


class ChessError(RuntimeError):
    pass


class _CConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("n_q_heads", "n_kv_heads", "head_dim", "page_size", "pages_per_chunk", "chunks_per_grid",
                 "max_batch", "max_pages_per_seq", "max_selected_pages")] + [("sm_scale", ctypes.c_float),
                                                                              ("summary_dtype", ctypes.c_int32),
                                                                              ("shared_device", ctypes.c_int32)]


class _CPlan(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("plan", "sink_pages", "window_pages", "budget_pages", "budget_bp", "over_chunk", "over_grid",
                 "rho_g_bp", "rho_c_bp", "rho_p_bp", "probe", "cut_rule")] + [("budget_per_seq", ctypes.c_void_p)]


class _CRotary(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("inv_freq", "q_norm", "k_norm")] + [
        (n, ctypes.c_int32) for n in ("rotary_dim", "interleaved", "norm_per_head", "n_axes")] + [
        ("axis", ctypes.c_uint8 * 64), ("eps", ctypes.c_float), ("scale", ctypes.c_float)]


class _CScores(ctypes.Structure):
    _fields_ = [("cap", ctypes.c_float), ("window", ctypes.c_int32)] + [(n, ctypes.c_void_p) for n in ("slopes", "prefix_lens", "first_keys")]


@dataclass(frozen=True)
class Config:
    n_q_heads: int
    n_kv_heads: int
    page_size: int
    max_batch: int
    max_pages_per_seq: int
    max_selected_pages: int
    pages_per_chunk: int = 8
    chunks_per_grid: int = 8
    head_dim: int = 128
    sm_scale: float = 0.0
    summary_dtype: int = SUMMARY_F32
    shared_device: bool = False


@dataclass(frozen=True)
class SelectPlan:
    plan: int = PLAN_BUDGET
    sink_pages: int = 1
    window_pages: int = 4
    budget_pages: int = 0
    budget_bp: int = 100
    over_chunk: int = 10
    over_grid: int = 5
    rho_g_bp: int = 10000
    rho_c_bp: int = 10000
    rho_p_bp: int = 10000
    probe: int = PROBE_QUERY
    cut_rule: int = CUT_COUNT
    budget_per_seq: object = None      # device int32 tensor [batch] or None (the caller keeps it alive)

    def _c(self) -> _CPlan:
        per = None if self.budget_per_seq is None else ctypes.c_void_p(self.budget_per_seq.data_ptr())
        return _CPlan(self.plan, self.sink_pages, self.window_pages, self.budget_pages, self.budget_bp,
                      self.over_chunk, self.over_grid, self.rho_g_bp, self.rho_c_bp, self.rho_p_bp, self.probe,
                      self.cut_rule, per)


def _plain(t, name, dtype):
    """A contiguous tensor of the type, or None: (elements, device index) of it."""
    if t is None:
        return 0, None
    if t.dtype is not dtype or not t.is_contiguous():
        raise ChessError(f"{name}: a contiguous {dtype} tensor is wanted, got {t.dtype} {tuple(t.shape)} of strides {t.stride()}")
    return t.numel(), t.get_device()


class Rotary:
    """How queries and keys are normed and turned (``chess_rotary``); holds its tensors.

    inv_freq: device fp32 [rotary_dim / 2]; axis: for each pair the row of ``positions`` that turns it (None: row 0); q_norm, k_norm: device fp32
    [128], or [heads, 128] both, or None; interleaved: pairs are neighbours."""

    def __init__(self, inv_freq, axis=None, interleaved: bool = False, q_norm=None, k_norm=None, eps: float = 1e-6, scale: float = 1.0):
        pairs, dev = _plain(inv_freq, "inv_freq", torch.float32)
        axis = [0] * pairs if axis is None else [int(i) for i in axis]
        if len(axis) != pairs or pairs > 64 or min(axis, default=0) < 0 or max(axis, default=0) > 3:
            raise ChessError(f"axis: one of 0 to 3 for each of at most 64 pairs is wanted, got {axis} for {pairs}")
        if q_norm is not None and k_norm is not None and q_norm.dim() != k_norm.dim():
            raise ChessError(f"q_norm, k_norm: weights a head, or for all heads, in both, got {tuple(q_norm.shape)} and {tuple(k_norm.shape)}")
        if scale == 0:
            raise ChessError("scale: not 0")
        self.inv_freq, self.q_norm, self.k_norm, self.device = inv_freq, q_norm, k_norm, dev
        self.n_axes = max(axis, default=0) + 1
        per_head = any(t is not None and t.dim() == 2 for t in (q_norm, k_norm))
        self.weights = []                  # (heads that each kind's weights are for, or None: for any)
        for t, name in ((q_norm, "q_norm"), (k_norm, "k_norm")):
            n, at = _plain(t, name, torch.float32)
            if t is not None and (at != dev or (t.shape[-1] if t.dim() else 0) != 128 or t.dim() > 2):
                raise ChessError(f"{name}: [128] or [heads, 128] on the device of inv_freq is wanted, got {tuple(t.shape)} on {t.device}")
            self.weights.append(n // 128 if t is not None and per_head else None)
        self._c = _CRotary(inv_freq.data_ptr(), _ptr(q_norm), _ptr(k_norm), 2 * pairs, int(bool(interleaved)), int(per_head), self.n_axes,
                           (ctypes.c_uint8 * 64)(*axis), eps, scale)
        self._ref = ctypes.byref(self._c)


class Scores:
    """What a query sees and how a score is formed (``chess_scores``); holds its tensors.

    slopes: device fp32 [n_q_heads]; prefix_lens: device int32 [batch]; first_keys: device int32 [rows]; each or None."""

    def __init__(self, cap: float = 0.0, slopes=None, window: int = 0, prefix_lens=None, first_keys=None):
        self.slopes, self.prefix_lens, self.first_keys = slopes, prefix_lens, first_keys
        self.has = [(*_plain(t, name, dtype), name) for t, name, dtype in
                    ((slopes, "slopes", torch.float32), (prefix_lens, "prefix_lens", torch.int32), (first_keys, "first_keys", torch.int32))]
        self.any = any(dev is not None for _, dev, _ in self.has)
        self._c = _CScores(cap, window, _ptr(slopes), _ptr(prefix_lens), _ptr(first_keys))
        self._ref = ctypes.byref(self._c)

    def _need(self, *numels, dev):
        for (n, at, name), numel in zip(self.has, numels):
            if at is not None and (at != dev or n < numel):
                raise ChessError(f"{name}: at least {numel} elements on the context's device are wanted, got {n} on device {at}")


def library_path() -> str:
    return _LIB_PATH


def load_library() -> ctypes.CDLL:
    """Load the built library; raises if it is missing (build it with ``__graft_entry__.build()``)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ChessError(f"{_LIB_PATH} is not built; run `python -c 'import __graft_entry__ as g; g.build()'`")
        lib = ctypes.CDLL(_LIB_PATH)
        vp, i32p = ctypes.c_void_p, ctypes.c_void_p
        lib.chess_create.argtypes = [ctypes.POINTER(_CConfig), ctypes.POINTER(vp)]
        lib.chess_destroy.argtypes = [vp]
        lib.chess_destroy.restype = None
        lib.chess_summary_bytes.argtypes = [vp, ctypes.POINTER(ctypes.c_size_t)]
        lib.chess_summary_layout.argtypes = [vp] + [ctypes.POINTER(ctypes.c_size_t)] * 3
        lib.chess_workspace_bytes.argtypes = [vp, ctypes.POINTER(ctypes.c_size_t)]
        lib.chess_summarize.argtypes = [vp, vp, i32p, i32p, ctypes.c_int32, i32p, vp, vp]
        lib.chess_summarize_tail.argtypes = [vp, vp, i32p, i32p, ctypes.c_int32, vp, vp]
        lib.chess_summarize_recent.argtypes = [vp, vp, i32p, i32p, ctypes.c_int32, ctypes.c_int32, vp, vp]
        lib.chess_workspace_init.argtypes = [vp, vp, vp]
        lib.chess_select.argtypes = [vp, vp, vp, i32p, ctypes.c_int32, ctypes.POINTER(_CPlan), i32p, i32p, vp, vp]
        lib.chess_entropy.argtypes = [vp, vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int64, vp, vp, vp]
        lib.chess_monitor_step.argtypes = [vp, vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int64, ctypes.c_int32, ctypes.c_double,
                                           ctypes.c_double, vp, vp, i32p, i32p, vp, vp, vp]
        lib.chess_trigger_update.argtypes = [vp, vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_double, ctypes.c_double, vp, i32p, i32p, vp, vp]
        lib.chess_reuse_step.argtypes = [vp, vp, vp, vp, vp, vp, i32p, i32p, i32p, i32p, ctypes.c_int32, vp, vp, vp]
        lib.chess_extend_window.argtypes = [vp, i32p, ctypes.c_int32, i32p, i32p, vp]
        lib.chess_append_kv.argtypes = [vp, vp, vp, vp, vp, i32p, i32p, ctypes.c_int32, i32p, i32p, vp]
        lib.chess_anchor.argtypes = [vp, ctypes.POINTER(vp), ctypes.c_int32, i32p, ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(vp), vp]
        lib.chess_select_shared.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.c_int32, i32p, ctypes.c_int32,
                                            ctypes.POINTER(_CPlan), i32p, i32p, vp, vp]
        lib.chess_sparse_decode.argtypes = [vp, vp, vp, vp, i32p, i32p, i32p, i32p, ctypes.c_int32, vp, vp, vp]
        lib.chess_sparse_decode_static.argtypes = [vp, vp, vp, vp, i32p, i32p, i32p, i32p, ctypes.c_int32, vp, vp]
        lib.chess_dense_decode.argtypes = [vp, vp, vp, vp, i32p, i32p, ctypes.c_int32, vp, vp, vp]
        lib.chess_decode_step.argtypes = [vp, vp, vp, vp, i32p, i32p, vp, ctypes.c_int32, ctypes.c_int32, vp, i32p, i32p, vp, vp, vp]
        lib.chess_write_rows.argtypes = [vp, ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)]
        lib.chess_release_pages.argtypes = [vp, i32p, i32p, ctypes.c_int32, i32p, i32p, ctypes.c_int32, i32p, i32p, i32p, vp, vp]
        lib.chess_map_tokens.argtypes = [vp, i32p, i32p, ctypes.c_int32, ctypes.c_int32] + [vp] * 11
        lib.chess_quant_store.argtypes = [vp, vp, ctypes.c_int64, vp, ctypes.c_int64, i32p, i32p, ctypes.c_int32, vp, vp, vp, vp]
        lib.chess_quant_store_bounded.argtypes = [vp, vp, ctypes.c_int64, vp, ctypes.c_int64, ctypes.c_int32, i32p, i32p, ctypes.c_int32, vp, vp, vp,
                                                  ctypes.c_int32, vp]
        lib.chess_quant_summarize.argtypes = [vp, vp, vp, i32p, i32p, ctypes.c_int32, i32p, ctypes.c_int32, vp, vp]
        lib.chess_quant_sparse_decode.argtypes = [vp, vp, vp, vp, vp, i32p, i32p, i32p, i32p, ctypes.c_int32, vp, vp, vp]
        lib.chess_quant_dense_decode.argtypes = [vp, vp, vp, vp, vp, i32p, i32p, ctypes.c_int32, vp, vp, vp]
        i32, i64 = ctypes.c_int32, ctypes.c_int64
        lib.chess_rotate.argtypes = [vp, vp, vp, i64, vp, i64, i32p, i32, i32p, vp, vp, vp]
        lib.chess_rotate_store.argtypes = [vp, vp, vp, i64, vp, i64, vp, i64, i32p, i32, i32p, i32p, i32, vp, vp, vp, i32, vp]
        lib.chess_attend_scratch_bytes.argtypes = [vp, i32, i32, i32, ctypes.POINTER(ctypes.c_size_t)]
        lib.chess_dense_attend.argtypes = [vp, vp, vp, i32, i32p, i32, vp, vp, i32p, i32p, i32, vp, vp, vp, ctypes.c_size_t, vp]
        lib.chess_sparse_attend.argtypes = [vp, vp, vp, i32, i32p, i32, vp, vp, i32p, i32p, i32p, i32p, i32, vp, vp, vp, ctypes.c_size_t, vp]
        lib.chess_verify.argtypes = [vp, vp, i64, vp, i64, i64, i32, i32p, i32, i32p, vp, i32, i32p, i32, i32p, i32p, i32p, vp, vp]
        lib.chess_trim_pages.argtypes = [vp, i32p, i32p, i32, i32p, i32p, i32, i32p, i32p, vp, vp]
        lib.chess_debug_force_splits.argtypes = [vp, ctypes.c_int32, ctypes.c_int32]
        lib.chess_debug_force_cluster.argtypes = [vp, ctypes.c_int32]
        lib.chess_debug_force_general_cut.argtypes = [vp, ctypes.c_int32]
        lib.chess_debug_force_schedule.argtypes = [vp, ctypes.c_int32]
        lib.chess_debug_set_poll_limit.argtypes = [vp, ctypes.c_int32]
        lib.chess_workspace_error.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_int32), vp]
        lib.chess_strerror.argtypes = [ctypes.c_int]
        lib.chess_strerror.restype = ctypes.c_char_p
        lib.chess_version.restype = ctypes.c_int
        _lib = lib
    return _lib


# Plain integers: the entry points' argtypes make the pointers of them.  A launch made from Python costs the host
# more than the smaller kernels run for; without an object per pointer and one for the stream, 34 calls of 4
# sequences at 24-32K (32 layers, model-wide scope) take 288 -> 205 us of host time.
def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream():
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


_BYTES = (torch.uint8, torch.float8_e4m3fn)
_INT, _LONG, _FLOAT, _BF16, _BYTE = (torch.int32,), (torch.int64,), (torch.float32,), (torch.bfloat16,), (torch.uint8,)


def _need(t, name, dtypes, numel, dev):
    """A contiguous tensor on device `dev`, the context's, of one of the types, with that many elements at least.  (The library sees a pointer
    only.  About 0.3 us a tensor: what these calls cost the host matters as much as what the smaller kernels take.)"""
    if t.dtype not in dtypes or t.numel() < numel or not t.is_contiguous() or t.get_device() != dev:
        raise ChessError(f"{name}: a contiguous {' or '.join(str(d) for d in dtypes)} tensor of at least {numel} elements on the context's device is wanted, "
                         f"got {t.dtype} {tuple(t.shape)} of strides {t.stride()} on {t.device}")


class Chess:
    """One configured instance of the library (one layer's shapes).  Methods launch asynchronously on the
    current torch stream and return nothing; outputs are the tensors passed in."""

    device = None     # index of the device the context was created on

    def __init__(self, cfg: Config):
        self.lib = load_library()
        self.cfg = cfg
        c = _CConfig(cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, cfg.page_size, cfg.pages_per_chunk,
                     cfg.chunks_per_grid, cfg.max_batch, cfg.max_pages_per_seq, cfg.max_selected_pages, cfg.sm_scale,
                     cfg.summary_dtype, int(bool(cfg.shared_device)))
        h = ctypes.c_void_p()
        self._check(self.lib.chess_create(ctypes.byref(c), ctypes.byref(h)))
        self._h = h
        self.device = torch.cuda.current_device()
        n = ctypes.c_size_t()
        self._check(self.lib.chess_summary_bytes(h, ctypes.byref(n)))
        self.summary_bytes = n.value
        self._check(self.lib.chess_workspace_bytes(h, ctypes.byref(n)))
        self.workspace_bytes = n.value
        a, b, c3 = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
        self._check(self.lib.chess_summary_layout(h, ctypes.byref(a), ctypes.byref(b), ctypes.byref(c3)))
        self.summary_offsets = (a.value, b.value, c3.value)

    def close(self):
        if getattr(self, "_h", None):
            self.lib.chess_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc: int):
        if rc != 0:
            raise ChessError(f"libchess error {rc}: {self.lib.chess_strerror(rc).decode()}")

    # ---- buffers the caller owns (torch is only the allocator here)
    def new_summaries(self, device="cuda") -> torch.Tensor:
        return torch.zeros(self.summary_bytes, dtype=torch.uint8, device=device)

    def new_workspace(self, device="cuda") -> torch.Tensor:
        ws = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=device)
        self._check(self.lib.chess_workspace_init(self._h, _ptr(ws), _stream()))
        return ws

    def summary_views(self, summaries: torch.Tensor):
        """(pages, chunks, grids) views [max_batch, H_kv, units, d] of a summaries buffer, fp32 or bf16 by the
        configuration's summary_dtype."""
        c = self.cfg
        mc = -(-c.max_pages_per_seq // c.pages_per_chunk)
        mg = -(-mc // c.chunks_per_grid)
        dt, size = (torch.bfloat16, 2) if c.summary_dtype == SUMMARY_BF16 else (torch.float32, 4)
        out = []
        for off, units in zip(self.summary_offsets, (c.max_pages_per_seq, mc, mg)):
            n = c.max_batch * c.n_kv_heads * units * c.head_dim
            out.append(summaries[off:off + size * n].view(dt).view(c.max_batch, c.n_kv_heads, units, c.head_dim))
        return tuple(out)

    # ---- the C entry points
    def summarize(self, k_pool, block_table, seq_lens, summaries, from_page=None):
        self._check(self.lib.chess_summarize(self._h, _ptr(k_pool), _ptr(block_table), _ptr(seq_lens),
                                             seq_lens.shape[0], _ptr(from_page), _ptr(summaries), _stream()))

    def summarize_tail(self, k_pool, block_table, seq_lens, summaries):
        self._check(self.lib.chess_summarize_tail(self._h, _ptr(k_pool), _ptr(block_table), _ptr(seq_lens),
                                                  seq_lens.shape[0], _ptr(summaries), _stream()))

    def summarize_recent(self, k_pool, block_table, seq_lens, recent_pages: int, summaries):
        self._check(self.lib.chess_summarize_recent(self._h, _ptr(k_pool), _ptr(block_table), _ptr(seq_lens),
                                                    seq_lens.shape[0], recent_pages, _ptr(summaries), _stream()))

    def select(self, q, summaries, seq_lens, plan: SelectPlan, page_ids, n_selected, workspace):
        p = plan._c()
        self._check(self.lib.chess_select(self._h, _ptr(q), _ptr(summaries), _ptr(seq_lens), seq_lens.shape[0],
                                          ctypes.byref(p), _ptr(page_ids), _ptr(n_selected), _ptr(workspace), _stream()))

    def entropy(self, logits, entropy, workspace, vocab=None):
        self._check(self.lib.chess_entropy(self._h, _ptr(logits), logits.shape[0], logits.shape[1] if vocab is None else vocab,
                                           logits.stride(0), _ptr(entropy), _ptr(workspace), _stream()))

    def monitor_step(self, logits, page_steps: int, tau_entropy: float, tau_variance: float, entropy, history, count, fire,
                     workspace, stats=None, vocab=None):
        self._check(self.lib.chess_monitor_step(self._h, _ptr(logits), logits.shape[0],
                                                logits.shape[1] if vocab is None else vocab, logits.stride(0), page_steps,
                                                tau_entropy, tau_variance, _ptr(entropy), _ptr(history), _ptr(count),
                                                _ptr(fire), _ptr(stats), _ptr(workspace), _stream()))

    def trigger_update(self, entropy, page_steps: int, tau_entropy: float, tau_variance: float, history, count, fire,
                       stats=None):
        self._check(self.lib.chess_trigger_update(self._h, _ptr(entropy), entropy.shape[0], page_steps, tau_entropy,
                                                  tau_variance, _ptr(history), _ptr(count), _ptr(fire), _ptr(stats), _stream()))

    def reuse_step(self, q, k_new, v_new, k_pool, v_pool, block_table, seq_lens, page_ids, n_selected, out, workspace):
        self._check(self.lib.chess_reuse_step(self._h, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_pool), _ptr(v_pool),
                                              _ptr(block_table), _ptr(seq_lens), _ptr(page_ids), _ptr(n_selected),
                                              seq_lens.shape[0], _ptr(out), _ptr(workspace), _stream()))

    def extend_window(self, seq_lens, page_ids, n_selected):
        self._check(self.lib.chess_extend_window(self._h, _ptr(seq_lens), seq_lens.shape[0], _ptr(page_ids), _ptr(n_selected),
                                                 _stream()))

    def append_kv(self, k_new, v_new, k_pool, v_pool, block_table, seq_lens, page_ids=None, n_selected=None):
        self._check(self.lib.chess_append_kv(self._h, _ptr(k_new), _ptr(v_new), _ptr(k_pool), _ptr(v_pool), _ptr(block_table),
                                             _ptr(seq_lens), seq_lens.shape[0], _ptr(page_ids), _ptr(n_selected), _stream()))

    def anchor(self, summaries, seq_lens, window_pages: int, anchors):
        """summaries / anchors: one device tensor each, or sequences of per-layer tensors (one launch)."""
        if isinstance(summaries, torch.Tensor):
            summaries, anchors = [summaries], [anchors]
        n = len(summaries)
        assert len(anchors) == n
        st = (ctypes.c_void_p * n)(*[t.data_ptr() for t in summaries])
        at = (ctypes.c_void_p * n)(*[t.data_ptr() for t in anchors])
        self._check(self.lib.chess_anchor(self._h, st, n, _ptr(seq_lens), seq_lens.shape[0], window_pages, at, _stream()))

    def select_shared(self, probes, summaries, seq_lens, plan: SelectPlan, page_ids, n_selected, workspace):
        """probes / summaries: sequences of per-layer device tensors."""
        n = len(probes)
        assert len(summaries) == n
        pt = (ctypes.c_void_p * n)(*[t.data_ptr() for t in probes])
        st = (ctypes.c_void_p * n)(*[t.data_ptr() for t in summaries])
        p = plan._c()
        self._check(self.lib.chess_select_shared(self._h, pt, st, n, _ptr(seq_lens), seq_lens.shape[0], ctypes.byref(p),
                                                 _ptr(page_ids), _ptr(n_selected), _ptr(workspace), _stream()))

    def sparse_decode(self, q, k_pool, v_pool, block_table, seq_lens, page_ids, n_selected, out, workspace):
        self._check(self.lib.chess_sparse_decode(self._h, _ptr(q), _ptr(k_pool), _ptr(v_pool), _ptr(block_table),
                                                 _ptr(seq_lens), _ptr(page_ids), _ptr(n_selected), seq_lens.shape[0],
                                                 _ptr(out), _ptr(workspace), _stream()))

    def sparse_decode_static(self, q, k_pool, v_pool, block_table, seq_lens, page_ids, n_selected, out):
        self._check(self.lib.chess_sparse_decode_static(self._h, _ptr(q), _ptr(k_pool), _ptr(v_pool), _ptr(block_table),
                                                        _ptr(seq_lens), _ptr(page_ids), _ptr(n_selected), seq_lens.shape[0],
                                                        _ptr(out), _stream()))

    def dense_decode(self, q, k_pool, v_pool, block_table, seq_lens, out, workspace):
        self._check(self.lib.chess_dense_decode(self._h, _ptr(q), _ptr(k_pool), _ptr(v_pool), _ptr(block_table),
                                                _ptr(seq_lens), seq_lens.shape[0], _ptr(out), _ptr(workspace), _stream()))

    def decode_step(self, q, k_pool, v_pool, block_table, seq_lens, summaries, plan: SelectPlan, page_ids, n_selected,
                    out, workspace, refresh_tail: bool = False):
        p = plan._c()
        self._check(self.lib.chess_decode_step(self._h, _ptr(q), _ptr(k_pool), _ptr(v_pool), _ptr(block_table),
                                               _ptr(seq_lens), _ptr(summaries), int(bool(refresh_tail)),
                                               seq_lens.shape[0], ctypes.byref(p),
                                               _ptr(page_ids), _ptr(n_selected), _ptr(out), _ptr(workspace), _stream()))

    # ---- pages handed out on the device
    def write_rows(self, max_tokens: int, batch: int) -> int:
        """Entries `writes` must have room for."""
        n = ctypes.c_size_t()
        self._check(self.lib.chess_write_rows(self._h, max_tokens, batch, ctypes.byref(n)))
        return n.value

    def release_pages(self, seq_lens, done, block_table, free_pages, n_free, lens_after, n_left, workspace):
        batch, dev = seq_lens.numel(), self.device
        _need(seq_lens, "seq_lens", _INT, batch, dev)
        _need(done, "done", _INT, batch, dev)
        _need(block_table, "block_table", _INT, batch * self.cfg.max_pages_per_seq, dev)
        _need(free_pages, "free_pages", _INT, 1, dev)
        _need(n_free, "n_free", _INT, 1, dev)
        _need(lens_after, "lens_after", _INT, batch, dev)
        _need(n_left, "n_left", _INT, 1, dev)
        _need(workspace, "workspace", _BYTE, self.workspace_bytes, dev)
        self._check(self.lib.chess_release_pages(self._h, seq_lens.data_ptr(), done.data_ptr(), batch, block_table.data_ptr(), free_pages.data_ptr(),
                                                 free_pages.numel(), n_free.data_ptr(), lens_after.data_ptr(), n_left.data_ptr(),
                                                 workspace.data_ptr(), torch._C._cuda_getCurrentRawStream(dev)))

    def map_tokens(self, seq_lens, new_lens, block_table, free_pages, n_free, lens_after, n_left, token_start, slots, writes, counts, workspace,
                   max_tokens=None):
        """max_tokens: by default what `slots` has room for; slots may be None if it is given."""
        if max_tokens is None:
            if slots is None:
                raise ChessError("map_tokens: slots or max_tokens is wanted")
            max_tokens = slots.numel()
        batch, dev = seq_lens.numel(), self.device
        _need(seq_lens, "seq_lens", _INT, batch, dev)
        _need(new_lens, "new_lens", _INT, batch, dev)
        _need(block_table, "block_table", _INT, batch * self.cfg.max_pages_per_seq, dev)
        _need(free_pages, "free_pages", _INT, 1, dev)
        _need(n_free, "n_free", _INT, 1, dev)
        _need(lens_after, "lens_after", _INT, batch, dev)
        _need(n_left, "n_left", _INT, 1, dev)
        _need(workspace, "workspace", _BYTE, self.workspace_bytes, dev)
        _need(token_start, "token_start", _INT, batch + 1, dev)
        if slots is not None:
            _need(slots, "slots", _LONG, max_tokens, dev)
        _need(writes, "writes", _INT, 4 * min(max_tokens, max_tokens // self.cfg.page_size + 2 * batch), dev)
        _need(counts, "counts", _INT, 4, dev)
        self._check(self.lib.chess_map_tokens(self._h, seq_lens.data_ptr(), new_lens.data_ptr(), batch, max_tokens, block_table.data_ptr(),
                                              free_pages.data_ptr(), n_free.data_ptr(), lens_after.data_ptr(), n_left.data_ptr(),
                                              token_start.data_ptr(), _ptr(slots), writes.data_ptr(), counts.data_ptr(), workspace.data_ptr(),
                                              torch._C._cuda_getCurrentRawStream(dev)))

    # ---- the cache in 8 bits: pools uint8 or float8_e4m3fn, scales fp32 [physical page, H_kv, 2]
    def _need_pool(self, pool, scales, name, dev):
        block = self.cfg.page_size * self.cfg.head_dim
        _need(pool, name, _BYTES, block, dev)
        if pool.numel() * 2 != scales.numel() * block:
            raise ChessError(f"{name}: {pool.numel()} bytes and {scales.numel()} scales are not of the same pages")

    def quant_store(self, k_new, v_new, writes, counts, k_pool, v_pool, scales):
        """k_new / v_new: bf16 [tokens, H_kv, 128], the rows of a token contiguous (slices of a wider projection will do); no tokens, nothing
        stored.  An entry that names a token or a page beyond these tensors stores nothing."""
        cfg, dev = self.cfg, self.device
        n, H, d = k_new.size(0), cfg.n_kv_heads, cfg.head_dim
        for t, name in ((k_new, "k_new"), (v_new, "v_new")):
            if (t.dtype is not torch.bfloat16 or t.dim() != 3 or t.size(0) != n or t.size(1) != H or t.size(2) != d or t.stride(2) != 1 or
                    (t.stride(1) != d and H > 1) or t.get_device() != dev):
                raise ChessError(f"{name}: a bf16 tensor [{n}, {H}, {d}] on the context's device with contiguous token rows is wanted, "
                                 f"got {t.dtype} {tuple(t.shape)} of strides {t.stride()} on {t.device}")
        _need(writes, "writes", _INT, 4, dev)
        _need(counts, "counts", _INT, 4, dev)
        _need(scales, "scales", _FLOAT, 2 * H, dev)
        self._need_pool(k_pool, scales, "k_pool", dev)
        self._need_pool(v_pool, scales, "v_pool", dev)
        if n == 0:
            return
        # (one token's stride leads nowhere and may be any number: of [H, 1, 128] transposed it is 128)
        k_stride, v_stride = (k_new.stride(0), v_new.stride(0)) if n > 1 else (H * d, H * d)
        self._check(self.lib.chess_quant_store_bounded(self._h, k_new.data_ptr(), k_stride, v_new.data_ptr(), v_stride, n,
                                                       writes.data_ptr(), counts.data_ptr(), writes.numel() // 4, k_pool.data_ptr(), v_pool.data_ptr(),
                                                       scales.data_ptr(), scales.numel() // (2 * H), torch._C._cuda_getCurrentRawStream(dev)))

    def quant_summarize(self, k_pool, scales, block_table, seq_lens, summaries, from_page=None, recent_pages: int = 0):
        batch, dev = seq_lens.numel(), self.device
        _need(scales, "scales", _FLOAT, 2 * self.cfg.n_kv_heads, dev)
        self._need_pool(k_pool, scales, "k_pool", dev)
        _need(block_table, "block_table", _INT, batch * self.cfg.max_pages_per_seq, dev)
        _need(seq_lens, "seq_lens", _INT, batch, dev)
        if from_page is not None:
            _need(from_page, "from_page", _INT, batch, dev)
        _need(summaries, "summaries", _BYTE, self.summary_bytes, dev)
        self._check(self.lib.chess_quant_summarize(self._h, k_pool.data_ptr(), scales.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(), batch,
                                                   _ptr(from_page), recent_pages, summaries.data_ptr(), torch._C._cuda_getCurrentRawStream(dev)))

    def _need_attention(self, q, k_pool, v_pool, scales, block_table, seq_lens, out, workspace, batch, dev):
        c = self.cfg
        values = batch * c.n_q_heads * c.head_dim
        _need(q, "q", _BF16, values, dev)
        _need(scales, "scales", _FLOAT, 2 * c.n_kv_heads, dev)
        self._need_pool(k_pool, scales, "k_pool", dev)
        self._need_pool(v_pool, scales, "v_pool", dev)
        _need(block_table, "block_table", _INT, batch * c.max_pages_per_seq, dev)
        _need(seq_lens, "seq_lens", _INT, batch, dev)
        _need(out, "out", _FLOAT, values, dev)
        _need(workspace, "workspace", _BYTE, self.workspace_bytes, dev)

    def quant_sparse_decode(self, q, k_pool, v_pool, scales, block_table, seq_lens, page_ids, n_selected, out, workspace):
        batch, dev = seq_lens.numel(), self.device
        self._need_attention(q, k_pool, v_pool, scales, block_table, seq_lens, out, workspace, batch, dev)
        _need(page_ids, "page_ids", _INT, batch * self.cfg.n_kv_heads * self.cfg.max_selected_pages, dev)
        _need(n_selected, "n_selected", _INT, batch * self.cfg.n_kv_heads, dev)
        self._check(self.lib.chess_quant_sparse_decode(self._h, q.data_ptr(), k_pool.data_ptr(), v_pool.data_ptr(), scales.data_ptr(),
                                                       block_table.data_ptr(), seq_lens.data_ptr(), page_ids.data_ptr(), n_selected.data_ptr(),
                                                       batch, out.data_ptr(), workspace.data_ptr(), torch._C._cuda_getCurrentRawStream(dev)))

    def quant_dense_decode(self, q, k_pool, v_pool, scales, block_table, seq_lens, out, workspace):
        batch, dev = seq_lens.numel(), self.device
        self._need_attention(q, k_pool, v_pool, scales, block_table, seq_lens, out, workspace, batch, dev)
        self._check(self.lib.chess_quant_dense_decode(self._h, q.data_ptr(), k_pool.data_ptr(), v_pool.data_ptr(), scales.data_ptr(),
                                                      block_table.data_ptr(), seq_lens.data_ptr(), batch, out.data_ptr(), workspace.data_ptr(),
                                                      torch._C._cuda_getCurrentRawStream(dev)))

    # ---- several tokens of a sequence in a step
    def _need_rows(self, t, name, heads, n, dev):
        """bf16 [n, heads, 128] whose token rows are contiguous; the stride from one to the next."""
        stride = t.stride()
        if t.dtype is not torch.bfloat16 or t.shape != (n, heads, 128) or stride[2] != 1 or (stride[1] != 128 and heads > 1) or t.get_device() != dev:
            raise ChessError(f"{name}: a bf16 tensor [{n}, {heads}, 128] on the context's device with contiguous token rows is wanted, "
                             f"got {t.dtype} {tuple(t.shape)} of strides {stride} on {t.device}")
        return stride[0] if n > 1 else heads * 128    # (one token's stride leads nowhere)

    def _need_rotary(self, rotary, positions, n, dev):
        c = self.cfg
        if rotary.device != dev or rotary.weights[0] not in (None, c.n_q_heads) or rotary.weights[1] not in (None, c.n_kv_heads):
            raise ChessError(f"rotary: of the context's device ({dev}) and, with weights a head, {c.n_q_heads} and {c.n_kv_heads} heads is wanted, "
                             f"got device {rotary.device}, heads {rotary.weights}")
        _need(positions, "positions", _INT, rotary.n_axes * n, dev)
        # (one axis in any shape of as many; [rows, axes] would be read as [axes, rows])
        if positions.numel() != rotary.n_axes * n or rotary.n_axes > 1 and positions.dim() > 1 and positions.shape[-1] != n:
            raise ChessError(f"positions: [{rotary.n_axes}, {n}] is wanted, got {tuple(positions.shape)}")

    def rotate(self, rotary: Rotary, q, k, positions, q_out=None, k_out=None, counts=None):
        """q: bf16 [rows, n_q_heads, 128] or None, k: bf16 [rows, H_kv, 128] or None (slices of a wider projection will do); positions: int32
        [axes, rows] (or [rows] for one axis); no rows, nothing done."""
        c, dev = self.cfg, self.device
        if q is None and k is None:
            raise ChessError("rotate: q or k is wanted")
        n = (k if q is None else q).size(0)
        q_stride = k_stride = 0
        if q is not None:
            q_stride = self._need_rows(q, "q", c.n_q_heads, n, dev)
            _need(q_out, "q_out", _BF16, n * c.n_q_heads * c.head_dim, dev)
        if k is not None:
            k_stride = self._need_rows(k, "k", c.n_kv_heads, n, dev)
            _need(k_out, "k_out", _BF16, n * c.n_kv_heads * c.head_dim, dev)
        self._need_rotary(rotary, positions, n, dev)
        if counts is not None:
            _need(counts, "counts", _INT, 1, dev)
        if n == 0:
            return
        self._check(self.lib.chess_rotate(self._h, rotary._ref, _ptr(q), q_stride, _ptr(k), k_stride, positions.data_ptr(), n, _ptr(counts),
                                          None if q is None else q_out.data_ptr(), None if k is None else k_out.data_ptr(),
                                          torch._C._cuda_getCurrentRawStream(dev)))

    def rotate_store(self, rotary: Rotary, q, k_new, v_new, positions, writes, counts, q_out, k_pool, v_pool):
        """q: bf16 [rows, n_q_heads, 128] or None (with q_out), k_new / v_new: bf16 [rows, H_kv, 128] (slices of a wider projection will do); no
        rows, nothing stored.  An entry that names a row or a page beyond these tensors does nothing."""
        c, dev = self.cfg, self.device
        n, H, d, B = k_new.size(0), c.n_kv_heads, c.head_dim, c.page_size
        k_stride, v_stride, q_stride = self._need_rows(k_new, "k_new", H, n, dev), self._need_rows(v_new, "v_new", H, n, dev), 0
        if q is not None:
            q_stride = self._need_rows(q, "q", c.n_q_heads, n, dev)
            _need(q_out, "q_out", _BF16, n * c.n_q_heads * d, dev)
        self._need_rotary(rotary, positions, n, dev)
        _need(writes, "writes", _INT, 4, dev)
        _need(counts, "counts", _INT, 2, dev)
        _need(k_pool, "k_pool", _BF16, H * B * d, dev)
        _need(v_pool, "v_pool", _BF16, H * B * d, dev)
        if k_pool.numel() != v_pool.numel():
            raise ChessError(f"k_pool, v_pool: {k_pool.numel()} and {v_pool.numel()} values are not of the same pages")
        if n == 0:
            return
        self._check(self.lib.chess_rotate_store(self._h, rotary._ref, _ptr(q), q_stride, k_new.data_ptr(), k_stride, v_new.data_ptr(), v_stride,
                                                positions.data_ptr(), n, writes.data_ptr(), counts.data_ptr(), writes.numel() // 4,
                                                None if q is None else q_out.data_ptr(), k_pool.data_ptr(), v_pool.data_ptr(),
                                                k_pool.numel() // (H * B * d), torch._C._cuda_getCurrentRawStream(dev)))

    def attend_scratch_bytes(self, n_rows: int, max_new: int, batch: int) -> int:
        n = ctypes.c_size_t()
        self._check(self.lib.chess_attend_scratch_bytes(self._h, n_rows, max_new, batch, ctypes.byref(n)))
        return n.value

    def new_attend_scratch(self, n_rows: int, max_new: int, batch: int, device="cuda") -> torch.Tensor:
        return torch.empty(self.attend_scratch_bytes(n_rows, max_new, batch), dtype=torch.uint8, device=device)

    def _need_attend(self, q, token_start, k_pool, v_pool, block_table, seq_lens, out, workspace, scratch, scores, batch, dev):
        c = self.cfg
        shape = q.shape
        if len(shape) != 3 or shape[1] != c.n_q_heads or shape[2] != c.head_dim:
            raise ChessError(f"q: [rows, {c.n_q_heads}, {c.head_dim}] is wanted, got {tuple(shape)}")
        n = shape[0]
        values = n * c.n_q_heads * c.head_dim
        _need(q, "q", _BF16, values, dev)
        _need(out, "out", _BF16, values, dev)
        _need(token_start, "token_start", _INT, batch + 1, dev)
        page = c.n_kv_heads * c.page_size * c.head_dim
        _need(k_pool, "k_pool", _BF16, page, dev)
        _need(v_pool, "v_pool", _BF16, page, dev)
        _need(block_table, "block_table", _INT, batch * c.max_pages_per_seq, dev)
        _need(seq_lens, "seq_lens", _INT, batch, dev)
        _need(workspace, "workspace", _BYTE, self.workspace_bytes, dev)
        _need(scratch, "scratch", _BYTE, 1, dev)
        if scores is not None and scores.any:
            scores._need(c.n_q_heads, batch, n, dev=dev)
        return n

    def dense_attend(self, q, token_start, max_new: int, k_pool, v_pool, block_table, seq_lens, out, workspace, scratch, scores: Scores = None):
        """q, out: bf16 [rows, n_q_heads, 128]; scratch: of new_attend_scratch for as many rows, new tokens of a sequence and sequences; no rows, nothing done."""
        batch, dev = seq_lens.numel(), self.device
        n = self._need_attend(q, token_start, k_pool, v_pool, block_table, seq_lens, out, workspace, scratch, scores, batch, dev)
        if n == 0:
            return
        self._check(self.lib.chess_dense_attend(self._h, None if scores is None else scores._ref, q.data_ptr(), n, token_start.data_ptr(), min(max_new, n),
                                                k_pool.data_ptr(), v_pool.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(), batch,
                                                out.data_ptr(), workspace.data_ptr(), scratch.data_ptr(), scratch.numel(),
                                                torch._C._cuda_getCurrentRawStream(dev)))

    def sparse_attend(self, q, token_start, max_new: int, k_pool, v_pool, block_table, seq_lens, page_ids, n_selected, out, workspace, scratch,
                      scores: Scores = None):
        batch, dev = seq_lens.numel(), self.device
        n = self._need_attend(q, token_start, k_pool, v_pool, block_table, seq_lens, out, workspace, scratch, scores, batch, dev)
        _need(page_ids, "page_ids", _INT, batch * self.cfg.n_kv_heads * self.cfg.max_selected_pages, dev)
        _need(n_selected, "n_selected", _INT, batch * self.cfg.n_kv_heads, dev)
        if n == 0:
            return
        self._check(self.lib.chess_sparse_attend(self._h, None if scores is None else scores._ref, q.data_ptr(), n, token_start.data_ptr(), min(max_new, n),
                                                 k_pool.data_ptr(), v_pool.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(),
                                                 page_ids.data_ptr(), n_selected.data_ptr(), batch, out.data_ptr(), workspace.data_ptr(),
                                                 scratch.data_ptr(), scratch.numel(), torch._C._cuda_getCurrentRawStream(dev)))

    def verify(self, target, draft, tokens, token_start, uniforms, seq_lens, n_accepted, out_tokens, lens_after, workspace):
        """target: fp32 [rows, vocab]; draft: fp32 [batch, at least max_drafts, vocab] or None (words of a row next to one another in both; rows may be
        slices of wider ones); tokens: int32 [rows]; uniforms: fp32 [batch, max_drafts + 1]."""
        batch, dev = seq_lens.numel(), self.device
        if uniforms.dim() != 2 or uniforms.size(0) != batch or uniforms.size(1) < 1:
            raise ChessError(f"uniforms: [{batch}, max_drafts + 1] is wanted, got {tuple(uniforms.shape)}")
        shape, stride = target.shape, target.stride()
        if len(shape) != 2 or target.dtype is not torch.float32 or stride[1] != 1 and shape[1] > 1 or target.get_device() != dev or shape[0] < 1 or shape[1] < 1:
            raise ChessError(f"target: an fp32 tensor [rows, vocab] with contiguous rows on the context's device is wanted, got {target.dtype} "
                             f"{tuple(shape)} of strides {stride} on {target.device}")
        n, vocab = shape
        target_stride = stride[0] if n > 1 else vocab
        most = uniforms.size(1) - 1
        draft_seq = draft_row = 0
        if draft is not None:
            shape, stride = draft.shape, draft.stride()
            if (len(shape) != 3 or draft.dtype is not torch.float32 or shape[0] != batch or shape[1] < most or shape[2] != vocab or
                    stride[2] != 1 and vocab > 1 or draft.get_device() != dev):
                raise ChessError(f"draft: an fp32 tensor [{batch}, {most}, {vocab}] with contiguous rows on the context's device is wanted, got {draft.dtype} "
                                 f"{tuple(shape)} of strides {stride} on {draft.device}")
            draft_seq, draft_row = stride[0] if batch > 1 else vocab, stride[1] if shape[1] > 1 else vocab
        _need(tokens, "tokens", _INT, n, dev)
        _need(token_start, "token_start", _INT, batch + 1, dev)
        _need(uniforms, "uniforms", _FLOAT, batch * (most + 1), dev)
        _need(seq_lens, "seq_lens", _INT, batch, dev)
        _need(n_accepted, "n_accepted", _INT, batch, dev)
        _need(out_tokens, "out_tokens", _INT, batch * (most + 1), dev)
        _need(lens_after, "lens_after", _INT, batch, dev)
        _need(workspace, "workspace", _BYTE, self.workspace_bytes, dev)
        self._check(self.lib.chess_verify(self._h, target.data_ptr(), target_stride, _ptr(draft), draft_seq, draft_row, vocab,
                                          tokens.data_ptr(), n, token_start.data_ptr(), uniforms.data_ptr(), most, seq_lens.data_ptr(), batch,
                                          n_accepted.data_ptr(), out_tokens.data_ptr(), lens_after.data_ptr(), workspace.data_ptr(),
                                          torch._C._cuda_getCurrentRawStream(dev)))

    def trim_pages(self, seq_lens, keep_lens, block_table, free_pages, n_free, n_left, workspace):
        batch, dev = seq_lens.numel(), self.device
        _need(seq_lens, "seq_lens", _INT, batch, dev)
        _need(keep_lens, "keep_lens", _INT, batch, dev)
        _need(block_table, "block_table", _INT, batch * self.cfg.max_pages_per_seq, dev)
        _need(free_pages, "free_pages", _INT, 1, dev)
        _need(n_free, "n_free", _INT, 1, dev)
        _need(n_left, "n_left", _INT, 1, dev)
        _need(workspace, "workspace", _BYTE, self.workspace_bytes, dev)
        self._check(self.lib.chess_trim_pages(self._h, seq_lens.data_ptr(), keep_lens.data_ptr(), batch, block_table.data_ptr(), free_pages.data_ptr(),
                                              free_pages.numel(), n_free.data_ptr(), n_left.data_ptr(), workspace.data_ptr(),
                                              torch._C._cuda_getCurrentRawStream(dev)))

    def workspace_error(self, workspace) -> int:
        flag = ctypes.c_int32()
        self._check(self.lib.chess_workspace_error(self._h, _ptr(workspace), ctypes.byref(flag), _stream()))
        return flag.value

    def debug_force_cluster(self, cluster: int):
        self._check(self.lib.chess_debug_force_cluster(self._h, cluster))

    def debug_force_schedule(self, schedule: int):
        """0 = automatic, 1 = lazy, 2 = merged, 3 = eager."""
        self._check(self.lib.chess_debug_force_schedule(self._h, schedule))

    def debug_force_general_cut(self, on: bool):
        self._check(self.lib.chess_debug_force_general_cut(self._h, int(bool(on))))

    def debug_set_poll_limit(self, polls: int):
        self._check(self.lib.chess_debug_set_poll_limit(self._h, polls))

    def debug_force_splits(self, n_splits: int, waves: int = 4):
        self._check(self.lib.chess_debug_force_splits(self._h, n_splits, waves))
