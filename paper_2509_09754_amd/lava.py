"""ctypes binding over liblava.so: the same entry points as include/lava.h, taking torch tensors.

Argument marshalling only — every step of the path runs in the HIP kernels.  PyTorch supplies
device memory and the current stream.  If the library has not been built the import fails
loudly; there is no fallback implementation.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# LAVA_LIBRARY names another build of the same library (the host-sanitizer build of build.py --sanitize);
# it is read by this binding only, never by the library itself
LIB_PATH = os.environ.get("LAVA_LIBRARY") or os.path.join(_HERE, "liblava.so")

LAVA_OK, LAVA_ERR_INVALID_ARG, LAVA_ERR_SHAPE, LAVA_ERR_BUDGET, LAVA_ERR_WORKSPACE, LAVA_ERR_HIP = range(6)
LAVA_F32, LAVA_BF16 = 0, 1
LAVA_SCORE_LAVA, LAVA_SCORE_ATTENTION, LAVA_SCORE_TOKEN_NORM = 0, 1, 2

EXPORTS = [
    "lava_status_string", "lava_set_tuning", "lava_get_tuning", "lava_window_scores_workspace_bytes", "lava_window_scores",
    "lava_window_scores_primed", "lava_select_topk_primed", "lava_window_scores_planned",
    "lava_layer_budgets", "lava_select_workspace_bytes", "lava_select_topk", "lava_select_status",
    "lava_select_topk_static",
    "lava_select_batch_workspace_bytes", "lava_select_topk_batch", "lava_select_batch_status",
    "lava_compact_kv", "lava_compact_packed", "lava_compact_batch",
    "lava_cascade_workspace_bytes", "lava_cascade_step",
    "lava_decode_workspace_bytes", "lava_decode_attention",
    "lava_page_tables_workspace_bytes", "lava_page_tables", "lava_compact_paged", "lava_rotary_turns", "lava_rotary",
    "lava_rotary_append", "lava_paged_decode_workspace_bytes", "lava_paged_decode",
    "lava_beam_step_workspace_bytes", "lava_beam_step", "lava_page_fork_workspace_bytes", "lava_page_fork", "lava_page_compact",
    "lava_shared_decode_workspace_bytes", "lava_shared_decode",
    "lava_prof_kernel_count", "lava_prof_kernel_name", "lava_prof_enable", "lava_prof_reset",
    "lava_prof_read", "lava_probe_stream",
]


class LayerDesc(ctypes.Structure):
    """Mirror of lava_layer_desc."""
    _fields_ = [
        ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
        ("window", ctypes.c_int32), ("pool_kernel", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("softmax_scale", ctypes.c_float), ("score_kind", ctypes.c_int32),
    ]

    @classmethod
    def make(cls, n_q_heads, n_kv_heads, head_dim, window, dtype, pool_kernel=7, softmax_scale=0.0,
             score_kind=LAVA_SCORE_LAVA):
        code = {"f32": LAVA_F32, "bf16": LAVA_BF16, LAVA_F32: LAVA_F32, LAVA_BF16: LAVA_BF16}[dtype]
        return cls(n_q_heads, n_kv_heads, head_dim, window, pool_kernel, code, softmax_scale, score_kind)

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.dtype == LAVA_BF16 else torch.float32


class Tuning(ctypes.Structure):
    """Mirror of lava_tuning (zero = the library's own choice)."""
    _fields_ = [
        ("sweep_shape", ctypes.c_int32), ("sweep_workgroups", ctypes.c_int32), ("sweep_schedule", ctypes.c_int32),
        ("decode_rows_per_unit", ctypes.c_int32), ("barrier_spin_limit", ctypes.c_int32),
        ("sweep_orphan_units", ctypes.c_int32), ("reserved", ctypes.c_int32 * 2),
    ]


class BudgetPlan(ctypes.Structure):
    """Mirror of lava_budget_plan (device pointers; see make_budget_plan)."""
    _fields_ = [("n_layers", ctypes.c_int32), ("layer", ctypes.c_int32), ("e", ctypes.c_void_p),
                ("total", ctypes.c_void_p), ("lo", ctypes.c_void_p), ("hi", ctypes.c_void_p),
                ("budgets", ctypes.c_void_p)]


LAVA_PLAN_MAX_LAYERS = 128
SWEEP_SHAPES = {"auto": 0, "wide": 1, "narrow": 2}
SWEEP_SCHEDULES = {"auto": 0, "separate": 1, "persistent": 2, "prepass": 3}


class LavaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2509_09754_amd.build` "
            "(there is no CPU fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    dp = ctypes.POINTER(LayerDesc)
    lib.lava_status_string.restype = ctypes.c_char_p
    lib.lava_status_string.argtypes = [i32]
    lib.lava_set_tuning.restype = i32
    lib.lava_set_tuning.argtypes = [ctypes.POINTER(Tuning)]
    lib.lava_get_tuning.restype = i32
    lib.lava_get_tuning.argtypes = [ctypes.POINTER(Tuning)]
    lib.lava_window_scores_workspace_bytes.restype = sz
    lib.lava_window_scores_workspace_bytes.argtypes = [dp, i32, i64]
    lib.lava_window_scores.restype = i32
    lib.lava_window_scores.argtypes = [dp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.lava_window_scores_primed.restype = i32
    lib.lava_window_scores_primed.argtypes = [dp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp, sz, vp]
    lib.lava_window_scores_planned.restype = i32
    lib.lava_window_scores_planned.argtypes = [dp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp, sz, vp, vp]
    lib.lava_select_topk_primed.restype = i32
    lib.lava_select_topk_primed.argtypes = [i32, vp, i64, i64, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.lava_layer_budgets.restype = i32
    lib.lava_layer_budgets.argtypes = [i32, i32, vp, vp, vp, vp, vp, i32, vp]
    lib.lava_select_workspace_bytes.restype = sz
    lib.lava_select_workspace_bytes.argtypes = [i64]
    lib.lava_select_topk.restype = i32
    lib.lava_select_topk.argtypes = [i32, vp, vp, i64, i64, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.lava_select_topk_static.restype = i32
    lib.lava_select_topk_static.argtypes = [i32, vp, vp, i64, i64, vp, vp, vp, vp, vp, vp]
    lib.lava_select_status.restype = i32
    lib.lava_select_status.argtypes = [vp, i64, vp]
    lib.lava_compact_kv.restype = i32
    lib.lava_compact_kv.argtypes = [dp, i64, vp, vp, vp, vp, i64, vp, vp, vp]
    lib.lava_compact_packed.restype = i32
    lib.lava_compact_packed.argtypes = [dp, vp, i64, vp, vp, vp, vp, vp, i64, vp, vp, vp, vp]
    lib.lava_cascade_workspace_bytes.restype = sz
    lib.lava_cascade_workspace_bytes.argtypes = [dp, i64, i32, i64]
    lib.lava_select_batch_workspace_bytes.restype = sz
    lib.lava_select_batch_workspace_bytes.argtypes = [i32, i64]
    lib.lava_select_topk_batch.restype = i32
    lib.lava_select_topk_batch.argtypes = [i32, i32, vp, i64, vp, sz, vp]
    lib.lava_select_batch_status.restype = i32
    lib.lava_select_batch_status.argtypes = [vp, i32, i64, vp]
    lib.lava_compact_batch.restype = i32
    lib.lava_compact_batch.argtypes = [dp, i32, vp, vp]
    lib.lava_cascade_step.restype = i32
    lib.lava_cascade_step.argtypes = [dp, i32, i64, vp, vp, vp, vp, i64, vp, vp, vp, sz, vp]
    lib.lava_decode_workspace_bytes.restype = sz
    lib.lava_decode_workspace_bytes.argtypes = [dp, i32, i64, i64]
    lib.lava_decode_attention.restype = i32
    lib.lava_decode_attention.argtypes = [dp, i32, vp, vp, vp, vp, vp, i64, vp, vp, i64, i64, vp, vp, vp, sz, vp]
    lib.lava_page_tables_workspace_bytes.restype = sz
    lib.lava_page_tables_workspace_bytes.argtypes = [i32, i32]
    lib.lava_page_tables.restype = i32
    lib.lava_page_tables.argtypes = [vp, i32, i32, vp, vp, vp, vp, i64, vp, vp, vp, sz, vp]
    lib.lava_compact_paged.restype = i32
    lib.lava_compact_paged.argtypes = [dp, i32, vp, vp, vp]
    lib.lava_rotary_turns.restype = i32
    lib.lava_rotary_turns.argtypes = [vp, vp]
    lib.lava_rotary.restype = i32
    lib.lava_rotary.argtypes = [vp, vp, i32, i32, i64, i32, vp, vp, i64, i64, vp, i64, i64, i32, vp]
    lib.lava_rotary_append.restype = i32
    lib.lava_rotary_append.argtypes = [dp, vp, vp, i64, vp, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp]
    lib.lava_paged_decode_workspace_bytes.restype = sz
    lib.lava_paged_decode_workspace_bytes.argtypes = [dp]
    lib.lava_paged_decode.restype = i32
    lib.lava_paged_decode.argtypes = [dp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.lava_beam_step_workspace_bytes.restype = sz
    lib.lava_beam_step_workspace_bytes.argtypes = [i32, i32, i64, i32]
    lib.lava_beam_step.restype = i32
    lib.lava_beam_step.argtypes = [i32, i32, i32, i64, vp, i64, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, i32, vp, sz, vp]
    lib.lava_page_fork_workspace_bytes.restype = sz
    lib.lava_page_fork_workspace_bytes.argtypes = [i32, i32, i32, i64]
    lib.lava_page_fork.restype = i32
    lib.lava_page_fork.argtypes = [dp, vp, i32, vp, vp, vp, vp, vp, sz, vp]
    lib.lava_page_compact.restype = i32
    lib.lava_page_compact.argtypes = [dp, vp, i32, vp, vp, vp, i64, vp, vp, vp, vp, sz, vp]
    lib.lava_shared_decode_workspace_bytes.restype = sz
    lib.lava_shared_decode_workspace_bytes.argtypes = [dp, i32, i32]
    lib.lava_shared_decode.restype = i32
    lib.lava_shared_decode.argtypes = [dp, i32, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.lava_prof_kernel_count.restype = i32
    lib.lava_prof_kernel_name.restype = ctypes.c_char_p
    lib.lava_prof_kernel_name.argtypes = [i32]
    lib.lava_prof_enable.restype = i32
    lib.lava_prof_enable.argtypes = [i32]
    lib.lava_prof_reset.restype = i32
    lib.lava_prof_read.restype = i32
    lib.lava_prof_read.argtypes = [i32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)]
    lib.lava_probe_stream.restype = i32
    lib.lava_probe_stream.argtypes = [vp, vp, i64, i32, i32, vp]
    return lib


lib = _load()


def status_string(status: int) -> str:
    return lib.lava_status_string(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != LAVA_OK:
        raise LavaError(status, where)


# What a call costs on the host decides how fast short layers run: the three calls of a layer took 34 us of
# which the library's own launches are 13.  Addresses go to ctypes as plain integers (no c_void_p objects),
# lengths as a C array (no numpy), and the current stream comes as its raw handle: a Stream object takes
# 3 us per call.
def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


try:
    from torch._C import _cuda_getCurrentRawStream as _raw_stream, _cuda_getDevice as _device_index
except ImportError:          # a torch without these: the public, slower way
    _raw_stream = _device_index = None


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_device_index())


def _empty(*shape, dtype, device, stream) -> torch.Tensor:
    """A buffer the call makes itself, a workspace or an output.  Its memory is the stream's the call is enqueued on, so that it is given to
    nobody else before the call has run, whenever the binding lets go of it; the stream that is current (whose caller may read
    an output) is noted as a user of it as well."""
    if stream is None:
        return torch.empty(*shape, dtype=dtype, device=device)
    if not isinstance(stream, torch.cuda.Stream):            # anything that has a handle
        stream = torch.cuda.ExternalStream(stream.cuda_stream, device)
    with torch.cuda.stream(stream):
        t = torch.empty(*shape, dtype=dtype, device=device)
    t.record_stream(torch.cuda.current_stream(device))
    return t


def _lengths(seq_lens):
    """(C array of int64, number of sequences, their sum)."""
    if type(seq_lens) in (list, tuple) and all(type(n) is int and 0 <= n < 1 << 40 for n in seq_lens):
        return (ctypes.c_int64 * len(seq_lens))(*seq_lens), len(seq_lens), sum(seq_lens)
    lens = np.asarray(seq_lens, dtype=np.int64)
    n = int(lens.shape[0])
    return (ctypes.c_int64 * n)(*lens.ravel()[:n].tolist()), n, int(lens.sum())


def _dev(t: torch.Tensor, name: str, dtype=None) -> torch.Tensor:
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous device tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must have dtype {dtype}")
    return t


def to_device(arr: np.ndarray, dtype: str, device="cuda") -> torch.Tensor:
    """Upload a stored array from the generator (float32, or uint16 bf16 bit patterns)."""
    if dtype in ("bf16", LAVA_BF16):
        return torch.from_numpy(np.ascontiguousarray(arr).view(np.int16)).to(device).view(torch.bfloat16)
    return torch.from_numpy(np.ascontiguousarray(arr, dtype=np.float32)).to(device)


def to_host_bits(t: torch.Tensor) -> np.ndarray:
    """Download rows bit for bit (bf16 as uint16 patterns, f32 as float32)."""
    if t.dtype == torch.bfloat16:
        return t.view(torch.int16).cpu().numpy().view(np.uint16)
    return t.cpu().numpy()


# ------------------------------------------------------------------------------ entry points
def set_tuning(sweep_shape="auto", sweep_workgroups=0, sweep_schedule="auto", decode_rows_per_unit=0,
               barrier_spin_limit=0, sweep_orphan_units=0) -> None:
    """lava_set_tuning; called without arguments it restores the library's own choices."""
    t = Tuning(SWEEP_SHAPES[sweep_shape], int(sweep_workgroups), SWEEP_SCHEDULES[sweep_schedule],
               int(decode_rows_per_unit), int(barrier_spin_limit), int(sweep_orphan_units))
    _check(lib.lava_set_tuning(ctypes.byref(t)), "lava_set_tuning")


def get_tuning() -> Tuning:
    t = Tuning()
    _check(lib.lava_get_tuning(ctypes.byref(t)), "lava_get_tuning")
    return t


def lava_window_scores_workspace_bytes(desc: LayerDesc, batch: int, total_tokens: int) -> int:
    return int(lib.lava_window_scores_workspace_bytes(ctypes.byref(desc), batch, total_tokens))


def lava_window_scores(desc: LayerDesc, seq_lens: Sequence[int], q_win: torch.Tensor, k: torch.Tensor,
                       v: torch.Tensor, lse: Optional[torch.Tensor] = None, scores=None, vbar=None,
                       layer_stat=None, workspace=None, stream=None, select_workspace=None, budget_plan=None):
    """Scores [sum_b H_kv * N_b] (per sequence [H_kv][N_b]), vbar [batch, H_kv], layer_stat [batch].
    With select_workspace the call is lava_window_scores_primed; with budget_plan (see make_budget_plan)
    it is lava_window_scores_planned, which also accepts select_workspace."""
    lens, batch, total = _lengths(seq_lens)
    dtype = desc.torch_dtype
    _dev(q_win, "q_win", dtype), _dev(k, "k", dtype), _dev(v, "v", dtype)
    row = desc.n_kv_heads * desc.head_dim
    if k.numel() != total * row or v.numel() != total * row:
        raise ValueError("k / v hold a different number of tokens than seq_lens")
    if q_win.numel() != batch * desc.n_q_heads * desc.window * desc.head_dim:
        raise ValueError("q_win must be [batch, H, w, d_h]")
    if lse is not None:
        _dev(lse, "lse", torch.float32)
        if lse.numel() != batch * desc.n_q_heads * desc.window:
            raise ValueError("lse must be [batch, H, w]")
    if scores is None:
        scores = _empty(total * desc.n_kv_heads, dtype=torch.float32, device=k.device, stream=stream)
    if vbar is None:
        vbar = _empty(batch, desc.n_kv_heads, dtype=torch.float32, device=k.device, stream=stream)
    if layer_stat is None:
        layer_stat = _empty(batch, dtype=torch.float32, device=k.device, stream=stream)
    if workspace is None:
        nbytes = lava_window_scores_workspace_bytes(desc, batch, total)
        workspace = _empty(max(nbytes, 256), dtype=torch.uint8, device=k.device, stream=stream)
    if budget_plan is not None:
        st = lib.lava_window_scores_planned(ctypes.byref(desc), batch, lens, _ptr(q_win),
                                            _ptr(k), _ptr(v), _ptr(lse), _ptr(scores), _ptr(vbar), _ptr(layer_stat),
                                            _ptr(workspace), workspace.numel(), _ptr(select_workspace),
                                            select_workspace.numel() if select_workspace is not None else 0,
                                            ctypes.byref(budget_plan), _stream(stream))
        _check(st, "lava_window_scores_planned")
        return scores, vbar, layer_stat
    if select_workspace is not None:
        st = lib.lava_window_scores_primed(ctypes.byref(desc), batch, lens, _ptr(q_win),
                                           _ptr(k), _ptr(v), _ptr(lse), _ptr(scores), _ptr(vbar), _ptr(layer_stat),
                                           _ptr(workspace), workspace.numel(), _ptr(select_workspace),
                                           select_workspace.numel(), _stream(stream))
        _check(st, "lava_window_scores_primed")
        return scores, vbar, layer_stat
    st = lib.lava_window_scores(ctypes.byref(desc), batch, lens, _ptr(q_win),
                                _ptr(k), _ptr(v), _ptr(lse), _ptr(scores), _ptr(vbar), _ptr(layer_stat),
                                _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, "lava_window_scores")
    return scores, vbar, layer_stat


def make_budget_plan(e: torch.Tensor, layer: int, total: torch.Tensor, lo: torch.Tensor, hi: torch.Tensor,
                     budgets: torch.Tensor) -> "BudgetPlan":
    """lava_budget_plan over device tensors e [batch, L] float32 (column `layer` is written by the scores
    call), total [batch], lo / hi / budgets [batch, L] int64.  The plan holds pointers only: keep the tensors."""
    batch, L = e.shape
    for name, t, dt in (("e", e, torch.float32), ("total", total, torch.int64), ("lo", lo, torch.int64),
                        ("hi", hi, torch.int64), ("budgets", budgets, torch.int64)):
        _dev(t, name, dt)
    if total.numel() != batch or lo.numel() != batch * L or hi.numel() != batch * L or budgets.numel() != batch * L:
        raise ValueError("budget plan tables must be [batch] / [batch, L]")
    return BudgetPlan(L, int(layer), e.data_ptr(), total.data_ptr(), lo.data_ptr(), hi.data_ptr(), budgets.data_ptr())


def lava_layer_budgets(e, total, lo, hi, budgets=None, stream=None):
    """e [batch, L] float32; total [batch], lo / hi [batch, L] int64.  All numpy (host path) or all
    device tensors (device path)."""
    on_device = isinstance(e, torch.Tensor) and e.is_cuda
    if on_device:
        batch, L = e.shape
        for name, t, dt in (("e", e, torch.float32), ("total", total, torch.int64), ("lo", lo, torch.int64),
                            ("hi", hi, torch.int64)):
            _dev(t, name, dt)
        if budgets is None:
            budgets = _empty(batch, L, dtype=torch.int64, device=e.device, stream=stream)
        st = lib.lava_layer_budgets(batch, L, _ptr(e), _ptr(total), _ptr(lo), _ptr(hi), _ptr(budgets), 1,
                                    _stream(stream))
        _check(st, "lava_layer_budgets")
        return budgets
    e = np.ascontiguousarray(np.asarray(e, dtype=np.float32))
    if e.ndim == 1:
        e = e[None, :]
    batch, L = e.shape
    total = np.ascontiguousarray(np.asarray(total, dtype=np.int64).reshape(batch))
    lo = np.ascontiguousarray(np.broadcast_to(np.asarray(lo, dtype=np.int64), (batch, L)))
    hi = np.ascontiguousarray(np.broadcast_to(np.asarray(hi, dtype=np.int64), (batch, L)))
    out = np.zeros((batch, L), dtype=np.int64)
    as_vp = lambda a: a.ctypes.data_as(ctypes.c_void_p)
    st = lib.lava_layer_budgets(batch, L, as_vp(e), as_vp(total), as_vp(lo), as_vp(hi), as_vp(out), 0, None)
    _check(st, "lava_layer_budgets")
    return out


def lava_select_workspace_bytes(total_entries: int) -> int:
    return int(lib.lava_select_workspace_bytes(total_entries))


def lava_select_topk(n_heads: int, scores: torch.Tensor, budget: int, seg_offsets: Optional[torch.Tensor] = None,
                     budget_dev: Optional[torch.Tensor] = None, total_entries: Optional[int] = None,
                     head_counts=None, head_offsets=None, kept_idx=None, kept_scores=None,
                     want_scores: bool = True, workspace=None, stream=None, primed: bool = False):
    """primed: `workspace` was prepared by lava_window_scores(select_workspace=workspace) for these scores."""
    _dev(scores, "scores", torch.float32)
    total = scores.numel() if total_entries is None else int(total_entries)
    if seg_offsets is not None:
        _dev(seg_offsets, "seg_offsets", torch.int64)
    if budget_dev is not None:
        _dev(budget_dev, "budget_dev", torch.int64)
    if head_counts is None:
        head_counts = _empty(n_heads, dtype=torch.int32, device=scores.device, stream=stream)
    if head_offsets is None:
        head_offsets = _empty(n_heads + 1, dtype=torch.int64, device=scores.device, stream=stream)
    if kept_idx is None:
        kept_idx = _empty(max(int(budget), 1), dtype=torch.int32, device=scores.device, stream=stream)
    if kept_scores is None and want_scores:
        kept_scores = _empty(max(int(budget), 1), dtype=torch.float32, device=scores.device, stream=stream)
    if workspace is None:
        workspace = _empty(max(lava_select_workspace_bytes(total), 256), dtype=torch.uint8, device=scores.device, stream=stream)
    if primed:
        if seg_offsets is not None:
            raise ValueError("a prepared workspace serves equal segments only")
        st = lib.lava_select_topk_primed(n_heads, _ptr(scores), total, int(budget), _ptr(budget_dev),
                                         _ptr(head_counts), _ptr(head_offsets), _ptr(kept_idx), _ptr(kept_scores),
                                         _ptr(workspace), workspace.numel(), _stream(stream))
        _check(st, "lava_select_topk_primed")
        return head_counts, head_offsets, kept_idx, kept_scores
    st = lib.lava_select_topk(n_heads, _ptr(scores), _ptr(seg_offsets), total, int(budget), _ptr(budget_dev),
                              _ptr(head_counts), _ptr(head_offsets), _ptr(kept_idx), _ptr(kept_scores),
                              _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, "lava_select_topk")
    return head_counts, head_offsets, kept_idx, kept_scores


SELECT_STATIC_MAX_ENTRIES = 1 << 22


def lava_select_topk_static(n_heads: int, scores: torch.Tensor, budget: int, head_counts: torch.Tensor,
                            head_offsets: torch.Tensor, kept_idx: torch.Tensor,
                            kept_scores: Optional[torch.Tensor] = None, seg_offsets: Optional[torch.Tensor] = None,
                            budget_dev: Optional[torch.Tensor] = None, total_entries: Optional[int] = None,
                            stream=None) -> None:
    """lava_select_topk on the library's built-in scratch array.  Allocates nothing: every buffer is the caller's."""
    _dev(scores, "scores", torch.float32), _dev(head_counts, "head_counts", torch.int32)
    _dev(head_offsets, "head_offsets", torch.int64), _dev(kept_idx, "kept_idx", torch.int32)
    for name, t, dt in (("kept_scores", kept_scores, torch.float32), ("seg_offsets", seg_offsets, torch.int64),
                        ("budget_dev", budget_dev, torch.int64)):
        if t is not None:
            _dev(t, name, dt)
    total = scores.numel() if total_entries is None else int(total_entries)
    st = lib.lava_select_topk_static(n_heads, _ptr(scores), _ptr(seg_offsets), total, int(budget), _ptr(budget_dev),
                                     _ptr(head_counts), _ptr(head_offsets), _ptr(kept_idx), _ptr(kept_scores),
                                     _stream(stream))
    _check(st, "lava_select_topk_static")


def lava_select_status(workspace: torch.Tensor, total_entries: int, stream=None) -> int:
    """Synchronises; LAVA_OK, or LAVA_ERR_HIP if the selection's bounded barrier wait gave up."""
    return int(lib.lava_select_status(_ptr(workspace), int(total_entries), _stream(stream)))


class SelectProblem(ctypes.Structure):
    """Mirror of lava_select_problem."""
    _fields_ = [
        ("scores", ctypes.c_void_p), ("seg_offsets", ctypes.c_void_p), ("total_entries", ctypes.c_int64),
        ("budget", ctypes.c_int64), ("budget_dev", ctypes.c_void_p), ("head_counts", ctypes.c_void_p),
        ("head_offsets", ctypes.c_void_p), ("kept_idx", ctypes.c_void_p), ("kept_scores", ctypes.c_void_p),
        ("in_offset_dev", ctypes.c_void_p), ("out_offset_dev", ctypes.c_void_p), ("error_dev", ctypes.c_void_p),
        ("primed", ctypes.c_int32),
    ]


class CompactProblem(ctypes.Structure):
    """Mirror of lava_compact_problem."""
    _fields_ = [
        ("src_rows", ctypes.c_int64), ("src_offsets", ctypes.c_void_p), ("k_src", ctypes.c_void_p),
        ("v_src", ctypes.c_void_p), ("pos_src", ctypes.c_void_p), ("head_offsets", ctypes.c_void_p),
        ("kept_idx", ctypes.c_void_p), ("capacity", ctypes.c_int64), ("k_out", ctypes.c_void_p),
        ("v_out", ctypes.c_void_p), ("pos_out", ctypes.c_void_p),
        ("src_offset_dev", ctypes.c_void_p), ("out_offset_dev", ctypes.c_void_p),
    ]


def _addr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def select_problem(scores, budget, head_counts, head_offsets, kept_idx, kept_scores=None, seg_offsets=None,
                   budget_dev=None, total_entries=None, in_offset_dev=None, out_offset_dev=None,
                   error_dev=None, primed=False) -> SelectProblem:
    """One row of the table of lava_select_topk_batch from device tensors (the caller keeps them alive)."""
    _dev(scores, "scores", torch.float32), _dev(head_counts, "head_counts", torch.int32)
    _dev(head_offsets, "head_offsets", torch.int64), _dev(kept_idx, "kept_idx", torch.int32)
    for name, t, dt in (("kept_scores", kept_scores, torch.float32), ("seg_offsets", seg_offsets, torch.int64),
                        ("budget_dev", budget_dev, torch.int64), ("in_offset_dev", in_offset_dev, torch.int64),
                        ("out_offset_dev", out_offset_dev, torch.int64), ("error_dev", error_dev, torch.int32)):
        if t is not None:
            _dev(t, name, dt)
    total = scores.numel() if total_entries is None else int(total_entries)
    return SelectProblem(_addr(scores), _addr(seg_offsets), total, int(budget), _addr(budget_dev),
                         _addr(head_counts), _addr(head_offsets), _addr(kept_idx), _addr(kept_scores),
                         _addr(in_offset_dev), _addr(out_offset_dev), _addr(error_dev), 1 if primed else 0)


def compact_problem(desc: LayerDesc, src_rows, k_src, v_src, head_offsets, kept_idx, capacity, k_out, v_out,
                    src_offsets=None, pos_src=None, pos_out=None, src_offset_dev=None,
                    out_offset_dev=None) -> CompactProblem:
    """One row of the table of lava_compact_batch (dense source when src_offsets is None)."""
    for name, t in (("k_src", k_src), ("v_src", v_src), ("k_out", k_out), ("v_out", v_out)):
        _dev(t, name, desc.torch_dtype)
    _dev(head_offsets, "head_offsets", torch.int64), _dev(kept_idx, "kept_idx", torch.int32)
    for name, t, dt in (("src_offsets", src_offsets, torch.int64), ("pos_src", pos_src, torch.int32),
                        ("pos_out", pos_out, torch.int32), ("src_offset_dev", src_offset_dev, torch.int64),
                        ("out_offset_dev", out_offset_dev, torch.int64)):
        if t is not None:
            _dev(t, name, dt)
    return CompactProblem(int(src_rows), _addr(src_offsets), _addr(k_src), _addr(v_src), _addr(pos_src),
                          _addr(head_offsets), _addr(kept_idx), int(capacity), _addr(k_out), _addr(v_out),
                          _addr(pos_out), _addr(src_offset_dev), _addr(out_offset_dev))


def lava_select_batch_workspace_bytes(n_problems: int, max_total_entries: int) -> int:
    return int(lib.lava_select_batch_workspace_bytes(int(n_problems), int(max_total_entries)))


def lava_select_topk_batch(n_heads: int, problems, max_total_entries=None, workspace=None, device="cuda",
                           stream=None):
    """problems: sequence of SelectProblem, or a ready (SelectProblem * n) array that a caller reuses from
    step to step.  Returns the workspace (for lava_select_batch_status)."""
    table = problems if isinstance(problems, ctypes.Array) else (SelectProblem * len(problems))(*problems)
    widest = max((p.total_entries for p in problems), default=0) if max_total_entries is None else int(max_total_entries)
    if workspace is None:
        need = lava_select_batch_workspace_bytes(len(problems), widest)
        workspace = _empty(max(need, 256), dtype=torch.uint8, device=device, stream=stream)
    st = lib.lava_select_topk_batch(int(n_heads), len(problems), ctypes.cast(table, ctypes.c_void_p), widest,
                                    _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, "lava_select_topk_batch")
    return workspace


def lava_select_batch_status(workspace: torch.Tensor, n_problems: int, max_total_entries: int, stream=None) -> int:
    return int(lib.lava_select_batch_status(_ptr(workspace), int(n_problems), int(max_total_entries),
                                            _stream(stream)))


def lava_compact_batch(desc: LayerDesc, problems, stream=None) -> None:
    """problems: sequence of CompactProblem, or a ready (CompactProblem * n) array."""
    table = problems if isinstance(problems, ctypes.Array) else (CompactProblem * len(problems))(*problems)
    st = lib.lava_compact_batch(ctypes.byref(desc), len(problems), ctypes.cast(table, ctypes.c_void_p),
                                _stream(stream))
    _check(st, "lava_compact_batch")


def lava_compact_kv(desc: LayerDesc, n: int, k: torch.Tensor, v: torch.Tensor, head_offsets: torch.Tensor,
                    kept_idx: torch.Tensor, capacity: int, k_out=None, v_out=None, stream=None):
    _dev(k, "k", desc.torch_dtype), _dev(v, "v", desc.torch_dtype)
    _dev(head_offsets, "head_offsets", torch.int64), _dev(kept_idx, "kept_idx", torch.int32)
    if k_out is None:
        k_out = _empty(max(int(capacity), 1), desc.head_dim, dtype=desc.torch_dtype, device=k.device, stream=stream)
    if v_out is None:
        v_out = _empty(max(int(capacity), 1), desc.head_dim, dtype=desc.torch_dtype, device=k.device, stream=stream)
    st = lib.lava_compact_kv(ctypes.byref(desc), int(n), _ptr(k), _ptr(v), _ptr(head_offsets), _ptr(kept_idx),
                             int(capacity), _ptr(k_out), _ptr(v_out), _stream(stream))
    _check(st, "lava_compact_kv")
    return k_out, v_out


def lava_compact_packed(desc: LayerDesc, src_offsets: torch.Tensor, k_src: torch.Tensor, v_src: torch.Tensor,
                        head_offsets: torch.Tensor, kept_idx: torch.Tensor, capacity: int, pos_src=None,
                        k_out=None, v_out=None, pos_out=None, stream=None):
    """Gather from an already packed cache (re-eviction).  Returns (k_out, v_out, pos_out)."""
    _dev(k_src, "k_src", desc.torch_dtype), _dev(v_src, "v_src", desc.torch_dtype)
    _dev(src_offsets, "src_offsets", torch.int64), _dev(head_offsets, "head_offsets", torch.int64)
    _dev(kept_idx, "kept_idx", torch.int32)
    if pos_src is not None:
        _dev(pos_src, "pos_src", torch.int32)
    rows = max(int(capacity), 1)
    if k_out is None:
        k_out = _empty(rows, desc.head_dim, dtype=desc.torch_dtype, device=k_src.device, stream=stream)
    if v_out is None:
        v_out = _empty(rows, desc.head_dim, dtype=desc.torch_dtype, device=k_src.device, stream=stream)
    if pos_out is None:
        pos_out = _empty(rows, dtype=torch.int32, device=k_src.device, stream=stream)
    st = lib.lava_compact_packed(ctypes.byref(desc), _ptr(src_offsets), k_src.shape[0], _ptr(k_src), _ptr(v_src),
                                 _ptr(pos_src), _ptr(head_offsets), _ptr(kept_idx), int(capacity), _ptr(k_out),
                                 _ptr(v_out), _ptr(pos_out), _stream(stream))
    _check(st, "lava_compact_packed")
    return k_out, v_out, pos_out


class CascadeStateStruct(ctypes.Structure):
    """Mirror of lava_cascade_state."""
    _fields_ = [
        ("k", ctypes.c_void_p * 2), ("v", ctypes.c_void_p * 2), ("pos", ctypes.c_void_p * 2),
        ("scores", ctypes.c_void_p * 2), ("head_offsets", ctypes.c_void_p * 2), ("layer_start", ctypes.c_void_p * 2),
        ("head_counts", ctypes.c_void_p), ("kept_idx", ctypes.c_void_p), ("error", ctypes.c_void_p),
        ("capacity", ctypes.c_int64), ("max_layers", ctypes.c_int32), ("cur", ctypes.c_int32),
    ]


class CascadeState:
    """Device buffers of a stack of layers for lava_cascade_step (allocation and views only): two arenas of
    `capacity` rows in which the layers sit back to back, plus the per-layer offsets.  in_place: K and V
    share ONE arena (the step re-compacts the earlier layers inside it), which halves the state."""

    def __init__(self, desc: LayerDesc, max_layers: int, capacity: int, device="cuda", in_place: bool = False):
        self.desc, self.n_layers, self.capacity = desc, int(max_layers), int(capacity)
        self.in_place = bool(in_place)
        hk = desc.n_kv_heads
        self.k = [torch.empty(capacity, desc.head_dim, dtype=desc.torch_dtype, device=device)]
        self.v = [torch.empty(capacity, desc.head_dim, dtype=desc.torch_dtype, device=device)]
        self.k.append(self.k[0] if in_place else torch.empty_like(self.k[0]))
        self.v.append(self.v[0] if in_place else torch.empty_like(self.v[0]))
        self.pos = [torch.empty(capacity, dtype=torch.int32, device=device) for _ in range(2)]
        self.scores = [torch.empty(capacity, dtype=torch.float32, device=device) for _ in range(2)]
        self.head_offsets = [torch.zeros(max_layers, hk + 1, dtype=torch.int64, device=device) for _ in range(2)]
        self.layer_start = [torch.zeros(max_layers + 1, dtype=torch.int64, device=device) for _ in range(2)]
        self.head_counts = torch.zeros(max_layers, hk, dtype=torch.int32, device=device)
        self.kept_idx = torch.empty(capacity, dtype=torch.int32, device=device)
        self.error = torch.zeros(1, dtype=torch.int32, device=device)
        self.e = torch.zeros(max_layers, dtype=torch.float32, device=device)
        self.budgets = torch.zeros(max_layers, dtype=torch.int64, device=device)
        c = self.c = CascadeStateStruct()
        for i in range(2):
            c.k[i], c.v[i], c.pos[i] = self.k[i].data_ptr(), self.v[i].data_ptr(), self.pos[i].data_ptr()
            c.scores[i] = self.scores[i].data_ptr()
            c.head_offsets[i], c.layer_start[i] = self.head_offsets[i].data_ptr(), self.layer_start[i].data_ptr()
        c.head_counts, c.kept_idx = self.head_counts.data_ptr(), self.kept_idx.data_ptr()
        c.error = self.error.data_ptr()
        c.capacity, c.max_layers, c.cur = self.capacity, self.n_layers, 0

    @property
    def cur(self) -> int:
        return int(self.c.cur)

    def reset(self) -> None:
        self.c.cur = 0
        self.error.zero_()

    def bytes(self) -> int:
        """Device bytes the state holds."""
        ts = (self.k[:1] + self.v[:1] if self.in_place else self.k + self.v)
        ts = ts + self.pos + self.scores + self.head_offsets + self.layer_start
        ts += [self.head_counts, self.kept_idx, self.e, self.budgets]
        return sum(t.numel() * t.element_size() for t in ts)

    def decode_args(self, t: int) -> dict:
        """What lava_decode_attention needs to read layer t in place (nothing is read back)."""
        c = self.cur
        return dict(k_hat=self.k[c], v_hat=self.v[c], head_offsets=self.head_offsets[c][t: t + 1],
                    seq_base=self.layer_start[c][t: t + 1], rows_capacity=self.capacity)

    def current(self, t: int) -> dict:
        """Views of layer t's current state (reads the layer's extent back: synchronises)."""
        c = self.cur
        start, end = (int(x) for x in self.layer_start[c][t: t + 2].cpu())
        return dict(k_hat=self.k[c][start:end], v_hat=self.v[c][start:end], pos=self.pos[c][start:end],
                    scores=self.scores[c][start:end], head_offsets=self.head_offsets[c][t],
                    head_counts=self.head_counts[t], start=start)


def lava_cascade_workspace_bytes(desc: LayerDesc, n: int, n_layers: int, total_budget: int) -> int:
    return int(lib.lava_cascade_workspace_bytes(ctypes.byref(desc), int(n), int(n_layers), int(total_budget)))


def lava_cascade_step(desc: LayerDesc, layer: int, n: int, k_new: torch.Tensor, v_new: torch.Tensor,
                      scores_new: torch.Tensor, state: CascadeState, total_budget: int, workspace=None, stream=None):
    """Alg. 2, one outer iteration; state.e[: layer + 1] must hold the layers' statistics."""
    _dev(k_new, "k_new", desc.torch_dtype), _dev(v_new, "v_new", desc.torch_dtype)
    _dev(scores_new, "scores_new", torch.float32)
    if workspace is None:
        need = lava_cascade_workspace_bytes(desc, n, state.n_layers, total_budget)
        workspace = _empty(max(need, 256), dtype=torch.uint8, device=k_new.device, stream=stream)
    st = lib.lava_cascade_step(ctypes.byref(desc), int(layer), int(n), _ptr(k_new), _ptr(v_new), _ptr(scores_new),
                               _ptr(state.e), int(total_budget), ctypes.byref(state.c),
                               _ptr(state.budgets), _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, "lava_cascade_step")
    return workspace


def lava_decode_workspace_bytes(desc: LayerDesc, batch: int, rows_capacity: int, tail_len: int = 0) -> int:
    return int(lib.lava_decode_workspace_bytes(ctypes.byref(desc), int(batch), int(rows_capacity), int(tail_len)))


def lava_decode_attention(desc: LayerDesc, batch: int, q: torch.Tensor, k_hat, v_hat, head_offsets: torch.Tensor,
                          rows_capacity: int, seq_base=None, k_tail=None, v_tail=None, tail_len: int = 0,
                          tail_capacity: int = 0, out=None, lse=None, workspace=None, stream=None):
    """One new token per sequence attends to the packed cache (+ dense tail).  Returns (out, lse)."""
    _dev(q, "q", desc.torch_dtype), _dev(head_offsets, "head_offsets", torch.int64)
    for name, t in (("k_hat", k_hat), ("v_hat", v_hat), ("k_tail", k_tail), ("v_tail", v_tail)):
        if t is not None:
            _dev(t, name, desc.torch_dtype)
    if seq_base is not None:
        _dev(seq_base, "seq_base", torch.int64)
    if out is None:
        out = _empty(batch, desc.n_q_heads, desc.head_dim, dtype=torch.float32, device=q.device, stream=stream)
    if lse is None:
        lse = _empty(batch, desc.n_q_heads, dtype=torch.float32, device=q.device, stream=stream)
    if workspace is None:
        need = lava_decode_workspace_bytes(desc, batch, rows_capacity, tail_len)
        workspace = _empty(max(need, 256), dtype=torch.uint8, device=q.device, stream=stream)
    st = lib.lava_decode_attention(ctypes.byref(desc), int(batch), _ptr(q), _ptr(k_hat), _ptr(v_hat),
                                   _ptr(head_offsets), _ptr(seq_base), int(rows_capacity), _ptr(k_tail),
                                   _ptr(v_tail), int(tail_len), int(tail_capacity), _ptr(out), _ptr(lse),
                                   _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, "lava_decode_attention")
    return out, lse


# ------------------------------------------------------------------------------ the paged cache
LAVA_PAGES_EXHAUSTED, LAVA_PAGES_BLOCKS, LAVA_PAGES_INVALID, LAVA_PAGES_TOKENS = 1, 2, 4, 8


class PagePoolStruct(ctypes.Structure):
    """Mirror of lava_page_pool."""
    _fields_ = [("n_pages", ctypes.c_int64), ("page_rows", ctypes.c_int32), ("max_blocks", ctypes.c_int32),
                ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("pos", ctypes.c_void_p)]


class PagePool:
    """A pool of pages over device tensors k, v [n_pages, page_rows, d_h] and pos [n_pages, page_rows] int32 or None
    (the tensors are kept).  max_blocks: pages a head's block table has room for (not needed to append)."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, pos: Optional[torch.Tensor] = None, max_blocks: int = 1):
        _dev(k, "k"), _dev(v, "v", k.dtype)
        if k.dim() != 3 or v.shape != k.shape:
            raise ValueError("k and v must be [n_pages, page_rows, d_h]")
        if pos is not None and tuple(_dev(pos, "pos", torch.int32).shape) != tuple(k.shape[:2]):
            raise ValueError("pos must be [n_pages, page_rows]")
        self.k, self.v, self.pos, self.max_blocks = k, v, pos, int(max_blocks)
        self.c = PagePoolStruct(k.shape[0], k.shape[1], self.max_blocks, _ptr(k), _ptr(v), _ptr(pos))
        self._ref = ctypes.byref(self.c)

    def _check(self, desc: LayerDesc) -> None:
        if self.k.dtype != desc.torch_dtype or self.k.shape[2] != desc.head_dim:
            raise ValueError("the pool's pages have another type or head dimension than the descriptor")


class PageStateStruct(ctypes.Structure):
    """Mirror of lava_page_state."""
    _fields_ = [(name, ctypes.c_void_p) for name in (
        "block_table", "head_rows", "seq_pos", "free_pages", "n_free", "head_rows_out", "seq_pos_out", "n_free_out", "error")]


class PageState:
    """What lava_page_tables keeps between steps, over device tensors (all int32): block_table
    [batch, H_kv, max_blocks], head_rows [batch, H_kv], seq_pos [batch], free_pages [n_pages] (a stack), n_free [1].
    The *_out tensors receive the counts after a step; left out, a step is made in place."""

    def __init__(self, block_table, head_rows, seq_pos, free_pages, n_free, page_rows: int, head_rows_out=None,
                 seq_pos_out=None, n_free_out=None, error=None):
        if block_table.dim() != 3:
            raise ValueError("block_table must be [batch, H_kv, max_blocks]")
        self.batch, self.n_kv_heads, self.max_blocks = block_table.shape
        self.page_rows, self.n_pages = int(page_rows), free_pages.numel()
        self.block_table, self.free_pages, self.error = block_table, free_pages, error
        self.head_rows, self.seq_pos, self.n_free = head_rows, seq_pos, n_free
        self.head_rows_out = head_rows if head_rows_out is None else head_rows_out
        self.seq_pos_out = seq_pos if seq_pos_out is None else seq_pos_out
        self.n_free_out = n_free if n_free_out is None else n_free_out
        heads = self.batch * self.n_kv_heads
        for name, t, n in (("block_table", block_table, None), ("free_pages", free_pages, None), ("head_rows", head_rows, heads),
                           ("head_rows_out", self.head_rows_out, heads), ("seq_pos", seq_pos, self.batch),
                           ("seq_pos_out", self.seq_pos_out, self.batch), ("n_free", n_free, 1), ("n_free_out", self.n_free_out, 1),
                           ("error", error, 1)):
            if t is None:
                continue
            _dev(t, name, torch.int32)
            if n is not None and t.numel() != n:
                raise ValueError(f"{name} must hold {n} values")
        self.c = PageStateStruct(*(_ptr(t) for t in (block_table, head_rows, seq_pos, free_pages, n_free, self.head_rows_out,
                                                     self.seq_pos_out, self.n_free_out, error)))
        self._sizes = PagePoolStruct(self.n_pages, self.page_rows, self.max_blocks, None, None, None)
        self._ref, self._sizes_ref = ctypes.byref(self.c), ctypes.byref(self._sizes)

    @classmethod
    def empty(cls, batch: int, n_kv_heads: int, max_blocks: int, n_pages: int, page_rows: int, device="cuda") -> "PageState":
        """No sequence holds a row and every page is free; steps are made in place."""
        new = lambda *shape: torch.zeros(*shape, dtype=torch.int32, device=device)
        free = torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device=device)     # page 0 is taken first
        return cls(new(batch, n_kv_heads, max_blocks), new(batch, n_kv_heads), new(batch), free,
                   torch.full((1,), n_pages, dtype=torch.int32, device=device), page_rows, error=new(1))


def lava_page_tables_workspace_bytes(batch: int, n_kv_heads: int) -> int:
    return int(lib.lava_page_tables_workspace_bytes(int(batch), int(n_kv_heads)))


def lava_page_tables(state: PageState, n_new: Optional[torch.Tensor] = None, head_counts: Optional[torch.Tensor] = None,
                     release: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None,
                     positions: Optional[torch.Tensor] = None, workspace=None, stream=None):
    """Pages, block tables and slots of one step; n_new / release [batch], head_counts [batch, H_kv] int32; slots
    [max_tokens, H_kv] int64 and positions [max_tokens] int32 are written.  Returns (slots, positions)."""
    for name, t, n in (("n_new", n_new, state.batch), ("release", release, state.batch),
                       ("head_counts", head_counts, state.batch * state.n_kv_heads)):
        if t is not None and _dev(t, name, torch.int32).numel() != n:
            raise ValueError(f"{name} must hold {n} values")
    _here(state.block_table)
    max_tokens = 0
    if slots is not None:
        max_tokens = _dev(slots, "slots", torch.int64).numel() // state.n_kv_heads
        if slots.numel() != max_tokens * state.n_kv_heads:
            raise ValueError("slots must be [max_tokens, H_kv]")
    if positions is not None:
        _dev(positions, "positions", torch.int32)
        if slots is not None and positions.numel() != max_tokens:
            raise ValueError("slots and positions must be for the same number of tokens")
        max_tokens = positions.numel()
    if workspace is None:
        need = lava_page_tables_workspace_bytes(state.batch, state.n_kv_heads)
        workspace = _empty(max(need, 256), dtype=torch.uint8, device=state.block_table.device, stream=stream)
    st = lib.lava_page_tables(state._sizes_ref, state.batch, state.n_kv_heads, state._ref, _ptr(n_new), _ptr(head_counts),
                              _ptr(release), max_tokens, _ptr(slots), _ptr(positions), _ptr(workspace), workspace.numel(),
                              _stream(stream))
    _check(st, "lava_page_tables")
    return slots, positions


class PagedCompactProblem(ctypes.Structure):
    """Mirror of lava_paged_compact_problem."""
    _fields_ = [
        ("src_rows", ctypes.c_int64), ("src_offsets", ctypes.c_void_p), ("k_src", ctypes.c_void_p),
        ("v_src", ctypes.c_void_p), ("pos_src", ctypes.c_void_p), ("head_offsets", ctypes.c_void_p),
        ("kept_idx", ctypes.c_void_p), ("capacity", ctypes.c_int64), ("block_table", ctypes.c_void_p),
        ("first_rows", ctypes.c_void_p), ("table_blocks", ctypes.c_int32),
    ]


def paged_compact_problem(desc: LayerDesc, src_rows, k_src, v_src, head_offsets, kept_idx, capacity, block_table,
                          first_rows=None, src_offsets=None, pos_src=None) -> PagedCompactProblem:
    """One row of the table of lava_compact_paged (dense source when src_offsets is None); block_table: the sequence's
    [H_kv, max_blocks], as many blocks as the pool's.  The caller keeps the tensors."""
    for name, t in (("k_src", k_src), ("v_src", v_src)):
        _dev(t, name, desc.torch_dtype)
    _dev(head_offsets, "head_offsets", torch.int64), _dev(kept_idx, "kept_idx", torch.int32)
    for name, t, dt in (("block_table", block_table, torch.int32), ("first_rows", first_rows, torch.int32),
                        ("src_offsets", src_offsets, torch.int64), ("pos_src", pos_src, torch.int32)):
        if t is not None:
            _dev(t, name, dt)
    if head_offsets.numel() != desc.n_kv_heads + 1 or kept_idx.numel() < int(capacity):
        raise ValueError("head_offsets must hold H_kv + 1 values and kept_idx `capacity` ones")
    hkv = desc.n_kv_heads
    rows = int(src_rows) * (1 if src_offsets is not None else hkv)
    if k_src.numel() != rows * desc.head_dim or v_src.numel() != rows * desc.head_dim:
        raise ValueError("k_src / v_src hold a different number of rows than src_rows")
    for name, t, n in (("src_offsets", src_offsets, hkv + 1), ("pos_src", pos_src, rows), ("first_rows", first_rows, hkv)):
        if t is not None and t.numel() != n:
            raise ValueError(f"{name} must hold {n} values")
    blocks = block_table.numel() // hkv
    if blocks < 1 or block_table.numel() != blocks * hkv:
        raise ValueError("block_table must be [H_kv, max_blocks]")
    return PagedCompactProblem(int(src_rows), _addr(src_offsets), _addr(k_src), _addr(v_src), _addr(pos_src),
                               _addr(head_offsets), _addr(kept_idx), int(capacity), _addr(block_table), _addr(first_rows), blocks)


def lava_compact_paged(desc: LayerDesc, problems, pool: PagePool, stream=None) -> None:
    """problems: sequence of PagedCompactProblem, or a ready (PagedCompactProblem * n) array."""
    pool._check(desc)
    _here(pool.k)
    table = problems if isinstance(problems, ctypes.Array) else (PagedCompactProblem * len(problems))(*problems)
    st = lib.lava_compact_paged(ctypes.byref(desc), len(problems), ctypes.cast(table, ctypes.c_void_p), pool._ref, _stream(stream))
    _check(st, "lava_compact_paged")


class RotaryDesc(ctypes.Structure):
    """Mirror of lava_rotary_desc."""
    _fields_ = [("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("magnitude", ctypes.c_float),
                ("original_context", ctypes.c_int32), ("base", ctypes.c_double), ("factor", ctypes.c_double),
                ("low_turns", ctypes.c_double), ("high_turns", ctypes.c_double)]

    @classmethod
    def make(cls, rotary_dim, interleaved=False, magnitude=1.0, base=10000.0, factor=1.0, original_context=0, low_turns=1.0,
             high_turns=4.0):
        return cls(int(rotary_dim), 1 if interleaved else 0, magnitude, int(original_context), base, factor, low_turns, high_turns)


def lava_rotary_turns(rot: RotaryDesc, device=None) -> torch.Tensor:
    """The angles of one token in 2^-64 turns [rotary_dim / 2]: the table lava_rotary takes, as int64 bit patterns."""
    out = torch.empty(max(rot.rotary_dim // 2, 1), dtype=torch.int64)
    _check(lib.lava_rotary_turns(ctypes.byref(rot), out.data_ptr()), "lava_rotary_turns")
    return out if device is None else out.to(device)


def _here(t: torch.Tensor) -> None:
    """The library works on the current device, on whose stream the call is enqueued."""
    if _device_index is not None and t.is_cuda and t.get_device() != _device_index():
        raise ValueError("the tensors are on another device than the current one")


def _rows_of_heads(t: torch.Tensor, name: str, dtype) -> torch.Tensor:
    """[tokens, heads, d_h] whose heads are contiguous rows (any strides between them)."""
    if not t.is_cuda or t.dim() != 3 or t.stride(2) != 1 or t.dtype != dtype:
        raise ValueError(f"{name} must be a device tensor [tokens, heads, d_h] of {dtype} with contiguous heads")
    return t


def _token_stride(t: torch.Tensor, name: str, dtype, shape) -> int:
    """The stride of the tokens of t, of that shape, whose heads lie one after another."""
    if t.shape != shape or not t.is_cuda or t.dtype != dtype:
        raise ValueError(f"{name} must be a device tensor {list(shape)} of {dtype}")
    stride = t.stride()
    if stride[2] != 1 or (stride[1] != shape[2] and shape[1] > 1):
        raise ValueError(f"{name} must have its heads one after another")
    return stride[0]


def _check_turns(rot: RotaryDesc, turns: torch.Tensor, positions: torch.Tensor, tokens: int) -> None:
    if _dev(turns, "turns", torch.int64).numel() < rot.rotary_dim // 2:
        raise ValueError("turns must hold rotary_dim / 2 values")
    if _dev(positions, "positions", torch.int32).numel() != tokens:
        raise ValueError("positions must be [tokens]")


def lava_rotary(rot: RotaryDesc, turns: torch.Tensor, positions: torch.Tensor, x: torch.Tensor,
                out: Optional[torch.Tensor] = None, transpose: bool = False, stream=None) -> torch.Tensor:
    """x [tokens, heads, d_h] turned by its tokens' positions into `out` (x itself, or any view of that shape)."""
    dt = torch.bfloat16 if x.dtype == torch.bfloat16 else torch.float32
    _rows_of_heads(x, "x", dt)
    tokens, heads, d = x.shape
    _here(x)
    _check_turns(rot, turns, positions, tokens)
    if out is None:
        out = _empty(x.shape, dtype=dt, device=x.device, stream=stream)
    if _rows_of_heads(out, "out", dt).shape != x.shape:
        raise ValueError("out must have the shape of x")
    st = lib.lava_rotary(ctypes.byref(rot), _ptr(turns), LAVA_BF16 if dt == torch.bfloat16 else LAVA_F32, d, tokens, heads,
                         _ptr(positions), _ptr(x), x.stride(0), x.stride(1), _ptr(out), out.stride(0), out.stride(1),
                         1 if transpose else 0, _stream(stream))
    _check(st, "lava_rotary")
    return out


def lava_rotary_append(desc: LayerDesc, rot: RotaryDesc, turns: torch.Tensor, positions: torch.Tensor,
                       q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, pool: PagePool, slots: torch.Tensor,
                       q_out: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
    """New tokens into the paged cache; q [tokens, H, d_h] (or None), k, v [tokens, H_kv, d_h], parts of one projection's
    output allowed.  Returns q_out, the rotated queries [tokens, H, d_h]."""
    dt, d, hq, hkv = desc.torch_dtype, desc.head_dim, desc.n_q_heads, desc.n_kv_heads
    tokens = k.shape[0]
    _here(k)
    k_stride, v_stride = _token_stride(k, "k", dt, (tokens, hkv, d)), _token_stride(v, "v", dt, (tokens, hkv, d))
    q_stride = 0
    if q is not None:
        q_stride = _token_stride(q, "q", dt, (tokens, hq, d))
        if q_out is None:
            q_out = _empty(tokens, hq, d, dtype=dt, device=q.device, stream=stream)
        elif q_out.numel() != tokens * hq * d:
            raise ValueError("q_out must be [tokens, H, d_h]")
        elif q_out is not q:
            _dev(q_out, "q_out", dt)
    _check_turns(rot, turns, positions, tokens)
    pool._check(desc)
    if _dev(slots, "slots", torch.int64).numel() != tokens * hkv:
        raise ValueError("slots must be [tokens, H_kv]")
    st = lib.lava_rotary_append(ctypes.byref(desc), ctypes.byref(rot), _ptr(turns), tokens, _ptr(positions), _ptr(q),
                                q_stride, _ptr(k), k_stride, _ptr(v), v_stride,
                                _ptr(q_out) if q is not None else None, pool._ref, _ptr(slots), _stream(stream))
    _check(st, "lava_rotary_append")
    return q_out


class DecodeOptions(ctypes.Structure):
    """Mirror of lava_decode_options."""
    _fields_ = [("softcap", ctypes.c_float), ("window", ctypes.c_int32), ("slopes", ctypes.c_void_p)]

    @classmethod
    def make(cls, softcap=0.0, window=0, slopes: Optional[torch.Tensor] = None) -> "DecodeOptions":
        o = cls(softcap, int(window), _ptr(None if slopes is None else _dev(slopes, "slopes", torch.float32)))
        o.tensor = slopes                                  # kept: the structure holds its address only
        return o


def lava_paged_decode_workspace_bytes(desc: LayerDesc) -> int:
    return int(lib.lava_paged_decode_workspace_bytes(ctypes.byref(desc)))


def _decode_tensors(desc: LayerDesc, q: torch.Tensor, pool: PagePool, block_table: torch.Tensor, head_rows: torch.Tensor, options, q_pos, out,
                    lse, stream):
    """The checks of a decode step over pages.  Returns (batch, out, lse)."""
    _dev(q, "q", desc.torch_dtype), _dev(block_table, "block_table", torch.int32), _dev(head_rows, "head_rows", torch.int32)
    _here(q)
    batch = q.numel() // (desc.n_q_heads * desc.head_dim)
    heads = batch * desc.n_kv_heads
    if q.numel() != batch * desc.n_q_heads * desc.head_dim:
        raise ValueError("q must be [batch, H, d_h]")
    if head_rows.numel() != heads or block_table.numel() != heads * pool.max_blocks:
        raise ValueError("head_rows must be [batch, H_kv] and block_table [batch, H_kv, max_blocks]")
    pool._check(desc)
    if q_pos is not None and _dev(q_pos, "q_pos", torch.int32).numel() != batch:
        raise ValueError("q_pos must be [batch]")
    slopes = getattr(options, "tensor", None)
    if slopes is not None and slopes.numel() != desc.n_q_heads:
        raise ValueError("slopes must be [H]")
    if out is None:
        out = _empty(batch, desc.n_q_heads, desc.head_dim, dtype=torch.float32, device=q.device, stream=stream)
    if lse is None:
        lse = _empty(batch, desc.n_q_heads, dtype=torch.float32, device=q.device, stream=stream)
    for name, t, n in (("out", out, q.numel()), ("lse", lse, batch * desc.n_q_heads)):
        if _dev(t, name, torch.float32).numel() != n:
            raise ValueError(f"{name} must hold {n} values")
    return batch, out, lse


def lava_paged_decode(desc: LayerDesc, q: torch.Tensor, pool: PagePool, block_table: torch.Tensor, head_rows: torch.Tensor,
                      options: Optional[DecodeOptions] = None, q_pos: Optional[torch.Tensor] = None, out=None, lse=None,
                      workspace=None, stream=None):
    """One new token per sequence, q [batch, H, d_h], attends to the pages of its heads; block_table
    [batch, H_kv, pool.max_blocks], head_rows [batch, H_kv], q_pos [batch] int32.  Returns (out, lse).  Where n_new of the step is zero for some
    sequences, q is q_out.index_select(0, (n_new.cumsum(0) - 1).clamp(min=0)) of lava_rotary_append's."""
    batch, out, lse = _decode_tensors(desc, q, pool, block_table, head_rows, options, q_pos, out, lse, stream)
    if workspace is None:
        workspace = _empty(max(lava_paged_decode_workspace_bytes(desc), 256), dtype=torch.uint8, device=q.device, stream=stream)
    st = lib.lava_paged_decode(ctypes.byref(desc), batch, _ptr(q), pool._ref, _ptr(block_table), _ptr(head_rows),
                               ctypes.byref(options) if options is not None else None, _ptr(q_pos), _ptr(out), _ptr(lse),
                               _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, "lava_paged_decode")
    return out, lse


# ------------------------------------------------------------------------------ sequences that share pages
def lava_beam_step_workspace_bytes(batch: int, beams: int, vocab: int, n_out: int) -> int:
    return int(lib.lava_beam_step_workspace_bytes(int(batch), int(beams), int(vocab), int(n_out)))


def lava_beam_step(logits: torch.Tensor, scores: torch.Tensor, n_out: Optional[int] = None, done: Optional[torch.Tensor] = None,
                   end_token: int = -1, pad_token: int = 0, parents=None, tokens=None, scores_out=None, done_out=None,
                   sources: Optional[torch.Tensor] = None, workspace=None, stream=None):
    """The best n_out (None: as many as there are) continuations of every group of beams: logits [batch, beams, V] float32 or bfloat16 (rows of
    any distance), scores [batch, beams] float32, done [batch, beams] int32 or None.  sources [n_tables, batch * n_out] int32, if given, receives the
    parents for a state that holds n_tables layers as sequences of their own.  Returns (parents, tokens, scores_out, done_out), each
    [batch, n_out]; parents are rows b * beams + i, what lava_page_fork takes where n_out = beams (with another n_out the caller puts them where
    the beams that go on are to be in its state, and -1 elsewhere)."""
    if logits.dtype not in (torch.float32, torch.bfloat16) or not logits.is_cuda or logits.dim() != 3 or (logits.shape[2] > 1 and logits.stride(2) != 1):
        raise ValueError("logits must be a device tensor [batch, beams, V] of float32 or bfloat16 with contiguous rows")
    batch, beams, vocab = logits.shape
    if batch > 1 and beams > 1 and logits.stride(0) != beams * logits.stride(1):
        raise ValueError("the rows of logits must all be the same distance apart")
    stride = logits.stride(1) if beams > 1 else logits.stride(0)
    _here(logits)
    n_out = beams if n_out is None else int(n_out)
    if _dev(scores, "scores", torch.float32).numel() != batch * beams:
        raise ValueError("scores must be [batch, beams]")
    if done is not None and _dev(done, "done", torch.int32).numel() != batch * beams:
        raise ValueError("done must be [batch, beams]")
    new = lambda dtype: _empty(batch, n_out, dtype=dtype, device=logits.device, stream=stream)
    parents = new(torch.int32) if parents is None else parents
    tokens = new(torch.int32) if tokens is None else tokens
    scores_out = new(torch.float32) if scores_out is None else scores_out
    done_out = new(torch.int32) if done_out is None else done_out
    for name, t, dt in (("parents", parents, torch.int32), ("tokens", tokens, torch.int32), ("scores_out", scores_out, torch.float32),
                        ("done_out", done_out, torch.int32)):
        if _dev(t, name, dt).numel() != batch * n_out:
            raise ValueError(f"{name} must be [batch, n_out]")
    n_tables = 0
    if sources is not None:
        n_tables = _dev(sources, "sources", torch.int32).numel() // max(batch * n_out, 1)
        if sources.numel() != n_tables * batch * n_out or n_tables < 1:
            raise ValueError("sources must be [n_tables, batch * n_out]")
    if workspace is None:
        need = lava_beam_step_workspace_bytes(batch, beams, vocab, n_out)
        workspace = _empty(max(need, 256), dtype=torch.uint8, device=logits.device, stream=stream)
    st = lib.lava_beam_step(LAVA_BF16 if logits.dtype == torch.bfloat16 else LAVA_F32, batch, beams, vocab, _ptr(logits), stride, _ptr(scores),
                            _ptr(done), int(end_token), int(pad_token), n_out, _ptr(parents), _ptr(tokens), _ptr(scores_out), _ptr(done_out),
                            _ptr(sources), n_tables, _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, "lava_beam_step")
    return parents, tokens, scores_out, done_out


def lava_page_fork_workspace_bytes(batch: int, n_kv_heads: int, max_blocks: int, n_pages: int) -> int:
    return int(lib.lava_page_fork_workspace_bytes(int(batch), int(n_kv_heads), int(max_blocks), int(n_pages)))


def _change_tensors(desc: LayerDesc, pool: PagePool, state: PageState, block_table_out, free_pages_out, workspace, stream):
    """The checks of a change of a state's sequences.  Returns the workspace."""
    pool._check(desc)
    _here(state.block_table)
    if (state.n_kv_heads, state.max_blocks, state.n_pages, state.page_rows) != (desc.n_kv_heads, pool.max_blocks, *pool.k.shape[:2]):
        raise ValueError("the state's heads, blocks or pages are not those of the descriptor and the pool")
    for name, t, n in (("block_table_out", block_table_out, state.block_table.numel()), ("free_pages_out", free_pages_out, state.n_pages)):
        if t is not None and _dev(t, name, torch.int32).numel() != n:
            raise ValueError(f"{name} must hold {n} values")
    if workspace is None:
        need = lava_page_fork_workspace_bytes(state.batch, state.n_kv_heads, state.max_blocks, state.n_pages)
        workspace = _empty(max(need, 256), dtype=torch.uint8, device=state.block_table.device, stream=stream)
    return workspace


def lava_page_fork(desc: LayerDesc, pool: PagePool, state: PageState, source: torch.Tensor, block_table_out: Optional[torch.Tensor] = None,
                   free_pages_out: Optional[torch.Tensor] = None, workspace=None, stream=None) -> None:
    """Sequence b of the state becomes what sequence source[b] was ([batch] int32; -1: empty); full pages are shared.  In place, or into
    block_table_out / free_pages_out and the state's *_out tensors."""
    workspace = _change_tensors(desc, pool, state, block_table_out, free_pages_out, workspace, stream)
    if _dev(source, "source", torch.int32).numel() != state.batch:
        raise ValueError("source must be [batch]")
    st = lib.lava_page_fork(ctypes.byref(desc), pool._ref, state.batch, state._ref, _ptr(source), _ptr(block_table_out), _ptr(free_pages_out),
                            _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, "lava_page_fork")


def lava_page_compact(desc: LayerDesc, pool: PagePool, state: PageState, head_counts: torch.Tensor, kept_idx: torch.Tensor,
                      evict: Optional[torch.Tensor] = None, block_table_out: Optional[torch.Tensor] = None,
                      free_pages_out: Optional[torch.Tensor] = None, workspace=None, stream=None) -> None:
    """Every head of the sequences with evict[b] != 0 (None: of all) keeps head_counts[b, g] of its rows: kept_idx [batch, capacity] int32, a
    sequence's heads one after another, ascending in each.  In place, or into the outputs as for lava_page_fork."""
    workspace = _change_tensors(desc, pool, state, block_table_out, free_pages_out, workspace, stream)
    if _dev(head_counts, "head_counts", torch.int32).numel() != state.batch * state.n_kv_heads:
        raise ValueError("head_counts must be [batch, H_kv]")
    if _dev(kept_idx, "kept_idx", torch.int32).dim() != 2 or kept_idx.shape[0] != state.batch:
        raise ValueError("kept_idx must be [batch, capacity]")
    if evict is not None and _dev(evict, "evict", torch.int32).numel() != state.batch:
        raise ValueError("evict must be [batch]")
    st = lib.lava_page_compact(ctypes.byref(desc), pool._ref, state.batch, state._ref, _ptr(head_counts), _ptr(kept_idx), kept_idx.shape[1],
                               _ptr(evict), _ptr(block_table_out), _ptr(free_pages_out), _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, "lava_page_compact")


def lava_shared_decode_workspace_bytes(desc: LayerDesc, batch: int, max_blocks: int) -> int:
    return int(lib.lava_shared_decode_workspace_bytes(ctypes.byref(desc), int(batch), int(max_blocks)))


def lava_shared_decode(desc: LayerDesc, q: torch.Tensor, pool: PagePool, block_table: torch.Tensor, head_rows: torch.Tensor,
                       group_start: torch.Tensor, options: Optional[DecodeOptions] = None, q_pos: Optional[torch.Tensor] = None, out=None,
                       lse=None, workspace=None, stream=None):
    """lava_paged_decode for groups of sequences (group i is group_start[i] .. group_start[i + 1] - 1, [n_groups + 1] int32): pages that a group's
    tables begin with alike are read once for all of it.  Returns (out, lse)."""
    batch, out, lse = _decode_tensors(desc, q, pool, block_table, head_rows, options, q_pos, out, lse, stream)
    if _dev(group_start, "group_start", torch.int32).numel() < 2:
        raise ValueError("group_start must be [n_groups + 1]")
    if workspace is None:
        need = lava_shared_decode_workspace_bytes(desc, batch, pool.max_blocks)
        workspace = _empty(max(need, 256), dtype=torch.uint8, device=q.device, stream=stream)
    st = lib.lava_shared_decode(ctypes.byref(desc), batch, _ptr(q), pool._ref, _ptr(block_table), _ptr(head_rows), group_start.numel() - 1,
                                _ptr(group_start), ctypes.byref(options) if options is not None else None, _ptr(q_pos), _ptr(out),
                                _ptr(lse), _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, "lava_shared_decode")
    return out, lse


# ------------------------------------------------------------------------------ timing hook
def prof_enable(on: bool = True) -> None:
    lib.lava_prof_enable(1 if on else 0)


def prof_reset() -> None:
    lib.lava_prof_reset()


def prof_read() -> dict:
    """{kernel name: (total milliseconds, launches)} since the last reset."""
    out = {}
    for i in range(lib.lava_prof_kernel_count()):
        ms, cnt = ctypes.c_double(0.0), ctypes.c_int64(0)
        lib.lava_prof_read(i, ctypes.byref(ms), ctypes.byref(cnt))
        out[lib.lava_prof_kernel_name(i).decode()] = (ms.value, cnt.value)
    return out


def probe_stream(src: torch.Tensor, dst: torch.Tensor, nbytes: int, mode: int, blocks: int = 2048, stream=None):
    """mode 0: copy nbytes from src to dst; mode 1: read nbytes of src."""
    _check(lib.lava_probe_stream(_ptr(src), _ptr(dst), int(nbytes), int(mode), int(blocks), _stream(stream)),
           "lava_probe_stream")


def evict_layer(desc: LayerDesc, n: int, q_win, k, v, budget: int, lse=None, stream=None, primed: bool = True):
    """The calls of one layer in order for one sequence (fixed budget): scores, selection, compaction.
    primed: the scores call prepares the selection's workspace (lava_window_scores_primed +
    lava_select_topk_primed) instead of the plain pair; the results are the same."""
    ws = None
    if primed:
        ws = _empty(max(lava_select_workspace_bytes(desc.n_kv_heads * n), 256), dtype=torch.uint8, device=k.device, stream=stream)
    scores, vbar, stat = lava_window_scores(desc, [n], q_win, k, v, lse=lse, stream=stream, select_workspace=ws)
    counts, offs, idx, kept_s = lava_select_topk(desc.n_kv_heads, scores, budget, stream=stream, workspace=ws,
                                                 primed=primed)
    k_hat, v_hat = lava_compact_kv(desc, n, k, v, offs, idx, budget, stream=stream)
    return dict(scores=scores, vbar=vbar, layer_stat=stat, head_counts=counts, head_offsets=offs,
                kept_idx=idx, kept_scores=kept_s, k_hat=k_hat, v_hat=v_hat)
