"""GB300 tree-verification library: Python binding of libtreeverify.so.

Thin ctypes marshalling over the C ABI declared in include/treeverify.h; the
functions keep the C names.  Every step of the verification pass runs in the
library's CUDA kernels; this module only turns torch tensors into pointers
and sizes.  PyTorch provides device memory and streams.

Importing this module does not require a GPU; calling the compute entry
points does, and a missing library raises immediately (there is no CPU
fallback).
"""
from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
# TB_DEBUG_BOUNDS=1 in the environment selects the debug build of the library,
# whose kernels check their global indices (build.build(debug_bounds=True))
LIB_PATH = os.path.join(_HERE, "libtreeverify_debug.so" if os.environ.get("TB_DEBUG_BOUNDS") == "1"
                        else "libtreeverify.so")

TB_OK, TB_EINVAL, TB_ENOMEM, TB_ECUDA, TB_ENOTFOUND, TB_ECAPACITY, TB_ETIMEOUT, TB_EUNSUPPORTED = (
    0, -1, -2, -3, -4, -5, -6, -7)
TB_MAX_NODES = 64
TB_NO_COMPACT = 1
TB_DEBUG_EXPIRE_WAIT = 1 << 30
RESULT_INTS = 4 + TB_MAX_NODES  # sizeof(tb_result) / 4

API = ("tb_canonicalize", "tb_create", "tb_add_topology", "tb_get_topology", "tb_destroy", "tb_workspace_size",
       "tb_workspace_init", "tb_workspace_status", "tree_attention", "lm_head_stats", "greedy_accept",
       "kv_compact", "verify_step", "verify_step_batched", "lm_head_stats_noalloc", "lm_head_stats_noalloc_status",
       "tb_last_error",
       "tb_schedule_hysteretic_ladder", "tb_schedule_binary", "tb_schedule_threshold_ladder",
       "lm_head_stats_typical", "typical_accept", "verify_step_typical", "verify_step_batched_typical",
       "verify_step_scheduled", "spec_sample_accept", "verify_step_sampled", "tb_debug_bounds_violations",
       "tb_debug_bounds_build", "tb_launch_count", "tb_paged_plan_size", "paged_plan", "paged_kv_store",
       "paged_tree_attention", "logits_process", "tb_logits_workspace_size", "paged_accept", "paged_kv_store_norm",
       "paged_kv_store_q4", "paged_kv_load_q4", "paged_tree_attention_q4", "paged_accept_q4")


class TreeVerifyError(RuntimeError):
    def __init__(self, status: int, where: str, message: str):
        super().__init__(f"{where} failed ({status}): {message}")
        self.status = status


class TbKv(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("layer_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64), ("n_layers", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("L", ctypes.c_int32), ("L_cap", ctypes.c_int32),
                ("rope_theta", ctypes.c_float)]


class TbSeq(ctypes.Structure):
    _fields_ = [("bank_id", ctypes.c_int32), ("reserved", ctypes.c_int32), ("kv", TbKv), ("q", ctypes.c_void_p),
                ("draft_tokens", ctypes.c_void_p), ("attn_out", ctypes.c_void_p), ("result", ctypes.c_void_p)]


class TbTypical(ctypes.Structure):
    _fields_ = [("temperature", ctypes.c_float), ("eps", ctypes.c_float), ("alpha", ctypes.c_float),
                ("reserved", ctypes.c_int32)]


TB_POLICY_HYSTERETIC_LADDER, TB_POLICY_BINARY, TB_POLICY_THRESHOLD_LADDER = 0, 1, 2
TB_FEATURE_TRACE, TB_FEATURE_PATH_VALUE, TB_FEATURE_ENTROPY = 0, 1, 2
STATE_INTS = 8  # sizeof(tb_state) / 4


class TbPolicy(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("feature", ctypes.c_int32), ("n_rungs", ctypes.c_int32),
                ("bank_ids", ctypes.c_int32 * 8), ("a", ctypes.c_float), ("b", ctypes.c_float),
                ("edges", ctypes.c_float * 7), ("trace", ctypes.c_void_p), ("n_trace", ctypes.c_int32),
                ("n_heads", ctypes.c_int32), ("node_stride", ctypes.c_int32)]


TB_MAX_REQUESTS = 4096
TB_BF16, TB_F16, TB_F32 = 0, 1, 2


class TbPages(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("layer_stride", ctypes.c_int64),
                ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("slot_stride", ctypes.c_int64),
                ("n_layers", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class TbPagesQ4(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("layer_stride", ctypes.c_int64),
                ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("n_layers", ctypes.c_int32),
                ("n_pages", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class TbRequests(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("tree", ctypes.c_void_p), ("n_new", ctypes.c_void_p),
                ("lens", ctypes.c_void_p), ("key_begin", ctypes.c_void_p), ("table", ctypes.c_void_p),
                ("row_start", ctypes.c_void_p)]


class TbPagePool(ctypes.Structure):
    _fields_ = [("n_pages", ctypes.c_int32), ("reserved", ctypes.c_int32), ("ring", ctypes.c_void_p),
                ("state", ctypes.c_void_p), ("state_out", ctypes.c_void_p), ("held", ctypes.c_void_p),
                ("held_out", ctypes.c_void_p)]


class TbRope(ctypes.Structure):
    _fields_ = [("theta", ctypes.c_float), ("n_axes", ctypes.c_int32), ("sections", ctypes.c_int32 * 4),
                ("positions", ctypes.c_void_p), ("axis_stride", ctypes.c_int64)]


class TbRows(ctypes.Structure):
    _fields_ = [("ptr", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class TbHeadNorm(ctypes.Structure):
    _fields_ = [("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("eps", ctypes.c_float),
                ("weight_offset", ctypes.c_float)]


class TbLogitRules(ctypes.Structure):
    _fields_ = [("history", ctypes.c_void_p), ("history_stride", ctypes.c_int64), ("history_len", ctypes.c_void_p),
                ("prompt_len", ctypes.c_void_p), ("draft", ctypes.c_void_p), ("repetition", ctypes.c_void_p),
                ("presence", ctypes.c_void_p), ("frequency", ctypes.c_void_p), ("bias_start", ctypes.c_void_p),
                ("bias_token", ctypes.c_void_p), ("bias_value", ctypes.c_void_p), ("mask", ctypes.c_void_p),
                ("mask_stride", ctypes.c_int64), ("mask_row", ctypes.c_void_p), ("mask_rows", ctypes.c_int64),
                ("n_bias", ctypes.c_int64)]


class TbLogitStats(ctypes.Structure):
    _fields_ = [("argmax", ctypes.c_void_p), ("top1", ctypes.c_void_p), ("entropy", ctypes.c_void_p),
                ("logz_t", ctypes.c_void_p), ("entropy_t", ctypes.c_void_p), ("draft_logit", ctypes.c_void_p)]


# the paper's verification settings (temperature, posterior threshold, mixing coefficient)
PAPER_TYPICAL = (0.7, 0.09, 0.3)

TB_MAX_BATCH = 16

_lib = None


def load(path: str = LIB_PATH):
    """Loads libtreeverify.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with paper_2606_27550_gb300.build.build()")
    lib = ctypes.CDLL(path)
    P, i32, i64, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
    sig = {
        "tb_canonicalize": [P, i32, P, P, P, P],
        "tb_create": [P, i32, i32],
        "tb_add_topology": [P, P, i32, P, P],
        "tb_get_topology": [P, i32, P, P, P, P],
        "tb_destroy": [P],
        "tb_workspace_size": [i32, i32, i32, i32, i32, i32, i32],
        "tb_workspace_init": [P, sz, P],
        "tb_workspace_status": [P, P],
        "tree_attention": [P, i32, P, i32, i32, P, i32, P, P, sz, P],
        "lm_head_stats": [P, i32, P, i32, i32, P, P, P, P, sz, P],
        "greedy_accept": [P, i32, P, P, i32, i32, P, P],
        "kv_compact": [P, P, P, P],
        "verify_step": [P, i32, P, P, i32, P, P, i32, i32, P, P, P, P, P, P, P, sz, i32, P],
        "lm_head_stats_noalloc": [P, i32, P, i32, i32, P, P, P, i32, P],
        "lm_head_stats_noalloc_status": [P, P],
        "tb_debug_bounds_violations": [P],
        "tb_debug_bounds_build": [],
        "tb_launch_count": [P],
        "verify_step_batched": [P, i32, P, i32, P, P, i32, i32, P, P, P, P, sz, i32, P],
        "tb_last_error": [],
        "lm_head_stats_typical": [P, i32, P, P, i32, i32, ctypes.c_float, P, P, P, P, P, P, P, P, sz, P],
        "typical_accept": [P, i32, P, P, P, P, P, i32, i32, P, P, P],
        "verify_step_typical": [P, i32, P, P, i32, P, P, i32, i32, P, P, P, P, P, P, P, P, sz, i32, P],
        "verify_step_batched_typical": [P, i32, P, i32, P, P, i32, i32, P, P, P, P, P, sz, i32, P],
        "verify_step_scheduled": [P, P, P, P, P, i32, P, P, i32, i32, P, P, P, P, P, P, P, sz, i32, P],
        "spec_sample_accept": [P, i32, P, P, P, P, P, i32, i32, ctypes.c_float, P, P, P],
        "verify_step_sampled": [P, i32, P, P, i32, P, P, i32, i32, P, P, P, ctypes.c_float, P, P, P, P, P, P, P, sz,
                                i32, P],
        "tb_paged_plan_size": [i32, i32],
        "paged_plan": [P, P, P, P, P, i32, P, i32, i32, i32, i32, P, sz, P],
        "paged_kv_store": [P, i32, P, i32, P, P, P, P, i32, P, P],
        "paged_tree_attention": [P, P, P, i32, P, sz, P, i32, i32, ctypes.c_float, ctypes.c_float, P, P, P, P, sz, P],
        "tb_logits_workspace_size": [i32, i32, i32],
        "logits_process": [P, P, P, i32, i64, i32, i32, P, ctypes.c_float, P, i64, P, P, sz, P],
        "paged_accept": [P, P, P, P, P, i32, i32, P, P, P],
        "paged_kv_store_norm": [P, i32, P, i32, P, P, P, P, i32, P, P, P],
        "paged_kv_store_q4": [P, i32, P, i32, P, P, P, P, i32, P, P, P],
        "paged_kv_load_q4": [P, i32, i32, P, i32, P, P, i64, P],
        "paged_tree_attention_q4": [P, P, P, i32, P, sz, P, i32, i32, ctypes.c_float, ctypes.c_float, P, P, P, P, sz, P],
        "paged_accept_q4": [P, P, P, P, P, i32, i32, P, P, P],
    }
    for name, args in sig.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = ctypes.c_int
    d = ctypes.c_double
    lib.tb_schedule_hysteretic_ladder.argtypes = [i32, i32, d, d, d]
    lib.tb_schedule_binary.argtypes = [i32, d, d, d]
    lib.tb_schedule_threshold_ladder.argtypes = [d, P, i32]
    for f in (lib.tb_schedule_hysteretic_ladder, lib.tb_schedule_binary, lib.tb_schedule_threshold_ladder):
        f.restype = ctypes.c_int
    for f in (lib.tb_workspace_size, lib.tb_paged_plan_size, lib.tb_logits_workspace_size):
        f.restype = ctypes.c_size_t
    lib.tb_last_error.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _check(rc: int, where: str):
    if rc:
        raise TreeVerifyError(rc, where, load().tb_last_error().decode())


def _ptr(t) -> int | None:
    try:
        return t.data_ptr()  # a tensor, on every call's path: no checks first
    except AttributeError:
        return None if t is None else t.ctypes.data


_current_stream = None


def _find_current_stream():
    """A function that returns the raw handle of torch's current stream: torch's
    own raw getter where it has one (a Stream object per call costs 1 us)."""
    import torch

    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    device = getattr(torch._C, "_cuda_getDevice", None)
    if raw is None or device is None or not torch.cuda.is_initialized():
        return lambda: torch.cuda.current_stream().cuda_stream
    return lambda: raw(device())


def _stream(stream) -> int | None:
    if stream is None:
        global _current_stream
        if _current_stream is None:
            import torch

            torch.cuda.current_stream()  # initialises CUDA, as the getter expects
            _current_stream = _find_current_stream()
        return _current_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


# --------------------------------------------------------------------- topologies


def tb_canonicalize(parent):
    """(order, bfs_parent, depth, anc) of a parent array (pure host)."""
    parent = np.ascontiguousarray(parent, dtype=np.int32)
    n = len(parent)
    order = np.zeros(n, np.int32)
    bp = np.zeros(n, np.int32)
    depth = np.zeros(n, np.int32)
    anc = np.zeros(n, np.uint64)
    _check(load().tb_canonicalize(_ptr(parent), n, _ptr(order), _ptr(bp), _ptr(depth), _ptr(anc)), "tb_canonicalize")
    return order, bp, depth, anc


class Bank:
    """A TopologyBank on one device (tb_create / tb_add_topology / tb_destroy)."""

    def __init__(self, max_topologies: int = 64, device: int = 0):
        h = ctypes.c_void_p()
        _check(load().tb_create(ctypes.byref(h), max_topologies, device), "tb_create")
        self.handle = h
        self.device = device
        self.sizes: list[int] = []

    def add(self, parent):
        """Adds a topology; returns (bank_id, order) with order[canonical] = caller index."""
        parent = np.ascontiguousarray(parent, dtype=np.int32)
        out = ctypes.c_int()
        order = np.zeros(len(parent), np.int32)
        _check(load().tb_add_topology(self.handle, _ptr(parent), len(parent), ctypes.byref(out), _ptr(order)),
               "tb_add_topology")
        self.sizes.append(len(parent))
        return out.value, order

    def get(self, bank_id: int):
        n = ctypes.c_int()
        parent = np.zeros(TB_MAX_NODES, np.int32)
        depth = np.zeros(TB_MAX_NODES, np.int32)
        anc = np.zeros(TB_MAX_NODES, np.uint64)
        _check(load().tb_get_topology(self.handle, bank_id, ctypes.byref(n), _ptr(parent), _ptr(depth), _ptr(anc)),
               "tb_get_topology")
        k = n.value
        return parent[:k].copy(), depth[:k].copy(), anc[:k].copy()

    def n_nodes(self, bank_id: int) -> int:
        return self.sizes[bank_id]

    def close(self):
        if self.handle:
            _check(load().tb_destroy(self.handle), "tb_destroy")
            self.handle = None

    def __del__(self):  # pragma: no cover
        try:
            self.close()
        except Exception:
            pass


# --------------------------------------------------------------------- KV cache, workspace, result


@dataclass
class KvCache:
    """bf16 K and V caches shaped [n_layers][n_kv_heads][L_cap][head_dim]."""

    k: object
    v: object
    L: int
    rope_theta: float = 0.0  # > 0: the call rotary-embeds q and the tree keys at L + depth

    def as_c(self) -> TbKv:
        k = self.k
        n_layers, n_kv_heads, L_cap, head_dim = k.shape
        s = k.stride()
        return TbKv(k.data_ptr(), self.v.data_ptr(), s[0], s[1], n_layers, n_kv_heads, head_dim, self.L, L_cap,
                    float(self.rope_theta))


def tb_workspace_size(max_rows: int, n_layers: int, n_kv_heads: int, n_q_heads: int, head_dim: int, vocab: int,
                      device: int = -1) -> int:
    return int(load().tb_workspace_size(max_rows, n_layers, n_kv_heads, n_q_heads, head_dim, vocab, device))


def make_workspace(nbytes: int, device="cuda"):
    """Zero-filled device workspace (torch uint8)."""
    import torch

    return torch.zeros(nbytes, dtype=torch.uint8, device=device)


def tb_workspace_init(ws, stream=None):
    _check(load().tb_workspace_init(_ptr(ws), ws.numel(), _stream(stream)), "tb_workspace_init")


def tb_workspace_status(ws) -> int:
    st = ctypes.c_int32()
    _check(load().tb_workspace_status(_ptr(ws), ctypes.byref(st)), "tb_workspace_status")
    return st.value


def make_result(device="cuda"):
    """Device buffer for one tb_result (int32[68])."""
    import torch

    return torch.zeros(RESULT_INTS, dtype=torch.int32, device=device)


def parse_result(res) -> dict:
    """The tb_result block (a device or host tensor, or a sequence of ints) as a dict."""
    if hasattr(res, "cpu"):
        r = res.cpu().tolist()  # one copy and one conversion (iterating a tensor makes a tensor per element)
    else:
        r = [int(x) for x in res]
    k = r[0]
    return {"accept_len": k, "bonus_token": r[1], "new_L": r[2], "status": r[3], "path": r[4:4 + k]}


# --------------------------------------------------------------------- the pass


def tree_attention(bank: Bank, bank_id: int, kv: KvCache, q, out, ws, layer_begin: int = 0, n_layers: int | None = None,
                   stream=None):
    """q, out: bf16 [n_layers][N][n_q_heads][head_dim]."""
    c = kv.as_c()
    nl = c.n_layers - layer_begin if n_layers is None else n_layers
    _check(load().tree_attention(bank.handle, bank_id, ctypes.byref(c), layer_begin, nl, _ptr(q), q.shape[2],
                                 _ptr(out), _ptr(ws), ws.numel(), _stream(stream)), "tree_attention")


def lm_head_stats(hidden, lm_head, argmax, top1, entropy, ws, stream=None):
    """hidden bf16 [R][d_model]; lm_head bf16 [V][d_model]; outputs [R]."""
    R, D = hidden.shape
    _check(load().lm_head_stats(_ptr(hidden), R, _ptr(lm_head), D, lm_head.shape[0], _ptr(argmax), _ptr(top1),
                                _ptr(entropy), _ptr(ws), ws.numel(), _stream(stream)), "lm_head_stats")


def greedy_accept(bank: Bank, bank_id: int, draft, argmax, vocab: int, L: int, result, stream=None):
    _check(load().greedy_accept(bank.handle, bank_id, _ptr(draft), _ptr(argmax), vocab, L, _ptr(result),
                                _stream(stream)), "greedy_accept")


def kv_compact_path(kv: KvCache, path, accept_len, stream=None):
    """KV-cache update from a device path (int32 [accept_len]) and a device
    accept_len (int32 [1])."""
    c = kv.as_c()
    _check(load().kv_compact(ctypes.byref(c), _ptr(path), _ptr(accept_len), _stream(stream)), "kv_compact")


def kv_compact(kv: KvCache, result, stream=None):
    """KV-cache update from a device result block (greedy_accept's): its path
    and accept_len fields."""
    kv_compact_path(kv, result[4:], result[:1], stream)


def verify_step(bank: Bank, bank_id: int, kv: KvCache, q, hidden, lm_head, draft, attn_out, argmax, top1, entropy,
                result, ws, flags: int = 0, stream=None):
    c = kv.as_c()
    _check(load().verify_step(bank.handle, bank_id, ctypes.byref(c), _ptr(q), q.shape[2], _ptr(hidden),
                              _ptr(lm_head), hidden.shape[1], lm_head.shape[0], _ptr(draft), _ptr(attn_out),
                              _ptr(argmax), _ptr(top1), _ptr(entropy), _ptr(result), _ptr(ws), ws.numel(), flags,
                              _stream(stream)), "verify_step")


def lm_head_stats_noalloc(hidden, lm_head, argmax, top1, entropy, flags: int = 0, stream=None):
    """lm_head_stats with the library's built-in scratch array instead of a
    caller workspace, for callers that cannot allocate device memory."""
    R, D = hidden.shape
    _check(load().lm_head_stats_noalloc(_ptr(hidden), R, _ptr(lm_head), D, lm_head.shape[0], _ptr(argmax),
                                        _ptr(top1), _ptr(entropy), flags, _stream(stream)), "lm_head_stats_noalloc")


def tb_debug_bounds_violations() -> int:
    """Failed index checks of the debug build's kernels since the last call
    (0 in a normal build); synchronises the device."""
    n = ctypes.c_uint32(0)
    _check(load().tb_debug_bounds_violations(ctypes.byref(n)), "tb_debug_bounds_violations")
    return int(n.value)


def tb_debug_bounds_build() -> bool:
    return bool(load().tb_debug_bounds_build())


def tb_launch_count() -> int:
    """Kernels the library has enqueued in this process (host-side count; a
    CUDA graph's replays are not counted again)."""
    n = ctypes.c_uint64(0)
    _check(load().tb_launch_count(ctypes.byref(n)), "tb_launch_count")
    return int(n.value)


def lm_head_stats_noalloc_status(stream=None) -> int:
    """Device-detected status (TB_OK or TB_ETIMEOUT) of the last
    lm_head_stats_noalloc call on `stream`; waits for the stream."""
    st = ctypes.c_int32(0)
    _check(load().lm_head_stats_noalloc_status(ctypes.byref(st), _stream(stream)), "lm_head_stats_noalloc_status")
    return st.value


@dataclass
class Seq:
    """One sequence of verify_step_batched."""

    bank_id: int
    kv: KvCache
    q: object
    draft_tokens: object
    attn_out: object
    result: object

    def as_c(self) -> TbSeq:
        return TbSeq(self.bank_id, 0, self.kv.as_c(), _ptr(self.q), _ptr(self.draft_tokens), _ptr(self.attn_out),
                     _ptr(self.result))


def verify_step_batched(bank: Bank, seqs, hidden, lm_head, argmax, top1, entropy, ws, flags: int = 0, stream=None):
    """hidden bf16 [sum N_b][d_model] (sequence 0 first); argmax/top1/entropy [sum N_b]."""
    arr = (TbSeq * len(seqs))(*[s.as_c() for s in seqs])
    _check(load().verify_step_batched(bank.handle, len(seqs), arr, seqs[0].q.shape[2], _ptr(hidden), _ptr(lm_head),
                                      hidden.shape[1], lm_head.shape[0], _ptr(argmax), _ptr(top1), _ptr(entropy),
                                      _ptr(ws), ws.numel(), flags, _stream(stream)), "verify_step_batched")


# --------------------------------------------------------------------- typical acceptance


def _typical(temperature: float, eps: float, alpha: float) -> TbTypical:
    return TbTypical(float(temperature), float(eps), float(alpha), 0)


def lm_head_stats_typical(bank: Bank, bank_id: int, hidden, lm_head, temperature: float, draft, argmax, top1, entropy,
                          logz_t, entropy_t, draft_logit, ws, stream=None):
    """hidden bf16 [N][d_model] (the tree's rows); every output [N]."""
    _check(load().lm_head_stats_typical(bank.handle, bank_id, _ptr(hidden), _ptr(lm_head), hidden.shape[1],
                                        lm_head.shape[0], float(temperature), _ptr(draft), _ptr(argmax), _ptr(top1),
                                        _ptr(entropy), _ptr(logz_t), _ptr(entropy_t), _ptr(draft_logit), _ptr(ws),
                                        ws.numel(), _stream(stream)), "lm_head_stats_typical")


def typical_accept(bank: Bank, bank_id: int, draft, argmax, logz_t, entropy_t, draft_logit, vocab: int, L: int,
                   result, temperature: float, eps: float, alpha: float, stream=None):
    t = _typical(temperature, eps, alpha)
    _check(load().typical_accept(bank.handle, bank_id, _ptr(draft), _ptr(argmax), _ptr(logz_t), _ptr(entropy_t),
                                 _ptr(draft_logit), vocab, L, ctypes.byref(t), _ptr(result), _stream(stream)),
           "typical_accept")


def verify_step_typical(bank: Bank, bank_id: int, kv: KvCache, q, hidden, lm_head, draft, attn_out, argmax, top1,
                        entropy, result, ws, temperature: float, eps: float, alpha: float, flags: int = 0,
                        stream=None):
    c = kv.as_c()
    t = _typical(temperature, eps, alpha)
    _check(load().verify_step_typical(bank.handle, bank_id, ctypes.byref(c), _ptr(q), q.shape[2], _ptr(hidden),
                                      _ptr(lm_head), hidden.shape[1], lm_head.shape[0], _ptr(draft), _ptr(attn_out),
                                      _ptr(argmax), _ptr(top1), _ptr(entropy), ctypes.byref(t), _ptr(result),
                                      _ptr(ws), ws.numel(), flags, _stream(stream)), "verify_step_typical")


def verify_step_batched_typical(bank: Bank, seqs, hidden, lm_head, argmax, top1, entropy, ws, temperature: float,
                                eps: float, alpha: float, flags: int = 0, stream=None):
    arr = (TbSeq * len(seqs))(*[s.as_c() for s in seqs])
    t = _typical(temperature, eps, alpha)
    _check(load().verify_step_batched_typical(bank.handle, len(seqs), arr, seqs[0].q.shape[2], _ptr(hidden),
                                              _ptr(lm_head), hidden.shape[1], lm_head.shape[0], _ptr(argmax),
                                              _ptr(top1), _ptr(entropy), ctypes.byref(t), _ptr(ws), ws.numel(),
                                              flags, _stream(stream)), "verify_step_batched_typical")


# --------------------------------------------------------------------- speculative sampling


def spec_sample_accept(bank: Bank, bank_id: int, draft, logits, logz_t, draft_probs, uniforms, L: int,
                       temperature: float, scratch, result, stream=None):
    """logits, draft_probs float [N][V]; logz_t [N]; uniforms [2N]; scratch [V]."""
    _check(load().spec_sample_accept(bank.handle, bank_id, _ptr(draft), _ptr(logits), _ptr(logz_t),
                                     _ptr(draft_probs), _ptr(uniforms), logits.shape[1], L, float(temperature),
                                     _ptr(scratch), _ptr(result), _stream(stream)), "spec_sample_accept")


def verify_step_sampled(bank: Bank, bank_id: int, kv: KvCache, q, hidden, lm_head, draft, draft_probs, uniforms,
                        temperature: float, attn_out, argmax, top1, entropy, logits, result, ws, flags: int = 0,
                        stream=None):
    """logits: float [N + 1][V] scratch (rows 0..N-1 receive the target logits)."""
    c = kv.as_c()
    _check(load().verify_step_sampled(bank.handle, bank_id, ctypes.byref(c), _ptr(q), q.shape[2], _ptr(hidden),
                                      _ptr(lm_head), hidden.shape[1], lm_head.shape[0], _ptr(draft),
                                      _ptr(draft_probs), _ptr(uniforms), float(temperature), _ptr(attn_out),
                                      _ptr(argmax), _ptr(top1), _ptr(entropy), _ptr(logits), _ptr(result), _ptr(ws),
                                      ws.numel(), flags, _stream(stream)), "verify_step_sampled")


# --------------------------------------------------------------------- device-driven loop


def make_policy(kind: int, feature: int, bank_ids, a: float = 0.0, b: float = 0.0, edges=(), trace=None,
                n_heads: int = 0, node_stride: int = 0) -> TbPolicy:
    """tb_policy; `trace` is a device float tensor, which the returned policy
    keeps alive (the library holds only its address)."""
    pol = TbPolicy()
    pol.kind, pol.feature, pol.n_rungs = kind, feature, len(bank_ids)
    for i, x in enumerate(bank_ids):
        pol.bank_ids[i] = int(x)
    pol.a, pol.b = float(a), float(b)
    for i, x in enumerate(edges):
        pol.edges[i] = float(x)
    if trace is not None:
        pol.trace = _ptr(trace)
        pol._trace_ref = trace
        pol.n_trace = trace.numel() // max(1, n_heads) if feature == TB_FEATURE_PATH_VALUE else trace.numel()
    pol.n_heads = n_heads
    pol.node_stride = node_stride
    return pol


def make_state(rung: int, L: int, device="cuda"):
    """A device tb_state (int32 words) at the given rung and prefix length."""
    import torch

    t = torch.zeros(STATE_INTS, dtype=torch.int32)
    t[0], t[1] = rung, L
    return t.to(device)


def parse_state(st) -> dict:
    import numpy as np

    h = st.cpu().numpy()
    return {"rung": int(h[0]), "L": int(h[1]), "step": int(h[2]), "feature": float(h[3:4].view(np.float32)[0]),
            "accept_len": int(h[4])}


def verify_step_scheduled(bank: Bank, policy: TbPolicy, state, kv: KvCache, q, hidden, lm_head, drafts, attn_out,
                          argmax, top1, entropy, result, ws, flags: int = 0, stream=None):
    """q / attn_out [n_layers][N_max][Hq][head_dim]; hidden [N_max][d_model]; drafts [n_rungs][N_max]."""
    c = kv.as_c()
    _check(load().verify_step_scheduled(bank.handle, ctypes.byref(policy), _ptr(state), ctypes.byref(c), _ptr(q),
                                        q.shape[2], _ptr(hidden), _ptr(lm_head), hidden.shape[1], lm_head.shape[0],
                                        _ptr(drafts), _ptr(attn_out), _ptr(argmax), _ptr(top1), _ptr(entropy),
                                        _ptr(result), _ptr(ws), ws.numel(), flags, _stream(stream)),
           "verify_step_scheduled")


# --------------------------------------------------------------------- serving over a paged cache


_I32 = _I64 = _F32 = _KINDS = None  # torch's types and the C ABI's numbers for element types


def _torch_types():
    global _I32, _I64, _F32, _KINDS
    import torch

    _I32, _I64, _F32 = torch.int32, torch.int64, torch.float32
    _KINDS = {torch.bfloat16: TB_BF16, torch.float16: TB_F16, torch.float32: TB_F32}


def _bad_array(t, kind, n: int, what: str):
    if t.dtype is not kind:
        raise TypeError(f"{what}: {t.dtype}, {kind} expected")
    raise ValueError(f"{what}: shape {tuple(t.shape)}, {n} contiguous entries expected")


def _arr(t, kind, n: int, what: str) -> int | None:
    """The address of an array of at least n contiguous entries of the type that the call reads it as."""
    if t is None:
        return None
    if t.dtype is not kind or t.numel() < n or not t.is_contiguous():
        _bad_array(t, kind, n, what)
    return t.data_ptr()


class Pages:
    """The paged cache: k and v shaped [n_layers][n_pages][n_kv_heads][page_size][head_dim],
    views of any strides (multiples of 8, elements of a row contiguous), the same for both.
    Which tensors they are is fixed; what they hold is read and written by every call."""

    __slots__ = ("_k", "_v", "_c", "dtype")
    k = property(lambda self: self._k)
    v = property(lambda self: self._v)

    def __init__(self, k, v):
        s, shape, dtype = k.stride(), k.shape, k.dtype
        if len(s) != 5 or s[4] != 1 or v.stride() != s or v.shape != shape or v.dtype is not dtype:
            raise ValueError("pages: k and v of one 5-D shape, type and strides, rows contiguous")
        if _KINDS is None:
            _torch_types()
        kind = _KINDS.get(dtype, TB_F32)
        if kind == TB_F32:
            raise TypeError(f"pages: {dtype}, bfloat16 or float16 expected")
        self._k, self._v, self.dtype = k, v, dtype
        self._c = TbPages(k.data_ptr(), v.data_ptr(), *s[:4], *shape, kind)

    def as_c(self) -> TbPages:
        return self._c


@dataclass(frozen=True)
class Requests:
    """A batch of request slots (device int32 tensors): lens [B], table [B][max_pages],
    row_start [B + 1], and tree [B] (bank ids, -1 for none) or n_new [B]; key_begin [B] or None.
    Which tensors they are is fixed; what they hold is read by every call."""

    row_start: object
    tree: object = None
    lens: object = None
    table: object = None
    page_size: int = 16
    n_new: object = None
    key_begin: object = None

    def __post_init__(self):
        if _I32 is None:
            _torch_types()
        B = self.row_start.shape[0] - 1
        width = 0 if self.table is None else self.table.shape[1]
        c = TbRequests(B, width, self.page_size, 0, _arr(self.tree, _I32, B, "tree"), _arr(self.n_new, _I32, B, "n_new"),
                       _arr(self.lens, _I32, B, "lens"), _arr(self.key_begin, _I32, B, "key_begin"),
                       _arr(self.table, _I32, B * width, "table"), _arr(self.row_start, _I32, B + 1, "row_start"))
        object.__setattr__(self, "_c", c)

    def as_c(self) -> TbRequests:
        return self._c


@dataclass
class PagePool:
    """The free pages (device int32 tensors): ring [n_pages], state [2] = (first, free), held [B];
    state_out / held_out receive the new values (None: in place).  ring and state None: no page
    changes hands (see held_only)."""

    ring: object
    state: object
    held: object
    state_out: object = None
    held_out: object = None

    def held_only(self) -> PagePool:
        """The pool for the further plans of a step: what the first one left with every request.  They
        refuse what the first refused, and write the same rows."""
        return PagePool(None, None, self.held if self.held_out is None else self.held_out)

    def as_c(self, batch: int) -> TbPagePool:
        state = _arr(self.state, _I32, 2, "state")
        held = _arr(self.held, _I32, batch, "held")
        if self.ring is None:
            return TbPagePool(0, 0, None, state, _arr(self.state_out, _I32, 2, "state_out"), held,
                              _arr(self.held_out, _I32, batch, "held_out"))
        n = self.ring.numel()
        return TbPagePool(n, 0, _arr(self.ring, _I32, n, "ring"), state,
                          state if self.state_out is None else _arr(self.state_out, _I32, 2, "state_out"), held,
                          held if self.held_out is None else _arr(self.held_out, _I32, batch, "held_out"))


def make_page_pool(n_pages: int, batch: int, device="cuda") -> PagePool:
    """A pool whose pages 0 .. n_pages - 1 are all free."""
    import torch

    return PagePool(torch.arange(n_pages, dtype=torch.int32, device=device),
                    torch.tensor([0, n_pages], dtype=torch.int32, device=device),
                    torch.zeros(batch, dtype=torch.int32, device=device))


def tb_paged_plan_size(batch: int, device: int = -1) -> int:
    return int(load().tb_paged_plan_size(batch, device))


def make_paged_plan(batch: int, device="cuda"):
    """Zero-filled device memory for the plan of a batch (torch uint8)."""
    return make_workspace(tb_paged_plan_size(batch), device)


def _ref(c):
    return None if c is None else ctypes.byref(c)


def paged_plan(bank, req: Requests, slots, positions, status, plan, pool: PagePool | None = None, n_q_heads: int = 0,
               n_kv_heads: int = 1, window: int = 0, sink: int = 0, stream=None):
    """slots int64, positions int32 [max_rows]; status int32 [B]; bank may be None with n_new."""
    r = req._c
    c = None if pool is None else pool.as_c(r.batch)
    rows = slots.shape[0]
    rc = load().paged_plan(None if bank is None else bank.handle, ctypes.byref(r), _ref(c),
                           _arr(slots, _I64, rows, "slots"), _arr(positions, _I32, rows, "positions"), rows,
                           _arr(status, _I32, r.batch, "status"), n_q_heads, n_kv_heads, window, sink, plan.data_ptr(),
                           plan.numel(), _stream(stream))
    if rc:
        _check(rc, "paged_plan")


# The operands of the stores and the load as the bytes of their C structs (TbRows, TbRope, TbHeadNorm), which ctypes
# passes by address: building a Structure and a reference to it costs two to three times as much.
_ROWS, _ROPE, _NORM = (struct.Struct(f).pack for f in ("=Qqq", "=fi4iQq", "=QQff"))


def _rows_of(t, rows: int, heads: int, d: int, dtype, what: str, dims: int = 3) -> bytes:
    """The TbRows of a (rows, heads, d) tensor, or with dims 4 of the first layer of a (layers, rows, heads, d) one."""
    shape, s = t.shape, t.stride()
    if dims == 4:
        shape, s = shape[1:], s[1:]
    if len(s) != 3 or s[2] != 1 or shape[0] < rows or shape[1] != heads or shape[2] != d:
        raise ValueError(f"{what}: shape {tuple(shape)}, ({rows}, {heads}, {d}) expected, rows contiguous")
    if t.dtype is not dtype:
        raise TypeError(f"{what}: {t.dtype}, the pages' {dtype} expected")
    return _ROWS(t.data_ptr(), s[0], s[1])


def _queries_and_rope(q, q_out, rows: int, d: int, dtype, positions, sections, rope_theta: float):
    """(heads, q, q_out, rope) of a store's arguments, None for what is not there."""
    heads, cq, co, rope = 0, None, None, None
    if q is not None:
        heads = q.shape[1]
        cq = _rows_of(q, rows, heads, d, dtype, "q")
        co = cq if q_out is None else _rows_of(q_out, rows, heads, d, dtype, "q_out")
    if rope_theta:
        sections = (d // 2,) if sections is None else sections
        axes, stride = len(sections), positions.shape[-1]
        if axes > 4:
            raise ValueError(f"{axes} position axes: at most 4")
        if stride < rows:
            raise ValueError(f"positions: {stride} of {rows} rows")
        address = _arr(positions, _I32, axes * stride, "positions")
        try:
            rope = _ROPE(rope_theta, axes, *(*sections, 0, 0, 0, 0)[:4], address, stride)
        except (OverflowError, struct.error):  # past 32 bits: as C takes it (a theta is infinite), for the library to refuse
            rope = bytes(TbRope(rope_theta, axes, (*sections,), address, stride))
    return heads, cq, co, rope


def paged_kv_store(pages: Pages, slots, k, v, layer: int = 0, q=None, q_out=None, positions=None, sections=None,
                   rope_theta: float = 0.0, stream=None):
    """k, v [rows][n_kv_heads][head_dim] and q, q_out [rows][n_q_heads][head_dim] (views of any row
    and head strides); positions int32 [rows] or [axes][rows]; sections: pairs per axis (None: one axis)."""
    c, dtype = _page_kind(pages, Pages), pages.dtype
    rows, H, d = slots.shape[0], c.n_kv_heads, c.head_dim
    ck, cv = _rows_of(k, rows, H, d, dtype, "k"), _rows_of(v, rows, H, d, dtype, "v")
    heads, cq, co, rope = _queries_and_rope(q, q_out, rows, d, dtype, positions, sections, rope_theta)
    rc = load().paged_kv_store(ctypes.byref(c), layer, _arr(slots, _I64, rows, "slots"), rows, ck, cv, cq, co, heads,
                               rope, _stream(stream))
    if rc:
        _check(rc, "paged_kv_store")


def _norm_of(q_norm, k_norm, eps: float, weight_offset: float, d: int, dtype):
    if q_norm is None and k_norm is None:
        return None
    weights = _arr(q_norm, dtype, d, "q_norm") or 0, _arr(k_norm, dtype, d, "k_norm") or 0
    try:
        return _NORM(*weights, eps, weight_offset)
    except OverflowError:
        return bytes(TbHeadNorm(*weights, eps, weight_offset))


def _page_kind(pages, kind):
    """The C struct of pages, which has to be of the kind that the call reads it as (whatever class holds it)."""
    c = getattr(pages, "_c", None)
    if c is None or isinstance(c, TbPagesQ4) is not (kind is PagesQ4):
        raise TypeError(f"pages: {type(pages).__name__}, {kind.__name__} expected")
    return c


def _store_rows(name: str, kind, pages, layer: int, slots, k, v, q, q_out, q_norm, k_norm, eps, weight_offset,
                positions, sections, rope_theta, stream):
    c, dtype = _page_kind(pages, kind), pages.dtype
    rows, H, d = slots.shape[0], c.n_kv_heads, c.head_dim
    ck, cv = _rows_of(k, rows, H, d, dtype, "k"), _rows_of(v, rows, H, d, dtype, "v")
    heads, cq, co, rope = _queries_and_rope(q, q_out, rows, d, dtype, positions, sections, rope_theta)
    norm = _norm_of(q_norm, k_norm, eps, weight_offset, d, dtype)
    rc = getattr(load(), name)(ctypes.byref(c), layer, _arr(slots, _I64, rows, "slots"), rows, ck, cv, cq, co, heads,
                               norm, rope, _stream(stream))
    if rc:
        _check(rc, name)


def paged_kv_store_norm(pages: Pages, slots, k, v, layer: int = 0, q=None, q_out=None, q_norm=None, k_norm=None,
                        eps: float = 1e-6, weight_offset: float = 0.0, positions=None, sections=None,
                        rope_theta: float = 0.0, stream=None):
    """paged_kv_store with norms of the heads before the rotation: q_norm, k_norm [head_dim] of the pages'
    type, None where that operand is left as it is."""
    _store_rows("paged_kv_store_norm", Pages, pages, layer, slots, k, v, q, q_out, q_norm, k_norm, eps,
                weight_offset, positions, sections, rope_theta, stream)


class PagesQ4:
    """The paged cache in 4 bits: k and v uint8 [n_layers][n_pages][n_kv_heads][q4_page_bytes], views of any strides
    (multiples of 16, a page's bytes contiguous), the same for both; dtype: the type of the rows that go in and out.
    Which tensors they are is fixed; what they hold is read and written by every call."""

    __slots__ = ("_k", "_v", "_c", "dtype")
    k = property(lambda self: self._k)
    v = property(lambda self: self._v)

    def __init__(self, k, v, page_size: int, head_dim: int, dtype):
        import torch

        s, shape = k.stride(), k.shape
        n = q4_page_bytes(page_size, head_dim)
        if len(s) != 4 or s[3] != 1 or shape[3] != n or v.stride() != s or v.shape != shape:
            raise ValueError(f"4-bit pages: k and v of one 4-D shape and strides, {n} contiguous bytes per page and head")
        if k.dtype is not torch.uint8 or v.dtype is not torch.uint8:
            raise TypeError(f"4-bit pages: {k.dtype}, {v.dtype}, uint8 expected")
        if _KINDS is None:
            _torch_types()
        kind = _KINDS.get(dtype, TB_F32)
        if kind == TB_F32:
            raise TypeError(f"4-bit pages: rows of {dtype}, bfloat16 or float16 expected")
        self._k, self._v, self.dtype = k, v, dtype
        self._c = TbPagesQ4(k.data_ptr(), v.data_ptr(), *s[:3], *shape[:3], page_size, head_dim, kind)

    def as_c(self) -> TbPagesQ4:
        return self._c


def q4_page_bytes(page_size: int, head_dim: int) -> int:
    """Bytes of one head's block of a 4-bit page: codes, then a scale byte per 32 elements."""
    return page_size * (head_dim // 2 + head_dim // 32)


def make_pages_q4(n_layers: int, n_pages: int, n_kv_heads: int, page_size: int, head_dim: int, dtype,
                  device="cuda") -> PagesQ4:
    """Zero-filled 4-bit pages (every element 0)."""
    import torch

    shape = (n_layers, n_pages, n_kv_heads, q4_page_bytes(page_size, head_dim))
    return PagesQ4(*(torch.zeros(shape, dtype=torch.uint8, device=device) for _ in range(2)), page_size, head_dim, dtype)


def paged_kv_store_q4(pages: PagesQ4, slots, k, v, layer: int = 0, q=None, q_out=None, q_norm=None, k_norm=None,
                      eps: float = 1e-6, weight_offset: float = 0.0, positions=None, sections=None,
                      rope_theta: float = 0.0, stream=None):
    """paged_kv_store_norm into 4-bit pages; the operands have the pages' row type."""
    _store_rows("paged_kv_store_q4", PagesQ4, pages, layer, slots, k, v, q, q_out, q_norm, k_norm, eps,
                weight_offset, positions, sections, rope_theta, stream)


def paged_kv_load_q4(pages: PagesQ4, slots, k, v, layer: int = 0, stream=None):
    """Rows of 4-bit pages in 16 bits: k, v [rows][n_kv_heads][head_dim] of one layer, or [n_layers][rows][n_kv_heads]
    [head_dim] of `layer` and the ones behind it (views of any layer, row and head strides, the same layer stride)."""
    c, dtype = _page_kind(pages, PagesQ4), pages.dtype
    rows, layers, stride = slots.shape[0], 1, 0
    if len(k.shape) == 4:  # (no k[0]: a view costs more than the rest of the call)
        layers, stride = k.shape[0], k.stride(0)
        if len(v.shape) != 4 or v.shape[0] != layers or (v.stride(0) != stride and layers > 1):
            raise ValueError(f"k {tuple(k.shape)}, v {tuple(v.shape)}: one number of layers and one layer stride expected")
        if layers < 1:
            raise ValueError("no layers")
    ck = _rows_of(k, rows, c.n_kv_heads, c.head_dim, dtype, "k", len(k.shape))
    cv = _rows_of(v, rows, c.n_kv_heads, c.head_dim, dtype, "v", len(k.shape))
    rc = load().paged_kv_load_q4(ctypes.byref(c), layer, layers, _arr(slots, _I64, rows, "slots"), rows, ck, cv, stride,
                                 _stream(stream))
    if rc:
        _check(rc, "paged_kv_load_q4")


def paged_tree_attention(bank: Bank, req: Requests, pages: Pages, plan, q, out, ws, layer: int = 0,
                         scale: float | None = None, softcap: float = 0.0, slopes=None, lse=None, stream=None):
    """q, out [rows][n_q_heads][head_dim] of the pages' type; lse float [rows][n_q_heads]; slopes float [n_q_heads];
    scale: 1 / sqrt(head_dim) unless given."""
    _attend("paged_tree_attention", Pages, bank, req, pages, plan, q, out, ws, layer, scale, softcap, slopes, lse, stream)


def paged_tree_attention_q4(bank: Bank, req: Requests, pages: PagesQ4, plan, q, out, ws, layer: int = 0,
                            scale: float | None = None, softcap: float = 0.0, slopes=None, lse=None, stream=None):
    """paged_tree_attention over 4-bit pages; q and out have the pages' row type."""
    _attend("paged_tree_attention_q4", PagesQ4, bank, req, pages, plan, q, out, ws, layer, scale, softcap, slopes, lse, stream)


def _attend(name: str, kind, bank, req, pages, plan, q, out, ws, layer, scale, softcap, slopes, lse, stream):
    c, dtype = _page_kind(pages, kind), pages.dtype
    shape = q.shape
    rows, heads, d = shape
    if (q.dtype is not dtype or out.dtype is not dtype or out.shape != shape or d != c.head_dim or
            not q.is_contiguous() or not out.is_contiguous()):
        raise ValueError(f"q {q.dtype} {tuple(shape)}, out {out.dtype} {tuple(out.shape)}: contiguous {dtype} "
                         f"(rows, heads, {c.head_dim}) expected for both")
    rc = getattr(load(), name)(bank.handle, ctypes.byref(req._c), ctypes.byref(c), layer, plan.data_ptr(),
                               plan.numel(), q.data_ptr(), rows, heads, d ** -0.5 if scale is None else scale,
                               softcap, _arr(slopes, _F32, heads, "slopes"), out.data_ptr(),
                               _arr(lse, _F32, rows * heads, "lse"), ws.data_ptr(), ws.numel(), _stream(stream))
    if rc:
        _check(rc, name)


def tb_logits_workspace_size(batch: int, n_rows: int, vocab: int) -> int:
    return int(load().tb_logits_workspace_size(batch, n_rows, vocab))


def logits_process(bank, req: Requests, logits, out, ws, draft=None, history=None, history_len=None, prompt_len=None,
                   repetition=None, presence=None, frequency=None, bias_start=None, bias_token=None, bias_value=None,
                   mask=None, mask_row=None, temperature: float = 1.0, argmax=None, top1=None, entropy=None,
                   logz_t=None, entropy_t=None, draft_logit=None, stream=None):
    """logits [rows][vocab] (float32, bfloat16 or float16; rows may be strided), out float32 (may be logits);
    history int32 [B][width], mask int32 words [mask rows][width], the rest as the C struct names them."""
    r = req._c
    B = r.batch
    shape, s_in, s_out = logits.shape, logits.stride(), out.stride()
    if len(shape) != 2 or out.shape != shape or (s_in[1] != 1 and shape[1] > 1) or (s_out[1] != 1 and shape[1] > 1):
        raise ValueError(f"logits {tuple(shape)} of strides {s_in}, out {tuple(out.shape)} of strides {s_out}: two "
                         "matrices of one shape with contiguous rows expected")
    kind = _KINDS.get(logits.dtype)
    if kind is None or out.dtype is not _F32:
        raise TypeError(f"logits {logits.dtype}, out {out.dtype}: a 32- or 16-bit float type and float32 expected")
    rows, vocab = shape
    n_bias = 0
    if bias_token is not None:
        n_bias = bias_token.numel()
        if n_bias == 0:
            bias_start = None  # an empty list has no address
    width = words = mask_rows = 0
    if history is not None:
        width = history.shape[-1]
    if mask is not None:
        words = mask.shape[-1]
        mask_rows = mask.numel() // max(words, 1)
    rules = TbLogitRules(
        _arr(history, _I32, B * width, "history"), width, _arr(history_len, _I32, B, "history_len"),
        _arr(prompt_len, _I32, B, "prompt_len"), _arr(draft, _I32, rows, "draft"), _arr(repetition, _F32, B, "repetition"),
        _arr(presence, _F32, B, "presence"), _arr(frequency, _F32, B, "frequency"),
        _arr(bias_start, _I32, B + 1, "bias_start"), _arr(bias_token, _I32, 0, "bias_token"),
        _arr(bias_value, _F32, n_bias, "bias_value"), _arr(mask, _I32, 0 if mask_row is not None else rows * words, "mask"),
        words, _arr(mask_row, _I32, rows, "mask_row"), mask_rows, n_bias)
    st = TbLogitStats(_arr(argmax, _I32, rows, "argmax"), _arr(top1, _F32, rows, "top1"),
                      _arr(entropy, _F32, rows, "entropy"), _arr(logz_t, _F32, rows, "logz_t"),
                      _arr(entropy_t, _F32, rows, "entropy_t"), _arr(draft_logit, _F32, rows, "draft_logit"))
    rc = load().logits_process(None if bank is None else bank.handle, ctypes.byref(r), logits.data_ptr(), kind,
                               s_in[0] if rows > 1 else max(vocab, s_in[0]), rows, vocab, ctypes.byref(rules),
                               temperature, out.data_ptr(), s_out[0] if rows > 1 else max(vocab, s_out[0]),
                               ctypes.byref(st), ws.data_ptr(), ws.numel(), _stream(stream))
    if rc:
        _check(rc, "logits_process")


def make_results(batch: int, device="cuda"):
    """Device buffer for a batch of tb_result blocks (int32 [batch][68])."""
    import torch

    return torch.zeros((batch, RESULT_INTS), dtype=torch.int32, device=device)


def paged_accept(bank: Bank, req: Requests, pages, results, draft=None, argmax=None, vocab: int = 0, lens_out=None,
                 stream=None):
    """results int32 [B][68] (make_results); draft, argmax int32 [rows], or draft None to move by the results given;
    lens_out: None for lens itself; pages None: nothing to move."""
    _accept("paged_accept", Pages, bank, req, pages, results, draft, argmax, vocab, lens_out, stream)


def paged_accept_q4(bank: Bank, req: Requests, pages, results, draft=None, argmax=None, vocab: int = 0, lens_out=None,
                    stream=None):
    """paged_accept over 4-bit pages (PagesQ4, or None: nothing to move)."""
    _accept("paged_accept_q4", PagesQ4, bank, req, pages, results, draft, argmax, vocab, lens_out, stream)


def _accept(name: str, kind, bank, req, pages, results, draft, argmax, vocab, lens_out, stream):
    r = req._c
    c = None if pages is None else _page_kind(pages, kind)
    rows = 0x7FFFFFFF if draft is None else min(draft.shape[0], argmax.shape[0])
    block = _arr(results, _I32, r.batch * RESULT_INTS, "results")
    tokens, greedy = _arr(draft, _I32, 0, "draft"), _arr(argmax, _I32, 0, "argmax")
    if rows == 0:
        tokens = greedy = block  # a step without rows: no address, and none is read, but not "results given" either
    rc = getattr(load(), name)(bank.handle, ctypes.byref(r), _ref(c), tokens, greedy, rows, vocab, block,
                               r.lens if lens_out is None else _arr(lens_out, _I32, r.batch, "lens_out"),
                               _stream(stream))
    if rc:
        _check(rc, name)


# --------------------------------------------------------------------- per-step tree selection


def tb_schedule_hysteretic_ladder(current: int, n_trees: int, feature: float, up_below: float,
                                  down_above: float) -> int:
    return int(load().tb_schedule_hysteretic_ladder(current, n_trees, feature, up_below, down_above))


def tb_schedule_binary(aggressive: int, s: float, tau_on: float, tau_off: float) -> int:
    return int(load().tb_schedule_binary(int(aggressive), s, tau_on, tau_off))


def tb_schedule_threshold_ladder(s: float, edges) -> int:
    e = np.ascontiguousarray(edges, dtype=np.float64)
    return int(load().tb_schedule_threshold_ladder(s, _ptr(e), len(e) + 1))
