"""Python binding of librolekv: argument marshalling only.

Every function here forwards torch tensors' device pointers and the current
CUDA stream to the C ABI of the same name (include/rolekv.h); all work runs
in the library's sm_103a kernels.  There is no fallback: if the shared
library is missing the first call raises.
"""

from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import torch

# ROLEKV_CHECKED=1 in the environment selects the checked build (every
# computed global access checked against its buffer's extent; a miss sets
# STATUS_BOUNDS and is skipped), which has the same entry points.
_LIB_NAME = "librolekv_checked.so" if os.environ.get("ROLEKV_CHECKED") == "1" else "librolekv.so"
_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), _LIB_NAME)

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_CUDA = 0, 1, 2, 3, 4
STATUS_NONFINITE, STATUS_BAD_INDEX, STATUS_TIMEOUT, STATUS_BOUNDS, STATUS_NO_PAGES = 1, 2, 4, 8, 16
POLICY_ROLE_QUOTA, POLICY_GLOBAL, POLICY_FAIR, POLICY_SLACK, POLICY_CEIL = 0, 1, 2, 3, 4
MAX_ROLES = 8
SELECT_MAX_N = 262144
OP_SNAPKV, OP_H2O, OP_COMPRESS = 0, 1, 2


class RolekvError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"rolekv error {code}: {msg}")
        self.code = code


class Tensor(ctypes.Structure):
    _fields_ = [("ptr", ctypes.c_void_p), ("s_layer", ctypes.c_int64), ("s_seq", ctypes.c_int64),
                ("s_head", ctypes.c_int64), ("s_tok", ctypes.c_int64)]


class BatchDesc(ctypes.Structure):
    _fields_ = [("L", ctypes.c_int32), ("b", ctypes.c_int32), ("Hq", ctypes.c_int32),
                ("Hkv", ctypes.c_int32), ("d", ctypes.c_int32), ("n_max", ctypes.c_int32),
                ("seqlens_host", ctypes.POINTER(ctypes.c_int32)),
                ("cu_seqlens_dev", ctypes.c_void_p), ("kept_extra", ctypes.c_int32)]


class SelectParams(ctypes.Structure):
    _fields_ = [("n_roles", ctypes.c_int32), ("alpha", ctypes.c_float * MAX_ROLES),
                ("key_role", ctypes.c_int32), ("alpha_key", ctypes.c_float),
                ("budget", ctypes.c_float), ("policy", ctypes.c_int32),
                ("ban_mask", ctypes.c_uint32), ("keep_last", ctypes.c_int32)]


class PoolDesc(ctypes.Structure):
    _fields_ = [("ptr", ctypes.c_void_p), ("L", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("d", ctypes.c_int32),
                ("s_layer", ctypes.c_int64), ("s_page", ctypes.c_int64)]


class PagesDesc(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("n_pages", ctypes.c_int32),
                ("page_rows", ctypes.c_int32), ("table", ctypes.c_void_p), ("lens", ctypes.c_void_p),
                ("refs", ctypes.c_void_p)]


_lib = None

# The handle of a device's current stream.  torch.cuda.current_stream() makes a
# Stream object around it first.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda device: torch.cuda.current_stream(device).cuda_stream)

# The index of the current device.  torch.cuda.current_device() checks first that
# CUDA is initialised, which a call's own tensors have seen to.
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device

# (name, restype, argtypes) of every exported function
_SIGNATURES = [
    ("rolekv_kept_count", ctypes.c_int64, [ctypes.c_int64, ctypes.c_float]),
    ("rolekv_kept_rows", ctypes.c_int64, [ctypes.c_int64, ctypes.c_float, ctypes.c_int32]),
    ("rolekv_workspace_size", ctypes.c_int,
     [ctypes.c_int, ctypes.POINTER(BatchDesc), ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)]),
    ("snapkv_score", ctypes.c_int,
     [ctypes.POINTER(BatchDesc), Tensor, Tensor, ctypes.c_int32, ctypes.c_int32, ctypes.c_float,
      ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
      ctypes.c_void_p, ctypes.c_void_p]),
    ("snapkv_score_noalloc", ctypes.c_int,
     [ctypes.POINTER(BatchDesc), Tensor, Tensor, ctypes.c_int32, ctypes.c_int32, ctypes.c_float,
      ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]),
    ("quest_score", ctypes.c_int,
     [ctypes.POINTER(BatchDesc), Tensor, Tensor, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p,
      ctypes.c_void_p]),
    ("rolekv_selftest_wait", ctypes.c_int, [ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p]),
    ("rolekv_decode_workspace_size", ctypes.c_int,
     [ctypes.POINTER(BatchDesc), ctypes.c_float, ctypes.POINTER(ctypes.c_size_t)]),
    ("decode_attention", ctypes.c_int,
     [ctypes.POINTER(BatchDesc), Tensor, Tensor, Tensor, ctypes.c_void_p, ctypes.c_float,
      ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p,
      ctypes.c_void_p]),
    ("h2o_score", ctypes.c_int,
     [ctypes.POINTER(BatchDesc), Tensor, Tensor, ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p,
      ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p]),
    ("rolekv_selftest_score_timeout", ctypes.c_int, [ctypes.c_int64]),
    ("rolekv_checked_build", ctypes.c_int, []),
    ("rolekv_selftest_shrink_extent", ctypes.c_int, [ctypes.c_int64]),
    ("role_alloc_select", ctypes.c_int,
     [ctypes.POINTER(BatchDesc), ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(SelectParams),
      ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
      ctypes.c_void_p]),
    ("kv_compact", ctypes.c_int,
     [ctypes.POINTER(BatchDesc), Tensor, Tensor, ctypes.c_void_p, ctypes.c_float, ctypes.c_void_p,
      ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]),
    ("rolekv_compress", ctypes.c_int,
     [ctypes.POINTER(BatchDesc), Tensor, Tensor, Tensor, ctypes.c_int32, ctypes.c_int32,
      ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(SelectParams),
      ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
      ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p]),
    ("rolekv_q4_page_bytes", ctypes.c_int64, [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]),
    ("rolekv_pages_workspace_size", ctypes.c_int, [ctypes.POINTER(PagesDesc), ctypes.POINTER(ctypes.c_size_t)]),
    ("kv_pages_reserve", ctypes.c_int,
     [ctypes.POINTER(PagesDesc), ctypes.POINTER(PoolDesc), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
      ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p]),
    ("kv_pages_fork", ctypes.c_int,
     [ctypes.POINTER(PagesDesc), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p]),
    ("kv_pages_pack", ctypes.c_int,
     [ctypes.POINTER(PagesDesc), ctypes.POINTER(PoolDesc), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
      ctypes.c_void_p, ctypes.c_void_p]),
    ("kv_compact_q4", ctypes.c_int,
     [ctypes.POINTER(BatchDesc), Tensor, Tensor, ctypes.c_void_p, ctypes.c_float, ctypes.POINTER(PoolDesc),
      ctypes.POINTER(PagesDesc), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]),
    ("kv_append_q4", ctypes.c_int,
     [ctypes.POINTER(PoolDesc), ctypes.POINTER(PagesDesc), ctypes.c_void_p, ctypes.c_int32, Tensor, Tensor,
      ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]),
    ("kv_expand_q4", ctypes.c_int,
     [ctypes.POINTER(PoolDesc), ctypes.POINTER(PagesDesc), ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p,
      ctypes.c_int32, Tensor, Tensor, ctypes.c_void_p, ctypes.c_void_p]),
    ("rolekv_decode_q4_workspace_size", ctypes.c_int,
     [ctypes.c_int32] * 5 + [ctypes.POINTER(ctypes.c_size_t)]),
    ("decode_attention_q4", ctypes.c_int,
     [ctypes.POINTER(PoolDesc), ctypes.POINTER(PagesDesc), ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, Tensor,
      ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p]),
    ("rolekv_set_stage_events", ctypes.c_int, [ctypes.POINTER(ctypes.c_void_p), ctypes.c_int32]),
    ("rolekv_last_error", ctypes.c_char_p, []),
    ("rolekv_version", ctypes.c_char_p, []),
]


def library_path() -> str:
    return _LIB_PATH


def lib():
    """The loaded librolekv (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with "
                               "`python -c 'import __graft_entry__ as g; g.build()'`")
        L = ctypes.CDLL(_LIB_PATH)
        for name, res, args in _SIGNATURES:
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _lib = L
    return _lib


def _check(rc: int):
    if rc != OK:
        raise RolekvError(rc, lib().rolekv_last_error().decode())


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream(stream=None):
    if stream is not None:
        return stream.cuda_stream
    # the current stream's handle without a Stream object (3.0 us of a call's 23)
    return _raw_stream(torch.cuda.current_device())


# ---------------------------------------------------------------- descriptors

class Batch:
    """Shapes of one call.  seqlens (list of ints) makes it a varlen batch; the
    device copy of the prefix sums is created here, once.  kept_extra widens
    every kept row beyond ceil(B n) (the ceiling policy needs it)."""

    def __init__(self, L, b, Hq, Hkv, d, n_max, seqlens: Optional[Sequence[int]] = None,
                 device="cuda", kept_extra: int = 0):
        self.L, self.b, self.Hq, self.Hkv, self.d, self.n_max = L, b, Hq, Hkv, d, n_max
        self.kept_extra = int(kept_extra)
        self._kept = {}
        self.seqlens = list(seqlens) if seqlens is not None else None
        self._host = None
        self.cu_seqlens = None
        if self.seqlens is not None:
            self._host = (ctypes.c_int32 * len(self.seqlens))(*self.seqlens)
            cu = [0]
            for n in self.seqlens:
                cu.append(cu[-1] + n)
            self.cu_seqlens = torch.tensor(cu, dtype=torch.int32, device=device)
        self.desc = BatchDesc(L, b, Hq, Hkv, d, n_max,
                              self._host if self._host is not None else None,
                              ctypes.c_void_p(self.cu_seqlens.data_ptr()) if self.cu_seqlens is not None else None,
                              self.kept_extra)

    @property
    def varlen(self) -> bool:
        return self.seqlens is not None

    @property
    def T(self) -> int:
        return sum(self.seqlens) if self.varlen else self.b * self.n_max

    @property
    def n_units(self) -> int:
        return self.L * self.b * self.Hkv

    def score_shape(self):
        return (self.L, self.Hkv, self.T) if self.varlen else (self.L, self.b, self.Hkv, self.n_max)

    def role_shape(self):
        return (self.T,) if self.varlen else (self.b, self.n_max)

    def kept_total(self, budget: float) -> int:
        """Slots of all kept rows of a layer and head (summed once a budget)."""
        total = self._kept.get(budget)
        if total is None:
            lens = self.seqlens if self.varlen else [self.n_max] * self.b
            total = self._kept[budget] = sum(kept_rows(n, budget, self.kept_extra) for n in lens)
        return total

    def kept_shape(self, budget: float):
        if self.varlen:
            return (self.L, self.Hkv, sum(kept_rows(n, budget, self.kept_extra) for n in self.seqlens))
        return (self.L, self.b, self.Hkv, kept_rows(self.n_max, budget, self.kept_extra))


def tensor_desc(t: torch.Tensor, packed: bool = False) -> Tensor:
    """Strides of a 5-D [L][b][H][n][d] tensor, or of a packed 4-D [L][T][H][d]
    tensor, as a rolekv_tensor."""
    if t.dtype != torch.bfloat16:
        raise TypeError("rolekv tensors are bf16")
    stride = t.stride()
    if stride[-1] != 1:
        raise ValueError("the head-dim axis must be contiguous")
    if packed:
        if len(stride) != 4:
            raise ValueError("packed tensors are [L][T][H][d]")
        sl, st, sh, _ = stride
        return Tensor(t.data_ptr(), sl, 0, sh, st)
    if len(stride) != 5:
        raise ValueError("dense tensors are [L][b][H][n][d]")
    sl, ss, sh, st, _ = stride
    return Tensor(t.data_ptr(), sl, ss, sh, st)


def select_params(budget: float, alpha: Sequence[float], alpha_key: float = 0.0, key_role: int = 1,
                  policy: int = POLICY_ROLE_QUOTA, ban_mask: int = 0,
                  keep_last: int = 0) -> SelectParams:
    al = (ctypes.c_float * MAX_ROLES)(*([float(x) for x in alpha] + [0.0] * (MAX_ROLES - len(alpha))))
    return SelectParams(len(alpha), al, key_role, alpha_key, budget, policy, ban_mask, keep_last)


# ----------------------------------------------------------------- entry points

def kept_count(n: int, budget: float) -> int:
    return int(lib().rolekv_kept_count(int(n), float(budget)))


def kept_rows(n: int, budget: float, kept_extra: int = 0) -> int:
    return int(lib().rolekv_kept_rows(int(n), float(budget), int(kept_extra)))


def workspace_size(op: int, batch: Batch, W: int = 0) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().rolekv_workspace_size(op, ctypes.byref(batch.desc), W, ctypes.byref(out)))
    return int(out.value)


def workspace(op: int, batch: Batch, W: int = 0, device="cuda") -> torch.Tensor:
    return torch.empty(max(workspace_size(op, batch, W), 256), dtype=torch.uint8, device=device)


def _scratch(make, stream, *args, **kw) -> torch.Tensor:
    """A call's own workspace, allocated on the stream the call runs on: the
    caching allocator hands a freed block to its own stream alone."""
    if stream is None:
        return make(*args, **kw)
    with torch.cuda.stream(stream):
        return make(*args, **kw)


def snapkv_score(batch: Batch, q_win: torch.Tensor, k: torch.Tensor, W: int, pool_k: int,
                 scores: torch.Tensor, scores_prepool: Optional[torch.Tensor] = None,
                 lse_win: Optional[torch.Tensor] = None, scale: float = 0.0,
                 ws: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                 stream=None) -> torch.Tensor:
    if ws is None:
        ws = _scratch(workspace, stream, OP_SNAPKV, batch, W, device=k.device)
    _check(lib().snapkv_score(ctypes.byref(batch.desc), tensor_desc(q_win), tensor_desc(k, batch.varlen),
                              W, pool_k, scale, _ptr(lse_win), _ptr(scores), _ptr(scores_prepool),
                              _ptr(ws), ws.numel(), _ptr(status), _stream(stream)))
    return scores


def snapkv_score_noalloc(batch: Batch, q_win: torch.Tensor, k: torch.Tensor, W: int, pool_k: int,
                         scores: torch.Tensor, scores_prepool: Optional[torch.Tensor] = None,
                         lse_win: Optional[torch.Tensor] = None, scale: float = 0.0,
                         status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """snapkv_score for callers that cannot allocate device memory: no
    workspace argument, the library's own static scratch is used instead
    (see rolekv.h for its limit and sharing rules)."""
    _check(lib().snapkv_score_noalloc(ctypes.byref(batch.desc), tensor_desc(q_win),
                                      tensor_desc(k, batch.varlen), W, pool_k, scale, _ptr(lse_win),
                                      _ptr(scores), _ptr(scores_prepool), _ptr(status), _stream(stream)))
    return scores


def quest_score(batch: Batch, q_win: torch.Tensor, k: torch.Tensor, W: int, page: int,
                scores: torch.Tensor, stream=None) -> torch.Tensor:
    _check(lib().quest_score(ctypes.byref(batch.desc), tensor_desc(q_win, False),
                             tensor_desc(k, batch.varlen), W, page, _ptr(scores), _stream(stream)))
    return scores


def selftest_wait(limit_ns: int, status: torch.Tensor, stream=None) -> None:
    _check(lib().rolekv_selftest_wait(int(limit_ns), _ptr(status), _stream(stream)))


def decode_workspace(batch: Batch, budget: float, device="cuda") -> torch.Tensor:
    out = ctypes.c_size_t(0)
    _check(lib().rolekv_decode_workspace_size(ctypes.byref(batch.desc), budget, ctypes.byref(out)))
    return torch.empty(max(int(out.value), 256), dtype=torch.uint8, device=device)


def cache_desc(t: torch.Tensor, batch: Batch, compacted: bool) -> Tensor:
    """Strides of a cache tensor: kv_compact's output (compacted=True:
    dense [L][b][Hkv][K][d], varlen [L][Hkv][Ktot][d]) or an uncompacted K/V
    in the library's own layouts."""
    if compacted and batch.varlen:
        return tensor_desc(t.transpose(1, 2), True)
    return tensor_desc(t, batch.varlen)


def decode_attention(batch: Batch, q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                     keep_idx: Optional[torch.Tensor], budget: float, out: torch.Tensor,
                     compacted: bool = True, scale: float = 0.0, ws: Optional[torch.Tensor] = None,
                     status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """q bf16 [L][b][Hq][d] -> out fp32 [L][b][Hq][d]."""
    if ws is None:
        ws = _scratch(decode_workspace, stream, batch, budget, device=q.device)
    if q.dtype != torch.bfloat16 or q.dim() != 4 or q.stride(-1) != 1:
        raise ValueError("q is a bf16 [L][b][Hq][d] tensor with a contiguous last axis")
    sl, ss, sh, _ = q.stride()
    qd = Tensor(q.data_ptr(), sl, ss, sh, q.shape[-1])
    _check(lib().decode_attention(ctypes.byref(batch.desc), qd, cache_desc(k_cache, batch, compacted),
                                  cache_desc(v_cache, batch, compacted), _ptr(keep_idx), budget, scale,
                                  _ptr(out), _ptr(ws), ws.numel(), _ptr(status), _stream(stream)))
    return out


def h2o_score(batch: Batch, q: torch.Tensor, k: torch.Tensor, scores: torch.Tensor, scale: float = 0.0,
              lse: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
              status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """lse: optional fp32 natural-log normalisers of every query row (dense
    [L][b][Hq][n], varlen [L][Hq][T]); given, the score is one pass over K."""
    if ws is None:
        ws = _scratch(workspace, stream, OP_H2O, batch, 0, device=k.device)
    _check(lib().h2o_score(ctypes.byref(batch.desc), tensor_desc(q, batch.varlen),
                           tensor_desc(k, batch.varlen), scale, _ptr(lse), _ptr(scores), _ptr(ws),
                           ws.numel(), _ptr(status), _stream(stream)))
    return scores


def selftest_score_timeout(limit_ns: int) -> None:
    """Arm the next two-pass SnapKV score on this thread to time out at its
    per-unit meeting point after limit_ns (diagnostic; see rolekv.h)."""
    _check(lib().rolekv_selftest_score_timeout(int(limit_ns)))


def checked_build() -> bool:
    """Whether the loaded library is the checked build."""
    return lib().rolekv_checked_build() == 1


def selftest_shrink_extent(rows: int) -> None:
    """Checked build only: the next kv_compact on this thread takes its output
    extent as `rows` rows smaller, so its checks on the last rows fire
    (diagnostic; see rolekv.h)."""
    _check(lib().rolekv_selftest_shrink_extent(int(rows)))


def role_alloc_select(batch: Batch, scores: torch.Tensor, roles: torch.Tensor, params: SelectParams,
                      keep_idx: torch.Tensor, pool_k: int = 1, keep_mask: Optional[torch.Tensor] = None,
                      kept_per_role: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                      stream=None) -> torch.Tensor:
    _check(lib().role_alloc_select(ctypes.byref(batch.desc), _ptr(scores), _ptr(roles), ctypes.byref(params),
                                   pool_k, _ptr(keep_idx), _ptr(keep_mask), _ptr(kept_per_role),
                                   _ptr(status), _stream(stream)))
    return keep_idx


def kv_compact(batch: Batch, k: torch.Tensor, v: torch.Tensor, keep_idx: torch.Tensor, budget: float,
               k_out: torch.Tensor, v_out: torch.Tensor, status: Optional[torch.Tensor] = None,
               stream=None):
    _check(lib().kv_compact(ctypes.byref(batch.desc), tensor_desc(k, batch.varlen),
                            tensor_desc(v, batch.varlen), _ptr(keep_idx), budget, _ptr(k_out),
                            _ptr(v_out), _ptr(status), _stream(stream)))
    return k_out, v_out


def rolekv_compress(batch: Batch, q_win: torch.Tensor, k: torch.Tensor, v: torch.Tensor, W: int,
                    pool_k: int, roles: torch.Tensor, params: SelectParams, keep_idx: torch.Tensor,
                    k_out: torch.Tensor, v_out: torch.Tensor, ws: torch.Tensor,
                    kept_per_role: Optional[torch.Tensor] = None, lse_win: Optional[torch.Tensor] = None,
                    scale: float = 0.0, status: Optional[torch.Tensor] = None, stream=None):
    _check(lib().rolekv_compress(ctypes.byref(batch.desc), tensor_desc(q_win), tensor_desc(k, batch.varlen),
                                 tensor_desc(v, batch.varlen), W, pool_k, scale, _ptr(lse_win), _ptr(roles),
                                 ctypes.byref(params), _ptr(keep_idx), _ptr(k_out), _ptr(v_out),
                                 _ptr(kept_per_role), _ptr(ws), ws.numel(), _ptr(status), _stream(stream)))
    return keep_idx, k_out, v_out


def set_stage_events(events: Sequence[torch.cuda.Event]):
    """Record events[i] after the i-th kernel launch of every later call on
    this thread (empty sequence: off).  The events must have been recorded
    once so that they exist."""
    arr = (ctypes.c_void_p * max(1, len(events)))(*[ctypes.c_void_p(e.cuda_event) for e in events])
    _check(lib().rolekv_set_stage_events(arr, len(events)))


def compact_shape(batch: Batch, budget: float):
    return batch.kept_shape(budget) + (batch.d,)


# ------------------------------------------------- the cache in four bits ----

_U8, _I32, _BF16, _F32 = torch.uint8, torch.int32, torch.bfloat16, torch.float32


class Pages:
    """The tables of a paged 4-bit cache: n_seqs slots of at most max_pages
    pages each, out of n_pages pages of page_rows rows.  table [n_seqs]
    [max_pages], lens [n_seqs] and refs [n_pages] are int32 views of one device
    array, `state`, in this order (copy it to keep or restore a state)."""

    def __init__(self, n_seqs: int, n_pages: int, page_rows: int, max_pages: int, device="cuda"):
        self.n_seqs, self.n_pages, self.page_rows, self.max_pages = n_seqs, n_pages, page_rows, max_pages
        t = n_seqs * max_pages
        self.state = torch.zeros(t + n_seqs + n_pages, dtype=torch.int32, device=device)
        self.table = self.state[:t].view(n_seqs, max_pages)
        self.lens = self.state[t:t + n_seqs]
        self.refs = self.state[t + n_seqs:]
        self.table.fill_(-1)
        self.desc = PagesDesc(n_seqs, max_pages, n_pages, page_rows, self.table.data_ptr(), self.lens.data_ptr(),
                              self.refs.data_ptr())


def q4_pool_shape(L: int, n_pages: int, Hkv: int, d: int, page_rows: int):
    """Shape of a pool: uint8, a record of 18 d bytes for 16 rows."""
    if int(lib().rolekv_q4_page_bytes(Hkv, d, page_rows)) < 0:
        raise ValueError(f"no 4-bit pages of Hkv={Hkv}, d={d}, page_rows={page_rows}")
    return (L, n_pages, Hkv, page_rows // 16, 18 * d)


def pool_desc(pool: torch.Tensor, pages: Pages) -> PoolDesc:
    """Strides of a uint8 [L][n_pages][Hkv][page_rows / 16][18 d] pool, whose
    pages are contiguous."""
    try:
        L, n, h, r, rec = pool.shape
        sl, sp, sh, sr, se = pool.stride()
    except ValueError:
        rec = 0
    if not rec or pool.dtype is not _U8:
        raise TypeError("a pool is a uint8 [L][n_pages][Hkv][page_rows / 16][18 d] tensor")
    if n != pages.n_pages or r * 16 != pages.page_rows or rec % 18:
        raise ValueError(f"pool of {n} pages of {r * 16} rows for tables of {pages.n_pages} of {pages.page_rows}")
    if se != 1 or sr != rec or sh != r * rec:
        raise ValueError("the pages of a pool are contiguous")
    return PoolDesc(pool.data_ptr(), L, h, rec // 18, sl, sp)


def _here(stream, *tensors):
    """The call's stream; its tensors (None: not given) are on the current
    device, and so is the stream."""
    dev = _current_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"a tensor on {t.device}, the current device is cuda:{dev}")
    if stream is None:
        return _raw_stream(dev)
    if stream.device_index != dev:
        raise ValueError(f"a stream of cuda:{stream.device_index}, the current device is cuda:{dev}")
    return stream.cuda_stream


def _int32(t: Optional[torch.Tensor], n: int, name: str):
    """The pointer of a contiguous int32 array of n elements, or None."""
    if t is None:
        return None
    if t.dtype is not _I32 or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} is a contiguous int32 array of {n} elements")
    return t.data_ptr()


def pages_workspace(pages: Pages, device="cuda") -> torch.Tensor:
    out = ctypes.c_size_t(0)
    _check(lib().rolekv_pages_workspace_size(ctypes.byref(pages.desc), ctypes.byref(out)))
    return torch.empty(int(out.value), dtype=torch.uint8, device=device)


def kv_pages_reserve(pages: Pages, pool: torch.Tensor, add: torch.Tensor, pos: torch.Tensor,
                     ws: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None, stream=None):
    """Room for add[x] more rows of every slot; pos[x] becomes the first of them."""
    st = _here(stream, pages.state, pool, add, pos, ws, status)
    if ws is None:
        ws = _scratch(pages_workspace, stream, pages, device=pool.device)
    _check(lib().kv_pages_reserve(ctypes.byref(pages.desc), ctypes.byref(pool_desc(pool, pages)),
                                  _int32(add, pages.n_seqs, "add"), _int32(pos, pages.n_seqs, "pos"), _ptr(ws),
                                  ws.numel(), _ptr(status), st))
    return pos


def kv_pages_fork(pages: Pages, parent: torch.Tensor, ws: Optional[torch.Tensor] = None,
                  status: Optional[torch.Tensor] = None, stream=None):
    """Slot x takes over the pages of slot parent[x] (-1: none, x: its own)."""
    st = _here(stream, pages.state, parent, ws, status)
    if ws is None:
        ws = _scratch(pages_workspace, stream, pages, device=parent.device)
    _check(lib().kv_pages_fork(ctypes.byref(pages.desc), _int32(parent, pages.n_seqs, "parent"), _ptr(ws), ws.numel(),
                               _ptr(status), st))


def kv_pages_pack(pages: Pages, pool: torch.Tensor, n_live: Optional[torch.Tensor] = None,
                  ws: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None, stream=None):
    """The pages in use moved to the front of the pool."""
    st = _here(stream, pages.state, pool, n_live, ws, status)
    if ws is None:
        ws = _scratch(pages_workspace, stream, pages, device=pool.device)
    _check(lib().kv_pages_pack(ctypes.byref(pages.desc), ctypes.byref(pool_desc(pool, pages)),
                               _int32(n_live, 1, "n_live"), _ptr(ws), ws.numel(), _ptr(status), st))
    return n_live


def kv_compact_q4(batch: Batch, k: torch.Tensor, v: torch.Tensor, keep_idx: torch.Tensor, budget: float,
                  pool: torch.Tensor, pages: Pages, pos: torch.Tensor, seqs: Optional[torch.Tensor] = None,
                  status: Optional[torch.Tensor] = None, stream=None):
    """The kept rows of K and V into rows pos[x] .. of the cache.  K and V may
    lie in pinned host memory, of which the kept rows alone are read."""
    st = _here(stream, pages.state, pool, keep_idx, pos, seqs, status, batch.cu_seqlens)
    dev = pool.get_device()
    for t in (k, v):
        if t.get_device() != dev and not (t.device.type == "cpu" and t.is_pinned()):
            raise ValueError(f"k or v on {t.device}: not on the current device, cuda:{dev}, nor in pinned host memory")
    _check(lib().kv_compact_q4(ctypes.byref(batch.desc), _rows_desc(batch, k, "k"), _rows_desc(batch, v, "v"),
                               _int32(keep_idx, batch.L * batch.Hkv * max(0, batch.kept_total(budget)), "keep_idx"),
                               budget, ctypes.byref(pool_desc(pool, pages)),
                               ctypes.byref(pages.desc), _int32(seqs, batch.b, "seqs"),
                               _int32(pos, pages.n_seqs, "pos"), _ptr(status), st))
    return pool


def _rows_desc(batch: Batch, t: torch.Tensor, name: str) -> Tensor:
    """Strides of a batch's K or V, bf16 [L][b][Hkv][n][d] or packed
    [L][T][Hkv][d]."""
    shape, stride = t.shape, t.stride()
    if t.dtype is not _BF16 or stride[-1] != 1:
        raise TypeError(f"{name} is bf16 with a contiguous last axis")
    if batch.varlen:
        if len(shape) == 4 and shape[1] >= batch.T and (shape[0], shape[2], shape[3]) == (batch.L, batch.Hkv, batch.d):
            return Tensor(t.data_ptr(), stride[0], 0, stride[2], stride[1])
    elif len(shape) == 5 and shape[3] >= batch.n_max and \
            (shape[0], shape[1], shape[2], shape[4]) == (batch.L, batch.b, batch.Hkv, batch.d):
        return Tensor(t.data_ptr(), stride[0], stride[1], stride[2], stride[3])
    raise ValueError(f"{name} is [L][b][Hkv][n][d], packed [L][T][Hkv][d], of the batch's sizes")


def _pair_desc(k: torch.Tensor, v: torch.Tensor, pool: PoolDesc, name: str):
    """Strides of bf16 [L][b][Hkv][rows][d] K and V over a pool, b and rows."""
    shape, ks, vs = k.shape, k.stride(), v.stride()
    if len(shape) != 5 or (shape[0], shape[2], shape[4]) != (pool.L, pool.Hkv, pool.d) or v.shape != shape:
        raise ValueError(f"k_{name} and v_{name} are [L={pool.L}][b][Hkv={pool.Hkv}][rows][d={pool.d}] tensors")
    if k.dtype is not _BF16 or v.dtype is not _BF16 or ks[4] != 1 or vs[4] != 1:
        raise TypeError(f"k_{name} and v_{name} are bf16 with a contiguous last axis")
    return (Tensor(k.data_ptr(), ks[0], ks[1], ks[2], ks[3]), Tensor(v.data_ptr(), vs[0], vs[1], vs[2], vs[3]),
            shape[1], shape[3])


def kv_append_q4(pool: torch.Tensor, pages: Pages, k_new: torch.Tensor, v_new: torch.Tensor, pos: torch.Tensor,
                 count: Optional[torch.Tensor] = None, seqs: Optional[torch.Tensor] = None,
                 status: Optional[torch.Tensor] = None, stream=None):
    """bf16 k_new, v_new [L][b][Hkv][T][d] into rows pos[x] .. of the cache."""
    st = _here(stream, pages.state, pool, k_new, v_new, pos, count, seqs, status)
    pd = pool_desc(pool, pages)
    kd, vd, b, T = _pair_desc(k_new, v_new, pd, "new")
    _check(lib().kv_append_q4(ctypes.byref(pd), ctypes.byref(pages.desc),
                              _int32(seqs, b, "seqs"), b, kd, vd, T,
                              _int32(count, pages.n_seqs, "count"), _int32(pos, pages.n_seqs, "pos"), _ptr(status),
                              st))
    return pool


def kv_expand_q4(pool: torch.Tensor, pages: Pages, k_out: torch.Tensor, v_out: torch.Tensor,
                 start: Optional[torch.Tensor] = None, seqs: Optional[torch.Tensor] = None,
                 status: Optional[torch.Tensor] = None, stream=None):
    """Rows start[x] .. of the cache as bf16 [L][b][Hkv][rows][d]."""
    st = _here(stream, pages.state, pool, k_out, v_out, start, seqs, status)
    pd = pool_desc(pool, pages)
    kd, vd, b, rows = _pair_desc(k_out, v_out, pd, "out")
    _check(lib().kv_expand_q4(ctypes.byref(pd), ctypes.byref(pages.desc), _int32(seqs, b, "seqs"), b,
                              _int32(start, pages.n_seqs, "start"), rows, kd, vd, _ptr(status), st))
    return k_out, v_out


def decode_q4_workspace(L: int, b: int, Hq: int, Hkv: int, d: int, device="cuda") -> torch.Tensor:
    out = ctypes.c_size_t(0)
    _check(lib().rolekv_decode_q4_workspace_size(L, b, Hq, Hkv, d, ctypes.byref(out)))
    return torch.empty(int(out.value), dtype=torch.uint8, device=device)


def decode_attention_q4(q: torch.Tensor, pool: torch.Tensor, pages: Pages, out: torch.Tensor, scale: float = 0.0,
                        seqs: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                        status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """q bf16 [L][b][Hq][d] -> out fp32 [L][b][Hq][d]."""
    st = _here(stream, pages.state, q, pool, out, seqs, ws, status)
    pd = pool_desc(pool, pages)
    shape, stride = q.shape, q.stride()
    if q.dtype is not _BF16 or len(shape) != 4 or stride[3] != 1:
        raise ValueError("q is a bf16 [L][b][Hq][d] tensor with a contiguous last axis")
    L, b, Hq, d = shape
    if L != pd.L or d != pd.d or out.shape != shape or out.dtype is not _F32 or not out.is_contiguous():
        raise ValueError("q and a contiguous fp32 out are [L][b][Hq][d] of the pool's L and d")
    if ws is None:
        ws = _scratch(decode_q4_workspace, stream, L, b, Hq, pd.Hkv, d, device=q.device)
    _check(lib().decode_attention_q4(ctypes.byref(pd), ctypes.byref(pages.desc), _int32(seqs, b, "seqs"), b, Hq,
                                     Tensor(q.data_ptr(), stride[0], stride[1], stride[2], d), scale, _ptr(out),
                                     _ptr(ws), ws.numel(), _ptr(status), st))
    return out
