"""Thin binding of the C-ABI library ``libdpaps.so`` (see ``include/dpaps.h``).

Argument marshalling only: every function here hands device pointers of torch
tensors (torch is used for device memory and streams, nothing else) and host
pointers of numpy arrays to the entry point of the same name.  There is no
fallback: if the library has not been built, importing fails loudly.
"""
from __future__ import annotations

import ctypes as C
import math
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdpaps.so")

PS_OK, PS_EINVAL, PS_EKEY, PS_EWORKER, PS_ECONFLICT, PS_ENOMEM, PS_EHIP, PS_EREMOTE, PS_ELAYOUT, PS_ELIMIT, PS_ESTALL = \
    0, -1, -2, -3, -4, -5, -6, -7, -8, -9, -10
STAT_NAMES = ["pull_local", "pull_remote", "push_local", "push_remote", "relocated", "localize_keys",
              "msg_acc_req", "msg_acc_fwd", "msg_acc_reply", "msg_loc_req", "msg_loc_instruct", "msg_loc_transfer",
              "cache_hit", "cache_stale"]
OPT_MF_EXACT, OPT_MF_CACHE_ROWS, OPT_MF_WAVES, OPT_MF_PROFILE, OPT_MF_GROUPED, OPT_MF_HEAVY_LEN, OPT_PUSH_SEQUENTIAL, OPT_MF_TEAM_MAX, OPT_MF_CLASSIC, OPT_LOCATION_CACHES, OPT_KGE_EXACT = 1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11

EXPORTS = ["ps_create", "ps_destroy", "ps_pull", "ps_push", "ps_push_noalloc", "ps_localize", "ps_owner", "ps_stats", "ps_status",
           "ps_set_option", "ps_last_error", "mf_block_ratings", "mf_load_ratings", "mf_sgd_epoch", "mf_sgd_epoch_handoff", "mf_train_sse",
           "mf_profile_read", "kge_sgd_step", "kge_sgd_epoch", "emb_lookup", "emb_grad", "emb_adagrad_step",
           "muon_orthogonalize", "muon_step", "group_rows", "expert_matmul", "expert_grad", "adapter_matmul", "adapter_grad"]

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}         # PS_F32, PS_BF16, PS_F16
_TOKENS = {torch.int32: 0, torch.int64: 1}                              # PS_I32, PS_I64
_NO_PAD = -(1 << 63)                                                     # PS_NO_PAD


class PSError(RuntimeError):
    def __init__(self, code: int, what: str, detail: str = ""):
        super().__init__(f"{what}: status {code}" + (f" ({detail})" if detail else ""))
        self.code = code


def load_library() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2002_00655_amd.build` "
                          "(there is no CPU fallback)")
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float
    lib.ps_create.argtypes = [i64, i32, i32, C.POINTER(vp)]
    lib.ps_destroy.argtypes = [vp]
    lib.ps_pull.argtypes = [vp, i32, vp, i64, vp, vp]
    lib.ps_push.argtypes = [vp, i32, vp, i64, vp, vp]
    lib.ps_push_noalloc.argtypes = [vp, i32, vp, i64, vp, vp]
    lib.ps_localize.argtypes = [vp, vp, i64, i32, vp]
    lib.ps_owner.argtypes = [vp, vp, i64, vp, vp]
    lib.ps_stats.argtypes = [vp, vp, vp]
    lib.ps_status.argtypes = [vp, vp]
    lib.ps_set_option.argtypes = [vp, i32, i64]
    lib.ps_last_error.argtypes = [vp]
    lib.ps_last_error.restype = C.c_char_p
    lib.mf_block_ratings.argtypes = [i64, i64, i64, vp, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp, vp]
    lib.mf_load_ratings.argtypes = [vp, i64, i64, i64, vp, vp, vp, i32, i32, vp, vp, vp, vp]
    lib.mf_sgd_epoch.argtypes = [vp, vp, vp, i32, f32, f32, vp]
    lib.mf_sgd_epoch_handoff.argtypes = [vp, f32, f32, vp, vp]
    lib.mf_train_sse.argtypes = [vp, vp, vp]
    lib.mf_profile_read.argtypes = [vp, vp, vp, vp]
    lib.kge_sgd_step.argtypes = [vp, i32, i64, i32, i64, vp, vp, vp, i32, vp, i32, vp, f32, f32, vp, vp]
    lib.kge_sgd_epoch.argtypes = [vp, i64, i32, i64, vp, vp, vp, i32, vp, i32, vp, vp, i32, i64, i32, f32, f32, vp, vp]
    lib.emb_lookup.argtypes = [vp, i32, i64, i64, i32, vp, i32, i64, i64, f32, vp, i32, i64, vp]
    lib.emb_grad.argtypes = [vp, i64, i32, vp, i32, i64, i64, f32, vp, i32, i64, vp, i32, vp]
    lib.emb_adagrad_step.argtypes = [vp, i32, i64, i64, i32, vp, i32, i64, i64, f32, vp, i32, i64, f32, f32, vp]
    lib.muon_orthogonalize.argtypes = [vp, i32, i32, i32, vp, i32, i64, vp, i32, i64, i32, f32, vp]
    lib.muon_step.argtypes = [vp, i32, i64, i32, i32, i32, vp, i32, i64, f32, f32, i32, f32, i32, f32, vp]
    lib.group_rows.argtypes = [vp, i32, vp, i32, i64, i64, vp, vp, vp]
    lib.expert_matmul.argtypes = [vp, i32, i64, i32, i32, i32, i32, vp, vp, i64, vp, i32, i64, i32, vp, i32, i64, i32, vp]
    lib.expert_grad.argtypes = [vp, i32, i32, i32, vp, vp, i64, vp, i64, i32, vp, i64, i32, i32, vp, i32, vp]
    lib.adapter_matmul.argtypes = [vp, i32, i64, i32, i32, i64, i64, i32, i32, f32, vp, vp, i64, vp, i32, i64, vp, i32, i64, vp]
    lib.adapter_grad.argtypes = [vp, i32, i64, i32, i32, i64, i64, i32, i32, f32, vp, vp, i64, vp, i64, vp, i64, i32, vp, i32, i64, vp, vp, vp]
    for name in EXPORTS:
        if name != "ps_last_error":
            getattr(lib, name).restype = C.c_int
    return lib


_lib = load_library()


def _stream() -> int:
    # (the handle itself: as a torch.cuda.Stream object it takes 2.7 us, a third of a pull of 100 keys)
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _dev(t: torch.Tensor, dtype: torch.dtype) -> torch.Tensor:
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"expected a contiguous CUDA tensor of {dtype}, got {t.dtype} on {t.device}")
    return t


def _per_row(t: torch.Tensor, rows: int) -> tuple[int, int]:
    """Values per row of an int32 tensor of `rows` rows, and where it is.  (Its own shape where it has that one: a view is 1 us.)"""
    if rows == 0:
        return 0, 0
    _dev(t, torch.int32)
    return (t.shape[1] if t.dim() == 2 and t.shape[0] == rows else t.reshape(rows, -1).shape[1]), t.data_ptr()


def _tokens(t: torch.Tensor) -> tuple[int, int, int]:
    """Where the tokens are, their type, how many."""
    kind = _TOKENS.get(t.dtype)
    if kind is None or not t.is_cuda or not t.is_contiguous():
        raise TypeError(f"expected contiguous CUDA tokens of int32 or int64, got {t.dtype} on {t.device}")
    return t.data_ptr(), kind, t.numel()


def _rows(t: torch.Tensor, n: int, copy: bool = True, apart: bool = False) -> tuple[torch.Tensor, int, int, int]:
    """A tensor of n rows (its last dimension a row, the others counted together): what has to stay alive until the call is made, where
    it is, its type, the rows' distance in elements.  What is read (copy): a matrix is taken as it lies, or refused where it is transposed; rows of
    more dimensions that do not lie at one distance are copied, and so are numbers that were expanded to rows (the gradient of a sum) and, if they
    have to be apart, rows that were expanded.  What is written lies as the call can write it, or is refused."""
    kind = _TYPES.get(t.dtype)
    if kind is None or not t.is_cuda or t.dim() == 0:
        raise TypeError(f"expected a CUDA tensor of float32, bfloat16 or float16, got {t.dtype} on {t.device}")
    if t.dim() != 2:
        r = t.reshape(n, t.shape[-1])
        if not copy and r.data_ptr() != t.data_ptr():
            raise ValueError(f"the rows of a result have to lie at one distance, got shape {tuple(t.shape)}, strides {t.stride()}")
        t = r
    rows, cols = t.shape
    if copy and rows == n > 0 and cols > 1:
        if t.stride(1) == 0:
            t = t[:1].contiguous().expand(n, cols) if t.stride(0) == 0 else t.contiguous()
        if apart and n > 1 and t.stride(0) == 0:
            t = t.contiguous()
    if rows != n or (n > 0 and cols > 1 and t.stride(1) != 1):
        raise ValueError(f"expected {n} rows whose elements are contiguous, got shape {tuple(t.shape)}, strides {t.stride()}")
    return t, t.data_ptr(), kind, (t.stride(0) if n > 1 else cols)


def _matrices(t: torch.Tensor) -> tuple[int, int, int]:
    if t.dim() < 2:
        raise ValueError(f"expected matrices, got shape {tuple(t.shape)}")
    batch = 1
    for d in t.shape[:-2]:
        batch *= d
    return batch, t.shape[-2], t.shape[-1]


def _groups(groups) -> tuple[int, int, int, int]:
    """What group_rows has returned: where the order and the offsets are, the number of groups, of rows."""
    order, offsets = groups
    _dev(order, torch.int32), _dev(offsets, torch.int32)
    if offsets.numel() < 2:
        raise ValueError("the offsets of groups are one more than there are groups")
    return order.data_ptr(), offsets.data_ptr(), offsets.numel() - 1, order.numel()


def _count_of(t: torch.Tensor) -> int:
    """The rows of a tensor, its last dimension being a row."""
    return t.shape[0] if t.dim() == 2 else math.prod(t.shape[:-1])


def _result(shape, like: torch.Tensor, dtype: torch.dtype | None) -> tuple[torch.Tensor, int, int, int]:
    """A new tensor of rows, in `dtype` or the type of `like`: itself, where it is, its type, the rows' distance."""
    dtype = like.dtype if dtype is None else dtype
    if dtype not in _TYPES:
        raise TypeError(f"the result is float32, bfloat16 or float16, not {dtype}")
    out = torch.empty(shape, dtype=dtype, device=like.device)
    return out, out.data_ptr(), _TYPES[dtype], shape[-1]


def _pairs_of(t: torch.Tensor, n: int, what: str) -> tuple[int, int]:
    """Rows of a tensor that stand for n rows, and for how many each of them stands."""
    rows = _count_of(t) if t.dim() else 0
    if n == 0 and rows == 0:
        return 0, 1
    if rows <= 0 or n % rows or n == 0:
        raise ValueError(f"{what} has {rows} rows, which cannot stand for the {n} of the groups")
    return rows, n // rows


def _host(a, dtype) -> np.ndarray:
    return np.ascontiguousarray(a, dtype=dtype)


def _flatten_schedule(schedule):
    strata = [np.ascontiguousarray(s, dtype=np.int32).reshape(-1, 3) for s in schedule]
    tasks = np.concatenate(strata) if strata else np.zeros((0, 3), np.int32)
    sptr = np.concatenate([[0], np.cumsum([s.shape[0] for s in strata])]).astype(np.int32)
    return np.ascontiguousarray(tasks), sptr, len(strata)


class ParameterServer:
    """Handle of one server: ``num_keys`` keys x ``value_len`` fp32 values, ``num_workers`` workers."""

    def __init__(self, num_keys: int, value_len: int, num_workers: int):
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU: the parameter server runs on the device only")
        torch.cuda.init()
        torch.cuda.current_stream()
        self.K, self.L, self.W = int(num_keys), int(value_len), int(num_workers)
        h = C.c_void_p()
        rc = _lib.ps_create(self.K, self.L, self.W, C.byref(h))
        if rc:
            raise PSError(rc, "ps_create")
        self._h = h

    def close(self) -> None:
        if getattr(self, "_h", None) and _lib is not None:       # (at interpreter exit the module's globals may be gone)
            _lib.ps_destroy(self._h)
            self._h = None

    __del__ = close

    def _check(self, rc: int, what: str) -> None:
        if rc:
            raise PSError(rc, what, (_lib.ps_last_error(self._h) or b"").decode())

    # -- primitives -----------------------------------------------------------
    def pull(self, keys: torch.Tensor, worker: int = -1, out: torch.Tensor | None = None) -> torch.Tensor:
        keys = _dev(keys, torch.int64)
        n = keys.numel()
        if out is None:
            out = torch.empty((n, self.L), dtype=torch.float32, device=keys.device)
        _dev(out, torch.float32)
        self._check(_lib.ps_pull(self._h, worker, keys.data_ptr(), n, out.data_ptr(), _stream()), "ps_pull")
        return out

    def push(self, keys: torch.Tensor, deltas: torch.Tensor, worker: int = -1) -> None:
        keys, deltas = _dev(keys, torch.int64), _dev(deltas, torch.float32)
        if deltas.numel() != keys.numel() * self.L:
            raise ValueError("deltas must hold value_len floats per key")
        self._check(_lib.ps_push(self._h, worker, keys.data_ptr(), keys.numel(), deltas.data_ptr(), _stream()), "ps_push")

    def push_noalloc(self, keys: torch.Tensor, deltas: torch.Tensor, worker: int = -1) -> None:
        """ps_push with the library's fixed scratch array: no device allocation (see include/dpaps.h)."""
        keys, deltas = _dev(keys, torch.int64), _dev(deltas, torch.float32)
        if deltas.numel() != keys.numel() * self.L:
            raise ValueError("deltas must hold value_len floats per key")
        self._check(_lib.ps_push_noalloc(self._h, worker, keys.data_ptr(), keys.numel(), deltas.data_ptr(), _stream()), "ps_push_noalloc")

    def localize(self, keys: torch.Tensor, worker: int) -> None:
        keys = _dev(keys, torch.int64)
        self._check(_lib.ps_localize(self._h, keys.data_ptr(), keys.numel(), worker, _stream()), "ps_localize")

    def owner(self, keys: torch.Tensor | None = None) -> torch.Tensor:
        if keys is None:
            keys = torch.arange(self.K, dtype=torch.int64, device="cuda")
        keys = _dev(keys, torch.int64)
        out = torch.empty(keys.numel(), dtype=torch.int32, device=keys.device)
        self._check(_lib.ps_owner(self._h, keys.data_ptr(), keys.numel(), out.data_ptr(), _stream()), "ps_owner")
        return out

    def stats(self) -> dict:
        out = np.zeros(len(STAT_NAMES), dtype=np.int64)
        self._check(_lib.ps_stats(self._h, out.ctypes.data, _stream()), "ps_stats")
        return dict(zip(STAT_NAMES, (int(x) for x in out)))

    def status(self) -> None:
        self._check(_lib.ps_status(self._h, _stream()), "ps_status")

    def set_option(self, option: int, value: int) -> None:
        self._check(_lib.ps_set_option(self._h, option, value), "ps_set_option")

    # -- matrix factorization ---------------------------------------------------
    def mf_load_ratings(self, m, n, rows, cols, vals, row_bounds, col_bounds, block_ptr) -> None:
        rows, cols, vals = _dev(rows, torch.int32), _dev(cols, torch.int32), _dev(vals, torch.float32)
        rb, cb, bp = _host(row_bounds, np.int64), _host(col_bounds, np.int64), _host(block_ptr, np.int64)
        if bp.size != (rb.size - 1) * (cb.size - 1) + 1:
            raise ValueError("block_ptr must have d_row*d_col+1 entries")
        self._check(_lib.mf_load_ratings(self._h, m, n, rows.numel(), rows.data_ptr(), cols.data_ptr(), vals.data_ptr(),
                                         rb.size - 1, cb.size - 1, rb.ctypes.data, cb.ctypes.data, bp.ctypes.data,
                                         _stream()), "mf_load_ratings")
        self._mf_grid = (rb.size - 1, cb.size - 1)

    def mf_sgd_epoch(self, schedule, lr: float, lam: float) -> None:
        """schedule: int32 [S, T, 3] array or list of [T_s, 3] arrays of (worker, row block, column block)."""
        tasks, sptr, ns = _flatten_schedule(schedule)
        self._check(_lib.mf_sgd_epoch(self._h, tasks.ctypes.data, sptr.ctypes.data, ns, float(lr), float(lam), _stream()),
                    "mf_sgd_epoch")

    def mf_sgd_epoch_raw(self, tasks: np.ndarray, sptr: np.ndarray, lr: float, lam: float) -> None:
        self._check(_lib.mf_sgd_epoch(self._h, tasks.ctypes.data, sptr.ctypes.data, sptr.size - 1, float(lr), float(lam),
                                      _stream()), "mf_sgd_epoch")

    def mf_sgd_epoch_handoff(self, lr: float, lam: float, want_order: bool = True):
        """An epoch with column blocks handed from worker to worker (see include/dpaps.h).  Returns the recorded
        order as an int32 array [d_row, d_col, 2] of (column block, workers that had it before), or None."""
        d_row, d_col = self._mf_grid
        order = np.empty((d_row, d_col, 2), dtype=np.int32) if want_order else None
        self._check(_lib.mf_sgd_epoch_handoff(self._h, float(lr), float(lam), order.ctypes.data if want_order else None,
                                              _stream()), "mf_sgd_epoch_handoff")
        return order

    def mf_profile_read(self):
        """(summed SGD kernel time in ms, number of launches) since the last call; needs OPT_MF_PROFILE."""
        ms, cnt = C.c_double(0.0), C.c_int64(0)
        self._check(_lib.mf_profile_read(self._h, C.addressof(ms), C.addressof(cnt), _stream()), "mf_profile_read")
        return float(ms.value), int(cnt.value)

    def mf_train_sse(self) -> float:
        out = C.c_double(0.0)
        self._check(_lib.mf_train_sse(self._h, C.addressof(out), _stream()), "mf_train_sse")
        return float(out.value)

    def kge_sgd_step(self, num_entities, dim, subj, rel, obj, neg_subj, neg_obj, lr, eps, worker: int = -1,
                     want_loss: bool = True):
        """One mini-batch step of ComplEx training (see include/dpaps.h); returns the summed loss or None."""
        subj, rel, obj = _dev(subj, torch.int32), _dev(rel, torch.int32), _dev(obj, torch.int32)
        batch = subj.numel()
        (ns, ns_ptr), (no, no_ptr) = _per_row(neg_subj, batch), _per_row(neg_obj, batch)
        loss = C.c_double(0.0)
        self._check(_lib.kge_sgd_step(self._h, worker, num_entities, dim, batch, subj.data_ptr(), rel.data_ptr(), obj.data_ptr(),
                                      ns, ns_ptr, no, no_ptr, float(lr), float(eps),
                                      C.addressof(loss) if want_loss else None, _stream()), "kge_sgd_step")
        return float(loss.value) if want_loss else None

    def kge_sgd_epoch(self, num_entities, dim, subj, rel, obj, neg_subj, neg_obj, part_ptr, batch, lookahead, lr, eps,
                      want_loss: bool = True):
        """One epoch over workers with relation partitioning and pre-localization (see include/dpaps.h)."""
        subj, rel, obj = _dev(subj, torch.int32), _dev(rel, torch.int32), _dev(obj, torch.int32)
        n = subj.numel()
        (ns, ns_ptr), (no, no_ptr) = _per_row(neg_subj, n), _per_row(neg_obj, n)
        pp = _host(part_ptr, np.int64)
        loss = C.c_double(0.0)
        self._check(_lib.kge_sgd_epoch(self._h, num_entities, dim, n, subj.data_ptr(), rel.data_ptr(), obj.data_ptr(), ns,
                                       ns_ptr, no, no_ptr, pp.ctypes.data, pp.size - 1, int(batch),
                                       int(lookahead), float(lr), float(eps), C.addressof(loss) if want_loss else None, _stream()),
                    "kge_sgd_epoch")
        return float(loss.value) if want_loss else None

    # -- token models -------------------------------------------------------------
    def emb_lookup(self, tokens, first_key: int = 0, num_tokens: int | None = None, dim: int | None = None, scale: float = 1.0,
                   pad_token: int | None = None, worker: int = -1, dtype: torch.dtype = torch.float32, out: torch.Tensor | None = None):
        """The scaled embeddings of `tokens` (any shape), in `dtype`, shape [*tokens.shape, dim] (see include/dpaps.h)."""
        at, kind, n = _tokens(tokens)
        dim = self.L if dim is None else dim
        if out is None:
            if dtype not in _TYPES:
                raise TypeError(f"the result is float32, bfloat16 or float16, not {dtype}")
            out = tokens.new_empty((*tokens.shape, dim), dtype=dtype)
            to, out_kind, stride = out.data_ptr(), _TYPES[dtype], dim
        else:
            if out.shape != (*tokens.shape, dim):
                raise ValueError(f"out must have the shape {(*tokens.shape, dim)}")
            _, to, out_kind, stride = _rows(out, n, copy=False)
        self._check(_lib.emb_lookup(self._h, worker, first_key, self.K - first_key if num_tokens is None else num_tokens, dim, at, kind, n,
                                    _NO_PAD if pad_token is None else pad_token, scale, to, out_kind, stride, _stream()), "emb_lookup")
        return out

    def emb_grad(self, tokens, dout, num_tokens: int, scale: float = 1.0, pad_token: int | None = None, grad: torch.Tensor | None = None,
                 accumulate: bool = False):
        """The gradient of a lookup with respect to its table, [num_tokens, dim] in fp32, from that of its output (see include/dpaps.h)."""
        (at, kind, n), dim = _tokens(tokens), dout.shape[-1]
        kept, frm, dout_kind, stride = _rows(dout, n)
        if grad is None:
            if accumulate:
                raise ValueError("accumulate needs the gradient to add to")
            grad = torch.empty((num_tokens, dim), dtype=torch.float32, device=tokens.device)
        _dev(grad, torch.float32)
        if grad.shape != (num_tokens, dim):
            raise ValueError(f"grad must have the shape {(num_tokens, dim)}")
        self._check(_lib.emb_grad(self._h, num_tokens, dim, at, kind, n, _NO_PAD if pad_token is None else pad_token, scale, frm, dout_kind, stride,
                                  grad.data_ptr(), int(accumulate), _stream()), "emb_grad")
        return grad

    def emb_adagrad_step(self, tokens, dout, lr: float, eps: float, first_key: int = 0, num_tokens: int | None = None, scale: float = 1.0,
                         pad_token: int | None = None, worker: int = -1) -> None:
        """One step of AdaGrad on the rows that `tokens` mention, from the gradient of their lookup's output (see include/dpaps.h)."""
        (at, kind, n), dim = _tokens(tokens), dout.shape[-1]
        kept, frm, dout_kind, stride = _rows(dout, n)
        self._check(_lib.emb_adagrad_step(self._h, worker, first_key, self.K - first_key if num_tokens is None else num_tokens, dim, at, kind, n,
                                          _NO_PAD if pad_token is None else pad_token, scale, frm, dout_kind, stride, lr, eps, _stream()),
                    "emb_adagrad_step")

    def muon_orthogonalize(self, x: torch.Tensor, steps: int = 5, eps: float = 1e-7, dtype: torch.dtype | None = None, out: torch.Tensor | None = None):
        """Matrices [..., rows, cols] orthogonalised by Newton-Schulz products, in x's type or `dtype`, of which the precision of the
        products follows (see include/dpaps.h)."""
        batch, rows, cols = _matrices(x)
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype if dtype is None else dtype, device=x.device)
        elif out.shape != x.shape:
            raise ValueError(f"out must have the shape {tuple(x.shape)}")
        kept, frm, in_kind, in_ld = _rows(x, batch * rows, apart=True)
        _, to, out_kind, out_ld = _rows(out, batch * rows, copy=False)
        self._check(_lib.muon_orthogonalize(self._h, batch, rows, cols, frm, in_kind, in_ld, to, out_kind, out_ld, steps, eps, _stream()), "muon_orthogonalize")
        return out

    def muon_step(self, first_key: int, grad: torch.Tensor, lr: float, momentum: float = 0.95, nesterov: bool = True, weight_decay: float = 0.0,
                  steps: int = 5, eps: float = 1e-7, worker: int = -1) -> None:
        """One step of weight matrices in the server, from their gradients [..., rows, dim] (see include/dpaps.h)."""
        batch, rows, dim = _matrices(grad)
        kept, frm, kind, ld = _rows(grad, batch * rows, apart=True)
        self._check(_lib.muon_step(self._h, worker, first_key, batch, rows, dim, frm, kind, ld, lr, momentum, int(nesterov), weight_decay, steps, eps,
                                   _stream()), "muon_step")

    # -- models of many matrices ------------------------------------------------------
    def group_rows(self, ids: torch.Tensor, num_groups: int, pad: int | None = None) -> tuple[torch.Tensor, torch.Tensor]:
        """The rows, numbered as `ids` lie, ordered by the group that they name, and where the groups start, num_groups + 1 places; rows whose id is `pad`
        are of no group (see include/dpaps.h)."""
        at, kind, n = _tokens(ids)
        order = torch.empty(n, dtype=torch.int32, device=ids.device)
        offsets = torch.empty(num_groups + 1, dtype=torch.int32, device=ids.device)
        self._check(_lib.group_rows(self._h, num_groups, at, kind, n, _NO_PAD if pad is None else pad, order.data_ptr(), offsets.data_ptr(), _stream()), "group_rows")
        return order, offsets

    def expert_matmul(self, x: torch.Tensor, groups, first_key: int, rows: int, dim: int | None = None, transposed: bool = False, sum_pairs: int = 1,
                      worker: int = -1, dtype: torch.dtype | None = None, out: torch.Tensor | None = None):
        """The grouped rows times their expert's matrix (rows x dim, keys of the server), or its transpose; `groups` from group_rows (see include/dpaps.h).  x has
        the groups' n rows, or fewer, each of which then stands for as many neighbouring ones.  The result, in x's type or `dtype`, is [n / sum_pairs, columns]:
        of sum_pairs neighbouring rows the sum."""
        order, offsets, experts, n = _groups(groups)
        dim = self.L if dim is None else dim
        given, columns = (rows, dim) if transposed else (dim, rows)
        if x.dim() == 0 or x.shape[-1] != given:
            raise ValueError(f"expected rows of {given} numbers, got shape {tuple(x.shape)}")
        x_rows, x_pairs = _pairs_of(x, n, "x")
        if sum_pairs < 1 or n % sum_pairs:
            raise ValueError(f"sums of {sum_pairs} of {n} rows")
        kept, frm, kind, stride = _rows(x, x_rows)
        out_rows = n // sum_pairs
        if out is None:
            out, to, out_kind, out_stride = _result((out_rows, columns), x, dtype)
        elif out.dim() == 0 or out.shape[-1] != columns or _count_of(out) != out_rows:
            raise ValueError(f"out must have the shape {(out_rows, columns)}")
        else:
            _, to, out_kind, out_stride = _rows(out, out_rows, copy=False)
        self._check(_lib.expert_matmul(self._h, worker, first_key, experts, rows, dim, int(transposed), order, offsets, n, frm, kind, stride, x_pairs, to, out_kind,
                                       out_stride, sum_pairs, _stream()), "expert_matmul")
        return out

    def expert_grad(self, left: torch.Tensor, right: torch.Tensor, groups, dtype: torch.dtype = torch.float32, out: torch.Tensor | None = None):
        """Per group the sum of its rows' products left_i right_j, [groups, rows, dim]: the gradients of experts' matrices (see include/dpaps.h)."""
        order, offsets, experts, n = _groups(groups)
        if left.dtype != right.dtype:
            raise TypeError(f"left and right have one type, not {left.dtype} and {right.dtype}")
        (left_rows, left_pairs), (right_rows, right_pairs) = _pairs_of(left, n, "left"), _pairs_of(right, n, "right")
        shape = (experts, left.shape[-1], right.shape[-1])
        if out is None:
            out = torch.empty(shape, dtype=dtype, device=left.device)
        elif out.shape != shape or not out.is_contiguous():
            raise ValueError(f"out must be contiguous and have the shape {shape}")
        kept_left, l, kind, l_stride = _rows(left, left_rows)
        kept_right, r, _, r_stride = _rows(right, right_rows)
        _, to, out_kind, _ = _rows(out, experts * shape[1], copy=False)
        self._check(_lib.expert_grad(self._h, experts, shape[1], shape[2], order, offsets, n, l, l_stride, left_pairs, r, r_stride, right_pairs, kind, to, out_kind,
                                     _stream()), "expert_grad")
        return out

    def adapter_matmul(self, x: torch.Tensor, groups, first_key: int, rows: int, first_a: int, first_b: int, rank: int, scale: float = 1.0, dim: int | None = None,
                       worker: int = -1, dtype: torch.dtype | None = None, out: torch.Tensor | None = None):
        """Rows [..., dim] times a shared matrix and, beside it, scaled, their adapter's two of low rank, [..., rows]; `groups` from group_rows of the rows' adapters (see
        include/dpaps.h)."""
        order, offsets, adapters, n = _groups(groups)
        dim = self.L if dim is None else dim
        if x.dim() == 0 or x.shape[-1] != dim or _count_of(x) != n:
            raise ValueError(f"expected {n} rows of {dim} numbers, got shape {tuple(x.shape)}")
        kept, frm, kind, stride = _rows(x, n)
        if out is None:
            out, to, out_kind, out_stride = _result((*x.shape[:-1], rows), x, dtype)
        elif out.shape != (*x.shape[:-1], rows):
            raise ValueError(f"out must have the shape {(*x.shape[:-1], rows)}")
        else:
            _, to, out_kind, out_stride = _rows(out, n, copy=False)
        self._check(_lib.adapter_matmul(self._h, worker, first_key, rows, dim, first_a, first_b, adapters, rank, scale, order, offsets, n, frm, kind, stride, to, out_kind,
                                        out_stride, _stream()), "adapter_matmul")
        return out

    def adapter_grad(self, x: torch.Tensor, dout: torch.Tensor, groups, first_key: int, first_a: int, first_b: int, rank: int, scale: float = 1.0, worker: int = -1,
                     want_dx: bool = True, dtype: torch.dtype | None = None):
        """The gradients of adapter_matmul with respect to x (or None), in x's type or `dtype`, and to all adapters' A and B transposed, fp32, [adapters, rank, dim] and
        [adapters, rank, rows] (see include/dpaps.h)."""
        order, offsets, adapters, n = _groups(groups)
        if x.dtype != dout.dtype:
            raise TypeError(f"x and dout have one type, not {x.dtype} and {dout.dtype}")
        if x.dim() == 0 or dout.shape[:-1] != x.shape[:-1] or _count_of(x) != n:
            raise ValueError(f"expected {n} rows, got shapes {tuple(x.shape)} and {tuple(dout.shape)}")
        dim, rows = x.shape[-1], dout.shape[-1]
        dx, to, to_kind, to_stride = _result(x.shape, x, dtype) if want_dx else (None, None, _TYPES.get(x.dtype, 0), dim)
        da, db = (torch.empty((adapters, rank, c), dtype=torch.float32, device=x.device) for c in (dim, rows))
        kept_x, frm, kind, stride = _rows(x, n)
        kept_d, d, _, d_stride = _rows(dout, n)
        self._check(_lib.adapter_grad(self._h, worker, first_key, rows, dim, first_a, first_b, adapters, rank, scale, order, offsets, n, frm, stride, d, d_stride, kind, to,
                                      to_kind, to_stride, da.data_ptr(), db.data_ptr(), _stream()), "adapter_grad")
        return dx, da, db


def mf_block_ratings(m, n, rows, cols, vals, row_bounds, col_bounds):
    """Device version of the block-by-block data layout; returns (rows, cols, vals, block_ptr[host])."""
    rows, cols, vals = _dev(rows, torch.int32), _dev(cols, torch.int32), _dev(vals, torch.float32)
    rb, cb = _host(row_bounds, np.int64), _host(col_bounds, np.int64)
    ro, co, vo = torch.empty_like(rows), torch.empty_like(cols), torch.empty_like(vals)
    bp = np.zeros((rb.size - 1) * (cb.size - 1) + 1, dtype=np.int64)
    rc = _lib.mf_block_ratings(m, n, rows.numel(), rows.data_ptr(), cols.data_ptr(), vals.data_ptr(), rb.size - 1,
                               cb.size - 1, rb.ctypes.data, cb.ctypes.data, ro.data_ptr(), co.data_ptr(), vo.data_ptr(),
                               bp.ctypes.data, _stream())
    if rc:
        raise PSError(rc, "mf_block_ratings")
    return ro, co, vo, bp
