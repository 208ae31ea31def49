"""Python binding of the serving calls of libseedq.so: page bookkeeping, the
8-bit key/value cache, the attention that reads it, and token log probabilities.

Like the rest of the binding it marshals arguments and computes nothing: every
buffer is the caller's torch tensor, every length and page number stays on the
device, and calls only enqueue work on the given stream (torch's current stream
by default).  The tensors' device must be the current one.  What the C ABI
cannot see (shapes, types, devices) is checked here and raises ValueError; what it
refuses itself raises SeedQError.
"""
from __future__ import annotations

import ctypes as C
import struct

import torch

from . import seedq as Q

DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
KINDS = {"int8": 0, "e4m3": 1}
STATUS = {0: "ok", 1: "no pages", 2: "bad lengths", 3: "no room"}
_CODE_TYPES = (torch.int8, torch.uint8, torch.float8_e4m3fn)


def _want(ok, what: str):
    if not ok:
        raise ValueError(what)


_current_device = torch._C._cuda_getDevice  # torch.cuda.current_device takes twice as long


def _stream(s, device) -> int:
    # The library launches on the current device, whose kernels another device's pointers would reach.
    index = device.index
    if index != _current_device():
        raise ValueError(f"the current device ({_current_device()}) is not the tensors' ({device})")
    if s is None:
        return torch._C._cuda_getCurrentRawStream(index)
    return s if isinstance(s, int) else s.cuda_stream


def _check(status: int, where: str):
    if status != 0:
        raise Q.SeedQError(status, where)


# Messages are put together only when a check fails: these run on every call of
# a decode step, whose kernels take a few microseconds.

def _ints(t, n, dtype, device, name: str):
    if not (t.dtype is dtype and t.ndim == 1 and t.shape[0] >= n and t.is_contiguous() and t.device == device):
        raise ValueError(f"{name}: a contiguous {dtype} vector of at least {n} on {device} is wanted")


def _table(t, n, device):
    if not (t.dtype is torch.int32 and t.ndim == 2 and t.shape[0] >= n and (t.stride(1) == 1 or t.shape[1] == 1) and t.device == device):
        raise ValueError(f"block_table: int32, {n} or more rows with contiguous entries on {device} are wanted")


def _row_stride(t) -> int:
    """The row stride of a matrix; torch leaves that of a single row open."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _same_strides(a, b) -> bool:
    """Of tensors of one shape, but for those of single entries."""
    return all(x == y or n < 2 for n, x, y in zip(a.shape, a.stride(), b.stride()))


def _code_strides(t):
    """Strides of the code tensor in bytes; those of single entries, which torch leaves open, as head_dim."""
    return tuple(st if n > 1 else t.shape[3] for n, st in zip(t.shape[:3], t.stride()))


def _rows(t, name: str, tokens, heads, dim, device):
    """Checks a (tokens, heads, dim) tensor of any strides but the last, and returns its type's code and the strides."""
    dt, st = DTYPES.get(t.dtype), t.stride()
    if dt is None or t.shape != (tokens, heads, dim) or t.device != device or st[2] != 1:
        raise ValueError(f"{name}: ({tokens}, {heads}, {dim}) float32, bfloat16 or float16 with contiguous last dimension "
                         f"on {device} is wanted, got {tuple(t.shape)} {t.dtype}")
    return dt, st


class BatchPlan:
    """The outputs of seedq_batch_plan for up to max_requests requests and
    max_tokens new tokens a step: slots, positions, requests (per token),
    seq_lens, starts, status (per request), free_count.  They are allocated
    once, so a captured graph keeps its addresses; seq_lens, starts and status
    are as long as the last build had requests, starts one more."""

    def __init__(self, max_requests: int, max_tokens: int, device="cuda"):
        r, t = int(max_requests), int(max_tokens)
        self.max_requests, self.max_tokens = r, t
        self.slots = torch.full((t,), -1, dtype=torch.int64, device=device)
        ints = torch.zeros(2 * t + 3 * r + 2, dtype=torch.int32, device=device)
        self.positions, self.requests, *self._per_request, self.free_count = ints.split([t, t, r, r + 1, r, 1])
        self._out = tuple(C.c_void_p(t.data_ptr()) for t in (
            self.slots, self.positions, self.requests, *self._per_request, self.free_count))
        self._resize(r)

    def _resize(self, n: int):
        # What lies past n requests is an earlier step's.
        lens, starts, status = self._per_request
        self.n_requests, self.seq_lens, self.starts, self.status = n, lens[:n], starts[:n + 1], status[:n]

    def build(self, seq_lens, n_new, block_table, free_pages, free_count, page_size: int, stream=None):
        """seedq_batch_plan: lengths and new-token counts (int32 vectors) in,
        this object's tensors out; block_table and free_pages change in place."""
        n, dev = n_new.shape[0], self.slots.device
        if not 1 <= n <= self.max_requests:
            raise ValueError(f"n_new: 1..{self.max_requests} requests are wanted, got {n}")
        _ints(n_new, n, torch.int32, dev, "n_new")
        _ints(seq_lens, n, torch.int32, dev, "seq_lens")
        _ints(free_pages, 0, torch.int32, dev, "free_pages")
        _ints(free_count, 1, torch.int32, dev, "free_count")
        _table(block_table, n, dev)
        _check(Q.lib().seedq_batch_plan(
            n, seq_lens.data_ptr(), n_new.data_ptr(), page_size, block_table.data_ptr(), _row_stride(block_table),
            block_table.shape[1], free_pages.data_ptr(), free_pages.shape[0], free_count.data_ptr(),
            self.max_tokens, *self._out, _stream(stream, dev)), "seedq_batch_plan")
        if n != self.n_requests:
            self._resize(n)


class KVCache:
    """A paged 8-bit key/value cache over the caller's tensors (seedq_kv_cache).

    k, v: codes, (n_pages, n_kv_heads, page_size, head_dim) in any order of the
    first three dimensions (a transposed view of (n_pages, page_size,
    n_kv_heads, head_dim) is as good), int8, uint8 or float8_e4m3fn, the same
    strides for both.  k_scale, v_scale: (n_pages, n_kv_heads) float32.
    kind: "int8" or "e4m3".  KVCache.empty allocates all four."""

    def __init__(self, k, v, k_scale, v_scale, kind: str = "int8"):
        _want(kind in KINDS, f"kind: one of {sorted(KINDS)} is wanted, got {kind!r}")
        _want(k.dim() == 4 and k.shape == v.shape and _code_strides(k) == _code_strides(v) and k.stride(3) == v.stride(3) == 1,
              "k, v: four dimensions, equal shapes and strides, and contiguous codes are wanted")
        _want(k.dtype in _CODE_TYPES and v.dtype == k.dtype, "k, v: int8, uint8 or float8_e4m3fn codes are wanted")
        self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = k.shape
        for t in (k_scale, v_scale):
            _want(t.dtype is torch.float32 and t.shape == (self.n_pages, self.n_kv_heads) and t.is_contiguous(),
                  "k_scale, v_scale: contiguous float32 (n_pages, n_kv_heads) are wanted")
        _want(k.is_cuda and all(t.device == k.device for t in (v, k_scale, v_scale)),
              "k, v, k_scale, v_scale: tensors of one CUDA device are wanted")
        self.k, self.v, self.k_scale, self.v_scale, self.kind, self.device = k, v, k_scale, v_scale, kind, k.device
        self.desc = Q.KvCacheDesc(KINDS[kind], self.n_kv_heads, self.head_dim, self.page_size, self.n_pages,
                                  k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(),
                                  *_code_strides(k))
        self._ref = C.byref(self.desc)

    @classmethod
    def empty(cls, n_pages: int, n_kv_heads: int, head_dim: int, page_size: int = 16, kind: str = "int8",
              device="cuda"):
        """A cache of its own; pages hold nothing until they are written."""
        shape = (n_pages, n_kv_heads, page_size, head_dim)
        k, v = (torch.empty(shape, dtype=torch.int8, device=device) for _ in range(2))
        ks, vs = (torch.zeros(shape[:2], dtype=torch.float32, device=device) for _ in range(2))
        return cls(k, v, ks, vs, kind)

    def append(self, k, v, slots, stream=None):
        """seedq_kv_append: k, v (n_tokens, n_kv_heads, head_dim) to slots (int64)."""
        n, dt, st = self._pair(k, v, slots)
        _check(Q.lib().seedq_kv_append(self._ref, k.data_ptr(), v.data_ptr(), dt, st[0], st[1],
                                       slots.data_ptr(), n, _stream(stream, self.device)), "seedq_kv_append")

    def gather(self, slots, k, v, stream=None):
        """seedq_kv_gather: the cached numbers at slots into k, v."""
        n, dt, st = self._pair(k, v, slots)
        _check(Q.lib().seedq_kv_gather(self._ref, slots.data_ptr(), n, k.data_ptr(), v.data_ptr(), dt,
                                       st[0], st[1], _stream(stream, self.device)), "seedq_kv_gather")

    def _pair(self, k, v, slots):
        n, dev = k.shape[0], self.device
        dt, st = _rows(k, "k", n, self.n_kv_heads, self.head_dim, dev)
        if v.shape != k.shape or v.dtype is not k.dtype or v.device != dev or (v.stride() != st and not _same_strides(k, v)):
            raise ValueError("v: the shape, type, strides and device of k are wanted")
        _ints(slots, n, torch.int64, dev, "slots")
        return n, dt, st

    def attend_workspace(self, n_heads: int, max_new: int = 1):
        """A zeroed workspace for attend() with that many query heads and, per
        request, up to max_new query tokens."""
        n = Q.lib().seedq_kv_attend_workspace_bytes(self._ref, n_heads, max_new)
        _want(n > 0, "attend_workspace: n_heads a multiple of n_kv_heads, max_new >= 1 and a supported cache are wanted")
        return torch.zeros(n, dtype=torch.uint8, device=self.device)

    def attend(self, q, out, seq_lens, starts, block_table, workspace, max_new: int = 1, scale: float | None = None,
               window: int = 0, lse=None, stream=None):
        """seedq_kv_attend: q, out (n_tokens, n_heads, head_dim), lse
        (n_tokens, n_heads) float32 or None; scale defaults to head_dim^-1/2."""
        n, heads, _ = q.shape
        dev = self.device
        qt, qs = _rows(q, "q", n, heads, self.head_dim, dev)
        ot, os = _rows(out, "out", n, heads, self.head_dim, dev)
        b = starts.shape[0] - 1
        _ints(starts, 2, torch.int32, dev, "starts")
        _ints(seq_lens, b, torch.int32, dev, "seq_lens")
        _table(block_table, b, dev)
        if not workspace.is_contiguous() or workspace.device != dev:
            raise ValueError("workspace: a tensor of attend_workspace is wanted")
        if lse is not None and not (lse.dtype is torch.float32 and lse.shape == (n, heads) and lse.is_contiguous()
                                    and lse.device == dev):
            raise ValueError(f"lse: contiguous float32 ({n}, {heads}) on {dev} is wanted")
        try:
            a = Q.ATTEND_ARGS.pack(b, heads, n, q.data_ptr(), qs[0], qs[1], out.data_ptr(), os[0], os[1],
                                   qt, ot, 0 if lse is None else lse.data_ptr(), seq_lens.data_ptr(), starts.data_ptr(),
                                   block_table.data_ptr(), _row_stride(block_table), block_table.shape[1], max_new, window,
                                   self.head_dim ** -0.5 if scale is None else scale, workspace.data_ptr(), workspace.nbytes)
        except struct.error as e:
            raise ValueError(f"max_new, window: 32-bit integers, scale: a number are wanted ({e})") from None
        _check(Q.lib().seedq_kv_attend(self._ref, a, _stream(stream, dev)), "seedq_kv_attend")


def score_workspace(n_rows: int, vocab: int, device="cuda"):
    """A zeroed workspace for token_logprobs over that many rows or fewer."""
    return torch.zeros(Q.lib().seedq_token_logprobs_workspace_bytes(n_rows, vocab), dtype=torch.uint8, device=device)


def token_logprobs(logits, targets, logprob, entropy, rank, top_logprob, top_index, workspace, scale: float = 1.0,
                   stream=None):
    """seedq_token_logprobs: logits (n, vocab), targets (n,) int64 or None;
    logprob, entropy (n,) float32, rank (n,) int32, top_logprob (n, k) float32
    and top_index (n, k) int32 are written.  Each of them may be None (logprob
    and rank only without targets, the two top tensors only together)."""
    dt, st = DTYPES.get(logits.dtype), logits.stride()
    if len(st) != 2 or dt is None or (st[1] != 1 and logits.shape[1] != 1) or not logits.is_cuda:
        raise ValueError("logits: (rows, vocab) float32, bfloat16 or float16 with contiguous rows on a CUDA device is wanted")
    (n, vocab), dev = logits.shape, logits.device
    pt = pl = pe = pr = px = pi = None
    if targets is not None:
        if logprob is None or rank is None:
            raise ValueError("logprob and rank: wanted beside targets")
        _ints(targets, n, torch.int64, dev, "targets")
        pt = targets.data_ptr()
    if logprob is not None:
        _ints(logprob, n, torch.float32, dev, "logprob")
        pl = logprob.data_ptr()
    if entropy is not None:
        _ints(entropy, n, torch.float32, dev, "entropy")
        pe = entropy.data_ptr()
    if rank is not None:
        _ints(rank, n, torch.int32, dev, "rank")
        pr = rank.data_ptr()
    k = 0
    if top_index is not None or top_logprob is not None:
        if top_index is None or top_logprob is None:
            raise ValueError("top_logprob and top_index: wanted together")
        k = top_index.shape[-1]
        if not (top_logprob.dtype is torch.float32 and top_index.dtype is torch.int32
                and top_logprob.shape == top_index.shape == (n, k) and top_logprob.is_contiguous()
                and top_index.is_contiguous() and top_logprob.device == dev and top_index.device == dev):
            raise ValueError(f"top_logprob, top_index: contiguous float32 and int32 ({n}, k) on {dev} are wanted")
        px, pi = top_logprob.data_ptr(), top_index.data_ptr()
    if not workspace.is_contiguous() or workspace.device != dev:
        raise ValueError("workspace: a tensor of score_workspace is wanted")
    _check(Q.lib().seedq_token_logprobs(
        logits.data_ptr(), dt, n, vocab, st[0] if n > 1 else vocab, scale, pt, pl, pe, pr, k, px, pi, workspace.data_ptr(),
        workspace.nbytes, _stream(stream, dev)), "seedq_token_logprobs")
