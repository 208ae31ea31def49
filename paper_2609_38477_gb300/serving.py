"""Python binding of the serving calls of libseedq.so: page bookkeeping, the
8-bit key/value cache, the attention that reads it, rotary positions, token log
probabilities, and beam search's choice with the pages of the chosen beams.

Like the rest of the binding it marshals arguments and computes nothing: every
buffer is the caller's torch tensor, every length and page number stays on the
device, and calls only enqueue work on the given stream (torch's current stream
by default).  The tensors' device must be the current one.  What the C ABI
cannot see (shapes, types, devices) is checked here and raises ValueError; what it
refuses itself raises SeedQError.
"""
from __future__ import annotations

import ctypes as C
import math
import struct
from fractions import Fraction

import torch

from . import seedq as Q

DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
KINDS = {"int8": 0, "e4m3": 1}
LAYOUTS = {"half": 0, "pairs": 1}
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

    def append_rotary(self, k, v, slots, rotary, cos_sin, q=None, q_out=None, stream=None):
        """seedq_kv_append_rotary: k (n_tokens, n_kv_heads, head_dim) rotated as
        by rotary.rotate, then written with v at slots; q (n_tokens, n_heads,
        head_dim) of k's type, if given, is rotated to q_out, by the same launch
        or, many of them, by one before it.  q_out may be q, and lies on no other
        input."""
        n, dt, st = self._pair(k, v, slots)
        rotary._want_angles(cos_sin, n, self.device)
        heads, ot, qs, os, qp, op = 0, dt, (0, 0), (0, 0), 0, 0
        if q is not None:
            shape = q.shape
            if q_out is None or q.dtype is not k.dtype or len(shape) != 3 or shape[0] != n or shape[2] != self.head_dim or q.device != self.device:
                raise ValueError(f"q: ({n}, n_heads, {self.head_dim}) of the type and device of k, and q_out beside it are wanted")
            heads = shape[1]
            _, qs, ot, os = _turned_rows(q, q_out, "q_out")
            qp, op = q.data_ptr(), q_out.data_ptr()
        elif q_out is not None:
            raise ValueError("q_out: wanted beside q alone")
        a = Q.APPEND_ROTARY_ARGS.pack(cos_sin.data_ptr(), rotary.rot_dim, rotary.layout, heads, ot, qp, qs[0], qs[1], op, os[0], os[1])
        _check(Q.lib().seedq_kv_append_rotary(self._ref, k.data_ptr(), v.data_ptr(), dt, st[0], st[1], slots.data_ptr(), n, a,
                                              _stream(stream, self.device)), "seedq_kv_append_rotary")

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


def _turned_rows(x, out, name: str):
    """Types and strides of (tokens, heads, dim) rows and of those that they are rotated to, which must not lie on one another."""
    shape, xt, ot, xs, os = x.shape, DTYPES.get(x.dtype), DTYPES.get(out.dtype), x.stride(), out.stride()
    if (xt is None or ot is None or len(shape) != 3 or out.shape != shape or xs[2] != 1 or os[2] != 1 or out.device != x.device
            or not ((os[1] >= shape[2] or shape[1] < 2) and (os[0] >= os[1] * (shape[1] - 1) + shape[2] or shape[0] < 2))
            and not ((os[0] >= shape[2] or shape[0] < 2) and (os[1] >= os[0] * (shape[0] - 1) + shape[2] or shape[1] < 2))):
        raise ValueError(f"{name}: (tokens, heads, dim) float32, bfloat16 or float16 in and out, of one shape and device, with contiguous "
                         f"last dimension and no rows of {name} on one another are wanted, got {tuple(shape)} {x.dtype} and {tuple(out.shape)} {out.dtype}")
    return xt, xs, ot, os


def rotary_frequencies(rot_dim: int, base: float = 10000.0, rule: str = "none", factor: float = 1.0, original: int = 8192,
                       low: float = 1.0, high: float = 4.0):
    """(frequencies, scale) for Rotary: radians per position of the rot_dim / 2
    pairs, w_i = base^(-2 i / rot_dim), and the factor of cos and sin, for contexts
    `factor` times as long as the `original` ones:
      "none"    w_i
      "linear"  w_i / factor
      "base"    w_i of base * factor^(rot_dim / (rot_dim - 2)): the slowest pair is
                stretched by factor, the fastest not at all
      "bands"   by the turns t that a pair makes over the original context: w_i where
                t >= high, w_i / factor where t <= low, between them both, mixed in
                proportion to t
      "ramp"    the same, mixed in proportion to the pair's number between the
                (whole) numbers at which pairs make high and low turns (32 and 1
                are usual); scale 1 + 0.1 ln factor"""
    _want(rot_dim >= 2 and rot_dim % 2 == 0, f"rot_dim: an even number is wanted, got {rot_dim}")
    _want(base > 1 and factor >= 1 and original >= 1 and 0 < low < high, "base > 1, factor >= 1, original >= 1, 0 < low < high are wanted")
    half, scale = rot_dim // 2, 1.0
    if rule == "base" and half > 1:
        base = base * factor ** (rot_dim / (rot_dim - 2))
    w = [base ** (-2.0 * i / rot_dim) for i in range(half)]
    if rule == "linear":
        keep = [0.0] * half
    elif rule == "bands":
        keep = [min(max((original * x / (2 * math.pi) - low) / (high - low), 0.0), 1.0) for x in w]
    elif rule == "ramp":
        at = lambda turns: rot_dim * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        first, last = max(math.floor(at(high)), 0), min(math.ceil(at(low)), rot_dim - 1)
        keep = [1.0 - min(max((i - first) / max(last - first, 0.001), 0.0), 1.0) for i in range(half)]
        scale = 1.0 + 0.1 * math.log(factor)
    else:
        _want(rule in ("none", "base"), f"rule: none, linear, base, bands or ramp is wanted, got {rule!r}")
        keep = [1.0] * half
    return [x * k + x / factor * (1.0 - k) if k < 1.0 else x for x, k in zip(w, keep)], scale


_TWO_PI = Fraction(6283185307179586476925286766559005768394, 10 ** 39)


class Rotary:
    """Rotary positions of one kind (see seedq_rotary_angles and seedq_rotate).

    frequencies: radians per position of each pair (rot_dim / 2 numbers, as
    rotary_frequencies gives them).  layout: "half" (numbers i and i + rot_dim / 2
    of a head are a pair) or "pairs" (2i and 2i + 1).  scale: factor of cos and
    sin.  Keeps the frequencies on the device in whole parts of a turn."""

    def __init__(self, frequencies, layout: str = "half", scale: float = 1.0, device="cuda"):
        _want(layout in LAYOUTS, f"layout: one of {sorted(LAYOUTS)} is wanted, got {layout!r}")
        w = [float(x) for x in frequencies]
        _want(w and all(math.isfinite(x) for x in w), "frequencies: one or more finite numbers are wanted")
        self.half, self.rot_dim, self.layout, self.scale = len(w), 2 * len(w), LAYOUTS[layout], float(scale)
        whole = [round(Fraction(x) / _TWO_PI * 2 ** 64) % 2 ** 64 for x in w]
        self.turns = torch.tensor([x - 2 ** 64 if x >= 2 ** 63 else x for x in whole], dtype=torch.int64, device=device)
        self.device = self.turns.device

    def _want_angles(self, cos_sin, n, device):
        if not (cos_sin.dtype is torch.float32 and cos_sin.shape == (n, self.half, 2) and cos_sin.is_contiguous()
                and cos_sin.device == device):
            raise ValueError(f"cos_sin: contiguous float32 ({n}, {self.half}, 2) on {device} is wanted")

    def angles(self, positions, cos_sin, stream=None):
        """seedq_rotary_angles: cos_sin (n_tokens, rot_dim / 2, 2) float32 of
        positions (int32, at least n_tokens)."""
        n = cos_sin.shape[0]
        self._want_angles(cos_sin, n, self.device)
        _ints(positions, n, torch.int32, self.device, "positions")
        _check(Q.lib().seedq_rotary_angles(self.turns.data_ptr(), self.half, self.scale, positions.data_ptr(), n, cos_sin.data_ptr(),
                                           _stream(stream, self.device)), "seedq_rotary_angles")

    def rotate(self, x, cos_sin, out, stream=None):
        """seedq_rotate: x, out (n_tokens, n_heads, head_dim); out may be x, or lies on no row of it."""
        xt, xs, ot, os = _turned_rows(x, out, "out")
        n, heads, dim = x.shape
        self._want_angles(cos_sin, n, x.device)
        _check(Q.lib().seedq_rotate(x.data_ptr(), xt, xs[0], xs[1], n, heads, dim, self.rot_dim, self.layout, cos_sin.data_ptr(),
                                    out.data_ptr(), ot, os[0], os[1], _stream(stream, x.device)), "seedq_rotate")


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


def beam_workspace(n_groups: int, n_beams: int, vocab: int, device="cuda"):
    """A zeroed workspace for beam_select over that many rows and tokens or fewer."""
    n = Q.lib().seedq_beam_select_workspace_bytes(n_groups, n_beams, vocab)
    _want(n > 0, "beam_workspace: 1..32 beams, up to 8192 rows and a vocabulary of up to 2^27 are wanted")
    return torch.zeros(n, dtype=torch.uint8, device=device)


def _beams(t, name, dtype, shape, device):
    if not (t.dtype in dtype and t.shape == shape and t.is_contiguous() and t.device == device):
        raise ValueError(f"{name}: contiguous {' or '.join(map(str, dtype))} {tuple(shape)} on {device} is wanted")
    return t.data_ptr()


_F32, _I32, _BYTES = (torch.float32,), (torch.int32,), (torch.bool, torch.uint8)


def beam_select(logits, scores, out_score, out_beam, out_token, workspace, scale: float = 1.0, done=None, end_token: int = -1,
                weights=None, stream=None):
    """seedq_beam_select: logits (n_groups * n_beams, vocab); scores, done (bool or
    uint8, or None) and weights (or None) (n_groups, n_beams); out_score,
    out_beam and out_token (n_groups, n_out) are written."""
    dt, st = DTYPES.get(logits.dtype), logits.stride()
    if len(st) != 2 or dt is None or (st[1] != 1 and logits.shape[1] != 1) or not logits.is_cuda:
        raise ValueError("logits: (rows, vocab) float32, bfloat16 or float16 with contiguous rows on a CUDA device is wanted")
    if scores.ndim != 2 or out_score.ndim != 2:
        raise ValueError("scores, out_score: (n_groups, n_beams) and (n_groups, n_out) are wanted")
    (rows, vocab), (groups, beams), n_out, dev = logits.shape, scores.shape, out_score.shape[1], logits.device
    if rows != groups * beams:
        raise ValueError(f"logits: a row for each of {groups} x {beams} beams is wanted, got {rows}")
    shape, out = (groups, beams), (groups, n_out)
    if not workspace.is_contiguous() or workspace.device != dev:
        raise ValueError("workspace: a tensor of beam_workspace is wanted")
    try:
        a = Q.BEAM_SELECT_ARGS.pack(
            logits.data_ptr(), st[0] if rows > 1 else vocab, dt, beams, groups, vocab, scale, end_token,
            _beams(scores, "scores", _F32, shape, dev), 0 if done is None else _beams(done, "done", _BYTES, shape, dev),
            0 if weights is None else _beams(weights, "weights", _F32, shape, dev), n_out,
            _beams(out_score, "out_score", _F32, out, dev), _beams(out_beam, "out_beam", _I32, out, dev),
            _beams(out_token, "out_token", _I32, out, dev), workspace.data_ptr(), workspace.nbytes)
    except struct.error as e:
        raise ValueError(f"end_token: a 32-bit integer, scale: a number are wanted ({e})") from None
    _check(Q.lib().seedq_beam_select(a, _stream(stream, dev)), "seedq_beam_select")


class BeamPages:
    """The outputs of seedq_beam_reorder for n_groups requests of n_beams beams
    over the caches of all layers (KVCache, alike but for their tensors):
    seq_lens, status (per row) and free_count.  Allocated once, so a captured
    graph keeps its addresses."""

    def __init__(self, caches, n_groups: int, n_beams: int):
        caches = list(caches)
        _want(caches and all(isinstance(c, KVCache) and c.device == caches[0].device for c in caches),
              "caches: KVCache objects of one device are wanted")
        self.caches, self.n_groups, self.n_beams, self.device = caches, int(n_groups), int(n_beams), caches[0].device
        n = Q.lib().seedq_beam_reorder_workspace_bytes(self.n_groups, self.n_beams)
        _want(n > 0, "n_groups, n_beams: 1..32 beams and 1..8192 rows are wanted")
        self.descs = (Q.KvCacheDesc * len(caches))(*(c.desc for c in caches))
        self.rows = self.n_groups * self.n_beams
        ints = torch.zeros(2 * self.rows + 1, dtype=torch.int32, device=self.device)
        self.seq_lens, self.status, self.free_count = ints.split([self.rows, self.rows, 1])
        self.workspace = torch.zeros(n, dtype=torch.uint8, device=self.device)

    def reorder(self, parents, seq_lens, block_table, free_pages, free_count, out=None, stream=None):
        """seedq_beam_reorder: parents (n_groups, n_beams) int32, seq_lens int32 of
        at least as many rows (this object's own after a first call); block_table changes in place, or out (the same
        shape) gets the new one; free_pages changes in place."""
        n, dev = self.rows, self.device
        _ints(seq_lens, n, torch.int32, dev, "seq_lens")
        _ints(free_pages, 0, torch.int32, dev, "free_pages")
        _ints(free_count, 1, torch.int32, dev, "free_count")
        _table(block_table, n, dev)
        to = block_table if out is None else out
        if out is not None:
            _table(out, n, dev)
            if out.shape[1] != block_table.shape[1]:
                raise ValueError("out: as wide as block_table is wanted")
        if n > 1 and to.stride(0) < to.shape[1]:
            raise ValueError("out: rows that overlap")
        a = Q.BEAM_REORDER_ARGS.pack(
            self.n_groups, self.n_beams, _beams(parents, "parents", _I32, (self.n_groups, self.n_beams), dev), seq_lens.data_ptr(),
            block_table.data_ptr(), _row_stride(block_table), to.data_ptr(), _row_stride(to), block_table.shape[1],
            free_pages.shape[0], free_pages.data_ptr(), free_count.data_ptr(), self.seq_lens.data_ptr(), self.status.data_ptr(),
            self.free_count.data_ptr(), self.workspace.data_ptr(), self.workspace.nbytes)
        _check(Q.lib().seedq_beam_reorder(self.descs, len(self.caches), a, _stream(stream, dev)), "seedq_beam_reorder")
