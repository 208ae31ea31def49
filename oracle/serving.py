"""CPU oracle of the serving calls (numpy, fp64); test infrastructure only.

Page bookkeeping, the 8-bit cache's append and gather, attention over it, and
token log probabilities, each written from its definition in include/seedq.h
and sharing nothing with the CUDA library.
"""
import numpy as np

OK, NO_PAGES, BAD, NO_ROOM = 0, 1, 2, 3


def cdiv(a, b):
    return -(-a // b)


def batch_plan(seq_lens, n_new, table, free_pages, free_count, page, max_tokens):
    """Returns (table, free_pages, slots, positions, requests, seq_lens, starts, status, free_count)."""
    table, free = np.array(table, np.int32), np.array(free_pages, np.int32)
    n, width = len(n_new), table.shape[1]
    count = min(max(int(free_count), 0), free.size)
    lens, new = [int(x) for x in seq_lens], [int(x) for x in n_new]
    starts = [0]
    for x in new:
        starts.append(starts[-1] + max(x, 0))
    status = [OK] * n
    for i in range(n):
        total = lens[i] + max(new[i], 0)
        if new[i] < -1 or lens[i] < 0 or total >= 2 ** 31 or cdiv(total, page) > width:
            status[i] = BAD
        elif new[i] >= 0 and starts[i + 1] > max_tokens:
            status[i] = NO_ROOM
    back, top = 0, count
    for i in range(n):
        if status[i] == OK and new[i] == -1:
            h = cdiv(lens[i], page)
            back += h
            if count + back > free.size:
                status[i] = NO_ROOM
            else:
                free[top:top + h] = table[i, :h]
                top += h
    stack = free.copy()
    need, left = 0, top
    for i in range(n):
        if status[i] == OK and new[i] >= 0:
            a, b = cdiv(lens[i], page), cdiv(lens[i] + new[i], page)
            need += b - a
            if b > a and need > top:
                status[i] = NO_PAGES
            elif b > a:
                table[i, a:b] = [stack[top - 1 - (need - (b - a)) - c] for c in range(b - a)]
                left -= b - a
    slots, pos, req = np.full(max_tokens, -1, np.int64), np.zeros(max_tokens, np.int32), np.full(max_tokens, -1, np.int32)
    for i in range(n):
        for d in range(max(new[i], 0)):
            t = starts[i] + d
            if t >= max_tokens:
                break
            p = min(lens[i] + d, 2 ** 31 - 1)
            pos[t], req[t] = p, i
            if status[i] == OK:
                slots[t] = int(table[i, p // page]) * page + p % page
    out = [0 if status[i] == OK and new[i] == -1 else lens[i] + new[i] if status[i] == OK else lens[i] for i in range(n)]
    clip = np.minimum(np.array(starts, np.int64), max_tokens).astype(np.int32)
    return table, free, slots, pos, req, np.array(out, np.int32), clip, np.array(status, np.int32), np.int32(left)


# ---------------------------------------------------------------- the cache

LIMIT = {"int8": 127.0, "e4m3": 448.0}


def e4m3_table():
    """The 256 numbers of the E4M3 codes (sign, 4 exponent bits of bias 7, 3
    fraction bits; all of both set is NaN)."""
    v = np.zeros(256)
    for c in range(256):
        e, f = (c >> 3) & 15, c & 7
        m = np.nan if c & 127 == 127 else f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7)
        v[c] = -m if c >> 7 else m
    return v


_E4M3 = e4m3_table()


def decode(codes, kind):
    u = np.asarray(codes).view(np.uint8)
    return u.view(np.int8).astype(np.float64) if kind == "int8" else _E4M3[u]


def encode(x, kind):
    """Nearest code, ties to even, of |x| within the kind's range (uint8 bits)."""
    x = np.asarray(x, np.float64)
    if kind == "int8":
        return np.clip(np.rint(x), -127, 127).astype(np.int8).view(np.uint8)
    pos = _E4M3[:127]  # 0 .. 448, ascending with the code
    a = np.minimum(np.abs(x), 448.0)
    lo = np.clip(np.searchsorted(pos, a, side="right") - 1, 0, 125)
    mid = (pos[lo] + pos[lo + 1]) / 2
    up = (a > mid) | ((a == mid) & (lo % 2 == 1))
    return ((lo + up) | (np.signbit(x) << 7)).astype(np.uint8)


def block_scale(amax, kind):
    """Smallest power of two s >= 2^-126 with amax <= limit s; 0 for 0, NaN for what is not finite."""
    if not np.isfinite(amax):
        return np.nan
    if amax == 0:
        return 0.0
    e = -126
    while LIMIT[kind] * 2.0 ** e < amax:
        e += 1
    return 2.0 ** e


def append(codes, scales, new, slots, page, kind):
    """codes: (pages, heads, page, dim) uint8 and scales (pages, heads) float64, changed in place."""
    slots = [int(s) for s in slots]
    n_pages, heads = scales.shape
    t = 0
    while t < len(slots):
        b = slots[t] // page if slots[t] >= 0 else -1
        if b < 0 or b >= n_pages:
            t += 1
            continue
        m = 1
        while t + m < len(slots) and slots[t + m] == slots[t] + m and slots[t + m] // page == b:
            m += 1
        off = slots[t] % page
        for h in range(heads):
            x = new[t:t + m, h].astype(np.float64)
            a = np.abs(x).max()
            want = block_scale(a, kind)
            now = want
            if off > 0:
                old = scales[b, h]
                now = want if np.isnan(want) or want > old else old
                if now > old:
                    codes[b, h, :off] = encode(decode(codes[b, h, :off], kind) * (old / now), kind)
            codes[b, h, off:off + m] = encode(x / now, kind) if now > 0 else 0
            scales[b, h] = now
        t += m


def gather(codes, scales, slots, page, kind):
    out = np.zeros((len(slots), codes.shape[1], codes.shape[3]))
    for i, s in enumerate(int(s) for s in slots):
        b = s // page if s >= 0 else -1
        if 0 <= b < codes.shape[0]:
            out[i] = decode(codes[b, :, s % page], kind) * scales[b][:, None]
    return out


def attend(q, kc, vc, ks, vs, seq_lens, starts, table, page, kind, scale, window=0):
    """(out, lse, spread, reach) in fp64: spread = the largest scale * sum |q_d k_d|
    and reach = the largest |v| among a query's visible keys, for error bounds."""
    n, hq, d = q.shape
    h = kc.shape[1]
    out, lse = np.zeros((n, hq, d)), np.full((n, hq), -np.inf)
    spread, reach = np.zeros((n, hq)), np.zeros((n, hq))
    for i in range(len(seq_lens)):
        fresh = int(starts[i + 1]) - int(starts[i])
        for t in range(fresh):
            row = int(starts[i]) + t
            p = int(seq_lens[i]) - fresh + t
            lo = max(0, p - window + 1) if window else 0
            keys = np.arange(lo, min(p + 1, table.shape[1] * page))
            if keys.size:
                keys = keys[(table[i, keys // page] >= 0) & (table[i, keys // page] < kc.shape[0])]
            if not keys.size:
                continue
            b, o = table[i, keys // page], keys % page
            k = decode(kc[b, :, o], kind) * ks[b][:, :, None]
            v = decode(vc[b, :, o], kind) * vs[b][:, :, None]
            for g in range(hq):
                kv = g // (hq // h)
                x = q[row, g].astype(np.float64)
                z = scale * (k[:, kv] @ x)
                m = z.max()
                e = np.exp(z - m)
                out[row, g] = e @ v[:, kv] / e.sum()
                lse[row, g] = m + np.log(e.sum())
                spread[row, g] = abs(scale) * (np.abs(k[:, kv]) @ np.abs(x)).max()
                reach[row, g] = np.abs(v[:, kv]).max()
    return out, lse, spread, reach


# ---------------------------------------------------------------- log probabilities

def token_logprobs(x, targets, scale, top_k):
    """x: (rows, vocab) numbers as float64.  Returns (logprob, entropy, rank, top_logprob, top_index)."""
    n, v = x.shape
    lp, en, rk = np.zeros(n), np.zeros(n), np.full(n, -1, np.int32)
    tl, ti = np.full((n, top_k), -np.inf), np.full((n, top_k), -1, np.int32)
    for r in range(n):
        row = np.where(x[r] == 0, 0.0, x[r])
        nan, inf = np.isnan(row), np.isposinf(row)
        order = sorted(range(v), key=lambda i: (0 if nan[i] else 1, 0.0 if nan[i] else -row[i], i))
        place = {c: i for i, c in enumerate(order)}
        z = scale * row
        if nan.any() or inf.any():
            logp, en[r] = np.full(v, np.nan), np.nan
        elif np.isneginf(z).all():
            logp = z
        else:
            m = z.max()
            logp = z - m - np.log(np.exp(z - m).sum())
            p = np.exp(logp)
            en[r] = -(p[p > 0] * logp[p > 0]).sum()
        t = -1 if targets is None else int(targets[r])
        if 0 <= t < v:
            lp[r], rk[r] = logp[t], -1 if nan.any() else place[t]
        elif t != -1:
            lp[r] = np.nan
        for k, c in enumerate(order[:top_k]):
            tl[r, k], ti[r, k] = logp[c], c
    return lp, en, rk, tl, ti
