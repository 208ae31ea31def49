"""The serving calls on the GPU against the fp64 oracle.

Whole numbers (plans, codes, scales, ranks, indices) compare exactly.
Tolerances, with u = 2^-24:

Attention.  A score is a float32 sum of head_dim products of exact codes with
query values held to at least 2^-21 of the query's largest; the products may be
accumulated with truncation, at most 2^-23 of the partial sums per step and at
most 32 steps, so a score is off by at most 2^-18 A, A = the largest
scale * sum |q_d k_d| (the oracle's `spread`).  exp turns that into a relative
error of each weight, so outputs move by at most 2 * 2^-18 A max|v|; the weights
and sums add at most 2^-16 max|v| (weights held to 2^-21, float32 sums of a few
hundred terms per worker, a handful of joins).  Rounding to the output's type is
monotonic, so the output lies between the rounded ends of that interval.

Log probabilities.  All terms of sum exp are positive and each thread adds at
most vocab / 128 + 64 of them in order, so its relative error is at most
(vocab / 128 + 64 + 8) u, and that is the error of its logarithm; the rounding
of scale * x and of the differences adds 4 u (|z_t| + |max|) + 4 u.  The entropy's
second sum is off by the same factor of sum |d| e^d / sum e^d.
"""
import os
import random
import sys

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)
sys.path.insert(0, os.path.join(ROOT, "oracle"))

import serving as S  # noqa: E402

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def V():
    from paper_2609_38477_gb300 import build

    build.build()
    from paper_2609_38477_gb300 import seedq, serving

    seedq.lib()
    return serving


def dev(x, dtype=None):
    return torch.as_tensor(np.ascontiguousarray(x), dtype=dtype).cuda()


# ---------------------------------------------------------------- plan

def run_plan(V, seq, new, table, free, count, page, max_tokens):
    p = V.BatchPlan(len(new), max_tokens)
    t, f = dev(table), dev(free)
    for _ in range(2):  # the same inputs again: nothing an earlier call left behind matters
        p.build(dev(seq, torch.int32), dev(new, torch.int32), t, f, dev([count], torch.int32), page)
    want = S.batch_plan(seq, new, table, free, count, page, max_tokens)
    got = [t, f, p.slots, p.positions, p.requests, p.seq_lens, p.starts, p.status, p.free_count[0]]
    for g, w, name in zip(got, want, "table free slots positions requests seq_lens starts status left".split()):
        assert np.array_equal(g.cpu().numpy(), w), name
    return want


def pool(rng, seq, page, width, spare, extra=0):
    held = [S.cdiv(max(x, 0), page) if S.cdiv(max(x, 0), page) <= width else 0 for x in seq]
    ids = rng.permutation(sum(held) + spare + 3).astype(np.int32)
    table = np.full((len(seq), width), -1, np.int32)
    at = 0
    for i, h in enumerate(held):
        table[i, :h] = ids[at:at + h]
        at += h
    free = np.full(sum(held) + spare + extra, -1, np.int32)
    free[:spare] = ids[at:at + spare]
    return table, free


@pytest.mark.parametrize("n,page,most,new,spare", [
    (1, 16, 1, 1, 4), (1, 16, 100, 40, 0), (5, 1, 9, 4, 30), (33, 16, 70, 30, 40), (33, 48, 400, 100, 2), (513, 32, 90, 3, 200),
    (1000, 16, 300, 60, 3000), (8192, 64, 200, 2, 9000)])
def test_plan(V, n, page, most, new, spare):
    rng = np.random.RandomState(n + page)
    seq = rng.randint(0, most + 1, n)
    fresh = rng.randint(-1, new + 1, n)
    width = S.cdiv(most + new, page)
    table, free = pool(rng, seq, page, width, spare)
    total = int(np.maximum(fresh, 0).sum())
    run_plan(V, seq, fresh, table, free, spare, page, total + 5)


def test_plan_bad_requests_and_short_buffers(V):
    rng = np.random.RandomState(3)
    big = 2 ** 31 - 1
    seq = np.array([5, -3, 17, 40, 0, 900, big, big, 31, 16, 12])
    new = np.array([3, 2, -7, 9, -1, 1, 1, -1, 1, -1, 0])
    table, free = pool(rng, seq, 16, 4, 6)
    for tokens in (1, 4, 8, 13, 14, 40):  # from too few for the first request to enough for all
        w = run_plan(V, seq, new, table, free, 6, 16, tokens)
    assert w[7].tolist() == [0, 2, 2, 0, 0, 2, 2, 2, 0, 0, 0]
    run_plan(V, np.array([1, 2]), np.array([big, big]), table[:2], free, 6, 16, 50)  # sums past 32 bits


@pytest.mark.parametrize("count", [-5, 0, 2, 6, 7, 10 ** 9])
def test_plan_returned_pages_that_do_not_fit(V, count):
    rng = np.random.RandomState(4)
    seq = np.array([30, 64, 3, 20, 16])
    new = np.array([-1, -1, 20, -1, 17])
    table, free = pool(rng, seq, 16, 4, 0)
    free = np.arange(100, 107, dtype=np.int32)
    run_plan(V, seq, new, table, free, count, 16, 64)


def test_plan_wide_strided_table(V):
    rng = np.random.RandomState(5)
    seq, new = rng.randint(0, 50, 9), rng.randint(0, 20, 9)
    table, free = pool(rng, seq, 16, 5, 40)
    wide = torch.full((9, 11), -9, dtype=torch.int32, device="cuda")
    wide[:, :5] = dev(table)
    p = V.BatchPlan(9, 300)
    p.build(dev(seq, torch.int32), dev(new, torch.int32), wide[:, :5], dev(free), dev([40], torch.int32), 16)
    want = S.batch_plan(seq, new, table, free, 40, 16, 300)
    assert np.array_equal(wide[:, :5].cpu().numpy(), want[0]) and bool((wide[:, 5:] == -9).all())
    assert np.array_equal(p.slots.cpu().numpy(), want[2])


# ---------------------------------------------------------------- cache

def new_cache(V, pages, heads, page, dim, kind, order="head", fill=None):
    shape = (pages, heads, page, dim) if order == "head" else (pages, page, heads, dim)
    t = []
    for i in range(2):
        c = torch.full(shape, 0x55, dtype=torch.uint8, device="cuda")
        t.append(c if order == "head" else c.transpose(1, 2))
    ks, vs = (torch.full((pages, heads), 77.0, device="cuda") for _ in range(2))
    return V.KVCache(t[0], t[1], ks, vs, kind)


def codes_of(c):
    return [x.contiguous().cpu().numpy().view(np.uint8).copy() for x in (c.k, c.v)], [x.double().cpu().numpy().copy()
                                                                                     for x in (c.k_scale, c.v_scale)]


def same_cache(c, codes, scales, what=""):
    got, gs = codes_of(c)
    for a, b, x, y in zip(got, codes, gs, scales):
        assert np.array_equal(x, y, equal_nan=True), what
        assert np.array_equal(a, b), what


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("heads,page,dim,order", [(1, 16, 16, "head"), (3, 32, 80, "token"), (8, 16, 128, "head"),
                                                  (2, 256, 64, "token"), (5, 48, 256, "head")])
def test_append_in_steps(V, kind, dtype, heads, page, dim, order):
    """Runs of every length and offset, in an order that reuses pages, each step exact; then the gather."""
    rng = np.random.RandomState(heads * page + dim)
    c = new_cache(V, 6, heads, page, dim, kind, order)
    codes, scales = codes_of(c)
    at = {}
    for step in range(9):
        slots = []
        for b in rng.permutation(6)[:rng.randint(1, 6)]:
            o = at.get(b, 0)
            if o >= page or rng.rand() < 0.2:
                o = 0  # a reused page
            m = min(page - o, int(rng.choice([1, 2, 3, 15, 16, 17, page])))
            slots += list(range(b * page + o, b * page + o + m))
            at[b] = o + m
            if rng.rand() < 0.3:
                slots.append(int(rng.choice([-1, 6 * page, 2 ** 40, -2 ** 40])))
        n = len(slots)
        size = 2.0 ** rng.randint(-9, 9, (2, n, 1, 1))
        x = torch.from_numpy((size * rng.randn(2, n, heads, dim)).astype(np.float32)).to(DT[dtype])
        c.append(x[0].cuda(), x[1].cuda(), dev(slots, torch.int64))
        for i in range(2):
            S.append(codes[i], scales[i], x[i].float().numpy(), slots, page, kind)
        same_cache(c, codes, scales, step)
    read = np.concatenate([rng.permutation(6 * page)[:50], [-1, 6 * page, 2 ** 50]])
    k, v = (torch.full((read.size, heads, dim), 9.0, dtype=DT[dtype], device="cuda") for _ in range(2))
    c.gather(dev(read, torch.int64), k, v)
    for i, t in enumerate((k, v)):
        want = torch.from_numpy(S.gather(codes[i], scales[i], read, page, kind)).to(DT[dtype])
        assert torch.equal(t.cpu(), want)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_append_extremes(V, kind):
    """Zeros, the smallest and largest numbers, infinities and NaN, alone and joining a page that holds tokens."""
    f = np.float32
    rows = [f(0), f(1e-45), f(1e-39), f(1.1754944e-38), f(3.4028235e38), f(127), np.nextafter(f(127), f(200)), f(448),
            np.nextafter(f(448), f(500)), f(-0.0), f(np.inf), f(-np.inf), f(np.nan)]
    D, P = 16, 16
    for first in (None, f(0), f(3.0), f(np.nan)):
        c = new_cache(V, len(rows), 1, P, D, kind)
        codes, scales = codes_of(c)
        off = 0
        if first is not None:
            slots = [b * P for b in range(len(rows))]
            x = np.full((len(rows), 1, D), first)
            c.append(dev(x), dev(x), dev(slots, torch.int64))
            for i in range(2):
                S.append(codes[i], scales[i], x, slots, P, kind)
            same_cache(c, codes, scales, first)
            off = 1
        x = np.zeros((len(rows), 1, D), f)
        x[:, 0, 5] = rows
        x[:, 0, 6] = [-r if np.isfinite(r) else f(1) for r in rows]
        slots = [b * P + off for b in range(len(rows))]
        c.append(dev(x), dev(x), dev(slots, torch.int64))
        for i in range(2):
            S.append(codes[i], scales[i], x, slots, P, kind)
        same_cache(c, codes, scales, first)


def test_append_strides_and_alignment(V):
    """Keys and values as slices of one projection's output, at an odd element offset, heads before tokens."""
    n, h, d, P = 7, 3, 48, 16
    rng = np.random.RandomState(8)
    for dtype in DT.values():
        flat = torch.from_numpy(rng.randn(n * (2 * h * d + 5) + 1).astype(np.float32)).to(dtype).cuda()
        rows = flat[1:].view(n, -1)
        k, v = rows[:, :h * d].view(n, h, d), rows[:, h * d:2 * h * d].view(n, h, d)
        slots = [3, 4, 5, 20, 21, 32, 47]
        c = new_cache(V, 3, h, P, d, "int8")
        codes, scales = codes_of(c)
        c.append(k, v, dev(slots, torch.int64))
        for i, t in enumerate((k, v)):
            S.append(codes[i], scales[i], t.float().cpu().numpy(), slots, P, "int8")
        same_cache(c, codes, scales)
        kt, vt = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (k, v))
        c2 = new_cache(V, 3, h, P, d, "int8")
        c2.append(kt, vt, dev(slots, torch.int64))
        same_cache(c2, codes, scales)
        out = torch.zeros_like(flat)
        o = out[1:].view(n, -1)
        c.gather(dev(slots, torch.int64), o[:, :h * d].view(n, h, d), o[:, h * d:2 * h * d].view(n, h, d))
        want = torch.from_numpy(S.gather(codes[1], scales[1], slots, P, "int8")).to(dtype)
        assert torch.equal(o[:, h * d:2 * h * d].view(n, h, d).cpu(), want)
        assert bool((o[:, 2 * h * d:] == 0).all()) and out[0] == 0


def test_strides_of_single_entries(V):
    """One token's or one head's keys and values with unlike strides there, a table of one page, logits of one token."""
    for n, h in ((1, 4), (5, 1), (1, 1)):
        x = torch.randn(2, n, h, 64, device="cuda")
        k = x[0]
        v = torch.zeros(4096, device="cuda").as_strided((n, h, 64), [y if m > 1 else 777 for m, y in zip(k.shape, k.stride())])
        v.copy_(x[1])
        slots = torch.arange(n, device="cuda")
        a, b = (new_cache(V, 2, h, 16, 64, "int8") for _ in range(2))
        a.append(k, x[1], slots)
        b.append(k, v, slots)
        assert torch.equal(a.k[0, :, :n], b.k[0, :, :n]) and torch.equal(a.v[0, :, :n], b.v[0, :, :n])
        got = torch.zeros_like(k)
        v.zero_()
        b.gather(slots, got, v)
        for i, y in enumerate((got, v)):
            assert float((y - x[i]).abs().max()) < 0.05
    table = torch.zeros(6, dtype=torch.int32, device="cuda").as_strided((3, 1), (1, 7))
    table.fill_(-1)
    plan, seq = V.BatchPlan(3, 8), torch.zeros(3, dtype=torch.int32, device="cuda")
    plan.build(seq, dev([1, 2, 3], torch.int32), table, torch.arange(5, dtype=torch.int32, device="cuda"), dev([5], torch.int32), 16)
    assert table[:, 0].tolist() == [4, 3, 2] and plan.slots.tolist() == [64, 48, 49, 32, 33, 34, -1, -1]
    check_score(V, torch.randn(6, device="cuda").as_strided((3, 1), (1, 7)), [0, -1, 1], 1.0, 2)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("heads,page,dim", [(3, 256, 128), (5, 256, 16), (2, 144, 256), (1, 240, 96), (7, 128, 64)])
def test_append_long_runs(V, kind, dtype, heads, page, dim):
    """Runs longer than a warp keeps beside short ones of the same page, each step exact; odd offsets of the rows."""
    rng = np.random.RandomState(heads * page + dim)
    c = new_cache(V, 4, heads, page, dim, kind)
    codes, scales = codes_of(c)
    for step in range(5):
        slots = []
        for b in rng.permutation(4)[:3]:
            cuts = np.sort(rng.permutation(page + 1)[:6])
            for a, e in zip(cuts[::2], cuts[1::2]):  # three runs of the page, gaps between
                slots += list(range(b * page + a, b * page + e))
            if rng.rand() < 0.5:
                slots.append(-1)
        n = len(slots)
        size = 2.0 ** rng.randint(-9, 9, (2, n, 1, 1))
        x = torch.from_numpy((size * rng.randn(2, n, heads, dim)).astype(np.float32)).to(DT[dtype])
        odd = step % 2
        y = torch.zeros(2 * n * heads * dim + odd, dtype=DT[dtype], device="cuda")[odd:].view(2, n, heads, dim)
        y.copy_(x)
        c.append(y[0], y[1], dev(slots, torch.int64))
        for i in range(2):
            S.append(codes[i], scales[i], x[i].float().numpy(), slots, page, kind)
        same_cache(c, codes, scales, step)
        out = torch.full((2 * n * heads * dim + odd,), 9.0, dtype=DT[dtype], device="cuda")[odd:].view(2, n, heads, dim)
        c.gather(dev(slots, torch.int64), out[0], out[1])
        for i in range(2):
            want = torch.from_numpy(S.gather(codes[i], scales[i], slots, page, kind)).to(DT[dtype])
            assert torch.equal(out[i].cpu(), want)


# ---------------------------------------------------------------- attention

def fill_cache(c, seed, kind):
    g = torch.Generator("cuda").manual_seed(seed)
    for t in (c.k, c.v):
        x = torch.randn(t.shape, generator=g, device="cuda")
        if kind == "int8":
            t.copy_((x * 40).round().clamp(-127, 127).to(torch.int8).view(torch.uint8))
        else:
            t.copy_((x * 60).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
    for t in (c.k_scale, c.v_scale):
        t.copy_(torch.pow(2.0, torch.randint(-7, -3, t.shape, generator=g, device="cuda").float()))


def check_attend(V, c, kind, lens, fresh, hq, q_dtype, out_dtype, window=0, scale=None, max_new=None, table=None, seed=0,
                 q=None, pad=0, q_size=1.0):
    rng = np.random.RandomState(seed)
    P, D = c.page_size, c.head_dim
    starts = np.concatenate([[0], np.cumsum(fresh)]).astype(np.int32)
    n = int(starts[-1]) + pad
    if table is None:
        width = max(1, max(S.cdiv(x, P) for x in lens))
        table = np.full((len(lens), width), -1, np.int32)
        ids = rng.permutation(c.n_pages).astype(np.int32)
        at = 0
        for i, x in enumerate(lens):
            h = S.cdiv(x, P)
            table[i, :h] = ids[at:at + h]
            at += h
    if q is None:
        q = torch.from_numpy((q_size * rng.randn(n, hq, D)).astype(np.float32)).to(DT[q_dtype]).cuda()
    out = torch.full((n, hq, D), 7.0, dtype=DT[out_dtype], device="cuda")
    lse = torch.full((n, hq), 7.0, device="cuda")
    ws = c.attend_workspace(hq, max_new or max(max(fresh), 1))
    args = (dev(lens, torch.int32), dev(starts), dev(table), ws)
    kw = dict(max_new=max_new or max(max(fresh), 1), window=window, scale=scale)
    c.attend(q, out, *args, lse=lse, **kw)
    first = out.clone(), lse.clone()
    c.attend(q, out, *args, lse=lse, **kw)  # the workspace is left as it was found
    assert torch.equal(first[0].float().nan_to_num(-3), out.float().nan_to_num(-3))
    assert torch.equal(first[1].nan_to_num(-3), lse.nan_to_num(-3))
    (kc, vc), (ks, vs) = codes_of(c)
    s = float(np.float32(D ** -0.5 if scale is None else scale))
    o64, l64, spread, reach = S.attend(q.double().cpu().numpy(), kc, vc, ks, vs, lens, starts, table, P, kind, s, window)
    m = int(starts[-1])
    got, gl = out[:m].double().cpu().numpy(), lse[:m].double().cpu().numpy()
    o64, l64, spread, reach = o64[:m], l64[:m], spread[:m], reach[:m]
    none = np.isneginf(l64)
    assert np.array_equal(none, np.isneginf(gl)) and np.all(got[none] == 0)
    ok = ~none
    tol = ((2.0 ** -17 * spread + 2.0 ** -16) * reach)[:, :, None]
    lo, hi = (torch.from_numpy(x).to(DT[out_dtype]).double().numpy() for x in (o64 - tol, o64 + tol))
    assert np.all(((lo <= got) & (got <= hi))[ok]), np.max((np.abs(got - o64) / np.maximum(tol, 1e-300))[ok])
    ltol = 2.0 ** -18 * spread + 2.0 ** -18 * (1 + np.abs(np.where(none, 0, l64)))
    assert np.all(np.abs(gl[ok] - l64[ok]) <= ltol[ok])
    assert bool((out[m:] == 7).all()) and bool((lse[m:] == 7).all())
    return out, lse


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("hq,h,d", [(1, 1, 16), (5, 1, 32), (4, 2, 64), (6, 2, 80), (12, 4, 96), (8, 8, 128), (32, 4, 128),
                                    (4, 2, 208), (16, 2, 256), (24, 1, 64), (71, 1, 64), (33, 1, 128)])
def test_attend_heads(V, kind, hq, h, d):
    c = new_cache(V, 40, h, 16, d, kind)
    fill_cache(c, d + hq, kind)
    check_attend(V, c, kind, [1, 15, 16, 17, 33, 0, 130, 64], [1] * 8, hq, "f32", "f32", seed=hq)


@pytest.mark.parametrize("page,order", [(16, "token"), (32, "head"), (48, "token"), (80, "head"), (128, "token"), (256, "head")])
@pytest.mark.parametrize("q_dtype,out_dtype", [("f32", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("bf16", "bf16")])
def test_attend_pages_and_types(V, page, order, q_dtype, out_dtype):
    c = new_cache(V, 30, 2, page, 64, "int8", order)
    fill_cache(c, page, "int8")
    check_attend(V, c, "int8", [page * 3 + 5, 1, page, page + 1, 2 * page - 1], [1, 1, 2, 3, 16], 8, q_dtype, out_dtype, seed=page)


@pytest.mark.parametrize("window", [0, 1, 2, 16, 33, 1000])
@pytest.mark.parametrize("fresh", [[1, 1, 1, 1], [7, 0, 3, 16], [0, 40, 1, 0], [90, 5, 31, 2]])
def test_attend_windows_and_pieces(V, window, fresh):
    c = new_cache(V, 40, 2, 16, 64, "e4m3")
    fill_cache(c, window, "e4m3")
    lens = [max(x, f) for x, f in zip([200, 40, 31, 90], fresh)]
    check_attend(V, c, "e4m3", lens, fresh, 6, "f32", "f32", window=window, seed=window + sum(fresh), pad=3)


def test_attend_long_context_splits(V):
    """Contexts far longer than a worker's share, beside short ones: the joins across workers."""
    for hq, h, d, lens in ((4, 1, 128, [40000]), (8, 2, 64, [30000, 5, 0, 12345]), (2, 2, 32, [9001] * 3), (16, 1, 256, [7000, 9])):
        c = new_cache(V, sum(S.cdiv(x, 64) for x in lens) + 1, h, 64, d, "int8")
        fill_cache(c, d, "int8")
        check_attend(V, c, "int8", lens, [1] * len(lens), hq, "f32", "f32", seed=d, q_size=2.0)


def test_attend_many_requests(V):
    rng = np.random.RandomState(11)
    lens = [int(x) for x in rng.randint(0, 60, 700)]
    fresh = [int(min(x, f)) for x, f in zip(lens, rng.randint(0, 4, 700))]
    c = new_cache(V, sum(S.cdiv(x, 16) for x in lens), 1, 16, 32, "int8")
    fill_cache(c, 1, "int8")
    check_attend(V, c, "int8", lens, fresh, 3, "bf16", "bf16", seed=3)


def test_attend_large_scores_and_scales(V):
    """Scores of a few hundred, scales far apart between blocks and as small and large as float32 allows, a zero scale."""
    c = new_cache(V, 12, 2, 16, 64, "int8")
    fill_cache(c, 5, "int8")
    check_attend(V, c, "int8", [150, 20], [2, 1], 8, "f32", "f32", q_size=30.0)
    for lo, hi in ((-60, 3), (-126, -120), (90, 100)):
        c.v_scale.copy_(torch.pow(2.0, torch.randint(lo, hi, c.v_scale.shape, device="cuda").double()).float())
        check_attend(V, c, "int8", [150, 20], [2, 1], 8, "f32", "f32", seed=2)
    c.v_scale.zero_()
    check_attend(V, c, "int8", [150, 20], [2, 1], 8, "f32", "f32", seed=2)
    fill_cache(c, 5, "int8")
    c.k_scale.mul_(2.0 ** -40)
    check_attend(V, c, "int8", [150, 20], [2, 1], 8, "f32", "f32", seed=2, q_size=2.0 ** 38)
    check_attend(V, c, "int8", [150, 20], [2, 1], 8, "f32", "f32", seed=2, q_size=2.0 ** -100)
    c.k_scale.zero_()
    check_attend(V, c, "int8", [150, 20], [2, 1], 8, "f32", "f32", seed=2)
    fill_cache(c, 5, "int8")
    check_attend(V, c, "int8", [150, 20], [2, 1], 8, "f32", "f32", seed=2, scale=-0.3)
    check_attend(V, c, "int8", [150, 20], [2, 1], 8, "f32", "f32", seed=2, scale=0.0)


def check_rows_by_themselves(c, kind, lens, fresh, hq, table, q, window=0):
    """Outputs against the definition, each row by its own terms alone: the bound
    at the head of this file with the row's largest sum of p_j |v_jd| over sum p_j
    in place of the largest |v|.  A weight in two binary16 halves, its row's
    largest at 2^12 or more, adds half of 2^-24 per key, 2^-37 of the largest term:
    below 2^-20 of that sum for a few hundred keys of codes up to 448."""
    starts = np.concatenate([[0], np.cumsum(fresh)]).astype(np.int32)
    n, D, P, h = int(starts[-1]), c.head_dim, c.page_size, c.n_kv_heads
    out, lse = torch.zeros(n, hq, D, device="cuda"), torch.zeros(n, hq, device="cuda")
    c.attend(q, out, dev(lens, torch.int32), dev(starts), dev(table), c.attend_workspace(hq, max(fresh)), max_new=max(fresh),
             window=window, lse=lse)
    (kc, vc), (ks, vs) = codes_of(c)
    q64, got = q.double().cpu().numpy(), out.double().cpu().numpy()
    for i, f in enumerate(fresh):
        for t in range(f):
            p = lens[i] - f + t
            keys = np.arange(max(0, p - window + 1) if window else 0, p + 1)
            b, o = table[i, keys // P], keys % P
            k, v = (S.decode(x[b, :, o], kind) * s[b][:, :, None] for x, s in ((kc, ks), (vc, vs)))
            for y in range(hq):
                kv = y // (hq // h)
                x = q64[starts[i] + t, y] * float(np.float32(D ** -0.5))
                z = k[:, kv] @ x
                e = np.exp(z - z.max())
                own = (e @ np.abs(v[:, kv]) / e.sum()).max()
                tol = (2.0 ** -17 * (np.abs(k[:, kv]) @ np.abs(x)).max() + 2.0 ** -16) * own
                err = np.abs(got[starts[i] + t, y] - e @ v[:, kv] / e.sum()).max()
                assert err <= tol, (i, t, y, err / own, tol / own)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("hq,fresh,d", [(1, 4, 64), (4, 1, 128), (4, 2, 128), (4, 7, 64), (2, 2, 256), (6, 2, 256), (3, 5, 80)])
def test_attend_scales_far_apart(V, kind, hq, fresh, d):
    """Value scales of the pages up to 2^100 apart.  A row is exact by its own
    terms, whatever the scales of pages that it does not see (a later token's,
    those before its window) and of pages that it weighs at almost nothing."""
    c = new_cache(V, 30, 1, 16, d, kind)
    fill_cache(c, d, kind)
    g = torch.Generator("cuda").manual_seed(hq)
    q = torch.randn(2 * fresh, hq, d, generator=g, device="cuda")
    table = np.arange(30, dtype=np.int32).reshape(2, 15)
    # the last token alone sees page 1; the pages of the window's first rows
    c.v_scale[1] *= 2.0 ** 40
    for lens in ([16 + fresh - 1, 16 + fresh], [17, 18 + fresh]):
        check_rows_by_themselves(c, kind, [max(x, fresh) for x in lens], [fresh] * 2, hq, table, q)
    c.v_scale.copy_(torch.pow(2.0, 8.0 * torch.arange(30, device="cuda").flip(0) - 120)[:, None])
    check_rows_by_themselves(c, kind, [230, 37], [fresh] * 2, hq, table, q, window=17)
    check_rows_by_themselves(c, kind, [230, 37], [fresh] * 2, hq, table, q)
    # any order of scales, scores from -60 to 60
    for seed in range(3):
        c.v_scale.copy_(torch.pow(2.0, torch.randint(-50, 50, c.v_scale.shape, generator=g, device="cuda").float()))
        size = 15 / float((q[0, 0] @ (c.k[0, 0].view(torch.int8).float() if kind == "int8" else
                                      c.k[0, 0].view(torch.float8_e4m3fn).float()).T).abs().max()) / float(c.k_scale[0, 0])
        check_rows_by_themselves(c, kind, [240, 100], [fresh] * 2, hq, table, q * size * d ** 0.5)


@pytest.mark.parametrize("hq,h,d", [(32, 8, 128), (8, 8, 128), (4, 2, 64), (8, 1, 256)])
def test_attend_workspace_for_more_tokens(V, hq, h, d):
    """A workspace for up to n new tokens serves every smaller number, one after another."""
    c = new_cache(V, 60, h, 16, d, "int8")
    fill_cache(c, d, "int8")
    lens, table = [400, 90], np.array([list(range(25)), list(range(25, 50))], np.int32)
    for most in (2, 5, 16):
        ws = c.attend_workspace(hq, most)
        for n in (1, 2, 5, 16, 1):
            if n > most:
                continue
            q = torch.randn(2 * n, hq, d, device="cuda")
            res = []
            for w in (ws, c.attend_workspace(hq, n)):
                out = torch.zeros(2 * n, hq, d, device="cuda")
                c.attend(q, out, dev(lens, torch.int32), dev([0, n, 2 * n], torch.int32), dev(table), w, max_new=n)
                res.append(out)
            assert torch.equal(*res), (most, n)


def test_attend_joins_of_large_values(V):
    """Values near float32's largest over a context of many parts: an average of them is no larger."""
    for hq, h, d, lens in ((4, 1, 128, [9000]), (8, 1, 64, [5000, 40]), (16, 1, 256, [7000])):
        c = new_cache(V, sum(S.cdiv(x, 64) for x in lens), h, 64, d, "int8")
        fill_cache(c, d, "int8")
        c.v_scale.fill_(2.0 ** 119)
        check_attend(V, c, "int8", lens, [1] * len(lens), hq, "f32", "f32", seed=d, q_size=0.1)


def test_attend_query_zero_and_wide_range(V):
    c = new_cache(V, 12, 1, 16, 64, "int8")
    fill_cache(c, 6, "int8")
    q = torch.randn(2, 4, 64, device="cuda") * torch.pow(10.0, torch.randint(-6, 1, (2, 4, 64), device="cuda").float())
    q[0, 1] = 0
    check_attend(V, c, "int8", [100, 60], [1, 1], 4, "f32", "f32", q=q)


def test_attend_garbage_outside_the_request_is_not_seen(V):
    """Codes and scales past a request's length, before its window and on pages
    it does not own are NaN or huge; pages outside the cache are left out."""
    for kind in ("int8", "e4m3"):
        c = new_cache(V, 20, 2, 16, 64, kind)
        fill_cache(c, 7, kind)
        table = np.array([[4, 9, 2, 99], [7, 1, -1, 3], [5, 6, 8, 10]], np.int32)
        lens, fresh = [37, 60, 64], [1, 2, 1]
        base, bl = check_attend(V, c, kind, lens, fresh, 4, "f32", "f32", table=table, window=30)
        seen = {4, 9, 2, 7, 1, 3, 6, 8, 10}
        for b in set(range(20)) - seen | {5}:  # page 5: tokens 0..15 of request 2, before its window
            c.k_scale[b], c.v_scale[b] = float("nan"), float("inf")
            c.k[b], c.v[b] = 0x7f, 0x7f
        c.k[2, :, 5:], c.v[2, :, 5:] = 0x7f, 0xff  # past the length of request 0
        again, al = check_attend_raw(c, lens, fresh, 4, table, 30)
        assert torch.equal(base, again) and torch.equal(bl, al)


def check_attend_raw(c, lens, fresh, hq, table, window, seed=0):
    rng = np.random.RandomState(seed)
    starts = np.concatenate([[0], np.cumsum(fresh)]).astype(np.int32)
    n = int(starts[-1])
    q = torch.from_numpy(rng.randn(n, hq, c.head_dim).astype(np.float32)).cuda()
    out, lse = torch.zeros((n, hq, c.head_dim), device="cuda"), torch.zeros((n, hq), device="cuda")
    c.attend(q, out, dev(lens, torch.int32), dev(starts), dev(table), c.attend_workspace(hq, max(fresh)), max_new=max(fresh),
             window=window, lse=lse)
    return out, lse


def test_attend_nan_block_reaches_only_who_sees_it(V):
    c = new_cache(V, 8, 2, 16, 64, "int8")
    fill_cache(c, 8, "int8")
    table = np.array([[0, 1, 2, 3], [4, 5, 6, 7]], np.int32)
    clean, cl = check_attend_raw(c, [64, 50], [1, 1], 4, table, 0)
    c.v_scale[1, 0] = float("nan")
    out, lse = check_attend_raw(c, [64, 50], [1, 1], 4, table, 0)
    assert bool(out[0, :2].isnan().all()) and torch.equal(out[0, 2:], clean[0, 2:]) and torch.equal(out[1], clean[1])
    c.v_scale[1, 0] = 0.5
    c.k_scale[5, 1] = float("nan")
    out, lse = check_attend_raw(c, [64, 50], [1, 1], 4, table, 0)
    assert bool(out[1, 2:].isnan().all()) and bool(lse[1, 2:].isnan().all())
    assert not bool(out[1, :2].isnan().any()) and not bool(out[0].isnan().any())
    out, _ = check_attend_raw(c, [64, 50], [1, 1], 4, table, 10)  # the window leaves page 5 out
    assert not bool(out.isnan().any())


@pytest.mark.parametrize("hq,fresh", [(4, 1), (8, 1), (8, 2), (4, 9)])
@pytest.mark.parametrize("dtype", list(DT))
def test_attend_query_that_is_no_number(V, hq, fresh, dtype):
    """A NaN or an infinity in a row of the query spoils that row alone."""
    c = new_cache(V, 30, 2, 16, 64, "int8")
    fill_cache(c, 10, "int8")
    n = 2 * fresh
    g = torch.Generator("cuda").manual_seed(hq)
    q = torch.randn(n, hq, 64, generator=g, device="cuda").to(DT[dtype])
    starts, lens = dev([0, fresh, n], torch.int32), dev([400, 33], torch.int32)
    table = dev(np.array([list(range(25)), [25, 26, 27] + [-1] * 22]), torch.int32)
    res = []
    for bad in (False, True):
        if bad:
            q[0, 1, 5], q[n - 1, hq - 1, 63], q[n - 1, 0, 0] = float("nan"), float("inf"), -float("inf")
        out, lse = torch.zeros(n, hq, 64, device="cuda"), torch.zeros(n, hq, device="cuda")
        c.attend(q, out, lens, starts, table, c.attend_workspace(hq, fresh), max_new=fresh, lse=lse)
        res.append((out, lse))
    spoilt = torch.zeros(n, hq, dtype=torch.bool, device="cuda")
    spoilt[0, 1] = spoilt[n - 1, hq - 1] = spoilt[n - 1, 0] = True
    assert torch.equal(res[0][0][~spoilt], res[1][0][~spoilt]) and torch.equal(res[0][1][~spoilt], res[1][1][~spoilt])
    assert bool(res[1][0][spoilt].isnan().all()) and bool(res[1][1][spoilt].isnan().all())


def test_attend_strided_query_and_output(V):
    """Query and output as slices of wider rows at odd offsets, heads before tokens in memory."""
    c = new_cache(V, 10, 2, 16, 64, "int8")
    fill_cache(c, 9, "int8")
    lens, fresh, hq = [70, 33], [3, 1], 4
    table = np.arange(10, dtype=np.int32).reshape(2, 5)
    starts = dev([0, 3, 4], torch.int32)
    for dt in DT.values():
        q = torch.randn(4, hq, 64, device="cuda").to(dt)
        ref = torch.zeros(4, hq, 64, dtype=dt, device="cuda")
        ws = c.attend_workspace(hq, 3)
        args = (dev(lens, torch.int32), starts, dev(table), ws)
        c.attend(q, ref, *args, max_new=3)
        flat = torch.zeros(4 * (hq * 64 + 3) + 1, dtype=dt, device="cuda")
        q2 = flat[1:].view(4, -1)[:, :hq * 64].view(4, hq, 64)
        q2.copy_(q)
        o2 = torch.zeros(hq, 4, 70, dtype=dt, device="cuda")[:, :, 1:65].transpose(0, 1)
        c.attend(q2, o2, *args, max_new=3)
        assert torch.equal(o2, ref)


def test_attend_cache_past_32_bits(V):
    """A page whose codes begin more than 2^32 bytes into the cache."""
    h, p, d = 8, 64, 128
    pages = (2 ** 32) // (h * p * d) + 40
    k = torch.zeros((pages, h, p, d), dtype=torch.uint8, device="cuda")
    v = torch.zeros_like(k)
    s = torch.zeros((2, pages, h), device="cuda")
    big = V.KVCache(k, v, s[0], s[1], "int8")
    c = new_cache(V, 4, h, p, d, "int8")
    x = torch.randn(2, 200, h, d, device="cuda")
    slots = torch.arange(200, device="cuda")
    c.append(x[0], x[1], slots)
    far = pages - 4
    big.append(x[0], x[1], slots + far * p)
    assert torch.equal(big.k[far:], c.k.where(torch.arange(256, device="cuda").view(4, 1, 64, 1) < 200, torch.zeros_like(c.k)))
    table = np.arange(4, dtype=np.int32)[None]
    a, al = check_attend_raw(c, [200], [1], 16, table, 0)
    b, bl = check_attend_raw(big, [200], [1], 16, table + far, 0)
    assert torch.equal(a, b) and torch.equal(al, bl)
    ga, gb = (torch.zeros(200, h, d, device="cuda") for _ in range(2))
    big.gather(slots + far * p, ga, gb)
    assert float((ga - x[0]).abs().max()) < 0.05


# ---------------------------------------------------------------- log probabilities

def check_score(V, x, targets, scale, k, ws=None):
    n, v = x.shape
    t = None if targets is None else dev(targets, torch.int64)
    f = lambda *s, d=torch.float32: torch.full(s, 5, dtype=d, device="cuda")  # noqa: E731
    lp, en, rk, tl, ti = f(n), f(n), f(n, d=torch.int32), f(n, k), f(n, k, d=torch.int32)
    ws = V.score_workspace(n, v) if ws is None else ws
    for _ in range(2):
        V.token_logprobs(x, t, lp, en, rk, tl, ti, ws, scale=scale)
    x64 = x.double().cpu().numpy()
    s = float(np.float32(scale))
    wl, we, wr, wt, wi = S.token_logprobs(x64, targets, s, k)
    fin = np.where(np.isfinite(x64), x64, 0)
    u, top = 2.0 ** -24, s * np.abs(fin).max(1)
    rel = (v / 128 + 72) * u
    for got, want, tol in ((tl, wt, (rel + 8 * u * top + 4 * u)[:, None]), (en, we, (2 * rel + 16 * u * (1 + top)) * (1 + np.abs(we)) * 2)):
        g = got.double().cpu().numpy()
        bad = ~np.isfinite(want)
        assert np.array_equal(g[bad], want[bad], equal_nan=True)
        assert np.all(np.abs(g - np.where(bad, g, want))[~bad] <= np.broadcast_to(tol, want.shape)[~bad])
    assert np.array_equal(ti.cpu().numpy(), wi)
    if targets is not None:
        g = lp.double().cpu().numpy()
        bad = ~np.isfinite(wl)
        assert np.array_equal(g[bad], wl[bad], equal_nan=True)
        assert np.all(np.abs(g - wl)[~bad] <= (rel + 8 * u * top + 4 * u)[~bad])
        assert np.array_equal(rk.cpu().numpy(), wr)
    else:
        assert bool((lp == 5).all()) and bool((rk == 5).all())


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("n,v,k,scale", [(1, 1, 1, 1.0), (3, 2, 5, 0.7), (5, 77, 0, 1.0), (4, 300, 32, 1.25), (17, 1025, 20, 1.0),
                                         (2, 32000, 20, 1.3), (1, 128256, 32, 1.0), (300, 272, 3, 2.0)])
def test_score(V, dtype, n, v, k, scale):
    g = torch.Generator("cuda").manual_seed(n + v)
    x = (2.5 * torch.randn((n, v), generator=g, device="cuda")).to(DT[dtype])
    rng = np.random.RandomState(v)
    t = rng.randint(0, v, n)
    t[0] = int(x[0].float().argmax())
    if n > 2:
        t[1], t[2] = -1, v
    check_score(V, x, t, scale, k)


def test_score_orders_that_go_wrong(V):
    """Ascending and descending rows, all equal, ties at the edge of the list, excluded tokens, NaN and infinities."""
    v = 5000
    inf, nan = float("inf"), float("nan")
    rows = [torch.arange(v).float() / 100, -torch.arange(v).float() / 100, torch.zeros(v), torch.full((v,), -inf),
            torch.full((v,), -inf), torch.randn(v), torch.randn(v), (torch.arange(v) % 7).float(), torch.randn(v),
            torch.randn(v) * 1e4, torch.full((v,), 3e38), torch.randn(v), torch.full((v,), -0.0)]
    rows[4][[7, 4000, 4999]] = torch.tensor([1.0, 2.0, 1.0])
    rows[5][::3] = -inf
    rows[6][123] = nan
    rows[8][77] = inf
    rows[11][4321], rows[11][5] = nan, inf
    rows[12][::2] = 0.0
    x = torch.stack(rows).cuda()
    t = np.array([v - 1, 0, 1234, 3, 4999, 3, 9, 3500, 77, 5, 4000, 1, 4999])
    for k in (1, 3, 32):
        check_score(V, x, t, 1.0, k)
    check_score(V, x, None, 1.0, 5)
    b = x.bfloat16()
    check_score(V, b, t, 0.5, 20)


@pytest.mark.parametrize("v", [900, 3000])
def test_score_orders_in_long_batches(V, v):
    """The same kinds of rows where every row is a warp's work, and among thousands of others."""
    inf, nan = float("inf"), float("nan")
    g = torch.Generator("cuda").manual_seed(v)
    x = torch.randn((13, v), generator=g, device="cuda")
    x[0], x[1], x[2] = torch.arange(v, device="cuda") / 100, -torch.arange(v, device="cuda") / 100, 0
    x[3] = -inf
    x[4] = -inf
    x[4, [7, v // 2, v - 1]] = torch.tensor([1.0, 2.0, 1.0], device="cuda")
    x[5, ::3] = -inf
    x[6, 123] = nan
    x[7] = torch.arange(v, device="cuda") % 7
    x[8, 77] = inf
    x[9] *= 1e4
    x[10] = -3.4e38
    x[11, v - 5], x[11, 5] = nan, inf
    x[12] = torch.finfo(torch.float32).min
    x[12, 300:310] = 1.0
    t = np.array([v - 1, 0, v // 3, 3, v - 1, 3, 9, v // 2 + 1, 77, 5, v - 2, 1, 305])
    for dtype in DT.values():
        y = x.to(dtype)
        check_score(V, y, t, 1.0, 20)  # 13 rows
        n = 13 * 260
        many, tt = y.repeat(260, 1), dev(np.tile(t, 260), torch.int64)
        f = lambda *s, d=torch.float32: torch.full(s, 5, dtype=d, device="cuda")  # noqa: E731
        out = [[f(k), f(k), f(k, d=torch.int32), f(k, 20), f(k, 20, d=torch.int32)] for k in (13, n)]
        V.token_logprobs(y, tt[:13], *out[0], V.score_workspace(13, v))
        V.token_logprobs(many, tt, *out[1], V.score_workspace(n, v))
        for a, b, name in zip(out[0], out[1], ("logprob", "entropy", "rank", "top", "index")):
            a = a.repeat((260,) + (1,) * (a.dim() - 1))
            if a.dtype is torch.int32:
                assert torch.equal(a, b), name
            else:
                assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.isinf(), b.isinf()), name
                ok = a.isfinite()
                assert torch.allclose(a[ok], b[ok], rtol=2e-5, atol=2e-5), name


def test_score_logits_further_apart_than_float32(V):
    """Logits whose difference passes float32's largest while the scaled one does not."""
    x = (torch.rand(4, 3000, device="cuda") * 2 - 1) * 3e38
    x[:, 5], x[:, 2500], x[1, 7] = 3.3e38, -3.3e38, -float("inf")
    x[2] = torch.where(x[2] > 0, 3.0e38, -3.0e38)
    for dt in (torch.float32, torch.bfloat16):
        for scale in (0.25, 1e-3, 2.0 ** -100):
            check_score(V, x.to(dt), [2500, 7, 2999, 5], scale, 32)
        many = x.to(dt).repeat(2000, 1)
        t = torch.tensor([2500, 7, 2999, 5], device="cuda")
        few, all_ = (torch.empty(n, device="cuda") for n in (4, 8000))
        rk = torch.empty(8000, dtype=torch.int32, device="cuda")
        V.token_logprobs(many[:4], t, few, None, rk, None, None, V.score_workspace(4, 3000), scale=0.25)
        V.token_logprobs(many, t.repeat(2000), all_, None, rk, None, None, V.score_workspace(8000, 3000), scale=0.25)
        assert torch.equal(few.repeat(2000), all_)
    low = torch.full((1, 3000), -3.3e38, device="cuda")  # the list reaches logits that far below its first
    low[0, 9] = 3.3e38
    check_score(V, low, [17], 0.25, 32)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("n,v", [(1, 20000), (3, 20003), (2500, 1500), (2500, 2047), (2000, 9000)])
def test_score_rank_of_a_negative_zero(V, dtype, n, v):
    """-0 and +0 are equal logits, placed by their index: targets of either sign
    at a row's start, middle and end, among larger and smaller logits, and zeros
    behind them in every tile; few rows and many, wide loads and single ones."""
    g = torch.Generator("cuda").manual_seed(n + v)
    for odd in (0, 1):
        flat = torch.randint(-1, 2, (n * v + odd,), generator=g, device="cuda").float()
        flat[torch.rand(flat.shape, generator=g, device="cuda") < 0.5] *= -1  # zeros of both signs
        x = flat.to(DT[dtype])[odd:].view(n, v)
        f = lambda *s, d=torch.float32: torch.empty(s, dtype=d, device="cuda")  # noqa: E731
        lp, en, rk, tl, ti, ws = f(n), f(n), f(n, d=torch.int32), f(n, 0), f(n, 0, d=torch.int32), V.score_workspace(n, v)
        for at in (0, v // 2, v - 1):
            for zero in (-0.0, 0.0):
                x[:, at] = zero
                t = torch.full((n,), at, device="cuda")
                V.token_logprobs(x, t, lp, en, rk, tl, ti, ws)
                want = (x > 0).sum(1) + (x[:, :at] == 0).sum(1)
                assert torch.equal(rk.long(), want), (odd, at, zero)


def test_score_strided_unaligned_rows(V):
    for dt in DT.values():
        flat = torch.randn(6 * 1003 + 5, device="cuda").to(dt)
        for off in (0, 1, 3):
            x = flat[off:off + 6 * 1003].view(6, 1003)[:, :997]
            check_score(V, x, [0, 996, 500, -1, 3, 4], 1.0, 8)
        check_score(V, flat[:4096].view(4, 1024)[:1], [1000], 1.0, 4)


def test_score_workspace_of_a_larger_batch(V):
    ws = V.score_workspace(64, 128256)
    for n, v in ((3, 40000), (64, 500), (1, 128256), (40, 9000)):
        x = torch.randn(n, v, device="cuda")
        check_score(V, x, [v // 2] * n, 1.0, 6, ws)


def test_workspaces_elsewhere_are_refused(V):
    x = torch.zeros(2, 50, device="cuda")
    e = torch.zeros(2, device="cuda")
    for ws in (V.score_workspace(2, 50).cpu(), V.score_workspace(2, 50).view(-1, 2)[:, 0]):
        with pytest.raises(ValueError, match="workspace"):
            V.token_logprobs(x, None, None, e, None, None, None, ws)
    c = new_cache(V, 4, 2, 16, 64, "int8")
    q = torch.zeros(1, 2, 64, device="cuda")
    z = dev([1, 0], torch.int32)
    a = (q, q.clone(), z[:1], z, z[None])
    with pytest.raises(ValueError, match="workspace"):
        c.attend(*a, c.attend_workspace(2).cpu())
    for kw in (dict(window=1 << 40), dict(max_new=1.5)):
        with pytest.raises(ValueError):
            c.attend(*a, c.attend_workspace(2), **kw)
    with pytest.raises(V.Q.SeedQError):  # an infinity in float32
        c.attend(*a, c.attend_workspace(2), scale=1e300)


def test_score_lists_that_overflow(V):
    """Few rows, cut into chunks: one of equal logits, small whole numbers with
    ties at every edge, and chunks of which all but one reach the list with almost
    all of their alternatives."""
    v = 40 * 4096 + 77
    g = torch.Generator("cuda").manual_seed(1)
    rows = [torch.zeros(v, device="cuda"), torch.randint(0, 9, (v,), generator=g, device="cuda").float(),
            torch.full((v,), -5.0, device="cuda")]
    for c in range(41):
        if c != 7:
            at = c * 4096 + torch.randperm(77, generator=g, device="cuda")[:31]
            rows[2][at] = 5 + torch.rand(31, generator=g, device="cuda")
    x = torch.stack(rows)
    check_score(V, x, [v - 1, 4000, 8], 1.0, 32)
    check_score(V, x.bfloat16(), [0, 4000, 8], 1.0, 32)
    check_score(V, x[1:2, 1:], [17], 2.0, 9)


def test_score_row_counts_around_the_split(V):
    """Row counts and lengths on both sides of every choice between the kernels."""
    for n, v in ((1, 1024), (1, 1025), (3, 2049), (2432, 1500), (2433, 1500), (76, 128256), (77, 128256), (608, 16384), (609, 16384)):
        x = torch.randn((n, v), device="cuda") * 3
        lp, en = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        rk, t = torch.empty(n, dtype=torch.int32, device="cuda"), torch.randint(0, v, (n,), device="cuda")
        tl, ti = torch.empty(n, 6, device="cuda"), torch.empty(n, 6, dtype=torch.int32, device="cuda")
        V.token_logprobs(x, t, lp, en, rk, tl, ti, V.score_workspace(n, v))
        ref = torch.log_softmax(x.double(), 1)
        tol = (v / 128 + 72) * 2.0 ** -24 + 8 * 2.0 ** -24 * float(x.abs().max()) + 2.0 ** -22
        assert float((lp - ref.gather(1, t[:, None])[:, 0]).abs().max()) <= tol
        assert float((en + (ref.exp() * ref).sum(1)).abs().max()) <= 40 * tol
        best = torch.sort(x.double(), dim=1, descending=True, stable=True).indices[:, :6]
        assert torch.equal(ti.long(), best)
        assert float((tl - ref.gather(1, best)).abs().max()) <= tol
        xt = x.gather(1, t[:, None])
        assert torch.equal(rk.long(), ((x > xt) | ((x == xt) & (torch.arange(v, device="cuda") < t[:, None]))).sum(1))


# ---------------------------------------------------------------- together

def test_batch_that_shrinks_on_one_plan(V):
    """Fewer requests than the plan was made for, after a step of more: what the
    plan then hands on has no request of the earlier step in it."""
    H, HQ, D, P = 2, 4, 64, 16
    plan = V.BatchPlan(4, 16)
    c = V.KVCache.empty(20, H, D, P)
    table = torch.full((4, 4), -1, dtype=torch.int32, device="cuda")
    free, count = torch.arange(20, dtype=torch.int32, device="cuda"), dev([20], torch.int32)
    seq = torch.zeros(4, dtype=torch.int32, device="cuda")
    g = torch.Generator("cuda").manual_seed(0)
    for new in ([9, 1, 3, 2], [1, 1, 1, 1], [3, 3], [1, 2, 1], [5], [2, 1, 4, 1]):
        r, n = len(new), sum(new)
        plan.build(seq, dev(new, torch.int32), table, free, count, P)
        assert plan.starts.tolist() == [sum(new[:i]) for i in range(r + 1)] and plan.status.tolist() == [0] * r
        kv, q = (torch.randn(s, generator=g, device="cuda") for s in ((2, n, H, D), (n, HQ, D)))
        c.append(kv[0], kv[1], plan.slots)
        out, alone = torch.zeros(n, HQ, D, device="cuda"), torch.zeros(n, HQ, D, device="cuda")
        ws = c.attend_workspace(HQ, max(new))
        c.attend(q, out, plan.seq_lens, plan.starts, table, ws, max_new=max(new))
        for i in range(r):  # a request at a time
            a, b = sum(new[:i]), sum(new[:i + 1])
            c.attend(q[a:b], alone[a:b], plan.seq_lens[i:], dev([0, b - a], torch.int32), table[i:], ws, max_new=max(new))
        assert torch.allclose(out, alone, atol=1e-5)
        assert plan.seq_lens.tolist() == [x + y for x, y in zip(seq.tolist(), new)]
        seq[:r] = plan.seq_lens
        count.copy_(plan.free_count)


def test_side_stream_and_graph(V):
    """plan, append, attend and score captured in a graph on a stream of their own, replayed for
    new lengths, against the calls one by one."""
    B, H, HQ, D, P, vocab = 5, 2, 4, 64, 16, 500
    c = [V.KVCache.empty(40, H, D, P) for _ in range(2)]
    table = [torch.full((B, 8), -1, dtype=torch.int32, device="cuda") for _ in range(2)]
    free = [torch.arange(40, dtype=torch.int32, device="cuda") for _ in range(2)]
    count = [torch.full((1,), 40, dtype=torch.int32, device="cuda") for _ in range(2)]
    seq = [torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2)]
    plan = [V.BatchPlan(B, 16) for _ in range(2)]
    ws = [c[i].attend_workspace(HQ, 4) for i in range(2)]
    sw = [V.score_workspace(16, vocab) for _ in range(2)]
    out = [torch.zeros(16, HQ, D, device="cuda") for _ in range(2)]
    sc = [[torch.zeros(16, device="cuda"), torch.zeros(16, device="cuda"), torch.zeros(16, dtype=torch.int32, device="cuda"),
           torch.zeros(16, 3, device="cuda"), torch.zeros(16, 3, dtype=torch.int32, device="cuda")] for _ in range(2)]
    new = torch.zeros(B, dtype=torch.int32, device="cuda")
    kv, q = torch.zeros(2, 16, H, D, device="cuda"), torch.zeros(16, HQ, D, device="cuda")
    x, t = torch.zeros(16, vocab, device="cuda"), torch.zeros(16, dtype=torch.int64, device="cuda")

    def step(i):
        plan[i].build(seq[i], new, table[i], free[i], count[i], P)
        c[i].append(kv[0], kv[1], plan[i].slots)
        c[i].attend(q, out[i], plan[i].seq_lens, plan[i].starts, table[i], ws[i], max_new=4)
        V.token_logprobs(x, t, *sc[i], sw[i])
        seq[i].copy_(plan[i].seq_lens)
        count[i].copy_(plan[i].free_count)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(0)  # loads the kernels; no new tokens, so nothing changes
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        step(0)
    rng = random.Random(0)
    for it in range(12):
        new.copy_(torch.tensor([rng.choice([0, 1, 2, 4]) if it else 3 for _ in range(B)], dtype=torch.int32))
        if it == 8:
            new[2] = -1
        for z in (kv, q, x):
            z.normal_()
        t.random_(0, vocab)
        g.replay()
        step(1)
        for a, b in zip([out[0], seq[0], count[0], table[0], c[0].k_scale, *sc[0]], [out[1], seq[1], count[1], table[1], c[1].k_scale, *sc[1]]):
            assert torch.equal(a, b), it
