"""Beam search's choice and the pages of the chosen beams on the GPU against the fp64 oracle.

Whole numbers compare exactly, where neighbours of different beams in the order lie
further apart (the oracle's `room`) than twice what the float32 log sums may be off
by; inputs are drawn until they do.  All terms of sum exp are positive.  A lane adds
at most 32 of them in order, then 8 + 5 sums of sums join (and one more for each 2^18
logits), at most 50 u with u = 2^-24; a term's 2^x is within 4 u, and the roundings of
its difference, of the product and of scale * log2(e) are 3 u of |z - m|, which
weighted by the terms themselves stays below ln(vocab) <= 12: 36 u.  So a log sum is
off by less than 110 u (1 + its logarithm's own 4 u), and a total rounds once to float32.
"""
import os
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
U = 2.0 ** -24
OFF = 120 * U


@pytest.fixture(scope="module")
def V():
    from paper_2609_38477_gb300 import build

    build.build()
    from paper_2609_38477_gb300 import seedq, serving

    seedq.lib()
    return serving


def select(V, x, scores, n_out, scale=1.0, done=None, end=-1, weights=None, work=None):
    g, b = scores.shape
    out = (torch.full((g, n_out), 3.0, device="cuda"), *(torch.full((g, n_out), 3, dtype=torch.int32, device="cuda") for _ in range(2)))
    V.beam_select(x, scores, *out, V.beam_workspace(g, b, x.shape[1]) if work is None else work, scale=scale, done=done, end_token=end,
                  weights=weights)
    return out


def check_select(V, x, scores, n_out, scale=1.0, done=None, end=-1, weights=None, work=None):
    """x: (rows, vocab) on the device.  False where neighbours lie too close to tell."""
    g, b = scores.shape
    args = [None if t is None else torch.as_tensor(t).cuda() for t in (scores, done, weights)]
    cpu = lambda t: None if t is None else t.cpu().numpy()  # noqa: E731
    got = select(V, x, args[0], n_out, scale, args[1], end, args[2], work)
    want = S.beam_select(x.double().cpu().numpy().reshape(g, b, -1), args[0].double().cpu().numpy(), float(np.float32(scale)), n_out,
                         cpu(args[1]), end, None if weights is None else args[2].double().cpu().numpy())
    if not want[3] > 2 * OFF:
        return False
    assert np.array_equal(got[1].cpu().numpy(), want[1]) and np.array_equal(got[2].cpu().numpy(), want[2])
    gs = got[0].double().cpu().numpy()
    fine = np.isfinite(want[0])
    assert np.array_equal(np.isnan(gs), np.isnan(want[0])) and np.array_equal(gs[~fine & ~np.isnan(gs)], want[0][~fine & ~np.isnan(gs)])
    assert np.all(np.abs(gs[fine] - want[0][fine]) <= OFF + np.abs(want[0][fine]) * U)
    return True


def some(check):
    """check(seed) of the first seed whose inputs can be told apart."""
    assert any(check(seed) for seed in range(20))


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("g,b,v,n", [(1, 1, 1, 1), (1, 1, 1, 32), (1, 3, 2, 5), (2, 4, 77, 8), (1, 1, 300, 32), (3, 32, 40, 32),
                                     (1, 4, 8192, 4), (2, 2, 8193, 20), (1, 5, 32000, 32), (7, 8, 4097, 16), (2, 3, 128256, 6),
                                     (1, 2, 100003, 32), (65, 1, 513, 2), (60, 5, 32000, 12), (400, 1, 33000, 3), (9, 32, 50004, 32)])
def test_select(V, dtype, g, b, v, n):
    def check(seed):
        rng = np.random.RandomState(g * 7 + b + v + n + 1000 * seed)
        x = torch.from_numpy((3 * rng.randn(g * b, v)).astype(np.float32)).to(DT[dtype]).cuda()
        return check_select(V, x, (-5 + 2 * rng.randn(g, b)).astype(np.float32), n)

    some(check)


@pytest.mark.parametrize("seed", range(6))
def test_select_masks_ends_and_weights(V, seed):
    """Masked tokens and whole rows, finished and empty beams, weights, a scale, rows at odd offsets and apart."""
    g, b, v = [(3, 4, 700), (2, 8, 5000), (5, 2, 61), (1, 32, 1000), (4, 6, 257), (2, 3, 40000)][seed]
    dtype = list(DT.values())[seed % 3]
    flat = torch.full((g * b * (v + 13) + 1,), float("nan"), dtype=dtype, device="cuda")  # between rows: nothing that may be read
    x = flat[seed % 2:][:g * b * (v + 13)].view(g * b, v + 13)[:, :v]
    work = V.beam_workspace(g, b, v)

    def check(k, weighted, as_bytes):
        nonlocal scores, done, end
        rng = np.random.RandomState(100 + seed + 1000 * k)
        z = 3 * rng.randn(g * b, v)
        z[rng.rand(g * b, v) < 0.4] = -np.inf
        z[rng.randint(g * b)] = -np.inf
        x.copy_(torch.from_numpy(z.astype(np.float32)))
        scores = (-5 + 2 * rng.randn(g, b)).astype(np.float32)
        scores[rng.rand(g, b) < 0.2] = -np.inf
        done = rng.rand(g, b) < 0.3
        weights = (rng.randint(3, 30, (g, b)) ** -0.7).astype(np.float32) if weighted else None
        end = int(rng.randint(v))
        return check_select(V, x, scores, 1 + seed * 6, [0.5, 1.0, 2.0][seed % 3], done.astype(np.uint8) * 7 if as_bytes else done, end,
                            weights, work)

    scores = done = end = None
    for weighted in (False, True):
        for as_bytes in (False, True):
            some(lambda k: check(k, weighted, as_bytes))
    # what is not read may hold anything
    for r in range(g * b):
        if done.reshape(-1)[r] or scores.reshape(-1)[r] == -np.inf:
            x[r] = float("nan")
    got = select(V, x, torch.from_numpy(scores).cuda(), 9, done=torch.from_numpy(done).cuda(), end=end, work=work)
    assert not bool(got[0].isnan().any())


def test_select_equal_logits(V):
    """Ties go to the lower beam, then the lower token: whole rows of one value, pairs of equal rows, -0 beside +0."""
    for v, n in ((1000, 32), (70, 7), (9001, 20)):
        for dtype in DT.values():
            x = torch.zeros((6, v), dtype=dtype, device="cuda")
            x[1, ::2] = -0.0
            x[4:, 3::5] = 2.0
            scores = torch.full((2, 3), -1.5, device="cuda")
            got = select(V, x, scores, n)
            assert got[1][0].tolist() == [0] * n and got[2][0].tolist() == list(range(n))
            top = list(range(3, v, 5))
            two = [(1, t) for t in top] + [(2, t) for t in top]
            assert list(zip(got[1][1].tolist(), got[2][1].tolist())) == two[:n]
    # equal rows at addresses of every alignment, the same tokens from each in turn of the beam
    rng = np.random.RandomState(5)
    row = torch.from_numpy(rng.randn(1003).astype(np.float32)).cuda()
    x = row.expand(8, 1003).contiguous()
    got = select(V, x, torch.zeros((1, 8), device="cuda"), 32)
    order = torch.sort(row, descending=True, stable=True).indices.tolist()
    assert got[1][0].tolist() == list(range(8)) * 4 and got[2][0].tolist() == [t for t in order[:4] for _ in range(8)]


def test_select_equal_rows_of_many(V):
    """Equal rows in a large batch, dealt to the SMs at other places each: sums equal to the bit, ties by the beam."""
    for v, dtype in ((40000, "f32"), (128256, "bf16")):
        row = (3 * torch.randn(v, generator=torch.Generator("cuda").manual_seed(v), device="cuda")).to(DT[dtype])
        x = row.expand(200, v).contiguous()
        scores = torch.zeros((40, 5), device="cuda")
        scores[7], scores[8, :4], scores[9, 0] = -float("inf"), -float("inf"), -float("inf")
        got = select(V, x, scores, 10)
        order = torch.sort(row.float(), descending=True, stable=True)
        ties = [order.indices[order.values == y].tolist() for y in torch.unique(order.values).flip(0)[:10]]
        for g in range(40):
            beams = [] if g == 7 else [4] if g == 8 else [1, 2, 3, 4] if g == 9 else list(range(5))
            want = [(b, t) for same in ties for b in beams for t in same][:10]
            assert list(zip(got[1][g].tolist(), got[2][g].tolist())) == (want or [(-1, -1)] * 10)
            assert len(set(got[0][g].tolist())) <= 10 and bool((got[0][g] == got[0][0])[:2].all()) or g in (7, 8)


def test_select_of_a_large_batch_repeats(V):
    """Whoever joins a request, the results are the same bits, and the workspace is left as it was."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    g, b, v = 70, 6, 128256
    x = torch.randn((g * b, v), device="cuda", generator=gen).bfloat16()
    scores = -torch.rand((g, b), device="cuda", generator=gen)
    scores[3] = scores[40:44] = -np.inf
    work = V.beam_workspace(g, b, v)
    first = select(V, x, scores, 12, work=work)
    head = work[: 2 * 8192 * 4 + 16]  # the counters
    assert int(head.max()) == 0
    for i in (0, 3, 33, 69):  # alone, other chunks: both sums may be off, and totals of less than 16 round
        score, beam, token = select(V, x[i * b:(i + 1) * b], scores[i:i + 1], 12)
        assert torch.allclose(score, first[0][i:i + 1], rtol=0, atol=2 * OFF + 32 * U)
        assert i != 3 or (bool((first[1][3] == -1).all()) and bool((first[2][3] == -1).all()))
    for _ in range(60):
        assert all(torch.equal(p, q) for p, q in zip(select(V, x, scores, 12, work=work), first))
    assert int(head.max()) == 0


def test_select_nothing_alive_in_a_large_batch(V):
    x = torch.randn((300, 32768), device="cuda")
    done = torch.zeros((100, 3), dtype=torch.bool, device="cuda")
    done[::3] = True
    scores = torch.randn((100, 3), device="cuda")
    scores[::5] = -float("inf")
    x[3:6], x[299] = -float("inf"), float("nan")
    for _ in range(3):
        got = select(V, x, scores, 2, done=done, end=9)
        for g in range(100):
            if g % 5 == 0 or g == 1:
                assert got[1][g].tolist() == [-1, -1] and bool((got[0][g] == -float("inf")).all())
            elif g == 99:
                assert g % 3 == 0 and not bool(got[0][g].isnan().any())
            elif g % 3 == 0:
                assert sorted(got[0][g].tolist(), reverse=True) == got[0][g].tolist() == torch.sort(scores[g], descending=True).values[:2].tolist()
                assert got[2][g].tolist() == [9, 9]
            else:
                assert not bool(got[0][g].isnan().any()) and min(got[1][g].tolist()) >= 0


def test_select_all_candidates_in_one_segment(V):
    """The first 32 of 33 best tokens side by side, across borders of segments and chunks, and at both ends of a row."""
    for v, at in ((20000, 0), (20000, 240), (20000, 8180), (20000, 16370), (20000, 19967), (33, 0)):
        for dtype in DT.values():
            x = torch.zeros((2, v), dtype=dtype, device="cuda")
            x[1, at:at + 33] = 5.0 + torch.arange(33, device="cuda") % 7
            scores = torch.tensor([[0.0, -1.0]], device="cuda")
            assert check_select(V, x, scores.cpu(), 32)


def test_select_values_at_the_ends(V):
    """Masks of the type's lowest value, logits far apart, far common parts, scores far down."""
    for dtype in DT.values():
        low, high = torch.finfo(dtype).min, torch.finfo(dtype).max
        x = torch.full((4, 600), low, dtype=dtype, device="cuda")
        x[0, 5], x[0, 7] = 1.0, 3.0
        x[1] = high
        x[1, 9] = low
        x[2, 30] = high
        got = select(V, x, torch.tensor([[-3.0, -4.0, -1e30, 0.0]], device="cuda"), 12)
        # row 3: all of the lowest value, so equal and ahead of row 1's 599 equal ones; rows 0 and 2 by their gaps
        lse0 = np.log(np.exp(1.0) + np.exp(3.0))
        assert got[1][0, :2].tolist() == [0, 0] and got[2][0, :2].tolist() == [7, 5]
        assert abs(float(got[0][0, 0]) - (-3 + 3 - lse0)) < 1e-5
        assert got[1][0, 2:].tolist() == [3] * 10 and got[2][0, 2:].tolist() == list(range(10))
        assert abs(float(got[0][0, 2]) + np.log(600)) < 1e-5


@pytest.mark.parametrize("vocab", [300, 40000])
def test_select_weights_of_any_size(V, vocab):
    """Weights of powers of two leave the choice as it is, from denormals to the largest."""
    rng = np.random.RandomState(vocab)
    x = torch.from_numpy(rng.randn(9, vocab).astype(np.float32)).cuda()
    scores = torch.from_numpy(-rng.rand(3, 3).astype(np.float32)).cuda()
    weights = torch.tensor([[1.0, 0.5, 1.0], [2.0, 1.0, 1.0], [1.0, 1.0, 1.0]], device="cuda")
    done = torch.tensor([[0, 0, 0], [0, 1, 0], [0, 0, 1]], dtype=torch.uint8, device="cuda")
    want = select(V, x, scores, 12, 1.5, done, 7, weights)
    for power in (-140, -100, -78, -60, 60, 100, 125):
        got = select(V, x, scores, 12, 1.5, done, 7,
                     torch.from_numpy(np.ldexp(weights.cpu().numpy(), power)).cuda())
        assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])
        assert torch.all((got[0] - want[0]).abs() <= want[0].abs() * 2.0 ** -23)  # pairs or float64: roundings of neighbours


def test_select_spoiled_requests(V):
    """NaN or infinity in a live beam, its score or its weight: that request alone."""
    nan, inf = float("nan"), float("inf")
    x = torch.randn((16, 900), device="cuda")
    scores, weights = torch.randn((8, 2), device="cuda") - 3, torch.ones((8, 2), device="cuda")
    x[2, 899], x[5, 0], scores[3, 1], scores[4, 0], weights[5, 1], weights[6, 0] = nan, inf, nan, inf, 0.0, nan
    got = select(V, x, scores, 4, weights=weights)
    bad = torch.tensor([0, 1, 1, 1, 1, 1, 1, 0], dtype=torch.bool)
    assert torch.equal(got[0].isnan().all(1).cpu(), bad) and torch.equal(got[0].isnan().any(1).cpu(), bad)
    assert bool((got[1][bad] == -1).all()) and bool((got[2][bad] == -1).all())
    good = [0, 1, 14, 15]
    again = select(V, x[good], scores[[0, 7]], 4)
    for p, q in zip(got, again):
        assert torch.equal(p[[0, 7]], q)
    scores[3, 1] = scores[4, 0] = -inf  # a beam that brings nothing spoils nothing
    weights[5, 1] = weights[6, 0] = 1.0
    scores[1, 0] = scores[2, 1] = -inf
    got = select(V, x, scores, 4, weights=weights)
    assert not bool(got[0].isnan().any())


def test_select_nothing_left(V):
    x = torch.full((4, 50), -float("inf"), device="cuda")
    got = select(V, x, torch.zeros((2, 2), device="cuda"), 5)
    assert bool((got[0] == -float("inf")).all()) and bool((got[1] == -1).all()) and bool((got[2] == -1).all())
    x[2, 3] = 1.0
    got = select(V, x, torch.zeros((2, 2), device="cuda"), 5)
    assert got[1][1].tolist() == [0, -1, -1, -1, -1] and got[2][1].tolist() == [3, -1, -1, -1, -1] and float(got[0][1, 0]) == 0.0
    got = select(V, x[:0], torch.zeros((0, 2), device="cuda"), 5)
    assert got[0].shape == (0, 5)


def test_select_workspace_of_other_calls(V):
    """One workspace for calls of other sizes and types, one after the other."""
    work = V.beam_workspace(6, 8, 9000)
    for g, b, v, dtype in ((6, 8, 9000, "f32"), (1, 2, 100, "bf16"), (3, 4, 8999, "f16"), (6, 1, 9000, "f32"), (2, 8, 300, "bf16"), (6, 8, 9000, "bf16")):
        def check(seed):
            rng = np.random.RandomState(9 + seed)
            x = torch.from_numpy((3 * rng.randn(g * b, v)).astype(np.float32)).to(DT[dtype]).cuda()
            return check_select(V, x, (rng.randn(g, b) * 2).astype(np.float32), 7, work=work)

        some(check)


# ---------------------------------------------------------------- pages

def make_caches(V, layers, pages, heads, page, dim, order, gen):
    shape = (pages, heads, page, dim) if order == "head" else (pages, page, heads, dim)
    out = []
    for i in range(layers):
        k, v = (torch.randint(0, 256, shape, generator=gen, device="cuda", dtype=torch.uint8) for _ in range(2))
        if order == "token":
            k, v = k.transpose(1, 2), v.transpose(1, 2)
        out.append(V.KVCache(k, v, *(torch.rand((pages, heads), generator=gen, device="cuda") for _ in range(2)), ["int8", "e4m3"][i % 2]))
    return out


def check_reorder(V, caches, parents, lens, table, free, count, in_place, wide=0):
    g, b = parents.shape
    page = caches[0].page_size
    before = [[t.clone() for t in (c.k, c.v, c.k_scale, c.v_scale)] for c in caches]
    pages = V.BeamPages(caches, g, b)
    i32 = lambda x: torch.as_tensor(np.asarray(x, np.int32)).cuda()  # noqa: E731
    held = i32(np.full((table.shape[0], table.shape[1] + wide), -7))
    held[:, :table.shape[1]] = i32(table)
    t, f = held[:, :table.shape[1]], i32(free)
    out = None if in_place else torch.full_like(t, -9)
    was = table if in_place else np.full_like(table, -9)
    pages.reorder(i32(parents), i32(lens), t, f, i32([count]), out=out)
    want = S.beam_reorder(parents, lens, table, was, free, count, page)
    got = [t if in_place else out, pages.seq_lens, pages.status, f, pages.free_count[0]]
    for x, w, name in zip(got, want, "table lens status free left".split()):
        assert np.array_equal(x.cpu().numpy(), w), name
    if not in_place:
        assert np.array_equal(t.cpu().numpy(), table)
    assert bool((held[:, table.shape[1]:] == -7).all())
    for (k, v, ks, vs), c in zip(before, caches):
        for src, dst, used in want[5]:
            if not (0 <= src < c.n_pages and 0 <= dst < c.n_pages):
                continue
            k[dst, :, :used], v[dst, :, :used], ks[dst], vs[dst] = k[src, :, :used], v[src, :, :used], ks[src], vs[src]
        for x, y in zip((k, v, ks, vs), (c.k, c.v, c.k_scale, c.v_scale)):
            assert torch.equal(x, y)
    return want


def beams_state(rng, g, b, page, most, width, spare, first=False):
    """Lists of every request's beams with a shared part, lengths of their own behind it, and a free stack."""
    lens, table, at = np.zeros(g * b, np.int32), np.full((g * b, width), -1, np.int32), 0
    ids = rng.permutation(g * b * width + spare + 5).astype(np.int32)
    for i in range(g):
        length = int(rng.randint(0, most + 1))
        shared = int(rng.randint(0, length // page + 1))
        common = ids[at:at + shared]
        at += shared
        for j in range(b):
            n = length if rng.rand() < 0.6 else int(rng.randint(shared * page, most + 1))
            if first and j:
                n = 0
            m = S.cdiv(n, page)
            table[i * b + j, :min(shared, m)] = common[:m]
            table[i * b + j, shared:m] = ids[at:at + max(m - shared, 0)]
            at += max(m - shared, 0)
            lens[i * b + j] = n
    n_pages = g * b * width + spare + 5
    free = np.full(n_pages, -1, np.int32)
    free[:spare] = ids[at:at + spare]
    return lens, table, free, n_pages


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("g,b,page,most,width,layers,heads,dim,order", [
    (1, 1, 16, 40, 3, 1, 1, 16, "head"), (1, 4, 16, 70, 6, 2, 2, 64, "head"), (3, 5, 32, 400, 13, 2, 3, 48, "token"),
    (2, 32, 16, 90, 8, 1, 1, 32, "head"), (40, 3, 16, 64, 5, 1, 2, 16, "token"), (1, 8, 16, 5000, 313, 1, 1, 16, "head"),
    (9, 7, 48, 3000, 70, 1, 1, 32, "token"), (2, 2, 256, 700, 3, 65, 1, 16, "head"), (600, 2, 16, 40, 40, 1, 1, 16, "head")])
def test_reorder(V, in_place, g, b, page, most, width, layers, heads, dim, order):
    rng = np.random.RandomState(g * 31 + b + most)
    gen = torch.Generator("cuda").manual_seed(g + b)
    for kind in range(4):
        spare = g * b if kind != 3 else rng.randint(0, max(g * b // 3, 1))  # a stack that runs out
        lens, table, free, n = beams_state(rng, g, b, page, most, width, spare, first=kind == 0)
        if kind == 0:
            parents = np.zeros((g, b), np.int32)  # forked
        elif kind == 1:
            parents = rng.randint(-1, b, (g, b)).astype(np.int32)
        else:
            parents = np.minimum(rng.geometric(0.5, (g, b)) - 1, b - 1).astype(np.int32)
            parents[rng.rand(g) < 0.2] = -1
            parents[rng.rand(g) < 0.2] = np.arange(b)
        caches = make_caches(V, layers, n, heads, page, dim, order, gen)
        check_reorder(V, caches, parents, lens, table, free, spare, in_place, wide=kind)


@pytest.mark.parametrize("spare", [0, 1, 5, 13])
def test_reorder_short_of_pages(V, spare):
    """Forks that want a page for 7 children each from a stack that covers the first few: the others are empty."""
    lens = np.zeros(24, np.int32)
    lens[[0, 8, 16]] = 21, 5, 40
    table = np.full((24, 4), -1, np.int32)
    table[0, :2], table[8, 0], table[16, :3] = (3, 9), 4, (7, 1, 2)
    free = np.resize(np.arange(10, 34), 40).astype(np.int32)
    caches = make_caches(V, 1, 40, 2, 16, 16, "token", torch.Generator("cuda").manual_seed(spare))
    for in_place in (False, True):
        w = check_reorder(V, caches, np.zeros((3, 8), np.int32), lens, table, free, spare, in_place)
        assert (w[2] == S.NO_PAGES).sum() == 21 - spare and w[4] == 0


def test_reorder_bad_parents_and_lengths(V):
    rng = np.random.RandomState(2)
    gen = torch.Generator("cuda").manual_seed(2)
    lens, table, free, n = beams_state(rng, 4, 4, 16, 60, 4, 16)
    parents = np.array([[0, 4, -2, 2 ** 31 - 1], [1, 1, 1, 0], [3, 3, -2 ** 31, 3], [0, 0, 0, 0]], np.int32)
    lens[5], lens[11], lens[12] = -1, 65, 2 ** 31 - 1
    caches = make_caches(V, 1, n, 1, 16, 16, "head", gen)
    for in_place in (False, True):
        w = check_reorder(V, caches, parents, lens, table, free, 16, in_place)
    assert w[2].tolist() == [0, 2, 2, 2, 2, 2, 2, 0, 2, 2, 2, 2, 2, 2, 2, 2]
    # pages outside the cache, and a count that makes no sense, move but nothing is copied or lost
    lens, table, free, n = beams_state(rng, 2, 3, 16, 50, 4, 6)
    table[0, 0], table[3, 0] = 10 ** 9, -5
    free[4] = 2 ** 31 - 1
    for count in (-3, 0, 6, 10 ** 9):
        check_reorder(V, caches[:1], np.array([[0, 0, 0], [1, 1, 2]], np.int32), lens, table, np.resize(free, caches[0].n_pages), count, False)


def test_reorder_from_its_own_outputs(V):
    """An earlier call's lengths and count as the next one's, changed in place."""
    rng = np.random.RandomState(6)
    g, b, page = 300, 4, 16
    lens, table, free, n = beams_state(rng, g, b, page, 50, 4, g * b)
    caches = make_caches(V, 1, n, 1, page, 16, "head", torch.Generator("cuda").manual_seed(1))
    pages = V.BeamPages(caches, g, b)
    i32 = lambda x: torch.as_tensor(np.asarray(x, np.int32)).cuda()  # noqa: E731
    t, f = i32(table), i32(free)
    pages.seq_lens.copy_(i32(lens))
    pages.free_count.fill_(g * b)
    count = g * b
    for _ in range(4):
        parents = np.minimum(rng.geometric(0.5, (g, b)) - 1, b - 1).astype(np.int32)
        pages.reorder(i32(parents), pages.seq_lens, t, f, pages.free_count)
        table, lens, status, free, count, _ = S.beam_reorder(parents, lens, table, table, free, count, page)
        assert np.array_equal(t.cpu().numpy(), table) and np.array_equal(pages.seq_lens.cpu().numpy(), lens)
        assert np.array_equal(f.cpu().numpy(), free) and int(pages.free_count) == count and not status.any()


def test_two_searches_at_once(V):
    """Choices and pages of two batches on two streams, each with a workspace of its own, as they are alone."""
    gen = torch.Generator("cuda").manual_seed(8)
    rng = np.random.RandomState(8)
    i32 = lambda x: torch.as_tensor(np.asarray(x, np.int32)).cuda()  # noqa: E731
    cases = []
    for g, b, v in ((3, 5, 90000), (64, 4, 128256)):
        lens, table, free, n = beams_state(rng, g, b, 16, 60, 4, g * b)
        caches = make_caches(V, 2, n, 2, 16, 32, "head", gen)
        x = (3 * torch.randn((g * b, v), generator=gen, device="cuda")).bfloat16()
        cases.append(dict(x=x, scores=torch.randn((g, b), generator=gen, device="cuda"), work=V.beam_workspace(g, b, v), pages=V.BeamPages(caches, g, b),
                          lens=i32(lens), table=i32(table), free=i32(free), count=i32([g * b]), caches=caches, g=g, b=b, start=[c.k.clone() for c in caches]))
    done = []
    for together in (False, True):
        out = [[] for _ in cases]
        streams = [torch.cuda.Stream() for _ in cases]
        for c in cases:
            for k, s in zip(c["caches"], c["start"]):
                k.k.copy_(s)
        torch.cuda.synchronize()
        for _ in range(5):
            for i, (c, s) in enumerate(zip(cases, streams)):
                with torch.cuda.stream(s):
                    res = select(V, c["x"], c["scores"], c["b"], work=c["work"])
                    t, f = c["table"].clone(), c["free"].clone()
                    c["pages"].reorder(res[1], c["lens"], t, f, c["count"])
                    out[i].append([*res, t, f, c["pages"].seq_lens.clone()] + [k.k.clone() for k in c["caches"]])
                if not together:
                    s.synchronize()
        torch.cuda.synchronize()
        done.append(out)
    for one, two in zip(*done):
        for p, q in zip(one, two):
            assert all(torch.equal(y, z) for y, z in zip(p, q))


def test_reorder_steps_with_the_plan(V):
    """Forks, steps of the plan and choices in turn: pages are neither lost nor held twice, shared ones are full, and
    every row reads back the tokens of its own history."""
    g, b, P, H, D = 2, 4, 16, 1, 16
    rows, n_pages = g * b, 60
    cache = V.KVCache.empty(n_pages, H, D, P)
    pages = V.BeamPages([cache], g, b)
    plan = V.BatchPlan(rows, 64)
    i32 = dict(dtype=torch.int32, device="cuda")
    table, free = torch.full((rows, 12), -1, **i32), torch.arange(n_pages, **i32)
    count, lens = torch.tensor([n_pages], **i32), torch.zeros(rows, **i32)
    rng = np.random.RandomState(3)
    history = [[] for _ in range(rows)]

    def add(n_new):
        nonlocal count
        plan.build(lens, torch.tensor(n_new, **i32), table, free, count, P)
        assert not bool(plan.status.any())
        fresh = [rng.randint(-100, 101, n).tolist() for n in n_new]
        x = torch.zeros((64, H, D), device="cuda")
        flat = sum(fresh, [])
        x[:len(flat)] = torch.tensor(flat, device="cuda").float()[:, None, None]
        x[:len(flat), :, 0] = 127.0  # a scale of one for every page
        cache.append(x, -x, plan.slots)
        lens.copy_(plan.seq_lens)
        count = plan.free_count.clone()
        for r in range(rows):
            history[r] += fresh[r]

    def choose(parents):
        nonlocal count, history
        pages.reorder(torch.tensor(parents, **i32), lens, table, free, count)
        assert not bool(pages.status.any())
        lens.copy_(pages.seq_lens)
        count = pages.free_count.clone()
        history = [history[r // b * b + parents[r // b][r % b]][:] if parents[r // b][r % b] >= 0 else [] for r in range(rows)]

    def look():
        assert lens.tolist() == [len(h) for h in history]
        t, left = table.tolist(), int(count)
        held = {}
        for r in range(rows):
            for c in range(S.cdiv(len(history[r]), P)):
                held.setdefault(t[r][c], []).append((r, c))
        assert len(held) + left == n_pages and not set(held) & set(free[:left].tolist()) and len(set(free[:left].tolist())) == left
        for where in held.values():
            assert len({(r // b, c) for r, c in where}) == 1
            if len(where) > 1:
                assert all((c + 1) * P <= len(history[r]) for r, c in where)
        for r in range(rows):
            pos = torch.arange(len(history[r]), device="cuda")
            slots = table[r, pos // P].long() * P + pos % P
            k, v = (torch.empty((len(pos), H, D), device="cuda") for _ in range(2))
            cache.gather(slots, k, v)
            assert k[:, 0, 5].tolist() == history[r] and (-v[:, 0, 5]).tolist() == history[r]

    add([19, 0, 0, 0, 32, 0, 0, 0])
    choose([[0] * 4, [0] * 4])
    look()
    for i in range(24):
        add([1] * rows)
        look()
        choose([np.minimum(rng.geometric(0.5, b) - 1, b - 1).tolist() for _ in range(g)])
        look()
        if i == 12:  # one request ends, another begins in its rows
            choose([[-1] * 4, [0, 1, 2, 3]])
            look()
            add([5, 0, 0, 0, 0, 0, 0, 0])
            choose([[0] * 4, [0, 1, 2, 3]])
            look()
    choose([[-1] * 4, [-1] * 4])
    look()
    assert int(count) == n_pages


def test_search_step_captured_and_replayed(V):
    """Choice and pages in a graph; replays with other logits, each checked against the calls one by one."""
    g, b, v, P = 2, 3, 5000, 16
    gen = torch.Generator("cuda").manual_seed(4)
    rng = np.random.RandomState(4)
    lens, table, free, n = beams_state(rng, g, b, P, 60, 4, 12)
    caches, other = (make_caches(V, 2, n, 2, P, 32, "head", torch.Generator("cuda").manual_seed(5)) for _ in range(2))
    c = lambda a: torch.as_tensor(np.asarray(a, np.int32)).cuda()  # noqa: E731
    x, scores = torch.empty((g * b, v), device="cuda"), torch.zeros((g, b), device="cuda")
    work, pages = V.beam_workspace(g, b, v), V.BeamPages(caches, g, b)
    out = (torch.empty((g, b), device="cuda"), *(torch.empty((g, b), dtype=torch.int32, device="cuda") for _ in range(2)))
    t, f, cnt, ln, to = c(table), c(free), c([12]), c(lens), c(np.full_like(table, -1))

    def step():
        V.beam_select(x, scores, *out, work)
        pages.reorder(out[1], ln, t, f, cnt, out=to)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step()
    for _ in range(4):
        x.normal_(generator=gen).mul_(3)
        scores.normal_(generator=gen)
        f.copy_(c(free))
        graph.replay()
        want = select(V, x, scores, b)
        for p, q in zip(out, want):
            assert torch.equal(p, q)
        again, f2, to2 = V.BeamPages(other, g, b), c(free), c(np.full_like(table, -1))
        again.reorder(want[1], ln, t, f2, cnt, out=to2)
        m = S.beam_reorder(want[1].cpu().numpy(), lens, table, np.full_like(table, -1), free, 12, P)
        assert np.array_equal(again.seq_lens.cpu().numpy(), m[1]) and torch.equal(pages.seq_lens, again.seq_lens)
        assert torch.equal(f, f2) and torch.equal(pages.free_count, again.free_count)
        for r, length in enumerate(m[1]):
            assert torch.equal(to[r, :S.cdiv(int(length), P)], to2[r, :S.cdiv(int(length), P)])
        for p, q in zip(caches, other):
            for y, z in ((p.k, q.k), (p.v, q.v), (p.k_scale, q.k_scale), (p.v_scale, q.v_scale)):
                assert torch.equal(y, z)


# ---------------------------------------------------------------- the search

@pytest.fixture(scope="module")
def G(V):
    from paper_2609_38477_gb300 import generate

    return generate


def follow(d, prompt, tokens):
    """Log probability of each of tokens after the prompt, one at a time, in row 0 of an idle decoder."""
    row = lambda n: torch.tensor([n], dtype=torch.int32, device="cuda")  # noqa: E731
    for at in range(0, len(prompt), 16):
        logits = d.step(torch.tensor(prompt[at:at + 16], device="cuda"), row(len(prompt[at:at + 16])))
    out = []
    for t in tokens:
        out.append(torch.log_softmax(logits[-1].double(), 0).cpu().numpy())
        logits = d.step(torch.tensor([t], device="cuda"), row(1))
    d.step(torch.empty(0, dtype=torch.int64, device="cuda"), row(-1))
    return out


@pytest.mark.parametrize("power", [0.0, 0.8])
def test_beam_search(G, power, monkeypatch):
    """The choices are the oracle's on the logits that the search's own steps gave, and those are, for every row and
    step, the logits of the row's hypothesis decoded alone: within 1% of the largest, as another batch's float32 sums
    and the roundings to 16 and 8 bits that they tip over may move them."""
    d = G.synthetic_decoder("tiny", max_requests=8, n_pages=40)
    prompts, b, steps = [[5, 17, 42, 7, 99, 3, 8, 21, 6, 5, 4, 3, 2, 1, 9, 11, 13, 30], [200]], 4, 18
    plain, _ = d.beam_search(prompts, b, steps)
    end = int(plain[0, 0, 6])  # a token that a good hypothesis chooses early
    seen, step = [], d.step
    monkeypatch.setattr(d, "step", lambda tokens, n_new: seen.append(step(tokens, n_new)) or seen[-1])
    found, scores = d.beam_search(prompts, b, steps, end_token=end, length_power=power)
    monkeypatch.undo()
    assert int(d.free_count) == 40 and not bool(d.seq_lens.any())
    first = torch.zeros((2 * b, d.spec.vocab), device="cuda")
    first[0], first[b] = seen[1][-1], seen[2][-1]
    logits = [first] + seen[3:]
    assert len(logits) == steps
    history = [[()] * b for _ in prompts]
    sums, done = np.full((2, b), -np.inf), np.zeros((2, b), bool)
    sums[:, 0] = 0
    alone = {}
    for i, x in enumerate(logits):
        length = np.array([[len(h) if e else i + 1 for h, e in zip(hs, ds)] for hs, ds in zip(history, done)])
        s, beam, token, room = S.beam_select(x.double().cpu().numpy().reshape(2, b, -1), sums.astype(np.float32), 1.0, b, done, end,
                                             (length ** -power).astype(np.float32))
        assert room > 1e-5
        for g, prompt in enumerate(prompts):
            for r in range(b):
                if sums[g, r] > -np.inf and not done[g, r]:
                    h = history[g][r]
                    if (g, h) not in alone:
                        for n, row in enumerate(follow(d, prompt, list(h) + [0])):
                            alone[g, h[:n]] = row
                    want = alone[g, h]
                    assert float((torch.log_softmax(x[g * b + r].double(), 0).cpu() - torch.from_numpy(want)).abs().max()) <= 0.02 * np.abs(want).max()
        history = [[history[g][p] + (() if done[g, p] else (int(t),)) for p, t in zip(beam[g], token[g])] for g in range(2)]
        done = np.array([[done[g, p] or t == end for p, t in zip(beam[g], token[g])] for g in range(2)])
        sums = s.astype(np.float32)
    assert done.any() and not done.all()
    for g in range(2):
        for r in range(b):
            h = history[g][r]
            assert found[g, r].tolist() == list(h) + [end] * (steps - len(h))
            assert abs(float(scores[g, r]) - sums[g, r]) <= steps * OFF


def test_beam_search_without_pages(G):
    """Pages that do not last for the copies: NaN and -1, and all of them back at the end."""
    d = G.synthetic_decoder("tiny", max_requests=4, n_pages=3)
    found, scores = d.beam_search([[1, 2, 3]], 4, 4)
    assert bool(scores.isnan().all()) and bool((found[..., -1] == -1).all())
    assert int(d.free_count) == 3 and sorted(d.free[:3].tolist()) == [0, 1, 2]
    with pytest.raises(ValueError, match="max_requests"):
        d.beam_search([[1]], 5, 2)
    for bad in (([[]], 2, 2), ([[1]], 0, 2), ([[1]], 2, 0), ([], 2, 2), ([[1], [300]], 2, 2), ([[-1]], 2, 2), ([[1]], 2, 2, 300)):
        with pytest.raises(ValueError):
            d.beam_search(*bad)
    d.step(torch.tensor([5], device="cuda"), torch.tensor([1], dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError, match="under way"):
        d.beam_search([[1]], 2, 2)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("b,vocab", [(2, 40), (8, 128256)])
def test_select_slope_past_float32(V, dtype, b, vocab):
    """A weight times a scale above the largest float32: the beam's best token, whose total is 0 whatever they are,
    comes first, and its others last."""
    for weight, scale in ((2.0 ** 120, 2.0 ** 20), (3e38, 1.25), (2.0 ** 64, 2.0 ** 64)):
        x = torch.full((b, vocab), -200.0, dtype=DT[dtype], device="cuda")
        x[0, 7], x[1, 30] = 3.0, 4.0
        scores = torch.full((1, b), -float("inf"), device="cuda")
        scores[0, 0], scores[0, 1] = 0.0, -5.0
        weights = torch.ones((1, b), device="cuda")
        weights[0, 0] = weight
        for n in (1, 3):
            got = select(V, x, scores, n, scale, weights=weights)
            down = float(np.float32(-5 - scale * 204))
            assert got[1][0].tolist() == [0, 1, 1][:n] and got[2][0].tolist() == [7, 30, 0][:n]
            assert got[0][0].tolist() == [0.0, -5.0, down][:n]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,vocab", [(2, 4000), (8, 128256)])
def test_select_logits_further_apart_than_float32(V, dtype, b, vocab):
    """A beam's logits at both ends of the type, under a small weight: -6e35 of it comes before another's -1e36."""
    x = torch.full((b, vocab), -float("inf"), dtype=DT[dtype], device="cuda")
    x[0, 1], x[0, 300] = 3e38, -3e38
    x[1, 1], x[1, 300:2701:300] = 0.0, -1e37 * torch.arange(1, 10, device="cuda")  # segments of their own
    scores = torch.full((1, b), -float("inf"), device="cuda")
    scores[0, :2] = 0.0
    weights = torch.ones((1, b), device="cuda")
    weights[0, 0] = 0.01
    got = select(V, x, scores, 5, 0.1, weights=weights)
    assert list(zip(got[1][0].tolist(), got[2][0].tolist())) == [(0, 1), (1, 1), (0, 300), (1, 300), (1, 600)]
    want = torch.tensor([0.0, 0.0, 2 * float(x[0, 300]), float(x[1, 300]), float(x[1, 600])], dtype=torch.float64) * float(np.float32(0.1))
    assert bool(((got[0][0].double().cpu() - want).abs() <= want.abs() * U * (1 + 2.0 ** -20)).all())


def test_beam_search_steps_live_beams_alone(G, monkeypatch):
    """Ended hypotheses take part in no step and hold no page: as many tokens a step as there are hypotheses
    that go on, and as many pages as their rows list."""
    d = G.synthetic_decoder("tiny", max_requests=8, n_pages=60)
    prompts, b, steps = [[5, 17, 42, 7, 99, 3, 8, 21, 6, 5, 4, 3, 2, 1, 9, 11, 13, 30], [200]], 4, 16
    plain, _ = d.beam_search(prompts, b, steps)
    end = int(plain[0, 0, 6])  # a token that a good hypothesis chooses early
    live = []
    for n in range(1, steps):
        last = d.beam_search(prompts, b, n, end_token=end)[0][..., -1]
        live.append(int(((last != end) & (last >= 0)).sum()))
    assert min(live) < 2 * b  # some end
    taken, step = [], d.step

    def counted(tokens, n_new):
        out = step(tokens, n_new)
        pages = {p for row, n in zip(d.table.tolist(), d.seq_lens.tolist()) for p in row[:-(-max(n, 0) // d.page_size)]}
        taken.append((int((d.plan.slots >= 0).sum()), 60 - int(d.free_count), len(pages), int((d.seq_lens > 0).sum())))
        return out

    monkeypatch.setattr(d, "step", counted)
    d.beam_search(prompts, b, steps, end_token=end)
    assert [t[0] for t in taken[3:]] == live  # behind the prompts' three steps
    assert all(held == listed for _, held, listed, _ in taken)
    assert [t[3] for t in taken[3:]] == live
    assert int(d.free_count) == 60 and not bool(d.seq_lens.any())


@pytest.mark.parametrize("first,n_pages", [(70, 4), (30, 5)])
def test_beam_search_of_a_prompt_beside_one_without_pages(G, first, n_pages):
    """A prompt that finds no pages, for its own tokens or for those behind it, gives back what it has, and its
    neighbour is searched as if alone: the sums are those of the same tokens decoded one by one."""
    d = G.synthetic_decoder("tiny", max_requests=4, n_pages=n_pages)
    long, short, steps = [int(x) for x in np.random.RandomState(1).randint(0, 300, first)], [7, 30, 2, 41, 5, 99, 8], 14
    found, scores = d.beam_search([long, short], 2, steps)
    assert bool(scores[0].isnan().all()) and bool((found[0, :, -1] == -1).all())
    assert bool(scores[1].isfinite().all()) and bool((found[1] >= 0).all())
    assert int(d.free_count) == n_pages and not bool(d.seq_lens.any())
    for r in range(2):
        tokens = found[1, r].tolist()
        rows = follow(d, short, tokens)
        want = sum(row[t] for row, t in zip(rows, tokens))
        assert abs(float(scores[1, r]) - want) <= 0.02 * sum(np.abs(row).max() for row in rows)


# ---------------------------------------------------------------- large batches (100 MB of logits and more: warps stream through them)

def large_logits(dtype, rows, v, stride, gen):
    assert rows * v * torch.empty(0, dtype=DT[dtype]).element_size() >= 96 << 20 and v >= 16384
    flat = torch.full((rows, stride), float("nan"), dtype=DT[dtype], device="cuda")  # between rows: nothing that may be read
    x = flat[:, :v]
    for r in range(0, rows, 64):
        x[r:r + 64] = 3 * torch.randn((min(64, rows - r), v), generator=gen, device="cuda")
    return x


@pytest.mark.parametrize("dtype,g,b,v,stride,n,scale", [("f32", 63, 8, 50003, 50008, 5, 0.7), ("bf16", 126, 8, 50003, 50008, 8, 1.0),
                                                        ("f16", 100, 4, 128256, 128256, 3, 1.5), ("bf16", 30, 32, 56001, 56008, 32, 1.0),
                                                        ("f32", 1501, 1, 16777, 16780, 2, 1.0)])
def test_select_large(V, dtype, g, b, v, stride, n, scale):
    """Every request of a large batch against the oracle: masked tokens and rows, finished and empty beams, weights,
    and requests spoiled by a logit, a score or a weight."""
    def check(seed):
        rng, gen = np.random.RandomState(g + b + 1000 * seed), torch.Generator("cuda").manual_seed(v + seed)
        x = large_logits(dtype, g * b, v, stride, gen)
        for r in rng.randint(0, g * b, g):
            x[r, rng.randint(0, v, v // 3)] = -float("inf")
        x[rng.randint(0, g * b, 3)] = -float("inf")
        scores = (-5 + 2 * rng.randn(g, b)).astype(np.float32)
        scores[rng.rand(g, b) < 0.1] = -np.inf
        done = rng.rand(g, b) < 0.2
        weights = (rng.randint(3, 30, (g, b)) ** -0.7).astype(np.float32)
        scores[:5, 0], done[:5, 0] = -1.0, False
        x[0, v - 1], x[b, 4096] = float("nan"), float("inf")
        scores[2, 0], weights[3, 0], scores[4, 0] = np.nan, 0.0, np.inf
        return check_select(V, x, scores, n, scale, done, int(rng.randint(v)), weights)

    some(check)


@pytest.mark.parametrize("dtype,rows", [("f32", 200), ("bf16", 400), ("f16", 400)])
def test_select_equal_rows_of_a_large_batch(V, dtype, rows):
    """Equal rows, dealt to the SMs at other places each: scores that are each token's log probability and equal to the
    bit, ties by beam and token."""
    v, b, n = 128256, 5, 12
    g = rows // b
    row = (3 * torch.randn(v, generator=torch.Generator("cuda").manual_seed(7), device="cuda")).to(DT[dtype])
    x = row.expand(rows, v).contiguous()
    assert x.nbytes >= 96 << 20
    scores = torch.zeros((g, b), device="cuda")
    scores[7], scores[8, :4], scores[9, 0] = -float("inf"), -float("inf"), -float("inf")
    score, beam, token = select(V, x, scores, n)
    logp = torch.log_softmax(row.double(), 0)
    order = torch.sort(row.float(), descending=True, stable=True)
    ties = [order.indices[order.values == y].tolist() for y in torch.unique(order.values).flip(0)[:n]]
    of_token = {}
    for i in range(g):
        beams = [] if i == 7 else [4] if i == 8 else [1, 2, 3, 4] if i == 9 else list(range(b))
        want = [(k, t) for same in ties for k in beams for t in same][:n] or [(-1, -1)] * n
        assert list(zip(beam[i].tolist(), token[i].tolist())) == want
        for t, s in zip(token[i].tolist(), score[i].tolist()):
            if t < 0:
                assert s == -float("inf")
                continue
            assert abs(s - float(logp[t])) <= OFF + abs(s) * U
            assert of_token.setdefault(float(row[t]), s) == s


def test_select_nothing_alive_in_a_batch_that_streams(V):
    """Requests of finished, empty and masked beams between live ones, 100 MB of logits; the workspace stays good."""
    g, b, v = 260, 3, 32768
    x = torch.randn((g * b, v), device="cuda")
    assert x.nbytes >= 96 << 20
    done = torch.zeros((g, b), dtype=torch.bool, device="cuda")
    done[::3] = True
    scores = torch.randn((g, b), device="cuda")
    scores[::5] = -float("inf")
    x[3:6] = -float("inf")
    x[9:12] = float("nan")  # request 3: finished, so nothing of it is read
    work = V.beam_workspace(g, b, v)
    for _ in range(3):
        score, beam, token = (t.tolist() for t in select(V, x, scores, 2, done=done, end=9, work=work))
        for i in range(g):
            if i % 5 == 0 or i == 1:
                assert beam[i] == token[i] == [-1, -1] and score[i] == [-float("inf")] * 2
            elif i % 3 == 0:
                assert token[i] == [9, 9] and score[i] == torch.sort(scores[i], descending=True).values[:2].tolist()
                assert score[i] == [float(scores[i, k]) for k in beam[i]]
            else:
                assert min(beam[i]) >= 0 and score[i][0] >= score[i][1] > -20
    scores[:] = -float("inf")  # nobody's
    got = select(V, x, scores, 2, done=done, end=9, work=work)
    assert bool((got[0] == -float("inf")).all()) and bool((got[1] == -1).all()) and bool((got[2] == -1).all())
    assert int(work[:2 * 8192 * 4 + 16].max()) == 0


# ---------------------------------------------------------------- pages of models of real size (copies by a launch of their own)

LARGE = [(32, 8, 16, 600, 40, 2, 8, 128, "head"), (120, 4, 16, 1400, 90, 1, 2, 64, "token"), (60, 6, 48, 4000, 84, 3, 2, 80, "token"),
         (9, 32, 32, 2000, 63, 70, 1, 64, "head")]


def copies_apart(g, b, page, layers, heads, dim, width):
    """More than 1 MB may have to be copied, and the lists take more CTAs than one."""
    return g * b * layers * 2 * heads * (page - 1) * dim > 1 << 20 and g * -(-width // 32) > 16


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("g,b,page,most,width,layers,heads,dim,order", LARGE)
def test_reorder_large(V, in_place, g, b, page, most, width, layers, heads, dim, order):
    assert copies_apart(g, b, page, layers, heads, dim, width)
    rng = np.random.RandomState(g + b)
    gen = torch.Generator("cuda").manual_seed(g)
    for kind in range(3):
        spare = g * b if kind < 2 else g  # a stack that runs out
        lens, table, free, n = beams_state(rng, g, b, page, most, width, spare, first=kind == 0)
        parents = np.zeros((g, b), np.int32) if kind == 0 else np.minimum(rng.geometric(0.5, (g, b)) - 1, b - 1).astype(np.int32)
        if kind:
            parents[rng.rand(g) < 0.1] = -1
            parents[rng.rand(g, b) < 0.05] = -1
        caches = make_caches(V, layers, n, heads, page, dim, order, gen)
        want = check_reorder(V, caches, parents, lens, table, free, spare, in_place)
        assert len(want[5]) > 8
        del caches


def test_reorder_large_captured_and_replayed(V):
    """Both launches in a graph, replayed with other parents, each against the oracle; and the graph beside calls on another stream."""
    g, b, page, most, width, layers, heads, dim, order = LARGE[0]
    rng = np.random.RandomState(11)
    i32 = lambda x: torch.as_tensor(np.asarray(x, np.int32)).cuda()  # noqa: E731
    lens, table, free, n = beams_state(rng, g, b, page, most, width, g * b)
    caches, others = (make_caches(V, layers, n, heads, page, dim, order, torch.Generator("cuda").manual_seed(3)) for _ in range(2))
    start = [t.clone() for c in caches for t in (c.k, c.v, c.k_scale, c.v_scale)]
    state = lambda cs: [t for c in cs for t in (c.k, c.v, c.k_scale, c.v_scale)]  # noqa: E731
    pages, beside = V.BeamPages(caches, g, b), V.BeamPages(others, g, b)
    parents, t, f, cnt, ln = i32(np.zeros((g, b))), i32(table), i32(free), i32([g * b]), i32(lens)
    to = torch.full_like(t, -9)
    s, other = torch.cuda.Stream(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        pages.reorder(parents, ln, t, f, cnt, out=to)
    for _ in range(3):
        p = np.minimum(rng.geometric(0.5, (g, b)) - 1, b - 1).astype(np.int32)
        p2 = p[::-1].copy()
        parents.copy_(i32(p))
        f.copy_(i32(free))
        to.fill_(-9)
        f2, to2, parents2 = i32(free), torch.full_like(t, -9), i32(p2)
        for now in (caches, others):
            for x, y in zip(state(now), start):
                x.copy_(y)
        torch.cuda.synchronize()
        graph.replay()
        beside.reorder(parents2, ln, t, f2, cnt, out=to2, stream=other)
        torch.cuda.synchronize()
        for q, now, got_to, got_f, obj in ((p, caches, to, f, pages), (p2, others, to2, f2, beside)):
            want = S.beam_reorder(q, lens, table, np.full_like(table, -9), free, g * b, page)
            for x, y in ((got_to, want[0]), (obj.seq_lens, want[1]), (obj.status, want[2]), (got_f, want[3]), (obj.free_count[0], want[4])):
                assert np.array_equal(x.cpu().numpy(), y)
            model = [x.clone() for x in start]
            for src, dst, used in want[5]:
                for i, x in enumerate(model):
                    if i % 4 < 2:
                        x[dst, :, :used] = x[src, :, :used]
                    else:
                        x[dst] = x[src]
            assert all(torch.equal(x, y) for x, y in zip(state(now), model))


# ---------------------------------------------------------------- the largest sizes

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("odd", [0, 1])
def test_select_of_the_largest_vocabulary(V, dtype, odd):
    """2^27 tokens, by streaming warps and (rows that do not allow wide loads) by a CTA per chunk: tokens exactly, the score
    to the roundings of 2^14 sums of sums that an eighth of a row's chunks join (2^15 u at most, u = 2^-24; 2^13 sums of
    2048 logits or more in order, and a term's own)."""
    v, n = 1 << 27, 20
    x = torch.randn(v + odd, generator=torch.Generator("cuda").manual_seed(odd), device="cuda").to(DT[dtype])[odd:].view(1, v)
    x[0, [5, v // 2, v - 1]] = torch.tensor([9.0, 8.0, 10.0], device="cuda").to(DT[dtype])
    score, beam, token = select(V, x, torch.zeros((1, 1), device="cuda"), n)
    top = torch.topk(x[0].float(), 4 * n)
    order = sorted(zip((-top.values).tolist(), top.indices.tolist()))[:n]
    assert order[-1][0] < -float(top.values[-1])  # no ties at the end
    assert token[0].tolist() == [t for _, t in order] and token[0, :3].tolist() == [v - 1, 5, v // 2] and bool((beam == 0).all())
    lse = float(torch.logsumexp(x[0].double(), 0))
    for s, (z, _) in zip(score[0].tolist(), order):
        assert abs(s - (-z - lse)) <= 2.0 ** -9 + abs(s) * U


@pytest.mark.parametrize("g,b,v", [(8192, 1, 16384), (256, 32, 16384), (8192, 1, 200), (256, 32, 300)])
def test_select_of_the_most_rows(V, g, b, v):
    """8192 rows, streaming and not, two thirds of whose requests bring nothing or one finished beam: as in smaller batches."""
    x = (3 * torch.randn((g * b, v), generator=torch.Generator("cuda").manual_seed(b), device="cuda")).half()
    scores = torch.rand((g, b), generator=torch.Generator("cuda").manual_seed(v), device="cuda") - 3
    done = torch.zeros((g, b), dtype=torch.bool, device="cuda")
    scores[1::3], done[2::3] = -float("inf"), True
    work = V.beam_workspace(g, b, v)
    for _ in range(2):
        score, beam, token = select(V, x, scores, 3, done=done, end=7, work=work)
        assert bool((token[1::3] == -1).all()) and bool((score[1::3] == -float("inf")).all())
        best = scores[2::3].topk(min(b, 3), 1)
        assert torch.equal(score[2::3, :min(b, 3)], best.values) and bool((token[2::3, :min(b, 3)] == 7).all())
        live = torch.arange(0, g, 3, device="cuda")
        total = torch.log_softmax(x.double().view(g, b, v)[live], 2) + scores[live].double()[..., None]
        want = total.flatten(1).topk(4, 1)
        apart = (want.values[:, :3] - want.values[:, 1:] > 2 * OFF).all(1)  # no neighbours too close to tell, and no ties
        assert float(apart.double().mean()) > 0.7
        got = (beam[live].long() * v + token[live])[apart]
        assert torch.equal(got, want.indices[:, :3][apart])
        assert bool(((score[live].double() - want.values[:, :3]).abs() <= OFF + want.values[:, :3].abs() * U).all())
    assert int(work[:2 * 8192 * 4 + 16].max()) == 0


@pytest.mark.parametrize("g,b,page,most,width", [(8192, 1, 16, 40, 3), (256, 32, 16, 60, 4), (1, 4, 16, 300000, 18750), (2, 32, 16, 20000, 1250)])
def test_reorder_of_the_most_rows_and_the_longest_lists(V, g, b, page, most, width):
    rng = np.random.RandomState(g + width)
    for in_place in (True, False):
        lens, table, free, n = beams_state(rng, g, b, page, most, width, g * b)
        parents = rng.randint(-1, b, (g, b)).astype(np.int32)
        check_reorder(V, make_caches(V, 1, n, 1, page, 16, "head", torch.Generator("cuda").manual_seed(g)), parents, lens, table, free, g * b, in_place)
