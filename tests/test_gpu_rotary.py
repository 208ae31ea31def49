"""Rotary positions and the rotating cache write on the GPU against the fp64 oracle.

Tolerances, with u = 2^-24.  Angles: the fraction of a turn is cut to 2^-32 of one
and its rest, at most an eighth, rounded to 25 bits (2^-28 of a turn at most):
together 2 pi 2^-27.9 < 0.42 u' with u' = 2^-24; sincospif is within 2 units in the
last place of numbers up to 1 (2 u), and the factor `scale` rounds once more (u): at
most 4 u scale.  Rotation: a product and a fused sum, each rounded once: 2 u times
the sum of the two products' magnitudes, then half a step of the output's type.
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


@pytest.fixture(scope="module")
def V():
    from paper_2609_38477_gb300 import build

    build.build()
    from paper_2609_38477_gb300 import seedq, serving

    seedq.lib()
    return serving


def angles_of(V, rotary, positions):
    cs = torch.empty((len(positions), rotary.half, 2), device="cuda")
    rotary.angles(torch.tensor(positions, dtype=torch.int32, device="cuda"), cs)
    return cs


# ---------------------------------------------------------------- angles

@pytest.mark.parametrize("rot,rule,factor", [(2, "none", 1.0), (24, "linear", 4.0), (128, "bands", 8.0), (96, "ramp", 4.0), (64, "base", 2.0),
                                             (1024, "none", 1.0)])
def test_angles(V, rot, rule, factor):
    w, scale = V.rotary_frequencies(rot, 500000.0 if rot == 128 else 10000.0, rule, factor)
    positions = [0, 1, 2, 7, 1000, 131071, 10 ** 6 + 3, 2 ** 24 + 1, 2 ** 31 - 1, -1, -5, -131071, -2 ** 31]
    cs = angles_of(V, V.Rotary(w, scale=scale), positions)
    want = S.rotary_angles(positions, w, scale)
    assert np.abs(cs.double().cpu().numpy() - want).max() <= 4 * U * scale
    assert bool((cs[0, :, 0] == torch.tensor(scale, dtype=torch.float32)).all()) and bool((cs[0, :, 1] == 0).all())


def test_angles_of_frequencies_above_a_turn_and_below_zero(V):
    """Whole turns vanish, negative frequencies turn backwards; and a factor of any size."""
    w = [2 * np.pi * 5, -0.3, 100.0, 0.0, 1e-12, 3.0]
    positions = [0, 1, 3, -7, 12345, 2 ** 30]
    for scale in (1.0, -2.5, 0.0, 1e30):
        cs = angles_of(V, V.Rotary(w, scale=scale), positions)
        assert np.abs(cs.double().cpu().numpy() - S.rotary_angles(positions, w, scale)).max() <= 4 * U * abs(scale)


# ---------------------------------------------------------------- rotation

def check_rotate(V, x, cs, rotary, layout, out, inplace=False):
    want, size = S.rotate(x.double().cpu().numpy(), cs.double().cpu().numpy(), layout)
    rotary.rotate(x, cs, out)
    got = out.double().cpu().numpy()
    info = torch.finfo(out.dtype)
    # half a step of the type (of its subnormals: half their distance) on what the sums may be off by
    off = 2 * U * size
    tol = off + (np.abs(want) + off) * info.eps / 2 + info.tiny * info.eps / 2
    tol = np.where(size > 0, tol, np.abs(want) * info.eps / 2 + info.tiny * info.eps / 2)
    assert np.all(np.abs(got - want) <= tol)
    return got


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("ti,to", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16"), ("bf16", "f32"), ("f16", "bf16"), ("f32", "f16")])
@pytest.mark.parametrize("n,heads,dim,rot", [(1, 1, 2, 2), (1, 40, 128, 128), (16, 5, 32, 32), (333, 3, 96, 24), (7, 4, 80, 20), (65, 2, 64, 6),
                                             (5, 9, 256, 128), (3, 1, 99, 50), (2, 3, 1000, 998), (1100, 33, 64, 64)])
def test_rotate(V, layout, ti, to, n, heads, dim, rot):
    rng = np.random.RandomState(n + heads + dim + rot)
    rotary = V.Rotary(V.rotary_frequencies(rot)[0], layout, scale=1.25)
    cs = angles_of(V, rotary, rng.randint(0, 200000, n).tolist())
    x = torch.from_numpy(rng.randn(n, heads, dim).astype(np.float32)).to(DT[ti]).cuda()
    out = torch.full((n, heads, dim), 9.0, dtype=DT[to], device="cuda")
    check_rotate(V, x, cs, rotary, layout, out)
    if ti == to:  # where it lies: the same numbers
        y = x.clone()
        rotary.rotate(y, cs, y)
        assert torch.equal(y, out)


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("dtype", list(DT))
def test_rotate_strides(V, layout, dtype):
    """Heads of a fused projection at odd offsets, heads before tokens, one row for all tokens; neighbours stay."""
    n, h, d, r = 9, 4, 64, 48
    rng = np.random.RandomState(1)
    rotary = V.Rotary(V.rotary_frequencies(r)[0], layout)
    cs = angles_of(V, rotary, rng.randint(0, 5000, n).tolist())
    for shift, width in ((0, 3 * h * d), (1, 3 * h * d + 1), (4, 3 * h * d + 4), (2, 3 * h * d + 2)):
        flat = torch.from_numpy(rng.randn(shift + n * width).astype(np.float32)).to(DT[dtype]).cuda()
        before = flat.clone()
        x = flat[shift:].view(n, width)[:, h * d:2 * h * d].view(n, h, d)
        out = torch.empty((n, h, d), dtype=DT[dtype], device="cuda")
        check_rotate(V, x, cs, rotary, layout, out)
        rotary.rotate(x, cs, x)  # in its place
        assert torch.equal(x, out)
        x.copy_(before[shift:].view(n, width)[:, h * d:2 * h * d].view(n, h, d))
        assert torch.equal(flat, before)
    x = torch.from_numpy(rng.randn(h, n, d).astype(np.float32)).to(DT[dtype]).cuda().transpose(0, 1)
    out = torch.empty((h, n, d), dtype=DT[dtype], device="cuda").transpose(0, 1)
    check_rotate(V, x, cs, rotary, layout, out)
    x = x[:1].expand(n, h, d)
    check_rotate(V, x, cs, rotary, layout, out)


def test_rotate_not_a_number_stays_in_its_pair(V):
    rotary = V.Rotary(V.rotary_frequencies(32)[0])
    cs = angles_of(V, rotary, [5, 6])
    x = torch.randn(2, 2, 48, device="cuda")
    clean, out = torch.empty_like(x), torch.empty_like(x)
    rotary.rotate(x, cs, clean)
    x[0, 1, 3], x[1, 0, 40], x[1, 1, 20] = float("nan"), float("inf"), float("nan")
    rotary.rotate(x, cs, out)
    bad = torch.zeros_like(x, dtype=torch.bool)
    bad[0, 1, [3, 19]] = bad[1, 1, [4, 20]] = True
    assert bool(out[bad].isnan().all()) and out[1, 0, 40] == float("inf")
    bad[1, 0, 40] = True
    assert torch.equal(out[~bad], clean[~bad])


def test_nothing_to_rotate(V):
    rotary = V.Rotary([1.0])
    cs = torch.empty((0, 1, 2), device="cuda")
    rotary.angles(torch.empty(0, dtype=torch.int32, device="cuda"), cs)
    rotary.rotate(torch.empty((0, 3, 2), device="cuda"), cs, torch.empty((0, 3, 2), device="cuda"))
    cs = angles_of(V, rotary, [1, 2])
    rotary.rotate(torch.empty((2, 0, 2), device="cuda"), cs, torch.empty((2, 0, 2), device="cuda"))


# ---------------------------------------------------------------- on the way into the cache

def new_cache(V, pages, heads, page, dim, kind, order="head"):
    shape = (pages, heads, page, dim) if order == "head" else (pages, page, heads, dim)
    t = [torch.full(shape, 0x55, dtype=torch.uint8, device="cuda") for _ in range(2)]
    if order == "token":
        t = [x.transpose(1, 2) for x in t]
    return V.KVCache(*t, *(torch.full((pages, heads), 77.0, device="cuda") for _ in range(2)), kind)


def same(a, b):
    for x, y in ((a.k, b.k), (a.v, b.v)):
        assert torch.equal(x, y)
    for x, y in ((a.k_scale, b.k_scale), (a.v_scale, b.v_scale)):
        assert torch.equal(x.nan_to_num(-1), y.nan_to_num(-1))


def both_ways(V, a, b, k, v, slots, rotary, cs, q=None, q_out=None):
    """The call, and its two halves: keys rotated in float32, then appended."""
    a.append_rotary(k, v, slots, rotary, cs, q=q, q_out=q_out)
    turned = torch.empty(k.shape, device="cuda")
    rotary.rotate(k, cs, turned)
    b.append(turned, v.float().contiguous(), slots)
    same(a, b)
    if q is not None:
        want = torch.empty_like(q_out)
        rotary.rotate(q, cs, want)
        assert torch.equal(q_out, want)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("heads,page,dim,rot,order", [(1, 16, 16, 16, "head"), (3, 32, 80, 80, "token"), (8, 16, 128, 128, "head"),
                                                      (2, 256, 64, 32, "token"), (5, 48, 256, 64, "head"), (3, 64, 96, 24, "head"),
                                                      (4, 256, 128, 128, "token"), (2, 32, 48, 38, "head"), (7, 128, 32, 2, "token"),
                                                      (2, 240, 112, 112, "head")])
def test_append_rotary_in_steps(V, kind, dtype, layout, heads, page, dim, rot, order):
    """Runs of every length and offset, pages that fill up and are reused, slots outside; queries of another type out."""
    rng = np.random.RandomState(heads * page + dim)
    a, b = (new_cache(V, 6, heads, page, dim, kind, order) for _ in range(2))
    rotary = V.Rotary(V.rotary_frequencies(rot)[0], layout, scale=1.1)
    at = {}
    for step in range(7):
        slots = []
        for p in rng.permutation(6)[:rng.randint(1, 6)]:
            o = at.get(p, 0)
            if o >= page or rng.rand() < 0.2:
                o = 0
            m = min(page - o, int(rng.choice([1, 2, 3, 15, 16, 17, 33, page])))
            slots += list(range(p * page + o, p * page + o + m))
            at[p] = o + m
            if rng.rand() < 0.3:
                slots.append(int(rng.choice([-1, 6 * page, 2 ** 40, -2 ** 40])))
        n = len(slots)
        size = 2.0 ** rng.randint(-9, 9, (2, n, 1, 1))
        odd = step % 2  # rows that begin at an odd element
        flat = torch.zeros(2 * n * heads * dim + odd, dtype=DT[dtype], device="cuda")
        x = flat[odd:].view(2, n, heads, dim)
        x.copy_(torch.from_numpy((size * rng.randn(2, n, heads, dim)).astype(np.float32)))
        cs = angles_of(V, rotary, rng.randint(0, 100000, n).tolist())
        q = torch.from_numpy(rng.randn(n, 3 * heads, dim).astype(np.float32)).to(DT[dtype]).cuda() if step != 3 else None
        q_out = torch.full((n, 3 * heads, dim), 5.0, dtype=list(DT.values())[step % 3], device="cuda") if q is not None else None
        both_ways(V, a, b, x[0], x[1], torch.tensor(slots, device="cuda"), rotary, cs, q, q_out)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("layout,rot", [("half", 64), ("pairs", 64), ("half", 32), ("half", 20)])
def test_append_rotary_against_the_oracle(V, kind, layout, rot):
    """Codes of keys turned in fp64: equal, or where the number lies within the rotation's
    rounding of the border between two codes, one of the two."""
    rng = np.random.RandomState(rot)
    P, H, D, n = 16, 3, 64, 40
    rotary = V.Rotary(V.rotary_frequencies(rot)[0], layout)
    c = new_cache(V, 4, H, P, D, kind)
    slots = list(range(16, 56))
    cs = angles_of(V, rotary, (3000 + np.arange(n)).tolist())
    x = torch.from_numpy(rng.randn(2, n, H, D).astype(np.float32)).bfloat16().cuda()
    c.append_rotary(x[0], x[1], torch.tensor(slots, device="cuda"), rotary, cs)
    turned, size = S.rotate(x[0].double().cpu().numpy(), cs.double().cpu().numpy(), layout)
    for codes, scales, want, off in ((c.k, c.k_scale, turned, 2 * U * size), (c.v, c.v_scale, x[1].double().cpu().numpy(), 0 * size)):
        wc, ws = np.zeros((4, H, P, D), np.uint8), np.zeros((4, H))
        S.append(wc, ws, want, slots, P, kind)
        got, gs = codes.cpu().numpy().view(np.uint8), scales.double().cpu().numpy()
        for t, s in enumerate(slots):
            b, o = s // P, s % P
            assert np.array_equal(gs[b], ws[b])
            g, w = S.decode(got[b, :, o], kind), S.decode(wc[b, :, o], kind)
            border = (g + w) / 2 * ws[b][:, None]
            assert np.all((g == w) | (np.abs(want[t] - border) <= off[t]))
        assert np.mean(got[1:3] == wc[1:3]) > 0.999


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_append_rotary_extremes(V, kind):
    """Zeros, numbers at the type's ends, NaN and infinities; scales that are no powers of two, as a caller may have."""
    rotary = V.Rotary(V.rotary_frequencies(16)[0])
    for first in (0.0, 3.0, float("nan"), 0.3):
        a, b = (new_cache(V, 12, 1, 16, 16, kind) for _ in range(2))
        rows = [0.0, 1e-45, 1e-39, 1.1754944e-38, 1e38, 127.0, 448.0, -0.0, float("inf"), float("-inf"), float("nan"), 5.0]
        if first == 0.3:
            for c in (a, b):
                c.k_scale.fill_(0.3)
                c.v_scale.fill_(0.3)
                c.k.fill_(3)
                c.v.fill_(3)
        else:
            x = torch.full((12, 1, 16), first, device="cuda")
            cs = angles_of(V, rotary, [3] * 12)
            both_ways(V, a, b, x, x, torch.arange(12, device="cuda") * 16, rotary, cs)
        x = torch.zeros((12, 1, 16), device="cuda")
        x[:, 0, 5] = torch.tensor(rows)
        cs = angles_of(V, rotary, list(range(12)))
        both_ways(V, a, b, x, x, torch.arange(12, device="cuda") * 16 + 1, rotary, cs)


def test_append_rotary_without_tokens(V):
    rotary = V.Rotary([1.0, 0.5])
    c = new_cache(V, 2, 2, 16, 16, "int8")
    e = torch.empty((0, 2, 16), device="cuda")
    c.append_rotary(e, e, torch.empty(0, dtype=torch.int64, device="cuda"), rotary, torch.empty((0, 2, 2), device="cuda"), q=e, q_out=e)
    assert bool((c.k == 0x55).all())


def test_append_rotary_of_many_single_tokens(V):
    """Every token a page of its own, more than the warps of a launch's first wave, queries in place."""
    rotary = V.Rotary(V.rotary_frequencies(128)[0])
    n, h = 700, 9
    a, b = (new_cache(V, n, h, 16, 128, "int8") for _ in range(2))
    x = torch.randn((2, n, h, 128), device="cuda")
    cs = angles_of(V, rotary, list(range(n)))
    q = torch.randn((n, 2 * h, 128), device="cuda")
    want = torch.empty_like(q)
    rotary.rotate(q, cs, want)
    slots = torch.randperm(n, device="cuda") * 16
    a.append_rotary(x[0], x[1], slots, rotary, cs, q=q, q_out=q)
    assert torch.equal(q, want)
    k = torch.empty_like(x[0])
    rotary.rotate(x[0], cs, k)
    b.append(k, x[1], slots)
    for y, z in ((a.k, b.k), (a.v, b.v)):
        assert torch.equal(y[:, :, 0], z[:, :, 0])


@pytest.mark.parametrize("page", [16, 64])
def test_rotation_captured_and_replayed(V, page):
    """A step's angles, rotation and cache write in a graph, replayed with other positions and numbers."""
    n, h, d = 5, 3, 64
    rotary = V.Rotary(V.rotary_frequencies(d)[0])
    a, b = (new_cache(V, 8, h, page, d, "int8") for _ in range(2))
    for c in (a, b):
        c.k.zero_()
        c.v.zero_()
    pos = torch.zeros(n, dtype=torch.int32, device="cuda")
    slots = torch.zeros(n, dtype=torch.int64, device="cuda")
    x, q = torch.randn((2, n, h, d), device="cuda"), torch.randn((n, 2 * h, d), device="cuda")
    cs, q_out, direct = torch.empty((n, d // 2, 2), device="cuda"), torch.empty_like(q), torch.empty_like(q)

    def step():
        rotary.angles(pos, cs)
        a.append_rotary(x[0], x[1], slots, rotary, cs, q=q, q_out=q_out)
        rotary.rotate(q, cs, direct)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step()
    for i in range(3):
        pos.copy_(torch.randint(0, 50000, (n,)))
        slots.copy_(torch.arange(n) + i * n + page)
        x.normal_()
        q.normal_()
        graph.replay()
        cs2 = torch.empty_like(cs)
        rotary.angles(pos, cs2)
        assert torch.equal(cs, cs2) and torch.equal(q_out, direct)
        k = torch.empty_like(x[0])
        rotary.rotate(x[0], cs2, k)
        b.append(k, x[1], slots)
        same(a, b)


def test_other_streams(V):
    """Calls on a stream of their own, given and current."""
    rotary = V.Rotary(V.rotary_frequencies(64)[0])
    x = torch.randn((300, 8, 64), device="cuda")
    pos = torch.arange(300, dtype=torch.int32, device="cuda")
    want = torch.empty_like(x)
    rotary.rotate(x, angles_of(V, rotary, list(range(300))), want)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for given in (True, False):
        cs, out = torch.empty((300, 32, 2), device="cuda"), torch.empty_like(x)
        s.wait_stream(torch.cuda.current_stream())
        if given:
            rotary.angles(pos, cs, stream=s)
            rotary.rotate(x, cs, out, stream=s)
        else:
            with torch.cuda.stream(s):
                rotary.angles(pos, cs)
                rotary.rotate(x, cs, out)
        s.synchronize()
        assert torch.equal(out, want)


def test_offsets_past_32_bits(V):
    """Tokens that lie gigabytes apart, in the numbers, in the cache and between tokens of one page."""
    rotary = V.Rotary(V.rotary_frequencies(64)[0])
    n, h, d = 17, 2, 64
    cs = angles_of(V, rotary, list(range(n)))
    near = torch.randn((2, n, h, d), device="cuda").bfloat16()
    far = torch.empty(17 * (1 << 28) + 4096, dtype=torch.bfloat16, device="cuda")  # 9 GB
    x = far.as_strided((n, h, d), ((1 << 28) + 16, d, 1))
    x.copy_(near[0])
    out, want = torch.empty((n, h, d), device="cuda"), torch.empty((n, h, d), device="cuda")
    rotary.rotate(x, cs, out)
    rotary.rotate(near[0], cs, want)
    assert torch.equal(out, want)
    rotary.rotate(x, cs, x)
    assert torch.equal(x.float(), want.bfloat16().float())
    x.copy_(near[0])
    v = x.as_strided((n, h, d), ((1 << 28) + 16, d, 1), 2048)
    v.copy_(near[1])
    # a cache whose tokens lie 512 MB apart: a page spans 16 GB
    codes = torch.empty(32 * (1 << 29), dtype=torch.int8, device="cuda")
    page = lambda at: codes.as_strided((2, h, 32, d), (4096, 256, 1 << 29, 1), at)  # noqa: E731
    a = V.KVCache(page(0), page(1 << 20), *(torch.zeros((2, h), device="cuda") for _ in range(2)))
    b = new_cache(V, 2, h, 32, d, "int8")
    for c in (a, b):
        for t in (c.k, c.v, c.k_scale, c.v_scale):
            t.zero_()
    slots = torch.arange(n, device="cuda") + 32 + 13
    for keys, values in ((x, v), (near[0], near[1])):
        a.append_rotary(keys, values, slots, rotary, cs)
        assert a.k.stride(2) == 1 << 29
    turned = torch.empty((n, h, d), device="cuda")
    rotary.rotate(near[0], cs, turned)
    for _ in range(2):
        b.append(turned, near[1].float(), slots)
    assert torch.equal(a.k.view(torch.uint8), b.k) and torch.equal(a.v.view(torch.uint8), b.v)
    assert torch.equal(a.k_scale[1], b.k_scale[1]) and torch.equal(a.v_scale[1], b.v_scale[1])


def test_cache_pages_of_every_order(V):
    """Pages whose heads or tokens lie outermost, as views of one buffer."""
    rotary = V.Rotary(V.rotary_frequencies(48)[0], "pairs")
    n, h, d, P = 50, 3, 48, 16
    x = torch.randn((2, n, h, d), device="cuda")
    cs = angles_of(V, rotary, list(range(100, 100 + n)))
    slots = torch.arange(n, device="cuda") + 5
    want = new_cache(V, 4, h, P, d, "e4m3")
    k = torch.empty_like(x[0])
    rotary.rotate(x[0], cs, k)
    want.append(k, x[1], slots)
    for order in ((0, 1, 2), (0, 2, 1), (1, 0, 2), (1, 2, 0), (2, 0, 1), (2, 1, 0)):
        shape = (4, h, P)
        t = [torch.full([shape[i] for i in order] + [d], 0x55, dtype=torch.uint8, device="cuda").permute(*[order.index(i) for i in range(3)], 3) for _ in range(2)]
        c = V.KVCache(*t, *(torch.full((4, h), 77.0, device="cuda") for _ in range(2)), "e4m3")
        c.append_rotary(x[0], x[1], slots, rotary, cs)
        same(c, want)


@pytest.mark.parametrize("base", [10000.0, 5e5, 1e7])
def test_sines_of_small_angles(V, base):
    """Angles of less than an eighth of a turn, however small: sines within a few roundings of themselves.  The
    frequency is a whole number of 2^-64 turns (off by 2^-65 of w / 2 pi > 2^-26), the phase rounds to 24 bits (u),
    sincospif is within 2 units in the last place (4 u of the number at most), the scale rounds once more (u)."""
    w = V.rotary_frequencies(128, base)[0]
    positions = [1, -1, 3, -7, 1000, -131071, 2 ** 24 + 1]
    for scale in (1.0, 1.4):
        got = angles_of(V, V.Rotary(w, scale=scale), positions)[..., 1].double().cpu().numpy()
        angle = np.array(positions, np.float64)[:, None] * np.array(w)
        want = scale * np.sin(angle)
        small = np.abs(angle) < np.pi / 4
        assert small.sum() > 100 and np.all(np.abs(got - want)[small] <= 6.1 * U * np.abs(want)[small])


@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_rotate_between_the_rows_of_its_input(V, layout):
    """Out in the same buffer as x: beside it in every token, in every head, and behind it; neighbours stay."""
    n, h, d = 33, 6, 64
    rotary = V.Rotary(V.rotary_frequencies(d)[0], layout)
    cs = angles_of(V, rotary, list(range(n)))
    for place in (lambda t, i: t.view(n, 3, h, d)[:, i], lambda t, i: t.view(n, h, 3, d)[:, :, i], lambda t, i: t.view(3, n, h, d)[i],
                  lambda t, i: t.view(h, n, 3, d)[:, :, i].transpose(0, 1)):
        flat = torch.randn(3 * n * h * d, device="cuda")
        before = flat.clone()
        want = torch.empty((n, h, d), device="cuda")
        rotary.rotate(place(before, 2).contiguous(), cs, want)
        rotary.rotate(place(flat, 2), cs, place(flat, 1))
        assert torch.equal(place(flat, 1), want)
        place(flat, 1).copy_(place(before, 1))
        assert torch.equal(flat, before)
        with pytest.raises(V.Q.SeedQError):
            rotary.rotate(flat[:n * h * d].view(n, h, d), cs, flat[d:d + n * h * d].view(n, h, d))


@pytest.mark.parametrize("n,h", [(6, 2), (700, 8)])
def test_append_rotary_from_a_fused_projection(V, n, h):
    """Queries turned in their place in rows that hold queries, keys and values; or into other rows' gaps."""
    d, P = 128, 16
    rotary = V.Rotary(V.rotary_frequencies(d)[0])
    cs = angles_of(V, rotary, list(range(n)))
    flat = torch.randn((n, 6 * h * d), device="cuda").bfloat16()
    before = flat.clone()
    q, k, v, gap = (flat[:, i * d:j * d].view(n, -1, d) for i, j in ((0, 3 * h), (3 * h, 4 * h), (4 * h, 5 * h), (5 * h, 6 * h)))
    slots = torch.arange(n, device="cuda")
    a, b = (new_cache(V, n // P + 1, h, P, d, "int8") for _ in range(2))
    want = torch.empty_like(q)
    both_ways(V, b, a, k, v, slots, rotary, cs, q, want)
    for out in (gap, q):
        x = q[:, :out.shape[1]]
        c = new_cache(V, n // P + 1, h, P, d, "int8")
        c.append_rotary(k, v, slots, rotary, cs, q=x, q_out=out)
        same(c, a)
        assert torch.equal(out, want[:, :out.shape[1]])
    flat[:, 5 * h * d:], flat[:, :3 * h * d] = before[:, 5 * h * d:], before[:, :3 * h * d]
    assert torch.equal(flat, before)
    for out in (k, v):
        with pytest.raises(V.Q.SeedQError):
            a.append_rotary(k, v, slots, rotary, cs, q=q[:, :h], q_out=out)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("dim,rot", [(128, 64), (64, 40), (32, 2), (112, 90), (48, 24), (16, 14)])
@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_append_rotary_leaves_zeros_behind_the_rotation(V, kind, layout, dim, rot):
    """Numbers from rot_dim on go into the cache as they are, a zero's sign among them."""
    n, h, P = 21, 3, 16
    rotary = V.Rotary(V.rotary_frequencies(rot)[0], layout)
    cs = angles_of(V, rotary, list(range(7, 7 + n)))
    x = torch.randn((2, n, h, dim), generator=torch.Generator("cuda").manual_seed(dim), device="cuda")
    x[..., rot:] = torch.where(x[..., rot:] > 0.5, x[..., rot:], torch.where(x[..., rot:] > -0.5, -0.0, 0.0))
    a, b = (new_cache(V, 2, h, P, dim, kind) for _ in range(2))
    both_ways(V, a, b, x[0], x[1], torch.arange(n, device="cuda"), rotary, cs)
    code = torch.where(x[0, :P, :, rot:].signbit(), 0x80 if kind == "e4m3" else 0, 0)[x[0, :P, :, rot:] == 0]
    assert torch.equal(a.k[0].transpose(0, 1)[..., rot:][x[0, :P, :, rot:] == 0], code.byte())


# ---------------------------------------------------------------- large calls

@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("ti,to,n,heads,dim,rot", [("bf16", "bf16", 4099, 41, 128, 128), ("f16", "f32", 4099, 38, 128, 64), ("bf16", "f16", 3001, 37, 96, 24),
                                                   ("f16", "f16", 701, 39, 100, 50)])
def test_rotate_large(V, layout, ti, to, n, heads, dim, rot):
    """Heads four to a thread, numbers of them that four does not divide; out of place and in it."""
    rng = np.random.RandomState(n + heads)
    rotary = V.Rotary(V.rotary_frequencies(rot)[0], layout)
    cs = angles_of(V, rotary, rng.randint(0, 131072, n).tolist())
    x = torch.randn((n, heads, dim), generator=torch.Generator("cuda").manual_seed(n), device="cuda").to(DT[ti])
    out = torch.full((n, heads, dim), 9.0, dtype=DT[to], device="cuda")
    check_rotate(V, x, cs, rotary, layout, out)
    if ti == to:
        wide = torch.full((n, heads + 1, dim), 4.0, dtype=DT[ti], device="cuda")  # a head more, which stays
        wide[:, :heads] = x
        rotary.rotate(wide[:, :heads], cs, wide[:, :heads])
        assert torch.equal(wide[:, :heads], out) and bool((wide[:, heads] == 4.0).all())


@pytest.mark.parametrize("kind,dtype,layout,heads,q_heads,page,dim,rot,order,lens", [
    ("int8", "bf16", "half", 8, 32, 16, 128, 128, "head", (1024, 1024, 1024, 1024)),
    ("e4m3", "bf16", "half", 32, 32, 16, 128, 128, "head", (1024, 1024, 1024, 1024)),
    ("int8", "f32", "pairs", 8, 9, 64, 128, 128, "token", (1500, 1, 700, 33)),
    ("e4m3", "f16", "pairs", 32, 33, 256, 128, 64, "head", (1024, 300, 777)),
    ("int8", "f16", "half", 9, 0, 256, 64, 64, "token", (2000, 1, 1, 1, 511)),
    ("e4m3", "f32", "half", 11, 11, 240, 256, 64, "head", (900, 241)),
    ("int8", "bf16", "half", 17, 0, 48, 96, 24, "token", (333, 1000)),
    ("e4m3", "bf16", "pairs", 10, 40, 128, 112, 112, "head", (1025,)),
    ("int8", "f32", "half", 64, 64, 256, 16, 6, "head", (600, 600))])
def test_append_rotary_prompts(V, kind, dtype, layout, heads, q_heads, page, dim, rot, order, lens):
    """Prompts whose heads a CTA takes several of, three times, on from where the last ended within a page (the first pieces small
    numbers, the next ones larger, so that pages' scales grow): codes, scales and queries as of the rotation and the plain append."""
    rng = np.random.RandomState(heads + dim)
    most = [-(-3 * n // page) + 1 for n in lens]
    pages = [p.tolist() for p in np.split(rng.permutation(sum(most)), np.cumsum(most)[:-1])]
    a, b = (new_cache(V, sum(most), heads, page, dim, kind, order) for _ in range(2))
    rotary = V.Rotary(V.rotary_frequencies(rot)[0], layout)
    gen = torch.Generator("cuda").manual_seed(heads)
    at = [int(x) for x in rng.randint(0, page, len(lens))]  # in the middle of a page, which holds what it held
    for step, size in enumerate((0.01, 1.0, 30.0)):
        slots = []
        for i, n in enumerate(lens):
            n = n if step != 1 else max(n - 5, 1)
            slots += [pages[i][p // page] * page + p % page for p in range(at[i], at[i] + n)]
            at[i] += n
            if step == 2:
                slots.append(-1)  # an unused token between requests
        n = len(slots)
        assert 2 * n * heads > 8192
        odd = step if dtype != "f32" else 0  # rows that do not allow wide loads
        flat = torch.zeros(2 * n * heads * dim + odd, dtype=DT[dtype], device="cuda")
        x = flat[odd:].view(2, n, heads, dim)
        x.copy_(size * torch.randn((2, n, heads, dim), generator=gen, device="cuda"))
        x[:, ::7] *= 4
        cs = angles_of(V, rotary, rng.randint(0, 100000, n).tolist())
        q = torch.randn((n, q_heads, dim), generator=gen, device="cuda").to(DT[dtype]) if q_heads else None
        q_out = torch.full((n, q_heads, dim), 5.0, dtype=DT[dtype if step else "bf16"], device="cuda") if q_heads else None
        both_ways(V, a, b, x[0], x[1], torch.tensor(slots, device="cuda"), rotary, cs, q, q_out)
        if q_heads and step:  # the same in place
            turned = q.clone()
            a.append_rotary(x[0], x[1], torch.full((n,), -1, device="cuda"), rotary, cs, q=turned, q_out=turned)
            assert torch.equal(turned, q_out)
            same(a, b)


def test_append_rotary_prompts_captured_and_replayed(V):
    """A prompts' write with its queries' own launch in a graph, replayed with other positions, numbers and slots."""
    n, h, d, P = 1100, 8, 128, 16
    rotary = V.Rotary(V.rotary_frequencies(d)[0])
    a, b = (new_cache(V, 3 * (n // P + 1), h, P, d, "int8") for _ in range(2))
    pos, slots = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int64, device="cuda")
    x, q = torch.randn((2, n, h, d), device="cuda").bfloat16(), torch.randn((n, 5 * h, d), device="cuda").bfloat16()
    cs, q_out = torch.empty((n, d // 2, 2), device="cuda"), torch.empty_like(q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        rotary.angles(pos, cs)
        a.append_rotary(x[0], x[1], slots, rotary, cs, q=q, q_out=q_out)
    for i in range(3):
        pos.copy_(torch.randint(0, 50000, (n,)))
        slots.copy_(torch.arange(n) + i * (n + 3))
        x.normal_()
        q.normal_()
        graph.replay()
        want, turned = torch.empty_like(q), torch.empty((n, h, d), device="cuda")
        rotary.rotate(q, cs, want)
        rotary.rotate(x[0], cs, turned)
        b.append(turned, x[1].float(), slots)
        assert torch.equal(q_out, want)
        same(a, b)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("heads,dim,page,reps", [(2, 32, 32, 1), (40, 128, 64, 60)])
def test_append_rotary_runs_of_a_page_in_any_order(V, kind, heads, dim, page, reps):
    """Runs of one page's slots that go back, meet or repeat a slot: as calls of their own, one after the other."""
    rng = np.random.RandomState(heads)
    rotary = V.Rotary(V.rotary_frequencies(dim)[0])
    once = [[5, 6, 7], [5], [5], [3, 4], [0, 1], [30, 31], [2], [2, 3, 4, 5, 6, 7, 8], [9], list(range(page))[10:], [0]]
    a, b, c = (new_cache(V, reps, heads, page, dim, kind) for _ in range(3))
    slots = [p * page + s for p in range(reps) for run in once for s in run]
    x = torch.from_numpy((2.0 ** rng.randint(-6, 6, (2, len(slots), 1, 1)) * rng.randn(2, len(slots), heads, dim)).astype(np.float32)).cuda()
    cs = angles_of(V, rotary, rng.randint(0, 9999, len(slots)).tolist())
    both_ways(V, a, b, x[0], x[1], torch.tensor(slots, device="cuda"), rotary, cs)
    cuts = [0] + [i for i in range(1, len(slots)) if slots[i] != slots[i - 1] + 1] + [len(slots)]  # what follows on is one run
    for at, to in zip(cuts, cuts[1:]):
        if slots[at] < 5 * page:
            c.append_rotary(x[0, at:to], x[1, at:to], torch.tensor(slots[at:to], device="cuda"), rotary, cs[at:to])
    for y, z in ((a.k, c.k), (a.v, c.v), (a.k_scale, c.k_scale), (a.v_scale, c.v_scale)):
        assert torch.equal(y[:5], z[:5])


def test_append_rotary_of_the_most_heads(V):
    """1024 heads of 16 dims, a few tokens and some prompts' worth."""
    rotary = V.Rotary(V.rotary_frequencies(16)[0])
    for n in (3, 200):
        a, b = (new_cache(V, 20, 1024, 16, 16, "int8") for _ in range(2))
        x = torch.randn((2, n, 1024, 16), device="cuda").half()
        q = torch.randn((n, 3000, 16), device="cuda").half()
        cs = angles_of(V, rotary, list(range(n)))
        both_ways(V, a, b, x[0], x[1], torch.arange(n, device="cuda") + 7, rotary, cs, q, torch.empty_like(q))


def test_rotate_the_most_heads_and_the_widest(V):
    for n, heads, dim, rot in ((2, 65536, 2, 2), (1, 65536, 16, 10), (5, 3, 1024, 1024)):
        for layout in ("half", "pairs"):
            rotary = V.Rotary(V.rotary_frequencies(rot)[0], layout)
            x = torch.randn((n, heads, dim), device="cuda")
            check_rotate(V, x, angles_of(V, rotary, list(range(n))), rotary, layout, torch.empty_like(x))
