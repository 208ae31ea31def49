"""Overlaps of rows of bytes (csrc/overlap.h, host code) against sets of bytes, and the calls that refuse them."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = """
#include "overlap.h"
using namespace seedq;
static ByteRows rows(const long long *r) { return byte_rows((const void *)r[0], r[1], r[2], r[3], r[4], r[5]); }
extern "C" int meet(const long long *x, const long long *y) { return overlap(rows(x), rows(y)); }
extern "C" int itself(const long long *x) { return overlaps_itself(rows(x)); }
"""


@pytest.fixture(scope="module")
def L(tmp_path_factory):
    d = tmp_path_factory.mktemp("overlap")
    (d / "o.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2609_38477_gb300", "csrc"),
                    str(d / "o.cpp"), "-o", str(d / "o.so")], check=True)
    return C.CDLL(str(d / "o.so"))


def as_c(r):
    return (C.c_longlong * 6)(*r)


def bytes_of(r):
    at, size, n0, s0, n1, s1 = r
    return [set(range(at + i * s0 + j * s1, at + i * s0 + j * s1 + size)) for i in range(n0) for j in range(n1)]


def some_rows(rng):
    """Rows as callers have them (heads of tokens, of a fused row, heads before tokens) and of any strides."""
    size, n0, n1 = (int(rng.randint(1, k)) for k in (9, 7, 6))
    kind = rng.randint(4)
    if kind == 0:
        s1 = size + int(rng.choice([0, 0, 3]))
        s0 = n1 * s1 + int(rng.choice([0, 0, 5, 40]))
    elif kind == 1:
        s0 = size + int(rng.choice([0, 2]))
        s1 = n0 * s0 + int(rng.choice([0, 7]))
    else:
        s0, s1 = (int(x) for x in rng.randint(0, 60, 2))
    if kind == 3:
        s0, s1 = (int(s * rng.choice([-1, 1])) for s in (s0, s1))
    return [int(rng.randint(400, 800)), size, n0, s0, n1, s1]


def test_overlap_against_sets(L):
    rng = np.random.RandomState(0)
    met = 0
    for _ in range(30000):
        x, y = some_rows(rng), some_rows(rng)
        if rng.rand() < 0.5:  # of equal strides, as slices of one buffer are
            y[2:] = x[2:]
            y[0] = x[0] + int(rng.randint(-60, 61))
        want = bool(set.union(*bytes_of(x)) & set.union(*bytes_of(y)))
        assert bool(L.meet(as_c(x), as_c(y))) == bool(L.meet(as_c(y), as_c(x))) == want, (x, y)
        met += want
    assert 5000 < met < 25000


def test_overlap_of_a_set_with_itself(L):
    rng = np.random.RandomState(1)
    met = 0
    for _ in range(20000):
        x = some_rows(rng)
        parts = bytes_of(x)
        want = len(set.union(*parts)) < sum(map(len, parts))
        assert bool(L.itself(as_c(x))) == want, x
        met += want
    assert 2000 < met < 18000


def test_overlap_of_many_rows(L):
    """Slices of a fused projection of thousands of tokens, far addresses and strides: by arithmetic, not by search."""
    t, h, d = 1 << 20, 72, 256
    row = 3 * h * d
    q, k, v = ([1 << 40 | i * h * d, d, t, row, h, d] for i in range(3))
    assert not any(L.meet(as_c(x), as_c(y)) for x, y in ((q, k), (k, v), (v, q)))
    assert L.meet(as_c(q), as_c([q[0] + d, *q[1:]])) and L.meet(as_c(k), as_c([k[0] - 1, *k[1:]])) and L.meet(as_c(q), as_c(q))
    apart = [q[0] + d * h, 1, 1, 0, 1, 0]
    assert not L.meet(as_c(q), as_c(apart)) and L.meet(as_c(k), as_c(apart))
    per_head = [[1 << 40 | i * d, d, t, h * 3 * d, h, 3 * d] for i in range(3)]  # q, k, v side by side in each head
    assert not any(L.meet(as_c(x), as_c(y)) for x, y in zip(per_head, per_head[1:]))
    assert not L.itself(as_c(q)) and not L.itself(as_c(per_head[0])) and L.itself(as_c([1 << 40, d, t, 0, h, d]))
    for heads, met in ((2, False), (3, True)):  # tokens 2^61 apart, heads 2^60 downwards: token 1's head 2 is token 0's head 0
        assert bool(L.itself(as_c([1 << 40, 16, 5, 1 << 61, heads, -(1 << 60)]))) == met


# ---------------------------------------------------------------- calls (refused before a GPU is touched: the addresses are none)

FAKE = 1 << 20


@pytest.fixture(scope="module")
def Q():
    pytest.importorskip("torch")
    from paper_2609_38477_gb300 import build

    build.build()
    from paper_2609_38477_gb300 import seedq

    seedq.lib()
    return seedq


@pytest.mark.parametrize("kw", [
    dict(out=FAKE + 4), dict(out=FAKE - 64), dict(out=FAKE + 256), dict(out=FAKE + 4 * 3 * 256 - 4), dict(out=FAKE - 4 * 3 * 256 + 4),  # moved views of x
    dict(out=FAKE + 8, odt=1), dict(x=FAKE + 64 * 4, xt=512, out=FAKE, ot=512, oh=32),  # another type or strides, part of x
    dict(cs=2 * FAKE + 64), dict(cs=2 * FAKE - 3 * 16 * 8 + 8),  # over cos and sin
    dict(oh=32), dict(ot=128), dict(ot=0), dict(ot=64, oh=64)])  # rows of out on one another
def test_rotate_refuses_overlaps(Q, kw):
    a = dict(x=FAKE, dt=0, xt=256, xh=64, n=3, heads=4, dim=64, rot=32, layout=0, cs=8 * FAKE, out=2 * FAKE, odt=0, ot=256, oh=64)
    a.update(kw)
    assert Q.lib().seedq_rotate(*a.values(), None) == 1


@pytest.mark.parametrize("kw", [
    dict(out=FAKE + 64 * 4), dict(out=FAKE + 2, odt=1),  # over q, moved
    dict(out=3 * FAKE), dict(out=3 * FAKE + 4 * 128 - 4), dict(out=4 * FAKE - 512, odt=1), dict(out=4 * FAKE + 4 * 128 * 4 - 4),  # keys, values
    dict(out=5 * FAKE - 4 * 256 * 4 + 8), dict(out=6 * FAKE + 4), dict(oh=32), dict(ot=128)])  # slots, cos and sin, itself
def test_append_rotary_refuses_overlaps(Q, kw):
    c = Q.KvCacheDesc(0, 2, 64, 16, 4, 10 * FAKE, 11 * FAKE, 12 * FAKE, 13 * FAKE, 2 * 16 * 64, 16 * 64, 64)
    a = dict(cs=6 * FAKE, rot=32, layout=0, heads=4, odt=0, q=FAKE, qt=256, qh=64, out=2 * FAKE, ot=256, oh=64)
    a.update(kw)
    args = Q.AppendRotaryArgs(*a.values())
    assert Q.lib().seedq_kv_append_rotary(C.byref(c), 3 * FAKE, 4 * FAKE, 0, 128, 64, 5 * FAKE, 4, C.byref(args), None) == 1


@pytest.mark.parametrize("kw", [dict(cs=2 * FAKE + 8), dict(cs=2 * FAKE - 3 * 4 * 8 + 8), dict(cs=FAKE + 24), dict(cs=FAKE - 3 * 4 * 8 + 8)])
def test_angles_refuse_overlaps(Q, kw):
    a = dict(turns=FAKE, half=4, scale=1.0, pos=2 * FAKE, n=3, cs=3 * FAKE)
    a.update(kw)
    assert Q.lib().seedq_rotary_angles(*a.values(), None) == 1


@pytest.mark.parametrize("kw", [
    dict(beam=3 * FAKE), dict(token=4 * FAKE + 124), dict(score=5 * FAKE - 124), dict(beam=5 * FAKE + 4),  # one output over another
    dict(score=7 * FAKE), dict(token=7 * FAKE - 124), dict(beam=7 * FAKE + 31 * 416 + 396), dict(score=7 * FAKE + 2 * 416 - 4)])  # over logits
def test_select_refuses_overlaps(Q, kw):
    a = dict(logits=7 * FAKE, stride=104, dtype=0, beams=4, groups=8, vocab=100, scale=1.0, end=3, scores=FAKE, done=FAKE, weights=None, n_out=4,
             score=3 * FAKE, beam=4 * FAKE, token=5 * FAKE, work=FAKE, bytes=1 << 40)
    a.update(kw)
    assert Q.lib().seedq_beam_select(C.byref(Q.BeamSelectArgs(*a.values())), None) == 1


@pytest.mark.parametrize("kw", [
    dict(lens_out=3 * FAKE - 28), dict(lens_out=2 * FAKE + 4), dict(lens_out=4 * FAKE), dict(lens_out=7 * FAKE),  # over inputs, moved
    dict(status=2 * FAKE + 28), dict(status=3 * FAKE + 4), dict(status=8 * FAKE - 28), dict(left=2 * FAKE + 12), dict(left=3 * FAKE + 8),
    dict(left=9 * FAKE + 4), dict(left=8 * FAKE + 28), dict(left=6 * FAKE + 12),  # over other outputs
    dict(out=4 * FAKE + 4), dict(out=4 * FAKE - 32 * 7), dict(out=4 * FAKE + 4, ostride=9), dict(out=6 * FAKE - 64), dict(out=9 * FAKE), dict(out=2 * FAKE - 8),
    dict(free=4 * FAKE + 32 * 7), dict(free=2 * FAKE), dict(free=3 * FAKE + 28), dict(free=8 * FAKE)])
def test_reorder_refuses_overlaps(Q, kw):
    a = dict(groups=2, beams=4, parents=2 * FAKE, lens=3 * FAKE, table=4 * FAKE, stride=8, out=4 * FAKE, ostride=8, width=8, cap=4,
             free=6 * FAKE, count=7 * FAKE, lens_out=8 * FAKE, status=9 * FAKE, left=10 * FAKE, work=11 * FAKE, bytes=1 << 20)
    a.update(kw)
    caches = (Q.KvCacheDesc * 1)(Q.KvCacheDesc(0, 2, 64, 16, 4, 20 * FAKE, 21 * FAKE, 22 * FAKE, 23 * FAKE, 2 * 16 * 64, 16 * 64, 64))
    assert Q.lib().seedq_beam_reorder(caches, 1, C.byref(Q.BeamReorderArgs(*a.values())), None) == 1
