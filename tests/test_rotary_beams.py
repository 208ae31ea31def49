"""CPU checks of rotary positions, the rotating cache write and beam search: the
oracle against independent forms, the frequencies, and every refusal of the C ABI
and of the binding, before a GPU is touched."""
import ctypes as C
import math
import os
import sys

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "oracle"))

import serving as S  # noqa: E402

torch = pytest.importorskip("torch")
FAKE = 1 << 20  # 16-byte aligned, never dereferenced: validation comes first


@pytest.fixture(scope="module")
def Q():
    from paper_2609_38477_gb300 import build

    build.build()
    from paper_2609_38477_gb300 import seedq

    seedq.lib()
    return seedq


@pytest.fixture(scope="module")
def V(Q):
    from paper_2609_38477_gb300 import serving

    return serving


# ---------------------------------------------------------------- oracle

def test_rotation_by_hand():
    """A quarter turn of pair 0 and none of pair 1, in both layouts; the rest of the head stays."""
    cs = np.array([[[0.0, 1.0], [1.0, 0.0]]])
    x = np.arange(1.0, 7.0).reshape(1, 1, 6)
    assert S.rotate(x, cs, "half")[0][0, 0].tolist() == [-3, 2, 1, 4, 5, 6]
    assert S.rotate(x, cs, "pairs")[0][0, 0].tolist() == [-2, 1, 3, 4, 5, 6]


def test_rotation_scores_by_distance():
    """Products of rotated queries and keys go by the distance of their positions."""
    rng = np.random.RandomState(0)
    w = [10000.0 ** (-i / 8) for i in range(8)]
    q, k = rng.randn(1, 1, 16), rng.randn(1, 1, 16)
    for layout in ("half", "pairs"):
        at = lambda x, p: S.rotate(x, S.rotary_angles([p], w, 1.0), layout)[0][0, 0]  # noqa: E731
        d = [at(q, p) @ at(k, p - 7) for p in (7, 100, 131072, -3)]
        assert np.allclose(d, d[0], rtol=0, atol=1e-10)


def test_beam_select_oracle_by_hand():
    """Two beams of two tokens, even odds and 3 to 1; a finished one; a weight that turns the order."""
    x = np.log(np.array([[[1.0, 1.0], [3.0, 1.0], [9.0, 9.0]]]))
    scores = np.log(np.array([[0.5, 0.4, 0.09]]))
    s, b, t, _ = S.beam_select(x, scores, 1.0, 5, np.array([[False, False, True]]), 1)
    assert np.allclose(np.exp(s), [[0.3, 0.25, 0.25, 0.1, 0.09]])
    assert b.tolist() == [[1, 0, 0, 1, 2]] and t.tolist() == [[0, 0, 1, 1, 1]]
    s, b, t, _ = S.beam_select(x, scores, 1.0, 3, None, -1, np.array([[1.0, 1.0, 0.01]]))
    assert b.tolist() == [[2, 2, 1]] and t.tolist() == [[0, 1, 0]] and np.allclose(np.exp(s), [[0.045, 0.045, 0.3]])
    s, b, t, _ = S.beam_select(np.full((1, 1, 2), -np.inf), np.zeros((1, 1)), 1.0, 2)
    assert b.tolist() == [[-1, -1]] and np.isneginf(s).all()


def test_beam_reorder_oracle_by_hand():
    """Pages of 4: beam 0 (10 tokens) has two children, beam 1 one, beam 2 none; page 1 is shared."""
    table = np.array([[1, 2, 3], [1, 4, -1], [1, 5, 6]])
    free = np.array([7, 8, -1, -1, -1])
    out, lens, status, f, left, copies = S.beam_reorder(np.array([[0, 0, 1]]), [10, 8, 9], table, np.full((3, 3), -9), free, 2, 4)
    assert f.tolist() == [7, 8, 5, 6, -1] and left == 3 and copies == [(3, 6, 2)]
    assert out.tolist() == [[1, 2, 3], [1, 2, 6], [1, 4, -9]] and lens.tolist() == [10, 10, 8] and not status.any()


# ---------------------------------------------------------------- frequencies

def test_frequencies(V):
    w, scale = V.rotary_frequencies(8, 10000.0)
    assert np.allclose(w, [1, 0.1, 0.01, 0.001]) and scale == 1
    assert np.allclose(V.rotary_frequencies(8, rule="linear", factor=4)[0], np.array(w) / 4)
    b = V.rotary_frequencies(8, rule="base", factor=4)[0]
    assert b[0] == 1 and math.isclose(b[-1], w[-1] / 4)
    assert V.rotary_frequencies(2, rule="base", factor=4)[0] == [1.0]
    # bands: turns over 8192 positions are 1304, 130, 13 and 1.3; kept from 4 turns on, a quarter of the way at 1.3
    m, scale = V.rotary_frequencies(8, rule="bands", factor=8)
    keep = (8192 * w[3] / (2 * math.pi) - 1) / 3
    assert m[:3] == w[:3] and math.isclose(m[3], w[3] * keep + w[3] / 8 * (1 - keep)) and scale == 1
    m, scale = V.rotary_frequencies(128, rule="ramp", factor=16, original=4096, low=1, high=32)
    w = V.rotary_frequencies(128)[0]
    ratio = np.array(m) / np.array(w)
    lo = math.floor(128 * math.log(4096 / (32 * 2 * math.pi)) / (2 * math.log(10000)))
    hi = math.ceil(128 * math.log(4096 / (2 * math.pi)) / (2 * math.log(10000)))
    assert np.all(ratio[:lo + 1] == 1) and np.allclose(ratio[hi:], 1 / 16) and np.all(np.diff(ratio[lo:hi + 1]) < 0)
    assert math.isclose(scale, 1 + 0.1 * math.log(16))
    for rule in ("none", "linear", "base", "bands", "ramp"):
        assert np.allclose(V.rotary_frequencies(64, rule=rule)[0], V.rotary_frequencies(64)[0])  # a factor of one
    for bad in (dict(rot_dim=7), dict(rot_dim=0), dict(base=1.0), dict(factor=0.5), dict(rule="other"), dict(low=4.0), dict(original=0)):
        with pytest.raises(ValueError):
            V.rotary_frequencies(**{**dict(rot_dim=8), **bad})


def test_rotary_turns(V):
    r = V.Rotary([2 * math.pi, math.pi, 1.0, -1.0, 0.0], device="cpu", layout="pairs", scale=2.0)
    assert (r.half, r.rot_dim, r.layout, r.scale) == (5, 10, 1, 2.0)
    t = [x % 2 ** 64 for x in r.turns.tolist()]
    near = lambda x, y: min((x - y) % 2 ** 64, (y - x) % 2 ** 64)  # noqa: E731
    assert near(t[0], 0) < 2 ** 12 and near(t[1], 2 ** 63) < 2 ** 11 and t[4] == 0 and (t[2] + t[3]) % 2 ** 64 == 0
    assert near(t[2], round(2 ** 64 / (2 * math.pi))) < 2 ** 12
    for bad in ([], [float("nan")], [1.0, float("inf")]):
        with pytest.raises(ValueError, match="frequencies"):
            V.Rotary(bad, device="cpu")
    with pytest.raises(ValueError, match="layout"):
        V.Rotary([1.0], "other", device="cpu")


# ---------------------------------------------------------------- refusals of the library

@pytest.mark.parametrize("kw,status", [
    (dict(turns=None), 1), (dict(half=0), 1), (dict(half=513), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1),
    (dict(pos=None), 1), (dict(n=-1), 1), (dict(n=1 << 31), 1), (dict(cs=None), 1), (dict(cs=FAKE + 4), 1),
    (dict(half=512, n=(1 << 31) - 1), 6)])
def test_angles_refuse(Q, kw, status):
    a = dict(turns=FAKE, half=4, scale=1.0, pos=FAKE, n=3, cs=FAKE)
    a.update(kw)
    assert Q.lib().seedq_rotary_angles(*a.values(), None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), 1), (dict(dt=3), 1), (dict(n=-1), 1), (dict(n=1 << 31), 1), (dict(heads=-1), 1), (dict(heads=65537), 1),
    (dict(rot=0), 1), (dict(rot=7), 1), (dict(rot=66), 1), (dict(dim=1026, rot=64), 1), (dict(layout=2), 1), (dict(layout=-1), 1),
    (dict(cs=None), 1), (dict(cs=FAKE + 4), 1), (dict(out=None), 1), (dict(odt=-1), 1), (dict(out=FAKE, odt=1), 1),
    (dict(out=FAKE, ot=512), 1), (dict(out=FAKE, oh=128), 1), (dict(n=(1 << 31) - 1, heads=65536, dim=1024, rot=2), 6)])
def test_rotate_refuses(Q, kw, status):
    a = dict(x=FAKE, dt=0, xt=256, xh=64, n=3, heads=4, dim=64, rot=32, layout=0, cs=FAKE, out=2 * FAKE, odt=0, ot=256, oh=64)
    a.update(kw)
    assert Q.lib().seedq_rotate(*a.values(), None) == status


def _desc(Q, **kw):
    d = dict(kind=0, n_kv_heads=2, head_dim=64, page_size=16, n_pages=4, k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE,
             page_stride=2 * 16 * 64, head_stride=16 * 64, token_stride=64)
    d.update(kw)
    return Q.KvCacheDesc(*d.values())


def _rotary_args(Q, **kw):
    a = dict(cs=FAKE, rot=32, layout=0, heads=4, odt=1, q=FAKE, qt=256, qh=64, out=2 * FAKE, ot=256, oh=64)
    a.update(kw)
    return Q.AppendRotaryArgs(*a.values())


@pytest.mark.parametrize("kw", [
    dict(cs=None), dict(cs=FAKE + 4), dict(rot=0), dict(rot=33), dict(rot=66), dict(layout=2), dict(heads=-1), dict(heads=65537),
    dict(odt=3), dict(q=None), dict(out=None), dict(out=FAKE, odt=1), dict(out=FAKE, odt=0, ot=512)])
def test_append_rotary_refuses(Q, kw):
    L, d = Q.lib(), C.byref(_desc(Q))
    assert L.seedq_kv_append_rotary(d, FAKE, FAKE, 0, 128, 64, FAKE, 4, C.byref(_rotary_args(Q, **kw)), None) == 1
    assert L.seedq_kv_append_rotary(d, FAKE, FAKE, 0, 128, 64, FAKE, 4, None, None) == 1


@pytest.mark.parametrize("a,status", [
    ((None, FAKE, 0, 128, 64, FAKE, 4), 1), ((FAKE, None, 0, 128, 64, FAKE, 4), 1), ((FAKE, FAKE, 3, 128, 64, FAKE, 4), 1),
    ((FAKE, FAKE, 0, 128, 64, FAKE, -1), 1), ((FAKE, FAKE, 0, 128, 64, None, 4), 1), ((FAKE, FAKE, 0, 128, 64, FAKE, 1 << 31), 1),
    ((FAKE, FAKE, 0, 0, 0, FAKE, (1 << 31) - 1), 6)])
def test_append_rotary_refuses_what_append_does(Q, a, status):
    big = dict(n_kv_heads=1024, head_dim=256, token_stride=256, head_stride=16 * 256, page_stride=1024 * 16 * 256) if status == 6 else {}
    r = _rotary_args(Q, heads=0, q=None, out=None)
    assert Q.lib().seedq_kv_append_rotary(C.byref(_desc(Q, **big)), *a, C.byref(r), None) == status
    for bad, code in ((dict(kind=2), 1), (dict(head_dim=24), 6), (dict(page_size=8), 6), (dict(k=None), 1), (dict(k=FAKE + 8), 6)):
        assert Q.lib().seedq_kv_append_rotary(C.byref(_desc(Q, **bad)), FAKE, FAKE, 0, 128, 64, FAKE, 4, C.byref(r), None) == code
    assert Q.lib().seedq_kv_append_rotary(None, FAKE, FAKE, 0, 128, 64, FAKE, 4, C.byref(r), None) == 1


def _select(Q, **kw):
    a = dict(logits=FAKE, stride=100, dtype=0, beams=4, groups=8, vocab=100, scale=1.0, end=3, scores=FAKE, done=FAKE, weights=None, n_out=4,
             score=3 * FAKE, beam=4 * FAKE, token=5 * FAKE, work=FAKE, bytes=1 << 40)
    a.update(kw)
    return Q.BeamSelectArgs(*a.values())


@pytest.mark.parametrize("kw", [
    dict(logits=None), dict(logits=FAKE + 2), dict(stride=99), dict(dtype=3), dict(beams=0), dict(beams=33), dict(groups=-1),
    dict(groups=2049), dict(groups=1 << 40), dict(vocab=0), dict(vocab=(1 << 27) + 1, stride=1 << 28), dict(scale=0.0), dict(scale=-1.0),
    dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=2.0 ** -65), dict(scale=2.0 ** 65), dict(end=-1), dict(end=100),
    dict(scores=3 * FAKE + 4 * 31), dict(weights=3 * FAKE - 4 * 7), dict(done=4 * FAKE + 127), dict(scores=5 * FAKE),
    dict(scores=None), dict(n_out=0), dict(n_out=33), dict(score=None), dict(beam=None), dict(token=None), dict(work=None),
    dict(work=FAKE + 8), dict(bytes=1000)])
def test_select_refuses(Q, kw):
    assert Q.lib().seedq_beam_select(C.byref(_select(Q, **kw)), None) == 1
    assert Q.lib().seedq_beam_select(None, None) == 1


def test_select_workspace(Q):
    size = Q.lib().seedq_beam_select_workspace_bytes
    assert size(2, 4, 100) > 0 and size(2, 4, 100) <= size(2, 4, 30000) <= size(3, 4, 30000) <= size(3, 5, 30000)
    for bad in ((-1, 4, 100), (2, 0, 100), (2, 33, 100), (2, 4, 0), (2, 4, (1 << 27) + 1), (8193, 1, 10), (300, 32, 10)):
        assert size(*bad) == 0
    short = size(2, 4, 100) - 1
    assert Q.lib().seedq_beam_select(C.byref(_select(Q, bytes=short)), None) == 1


def _reorder(Q, **kw):
    a = dict(groups=2, beams=4, parents=FAKE, lens=FAKE + 64, table=FAKE + 128, stride=8, out=FAKE + 128, ostride=8, width=8, cap=4,
             free=FAKE + 512, count=FAKE + 768, lens_out=FAKE + 1024, status=FAKE + 1088, left=FAKE + 1152, work=FAKE, bytes=1 << 40)
    a.update(kw)
    return Q.BeamReorderArgs(*a.values())


@pytest.mark.parametrize("kw", [
    dict(groups=0), dict(beams=0), dict(beams=33), dict(groups=2049), dict(parents=None), dict(lens=None), dict(table=None), dict(out=None),
    dict(width=0), dict(width=9), dict(width=(1 << 20) + 1, stride=1 << 21, ostride=1 << 21), dict(out=FAKE + 256, ostride=7),
    dict(ostride=9), dict(cap=3), dict(cap=(1 << 31) - 1), dict(free=None), dict(count=None), dict(lens_out=None), dict(status=None),
    dict(left=None), dict(lens_out=FAKE), dict(lens_out=FAKE + 768), dict(status=FAKE), dict(status=FAKE + 64), dict(status=FAKE + 768),
    dict(left=FAKE + 64), dict(left=FAKE), dict(work=None), dict(work=FAKE + 8), dict(bytes=100)])
def test_reorder_refuses(Q, kw):
    caches = (Q.KvCacheDesc * 2)(_desc(Q), _desc(Q, kind=1))
    assert Q.lib().seedq_beam_reorder(caches, 2, C.byref(_reorder(Q, **kw)), None) == 1


@pytest.mark.parametrize("kw,status", [
    (dict(n_kv_heads=3), 1), (dict(head_dim=48), 1), (dict(page_size=32), 1), (dict(n_pages=5), 1), (dict(page_stride=4096), 1),
    (dict(head_stride=2048), 1), (dict(token_stride=128), 1), (dict(kind=5), 1), (dict(v=None), 1), (dict(head_dim=24), 6)])
def test_reorder_refuses_caches(Q, kw, status):
    caches = (Q.KvCacheDesc * 2)(_desc(Q), _desc(Q, **kw))
    L, a = Q.lib(), C.byref(_reorder(Q))
    assert L.seedq_beam_reorder(caches, 2, a, None) == status
    assert L.seedq_beam_reorder(None, 2, a, None) == 1 and L.seedq_beam_reorder(caches, 0, a, None) == 1
    assert L.seedq_beam_reorder(caches, 4097, a, None) == 1 and L.seedq_beam_reorder(caches, 1, None, None) == 1


def test_nothing_to_do_is_ok(Q):
    L = Q.lib()
    assert L.seedq_rotary_angles(None, 4, 1.0, None, 0, None, None) == 0
    assert L.seedq_rotate(None, 0, 0, 0, 0, 4, 64, 32, 0, None, None, 0, 0, 0, None) == 0
    assert L.seedq_rotate(None, 0, 0, 0, 5, 0, 64, 32, 0, None, None, 0, 0, 0, None) == 0
    assert L.seedq_kv_append_rotary(C.byref(_desc(Q)), None, None, 0, 0, 0, None, 0, C.byref(_rotary_args(Q, cs=None, q=None, out=None)), None) == 0
    assert L.seedq_beam_select(C.byref(_select(Q, groups=0, logits=None, scores=None, work=None)), None) == 0


# ---------------------------------------------------------------- refusals of the binding

def _meta(*shape, dt=torch.float32):
    return torch.zeros(shape, dtype=dt, device="meta")


class NoLibrary:
    def __getattr__(self, name):
        return lambda *a: pytest.fail(f"{name} is called")


def _cache(V, device):
    c = V.KVCache.__new__(V.KVCache)
    c.n_pages, c.n_kv_heads, c.page_size, c.head_dim, c.device, c._ref = 4, 2, 16, 64, torch.device(device), None
    return c


def test_binding_refuses_rotary(Q, V, monkeypatch):
    monkeypatch.setattr(Q, "lib", NoLibrary)
    r = V.Rotary([1.0] * 16, device="cpu")
    z = torch.zeros
    i32, cs = z(3, dtype=torch.int32), z(3, 16, 2)
    for pos, out in ((i32.long(), cs), (i32[:2], cs), (i32, z(3, 15, 2)), (i32, cs.double()), (i32, z(3, 2, 16).transpose(1, 2)), (i32, _meta(3, 16, 2))):
        with pytest.raises(ValueError):
            r.angles(pos, out, stream=0)
    x = z(3, 4, 64)
    for a, c, o in ((x[0], cs, x), (x, cs[:2], x), (x, cs, z(3, 4, 63)), (x, cs, x.double()), (z(3, 64, 4).transpose(1, 2), cs, x),
                    (x, cs, z(3, 1, 64).expand(3, 4, 64)), (x, cs, z(999).as_strided((3, 4, 64), (64, 64, 1))),
                    (x, cs, z(999).as_strided((3, 4, 64), (128, 64, 1))), (x, cs, z(999).as_strided((3, 4, 64), (64, 128, 1))), (x, cs, _meta(3, 4, 64)), (x, cs, z(64 * 12).as_strided((3, 4, 64), (32, 192, 1)))):
        with pytest.raises(ValueError):
            r.rotate(a, c, o, stream=0)
    cache = _cache(V, "cpu")
    k, slots = z(3, 2, 64), z(3, dtype=torch.int64)
    for kw in (dict(q=x), dict(q_out=x), dict(q=x.half(), q_out=x), dict(q=z(2, 4, 64), q_out=x), dict(q=x, q_out=z(3, 5, 64)),
               dict(q=x, q_out=z(3, 1, 64).expand(3, 4, 64)), dict(cos_sin=cs[:2]), dict(slots=slots[:2]), dict(v=z(3, 2, 63)), dict(k=z(3, 3, 64)),
               dict(q=x[0], q_out=x[0])):
        a = dict(k=k, v=k, slots=slots, rotary=r, cos_sin=cs, stream=0)
        a.update(kw)
        with pytest.raises(ValueError):
            cache.append_rotary(**a)


def test_binding_refuses_beams(Q, V, monkeypatch):
    z = torch.zeros
    with pytest.raises(ValueError, match="logits"):
        V.beam_select(z(4, 9), z(2, 2), z(2, 3), z(2, 3), z(2, 3), z(8, dtype=torch.uint8))
    for bad in ((2, 0, 10), (2, 33, 10), (9000, 1, 10), (2, 4, 0)):
        with pytest.raises(ValueError, match="beam_workspace"):
            V.beam_workspace(*bad, device="cpu")
    with pytest.raises(ValueError, match="caches"):
        V.BeamPages([], 1, 2)
    with pytest.raises(ValueError, match="caches"):
        V.BeamPages([z(3)], 1, 2)
    cache = _cache(V, "cpu")
    cache.desc = _desc(Q)
    for g, b in ((0, 4), (1, 0), (1, 33), (8193, 1)):
        with pytest.raises(ValueError, match="n_groups"):
            V.BeamPages([cache], g, b)
    pages = V.BeamPages([cache], 2, 3)
    assert [t.shape[0] for t in (pages.seq_lens, pages.status, pages.free_count)] == [6, 6, 1]
    monkeypatch.setattr(Q, "lib", NoLibrary)
    i = z(6, dtype=torch.int32)
    table, free = z((6, 5), dtype=torch.int32), z(9, dtype=torch.int32)
    for kw in (dict(parents=i), dict(parents=z(2, 3)), dict(parents=z((3, 2), dtype=torch.int32).t()), dict(seq_lens=i[:5]), dict(block_table=table[:5]),
               dict(block_table=z((5, 6), dtype=torch.int32).t()), dict(free_pages=free[::2]), dict(free_count=i[:0]), dict(out=z((6, 4), dtype=torch.int32)),
               dict(out=z((6, 5))), dict(out=z((1, 5), dtype=torch.int32).expand(6, 5)), dict(out=_meta(6, 5, dt=torch.int32))):
        a = dict(parents=i.view(2, 3), seq_lens=i, block_table=table, free_pages=free, free_count=i[:1], stream=0)
        a.update(kw)
        with pytest.raises(ValueError):
            pages.reorder(**a)


@pytest.mark.parametrize("stream", [None, 0])
def test_binding_refuses_another_device_than_the_current_one(Q, V, monkeypatch, stream):
    cache = _cache(V, "cpu")
    cache.desc = _desc(Q)
    pages = V.BeamPages([cache], 2, 3)
    monkeypatch.setattr(Q, "lib", NoLibrary)
    r = V.Rotary([1.0] * 16, device="cpu")
    z = torch.zeros
    i = z(6, dtype=torch.int32)
    x, cs = z(3, 2, 64), z(3, 16, 2)
    calls = [lambda: r.angles(i, cs, stream=stream), lambda: r.rotate(x, cs, x, stream=stream),
             lambda: cache.append_rotary(x, x, z(3, dtype=torch.int64), r, cs, stream=stream),
             lambda: pages.reorder(i.view(2, 3), i, z((6, 5), dtype=torch.int32), i, i[:1], stream=stream)]
    for current in (0, 1):  # the CPU's tensors are on no device of these
        monkeypatch.setattr(V, "_current_device", lambda: current)
        for call in calls:
            with pytest.raises(ValueError, match="current device"):
                call()


def test_strides_of_single_entries_do_not_matter(Q, V, monkeypatch):
    """One token's or one head's rows, whatever their strides there; a single row of logits or of a table."""
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: calls.append((name, a)) or 0

    r = V.Rotary([1.0] * 16, device="cpu")
    cache = _cache(V, "cpu")
    cache.desc = _desc(Q)
    pages = V.BeamPages([cache], 1, 1)
    monkeypatch.setattr(Q, "lib", Library)
    monkeypatch.setattr(V, "_current_device", lambda: None)
    for n, h in ((1, 4), (5, 1), (1, 1)):
        x = torch.zeros(4096).as_strided((n, h, 64), [7 if m == 1 else s for m, s in zip((n, h), (64 * h, 64))] + [1])
        r.rotate(x, torch.zeros(n, 16, 2), x, stream=0)
        assert calls[-1][0] == "seedq_rotate" and calls[-1][1][4:6] == (n, h)
    i = torch.zeros(1, dtype=torch.int32)
    pages.reorder(i.view(1, 1), i, torch.zeros(9, dtype=torch.int32).as_strided((1, 5), (2, 1)), torch.zeros(9, dtype=torch.int32), i, stream=0)
    assert calls[-1][0] == "seedq_beam_reorder" and Q.BEAM_REORDER_ARGS.unpack(calls[-1][1][2])[5] == 5


def test_search_refuses_powers_past_float32(monkeypatch):
    """Lengths to a power that float32 cannot hold would make a weight of 0 or infinity: refused before any work."""
    from types import SimpleNamespace

    from paper_2609_38477_gb300 import generate

    d = generate.Decoder.__new__(generate.Decoder)
    d.spec, d.plan, d.seq_lens = SimpleNamespace(vocab=50), SimpleNamespace(max_requests=4), torch.ones(4)
    for power, steps in ((64.0, 4), (-64.0, 4), (20.0, 100), (float("nan"), 4), (float("inf"), 4), (-float("inf"), 2)):
        with pytest.raises(ValueError, match="length_power"):
            d.beam_search([[1]], 2, steps, length_power=power)
    for power, steps in ((63.0, 4), (-63.0, 4), (1.0, 10 ** 6), (1e30, 1)):
        with pytest.raises(ValueError, match="under way"):
            d.beam_search([[1]], 2, steps, length_power=power)


def test_rotate_of_the_decode_loop():
    """generate.rotate turns numbers i and i + dim / 2 of every head by the angles, in plain torch."""
    from paper_2609_38477_gb300 import generate

    rng = np.random.RandomState(4)
    x, angles = torch.from_numpy(rng.randn(3, 2, 10)), torch.from_numpy(rng.randn(3, 5))
    want, _ = S.rotate(x.numpy(), np.stack([np.cos(angles.numpy()), np.sin(angles.numpy())], 2), "half")
    got = generate.rotate(x, angles)
    assert got.shape == x.shape and np.abs(got.numpy() - want).max() < 1e-14
