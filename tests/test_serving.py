"""CPU checks of the serving calls: the oracle against independent forms, and
every refusal of the C ABI and of the binding, before a GPU is touched."""
import ctypes as C
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


# ---------------------------------------------------------------- oracle

def test_e4m3_codes_agree_with_torch():
    """Every code's value, and the rounding of a dense set of numbers with its ties."""
    t = torch.arange(256, dtype=torch.int16).to(torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    mine = S.e4m3_table()
    ok = ~np.isnan(t)
    assert ok.sum() == 254 and np.array_equal(mine[ok], t[ok])
    grid = np.unique(mine[:127])
    x = np.concatenate([grid, (grid[1:] + grid[:-1]) / 2, np.linspace(0, 448, 20011)]).astype(np.float32)
    x = np.concatenate([x, -x])
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(S.encode(x, "e4m3"), want)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_block_scale_is_the_smallest_power_of_two(kind):
    lim = S.LIMIT[kind]
    for a in [1e-45, 1e-38, 0.49, 1.0, lim, np.nextafter(lim, 1e9), 3.0e38]:
        s = S.block_scale(a, kind)
        assert a <= lim * s and np.log2(s) % 1 == 0
        assert s == 2.0 ** -126 or a > lim * s / 2
    assert S.block_scale(0.0, kind) == 0 and np.isnan(S.block_scale(np.inf, kind)) and np.isnan(S.block_scale(np.nan, kind))


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_growing_scale_stays_below_one_step(kind):
    """A page whose scale doubles with every token rounds its first values again
    and again; int8 values stay within one step of the final scale."""
    rng = np.random.RandomState(0)
    P, D = 16, 16
    codes, sc = np.zeros((1, 1, P, D), np.uint8), np.zeros((1, 1))
    x = (rng.randn(P, 1, D) * 2.0 ** np.arange(P)[:, None, None]).astype(np.float32)
    for t in range(P):
        S.append(codes, sc, x[t:t + 1], [t], P, kind)
    got = S.gather(codes, sc, np.arange(P), P, kind)[:, 0]
    err = np.abs(got - x[:, 0])
    step = sc[0, 0] if kind == "int8" else np.maximum(np.abs(x[:, 0]) * 2.0 ** -3, sc[0, 0] * 2.0 ** -9)
    assert np.all(err < step)


def test_attend_oracle_against_torch():
    rng = np.random.RandomState(1)
    P, H, G, D, T, F = 16, 2, 3, 32, 37, 4
    kc, vc = (rng.randint(0, 256, (5, H, P, D)).astype(np.uint8) for _ in range(2))
    ks, vs = (2.0 ** rng.randint(-8, -4, (5, H)) for _ in range(2))
    table = np.array([[3, 0, 4]], np.int32)
    q = rng.randn(F, H * G, D)
    out, lse, _, _ = S.attend(q, kc, vc, ks, vs, [T], [0, F], table, P, "int8", 0.3)
    slots = table[0, np.arange(T) // P] * P + np.arange(T) % P
    k = torch.from_numpy(S.gather(kc, ks, slots, P, "int8")).repeat_interleave(G, 1)
    v = torch.from_numpy(S.gather(vc, vs, slots, P, "int8")).repeat_interleave(G, 1)
    z = torch.einsum("thd,jhd->thj", torch.from_numpy(q), k) * 0.3
    z = z.masked_fill((torch.arange(T) > T - F + torch.arange(F)[:, None])[:, None], -np.inf)
    assert np.allclose(out, torch.einsum("thj,jhd->thd", z.softmax(2), v).numpy(), atol=1e-12)
    assert np.allclose(lse, z.logsumexp(2).numpy(), atol=1e-12)


def test_score_oracle_against_torch():
    rng = np.random.RandomState(2)
    x = np.round(rng.randn(4, 50), 1)  # with ties
    lp, en, rk, tl, ti = S.token_logprobs(x, [3, 49, -1, 50], 1.5, 7)
    d = torch.distributions.Categorical(logits=torch.from_numpy(x) * 1.5)
    assert np.allclose(en, d.entropy().numpy(), atol=1e-12)
    ref = torch.log_softmax(torch.from_numpy(x) * 1.5, 1).numpy()
    assert np.allclose(lp[:2], ref[[0, 1], [3, 49]], atol=1e-12) and lp[2] == 0 and np.isnan(lp[3])
    st = np.argsort(-x, 1, kind="stable")
    assert np.array_equal(ti, st[:, :7]) and np.allclose(tl, np.take_along_axis(ref, st[:, :7], 1), atol=1e-12)
    assert rk[0] == list(st[0]).index(3) and rk[2] == -1 and rk[3] == -1


def test_plan_oracle_by_hand():
    """Page size 4: request 0 grows into its second page, 1 ends and returns
    two, 2 starts with three, 3 finds the stack short, 4 needs none."""
    table = np.array([[5, -1, -1], [7, 8, -1], [-1, -1, -1], [-1, -1, -1], [9, -1, -1]], np.int32)
    free = np.array([1, 2, -1, -1], np.int32)
    got = S.batch_plan([4, 6, 0, 0, 2], [1, -1, 9, 1, 2], table, free, 2, 4, 16)
    t2, f2, slots, pos, req, lens, starts, status, left = got
    assert f2.tolist() == [1, 2, 7, 8] and status.tolist() == [0, 0, 0, 1, 0] and left == 0
    assert t2[0].tolist() == [5, 8, -1] and t2[2].tolist() == [7, 2, 1] and lens.tolist() == [5, 0, 9, 0, 4]
    assert starts.tolist() == [0, 1, 1, 10, 11, 13]
    assert slots.tolist() == [32, 28, 29, 30, 31, 8, 9, 10, 11, 4, -1, 38, 39, -1, -1, -1]
    assert pos[:13].tolist() == [4, 0, 1, 2, 3, 4, 5, 6, 7, 8, 0, 2, 3] and req[13:].tolist() == [-1] * 3


# ---------------------------------------------------------------- refusals

def _plan(Q, **kw):
    a = dict(n=2, seq=FAKE, new=FAKE + 64, page=16, table=FAKE + 128, stride=8, width=8, free=FAKE, cap=4, count=FAKE + 192,
             tokens=16, slots=FAKE, pos=FAKE + 256, req=FAKE + 320, lens=FAKE + 384, starts=FAKE + 448, status=FAKE + 512,
             left=FAKE + 576)
    a.update(kw)
    return Q.lib().seedq_batch_plan(*a.values(), None)


@pytest.mark.parametrize("kw", [
    dict(seq=None), dict(new=None), dict(table=None), dict(free=None), dict(count=None), dict(slots=None), dict(pos=None),
    dict(req=None), dict(lens=None), dict(starts=None), dict(status=None), dict(left=None), dict(n=0), dict(n=8193),
    dict(page=0), dict(width=0), dict(width=9), dict(width=(1 << 20) + 1, stride=1 << 21), dict(cap=-1), dict(tokens=0),
    dict(lens=FAKE), dict(left=FAKE + 192), dict(starts=FAKE + 64)])
def test_plan_refuses(Q, kw):
    assert _plan(Q, **kw) == 1


def _desc(Q, **kw):
    a = dict(kind=0, n_kv_heads=2, head_dim=64, page_size=16, n_pages=8, k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE,
             page_stride=2 * 16 * 64, head_stride=16 * 64, token_stride=64)
    a.update(kw)
    return Q.KvCacheDesc(*a.values())


BAD_CACHES = [(dict(kind=2), 1), (dict(n_kv_heads=0), 1), (dict(n_pages=0), 1), (dict(k=None), 1), (dict(v_scale=None), 1),
              (dict(head_dim=24), 6), (dict(head_dim=0), 6), (dict(head_dim=272), 6), (dict(page_size=8), 6),
              (dict(page_size=40), 6), (dict(page_size=512), 6), (dict(token_stride=48), 6), (dict(token_stride=72), 6),
              (dict(head_stride=0), 6), (dict(page_stride=-1024), 6), (dict(k=FAKE + 8), 6), (dict(n_kv_heads=2000), 6)]


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_cache_calls_refuse_bad_caches(Q, kw, status):
    L, d = Q.lib(), _desc(Q, **kw)
    r = C.byref(d)
    assert L.seedq_kv_append(r, FAKE, FAKE, 0, 128, 64, FAKE, 4, None) == status
    assert L.seedq_kv_gather(r, FAKE, 4, FAKE, FAKE, 0, 128, 64, None) == status
    assert L.seedq_kv_attend_workspace_bytes(r, 2000 if kw.get("n_kv_heads") == 2000 else 4, 1) == 0
    assert L.seedq_kv_attend(r, C.byref(_attend(Q)), None) == status


@pytest.mark.parametrize("a", [
    (None, FAKE, 0, 128, 64, FAKE, 4), (FAKE, None, 0, 128, 64, FAKE, 4), (FAKE, FAKE, 3, 128, 64, FAKE, 4),
    (FAKE, FAKE, -1, 128, 64, FAKE, 4), (FAKE, FAKE, 0, 128, 64, None, 4), (FAKE, FAKE, 0, 128, 64, FAKE, -1),
    (FAKE, FAKE, 0, 128, 64, FAKE, 1 << 31)])
def test_append_and_gather_refuse(Q, a):
    L, r = Q.lib(), C.byref(_desc(Q))
    k, v, dt, ts, hs, slots, n = a
    assert L.seedq_kv_append(r, *a, None) == 1
    assert L.seedq_kv_gather(r, slots, n, k, v, dt, ts, hs, None) == 1
    assert L.seedq_kv_append(None, *a, None) == 1


@pytest.mark.parametrize("n", [(1 << 31) - 1, 1 << 30, (1 << 28) + 1])
def test_append_and_gather_refuse_more_than_a_grid_takes(Q, n):
    """More CTAs than a launch counts (rows of stride 0 make such sizes possible): refused, not cut short."""
    d = _desc(Q, n_kv_heads=1024, head_dim=256, token_stride=256, head_stride=16 * 256, page_stride=1024 * 16 * 256)
    assert Q.lib().seedq_kv_append(C.byref(d), FAKE, FAKE, 0, 0, 0, FAKE, n, None) == 6
    assert Q.lib().seedq_kv_gather(C.byref(d), FAKE, n, FAKE, FAKE, 0, 0, 0, None) == 6


def test_nothing_to_do_is_ok(Q):
    L, r = Q.lib(), C.byref(_desc(Q))
    assert L.seedq_kv_append(r, None, None, 0, 0, 0, None, 0, None) == 0
    assert L.seedq_kv_gather(r, None, 0, None, None, 0, 0, 0, None) == 0
    assert L.seedq_token_logprobs(None, 0, 0, 10, 10, 1.0, None, None, None, None, 0, None, None, None, 0, None) == 0


def _attend(Q, **kw):
    a = dict(n_requests=2, n_heads=4, n_tokens=2, q=FAKE, qt=256, qh=64, out=FAKE, ot=256, oh=64, q_dtype=0, out_dtype=1,
             lse=None, seq_lens=FAKE, starts=FAKE, block_table=FAKE, table_stride=8, table_width=8, max_new=1, window=0,
             scale=0.125, workspace=FAKE, workspace_bytes=1 << 40)
    a.update(kw)
    return Q.AttendArgs(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(n_requests=0), 1), (dict(n_requests=8193), 1), (dict(n_heads=0), 1), (dict(n_heads=3), 6), (dict(n_tokens=-1), 1),
    (dict(q=None), 1), (dict(out=None), 1), (dict(q_dtype=3), 1), (dict(out_dtype=-1), 1), (dict(seq_lens=None), 1),
    (dict(starts=None), 1), (dict(block_table=None), 1), (dict(table_width=0), 1), (dict(table_width=9), 1),
    (dict(max_new=0), 1), (dict(window=-1), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1),
    (dict(workspace=None), 1), (dict(workspace=FAKE + 8), 1), (dict(workspace_bytes=0), 1)])
def test_attend_refuses(Q, kw, status):
    L, d = Q.lib(), _desc(Q)
    assert L.seedq_kv_attend(C.byref(d), C.byref(_attend(Q, **kw)), None) == status
    assert L.seedq_kv_attend(C.byref(d), None, None) == 1
    assert L.seedq_kv_attend(None, C.byref(_attend(Q)), None) == 1


@pytest.mark.parametrize("dim", [16, 64, 80, 128, 144, 256])
@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 8, 9, 17])
def test_attend_workspace_serves_fewer_tokens(Q, dim, group):
    d = _desc(Q, head_dim=dim, token_stride=dim, head_stride=16 * dim, page_stride=32 * dim)
    n = [Q.lib().seedq_kv_attend_workspace_bytes(C.byref(d), 2 * group, m) for m in [*range(1, 34), 1000, (1 << 31) - 1]]
    assert n[0] > 0 and n == sorted(n)


@pytest.mark.parametrize("n,heads", [(1 << 30, 4), ((1 << 31) - 1, 2), (((1 << 31) - 32) // 8, 16)])
def test_attend_refuses_more_rows_than_it_numbers(Q, n, heads):
    d = _desc(Q)
    assert Q.lib().seedq_kv_attend(C.byref(d), C.byref(_attend(Q, n_tokens=n, n_heads=heads)), None) == 6


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(dt=3), dict(rows=-1), dict(vocab=0), dict(vocab=(1 << 30) + 1, stride=1 << 31), dict(stride=9),
    dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(lp=None), dict(rank=None), dict(k=-1), dict(k=33),
    dict(tl=None), dict(ti=None), dict(ws=None), dict(ws=FAKE + 4), dict(wb=0)])
def test_logprobs_refuse(Q, kw):
    a = dict(x=FAKE, dt=0, rows=3, vocab=10, stride=10, scale=1.0, t=FAKE, lp=FAKE, en=FAKE, rank=FAKE, k=2, tl=FAKE, ti=FAKE,
             ws=FAKE, wb=1 << 40)
    a.update(kw)
    assert Q.lib().seedq_token_logprobs(*a.values(), None) == 1


def test_binding_refuses_what_the_abi_cannot_see(Q):
    from paper_2609_38477_gb300 import serving as V

    z = torch.zeros
    k = z((4, 2, 16, 64), dtype=torch.int8)
    s = z((4, 2))
    with pytest.raises(ValueError, match="kind"):
        V.KVCache(k, k, s, s, "int4")
    with pytest.raises(ValueError, match="strides"):
        V.KVCache(k, z((4, 16, 2, 64), dtype=torch.int8).transpose(1, 2), s, s)
    with pytest.raises(ValueError, match="codes"):
        V.KVCache(k.float(), k.float(), s, s)
    with pytest.raises(ValueError, match="n_pages"):
        V.KVCache(k, k, s.t().contiguous().t(), s)
    with pytest.raises(ValueError, match="CUDA"):
        V.KVCache(k, k, s, s)
    with pytest.raises(ValueError, match="logits"):
        V.token_logprobs(z((2, 8)), None, None, None, None, None, None, z(1))
    plan = V.BatchPlan(4, 16, device="cpu")
    i = z(4, dtype=torch.int32)
    t = z((4, 3), dtype=torch.int32)
    for bad in (dict(seq_lens=i.long()), dict(n_new=z(5, dtype=torch.int32)), dict(seq_lens=i[:2]), dict(block_table=t.t()),
                dict(block_table=t[:2]), dict(free_count=z(2, dtype=torch.int64)), dict(free_pages=z(8, dtype=torch.int32)[::2])):
        a = dict(seq_lens=i, n_new=i, block_table=t, free_pages=i, free_count=i[:1], page_size=16, stream=0)
        a.update(bad)
        with pytest.raises(ValueError):
            plan.build(**a)


def test_plan_of_fewer_requests_hands_on_no_others(Q, monkeypatch):
    """A build with fewer requests writes fewer offsets; what is handed on ends there, at the same addresses."""
    from paper_2609_38477_gb300 import serving as V

    class Library:
        def seedq_batch_plan(self, n, *a):
            return 0

    plan = V.BatchPlan(4, 16, device="cpu")
    base = [t.data_ptr() for t in (plan.seq_lens, plan.starts, plan.status)]
    monkeypatch.setattr(Q, "lib", Library)
    monkeypatch.setattr(V, "_current_device", lambda: None)  # as the CPU's tensors have it
    i = torch.zeros(4, dtype=torch.int32)
    for n in (4, 2, 2, 3, 1, 4):
        plan.build(i, i[:n], torch.zeros((4, 3), dtype=torch.int32), i, i[:1], 16, stream=0)
        assert (plan.seq_lens.shape[0], plan.starts.shape[0], plan.status.shape[0]) == (n, n + 1, n)
        assert [t.data_ptr() for t in (plan.seq_lens, plan.starts, plan.status)] == base


@pytest.mark.parametrize("stream", [None, 0])
def test_binding_refuses_another_device_than_the_current_one(Q, monkeypatch, stream):
    """The library launches on the current device; tensors of another one never reach it."""
    from paper_2609_38477_gb300 import serving as V

    class Library:
        def __getattr__(self, name):
            return lambda *a: pytest.fail(f"{name} is called")

    monkeypatch.setattr(Q, "lib", Library)
    z = lambda *shape, dt=torch.int32: torch.zeros(shape, dtype=dt, device="meta")  # noqa: E731
    cache = V.KVCache.__new__(V.KVCache)
    cache.n_pages, cache.n_kv_heads, cache.page_size, cache.head_dim, cache.device, cache._ref = 4, 2, 16, 64, z(1).device, None
    plan = V.BatchPlan(2, 4, device="meta")
    f = lambda *shape: z(*shape, dt=torch.float32)  # noqa: E731
    calls = [lambda: plan.build(z(2), z(2), z(2, 3), z(4), z(1), 16, stream=stream),
             lambda: cache.append(f(3, 2, 64), f(3, 2, 64), z(3, dt=torch.int64), stream=stream),
             lambda: cache.gather(z(3, dt=torch.int64), f(3, 2, 64), f(3, 2, 64), stream=stream),
             lambda: cache.attend(f(2, 4, 64), f(2, 4, 64), z(2), z(3), z(2, 3), z(8, dt=torch.uint8), stream=stream)]
    for current in (0, 1):
        monkeypatch.setattr(V, "_current_device", lambda: current)
        for call in calls:
            with pytest.raises(ValueError, match="current device"):
                call()
    monkeypatch.setattr(V, "_current_device", lambda: 0)
    with pytest.raises(ValueError, match="current device"):  # where the log probabilities, for which no tensor can stand in, ask
        V._stream(stream, torch.device("cuda", 1))
    assert V._stream(7, torch.device("cuda", 0)) == 7


def test_strides_of_single_entries_do_not_matter(Q, monkeypatch):
    """torch leaves the stride of a dimension of one entry open: keys and values of
    one token or one head, a table of one page, whatever their strides there."""
    from paper_2609_38477_gb300 import serving as V

    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: calls.append((name, a)) or 0

    monkeypatch.setattr(Q, "lib", Library)
    monkeypatch.setattr(V, "_current_device", lambda: None)
    cache = V.KVCache.__new__(V.KVCache)
    cache.page_size, cache.head_dim, cache.device, cache._ref = 16, 64, torch.device("cpu"), None
    i64 = torch.zeros(9, dtype=torch.int64)
    for n, h in ((1, 4), (5, 1), (1, 1), (0, 4)):
        cache.n_kv_heads = h
        k = torch.zeros(n, h, 64)
        v = torch.zeros(4096).as_strided((n, h, 64), [x if m > 1 else 777 for m, x in zip(k.shape, k.stride())])
        for a, b in ((k, v), (v, k)):
            assert a.stride() != b.stride()
            cache.append(a, b, i64, stream=0)
            cache.gather(i64, a, b, stream=0)
            for name, at in (("seedq_kv_append", 4), ("seedq_kv_gather", 6)):
                args = next(c for f, c in reversed(calls) if f == name)
                assert all(m < 2 or x == s for m, x, s in zip((n, h), args[at:at + 2], a.stride()))
    cache.n_kv_heads = 4
    with pytest.raises(ValueError, match="strides"):
        cache.append(torch.zeros(2, 4, 64), torch.zeros(4, 2, 64).transpose(0, 1), i64, stream=0)
    plan = V.BatchPlan(3, 4, device="cpu")
    i = torch.zeros(4, dtype=torch.int32)
    table = torch.zeros(6, dtype=torch.int32).as_strided((3, 1), (1, 7))
    plan.build(i, i[:3], table, i, i[:1], 16, stream=0)
    assert calls[-1][0] == "seedq_batch_plan" and calls[-1][1][5:7] == (1, 1)
