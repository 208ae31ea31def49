"""The decode loop over compressed layers against a plain recomputation in fp64.

The reference multiplies the decoded weights, rounds to bfloat16 where the loop
does, and attends over the numbers that the loop's caches hold (read back by
gather), so what remains are float32 sums and bfloat16 roundings that fall the
other way: each of those moves a product's input by 2^-8 of a number, a few per
row of hundreds, and two layers of them stay well below 1% of the largest logit.
A wrong page, slot, position, head or mask moves logits by their own size.
"""
import os
import sys

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    from paper_2609_38477_gb300 import build

    build.build()
    from paper_2609_38477_gb300 import generate

    return generate


def dense(layer):
    w = torch.empty((layer.rows, layer.cols), device="cuda")
    layer.decode_weights(w)
    return w.double()


def bf(x):
    return x.float().bfloat16().double()


def norm(x, gain):
    return bf(x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-5) * gain.double())


def rope(x, pos, freqs):
    a = pos[:, None].double() * freqs.double()
    c, s = torch.cos(a)[:, None], torch.sin(a)[:, None]
    u, v = x.chunk(2, 2)
    return torch.cat([u * c - v * s, v * c + u * s], 2)


def reference(d, weights, history, r, count):
    """Logits of the last `count` tokens of request r, whose tokens are history."""
    s = d.spec
    n = len(history)
    slots = d.table[r, torch.arange(n, device="cuda") // d.page_size].long() * d.page_size + torch.arange(n, device="cuda") % d.page_size
    pos = torch.arange(n - count, n, device="cuda")
    x = d.embedding[torch.tensor(history[n - count:], device="cuda")].double()
    for block, cache, w in zip(d.blocks, d.caches, weights):
        h = norm(x, block["attn_norm"])
        q = rope((h @ w["q"].T).view(count, s.n_heads, s.head_dim), pos, d.freqs)
        k, v = (torch.empty((n, s.n_kv_heads, s.head_dim), device="cuda") for _ in range(2))
        cache.gather(slots, k, v)
        own = rope((h @ w["k"].T).view(count, s.n_kv_heads, s.head_dim), pos, d.freqs)
        # A page's power-of-two scale is at most its largest number / 63.5, and older tokens on the page count.
        step = max(float(own.abs().max()), float(k.abs().max())) / 63
        assert float((k[n - count:].double() - own).abs().max()) <= (step if cache.kind == "int8" else 4 * step)
        g = s.n_heads // s.n_kv_heads
        z = torch.einsum("thd,jhd->thj", q, k.double().repeat_interleave(g, 1)) * s.head_dim ** -0.5
        z = z.masked_fill((torch.arange(n, device="cuda") > pos[:, None])[:, None], -np.inf)
        o = torch.einsum("thj,jhd->thd", z.softmax(2), v.double().repeat_interleave(g, 1))
        x = x + bf(o).reshape(count, -1) @ w["o"].T
        h = norm(x, block["mlp_norm"])
        x = x + bf(torch.nn.functional.silu(h @ w["gate"].T) * (h @ w["up"].T)) @ w["down"].T
    return norm(x, d.final_norm) @ weights[-1]["head"].T


@pytest.mark.parametrize("name,kind,page", [("tiny", "int8", 16), ("tiny", "e4m3", 32), ("tiny_odd", "int8", 16)])
def test_decode_loop(G, name, kind, page):
    d = G.synthetic_decoder(name, max_requests=3, n_pages=7, page_size=page, kind=kind)
    weights = [{k: dense(b[k]) for k in ("q", "k", "v", "o", "gate", "up", "down")} for b in d.blocks] + [{"head": dense(d.head)}]
    rng = np.random.RandomState(3)
    vocab = d.spec.vocab
    history = [[], [], []]
    # prompts in pieces, single tokens, a pause, an end whose pages another request takes
    for new in ([5, 1, 9], [7, 9, 0], [1, 1, 1], [1, 0, 1], [16, 0, 0], [-1, 1, 1], [4, 0, 12], [1, 1, 1]):
        tokens = []
        for r, n in enumerate(new):
            if n < 0:
                history[r] = []
            fresh = [int(t) for t in rng.randint(0, vocab, max(n, 0))]
            history[r] += fresh
            tokens += fresh
        logits = d.step(torch.tensor(tokens, device="cuda"), torch.tensor(new, dtype=torch.int32, device="cuda"))
        assert d.plan.status.tolist() == [0, 0, 0]
        assert d.seq_lens.tolist() == [len(h) for h in history]
        at = 0
        for r, n in enumerate(new):
            if n <= 0:
                continue
            want = reference(d, weights, history[r], r, n)
            got = logits[at:at + n].double()
            assert float((got - want).abs().max()) <= 0.01 * float(want.abs().max())
            at += n
        targets = torch.tensor([int(t) for t in rng.randint(0, vocab, at)], device="cuda")
        logp, entropy, rank, top, best = d.score(logits, targets, top_k=4, temperature=0.8)
        ref = torch.log_softmax(logits.double() / 0.8, 1)
        assert torch.allclose(logp.double(), ref.gather(1, targets[:, None])[:, 0], atol=1e-5)
        assert torch.allclose(entropy.double(), -(ref.exp() * ref).sum(1), atol=1e-5)
        assert torch.equal(best[:, 0].long(), logits.argmax(1)) and torch.allclose(top.double(), ref.topk(4).values, atol=1e-5)
    assert int(d.free_count) + int((-(-d.seq_lens // page)).sum()) == 7
    with_room = d.table.clone()
    # a request that the pages cannot hold is told so, and its neighbours go on
    d.step(torch.tensor([1] * 16, device="cuda"), torch.tensor([0, 16, 0], dtype=torch.int32, device="cuda"))
    while int(d.plan.status[1]) == 0:
        d.step(torch.tensor([1] * 16, device="cuda"), torch.tensor([0, 16, 0], dtype=torch.int32, device="cuda"))
    assert d.plan.status.tolist() == [0, 1, 0] and bool((d.plan.slots == -1).all())
    assert torch.equal(d.table[0], with_room[0]) and torch.equal(d.table[2], with_room[2])


def test_example_runs(G, capsys):
    G.main()
    assert capsys.readouterr().out.count("step") == 6


def test_step_of_fewer_requests(G):
    """A step of the first requests alone: the others keep their lengths, and the logits are those of a smaller batch."""
    t = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    d, e = (G.synthetic_decoder("tiny", max_requests=r, n_pages=6) for r in (3, 2))
    tokens = torch.arange(16, device="cuda")
    d.step(tokens, t(5, 4, 7))
    e.step(tokens[:9], t(5, 4))
    for new in ((3, 6), (1, 1), (0, 2)):
        a, b = (x.step(tokens[:sum(new)], t(*new)) for x in (d, e))
        assert float((a - b).abs().max()) <= 0.01 * float(b.abs().max())
    assert d.seq_lens.tolist() == [9, 13, 7] and e.seq_lens.tolist() == [9, 13]


def test_step_that_only_ends_requests(G):
    """The last requests of a batch end together, alone in a step; their pages are there again."""
    d = G.synthetic_decoder("tiny", max_requests=2, n_pages=3)
    t = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    for _ in range(3):
        logits = d.step(torch.arange(12, device="cuda"), t(4, 8))
        assert logits.shape == (12, d.spec.vocab) and int(d.free_count) == 1
        assert d.step(none, t(0, 0)).shape == (0, d.spec.vocab) and d.seq_lens.tolist() == [4, 8] and int(d.free_count) == 1
        assert d.step(none, t(-1, -1)).shape == (0, d.spec.vocab)
        assert d.seq_lens.tolist() == [0, 0] and int(d.free_count) == 3
        assert sorted(d.free.tolist()) == [0, 1, 2]


def test_step_that_refuses_a_request(G):
    """The logits of a request that got no pages are NaN, its neighbours' what they are without it."""
    t = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    tokens = torch.arange(16, device="cuda")
    got = []
    for new in ((1, 12, 3), (1, 0, 3)):
        d = G.synthetic_decoder("tiny", max_requests=3, n_pages=3)
        d.step(tokens, t(12, 1, 3))
        mine = tokens[:16] if new[1] else torch.cat([tokens[:1], tokens[13:]])
        d.free_count.fill_(0)
        d.seq_lens[1] = 16 if new[1] else 1  # a full page: the next tokens want another
        got.append((d.step(mine, t(*new)), d))
    (a, d), (b, _) = got
    assert d.plan.status.tolist() == [0, 1, 0] and d.seq_lens.tolist() == [13, 16, 6]
    assert bool(a[1:13].isnan().all()) and not bool(a[:1].isnan().any()) and not bool(a[13:].isnan().any())
    own = torch.cat([a[:1], a[13:]])
    assert float((own - b).abs().max()) <= 0.01 * float(b.abs().max())
    logp, entropy, rank, top, _ = d.score(a, torch.zeros(16, dtype=torch.int64, device="cuda"), top_k=2)
    assert bool(logp[1:13].isnan().all()) and bool(top[1:13].isnan().all()) and bool((rank[1:13] == -1).all())


def test_example_says_what_the_plan_refused(G, monkeypatch):
    """A page too few for the prompts: an error, and no token is taken from logits of NaN."""
    make = G.synthetic_decoder
    monkeypatch.setattr(G, "synthetic_decoder", lambda: make("tiny", n_pages=2))
    with pytest.raises(RuntimeError, match="no pages"):
        G.main()


@pytest.mark.parametrize("name,kind", [("tiny", "int8"), ("tiny_odd", "e4m3")])
def test_decode_loop_caches_values(G, name, kind):
    """The cached values of every layer against their own product: one rounding
    under the page's scale, at most its largest number / 63.5 (E4M3: a sixteenth of a
    number at most), and neither the keys nor another layer's values."""
    d = G.synthetic_decoder(name, max_requests=2, n_pages=6, kind=kind)
    s = d.spec
    weights = [{k: dense(b[k]) for k in ("q", "v", "o", "gate", "up", "down")} for b in d.blocks]
    rng = np.random.RandomState(5)
    history = [[], []]
    for new in ([7, 9], [1, 1], [1, 15], [12, 1]):
        fresh = [[int(t) for t in rng.randint(0, s.vocab, n)] for n in new]
        d.step(torch.tensor(fresh[0] + fresh[1], device="cuda"), torch.tensor(new, dtype=torch.int32, device="cuda"))
        for r, m in enumerate(new):
            history[r] += fresh[r]
            n = len(history[r])
            at = torch.arange(n, device="cuda")
            slots, pos = d.table[r, at // d.page_size].long() * d.page_size + at % d.page_size, at[n - m:]
            x = d.embedding[torch.tensor(fresh[r], device="cuda")].double()
            for block, cache, w in zip(d.blocks, d.caches, weights):
                h = norm(x, block["attn_norm"])
                k, v = (torch.empty((n, s.n_kv_heads, s.head_dim), device="cuda") for _ in range(2))
                cache.gather(slots, k, v)
                own = (h @ w["v"].T).view(m, s.n_kv_heads, s.head_dim)
                step = max(float(own.abs().max()), float(v.abs().max())) / 63
                off = float((v[n - m:].double() - own).abs().max())
                assert off <= (step if kind == "int8" else 4 * step) < 0.2 * float((k[n - m:].double() - own).abs().max())
                q = rope((h @ w["q"].T).view(m, s.n_heads, s.head_dim), pos, d.freqs)
                g = s.n_heads // s.n_kv_heads
                z = torch.einsum("thd,jhd->thj", q, k.double().repeat_interleave(g, 1)) * s.head_dim ** -0.5
                z = z.masked_fill((at > pos[:, None])[:, None], -np.inf)
                o = torch.einsum("thj,jhd->thd", z.softmax(2), v.double().repeat_interleave(g, 1))
                x = x + bf(o).reshape(m, -1) @ w["o"].T
                h = norm(x, block["mlp_norm"])
                x = x + bf(torch.nn.functional.silu(h @ w["gate"].T) * (h @ w["up"].T)) @ w["down"].T
