"""The serving operators between the compressed products, as cases that can be timed and compared.

Four groups, named by a case's "op":
  plan    block tables, slot maps and token positions from request lengths
  append  new keys and values written to the 8-bit paged cache, and the blocks they touch read back
  attend  attention of new tokens over the 8-bit paged cache
  score   log probability, rank, entropy and top alternatives of given tokens under a row of logits

`run` computes them in plain torch operations where `own` is false and through
the package's entry points where it is true.  `exact` computes the same in 64 bits.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
WIDTH = {"f32": 4, "bf16": 2, "f16": 2}
# (query heads, key-value heads, head dim): the Llama-2-7B, Llama-3-8B and Llama-2-70B shapes, the small test
# models (head dims 64 and 32, five heads on one), and two generic ones
HEADS = [(32, 32, 128), (32, 8, 128), (64, 8, 128), (4, 2, 64), (5, 1, 32), (16, 2, 256), (12, 4, 96)]
VOCABS = [77, 272, 300, 32000, 128256]
MOST_ELEMENTS = 4 * 131072 * 8 * 128  # cache values a drawn attention case may hold, padded to the longest request


# ---------------------------------------------------------------- cases

def listed():
    return [
        # a decode step's bookkeeping: 16 requests, one token each
        dict(name="plan_decode", op="plan", requests=16, max_len=4096, new="one", max_new=1, page=16, tight=False, mix=1),
        # a mixed step: prompts beside running requests, some finishing, the page pool running out
        dict(name="plan_mixed", op="plan", requests=600, max_len=8192, new="mixed", max_new=512, page=64, tight=True, mix=2),
        # the cache write of a decode step, f32 as the products leave it
        dict(name="append_decode", op="append", requests=16, max_len=4096, new="one", max_new=1, heads=8, dim=128,
             page=16, kind="int8", order="head", dtype="f32", mix=3),
        # prompts of the Llama-2-7B shape, 4096 tokens in all
        dict(name="append_prompt", op="append", requests=4, max_len=100, new="full", max_new=1024, heads=32, dim=128,
             page=64, kind="e4m3", order="head", dtype="bf16", mix=4),
        # ragged prompts of a small model, tokens before heads in a page
        dict(name="append_ragged", op="append", requests=7, max_len=333, new="mixed", max_new=217, heads=4, dim=64,
             page=32, kind="int8", order="token", dtype="f16", mix=5),
        # one user's next token on a short context: latency
        dict(name="attend_one", op="attend", requests=1, max_len=1000, new="one", max_new=1, q_heads=32, heads=8, dim=128,
             page=16, kind="int8", order="head", dtype="f32", out="bf16", window=0, mix=6),
        # a full decode batch of the Llama-2-70B shape, contexts of very different lengths
        dict(name="attend_batch", op="attend", requests=16, max_len=8192, new="one", max_new=1, q_heads=64, heads=8, dim=128,
             page=16, kind="int8", order="head", dtype="f32", out="bf16", window=0, mix=7),
        # four long contexts of the Llama-3-8B shape
        dict(name="attend_long", op="attend", requests=4, max_len=131072, new="one", max_new=1, q_heads=32, heads=8, dim=128,
             page=64, kind="e4m3", order="head", dtype="bf16", out="f32", window=0, even=True, mix=8),
        # a 16-token piece of a prompt (the widest product) of the Llama-2-7B shape behind a sliding window
        dict(name="attend_piece", op="attend", requests=1, max_len=4001, new="full", max_new=16, q_heads=32, heads=32, dim=128,
             page=32, kind="int8", order="token", dtype="bf16", out="bf16", window=3000, mix=9),
        # the smallest: a few rows of a small model's head
        dict(name="score_tiny", op="score", rows=5, vocab=300, dtype="bf16", top=3, scale=1.0, masked=False),
        # a decode step of the Llama-3-8B head with 20 alternatives
        dict(name="score_decode", op="score", rows=16, vocab=128256, dtype="f32", top=20, scale=1.25, masked=False),
        # scoring a text of 2048 tokens
        dict(name="score_text", op="score", rows=2048, vocab=128256, dtype="f32", top=5, scale=1.0, masked=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["plan", "append", "append", "attend", "attend", "attend", "score", "score"])
    page = rng.choice([16, 32, 64, 128])
    mix = rng.randrange(1 << 20)
    if op == "plan":
        return dict(op=op, requests=_log_int(rng, 1, 600), max_len=_log_int(rng, 1, 8192), new=rng.choice(["one", "mixed", "full"]),
                    max_new=_log_int(rng, 1, 128), page=page, tight=rng.random() < 0.4, mix=mix)
    common = dict(page=page, kind=rng.choice(["int8", "e4m3"]), order=rng.choice(["head", "token"]),
                  dtype=rng.choice(list(DTYPES)), mix=mix)
    if op == "append":
        _, h, d = rng.choice(HEADS)
        n = _log_int(rng, 1, 64)
        most = max(1, 4096 * 32 * 128 // (n * h * d))  # new values within the largest listed case's
        return dict(op=op, requests=n, max_len=_log_int(rng, 1, 4096), new=rng.choice(["one", "mixed", "full"]),
                    max_new=_log_int(rng, 1, min(1024, most)), heads=h, dim=d, **common)
    if op == "attend":
        q, h, d = rng.choice(HEADS)
        n = _log_int(rng, 1, 64)
        new = _log_int(rng, 1, 16)
        # the plain form's longest request decides its cost: cache values, and scores of every query head and token
        most = min(131072, MOST_ELEMENTS // (n * h * d), 4 * 131072 * 32 // (n * q * new))
        return dict(op=op, requests=n, max_len=_log_int(rng, new, max(new, most)), new=rng.choice(["one", "mixed", "full"]),
                    max_new=new, q_heads=q, heads=h, dim=d, out=rng.choice(list(DTYPES)), even=rng.random() < 0.3,
                    window=rng.choice([0, 0, _log_int(rng, 1, 4096)]), **common)
    vocab = rng.choice([rng.choice(VOCABS), _log_int(rng, 40, 128256)])
    return dict(op=op, rows=_log_int(rng, 1, min(4096, 2048 * 128256 // vocab)), vocab=vocab, dtype=rng.choice(list(DTYPES)),
                top=rng.choice([0, 1, 5, 20, 32]), scale=rng.choice([1.0, 0.7, 1.25]), masked=rng.random() < 0.4)


# ---------------------------------------------------------------- inputs

def _lengths(case):
    """Lengths before the step and new tokens of every request, from the case alone.

    One request has the longest context; the others are spread over the range,
    among them (in a batch of four or more) an empty one and one of one token.
    With "even" all of them are long."""
    rng = random.Random(case["mix"])
    n, most, new = case["requests"], case["max_len"], case["max_new"]
    even = case.get("even", False)
    before = [rng.randint(most - most // 4, most) if even else _log_int(rng, 1, most) for _ in range(n)]
    before[0] = most
    if n >= 4 and not even:
        before[1], before[2] = 0, 1
    if case["new"] == "one":
        fresh = [1] * n
    elif case["new"] == "full":
        fresh = [new] * n
    else:
        fresh = [1 if rng.random() < 0.5 else rng.randint(1, new) for _ in range(n)]
        if n >= 4:
            fresh[3] = 0
    return before, fresh


def _ceil(a, b):
    return -(-a // b)


def _pages(total, seed):
    return np.random.RandomState(seed % (1 << 31)).permutation(total).astype(np.int32)


def _prepare_plan(case, seed):
    before, fresh = _lengths(case)
    page, n = case["page"], case["requests"]
    if case["new"] == "mixed":  # some requests end with this step
        fresh = [-1 if i % 11 == 10 else f for i, f in enumerate(fresh)]
    held = [_ceil(x, page) for x in before]
    need = [_ceil(x + f, page) - h if f >= 0 else 0 for x, f, h in zip(before, fresh, held)]
    spare = sum(need) // 2 if case["tight"] else sum(need) + 5
    total = sum(held) + spare
    width = _ceil(case["max_len"] + case["max_new"], page)
    ids = _pages(total + 64, seed)
    table = np.full((n, width), -1, np.int32)
    at = 0
    for i, h in enumerate(held):
        table[i, :h] = ids[at:at + h]
        at += h
    free = np.full(total + 1, -1, np.int32)
    free[:spare] = ids[at:at + spare]
    tokens = max(1, sum(max(f, 0) for f in fresh))
    tokens = _ceil(tokens, 64) * 64  # a step's buffers have a fixed size: the rest is marked unused
    g = lambda v: torch.tensor(np.asarray(v, np.int32), device="cuda")  # noqa: E731
    s = dict(case=case, seq=g(before), new=g(fresh), table=g(table), free=g(free), count=g([spare]), tokens=tokens)
    if own:
        from paper_2609_38477_gb300 import serving

        s["plan"] = serving.BatchPlan(n, tokens)
    return s


def _cache(case, gen, pages):
    """A cache that already holds tokens: random codes under power-of-two scales, in either page order."""
    p, h, d = case["page"], case["heads"], case["dim"]
    shape = (pages, h, p, d) if case["order"] == "head" else (pages, p, h, d)
    out = []
    for _ in range(2):
        codes = torch.empty(shape, dtype=torch.int8, device="cuda")
        for part in codes.split(max(1, (1 << 26) // (p * h * d))):
            x = torch.randn(part.shape, generator=gen, device="cuda")
            if case["kind"] == "int8":
                part.copy_((x * 32).round_().clamp_(-127, 127))
            else:
                part.copy_((x * 96).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.int8))
        e = torch.randint(-6, -3, (pages, h), generator=gen, device="cuda")
        scale = torch.pow(2.0, e.float() - (0 if case["kind"] == "int8" else 2))
        out.append((codes if case["order"] == "head" else codes.transpose(1, 2), scale))
    return out


def _tables(case, before, fresh, seed):
    """A block table over shuffled pages, and slots and offsets of the step's tokens."""
    page = case["page"]
    after = [x + f for x, f in zip(before, fresh)]
    held = [_ceil(x, page) for x in after]
    ids = _pages(max(1, sum(held)), seed)
    table = np.full((len(before), max(1, max(held))), -1, np.int32)
    at, slots, touched = 0, [], []
    for i, h in enumerate(held):
        table[i, :h] = ids[at:at + h]
        at += h
        pos = np.arange(before[i], after[i])
        slots.append(table[i, pos // page].astype(np.int64) * page + pos % page)
        if fresh[i]:  # what the blocks hold that this step writes to
            pos = np.arange(before[i] // page * page, after[i])
            touched.append(table[i, pos // page].astype(np.int64) * page + pos % page)
    cat = lambda v: np.concatenate(v) if v else np.zeros(0, np.int64)  # noqa: E731
    return ids.size, table, cat(slots), cat(touched), after


def _prepare_append(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    before, fresh = _lengths(case)
    pages, _, slots, touched, _ = _tables(case, before, fresh, seed)
    (k, ks), (v, vs) = _cache(case, gen, pages)
    n, h, d = slots.size, case["heads"], case["dim"]
    dt = DTYPES[case["dtype"]]
    # tokens differ in size: some outgrow the scale of the block they join
    size = torch.exp(0.8 * torch.randn((2, n, 1, 1), generator=gen, device="cuda"))
    kv = (size * torch.randn((2, n, h, d), generator=gen, device="cuda")).to(dt)
    s = dict(case=case, k=k, v=v, ks=ks, vs=vs, new_k=kv[0], new_v=kv[1], slots=torch.from_numpy(slots).cuda(),
             read=torch.from_numpy(touched).cuda())
    s["out_k"] = torch.empty((touched.size, h, d), dtype=dt, device="cuda")
    s["out_v"] = torch.empty_like(s["out_k"])
    if own:
        from paper_2609_38477_gb300 import serving

        s["cache"] = serving.KVCache(k, v, ks, vs, case["kind"])
    return s


def _prepare_attend(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    after, fresh = _lengths(case)  # here the range is of lengths that count the new tokens
    after = [max(x, f) for x, f in zip(after, fresh)]
    before = [x - f for x, f in zip(after, fresh)]
    pages, table, _, _, _ = _tables(case, before, fresh, seed)
    (k, ks), (v, vs) = _cache(case, gen, pages)
    n, hq, d = sum(fresh), case["q_heads"], case["dim"]
    start = np.concatenate([[0], np.cumsum(fresh)]).astype(np.int32)
    s = dict(case=case, k=k, v=v, ks=ks, vs=vs, table=torch.from_numpy(table).cuda(), start=torch.from_numpy(start).cuda(),
             seq=torch.tensor(np.asarray(after, np.int32), device="cuda"), longest=max(after), widest=max(max(fresh), 1),
             q=(2.0 * torch.randn((n, hq, d), generator=gen, device="cuda")).to(DTYPES[case["dtype"]]))
    req = np.repeat(np.arange(len(fresh)), fresh)
    s["req"] = torch.from_numpy(req).cuda()
    s["step"] = torch.from_numpy(np.arange(n) - start[req]).cuda()
    s["out"] = torch.empty((n, hq, d), dtype=DTYPES[case["out"]], device="cuda")
    s["lse"] = torch.empty((n, hq), dtype=torch.float32, device="cuda")
    if own:
        from paper_2609_38477_gb300 import serving

        s["cache"] = serving.KVCache(k, v, ks, vs, case["kind"])
        s["work"] = s["cache"].attend_workspace(hq, s["widest"])
    return s


def _prepare_score(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    n, v = case["rows"], case["vocab"]
    x = torch.empty((n, v), dtype=DTYPES[case["dtype"]], device="cuda")
    for part in x.split(max(1, (1 << 27) // v)):
        z = 2.5 * torch.randn(part.shape, generator=gen, device="cuda")
        if case["masked"]:  # tokens that a grammar or a ban list rules out
            z.masked_fill_(torch.rand(part.shape, generator=gen, device="cuda") < 0.3, -math.inf)
        part.copy_(z)
    t = torch.randint(0, v, (n,), generator=gen, device="cuda")
    t[n // 2:] = x[n // 2:].argmax(1)  # half of them the likeliest token, as in a text that the model wrote
    if n >= 4:
        t[1] = -1  # a row with no target (padding)
    g = lambda *shape, dt=torch.float32: torch.empty(shape, dtype=dt, device="cuda")  # noqa: E731
    s = dict(case=case, x=x, t=t, logprob=g(n), entropy=g(n), rank=g(n, dt=torch.int32), top=g(n, case["top"]),
             top_id=g(n, case["top"], dt=torch.int32))
    if own:
        from paper_2609_38477_gb300 import serving

        s["work"] = serving.score_workspace(n, v)
    return s


def prepare(case, seed):
    return {"plan": _prepare_plan, "append": _prepare_append, "attend": _prepare_attend, "score": _prepare_score}[case["op"]](case, seed)


# ---------------------------------------------------------------- the package's calls

def _own_plan(s):
    p = s["plan"]
    p.build(s["seq"], s["new"], s["table"], s["free"], s["count"], s["case"]["page"])
    return [s["table"], s["free"], p.slots, p.positions, p.requests, p.seq_lens, p.starts, p.status, p.free_count]


def _own_append(s):
    s["cache"].append(s["new_k"], s["new_v"], s["slots"])
    s["cache"].gather(s["read"], s["out_k"], s["out_v"])
    return [s["out_k"], s["out_v"]]


def _own_attend(s):
    s["cache"].attend(s["q"], s["out"], s["seq"], s["start"], s["table"], s["work"], max_new=s["widest"],
                      window=s["case"]["window"], lse=s["lse"])
    return [s["out"], s["lse"]]


def _own_score(s):
    from paper_2609_38477_gb300 import serving

    serving.token_logprobs(s["x"], s["t"], s["logprob"], s["entropy"], s["rank"], s["top"], s["top_id"], s["work"],
                           scale=s["case"]["scale"])
    return [s["logprob"], s["entropy"], s["rank"], s["top"], s["top_id"]]


# ---------------------------------------------------------------- the plain forms

def _plain_plan(s):
    page, table, free = s["case"]["page"], s["table"], s["free"]
    seq, new = s["seq"].long(), s["new"].long()
    width, dev = table.shape[1], table.device
    n = new.clamp(min=0)
    ends = n.cumsum(0)
    starts = torch.cat([ends.new_zeros(1), ends]).clamp(max=s["tokens"])
    held, wanted = (seq + page - 1) // page, (seq + n + page - 1) // page
    bad = (new < -1) | (seq < 0) | (wanted > width)
    full = ends > s["tokens"]
    gone = (new == -1) & ~bad
    # finished requests' pages go on the stack first, in order
    back = torch.where(gone, held, 0)
    back_at = back.cumsum(0) - back
    col = torch.arange(width, device=dev)
    r, c = torch.nonzero(gone[:, None] & (col < held[:, None]), as_tuple=True)
    free[s["count"] + back_at[r] + c] = table[r, c]
    total = s["count"][0] + back.sum()
    need = torch.where(bad | full | gone, 0, wanted - held)
    upto = need.cumsum(0)
    short = (need > 0) & (upto > total)
    status = torch.where(bad, 2, torch.where(full, 3, torch.where(short, 1, 0)))
    served = (status == 0) & ~gone
    take = torch.where(served, need, 0)
    r, c = torch.nonzero(served[:, None] & (col >= held[:, None]) & (col < wanted[:, None]), as_tuple=True)
    table[r, c] = free[total - 1 - (upto[r] - need[r]) - (c - held[r])]
    tok = torch.arange(s["tokens"], device=dev)
    used = tok < starts[-1]
    req = torch.searchsorted(starts, tok, right=True).clamp(max=new.numel()) - 1
    pos = seq[req] + tok - starts[req]
    ok = used & served[req]
    slots = torch.where(ok, table[req, torch.where(ok, pos // page, 0)].long() * page + pos % page, -1)
    seq_out = torch.where(gone, 0, torch.where(served, seq + n, seq))
    i32 = lambda v: v.to(torch.int32)  # noqa: E731
    return [table, free, slots, i32(torch.where(used, pos, 0)), i32(torch.where(used, req, -1)), i32(seq_out), i32(starts),
            i32(status), i32(total - take.sum()).reshape(1)]


def _values(codes, kind):
    return codes.float() if kind == "int8" else codes.view(torch.float8_e4m3fn).float()


def _codes(x, kind):
    return x.round().to(torch.int8) if kind == "int8" else x.to(torch.float8_e4m3fn).view(torch.int8)


def _block_scale(amax, kind):
    """The smallest power of two s with amax <= s * (127 or 448); 0 for a block of zeros."""
    m, e = torch.frexp(amax)
    e = e - 7 + (m > 127 / 128).int() if kind == "int8" else e - 9 + (m > 448 / 512).int()
    return torch.where(amax > 0, ((e.clamp(min=-126) + 127) << 23).view(torch.float32), 0.0)


def _plain_append(s):
    case = s["case"]
    page, kind = case["page"], case["kind"]
    block, off = s["slots"] // page, s["slots"] % page
    outs = []
    for codes, scales, new, out in ((s["k"], s["ks"], s["new_k"], s["out_k"]), (s["v"], s["vs"], s["new_v"], s["out_v"])):
        x = new.float()
        amax = torch.zeros_like(scales).index_reduce_(0, block, x.abs().amax(2), "amax")
        first = torch.full_like(scales[:, 0], page).index_reduce_(0, block, off.float(), "amin")
        want = _block_scale(amax, kind)
        now = torch.where(first[:, None] == 0, want, torch.maximum(scales, want))
        hit = torch.where(first < page)[0]
        old = torch.where(first[hit] > 0, 1.0, 0.0)[:, None] * scales[hit]
        grown = _values(codes[hit], kind) * torch.where(now[hit] > 0, old / now[hit], 0.0)[:, :, None, None]
        codes[hit] = _codes(grown, kind)
        scales[hit] = now[hit]
        sc = scales[block][:, :, None]
        codes[block, :, off] = _codes(torch.where(sc > 0, x / sc, 0.0), kind)
        rb, ro = s["read"] // page, s["read"] % page
        outs.append((_values(codes[rb, :, ro], kind) * scales[rb][:, :, None]).to(out.dtype))
    return outs


def _plain_attend(s):
    case = s["case"]
    page, hq, h, d = case["page"], case["q_heads"], case["heads"], case["dim"]
    n, width = s["seq"].numel(), s["widest"]
    pages = -(-s["longest"] // page)
    at = s["table"][:, :pages].long().clamp(min=0)
    wide = lambda codes, scales: (_values(codes[at], case["kind"]) * scales[at][..., None, None]).transpose(1, 2).reshape(  # noqa: E731
        n, h, pages * page, d)
    k, v = wide(s["k"], s["ks"]), wide(s["v"], s["vs"])
    tok = (s["start"][:-1, None] + torch.arange(width, device=at.device)).clamp(max=max(s["q"].shape[0] - 1, 0))
    q = s["q"].float()[tok.long()].reshape(n, width, h, hq // h, d).permute(0, 2, 1, 3, 4).reshape(n, h, width * (hq // h), d)
    z = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(d))
    pos = (s["seq"] - (s["start"][1:] - s["start"][:-1]))[:, None] + torch.arange(width, device=at.device)
    key = torch.arange(pages * page, device=at.device)
    see = (key <= pos[:, :, None]) & (key < s["seq"][:, None, None])
    if case["window"]:
        see &= key > pos[:, :, None] - case["window"]
    see = see[:, None, :, None].expand(n, 1, width, hq // h, key.numel()).reshape(n, 1, width * (hq // h), key.numel())
    z = z.masked_fill_(~see, -math.inf)
    m = z.amax(3, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    e = torch.exp(z - m)
    total = e.sum(3, keepdim=True)
    o = torch.matmul(e, v * see.any(2)[..., None]) / torch.where(total > 0, total, 1.0)
    lse = m + torch.log(total)
    back = lambda x: x.reshape(n, h, width, hq // h, -1).permute(0, 2, 1, 3, 4).reshape(n, width, hq, -1)[s["req"], s["step"]]  # noqa: E731
    return [back(o).to(s["out"].dtype), back(lse)[..., 0]]


def _plain_score(s):
    case, t = s["case"], s["t"]
    v, k = case["vocab"], case["top"]
    x = s["x"].float()
    z = x * case["scale"]
    m = z.amax(1, keepdim=True)
    empty = m == -math.inf
    e = torch.exp(z - torch.where(empty, 0.0, m))
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total)
    entropy = torch.where(empty, 0.0, log_total - torch.where(e > 0, e * (z - m), 0.0).sum(1, keepdim=True) / total)
    has = t >= 0
    at = t.clamp(min=0)[:, None]
    logp = torch.where(empty, -math.inf, z.gather(1, at) - m - log_total)[:, 0]
    xt, ids = x.gather(1, at), torch.arange(v, device=x.device)
    rank = ((x > xt) | ((x == xt) & (ids < at))).sum(1)
    # values in order as whole numbers, the lower index first among equals
    bits = (x + 0.0).view(torch.int32)
    key = (torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() << 32) | (v - 1 - ids)
    best = min(k, v)
    top_id = torch.full((x.shape[0], k), -1, dtype=torch.int32, device=x.device)
    top = torch.full((x.shape[0], k), -math.inf, device=x.device)
    if best:
        i = v - 1 - (torch.topk(key, best, 1).values & 0xFFFFFFFF)
        top_id[:, :best] = i.to(torch.int32)
        top[:, :best] = torch.where(empty, -math.inf, z.gather(1, i) - m - log_total)
    return [torch.where(has, logp, 0.0), entropy[:, 0], torch.where(has, rank, -1).to(torch.int32), top, top_id]


def run(state):
    op = state["case"]["op"]
    if own:
        return {"plan": _own_plan, "append": _own_append, "attend": _own_attend, "score": _own_score}[op](state)
    return {"plan": _plain_plan, "append": _plain_append, "attend": _plain_attend, "score": _plain_score}[op](state)


# ---------------------------------------------------------------- what a pass cannot do without

def _seen(case):
    """(keys read, (query token, key) pairs, query tokens) summed over the requests."""
    after, fresh = _lengths(case)
    keys = pairs = 0
    for x, f in zip(after, fresh):
        x = max(x, f)
        window = case["window"] or x + 1
        if f:
            keys += x - max(0, x - f + 1 - window)
        pairs += sum(min(x - f + 1 + i, window) for i in range(f))
    return keys, pairs, sum(fresh)


def work(case):
    if case["op"] == "plan":
        before, fresh = _lengths(case)
        page = case["page"]
        need = sum(_ceil(x + f, page) - _ceil(x, page) for x, f in zip(before, fresh))
        n = sum(fresh)
        return {"bytes": 20 * case["requests"] + 8 * need + 16 * n, "flops": 4 * n}
    if case["op"] == "append":
        before, fresh = _lengths(case)
        page, row = case["page"], 2 * case["heads"] * case["dim"]
        n = sum(fresh)
        read = sum(x % page + f for x, f in zip(before, fresh) if f)
        w = WIDTH[case["dtype"]]
        return {"bytes": row * (n * (w + 1) + read * (1 + w)) + 8 * (n + read), "flops": 2 * row * (n + read)}
    if case["op"] == "attend":
        keys, pairs, n = _seen(case)
        h, hq, d = case["heads"], case["q_heads"], case["dim"]
        pages = keys / case["page"]
        return {"bytes": 2 * h * (keys * d + 4 * pages) + 4 * pages + n * hq * (d * (WIDTH[case["dtype"]] + WIDTH[case["out"]]) + 4),
                "flops": 4 * hq * d * pairs}
    n, v = case["rows"], case["vocab"]
    return {"bytes": n * (v * WIDTH[case["dtype"]] + 20 + 8 * case["top"]), "flops": 6 * n * v}


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_plan(s, case):
    page = case["page"]
    seq, new, free = (s[x].cpu().tolist() for x in ("seq", "new", "free"))
    table = s["table"].cpu().numpy().copy()
    count, tokens = s["count"].item(), s["tokens"]
    width = table.shape[1]
    top = count
    for i, (x, f) in enumerate(zip(seq, new)):
        if f == -1 and x >= 0 and _ceil(x, page) <= width:
            for j in range(_ceil(x, page)):
                free[top] = int(table[i, j])
                top += 1
    stack_end = top
    slots, pos, req = [], [], []
    seq_out, starts, status, asked = [], [0], [], 0
    for i, (x, f) in enumerate(zip(seq, new)):
        f0 = max(f, 0)
        first = len(slots)
        end = starts[-1] + f0
        state = 2 if f < -1 or x < 0 or _ceil(x + f0, page) > width else 3 if end > tokens else 0
        if state == 0 and f >= 0:
            need = _ceil(x + f, page) - _ceil(x, page)
            asked += need
            if need and asked > stack_end:
                state = 1
            elif need:
                table[i, _ceil(x, page):_ceil(x + f, page)] = [free[stack_end - 1 - (asked - need) - j] for j in range(need)]
                top -= need
        good = state == 0 and f >= 0
        for p in range(x, x + f0):
            slots.append(int(table[i, p // page]) * page + p % page if good else -1)
            pos.append(p)
            req.append(i)
        assert len(slots) - first == f0
        seq_out.append(0 if state == 0 and f == -1 else x + f if good else x)
        starts.append(end)
        status.append(state)
    pad = tokens - len(slots)
    i32 = lambda v: np.asarray(v, np.int32)  # noqa: E731
    return [table, i32(free), np.asarray(slots + [-1] * pad, np.int64), i32(pos + [0] * pad), i32(req + [-1] * pad), i32(seq_out),
            i32(starts), i32(status), i32([top])]


def _decode64(codes, kind):
    """The numbers that codes stand for: two's complement, or sign, four exponent bits of bias 7 and three fraction bits."""
    c = codes.cpu().numpy()
    if kind == "int8":
        return c.astype(np.float64)
    u = c.view(np.uint8).astype(np.int64)
    e, f = (u >> 3) & 15, u & 7
    mag = np.where(e > 0, np.ldexp(8.0 + f, e - 10), np.ldexp(f.astype(np.float64), -9))
    return np.where(u >> 7, -mag, mag)


def _round64(x, kind):
    """To the nearest number that a code can hold, ties to even."""
    if kind == "int8":
        return np.rint(x)
    step = np.ldexp(1.0, np.maximum(np.frexp(x)[1] - 1, -6) - 3)
    return np.rint(x / step) * step


def _exact_append(s, case):
    page, kind = case["page"], case["kind"]
    limit = 127.0 if kind == "int8" else 448.0
    slots, read = s["slots"].cpu().numpy(), s["read"].cpu().numpy()
    outs = []
    for codes, scales, new in ((s["k"], s["ks"], s["new_k"]), (s["v"], s["vs"], s["new_v"])):
        value = _decode64(codes.contiguous(), kind)  # pages, heads, tokens, dims
        scale = scales.cpu().double().numpy()
        x = new.cpu().double().numpy()
        cuts = np.flatnonzero(np.diff(slots // page) != 0) + 1
        for run_ in np.split(np.arange(slots.size), cuts):
            if not run_.size:
                continue
            b, o = slots[run_[0]] // page, slots[run_] % page
            amax = np.abs(x[run_]).max((0, 2))
            want = np.zeros_like(amax)
            want[amax > 0] = np.exp2(np.maximum(np.ceil(np.log2(amax[amax > 0] / limit)), -126))
            want = np.where((amax > 0) & (want > 2.0 ** -126) & (amax <= limit * want / 2), want / 2, want)  # log2 rounds
            want = np.where(amax > limit * want, want * 2, want)
            now = want if o[0] == 0 else np.maximum(scale[b], want)
            safe = np.where(now > 0, now, 1.0)[:, None]
            for t in range(o[0]):
                value[b, :, t] = _round64(value[b, :, t] * scale[b][:, None] / safe, kind)
            for j, t in zip(run_, o):
                value[b, :, t] = _round64(x[j] / safe, kind)
            scale[b] = now
        outs.append(value[read // page, :, read % page] * scale[read // page][:, :, None])
    return outs


def _exact_attend(s, case):
    page, hq, h, d = case["page"], case["q_heads"], case["heads"], case["dim"]
    q = s["q"].double()
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
    table, start, seq = s["table"].long(), s["start"].tolist(), s["seq"].tolist()
    for i, length in enumerate(seq):
        fresh = start[i + 1] - start[i]
        if not fresh or not length:
            continue
        at = table[i, :_ceil(length, page)]
        k = _values(s["k"][at], case["kind"]).double() * s["ks"][at].double()[:, :, None, None]
        v = _values(s["v"][at], case["kind"]).double() * s["vs"][at].double()[:, :, None, None]
        k, v = (x.transpose(1, 2).reshape(-1, h, d)[:length] for x in (k, v))
        for j in range(fresh):
            p = length - fresh + j
            lo = max(0, p + 1 - case["window"]) if case["window"] else 0
            qj = q[start[i] + j].reshape(h, hq // h, d)
            z = torch.matmul(qj, k[lo:p + 1].permute(1, 2, 0)) / math.sqrt(d)
            out[start[i] + j] = torch.matmul(torch.softmax(z, 2), v[lo:p + 1].transpose(0, 1)).reshape(hq, d)
            lse[start[i] + j] = torch.logsumexp(z, 2).reshape(hq)
    return [out.cpu().numpy(), lse.cpu().numpy()]


def _exact_score(s, case):
    x, t, k = s["x"], s["t"].tolist(), case["top"]
    n, v = x.shape
    logp, entropy, rank = np.zeros(n), np.zeros(n), np.full(n, -1, np.int32)
    top, top_id = np.full((n, k), -np.inf), np.full((n, k), -1, np.int32)
    for i in range(n):
        z = x[i].double() * case["scale"]
        lp = z - torch.logsumexp(z, 0)
        if bool((z == -math.inf).all()):
            lp = z
        p = torch.exp(lp)
        entropy[i] = -(torch.where(p > 0, p * lp, 0.0)).sum().item()
        if t[i] >= 0:
            logp[i] = lp[t[i]].item()
            rank[i] = int((x[i] > x[i, t[i]]).sum()) + int((x[i, :t[i]] == x[i, t[i]]).sum())
        if k:
            b = min(k, v)
            ids = torch.sort(x[i].double(), descending=True, stable=True).indices[:b]
            top[i, :b], top_id[i, :b] = lp[ids].cpu().numpy(), ids.cpu().numpy()
    return [logp, entropy, rank, top, top_id]


def exact(case, seed):
    s = prepare(case, seed)
    return {"plan": _exact_plan, "append": _exact_append, "attend": _exact_attend, "score": _exact_score}[case["op"]](s, case)
