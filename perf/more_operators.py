"""The operators around positions and beams of a decode step, as cases that can be timed and compared.

Four groups, named by a case's "op":
  rotary   cos and sin of a step's positions, and queries and keys rotated by them
  write    new keys and values written to the 8-bit paged cache, the keys rotated on the way and the step's
           queries beside them, and the blocks they touch read back
  select   beam search's choice over beams and vocabulary from the logits of a step
  reorder  the pages of the chosen beams: shared where full, the last one copied for every further child

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
MOST_ROTARY = 8192 * 72 * 128 * 4   # bytes that a drawn case rotates, in and out
MOST_WRITE = 4096 * 32 * 128        # keys that a drawn case writes (half of them in 32 bits)
MOST_LOGITS = 64 * 8 * 128256 * 2   # bytes of logits
MOST_CODES = 900 << 20              # bytes of keys that a drawn reorder holds, all layers


# ---------------------------------------------------------------- cases

def listed():
    return [
        # a decode step of the Llama-3-8B shape: 16 tokens, query and key heads of the fused projection
        dict(name="rotary_step", op="rotary", tokens=16, heads=40, spare=8, dim=128, rot=128, layout="half", rule="none", factor=1.0,
             base=500000.0, dtype="f32", out="f32", most=8192),
        # a ragged prompt of a small model: part of the head, neighbours paired, stretched positions
        dict(name="rotary_part", op="rotary", tokens=333, heads=16, spare=4, dim=96, rot=24, layout="pairs", rule="ramp", factor=4.0,
             base=10000.0, dtype="f16", out="f16", most=32768),
        # a long prompt of the Llama-2-70B shape at positions up to 131072, frequencies scaled by wavelength
        dict(name="rotary_prompt", op="rotary", tokens=8192, heads=72, spare=8, dim=128, rot=128, layout="half", rule="bands", factor=8.0,
             base=500000.0, dtype="bf16", out="bf16", most=131072),
        # the cache write of a decode step, f32 as the products leave it, queries rotated beside it
        dict(name="write_step", op="write", requests=16, max_len=4096, new="one", max_new=1, q_heads=32, heads=8, dim=128, rot=128,
             layout="half", page=16, kind="int8", order="head", dtype="f32", out="f32", mix=3),
        # prompts of the Llama-2-7B shape, 4096 tokens in all
        dict(name="write_prompt", op="write", requests=4, max_len=100, new="full", max_new=1024, q_heads=32, heads=32, dim=128, rot=128,
             layout="half", page=64, kind="e4m3", order="head", dtype="bf16", out="bf16", mix=4),
        # ragged prompts of a small model, tokens before heads in a page, a quarter of the head rotated
        dict(name="write_ragged", op="write", requests=7, max_len=333, new="mixed", max_new=217, q_heads=12, heads=4, dim=96, rot=24,
             layout="pairs", page=32, kind="int8", order="token", dtype="f16", out="f16", mix=5),
        # one request's four beams over the Llama-2-7B vocabulary: latency
        dict(name="select_one", op="select", groups=1, beams=4, vocab=32000, top=4, dtype="f32", scale=1.0, first=False, weighted=False,
             masked=False, mix=6),
        # four requests of four beams, the widest product, over the Llama-3-8B head, some beams at their end
        dict(name="select_step", op="select", groups=4, beams=4, vocab=128256, top=8, dtype="f32", scale=1.0, first=False, weighted=True,
             masked=True, mix=7),
        # a large batch of beams
        dict(name="select_batch", op="select", groups=64, beams=8, vocab=128256, top=16, dtype="bf16", scale=1.25, first=False,
             weighted=True, masked=False, mix=8),
        # two layers of a small model, one request forked from its prompt
        dict(name="reorder_fork", op="reorder", groups=1, beams=5, max_len=77, heads=2, dim=64, page=16, layers=2, order="head", first=True,
             mix=9),
        # four requests of four beams, Llama-3-8B shape, all layers
        dict(name="reorder_step", op="reorder", groups=4, beams=4, max_len=600, heads=8, dim=128, page=16, layers=32, order="head",
             first=False, mix=10),
        # 32 requests of eight beams, larger pages
        dict(name="reorder_batch", op="reorder", groups=32, beams=8, max_len=2048, heads=8, dim=128, page=64, layers=8, order="token",
             first=False, mix=11),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def _parts(rng, dim):
    """Rotated dims of a head: all of them, a half, a quarter, or some even number."""
    return rng.choice([dim, dim, dim // 2, dim // 4, 2 * rng.randint(1, dim // 2)])


def draw(rng):
    op = rng.choice(["rotary", "rotary", "write", "write", "select", "select", "reorder"])
    mix = rng.randrange(1 << 20)
    if op == "rotary":
        q, h, d = rng.choice(HEADS)
        heads, dt, out = rng.choice([q, h, q + h]), rng.choice(list(DTYPES)), rng.choice(list(DTYPES))
        most = MOST_ROTARY // (heads * d * (WIDTH[dt] + WIDTH[out]))
        return dict(op=op, tokens=_log_int(rng, 1, min(16384, most)), heads=heads, spare=rng.choice([0, h]), dim=d,
                    rot=_parts(rng, d), layout=rng.choice(["half", "pairs"]), rule=rng.choice(["none", "linear", "base", "bands", "ramp"]),
                    factor=rng.choice([2.0, 4.0, 8.0]), base=rng.choice([10000.0, 500000.0]), dtype=dt, out=out,
                    most=_log_int(rng, 16, 1 << 20))
    if op == "write":
        q, h, d = rng.choice(HEADS)
        n, dt, out = _log_int(rng, 1, 64), rng.choice(list(DTYPES)), rng.choice(list(DTYPES))
        most = max(1, MOST_WRITE // (n * max(h, q // 2) * d * (2 if "f32" in (dt, out) else 1)))
        return dict(op=op, requests=n, max_len=_log_int(rng, 1, 4096), new=rng.choice(["one", "mixed", "full"]),
                    max_new=_log_int(rng, 1, min(1024, most)), q_heads=q, heads=h, dim=d, rot=_parts(rng, d),
                    layout=rng.choice(["half", "pairs"]), page=rng.choice([16, 32, 64, 128]), kind=rng.choice(["int8", "e4m3"]),
                    order=rng.choice(["head", "token"]), dtype=dt, out=out, mix=mix)
    if op == "select":
        vocab = rng.choice([rng.choice(VOCABS), _log_int(rng, 40, 128256)])
        beams, dt = _log_int(rng, 1, 32), rng.choice(list(DTYPES))
        return dict(op=op, groups=_log_int(rng, 1, max(1, min(64, MOST_LOGITS // (beams * vocab * WIDTH[dt])))), beams=beams, vocab=vocab,
                    top=rng.choice([1, beams, min(2 * beams, 32), 32]), dtype=dt, scale=rng.choice([1.0, 0.7, 1.25]),
                    first=rng.random() < 0.2, weighted=rng.random() < 0.5, masked=rng.random() < 0.4, mix=mix)
    _, h, d = rng.choice(HEADS)
    layers, beams, page = rng.choice([1, 2, 8, 32]), _log_int(rng, 1, 32), rng.choice([16, 32, 64, 128])
    groups = _log_int(rng, 1, max(1, min(32, 512 // beams)))
    pages = MOST_CODES // (layers * h * d * page)  # of all rows: a shared part and up to four of each beam
    most = max(1, min(8192, (pages // (groups + 1) - 5 * beams) * page))
    while most < 2 * page and groups > 1:
        groups //= 2
        most = max(1, min(8192, (pages // (groups + 1) - 5 * beams) * page))
    return dict(op=op, groups=groups, beams=beams, max_len=_log_int(rng, 1, most), heads=h, dim=d, page=page, layers=layers,
                order=rng.choice(["head", "token"]), first=rng.random() < 0.2, mix=mix)


# ---------------------------------------------------------------- inputs

def _ceil(a, b):
    return -(-a // b)


def _frequencies(case):
    """Radians per position of each pair (float64) and the factor of cos and sin, by the published rules."""
    r, base, s = case["rot"], case["base"], case["factor"]
    i = np.arange(r // 2, dtype=np.float64)
    if case["rule"] == "base" and r > 2:
        base = base * s ** (r / (r - 2))
    w = base ** (-2.0 * i / r)
    if case["rule"] == "linear":
        return w / s, 1.0
    if case["rule"] == "bands":  # long waves stretched, short ones kept, between them a mixture
        turns = 8192.0 * w / (2 * math.pi)
        mix = np.clip((turns - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        return w * (mix + (1 - mix) / s), 1.0
    if case["rule"] == "ramp":  # by the dimension, between those that turn 32 times and once over the trained length
        at = lambda turns: r * math.log(4096.0 / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), r - 1)
        keep = 1 - np.clip((i - lo) / max(hi - lo, 0.001), 0.0, 1.0)
        return w * (keep + (1 - keep) / s), 0.1 * math.log(s) + 1.0
    return w, 1.0


def _pages(total, seed):
    return np.random.RandomState(seed % (1 << 31)).permutation(total).astype(np.int32)


def _prepare_rotary(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    n, heads, d = case["tokens"], case["heads"], case["dim"]
    # the heads to rotate are the first of a fused projection's; a prompt's tokens follow one another, a step's do not
    x = torch.randn((n, heads + case["spare"], d), generator=gen, device="cuda").to(DTYPES[case["dtype"]])[:, :heads]
    rng = random.Random(seed)
    if n > 64:
        pos = torch.arange(n, device="cuda") + rng.randint(0, max(0, case["most"] - n))
    else:
        pos = torch.tensor([rng.randint(0, case["most"]) for _ in range(n)], device="cuda")
    w, m = _frequencies(case)
    s = dict(case=case, x=x, pos=pos.to(torch.int32), w=torch.from_numpy(w).cuda(), m=m,
             cs=torch.empty((n, case["rot"] // 2, 2), device="cuda"),
             out=torch.empty((n, heads, d), dtype=DTYPES[case["out"]], device="cuda"))
    if own:
        from paper_2609_38477_gb300 import serving

        s["rotary"] = serving.Rotary(w, layout=case["layout"], scale=m)
    return s


def _lengths(case):
    """Lengths before the step and new tokens of every request, from the case alone: one as long as the longest, in
    a batch of four or more an empty one and one of a single token."""
    rng = random.Random(case["mix"])
    n, most, new = case["requests"], case["max_len"], case["max_new"]
    before = [_log_int(rng, 1, most) for _ in range(n)]
    before[0] = most
    if n >= 4:
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


def _cache(case, gen, pages):
    """A cache that already holds tokens: random codes under power-of-two scales, in either page order."""
    p, h, d = case["page"], case["heads"], case["dim"]
    shape = (pages, h, p, d) if case["order"] == "head" else (pages, p, h, d)
    out = []
    for _ in range(2):
        x = torch.randn(shape, generator=gen, device="cuda")
        codes = (x * 32).round_().clamp_(-127, 127).to(torch.int8) if case["kind"] == "int8" else (
            (x * 96).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.int8))
        e = torch.randint(-6, -3, (pages, h), generator=gen, device="cuda")
        scale = torch.pow(2.0, e.float() - (0 if case["kind"] == "int8" else 2))
        out.append((codes if case["order"] == "head" else codes.transpose(1, 2), scale))
    return out


def _prepare_write(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    before, fresh = _lengths(case)
    page, h, hq, d, r = case["page"], case["heads"], case["q_heads"], case["dim"], case["rot"]
    held = [_ceil(x + f, page) for x, f in zip(before, fresh)]
    ids = _pages(max(1, sum(held)), seed)
    at, slots, touched, pos = 0, [], [], []
    for x, f, m in zip(before, fresh, held):
        own_pages = ids[at:at + m].astype(np.int64)
        at += m
        p = np.arange(x, x + f)
        slots.append(own_pages[p // page] * page + p % page)
        pos.append(p)
        if f:  # what the blocks hold that this step writes to
            p = np.arange(x // page * page, x + f)
            touched.append(own_pages[p // page] * page + p % page)
    slots, touched, pos = (np.concatenate(v) for v in (slots, touched, pos))
    (k, ks), (v, vs) = _cache(case, gen, ids.size)
    n, dt = slots.size, DTYPES[case["dtype"]]
    # tokens differ in size: some outgrow the scale of the block they join
    size = torch.exp(0.8 * torch.randn((2, n, 1, 1), generator=gen, device="cuda"))
    kv = (size * torch.randn((2, n, h, d), generator=gen, device="cuda")).to(dt)
    q = torch.randn((n, hq, d), generator=gen, device="cuda").to(dt)
    # the step's cos and sin, which all its layers share
    w = 10000.0 ** (-2.0 * torch.arange(r // 2, device="cuda", dtype=torch.float64) / r)
    angle = torch.from_numpy(pos).cuda().double()[:, None] * w
    s = dict(case=case, k=k, v=v, ks=ks, vs=vs, new_k=kv[0], new_v=kv[1], q=q, slots=torch.from_numpy(slots).cuda(),
             read=torch.from_numpy(touched).cuda(), cs=torch.stack([torch.cos(angle), torch.sin(angle)], 2).float().contiguous())
    s["q_out"] = torch.empty((n, hq, d), dtype=DTYPES[case["out"]], device="cuda")
    s["out_k"] = torch.empty((touched.size, h, d), dtype=torch.bfloat16, device="cuda")
    s["out_v"] = torch.empty_like(s["out_k"])
    if own:
        from paper_2609_38477_gb300 import serving

        s["cache"] = serving.KVCache(k, v, ks, vs, case["kind"])
        s["rotary"] = serving.Rotary(w.cpu().numpy(), layout=case["layout"])
    return s


def _prepare_select(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    g, b, v = case["groups"], case["beams"], case["vocab"]
    x = torch.empty((g * b, v), dtype=DTYPES[case["dtype"]], device="cuda")
    for part in x.split(max(1, (1 << 27) // v)):
        z = 2.5 * torch.randn(part.shape, generator=gen, device="cuda")
        if case["masked"]:  # tokens that a grammar or a ban list rules out
            z.masked_fill_(torch.rand(part.shape, generator=gen, device="cuda") < 0.3, -math.inf)
        part.copy_(z)
    # sums of log probabilities, close to one another as those of beams are
    scores = -20.0 + 2.0 * torch.randn((g, b), generator=gen, device="cuda")
    length = torch.randint(4, 40, (g, b), generator=gen, device="cuda").float()
    done = (torch.rand((g, b), generator=gen, device="cuda") < 0.2).to(torch.uint8)
    if case["first"]:  # after the prompt only the first beam says anything
        scores[:, 1:] = -math.inf
        scores[:, 0] = 0.0
        done.zero_()
    n = case["top"]
    s = dict(case=case, x=x, scores=scores, done=done, weights=length ** -0.6 if case["weighted"] else None, end=min(2, v - 1),
             score=torch.empty((g, n), device="cuda"), beam=torch.empty((g, n), dtype=torch.int32, device="cuda"),
             token=torch.empty((g, n), dtype=torch.int32, device="cuda"))
    if own:
        from paper_2609_38477_gb300 import serving

        s["work"] = serving.beam_workspace(g, b, v)
    return s


def _beams(case):
    """Length, shared pages and parents of every request's beams, from the case alone."""
    rng = random.Random(case["mix"])
    b, page, out = case["beams"], case["page"], []
    for i in range(case["groups"]):
        length = case["max_len"] if i == 0 else _log_int(rng, 1, case["max_len"])
        if case["first"]:  # the prompt's row is forked
            out.append((length, 0, [0] * b))
            continue
        shared = max(0, length // page - rng.randint(0, 3))
        if i % 7 == 5:  # a request that ends
            parents = [-1] * b
        elif i % 7 == 3:  # nothing changes
            parents = list(range(b))
        else:  # few beams have most of the children, as the better ones do
            parents = [min(b - 1, int(rng.expovariate(1.0) * b / 3)) for _ in range(b)]
        out.append((length, shared, parents))
    return out


def _prepare_reorder(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    g, b, page, h, d, layers = (case[x] for x in ("groups", "beams", "page", "heads", "dim", "layers"))
    groups = _beams(case)
    width = _ceil(case["max_len"], page) + 1
    used = sum(_ceil(x, page) if case["first"] else sh + b * (_ceil(x, page) - sh) for x, sh, _ in groups)
    spare = g * b
    pages = used + spare
    ids = _pages(pages, seed)
    table, lens, at = np.full((g * b, width), -1, np.int32), np.zeros(g * b, np.int32), 0
    for i, (x, sh, _) in enumerate(groups):
        rows = [i * b] if case["first"] else range(i * b, i * b + b)
        table[list(rows), :sh] = ids[at:at + sh]
        at += sh
        for r in rows:
            m = _ceil(x, page) - sh
            table[r, sh:sh + m] = ids[at:at + m]
            at += m
            lens[r] = x
    free = np.full(pages, -1, np.int32)
    free[:spare] = ids[used:]
    shape = (layers, pages, h, page, d) if case["order"] == "head" else (layers, pages, page, h, d)
    k, v = (torch.randint(-127, 128, shape, generator=gen, device="cuda", dtype=torch.int8) for _ in range(2))
    ks, vs = (torch.rand((layers, pages, h), generator=gen, device="cuda") for _ in range(2))
    cu = lambda a: torch.from_numpy(np.asarray(a, np.int32)).cuda()  # noqa: E731
    s = dict(case=case, k=k, v=v, ks=ks, vs=vs, table=cu(table), lens=cu(lens), free=cu(free), count=cu([spare]),
             parents=cu([p for _, _, p in groups]), new_table=torch.full((g * b, width), -1, dtype=torch.int32, device="cuda"))
    if own:
        from paper_2609_38477_gb300 import serving

        view = (lambda x: x) if case["order"] == "head" else (lambda x: x.transpose(1, 2))
        s["pages"] = serving.BeamPages([serving.KVCache(view(k[i]), view(v[i]), ks[i], vs[i]) for i in range(layers)], g, b)
    return s


def prepare(case, seed):
    return {"rotary": _prepare_rotary, "write": _prepare_write, "select": _prepare_select, "reorder": _prepare_reorder}[case["op"]](case, seed)


# ---------------------------------------------------------------- the package's calls

def _own_rotary(s):
    s["rotary"].angles(s["pos"], s["cs"])
    s["rotary"].rotate(s["x"], s["cs"], s["out"])
    return [s["cs"], s["out"]]


def _own_write(s):
    s["cache"].append_rotary(s["new_k"], s["new_v"], s["slots"], s["rotary"], s["cs"], q=s["q"], q_out=s["q_out"])
    s["cache"].gather(s["read"], s["out_k"], s["out_v"])
    return [s["q_out"], s["out_k"], s["out_v"]]


def _own_select(s):
    from paper_2609_38477_gb300 import serving

    serving.beam_select(s["x"], s["scores"], s["score"], s["beam"], s["token"], s["work"], scale=s["case"]["scale"], done=s["done"],
                        end_token=s["end"], weights=s["weights"])
    return [s["score"], s["beam"], s["token"]]


def _own_reorder(s):
    p = s["pages"]
    p.reorder(s["parents"], s["lens"], s["table"], s["free"], s["count"], out=s["new_table"])
    return [s["new_table"], p.seq_lens, p.status, s["free"], p.free_count, s["k"], s["v"], s["ks"], s["vs"]]


# ---------------------------------------------------------------- the plain forms

def _turn(x, cs, case):
    """x (tokens, heads, dim) in 32 bits, its first `rot` dims rotated."""
    r, c, s = case["rot"], cs[:, None, :, 0], cs[:, None, :, 1]
    if case["layout"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([a * c - b * s, b * c + a * s], 2)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * c - b * s, b * c + a * s], 3).flatten(2)
    return torch.cat([y, x[..., r:]], 2)


def _plain_rotary(s):
    angle = s["pos"].double()[:, None] * s["w"]  # in 64 bits: far positions
    cs = (torch.stack([torch.cos(angle), torch.sin(angle)], 2) * s["m"]).float()
    return [cs, _turn(s["x"].float(), cs, s["case"]).to(s["out"].dtype)]


def _values(codes, kind):
    return codes.float() if kind == "int8" else codes.view(torch.float8_e4m3fn).float()


def _codes(x, kind):
    return x.round().to(torch.int8) if kind == "int8" else x.to(torch.float8_e4m3fn).view(torch.int8)


def _block_scale(amax, kind):
    """The smallest power of two s with amax <= s * (127 or 448); 0 for a block of zeros."""
    m, e = torch.frexp(amax)
    e = e - 7 + (m > 127 / 128).int() if kind == "int8" else e - 9 + (m > 448 / 512).int()
    return torch.where(amax > 0, ((e.clamp(min=-126) + 127) << 23).view(torch.float32), 0.0)


def _put(s, codes, scales, x):
    """x (tokens, heads, dim) at the step's slots, and what the touched blocks hold afterwards."""
    page, kind = s["case"]["page"], s["case"]["kind"]
    block, off = s["slots"] // page, s["slots"] % page
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
    return (_values(codes[rb, :, ro], kind) * scales[rb][:, :, None]).to(torch.bfloat16)


def _plain_write(s):
    q = _turn(s["q"].float(), s["cs"], s["case"]).to(s["q_out"].dtype)
    k = _put(s, s["k"], s["ks"], _turn(s["new_k"].float(), s["cs"], s["case"]))
    return [q, k, _put(s, s["v"], s["vs"], s["new_v"].float())]


def _plain_select(s):
    case = s["case"]
    g, b, v, n = (case[x] for x in ("groups", "beams", "vocab", "top"))
    done, scores = s["done"].bool(), s["scores"].double()
    z = s["x"].double().reshape(g, b, v) * case["scale"]  # in 64 bits: candidates of different beams lie close together
    m = z.amax(2, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    total = scores[..., None] + (z - m) - torch.log(torch.exp(z - m).sum(2, keepdim=True))
    none = (scores == -math.inf)[..., None] | (z == -math.inf)
    at = torch.arange(v, device=z.device)
    total = torch.where(done[..., None], torch.where(at == s["end"], scores[..., None], -math.inf), torch.where(none, -math.inf, total))
    key = (total if s["weights"] is None else total * s["weights"].double()[..., None]).reshape(g, b * v)
    # the n best, equal ones by their place: all above the n-th best, and as many of its equals as are left, the first ones
    most = min(n, b * v)
    border = torch.topk(key, most, 1).values[:, -1:]
    above, equal = key > border, key == border
    room = most - above.sum(1, keepdim=True)
    take = above | (equal & (equal.cumsum(1) <= room))
    place = torch.nonzero(take)[:, 1].reshape(g, most)
    order = torch.sort(key.gather(1, place), dim=1, descending=True, stable=True)
    place = place.gather(1, order.indices)
    best = total.reshape(g, b * v).gather(1, place)
    real = best > -math.inf
    pad = lambda x, by, dt: torch.nn.functional.pad(x.to(dt), (0, n - most), value=by)  # noqa: E731
    return [pad(best, -math.inf, torch.float32), pad(torch.where(real, place // v, -1), -1, torch.int32),
            pad(torch.where(real, place % v, -1), -1, torch.int32)]


def _plain_reorder(s):
    case = s["case"]
    g, b, page = case["groups"], case["beams"], case["page"]
    table, free, lens, parents = s["table"].reshape(g, b, -1), s["free"], s["lens"].reshape(g, b).long(), s["parents"].long()
    width, dev = table.shape[2], table.device
    lives = parents >= 0
    source = parents.clamp(min=0)
    new_len = torch.where(lives, lens.gather(1, source), 0)
    held, new_held = (lens + page - 1) // page, (new_len + page - 1) // page
    col, row = torch.arange(width, device=dev), torch.arange(b, device=dev)
    has, keeps = col < held[..., None], col < new_held[..., None]
    moved = table.gather(1, source[..., None].expand(g, b, width))
    # pages that no beam keeps, each once, column by column
    same = lambda x, y, ok: (x[:, :, None] == y[:, None]) & ok[:, None]  # noqa: E731
    kept = same(table, moved, keeps).any(2)
    before = (same(table, table, has) & (row[:, None] > row)[None, :, :, None]).any(2)
    gi, ci, ri = torch.nonzero((has & ~kept & ~before).transpose(1, 2), as_tuple=True)
    back = table[gi, ri, ci]
    free[s["count"] + torch.arange(back.numel(), device=dev)] = back
    total = s["count"][0].long() + back.numel()
    # further children of a beam whose last page is partly filled get a copy of it
    sibling = ((parents[:, :, None] == parents[:, None]) & (row[:, None] > row)).any(2)
    copy = lives & sibling & (new_len % page > 0)
    nth = copy.reshape(-1).cumsum(0).reshape(g, b) - 1
    ok = copy & (nth < total)
    dst = free[torch.where(ok, total - 1 - nth, 0)]
    last = torch.where(new_len > 0, (new_len - 1) // page, 0)
    src = moved.gather(2, last[..., None])[..., 0]
    moved = torch.where(ok[..., None] & (col == last[..., None]), dst[..., None], moved)
    short = copy & ~ok
    new_len = torch.where(short, 0, new_len)
    out = torch.where(keeps & ~short[..., None], moved, s["new_table"].reshape(g, b, width))
    s["new_table"].copy_(out.reshape(g * b, width))
    a, z, used = src[ok].long(), dst[ok].long(), (new_len % page)[ok]
    tok = torch.arange(page, device=dev)
    for codes in (s["k"], s["v"]):
        x = codes if case["order"] == "head" else codes.transpose(2, 3)
        x[:, z] = torch.where((tok < used[:, None])[None, :, None, :, None], x[:, a], x[:, z])
    for scales in (s["ks"], s["vs"]):
        scales[:, z] = scales[:, a]
    i32 = lambda x: x.reshape(-1).to(torch.int32)  # noqa: E731
    return [s["new_table"], i32(new_len), i32(short), free, i32(total - ok.sum()), s["k"], s["v"], s["ks"], s["vs"]]


def run(state):
    op = state["case"]["op"]
    if own:
        return {"rotary": _own_rotary, "write": _own_write, "select": _own_select, "reorder": _own_reorder}[op](state)
    return {"rotary": _plain_rotary, "write": _plain_write, "select": _plain_select, "reorder": _plain_reorder}[op](state)


# ---------------------------------------------------------------- what a pass cannot do without

def _copies(case):
    """(pages held before, pages held after, copied tokens) over all rows."""
    page, b = case["page"], case["beams"]
    old = new = tokens = 0
    for length, _, parents in _beams(case):
        old += _ceil(length, page) * (1 if case["first"] else b)
        new += _ceil(length, page) * sum(p >= 0 for p in parents)
        tokens += length % page * (sum(p >= 0 for p in parents) - len({p for p in parents if p >= 0}))
    return old, new, tokens


def work(case):
    if case["op"] == "rotary":
        n, r = case["tokens"], case["rot"]
        x = n * case["heads"] * case["dim"]
        return {"bytes": x * (WIDTH[case["dtype"]] + WIDTH[case["out"]]) + n * (4 + 4 * r), "flops": 3 * n * case["heads"] * r + 20 * n * r}
    if case["op"] == "write":
        before, fresh = _lengths(case)
        page, row, q, r = case["page"], 2 * case["heads"] * case["dim"], case["q_heads"] * case["dim"], case["rot"]
        n = sum(fresh)
        read = sum(x % page + f for x, f in zip(before, fresh) if f)
        w = WIDTH[case["dtype"]]
        return {"bytes": row * (n * (w + 1) + read * 3) + n * q * (w + WIDTH[case["out"]]) + n * (8 + 4 * r) + 8 * read,
                "flops": 2 * row * (n + read) + 3 * n * r * (case["heads"] + case["q_heads"])}
    if case["op"] == "select":
        rows, v = case["groups"] * case["beams"], case["vocab"]
        live = case["groups"] if case["first"] else rows * 0.8
        return {"bytes": live * v * WIDTH[case["dtype"]] + 9 * rows + 12 * case["groups"] * case["top"], "flops": 4 * live * v}
    old, new, tokens = _copies(case)
    row = 2 * case["layers"] * case["heads"] * case["dim"]
    return {"bytes": 4 * (old + new) + 20 * case["groups"] * case["beams"] + 2 * row * tokens, "flops": old + new}


# ---------------------------------------------------------------- the definitions in 64 bits

def _rotated64(x, cs, case):
    """x and cs as float64 arrays on the GPU; pair by pair through complex numbers."""
    r = case["rot"]
    z = torch.complex(cs[:, None, :, 0].contiguous(), cs[:, None, :, 1].contiguous())
    y = x.clone()
    even = torch.arange(r // 2, device=x.device)
    a, b = (even, even + r // 2) if case["layout"] == "half" else (2 * even, 2 * even + 1)
    turned = torch.complex(x[..., a], x[..., b]) * z
    y[..., a], y[..., b] = turned.real, turned.imag
    return y


def _exact_rotary(s, case):
    angle = s["pos"].cpu().numpy().astype(np.float64)[:, None] * s["w"].cpu().numpy()
    cs = s["m"] * np.stack([np.cos(angle), np.sin(angle)], 2)
    out = torch.cat([_rotated64(x.double(), c, case).cpu() for x, c in zip(s["x"].split(512), torch.from_numpy(cs).cuda().split(512))])
    return [cs, out.numpy()]


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


def _exact_write(s, case):
    page, kind = case["page"], case["kind"]
    limit = 127.0 if kind == "int8" else 448.0
    slots, read = s["slots"].cpu().numpy(), s["read"].cpu().numpy()
    cs = s["cs"].double()
    outs = [_rotated64(s["q"].double(), cs, case).cpu().numpy()]
    for codes, scales, new in ((s["k"], s["ks"], _rotated64(s["new_k"].double(), cs, case)), (s["v"], s["vs"], s["new_v"].double())):
        value = _decode64(codes.contiguous(), kind)  # pages, heads, tokens, dims
        scale, x = scales.cpu().double().numpy(), new.cpu().numpy()
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
            value[b, :, :o[0]] = _round64(value[b, :, :o[0]] * (scale[b][:, None] / safe)[:, None], kind)
            value[b, :, o] = _round64(x[run_] / safe, kind)
            scale[b] = now
        outs.append(value[read // page, :, read % page] * scale[read // page][:, :, None])
    return outs


def _exact_select(s, case):
    g, b, v, n = (case[x] for x in ("groups", "beams", "vocab", "top"))
    score, beam, token = np.full((g, n), -np.inf), np.full((g, n), -1, np.int32), np.full((g, n), -1, np.int32)
    scores, done = s["scores"].double().cpu().numpy(), s["done"].cpu().numpy()
    weights = np.ones((g, b)) if s["weights"] is None else s["weights"].double().cpu().numpy()
    for i in range(g):
        found = []  # (-weighted total, beam, token, total)
        for j in range(b):
            if scores[i, j] == -np.inf:
                continue
            if done[i, j]:
                found.append((-weights[i, j] * scores[i, j], j, s["end"], scores[i, j]))
                continue
            z = s["x"][i * b + j].double() * case["scale"]
            lp = torch.log_softmax(z, 0)
            ids = torch.sort(z, descending=True, stable=True).indices[:n].cpu().numpy()
            for t, p in zip(ids, lp.cpu().numpy()[ids]):
                if p > -np.inf:
                    found.append((-weights[i, j] * (scores[i, j] + p), j, int(t), scores[i, j] + p))
        for m, (_, j, t, total) in enumerate(sorted(found)[:n]):
            score[i, m], beam[i, m], token[i, m] = total, j, t
    return [score, beam, token]


def _exact_reorder(s, case):
    g, b, page = case["groups"], case["beams"], case["page"]
    table, lens, parents, free = (s[x].cpu().numpy() for x in ("table", "lens", "parents", "free"))
    out, free, new_len = s["new_table"].cpu().numpy().copy(), free.copy(), np.zeros(g * b, np.int32)
    top, wants = int(s["count"]), []
    for i in range(g):
        rows = range(i * b, i * b + b)
        kept = set()
        for r, p in zip(rows, parents[i]):
            if p >= 0:
                new_len[r] = lens[i * b + p]
                m = _ceil(int(new_len[r]), page)
                out[r, :m] = table[i * b + p, :m]
                kept |= set(out[r, :m].tolist())
                if new_len[r] % page and p in parents[i, :r - i * b]:
                    wants.append(r)
        for c in range(table.shape[1]):
            for r in rows:
                page_id = int(table[r, c])
                if c < _ceil(int(lens[r]), page) and page_id not in kept:
                    kept.add(page_id)
                    free[top] = page_id
                    top += 1
    state = np.zeros(g * b, np.int32)
    k, v, ks, vs = (s[x].clone() for x in ("k", "v", "ks", "vs"))
    for nth, r in enumerate(wants):
        c, used = int(new_len[r]) // page, int(new_len[r]) % page
        if nth >= top:
            raise ValueError("the cases have pages enough")
        src, dst = int(out[r, c]), int(free[top - 1 - nth])
        out[r, c] = dst
        for x in (k, v):
            if case["order"] == "head":
                x[:, dst, :, :used] = x[:, src, :, :used]
            else:
                x[:, dst, :used] = x[:, src, :used]
        for x in (ks, vs):
            x[:, dst] = x[:, src]
    return [out, new_len, state, free, np.asarray([top - len(wants)], np.int32), k, v, ks, vs]


def exact(case, seed):
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "write": _exact_write, "select": _exact_select, "reorder": _exact_reorder}[case["op"]](s, case)
