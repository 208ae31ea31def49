"""A decode loop over compressed layers: page bookkeeping, rotary positions, the
8-bit cache, its attention, token log probabilities and beam search around the
fused products.

Decoder.step takes the next tokens of a batch of requests (single tokens, or
pieces of prompts; at most 16 in all, the widest product), and everything after
the token ids stays on the device; Decoder.beam_search follows several
hypotheses of each prompt.  RMSNorm, SiLU and the residual sums are plain torch
operations.

    python -m paper_2609_38477_gb300.generate

compresses the small synthetic checkpoint (2 layers, 4 query and 2 key-value
heads) by the seed search, continues three prompts of different lengths, and
searches the likeliest continuations of one of them.
"""
from __future__ import annotations

import math

import torch

from . import seedq as Q
from . import serving

MAX_COLUMNS = 16  # of a product


def compress(weight, rung=(12, 3), max_batch: int = MAX_COLUMNS) -> Q.Layer:
    """A bound Layer that holds weight (rows x cols, float32 on the device) at
    one rung of the seed search, without outlier columns."""
    rows, cols = weight.shape
    layer = Q.Layer(rows, cols, [1.0] * cols, None, [rung], [], -1, 0.0, 0, max_batch=max_batch)
    nb = rows * (cols // 8)
    seed = torch.empty(nb, dtype=torch.int32, device="cuda")
    e, t = (torch.empty(n, dtype=torch.int8, device="cuda") for n in (nb, 6 * nb))
    layer.encode(weight.contiguous(), seed, e, t)
    bits = layer.stream_bits
    nbytes = Q.stream_bytes_required(bits)
    buf = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    layer.pack_stream(seed, e, t, buf, nbytes)
    layer.bind_stream(buf, bits, nbytes)
    return layer


def rms_norm(x, gain):
    return (x * torch.rsqrt((x * x).mean(1, keepdim=True) + 1e-5) * gain).bfloat16()


def rotate(x, angles):
    """Rotary positions in plain torch: x (tokens, heads, dim), angles (tokens, dim / 2)."""
    c, s = torch.cos(angles)[:, None], torch.sin(angles)[:, None]
    a, b = x.chunk(2, 2)
    return torch.cat([a * c - b * s, b * c + a * s], 2)


class Decoder:
    """A Llama-shaped decoder over compressed layers.

    spec: dimensions (n_layers, d_model, n_heads, n_kv_heads, head_dim, d_ff,
    vocab).  blocks: per layer a dict of bound Layers q, k, v, o, gate, up, down
    and float32 gains attn_norm, mlp_norm.  embedding: (vocab, d_model)."""

    def __init__(self, spec, blocks, final_norm, head, embedding, max_requests: int, n_pages: int, page_size: int = 16,
                 max_pages: int = 64, kind: str = "int8"):
        self.spec, self.blocks, self.final_norm, self.head, self.embedding = spec, blocks, final_norm, head, embedding
        self.page_size = page_size
        self.caches = [serving.KVCache.empty(n_pages, spec.n_kv_heads, spec.head_dim, page_size, kind) for _ in blocks]
        self.work = self.caches[0].attend_workspace(spec.n_heads, MAX_COLUMNS)
        # one set of pages for all layers: page p of every layer's cache holds the same tokens
        self.plan = serving.BatchPlan(max_requests, MAX_COLUMNS)
        self.table = torch.full((max_requests, max_pages), -1, dtype=torch.int32, device="cuda")
        self.free = torch.arange(n_pages, dtype=torch.int32, device="cuda")
        self.free_count = torch.full((1,), n_pages, dtype=torch.int32, device="cuda")
        self.seq_lens = torch.zeros(max_requests, dtype=torch.int32, device="cuda")
        freqs, scale = serving.rotary_frequencies(spec.head_dim)
        self.freqs = torch.tensor(freqs, device="cuda")
        self.rotary = serving.Rotary(freqs, scale=scale)
        self.score_work = serving.score_workspace(MAX_COLUMNS, spec.vocab)

    def _products(self, x, names, block):
        """x (tokens, cols) bfloat16 times several layers in one launch."""
        layers = [block[n] for n in names]
        out = [torch.empty((x.shape[0], l.rows), dtype=torch.float32, device="cuda") for l in layers]
        Q.gemm_multi(layers, [x] * len(layers), x.shape[0], out)
        return out

    def _advance(self):
        self.seq_lens[:self.plan.n_requests].copy_(self.plan.seq_lens)
        self.free_count.copy_(self.plan.free_count)

    def step(self, tokens, n_new):
        """The next tokens (int64, one request's after another's) of every
        request, n_new of each (int32; -1 ends a request); of fewer requests
        than the decoder was made for, the others wait.  Returns the logits
        of every token, none where requests only end; plan and seq_lens describe
        the step.  Tokens of a request that the plan could not serve (plan.status)
        have logits of NaN, and the request is as it was before."""
        s, n = self.spec, tokens.shape[0]
        p = self.plan
        p.build(self.seq_lens, n_new, self.table, self.free, self.free_count, self.page_size)
        if n == 0:  # requests only end or wait
            self._advance()
            return torch.empty((0, s.vocab), device="cuda")
        # tokens without a slot have no keys to attend to: NaN, which stays in its row
        x = self.embedding[tokens].float().masked_fill(p.slots[:n, None] < 0, float("nan"))
        cos_sin = torch.empty((n, self.rotary.half, 2), device="cuda")
        self.rotary.angles(p.positions, cos_sin)
        for block, cache in zip(self.blocks, self.caches):
            h = rms_norm(x, block["attn_norm"])
            q, k, v = self._products(h, ("q", "k", "v"), block)
            q = q.view(n, s.n_heads, s.head_dim)
            k, v = (y.view(n, s.n_kv_heads, s.head_dim) for y in (k, v))
            cache.append_rotary(k, v, p.slots, self.rotary, cos_sin, q=q, q_out=q)
            out = torch.empty((n, s.n_heads, s.head_dim), dtype=torch.bfloat16, device="cuda")
            cache.attend(q, out, p.seq_lens, p.starts, self.table, self.work, max_new=n)
            x = x + self._products(out.view(n, -1), ("o",), block)[0]
            gate, up = self._products(rms_norm(x, block["mlp_norm"]), ("gate", "up"), block)
            act = (torch.nn.functional.silu(gate) * up).bfloat16()
            x = x + self._products(act, ("down",), block)[0]
        self._advance()
        return self._products(rms_norm(x, self.final_norm), ("head",), {"head": self.head})[0]

    def score(self, logits, targets=None, top_k: int = 1, temperature: float = 1.0):
        """(logprob, entropy, rank, top_logprob, top_index) of a step's logits."""
        n = logits.shape[0]
        f, i = dict(dtype=torch.float32, device="cuda"), dict(dtype=torch.int32, device="cuda")
        out = (torch.empty(n, **f), torch.empty(n, **f), torch.empty(n, **i), torch.empty((n, top_k), **f),
               torch.empty((n, top_k), **i))
        serving.token_logprobs(logits, targets, *out, self.score_work, scale=1.0 / temperature)
        return out

    def beam_search(self, prompts, n_beams: int, max_new: int, end_token: int = -1, length_power: float = 0.0):
        """The likeliest continuations of every prompt (lists of tokens; no request
        may be under way, and prompts x n_beams be at most 16): tokens (prompts,
        n_beams, max_new), likeliest first, with -1 where there is no hypothesis,
        and the sums of their log probabilities.  A hypothesis that has chosen
        end_token keeps its sum and repeats it.  Sums are compared after division
        by the number of chosen tokens to the length_power.  Where the pages do not
        last, a prompt's sums are NaN and its tokens -1."""
        g, b, vocab = len(prompts), n_beams, self.spec.vocab
        rows = g * b
        if not 1 <= rows <= min(MAX_COLUMNS, self.plan.max_requests) or not all(prompts) or max_new < 1:
            raise ValueError("1..16 beams in all and no more than max_requests, prompts of a token or more and max_new >= 1 are wanted")
        if not all(0 <= t < vocab for prompt in prompts for t in prompt) or end_token >= vocab:
            raise ValueError(f"prompts, end_token: tokens below {vocab} are wanted")
        if not abs(length_power) * math.log2(max_new) <= 126:
            raise ValueError("length_power: max_new to this power passes float32")
        if bool(self.seq_lens.any()):
            raise ValueError("a request is under way")
        i32 = dict(dtype=torch.int32, device="cuda")
        pages = serving.BeamPages(self.caches, g, b)
        work = serving.beam_workspace(g, b, vocab)

        def reorder(parents, length=0):
            """The chosen beams' pages; rows that go on from none get that length."""
            pages.reorder(parents, self.seq_lens, self.table, self.free, self.free_count)
            self.seq_lens[:rows].copy_(torch.where(parents.view(-1) < 0, length, pages.seq_lens))
            self.free_count.copy_(pages.free_count)

        # prompts in the first row of each request, which its beams then fork; one that finds no pages ends at once
        logits = torch.zeros((rows, vocab), device="cuda")
        lost = torch.zeros(rows, dtype=torch.bool, device="cuda")
        for i, prompt in enumerate(prompts):
            for at in range(0, len(prompt), MAX_COLUMNS):
                piece = torch.tensor(prompt[at:at + MAX_COLUMNS], device="cuda")
                n_new = torch.zeros(rows, **i32)
                n_new[i * b] = piece.shape[0]
                logits[i * b] = self.step(piece, n_new.masked_fill_(lost, -1))[-1]
                lost |= self.plan.status != 0
        scores = torch.full((g, b), float("-inf"), device="cuda")
        scores[:, 0] = 0.0
        done = torch.zeros((g, b), dtype=torch.bool, device="cuda")
        chosen = torch.zeros((g, b), device="cuda")
        history = torch.full((g, b, max_new), -1, dtype=torch.int64, device="cuda")
        for i in range(max_new):
            new_scores, beam, token = torch.empty_like(scores), torch.empty((g, b), **i32), torch.empty((g, b), **i32)
            weights = (chosen + ~done) ** -length_power if length_power else None
            serving.beam_select(logits, scores, new_scores, beam, token, work, done=done if end_token >= 0 else None,
                                end_token=end_token, weights=weights)
            source = beam.clamp(min=0).long()
            history = history.gather(1, source[..., None].expand_as(history))
            history[..., i] = token
            history.masked_fill_(beam[..., None] < 0, -1)
            chosen, done = (chosen + ~done).gather(1, source), done.gather(1, source) | (token == end_token)
            if i + 1 == max_new:
                scores = new_scores
                break
            # A hypothesis that has ended needs no context, and a row without one has none.  Their rows are given
            # up; a negative length makes the plan refuse their tokens, so the others' stay at their rows' places.
            reorder(beam.masked_fill(done, -1), -1)
            # a beam whose copy found no page has no context any more: NaN, which the next choice passes on
            scores = new_scores.masked_fill(pages.status.view(g, b) != 0, float("nan"))
            logits = self.step(token.flatten().clamp(min=0).long(), torch.ones(rows, **i32))
        reorder(torch.full((g, b), -1, **i32))
        return history, scores


def synthetic_decoder(name: str = "tiny", max_requests: int = 4, n_pages: int = 64, page_size: int = 16, kind: str = "int8"):
    """A Decoder over a synthetic checkpoint's weights (workloads.MODELS)."""
    from . import workload_gpu as G
    from . import workloads as W

    spec = W.MODELS[name]
    m = G.synth_model_device(spec)

    def num(t):
        return t.view(torch.float16).float()

    blocks = []
    for y in m.layers:
        b = {k: compress(num(y["w" + k])) for k in W.MODEL_KINDS}
        b.update({k: num(y[k]) for k in ("attn_norm", "mlp_norm")})
        blocks.append(b)
    gen = torch.Generator("cuda").manual_seed(spec.seed)
    embedding = torch.randn((spec.vocab, spec.d_model), generator=gen, device="cuda")
    return Decoder(spec, blocks, num(m.final_norm), compress(num(m.lm_head)), embedding, max_requests, n_pages, page_size,
                   kind=kind)


def main():
    d = synthetic_decoder()
    prompts = [[5, 17, 42, 7, 99], [1], [200, 13, 8, 60, 61, 62, 63, 64, 65, 66]]
    n_new = torch.tensor([len(x) for x in prompts] + [0], dtype=torch.int32, device="cuda")
    tokens = torch.tensor(sum(prompts, []), device="cuda")
    for step in range(6):
        logits = d.step(tokens, n_new)
        if any(d.plan.status.tolist()):
            raise RuntimeError(f"step {step}: {[serving.STATUS[x] for x in d.plan.status.tolist()]}")
        last = (d.plan.starts[1:4] - 1).long()  # each request's newest token
        _, entropy, _, top, best = d.score(logits[last].contiguous(), top_k=3)
        tokens = best[:, 0].long()
        n_new = torch.tensor([1, 1, 1, 0], dtype=torch.int32, device="cuda")
        print(f"step {step}: lengths {d.seq_lens[:3].tolist()}, next {tokens.tolist()}, "
              f"logprob {[round(x, 3) for x in top[:, 0].tolist()]}, entropy {[round(x, 3) for x in entropy.tolist()]}")
    d.step(torch.empty(0, dtype=torch.int64, device="cuda"), torch.full((4,), -1, dtype=torch.int32, device="cuda"))
    found, scores = d.beam_search(prompts[:1], 4, 6)
    for hypothesis, score in zip(found[0].tolist(), scores[0].tolist()):
        print(f"beam: {hypothesis}, logprob {score:.3f}")


if __name__ == "__main__":
    main()
