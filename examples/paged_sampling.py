"""Speculative decoding with sampling over a paged 8-bit cache.

    python examples/paged_sampling.py

A looped Transformer with random weights (an embedding, L core layers applied
R times, a readout) serves several sequences of different lengths at once.
Per step, on the device and without a copy to the host:

    1. the verifier's block [x_t, y_1 .. y_{W-1}] runs through every depth and
       layer; das_mature_v_attention_paged attends over each sequence's pages
       (key_depth = value_depth = the depth) and the block itself;
    2. das_sample_accept draws the target's tokens with the step's random
       numbers and accepts the proposals while they equal the draws, so that
       every emitted token is a draw from the target's own distribution;
    3. das_page_assign takes pages for the committed tokens, and gives the
       pages of the sequences that have ended back;
    4. das_kv_append_paged stores the committed inputs' K/V at every depth.

The host reads the accepted tokens to make the next proposals (here, the
tokens that followed the last time the same token was emitted).
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2609_34538_gb300 as das  # noqa: E402


class LoopedModel:
    """h = E[token]; R times the L core layers: h += tanh(attention(h) Wo);
    logits = h U."""

    def __init__(self, vocab=512, width=256, heads=8, kv_heads=2, head_dim=64, layers=2, depths=4, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=g, device="cuda") / s[-2] ** 0.5
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.layers, self.depths, self.vocab = layers, depths, vocab
        self.E = torch.randn((vocab, width), generator=g, device="cuda")
        self.Wq, self.Wk, self.Wv = (rand(layers, width, n * head_dim) for n in (heads, kv_heads, kv_heads))
        self.Wo, self.U = rand(layers, heads * head_dim, width), 3 * rand(width, vocab)

    def forward(self, tokens, attend):
        """tokens [B][T] -> logits [B][T][vocab] fp32 and the K/V of every depth and layer,
        [depths][layers][B][T][kv_heads][head_dim] bf16.  attend(layer, depth, q, k, v) -> out."""
        B, T = tokens.shape
        h = self.E[tokens.long()]
        shape = (self.depths, self.layers, B, T, self.kv_heads, self.head_dim)
        keys, values = (torch.empty(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        for d in range(self.depths):
            for l in range(self.layers):
                q = (h @ self.Wq[l]).to(torch.bfloat16).view(B, T, self.heads, self.head_dim)
                keys[d, l] = (h @ self.Wk[l]).to(torch.bfloat16).view(shape[2:])
                values[d, l] = (h @ self.Wv[l]).to(torch.bfloat16).view(shape[2:])
                out = attend(l, d + 1, q, keys[d, l], values[d, l])
                h = h + torch.tanh(out.float().view(B, T, -1) @ self.Wo[l])
        return h @ self.U, keys, values


class PagedDecoder:
    """The cache, its pages and the sequences' lengths."""

    def __init__(self, model, batch, pages, max_pages, block):
        self.model, self.batch, self.block = model, batch, block
        self.cache = das.PagedKVCache.empty(model.depths, model.layers, pages, model.kv_heads, model.head_dim)
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
        self.table, self.length, self.flag = i32(batch, max_pages), i32(batch), i32(1)
        self.free = torch.arange(pages, dtype=torch.int32, device="cuda")
        self.free_count = torch.full((1,), pages, dtype=torch.int32, device="cuda")
        self.ws = das.new_workspace_paged(self.cache, batch, model.heads, block)

    def attend(self, block_len):
        def call(layer, depth, q, k, v):
            return das.das_mature_v_attention_paged(self.cache, layer, depth, depth, self.table, self.length,
                                                    block_len, q, k, v, self.ws)[0]
        return call

    def store(self, keys, values, grow):
        """Take grow[b] tokens more of each sequence (negative: give back) and store them."""
        slots = torch.empty(self.batch * keys.shape[3], dtype=torch.int32, device="cuda")
        _, _, start = das.das_page_assign(self.length, grow, self.table, self.free, self.free_count, slots,
                                          self.flag, new_len=self.length, new_free_count=self.free_count)
        das.das_kv_append_paged(self.cache, keys, values, slots, start, self.flag)

    def prefill(self, prompts):
        """The prompts' tokens but the last, `block` at a time; returns the last ones [B]."""
        done = [0] * self.batch
        while any(done[b] < len(p) - 1 for b, p in enumerate(prompts)):
            part = [p[done[b]:min(done[b] + self.block, len(p) - 1)] for b, p in enumerate(prompts)]
            tokens = torch.tensor([t + [0] * (self.block - len(t)) for t in part], dtype=torch.int32, device="cuda")
            n = torch.tensor([len(t) for t in part], dtype=torch.int32, device="cuda")
            _, keys, values = self.model.forward(tokens, self.attend(n))
            self.store(keys, values, n)
            done = [d + len(t) for d, t in zip(done, part)]
        return torch.tensor([p[-1] for p in prompts], dtype=torch.int32, device="cuda")

    def step(self, anchor, proposals, uniforms, live, **sampling):
        """One verify-and-commit step of W = proposals.shape[1] proposals a sequence; sequences
        with live[b] = 0 take no part.  Returns (accepted, target_ids, next_token, logprobs)."""
        W = proposals.shape[1]
        tokens = torch.cat([anchor[:, None], proposals[:, :-1]], 1)
        logits, keys, values = self.model.forward(tokens, self.attend(live * W))
        accepted, ids, token, committed, logprobs = das.das_sample_accept(logits, proposals, uniforms, **sampling)
        self.store(keys, values, committed * live)
        return accepted, ids, token, logprobs

    def release(self, ended):
        """Gives the pages of the sequences with ended[b] = 1 back."""
        das.das_page_assign(self.length, -self.length * ended, self.table, self.free, self.free_count,
                            torch.empty(1, dtype=torch.int32, device="cuda"), self.flag, new_len=self.length,
                            new_free_count=self.free_count)


def decode(prompts, new_tokens, W=4, temperature=0.8, top_k=40, top_p=0.95, min_p=0.01, seed=0, model=None):
    """Emits new_tokens[b] tokens after each prompt; returns (tokens, their logprobs, decoder,
    accepted proposals a step)."""
    model = LoopedModel() if model is None else model
    B, g = len(prompts), torch.Generator(device="cuda").manual_seed(seed)
    longest = max(len(p) + n + W for p, n in zip(prompts, new_tokens))
    max_pages = -(-longest // das.PAGE_TOKENS)
    dec = PagedDecoder(model, B, pages=B * max_pages, max_pages=max_pages, block=max(W, 16))
    each = lambda x, dt: torch.full((B,), x, dtype=dt, device="cuda")
    sampling = dict(temperature=each(temperature, torch.float32), top_k=each(top_k, torch.int32),
                    top_p=each(top_p, torch.float32), min_p=each(min_p, torch.float32))
    anchor = dec.prefill(prompts)
    # the block buffers of a step have W rows: a workspace for that shape
    dec.block, dec.ws = W, das.new_workspace_paged(dec.cache, B, model.heads, W)
    out, logp = [[] for _ in range(B)], [[] for _ in range(B)]
    follow = [{} for _ in range(B)]
    accepts = []
    live = torch.ones(B, dtype=torch.int32, device="cuda")
    while any(len(o) < n for o, n in zip(out, new_tokens)):
        last = anchor.tolist()
        guess = []
        for b in range(B):
            row, t = [], last[b]
            for _ in range(W):
                t = follow[b].get(t, t)
                row.append(t)
            guess.append(row)
        u = torch.rand((B, W), generator=g, device="cuda")
        proposals = torch.tensor(guess, dtype=torch.int32, device="cuda")
        accepted, ids, anchor, lp = dec.step(anchor, proposals, u, live, **sampling)
        was = live.tolist()
        for b, (a, row, l) in enumerate(zip(accepted.tolist(), ids.tolist(), lp.tolist())):
            if not was[b]:
                continue
            accepts.append(a)
            for t, x in zip(row[:min(a + 1, W)], l):
                follow[b][last[b]] = t
                last[b] = t
                out[b].append(t)
                logp[b].append(x)
        ended = torch.tensor([int(w and len(o) >= n) for w, o, n in zip(was, out, new_tokens)], dtype=torch.int32,
                             device="cuda")
        dec.release(ended)
        live = live * (1 - ended)
    return [o[:n] for o, n in zip(out, new_tokens)], [l[:n] for l, n in zip(logp, new_tokens)], dec, accepts


def main():
    prompts = [list(range(3, 3 + n)) for n in (5, 130, 64, 17)]
    tokens, logprobs, dec, accepts = decode(prompts, [60, 20, 40, 90])
    for p, t, l in zip(prompts, tokens, logprobs):
        print(f"prompt of {len(p)}: {len(t)} tokens, mean logprob {sum(l) / len(l):.3f}: {t[:10]} ...")
    print(f"{sum(accepts) / len(accepts):.2f} proposals accepted a step; {dec.free_count.item()} of "
          f"{dec.free.numel()} pages free; flag {dec.flag.item()}, status {das.workspace_status(dec.ws)}")


if __name__ == "__main__":
    main()
