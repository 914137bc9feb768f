"""Speculative decoding with drawn proposals over a paged 4-bit cache.

    python examples/paged_speculative.py

A looped Transformer with random weights, norms of queries and keys, and rotation by position serves
several sequences of different lengths at once.  Its drafter is the model without its loop: the
embedding and the readout.  Per step, on the device and without a copy to the host:

    1. the drafter proposes W tokens in turn, each drawn by das_sample;
    2. the verifier's block [x_t, y_1 .. y_{W-1}] runs through every depth and layer:
       das_qk_norm_rope makes queries, keys and values of one projection's rows, and
       das_mature_v_attention_paged4 attends over each sequence's pages and the block itself;
    3. das_speculative_accept accepts proposals and draws the token after them, so that what is
       emitted is distributed as if the target alone had drawn it;
    4. das_page_assign takes pages for the committed tokens, and gives the pages of the sequences
       that have ended back;
    5. das_kv_append_paged4 stores the committed inputs' keys and values at every depth.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2609_34538_gb300 as das  # noqa: E402


class LoopedModel:
    """h = E[token]; R times the L core layers: h += tanh(attention(h) Wo); logits = h U."""

    def __init__(self, vocab=512, width=256, heads=8, kv_heads=2, head_dim=64, layers=2, depths=4, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=g, device="cuda") / s[-2] ** 0.5
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.layers, self.depths, self.vocab = layers, depths, vocab
        self.E = torch.randn((vocab, width), generator=g, device="cuda")
        self.Wqkv = rand(layers, width, (heads + 2 * kv_heads) * head_dim)
        self.Wo, self.U = 0.2 * rand(layers, heads * head_dim, width), rand(width, vocab)
        self.q_norm, self.k_norm = (1 + 0.1 * torch.randn((layers, head_dim), generator=g, device="cuda") for _ in range(2))
        self.inv_freq = 10000.0 ** (-torch.arange(0, head_dim, 2, device="cuda") / head_dim)

    def draft(self, tokens):
        return self.E[tokens.long()] @ self.U

    def forward(self, tokens, length, block_len, attend):
        """tokens [B][T] at positions length[b] on -> logits [B][T][vocab] fp32 and the K/V of every depth and
        layer, [depths][layers][B][T][kv_heads][head_dim] bf16.  attend(layer, depth, q, k, v) -> out."""
        B, T = tokens.shape
        h = self.E[tokens.long()]
        shape = (self.depths, self.layers, B, T, self.kv_heads, self.head_dim)
        keys, values = (torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        for d in range(self.depths):
            for l in range(self.layers):
                rows = (h @ self.Wqkv[l]).to(torch.bfloat16).view(B, T, -1, self.head_dim)
                q, k, v = rows.split([self.heads, self.kv_heads, self.kv_heads], 2)
                q, _, _ = das.das_qk_norm_rope(q, k, v, self.inv_freq, length, block_len, self.q_norm[l],
                                               self.k_norm[l], k_out=keys[d, l], v_out=values[d, l])
                out = attend(l, d + 1, q, keys[d, l], values[d, l])
                h = h + torch.tanh(out.float().view(B, T, -1) @ self.Wo[l])
        return h @ self.U, keys, values


class Decoder:
    """The cache, its pages and the sequences' lengths."""

    def __init__(self, model, batch, pages, max_pages, block):
        self.model, self.batch, self.block = model, batch, block
        self.cache = das.PagedKVCache4.empty(model.depths, model.layers, pages, model.kv_heads, model.head_dim)
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
        self.table, self.length, self.flag = i32(batch, max_pages), i32(batch), i32(1)
        self.free = torch.arange(pages, dtype=torch.int32, device="cuda")
        self.free_count = torch.full((1,), pages, dtype=torch.int32, device="cuda")
        # one workspace for blocks of up to `block` rows
        self.ws = das.new_workspace_paged4(self.cache, batch, model.heads, block)

    def attend(self, block_len):
        def call(layer, depth, q, k, v):
            return das.das_mature_v_attention_paged4(self.cache, layer, depth, depth, self.table, self.length,
                                                     block_len, q, k, v, self.ws)[0]
        return call

    def forward(self, tokens, n):
        return self.model.forward(tokens, self.length, n, self.attend(n))

    def store(self, keys, values, grow):
        """Take grow[b] tokens more of each sequence (negative: give back) and store them."""
        slots = torch.empty(self.batch * keys.shape[3], dtype=torch.int32, device="cuda")
        _, _, start = das.das_page_assign(self.length, grow, self.table, self.free, self.free_count, slots,
                                          self.flag, new_len=self.length, new_free_count=self.free_count)
        das.das_kv_append_paged4(self.cache, keys, values, slots, start, self.flag)

    def prefill(self, prompts):
        """The prompts' tokens but the last, `block` at a time; returns the last ones [B]."""
        done = [0] * self.batch
        while any(done[b] < len(p) - 1 for b, p in enumerate(prompts)):
            part = [p[done[b]:min(done[b] + self.block, len(p) - 1)] for b, p in enumerate(prompts)]
            tokens = torch.tensor([t + [0] * (self.block - len(t)) for t in part], dtype=torch.int32, device="cuda")
            n = torch.tensor([len(t) for t in part], dtype=torch.int32, device="cuda")
            _, keys, values = self.forward(tokens, n)
            self.store(keys, values, n)
            done = [d + len(t) for d, t in zip(done, part)]
        return torch.tensor([p[-1] for p in prompts], dtype=torch.int32, device="cuda")

    def step(self, anchor, numbers, live, W, **sampling):
        """W proposals a sequence, their verification and the commit; sequences with live[b] = 0 take no part.
        numbers: uniform ones [2 W + 1][B].  Returns (proposals, accepted, next_token)."""
        last, drafts, ids = anchor, [], []
        for i in range(W):
            logits = self.model.draft(last)
            last = das.das_sample(logits[:, None], numbers[i][:, None], **sampling)[0][:, 0]
            drafts.append(logits)
            ids.append(last)
        proposals = torch.stack(ids, 1)
        tokens = torch.cat([anchor[:, None], proposals[:, :-1]], 1)
        logits, keys, values = self.forward(tokens, live * W)
        accepted, token, committed = das.das_speculative_accept(
            logits, torch.stack(drafts, 1), proposals, numbers[W:2 * W].t().contiguous(), numbers[2 * W], **sampling)
        self.store(keys, values, committed * live)
        return proposals, accepted, token

    def release(self, ended):
        """Gives the pages of the sequences with ended[b] = 1 back."""
        das.das_page_assign(self.length, -self.length * ended, self.table, self.free, self.free_count,
                            torch.empty(1, dtype=torch.int32, device="cuda"), self.flag, new_len=self.length,
                            new_free_count=self.free_count)


def decode(prompts, new_tokens, W=4, temperature=0.8, top_k=40, top_p=0.95, min_p=0.01, seed=0, model=None):
    """Emits new_tokens[b] tokens after each prompt; returns (tokens, decoder, accepted proposals a step)."""
    model = LoopedModel() if model is None else model
    B, g = len(prompts), torch.Generator(device="cuda").manual_seed(seed)
    longest = max(len(p) + n + W for p, n in zip(prompts, new_tokens))
    max_pages = -(-longest // das.PAGE_TOKENS)
    dec = Decoder(model, B, pages=B * max_pages, max_pages=max_pages, block=max(W, 16))
    each = lambda x, dt: torch.full((B,), x, dtype=dt, device="cuda")
    sampling = dict(temperature=each(temperature, torch.float32), top_k=each(top_k, torch.int32),
                    top_p=each(top_p, torch.float32), min_p=each(min_p, torch.float32))
    anchor = dec.prefill(prompts)
    out, accepts = [[] for _ in range(B)], []
    live = torch.ones(B, dtype=torch.int32, device="cuda")
    while any(len(o) < n for o, n in zip(out, new_tokens)):
        numbers = torch.rand((2 * W + 1, B), generator=g, device="cuda")
        proposals, accepted, anchor = dec.step(anchor, numbers, live, W, **sampling)
        was = live.tolist()
        for b, (row, a, t) in enumerate(zip(proposals.tolist(), accepted.tolist(), anchor.tolist())):
            if was[b]:
                accepts.append(a)
                out[b] += row[:a] + ([t] if a < W else [])
        ended = torch.tensor([int(w and len(o) >= n) for w, o, n in zip(was, out, new_tokens)], dtype=torch.int32,
                             device="cuda")
        dec.release(ended)
        live = live * (1 - ended)
    return [o[:n] for o, n in zip(out, new_tokens)], dec, accepts


def main():
    prompts = [list(range(3, 3 + n)) for n in (5, 130, 64, 17)]
    tokens, dec, accepts = decode(prompts, [60, 20, 40, 90])
    for p, t in zip(prompts, tokens):
        print(f"prompt of {len(p)}: {len(t)} tokens: {t[:10]} ...")
    print(f"{sum(accepts) / len(accepts):.2f} proposals accepted a step; {dec.free_count.item()} of "
          f"{dec.free.numel()} pages free; flag {dec.flag.item()}, status {das.workspace_status(dec.ws)}")


if __name__ == "__main__":
    main()
