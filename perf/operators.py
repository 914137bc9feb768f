"""Cases, inputs and plain forms of the paged-cache and sampling operators.

    assign     das_page_assign: block table and slot map from request lengths
    append     das_kv_append_paged: commit into the paged block-scaled e4m3 cache
    attention  das_mature_v_attention_paged: attention over that cache
    sample     das_sample_accept: sampled acceptance (temperature, top-k, top-p, min-p)

With `own` false, run() computes an operator in elementary torch operations in 32 bits; with `own` true it
makes the library's calls on the same state.
"""
import math

import numpy as np
import torch

own = False

PAGE = 64                       # tokens per page
E_MIN, E_MAX = -40, 120         # exponents of a block's scale
ONE = float(2 ** 32)            # weight of the most likely token


# ---- cases ---------------------------------------------------------------------------------------------------------

def listed():
    return [
        # one decoding step of 16 ragged requests: each takes 1 to 17 tokens, two have ended
        dict(name="assign decode", op="assign", batch=16, max_len=8192, max_grow=17, released=2),
        # the prompts of 256 new requests are admitted at once
        dict(name="assign prompts", op="assign", batch=256, max_len=1, max_grow=8192, released=0),
        # the verify-and-commit pass: 16 candidates, 32 depths, 4 layers, 8 heads of 128
        dict(name="append verify", op="append", depths=32, layers=4, batch=8, width=16, kv_heads=8, head_dim=128,
             held=16384),
        # a prompt's keys and values, an odd number of tokens, 8 depths
        dict(name="append prompt", op="append", depths=8, layers=4, batch=4, width=1001, kv_heads=8, head_dim=128,
             held=0),
        # the smallest model: 4 heads of 64, 256 tokens, 4 drafted
        dict(name="attention tiny", op="attention", batch=1, q_heads=4, kv_heads=4, head_dim=64, lo=256, hi=256,
             block=4),
        # one token at a time, one sequence, every query head with a kv head of its own
        dict(name="attention single token", op="attention", batch=1, q_heads=32, kv_heads=32, head_dim=128, lo=4096,
             hi=4096, block=1),
        # one sequence drafting a block of 8
        dict(name="attention decode", op="attention", batch=1, q_heads=32, kv_heads=32, head_dim=128, lo=4096,
             hi=4096, block=8),
        # 16 ragged sequences, blocks of 4 to 16, four query heads to a kv head
        dict(name="attention batched", op="attention", batch=16, q_heads=32, kv_heads=8, head_dim=128, lo=1024,
             hi=8192, block=16),
        # long prefixes, blocks of 16
        dict(name="attention long", op="attention", batch=4, q_heads=32, kv_heads=8, head_dim=128, lo=32768, hi=32768,
             block=16),
        # the next token of one sequence, nucleus sampling
        dict(name="sample one", op="sample", batch=1, width=1, vocab=32000, dtype="f32", temperature=0.8, top_k=0,
             top_p=0.95, min_p=0.0),
        # the verifier's 16 conditionals of 8 sequences, all filters
        dict(name="sample verify", op="sample", batch=8, width=16, vocab=32000, dtype="f32", temperature=0.8,
             top_k=200, top_p=0.95, min_p=0.02),
        # 64 sequences with a large odd vocabulary, 16-bit logits with many equal ones, no top-k
        dict(name="sample wide", op="sample", batch=64, width=1, vocab=128257, dtype="bf16", temperature=1.0, top_k=0,
             top_p=0.9, min_p=0.0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["assign", "append", "attention", "attention", "sample", "sample"])
    if op == "assign":
        batch = _log_int(rng, 1, 700)
        return dict(op=op, batch=batch, max_len=_log_int(rng, 1, 32768),
                    max_grow=_log_int(rng, 1, max(1, min(8192, 2000000 // batch))), released=rng.randint(0, batch // 4))
    if op == "append":
        depths, layers, kv_heads = rng.randint(1, 32), rng.randint(1, 4), rng.choice([1, 2, 4, 8, 32])
        head_dim, batch = rng.choice([64, 128]), _log_int(rng, 1, 16)
        room = 120_000_000 // (depths * layers * kv_heads * head_dim * batch)
        return dict(op=op, depths=depths, layers=layers, batch=batch, width=_log_int(rng, 1, max(1, min(1500, room))),
                    kv_heads=kv_heads, head_dim=head_dim, held=_log_int(rng, 1, 20000) - 1)
    if op == "attention":
        kv_heads, group = rng.choice([1, 2, 4, 8, 32]), rng.choice([1, 1, 2, 4, 5, 8])
        batch = _log_int(rng, 1, 24)
        hi = _log_int(rng, 1, min(32768, 4 * 8 * 32768 // (batch * kv_heads)))
        return dict(op=op, batch=batch, q_heads=kv_heads * group, kv_heads=kv_heads, head_dim=rng.choice([64, 128]),
                    lo=rng.choice([1, max(1, hi // 3), hi]), hi=hi, block=_log_int(rng, 1, 64 // group))
    batch, width = _log_int(rng, 1, 64), _log_int(rng, 1, 16)
    return dict(op=op, batch=batch, width=width, vocab=_log_int(rng, 1000, min(160000, 8_000_000 // (batch * width))),
                dtype=rng.choice(["f32", "bf16"]), temperature=round(rng.uniform(0.3, 1.5), 3),
                top_k=rng.choice([0, 1, _log_int(rng, 2, 2000)]), top_p=rng.choice([1.0, round(rng.uniform(0.3, 0.999), 3)]),
                min_p=rng.choice([0.0, round(rng.uniform(0.001, 0.2), 4)]))


def work(case):
    op = case["op"]
    if op == "assign":
        _, grow, held = _lengths(case)
        slots = int(np.maximum(grow, 0).sum())
        moved = int(np.abs(-(-(held + grow) // PAGE) - -(-held // PAGE)).sum())
        return {"bytes": 16 * case["batch"] + 8 * moved + 4 * slots, "flops": 0}
    if op == "append":
        n = int(_appended(case).sum())
        per = case["depths"] * case["layers"] * case["kv_heads"] * case["head_dim"] * 2
        return {"bytes": n * per * 3, "flops": n * per * 3}
    if op == "attention":
        P, T = _prefix_and_block(case)
        tiles = int((-(-P // PAGE)).sum())
        D, H, Hq = case["head_dim"], case["kv_heads"], case["q_heads"]
        rows = int(T.sum())
        return {"bytes": int(P.sum()) * H * D * 2 + tiles * (8 * H + 4) + rows * (Hq * (4 * D + 4) + H * D * 4),
                "flops": int((4 * T * Hq * D * (P + (T + 1) / 2)).sum())}
    n = case["batch"] * case["width"]
    return {"bytes": n * (case["vocab"] * (4 if case["dtype"] == "f32" else 2) + 16) + case["batch"] * 28,
            "flops": 4 * n * case["vocab"]}


# ---- inputs --------------------------------------------------------------------------------------------------------

def _rng(case, salt):
    return np.random.default_rng([case["batch"], salt])


def _lengths(case):
    """Tokens held by each request, and what each takes (negative: gives back)."""
    g = _rng(case, 1)
    B = case["batch"]
    held = g.integers(case["max_len"] // 8, case["max_len"] + 1, B)
    if case["max_len"] == 1:
        held = np.zeros(B, dtype=np.int64)
    grow = g.integers(max(1, case["max_grow"] // 8), case["max_grow"] + 1, B)
    ended = g.permutation(B)[:case["released"]]
    grow[ended] = -held[ended]
    return B, grow.astype(np.int64), held.astype(np.int64)


def _appended(case):
    g = _rng(case, 2)
    W = case["width"]
    return g.integers((W + 1) // 2, W + 1, case["batch"])


def _prefix_and_block(case):
    g = _rng(case, 3)
    B = case["batch"]
    P = g.integers(case["lo"], case["hi"] + 1, B)
    T = g.integers(max(1, case["block"] // 4), case["block"] + 1, B) if B > 1 else np.full(1, case["block"])
    return P.astype(np.int64), T.astype(np.int64)


def _i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _block_scaled(shape, g):
    """Codes and power-of-two scales of normal values whose size differs from block to block."""
    codes = torch.empty(shape, dtype=torch.uint8, device="cuda")
    scales = torch.empty(shape[:4], dtype=torch.float32, device="cuda")
    for d in range(shape[0]):
        for layer in range(shape[1]):
            x = torch.randn(shape[2:], generator=g, device="cuda")
            x *= torch.rand(shape[2:4], generator=g, device="cuda")[..., None, None] * 1.5 + 0.5
            s = _scale_of(x.abs().amax((-1, -2)))
            codes[d, layer] = (x / s[..., None, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
            scales[d, layer] = s
    return codes, scales


def _scale_of(amax):
    """2^e, the least e in [E_MIN, E_MAX] with amax <= 448 * 2^e."""
    m, e = torch.frexp(amax)                         # amax = m 2^e, m in [0.5, 1); 448 = 0.875 * 2^9
    e = e - 9 + (m > 0.875).to(e.dtype)
    e = torch.where(amax > 0, e, torch.full_like(e, E_MIN)).clamp(E_MIN, E_MAX)
    return torch.ldexp(torch.ones_like(amax), e)


def _library():
    if not own:
        return None
    import paper_2609_34538_gb300 as das
    return das


def prepare(case, seed):
    g = _gen(seed)
    host = np.random.default_rng(seed)
    op = case["op"]
    das = _library()
    s = {"case": case, "op": op}
    if op == "assign":
        B, grow, held = _lengths(case)
        rows = max(1, int((-(-(held + np.maximum(grow, 0)) // PAGE)).max()))
        have = -(-held // PAGE)
        new = int((-(-np.maximum(held + grow, 0) // PAGE)).sum())
        pages = max(int(have.sum()), new) + 64
        ids = host.permutation(pages)
        table = host.integers(0, pages, (B, rows))
        used = np.arange(rows)[None, :] < have[:, None]
        table[used] = ids[:used.sum()]
        free = np.zeros(pages, dtype=np.int64)
        count = pages - int(used.sum())
        free[:count] = ids[used.sum():]
        s.update(seq_len=_i32(held), grow=_i32(grow), table=_i32(table), free=_i32(free), count=_i32([count]),
                 slots=torch.empty(max(1, int(np.maximum(grow, 0).sum())), dtype=torch.int32, device="cuda"),
                 flag=_i32([0]), new_len=_i32(held), new_count=_i32([0]), start=_i32([0] * (B + 1)))
    elif op == "append":
        B, W, R, L, H, D = (case[k] for k in ("batch", "width", "depths", "layers", "kv_heads", "head_dim"))
        n = _appended(case)
        first = case["held"] % PAGE + np.arange(B) * 7 if case["held"] else np.zeros(B, dtype=np.int64)
        first = first % PAGE                          # the place of the first new token in its page
        touched = -(-(first + n) // PAGE)
        pages = int(touched.sum())
        ids = host.permutation(pages)
        at = np.concatenate([[0], np.cumsum(touched)])
        slots = np.concatenate([ids[at[b] + (first[b] + np.arange(n[b])) // PAGE] * PAGE
                                + (first[b] + np.arange(n[b])) % PAGE for b in range(B)])
        start = np.concatenate([[0], np.cumsum(n)])
        k, ks = _block_scaled((R, L, pages, H, PAGE, D), g)
        v, vs = _block_scaled((R, L, pages, H, PAGE, D), g)
        s.update(k=k, v=v, ks=ks, vs=vs, slots=_i32(slots), start=_i32(start), flag=_i32([0]),
                 kn=torch.empty((R, L, B, W, H, D), dtype=torch.bfloat16, device="cuda"),
                 vn=torch.empty((R, L, B, W, H, D), dtype=torch.bfloat16, device="cuda"))
        for d in range(R):
            s["kn"][d] = torch.randn((L, B, W, H, D), generator=g, device="cuda")
            s["vn"][d] = torch.randn((L, B, W, H, D), generator=g, device="cuda") * 2
    elif op == "attention":
        B, H, Hq, D, T = (case[k] for k in ("batch", "kv_heads", "q_heads", "head_dim", "block"))
        P, Tb = _prefix_and_block(case)
        need = -(-P // PAGE)
        rows, pages = max(1, int(need.max())), max(1, int(need.sum()))
        table = host.integers(0, pages, (B, rows))
        used = np.arange(rows)[None, :] < need[:, None]
        table[used] = host.permutation(pages)[:used.sum()]
        k, ks = _block_scaled((2, 1, pages, H, PAGE, D), g)
        v, vs = _block_scaled((2, 1, pages, H, PAGE, D), g)
        bf = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)
        s.update(k=k, v=v, ks=ks, vs=vs, table=_i32(table), P=_i32(P), T=_i32(Tb), q=bf(B, T, Hq, D),
                 kb=bf(B, T, H, D), vb=bf(B, T, H, D))
    else:
        B, W, V = case["batch"], case["width"], case["vocab"]
        logits = 2 * torch.randn((B, W, V), generator=g, device="cuda")
        logits = logits.to(torch.float32 if case["dtype"] == "f32" else torch.bfloat16)
        u = torch.rand((B, W), generator=g, device="cuda")
        full = lambda x, dt=torch.float32: torch.full((B,), x, dtype=dt, device="cuda")
        s.update(logits=logits, u=u, temperature=full(case["temperature"]), top_k=full(case["top_k"], torch.int32),
                 top_p=full(case["top_p"]), min_p=full(case["min_p"]))
        # the drafter's proposals: mostly what the target would draw with these numbers
        target = _sample(s)[0]
        other = torch.randint(0, V, (B, W), generator=g, device="cuda", dtype=torch.int32)
        s["draft"] = torch.where(torch.rand((B, W), generator=g, device="cuda") < 0.85, target, other)
    if das is not None and op in ("append", "attention"):
        s["cache"] = das.PagedKVCache(s["k"], s["v"], s["ks"], s["vs"])
        if op == "attention":
            s["ws"] = das.new_workspace_paged(s["cache"], case["batch"], case["q_heads"], case["block"])
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------

def run(s):
    return {"assign": _run_assign, "append": _run_append, "attention": _run_attention, "sample": _run_sample}[s["op"]](s)


def _run_assign(s):
    das = _library()
    if das is not None:
        das.das_page_assign(s["seq_len"], s["grow"], s["table"], s["free"], s["count"], s["slots"], s["flag"],
                            new_len=s["new_len"], new_free_count=s["new_count"], slot_start=s["start"])
        new_len, count, start, table, slots = s["new_len"], s["new_count"], s["start"], s["table"], s["slots"]
    else:
        new_len, count, start, table, slots = _assign(s)
    return {"new_len": new_len, "free_count": count, "slot_start": start, "table": table, "slots": slots,
            "flag": s["flag"]}


def _assign(s):
    old, grow, table, free = s["seq_len"].long(), s["grow"].long(), s["table"], s["free"]
    B, rows = table.shape
    cap = s["slots"].numel()
    new = (old + grow).clamp(min=0)
    have, want = (old + PAGE - 1) // PAGE, (new + PAGE - 1) // PAGE
    give, take = (have - want).clamp(min=0), (want - have).clamp(min=0)
    fits = (grow > 0) & (new <= rows * PAGE)
    take = torch.where(fits, take, 0)
    avail = s["count"].long() + give.sum()
    served = fits & ((take == 0) | (take.cumsum(0) <= avail)) & (torch.where(fits, grow, 0).cumsum(0) <= cap)
    s["flag"].bitwise_or_(((grow > 0) & ~served).any().to(torch.int32))
    take, count = torch.where(served, take, 0), torch.where(served, grow, 0)
    new_len = torch.where(grow > 0, torch.where(served, new, old), new)
    # what is given back goes on the stack in request order, then pages are taken from its top
    col = torch.arange(rows, device=table.device)[None, :]
    giving = (col >= want[:, None]) & (col < have[:, None]) & (give > 0)[:, None]
    place = s["count"].long() + (give.cumsum(0) - give)[:, None] + col - want[:, None]
    stack = torch.cat([free, free.new_zeros(1)])
    stack[torch.where(giving, place, free.numel())] = table
    taking = (col >= have[:, None]) & (col < (have + take)[:, None])
    top = avail - 1 - (take.cumsum(0) - take)[:, None] - (col - have[:, None])
    table = torch.where(taking, stack[top.clamp(0, free.numel() - 1)], table)
    start = torch.cat([count.new_zeros(1), count.cumsum(0)])
    i = torch.arange(cap, device=table.device)
    b = torch.bucketize(i, start[1:], right=True).clamp(max=B - 1)
    pos = old[b] + i - start[b]
    slots = table[b, (pos // PAGE).clamp(max=rows - 1)] * PAGE + (pos % PAGE).int()
    slots = torch.where(i < start[-1], slots, -1)
    return new_len.int(), (avail - take.sum()).int().view(1), start.int(), table, slots.int()


def _run_append(s):
    das = _library()
    if das is not None:
        das.das_kv_append_paged(s["cache"], s["kn"], s["vn"], s["slots"], s["start"], s["flag"])
    else:
        for codes, scales, new in ((s["k"], s["ks"], s["kn"]), (s["v"], s["vs"], s["vn"])):
            _append(s, codes, scales, new)
    f8 = torch.float8_e4m3fn
    return {"k": s["k"].view(f8), "v": s["v"].view(f8), "k_scale": s["ks"], "v_scale": s["vs"], "flag": s["flag"]}


def _append(s, codes, scales, new):
    R, L, B, W, H, D = new.shape
    most = (W + 2 * PAGE - 2) // PAGE
    start = s["start"].long()
    n, slots = start[1:] - start[:-1], s["slots"].long()
    first = slots[start[:-1]] % PAGE                                            # [B]
    p = torch.arange(most, device=codes.device)[None, :]                        # [B, most]: a request's pages
    p = torch.where(p * PAGE < (first + n)[:, None], p, 0)                      # past its last: its first again
    page = slots[start[:-1, None] + (p * PAGE - first[:, None]).clamp(min=0)] // PAGE
    i = torch.arange(PAGE, device=codes.device)
    t = p[..., None] * PAGE + i - first[:, None, None]                          # the new token at a place, if any
    fresh = (t >= 0) & (t < n[:, None, None])
    older = (p[..., None] == 0) & (i < first[:, None, None])
    x = new[:, :, torch.arange(B, device=codes.device)[:, None, None], t.clamp(0, W - 1)]  # [R,L,B,most,64,H,D]
    x = torch.where(fresh[..., None, None], x.float(), 0.0).transpose(-3, -2)   # [R,L,B,most,H,64,D]
    scale = _scale_of(x.abs().amax((-1, -2)))
    held = scales[:, :, page]                                                   # [R,L,B,most,H]
    scale = torch.where(older.any(-1)[..., None], torch.maximum(scale, held), scale)
    was = codes[:, :, page]
    again = was.view(torch.float8_e4m3fn).float() * (held / scale)[..., None, None]
    x = torch.where(older[:, :, None, :, None], again, x / scale[..., None, None])
    x = x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    codes[:, :, page] = torch.where((fresh | older)[:, :, None, :, None], x, was)
    scales[:, :, page] = scale


def _run_attention(s):
    das = _library()
    if das is not None:
        out, lse = das.das_mature_v_attention_paged(s["cache"], 0, 1, 2, s["table"], s["P"], s["T"], s["q"], s["kb"],
                                                    s["vb"], s["ws"])
    else:
        out, lse = _attention(s)
    return {"out": out, "lse": lse}


def _attention(s):
    B, T, Hq, D = s["q"].shape
    H = s["kb"].shape[2]
    table = s["table"].long()

    def gathered(codes, scales):
        x = codes[table].view(torch.float8_e4m3fn).float() * scales[table][..., None, None]   # [B, pages, H, 64, D]
        return x.transpose(1, 2).reshape(B, H, -1, D)

    k, v = gathered(s["k"][0, 0], s["ks"][0, 0]), gathered(s["v"][1, 0], s["vs"][1, 0])
    N = k.shape[2]
    seen = (torch.arange(N, device=k.device) < s["P"][:, None])[:, None, None, :]             # [B, 1, 1, N]
    v = v.mul_(seen[:, :, 0, :, None])
    q = s["q"].float().view(B, T, H, Hq // H, D).permute(0, 2, 3, 1, 4).reshape(B, H, -1, D)  # rows: group, place
    scale = 1 / math.sqrt(D)
    a = torch.where(seen, torch.matmul(q, k.transpose(2, 3)) * scale, -math.inf)
    kb, vb = s["kb"].float().transpose(1, 2), s["vb"].float().transpose(1, 2)                 # [B, H, T, D]
    i = torch.arange(T, device=k.device)
    live = (i[None, :] < s["T"][:, None])                                                     # [B, T]
    causal = (i[None, :] <= i[:, None]).repeat(Hq // H, 1)
    c = torch.where(causal, torch.matmul(q, kb.transpose(2, 3)) * scale, -math.inf)
    m = torch.maximum(a.amax(-1), c.amax(-1))[..., None]
    a, c = torch.exp(a - m), torch.exp(c - m)
    total = a.sum(-1) + c.sum(-1)
    out = (torch.matmul(a, v) + torch.matmul(c, vb)) / total[..., None]
    lse = m[..., 0] + torch.log(total)
    out = out.view(B, H, Hq // H, T, D).permute(0, 3, 1, 2, 4).reshape(B, T, Hq, D)
    out = torch.where(live[:, :, None, None], out, 0.0).to(torch.bfloat16)
    lse = torch.where(live[:, None, :], lse.view(B, Hq, T), -math.inf)
    return out, lse


def _run_sample(s):
    das = _library()
    if das is not None:
        accepted, ids, token, committed, logprob = das.das_sample_accept(
            s["logits"], s["draft"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
            min_p=s["min_p"])
    else:
        ids, logprob = _sample(s)
        W = ids.shape[1]
        accepted = (ids == s["draft"]).int().cumprod(1).sum(1)
        at = accepted.clamp(max=W - 1)[:, None]
        token = torch.where(accepted[:, None] < W, ids.gather(1, at), s["draft"].gather(1, at))[:, 0]
        accepted, committed = accepted.int(), (accepted + 1).clamp(max=W).int()
    return {"accepted": accepted, "ids": ids, "next": token, "committed": committed, "logprob": logprob}


def _sample(s):
    z = s["logits"].float() + 0.0                                          # -0 counts as 0
    B, W, V = z.shape
    each = lambda name: s[name][:, None, None]
    T, k, p, floor = each("temperature"), each("top_k").long(), each("top_p"), each("min_p")
    z, order = torch.sort(z, dim=-1, descending=True, stable=True)
    e = torch.where(z == z[..., :1], 1.0, torch.exp((z - z[..., :1]) / T))
    w = (e.double() * ONE).round().long()                                  # whole numbers: sums do not depend on order
    rank = torch.arange(V, device=z.device)
    kept = (k <= 0) | (rank < k)
    w = torch.where(kept, w, 0)
    before = w.cumsum(-1) - w
    least = torch.ceil(p.double() * w.sum(-1, keepdim=True).double()).long().clamp(min=1)
    kept = kept & ((p >= 1) | (before < least)) & (e >= floor.clamp(max=1.0))
    w = torch.where(kept, w, 0)
    total = w.sum(-1, keepdim=True)
    r = torch.minimum((s["u"].double()[..., None] * total.double()).floor().long(), total - 1)
    w = torch.zeros_like(w).scatter_(-1, order, w)                          # by index again
    token = (w.cumsum(-1) <= r).sum(-1, keepdim=True)
    chosen = s["logits"].float().gather(-1, token)
    logprob = (chosen - z[..., :1]) / T - torch.log((total.double() / ONE).float())
    return token[..., 0].int(), logprob[..., 0]


# ---- in 64 bits ----------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "assign":
        return None
    if s["op"] == "append":
        return _exact_append(s)
    if s["op"] == "attention":
        return _exact_attention(s)
    lg, u = s["logits"].double().cpu().numpy(), s["u"].double().cpu().numpy()
    B, W, V = lg.shape
    T, p, floor = float(s["temperature"][0]), float(s["top_p"][0]), float(s["min_p"][0])
    logprob = np.empty((B, W), dtype=np.float64)
    for b in range(B):
        for i in range(W):
            x = (lg[b, i] - lg[b, i].max()) / T
            order = np.argsort(-x, kind="stable")
            if case["top_k"] > 0:
                order = order[:case["top_k"]]
            weight = np.exp(x[order])
            if p < 1:
                run_ = np.cumsum(weight)
                order = order[:int(np.searchsorted(run_, p * run_[-1])) + 1]
            order = np.sort(order[np.exp(x[order]) >= floor])
            run_ = np.cumsum(np.exp(x[order]))
            at = min(int(np.searchsorted(run_, u[b, i] * run_[-1], side="right")), len(order) - 1)
            logprob[b, i] = x[order[at]] - math.log(run_[-1])
    return {"accepted": None, "ids": None, "next": None, "committed": None, "logprob": torch.from_numpy(logprob)}


def _exact_append(s):
    if s["kn"].numel() > 40_000_000:
        return None
    out = {"flag": None}
    start, slots = s["start"].cpu().numpy(), s["slots"].cpu().numpy()
    for name, codes, scales, new in (("k", s["k"], s["ks"], s["kn"]), ("v", s["v"], s["vs"], s["vn"])):
        values = codes.view(torch.float8_e4m3fn).to(torch.float64)
        scales = scales.to(torch.float64).clone()
        for b in range(len(start) - 1):
            t = start[b]
            while t < start[b + 1]:
                page, at = divmod(int(slots[t]), PAGE)
                n = min(PAGE - at, int(start[b + 1] - t))
                x = new[:, :, b, t - start[b]:t - start[b] + n].to(torch.float64).transpose(2, 3)  # [R, L, H, n, D]
                e = torch.ceil(torch.log2(x.abs().amax((-1, -2)) / 448) - 1e-9).clamp(E_MIN, E_MAX)
                sc = torch.exp2(e)
                if at:
                    sc = torch.maximum(sc, scales[:, :, page])
                    values[:, :, page, :, :at] = _e4m3(values[:, :, page, :, :at]
                                                       * (scales[:, :, page] / sc)[..., None, None])
                values[:, :, page, :, at:at + n] = _e4m3(x / sc[..., None, None])
                scales[:, :, page] = sc
                t += n
        out[name], out[name + "_scale"] = values, scales
    return out


def _e4m3(x):
    """x rounded to 4 significant bits (no finer than 2^-9), halves to even, at most 448 in size."""
    _, e = torch.frexp(x)
    step = torch.exp2((e - 4).clamp(min=-9).double())
    return (torch.round(x / step) * step).clamp(-448, 448)


def _exact_attention(s):
    P, T = s["P"].cpu().numpy(), s["T"].cpu().numpy()
    B, Tmax, Hq, D = s["q"].shape
    H = s["kb"].shape[2]
    out = torch.zeros((B, Tmax, Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.full((B, Hq, Tmax), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(B):
        pages = s["table"][b, :-(-int(P[b]) // PAGE)].long()
        for h in range(H):
            k, v = ((c[pages, h].view(torch.float8_e4m3fn).double() * sc[pages, h].double()[:, None, None])
                    .reshape(-1, D)[:P[b]] for c, sc in ((s["k"][0, 0], s["ks"][0, 0]), (s["v"][1, 0], s["vs"][1, 0])))
            k = torch.cat([k, s["kb"][b, :T[b], h].double()])
            v = torch.cat([v, s["vb"][b, :T[b], h].double()])
            heads = slice(h * (Hq // H), (h + 1) * (Hq // H))
            a = torch.einsum("tgd,nd->gtn", s["q"][b, :T[b], heads].double(), k) / math.sqrt(D)
            j = torch.arange(k.shape[0], device="cuda")
            hidden = j[None, :] > P[b] + torch.arange(T[b], device="cuda")[:, None]
            a = a.masked_fill(hidden, -math.inf)
            lse[b, heads, :T[b]] = torch.logsumexp(a, -1)
            out[b, :T[b], heads] = torch.einsum("gtn,nd->tgd", torch.softmax(a, -1), v)
    return {"out": out, "lse": lse}
