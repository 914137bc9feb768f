"""Cases, inputs and plain forms of the operators around the paged 4-bit cache.

    rope       das_qk_norm_rope: norms of queries and keys per head, and their rotation by position
    append     das_kv_append_paged4: commit into the paged 4-bit cache
    attention  das_mature_v_attention_paged4: attention over that cache
    accept     das_speculative_accept: verification of proposals that were drawn from a drafter's distribution

With `own` false, run() computes an operator in elementary torch operations in 32 bits (angles in 64); with `own`
true it makes the library's calls on the same state.
"""
import math

import numpy as np
import torch

own = False

PAGE = 64                       # tokens per page
GROUP = 32                      # elements that share a scale
ONE = float(2 ** 32)            # weight of the most likely token
PART = float(2 ** 40)           # of a probability of 1 in the draw after a refusal


# ---- cases ---------------------------------------------------------------------------------------------------------

def listed():
    return [
        # the next token of one sequence: one row of queries, keys and values, the smallest call
        dict(name="rope single token", op="rope", batch=1, block=1, q_heads=32, kv_heads=32, head_dim=128, held=4096,
             rotary=128, interleaved=False, norm=True),
        # the verifier's candidates of 16 sequences, 4 to 16 each, half of every head rotated in neighbouring pairs
        dict(name="rope verify", op="rope", batch=16, block=16, q_heads=32, kv_heads=8, head_dim=128, held=8192,
             rotary=64, interleaved=True, norm=True),
        # prompts of odd lengths
        dict(name="rope prompt", op="rope", batch=4, block=2001, q_heads=32, kv_heads=8, head_dim=128, held=0,
             rotary=128, interleaved=False, norm=True),
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
        # 16 ragged sequences, blocks of 4 to 16, four query heads to a kv head
        dict(name="attention batched", op="attention", batch=16, q_heads=32, kv_heads=8, head_dim=128, lo=1024,
             hi=8192, block=16),
        # long prefixes, blocks of 16
        dict(name="attention long", op="attention", batch=4, q_heads=32, kv_heads=8, head_dim=128, lo=32768, hi=32768,
             block=16),
        # a drafted block of one sequence
        dict(name="accept one", op="accept", batch=1, width=8, vocab=32000, dtype="f32", temperature=0.8, top_k=0,
             top_p=0.95, min_p=0.0),
        # the verifier's 8 x 16 rows, every filter in use
        dict(name="accept verify", op="accept", batch=8, width=16, vocab=32000, dtype="f32", temperature=0.7, top_k=200,
             top_p=0.95, min_p=0.02),
        # a large vocabulary of odd size in bf16, whose rows start at any alignment
        dict(name="accept wide", op="accept", batch=8, width=8, vocab=128257, dtype="bf16", temperature=1.0, top_k=0,
             top_p=0.9, min_p=0.0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["rope", "append", "attention", "attention", "accept"])
    if op == "rope":
        head_dim, kv_heads, group = rng.choice([64, 128]), rng.choice([1, 2, 4, 8, 32]), rng.choice([1, 2, 4, 5, 8])
        batch = _log_int(rng, 1, 64)
        most = 49_000_000 // (batch * kv_heads * (group + 2) * head_dim)
        return dict(op=op, batch=batch, block=_log_int(rng, 1, max(1, min(8192, most))), q_heads=kv_heads * group,
                    kv_heads=kv_heads, head_dim=head_dim, held=_log_int(rng, 1, 1 << 20) - 1,
                    rotary=rng.choice([0, 16, 32, head_dim // 2, head_dim, head_dim]),
                    interleaved=rng.random() < 0.5, norm=rng.random() < 0.8)
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
                dtype=rng.choice(["f32", "bf16"]), temperature=rng.choice([0.0, 1.0, round(rng.uniform(0.3, 1.5), 3)]),
                top_k=rng.choice([0, 1, _log_int(rng, 2, 2000)]),
                top_p=rng.choice([1.0, round(rng.uniform(0.3, 0.999), 3)]),
                min_p=rng.choice([0.0, round(rng.uniform(0.001, 0.2), 4)]))


def work(case):
    op = case["op"]
    if op == "rope":
        rows = int(_blocks(case).sum())
        elements = rows * (case["q_heads"] + 2 * case["kv_heads"]) * case["head_dim"]
        return {"bytes": 4 * elements + 2 * case["rotary"] + 4 * case["head_dim"] + 8 * case["batch"],
                "flops": 8 * elements}
    if op == "append":
        n = int(_appended(case).sum())
        per = case["depths"] * case["layers"] * case["kv_heads"] * case["head_dim"] * 2
        return {"bytes": n * per * 2 + n * per // 2 + n * per // GROUP, "flops": n * per * 4}
    if op == "attention":
        P, T = _prefix_and_block(case)
        D, H, Hq = case["head_dim"], case["kv_heads"], case["q_heads"]
        rows = int(T.sum())
        return {"bytes": int(P.sum()) * H * (D + D // 16) + 4 * int((-(-P // PAGE)).sum())
                + rows * (Hq * (4 * D + 4) + H * D * 4),
                "flops": int((4 * T * Hq * D * (P + (T + 1) / 2)).sum())}
    n = case["batch"] * case["width"]
    return {"bytes": n * (2 * case["vocab"] * (4 if case["dtype"] == "f32" else 2) + 8) + case["batch"] * 32,
            "flops": 8 * n * case["vocab"]}


# ---- inputs --------------------------------------------------------------------------------------------------------

def _rng(case, salt):
    return np.random.default_rng([case["batch"], salt])


def _blocks(case):
    g = _rng(case, 1)
    B = case["batch"]
    return g.integers(max(1, case["block"] // 4), case["block"] + 1, B) if B > 1 else np.full(1, case["block"])


def _appended(case):
    g = _rng(case, 2)
    W = case["width"]
    return g.integers((W + 1) // 2, W + 1, case["batch"])


def _prefix_and_block(case):
    P = _rng(case, 3).integers(case["lo"], case["hi"] + 1, case["batch"])
    return P.astype(np.int64), _blocks(case).astype(np.int64)


def _i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _random_codes(shape, g):
    """Packed 4-bit codes of rounded normal values (1 to 15), two to a byte."""
    out = torch.empty(shape, dtype=torch.uint8, device="cuda")
    for d in range(shape[0]):
        for layer in range(shape[1]):
            lo, hi = (torch.randn(shape[2:], generator=g, device="cuda").mul_(2.6).round_().clamp_(-7, 7).add_(8)
                      .to(torch.uint8) for _ in range(2))
            out[d, layer] = lo | hi << 4
    return out


def _random_scales(shape, g):
    """Scales of 0.19 to 0.75, as bytes."""
    return torch.randint(100, 117, shape, generator=g, device="cuda", dtype=torch.uint8)


def _random_units(shape, g):
    """Powers of two, a half to two."""
    return torch.exp2(torch.randint(-1, 2, shape, generator=g, device="cuda").float())


def _cache(s, R, L, pages, H, D, g):
    s.update(k=_random_codes((R, L, pages, H, PAGE, D // 2), g), ks=_random_scales((R, L, pages, H, PAGE, D // GROUP), g),
             v=_random_codes((R, L, pages, H, PAGE // 8, D, 4), g),
             vs=_random_scales((R, L, pages, H, D // GROUP, PAGE), g),
             ku=_random_units((R, L, H), g), vu=_random_units((R, L, H), g))


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
    if op == "rope":
        B, T, H, Hq, D, rd = (case[x] for x in ("batch", "block", "kv_heads", "q_heads", "head_dim", "rotary"))
        rows = torch.randn((B, T, Hq + 2 * H, D), generator=g, device="cuda")      # a projection's rows, all heads
        rows *= torch.rand((1, 1, Hq + 2 * H, 1), generator=g, device="cuda") * 3 + 0.5
        rows = rows.to(torch.bfloat16)
        weight = lambda: (1 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(torch.bfloat16)
        s.update(q=rows[:, :, :Hq], k=rows[:, :, Hq:Hq + H], v=rows[:, :, Hq + H:], T=_i32(_blocks(case)),
                 P=_i32(host.integers(case["held"] // 2, case["held"] + 1, B)), qw=weight(), kw=weight(),
                 freq=(500000.0 ** (-torch.arange(0, rd, 2, device="cuda", dtype=torch.float64) / max(1, rd))).float(),
                 q_out=torch.zeros((B, T, Hq, D), dtype=torch.bfloat16, device="cuda"),
                 k_out=torch.zeros((B, T, H, D), dtype=torch.bfloat16, device="cuda"),
                 v_out=torch.zeros((B, T, H, D), dtype=torch.bfloat16, device="cuda"))
    elif op == "append":
        B, W, R, L, H, D = (case[x] for x in ("batch", "width", "depths", "layers", "kv_heads", "head_dim"))
        n = _appended(case)
        first = (case["held"] % PAGE + np.arange(B) * 7) % PAGE if case["held"] else np.zeros(B, dtype=np.int64)
        touched = -(-(first + n) // PAGE)                                            # pages of each request's new tokens
        pages = int(touched.sum())
        ids = host.permutation(pages)
        at = np.concatenate([[0], np.cumsum(touched)])
        slots = np.concatenate([ids[at[b] + (first[b] + np.arange(n[b])) // PAGE] * PAGE
                                + (first[b] + np.arange(n[b])) % PAGE for b in range(B)])
        _cache(s, R, L, pages, H, D, g)
        s.update(slots=_i32(slots), start=_i32(np.concatenate([[0], np.cumsum(n)])), flag=_i32([0]),
                 kn=torch.empty((R, L, B, W, H, D), dtype=torch.bfloat16, device="cuda"),
                 vn=torch.empty((R, L, B, W, H, D), dtype=torch.bfloat16, device="cuda"))
        for d in range(R):
            s["kn"][d] = torch.randn((L, B, W, H, D), generator=g, device="cuda")
            s["vn"][d] = torch.randn((L, B, W, H, D), generator=g, device="cuda") * 2
    elif op == "attention":
        B, H, Hq, D, T = (case[x] for x in ("batch", "kv_heads", "q_heads", "head_dim", "block"))
        P, Tb = _prefix_and_block(case)
        need = -(-P // PAGE)
        rows, pages = max(1, int(need.max())), max(1, int(need.sum()))
        table = host.integers(0, pages, (B, rows))
        used = np.arange(rows)[None, :] < need[:, None]
        table[used] = host.permutation(pages)[:used.sum()]
        _cache(s, 2, 1, pages, H, D, g)
        bf = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)
        s.update(table=_i32(table), P=_i32(P), T=_i32(Tb), q=bf(B, T, Hq, D), kb=bf(B, T, H, D), vb=bf(B, T, H, D))
    else:
        B, W, V = case["batch"], case["width"], case["vocab"]
        dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        target = 2 * torch.randn((B, W, V), generator=g, device="cuda")
        drafter = target + 0.5 * torch.randn((B, W, V), generator=g, device="cuda")  # a shallower look at the same text
        full = lambda x, dt=torch.float32: torch.full((B,), x, dtype=dt, device="cuda")
        uniform = lambda *shape: torch.rand(shape, generator=g, device="cuda")
        s.update(target=target.to(dtype), drafter=drafter.to(dtype), u=uniform(B, W), again=uniform(B),
                 temperature=full(case["temperature"]), top_k=full(case["top_k"], torch.int32),
                 top_p=full(case["top_p"]), min_p=full(case["min_p"]))
        _, w, total = _truncated(s, s["drafter"])
        s["ids"] = _drawn(w, total, uniform(B, W))
    if das is not None and op in ("append", "attention"):
        s["cache"] = das.PagedKVCache4(s["k"], s["v"], s["ks"], s["vs"], s["ku"], s["vu"])
        if op == "attention":
            s["ws"] = das.new_workspace_paged4(s["cache"], case["batch"], case["q_heads"], case["block"])
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------

def run(s):
    return {"rope": _run_rope, "append": _run_append, "attention": _run_attention, "accept": _run_accept}[s["op"]](s)


def _run_rope(s):
    das = _library()
    eps = 1e-6 if s["case"]["norm"] else None
    if das is not None:
        q, k, v = das.das_qk_norm_rope(s["q"], s["k"], s["v"], s["freq"], s["P"], s["T"], q_weight=s["qw"],
                                       k_weight=s["kw"], eps=eps, interleaved=s["case"]["interleaved"],
                                       q_out=s["q_out"], k_out=s["k_out"], v_out=s["v_out"])
    else:
        live = (torch.arange(s["q"].shape[1], device="cuda") < s["T"][:, None])[:, :, None, None]
        q = torch.where(live, _norm_rope(s, s["q"], s["qw"], eps), s["q_out"])
        k = torch.where(live, _norm_rope(s, s["k"], s["kw"], eps), s["k_out"])
        v = torch.where(live, s["v"], s["v_out"])
    return {"q": q, "k": k, "v": v}


def _norm_rope(s, x, weight, eps):
    x = x.float()
    if eps is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps) * weight.float()
    rd = s["case"]["rotary"]
    place = s["P"][:, None] + torch.arange(x.shape[1], device=x.device)
    angle = torch.remainder(place[..., None].double() * s["freq"].double(), 2 * math.pi).float()[:, :, None]
    cos, sin = torch.cos(angle), torch.sin(angle)
    turned, rest = x[..., :rd], x[..., rd:]
    if s["case"]["interleaved"]:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = turned[..., :rd // 2], turned[..., rd // 2:]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, rest), -1).to(torch.bfloat16)


def _run_append(s):
    das = _library()
    if das is not None:
        das.das_kv_append_paged4(s["cache"], s["kn"], s["vn"], s["slots"], s["start"], s["flag"])
    else:
        _append(s)
    # (the codes as they are packed: whole numbers)
    return {"k": s["k"], "v": s["v"], "k_scale": s["ks"], "v_scale": s["vs"], "flag": s["flag"]}


def _append(s):
    R, L, B, W, H, D = s["kn"].shape
    start, slots = s["start"].long(), s["slots"].long()
    new = torch.arange(slots.numel(), device=slots.device)
    b = torch.bucketize(new, start[1:], right=True)
    page, place = slots // PAGE, slots % PAGE
    codes, scales = _quantised(s["kn"][:, :, b, new - start[b]], s["ku"])           # [R, L, tokens, H, D]
    s["k"][:, :, page, :, place] = (codes[..., 0::2] | codes[..., 1::2] << 4).permute(2, 0, 1, 3, 4)
    s["ks"][:, :, page, :, place] = scales.permute(2, 0, 1, 3, 4)
    codes, scales = _quantised(s["vn"][:, :, b, new - start[b]], s["vu"])
    s["vs"][:, :, page, :, :, place] = scales.permute(2, 0, 1, 3, 4)
    # a byte holds two tokens: the even places first, then the odd ones
    for odd in (0, 1):
        pick = (place % 2 == odd).nonzero()[:, 0]
        at = (slice(None), slice(None), page[pick], slice(None), place[pick] // 8, slice(None), place[pick] % 8 // 2)
        s["v"][at] = s["v"][at] & (15 << 4 * (1 - odd)) | codes[:, :, pick].permute(2, 0, 1, 3, 4) << 4 * odd


def _quantised(x, unit):
    """Codes and scale bytes of values [R, L, tokens, H, D]: a scale to 32, four significant bits of amax / 7."""
    shape = x.shape
    x = (x.float() / unit[:, :, None, :, None]).unflatten(-1, (-1, GROUP))
    nan = x.isnan().any(-1)
    amax = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1)
    m, e = torch.frexp(amax / 7)                                                   # m 2^e, m in [0.5, 1)
    step = torch.exp2((e - 4).clamp(min=-17).float())                              # of four bits; none below 2^-17
    scale = ((amax / 7 / step).round() * step).clamp(max=60.0)
    code = (x / torch.where(scale > 0, scale, 1.0)[..., None]).nan_to_num().round().clamp(-7, 7)
    code = torch.where(scale[..., None] > 0, code, 0.0).to(torch.int32) + 8
    byte = scale.to(torch.float16).view(torch.int16) >> 7                          # sign 0, five bits, three bits
    byte = torch.where(nan, 255, byte)
    return code.to(torch.uint8).view(shape), byte.to(torch.uint8)


def _scale(byte):
    return (byte.to(torch.int16) << 7).view(torch.float16).float()


def _keys(codes, scales, unit):
    """Values [..., H, 64, D] of packed codes [..., H, 64, D / 2]."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float() - 8
    return (c.unflatten(-1, (-1, GROUP)) * _scale(scales)[..., None]).flatten(-2) * unit[:, None, None]


def _values(codes, scales, unit):
    """Values [..., H, 64, D] of packed codes [..., H, 8, D, 4]."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float() - 8          # [..., 8, D, 8]
    c = c.transpose(-1, -2).flatten(-3, -2).unflatten(-1, (-1, GROUP))             # [..., 64, D / 32, 32]
    return (c * _scale(scales).transpose(-1, -2)[..., None]).flatten(-2) * unit[:, None, None]


def _run_attention(s):
    das = _library()
    if das is not None:
        out, lse = das.das_mature_v_attention_paged4(s["cache"], 0, 1, 2, s["table"], s["P"], s["T"], s["q"], s["kb"],
                                                     s["vb"], s["ws"])
    else:
        out, lse = _attention(s)
    return {"out": out, "lse": lse}


def _attention(s):
    B, T, Hq, D = s["q"].shape
    H = s["kb"].shape[2]
    table = s["table"].long()
    flat = lambda x: x.transpose(1, 2).reshape(B, H, -1, D)
    k = flat(_keys(s["k"][0, 0][table], s["ks"][0, 0][table], s["ku"][0, 0]))               # [B, H, N, D]
    v = flat(_values(s["v"][1, 0][table], s["vs"][1, 0][table], s["vu"][1, 0]))
    seen = (torch.arange(k.shape[2], device=k.device) < s["P"][:, None])[:, None, None, :]    # [B, 1, 1, N]
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


def _run_accept(s):
    das = _library()
    if das is not None:
        accepted, token, committed = das.das_speculative_accept(
            s["target"], s["drafter"], s["ids"], s["u"], s["again"], temperature=s["temperature"], top_k=s["top_k"],
            top_p=s["top_p"], min_p=s["min_p"])
    else:
        accepted, token, committed = _accept(s)
    return {"accepted": accepted, "next": token, "committed": committed}


def _truncated(s, logits):
    """What temperature, top-k, top-p and min-p leave of each row: e = exp((l - m) / T) in binary32, 0 where a token is
    left out; the whole numbers round(e 2^32); and their sum."""
    z = logits.float() + 0.0                                               # -0 counts as 0
    each = lambda name: s[name][:, None, None]
    T, k, p, floor = each("temperature"), each("top_k").long(), each("top_p"), each("min_p")
    k = torch.where(T > 0, k, 1)
    T = torch.where(T > 0, T, 1.0)
    z, order = torch.sort(z, dim=-1, descending=True, stable=True)
    e = torch.where(z == z[..., :1], 1.0, torch.exp((z - z[..., :1]) / T))
    w = (e.double() * ONE).round().long()                                  # whole numbers: sums do not depend on order
    kept = (k <= 0) | (torch.arange(z.shape[-1], device=z.device) < k)
    w = torch.where(kept, w, 0)
    before = w.cumsum(-1) - w
    least = torch.ceil(p.double() * w.sum(-1, keepdim=True).double()).long().clamp(min=1)
    kept = kept & ((p >= 1) | (before < least)) & (e >= floor.clamp(max=1.0))
    w, e = torch.where(kept, w, 0), torch.where(kept, e, 0.0)
    total = w.sum(-1, keepdim=True)
    by_index = lambda x: torch.zeros_like(x).scatter_(-1, order, x)
    return by_index(e), by_index(w), total


def _drawn(w, total, u):
    """The least index up to which the weights sum to more than floor(u total)."""
    r = torch.minimum((u.double()[..., None] * total.double()).floor().long(), total - 1)
    return (w.cumsum(-1) <= r).sum(-1).int()


def _accept(s):
    W = s["ids"].shape[1]
    e, w, total = _truncated(s, s["target"])
    p = e * (1 / (total.double() / ONE).float())                           # probabilities, in binary32
    e, _, q_total = _truncated(s, s["drafter"])
    q = e * (1 / (q_total.double() / ONE).float())
    at = s["ids"].long()[..., None]
    taken = s["u"].double() * q.gather(-1, at)[..., 0].double() < p.gather(-1, at)[..., 0].double()
    accepted = taken.int().cumprod(1).sum(1)
    row = accepted.clamp(max=W - 1)[:, None, None]                         # the first refused proposal's
    pick = lambda x: x.gather(1, row.expand(-1, 1, x.shape[-1]))[:, 0]
    rest = ((pick(p) - pick(q)).clamp(min=0).double() * PART).round().long()
    some = rest.sum(-1, keepdim=True)
    rest = torch.where(some > 0, rest, pick(w))                            # nothing left by rounding: the target's own
    drawn = _drawn(rest, rest.sum(-1, keepdim=True), s["again"])
    token = torch.where(accepted < W, drawn, s["ids"][:, -1])
    return accepted.int(), token, (accepted + 1).clamp(max=W).int()


# ---- in 64 bits ----------------------------------------------------------------------------------------------------

def exact(case, seed):
    if case["op"] not in ("rope", "attention"):
        return None                                                        # whole numbers alone
    s = prepare(case, seed)
    return _exact_rope(s) if s["op"] == "rope" else _exact_attention(s)


def _exact_rope(s):
    case = s["case"]
    rd, half = case["rotary"], case["rotary"] // 2
    out = {"v": s["v"].double().clone()}
    n = s["P"].double()[:, None] + torch.arange(case["block"], device="cuda", dtype=torch.float64)
    for name, weight in (("q", s["qw"]), ("k", s["kw"])):
        x = s[name].double().clone()
        if case["norm"]:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + 1e-6) * weight.double()
        for j in range(half):
            a, b = (2 * j, 2 * j + 1) if case["interleaved"] else (j, j + half)
            turn = torch.polar(torch.ones_like(n), n * s["freq"][j].double())[..., None]
            z = torch.complex(x[..., a], x[..., b]) * turn
            x[..., a], x[..., b] = z.real, z.imag
        out[name] = x
    for b, t in enumerate(s["T"].tolist()):
        for x in out.values():
            x[b, t:] = 0                                                   # as the rows were
    return {name: out[name] for name in ("q", "k", "v")}


def _exact_attention(s):
    P, T = s["P"].cpu().numpy(), s["T"].cpu().numpy()
    B, Tmax, Hq, D = s["q"].shape
    H = s["kb"].shape[2]
    out = torch.zeros((B, Tmax, Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.full((B, Hq, Tmax), -math.inf, dtype=torch.float64, device="cuda")
    byte = torch.arange(256, device="cuda")
    size = torch.where(byte < 8, byte.double() * 2.0 ** -17, (8 + byte % 8).double() * torch.exp2((byte // 8 - 18).double()))
    for b in range(B):
        pages = s["table"][b, :-(-int(P[b]) // PAGE)].long()
        for h in range(H):
            c = s["k"][0, 0][pages, h].reshape(-1, D // 2)[:P[b]]
            k = torch.empty((int(P[b]), D), dtype=torch.float64, device="cuda")
            k[:, 0::2], k[:, 1::2] = (c % 16).double() - 8, (c // 16).double() - 8
            sk = size[s["ks"][0, 0][pages, h].reshape(-1, D // GROUP)[:P[b]].long()]
            c = s["v"][1, 0][pages, h]                                     # [pages, 8, D, 4]
            v = torch.empty((len(pages), 8, 8, D), dtype=torch.float64, device="cuda")
            v[:, :, 0::2] = (c % 16).double().transpose(2, 3) - 8
            v[:, :, 1::2] = (c // 16).double().transpose(2, 3) - 8
            v = v.reshape(-1, D)[:P[b]]
            sv = size[s["vs"][1, 0][pages, h].transpose(1, 2).reshape(-1, D // GROUP)[:P[b]].long()]
            k = k * sk.repeat_interleave(GROUP, 1) * s["ku"][0, 0, h].double()
            v = v * sv.repeat_interleave(GROUP, 1) * s["vu"][1, 0, h].double()
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
