"""What a fitted block is served with, as cases that can be timed and checked one by one.

A block whose weights have been quantised (codes and one scale per output channel) is run on new
tokens by four calls: the joint projection in 8-bit integers (jab_quantized_linear), the rotation of
Q and K with the quantising write of K and V into a paged cache (jab_kv_write), attention over the
quantised pages (jab_kv_attention), and the read-back of cached tokens (jab_kv_read). The blocks are
those of `workloads/` (GPT-2 small and Mistral-7B shapes) and small generic ones that reach the other
head ratios.

listed() and draw(rng) give cases, prepare(case, seed) the inputs, run(state) one pass, work(case) the
bytes and operations that the pass cannot do without, exact(case, seed) the outputs in 64 bits. With
`own` false run() computes the operators by elementary torch operations in 32 bits.

Cache layout (the one of the public header): codes [pages, KV heads, tokens of a page, head_dim * bits
/ 8] as bytes, code + 128 for 8 bits; for 4 bits code + 8, element 2i in the low half of byte i and
2i + 1 in the high half. Scales fp32 [pages, KV heads, tokens of a page]. A code is
clip(rint(fl32(x / s)), -qmax, qmax) with s = fl32(max|x| / qmax), both roundings part of the definition.
"""
import math

import torch

own = False

#           d_model, query heads, KV heads, head_dim, RoPE theta (0: none)
BLOCKS = {
    "gpt2": (768, 12, 12, 64, 0.0),
    "mistral": (4096, 32, 8, 128, 10000.0),
    "gqa2": (512, 4, 2, 128, 10000.0),
    "gqa4_dh64": (256, 4, 1, 64, 500.0),
    "gqa3": (1024, 12, 4, 128, 10000.0),
}
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _linear(name, block, M, bits, x, y):
    return {"name": name, "kind": "linear", "block": block, "M": M, "bits": bits, "x": x, "y": y}


def _cache(name, block, B, T, start, bits, page, x, y):
    return {"name": name, "kind": "cache", "block": block, "B": B, "T": T, "start": start, "bits": bits,
            "page": page, "x": x, "y": y}


def _attn(name, block, B, q, shortest, longest, shared, window, bits, page, x):
    return {"name": name, "kind": "attention", "block": block, "B": B, "q": q, "shortest": shortest,
            "longest": longest, "shared": shared, "window": window, "bits": bits, "page": page, "x": x}


def listed():
    return [
        # the projection of one new token: the weights are read for a single row
        _linear("linear_mistral_1", "mistral", 1, 8, "bf16", "bf16"),
        # a few dozen tokens of a small block at 3 bits, an odd number of rows: launches and latency
        _linear("linear_gpt2_37", "gpt2", 37, 3, "fp16", "fp32"),
        # a decoding step of 64 sequences
        _linear("linear_mistral_64", "mistral", 64, 4, "bf16", "fp16"),
        # prompts of 8192 tokens in all: the largest product
        _linear("linear_mistral_8192", "mistral", 8192, 8, "bf16", "bf16"),
        # a decoding step of 64 sequences: one token each is rotated, quantised, written and read back
        _cache("cache_mistral_64x1", "mistral", 64, 1, 1027, 8, 64, "fp16", "fp16"),
        # three ragged-length prompts in 4 bits, pages that end inside the prompt
        _cache("cache_gpt2_3x1001", "gpt2", 3, 1001, 0, 4, 16, "bf16", "fp32"),
        # prompts of 2048 tokens: written, and read back for a consumer that wants 16-bit keys and values
        _cache("cache_mistral_8x2048", "mistral", 8, 2048, 0, 8, 64, "fp16", "bf16"),
        # a single sequence of a small block, one token: latency
        _attn("attn_gpt2_1x1000", "gpt2", 1, 1, 1000, 1000, 0, 0, 8, 16, "fp16"),
        # a decoding step of 64 sequences of all lengths
        _attn("attn_mistral_64x8192", "mistral", 64, 1, 300, 8192, 0, 0, 8, 64, "bf16"),
        # a few long contexts in 4 bits
        _attn("attn_mistral_4x65536", "mistral", 4, 1, 40001, 65536, 0, 0, 4, 128, "fp16"),
        # 64 sequences behind one prompt of 8192 tokens, each with up to 700 tokens of its own
        _attn("attn_mistral_prefix8192", "mistral", 64, 1, 8193, 8892, 8192, 0, 8, 64, "bf16"),
        # two prompts taken in chunks of 512 tokens, in the sliding window of 4096
        _attn("attn_mistral_chunk512", "mistral", 2, 512, 4100, 6000, 0, 4096, 8, 64, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / 1e15)


def draw(rng):
    kind = rng.choice(("linear", "linear", "cache", "attention", "attention", "attention"))
    most = max(_cost(c) for c in listed() if c["kind"] == kind)
    while True:
        block = rng.choice(("gpt2", "mistral", "mistral", "gqa2", "gqa3", "gqa4_dh64"))
        x = rng.choice(("bf16", "fp16"))
        if kind == "linear":
            case = _linear("", block, _log_int(rng, 1, 8192), rng.choice((2, 3, 4, 8, 8)), x,
                           rng.choice(("bf16", "fp16", "fp32")))
        elif kind == "cache":
            T = _log_int(rng, 1, 4096)
            case = _cache("", block, _log_int(rng, 1, max(1, min(128, 16384 // T))), T, rng.choice((0, 0, _log_int(rng, 1, 4000))),
                          rng.choice((4, 8)), rng.choice((16, 32, 64, 128)), x, rng.choice(("bf16", "fp16", "fp32")))
        else:
            q = rng.choice((1, 1, 1, 2, 4, 7, _log_int(rng, 8, 512)))
            longest = max(q, _log_int(rng, 1, 65536))
            B = _log_int(rng, 1, 128)
            page = rng.choice((16, 32, 64, 128))
            shared = longest // rng.choice((2, 4)) // page * page if rng.random() < 0.3 else 0
            case = _attn("", block, B, q, max(1, shared, int(longest * rng.uniform(0.05, 1.0))), longest, shared,
                         rng.choice((0, 0, 0, 1024, 4096)), rng.choice((4, 8)), page, x)
            d, hq, hkv, dh, _ = BLOCKS[block]
            # the plain form holds every sequence at the longest's length, in 32 bits, and all of its scores
            if B * longest * hkv * dh > 64 * 8192 * 1024 or B * q * hq * longest > 2 ** 28:
                continue
        del case["name"]
        if 3072 not in case.values() and _cost(case) <= most:
            return case


# ------------------------------------------------------------------ sizes
def _lens(case):
    """Keys of each sequence, the new tokens among them: spread over the logarithm, in mixed order."""
    B, lo, hi = case["B"], case["shortest"], case["longest"]
    if B == 1:
        return [hi]
    v = [int(round(lo * (hi / lo) ** (i / (B - 1)))) for i in range(B)]
    return [v[(i * 37) % B] if B % 37 else v[i] for i in range(B)]


def _visible(case):
    """(pairs of a query and a key that it sees, keys that any query sees, the shared ones counted once)."""
    q, w, shared = case["q"], case["window"], case["shared"]
    pairs, keys, first = 0, 0, shared
    for n in _lens(case):
        for p in range(n - q, n):
            pairs += max(0, min(p + 1, w) if w else p + 1)
        lo = max(0, n - q + 1 - w) if w else 0
        keys += max(0, n - max(lo, shared))
        first = min(first, lo)
    return pairs, keys + shared - first


def work(case):
    d, hq, hkv, dh, _ = BLOCKS[case["block"]]
    D = (hq + 2 * hkv) * dh
    if case["kind"] == "linear":
        M, out = case["M"], 4 if case["y"] == "fp32" else 2
        return {"bytes": M * d * 2 + D * d + D * 4 + M * D * out, "flops": 2 * M * D * d}
    row = dh * case["bits"] // 8 + 4
    if case["kind"] == "cache":
        N, out = case["B"] * case["T"], 4 if case["y"] == "fp32" else 2
        # the joint rows in, Q out, the pages written and read once, K and V out, slots, positions and table rows
        return {"bytes": N * D * 2 + N * hq * dh * 2 + 2 * (2 * N * hkv * row) + 2 * N * hkv * dh * out + N * 12
                + (N * dh * 4 if BLOCKS[case["block"]][4] else 0), "flops": 6 * N * D}
    pairs, keys = _visible(case)
    N = case["B"] * case["q"]
    return {"bytes": keys * hkv * 2 * row + N * hq * (dh * 4 + 4), "flops": 4 * dh * hq * pairs}


# ------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _activations(g, n, d):
    """Rows of N(0, 1) with 1 % of the channels ten times as large."""
    x = torch.randn((n, d), generator=g, device="cuda")
    x[:, torch.randperm(d, generator=g, device="cuda")[: d // 100 + 1]] *= 10
    return x


def _rope_table(case, length):
    dh, theta = BLOCKS[case["block"]][3:]
    if not theta:
        return None
    j = torch.arange(dh // 2, device="cuda", dtype=torch.float64)
    a = torch.arange(length, device="cuda", dtype=torch.float64)[:, None] * theta ** (-2 * j / dh)
    return a.cos().float().contiguous(), a.sin().float().contiguous()


def _fp32(x, bits):
    """(whole-numbered codes in fp32, scales) of rows of fp32 values."""
    qmax = 2 ** (bits - 1) - 1
    # divided on the device: torch turns a division by a host number into a product with its reciprocal
    s = x.abs().amax(-1) / torch.full((), float(qmax), device=x.device)
    c = torch.round(x / s[..., None]).clamp(-qmax, qmax)
    return torch.where(s[..., None] > 0, c, torch.zeros_like(c)), s


def _pack(codes, bits):
    if bits == 8:
        return (codes + 128).to(torch.uint8)
    u = (codes + 8).to(torch.uint8)
    return u[..., 0::2] | (u[..., 1::2] << 4)


def _unpack(b, bits, dtype):
    if bits == 8:
        return b.to(dtype) - 128
    return torch.stack((b & 15, b >> 4), -1).flatten(-2).to(dtype) - 8


def _tables(case, g, lens):
    """Page numbers of every sequence, int32 [B, pages of the longest], in no order; the shared pages of a
    prefix are the same in each row; the number of pages of the cache."""
    page = case["page"]
    width = max(1, -(-max(lens) // page))
    same = case.get("shared", 0) // page
    own_pages = [max(0, -(-n // page) - same) for n in lens]
    total = same + sum(own_pages) + 3
    ids = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros((len(lens), width), dtype=torch.int32, device="cuda")
    table[:, :same] = ids[:same]
    at = same
    for b, n in enumerate(own_pages):
        table[b, same : same + n] = ids[at : at + n]
        at += n
    return table, total


def prepare(case, seed):
    g = _generator(seed)
    d, hq, hkv, dh, theta = BLOCKS[case["block"]]
    D = (hq + 2 * hkv) * dh
    s = {"case": case, "hq": hq, "hkv": hkv, "dh": dh}
    i32 = dict(dtype=torch.int32, device="cuda")
    if case["kind"] == "linear":
        M = case["M"]
        s["x"] = _activations(g, M, d).to(DTYPES[case["x"]])
        codes, s["w_scales"] = _fp32(torch.randn((D, d), generator=g, device="cuda") * 0.02, case["bits"])
        s["codes"] = codes.to(torch.int8)
        if own:
            import paper_2609_34866_gb300 as J
            s["y"] = torch.empty((M, D), dtype=DTYPES[case["y"]], device="cuda")
            s["ws"] = torch.empty(J.jab_quantized_linear_workspace_size(M, D, d), dtype=torch.uint8, device="cuda")
        return s
    bits, page, B = case["bits"], case["page"], case["B"]
    if case["kind"] == "cache":
        T, start = case["T"], case["start"]
        s["pages"], n_pages = _tables(case, g, [start + T] * B)
        s["qkv"] = _activations(g, B * T, D).to(DTYPES[case["x"]])
        pos = torch.arange(start, start + T, device="cuda").repeat(B)
        row = torch.arange(B, device="cuda").repeat_interleave(T)
        s["slots"] = s["pages"][row, pos // page].long() * page + pos % page
        s["positions"] = pos.int()
        s["rope"] = _rope_table(case, start + T)
        s["starts"], s["counts"] = torch.full((B,), start, **i32), torch.full((B,), T, **i32)
        if own:
            import paper_2609_34866_gb300 as J
            s["cache"] = J.KvCache(hkv, dh, bits, page, n_pages)
            s["q"] = torch.empty((B * T, hq * dh), dtype=DTYPES[case["x"]], device="cuda")
            s["k"], s["v"] = (torch.empty((B, T, hkv, dh), dtype=DTYPES[case["y"]], device="cuda") for _ in range(2))
        return s
    q, lens = case["q"], _lens(case)
    s["pages"], n_pages = _tables(case, g, lens)
    for name in ("k", "v"):
        codes = torch.empty((n_pages, hkv, page, dh * bits // 8), dtype=torch.uint8, device="cuda")
        scales = torch.empty((n_pages, hkv, page), device="cuda")
        for lo in range(0, n_pages, 1024):
            n = min(1024, n_pages - lo)
            x = _activations(g, n * hkv * page, dh) * (0.5 if name == "k" else 1.0)
            c, sc = _fp32(x, bits)
            codes[lo : lo + n] = _pack(c, bits).view(n, hkv, page, -1)
            scales[lo : lo + n] = sc.view(n, hkv, page)
        s[name + "_codes"], s[name + "_scales"] = codes, scales
    s["q"] = (2 * torch.randn((B * q, hq, dh), generator=g, device="cuda")).to(DTYPES[case["x"]])
    s["lens"] = torch.tensor(lens, **i32)
    s["q_start"] = torch.arange(0, B * q + 1, q, **i32)
    if own:
        import paper_2609_34866_gb300 as J
        s["cache"] = J.KvCache(hkv, dh, bits, page, n_pages, k_codes=s["k_codes"], v_codes=s["v_codes"],
                               k_scales=s["k_scales"], v_scales=s["v_scales"])
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((B * q, hq), device="cuda")
        s["ws"] = torch.empty(J.jab_kv_attention_workspace_size(s["cache"], B, B * q, hq, q, case["longest"],
                                                                case["shared"]), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    return _compute(s, case, torch.float32)


def _run_own(s, case):
    import paper_2609_34866_gb300 as J
    if case["kind"] == "linear":
        J.jab_quantized_linear(s["x"], s["codes"], s["w_scales"], s["y"], s["ws"])
        return s["y"]
    if case["kind"] == "cache":
        J.jab_kv_write(s["cache"], s["qkv"], s["hq"], s["slots"], q_out=s["q"], positions=s["positions"], rope=s["rope"])
        J.jab_kv_read(s["cache"], s["pages"], s["counts"], s["k"], s["v"], starts=s["starts"])
        return {"q": s["q"], "k": s["k"], "v": s["v"]}
    J.jab_kv_attention(s["cache"], s["q"], s["q_start"], s["pages"], s["lens"], s["out"], s["ws"], max_q_len=case["q"],
                       max_seq_len=case["longest"], shared_len=case["shared"], window=case["window"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def _compute(s, case, dt):
    hq, hkv, dh = s["hq"], s["hkv"], s["dh"]
    if case["kind"] == "linear":
        codes, scales = _fp32(s["x"].to(torch.float32), 8)
        y = codes.to(dt) @ s["codes"].to(dt).t()
        return (y * scales.to(dt)[:, None] * s["w_scales"].to(dt)).to(DTYPES[case["y"]])
    if case["kind"] == "cache":
        B, T = case["B"], case["T"]
        x = s["qkv"].to(dt).view(B * T, hq + 2 * hkv, dh)
        turned = x[:, : hq + hkv]
        if s["rope"] is not None:
            cos, sin = (t.to(dt)[s["positions"].long()][:, None] for t in s["rope"])
            a, b = turned[..., : dh // 2], turned[..., dh // 2 :]
            turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
        k, v = (c * sc[..., None] for c, sc in (_fp32(t, case["bits"]) for t in (turned[:, hq:], x[:, hq + hkv :])))
        y = DTYPES[case["y"]]
        return {"q": turned[:, :hq].reshape(B * T, hq * dh).to(s["qkv"].dtype), "k": k.view(B, T, hkv, dh).to(y),
                "v": v.reshape(B, T, hkv, dh).to(y)}
    B, q, page, bits = case["B"], case["q"], case["page"], case["bits"]
    pages = s["pages"].long()
    L = pages.shape[1] * page
    k, v = (((_unpack(s[n + "_codes"][pages], bits, dt) * s[n + "_scales"][pages].to(dt)[..., None])
             .transpose(2, 3).reshape(B, L, hkv, dh)).permute(0, 2, 1, 3) for n in ("k", "v"))
    x = s["q"].to(dt).view(B, q, hkv, hq // hkv, dh).permute(0, 2, 3, 1, 4).reshape(B, hkv, -1, dh)
    sc = (x @ k.transpose(-1, -2)) * (1.0 / math.sqrt(dh))
    pos = (s["lens"].long()[:, None] - q + torch.arange(q, device="cuda")).repeat(1, hq // hkv)[:, None, :, None]
    key = torch.arange(L, device="cuda")
    seen = key <= pos
    if case["window"]:
        seen = seen & (key > pos - case["window"])
    sc = torch.where(seen, sc, torch.full((), -math.inf, dtype=dt, device="cuda"))
    m = sc.amax(-1, keepdim=True)
    m = torch.where(m > -math.inf, m, torch.zeros_like(m))
    p = torch.exp(sc - m)
    del sc
    l = p.sum(-1, keepdim=True)
    o = (p @ v) / torch.where(l > 0, l, torch.ones_like(l))
    back = lambda t: t.view(B, hkv, hq // hkv, q, -1).permute(0, 3, 1, 2, 4).reshape(B * q, hq, -1)  # noqa: E731
    return {"out": back(o).to(s["q"].dtype), "lse": back(m + torch.log(l))[..., 0].float()}


# ------------------------------------------------------------------ 64 bits
def _exact_codes(x, bits):
    """Codes and scales of fp64 rows; the scale and the quotient are rounded to 32 bits by definition."""
    qmax = 2 ** (bits - 1) - 1
    s = (x.abs().amax(-1) / torch.full((), qmax, dtype=torch.float64, device="cuda")).float()
    v = (x / s.double()[..., None]).float().double()
    c = torch.nan_to_num(torch.round(v), nan=0.0, posinf=qmax, neginf=-qmax).clamp(-qmax, qmax)
    return torch.where(s.double()[..., None] == 0, torch.zeros_like(c), c), s.double()


def exact(case, seed):
    s = prepare(case, seed)
    d, hq, hkv, dh, theta = BLOCKS[case["block"]]
    if case["kind"] == "linear":
        c, sx = _exact_codes(s["x"].double(), 8)
        return torch.einsum("mk,nk->mn", c, s["codes"].double()) * (sx[:, None] * s["w_scales"].double()[None, :])
    if case["kind"] == "cache":
        B, T = case["B"], case["T"]
        x = s["qkv"].double().reshape(B * T, hq + 2 * hkv, dh)
        qk, v = x[:, : hq + hkv], x[:, hq + hkv :]
        if theta:
            cos, sin = (t.double()[s["positions"].long()] for t in s["rope"])
            z = torch.complex(qk[..., : dh // 2], qk[..., dh // 2 :]) * torch.complex(cos, sin)[:, None]
            qk = torch.cat((z.real, z.imag), -1)
        kc, ks = _exact_codes(qk[:, hq:], case["bits"])
        vc, vs = _exact_codes(v, case["bits"])
        return {"q": qk[:, :hq].reshape(B * T, hq * dh), "k": (kc * ks[..., None]).reshape(B, T, hkv, dh),
                "v": (vc * vs[..., None]).reshape(B, T, hkv, dh)}
    q, page, bits, w = case["q"], case["page"], case["bits"], case["window"]
    outs, lses = [], []
    for b, n in enumerate(_lens(case)):
        at = torch.arange(n, device="cuda")
        ids = s["pages"][b].long()[at // page]
        kv = []
        for name in ("k", "v"):
            raw = s[name + "_codes"][ids, :, at % page].long()
            if bits == 4:
                raw = torch.stack((raw % 16, raw // 16), -1).reshape(n, hkv, dh)
            kv.append((raw.double() - 2 ** (bits - 1)) * s[name + "_scales"][ids, :, at % page].double()[..., None])
        x = s["q"][b * q : (b + 1) * q].double()
        i = torch.arange(n - q, n, device="cuda")[:, None]
        hidden = (at[None] > i) | ((at[None] <= i - w) if w else torch.zeros_like(at[None] > i))
        o, l = [], []
        for h in range(hq):
            t = (x[:, h] @ kv[0][:, h // (hq // hkv)].t() / math.sqrt(dh)).masked_fill(hidden, -math.inf)
            l.append(torch.logsumexp(t, -1))
            e = torch.where(hidden, torch.zeros_like(t), torch.exp(t - torch.where(l[-1] > -math.inf, l[-1], 0.0)[:, None]))
            o.append(e @ kv[1][:, h // (hq // hkv)])
        outs.append(torch.stack(o, 1))
        lses.append(torch.stack(l, 1))
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}
