"""More of what a fitted block is served and trained with, as cases that can be timed and checked one by one.

Five operators beside those of `operators.py`:

  linear    jab_fp8_linear: a projection whose weights are e4m3 numbers with an fp32 scale for every 128 of K, per row or
            per 128 rows. Fitted codes of up to 5 bits at group size 128 are e4m3 numbers as they are
  quantize  jab_fp8_quantize: the weights of such a projection (or any rows) into codes and scales
  write     jab_kv_write_norm_rope: rows [Q | K | V] with a norm for each head and the rotation (halves or
            neighbours, part of the head, tables scaled for long contexts) into the quantised paged cache
  rotate    jab_qk_norm_rope and jab_qk_norm_rope_backward: the same norm and rotation of prompts or training
            batches, with the gradients of rows and norm weights
  plan      jab_kv_release and jab_kv_plan: a server step's bookkeeping, pages of ended sequences back to the
            free list, pages, slots and positions for the new tokens

listed() and draw(rng) give cases, prepare(case, seed) the inputs, run(state) one pass, work(case) the
bytes and operations that the pass cannot do without, exact(case, seed) the outputs in 64 bits. With
`own` false run() computes the operators by elementary torch operations in 32 bits.

Definitions. A scale is fl32(max|x| / 448) of its block, a code e4m3(fl32(x / scale)), rounded to nearest even, at most
448 in magnitude; a block of zeros has scale 0 and codes 0. A head's norm is fl32(1 / sqrt(mean x^2 + eps)), a normed
element fl32(fl32(x norm) weight); the rotation's products and sums are each rounded to 32 bits, so that the
cache's codes are a function of the inputs. Pages of 16 to 4096 tokens; the free list is a stack.
"""
import math

import torch

own = False

#           d_model, query heads, KV heads, head_dim, RoPE theta
BLOCKS = {
    "gpt2": (768, 12, 12, 64, 10000.0),
    "mistral": (4096, 32, 8, 128, 10000.0),
    "gqa2": (512, 4, 2, 128, 10000.0),
    "gqa4_dh64": (256, 4, 1, 64, 500.0),
    "gqa3": (1024, 12, 4, 128, 10000.0),
}
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BLOCK, TOP, EPS = 128, 448.0, 1e-6


def _linear(name, block, M, weights, x, y):
    return {"name": name, "kind": "linear", "block": block, "M": M, "weights": weights, "x": x, "y": y}


def _quantize(name, M, K, rows, x):
    return {"name": name, "kind": "quantize", "M": M, "K": K, "rows": rows, "x": x}


def _rows(name, kind, block, B, T, start, x, part, neighbours, norm, scaled):
    return {"name": name, "kind": kind, "block": block, "B": B, "T": T, "start": start, "x": x, "part": part,
            "neighbours": neighbours, "norm": norm, "scaled": scaled}


def _write(name, block, B, T, start, x, part, neighbours, norm, scaled, bits, page):
    return dict(_rows(name, "write", block, B, T, start, x, part, neighbours, norm, scaled), bits=bits, page=page)


def _plan(name, B, page, longest, new, ended, padding):
    return {"name": name, "kind": "plan", "B": B, "page": page, "longest": longest, "new": new, "ended": ended,
            "padding": padding}


def listed():
    return [
        # the projection of one new token, scales for every 128 x 128 weights: the weights are read for a single row
        _linear("linear_mistral_1", "mistral", 1, "blocks", "bf16", "bf16"),
        # a few dozen tokens of a small block fitted at 4 bits in groups of 128, an odd number of rows: launches and latency
        _linear("linear_gpt2_37", "gpt2", 37, "fit4", "fp16", "fp32"),
        # a decoding step of 64 sequences, a scale for every row's 128 weights
        _linear("linear_mistral_64", "mistral", 64, "rows", "bf16", "fp16"),
        # prompts of 8192 tokens in all: the largest product
        _linear("linear_mistral_8192", "mistral", 8192, "blocks", "bf16", "bf16"),
        # the weights of a small block in fp32, a scale for every row's 128: latency
        _quantize("quantize_gpt2", 2304, 768, 1, "fp32"),
        # a large block's weights, 128 x 128 to a scale
        _quantize("quantize_mistral", 6144, 4096, 128, "bf16"),
        # a decoding step of 64 sequences in a context stretched four times
        _write("write_mistral_64x1", "mistral", 64, 1, 16001, "bf16", 1, False, True, True, 8, 64),
        # three prompts of odd length, a quarter of each head turned, neighbours together, no norm, 4 bits
        _write("write_gpt2_3x1001", "gpt2", 3, 1001, 0, "fp16", 4, True, False, False, 4, 16),
        # a short training batch of a small block: launches and latency
        _rows("rotate_gqa4_4x128", "rotate", "gqa4_dh64", 4, 128, 0, "fp32", 2, True, True, False),
        # a training batch of 8 sequences of 2048 tokens
        _rows("rotate_mistral_8x2048", "rotate", "mistral", 8, 2048, 0, "bf16", 1, False, True, False),
        # a decoding step of 64 sequences: most need no page
        _plan("plan_64_decode", 64, 64, 8192, 1, 2, 0),
        # prompts of 1000 requests that come in chunks, and the pages of those that ended
        _plan("plan_1000_prompts", 1000, 16, 4096, 250, 100, 3001),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / 1e15)


def draw(rng):
    kind = rng.choice(("linear", "linear", "quantize", "write", "write", "rotate", "plan"))
    most = max(_cost(c) for c in listed() if c["kind"] == kind)
    if kind == "write":  # (the range goes to prompts; the listed ones stand for the calls where latency counts)
        most = max(_cost(c) for c in listed() if c["kind"] == "rotate")
    while True:
        block = rng.choice(("gpt2", "mistral", "mistral", "gqa2", "gqa3", "gqa4_dh64"))
        x = rng.choice(("bf16", "bf16", "fp16", "fp16", "fp32"))
        if kind == "linear":
            case = _linear("", block, _log_int(rng, 1, 8192), rng.choice(("blocks", "blocks", "rows", "fit3", "fit5")), x,
                           rng.choice(("bf16", "fp16", "fp32")))
        elif kind == "quantize":
            case = _quantize("", _log_int(rng, 1, 8192), 16 * _log_int(rng, 1, 512), rng.choice((1, 128)), x)
        elif kind == "plan":
            case = _plan("", _log_int(rng, 1, 2048), rng.choice((16, 32, 64, 128, 48)), _log_int(rng, 1, 8192),
                         rng.choice((1, 1, 2, _log_int(rng, 1, 500))), rng.choice((0, 1, 7)), rng.choice((0, 0, 1, 100)))
        else:
            T = _log_int(rng, 1, 4096)
            B = _log_int(rng, 1, max(1, min(128, 16384 // T)))
            args = (block, B, T, rng.choice((0, 0, _log_int(rng, 1, 20000))), x, rng.choice((1, 1, 2, 4)),
                    rng.random() < 0.5, rng.random() < 0.7, rng.random() < 0.3)
            case = (_write("", *args, rng.choice((4, 8)), rng.choice((16, 32, 64, 128))) if kind == "write"
                    else _rows("", "rotate", *args))
        del case["name"]
        if _cost(case) <= most:
            return case


# ------------------------------------------------------------------ sizes
def _up(n, d):
    return -(-n // d)


def _plan_sizes(case):
    """(cached tokens, new tokens, whether it ends) of every sequence: those that end get no new ones."""
    B, hi, new = case["B"], case["longest"], case["new"]
    lens = [int(hi ** (((i * 29) % B + 0.5) / B)) for i in range(B)]
    ends = [i % max(1, B // max(1, case["ended"])) == 0 and case["ended"] > 0 for i in range(B)]
    counts = [0 if e else new if new < 3 else 1 + (i * 7919) % (2 * new - 1) for i, e in enumerate(ends)]
    return lens, counts, ends


def work(case):
    size = 4 if case.get("x") == "fp32" else 2
    if case["kind"] == "quantize":
        M, K = case["M"], case["K"]
        return {"bytes": M * K * (size + 1) + _up(M, case["rows"]) * _up(K, BLOCK) * 4, "flops": 2 * M * K}
    if case["kind"] == "plan":
        lens, counts, ends = _plan_sizes(case)
        page, rows = case["page"], sum(counts) + case["padding"]
        back = sum(_up(n, page) for n, e in zip(lens, ends) if e)
        taken = sum(_up(n + c, page) - _up(n, page) for n, c, e in zip(lens, counts, ends) if not e)
        used = sum(_up(n + c, page) - n // page for n, c, e in zip(lens, counts, ends) if not e and c)
        # lengths, counts and ends in, lengths and starts out, pages given back and taken, pages of the new tokens, rows
        return {"bytes": case["B"] * 20 + 8 * (back + taken) + 4 * used + rows * 12, "flops": rows}
    d, hq, hkv, dh, _ = BLOCKS[case["block"]]
    D = (hq + 2 * hkv) * dh
    if case["kind"] == "linear":
        M, out = case["M"], 4 if case["y"] == "fp32" else 2
        scales = (_up(D, BLOCK) if case["weights"] == "blocks" else D) * _up(d, BLOCK) * 4
        return {"bytes": M * d * size + D * d + scales + M * D * out, "flops": 2 * M * D * d}
    N, turned = case["B"] * case["T"], (hq + hkv) * dh
    table = N * dh // case["part"] * 4 + N * 4
    if case["kind"] == "write":
        row = dh * case["bits"] // 8 + 4
        # the joint rows in, Q out, the pages written and read once, K and V out, slots, positions and table rows
        return {"bytes": N * D * size + N * hq * dh * size + 2 * (2 * N * hkv * row) + 2 * N * hkv * dh * 2 + N * 8 + table,
                "flops": 12 * N * D}
    # rows in, rows out; rows and gradients in, gradients out; the norms' weights and their gradients
    return {"bytes": 5 * N * turned * size + 2 * table + 4 * dh * 4, "flops": 30 * N * turned}


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


def _blocked(x):
    """[M, blocks of K, 128], zeros behind the last column."""
    M, K = x.shape
    return torch.nn.functional.pad(x, (0, _up(K, BLOCK) * BLOCK - K)).view(M, -1, BLOCK)


def _fp8(x, rows):
    """(codes as fp32 numbers [M, K], scales [blocks of rows, blocks of K]) of rows of fp32 values."""
    M, K = x.shape
    b = _blocked(x)
    s = torch.nn.functional.pad(b.abs().amax(-1), (0, 0, 0, _up(M, rows) * rows - M))
    # divided on the device: torch turns a division by a host number into a product with its reciprocal
    s = s.view(-1, rows, b.shape[1]).amax(1) / torch.full((), TOP, device=x.device)
    each = s.repeat_interleave(rows, 0)[:M, :, None] if rows > 1 else s[:, :, None]
    c = (b / each).clamp(-TOP, TOP).to(torch.float8_e4m3fn).float()
    return torch.where(each > 0, c, torch.zeros_like(c)).flatten(1)[:, :K], s


def _fit(x, bits):
    """(whole-numbered codes, scales) of rows in groups of 128: what a fit with that group size leaves."""
    b, qmax = _blocked(x), float(2 ** (bits - 1) - 1)
    s = b.abs().amax(-1) / torch.full((), qmax, device=x.device)
    return torch.round(b / s[..., None]).clamp(-qmax, qmax).flatten(1)[:, : x.shape[1]], s


def _table(dim, theta, length, scaled):
    """cos and sin [length, dim / 2]; scaled: four times a context of 4096, by parts: frequencies of 32 turns and more in it
    stay, those of one and less are divided by four, both with the factor 0.1 ln 4 + 1."""
    f = theta ** (-2 * torch.arange(dim // 2, device="cuda", dtype=torch.float64) / dim)
    by = 1.0
    if scaled:
        stay = ((4096 * f / (2 * math.pi) - 1) / 31).clamp(0, 1)
        f, by = f / 4 * (1 - stay) + f * stay, 0.1 * math.log(4) + 1
    a = torch.arange(length, device="cuda", dtype=torch.float64)[:, None] * f
    return (a.cos() * by).float().contiguous(), (a.sin() * by).float().contiguous()


def _pages(g, lens, page, width):
    """Page numbers of every sequence in no order, int32 [B, width]; the free ones; their number in all."""
    each = torch.tensor([_up(n, page) for n in lens], device="cuda")
    used = int(each.sum())
    total = used + sum(width - _up(n, page) for n in lens) + 3
    ids = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    at = (each.cumsum(0) - each)[:, None] + torch.arange(width, device="cuda")
    table = torch.where(torch.arange(width, device="cuda") < each[:, None], ids[at.clamp(max=total - 1)], 0)
    return table.to(torch.int32).contiguous(), ids[used:], total


def prepare(case, seed):
    g = _generator(seed)
    s = {"case": case}
    i32 = dict(dtype=torch.int32, device="cuda")
    if case["kind"] == "quantize":
        M, K, rows = case["M"], case["K"], case["rows"]
        s["x"] = (torch.randn((M, K), generator=g, device="cuda") * 0.02).to(DTYPES[case["x"]])
        if own:
            s["codes"] = torch.empty((M, K), dtype=torch.float8_e4m3fn, device="cuda")
            s["scales"] = torch.empty((_up(M, rows), _up(K, BLOCK)), device="cuda")
        return s
    if case["kind"] == "plan":
        lens, counts, ends = _plan_sizes(case)
        page = case["page"]
        width = max(1, max(_up(n + c, page) for n, c in zip(lens, counts)))
        s["pages"], free, s["n_pages"] = _pages(g, lens, page, width)
        s["lens"], s["counts"], s["ends"] = (torch.tensor(v, **i32) for v in (lens, counts, [int(e) for e in ends]))
        s["free"] = torch.zeros(s["n_pages"], **i32)
        s["free"][: len(free)] = free
        s["n_free"] = torch.tensor([len(free)], **i32)
        s["rows"] = sum(counts) + case["padding"]
        if own:
            import paper_2609_34866_gb300 as J
            s["cache"] = J.KvCache(1, 64, 8, page, s["n_pages"])
            s["lens_kept"], s["lens_new"] = torch.empty_like(s["lens"]), torch.empty_like(s["lens"])
            s["free_back"], s["free_new"] = torch.empty_like(s["n_free"]), torch.empty_like(s["n_free"])
            s["q_start"] = torch.empty(case["B"] + 1, **i32)
            s["slots"] = torch.empty(s["rows"], dtype=torch.int64, device="cuda")
            s["positions"] = torch.empty(s["rows"], **i32)
        return s
    d, hq, hkv, dh, theta = BLOCKS[case["block"]]
    D = (hq + 2 * hkv) * dh
    dt = DTYPES[case["x"]]
    if case["kind"] == "linear":
        M = case["M"]
        s["x"] = _activations(g, M, d).to(dt)
        w = torch.randn((D, d), generator=g, device="cuda") * 0.02
        s["rows"] = 128 if case["weights"] == "blocks" else 1
        codes, s["scales"] = _fit(w, int(case["weights"][3:])) if case["weights"].startswith("fit") else _fp8(w, s["rows"])
        s["codes"] = codes.to(torch.float8_e4m3fn).contiguous()
        if own:
            import paper_2609_34866_gb300 as J
            s["y"] = torch.empty((M, D), dtype=DTYPES[case["y"]], device="cuda")
            s["ws"] = torch.empty(J.jab_fp8_linear_workspace_size(M, D, d), dtype=torch.uint8, device="cuda")
        return s
    B, T, start = case["B"], case["T"], case["start"]
    N, dim = B * T, dh // case["part"]
    pos = torch.arange(start, start + T, device="cuda").repeat(B)
    s["positions"] = pos.int()
    s["rope"] = _table(dim, theta, start + T, case["scaled"])
    s["qkv"] = _activations(g, N, D).to(dt)
    s["eps"] = EPS if case["norm"] else None
    s["wq"], s["wk"] = ((1 + 0.2 * torch.randn(dh, generator=g, device="cuda")) if case["norm"] else None for _ in range(2))
    if case["kind"] == "write":
        s["pages"], _, n_pages = _pages(g, [start + T] * B, case["page"], _up(start + T, case["page"]))
        row = torch.arange(B, device="cuda").repeat_interleave(T)
        s["slots"] = s["pages"][row, pos // case["page"]].long() * case["page"] + pos % case["page"]
        s["starts"], s["counts"] = torch.full((B,), start, **i32), torch.full((B,), T, **i32)
        if own:
            import paper_2609_34866_gb300 as J
            s["cache"] = J.KvCache(hkv, dh, case["bits"], case["page"], n_pages)
            s["q"] = torch.empty((N, hq * dh), dtype=dt, device="cuda")
            s["k"], s["v"] = (torch.empty((B, T, hkv, dh), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        return s
    s["dq"], s["dk"] = ((torch.randn((N, h * dh), generator=g, device="cuda") * 0.01).to(dt) for h in (hq, hkv))
    if own:
        import paper_2609_34866_gb300 as J
        s["q"], s["k"] = torch.empty_like(s["dq"]), torch.empty_like(s["dk"])
        s["dx"] = torch.empty((N, (hq + hkv) * dh), dtype=dt, device="cuda")
        s["dwq"], s["dwk"] = (torch.empty(dh, device="cuda") if case["norm"] else None for _ in range(2))
        s["ws"] = torch.empty(J.jab_qk_norm_rope_backward_workspace_size(N, hq, hkv, dh), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    return {"linear": _plain_linear, "quantize": _plain_quantize, "write": _plain_write, "rotate": _plain_rotate,
            "plan": _plain_plan}[case["kind"]](s, case)


def _run_own(s, case):
    import paper_2609_34866_gb300 as J
    if case["kind"] == "linear":
        J.jab_fp8_linear(s["x"], s["codes"], s["scales"], s["y"], s["ws"], block_rows=s["rows"])
        return s["y"]
    if case["kind"] == "quantize":
        J.jab_fp8_quantize(s["x"], s["codes"], s["scales"], block_rows=case["rows"])
        return {"values": s["codes"], "scales": s["scales"]}
    if case["kind"] == "plan":
        J.jab_kv_release(s["cache"], s["lens"], s["ends"], s["pages"], s["free"], s["n_free"], new_lens=s["lens_kept"],
                         new_free=s["free_back"])
        J.jab_kv_plan(s["cache"], s["lens_kept"], s["counts"], s["pages"], s["free"], s["free_back"], s["q_start"], s["slots"],
                      s["positions"], new_lens=s["lens_new"], new_free=s["free_new"])
        return {k: s[k] for k in ("lens_new", "free_new", "free", "pages", "q_start", "slots", "positions")}
    _, hq, hkv, dh, _ = BLOCKS[case["block"]]
    how = dict(positions=s["positions"], rope=s["rope"], interleaved=case["neighbours"], norm_eps=s["eps"],
               q_weight=s["wq"], k_weight=s["wk"])
    if case["kind"] == "write":
        J.jab_kv_write_norm_rope(s["cache"], s["qkv"], hq, s["slots"], q_out=s["q"], **how)
        J.jab_kv_read(s["cache"], s["pages"], s["counts"], s["k"], s["v"], starts=s["starts"])
        return {"q": s["q"], "k": s["k"], "v": s["v"]}
    J.jab_qk_norm_rope(s["qkv"], hq, hkv, dh, s["q"], s["k"], **how)
    J.jab_qk_norm_rope_backward(s["qkv"], hq, hkv, dh, s["dq"], s["dk"], s["dx"], s["ws"], dq_weight=s["dwq"],
                                dk_weight=s["dwk"], **how)
    out = {"q": s["q"], "k": s["k"], "dx": s["dx"]}
    return dict(out, dwq=s["dwq"], dwk=s["dwk"]) if case["norm"] else out


def _plain_linear(s, case):
    x = s["x"].float()
    c, sx = _fp8(x, 1)
    K = x.shape[1]
    spread = lambda t: t.repeat_interleave(BLOCK, 1)[:, :K]  # noqa: E731
    w = s["codes"].float()
    sw = s["scales"].repeat_interleave(s["rows"], 0)[: w.shape[0]] if s["rows"] > 1 else s["scales"]
    return ((c * spread(sx)) @ (w * spread(sw)).t()).to(DTYPES[case["y"]])


def _plain_quantize(s, case):
    c, scales = _fp8(s["x"].float(), case["rows"])
    return {"values": c.to(torch.float8_e4m3fn), "scales": scales}


def _norm_of(x, eps):
    """The factor of every head's norm: in 64 bits, since one ulp of it moves codes that lie at a border."""
    return (x.double().square().mean(-1, keepdim=True) + eps).rsqrt().float()


def _turn(x, cos, sin, neighbours, back=False):
    """Heads [N, heads, dh] with their first 2 * cos.shape[-1] elements turned by the rows' angles; back: by the transpose."""
    half = cos.shape[-1]
    cos, sin = cos[:, None], -sin[:, None] if back else sin[:, None]
    t, rest = x[..., : 2 * half], x[..., 2 * half :]
    a, b = (t[..., 0::2], t[..., 1::2]) if neighbours else (t[..., :half], t[..., half:])
    y, z = a * cos - b * sin, b * cos + a * sin
    t = torch.stack((y, z), -1).flatten(-2) if neighbours else torch.cat((y, z), -1)
    return torch.cat((t, rest), -1)


def _rows_of(s, case):
    """(heads in fp32 [N, heads of Q, K and V, dh], the rows' angles, weights of the norm for each of the heads of Q and K)"""
    _, hq, hkv, dh, _ = BLOCKS[case["block"]]
    x = s["qkv"].float().view(-1, hq + 2 * hkv, dh)
    cos, sin = (t[s["positions"].long()] for t in s["rope"])
    w = torch.cat((s["wq"].expand(hq, dh), s["wk"].expand(hkv, dh))) if case["norm"] else None
    return x, cos, sin, w


def _plain_forward(s, case):
    _, hq, hkv, dh, _ = BLOCKS[case["block"]]
    x, cos, sin, w = _rows_of(s, case)
    qk = x[:, : hq + hkv]
    if case["norm"]:
        qk = qk * _norm_of(qk, EPS) * w
    return _turn(qk, cos, sin, case["neighbours"]), x[:, hq + hkv :]


def _plain_write(s, case):
    _, hq, hkv, dh, _ = BLOCKS[case["block"]]
    B, T = case["B"], case["T"]
    qk, v = _plain_forward(s, case)
    qmax = float(2 ** (case["bits"] - 1) - 1)
    kv = torch.stack((qk[:, hq:], v))
    sc = kv.abs().amax(-1, keepdim=True) / torch.full((), qmax, device=kv.device)
    c = torch.round(kv / sc).clamp(-qmax, qmax)
    kv = (torch.where(sc > 0, c, torch.zeros_like(c)) * sc).bfloat16().view(2, B, T, hkv, dh)
    return {"q": qk[:, :hq].reshape(-1, hq * dh).to(DTYPES[case["x"]]), "k": kv[0], "v": kv[1]}


def _plain_rotate(s, case):
    _, hq, hkv, dh, _ = BLOCKS[case["block"]]
    dt = DTYPES[case["x"]]
    x, cos, sin, w = _rows_of(s, case)
    y, _ = _plain_forward(s, case)
    N = x.shape[0]
    g = torch.cat((s["dq"].float().view(N, hq, dh), s["dk"].float().view(N, hkv, dh)), 1)
    g = _turn(g, cos, sin, case["neighbours"], back=True)
    out = {"q": y[:, :hq].reshape(N, -1).to(dt), "k": y[:, hq:].reshape(N, -1).to(dt)}
    if case["norm"]:
        r = _norm_of(x[:, : hq + hkv], EPS)
        n = x[:, : hq + hkv] * r
        dw = g * n
        out.update(dwq=dw[:, :hq].sum((0, 1)), dwk=dw[:, hq:].sum((0, 1)))
        u = g * w
        g = r * (u - n * (u * n).mean(-1, keepdim=True))
    return dict(out, dx=g.reshape(N, -1).to(dt))


def _plain_plan(s, case):
    page, B, rows = case["page"], case["B"], s["rows"]
    lens, counts, ends = s["lens"].long(), s["counts"].long(), s["ends"].long() != 0
    dev = lens.device
    width = s["pages"].shape[1]
    entry = torch.arange(width, device=dev)
    # pages of the ended sequences, in the sequences' order and their own, onto the stack
    have = (lens + page - 1) // page
    back = torch.where(ends, have, torch.zeros_like(have))
    at = s["n_free"].long() + (back.cumsum(0) - back)[:, None] + entry
    out = entry < back[:, None]
    s["free"][at[out]] = s["pages"][out]
    n_free = s["n_free"].long() + back.sum()
    kept = torch.where(ends, torch.zeros_like(lens), lens)
    # pages for the new tokens, from the top of the stack
    have = (kept + page - 1) // page
    need = (kept + counts + page - 1) // page - have
    before = need.cumsum(0) - need
    new = (entry >= have[:, None]) & (entry < (have + need)[:, None])
    at = n_free - 1 - (before[:, None] + entry - have[:, None])
    s["pages"][new] = s["free"][at[new]]
    ends_at = counts.cumsum(0)
    row = torch.arange(rows, device=dev)
    seq = torch.searchsorted(ends_at, row, right=True)
    real = seq < B
    seq = seq.clamp(max=B - 1)
    pos = kept[seq] + row - (ends_at - counts)[seq]
    pos = torch.where(real, pos, torch.zeros_like(pos))
    slots = s["pages"][seq, (pos // page).clamp(max=width - 1)].long() * page + pos % page
    return {"lens_new": (kept + counts).int(), "free_new": (n_free - need.sum()).int(), "free": s["free"], "pages": s["pages"],
            "q_start": torch.cat((torch.zeros_like(ends_at[:1]), ends_at)).int(),
            "slots": torch.where(real, slots, torch.full_like(slots, -1)), "positions": pos.int()}


# ------------------------------------------------------------------ 64 bits
def _exact_e4m3(v):
    """Numbers rounded to 4 significant bits, half to even, steps of 2^-9 at least, 448 at most."""
    e = torch.frexp(v.abs()).exponent - 1
    step = ((e.clamp(min=-6) - 3 + 1023).long() << 52).view(torch.float64)  # (2 to that power, without a rounding)
    return (torch.round(v / step) * step).clamp(-TOP, TOP)


def _exact_fp8(x, rows):
    """Codes and scales [M, K] (each element's) of fp64 rows; scale and quotient are rounded to 32 bits by definition."""
    M, K = x.shape
    kb, mb = torch.arange(K, device="cuda") // BLOCK, torch.arange(M, device="cuda") // rows
    top = torch.zeros((M, _up(K, BLOCK)), dtype=torch.float64, device="cuda")
    top.scatter_reduce_(1, kb.expand(M, K), x.abs(), "amax")
    by = torch.zeros((_up(M, rows), top.shape[1]), dtype=torch.float64, device="cuda")
    by.scatter_reduce_(0, mb[:, None].expand_as(top), top, "amax")
    s = (by / torch.full((), TOP, dtype=torch.float64, device="cuda")).float()
    each = s.double()[mb][:, kb]
    v = torch.where(each > 0, (x / each).float().double(), 0.0)
    return _exact_e4m3(v), each, s


def _exact_rows(s, case):
    """(Q and K normed and turned, V) as fp64 heads, and what the gradients need."""
    _, hq, hkv, dh, _ = BLOCKS[case["block"]]
    x = s["qkv"].double().reshape(-1, hq + 2 * hkv, dh)
    qk, v = x[:, : hq + hkv], x[:, hq + hkv :]
    r = torch.ones_like(qk[..., :1])
    w = torch.ones((hq + hkv, dh), dtype=torch.float64, device="cuda")
    if case["norm"]:
        r = 1 / torch.sqrt(torch.linalg.vector_norm(qk, dim=-1, keepdim=True) ** 2 / dh + EPS)
        w = torch.cat([s["wq"].double()[None]] * hq + [s["wk"].double()[None]] * hkv)
    c, sn = (t.double()[s["positions"].long()][:, None] for t in s["rope"])
    z = torch.complex(c, sn)
    dim = 2 * c.shape[-1]

    def turned(t, by):
        head, rest = t[..., :dim], t[..., dim:]
        if case["neighbours"]:
            p = torch.view_as_real(torch.view_as_complex(head.reshape(*head.shape[:-1], -1, 2).contiguous()) * by).flatten(-2)
        else:
            q = torch.complex(head[..., : dim // 2], head[..., dim // 2 :]) * by
            p = torch.cat((q.real, q.imag), -1)
        return torch.cat((p, rest), -1)

    return qk, v, r, w, z, turned


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "plan":
        return None
    if case["kind"] == "quantize":
        c, _, scales = _exact_fp8(s["x"].double(), case["rows"])
        return {"values": c, "scales": scales.double()}
    _, hq, hkv, dh, _ = BLOCKS[case["block"]]
    if case["kind"] == "linear":
        c, sx, _ = _exact_fp8(s["x"].double(), 1)
        D, K = s["codes"].shape
        n, k = torch.arange(D, device="cuda") // s["rows"], torch.arange(K, device="cuda") // BLOCK
        return torch.einsum("mk,nk->mn", c * sx, s["codes"].double() * s["scales"].double()[n][:, k])
    qk, v, r, w, z, turned = _exact_rows(s, case)
    y = turned(qk * r * w, z)
    N = qk.shape[0]
    if case["kind"] == "write":
        kv = torch.stack((y[:, hq:], v)).reshape(2, case["B"], case["T"], hkv, dh)
        qmax = 2 ** (case["bits"] - 1) - 1
        top = kv.float().abs().amax(-1, keepdim=True)  # (scales, quotients and what they are of in 32 bits, by definition)
        sc = (top.double() / qmax).float().double()
        c = torch.where(sc > 0, torch.round((kv.float().double() / sc).float().double()), 0.0).clamp(-qmax, qmax)
        return {"q": y[:, :hq].reshape(N, -1), "k": (c * sc)[0], "v": (c * sc)[1]}
    g = turned(torch.cat((s["dq"].double().reshape(N, hq, dh), s["dk"].double().reshape(N, hkv, dh)), 1), z.conj())
    out = {"q": y[:, :hq].reshape(N, -1), "k": y[:, hq:].reshape(N, -1)}
    if case["norm"]:
        xn = qk * r
        out["dwq"], out["dwk"] = (torch.einsum("nhd,nhd->d", g[:, h], xn[:, h]) for h in (slice(0, hq), slice(hq, None)))
        gw = g * w
        g = (gw - xn * torch.einsum("nhd,nhd->nh", gw, xn)[..., None] / dh) * r
    return dict(out, dx=g.reshape(N, -1))
