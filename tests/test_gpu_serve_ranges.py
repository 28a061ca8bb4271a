"""The serving operators over their whole ranges: calls whose blocks go round their loops more than once, values at
the edges of what the kernels hold, and inputs that have to be reported. Everything against plain float64
implementations (serve_ref.py); the projection, codes, scales and read-back bit for bit."""
import math

import pytest
import torch

import serve_ref as R
from test_gpu_serve import HALF_ULP, _filled, _gen, _linear, _pages

pytestmark = pytest.mark.gpu

import paper_2609_34866_gb300 as J  # noqa: E402


@pytest.fixture(autouse=True)
def _status():
    J.jab_get_device_status()
    yield
    torch.cuda.synchronize()


def _attention(cache, q, q_lens, lens, pages, shared=0, window=0, max_q=None, max_len=None, scale=0.0):
    """(out, lse) of a call."""
    n, hq, _ = q.shape
    max_q, max_len = max_q or max(q_lens), max_len or max(lens)
    start = torch.tensor([0] + list(torch.tensor(q_lens).cumsum(0)), dtype=torch.int32, device="cuda")
    out, lse = torch.full_like(q, 77.0), torch.full((n, hq), 77.0, device="cuda")
    ws = torch.full((J.jab_kv_attention_workspace_size(cache, len(lens), n, hq, max_q, max_len, shared),), 0xFF, dtype=torch.uint8,
                    device="cuda")
    J.jab_kv_attention(cache, q, start, pages, torch.tensor(lens, dtype=torch.int32, device="cuda"), out, ws, max_q, max_len,
                       shared_len=shared, window=window, softmax_scale=scale, lse=lse)
    return out, lse


def _exact(cache, kd, vd, q, q_lens, lens, pages, window=0, scale=0.0):
    """Per (token, head) in float64: o, log-sum-exp, sum p |v|, the longest row, and the largest p_j max|v_j|."""
    n, hq, dh = q.shape
    page, hkv, at = cache.page_tokens, cache.n_kv_heads, 0
    f64 = dict(dtype=torch.float64, device="cuda")
    o, mag = torch.zeros((n, hq, dh), **f64), torch.zeros((n, hq, dh), **f64)
    lse, top, keys = torch.full((n, hq), -math.inf, **f64), torch.zeros((n, hq, 1), **f64), torch.zeros((n, hq, 1), **f64)
    for b, (nq, length) in enumerate(zip(q_lens, lens)):
        j = torch.arange(length, device="cuda")
        ids = pages[b].long()[j // page]
        k, v = kd[ids, j % page], vd[ids, j % page]
        pos = torch.arange(length - nq, length, device="cuda")[:, None]
        seen = (j <= pos) & ((j > pos - window) if window else torch.ones_like(j <= pos))
        rows = slice(at, at + nq)
        for h in range(hq):
            kh, vh = k[:, h // (hq // hkv)], v[:, h // (hq // hkv)]
            s = (q[rows, h].double() @ kh.t() * (scale or 1 / math.sqrt(dh))).masked_fill(~seen, -math.inf)
            ls = torch.logsumexp(s, -1)
            p = torch.where(seen, torch.exp(s - torch.where(ls > -math.inf, ls, 0.0)[:, None]), 0.0)
            o[rows, h], mag[rows, h], lse[rows, h] = p @ vh, p @ vh.abs(), ls
            if length:
                top[rows, h, 0] = (p * vh.abs().amax(-1)).amax(-1)
            keys[rows, h, 0] = seen.sum(-1).double()
        at += nq
    return o, lse, mag, keys, top


def _one_ahead(dh, bits, page, length):
    """A cache whose key 0 is 1 everywhere, all others 0; values 1, of key 0 every other one 0."""
    n_pages = -(-length // page)
    cache = J.KvCache(1, dh, bits, page, n_pages)
    zero, top = (128, 127) if bits == 8 else (8, 7)
    full = zero + top
    cache.k_codes.fill_(zero if bits == 8 else zero * 17)
    cache.v_codes.fill_(full if bits == 8 else full * 17)
    cache.k_scales.fill_(1.0 / top)
    cache.v_scales.fill_(1.0 / top)
    cache.k_codes[0, 0, 0] = full if bits == 8 else full * 17
    if bits == 8:
        cache.v_codes[0, 0, 0, 1::2] = zero
    else:
        cache.v_codes[0, 0, 0] = full + 16 * zero
    kd = R.unpack(cache.k_codes, bits) * cache.k_scales.double()[..., None]
    vd = R.unpack(cache.v_codes, bits) * cache.v_scales.double()[..., None]
    return cache, kd.transpose(1, 2), vd.transpose(1, 2), torch.arange(n_pages, dtype=torch.int32, device="cuda").view(1, -1)


def _held(out, want, o, rel, floor):
    tol = rel + floor + HALF_ULP[out.dtype] * o.abs() + 1e-30
    err = (out.double() - want).abs()
    assert bool((err <= tol).all()), (err / tol).max().item()


def _lse_held(lse, want):
    fin = torch.isfinite(want)
    assert bool((lse[~fin].double() == want[~fin]).all())
    assert bool(((lse.double() - want).abs()[fin] <= 2.0 ** -16 + 2.0 ** -21 * want.abs()[fin]).all()), (lse.double() - want).abs()[fin].max().item()


# ------------------------------------------------------------------ attention: bits of the weights
# A weight is an fp16 number and what that leaves over: within 2^-22 of it, or 2^-25 where that is more (twice that
# after the reference has moved). The largest of a row, p_a v_a, is at least 2^-1 as held, so that the second is at
# most 2^-23 p_a v_a of the result a key. Scores up to 10 in magnitude are within 2^-16 (eight truncated fp32 sums and
# their exponential), and two truncated products for 16 keys lose 2^-26 of the result a key.
@pytest.mark.parametrize("q_lens,lens,shared,window", [
    ([300, 77], [1000, 900], 0, 0),
    ([40], [513], 0, 0),
    ([260, 33], [1700, 500], 0, 400),
    ([1] * 40, [520 + 7 * i for i in range(40)], 512, 0),
])
@pytest.mark.parametrize("dh,hq,hkv,bits,dt", [(128, 8, 2, 8, torch.float16), (64, 4, 4, 4, torch.float16), (128, 6, 2, 4, torch.bfloat16)])
def test_weights_keep_their_bits_in_every_tile(q_lens, lens, shared, window, dh, hq, hkv, bits, dt):
    g = _gen(sum(lens) + dh + bits)
    page = 64
    cache, kd, vd = _filled(g, hkv, dh, bits, page, sum(-(-max(n, shared) // page) for n in lens) + 3)
    q = (torch.randn((sum(q_lens), hq, dh), generator=g, device="cuda") * 2).to(dt)
    pages = _pages(g, [max(n, shared) for n in lens], page, cache.n_pages, shared)
    out, lse = _attention(cache, q, q_lens, lens, pages, shared, window)
    assert J.jab_get_device_status() == 0
    o, ls, mag, keys, top = _exact(cache, kd, vd, q, q_lens, lens, pages, window)
    _held(out, o, o, (2.0 ** -22 + 2.0 ** -16 + keys * 2.0 ** -26) * mag, keys * 2.0 ** -23 * top)
    _lse_held(lse, ls)


@pytest.mark.parametrize("q_lens,lens", [([130, 4, 1, 3, 2, 5, 4], [700, 1500, 40, 3, 900, 77, 65]), ([600, 1, 1, 2], [600, 1000, 17, 2])])
@pytest.mark.parametrize("dh,hq,hkv,bits,dt", [(128, 8, 2, 8, torch.float16), (64, 16, 1, 4, torch.float16), (128, 6, 2, 4, torch.bfloat16)])
def test_short_runs_beside_a_chunk(q_lens, lens, dh, hq, hkv, bits, dt):
    """Sequences of 1 to 80 rows in one batch with a chunk: the two kernels share the work between them."""
    g = _gen(sum(lens) + dh + bits)
    cache, kd, vd = _filled(g, hkv, dh, bits, 64, sum(-(-n // 64) for n in lens) + 3)
    q = (torch.randn((sum(q_lens), hq, dh), generator=g, device="cuda") * 2).to(dt)
    pages = _pages(g, lens, 64, cache.n_pages)
    out, lse = _attention(cache, q, q_lens, lens, pages)
    assert J.jab_get_device_status() == 0
    o, ls, mag, keys, top = _exact(cache, kd, vd, q, q_lens, lens, pages)
    _held(out, o, o, (2.0 ** -22 + 2.0 ** -16 + keys * 2.0 ** -26) * mag, keys * 2.0 ** -23 * top)
    _lse_held(lse, ls)


# ------------------------------------------------------------------ attention: small weights
# Weights 2^-26 of the largest are held within 2^-31 of it (2^-30 by tiles, twice that after a move), where a share of
# the work has all of a sequence's keys: many sequences, here of the same pages.
@pytest.mark.parametrize("nq,B,bits,dh", [(1, 2048, 8, 128), (1, 2048, 4, 64), (40, 600, 8, 128), (40, 600, 4, 64)])
@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
def test_a_long_flat_tail_behind_one_key(nq, B, bits, dh, dt):
    length = 4096
    cache, kd, vd, pages = _one_ahead(dh, bits, 64, length)
    q = torch.full((nq, 2, dh), 1.0, device="cuda").to(dt)
    scale = 26 * math.log(2) / dh
    out, lse = _attention(cache, q.repeat(B, 1, 1), [nq] * B, [length] * B, pages.repeat(B, 1), scale=scale)
    assert J.jab_get_device_status() == 0
    o, ls, mag, keys, top = _exact(cache, kd, vd, q, [nq], [length], pages, scale=scale)
    assert 0.98 * 2.0 ** -14 < o[0, 0, 1].item() < 2.0 ** -14
    _held(out.view(B, nq, 2, dh), o, o, 2.0 ** -11 * mag * (vd[0, 0, 0] > 0), keys * 2.0 ** -29 * top)
    _lse_held(lse.view(B, nq, 2), ls.expand(B, nq, 2))


def test_bf16_query_elements_far_below_the_largest():
    """Elements 2^-22 of a row's largest are used with all of their bits: the largest meets codes of 0."""
    dh, page, length = 128, 16, 48
    g = _gen(11)
    cache, kd, vd = _filled(g, 1, dh, 8, page, 3)
    cache.k_codes[..., 0] = 128
    kd[..., 0] = 0
    q = torch.randn((1, 4, dh), generator=g, device="cuda").to(torch.bfloat16)
    q[..., 0] = 2.0 ** 22
    pages = torch.arange(3, dtype=torch.int32, device="cuda").view(1, 3)
    for qq, nq in ((q, 1), (q.expand(40, 4, dh).contiguous(), 40)):
        out, lse = _attention(cache, qq, [nq], [length], pages, scale=0.3)
        assert J.jab_get_device_status() == 0
        o, ls, mag, keys, top = _exact(cache, kd, vd, qq, [nq], [length], pages, scale=0.3)
        _held(out, o, o, (2.0 ** -22 + 2.0 ** -15 + keys * 2.0 ** -26) * mag, keys * 2.0 ** -23 * top)
        _lse_held(lse, ls)


# ------------------------------------------------------------------ attention: values of zero, NaN
# (Many sequences, here of the same pages, so that a share of the work has several key tiles of a row in turn.)
@pytest.mark.parametrize("nq,B", [(1, 2048), (40, 400)])
@pytest.mark.parametrize("ahead", [60.0, 83.0, 88.0, 300.0])
def test_keys_far_ahead_whose_values_are_zero(nq, B, ahead):
    """Their scores alone decide the log-sum-exp; their weights are 0 whatever the scores are."""
    dh, page, length = 64, 64, 700
    cache, kd, vd, pages = _one_ahead(dh, 8, page, length)
    cache.k_codes[0, 0, 0], cache.v_codes[0, 0, 0] = 128, 255
    cache.k_codes[4], cache.v_codes[4] = 255, 128  # keys 256 to 319, in a tile that no mask cuts
    cache.v_scales[4] = 0.0
    kd[0, 0], kd[4], vd[0, 0], vd[4] = 0, 1, 1, 0
    q = torch.ones((nq, 2, dh), device="cuda").to(torch.float16)
    out, lse = _attention(cache, q.repeat(B, 1, 1), [nq] * B, [length] * B, pages.repeat(B, 1), scale=ahead / dh)
    assert J.jab_get_device_status() == 0
    o, ls, mag, keys, top = _exact(cache, kd, vd, q, [nq], [length], pages, scale=ahead / dh)
    _held(out.view(B, nq, 2, dh), o, o, 2.0 ** -10 * mag, 2.0 ** -60)
    _lse_held(lse.view(B, nq, 2), ls.expand(B, nq, 2))


@pytest.mark.parametrize("nq", [1, 40])
@pytest.mark.parametrize("size", [1e-25, 1e-40])
def test_values_near_the_end_of_fp32(nq, size):
    g = _gen(21)
    dh, page, length = 64, 64, 700
    cache, kd, vd = _filled(g, 1, dh, 8, page, 11)
    pages = torch.arange(11, dtype=torch.int32, device="cuda").view(1, -1)
    vd *= (size / cache.v_scales.double()).transpose(1, 2)[..., None]
    cache.v_scales.fill_(size)
    q = torch.randn((nq, 2, dh), generator=g, device="cuda").to(torch.bfloat16)
    out, lse = _attention(cache, q, [nq], [length], pages)
    assert J.jab_get_device_status() == 0
    o, ls, mag, keys, top = _exact(cache, kd, vd, q, [nq], [length], pages)
    tol = 2.0 ** -11 * mag + 2.0 ** -8 * o.abs() + 1e-37
    assert bool(((out.double() - o).abs() <= tol).all())
    _lse_held(lse, ls)


@pytest.mark.parametrize("nq", [1, 40])
@pytest.mark.parametrize("key", [5, 265, 650])
def test_a_value_that_is_nan_leaves_the_log_sum_exp(nq, key):
    g = _gen(key)
    dh, page, length = 64, 64, 700
    cache, kd, vd = _filled(g, 1, dh, 8, page, 11)
    pages = torch.arange(11, dtype=torch.int32, device="cuda").view(1, -1)
    q = torch.randn((nq, 2, dh), generator=g, device="cuda").to(torch.float16)
    cache.v_scales[key // page, 0, key % page] = math.nan
    out, lse = _attention(cache, q, [nq], [length], pages)
    o, ls, *_ = _exact(cache, kd, vd, q, [nq], [length], pages)
    assert bool(torch.isnan(out).all())
    _lse_held(lse, ls)


# ------------------------------------------------------------------ attention: inputs that are reported
def test_rows_that_no_sequence_owns_are_reported():
    cache, _, _ = _filled(_gen(1), 1, 64, 8, 16, 4)
    pages = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2)
    for hq, max_q in ((1, 2), (64, 40)):  # by keys, and by tiles
        n = 2 * max_q
        q = torch.randn((n, hq, 64), device="cuda").to(torch.float16)
        ws = torch.empty(J.jab_kv_attention_workspace_size(cache, 2, n, hq, max_q, 32), dtype=torch.uint8, device="cuda")
        lens = torch.tensor([32, 32], dtype=torch.int32, device="cuda")
        for start, status in (((0, max_q, n), 0), ((1, max_q, n), 1), ((0, max_q, n - 1), 1), ((0, 0, 0), 1), ((n, n, n), 1)):
            out = torch.full_like(q, 5.0)
            J.jab_kv_attention(cache, q, torch.tensor(start, dtype=torch.int32, device="cuda"), pages, lens, out, ws, max_q, 32)
            assert J.jab_get_device_status() == status, start
            assert bool((out[: start[0]] == 5).all()) and bool((out[start[2]:] == 5).all())


def test_a_list_of_work_too_long_to_count_is_reported():
    """2048 sequences that all claim the same rows, behind tables for 2^20 keys: 2^31 pairs of a row tile and a key
    tile. Nothing is computed."""
    page, B, n = 4096, 2048, 8192
    cache, _, _ = _filled(_gen(1), 1, 64, 8, page, 1)
    pages = torch.zeros((B, 256), dtype=torch.int32, device="cuda")
    lens = torch.full((B,), 256 * page, dtype=torch.int32, device="cuda")
    start = (torch.arange(B + 1, dtype=torch.int32, device="cuda") % 2) * n
    q = torch.randn((n, 4, 64), device="cuda").to(torch.float16)
    for shared in (0, page):
        out = torch.full_like(q, 5.0)
        ws = torch.empty(J.jab_kv_attention_workspace_size(cache, B, n, 4, n, 256 * page, shared), dtype=torch.uint8, device="cuda")
        J.jab_kv_attention(cache, q, start, pages, lens, out, ws, n, 256 * page, shared_len=shared)
        assert J.jab_get_device_status() == 1
        assert bool((out == 5).all())


@pytest.mark.parametrize("max_q,max_len", [(1 << 20, 1 << 20), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_hints_of_any_size_leave_the_work_to_all_blocks(max_q, max_len):
    """The longest of the sequences "or more": the same values, and no call of one block (a hundred times as long)."""
    g = _gen(31)
    B, page, dh = 64, 64, 128
    lens = [1024 + 16 * i for i in range(B)]
    cache, kd, vd = _filled(g, 8, dh, 8, page, sum(-(-n // page) for n in lens))
    pages = _pages(g, lens, page, cache.n_pages)
    q = torch.randn((B, 32, dh), generator=g, device="cuda").to(torch.float16)
    start, length = torch.arange(B + 1, dtype=torch.int32, device="cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda")
    times, outs = [], []
    for hints in ((max_q, max_len), (1, max(lens))):
        out = torch.empty_like(q)
        ws = torch.empty(J.jab_kv_attention_workspace_size(cache, B, B, 32, *hints), dtype=torch.uint8, device="cuda")
        best = math.inf
        for _ in range(5):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            J.jab_kv_attention(cache, q, start, pages, length, out, ws, *hints)
            b.record()
            b.synchronize()
            best = min(best, a.elapsed_time(b))
        times.append(best)
        outs.append(out)
    assert J.jab_get_device_status() == 0
    o, ls, mag, keys, top = _exact(cache, kd, vd, q, [1] * B, lens, pages)
    for out in outs:
        _held(out, o, o, (2.0 ** -22 + 2.0 ** -16 + keys * 2.0 ** -26) * mag, keys * 2.0 ** -23 * top)
    assert times[0] < 10 * times[1], times


def test_launches_are_counted():
    """One kernel for the work and one that joins; one more where a chunk and short runs share a call."""
    cache, _, _ = _filled(_gen(1), 1, 64, 8, 16, 40)
    pages = torch.arange(40, dtype=torch.int32, device="cuda").view(2, 20)
    q = torch.randn((101, 1, 64), generator=_gen(2), device="cuda").to(torch.float16)
    for q_lens, launches in (([1, 1], 2), ([50, 50], 2), ([100, 1], 3)):
        J.jab_timing_reset()
        J.jab_timing_enable(True)
        try:
            _attention(cache, q[: sum(q_lens)], q_lens, [300, 300], pages)
        finally:
            J.jab_timing_enable(False)
        assert J.jab_timing_read()["kv_attention"][1:] == (1, launches)
    J.jab_timing_reset()


# ------------------------------------------------------------------ cache
def _write_check(n, hq, hkv, dh, bits, page, dt, rope):
    g = _gen(n + hq + dh + bits)
    n_pages = -(-n // page) + 2
    qkv = torch.randn((n, (hq + 2 * hkv) * dh), generator=g, device="cuda").to(dt)
    slots = torch.randperm(n_pages * page, generator=g, device="cuda")[:n].clone()
    slots[::7] = -1
    qkv[::7] = math.nan  # padding: not read
    cache = J.KvCache(hkv, dh, bits, page, n_pages)
    cos = sin = pos = None
    if rope:
        cos, sin = (torch.empty((777, dh // 2), device="cuda") for _ in range(2))
        J.jab_rope_table(cos, sin, 10000.0)
        pos = torch.randint(0, 777, (n,), generator=g, device="cuda").int()
    q_out = torch.full((n, hq * dh), 9.0, dtype=dt, device="cuda") if hq else None
    J.jab_kv_write(cache, qkv, hq, slots, q_out=q_out, positions=pos, rope=(cos, sin) if rope else None)
    assert J.jab_get_device_status() == 0
    live = slots >= 0
    x = qkv.float().view(n, hq + 2 * hkv, dh)[live]
    turned = R.rotate(x[:, : hq + hkv], cos[pos[live].long()], sin[pos[live].long()]) if rope else x[:, : hq + hkv]
    if hq:
        assert torch.equal(q_out[live], turned[:, :hq].reshape(-1, hq * dh).to(dt)) and bool((q_out[~live] == 9).all())
    pg, at = slots[live] // page, slots[live] % page
    for rows, codes, scales in ((turned[:, hq:], cache.k_codes, cache.k_scales), (x[:, hq + hkv:], cache.v_codes, cache.v_scales)):
        c, s = R.quantize_rows(rows, bits)
        assert torch.equal(scales[pg, :, at], s) and torch.equal(codes[pg, :, at], R.pack(c, bits))


@pytest.mark.parametrize("hq,hkv,dh", [(64, 64, 128), (52, 52, 128), (104, 104, 64), (160, 16, 128)])
@pytest.mark.parametrize("few", [True, False])
def test_write_of_wide_blocks(hq, hkv, dh, few):
    """More heads than a block's threads: few tokens, and four for every SM and more."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    for n in (4 * sms - 1,) if few else (4 * sms, 700):
        for dt, bits in ((torch.float16, 8), (torch.bfloat16, 4), (torch.float32, 8)):
            _write_check(n, hq, hkv, dh, bits, 32, dt, True)


@pytest.mark.parametrize("hq,hkv,dh,bits,page", [(32, 8, 128, 8, 64), (12, 12, 64, 4, 16), (0, 3, 64, 8, 48), (71, 1, 128, 4, 32)])
@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rope", [False, True])
def test_write_of_many_tokens(hq, hkv, dh, bits, page, dt, rope):
    """A block takes many tokens one after the other, and several rounds of heads."""
    _write_check(6007, hq, hkv, dh, bits, page, dt, rope)


@pytest.mark.parametrize("hkv,dh,bits,page", [(8, 128, 8, 64), (3, 64, 4, 48), (40, 128, 4, 16)])
@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16, torch.float32])
def test_read_of_many_tokens(hkv, dh, bits, page, dt):
    """Several tokens a block, blocks that cross from one sequence to the next."""
    g = _gen(hkv + dh)
    B, T = 9, 1111
    counts = torch.tensor([1111, 0, 1, 1000, 1111, 513, 7, 1110, 999], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 3, 900, 111, 17, 0, 1000, 1, 64], dtype=torch.int32, device="cuda")
    width = -(-2300 // page)
    cache, kd, vd = _filled(g, hkv, dh, bits, page, 200)
    pages = torch.randint(0, 200, (B, width), generator=g, device="cuda").int()
    k, v = (torch.full((B, T, hkv, dh), 3.0, dtype=dt, device="cuda") for _ in range(2))
    J.jab_kv_read(cache, pages, counts, k, v, starts=starts)
    assert J.jab_get_device_status() == 0
    for b in range(B):
        j = torch.arange(int(counts[b]), device="cuda") + starts[b]
        ids = pages[b].long()[j // page]
        for got, codes, scales in ((k, cache.k_codes, cache.k_scales), (v, cache.v_codes, cache.v_scales)):
            want = (R.unpack(codes[ids, :, j % page], bits).float() * scales[ids, :, j % page][..., None]).to(dt)
            assert torch.equal(got[b, : j.numel()], want) and bool((got[b, j.numel():] == 0).all())


# ------------------------------------------------------------------ projection
@pytest.mark.parametrize("M,N,K", [(1500, 3500, 64), (1500, 3501, 336), (2100, 2600, 1200), (1411, 6144, 2064), (64, 21000, 1104), (9, 40001, 144)])
@pytest.mark.parametrize("xt,yt", [(torch.bfloat16, torch.bfloat16), (torch.float16, torch.float32), (torch.bfloat16, torch.float16)])
def test_linear_of_several_tiles_a_block(M, N, K, xt, yt):
    """More than two tiles for every SM: the accumulators and the rings go on from one tile to the next."""
    g = _gen(M + N + K)
    x = torch.randn((M, K), generator=g, device="cuda")
    x[:, :: max(1, K // 5)] *= 20
    x = x.to(xt)
    codes = torch.randint(-127, 128, (N, K), generator=g, device="cuda").to(torch.int8)
    ws = torch.rand((N,), generator=g, device="cuda") * 0.01 + 1e-4
    assert torch.equal(_linear(x, codes, ws, yt), R.linear(x, codes, ws, yt))
    assert J.jab_get_device_status() == 0
