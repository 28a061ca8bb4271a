"""The serving operators on the GPU (8-bit projection, quantised paged cache, attention over it) against plain
float64 implementations.

Tolerances. The projection, the codes, the scales and the read-back are compared bit for bit: their sums
are exact and their roundings are part of the definition. Attention keeps each weight to 2^-12 of it (two fp16 parts where rows see few keys;
weights below 2^-14 of the largest by 2^-25 of the largest) and the result to its type; scores are
fp32 sums of at most 128 exact products, their exponentials good to 2^-22, which stays below 2^-16 of the
result for scores of the size used here. So |error| <= (2^-12 + 2^-16) sum p |v| + n 2^-25 max|v| + ulp(type) / 2,
and the log-sum-exp is within 2^-16 + 2^-21 |lse|."""
import math

import pytest
import torch

import serve_ref as R

pytestmark = pytest.mark.gpu

import paper_2609_34866_gb300 as J  # noqa: E402

HALF_ULP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(autouse=True)
def _status():
    J.jab_get_device_status()
    yield
    torch.cuda.synchronize()


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


# ------------------------------------------------------------------ projection
def _linear(x, codes, ws, dtype, y=None):
    M, K = x.shape
    N = codes.shape[0]
    y = torch.empty((M, N), dtype=dtype, device="cuda") if y is None else y
    buf = torch.full((J.jab_quantized_linear_workspace_size(M, N, K),), 0x5A, dtype=torch.uint8, device="cuda")
    J.jab_quantized_linear(x, codes, ws, y, buf)
    return y


@pytest.mark.parametrize("M,N,K", [(1, 128, 64), (1, 6144, 4096), (2, 100, 16), (7, 2304, 768), (16, 129, 80), (17, 1, 1040),
                                   (33, 384, 256), (64, 1000, 2064), (65, 2560, 1024), (128, 640, 8208), (129, 257, 4096),
                                   (300, 2304, 768), (1500, 1024, 512)])
@pytest.mark.parametrize("xt,yt", [(torch.bfloat16, torch.bfloat16), (torch.float16, torch.float32), (torch.bfloat16, torch.float16)])
def test_linear_bit_for_bit(M, N, K, xt, yt):
    g = _gen(M * 7 + N + K)
    x = torch.randn((M, K), generator=g, device="cuda")
    x[:, :: max(1, K // 5)] *= 20
    x = x.to(xt)
    codes = torch.randint(-127, 128, (N, K), generator=g, device="cuda").to(torch.int8)
    ws = torch.rand((N,), generator=g, device="cuda") * 0.01 + 1e-4
    assert torch.equal(_linear(x, codes, ws, yt), R.linear(x, codes, ws, yt))
    assert J.jab_get_device_status() == 0


@pytest.mark.parametrize("M,K", [(3, 4096), (40, 16384), (130, 20016)])
def test_linear_largest_sums(M, K):
    """Every product 127^2 (or -127 * 128): sums far past 2^24, still exact."""
    x = torch.full((M, K), 3.0, device="cuda", dtype=torch.bfloat16)
    codes = torch.full((130, K), 127, dtype=torch.int8, device="cuda")
    codes[1] = -128
    codes[2, ::2] = -127
    codes[3, K // 2:] = -127
    codes[4, -1] = -126
    ws = torch.ones((130,), device="cuda")
    assert torch.equal(_linear(x, codes, ws, torch.float32), R.linear(x, codes, ws, torch.float32))


def test_linear_rows_of_zeros_tiny_and_nonfinite():
    K = 256
    x = torch.zeros((5, K), dtype=torch.bfloat16, device="cuda")
    x[1] = 1e-38
    x[2, 3], x[2, 4] = 3e38, -1.0
    x[3, 0] = math.inf
    x[4, K - 1] = math.nan
    codes = torch.randint(-7, 8, (130, K), generator=_gen(1), device="cuda").to(torch.int8)
    ws = torch.ones((130,), device="cuda")
    y = _linear(x, codes, ws, torch.float32)
    assert J.jab_get_device_status() == 4  # JAB_ERR_NONFINITE
    assert torch.equal(y[:3], R.linear(x[:3], codes, ws, torch.float32)) and bool((y[0] == 0).all())
    assert bool(torch.isnan(y[3:]).all())


def test_linear_pitched_rows_and_streams():
    g = _gen(5)
    big = torch.randn((21, 1000), generator=g, device="cuda").to(torch.bfloat16)
    x = big[:, 8:8 + 768]
    codes = torch.randint(-3, 4, (2304, 768), generator=g, device="cuda").to(torch.int8)
    ws = torch.rand((2304,), generator=g, device="cuda")
    out = torch.full((21, 2400), -5.0, device="cuda")
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    buf = torch.empty(J.jab_quantized_linear_workspace_size(21, 2304, 768), dtype=torch.uint8, device="cuda")
    for _ in range(3):
        J.jab_quantized_linear(x, codes, ws, out[:, :2304], buf, stream=st)
    st.synchronize()
    assert torch.equal(out[:, :2304], R.linear(x, codes, ws, torch.float32)) and bool((out[:, 2304:] == -5).all())
    J.jab_quantized_linear(x[:0], codes, ws, out[:0, :2304], buf)  # no rows: nothing to do


def test_linear_on_codes_of_jab_quantize():
    """Codes and scales as the fit leaves them, one group per output channel."""
    d, hq, dh = 768, 12, 64
    desc = J.BlockDesc(d, hq, hq, dh, d, 0, 10000.0, 0.0)
    g = _gen(9)
    W = (torch.randn((3 * hq * dh, d), generator=g, device="cuda") * 0.02).to(torch.bfloat16)
    scales = torch.empty((3 * hq * dh, 1), device="cuda")
    codes = torch.empty((3 * hq * dh, d), dtype=torch.int8, device="cuda")
    J.jab_init_scales(desc, 3, 1, W, scales)
    J.jab_quantize(desc, 3, W, scales, codes=codes)
    x = torch.randn((5, d), generator=g, device="cuda").to(torch.float16)
    assert torch.equal(_linear(x, codes, scales.view(-1), torch.float16), R.linear(x, codes, scales.view(-1), torch.float16))


# ------------------------------------------------------------------ cache
def _filled(g, hkv, dh, bits, page, n_pages, k_scale=0.5):
    """A cache of random codes, its tokens as float64 [n_pages, page, hkv, dh], and the KvCache."""
    cache = J.KvCache(hkv, dh, bits, page, n_pages)
    vals = []
    for codes, scales, f in ((cache.k_codes, cache.k_scales, k_scale), (cache.v_codes, cache.v_scales, 1.0)):
        c, s = R.quantize_rows(torch.randn((n_pages, hkv, page, dh), generator=g, device="cuda") * f, bits)
        codes.copy_(R.pack(c, bits))
        scales.copy_(s)
        vals.append((c * s.double()[..., None]).transpose(1, 2))
    return cache, vals[0], vals[1]


@pytest.mark.parametrize("dh,hq,hkv", [(64, 12, 12), (128, 32, 8), (128, 3, 1), (64, 0, 2)])
@pytest.mark.parametrize("bits,page", [(8, 16), (4, 48), (8, 64)])
@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rope", [False, True])
def test_write_and_read(dh, hq, hkv, bits, page, dt, rope):
    g = _gen(dh + hq + bits)
    n, n_pages = 53, 9
    qkv = torch.randn((n, (hq + 2 * hkv) * dh), generator=g, device="cuda")
    qkv[3] = 0
    qkv[5] *= 1e-30 if dt != torch.float16 else 1e-5
    qkv = qkv.to(dt)
    slots = torch.randperm(n_pages * page, generator=g, device="cuda")[:n].clone()
    slots[7] = slots[11] = -1
    qkv[7] = math.nan  # padding: not read
    cache = J.KvCache(hkv, dh, bits, page, n_pages)
    cos = sin = pos = None
    if rope:
        cos, sin = (torch.empty((1000, dh // 2), device="cuda") for _ in range(2))
        J.jab_rope_table(cos, sin, 10000.0)
        t = torch.arange(1000, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (
            -2 * torch.arange(dh // 2, device="cuda", dtype=torch.float64) / dh)
        assert (cos.double() - t.cos()).abs().max() < 1e-7 and (sin.double() - t.sin()).abs().max() < 1e-7
        pos = torch.randint(0, 1000, (n,), generator=g, device="cuda").int()
        pos[7] = 5000
    q_out = torch.full((n, hq * dh), 9.0, dtype=dt, device="cuda") if hq else None
    J.jab_kv_write(cache, qkv, hq, slots, q_out=q_out, positions=pos, rope=(cos, sin) if rope else None)
    assert J.jab_get_device_status() == 0
    live = slots >= 0
    x = qkv.float().view(n, hq + 2 * hkv, dh)[live]
    turned = R.rotate(x[:, : hq + hkv], cos[pos[live].long()], sin[pos[live].long()]) if rope else x[:, : hq + hkv]
    if hq:
        want = turned[:, :hq].reshape(-1, hq * dh).to(dt)
        assert torch.equal(q_out[live], want) and bool((q_out[~live] == 9).all())
    want_k, want_v = R.quantize_rows(turned[:, hq:], bits), R.quantize_rows(x[:, hq + hkv:], bits)
    pg, at = slots[live] // page, slots[live] % page
    for (c, s), codes, scales in ((want_k, cache.k_codes, cache.k_scales), (want_v, cache.v_codes, cache.v_scales)):
        assert torch.equal(scales[pg, :, at], s)
        assert torch.equal(codes[pg, :, at], R.pack(c, bits))
    # untouched slots stay as they were
    left = torch.ones(n_pages * page, dtype=torch.bool, device="cuda")
    left[slots[live]] = False
    assert bool((cache.k_scales.transpose(1, 2).reshape(-1, hkv)[left] == 0).all())
    # and back: sequences of pages in any order, ranges that start and end inside pages
    pages = torch.randperm(n_pages, generator=g, device="cuda")[:8].view(2, 4).int()
    starts = torch.tensor([0, 5], dtype=torch.int32, device="cuda")
    counts = torch.tensor([page + 3, 0], dtype=torch.int32, device="cuda")
    T = page + 5
    for out_t in (torch.float32, torch.float16, torch.bfloat16):
        k, v = (torch.full((2, T, hkv, dh), 3.0, dtype=out_t, device="cuda") for _ in range(2))
        J.jab_kv_read(cache, pages, counts, k, v, starts=starts)
        j = torch.arange(page + 3, device="cuda")
        ids = pages[0].long()[j // page]
        for got, codes, scales in ((k, cache.k_codes, cache.k_scales), (v, cache.v_codes, cache.v_scales)):
            want = (R.unpack(codes[ids, :, j % page], bits).float() * scales[ids, :, j % page][..., None]).to(out_t)
            assert torch.equal(got[0, : page + 3], want)
            assert bool((got[0, page + 3:] == 0).all()) and bool((got[1] == 0).all())
    assert J.jab_get_device_status() == 0


def test_write_nonfinite_and_bad_indices():
    cache = J.KvCache(2, 64, 8, 16, 2)
    qkv = torch.ones((4, 4 * 64), device="cuda")
    qkv[1, 5] = math.inf
    J.jab_kv_write(cache, qkv, 0, torch.tensor([0, 1, 2, 3], device="cuda"))
    assert J.jab_get_device_status() == 4
    assert math.isnan(cache.k_scales[0, 0, 1].item()) and cache.k_scales[0, 1, 1].item() > 0
    J.jab_kv_write(cache, torch.ones_like(qkv), 0, torch.tensor([4, 32, 5, 1 << 40], device="cuda"))
    assert J.jab_get_device_status() == 1  # slots past the cache
    cos = torch.ones((4, 32), device="cuda")
    J.jab_kv_write(cache, torch.ones_like(qkv), 0, torch.tensor([4, 6, 5, 7], device="cuda"), rope=(cos, cos),
                   positions=torch.tensor([0, 4, -1, 3], dtype=torch.int32, device="cuda"))
    assert J.jab_get_device_status() == 1
    assert cache.v_scales[0, 0, 6].item() > 0 and cache.k_scales[0, 0, 6].item() == 0
    k, v = (torch.ones((1, 20, 2, 64), device="cuda") for _ in range(2))
    J.jab_kv_read(cache, torch.tensor([[0, 7]], dtype=torch.int32, device="cuda"), torch.tensor([18], dtype=torch.int32, device="cuda"), k, v)
    assert J.jab_get_device_status() == 1
    assert bool((k[0, 16:] == 0).all())


# ------------------------------------------------------------------ attention
def _attend(cache, kd, vd, q, q_lens, lens, pages, shared=0, window=0, scale=0.0, max_q=None, max_len=None, out=None, stream=None):
    """Runs jab_kv_attention and checks it against the float64 form."""
    n, hq, dh = q.shape
    page = cache.page_tokens
    q_start = torch.tensor([0] + list(torch.tensor(q_lens).cumsum(0)), dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 77.0) if out is None else out
    lse = torch.full((n, hq), 77.0, device="cuda")
    max_q, max_len = max_q or max(max(q_lens), 1), max_len or max(lens)
    ws = torch.full((J.jab_kv_attention_workspace_size(cache, len(lens), n, hq, max_q, max_len, shared),), 0xFF, dtype=torch.uint8,
                    device="cuda")
    J.jab_kv_attention(cache, q, q_start, pages, torch.tensor(lens, dtype=torch.int32, device="cuda"), out, ws, max_q, max_len,
                       shared_len=shared, window=window, softmax_scale=scale, lse=lse, stream=stream)
    if stream is not None:
        stream.synchronize()
    assert J.jab_get_device_status() == 0
    at = 0
    for b, (nq, length) in enumerate(zip(q_lens, lens)):
        j = torch.arange(length, device="cuda")
        ids = pages[b].long()[j // page]
        k, v = kd[ids, j % page], vd[ids, j % page]
        o, ls, mag = R.attention(q[at:at + nq].double(), k, v, window, scale or 1 / math.sqrt(dh))
        vmax = v.abs().max() if length else 0.0
        tol = (2.0 ** -12 + 2.0 ** -16) * mag + length * 2.0 ** -25 * vmax + HALF_ULP[q.dtype] * o.abs() + 1e-30
        err = (out[at:at + nq].double() - o).abs()
        assert bool((err <= tol).all()), (b, nq, length, (err / tol).max().item())
        fin = torch.isfinite(ls)
        got = lse[at:at + nq].double()
        assert torch.equal(torch.isfinite(got), fin) and bool((got[~fin] == -math.inf).all())
        if bool(fin.any()):
            assert bool(((got - ls).abs()[fin] <= 2.0 ** -16 + 2.0 ** -21 * ls.abs()[fin]).all())
        at += nq
    return out, lse


def _pages(g, lens, page, n_pages, shared=0):
    width = max(1, max(-(-n // page) for n in lens)) + 1
    ids = torch.randperm(n_pages, generator=g, device="cuda")
    t = torch.zeros((len(lens), width), dtype=torch.int32, device="cuda")
    same = shared // page
    at = same
    for b, n in enumerate(lens):
        t[b, :same] = ids[:same]
        m = max(0, -(-n // page) - same)
        t[b, same:same + m] = ids[at:at + m]
        at += m
    assert at <= n_pages
    return t


@pytest.mark.parametrize("dh,hq,hkv", [(64, 12, 12), (128, 8, 2), (128, 16, 1), (64, 6, 2), (128, 5, 1)])
@pytest.mark.parametrize("bits,page", [(8, 16), (4, 48), (8, 128), (4, 64)])
@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
def test_attention_single_tokens(dh, hq, hkv, bits, page, dt):
    g = _gen(dh + hq * 3 + bits)
    lens = [1, 0, 17, 16, 15, 700, 64, 33, 2]
    cache, kd, vd = _filled(g, hkv, dh, bits, page, 120 if page == 16 else 40)
    q = (torch.randn((len(lens), hq, dh), generator=g, device="cuda") * 2).to(dt)
    _attend(cache, kd, vd, q, [1] * len(lens), lens, _pages(g, lens, page, cache.n_pages))


@pytest.mark.parametrize("q_lens,lens", [([3, 1, 0, 5, 2], [3, 40, 9, 2, 130]), ([20, 33], [90, 33]), ([70], [333]), ([1, 130, 7], [257, 131, 64])])
@pytest.mark.parametrize("dh,hq,hkv,bits,page", [(128, 4, 1, 8, 16), (64, 3, 3, 4, 32), (64, 4, 2, 8, 64), (128, 6, 2, 4, 16)])
@pytest.mark.parametrize("window", [0, 1, 50])
def test_attention_chunks_and_windows(q_lens, lens, dh, hq, hkv, bits, page, window):
    g = _gen(sum(lens) + dh + window)
    cache, kd, vd = _filled(g, hkv, dh, bits, page, 50)
    q = torch.randn((sum(q_lens), hq, dh), generator=g, device="cuda").to(torch.float16)
    _attend(cache, kd, vd, q, q_lens, lens, _pages(g, lens, page, 50), window=window)


@pytest.mark.parametrize("q_lens,lens,shared", [([1] * 6, [300, 257, 256, 290, 400, 260], 256), ([2, 1, 3], [130, 128, 200], 128),
                                                ([1, 1], [20, 500], 64), ([40, 9], [160, 99], 64), ([1] * 3, [128] * 3, 128)])
@pytest.mark.parametrize("dh,hq,hkv,bits", [(128, 8, 2, 8), (64, 2, 2, 4)])
@pytest.mark.parametrize("window", [0, 100])
def test_attention_shared_prefix(q_lens, lens, shared, dh, hq, hkv, bits, window):
    """The same as without the hint (a sequence shorter than the prefix sees its part of it)."""
    g = _gen(sum(lens) + shared)
    cache, kd, vd = _filled(g, hkv, dh, bits, 64, 40)
    q = torch.randn((sum(q_lens), hq, dh), generator=g, device="cuda").to(torch.bfloat16)
    pages = _pages(g, [max(n, shared) for n in lens], 64, 40, shared)
    _attend(cache, kd, vd, q, q_lens, lens, pages, shared=shared, window=window)


def test_attention_long_and_split():
    g = _gen(2)
    lens = [20011, 8192]
    cache, kd, vd = _filled(g, 1, 128, 8, 64, 460)
    q = torch.randn((2, 4, 128), generator=g, device="cuda").to(torch.float16)
    pages = _pages(g, lens, 64, 460)
    _attend(cache, kd, vd, q, [1, 1], lens, pages)
    # hints that are too large or too small change the cuts, not the result
    _attend(cache, kd, vd, q, [1, 1], lens, pages, max_len=1 << 20)
    _attend(cache, kd, vd, q, [1, 1], lens, pages, max_len=16)


def test_attention_hidden_garbage_and_extreme_scales():
    """Slots past a sequence's end hold NaN scales; V rows of zeros, of 1e-6 and of 1e4 side by side; one key far ahead."""
    g = _gen(3)
    lens = [45, 100]
    cache, kd, vd = _filled(g, 2, 64, 8, 16, 20)
    pages = _pages(g, lens, 16, 20)
    for b, n in enumerate(lens):
        p, at = int(pages[b, n // 16]), n % 16
        for t in (cache.k_scales, cache.v_scales):
            t[p, :, at:] = math.nan
    p0 = int(pages[1, 0])
    for i, f in ((0, 0.0), (1, 1e-6), (2, 1e4), (3, 1e-30)):
        cache.v_scales[p0, :, i] *= f
    vd[p0] = (R.unpack(cache.v_codes[p0], 8) * cache.v_scales[p0].double()[..., None]).transpose(0, 1)
    q = torch.randn((2, 2, 64), generator=g, device="cuda").to(torch.float16)
    _attend(cache, kd, vd, q, [1, 1], lens, pages)
    cache.k_scales[p0, :, 5] *= 20
    kd[p0] = (R.unpack(cache.k_codes[p0], 8) * cache.k_scales[p0].double()[..., None]).transpose(0, 1)
    _attend(cache, kd, vd, q, [1, 1], lens, pages, scale=0.2)
    # all of a sequence's values zero: the output is zero, the log-sum-exp is not -inf
    cache.v_scales.zero_()
    vd.zero_()
    _attend(cache, kd, vd, q, [1, 1], lens, pages)


def test_attention_bf16_query_range():
    """bf16 queries outside fp16's range (1e30 and 1e-30) are used as they are."""
    g = _gen(4)
    cache, kd, vd = _filled(g, 1, 128, 8, 16, 10)
    q = torch.randn((1, 4, 128), generator=g, device="cuda")
    pages = _pages(g, [90], 16, 10)
    for f in (1e30, 1e-30, 1e-38):
        qq = (q * f).to(torch.bfloat16)
        _attend(cache, kd, vd, qq, [1], [90], pages, scale=float(0.1 / f) if f < 1e30 else 1e-31)
    qq = torch.zeros_like(q).to(torch.bfloat16)
    _attend(cache, kd, vd, qq, [1], [90], pages)


def test_attention_pitched_stream_and_repeat():
    g = _gen(6)
    lens = [333, 64, 1]
    cache, kd, vd = _filled(g, 2, 64, 4, 32, 20)
    wide = torch.randn((3, 4 * 64 + 24), generator=g, device="cuda").to(torch.bfloat16)
    q = wide[:, 8:8 + 256].view(3, 4, 64)
    res = torch.full((3, 304), 5.0, device="cuda", dtype=torch.bfloat16)
    pages = _pages(g, lens, 32, 20)
    torch.cuda.synchronize()
    o1, l1 = _attend(cache, kd, vd, q, [1] * 3, lens, pages, out=res[:, :256].view(3, 4, 64), stream=torch.cuda.Stream())
    assert bool((res[:, 256:] == 5).all())
    o2, l2 = _attend(cache, kd, vd, q, [1] * 3, lens, pages)
    assert torch.equal(o1, o2) and torch.equal(l1, l2)


def test_attention_past_32_bit_offsets():
    """A cache of more than 2^32 bytes of codes a side, its last pages in use."""
    hkv, dh, page = 8, 128, 64
    n_pages = (1 << 32) // (hkv * dh * page) + 40
    cache = J.KvCache(hkv, dh, 8, page, n_pages)
    g = _gen(8)
    top = 30
    small, kd, vd = _filled(g, hkv, dh, 8, page, top)
    for a, b in ((cache.k_codes, small.k_codes), (cache.v_codes, small.v_codes), (cache.k_scales, small.k_scales), (cache.v_scales, small.v_scales)):
        a[-top:] = b
    lens = [500, 1000]
    local = _pages(g, lens, page, top)
    q = torch.randn((2, 32, dh), generator=g, device="cuda").to(torch.float16)
    o1, _ = _attend(small, kd, vd, q, [1, 1], lens, local)
    out = torch.empty_like(q)
    ws = torch.empty(J.jab_kv_attention_workspace_size(cache, 2, 2, 32, 1, 1000), dtype=torch.uint8, device="cuda")
    J.jab_kv_attention(cache, q, torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"), (local + n_pages - top).int().contiguous(),
                       torch.tensor(lens, dtype=torch.int32, device="cuda"), out, ws, 1, 1000)
    assert torch.equal(out, o1)
    qkv = torch.randn((1, 16 * dh), generator=g, device="cuda")
    slot = torch.tensor([n_pages * page - 1], device="cuda")
    J.jab_kv_write(cache, qkv, 0, slot)
    c, s = R.quantize_rows(qkv.view(16, dh), 8)
    assert torch.equal(cache.v_codes[-1, :, -1], R.pack(c[8:], 8))
    k, v = (torch.empty((1, 1, hkv, dh), device="cuda") for _ in range(2))
    J.jab_kv_read(cache, torch.tensor([[n_pages - 1]], dtype=torch.int32, device="cuda"), torch.tensor([1], dtype=torch.int32, device="cuda"),
                  k, v, starts=torch.tensor([page - 1], dtype=torch.int32, device="cuda"))
    assert torch.equal(k[0, 0], (c[:8].float() * s[:8, None]))
    assert J.jab_get_device_status() == 0


def test_attention_bad_indices_are_reported():
    """Page numbers and lengths outside the cache: reported, nothing outside it is read."""
    cache, kd, vd = _filled(_gen(1), 1, 64, 8, 16, 4)
    q = torch.randn((1, 1, 64), device="cuda").to(torch.float16)
    out = torch.empty_like(q)
    ws = torch.empty(J.jab_kv_attention_workspace_size(cache, 1, 1, 1, 1, 64), dtype=torch.uint8, device="cuda")
    i = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    for pages, lens, start in ((i(9, 0), 20, (0, 1)), (i(-1, 0), 20, (0, 1)), (i(0, 1), 33, (0, 1)), (i(0, 1), -1, (0, 1)), (i(0, 1), 20, (0, 2)), (i(0, 1), 20, (-1, 1))):
        J.jab_kv_attention(cache, q, i(*start), pages.view(1, 2), i(lens), out, ws, 1, 64)
        assert J.jab_get_device_status() == 1, (pages, lens, start)


# 128-row tiles round a weight once in key tiles that no mask cuts (2^-11 of it); the rest of the bound as above.
def _attend_tiles(cache, kd, vd, q, q_lens, lens, pages, shared=0, window=0):
    n, hq, dh = q.shape
    q_start = torch.tensor([0] + list(torch.tensor(q_lens).cumsum(0)), dtype=torch.int32, device="cuda")
    out, lse = torch.full_like(q, 77.0), torch.full((n, hq), 77.0, device="cuda")
    ws = torch.full((J.jab_kv_attention_workspace_size(cache, len(lens), n, hq, max(q_lens), max(lens), shared),), 0xFF, dtype=torch.uint8,
                    device="cuda")
    J.jab_kv_attention(cache, q, q_start, pages, torch.tensor(lens, dtype=torch.int32, device="cuda"), out, ws, max(q_lens), max(lens),
                       shared_len=shared, window=window, lse=lse)
    assert J.jab_get_device_status() == 0
    at, page, hkv = 0, cache.page_tokens, cache.n_kv_heads
    for b, (nq, length) in enumerate(zip(q_lens, lens)):
        if nq == 0:
            continue
        j = torch.arange(length, device="cuda")
        ids = pages[b].long()[j // page]
        k, v = kd[ids, j % page], vd[ids, j % page]
        pos = torch.arange(length - nq, length, device="cuda")[:, None]
        seen = (j <= pos) & ((j > pos - window) if window else torch.ones_like(j <= pos))
        for h in range(hq):
            s = (q[at:at + nq, h].double() @ k[:, h // (hq // hkv)].t() / math.sqrt(dh)).masked_fill(~seen, -math.inf)
            ls = torch.logsumexp(s, -1)
            w = torch.where(seen, torch.exp(s - torch.where(ls > -math.inf, ls, 0.0)[:, None]), 0.0)
            vv = v[:, h // (hq // hkv)]
            o, mag = w @ vv, w @ vv.abs()
            tol = (2.0 ** -11 + 2.0 ** -16) * mag + length * 2.0 ** -25 * vv.abs().max() + HALF_ULP[q.dtype] * o.abs() + 1e-30
            err = (out[at:at + nq, h].double() - o).abs()
            assert bool((err <= tol).all()), (b, h, (err / tol).max().item())
            fin = ls > -math.inf
            got = lse[at:at + nq, h].double()
            assert bool((got[~fin] == -math.inf).all()) and bool(((got - ls).abs()[fin] <= 2.0 ** -16 + 2.0 ** -21 * ls.abs()[fin]).all())
        at += nq


@pytest.mark.parametrize("q_lens,lens,shared,window", [
    ([300, 77], [1000, 900], 0, 0),            # chunks behind a context, several row and key tiles
    ([513], [513], 0, 0),                      # a prompt from its first token
    ([129, 1, 40, 2], [700, 1500, 40, 3], 0, 0),   # a chunk, single tokens and a short prompt in one batch
    ([260, 33], [1700, 500], 0, 200),          # sliding window: key tiles before it are skipped
    ([100], [60], 0, 0),                       # more queries than tokens: the first rows see nothing
    ([1] * 40, [520 + 7 * i for i in range(40)], 512, 0),     # single tokens behind a prefix
    ([1] * 40, [520 + 7 * i for i in range(40)], 512, 300),
    ([50, 3, 70], [900, 785, 1001], 768, 0),   # chunks behind a prefix
    ([64, 64], [64, 300], 192, 0),             # a sequence shorter than the prefix
])
@pytest.mark.parametrize("dh,hq,hkv,bits,dt", [(128, 8, 2, 8, torch.float16), (64, 4, 4, 8, torch.bfloat16), (128, 6, 2, 4, torch.bfloat16),
                                               (64, 4, 1, 4, torch.float16)])
def test_attention_many_rows(q_lens, lens, shared, window, dh, hq, hkv, bits, dt):
    g = _gen(sum(lens) + dh + bits)
    page = 64 if shared else 48
    cache, kd, vd = _filled(g, hkv, dh, bits, page, sum(-(-max(n, shared) // page) for n in lens) + 3)
    q = torch.randn((sum(q_lens), hq, dh), generator=g, device="cuda").to(dt)
    pages = _pages(g, [max(n, shared) for n in lens], page, cache.n_pages, shared)
    for b, n in enumerate(lens):  # entries past a sequence's pages are not looked at
        pages[b, -(-max(n, shared) // page):] = -1
    _attend_tiles(cache, kd, vd, q, q_lens, lens, pages, shared=shared, window=window)


def test_attention_unused_table_entries():
    cache, kd, vd = _filled(_gen(1), 2, 64, 8, 16, 8)
    pages = torch.full((3, 4), -1, dtype=torch.int32, device="cuda")
    pages[1, 0], pages[2, :2] = 5, torch.tensor([1, 7], dtype=torch.int32, device="cuda")
    q = torch.randn((3, 4, 64), generator=_gen(2), device="cuda").to(torch.float16)
    _attend(cache, kd, vd, q, [1, 1, 1], [0, 9, 20], pages)


@pytest.mark.parametrize("dh,bits,page,q,longest,window", [(64, 8, 64, 33, 127, 0), (128, 4, 16, 34, 128, 0), (64, 4, 32, 40, 250, 20), (128, 8, 128, 33, 300, 0)])
def test_attention_many_short_items(dh, bits, page, q, longest, window):
    """Several row tiles of one or a few key tiles for every block: the parts of the kernel run ahead of each other."""
    g = _gen(q + longest)
    B, h = 84, 8
    lens = [q + (i * 37) % (longest - q + 1) for i in range(B)]
    cache, kd, vd = _filled(g, h, dh, bits, page, sum(-(-n // page) for n in lens) + 1)
    qs = torch.randn((B * q, h, dh), generator=g, device="cuda").to(torch.bfloat16)
    pages = _pages(g, lens, page, cache.n_pages)
    outs = []
    for _ in range(20):
        out, lse = torch.empty_like(qs), torch.empty((B * q, h), device="cuda")
        start = torch.arange(B + 1, dtype=torch.int32, device="cuda") * q
        ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
        ws = torch.empty(J.jab_kv_attention_workspace_size(cache, B, B * q, h, q, longest), dtype=torch.uint8, device="cuda")
        J.jab_kv_attention(cache, qs, start, pages, ln, out, ws, q, longest, window=window, lse=lse)
        outs.append((out, lse))
    assert J.jab_get_device_status() == 0
    assert all(torch.equal(o, outs[0][0]) and torch.equal(l, outs[0][1]) for o, l in outs)
    at = torch.arange(longest, device="cuda")
    for b in range(0, B, 9):
        n = lens[b]
        ids = pages[b].long()[at[:n] // page]
        o, ls, mag = R.attention(qs[b * q:(b + 1) * q].double(), kd[ids, at[:n] % page], vd[ids, at[:n] % page], window, 1 / math.sqrt(dh))
        tol = (2.0 ** -11 + 2.0 ** -16) * mag + n * 2.0 ** -25 * vd.abs().max() + HALF_ULP[qs.dtype] * o.abs() + 1e-30
        assert bool(((outs[0][0][b * q:(b + 1) * q].double() - o).abs() <= tol).all()), b
        assert bool(((outs[0][1][b * q:(b + 1) * q].double() - ls).abs() <= 2.0 ** -16 + 2.0 ** -21 * ls.abs()).all()), b
