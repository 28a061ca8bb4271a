"""The 8-bit floating-point projection and its quantiser on the GPU against plain float64 implementations.

Codes and scales are compared bit for bit: their roundings are part of the definition. A product instruction adds 32
products of codes to an accumulator; each addend is cut to 24 bits or more below the largest, so that 33 of them lose at
most 33 * 2^-24 of the sum of the magnitudes A, four instructions of a block less than 2^-16. Two products with
scales and one addition for each of nb blocks are fp32: (nb + 4) 2^-24 A. Then half a step of the result's type."""
import pytest
import torch

import more_ref as R

pytestmark = pytest.mark.gpu

import paper_2609_34866_gb300 as J  # noqa: E402

HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
F8 = torch.float8_e4m3fn
BF, HF, F = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(autouse=True)
def _status():
    J.jab_get_device_status()
    yield
    torch.cuda.synchronize()


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _quantize(x, rows):
    M, K = x.shape
    codes = torch.full((M, K), 1, dtype=torch.uint8, device="cuda").view(F8)
    scales = torch.full((-(-M // rows), -(-K // 128)), -7.0, device="cuda")
    J.jab_fp8_quantize(x, codes, scales, block_rows=rows)
    return codes, scales


@pytest.mark.parametrize("M,K", [(1, 16), (3, 128), (130, 144), (256, 1040), (700, 4096), (129, 2032), (4097, 64)])
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("dt", [BF, HF, F])
def test_quantize_bit_for_bit(M, K, rows, dt):
    g = _gen(M + K)
    x = torch.randn((M, K + 16), generator=g, device="cuda") * torch.rand((M, 1), generator=g, device="cuda") * 3
    x[:, ::7] *= 30
    x[M // 2] = 0
    x = x.to(dt)[:, 8 : 8 + K] if dt != F else x[:, 4 : 4 + K]  # (a pitch, and a start on 16 bytes)
    codes, scales = _quantize(x, rows)
    want, s = R.fp8(x.float(), rows)
    assert torch.equal(scales, s)
    assert torch.equal(codes.float().double(), want)
    assert J.jab_get_device_status() == 0


def test_quantize_every_rounding():
    """A block whose scale is 1 (largest 448): codes are e4m3 of the numbers themselves; all codes, the ties between them and
    the numbers beside the ties."""
    top = torch.arange(127, dtype=torch.uint8).view(F8).float()  # 0 .. 448
    mid = (top[1:] + top[:-1]) / 2
    v = torch.cat((top, mid, torch.nextafter(mid, mid + 1), torch.nextafter(mid, mid - 1)))
    v = torch.cat((v, -v))
    x = torch.full((1, 128 * 16), 448.0)
    n = 0
    for b in range(16):  # 127 numbers and a 448 a block
        part = v[127 * b : 127 * b + 127]
        x[0, 128 * b : 128 * b + len(part)] = part
        n += len(part)
    assert n == len(v)
    codes, scales = _quantize(x.cuda(), 1)
    assert torch.equal(scales, torch.ones_like(scales))
    assert torch.equal(codes.float().double(), R.e4m3(x.cuda().double()))


@pytest.mark.parametrize("dt,top", [(F, 3e38), (F, 1e-37), (F, 1e-44), (BF, 3e38), (BF, 1e-38), (HF, 6e-8)])
def test_quantize_scales_of_any_size(dt, top):
    x = (torch.randn((200, 256), generator=_gen(3), device="cuda").clamp(-1, 1) * top).to(dt)
    for rows in (1, 128):
        codes, scales = _quantize(x, rows)
        want, s = R.fp8(x.float(), rows)
        assert torch.equal(scales, s) and torch.equal(codes.float().double(), want)


@pytest.mark.parametrize("dt", [BF, HF, F])
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("exponent", [0, -14, 70, -90])
def test_quantize_signs_of_zeros(dt, rows, exponent):
    """The bytes themselves: zeros of both signs, and numbers of both signs that round to zero, beside scales that are divided by and scales
    whose reciprocal is taken."""
    if dt == HF and exponent not in (0, -14):
        pytest.skip("not in fp16")
    x = torch.randn((130, 400), generator=_gen(6), device="cuda").clamp(-1, 1)
    x[:, 1::4], x[:, 2::8], x[:, 6::8] = -0.0, 0.0, -(2.0 ** -20)
    x[:, 7::8] = 2.0 ** -20
    x[:, ::128] = 1.0
    x[3], x[4] = -0.0, 0.0
    x = (x * 2.0 ** exponent).to(dt)
    codes, scales = _quantize(x, rows)
    want, s = R.fp8(x.float(), rows)
    minus = torch.signbit(x.float()) & (R.spread(s, rows, *x.shape) > 0)
    top = torch.arange(127, dtype=torch.uint8, device="cuda")
    magnitude = torch.searchsorted(top.view(F8).double(), want.abs())  # (the numbers of codes 0 .. 126 in their order)
    assert torch.equal(codes.view(torch.uint8).long(), magnitude + 128 * minus) and torch.equal(scales, s)
    assert bool((codes.view(torch.uint8) == 0x80).any()) and J.jab_get_device_status() == 0


def test_quantize_nonfinite():
    x = torch.randn((300, 384), generator=_gen(4), device="cuda")
    x[5, 200], x[290, 0] = float("inf"), float("nan")
    codes, scales = _quantize(x, 128)
    bad = torch.zeros((3, 3), dtype=torch.bool, device="cuda")
    bad[0, 1] = bad[2, 0] = True
    assert torch.equal(scales.isnan(), bad)
    assert not codes[:128, 128:256].float().any() and codes[128:].float().isfinite().all()
    assert J.jab_get_device_status() == 4


# ------------------------------------------------------------------ product
def _weights(N, K, rows, g, kind="random"):
    if kind == "fit":  # whole-numbered codes of a fit at 5 bits in groups of 128
        codes = torch.randint(-15, 16, (N, K), generator=g, device="cuda").float().to(F8)
    else:
        codes = torch.randint(0, 256, (N, K), generator=g, device="cuda").to(torch.uint8)
        codes = torch.where(codes & 127 == 127, codes - 1, codes).view(F8)  # (no NaN)
    scales = torch.rand((-(-N // rows), -(-K // 128)), generator=g, device="cuda") * 0.01 + 1e-4
    return codes, scales


def _linear(x, codes, scales, rows, dt, y=None):
    (M, K), N = x.shape, codes.shape[0]
    y = torch.empty((M, N), dtype=dt, device="cuda") if y is None else y
    ws = torch.full((J.jab_fp8_linear_workspace_size(M, N, K),), 0xFF, dtype=torch.uint8, device="cuda")
    J.jab_fp8_linear(x, codes, scales, y, ws, block_rows=rows)
    return y


def _held(y, x, codes, scales, rows):
    want, mag = R.fp8_linear(x, codes, scales, rows)
    nb = scales.shape[1]
    tiny = 2.0 ** -24 if y.dtype == HF else 2.0 ** -126
    bound = mag * (2.0 ** -16 + (nb + 4) * 2.0 ** -24) * (1 + HALF_STEP[y.dtype]) + want.abs() * HALF_STEP[y.dtype] + tiny
    off = (y.double() - want).abs()
    assert bool((off <= bound).all()), float((off / bound).max())


SIZES = [(1, 128, 128), (1, 6144, 4096), (2, 100, 16), (7, 2304, 768), (16, 129, 80), (17, 1, 1040), (33, 384, 256), (64, 1000, 2064),
         (65, 2560, 1024), (128, 640, 8208), (129, 257, 4096), (300, 2304, 768), (1500, 1024, 512), (700, 6144, 4096), (3001, 6144, 640)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("xt,yt,rows,kind", [(BF, BF, 128, "random"), (HF, F, 1, "fit"), (F, HF, 1, "random"), (BF, F, 128, "random")])
def test_linear(M, N, K, xt, yt, rows, kind):
    g = _gen(M * 7 + N + K)
    x = torch.randn((M, K), generator=g, device="cuda") * 0.05
    x[:, :: max(1, K // 5)] *= 20
    x = x.to(xt)
    codes, scales = _weights(N, K, rows, g, kind)
    y = _linear(x, codes, scales, rows, yt)
    _held(y, x, codes, scales, rows)
    assert torch.equal(y, _linear(x, codes, scales, rows, yt))
    assert J.jab_get_device_status() == 0


@pytest.mark.parametrize("M,N,K", [(5, 25000, 272), (20, 21000, 144), (40, 25003, 272), (100, 30000, 400), (2600, 5003, 400), (4000, 4010, 16), (2700, 4872, 528),
                                   (2, 130, 131072), (130, 200, 65552)])
@pytest.mark.parametrize("yt,rows", [(BF, 128), (F, 1)])
def test_linear_many_tiles_for_a_block_and_long_sums(M, N, K, yt, rows):
    """More tiles than blocks at every tile size, odd numbers of channels, a single block of K, and the longest K."""
    g = _gen(M + N + K)
    x = (torch.randn((M, K), generator=g, device="cuda") * 0.05).to(HF)
    codes, scales = _weights(N, K, rows, g)
    y = _linear(x, codes, scales, rows, yt)
    _held(y, x, codes, scales, rows)
    assert torch.equal(y, _linear(x, codes, scales, rows, yt)) and J.jab_get_device_status() == 0


@pytest.mark.parametrize("M", [5, 40, 200, 1000])
@pytest.mark.parametrize("yt", [BF, F])
def test_linear_pitches_and_margins(M, yt):
    """Rows with pitches, an odd one for y; what lies around y stays."""
    N, K = 392, 272
    g = _gen(M)
    wide = torch.randn((M, K + 40), generator=g, device="cuda").to(HF)
    x = wide[:, 8 : 8 + K]
    codes, scales = _weights(N, K, 128, g)
    for pitch in (N + 8, N + 9):
        out = torch.full((M + 2, pitch), 7.0, dtype=yt, device="cuda")
        y = out[1 : M + 1, :N]
        _linear(x, codes, scales, 128, yt, y)
        _held(y, x, codes, scales, 128)
        assert bool((out[0] == 7).all() and (out[M + 1] == 7).all() and (out[1 : M + 1, N:] == 7).all())


def test_linear_serves_a_fitted_block():
    """Codes and scales of a fit in groups of 128, up to 5 bits, as they are: whole numbers are e4m3 numbers."""
    desc = J.BlockDesc(256, 4, 1, 64, 128, 1, 10000.0, 0.0)
    D = 6 * 64
    W = (torch.randn((D, 256), generator=_gen(1), device="cuda") * 0.02).to(BF)
    for bits in (2, 3, 4, 5):
        scales, codes = torch.empty((D, 2), device="cuda"), torch.empty((D, 256), dtype=torch.int8, device="cuda")
        J.jab_init_scales(desc, bits, 0, W, scales)
        J.jab_quantize(desc, bits, W, scales, codes=codes)
        c8 = codes.float().to(F8)
        assert torch.equal(c8.float(), codes.float())
        x = torch.randn((9, 256), generator=_gen(2), device="cuda").to(HF)
        _held(_linear(x, c8, scales, 1, F), x, c8, scales, 1)


def test_linear_zeros_and_nonfinite():
    g = _gen(9)
    x = torch.randn((70, 512), generator=g, device="cuda").to(BF)
    x[3], x[4, 130], x[69, 500] = 0, float("inf"), float("nan")
    codes, scales = _weights(300, 512, 1, g)
    y = _linear(x, codes, scales, 1, F)
    assert not y[3].any() and y[4].isnan().all() and y[69].isnan().all()
    rest = [i for i in range(70) if i not in (4, 69)]
    _held(y[rest], x[rest], codes, scales, 1)
    assert J.jab_get_device_status() == 4
    # a NaN weight is in its channel alone
    codes.view(torch.uint8)[7, 9] = 0x7F
    y = _linear(x[:2], codes, scales, 1, F)
    assert y[:, 7].isnan().all() and y[:, :7].isfinite().all() and y[:, 8:].isfinite().all()


@pytest.mark.parametrize("M,N,K", [(1, 129, 256), (1, 256, 2048), (40, 130, 2048), (130, 384, 2048), (130, 20000, 272), (3000, 1024, 256), (3000, 1021, 272)])
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("left_over", [0xFF, 0x7F])
def test_linear_results_that_do_not_fit_fp16(M, N, K, rows, left_over):
    """One result of 448 * 2 * 73.125 = 65520, halfway between the largest fp16 and what would come next, which rounds to an infinity;
    the fp32 below it rounds to 65504. Whatever the workspace holds."""
    ws = torch.empty(J.jab_fp8_linear_workspace_size(M, N, K), dtype=torch.uint8, device="cuda")
    for m, n, k, sign in ((0, 0, 0, 1), (M - 1, N - 1, K - 1, -1), (M // 2, N // 2, K // 2, 1)):
        x = torch.zeros((M, K), dtype=BF, device="cuda")
        codes, scales = torch.zeros((N, K), device="cuda"), torch.ones((-(-N // rows), -(-K // 128)), device="cuda")
        x[m, k], codes[n, k] = 448.0, 2.0 * sign
        edge = torch.tensor(73.125)
        for s, dt, status in ((edge, HF, 5), (torch.nextafter(edge, torch.zeros(())), HF, 0), (edge, BF, 0), (edge, F, 0), (edge * 1e30, HF, 5)):
            scales[n // rows, k // 128] = s
            ws.fill_(left_over)
            y = torch.full((M, N), 7.0, dtype=dt, device="cuda")
            J.jab_fp8_linear(x, codes.to(F8), scales, y, ws, block_rows=rows)
            assert J.jab_get_device_status() == status
            want = torch.zeros((M, N), device="cuda")
            want[m, n] = 896.0 * sign * s.item()
            assert torch.equal(y, want.to(dt))


def test_linear_in_a_graph_and_on_another_stream():
    g = _gen(11)
    x = torch.randn((37, 768), generator=g, device="cuda").to(HF)
    codes, scales = _weights(2304, 768, 1, g)
    y, ws = torch.zeros((37, 2304), device="cuda"), torch.empty(J.jab_fp8_linear_workspace_size(37, 2304, 768), dtype=torch.uint8, device="cuda")
    J.jab_fp8_linear(x, codes, scales, y, ws, block_rows=1)
    want = y.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        J.jab_fp8_linear(x, codes, scales, y, ws, block_rows=1)
    for _ in range(3):
        y.zero_()
        graph.replay()
        assert torch.equal(y, want)
    x.mul_(2)  # a replay reads what is there now
    graph.replay()
    assert torch.equal(y, 2 * want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y2, ws2 = torch.zeros_like(y), torch.empty_like(ws)
    J.jab_fp8_linear(x, codes, scales, y2, ws2, block_rows=1, stream=side)
    side.synchronize()
    assert torch.equal(y2, y)


@pytest.mark.parametrize("M", [3, 100, 700])
def test_linear_two_calls_at_once(M):
    """Two streams, buffers of their own: the values of one call after the other."""
    N, K = 2048, 1040
    sets = []
    for i in range(2):
        g = _gen(M + i)
        x = torch.randn((M, K), generator=g, device="cuda").to(BF)
        sets.append((x, *_weights(N, K, 128 if i else 1, g), torch.empty((M, N), dtype=BF, device="cuda"),
                     torch.empty(J.jab_fp8_linear_workspace_size(M, N, K), dtype=torch.uint8, device="cuda"), torch.cuda.Stream(), 128 if i else 1))
    want = [_linear(s[0], s[1], s[2], s[6], BF) for s in sets]
    torch.cuda.synchronize()
    for _ in range(20):
        for x, codes, scales, y, ws, st, rows in sets:
            J.jab_fp8_linear(x, codes, scales, y, ws, block_rows=rows, stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(s[3], w) for s, w in zip(sets, want)) and J.jab_get_device_status() == 0


def test_linear_without_rows_and_refusals():
    codes, scales = _weights(128, 256, 128, _gen(1))
    ws = torch.empty(J.jab_fp8_linear_workspace_size(4, 128, 256), dtype=torch.uint8, device="cuda")
    J.jab_fp8_linear(torch.empty((0, 256), dtype=BF, device="cuda"), codes, scales, torch.empty((0, 128), device="cuda"), ws)
    x, y = torch.zeros((4, 256), dtype=BF, device="cuda"), torch.zeros((4, 128), device="cuda")
    for bad in (lambda: J.jab_fp8_linear(x, codes.view(torch.uint8), scales, y, ws), lambda: J.jab_fp8_linear(x, codes, scales, y, ws, block_rows=1),
                lambda: J.jab_fp8_linear(x, codes, scales, y[:3], ws), lambda: J.jab_fp8_linear(x, codes, scales, y, ws, block_rows=64),
                lambda: J.jab_fp8_quantize(x, codes, scales)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(J.JabError):
        J.jab_fp8_linear(x, codes, scales, y, ws[:16])
