"""Norms and rotations of heads on the GPU, into the cache and not, with their gradients, against plain implementations.

Without a norm the forward is compared bit for bit (its roundings are the definition); with one, all but the rows whose factor is
rounded the other way, one in 2^16 or fewer: at most 2 + rows / 2^14 here. Against float64: the factor, two products and the
rotation's three roundings are 6 of 2^-24 (a factor rounded the other way 7) of |a c| + |b s|, then half a step of the type.
Gradients, each of at most 32 roundings in a chain (products with r, w, cos and sin, a sum of 16 products and one over 8
lanes): 2^-19 of the sums of magnitudes; a weight's gradient adds up `per` rows a thread, 32 to 64 heads and the blocks' parts
as pairs: (per + 64 + 8) 2^-24 more."""
import math

import pytest
import torch

import more_ref as R

pytestmark = pytest.mark.gpu

import paper_2609_34866_gb300 as J  # noqa: E402

BF, HF, F = torch.bfloat16, torch.float16, torch.float32
HALF_STEP = {HF: 2.0 ** -11, BF: 2.0 ** -8, F: 2.0 ** -24}


@pytest.fixture(autouse=True)
def _status():
    J.jab_get_device_status()
    yield
    torch.cuda.synchronize()


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _inputs(n, hq, hk, hv, dh, dt, part, seed, norm=True, length=600, pad=0):
    g = _gen(seed)
    x = torch.randn((n, (hq + hk + hv) * dh + pad), generator=g, device="cuda") * torch.exp(torch.randn((n, 1), generator=g, device="cuda"))
    x[:, 3] *= 30
    if n > 2:
        x[n // 2] = 0
    cos, sin = (t.float().cuda() for t in R.table(length, dh // part, 1e4))
    return dict(x=x.to(dt), pos=torch.randint(0, length, (n,), generator=g, device="cuda").int(), rope=(cos, sin),
                wq=1 + 0.3 * torch.randn(dh, generator=g, device="cuda") if norm else None,
                wk=1 + 0.3 * torch.randn(dh, generator=g, device="cuda") if norm else None, eps=1e-6 if norm else None)


def _how(s, inter):
    return dict(positions=s["pos"], rope=s["rope"], interleaved=inter, norm_eps=s["eps"], q_weight=s["wq"], k_weight=s["wk"])


def _want(s, hq, hk, dh, inter, fn=R.norm_rope, dt=F):
    h = s["x"][:, : (hq + hk) * dh].to(dt).reshape(-1, hq + hk, dh)
    w = None if s["wq"] is None else torch.cat((s["wq"].expand(hq, dh), s["wk"].expand(hk, dh))).to(dt)
    cos, sin = (t[s["pos"].long()].to(dt) for t in s["rope"])
    return fn(h, w, s["eps"], cos, sin, inter)


def _same_rows(got, want, norm):
    """got, want [rows, dh] in the output's type."""
    off = (got != want).any(-1).sum().item()
    assert off <= (2 + got.shape[0] // 2 ** 14 if norm else 0), off


CASES = [(1, 1, 1, 64), (1, 32, 8, 128), (3, 12, 12, 64), (64, 32, 8, 128), (37, 4, 1, 64), (1001, 12, 4, 128), (700, 5, 0, 64), (5, 0, 3, 128), (130, 96, 8, 128), (20, 300, 56, 64)]


@pytest.mark.parametrize("n,hq,hk,dh", CASES)
@pytest.mark.parametrize("dt", [BF, HF, F])
@pytest.mark.parametrize("part,inter,norm", [(1, False, True), (2, True, True), (4, False, False), (1, True, False), (4, True, True)])
def test_forward(n, hq, hk, dh, dt, part, inter, norm):
    s = _inputs(n, hq, hk, 1, dh, dt, part, n + hq, norm, pad=8)
    q = torch.full((n, hq * dh + 8), 3.0, dtype=dt, device="cuda")
    k = torch.full((n, hk * dh + 16), 3.0, dtype=dt, device="cuda")
    J.jab_qk_norm_rope(s["x"], hq, hk, dh, q[:, : hq * dh], k[:, : hk * dh], **_how(s, inter))
    got = torch.cat((q[:, : hq * dh], k[:, : hk * dh]), 1).view(n, hq + hk, dh)
    want = _want(s, hq, hk, dh, inter)
    _same_rows(got.reshape(-1, dh), want.to(dt).reshape(-1, dh), norm)
    if hq:
        assert bool((q[:, hq * dh :] == 3).all())
    if hk:
        assert bool((k[:, hk * dh :] == 3).all())
    exact = _want(s, hq, hk, dh, inter, R.norm_rope64, torch.float64)
    mag = _want(dict(s, rope=tuple(t.abs() for t in s["rope"]), x=s["x"].abs(), wq=None if not norm else s["wq"].abs(), wk=None if not norm else s["wk"].abs()),
                hq, hk, dh, inter, _sums, torch.float64)
    bound = mag * 7 * 2.0 ** -24 * 1.01 + exact.abs() * HALF_STEP[dt] * 1.01 + (2.0 ** -24 if dt == HF else 2.0 ** -126)
    assert bool(((got.double() - exact).abs() <= bound).all())
    assert J.jab_get_device_status() == 0


def _sums(x, w, eps, cos, sin, inter):
    """|a c| + |b s| of everything that norm_rope64 adds up, from magnitudes."""
    x = R.norm_rope64(x, w, eps, None, None, inter)
    half = cos.shape[-1]
    t, rest = x[..., : 2 * half], x[..., 2 * half :]
    a, b = (t[..., 0::2], t[..., 1::2]) if inter else (t[..., :half], t[..., half:])
    c, s = cos[:, None], sin[:, None]
    y, z = a * c + b * s, b * c + a * s
    return torch.cat((torch.stack((y, z), -1).flatten(-2) if inter else torch.cat((y, z), -1), rest), -1)


def test_forward_in_place():
    s = _inputs(300, 12, 4, 4, 128, BF, 1, 5)
    q, k = (torch.empty((300, h * 128), dtype=BF, device="cuda") for h in (12, 4))
    J.jab_qk_norm_rope(s["x"], 12, 4, 128, q, k, **_how(s, False))
    v = s["x"][:, 16 * 128 :].clone()
    J.jab_qk_norm_rope(s["x"], 12, 4, 128, s["x"][:, : 12 * 128], s["x"][:, 12 * 128 : 16 * 128], **_how(s, False))
    assert torch.equal(s["x"], torch.cat((q, k, v), 1))


def test_norm_without_weights_or_rotation():
    s = _inputs(50, 4, 2, 0, 64, F, 1, 6)
    q, k = (torch.empty((50, h * 64), device="cuda") for h in (4, 2))
    J.jab_qk_norm_rope(s["x"], 4, 2, 64, q, k, norm_eps=1e-5)
    want = R.norm_rope(s["x"].view(50, 6, 64), None, 1e-5, None, None, False)
    _same_rows(torch.cat((q, k), 1).reshape(-1, 64), want.reshape(-1, 64), True)
    J.jab_qk_norm_rope(s["x"], 4, 2, 64, q, k)  # nothing at all: a copy
    assert torch.equal(torch.cat((q, k), 1), s["x"])


@pytest.mark.parametrize("eps", [1e-30, 1e-5, 10.0, 1e30])
@pytest.mark.parametrize("size", [1e-12, 1.0, 1e15])
def test_norm_of_any_size(eps, size):
    x = torch.randn((400, 128), generator=_gen(7), device="cuda") * size
    q, k = torch.empty_like(x[:, :64]).contiguous(), torch.empty_like(x[:, :64]).contiguous()
    J.jab_qk_norm_rope(x, 1, 1, 64, q, k, norm_eps=eps)
    want = R.norm_rope(x.view(-1, 2, 64), None, eps, None, None, False)
    _same_rows(torch.stack((q, k), 1).view(-1, 64), want.reshape(-1, 64), True)
    assert J.jab_get_device_status() == 0


def test_norm_nonfinite_and_positions_out_of_range():
    x = torch.randn((6, 128), generator=_gen(8), device="cuda")
    x[1, 5], x[2, 70], x[3, 0] = float("nan"), float("inf"), 1e25  # (the square of the last leaves fp32)
    q, k = torch.zeros((6, 64), device="cuda"), torch.zeros((6, 64), device="cuda")
    J.jab_qk_norm_rope(x, 1, 1, 64, q, k, norm_eps=1e-6)
    nan = torch.stack((q.isnan().all(1), k.isnan().all(1)), 1).cpu().tolist()
    assert nan == [[False, False], [True, False], [False, True], [True, False], [False, False], [False, False]]
    assert J.jab_get_device_status() == 4
    s = _inputs(6, 1, 1, 0, 64, F, 1, 9, length=10)
    s["pos"][:] = torch.tensor([0, 9, 10, -1, 2 ** 31 - 1, 3], dtype=torch.int32)
    q.fill_(5), k.fill_(5)
    J.jab_qk_norm_rope(s["x"], 1, 1, 64, q, k, **_how(s, False))
    assert (q == 5).all(1).cpu().tolist() == [False, False, True, True, True, False]
    assert J.jab_get_device_status() == 1
    dx, dw = torch.full_like(x, 5), torch.zeros(64, device="cuda")
    ws = torch.empty(J.jab_qk_norm_rope_backward_workspace_size(6, 1, 1, 64), dtype=torch.uint8, device="cuda")
    dy = torch.ones_like(q)
    J.jab_qk_norm_rope_backward(s["x"], 1, 1, 64, dy, dy, dx, ws, dq_weight=dw, **_how(s, False))
    assert (dx == 5).all(1).cpu().tolist() == [False, False, True, True, True, False]
    assert J.jab_get_device_status() == 1
    s["x"][3] = float("nan")  # whatever such a token holds
    with_nan = torch.zeros_like(dw)
    J.jab_qk_norm_rope_backward(s["x"], 1, 1, 64, dy, dy, dx, ws, dq_weight=with_nan, **_how(s, False))
    assert torch.equal(with_nan, dw) and J.jab_get_device_status() == 1
    keep = torch.tensor([0, 1, 5], device="cuda")
    t = dict(s, x=s["x"][keep].contiguous(), pos=s["pos"][keep].contiguous())
    only = torch.zeros_like(dw)
    J.jab_qk_norm_rope_backward(t["x"], 1, 1, 64, dy[:3], dy[:3], torch.empty_like(t["x"]), ws, dq_weight=only, **_how(t, False))
    assert torch.allclose(dw, only, rtol=0, atol=3 * 2.0 ** -24 * 3 * 8 * 2)  # three rows of |g x r| < 8 in another order


# ------------------------------------------------------------------ into the cache
@pytest.mark.parametrize("n,hq,hk,dh,page", [(1, 32, 8, 128, 64), (64, 32, 8, 128, 64), (1001, 12, 12, 64, 16), (333, 4, 1, 64, 48), (700, 12, 4, 128, 32)])
@pytest.mark.parametrize("dt,bits", [(BF, 8), (HF, 4), (F, 8)])
@pytest.mark.parametrize("part,inter,norm", [(1, False, True), (2, True, True), (4, False, False), (1, True, False)])
def test_write(n, hq, hk, dh, page, dt, bits, part, inter, norm):
    s = _inputs(n, hq, hk, hk, dh, dt, part, n, norm)
    pages = -(-n // page) + 2
    cache = J.KvCache(hk, dh, bits, page, pages)
    slots = torch.randperm(pages * page, generator=_gen(n), device="cuda")[:n].contiguous()
    slots[n // 3] = -1
    q = torch.zeros((n, hq * dh), dtype=dt, device="cuda")
    J.jab_kv_write_norm_rope(cache, s["x"], hq, slots, q_out=q, **_how(s, inter))
    want = _want(s, hq, hk, dh, inter)
    live = slots >= 0
    _same_rows(q.view(n, hq, dh)[live].reshape(-1, dh), want[:, :hq].to(dt)[live].reshape(-1, dh), norm)
    v = s["x"].float()[:, (hq + hk) * dh :].reshape(n, hk, dh)
    at = slots[live]
    for rows, codes, scales, normed in ((want[:, hq:], cache.k_codes, cache.k_scales, norm), (v, cache.v_codes, cache.v_scales, False)):
        qmax = 2 ** (bits - 1) - 1
        sc = rows.abs().amax(-1) / torch.full((), float(qmax), device="cuda")
        c = torch.round(rows / sc[..., None]).clamp(-qmax, qmax)
        c = torch.where(sc[..., None] > 0, c, torch.zeros_like(c)).long() + 2 ** (bits - 1)
        c = c if bits == 8 else c[..., 0::2] + 16 * c[..., 1::2]
        got_c, got_s = codes[at // page, :, at % page], scales[at // page, :, at % page]
        off = ((got_c.long() != c[live]).any(-1) | (got_s != sc[live])).sum().item()
        assert off <= (2 + n * hk // 2 ** 14 if normed else 0), off
    touched = torch.zeros((pages, page), dtype=torch.bool, device="cuda")
    touched[at // page, at % page] = True
    assert not cache.k_scales.transpose(1, 2)[~touched].any() and not cache.v_codes.transpose(1, 2)[~touched].any()
    assert J.jab_get_device_status() == 0


def _near(got, exact, mag, dt):
    """Outputs in type dt: seven roundings of 2^-24 of the magnitudes (the norm's factor rounded the other way is two of them), then half
    a step."""
    bound = mag * 7 * 2.0 ** -24 * 1.01 + exact.abs() * HALF_STEP[dt] * 1.01 + (2.0 ** -24 if dt == HF else 2.0 ** -126)
    assert bool(((got.double() - exact).abs() <= bound).all())


def _written(codes, scales, bits, exact, mag):
    """Codes and scales of rows [..., dh] against the 64-bit rows: a scale is the largest element (off by e) over qmax, rounded; a code
    lies within half a step of the element over its scale, the element off by e and the quotient by 2^-24 of itself."""
    qmax = 2 ** (bits - 1) - 1
    c = (codes if bits == 8 else torch.stack((codes & 15, codes >> 4), -1).flatten(-2)).double() - 2 ** (bits - 1)
    e, s = mag * 7 * 2.0 ** -24 * 1.01, scales.double()
    assert bool(((s - exact.abs().amax(-1) / qmax).abs() <= e.amax(-1) / qmax * 1.01 + s * 2.0 ** -24 * 1.01).all())
    zero = s == 0
    assert not c[zero].any() and not exact[zero].any()
    c, e, exact, s = c[~zero], e[~zero], exact[~zero], s[~zero][:, None]
    assert bool((c.abs() <= qmax).all()) and bool(((c - exact / s).abs() <= 0.5 + e / s + (exact / s).abs() * 2.0 ** -24 * 1.01).all())


def _ones(s):
    """The weights that a missing one stands for."""
    one = torch.ones_like(s["wq"] if s["wq"] is not None else s["wk"]) if s["wq"] is not None or s["wk"] is not None else None
    return dict(s, wq=one if s["wq"] is None else s["wq"], wk=one if s["wk"] is None else s["wk"])


def _exact(s, hq, hk, dh, inter):
    """(outputs, magnitudes) of the heads of Q and K in 64 bits."""
    s = _ones(s)
    a = dict(s, x=s["x"].abs(), rope=tuple(t.abs() for t in s["rope"]), wq=None if s["wq"] is None else s["wq"].abs(), wk=None if s["wk"] is None else s["wk"].abs())
    return _want(s, hq, hk, dh, inter, R.norm_rope64, torch.float64), _want(a, hq, hk, dh, inter, _sums, torch.float64)


def _check_write(s, n, hq, hk, dh, dt, bits, page, inter, slots):
    """Every row that has a slot, Q and cache, within bounds of the 64-bit values; nothing else is touched."""
    pages = -(-(int(slots.max()) + 1) // page) + 1
    cache = J.KvCache(hk, dh, bits, page, pages)
    q = torch.full((n, hq * dh), 3.0, dtype=dt, device="cuda")
    J.jab_kv_write_norm_rope(cache, s["x"], hq, slots, q_out=q, **_how(s, inter))
    exact, mag = _exact(s, hq, hk, dh, inter)
    live = slots >= 0
    assert bool(live.any())
    _near(q.view(n, hq, dh)[live], exact[live, :hq], mag[live, :hq], dt)
    assert bool((q[~live] == 3).all())
    at = slots[live]
    v = s["x"].double()[:, (hq + hk) * dh : (hq + 2 * hk) * dh].reshape(n, hk, dh)[live]
    take = lambda t: t[at // page, :, at % page]  # noqa: E731
    _written(take(cache.k_codes), take(cache.k_scales), bits, exact[live, hq:], mag[live, hq:])
    _written(take(cache.v_codes), take(cache.v_scales), bits, v, torch.zeros_like(v))
    touched = torch.zeros((pages, page), dtype=torch.bool, device="cuda")
    touched[at // page, at % page] = True
    for t in cache._tensors:
        assert not t.transpose(1, 2)[~touched].any()
    assert J.jab_get_device_status() == 0


@pytest.mark.parametrize("n,hq,hk,dh,page", [(1, 32, 8, 128, 64), (1, 4, 1, 64, 16), (1, 1, 3, 128, 48), (2, 12, 12, 64, 16), (130, 5, 1, 64, 32), (700, 12, 4, 128, 16)])
@pytest.mark.parametrize("dt,bits", [(BF, 8), (BF, 4), (HF, 8), (HF, 4), (F, 8), (F, 4)])
@pytest.mark.parametrize("part,inter,norm", [(1, False, True), (2, True, True), (4, False, False), (1, True, False)])
def test_write_of_every_row(n, hq, hk, dh, page, dt, bits, part, inter, norm):
    s = _inputs(n, hq, hk, hk, dh, dt, part, n + 3, norm)
    slots = torch.randperm((n // page + 2) * page, generator=_gen(n), device="cuda")[:n].contiguous()
    if n > 2:
        slots[n // 3] = -1
    _check_write(s, n, hq, hk, dh, dt, bits, page, inter, slots)


WIDTHS = [(128, w) for w in range(16, 129, 16)] + [(64, w) for w in range(16, 65, 16)]


@pytest.mark.parametrize("dh,rotary", WIDTHS)
@pytest.mark.parametrize("dt", [BF, HF, F])
@pytest.mark.parametrize("inter", [False, True])
def test_rotations_of_every_width(dh, rotary, dt, inter):
    """Forward, gradient and cache for every number of elements that may be turned, with and without a norm."""
    n, hq, hk = 45, 5, 2
    for norm in (False, True):
        s = _inputs(n, hq, hk, hk, dh, dt, 1, rotary, norm)
        s["rope"] = tuple(t.float().cuda() for t in R.table(600, rotary, 1e4))
        q, k = (torch.full((n, h * dh), 3.0, dtype=dt, device="cuda") for h in (hq, hk))
        J.jab_qk_norm_rope(s["x"], hq, hk, dh, q, k, **_how(s, inter))
        got = torch.cat((q, k), 1).view(n, hq + hk, dh)
        _near(got, *_exact(s, hq, hk, dh, inter), dt)
        _same_rows(got.reshape(-1, dh), _want(s, hq, hk, dh, inter).to(dt).reshape(-1, dh), norm)
        for bits in (8, 4):
            _check_write(s, n, hq, hk, dh, dt, bits, 16, inter, torch.randperm(48, generator=_gen(1), device="cuda")[:n].contiguous())
        _check_backward(s, n, hq, hk, dh, dt, inter)


def _check_backward(s, n, hq, hk, dh, dt, inter):
    """dx and the weights' gradients (of the weights that there are, or of all) against autograd in 64 bits: bounds as in test_backward,
    for fewer than 256 tokens (a thread adds up at most two rows)."""
    norm = s["eps"] is not None
    g = _gen(n)
    dq, dk = ((torch.randn((n, h * dh), generator=g, device="cuda")).to(dt) for h in (hq, hk))
    dx, dwq, dwk = _backward(s, hq, hk, dh, dq, dk, inter, norm)
    x = s["x"][:, : (hq + hk) * dh].double().reshape(n, hq + hk, dh).requires_grad_()
    cos, sin = (t[s["pos"].long()].double() for t in s["rope"])
    one = torch.ones(dh, device="cuda")
    ws = [(one if s[k] is None else s[k]).double().requires_grad_() for k in ("wq", "wk")] if norm else []
    w = torch.cat((ws[0].expand(hq, dh), ws[1].expand(hk, dh))) if norm else None
    R.norm_rope64(x, w, s["eps"], cos, sin, inter).backward(torch.cat((dq, dk), 1).double().view(n, hq + hk, dh))
    mag = gm = _sums(torch.cat((dq, dk), 1).double().view(n, hq + hk, dh).abs(), None, None, cos.abs(), sin.abs(), inter)
    if norm:
        r = 1 / torch.sqrt(x.detach().square().mean(-1, keepdim=True) + 1e-6)
        xn, um = (x.detach() * r).abs(), gm * w.detach().abs()
        mag = r * (um + xn * (um * xn).mean(-1, keepdim=True))
        for got, want, sl in ((dwq, ws[0].grad, slice(0, hq)), (dwk, ws[1].grad, slice(hq, None))):
            top = (gm * xn)[:, sl].sum((0, 1))
            assert bool(((got.double() - want).abs() <= top * (2.0 ** -19 + 74 * 2.0 ** -24) + 2.0 ** -126).all())
    bound = mag * 2.0 ** -19 + x.grad.abs() * HALF_STEP[dt] * 1.01 + (2.0 ** -24 if dt == HF else 2.0 ** -126)
    assert bool(((dx.double().view_as(x) - x.grad).abs() <= bound).all()) and J.jab_get_device_status() == 0


@pytest.mark.parametrize("dt", [BF, HF, F])
@pytest.mark.parametrize("which", ["wq", "wk", "neither"])
def test_weights_of_q_or_of_k_alone(dt, which):
    n, hq, hk, dh = 60, 6, 2, 128
    s = _inputs(n, hq, hk, hk, dh, dt, 2, 8)
    for k in ("wq", "wk"):
        if k != which:
            s[k] = None
    q, k = (torch.empty((n, h * dh), dtype=dt, device="cuda") for h in (hq, hk))
    J.jab_qk_norm_rope(s["x"], hq, hk, dh, q, k, **_how(s, True))
    _near(torch.cat((q, k), 1).view(n, hq + hk, dh), *_exact(s, hq, hk, dh, True), dt)
    _check_write(s, n, hq, hk, dh, dt, 8, 32, True, torch.arange(n, device="cuda"))
    _check_backward(s, n, hq, hk, dh, dt, True)


@pytest.mark.parametrize("eps", [1e-30, 1e-5, 10.0, 1e30])
@pytest.mark.parametrize("size", [1e-12, 1.0, 1e15, 1e18])
def test_norm_of_any_size_in_64_bits(eps, size):
    """Every row: the factor at most two of 2^-24 off, the product one."""
    x = torch.randn((400, 128), generator=_gen(7), device="cuda").clamp(-2, 2) * size
    q, k = torch.empty_like(x[:, :64]).contiguous(), torch.empty_like(x[:, :64]).contiguous()
    J.jab_qk_norm_rope(x, 1, 1, 64, q, k, norm_eps=eps)
    want = R.norm_rope64(x.double().view(-1, 2, 64), None, eps, None, None, False)
    assert bool(((torch.stack((q, k), 1).double() - want).abs() <= want.abs() * 3 * 2.0 ** -24 * 1.01 + 2.0 ** -126).all())
    assert J.jab_get_device_status() == 0


def test_write_without_norm_is_the_plain_write():
    s = _inputs(200, 12, 4, 4, 128, HF, 1, 3, norm=False)
    a, b = (J.KvCache(4, 128, 8, 32, 8) for _ in range(2))
    slots = torch.arange(200, device="cuda")
    qa, qb = (torch.empty((200, 12 * 128), dtype=HF, device="cuda") for _ in range(2))
    J.jab_kv_write(a, s["x"], 12, slots, q_out=qa, positions=s["pos"], rope=s["rope"])
    J.jab_kv_write_norm_rope(b, s["x"], 12, slots, q_out=qb, positions=s["pos"], rope=s["rope"])
    assert torch.equal(qa, qb) and all(torch.equal(u, v) for u, v in zip(a._tensors, b._tensors))
    J.jab_kv_write_norm_rope(b, s["x"], 12, slots, positions=s["pos"], rope=s["rope"])  # Q is not wanted
    assert all(torch.equal(u, v) for u, v in zip(a._tensors, b._tensors))
    assert J.jab_get_device_status() == 0


# ------------------------------------------------------------------ gradients
def _backward(s, hq, hk, dh, dq, dk, inter, weights=True):
    n = s["x"].shape[0]
    dx = torch.full((n, (hq + hk) * dh + 8), 3.0, dtype=s["x"].dtype, device="cuda")
    dwq, dwk = (torch.full((dh,), 9.0, device="cuda") if weights else None for _ in range(2))
    ws = torch.full((J.jab_qk_norm_rope_backward_workspace_size(n, hq, hk, dh),), 0xFF, dtype=torch.uint8, device="cuda")
    J.jab_qk_norm_rope_backward(s["x"], hq, hk, dh, dq, dk, dx, ws if weights else None, dq_weight=dwq, dk_weight=dwk, **_how(s, inter))
    assert bool((dx[:, (hq + hk) * dh :] == 3).all())
    return dx[:, : (hq + hk) * dh], dwq, dwk


@pytest.mark.parametrize("n,hq,hk,dh", CASES + [(5000, 2, 1, 64)])
@pytest.mark.parametrize("dt", [BF, HF, F])
@pytest.mark.parametrize("part,inter,norm", [(1, False, True), (2, True, True), (4, False, False)])
def test_backward(n, hq, hk, dh, dt, part, inter, norm):
    s = _inputs(n, hq, hk, 1, dh, dt, part, n + 1, norm)
    g = _gen(n)
    dq, dk = ((torch.randn((n, h * dh + 8), generator=g, device="cuda")).to(dt)[:, : h * dh] for h in (hq, hk))
    dx, dwq, dwk = _backward(s, hq, hk, dh, dq, dk, inter, norm)
    # the formula, by autograd in 64 bits
    x = s["x"][:, : (hq + hk) * dh].double().reshape(n, hq + hk, dh).requires_grad_()
    ws = [None if not norm else s[k].double().requires_grad_() for k in ("wq", "wk")]
    w = None if not norm else torch.cat((ws[0].expand(hq, dh), ws[1].expand(hk, dh)))
    cos, sin = (t[s["pos"].long()].double() for t in s["rope"])
    y = R.norm_rope64(x, w, s["eps"], cos, sin, inter)
    dy = torch.cat((dq, dk), 1).double().view(n, hq + hk, dh)
    y.backward(dy)
    # magnitudes
    gm = _sums(dy.abs(), None, None, cos.abs(), sin.abs(), inter)
    if norm:
        r = 1 / torch.sqrt(x.detach().square().mean(-1, keepdim=True) + 1e-6)
        xn = (x.detach() * r).abs()
        um = gm * w.detach().abs()
        mag = r * (um + xn * (um * xn).mean(-1, keepdim=True))
    else:
        mag = gm
    bound = mag * 2.0 ** -19 + x.grad.abs() * HALF_STEP[dt] * 1.01 + (2.0 ** -24 if dt == HF else 2.0 ** -126)
    assert bool(((dx.double().view_as(x) - x.grad).abs() <= bound).all())
    if norm:
        heads_a_block = 256 // (dh // 16)
        per = -(-n // max(1, 304 // -(-(hq + hk) // heads_a_block)))  # (two blocks an SM at least)
        for got, want, sl in ((dwq, ws[0], slice(0, hq)), (dwk, ws[1], slice(hq, None))):
            want = torch.zeros(dh, device="cuda", dtype=torch.float64) if want.grad is None else want.grad
            top = (gm * xn)[:, sl].sum((0, 1))
            assert bool(((got.double() - want).abs() <= top * (2.0 ** -19 + (per + 72) * 2.0 ** -24) + 2.0 ** -126).all())
    again = _backward(s, hq, hk, dh, dq, dk, inter, norm)
    assert torch.equal(again[0], dx) and (not norm or (torch.equal(again[1], dwq) and torch.equal(again[2], dwk)))
    assert J.jab_get_device_status() == 0


def test_backward_against_differences():
    """The slope of sum(c y) along a direction v: differences of the 64-bit forward at h = 2^-12 are h^2 / 6 of the third derivative
    off, some 2^-24 of the terms' magnitudes here; the kernel's fp32 gradient 2^-19 of them: 2^-18 of the sum of |dx v| in all."""
    n, hq, hk, dh = 20, 3, 2, 64
    s = _inputs(n, hq, hk, 0, dh, F, 2, 4)
    s["x"] = torch.randn((n, 5 * dh), generator=_gen(1), device="cuda")
    c = torch.randn((n, 5, dh), generator=_gen(2), device="cuda")
    v = torch.randn((n, 5, dh), generator=_gen(3), device="cuda").double()
    dq, dk = c[:, :3].reshape(n, -1).contiguous(), c[:, 3:].reshape(n, -1).contiguous()
    dx, dwq, dwk = _backward(s, hq, hk, dh, dq, dk, True)
    x = s["x"].double().view(n, 5, dh)
    cos, sin = (t[s["pos"].long()].double() for t in s["rope"])

    def f(x, wq, wk):
        w = torch.cat((wq.expand(3, dh), wk.expand(2, dh)))
        return (R.norm_rope64(x, w, s["eps"], cos, sin, True) * c.double()).sum().item()

    wq, wk, h = s["wq"].double(), s["wk"].double(), 2.0 ** -12
    dx = dx.double().view_as(x)
    assert abs((f(x + h * v, wq, wk) - f(x - h * v, wq, wk)) / (2 * h) - (dx * v).sum().item()) <= 2.0 ** -18 * (dx * v).abs().sum().item()
    u = v[0, 0]
    for got, a, b in ((dwq, (wq + h * u, wk), (wq - h * u, wk)), (dwk, (wq, wk + h * u), (wq, wk - h * u))):
        assert abs((f(x, *a) - f(x, *b)) / (2 * h) - (got.double() * u).sum().item()) <= 2.0 ** -16 * (got.double() * u).abs().sum().item()


def test_results_that_do_not_fit_fp16():
    x = torch.randn((9, 128), generator=_gen(5), device="cuda").to(HF)
    big, q, k = torch.full((64,), 1e6, device="cuda"), torch.empty((9, 64), dtype=HF, device="cuda"), torch.empty((9, 64), dtype=HF, device="cuda")
    J.jab_qk_norm_rope(x, 1, 1, 64, q, k, norm_eps=1e-6, k_weight=big)
    assert J.jab_get_device_status() == 5
    J.jab_qk_norm_rope_backward(x, 1, 1, 64, torch.ones_like(q), torch.ones_like(k) + k.sign(), torch.empty_like(x), norm_eps=1e-6, q_weight=big)
    assert J.jab_get_device_status() == 5
    J.jab_qk_norm_rope_backward(x, 1, 1, 64, torch.ones_like(q), torch.ones_like(k), torch.empty_like(x), norm_eps=1e-6)
    assert J.jab_get_device_status() == 0


def test_backward_of_no_tokens():
    dw = torch.full((128,), 9.0, device="cuda")
    x = torch.empty((0, 512), dtype=BF, device="cuda")
    ws = torch.empty(J.jab_qk_norm_rope_backward_workspace_size(0, 2, 1, 128), dtype=torch.uint8, device="cuda")
    J.jab_qk_norm_rope_backward(x, 2, 1, 128, x[:, :256], x[:, :128], x, ws, norm_eps=1e-6, dk_weight=dw)
    assert not dw.any()
    J.jab_qk_norm_rope(x, 2, 1, 128, x[:, :256], x[:, :128], norm_eps=1e-6)


# ------------------------------------------------------------------ tables
@pytest.mark.parametrize("length,dim", [(1, 16), (37, 48), (5000, 128), (131072, 64)])
@pytest.mark.parametrize("how", [dict(), dict(kind="linear", factor=4.0), dict(kind="by_parts", factor=8.0, original_length=4096.0, attention=1.2),
                                 dict(kind="by_parts", factor=8.0, original_length=8192.0, low_turns=1.0, high_turns=4.0)])
def test_tables(length, dim, how):
    """Angles in 64 bits: the table is within half a step of fp32 of the 64-bit one, and 2^-33 for the angles' rounding (2^17 positions
    times 2^-53 and sixteen rotations on each side)."""
    cos, sin = (torch.empty((length, dim // 2), device="cuda") for _ in range(2))
    J.jab_rope_table_scaled(cos, sin, 500000.0, **how)
    att = torch.tensor(how.get("attention", 1.0), dtype=torch.float32).double().item()
    want = R.table(length, dim, 500000.0, how.get("kind", "plain"), how.get("factor", 1.0), how.get("original_length", 0.0), how.get("low_turns", 1.0),
                   how.get("high_turns", 32.0), att)
    for got, w in zip((cos, sin), want):
        assert bool(((got.cpu().double() - w).abs() <= w.abs() * 2.0 ** -24 + 2.0 ** -33).all())


def test_plain_table_is_the_table():
    a, b = ([torch.empty((700, 64), device="cuda") for _ in range(2)] for _ in range(2))
    J.jab_rope_table(*a, 10000.0)
    J.jab_rope_table_scaled(*b, 10000.0)
    assert bool((torch.stack(a) - torch.stack(b)).abs().max() <= 2.0 ** -24)


def test_the_longest_table():
    """Every length that the call takes. Positions of 2^31 over pi are rounded twice to 2^-53 of themselves: 2^-22 of the angle, and half a
    step of fp32."""
    if torch.cuda.mem_get_info()[0] < 160 << 30:
        pytest.skip("139 GB of tables")
    length = 2 ** 31 - 1
    cos, sin = (torch.empty((length, 8), device="cuda") for _ in range(2))
    try:
        cos[-40:], sin[-40:] = 7.0, 7.0
        J.jab_rope_table_scaled(cos, sin, 1e4)
        for p in (0, 1, 2 ** 30 + 3, length - 17, length - 16, length - 15, length - 1):
            assert abs(cos[p, 0].item() - math.cos(p)) <= 2.0 ** -21 and abs(sin[p, 0].item() - math.sin(p)) <= 2.0 ** -21, p
        assert bool((cos[-40:].square() + sin[-40:].square() - 1).abs().max() <= 2.0 ** -22)
    finally:
        del cos, sin
        torch.cuda.empty_cache()
