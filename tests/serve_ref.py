"""Plain implementations of the serving operators, in float64 but for the roundings that their definition
names (the scale of a row, the quotient by it, the products and sums of the rotation, the two products by
the scales of a projection), on whatever device their arguments are."""
import math

import torch


def quantize_rows(x32, bits):
    """(codes as float64, scales fp32) of fp32 rows: s = fl32(max|x| / qmax), q = clip(rint(fl32(x / s)))."""
    qmax = 2 ** (bits - 1) - 1
    s = x32.abs().amax(-1) / torch.full((), float(qmax), device=x32.device)
    q = torch.round(x32 / s[..., None]).clamp(-qmax, qmax)
    q = torch.where(s[..., None] > 0, q, torch.zeros_like(q))
    return q.double(), s


def pack(codes, bits):
    c = codes.long() + 2 ** (bits - 1)
    if bits == 8:
        return c.to(torch.uint8)
    return (c[..., 0::2] + 16 * c[..., 1::2]).to(torch.uint8)


def unpack(raw, bits):
    r = raw.long()
    if bits == 4:
        r = torch.stack((r % 16, r // 16), -1).flatten(-2)
    return (r - 2 ** (bits - 1)).double()


def linear(x, codes, w_scales, out_dtype):
    q, s = quantize_rows(x.float(), 8)
    acc = q @ codes.double().t()  # whole numbers below 2^53
    return ((acc.float() * s[:, None]) * w_scales[None, :]).to(out_dtype)


def rotate(x32, cos, sin):
    """x [n, heads, dh] fp32, cos / sin [n, dh / 2] fp32; every product and sum rounded to fp32."""
    h = x32.shape[-1] // 2
    a, b, c, s = x32[..., :h], x32[..., h:], cos[:, None], sin[:, None]
    return torch.cat((a * c - b * s, b * c + a * s), -1)


def attention(q, k, v, window, scale):
    """One sequence: q [n, Hq, dh], k and v [len, Hkv, dh] in float64; the queries are the last n of the tokens.
    Returns out, lse and sum of p |v| (what the weights' rounding errors scale with)."""
    n, hq, dh = q.shape
    length, hkv = k.shape[0], k.shape[1]
    out = torch.zeros((n, hq, dh), dtype=torch.float64, device=q.device)
    mag = torch.zeros_like(out)
    lse = torch.full((n, hq), -math.inf, dtype=torch.float64, device=q.device)
    key = torch.arange(length, device=q.device)
    for i in range(n):
        p = length - n + i
        seen = key <= p
        if window:
            seen &= key > p - window
        idx = key[seen]
        if idx.numel() == 0:
            continue
        for h in range(hq):
            s = (k[idx, h // (hq // hkv)] @ q[i, h]) * scale
            lse[i, h] = torch.logsumexp(s, 0)
            w = torch.exp(s - lse[i, h])
            vv = v[idx, h // (hq // hkv)]
            out[i, h] = w @ vv
            mag[i, h] = w @ vv.abs()
    return out, lse, mag
