"""Plain implementations, in float64 but for the roundings that their definitions name, of the 8-bit floating-point
projection, the norm and rotation of heads with its gradient, and the bookkeeping of pages. On whatever device their arguments are."""
import math

import torch

TOP = 448.0


def blocks_max(x, rows):
    """Largest magnitudes [blocks of rows, blocks of 128 columns]."""
    M, K = x.shape
    out = torch.zeros((-(-M // rows), -(-K // 128)), dtype=x.dtype, device=x.device)
    for i in range(out.shape[1]):
        top = x[:, 128 * i : 128 * i + 128].abs().amax(1)
        for m in range(out.shape[0]):
            out[m, i] = top[rows * m : rows * m + rows].max()
    return out if rows > 1 else torch.stack([x[:, 128 * i : 128 * i + 128].abs().amax(1) for i in range(out.shape[1])], 1)


def e4m3(v):
    """float64 numbers rounded to e4m3 (half to even, 448 at most)."""
    e = (torch.frexp(v.abs()).exponent - 1).clamp(min=-6).long()
    step = ((e - 3 + 1023) << 52).view(torch.float64)
    return (torch.round(v / step) * step).clamp(-TOP, TOP)


def spread(scales, rows, M, K):
    """Each element's scale [M, K]."""
    return scales.repeat_interleave(rows, 0)[:M].repeat_interleave(128, 1)[:, :K]


def fp8(x32, rows):
    """(codes as float64, scales fp32) of fp32 rows."""
    s = blocks_max(x32, rows) / torch.full((), TOP, device=x32.device)
    each = spread(s, rows, *x32.shape)
    q = (x32 / each).double()
    return e4m3(torch.where(each > 0, q, torch.zeros_like(q))), s


def fp8_linear(x, codes, w_scales, rows):
    """(y, sum of magnitudes) in float64."""
    q, s = fp8(x.float(), 1)
    a = q * spread(s, 1, *q.shape).double()
    w = codes.to(torch.float32).double() * spread(w_scales, rows, *codes.shape).double()
    return a @ w.t(), a.abs() @ w.abs().t()


# ------------------------------------------------------------------ norm and rotation
def turn(x, cos, sin, interleaved, back=False):
    """Heads [n, heads, dh], their first 2 * cos.shape[-1] elements turned by the rows' angles; each operation in x's type."""
    half = cos.shape[-1]
    c, s = cos[:, None], -sin[:, None] if back else sin[:, None]
    t, rest = x[..., : 2 * half], x[..., 2 * half :]
    a, b = (t[..., 0::2], t[..., 1::2]) if interleaved else (t[..., :half], t[..., half:])
    y, z = a * c - b * s, b * c + a * s
    return torch.cat((torch.stack((y, z), -1).flatten(-2) if interleaved else torch.cat((y, z), -1), rest), -1)


def factor(x, eps):
    """fl32(1 / sqrt(mean x^2 + eps)) of heads; eps as the fp32 number that the call gets."""
    eps = torch.tensor(eps, dtype=torch.float32).double().item()
    return (1 / torch.sqrt(x.double().square().mean(-1, keepdim=True) + eps)).float()


def norm_rope(x, w, eps, cos, sin, interleaved):
    """The forward with its roundings, on fp32 heads. w [heads, dh] or None."""
    if eps is not None:
        x = x * factor(x, eps)
        x = x if w is None else x * w
    return x if cos is None else turn(x, cos, sin, interleaved)


def norm_rope64(x, w, eps, cos, sin, interleaved):
    """The same without roundings, in float64."""
    if eps is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + torch.tensor(eps, dtype=torch.float32).double().item())
        x = x if w is None else x * w
    return x if cos is None else turn(x, cos, sin, interleaved)


def table(length, dim, theta, kind="plain", factor=1.0, original=0.0, low=1.0, high=32.0, attention=1.0):
    f = torch.tensor([theta ** (-2 * j / dim) for j in range(dim // 2)], dtype=torch.float64)
    if kind == "linear":
        f = f / factor
    if kind == "by_parts":
        g = ((original * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        f = g * f + (1 - g) * f / factor
    a = torch.arange(length, dtype=torch.float64)[:, None] * f
    return a.cos() * attention, a.sin() * attention


# ------------------------------------------------------------------ bookkeeping (lists)
def release(lens, ended, pages, free, n_free, page, shared):
    free, lens = list(free), list(lens)
    for b, e in enumerate(ended):
        if e:
            for i in range(shared // page, -(-lens[b] // page)):
                free[n_free] = pages[b][i]
                n_free += 1
            lens[b] = min(lens[b], shared)
    return lens, free, n_free


def plan(lens, counts, pages, free, n_free, page, rows):
    lens, pages = list(lens), [list(p) for p in pages]
    start, slots, positions = [0], [], []
    for b, c in enumerate(counts):
        for i in range(-(-lens[b] // page), -(-(lens[b] + c) // page)):
            n_free -= 1
            pages[b][i] = free[n_free]
        for p in range(lens[b], lens[b] + c):
            positions.append(p)
            slots.append(pages[b][p // page] * page + p % page)
        lens[b] += c
        start.append(start[-1] + c)
    pad = rows - len(slots)
    return lens, pages, n_free, start, slots + [-1] * pad, positions + [0] * pad
