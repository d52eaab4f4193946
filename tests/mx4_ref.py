"""Plain 64-bit forms of the 4-bit cache pages (codes 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign, a scale 2^e to each 32 channels), on
the host."""
import math

import torch

import paged_ref as R

GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def encode(rows):
    """Rows [.., d] (64 bits): (code of each channel 0..15, scale byte of each 32 channels)."""
    x = rows.double().unflatten(-1, (-1, 32))
    fine = x.isfinite()
    top = torch.where(fine, x.abs(), 0.0).amax(-1)
    e = torch.full_like(top, -126.0)
    for s in range(-126, 125):  # the least e with top <= 6 2^e, up to 125
        e = torch.where(top > 6 * 2.0 ** s, float(s + 1), e)
    e = torch.where(top == 0, 0.0, e)
    u = (x / (2.0 ** e)[..., None]).abs().clamp(max=6.0)
    # nearest of the grid; of two that are as near, the one with the even code
    gap = (u[..., None] - GRID).abs()
    near = gap == gap.amin(-1, keepdim=True)
    even = near & (torch.arange(8) % 2 == 0)
    code = torch.where(even.any(-1), even.int().argmax(-1), near.int().argmax(-1))
    code = code | (torch.signbit(x).long() << 3)
    scale = torch.where(x.isnan().any(-1), 255, (e + 127).long())
    return code.flatten(-2), scale


def decode(codes, scale):
    """Rows (64 bits) of packed codes [.., d / 2] (bytes) and scale bytes [.., d / 32]."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    x = GRID[c & 7] * (1 - 2 * (c >> 3).double())
    s = torch.where(scale == 255, math.nan, 2.0 ** (scale.double() - 127))
    return x * s.repeat_interleave(32, -1)


def packed(code):
    return (code[..., 0::2] | (code[..., 1::2] << 4)).to(torch.uint8)


def rows_of(kv, l, b, h, n):
    """K and V rows [0, n) of a sequence of 4-bit pages in 64 bits, and which rows have a page."""
    page, out, has = kv.page, [], torch.zeros(n, dtype=torch.bool)
    for pages, scale in ((kv.k_pages, kv.k_scale), (kv.v_pages, kv.v_scale)):
        x = torch.full((n, kv.d), math.nan, dtype=torch.float64)
        for j0 in range(0, n, page):
            m, id = min(page, n - j0), int(kv.table[b, j0 // page])
            if 0 <= id < pages.shape[1]:
                x[j0:j0 + m] = decode(pages[l, id, h, :m].cpu(), scale[l, id, h, :, :m].T.cpu())
                has[j0:j0 + m] = True
        out.append(x)
    return out[0], out[1], has


def bounds(q, k, v, idx, w, out, lse, sm, dtype):
    """Largest errors of the attention over 4-bit rows. As paged_ref.bounds, but for the scores' products: fp16 queries are added up
    in two parts, so 2 d terms (at most) in fp32 in any order; the rows are exact, and a weight in two bf16 parts is off by at
    most half a step of half a step of bf16, 2^-8 2^-8."""
    if w is None or idx.numel() == 0:
        return torch.zeros_like(out), 0.0
    top = float((k[idx].abs() @ q.abs()).max()) * abs(sm)
    ds = (2 * q.numel() + 8) * R.U32 * top + 4 * R.U32
    n = idx.numel()
    rel = 2 * ds + (n + 16) * R.U32
    weight = 2.0 ** -16 if dtype != torch.float32 else 0.0
    tiny = 2.0 ** -24 if dtype == torch.float16 else 0.0  # fp16 below its normal range
    return (2 * rel + weight) * (w @ v[idx].abs()) + R.half_step(dtype) * out.abs() + tiny, 2 * ds + (n + 16) * R.U32 + 4 * R.U32 * abs(lse)
