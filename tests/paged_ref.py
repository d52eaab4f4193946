"""Plain 64-bit forms of the paged-cache operators, on the host, and the error bounds their GPU results are held to."""
import math

import torch

E4M3 = torch.float8_e4m3fn
U32 = 2.0 ** -24  # half a step of fp32, relative


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def rope_table(n_pos, rot, base=10000.0):
    f = base ** (-2 * torch.arange(rot // 2, dtype=torch.float64) / rot)
    a = torch.arange(n_pos, dtype=torch.float64)[:, None] * f
    return torch.stack([a.cos(), a.sin()], -1).float()


def rotated(x, table, style, pos):
    """Row x [.., d] (64 bits) at position pos, in 64 bits: (row, magnitude of the products for its error bound)."""
    y, mag = x.clone(), x.abs()
    rot = 2 * table.shape[1]
    if not 0 <= pos < table.shape[0]:
        y[..., :rot] = math.nan
        return y, mag
    c, s = table[pos, :, 0].double(), table[pos, :, 1].double()
    i = torch.arange(rot // 2)
    a, b = (i, i + rot // 2) if style == "half" else (2 * i, 2 * i + 1)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    mag = mag.clone()
    mag[..., a] = mag[..., b] = x[..., a].abs() + x[..., b].abs()
    return y, mag


def encode(rows):
    """A page's rows [page][d] (64 bits): (codes as the values they stand for in units of the scale, scale)."""
    fine = rows.isfinite()
    top = float(torch.where(fine, rows.abs(), 0.0).max())
    e = 0
    if top > 0:
        e = max(-126, math.frexp(top / 448)[1] - 1)
        if top > 448 * 2.0 ** e:
            e += 1
    u = rows / 2.0 ** e
    mag = u.abs().clamp(max=448.0)
    step = 2.0 ** (torch.frexp(mag.clamp(min=2.0 ** -6))[1].double() - 4)  # three places behind the first, from 2^-6 up
    q = torch.round(mag / step) * step  # halves to even
    return torch.where(u.isnan(), u, torch.copysign(q, u)), 2.0 ** e


def attend(q, k, v, pos, sm, window, sinks, has=None):
    """One row q [d] over k, v [T][d] in 64 bits -> (out [d], lse, seen, weights)."""
    j = torch.arange(k.shape[0])
    see = j <= pos
    if window:
        see &= (j > pos - window) | (j < sinks)
    if has is not None:
        see &= has
    idx = j[see]
    s = (k[idx] @ q) * sm
    if idx.numel() == 0 or bool((s == -math.inf).all()):
        return torch.zeros(v.shape[1], dtype=torch.float64), -math.inf, idx, None
    lse = torch.logsumexp(s, 0)
    if not bool(s.isfinite().any()) or bool((s == math.inf).any()) or bool(s.isnan().any()):
        return torch.full((v.shape[1],), math.nan, dtype=torch.float64), math.nan, idx, None
    w = torch.exp(s - lse)
    return w @ v[idx], float(lse), idx, w


def bounds(q, k, v, idx, w, out, lse, sm, dtype):
    """Largest errors of out [d] and lse that the kernels' roundings allow. Scores: fp32 products and sums of d terms in
    any order, the scale and the exponent's own rounding; weights: exp2 of one step, their sum over the keys in fp32, and
    for 16-bit types one rounding of each weight to the type; out: one rounding to its type."""
    if w is None or idx.numel() == 0:
        return torch.zeros_like(out), 0.0
    d = q.numel()
    top = float((k[idx].abs() @ q.abs()).max()) * abs(sm)
    ds = (d + 8) * U32 * top + 4 * U32
    n = idx.numel()
    rel = 2 * ds + (n + 16) * U32
    weight = half_step(dtype) if dtype != torch.float32 else 0.0
    spread = w @ v[idx].abs()
    tiny = 2.0 ** -24 if dtype == torch.float16 else 0.0  # fp16 below its normal range
    return (2 * rel + weight) * spread + half_step(dtype) * out.abs() + tiny, 2 * ds + (n + 16) * U32 + 4 * U32 * abs(lse)


def check(got, want, bound, what):
    """got (any type) against want (64 bits) within bound; NaN and infinities where want has them."""
    got = torch.as_tensor(got).double()
    want, bound = torch.as_tensor(want, dtype=torch.float64), torch.as_tensor(bound, dtype=torch.float64)
    fine = want.isfinite()
    assert torch.equal(got.isnan(), want.isnan()), f"{what}: NaN in other places"
    rest = ~fine & ~want.isnan()
    assert torch.equal(got[rest], want[rest]), f"{what}: infinities in other places"
    err = (got - want).abs()[fine]
    over = err > bound.expand_as(want)[fine]
    assert not bool(over.any()), (f"{what}: {int(over.sum())} of {over.numel()} outside, worst {float(err.max()):.3e}, "
                                  f"bound there {float(bound.expand_as(want)[fine][err.argmax()]):.3e}")
