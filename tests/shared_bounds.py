"""Error bounds of the attention behind shared rows that tell a weight in two parts from a weight rounded once."""
import torch

import mx4_ref as X
import paged_ref as R


def parts(dtype, fmt):
    """Largest error of a weight (relative) that enters the value product in two parts: half a step of half a step of the type they
    have (bf16 over codes, else the element type); none in fp32."""
    if dtype == torch.float32:
        return 0.0
    return R.half_step(torch.float16 if fmt == "same" and dtype == torch.float16 else torch.bfloat16) ** 2


def bounds(q, k, v, idx, w, out, lse, sm, dtype, fmt):
    """Largest errors of out [d] and lse: mx4_ref.bounds (scores, sums and the output's own rounding; its term for the weights
    replaced by the parts'), and fp16 parts below the normal range, off by 2^-25 at most where the largest weight is 2^7 or
    more."""
    if w is None or idx.numel() == 0:
        return torch.zeros_like(out), 0.0
    b, l = X.bounds(q, k, v, idx, w, out, lse, sm, dtype)
    size = w @ v[idx].abs()
    in_x = 2.0 ** -16 if dtype != torch.float32 else 0.0
    tiny = 2.0 ** -32 * v[idx].abs().sum(0) if dtype == torch.float16 else 0.0
    return b + (parts(dtype, fmt) - in_x) * size + tiny, l


def attend_rounded(q, k, v, pos, sm, weight_type, two):
    """The attention of one row (64 bits) with weights (the largest 2^7) in weight_type, in two parts or rounded once."""
    s = (k[: pos + 1] @ q) * sm
    w = torch.exp(s - s.max()) * 2.0 ** 7
    hi = w.to(weight_type).double()
    if two:
        hi = hi + (w - hi).to(weight_type).double()
    return (hi @ v[: pos + 1]) / w.sum()
