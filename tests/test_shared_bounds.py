"""The bounds of the shared attention's precision tests, on the host: weights in two parts stay inside, weights rounded once do not."""
import pytest
import torch

import paged_ref as R
import shared_bounds as S


@pytest.mark.parametrize("dtype,fmt,parts", [("bf16", "same", "bf16"), ("fp16", "same", "fp16"), ("bf16", "mx4", "bf16"), ("fp16", "mx4", "bf16"), ("fp16", "e4m3", "bf16"),
                                             ("fp32", "mx4", "bf16")])
def test_a_weight_rounded_once_is_outside(dtype, fmt, parts):
    """At few keys and scores of about one: the terms of fp32 sums and scores, which hold for any order, do not hide it there."""
    t = dict(fp32=torch.float32, fp16=torch.float16, bf16=torch.bfloat16)
    g = torch.Generator().manual_seed(1)
    over = {True: 0, False: 0}
    for _ in range(8):
        q, k, v = (torch.randn(n, 64, generator=g).to(t[dtype]).double() for n in (1, 70, 70))
        o, lse, idx, w = R.attend(q[0], k, v, 69, 0.01, 0, 0)
        b, _ = S.bounds(q[0], k, v, idx, w, o, lse, 0.01, t[dtype], fmt)
        for two in (True, False):
            got = S.attend_rounded(q[0], k, v, 69, 0.01, t[parts], two).to(t[dtype]).double()
            over[two] += int(((got - o).abs() > b).sum())
    assert over[False] >= 5 and (over[True] == 0 or dtype == "fp32")  # (fp32 has no room for 16-bit parts at all)
