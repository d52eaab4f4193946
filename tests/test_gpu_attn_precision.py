"""What the attentions' roundings cost, where it would show: scores far from zero that lie close together, and products of a
score that are small beside others, and weights of 16-bit types over values that cancel."""
import math

import pytest
import torch

import paged_ref as R
from test_gpu_attn import fill, rows_of, run_paged
from test_gpu_paged_append import DT, make, tokens

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", ["pages", "codes", "prompt"])
@pytest.mark.parametrize("sm", [0.3125, -0.3125, 0.28125])
def test_large_scores_that_lie_close(form, sm):
    """fp32 scores of 4032 to 4039, each exact. A score times the scale and log2(e) is about 1800, where half a step of fp32
    is 2^-14: rounded there, a weight would be off by up to 2^-14 ln 2, 700 U32. Taken against the reference in one rounding,
    an exponent e of [-4, 0] is off by 4 U32, and by twice U32 of its difference to the reference's, 8 U32, for the two
    roundings of the factor: 12 ln 2 U32 of the weight. exp2 adds a step, 2 U32, each of three moves (the reference's, the
    join of waves, of parts) 3 U32, the division 3: below 24 U32 for a weight, and T U32 for the sums. Channel c of the output is
    the sum of the weights of one score out of eight."""
    import paper_2501_06807_amd as M
    d, T, page = 64, 64, 16
    step = torch.arange(T) * 5 % 8
    k, q = torch.zeros(1, 1, 1, T, d), torch.zeros(1, 1, 2, 1, d)
    k[..., 0], k[..., 1] = 448.0, step / 8.0  # (codes hold these too, with a scale of 1)
    q[..., 0], q[..., 1] = 9.0, 8.0
    q[0, 0, 1] *= -1
    v = (torch.arange(d) % 8 == step[:, None]).float().expand(1, 1, 1, T, d).contiguous()
    if form == "prompt":
        out, lse = torch.empty_like(q).cuda(), torch.empty(1, 1, 2, 1, device="cuda")
        M.mpc_prompt_attn(q.cuda(), k.cuda(), v.cuda(), out, sm_scale=sm, lse=lse)
    else:
        kv = make(M, 1, 1, 1, d, "fp32", page, cap=5, fp8=form == "codes")
        kv.lens.fill_(T)
        M.mpc_paged_append(k.cuda(), v.cuda(), kv)
        out, lse = run_paged(kv, q.cuda(), [1], sm=sm)
    for h in range(2):
        o, ls, idx, w = R.attend(q[0, 0, h, 0].double(), k[0, 0, 0].double(), v[0, 0, 0].double(), T - 1, sm, 0, 0)
        R.check(out[0, 0, h, 0].cpu(), o, (2 * (24 + T) + 1) * R.U32 * o, f"{form} h{h}")


@pytest.mark.parametrize("dtype,fp8", [("bf16", False), ("fp16", False), ("bf16", True), ("fp16", True), ("fp32", False)])
def test_infinite_values_that_every_row_sees(dtype, fp8):
    """A value of infinity makes the channel's output infinite, of both signs or NaN makes it NaN, for every row that sees it,
    wherever in the cache it lies, and no other channel."""
    import paper_2501_06807_amd as M
    d, T, page, n = 64, 75, 16, 2
    k, v = tokens((1, 1, 1, T, d), dtype, 1, spread=False), tokens((1, 1, 1, T, d), dtype, 2)
    at = (70, 66) if fp8 else (20, 40)  # codes have no infinities: those of a cache in codes stand in its tail
    v[0, 0, 0, at[0], 3] = math.inf
    v[0, 0, 0, at[0], 5] = -math.inf
    v[0, 0, 0, at[0], 9] = math.inf
    v[0, 0, 0, at[1], 9] = -math.inf
    v[0, 0, 0, at[1], 11] = math.nan
    v[0, 0, 0, at[1], 12] = math.inf
    v[0, 0, 0, at[0], 12] = math.inf
    kv = make(M, 1, 1, 1, d, dtype, page, cap=5, fp8=fp8)
    kv.lens.fill_(T)
    M.mpc_paged_append(k.cuda(), v.cuda(), kv)
    q = tokens((1, 1, 4, n, d), dtype, 3, spread=False).cuda()
    want = {3: math.inf, 5: -math.inf, 9: math.nan, 11: math.nan, 12: math.inf}
    for m in (1, 2):
        out, lse = run_paged(kv, q[:, :, :, :m].contiguous(), [m])
        assert bool(lse.isfinite().all())
        for c in range(d):
            x = out[..., c].cpu().float()
            if c not in want:
                assert bool(x.isfinite().all()), c
            elif math.isnan(want[c]):
                assert bool(x.isnan().all()), c
            else:
                assert bool((x == want[c]).all()), c


@pytest.mark.parametrize("form", ["pages", "codes", "prompt"])
@pytest.mark.parametrize("d", [64, 128])
def test_small_products_beside_a_large_one(form, d):
    """fp32 scores of 2^20 for one key and 2^20 and d - 1 products of 0.12 steps of that size for the other. A score is added up
    in four chains of d / 4 products, of which one starts with the large product and may lose what follows it: 0.12 (d / 4 - 1)
    steps, and half a step in each of the two sums that join the chains, for either key. The output, the second key's weight
    against the first's, moves by a quarter of an error of the score at most; one chain would lose all of 0.12 (d - 1)."""
    import paper_2501_06807_amd as M
    step, T = 2.0 ** -3, 2  # (fp32 between 2^20 and 2^21)
    k, q, v = torch.zeros(1, 1, 1, 16, d), torch.full((1, 1, 1, 1, d), 0.12 * step), torch.zeros(1, 1, 1, 16, d)
    k[..., 0], k[:, :, :, 1, 1:], q[..., 0] = 256.0, 1.0, 4096.0
    v[:, :, :, 1] = 1.0
    if form == "prompt":
        out = torch.empty_like(q).cuda()
        M.mpc_prompt_attn(q.cuda(), k[:, :, :, :T].contiguous().cuda(), v[:, :, :, :T].contiguous().cuda(), out, sm_scale=1.0)
    else:
        n = T if form == "pages" else 16  # a page of codes is whole: the other keys' scores are zero
        k[:, :, :, T:] = 0
        kv = make(M, 1, 1, 1, d, "fp32", 16, cap=2, fp8=form == "codes")
        kv.lens.fill_(n)
        M.mpc_paged_append(k[:, :, :, :n].cuda(), v[:, :, :, :n].cuda(), kv)
        out, _ = run_paged(kv, q.cuda(), [1], sm=1.0)
    diff = 0.12 * (d - 1) * step
    want = 1 / (1 + math.exp(-diff))
    bound = (0.12 * (d / 4 - 1) + 2) * step / 4
    assert bound < 0.7 * (want - 0.5)
    R.check(out.cpu(), torch.full_like(out.cpu(), want), bound, form)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("fp8,page", [(False, 16), (True, 16), (True, 64)])
@pytest.mark.parametrize("n,window,sinks", [(1, 0, 0), (3, 0, 0), (5, 90, 3)])
def test_weights_of_16_bit_caches_keep_twice_their_bits(dtype, fp8, page, n, window, sinks):
    """Weights enter the product with the values in two parts of the type, what the first part leaves being rounded once
    more: half a step of half a step each, beside the fp32 roundings (R.bounds without a 16-bit weight) and the output's
    one rounding to the type. fp16 weights are lifted by 2^14, below which their second part keeps 2^-25 at least."""
    import paper_2501_06807_amd as M
    d, Hq, Hkv, lens = 128, 8, 2, [300, 77, 512]
    kv = make(M, 1, 3, Hkv, d, dtype, page, cap=-(-512 // page), fp8=fp8)
    fill(kv, lens, 21, dtype)
    q = tokens((1, 3, Hq, n, d), dtype, 3, spread=False).cuda()
    out, lse = run_paged(kv, q, [n] * 3, window, sinks)
    sm, half = d ** -0.5, R.half_step(DT[dtype])
    for b in range(3):
        for h in range(Hkv):
            k, v, _ = rows_of(kv, 0, b, h, lens[b])
            for hq in range(4 * h, 4 * h + 4):
                for t in range(n):
                    x = q[0, b, hq, t].cpu().double()
                    o, ls, idx, w = R.attend(x, k, v, lens[b] - n + t, sm, window, sinks)
                    bo, _ = R.bounds(x, k, v, idx, w, o, ls, sm, torch.float32)
                    spread = w @ v[idx].abs()
                    tiny = 2.0 ** -24 + 2.0 ** -39 * v[idx].abs().sum(0) if dtype == "fp16" else 0.0
                    R.check(out[0, b, hq, t].cpu(), o, bo + half * half * spread + half * o.abs() + tiny, f"b{b} h{hq} t{t}")
