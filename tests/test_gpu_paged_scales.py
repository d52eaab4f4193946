"""Page scales that a caller wrote, or nobody did, in pages that a row does not see; score scales far below one."""
import math

import pytest
import torch

import paged_ref as R
from test_gpu_attn import fill, rows_of, run_paged
from test_gpu_paged_append import DT, make, tokens

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("side,bad", [("v", math.nan), ("v", math.inf), ("k", math.nan)])
@pytest.mark.parametrize("n,lens,pages,carry", [
    # rows 76 .. 79 see from 47 .. 50 on: page 2 (32 .. 47) is seen by the first one alone; rows 80 .. 83 see from 51 on, none
    # of them page 2, the other half of their first tile in the 16-bit types
    (4, [80, 84], [2, 2], [{0}, set()]),
    # the same with 20 rows, and page 5 (80 .. 95) ahead of rows 76 .. 79
    (20, [96, 100, 96], [2, 2, 5], [{0}, set(), set(range(4, 20))]),
])
def test_scales_of_pages_that_a_row_does_not_see(dtype, side, bad, n, lens, pages, carry):
    """Rows that see a page with such a scale are not finite; the others are as if it were an ordinary one."""
    import paper_2501_06807_amd as M
    d, page, window, Hkv = 64, 16, 30, 2
    kv = make(M, 1, len(lens), Hkv, d, dtype, page, cap=7)
    fill(kv, lens, 7, dtype)
    q = tokens((1, len(lens), 4, n, d), dtype, 3, spread=False).cuda()
    want = [[rows_of(kv, 0, b, h, lens[b]) for h in range(Hkv)] for b in range(len(lens))]
    for b, pg in enumerate(pages):
        (kv.v_scale if side == "v" else kv.k_scale)[0, int(kv.table[b, pg])] = bad
    out, lse = run_paged(kv, q, [n] * len(lens), window)
    for b in range(len(lens)):
        for hq in range(4):
            k, v, _ = want[b][hq // 2]
            for t in range(n):
                if t in carry[b]:
                    assert not bool(out[0, b, hq, t].isfinite().any())
                    assert math.isnan(float(lse[0, b, hq, t])) == (side == "k")
                    continue
                x = q[0, b, hq, t].cpu().double()
                o, ls, idx, w = R.attend(x, k, v, lens[b] - n + t, d ** -0.5, window, 0)
                bo, bl = R.bounds(x, k, v, idx, w, o, ls, d ** -0.5, DT[dtype])
                R.check(out[0, b, hq, t].cpu(), o, bo, f"b{b} h{hq} t{t}")
                R.check(lse[0, b, hq, t].cpu(), ls, bl, f"lse b{b} h{hq} t{t}")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_score_scales_far_below_one(dtype):
    """Products of 2^116 to 2^117 with a scale of 2^-116 are scores of 1 to 2: the scale is taken as it is."""
    import paper_2501_06807_amd as M
    d, T, sm = 64, 70, 2.0 ** -116
    k, q = torch.zeros(1, 1, 1, T, d), torch.zeros(1, 1, 2, T, d)
    k[..., 0] = (1 + torch.arange(T) % 8 / 8.0) * 2.0 ** 58
    q[..., 0] = 2.0 ** 58
    q[0, 0, 1] *= -1
    v = tokens((1, 1, 1, T, d), dtype, 2, spread=False)
    k, q = k.to(DT[dtype]), q.to(DT[dtype])
    out, lse = torch.empty_like(q).cuda(), torch.empty(1, 1, 2, T, device="cuda")
    M.mpc_prompt_attn(q.cuda(), k.cuda(), v.cuda(), out, sm_scale=sm, window=20, sinks=2, lse=lse)
    kv = make(M, 1, 1, 1, d, dtype, 16, cap=5, fp8=False)
    kv.lens.fill_(T)
    M.mpc_paged_append(k.cuda(), v.cuda(), kv)
    po, pl = run_paged(kv, q.cuda(), [T], 20, 2, sm=sm)
    for h in range(2):
        for t in (0, 5, 40, 69):
            x, kd, vd = q[0, 0, h, t].double(), k[0, 0, 0].double(), v[0, 0, 0].double()
            o, ls, idx, w = R.attend(x, kd, vd, t, sm, 20, 2)
            bo, bl = R.bounds(x, kd, vd, idx, w, o, ls, sm, DT[dtype])
            for got, gl, what in ((out, lse, "prompt"), (po, pl, "pages")):
                R.check(got[0, 0, h, t].cpu(), o, bo, f"{what} h{h} t{t}")
                R.check(gl[0, 0, h, t].cpu(), ls, bl, f"{what} lse h{h} t{t}")
