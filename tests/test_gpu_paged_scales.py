"""Page scales that a caller wrote, or nobody did, in pages that a row does not see."""
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
