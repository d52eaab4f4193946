"""mpc_shared_attn's weights enter the value product in two parts of their type, as mpc_paged_attn's, however many query rows a group has
and whatever the pages hold: bounds without a term for weights rounded once."""
import pytest
import torch

import paged_ref as R
import shared_bounds as S
from test_gpu_paged_append import tokens
from test_gpu_shared_attn import FORMATS, behind, held, run

pytestmark = pytest.mark.gpu

T, LENS = 64, [70, 66, 65, 71, 69]


def inside(kv, fmt, q, out, lse, lens, sm, window=0):
    """Every row of `out` and `lse` within the bounds; all sequences share the first one's T rows."""
    L, B, Hq, n, d = q.shape
    G = Hq // kv.Hkv
    qc, oc, lc = q.cpu(), out.cpu(), lse.cpu()
    for l in range(L):
        for h in range(kv.Hkv):
            lead = held(kv, l, 0, h, lens[0])
            for b in range(B):
                k, v, has = held(kv, l, b, h, lens[b])
                for x, y in zip((k, v, has), lead):
                    x[:T] = y[:T]
                for hq in range(h * G, (h + 1) * G):
                    for t in range(n):
                        x = qc[l, b, hq, t].double()
                        o, ls, idx, w = R.attend(x, k, v, lens[b] - n + t, sm, window, 0, has)
                        bo, bl = S.bounds(x, k, v, idx, w, o, ls, sm, q.dtype, fmt)
                        R.check(oc[l, b, hq, t], o, bo, f"out l{l} b{b} h{hq} t{t}")
                        R.check(lc[l, b, hq, t], ls, bl, f"lse l{l} b{b} h{hq} t{t}")


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("G,n,d", [(1, 1, 64), (4, 1, 128), (2, 3, 64), (4, 5, 64), (8, 4, 128)])  # 5, 20, 30, 100, 160 rows to a kv head
def test_weights_in_two_parts(fmt, dtype, G, n, d):
    """Whole tiles (no window) and tiles that a window cuts. Scores of about one, as in the bounds' own test."""
    import paper_2501_06807_amd as M
    kv = behind(M, fmt, dtype, LENS, [0, 5], [T], 2, 2, d)
    q = tokens((2, 5, 2 * G, n, d), dtype, 9, spread=False).cuda()
    for window in (0, 40):
        out, lse = run(M, kv, q, [0, 5], [T], window=window, sm=0.002)
        inside(kv, fmt, q, out, lse, LENS, 0.002, window)
