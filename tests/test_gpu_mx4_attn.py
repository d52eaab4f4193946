"""mpc_paged_attn over pages of 4-bit codes against the softmax's definition in 64 bits: types, head layouts, lengths from one row
to several pages, windows, sinks, ragged batches, and values that a row may not see."""
import math

import pytest
import torch

import mx4_ref as X
import paged_ref as R
from test_gpu_mx4_append import make4
from test_gpu_paged_append import DT, bits, tokens

pytestmark = pytest.mark.gpu


def fill4(kv, lens, seed, dtype):
    import paper_2501_06807_amd as M
    n = max(max(lens), 1)
    k, v = tokens((kv.L, kv.B, kv.Hkv, n, kv.d), dtype, seed), tokens((kv.L, kv.B, kv.Hkv, n, kv.d), dtype, seed + 1, spread=False)
    kv.lens.copy_(torch.tensor(lens))
    M.mpc_paged_append(k.cuda(), v.cuda(), kv, n_valid=torch.tensor(lens, dtype=torch.int32, device="cuda"))


def run4(kv, q, new=None, window=0, sinks=0, sm=None, ws=None, out=None):
    import paper_2501_06807_amd as M
    out = torch.full_like(q, 7.0) if out is None else out
    lse = torch.full(q.shape[:4], 7.0, device="cuda")
    M.mpc_paged_attn(q, kv, out, sm_scale=sm or 1 / math.sqrt(kv.d), window=window, sinks=sinks, lse=lse, ws=ws,
                     n_valid=None if new is None else torch.tensor(new, dtype=torch.int32, device="cuda"))
    return out, lse


def check4(kv, q, out, lse, lens, new=None, window=0, sinks=0, sm=None, units=None):
    L, B, Hq, n, d = q.shape
    G, sm = Hq // kv.Hkv, sm or 1 / math.sqrt(d)
    qc, oc, lc = q.cpu(), out.cpu(), lse.cpu()
    for l in range(L):
        for b in range(B):
            m = n if new is None else new[b]
            for h in range(kv.Hkv):
                if units is not None and (l, b, h) not in units:
                    continue
                k, v, has = X.rows_of(kv, l, b, h, lens[b])
                for hq in range(h * G, (h + 1) * G):
                    assert bool((oc[l, b, hq, m:] == 7).all()) and bool((lc[l, b, hq, m:] == 7).all())
                    for t in range(m):
                        x = qc[l, b, hq, t].double()
                        o, ls, idx, w = R.attend(x, k, v, lens[b] - m + t, sm, window, sinks, has)
                        bo, bl = X.bounds(x, k, v, idx, w, o, ls, sm, q.dtype)
                        R.check(oc[l, b, hq, t], o, bo, f"out l{l} b{b} h{hq} t{t}")
                        R.check(lc[l, b, hq, t], ls, bl, f"lse l{l} b{b} h{hq} t{t}")


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,d,page,n,lens,new", [
    (2, 2, 64, 16, 1, [1, 17, 500], None), (8, 2, 128, 32, 1, [33, 64, 1000], None), (8, 1, 128, 16, 3, [3, 47, 259], [3, 0, 2]),
    (4, 4, 64, 64, 5, [5, 130, 64], [5, 5, 1]), (4, 1, 128, 128, 9, [300, 9, 129], [9, 4, 9]), (2, 1, 64, 256, 33, [600, 33, 256], [33, 1, 20]),
])
def test_against_the_definition(dtype, Hq, Hkv, d, page, n, lens, new):
    import paper_2501_06807_amd as M
    kv = make4(M, 2, 3, Hkv, d, dtype, page, cap=-(-max(lens) // page) + 1)
    fill4(kv, lens, 3, dtype)
    q = tokens((2, 3, Hq, n, d), dtype, 9).cuda()
    out, lse = run4(kv, q, new)
    check4(kv, q, out, lse, lens, new)


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (20, 0), (100, 4), (33, 40), (5000, 7)])
def test_windows_and_sinks(dtype, window, sinks):
    import paper_2501_06807_amd as M
    lens, new = [257, 40, 130], [4, 2, 4]
    kv = make4(M, 1, 3, 2, 64, dtype, 16, cap=17)
    fill4(kv, lens, 3, dtype)
    q = tokens((1, 3, 4, 4, 64), dtype, 9).cuda()
    out, lse = run4(kv, q, new, window, sinks)
    check4(kv, q, out, lse, lens, new, window, sinks)


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
def test_rows_that_see_nothing(dtype):
    """A sequence without rows, and one whose window holds only rows without a page."""
    import paper_2501_06807_amd as M
    lens = [1, 60, 3]
    kv = make4(M, 1, 3, 1, 64, dtype, 16, cap=4)
    fill4(kv, lens, 3, dtype)
    lens = [0, 60, 1]
    kv.lens.copy_(torch.tensor(lens))
    kv.table[1, 2:] = -1
    q = tokens((1, 3, 2, 2, 64), dtype, 9).cuda()
    out, lse = run4(kv, q, window=8)
    assert bool((out[0, 0] == 0).all()) and bool((lse[0, 0] == -math.inf).all())
    assert bool((out[0, 1] == 0).all()) and bool((lse[0, 1] == -math.inf).all())
    check4(kv, q, out, lse, lens, window=8)


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
def test_what_a_row_does_not_see_does_not_reach_it(dtype):
    """NaN blocks of a later token's key and value, behind a window and behind the last row."""
    import paper_2501_06807_amd as M
    lens = [70]
    kv = make4(M, 1, 1, 1, 64, dtype, 16, cap=6)
    fill4(kv, [75], 3, dtype)
    for j in (10, 69, 70, 74):
        id = int(kv.table[0, j // 16])
        kv.k_scale[0, id, 0, :, j % 16] = 255
        kv.v_scale[0, id, 0, 1, j % 16] = 255
    kv.lens.fill_(70)
    q = tokens((1, 1, 2, 3, 64), dtype, 9).cuda()
    out, lse = run4(kv, q, window=50)
    assert bool(out[0, 0, :, :2].isfinite().all()) and bool(out[0, 0, :, 2].isnan().all()) and bool(lse[0, 0, :, 2].isnan().all())
    check4(kv, q, out, lse, lens, window=50)
    kv.k_scale[0, int(kv.table[0, 4]), 0, :, 5] = 127  # row 69: its key is a number, its value NaN in channels 32 on
    out, lse = run4(kv, q, window=50)
    assert bool(out[0, 0, :, 2, :32].isfinite().all()) and bool(out[0, 0, :, 2, 32:].isnan().all())
    check4(kv, q, out, lse, lens, window=50)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("size", [2.0 ** -14, 1.0, 2.0 ** 10])
def test_queries_and_values_of_any_size(dtype, size):
    """fp16 queries are exact in two parts, and values beyond fp16's exact range come through."""
    import paper_2501_06807_amd as M
    lens = [200, 31]
    kv = make4(M, 1, 2, 2, 128, dtype, 32, cap=8)
    k, v = tokens((1, 2, 2, 200, 128), dtype, 1), tokens((1, 2, 2, 200, 128), dtype, 2)
    v = (v.float() * size).to(DT[dtype])
    kv.lens.copy_(torch.tensor(lens))
    M.mpc_paged_append(k.cuda(), v.cuda(), kv, n_valid=kv.lens.clone())
    q = (tokens((1, 2, 4, 2, 128), dtype, 3).float() * size).to(DT[dtype]).cuda()
    sm = 1 / math.sqrt(128) / size
    out, lse = run4(kv, q, sm=sm)
    check4(kv, q, out, lse, lens, sm=sm)


def test_fp16_queries_that_are_not_finite():
    import paper_2501_06807_amd as M
    kv = make4(M, 1, 1, 1, 64, "fp16", 16, cap=3)
    k = torch.ones(1, 1, 1, 40, 64, dtype=torch.float16)
    k[..., 0] = -1
    kv.lens.fill_(40)
    M.mpc_paged_append(k.cuda(), k.cuda(), kv)
    q = torch.ones(1, 1, 4, 1, 64, dtype=torch.float16, device="cuda")
    q[0, 0, 0, 0, 0] = math.inf  # every score -infinity
    q[0, 0, 1, 0, 0] = -math.inf  # every score +infinity
    q[0, 0, 2, 0, 5] = math.nan
    out, lse = run4(kv, q)
    assert bool((out[0, 0, 0] == 0).all()) and float(lse[0, 0, 0]) == -math.inf
    assert bool(out[0, 0, 1:3].isnan().all()) and bool(lse[0, 0, 1:3].isnan().all())
    assert bool(out[0, 0, 3].isfinite().all())


def test_strides_workspaces_and_order_of_calls():
    """Queries and outputs with tokens before heads; one workspace for calls of several shapes; results do not depend on it."""
    import paper_2501_06807_amd as M
    lens = [1500, 2]
    kv = make4(M, 2, 2, 2, 128, "bf16", 64, cap=24)
    fill4(kv, lens, 3, "bf16")
    q = tokens((2, 2, 8, 8, 128), "bf16", 9).cuda()
    ws = M.workspace(M.paged_attn_workspace_bytes(q, kv))
    first = run4(kv, q, ws=ws)
    check4(kv, q, *first, lens, units=[(1, 0, 1), (0, 1, 0)])
    one = run4(kv, q[:, :, :, 7:].contiguous(), ws=ws)
    assert torch.equal(bits(one[0][:, :, :, 0]), bits(run4(kv, q[:, :, :, 7:].contiguous())[0][:, :, :, 0]))
    qt = q.transpose(2, 3).contiguous().transpose(2, 3)
    out = torch.full((2, 2, 8, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda").transpose(2, 3)
    again = run4(kv, qt, ws=ws, out=out)
    assert torch.equal(bits(first[0]), bits(again[0])) and torch.equal(bits(first[1]), bits(again[1]))


def test_long_caches_of_many_splits():
    import paper_2501_06807_amd as M
    lens = [20011]
    kv = make4(M, 1, 1, 1, 128, "bf16", 64, cap=320)
    fill4(kv, lens, 3, "bf16")
    q = tokens((1, 1, 8, 1, 128), "bf16", 9).cuda()
    out, lse = run4(kv, q)
    check4(kv, q, out, lse, lens)
