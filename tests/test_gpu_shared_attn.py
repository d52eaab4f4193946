"""mpc_shared_attn against the softmax's definition in 64 bits: groups of any size and number, page formats, types, lengths on both
sides of the shared rows, windows, sinks, values that a row may not see, captured calls."""
import math

import pytest
import torch

import mx4_ref as X
import paged_ref as R
from test_gpu_attn import rows_of
from test_gpu_mx4_append import make4
from test_gpu_paged_append import DT, bits, make, tokens

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def held(kv, l, b, h, n):
    return (X.rows_of if kv.k_scale is not None and kv.k_tail is None else rows_of)(kv, l, b, h, n)


def behind(M, fmt, dtype, lens, first, shared, L=1, Hkv=2, d=64, page=16, seed=3, cap=None):
    """A cache whose groups share the pages of their first rows: each sequence's rows are appended, then the groups' tables are
    pointed to the first sequence's pages (whole ones) for them."""
    B, cap = len(lens), cap or -(-max(lens) // page) + 1
    kw = dict(L=L, B=B, Hkv=Hkv, d=d, dtype=dtype, page=page, cap=cap)
    kv = make4(M, **kw) if fmt == "mx4" else make(M, fp8=fmt == "e4m3", **kw)
    n = max(lens)
    k, v = tokens((L, B, Hkv, n, d), dtype, seed), tokens((L, B, Hkv, n, d), dtype, seed + 1, spread=False)
    kv.lens.copy_(torch.tensor(lens))
    M.mpc_paged_append(k.cuda(), v.cuda(), kv, n_valid=kv.lens.clone())
    torch.cuda.synchronize()
    for g, rows in enumerate(shared):
        for b in range(first[g] + 1, first[g + 1]):
            # in the sequence's own table these entries are not read for shared rows: nothing good stands there
            kv.table[b, : rows // page] = 2 ** 30
    return kv


def run(M, kv, q, first, shared, new=None, window=0, sinks=0, ws=None, sm=None):
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:4], 7.0, device="cuda")
    M.mpc_shared_attn(q, kv, out, first=ints(first), shared_rows=ints(shared), sm_scale=sm or 1 / math.sqrt(kv.d), window=window, sinks=sinks,
                      n_valid=None if new is None else ints(new), lse=lse, ws=ws)
    return out, lse


def bounded(kv, *args):
    """The bound of the unshared form, and one rounding of each weight to the type: paged_ref.bounds has that for every type; fp16
    queries over 4-bit codes are added up in two parts as well."""
    b, l = R.bounds(*args)
    if kv.k_tail is None and kv.k_scale is not None:
        b2, l2 = X.bounds(*args)
        w, v = args[4], args[2][args[3]]
        b, l = torch.maximum(b, b2) + (0 if w is None else 2.0 ** -8 * (w @ v.abs())), max(l, l2)
    return b, l


def check(kv, q, out, lse, lens, first, shared, new=None, window=0, sinks=0, units=None, sm=None):
    L, B, Hq, n, d = q.shape
    G, sm, page, cap = Hq // kv.Hkv, sm or 1 / math.sqrt(d), kv.page, kv.table.shape[1] * kv.page
    leader, base = list(range(B)), [0] * B
    for g, rows in enumerate(shared):
        for b in range(first[g], first[g + 1]):
            leader[b], base[b] = first[g], min(max(rows, 0), cap) // page * page
    qc, oc, lc = q.cpu(), out.cpu(), lse.cpu()
    for l in range(L):
        for b in range(B):
            m = n if new is None else new[b]
            for h in range(kv.Hkv):
                if units is not None and (l, b, h) not in units:
                    continue
                T = min(lens[b], cap)
                k, v, has = held(kv, l, b, h, T)
                if base[b]:
                    z = min(base[b], T)
                    for x, y in zip((k, v, has), held(kv, l, leader[b], h, max(base[b], lens[leader[b]]))):
                        x[:z] = y[:z]
                for hq in range(h * G, (h + 1) * G):
                    assert bool((oc[l, b, hq, m:] == 7).all()) and bool((lc[l, b, hq, m:] == 7).all())
                    for t in range(m):
                        x = qc[l, b, hq, t].double()
                        o, ls, idx, w = R.attend(x, k, v, lens[b] - m + t, sm, window, sinks, has)
                        bo, bl = bounded(kv, x, k, v, idx, w, o, ls, sm, q.dtype)
                        R.check(oc[l, b, hq, t], o, bo, f"out l{l} b{b} h{hq} t{t}")
                        R.check(lc[l, b, hq, t], ls, bl, f"lse l{l} b{b} h{hq} t{t}")


FORMATS = ["same", "e4m3", "mx4"]
CASES = [
    # Hq, Hkv, d, page, n, lens, new, first, shared
    (2, 2, 64, 16, 1, [100, 81, 130], None, [0, 3], [80]),
    (8, 2, 128, 32, 1, [300, 257, 290, 70, 69], None, [0, 3, 5], [256, 64]),
    (8, 1, 128, 16, 3, [50, 51, 49, 60, 200, 53, 48], [3, 0, 1, 3, 2, 3, 3], [0, 7], [48]),
    (4, 4, 64, 64, 2, [130, 70, 200, 300], None, [1, 2, 4], [64, 192]),  # one outside, one alone, a pair
    (4, 1, 64, 128, 17, [400, 390, 300], [17, 9, 1], [0, 2, 3], [383, 0]),  # rows that are no whole pages; none
    (8, 2, 128, 16, 9, [600, 590, 610, 580, 577, 1000, 576, 999, 640], [9, 9, 1, 0, 1, 9, 2, 9, 9], [0, 9], [560]),
]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_the_definition(fmt, dtype, case):
    import paper_2501_06807_amd as M
    Hq, Hkv, d, page, n, lens, new, first, shared = CASES[case]
    kv = behind(M, fmt, dtype, lens, first, shared, 2, Hkv, d, page)
    q = tokens((2, len(lens), Hq, n, d), dtype, 9).cuda()
    out, lse = run(M, kv, q, first, shared, new)
    check(kv, q, out, lse, lens, first, shared, new)


@pytest.mark.parametrize("fmt,dtype", [("same", "fp32"), ("same", "bf16"), ("e4m3", "fp16"), ("mx4", "fp16"), ("e4m3", "bf16")])
@pytest.mark.parametrize("window,sinks", [(1, 0), (20, 0), (100, 4), (33, 40), (150, 100), (5000, 7)])
def test_windows_and_sinks(fmt, dtype, window, sinks):
    """Windows that reach some of the shared rows, none of them, or not all of a sequence's own; sinks on both sides."""
    import paper_2501_06807_amd as M
    lens, new, first, shared = [170, 97, 130, 260, 96], [4, 1, 0, 4, 2], [0, 4, 5], [96, 64]
    kv = behind(M, fmt, dtype, lens, first, shared)
    q = tokens((1, 5, 4, 4, 64), dtype, 9).cuda()
    out, lse = run(M, kv, q, first, shared, new, window, sinks)
    check(kv, q, out, lse, lens, first, shared, new, window, sinks)


@pytest.mark.parametrize("fmt", ["same", "mx4"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_sequences_shorter_than_the_shared_rows(fmt, dtype):
    """They see their first rows of them; an empty one sees nothing."""
    import paper_2501_06807_amd as M
    lens, first, shared = [100, 20, 33, 90], [0, 4], [64]
    kv = behind(M, fmt, dtype, [100, 70, 70, 90], first, shared)
    lens[2] = 0
    kv.lens.copy_(torch.tensor(lens))
    q = tokens((1, 4, 4, 2, 64), dtype, 9).cuda()
    out, lse = run(M, kv, q, first, shared)
    check(kv, q, out, lse, lens, first, shared)
    assert bool((out[0, 2] == 0).all()) and bool((lse[0, 2] == -math.inf).all())


@pytest.mark.parametrize("first,means", [([3, 1, 5], [3, 3, 5]), ([-7, 2, 1 << 30], [0, 2, 5]), ([9, -1, 4], [5, 5, 5]), ([0, 0, 0], [0, 0, 0])])
def test_groups_that_are_out_of_order(first, means):
    import paper_2501_06807_amd as M
    lens, shared = [100, 90, 95, 81, 99], [64, 80]
    kv = behind(M, "same", "bf16", lens, [0, 0, 0], [0, 0])
    q = tokens((1, 5, 4, 1, 64), "bf16", 9).cuda()
    out, lse = run(M, kv, q, first, shared)
    check(kv, q, out, lse, lens, means, shared)


@pytest.mark.parametrize("rows", [-5, 15, 16, 2 ** 31 - 1])
def test_numbers_of_shared_rows(rows):
    """Below a page, and beyond the table: what is not there is seen by nobody."""
    import paper_2501_06807_amd as M
    lens, first = [100, 90, 95], [0, 3]
    kv = behind(M, "same", "bf16", lens, first, [0])
    q = tokens((1, 3, 4, 1, 64), "bf16", 9).cuda()
    out, lse = run(M, kv, q, first, [rows])
    check(kv, q, out, lse, lens, first, [rows])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
def test_what_a_row_does_not_see_does_not_reach_it(fmt, dtype):
    """NaN among the shared rows: in one that only a window's rows see, and behind all rows of a sequence."""
    import paper_2501_06807_amd as M
    lens, first, shared = [120, 100, 103], [0, 3], [96]
    kv = behind(M, fmt, dtype, lens, first, shared, Hkv=1)
    lens[1] = 40
    kv.lens.copy_(torch.tensor(lens))
    id = int(kv.table[0, 3])  # rows 48..63
    for pages, scale in ((kv.k_pages, kv.k_scale), (kv.v_pages, kv.v_scale)):
        if fmt == "mx4":
            scale[0, id, 0, 1, 7] = 255
        else:
            pages[0, id, 0, 7, 5] = math.nan
    q = tokens((1, 3, 2, 2, 64), dtype, 9).cuda()
    out, lse = run(M, kv, q, first, shared, window=60)
    check(kv, q, out, lse, lens, first, shared, window=60)
    assert bool(out[0, 1].isfinite().all()) and bool(out[0, 2].isnan().all()) and bool(out[0, 0].isfinite().all())


@pytest.mark.parametrize("fmt", FORMATS)
def test_pages_that_are_missing(fmt):
    import paper_2501_06807_amd as M
    lens, first, shared = [120, 100, 103], [0, 3], [96]
    kv = behind(M, fmt, "bf16", lens, first, shared)
    kv.table[0, 2], kv.table[0, 5] = -1, kv.k_pages.shape[1]
    q = tokens((1, 3, 4, 2, 64), "bf16", 9).cuda()
    out, lse = run(M, kv, q, first, shared)
    check(kv, q, out, lse, lens, first, shared)


@pytest.mark.parametrize("fmt,dtype", [("same", "bf16"), ("same", "fp16"), ("e4m3", "bf16"), ("e4m3", "fp16"), ("mx4", "bf16"), ("mx4", "fp16"), ("mx4", "fp32")])
@pytest.mark.parametrize("B,G,n,T", [(40, 4, 1, 3000), (6, 8, 40, 2000), (70, 1, 1, 1504), (3, 2, 130, 5008)])
def test_many_rows_behind_long_prompts(fmt, dtype, B, G, n, T):
    """Units of several hundred rows that many workgroups share."""
    import paper_2501_06807_amd as M
    base = T // 16 * 16
    lens = [base + n + (7 * b) % 50 for b in range(B)]
    new = [n - (3 * b) % n for b in range(B)]
    first, shared = [0, B], [T]
    kv = behind(M, fmt, dtype, lens, first, shared, Hkv=1, d=128)
    q = tokens((1, B, G, n, 128), dtype, 9).cuda()
    out, lse = run(M, kv, q, first, shared, new)
    check(kv, q[:, :, :1], out[:, :, :1], lse[:, :, :1], lens, first, shared, new, units=[(0, 0, 0), (0, 1, 0), (0, B - 1, 0)])
    # the other heads and sequences against the form that shares nothing
    for b in range(1, B):
        kv.table[b, : base // 16] = kv.table[0, : base // 16]
    ref, lse2 = torch.full_like(q, 7.0), torch.full(q.shape[:4], 7.0, device="cuda")
    M.mpc_paged_attn(q, kv, ref, sm_scale=1 / math.sqrt(128), n_valid=ints(new), lse=lse2)
    # each is within its bound of the exact one: weights rounded to the type (in one of them, or both), outputs rounded twice
    tol = 4 * R.half_step(DT[dtype]) if dtype != "fp32" else 2e-5
    assert float((out.float() - ref.float()).norm() / ref.float().norm()) < tol
    assert float((lse - lse2).abs().max()) < 1e-4


def test_hundreds_of_groups_and_sequences():
    import paper_2501_06807_amd as M
    B, page = 1100, 16
    lens = [17 + b % 30 for b in range(B)]
    first = [min(b, B) for b in range(0, 1023)] + [B]  # 1022 of one sequence, one of 78
    shared = [16] * 1023
    kv = behind(M, "same", "bf16", lens, first, shared, Hkv=1, cap=4)
    q = tokens((1, B, 2, 1, 64), "bf16", 9).cuda()
    out, lse = run(M, kv, q, first, shared)
    check(kv, q, out, lse, lens, first, shared, units=[(0, b, 0) for b in list(range(0, B, 97)) + [1021, 1022, 1023, B - 1]])


def test_one_workspace_for_every_call():
    """Of other shapes, of the paged attention, and again: the same bits."""
    import paper_2501_06807_amd as M
    lens, first, shared = [700, 590, 650, 581], [0, 4], [576]
    kv = behind(M, "e4m3", "bf16", lens, first, shared, Hkv=2, d=128)
    q = tokens((1, 4, 16, 5, 128), "bf16", 9).cuda()
    ws = M.workspace(M.shared_attn_workspace_bytes(q, kv, 4))
    a = run(M, kv, q, first, shared, ws=ws)
    check(kv, q, *a, lens, first, shared, units=[(0, 1, 0), (0, 3, 1)])
    one = q[:, :, :2, :1].contiguous()
    b = run(M, kv, one, [0, 1, 2, 4], [576, 0, 320], ws=ws)
    check(kv, one, *b, lens, [0, 1, 2, 4], [576, 0, 320])
    out = torch.zeros_like(one)
    for t in range(1, 4):
        kv.table[t, :36] = kv.table[0, :36]
    M.mpc_paged_attn(one, kv, out, sm_scale=1 / math.sqrt(128), ws=ws)
    fresh = torch.zeros_like(one)
    M.mpc_paged_attn(one, kv, fresh, sm_scale=1 / math.sqrt(128))
    assert torch.equal(bits(out), bits(fresh))
    again = run(M, kv, q, first, shared, ws=ws)
    assert torch.equal(bits(a[0]), bits(again[0])) and torch.equal(bits(a[1]), bits(again[1]))


def test_a_captured_call_follows_lengths_tables_and_groups():
    import paper_2501_06807_amd as M
    page, lens, first, shared = 16, [200, 170, 180, 190], [0, 4], [160]
    kv = behind(M, "mx4", "bf16", lens, first, shared, cap=16)
    q = tokens((1, 4, 8, 1, 64), "bf16", 9).cuda()
    f, r, ws = ints(first + [0]), ints(shared + [0]), M.workspace(M.shared_attn_workspace_bytes(q, kv, 2))
    f[2] = 4
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:4], device="cuda")

    def step():
        M.mpc_shared_attn(q, kv, out, first=f, shared_rows=r, sm_scale=0.125, lse=lse, ws=ws)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for lens, first, shared in (([200, 170, 180, 190], [0, 4, 4], [160, 0]), ([201, 165, 180, 191], [0, 4, 4], [160, 0]),
                                ([150, 165, 170, 190], [0, 2, 4], [64, 160]), ([200, 170, 180, 190], [1, 1, 1], [16, 16])):
        kv.lens.copy_(torch.tensor(lens))
        f.copy_(torch.tensor(first))
        r.copy_(torch.tensor(shared))
        kv.table[1:, :10] = kv.table[0, :10]
        out.fill_(9)
        g.replay()
        torch.cuda.synchronize()
        got = (out.clone(), lse.clone())
        check(kv, q, *got, lens, first, shared)
        step()
        torch.cuda.synchronize()
        assert torch.equal(bits(out), bits(got[0])) and torch.equal(bits(lse), bits(got[1]))


def test_strides_and_another_stream():
    import paper_2501_06807_amd as M
    lens, first, shared = [200, 170, 180], [0, 3], [160]
    kv = behind(M, "same", "fp16", lens, first, shared, L=2)
    q = tokens((2, 3, 4, 3, 64), "fp16", 9).cuda()
    a = run(M, kv, q, first, shared)
    qt = q.transpose(2, 3).contiguous().transpose(2, 3)
    out = torch.zeros(2, 3, 3, 4, 64, dtype=torch.float16, device="cuda").transpose(2, 3)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    M.mpc_shared_attn(qt, kv, out, first=ints(first), shared_rows=ints(shared), sm_scale=0.125, stream=st)
    st.synchronize()
    assert torch.equal(bits(out), bits(a[0]))
