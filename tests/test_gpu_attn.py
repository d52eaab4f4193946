"""mpc_paged_attn and mpc_prompt_attn against the softmax's definition in 64 bits: types, head layouts, lengths from none to
several pages, windows, sinks, ragged batches, and values that a row may not see."""
import math

import pytest
import torch

import paged_ref as R
from gpu_util import say
from test_gpu_paged_append import DT, bits, make, tokens

pytestmark = pytest.mark.gpu


def rows_of(kv, l, b, h, n):
    """K and V rows [0, n) of a sequence as the cache holds them, in 64 bits, and which rows have a page."""
    page, out, has = kv.page, [], torch.zeros(n, dtype=torch.bool)
    codes = kv.k_scale is not None
    done = n // page * page if codes else n
    for pages, scale, ring in ((kv.k_pages, kv.k_scale, kv.k_tail), (kv.v_pages, kv.v_scale, kv.v_tail)):
        x = torch.full((n, kv.d), math.nan, dtype=torch.float64)
        for j0 in range(0, n, page):
            m, id = min(page, n - j0), int(kv.table[b, j0 // page])
            if j0 >= done:
                x[j0:n] = ring[l, b, h, [j % (2 * page) for j in range(j0, n)]].cpu().double()
                has[j0:n] = True
            elif 0 <= id < pages.shape[1]:
                x[j0:j0 + m] = pages[l, id, h, :m].cpu().double() * (float(scale[l, id, h]) if codes else 1.0)
                has[j0:j0 + m] = True
        out.append(x)
    return out[0], out[1], has


def fill(kv, lens, seed, dtype, scale=1.0):
    """Appends random rows, sequence by sequence lengths `lens`."""
    import paper_2501_06807_amd as M
    n = max(max(lens), 1)
    k = tokens((kv.L, kv.B, kv.Hkv, n, kv.d), dtype, seed)
    v = tokens((kv.L, kv.B, kv.Hkv, n, kv.d), dtype, seed + 1, spread=False) * scale
    kv.lens.copy_(torch.tensor(lens))
    M.mpc_paged_append(k.cuda(), v.cuda(), kv, n_valid=torch.tensor(lens, dtype=torch.int32, device="cuda"))


def check_paged(kv, q, out, lse, lens, new, window, sinks, sm, what, units=None):
    L, B, Hq, n, d = q.shape
    G = Hq // kv.Hkv
    qc, oc, lc = q.cpu(), out.cpu(), lse.cpu()
    cap = kv.table.shape[1] * kv.page
    for l in range(L):
        for b in range(B):
            for h in range(kv.Hkv):
                if units is not None and (l, b, h) not in units:
                    continue
                k, v, has = rows_of(kv, l, b, h, min(lens[b], cap))
                for hq in range(h * G, (h + 1) * G):
                    for t in range(n):
                        w_ = f"{what} l{l} b{b} h{hq} t{t}"
                        if t >= new[b]:
                            assert bool((oc[l, b, hq, t] == 7).all()) and float(lc[l, b, hq, t]) == 7, w_
                            continue
                        x = qc[l, b, hq, t].double()
                        o, ls, idx, w = R.attend(x, k, v, lens[b] - new[b] + t, sm, window, sinks, has)
                        bo, bl = R.bounds(x, k, v, idx, w, o, ls, sm, q.dtype)
                        R.check(oc[l, b, hq, t], o, bo, "out " + w_)
                        R.check(lc[l, b, hq, t], ls, bl, "lse " + w_)


def run_paged(kv, q, new, window=0, sinks=0, sm=None, ws=None, stream=None):
    import paper_2501_06807_amd as M
    out = torch.full_like(q, 7.0)
    lse = torch.full(q.shape[:4], 7.0, device="cuda")
    M.mpc_paged_attn(q, kv, out, sm_scale=q.shape[-1] ** -0.5 if sm is None else sm, window=window, sinks=sinks,
                     n_valid=torch.tensor(new, dtype=torch.int32, device="cuda"), lse=lse, ws=ws, stream=stream)
    torch.cuda.synchronize()
    return out, lse


PAGED = [  # dtype, fp8, page, d, Hq, Hkv, n, window, sinks
    ("bf16", True, 16, 128, 4, 4, 1, 0, 0), ("bf16", True, 64, 128, 8, 2, 1, 0, 0), ("fp16", True, 32, 64, 8, 1, 3, 0, 0),
    ("fp32", True, 16, 64, 2, 2, 2, 0, 0), ("fp32", False, 16, 128, 4, 2, 1, 0, 0), ("bf16", False, 16, 64, 8, 1, 5, 0, 0),
    ("fp16", False, 64, 128, 4, 4, 2, 0, 0), ("fp32", False, 32, 64, 8, 1, 9, 0, 0), ("bf16", True, 256, 64, 4, 1, 1, 0, 0),
    ("bf16", True, 16, 128, 8, 2, 4, 37, 4), ("fp16", False, 16, 64, 4, 4, 3, 1, 0), ("fp32", True, 32, 128, 4, 1, 2, 50, 33),
    ("bf16", False, 64, 128, 8, 1, 4, 16, 1), ("fp16", True, 64, 64, 2, 1, 1, 300, 200), ("bf16", True, 128, 128, 4, 4, 19, 70, 2),
    ("bf16", False, 16, 128, 8, 1, 40, 0, 0), ("fp32", False, 64, 64, 4, 4, 33, 20, 3),
]


@pytest.mark.parametrize("dtype,fp8,page,d,Hq,Hkv,n,window,sinks", PAGED)
def test_paged_attention_of_ragged_batches(dtype, fp8, page, d, Hq, Hkv, n, window, sinks):
    import paper_2501_06807_amd as M
    lens = [1, n, 2 * page, 2 * page + 1, 15, 3 * page - 1, 200 + page, 0]
    new = [min(1, n), n, n, max(1, n - 1), 0, n, n, n]
    cap = -(-max(lens) // page)
    kv = make(M, 1, len(lens), Hkv, d, dtype, page, cap=cap, fp8=fp8)
    fill(kv, lens, 11, dtype)
    q = tokens((1, len(lens), Hq, n, d), dtype, 3, spread=False).cuda()
    out, lse = run_paged(kv, q, new, window, sinks)
    check_paged(kv, q, out, lse, lens, new, window, sinks, d ** -0.5, f"{dtype} {fp8}")


@pytest.mark.parametrize("dtype,fp8", [("bf16", True), ("fp16", False), ("fp32", False)])
def test_paged_attention_of_a_long_cache(dtype, fp8):
    """Few rows and a long axis: the keys are divided over workgroups and joined; two calls with one workspace agree."""
    import paper_2501_06807_amd as M
    lens, page, d = [20011, 130, 9000], 32, 128
    kv = make(M, 2, 3, 2, d, dtype, page, cap=626, fp8=fp8)
    fill(kv, lens, 5, dtype)
    q = tokens((2, 3, 8, 1, d), dtype, 3, spread=False).cuda()
    ws = M.workspace(M.paged_attn_workspace_bytes(q, kv))
    out, lse = run_paged(kv, q, [1, 1, 1], ws=ws)
    for _ in range(3):
        again = run_paged(kv, q, [1, 1, 1], ws=ws)
        assert torch.equal(bits(out), bits(again[0])) and torch.equal(bits(lse), bits(again[1]))
    check_paged(kv, q, out, lse, lens, [1, 1, 1], 0, 0, d ** -0.5, dtype)
    out, lse = run_paged(kv, q, [1, 1, 1], 4000, 5, ws=ws)
    check_paged(kv, q, out, lse, lens, [1, 1, 1], 4000, 5, d ** -0.5, dtype + " window", {(0, 0, 0), (1, 2, 1), (1, 1, 0)})


@pytest.mark.parametrize("dtype,fp8", [("fp16", False), ("fp16", True), ("bf16", False), ("bf16", True)])
def test_small_weights_of_large_values(dtype, fp8):
    """One key in a page of its own has a weight of 2^-14 to 2^-22 of the largest and a value 2^15 times theirs."""
    import paper_2501_06807_amd as M
    d, page, T = 64, 16, 64
    k = torch.zeros(1, 1, 1, T, d)
    k[..., 0] = 4 + 0.001 * torch.arange(T)
    v = tokens((1, 1, 1, T, d), dtype, 2, spread=False).float()
    q = torch.zeros(1, 1, 2, 1, d)
    q[..., 0] = torch.tensor([1.0, 1.5])[None, None, :, None]
    k[0, 0, 0, 20, 0] = -6.0
    v[0, 0, 0, 16:32] = 0
    v[0, 0, 0, 20] = 30000.0
    k, v, q = (x.to(DT[dtype]) for x in (k, v, q))
    kv = make(M, 1, 1, 1, d, dtype, page, cap=5, fp8=fp8)
    kv.lens.fill_(T)
    M.mpc_paged_append(k.cuda(), v.cuda(), kv)
    out, lse = run_paged(kv, q.cuda(), [1], sm=1.0)
    check_paged(kv, q.cuda(), out, lse, [T], [1], 0, 0, 1.0, f"{dtype} {fp8}")
    po, pl = torch.empty_like(q).cuda(), torch.empty(1, 1, 2, 1, device="cuda")
    M.mpc_prompt_attn(q.cuda(), k.cuda(), v.cuda(), po, sm_scale=1.0, lse=pl)
    for h in range(2):
        x, kd, vd = q[0, 0, h, 0].double(), k[0, 0, 0].double(), v[0, 0, 0].double()
        o, ls, idx, w = R.attend(x, kd, vd, T - 1, 1.0, 0, 0)
        assert 2.0 ** -22 < float(w[20] / w.max()) < 2.0 ** -14
        bo, bl = R.bounds(x, kd, vd, idx, w, o, ls, 1.0, DT[dtype])
        R.check(po[0, 0, h, 0].cpu(), o, bo, f"prompt h{h}")
        R.check(pl[0, 0, h, 0].cpu(), ls, bl, f"prompt lse h{h}")


@pytest.mark.parametrize("fp8", [False, True])
def test_paged_attention_of_more_sequences_than_a_wave_has_lanes(fp8):
    import paper_2501_06807_amd as M
    B = 150
    g = torch.Generator().manual_seed(4)
    lens = torch.randint(0, 90, (B,), generator=g).tolist()
    new = [min(n, 2) if b % 7 else 0 for b, n in enumerate(lens)]
    kv = make(M, 2, B, 1, 64, "bf16", 16, cap=6, fp8=fp8)
    fill(kv, lens, 3, "bf16")
    q = tokens((2, B, 4, 2, 64), "bf16", 9, spread=False).cuda()
    out, lse = run_paged(kv, q, new)
    check_paged(kv, q, out, lse, lens, new, 0, 0, 0.125, "many", {(l, b, 0) for l in range(2) for b in range(0, B, 5)} | {(1, 149, 0), (0, 63, 0), (0, 64, 0)})


@pytest.mark.parametrize("sm", [-0.2, 0.0])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_scales_of_zero_and_below(sm, dtype):
    import paper_2501_06807_amd as M
    lens = [77, 5]
    kv = make(M, 1, 2, 2, 64, dtype, 16, cap=5, fp8=dtype == "bf16")
    fill(kv, lens, 3, dtype)
    q = tokens((1, 2, 4, 3, 64), dtype, 9, spread=False).cuda()
    out, lse = run_paged(kv, q, [3, 3], 20, 2, sm=sm)
    check_paged(kv, q, out, lse, lens, [3, 3], 20, 2, sm, "scale")
    T = 100
    q, k, v = (tokens((1, 1, 2, T, 64), dtype, s, spread=False) for s in (1, 2, 3))
    out, lse = torch.empty_like(q).cuda(), torch.empty(1, 1, 2, T, device="cuda")
    M.mpc_prompt_attn(q.cuda(), k.cuda(), v.cuda(), out, sm_scale=sm, window=30, sinks=2, lse=lse)
    for h in range(2):
        for t in (0, 1, 31, 32, 99):
            x, kd, vd = q[0, 0, h, t].double(), k[0, 0, h].double(), v[0, 0, h].double()
            o, ls, idx, w = R.attend(x, kd, vd, t, sm, 30, 2)
            bo, bl = R.bounds(x, kd, vd, idx, w, o, ls, sm, DT[dtype])
            R.check(out[0, 0, h, t].cpu(), o, bo, f"h{h} t{t}")
            R.check(lse[0, 0, h, t].cpu(), ls, bl, f"lse h{h} t{t}")


def test_paged_scales_far_from_one():
    """Values of 2^-16 and 2^10 times the ordinary size, in 8-bit pages of each type: no range is lost on the way."""
    import paper_2501_06807_amd as M
    for dtype, scale in (("fp16", 2.0 ** -10), ("fp16", 2.0 ** 10), ("bf16", 2.0 ** -40), ("bf16", 2.0 ** 60), ("fp32", 2.0 ** -60)):
        kv = make(M, 1, 1, 1, 64, dtype, 16, cap=8)
        fill(kv, [100], 2, dtype, scale)
        q = tokens((1, 1, 2, 1, 64), dtype, 3, spread=False).cuda()
        out, lse = run_paged(kv, q, [1])
        tiny = 2.0 ** -24 if dtype == "fp16" else 0.0
        k, v, _ = rows_of(kv, 0, 0, 0, 100)
        for hq in range(2):
            x = q[0, 0, hq, 0].cpu().double()
            o, ls, idx, w = R.attend(x, k, v, 99, 0.125, 0, 0)
            bo, bl = R.bounds(x, k, v, idx, w, o, ls, 0.125, q.dtype)
            assert float(bo.max()) < 0.1 * float(o.abs().max()) + 2 * tiny
            R.check(out[0, 0, hq, 0].cpu(), o, bo, f"{dtype} {scale}")
            R.check(lse[0, 0, hq, 0].cpu(), ls, bl, f"{dtype} {scale} lse")


@pytest.mark.parametrize("dtype,fp8", [("bf16", False), ("bf16", True), ("fp16", False), ("fp32", False), ("fp32", True)])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_paged_values_that_a_row_does_not_see(dtype, fp8, bad):
    """Rows behind the window, ahead of a drafted token's position and behind the length hold NaN or infinities."""
    import paper_2501_06807_amd as M
    d, page, n, window, sinks, length = 64, 16, 4, 20, 2, 75
    kv = make(M, 1, 1, 2, d, dtype, page, cap=7, fp8=fp8)
    k, v = tokens((1, 1, 2, length, d), dtype, 1), tokens((1, 1, 2, length, d), dtype, 2)
    for j in (5, 30, 40, 73):  # 5, 30, 40: behind the window of every new token; 73: ahead of rows 71 and 72
        k[0, 0, 0, j] = bad
        v[0, 0, :, j, ::3] = bad
    kv.lens.fill_(length)
    M.mpc_paged_append(k.cuda(), v.cuda(), kv)
    if fp8:  # slots of the ring that hold no row of the sequence's last page yet
        free = [j % (2 * page) for j in range(length, length + page)]
        for t in (kv.k_tail, kv.v_tail):
            t[:, :, :, free] = bad
    q = tokens((1, 1, 4, n, d), dtype, 3, spread=False).cuda()
    out, lse = run_paged(kv, q, [n], window, sinks)
    assert bool(out[0, 0, :, :2].isfinite().all()) and bool(lse[0, 0, :, :2].isfinite().all())
    for h in range(2):
        kr, vr, _ = rows_of(kv, 0, 0, h, length)
        for hq in (2 * h, 2 * h + 1):
            for t in range(2):
                x = q[0, 0, hq, t].cpu().double()
                o, ls, idx, w = R.attend(x, kr, vr, length - n + t, d ** -0.5, window, sinks)
                bo, bl = R.bounds(x, kr, vr, idx, w, o, ls, d ** -0.5, q.dtype)
                R.check(out[0, 0, hq, t].cpu(), o, bo, f"h{hq} t{t}")
                R.check(lse[0, 0, hq, t].cpu(), ls, bl, f"lse h{hq} t{t}")
    # rows 73 and 74 see row 73: their outputs carry what stands in V there (codes hold an infinity as 448 scales)
    assert bool(out[0, 0, 2:, 2:, 1::3].isfinite().all())
    if not fp8 or math.isnan(bad):
        assert not bool(out[0, 0, 2:, 2:, ::3].isfinite().any())


def test_scores_of_infinity():
    """A weight of -infinity is zero, a row of nothing but those is empty, +infinity makes a row NaN."""
    import paper_2501_06807_amd as M
    for dtype, fp8 in (("fp32", False), ("bf16", False)):
        kv = make(M, 1, 3, 1, 64, dtype, 16, cap=3, fp8=fp8)
        k, v = tokens((1, 3, 1, 40, 64), dtype, 1).abs(), tokens((1, 3, 1, 40, 64), dtype, 2)
        k[0, 0, 0, 7, 0] = -math.inf
        k[0, 1, 0, :, 0] = -math.inf
        k[0, 2, 0, 39, 0] = math.inf
        kv.lens.fill_(40)
        M.mpc_paged_append(k.cuda(), v.cuda(), kv)
        q = tokens((1, 3, 1, 1, 64), dtype, 3).abs().cuda()
        out, lse = run_paged(kv, q, [1, 1, 1])
        x, kr, vr = q[0, 0, 0, 0].cpu().double(), k[0, 0, 0].double(), v[0, 0, 0].double()
        keep = [j for j in range(40) if j != 7]
        o, ls, idx, w = R.attend(x, kr[keep], vr[keep], 38, 0.125, 0, 0)
        bo, bl = R.bounds(x, kr[keep], vr[keep], idx, w, o, ls, 0.125, q.dtype)
        R.check(out[0, 0, 0, 0].cpu(), o, bo, dtype)
        assert bool((out[0, 1] == 0).all()) and float(lse[0, 1, 0, 0]) == -math.inf
        assert bool(out[0, 2].isnan().all()) and math.isnan(float(lse[0, 2, 0, 0]))


def test_paged_pages_out_of_range_are_absent():
    import paper_2501_06807_amd as M
    for fp8 in (False, True):
        kv = make(M, 1, 3, 2, 64, "bf16", 16, cap=6, fp8=fp8)
        lens = [90, 96, 500]  # the last one is longer than its table: its rows end at 96
        fill(kv, [90, 96, 96], 3, "bf16")
        kv.table[0, 2], kv.table[1, 0], kv.table[1, 5] = -1, kv.k_pages.shape[1], -(2 ** 31)
        kv.lens.copy_(torch.tensor(lens))
        q = tokens((1, 3, 4, 2, 64), "bf16", 3, spread=False).cuda()
        out, lse = run_paged(kv, q, [2, 2, 2])
        check_paged(kv, q, out, lse, lens, [2, 2, 2], 0, 0, 0.125, f"fp8 {fp8}")


def test_paged_prefix_pages_shared_between_sequences():
    import paper_2501_06807_amd as M
    kv = make(M, 1, 2, 1, 128, "bf16", 32, cap=5)
    fill(kv, [150, 150], 3, "bf16")
    kv.table[1, :3] = kv.table[0, :3]
    q = tokens((1, 2, 4, 1, 128), "bf16", 3, spread=False).cuda()
    out, lse = run_paged(kv, q, [1, 1])
    check_paged(kv, q, out, lse, [150, 150], [1, 1], 0, 0, 128 ** -0.5, "shared")


def test_a_decode_loop_captured_once_follows_the_lengths():
    """One graph of append + attention, replayed while lengths, tables and inputs change on the device, equals the eager
    calls bit for bit; eager work of the same cache's twin runs between the replays."""
    import paper_2501_06807_amd as M
    L, B, Hq, Hkv, d, page = 2, 3, 8, 2, 128, 16
    rope = R.rope_table(512, d).cuda()
    start = [31, 300, 64]
    twins = []
    for _ in range(2):
        kv = make(M, L, B, Hkv, d, "bf16", page, cap=25)
        fill(kv, start, 7, "bf16")
        twins.append(kv)
    k, v = (torch.zeros(L, B, Hkv, 1, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.zeros(L, B, Hq, 1, d, dtype=torch.bfloat16, device="cuda")
    qr, out, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(L, B, Hq, 1, device="cuda")
    ws = M.workspace(M.paged_attn_workspace_bytes(q, twins[0]))
    ws2 = M.workspace(M.paged_attn_workspace_bytes(q, twins[0]))

    def step(kv, o, ls, w):
        kv.lens.add_(1)
        M.mpc_paged_append(k, v, kv, q=q, q_out=qr, rope=rope)
        M.mpc_paged_attn(qr, kv, o, sm_scale=d ** -0.5, lse=ls, ws=w)

    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(twins[0], out, lse, ws)
    out2, lse2 = torch.empty_like(out), torch.empty_like(lse)
    for i in range(20):
        for t, s, h in ((q, 1, Hq), (k, 2, Hkv), (v, 3, Hkv)):
            t.copy_(tokens((L, B, h, 1, d), "bf16", 100 * i + s))
        g.replay()
        step(twins[1], out2, lse2, ws2)
        torch.cuda.synchronize()
        assert torch.equal(bits(out), bits(out2)) and torch.equal(bits(lse), bits(lse2)), i
    lens = [s + 20 for s in start]
    assert twins[0].lens.tolist() == lens
    check_paged(twins[0], qr, out, lse, lens, [1] * B, 0, 0, d ** -0.5, "graph")


def test_single_tokens_without_their_axis():
    """[L][B][H][d] tensors are taken as one token each, as the other decode calls take them."""
    import paper_2501_06807_amd as M
    kv = make(M, 2, 3, 2, 64, "bf16", 16, cap=3)
    fill(kv, [20, 33, 48], 3, "bf16")
    kv.lens.sub_(1)
    k, v, q = (tokens((2, 3, h, 64), "bf16", s).cuda() for s, h in ((1, 2), (2, 2), (3, 8)))
    kv.lens.add_(1)
    M.mpc_paged_append(k, v, kv)
    out, lse = torch.empty_like(q), torch.empty(2, 3, 8, device="cuda")
    M.mpc_paged_attn(q, kv, out, sm_scale=0.125, lse=lse)
    torch.cuda.synchronize()
    check_paged(kv, q[:, :, :, None], out[:, :, :, None], lse[..., None], [20, 33, 48], [1] * 3, 0, 0, 0.125, "one")


def prompt_case(dtype, L, B, Hq, Hkv, d, Tq, T, q_lens, k_lens, window, sinks, seed=0, rows=None, token_major=False):
    import paper_2501_06807_amd as M
    q, k, v = (tokens((L, B, h, n, d), dtype, seed + s, spread=s == 2) for s, h, n in ((1, Hq, Tq), (2, Hkv, T), (3, Hkv, T)))
    if k_lens is not None:  # rows behind a sequence's keys are not looked at
        for b in range(B):
            k[:, b, :, max(0, k_lens[b]):] = math.nan
            v[:, b, :, max(0, k_lens[b]):] = math.inf
    dev = [x.cuda() for x in (q, k, v)]
    out = torch.full_like(dev[0], 7.0)
    if token_major:
        dev = [x.transpose(2, 3).contiguous().transpose(2, 3) for x in dev]
        out = out.transpose(2, 3).contiguous().transpose(2, 3)
    lse = torch.full((L, B, Hq, Tq), 7.0, device="cuda")
    ints = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    sm = d ** -0.5
    M.mpc_prompt_attn(*dev, out, sm_scale=sm, window=window, sinks=sinks, q_lens=ints(q_lens), k_lens=ints(k_lens), lse=lse)
    torch.cuda.synchronize()
    oc, lc, G = out.cpu(), lse.cpu(), Hq // Hkv
    for l in range(L):
        for b in range(B):
            ql = Tq if q_lens is None else min(max(q_lens[b], 0), Tq)
            kl = T if k_lens is None else min(max(k_lens[b], 0), T)
            for hq in range(Hq):
                kd, vd = k[l, b, hq // G, :kl].double(), v[l, b, hq // G, :kl].double()
                for t in range(Tq) if rows is None else rows:
                    what = f"l{l} b{b} h{hq} t{t}"
                    if t >= ql:
                        assert bool((oc[l, b, hq, t] == 7).all()) and float(lc[l, b, hq, t]) == 7, what
                        continue
                    x = q[l, b, hq, t].double()
                    o, ls, idx, w = R.attend(x, kd, vd, kl - ql + t, sm, window, sinks)
                    bo, bl = R.bounds(x, kd, vd, idx, w, o, ls, sm, DT[dtype])
                    R.check(oc[l, b, hq, t], o, bo, "out " + what)
                    R.check(lc[l, b, hq, t], ls, bl, "lse " + what)


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("d,Hq,Hkv", [(64, 2, 2), (128, 4, 1), (128, 8, 1), (64, 4, 2)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (33, 4), (100, 70)])
def test_prompt_attention(dtype, d, Hq, Hkv, window, sinks):
    prompt_case(dtype, 1, 1, Hq, Hkv, d, 140, 140, None, None, window, sinks)


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("Tq,T", [(1, 1), (1, 300), (5, 131), (129, 257), (64, 64), (300, 40)])
def test_prompt_attention_of_odd_lengths(dtype, Tq, T):
    """More rows than keys too: the first rows stand before key 0 and see nothing."""
    prompt_case(dtype, 2, 1, 2, 1, 64, Tq, T, None, None, 0, 0, seed=Tq, token_major=Tq % 2 == 1)
    prompt_case(dtype, 1, 1, 2, 2, 128, Tq, T, None, None, 20, 3, seed=Tq)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 5)])
def test_prompt_attention_of_padded_batches(dtype, window, sinks):
    prompt_case(dtype, 1, 7, 2, 1, 64, 130, 200, [130, 0, 1, 77, 130, 500, 64], [200, 50, 1, 77, 0, 130, -4], window, sinks)


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
def test_prompt_attention_of_long_prompts(dtype):
    rows = [0, 1, 31, 32, 127, 128, 129, 1000, 1023, 1024, 2047, 2999]
    prompt_case(dtype, 1, 1, 4, 2, 128, 3000, 3000, None, None, 0, 0, rows=rows)
    prompt_case(dtype, 1, 1, 4, 2, 128, 3000, 3000, None, None, 513, 9, rows=rows)
    prompt_case(dtype, 1, 1, 2, 1, 64, 200, 5000, None, None, 0, 0, rows=[0, 7, 100, 199])


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_prompt_values_that_a_row_does_not_see(dtype, d, bad):
    """K and V hold NaN or infinities at keys that some rows see and others do not: only those that see them carry it."""
    import paper_2501_06807_amd as M
    T, window, sinks = 300, 50, 3
    q, k, v = (tokens((1, 1, 2, T, d), dtype, s, spread=False) for s in (1, 2, 3))
    at = (40, 200, 207)
    clean = v.clone()
    for j in at:
        v[0, 0, :, j, ::5] = bad
        k[0, 0, 1, j] = bad
    out, lse = torch.empty_like(q).cuda(), torch.empty(1, 1, 2, T, device="cuda")
    M.mpc_prompt_attn(q.cuda(), k.cuda(), v.cuda(), out, sm_scale=d ** -0.5, window=window, sinks=sinks, lse=lse)
    out, lse = out.cpu(), lse.cpu()
    for t in range(T):
        sees = any(j <= t and t - window < j for j in at)
        for h in range(2):
            row = out[0, 0, h, t]
            if not sees or h == 0:
                x = q[0, 0, h, t].double()
                o, ls, idx, w = R.attend(x, k[0, 0, h].double(), clean[0, 0, h].double(), t, d ** -0.5, window, sinks)
                bo, bl = R.bounds(x, k[0, 0, h].double(), clean[0, 0, h].double(), idx, w, o, ls, d ** -0.5, DT[dtype])
                part = torch.arange(d) % 5 != 0 if sees else torch.ones(d, dtype=torch.bool)
                R.check(row[part], o[part], bo[part], f"t{t} h{h}")
                R.check(lse[0, 0, h, t], ls, bl, f"lse t{t} h{h}")
            if sees and h == 0:
                assert not bool(row[::5].isfinite().any()), t


def test_prompt_then_decode_as_they_are_used():
    """A prompt's attention equals, row by row within the bounds, the attention over the cache it was appended to."""
    import paper_2501_06807_amd as M
    L, B, Hq, Hkv, d, T = 1, 2, 4, 2, 64, 90
    rope = R.rope_table(200, d).cuda()
    for dtype in ("bf16", "fp32"):
        kv = make(M, L, B, Hkv, d, dtype, 16, cap=8, fp8=False)
        q, k, v = (tokens((L, B, h, T, d), dtype, s).cuda() for s, h in ((1, Hq), (2, Hkv), (3, Hkv)))
        kv.lens.fill_(T)
        qr = torch.empty_like(q)
        M.mpc_paged_append(k, v, kv, q=q, q_out=qr, rope=rope)
        pages = kv.k_pages[:, kv.table.long()[:, :6]].transpose(2, 3).flatten(3, 4)[:, :, :, :T].contiguous()
        out, lse = torch.empty_like(q), torch.empty(L, B, Hq, T, device="cuda")
        M.mpc_prompt_attn(qr, pages, v, out, sm_scale=d ** -0.5, window=30, sinks=4, lse=lse)
        got, gl = run_paged(kv, qr, [T, T], 30, 4)
        check_paged(kv, qr, got, gl, [T, T], [T, T], 30, 4, d ** -0.5, dtype)
        check_paged(kv, qr, out, lse, [T, T], [T, T], 30, 4, d ** -0.5, dtype + " prompt")
    say("[attn] prompt and paged forms agree")
