"""mpc_shared_attn where a group has many query rows (units of 128 of them in 16-bit types): windows, sinks, missing pages, values and scales
that a row may not see, sequences shorter than the shared rows, scales of scores, strides, captured calls, large batches and pools."""
import math

import pytest
import torch

from test_gpu_mx4_append import make4
from test_gpu_paged_append import bits, make, tokens
from test_gpu_shared_attn import FORMATS, behind, check, ints, run

pytestmark = pytest.mark.gpu

LENS = [190, 161, 300, 175, 164]  # behind 160 shared rows
KINDS = [("same", "bf16"), ("same", "fp16"), ("e4m3", "bf16"), ("e4m3", "fp16"), ("mx4", "bf16"), ("mx4", "fp16"), ("same", "fp32")]


def wide(M, fmt, dtype, lens=LENS, T=160, Hkv=1, G=4, n=5, d=64, page=16, L=1, **kw):
    """100 query rows of one group (and more of larger ones)."""
    kv = behind(M, fmt, dtype, lens, [0, len(lens)], [T], L, Hkv, d, page, **kw)
    return kv, tokens((L, len(lens), Hkv * G, n, d), dtype, 9).cuda(), [0, len(lens)], [T]


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (20, 0), (100, 4), (33, 40), (150, 100), (64, 33), (5000, 7)])
def test_windows_and_sinks(fmt, dtype, window, sinks):
    import paper_2501_06807_amd as M
    kv, q, first, shared = wide(M, fmt, dtype)
    new = [5, 1, 0, 5, 3]
    out, lse = run(M, kv, q, first, shared, new, window, sinks)
    check(kv, q, out, lse, LENS, first, shared, new, window, sinks)


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("page,d", [(16, 128), (32, 64), (64, 128), (128, 64), (256, 128)])
def test_page_sizes(fmt, dtype, page, d):
    """Shared rows of more than 64 halves of 16 keys, pages of every size, tiles that end inside a page and behind the last one."""
    import paper_2501_06807_amd as M
    T = 1040 if page == 16 else 4 * 256 + page
    lens = [T + 20, T + 5, T + 40]
    kv, q, first, shared = wide(M, fmt, dtype, lens, T, n=9, d=d, page=page)
    out, lse = run(M, kv, q, first, shared)
    check(kv, q, out, lse, lens, first, shared, units=[(0, 1, 0)])


@pytest.mark.parametrize("fmt,dtype", [k for k in KINDS if k[0] != "e4m3"])
@pytest.mark.parametrize("short", [1, 17, 100, 159])
def test_sequences_shorter_than_the_shared_rows(fmt, dtype, short):
    import paper_2501_06807_amd as M
    kv, q, first, shared = wide(M, fmt, dtype)
    lens = [190, short, 300, 0, 164]
    kv.lens.copy_(torch.tensor(lens))
    out, lse = run(M, kv, q, first, shared)
    check(kv, q, out, lse, lens, first, shared)
    assert bool((out[0, 3] == 0).all()) and bool((lse[0, 3] == -math.inf).all())


@pytest.mark.parametrize("fmt,dtype", KINDS)
def test_pages_that_are_missing(fmt, dtype):
    """Whatever lies in page 0, which stands in for them."""
    import paper_2501_06807_amd as M
    kv, q, first, shared = wide(M, fmt, dtype)
    hold = (kv.table == 0).nonzero()
    for t in (kv.k_pages, kv.v_pages):
        if hold.numel() == 0 or int(hold[0, 1]) >= 10:
            t[:, 0].view(torch.uint8).fill_(0x7F if fmt == "e4m3" else 0xFF)
    kv.table[0, 2], kv.table[0, 5], kv.table[0, 9] = -1, kv.k_pages.shape[1], 2 ** 31 - 1
    for window in (0, 90):
        out, lse = run(M, kv, q, first, shared, window=window)
        check(kv, q, out, lse, LENS, first, shared, window=window, units=[(0, 0, 0), (0, 2, 0)])


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("row", [0, 39, 151])
def test_nan_in_a_shared_row(fmt, dtype, row):
    """Rows whose window ends behind it stay numbers; the others become NaN, in the channels that hold it."""
    import paper_2501_06807_amd as M
    kv, q, first, shared = wide(M, fmt, dtype)
    id = int(kv.table[0, row // 16])
    if fmt == "mx4":
        kv.v_scale[0, id, 0, 1, row % 16] = 255
    else:
        kv.v_pages[0, id, 0, row % 16, 33] = math.nan
    for window in (0, 60):
        out, lse = run(M, kv, q, first, shared, window=window)
        check(kv, q, out, lse, LENS, first, shared, window=window)
        assert bool(lse.isfinite().all())


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("scale", [math.inf, math.nan, 0.0, -0.5, 2.0 ** -100, 3.0 ** 20])
def test_scales_of_a_page_that_rows_do_not_see(dtype, scale):
    """8-bit pages: what a window leaves out does not reach a row, whatever its page's scales are; seen ones multiply."""
    import paper_2501_06807_amd as M
    kv, q, first, shared = wide(M, "e4m3", dtype)
    id = int(kv.table[0, 1])  # rows 16..31
    clean, _ = run(M, kv, q, first, shared, window=60)
    kv.k_scale[0, id, 0] = kv.v_scale[0, id, 0] = scale
    out, lse = run(M, kv, q, first, shared, window=60)
    assert torch.equal(bits(out), bits(clean))
    if math.isfinite(scale) and 0 < abs(scale) < 100:
        out, lse = run(M, kv, q, first, shared)
        check(kv, q, out, lse, LENS, first, shared, units=[(0, 1, 0)])


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("sm", [-0.125, 1e-30, 0.5])
def test_scales_of_the_scores(fmt, dtype, sm):
    import paper_2501_06807_amd as M
    kv, q, first, shared = wide(M, fmt, dtype)
    out, lse = run(M, kv, q, first, shared, sm=sm)
    check(kv, q, out, lse, LENS, first, shared, sm=sm, units=[(0, 0, 0), (0, 4, 0)])


@pytest.mark.parametrize("fmt,dtype", [("same", "bf16"), ("mx4", "fp16"), ("e4m3", "fp16"), ("same", "fp32")])
def test_queries_that_are_not_finite_stay_by_themselves(fmt, dtype):
    import paper_2501_06807_amd as M
    kv, q, first, shared = wide(M, fmt, dtype)
    clean, l0 = run(M, kv, q, first, shared)
    q[0, 1, 2, 3, 7], q[0, 3, 0, 0, 0] = math.nan, math.inf
    out, lse = run(M, kv, q, first, shared)
    odd = torch.zeros(q.shape[:4], dtype=torch.bool, device="cuda")
    odd[0, 1, 2, 3] = odd[0, 3, 0, 0] = True
    assert bool(out[0, 1, 2, 3].isnan().all()) and bool(out[0, 3, 0, 0].isnan().all())
    assert torch.equal(bits(out[~odd]), bits(clean[~odd])) and torch.equal(bits(lse[~odd]), bits(l0[~odd]))


@pytest.mark.parametrize("fmt", FORMATS)
def test_strides_layers_and_heads(fmt):
    """Tokens before heads; two layers of three kv heads; the same bits as contiguous ones."""
    import paper_2501_06807_amd as M
    kv, q, first, shared = wide(M, fmt, "bf16", Hkv=3, L=2, d=128)
    a = run(M, kv, q, first, shared)
    check(kv, q, *a, LENS, first, shared, units=[(1, 2, 2), (0, 4, 0)])
    qt = q.permute(1, 3, 0, 2, 4).contiguous().permute(2, 0, 3, 1, 4)
    out = torch.zeros(5, 5, 2, 12, 128, dtype=torch.bfloat16, device="cuda").permute(2, 0, 3, 1, 4)
    M.mpc_shared_attn(qt, kv, out, first=ints(first), shared_rows=ints(shared), sm_scale=1 / math.sqrt(128))
    assert torch.equal(bits(out), bits(a[0]))


@pytest.mark.parametrize("B", [64, 65, 130])
@pytest.mark.parametrize("fmt", ["e4m3", "mx4"])
def test_captured_calls_of_batches_on_both_sides_of_a_waves_lanes(B, fmt):
    import paper_2501_06807_amd as M
    T, first = 96, [0, 3, 50, B]
    lens = [T + 1 + (5 * b) % 23 for b in range(B)]
    kv = behind(M, fmt, "bf16", lens, first, [T] * 3, Hkv=1)
    q = tokens((1, B, 4, 1, 64), "bf16", 9).cuda()
    f, r, n_valid = ints(first), ints([T] * 3), ints([1] * B)
    ws = M.workspace(M.shared_attn_workspace_bytes(q, kv, 3))
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:4], device="cuda")

    def step():
        M.mpc_shared_attn(q, kv, out, first=f, shared_rows=r, sm_scale=0.125, n_valid=n_valid, lse=lse, ws=ws)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for new, first, lens in (([1] * B, first, lens), ([1, 0] * (B // 2) + [1] * (B % 2), [0, 1, 33, 60], lens), ([1] * B, [0, B, B, B], [x - 1 for x in lens])):
        for b in range(B):
            leader = max(a for a in first if a <= b) if b < first[-1] else b
            if leader < B:
                kv.table[b, :6] = kv.table[leader, :6] if int(kv.table[leader, 0]) < 2 ** 30 else kv.table[0, :6]
        n_valid.copy_(torch.tensor(new))
        f.copy_(torch.tensor(first))
        kv.lens.copy_(torch.tensor(lens))
        out.fill_(7)
        lse.fill_(7)
        g.replay()
        torch.cuda.synchronize()
        got = (out.clone(), lse.clone())
        check(kv, q, *got, lens, first, [T] * 3, new, units=[(0, b, 0) for b in (0, 1, 2, 3, 49, 50, B - 1)])
        out.fill_(7)
        step()
        torch.cuda.synchronize()
        assert torch.equal(bits(out), bits(got[0]))


@pytest.mark.parametrize("fmt", ["mx4", "e4m3"])
def test_pools_beyond_32_bits_of_bytes(fmt):
    """Pages in the last megabytes of pools of 4.5 GiB: append, read, both attentions."""
    import paper_2501_06807_amd as M
    d, page, B = 128, 256, 3
    row = d // 2 if fmt == "mx4" else d
    P = (9 << 29) // (page * row)
    kv = M.paged_kv(n_layers=1, batch=B, n_kv_heads=1, head_dim=d, dtype=torch.bfloat16, n_pages=P, max_pages=5, page_size=page, fmt=fmt)
    small = make4(M, 1, B, 1, d, "bf16", page, cap=5) if fmt == "mx4" else make(M, 1, B, 1, d, "bf16", page, cap=5, fp8=True)
    kv.table.copy_(P - 1 - torch.arange(B * 5).view(B, 5))
    lens, first, shared = [1100, 1030, 1200], [0, 3], [1024]
    k, v = tokens((1, B, 1, 1200, d), "bf16", 1).cuda(), tokens((1, B, 1, 1200, d), "bf16", 2, spread=False).cuda()
    q = tokens((1, B, 8, 4, d), "bf16", 9).cuda()
    res = []
    for c in (kv, small):
        c.lens.copy_(torch.tensor(lens))
        M.mpc_paged_append(k, v, c, n_valid=c.lens.clone())
        c.table[1:, :4] = c.table[0, :4]
        back = [torch.zeros_like(k) for _ in range(2)]
        M.mpc_paged_read(c, *back)
        out = torch.zeros_like(q)
        M.mpc_paged_attn(q, c, out, sm_scale=0.1)
        one = q[:, :, :2, :1].contiguous()
        res.append(back + [out] + list(run(M, c, q, first, shared)) + list(run(M, c, one, first, shared)))
    for x, y in zip(*res):
        assert torch.equal(bits(x), bits(y))
