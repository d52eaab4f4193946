"""mpc_paged_append against its definition in 64 bits: rotated rows, pages, codes, scales and rings, however the tokens are
cut into calls, and what has to stay as it was."""
import pytest
import torch

import paged_ref as R
from gpu_util import say

pytestmark = pytest.mark.gpu

DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


def make(M, L=1, B=2, Hkv=2, d=64, dtype="bf16", page=16, cap=8, fp8=True, seed=0, spare=3):
    g = torch.Generator().manual_seed(seed)
    kv = M.paged_kv(n_layers=L, batch=B, n_kv_heads=Hkv, head_dim=d, dtype=DT[dtype], n_pages=B * cap + spare, max_pages=cap,
                    page_size=page, fp8=fp8)
    kv.table.copy_(torch.randperm(B * cap + spare, generator=g)[: B * cap].int().view(B, cap))
    for t in (kv.k_pages, kv.v_pages):  # nothing that is not written may be read
        t.view(torch.uint8).fill_(0x7F if fp8 else 0xFF)
    if fp8:
        for t in (kv.k_tail, kv.v_tail, kv.k_scale, kv.v_scale):
            t.fill_(float("nan"))
    return kv


def tokens(shape, dtype, seed, spread=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g)
    if spread:
        x[..., :4] *= 8
    return x.to(DT[dtype])


def bits(t):
    return t.contiguous().view(torch.uint8).cpu()


def state(kv):
    names = ["k_pages", "v_pages"] + (["k_scale", "v_scale", "k_tail", "v_tail"] if kv.k_scale is not None else [])
    return {n: bits(getattr(kv, n)) for n in names}


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("style,d,rot", [("half", 64, 64), ("interleaved", 128, 128), ("half", 128, 32), ("interleaved", 64, 16)])
def test_rows_and_queries_are_the_rotated_ones(dtype, style, d, rot):
    import paper_2501_06807_amd as M
    L, B, Hq, Hkv, n, page = 2, 3, 4, 2, 21, 16
    kv = make(M, L, B, Hkv, d, dtype, page, cap=4, fp8=False)
    before = state(kv)
    new, lens = [21, 0, 13], [21, 5, 30]
    kv.lens.copy_(torch.tensor(lens))
    q, k, v = (tokens((L, B, h, n, d), dtype, s) for s, h in ((1, Hq), (2, Hkv), (3, Hkv)))
    tab = R.rope_table(64, rot)
    q_out = torch.full((L, B, Hq, n, d), 7.0, dtype=DT[dtype], device="cuda")
    M.mpc_paged_append(k.cuda(), v.cuda(), kv, q=q.cuda(), q_out=q_out, rope=tab.cuda(), rope_style=style,
                       n_valid=torch.tensor(new, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    kp, vp, table = kv.k_pages.cpu(), kv.v_pages.cpu(), kv.table.cpu()
    written = torch.zeros(kp.shape[:4], dtype=torch.bool)
    for b in range(B):
        for t in range(n):
            if t >= new[b]:
                assert bool((q_out[:, b, :, t] == 7.0).all())
                continue
            j = lens[b] - new[b] + t
            pg, r = int(table[b, j // page]), j % page
            written[:, pg, :, r] = True
            for x, got, what in ((q, q_out.cpu()[:, b, :, t], "q"), (k, kp[:, pg, :, r], "k")):
                want, mag = R.rotated(x[:, b, :, t].double(), tab, style, j)
                R.check(got, want, R.half_step(DT[dtype]) * want.abs() + 4 * R.U32 * mag + 2.0 ** -25, f"{what} {b} {t}")
            assert torch.equal(bits(vp[:, pg, :, r]), bits(v[:, b, :, t]))
    for name in ("k_pages", "v_pages"):
        was = before[name].view(getattr(kv, name).dtype).view(kp.shape)[~written]
        assert torch.equal(bits(getattr(kv, name).cpu()[~written]), bits(was)), "rows outside the call changed"


def plain_rows(M, kv, k, v, rope, style, start, pos0):
    """K rows as a 16- or 32-bit cache holds them (their own test is above): [L][B][Hkv][n][d]."""
    L, B, H, n, d = k.shape
    page = 16
    cap = -(-n // page)
    flat = M.paged_kv(n_layers=L, batch=B, n_kv_heads=H, head_dim=d, dtype=k.dtype, n_pages=B * cap, max_pages=cap, page_size=page)
    flat.table.copy_(torch.arange(B * cap).int().view(B, cap))
    flat.lens.fill_(n)
    M.mpc_paged_append(k.cuda(), v.cuda(), flat, rope=rope, rope_style=style, pos0=pos0)
    rows = lambda t: t.cpu().view(L, B, cap, H, page, d).transpose(2, 3).reshape(L, B, H, cap * page, d)[:, :, :, :n]  # noqa: E731
    return rows(flat.k_pages), rows(flat.v_pages)


@pytest.mark.parametrize("dtype,page,d", [("bf16", 16, 64), ("fp16", 32, 128), ("fp32", 64, 64), ("bf16", 256, 128),
                                          ("fp32", 16, 128), ("bf16", 128, 64)])
@pytest.mark.parametrize("extra", [0, 1, -1, 7])
def test_codes_scales_and_ring(dtype, page, d, extra):
    import paper_2501_06807_amd as M
    L, B, H = 2, 2, 2
    n = 3 * page + extra
    kv = make(M, L, B, H, d, dtype, page, cap=5)
    k, v = tokens((L, B, H, n, d), dtype, 5), tokens((L, B, H, n, d), dtype, 6)
    v[:, 0, 0, :page] = 0  # a page of zeros: scale 1
    v[:, 1, 1, :page] *= 2.0 ** -12
    v[0, 0, 1, 3, 5] = float("nan")
    v[0, 0, 1, 4, 6] = float("-inf")
    kv.lens.fill_(n)
    rope = R.rope_table(n, d).cuda()
    M.mpc_paged_append(k.cuda(), v.cuda(), kv, rope=rope, rope_style="half")
    kr, vr = plain_rows(M, kv, k, v, rope, "half", 0, None)
    table = kv.table.cpu()
    last = (n - 1) // page
    for rows, codes, scale, ring, what in ((kr, kv.k_pages, kv.k_scale, kv.k_tail, "k"), (vr, kv.v_pages, kv.v_scale, kv.v_tail, "v")):
        codes, scale, ring = codes.cpu(), scale.cpu(), ring.cpu()
        for l in range(L):
            for b in range(B):
                for h in range(H):
                    for pg in range(n // page):
                        want, e = R.encode(rows[l, b, h, pg * page:(pg + 1) * page].double())
                        at = (l, int(table[b, pg]), h)
                        assert float(scale[at]) == e, (what, l, b, h, pg)
                        got = codes[at].double()
                        assert torch.equal(got.isnan(), want.isnan())
                        assert torch.equal(got[~want.isnan()], want[~want.isnan()]), (what, l, b, h, pg)
                    for j in range((max(last - 1, 0)) * page, n):
                        assert torch.equal(bits(ring[l, b, h, j % (2 * page)]), bits(rows[l, b, h, j])), (what, l, b, h, j)
    for l in range(L):  # a page that is not complete is not written
        for b in range(B):
            if n % page:
                assert bool((kv.k_pages[l, int(table[b, last])].view(torch.uint8) == 0x7F).all())


@pytest.mark.parametrize("dtype,page", [("bf16", 16), ("fp32", 32)])
@pytest.mark.parametrize("cuts", [[1] * 100, [37, 5, 58], [16, 16, 32, 36], [3, 1, 70, 26], [10, 40, 40, 10], [99, 1]])
def test_any_division_into_calls_gives_the_same_cache(dtype, page, cuts):
    import paper_2501_06807_amd as M
    L, B, H, d, n = 1, 2, 2, 64, 100
    rope = R.rope_table(200, d).cuda()
    pos0 = torch.tensor([0, 50], dtype=torch.int32, device="cuda")
    k, v, q = (tokens((L, B, h, n, d), dtype, s).cuda() for s, h in ((1, H), (2, H), (3, 2 * H)))
    one = make(M, L, B, H, d, dtype, page, cap=8)
    one.lens.fill_(n)
    q1 = torch.empty_like(q)
    M.mpc_paged_append(k, v, one, q=q, q_out=q1, rope=rope, pos0=pos0)
    many = make(M, L, B, H, d, dtype, page, cap=8)
    at, q2 = 0, torch.empty_like(q)
    for m in cuts:
        many.lens.fill_(at + m)
        part = q[:, :, :, at:at + m].contiguous()
        M.mpc_paged_append(k[:, :, :, at:at + m], v[:, :, :, at:at + m], many, q=part, rope=rope, pos0=pos0 + at)
        q2[:, :, :, at:at + m] = part  # rotated in place
        at += m
    torch.cuda.synchronize()
    a, b = state(one), state(many)
    ring = lambda s, name: s[name].view(one.k_tail.dtype).view(one.k_tail.shape)[:, :, :, torch.arange(((n - 1) // page - 1) * page, n) % (2 * page)]  # noqa: E731
    for name in a:
        x, y = (ring(s, name) if "tail" in name else s[name] for s in (a, b))
        assert torch.equal(bits(x), bits(y)), name
    assert torch.equal(bits(q1), bits(q2))


def test_rows_taken_back_and_appended_again():
    """Lowering a length by up to a page and appending other tokens gives the cache of those tokens."""
    import paper_2501_06807_amd as M
    L, B, H, d, page, n = 1, 2, 1, 64, 16, 50
    k, v = tokens((L, B, H, n, d), "bf16", 1).cuda(), tokens((L, B, H, n, d), "bf16", 2).cuda()
    k2, v2 = tokens((L, B, H, n, d), "bf16", 3).cuda(), tokens((L, B, H, n, d), "bf16", 4).cuda()
    for back in (1, 2, 7, 16):
        got, want = (make(M, L, B, H, d, "bf16", page, cap=5) for _ in range(2))
        got.lens.fill_(n)
        M.mpc_paged_append(k, v, got)
        keep = n - back
        new = torch.cat([k[:, :, :, :keep], k2[:, :, :, :back + 3]], 3), torch.cat([v[:, :, :, :keep], v2[:, :, :, :back + 3]], 3)
        got.lens.fill_(n + 3)
        M.mpc_paged_append(k2[:, :, :, :back + 3], v2[:, :, :, :back + 3], got)
        want.lens.fill_(n + 3)
        M.mpc_paged_append(*new, want)
        for name in ("k_pages", "v_pages", "k_scale", "v_scale"):
            for pg in range((n + 3) // page):
                ids = want.table[:, pg].long()
                assert torch.equal(bits(getattr(got, name)[:, ids]), bits(getattr(want, name)[:, ids])), (back, name, pg)


def test_pages_lengths_and_positions_out_of_range_write_nothing():
    import paper_2501_06807_amd as M
    L, B, H, d, page = 1, 5, 2, 64, 16
    for fp8 in (False, True):
        kv = make(M, L, B, H, d, "bf16", page, cap=2, fp8=fp8)
        kv.table[0, 0], kv.table[1, 0], kv.table[1, 1] = -1, kv.k_pages.shape[1], 2 ** 31 - 1
        # rows 0..19 into no page and a good one; into none; ending behind the table; starting before row 0; no length
        kv.lens.copy_(torch.tensor([20, 20, 40, 6, -3]))
        before = state(kv)
        n = 20
        k, v = tokens((L, B, H, n, d), "bf16", 1).cuda(), tokens((L, B, H, n, d), "bf16", 2).cuda()
        valid = torch.tensor([20, 99, 20, 10, -5], dtype=torch.int32, device="cuda")
        rope = R.rope_table(10, d).cuda()  # positions from 10 on are outside
        M.mpc_paged_append(k, v, kv, rope=rope, n_valid=valid)
        torch.cuda.synchronize()
        good = torch.zeros(kv.k_pages.shape[:4], dtype=torch.bool)
        if not fp8:
            good[:, int(kv.table[0, 1]), :, :4] = True
            good[:, int(kv.table[2, 1])] = True  # rows 20 .. 31 of a capacity of 32
            good[:, int(kv.table[2, 1]), :, :4] = False
            good[:, int(kv.table[3, 0]), :, :6] = True
        else:
            good[:, int(kv.table[2, 1])] = True
        for name in ("k_pages", "v_pages"):
            t = getattr(kv, name)
            was = before[name].view(t.dtype).view(t.shape)
            assert torch.equal(bits(t.cpu()[~good]), bits(was[~good])), name
        if not fp8:
            got = kv.k_pages.cpu().double()
            assert bool(got[0, int(kv.table[3, 0]), :, :6].isfinite().all())
            assert bool(got[0, int(kv.table[0, 1]), :, :4].isnan().all())  # positions 16 .. 19
            assert torch.equal(bits(kv.v_pages[0, int(kv.table[3, 0]), :, :6]), bits(v[0, 3, :, 4:10]))


def test_token_major_inputs_and_another_stream():
    import paper_2501_06807_amd as M
    L, B, Hq, H, d, n = 1, 2, 8, 2, 128, 33
    rope = R.rope_table(64, d).cuda()
    qkv = tokens((B, n, (Hq + 2 * H) * d), "bf16", 1).cuda()
    heads = qkv.view(1, B, n, Hq + 2 * H, d).permute(0, 1, 3, 2, 4)  # one projection's rows, as [L][B][H][n][d] views
    q, k, v = heads[:, :, :Hq], heads[:, :, Hq:Hq + H], heads[:, :, Hq + H:]
    want = make(M, L, B, H, d, "bf16", 32, cap=3)
    want.lens.fill_(n)
    q1 = torch.empty_like(q.contiguous())
    M.mpc_paged_append(k.contiguous(), v.contiguous(), want, q=q.contiguous(), q_out=q1, rope=rope)
    got = make(M, L, B, H, d, "bf16", 32, cap=3)
    got.lens.fill_(n)
    q2 = torch.empty(B, n, Hq, d, dtype=torch.bfloat16, device="cuda").permute(0, 2, 1, 3)[None]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    M.mpc_paged_append(k, v, got, q=q, q_out=q2, rope=rope, stream=side)
    side.synchronize()
    assert torch.equal(bits(q1), bits(q2))
    a, b = state(want), state(got)
    for name in ("k_pages", "v_pages", "k_scale", "v_scale"):
        assert torch.equal(a[name], b[name]), name


def test_pool_beyond_four_gib():
    """Page ids whose byte and element offsets need more than 32 bits."""
    import paper_2501_06807_amd as M
    H, page, d = 8, 64, 128
    P = (1 << 32) // (H * page * d) + 5
    say(f"[paged] pool of {P} pages, {P * H * page * d / 2**30:.2f} GiB for K")
    kv = M.PagedKV(*(torch.empty(1, P, H, page, d, dtype=R.E4M3, device="cuda") for _ in range(2)),
                   torch.tensor([[P - 1, 3, P - 2]], dtype=torch.int32, device="cuda"),
                   torch.tensor([130], dtype=torch.int32, device="cuda"),
                   k_scale=torch.zeros(1, P, H, device="cuda"), v_scale=torch.zeros(1, P, H, device="cuda"),
                   k_tail=torch.zeros(1, 1, H, 2 * page, d, dtype=torch.bfloat16, device="cuda"),
                   v_tail=torch.zeros(1, 1, H, 2 * page, d, dtype=torch.bfloat16, device="cuda"))
    k, v = tokens((1, 1, H, 130, d), "bf16", 1), tokens((1, 1, H, 130, d), "bf16", 2)
    M.mpc_paged_append(k.cuda(), v.cuda(), kv)
    for x, codes, scale in ((k, kv.k_pages, kv.k_scale), (v, kv.v_pages, kv.v_scale)):
        for pg, id in ((0, P - 1), (1, 3)):
            for h in (0, H - 1):
                want, e = R.encode(x[0, 0, h, pg * page:(pg + 1) * page].double())
                assert float(scale[0, id, h]) == e and torch.equal(codes[0, id, h].cpu().double(), want)
    out = torch.empty(1, 1, H, d, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(1, 1, H, 1, device="cuda")
    q = tokens((1, 1, H, d), "bf16", 3)
    M.mpc_paged_attn(q.cuda(), kv, out, sm_scale=d ** -0.5, lse=lse)
    for h in (0, H - 1):
        rows = []
        for x, codes, scale, ring in ((k, kv.k_pages, kv.k_scale, kv.k_tail), (v, kv.v_pages, kv.v_scale, kv.v_tail)):
            rows.append(torch.cat([codes[0, P - 1, h].cpu().double() * float(scale[0, P - 1, h]),
                                   codes[0, 3, h].cpu().double() * float(scale[0, 3, h]), x[0, 0, h, 128:].double()]))
        o, ls, idx, w = R.attend(q[0, 0, h].double(), *rows, 129, d ** -0.5, 0, 0)
        bo, bl = R.bounds(q[0, 0, h].double(), *rows, idx, w, o, ls, d ** -0.5, torch.bfloat16)
        R.check(out[0, 0, h].cpu(), o, bo, f"out {h}")
        R.check(lse[0, 0, h, 0].cpu(), ls, bl, f"lse {h}")


@pytest.mark.parametrize("dtype,fp8,page", [("bf16", False, 16), ("bf16", True, 32), ("fp32", True, 16), ("fp16", True, 256)])
def test_rotated_keys_are_returned_too(dtype, fp8, page):
    """k_out holds K's rows as the cache takes them, of every token that becomes a row, and nothing else."""
    import paper_2501_06807_amd as M
    L, B, H, d, n = 2, 3, 2, 64, 75
    kv = make(M, L, B, H, d, dtype, page, cap=-(-60 // page), fp8=fp8)
    cap = kv.table.shape[1] * page
    lens, new = [min(75, cap), 3, cap + 5], [75, 2, 10]  # ten rows, five of them behind the table's end
    kv.lens.copy_(torch.tensor(lens))
    k, v = tokens((L, B, H, n, d), dtype, 1).cuda(), tokens((L, B, H, n, d), dtype, 2).cuda()
    k_out = torch.full((B, n, L, H, d), 7.0, dtype=DT[dtype], device="cuda").permute(2, 0, 3, 1, 4)
    rope = R.rope_table(400, d)
    M.mpc_paged_append(k, v, kv, k_out=k_out, rope=rope.cuda(), rope_style="half",
                       n_valid=torch.tensor(new, dtype=torch.int32, device="cuda"))
    got = k_out.cpu()
    for b in range(B):
        for t in range(n):
            j = lens[b] - new[b] + t
            if t >= new[b] or not 0 <= j < cap:
                assert bool((got[:, b, :, t] == 7.0).all()), (b, t)
                continue
            want, mag = R.rotated(k[:, b, :, t].cpu().double(), rope, "half", j)
            R.check(got[:, b, :, t], want, R.half_step(DT[dtype]) * want.abs() + 4 * R.U32 * mag + 2.0 ** -25, f"{b} {t}")
