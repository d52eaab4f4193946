"""The forms that large calls take, which the small tests of the same operators do not reach: prompts of more than 256 blocks of
128 rows, two 16-row tiles to a wave in fp32, and appends whose threads share a position's angles over four heads. Some rows
of each, against the 64-bit forms over the inputs."""
import pytest
import torch

import paged_ref as R
from test_gpu_attn import prompt_case
from test_gpu_paged_append import DT, bits, make, tokens

pytestmark = pytest.mark.gpu


def spots(T):
    return [t for t in (0, 1, 31, 32, 127, 128, 129, 500, 640, 1023, 1024, T - 130, T - 1) if 0 <= t < T]


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp16", 128), ("bf16", 64), ("fp16", 64)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 5), (33, 70)])
def test_prompts_of_many_blocks(dtype, d, window, sinks):
    """32 heads of 1200 rows are 320 blocks: a workgroup of four waves to each, all of its keys."""
    prompt_case(dtype, 1, 1, 32, 8, d, 1200, 1200, None, None, window, sinks, rows=spots(1200))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (200, 3)])
def test_padded_batches_of_many_blocks(dtype, window, sinks):
    """Sequences of other lengths side by side, with NaN and infinities behind their keys; one has more rows than keys."""
    prompt_case(dtype, 2, 4, 8, 2, 128, 700, 900, [700, 1, 333, 690], [900, 900, 333, 257], window, sinks,
                rows=[0, 1, 127, 128, 332, 333, 432, 433, 434, 512, 689, 690, 699], token_major=True)


@pytest.mark.parametrize("d,Hq,Hkv", [(64, 8, 8), (128, 8, 2)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (400, 20)])
def test_prompts_of_two_tiles_to_a_wave_in_fp32(d, Hq, Hkv, window, sinks):
    """2100 rows of 8 heads are more than 16384 rows."""
    prompt_case("fp32", 1, 1, Hq, Hkv, d, 2100, 2100, None, None, window, sinks, rows=spots(2100))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_values_that_a_row_does_not_see_in_many_blocks(dtype):
    """Infinities and NaN in K and V at keys behind the window or ahead of a row: rows that see them carry them, no others."""
    import math

    import paper_2501_06807_amd as M
    T, Hq, d, window, sinks = 1200, 32 if dtype == "bf16" else 16, 64, 50, 3
    q, k, v = (tokens((1, 1, h, T, d), dtype, s, spread=False) for s, h in ((1, Hq), (2, Hq), (3, Hq)))
    at, clean = (40, 700, 707), v.clone()
    for i, j in enumerate(at):
        v[0, 0, ::2, j, ::5] = (math.inf, math.nan, -math.inf)[i]
        k[0, 0, 1::2, j] = math.nan
    out, lse = torch.empty_like(q).cuda(), torch.empty(1, 1, Hq, T, device="cuda")
    M.mpc_prompt_attn(q.cuda(), k.cuda(), v.cuda(), out, sm_scale=d ** -0.5, window=window, sinks=sinks, lse=lse)
    out, lse = out.cpu(), lse.cpu()
    for t in (2, 39, 40, 41, 89, 90, 91, 500, 699, 700, 706, 707, 749, 750, 756, 757, 1199):
        sees = any(j <= t and t - window < j for j in at)
        for h in (0, 1, 6, 7):
            if sees and h % 2:
                assert bool(out[0, 0, h, t].isnan().all()) and math.isnan(float(lse[0, 0, h, t])), (t, h)
                continue
            x, kd, vd = q[0, 0, h, t].double(), k[0, 0, h].double(), clean[0, 0, h].double()
            o, ls, idx, w = R.attend(x, kd, vd, t, d ** -0.5, window, sinks)
            bo, bl = R.bounds(x, kd, vd, idx, w, o, ls, d ** -0.5, DT[dtype])
            part = torch.arange(d) % 5 != 0 if sees else torch.ones(d, dtype=torch.bool)
            R.check(out[0, 0, h, t, part], o[part], bo[part], f"t{t} h{h}")
            R.check(lse[0, 0, h, t], ls, bl, f"lse t{t} h{h}")
            if sees:
                assert not bool(out[0, 0, h, t, ::5].isfinite().any()), (t, h)


# (dtype, 8-bit, page, d, Hq, Hkv, rows, style, rotated channels): 1024 workgroups of four heads to a thread, and more
APPENDS = [
    ("bf16", False, 16, 128, 32, 8, 3000, "half", 128), ("fp16", False, 64, 64, 16, 16, 6200, "interleaved", 64),
    ("fp32", False, 32, 128, 32, 4, 1800, "interleaved", 64), ("bf16", True, 64, 128, 32, 8, 2200, "half", 128),
    ("fp16", True, 32, 128, 32, 8, 2200, "interleaved", 96), ("fp32", True, 16, 64, 32, 4, 2200, "half", 64),
    ("bf16", True, 16, 64, 32, 4, 2300, "interleaved", 64),
]


@pytest.mark.parametrize("dtype,fp8,page,d,Hq,Hkv,n,style,rot", APPENDS)
def test_appended_prompts(dtype, fp8, page, d, Hq, Hkv, n, style, rot):
    """Two sequences of other lengths, the second one beginning in the middle of a page; token-major inputs."""
    import paper_2501_06807_amd as M
    B, lens, new = 2, [n, n - 77], [n, n - 100]
    kv = make(M, 1, B, Hkv, d, dtype, page, cap=-(-n // page), fp8=fp8)
    kv.lens.copy_(torch.tensor([0, 23]))
    first = [tokens((1, B, Hkv, 23, d), dtype, s) for s in (11, 12)]
    tab = R.rope_table(n, rot)
    M.mpc_paged_append(*(x.cuda() for x in first), kv, rope=tab.cuda(), rope_style=style,
                       n_valid=torch.tensor([0, 23], dtype=torch.int32, device="cuda"))
    major = lambda t: t.transpose(2, 3).contiguous().transpose(2, 3)  # noqa: E731
    q, k, v = (major(tokens((1, B, h, n, d), dtype, s)) for s, h in ((1, Hq), (2, Hkv), (3, Hkv)))
    kv.lens.copy_(torch.tensor(lens))
    q_out, k_out = torch.full_like(q, 7.0, device="cuda"), torch.full_like(k, 7.0, device="cuda")
    M.mpc_paged_append(k.cuda(), v.cuda(), kv, q=q.cuda(), q_out=q_out, k_out=k_out, rope=tab.cuda(), rope_style=style,
                       n_valid=torch.tensor(new, dtype=torch.int32, device="cuda"))
    q_out, k_out, table = q_out.cpu(), k_out.cpu(), kv.table.cpu()
    kp, vp = kv.k_pages.cpu(), kv.v_pages.cpu()
    for b in range(B):
        base = lens[b] - new[b]
        for t in (0, 1, 15, 16, 31, 33, 1000, new[b] // 2, new[b] - 33, new[b] - 1, min(new[b], n - 1), n - 1):
            if t >= new[b]:
                assert bool((q_out[0, b, :, t] == 7).all()) and bool((k_out[0, b, :, t] == 7).all())
                continue
            for x, got, what in ((q, q_out, "q"), (k, k_out, "k")):
                want, mag = R.rotated(x[0, b, :, t].double(), tab, style, base + t)
                R.check(got[0, b, :, t], want, R.half_step(DT[dtype]) * want.abs() + 4 * R.U32 * mag + 2.0 ** -25, f"{what} {b} {t}")
            if not fp8:
                at = int(table[b, (base + t) // page]), (base + t) % page
                assert torch.equal(bits(kp[0, at[0], :, at[1]]), bits(k_out[0, b, :, t])), (b, t)
                assert torch.equal(bits(vp[0, at[0], :, at[1]]), bits(v[0, b, :, t])), (b, t)
        if fp8:
            ks, vs = kv.k_scale.cpu(), kv.v_scale.cpu()
            last, full = (lens[b] - 1) // page, lens[b] // page
            for pg in {1, 2, full // 2, full - 1} | ({0} if base == 0 else set()):
                for rows, codes, scale, what in ((k_out, kp, ks, "k"), (v, vp, vs, "v")):
                    id = int(table[b, pg])
                    for h in range(Hkv):
                        lo, hi = pg * page - base, (pg + 1) * page - base
                        x = rows[0, b, h, max(lo, 0):hi].double()
                        if lo < 0:  # its first rows are those of the call before
                            if what == "k":
                                continue
                            x = torch.cat([first[1][0, b, h, pg * page:23].double(), x])
                        want, e = R.encode(x)
                        assert float(scale[0, id, h]) == e and torch.equal(codes[0, id, h].double(), want), (b, what, pg, h)
            for j in range((last - 1) * page, lens[b]):
                at = j % (2 * page)
                assert torch.equal(bits(kv.k_tail[0, b, :, at]), bits(k_out[0, b, :, j - base])), (b, j)
                assert torch.equal(bits(kv.v_tail[0, b, :, at]), bits(v[0, b, :, j - base])), (b, j)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 4)])
def test_chunks_over_a_paged_cache(dtype, fp8, d, window, sinks):
    """48 query rows to a kv head: two units of two 16-row tiles each, their keys divided over workgroups and joined."""
    import paper_2501_06807_amd as M
    from test_gpu_attn import check_paged, fill, run_paged
    lens, new, n = [3000, 12, 701], [12, 12, 5], 12
    kv = make(M, 1, 3, 2, d, dtype, 32, cap=94, fp8=fp8)
    fill(kv, lens, 5, dtype)
    q = tokens((1, 3, 8, n, d), dtype, 3, spread=False).cuda()
    out, lse = run_paged(kv, q, new, window, sinks)
    check_paged(kv, q, out, lse, lens, new, window, sinks, d ** -0.5, f"{dtype} {fp8} {d}")
