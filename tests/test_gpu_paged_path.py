"""PagedPath: prompts, decoded and drafted tokens, rows taken back, a captured step and an evicted cache, each against the 64-bit
forms over what the cache holds."""
import math

import pytest
import torch

import paged_ref as R
import synth
from gpu_util import bits_to_torch
from test_gpu_attn import check_paged, rows_of
from test_gpu_paged_append import DT, bits, tokens

pytestmark = pytest.mark.gpu


def make(dtype="bf16", fp8=True, L=2, B=3, Hq=4, Hkv=2, d=64, page=16, rope=True, **kw):
    import paper_2501_06807_amd as M
    return M.PagedPath(n_layers=L, batch=B, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, dtype=DT[dtype], max_rows=200, page_size=page,
                       fp8=fp8, rope=R.rope_table(256, d).cuda() if rope else None, **kw)


def inputs(path, n, dtype, seed):
    kv = path.kv
    return [tokens((kv.L, kv.B, h, n, kv.d), dtype, seed + s).cuda() for s, h in ((1, path.Hq), (2, kv.Hkv), (3, kv.Hkv))]


@pytest.mark.parametrize("dtype,fp8,window,sinks", [("bf16", True, 0, 0), ("fp16", False, 30, 4), ("fp32", True, 0, 0), ("bf16", True, 25, 2)])
def test_prompts_then_tokens_then_drafts(dtype, fp8, window, sinks):
    path = make(dtype, fp8, window=window, sinks=sinks)
    lens = [70, 1, 33]
    q, k, v = inputs(path, 70, dtype, 0)
    k0 = k.clone()
    lse = torch.full((2, 3, 4, 70), 7.0, device="cuda")
    out = path.prefill(q, k, v, lens, out=torch.full_like(q, 7.0), lse=lse)
    assert torch.equal(k, k0) and path.kv.lens.tolist() == lens and path.pos.tolist() == lens
    sm = path.kv.d ** -0.5
    if not fp8:  # with pages of the element type the cache's rows are the prompt's
        check_paged(path.kv, q, out, lse, lens, lens, window, sinks, sm, "prompt")
    else:
        turned = torch.stack([torch.stack([R.rotated(k0[l, b, :, t].cpu().double(), R.rope_table(256, 64), "interleaved", t)[0]
                                           for t in range(lens[b])], 1).to(DT[dtype]).double() for l in range(2) for b in (0,)])
        for hq in (0, 3):
            for t in (0, 40, 69):
                x = q[1, 0, hq, t].cpu().double()
                o, ls, idx, w = R.attend(x, turned[1, hq // 2], v[1, 0, hq // 2].cpu().double(), t, sm, window, sinks)
                bo, bl = R.bounds(x, turned[1, hq // 2], v[1, 0, hq // 2].cpu().double(), idx, w, o, ls, sm, DT[dtype])
                # the reference's K is rounded once from 64 bits, the cache's after fp32 sums: at most one step of the type
                # in a channel apart, a score by at most that step of sum |q| |k|, weights by twice it
                step = 2 * R.half_step(DT[dtype]) * float((turned[1, hq // 2].abs() @ x.abs()).max()) * sm * 2.0 ** -6
                R.check(out[1, 0, hq, t].cpu(), o, bo + 2 * step * float(v.abs().max()), f"prompt h{hq} t{t}")
    for i, (n, new) in enumerate([(1, None), (1, None), (4, [4, 2, 1]), (1, [1, 0, 1])]):
        q, k, v = inputs(path, n, dtype, 50 + 10 * i)
        lse = torch.full((2, 3, 4, n), 7.0, device="cuda")
        out = path.extend(q, k, v, new, out=torch.full_like(q, 7.0), lse=lse)
        new = [n] * 3 if new is None else new
        lens = [x + y for x, y in zip(lens, new)]
        assert path.kv.lens.tolist() == lens == path.rows
        check_paged(path.kv, q, out, lse, lens, new, window, sinks, sm, f"step {i}")


def test_rejected_drafts_leave_the_cache_as_if_they_had_not_been():
    a, b = make(), make()
    q, k, v = inputs(a, 30, "bf16", 0)
    for p in (a, b):
        p.prefill(q.clone(), k, v)
    dq, dk, dv = inputs(a, 5, "bf16", 10)
    a.extend(dq, dk, dv)
    a.take_back([5, 3, 4])
    b.extend(dq[:, :, :, :2].clone().contiguous(), dk[:, :, :, :2], dv[:, :, :, :2], [0, 2, 1])
    assert a.rows == b.rows and a.kv.lens.tolist() == b.kv.lens.tolist() and a.pos.tolist() == b.pos.tolist()
    for i in range(20):
        x = inputs(a, 1, "bf16", 100 + 10 * i)
        o = [p.extend(x[0].clone(), x[1], x[2]) for p in (a, b)]
        if i > 0:  # (the first of them was rotated in place above by the same step of each)
            assert torch.equal(bits(o[0]), bits(o[1])), i
    with pytest.raises(ValueError):  # the tail holds the last two pages: rows from 32 on
        a.take_back([a.rows[0] - 31, 0, 0])
    a.take_back([a.rows[0] - 33, 0, 0])
    with pytest.raises(ValueError):  # also for a second time
        a.take_back([2, 0, 0])
    a.take_back([1, 0, 0])  # row 32 begins a page: nothing of it is needed
    with pytest.raises(ValueError):
        a.take_back([0, 0, -1])


def test_a_captured_step_follows_the_eager_one():
    import paper_2501_06807_amd as M
    a, b = make(page=16), make(page=16)
    q, k, v = inputs(a, 40, "bf16", 0)
    for p in (a, b):
        p.prefill(q.clone(), k, v)
        p.reserve([80] * 3)
    q, k, v = inputs(a, 1, "bf16", 5)
    out = torch.zeros_like(q)
    a.step(q.clone(), k, v)  # (its workspace exists before the capture)
    a.kv.lens.sub_(1)
    a.pos.sub_(1)
    g = M.MPCachePath.capture(a, a.step, q, k, v, None, out)
    for i in range(25):
        x = inputs(a, 1, "bf16", 100 + 10 * i)
        for dst, src in zip((q, k, v), x):
            dst.copy_(src)
        a.grown([1] * 3)
        g.replay()
        want = b.extend(x[0].clone(), x[1], x[2])
        torch.cuda.synchronize()
        assert torch.equal(bits(out), bits(want)), i
    assert a.kv.lens.tolist() == b.kv.lens.tolist() == a.rows


def test_an_evicted_cache_goes_on_in_pages():
    """Static eviction keeps 256 of 512 tokens; the kept rows, different ones for each head, become a paged cache, and decoding
    goes on from position 512."""
    import paper_2501_06807_amd as M
    w = synth.get("C1")
    qw, k, v = (bits_to_torch(x[None], w.dtype) for x in synth.prefill_host(w, 0))
    path = M.MPCachePath(n_layers=1, batch=1, n_q_heads=w.n_q_heads, n_kv_heads=w.n_kv_heads, head_dim=w.head_dim,
                         dtype=torch.float32, T=w.T, window=w.window, keep=w.keep, local_keep=w.local_keep, cluster=w.cluster,
                         fanout=w.fanout, k_super=w.k_super, k_clusters=w.k_clusters, share_period=1)
    path.prefill(qw, k, v)
    for fp8 in (False, True):
        d = w.head_dim
        paged = M.PagedPath(n_layers=1, batch=1, n_q_heads=w.n_q_heads, n_kv_heads=w.n_kv_heads, head_dim=d, dtype=torch.float32,
                            max_rows=w.keep + 40, page_size=32, fp8=fp8, rope=R.rope_table(600, d).cuda())
        paged.adopt(path, position=w.T)
        rows = rows_of(paged.kv, 0, 0, 3, w.keep)
        if not fp8:
            assert torch.equal(rows[0], path.k_s[0, 0, 3].cpu().double()) and torch.equal(rows[1], path.v_s[0, 0, 3].cpu().double())
        for i in range(3):
            q, kn, vn = (tokens((1, 1, w.n_kv_heads, 1, d), "fp32", 10 * i + s).cuda() for s in (1, 2, 3))
            k_before = kn.clone()
            lse = torch.empty(1, 1, w.n_q_heads, 1, device="cuda")
            out = paged.extend(q, kn, vn, lse=lse)
            assert torch.equal(kn, k_before)
            n = w.keep + i + 1
            got = rows_of(paged.kv, 0, 0, 2, n)[0][-1]
            want, mag = R.rotated(kn[0, 0, 2, 0].cpu().double(), R.rope_table(600, d), "interleaved", w.T + i)
            R.check(got, want, R.half_step(torch.float32) * want.abs() + 4 * R.U32 * mag, "position of the new token")
            check_paged(paged.kv, q, out, lse, [n], [1], 0, 0, 1 / math.sqrt(d), f"fp8 {fp8} token {i}")


def test_pages_run_out_and_lengths_end_with_an_error():
    import paper_2501_06807_amd as M
    path = M.PagedPath(n_layers=1, batch=2, n_q_heads=2, n_kv_heads=2, head_dim=64, dtype=torch.bfloat16, max_rows=64, page_size=16,
                       n_pages=5, rope=None)
    q = torch.zeros(1, 2, 2, 40, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="pages wanted"):
        path.prefill(q, q, q)
    path.prefill(q, q, q, [40, 20])
    x = q[:, :, :, :1].contiguous()
    with pytest.raises(ValueError, match="more than 64 rows"):
        path.grown([25, 0])
    assert path.rows == [40, 20]
    path.extend(x, x, x)
    path.clear()
    path.prefill(q, q, q, [16, 40])
    assert path.rows == [16, 40] and sorted(path._free + path._pages[0] + path._pages[1]) == list(range(5))
