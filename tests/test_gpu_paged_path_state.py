"""PagedPath: a call that is refused leaves the path as it was, on the host and on the device; rows taken back far."""
import math

import pytest
import torch

from test_gpu_paged_append import bits, tokens
from test_gpu_paged_path import inputs, make

pytestmark = pytest.mark.gpu


def snapshot(path):
    kv = path.kv
    return (list(path.rows), list(path._kept), [list(p) for p in path._pages], list(path._free), kv.table.tolist(),
            kv.lens.tolist(), path.pos.tolist(), bits(kv.k_pages), bits(kv.v_pages),
            *(bits(t) for t in (kv.k_tail, kv.v_tail, kv.k_scale, kv.v_scale) if t is not None))


def same(a, b):
    return all(torch.equal(x, y) if torch.is_tensor(x) else x == y for x, y in zip(a, b))


def refused(path, call, *args, **kw):
    before = snapshot(path)
    ins = [x.clone() for x in args if torch.is_tensor(x)]
    with pytest.raises((ValueError, TypeError)):
        call(*args, **kw)
    torch.cuda.synchronize()
    assert same(before, snapshot(path))
    assert all(torch.equal(bits(x), bits(y)) for x, y in zip(ins, (x for x in args if torch.is_tensor(x))))


@pytest.mark.parametrize("fp8", [True, False])
def test_refused_calls_change_nothing(fp8):
    path = make(fp8=fp8)
    q, k, v = inputs(path, 40, "bf16", 0)
    path.prefill(q, k, v, [40, 7, 20])
    q, k, v = inputs(path, 2, "bf16", 10)
    no = lambda *a, **kw: refused(path, path.extend, *a, **kw)  # noqa: E731
    # counts: more than there are, fewer than none, too few, too many, not whole
    for new in ([3, 0, 0], [2, -1, 1], [2, 2], [2, 2, 2, 2], [1.5, 1, 1]):
        no(q, k, v, new)
    # tensors: types, heads, tokens, sequences, channels, channels apart, off their alignment, on the host
    no(q.half(), k, v)
    no(q, k.float(), v)
    no(q, k, v.half())
    no(q[:, :, :3].contiguous(), k, v)
    no(q, k[:, :, :1], v)
    no(q, k[:, :, :, :1], v)
    no(q, k, v[:, :2])
    no(q[:1], k[:1], v[:1])
    no(q[..., :32].contiguous(), k, v)
    no(q, k.transpose(3, 4).contiguous().transpose(3, 4), v)
    no(q, torch.zeros(k.numel() + 1, dtype=k.dtype, device="cuda")[1:].view(k.shape), v)
    no(q, k, v.cpu())
    no(q, torch.zeros(*k.shape[:4], 66, dtype=k.dtype, device="cuda")[..., :64], v)  # rows 132 bytes apart
    no(q[:, :, :, :1].expand(-1, -1, -1, 2, -1), k, v)  # q becomes rotated in place: its rows may not lie on each other
    # results
    no(q, k, v, out=torch.zeros_like(q).half())
    no(q, k, v, out=torch.zeros_like(q)[:, :, :2])
    no(q, k, v, out=torch.zeros_like(q)[:, :, :1].expand(-1, -1, 4, -1, -1))
    no(q, k, v, lse=torch.zeros(2, 3, 4, 1, device="cuda"))
    no(q, k, v, lse=torch.zeros(2, 3, 4, 2, device="cuda", dtype=torch.float64))
    no(q, k, v, lse=torch.zeros(2, 3, 4, 2))
    # the device's part by itself
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    step = lambda *a, **kw: refused(path, path.step, *a, **kw)  # noqa: E731
    step(q, k, v, ints(1))
    step(q, k, v, ints(1, 1, 1).long())
    step(q, k, v, ints(1, 1, 1).cpu())
    step(q, k.half(), v)
    # longer than the table, more pages than there are, and the other ways to book
    refused(path, path.extend, *inputs(path, 200, "bf16", 20))
    for new in ([1, 1], [1, 1, -1], [500, 0, 0]):
        refused(path, path.grown, new)
    for rows in ([50, 50], [50, 50, 500], [50, -1, 50]):
        refused(path, path.reserve, rows)
    for back in ([1, 1], [8, 8, 8], [0, -1, 0], [1, 1, 1, 1]):
        refused(path, path.take_back, back)
    # a prompt that is refused leaves the sequences that are there
    no = lambda *a, **kw: refused(path, path.prefill, *a, **kw)  # noqa: E731
    q, k, v = inputs(path, 30, "bf16", 30)
    for lens in ([31, 1, 1], [30, -1, 3], [30, 30]):
        no(q, k, v, lens)
    no(q.half(), k, v)
    no(q, k, v[:, :, :, :29])
    no(q, k, v, out=torch.zeros_like(q)[:, :, :1].expand(-1, -1, 4, -1, -1))
    no(q, k, v, lse=torch.zeros(2, 3, 4, 29, device="cuda"))
    no(*inputs(path, 209, "bf16", 40))  # (13 pages of 16 rows are 208)
    # and the path goes on as one that was not asked for any of it
    twin = make(fp8=fp8)
    a, b, c = inputs(path, 40, "bf16", 0)
    twin.prefill(a, b, c, [40, 7, 20])
    for i in range(3):
        x = inputs(path, 2, "bf16", 50 + 10 * i)
        got, want = (p.extend(x[0].clone(), x[1], x[2], [2, 1, 0]) for p in (path, twin))
        assert torch.equal(bits(got), bits(want)), i


def test_a_prompt_that_the_pool_has_no_pages_for_leaves_the_sequences():
    import paper_2501_06807_amd as M
    path = M.PagedPath(n_layers=1, batch=2, n_q_heads=2, n_kv_heads=2, head_dim=64, dtype=torch.bfloat16, max_rows=64, page_size=16,
                       n_pages=5, rope=None)
    q = tokens((1, 2, 2, 40, 64), "bf16", 1).cuda()
    path.prefill(q, q, q, [30, 20])
    refused(path, path.prefill, q, q, q)
    path.prefill(q, q, q, [16, 40])  # four pages: those of the sequences before are free for it
    assert path.rows == [16, 40]


@pytest.mark.parametrize("kw", [dict(window=-1), dict(sinks=-2), dict(window=2 ** 32 + 5), dict(sm_scale=math.nan), dict(rope_style="whole"),
                                dict(Hq=3), dict(Hq=32), dict(d=96), dict(page=48)])
def test_a_path_that_could_not_run_is_not_made(kw):
    """Refused when it is made, not by its first call, which would have booked its rows by then."""
    with pytest.raises((ValueError, RuntimeError)):
        make(**kw)


@pytest.mark.parametrize("rope", ["long", "half", "flat", "host", "odd"])
def test_a_rotary_table_that_does_not_fit_is_refused_at_once(rope):
    import paper_2501_06807_amd as M
    t = torch.zeros(10, 32, 2, device="cuda")
    t = {"long": torch.zeros(10, 40, 2, device="cuda"), "half": t.half(), "flat": t.view(10, 64), "host": t.cpu(),
         "odd": torch.zeros(10, 4, 2, device="cuda")}[rope]
    with pytest.raises(ValueError):
        M.PagedPath(n_layers=1, batch=1, n_q_heads=2, n_kv_heads=2, head_dim=64, dtype=torch.bfloat16, max_rows=64, rope=t)


def test_an_evicted_cache_of_another_shape_is_refused():
    import paper_2501_06807_amd as M
    path = make("fp32")
    q, k, v = inputs(path, 20, "fp32", 0)
    path.prefill(q, k, v)
    kw = dict(n_layers=2, batch=3, n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=torch.float32, T=64, window=8, keep=32, local_keep=8,
              cluster=16, fanout=2, k_super=1, k_clusters=1, share_period=1)
    for other in (dict(batch=2), dict(n_layers=1), dict(n_kv_heads=1), dict(head_dim=128), dict(dtype=torch.float16),
                  dict(T=512, keep=256)):
        refused(path, path.adopt, M.MPCachePath(**dict(kw, **other)), 64)
    refused(path, path.adopt, M.MPCachePath(**kw), -1)


def test_rows_taken_back_to_a_page_far_behind():
    """From row 161 to row 32, where a page begins, and on from there: drafts are taken back again as on a path that never
    went further, and the other sequences' too."""
    a, b = make(page=16), make(page=16)
    q, k, v = inputs(a, 161, "bf16", 0)
    a.prefill(q.clone(), k, v, [161, 30, 161])
    a.take_back([161 - 32, 0, 161 - 32])
    b.prefill(q[:, :, :, :32].contiguous(), k[:, :, :, :32], v[:, :, :, :32], [32, 30, 32])
    for i, (new, back) in enumerate([([5, 5, 1], [2, 1, 0]), ([4, 0, 5], [0, 2, 3]), ([5, 5, 5], [5, 1, 0]), ([5, 5, 5], [0, 5, 5]),
                                     ([5, 3, 5], [1, 3, 5])]):
        x = inputs(a, 5, "bf16", 10 + 10 * i)
        got, want = (p.extend(x[0].clone(), x[1], x[2], new) for p in (a, b))
        assert torch.equal(bits(got), bits(want)), i
        for p in (a, b):
            p.take_back(back)
        assert a.rows == b.rows and a.kv.lens.tolist() == b.kv.lens.tolist() == a.rows
    for p in (a, b):
        with pytest.raises(ValueError):  # row 20 lies in a page that neither tail holds now
            p.take_back([p.rows[0] - 20, 0, 0])
