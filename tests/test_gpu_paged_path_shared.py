"""PagedPath over pages of every format with sequences that go on from one prompt: fork() against a path whose sequences have the prompt
each, captured steps, rows taken back, pages given back, and 4-bit pages in the path's other calls."""
import pytest
import torch

import paged_ref as R
from test_gpu_mx4_attn import check4
from test_gpu_paged_append import DT, bits
from test_gpu_paged_path import inputs

pytestmark = pytest.mark.gpu

FORMATS = ["same", "e4m3", "mx4"]


def make(fmt, dtype="bf16", B=5, L=2, Hq=4, Hkv=2, d=64, page=16, rows=200, **kw):
    import paper_2501_06807_amd as M
    return M.PagedPath(n_layers=L, batch=B, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, dtype=DT[dtype], max_rows=rows, page_size=page,
                       fmt=fmt, rope=R.rope_table(256, d).cuda(), **kw)


def alone(x, b):
    """The prompt of sequence b in every sequence's place."""
    return x[:, b:b + 1].expand_as(x).contiguous()


def close(a, b, dtype):
    """Two results that are each within their bounds of the exact one: weights rounded to the type at most, outputs rounded once."""
    tol = 4 * R.half_step(DT[dtype]) if dtype != "fp32" else 2e-5
    return float((a.float() - b.float()).norm() / b.float().norm()) < tol


def start(path, T, first, seed=0, dtype="bf16"):
    """A prompt of T tokens in the first sequence of each group, then the fork."""
    q, k, v = inputs(path, T, dtype, seed)
    lens = [0] * path.kv.B
    for a in first[:-1]:
        lens[a] = T
    path.prefill(q.clone(), k, v, lens)
    path.fork(first, n_new=4)
    return q, k, v


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("T", [64, 71, 9])
def test_forked_sequences_go_on_as_if_each_had_the_prompt(fmt, dtype, T):
    first = [0, 3, 5]
    a, b = make(fmt, dtype), make(fmt, dtype)
    q, k, v = start(a, T, first, dtype=dtype)
    for x in (q, k, v):  # the same prompt in the other path's sequences
        x[:, 1:3], x[:, 4:] = x[:, :1], x[:, 3:4]
    b.prefill(q, k, v)
    assert a.rows == b.rows == [T] * 5 and a.kv.lens.tolist() == [T] * 5 and a.pos.tolist() == [T] * 5
    whole = T // 16
    assert all(a._pages[i][:whole] == a._pages[0][:whole] for i in (1, 2)) and len({p[-1] for p in a._pages}) == (5 if T % 16 else 2)
    for i, (n, new) in enumerate([(1, None), (4, [4, 2, 1, 0, 3]), (1, [1, 1, 1, 1, 0]), (6, None), (30, [30, 1, 17, 0, 30]), (1, None)]):
        x = inputs(a, n, dtype, 50 + 10 * i)
        o = [p.extend(x[0].clone(), x[1], x[2], new) for p in (a, b)]
        assert close(*o, dtype), i
        assert a.rows == b.rows
        for s, t in zip(a.held(100), b.held(100)):
            assert torch.equal(bits(s), bits(t)), i
    a.take_back([2, 0, 1, 0, 0])
    b.take_back([2, 0, 1, 0, 0])
    x = inputs(a, 1, dtype, 200)
    o = [p.extend(x[0].clone(), x[1], x[2]) for p in (a, b)]
    assert close(*o, dtype)


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_captured_step_behind_a_fork_and_behind_the_next_one(fmt):
    """The step's graph follows the tables and lengths; when the path starts again, a graph of an earlier fork shares nothing."""
    a, b = make(fmt), make(fmt)
    start(a, 70, [0, 5])
    q, k, v = inputs(b, 70, "bf16", 0)
    b.prefill(*(alone(x, 0) for x in (q, k, v)))
    x = inputs(a, 1, "bf16", 50)
    src = [t.clone() for t in x]
    out = torch.zeros_like(x[0])
    a.extend(x[0].clone(), x[1], x[2])
    b.extend(x[0].clone(), x[1], x[2])
    a.reserve([200] * 5)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a.step(x[0], x[1], x[2], out=out)

    def replay(i):
        y = inputs(a, 1, "bf16", 60 + 10 * i)
        for s, t in zip(x, y):
            s.copy_(t)
        a.grown([1] * 5)
        g.replay()
        torch.cuda.synchronize()
        want = b.extend(y[0], y[1], y[2])
        assert close(out, want, "bf16"), i
        for s, t in zip(a.held(90), b.held(90)):
            assert torch.equal(bits(s), bits(t)), i

    for i in range(4):
        replay(i)
    assert src[0].shape == x[0].shape
    q, k, v = start(a, 40, [0, 2, 5], seed=7)
    for t in (q, k, v):
        t[:, 1:2], t[:, 3:] = t[:, :1], t[:, 2:3]
    b.prefill(q, k, v)
    a.reserve([200] * 5)
    for i in range(4, 7):
        replay(i)


def test_pages_are_lent_and_given_back():
    a = make("mx4", n_pages=5 * 13)
    assert len(a._free) == 65
    start(a, 70, [0, 4])
    assert len(a._free) == 65 - 5 - 3  # the prompt's, and a copy of the last one for each of the others
    x = inputs(a, 1, "bf16", 50)
    a.extend(x[0], x[1], x[2])
    with pytest.raises(ValueError):  # into the shared rows: 64 of them
        a.take_back([8, 0, 0, 0, 0])
    with pytest.raises(ValueError):
        a.take_back([0, 8, 0, 0, 0])
    a.take_back([7, 7, 1, 0, 1])
    assert a.rows == [64, 64, 70, 71, 0]
    with pytest.raises(ValueError):  # once is enough
        a.fork([0, 4])
    a.clear()
    assert sorted(a._free) == list(range(65))
    q, k, v = inputs(a, 200, "bf16", 3)
    a.prefill(q, k, v)
    assert not a._free


def test_forks_one_after_another_take_no_more_memory():
    """A server forks for every batch: the arrays of the groups and the workspace are the same ones."""
    a, b = make("mx4"), make("mx4")
    seen = set()
    for i, first in enumerate([[0, 5], [1, 3, 5], [0, 1, 2, 3, 4, 5], [0, 2], [2, 5]]):
        q, k, v = start(a, 40, first, seed=i)
        for g, z in zip(first, first[1:]):
            for t in (q, k, v):
                t[:, g + 1:z] = t[:, g:g + 1]
        lens = [40 if first[0] <= s < first[-1] else 0 for s in range(5)]
        b.prefill(q, k, v, lens)
        x = inputs(a, 2, "bf16", 50 + i)
        o = [p.extend(x[0].clone(), x[1], x[2]) for p in (a, b)]
        assert close(*o, "bf16"), first
        seen.add((a._first.data_ptr(), a._shared.data_ptr(), len(a._shared_ws), a._shared_ws[-1].data_ptr()))
        torch.cuda.synchronize()
        used = torch.cuda.memory_allocated()
        if i > 2:
            assert used <= most
        most = used
    assert len(seen) <= 2  # (the second fork has more groups: a larger plan)
    a.clear()
    assert a._groups is None and not a._shared.any()


def test_forks_that_are_refused_change_nothing():
    a = make("e4m3", n_pages=8)
    q, k, v = inputs(a, 70, "bf16", 0)
    a.prefill(q, k, v, [70, 0, 0, 1, 0])

    def state():
        return (list(a.rows), [list(p) for p in a._pages], list(a._free), a.kv.lens.tolist(), a.kv.table.tolist(), a._groups is None)

    before = state()
    for first, n in (([0, 4], 1), ([0, 3, 5], 1), ([0], 1), ([], 1), ([0, 6], 1), ([-1, 3], 1), ([0, 0, 2], 1), ([2, 1], 1), ([0, 2], 0)):
        with pytest.raises(ValueError):
            if (first, n) == ([0, 3, 5], 1):
                a.grown([0, 0, 0, 0, 16])  # (books a page of sequence 4: it is not empty)
                try:
                    a.fork(first, n)
                finally:
                    a.clear()
                    a.prefill(q, k, v, [70, 0, 0, 1, 0])
                    before = state()
            else:
                a.fork(first, n)
        assert state() == before
    a.fork([0, 3])  # two copies of the fifth page: the last ones that are free
    assert not a._free


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
def test_four_bit_pages_in_a_path(dtype):
    """Prompts, tokens, drafts taken back however far, each against the 64-bit form over what the cache holds."""
    path = make("mx4", dtype, B=3)
    lens = [70, 1, 33]
    q, k, v = inputs(path, 70, dtype, 0)
    path.prefill(q, k, v, lens)
    for i, (n, new, back) in enumerate([(1, None, None), (4, [4, 2, 1], [3, 1, 0]), (1, [1, 0, 1], [60, 0, 30]), (2, None, None)]):
        q, k, v = inputs(path, n, dtype, 50 + 10 * i)
        lse = torch.full(q.shape[:4], 7.0, device="cuda")
        out = path.extend(q, k, v, new, out=torch.full_like(q, 7.0), lse=lse)
        new = [n] * 3 if new is None else new
        lens = [x + y for x, y in zip(lens, new)]
        check4(path.kv, q, out, lse, lens, new)
        if back:
            path.take_back(back)
            lens = [x - y for x, y in zip(lens, back)]
        assert path.kv.lens.tolist() == lens == path.rows


@pytest.mark.parametrize("fmt", FORMATS)
def test_rows_that_a_path_holds(fmt):
    path = make(fmt, B=3)
    q, k, v = inputs(path, 40, "bf16", 0)
    path.prefill(q, k, v, [40, 7, 0])
    a, b = path.held(40, [0, 0, 0]), path.held(7)
    for x, y in zip(a, b):
        assert torch.equal(bits(x[:, 0, :, 33:]), bits(y[:, 0])) and torch.equal(bits(x[:, 1, :, :7]), bits(y[:, 1]))
        assert not x[:, 2].any() and not x[:, 1, :, 7:].any() and bool(x[:, 0].any())
    if fmt == "same":
        assert torch.equal(bits(a[1][:, 0]), bits(v[:, 0]))
    for bad in ((0, None), (3, [0, 0]), (3, [0, -1, 0])):
        with pytest.raises(ValueError):
            path.held(*bad)


def test_an_evicted_cache_in_four_bits():
    """adopt() takes the kept rows of a MPCachePath into pages of any format."""
    import paper_2501_06807_amd as M
    path = make("mx4", B=2, page=16)

    class Kept:
        Ts, n_tail = 32, 3
        k_s = torch.randn(2, 2, 2, 40, 64, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).bfloat16()
        v_s = torch.randn(2, 2, 2, 40, 64, device="cuda", generator=torch.Generator("cuda").manual_seed(2)).bfloat16()

    path.adopt(Kept, 500)
    k, v = path.held(35)
    again = M.paged_kv(n_layers=2, batch=2, n_kv_heads=2, head_dim=64, dtype=torch.bfloat16, n_pages=6, max_pages=3, page_size=16, fmt="mx4")
    again.table.copy_(torch.arange(6).view(2, 3))
    again.lens.fill_(35)
    M.mpc_paged_append(Kept.k_s[:, :, :, :35], Kept.v_s[:, :, :, :35], again)
    k2, v2 = torch.zeros_like(k), torch.zeros_like(v)
    M.mpc_paged_read(again, k2, v2)
    assert torch.equal(bits(k), bits(k2)) and torch.equal(bits(v), bits(v2))
    assert float((k.float() - Kept.k_s[:, :, :, :35].float()).norm() / k.float().norm()) < 0.2
