"""One workspace of the paged attention for calls of different shapes, the one that a call makes for itself on another stream,
and a step of PagedPath whose first use is its capture."""
import pytest
import torch

from test_gpu_attn import fill, run_paged
from test_gpu_paged_append import bits, make, tokens
from test_gpu_paged_path import inputs
from test_gpu_paged_path import make as make_path

pytestmark = pytest.mark.gpu


def test_one_workspace_for_calls_of_different_shapes():
    """Calls of one token and of sixteen, over two caches, in turn on the largest workspace, as a server makes them: each
    gives what it gives on a workspace of its own, with the keys of every head divided over workgroups."""
    import paper_2501_06807_amd as M
    kvs = [make(M, 2, 4, 8, 128, "bf16", 32, cap=64), make(M, 1, 1, 2, 128, "bf16", 32, cap=200)]
    fill(kvs[0], [2000, 1500, 2048, 1999], 3, "bf16")
    fill(kvs[1], [6400], 4, "bf16")
    calls = []
    for kv, n in ((kvs[0], 1), (kvs[0], 16), (kvs[1], 1), (kvs[1], 40)):
        q = tokens((kv.L, kv.B, 4 * kv.Hkv, n, 128), "bf16", 5 + n, spread=False).cuda()
        calls.append((kv, q, [n] * kv.B, run_paged(kv, q, [n] * kv.B)))
    ws = M.workspace(max(M.paged_attn_workspace_bytes(q, kv) for kv, q, _, _ in calls))
    for i in (1, 0, 1, 2, 3, 0, 1, 3, 2, 1):
        kv, q, new, want = calls[i]
        got = run_paged(kv, q, new, ws=ws)
        assert torch.equal(bits(got[0]), bits(want[0])) and torch.equal(bits(got[1]), bits(want[1])), i


def test_workspace_of_a_call_on_another_stream():
    """A call without ws, on a stream that is not the current one: its workspace is made and cleared there."""
    import paper_2501_06807_amd as M
    kv = make(M, 1, 2, 2, 128, "bf16", 32, cap=100)
    fill(kv, [3200, 2000], 3, "bf16")
    q = tokens((1, 2, 8, 1, 128), "bf16", 5, spread=False).cuda()
    want = run_paged(kv, q, [1, 1])
    side = torch.cuda.Stream()
    new = torch.tensor([1, 1], dtype=torch.int32, device="cuda")
    outs = [torch.full_like(q, 7.0) for _ in range(8)]
    torch.cuda.synchronize()
    busy = torch.randn(4096, 4096, device="cuda")
    for out in outs:
        busy = busy @ busy * 1e-4  # what the current stream has before the zeros, if they were put there
        M.mpc_paged_attn(q, kv, out, sm_scale=128 ** -0.5, n_valid=new, stream=side)
    side.synchronize()
    for out in outs:
        assert torch.equal(bits(out), bits(want[0]))


def test_a_step_whose_first_use_is_its_capture():
    """The capture makes nothing that later steps use (its clearing would wait for the first replay): eager steps of the same
    shape run right after it, before the first replay, and between the replays."""
    import paper_2501_06807_amd as M
    a, b = make_path(page=16), make_path(page=16)
    q, k, v = inputs(a, 100, "bf16", 0)
    for p in (a, b):
        p.prefill(q.clone(), k, v)
        p.reserve([150] * 3)
    q, k, v = inputs(a, 1, "bf16", 5)
    out = torch.zeros_like(q)
    torch.cuda.synchronize()
    held = torch.cuda.memory_allocated()
    g = M.MPCachePath.capture(a, a.step, q, k, v, None, out)
    # (a graph keeps two words of its own; a workspace of two query rows has 270 KB)
    assert torch.cuda.memory_allocated() - held <= 4096
    for i in range(12):
        x = inputs(a, 1, "bf16", 100 + 10 * i)
        if i % 3 == 0:
            got = a.extend(x[0].clone(), x[1], x[2])
        else:
            for dst, src in zip((q, k, v), x):
                dst.copy_(src)
            a.grown([1] * 3)
            g.replay()
            got = out
        want = b.extend(x[0].clone(), x[1], x[2])
        torch.cuda.synchronize()
        assert torch.equal(bits(got), bits(want)), i
    assert a.kv.lens.tolist() == b.kv.lens.tolist() == a.rows
