"""One workspace of the paged attention for calls of different shapes."""
import pytest
import torch

from test_gpu_attn import fill, run_paged
from test_gpu_paged_append import bits, make, tokens

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
