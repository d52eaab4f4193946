"""Sizes of the paged attention's workspace (no GPU): one made for the most rows serves every call of that head_dim."""
from test_paged_refusals import cache, dims, ref

from paper_2501_06807_amd import _lib as L


def size(d, n, kv):
    return L.lib().mpc_workspace_bytes(L.MPC_OP_PAGED_ATTN, ref(d), n, ref(kv))


def test_bytes_follow_the_query_rows_and_head_dim_only():
    most = size(dims(), 8, cache())  # four heads to a kv head: 32 rows
    last = 0
    for n in (1, 2, 3, 4, 5, 8, 9, 100, 5000):
        got = size(dims(), n, cache())
        assert last <= got <= most
        last = got
    assert last == most
    for d in (dims(batch=1, n_layers=1, n_q_heads=1, n_kv_heads=1), dims(batch=100, n_layers=32), dims(dtype=0), dims(head_dim=64)):
        for kv in (cache(max_pages=1), cache(max_pages=1 << 12), cache(format=0), cache(page_size=256)):
            for n in (1, 7, 64, 300):
                assert 0 < size(d, n, kv) <= most
    assert size(dims(batch=100, n_layers=32), 1, cache(max_pages=1 << 12)) == size(dims(), 1, cache())
