"""The sizes that mpc_shared_attn takes: those of mpc_paged_attn, and the limits that the header adds (no GPU)."""
import pytest
from test_paged_refusals import cache, dims, ref
from test_shared_refusals import size

from paper_2501_06807_amd import _lib as L


def paged_size(d, n, kv):
    return L.lib().mpc_workspace_bytes(L.MPC_OP_PAGED_ATTN, ref(d), n, ref(kv))


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("fmt", [0, 1, 4])
@pytest.mark.parametrize("heads", [(32, 32), (32, 8), (8, 1)])
def test_what_the_paged_attention_takes_is_taken(dtype, fmt, heads):
    """Up to the largest table with which mpc_paged_attn takes the other sizes."""
    for layers, batch, n in ((32, 128, 1), (32, 100, 1), (80, 64, 1), (4, 1000, 1), (8, 32, 40), (2, 4, 5000), (1, 1, 1), (1, 2000, 1)):
        d = dims(batch=batch, n_layers=layers, n_q_heads=heads[0], n_kv_heads=heads[1], dtype=dtype)
        taken = [m for m in range(23) if paged_size(d, n, cache(page_size=256, max_pages=1 << m, format=fmt))]
        assert taken == list(range(len(taken))) and taken
        edge = 1 << taken[-1]
        for M in {edge, max(1, edge - 1), edge // 2 + 1, 1}:
            kv = cache(page_size=256, max_pages=M, format=fmt)
            assert paged_size(d, n, kv)
            for groups in {1, 2, batch // 2, min(batch, 1024)}:
                if 1 <= groups <= batch:
                    assert layers * heads[1] * groups < 2 ** 29 and layers * batch * heads[0] * n < 2 ** 31
                    assert size(d, n, kv, groups), (layers, batch, n, M, groups)


@pytest.mark.parametrize("layers,batch,n,M", [(32, 128, 1, 1 << 22), (1 << 10, 1 << 10, 1, 1 << 16)])
def test_what_it_refuses_is_refused(layers, batch, n, M):
    d, kv = dims(batch=batch, n_layers=layers, n_q_heads=32, n_kv_heads=32), cache(page_size=256, max_pages=M)
    assert paged_size(d, n, kv) == 0 and size(d, n, kv, 1) == 0
