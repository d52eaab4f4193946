"""Sequences that end among the shared rows of 8-bit pages: mpc_shared_attn gives them the group's rows, as the first sequence's pages hold them,
also where the sequence's own table and tail would say otherwise."""
import math

import pytest
import torch

from test_gpu_paged_append import tokens
from test_gpu_shared_attn import behind, check, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("G,n,room", [(1, 1, None), (4, 5, None), (4, 5, 1 << 14)])  # units of 16, 32 and 128 query rows
@pytest.mark.parametrize("short", [1, 16, 17, 100, 159])
def test_the_groups_rows_are_the_first_sequences(dtype, G, n, room, short):
    import paper_2501_06807_amd as M
    lens, first, shared = [190, 161, 300, 175, 164], [0, 5], [160]
    kv = behind(M, "e4m3", dtype, lens, first, shared, 1, 1)
    if room:
        table = torch.full((5, room), -1, dtype=torch.int32, device="cuda")
        table[:, : kv.table.shape[1]] = kv.table
        kv = M.PagedKV(kv.k_pages, kv.v_pages, table, kv.lens, k_scale=kv.k_scale, v_scale=kv.v_scale, k_tail=kv.k_tail, v_tail=kv.v_tail)
    kv.k_tail[0, 1], kv.v_tail[0, 1] = math.nan, math.nan  # what a sequence has in its tail is not read for shared rows
    lens[1], lens[3] = short, 0
    kv.lens.copy_(torch.tensor(lens))
    q = tokens((1, 5, G, n, 64), dtype, 9).cuda()
    out, lse = run(M, kv, q, first, shared)
    check(kv, q, out, lse, lens, first, shared)
    assert bool((out[0, 3] == 0).all()) and bool((lse[0, 3] == -math.inf).all())
    assert bool(out[0, 1, :, -1].isfinite().all())
