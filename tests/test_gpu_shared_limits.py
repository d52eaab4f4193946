"""mpc_shared_attn over tables with room for so many rows that its blocks of keys become larger, against mpc_paged_attn."""
import math

import pytest
import torch

import paged_ref as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,cap,first,fmt", [
    (128, 1 << 20, [0, 64, 128], "same"),  # own rows: 2^31 blocks of 64 keys, more than the paged attention has
    (120, 1 << 22, list(range(121)), "same"),  # shared rows too: a group for each sequence
    (128, 1 << 20, [0, 1, 128], "mx4"),
])
def test_large_tables(B, cap, first, fmt):
    import paper_2501_06807_amd as M
    L, H, d, page, P, n = 32, 32, 64, 256, 4, 1
    kv = M.paged_kv(n_layers=L, batch=B, n_kv_heads=H, head_dim=d, dtype=torch.bfloat16, n_pages=P, max_pages=cap // page, page_size=page, fmt=fmt)
    g = torch.Generator(device="cuda").manual_seed(1)
    for t in (kv.k_pages, kv.v_pages):
        if fmt == "mx4":
            t.random_(0, 256, generator=g)
        else:
            t.normal_(generator=g)
    if fmt == "mx4":
        kv.k_scale.random_(124, 128, generator=g)
        kv.v_scale.random_(124, 128, generator=g)
    kv.table.copy_((torch.arange(B)[:, None] + torch.arange(cap // page)).remainder(P - 1) + 1)
    kv.table[:, :1] = 0  # the shared page
    lens = [256 + 1 + (37 * b) % 700 for b in range(B)]
    kv.lens.copy_(torch.tensor(lens))
    q = torch.randn(L, B, H, n, d, device="cuda", generator=g).bfloat16()
    out, want, lse, lse2 = torch.zeros_like(q), torch.zeros_like(q), torch.zeros(q.shape[:4], device="cuda"), torch.zeros(q.shape[:4], device="cuda")
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    M.mpc_shared_attn(q, kv, out, first=ints(first), shared_rows=ints([256] * (len(first) - 1)), sm_scale=1 / math.sqrt(d), lse=lse)
    M.mpc_paged_attn(q, kv, want, sm_scale=1 / math.sqrt(d), lse=lse2)
    torch.cuda.synchronize()
    # each is within half a step of the exact one, and a few steps of fp32
    rows = lambda x: x.float().transpose(0, 1).flatten(1)  # noqa: E731
    err = (rows(out) - rows(want)).norm(dim=1) / rows(want).norm(dim=1)
    assert float(err.max()) < 2 * R.half_step(torch.bfloat16) and float((lse - lse2).abs().max()) < 1e-4
