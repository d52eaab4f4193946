"""Infinite values among the shared rows of mpc_shared_attn: what a row sees of them reaches it as an infinity, however small its weight,
as in mpc_paged_attn, and whichever kind of tile they lie in."""
import math

import pytest
import torch

from test_gpu_paged_append import bits, tokens
from test_gpu_shared_attn import behind, check, run

pytestmark = pytest.mark.gpu

LENS, T = [190, 161, 300, 175, 164], 160


def cache(M, dtype, rows, d=64, G=4, n=5, big=7):
    """A score of about 32 nats above the others in shared row `big`, and infinities in the values of `rows`: whose weights are far below
    what either 16-bit type holds beside it."""
    kv = behind(M, "same", dtype, LENS, [0, 5], [T], 1, 1, d)
    q = tokens((1, 5, G, n, d), dtype, 9, spread=False).abs().cuda()
    kv.k_pages[0, int(kv.table[0, big // 16]), 0, big % 16] = 5.0 * math.sqrt(64 / d)
    for i, row in enumerate(rows):
        id, slot = int(kv.table[0, row // 16]), row % 16
        kv.k_pages[0, id, 0, slot] = 0
        kv.v_pages[0, id, 0, slot, 33] = math.inf
        kv.v_pages[0, id, 0, slot, 40] = -math.inf
        kv.v_pages[0, id, 0, slot, 50] = math.inf if i % 2 else -math.inf
    return kv, q


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("G,n,d", [(1, 1, 64), (4, 1, 128), (4, 5, 64), (8, 4, 128)])
@pytest.mark.parametrize("rows", [[40], [0, 159], [33, 100, 101]])
def test_infinities_that_every_row_sees(dtype, G, n, d, rows):
    import paper_2501_06807_amd as M
    kv, q = cache(M, dtype, rows, d, G, n)
    for window in (0, 100, 5000):
        out, lse = run(M, kv, q, [0, 5], [T], window=window)
        check(kv, q, out, lse, LENS, [0, 5], [T], window=window)
        assert bool(lse.isfinite().all())
        if window != 100:
            x = out[:, [0, 2]]  # whose rows stand behind all of the shared ones
            assert bool((x[..., 33] == math.inf).all()) and bool((x[..., 40] == -math.inf).all())
            assert bool(x[..., 50].isnan().all() if len(rows) > 1 else (x[..., 50] == -math.inf).all())
            assert bool(x[..., :33].isfinite().all())


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_as_the_paged_attention_has_them(dtype):
    """The same places that are not finite, and the same values in them; the rest as if the infinities were not there."""
    import paper_2501_06807_amd as M
    kv, q = cache(M, dtype, [40, 90])
    out, lse = run(M, kv, q, [0, 5], [T])
    for b in range(1, 5):
        kv.table[b, : T // 16] = kv.table[0, : T // 16]
    want, lse2 = torch.zeros_like(out), torch.zeros_like(lse)
    M.mpc_paged_attn(q, kv, want, sm_scale=1 / math.sqrt(64), lse=lse2)
    fine = want.isfinite()
    assert torch.equal(fine, out.isfinite()) and torch.equal(want.isnan(), out.isnan())
    rest = ~fine & ~want.isnan()
    assert torch.equal(want[rest], out[rest]) and int(rest.sum()) > 0
    for row in (40, 90):
        id = int(kv.table[0, row // 16])
        kv.v_pages[0, id, 0, row % 16, [33, 40, 50]] = 0
    clean, l0 = run(M, kv, q, [0, 5], [T])
    assert torch.equal(bits(lse), bits(l0))
    err = (out[fine].float() - clean[fine].float()).norm() / clean[fine].float().norm()
    assert float(err) < 4 * torch.finfo(out.dtype).eps / 2


def test_many_runs_of_which_one_has_an_infinity():
    """Hundreds of rows behind a long prompt: other heads, and other workgroups' runs, are as without it."""
    import paper_2501_06807_amd as M
    B, G, n, T_ = 6, 8, 40, 2000
    lens = [T_ + n + (7 * b) % 50 for b in range(B)]
    kv = behind(M, "same", "bf16", lens, [0, B], [T_], Hkv=2, d=128)
    q = tokens((1, B, 2 * G, n, 128), "bf16", 9).cuda()
    clean, l0 = run(M, kv, q, [0, B], [T_])
    id = int(kv.table[0, 70])
    kv.v_pages[0, id, 1, 3, 77] = math.inf
    out, lse = run(M, kv, q, [0, B], [T_])
    assert bool((out[0, :, G:, :, 77] == math.inf).all()) and torch.equal(bits(out[:, :, :G]), bits(clean[:, :, :G]))
    out[0, :, G:, :, 77] = 0
    clean[0, :, G:, :, 77] = 0
    assert bool(out.isfinite().all()) and torch.equal(bits(lse[:, :, :G]), bits(l0[:, :, :G]))
    assert float((out.float() - clean.float()).norm() / clean.float().norm()) < 2.0 ** -7 and float((lse - l0).abs().max()) < 1e-4
