"""PagedPath.fork() with a sequence that is alone in its group: nothing of it is shared, so its rows can be taken back like any other's."""
import math

import pytest
import torch

import paged_ref as R
from test_gpu_paged_append import DT, bits
from test_gpu_paged_path import inputs
from test_gpu_paged_path_shared import FORMATS, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
def test_rows_of_a_sequence_alone_in_its_group_are_taken_back(fmt, dtype):
    """Into its last whole page: with 8-bit pages what follows stands in the tail, not yet in the page's codes."""
    import paper_2501_06807_amd as M
    path = make(fmt, dtype, B=4)
    q, k, v = inputs(path, 70, dtype, 0)
    path.prefill(q, k, v, [70, 70, 0, 0])
    path.fork([0, 1, 4], n_new=4)
    path.take_back([10, 0, 0, 0])
    for i, (n, back) in enumerate([(3, 1), (1, 0), (4, 2), (1, 0)]):
        x = inputs(path, n, dtype, 50 + 10 * i)
        rows = x[0].clone()
        out = path.extend(rows, x[1], x[2])  # (turns the queries in place)
        want = torch.zeros_like(out)
        M.mpc_paged_attn(rows, path.kv, want, sm_scale=1 / math.sqrt(64))
        # each row is within its bounds of the exact one: a weight's parts, and two outputs rounded once each
        tol = 4 * R.half_step(DT[dtype]) if dtype != "fp32" else 2e-5
        for b in range(4):
            err = float((out[:, b].float() - want[:, b].float()).norm() / want[:, b].float().norm())
            assert err < tol, (i, b, err)
        path.take_back([back] * 4)


def test_what_a_step_behind_such_a_fork_gives_is_what_an_unforked_path_gives():
    a, b = make("e4m3", B=3), make("e4m3", B=3)
    q, k, v = inputs(a, 100, "bf16", 0)
    for p in (a, b):
        p.prefill(q.clone(), k, v, [100, 33, 80])
    a.fork([0, 1, 2, 3], n_new=1)  # three sequences, each by itself
    for back, n in (([19, 2, 15], 1), ([0, 0, 0], 1), ([1, 1, 1], 5), ([0, 0, 0], 1)):
        for p in (a, b):
            p.take_back(back)
        x = inputs(a, n, "bf16", 60 + n)
        out = [p.extend(x[0].clone(), x[1], x[2]) for p in (a, b)]
        assert float((out[0].float() - out[1].float()).norm() / out[1].float().norm()) < 4 * R.half_step(torch.bfloat16)
        for s, t in zip(a.held(100), b.held(100)):
            assert torch.equal(bits(s), bits(t))
