"""Host-side refusals around 4-bit pages and reading back (no GPU): nothing reaches a launch."""
import ctypes

import pytest
import torch
from test_paged_refusals import FAKE, ODD, append, cache, dims, paged, ref

from paper_2501_06807_amd import _lib as L


def cache4(**kw):
    return cache(**dict(dict(format=4, k_tail=None, v_tail=None), **kw))


def read(d=None, kv=None, n=1, k=FAKE, ks=None, v=FAKE, vs=None, no_kv=False):
    lib = L.lib()
    s = lib.mpc_paged_read(ref(d or dims()), None if no_kv else ref(kv or cache4()), n, None, None, k, ref(ks), v, ref(vs), None)
    return s, lib.mpc_last_error().decode()


@pytest.mark.parametrize("call", [append, paged, read])
@pytest.mark.parametrize("kv,expect", [
    (cache4(k_scale=None), L.MPC_EINVAL), (cache4(v_scale=None), L.MPC_EINVAL), (cache4(k_scale=(1 << 20) + 4), L.MPC_EINVAL),
    (cache4(v_pages=(1 << 20) + 8), L.MPC_EINVAL), (cache4(page_size=8), L.MPC_EUNSUPPORTED), (cache(format=3), L.MPC_EINVAL),
    (cache(format=5), L.MPC_EINVAL),
])
def test_caches(call, kv, expect):
    s, msg = call(kv=kv)
    assert s == expect and msg


@pytest.mark.parametrize("kw,expect", [
    (dict(no_kv=True), L.MPC_EINVAL), (dict(n=0), L.MPC_EINVAL), (dict(n=(1 << 31) - 1), L.MPC_EINVAL), (dict(n=1 << 29), L.MPC_EUNSUPPORTED), (dict(k=None, v=None), L.MPC_EINVAL),
    (dict(k=ODD), L.MPC_EINVAL), (dict(v=ODD), L.MPC_EINVAL), (dict(n=4, ks=L.MpcStrides(4096, 2048, 0, 128)), L.MPC_ESHAPE),
    (dict(n=4, vs=L.MpcStrides(4096, 2048, 1024, 100)), L.MPC_EINVAL), (dict(d=dims(head_dim=96)), L.MPC_EUNSUPPORTED),
    (dict(d=dims(dtype=3)), L.MPC_EINVAL),
])
def test_reads(kw, expect):
    s, msg = read(**kw)
    assert s == expect and msg


def test_tails_are_not_asked_for():
    """A 4-bit cache passes without tails: the call is refused for the workspace only."""
    assert paged(kv=cache4(), ws=None)[0] == L.MPC_EWORKSPACE
    size = L.lib().mpc_workspace_bytes(L.MPC_OP_PAGED_ATTN, ref(dims()), 1, ref(cache4()))
    assert size == L.lib().mpc_workspace_bytes(L.MPC_OP_PAGED_ATTN, ref(dims()), 1, ref(cache()))


def test_formats_by_name():
    assert L._page_format(None, False) == "same" and L._page_format(None, True) == "e4m3" and L._page_format("mx4", False) == "mx4"
    for fmt, fp8 in (("mx4", True), ("same", True), ("fp8", False), ("", False)):
        with pytest.raises(ValueError):
            L._page_format(fmt, fp8)


def test_the_handle_refuses_tensors_on_the_host():
    z = lambda t, *s: torch.zeros(s, dtype=t)  # noqa: E731
    pages, scale = z(torch.uint8, 1, 4, 2, 16, 32), z(torch.uint8, 1, 4, 2, 2, 16)
    with pytest.raises(ValueError):  # (a host tensor; no scales; tails)
        L.PagedKV(pages, pages, z(torch.int32, 1, 4), z(torch.int32, 1), k_scale=scale, v_scale=scale, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        L.PagedKV(pages, pages, z(torch.int32, 1, 4), z(torch.int32, 1), k_scale=scale, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        L.PagedKV(pages, pages, z(torch.int32, 1, 4), z(torch.int32, 1), k_scale=scale, v_scale=scale, k_tail=pages, v_tail=pages)
