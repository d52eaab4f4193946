"""Host-side refusals of the attention behind shared rows, and the sizes of its workspace (no GPU)."""
import ctypes

import pytest
from test_paged_refusals import FAKE, ODD, cache, dims, ref

from paper_2501_06807_amd import _lib as L


def shared(d=None, kv=None, n=1, cfg=True, q=FAKE, out=FAKE, os_=None, ws=FAKE, ws_bytes=0, groups=2, first=1 << 20, rows=1 << 20,
           no_shared=False, **kw):
    lib = L.lib()
    c = L.MpcAttnCfg(**dict(dict(sm_scale=0.1, window=0, sinks=0), **kw)) if cfg else None
    s = lib.mpc_shared_attn(ref(d or dims()), ref(kv or cache()), n, None, None if no_shared else ref(L.MpcShared(groups, first, rows)),
                            ref(c), q, None, out, ref(os_), None, ws, ws_bytes, None)
    return s, lib.mpc_last_error().decode()


def size(d, n, kv, groups):
    z = L.MpcSharedSizes(None if kv is None else ctypes.pointer(kv), groups)
    return L.lib().mpc_workspace_bytes(L.MPC_OP_SHARED_ATTN, ref(d), n, ctypes.byref(z))


@pytest.mark.parametrize("kw,expect", [
    (dict(n=0), L.MPC_EINVAL), (dict(no_shared=True), L.MPC_EINVAL), (dict(first=None), L.MPC_EINVAL), (dict(rows=None), L.MPC_EINVAL),
    (dict(groups=0), L.MPC_EINVAL), (dict(groups=-3), L.MPC_EINVAL), (dict(groups=3), L.MPC_EINVAL),  # (two sequences)
    (dict(d=dims(batch=2000), groups=1025), L.MPC_EUNSUPPORTED), (dict(cfg=False), L.MPC_EINVAL), (dict(window=-1), L.MPC_EINVAL),
    (dict(sm_scale=float("nan")), L.MPC_EINVAL), (dict(q=None), L.MPC_EINVAL), (dict(out=ODD), L.MPC_EINVAL),
    (dict(os_=L.MpcStrides(2048, 1024, 0, 128)), L.MPC_ESHAPE), (dict(kv=cache(format=2)), L.MPC_EINVAL), (dict(d=dims(head_dim=96)), L.MPC_EUNSUPPORTED),
    (dict(n=1 << 26, ws_bytes=1 << 62), L.MPC_EUNSUPPORTED),  # 2^31 query rows over two layers, two sequences and eight heads
    (dict(n=1 << 28, ws_bytes=1 << 62), L.MPC_EUNSUPPORTED),  # 2^28 tokens of two sequences of four heads to a kv head
])
def test_calls(kw, expect):
    s, msg = shared(**kw)
    assert s == expect and msg


def test_workspace():
    need = size(dims(), 1, cache(), 2)
    assert need > L.lib().mpc_workspace_bytes(L.MPC_OP_PAGED_ATTN, ref(dims()), 1, ref(cache())) > 0
    assert shared(ws_bytes=need - 1)[0] == L.MPC_EWORKSPACE and shared(ws=None, ws_bytes=need)[0] == L.MPC_EWORKSPACE
    assert shared(ws=ODD, ws_bytes=need)[0] == L.MPC_EINVAL
    for bad in (size(dims(), 0, cache(), 1), size(dims(), 1, None, 1), size(dims(), 1, cache(), 3), size(dims(), 1, cache(), 0),
                size(dims(), 1, cache(page_size=8), 1), L.lib().mpc_workspace_bytes(L.MPC_OP_SHARED_ATTN, ref(dims()), 1, None)):
        assert bad == 0
    huge = cache(max_pages=1 << 24, page_size=64)
    assert size(dims(batch=1024), 1, huge, 1) == 0 and shared(d=dims(batch=1024), kv=huge, groups=1, ws_bytes=1 << 50)[0] == L.MPC_EUNSUPPORTED


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("heads", [(8, 8), (8, 2), (8, 1)])
def test_bytes_never_fall(dtype, heads):
    """A workspace made for the most tokens, sequences and groups serves calls of fewer, whatever form each takes."""
    make = lambda b, L=2: dims(batch=b, n_layers=L, n_q_heads=heads[0], n_kv_heads=heads[1], dtype=dtype)  # noqa: E731
    for groups in (1, 3, 16):
        sizes = [size(make(16), n, cache(), groups) for n in (1, 2, 3, 4, 5, 8, 9, 16, 17, 33, 64, 100, 1000)]
        assert sizes == sorted(sizes) and sizes[0] > 0
    for n in (1, 4, 40):
        assert sorted(s := [size(make(16), n, cache(), g) for g in range(1, 17)]) == s
        assert sorted(s := [size(make(b), n, cache(), 1) for b in range(1, 80)]) == s
        assert size(make(8, 1), n, cache(), 2) <= size(make(8, 5), n, cache(), 2)
