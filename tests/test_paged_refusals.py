"""Host-side refusals of the paged-cache entry points (no GPU): nothing reaches a launch."""
import ctypes

import pytest

from paper_2501_06807_amd import _lib as L

FAKE = ctypes.c_void_p(1 << 20)  # never dereferenced: validation fails before any launch
ODD = ctypes.c_void_p((1 << 20) + 8)


def dims(**kw):
    return L.MpcDims(**dict(dict(batch=2, layer0=0, n_layers=2, n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=2), **kw))


def cache(**kw):
    p = 1 << 20
    return L.MpcPagedKv(**dict(dict(page_size=32, n_pages=10, max_pages=5, format=1, k_pages=p, v_pages=p, k_scale=p, v_scale=p,
                                    k_tail=p, v_tail=p, table=p, lens=p), **kw))


def rope(**kw):
    return L.MpcRope(**dict(dict(table=1 << 20, n_pos=100, rot_dim=64, style=1), **kw))


def ref(x):
    return None if x is None else ctypes.byref(x)


def append(d=None, kv=None, n=1, r=None, k=FAKE, ks=None, v=FAKE, q=None, q_out=None, os_=None, no_kv=False, k_out=None, ko=None):
    lib = L.lib()
    s = lib.mpc_paged_append(ref(d or dims()), None if no_kv else ref(kv or cache()), n, None, ref(r), None, k, ref(ks), v, None, q,
                             None, q_out, ref(os_), k_out, ref(ko), None)
    return s, lib.mpc_last_error().decode()


def paged(d=None, kv=None, n=1, cfg=True, q=FAKE, out=FAKE, os_=None, ws=FAKE, ws_bytes=0, **kw):
    lib = L.lib()
    c = L.MpcAttnCfg(**dict(dict(sm_scale=0.1, window=0, sinks=0), **kw)) if cfg else None
    s = lib.mpc_paged_attn(ref(d or dims()), ref(kv or cache()), n, None, ref(c), q, None, out, ref(os_), None, ws, ws_bytes, None)
    return s, lib.mpc_last_error().decode()


def prompt(d=None, Tq=5, T=5, cfg=True, q=FAKE, k=FAKE, ks=None, v=FAKE, out=FAKE, os_=None, **kw):
    lib = L.lib()
    c = L.MpcAttnCfg(**dict(dict(sm_scale=0.1, window=0, sinks=0), **kw)) if cfg else None
    s = lib.mpc_prompt_attn(ref(d or dims()), Tq, T, None, None, ref(c), q, None, k, ref(ks), v, None, out, ref(os_), None, None)
    return s, lib.mpc_last_error().decode()


@pytest.mark.parametrize("call", [append, paged, prompt])
@pytest.mark.parametrize("d,expect", [
    (dims(batch=0), L.MPC_EINVAL), (dims(dtype=5), L.MPC_EINVAL), (dims(head_dim=96), L.MPC_EUNSUPPORTED),
    (dims(n_q_heads=7), L.MPC_ESHAPE), (dims(n_q_heads=6), L.MPC_EUNSUPPORTED), (dims(n_q_heads=32), L.MPC_EUNSUPPORTED),
])
def test_dims(call, d, expect):
    s, msg = call(d=d)
    assert s == expect and msg


@pytest.mark.parametrize("call", [append, paged])
@pytest.mark.parametrize("kv,expect", [
    (cache(page_size=8), L.MPC_EUNSUPPORTED), (cache(page_size=48), L.MPC_EUNSUPPORTED), (cache(page_size=512), L.MPC_EUNSUPPORTED),
    (cache(n_pages=0), L.MPC_EINVAL), (cache(max_pages=-1), L.MPC_EINVAL), (cache(max_pages=1 << 26), L.MPC_EUNSUPPORTED),
    (cache(format=2), L.MPC_EINVAL), (cache(k_pages=None), L.MPC_EINVAL), (cache(table=None), L.MPC_EINVAL),
    (cache(lens=None), L.MPC_EINVAL), (cache(k_scale=None), L.MPC_EINVAL), (cache(v_tail=None), L.MPC_EINVAL),
    (cache(v_pages=(1 << 20) + 4), L.MPC_EINVAL),
])
def test_caches(call, kv, expect):
    s, msg = call(kv=kv)
    assert s == expect and msg


@pytest.mark.parametrize("kw,expect", [
    (dict(no_kv=True), L.MPC_EINVAL), (dict(n=0), L.MPC_EINVAL), (dict(k=None), L.MPC_EINVAL), (dict(v=ODD), L.MPC_EINVAL),
    (dict(q=FAKE, q_out=FAKE), L.MPC_EINVAL),  # queries without a rotation
    (dict(q=FAKE, r=rope()), L.MPC_EINVAL), (dict(q_out=FAKE, r=rope()), L.MPC_EINVAL),
    (dict(r=rope(rot_dim=24)), L.MPC_ESHAPE), (dict(r=rope(rot_dim=256)), L.MPC_ESHAPE), (dict(r=rope(rot_dim=0)), L.MPC_ESHAPE),
    (dict(r=rope(style=2)), L.MPC_EINVAL), (dict(r=rope(table=None)), L.MPC_EINVAL), (dict(r=rope(n_pos=0)), L.MPC_EINVAL),
    (dict(r=rope(table=(1 << 20) + 8)), L.MPC_EINVAL),
    (dict(ks=L.MpcStrides(-8, 1024, 128, 128)), L.MPC_EINVAL), (dict(ks=L.MpcStrides(4096, 1024, 132, 128)), L.MPC_EINVAL),
    (dict(ks=L.MpcStrides(1 << 60, 1024, 128, 128)), L.MPC_EINVAL),
    (dict(k_out=FAKE), L.MPC_EINVAL), (dict(k_out=ODD), L.MPC_EINVAL),  # k itself, and off its alignment
    (dict(k_out=ctypes.c_void_p(1 << 22), ko=L.MpcStrides(4096, 1024, 0, 128)), L.MPC_ESHAPE),
    # rows that are written may not lie on each other: heads a half row apart, sequences on one place
    (dict(q=FAKE, q_out=FAKE, r=rope(), os_=L.MpcStrides(4096, 1024, 64, 128)), L.MPC_ESHAPE),
    (dict(q=FAKE, q_out=FAKE, r=rope(), os_=L.MpcStrides(4096, 0, 128, 128)), L.MPC_ESHAPE),
])
def test_append(kw, expect):
    s, msg = append(**kw)
    assert s == expect and msg


@pytest.mark.parametrize("kw,expect", [
    (dict(n=0), L.MPC_EINVAL), (dict(n=-1), L.MPC_EINVAL), (dict(cfg=False), L.MPC_EINVAL), (dict(window=-1), L.MPC_EINVAL),
    (dict(sinks=-2), L.MPC_EINVAL), (dict(sm_scale=float("nan")), L.MPC_EINVAL), (dict(sm_scale=float("inf")), L.MPC_EINVAL),
    (dict(q=None), L.MPC_EINVAL), (dict(out=ODD), L.MPC_EINVAL), (dict(os_=L.MpcStrides(2048, 1024, 0, 128)), L.MPC_ESHAPE),
])
def test_paged_attn(kw, expect):
    s, msg = paged(**kw)
    assert s == expect and msg


@pytest.mark.parametrize("kw,expect", [
    (dict(Tq=0), L.MPC_EINVAL), (dict(T=-4), L.MPC_EINVAL), (dict(T=(1 << 30) + 1), L.MPC_EUNSUPPORTED), (dict(cfg=False), L.MPC_EINVAL),
    (dict(window=-1), L.MPC_EINVAL), (dict(sm_scale=float("inf")), L.MPC_EINVAL), (dict(v=None), L.MPC_EINVAL), (dict(k=ODD), L.MPC_EINVAL),
    (dict(ks=L.MpcStrides(4096, 1024, 128, 129)), L.MPC_EINVAL), (dict(os_=L.MpcStrides(65536, 16384, 128, 512)), L.MPC_ESHAPE),
])
def test_prompt_attn(kw, expect):
    s, msg = prompt(**kw)
    assert s == expect and msg


def test_workspace_of_the_paged_attention():
    lib = L.lib()
    size = lambda d, n, kv: lib.mpc_workspace_bytes(L.MPC_OP_PAGED_ATTN, ref(d), n, ref(kv))  # noqa: E731
    assert size(dims(), 1, None) == 0 and size(dims(), 0, cache()) == 0 and size(dims(), 1, cache(page_size=8)) == 0
    assert size(None, 1, cache()) == 0
    assert size(dims(), 1, cache()) > 0
    huge = cache(max_pages=1 << 24, page_size=64)
    assert size(dims(batch=1024), 1, huge) == 0  # more than 2^31 key blocks
    assert paged(d=dims(batch=1024), kv=huge, ws_bytes=1 << 40)[0] == L.MPC_EUNSUPPORTED
    need = size(dims(), 1, cache())
    assert paged(ws_bytes=need - 1)[0] == L.MPC_EWORKSPACE and paged(ws=None, ws_bytes=need)[0] == L.MPC_EWORKSPACE
    assert paged(ws=ODD, ws_bytes=need)[0] == L.MPC_EINVAL


@pytest.mark.parametrize("n", [1 << 29, 1 << 30])
def test_query_rows_beyond_the_limit(n):
    assert paged(n=n, ws_bytes=1 << 60)[0] == L.MPC_EUNSUPPORTED  # four heads to a kv head
    assert append(n=n)[0] == L.MPC_EUNSUPPORTED
    assert prompt(Tq=n, T=5)[0] == L.MPC_EUNSUPPORTED
