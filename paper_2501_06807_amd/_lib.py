"""ctypes binding of libmpcache.so: the entry points of the C ABI with the same names.

Argument marshalling only: shapes are read off torch CUDA tensors, pointers and the current
stream are handed to the library, and a non-zero status raises MpcError. Every step of the path
runs in the HIP kernels; there is no fallback.
"""
import ctypes
import os

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libmpcache.so")

MPC_OK, MPC_EINVAL, MPC_ESHAPE, MPC_EUNSUPPORTED, MPC_EWORKSPACE, MPC_EHIP = range(6)
MPC_OP_STATIC_EVICT, MPC_OP_SELECT, MPC_OP_DECODE_ATTN, MPC_OP_DECODE_STEP, MPC_OP_PAGED_ATTN, MPC_OP_SHARED_ATTN = range(6)
DTYPE_CODE = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


class MpcDims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("batch", "layer0", "n_layers", "n_q_heads", "n_kv_heads", "head_dim", "dtype", "kv_capacity")]


class MpcSelectCfg(ctypes.Structure):
    _fields_ = [("cluster_size", ctypes.c_int32), ("fanout", ctypes.c_int32),
                ("k_super", ctypes.c_int32), ("k_clusters", ctypes.c_int32),
                ("alpha", ctypes.c_float), ("share_period", ctypes.c_int32),
                ("share_start", ctypes.c_int32), ("similarity", ctypes.c_int32), ("group", ctypes.c_int32)]


class MpcEvictCfg(ctypes.Structure):
    _fields_ = [("window", ctypes.c_int32), ("keep", ctypes.c_int32),
                ("local_keep", ctypes.c_int32), ("sm_scale", ctypes.c_float),
                ("causal", ctypes.c_int32), ("share_period", ctypes.c_int32),
                ("share_start", ctypes.c_int32)]


class MpcStrides(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("layer", "batch", "head", "token")]


class MpcPagedKv(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("page_size", "n_pages", "max_pages", "format")] +
                [(n, ctypes.c_void_p) for n in ("k_pages", "v_pages", "k_scale", "v_scale", "k_tail", "v_tail", "table",
                                                "lens")])


class MpcRope(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("n_pos", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("style", ctypes.c_int32)]


class MpcAttnCfg(ctypes.Structure):
    _fields_ = [("sm_scale", ctypes.c_float), ("window", ctypes.c_int32), ("sinks", ctypes.c_int32)]


class MpcShared(ctypes.Structure):
    _fields_ = [("n_groups", ctypes.c_int32), ("first", ctypes.c_void_p), ("rows", ctypes.c_void_p)]


class MpcSharedSizes(ctypes.Structure):
    _fields_ = [("kv", ctypes.POINTER(MpcPagedKv)), ("n_groups", ctypes.c_int32)]


class MpcError(RuntimeError):
    def __init__(self, fn, status, msg):
        super().__init__(f"{fn}: status {status} ({msg})")
        self.status = status


_LIB = None
EXPORTS = ("mpc_workspace_bytes", "mpc_static_evict", "mpc_static_evict_noalloc", "mpc_static_evict_noalloc_limit",
           "mpc_build_clusters", "mpc_prefill", "mpc_select_clusters",
           "mpc_sparse_decode_attn", "mpc_decode_step", "mpc_decode_step_status", "mpc_append_kv", "mpc_commonality",
           "mpc_paged_append", "mpc_paged_read", "mpc_paged_attn", "mpc_shared_attn", "mpc_prompt_attn", "mpc_owner_layer",
           "mpc_status_string", "mpc_last_error")


def lib():
    """Loads libmpcache.so; raises if it has not been built (no fallback path exists)."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
        L = ctypes.CDLL(LIB_PATH)
        P, V, I, F = ctypes.POINTER, ctypes.c_void_p, ctypes.c_int32, ctypes.c_float
        L.mpc_workspace_bytes.argtypes = [I, P(MpcDims), I, V]
        L.mpc_workspace_bytes.restype = ctypes.c_size_t
        L.mpc_static_evict.argtypes = [P(MpcDims), I, P(MpcEvictCfg)] + [V] * 8 + [V, ctypes.c_size_t, V]
        L.mpc_static_evict_noalloc.argtypes = [P(MpcDims), I, P(MpcEvictCfg)] + [V] * 8 + [V]
        L.mpc_static_evict_noalloc.restype = ctypes.c_int
        L.mpc_static_evict_noalloc_limit.argtypes = []
        L.mpc_static_evict_noalloc_limit.restype = ctypes.c_size_t
        L.mpc_build_clusters.argtypes = [P(MpcDims), I, P(MpcSelectCfg), V, V, V, V]
        L.mpc_prefill.argtypes = [P(MpcDims), I, P(MpcEvictCfg), P(MpcSelectCfg)] + [V] * 10 + [V, ctypes.c_size_t, V]
        L.mpc_select_clusters.argtypes = [P(MpcDims), I, P(MpcSelectCfg)] + [V] * 5 + [V, ctypes.c_size_t, V]
        L.mpc_sparse_decode_attn.argtypes = [P(MpcDims), I, I, I, V, V, V, V, I, I, F, V, V, V, ctypes.c_size_t, V]
        L.mpc_decode_step.argtypes = [P(MpcDims), I, I, P(MpcSelectCfg)] + [V] * 5 + [F] + [V] * 4 + [
            V, ctypes.c_size_t, V]
        L.mpc_append_kv.argtypes = [P(MpcDims), I, I, P(MpcSelectCfg)] + [V] * 6 + [P(I), P(I), V]
        L.mpc_decode_step_status.argtypes = [V, ctypes.c_size_t, I, P(I)]
        L.mpc_commonality.argtypes = [I, I, I, I, V, V, V]
        KV, S, A = P(MpcPagedKv), P(MpcStrides), P(MpcAttnCfg)
        L.mpc_paged_append.argtypes = [P(MpcDims), KV, I, V, P(MpcRope), V] + [V, S] * 5 + [V]
        L.mpc_paged_read.argtypes = [P(MpcDims), KV, I, V, V] + [V, S] * 2 + [V]
        L.mpc_paged_attn.argtypes = [P(MpcDims), KV, I, V, A] + [V, S] * 2 + [V, V, ctypes.c_size_t, V]
        L.mpc_shared_attn.argtypes = [P(MpcDims), KV, I, V, P(MpcShared), A] + [V, S] * 2 + [V, V, ctypes.c_size_t, V]
        L.mpc_prompt_attn.argtypes = [P(MpcDims), I, I, V, V, A] + [V, S] * 4 + [V, V]
        for fn in ("mpc_paged_append", "mpc_paged_read", "mpc_paged_attn", "mpc_shared_attn", "mpc_prompt_attn", "mpc_static_evict", "mpc_build_clusters", "mpc_prefill", "mpc_select_clusters", "mpc_sparse_decode_attn",
                   "mpc_decode_step", "mpc_decode_step_status", "mpc_append_kv", "mpc_commonality"):
            getattr(L, fn).restype = ctypes.c_int
        L.mpc_owner_layer.argtypes = [I, I, I]
        L.mpc_owner_layer.restype = I
        L.mpc_status_string.argtypes = [ctypes.c_int]
        L.mpc_status_string.restype = ctypes.c_char_p
        L.mpc_last_error.argtypes = []
        L.mpc_last_error.restype = ctypes.c_char_p
        _LIB = L
    return _LIB


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _check(fn, status):
    if status != MPC_OK:
        raise MpcError(fn, status, lib().mpc_last_error().decode())


def dims_of(q_like, kv, layer0=0):
    """mpc_dims from a query-like tensor [L][B][Hq][..][d] and a cache [L][B][Hkv][Tcap][d]; the
    cache's row axis is its capacity."""
    if kv.dtype not in DTYPE_CODE:
        raise TypeError(f"unsupported dtype {kv.dtype}")
    cap = kv.shape[3] if kv.dim() == 5 else 0
    return MpcDims(batch=kv.shape[1], layer0=layer0, n_layers=kv.shape[0], n_q_heads=q_like.shape[2],
                   n_kv_heads=kv.shape[2], head_dim=kv.shape[-1], dtype=DTYPE_CODE[kv.dtype], kv_capacity=cap)


def _contig(*ts):
    for t in ts:
        if t is not None and not (t.is_cuda and t.is_contiguous()):
            raise ValueError("tensors must be contiguous CUDA tensors")


def owner_layer(layer, period, start=2):
    return lib().mpc_owner_layer(layer, period, start)


def workspace_bytes(op, dims, T_or_Ts, cfg=None):
    c = None if cfg is None else ctypes.byref(cfg)
    return lib().mpc_workspace_bytes(op, ctypes.byref(dims), T_or_Ts, c)


def workspace(nbytes, device="cuda"):
    """A zero-filled workspace buffer (the counters in it must start at zero)."""
    return torch.zeros(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def _call_ws(nbytes, device, stream):
    """The workspace of one call that was given none, made and cleared on the stream that the call runs on: the zeros come
    before its kernels, and the memory goes back to the allocator in that stream's order."""
    if stream is None:
        return workspace(nbytes, device)
    with torch.cuda.stream(stream):
        return workspace(nbytes, device)


def mpc_static_evict(q_win, k, v, kept_idx, k_out, v_out, *, keep, local_keep, sm_scale, causal=True,
                     layer0=0, share_period=1, share_start=2, token_score=None, row_lse=None, ws=None,
                     stream=None):
    """q_win [L][B][Hq][W][d], k/v [L][B][Hkv][T][d] -> kept_idx [L][B][Hkv][keep], k_out/v_out."""
    _contig(q_win, k, v, kept_idx, k_out, v_out, token_score, row_lse, ws)
    dims = dims_of(q_win, k, layer0)
    dims.kv_capacity = k_out.shape[3]
    T, W = k.shape[3], q_win.shape[3]
    cfg = MpcEvictCfg(window=W, keep=keep, local_keep=local_keep, sm_scale=sm_scale, causal=int(causal),
                      share_period=share_period, share_start=share_start)
    if ws is None:
        ws = _call_ws(workspace_bytes(MPC_OP_STATIC_EVICT, dims, T, cfg), k.device, stream)
    _check("mpc_static_evict", lib().mpc_static_evict(
        ctypes.byref(dims), T, ctypes.byref(cfg), _ptr(q_win), _ptr(k), _ptr(v), _ptr(kept_idx), _ptr(k_out),
        _ptr(v_out), _ptr(token_score), _ptr(row_lse), _ptr(ws), ws.numel(), _stream(stream)))


def mpc_static_evict_noalloc(q_win, k, v, kept_idx, k_out, v_out, *, keep, local_keep, sm_scale, causal=True,
                             layer0=0, share_period=1, share_start=2, token_score=None, row_lse=None, stream=None):
    """mpc_static_evict with the library's static scratch array as its workspace (nothing is
    allocated); fails with MpcError (MPC_EWORKSPACE) when the block needs more than
    noalloc_limit() scratch bytes."""
    _contig(q_win, k, v, kept_idx, k_out, v_out, token_score, row_lse)
    dims = dims_of(q_win, k, layer0)
    dims.kv_capacity = k_out.shape[3]
    T, W = k.shape[3], q_win.shape[3]
    cfg = MpcEvictCfg(window=W, keep=keep, local_keep=local_keep, sm_scale=sm_scale, causal=int(causal),
                      share_period=share_period, share_start=share_start)
    _check("mpc_static_evict_noalloc", lib().mpc_static_evict_noalloc(
        ctypes.byref(dims), T, ctypes.byref(cfg), _ptr(q_win), _ptr(k), _ptr(v), _ptr(kept_idx), _ptr(k_out),
        _ptr(v_out), _ptr(token_score), _ptr(row_lse), _stream(stream)))


def noalloc_limit():
    """Bytes of the static scratch array behind mpc_static_evict_noalloc."""
    return lib().mpc_static_evict_noalloc_limit()


SIMILARITY = {"linear": 0, "maxprod": 1, "mean": 2}
GROUP = {"sum": 0, "max": 1, "head": 2}


def rep_rows(similarity):
    """Rows of d floats per cluster representative (r^max and r^min for the max-product bound)."""
    return 2 if SIMILARITY[similarity] == 1 else 1


def select_cfg(cluster, fanout, k_super, k_clusters, alpha=0.6, share_period=1, share_start=2,
               similarity="linear", group="sum"):
    """group: "sum" / "max" (the q-heads of a kv head share one selection scored by the sum / the
    maximum of their similarities) or "head" (one selection per q-head)."""
    return MpcSelectCfg(cluster_size=cluster, fanout=fanout, k_super=k_super, k_clusters=k_clusters,
                        alpha=alpha, share_period=share_period, share_start=share_start,
                        similarity=SIMILARITY[similarity], group=GROUP[group])


def sel_heads(cfg, n_q_heads, n_kv_heads):
    """Selection lists per (layer, sequence) under the config's group rule."""
    return n_q_heads if cfg.group == GROUP["head"] else n_kv_heads


def _slots(cap, cfg):
    C = -(-cap // cfg.cluster_size)
    return C, -(-C // cfg.fanout)


def mpc_build_clusters(k_cache, cent, scent, cfg, *, Ts=None, layer0=0, stream=None):
    """k_cache [L][B][Hkv][Tcap][d] (rows [0, Ts) used, Ts = Tcap by default) -> cent
    [L][B][Hkv][Ccap][R][d], scent [L][B][Hkv][Scap][R][d] (float32; R = 2 rows r^max, r^min for the
    max-product bound, else 1 and the R axis may be omitted)."""
    _contig(k_cache, cent, scent)
    dims = dims_of(k_cache, k_cache, layer0)
    Ts = k_cache.shape[3] if Ts is None else Ts
    _check_reps(k_cache, cent, scent, cfg)
    _check("mpc_build_clusters", lib().mpc_build_clusters(
        ctypes.byref(dims), Ts, ctypes.byref(cfg), _ptr(k_cache), _ptr(cent), _ptr(scent), _stream(stream)))


def _check_reps(k_cache, cent, scent, cfg):
    L, B, Hkv, cap, d = k_cache.shape
    C, S = _slots(cap, cfg)
    R = 2 if cfg.similarity == SIMILARITY["maxprod"] else 1
    if cent.numel() != L * B * Hkv * C * R * d or scent.numel() != L * B * Hkv * S * R * d:
        raise ValueError(f"cent / scent must hold [L][B][Hkv][C or S][{R}][d] floats")
    if cent.dtype != torch.float32 or scent.dtype != torch.float32:
        raise TypeError("cent / scent must be float32")


def mpc_prefill(q_win, k, v, kept_idx, k_out, v_out, cent, scent, cfg, *, keep, local_keep, sm_scale, causal=True,
                layer0=0, share_period=1, share_start=2, token_score=None, row_lse=None, ws=None, stream=None):
    """mpc_static_evict then mpc_build_clusters over the kept rows (Ts = keep) in one call, with the
    selection owners' rows gathered inside the build; the eviction's sharing rule is
    share_period / share_start, the representatives' that of cfg."""
    _contig(q_win, k, v, kept_idx, k_out, v_out, cent, scent, token_score, row_lse, ws)
    _check_reps(k_out, cent, scent, cfg)
    dims = dims_of(q_win, k, layer0)
    dims.kv_capacity = k_out.shape[3]
    T, W = k.shape[3], q_win.shape[3]
    ecfg = MpcEvictCfg(window=W, keep=keep, local_keep=local_keep, sm_scale=sm_scale, causal=int(causal),
                       share_period=share_period, share_start=share_start)
    if ws is None:
        ws = _call_ws(workspace_bytes(MPC_OP_STATIC_EVICT, dims, T, ecfg), k.device, stream)
    _check("mpc_prefill", lib().mpc_prefill(
        ctypes.byref(dims), T, ctypes.byref(ecfg), ctypes.byref(cfg), _ptr(q_win), _ptr(k), _ptr(v), _ptr(kept_idx),
        _ptr(k_out), _ptr(v_out), _ptr(cent), _ptr(scent), _ptr(token_score), _ptr(row_lse), _ptr(ws), ws.numel(),
        _stream(stream)))


def mpc_select_clusters(q, cent, scent, sel, cfg, *, Ts, sel_score=None, layer0=0, stream=None):
    """q [L][B][Hq][d], cent / scent with Ccap / Scap slots (the first ceil(Ts / s) used) ->
    sel [L][B][H][k_clusters] (int32, ascending), H = Hq for the "head" group rule, else Hkv."""
    _contig(q, cent, scent, sel, sel_score)
    dims = dims_of(q, cent, layer0)
    dims.head_dim = q.shape[-1]
    dims.dtype = DTYPE_CODE[q.dtype]
    dims.kv_capacity = cent.shape[3] * cfg.cluster_size
    if scent.shape[3] != _slots(dims.kv_capacity, cfg)[1]:
        raise ValueError("scent must have ceil(Ccap / fanout) super-cluster slots")
    if sel.shape[2] != sel_heads(cfg, q.shape[2], cent.shape[2]):
        raise ValueError("sel must have one list per q-head for the head rule, per kv head otherwise")
    _check("mpc_select_clusters", lib().mpc_select_clusters(
        ctypes.byref(dims), Ts, ctypes.byref(cfg), _ptr(q), _ptr(cent), _ptr(scent), _ptr(sel), _ptr(sel_score),
        None, 0, _stream(stream)))


def mpc_sparse_decode_attn(q, k_cache, v_cache, sel, out, *, cluster_size, sm_scale, Ts=None, n_tail=0, lse=None,
                           ws=None, layer0=0, stream=None):
    """q [L][B][Hq][d], k/v [L][B][Hkv][Tcap][d], sel [L][B][H][k] (H = Hkv: one list per kv head;
    H = Hq: one per q-head) -> out [L][B][Hq][d]. Clustered rows [0, Ts) (Ts = Tcap - n_tail by
    default) and tail rows [Ts, Ts + n_tail)."""
    _contig(q, k_cache, v_cache, sel, out, lse, ws)
    dims = dims_of(q, k_cache, layer0)
    Ts = k_cache.shape[3] - n_tail if Ts is None else Ts
    if ws is None:
        ws = _call_ws(workspace_bytes(MPC_OP_DECODE_ATTN, dims, Ts), q.device, stream)
    _check("mpc_sparse_decode_attn", lib().mpc_sparse_decode_attn(
        ctypes.byref(dims), Ts, n_tail, cluster_size, _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(sel), sel.shape[2],
        sel.shape[-1], sm_scale, _ptr(out), _ptr(lse), _ptr(ws), ws.numel(), _stream(stream)))


def mpc_decode_step(q, cent, scent, k_cache, v_cache, sel, out, cfg, *, sm_scale, Ts=None, n_tail=0, sel_score=None,
                    lse=None, ws=None, layer0=0, stream=None):
    """Selection of every owner head then sparse attention of every head, in one call.

    q [L][B][Hq][d], cent/scent as built, k/v [L][B][Hkv][Tcap][d] (clustered rows [0, Ts), Ts = Tcap - n_tail
    by default, then the tail) -> sel [L][B][H][k] (H as for mpc_select_clusters), out [L][B][Hq][d].
    ws must come from workspace() (zero-filled) and be reused by later calls of the same shape.
    """
    _contig(q, cent, scent, k_cache, v_cache, sel, out, sel_score, lse, ws)
    dims = dims_of(q, k_cache, layer0)
    Ts = k_cache.shape[3] - n_tail if Ts is None else Ts
    if ws is None:
        ws = _call_ws(workspace_bytes(MPC_OP_DECODE_STEP, dims, Ts, cfg), q.device, stream)
    _check("mpc_decode_step", lib().mpc_decode_step(
        ctypes.byref(dims), Ts, n_tail, ctypes.byref(cfg), _ptr(q), _ptr(cent), _ptr(scent), _ptr(k_cache), _ptr(v_cache),
        sm_scale, _ptr(sel), _ptr(sel_score), _ptr(out), _ptr(lse), _ptr(ws), ws.numel(), _stream(stream)))
    return ws


def mpc_commonality(idx, out, m, stream=None):
    """idx [L][...][k] int32 top-k sets per layer -> out [...] float64: commonality score of m + 1
    adjacent layers (Sec. 3, Observation 3) for every unit of the middle axes."""
    _contig(idx, out)
    if idx.dtype != torch.int32 or out.dtype != torch.float64:
        raise TypeError("idx must be int32 and out float64")
    L, k = idx.shape[0], idx.shape[-1]
    units = idx[0, ..., 0].numel()
    if out.numel() != units:
        raise ValueError("out must hold one value per unit")
    _check("mpc_commonality", lib().mpc_commonality(L, units, k, m, _ptr(idx), _ptr(out), _stream(stream)))


def mpc_append_kv(k_new, v_new, k_cache, v_cache, cent, scent, cfg, *, Ts, n_tail, layer0=0, stream=None):
    """Appends one decoded token: k_new / v_new [L][B][Hkv][d] into k/v [L][B][Hkv][Tcap][d] (sealing a full
    tail into a cluster, whose representatives in cent / scent are rebuilt). Returns the new (Ts, n_tail)."""
    _contig(k_new, v_new, k_cache, v_cache, cent, scent)
    dims = dims_of(k_cache, k_cache, layer0)
    if k_new.shape != k_cache.shape[:3] + k_cache.shape[4:] or v_new.shape != k_new.shape:
        raise ValueError("k_new / v_new must be [L][B][Hkv][d] like the cache")
    if k_new.dtype != k_cache.dtype or v_new.dtype != k_cache.dtype or v_cache.dtype != k_cache.dtype:
        raise TypeError("k_new / v_new / v_cache must have the cache's dtype")
    C, S = _slots(k_cache.shape[3], cfg)
    if cent.shape[3] != C or scent.shape[3] != S:
        raise ValueError(f"cent / scent must have {C} / {S} slots for a capacity of {k_cache.shape[3]} rows")
    ts_out, tail_out = ctypes.c_int32(), ctypes.c_int32()
    _check("mpc_append_kv", lib().mpc_append_kv(
        ctypes.byref(dims), Ts, n_tail, ctypes.byref(cfg), _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache),
        _ptr(cent), _ptr(scent), ctypes.byref(ts_out), ctypes.byref(tail_out), _stream(stream)))
    return ts_out.value, tail_out.value


def mpc_decode_step_status(ws, clear=False):
    """Error word of a decode-step workspace (bit 0: a unit gave up waiting for its selection and
    wrote NaN outputs); blocking, call after the steps' stream has completed."""
    _contig(ws)
    flags = ctypes.c_int32()
    _check("mpc_decode_step_status", lib().mpc_decode_step_status(_ptr(ws), ws.numel() * ws.element_size(),
                                                                  int(bool(clear)), ctypes.byref(flags)))
    return flags.value


ROPE_STYLE = {"interleaved": 0, "half": 1}
PAGE_FORMAT = {"same": 0, "e4m3": 1, "mx4": 4}
MX4_BLOCK = 32  # channels to a scale of 4-bit codes


def _rows(t, what, dtype, heads=None):
    """A tensor [L][B][H][n][d] (or [L][B][H][d], n = 1): (pointer, strides or None where contiguous, shape). The last axis
    must have stride 1; the other strides are the caller's."""
    if t.dim() == 4:
        t = t.unsqueeze(3)
    if t.dim() != 5 or not t.is_cuda or t.dtype is not dtype:
        raise ValueError(f"{what} must be a CUDA tensor [L][B][H][n][d] of type {dtype}")
    shape = t.shape
    if heads is not None and shape[2] != heads:
        raise ValueError(f"{what} must have {heads} heads")
    if t.is_contiguous():
        return t.data_ptr(), None, shape
    if t.stride(4) != 1:
        raise ValueError(f"{what}: the channels of a row must be contiguous")
    return t.data_ptr(), ctypes.byref(MpcStrides(*t.stride()[:4])), shape


def _placed(t, what, written=False):
    """Refuses the address and strides that the library would refuse: off 16 bytes, or of rows that are written and overlap."""
    size = t.element_size()
    if t.data_ptr() % 16:
        raise ValueError(f"{what} must be 16-byte aligned")
    if t.is_contiguous():
        return
    axes = sorted((s, n) for s, n in zip(t.stride()[:-1], t.shape[:-1]) if n > 1)
    if any(s * size % 16 for s, _ in axes):
        raise ValueError(f"{what}: strides must be whole numbers of 16 bytes")
    span = t.shape[-1]  # elements from the first to behind the last of the axes so far
    for s, n in axes if written else ():
        if s < span:
            raise ValueError(f"{what}: rows that are written overlap")
        span += (n - 1) * s


def _rope_of(rope):
    """(pointer, positions, rotated channels) of a rotary table."""
    if rope.dtype != torch.float32 or rope.dim() != 3 or rope.shape[2] != 2 or not rope.is_contiguous():
        raise ValueError("rope must be contiguous float32 [n_pos][rot_dim / 2][2]")
    return rope.data_ptr(), rope.shape[0], 2 * rope.shape[1]


def _batch_ints(t, what, B, device):
    if t is None:
        return None
    if t.dtype is not torch.int32 or t.shape != (B,) or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{what} must be a contiguous int32 tensor [{B}] on {device}")
    return t.data_ptr()


def _on(device, stream, *tensors):
    """The stream of a call on `device` (its current one by default); every tensor has to lie there."""
    for t in tensors:
        if t is not None and t.device != device:
            raise ValueError(f"a tensor on {t.device} in a call on {device}")
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device.index)  # (current_stream() without its object)
    if stream.device != device:
        raise ValueError(f"a stream of {stream.device} in a call on {device}")
    return stream.cuda_stream


def _call(name, fn, device, *args):
    """One library call with `device` as the current one, which its launches go to."""
    if device.index == torch._C._cuda_getDevice():
        status = fn(*args)
    else:
        with torch.cuda.device(device):
            status = fn(*args)
    if status != MPC_OK:
        _check(name, status)


class PagedKV:
    """A paged cache over the caller's tensors, as the mpc_paged_* calls and mpc_shared_attn take it.

    k_pages, v_pages [L][P][Hkv][page][d] of the element type, or torch.float8_e4m3fn codes with k_scale, v_scale
    [L][P][Hkv] float32 and the rings k_tail, v_tail [L][B][Hkv][2 page][d] of the element type, or torch.uint8 [L][P][Hkv]
    [page][d / 2], two 4-bit codes to a byte, with k_scale, v_scale torch.uint8 [L][P][Hkv][d / 32][page]; table [B][M] int32
    page ids; lens [B] int32, rows of each sequence with those of the next call's new tokens. dtype: the element type, which
    4-bit pages do not tell. The tables and lengths live on the device: a caller writes them there, and a captured graph reads
    what they hold at its replay."""

    def __init__(self, k_pages, v_pages, table, lens, *, k_scale=None, v_scale=None, k_tail=None, v_tail=None, dtype=None):
        codes, codes4 = k_pages.dtype == torch.float8_e4m3fn, k_pages.dtype == torch.uint8
        extra = (k_scale, v_scale, k_tail, v_tail)
        if codes4:
            if k_scale is None or v_scale is None or k_tail is not None or v_tail is not None:
                raise ValueError("4-bit pages have scales and no tails")
        elif codes != all(t is not None for t in extra) or (not codes and any(t is not None for t in extra)):
            raise ValueError("scales and tails belong to float8_e4m3fn pages, all four of them")
        _contig(k_pages, v_pages, table, lens, *extra)
        if k_pages.dim() != 5 or v_pages.shape != k_pages.shape or v_pages.dtype != k_pages.dtype:
            raise ValueError("k_pages and v_pages must be alike, [L][P][Hkv][page][d]")
        self.L, P, self.Hkv, self.page, self.d = k_pages.shape
        self.dtype = dtype if codes4 else k_tail.dtype if codes else k_pages.dtype
        if self.dtype not in DTYPE_CODE:
            raise TypeError(f"unsupported dtype {self.dtype}")
        if dtype is not None and dtype != self.dtype:
            raise TypeError(f"the cache's element type is {self.dtype}")
        if codes4:
            self.d *= 2
            if any(t.dtype != torch.uint8 or t.shape != (self.L, P, self.Hkv, self.d // MX4_BLOCK, self.page) for t in (k_scale, v_scale)):
                raise ValueError("k_scale and v_scale must be uint8 [L][P][Hkv][d / 32][page]")
        if table.dtype != torch.int32 or table.dim() != 2 or lens.dtype != torch.int32 or lens.shape != table.shape[:1]:
            raise ValueError("table must be int32 [B][M] and lens int32 [B]")
        self.B, M = table.shape
        if codes:
            ring = (self.L, self.B, self.Hkv, 2 * self.page, self.d)
            if k_tail.shape != ring or v_tail.shape != ring or v_tail.dtype != k_tail.dtype:
                raise ValueError(f"k_tail and v_tail must be alike, {list(ring)}")
            if any(t.shape != k_pages.shape[:3] or t.dtype != torch.float32 for t in (k_scale, v_scale)):
                raise ValueError("k_scale and v_scale must be float32 [L][P][Hkv]")
        self.device = k_pages.device
        if any(t is not None and t.device != self.device for t in (v_pages, table, lens) + extra):
            raise ValueError("the cache's tensors must lie on one device")
        self.k_pages, self.v_pages, self.table, self.lens = k_pages, v_pages, table, lens
        self.k_scale, self.v_scale, self.k_tail, self.v_tail = extra
        p = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        self.c = MpcPagedKv(self.page, P, M, PAGE_FORMAT["mx4" if codes4 else "e4m3" if codes else "same"], p(k_pages), p(v_pages), p(k_scale),
                            p(v_scale), p(k_tail), p(v_tail), p(table), p(lens))
        self.ref = ctypes.byref(self.c)
        self._dims = {}

    def dims(self, n_q_heads):
        """The mpc_dims (as an argument) of a call with that many query heads."""
        if n_q_heads not in self._dims:
            self._dims[n_q_heads] = ctypes.byref(MpcDims(self.B, 0, self.L, n_q_heads, self.Hkv, self.d, DTYPE_CODE[self.dtype], 0))
        return self._dims[n_q_heads]


def _page_format(fmt, fp8):
    if fmt is None:
        return "e4m3" if fp8 else "same"
    if fmt not in PAGE_FORMAT or (fp8 and fmt != "e4m3"):
        raise ValueError(f"the page format must be one of {list(PAGE_FORMAT)}, and \"e4m3\" with fp8")
    return fmt


def paged_kv(*, n_layers, batch, n_kv_heads, head_dim, dtype, n_pages, max_pages, page_size=64, fp8=False, fmt=None, device="cuda"):
    """An empty PagedKV: table entries -1 (no page), lengths 0. fmt: the pages' format, "same" (as the element type), "e4m3" or
    "mx4"; fp8 is another way to say "e4m3"."""
    fmt = _page_format(fmt, fp8)
    dev = torch.device(device)
    new = lambda t, *shape: torch.zeros(shape, dtype=t, device=dev)  # noqa: E731
    pool = (n_layers, n_pages, n_kv_heads, page_size, head_dim)
    ring = (n_layers, batch, n_kv_heads, 2 * page_size, head_dim)
    table = torch.full((batch, max_pages), -1, dtype=torch.int32, device=dev)
    if fmt == "mx4":
        pool, scales = pool[:4] + (head_dim // 2,), pool[:3] + (head_dim // MX4_BLOCK, page_size)
        return PagedKV(new(torch.uint8, *pool), new(torch.uint8, *pool), table, new(torch.int32, batch),
                       k_scale=new(torch.uint8, *scales), v_scale=new(torch.uint8, *scales), dtype=dtype)
    extra = {}
    if fmt == "e4m3":
        extra = dict(k_scale=new(torch.float32, *pool[:3]), v_scale=new(torch.float32, *pool[:3]), k_tail=new(dtype, *ring),
                     v_tail=new(dtype, *ring))
    t = torch.float8_e4m3fn if fmt == "e4m3" else dtype
    return PagedKV(new(t, *pool), new(t, *pool), table, new(torch.int32, batch), **extra)


def _like(shape, kv, n, what):
    if shape[0] != kv.L or shape[1] != kv.B or shape[3] != n or shape[4] != kv.d:
        raise ValueError(f"{what} must be [{kv.L}][{kv.B}][H][{n}][{kv.d}]")


def mpc_paged_append(k, v, kv, *, q=None, q_out=None, k_out=None, rope=None, rope_style="interleaved", pos0=None,
                     n_valid=None, stream=None):
    """k, v [L][B][Hkv][n][d] (or [L][B][Hkv][d]), any strides, into the cache `kv` at the rows before kv.lens. rope
    [n_pos][rot_dim / 2][2] float32 (cos, sin) rotates K, and q [L][B][Hq][n][d] into q_out (q itself by default), by the
    positions pos0 [B] + t (the row numbers by default); k_out (shaped like k) also receives K's rows as the cache takes
    them. n_valid [B]: new tokens of each sequence (n by default)."""
    kp, ks, shape = _rows(k, "k", kv.dtype, kv.Hkv)
    n = shape[3]
    _like(shape, kv, n, "k")
    vp, vs, shape = _rows(v, "v", kv.dtype, kv.Hkv)
    _like(shape, kv, n, "v")
    Hq, qp, qs, op, os_, r = kv.Hkv, None, None, None, None, None
    if rope is not None:
        r = ctypes.byref(MpcRope(*_rope_of(rope), ROPE_STYLE[rope_style]))
    if q is not None:
        q_out = q if q_out is None else q_out
        qp, qs, shape = _rows(q, "q", kv.dtype)
        Hq = shape[2]
        _like(shape, kv, n, "q")
        op, os_, shape = _rows(q_out, "q_out", kv.dtype, Hq)
        _like(shape, kv, n, "q_out")
    elif q_out is not None:
        raise ValueError("q_out is given without q")
    kop = kos = None
    if k_out is not None:
        kop, kos, shape = _rows(k_out, "k_out", kv.dtype, kv.Hkv)
        _like(shape, kv, n, "k_out")
    st = _on(kv.device, stream, k, v, q, q_out, k_out, rope)
    _call("mpc_paged_append", lib().mpc_paged_append, kv.device, kv.dims(Hq), kv.ref, n, _batch_ints(n_valid, "n_valid", kv.B, kv.device),
          r, _batch_ints(pos0, "pos0", kv.B, kv.device), kp, ks, vp, vs, qp, qs, op, os_, kop, kos, st)


def mpc_paged_read(kv, k_out=None, v_out=None, *, first=None, n_valid=None, stream=None):
    """Rows of the cache `kv`, in the element type, into k_out, v_out [L][B][Hkv][n][d] (or [L][B][Hkv][d], any strides; either may be
    None): row t < n_valid[b] (n by default) of sequence b is row first[b] + t of the cache (the newest n_valid[b] rows by
    default). Rows that the cache does not have are left as they were."""
    out = [(t, what, _rows(t, what, kv.dtype, kv.Hkv)) for t, what in ((k_out, "k_out"), (v_out, "v_out")) if t is not None]
    if not out:
        raise ValueError("neither k_out nor v_out is given")
    n = out[0][2][2][3]
    for _, what, (_, _, shape) in out:
        _like(shape, kv, n, what)
    args = [x for t in (k_out, v_out) for x in ((None, None) if t is None else next(r[:2] for u, _, r in out if u is t))]
    st = _on(kv.device, stream, k_out, v_out)
    _call("mpc_paged_read", lib().mpc_paged_read, kv.device, kv.dims(kv.Hkv), kv.ref, n, _batch_ints(n_valid, "n_valid", kv.B, kv.device),
          _batch_ints(first, "first", kv.B, kv.device), *args, st)


def paged_attn_workspace_bytes(q, kv):
    """Workspace bytes of mpc_paged_attn for queries shaped like q [L][B][Hq][n][d] (or [L][B][Hq][d])."""
    return lib().mpc_workspace_bytes(MPC_OP_PAGED_ATTN, kv.dims(q.shape[2]), q.shape[3] if q.dim() == 5 else 1,
                                     kv.ref)


def _attn_cfg(sm_scale, window, sinks):
    for what, x in (("window", window), ("sinks", sinks)):
        if not -2 ** 31 <= x < 2 ** 31:  # (a field would keep the lower 32 bits)
            raise ValueError(f"{what} {x} does not fit 32 bits")
    return MpcAttnCfg(sm_scale, window, sinks)


def _lse_of(lse, shape):
    if lse is None:
        return None
    if lse.dtype != torch.float32 or not lse.is_contiguous() or lse.numel() != shape[0] * shape[1] * shape[2] * shape[3]:
        raise ValueError("lse must be contiguous float32 [L][B][Hq][n]")
    return lse.data_ptr()


def mpc_paged_attn(q, kv, out, *, sm_scale, window=0, sinks=0, n_valid=None, lse=None, ws=None, stream=None):
    """Attention of the newest tokens' queries q [L][B][Hq][n][d] (or [L][B][Hq][d]) over the cache `kv`, which holds their
    keys and values already -> out (shaped like q), lse [L][B][Hq][n] float32. window, sinks: a row at position p sees
    the rows j <= p with j > p - window (0: all) or j < sinks. ws: from workspace(paged_attn_workspace_bytes(q, kv)),
    reused by later calls of any shape that needs no more bytes (made for the call by default)."""
    qp, qs, shape = _rows(q, "q", kv.dtype)
    n = shape[3]
    _like(shape, kv, n, "q")
    op, os_, oshape = _rows(out, "out", kv.dtype, shape[2])
    _like(oshape, kv, n, "out")
    if ws is None:
        ws = _call_ws(paged_attn_workspace_bytes(q, kv), kv.device, stream)
    _contig(ws)
    st = _on(kv.device, stream, q, out, lse, ws)
    cfg = _attn_cfg(sm_scale, window, sinks)
    _call("mpc_paged_attn", lib().mpc_paged_attn, kv.device, kv.dims(shape[2]), kv.ref, n,
          _batch_ints(n_valid, "n_valid", kv.B, kv.device), ctypes.byref(cfg), qp, qs, op, os_, _lse_of(lse, shape),
          ws.data_ptr(), ws.numel() * ws.element_size(), st)


def shared_attn_workspace_bytes(q, kv, n_groups):
    """Workspace bytes of mpc_shared_attn for queries shaped like q [L][B][Hq][n][d] (or [L][B][Hq][d]) and that many groups."""
    sizes = MpcSharedSizes(ctypes.pointer(kv.c), n_groups)
    return lib().mpc_workspace_bytes(MPC_OP_SHARED_ATTN, kv.dims(q.shape[2]), q.shape[3] if q.dim() == 5 else 1, ctypes.byref(sizes))


def mpc_shared_attn(q, kv, out, *, first, shared_rows, sm_scale, window=0, sinks=0, n_valid=None, lse=None, ws=None, stream=None):
    """mpc_paged_attn for sequences that share their first rows, in groups of neighbours: group g is the sequences first[g] <= b <
    first[g + 1] (int32 [n_groups + 1] on the device), and their first shared_rows[g] rows (int32 [n_groups]; whole pages of them)
    are read once for all of them, from the pages of the group's first sequence. ws: from
    workspace(shared_attn_workspace_bytes(q, kv, n_groups)); it serves mpc_paged_attn too."""
    qp, qs, shape = _rows(q, "q", kv.dtype)
    n = shape[3]
    _like(shape, kv, n, "q")
    op, os_, oshape = _rows(out, "out", kv.dtype, shape[2])
    _like(oshape, kv, n, "out")
    if shared_rows.dim() != 1 or shared_rows.numel() == 0:
        raise ValueError("shared_rows must be int32 [n_groups]")
    ng = shared_rows.numel()
    groups = MpcShared(ng, _batch_ints(first, "first", ng + 1, kv.device), _batch_ints(shared_rows, "shared_rows", ng, kv.device))
    if ws is None:
        ws = _call_ws(shared_attn_workspace_bytes(q, kv, ng), kv.device, stream)
    _contig(ws)
    st = _on(kv.device, stream, q, out, lse, ws)
    cfg = _attn_cfg(sm_scale, window, sinks)
    _call("mpc_shared_attn", lib().mpc_shared_attn, kv.device, kv.dims(shape[2]), kv.ref, n,
          _batch_ints(n_valid, "n_valid", kv.B, kv.device), ctypes.byref(groups), ctypes.byref(cfg), qp, qs, op, os_,
          _lse_of(lse, shape), ws.data_ptr(), ws.numel() * ws.element_size(), st)


def mpc_prompt_attn(q, k, v, out, *, sm_scale, window=0, sinks=0, q_lens=None, k_lens=None, lse=None, stream=None):
    """Attention of a prompt's rows q [L][B][Hq][Tq][d] over its keys k, v [L][B][Hkv][T][d] (any strides) -> out (shaped like
    q), lse [L][B][Hq][Tq] float32: row t of sequence b stands at position k_lens[b] - q_lens[b] + t (T, Tq by default);
    window, sinks as in mpc_paged_attn."""
    if q.dtype not in DTYPE_CODE:
        raise TypeError(f"unsupported dtype {q.dtype}")
    if q.dim() != 5 or k.dim() != 5:
        raise ValueError("q, k, v and out must be [L][B][H][n][d]")
    qp, qs, shape = _rows(q, "q", q.dtype)
    op, os_, oshape = _rows(out, "out", q.dtype)
    kp, ks, kshape = _rows(k, "k", q.dtype)
    vp, vs, vshape = _rows(v, "v", q.dtype)
    if oshape != shape or vshape != kshape or kshape[:2] != shape[:2] or kshape[4] != shape[4]:
        raise ValueError("out must be shaped like q, and k and v like q but for their heads and rows")
    L, B, Hq, Tq, d = shape
    dev = q.device
    st = _on(dev, stream, k, v, out, lse)
    dims = MpcDims(B, 0, L, Hq, kshape[2], d, DTYPE_CODE[q.dtype], 0)
    cfg = _attn_cfg(sm_scale, window, sinks)
    _call("mpc_prompt_attn", lib().mpc_prompt_attn, dev, ctypes.byref(dims), Tq, kshape[3], _batch_ints(q_lens, "q_lens", B, dev),
          _batch_ints(k_lens, "k_lens", B, dev), ctypes.byref(cfg), qp, qs, kp, ks, vp, vs, op, os_, _lse_of(lse, shape), st)
