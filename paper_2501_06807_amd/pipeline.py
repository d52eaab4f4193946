"""Preallocated prefill + decode paths over the C-ABI entry points: the kept cache of the method, and a paged cache."""
import ctypes
import math
import operator

import torch

from . import _lib as L


class MPCachePath:
    """Buffers and calls for one workload: static eviction and cluster build at prefill, then
    selection + sparse attention for every decode step, all layers of the block per call.

    decode() runs them as two calls (mpc_select_clusters, mpc_sparse_decode_attn); decode_fused()
    runs both in one launch (mpc_decode_step) with the same results. With `capacity` rows per
    (layer, sequence, kv head) above `keep`, append() adds each decoded token's k, v to the cache
    (mpc_append_kv) and later steps select over the grown clusters and attend the tail."""

    def __init__(self, *, n_layers, batch, n_q_heads, n_kv_heads, head_dim, dtype, T, window, keep,
                 local_keep, cluster, fanout, k_super, k_clusters, share_period, share_start=2,
                 alpha=0.6, causal=True, layer0=0, device="cuda", keep_scores=False, similarity="linear",
                 group="sum", capacity=None):
        self.L, self.B, self.Hq, self.Hkv, self.d = n_layers, batch, n_q_heads, n_kv_heads, head_dim
        self.dtype, self.T, self.W, self.keep = dtype, T, window, keep
        self.local_keep, self.causal, self.layer0 = local_keep, causal, layer0
        self.cluster, self.k_clusters = cluster, k_clusters
        self.share_period, self.share_start = share_period, share_start
        self.sm_scale = 1.0 / math.sqrt(head_dim)
        self.rows = keep if capacity is None else capacity
        if self.rows < keep:
            raise ValueError("capacity below the kept tokens")
        self.C = -(-keep // cluster)
        self.S = -(-self.C // fanout)
        n_c = -(-self.rows // cluster)
        self.Ts, self.n_tail = keep, 0
        self.cfg = L.select_cfg(cluster, fanout, k_super, k_clusters, alpha, share_period, share_start, similarity,
                                group)
        self.Hsel = L.sel_heads(self.cfg, n_q_heads, n_kv_heads)  # selection lists per (layer, sequence)
        R = L.rep_rows(similarity)
        rep = (R, head_dim) if R > 1 else (head_dim,)
        dev = torch.device(device)
        kv_shape = (n_layers, batch, n_kv_heads)
        self.kept = torch.zeros(*kv_shape, keep, dtype=torch.int32, device=dev)
        self.k_s = torch.empty(*kv_shape, self.rows, head_dim, dtype=dtype, device=dev)
        self.v_s = torch.empty_like(self.k_s)
        self.cent = torch.zeros(*kv_shape, n_c, *rep, dtype=torch.float32, device=dev)
        self.scent = torch.zeros(*kv_shape, -(-n_c // fanout), *rep, dtype=torch.float32, device=dev)
        self.sel = torch.zeros(n_layers, batch, self.Hsel, k_clusters, dtype=torch.int32, device=dev)
        self.sel_score = torch.zeros(n_layers, batch, self.Hsel, k_clusters, dtype=torch.float32, device=dev)
        self.out = torch.empty(n_layers, batch, n_q_heads, head_dim, dtype=dtype, device=dev)
        self.lse = torch.empty(n_layers, batch, n_q_heads, dtype=torch.float32, device=dev)
        self.token_score = (torch.zeros(*kv_shape, T, dtype=torch.float32, device=dev)
                            if keep_scores else None)
        self.row_lse = (torch.zeros(n_layers, batch, n_q_heads, window, dtype=torch.float32, device=dev)
                        if keep_scores else None)
        qd = L.MpcDims(batch=batch, layer0=layer0, n_layers=n_layers, n_q_heads=n_q_heads,
                       n_kv_heads=n_kv_heads, head_dim=head_dim, dtype=L.DTYPE_CODE[dtype])
        ecfg = L.MpcEvictCfg(window=window, keep=keep, local_keep=local_keep, sm_scale=self.sm_scale,
                             causal=int(causal), share_period=share_period, share_start=share_start)
        self.ws_evict = L.workspace(L.workspace_bytes(L.MPC_OP_STATIC_EVICT, qd, T, ecfg), dev)
        self.ws_decode = L.workspace(L.workspace_bytes(L.MPC_OP_DECODE_ATTN, qd, keep), dev)
        self.ws_step = L.workspace(L.workspace_bytes(L.MPC_OP_DECODE_STEP, qd, keep, self.cfg), dev)

        # argument tuples of the per-step calls, built once per cache state (only the query pointer
        # and the stream change between decode steps that do not grow the cache)
        self._qdims = qd
        kvd = L.dims_of(self.out, self.k_s, layer0)
        self._kvdims = kvd
        lib = L.lib()
        self._select_fn = lib.mpc_select_clusters
        self._attend_fn = lib.mpc_sparse_decode_attn
        self._step_fn = lib.mpc_decode_step
        self._prepare()

    def _prepare(self):
        P = lambda t: None if t is None else ctypes.c_void_p(t.data_ptr())
        kvd, Ts, nt = self._kvdims, self.Ts, self.n_tail
        self.C = -(-Ts // self.cluster)  # selectable clusters of the current cache
        self._select_args = (ctypes.byref(kvd), Ts, ctypes.byref(self.cfg))
        self._select_tail = (P(self.cent), P(self.scent), P(self.sel), P(self.sel_score), None, 0)
        self._attend_args = (ctypes.byref(kvd), Ts, nt, self.cluster)
        self._attend_mid = (P(self.k_s), P(self.v_s), P(self.sel), self.Hsel, self.k_clusters, self.sm_scale,
                            P(self.out), P(self.lse), P(self.ws_decode), self.ws_decode.numel())
        self._step_args = (ctypes.byref(kvd), Ts, nt, ctypes.byref(self.cfg))
        self._step_tail = (P(self.cent), P(self.scent), P(self.k_s), P(self.v_s), self.sm_scale, P(self.sel),
                           P(self.sel_score), P(self.out), P(self.lse), P(self.ws_step), self.ws_step.numel())

    def prefill(self, q_win, k, v, stream=None, fused=True):
        """Static eviction into rows [0, keep) of the kept cache and the cluster build; the cache
        state returns to (keep, 0). fused: one call (mpc_prefill), else mpc_static_evict then
        mpc_build_clusters (same results)."""
        kw = dict(keep=self.keep, local_keep=self.local_keep, sm_scale=self.sm_scale, causal=self.causal,
                  layer0=self.layer0, share_period=self.share_period, share_start=self.share_start,
                  token_score=self.token_score, row_lse=self.row_lse, ws=self.ws_evict, stream=stream)
        if fused:
            L.mpc_prefill(q_win, k, v, self.kept, self.k_s, self.v_s, self.cent, self.scent, self.cfg, **kw)
        else:
            L.mpc_static_evict(q_win, k, v, self.kept, self.k_s, self.v_s, **kw)
            L.mpc_build_clusters(self.k_s, self.cent, self.scent, self.cfg, Ts=self.keep, layer0=self.layer0,
                                 stream=stream)
        if (self.Ts, self.n_tail) != (self.keep, 0):
            self.Ts, self.n_tail = self.keep, 0
            self._prepare()

    def append(self, k_new, v_new, stream=None):
        """Adds one decoded token's k, v ([L][B][Hkv][d]) to every layer's cache."""
        self.Ts, self.n_tail = L.mpc_append_kv(k_new, v_new, self.k_s, self.v_s, self.cent, self.scent, self.cfg,
                                               Ts=self.Ts, n_tail=self.n_tail, layer0=self.layer0, stream=stream)
        self._prepare()

    def select(self, q, stream=None):
        """q: [L][B][Hq][d] contiguous CUDA tensor of the path's dtype."""
        st = L._stream(stream)
        L._check("mpc_select_clusters",
                 self._select_fn(*self._select_args, ctypes.c_void_p(q.data_ptr()), *self._select_tail, st))

    def attend(self, q, stream=None):
        st = L._stream(stream)
        L._check("mpc_sparse_decode_attn",
                 self._attend_fn(*self._attend_args, ctypes.c_void_p(q.data_ptr()), *self._attend_mid, st))

    def attend_call(self, sel):
        """A prepared attention call that reads the selection from `sel` (same shape as self.sel)
        instead of self.sel: returns f(q, stream=None)."""
        if sel.shape != self.sel.shape or sel.dtype != torch.int32 or not sel.is_contiguous():
            raise ValueError("sel must be a contiguous int32 tensor shaped like the path's selection")
        mid = (self._attend_mid[0], self._attend_mid[1], ctypes.c_void_p(sel.data_ptr())) + self._attend_mid[3:]

        def call(q, stream=None):
            L._check("mpc_sparse_decode_attn",
                     self._attend_fn(*self._attend_args, ctypes.c_void_p(q.data_ptr()), *mid, L._stream(stream)))
        return call

    def decode(self, q, stream=None):
        self.select(q, stream)
        self.attend(q, stream)
        return self.out

    def capture(self, fn, *args):
        """A HIP graph (torch.cuda.CUDAGraph) of fn(*args), e.g. capture(self.decode, q_buf) or
        capture(self.prefill, q_win, k, v). Replaying it reruns the same kernels on the same buffers,
        so the caller refills the input buffers between replays. The entry points only enqueue kernels
        (no allocation, memset or host wait), so capture needs nothing else from them. A graph keeps
        the cache state (Ts, n_tail) it was captured with: capture again after append()."""
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            fn(*args)
        return g

    def decode_fused(self, q, stream=None):
        st = L._stream(stream)
        L._check("mpc_decode_step",
                 self._step_fn(*self._step_args, ctypes.c_void_p(q.data_ptr()), *self._step_tail, st))
        return self.out


class PagedPath:
    """Serving from a paged cache over mpc_paged_append, mpc_paged_attn, mpc_shared_attn, mpc_paged_read and mpc_prompt_attn: a
    batch of `batch` sequences of up to `max_rows` rows each, all layers of the block per call, the pages drawn from one pool as
    the sequences grow.

    prefill() starts every sequence with a prompt, extend() adds tokens to them (one each, drafted ones, or a chunk of a
    prompt) and attends over the cache, take_back() drops the newest rows again (rejected drafts), fork() lets sequences go on
    from the rows of another, whose whole pages they share, held() gives rows of the cache back, and adopt() starts the
    sequences with the rows that a MPCachePath kept. A call that is refused has changed nothing. All calls of a path, and the
    replays of its captured steps, share its cache and workspaces, so they run in one stream's order. fmt: the pages' format,
    "same", "e4m3" (codes with a scale for each page and head) or "mx4" (4-bit codes with a scale for each 32 channels of a
    row); by default what fp8 says, "e4m3" or "same". window, sinks: what a row sees of the rows before it (0: all of them). rope: a table [n_pos][rot_dim / 2][2] of
    (cos, sin); None where q and k arrive rotated."""

    def __init__(self, *, n_layers, batch, n_q_heads, n_kv_heads, head_dim, dtype, max_rows, page_size=64, n_pages=None,
                 fp8=True, fmt=None, window=0, sinks=0, rope=None, rope_style="interleaved", sm_scale=None, device="cuda"):
        self.Hq, self.window, self.sinks, self.rope, self.rope_style = n_q_heads, window, sinks, rope, rope_style
        self.sm_scale = 1.0 / math.sqrt(head_dim) if sm_scale is None else sm_scale
        if not 0 <= window < 2 ** 31 or not 0 <= sinks < 2 ** 31 or not math.isfinite(self.sm_scale):
            raise ValueError("window and sinks must be from 0 on, and sm_scale finite")
        if rope_style not in L.ROPE_STYLE:
            raise ValueError(f"rope_style must be one of {list(L.ROPE_STYLE)}")
        max_pages = -(-max_rows // page_size)
        n_pages = batch * max_pages if n_pages is None else n_pages
        self.kv = L.paged_kv(n_layers=n_layers, batch=batch, n_kv_heads=n_kv_heads, head_dim=head_dim, dtype=dtype,
                             n_pages=n_pages, max_pages=max_pages, page_size=page_size, device=device,
                             fmt=("e4m3" if fp8 else "same") if fmt is None else fmt)
        if rope is not None:
            p, n_pos, rot = L._rope_of(rope)
            if rope.device != self.kv.device or p % 16 or n_pos == 0 or rot == 0 or rot % 16 or rot > head_dim:
                raise ValueError(f"rope must turn a multiple of 16 channels up to {head_dim} and lie 16-byte aligned on {self.kv.device}")
        self.pos = torch.zeros(batch, dtype=torch.int32, device=self.kv.device)  # position of each sequence's next token
        self.rows = [0] * batch  # the lengths again, on the host
        self._kept = [0] * batch  # first row of each sequence that its tail still holds
        self._pages = [[] for _ in range(batch)]
        self._lent = [0] * batch  # pages at the front of each that belong to another sequence
        self._floor = [0] * batch  # rows that other sequences share, or that are shared with them
        # what mpc_shared_attn takes: how many groups and the most new tokens of a step (None: nothing is shared), and their arrays, the
        # same ones for every fork, since captured steps read them: to a step of another fork they name other groups, and what it
        # computes does not depend on which rows are read once
        self._groups = None
        n = min(batch, 1024)
        self._first = torch.zeros(n + 1, dtype=torch.int32, device=self.kv.device)
        self._shared = torch.zeros(n, dtype=torch.int32, device=self.kv.device)
        self._shared_ws = []  # the last one is the largest; smaller ones may be a captured step's
        self._free = list(range(n_pages - 1, -1, -1))
        # for steps of any number of tokens (the bytes do not grow beyond 32 query rows to a kv head), and cleared here, so
        # that a step may be captured before one has run
        size = lambda n: L.lib().mpc_workspace_bytes(L.MPC_OP_PAGED_ATTN, self.kv.dims(n_q_heads), n, self.kv.ref)  # noqa: E731
        if size(1) == 0:
            raise ValueError(f"sizes that the library does not take ({L.lib().mpc_last_error().decode()})")
        self.ws = L.workspace(max(size(1), size(32)), self.kv.device)

    def _ints(self, x):
        return torch.tensor(x, dtype=torch.int32, device=self.kv.device)

    def _counts(self, x, what, most=math.inf):
        """One whole number from 0 to `most` for each sequence."""
        x = [operator.index(n) for n in x]
        if len(x) != self.kv.B or any(not 0 <= n <= most for n in x):
            raise ValueError(f"{what}: {self.kv.B} numbers from 0 to {most} are wanted")
        return x

    def _check(self, n, q, k, v, out, lse):
        """Refuses the tensors that the calls of a step or a prompt would refuse, before any of them has run."""
        kv, turned = self.kv, self.rope is not None
        if n < 1:
            raise ValueError("no tokens")
        for what, t, heads, written in (("q", q, self.Hq, turned), ("k", k, kv.Hkv, False), ("v", v, kv.Hkv, False),
                                        ("out", out, self.Hq, True)):
            if t is None or (t.dtype is kv.dtype and t.shape == (kv.L, kv.B, heads, n, kv.d) and t.device == kv.device and
                             t.is_contiguous() and t.data_ptr() % 16 == 0):  # (a step's host time: nothing else can be wrong)
                continue
            L._like(L._rows(t, what, kv.dtype, heads)[2], kv, n, what)
            L._placed(t, what, written)
        if lse is not None:
            L._lse_of(lse, (kv.L, kv.B, self.Hq, n))
        L._on(kv.device, None, q, k, v, out, lse)

    def _lacking(self, rows, held, free):
        """The pages that rows[b] rows of each sequence want beyond the held[b] that it has, of `free` ones."""
        page, M = self.kv.page, self.kv.table.shape[1]
        if any(r > M * page for r in rows):
            raise ValueError(f"a sequence of more than {M * page} rows")
        want = [max(0, -(-r // page) - n) for r, n in zip(rows, held)]
        if sum(want) > free:
            raise ValueError(f"{sum(want)} pages wanted, {free} free")
        return want

    def _start(self, rows):
        """Empties every sequence and books rows[b] rows for each, if the whole pool has pages for them."""
        self._lacking(rows, [0] * self.kv.B, len(self._free) + sum(len(p) - n for p, n in zip(self._pages, self._lent)))
        self.clear()
        self.grown(rows)

    def clear(self):
        """Empties every sequence; the pages go back to the pool."""
        for b, pages in enumerate(self._pages):
            self._free += pages[self._lent[b]:][::-1]
            self._pages[b] = []
        self._lent = [0] * self.kv.B
        self._floor = [0] * self.kv.B
        if self._groups is not None:
            self._shared.zero_()
            self._groups = None
        self.rows = [0] * self.kv.B
        self._kept = [0] * self.kv.B
        self.kv.table.fill_(-1)
        self.kv.lens.zero_()
        self.pos.zero_()

    def reserve(self, rows):
        """Pages for rows[b] rows of each sequence, for steps that are replayed from a graph; extend() does it by itself."""
        want, M = self._lacking(self._counts(rows, "rows"), [len(p) for p in self._pages], len(self._free)), self.kv.table.shape[1]
        if sum(want) == 0:
            return
        for b, n in enumerate(want):
            self._pages[b] += [self._free.pop() for _ in range(n)]
        self.kv.table.copy_(self._ints([p + [-1] * (M - len(p)) for p in self._pages]))

    def step(self, q, k, v, n_valid=None, out=None, lse=None):
        """The device's part of extend(), which can be captured as a HIP graph: rotates, appends and attends, for sequences
        whose pages are reserved. n_valid[b] (int32 on the device) is from 0 to n. q becomes rotated in place."""
        n = q.shape[3] if q.dim() == 5 else 1
        self._check(n, q, k, v, out, lse)
        L._batch_ints(n_valid, "n_valid", self.kv.B, self.kv.device)
        return self._step(n, q, k, v, n_valid, out, lse)

    def _step(self, n, q, k, v, n_valid, out, lse):
        self.kv.lens.add_(n if n_valid is None else n_valid)
        L.mpc_paged_append(k, v, self.kv, q=q if self.rope is not None else None, rope=self.rope, rope_style=self.rope_style,
                           pos0=self.pos, n_valid=n_valid)
        self.pos.add_(n if n_valid is None else n_valid)
        out = torch.zeros_like(q) if out is None else out
        kw = dict(sm_scale=self.sm_scale, window=self.window, sinks=self.sinks, n_valid=n_valid, lse=lse)
        if self._groups is not None and n <= self._groups[1]:
            ng = self._groups[0]
            L.mpc_shared_attn(q, self.kv, out, first=self._first[:ng + 1], shared_rows=self._shared[:ng], ws=self._shared_ws[-1], **kw)
        else:
            L.mpc_paged_attn(q, self.kv, out, ws=self.ws, **kw)
        return out

    def extend(self, q, k, v, new=None, out=None, lse=None):
        """Adds the tokens q [L][B][Hq][n][d], k, v [L][B][Hkv][n][d] (new[b] <= n of sequence b, n by default) and returns their
        attention over the cache, shaped like q."""
        n = q.shape[3] if q.dim() == 5 else 1
        new = None if new is None else self._counts(new, "new", n)
        self._check(n, q, k, v, out, lse)
        self.grown([n] * self.kv.B if new is None else new)
        return self._step(n, q, k, v, None if new is None else self._ints(new), out, lse)

    def grown(self, new):
        """Books new[b] rows of each sequence on the host and reserves their pages (before the step, or the replays of one)."""
        rows = [r + n for r, n in zip(self.rows, self._counts(new, "new"))]
        self.reserve(rows)
        self.rows = rows
        page = self.kv.page
        self._kept = [max(k, ((r - 1) // page - 1) * page) for k, r in zip(self._kept, rows)]

    def take_back(self, dropped):
        """Drops the newest dropped[b] rows of each sequence; the pages stay reserved, and rows that sequences share stay. With
        8-bit pages the page that a
        sequence then ends in has to be in its tail still, which holds the last two pages that it ever reached: a page's
        rows at least."""
        dropped = self._counts(dropped, "dropped")
        page, rows = self.kv.page, [r - d for r, d in zip(self.rows, dropped)]
        for r, d, kept in zip(rows, dropped, self._kept):
            if r < 0 or (d and self.kv.k_tail is not None and r % page and r // page * page < kept):
                raise ValueError("more rows than the sequence has, or than its tail keeps")
        if any(d and r < f for r, d, f in zip(rows, dropped, self._floor)):
            raise ValueError("rows that sequences share cannot be dropped")
        d = self._ints(dropped)
        self.rows = rows
        # where a page begins nothing of the tail is needed, and what follows is written into it again
        self._kept = [min(k, r) if r % page == 0 else k for k, r in zip(self._kept, rows)]
        self.kv.lens.sub_(d)
        self.pos.sub_(d)

    def prefill(self, q, k, v, lens=None, out=None, lse=None):
        """Starts every sequence with its prompt, q [L][B][Hq][T][d], k, v [L][B][Hkv][T][d] (lens[b] tokens of sequence b, T by
        default, lens[b] <= T): the rows go into the cache, and the attention of the prompt's rows among themselves is returned. q
        becomes rotated in place."""
        if q.dim() != 5 or k.dim() != 5 or v.dim() != 5:
            raise ValueError("q, k and v must be [L][B][H][T][d]")
        T = q.shape[3]
        new = [T] * self.kv.B if lens is None else self._counts(lens, "lens", T)
        self._check(T, q, k, v, out, lse)
        self._start(new)
        n = None if lens is None else self._ints(new)
        self.kv.lens.copy_(self._ints(new))
        turned = torch.empty_like(k) if self.rope is not None else None
        L.mpc_paged_append(k, v, self.kv, q=q if self.rope is not None else None, k_out=turned, rope=self.rope,
                           rope_style=self.rope_style, pos0=self.pos, n_valid=n)
        self.pos.add_(self.kv.lens)
        out = torch.zeros_like(q) if out is None else out
        L.mpc_prompt_attn(q, k if turned is None else turned, v, out, sm_scale=self.sm_scale, window=self.window,
                          sinks=self.sinks, q_lens=n, k_lens=n, lse=lse)
        return out

    def fork(self, first, n_new=1):
        """Groups of neighbours, sequences first[g] <= b < first[g + 1]: each of them goes on from the rows of its group's first one,
        whose whole pages they share from then on (the rows behind these are copied); the others of a group have to be empty. A
        sequence alone in its group shares nothing, as one outside all groups. Steps of up to n_new tokens read the shared rows once
        for a group (mpc_shared_attn), longer ones once for each sequence. The workspace grows with n_new, by about
        8 (head_dim + 4) bytes for each token, query head, layer and sequence; one that a fork of fewer tokens made stays, since
        captured steps may use it."""
        kv, page = self.kv, self.kv.page
        first, n_new = [operator.index(b) for b in first], operator.index(n_new)
        if not 2 <= len(first) <= 1025 or first[0] < 0 or first[-1] > kv.B or any(x >= y for x, y in zip(first, first[1:])) or n_new < 1:
            raise ValueError(f"first: numbers from 0 to {kv.B}, each larger than the one before it, and n_new from 1 on are wanted")
        if self._groups is not None:
            raise ValueError("the sequences share rows already: clear() first")
        others = [(a, b) for a, z in zip(first, first[1:]) for b in range(a + 1, z)]
        if any(self.rows[b] or self._pages[b] for _, b in others):
            raise ValueError("a sequence that goes on from another's rows has to be empty")
        n_copies = sum(1 for a, _ in others if self.rows[a] % page)
        if n_copies > len(self._free):
            raise ValueError(f"{n_copies} pages wanted, {len(self._free)} free")
        shape = torch.empty(kv.L, kv.B, self.Hq, n_new, kv.d, device="meta")
        size = L.shared_attn_workspace_bytes(shape, kv, len(first) - 1)
        if size == 0:
            raise ValueError(f"sizes that the library does not take ({L.lib().mpc_last_error().decode()})")
        # (a sequence alone in its group shares nothing: its rows may be taken back, and 8-bit pages that end up incomplete must
        # not be read as shared ones)
        shared = [self.rows[a] // page * page if z > a + 1 else 0 for a, z in zip(first, first[1:])]
        if not self._shared_ws or self._shared_ws[-1].numel() < size:
            self._shared_ws.append(L.workspace(size, kv.device))
        src, dst = [], []
        for a, b in others:
            whole = self.rows[a] // page
            self._pages[b] = self._pages[a][:whole]
            self._lent[b] = whole
            if self.rows[a] % page:
                src.append(self._pages[a][whole])
                dst.append(self._free.pop())
                self._pages[b].append(dst[-1])
            self.rows[b], self._kept[b], self._floor[b], self._floor[a] = self.rows[a], self._kept[a], whole * page, whole * page
        if others:
            a, b = (torch.tensor(x, device=kv.device) for x in zip(*others))
            for t in (kv.lens, self.pos):
                t[b] = t[a]
            for t in (kv.k_tail, kv.v_tail):
                if t is not None:
                    t[:, b] = t[:, a]
            if src and kv.k_tail is None:  # (with 8-bit pages the rows behind the whole pages are in the tail)
                s, d = (torch.tensor(x, device=kv.device) for x in (src, dst))
                for t in (kv.k_pages, kv.v_pages, kv.k_scale, kv.v_scale):
                    if t is not None:
                        t[:, d] = t[:, s]
            M = kv.table.shape[1]
            kv.table.copy_(self._ints([p + [-1] * (M - len(p)) for p in self._pages]))
        spare = self._shared.numel() - len(shared)
        self._first.copy_(self._ints(first + [first[-1]] * spare))
        self._shared.copy_(self._ints(shared + [0] * spare))
        self._groups = (len(shared), n_new)

    def held(self, n, first=None):
        """(k, v), each [L][B][Hkv][n][d] in the element type: rows first[b] .. first[b] + n - 1 of each sequence as the cache has them
        (the newest n by default), zeros for rows that it does not have."""
        kv, n = self.kv, operator.index(n)
        if n < 1:
            raise ValueError("no rows")
        first = None if first is None else self._ints(self._counts(first, "first", 2 ** 31 - 1))
        k, v = (torch.zeros(kv.L, kv.B, kv.Hkv, n, kv.d, dtype=kv.dtype, device=kv.device) for _ in range(2))
        L.mpc_paged_read(kv, k, v, first=first)
        return k, v

    def adopt(self, path, position):
        """Starts every sequence with the rows that `path` (a MPCachePath of the same shape) keeps, as they are: its evicted
        prompt and what was appended to it. `position`: that of the next token."""
        kv, n = self.kv, path.Ts + path.n_tail
        for what, t in (("path.k_s", path.k_s), ("path.v_s", path.v_s)):
            L._like(L._rows(t[:, :, :, :n], what, kv.dtype, kv.Hkv)[2], kv, n, what)
        L._on(kv.device, None, path.k_s, path.v_s)
        position = operator.index(position)
        if not 0 <= position < 2 ** 31:
            raise ValueError("position must be from 0 on")
        self._start([n] * kv.B)
        self.kv.lens.fill_(n)
        L.mpc_paged_append(path.k_s[:, :, :, :n], path.v_s[:, :, :, :n], self.kv)
        self.pos.fill_(position)
