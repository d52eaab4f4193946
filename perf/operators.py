"""Cases of the paged-cache operators: appending rotated keys and values to a paged cache, attention over
that cache (pages in the element type or in 8 bits with a scale for each page and head), and the attention of
a prompt with a sliding window and a few first tokens that stay visible.

Sizes are those of this repository's workloads (12 heads of 64, 32 heads of 128, 32 query heads over 8 kv heads;
512 to 128K tokens) or lie between them. `own` False computes the plain forms; True makes the package's calls.
"""
import math

import torch

own = False

DTYPE = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
ROPE_BASE = 10000.0


def _append(name, **kw):
    return dict(name=name, op="append", **kw)


def _paged(name, **kw):
    return dict(name=name, op="paged", **kw)


def _prompt(name, **kw):
    return dict(name=name, op="prompt", **kw)


def listed():
    return [
        # one decoded token of one layer, as inside a model's layer loop: latency of the smallest call
        _append("append-token", L=1, B=1, Hq=32, Hkv=8, d=128, dtype="bf16", fp8=True, page=64, T=8192, n=1, ragged=False,
                style="half"),
        # one decoded token of every layer of four sequences at four lengths, all heads of the 7B shape
        _append("append-step-b4", L=32, B=4, Hq=32, Hkv=32, d=128, dtype="bf16", fp8=True, page=32, T=2048, n=1,
                ragged=True, style="interleaved"),
        # four prompts of different lengths into pages of the element type, one layer
        _append("append-prompts-16bit", L=1, B=4, Hq=32, Hkv=32, d=128, dtype="bf16", fp8=False, page=16, T=8192, n=8192,
                ragged=True, style="half"),
        # one long prompt into 8-bit pages, grouped heads, two layers
        _append("append-prompt-8bit", L=2, B=1, Hq=32, Hkv=8, d=128, dtype="fp16", fp8=True, page=64, T=32767, n=32767,
                ragged=False, style="interleaved"),
        # one token of a small fp32 model over a short cache: latency
        _paged("decode-short-fp32", L=1, B=1, Hq=12, Hkv=12, d=64, dtype="fp32", fp8=False, page=16, T=500, n=1,
               ragged=False, window=0, sinks=0),
        # a decode step of four 32K sequences over 8-bit pages, two layers: bandwidth
        _paged("decode-32k-b4-8bit", L=2, B=4, Hq=32, Hkv=32, d=128, dtype="bf16", fp8=True, page=32, T=32768, n=1,
               ragged=False, window=0, sinks=0),
        # the longest cache, grouped heads, one layer: few rows, a long axis
        _paged("decode-128k-gqa-8bit", L=1, B=1, Hq=32, Hkv=8, d=128, dtype="bf16", fp8=True, page=64, T=131072 - 17,
               n=1, ragged=False, window=0, sinks=0),
        # four drafted tokens for each of 32 sequences of very different lengths, window and sinks, 16-bit pages
        _paged("drafts-window-b32", L=1, B=32, Hq=32, Hkv=8, d=128, dtype="fp16", fp8=False, page=16, T=20000, n=4,
               ragged=True, window=1024, sinks=4),
        # a short prompt of a small fp32 model
        _prompt("prompt-512-fp32", L=1, B=1, Hq=12, Hkv=12, d=64, dtype="fp32", Tq=512, T=512, ragged=False, window=0,
                sinks=0),
        # one layer of an 8K prompt, 7B shape, every key visible
        _prompt("prompt-8k", L=1, B=1, Hq=32, Hkv=32, d=128, dtype="bf16", Tq=8192, T=8192, ragged=False, window=0,
                sinks=0),
        # four prompts of different lengths behind a sliding window with sinks, grouped heads
        _prompt("prompt-window-b4", L=1, B=4, Hq=32, Hkv=8, d=128, dtype="bf16", Tq=16384, T=16384, ragged=True,
                window=1024, sinks=4),
        # the last 1000 tokens of a long prompt that is taken in chunks
        _prompt("prompt-chunk-20k", L=1, B=1, Hq=32, Hkv=8, d=128, dtype="fp16", Tq=1000, T=20000, ragged=False,
                window=0, sinks=0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "paged", "prompt"])
    heads = rng.choice([(12, 12, 64), (32, 32, 128), (32, 8, 128), (16, 4, 64), (8, 1, 128), (16, 8, 128)])
    c = dict(op=op, Hq=heads[0], Hkv=heads[1], d=heads[2], dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]),
             ragged=rng.random() < 0.5)
    if op == "append":
        c.update(fp8=rng.random() < 0.6, page=rng.choice([16, 32, 64, 128]), style=rng.choice(["half", "interleaved"]))
        if rng.random() < 0.5:  # decoded or drafted tokens
            L, T = _log_int(rng, 1, 32), _log_int(rng, 64, 4096)
            c.update(L=L, B=_log_int(rng, 1, max(1, min(32, 131072 // (L * T)))), n=rng.choice([1, 1, 2, 5]), T=T)
        else:  # prompts
            n = _log_int(rng, 32, 16384)
            c.update(L=1, B=max(1, min(8, _log_int(rng, 1, 16384) // n)), n=n, T=n)
        return c
    window = rng.choice([0, 0, rng.randint(1, 300), rng.randint(300, 4096)])
    c.update(window=window, sinks=rng.choice([0, 4, rng.randint(1, 64)]) if window else 0)
    if op == "paged":
        T = _log_int(rng, 1, 65536)
        c.update(fp8=rng.random() < 0.6, page=rng.choice([16, 32, 64, 128]), n=rng.choice([1, 1, 1, 3, 8]), T=max(T, 8),
                 B=max(1, min(32, _log_int(rng, 1, 131072) // T)), L=1)
        return c
    T = _log_int(rng, 16, 8192)
    c.update(L=1, B=1 if T > 1500 else rng.randint(1, 6), T=T, Tq=T if rng.random() < 0.7 else rng.randint(1, T))
    if c["dtype"] == "fp32":
        c.update(T=min(T, 4096), Tq=min(c["Tq"], 4096))
    return c


def _rows(c):
    """(rows in the cache, new rows) of each sequence, this call's rows included."""
    B, T, n = c["B"], c["T"], c["n"] if c["op"] != "prompt" else c["Tq"]
    lens = [T if b == 0 or not c["ragged"] else max(1, T * ((5 * b) % 11 + 1) // 12 - b) for b in range(B)]
    if c["op"] == "append" and n == T:
        return lens, list(lens)  # whole prompts: every row is new
    new = [n if b == 0 or not c["ragged"] else max(1, n - b % n) for b in range(B)]
    return lens, [min(x, y) for x, y in zip(new, lens)]


def _visible(c):
    """Pairs (row, key) that see each other, over the sequences of one layer and one query head; keys read."""
    lens, new = _rows(c)
    w, s, pairs, keys = c["window"], c["sinks"], 0, 0
    for length, m in zip(lens, new):
        p = torch.arange(length - m, length, dtype=torch.int64)
        if not w:
            pairs += int((p + 1).sum())
            keys += length
        else:
            lo = (p - w + 1).clamp(min=0)
            pairs += int((p + 1 - lo).sum() + torch.minimum(lo, torch.tensor(s)).sum())
            keys += length - int(lo[0]) + min(s, int(lo[0]))
    return pairs, keys


def work(c):
    e, d, lens = DTYPE[c["dtype"]].itemsize, c["d"], _rows(c)
    if c["op"] == "append":
        new = sum(lens[1])
        rows = c["L"] * new * d
        moved = rows * e * (c["Hq"] + 2 * c["Hkv"]) + rows * c["Hq"] * e  # inputs, rotated queries
        if not c["fp8"]:
            moved += rows * e * 2 * c["Hkv"]
        else:
            full = fresh = old = 0
            for length, m in zip(*lens):
                first, done = (length - m) // c["page"], length // c["page"]
                full += max(0, done - first) * c["page"]
                fresh += length - max(length - m, max(0, (length - 1) // c["page"] - 1) * c["page"])
                old += (length - m) % c["page"] if done > first else 0
            moved += 2 * c["L"] * c["Hkv"] * d * (full + (fresh + old) * e)
        return {"bytes": moved, "flops": rows * 3 * (c["Hq"] + c["Hkv"])}
    pairs, keys = _visible(c)
    kv = c["L"] * c["Hkv"] * d
    q = c["L"] * c["Hq"] * sum(lens[1]) * d * e
    return {"bytes": 2 * kv * keys * (1 if c.get("fp8") else e) + 2 * q, "flops": 4 * c["L"] * c["Hq"] * d * pairs}


def _pow2(s):
    """2^s in fp32 for whole s."""
    return ((s + 127) << 23).to(torch.int32).view(torch.float32)


def _encode(x):
    """Codes and scale (the least power of two that brings the block's largest value to 448 or less) of fp32
    blocks over the last two axes."""
    m, e = torch.frexp(x.abs().amax((-1, -2)))
    scale = _pow2(torch.where(m == 0, 0, (e - torch.where(m <= 0.875, 9, 8)).clamp(-126, 127)))
    return (x / scale[..., None, None]).to(E4M3), scale


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, L, B, Hkv, Hq, d = DTYPE[c["dtype"]], c["L"], c["B"], c["Hkv"], c["Hq"], c["d"]
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=dt)  # noqa: E731
    # keys have four channels of eight times the spread, as trained models' keys do
    spread = torch.ones(d, device="cuda", dtype=dt)
    spread[torch.randperm(d, generator=g, device="cuda")[:4]] = 8
    lens, new = _rows(c)
    on = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    s = dict(case=c, sm=1.0 / math.sqrt(d))
    if c["op"] == "prompt":
        s.update(q=normal(L, B, Hq, c["Tq"], d), k=normal(L, B, Hkv, c["T"], d) * spread, v=normal(L, B, Hkv, c["T"], d),
                 out=torch.zeros(L, B, Hq, c["Tq"], d, device="cuda", dtype=dt),
                 lse=torch.zeros(L, B, Hq, c["Tq"], device="cuda"), q_lens=on(new) if c["ragged"] else None,
                 k_lens=on(lens) if c["ragged"] else None)
        return s
    n, page = c["n"], c["page"]
    M = -(-c["T"] // page) + 2
    P = B * M
    table = torch.randperm(P, generator=g, device="cuda").to(torch.int32).view(B, M)
    s.update(q=normal(L, B, Hq, n, d), table=table, lens=on(lens), n_valid=on(new) if c["ragged"] else None)
    pool = (L, P, Hkv, page, d)
    if c["op"] == "append":
        s.update(k=normal(L, B, Hkv, n, d) * spread, v=normal(L, B, Hkv, n, d), q_out=torch.zeros_like(s["q"]))
        half = torch.arange(d // 2, dtype=torch.float64, device="cuda")
        angle = torch.arange(c["T"], dtype=torch.float64, device="cuda")[:, None] * ROPE_BASE ** (-2 * half / d)
        s["rope"] = torch.stack([angle.cos(), angle.sin()], -1).float()
        kp, vp = (torch.zeros(pool, device="cuda", dtype=E4M3 if c["fp8"] else dt) for _ in range(2))
    else:
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(L, B, Hq, n, device="cuda")
        kp, vp = normal(*pool) * spread, normal(*pool)
    ks = vs = kt = vt = None
    if c["fp8"]:
        kt, vt = normal(L, B, Hkv, 2 * page, d) * spread, normal(L, B, Hkv, 2 * page, d)
        if c["op"] == "append":
            ks, vs = (torch.zeros(L, P, Hkv, device="cuda") for _ in range(2))
        else:
            (kp, ks), (vp, vs) = _encode(kp.float()), _encode(vp.float())
    s.update(k_pages=kp, v_pages=vp, k_scale=ks, v_scale=vs, k_tail=kt, v_tail=vt)
    if own:  # the handle that a program keeps: the cache's tensors as one object, and the workspace
        import paper_2501_06807_amd as mpc
        s["kv"] = mpc.PagedKV(kp, vp, table, s["lens"], k_scale=ks, v_scale=vs, k_tail=kt, v_tail=vt)
        if c["op"] == "paged":
            s["ws"] = mpc.workspace(mpc.paged_attn_workspace_bytes(s["q"], s["kv"]), "cuda")
    return s


def _own(s):
    import paper_2501_06807_amd as mpc
    c = s["case"]
    if c["op"] == "append":
        mpc.mpc_paged_append(s["k"], s["v"], s["kv"], q=s["q"], q_out=s["q_out"], rope=s["rope"], rope_style=c["style"],
                             n_valid=s["n_valid"])
        return _appended(s)
    if c["op"] == "paged":
        mpc.mpc_paged_attn(s["q"], s["kv"], s["out"], sm_scale=s["sm"], window=c["window"], sinks=c["sinks"],
                           n_valid=s["n_valid"], lse=s["lse"], ws=s["ws"])
    else:
        mpc.mpc_prompt_attn(s["q"], s["k"], s["v"], s["out"], sm_scale=s["sm"], window=c["window"], sinks=c["sinks"],
                            q_lens=s["q_lens"], k_lens=s["k_lens"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def _appended(s):
    names = ["k_pages", "v_pages", "q_out"] + (["k_scale", "v_scale", "k_tail", "v_tail"] if s["case"]["fp8"] else [])
    return {k: s[k] for k in names}


def _rotate(x, cs, style):
    """Rows x [..., n, d] by (cos, sin) pairs cs [B, 1, n, d / 2, 2]; fp32, rounded to x's type."""
    d, y = x.shape[-1], x.float()
    a, b = (y[..., : d // 2], y[..., d // 2:]) if style == "half" else (y[..., 0::2], y[..., 1::2])
    co, si = cs[..., 0], cs[..., 1]
    r0, r1 = a * co - b * si, a * si + b * co
    return (torch.cat([r0, r1], -1) if style == "half" else torch.stack([r0, r1], -1).flatten(-2)).to(x.dtype)


def _plain_append(s):
    c = s["case"]
    L, B, Hkv, n, d = s["k"].shape
    page, M = c["page"], s["table"].shape[1]
    lens = s["lens"].long()
    new = s["n_valid"].long() if s["n_valid"] is not None else torch.full_like(lens, n)
    start = lens - new
    t = torch.arange(n, device="cuda")
    at = (start[:, None] + t).clamp(0, c["T"] - 1)  # [B, n]: rows, and positions
    live = t < new[:, None]
    cs = s["rope"][at][:, None]
    q, k, v = _rotate(s["q"], cs, c["style"]), _rotate(s["k"], cs, c["style"]), s["v"]
    s["q_out"].copy_(torch.where(live[:, None, :, None], q, s["q_out"]))
    # every page from the first new row's on: its rows are new ones, rows of the tail ring, or not there yet
    NP = (n + page - 2) // page + 1
    p = (start // page)[:, None] + torch.arange(NP, device="cuda")  # [B, NP]
    ids = torch.gather(s["table"].long(), 1, p.clamp(max=M - 1))
    j = (p[..., None] * page + torch.arange(page, device="cuda")).flatten(1)  # [B, NP * page]
    src, is_new, is_row = (j - start[:, None]).clamp(0, n - 1), j >= start[:, None], j < lens[:, None]
    wide = lambda m: m[None, :, None, :, None]  # noqa: E731
    pick = lambda x, i: torch.gather(x, 3, wide(i).expand(L, B, Hkv, i.shape[1], d))  # noqa: E731
    for x, name in ((k, "k"), (v, "v")):
        pool = s[name + "_pages"]
        fresh = pick(x, src)
        cut = lambda y: y.unflatten(3, (NP, page)).permute(0, 1, 3, 2, 4, 5)  # noqa: E731
        old = pool.view(torch.uint8)[:, ids].view(pool.dtype)  # [L, B, NP, Hkv, page, d]
        if not c["fp8"]:
            pool[:, ids] = torch.where(cut(wide(is_new & is_row)), cut(fresh), old)
            continue
        tail = s[name + "_tail"]
        rows = torch.where(wide(is_new), fresh, pick(tail, j % (2 * page)))
        codes, scale = _encode(cut(rows).float())
        done = ((p + 1) * page <= lens[:, None])[None, :, :, None]
        pool.view(torch.uint8)[:, ids] = torch.where(done[..., None, None], codes.view(torch.uint8), old.view(torch.uint8))
        s[name + "_scale"][:, ids] = torch.where(done, scale, s[name + "_scale"][:, ids])
        # the ring keeps the new rows of the last two pages; slot r holds the last row j with j mod 2 page = r
        r = torch.arange(2 * page, device="cuda")
        last = (lens - 1)[:, None]
        top = last - (last - r) % (2 * page)
        keep = (top >= start[:, None]) & (top >= 0) & (top // page >= last // page - 1)
        tail.copy_(torch.where(wide(keep), pick(x, (top - start[:, None]).clamp(0, n - 1)), tail))
    return _appended(s)


def _softmax_out(scores, see, v, dt):
    """Weights of masked scores on v: (out, natural log of the weights' sum); rows that see nothing give 0 and -inf."""
    scores = scores.masked_fill(~see, -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    w = torch.exp(scores - top)
    total = w.sum(-1, keepdim=True)
    out = torch.matmul(w, v) / torch.where(total == 0, 1.0, total)
    return out.to(dt), (total.log() + top)[..., 0]


def _sees(p, j, c):
    see = j <= p
    if c["window"]:
        see = see & ((j > p - c["window"]) | (j < c["sinks"]))
    return see


def _plain_paged(s):
    c = s["case"]
    L, B, Hq, n, d = s["q"].shape
    Hkv, page, T = c["Hkv"], c["page"], c["T"]
    lens = s["lens"].long()
    new = s["n_valid"].long() if s["n_valid"] is not None else torch.full_like(lens, n)
    NP = -(-T // page)
    ids = s["table"][:, :NP].long()
    j = torch.arange(NP * page, device="cuda")
    row = (j < lens[:, None])[None, :, None, :, None]
    kv = []
    for name in ("k", "v"):
        x = s[name + "_pages"]
        x = x.view(torch.uint8)[:, ids].view(x.dtype).float()  # [L, B, NP, Hkv, page, d]
        if c["fp8"]:
            x = x * s[name + "_scale"][:, ids][..., None, None]
        x = x.transpose(2, 3).flatten(3, 4)
        if c["fp8"]:
            in_ring = (j >= (lens // page * page)[:, None])[None, :, None, :, None]
            ring = s[name + "_tail"].repeat(1, 1, 1, -(-NP // 2), 1)[..., : NP * page, :].float()
            x = torch.where(in_ring, ring, x)
        kv.append(torch.where(row, x, 0.0))
    q = s["q"].float().reshape(L, B, Hkv, -1, d)
    scores = torch.matmul(q, kv[0].transpose(-1, -2)) * s["sm"]
    t = torch.arange(n, device="cuda")
    pos = ((lens - new)[:, None] + t).repeat(1, Hq // Hkv)[None, :, None, :, None]
    out, lse = _softmax_out(scores, _sees(pos, j, c) & row.squeeze(-1)[..., None, :], kv[1], s["q"].dtype)
    live = (t < new[:, None])[None, :, None]
    return {"out": torch.where(live[..., None], out.reshape(s["q"].shape), s["out"]),
            "lse": torch.where(live, lse.reshape(L, B, Hq, n), s["lse"])}


def _plain_prompt(s):
    c = s["case"]
    L, B, Hq, Tq, d = s["q"].shape
    Hkv, T, w, dt = c["Hkv"], c["T"], c["window"], s["q"].dtype
    every = lambda x, n: x.long() if x is not None else torch.full((B,), n, device="cuda")  # noqa: E731
    q_len, k_len = every(s["q_lens"], Tq), every(s["k_lens"], T)
    start = k_len - q_len
    q, k, v = s["q"].float().unflatten(2, (Hkv, -1)), s["k"].float(), s["v"].float()
    t = torch.arange(Tq, device="cuda")
    if not w or w >= T:
        j = torch.arange(T, device="cuda")
        see = _sees((start[:, None] + t)[..., None], j, c) & (j < k_len[:, None, None])  # [B, Tq, T]
        scores = torch.matmul(q.flatten(3, 4), k.transpose(-1, -2)).mul_(s["sm"])
        out, lse = _softmax_out(scores.unflatten(3, (-1, Tq)), see[None, :, None, None], v[:, :, :, None], dt)
    else:
        # blocks of rows, each with the keys that its window can reach and the sinks before them
        step = min(max(w, 16), 1024, Tq)
        nb = -(-Tq // step)
        rows = torch.arange(nb * step, device="cuda").view(nb, step)
        lo = start[:, None] + rows[:, 0] - w + 1  # [B, nb]
        band = lo[..., None] + torch.arange(w - 1 + step, device="cuda")
        sink = torch.arange(c["sinks"], device="cuda").expand(B, nb, -1)
        j = torch.cat([sink, band], -1)  # [B, nb, span]
        fine = (j >= 0) & (j < k_len[:, None, None])
        fine[..., c["sinks"]:] &= band >= c["sinks"]  # sinks count once
        at = j.clamp(0, T - 1)
        take = lambda x: torch.gather(x, 3, at.flatten(1)[None, :, None, :, None].expand(L, B, Hkv, -1, d)).unflatten(3, (nb, -1))  # noqa: E731
        q = torch.nn.functional.pad(q, (0, 0, 0, nb * step - Tq)).unflatten(4, (nb, step)).transpose(3, 4)  # L B Hkv nb G step d
        pos = start[:, None, None] + rows  # [B, nb, step]
        see = _sees(pos[..., None], j[:, :, None], c) & fine[:, :, None]
        scores = torch.matmul(q.flatten(4, 5), take(k).transpose(-1, -2)).mul_(s["sm"]).unflatten(4, (-1, step))
        out, lse = _softmax_out(scores, see[None, :, None, :, None], take(v).unsqueeze(4), dt)
        out = out.transpose(3, 4).flatten(4, 5)[..., :Tq, :]
        lse = lse.transpose(3, 4).flatten(4, 5)[..., :Tq]
    live = (t < q_len[:, None])[None, :, None]
    return {"out": torch.where(live[..., None], out.reshape(s["q"].shape), s["out"]),
            "lse": torch.where(live, lse.reshape(L, B, Hq, Tq), s["lse"])}


def run(s):
    if own:
        return _own(s)
    return {"append": _plain_append, "paged": _plain_paged, "prompt": _plain_prompt}[s["case"]["op"]](s)


def _exact_append(s, lens, new):
    c, page = s["case"], s["case"]["page"]
    L, B, Hkv, n, d = s["k"].shape
    dt, res = s["k"].dtype, {k: x.double() for k, x in _appended(s).items()}
    freq = ROPE_BASE ** (-2 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
    first = torch.arange(d // 2, device="cuda") * (1 if c["style"] == "half" else 2)
    second = first + (d // 2 if c["style"] == "half" else 1)
    for b in range(B):
        m, base = new[b], lens[b] - new[b]
        ang = torch.arange(base, lens[b], dtype=torch.float64, device="cuda")[:, None] * freq

        def turned(x):
            z = torch.view_as_complex(torch.stack([x[..., first], x[..., second]], -1)) * torch.polar(torch.ones_like(ang), ang)
            y = torch.empty_like(x)
            y[..., first], y[..., second] = z.real, z.imag
            return y

        res["q_out"][:, b, :, :m] = turned(s["q"][:, b, :, :m].double())
        for name in ("k", "v"):
            x = s[name][:, b, :, :m].double()
            x = turned(x) if name == "k" else x
            pages, spots = s["table"][b].tolist(), 2 * page
            rows = x.to(dt).double()  # the rows as the element type holds them: what codes are made from
            before = [(base // page) * page, base]
            old = torch.stack([s[name + "_tail"][:, b, :, i % spots].double() for i in range(*before)], 2) if c["fp8"] and before[0] < base else rows[:, :, :0]
            both = torch.cat([old, rows], 2)  # rows before[0] .. lens[b] - 1
            for p in range(base // page, -(-lens[b] // page)):
                lo, hi = p * page, min((p + 1) * page, lens[b])
                if not c["fp8"]:
                    lo = max(lo, base)
                    res[name + "_pages"][:, pages[p], :, lo - p * page:hi - p * page] = x[:, :, lo - base:hi - base]
                elif hi - lo == page:
                    y = both[:, :, lo - before[0]:hi - before[0]]
                    top = y.abs().amax((2, 3))
                    e = torch.where(top > 0, torch.ceil(torch.log2(top / E4M3_MAX)), torch.zeros_like(top)).clamp(-126, 127)
                    res[name + "_scale"][:, pages[p]] = 2.0 ** e
                    u = y / (2.0 ** e)[..., None, None]
                    grid = 2.0 ** torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -6))) / 8  # steps of three binary places
                    res[name + "_pages"][:, pages[p]] = torch.round(u / grid) * grid
            if c["fp8"]:
                for i in range(max(base, ((lens[b] - 1) // page - 1) * page), lens[b]):
                    res[name + "_tail"][:, b, :, i % spots] = x[:, :, i - base]
    return res


def _exact_rows(s, q, k, v, pos):
    """q [H, G, m, d], k / v [H, T, d] in 64 bits, pos [m] -> out, lse by the definition."""
    c, T = s["case"], k.shape[1]
    j = torch.arange(T, device="cuda")
    see = j[None] <= pos[:, None]
    if c["window"]:
        see &= (j[None] > pos[:, None] - c["window"]) | (j[None] < c["sinks"])
    score = (q @ k[:, None].transpose(-1, -2)) * s["sm"]
    score[..., ~see] = -math.inf
    lse = torch.logsumexp(score, -1)
    weight = torch.exp(score - torch.where(lse == -math.inf, 0.0, lse)[..., None])
    return weight @ v[:, None], lse


def exact(c, seed):
    s = prepare(c, seed)
    lens, new = _rows(c)
    if c["op"] == "append":
        return _exact_append(s, lens, new)
    out, lse = s["out"].double(), s["lse"].double()
    G = c["Hq"] // c["Hkv"]
    for l in range(c["L"]):
        for b in range(c["B"]):
            n, m = lens[b], new[b]
            if c["op"] == "prompt":
                k, v = s["k"][l, b, :, :n], s["v"][l, b, :, :n]
            else:
                page, kv = c["page"], []
                for name in ("k", "v"):
                    done = n // page if c["fp8"] else -(-n // page)
                    ids = s["table"][b, :done].long()
                    x = s[name + "_pages"][l].view(torch.uint8)[ids].view(s[name + "_pages"].dtype).double()
                    if c["fp8"]:
                        x = x * s[name + "_scale"][l, ids].double()[..., None, None]
                    x = x.transpose(0, 1).flatten(1, 2)[:, :n]
                    if c["fp8"]:
                        slots = torch.arange(done * page, n, device="cuda") % (2 * page)
                        x = torch.cat([x, s[name + "_tail"][l, b][:, slots].double()], 1)
                    kv.append(x)
                k, v = kv
            step = max(1, (1 << 28) // (n * G))
            for h in range(c["Hkv"]):
                for i in range(0, m, step):
                    e = min(i + step, m)
                    hq = slice(h * G, (h + 1) * G)
                    pos = torch.arange(n - m + i, n - m + e, device="cuda")
                    out[l, b, hq, i:e], lse[l, b, hq, i:e] = (x[0] for x in _exact_rows(
                        s, s["q"][l, b, hq, i:e].double()[None], k[h:h + 1].double(), v[h:h + 1].double(), pos))
    return {"out": out, "lse": lse}
