"""Cases of the second set of paged-cache operators: pages of 4-bit floating-point codes with a scale for each 32 channels of a
row (written as tokens arrive, read back, and attended to), and the attention of a batch whose sequences share their first
pages, which are read once for all of them.

Sizes are those of this repository's workloads (12 heads of 64, 32 heads of 128, 32 query heads over 8 kv heads;
512 to 128K tokens) or lie between them. `own` False computes the plain forms; True makes the package's calls.
"""
import math

import torch

own = False

DTYPE = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # magnitudes of the 4-bit codes; the fourth bit is the sign
BLOCK = 32  # channels to a scale of the 4-bit codes
ROPE_BASE = 10000.0


def listed():
    return [
        # one decoded token of one layer into 4-bit pages, and its row as the cache has it: latency of the smallest calls
        dict(name="store-token", op="store", fmt="mx4", L=1, B=1, Hq=32, Hkv=8, d=128, dtype="bf16", page=64, T=8192, n=1,
             ragged=False, style="half"),
        # four prompts of different lengths into 4-bit pages, and back for the attention of the prompts over what was kept
        dict(name="store-prompts-b4", op="store", fmt="mx4", L=1, B=4, Hq=32, Hkv=32, d=128, dtype="fp16", page=16, T=8192, n=8192,
             ragged=True, style="interleaved"),
        # a long sequence of a 4-bit cache back into plain rows, two layers (to evict from it, or to move it)
        dict(name="read-32k-4bit", op="read", fmt="mx4", L=2, B=1, Hq=32, Hkv=8, d=128, dtype="bf16", page=64, T=32767, n=32767,
             ragged=False),
        # the newest rows of four sequences of 8-bit pages, those of the pages that are not complete among them
        dict(name="read-newest-8bit", op="read", fmt="e4m3", L=2, B=4, Hq=12, Hkv=12, d=64, dtype="fp16", page=32, T=5000, n=500,
             ragged=True),
        # one token of a small fp32 model over a short 4-bit cache: latency
        dict(name="decode-short-4bit", op="paged", fmt="mx4", L=1, B=1, Hq=12, Hkv=12, d=64, dtype="fp32", page=16, T=500, n=1,
             ragged=False, window=0, sinks=0),
        # a decode step of four 32K sequences over 4-bit pages, two layers: bandwidth
        dict(name="decode-32k-b4-4bit", op="paged", fmt="mx4", L=2, B=4, Hq=32, Hkv=32, d=128, dtype="bf16", page=32, T=32768, n=1,
             ragged=False, window=0, sinks=0),
        # the longest cache, grouped heads, three drafted tokens, one layer: a long axis
        dict(name="drafts-128k-gqa-4bit", op="paged", fmt="mx4", L=1, B=1, Hq=32, Hkv=8, d=128, dtype="fp16", page=64,
             T=131072 - 17, n=3, ragged=False, window=0, sinks=0),
        # eight short sequences of a small fp32 model behind one prompt of 512 tokens: latency
        dict(name="shared-short-fp32", op="shared", fmt="same", L=1, B=8, groups=1, Hq=12, Hkv=12, d=64, dtype="fp32", page=16, T=512,
             S=40, n=1, ragged=True, window=0, sinks=0),
        # a decode step of 32 conversations behind one document of 32K tokens, grouped heads, 16-bit pages: bandwidth
        dict(name="shared-32k-b32", op="shared", fmt="same", L=1, B=32, groups=1, Hq=32, Hkv=8, d=128, dtype="bf16", page=32, T=32768,
             S=700, n=1, ragged=True, window=0, sinks=0),
        # 64 sequences in four groups of different sizes, each behind its own 8K prompt, all heads of the 7B shape, 8-bit pages
        dict(name="shared-8k-groups", op="shared", fmt="e4m3", L=1, B=64, groups=4, Hq=32, Hkv=32, d=128, dtype="bf16", page=64, T=8192,
             S=300, n=1, ragged=True, window=0, sinks=0),
        # four drafted tokens of each of 48 sequences behind 20K tokens of 4-bit pages
        dict(name="shared-drafts-4bit", op="shared", fmt="mx4", L=1, B=48, groups=1, Hq=32, Hkv=8, d=128, dtype="bf16", page=64, T=20000,
             S=500, n=4, ragged=True, window=0, sinks=0),
        # eight questions of up to 256 tokens each, taken as prompts behind 16K shared tokens
        dict(name="shared-prompts-16k", op="shared", fmt="same", L=1, B=8, groups=1, Hq=32, Hkv=8, d=128, dtype="fp16", page=16, T=16384,
             S=256, n=256, ragged=True, window=0, sinks=0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["store", "read", "paged", "shared", "shared"])
    heads = rng.choice([(12, 12, 64), (32, 32, 128), (32, 8, 128), (16, 4, 64), (8, 1, 128), (16, 8, 128)])
    c = dict(op=op, Hq=heads[0], Hkv=heads[1], d=heads[2], dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), L=1,
             ragged=rng.random() < 0.5, page=rng.choice([16, 32, 64, 128]))
    if op == "store":
        c.update(fmt="mx4", style=rng.choice(["half", "interleaved"]))
        if rng.random() < 0.5:  # decoded or drafted tokens
            L, T = _log_int(rng, 1, 32), _log_int(rng, 64, 4096)
            c.update(L=L, B=_log_int(rng, 1, max(1, min(32, 131072 // (L * T)))), n=rng.choice([1, 1, 2, 5]), T=T)
        else:  # prompts
            n = _log_int(rng, 32, 16384)
            c.update(B=max(1, min(8, _log_int(rng, 1, 16384) // n)), n=n, T=n)
        return c
    c.update(fmt=rng.choice(["mx4", "mx4", "e4m3", "same"]))
    if op == "read":
        T = _log_int(rng, 8, 32768)
        c.update(T=T, n=_log_int(rng, 1, T), B=max(1, min(32, _log_int(rng, 1, 32768) // T)))
        return c
    window = rng.choice([0, 0, 0, rng.randint(1, 300), rng.randint(300, 4096)])
    c.update(window=window, sinks=rng.choice([0, 4, rng.randint(1, 64)]) if window else 0)
    if op == "paged":
        T = _log_int(rng, 8, 65536)
        c.update(fmt="mx4", n=rng.choice([1, 1, 1, 3, 8]), T=T, B=max(1, min(32, _log_int(rng, 1, 131072) // T)))
        return c
    n = rng.choice([1, 1, 1, 3, 8, rng.randint(16, 128)])
    T, B = _log_int(rng, 16, 16384), _log_int(rng, 1, 64 if n < 16 else 8)
    c.update(n=n, T=T, B=B, groups=min(B, rng.choice([1, 1, 2, 3, rng.randint(1, 16)])), S=n + _log_int(rng, 1, 600))
    while c["groups"] > 1 and c["groups"] * T > 32768:  # the pages of all groups' prompts
        c["groups"] -= 1
    return c


def _rows(c):
    """(rows in the cache, new rows) of each sequence, this call's rows included."""
    B, T, n = c["B"], c["T"], c["n"]
    if c["op"] == "shared":  # the shared pages, then rows of each sequence's own
        base = T // c["page"] * c["page"]
        own_rows = [c["S"] if b == 0 or not c["ragged"] else max(1, c["S"] * ((5 * b) % 11 + 1) // 12 - b % 7) for b in range(B)]
        new = [n if b == 0 or not c["ragged"] or n < 16 else max(1, n - 13 * b) for b in range(B)]
        return [base + max(x, y) for x, y in zip(own_rows, new)], new
    lens = [T if b == 0 or not c["ragged"] else max(1, T * ((5 * b) % 11 + 1) // 12 - b) for b in range(B)]
    if c["op"] == "store" and n == T:
        return lens, list(lens)  # whole prompts: every row is new
    new = [n if b == 0 or not c["ragged"] else max(1, n - b % n) for b in range(B)]
    return lens, [min(x, y) for x, y in zip(new, lens)]


def _first(c):
    """First sequence of each group, and B behind the last: sizes that differ where the case is ragged."""
    B, ng = c["B"], c["groups"]
    cut = [B * g // ng for g in range(ng + 1)]
    return [x + (1 if c["ragged"] and 0 < g < ng and g % 2 and x + 1 < cut[g + 1] else 0) for g, x in enumerate(cut)]


def _page_bytes(c, e):
    """Bytes of an element of the pages, scales of 4-bit codes included."""
    return {"same": e, "e4m3": 1.0, "mx4": 0.5 + 1 / BLOCK}[c["fmt"]]


def work(c):
    e, d, (lens, new) = DTYPE[c["dtype"]].itemsize, c["d"], _rows(c)
    kv, q = c["L"] * c["Hkv"] * d, c["L"] * c["Hq"] * sum(new) * d * e
    stored = _page_bytes(c, e)
    if c["op"] == "store":  # k and v in, codes out and in again, rows out; queries in and out
        return {"bytes": int(2 * kv * sum(new) * (2 * e + 2 * stored)) + 2 * q,
                "flops": c["L"] * sum(new) * d * (3 * (c["Hq"] + c["Hkv"]) + 4 * c["Hkv"])}
    if c["op"] == "read":
        return {"bytes": int(2 * kv * sum(new) * (e + stored)), "flops": 2 * kv * sum(new)}
    w, s, base = c["window"], c["sinks"], c["T"] // c["page"] * c["page"] if c["op"] == "shared" else 0
    pairs = keys = 0
    for length, m in zip(lens, new):
        p = torch.arange(length - m, length, dtype=torch.int64)
        lo = (p - w + 1).clamp(min=0) if w else torch.zeros_like(p)
        pairs += int((p + 1 - lo).sum() + torch.minimum(lo, torch.tensor(s)).sum())
        first = int(lo[0])
        keys += length - max(first, base) + max(0, min(s, first) - base)
    if base:  # the shared rows that some sequence of a group sees, once for the group
        f = _first(c)
        for a, z in zip(f, f[1:]):
            first = min(max(0, lens[b] - new[b] - w + 1) if w else 0 for b in range(a, z))
            keys += max(0, base - first) + min(s, first, base)
    return {"bytes": int(2 * kv * keys * stored) + 2 * q, "flops": 4 * c["L"] * c["Hq"] * d * pairs}


def _pow2(s):
    """2^s in fp32 for whole s."""
    return ((s + 127) << 23).to(torch.int32).view(torch.float32)


def _encode8(x):
    """Codes and scale (the least power of two that brings the block's largest value to 448 or less) of fp32
    blocks over the last two axes."""
    m, e = torch.frexp(x.abs().amax((-1, -2)))
    scale = _pow2(torch.where(m == 0, 0, (e - torch.where(m <= 0.875, 9, 8)).clamp(-126, 127)))
    return (x / scale[..., None, None]).to(E4M3), scale


def _encode4(x):
    """4-bit codes of fp32 rows x [.., d], packed two to a byte (the even channel low), and their scales' exponents + 127 for
    each 32 channels: the least power of two that brings the block's largest value to 6 or less; codes to nearest, halves to
    even codes."""
    y = x.unflatten(-1, (-1, BLOCK))
    m, e = torch.frexp(y.abs().amax(-1))
    s = torch.where(m == 0, 0, (e - torch.where(m <= 0.75, 3, 2)).clamp(-126, 125))
    y = y * _pow2(-s)[..., None]
    a = y.abs()
    code = sum(t.to(torch.uint8) for t in (a > 0.25, a >= 0.75, a > 1.25, a >= 1.75, a > 2.5, a >= 3.5, a > 5))
    code = (code | (torch.signbit(y).to(torch.uint8) << 3)).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (s + 127).to(torch.uint8)


def _decode4(codes, scale):
    """fp32 rows of packed codes [.., d / 2] and scale bytes [.., d / 32]."""
    value = torch.tensor(E2M1 + tuple(-x for x in E2M1), device=codes.device)
    x = value[torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()]
    return (x.unflatten(-1, (-1, BLOCK)) * _pow2(scale.to(torch.int32) - 127)[..., None]).flatten(-2)


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, L, B, Hkv, Hq, d, n, page = DTYPE[c["dtype"]], c["L"], c["B"], c["Hkv"], c["Hq"], c["d"], c["n"], c["page"]
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=dt)  # noqa: E731
    # keys have four channels of eight times the spread, as trained models' keys do
    spread = torch.ones(d, device="cuda", dtype=dt)
    spread[torch.randperm(d, generator=g, device="cuda")[:4]] = 8
    lens, new = _rows(c)
    on = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    s = dict(case=c, sm=1.0 / math.sqrt(d))
    M = -(-max(lens) // page) + 2
    if c["op"] == "shared":  # each group's pages, then each sequence's own
        f, NP = _first(c), c["T"] // page
        P = c["groups"] * NP + B * (M - NP)
        pages = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
        member = on([sum(b >= x for x in f[1:-1]) for b in range(B)])
        table = torch.cat([pages[: c["groups"] * NP].view(c["groups"], NP)[member.long()], pages[c["groups"] * NP:].view(B, M - NP)], 1)
        s.update(first=on(f), shared_rows=on([NP * page] * c["groups"]), member=member.long(), table=table.contiguous())
    else:
        P = B * M
        s["table"] = torch.randperm(P, generator=g, device="cuda").to(torch.int32).view(B, M)
    s.update(lens=on(lens), n_valid=on(new) if c["ragged"] else None)
    pool, ks, vs, kt, vt = (L, P, Hkv, page, d), None, None, None, None
    if c["op"] == "store":
        s.update(q=normal(L, B, Hq, n, d), k=normal(L, B, Hkv, n, d) * spread, v=normal(L, B, Hkv, n, d))
        s["q_out"] = torch.zeros_like(s["q"])
        half = torch.arange(d // 2, dtype=torch.float64, device="cuda")
        angle = torch.arange(c["T"], dtype=torch.float64, device="cuda")[:, None] * ROPE_BASE ** (-2 * half / d)
        s["rope"] = torch.stack([angle.cos(), angle.sin()], -1).float()
        kp, vp = (torch.zeros(L, P, Hkv, page, d // 2, device="cuda", dtype=torch.uint8) for _ in range(2))
        ks, vs = (torch.zeros(L, P, Hkv, d // BLOCK, page, device="cuda", dtype=torch.uint8) for _ in range(2))
    else:
        kp, vp = normal(*pool) * spread, normal(*pool)
        if c["fmt"] == "mx4":
            (kp, ks), (vp, vs) = _encode4(kp.float()), _encode4(vp.float())
            ks, vs = ks.transpose(-1, -2).contiguous(), vs.transpose(-1, -2).contiguous()
        elif c["fmt"] == "e4m3":
            kt, vt = normal(L, B, Hkv, 2 * page, d) * spread, normal(L, B, Hkv, 2 * page, d)
            (kp, ks), (vp, vs) = _encode8(kp.float()), _encode8(vp.float())
    if c["op"] in ("store", "read"):
        s["k_back"], s["v_back"] = (torch.zeros(L, B, Hkv, n, d, device="cuda", dtype=dt) for _ in range(2))
    else:
        s["q"] = normal(L, B, Hq, n, d)
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(L, B, Hq, n, device="cuda")
    s.update(k_pages=kp, v_pages=vp, k_scale=ks, v_scale=vs, k_tail=kt, v_tail=vt)
    if own:  # the handle that a program keeps: the cache's tensors as one object, and the workspace
        import paper_2501_06807_amd as mpc
        s["kv"] = mpc.PagedKV(kp, vp, s["table"], s["lens"], k_scale=ks, v_scale=vs, k_tail=kt, v_tail=vt, dtype=dt)
        if c["op"] == "paged":
            s["ws"] = mpc.workspace(mpc.paged_attn_workspace_bytes(s["q"], s["kv"]), "cuda")
        if c["op"] == "shared":
            s["ws"] = mpc.workspace(mpc.shared_attn_workspace_bytes(s["q"], s["kv"], c["groups"]), "cuda")
    return s


def _own(s):
    import paper_2501_06807_amd as mpc
    c = s["case"]
    if c["op"] == "store":
        mpc.mpc_paged_append(s["k"], s["v"], s["kv"], q=s["q"], q_out=s["q_out"], rope=s["rope"], rope_style=c["style"],
                             n_valid=s["n_valid"])
    if c["op"] in ("store", "read"):
        mpc.mpc_paged_read(s["kv"], s["k_back"], s["v_back"], n_valid=s["n_valid"])
        return _read(s)
    kw = dict(sm_scale=s["sm"], window=c["window"], sinks=c["sinks"], n_valid=s["n_valid"], lse=s["lse"], ws=s["ws"])
    if c["op"] == "paged":
        mpc.mpc_paged_attn(s["q"], s["kv"], s["out"], **kw)
    else:
        mpc.mpc_shared_attn(s["q"], s["kv"], s["out"], first=s["first"], shared_rows=s["shared_rows"], **kw)
    return {"out": s["out"], "lse": s["lse"]}


def _read(s):
    return {k: s[k] for k in ["k_back", "v_back"] + (["q_out"] if s["case"]["op"] == "store" else [])}


def _new(s):
    """(row of the cache of each new token, whether it is one) [B][n]."""
    lens = s["lens"].long()
    new = s["n_valid"].long() if s["n_valid"] is not None else torch.full_like(lens, s["case"]["n"])
    t = torch.arange(s["case"]["n"], device="cuda")
    return (lens - new)[:, None] + t, t < new[:, None]


def _plain_store(s):
    c = s["case"]
    L, B, Hkv, n, d = s["k"].shape
    at, live = _new(s)
    at = at.clamp(0, c["T"] - 1)
    cs = s["rope"][at][:, None]
    co, si = cs[..., 0], cs[..., 1]

    def turn(x):
        y = x.float()
        a, b = (y[..., : d // 2], y[..., d // 2:]) if c["style"] == "half" else (y[..., 0::2], y[..., 1::2])
        r0, r1 = a * co - b * si, a * si + b * co
        return (torch.cat([r0, r1], -1) if c["style"] == "half" else torch.stack([r0, r1], -1).flatten(-2)).to(x.dtype)

    s["q_out"].copy_(torch.where(live[:, None, :, None], turn(s["q"]), s["q_out"]))
    b, t = torch.nonzero(live, as_tuple=True)
    row = at[b, t]
    page, slot = s["table"].long()[b, row // c["page"]], row % c["page"]
    for name, x in (("k", turn(s["k"])), ("v", s["v"])):
        codes, scale = _encode4(x.transpose(2, 3)[:, b, t].float())  # [L][tokens][Hkv][..]
        s[name + "_pages"][:, page, :, slot] = codes.transpose(0, 1)
        s[name + "_scale"].transpose(3, 4)[:, page, :, slot] = scale.transpose(0, 1)


def _plain_read(s):
    """Rows of the cache by (sequence, row): the newest ones, as the element type holds them."""
    c = s["case"]
    at, live = _new(s)
    b, t = torch.nonzero(live, as_tuple=True)
    row, length = at[b, t], s["lens"].long()[b]
    page, slot = s["table"].long()[b, row // c["page"]], row % c["page"]
    for name in ("k", "v"):
        x = s[name + "_pages"]
        x = x.view(torch.uint8)[:, page, :, slot].view(x.dtype)  # [tokens][L][Hkv][d]
        if c["fmt"] == "mx4":
            x = _decode4(x, s[name + "_scale"].transpose(3, 4)[:, page, :, slot])
        elif c["fmt"] == "e4m3":
            x = x.float() * s[name + "_scale"][:, page].transpose(0, 1)[..., None]
            ring = s[name + "_tail"][:, b, :, row % (2 * c["page"])]
            x = torch.where((row >= length // c["page"] * c["page"])[:, None, None, None], ring.float(), x)
        s[name + "_back"].transpose(2, 3)[:, b, t] = x.transpose(0, 1).to(s[name + "_back"].dtype)
    return _read(s)


def _pages(s, name, ids):
    """fp32 rows [L][X][Hkv][N page][d] of the pages ids [X][N]."""
    x, fmt = s[name + "_pages"], s["case"]["fmt"]
    x = x.view(torch.uint8)[:, ids].view(x.dtype)  # [L][X][N][Hkv][page][..]
    if fmt == "mx4":
        x = _decode4(x, s[name + "_scale"][:, ids].transpose(-1, -2))
    elif fmt == "e4m3":
        x = x.float() * s[name + "_scale"][:, ids][..., None, None]
    return x.float().transpose(2, 3).flatten(3, 4)


def _part(s, q, k, v, see):
    """Largest score, sum of weights and weighted values of rows q [L][X][Hkv][m][d] over k, v [L][X][Hkv][N][d]; see
    [X][m][N], or None where every row sees every key."""
    scores = torch.matmul(q, k.transpose(-1, -2)).mul_(s["sm"])
    if see is not None:
        scores.masked_fill_(~see[None, :, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    w = scores.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    return top, w.sum(-1, keepdim=True), torch.matmul(w, v)


def _plain_attn(s):
    c = s["case"]
    L, B, Hq, n, d = s["q"].shape
    Hkv, page, w, lens = c["Hkv"], c["page"], c["window"], s["lens"].long()
    pos, live = _new(s)
    base = c["T"] // page if c["op"] == "shared" else 0  # shared pages
    see = lambda p, j: (j <= p) & ((j > p - w) | (j < c["sinks"])) if w else j <= p  # noqa: E731
    # each sequence's own rows
    NP = max(1, -(-(c["T"] if c["op"] != "shared" else max(_rows(c)[0])) // page) - base)
    j = torch.arange(base * page, (base + NP) * page, device="cuda")
    have = j < lens[:, None]
    kv = []
    for name in ("k", "v"):
        x = _pages(s, name, s["table"][:, base:base + NP].long())
        if c["fmt"] == "e4m3":
            ring = s[name + "_tail"][:, :, :, j % (2 * page)].float()
            x = torch.where((j >= (lens // page * page)[:, None])[None, :, None, :, None], ring, x)
        kv.append(torch.where(have[None, :, None, :, None], x, 0.0))
    rows = s["q"].float().reshape(L, B, Hkv, -1, d)
    at = pos.repeat(1, Hq // Hkv)  # [B][G n]
    top, total, acc = _part(s, rows, *kv, see(at[..., None], j) & have[:, None])
    if base:  # the shared rows, once for the rows of all sequences of a group
        f = s["first"].long()
        m = int(max(b - a for a, b in zip(_first(c), _first(c)[1:])))
        who = (f[:-1, None] + torch.arange(m, device="cuda")).clamp(max=B - 1)  # [groups][m]
        ids = s["table"][f[:-1], :base].long()
        j = torch.arange(base * page, device="cuda")
        block = rows[:, who].transpose(2, 3).flatten(3, 4)  # [L][groups][Hkv][m G n][d]
        part = _part(s, block, _pages(s, "k", ids), _pages(s, "v", ids), see(at[who].flatten(1)[..., None], j) if w else None)
        idx = torch.arange(B, device="cuda") - f[:-1][s["member"]]
        t2, l2, a2 = (x.unflatten(3, (m, -1)).transpose(2, 3)[:, s["member"], idx] for x in part)
        both = torch.maximum(top, t2)
        ref = torch.where(both == -math.inf, 0.0, both)
        f1, f2 = torch.exp(top - ref), torch.exp(t2 - ref)
        top, total, acc = both, total * f1 + l2 * f2, acc * f1 + a2 * f2
    out = (acc / torch.where(total == 0, 1.0, total)).to(s["q"].dtype).reshape(s["q"].shape)
    lse = (total.log() + torch.where(top == -math.inf, 0.0, top)).reshape(L, B, Hq, n)
    live = live[None, :, None]
    return {"out": torch.where(live[..., None], out, s["out"]), "lse": torch.where(live, lse, s["lse"])}


def run(s):
    if own:
        return _own(s)
    op = s["case"]["op"]
    if op == "store":
        _plain_store(s)
    return _plain_read(s) if op in ("store", "read") else _plain_attn(s)


def _nearest4(y):
    """64-bit rows as their 4-bit codes give them back."""
    u = y.unflatten(-1, (-1, BLOCK))
    top = u.abs().amax(-1, keepdim=True)
    scale = 2.0 ** torch.where(top > 0, torch.ceil(torch.log2(top / 6)), torch.zeros_like(top)).clamp(-126, 125)
    u = u / scale
    grid = 2.0 ** torch.floor(torch.log2(u.abs().clamp(min=1.0))) / 2  # steps of one binary place
    return (torch.round(u / grid) * grid * scale).flatten(-2)


def _stored(s, l, b, a, z):
    """K and V rows [a, z) of sequence b in layer l, [Hkv][z - a][d] in 64 bits."""
    c, page = s["case"], s["case"]["page"]
    r = torch.arange(a, z, device="cuda")
    ids, slot = s["table"][b].long()[r // page], r % page
    value = torch.tensor(E2M1, dtype=torch.float64, device="cuda")
    both = []
    for name in ("k", "v"):
        x = s[name + "_pages"][l]
        x = x.view(torch.uint8)[ids, :, slot].view(x.dtype)  # [rows][Hkv][..]
        if c["fmt"] == "mx4":
            y = torch.empty(x.shape[0], c["Hkv"], c["d"], dtype=torch.float64, device="cuda")
            for i, code in enumerate((x & 15, x >> 4)):
                y[..., i::2] = value[(code & 7).long()] * (1 - 2 * (code >> 3).double())
            e = s[name + "_scale"][l][ids, :, :, slot].double() - 127
            x = y * (2.0 ** e).repeat_interleave(BLOCK, -1)
        elif c["fmt"] == "e4m3":
            x = x.double() * s[name + "_scale"][l, ids].double()[..., None]
            done = int(s["lens"][b]) // page * page
            if z > done:
                newest = slice(max(done - a, 0), None)
                x[newest] = s[name + "_tail"][l, b][:, r[newest] % (2 * page)].transpose(0, 1).double()
        both.append(x.double().transpose(0, 1))
    return both


def exact(c, seed):
    s = prepare(c, seed)
    lens, new = _rows(c)
    if c["op"] == "store":
        d = c["d"]
        first = torch.arange(d // 2, device="cuda") * (1 if c["style"] == "half" else 2)
        second = first + (d // 2 if c["style"] == "half" else 1)
        freq = ROPE_BASE ** (-2 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
        res = {k: x.double() for k, x in _read(s).items()}
        for b, (length, m) in enumerate(zip(lens, new)):
            angle = torch.arange(length - m, length, dtype=torch.float64, device="cuda")[:, None] * freq
            rows = {}
            for name in ("q", "k"):
                x = s[name][:, b, :, :m].double()
                z = torch.complex(x[..., first], x[..., second]) * torch.polar(torch.ones_like(angle), angle)
                x[..., first], x[..., second] = z.real, z.imag
                rows[name] = x
            res["q_out"][:, b, :, :m] = rows["q"]
            # codes are made from the rows as the element type holds them
            res["k_back"][:, b, :, :m] = _nearest4(rows["k"].to(DTYPE[c["dtype"]]).double())
            res["v_back"][:, b, :, :m] = _nearest4(s["v"][:, b, :, :m].double())
        return res
    if c["op"] == "read":
        res = {k: x.double() for k, x in _read(s).items()}
        for l in range(c["L"]):
            for b, (length, m) in enumerate(zip(lens, new)):
                res["k_back"][l, b, :, :m], res["v_back"][l, b, :, :m] = _stored(s, l, b, length - m, length)
        return res
    out, lse = s["out"].double(), s["lse"].double()
    G = c["Hq"] // c["Hkv"]
    for l in range(c["L"]):
        for b, (length, m) in enumerate(zip(lens, new)):
            k, v = _stored(s, l, b, 0, length)
            j = torch.arange(length, device="cuda")
            for h in range(c["Hkv"]):
                heads, p = slice(h * G, (h + 1) * G), torch.arange(length - m, length, device="cuda")[:, None]
                score = (s["q"][l, b, heads, :m].double().flatten(0, 1) @ k[h].T).unflatten(0, (G, m)) * s["sm"]
                gone = j > p
                if c["window"]:
                    gone |= (j <= p - c["window"]) & (j >= c["sinks"])
                score.masked_fill_(gone, -math.inf)
                norm = torch.logsumexp(score, -1)
                out[l, b, heads, :m] = torch.exp(score - norm[..., None]) @ v[h]
                lse[l, b, heads, :m] = norm
    return {"out": out, "lse": lse}
