"""The measured cases of the paged cache and its rotary positions: what a
decode loop, or the prefill before it, has each of these operators do.

A case is a dict of plain values; ``op`` names the operator:

  rope    rope_rows: the query and key rows of some tokens rotated by their
          positions (half or interleaved pairs, all or part of the head), or
          rotated back by the same angles, which is the gradient
  write   paged_write: new key and value rows into their pages, in bf16 or
          quantised (e4m3 with a power-of-two exponent a row), keys and
          queries rotated on the way if asked
  read    paged_read: rows of the pages, selected ones or all from the start,
          back as bf16 rows in slot order
  score   paged_score_keys: the group's best logit of every position
  attn    paged_decode_attn: attention of the last one or few tokens over
          everything a request has in its pages

Shapes are the ones of the synthetic workloads and the other performance cases
(head_dim 128, 8 to 64 query heads on 1 to 8 KV heads, contexts from one token
to 2^18) and others of the ranges the interface accepts.  Keys have a
log-normal scale per channel, values are normal.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

D = 128
SCALE = float(np.float32(1.0 / math.sqrt(D)))
MIB = 1 << 20


# ---- the cases -------------------------------------------------------------------
def _rope(tokens, q_heads, kv_heads, first, pairs="half", rot=D, dtype="bf16", back=False,
          scaling="none", **more):
    return {"op": "rope", "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads,
            "first": first, "pairs": pairs, "rot": rot, "dtype": dtype, "back": back,
            "scaling": scaling, **more}


def _cache(op, batch, q_heads, kv_heads, max_ctx, ctx_min, kind, page, **more):
    return {"op": op, "batch": batch, "q_heads": q_heads, "kv_heads": kv_heads,
            "max_ctx": max_ctx, "ctx_min": ctx_min, "kind": kind, "page": page, **more}


def listed():
    return [
        # one decode step of an ordinary batch, far into long contexts: a launch's latency
        _rope(16, 32, 8, 120000, name="rope_decode"),
        # a prefill chunk of a model with stretched frequencies: bandwidth
        _rope(16384, 32, 8, 0, scaling="bands", name="rope_prefill"),
        # the gradient's rotation in fp32, neighbouring pairs, half of the head, odd count
        _rope(4097, 64, 8, 77, pairs="interleaved", rot=64, dtype="f32", back=True,
              name="rope_gradient"),
        # the step's new tokens: queries and keys rotated, rows into bf16 pages
        _cache("write", 64, 32, 8, 2000, 100, "bf16", 16, new=1, rope=True, name="write_decode"),
        # a prefill into a quantised cache, prompts of different lengths
        _cache("write", 5, 32, 8, 6001, 2500, "e4m3", 64, new=0, rope=True,
               name="write_prefill"),
        # the selected rows of a quantised cache, assembled for the sparse attention
        _cache("read", 16, 32, 8, 32768, 32768, "e4m3", 64, k=2048, idx=True,
               name="read_selected"),
        # whole short contexts read back, small pages
        _cache("read", 3, 32, 8, 5003, 1200, "bf16", 16, k=5003, idx=False, name="read_whole"),
        # selection scores of one short request
        _cache("score", 1, 8, 2, 4096, 4096, "bf16", 16, name="score_single"),
        # and of the ordinary serving batch over quantised keys
        _cache("score", 16, 32, 8, 32768, 32768, "e4m3", 64, name="score_batch"),
        # one user alone, a short context: latency of the split and the join
        _cache("attn", 1, 32, 8, 2001, 2001, "bf16", 16, new=1, evict=False, name="attn_single"),
        # a serving batch of very different lengths
        _cache("attn", 64, 32, 8, 32768, 1000, "bf16", 16, new=1, evict=False,
               name="attn_batch"),
        # two long documents, the current and the speculative token together, quantised
        _cache("attn", 2, 64, 8, 200001, 150000, "e4m3", 64, new=2, evict=False,
               name="attn_long"),
    ]


def _logu(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "write", "read", "score", "attn", "attn"])
    kv = rng.choice([1, 2, 4, 8, 8, 8])
    if op == "rope":
        return _rope(_logu(rng, 1, 16384), kv * rng.choice([1, 2, 4, 4, 8]), kv,
                     rng.choice([0, 5, 4000, 131072, 1000003]),
                     pairs=rng.choice(["half", "interleaved"]),
                     rot=rng.choice([128, 128, 64, 96, 32, 20]),
                     dtype=rng.choice(["bf16", "bf16", "f32"]), back=rng.random() < 0.4,
                     scaling=rng.choice(["none", "linear", "bands"]))
    g = rng.choice([1, 2, 4, 4, 8, 16])
    kind = rng.choice(["bf16", "e4m3"])
    page = rng.choice([1, 4, 16, 16, 32, 64, 64, 128, 256])
    # positions over all units: up to what the largest listed case of the operator has
    rows = {"write": 160000, "read": 260000, "score": 4 << 20, "attn": 6 << 20}[op]
    n = min(_logu(rng, 1, {"write": 8192, "read": 32768}.get(op, 262144)), rows // kv)
    if page < 16:
        n = min(n, 20000)
    batch = max(1, min(_logu(rng, 1, 96), rows // (kv * n)))
    lo = n if batch == 1 or rng.random() < 0.3 else max(1, int(n * rng.uniform(0.05, 1.0)))
    more = {}
    if op == "write":
        more = {"new": rng.choice([0, 1, 1, 2]), "rope": rng.random() < 0.7}
    if op == "read":
        more["idx"] = rng.random() < 0.6
        more["k"] = max(1, min(_logu(rng, 1, 4096), n)) if more["idx"] else n
    if op == "attn":
        more["new"] = rng.choice([t for t in (1, 1, 1, 2, 3, 4) if t * g <= 16])
        more["evict"] = rng.random() < 0.2
    return _cache(op, batch, kv * g, kv, n, lo, kind, page, **more)


# ---- sizes -------------------------------------------------------------------------
def _lens(c):
    """Context lengths of the requests, spread over [ctx_min, max_ctx]."""
    lo, hi = c["ctx_min"], c["max_ctx"]
    return [hi - int((hi - lo) * ((b * 0.6180339887498949) % 1.0)) for b in range(c["batch"])]


def _written(c):
    """(request, position) of every token that a write case writes: the last
    `new` ones of each request, or (0) all of them."""
    lens = _lens(c)
    first = [0 if c["new"] == 0 else max(0, n - c["new"]) for n in lens]
    req = np.concatenate([np.full(n - f, b) for b, (n, f) in enumerate(zip(lens, first))])
    pos = np.concatenate([np.arange(f, n) for n, f in zip(lens, first)])
    return req, pos


def _kept(c):
    """For each request the pages it still has: all, or, when the middle of its
    context is evicted, the first page and those of the last 1024 positions."""
    out = []
    for n in _lens(c):
        pages = -(-n // c["page"])
        keep = np.ones(pages, bool)
        if c.get("evict"):
            keep[1:max(1, (n - 1024) // c["page"])] = False
        out.append(keep)
    return out


def _row_bytes(kind):
    return 2 * D if kind == "bf16" else D + 1


def work(c):
    op = c["op"]
    if op == "rope":
        size = 2 if c["dtype"] == "bf16" else 4
        rows = c["tokens"] * (c["q_heads"] + c["kv_heads"])
        return {"bytes": 2.0 * rows * D * size + 4 * c["tokens"], "flops": 3.0 * rows * c["rot"]}
    H, Hq, row = c["kv_heads"], c["q_heads"], _row_bytes(c["kind"])
    lens = _lens(c)
    if op == "write":
        n = len(_written(c)[0])
        by = n * H * 2 * (2 * D + row) + 8 * n
        fl = 2.0 * n * H * 2 * D
        if c["rope"]:
            by += 2 * n * Hq * 2 * D
            fl += 3.0 * n * (H + Hq) * D
        return {"bytes": float(by), "flops": fl}
    if op == "read":
        n = H * sum(min(c["k"], x) for x in lens)
        return {"bytes": float(n * 2 * (row + 2 * D) + (4 * n if c["idx"] else 0)),
                "flops": 2.0 * n * D}
    if op == "score":
        n = H * sum(lens)
        return {"bytes": float(n * row + 4 * len(lens) * H * c["max_ctx"] + 2 * D * len(lens) * Hq),
                "flops": 2.0 * n * (Hq // H) * D}
    n = H * sum(min(int(k.sum()) * c["page"], x) for k, x in zip(_kept(c), lens))
    return {"bytes": float(2 * n * row + 6 * D * len(lens) * Hq * c["new"]),
            "flops": 4.0 * n * (Hq // H) * c["new"] * D}


# ---- inputs ------------------------------------------------------------------------
def _inv_freq(rot, scaling):
    """Radians a position for every pair, float64: base 500000; "linear" for
    contexts eight times as long; "bands" stretches the long wavelengths only."""
    f = 500000.0 ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)
    if scaling == "linear":
        return f / 8
    if scaling == "bands":
        turns = 8192 * f / (2 * math.pi)
        keep = np.clip((turns - 1.0) / (4.0 - 1.0), 0, 1)
        return f * keep + f / 8 * (1 - keep)
    return f


def _pool(c, g, dev):
    """Pages in a shuffled order, as a server that has run for a while has them,
    their table (-1: none) and their rows."""
    H, ps, kind = c["kv_heads"], c["page"], c["kind"]
    keeps = _kept(c)
    per = -(-c["max_ctx"] // ps)
    total = int(sum(k.sum() for k in keeps)) + 3
    order = torch.randperm(total, generator=g, device=dev).to(torch.int32).cpu().numpy()
    table = np.full((c["batch"], per), -1, np.int32)
    at = 0
    for b, k in enumerate(keeps):
        m = int(k.sum())
        table[b, :len(k)][k] = order[at:at + m]
        at += m
    s = {"table": torch.from_numpy(table).to(dev)}
    shape = (total, H, ps, D)
    if kind == "bf16":
        chan = torch.exp(0.5 * torch.randn((1, H, 1, D), generator=g, device=dev)).to(torch.bfloat16)
        s["k_pages"] = torch.randn(shape, generator=g, device=dev, dtype=torch.bfloat16).mul_(chan)
        s["v_pages"] = torch.randn(shape, generator=g, device=dev, dtype=torch.bfloat16)
    else:  # codes of normal values, rows of different exponents
        for name in ("k", "v"):
            codes = torch.empty(shape, dtype=torch.uint8, device=dev)
            flat, piece = codes.view(-1), 256 * MIB
            for i in range(0, flat.numel(), piece):
                part = flat[i:i + piece]
                part.copy_((100 * torch.randn(part.shape, generator=g, device=dev,
                                              dtype=torch.bfloat16)).clamp_(-448, 448)
                           .to(torch.float8_e4m3fn).view(torch.uint8))
            s[name + "_pages"] = codes
            s[name + "_exps"] = torch.randint(119, 122, shape[:3], generator=g, device=dev,
                                              dtype=torch.uint8)
    return s


def prepare(c, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    op, Hq, H = c["op"], c["q_heads"], c["kv_heads"]

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(shape, generator=g, device=dev, dtype=dtype)

    s = {"case": c}
    if op == "rope":
        N, dt = c["tokens"], torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
        s["freq"] = torch.from_numpy(_inv_freq(c["rot"], c["scaling"])).to(dev)
        s["pos"] = torch.arange(c["first"], c["first"] + N, dtype=torch.int32, device=dev)
        # slices of the projection's output, as a model has them
        qkv = normal(N, Hq + 2 * H, D, dtype=dt)
        s["q"], s["k"] = qkv[:, :Hq], qkv[:, Hq:Hq + H]
        s["q_out"] = torch.empty((N, Hq, D), dtype=dt, device=dev)
        s["k_out"] = torch.empty((N, H, D), dtype=dt, device=dev)
        return s
    s.update(_pool(c, g, dev))
    lens = _lens(c)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    if op == "write":
        req, pos = _written(c)
        s["req"] = torch.from_numpy(req.astype(np.int32)).to(dev)
        s["pos"] = torch.from_numpy(pos.astype(np.int32)).to(dev)
        qkv = normal(len(req), Hq + 2 * H, D)
        s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
        s["freq"] = torch.from_numpy(_inv_freq(D, "none")).to(dev)
        s["q_out"] = torch.empty((len(req), Hq, D), dtype=torch.bfloat16, device=dev)
    elif op == "read":
        k = c["k"]
        if c["idx"]:
            top = torch.rand((c["batch"], H, c["max_ctx"]), generator=g, device=dev)
            top.masked_fill_(torch.arange(c["max_ctx"], device=dev) >= s["lens"][:, None, None], -1)
            m = s["lens"].clamp(max=k)
            idx = torch.topk(top, k, dim=-1).indices
            past = (torch.arange(k, device=dev) >= m[:, None, None]).expand_as(idx)
            idx = idx.masked_fill(past, c["max_ctx"]).sort(dim=-1).values
            s["idx"] = idx.masked_fill(past, -1).to(torch.int32)
            s["n_sel"] = m[:, None].expand(-1, H).contiguous()
        s["k_dst"] = torch.zeros((c["batch"], H, k, D), dtype=torch.bfloat16, device=dev)
        s["v_dst"] = torch.zeros_like(s["k_dst"])
    elif op == "score":
        s["q"] = normal(c["batch"], Hq, D)
        s["scores"] = torch.empty((c["batch"], H, c["max_ctx"]), device=dev)
    else:
        s["q"] = normal(c["batch"], c["new"], Hq, D)
        s["out"] = torch.empty((c["batch"], c["new"], Hq, D), device=dev)
        s["lse"] = torch.empty((c["batch"], c["new"], Hq), device=dev)
    return s


# ---- one pass, plain -----------------------------------------------------------------
def _rotate(x, pos, freq, rot, pairs, back):
    """x [N][heads][D] by the angles pos * freq, in fp32 (the angles in fp64)."""
    a = pos.double()[:, None, None] * freq
    cos, sin = torch.cos(a).float(), torch.sin(a).float()
    sin = -sin if back else sin
    y = x.float()
    if pairs == "half":
        x1, x2 = y[..., :rot // 2], y[..., rot // 2:rot]
        r = torch.cat([x1 * cos - x2 * sin, x2 * cos + x1 * sin], -1)
    else:
        x1, x2 = y[..., 0:rot:2], y[..., 1:rot:2]
        r = torch.stack([x1 * cos - x2 * sin, x2 * cos + x1 * sin], -1).flatten(-2)
    return torch.cat([r, y[..., rot:]], -1)


def _quantise(x):
    """fp32 rows -> (e4m3 codes, exponent bytes): the smallest e with
    max |x| <= 448 * 2^e, codes of x / 2^e."""
    m, e = torch.frexp(x.abs().amax(-1))
    e = torch.where(m == 0, -127, torch.where(m <= 0.875, e - 9, e - 8)).clamp(-127, 127)
    codes = torch.ldexp(x, -e[..., None]).to(torch.float8_e4m3fn)
    return codes.view(torch.uint8), (e + 127).to(torch.uint8)


def _rows(pages, exps, table, pos, page):
    """fp32 rows [B][H][n][D] at positions pos ([B][1 or H][n], at least 0), and
    whether each has a page."""
    H = pages.shape[1]
    B = table.shape[0]
    slot = (pos // page).long()
    p = table.gather(1, slot.reshape(B, -1)).view(slot.shape).long()
    at = (p.clamp(min=0), torch.arange(H, device=table.device)[None, :, None], (pos % page).long())
    if exps is None:
        return pages[at].float(), p >= 0
    return torch.ldexp(pages[at].view(torch.float8_e4m3fn).float(),
                       exps[at].int()[..., None] - 127), p >= 0


def _plain(s):
    c = s["case"]
    op, H = c["op"], c["kv_heads"]
    if op == "rope":
        return {n: _rotate(s[n], s["pos"], s["freq"], c["rot"], c["pairs"], c["back"]).to(s[n].dtype)
                for n in ("q", "k")}
    kp, vp, ke, ve = s["k_pages"], s["v_pages"], s.get("k_exps"), s.get("v_exps")
    if op == "write":
        k, v, q = s["k"].float(), s["v"].float(), None
        if c["rope"]:
            k = _rotate(k, s["pos"], s["freq"], D, "half", False)
            q = _rotate(s["q"], s["pos"], s["freq"], D, "half", False).to(torch.bfloat16)
        p = s["table"][s["req"].long(), (s["pos"] // c["page"]).long()].long()
        at = (p[:, None], torch.arange(H, device=p.device)[None], (s["pos"] % c["page"]).long()[:, None])
        for x, pages, exps in ((k, kp, ke), (v, vp, ve)):
            if exps is None:
                pages[at] = x.to(torch.bfloat16)
            else:
                pages[at], exps[at] = _quantise(x)
        return _pages_out(s, q)
    if op == "read":
        k = c["k"]
        pos = s["idx"] if c["idx"] else torch.arange(k, device=kp.device).expand(c["batch"], 1, k)
        n = s["n_sel"][..., None] if c["idx"] else s["lens"][:, None, None]
        ok = (torch.arange(k, device=kp.device) < n)[..., None]
        for pages, exps, dst in ((kp, ke, s["k_dst"]), (vp, ve, s["v_dst"])):
            rows, has = _rows(pages, exps, s["table"], pos.clamp(min=0), c["page"])
            torch.where(ok & has[..., None], rows.to(torch.bfloat16), dst, out=dst)
        return {"k": s["k_dst"], "v": s["v_dst"]}
    B, n, Hq, G = c["batch"], c["max_ctx"], c["q_heads"], c["q_heads"] // H
    pos = torch.arange(n, device=kp.device).expand(B, 1, n)
    k, has = _rows(kp, ke, s["table"], pos, c["page"])
    T = c.get("new", 1)
    q = s["q"].float().view(B, T, H, G, D).permute(0, 2, 4, 1, 3).reshape(B, H, D, T * G)
    logits = torch.matmul(k, q).mul_(SCALE)  # [B][H][n][T*G]
    del k
    end = s["lens"][:, None] - torch.arange(T - 1, -1, -1, device=kp.device)  # [B][T]
    ok = (pos[..., None] < end[:, None, None]) & has[..., None]               # [B][1][n][T]
    logits.masked_fill_(~ok.repeat_interleave(G, -1), -math.inf)
    if op == "score":
        return {"scores": logits.amax(-1)}
    top = logits.amax(2, keepdim=True)
    top = torch.where(top == -math.inf, 0, top)
    w = torch.exp(logits.sub_(top))
    total = w.sum(2)                                                           # [B][H][T*G]
    v, _ = _rows(vp, ve, s["table"], pos, c["page"])
    o = torch.matmul(w.transpose(2, 3).contiguous(), v) / total.clamp(min=1e-30)[..., None]
    lse = top[:, :, 0] + torch.log(total)
    return {"out": o.view(B, H, T, G, D).transpose(1, 2).reshape(B, T, Hq, D),
            "lse": lse.view(B, H, T, G).transpose(1, 2).reshape(B, T, Hq)}


def _pages_out(s, q):
    """What a write leaves: every page (codes and exponents as the numbers they
    stand for) and the rotated queries."""
    r = {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if "k_exps" in s:
        r = {n: t.view(torch.float8_e4m3fn) for n, t in r.items()}
        r["k_exps"] = s["k_exps"].view(torch.float8_e8m0fnu)
        r["v_exps"] = s["v_exps"].view(torch.float8_e8m0fnu)
    if q is not None:
        r["q"] = q
    return r


# ---- one pass, through the framework ---------------------------------------------------
def _plan(s):
    """What a program keeps between calls: shape, cache and rotation handles,
    the workspace."""
    import paper_2607_26475_amd as ckv
    c = s["case"]
    p = {"ckv": ckv}
    if c["op"] == "rope":
        dt = ckv.ROPE_BF16 if c["dtype"] == "bf16" else ckv.ROPE_F32
        p["rope"] = ckv.rope_for(s["freq"], head_dim=D, rot_dim=c["rot"], dtype=dt,
                                 layout=ckv.ROPE_HALF if c["pairs"] == "half" else ckv.ROPE_INTERLEAVED,
                                 inverse=c["back"])
        p["q"], p["k"] = ckv.rows_for(s["q"], s["q_out"]), ckv.rows_for(s["k"], s["k_out"])
        return p
    p["shape"] = ckv.shape_for(c["batch"], c["q_heads"], c["kv_heads"], c["max_ctx"])
    p["cache"] = ckv.paged_cache_for(s["k_pages"], s["v_pages"], s["table"], s.get("k_exps"),
                                     s.get("v_exps"))
    if c["op"] == "write":
        p["rope"] = ckv.rope_for(s["freq"], head_dim=D) if c["rope"] else None
        p["q"] = ckv.rows_for(s["q"], s["q_out"]) if c["rope"] else None
    if c["op"] == "attn":
        p["ws"] = ckv.workspace(p["shape"], c["new"], ckv.ENTRY_PAGED_DECODE_ATTN)
    return p


def run(s):
    if not own:
        return _plain(s)
    if "plan" not in s:
        s["plan"] = _plan(s)
    c, p = s["case"], s["plan"]
    ckv, op = p["ckv"], c["op"]
    if op == "rope":
        ckv.rope_rows(p["rope"], s["pos"], p["q"], p["k"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "write":
        ckv.paged_write(p["shape"], p["cache"], s["req"], s["pos"], s["k"], s["v"],
                        rope=p["rope"], q=p["q"])
        return _pages_out(s, s["q_out"] if c["rope"] else None)
    if op == "read":
        ckv.paged_read(p["shape"], p["cache"], s["lens"], s.get("idx"), s.get("n_sel"), c["k"],
                       s["k_dst"], s["v_dst"])
        return {"k": s["k_dst"], "v": s["v_dst"]}
    if op == "score":
        ckv.paged_score_keys(p["shape"], p["cache"], s["q"], s["lens"], SCALE, s["scores"])
        return {"scores": s["scores"]}
    ckv.paged_decode_attn(p["shape"], p["cache"], c["new"], s["q"], s["lens"], SCALE, s["out"],
                          s["lse"], p["ws"])
    return {"out": s["out"], "lse": s["lse"]}


# ---- the definition, in 64 bits ----------------------------------------------------------
def _turned(x, angle, pairs, rot):
    """Each pair as one complex number, times exp(i angle)."""
    x = x.double()
    a, b = ((slice(0, rot // 2), slice(rot // 2, rot)) if pairs == "half"
            else (slice(0, rot, 2), slice(1, rot, 2)))
    z = torch.complex(x[..., a].contiguous(), x[..., b].contiguous())
    z = z * torch.polar(torch.ones_like(angle), angle)[:, None]
    y = x.clone()
    y[..., a], y[..., b] = z.real, z.imag
    return y


def _e4m3(x):
    """Nearest e4m3 numbers (steps of 2^-3 of the leading power, 2^-9 at least)
    of rows over their power of two, and that power."""
    most = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2((most / 448).clamp(min=2.0 ** -127)))
    e = torch.where(most > 448 * 2.0 ** e, e + 1, e)
    e = torch.where((e > -127) & (most <= 448 * 2.0 ** (e - 1)), e - 1, e)
    y = x / 2.0 ** e
    step = 2.0 ** (torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step, 2.0 ** e[..., 0]


def exact(c, seed):
    s = prepare(c, seed)
    op, H = c["op"], c["kv_heads"]
    if op == "rope":
        angle = s["pos"].double()[:, None] * s["freq"]
        angle = -angle if c["back"] else angle
        return {n: _turned(s[n], angle, c["pairs"], c["rot"]) for n in ("q", "k")}
    table, page = s["table"].long(), c["page"]

    def number(name):  # a stored tensor as the numbers it stands for
        t = s[name]
        if name.endswith("exps"):
            return 2.0 ** (t.double() - 127)
        return t.double() if c["kind"] == "bf16" else t.view(torch.float8_e4m3fn).double()

    if op == "write":
        k, q = s["k"].double(), None
        if c["rope"]:
            angle = s["pos"].double()[:, None] * s["freq"]
            k, q = _turned(k, angle, "half", D), _turned(s["q"], angle, "half", D)
        r = {n: number(n) for n in ("k_pages", "v_pages", "k_exps", "v_exps") if n in s}
        p = table[s["req"].long(), s["pos"].long() // page]
        row = s["pos"].long() % page
        for n, x in (("k", k), ("v", s["v"].double())):
            if c["kind"] == "bf16":
                r[n + "_pages"][p, :, row] = x
            else:
                r[n + "_pages"][p, :, row], r[n + "_exps"][p, :, row] = _e4m3(x)
        if q is not None:
            r["q"] = q
        return r

    def request(name, b, at):  # rows [H][len(at)][D] of one request, fp64
        p, row = table[b, at // page].clamp(min=0), at % page
        x = s[name + "_pages"][p, :, row]
        if c["kind"] == "bf16":
            return x.double().transpose(0, 1)
        e = s[name + "_exps"][p, :, row].double() - 127
        return (x.view(torch.float8_e4m3fn).double() * (2.0 ** e)[..., None]).transpose(0, 1)

    dev, lens = table.device, _lens(c)
    if op == "read":
        r = {"k": s["k_dst"].double(), "v": s["v_dst"].double()}
        for b, n in enumerate(lens):
            m = min(c["k"], n)
            for name in ("k", "v"):
                rows = request(name, b, torch.arange(n, device=dev))
                if c["idx"]:
                    at = s["idx"][b, :, :m].long()
                    rows = rows.gather(1, at[..., None].expand(-1, -1, D))
                r[name][b, :, :m] = rows[:, :m]
        return r
    G, T = c["q_heads"] // H, c.get("new", 1)
    outs, lses = [], []
    for b, n in enumerate(lens):
        at = torch.arange(n, device=dev)
        at = at[table[b, at // page] >= 0]
        k = request("k", b, at)
        if op == "score":
            x = torch.stack([(k * s["q"][b, g::G].double()[:, None]).sum(-1) for g in range(G)])
            full = torch.full((H, c["max_ctx"]), -math.inf, dtype=torch.float64, device=dev)
            full[:, at] = x.amax(0) * SCALE
            outs.append(full)
            continue
        v = request("v", b, at)
        o = torch.zeros((T, H, G, D), dtype=torch.float64, device=dev)
        l = torch.full((T, H, G), -math.inf, dtype=torch.float64, device=dev)
        for t in range(T):
            m = int((at < n - (T - 1 - t)).sum())
            if m == 0:
                continue
            x = torch.bmm(s["q"][b, t].double().view(H, G, D), k[:, :m].transpose(1, 2)) * SCALE
            l[t] = torch.logsumexp(x, -1)
            o[t] = torch.bmm(torch.softmax(x, -1), v[:, :m].contiguous())
        outs.append(o.view(T, H * G, D))
        lses.append(l.view(T, H * G))
    if op == "score":
        return {"scores": torch.stack(outs)}
    return {"out": torch.stack(outs), "lse": torch.stack(lses)}
