"""The operators of serving many sequences at once, and the sizes that work on them is measured at:
the paged key / value cache (quantising what is written, reading it back), the attention of a few
new positions of every sequence over it, and drawing tokens from logits.

Each has a plain form in elementary torch operations and 32 bits, a definition in 64 bits
(`exact`), and the framework's call.  Sizes are those of the repository's model shapes (32 heads;
28 query / 4 kv heads; 4 and 12 / 4 heads of 64) and workloads (prompt 256 + generation 256,
512 + 1024, 384 + 512, blocks of 32 positions), and generic ones.
"""
import math

import torch

own = False  # True: run() makes the framework's calls

E_MIN = -64  # smallest exponent of a cached vector's power-of-two scale
_context = None


def _ctx():
    """One context for all cases; its stream is ordered with the default stream that torch works on."""
    global _context
    import paper_2607_20467_gb300 as dcl
    if _context is None:
        _context = dcl.Context(None, 1, 1)
    return dcl, _context


# ------------------------------------------------------------------ cases
def _cache(op, name, fmt, heads, kv, hd, page, **more):
    return dict(name=name, op=op, fmt=fmt, heads=heads, kv=kv, hd=hd, page=page, **more)


def _attn(name, fmt, heads, kv, hd, page, batch, length, new, causal=0, ragged=0):
    return _cache("attention", name, fmt, heads, kv, hd, page, batch=batch, length=length, new=new, causal=causal,
                  ragged=ragged)


def listed():
    return [
        # one block of 32 positions of one sequence, 32 kv heads: what a step between refreshes writes
        _cache("write", "write-block", "fp8", 32, 32, 128, 64, rows=32, pad=0),
        # a refresh of 8 sequences of 1536 positions, taken out of the fused q | k | v rows
        _cache("write", "write-refresh", "fp8", 32, 32, 128, 64, rows=12288, pad=0),
        # one ragged sequence's 1001 positions read back, few kv heads
        _cache("read", "read-sequence", "fp8", 28, 4, 128, 16, rows=1001, pad=0),
        # 8 sequences of 1536 positions read back (moved to another pool, or to a dense step)
        _cache("read", "read-pool", "fp8", 32, 32, 128, 64, rows=12288, pad=0),
        # one new token of one sequence of 512 positions: latency
        _attn("token-b1", "fp8", 32, 32, 128, 64, 1, 512, 1),
        # one new token of each of 64 sequences of up to 4096 positions, grouped heads
        _attn("token-b64", "fp8", 28, 4, 128, 16, 64, 4096, 1, ragged=1),
        # one new token of two sequences of 131071 positions, grouped heads
        _attn("token-long", "fp8", 28, 4, 128, 64, 2, 131071, 1),
        # the block of 32 positions of 8 sequences of 1536, unquantised cache
        _attn("block-b8", "bf16", 32, 32, 128, 64, 8, 1536, 32),
        # the block of 32 positions of 16 long sequences, grouped heads: 224 rows share a kv head
        _attn("block-gqa-b16", "fp8", 28, 4, 128, 32, 16, 8192, 32),
        # one row of a small odd vocabulary: latency
        dict(name="sample-row", op="sample", rows=1, vocab=4095, top_k=0, top_p=0.9, min_p=0.0, temperature=0.8),
        # the block of 32 positions of one sequence, all three truncations
        dict(name="sample-block", op="sample", rows=32, vocab=126464, top_k=50, top_p=0.95, min_p=0.02,
             temperature=0.7),
        # 512 positions (blocks of 16 sequences) over the whole vocabulary
        dict(name="sample-batch", op="sample", rows=512, vocab=152064, top_k=0, top_p=1.0, min_p=0.0,
             temperature=1.0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


_HEADS = ((32, 32, 128), (28, 4, 128), (4, 4, 64), (12, 4, 64), (16, 2, 128), (8, 1, 128))


def draw(rng):
    op = rng.choice(("write", "read", "attention", "attention", "sample", "sample"))
    if op == "sample":
        vocab = _log(rng, 257, 152064)
        rows = _log(rng, 1, min(512, 40_000_000 // vocab))
        return dict(op=op, rows=rows, vocab=vocab, top_k=rng.choice((0, _log(rng, 1, vocab))),
                    top_p=rng.choice((1.0, round(rng.uniform(0.1, 0.99), 3))),
                    min_p=rng.choice((0.0, round(rng.uniform(0.001, 0.3), 3))),
                    temperature=round(rng.uniform(0.2, 2.0), 2))
    heads, kv, hd = rng.choice(_HEADS)
    fmt, page = rng.choice(("fp8", "fp8", "bf16")), rng.choice((16, 32, 64, 128))
    token = 2 * kv * hd * (1 if fmt == "fp8" else 2)  # bytes of a cached position
    if op != "attention":
        rows = _log(rng, 1, min(65536, 60_000_000 // token))
        return dict(op=op, fmt=fmt, heads=heads, kv=kv, hd=hd, page=page, rows=rows, pad=rng.choice((0, 1)))
    batch, new = _log(rng, 1, 64), rng.choice((1, 1, _log(rng, 2, 64)))
    most = min(131072, 200_000_000 // (token * batch), 110_000_000 // (batch * heads * new))
    return dict(op=op, fmt=fmt, heads=heads, kv=kv, hd=hd, page=page, batch=batch, length=_log(rng, max(new, 16), most),
                new=new, causal=rng.choice((0, 1)), ragged=rng.choice((0, 1)))


def _lengths(c):
    """Cached positions and new positions of each sequence: sequence 0 has the most of both; the ragged
    others are spread evenly, each from another place."""
    n, new = [c["length"]] * c["batch"], [c["new"]] * c["batch"]
    if c["ragged"]:
        for b in range(1, c["batch"]):
            u = (b * 0.6180339887498949) % 1.0
            new[b] = 1 + int((b * 0.7548776662466927) % 1.0 * c["new"])
            n[b] = max(new[b], int(c["length"] * u))
    return n, new


def work(c):
    if c["op"] == "sample":
        whole = c["top_k"] == 0 and c["top_p"] >= 1.0 and c["min_p"] <= 0.0
        n = c["rows"] * c["vocab"]  # logits once; the random numbers of the kept tokens
        return {"bytes": n * (6 if whole else 2) + 12 * c["rows"], "flops": (8 if whole else 6) * n}
    es, vec = (1, 1) if c["fmt"] == "fp8" else (2, 0)
    token = 2 * c["kv"] * (c["hd"] * es + vec)  # a cached position: keys and values, and their exponents
    if c["op"] != "attention":
        return {"bytes": c["rows"] * (token + 4 * c["kv"] * c["hd"] + 4), "flops": 2 * c["rows"] * c["kv"] * c["hd"]}
    n, new = _lengths(c)
    q = c["heads"] * c["hd"]
    seen = sum(a * b - (b * (b - 1) // 2 if c["causal"] else 0) for a, b in zip(n, new))
    return {"bytes": sum(n) * token + sum(new) * (4 * q + 4 * c["heads"]), "flops": 4 * seen * q}


# ------------------------------------------------------------------ inputs
def _bf16(shape, gen, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(torch.bfloat16)


def _vectors(shape, gen):
    """Keys or values [tokens][heads][hd]: a channel pattern of each head, and tokens of unlike size."""
    t, h, d = shape
    chan = torch.exp(0.5 * torch.randn(1, h, d, generator=gen, device="cuda"))
    size = torch.exp(0.4 * torch.randn(t, h, 1, generator=gen, device="cuda"))
    return (torch.randn(shape, generator=gen, device="cuda") * chan * size).to(torch.bfloat16)


def _store(c, pages, gen):
    """A pool of `pages` pages in use: k, v [pages][kv][page][hd] and (fp8) their exponents."""
    shape, out = (pages, c["kv"], c["page"], c["hd"]), {}
    for name in ("k", "v"):
        a = _vectors((pages * c["page"], c["kv"], c["hd"]), gen).view(pages, c["page"], c["kv"], c["hd"])
        a = a.transpose(1, 2).contiguous()
        if c["fmt"] == "fp8":
            out[name], out[name + "_exp"] = _quantise(a)
        else:
            out[name] = a
        assert out[name].shape == shape
    return out


def _slots(c, pages, gen):
    """Cache places of the rows: whole pages in a random order; every 17th row is padding where asked."""
    order = torch.randperm(pages, generator=gen, device="cuda")
    at = torch.arange(c["rows"], device="cuda")
    slots = order[at // c["page"]] * c["page"] + at % c["page"]
    if c["pad"]:
        slots = torch.where(at % 17 == 16, torch.full_like(slots, -1), slots)
    return slots.to(torch.int32)


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if c["op"] == "sample":
        R, V = c["rows"], c["vocab"]
        # a trained model's rows: a wide bulk and a few dozen tokens that stand out
        z = 2.0 * torch.randn(R, V, generator=gen, device="cuda")
        top = torch.randint(0, V, (R, min(V, 48)), generator=gen, device="cuda")
        lift = 6.0 + 5.0 * torch.rand(R, min(V, 48), generator=gen, device="cuda")
        z.scatter_add_(1, top, lift)
        s["logits"] = z.to(torch.bfloat16)
        u = torch.rand(R, V, generator=gen, device="cuda").clamp_(1e-20, 1 - 2.0 ** -24)
        s["noise"] = -torch.log(-torch.log(u))
        full = lambda x, t: torch.full((R,), x, dtype=t, device="cuda")
        s["temperature"], s["top_k"] = full(c["temperature"], torch.float32), full(c["top_k"], torch.int32)
        s["top_p"], s["min_p"] = full(c["top_p"], torch.float32), full(c["min_p"], torch.float32)
        s["truncated"] = not (c["top_k"] == 0 and c["top_p"] >= 1.0 and c["min_p"] <= 0.0)
        s["token"], s["prob"], s["conf"] = full(0, torch.int32), full(0, torch.float32), full(0, torch.float32)
        if own:
            s["ctx"] = _ctx()[1]
        return s
    H, G, hd, P = c["heads"], c["kv"], c["hd"], c["page"]
    if c["op"] == "attention":
        n, new = _lengths(c)
        need = [-(-x // P) for x in n]
        pages = sum(need) + 3
        s.update(_store(c, pages, gen))
        order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
        width = max(need)
        table = torch.full((c["batch"], width), -1, dtype=torch.int32)
        at, order = 0, order.cpu()
        for b, k in enumerate(need):
            table[b, :k] = order[at:at + k]
            at += k
        s["table"], s["lens"] = table.cuda(), torch.tensor(n, dtype=torch.int32, device="cuda")
        starts = [0]
        for k in new:
            starts.append(starts[-1] + k)
        s["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
        s["rows"], s["most"], s["longest"], s["scale"] = starts[-1], max(new), max(n), hd ** -0.5
        s["q"] = _bf16((starts[-1], (H + 2 * G) * hd), gen)[:, :H * hd].unflatten(1, (H, hd))
        s["out"] = torch.empty(starts[-1], H, hd, dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.empty(starts[-1], H, dtype=torch.float32, device="cuda")
    else:
        pages = -(-c["rows"] // P) + 3
        s["slots"] = _slots(c, pages, gen)
        if c["op"] == "write":  # k and v stand in the fused q | k | v rows
            qkv = torch.empty(c["rows"], (H + 2 * G) * hd, dtype=torch.bfloat16, device="cuda")
            qkv[:, H * hd:] = torch.cat([_vectors((c["rows"], G, hd), gen).flatten(1) for _ in range(2)], 1)
            s["k_new"] = qkv[:, H * hd:(H + G) * hd].unflatten(1, (G, hd))
            s["v_new"] = qkv[:, (H + G) * hd:].unflatten(1, (G, hd))
            t = torch.float8_e4m3fn if c["fmt"] == "fp8" else torch.bfloat16
            for name in ("k", "v"):
                s[name] = torch.zeros(pages, G, P, hd, device="cuda").to(t)
                if c["fmt"] == "fp8":
                    s[name + "_exp"] = torch.zeros(pages, G, P, dtype=torch.int8, device="cuda")
        else:
            s.update(_store(c, pages, gen))
            s["k_out"] = torch.empty(c["rows"], G, hd, dtype=torch.bfloat16, device="cuda")
            s["v_out"] = torch.empty_like(s["k_out"])
    if own:
        dcl, s["ctx"] = _ctx()
        s["cache"] = dcl.KvCache(s["k"], s["v"], s.get("k_exp"), s.get("v_exp"))
    return s


# ------------------------------------------------------------------ plain forms
def _pow2(e):
    """2^e of whole numbers in [-126, 127], exactly."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _quantise(a):
    """codes (E4M3) and exponents of the last dimension's vectors: e the least integer with
    max|a| <= 448 * 2^e (at least E_MIN; 0 for zeros), codes the nearest values to a / 2^e."""
    f = a.float()
    top = torch.where(torch.isfinite(f), f.abs(), torch.zeros_like(f)).amax(-1)
    m, x = torch.frexp(top)
    e = torch.where(top > 0, (x - 9 + (m > 0.875).to(torch.int32)).clamp_min(E_MIN), torch.zeros_like(x))
    return (f * _pow2(-e).unsqueeze(-1)).to(torch.float8_e4m3fn), e.to(torch.int8)


def _plain_write(s):
    P = s["case"]["page"]
    live = s["slots"] >= 0
    slots = s["slots"][live].long()
    for name in ("k", "v"):
        a = s[name + "_new"][live]
        if s["case"]["fmt"] == "fp8":
            codes, e = _quantise(a)
            s[name].view(torch.uint8)[slots // P, :, slots % P] = codes.view(torch.uint8)
            s[name + "_exp"][slots // P, :, slots % P] = e
        else:
            s[name][slots // P, :, slots % P] = a
    return _pools(s)


def _plain_read(s):
    P = s["case"]["page"]
    live, slots = s["slots"] >= 0, s["slots"].clamp_min(0).long()
    out = {}
    for name in ("k", "v"):
        f = s[name].view(torch.uint8 if s["case"]["fmt"] == "fp8" else torch.bfloat16)[slots // P, :, slots % P]
        if s["case"]["fmt"] == "fp8":
            f = f.view(torch.float8_e4m3fn).float() * _pow2(s[name + "_exp"][slots // P, :, slots % P]).unsqueeze(-1)
        out[name] = torch.where(live[:, None, None], f, torch.zeros_like(f)).to(torch.bfloat16)
    return out


def _plain_attention(s):
    c = s["case"]
    H, G, hd, B, P, new = c["heads"], c["kv"], c["hd"], c["batch"], c["page"], s["most"]
    width = s["table"].shape[1]
    L = width * P
    at = torch.arange(L, device="cuda")
    live = at < s["lens"][:, None]  # [B][L]
    pages = s["table"].clamp_min(0).long()
    k, v = (_gather(s, name, pages).permute(0, 2, 1, 3, 4).reshape(B, G, L, hd) for name in ("k", "v"))
    v = torch.where(live[:, None, :, None], v, torch.zeros_like(v))
    i = torch.arange(new, device="cuda")
    count = (s["starts"][1:] - s["starts"][:-1]).long()
    row = (s["starts"][:-1, None].long() + i).clamp_max(s["rows"] - 1)  # [B][new]
    q = s["q"][row].float().view(B, new, G, H // G, hd).permute(0, 2, 3, 1, 4).reshape(B, G, -1, hd)
    z = (q @ k.transpose(-1, -2)) * s["scale"]  # [B][G][(H / G) new][L]
    seen = live[:, None, :].expand(B, new, L)
    if c["causal"]:
        seen = seen & (at <= (s["lens"][:, None] - count[:, None] + i)[:, :, None])
    seen = seen[:, None, None].expand(B, G, H // G, new, L).reshape(B, G, -1, L)
    z = torch.where(seen, z, torch.full_like(z, -math.inf))
    top = z.amax(-1, keepdim=True)
    e = torch.where(seen, torch.exp(z - top), torch.zeros_like(z))
    total = e.sum(-1, keepdim=True)
    o = torch.where(total > 0, (e @ v) / total, torch.zeros_like(q))
    lse = torch.where(total > 0, top + torch.log(total), torch.full_like(total, -math.inf)).squeeze(-1)
    o = o.view(B, G, H // G, new, hd).permute(0, 3, 1, 2, 4).reshape(B, new, H, hd)
    lse = lse.view(B, G, H // G, new).permute(0, 3, 1, 2).reshape(B, new, H)
    kept = i < count[:, None]
    return {"out": o[kept].to(torch.bfloat16), "lse": lse[kept].contiguous()}


def _gather(s, name, pages):
    """The table's pages [B][width][kv][page][hd] in 32 bits."""
    if name + "_exp" not in s:
        return s[name][pages].float()
    codes = s[name].view(torch.uint8)[pages].view(torch.float8_e4m3fn)
    return codes.float() * _pow2(s[name + "_exp"][pages]).unsqueeze(-1)


def _plain_sample(s):
    V = s["case"]["vocab"]
    z = s["logits"].float()
    z = z - z.amax(-1, keepdim=True)
    y = z * (1.0 / s["temperature"])[:, None]
    w = torch.exp(y)
    if s["truncated"]:
        order = torch.sort(y, dim=-1, descending=True, stable=True).indices
        k = torch.where(s["top_k"] > 0, s["top_k"], torch.full_like(s["top_k"], V)).clamp_max(V)
        by = torch.gather(w, 1, order)
        by = torch.where(torch.arange(V, device="cuda") < k[:, None], by, torch.zeros_like(by))
        before = by.cumsum(-1) - by  # the mass of the tokens before each in that order
        in_p = (before < s["top_p"][:, None] * by.sum(-1, keepdim=True)) | (s["top_p"] >= 1)[:, None]
        in_p[:, 0] = True
        in_k = torch.arange(V, device="cuda") < k[:, None]
        kept = torch.empty_like(in_k).scatter_(1, order, in_p & in_k)
        kept &= (y >= torch.log(s["min_p"])[:, None]) | (s["min_p"] <= 0)[:, None]
        key = torch.where(kept, y + s["noise"], torch.full_like(y, -math.inf))
        total = torch.where(kept, w, torch.zeros_like(w)).sum(-1)
    else:
        key, total = y + s["noise"], w.sum(-1)
    token = key.argmax(-1)
    at = token[:, None]
    full = torch.exp(z)
    return {"token": token.to(torch.int32), "prob": torch.gather(w, 1, at).squeeze(1) / total,
            "conf": torch.gather(full, 1, at).squeeze(1) / full.sum(-1)}


def _pools(s):
    return {name: s[name] for name in ("k", "v", "k_exp", "v_exp") if name in s}


def run(s):
    op = s["case"]["op"]
    if not own:
        return {"write": _plain_write, "read": _plain_read, "attention": _plain_attention, "sample": _plain_sample}[op](s)
    ctx = s["ctx"]
    if op == "write":
        ctx.kv_write(s["cache"], s["k_new"], s["v_new"], s["slots"])
        return _pools(s)
    if op == "read":
        ctx.kv_read(s["cache"], s["slots"], s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"]}
    if op == "attention":
        ctx.kv_attention(s["cache"], s["q"], s["starts"], s["table"], s["lens"], s["out"], max_new=s["most"],
                         causal=bool(s["case"]["causal"]), scale=s["scale"], lse=s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    if s["truncated"]:
        ctx.sample(s["logits"], s["token"], noise=s["noise"], temperature=s["temperature"], top_k=s["top_k"],
                   top_p=s["top_p"], min_p=s["min_p"], prob=s["prob"], conf=s["conf"])
    else:
        ctx.sample(s["logits"], s["token"], noise=s["noise"], temperature=s["temperature"], prob=s["prob"],
                   conf=s["conf"])
    return {"token": s["token"], "prob": s["prob"], "conf": s["conf"]}


# ------------------------------------------------------------------ 64 bits
def _exact_pow2(e):
    return torch.tensor([2.0 ** k for k in range(-128, 128)], dtype=torch.float64, device="cuda")[e.long() + 128]


def _exact_codes(a):
    """E4M3 values of a / 2^e and e, from the grid of the format in 64 bits."""
    a = a.double()
    top = a.abs().amax(-1, keepdim=True)
    e = torch.zeros_like(top)
    for k in range(E_MIN, 121):  # the least exponent that holds the vector
        e = torch.where(top > 448.0 * 2.0 ** (k - 1), torch.full_like(e, float(k)), e)
    x = a / _exact_pow2(e)
    step = torch.full_like(x, 2.0 ** -9)
    for k in range(-5, 9):  # spacing 2^(k - 3) from 2^k on
        step = torch.where(x.abs() >= 2.0 ** k, torch.full_like(x, 2.0 ** (k - 3)), step)
    return torch.round(x / step) * step, e.squeeze(-1)


def exact(case, seed):
    s = prepare(dict(case), seed)
    c = s["case"]
    if c["op"] == "sample":
        z = s["logits"].double()
        if s["truncated"]:
            kept = torch.zeros_like(z, dtype=torch.bool)
            for r in range(c["rows"]):
                v, idx = torch.sort(z[r], descending=True, stable=True)
                w = torch.softmax(v / s["temperature"][r].double(), 0)
                n = c["top_k"] if c["top_k"] > 0 else c["vocab"]
                w = w[:n] / w[:n].sum()
                p = float(s["top_p"][r])
                if p < 1:
                    n = max(1, int((w.cumsum(0) - w < p).sum()))
                ok = w[:n] >= float(s["min_p"][r]) * w[0]
                kept[r, idx[:n][ok]] = True
            z = torch.where(kept, z, torch.full_like(z, -math.inf))
        p = torch.softmax(z / s["temperature"].double()[:, None], -1)
        token = (torch.log(p) + s["noise"].double()).argmax(-1, keepdim=True)
        full = torch.softmax(s["logits"].double(), -1)
        return {"token": None, "prob": p.gather(1, token).squeeze(1), "conf": full.gather(1, token).squeeze(1)}
    P = c["page"]
    if c["op"] == "write":
        out, slots = {}, s["slots"].tolist()
        live = torch.tensor([i for i, x in enumerate(slots) if x >= 0], device="cuda")
        at = s["slots"].long()[live]
        for name in ("k", "v"):
            pool = torch.zeros(s[name].shape[0], P, c["kv"], c["hd"], dtype=torch.float64, device="cuda").flatten(0, 1)
            a = s[name + "_new"][live]
            pool[at] = _exact_codes(a)[0] if c["fmt"] == "fp8" else a.double()
            out[name] = pool.view(-1, P, c["kv"], c["hd"]).transpose(1, 2).contiguous()
            if c["fmt"] == "fp8":
                out[name + "_exp"] = None
        return out
    value = {name: s[name].double() * (_exact_pow2(s[name + "_exp"])[..., None] if c["fmt"] == "fp8" else 1.0)
             for name in ("k", "v")}
    if c["op"] == "read":
        at = s["slots"].long()
        return {name: value[name].transpose(1, 2).flatten(0, 1)[at.clamp_min(0)] * (at >= 0).double()[:, None, None]
                for name in ("k", "v")}
    n, new = _lengths(c)
    H, G = c["heads"], c["kv"]
    out, lse, row = [], [], 0
    for b in range(c["batch"]):
        pages = s["table"][b, :-(-n[b] // P)].long()
        k, v = (value[name][pages].transpose(0, 1).flatten(1, 2)[:, :n[b]] for name in ("k", "v"))  # [G][n][hd]
        q = s["q"][row:row + new[b]].double().transpose(0, 1).unflatten(0, (G, H // G))  # [G][H / G][new][hd]
        z = torch.einsum("ghid,gjd->ghij", q, k) * s["scale"]
        if c["causal"]:
            j, i = torch.arange(n[b], device="cuda"), torch.arange(new[b], device="cuda")
            z = z.masked_fill(j[None, :] > (n[b] - new[b] + i)[:, None], -math.inf)
        lse.append(torch.logsumexp(z, -1).flatten(0, 1).T)
        out.append(torch.einsum("ghij,gjd->ghid", torch.softmax(z, -1), v).flatten(0, 1).transpose(0, 1))
        row += new[b]
    return {"out": torch.cat(out), "lse": torch.cat(lse).contiguous()}
