"""The operators around a paged cache that is held in 4 bits, and the sizes that work on them is
measured at: the plan of a step (pages handed out, rows and slots laid out on the device), the norm
and rotation of queries and keys, keys and values stored in 4 bits and read back, and the
attention over them.

Each has a plain form in elementary torch operations and 32 bits (64 for angles), a definition in 64
bits (`exact`), and the framework's call.  Sizes are those of the repository's model shapes (32
heads; 28 query / 4 kv heads; 4 and 12 / 4 heads of 64) and workloads (prompt 256 + generation 256,
512 + 1024, 384 + 512, blocks of 32 positions), and generic ones.
"""
import math

import torch

own = False  # True: run() makes the framework's calls

GROUP = 32     # components that share a scale
CODES = 252    # scale byte b < CODES: (4 + b % 4) 2^(b // 4 - SHIFT); the others mark a group that holds no numbers
SHIFT = 40
_context = None


def _ctx():
    """One context for all cases; its stream is ordered with the default stream that torch works on."""
    global _context
    import paper_2607_20467_gb300 as dcl
    if _context is None:
        _context = dcl.Context(None, 1, 1)
    return dcl, _context


# ------------------------------------------------------------------ cases
def _plan(name, batch, page, new, ragged, most, short=0):
    """`batch` sequences that have up to `most` positions cached and get `new` rows, or (ragged) up to as many."""
    return dict(name=name, op="plan", batch=batch, page=page, new=new, ragged=ragged, most=most, short=short)


def _rope(name, rows, heads, kv, hd, rot, norm=1, far=0, pad=0):
    return dict(name=name, op="rope", rows=rows, heads=heads, kv=kv, hd=hd, rot=rot, norm=norm, far=far, pad=pad)


def _store(name, rows, heads, kv, hd, page, pad=0):
    return dict(name=name, op="store", rows=rows, heads=heads, kv=kv, hd=hd, page=page, pad=pad)


def _attn(name, heads, kv, hd, page, batch, length, new, causal=0, ragged=0):
    return dict(name=name, op="attention", heads=heads, kv=kv, hd=hd, page=page, batch=batch, length=length, new=new,
                causal=causal, ragged=ragged)


def listed():
    return [
        # the current block of 32 positions of 8 sequences: what every step of a small server begins with
        _plan("plan-blocks", 8, 64, 32, 0, 1536),
        # 256 prompts of up to 1536 positions admitted at once, small pages
        _plan("plan-prompts", 256, 16, 1536, 1, 0),
        # one new token of one sequence, grouped heads: latency
        _rope("rope-token", 1, 28, 4, 128, 128),
        # blocks of 32 positions of 16 sequences in the middle of long contexts, half of a head rotated
        _rope("rope-blocks", 512, 28, 4, 128, 64, far=1, pad=1),
        # a refresh of 8 sequences of 1536 positions, 32 heads
        _rope("rope-refresh", 12288, 32, 32, 128, 128),
        # the block of 32 positions of one sequence stored and read back
        _store("store-block", 32, 32, 32, 128, 64),
        # 8 sequences of 1536 positions stored and read back (what a dense step would compute on)
        _store("store-refresh", 12288, 32, 32, 128, 64),
        # one new token of one sequence of 512 positions: latency
        _attn("token-b1", 32, 32, 128, 64, 1, 512, 1),
        # one new token of each of 64 sequences of up to 4096 positions, grouped heads
        _attn("token-b64", 28, 4, 128, 16, 64, 4096, 1, ragged=1),
        # one new token of two sequences of 131071 positions, grouped heads
        _attn("token-long", 28, 4, 128, 64, 2, 131071, 1),
        # the block of 32 positions of 8 sequences of 1536
        _attn("block-b8", 32, 32, 128, 64, 8, 1536, 32),
        # the block of 32 positions of 16 long sequences, grouped heads: 224 rows share a kv head
        _attn("block-gqa-b16", 28, 4, 128, 32, 16, 8192, 32),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


_HEADS = ((32, 32, 128), (28, 4, 128), (4, 4, 64), (12, 4, 64), (16, 2, 128), (8, 1, 128))


def draw(rng):
    op = rng.choice(("plan", "rope", "store", "attention", "attention"))
    page = rng.choice((16, 32, 64, 128))
    if op == "plan":
        batch = _log(rng, 1, 1024)
        new = _log(rng, 1, max(1, min(4096, 196608 // batch)))
        return _plan("", batch, page, new, rng.choice((0, 1)), rng.choice((0, _log(rng, 1, 4096))), rng.choice((0, 0, 1)))
    heads, kv, hd = rng.choice(_HEADS)
    if op == "rope":
        rows = _log(rng, 1, min(65536, 100_000_000 // ((heads + kv) * hd)))
        return _rope("", rows, heads, kv, hd, rng.choice((hd, hd, hd // 2, hd // 4)), rng.choice((0, 1, 1)),
                     rng.choice((0, 1)), rng.choice((0, 1)))
    if op == "store":
        return _store("", _log(rng, 1, min(65536, 50_000_000 // (kv * hd))), heads, kv, hd, page, rng.choice((0, 1)))
    batch, new = _log(rng, 1, 64), rng.choice((1, 1, _log(rng, 2, 64)))
    most = min(131072, 250_000_000 // (2 * kv * hd * batch), 110_000_000 // (batch * heads * new))
    return _attn("", heads, kv, hd, page, batch, _log(rng, max(new, 16), most), new, rng.choice((0, 1)),
                 rng.choice((0, 1)))


def _spread(c, b):
    """A number in [0, 1) of sequence b, spread evenly over the batch."""
    return (b * 0.6180339887498949) % 1.0


def _plan_rows(c):
    """New rows of each sequence: none for every eighth from the fifth on, which has ended."""
    return [0 if b % 8 == 4 else c["new"] if not c["ragged"] else 1 + int(_spread(c, b) * c["new"]) for b in range(c["batch"])]


def _lengths(c):
    """Cached positions and new positions of each sequence: sequence 0 has the most of both; the ragged
    others are spread evenly, each from another place."""
    n, new = [c["length"]] * c["batch"], [c["new"]] * c["batch"]
    if c["ragged"]:
        for b in range(1, c["batch"]):
            new[b] = 1 + int((b * 0.7548776662466927) % 1.0 * c["new"])
            n[b] = max(new[b], int(c["length"] * _spread(c, b)))
    return n, new


def work(c):
    if c["op"] == "plan":
        rows = sum(_plan_rows(c))  # their slots and positions; starts, counts, pages held; the pages they lie in
        return {"bytes": 8 * rows + 24 * c["batch"] + 4 * (rows // c["page"] + c["batch"]), "flops": 6 * rows}
    if c["op"] == "rope":
        n = c["rows"] * (c["heads"] + c["kv"]) * c["hd"]
        return {"bytes": 4 * n + 4 * c["rows"], "flops": (7 if c["norm"] else 3) * n}
    token = 2 * c["kv"] * (c["hd"] // 2 + c["hd"] // GROUP)  # a cached position: codes and scales
    if c["op"] == "store":  # rows in, codes out; codes in, rows out
        n = 2 * c["rows"] * c["kv"] * c["hd"]
        return {"bytes": 2 * (c["rows"] * (token + 4) + 2 * n), "flops": 4 * n}
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


def _i32(a):
    return torch.as_tensor(a, dtype=torch.int32).cuda()


def _prepare_plan(c, gen):
    P, B = c["page"], c["batch"]
    new = _plan_rows(c)
    start = [0] * B
    if c["most"]:
        at = torch.randint(0, c["most"] + 1, (B,), generator=gen, device="cuda").tolist()
        start = [0 if b % 8 == 4 else a for b, a in enumerate(at)]
    # pages held from the step before: those of what is cached, and some too many (of positions given up)
    more = torch.randint(0, 3, (B,), generator=gen, device="cuda").tolist()
    held = [(3 if b % 8 == 4 else -(-a // P)) + (m if a else 0) for b, (a, m) in enumerate(zip(start, more))]
    need = [-(-(a + k) // P) for a, k in zip(start, new)]
    width = max(3, -(-(c["most"] + max(new)) // P) + 2)
    grow = sum(max(0, k - h) for h, k in zip(held, need))
    back = sum(max(0, h - k) for h, k in zip(held, need))
    left = max(0, grow // 2 - back) if c["short"] else grow + 7  # free pages; short: not all get theirs
    pages = B * width + 8
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    count = _i32(held)
    base = torch.cumsum(count, 0) - count
    col = torch.arange(width, device="cuda")
    mine = col < count[:, None]
    s = {"table": torch.where(mine, order[(base[:, None] + col).clamp_max(pages - 1)], torch.full_like(order[:1], -1)).contiguous()}
    s["held"], s["n_free"] = count, _i32([left])
    s["free"] = torch.full((pages,), -1, dtype=torch.int32, device="cuda")
    s["free"][:left] = order[sum(held):sum(held) + left]
    s["start"], s["new"] = _i32(start), _i32(new)
    rows = sum(new) + 5  # a step's rows are as many as it was captured for: some lie past the last sequence
    s["q_start"], s["seq_len"] = _i32([0] * (B + 1)), _i32([0] * B)
    s["slots"], s["pos"] = _i32([0] * rows), _i32([0] * rows)
    return s


def _prepare_rope(c, gen):
    R, H, G, hd = c["rows"], c["heads"], c["kv"], c["hd"]
    qkv = torch.empty(R, (H + 2 * G) * hd, dtype=torch.bfloat16, device="cuda")  # the fused projection's rows
    qkv[:, :(H + G) * hd] = _vectors((R, H + G, hd), gen).flatten(1)
    qkv[:, (H + G) * hd:] = 0
    s = {"q": qkv[:, :H * hd].unflatten(1, (H, hd)), "k": qkv[:, H * hd:(H + G) * hd].unflatten(1, (G, hd))}
    pos = torch.arange(R, device="cuda") % 1536
    if c["far"]:
        pos = pos + torch.randint(0, 1 << 20, (1,), generator=gen, device="cuda")
    if c["pad"]:  # rows of no sequence, as a plan leaves them
        pos = torch.where(torch.arange(R, device="cuda") % 17 == 16, torch.full_like(pos, -1), pos)
    s["pos"] = pos.to(torch.int32)
    gain = lambda: (1.0 + 0.1 * torch.randn(hd, generator=gen, device="cuda")).to(torch.bfloat16) if c["norm"] else None
    s["q_gain"], s["k_gain"] = gain(), gain()
    s["q_out"] = torch.zeros(R, H, hd, dtype=torch.bfloat16, device="cuda")
    s["k_out"] = torch.zeros(R, G, hd, dtype=torch.bfloat16, device="cuda")
    s["theta"], s["eps"] = 1e6, 1e-6
    return s


def _pool(c, pages, gen=None):
    """A pool of `pages` pages: codes [pages][kv][page][hd / 2] and scales [pages][kv][page][hd / 32], zeros or (gen)
    pages in use."""
    G, P, hd, s = c["kv"], c["page"], c["hd"], {}
    for name in ("k", "v"):
        if gen is None:
            s[name] = torch.full((pages, G, P, hd // 2), 0x88, dtype=torch.uint8, device="cuda")
            s[name + "_exp"] = torch.zeros(pages, G, P, hd // GROUP, dtype=torch.uint8, device="cuda")
            continue
        s[name] = torch.empty(pages, G, P, hd // 2, dtype=torch.uint8, device="cuda")
        s[name + "_exp"] = torch.empty(pages, G, P, hd // GROUP, dtype=torch.uint8, device="cuda")
        step = max(1, 16_000_000 // (G * P * hd))
        for at in range(0, pages, step):
            n = min(step, pages - at)
            a = _vectors((n * P, G, hd), gen).view(n, P, G, hd).transpose(1, 2)
            s[name][at:at + n], s[name + "_exp"][at:at + n] = _quantise(a)
    return s


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if c["op"] == "plan":
        s.update(_prepare_plan(c, gen))
        if own:
            dcl, s["ctx"] = _ctx()
            s["pages"] = dcl.KvPages(s["table"], s["held"], s["free"], s["n_free"], c["page"])
        return s
    if c["op"] == "rope":
        s.update(_prepare_rope(c, gen))
        if own:
            s["ctx"] = _ctx()[1]
        return s
    H, G, hd, P = c["heads"], c["kv"], c["hd"], c["page"]
    if c["op"] == "store":
        R = c["rows"]
        pages = -(-R // P) + 3
        s.update(_pool(c, pages))
        qkv = torch.zeros(R, (H + 2 * G) * hd, dtype=torch.bfloat16, device="cuda")  # k and v in the fused rows
        qkv[:, H * hd:] = torch.cat([_vectors((R, G, hd), gen).flatten(1) for _ in range(2)], 1)
        s["k_new"] = qkv[:, H * hd:(H + G) * hd].unflatten(1, (G, hd))
        s["v_new"] = qkv[:, (H + G) * hd:].unflatten(1, (G, hd))
        order = torch.randperm(pages, generator=gen, device="cuda")
        at = torch.arange(R, device="cuda")
        slots = order[at // P] * P + at % P
        if c["pad"]:
            slots = torch.where(at % 17 == 16, torch.full_like(slots, -1), slots)
        s["slots"] = slots.to(torch.int32)
        s["k_out"] = torch.empty(R, G, hd, dtype=torch.bfloat16, device="cuda")
        s["v_out"] = torch.empty_like(s["k_out"])
    else:
        n, new = _lengths(c)
        need = [-(-x // P) for x in n]
        pages, width = sum(need) + 3, max(need)
        s.update(_pool(c, pages, gen))
        order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32).cpu()
        table, at = torch.full((c["batch"], width), -1, dtype=torch.int32), 0
        for b, k in enumerate(need):
            table[b, :k] = order[at:at + k]
            at += k
        starts = [0]
        for k in new:
            starts.append(starts[-1] + k)
        s["table"], s["lens"], s["starts"] = table.cuda(), _i32(n), _i32(starts)
        s["rows"], s["most"], s["scale"] = starts[-1], max(new), hd ** -0.5
        s["q"] = _bf16((starts[-1], (H + 2 * G) * hd), gen)[:, :H * hd].unflatten(1, (H, hd))
        s["out"] = torch.empty(starts[-1], H, hd, dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.empty(starts[-1], H, dtype=torch.float32, device="cuda")
    if own:
        dcl, s["ctx"] = _ctx()
        s["cache"] = dcl.KvCache(s["k"], s["v"], s["k_exp"], s["v_exp"])
    return s


# ------------------------------------------------------------------ plain forms
def _scales():
    """What the scale bytes stand for, exactly."""
    b = torch.arange(256, device="cuda")
    s = (4 + b % 4).float() * (((b // 4 - SHIFT + 127).int() << 23).view(torch.float32))
    return torch.where(b < CODES, s, torch.full_like(s, math.nan))


def _quantise(a):
    """Codes (two a byte, the even component in the lower half) and scale bytes of groups of 32 of the last
    dimension: the least scale with max|a| <= 7 scale, the nearest whole multiples of it, 8 added.  A group that
    holds NaN or an infinity is marked as none."""
    f = a.float().unflatten(-1, (-1, GROUP))
    fine = torch.isfinite(f).all(-1)
    f = torch.where(fine.unsqueeze(-1), f, torch.zeros_like(f))
    table = _scales()[:CODES]
    b = torch.searchsorted(7.0 * table, f.abs().amax(-1)).clamp_max(CODES - 1)
    u = (torch.round(f / table[b].unsqueeze(-1)).clamp(-7, 7) + 8).to(torch.uint8).flatten(-2)
    b = torch.where(fine, b, torch.full_like(b, 255)).to(torch.uint8)
    return u[..., 0::2] | (u[..., 1::2] << 4), b


def _values(codes, b):
    """What codes and scale bytes stand for, in 32 bits."""
    u = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float() - 8.0
    return (u.unflatten(-1, (-1, GROUP)) * _scales()[b.long()].unsqueeze(-1)).flatten(-2)


def _plain_plan(s):
    P, table, held, free = s["case"]["page"], s["table"], s["held"], s["free"]
    B, width = table.shape
    need = (s["start"] + s["new"] + (P - 1)) // P
    col = torch.arange(width, device="cuda")
    # pages past what a sequence needs go back
    back = (held - need).clamp_min(0)
    given = (col >= need[:, None]) & (col < held[:, None])
    to = s["n_free"] + (torch.cumsum(back, 0) - back)[:, None] + col - need[:, None]
    spare = torch.cat([free, free[:1]])
    spare[torch.where(given, to, torch.full_like(to, free.numel())).flatten()] = table.flatten()
    free.copy_(spare[:-1])
    table.masked_fill_(given, -1)
    held = torch.minimum(held, need)
    there = s["n_free"] + back.sum()
    # in order, sequences get what they lack, up to the first whose pages are not there
    lack = need - held
    upto = torch.cumsum(lack, 0)
    ok = (lack == 0) | (upto <= there)
    taken = (col >= held[:, None]) & (col < need[:, None]) & ok[:, None]
    at = there - 1 - ((upto - lack)[:, None] + col - held[:, None])
    table.copy_(torch.where(taken, free[at.clamp(0, free.numel() - 1)], table))
    s["held"].copy_(torch.where(ok, need, held))
    s["n_free"].copy_((there - torch.where(ok, lack, torch.zeros_like(lack)).sum()).view(1))
    # rows
    give = torch.where(ok, s["new"], torch.zeros_like(lack))
    s["q_start"][1:] = torch.cumsum(give, 0)
    s["seq_len"].copy_(torch.where(ok, s["start"] + s["new"], s["start"]))
    r = torch.arange(s["slots"].shape[0], device="cuda")
    b = torch.searchsorted(s["q_start"][1:], r, right=True).clamp_max(B - 1)
    pos = s["start"][b] + r - s["q_start"][b]
    live = r < s["q_start"][B]
    slot = table[b, (pos // P).clamp(0, width - 1)] * P + pos % P
    s["slots"].copy_(torch.where(live, slot, torch.full_like(slot, -1)))
    s["pos"].copy_(torch.where(live, pos, torch.full_like(pos, -1)))
    return _planned(s)


def _planned(s):
    return {name: s[name] for name in ("table", "held", "free", "n_free", "q_start", "seq_len", "slots", "pos")}


def _turned(x, gain, cos, sin, eps):
    """Heads [rows][heads][hd] normed (where there is a gain) and their first 2 * cos.shape[-1] components rotated."""
    f = x.float()
    if gain is not None:
        f = f / torch.sqrt((f * f).mean(-1, keepdim=True) + eps) * gain.float()
    half = cos.shape[-1]
    a, b = f[..., :half], f[..., half:2 * half]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, f[..., 2 * half:]], -1)


def _plain_rope(s):
    rot = s["case"]["rot"]
    i = torch.arange(rot // 2, device="cuda", dtype=torch.float64)
    angle = s["pos"].double()[:, None] * (s["theta"] ** (-2.0 * i / rot))
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    live = (s["pos"] >= 0)[:, None, None]
    out = {}
    for name in ("q", "k"):
        y = _turned(s[name], s[name + "_gain"], cos, sin, s["eps"]).to(torch.bfloat16)
        out[name] = torch.where(live, y, s[name + "_out"])
    return out


def _plain_store(s):
    P, out = s["case"]["page"], {}
    live = s["slots"] >= 0
    # (a row without a slot stands in for the first that has one, which stores the same once more)
    row = torch.where(live, torch.arange(live.shape[0], device="cuda"), live.to(torch.int32).argmax())
    slots = s["slots"].long()[row]
    page, place = slots // P, slots % P
    for name in ("k", "v"):
        codes, b = _quantise(s[name + "_new"])
        s[name][page, :, place], s[name + "_exp"][page, :, place] = codes[row], b[row]
        y = _values(s[name][page, :, place], s[name + "_exp"][page, :, place])
        out[name] = torch.where(live[:, None, None], y, torch.zeros_like(y)).to(torch.bfloat16)
    return out


def _plain_attention(s):
    c = s["case"]
    H, G, hd, B, P, new = c["heads"], c["kv"], c["hd"], c["batch"], c["page"], s["most"]
    width = s["table"].shape[1]
    L = width * P
    at = torch.arange(L, device="cuda")
    live = at < s["lens"][:, None]  # [B][L]
    pages = s["table"].clamp_min(0).long()
    k = _values(s["k"][pages], s["k_exp"][pages]).permute(0, 2, 1, 3, 4).reshape(B, G, L, hd)
    v = _values(s["v"][pages], s["v_exp"][pages]).permute(0, 2, 1, 3, 4).reshape(B, G, L, hd)
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


def run(s):
    op = s["case"]["op"]
    if not own:
        return {"plan": _plain_plan, "rope": _plain_rope, "store": _plain_store, "attention": _plain_attention}[op](s)
    ctx = s["ctx"]
    if op == "plan":
        ctx.kv_plan(s["pages"], s["start"], s["new"], s["q_start"], s["seq_len"], s["slots"], s["pos"])
        return _planned(s)
    if op == "rope":
        ctx.qk_norm_rope(s["q"], s["k"], s["pos"], s["q_out"], s["k_out"], theta=s["theta"], q_gain=s["q_gain"],
                         k_gain=s["k_gain"], eps=s["eps"], rot_dim=s["case"]["rot"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "store":
        ctx.kv_write(s["cache"], s["k_new"], s["v_new"], s["slots"])
        ctx.kv_read(s["cache"], s["slots"], s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"]}
    ctx.kv_attention(s["cache"], s["q"], s["starts"], s["table"], s["lens"], s["out"], max_new=s["most"],
                     causal=bool(s["case"]["causal"]), scale=s["scale"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


# ------------------------------------------------------------------ 64 bits
def _exact_pow2(k):
    return torch.tensor([2.0 ** x for x in range(-64, 65)], dtype=torch.float64, device="cuda")[k.long() + 64]


def _exact_group(a):
    """The values nearest to a (groups of 32 in the last dimension) among whole multiples -7 .. 7 of the least
    scale (4 .. 7) 2^k, -40 <= k <= 22, that reaches the largest."""
    g = a.double().unflatten(-1, (-1, GROUP))
    top = g.abs().amax(-1, keepdim=True)
    best = torch.full_like(top, math.inf)
    for m in (4.0, 5.0, 6.0, 7.0):
        x, e = torch.frexp(top / (7.0 * m))  # x in [0.5, 1): 2^e reaches it, 2^(e - 1) only where x is 0.5
        k = torch.where(x == 0.5, e - 1, e).clamp(-SHIFT, 22)
        s = m * _exact_pow2(k)
        best = torch.where((s < best) & ((7.0 * s >= top) | (m == 7.0)), s, best)
    return ((g / best).round().clamp(-7, 7) * best).flatten(-2)


def _exact_values(codes, b):
    b = b.double()
    k = torch.floor(b / 4)
    s = (4.0 + b - 4.0 * k) * _exact_pow2(k - SHIFT)
    hi = torch.floor(codes.double() / 16)
    u = torch.stack([codes.double() - 16 * hi, hi], -1).flatten(-2) - 8
    return u * s.repeat_interleave(GROUP, -1)


def exact(case, seed):
    if case["op"] == "plan":
        return None  # (whole numbers only)
    s = prepare(dict(case), seed)
    c = s["case"]
    if c["op"] == "rope":
        out, half = {}, c["rot"] // 2
        turn = s["pos"].double()[:, None] * torch.exp(-math.log(s["theta"]) * torch.arange(half, device="cuda").double() / half)
        w = torch.polar(torch.ones_like(turn), turn)[:, None]
        for name in ("q", "k"):
            x = s[name].double()
            if c["norm"]:
                x = x * torch.rsqrt(x.square().sum(-1, keepdim=True) / c["hd"] + s["eps"]) * s[name + "_gain"].double()
            z = torch.complex(x[..., :half], x[..., half:c["rot"]]) * w
            x = torch.cat([z.real, z.imag, x[..., c["rot"]:]], -1)
            out[name] = x * (s["pos"] >= 0).double()[:, None, None]
        return out
    if c["op"] == "store":
        live = (s["slots"] >= 0).double()[:, None, None]
        return {name: _exact_group(s[name + "_new"]) * live for name in ("k", "v")}
    n, new = _lengths(c)
    H, G, P = c["heads"], c["kv"], c["page"]
    out, lse, row = [], [], 0
    for b in range(c["batch"]):
        pages = s["table"][b, :-(-n[b] // P)].long()
        k, v = (_exact_values(s[name][pages], s[name + "_exp"][pages]).transpose(0, 1).flatten(1, 2)[:, :n[b]]
                for name in ("k", "v"))  # [G][n][hd]
        q = s["q"][row:row + new[b]].double().transpose(0, 1).unflatten(0, (G, H // G))  # [G][H / G][new][hd]
        z = torch.einsum("ghid,gjd->ghij", q, k) * s["scale"]
        if c["causal"]:
            j, i = torch.arange(n[b], device="cuda"), torch.arange(new[b], device="cuda")
            z = z.masked_fill(j[None, :] > (n[b] - new[b] + i)[:, None], -math.inf)
        lse.append(torch.logsumexp(z, -1).flatten(0, 1).T)
        out.append(torch.einsum("ghij,gjd->ghid", torch.softmax(z, -1), v).flatten(0, 1).transpose(0, 1))
        row += new[b]
    return {"out": torch.cat(out), "lse": torch.cat(lse).contiguous()}
