"""Block decoding of many sequences of different lengths over one paged cache, with sampled tokens.

A masked-diffusion model generates a block of positions at a time (semi-autoregressively).  Each
sequence's prompt is computed once and its keys and values go into its pages.  A step then runs the
current block of every sequence, all in one batch of rows: it writes the block's keys and values
over those of the last step (`Context.kv_write`), lets the block attend to everything its sequence
has cached (`Context.kv_attention`), draws a token for every position that is still masked
(`Context.sample`), and commits the ones whose confidence passes the threshold, or the most
confident one.  A block that is complete runs once more, so that the cache holds the keys and
values of its final tokens, and the next block begins.

    python examples/paged_decode.py                # a small random model, four prompts
    python examples/paged_decode.py --bf16 --greedy

The model's other parts are the library's single-kernel calls (RMSNorm, linear layers) and a few
torch lines (RoPE, SwiGLU); needs a GB300.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_20467_gb300 as dcl  # noqa: E402
import synthetic as syn  # noqa: E402


class PagedModel:
    """A model's weights and its layers' paged caches; `forward` runs any rows of any sequences."""

    def __init__(self, ctx, shape, weights, n_pages, page_len=16, fp8=True):
        self.ctx, self.shape, self.page_len = ctx, shape, page_len
        bf = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(torch.bfloat16).cuda()
        self.embed, self.head, self.norm = bf(weights["embed"]), bf(weights["lm_head"]), bf(weights["final_norm"])
        self.layers = [dict(norm=bf(w["attn_norm"]), qkv=bf(np.concatenate([w["wq"], w["wk"], w["wv"]])), o=bf(w["wo"]),
                            mlp_norm=bf(w["mlp_norm"]), up=bf(np.concatenate([w["w_gate"], w["w_up"]])),
                            down=bf(w["w_down"])) for w in weights["layers"]]
        self.caches = [dcl.KvCache.empty(n_pages, page_len, shape.n_kv_heads, shape.head_dim, fp8=fp8)
                       for _ in weights["layers"]]
        self.free = list(range(n_pages))

    def pages_for(self, positions):
        """Pages for a sequence of this many positions."""
        need = -(-positions // self.page_len)
        if need > len(self.free):
            raise MemoryError(f"{need} pages asked for, {len(self.free)} free")
        return [self.free.pop() for _ in range(need)]

    def release(self, pages):
        self.free.extend(pages)

    def _norm(self, h, gain):
        y = torch.empty(h.shape, dtype=torch.bfloat16, device="cuda")
        self.ctx.op_rmsnorm(h, gain, y, self.shape.rms_eps)
        return y

    def _linear(self, a, w):
        out = torch.empty(a.shape[0], w.shape[0], dtype=torch.bfloat16, device="cuda")
        self.ctx.op_linear(a, w, out)
        return out

    def forward(self, tokens, positions, slots, q_start, table, lens, max_new):
        """Logits [rows][V] of the rows (sequence b's are [q_start[b], q_start[b + 1])); their keys and
        values go to `slots` of every layer's cache, and each sees the first lens[b] positions of its
        sequence.  All arguments are int32 tensors on the device."""
        s = self.shape
        H, G, hd = s.n_heads, s.n_kv_heads, s.head_dim
        half = torch.arange(hd // 2, device="cuda", dtype=torch.float64)
        angle = positions.double()[:, None] * (s.rope_theta ** (-2.0 * half / hd))
        cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

        def rope(x):
            a, b = x.float().split(hd // 2, -1)
            return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(torch.bfloat16)

        h = self.embed[tokens.long()].float()
        for w, cache in zip(self.layers, self.caches):
            qkv = self._linear(self._norm(h, w["norm"]), w["qkv"]).view(-1, H + 2 * G, hd)
            qkv[:, :H + G] = rope(qkv[:, :H + G])
            self.ctx.kv_write(cache, qkv[:, H:H + G], qkv[:, H + G:], slots)
            att = torch.empty(qkv.shape[0], H, hd, dtype=torch.bfloat16, device="cuda")
            self.ctx.kv_attention(cache, qkv[:, :H], q_start, table, lens, att, max_new=max_new)
            self.ctx.op_linear(att.view(-1, H * hd), w["o"], h, mode=1)
            gate, up = self._linear(self._norm(h, w["mlp_norm"]), w["up"]).float().chunk(2, -1)
            self.ctx.op_linear((torch.nn.functional.silu(gate) * up).to(torch.bfloat16), w["down"], h, mode=1)
        return self._linear(self._norm(h, self.norm), self.head)


def generate(model, prompts, gen_len, block=32, tau=0.7, temperature=0.0, top_k=0, top_p=1.0, min_p=0.0, seed=0):
    """Tokens [batch][gen_len] after prompts of any lengths, and the number of denoise steps."""
    n = [len(p) for p in prompts]
    pages = []
    try:
        for k in n:
            pages.append(model.pages_for(k + gen_len))
        return _decode(model, prompts, pages, gen_len, block, tau, seed, temperature, top_k, top_p, min_p)
    finally:  # (also where there were not enough, or a step failed)
        for p in pages:
            model.release(p)


def _decode(model, prompts, pages, gen_len, block, tau, seed, temperature, top_k, top_p, min_p):
    """`generate` in these pages of the sequences."""
    ctx, s, P = model.ctx, model.shape, model.page_len
    B, n = len(prompts), [len(p) for p in prompts]
    i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(seed)
    width = max(len(p) for p in pages)
    table = i32([p + [-1] * (width - len(p)) for p in pages])

    def rows_of(first, count):
        """Positions and slots of rows [first[b], first[b] + count[b]) of every sequence."""
        pos = [np.arange(f, f + c) for f, c in zip(first, count)]
        slot = [np.asarray(pages[b])[x // P] * P + x % P for b, x in enumerate(pos)]
        return i32(np.concatenate(pos)), i32(np.concatenate(slot)), i32(np.concatenate([[0], np.cumsum(count)]))

    pos, slots, starts = rows_of([0] * B, n)  # the prompts: ragged, once
    model.forward(i32(np.concatenate(prompts)), pos, slots, starts, table, i32(n), max(n))

    out = np.full((B, gen_len), s.mask_id, np.int32)
    steps = 0
    for b0 in range(0, gen_len, block):
        size = min(block, gen_len - b0)
        first = [k + b0 for k in n]
        pos, slots, starts = rows_of(first, [size] * B)
        lens = i32([f + size for f in first])
        x = torch.full((B * size,), s.mask_id, dtype=torch.int32, device="cuda")
        done = torch.zeros(B * size, dtype=torch.bool, device="cuda")
        full = lambda v, t: torch.full((B * size,), v, dtype=t, device="cuda")
        token, conf = full(0, torch.int32), full(0.0, torch.float32)
        params = dict(temperature=full(temperature, torch.float32), top_k=full(top_k, torch.int32),
                      top_p=full(top_p, torch.float32), min_p=full(min_p, torch.float32))
        while True:
            logits = model.forward(x, pos, slots, starts, table, lens, size)
            if bool(done.all()):  # that pass left the final tokens' keys and values in the cache
                break
            steps += 1
            u = torch.rand(logits.shape, generator=gen, device="cuda").clamp_(1e-20, 1 - 2.0 ** -24)
            ctx.sample(logits, token, noise=-torch.log(-torch.log(u)), conf=conf, **params)
            c = torch.where(done, torch.full_like(conf, -1.0), conf).view(B, size)
            take = c > tau
            best = torch.zeros_like(take).scatter_(1, c.argmax(1, keepdim=True), True)
            take = (take | (best & ~take.any(1, keepdim=True))).view(-1) & ~done
            x = torch.where(take, token, x)
            done |= take
        out[:, b0:b0 + size] = x.view(B, size).cpu().numpy()
    ctx.synchronise()
    return out, steps


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--gen", type=int, default=64)
    ap.add_argument("--greedy", action="store_true", help="the largest logit instead of a draw")
    ap.add_argument("--bf16", action="store_true", help="an unquantised cache")
    args = ap.parse_args()
    shape = syn.SHAPES["tiny"]
    weights = syn.model_weights(shape, 0, lm_head_scale=40.0, norm_gain_std=0.1)
    prompts = [syn.prompt_ids(i, 1, k, shape.mask_id)[0] for i, k in enumerate((5, 32, 77, 130))]
    with dcl.Context(None, 1, 1) as ctx:
        model = PagedModel(ctx, shape, weights, n_pages=64, fp8=not args.bf16)
        how = {} if args.greedy else dict(temperature=0.8, top_k=50, top_p=0.95)
        out, steps = generate(model, prompts, args.gen, **how)
    for p, t in zip(prompts, out):
        print(f"prompt of {len(p)}: {t[:12].tolist()} ...")
    print(f"{out.size} tokens of {len(prompts)} sequences in {steps} steps")


if __name__ == "__main__":
    main()
