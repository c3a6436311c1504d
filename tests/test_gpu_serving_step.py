"""The calls of a decode step run together, as they are used: plan, norm and rotation in the fused rows, keys
and values into the cache, attention over it - several steps of sequences that grow, give positions up and
end, eagerly and as one captured graph (bit for bit the same), against 64 bits over what the cache holds.

Tolerance of the attention: see test_gpu_q4_attention.py (2^-8 of the result for its rounding, 2^-11 of sum p |v| for
scores of this size and fewer than 200 keys); of the rotation: test_gpu_qk_rope.py."""
import os
import sys

import numpy as np
import pytest
import torch

import paper_2607_20467_gb300 as dcl
import synthetic as syn
from oracle import fp8, q4

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import paged_decode  # noqa: E402
from test_gpu_kv_plan import Lists  # noqa: E402
from test_gpu_qk_rope import _check as check_rotation  # noqa: E402

pytestmark = pytest.mark.gpu

THETA, EPS = 1e6, 1e-6


def _i32(a):
    return torch.tensor(np.asarray(a, np.int64), dtype=torch.int32, device="cuda")


def _held(a, form):
    """What the cache returns of a [n][heads][hd]."""
    if form == "q4":
        return q4.decode(*q4.encode(a))
    if form == "fp8":
        flat = a.reshape(-1, a.shape[-1])
        return fp8.dequantise(*fp8.quantise(flat)).reshape(a.shape)
    return a


class Step:
    """Buffers of a step of up to `rows` rows, and its calls."""

    def __init__(self, ctx, cache, pages, gains, rows, heads, new):
        i32 = lambda k: torch.full((k,), 99, dtype=torch.int32, device="cuda")
        B, G, hd = pages.batch, cache.n_kv_heads, cache.head_dim
        self.ctx, self.cache, self.pages, self.gains, self.H, self.G, self.most = ctx, cache, pages, gains, heads, G, new
        self.start, self.new = i32(B), i32(B)
        self.q_start, self.seq_len, self.slots, self.pos = i32(B + 1), i32(B), i32(rows), i32(rows)
        self.qkv = torch.zeros(rows, heads + 2 * G, hd, dtype=torch.bfloat16, device="cuda")
        self.out = torch.full((rows, heads, hd), 7.0, dtype=torch.bfloat16, device="cuda")

    def calls(self):
        H, G = self.H, self.G
        q, k, v = self.qkv[:, :H], self.qkv[:, H:H + G], self.qkv[:, H + G:]
        self.ctx.kv_plan(self.pages, self.start, self.new, self.q_start, self.seq_len, self.slots, self.pos)
        self.ctx.qk_norm_rope(q, k, self.pos, q, k, theta=THETA, q_gain=self.gains[0], k_gain=self.gains[1], eps=EPS)
        self.ctx.kv_write(self.cache, k, v, self.slots)
        self.ctx.kv_attention(self.cache, q, self.q_start, self.pages.table, self.seq_len, self.out, max_new=self.most)


@pytest.mark.parametrize("form", ["q4", "fp8", "bf16"])
@pytest.mark.parametrize("heads,kv,hd,page_len,most", [(4, 4, 64, 16, 3), (14, 2, 128, 32, 1), (8, 1, 128, 16, 9)])
def test_steps_of_growing_and_ending_sequences(form, heads, kv, hd, page_len, most):
    import __graft_entry__
    __graft_entry__.build()
    rng = np.random.default_rng(hd + most)
    B, n_pages, width, rows = 5, 64, 12, 5 * most + 3
    stream = torch.cuda.Stream()
    gains = [torch.from_numpy(1 + 0.1 * rng.normal(0, 1, hd)).to(torch.bfloat16).cuda() for _ in range(2)]
    eager_ctx, ctx = dcl.Context(None, 1, 1), dcl.Context(None, 1, 1, stream=stream.cuda_stream)
    steps = []
    for c in (eager_ctx, ctx):
        cache = dcl.KvCache.empty(n_pages, page_len, kv, hd, fp8=form == "fp8", q4=form == "q4")
        steps.append(Step(c, cache, dcl.KvPages.new(n_pages, page_len, B, width), gains, rows, heads, most))
    one, two = steps
    torch.cuda.synchronize()
    two.start.zero_(), two.new.zero_()
    torch.cuda.synchronize()
    two.calls()  # (the attention's first call allocates, which a capture may not)
    ctx.synchronise()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        two.calls()
    lists = Lists(n_pages, page_len, B)
    start = np.zeros(B, np.int64)
    K, V = [np.zeros((0, kv, hd)) for _ in range(B)], [np.zeros((0, kv, hd)) for _ in range(B)]
    for step in range(40 if most == 1 else 12):
        new = rng.integers(0, most + 1, B)
        if step in (5, 9):  # one ends, one gives positions up
            start[0], new[0] = 0, 0
            start[1] = start[1] // 2
        raw = torch.from_numpy(rng.normal(0, 1, (rows, heads + 2 * kv, hd))).to(torch.bfloat16).cuda()
        for s in steps:
            s.start.copy_(_i32(start)), s.new.copy_(_i32(new)), s.qkv.copy_(raw), s.out.fill_(7)
        torch.cuda.synchronize()
        one.calls()
        graph.replay()
        torch.cuda.synchronize()
        eager_ctx.synchronise()
        ctx.synchronise()
        live = int(new.sum())
        for a in ("out", "qkv", "slots", "pos", "q_start", "seq_len"):
            assert torch.equal(getattr(one, a), getattr(two, a)), a
        slots, pos, q_start, lens = lists.plan(start.tolist(), new.tolist())
        assert one.slots.tolist() == slots + [-1] * (rows - live) and one.pos.tolist() == pos + [-1] * (rows - live)
        assert one.q_start.tolist() == q_start and one.seq_len.tolist() == lens
        assert torch.equal(one.qkv[live:], raw[live:]) and (one.out[live:] == 7).all()
        at = one.pos.cpu().numpy().astype(np.int64)
        check_rotation(one.qkv[:, :heads], raw[:, :heads], gains[0], at, hd, THETA, EPS)
        check_rotation(one.qkv[:, heads:heads + kv], raw[:, heads:heads + kv], gains[1], at, hd, THETA, EPS)
        x = one.qkv.double().cpu().numpy()
        got = one.out.double().cpu().numpy()
        for b in range(B):
            sl = slice(q_start[b], q_start[b + 1])
            K[b] = np.concatenate([K[b][:start[b]], _held(x[sl, heads:heads + kv], form)])
            V[b] = np.concatenate([V[b][:start[b]], _held(x[sl, heads + kv:], form)])
            for h in range(heads):
                if not new[b]:
                    continue
                z = x[sl, h] @ K[b][:, h // (heads // kv)].T * hd ** -0.5
                w = np.exp(z - z.max(1, keepdims=True))
                w /= w.sum(1, keepdims=True)
                o, A = w @ V[b][:, h // (heads // kv)], w @ np.abs(V[b][:, h // (heads // kv)])
                assert (np.abs(got[sl, h] - o) <= 2.0 ** -8 * np.abs(o) + 2.0 ** -11 * A).all()
        start = start + new
    for c in (eager_ctx, ctx):
        c.close()


def test_the_example_decodes_over_4_bits():
    shape = syn.SHAPES["tiny"]
    weights = syn.model_weights(shape, 0, lm_head_scale=40.0, norm_gain_std=0.1)
    with dcl.Context(None, 1, 1) as ctx:
        model = paged_decode.PagedModel(ctx, shape, weights, n_pages=64, q4=True)
        prompts = [syn.prompt_ids(i, 1, k, shape.mask_id)[0] for i, k in enumerate((3, 40, 90))]
        out, steps = paged_decode.generate(model, prompts, 40, block=16, seed=5)
        assert out.shape == (3, 40) and ((0 <= out) & (out < shape.vocab)).all() and 3 <= steps <= 40
        assert sorted(model.free) == list(range(64))
        alone, _ = paged_decode.generate(model, prompts[1:2], 40, block=16, seed=5)
        assert (alone[0] == out[1]).all()
