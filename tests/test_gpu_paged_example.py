"""The paged block decoding example (examples/paged_decode.py): its forward against the oracle's
(per block of rows over stored keys and values), and whole generations."""
import os
import sys

import numpy as np
import pytest
import torch

import paper_2607_20467_gb300 as dcl
import synthetic as syn
from oracle import fp8, model as oracle

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import paged_decode  # noqa: E402

pytestmark = pytest.mark.gpu

SHAPE = syn.SHAPES["tiny"]


@pytest.fixture(scope="module")
def setup():
    import __graft_entry__
    __graft_entry__.build()
    weights = syn.model_weights(SHAPE, 0, lm_head_scale=40.0, norm_gain_std=0.1)
    ctx = dcl.Context(None, 1, 1)
    yield ctx, weights
    ctx.close()


def _stored(a, on):
    """What an FP8 cache returns of keys or values [rows][heads][hd]."""
    if not on:
        return a
    flat = a.reshape(-1, a.shape[-1])
    return fp8.dequantise(*fp8.quantise(flat)).reshape(a.shape)


def _oracle_logits(weights, prompt, block, fp8_cache):
    """Logits of the block's rows: the prompt's own pass, then the block over both, keys and values as
    stored."""
    n, m = len(prompt), len(block)
    angles = oracle.rope_angles(n + m, SHAPE.head_dim, SHAPE.rope_theta)
    H, G, hd = SHAPE.n_heads, SHAPE.n_kv_heads, SHAPE.head_dim
    r = oracle.to_bf16
    hs = [np.asarray(weights["embed"], np.float64)[t] for t in (prompt, block)]
    for lw in weights["layers"]:
        w = {k: np.asarray(v, np.float64) for k, v in lw.items()}
        kept = []
        for i, at in enumerate((slice(0, n), slice(n, n + m))):
            h = hs[i]
            xn = r(oracle.rms_norm(h, w["attn_norm"], SHAPE.rms_eps))
            q, k, v = (r(xn @ w[name].T).reshape(len(h), -1, hd) for name in ("wq", "wk", "wv"))
            q, k = r(oracle.apply_rope(q, angles[at])), r(oracle.apply_rope(k, angles[at]))
            kept.append((_stored(k, fp8_cache), _stored(v, fp8_cache)))
            kk, vv = (np.concatenate([x[j] for x in kept]) for j in (0, 1))
            o = np.empty((len(h), H, hd))
            for head in range(H):
                s = q[:, head] @ kk[:, head // (H // G)].T / np.sqrt(hd)
                p = np.exp(s - s.max(1, keepdims=True))
                o[:, head] = (p / p.sum(1, keepdims=True)) @ vv[:, head // (H // G)]
            h = h + r(o.reshape(len(h), -1)) @ w["wo"].T
            xn = r(oracle.rms_norm(h, w["mlp_norm"], SHAPE.rms_eps))
            hs[i] = h + r(oracle.silu(r(xn @ w["w_gate"].T)) * r(xn @ w["w_up"].T)) @ w["w_down"].T
    hn = r(oracle.rms_norm(hs[1], weights["final_norm"], SHAPE.rms_eps))
    return hn @ np.asarray(weights["lm_head"], np.float64).T


@pytest.mark.parametrize("fp8_cache", [False, True])
def test_a_blocks_logits_match_the_oracle(setup, fp8_cache):
    """Ragged prompts, then a block of each, in one batch; logits within 2e-2 of the row's largest (the
    bound of the whole forward's logits, where the same bf16 roundings are)."""
    ctx, weights = setup
    model = paged_decode.PagedModel(ctx, SHAPE, weights, n_pages=32, fp8=fp8_cache)
    lens = (5, 32, 77)
    prompts = [syn.prompt_ids(10 + i, 1, k, SHAPE.mask_id)[0] for i, k in enumerate(lens)]
    m = 20
    blocks = [np.where(np.arange(m) % 3 == 0, SHAPE.mask_id, syn.prompt_ids(20 + i, 1, m, SHAPE.mask_id)[0])
              for i in range(3)]
    pages = [model.pages_for(k + m) for k in lens]
    table = np.full((3, max(map(len, pages))), -1, np.int32)
    for b, p in enumerate(pages):
        table[b, :len(p)] = p
    i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")
    P = model.page_len

    def run(tokens, first):
        pos = [np.arange(f, f + len(t)) for f, t in zip(first, tokens)]
        slots = [table[b][x // P] * P + x % P for b, x in enumerate(pos)]
        starts = np.concatenate([[0], np.cumsum([len(t) for t in tokens])])
        return model.forward(i32(np.concatenate(tokens)), i32(np.concatenate(pos)), i32(np.concatenate(slots)),
                             i32(starts), i32(table), i32([f + len(t) for f, t in zip(first, tokens)]),
                             max(len(t) for t in tokens))

    run(prompts, (0, 0, 0))
    got = run(blocks, lens)
    ctx.synchronise()
    got = got.float().cpu().numpy().astype(np.float64).reshape(3, m, -1)
    for b in range(3):
        want = _oracle_logits(weights, prompts[b], blocks[b], fp8_cache)
        err = np.abs(got[b] - want).max(1) / np.abs(want).max(1)
        assert err.max() <= 2e-2, (b, err.max())


@pytest.mark.parametrize("how", [dict(), dict(temperature=0.8, top_k=50, top_p=0.95, min_p=0.01)])
def test_generations_are_whole_and_repeat(setup, how):
    ctx, weights = setup
    model = paged_decode.PagedModel(ctx, SHAPE, weights, n_pages=64)
    prompts = [syn.prompt_ids(i, 1, k, SHAPE.mask_id)[0] for i, k in enumerate((3, 40, 90))]
    out, steps = paged_decode.generate(model, prompts, 40, block=16, seed=5, **how)
    assert out.shape == (3, 40) and ((0 <= out) & (out < SHAPE.vocab)).all()
    assert 3 <= steps <= 40  # at least a step a block, at most one position a step
    assert sorted(model.free) == list(range(64))  # every page came back
    again, steps2 = paged_decode.generate(model, prompts, 40, block=16, seed=5, **how)
    assert (again == out).all() and steps2 == steps
    alone, _ = paged_decode.generate(model, prompts[1:2], 40, block=16, seed=5)
    if not how:  # a sequence's tokens do not depend on its neighbours (no noise enters a greedy step)
        assert (alone[0] == out[1]).all()


def test_out_of_pages(setup):
    ctx, weights = setup
    model = paged_decode.PagedModel(ctx, SHAPE, weights, n_pages=2)
    with pytest.raises(MemoryError):
        paged_decode.generate(model, [np.zeros(40, np.int32)], 16)
