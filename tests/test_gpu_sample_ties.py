"""Ties of dcl_sample go to the lowest index, wherever a row begins in memory.

Equal logits and equal noise give exactly equal scores, so the token is compared exactly.  Rows of an odd
length (and strides of every remainder by 8) begin at every offset from a 16-byte boundary."""
import numpy as np
import pytest
import torch

import paper_2607_20467_gb300 as dcl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    import __graft_entry__
    __graft_entry__.build()
    ctx = dcl.Context(None, 1, 1)
    yield ctx
    ctx.close()


def _draw(ops, z, noise=None, **kw):
    R = z.shape[0]
    token = torch.full((R,), -7, dtype=torch.int32, device="cuda")
    full = lambda x, t: torch.full((R,), x, dtype=t, device="cuda")
    types = dict(temperature=torch.float32, top_k=torch.int32, top_p=torch.float32, min_p=torch.float32)
    ops.sample(z, token, noise=noise, **{k: full(v, types[k]) for k, v in kw.items()})
    ops.synchronise()
    return token.cpu().numpy()


def _rows(R, V, stride, value=0.0):
    wide = torch.full((R, stride), 9.0, dtype=torch.bfloat16, device="cuda")
    z = wide[:, :V]
    z.fill_(value)
    return z


WAYS = [dict(), dict(top_k=5), dict(top_k=100), dict(top_p=0.5), dict(min_p=0.5), dict(top_k=64, top_p=0.9, min_p=0.1),
        dict(temperature=0.0), dict(temperature=0.7, top_k=7)]


@pytest.mark.parametrize("V", [17, 101, 4095, 12345, 152063])
@pytest.mark.parametrize("way", range(len(WAYS)))
def test_flat_rows(ops, V, way):
    """All logits equal: token 0, without noise and with the same noise everywhere."""
    z = _rows(9, V, V)
    assert (_draw(ops, z, **WAYS[way]) == 0).all()
    noise = torch.full((9, V), 0.25, device="cuda")
    assert (_draw(ops, z, noise, **WAYS[way]) == 0).all()


@pytest.mark.parametrize("V", [101, 4095, 152063])
@pytest.mark.parametrize("pad", range(8))
def test_two_equal_leaders(ops, V, pad):
    """Two largest logits, at every distance from the row's beginning that a first vector has: the lower."""
    rng = np.random.default_rng(V + pad)
    R = 16
    z = _rows(R, V, V + pad, -3.0)
    lower = np.arange(R) % 9
    upper = np.minimum(lower + 1 + rng.integers(0, V - 20, R), V - 1)
    for r in range(R):
        z[r, int(lower[r])] = 2.0
        z[r, int(upper[r])] = 2.0
    flat = torch.full((R, V + 4), -0.5, device="cuda")
    for shift in range(4):  # (the noise's alignment chooses how it is read)
        noise = flat[:, shift:shift + V]
        for kw in WAYS:
            assert (_draw(ops, z, noise, **kw) == lower).all(), (shift, kw)
    for kw in WAYS:
        assert (_draw(ops, z, **kw) == lower).all(), kw


@pytest.mark.parametrize("V", [4096, 126464, 152064])
def test_noise_that_is_aligned_as_the_row(ops, V):
    """Whole rows read in vectors, by one CTA and by several: the token with the largest z / T + noise, of
    64-bit scores, where it leads by more than their rounding (1e-5 (1 + |y|)); its probabilities to 1e-5
    (1 + |y|) of themselves."""
    rng = np.random.default_rng(V)
    R = 12
    z = torch.from_numpy(rng.normal(0, 2, (R, V)).astype(np.float32)).to(torch.bfloat16).cuda()
    u = rng.uniform(1e-12, 1 - 1e-7, (R, V))
    noise = torch.from_numpy((-np.log(-np.log(u))).astype(np.float32)).cuda()
    T = torch.from_numpy(rng.uniform(0.3, 2, R).astype(np.float32)).cuda()
    token = torch.full((R,), -7, dtype=torch.int32, device="cuda")
    prob, conf = torch.zeros(R, device="cuda"), torch.zeros(R, device="cuda")
    ops.sample(z, token, noise=noise, temperature=T, prob=prob, conf=conf)
    ops.synchronise()
    d = z.double() - z.double().amax(1, keepdim=True)
    y = d / T.double()[:, None]
    top = torch.topk(y + noise.double(), 2, 1)
    at = token.long()[:, None]
    yt = y.gather(1, at)[:, 0].abs()
    clear = top.values[:, 0] - top.values[:, 1] > 1e-5 * (1 + y.gather(1, top.indices).abs().sum(1))
    assert clear.sum() >= R - 2
    assert (token.long() == top.indices[:, 0])[clear].all()
    want = torch.softmax(y, 1).gather(1, at)[:, 0]
    assert ((prob.double() - want).abs() <= 1e-5 * (1 + yt) * want).all()
    dt = d.gather(1, at)[:, 0].abs()
    want = torch.softmax(d, 1).gather(1, at)[:, 0]
    assert ((conf.double() - want).abs() <= 1e-5 * (1 + dt) * want).all()
