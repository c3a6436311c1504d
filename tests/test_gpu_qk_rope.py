"""dcl_qk_norm_rope against the formula in 64 bits.

Tolerance.  Sums of squares, the root and the gain leave 2^-19 of a normed component (19 additions of fp32, an
approximate root, three products); a sine or cosine is off by 2^-20 (2^-21 of the function, as much of its
argument: 24 bits of at most pi); so a rotated component by 2^-18 (|y_i| + |y_(i + h)|), and by half a step
of bf16, 2^-8 of itself."""
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


def _bf16(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.float64)).to(torch.bfloat16).cuda()


def _double(t):
    return t.double().cpu().numpy()


def _want(x, gain, pos, rot, theta, eps):
    """y and how large it is of what may be off."""
    if gain is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain
    h = rot // 2
    i = np.arange(h)
    f = np.longdouble(theta) ** (-i.astype(np.longdouble) / max(h, 1))
    angle = (pos[:, None].astype(np.longdouble) * f) % (2 * np.longdouble(np.pi))
    c, s = np.cos(angle).astype(np.float64)[:, None], np.sin(angle).astype(np.float64)[:, None]
    a, b = x[..., :h], x[..., h:rot]
    y = np.concatenate([a * c - b * s, b * c + a * s, x[..., rot:]], -1)
    size = np.concatenate([np.abs(a) + np.abs(b)] * 2 + [np.abs(x[..., rot:])], -1)
    return y, size


def _check(got, x, gain, pos, rot, theta, eps):
    live = pos >= 0
    y, size = _want(_double(x)[live], None if gain is None else _double(gain), pos[live], rot, theta, eps)
    err = np.abs(_double(got)[live] - y)
    most = 2.0 ** -8 * np.abs(y) + 2.0 ** -18 * size
    assert (err <= most + 1e-38).all(), (err / (most + 1e-38)).max()


def _run(ops, n, H, G, hd, rot, gains=(True, True), theta=5e5, eps=1e-5, pos=None, in_place=False, seed=0, size=1.0):
    rng = np.random.default_rng(seed)
    qkv = _bf16(rng.normal(0, size, (n, (H + 2 * G) * hd)) * np.exp2(rng.integers(-3, 4, (n, 1))))
    before = qkv.clone()
    q, k = qkv[:, :H * hd].unflatten(1, (H, hd)), qkv[:, H * hd:(H + G) * hd].unflatten(1, (G, hd))
    pos = np.asarray(rng.integers(0, 4096, n) if pos is None else pos, np.int64)
    gq, gk = (_bf16(1 + 0.2 * rng.normal(0, 1, hd)) if g else None for g in gains)
    if in_place:
        qo, ko = q, k
    else:
        wide = torch.full((n, H + G + 1, hd), 55.0, dtype=torch.bfloat16, device="cuda")
        qo, ko = wide[:, G + 1:], wide[:, 1:G + 1]
    ops.qk_norm_rope(q, k, torch.tensor(pos, dtype=torch.int32, device="cuda"), qo, ko, theta=theta, q_gain=gq, k_gain=gk,
                     eps=eps, rot_dim=rot)
    ops.synchronise()
    q0, k0 = before[:, :H * hd].unflatten(1, (H, hd)), before[:, H * hd:(H + G) * hd].unflatten(1, (G, hd))
    _check(qo, q0, gq, pos, rot, theta, eps)
    _check(ko, k0, gk, pos, rot, theta, eps)
    out = torch.from_numpy(pos < 0).cuda()
    if in_place:
        assert torch.equal(qkv[:, (H + G) * hd:], before[:, (H + G) * hd:]) and torch.equal(qkv[out], before[out])
    else:
        assert torch.equal(qkv, before) and (wide[:, 0] == 55).all() and (wide[out] == 55).all()
    return qo, ko


@pytest.mark.parametrize("H,G,hd", [(4, 4, 64), (28, 4, 128), (32, 32, 128), (1, 1, 64), (7, 3, 128), (12, 4, 64)])
@pytest.mark.parametrize("n", [1, 3, 37])
@pytest.mark.parametrize("part", [0, 1, 2, 4])
def test_heads_rows_and_parts_that_rotate(ops, H, G, hd, n, part):
    rot = hd // part // 16 * 16 if part else 0
    _run(ops, n, H, G, hd, rot, seed=n + hd, in_place=n == 3)


@pytest.mark.parametrize("rot", [16, 48, 80, 96, 112])
def test_odd_parts_that_rotate(ops, rot):
    _run(ops, 5, 3, 2, 128, rot)


@pytest.mark.parametrize("gains", [(True, False), (False, True), (False, False)])
@pytest.mark.parametrize("in_place", [False, True])
def test_norms_left_out(ops, gains, in_place):
    _run(ops, 9, 6, 2, 128, 128, gains=gains, in_place=in_place, eps=1e-6 if any(gains) else 0.0)


@pytest.mark.parametrize("theta", [1.0, 1e4, 1e6, 1e9])
def test_far_positions(ops, theta):
    pos = [0, 1, 2, 131071, 1 << 20, (1 << 24) + 1, (1 << 30) - 3, 2 ** 31 - 1]
    _run(ops, 8, 4, 2, 64, 64, pos=pos, theta=theta)


@pytest.mark.parametrize("in_place", [False, True])
def test_rows_of_no_sequence_are_left_as_they_are(ops, in_place):
    _run(ops, 40, 5, 3, 128, 64, pos=np.where(np.arange(40) % 3 == 1, -1 - np.arange(40), np.arange(40)), in_place=in_place)
    _run(ops, 4, 2, 2, 64, 64, pos=[-1] * 4, in_place=in_place)


def test_many_rows(ops):
    _run(ops, 3001, 12, 4, 64, 64, seed=3)
    _run(ops, 1100, 28, 4, 128, 128, seed=4, in_place=True)


def test_large_small_and_strange_values(ops):
    """Squares past fp32's range, zeros, values far below eps, and components that are no numbers (which take
    their head with them and no other)."""
    H, hd = 6, 64
    rng = np.random.default_rng(0)
    x = rng.normal(0, 1, (1, H, hd))
    x[0, 0] *= 1e37
    x[0, 1] *= 3e19
    x[0, 2] = 0
    x[0, 3] *= 1e-30
    x[0, 4, 7] = np.nan
    q, k = _bf16(x), _bf16(x[:, :2])
    gain = _bf16(np.ones(hd))
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    pos = torch.tensor([3], dtype=torch.int32, device="cuda")
    ops.qk_norm_rope(q, k, pos, qo, ko, theta=1e4, q_gain=gain, k_gain=gain, eps=1e-6)
    ops.synchronise()
    some = [0, 1, 2, 3, 5]
    _check(qo[:, some], q[:, some], gain, np.array([3]), hd, 1e4, 1e-6)
    _check(ko, k, gain, np.array([3]), hd, 1e4, 1e-6)
    assert torch.isnan(qo[0, 4]).all()
    q[0, 5, 0] = float("inf")
    ops.qk_norm_rope(q, k, pos, qo, ko, theta=1e4, q_gain=gain, k_gain=gain, eps=1e-6, rot_dim=32)
    ops.synchronise()
    assert torch.isnan(qo[0, 5, [0, 16]]).all() and (qo[0, 5, 32:] == 0).all()


def test_outputs_reproduce_and_capture(ops):
    stream = torch.cuda.Stream()
    rng = np.random.default_rng(2)
    q, k = _bf16(rng.normal(0, 1, (33, 8, 128))), _bf16(rng.normal(0, 1, (33, 2, 128)))
    gain = _bf16(np.ones(128))
    pos = torch.arange(33, dtype=torch.int32, device="cuda")
    outs = [torch.zeros_like(q), torch.zeros_like(k)]
    eager = [torch.zeros_like(q), torch.zeros_like(k)]
    with dcl.Context(None, 1, 1, stream=stream.cuda_stream) as ctx:
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            ctx.qk_norm_rope(q, k, pos, *outs, theta=1e4, q_gain=gain, k_gain=gain)
        for shift in (0, 100000):
            pos.add_(shift)
            ops.qk_norm_rope(q, k, pos, *eager, theta=1e4, q_gain=gain, k_gain=gain)
            ops.synchronise()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, eager))


@pytest.mark.parametrize("eps", [1e-30, 1e30])
def test_the_smallest_and_the_largest_eps(ops, eps):
    """Values so small and so large that eps is all of the root, or none of it."""
    _run(ops, 5, 4, 2, 64, 64, eps=eps, size=2.0 ** -60)
    _run(ops, 5, 4, 2, 64, 64, eps=eps, size=2.0 ** 60)
