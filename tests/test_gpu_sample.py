"""dcl_sample against its definition in 64 bits.

Which tokens are kept follows from the logits' order and counts (exact) and, for top-p, from sums: a
row whose prefix changes when top_p is moved by 1e-6 of itself is not decided by fp32 sums and is
left out (the cases are drawn so that this is rare, which the tests check).  A token is compared
where the best y + noise leads the next by 1e-5 (1 + |y|) (fp32 rounding of the two terms).
Probabilities are ratios of exponentials of fp32 arguments: 2^-24 |y| of an argument and a few ulp of
the exponential, within 1e-5 (1 + |y|) of themselves."""
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


def _prefix(w, top_p):
    """Tokens of the shortest prefix whose mass reaches top_p (w: weights in order)."""
    if top_p >= 1:
        return len(w)
    before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
    return max(1, int((before < top_p * w.sum()).sum()))


def _row(z, noise, T, k, p, mp):
    """(kept mask or None if top-p is not decided, y) of one row in 64 bits."""
    z = np.where(np.isnan(z), -np.inf, z)
    V = len(z)
    if not (T > 0):
        kept = np.zeros(V, bool)
        kept[np.argmax(z)] = True
        return kept, z - z.max()
    with np.errstate(invalid="ignore"):
        y = (z - z.max()) / T
    order = np.lexsort((np.arange(V), -z))
    n = k if 0 < k < V else V
    w = np.exp(y[order[:n]])
    counts = {_prefix(w, p * (1 + d)) if p < 1 else len(w) for d in (-1e-6, 0.0, 1e-6)}
    if len(counts) > 1:
        return None, y
    keep = order[:counts.pop()]
    kept = np.zeros(V, bool)
    kept[keep] = True
    if mp > 0:
        edge = np.log(min(mp, 1.0))
        if (np.abs(y[kept] - edge) < 1e-6 * (1 + abs(edge))).any() and mp < 1:
            return None, y
        kept &= y >= edge
    return kept & np.isfinite(y), y


def _check(ops, z, noise=None, T=None, k=None, p=None, mp=None, z_stride=None, most_undecided=0.05):
    """z [R][V] float (bf16 values), the rest arrays of R or None."""
    R, V = z.shape
    wide = torch.zeros(R, z_stride or V, dtype=torch.bfloat16, device="cuda")
    logits = wide[:, (z_stride or V) - V:]
    logits.copy_(torch.from_numpy(z.astype(np.float32)))
    dev = lambda a, t: None if a is None else torch.from_numpy(np.asarray(a)).to(t).cuda()
    token = torch.full((R,), -7, dtype=torch.int32, device="cuda")
    prob, conf = torch.full((R,), -7.0, device="cuda"), torch.full((R,), -7.0, device="cuda")
    nz = None
    if noise is not None:
        nw = torch.zeros(R, (z_stride or V) + 1, device="cuda")
        nz = nw[:, (z_stride or V) + 1 - V:]
        nz.copy_(torch.from_numpy(noise))
    kw = dict(noise=nz, temperature=dev(T, torch.float32), top_k=dev(k, torch.int32), top_p=dev(p, torch.float32),
              min_p=dev(mp, torch.float32))
    ops.sample(logits, token, prob=prob, conf=conf, **kw)
    ops.synchronise()
    got, gp, gc = token.cpu().numpy(), prob.cpu().numpy().astype(np.float64), conf.cpu().numpy().astype(np.float64)
    undecided = 0
    pick = lambda a, r, d: d if a is None else np.asarray(a)[r].item()
    for r in range(R):
        zr = z[r].astype(np.float64)
        if not (zr > -np.inf).any():  # all -inf or NaN
            assert got[r] == -1 and gp[r] == 0 and gc[r] == 0
            continue
        t32 = float(np.float32(pick(T, r, 1.0)))
        kept, y = _row(zr, None, t32, pick(k, r, 0), float(np.float32(pick(p, r, 1.0))),
                       float(np.float32(pick(mp, r, 0.0))))
        if kept is None:
            undecided += 1
            continue
        g = np.zeros(V) if noise is None or not t32 > 0 else noise[r].astype(np.float64)
        key = np.where(kept, y + g, -np.inf)
        tok = int(np.argmax(key))
        i = got[r]
        assert 0 <= i < V and kept[i], (r, i, tok)
        if i != tok:
            assert key[tok] - key[i] <= 1e-5 * (1 + abs(y[tok]) + abs(y[i])), (r, i, tok)
        want = np.exp(y[i]) / np.exp(y[kept]).sum() if t32 > 0 else 1.0
        assert abs(gp[r] - want) <= 1e-5 * (1 + abs(y[i])) * want, (r, gp[r], want)
        full = np.where(np.isnan(zr), -np.inf, zr)
        full = full - full.max()
        cw = np.exp(full[i]) / np.exp(full).sum()
        assert abs(gc[r] - cw) <= 1e-5 * (1 + abs(full[i])) * cw, (r, gc[r], cw)
    assert undecided <= most_undecided * R + 1, undecided
    again = torch.full_like(token, -7)
    p2, c2 = torch.zeros_like(prob), torch.zeros_like(conf)
    ops.sample(logits, again, prob=p2, conf=c2, **kw)
    alone = torch.full_like(token, -7)
    ops.sample(logits, alone, **kw)  # without the optional outputs
    ops.synchronise()
    assert torch.equal(again, token) and torch.equal(p2, prob) and torch.equal(c2, conf) and torch.equal(alone, token)
    return got


def _bf16(a):
    return torch.from_numpy(np.asarray(a, np.float32)).to(torch.bfloat16).float().numpy()


def _logits(rng, R, V, bulk=2.0, lifted=20):
    z = rng.normal(0, bulk, (R, V))
    for r in range(R):
        z[r, rng.integers(0, V, min(lifted, V))] += rng.uniform(3, 12)
    return _bf16(z)


def _gumbel(rng, R, V):
    return (-np.log(-np.log(rng.uniform(1e-12, 1 - 1e-7, (R, V))))).astype(np.float32)


SIZES = [(1, 1), (3, 2), (5, 31), (4, 257), (7, 1000), (2, 4096), (3, 12345), (2, 126464), (1, 152064)]


@pytest.mark.parametrize("R,V", SIZES)
def test_whole_vocabulary(ops, R, V):
    rng = np.random.default_rng(V)
    _check(ops, _logits(rng, R, V), _gumbel(rng, R, V), T=rng.uniform(0.2, 3, R))
    _check(ops, _logits(rng, R, V))  # the largest logit, temperature 1


@pytest.mark.parametrize("R,V", SIZES)
def test_truncations(ops, R, V):
    rng = np.random.default_rng(V + 1)
    z, g = _logits(rng, R, V), _gumbel(rng, R, V)
    T = rng.uniform(0.3, 2, R)
    _check(ops, z, g, T=T, k=rng.integers(1, V + 1, R))
    _check(ops, z, g, T=T, p=rng.uniform(0.05, 0.99, R))
    _check(ops, z, g, T=T, mp=rng.uniform(0.001, 0.5, R))
    _check(ops, z, g, T=T, k=rng.integers(1, min(V, 60) + 1, R), p=rng.uniform(0.3, 0.99, R),
           mp=rng.uniform(0.001, 0.1, R), z_stride=V + 3)


@pytest.mark.parametrize("V", [100, 5003, 152064])
def test_flat_rows_keep_most_of_the_vocabulary(ops, V):
    """High temperatures and logits about zero (both signs): the kept prefix runs far down the order."""
    rng = np.random.default_rng(V + 2)
    R = 6
    z = _bf16(rng.normal(0, 1, (R, V)))
    z[1] = _bf16(rng.normal(0, 1e-3, V))
    z[2] = _bf16(-np.abs(rng.normal(5, 2, V)))
    z[3] = _bf16(rng.normal(0, 1, V) * np.exp2(rng.integers(-30, 5, V)))
    _check(ops, z, _gumbel(rng, R, V), T=[1, 2, 1, 5, 20, 0.5], p=[0.95, 0.5, 0.9, 0.99, 0.7, 0.999],
           most_undecided=0.5)
    _check(ops, z, _gumbel(rng, R, V), T=[1, 2, 1, 5, 20, 0.5], k=rng.integers(V // 2, V, R))


def test_ties_go_to_the_lowest_index(ops):
    """Few distinct logits, so that every boundary falls inside a run of equal ones; k and the masses
    are chosen so that sums of powers of two decide exactly."""
    V, R = 4096, 8
    z = np.zeros((R, V), np.float32)
    z[:, 2048:2056] = 1.0
    z[4] = -0.0
    z[4, ::2] = 0.0  # -0 and +0 are equal logits
    g = _gumbel(np.random.default_rng(0), R, V)
    _check(ops, z, g, k=[1, 5, 8, 9, 3, 100, 4095, 4096])
    flat = np.full((R, V), -3.0, np.float32)
    for k in (1, 2, 1000, 4095):
        got = _check(ops, flat, g, k=[k] * R)
        assert (got < k).all()
        assert (got == g[:, :k].argmax(1)).all()
    got = _check(ops, flat, g, p=[(1000 - 0.5) / V] * R)  # 1000 of equal weight
    assert (got == g[:, :1000].argmax(1)).all()
    got = _check(ops, flat)
    assert (got == 0).all()


def test_masked_vocabularies(ops):
    """-inf, the lowest bf16 value and NaN in most places; rows of nothing else."""
    rng = np.random.default_rng(11)
    V, R = 3001, 9
    z = _logits(rng, R, V)
    low = float(torch.finfo(torch.bfloat16).min)
    z[0, 1:] = -np.inf
    z[1, :-1] = -np.inf
    z[2, rng.random(V) < 0.99] = -np.inf
    z[3] = -np.inf  # nothing
    z[4] = np.nan  # nothing
    z[5] = low  # all equal: a uniform draw
    z[6, rng.random(V) < 0.99] = low
    z[7, rng.random(V) < 0.5] = np.nan
    z[8, :] = np.where(rng.random(V) < 0.5, -np.inf, np.nan)
    g = _gumbel(rng, R, V)
    T = [0.5, 1, 2, 1, 1, 0.7, 0.3, 1.5, 1]
    got = _check(ops, z, g, T=T)
    assert got[5] == g[5].argmax()
    _check(ops, z, g, T=T, k=[3] * R, mp=[0.1] * R)
    _check(ops, z, g, T=T, p=[0.9] * R)
    _check(ops, z, g, T=T, k=[V - 1] * R)


def test_ends_of_the_parameters(ops):
    rng = np.random.default_rng(12)
    R, V = 8, 999
    z, g = _logits(rng, R, V), _gumbel(rng, R, V)
    first = z.argmax(1)
    nan = float("nan")
    got = _check(ops, z, g, T=[0.0, -1.0, nan, 0.0, 1e-3, 1e-6, 1e-30, 1e-44], k=[0, 5, 5, 1, 0, 3, 0, 0],
                 p=[0.5] * R)
    assert (got[:4] == first[:4]).all() and (got[6:] == first[6:]).all()
    assert (_check(ops, z, g, k=[1] * R) == first).all()
    assert (_check(ops, z, g, p=[0.0] * R) == first).all()
    _check(ops, z, g, k=[0, -5, V, V + 1, 2 ** 31 - 1, 1, 2, 3], p=[1.0, 2.0, nan, 1.5, 0.3, 0.0, -1.0, 0.99],
           mp=[0.0, -1.0, nan, 0.5, 1e-9, 0.2, 0.01, 0.0])
    got = _check(ops, z, g, mp=[1.0] * R)
    assert (z[np.arange(R), got] == z.max(1)).all()


def test_the_draws_follow_the_distribution(ops):
    """40000 rows of the same logits: the frequency of every token within 5 standard deviations."""
    rng = np.random.default_rng(13)
    R, V = 40000, 37
    z = np.broadcast_to(_bf16(rng.normal(0, 1.5, V)), (R, V))
    T, k, p = 0.8, 20, 0.9
    logits = torch.from_numpy(z.copy()).to(torch.bfloat16).cuda()
    token = torch.zeros(R, dtype=torch.int32, device="cuda")
    full = lambda x, t: torch.full((R,), x, dtype=t, device="cuda")
    ops.sample(logits, token, noise=torch.from_numpy(_gumbel(rng, R, V)).cuda(), temperature=full(T, torch.float32),
               top_k=full(k, torch.int32), top_p=full(p, torch.float32))
    ops.synchronise()
    kept, y = _row(z[0].astype(np.float64), None, float(np.float32(T)), k, p, 0.0)
    w = np.where(kept, np.exp(y), 0)
    w /= w.sum()
    freq = np.bincount(token.cpu().numpy(), minlength=V) / R
    assert (freq[~kept] == 0).all()
    assert (np.abs(freq - w) <= 5 * np.sqrt(w * (1 - w) / R) + 1e-9).all()


def test_rows_beyond_32_bits_of_elements(ops):
    """A row whose first logit lies past element 2^31 (a wide stride, two rows)."""
    V, stride = 1000, (1 << 31) + 64
    wide = torch.empty(stride + V, dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(14)
    z = _logits(rng, 2, V)
    logits = torch.as_strided(wide, (2, V), (stride, 1))
    logits.copy_(torch.from_numpy(z))
    token = torch.zeros(2, dtype=torch.int32, device="cuda")
    ops.sample(logits, token)
    ops.synchronise()
    assert (token.cpu().numpy() == z.argmax(1)).all()


def test_refusals(ops):
    z = torch.zeros(2, (1 << 19) + 1, dtype=torch.bfloat16, device="cuda")
    token = torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises(dcl.DcleapError, match="2\\^19") as e:
        ops.sample(z, token)
    assert e.value.status == dcl.DCL_ERR_UNSUPPORTED
    ops.sample(z[:0, :100], token[:0])  # no rows: nothing to do
    ops.synchronise()
