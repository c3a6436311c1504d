"""The angles of dcl_qk_norm_rope, by the sines of positions that come close to whole turns, where bf16 keeps small
differences.

Tolerance.  An angle is off by 2^-21 up to position 2^28 and by 2^-20 at any: the frequency, from double arithmetic, by
2^-55 of a turn a position, and the fraction of a turn, at most half of one, by its roundings to 24 bits, 2^-21.27 rad in all.  A
sine by 2^-21 (the approximation's 2^-21.4 between -pi and pi), and bf16's half step, 2^-8 of itself."""
from decimal import Decimal, getcontext

import numpy as np
import pytest
import torch

import paper_2607_20467_gb300 as dcl

pytestmark = pytest.mark.gpu
PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459")


@pytest.fixture(scope="module")
def ops():
    import __graft_entry__
    __graft_entry__.build()
    ctx = dcl.Context(None, 1, 1)
    yield ctx
    ctx.close()


@pytest.mark.parametrize("last,off", [(2 ** 28, 2.0 ** -21), (2 ** 31 - 1, 2.0 ** -20)])
@pytest.mark.parametrize("theta,rot", [(1.5, 128), (1e4, 128), (1e6, 128), (5e5, 64), (2.0, 80), (1e9, 112)])
def test_angles_close_to_whole_turns(ops, theta, rot, last, off):
    getcontext().prec = 60
    h, hd = rot // 2, 128
    rng = np.random.default_rng(rot + int(theta))
    rows, pos, want = [], [], []
    for i in range(0, h, max(1, h // 13)):
        turn = ((-Decimal(2 * i) / rot) * Decimal(theta).ln()).exp() / (2 * PI)  # of a position
        scaled = int(turn * 2 ** 128)
        at = [last - int(x) for x in rng.choice(1 << 20, 4000, replace=False)]
        part = [(p * scaled + (1 << 127)) % (1 << 128) - (1 << 127) for p in at]  # of a turn, from -1/2 to 1/2
        for j in np.argsort(np.abs(np.array([x / 2 ** 128 for x in part])))[:12]:
            if abs(part[j] / 2 ** 128) > 2.0 ** -9:  # (components that turn too slowly to come close)
                continue
            rows.append(i)
            pos.append(at[j])
            want.append(np.sin(part[j] / 2 ** 128 * 2 * np.pi))  # (what is close to nothing keeps its bits)
    n, want = len(rows), np.array(want)
    assert n >= 12
    x = torch.zeros(n, 1, hd, dtype=torch.bfloat16, device="cuda")
    x[torch.arange(n), 0, torch.tensor(rows)] = 1.0
    q, k = torch.empty_like(x), torch.empty_like(x)
    ops.qk_norm_rope(x, x, torch.tensor(pos, dtype=torch.int32, device="cuda"), q, k, theta=theta, rot_dim=rot)
    ops.synchronise()
    for out in (q, k):
        got = out[torch.arange(n), 0, torch.tensor(rows) + h].double().cpu().numpy()
        err = np.abs(got - want) - 2.0 ** -8 * np.abs(want)
        assert (err <= off + 2.0 ** -21).all(), err.max() / 2.0 ** -21
