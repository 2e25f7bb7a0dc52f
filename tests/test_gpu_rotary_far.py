"""sr_rotary up to its largest angles, 2^45.  The places and frequencies here multiply without a rounding, so the angle itself is
exact and the tolerance that of near positions: one rounding to the storage type, and in fp32 the sine and cosine (2^-23 each,
polynomial and rounding together) and three roundings of products of both channels, (|x0| + |x1|) 2^-21."""
import math

import numpy as np
import pytest

from paper_2607_02829_amd import abi

pytestmark = pytest.mark.gpu

FAR = 2.0 ** 45
FREQS = [1.0, 0.5, -0.25, 0.75, 2.0 ** -20, 2.0 ** -44, 0.0, -1.0]   # at most two bits each


@pytest.mark.parametrize("origin,step", [(FAR - 511.0, 1.0), (-FAR, 1.0), (FAR, -2.0), (-FAR + 1022.0, -2.0), (2.0 ** 44 + 1.0, 2.0 ** 34),
                                         (-3.0 * 2 ** 40, 2.0 ** 36 - 2.0 ** 10), (1.0e12, 1.0)])
@pytest.mark.parametrize("halves", [True, False])
@pytest.mark.parametrize("inverse", [0, 1])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_far_angles(origin, step, halves, inverse, dtype):
    import torch
    S, P = 512, len(FREQS)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.randn((S, 2 * P), generator=torch.Generator().manual_seed(7)).to(dt)
    y = torch.empty((S, 2 * P), dtype=dt, device="cuda")
    rot = abi.SrRotary([S], [P], abi.SR_ROT_HALVES if halves else abi.SR_ROT_NEIGHBOURS, origin=[origin], step=[step], freqs=FREQS)
    abi.sr_rotary(rot, inverse, abi.SR_BF16 if dtype == "bf16" else abi.SR_F32, 1, S, 1, 2 * P, x.cuda(), 2 * P, None, 0, y, 2 * P)
    t = np.array([[(origin + step * s) * f for f in FREQS] for s in range(S)])
    assert np.abs(t).max() <= FAR
    c = np.vectorize(math.cos)(t)
    s = np.vectorize(math.sin)(-t if inverse else t)
    lo, hi = (slice(0, P), slice(P, 2 * P)) if halves else (slice(0, None, 2), slice(1, None, 2))
    v, got = x.double().numpy(), y.cpu().double().numpy()
    want = np.empty_like(v)
    want[:, lo], want[:, hi] = v[:, lo] * c - v[:, hi] * s, v[:, hi] * c + v[:, lo] * s
    both = np.empty_like(v)
    both[:, lo] = both[:, hi] = np.abs(v[:, lo]) + np.abs(v[:, hi])
    err, tol = np.abs(got - want), torch.finfo(dt).eps / 2 * np.abs(want) + 2.0 ** -21 * both
    assert (err <= tol).all(), float((err / tol).max())


def test_the_longest_grid_is_within_it():
    # 2^31 - 1 places of a turn of one radian each: as far as an index reaches
    import torch
    n = (1 << 31) - 1
    idx = torch.tensor([[n - 1, 0, 1 << 30, 12345]], dtype=torch.int32)
    x, y = torch.randn((4, 32), generator=torch.Generator().manual_seed(1)), torch.empty((4, 32), device="cuda")
    abi.sr_rotary(abi.SrRotary([n], [16], freqs=[1.0] * 16), 0, abi.SR_F32, 1, 4, 1, 32, x.cuda(), 32, idx.cuda(), 0, y, 32)
    for r, l in enumerate(idx[0].tolist()):
        c, s = math.cos(l), math.sin(l)
        a, b, g = x[r, :16].double(), x[r, 16:].double(), y[r].cpu().double()
        tol = 2.0 ** -21 * (a.abs() + b.abs())
        assert bool(((g[:16] - (a * c - b * s)).abs() <= tol).all() and ((g[16:] - (b * c + a * s)).abs() <= tol).all())
