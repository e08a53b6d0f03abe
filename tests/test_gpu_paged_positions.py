"""Rotation at far positions: pos * inv_freq needs 55 bits, so an angle that is formed as one 64-bit product is off by up to 2^-22
there.  Shown where it can be seen behind a rounding to bf16: at positions whose angle lies next to a multiple of pi, where the
sine is no larger than a few of those errors."""
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2502_01068_b200 import binding as B
from tests.paged_reference import Pools
from tests.test_gpu_paged import bf16_rows, workspace

pytestmark = pytest.mark.gpu


def exact_sin_cos(pos, f):
    """Of the product of the two, whose second half (at most 2^-22) counts to first order."""
    a = Fraction(int(pos)) * Fraction(float(f))
    hi = float(a)
    lo = float(a - Fraction(hi))
    s, c = np.sin(hi), np.cos(hi)
    return s + c * lo, c - s * lo


def near_multiples_of_pi(f, n):
    pos = np.arange(2 ** 31 - 2 ** 20, 2 ** 31 - 1, dtype=np.int64)
    near = np.argsort(np.abs(np.sin(pos.astype(np.float64) * np.float64(f))))[:n]
    return pos[near]


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("fmt,new", [("bf16", 1), ("e4m3", 8), ("e4m3", 64)])
def test_angles_of_far_positions(fmt, new, adjacent):
    d, n = 64, 64
    f = np.exp(np.random.default_rng(9).uniform(-1, 0, d // 2)).astype(np.float32)
    pos = np.concatenate([near_multiples_of_pi(f[i], 8) for i in range(0, 32, 4)])
    pair = np.repeat(np.arange(0, 32, 4), 8)
    lo, hi = (2 * np.arange(32), 2 * np.arange(32) + 1) if adjacent else (np.arange(32), np.arange(32) + 32)
    q = torch.zeros((n, 1, d), dtype=torch.bfloat16)
    q[:, :, hi] = 1.0                                           # turns to (-sin, cos)
    pools = Pools(fmt, [0] * (n // new), [new] * (n // new), 16, 1, d, 3)
    rows = B.make_new_rows(batch=n // new, total=n, n_q_heads=1, n_kv_heads=1, head_dim=d, rot_dim=d,
                           rot_pairs=B.ROT_ADJACENT if adjacent else B.ROT_HALVES)
    q_out, ws = torch.zeros_like(q).cuda(), workspace()
    v = bf16_rows(np.random.default_rng(1), (n, 1, d)).cuda()
    B.fastkv_paged_append(pools.cache(), rows, pools.dev_lens, q.cuda(), q.cuda(), v, torch.from_numpy(pos.astype(np.int32)).cuda(),
                          torch.from_numpy(f).cuda(), None, q_out, None, ws)
    assert B.fastkv_device_status(ws) == (0, 0)
    got = q_out.cpu().double().numpy()[:, 0]
    small = 0
    for r in range(n):
        for i in range(32):
            s, c = exact_sin_cos(pos[r], f[i])
            # a rounding to fp32, one to bf16, and what the angle in 64 bits leaves (some 1e-15)
            assert abs(got[r, lo[i]] + s) <= (2.0 ** -8 + 2.0 ** -23) * abs(s) + 1e-14, (r, i)
            assert abs(got[r, hi[i]] - c) <= (2.0 ** -8 + 2.0 ** -23) * abs(c) + 1e-14, (r, i)
            small += i == pair[r] and abs(s) < 1e-5
    assert small >= 32
    if fmt == "bf16":                                           # the keys turn by the same angles
        k = np.stack([pools.read(b, 1)[0][0, 0] for b in range(n)])
        assert np.array_equal(k, got)
