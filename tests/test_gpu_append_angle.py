"""The append's angles, at any position and frequency: rows (1, 0) come out as (cos, sin), compared with the angle of the exact product
pos * inv_freq, in whole numbers of 400 bits.

Bounds.  The phase is off by 2^31 times 0.51 steps of 2^-64 turns: less than 2^-33 turns, 2 pi 2^-33 rad.  An eighth of a turn at most, it is rounded to float32 half turns: 2^-27 of them, pi 2^-27 rad.
sincospif is good to 2 units in the last place.  Products with 1 and 0 add nothing.
"""
import math

import numpy as np
import pytest
import torch

from paper_2608_04771_gb300 import reco

pytestmark = pytest.mark.gpu
DEV = "cuda"
BITS = 400


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2608_04771_gb300 import build
    build.build()
    reco.lib()


def _turns_per_radian():
    """2^BITS / (2 pi), from 4 (4 atan(1/5) - atan(1/239))."""
    one = 1 << (BITS + 64)

    def atan(x):
        t = s = one // x
        k = 1
        while t:
            t //= x * x
            k += 2
            s += -(t // k) if k % 4 == 3 else t // k
        return s
    pi = 4 * (4 * atan(5) - atan(239))
    return (1 << BITS) * one // (2 * pi)


def _exact(pos, freq):
    """cos and sin of pos * freq [T, F], reduced to a turn in whole numbers."""
    c = _turns_per_radian()
    out = np.empty((2, len(pos), len(freq)))
    for j, f in enumerate(freq):
        m, e = math.frexp(float(f))  # f = m 2^e
        step = int(m * 2 ** 53) * c  # times 2^(e - 53 - BITS) turns
        for i, p in enumerate(pos):
            shift = BITS + 53 - e  # bits behind the point
            part = (int(p) * step) & ((1 << shift) - 1)
            turn = (part >> (shift - 80)) / 2.0 ** 80
            a = 2 * math.pi * (turn - 1 if turn > 0.5 else turn)
            out[0, i, j], out[1, i, j] = math.cos(a), math.sin(a)
    return out


def test_the_reference_on_small_angles():
    pos, freq = np.array([0, 1, -3, 100]), np.array([1.0, 0.37, -0.001], np.float32)
    a = pos[:, None] * freq.astype(np.float64)
    want = _exact(pos, freq)
    assert np.abs(want - np.stack([np.cos(a), np.sin(a)])).max() < 1e-13


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("most", [1000, 2 ** 20, 2 ** 26, 2 ** 31])
def test_angles_at_any_position(most, interleaved):
    rng = np.random.default_rng(most + interleaved)
    F, T = 64, 300
    freq = (1e6 ** (-np.arange(F) / F)).astype(np.float32)
    freq[1::8] *= -1
    freq[2::8] = rng.uniform(1, 2 ** 20, 8)
    freq[[4, 12, 20, 28]] = 2.0 ** -140, 0.0, 3.4e38, -7e25
    pos = np.clip(rng.integers(-most, most, T), -2 ** 31, 2 ** 31 - 1)
    pos[:4] = max(-most, -2 ** 31), min(most, 2 ** 31 - 1), 0, -1
    row = np.zeros((T, 2, F), np.float32)
    row[:, 0] = 1
    x = torch.from_numpy(row.transpose(0, 2, 1).reshape(T, 2 * F).copy() if interleaved else row.reshape(T, 2 * F)).to(DEV)
    x = x.view(1, T, 1, 2 * F)
    K, V = (torch.zeros((1, 19, 1, 16, 2 * F), device=DEV) for _ in range(2))
    kv = reco.make_paged_kv(K, V, torch.arange(19, dtype=torch.int32, device=DEV).view(1, 19), 1)
    lens = torch.zeros((1, 1, 1), dtype=torch.int32, device=DEV)
    q_out = torch.zeros_like(x)
    reco.reco_paged_append(kv, x, x, torch.tensor([0, T], dtype=torch.int32, device=DEV), lens,
                           reco.paged_workspace(reco.RECO_OP_PAGED_APPEND, kv, DEV), pos=torch.from_numpy(pos.astype(np.int32)).to(DEV),
                           inv_freq=torch.from_numpy(freq).to(DEV), q=x, q_out=q_out, interleaved=interleaved)
    reco.reco_check()
    got = K.view(-1, 2 * F)[:T]
    assert torch.equal(got, q_out.view(T, 2 * F))
    got = got.cpu().numpy()
    got = np.stack([got[:, 0::2], got[:, 1::2]] if interleaved else [got[:, :F], got[:, F:]])
    want = _exact(pos, freq)
    tol = 2 * math.pi * 2.0 ** -33 + math.pi * 2.0 ** -27 + 2 * np.spacing(np.abs(want).astype(np.float32)).astype(np.float64)
    off = np.abs(got - want)
    assert (off <= tol).all(), (off / tol).max()
