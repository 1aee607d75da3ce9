"""Units beside one in error, against the float64 reference: their outputs, log-sum-exps, lengths and running weights
are those of a call without the error, with few units (a piece per CTA, weights where pieces join or by a launch of
their own), many (laid end to end) and short ones (whole to a stream), in a window and without."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2608_04771_gb300 import reco
from test_gpu_paged import BF, DEV, F32, Cache, _refused, bounds, decode, np64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2608_04771_gb300 import build
    build.build()
    reco.lib()


# (layers, B, H_q, H_kv, d, dtype, shortest and longest unit, window, sinks)
CASES = [
    (2, 2, 10, 2, 128, BF, 30, 700, 0, 0),
    (2, 2, 10, 2, 128, F32, 30, 700, 0, 0),
    (1, 2, 14, 2, 128, BF, 3000, 4500, 0, 0),
    (1, 3, 12, 1, 64, BF, 100, 3500, 600, 20),
    (10, 16, 7, 1, 128, BF, 300, 700, 0, 0),
    (10, 16, 6, 1, 64, F32, 300, 500, 100, 3),
    (10, 20, 4, 1, 64, BF, 60, 200, 0, 0),
    (10, 20, 12, 1, 128, F32, 60, 120, 0, 0),
]


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("what", ["length", "room", "page", "last page"])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_units_beside_an_error(i, what, weights):
    Ly, B, Hq, H, d, dtype, lo, hi, window, sinks = CASES[i]
    G = Hq // H
    lens = np.random.default_rng(400 + i).integers(lo, hi + 1, (Ly, B, H))
    lens[-1, -1] = hi  # the unit that a length or its room puts in error has blocks of its own otherwise
    c = Cache(400 + i, Ly, B, Hq, H, d, dtype, 16, lens)
    q, kn, vn = c.token()
    ref = c.host()
    bad = np.zeros((Ly, B, H), bool)
    if what in ("length", "room"):
        bad[-1, -1, -1] = True
        c.lens[-1, -1, -1] = -2 if what == "length" else c.cap
    else:  # a page of the newest rows of sequence 0's shortest or longest unit
        n = int(lens[:, 0].min() if what == "page" else lens[:, 0].max())
        c.table[0, n // 16] = -1
        at = n // 16 * 16
        bad[:, 0] = (lens[:, 0] >= at) if window == 0 else \
            (lens[:, 0] >= at) & ((lens[:, 0] + 1 - window) // 16 * 16 <= at)
    ro, rl, big, seen, absv = paged.decode(*ref[:4], *(np64(t) for t in (q, kn, vn)), c.scale, window, sinks, ref[4])
    before = c.weights.clone()
    lens0 = c.lens.cpu().numpy().copy()
    out, lse = decode(c, q, kn, vn, window, sinks, weights)
    assert {"length": "length", "room": "room"}.get(what, "page") in _refused()
    ok, okq = ~bad, ~np.repeat(bad, G, 2)
    t_prob, t_out, t_lse = bounds(c, big, seen, absv, ro, rl, torch.float32)
    go, gl = np64(out), np64(lse)
    assert (go[~okq] == 0).all() and np.isneginf(gl[~okq]).all()
    assert (np.abs(go - ro) <= t_out)[okq].all() and (np.abs(gl - rl) <= t_lse)[okq].all()
    assert np.array_equal(c.lens.cpu().numpy(), np.where(ok, lens + 1, lens0))
    W0, W, got = np64(before), ref[4], np64(c.weights)
    j = np.arange(c.cap)
    if not weights:
        assert torch.equal(c.weights, before)
        return
    of_bad = bad[..., None] & (j < np.minimum(lens, c.cap)[..., None])  # rows of the units in error
    assert np.array_equal(got[of_bad], W0[of_bad])
    tol = t_prob.reshape(Ly, B, H, G).max(3)[..., None]
    new = j == lens[..., None]
    added = np.where(new, W, W - W0)
    beside = np.broadcast_to(ok[..., None], W.shape)
    assert (np.abs(got - W) <= tol * added + 2 * 2.0 ** -24 * W)[beside].all()
    still = beside & (added == 0) & ~new
    assert np.array_equal(got[still], W0[still])
