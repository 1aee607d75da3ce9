"""NaN and infinite logits in decode attention, over contiguous and paged caches: a head that meets one gives NaN in
out and lse (never the zeros of a unit without rows), the weights of the rows it sees are NaN, and every other head
and unit keeps its bits.  On every path: units whole to a warp, cut between warps and CTAs, joined, laid end to end."""
import math

import numpy as np
import pytest
import torch

from paper_2608_04771_gb300 import reco
from test_gpu_paged import BF, DEV, F32, Cache, decode

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2608_04771_gb300 import build
    build.build()
    reco.lib()


# (layers, B, H_q, H_kv, d, dtype, length)
PAGED = [
    (1, 1, 7, 1, 128, BF, 20),       # one CTA, most streams without a block
    (1, 2, 14, 2, 128, BF, 3000),    # a piece per CTA, joined by the last
    (1, 2, 32, 2, 64, BF, 700),
    (1, 2, 12, 2, 128, F32, 900),
    (1, 1, 16, 1, 64, F32, 500),
    (10, 16, 8, 2, 128, BF, 450),    # laid end to end
    (10, 16, 24, 2, 64, BF, 400),
    (9, 18, 6, 1, 64, F32, 350),
    (10, 16, 8, 2, 64, BF, 150),     # whole to a stream
    (10, 16, 20, 2, 128, F32, 90),
]
PLACES = ["query", "key", "inf key", "minus inf key", "value", "new key", "all keys"]


def _poison(what, q, K, V, kn, at, h, n, G):
    """Poisons unit (0, 0, h) and returns the heads (of the unit) whose softmax it reaches, and whether lse is NaN.
    `at(pool, j)` is row j of the unit, a view."""
    heads = list(range(G))
    if what == "query":
        heads = [G - 1]
        q[0, 0, h * G + G - 1, 5] = NAN
    elif what == "key":
        at(K, n // 2)[3] = NAN
    elif what == "all keys":
        for j in range(n):
            at(K, j)[0] = NAN
    elif what == "new key":
        kn[0, 0, h, 7] = NAN
    elif what == "value":
        at(V, n // 3)[2] = NAN
        return heads, False
    else:  # an infinite logit for the heads whose query is of the sign
        sign = 1.0 if what == "inf key" else -1.0
        at(K, n - 2)[1] = sign * INF
        return [g for g in heads if float(q[0, 0, h * G + g, 1]) > 0], sign > 0
    return heads, True


@pytest.mark.parametrize("what", PLACES)
@pytest.mark.parametrize("i", range(len(PAGED)))
def test_paged(i, what):
    Ly, B, Hq, H, d, dtype, n = PAGED[i]
    G, h = Hq // H, H - 1
    lens = np.full((Ly, B, H), n)
    lens[:, 1:] -= 7
    clean, c = (Cache(700 + i, Ly, B, Hq, H, d, dtype, 16, lens) for _ in range(2))
    q, kn, vn = clean.token()
    table = c.table.cpu().numpy()
    row = lambda pool, j: pool[0, table[0, j // 16], h, j % 16]  # noqa: E731
    q2, kn2 = q.clone(), kn.clone()
    c.weights.copy_(clean.weights)
    start = clean.weights.clone()
    heads, is_nan = _poison(what, q2, c.K, c.V, kn2, row, h, n, G)
    hit = [h * G + g for g in heads]
    if what == "all keys":
        kn2[0, 0, h, 0] = NAN
    want, want_lse = decode(clean, q, kn, vn)
    out, lse = decode(c, q2, kn2, vn)
    reco.reco_check()
    other = torch.ones(want.shape[:3], dtype=torch.bool, device=DEV)
    other[0, 0, h * G:(h + 1) * G] = False
    keep = [g for g in range(h * G, (h + 1) * G) if g not in hit]
    assert torch.equal(out[other], want[other]) and torch.equal(lse[other], want_lse[other])
    seen = torch.arange(c.cap, device=DEV) <= n
    W, W0 = c.weights[0, 0, h], clean.weights[0, 0, h]
    if what == "minus inf key":  # that row has no weight for the heads it meets, and the others +inf
        neg = [g for g in range(h * G, (h + 1) * G) if g not in hit]
        assert torch.isfinite(out[0, 0, hit]).all() and torch.isfinite(lse[0, 0, hit]).all()
        assert torch.isnan(out[0, 0, neg]).all() and torch.isnan(lse[0, 0, neg]).all()
        is_nan, keep = bool(neg), []
    elif what == "value":  # the column of that value alone
        assert torch.isnan(out[0, 0, hit, 2]).all()
        cols = [x for x in range(d) if x != 2]
        assert torch.equal(out[0, 0, hit][:, cols], want[0, 0, hit][:, cols])
        assert torch.equal(lse, want_lse) and torch.equal(c.weights, clean.weights)
        return
    else:
        assert torch.isnan(out[0, 0, hit]).all() and torch.isnan(lse[0, 0, hit]).all()
        if what == "inf key":  # (and -inf for the heads whose query has the other sign)
            assert torch.isfinite(out[0, 0, keep]).all() and torch.isfinite(lse[0, 0, keep]).all()
            keep = []
        is_nan = is_nan and bool(hit)
    assert torch.equal(out[0, 0, keep], want[0, 0, keep]) and torch.equal(lse[0, 0, keep], want_lse[0, 0, keep])
    if is_nan:
        assert torch.isnan(W[seen]).all() and torch.equal(W[~seen], start[0, 0, h][~seen])
    whole = torch.ones(c.weights.shape[:3], dtype=torch.bool, device=DEV)
    whole[0, 0, h] = False
    assert torch.equal(c.weights[whole], clean.weights[whole])
    assert torch.equal(c.lens, clean.lens) and W0.isfinite().all()


@pytest.mark.parametrize("i", [1, 3, 5, 8])
def test_paged_out_of_sight(i):
    """The same in rows behind the window changes nothing."""
    Ly, B, Hq, H, d, dtype, n = PAGED[i]
    clean, c = (Cache(800 + i, Ly, B, Hq, H, d, dtype, 16, n) for _ in range(2))
    table = c.table.cpu().numpy()
    for j in (3, 40, n - 60):
        c.K[:, table[0, j // 16], :, j % 16] = NAN if j != 40 else INF
        c.V[:, table[0, j // 16], :, j % 16] = NAN
    q, kn, vn = clean.token()
    c.weights.copy_(clean.weights)
    a, b = (decode(x, q, kn, vn, window=50, sinks=3) for x in (clean, c))
    reco.reco_check()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.equal(clean.weights, c.weights)
    assert torch.isfinite(b[0]).all()


# (layers, B, H_q, H_kv, d, dtype, length)
FLAT = [
    (1, 1, 7, 1, 128, BF, 20), (1, 2, 14, 2, 128, BF, 4000), (1, 2, 32, 2, 64, BF, 3000), (1, 2, 12, 2, 128, F32, 3000),
    (1, 1, 16, 1, 64, F32, 2000), (1, 2, 2, 2, 64, F32, 600), (10, 16, 8, 2, 128, BF, 450), (10, 40, 24, 2, 64, BF, 400),
    (20, 40, 8, 2, 64, BF, 150), (20, 40, 6, 2, 64, F32, 90),
]


@pytest.mark.parametrize("what", ["query", "key", "inf key", "value", "new key", "all keys"])
@pytest.mark.parametrize("i", range(len(FLAT)))
def test_contiguous(i, what):
    Ly, B, Hq, H, d, dtype, n = FLAT[i]
    G, h = Hq // H, H - 1
    g = torch.Generator(device=DEV)
    g.manual_seed(900 + i)
    rand = lambda *s: torch.randn(s, generator=g, device=DEV).to(dtype)  # noqa: E731
    K, V, q = rand(Ly, B, H, n + 1, d), rand(Ly, B, H, n + 1, d), rand(Ly, B, Hq, d)
    kn, vn = rand(Ly, B, H, d), rand(Ly, B, H, d)

    def run(K, V, q, kn):
        kv = reco.make_kv(K, V, Hq)
        out, lse = torch.full(q.shape, 7.0, device=DEV), torch.full(q.shape[:3], 7.0, device=DEV)
        lens = torch.full((Ly, B, H), n, dtype=torch.int32, device=DEV)
        reco.reco_decode_attn(kv, q, kn, vn, lens, 1.0 / math.sqrt(d), out, lse,
                              reco.workspace(reco.RECO_OP_DECODE, kv, 0, DEV))
        reco.reco_check()
        assert (lens == n + 1).all()
        return out, lse

    K2, V2, q2, kn2 = K.clone(), V.clone(), q.clone(), kn.clone()
    want, want_lse = run(K.clone(), V, q, kn)
    heads, is_nan = _poison(what, q2, K2, V2, kn2, lambda pool, j: pool[0, 0, h, j], h, n, G)
    if what == "all keys":
        kn2[0, 0, h, 0] = NAN
    out, lse = run(K2, V2, q2, kn2)
    hit = [h * G + x for x in heads]
    other = torch.ones(want.shape[:3], dtype=torch.bool, device=DEV)
    other[0, 0, h * G:(h + 1) * G] = False
    assert torch.equal(out[other], want[other]) and torch.equal(lse[other], want_lse[other])
    if what == "value":
        cols = [x for x in range(d) if x != 2]
        assert torch.isnan(out[0, 0, hit, 2]).all() and torch.equal(lse, want_lse)
        assert torch.equal(out[0, 0, hit][:, cols], want[0, 0, hit][:, cols])
        return
    assert torch.isnan(out[0, 0, hit]).all() and torch.isnan(lse[0, 0, hit]).all()
    keep = [x for x in range(h * G, (h + 1) * G) if x not in hit]
    if what == "inf key":
        assert torch.isfinite(out[0, 0, keep]).all() and torch.isfinite(lse[0, 0, keep]).all()
    else:
        assert torch.equal(out[0, 0, keep], want[0, 0, keep]) and torch.equal(lse[0, 0, keep], want_lse[0, 0, keep])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [30, 2500])
def test_logits_that_are_all_minus_infinity(dtype, n):
    """Zeros and lse = -inf, nothing added to the sums; as documented."""
    c = Cache(950, 1, 1, 2, 1, 64, dtype, 16, n)
    q, kn, vn = c.token()
    q[0, 0, 0] = q[0, 0, 0].abs() + 0.5
    q[0, 0, 1] = -q[0, 0, 1].abs() - 0.5
    t = c.table.cpu().numpy()
    for j in range(n):
        c.K[0, t[0, j // 16], 0, j % 16, 0] = -INF
    kn[0, 0, 0, 0] = -INF
    start = c.weights.clone()
    out, lse = decode(c, q, kn, vn)
    reco.reco_check()
    assert (out[0, 0, 0] == 0).all() and float(lse[0, 0, 0]) == -INF
    assert torch.isnan(out[0, 0, 1]).all() and torch.isnan(lse[0, 0, 1])  # +inf for the other head
    assert torch.isnan(c.weights[0, 0, 0, :n + 1]).all() and torch.equal(c.weights[..., n + 1:], start[..., n + 1:])
    c = Cache(951, 1, 1, 1, 1, 64, dtype, 16, n)
    q, kn, vn = c.token()
    q, t = q.abs() + 0.5, c.table.cpu().numpy()
    for j in range(n):
        c.K[0, t[0, j // 16], 0, j % 16, 0] = -INF
    kn[0, 0, 0, 0] = -INF
    start = c.weights.clone()
    out, lse = decode(c, q, kn, vn)
    reco.reco_check()
    assert (out == 0).all() and float(lse[0, 0, 0]) == -INF
    start[0, 0, 0, n] = 0.0  # the new row starts at its own weight, which is none
    assert torch.equal(c.weights, start)
