"""The paged cache on the GPU against the fp64 reference (oracle/paged.py): decode attention over
pages with and without a window, the accumulated weights, the eviction, and a run of them together.

Bounds, from the number of roundings (u = 2^-24, half a step of float32):
  a logit       a sum of d products of up to `big` = scale * sum |q_i k_i| in all: (d + 4) u big, and
                what exp2 adds: its argument of up to about big * log2 e rounded (2 u big), its result
                within 2^-22
  a probability twice the logit's (itself and the normaliser's), and 2^-21
  an output     that times sum_j p_j |v_j|; the chain of additions into it (a block of 16 rows at a
                time, then pieces of a unit: 64 + n / 8 of them) u each; for bf16 caches the
                probabilities enter their product in two bf16 parts, 2^-17; a bf16 output half a bf16 step
  a lse         the logit's, the sum's (64 + n / 8 u) and its own rounding
  a weight      the probability's on the part that is added, u on the sum
"""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2608_04771_gb300 import reco

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2608_04771_gb300 import build
    build.build()
    reco.lib()


def np64(t):
    return t.detach().double().cpu().numpy()


class Cache:
    """A paged cache whose every row behind a unit's length is NaN and whose table entries behind the
    last needed page name no page."""

    def __init__(self, seed, Ly, B, Hq, H, d, dtype, page, lens, spare=2, room=1):
        self.shape = (Ly, B, Hq, H, d)
        self.dtype, self.page = dtype, page
        rng = np.random.default_rng(seed)
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)
        lens = np.broadcast_to(np.asarray(lens, np.int32), (Ly, B, H)).copy()
        self.max_pages = (int(lens.max()) + room + page - 1) // page + 1
        need = [-(-(int(lens[:, b].max()) + room) // page) for b in range(B)]
        n_pages = sum(need) + spare
        ids = rng.permutation(n_pages)
        table = np.where(rng.random((B, self.max_pages)) < 0.5, -1, 2 ** 31 - 1).astype(np.int32)
        at = 0
        for b in range(B):
            table[b, :need[b]] = ids[at:at + need[b]]
            at += need[b]
        self.K, self.V = self.rand(Ly, n_pages, H, page, d), self.rand(Ly, n_pages, H, page, d)
        live = torch.zeros((Ly, n_pages, H, page), dtype=torch.bool)
        for ly, b, h in np.ndindex(Ly, B, H):
            j = np.arange(lens[ly, b, h])
            live[ly, table[b, j // page], h, j % page] = True
        self.K[~live.to(DEV)] = float("nan")
        self.V[~live.to(DEV)] = float("nan")
        self.table = torch.from_numpy(table).to(DEV)
        self.lens = torch.from_numpy(lens).to(DEV)
        self.cap = self.max_pages * page
        self.weights = torch.rand((Ly, B, H, self.cap), generator=self.g, device=DEV)
        self.scale = float(d) ** -0.5
        self.kv = reco.make_paged_kv(self.K, self.V, self.table, Hq)

    def rand(self, *shape):
        return torch.randn(shape, generator=self.g, device=DEV).to(self.dtype)

    def token(self):
        Ly, B, Hq, H, d = self.shape
        return self.rand(Ly, B, Hq, d), self.rand(Ly, B, H, d), self.rand(Ly, B, H, d)

    def outputs(self, out_dtype):
        Ly, B, Hq, H, d = self.shape
        return (torch.full((Ly, B, Hq, d), 7.0, device=DEV, dtype=out_dtype),
                torch.full((Ly, B, Hq), 7.0, device=DEV))

    def host(self):
        return [np64(self.K), np64(self.V), self.table.cpu().numpy(), self.lens.cpu().numpy().copy(), np64(self.weights)]

    def workspace(self, op):
        return reco.paged_workspace(op, self.kv, DEV)


def decode(c, q, kn, vn, window=0, sinks=0, weights=True, out_dtype=torch.float32, ws=None):
    out, lse = c.outputs(out_dtype)
    if weights:
        ws = c.workspace(reco.RECO_OP_PAGED_WEIGHTS) if ws is None else ws
        reco.reco_paged_decode_attn_weights(c.kv, q, kn, vn, c.lens, c.scale, out, lse, c.weights, ws, window, sinks)
    else:
        ws = c.workspace(reco.RECO_OP_PAGED_DECODE) if ws is None else ws
        reco.reco_paged_decode_attn(c.kv, q, kn, vn, c.lens, c.scale, out, lse, ws, window, sinks)
    return out, lse


def bounds(c, big, seen, absv, out, lse, out_dtype):
    d = c.shape[4]
    prob = 2 * ((d + 6) * U * big) + 2.0 ** -21
    chain = (64 + seen / 8) * U
    t_out = (prob + chain + (2.0 ** -17 if c.dtype == torch.bfloat16 else 0.0))[..., None] * absv
    if out_dtype == torch.bfloat16:
        t_out = t_out * (1 + 2.0 ** -8) + np.abs(out) * 2.0 ** -8
    else:
        t_out = t_out + np.abs(out) * U
    t_lse = (d + 6) * U * big + 2.0 ** -21 + chain + 2 * U * np.abs(np.where(np.isfinite(lse), lse, 0.0))
    return prob + chain, t_out, t_lse


def check(c, q, kn, vn, window=0, sinks=0, weights=True, out_dtype=torch.float32, ws=None, exact_pool=True):
    """One call against the reference; returns the library's outputs."""
    K, V, table, lens, W = c.host()
    W0, before = W.copy(), [c.K.clone(), c.V.clone()] if exact_pool else None
    out, lse = decode(c, q, kn, vn, window, sinks, weights, out_dtype, ws)
    reco.reco_check()
    n64 = [None if t is None else np64(t) for t in (q, kn, vn)]
    ro, rl, big, seen, absv = paged.decode(K, V, table, lens, *n64, c.scale, window, sinks, W)
    t_prob, t_out, t_lse = bounds(c, big, seen, absv, ro, rl, out_dtype)
    go, gl = np64(out), np64(lse)
    assert (np.abs(go - ro) <= t_out).all(), (np.abs(go - ro) / (t_out + 1e-300)).max()
    none = seen == 0
    assert np.array_equal(np.isneginf(gl), none) and (go[none] == 0).all()
    off = np.abs(gl[~none] - rl[~none])
    assert (off <= t_lse[~none]).all(), (off / t_lse[~none]).max()
    assert np.array_equal(c.lens.cpu().numpy(), lens)
    if exact_pool:  # the new rows are where the table says, and nothing else has changed
        for t, b, ref in ((c.K, before[0], K), (c.V, before[1], V)):
            same = torch.from_numpy(ref).to(DEV).to(c.dtype)
            assert torch.equal(t.view(torch.int16 if c.dtype == torch.bfloat16 else torch.int32),
                               torch.where(torch.isnan(same), b, same).view(torch.int16 if c.dtype == torch.bfloat16 else torch.int32))
    got = np64(c.weights)
    if not weights:
        assert np.array_equal(got, W0)
        return out, lse
    H, G = c.shape[3], c.shape[2] // c.shape[3]
    tol = t_prob.reshape(*t_prob.shape[:2], H, G).max(3)[..., None]
    added = W - W0
    new = np.zeros_like(W, bool)
    if kn is not None:
        for i in np.ndindex(lens.shape):
            new[i + (lens[i] - 1,)] = True
            added[i + (lens[i] - 1,)] = W[i + (lens[i] - 1,)]
    assert np.array_equal(got[(added == 0) & ~new], W0[(added == 0) & ~new])
    assert (np.abs(got - W) <= tol * added + 2 * U * W).all(), (np.abs(got - W) / (tol * added + 2 * U * W + 1e-300)).max()
    return out, lse


BF, F32 = torch.bfloat16, torch.float32

# (layers, B, H_q, H_kv, d, dtype, page, lengths, window, sinks, append)
CASES = [
    # every group size, type and head dimension, lengths around blocks and pages
    (1, 2, 1, 1, 128, BF, 16, (0, 300), 0, 0, True),
    (2, 2, 4, 2, 64, BF, 16, (1, 100), 0, 0, True),
    (1, 3, 6, 2, 128, F32, 16, (1, 130), 0, 0, True),
    (1, 2, 8, 2, 64, F32, 32, (0, 70), 0, 0, True),
    (1, 2, 10, 2, 128, F32, 32, (0, 70), 0, 0, True),
    (2, 1, 6, 1, 128, F32, 64, (50, 200), 0, 0, False),
    (1, 2, 14, 2, 128, BF, 64, (1, 300), 0, 0, True),
    (1, 2, 8, 1, 64, F32, 128, (1, 300), 0, 0, True),
    (1, 2, 8, 1, 128, BF, 256, (200, 600), 0, 0, True),
    (1, 2, 18, 2, 128, BF, 16, (1, 200), 0, 0, True),
    (1, 2, 12, 1, 64, BF, 32, (1, 200), 0, 0, False),
    (1, 2, 24, 2, 128, F32, 16, (1, 90), 0, 0, True),
    (2, 2, 16, 1, 128, BF, 16, (1, 500), 0, 0, True),
    (1, 2, 16, 1, 64, F32, 16, (1, 90), 0, 0, True),
    # windows and sinks: of one row, inside a block, a block, across pages, longer than the unit
    (1, 2, 4, 2, 128, BF, 16, (1, 400), 1, 0, True),
    (1, 2, 4, 2, 64, F32, 16, (1, 400), 1, 1, True),
    (1, 3, 7, 1, 128, BF, 16, (1, 400), 15, 3, True),
    (1, 3, 5, 1, 128, F32, 16, (1, 400), 16, 16, True),
    (1, 3, 5, 1, 64, BF, 32, (1, 400), 17, 17, False),
    (1, 3, 9, 1, 128, BF, 64, (1, 400), 100, 33, True),
    (1, 3, 3, 1, 128, F32, 64, (1, 400), 100, 64, True),
    (1, 3, 2, 1, 128, BF, 16, (1, 400), 1000, 4, True),
    (1, 3, 2, 1, 128, BF, 16, (1, 400), 60, 1000, True),
    (1, 2, 8, 2, 128, BF, 256, (300, 1500), 256, 256, True),
    # cut over the length: few long units, beside short ones
    (1, 1, 7, 1, 128, BF, 16, (9000, 9000), 0, 0, True),
    (1, 2, 4, 2, 128, BF, 64, (1, 9000), 0, 0, True),
    (1, 1, 6, 1, 64, F32, 32, (7001, 7001), 0, 0, True),
    (1, 2, 16, 1, 128, BF, 32, (100, 6000), 0, 0, False),
    (1, 1, 5, 1, 128, BF, 16, (9001, 9001), 4097, 5, True),
    # more units than CTAs: ranges of blocks cut across units, joined in tiles of eight heads, heads shared by
    # the warps of a stream
    (10, 10, 6, 2, 128, BF, 16, (200, 900), 0, 0, True),
    (10, 10, 6, 2, 64, F32, 32, (200, 700), 0, 0, True),
    (9, 9, 24, 2, 128, BF, 16, (280, 600), 0, 0, True),
    (9, 9, 11, 1, 64, BF, 16, (280, 600), 300, 7, False),
    (9, 9, 14, 2, 128, F32, 16, (270, 500), 0, 0, True),
    (10, 16, 13, 1, 64, F32, 64, (270, 400), 0, 0, False),
    (10, 16, 3, 1, 128, BF, 64, (1, 3000), 200, 20, True),
    # and short units, each of which goes to the warps of one stream
    (12, 10, 6, 2, 128, BF, 16, (0, 200), 0, 0, True),
    (12, 10, 22, 2, 64, BF, 32, (0, 200), 30, 5, True),
    (12, 10, 8, 2, 128, F32, 16, (0, 200), 0, 0, True),
    (12, 10, 14, 2, 64, F32, 16, (0, 200), 50, 0, True),
    (9, 18, 10, 1, 128, F32, 16, (0, 100), 0, 0, True),
    (9, 18, 16, 1, 128, F32, 16, (0, 100), 0, 0, True),
    (9, 18, 1, 1, 64, F32, 16, (0, 100), 0, 0, True),
    # as many units as plan by warps, as fit a CTA each, and one more of each
    (4, 32, 2, 1, 64, BF, 16, (0, 300), 0, 0, True),
    (3, 43, 2, 1, 64, BF, 16, (0, 300), 0, 0, True),
    (8, 19, 2, 1, 64, BF, 16, (0, 600), 0, 0, True),
    (9, 17, 2, 1, 64, BF, 16, (0, 600), 0, 0, True),
    # units that one CTA sees through, one after another, and rows enough for the weights of cut ones to
    # take a launch of their own
    (5, 40, 7, 1, 128, BF, 64, (2000, 3500), 0, 0, True),
]


def _lens(seed, Ly, B, H, lo, hi, page):
    """Random lengths, some of them around the ends of blocks and pages."""
    rng = np.random.default_rng(seed)
    n = rng.integers(lo, hi + 1, (Ly, B, H))
    edge = np.array([0, 1, 15, 16, 17, page - 1, page, page + 1, 2 * page - 1])
    pick = rng.random(n.shape) < 0.4
    n[pick] = np.clip(edge[rng.integers(0, len(edge), pick.sum())], lo, hi)
    return n


@pytest.mark.parametrize("i", range(len(CASES)))
@pytest.mark.parametrize("weights", [False, True])
def test_decode_against_reference(i, weights):
    Ly, B, Hq, H, d, dtype, page, (lo, hi), window, sinks, append = CASES[i]
    c = Cache(100 + i, Ly, B, Hq, H, d, dtype, page, _lens(100 + i, Ly, B, H, lo, hi, page), room=3)
    op = reco.RECO_OP_PAGED_WEIGHTS if weights else reco.RECO_OP_PAGED_DECODE
    ws = c.workspace(op)
    for step in range(2):  # the second over what the first appended, through the same workspace
        q, kn, vn = c.token()
        check(c, q, kn if append else None, vn if append else None, window, sinks, weights,
              torch.bfloat16 if dtype == BF and i % 2 else torch.float32, ws)


def test_units_without_rows():
    c = Cache(1, 1, 2, 4, 2, 128, BF, 16, [[[0, 5], [0, 0]]])
    q, _, _ = c.token()
    out, lse = check(c, q, None, None)
    assert (out[0, 0, :2] == 0).all() and torch.isneginf(lse[0, 0, :2]).all() and torch.isfinite(lse[0, 0, 2:]).all()


@pytest.mark.parametrize("dtype,d", [(BF, 128), (F32, 64)])
@pytest.mark.parametrize("page", [16, 64])
def test_rows_outside_the_window_are_not_touched(dtype, d, page):
    """NaN and infinities in rows that are not seen, and no page at all behind their table entries."""
    n, window, sinks = 700, 130, 20
    c = Cache(7, 1, 2, 6, 2, d, dtype, page, n)
    K, V, table = c.K, c.V, c.table.cpu().numpy().copy()
    q, kn, vn = c.token()
    first, last = sinks, n + 1 - window  # rows [first, last) are not seen
    for b in range(2):
        for j in range(first, last):
            K[:, table[b, j // page], :, j % page] = float("nan") if j % 2 else float("inf")
            V[:, table[b, j // page], :, j % page] = float("-inf") if j % 3 else float("nan")
        for p in range(-(-first // page), last // page):  # whole pages of them
            c.table[b, p] = -5
    assert (c.table == -5).any()
    check(c, q, kn, vn, window, sinks)


def test_a_shared_prefix():
    """Two sequences whose first pages are the same: both read them, each appends to its own last page."""
    c = Cache(8, 2, 2, 8, 2, 128, BF, 16, [[[100, 100], [90, 90]]] * 2)
    c.table[1, :5] = c.table[0, :5]
    q, kn, vn = c.token()
    check(c, q, kn, vn)


@pytest.mark.parametrize("weights", [False, True])
def test_the_same_inputs_give_the_same_bits(weights):
    res = []
    for _ in range(3):
        c = Cache(9, 2, 3, 14, 2, 128, BF, 32, _lens(9, 2, 3, 2, 1, 4000, 32))
        out, lse = decode(c, *c.token(), weights=weights)
        res.append((out, lse, c.weights))
    for r in res[1:]:
        assert all(torch.equal(a, b) for a, b in zip(res[0], r))


def test_large_logits_and_one_dominant_row():
    """Logits in the hundreds: nothing overflows, and a row that takes all the weight gives its value."""
    c = Cache(10, 1, 1, 4, 1, 128, F32, 16, 500)
    q, kn, vn = c.token()
    q *= 20.0
    t = c.table.cpu().numpy()
    c.K[0, t[0, 123 // 16], 0, 123 % 16] = 20.0 * q[0, 0, 2] / q[0, 0, 2].norm() * 10
    check(c, q, kn, vn)
    c2 = Cache(11, 1, 1, 4, 1, 128, BF, 16, 500)
    q, kn, vn = c2.token()
    check(c2, (q.float() * 16).to(BF), kn, vn)


def test_more_units_than_one_plan_holds():
    Ly, B, H = 41, 25, 8  # 8200 units
    c = Cache(12, Ly, B, H, H, 64, BF, 16, _lens(12, Ly, B, H, 0, 40, 16))
    q, kn, vn = c.token()
    check(c, q, kn, vn, weights=True)


def test_more_units_than_lengths_staged_in_shared_memory():
    Ly, B, H = 50, 125, 8  # 50000 units
    c = Cache(14, Ly, B, H, H, 64, BF, 16, _lens(14, Ly, B, H, 0, 3, 16))
    q, kn, vn = c.token()
    check(c, q, kn, vn, weights=True)


def test_offsets_beyond_32_bits():
    """Rows behind the first 2^31 elements of the pools, in the last layer and the last pages."""
    H, page, d, n = 2, 64, 128, 200
    n_pages = (2 ** 31 // (H * page * d) // 2) + 300  # two layers of them: the second layer starts behind 2^30
    K = torch.zeros((2, n_pages, H, page, d), dtype=BF, device=DEV)
    V = torch.zeros((2, n_pages, H, page, d), dtype=BF, device=DEV)
    assert K.numel() > 2 ** 31
    table = torch.tensor([[n_pages - 1, n_pages - 7, 3, n_pages - 2]], dtype=torch.int32, device=DEV)
    small = Cache(13, 2, 1, 8, H, d, BF, page, n, room=1)
    st = small.table[0, :4].long()
    K[:, table[0].long()], V[:, table[0].long()] = small.K[:, st].nan_to_num(), small.V[:, st].nan_to_num()
    kv = reco.make_paged_kv(K, V, table, 8)
    q, kn, vn = small.token()
    ws = reco.paged_workspace(reco.RECO_OP_PAGED_WEIGHTS, kv, DEV)
    lens, (out, lse) = small.lens.clone(), small.outputs(BF)
    wts = small.weights[..., :256].clone().contiguous()
    reco.reco_paged_decode_attn_weights(kv, q, kn, vn, lens, small.scale, out, lse, wts, ws)
    o2, l2 = check(small, q, kn, vn, out_dtype=BF)
    assert torch.equal(out, o2) and torch.equal(lse, l2) and torch.equal(wts, small.weights[..., :256])
    assert torch.equal(K[:, table[0].long()], small.K[:, st].nan_to_num())
    budget = torch.tensor([150], dtype=torch.int32, device=DEV)
    ws = reco.paged_workspace(reco.RECO_OP_PAGED_EVICT, kv, DEV)
    reco.reco_paged_evict(kv, wts, lens, budget, 10, 2, None, ws)
    reco.reco_paged_evict(small.kv, small.weights, small.lens, budget, 10, 2, None,
                          small.workspace(reco.RECO_OP_PAGED_EVICT))
    reco.reco_check()
    assert (lens == 150).all() and torch.equal(K[:, table[0].long()], small.K[:, st].nan_to_num())
    assert torch.equal(V[:, table[0].long()], small.V[:, st].nan_to_num())


# ---------------------------------------------------------------- errors
def _refused():
    with pytest.raises(reco.RecoError) as e:
        reco.reco_check()
    assert e.value.status == reco.RECO_EDEVICE
    return str(e.value)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("what", ["negative", "long", "full", "page", "last page", "huge page"])
def test_units_in_error_are_skipped_and_the_others_are_right(dtype, weights, what):
    lens = np.array([[[500, 30], [700, 333]], [[90, 0], [65, 500]]])
    good = Cache(20, 2, 2, 10, 2, 128, dtype, 16, lens)
    c = Cache(20, 2, 2, 10, 2, 128, dtype, 16, lens)
    q, kn, vn = c.token()
    bad = torch.zeros((2, 2, 2), dtype=torch.bool)
    if what in ("negative", "long", "full"):
        c.lens[0, 1, 1] = {"negative": -3, "long": c.cap + 1, "full": c.cap}[what]
        bad[0, 1, 1] = True
    else:  # of sequence 0, the page of row 480, or of row 90: needed by the units that have that row
        at = 480 if what == "page" else 90
        c.table[0, at // 16] = c.kv.n_pages if what != "huge page" else 2 ** 31 - 1
        bad[:, 0] = torch.from_numpy(lens[:, 0] >= (at // 16) * 16)
    before = (c.lens.clone(), c.weights.clone(), c.K.clone())
    out, lse = decode(c, q, kn, vn, weights=weights)
    text = _refused()
    assert {"negative": "length", "long": "length", "full": "room"}.get(what, "page") in text
    wo, wl = decode(good, q, kn, vn, weights=weights)
    reco.reco_check()
    bq = bad.to(DEV).repeat_interleave(5, 2)
    assert (out[bq] == 0).all() and torch.isneginf(lse[bq]).all()
    # the other units: cut over their length elsewhere, so within rounding
    assert torch.allclose(out[~bq], wo[~bq], rtol=1e-4, atol=2e-5) and torch.allclose(lse[~bq], wl[~bq], rtol=1e-5)
    bad = bad.to(DEV)
    assert torch.equal(c.lens[bad], before[0][bad]) and torch.equal(c.lens[~bad], good.lens[~bad])
    assert torch.equal(c.weights[~bad][:, :400].isfinite(), good.weights[~bad][:, :400].isfinite())
    live = torch.arange(c.cap, device=DEV) < before[0].unsqueeze(-1)  # rows that the units in error have
    assert torch.equal(c.weights[bad.unsqueeze(-1) & live], before[1][bad.unsqueeze(-1) & live])
    # the call after it is sound
    c2 = Cache(21, 1, 2, 10, 2, 128, dtype, 16, 300)
    check(c2, *c2.token())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("hi", [100, 700])  # units that go whole to warps, and ranges cut across units
@pytest.mark.parametrize("what", ["length", "page"])
def test_errors_among_many_units(dtype, hi, what):
    lens = _lens(24, 10, 20, 2, 60, hi, 16)
    good, c = (Cache(24, 10, 20, 14, 2, 128, dtype, 16, lens) for _ in range(2))
    q, kn, vn = c.token()
    bad = torch.zeros((10, 20, 2), dtype=torch.bool)
    if what == "length":
        c.lens[3, 5, 1] = c.cap + 7
        c.lens[9, 19, 0] = -1
        bad[3, 5, 1] = bad[9, 19, 0] = True
    else:
        c.table[7, 3] = -1  # rows 48 to 63, which every unit has
        bad[:, 7] = True
    before = (c.lens.clone(), c.weights.clone())
    ws = c.workspace(reco.RECO_OP_PAGED_WEIGHTS)
    out, lse = decode(c, q, kn, vn, ws=ws)
    assert what in _refused()
    wo, wl = decode(good, q, kn, vn)
    reco.reco_check()
    bq, bad = bad.to(DEV).repeat_interleave(7, 2), bad.to(DEV)
    assert (out[bq] == 0).all() and torch.isneginf(lse[bq]).all()
    assert torch.allclose(out[~bq], wo[~bq], rtol=1e-4, atol=2e-5) and torch.allclose(lse[~bq], wl[~bq], rtol=1e-5)
    assert torch.equal(c.lens[bad], before[0][bad]) and torch.equal(c.lens[~bad], good.lens[~bad])
    live = torch.arange(c.cap, device=DEV) < torch.from_numpy(lens).to(DEV).unsqueeze(-1)
    assert torch.equal(c.weights[bad.unsqueeze(-1) & live], before[1][bad.unsqueeze(-1) & live])
    assert torch.allclose(c.weights[~bad], good.weights[~bad], rtol=1e-4, atol=1e-7)
    # the next call through the same workspace
    if what == "page":
        c.table[7, 3] = good.table[7, 3]
    c.lens.copy_(good.lens)
    c.K.copy_(good.K), c.V.copy_(good.V), c.weights.copy_(good.weights)
    o1, l1 = decode(c, q, None, None, ws=ws)
    o2, l2 = decode(good, q, None, None)
    reco.reco_check()
    assert torch.equal(o1, o2) and torch.equal(l1, l2) and torch.equal(c.weights, good.weights)


def test_a_workspace_survives_an_error():
    c = Cache(22, 1, 2, 6, 2, 128, BF, 16, [[[3000, 3000], [50, 50]]])
    ws = c.workspace(reco.RECO_OP_PAGED_WEIGHTS)
    q, kn, vn = c.token()
    keep = int(c.table[0, 100])
    c.table[0, 100] = -1
    decode(c, q, kn, vn, ws=ws)
    _refused()
    c.table[0, 100] = keep
    c.lens[:] = torch.tensor([[[3000, 3000], [50, 50]]], device=DEV)
    check(c, q, kn, vn, ws=ws, exact_pool=False)


# ---------------------------------------------------------------- streams and graphs
def test_captured_and_replayed_on_streams_of_their_own():
    """Two graphs, each with its workspace, replayed at the same time on two streams: as eager calls."""
    runs = []
    for seed in (30, 31):
        c, eager = (Cache(seed, 2, 2, 14, 2, 128, BF, 16, _lens(seed, 2, 2, 2, 1, 3000, 16), room=8) for _ in range(2))
        q, kn, vn = c.token()
        out, lse = c.outputs(BF)
        ws, wse = c.workspace(reco.RECO_OP_PAGED_WEIGHTS), c.workspace(reco.RECO_OP_PAGED_EVICT)
        budget = torch.tensor([500, 10 ** 6], dtype=torch.int32, device=DEV)
        warm = Cache(seed, 2, 2, 14, 2, 128, BF, 16, 20)
        decode(warm, *warm.token())
        torch.cuda.synchronize()
        st = torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st, capture_error_mode="relaxed"):
            reco.reco_paged_decode_attn_weights(c.kv, q, kn, vn, c.lens, c.scale, out, lse, c.weights, ws, 2000, 4)
            reco.reco_paged_evict(c.kv, c.weights, c.lens, budget, 16, 4, None, wse)
        runs.append((c, eager, graph, st, out, lse, (q, kn, vn), budget, ws, wse))  # (a graph keeps no workspace alive)
    torch.cuda.synchronize()
    for _ in range(5):
        for c, eager, graph, st, *_ in runs:
            with torch.cuda.stream(st):
                graph.replay()
    torch.cuda.synchronize()
    reco.reco_check()
    for c, eager, graph, st, out, lse, (q, kn, vn), budget, *_ in runs:
        e_out, e_lse = eager.outputs(BF)
        ws, wse = eager.workspace(reco.RECO_OP_PAGED_WEIGHTS), eager.workspace(reco.RECO_OP_PAGED_EVICT)
        for _ in range(5):
            reco.reco_paged_decode_attn_weights(eager.kv, q, kn, vn, eager.lens, eager.scale, e_out, e_lse, eager.weights,
                                                ws, 2000, 4)
            reco.reco_paged_evict(eager.kv, eager.weights, eager.lens, budget, 16, 4, None, wse)
        assert torch.equal(out, e_out) and torch.equal(lse, e_lse) and torch.equal(c.lens, eager.lens)
        assert torch.equal(c.weights, eager.weights)
        assert torch.equal(c.K.view(torch.int16), eager.K.view(torch.int16))


def test_a_stream_given_by_argument():
    c = Cache(32, 1, 2, 4, 2, 128, BF, 16, 200)
    q, kn, vn = c.token()
    out, lse = c.outputs(torch.float32)
    ws = c.workspace(reco.RECO_OP_PAGED_DECODE)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    reco.reco_paged_decode_attn(c.kv, q, kn, vn, c.lens, c.scale, out, lse, ws, stream=st)
    torch.cuda.current_stream().wait_stream(st)
    d = Cache(32, 1, 2, 4, 2, 128, BF, 16, 200)
    o2, l2 = check(d, q, kn, vn, weights=False)
    assert torch.equal(out, o2) and torch.equal(lse, l2)


# ---------------------------------------------------------------- eviction
def _gather_reference(c, budget, w, sinks):
    K, V, table, lens, W = c.host()
    kept = paged.evict(K, V, W, table, lens, budget, w, sinks)
    return K, V, W, lens, kept


def _check_evict(c, budget, w, sinks, with_kept=True):
    Ly, B, Hq, H, d = c.shape
    K, V, W, lens, kept = _gather_reference(c, budget, w, sinks)
    idx = torch.full((Ly, B, H, c.cap), -9, dtype=torch.int32, device=DEV) if with_kept else None
    ws = c.workspace(reco.RECO_OP_PAGED_EVICT)
    reco.reco_paged_evict(c.kv, c.weights, c.lens, torch.tensor(budget, dtype=torch.int32, device=DEV), w, sinks, idx, ws)
    reco.reco_check()
    assert np.array_equal(c.lens.cpu().numpy(), lens)
    table = c.table.cpu().numpy()
    for pool, ref in ((c.K, K), (c.V, V)):  # all rows, those behind the new lengths among them
        assert np.array_equal(np64(pool), ref, equal_nan=True)
    got = np64(c.weights)
    for i in np.ndindex(Ly, B, H):
        n = lens[i]
        assert np.array_equal(got[i][:n], W[i][:n], equal_nan=True)
        assert np.array_equal(got[i][n:], W[i][n:], equal_nan=True)
        if with_kept:
            k = idx[i].cpu().numpy()
            m = len(kept[i]) if i in kept else 0
            assert np.array_equal(k[:m], kept[i] if m else []) and (k[m:] == -9).all()
    del table


EVICT = [
    # (layers, B, H_kv, d, dtype, page, (lo, hi), budgets, w, sinks)
    (1, 1, 2, 64, F32, 16, (512, 512), [128], 16, 4),
    (2, 3, 2, 128, BF, 16, (1, 300), [100, 40, 10 ** 6], 8, 0),
    (1, 3, 1, 128, BF, 32, (200, 900), [150, 899, 333], 32, 5),
    (3, 2, 3, 64, BF, 64, (0, 700), [64, 65], 1, 0),
    (1, 2, 2, 128, F32, 128, (300, 1200), [299, 31], 0, 31),
    (1, 2, 2, 128, F32, 256, (300, 1200), [20, 256], 20, 0),  # nothing but the latest rows
    (1, 2, 1, 64, F32, 16, (20, 60), [0, 1], 0, 0),           # down to nothing
    (1, 2, 1, 128, BF, 16, (2000, 3500), [1999, 1000], 64, 17),
    (1, 1, 1, 64, BF, 64, (60000, 60000), [41111], 128, 4),   # more candidates than shared memory holds
    (28, 8, 4, 64, BF, 16, (30, 250), [60, 10 ** 6, 100, 10 ** 6, 10 ** 6, 10 ** 6, 33, 10 ** 6], 32, 1),
    (28, 10, 5, 64, BF, 16, (500, 1000), [600] * 10, 3, 3),   # a warp per unit
    # few long units: clusters of CTAs
    (1, 1, 1, 64, BF, 16, (131000, 131000), [50000], 32, 4),
    (1, 2, 1, 64, F32, 64, (2100, 9000), [2000, 1500], 0, 0),
    (2, 2, 2, 128, BF, 256, (9000, 30000), [8000, 29000], 64, 16),
    (1, 5, 4, 64, BF, 32, (5000, 8300), [4000, 10 ** 6, 64, 4999, 7000], 60, 4),
    (1, 3, 1, 64, BF, 16, (60000, 90000), [59999, 2, 41111], 1, 1),
    (1, 1, 2, 64, BF, 128, (400000, 400000), [100000], 128, 4),  # more keys than the cluster holds
    # many cut units, by columns: rows of 256 and 512 bytes, and of so few that a step does not fill
    (10, 10, 3, 128, BF, 32, (100, 300), [90] * 10, 8, 2),
    (8, 6, 3, 128, F32, 16, (100, 300), [40, 77, 90, 33, 50, 10 ** 6], 8, 2),
    (20, 10, 3, 64, BF, 16, (20, 60), [17] * 10, 2, 1),
]


@pytest.mark.parametrize("i", range(len(EVICT)))
@pytest.mark.parametrize("ties", [False, True])
def test_evict_against_reference(i, ties):
    Ly, B, H, d, dtype, page, (lo, hi), budget, w, sinks = EVICT[i]
    c = Cache(200 + i, Ly, B, 2 * H, H, d, dtype, page, _lens(200 + i, Ly, B, H, lo, hi, page))
    if ties:  # few values, and both zeros
        c.weights = (c.weights * 5).floor_() - 2.0
        c.weights[..., ::3] *= -0.0
    _check_evict(c, budget, w, sinks, with_kept=i % 2 == 0)


def test_evict_ranks_infinities_and_nan():
    c = Cache(220, 1, 1, 2, 1, 64, F32, 16, 100)
    c.weights[..., 10:20] = float("inf")
    c.weights[..., 30:40] = float("-inf")
    c.weights[0, 0, 0, 50] = float("nan")
    c.weights[0, 0, 0, 51] = -float("nan")
    rows = list(range(10, 20)) + [50, 51]
    idx = torch.zeros((1, 1, 1, c.cap), dtype=torch.int32, device=DEV)
    reco.reco_paged_evict(c.kv, c.weights, c.lens, torch.tensor([12], dtype=torch.int32, device=DEV), 0, 0, idx,
                          c.workspace(reco.RECO_OP_PAGED_EVICT))
    reco.reco_check()
    assert idx[0, 0, 0, :12].tolist() == rows


@pytest.mark.parametrize("what", ["negative", "long", "budget", "page"])
def test_evict_leaves_units_in_error_untouched(what):
    lens = np.array([[[300, 200], [280, 290]]])
    c = Cache(230, 1, 2, 4, 2, 128, BF, 16, lens)
    good = Cache(230, 1, 2, 4, 2, 128, BF, 16, lens)
    budget, bad = [150, 160], [(0, 1, 1)]
    if what in ("negative", "long"):
        c.lens[0, 1, 1] = -1 if what == "negative" else c.cap + 1
    elif what == "budget":
        budget, bad = [150, 11], [(0, 1, 0), (0, 1, 1)]
    else:
        c.table[1, 17] = c.kv.n_pages  # rows 272 to 287 of sequence 1
        bad = [(0, 1, 0), (0, 1, 1)]
    before = (c.K.clone(), c.V.clone(), c.weights.clone(), c.lens.clone())
    ws = c.workspace(reco.RECO_OP_PAGED_EVICT)
    reco.reco_paged_evict(c.kv, c.weights, c.lens, torch.tensor(budget, dtype=torch.int32, device=DEV), 8, 4, None, ws)
    text = _refused()
    assert {"budget": "keep", "page": "page"}.get(what, "length") in text
    reco.reco_paged_evict(good.kv, good.weights, good.lens, torch.tensor([150, 160], dtype=torch.int32, device=DEV), 8, 4,
                          None, ws)
    reco.reco_check()
    t = good.table.cpu().numpy()
    for i in np.ndindex(1, 2, 2):
        want = before if i in bad else (good.K, good.V, good.weights, good.lens)
        assert c.lens[i] == want[3][i] and torch.equal(c.weights[i], want[2][i])
        pages = torch.from_numpy(t[i[1]][:18].astype(np.int64)).to(DEV)
        for got, ref in ((c.K, want[0]), (c.V, want[1])):
            assert torch.equal(got[i[0], pages, i[2]].view(torch.int16), ref[i[0], pages, i[2]].view(torch.int16))


@pytest.mark.parametrize("what", ["negative", "long", "budget", "page"])
def test_evict_of_long_units_leaves_those_in_error_untouched(what):
    lens = np.array([[[9000, 8700], [8193, 8900], [12, 8888]]])
    c, good = (Cache(231, 1, 3, 4, 2, 64, BF, 64, lens) for _ in range(2))
    budget, bad = [150, 8192, 8000], [(0, 1, 1)]
    if what in ("negative", "long"):
        c.lens[0, 1, 1] = -1 if what == "negative" else c.cap + 1
    elif what == "budget":
        budget, bad = [150, 11, 8000], [(0, 1, 0), (0, 1, 1)]
    else:
        c.table[1, 100] = -1
        bad = [(0, 1, 0), (0, 1, 1)]
    before = (c.K.clone(), c.V.clone(), c.weights.clone(), c.lens.clone())
    ws = c.workspace(reco.RECO_OP_PAGED_EVICT)
    reco.reco_paged_evict(c.kv, c.weights, c.lens, torch.tensor(budget, dtype=torch.int32, device=DEV), 8, 4, None, ws)
    text = _refused()
    assert {"budget": "keep", "page": "page"}.get(what, "length") in text
    reco.reco_paged_evict(good.kv, good.weights, good.lens, torch.tensor([150, 8192, 8000], dtype=torch.int32, device=DEV),
                          8, 4, None, ws)
    reco.reco_check()
    assert good.lens.flatten().tolist() == [150, 150, 8192, 8192, 12, 8000]
    t = good.table.cpu().numpy()
    for i in np.ndindex(1, 3, 2):
        want = before if i in bad else (good.K, good.V, good.weights, good.lens)
        assert c.lens[i] == want[3][i] and torch.equal(c.weights[i], want[2][i])
        pages = torch.from_numpy(t[i[1]][:(int(lens[i]) + 63) // 64].astype(np.int64)).to(DEV)
        for got, ref in ((c.K, want[0]), (c.V, want[1])):
            assert torch.equal(got[i[0], pages, i[2]].view(torch.int16), ref[i[0], pages, i[2]].view(torch.int16))


def test_evict_of_long_units_ranks_infinities_and_nan():
    c = Cache(221, 1, 1, 2, 1, 64, F32, 16, 20000)
    c.weights[..., 5000:5010] = float("inf")
    c.weights[..., 30:40] = float("-inf")
    c.weights[0, 0, 0, 19999] = float("nan")
    c.weights[0, 0, 0, 51] = -float("nan")
    rows = [51] + list(range(5000, 5010)) + [19999]
    idx = torch.zeros((1, 1, 1, c.cap), dtype=torch.int32, device=DEV)
    reco.reco_paged_evict(c.kv, c.weights, c.lens, torch.tensor([12], dtype=torch.int32, device=DEV), 0, 0, idx,
                          c.workspace(reco.RECO_OP_PAGED_EVICT))
    reco.reco_check()
    assert idx[0, 0, 0, :12].tolist() == rows


# ---------------------------------------------------------------- together
@pytest.mark.parametrize("dtype,window", [(BF, 0), (F32, 0), (BF, 60)])
def test_a_run_of_tokens_with_evictions(dtype, window):
    """Forty tokens, decoded with their weights and evicted to a budget whenever a sequence is eight rows
    over it, against the reference in lock step (each eviction from the library's own sums)."""
    c = Cache(300, 2, 2, 6, 2, 64, dtype, 16, [[[70, 70], [90, 90]]] * 2, room=40)
    c.weights.zero_()
    ws, wse = c.workspace(reco.RECO_OP_PAGED_WEIGHTS), c.workspace(reco.RECO_OP_PAGED_EVICT)
    cuts = 0
    for t in range(40):
        q, kn, vn = c.token()
        check(c, q, kn, vn, window, 2 if window else 0, ws=ws)
        over = c.lens[0, :, 0].cpu().numpy() >= np.array([80, 80]) + 8
        if over.any():
            budget = np.where(over, 80, 10 ** 6).tolist()
            K, V, W, lens, kept = _gather_reference(c, budget, 10, 2)
            reco.reco_paged_evict(c.kv, c.weights, c.lens, torch.tensor(budget, dtype=torch.int32, device=DEV), 10, 2,
                                  None, wse)
            reco.reco_check()
            assert np.array_equal(c.lens.cpu().numpy(), lens) and np.array_equal(np64(c.K), K, equal_nan=True)
            assert np.array_equal(np64(c.weights), W) and np.array_equal(np64(c.V), V, equal_nan=True)
            cuts += len(kept)
    assert cuts >= 4 * 4
