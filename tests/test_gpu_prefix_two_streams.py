"""Decode attention over shared prefixes from bf16 caches to bf16 output: the form with two streams of products, whose row tiles have
one half of query rows (each stream takes half of the keys) or two (each takes a half of the rows), and whose output stays in tensor memory.

Bounds: test_gpu_prefix.py's, with two bf16 parts of the probabilities (2^-17).
"""
import numpy as np
import pytest
import torch

from paper_2608_04771_gb300 import reco
from test_gpu_prefix import BF, DEV, F32, U, Batch, _lib, bits, failing, np64  # noqa: F401

pytestmark = pytest.mark.gpu


class Two(Batch):
    def __init__(self, *a, **kw):
        super().__init__(*a, **{"out_dtype": BF, **kw})

    def check(self, ref, before, pool=True):
        super().check(ref, before, pool)
        (ro, rl, big, seen, absv), *_ = ref
        prob = 2 * ((self.dims[4] + 6) * U * big) + 2.0 ** -21 + 4 * U * np.where(np.isfinite(rl), np.abs(rl), 0.0)
        part = 2.0 ** -26 if self.out_dtype == F32 else 2.0 ** -17
        tol = (prob + (192 + 32 + seen / 8) * U + part)[..., None] * absv * (1 + 2.0 ** -8)
        tol = tol + np.abs(ro) * (2.0 ** -8 if self.out_dtype == BF else U)
        there = ~np.isnan(rl)
        off = np.abs(np64(self.out) - ro)[there]
        assert (off <= tol[there]).all(), (off / (tol[there] + 1e-300)).max()


# sequences and query heads per KV head: one half; two, the second with one row to 128; several row tiles, the last of one half or two
SHAPES = [(2, 1), (16, 8), (17, 8), (33, 4), (32, 8), (19, 7), (36, 7), (37, 7), (46, 7), (64, 5), (70, 3), (43, 16), (100, 5)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,G", SHAPES)
@pytest.mark.parametrize("P", [100, 700])
def test_rows_of_a_group(n, G, d, P):
    Two(n, 1, 2 * G, 2, d, BF, 16, [0] * n, [P] * n, np.random.default_rng(n).integers(0, 20, (1, n, 2))).go()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,G,P,Ly,H", [(3, 4, 9000, 4, 4), (33, 4, 20011, 1, 2), (46, 7, 6001, 2, 2), (64, 5, 5003, 2, 3), (9, 16, 30001, 1, 1)])
def test_long_prefixes_are_cut_between_ctas(n, G, P, Ly, H, d):
    """Pieces of several key tiles, of which CTAs keep a second partial: of up to 256 rows where a row tile has two halves."""
    c = Two(n, Ly, G * H, H, d, BF, 64, [0] * n, [P] * n, 17, garbage=False)
    c.go()
    out, lse = c.out.clone(), c.lse.clone()
    c.lens -= 1
    c.run()
    reco.reco_check()
    assert torch.equal(bits(out), bits(c.out)) and torch.equal(lse, c.lse)  # the same inputs, the same bits


def marked(n, G, P, page, dtype, d, out_dtype, size):
    """Rows of 16 tell themselves apart: a column of V each and, where columns repeat, other values.  `size` of the queries: small ones
    give every row a like weight (16 in another's place move a column by 1/10 of it and more), large ones weights that differ by
    factors (16 with another's weights move it likewise)."""
    c = (Two if dtype == BF else Batch)(n, 2, 2 * G, 2, d, dtype, page, [0] * n, [P] * n, 70, garbage=False, out_dtype=out_dtype)
    c.q.mul_(size)
    c.V.zero_()
    table = c.table.cpu().numpy()
    j = np.arange(P)
    at = torch.from_numpy(table[0, j // page].astype(np.int64)).to(DEV), torch.from_numpy(j % page).to(DEV)
    col, value = torch.from_numpy(j // 16 % d).to(DEV), torch.from_numpy(1.0 + j // 16 // d).to(DEV).to(dtype)
    c.V[:, at[0], :, at[1], col] = value.view(-1, 1, 1).expand(-1, 2, 2)
    return c, at


@pytest.mark.parametrize("size", [0.25, 1.5])
@pytest.mark.parametrize("out_dtype", [BF, F32])
@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F32, 128)])
@pytest.mark.parametrize("n,G,P,page", [(3, 4, 20011, 16), (3, 4, 9003, 256), (40, 4, 9001, 32), (80, 4, 5000, 64)])
def test_every_row_of_v_is_where_it_belongs(n, G, P, page, dtype, d, out_dtype, size):
    marked(n, G, P, page, dtype, d, out_dtype, size)[0].go()


@pytest.mark.parametrize("out_dtype", [BF, F32])
@pytest.mark.parametrize("size", [0.25, 1.5])
@pytest.mark.parametrize("rows", [16, 64, 128])
def test_rows_of_v_elsewhere_would_be_seen(rows, size, out_dtype):
    """The check itself: a reference in which a tile of V is read twice, or two have changed places, is out of its bounds."""
    c, at = marked(3, 4, 20011, 16, BF, 128, out_dtype, size)
    before = c.K.clone(), c.V.clone()
    good = c.reference()
    c.run()
    reco.reco_check()
    c.check(good, before)
    x, y = slice(5 * rows, 6 * rows), slice(1900 // rows * rows, (1900 // rows + 1) * rows)
    ids, off = at
    for other in ("twice", "exchanged"):
        if other == "exchanged" and size < 1:
            continue
        c.V.copy_(before[1])
        for ly in range(2):
            c.V[ly, ids[x], :, off[x]] = before[1][ly, ids[y], :, off[y]]
            if other == "exchanged":
                c.V[ly, ids[y], :, off[y]] = before[1][ly, ids[x], :, off[x]]
        c.lens -= 1
        wrong = c.reference()
        c.lens += 1
        with pytest.raises(AssertionError):
            c.check(wrong, before, pool=False)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,G,P,Ly,H,page", [(3, 2, 9000, 4, 4, 16), (40, 4, 1500, 2, 2, 32), (80, 4, 700, 2, 2, 16), (2, 1, 700, 1, 1, 16)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_logits_that_grow_along_the_rows(n, G, P, Ly, H, page, d, sign):
    """The maximum grows by far more than 2^12 from block to block (or falls): the output so far is rescaled where it lies."""
    c = Two(n, Ly, G * H, H, d, BF, page, [0] * n, [P] * n, 90, garbage=False)
    c.q[:] = sign * c.q.abs()
    table = c.table.cpu().numpy()
    for i in range(P // page):
        x = int(table[0, i])
        c.K[:, x] = (c.K[:, x].abs() * (0.25 * i * page / 16)).to(BF)
    c.scale = 0.5
    c.go()


@pytest.mark.parametrize("n,G", [(3, 2), (40, 4), (80, 4)])
@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0])
def test_scales(n, G, scale):
    c = Two(10, 1, 2 * G, 2, 64, BF, 16, [0] * n, [300] * n, 40)
    c.scale = scale
    c.go()


@pytest.mark.parametrize("n,G", [(3, 2), (40, 4), (80, 4)])
def test_nan_and_infinities_among_the_rows(n, G):
    """They reach the heads that see them, and no other: a row of the prefix all of the group, a query its head."""
    def batch():
        return Two(11, 1, 2 * G, 2, 64, BF, 16, [0] * n + [1] * 2, [140] * n + [200] * 2, 40)
    c = batch()
    c.K[0, int(c.table[0, 2]), 1, 3, 7] = float("nan")  # of the first group, KV head 1
    c.q[0, n + 1, 0, 5] = float("nan")
    ref, before = c.reference(), (c.K.clone(), c.V.clone())
    (_, rl, *_), *_ = ref
    assert np.isnan(rl[0, :n, G:]).all() and np.isnan(rl[0, n + 1, 0]) and np.isnan(rl).sum() == n * G + 1
    c.run()
    reco.reco_check()
    c.check(ref, before, pool=False)
    c = batch()  # an infinite key: logits of -inf (weight zero)
    c.q[:] = c.q.abs()
    c.K[0, int(c.table[0, 1]), 0, 2, 9] = float("-inf")
    c.go()
    c = batch()  # an infinite value, in its element alone
    c.V[0, int(c.table[n, 0]), 0, 2, 9] = float("inf")
    c.run()
    reco.reco_check()
    assert ~torch.isfinite(c.out[0, n:, :G, 9]).any() and torch.isfinite(c.out[0, n:, :G, :9]).all()
    assert torch.isfinite(c.lse).all() and torch.isfinite(c.out[0, :n]).all() and torch.isfinite(c.out[0, :, G:]).all()
    c = batch()  # a logit of +inf
    c.q[:] = c.q.abs()
    c.K[0, int(c.table[0, 1]), 0, 2, 9] = float("inf")
    c.run()
    reco.reco_check()
    assert torch.isnan(c.lse[0, :n, :G]).all() and torch.isfinite(c.lse[0, n:]).all() and torch.isfinite(c.lse[0, :, G:]).all()


@pytest.mark.parametrize("n,G", [(2, 2), (40, 4), (80, 4)])
def test_logits_that_are_all_minus_infinity(n, G):
    c = Two(12, 1, G, 1, 64, BF, 16, [0] * n, [300] * n, 4, append=False, garbage=False)
    c.q[:] = c.q.abs()
    c.K[0, :, 0, :, 3] = float("-inf")
    c.run()
    reco.reco_check()
    assert torch.isneginf(c.lse).all() and (c.out == 0).all()
    c = Two(13, 1, G, 1, 64, BF, 16, [0] * n, [300] * n, 4, append=False, garbage=False)  # of the first rows alone
    c.q[:] = c.q.abs()
    for i in range(9):
        c.K[0, int(c.table[0, i]), 0, :, 3] = float("-inf")
    c.go()


@pytest.mark.parametrize("n,G", [(3, 2), (40, 4), (80, 4)])
def test_units_prefixes_and_pages_in_error(n, G):
    group, shared = [0] * n + [1] * 2 + [2], [300] * n + [40] * 2 + [20]
    batch = lambda: Two(14, 2, 2 * G, 2, 64, BF, 16, group, shared, 40)  # noqa: E731
    every = lambda *bs: {(ly, b, h) for ly in range(2) for b in bs for h in range(2)}  # noqa: E731
    c = batch()
    c.lens[1, 1, 0] = 299
    c.lens[0, n + 2, 1] = -5
    failing(c, "length-out-of-range", {(1, 1, 0), (0, n + 2, 1)})
    c = batch()

    def wrong():
        c.shared[n - 1] = 299
    failing(c, "length-out-of-range", every(n - 1), wrong)
    # pages of prefixes (the whole group) and of own rows (more than 32 of them: the attention's)
    for b, k, units in ((0, 1, every(*range(n))), (0, 18, every(*range(n))), (n, 2, every(n, n + 1)), (n - 1, 20, every(n - 1)), (n + 2, 2, every(n + 2))):
        c = batch()
        last = [b, k]

        def bad():
            c.table[last[0], last[1]] = -1
        failing(c, "page-out-of-range", units, bad)


@pytest.mark.parametrize("n,P,mine,Ly,page", [(24, 140, 20, 6, 64), (39, 0, 130, 3, 16), (12, 1000, 60, 4, 128), (3, 300, 1, 28, 16)])
def test_the_same_bits_again_and_again(n, P, mine, Ly, page):
    """Many short items one after the other in every CTA, whose roles then run far apart: nothing depends on when."""
    own = np.random.default_rng(n).integers(0, mine, (Ly, n, 2))
    c = Two(n, Ly, 14, 2, 128, BF, page, np.repeat(np.arange(n // 3), 3).tolist(), [P] * n, own, garbage=False).go()
    out, lse = c.out.clone(), c.lse.clone()
    for _ in range(150):
        c.lens -= 1
        c.run()
        assert torch.equal(bits(out), bits(c.out)) and torch.equal(lse, c.lse)
    reco.reco_check()


@pytest.mark.parametrize("d,page", [(64, 16), (128, 64), (128, 256)])
def test_groups_of_many_sizes(d, page):
    """Short pieces of few and of many query rows in turn: one half, two, several row tiles."""
    sizes, prefix = [1, 2, 33, 1, 40, 3, 26, 64, 70], [0, 140, 129, 300, 260, 515, 31, 700, 400]
    group = [g for g, n in enumerate(sizes) for _ in range(n)]
    shared = [p for n, p in zip(sizes, prefix) for _ in range(n)]
    mine = np.random.default_rng(5).integers(0, 200, (3, len(group), 2))
    b = Two(34, 3, 8, 2, d, BF, page, group, shared, mine)
    lens = b.lens.clone()
    b.go()
    out, lse = b.out.clone(), b.lse.clone()
    for _ in range(20):
        b.lens.copy_(lens)
        b.run()
        reco.reco_check()
        assert torch.equal(bits(b.out), bits(out)) and torch.equal(bits(b.lse), bits(lse))


def test_plans_of_many_sequences_with_row_tiles_of_every_kind():
    rng = np.random.default_rng(8)
    group, shared = [], []
    while len(group) < 1500:
        k, p = int(rng.integers(1, 90)), int(rng.integers(0, 300))
        group += [len(group)] * k
        shared += [p] * k
    n = len(group)
    Two(n, 1, 4, 1, 64, BF, 16, group, shared, rng.integers(0, 9, (1, n, 1))).go()
