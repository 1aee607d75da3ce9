"""Decode attention over shared prefixes on the GPU against the fp64 reference (oracle/paged.py), and a run
of append, attention and eviction together.

Bounds as test_gpu_paged.py's (u = 2^-24): a logit (d + 4) u big and the exponential's 2 u big and 2^-22; a
probability twice that and 2^-21; an output that times sum_j p_j |v_j|, its chain of additions (blocks of up to 128
rows, then blocks, then pieces: 192 + n / 8 of them) and the parts' joining (32 more), u each; over bf16 caches the
probabilities enter in three bf16 parts, 2^-26, or, with bf16 output, in one, 2^-8; a bf16
output half a bf16 step.  A part's log2 is rounded where the parts join: 2 u of the lse's size more per probability.
"""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2608_04771_gb300 import reco

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2608_04771_gb300 import build
    build.build()
    reco.lib()


def np64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == BF else torch.int32)


class Batch:
    """A paged cache of sequences in groups.  Every row that no sequence may read is NaN, table entries that no
    row is needed from name no page.  mine [Ly, B, H]: rows behind the prefix."""

    def __init__(self, seed, Ly, Hq, H, d, dtype, page, group, shared, mine, append=True, out_dtype=None, garbage=True):
        B = len(group)
        self.dims, self.dtype, self.page, self.group, self.shared_list = (Ly, B, Hq, H, d), dtype, page, list(group), list(shared)
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.rand = lambda *s: torch.randn(s, generator=g, device=DEV).to(dtype)
        rng = np.random.default_rng(seed)
        mine = np.broadcast_to(np.asarray(mine), (Ly, B, H)).astype(np.int32)
        lens = mine + np.asarray(shared, np.int32)[None, :, None]
        lead = paged.prefix_lead(group)
        room = 1 if append else 0
        need = [-(-(int(lens[:, b].max()) + room) // page) for b in range(B)]
        first = [0 if lead[b] == b else shared[b] // page for b in range(B)]
        n_pages = sum(max(0, n - f) for n, f in zip(need, first)) + 2
        ids = rng.permutation(n_pages)
        table = rng.choice([-1, 2 ** 31 - 1, n_pages], (B, max(need) + 1)).astype(np.int32)
        at = 0
        for b in range(B):
            k = max(0, need[b] - first[b])
            table[b, first[b]:first[b] + k] = ids[at:at + k]
            at += k
        self.K, self.V = self.rand(Ly, n_pages, H, page, d), self.rand(Ly, n_pages, H, page, d)
        if garbage:
            live = torch.zeros((Ly, n_pages, H, page), dtype=torch.bool)
            for ly, b, h in np.ndindex(Ly, B, H):
                j = np.arange(0 if lead[b] == b else shared[b], lens[ly, b, h])
                live[ly, table[b, j // page], h, j % page] = True
            self.K[~live.to(DEV)] = float("nan")
            self.V[~live.to(DEV)] = float("nan")
        self.table, self.lens = torch.from_numpy(table).to(DEV), torch.from_numpy(lens).to(DEV)
        self.groups = torch.tensor(group, dtype=torch.int32, device=DEV)
        self.shared = torch.tensor(shared, dtype=torch.int32, device=DEV)
        self.kv = reco.make_paged_kv(self.K, self.V, self.table, Hq)
        self.scale = float(d) ** -0.5
        self.ws = reco.paged_workspace(reco.RECO_OP_PAGED_PREFIX, self.kv, DEV)
        self.ws[8192:] = 255  # NaN, should anything be read that was not written
        self.out_dtype = out_dtype or dtype
        self.token(append)

    def token(self, append=True):
        Ly, B, Hq, H, d = self.dims
        self.q = self.rand(Ly, B, Hq, d)
        self.kn, self.vn = (self.rand(Ly, B, H, d), self.rand(Ly, B, H, d)) if append else (None, None)
        self.out = torch.full((Ly, B, Hq, d), 7.0, device=DEV, dtype=self.out_dtype)
        self.lse = torch.full((Ly, B, Hq), 7.0, device=DEV)

    def run(self, **kw):
        a = dict(ws=self.ws, lse=self.lse)
        a.update(kw)
        reco.reco_paged_prefix_attn(self.kv, self.q, self.kn, self.vn, self.lens, self.groups, self.shared, self.scale,
                                    self.out, **a)

    def reference(self, skip=()):
        K, V, lens = np64(self.K), np64(self.V), self.lens.cpu().numpy().copy()
        r = paged.prefix_decode(K, V, self.table.cpu().numpy(), lens, np64(self.q), np64(self.kn), np64(self.vn), self.scale,
                                self.group, self.shared.tolist(), skip)
        return r, K, V, lens

    def check(self, ref, before, pool=True):
        (ro, rl, big, seen, absv), K, V, lens = ref
        d = self.dims[4]
        go, gl = np64(self.out), np64(self.lse)
        nan = np.isnan(rl)
        size = np.where(np.isfinite(rl), np.abs(rl), 0.0)
        prob = 2 * ((d + 6) * U * big) + 2.0 ** -21 + 4 * U * size
        chain = (192 + 32 + seen / 8) * U
        bf16 = self.dtype == BF
        part = 0.0 if not bf16 else (2.0 ** -26 if self.out_dtype == F32 else 2.0 ** -8)
        t_out = (prob + chain + part)[..., None] * absv
        t_out = t_out * (1 + 2.0 ** -8) + np.abs(ro) * 2.0 ** -8 if self.out_dtype == BF else t_out + np.abs(ro) * U
        t_lse = (d + 6) * U * big + 2.0 ** -21 + chain + 4 * U * size
        none = (seen == 0) & ~nan
        assert np.isnan(go[nan]).all() and np.isnan(gl[nan]).all() and not np.isnan(go[~nan]).any()
        assert np.array_equal(np.isneginf(gl), none) and (go[none] == 0).all()
        off = np.abs(go - ro)[~nan]
        assert (off <= t_out[~nan]).all(), (off / (t_out[~nan] + 1e-300)).max()
        live = ~none & ~nan
        off = np.abs(gl[live] - rl[live])
        assert (off <= t_lse[live]).all(), (off / t_lse[live]).max()
        assert np.array_equal(self.lens.cpu().numpy(), lens)
        if pool:
            for t, b, want in ((self.K, before[0], K), (self.V, before[1], V)):
                want = torch.from_numpy(want).to(DEV).to(self.dtype)
                assert torch.equal(bits(t), torch.where(torch.isnan(want), bits(b), bits(want)))

    def go(self, **kw):
        ref, before = self.reference(), (self.K.clone(), self.V.clone())
        self.run(**kw)
        reco.reco_check()
        self.check(ref, before)
        return self


@pytest.mark.parametrize("out_dtype", [BF, F32])
@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("append", [True, False])
def test_types_and_dims(dtype, d, out_dtype, append):
    mine = np.random.default_rng(1).integers(0, 70, (2, 7, 2))
    Batch(1, 2, 6, 2, d, dtype, 16, [0, 0, 0, 1, 2, 2, 2], [150, 150, 150, 40, 33, 33, 33], mine, append, out_dtype).go()


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("P", [1, 15, 16, 17, 127, 128, 129, 255, 256, 257, 300, 640])
def test_prefixes_end_anywhere(P, page):
    Batch(P, 1, 4, 2, 128, BF, page, [5, 5, 5], [P] * 3, [[[0], [1], [page]]]).go()


@pytest.mark.parametrize("P", [1, 16, 127, 128, 129, 300])
def test_float32_prefixes_end_anywhere(P):
    Batch(P, 1, 4, 2, 128, F32, 32, [5, 5, 5], [P] * 3, [[[0], [1], [32]]]).go()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,G", [(2, 1), (2, 4), (3, 3), (9, 7), (16, 8), (13, 5), (43, 3), (18, 7), (19, 7), (37, 7), (11, 16),
                                 (33, 16)])
def test_rows_of_a_group(n, G, dtype):
    """From two query rows to more than two row tiles, tiles that end inside a sequence's heads."""
    Batch(n, 1, 2 * G, 2, 64, dtype, 16, [0] * n, [200] * n, np.random.default_rng(n).integers(0, 20, (1, n, 2)), out_dtype=F32).go()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_no_prefix_no_company_no_rows(dtype):
    """Groups of one, groups that share nothing, equal groups apart from each other, units without a row."""
    group = [4, 4, 7, 4, 9, 9, -3, -3]
    shared = [30, 30, 25, 18, 0, 0, 0, 0]
    mine = [[[0], [3], [0], [5], [0], [9], [0], [0]]]
    Batch(3, 1, 4, 1, 128, dtype, 16, group, shared, mine, append=False).go()
    Batch(4, 1, 4, 1, 128, dtype, 16, group, shared, mine).go()
    Batch(5, 1, 4, 1, 128, dtype, 16, [0, 1, 2], [0, 0, 0], 0).go()


@pytest.mark.parametrize("dtype,P,Ly,H", [(BF, 20011, 1, 1), (BF, 9000, 3, 2), (F32, 7001, 1, 1), (F32, 2000, 5, 3)])
def test_long_prefixes_are_cut_between_ctas(dtype, P, Ly, H):
    c = Batch(6, Ly, 4 * H, H, 128, dtype, 64, [0, 0, 0], [P] * 3, 17, garbage=False)
    c.go()
    out, lse = c.out.clone(), c.lse.clone()
    c.lens -= 1
    c.run()
    reco.reco_check()
    assert torch.equal(bits(out), bits(c.out)) and torch.equal(lse, c.lse)  # the same inputs, the same bits


def test_many_short_groups():
    """More items than CTAs, several layers."""
    rng = np.random.default_rng(7)
    n = 60
    group = np.repeat(np.arange(n // 2), 2).tolist()
    shared = np.repeat(rng.integers(0, 50, n // 2), 2).tolist()
    Batch(7, 3, 4, 2, 64, BF, 16, group, shared, rng.integers(0, 30, (3, n, 2))).go()
    Batch(8, 3, 4, 2, 64, F32, 16, group, shared, rng.integers(0, 30, (3, n, 2))).go()


@pytest.mark.parametrize("n,P,mine,Ly,page", [(24, 140, 20, 6, 64), (39, 0, 130, 3, 16), (12, 1000, 60, 4, 128), (3, 300, 1, 28, 16)])
def test_the_same_bits_again_and_again(n, P, mine, Ly, page):
    """Many short items one after the other in every CTA, whose roles then run far apart: nothing depends on when."""
    own = np.random.default_rng(n).integers(0, mine, (Ly, n, 2))
    c = Batch(n, Ly, 14, 2, 128, BF, page, np.repeat(np.arange(n // 3), 3).tolist(), [P] * n, own, out_dtype=F32, garbage=False).go()
    out, lse = c.out.clone(), c.lse.clone()
    for _ in range(150):
        c.lens -= 1
        c.run()
        assert torch.equal(bits(out), bits(c.out)) and torch.equal(lse, c.lse)
    reco.reco_check()


@pytest.mark.parametrize("n", [255, 256, 257, 1023, 1024, 1025, 2500])
def test_plans_of_many_sequences(n):
    rng = np.random.default_rng(n)
    group, shared = [], []
    while len(group) < n:
        k, p = int(rng.integers(1, 9)), int(rng.integers(0, 40))
        group += [len(group)] * k
        shared += [p] * k
    Batch(n, 1, 2, 1, 64, BF, 16, group[:n], shared[:n], rng.integers(0, 9, (1, n, 1))).go()


def test_one_group_over_many_sequences():
    n = 1500
    Batch(9, 1, 2, 1, 64, BF, 16, [0] * n, [100] * n, np.random.default_rng(9).integers(0, 4, (1, n, 1))).go()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0])
def test_scales(dtype, scale):
    c = Batch(10, 1, 6, 2, 64, dtype, 16, [0, 0, 0], [140] * 3, [[[0], [5], [40]]], out_dtype=F32)
    c.scale = scale
    c.go()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_nan_and_infinities_among_the_rows(dtype):
    """They reach the heads that see them, and no other: a row of the prefix all of the group, a query its head."""
    def batch():
        return Batch(11, 1, 4, 2, 64, dtype, 16, [0, 0, 1, 1], [140] * 4, [[[3], [5], [40], [0]]], out_dtype=F32)
    c = batch()
    c.K[0, int(c.table[0, 2]), 1, 3, 7] = float("nan")  # of the first group, KV head 1
    c.q[0, 3, 0, 5] = float("nan")
    ref, before = c.reference(), (c.K.clone(), c.V.clone())
    (_, rl, *_), *_ = ref
    assert np.isnan(rl[0, :2, 2:]).all() and np.isnan(rl[0, 3, 0]) and np.isnan(rl).sum() == 5
    c.run()
    reco.reco_check()
    c.check(ref, before, pool=False)
    c = batch()  # an infinite key: logits of +inf (NaN) or -inf (weight zero)
    c.q[:] = c.q.abs()
    c.K[0, int(c.table[0, 1]), 0, 2, 9] = float("-inf")
    c.V[0, int(c.table[2, 0]), 0, 2, 9] = float("inf")
    c.run()
    reco.reco_check()
    assert torch.isfinite(c.lse).all() and torch.isfinite(c.out[0, :2]).all()
    # an infinite value: infinity, or NaN where a probability enters in two bf16 parts (the second is of either sign or
    # zero: hi * inf + lo * inf), in its element alone
    bad = c.out[0, 2:, :2, 9]
    assert (torch.isinf(bad) if dtype == F32 else ~torch.isfinite(bad)).all() and torch.isfinite(c.out[0, 2:, :2, :9]).all()
    c = batch()
    c.q[:] = c.q.abs()
    c.K[0, int(c.table[0, 1]), 0, 2, 9] = float("inf")
    c.run()
    reco.reco_check()
    assert torch.isnan(c.lse[0, :2, :2]).all() and torch.isfinite(c.lse[0, 2:]).all() and torch.isfinite(c.lse[0, :, 2:]).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_logits_that_are_all_minus_infinity(dtype):
    c = Batch(12, 1, 2, 1, 64, dtype, 16, [0, 0], [130] * 2, [[[0], [4]]], append=False, out_dtype=F32, garbage=False)
    c.q[:] = c.q.abs()
    c.K[0, :, 0, :, 3] = float("-inf")
    c.run()
    reco.reco_check()
    assert torch.isneginf(c.lse).all() and (c.out == 0).all()


def test_logits_far_apart_between_the_parts():
    """One part's weights vanish beside the other's, and the maximum grows along the prefix."""
    for dtype in (BF, F32):
        for sign in (1.0, -1.0):
            c = Batch(13, 1, 2, 1, 64, dtype, 16, [0, 0], [700] * 2, [[[50], [4]]], out_dtype=F32, garbage=False)
            c.q[:] = sign * c.q.abs()
            for i in range(44):
                c.K[0, int(c.table[0, i]), 0] = (c.K[0, int(c.table[0, i]), 0].abs() * (0.2 * i)).to(dtype)
            c.scale = 0.5
            c.go()


# ---------------------------------------------------------------- errors
def failing(c, word, skip, wrong=None):
    """The call sets the error word and does every unit not in `skip` as the reference."""
    ref, before = c.reference(skip), (c.K.clone(), c.V.clone())
    if wrong is not None:
        wrong()
    c.run()
    with pytest.raises(reco.RecoError) as e:
        reco.reco_check()
    assert word in str(e.value), str(e.value)
    c.check(ref, before, pool=False)
    reco.reco_check()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_units_shorter_than_their_prefix(dtype):
    c = Batch(14, 2, 4, 2, 64, dtype, 16, [0, 0, 0, 1], [50] * 3 + [20], 5, out_dtype=F32)
    c.lens[1, 1, 0] = 49
    c.lens[0, 3, 1] = 19
    c.lens[0, 2, 0] = -5
    failing(c, "length-out-of-range", {(1, 1, 0), (0, 3, 1), (0, 2, 0)})


@pytest.mark.parametrize("dtype", [BF, F32])
def test_prefixes_that_cannot_be(dtype):
    group, shared = [0, 0, 1, 1, 2, 3, 3, 4], [30, 30, 40, 40, 10, 20, 20, 3]
    every = lambda *bs: {(ly, b, h) for ly in range(2) for b in bs for h in range(2)}  # noqa: E731
    for at, value, bad in ((1, 29, (1,)), (3, 0, (3,)), (4, -1, (4,)), (7, 2 ** 30, (7,))):
        c = Batch(15, 2, 4, 2, 64, dtype, 16, group, shared, 6, out_dtype=F32)

        def wrong():
            c.shared[at] = value
        failing(c, "length-out-of-range", every(*bad), wrong)
    # the first one's is what the others differ from: negative, it leaves them without a prefix of their own
    c = Batch(15, 2, 4, 2, 64, dtype, 16, group, shared, 6, out_dtype=F32)

    def first():
        c.shared[5] = -7
    failing(c, "length-out-of-range", every(5, 6), first)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("bad", [-1, 1 << 29])
def test_bad_pages(dtype, bad):
    every = lambda *bs: {(0, b, h) for b in bs for h in range(2)}  # noqa: E731
    for b, k, units in ((0, 1, every(0, 1, 2)), (3, 2, every(3, 4)), (1, 3, every(1)), (5, 0, every(5))):
        c = Batch(16, 1, 4, 2, 64, dtype, 16, [0, 0, 0, 1, 1, 2], [50, 50, 50, 40, 40, 20], 5, out_dtype=F32)

        def wrong():
            c.table[b, k] = bad
        failing(c, "page-out-of-range", units, wrong)


def test_no_room_to_append():
    c = Batch(17, 1, 4, 2, 64, BF, 16, [0, 0, 1], [20, 20, 9], 3, out_dtype=F32)
    c.lens[0, 1, 1] = c.table.shape[1] * 16
    failing(c, "no-room", {(0, 1, 1)})


# ---------------------------------------------------------------- as it is used
def test_lse_may_be_left_out():
    c = Batch(18, 1, 4, 2, 128, BF, 16, [0, 0], [100] * 2, 5)
    ref, before = c.reference(), (c.K.clone(), c.V.clone())
    c.run(lse=None)
    reco.reco_check()
    assert (c.lse == 7).all()
    c.lse[:] = torch.from_numpy(ref[0][1]).to(DEV)
    c.check(ref, before)


def test_one_workspace_serves_every_call():
    """Calls of other sizes, types and kinds in one buffer, one after the other."""
    big = Batch(19, 2, 14, 2, 128, BF, 16, [0] * 9, [400] * 9, 30)
    others = [Batch(20, 1, 4, 2, 64, F32, 32, [0, 0, 1], [90, 90, 5], 7), Batch(21, 2, 7, 1, 128, BF, 16, [0, 0], [333] * 2, 1)]
    lens = [c.lens.clone() for c in (big, *others)]
    for _ in range(3):
        for c, at in zip((big, *others), lens):
            c.lens.copy_(at)  # (there is room for one row)
            c.token()
            ref, before = c.reference(), (c.K.clone(), c.V.clone())
            c.run(ws=big.ws)
            reco.reco_check()
            c.check(ref, before)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_captured_and_replayed(dtype):
    """A graph serves every token: lengths, groups and prefixes are read on the device."""
    c = Batch(22, 2, 14, 2, 128, dtype, 16, [0] * 6, [300] * 6, 30, garbage=False)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    lens0 = c.lens.clone()
    c.table[1:, :18] = c.table[0, :18]  # every sequence names the pages, so that any grouping will do
    with torch.cuda.stream(side):
        c.run()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            c.run()
    torch.cuda.synchronize()
    for group, shared in (([0] * 6, [288] * 6), ([0, 0, 0, 1, 1, 1], [100] * 3 + [288] * 3), ([0, 1, 2, 3, 4, 5], [0] * 6),
                          ([0, 0, 1, 1, 2, 2], [16] * 2 + [0] * 2 + [200] * 2)):
        c.group = group
        c.groups.copy_(torch.tensor(group))
        c.shared.copy_(torch.tensor(shared))
        c.lens.copy_(lens0)
        c.q.copy_(c.rand(*c.q.shape))
        ref, before = c.reference(), (c.K.clone(), c.V.clone())
        g.replay()
        reco.reco_check()
        c.check(ref, before)


def test_two_calls_at_once():
    a, b = (Batch(s, 4, 28, 4, 128, BF, 16, [0] * 8, [2000] * 8, 100) for s in (23, 24))
    refs = a.reference(), b.reference()
    before = [(c.K.clone(), c.V.clone()) for c in (a, b)]
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for c, s in zip((a, b), streams):
        c.run(stream=s)
    torch.cuda.synchronize()
    reco.reco_check()
    for c, x, r in zip((a, b), before, refs):
        c.check(r, x)


@pytest.mark.parametrize("d,page", [(64, 16), (128, 64), (128, 256)])
def test_float32_output_of_groups_of_many_sizes(d, page):
    """Short pieces of few and of many query rows in turn, whose warps have rows in one and none in the next."""
    sizes, prefix = [1, 2, 33, 1, 40, 3, 26, 64], [0, 140, 129, 300, 260, 515, 31, 700]
    group = [g for g, n in enumerate(sizes) for _ in range(n)]
    shared = [p for n, p in zip(sizes, prefix) for _ in range(n)]
    mine = np.random.default_rng(5).integers(0, 200, (3, len(group), 2))
    b = Batch(34, 3, 8, 2, d, BF, page, group, shared, mine, out_dtype=F32)
    lens = b.lens.clone()
    b.go()
    out, lse = b.out.clone(), b.lse.clone()
    for _ in range(20):
        b.lens.copy_(lens)
        b.run()
        reco.reco_check()
        assert torch.equal(bits(b.out), bits(out)) and torch.equal(bits(b.lse), bits(lse))


@pytest.mark.parametrize("dtype,d,G,out_dtype", [(BF, 128, 5, BF), (BF, 64, 16, F32), (F32, 128, 7, F32), (F32, 64, 2, F32), (BF, 128, 1, F32)])
@pytest.mark.parametrize("append", [True, False])
def test_many_units_with_few_rows_of_their_own(dtype, d, G, out_dtype, append):
    """Units with none, one, 31 to 33 and 200 rows behind prefixes and without any, among units in error."""
    sizes, prefix = [1, 9, 1, 14, 2, 8], [0, 65, 0, 130, 33, 0]
    group = [g for g, n in enumerate(sizes) for _ in range(n)]
    shared = [p for n, p in zip(sizes, prefix) for _ in range(n)]
    mine = np.random.default_rng(6).choice([0, 1, 2, 17, 30, 31, 32, 33, 200], (10, len(group), 2))
    b = Batch(35, 10, 2 * G, 2, d, dtype, 16, group, shared, mine, append=append, out_dtype=out_dtype)
    b.go()
    if append:  # a page of own rows that is none: that sequence's units alone
        mine[:, 3] = 20
        b = Batch(36, 10, 2 * G, 2, d, dtype, 16, group, shared, mine, append=True, out_dtype=out_dtype)
        whole = Batch(36, 10, 2 * G, 2, d, dtype, 16, group, shared, mine, append=True, out_dtype=out_dtype)
        whole.go()
        b.table[3, 4] = -1  # rows 64 to 79 of the sequence, whose prefix ends at 65
        lens = b.lens.clone()
        b.run()
        with pytest.raises(reco.RecoError):
            reco.reco_check()
        keep = [i for i in range(len(group)) if i != 3]
        assert (b.out[:, 3] == 0).all() and torch.isneginf(b.lse[:, 3]).all() and torch.equal(b.lens[:, 3], lens[:, 3])
        assert torch.equal(bits(b.out[:, keep]), bits(whole.out[:, keep])) and torch.equal(b.lens[:, keep], whole.lens[:, keep])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_pools_beyond_32_bits(dtype):
    """The same rows at the far end of a pool of more than 2^32 bytes: the same bits."""
    b = Batch(31, 2, 8, 2, 64, dtype, 64, [0, 0, 0, 1], [300, 300, 300, 0],
              np.ones((2, 4, 2), int) * [[[5], [130], [0], [77]]])
    n_pages, far = b.K.shape[1], 2 ** 33 // (b.K[0, 0].numel() * b.K.element_size()) // 2
    K, V = (torch.full((2, far, *b.K.shape[2:]), float("nan"), device=DEV, dtype=dtype) for _ in range(2))
    K[:, far - n_pages:], V[:, far - n_pages:] = b.K, b.V
    table = torch.where((b.table >= 0) & (b.table < n_pages), b.table + (far - n_pages), -1)
    lens = b.lens.clone()
    b.go()
    out, lse = torch.empty_like(b.out), torch.empty_like(b.lse)
    kv = reco.make_paged_kv(K, V, table, 8)
    ws = reco.paged_workspace(reco.RECO_OP_PAGED_PREFIX, kv, DEV)
    reco.reco_paged_prefix_attn(kv, b.q, b.kn, b.vn, lens, b.groups, b.shared, b.scale, out, lse, ws)
    reco.reco_check()
    assert K.numel() * K.element_size() >= 2 ** 33 and torch.equal(bits(out), bits(b.out)) and torch.equal(bits(lse), bits(b.lse))
    assert torch.equal(lens, b.lens)
    for pool, small in ((K, b.K), (V, b.V)):
        assert torch.equal(bits(pool[:, far - n_pages:]), bits(small))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_pages_named_twice(dtype):
    """Rows may be read through one page in several places: in one prefix, in two groups, as a sequence's own."""
    b = Batch(32, 1, 12, 2, 128, dtype, 32, [0, 0, 1, 1, 2], [192, 192, 192, 192, 0],
              np.ones((1, 5, 2), int) * [[[40], [40], [40], [40], [230]]])
    b.table[0, 3] = b.table[0, 1]
    b.table[2, :6] = b.table[0, :6]
    b.table[4, 2] = b.table[0, 1]
    b.go()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_call_for_another_stream_waits_for_nothing_else(dtype):
    """Calls that follow each other on two streams, ordered by events alone, with a workspace each."""
    b = Batch(33, 2, 14, 2, 128, dtype, 16, [0] * 6, [700] * 6, 40)
    ref, before = b.reference(), (b.K.clone(), b.V.clone())
    lens, ws = b.lens.clone(), reco.paged_workspace(reco.RECO_OP_PAGED_PREFIX, b.kv, DEV)
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b.run(stream=s)
    first = b.out, b.lse
    t.wait_stream(s)
    with torch.cuda.stream(t):
        b.lens.copy_(lens)
        b.out, b.lse = torch.empty_like(b.out), torch.empty_like(b.lse)
        b.run(ws=ws)
    torch.cuda.synchronize()
    reco.reco_check()
    assert torch.equal(bits(first[0]), bits(b.out)) and torch.equal(bits(first[1]), bits(b.lse))
    b.check(ref, before)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_prompt_once_then_its_answers(dtype):
    """Append of a prompt, answers over it, token by token with rotation, eviction of the answers' own rows: against
    the same calls on private copies of the prompt (reco_paged_decode_attn), bit for bit where rows are moved and
    within the bounds of both where attention is computed."""
    Ly, n, Hq, H, d, page, P, room = 2, 3, 6, 2, 64, 16, 100, 64
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    rand = lambda *s: torch.randn(s, generator=g, device=DEV).to(dtype)  # noqa: E731
    per = (P + room) // page + 1
    new = lambda pages: [torch.zeros((Ly, pages, H, page, d), device=DEV, dtype=dtype) for _ in range(2)]  # noqa: E731
    whole = P // page
    (Ks, Vs), (Kc, Vc) = new(n * per), new(n * per)
    copies = torch.arange(n * per, dtype=torch.int32, device=DEV).view(n, per)
    table = copies.clone()
    table[1:, :whole] = table[0, :whole]
    one, many = reco.make_paged_kv(Ks, Vs, table[:1].contiguous(), Hq), reco.make_paged_kv(Ks, Vs, table, Hq)
    priv = reco.make_paged_kv(Kc, Vc, copies, Hq)
    f = torch.from_numpy((1e4 ** (-np.arange(0, d, 2) / d)).astype(np.float32)).to(DEV)
    ws = torch.zeros(max(reco.reco_paged_workspace_bytes(op, many) for op in (reco.RECO_OP_PAGED_PREFIX, reco.RECO_OP_PAGED_EVICT)),
                     dtype=torch.uint8, device=DEV)
    k, v = rand(Ly, P, H, d), rand(Ly, P, H, d)
    pos = torch.arange(P, dtype=torch.int32, device=DEV)
    lens1 = torch.zeros((Ly, 1, H), dtype=torch.int32, device=DEV)
    starts = torch.tensor([0, P], dtype=torch.int32, device=DEV)
    reco.reco_paged_append(one, k, v, starts, lens1, ws, pos=pos, inv_freq=f)
    lens = lens1.expand(Ly, n, H).contiguous()
    lens_c = torch.zeros_like(lens)
    reco.reco_paged_append(priv, k.repeat(1, n, 1, 1), v.repeat(1, n, 1, 1), torch.arange(0, n * P + 1, P, dtype=torch.int32, device=DEV),
                           lens_c, ws, pos=pos.repeat(n), inv_freq=f)
    assert torch.equal(lens, lens_c)
    group, shared = torch.zeros(n, dtype=torch.int32, device=DEV), torch.full((n,), P, dtype=torch.int32, device=DEV)
    starts = torch.arange(n + 1, dtype=torch.int32, device=DEV)
    outs = [[torch.empty((Ly, n, Hq, d), device=DEV) for _ in range(2)] for _ in range(2)]
    for t in range(40):
        qkv = rand(Ly, n, Hq + 2 * H, d)
        q, kt, vt = qkv.split([Hq, H, H], dim=2)
        at = torch.full((n,), P + t, dtype=torch.int32, device=DEV)
        q_rot = torch.empty((Ly, n, Hq, d), device=DEV, dtype=dtype)
        reco.reco_paged_append(many, kt, vt, starts, lens, ws, pos=at, inv_freq=f, q=q, q_out=q_rot)
        reco.reco_paged_prefix_attn(many, q_rot, None, None, lens, group, shared, d ** -0.5, outs[0][0], None, ws)
        reco.reco_paged_append(priv, kt, vt, starts, lens_c, ws, pos=at, inv_freq=f, q=q, q_out=q_rot)
        reco.reco_paged_decode_attn(priv, q_rot, None, None, lens_c, d ** -0.5, outs[1][0], None, ws)
        reco.reco_check()
        assert torch.equal(lens, lens_c)
        # rows: |q k| of some tens at most; parts of 2^-17 (the decode's) or float32 sums
        assert (outs[0][0] - outs[1][0]).abs().max() < (2 ** -14 if dtype == BF else 2 ** -17)
        if t == 30:  # the same cut of both: the prefix's rows stay (sinks), answers lose all but their latest 12 rows and 8 more
            wts = torch.rand((Ly, n, H, per * page), generator=g, device=DEV)
            budget = torch.full((n,), P + 20, dtype=torch.int32, device=DEV)
            # the shared form moves no row of a shared page: the kept rows below P are where they were
            own_first = table.clone()
            own_first[1:, :whole] = copies[1:, :whole]
            for b in range(1, n):
                for src, dst in zip(table[0, :whole].tolist(), own_first[b, :whole].tolist()):
                    Ks[:, dst], Vs[:, dst] = Ks[:, src], Vs[:, src]
                last = (table[0, whole].item(), table[b, whole].item())
                Ks[:, last[1], :, :P % page], Vs[:, last[1], :, :P % page] = Ks[:, last[0], :, :P % page], Vs[:, last[0], :, :P % page]
            cut = reco.make_paged_kv(Ks, Vs, own_first, Hq)
            reco.reco_paged_evict(cut, wts.clone(), lens, budget, 12, P, None, ws)
            reco.reco_paged_evict(priv, wts.clone(), lens_c, budget, 12, P, None, ws)
            reco.reco_check()
            assert torch.equal(lens, lens_c) and (lens == P + 20).all()
