"""The append to a paged cache on the GPU against the fp64 reference (oracle/paged.py).

Bounds (u = 2^-24).  The angle is exact to 2^-32 turns, less than u, before it is rounded to float32
half turns in [-1, 1]: u of up to pi.  sincospif is good to 2 units in the last place, 4 u; its
products with x and y and their sum are rounded three times.  A rotated element is therefore within
(pi + 4 + 3) u, here 11 u, of |x| + |y|, and half a step of the cache's type of itself.  What does not
turn is moved bit for bit.
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


def bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)


class Call:
    """A cache whose rows are NaN but for the first `have` of each unit, and new tokens as views into one tensor."""

    def __init__(self, seed, Ly, B, Hq, H, d, dtype, page, have, new, rot=None, interleaved=False, pad=2, far=0, with_q=True):
        rng = np.random.default_rng(seed)
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.rand = lambda *s: torch.randn(s, generator=g, device=DEV).to(dtype)
        rot = d if rot is None else rot
        self.dims, self.dtype, self.interleaved = (Ly, B, Hq, H, d, page), dtype, interleaved
        have = np.broadcast_to(np.asarray(have, np.int32), (Ly, B, H)).copy()
        new = np.broadcast_to(np.asarray(new, np.int32), (B,))
        per = (int(have.max()) + int(new.max()) + page - 1) // page + 1
        need = [-(-(int(have[:, b].max()) + int(new[b])) // page) for b in range(B)]
        ids = rng.permutation(sum(need) + 2)
        table, at = np.full((B, per), -7, np.int32), 0
        for b in range(B):
            table[b, :need[b]] = ids[at:at + need[b]]
            at += need[b]
        shape = (Ly, sum(need) + 2, H, page, d)
        self.K, self.V = (torch.full(shape, float("nan"), device=DEV, dtype=dtype) for _ in range(2))
        self.table = torch.from_numpy(table).to(DEV)
        starts = np.concatenate([[1], 1 + np.cumsum(new)]).astype(np.int32)  # token 0 and the last `pad` are nobody's
        T = int(starts[-1]) + pad
        self.qkv = self.rand(Ly, T, Hq + 2 * H, d)
        self.q, self.k, self.v = self.qkv.split([Hq, H, H], dim=2)
        self.q_out = self.rand(Ly, T, Hq, d) if with_q else None
        if not with_q:
            self.q = None
        pos = rng.integers(0, 5000, T).astype(np.int32) + far
        self.pos, self.starts = torch.from_numpy(pos).to(DEV), torch.from_numpy(starts).to(DEV)
        f = (1e4 ** (-np.arange(0, rot, 2) / max(rot, 1))).astype(np.float32)
        self.inv_freq = torch.from_numpy(f).to(DEV) if rot else None
        self.lens = torch.from_numpy(have).to(DEV)
        self.kv = reco.make_paged_kv(self.K, self.V, self.table, Hq)
        self.ws = reco.paged_workspace(reco.RECO_OP_PAGED_APPEND, self.kv, DEV)

    def run(self, **kw):
        a = dict(pos=self.pos, inv_freq=self.inv_freq, q=self.q, q_out=self.q_out, interleaved=self.interleaved)
        a.update(kw)
        reco.reco_paged_append(self.kv, self.k, self.v, self.starts, self.lens, self.ws, **a)

    def reference(self):
        n = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
        K, V, lens, qo = n(self.K), n(self.V), self.lens.cpu().numpy().copy(), n(self.q_out)
        f = () if self.inv_freq is None else n(self.inv_freq)
        args = (self.table.cpu().numpy(), lens, n(self.k), n(self.v), self.starts.tolist(), self.pos.cpu().numpy(), f,
                self.interleaved)
        paged.append(K, V, *args, n(self.q), qo)
        # |x| + |y| of what turns, by the same way
        size = lambda x: paged.rotate(np.abs(x), 0, f, self.interleaved)  # noqa: E731

        def spread(x):
            x = np.abs(n(x))
            y = x.copy()
            h = len(f)
            lo, hi = (slice(0, 2 * h, 2), slice(1, 2 * h, 2)) if self.interleaved else (slice(0, h), slice(h, 2 * h))
            y[..., lo] = y[..., hi] = x[..., lo] + x[..., hi]
            y[..., 2 * h:] = 0.0
            return y
        big = np.zeros_like(K)
        paged.append(big, np.zeros_like(K), args[0], self.lens.cpu().numpy().copy(), spread(self.k), n(self.v), args[4])
        qbig = None if qo is None else spread(self.q)
        return K, V, lens, qo, big, qbig

    def check(self, before, ref):
        K0, V0, q0 = before
        K, V, lens, qo, big, qbig = ref
        half = 2.0 ** -8 if self.dtype == torch.bfloat16 else U

        def close(got, want, size, old):
            got64, was = got.double().cpu().numpy(), torch.from_numpy(np.isnan(want)).to(DEV)
            assert torch.equal(bits(got)[was], bits(old)[was])  # not written
            ok = ~np.isnan(want)
            off = np.abs(got64 - want)[ok]
            tol = (11 * U * size * (1 + half) + half * np.abs(want))[ok]
            assert (off <= tol).all(), (off / np.maximum(tol, 1e-300)).max()
        close(self.K, K, big, K0)
        assert torch.equal(bits(self.V), torch.where(torch.isnan(torch.from_numpy(V).to(DEV)), bits(V0),
                                                     bits(torch.from_numpy(V).to(DEV).to(self.dtype))))
        assert np.array_equal(self.lens.cpu().numpy(), lens)
        if qo is not None:
            there = np.zeros(qo.shape[1], bool)
            there[self.starts[0].item():self.starts[-1].item()] = True
            out = self.q_out.clone()
            assert torch.equal(bits(out[:, ~torch.from_numpy(there).to(DEV)]), bits(q0[:, ~torch.from_numpy(there).to(DEV)]))
            off = np.abs(out.double().cpu().numpy() - qo)[:, there]
            tol = (11 * U * qbig * (1 + half) + half * np.abs(qo))[:, there]
            assert (off <= tol).all(), (off / np.maximum(tol, 1e-300)).max()

    def go(self, **kw):
        ref = self.reference()
        before = self.K.clone(), self.V.clone(), None if self.q_out is None else self.q_out.clone()
        self.run(**kw)
        reco.reco_check()
        self.check(before, ref)


BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("rot", [0, 16, 48, 64])
def test_types_dims_and_partial_rotations(dtype, d, rot, interleaved):
    Call(1, 2, 3, 6, 2, d, dtype, 16, [[[0, 15], [16, 7], [31, 1]]] * 2, [1, 17, 0], rot, interleaved).go()


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_pages(page):
    Call(2, 1, 4, 5, 1, 128, BF, page, [[[page - 1], [page], [0], [2 * page + 3]]], [2, page, page + 1, 3 * page]).go()


@pytest.mark.parametrize("G", [1, 3, 7, 16])
def test_query_heads(G):
    Call(3, 1, 2, 3 * G, 3, 128, BF, 32, 40, [5, 1]).go()


@pytest.mark.parametrize("B", [1, 2, 31, 32, 33, 70, 1100])
def test_tokens_find_their_sequence(B):
    new = np.random.default_rng(B).integers(0, 4, B)
    new[-1] = 1
    Call(4, 1, B, 2, 1, 64, F32, 16, 3, new).go()


def test_one_token_of_one_sequence():
    Call(5, 1, 1, 8, 2, 64, F32, 16, 512, 1, pad=0).go()


def test_many_layers_share_counters():
    """More layers than counters: groups of layers whose lengths the same CTA advances."""
    Call(6, 1030, 1, 1, 1, 64, BF, 16, 1, 2, rot=16).go()


def test_far_and_negative_positions():
    c = Call(7, 1, 2, 2, 2, 128, F32, 16, 0, [40, 9])
    # (the reference's own product is off by 2^-53 of 2^26 radians here, 2^-27)
    c.pos[:] = torch.from_numpy(np.random.default_rng(1).integers(-2 ** 26, 2 ** 26, len(c.pos))).to(DEV)
    c.go()


def test_without_queries_and_without_rotation():
    Call(8, 2, 2, 4, 2, 128, BF, 16, 5, [3, 20], with_q=False).go()
    Call(8, 2, 2, 4, 2, 128, BF, 16, 5, [3, 20], rot=0, with_q=False).go(pos=None)


def test_queries_in_place_and_odd_strides():
    c = Call(9, 2, 2, 6, 2, 128, BF, 16, 5, [3, 20])
    ref, before = c.reference(), (c.K.clone(), c.V.clone(), c.qkv[:, :, :6].clone())
    # keys as [T, layers, heads, d], values with a repeated head dimension of stride zero
    kt = c.k.permute(1, 0, 2, 3).contiguous().permute(1, 0, 2, 3)
    c.k, c.q_out = kt, c.q
    c.run()
    reco.reco_check()
    c.check(before, ref)
    c = Call(10, 1, 2, 6, 2, 128, F32, 16, 5, [3, 20])
    c.v = c.v[:, :, :1].expand(-1, -1, 2, -1)
    c.k = c.k.flip(1).contiguous().flip(1)
    c.go()


def test_frequencies_that_are_not_finite_make_nan():
    c = Call(11, 1, 1, 2, 1, 64, F32, 16, 0, [4])
    c.inv_freq[3] = float("inf")
    c.inv_freq[5] = float("nan")
    c.run()
    reco.reco_check()
    got = torch.isnan(c.q_out[0, 1:5]).cpu().numpy()
    want = np.zeros(64, bool)
    want[[3, 5, 35, 37]] = True
    assert (got == want).all()


def test_nan_and_infinities_stay_in_their_pair():
    c = Call(12, 1, 1, 1, 1, 64, F32, 16, 0, [2])
    c.qkv[0, 1, 1, 4] = float("nan")
    c.qkv[0, 2, 2, 9] = float("inf")
    c.run()
    k = c.K[0, c.table[0, 0].long(), 0]
    assert torch.isnan(k[0]).nonzero().flatten().tolist() == [4, 36]
    assert torch.isinf(c.V[0, c.table[0, 0].long(), 0, 1]).nonzero().flatten().tolist() == [9]


def state(c):
    return [t.clone() for t in (c.K, c.V, c.q_out, c.lens)]


def test_no_room_and_bad_lengths_leave_units_as_they_are():
    have = np.full((1, 4, 2), 5, np.int32)
    c = Call(13, 1, 4, 4, 2, 128, BF, 16, have, [3, 2, 4, 0])
    cap = c.table.shape[1] * 16
    c.lens[0, 0, 1] = cap - 2
    c.lens[0, 1, 0] = -1
    c.lens[0, 2, 1] = cap + 1
    c.lens[0, 3, 0] = -9  # no tokens: not looked at
    K0, V0, _, lens0 = state(c)
    ok = c.lens.clone()
    c.run()
    with pytest.raises(reco.RecoError) as e:
        reco.reco_check()
    assert "length-out-of-range" in str(e.value) and "no-room" in str(e.value)
    want = lens0.clone()
    want[0, 0, 0] += 3
    want[0, 1, 1] += 2
    want[0, 2, 0] += 4
    assert torch.equal(c.lens, want)
    # written: only the new rows of the units that are in order
    for b, h in ((0, 0), (1, 1), (2, 0)):
        rows = range(int(ok[0, b, h]), int(want[0, b, h]))
        for i, r in enumerate(rows):
            at = (0, int(c.table[b, r // 16]), h, r % 16)
            assert torch.equal(c.V[at], c.v[0, int(c.starts[b]) + i, h])
            K0[at], V0[at] = c.K[at], c.V[at]
    assert torch.equal(bits(c.K), bits(K0)) and torch.equal(bits(c.V), bits(V0))


@pytest.mark.parametrize("bad", [-1, 1 << 30])
def test_bad_pages_keep_the_length(bad):
    c = Call(14, 2, 2, 4, 2, 64, F32, 16, [[[5, 20], [9, 3]]] * 2, [14, 3])
    c.table[0, 1] = bad  # rows 16 to 31: unit (., 0, 0) ends in them, (., 0, 1) starts in them
    want = c.lens.clone()
    want[:, 1] += 3
    K0 = c.K.clone()
    c.run()
    with pytest.raises(reco.RecoError) as e:
        reco.reco_check()
    assert "page-out-of-range" in str(e.value)
    assert torch.equal(c.lens, want)
    mine = torch.zeros(c.K.shape[1], dtype=torch.bool, device=DEV)
    for b in range(2):
        pages = c.table[b][(c.table[b] >= 0) & (c.table[b] < c.K.shape[1])].long()
        mine[pages] = True
    assert torch.equal(bits(c.K[:, ~mine]), bits(K0[:, ~mine]))
    c.table[0, 1] = int((~mine).nonzero()[0])  # the next call finds its counters as it left them
    c.lens[:] = want
    c.go()


@pytest.mark.parametrize("starts", [[5, 3, 9], [-1, 3, 9], [0, 3, 100], [9, 3, 0]])
def test_bad_starts_advance_nothing(starts):
    c = Call(15, 1, 2, 4, 2, 64, F32, 16, 3, [5, 6], pad=0)
    lens0 = c.lens.clone()
    good = c.starts.clone()
    c.starts[:] = torch.tensor(starts)
    c.run()
    with pytest.raises(reco.RecoError) as e:
        reco.reco_check()
    assert "length-out-of-range" in str(e.value) and torch.equal(c.lens, lens0)
    c.starts[:] = good
    c.K[:] = float("nan")
    c.V[:] = float("nan")
    c.go()


def test_empty_calls():
    c = Call(16, 1, 2, 4, 2, 64, F32, 16, 3, [0, 0])
    c.go()
    c = Call(16, 1, 2, 4, 2, 64, F32, 16, 3, [0, 0])
    reco.reco_paged_append(c.kv, c.k[:, :0], c.v[:, :0], c.starts, c.lens, c.ws)
    reco.reco_check()


def test_captured_and_replayed_with_other_lengths():
    """A graph serves every token: lengths, positions and whose tokens they are are read on the device."""
    c = Call(17, 2, 3, 4, 2, 128, BF, 16, 7, [4, 4, 4])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.run()  # first call outside the capture
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            c.run()
    torch.cuda.synchronize()
    for n in ([1, 2, 3], [0, 0, 12], [4, 4, 4]):
        c.starts[:] = torch.from_numpy(np.concatenate([[1], 1 + np.cumsum(n)]).astype(np.int32))
        c.lens[:] = torch.randint(0, 5, c.lens.shape, device=DEV)
        c.pos += 11
        c.qkv[:] = c.rand(*c.qkv.shape)
        c.K[:] = float("nan")
        c.V[:] = float("nan")
        c.q_out[:] = c.rand(*c.q_out.shape)
        if max(n) > 4:
            c.lens[:, 2] = 0
        ref, before = c.reference(), (c.K.clone(), c.V.clone(), c.q_out.clone())
        g.replay()
        reco.reco_check()
        c.check(before, ref)


def test_two_calls_at_once_with_a_workspace_each():
    a, b = Call(18, 1, 8, 28, 4, 128, BF, 16, 30, 50), Call(19, 1, 8, 28, 4, 128, BF, 16, 30, 50)
    refs = a.reference(), b.reference()
    before = [(c.K.clone(), c.V.clone(), c.q_out.clone()) for c in (a, b)]
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for c, s in zip((a, b), streams):
        c.run(stream=s)
    torch.cuda.synchronize()
    reco.reco_check()
    for c, x, r in zip((a, b), before, refs):
        c.check(x, r)


def test_pool_offsets_beyond_32_bits():
    """Rows behind the first 2^32 bytes of a pool, and new tokens behind 2^31 elements of their tensor."""
    H, d, page = 8, 128, 256
    n_pages = 9000  # 4.7 GB each
    K = torch.zeros((1, n_pages, H, page, d), dtype=BF, device=DEV)
    V = torch.zeros_like(K)
    table = torch.tensor([[n_pages - 1]], dtype=torch.int32, device=DEV)
    kv = reco.make_paged_kv(K, V, table, H)
    wide = torch.zeros((1, 2, 1 << 24, d), dtype=BF, device=DEV)  # token stride of 2^31 elements
    k = wide[:, :, -H:]
    k.copy_(torch.randn(1, 2, H, d, device=DEV))
    lens = torch.full((1, 1, H), 3, dtype=torch.int32, device=DEV)
    starts = torch.tensor([0, 2], dtype=torch.int32, device=DEV)
    reco.reco_paged_append(kv, k, k, starts, lens, reco.paged_workspace(reco.RECO_OP_PAGED_APPEND, kv))
    reco.reco_check()
    for t in range(2):
        assert torch.equal(K[0, -1, :, 3 + t], k[0, t]) and torch.equal(V[0, -1, :, 3 + t], k[0, t])
    assert int(K.count_nonzero()) <= 2 * H * d and int(K[0, :-1].count_nonzero()) == 0
