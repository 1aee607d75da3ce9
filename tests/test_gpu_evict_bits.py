"""Weights that an eviction moves keep their bits, whichever selection moves them: -0 (which ranks as +0 does), NaN of
either sign and any payload (all above everything), infinities and subnormals among the others; in candidates, in the
latest rows and in the sinks.  And the rows kept are those of the order documented, ties to the lower index."""
import numpy as np
import pytest
import torch

from paper_2608_04771_gb300 import reco

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2608_04771_gb300 import build
    build.build()
    reco.lib()


# units (layers, B, heads), rows of the shortest and the longest unit, w, sinks
PATHS = {
    "a warp, 256 candidates": ((1, 3, 2), 60, 240, 5, 3),
    "a warp, 512 candidates": ((20, 20, 2), 100, 480, 8, 1),
    "a warp, 1024 candidates": ((28, 10, 5), 200, 1000, 0, 0),
    "512 threads, few keys each": ((1, 2, 1), 300, 1500, 32, 4),
    "1024 threads, few keys each": ((1, 2, 2), 2100, 5000, 32, 4),
    "256 threads, few keys each": ((14, 10, 5), 300, 1800, 7, 2),
    "512 threads": ((4, 10, 5), 500, 6000, 32, 4),
    "256 threads": ((14, 10, 5), 500, 4000, 32, 0),
    "1024 threads": ((4, 10, 5), 9000, 17000, 16, 16),
    "a cluster": ((1, 3, 1), 9000, 60000, 100, 4),
    "from global memory": ((2, 8, 5), 2000, 60000, 2000, 17),
}


def _weights(g, shape):
    x = torch.rand(shape, generator=g, device=DEV) * 4.0 - 1.0
    x = torch.where(torch.rand(shape, generator=g, device=DEV) < 0.3, (x * 4).round() / 4, x).contiguous()  # ties
    bits = x.view(torch.int32)
    kinds = [0x80000000, 0, 0x7fc00000, 0x7f800001, 0xffc12345, 0xffffffff, 0x7f800000, 0xff800000, 0x80000001, 1]
    kinds = torch.from_numpy(np.array(kinds, np.uint32).view(np.int32)).to(DEV)
    pick = torch.randint(0, 14 * len(kinds), shape, generator=g, device=DEV)
    return torch.where(pick < len(kinds), kinds[pick.clamp(max=len(kinds) - 1)], bits).view(torch.float32).contiguous()


def _rank(weights):
    """A whole number per weight, in the order documented: NaN above everything, -0 as +0."""
    bits = (weights + 0.0).view(torch.int32).long()
    return torch.where(torch.isnan(weights), 2 ** 40, torch.where(bits < 0, -(bits & 0x7fffffff), bits))


@pytest.mark.parametrize("plain", [False, True])
@pytest.mark.parametrize("path", list(PATHS))
def test_weights_keep_their_bits(path, plain):
    (Ly, B, H), lo, hi, w, sinks = PATHS[path]
    g = torch.Generator(device=DEV)
    g.manual_seed(40 + len(path))
    rng = np.random.default_rng(40 + len(path))
    page, d = 16, 64
    per = -(-hi // page)
    table = torch.from_numpy(rng.permutation(B * per).astype(np.int32).reshape(B, per)).to(DEV)
    K = torch.randn((Ly, B * per, H, page, d), generator=g, device=DEV, dtype=torch.bfloat16)
    V = K.neg()
    kv = reco.make_paged_kv(K, V, table, H)
    lens0 = rng.integers(lo, hi + 1, (Ly, B, H)).astype(np.int32)
    lens = torch.from_numpy(lens0).to(DEV)
    budget = rng.integers(max(w + sinks, lo // 4), hi, B).astype(np.int32)
    budget[0] = w + sinks + 3  # fewer than there are NaNs
    weights = _weights(g, (Ly, B, H, per * page))
    if plain:  # nothing odd among the candidates: the keys stand for the weights
        weights = torch.where(torch.isnan(weights) | (weights == 0), 0.5, weights).contiguous()
    before = weights.clone()
    kept = torch.full((Ly, B, H, per * page), -7, dtype=torch.int32, device=DEV)
    reco.reco_paged_evict(kv, weights, lens, torch.from_numpy(budget).to(DEV), w, sinks, kept,
                          reco.paged_workspace(reco.RECO_OP_PAGED_EVICT, kv, DEV))
    reco.reco_check()
    L = torch.from_numpy(lens0).to(DEV).long().unsqueeze(-1)
    m = torch.from_numpy(budget).to(DEV).long().view(1, B, 1, 1).expand(L.shape)
    j = torch.arange(per * page, device=DEV)
    cut = L > m
    fixed = (j < sinks) | ((j >= L - w) & (j < L))
    rank = torch.where(fixed, 2 ** 41, torch.where(j < L, _rank(before), -2 ** 41))
    place = torch.empty_like(rank).scatter_(-1, torch.sort(-rank, dim=-1, stable=True).indices, j.expand(rank.shape).contiguous())
    source = torch.sort(torch.where(place < m, j, 2 ** 30), dim=-1).values
    moved = cut & (j < m)
    assert cut.any() and torch.equal(lens, torch.where(cut, m, L).squeeze(-1).int())
    assert torch.equal(kept, torch.where(moved, source, -7).int())
    source = torch.where(moved, source, j)
    assert torch.equal(weights.view(torch.int32), before.view(torch.int32).gather(-1, source))
