"""One workspace for paged calls of every kind and size: batches that grow and shrink, other heads, types
and head dimensions, calls with and without weights, evictions between them.  What a call leaves behind in
it must not count in the next."""
import numpy as np
import pytest
import torch

from paper_2608_04771_gb300 import reco
from test_gpu_paged import BF, DEV, F32, Cache, _check_evict, _lens, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2608_04771_gb300 import build
    build.build()
    reco.lib()


def _caches():
    """Few units cut into a piece per CTA; more units than CTAs, laid end to end and cut where the ranges end, many
    of them and fewer; other heads, types and pages; short units that are not cut."""
    return [Cache(60, 1, 2, 28, 4, 128, BF, 16, _lens(60, 1, 2, 4, 2000, 2600, 16), room=9),
            Cache(61, 7, 32, 28, 4, 128, BF, 16, _lens(61, 7, 32, 4, 280, 500, 16), room=9),
            Cache(62, 7, 16, 28, 4, 128, BF, 16, _lens(62, 7, 16, 4, 280, 500, 16), room=9),
            Cache(63, 1, 4, 6, 2, 64, F32, 32, _lens(63, 1, 4, 2, 700, 900, 32), room=9),
            Cache(64, 10, 20, 16, 1, 64, BF, 64, _lens(64, 10, 20, 1, 270, 400, 64), room=9),
            Cache(65, 10, 20, 2, 2, 128, BF, 16, _lens(65, 10, 20, 2, 0, 200, 16), room=9)]


ORDER = [0, 1, 0, 2, 1, 3, 1, 4, 2, 5, 1, 4, 0]


@pytest.mark.parametrize("weights", [False, True])
def test_growing_and_shrinking_batches_share_a_workspace(weights):
    caches = _caches()
    op = reco.RECO_OP_PAGED_WEIGHTS if weights else reco.RECO_OP_PAGED_DECODE
    ws = torch.zeros(max(reco.reco_paged_workspace_bytes(op, c.kv) for c in caches), dtype=torch.uint8, device=DEV)
    for i in ORDER:
        check(caches[i], *caches[i].token(), weights=weights, ws=ws, exact_pool=False)


def test_every_paged_call_shares_a_workspace_zero_in_its_first_bytes():
    """Decode with and without weights and evictions in turn, through a buffer that is no more than its first
    8192 bytes zero."""
    caches = _caches()
    ops = (reco.RECO_OP_PAGED_DECODE, reco.RECO_OP_PAGED_WEIGHTS, reco.RECO_OP_PAGED_EVICT)
    ws = torch.full((max(reco.reco_paged_workspace_bytes(op, c.kv) for c in caches for op in ops),), 0xA5,
                    dtype=torch.uint8, device=DEV)
    ws[:8192] = 0
    for step, i in enumerate(ORDER):
        c = caches[i]
        check(c, *c.token(), weights=step % 2 == 0, ws=ws, exact_pool=False)
        if step % 3 == 0:
            most = int(c.lens.max())
            c.workspace = lambda op: ws  # noqa: E731
            _check_evict(c, [most - 3 if b % 2 else 10 ** 6 for b in range(c.shape[1])], 16, 4, with_kept=False)
    assert not ws[:8].any()


def test_a_workspace_from_the_binding_is_zero_where_it_must_be():
    c = Cache(66, 1, 1, 2, 1, 64, BF, 16, 20)
    for op in (reco.RECO_OP_PAGED_DECODE, reco.RECO_OP_PAGED_WEIGHTS, reco.RECO_OP_PAGED_EVICT):
        ws = reco.paged_workspace(op, c.kv, DEV)
        assert ws.numel() >= reco.reco_paged_workspace_bytes(op, c.kv) >= 8192 and not ws[:8192].any()
    assert np.isfinite(float(c.scale))
