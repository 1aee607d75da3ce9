"""Forms of the paged decode that the documentation allows beside the common ones: no lse, outputs of either type over
caches of either type, negative and zero scales, calls at once on streams of their own; the same bits as the common form."""
import numpy as np
import pytest
import torch

from paper_2608_04771_gb300 import reco
from test_gpu_paged import BF, DEV, F32, Cache, _lens, check, decode

pytestmark = pytest.mark.gpu

# one CTA, pieces joined by the last CTA, ranges laid end to end, whole units, float32 and bf16
CASES = [(1, 1, 7, 1, 128, BF, 5, 30), (1, 2, 14, 2, 128, BF, 2000, 3000), (1, 2, 12, 2, 64, F32, 500, 900),
         (10, 16, 24, 2, 64, BF, 300, 500), (10, 16, 10, 1, 128, F32, 300, 400), (10, 20, 4, 1, 64, BF, 0, 150),
         (10, 20, 16, 1, 64, F32, 0, 100)]


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2608_04771_gb300 import build
    build.build()
    reco.lib()


def _cache(i):
    Ly, B, Hq, H, d, dtype, lo, hi = CASES[i]
    return Cache(350 + i, Ly, B, Hq, H, d, dtype, 16, _lens(350 + i, Ly, B, H, lo, hi, 16))


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_no_lse_and_either_output_type(i, weights):
    want = _cache(i)
    q, kn, vn = want.token()
    out, _ = decode(want, q, kn, vn, weights=weights)
    for out_dtype in (torch.float32, torch.bfloat16):
        c = _cache(i)
        got = torch.full_like(out, 7.0, dtype=out_dtype)
        if weights:
            ws = c.workspace(reco.RECO_OP_PAGED_WEIGHTS)
            reco.reco_paged_decode_attn_weights(c.kv, q, kn, vn, c.lens, c.scale, got, None, c.weights, ws)
        else:
            ws = c.workspace(reco.RECO_OP_PAGED_DECODE)
            reco.reco_paged_decode_attn(c.kv, q, kn, vn, c.lens, c.scale, got, None, ws)
        reco.reco_check()
        assert torch.equal(got, out.to(out_dtype)) and torch.equal(c.lens, want.lens)
        assert torch.equal(c.weights, want.weights)
        assert torch.equal(c.K.nan_to_num(), want.K.nan_to_num()) and torch.equal(c.V.nan_to_num(), want.V.nan_to_num())


@pytest.mark.parametrize("scale", [-0.3, 0.0])
@pytest.mark.parametrize("i", [1, 2, 3, 6])
def test_scales_that_are_not_positive(i, scale):
    c = _cache(i)
    q, kn, vn = c.token()
    c.scale = scale
    if scale < 0:  # (the reference's bounds take the scale's size)
        c2 = _cache(i)
        c2.scale = -scale
        out, lse = decode(c, q, kn, vn)
        reco.reco_check()
        o2, l2 = check(c2, -q, kn, vn)
        assert torch.equal(out, o2) and torch.equal(lse, l2) and torch.equal(c.weights, c2.weights)
    else:
        lens = c.lens.clone()
        _, lse = check(c, q, kn, vn)
        n = (lens + 1).repeat_interleave(c.shape[2] // c.shape[3], 2).double()
        # every logit is 0: the sum is n, its logarithm rounded twice and scaled by ln 2
        assert ((lse.double() - n.log()).abs() <= 2.0 ** -20 + 2.0 ** -21 * n.log()).all()


def test_eager_calls_at_once_on_streams_of_their_own():
    want, got = [], []
    for i in (1, 3, 4):
        c = _cache(i)
        t = c.token()
        want.append((*decode(c, *t), c.weights, c.lens))
    streams = [torch.cuda.Stream() for _ in range(3)]
    made = []
    for i in (1, 3, 4):
        c = _cache(i)
        made.append((c, c.token(), c.outputs(torch.float32), c.workspace(reco.RECO_OP_PAGED_WEIGHTS)))
    torch.cuda.synchronize()
    for (c, (q, kn, vn), (out, lse), ws), st in zip(made, streams):
        reco.reco_paged_decode_attn_weights(c.kv, q, kn, vn, c.lens, c.scale, out, lse, c.weights, ws, stream=st)
    torch.cuda.synchronize()
    reco.reco_check()
    for (c, _, (out, lse), _), w in zip(made, want):
        assert all(torch.equal(a, b) for a, b in zip((out, lse, c.weights, c.lens), w))
    assert np.isfinite(float(want[0][0].sum()))
