"""How exact decode attention over shared prefixes is with bf16 output, against 64 bits: as reco_paged_decode_attn, its
probabilities enter the product with V in two bf16 parts (2^-17 of each), not rounded to bf16 (2^-8 of each).

The bounds are test_gpu_prefix.py's with 2^-17 for the parts.  Small queries keep the logits' share of them below that of the parts
(big of some tenths: 2 (d + 6) u big is 2^-17), and rows of either sign leave outputs far smaller than their terms, so that the output's
own rounding, 2^-8 of it, hides nothing.
"""
import numpy as np
import pytest
import torch

from paper_2608_04771_gb300 import reco
from test_gpu_prefix import BF, U, Batch, _lib, np64  # noqa: F401

pytestmark = pytest.mark.gpu


def tight(c, ref):
    """Whether outputs are within the bounds of two bf16 parts."""
    (ro, rl, big, seen, absv), *_ = ref
    prob = 2 * ((c.dims[4] + 6) * U * big) + 2.0 ** -21 + 4 * U * np.where(np.isfinite(rl), np.abs(rl), 0.0)
    chain = (192 + 32 + seen / 8) * U
    tol = (prob + chain + 2.0 ** -17)[..., None] * absv * (1 + 2.0 ** -8) + np.abs(ro) * 2.0 ** -8
    off = np.abs(np64(c.out) - ro)
    assert (off <= tol).all(), (off / (tol + 1e-300)).max()


@pytest.mark.parametrize("d,G,n,P", [(128, 7, 3, 300), (128, 4, 40, 700), (64, 3, 2, 129), (64, 16, 9, 1000), (128, 1, 150, 260)])
def test_probabilities_keep_seventeen_bits(d, G, n, P):
    """One row tile of one half and of two, and several."""
    c = Batch(70 + G, 1, 2 * G, 2, d, BF, 32, [0] * n, [P] * n, np.random.default_rng(G).integers(0, 300, (1, n, 2)))
    c.q.mul_(2.0 ** -5)
    ref = c.reference()
    c.run()
    reco.reco_check()
    tight(c, ref)


def test_as_the_decode_that_reads_every_row_by_itself():
    """The same rows through reco_paged_decode_attn: both round the same value once, and differ where it falls between two."""
    c = Batch(78, 2, 14, 2, 128, BF, 16, [0] * 5, [320] * 5, 100)
    c.table[1:, :20] = c.table[0, :20]
    lens, out = c.lens.clone(), torch.empty_like(c.out)
    lse = torch.empty_like(c.lse)
    c.run()
    ws = reco.paged_workspace(reco.RECO_OP_PAGED_DECODE, c.kv, "cuda")
    reco.reco_paged_decode_attn(c.kv, c.q, c.kn, c.vn, lens, c.scale, out, lse, ws)
    reco.reco_check()
    # An error of e of an output's size moves its rounding with a probability of e over the spacing (2^-8 to 2^-7 of it, finer for
    # outputs near zero).  Errors in the probabilities are independent, and so is their share of a sum of terms of either sign: two
    # parts' 2^-18 of it and float32 sums make less than 1%, one part's 2^-9.8 more than 16%.
    assert (out != c.out).double().mean() < 0.08
