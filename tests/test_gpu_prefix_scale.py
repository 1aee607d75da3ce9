"""Scales of next to nothing and keys to match, in decode attention over shared prefixes: a logit is the product of the two, whatever
the size of either.

Bounds: test_gpu_prefix.py's.
"""
import pytest
import torch

from paper_2608_04771_gb300 import reco
from test_gpu_prefix import BF, F32, Batch, _lib  # noqa: F401

pytestmark = pytest.mark.gpu
FORMS = [(BF, BF), (BF, F32), (F32, F32)]


def batch(dtype, out_dtype, n, G, scale, size):
    c = Batch(81, 1, 2 * G, 2, 64, dtype, 16, [0] * n + [1] * 2, [300] * n + [40] * 2, 50, out_dtype=out_dtype)
    c.K.mul_(size)
    c.kn.mul_(size)
    c.scale = scale
    return c


@pytest.mark.parametrize("dtype,out_dtype", FORMS)
@pytest.mark.parametrize("n,G", [(3, 2), (40, 4)])
@pytest.mark.parametrize("scale,size", [(1e-32, 2.0 ** 103), (-1e-35, 2.0 ** 113), (1e30, 2.0 ** -103), (0.0, 2.0 ** 110), (-0.0, 1.0)])
def test_scales_of_any_size(dtype, out_dtype, n, G, scale, size):
    batch(dtype, out_dtype, n, G, scale, size).go()


@pytest.mark.parametrize("dtype,out_dtype", FORMS)
def test_a_scale_of_zero_makes_infinite_logits_nan(dtype, out_dtype):
    c = batch(dtype, out_dtype, 3, 2, 0.0, 1.0)
    c.q[:] = c.q.abs()
    c.K[0, int(c.table[0, 1]), 0, 2, 9] = float("inf")
    c.run()
    reco.reco_check()
    assert torch.isnan(c.lse[0, :3, :2]).all() and torch.isfinite(c.lse[0, 3:]).all() and torch.isfinite(c.lse[0, :, 2:]).all()
    assert torch.isnan(c.out[0, :3, :2]).all() and torch.isfinite(c.out[0, 3:]).all()
