"""Where the parts of decode attention over shared prefixes join: a CTA of 256 threads shares a unit's query heads and columns
out, evenly or (head dimension 64 with 3 or 5 query heads per KV head: 240 threads) not."""
import numpy as np
import pytest
import torch

from test_gpu_prefix import BF, F32, Batch, _lib, bits  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,Ly", [(G, 1) for G in range(1, 17)] + [(3, 52), (5, 52), (8, 52)])
def test_heads_that_fill_the_threads_or_not(dtype, d, G, Ly):
    """Prefixes cut between CTAs (16 units) or many units with few own rows (832)."""
    mine = np.random.default_rng(G).choice([0, 1, 5, 31, 32, 33, 70], (Ly, 8, 2))
    P = 1900 if Ly == 1 else 130
    b = Batch(60 + G, Ly, 2 * G, 2, d, dtype, 16, [0] * 5 + [1] * 3, [P] * 5 + [P - 100] * 3, mine, out_dtype=F32, garbage=Ly == 1)
    lens = b.lens.clone()
    b.go()
    out, lse = b.out.clone(), b.lse.clone()
    for _ in range(3):
        b.lens.copy_(lens)
        b.run()
        assert torch.equal(bits(out), bits(b.out)) and torch.equal(bits(lse), bits(b.lse))
