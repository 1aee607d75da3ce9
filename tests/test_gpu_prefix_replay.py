"""Graphs of decode attention over shared prefixes, replayed with other contents of the same buffers: every replay sees what
was written before it, in calls large and small (those of more than 600 units take short own rows where the parts join)."""
import pytest
import torch

from paper_2608_04771_gb300 import reco
from test_gpu_prefix import BF, DEV, F32, Batch, _lib, bits  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("Ly", [2, 40])
def test_replays_with_new_queries_rows_and_lengths(dtype, out_dtype, Ly):
    """32 or 640 units, 1 to 40 rows of their own; queries, new rows, groups and lengths change between replays, and between
    them a small kernel of the graph itself writes the queries."""
    n, H, G, d, page, P = 8, 2, 4, 128, 16, 160
    c = Batch(51, Ly, G * H, H, d, dtype, page, [0] * n, [P] * n, 39, out_dtype=out_dtype, garbage=False)
    c.table[1:, :P // page] = c.table[0, :P // page]  # every sequence names the prefix's pages, so that any grouping will do
    fresh = torch.empty_like(c.q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    lens = c.lens.clone()
    with torch.cuda.stream(side):
        c.run()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            c.q.copy_(fresh)
            c.run()
    torch.cuda.synchronize()
    for turn, group in enumerate(([0] * n, [0] * 3 + [1] * 5, list(range(n)), [0] * n)):
        c.group = group
        c.groups.copy_(torch.tensor(group))
        c.lens.copy_(lens - torch.randint(0, 39, lens.shape, device=DEV, dtype=torch.int32))
        c.kn.copy_(c.rand(*c.kn.shape))
        c.vn.copy_(c.rand(*c.vn.shape))
        fresh.copy_(c.rand(*c.q.shape))
        c.q.copy_(fresh)
        ref, before = c.reference(), (c.K.clone(), c.V.clone())
        c.q.fill_(float("nan"))
        c.out.fill_(7)
        g.replay()
        reco.reco_check()
        c.check(ref, before)
    # one replay after the other, nothing between them: each with the queries of the one before turned around
    first = fresh.clone()
    outs = []
    for _ in range(6):
        fresh.copy_(-fresh)
        c.lens -= 1
        g.replay()
        outs.append(c.out.clone())
    reco.reco_check()
    assert torch.equal(fresh, first)
    for i, x in enumerate(outs[2:]):
        assert torch.equal(bits(x), bits(outs[i % 2]))
    assert not torch.equal(outs[0], outs[1])
