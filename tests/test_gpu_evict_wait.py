"""The parallel compaction's wait for a chunk that nobody reads: it runs out, the error word says so, and nothing is
written over the rows that were waited for.  The kernel is compiled by itself and given its list by hand, since
no call leaves a chunk out."""
import ctypes
import subprocess

import numpy as np
import pytest
import torch

from paper_2608_04771_gb300 import build

pytestmark = pytest.mark.gpu
DEV = "cuda"

SOURCE = r"""
#include "evict.cu"
namespace reco {
int device_sm_count() { return 1; }
cudaError_t launch_select_budget(const reco_paged_kv &, float *, int32_t *, const int32_t *, int, int, int32_t *,
                                 const EvictWs &, unsigned *, cudaStream_t)
{
    return cudaErrorNotSupported;
}
}  // namespace reco
// one unit of 512 rows of 128 bytes in pages of 16
extern "C" int run_chunks(void *K, void *V, const int *table, const int *idx, const int *lens, int *counters, int *rank,
                          int *flags, void *list, int *ulist, unsigned *err, int ctas)
{
    reco::EvictWs ws{counters, nullptr, rank, flags, (int4 *)list, ulist, 0};
    reco::CompactArgs a{(char *)K, (char *)V, table, idx, lens, ws, 1, 1, 1, 32, 32, 4, 15, 16, 512, 4, 0, err};
    reco::compact_chunks<128><<<ctas, reco::kCompactThreads>>>(a);
    return (int)cudaDeviceSynchronize();
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("wait")
    (d / "wait.cu").write_text(SOURCE)
    cmd = [build.nvcc(), "-O3", "-std=c++17", "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr", "-I", str(build.INCLUDE),
           "-I", str(build.CSRC), *build.ARCH, "-shared", "-cudart", "static", "-o", str(d / "wait.so"), str(d / "wait.cu")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return ctypes.CDLL(str(d / "wait.so"))


def _run(lib, chunks):
    """Rows 128 to 383 of 512 move to 0 to 255, by the chunks that are listed; the second writes where the first
    one's rows come from."""
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    K, V = (torch.randn((32, 1, 16, 64), generator=g, device=DEV).bfloat16() for _ in range(2))
    K0, V0 = K.clone(), V.clone()
    i32 = lambda x: torch.tensor(np.asarray(x, np.int32), device=DEV)  # noqa: E731
    table, idx, lens = i32(np.random.default_rng(2).permutation(32)), i32(np.r_[128:384, np.zeros(256)]), i32([256])
    counters, rank = i32([0, len(chunks), 0, 1]), i32([0, 0, 128, 256, 256])
    flags, ulist, err = i32([0] * 4), i32([0]), i32([0])
    places = i32([[0, c, 256, 0] for c in chunks] + [[0, 0, 0, 0]] * (4 - len(chunks)))
    torch.cuda.synchronize()
    p = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    st = lib.run_chunks(*(p(t) for t in (K, V, table, idx, lens, counters, rank, flags, places, ulist, err)), 2)
    assert st == 0 and not counters.any()
    order = table.long()
    rows = lambda t: t[order].reshape(512, 64)  # noqa: E731
    return rows(K0), rows(K), rows(V0), rows(V), int(err), flags.tolist()


def test_listed_chunks_move(lib):
    K0, K, V0, V, err, flags = _run(lib, [0, 1])
    assert err == 0 and flags == [1, 1, 0, 0]
    for a, b in ((K0, K), (V0, V)):
        assert torch.equal(b[:256], a[128:384]) and torch.equal(b[256:], a[256:])


def test_a_chunk_that_is_waited_for_in_vain_is_not_written_over(lib):
    K0, K, V0, V, err, flags = _run(lib, [1])
    assert err == 32 and flags == [0, 1, 0, 0]  # an internal check has failed
    assert torch.equal(K, K0) and torch.equal(V, V0)
