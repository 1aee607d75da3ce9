"""Decode attention over shared prefixes when one of its own waits runs out: the error word says so, every unit of the call is
in error (zeros, lse = -inf, the length kept) whatever partials an earlier call has left in the workspace, and the next call
is as ever.  No call's waits run out by themselves: here the library is linked once more, with tensor maps whose boxes are smaller than
what the kernels wait for, and with a limit of 2^12 polls in place of 2^19."""
import concurrent.futures as cf
import ctypes
import re
import subprocess

import numpy as np
import pytest
import torch

from paper_2608_04771_gb300 import build, reco
from test_gpu_prefix import BF, F32, Batch

pytestmark = pytest.mark.gpu

API = r"""
#define encode_bf16_2d whole_bf16_2d
#define encode_bf16_heads whole_heads
#define encode_f32_2d whole_f32_2d
#include "api.cu"
#undef encode_bf16_2d
#undef encode_bf16_heads
#undef encode_f32_2d
namespace reco {
static int cut = 0, calls = 0;  // 1: queries, 2: keys, 4: values (keys and values take turns)
static int rows_of(int box_rows) { return cut & (calls++ & 1 ? 4 : 2) ? box_rows / 2 : box_rows; }
bool encode_bf16_heads(void *map, const void *base, unsigned long long rows, int heads, int d, int box_heads, int box_rows)
{
    return whole_heads(map, base, rows, heads, d, box_heads, cut & 1 && box_rows > 1 ? box_rows - 1 : box_rows);
}
bool encode_bf16_2d(void *map, const void *base, unsigned long long rows, int cols, int box_cols, int box_rows)
{
    return whole_bf16_2d(map, base, rows, cols, box_cols, rows_of(box_rows));
}
bool encode_f32_2d(void *map, const void *base, unsigned long long rows, int cols, int box_cols, int box_rows)
{
    return whole_f32_2d(map, base, rows, cols, box_cols, rows_of(box_rows));
}
}  // namespace reco
extern "C" void cut_boxes(int what) { reco::cut = what; }
"""
QUERIES, KEYS, VALUES = 1, 2, 4


@pytest.fixture(scope="module")
def cut_boxes(tmp_path_factory):
    """The binding on the library with smaller boxes, switched by the function that it gives."""
    build.build()
    d = tmp_path_factory.mktemp("wait")
    (d / "api.cu").write_text(API.replace('"api.cu"', '"%s"' % (build.CSRC / "api.cu")))
    for name in ("prefix.cu", "prefix_tc.cu"):
        text, n = re.subn(r"(Polls = 1LL <<) 19;", r"\1 12;", (build.CSRC / name).read_text())
        assert n == 1
        (d / name).write_text(text)

    def compile_one(name):
        cmd = [build.nvcc(), "-O3", "-std=c++17", "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr", "-I", str(build.INCLUDE), "-I",
               str(build.CSRC), *build.ARCH, "-c", "-o", str(d / name) + ".o", str(d / name)]
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
    with cf.ThreadPoolExecutor() as ex:
        list(ex.map(compile_one, ("api.cu", "prefix.cu", "prefix_tc.cu")))
    mine = {"api", "prefix", "prefix_tc"}
    objs = [str(build.OUT_DIR / (p.stem + ".o")) for p in sorted(build.CSRC.glob("*.cu")) if p.stem not in mine]
    objs += [str(d / (n + ".cu.o")) for n in sorted(mine)]
    r = subprocess.run([build.nvcc(), *build.ARCH, "-shared", "-cudart", "static", "-o", str(d / "wait.so"), *objs], capture_output=True,
                       text=True)
    assert r.returncode == 0, r.stderr
    old = reco._lib, reco._LIB_PATH
    reco._lib, reco._LIB_PATH = None, d / "wait.so"
    yield reco.lib().cut_boxes
    reco.lib().cut_boxes(ctypes.c_int(0))
    reco._lib, reco._LIB_PATH = old


@pytest.mark.parametrize("Ly", [1, 40])
@pytest.mark.parametrize("what,dtype,d,out_dtype", [
    (QUERIES, BF, 64, BF), (QUERIES, BF, 128, F32), (KEYS, F32, 64, F32), (VALUES, F32, 128, F32), (KEYS | VALUES, F32, 128, F32),
    (KEYS, BF, 128, BF), (VALUES, BF, 64, BF), (KEYS, BF, 64, F32), (VALUES, BF, 128, F32), (KEYS | VALUES, BF, 128, BF)])
def test_a_wait_that_runs_out(cut_boxes, what, dtype, d, out_dtype, Ly):
    """A few units and more than 600 of them, with few rows of their own and with many."""
    mine = np.random.default_rng(3).choice([1, 5, 40, 150], (Ly, 8, 2))
    c = Batch(41, Ly, 8, 2, d, dtype, 16, [0] * 5 + [1] * 3, [300] * 5 + [130] * 3, mine, out_dtype=out_dtype)
    lens = c.lens.clone()
    c.go()
    good = c.out.clone(), c.lse.clone()
    c.lens.copy_(lens)
    c.q.neg_()
    cut_boxes(ctypes.c_int(what))
    c.run()
    with pytest.raises(reco.RecoError) as e:
        reco.reco_check()
    cut_boxes(ctypes.c_int(0))
    assert "internal-check" in str(e.value)
    assert (c.out == 0).all() and torch.isneginf(c.lse).all() and torch.equal(c.lens, lens)
    c.q.neg_()
    c.run()
    reco.reco_check()
    assert torch.equal(c.out, good[0]) and torch.equal(c.lse, good[1]) and torch.equal(c.lens, lens + 1)
