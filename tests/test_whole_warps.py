"""Instructions that a whole warp must execute together, checked on the sources: barriers of a number of threads are of whole
warps, fixed when the kernel is compiled; lanes that waited for themselves, or stored where others did not, meet before they
touch tensor memory."""
import re

import pytest

from paper_2608_04771_gb300 import build

SOURCES = sorted([*build.CSRC.glob("*.cu"), *build.CSRC.glob("*.cuh")])


STATEMENT = re.compile(r"asm\s*(?:volatile)?\s*\((.*?)\);", re.S)


@pytest.mark.parametrize("path", SOURCES, ids=lambda p: p.name)
def test_counted_barriers_are_of_whole_warps(path):
    text = re.sub(r"//[^\n]*", "", path.read_text())
    for asm in STATEMENT.findall(text):
        if re.search(r"\bbar(?:\.sync|\.red|\.arrive|rier\.)", asm) and "barrier.cluster" not in asm and "%" in asm:
            assert re.search(r'"n"\((?:32 \* \w+|THREADS)\)', asm), asm


def test_lanes_meet_before_tensor_memory():
    """What a lane does by itself: a wait (await), a store of its row.  What all lanes do together: tmem_ leaves."""
    text = re.sub(r"//[^\n]*", "", (build.CSRC / "prefix_tc.cu").read_text())
    alone = None
    for m in re.finditer(r"\bawait\(|\bst_global_v8\(po|\bif \(there\) \{|__syncwarp\(\)|__(?:any|all)_sync\(|\bfine\(\)|__syncthreads\(\)|\btmem_(?:ld|st)\w+\(", text):
        word = m.group(0)
        if word.startswith(("await", "st_global", "if (there")):
            alone = m.start()
        elif word.startswith("tmem"):
            assert alone is None, text[alone:m.end()]
        else:
            alone = None
