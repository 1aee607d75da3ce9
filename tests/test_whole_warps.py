"""Instructions that a whole warp must execute together, checked on the sources: barriers of a number of threads are of whole
warps, fixed when the kernel is compiled."""
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
