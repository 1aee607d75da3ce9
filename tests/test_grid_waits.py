"""Kernels that may start while the one before them drains read nothing of global memory before their own wait for it:
only behind that wait is what earlier kernels wrote sure to be seen.  Checked on the sources."""
import re

import pytest

from paper_2608_04771_gb300 import build

READS = re.compile(r"__ld[a-z]+\(|\w+->|\b[a-z]\.[\w.]*\w\[|\*\s?[a-z]\.\w|\bld_\w+\(|pool_row\(|own_total\(")


def kernels():
    """(file, what stands before the wait) of every kernel that waits."""
    for path in sorted(build.CSRC.glob("*.cu")):
        text = re.sub(r"//[^\n]*", "", path.read_text())
        for m in re.finditer(r"__global__[^;{]*\)\s*\{", text):
            depth, i = 1, m.end()
            while depth:
                depth += (text[i] == "{") - (text[i] == "}")
                i += 1
            body = text[m.end():i]
            if "wait_prior_grid()" in body:
                name = re.findall(r"(\w+)\s*\(", re.sub(r"__launch_bounds__\((?:[^()]|\([^()]*\))*\)", "", m.group(0)))[0]
                yield pytest.param(body.split("wait_prior_grid()")[0], id=f"{path.stem}-{name}")


@pytest.mark.parametrize("before", list(kernels()))
def test_nothing_is_read_before_the_wait(before):
    assert not READS.findall(before)


def test_the_check_sees_a_read():
    for line in ("const int run = a.p.run_of[b];", "const T total = *a.p.total;", "x = __ldg(p);", "if (total->work)"):
        assert READS.search(line)
