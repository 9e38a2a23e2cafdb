"""Every device source with a kernel that starts before the one before it has ended and then reads what it wrote:
none reads through the read-only path, which may hold what was there before.  The files are found by what they
call, so that a new one is not left out."""
import os
import re

import pytest

from paper_2603_06492_gb300.build import CSRC


def _sources():
    out = {}
    for name in sorted(os.listdir(CSRC)):
        with open(os.path.join(CSRC, name)) as f:
            text = re.sub(r"//[^\n]*", "", f.read())
        if re.search(r"griddep_wait\(\)\s*;", text) and name.endswith(".cuh"):
            out[name] = text
    return out


def test_files():
    assert {"embed.cuh", "muon.cuh", "muon_gemm.cuh", "muon_small.cuh", "norm.cuh", "simt.cuh", "tc_cosnet.cuh"} <= set(_sources())


@pytest.mark.parametrize("name", sorted(_sources()))
def test_no_read_only_loads(name):
    assert re.findall(r"__ldg\w*|ld\.global\S*\.nc|__restrict__", _sources()[name]) == []
