"""Which form of the tree attention a call takes: the rule of csrc/tree_form.h, on the host."""
import ctypes
import shutil
import subprocess

import pytest

from paper_2504_05598_b200 import build


@pytest.fixture(scope="module")
def tcgen05(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    d = tmp_path_factory.mktemp("form")
    (d / "rule.cpp").write_text('#include "tree_form.h"\nextern "C" int rule(int hd, int nkv, int group, int nodes, int batch, int length, int streaming) {\n'
                                "    return tree::takes_tcgen05(hd, nkv, group, nodes, batch, (length + nodes + 15) / 16, 148, streaming != 0);\n}\n")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", build.CSRC, str(d / "rule.cpp"), "-o", str(d / "rule.so")], check=True)
    rule = ctypes.CDLL(str(d / "rule.so")).rule
    return lambda *a: bool(rule(*a))


@pytest.mark.parametrize("nodes", [5, 6, 8])
@pytest.mark.parametrize("length", [200, 3980, 4000, 8000, 16000, 32000])
def test_small_trees_between_streaming_gemms_stay_on_mma_sync(tcgen05, nodes, length):
    """8B shape: 5 to 8 rows a round are below the line of the tcgen05 layer GEMMs; with the tcgen05 attention between them a round behind 4000
    positions took 7.4 ms, with the other form 4.7."""
    assert not tcgen05(128, 8, 4, nodes, 1, length, 1)


def test_the_rule_between_other_kernels(tcgen05):
    for hd, nkv, group, nodes, batch, length, want in [(128, 8, 4, 8, 1, 200, 0), (128, 8, 4, 16, 1, 1000, 0), (128, 8, 4, 16, 1, 4000, 1), (128, 8, 4, 64, 1, 100, 0),
                                                       (128, 8, 4, 64, 1, 2000, 1), (128, 40, 1, 26, 1, 200, 0), (128, 40, 1, 26, 1, 3100, 1),
                                                       (128, 8, 4, 33, 4, 200, 1), (128, 8, 4, 4, 16, 4000, 0), (128, 40, 1, 17, 4, 4000, 0),
                                                       (64, 8, 4, 1, 32, 1100, 0), (64, 8, 4, 8, 4, 8000, 0), (64, 8, 4, 32, 1, 8000, 1), (128, 8, 4, 64, 8, 32700, 1)]:
        assert tcgen05(hd, nkv, group, nodes, batch, length, 0) == bool(want), (hd, nkv, group, nodes, batch, length)
    for length in (100, 4000, 30000):                            # head dimension 64: the same beside either kind of GEMM
        for nodes in (8, 32, 64):
            assert tcgen05(64, 8, 4, nodes, 1, length, 0) == tcgen05(64, 8, 4, nodes, 1, length, 1)
    assert not tcgen05(128, 12, 1, 64, 1, 8000, 1) and tcgen05(128, 12, 1, 64, 1, 16000, 1)      # 24 000 and 48 000 tile-pages
