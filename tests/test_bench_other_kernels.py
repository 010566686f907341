"""The HBM traffic that bench.py reports was measured with the codec's kernels as they are, whatever kernels stand beside them."""
import os
import re
import shutil
import sys

from conftest import ROOT

sys.path.insert(0, ROOT)
CSRC = os.path.join("paper_2604_03298_amd", "csrc")


def test_the_measured_traffic_is_the_present_codec_s():
    import bench
    assert bench.kernel_sources_sha256() == bench.MEASURED_TRAFFIC["kernel_sources_sha256"], "the codec changed: measure its traffic again"


def test_kernels_beside_the_codec_do_not_count(tmp_path, monkeypatch):
    import bench
    here = bench.kernel_sources_sha256()
    shutil.copytree(os.path.join(ROOT, CSRC), tmp_path / CSRC)
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    for name in ("sampling.hip", "lowbit_fp8.hip", "one_more.hip", "one_more.hpp"):
        with open(tmp_path / CSRC / name, "a") as f:
            f.write("\nstatic int one_more;\n")
        assert bench.kernel_sources_sha256() == here, name


def test_the_codec_includes_its_own_sources_only():
    """Which is what lets the others be left out."""
    names = [n for n in os.listdir(os.path.join(ROOT, CSRC)) if n.startswith("enec")]
    assert len(names) >= 10
    for name in names:
        with open(os.path.join(ROOT, CSRC, name), encoding="utf-8") as f:
            included = re.findall(r'#include "([^"]+)"', f.read())
        assert all(n.startswith("enec") for n in included), name
