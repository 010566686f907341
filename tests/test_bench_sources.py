"""bench.py reports HBM traffic only while the sources of the codec's kernels are those that it was measured with."""
import os
import shutil
import sys

from conftest import ROOT

sys.path.insert(0, ROOT)


def test_the_measured_traffic_goes_by_the_codec_s_sources_only(tmp_path, monkeypatch):
    import bench
    here = bench.kernel_sources_sha256()
    csrc = os.path.join("paper_2604_03298_amd", "csrc")
    shutil.copytree(os.path.join(ROOT, csrc), tmp_path / csrc)
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    assert bench.kernel_sources_sha256() == here

    def after(name):
        with open(tmp_path / csrc / name, "a") as f:
            f.write("\nstatic int one_more;\n")
        return bench.kernel_sources_sha256()

    for name in ("lowbit.hpp", "lowbit_attention.hip", "lowbit_matmul.hip"):
        assert after(name) == here, name                   # other kernels, which the codec does not include
    seen = {here}
    for name in ("enec_kernels.hip", "enec_device.hpp", "enec_decompress.hip"):
        seen.add(after(name))
    assert len(seen) == 4
