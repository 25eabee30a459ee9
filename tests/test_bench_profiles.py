"""bench.py takes a committed profile for current as long as the sources of the kernels that it is of are the same."""
import os
import shutil

import bench


def test_other_operators_sources_do_not_count(tmp_path, monkeypatch):
    csrc = os.path.join("paper_1908_11263_amd", "csrc")
    here = bench.kernel_source_sha()
    shutil.copytree(os.path.join(bench.ROOT, csrc), tmp_path / csrc)
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    assert bench.kernel_source_sha() == here
    for f in os.listdir(tmp_path / csrc):
        if f.startswith("lm_"):
            os.remove(tmp_path / csrc / f)
    assert bench.kernel_source_sha() == here
    with open(tmp_path / csrc / "conv_img_impl.h", "a") as f:
        f.write("// changed\n")
    assert bench.kernel_source_sha() != here
