"""The bench's counter and trace summaries are tied to the sources of the kernels
that it runs, and to no others."""
import os
import shutil

import bench


def test_measured_sources():
    """The row softmax's and the DAM attention's, with all that they include."""
    files = bench.measured_source_files()
    assert {"softmax_api.hip", "attention_api.hip", "sm_device.hpp", "sm_host.hpp"} <= set(files)
    assert not [name for name in files if "heads" in name or "cache" in name]
    for name in files:
        with open(os.path.join(bench.CSRC, name)) as f:
            for line in f:
                if line.startswith('#include "sm_'):
                    assert line.split('"')[1] in files, (name, line)


def test_other_sources_do_not_matter(tmp_path, monkeypatch):
    copy = tmp_path / "csrc"
    shutil.copytree(bench.CSRC, copy)
    monkeypatch.setattr(bench, "CSRC", str(copy))
    before = bench.kernel_source_sha256()
    (copy / "another.hip").write_text("// other kernels\n")
    assert bench.kernel_source_sha256() == before
    for name in ("softmax_api.hip", "sm_kernels.hpp", "sm_exchange.hpp", "sm_attention_wave.hpp"):
        text = (copy / name).read_text()
        (copy / name).write_text(text + "\n")
        assert bench.kernel_source_sha256() != before, name
        (copy / name).write_text(text)
    assert bench.kernel_source_sha256() == before
