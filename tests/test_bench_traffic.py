"""The bench reports measured HBM traffic only while the kernel's code is what the
counters were taken on: its source and the headers it includes.  Host-side only."""
import json
import os
import shutil

import pytest

import bench


@pytest.fixture
def tree(tmp_path, monkeypatch):
    csrc = shutil.copytree(bench.CSRC, tmp_path / "csrc")
    monkeypatch.setattr(bench, "CSRC", str(csrc))
    monkeypatch.setattr(bench, "PROFILES", str(tmp_path))
    for name, src in (("vocab_pass", "denoise.hip"), ("attn_bf16", "attention.hip")):
        rec = {"src_sha": bench.src_sha(src), "hbm_bytes_per_launch": 7}
        (tmp_path / f"{name}_w_traffic.txt").write_text("# taken\n" + json.dumps(rec, indent=1) + "\n")
    return csrc


def traffic():
    return (bench.measured_traffic("vocab_pass", "w", "denoise.hip"),
            bench.measured_traffic("attn_bf16", "w", "attention.hip"))


@pytest.mark.parametrize("changed,left", [
    (None, (7, 7)), ("denoise.hip", (None, 7)), ("vocab.h", (None, 7)), ("top.h", (None, 7)),
    ("attention.hip", (7, None)), ("internal.h", (None, None)), ("rules.hip", (7, 7))])
def test_a_changed_source_or_header_drops_the_figure(tree, changed, left):
    if changed:
        path = os.path.join(tree, changed)
        with open(path, "a") as f:
            f.write("// changed\n")
    assert traffic() == left


def test_files_of_a_kernel():
    assert bench.kernel_files("denoise.hip") == ["denoise.hip", "internal.h", "vocab.h", "top.h"]
    assert bench.kernel_files("attention.hip") == ["attention.hip", "internal.h"]
