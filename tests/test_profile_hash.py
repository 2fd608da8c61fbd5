"""The hash that ties stored profiler figures of the benchmark's step to its kernels: their sources and no others."""
import os
import shutil

from paper_2206_06257_amd import profile_summary as ps

CSRC = os.path.join(ps.ROOT, "paper_2206_06257_amd", "csrc")


def test_hash_goes_by_the_sources_of_the_step(tmp_path, monkeypatch):
    csrc = tmp_path / "paper_2206_06257_amd" / "csrc"
    shutil.copytree(CSRC, csrc)
    first = ps.source_hash()
    monkeypatch.setattr(ps, "ROOT", str(tmp_path))
    assert ps.source_hash() == first
    for name in ("attention.hip", "rotary.hip", "clip.hip", "groupnorm.hip", "logprobs.hip", "heads.h", "lanes.h"):
        (csrc / name).write_text("// another text\n")
    (csrc / "one_more.hip").write_text("// a new operator\n")
    assert ps.source_hash() == first
    for name in ("model.hip", "conv_mfma.hip", "conv_direct.hip", "layers.hip", "pgd.hip", "quantize.hip", "kernels.h", "common.h", "philox.h", "tensor_table.h"):
        text = (csrc / name).read_text()
        (csrc / name).write_text(text + "// changed\n")
        assert ps.source_hash() != first, name
        (csrc / name).write_text(text)
    assert ps.source_hash() == first
