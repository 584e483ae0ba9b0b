"""The traffic record's hash covers the sources that its kernels are built from."""
import shutil

import bench


def test_hash_leaves_out_sources_the_workloads_never_launch(tmp_path, monkeypatch):
    src = bench.ROOT / "paper_2609_34420_amd" / "csrc"
    dst = tmp_path / "paper_2609_34420_amd" / "csrc"
    shutil.copytree(src, dst)
    want = bench.kernel_sources_sha256()
    monkeypatch.setattr(bench, "ROOT", tmp_path)
    for name in ("pack_fwd.hpp", "pack_api.hip", "api.hip", "fwd_short.hip"):
        (dst / name).write_text("// changed")
    assert bench.kernel_sources_sha256() == want
    (dst / "fwd_mfma.hpp").write_text("// changed")
    assert bench.kernel_sources_sha256() != want
