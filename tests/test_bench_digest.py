"""Which sources a traffic figure in bench.py's line stands for."""
import os
import shutil


def test_every_source_but_the_paged_caches_counts(tmp_path, monkeypatch):
    import bench
    folder = tmp_path / "paper_2507_07990_amd" / "csrc"
    shutil.copytree(os.path.join(bench.ROOT, "paper_2507_07990_amd", "csrc"), folder)
    here = bench.source_digest()
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    assert bench.source_digest() == here
    for name in ("sttm_rope.hip", "sttm_attention.hip", "sttm_evict.hip", "sttm_cache.h"):
        (folder / name).write_text("// another one")
    assert bench.source_digest() == here
    (folder / "sttm_new_stage.hip").write_text("// a file that was not there")
    assert bench.source_digest() != here
