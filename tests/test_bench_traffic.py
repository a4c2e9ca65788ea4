"""The ncu traffic that the benchmark reports belongs to the eviction kernels' sources as they
are (CPU only)."""
import json
import os
import shutil

import bench

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_captured_row_is_of_the_current_sources():
    with open(os.path.join(ROOT, "profiles", "traffic.json")) as f:
        rows = json.load(f)
    assert {r["source_hash"] for r in rows.values()} == {bench.kernel_source_hash()}
    assert bench.ncu_traffic("prefill_wide") == rows["prefill_wide"]["dram_bytes_per_launch"]


def test_sources_of_the_4_bit_cache_do_not_count(tmp_path, monkeypatch):
    """A capture outlives changes of kernels that it did not run, and no others."""
    csrc = tmp_path / "paper_2609_23314_gb300" / "csrc"
    shutil.copytree(os.path.join(ROOT, "paper_2609_23314_gb300", "csrc"), csrc)
    before = bench.kernel_source_hash()
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    assert bench.kernel_source_hash() == before
    for name in ("vd_q4_attend.cuh", "vd_q4_rows.cu", "vd_qkv.cu", "vd_tcgen05.cuh"):
        (csrc / name).write_text("int changed;\n")
        assert bench.kernel_source_hash() == before
    for name in ("vd_device.cuh", "vd_evict.cuh", "vd_api.cu"):
        text = (csrc / name).read_text()
        (csrc / name).write_text(text + "\nint changed;\n")
        assert bench.kernel_source_hash() != before
        (csrc / name).write_text(text)
