"""Which changes void a row of the DRAM-traffic table: those to files that the kernel is made of."""
import os
import shutil

from paper_2603_14360_b200 import ncu_traffic


def test_a_change_voids_the_rows_of_kernels_that_see_it(tmp_path, monkeypatch):
    csrc = tmp_path / "csrc"
    shutil.copytree(ncu_traffic.CSRC, csrc)
    monkeypatch.setattr(ncu_traffic, "CSRC", str(csrc))
    was = {f: ncu_traffic.source_digest(f) for f in ("scan_fwd_bf16_cs.cu", "gated_norm.cu")}
    (csrc / "another.cuh").write_text("// of another kernel\n")      # not included
    (csrc / "reduce.cu").write_text("// of another kernel\n")
    assert was == {f: ncu_traffic.source_digest(f) for f in was}
    with open(csrc / "mma_tile.cuh", "a") as f:                       # included by the scan, not by the norm
        f.write("// changed\n")
    assert ncu_traffic.source_digest("gated_norm.cu") == was["gated_norm.cu"]
    assert ncu_traffic.source_digest("scan_fwd_bf16_cs.cu") != was["scan_fwd_bf16_cs.cu"]
    with open(csrc / "internal.h", "a") as f:
        f.write("// changed\n")
    assert ncu_traffic.source_digest("gated_norm.cu") != was["gated_norm.cu"]


def test_sources_include_what_headers_include():
    got = ncu_traffic.sources_of("scan_fwd_tc.cu")
    assert got[0] == "scan_fwd_tc.cu" and {"internal.h", "tc_common.cuh", "pipeline.cuh"} <= set(got) and "m2rnn.h" not in got
    assert "tile.cuh" in ncu_traffic.sources_of("scan_bwd_bf16.cu") and "delta.h" not in ncu_traffic.sources_of("scan_bwd_bf16.cu")
    assert all(os.path.exists(os.path.join(ncu_traffic.CSRC, f)) for f in got)


def test_the_committed_rows_are_of_the_sources_as_they_are():
    """A row that a change made void is captured again (or taken out), not carried along."""
    for line in open(ncu_traffic.TABLE):
        f = line.split()
        if f and not f[0].startswith("#"):
            assert f[5] == ncu_traffic.source_digest(f[2]), f[0]
