"""The key of a traffic row: the kernel's source and the device headers it includes, each by its hash."""
import os
import re

import bench


def _headers(name):
    """The .cuh files that a source includes, directly or through others."""
    found = set()
    for h in re.findall(r'#include "([^"/]+\.cuh)"', open(os.path.join(bench.CSRC, name)).read()):
        found |= {h} | _headers(h)
    return found


def test_a_changed_header_makes_a_row_stale(tmp_path, monkeypatch):
    (tmp_path / "k.cu").write_text('#include "waits.cuh"\n')
    (tmp_path / "waits.cuh").write_text("// one\n")
    monkeypatch.setattr(bench, "CSRC", str(tmp_path))
    key = " ".join(f"{f}:{bench.source_hash(f)}" for f in ("k.cu", "waits.cuh"))
    table = tmp_path / "dram_traffic.md"
    table.write_text(f"| cfg4 | denoise | 256 | 1.7e8 | 1.6e7 | {key} | a note: with a colon |\n| cfg4 | mix | 256 | 1e8 | - |  | no source |\n")
    monkeypatch.setattr(bench, "TRAFFIC_TABLE", str(table))
    assert bench.measured_traffic() == {("cfg4", "denoise"): (256, 1.7e8, 1.6e7)}
    (tmp_path / "waits.cuh").write_text("// two\n")
    assert bench.measured_traffic() == {}
    (tmp_path / "waits.cuh").write_text("// one\n")
    assert len(bench.measured_traffic()) == 1
    (tmp_path / "waits.cuh").unlink()
    assert bench.measured_traffic() == {}


def test_rows_of_the_table_name_every_header_of_their_kernel():
    rows = 0
    for ln in open(bench.TRAFFIC_TABLE):
        f = [x.strip() for x in ln.strip().strip("|").split("|")]
        if len(f) < 6 or not f[2].isdigit():
            continue
        files = [x.partition(":")[0] for x in f[5].split()]
        assert files[0].endswith(".cu") and set(files[1:]) == _headers(files[0]), ln
        rows += 1
    assert rows > 0
