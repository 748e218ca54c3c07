"""What the traffic figures of the profile are tied to: the sources of the kernels that they describe, and no others."""
import os
import re
import shutil

import bench

CSRC = os.path.join(bench.ROOT, "paper_2502_00299_amd", "csrc")
OTHER_CALLS = {"decode_plan.h", "chunkkv.h"}   # the plan of decode attention; the public header, most of it documentation


def test_includes_are_among_the_sources():
    for name in bench.TRAFFIC_SOURCES:
        for other in re.findall(r'#include "(\w+\.h)"', open(os.path.join(CSRC, name)).read()):
            assert other in bench.TRAFFIC_SOURCES or other in OTHER_CALLS, (name, other)


def test_hash_follows_these_sources_alone(tmp_path, monkeypatch):
    shutil.copytree(CSRC, tmp_path / "paper_2502_00299_amd" / "csrc")
    before = bench.csrc_hash()
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    assert bench.csrc_hash() == before
    for name in sorted(os.listdir(CSRC)):
        path = tmp_path / "paper_2502_00299_amd" / "csrc" / name
        text = path.read_text()
        path.write_text(text + "\n")
        assert (bench.csrc_hash() != before) == (name in bench.TRAFFIC_SOURCES), name
        path.write_text(text)
