"""The stored HBM traffic that bench.py reports beside the step's dominant kernel (no GPU needed)."""
import os
import re
import shutil

import pytest

import bench

CSRC = os.path.join(bench.ROOT, "paper_2609_14339_amd", "csrc")


def test_the_stored_traffic_is_of_these_sources():
    assert bench.measured_traffic("sc_ema", 5) > 25e9
    assert bench.measured_traffic("sc_ema", 2) is None and bench.measured_traffic("no such kernel", 5) is None


def test_the_block_shares_no_source_with_the_step():
    """No other file includes one of the block's."""
    for name in os.listdir(CSRC):
        if name not in bench.BLOCK_SOURCES:
            with open(os.path.join(CSRC, name)) as f:
                assert not set(re.findall(r'#include "([^"]+)"', f.read())) & set(bench.BLOCK_SOURCES), name
    assert all(os.path.exists(os.path.join(CSRC, name)) for name in bench.BLOCK_SOURCES)


@pytest.mark.parametrize("name,stands", [("lin_tile.hip", True), ("q8.h", True), ("new.hip", False), ("pass.hip", False),
                                         ("common.h", False)])
def test_a_changed_source(tmp_path, monkeypatch, name, stands):
    """The traffic stands when the block changes, and is withdrawn when anything else does."""
    csrc = tmp_path / "paper_2609_14339_amd" / "csrc"
    shutil.copytree(CSRC, csrc)
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    with open(csrc / name, "a") as f:
        f.write("// changed\n")
    assert (bench.measured_traffic("sc_ema", 5) is not None) == stands
