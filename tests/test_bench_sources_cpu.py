"""Which sources a profile's stamp covers: bench.py reads the linears' measured
traffic as long as what their calls are built from stays the same."""
import os
import shutil

import pytest

import bench

CSRC = os.path.join("paper_2412_04787_amd", "csrc")


@pytest.fixture
def tree(tmp_path, monkeypatch):
    shutil.copytree(os.path.join(bench.ROOT, CSRC), tmp_path / CSRC, ignore=shutil.ignore_patterns("_build"))
    shutil.copy(os.path.join(bench.ROOT, "paper_2412_04787_amd", "build_lib.py"), tmp_path / "paper_2412_04787_amd")
    (tmp_path / "profiles").mkdir()
    (tmp_path / "profiles" / "bwd_wl_counters.txt").write_text(
        f"kernel_source_hash = {bench.kernel_source_hash()}\nfetch_write_bytes_per_launch = 1234\n")
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    return tmp_path


def change(tree, f):
    with open(tree / CSRC / f, "a") as out:
        out.write("// changed\n")


@pytest.mark.parametrize("f", ["new_operator.hip", "new_operator.h", "kv_attn.hip", "kv_common.h", "cache_launch.h", "rope.h",
                               "abi_cache.hip", "attn.hip", "logprob.hip", "swiglu.hip"])
def test_other_operators_leave_the_linears_traffic(tree, f):
    every = bench.kernel_source_hash(None)
    assert bench.read_traffic("bwd", "wl") == 1234.0
    change(tree, f)
    assert bench.read_traffic("bwd", "wl") == 1234.0
    assert bench.kernel_source_hash(None) != every


@pytest.mark.parametrize("f", ["gemm_v3.hip", "abi.hip", "sr_update.hip", "abi_check.h", "gemm_common.h", "sr_rule.h", "dqt_launch.h",
                               "dqt_device.h", "../build_lib.py"])
def test_what_the_linears_are_built_from_does_not(tree, f):
    assert bench.read_traffic("bwd", "wl") == 1234.0
    change(tree, f)
    assert bench.read_traffic("bwd", "wl") is None


def test_sources_are_there():
    for f in bench.LINEAR_SOURCES:
        assert os.path.exists(os.path.join(bench.ROOT, CSRC, f))
