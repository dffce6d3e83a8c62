"""The traffic that bench.py quotes from counter runs goes with the kernels it was counted on, not with the library's version."""
import json
import os
import shutil

import pytest

import bench


@pytest.fixture
def tree(tmp_path, monkeypatch):
    csrc = tmp_path / "paper_2501_02573_amd" / "csrc"
    csrc.mkdir(parents=True)
    for name in bench.TRAFFIC_SOURCES:
        shutil.copy(os.path.join(bench.ROOT, "paper_2501_02573_amd", "csrc", name), csrc / name)
    (tmp_path / "profiles").mkdir()
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    record = {"_kernels": bench.traffic_key(), "job/kernel": {"hbm_bytes_per_launch": 7}}
    (tmp_path / "profiles" / "hbm_traffic.json").write_text(json.dumps(record))
    return csrc


def _append(tree, name, text):
    with open(tree / name, "a") as f:
        f.write(text)


def test_counts_stay_with_their_kernels(tree):
    assert bench.load_traffic("job", "kernel") == 7 and bench.load_traffic("job", "other") is None
    api = (tree / "leet_api.hip").read_text()
    assert 'leet_attn_version(void) { return "' in api
    head, tail = api.split('leet_attn_version(void) { return "')
    (tree / "leet_api.hip").write_text(head + 'leet_attn_version(void) { return "77.0.1' + tail[tail.index('"'):])
    _append(tree, "leet_fwd_16bit.hip", "\n   // a comment\n/* and\n another */\n")
    assert bench.load_traffic("job", "kernel") == 7


@pytest.mark.parametrize("name", bench.TRAFFIC_SOURCES)
def test_counts_of_other_kernels_are_not_quoted(tree, name):
    _append(tree, name, "\nstatic int one_more;\n")
    assert bench.load_traffic("job", "kernel") is None


def test_no_record(tree):
    os.remove(os.path.join(bench.ROOT, "profiles", "hbm_traffic.json"))
    assert bench.load_traffic("job", "kernel") is None
