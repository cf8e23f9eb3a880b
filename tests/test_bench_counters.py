"""The committed HBM counters that bench.py reports as an attention launch's
traffic: they are of the kernels that are there."""
import json

import pytest

import bench

CONFIGS = ["qwen7b", "qwen1.5b", "grpo", "longtail"]


def test_every_file_of_the_kernels_counts(tmp_path, monkeypatch):
    """The plan and combine kernels are in another file than the attention kernel:
    a change of either makes the counters stale."""
    files = []
    for p in bench.ATTN_SRC:
        text = open(p).read()
        files.append((tmp_path / p.split("/")[-1], text))
        files[-1][0].write_text(text)
    assert any("tree_attn_plan_kernel(AttnBase" in t for _, t in files)
    assert any("tree_attn_combine_kernel(AttnBase" in t for _, t in files)
    assert any("tree_attn_kernel(AttnArgs" in t for _, t in files)
    monkeypatch.setattr(bench, "ATTN_SRC", tuple(str(f) for f, _ in files))
    out = tmp_path / "c.json"
    monkeypatch.setattr(bench, "counters_path", lambda name: str(out))
    out.write_text(json.dumps({"source_sha256": bench.source_sha(bench.ATTN_SRC), "hbm_bytes_per_launch": 5.0}))
    assert bench.counter_traffic("tiny") == 5.0
    for f, text in files:
        f.write_text(text + "\n// changed\n")
        assert bench.counter_traffic("tiny") is None
        f.write_text(text)


@pytest.mark.parametrize("config", CONFIGS)
def test_the_committed_counters_are_of_these_kernels(config):
    """(After a change of the kernels the counters are taken again: profiles/ has the commands.)"""
    traffic = bench.counter_traffic(config)
    assert traffic is not None and traffic > 0
