"""The counter profiles that the benchmark quotes are those of the kernels in the tree (no GPU needed)."""

import argparse

import bench
from paper_2609_35465_amd import build


def test_recorded_traffic_and_instructions_hold():
    """Where a kernel or its flags change, its profile is taken again; a change to the way of linking is no such change."""
    args = argparse.Namespace(mode="chain", batch=1, model="14B", workload="tetra")
    assert bench.recorded_traffic(args, 40) is not None
    want = {"source_sha256": bench.encoder_source_hash(), "blocks": "20000"}
    assert bench.profile_record(bench.ENCODER_PROFILE, want, "valu_wave_instructions_per_launch") is not None


def test_sources_are_compiled_apart_and_linked_once(monkeypatch):
    calls = []
    monkeypatch.setattr(build, "generate_tables", lambda verbose=False: "inc")
    monkeypatch.setattr(build, "_run", lambda cmd, verbose, **kw: calls.append(cmd))
    monkeypatch.setattr(build.os, "replace", lambda a, b: None)
    build.build()
    assert [c for c in calls if "-c" not in c] == [calls[-1]] and "-shared" in calls[-1]
    assert len(calls) == len(build.SOURCES) + 1
    for c in calls[:-1]:
        assert "-shared" not in c and "-packed-fp32-ops" in c and "--offload-arch=gfx950" in c
