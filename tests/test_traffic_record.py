"""The recorded HBM traffic that bench.py reports is that of the current kernels: a
change of their sources, or of what they share, voids a record, and bench.py then
reports none (profile_summary.py makes a new one from counters)."""

import json

import bench


def test_traffic_is_recorded_for_the_current_kernels():
    with open(bench.TRAFFIC_FILE) as f:
        record = json.load(f)
    for phase in ("kpass", "gram", "leverage", "weights", "select", "compact", "kpass_tri", "qfactor", "qstats"):
        assert record[phase]["source_sha"] == bench.source_sha(phase), phase
        assert bench.recorded_traffic(phase, "long128k") > 0
