"""The traffic records that bench.py reads were taken on the kernels of this tree: once their
sources change, bench.py reports no traffic until the records are taken anew."""
import glob
import json
import os

from paper_2609_34977_amd import profiling as P

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_records_are_those_of_the_present_sources():
    paths = sorted(glob.glob(os.path.join(ROOT, "profiles", "gemm_gateup_traffic_*.json")))
    assert len(paths) >= 2
    for path in paths:
        rec = json.load(open(path))
        assert rec["source_sha256"] == P.kernel_source_hash(rec["kernel_class"]), path
        assert P.recorded_traffic(path, rec["kernel_class"], rec["workload"], rec["rows"]) == rec["bytes_per_launch"]
