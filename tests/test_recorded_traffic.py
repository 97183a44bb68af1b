"""bench.py reports the HBM traffic of a launch from the counters in profiles/decode_traffic.json as long as the sources are those they were taken
on, and nothing otherwise: a change to these files, a shared header's too, wants new counters."""
import hashlib
import json
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent
RECORDS = json.loads((ROOT / "profiles" / "decode_traffic.json").read_text())


@pytest.mark.parametrize("workload", sorted(RECORDS))
def test_the_recorded_traffic_is_that_of_the_present_kernels(workload):
    for name, digest in RECORDS[workload]["source_sha256_16"].items():
        source = ROOT / "paper_2502_07864_amd" / "csrc" / name
        assert hashlib.sha256(source.read_bytes()).hexdigest()[:16] == digest, f"{name} is not the one that the counters of {workload} were taken on"
