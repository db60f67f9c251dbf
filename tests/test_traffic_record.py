"""The roofline entry's traffic is a committed record, valid for the kernel's sources and compiler flags that it was taken
with: these have to be the present ones, or the benchmark reports none."""

import json
import re

import bench


def test_the_record_is_of_the_present_kernel():
    with open(bench.TRAFFIC_RECORD) as fh:
        rec = json.loads(re.search(r"^traffic_record: (\{.*\})$", fh.read(), re.M)[1])
    assert rec["source_sha256_16"] == bench.kernel_source_hash()
    assert bench.recorded_traffic(bench.WGRAD_KERNEL, rec["workload"], rec["workgroups"]) == rec["traffic_bytes"]
