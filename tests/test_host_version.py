"""The library's version tells its interfaces apart, and figures that were measured on a version are reported for that one only."""
import json
import os
import re
import sys

import paper_2507_11978_amd as nt

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_version_is_not_that_of_the_library_without_a_paged_cache():
    """0.7 had no nt_cache_write, nt_cache_read and nt_sdpa_paged, and neither of the 8-bit types."""
    assert hasattr(nt.load(), "nt_sdpa_paged")
    assert tuple(int(n) for n in re.match(r"nt-mi355x (\d+)\.(\d+) \(gfx950\)$", nt.version()).groups()) >= (0, 8)


def test_measured_traffic_names_its_kernel_and_version():
    sys.path.insert(0, ROOT)
    try:
        import bench
    finally:
        sys.path.remove(ROOT)
    with open(os.path.join(ROOT, "profiles", "traffic.json")) as f:
        records = json.load(f)
    assert "p_f16_8192" in records
    for workload, r in records.items():
        assert re.search(r"\w+_kernel", r["kernel"]) and r["library_version"].startswith("nt-mi355x ")
        assert bench.measured_traffic(workload, r["library_version"]) == r["hbm_bytes_per_launch"]
        assert bench.measured_traffic(workload, "nt-mi355x 0.1 (gfx950)") is None
