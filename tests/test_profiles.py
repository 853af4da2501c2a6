"""The recorded counters that bench.py quotes belong to the library as it is (CPU only)."""
import json
import os

import workloads

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_hbm_traffic_is_of_this_library():
    """bench.py quotes profiles/hbm_traffic.json only where it was taken with the library's version: one that is left behind is quoted no more."""
    from paper_2604_06746_amd import binding as B
    prof = json.load(open(os.path.join(ROOT, "profiles", "hbm_traffic.json")))
    assert prof["_library_version"] == B.structkv_version()
    measured = [name for name in workloads.WORKLOADS if name in prof]
    assert len(measured) >= 4
    for name in measured:
        wl = workloads.WORKLOADS[name]
        once = wl.n_kv_heads * wl.head_dim * wl.elem_bytes * wl.total_tokens       # K of a layer
        for kernel in ("score_pass1", "score_pass2"):
            assert 0.95 * once < prof[name][kernel] < 1.25 * once
