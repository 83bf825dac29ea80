"""A traffic record (profiles/traffic.json) that claims other sources than it was captured on says so, and only host
sources may have changed in between."""
import hashlib
import json
import os

import bench

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HOST = ("capi.cpp", "status.h")  # entry points and launch code: a change here is carried over by hand, with its reason


def kernels_digest():
    """The digest of the bench without the host sources: kernels, their headers, front ends and planner."""
    d = os.path.join(ROOT, "paper_2607_03574_gb300", "csrc")
    h = hashlib.sha256()
    for name in sorted(os.listdir(d)):
        path = os.path.join(d, name)
        if os.path.isfile(path) and name not in HOST:
            h.update(name.encode())
            with open(path, "rb") as f:
                h.update(f.read())
    return h.hexdigest()


def test_record_says_what_it_was_captured_on():
    with open(os.path.join(ROOT, "profiles", "traffic.json")) as f:
        rec = json.load(f)
    if rec["sources_sha256"] != bench.kernel_sources_digest():
        return  # it does not claim these sources: the bench reports no traffic
    assert rec["captured_kernels_sha256"] == kernels_digest(), "a kernel, a front end or the planner changed: capture again"
    if rec["captured_sources_sha256"] != rec["sources_sha256"]:
        assert all(name in rec["carried_over"] for name in HOST)
