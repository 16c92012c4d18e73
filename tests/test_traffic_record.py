"""The benchmark's record of measured traffic: it names every source that the
kernels of a phase are made of, and was taken with those sources as they are."""
import json
import os
import re

import bench

CSRC = os.path.join(bench.ROOT, "paper_2606_11867_amd", "csrc")
# headers without kernels of the phases or parts of them: conversions and error
# handling, and the fp32 path
OTHERS = {"common.h", "ffn_f32.h"}


def _headers(path):
    """The package's own headers that a source includes, and theirs."""
    got = set()
    for name in re.findall(r'#include "([^"]+)"', open(path).read()):
        if os.path.exists(os.path.join(CSRC, name)) and name not in OTHERS:
            got |= {name} | _headers(os.path.join(CSRC, name))
    return got


def test_sources_of_the_matrix_products_are_named():
    for sources in (bench.ROW_GEMM_SOURCES, bench.DISPATCH_SOURCES):
        named = {os.path.basename(s) for s in sources}
        for s in sources:
            assert _headers(os.path.join(bench.ROOT, s)) <= named, s


def test_record_is_of_these_sources():
    with open(bench.TRAFFIC_RECORD) as f:
        kernels = json.load(f)["kernels"]
    assert set(kernels) == set(bench.PHASES_ORDER)
    by_phase = {}
    for _, phases, sources in bench.PHASE_KERNELS:
        for p in phases:
            by_phase.setdefault(p, set()).update(sources)
    for p in bench.PHASES_ORDER:
        assert set(kernels[p]["sources"]) == by_phase[p]
        assert bench.measured_traffic(p) == kernels[p]["hbm_bytes_per_micro_step"], p
