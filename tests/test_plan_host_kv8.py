"""CPU tests of the launch plan of suffix attention over the 8-bit cache: the invariants of test_plan_host.py (every
query block meets every key once, split counts that kernel and merge read alike, the workspace the sum of the
partial slots) where the plan is priced for that kernel, with one sequence and several."""

import os
import shutil
import subprocess

import numpy as np
import pytest

from test_plan_host import CSRC, MAX_SPLIT_KEYS, ROOT, _check, _plans, _random_launch


@pytest.fixture(scope="module")
def harness(tmp_path_factory):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    exe = str(tmp_path_factory.mktemp("plan") / "plan_kv8_harness")
    subprocess.run([hipcc, "-x", "hip", "--offload-arch=gfx950", "-std=c++17", "-O1",
                    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-I", CSRC,
                    os.path.join(ROOT, "tests", "plan_kv8_harness.cpp"), "-o", exe],
                   check=True, capture_output=True)
    return exe


def _launch(hq, hkv, d, *seqs):
    """(head_dim 256 has the workgroups of 8 waves that test_plan_host's transposed V has.)"""
    return (hq, hkv, d, d == 256, 0, list(seqs))


def test_plans_of_random_launches(harness):
    r = np.random.default_rng([20397, 93])
    launches = []
    for _ in range(300):
        hq, hkv, d, _, _, seqs = _random_launch(r)
        launches.append(_launch(hq, hkv, d, *seqs))
    for _ in range(300):                                # one sequence, shallow to deep
        d, hkv = int(r.choice([64, 128, 256])), int(r.choice([1, 2, 4, 8, 32]))
        n = int(2 ** r.uniform(0, 11))
        launches.append(_launch(hkv * int(r.choice([1, 2, 5, 8])), hkv, d, (n, int(2 ** r.uniform(0, 16)))))
    for _ in range(60):                                 # several over short contexts
        d, hkv = int(r.choice([64, 128, 256])), int(r.choice([1, 8]))
        launches.append(_launch(hkv * 4, hkv, d, *[(int(r.integers(1, 64)), int(r.integers(0, 150)))
                                                   for _ in range(int(r.integers(2, 9)))]))
    plans = _plans(harness, launches)
    for launch, plan in zip(launches, plans):
        assert plan is not None, launch
        _check(launch, plan)
    for d in (64, 128, 256):
        own = [(x, p) for x, p in zip(launches, plans) if x[2] == d]
        # both orders, and splits and none, with one sequence and several
        assert {p["range_major"] for _, p in own} == {0, 1}
        for several in (False, True):
            assert {p["ws"] > 0 for x, p in own if (len(x[5]) > 1) == several} == {False, True}
        # the two-class cut: one sequence, groups of two split counts
        assert any(len(x[5]) == 1 and len({u[6] for u in p["unit"]}) == 2 for x, p in own), d
    assert _plans(harness, launches[:40]) == plans[:40]


def test_plans_of_long_contexts(harness):
    n = 64 * MAX_SPLIT_KEYS
    launches = [_launch(8, 2, d, (m, p)) for d in (64, 128, 256) for m, p in ((1, 70000), (16, 1000000), (300, n))]
    launches += [_launch(4, 1, 64, (8, n + 100000), (8, n + 50000)), _launch(4, 2, 256, (8, n - 8), (1, 5000)),
                 _launch(4, 2, 256, (64, 0), (1, n), (700, 20))]
    plans = _plans(harness, launches)
    for launch, plan in zip(launches, plans):
        assert plan is not None, launch
        _check(launch, plan)
    assert [p["range_major"] for p in plans[-3:]] == [0, 1, 0]


def test_the_plan_of_several_sequences_does_not_depend_on_their_order(harness):
    """A sequence keeps its cut wherever it stands, a prefill beside suffixes among them."""
    r = np.random.default_rng([20397, 94])
    launches = []
    for _ in range(150):
        seqs = [(int(r.integers(64, 2048)), 0)]
        seqs += [(int(2 ** r.uniform(0, 9)), int(2 ** r.uniform(9, 14))) for _ in range(int(r.integers(1, 6)))]
        hkv = int(r.choice([1, 2, 8]))
        for d in (64, 128, 256):
            launches += [_launch(hkv * 2, hkv, d, *seqs), _launch(hkv * 2, hkv, d, *seqs[::-1])]
    plans = _plans(harness, launches)
    for i in range(0, len(launches), 2):
        cuts = [sorted((s["len"], s["n_past"], u[5], u[6]) for s in p["seqs"] for u in p["unit"] if u[1] == s["b"])
                for p in plans[i:i + 2]]
        assert cuts[0] == cuts[1], launches[i]
        assert plans[i]["ws"] == plans[i + 1]["ws"]
