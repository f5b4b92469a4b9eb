"""The plans of the decode over a 4-bit cache, as the host makes them (csrc/validate.cpp,
built with g++ beside a driver that prints them): the workspace that a call is checked
against is its own plan's, and what rbq_workspace_bytes gives covers every plan (CPU)."""
import itertools
import os
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FORMS = range(8)      # 1: sparse, 2: with seq_n, 4: with seq_w


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ is not available")
    exe = str(tmp_path_factory.mktemp("plans") / "plans")
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-Werror", os.path.join(ROOT, "paper_2606_31519_amd/csrc/validate.cpp"),
                    os.path.join(ROOT, "tests/plans/decode_kv4_plans.cpp"), "-o", exe], check=True)

    def run(calls):
        text = "".join(" ".join(map(str, c)) + "\n" for c in calls)
        out = subprocess.run([exe], input=text, stdout=subprocess.PIPE, text=True, check=True, timeout=60).stdout
        return np.array([line.split() for line in out.splitlines()], np.int64).reshape(len(calls), -1)

    return run


def shapes():
    """(B, Hq, Hkv, D, n, w): batches from 1 to over 1024 groups, groups of 1 to 16 heads, every window."""
    rng = np.random.default_rng(8)
    fixed = [(1, 32, 8, 128, 0, 0), (1, 32, 8, 128, 130816, 256), (8, 32, 8, 128, 32000, 4096), (16, 32, 8, 128, 32000, 2048),
             (32, 32, 8, 128, 16000, 1024), (43, 32, 8, 128, 8000, 256), (64, 32, 8, 128, 8000, 256), (64, 32, 8, 128, 8000, 0),
             (129, 32, 8, 128, 8000, 0), (129, 32, 8, 64, 8000, 256), (1, 128, 8, 128, 130816, 256), (8, 128, 8, 64, 32000, 256),
             (1, 1, 1, 128, (1 << 24) - 1, 0), (1024, 1, 1, 64, 300, 1), (2000, 8, 8, 64, 40, 4096)]
    for _ in range(600):
        Hkv, G = 2 ** rng.integers(0, 4), 2 ** rng.integers(0, 5)
        fixed.append((int(np.exp(rng.uniform(0, np.log(300)))), int(Hkv * G), int(Hkv), int(rng.choice([64, 128])),
                      int(np.exp(rng.uniform(0, np.log(1e6)))), int(rng.choice([0, rng.integers(1, 4097)]))))
    return fixed


def test_a_call_is_checked_against_its_own_plans_states(plans):
    """Its plan's, or those of the same call over an 8-bit cache, where they are more."""
    calls = [(*s, f) for s, f in itertools.product(shapes(), FORMS)]
    for c, r in zip(calls, plans(calls)):
        if r[6] == 2:    # RBQ_EUNSUPPORTED: a ragged batch of 2^24 blocks and more
            assert c[6] > 1 and c[0] * c[2] * (r[1] + r[2]) >= 1 << 24
            continue
        assert (r[6], r[7]) == (0, 1), (c, r)     # RBQ_OK, RBQ_EINVAL


def test_the_workspace_size_covers_every_plan_and_every_shorter_window(plans):
    from paper_2606_31519_amd import rbq as R
    cases = [(s, w, f) for s in shapes() for w in sorted({0, 1, s[5] // 3, s[5]}) if w <= s[5] for f in FORMS]
    for (s, w, form), r in zip(cases, plans([(*s[:5], w, f) for s, w, f in cases])):
        states = s[0] * s[1] * (r[1] + r[2]) * (s[3] + 2) * 4
        assert states <= R.rbq_workspace_bytes(R.RBQ_OP_DECODE_KV4, *s), (s, w, form, r)
        if form == 1:    # the fused step's
            assert states <= R.rbq_workspace_bytes(R.RBQ_OP_DECODE_STEP_KV4, *s), (s, w, r)


def test_dense_plans_leave_no_part_of_the_gpu_empty(plans):
    """A uniform dense call's blocks of cached rows are no longer than 1 / 0.85 of what the blocks that run at once (4 a
    compute unit, 3 in groups of 16 at D = 128) would take if they shared them evenly, up to the 64 rows that they are
    rounded to, or they are the 8-bit plan's."""
    cases = shapes()
    short = 0
    for c, r in zip(cases, plans([(*c, 0) for c in cases])):
        B, Hq, Hkv, D, n, w = c
        places = 256 * (3 if D == 128 and Hq // Hkv == 16 else 4)
        even = n * B * Hkv / (0.85 * places)
        assert r[0] <= 64 * np.ceil(even / 64) or (r[:3] == r[3:6]).all(), (c, r)
        short += n > 0 and (r[:3] != r[3:6]).any()
        assert n == 0 or (r[1] - 1) * r[0] < n <= r[1] * r[0], (c, r)       # every row is in a split, none of them empty
    assert short > 20     # (plans of their own are among them)


def test_one_round_is_as_many_blocks_as_run_at_once(plans):
    """Waves take turns (a priority that belongs to blocks which start together) in such calls only, those of the window
    counted: not in groups of 16 at D = 128 beyond 768 blocks, nor beyond 1024."""
    cases = shapes()
    rounds = {True: 0, False: 0}
    for c, r in zip(cases, plans([(*c, 0) for c in cases])):
        places = 256 * (3 if c[3] == 128 and c[1] // c[2] == 16 else 4)
        assert bool(r[8]) == (c[0] * c[2] * (r[1] + r[2]) <= places), (c, r)
        rounds[bool(r[8])] += 1
    assert min(rounds.values()) > 20
