"""Evictions of one sequence, whose scores have no stride from sequence to sequence that means anything (no GPU: refused before the launch, or by it)."""
import os
import subprocess
import sys

import pytest

OK, INVALID, HIP = 0, 1, 4
TESTS = os.path.dirname(os.path.abspath(__file__))

STRIDES = [(0, 0), (1, 1), (7, 7), (400, 400), (-3, -3), (0, 400)]
# [2][100] scores of 50 rows each, the new ones of 20 rows from `at` on, `step` from head to head: what is to come of it
OVERLAP = [(4, 100), (49, 100), (100, 100), (149, 100), (-19, 100), (49, 120)]
BESIDE = [(50, 100), (60, 100), (80, 100), (200, 100), (200, 20), (0, 100)]

# in a process of its own, which a division by zero in the library would end; no device: what is not refused must not reach one with these addresses
CALLS = """
import sys
sys.path[:0] = [{tests!r}, {root!r}]
from paper_2412_20105_amd import binding as st3
from test_block_host import FAKE, cache, shape
for sb, tb, at, step in {cases}:
    print(sb, tb, at, step, st3.lib().st3_block_evict(shape(batch=1), cache(), cache(k_tail=1 << 40, v_tail=1 << 41), 50, 20, 0, 0, FAKE, sb, 100,
                                                      FAKE + 4 * at, tb, step, 1 << 42, 20, 20, None), flush=True)
"""


@pytest.mark.parametrize("which", ["overlap", "beside"])
def test_scores_of_one_sequence(which):
    """Scores that overlap are refused whatever the stride of sequences is; those between the rows of old ones, behind them, or rows on rows are not."""
    cases = [(sb, tb, at, step) for sb, tb in STRIDES for at, step in (OVERLAP if which == "overlap" else BESIDE)]
    r = subprocess.run([sys.executable, "-c", CALLS.format(tests=TESTS, root=os.path.dirname(TESTS), cases=cases)], capture_output=True, text=True,
                       env=dict(os.environ, HIP_VISIBLE_DEVICES="-1"))
    got = {tuple(map(int, line.split()[:4])): int(line.split()[4]) for line in r.stdout.splitlines() if len(line.split()) == 5}
    assert r.returncode == 0 and set(got) == set(cases), (r.returncode, sorted(set(cases) - set(got))[:3], r.stderr[-500:])
    wrong = [c for c in cases if got[c] not in ((INVALID,) if which == "overlap" else (OK, HIP))]
    assert not wrong
