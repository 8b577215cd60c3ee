"""Decode over blocks: where the output may lie beside the queries (no GPU: refused before the launch, or by it)."""
import os
import subprocess
import sys

import pytest

OK, INVALID, HIP = 0, 1, 4
TESTS = os.path.dirname(os.path.abspath(__file__))

# in a process that sees no device: what is not refused must not reach one with these addresses
CALLS = """
import sys
sys.path[:0] = [{tests!r}, {root!r}]
from paper_2412_20105_amd import binding as st3
from test_block_host import FAKE, cache, rows, shape
FAR = FAKE + (1 << 30)
for q, at, out, more in {cases}:
    print(st3.lib().st3_block_decode(shape(**more), rows(FAKE, *q), rows(FAR, 1024, 128), rows(2 * FAR, 1024, 128), cache(), 50, rows(FAKE + 2 * at, *out), None, 0, 0,
                                     FAKE, 1 << 30, None), flush=True)
"""

# strides of the queries, where the output begins (elements behind the queries), its strides, the shape's differences
REFUSED = [((1024, 128), 4 * 128, (1024, 128), {}), ((1024, 128), -128, (1024, 128), {}), ((1024, 128), 1024, (1024, 128), {}), ((1024, 128), 8, (1024, 128), {}),
           ((1024, 128), 0, (2048, 128), {}), ((2048, 128), 0, (2048, 256), {}), ((2048, 128), 1016, (2048, 128), {}), ((1024, 128), 0, (1024, 256), {"batch": 1}),
           ((1024, 128), 128, (1024, 128), {"batch": 1})]
TAKEN = [((1024, 128), 0, (1024, 128), {}),                                                    # the queries, row for row
         ((2048, 128), 1024, (2048, 128), {}), ((2048, 256), 128, (2048, 256), {}),            # slices of one buffer that alternate
         ((1024, 128), 0, (4096, 128), {"batch": 1}), ((1024, 128), 0, (1024, 512), {"heads": 1, "kv_heads": 1}), ((1024, 128), 1 << 20, (2048, 256), {})]


@pytest.mark.parametrize("cases,want", [(REFUSED, (INVALID,)), (TAKEN, (OK, HIP))], ids=["refused", "taken"])
def test_outputs_on_the_queries(cases, want):
    r = subprocess.run([sys.executable, "-c", CALLS.format(tests=TESTS, root=os.path.dirname(TESTS), cases=cases)], capture_output=True, text=True,
                       env=dict(os.environ, HIP_VISIBLE_DEVICES="-1"))
    assert r.returncode == 0, (r.returncode, r.stderr[-500:])
    got = [int(x) for x in r.stdout.split()]
    assert len(got) == len(cases) and not [(c, g) for c, g in zip(cases, got) if g not in want]
