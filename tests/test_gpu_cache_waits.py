"""Waits of the attention kernels that run out: in the debug build the first
keys of a call never arrive.  The call records DM_ERR_TIMEOUT and ends, and
the next one gives the bits that it gave before.  The calls run in a child
process, which loads the debug library (DM_LIBRARY=debug)."""

import os
import subprocess
import sys

import pytest

from parity_harness import lib_ready

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)

CHILD = r"""
import sys, time
sys.path.insert(0, {root!r})
sys.path.insert(0, {tests!r})
import torch
import cache_reference as R
from paper_2602_06502_gb300 import dualmap as D
assert D.LIB_PATH.endswith("libdualmap_debug.so"), D.LIB_PATH
wait = D.lib().dm_test_attend_wait
for dim, dtype in ((128, torch.bfloat16), (64, torch.float16)):
    for new in ([1, 2, 1, 1], [40, 2, 300, 700], [1, 1, 200, 1]):   # few rows, many, both
        b = R.make_batch(7, page=16, kv_heads=2, dim=dim, dtype=dtype, groups=[2], prefix=(640,), own=[30, 700, 2000, 5], new=new)
        c, T = b["cache"], b["tokens"]
        q = torch.randn(T, 8, dim, generator=b["gen"], device="cuda").to(dtype)
        plan = c.plan(b["seqs"], b["offsets"], T, 8, b["group_offsets"], b["group_prefix"])
        want = c.attend(plan, q)
        assert c.last_error() == 0
        held = c.k.clone(), c.v.clone()
        for _ in range(2):
            assert wait(20_000_000) == D.DM_OK
            t0 = time.perf_counter()
            c.attend(plan, q)
            assert c.last_error() == D.DM_ERR_TIMEOUT
            took = time.perf_counter() - t0
            assert wait(0) == D.DM_OK
            print(dim, new, "%.2f s" % took)
            assert took < {limit}, took
            assert torch.equal(c.attend(plan, q), want) and c.last_error() == 0
        assert all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in zip(held, (c.k, c.v)))
print("waits ran out and the calls after them are right")
"""


def test_waits_that_run_out():
    from paper_2602_06502_gb300 import build as B
    B.build(debug=True)
    env = dict(os.environ, DM_LIBRARY="debug")
    r = subprocess.run([sys.executable, "-c", CHILD.format(root=ROOT, tests=HERE, limit=30)], env=env, capture_output=True,
                       text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-4000:]
    assert "the calls after them are right" in r.stdout
    print(r.stdout)


def test_release_build_has_no_such_waits():
    lib_ready()
    from paper_2602_06502_gb300 import dualmap as D
    assert D.lib().dm_test_attend_wait(1) == D.DM_ERR_INVALID_ARG and D.lib().dm_test_attend_wait(0) == D.DM_OK
