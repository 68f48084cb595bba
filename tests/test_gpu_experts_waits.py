"""Waits of the product kernel that run out: in the debug build the first weights
of a product never arrive.  The call records DM_ERR_TIMEOUT and ends, and the
next one gives the bits that it gave before.  The calls run in a child process,
which loads the debug library (DM_LIBRARY=debug)."""

import os
import subprocess
import sys

import pytest

from parity_harness import lib_ready

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r"""
import sys, time
sys.path.insert(0, {root!r})
import torch
from paper_2602_06502_gb300 import dualmap as D
from paper_2602_06502_gb300 import experts as X
assert D.LIB_PATH.endswith("libdualmap_debug.so"), D.LIB_PATH
wait = D.lib().dm_test_product_wait
g = torch.Generator(device="cuda").manual_seed(1)
for eight in (False, True):
    for experts, rows, n, k, gated in ((3, [300, 0, 90], 520, 1024, False), (1, [2000], 3000, 256, False), (4, [40, 700, 1, 20], 256, 640, True)):
        real = torch.randn(experts, n, k, generator=g, device="cuda").bfloat16()
        w = X.Weights.quantized(real) if eight else X.Weights(real)
        x, xs = torch.randn(sum(rows), k, generator=g, device="cuda").bfloat16(), None
        if eight:
            x, xs = X.quantize(x)
        off = torch.tensor([0] + rows, device="cuda").cumsum(0).int()
        want = X.product(x, w, off, x_scale=xs, gated=gated)
        assert w.last_error() == 0
        for _ in range(2):
            assert wait(20_000_000) == D.DM_OK
            t0 = time.perf_counter()
            X.product(x, w, off, x_scale=xs, gated=gated)
            assert w.last_error() == D.DM_ERR_TIMEOUT
            took = time.perf_counter() - t0
            assert wait(0) == D.DM_OK
            print(eight, rows, "%.3f s" % took, flush=True)
            assert took < {limit}, took
            assert torch.equal(X.product(x, w, off, x_scale=xs, gated=gated), want) and w.last_error() == 0
print("waits ran out and the calls after them are right")
"""


def test_waits_that_run_out():
    from paper_2602_06502_gb300 import build as B
    B.build(debug=True)
    env = dict(os.environ, DM_LIBRARY="debug")
    r = subprocess.run([sys.executable, "-c", CHILD.format(root=ROOT, limit=30)], env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-4000:]
    assert "the calls after them are right" in r.stdout
    print(r.stdout)


def test_release_build_has_no_such_waits():
    lib_ready()
    from paper_2602_06502_gb300 import dualmap as D
    assert D.lib().dm_test_product_wait(1) == D.DM_ERR_INVALID_ARG and D.lib().dm_test_product_wait(0) == D.DM_OK
