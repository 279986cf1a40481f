"""Edges of the operators around the layer, on the CPU: calls of the checked CPU build of the kernels (tests/operators/edge_calls.py)."""
import os
import subprocess
import sys

import pytest

from test_operators_lanes import library  # noqa: F401

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.parametrize("kind,count,units", [("outlier", 32, 1), ("outlier", 16, 64)])
def test_edge_calls(library, kind, count, units):  # noqa: F811
    cmd = [sys.executable, os.path.join(HERE, "operators", "edge_calls.py"), kind, str(count)]
    r = subprocess.run(cmd, env={**os.environ, "QMOE_LIBRARY": library, "LANES_COMPUTE_UNITS": str(units)}, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600)
    assert r.returncode == 0 and r.stdout.rstrip().endswith("done"), r.stdout[-3000:]
