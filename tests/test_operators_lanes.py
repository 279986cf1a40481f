"""The operators around the layer in a CPU build of their kernels that checks every access (tests/operators, tests/lanes), against
their formulas in 64 bits: odd sizes, strides, types, masks, groups and token counts, with memory that ends, or begins, where the
arguments say."""
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def library(tmp_path_factory):
    import importlib.util

    spec = importlib.util.spec_from_file_location("operators_build", os.path.join(HERE, "operators", "operators_build.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod.build(str(tmp_path_factory.mktemp("operators")))


# on a GPU of so many compute units: few make a call one of much work
@pytest.mark.parametrize("kind,count,units", [("norm", 60, 6), ("route", 60, 6), ("int4", 60, 6), ("int4_many", 36, 1), ("int4_many", 30, 6), ("layer", 30, 6),
                                              ("layer_many", 18, 3)])
def test_results_and_every_access(library, kind, count, units):
    cmd = [sys.executable, os.path.join(HERE, "operators", "operator_calls.py"), kind, "1", str(count)]
    r = subprocess.run(cmd, env={**os.environ, "QMOE_LIBRARY": library, "LANES_COMPUTE_UNITS": str(units)}, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600)
    assert r.returncode == 0 and r.stdout.rstrip().endswith("done"), r.stdout[-3000:]
