"""More calls of the operators on their CPU build: `python edge_calls.py KIND COUNT`, as operator_calls.py does."""
import ctypes
import os
import sys

import numpy as np

import operator_calls as calls
import plain
import plain_exact
from operator_calls import L, q

SHAPES = [(30, 300, 3), (300, 200, 20), (300, 200, 40), (520, 390, 97)]  # rows, cols, batch: any kernel, on a GPU of few compute units


def outlier(rng, i):
    """One activation of a token is far larger than the others, in a column whose weights are 0 in every row: it takes no part in the result."""
    m = calls.Memory(i % 2)
    rows, cols, batch = SHAPES[i // 2 % len(SHAPES)]
    act, zeros, group, large = ["none", "silu"][i % 2], i % 4 < 2, [32, 64, 128, 256][i // 8 % 4], [1e4, 3e38][i // 2 % 2]
    values, _, s, zero = calls.weights(rng, rows, cols, group, zeros, False)
    at = rng.integers(0, cols, batch)
    x = rng.standard_normal((batch, cols))
    for t, c in enumerate(at):
        values[:, c] = 8 if zero is None else zero[:, c // group]
        x[t, c] = large * (-1) ** t
    x_at, x = m.rows(x, cols, q.BF16)
    results = rows // 2 if act == "silu" else rows
    y_at = m.new(4 * batch * results)
    W = q.qmoe_int4_matrix(m.put(plain.int4_pack(values), 16), m.put(s), m.put(zero), rows, cols, group, 0)
    print(f"outlier {i}: {rows} x {cols} batch {batch} group {group} zeros {zeros} act {act} of {large}", flush=True)
    st = L.qmoe_int4_matvec(ctypes.byref(W), x_at, cols, batch, q.ACTIVATIONS[act], y_at, q.F32, results, None)
    want, err = plain_exact.int4_product(x, values, s, zero, group, act)
    return st == 0 and calls.near(calls.read_rows(y_at, batch, results, results, q.F32)[0], want, err, q.F32, "y")


UNITS = int(os.environ.get("LANES_COMPUTE_UNITS", "256"))


def wide(rng, i):
    """More groups than a kernel holds at a time."""
    batch = [33, 40, 70, 130][i % 4]
    act, group = ["none", "silu"][i // 4 % 2], [32, 128][i // 8 % 2]
    rows, cols = 2 * int(rng.integers(100, 140)), int(rng.integers(33, 37)) * group
    print(f"wide {i}: {q.qmoe_hook_int4_kernel(rows, cols, group, q.ACTIVATIONS[act], batch, UNITS)}", flush=True)
    return one_product(rng, calls.Memory(i % 2), rows, cols, batch, group, i % 3 > 0, act)


def one_product(rng, m, rows, cols, batch, group, zeros, act):
    values, packed, s, zero = calls.weights(rng, rows, cols, group, zeros, False)
    x_at, x = m.rows(rng.standard_normal((batch, cols)), cols, q.BF16)
    results = rows // 2 if act == "silu" else rows
    y_at = m.new(4 * batch * results)
    W = q.qmoe_int4_matrix(m.put(packed, 16), m.put(s), m.put(zero), rows, cols, group, 0)
    st = L.qmoe_int4_matvec(ctypes.byref(W), x_at, cols, batch, q.ACTIVATIONS[act], y_at, q.F32, results, None)
    want, err = plain_exact.int4_product(x, values, s, zero, group, act)
    return st == 0 and calls.near(calls.read_rows(y_at, batch, results, results, q.F32)[0], want, err, q.F32, "y")


class _Groups:
    """A generator whose draws of a layer's group are of several blocks."""

    def __init__(self, rng, group):
        self.rng, self.group = rng, group

    def choice(self, of, *args):
        return self.group if list(of) == [32, 64, 128] else self.rng.choice(of, *args)

    def __getattr__(self, name):
        return getattr(self.rng, name)


def layer_groups(rng, i):
    """Layer calls with groups of several blocks."""
    sizes = (int(rng.choice([1, 3])), [5, 9, 40, 130][i % 4], 8 * int(rng.integers(20, 70)), 8 * int(rng.integers(20, 70)))
    return calls.layer(_Groups(rng, [256, 384, 512, 1152][i // 4 % 4]), i, sizes)


def layer_few(rng, i):
    """Up to eight tokens, many on one expert."""
    return calls.layer(rng, i, (int(rng.choice([1, 2, 3])), i % 8 + 1, 8 * int(rng.integers(1, 40)), 8 * int(rng.integers(1, 40))))


if __name__ == "__main__":
    kind, count = sys.argv[1], int(sys.argv[2])
    rng, ok = np.random.default_rng(7), True
    for i in range(count):
        before = L.lanes_reports()
        right = {"outlier": outlier, "wide": wide, "layer_groups": layer_groups, "layer_few": layer_few}[kind](rng, i)
        out = L.lanes_reports() - before
        ok &= bool(right) and out == 0
        if not right or out:
            print(f"  -> right {bool(right)}, {out} accesses out of range", flush=True)
    print("done" if ok else "failed", flush=True)
    sys.exit(0 if ok else 1)
