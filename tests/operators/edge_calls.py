"""More calls of the operators on their CPU build: `python edge_calls.py KIND COUNT`, as operator_calls.py does."""
import ctypes
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


if __name__ == "__main__":
    kind, count = sys.argv[1], int(sys.argv[2])
    rng, ok = np.random.default_rng(7), True
    for i in range(count):
        before = L.lanes_reports()
        right = {"outlier": outlier}[kind](rng, i)
        out = L.lanes_reports() - before
        ok &= bool(right) and out == 0
        if not right or out:
            print(f"  -> right {bool(right)}, {out} accesses out of range", flush=True)
    print("done" if ok else "failed", flush=True)
    sys.exit(0 if ok else 1)
