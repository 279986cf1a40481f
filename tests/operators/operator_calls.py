"""Calls of the operators on their CPU build (operators_build.py), seeded: `python operator_calls.py KIND SEED COUNT`.  Prints each call before it is
made and what came of it; the exit code is 1 when an access was out of range or a result wrong."""
import ctypes
import os
import sys

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, os.path.dirname(os.path.dirname(HERE)))
sys.path.insert(0, HERE)
import paper_2310_16795_amd as q  # noqa: E402
import plain  # noqa: E402

L = q.lib()
L.lanes_alloc.restype, L.lanes_alloc.argtypes = ctypes.c_void_p, [ctypes.c_size_t, ctypes.c_int, ctypes.c_size_t]
L.lanes_reports.restype = ctypes.c_long
SIZE = {q.F32: 4, q.BF16: 2}


class Memory:
    """Device memory of a call: all of it with its end, or all with its start, next to what may not be touched."""

    def __init__(self, at_start):
        self.at_start = at_start

    def new(self, n, align=4, fill=0xFF):
        p = L.lanes_alloc(n, self.at_start, align)
        ctypes.memset(p, fill, n)
        return p

    def put(self, a, align=None):
        if a is None:
            return None
        a = np.ascontiguousarray(a)
        p = L.lanes_alloc(a.nbytes, self.at_start, align or a.dtype.itemsize)
        ctypes.memmove(p, a.ctypes.data, a.nbytes)
        return p

    def rows(self, a, ld, kind):
        """A matrix with ld elements from row to row (nothing behind the last one's values); -> address, its values as stored"""
        n, d = a.shape
        bits = plain.bf16_bits(a) if kind == q.BF16 else a.astype(np.float32)
        flat = np.full((n - 1) * ld + d, 0x7F, dtype=np.uint8).astype(bits.dtype)
        for i in range(n):
            flat[i * ld:i * ld + d] = bits[i]
        return self.put(flat), plain.of_bits(bits) if kind == q.BF16 else bits.astype(np.float64)


def read(p, n, dtype):
    return np.frombuffer((ctypes.c_char * (n * np.dtype(dtype).itemsize)).from_address(p), dtype=dtype).copy()


def read_rows(p, n, d, ld, kind):
    """-> values [n, d], and whether what lies between the rows is untouched"""
    flat = read(p, (n - 1) * ld + d, np.float32 if kind == q.F32 else np.uint16)
    own = np.zeros(flat.size, dtype=bool)
    for i in range(n):
        own[i * ld:i * ld + d] = True
    untouched = bool((flat[~own].view(np.uint8) == 0xFF).all())
    v = flat[own].reshape(n, d)
    return (v.astype(np.float64) if kind == q.F32 else plain.of_bits(v)), untouched


def near(got, want, err, kind, label):
    tol = err + (plain.U32 if kind == q.F32 else plain.U_BF16) * (np.abs(want) + err) + 1e-37
    bad = ~(np.abs(got - want) <= tol)
    if bad.any():
        at = tuple(int(v[0]) for v in np.nonzero(bad))
        print(f"  {label}: {int(bad.sum())} of {bad.size} off, first at {at}: {got[at]} for {want[at]} (+- {tol[at]:.3g})", flush=True)
    return not bad.any()


def norm(rng, i):
    m = Memory(i % 2)
    n, d = int(rng.choice([1, 2, 5, 9])), int(np.exp(rng.uniform(0, np.log(2200)))) if i % 7 else 8200 + i
    k, copies = (int(rng.choice([1, 1, 2, 3])) for _ in range(2))
    ht, yt = int(rng.integers(0, 2)), int(rng.integers(0, 2))
    pad = lambda: d + int(rng.choice([0, 0, 1, 8]))  # noqa: E731
    ld_h, ld_y, ld_o, ld_x = pad(), pad(), pad(), pad()
    h_at, h = m.rows(3 * rng.standard_normal((n, d)), ld_h, ht)
    with_y, with_x, with_out = (rng.random() < 0.85 for _ in range(3))
    with_x = with_x or not with_out
    y_at, y = m.rows(rng.standard_normal((n * k, d)), ld_y, yt) if with_y else (None, None)
    gate = rng.random(n * k).astype(np.float32) if rng.random() < 0.5 else None
    channel = rng.random(d).astype(np.float32) if rng.random() < 0.4 else None
    specs, structs = [], []
    for _ in range(2):
        kind = str(rng.choice(["none", "rms", "layer"]))
        w = (1 + 0.2 * rng.standard_normal(d)).astype(np.float32) if rng.random() < 0.8 else None
        b = (0.1 * rng.standard_normal(d)).astype(np.float32) if rng.random() < 0.5 else None
        specs.append(None if kind == "none" else (kind, w, b, 1e-6))
        structs.append(None if kind == "none" else q.qmoe_norm(0 if kind == "rms" else 1, 1e-6, m.put(w), m.put(b)))
    post, pre = specs
    out_at = m.new(((n - 1) * ld_o + d) * SIZE[ht], SIZE[ht]) if with_out else None
    x_at = m.new(((n * copies - 1) * ld_x + d) * 2, 2) if with_x else None
    print(f"norm {i}: n {n} d {d} k {k} copies {copies} h {ht} y {yt if with_y else None} post {post and post[0]} pre {pre and pre[0]}", flush=True)
    st = L.qmoe_residual_norm(h_at, ht, ld_h, y_at, yt, ld_y, k, m.put(gate), structs[0] and ctypes.byref(structs[0]), 0.5, m.put(channel),
                              structs[1] and ctypes.byref(structs[1]), out_at, ld_o, x_at, ld_x, copies, n, d, None)
    want, err, x_want, x_err = plain.residual_norm(h, y, k, gate if with_y else None, post, 0.5, channel, pre, copies)
    ok = st == 0
    if with_out:
        got, kept = read_rows(out_at, n, d, ld_o, ht)
        ok &= near(got, want, err, ht, "h_out") and kept
    if with_x:
        got, kept = read_rows(x_at, n * copies, d, ld_x, q.BF16)
        ok &= near(got, x_want, x_err, q.BF16, "x") and kept
    return ok


def route(rng, i):
    m = Memory(i % 2)
    n = int(rng.choice([1, 3, 18, 37]))
    e = int(np.exp(rng.uniform(0, np.log(2300)))) if i % 5 else int(rng.choice([1, 64, 65, 256, 512, 2049, 4099, 8200]))
    n = min(n, 4) if e > 1000 else n
    k, lt, chosen = min(e, int(rng.choice([1, 2, 5, 8, 16]))), int(rng.integers(0, 2)), int(rng.integers(0, 2))
    l = 2 * rng.standard_normal((n, e))
    if i % 3 == 0:
        l = np.round(l)  # many equal ones
    if i % 4 == 1:
        l[rng.random((n, e)) < 0.4] = -np.inf
        l[n // 2] = -np.inf
    if i % 8 == 2:
        l[rng.random((n, e)) < 0.2] = np.inf
        l[rng.random((n, e)) < 0.2] = np.nan
        l[0] = np.finfo(np.float32).min if lt == q.F32 else -3.38953138925e38
    with np.errstate(invalid="ignore"):
        at, l = m.rows(l, ld := e + int(rng.choice([0, 0, 3])), lt)
    bias = rng.integers(-256, 257, e).astype(np.float32) / 64 if rng.random() < 0.5 else None
    mask = (rng.random(n) < 0.7).astype(np.uint8) if rng.random() < 0.5 else None
    idx_at, gate_at = m.new(4 * n * k), m.new(4 * n * k)
    print(f"route {i}: n {n} experts {e} k {k} type {lt} chosen {chosen} bias {bias is not None} mask {mask is not None}", flush=True)
    st = L.qmoe_route(at, lt, ld, m.put(bias), m.put(mask), n, e, k, chosen, idx_at, gate_at, None)
    idx, gate, rel = plain.route(l, bias, mask, k, chosen)
    got, g = read(idx_at, n * k, np.int32).reshape(n, k), read(gate_at, n * k, np.float32).reshape(n, k)
    same = np.array_equal(got, idx)
    if not same:
        print("  experts differ:", got[(got != idx).any(axis=1)][:3].tolist(), idx[(got != idx).any(axis=1)][:3].tolist())
    return st == 0 and same and near(g.astype(np.float64), gate, rel * gate, q.F32, "gates")


def weights(rng, rows, cols, group, zeros, whole):
    """whole: scales that are powers of two, so that sums of whole activations are exact"""
    values = rng.integers(0, 16, (rows, cols)).astype(np.uint8)
    groups = (cols + group - 1) // group
    s = 2.0 ** rng.integers(-3, 2, (rows, groups)) if whole else (0.5 + rng.random((rows, groups))) / (2 * np.sqrt(cols))
    zero = rng.integers(0, 16, (rows, groups)).astype(np.uint8) if zeros else None
    packed = plain.int4_pack(values)
    if cols % 128:  # what is stored past the last column must not matter
        other = rng.integers(0, 16, (rows, packed.shape[1] * 2)).astype(np.uint8)
        other[:, :cols] = values
        packed = plain.int4_pack(other)
    return values, packed, s.astype(np.float16).view(np.uint16), zero


def int4_many(rng, i):
    """Rows and tokens enough for the kernels that take 16, 32 or 64 tokens of a matrix at a time."""
    rows, cols = int(rng.integers(200, 700)), int(rng.choice([8, 64, 130, 200, 390]))
    return int4(rng, i, (rows, cols, [20, 40, 70, 66, 130, 97][i % 6]))


def int4(rng, i, sizes=None):
    m = Memory(i % 2)
    act = ["none", "none", "relu", "silu", "gelu"][i % 5]
    rows, cols = int(np.exp(rng.uniform(0, np.log(90)))), int(np.exp(rng.uniform(0, np.log(1100))))
    rows += rows % 2 if act in ("silu", "gelu") else 0
    batch = int(rng.choice([1, 2, 15, 16, 17, 33, 50, 65, 130])) if i % 4 else 1
    if sizes:
        rows, cols, batch = sizes
        rows -= rows % 2
    group, zeros, yt, whole = int(rng.choice([32, 64, 128, 256, 384])), rng.random() < 0.5, int(rng.integers(0, 2)), i % 2 == 0
    values, packed, s, zero = weights(rng, rows, cols, group, zeros, whole)
    results = rows // 2 if act in ("silu", "gelu") else rows
    x = rng.integers(-8, 9, (batch, cols)) if whole else rng.standard_normal((batch, cols))
    ld_x, ld_y = cols + int(rng.choice([0, 0, 1, 8])), results + int(rng.choice([0, 0, 3]))
    x_at, x = m.rows(x, ld_x, q.BF16)
    y_at = m.new(((batch - 1) * ld_y + results) * SIZE[yt], SIZE[yt])
    W = q.qmoe_int4_matrix(m.put(packed, 16), m.put(s), m.put(zero), rows, cols, group, 0)
    print(f"int4 {i}: {rows} x {cols} batch {batch} group {group} zeros {zeros} act {act} y {yt} whole {whole}", flush=True)
    st = L.qmoe_int4_matvec(ctypes.byref(W), x_at, ld_x, batch, q.ACTIVATIONS[act], y_at, yt, ld_y, None)
    want, err = plain.int4_product(x, values, s, zero, group, act)
    got, kept = read_rows(y_at, batch, results, ld_y, yt)
    if whole and act in ("none", "relu"):
        err = np.zeros_like(err)
    return st == 0 and kept and near(got, want, err, yt, "y")


def layer_many(rng, i):
    """Hidden vectors and tokens enough for tiles of 16 or 32 tokens of an expert."""
    return layer(rng, i, (int(rng.choice([1, 2, 4])), int(rng.choice([20, 60, 150])), 8 * int(rng.integers(1, 20)), 8 * int(rng.integers(30, 60))))


def layer(rng, i, sizes=None):
    m = Memory(i % 2)
    act, E, T = ["relu", "silu", "gelu"][i % 3], int(rng.choice([1, 2, 5, 9])), int(np.exp(rng.uniform(0, np.log(150))))
    d_model, d_ff = (8 * int(rng.integers(1, 24)) for _ in range(2))
    if sizes:
        E, T, d_model, d_ff = sizes
    group, yt = int(rng.choice([32, 64, 128])), int(rng.integers(0, 2))
    rows_i = d_ff if act == "relu" else 2 * d_ff
    ex = [[weights(rng, r, c, group, rng.random() < 0.5, False) for r, c in ((rows_i, d_model), (d_model, d_ff))] for _ in range(E)]
    idx = rng.integers(0, E, T).astype(np.int32)
    if T > 5:
        idx[[1, T - 2]], idx[T // 2:T // 2 + T // 3] = (-1, E), 0
    elif T > 1:
        idx[int(rng.integers(0, T))] = int(rng.choice([-1, E]))
    x_at, x = m.rows(rng.standard_normal((T, d_model)), d_model, q.BF16)
    x_at = m.put(plain.bf16_bits(x), 16)
    gate = rng.random(T).astype(np.float32) if i % 2 else None
    descs = [m.put(np.frombuffer(bytes((q.qmoe_int4_matrix * E)(*[
        q.qmoe_int4_matrix(m.put(w[1], 16), m.put(w[2]), m.put(w[3]), *w[0].shape, group, 0) for w in (e[p] for e in ex)])), dtype=np.uint8), 8)
        for p in range(2)]
    y_at, n_ws = m.new(T * d_model * SIZE[yt], 4), q.qmoe_moe_layer_workspace(E, d_model, d_ff, T)
    ws = m.new(n_ws, 256)
    print(f"layer {i}: {E} experts {d_model} x {d_ff}, {T} tokens, group {group} act {act} y {yt}", flush=True)
    st = L.qmoe_int4_layer_forward(*descs, group, q.ACTIVATIONS[act], E, d_model, d_ff, x_at, m.put(idx), m.put(gate), T, y_at, yt, ws, n_ws, None)
    lay = q.qmoe_moe_layer_ws_layout(E, d_model, d_ff, T)
    order = np.argsort(np.where((idx < 0) | (idx >= E), E, idx), kind="stable") if T > 8 else np.arange(T)  # slot -> token (few tokens: as they are)
    hidden = plain.of_bits(read(ws + lay.hidden, T * d_ff, np.uint16)).reshape(T, d_ff)
    y = read_rows(y_at, T, d_model, d_model, yt)[0]
    ok, none = st == 0, (idx < 0) | (idx >= E)
    ok &= not y[none].any()
    for e in range(E):
        slots = np.flatnonzero(idx[order] == e)
        toks = order[slots]
        if not toks.size:
            continue
        (vi, _, si, zi), (vo, _, so, zo) = ex[e]
        want, err = plain.int4_product(x[toks], vi, si, zi, group, act)
        ok &= near(hidden[slots], want, err, q.BF16, f"hidden of expert {e}")
        want, err = plain.int4_product(hidden[slots], vo, so, zo, group, "none")  # from the hidden vectors that were written
        g = np.ones(T) if gate is None else gate.astype(np.float64)
        ok &= near(y[toks], want * g[toks, None], (err + plain.U32 * np.abs(want)) * g[toks, None], yt, f"y of expert {e}")
    return bool(ok)


if __name__ == "__main__":
    kind, seed, count = sys.argv[1], int(sys.argv[2]), int(sys.argv[3])
    rng, ok = np.random.default_rng(seed), True
    for i in range(count):
        before = L.lanes_reports()
        right = {"norm": norm, "route": route, "int4": int4, "int4_many": int4_many, "layer": layer, "layer_many": layer_many}[kind](rng, i)
        out = L.lanes_reports() - before
        ok &= bool(right) and out == 0
        if not right or out:
            print(f"  -> right {bool(right)}, {out} accesses out of range", flush=True)
    print("done" if ok else "failed", flush=True)
    sys.exit(0 if ok else 1)
