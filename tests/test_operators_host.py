"""CPU tests of the operators around the layer: the stored form of four-bit weights, the quantiser, and every refusal (argument
errors are found before anything is enqueued, so no GPU is needed)."""
import ctypes
import os
import sys

import numpy as np
import pytest

import paper_2310_16795_amd as q

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "operators"))
import plain  # noqa: E402

INVALID, BAD_SYMBOL, WORKSPACE, LIMIT = -1, -3, -5, -10


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 31), (2, 128), (5, 129), (4, 391), (7, 1024)])
def test_pack_and_unpack(rows, cols):
    v = np.random.default_rng(cols).integers(0, 16, (rows, cols)).astype(np.uint8)
    packed = q.qmoe_int4_pack_host(v)
    assert packed.shape == (rows, 64 * -(-cols // 128)) and np.array_equal(packed, plain.int4_pack(v))
    assert np.array_equal(q.qmoe_int4_unpack_host(packed, cols), v)


def test_pack_refuses():
    v = np.full((2, 9), 15, dtype=np.uint8)
    v[1, 8] = 16
    with pytest.raises(q.QmoeError) as e:
        q.qmoe_int4_pack_host(v)
    assert e.value.status == BAD_SYMBOL
    L, buf = q.lib(), np.zeros(64, dtype=np.uint8).ctypes.data
    assert L.qmoe_int4_pack_host(None, 1, 1, buf) == L.qmoe_int4_pack_host(buf, 1, 1, None) == INVALID
    assert L.qmoe_int4_pack_host(buf, 0, 1, buf) == L.qmoe_int4_pack_host(buf, 1, 0, buf) == INVALID
    assert L.qmoe_int4_pack_host(buf, (1 << 24) + 1, 1, buf) == L.qmoe_int4_unpack_host(buf, 1, (1 << 20) + 1, buf) == LIMIT
    assert L.qmoe_int4_unpack_host(None, 1, 1, buf) == L.qmoe_int4_unpack_host(buf, 1, 1, None) == INVALID
    assert (q.qmoe_int4_row_bytes(0), q.qmoe_int4_row_bytes(1), q.qmoe_int4_row_bytes(128), q.qmoe_int4_row_bytes(129)) == (0, 64, 64, 128)


@pytest.mark.parametrize("zero", [False, True])
@pytest.mark.parametrize("rows,cols,group", [(1, 1, 32), (6, 200, 64), (3, 300, 128), (2, 130, 256), (4, 97, 32)])
def test_quantizer(rows, cols, group, zero):
    rng = np.random.default_rng(rows * cols)
    w = (rng.standard_normal((rows, cols)) * rng.choice([1e-6, 0.02, 30.0], (rows, 1))).astype(np.float32)
    w[0, :min(cols, 32)] = 0.0  # a group of zeros (or nearly)
    if zero:
        w[-1] = np.abs(w[-1])
    weights, scale, z = q.qmoe_int4_quantize_host(w, group, zero)
    groups = -(-cols // group)
    assert scale.shape == (rows, groups) and (z is None) == (not zero)
    values = q.qmoe_int4_unpack_host(weights, cols).astype(int)
    s = scale.view(np.float16).astype(np.float64)
    for r in range(rows):
        for g in range(groups):
            v = w[r, g * group:(g + 1) * group].astype(np.float64)
            lo, hi = min(0.0, v.min()), max(0.0, v.max())
            want = (hi - lo) / 15 if zero else max(hi, -lo) / 7
            assert s[r, g] == np.float64(np.float16(np.float32(want)))
            zp = int(z[r, g]) if zero else 8
            got = s[r, g] * (values[r, g * group:(g + 1) * group] - zp)
            if s[r, g] == 0:
                assert not got.any()
                continue
            if zero:
                assert zp == min(15, max(0, round(np.float32(-lo) / np.float32(s[r, g]))))
            # inside the grid a value is half a step away at most; its ends and the scale are rounded (2^-11 of 7 or 15 steps; subnormal scales more)
            ends = 15 * max(2.0 ** -11, 2.0 ** -25 / s[r, g]) + 0.5 * zero
            assert np.abs(got - v).max() <= s[r, g] * (0.5 + ends + 1e-5)


def test_quantizer_refuses():
    for bad in (np.nan, np.inf, -np.inf):
        with pytest.raises(q.QmoeError) as e:
            q.qmoe_int4_quantize_host(np.array([[1.0, bad]], dtype=np.float32), 32)
        assert e.value.status == INVALID
    with pytest.raises(q.QmoeError) as e:
        q.qmoe_int4_quantize_host(np.array([[1e7, 0.0]], dtype=np.float32), 32)
    assert e.value.status == LIMIT
    for group in (1, 31, 96, 129):
        with pytest.raises(q.QmoeError) as e:
            q.qmoe_int4_quantize_host(np.ones((1, 4), dtype=np.float32), group)
        assert e.value.status == INVALID


A = 256  # an address that no refused call touches


def _norm(**over):
    a = dict(h=A, h_type=0, ld_h=64, y=A, y_type=0, ld_y=64, k=1, gate=None, post=None, alpha=1.0, channel=None, pre=None, h_out=A, ld_out=64,
             x=A, ld_x=64, copies=1, n=4, d=64)
    a.update(over)
    return q.lib().qmoe_residual_norm(*a.values(), None)


def test_norm_refuses():
    for over in ({"h": None}, {"h_out": None, "x": None}, {"n": 0}, {"n": -1}, {"d": 0}, {"k": 0}, {"copies": 0}, {"h_type": 2}, {"y_type": -1},
                 {"ld_h": 63}, {"ld_y": 63}, {"ld_out": 63}, {"ld_x": 63}, {"ld_out": 65}):
        assert _norm(**over) == INVALID, over
    for kind, eps in ((2, 0.0), (-1, 0.0), (0, -1e-6), (0, float("nan"))):
        bad = ctypes.byref(q.qmoe_norm(kind, eps, None, None))
        assert _norm(pre=bad) == _norm(post=bad) == INVALID
    for over in ({"n": (1 << 20) + 1}, {"d": 32769, "ld_h": 40000, "ld_y": 40000, "ld_out": 40000, "ld_x": 40000}, {"k": 17}, {"copies": 17}):
        assert _norm(**over) == LIMIT, over


def _route(**over):
    a = dict(logits=A, type=0, ld=8, bias=None, mask=None, n=4, e=8, k=2, gates=0, idx=A, gate=A)
    a.update(over)
    return q.lib().qmoe_route(*a.values(), None)


def test_route_refuses():
    for over in ({"logits": None}, {"idx": None}, {"gate": None}, {"type": 2}, {"ld": 7}, {"n": 0}, {"e": 0}, {"k": 0}, {"k": 9}, {"gates": 2},
                 {"gates": -1}):
        assert _route(**over) == INVALID, over
    for over in ({"n": (1 << 20) + 1}, {"e": 16385, "ld": 16385}, {"e": 64, "ld": 64, "k": 17}):
        assert _route(**over) == LIMIT, over


def _int4(W=None, **over):
    w = dict(weights=A, scale=A, zero=None, rows=8, cols=100, group=64, reserved=0)
    w.update(W or {})
    a = dict(W=ctypes.byref(q.qmoe_int4_matrix(*w.values())), x=A, ld_x=100, batch=3, act=0, y=A, y_type=0, ld_y=8)
    a.update(over)
    return q.lib().qmoe_int4_matvec(*a.values(), None)


def test_int4_refuses():
    for W in ({"weights": None}, {"weights": 264}, {"scale": None}, {"rows": 0}, {"cols": 0}, {"group": 0}, {"group": 16}, {"group": 96},
              {"group": -128}, {"reserved": 1}):
        assert _int4(W) == INVALID, W
    assert q.lib().qmoe_int4_matvec(None, A, 100, 3, 0, A, 0, 8, None) == INVALID
    for over in ({"x": None}, {"y": None}, {"batch": 0}, {"act": -1}, {"act": 4}, {"y_type": 2}, {"ld_x": 99}, {"ld_y": 7},
                 {"act": 2, "ld_y": 3}):
        assert _int4(**over) == INVALID, over
    assert _int4({"rows": 7}, act=3) == INVALID
    assert _int4({"rows": (1 << 24) + 1}, ld_y=1 << 25) == _int4({"cols": (1 << 20) + 1}, ld_x=1 << 21) == _int4(batch=(1 << 20) + 1) == LIMIT


def _layer(**over):
    a = dict(wi=A, wo=A, group=64, act=1, e=4, d_model=64, d_ff=128, x=A, idx=A, gate=None, n=10, y=A, y_type=0, ws=A, ws_bytes=1 << 30)
    a.update(over)
    return q.lib().qmoe_int4_layer_forward(*a.values(), None)


def test_int4_layer_refuses():
    for over in ({"wi": None}, {"wo": None}, {"x": None}, {"idx": None}, {"y": None}, {"group": 48}, {"act": 0}, {"act": 4}, {"y_type": 2},
                 {"d_model": 60}, {"d_ff": 4}, {"x": 264}, {"y": 258}, {"e": 0}, {"n": 0}, {"d_model": 0}, {"d_ff": -8}):
        assert _layer(**over) == INVALID, over
    need = q.qmoe_moe_layer_workspace(4, 64, 128, 10)
    for over in ({"ws": None}, {"ws": 128}, {"ws_bytes": need - 32768 - 1}):
        assert _layer(**over) == WORKSPACE, over
    for over in ({"e": 16385}, {"n": (1 << 20) + 1}, {"d_model": 32776}, {"d_ff": 32776}):
        assert _layer(**over) == LIMIT, over


def test_structs_are_those_of_the_header():
    assert ctypes.sizeof(q.qmoe_norm) == 24 and q.qmoe_norm.weight.offset == 8
    assert ctypes.sizeof(q.qmoe_int4_matrix) == 40 and q.qmoe_int4_matrix.rows.offset == 24
