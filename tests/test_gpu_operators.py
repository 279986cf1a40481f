"""The operators around the layer on the GPU, against their formulas in 64 bits (tests/operators/plain.py).

Where activations are whole numbers and scales powers of two every sum is exact in fp32 and results must be equal; elsewhere
the tolerance is a number of fp32 roundings of the terms that are added up, and half a step of the result's type."""
import os
import sys

import numpy as np
import pytest
import torch

import paper_2310_16795_amd as q
from paper_2310_16795_amd import device as dev

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "operators"))
import plain  # noqa: E402

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("the GPU tests need a GPU: the HIP path has no fallback")
    return "cuda:0"


def _up(a, gpu, kind="f32", pad=0):
    """A host matrix as a device tensor of that type, `pad` elements between its rows; -> tensor, its values in 64 bits"""
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(DTYPES[kind])
    if pad:
        held = torch.full((t.shape[0], t.shape[1] + pad), 7.0, dtype=t.dtype, device=gpu)
        held[:, :t.shape[1]] = t.to(gpu)
        d = held[:, :t.shape[1]]
    else:
        d = t.to(gpu)
    return d, t.double().numpy()


def _out(n, d, gpu, kind, pad=0, behind=2):
    """An output filled with a sign, rows and columns around it: (tensor, all that it lies in)"""
    held = torch.full((n + behind, d + pad), -77.0, dtype=DTYPES[kind], device=gpu)
    return held[:n, :d], held


def _near(got, want, err, kind, label=""):
    got = got.double().cpu().numpy()
    tol = err + (plain.U32 if kind == "f32" else plain.U_BF16) * (np.abs(want) + err) + 1e-37
    ok = np.abs(got - want) <= tol
    ok |= np.isnan(got) & np.isnan(want)
    assert ok.all(), f"{label}: {(~ok).sum()} of {ok.size} off, worst {np.nanmax(np.abs(got - want) / tol):.3g} x the tolerance"


def _untouched(held, n, d):
    h = held.float().cpu().numpy().copy()
    h[:n, :d] = -77.0
    assert (h == -77.0).all()


# ---------------------------------------------------------------- residual stream and norm

NORMS = [  # tokens, d, k, copies, h, y, post, pre, padding between rows
    (1, 768, 1, 1, "f32", "f32", None, "rms", 0), (1, 1, 1, 1, "bf16", "bf16", "layer", "rms", 0), (3, 7, 2, 3, "f32", "bf16", "rms", "layer", 1),
    (65, 2080, 2, 2, "bf16", "f32", None, "rms", 0), (130, 513, 1, 1, "f32", "f32", "layer", "layer", 3), (7, 4099, 4, 1, "bf16", "bf16", "rms", "rms", 5),
    (5, 8193, 1, 2, "f32", "bf16", "layer", "rms", 0), (2, 32768, 16, 16, "bf16", "f32", "rms", "layer", 0), (2100, 1024, 1, 1, "f32", "bf16", "layer", "layer", 0),
    (40, 6144, 2, 1, "f32", "f32", None, None, 8), (1030, 256, 1, 1, "bf16", "bf16", None, "layer", 0), (3, 32767, 1, 1, "f32", "f32", None, "rms", 0),
]


@pytest.mark.parametrize("n,d,k,copies,ht,yt,post,pre,pad", NORMS)
def test_residual_norm(gpu, n, d, k, copies, ht, yt, post, pre, pad):
    rng = np.random.default_rng(n * 7 + d)
    h, h64 = _up(3 * rng.standard_normal((n, d)), gpu, ht, pad)
    y, y64 = _up(rng.standard_normal((n * k, d)), gpu, yt, 2 * pad)
    gate = rng.random(n * k).astype(np.float32) if k > 1 else None
    channel = (0.1 + rng.random(d)).astype(np.float32) if n % 2 else None
    spec, norms = [], []
    for kind in (post, pre):
        w = (1 + 0.2 * rng.standard_normal(d)).astype(np.float32) if d % 3 else None
        b = (0.1 * rng.standard_normal(d)).astype(np.float32) if kind == "layer" else None
        spec.append(None if kind is None else (kind, w, b, 1e-6))
        norms.append(None if kind is None else dev.DeviceNorm(kind, *(None if v is None else torch.from_numpy(v).to(gpu) for v in (w, b)), eps=1e-6))
    up = lambda v: None if v is None else torch.from_numpy(v).to(gpu)  # noqa: E731
    h_out, held_h = _out(n, d, gpu, ht, pad)
    x, held_x = _out(n * copies, d, gpu, "bf16", pad)
    q.qmoe_residual_norm(h, y, h_out, x, k=k, gate=up(gate), post=norms[0], alpha=0.75, channel_scale=up(channel), pre=norms[1], copies=copies)
    torch.cuda.synchronize()
    want, err, x_want, x_err = plain.residual_norm(h64, y64, k, gate, spec[0], 0.75, channel, spec[1], copies)
    _near(h_out, want, err, ht, "h_out")
    _near(x, x_want, x_err, "bf16", "x")
    _untouched(held_h, n, d)
    _untouched(held_x, n * copies, d)
    # in place, and each output alone, give the same bits
    h_in, x_alone = h.clone(), torch.empty_like(x)
    q.qmoe_residual_norm(h_in, y, h_in, None, k=k, gate=up(gate), post=norms[0], alpha=0.75, channel_scale=up(channel))
    q.qmoe_residual_norm(h, y, None, x_alone, k=k, gate=up(gate), post=norms[0], alpha=0.75, channel_scale=up(channel), pre=norms[1], copies=copies)
    assert torch.equal(h_in, h_out) and torch.equal(x_alone, x)


def test_norm_alone_and_tokens_that_are_not_finite(gpu):
    rng = np.random.default_rng(5)
    h = torch.from_numpy(rng.standard_normal((9, 300)).astype(np.float32)).to(gpu)
    h[2, 7], h[5, 299], h[7] = float("nan"), float("inf"), 0.0
    x = torch.empty((9, 300), dtype=torch.bfloat16, device=gpu)
    for kind in ("rms", "layer"):
        q.qmoe_residual_norm(h, x=x, pre=dev.DeviceNorm(kind, eps=1e-5))
        want, err, x_want, x_err = plain.residual_norm(h.cpu().numpy().astype(np.float64), None, 1, None, None, 1.0, None, (kind, None, None, 1e-5), 1)
        keep = [0, 1, 3, 4, 6, 7, 8]
        _near(x[keep], x_want[keep], x_err[keep], "bf16", kind)
        assert not x[7].any() and x[2].isnan().all() and x[5].isnan().any()
    # a gate of zero on the rows that dropped tokens left, all zero; a row that is all one value (its variance is zero)
    y = torch.zeros((18, 300), device=gpu)
    out = torch.empty_like(h)
    q.qmoe_residual_norm(h, y, out, None, k=2, gate=torch.zeros(18, device=gpu))
    assert torch.equal(out[[0, 1, 3]], h[[0, 1, 3]])
    ones = torch.full((2, 300), 3.0, device=gpu)
    q.qmoe_residual_norm(ones, x=x[:2], pre=dev.DeviceNorm("layer", eps=1e-6))
    assert x[:2].abs().max() < 2e-3  # (3 less its mean, which is rounded: 64 * 2^-24 * 3 over sqrt(eps) at most)


# ---------------------------------------------------------------- the router's choice

ROUTES = [  # tokens, experts, k, logits, chosen, bias, masked share, padding, kind of logits
    (1, 128, 1, "f32", 0, False, 0.0, 0, "normal"), (1, 1, 1, "bf16", 1, True, 0.0, 0, "normal"), (17, 2, 2, "f32", 0, True, 0.3, 1, "normal"),
    (333, 64, 6, "bf16", 1, True, 0.1, 0, "normal"), (70, 65, 8, "f32", 1, False, 0.0, 3, "equal"), (129, 256, 16, "bf16", 0, False, 0.5, 0, "equal"),
    (64, 257, 4, "f32", 0, True, 0.0, 0, "masked"), (31, 512, 2, "bf16", 1, False, 0.2, 5, "masked"), (40, 1000, 8, "f32", 1, True, 0.0, 0, "special"),
    (50, 2048, 1, "f32", 0, False, 0.0, 0, "normal"), (9, 2049, 5, "bf16", 0, True, 0.2, 1, "equal"), (6, 16384, 16, "f32", 1, False, 0.0, 0, "special"),
    (1025, 8, 2, "f32", 1, False, 0.0, 0, "lowest"), (8, 7, 7, "bf16", 0, True, 0.0, 0, "special"),
    (20, 4096, 8, "f32", 0, True, 0.1, 0, "equal"), (7, 4099, 16, "bf16", 0, True, 0.0, 1, "masked"), (5, 8192, 8, "bf16", 1, False, 0.3, 0, "lowest"),
    (6, 8193, 3, "f32", 0, True, 0.0, 2, "special"), (4, 16383, 16, "bf16", 0, False, 0.0, 0, "equal"),
]


def _logits(rng, n, e, kind):
    l = 2 * rng.standard_normal((n, e))
    if kind == "equal":
        l = np.round(l)
    if kind == "masked":
        l[rng.random((n, e)) < 0.6] = -np.inf
        l[n // 2] = -np.inf
        l[n // 3, 1:] = -np.inf
    if kind == "special":
        l[rng.random((n, e)) < 0.1] = np.inf
        l[rng.random((n, e)) < 0.2] = np.nan
        l[0] = np.nan
    if kind == "lowest":
        l[:, e // 2:] = -3.38953138925e38  # bf16's lowest value: very unlikely, not masked
        l[1] = -3.38953138925e38
    return l


@pytest.mark.parametrize("n,e,k,lt,chosen,bias,masked,pad,kind", ROUTES)
def test_route(gpu, n, e, k, lt, chosen, bias, masked, pad, kind):
    rng = np.random.default_rng(n + 3 * e)
    l, l64 = _up(_logits(rng, n, e, kind), gpu, lt, pad)
    b = rng.integers(-256, 257, e).astype(np.float32) / 64 if bias else None
    mask = (rng.random(n) >= masked) if masked else None
    idx = torch.full((n + 1, k), 99, dtype=torch.int32, device=gpu)
    gate = torch.full((n + 1, k), -77.0, device=gpu)
    up = lambda v: None if v is None else torch.from_numpy(v).to(gpu)  # noqa: E731
    q.qmoe_route(l, idx[:n], gate[:n], bias=up(b), token_mask=up(mask), gates=q.GATES_CHOSEN if chosen else q.GATES_ALL)
    torch.cuda.synchronize()
    want, g, rel = plain.route(l64.astype(np.float32), b, mask, k, chosen)
    assert np.array_equal(idx[:n].cpu().numpy(), want)
    _near(gate[:n], g, rel * g, "f32", "gates")
    assert (idx[n] == 99).all() and (gate[n] == -77.0).all()


# ---------------------------------------------------------------- four-bit weights

def _weights(rng, rows, cols, group, zeros, whole):
    values = rng.integers(0, 16, (rows, cols)).astype(np.uint8)
    groups = -(-cols // group)
    s = 2.0 ** rng.integers(-3, 2, (rows, groups)) if whole else (0.5 + rng.random((rows, groups))) / (2 * np.sqrt(cols))
    zero = rng.integers(0, 16, (rows, groups)).astype(np.uint8) if zeros else None
    held = np.random.default_rng(1).integers(0, 16, (rows, -(-cols // 128) * 128)).astype(np.uint8)  # past the last column: anything
    held[:, :cols] = values
    return values, q.qmoe_int4_pack_host(held), s.astype(np.float16).view(np.uint16), zero


def _matrix(gpu, w, cols, group):
    _, packed, s, z = w
    return dev.DeviceInt4Matrix(torch.from_numpy(packed).to(gpu), torch.from_numpy(s.view(np.int16)).to(gpu), cols, group,
                                None if z is None else torch.from_numpy(z).to(gpu))


INT4 = [  # rows, cols, batch, group, zeros, activation, y, padding
    (4096, 1024, 1, 128, False, "none", "f32", 0), (1, 1, 1, 32, True, "none", "bf16", 0), (17, 33, 3, 32, True, "relu", "f32", 1), (2, 129, 16, 64, False, "silu", "bf16", 0),
    (50, 391, 17, 64, True, "gelu", "f32", 3), (2080, 6144, 37, 64, True, "none", "f32", 0), (96, 2080, 64, 128, False, "relu", "bf16", 8), (130, 1000, 65, 256, True, "none", "f32", 0),
    (258, 777, 129, 384, False, "silu", "bf16", 1), (512, 2080, 300, 128, False, "none", "f32", 0), (640, 512, 513, 32, True, "gelu", "bf16", 0), (1024, 768, 1000, 128, True, "none", "bf16", 0),
    (31, 20000, 2, 128, False, "none", "f32", 0), (260, 130, 2000, 64, False, "none", "f32", 5), (40000, 64, 2, 64, False, "none", "f32", 0), (12, 256, 4100, 128, True, "none", "f32", 0),
]


@pytest.mark.parametrize("whole", [True, False])
@pytest.mark.parametrize("rows,cols,batch,group,zeros,act,yt,pad", INT4)
def test_int4_matvec(gpu, rows, cols, batch, group, zeros, act, yt, pad, whole):
    rng = np.random.default_rng(rows + cols + batch)
    w = _weights(rng, rows, cols, group, zeros, whole)
    results = rows // 2 if act in ("silu", "gelu") else rows
    x, x64 = _up(rng.integers(-8, 9, (batch, cols)) if whole else rng.standard_normal((batch, cols)), gpu, "bf16", pad)
    y, held = _out(batch, results, gpu, yt, pad)
    q.qmoe_int4_matvec(_matrix(gpu, w, cols, group).desc, x, y, activation=q.ACTIVATIONS[act])
    torch.cuda.synchronize()
    want, err = plain.int4_product(x64, w[0], w[2], w[3], group, act)
    _near(y, want, 0 * err if whole and act in ("none", "relu") else err, yt)
    _untouched(held, batch, results)
    if not whole and yt == "f32":  # roundings do not all go one way: as a whole far closer than the bound on each
        d = y.double().cpu().numpy() - want
        assert np.linalg.norm(d) <= 2e-6 * np.linalg.norm(want) + 1e-30


INT4_MANY = [  # rows, cols, batch, group, zeros, activation, y: enough work for the kernels of 16, 32 and 64 tokens a tile
    *((12000, 600, batch, group, zeros, act, yt) for batch in (33, 300) for group, zeros, act, yt in (
        (128, True, "none", "f32"), (64, False, "gelu", "bf16"), (32, True, "silu", "f32"), (32, False, "relu", "bf16"), (256, True, "none", "bf16"))),
    *((1601, 200, 3601, group, zeros, "none", "f32") for group in (32, 64, 128) for zeros in (False, True)),
    *((3202, 330, 3590, group, zeros, act, yt) for group, act, yt in ((32, "silu", "f32"), (64, "gelu", "bf16"), (256, "silu", "f32")) for zeros in (False, True)),
]


@pytest.mark.parametrize("rows,cols,batch,group,zeros,act,yt", INT4_MANY)
def test_int4_matvec_of_much_work(gpu, rows, cols, batch, group, zeros, act, yt):
    test_int4_matvec(gpu, rows, cols, batch, group, zeros, act, yt, 0, act in ("none", "relu"))


@pytest.mark.parametrize("batch", [3, 40, 200])
def test_int4_tokens_that_are_not_finite(gpu, batch):
    rng = np.random.default_rng(batch)
    w = _weights(rng, 200, 300, 64, True, True)
    x = rng.integers(-8, 9, (batch, 300)).astype(np.float32)
    x[1, 5], x[batch - 1, 299] = np.inf, np.nan
    xd, _ = _up(x, gpu, "bf16")
    y = torch.empty((batch, 200), device=gpu)
    q.qmoe_int4_matvec(_matrix(gpu, w, 300, 64).desc, xd, y)
    keep = [t for t in range(batch) if t not in (1, batch - 1)]
    want, err = plain.int4_product(x[keep].astype(np.float64), w[0], w[2], w[3], 64, "none")
    _near(y[keep], want, 0 * err, "f32")
    assert not y[1].isfinite().any() and y[batch - 1].isnan().all()


LAYERS = [  # experts, d_model, d_ff, tokens, group, zeros, activation, y, gate, routing
    (1, 8, 8, 1, 32, False, "relu", "f32", False, "uniform"), (5, 72, 40, 4, 32, True, "silu", "bf16", True, "crowded"), (6, 200, 64, 5, 64, False, "gelu", "f32", True, "crowded"), (5, 264, 136, 1, 64, True, "silu", "bf16", True, "uniform"),
    (12, 256, 520, 40, 128, False, "relu", "f32", True, "uniform"), (7, 136, 264, 300, 32, True, "gelu", "bf16", False, "crowded"),
    (3, 512, 384, 700, 128, True, "silu", "f32", True, "crowded"), (64, 128, 256, 64, 64, False, "relu", "bf16", True, "uniform"),
    (4, 768, 640, 1500, 128, False, "relu", "bf16", True, "uniform"), (9, 72, 88, 33, 64, False, "relu", "f32", False, "none"),
    (2000, 64, 64, 100, 32, True, "relu", "f32", True, "uniform"), (3, 264, 392, 8, 128, True, "gelu", "f32", True, "crowded"), (3, 264, 392, 9, 128, True, "gelu", "f32", True, "crowded"),
    (40, 128, 72, 8, 64, False, "relu", "bf16", False, "uniform"), (40, 128, 72, 9, 64, False, "relu", "bf16", False, "none"), (2, 64, 64, 8, 32, False, "silu", "bf16", True, "none"),
]


def _layer(gpu, rng, E, d_model, d_ff, group, zeros, act):
    rows_i = d_ff if act == "relu" else 2 * d_ff
    ex = [[_weights(rng, r, c, group, zeros, False) for r, c in ((rows_i, d_model), (d_model, d_ff))] for _ in range(E)]
    stacked = []
    for p in range(2):
        stacked.append((torch.from_numpy(np.stack([e[p][1] for e in ex])).to(gpu), torch.from_numpy(np.stack([e[p][2] for e in ex]).view(np.int16)).to(gpu),
                        torch.from_numpy(np.stack([e[p][3] for e in ex])).to(gpu) if zeros else None))
    return ex, dev.DeviceInt4Layer(*stacked, d_model, d_ff, group, act)


def _check_layer(ex, x64, idx, gate, group, act, yt, y, ws, d_model, d_ff):
    """Each expert's hidden vectors as the workspace holds them, and the results from those (a value next to a rounding border
    may go either way in the first product; the second is held to what the first wrote)."""
    E, T = len(ex), idx.size
    order = np.argsort(np.where((idx < 0) | (idx >= E), E, idx), kind="stable") if T > 8 else np.arange(T)  # slot -> token (few tokens: as they are)
    lay = q.qmoe_moe_layer_ws_layout(E, d_model, d_ff, T)
    hidden = plain.of_bits(ws.cpu().numpy()[lay.hidden:lay.hidden + 2 * T * d_ff].view(np.uint16)).reshape(T, d_ff)
    none = (idx < 0) | (idx >= E)
    assert not y[torch.from_numpy(none)].any()
    for e in range(E):
        slots = np.flatnonzero(idx[order] == e)
        toks = order[slots]
        if not toks.size:
            continue
        (vi, _, si, zi), (vo, _, so, zo) = ex[e]
        want, err = plain.int4_product(x64[toks], vi, si, zi, group, act)
        _near(torch.from_numpy(hidden[slots]), want, err, "bf16", f"hidden of expert {e}")
        want, err = plain.int4_product(hidden[slots], vo, so, zo, group, "none")
        g = np.ones((toks.size, 1)) if gate is None else gate[toks].astype(np.float64)[:, None]
        _near(y[torch.from_numpy(toks).long()], want * g, (err + plain.U32 * np.abs(want)) * g, yt, f"y of expert {e}")


@pytest.mark.parametrize("E,d_model,d_ff,T,group,zeros,act,yt,gated,routing", LAYERS)
def test_int4_layer(gpu, E, d_model, d_ff, T, group, zeros, act, yt, gated, routing):
    rng = np.random.default_rng(E + T)
    ex, layer = _layer(gpu, rng, E, d_model, d_ff, group, zeros, act)
    idx = rng.integers(0, E, T).astype(np.int32)
    if routing == "crowded":
        idx[: T // 2], idx[[min(3, T - 2), T - 1]] = E - 1, (-1, E)
    if routing == "none":
        idx[:] = -1
    gate = rng.random(T).astype(np.float32) if gated else None
    x, x64 = _up(rng.standard_normal((T, d_model)), gpu, "bf16")
    y, held = _out(T, d_model, gpu, yt)
    ws = layer.workspace(T)
    layer.forward(x, torch.from_numpy(idx).to(gpu), y, ws, None if gate is None else torch.from_numpy(gate).to(gpu))
    torch.cuda.synchronize()
    _check_layer(ex, x64, idx, gate, group, act, yt, y.cpu(), ws, d_model, d_ff)
    _untouched(held, T, d_model)


# ---------------------------------------------------------------- together

def _block(gpu, rng, T, E, d_model, d_ff, k):
    """A block's step as a user's program runs it: norm with k copies, logits, choice, experts, and the stream takes their rows."""
    ex, layer = _layer(gpu, rng, E, d_model, d_ff, 128, False, "relu")
    router = _weights(rng, E, d_model, 128, False, False)
    R = _matrix(gpu, router, d_model, 128)
    pre = dev.DeviceNorm("rms", torch.from_numpy((1 + 0.1 * rng.standard_normal(d_model)).astype(np.float32)).to(gpu))
    b = {"h": torch.from_numpy(rng.standard_normal((T, d_model)).astype(np.float32)).to(gpu), "x": torch.empty((T * k, d_model), dtype=torch.bfloat16, device=gpu),
         "logits": torch.empty((T, E), device=gpu), "idx": torch.empty((T, k), dtype=torch.int32, device=gpu), "gate": torch.empty((T, k), device=gpu),
         "y": torch.empty((T * k, d_model), device=gpu), "out": torch.empty((T, d_model), device=gpu), "next": torch.empty((T, d_model), dtype=torch.bfloat16, device=gpu),
         "mask": torch.ones(T, dtype=torch.uint8, device=gpu), "ws": layer.workspace(T * k)}
    b["mask"][T // 2] = 0

    def step(stream=None):
        q.qmoe_residual_norm(b["h"], x=b["x"], pre=pre, copies=k, stream=stream)
        q.qmoe_int4_matvec(R.desc, b["x"][::k], b["logits"], stream=stream)
        q.qmoe_route(b["logits"], b["idx"], b["gate"], token_mask=b["mask"], gates=q.GATES_CHOSEN, stream=stream)
        layer.forward(b["x"], b["idx"], b["y"], b["ws"], stream=stream)
        q.qmoe_residual_norm(b["h"], b["y"], b["out"], b["next"], k=k, gate=b["gate"], pre=pre, stream=stream)

    return ex, router, pre, b, step


@pytest.mark.parametrize("T,E,d_model,d_ff,k", [(1, 8, 256, 512, 2), (37, 8, 264, 136, 2), (200, 16, 128, 256, 4)])
def test_block_step(gpu, T, E, d_model, d_ff, k):
    rng = np.random.default_rng(T)
    ex, router, pre, b, step = _block(gpu, rng, T, E, d_model, d_ff, k)
    step()
    torch.cuda.synchronize()
    w = pre.weight.cpu().numpy()
    h = b["h"].cpu().numpy().astype(np.float64)
    _, _, x_want, x_err = plain.residual_norm(h, None, 1, None, None, 1.0, None, ("rms", w, None, 1e-6), k)
    _near(b["x"], x_want, x_err, "bf16", "x")
    x = b["x"].double().cpu().numpy()
    want, err = plain.int4_product(x[::k], router[0], router[2], router[3], 128, "none")
    _near(b["logits"], want, err, "f32", "logits")
    idx, gate, rel = plain.route(b["logits"].cpu().numpy(), None, b["mask"].cpu().numpy(), k, 1)
    assert np.array_equal(b["idx"].cpu().numpy(), idx)
    _near(b["gate"], gate, rel * gate, "f32", "gate")
    _check_layer(ex, x, idx.reshape(-1), None, 128, "relu", "f32", b["y"].cpu(), b["ws"], d_model, d_ff)
    g = b["gate"].cpu().numpy().reshape(-1)
    want, err, x_want, x_err = plain.residual_norm(h, b["y"].cpu().numpy().astype(np.float64), k, g, None, 1.0, None, ("rms", w, None, 1e-6), 1)
    _near(b["out"], want, err, "f32", "out")
    _near(b["next"], x_want, x_err, "bf16", "next x")


def test_block_step_in_a_graph_and_on_another_stream(gpu):
    """Captured and replayed several times over changed inputs, with eager work between the replays; and on a stream of its own."""
    rng = np.random.default_rng(11)
    _, _, _, b, step = _block(gpu, rng, 30, 8, 256, 512, 2)
    results = ("x", "logits", "idx", "gate", "y", "out", "next")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    on_side = {n: b[n].clone() for n in results}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(4):
        b["h"].copy_(torch.from_numpy(rng.standard_normal(b["h"].shape).astype(np.float32)).to(gpu) if turn else b["h"].clone())
        step()
        torch.cuda.synchronize()
        eager = {n: b[n].clone() for n in results}
        for n in results:
            b[n].zero_()
        graph.replay()
        torch.cuda.synchronize()
        for n in results:
            assert torch.equal(b[n], eager[n]), (turn, n)
            if turn == 0:
                assert torch.equal(b[n], on_side[n]), n


def test_two_streams_at_once(gpu):
    """Two programs with their own workspaces, each on a stream, give what each gives alone."""
    made = [_block(gpu, np.random.default_rng(seed), *sizes) for seed, sizes in ((3, (300, 8, 512, 1024, 2)), (4, (41, 16, 384, 640, 4)))]
    results = ("x", "logits", "idx", "gate", "y", "out", "next")
    alone = []
    for _, _, _, b, step in made:
        step()
        torch.cuda.synchronize()
        alone.append({n: b[n].clone() for n in results})
    streams = [torch.cuda.Stream() for _ in made]
    for (_, _, _, b, _), s in zip(made, streams):
        for n in results:
            b[n].zero_()
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(10):
        for (_, _, _, _, step), s in zip(made, streams):
            step(s)
    torch.cuda.synchronize()
    for (_, _, _, b, _), want in zip(made, alone):
        for n in results:
            assert torch.equal(b[n], want[n]), n


@pytest.mark.parametrize("T,k", [(1, 2), (40, 2), (300, 4)])
def test_block_step_on_ternary_experts(gpu, T, k):
    """The router's choice feeds the compressed layer, and the stream takes the rows that it leaves."""
    from paper_2310_16795_amd import synth

    w = synth.WORKLOADS["switch_base128"].scaled(n_experts=8, d_model=256, d_ff=512, n_tokens=8)
    dd = dev.DeviceDict(device=gpu)
    layer = dev.DeviceLayer(w.n_experts, w.d_model, w.d_ff, gpu)
    for e in range(w.n_experts):
        for which, tern, scale in (("wi", w.wi_ternary(e), w.wi_scale(e)), ("wo", w.wo_ternary(e), w.wo_scale(e))):
            layer.set_expert(e, which, *q.qmoe_encode_host(dd.handle, tern), scale)
    layer.finalize(device_order_of=dd)
    rng = np.random.default_rng(T)
    h, h64 = _up(rng.standard_normal((T, 256)), gpu)
    logits, _ = _up(rng.standard_normal((T, 8)), gpu)
    mask = torch.ones(T, dtype=torch.uint8, device=gpu)
    mask[T // 2:T // 2 + T // 4] = 0
    x = torch.empty((T * k, 256), dtype=torch.bfloat16, device=gpu)
    y, out = torch.empty((T * k, 256), device=gpu), torch.empty((T, 256), device=gpu)
    idx, gate = torch.empty((T, k), dtype=torch.int32, device=gpu), torch.empty((T, k), device=gpu)
    q.qmoe_residual_norm(h, x=x, pre=dev.DeviceNorm("rms"), copies=k)
    q.qmoe_route(logits, idx, gate, token_mask=mask, gates=q.GATES_CHOSEN)
    layer.forward(dd, x.view(torch.int16), idx, y, layer.workspace(T * k))
    q.qmoe_residual_norm(h, y, out, k=k, gate=gate)
    # the same layer call with the choice made on the host
    want, _, _ = plain.route(logits.cpu().numpy(), None, mask.cpu().numpy(), k, 1)
    y_host = torch.empty_like(y)
    layer.forward(dd, x.view(torch.int16), torch.from_numpy(want.astype(np.int32).reshape(-1)).to(gpu), y_host, layer.workspace(T * k))
    assert torch.equal(y, y_host) and y.isfinite().all() and y.any()
    assert not y[idx.view(-1) < 0].any() and torch.equal((idx < 0).all(1), mask == 0)
    want, err, _, _ = plain.residual_norm(h64, y.cpu().numpy().astype(np.float64), k, gate.cpu().numpy().reshape(-1), None, 1.0, None, None, 1)
    _near(out, want, err, "f32", "out")
    dd.close()


# ---------------------------------------------------------------- offsets past 32 bits

def _far(n, d, gpu, dtype):
    """A matrix whose rows are so far apart that the last begins more than 2^32 bytes behind the first"""
    step = (2 ** 32 // dtype.itemsize + 1024) // (n - 1)
    return torch.empty(step * (n - 1) + d, dtype=dtype, device=gpu).as_strided((n, d), (step, 1))


def test_rows_far_apart(gpu):
    rng = np.random.default_rng(8)
    n, d = 3, 200
    h, x = torch.from_numpy(rng.standard_normal((n, d)).astype(np.float32)).to(gpu), torch.empty((n, d), dtype=torch.bfloat16, device=gpu)
    near_h = torch.empty_like(h)
    pre = dev.DeviceNorm("layer", eps=1e-5)
    q.qmoe_residual_norm(h, h, near_h, x, pre=pre)
    far_h, far_out, far_x = _far(n, d, gpu, torch.float32), _far(n, d, gpu, torch.float32), _far(n, d, gpu, torch.bfloat16)
    far_h.copy_(h)
    q.qmoe_residual_norm(far_h, far_h, far_out, far_x, pre=pre)
    assert torch.equal(far_out, near_h) and torch.equal(far_x, x)
    idx, gate = torch.empty((2, n, 4), dtype=torch.int32, device=gpu), torch.empty((2, n, 4), device=gpu)
    q.qmoe_route(h, idx[0], gate[0])
    q.qmoe_route(far_h, idx[1], gate[1])
    assert torch.equal(idx[0], idx[1]) and torch.equal(gate[0], gate[1])
    M = _matrix(gpu, _weights(rng, 96, d, 64, True, False), d, 64)
    y, far_y = torch.empty((n, 96), device=gpu), _far(n, 96, gpu, torch.float32)
    q.qmoe_int4_matvec(M.desc, x, y)
    q.qmoe_int4_matvec(M.desc, far_x, far_y)
    assert torch.equal(y, far_y)


@pytest.mark.parametrize("batch", [1, 20])
def test_int4_matrix_of_more_than_32_bits(gpu, batch):
    rows, cols, group = 2 ** 20 + 300, 8192, 128
    weights = torch.randint(0, 256, (rows, cols // 2), dtype=torch.uint8, device=gpu)
    scale = (0.5 + torch.rand((rows, cols // group), device=gpu)).half().view(torch.int16)
    x, x64 = _up(np.random.default_rng(2).standard_normal((batch, cols)) / 64, gpu, "bf16")
    y = torch.empty((batch, rows), device=gpu)
    q.qmoe_int4_matvec(dev.DeviceInt4Matrix(weights, scale, cols, group).desc, x, y)
    for r0 in (0, 2 ** 19, rows - 300):
        values = q.qmoe_int4_unpack_host(weights[r0:r0 + 300].cpu().numpy(), cols)
        want, err = plain.int4_product(x64, values, scale[r0:r0 + 300].cpu().numpy().view(np.uint16), None, group, "none")
        _near(y[:, r0:r0 + 300], want, err, "f32", f"rows from {r0} on")


# ---------------------------------------------------------------- what is refused before anything is enqueued

def test_refusals_of_tensors(gpu):
    f = lambda *s, t=torch.float32, d=gpu: torch.zeros(s, dtype=t, device=d)  # noqa: E731
    b16, i32 = torch.bfloat16, torch.int32
    M = _matrix(gpu, _weights(np.random.default_rng(0), 32, 64, 32, False, True), 64, 32).desc
    bad = [
        lambda: q.qmoe_residual_norm(f(4, 8), f(4, 8, d="cpu"), f(4, 8)), lambda: q.qmoe_residual_norm(f(4, 8), f(4, 7), f(4, 8)),
        lambda: q.qmoe_residual_norm(f(4, 8), f(4, 8), f(4, 8, t=b16)), lambda: q.qmoe_residual_norm(f(8, 4).t(), f(4, 8), f(4, 8)),
        lambda: q.qmoe_residual_norm(f(4, 8, t=torch.float16), x=f(4, 8, t=b16)), lambda: q.qmoe_residual_norm(f(4, 8), x=f(4, 8)),
        lambda: q.qmoe_residual_norm(f(4, 8), x=f(4, 8, t=b16), pre=dev.DeviceNorm("rms", f(9))), lambda: q.qmoe_residual_norm(f(4, 8), f(8, 8), f(4, 8), k=2, gate=f(7)),
        lambda: q.qmoe_route(f(4, 8), f(4, 2, t=i32), f(4, 3)), lambda: q.qmoe_route(f(4, 8), f(4, 2), f(4, 2)),
        lambda: q.qmoe_route(f(4, 8), f(4, 2, t=i32), f(4, 2), bias=f(7)), lambda: q.qmoe_route(f(4, 8), f(4, 2, t=i32), f(4, 2), token_mask=f(4)),
        lambda: q.qmoe_int4_matvec(M, f(2, 63, t=b16), f(2, 32)), lambda: q.qmoe_int4_matvec(M, f(2, 64), f(2, 32)),
        lambda: q.qmoe_int4_matvec(M, f(2, 64, t=b16), f(2, 32), activation=q.ACTIVATIONS["silu"]), lambda: q.qmoe_int4_matvec(M, f(2, 64, t=b16), f(2, 32, t=torch.float16)),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was taken")
    with pytest.raises(q.QmoeError):
        q.qmoe_route(f(4, 8), f(4, 9, t=i32), f(4, 9))
