"""Edges of the operators around the layer on the GPU, against their formulas in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2310_16795_amd as q
from paper_2310_16795_amd import device as dev
from test_gpu_operators import _check_layer, _layer, _matrix, _near, _out, _untouched, _up, _weights, gpu  # noqa: F401

import plain
import plain_exact

pytestmark = pytest.mark.gpu

OUTLIERS = [  # rows, cols, batch, group, zeros, activation, y: little work, and tiles of 16, 32 and 64 tokens
    (30, 300, 1, 64, True, "none", "f32"), (16000, 600, 30, 32, True, "silu", "f32"), (20000, 600, 33, 128, False, "none", "f32"), (200, 390, 16, 128, False, "relu", "f32"), (12000, 600, 33, 32, True, "silu", "f32"), (12000, 600, 33, 256, False, "none", "bf16"),
    (12000, 600, 300, 128, True, "none", "f32"), (12000, 600, 300, 64, False, "gelu", "f32"), (1601, 200, 3601, 128, False, "none", "f32"),
    (1601, 200, 3601, 32, True, "none", "f32"), (3202, 330, 3590, 64, True, "silu", "f32"), (3202, 330, 3590, 128, False, "silu", "f32"),
]


@pytest.mark.parametrize("large", [1e4, 3e38])
@pytest.mark.parametrize("rows,cols,batch,group,zeros,act,yt", OUTLIERS)
def test_int4_weight_of_zero_takes_nothing_from_a_large_activation(gpu, rows, cols, batch, group, zeros, act, yt, large):  # noqa: F811
    rng = np.random.default_rng(rows + batch)
    values, _, s, zero = _weights(rng, rows, cols, group, zeros, False)
    x = rng.standard_normal((batch, cols))
    at = rng.choice(cols, 5)
    for c in at:
        values[:, c] = 8 if zero is None else zero[:, c // group]
    x[np.arange(batch), at[np.arange(batch) % 5]] = large * (-1.0) ** np.arange(batch)
    xd, x64 = _up(x, gpu, "bf16")
    y, held = _out(batch, rows // 2 if act in ("silu", "gelu") else rows, gpu, yt)
    W = _matrix(gpu, (values, q.qmoe_int4_pack_host(values), s, zero), cols, group)
    q.qmoe_int4_matvec(W.desc, xd, y, activation=q.ACTIVATIONS[act])
    want, err = plain_exact.int4_product(x64, values, s, zero, group, act)
    _near(y, want, err, yt)
    _untouched(held, *y.shape)
    d = y.double().cpu().numpy() - want  # as a whole far closer than the bound on each
    assert yt != "f32" or np.linalg.norm(d) <= 2e-6 * np.linalg.norm(want)


@pytest.mark.parametrize("rows,cols,batch", [(30, 300, 1), (12000, 600, 33), (12000, 600, 300), (1601, 200, 3601)])
def test_int4_product_of_the_largest_activation_is_finite(gpu, rows, cols, batch):  # noqa: F811
    """One activation near the end of bf16 times the largest weight, 15 steps of 2^-10: finite, with nothing else next to it to lose."""
    values, zero = np.full((rows, cols), 15, dtype=np.uint8), np.zeros((rows, -(-cols // 64)), dtype=np.uint8)
    s = np.full(zero.shape, 2.0 ** -10, dtype=np.float16).view(np.uint16)
    x = np.zeros((batch, cols))
    x[np.arange(batch), np.arange(batch) * 7 % cols] = 3e38
    xd, x64 = _up(x, gpu, "bf16")
    y = torch.empty((batch, rows), device=gpu)
    W = _matrix(gpu, (values, q.qmoe_int4_pack_host(values), s, zero), cols, 64)
    q.qmoe_int4_matvec(W.desc, xd, y)
    want, err = plain_exact.int4_product(x64, values, s, zero, 64, "none")
    _near(y, want, 0 * err, "f32")


@pytest.mark.parametrize("e", [2048, 4096, 16384])
def test_route_gates_over_equal_logits(gpu, e):  # noqa: F811
    """One expert at 0 and the others all at -d, 512 values of d where they make up most of the sum: an error of exp(-d) is the same in every term and stays.
    Done accurately the gate is off by the rounding of exp(-d), of quotient and sums (terms of one size add up exactly by halves; where the one joins, sums of
    1/2, 1/4, ... of the whole are rounded: the root of 1 + 1/4 + ... for all of them): each evenly spread over half a step, 1/sqrt(3) of it as a root mean square,
    together sqrt(1 + 1 + 4/3) / sqrt(3) = 1.05 half steps.  Twice that is allowed."""
    d = np.linspace(np.log(e) - 2.0, np.log(e) - 1.4, 512).astype(np.float32)
    l = np.repeat(-d[:, None], e, axis=1)
    l[:, 7] = 0.0
    idx, gate = torch.empty((512, 1), dtype=torch.int32, device=gpu), torch.empty((512, 1), device=gpu)
    q.qmoe_route(torch.from_numpy(l).to(gpu), idx, gate)
    want = 1.0 / (1.0 + (e - 1) * np.exp(-d.astype(np.float64)))
    rel = (gate.cpu().numpy()[:, 0].astype(np.float64) - want) / want
    assert (idx == 7).all()
    assert np.sqrt((rel ** 2).mean()) <= 2 * 1.05 * plain.U32, f"{np.sqrt((rel ** 2).mean()) / plain.U32:.2f} half steps"


def test_descriptors_of_another_device_are_refused(gpu):  # noqa: F811
    """(With one GPU another is a number that the descriptors say they are on.)"""
    x, y = torch.zeros((2, 64), dtype=torch.bfloat16, device=gpu), torch.zeros((2, 32), device=gpu)
    W = _matrix(gpu, _weights(np.random.default_rng(0), 32, 64, 32, False, True), 64, 32)
    h, norm = torch.zeros((2, 64), device=gpu), dev.DeviceNorm("rms", torch.ones(64, device=gpu))
    assert W.desc.device == norm.desc.device == x.get_device() and dev.DeviceNorm("rms").desc.device is None
    calls = [lambda: q.qmoe_int4_matvec(W.desc, x, y), lambda: q.qmoe_residual_norm(h, x=x, pre=norm), lambda: q.qmoe_residual_norm(h, x=x, pre=norm.desc),
             lambda: q.qmoe_residual_norm(h, h, torch.empty_like(h), post=norm)]
    for call in calls:
        call()
    W.desc.device = norm.desc.device = x.get_device() + 1
    for call in calls:
        with pytest.raises(ValueError, match="current device"):
            call()


# ---------------------------------------------------------------- every kernel, by what the library chooses

KERNELS = [  # kernel, rows, cols, batch, group, zeros, activation
    ("split", 200, 300, 40, 64, True, "none"), ("split", 300, 4300, 20, 32, False, "silu"), ("tile 16", 16000, 600, 30, 32, True, "silu"), ("tile 16", 20000, 1100, 33, 32, False, "none"),
    ("tile 16", 16000, 4300, 30, 128, True, "none"), ("tile 32", 12000, 600, 300, 128, True, "none"), ("tile 32", 12000, 1100, 300, 32, True, "gelu"), ("tile 32", 12000, 2300, 300, 128, False, "none"),
    ("mm", 1601, 200, 3601, 32, True, "none"), ("mm", 1601, 1100, 3601, 32, True, "none"), ("mm", 1601, 1100, 3601, 32, False, "none"), ("mm", 1601, 2300, 3601, 64, True, "none"),
    ("mm", 1601, 4300, 3601, 128, True, "none"), ("mm", 1601, 4300, 3601, 128, False, "none"), ("mm", 1601, 8400, 3601, 256, True, "none"), ("mm", 3202, 1100, 3590, 32, True, "silu"),
    ("mm", 3202, 4300, 3590, 128, False, "gelu"), ("mm", 3202, 4300, 3590, 128, True, "silu"),
]


@pytest.mark.parametrize("kernel,rows,cols,batch,group,zeros,act", KERNELS)
def test_int4_kernels_spoil_no_other_token_and_repeat_themselves(gpu, kernel, rows, cols, batch, group, zeros, act):  # noqa: F811
    """Matrices of more groups than a kernel holds at a time among them; two tokens are not finite; a second call gives the same bits."""
    assert q.qmoe_hook_int4_kernel(rows, cols, group, q.ACTIVATIONS[act], batch, torch.cuda.get_device_properties(0).multi_processor_count) == kernel
    rng = np.random.default_rng(cols + batch)
    w = _weights(rng, rows, cols, group, zeros, False)
    x = rng.standard_normal((batch, cols)).astype(np.float32)
    x[1, 5], x[batch - 1, cols - 1] = np.inf, np.nan
    xd, x64 = _up(x, gpu, "bf16")
    y, again = (torch.empty((batch, rows // 2 if act in ("silu", "gelu") else rows), device=gpu) for _ in range(2))
    W = _matrix(gpu, w, cols, group)
    for out in (y, again):
        q.qmoe_int4_matvec(W.desc, xd, out, activation=q.ACTIVATIONS[act])
    assert torch.equal(y.view(torch.int32), again.view(torch.int32))
    keep = np.r_[0, 2:batch - 1]
    want, err = plain_exact.int4_product(x64[keep], w[0], w[2], w[3], group, act)
    _near(y[torch.from_numpy(keep).to(gpu)], want, err, "f32")
    assert y[batch - 1].isnan().all() and not (act == "none" and y[1].isfinite().any())


def test_int4_more_units_than_workgroups(gpu):  # noqa: F811
    """k_int4_mm's workgroups take a second unit: 530000 tokens, whose results are compared on the GPU in 64 bits."""
    rows, cols, batch, group = 257, 8, 530000, 32
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    assert q.qmoe_hook_int4_kernel(rows, cols, group, 0, batch, cus) == "mm" and -(-batch // 64) * 2 > 64 * cus
    rng = np.random.default_rng(1)
    w = _weights(rng, rows, cols, group, True, True)
    x = torch.randint(-8, 9, (batch, cols), device=gpu).to(torch.bfloat16)
    y = torch.full((batch + 1, rows), -77.0, device=gpu)
    W = _matrix(gpu, w, cols, group)
    q.qmoe_int4_matvec(W.desc, x, y[:batch])
    matrix = torch.from_numpy(plain.int4_matrix(w[0], w[2], w[3], group)[0]).to(gpu).t().contiguous()
    for t0 in range(0, batch, 100000):  # (whole numbers and powers of two: exact)
        assert torch.equal(y[t0:t0 + 100000][:batch - t0].double(), x[t0:t0 + 100000].double() @ matrix)
    assert (y[batch] == -77.0).all()


LAYERS = [  # kernels of the two products, experts, d_model, d_ff, tokens, group, zeros, activation, y
    (("tile 16", "tile 16"), 40, 1160, 1288, 64, 32, True, "silu", "bf16"), (("tile 16", "tile 16"), 30, 2112, 2112, 100, 64, True, "gelu", "f32"),
    (("tile 16", "split"), 16, 1160, 3304, 40, 64, True, "silu", "f32"), (("tile 16", "tile 16"), 30, 1160, 1288, 300, 256, True, "silu", "bf16"),
    (("tile 32", "tile 32"), 16, 1096, 2112, 700, 32, True, "gelu", "f32"), (("tile 32", "tile 32"), 20, 1160, 1288, 700, 512, True, "silu", "f32"),
    (("split", "split"), 20, 776, 904, 90, 384, False, "relu", "bf16"), (("split", "split"), 5, 1288, 1160, 9, 1152, True, "gelu", "f32"), (("split", "split"), 3, 520, 776, 8, 256, True, "silu", "bf16"),
]


@pytest.mark.parametrize("kernels,E,d_model,d_ff,T,group,zeros,act,yt", LAYERS)
def test_int4_layer_kernels(gpu, kernels, E, d_model, d_ff, T, group, zeros, act, yt):  # noqa: F811
    """Gated experts with zero points and many groups in tiles, and groups of several blocks, in layer calls; a second call gives the same bits."""
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    assert q.qmoe_hook_int4_layer_kernels(group, q.ACTIVATIONS[act], E, d_model, d_ff, T, cus) == kernels
    rng = np.random.default_rng(E + T)
    ex, layer = _layer(gpu, rng, E, d_model, d_ff, group, zeros, act)
    idx = rng.integers(0, E, T).astype(np.int32)
    idx[: T // 3], idx[T // 2] = E - 1, -1
    gate = rng.random(T).astype(np.float32)
    x, x64 = _up(rng.standard_normal((T, d_model)), gpu, "bf16")
    (y, held), ws = _out(T, d_model, gpu, yt), layer.workspace(T)
    args = torch.from_numpy(idx).to(gpu), y, ws, torch.from_numpy(gate).to(gpu)
    layer.forward(x, *args)
    first = y.clone()
    _check_layer(ex, x64, idx, gate, group, act, yt, y.cpu(), ws, d_model, d_ff)
    _untouched(held, T, d_model)
    layer.forward(x, *args)
    assert torch.equal(y, first)


@pytest.mark.parametrize("idx", [[0] * 8, [2, 2, 1, 2, -1, 1, 2, 5], [1, 0, 1, 0, 1, 0, 1], [3, -1, 3, 99, 3], [4, 4], [-1] * 6, [0, 1, 2, 3, 4, 4, 3, 2]])
@pytest.mark.parametrize("act,zeros,group", [("relu", False, 128), ("silu", True, 64), ("gelu", True, 256)])
def test_int4_layer_of_few_tokens_that_share_experts(gpu, idx, act, zeros, group):  # noqa: F811
    """Up to eight tokens go without the dispatch; those of one expert are multiplied together, each where it stands."""
    rng = np.random.default_rng(len(idx))
    E, d_model, d_ff, T = 5, 392, 520, len(idx)
    ex, layer = _layer(gpu, rng, E, d_model, d_ff, group, zeros, act)
    idx = np.array(idx, dtype=np.int32)
    gate = rng.random(T).astype(np.float32)
    x, x64 = _up(rng.standard_normal((T, d_model)), gpu, "bf16")
    (y, held), ws = _out(T, d_model, gpu, "f32"), layer.workspace(T)
    layer.forward(x, torch.from_numpy(idx).to(gpu), y, ws, torch.from_numpy(gate).to(gpu))
    _check_layer(ex, x64, idx, gate, group, act, "f32", y.cpu(), ws, d_model, d_ff)
    _untouched(held, T, d_model)
