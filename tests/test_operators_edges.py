"""Edges of the operators around the layer, on the CPU: calls of the checked CPU build of the kernels (tests/operators/edge_calls.py), and what the
holders of device tensors keep and refuse."""
import gc
import os
import subprocess
import sys
import weakref

import pytest
import torch

from test_operators_lanes import library  # noqa: F401

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.parametrize("kind,count,units", [("outlier", 32, 1), ("outlier", 16, 64), ("wide", 16, 1), ("wide", 8, 6), ("layer_groups", 16, 1), ("layer_groups", 16, 8), ("layer_few", 24, 2), ("layer_few", 24, 256)])
def test_edge_calls(library, kind, count, units):  # noqa: F811
    cmd = [sys.executable, os.path.join(HERE, "operators", "edge_calls.py"), kind, str(count)]
    r = subprocess.run(cmd, env={**os.environ, "QMOE_LIBRARY": library, "LANES_COMPUTE_UNITS": str(units)}, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600)
    assert r.returncode == 0 and r.stdout.rstrip().endswith("done"), r.stdout[-3000:]


@pytest.fixture
def on_the_host(monkeypatch):
    """Descriptors of host tensors, for what does not launch anything."""
    from paper_2310_16795_amd import _binding

    monkeypatch.setattr(_binding, "_dev_ptr", lambda t: 0 if t is None else t.data_ptr())


def test_a_descriptor_keeps_its_tensors(on_the_host):
    """The calls take a descriptor alone: what it points to lives as long as it does."""
    from paper_2310_16795_amd import device as dev

    made = [torch.zeros((4, 64), dtype=torch.uint8), torch.zeros((4, 2), dtype=torch.float16), torch.zeros((4, 2), dtype=torch.uint8), torch.ones(8), torch.zeros(8)]
    alive = [weakref.ref(t) for t in made]
    matrix, norm = dev.DeviceInt4Matrix(made[0], made[1], 128, 64, made[2]).desc, dev.DeviceNorm("layer", made[3], made[4]).desc
    addresses = [t.data_ptr() for t in made]
    del made
    gc.collect()
    assert all(r() is not None for r in alive)
    assert [matrix.weights, matrix.scale_f16, matrix.zero, norm.weight, norm.bias] == addresses
    del matrix, norm
    gc.collect()
    assert all(r() is None for r in alive)


def test_what_a_descriptor_points_to_is_on_one_device(on_the_host):
    from paper_2310_16795_amd import device as dev

    host = dict(w=torch.zeros((4, 64), dtype=torch.uint8), s=torch.zeros((4, 2), dtype=torch.float16), z=torch.zeros((4, 2), dtype=torch.uint8))
    for name in host:
        t = {**host, name: host[name].to("meta")}
        with pytest.raises(ValueError, match="one device"):
            dev.DeviceInt4Matrix(t["w"], t["s"], 128, 64, t["z"])
        t = {k: v.view(1, 4, -1) for k, v in t.items()}
        with pytest.raises(ValueError, match="one device"):
            dev.DeviceInt4Layer(tuple(t.values()), tuple(t.values()), 128, 4, 64)
    layer = [tuple(v.view(1, 4, -1) for v in host.values()), (torch.zeros((1, 128, 64), dtype=torch.uint8, device="meta"), torch.zeros((1, 128, 1), dtype=torch.float16, device="meta"), None)]
    with pytest.raises(ValueError, match="one device"):
        dev.DeviceInt4Layer(*layer, 128, 4, 64)
    with pytest.raises(ValueError, match="one device"):
        dev.DeviceNorm("layer", torch.ones(8), torch.zeros(8, device="meta"))


def test_scales_are_binary16_and_weights_aligned(on_the_host):
    """A scale of another 16-bit type would be read as binary16; a layer's descriptors are not seen by the call, so what they point to is checked here."""
    from paper_2310_16795_amd import device as dev

    w, s = torch.zeros((2, 128, 64), dtype=torch.uint8), torch.ones((2, 128, 2), dtype=torch.float16)
    odd = torch.zeros(w.numel() + 8, dtype=torch.uint8)[8:].view(w.shape)
    for kind in (torch.float16, torch.int16, torch.uint16):
        dev.DeviceInt4Matrix(w[0], s[0].view(kind), 128, 64)
        dev.DeviceInt4Layer((w, s.view(kind), None), (w, s.view(kind), None), 128, 128, 64)
    for kind in (torch.bfloat16, torch.float32, torch.uint8):
        with pytest.raises(ValueError, match="binary16"):
            dev.DeviceInt4Matrix(w[0], s[0].to(kind), 128, 64)
        with pytest.raises(ValueError, match="binary16"):
            dev.DeviceInt4Layer((w, s, None), (w, s.to(kind), None), 128, 128, 64)
    with pytest.raises(ValueError, match="aligned"):
        dev.DeviceInt4Matrix(odd[0], s[0], 128, 64)
    with pytest.raises(ValueError, match="aligned"):
        dev.DeviceInt4Layer((w, s, None), (odd, s, None), 128, 128, 64)


def test_which_kernel_a_four_bit_product_takes():
    """The choice follows the sizes: few tokens, more, many; sizes that are none have no kernel."""
    import paper_2310_16795_amd as q

    one = lambda *a: q.qmoe_hook_int4_kernel(*a)  # noqa: E731
    assert [one(20000, 1100, 128, 0, batch) for batch in (1, 33, 150, 4001)] == ["split", "tile 16", "tile 32", "mm"]
    # one more workgroup than compute units is a turn of all its columns (2080 x 6144, 256 tokens: 272 workgroups 52 us, k_int4_split 39, tiles of 32 43)
    assert one(2080, 6144, 128, 0, 256) in ("split", "tile 32")
    assert [one(rows, 7, 32, 0, 4001) for rows in (8, 20000)] == ["split"] * 2  # (the other kernels load eight columns)
    L = q.lib()
    assert [L.qmoe_hook_int4_kernel(*bad) for bad in ((0, 8, 32, 0, 1, 256), (8, 0, 32, 0, 1, 256), (8, 8, 48, 0, 1, 256), (8, 8, 32, 0, 0, 256), (8, 8, 32, 0, 1, 0))] == [0] * 5
    assert q.qmoe_hook_int4_layer_kernels(128, q.ACT_RELU, 128, 768, 3072, 4001) == ("tile 32", "tile 32") and q.qmoe_hook_int4_layer_kernels(128, q.ACT_RELU, 128, 768, 3072, 8) == ("split", "split")
    with pytest.raises(q.QmoeError):
        q.qmoe_hook_int4_layer_kernels(128, q.ACT_RELU, 0, 768, 3072, 8)
