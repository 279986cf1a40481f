"""The operators around the compressed layer, as cases that can be timed.

What a decoder block does next to its compressed experts: the residual stream takes the layer's output and is normalised
for the next call (`qmoe_residual_norm`), the router's logits become experts and gates (`qmoe_route`), and the matrices
kept in four bits with a scale per group of columns are multiplied with the tokens, one at a time (`qmoe_int4_matvec`) or
as the experts of a layer (`qmoe_int4_layer_forward`).  Shapes are those of the SwitchTransformer layers the benchmark
uses, or generic ones of the same range; activations are normal, as a norm leaves them, and the four-bit values are
binomial around 7.5, as quantised weights are around their middle.

With `own` false, `run` computes the operators from elementary torch operations in 32 bits.

Four-bit rows: 64 bytes hold 128 columns; the 32-bit word 4 q + s of such a block holds columns 32 s + 8 q .. + 7 of it,
the even ones in its low half, the odd ones in its high half, four bits each, lowest first.
"""
import math

import numpy as np
import torch

own = False
GPU = "cuda:0"
POOL = 3  # distinct experts made per layer; every expert has its own copy in memory of one of them


def listed():
    return [
        # generating one token with the small model: the step between two layers, where the launch is what counts
        {"name": "norm_base_1", "op": "norm", "tokens": 1, "d": 768, "k": 1, "copies": 1, "h": "f32", "y": "f32", "gate": False,
         "pre": "rms", "post": "none", "channel": False},
        # a batch through the largest model, two experts a token: their rows are joined with their gates and x goes out twice
        {"name": "norm_c2048_2048_top2", "op": "norm", "tokens": 2048, "d": 2080, "k": 2, "copies": 2, "h": "bf16", "y": "f32",
         "gate": True, "pre": "rms", "post": "none", "channel": False},
        # a long prompt, norms on both sides of the block and a learnt scale a channel (the residual stream in 32 bits)
        {"name": "norm_prompt_8191_both", "op": "norm", "tokens": 8191, "d": 1024, "k": 1, "copies": 1, "h": "f32", "y": "bf16",
         "gate": False, "pre": "layer", "post": "layer", "channel": True},
        # the router of the small model, one token
        {"name": "route_base128_1", "op": "route", "tokens": 1, "experts": 128, "k": 1, "logits": "f32", "gates": "all",
         "bias": False, "padded": 0.0},
        # the router of the largest model, a batch: one expert of 2048 for every token
        {"name": "route_c2048_4096", "op": "route", "tokens": 4096, "experts": 2048, "k": 1, "logits": "f32", "gates": "all",
         "bias": False, "padded": 0.0},
        # a padded batch of prompts, eight of 256 experts, balanced by a bias, logits in bf16 (many of them equal)
        {"name": "route_prompt_16384_top8", "op": "route", "tokens": 16384, "experts": 256, "k": 8, "logits": "bf16",
         "gates": "chosen", "bias": True, "padded": 0.1},
        # one token through a dense projection of the middle model: the smallest product
        {"name": "int4_large_1", "op": "int4", "rows": 4096, "cols": 1024, "batch": 1, "group": 128, "zeros": False, "act": "none"},
        # a batch of tokens that all generate, zero points, a scale every 64 columns
        {"name": "int4_c2048_37_zeros", "op": "int4", "rows": 2080, "cols": 6144, "batch": 37, "group": 64, "zeros": True,
         "act": "none"},
        # a prompt through the first half of a gated feed-forward block: both projections, activation and product
        {"name": "int4_prompt_4001_gated", "op": "int4", "rows": 12288, "cols": 2080, "batch": 4001, "group": 128, "zeros": False,
         "act": "silu"},
        # generating one token with the middle model, two experts
        {"name": "layer_large128_1_top2", "op": "layer", "experts": 128, "d_model": 1024, "d_ff": 4096, "tokens": 1, "k": 2,
         "routing": "uniform", "padded": 0.0, "group": 128, "zeros": False, "act": "relu"},
        # 64 sequences that generate, gated experts of the largest shapes
        {"name": "layer_c2048_64_gated", "op": "layer", "experts": 256, "d_model": 2080, "d_ff": 6144, "tokens": 64, "k": 1,
         "routing": "uniform", "padded": 0.0, "group": 64, "zeros": True, "act": "silu"},
        # a prompt through the small model, skewed routing, some of the batch padding
        {"name": "layer_base128_prompt_4001", "op": "layer", "experts": 128, "d_model": 768, "d_ff": 3072, "tokens": 4001, "k": 1,
         "routing": "zipf", "padded": 0.05, "group": 128, "zeros": False, "act": "relu"},
    ]


def _log(rng, lo, hi):
    """An integer in lo .. hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _of8(v):
    return max(8, (v + 4) // 8 * 8)


def draw(rng):
    """One more case: any operator, over the sizes between the smallest and the largest listed."""
    op = rng.choice(("norm", "route", "int4", "int4", "layer"))
    if op == "norm":
        while True:
            n, d, k = _log(rng, 1, 8191), _log(rng, 500, 6200), rng.choice((1, 1, 2, 4))
            if n * d * k <= 8191 * 1024:
                break
        d = d if rng.random() < 0.2 else _of8(d)
        return {"op": op, "tokens": n, "d": d, "k": k, "copies": rng.choice((1, k)), "h": rng.choice(("f32", "bf16")),
                "y": rng.choice(("f32", "bf16")), "gate": k > 1 or rng.random() < 0.3, "pre": rng.choice(("rms", "rms", "layer")),
                "post": rng.choice(("none", "none", "rms", "layer")), "channel": rng.random() < 0.3}
    if op == "route":
        while True:
            n, e = _log(rng, 1, 16384), _log(rng, 8, 2048)
            if n * e <= 4096 * 2048:
                break
        return {"op": op, "tokens": n, "experts": e, "k": min(e, rng.choice((1, 1, 2, 4, 6, 8))), "logits": rng.choice(("f32", "bf16")),
                "gates": rng.choice(("all", "chosen")), "bias": rng.random() < 0.4, "padded": rng.choice((0.0, 0.0, 0.1, 0.4))}
    group, zeros, act = rng.choice((32, 64, 128, 128, 128, 256)), rng.random() < 0.4, rng.choice(("none", "none", "relu", "silu", "gelu"))
    if op == "int4":
        while True:
            rows, cols, batch = _log(rng, 500, 12288) // 2 * 2, _log(rng, 500, 6200), _log(rng, 1, 4001) if rng.random() < 0.7 else 1
            if rows * cols <= 12288 * 2080 and rows * cols * batch <= 12288 * 2080 * 4001:
                break
        cols = cols if rng.random() < 0.2 else _of8(cols)
        return {"op": op, "rows": rows, "cols": cols, "batch": batch, "group": group, "zeros": zeros, "act": act}
    while True:
        case = {"op": op, "experts": _log(rng, 4, 256), "d_model": _of8(_log(rng, 500, 2080)), "d_ff": _of8(_log(rng, 1000, 6144)),
                "tokens": _log(rng, 1, 4001), "k": rng.choice((1, 1, 2)), "routing": rng.choice(("uniform", "zipf")),
                "padded": rng.choice((0.0, 0.0, 0.1)), "group": group, "zeros": zeros, "act": "relu" if act == "none" else act}
        size = case["d_model"] * case["d_ff"]
        rows = case["tokens"] * case["k"]
        # within the listed layers' weights and work
        if _active(case) * size <= 57 * 2080 * 6144 and rows * size <= 4001 * 768 * 3072 * 3 and rows <= 4001:
            return case


# ---------------------------------------------------------------- inputs

def _binomial_bytes(gen, n):
    """n bytes, each of their two halves the number of heads in 15 throws."""
    half = torch.tensor([math.comb(15, i) for i in range(16)], dtype=torch.float64, device=GPU).cumsum(0) * (256.0 / 2 ** 15)
    level = torch.searchsorted(half, torch.arange(256, dtype=torch.float64, device=GPU) + 0.5).clamp(max=15).to(torch.uint8)
    lo, hi = (level[torch.randint(0, 256, (n,), generator=gen, device=GPU)] for _ in range(2))
    return lo | (hi << 4)


def _row_bytes(cols):
    return 64 * ((cols + 127) // 128)


def _int4(gen, count, rows, cols, group, zeros):
    """`count` matrices: bytes [count, rows, row bytes], scales [count, rows, groups], zero points or None."""
    groups = (cols + group - 1) // group
    w = _binomial_bytes(gen, count * rows * _row_bytes(cols)).view(count, rows, _row_bytes(cols))
    s = ((0.5 + torch.rand((count, rows, groups), generator=gen, device=GPU)) / (2 * math.sqrt(cols))).to(torch.float16)
    z = torch.randint(6, 10, (count, rows, groups), generator=gen, device=GPU).to(torch.uint8) if zeros else None
    return w, s, z


def _zipf(n_experts):
    w = np.arange(1, n_experts + 1, dtype=np.float64) ** -1.1
    return w / w.sum()


def _routing(case, seed):
    """The expert of every row that goes into the layer (k rows a token, different experts), -1 for padding."""
    rng = np.random.default_rng(seed)
    p = _zipf(case["experts"])[rng.permutation(case["experts"])] if case["routing"] == "zipf" else np.full(case["experts"], 1.0 / case["experts"])
    score = np.log(p)[None, :] + rng.gumbel(size=(case["tokens"], case["experts"]))
    idx = np.argsort(-score, axis=1)[:, :case["k"]].astype(np.int32)
    idx[rng.random(case["tokens"]) < case["padded"]] = -1
    return idx.reshape(-1)


def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def prepare(case, seed):
    gen = torch.Generator(device=GPU)
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=GPU)

    op, s = case["op"], {"case": dict(case)}
    if op == "norm":
        n, d, k = case["tokens"], case["d"], case["k"]
        s["h"] = (3.0 * normal(n, d)).to(_type(case["h"]))  # the stream grows with depth
        s["y"] = normal(n * k, d).to(_type(case["y"]))
        s["gate"] = torch.rand((n * k,), generator=gen, device=GPU) if case["gate"] else None
        s["channel"] = 0.1 + 0.2 * torch.rand((d,), generator=gen, device=GPU) if case["channel"] else None
        for side in ("pre", "post"):
            s[side + "_weight"] = 1.0 + 0.2 * normal(d) if case[side] != "none" else None
            s[side + "_bias"] = 0.1 * normal(d) if case[side] == "layer" else None
        s["h_out"], s["x"] = torch.empty_like(s["h"]), torch.empty((n * case["copies"], d), dtype=torch.bfloat16, device=GPU)
        if own:  # the descriptors of the two norms, as a program keeps them beside their weights
            from paper_2310_16795_amd import device as dev
            s["pre"], s["post"] = (None if case[side] == "none" else
                                   dev.DeviceNorm(case[side], s[side + "_weight"], s[side + "_bias"], eps=1e-6) for side in ("pre", "post"))
    elif op == "route":
        n, e, k = case["tokens"], case["experts"], case["k"]
        s["logits"] = (1.5 * normal(n, e)).to(_type(case["logits"]))
        # a balancing bias moves by steps of a fixed size
        s["bias"] = torch.randint(-256, 257, (e,), generator=gen, device=GPU).to(torch.float32) / 1024 if case["bias"] else None
        s["mask"] = (torch.rand((n,), generator=gen, device=GPU) >= case["padded"]).to(torch.uint8) if case["padded"] else None
        s["idx"], s["gate"] = torch.empty((n, k), dtype=torch.int32, device=GPU), torch.empty((n, k), device=GPU)
    elif op == "int4":
        rows, cols, batch = case["rows"], case["cols"], case["batch"]
        w, sc, z = _int4(gen, 1, rows, cols, case["group"], case["zeros"])
        s["w"], s["scale"], s["zero"] = w[0], sc[0], None if z is None else z[0]
        s["x"] = normal(batch, cols).to(torch.bfloat16)
        s["y"] = (torch.empty((batch, rows), device=GPU) if case["act"] == "none" else
                  torch.empty((batch, rows if case["act"] == "relu" else rows // 2), dtype=torch.bfloat16, device=GPU))
        if own:  # the matrix's descriptor, made when it is loaded
            from paper_2310_16795_amd import device as dev
            s["matrix"] = dev.DeviceInt4Matrix(s["w"], s["scale"], cols, case["group"], s["zero"])
    else:
        E, d_model, d_ff = case["experts"], case["d_model"], case["d_ff"]
        idx = _routing(case, seed)
        kept = idx[idx >= 0]
        pool = min(POOL, E)
        pick = torch.arange(E, device=GPU) % pool
        for name, rows, cols in (("wi", d_ff if case["act"] == "relu" else 2 * d_ff, d_model), ("wo", d_model, d_ff)):
            s[name] = tuple(None if v is None else v[pick] for v in _int4(gen, pool, rows, cols, case["group"], case["zeros"]))
        s["x"] = normal(idx.size, d_model).to(torch.bfloat16)
        s["idx"] = torch.from_numpy(idx).to(GPU)
        s["gate"] = 0.2 + 0.8 * torch.rand((idx.size,), generator=gen, device=GPU)
        s["y"] = torch.empty((idx.size, d_model), dtype=torch.bfloat16, device=GPU)
        # for the plain form: which experts have tokens, and the most that one has
        s["active"] = torch.from_numpy(np.unique(kept) if kept.size else np.zeros(1, dtype=np.int32)).to(GPU).long()
        s["most"] = int(np.bincount(kept, minlength=1).max())
        if own:  # the experts' descriptors, made when they are loaded, and the workspace
            from paper_2310_16795_amd import device as dev
            s["layer"] = dev.DeviceInt4Layer(s["wi"], s["wo"], d_model, d_ff, case["group"], case["act"])
            s["ws"] = s["layer"].workspace(idx.size)
    return s


# ---------------------------------------------------------------- plain forms

def _columns(cols):
    """Where column c's four bits stand in a row, counted in halves of bytes."""
    c = torch.arange(cols, device=GPU)
    block, s, q, j = c // 128, c % 128 // 32, c % 32 // 8, c % 8
    return 128 * block + 8 * (4 * q + s) + 4 * (j % 2) + j // 2


def _weights(w, scale, zero, cols, group):
    """The matrices [..., rows, cols] in 32 bits."""
    q = torch.stack((w & 15, w >> 4), dim=-1).flatten(-2).index_select(-1, _columns(cols)).float()
    g = torch.arange(cols, device=GPU) // group
    z = 8.0 if zero is None else zero.float().index_select(-1, g)
    return (q - z) * scale.float().index_select(-1, g)


def _activated(v, act):
    """v [..., rows, ...] with the rows in its dimension 1."""
    if act == "none":
        return v
    if act == "relu":
        return torch.where(v > 0, v, torch.zeros_like(v))
    half = v.shape[1] // 2
    g, u = v[:, :half], v[:, half:]
    if act == "silu":
        return g / (1 + torch.exp(-g)) * u
    return 0.5 * g * (1 + torch.tanh(0.7978845608028654 * (g + 0.044715 * g * g * g))) * u


def _normed(v, kind, weight, bias):
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.mean(dim=-1, keepdim=True)
    v = v * torch.rsqrt((v * v).mean(dim=-1, keepdim=True) + 1e-6) * weight
    return v if bias is None else v + bias


def _plain_norm(s, case):
    n, d, k = case["tokens"], case["d"], case["k"]
    b = s["y"].float().view(n, k, d)
    b = (b if s["gate"] is None else b * s["gate"].view(n, k, 1)).sum(dim=1)
    b = 0.5 * _normed(b, case["post"], s["post_weight"], s["post_bias"])
    h = s["h"].float() + (b if s["channel"] is None else b * s["channel"])
    x = _normed(h, case["pre"], s["pre_weight"], s["pre_bias"]).to(torch.bfloat16)
    return h.to(s["h"].dtype), x.repeat_interleave(case["copies"], dim=0)


def _plain_route(s, case):
    l = s["logits"].float()
    key = l if s["bias"] is None else l + s["bias"]
    idx = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :case["k"]]
    over = l if case["gates"] == "all" else l.gather(1, idx)
    top = over.max(dim=1, keepdim=True).values
    gate = torch.exp(l.gather(1, idx) - top) / torch.exp(over - top).sum(dim=1, keepdim=True)
    idx = idx.to(torch.int32)
    if s["mask"] is not None:
        there = (s["mask"] != 0).view(-1, 1)
        idx, gate = torch.where(there, idx, -1), torch.where(there, gate, 0.0)
    return idx, gate


def _plain_layer(s, case):
    idx, A, cap = s["idx"].long(), s["active"].numel(), s["most"]
    T, d_model = s["x"].shape
    # every row's place: its expert's number among the active ones, and how many rows of that expert come before it
    number = torch.searchsorted(s["active"], idx.clamp(min=0)).clamp(max=A - 1)
    number = torch.where(idx < 0, A, number)
    order = torch.sort(number, stable=True).indices
    count = torch.zeros(A + 1, dtype=torch.int64, device=GPU).scatter_add_(0, number, torch.ones_like(number))
    place = torch.arange(T, device=GPU) - (count.cumsum(0) - count)[number[order]]
    at = torch.empty_like(number)
    at[order] = torch.where(number[order] < A, number[order] * cap + place, A * cap)
    x = torch.zeros((A * cap + 1, d_model), device=GPU)
    x[at] = s["x"].float()
    x = x[:A * cap].view(A, cap, d_model).transpose(1, 2).contiguous()
    for name, cols in (("wi", case["d_model"]), ("wo", case["d_ff"])):
        w, scale, zero = (None if v is None else v[s["active"]] for v in s[name])
        x = torch.bmm(_weights(w, scale, zero, cols, case["group"]), x)
        if name == "wi":  # the hidden vector is bf16 by the operator's definition
            x = _activated(x, case["act"]).to(torch.bfloat16).float()
    y = torch.cat((x.transpose(1, 2).reshape(A * cap, d_model), torch.zeros((1, d_model), device=GPU)))[at]
    return (y * s["gate"].view(-1, 1) * (idx >= 0).view(-1, 1)).to(torch.bfloat16)


def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        import paper_2310_16795_amd as q
        if op == "norm":
            q.qmoe_residual_norm(s["h"], s["y"], s["h_out"], s["x"], k=case["k"], gate=s["gate"], post=s["post"], alpha=0.5,
                                 channel_scale=s["channel"], pre=s["pre"], copies=case["copies"])
            return s["h_out"], s["x"]
        if op == "route":
            q.qmoe_route(s["logits"], s["idx"], s["gate"], bias=s["bias"], token_mask=s["mask"],
                         gates=q.GATES_ALL if case["gates"] == "all" else q.GATES_CHOSEN)
            return s["idx"], s["gate"]
        if op == "int4":
            q.qmoe_int4_matvec(s["matrix"].desc, s["x"], s["y"], activation=q.ACTIVATIONS[case["act"]])
            return s["y"]
        s["layer"].forward(s["x"], s["idx"], s["y"], s["ws"], s["gate"])
        return s["y"]
    if op == "norm":
        return _plain_norm(s, case)
    if op == "route":
        return _plain_route(s, case)
    if op == "int4":
        v = torch.matmul(s["x"].float(), _weights(s["w"], s["scale"], s["zero"], case["cols"], case["group"]).t())
        return _activated(v, case["act"]).to(s["y"].dtype)
    return _plain_layer(s, case)


# ---------------------------------------------------------------- from the definitions, in 64 bits

def _exact_matrix(w, scale, zero, cols, group):
    """One matrix [rows, cols] in 64 bits, by blocks, words and halves of words."""
    rows = w.shape[0]
    words = w.contiguous().view(torch.int32).view(rows, -1, 4, 4).transpose(2, 3)  # [row][block][s][q]
    shifts = torch.tensor([0, 16, 4, 20, 8, 24, 12, 28], dtype=torch.int32, device=w.device)
    q = ((words.unsqueeze(-1) >> shifts) & 15).reshape(rows, -1)[:, :cols].double()
    z = torch.full_like(scale, 8.0).double() if zero is None else zero.double()
    return (q - z.repeat_interleave(group, dim=1)[:, :cols]) * scale.double().repeat_interleave(group, dim=1)[:, :cols]


def _exact_act(v, act):
    """v [tokens, rows]."""
    if act in ("none", "relu"):
        return v.clamp(min=0) if act == "relu" else v
    g, u = v.chunk(2, dim=1)
    if act == "silu":
        return g * torch.special.expit(g) * u
    return g * 0.5 * (torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)) + 1) * u


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        def norm(v, side):
            if case[side] == "none":
                return v
            var, mean = torch.var_mean(v, dim=1, unbiased=False, keepdim=True)
            if case[side] == "rms":
                var, mean = var + mean * mean, 0.0
            v = (v - mean) / torch.sqrt(var + 1e-6) * s[side + "_weight"].double()
            return v if s[side + "_bias"] is None else v + s[side + "_bias"].double()
        y = s["y"].double() * (1.0 if s["gate"] is None else s["gate"].double().unsqueeze(1))
        b = norm(sum(y[j::case["k"]] for j in range(case["k"])), "post")
        h = s["h"].double() + 0.5 * b * (1.0 if s["channel"] is None else s["channel"].double())
        x = norm(h, "pre")
        return h, torch.stack([x] * case["copies"], dim=1).flatten(0, 1)
    if op == "route":
        l = s["logits"].double()
        # the choice is defined on the sum rounded to 32 bits; equal ones go to the lowest index
        key = (l if s["bias"] is None else l + s["bias"].double()).float().cpu().numpy()
        idx = torch.from_numpy(np.argsort(-key, axis=1, kind="stable")[:, :case["k"]].copy()).to(GPU)
        if case["gates"] == "all":
            gate = torch.softmax(l, dim=1).gather(1, idx)
        else:
            gate = torch.softmax(l.gather(1, idx), dim=1)
        if s["mask"] is not None:
            gate, idx = gate * (s["mask"] != 0).double().unsqueeze(1), idx.masked_fill((s["mask"] == 0).unsqueeze(1), -1)
        return idx.to(torch.int32), gate
    if op == "int4":
        m = _exact_matrix(s["w"], s["scale"], s["zero"], case["cols"], case["group"])
        return _exact_act(s["x"].double() @ m.t(), case["act"])
    y = torch.zeros(s["y"].shape, dtype=torch.float64, device=GPU)
    for e in s["active"].tolist():
        rows = (s["idx"] == e).nonzero().flatten()
        wi, wo = ([None if v is None else v[e] for v in s[name]] for name in ("wi", "wo"))
        hidden = _exact_act(s["x"][rows].double() @ _exact_matrix(*wi, case["d_model"], case["group"]).t(), case["act"])
        y[rows] = hidden.to(torch.bfloat16).double() @ _exact_matrix(*wo, case["d_ff"], case["group"]).t()
    return y * s["gate"].double().unsqueeze(1)


# ---------------------------------------------------------------- what a pass cannot do without

def _active(case):
    """Experts that receive a row, about."""
    E, n = case["experts"], case["tokens"] * case["k"] * (1.0 - case["padded"])
    p = np.full(E, 1.0 / E) if case["routing"] == "uniform" else _zipf(E)
    return float((1.0 - (1.0 - p) ** n).sum())


def _matrix_bytes(rows, cols, group, zeros):
    return rows * (cols / 2 + (cols + group - 1) // group * (3 if zeros else 2))


def work(case):
    """Every input once and every output once; a multiplication and an addition for every weight and token."""
    op = case["op"]
    if op == "norm":
        values = case["tokens"] * case["d"]
        size = {"f32": 4, "bf16": 2}
        return {"bytes": values * (2 * size[case["h"]] + case["k"] * size[case["y"]] + 2 * case["copies"]),
                "flops": values * (2 * case["k"] + 6 + (4 if case["post"] != "none" else 0))}
    if op == "route":
        values = case["tokens"] * case["experts"]
        return {"bytes": values * (4 if case["logits"] == "f32" else 2) + 8 * case["tokens"] * case["k"],
                "flops": values * (case["k"] + (3 if case["gates"] == "all" else 0))}
    if op == "int4":
        rows, cols, b = case["rows"], case["cols"], case["batch"]
        out = 4 * rows if case["act"] == "none" else 2 * rows if case["act"] == "relu" else rows
        return {"bytes": _matrix_bytes(rows, cols, case["group"], case["zeros"]) + b * (2 * cols + out), "flops": 2 * rows * cols * b}
    d_model, d_ff, T = case["d_model"], case["d_ff"], case["tokens"] * case["k"]
    rows = d_ff if case["act"] == "relu" else 2 * d_ff
    matrices = _matrix_bytes(rows, d_model, case["group"], case["zeros"]) + _matrix_bytes(d_model, d_ff, case["group"], case["zeros"])
    return {"bytes": _active(case) * matrices + T * (4 * d_model + 8),
            "flops": 2 * T * (1.0 - case["padded"]) * (rows * d_model + d_model * d_ff)}
