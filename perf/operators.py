"""The operators of a feed-forward sublayer in training and serving, as cases that can be timed and compared.

A case is one pass through the public entry points of ``paper_2110_15362_amd.block`` on device tensors:

* ``gated_forward``   h = act(x Wg^T) * (x Wu^T): both projections, the activation and the product
* ``gated_step``      the same, kept for backward, and the gradients of x, Wg and Wu
* ``norms_forward``   what stands between two blocks: out = residual_scale x + scale gate * norm(block) wp, y = norm(out) wn
* ``norms_step``      the same and the gradients of x, block, gate and both weights
* ``clip``            the global norm over many gradients, and the gradients scaled to at most max_norm

``own`` says which side runs: the plain form (elementary torch operations in 32 bits) or the framework's kernels.
"""
import math
import random

import torch

own = False

_DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_EPS_NORM, _EPS_CLIP = 1e-6, 1e-6
_TOKENS = 8 * 2048                                          # a batch of the transformer MLP that the workloads hold, [8, 2048, .]
_MOST_FLOPS = 12.0 * _TOKENS * 2048 * 8192                  # of the largest listed step; fp32 an eighth of it, as its products take that much longer
_MOST_CELLS = _TOKENS * 4096                                # elements of the largest listed residual stream
_MOST_GRADS = 24 * (3 * 2048 * 8192 + 2 * 2048)             # and of the largest listed set of gradients


def listed():
    return [
        # one token through one layer, answering: the weights are read once, latency counts
        {"name": "gated_token_bf16", "op": "gated_forward", "dtype": "bf16", "rows": 1, "d": 1024, "f": 4096, "activation": "silu"},
        # a batch of sequences answering token by token, with a hidden size that no tile divides
        {"name": "gated_decode_f16_ragged", "op": "gated_forward", "dtype": "f16", "rows": 37, "d": 4096, "f": 11003, "activation": "gelu_tanh"},
        # the prompts of the transformer MLP [8, 2048, .], hidden size 4096, ReLU gates
        {"name": "gated_prompts_bf16", "op": "gated_forward", "dtype": "bf16", "rows": _TOKENS, "d": 1024, "f": 4096, "activation": "relu"},
        # a training step of a large layer: the largest products
        {"name": "gated_step_bf16", "op": "gated_step", "dtype": "bf16", "rows": _TOKENS, "d": 2048, "f": 8192, "activation": "silu"},
        # a training step on 500 rows in single precision, sizes odd, gates of ReLU
        {"name": "gated_step_f32_ragged", "op": "gated_step", "dtype": "f32", "rows": 500, "d": 1001, "f": 2731, "activation": "relu"},
        # one token between two blocks, answering
        {"name": "norms_token_bf16", "op": "norms_forward", "dtype": "bf16", "rows": 1, "cols": 4096, "gate_rows": 1},
        # the prompts between two blocks, one gate for each of the 8 sequences
        {"name": "norms_prompts_bf16", "op": "norms_forward", "dtype": "bf16", "rows": _TOKENS, "cols": 4096, "gate_rows": 8},
        # a training step on 8192 rows of 1024 features in single precision, one gate for all rows (a scale for each channel)
        {"name": "norms_step_f32", "op": "norms_step", "dtype": "f32", "rows": 8192, "cols": 1024, "gate_rows": 1},
        # a training step with odd sizes, a gate for each token
        {"name": "norms_step_bf16_ragged", "op": "norms_step", "dtype": "bf16", "rows": 4095, "cols": 1999, "gate_rows": 4095},
        # weights and biases of an MLP of four layers of 1024 features: few tensors, launches count
        {"name": "clip_mlp_f32", "op": "clip", "dtype": "f32", "set": "mlp", "max_norm": 1.0},
        # the parameters of a ResNet-50: 161 tensors from 64 elements to 2.4 million
        {"name": "clip_resnet50_f32", "op": "clip", "dtype": "f32", "set": "resnet50", "max_norm": 1.0},
        # 24 layers of gated blocks in bf16 with their norms' weights in fp32: the largest set
        {"name": "clip_layers_bf16", "op": "clip", "dtype": "bf16", "set": "layers", "max_norm": 1.0},
    ]


def _log(rng, low, high):
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def draw(rng):
    """One more case of the same ranges; none costs more than the largest listed one of its operator."""
    op = rng.choice(("gated_forward", "gated_forward", "gated_step", "norms_forward", "norms_step", "clip"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    if op.startswith("gated"):
        def width(high):
            n = _log(rng, 64, high)
            return n if rng.random() < 0.3 else (n + 7) // 8 * 8
        d, f = width(4096), width(16384)
        most = _MOST_FLOPS / (8 if dtype == "f32" else 1)
        rows = _log(rng, 1, max(1, min(_TOKENS, int(most / (12.0 * d * f)))))
        return {"op": op, "dtype": dtype, "rows": rows, "d": d, "f": f, "activation": rng.choice(("relu", "silu", "gelu_tanh"))}
    if op.startswith("norms"):
        cols = _log(rng, 64, 16384)
        if rng.random() < 0.6:
            cols = (cols + 7) // 8 * 8
        rows = _log(rng, 1, max(1, min(_TOKENS, _MOST_CELLS // (cols * (2 if dtype == "f32" else 1)))))
        gate_rows = rng.choice((1, "samples", rows))
        if gate_rows == "samples":
            gate_rows = min(rows, rng.randint(2, 16))
            rows = rows // gate_rows * gate_rows
        return {"op": op, "dtype": dtype, "rows": rows, "cols": cols, "gate_rows": gate_rows}
    return {"op": op, "dtype": dtype, "set": "random", "count": _log(rng, 1, 600), "sizes": rng.randrange(1 << 30),
            "max_norm": rng.choice((1.0, 1.0, 1e6))}


# ---- inputs ---------------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, dtype, *shape, std=1.0, mean=0.0):
    return torch.randn(shape, generator=g, device="cuda").mul_(std).add_(mean).to(dtype)


def _on_grid(t, step):
    return t.float().div_(step).round_().mul_(step).to(t.dtype)


def _resnet50():
    """Elements of a ResNet-50's parameters: convolutions, their norms' weights and biases, and the classifier."""
    sizes, width = [3 * 64 * 49, 64, 64], 64
    for planes, blocks in ((64, 3), (128, 4), (256, 6), (512, 3)):
        for b in range(blocks):
            sizes += [width * planes, planes, planes, 9 * planes * planes, planes, planes, 4 * planes * planes, 4 * planes, 4 * planes]
            if b == 0:
                sizes += [width * 4 * planes, 4 * planes, 4 * planes]
            width = 4 * planes
    return sizes + [2048 * 1000, 1000]


def _clip_set(case):
    """(elements, type) of each gradient of the set."""
    dtype = case["dtype"]
    if case["set"] == "mlp":
        return [(n, dtype) for _ in range(4) for n in (1024 * 1024, 1024)]
    if case["set"] == "resnet50":
        return [(n, dtype) for n in _resnet50()]
    if case["set"] == "layers":
        return [(n, t) for _ in range(24) for n, t in ((2048, "f32"), (2048 * 8192, dtype), (2048 * 8192, dtype), (8192 * 2048, dtype), (2048, "f32"))]
    rng, left, sizes = random.Random(case["sizes"]), _MOST_GRADS // 2, []
    for _ in range(case["count"]):
        n = min(_log(rng, 1, 1 << 24), left)
        if n > 0:
            sizes.append((n, dtype if n > 20000 or rng.random() < 0.5 else "f32"))
            left -= n
    return sizes


def _inputs(case, seed):
    g, op = _gen(seed), case["op"]
    dtype = _DTYPES[case["dtype"]]
    if op.startswith("gated"):
        rows, d, f = case["rows"], case["d"], case["f"]
        s = {"x": _normal(g, dtype, rows, d), "w_gate": _normal(g, dtype, f, d, std=d ** -0.5), "w_up": _normal(g, dtype, f, d, std=d ** -0.5)}
        if case["activation"] == "relu":
            # the gradient jumps where a ReLU closes: values on a grid so coarse that 32-bit sums are exact in any order, so that every
            # side closes the same gates
            s = {"x": _on_grid(s["x"], 2.0 ** -5), "w_gate": _on_grid(s["w_gate"], 2.0 ** -12), "w_up": s["w_up"]}
        if op == "gated_step":
            s["grad_h"] = _normal(g, dtype, rows, f, std=0.1)
        return s
    if op.startswith("norms"):
        rows, cols = case["rows"], case["cols"]
        s = {"x": _normal(g, dtype, rows, cols), "block": _normal(g, dtype, rows, cols, std=2.0), "gate": _normal(g, dtype, case["gate_rows"], cols, std=0.5),
             "post_weight": _normal(g, dtype, cols, std=0.1, mean=1.0), "pre_weight": _normal(g, dtype, cols, std=0.1, mean=1.0)}
        if op == "norms_step":
            s["grad_out"], s["grad_y"] = _normal(g, dtype, rows, cols, std=0.1), _normal(g, dtype, rows, cols, std=0.1)
        return s
    return {"grads": [_normal(g, _DTYPES[t], n, std=0.01) for n, t in _clip_set(case)]}


def _flat(grads, types):
    """A buffer of zeros for all gradients of each type, and each gradient's part of it (from a 256-byte step on, as an allocator would place it):
    where an optimizer reads them."""
    ends, starts = dict.fromkeys(types, 0), []
    for t in grads:
        starts.append(ends[t.dtype])
        ends[t.dtype] += (t.numel() + 127) // 128 * 128
    flat = {d: torch.zeros(ends[d], dtype=types[d], device="cuda") for d in types}
    return {str(d).split(".")[1]: t for d, t in flat.items()}, [flat[t.dtype][a:a + t.numel()] for t, a in zip(grads, starts)]


_SCALES = {"scale": 0.5, "residual_scale": 0.875}


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["op"] == "clip":
        s["flat"], s["outs"] = _flat(s["grads"], {t.dtype: t.dtype for t in s["grads"]})
    if not own:
        return s
    # the buffers that a program keeps from step to step
    from paper_2110_15362_amd import block
    op, dtype = case["op"], _DTYPES[case["dtype"]]
    empty = lambda *shape, dtype=dtype: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    if op.startswith("gated"):
        rows, d, f = case["rows"], case["d"], case["f"]
        s.update(h=empty(rows, f), gate=None, up=None, workspace=block.new_gated_workspace(rows, d, f, dtype, backward=op == "gated_step"))
        if op == "gated_step":
            s.update(gate=empty(rows, f), up=empty(rows, f), grad_x=empty(rows, d), grad_w_gate=empty(f, d), grad_w_up=empty(f, d))
    elif op.startswith("norms"):
        rows, cols = case["rows"], case["cols"]
        s.update(out=empty(rows, cols), y=empty(rows, cols), stats=None)
        if op == "norms_step":
            s.update(stats=empty(2, rows, dtype=torch.float32), grad_x=empty(rows, cols), grad_block=empty(rows, cols), grad_gate=empty(case["gate_rows"], cols),
                     grad_post_weight=empty(cols), grad_pre_weight=empty(cols),
                     workspace=block.new_residual_norm_workspace(rows, cols, case["gate_rows"], dtype))
    else:
        s.update(norm=empty(1, dtype=torch.float32), workspace=block.new_clip_workspace(s["grads"]))
    return s


# ---- the plain forms --------------------------------------------------------------------------------------------

def _activation(name, g):
    """act(g) and act'(g)."""
    if name == "relu":
        return torch.where(g <= 0, 0.0, g), torch.where(g <= 0, 0.0, 1.0)
    if name == "silu":
        s = 1.0 / (1.0 + torch.exp(-g))
        return g * s, s * (1.0 + g * (1.0 - s))
    c = math.sqrt(2.0 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * c * (1.0 + 3.0 * 0.044715 * g * g)


def _plain_gated(s, case):
    dtype = s["x"].dtype
    x, wg, wu = s["x"].float(), s["w_gate"].float(), s["w_up"].float()
    g, u = x @ wg.t(), x @ wu.t()
    a, slope = _activation(case["activation"], g)
    h = (a * u).to(dtype)
    if case["op"] == "gated_forward":
        return {"h": h}
    dh = s["grad_h"].float()
    dg, du = dh * u * slope, dh * a
    return {"h": h, "grad_x": (dg @ wg + du @ wu).to(dtype), "grad_w_gate": (dg.t() @ x).to(dtype), "grad_w_up": (du.t() @ x).to(dtype)}


def _plain_norms(s, case):
    dtype, rows, cols, groups = s["x"].dtype, case["rows"], case["cols"], case["gate_rows"]
    scale, keep = _SCALES["scale"], _SCALES["residual_scale"]
    x, b, wp, wn = s["x"].float(), s["block"].float(), s["post_weight"].float(), s["pre_weight"].float()
    gate = s["gate"].float().unsqueeze(1)                                  # [groups, 1, cols] against [groups, rows of a group, cols]
    grouped = lambda t: t.reshape(groups, rows // groups, cols)  # noqa: E731
    rb = torch.rsqrt((b * b).mean(dim=1, keepdim=True) + _EPS_NORM)
    z = b * rb
    out = keep * x + scale * (gate * grouped(z * wp)).reshape(rows, cols)
    ro = torch.rsqrt((out * out).mean(dim=1, keepdim=True) + _EPS_NORM)
    v = out * ro
    result = {"out": out.to(dtype), "y": (v * wn).to(dtype)}
    if case["op"] == "norms_forward":
        return result
    go, gy = s["grad_out"].float(), s["grad_y"].float()
    gv = gy * wn
    total = go + ro * (gv - v * (gv * v).mean(dim=1, keepdim=True))
    branch = scale * grouped(total)
    dn = (branch * gate).reshape(rows, cols)
    dz = dn * wp
    result.update(grad_x=keep * total, grad_block=rb * (dz - z * (dz * z).mean(dim=1, keepdim=True)), grad_gate=(branch * grouped(z * wp)).sum(dim=1),
                  grad_post_weight=(dn * z).sum(dim=0), grad_pre_weight=(gy * v).sum(dim=0))
    return {k: t.to(dtype) for k, t in result.items()}


def _plain_clip(s, case):
    total = torch.stack([(g.float() * g.float()).sum() for g in s["grads"]]).sum().sqrt()
    factor = (case["max_norm"] / (total + _EPS_CLIP)).clamp(max=1.0)
    for g, out in zip(s["grads"], s["outs"]):
        torch.mul(g.float(), factor, out=out)
    return {"norm": total.reshape(1), **s["flat"]}


# ---- one pass ---------------------------------------------------------------------------------------------------

def run(state):
    s, case = state, state["case"]
    op = case["op"]
    if not own:
        return (_plain_gated if op.startswith("gated") else _plain_norms if op.startswith("norms") else _plain_clip)(s, case)
    from paper_2110_15362_amd import block
    if op.startswith("gated"):
        block.bt_gated_forward(s["x"], s["w_gate"], s["w_up"], case["activation"], s["h"], s["gate"], s["up"], s["workspace"])
        if op == "gated_forward":
            return {"h": s["h"]}
        block.bt_gated_backward(s["grad_h"], s["x"], s["w_gate"], s["w_up"], s["gate"], s["up"], case["activation"],
                                s["grad_x"], s["grad_w_gate"], s["grad_w_up"], s["workspace"])
        return {k: s[k] for k in ("h", "grad_x", "grad_w_gate", "grad_w_up")}
    if op.startswith("norms"):
        block.bt_residual_norm_forward(s["x"], s["block"], s["post_weight"], s["gate"], s["pre_weight"], s["out"], s["y"], s["stats"], _EPS_NORM, **_SCALES)
        if op == "norms_forward":
            return {"out": s["out"], "y": s["y"]}
        block.bt_residual_norm_backward(s["grad_out"], s["grad_y"], s["out"], s["block"], s["post_weight"], s["gate"], s["pre_weight"], s["stats"],
                                        s["grad_x"], s["grad_block"], s["grad_post_weight"], s["grad_gate"], s["grad_pre_weight"], s["workspace"], **_SCALES)
        return {k: s[k] for k in ("out", "y", "grad_x", "grad_block", "grad_gate", "grad_post_weight", "grad_pre_weight")}
    block.bt_clip_grads(s["grads"], s["outs"], case["max_norm"], s["norm"], s["workspace"], _EPS_CLIP)
    return {"norm": s["norm"], **s["flat"]}


# ---- what a pass cannot do without, and how exactly it is defined -------------------------------------------------

def work(case):
    op = case["op"]
    if op == "clip":
        # read once for the norm, once more to be scaled, written once
        return {"bytes": sum(3 * n * _DTYPES[t].itemsize for n, t in _clip_set(case)), "flops": sum(3.0 * n for n, _ in _clip_set(case))}
    width = _DTYPES[case["dtype"]].itemsize
    if op.startswith("gated"):
        rows, d, f = case["rows"], case["d"], case["f"]
        if op == "gated_forward":
            return {"bytes": width * (rows * d + 2 * f * d + rows * f), "flops": 4.0 * rows * d * f}
        return {"bytes": width * (2 * rows * d + 4 * f * d + 2 * rows * f), "flops": 12.0 * rows * d * f}
    cells, gate = case["rows"] * case["cols"], case["gate_rows"] * case["cols"]
    if op == "norms_forward":
        return {"bytes": width * (4 * cells + gate + 2 * case["cols"]), "flops": 10.0 * cells}
    return {"bytes": width * (8 * cells + 2 * gate + 4 * case["cols"]), "flops": 34.0 * cells}


def exact(case, seed):
    """The definitions in double precision, their gradients by differentiation."""
    s = _inputs(case, seed)
    if case["op"] == "clip":
        norm = math.sqrt(math.fsum(float(torch.linalg.vector_norm(t.double())) ** 2 for t in s["grads"]))
        factor = min(1.0, case["max_norm"] / (norm + _EPS_CLIP))
        flat, outs = _flat(s["grads"], {t.dtype: torch.float64 for t in s["grads"]})
        for t, out in zip(s["grads"], outs):
            out.copy_(t.double() * factor)
        return {"norm": torch.tensor([norm], dtype=torch.float64, device="cuda"), **flat}
    step = case["op"].endswith("step")
    v = {k: t.double().requires_grad_(step and not k.startswith("grad")) for k, t in s.items()}
    f = torch.nn.functional
    if case["op"].startswith("gated"):
        g = f.linear(v["x"], v["w_gate"])
        a = f.relu(g) if case["activation"] == "relu" else f.silu(g) if case["activation"] == "silu" else f.gelu(g, approximate="tanh")
        h = a * f.linear(v["x"], v["w_up"])
        result, roots = {"h": h.detach()}, ((h, v.get("grad_h")),)
        names = ("x", "w_gate", "w_up")
    else:
        cols = case["cols"]
        norm = lambda t: t / (t.square().sum(dim=1, keepdim=True) / cols + _EPS_NORM).sqrt()  # noqa: E731
        gate = v["gate"].repeat_interleave(case["rows"] // case["gate_rows"], dim=0)
        out = v["x"] * _SCALES["residual_scale"] + norm(v["block"]) * v["post_weight"] * gate * _SCALES["scale"]
        y = norm(out) * v["pre_weight"]
        result, roots = {"out": out.detach(), "y": y.detach()}, ((out, v.get("grad_out")), (y, v.get("grad_y")))
        names = ("x", "block", "gate", "post_weight", "pre_weight")
    if step:
        grads = torch.autograd.grad([r for r, _ in roots], [v[k] for k in names], [t for _, t in roots])
        result.update(("grad_" + k, t) for k, t in zip(names, grads))
    return result
