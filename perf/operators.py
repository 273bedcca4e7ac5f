"""The calls of the feed-forward operators whose time matters to users of this library, as a list and as a way to draw more of them.

A case is one call: the quantisation of an activation or of a weight to 8-bit floats with a scale for each block of 128, the matrix
product of two such operands, the gated projection (bf16, fp32, and 8-bit operands), or its backward pass (with the projections that
the forward pass kept, or computing them again).  Tokens go from the single one of a decoding step to a training batch.  Sizes that
are powers of two and sizes that are nothing of the kind; some activations are columns of a wider array, some tokens are padding (zeros).

Where `own` is true, `run` calls the library; else it computes the same from elementary torch operations in 32 bits.
"""
import math

import torch

own = False

_BLOCK = 128
_E4M3_MAX = 448.0
_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
_SIZE = {"f32": 4, "bf16": 2, "e4m3": 1}
_ACTIVATIONS = ("silu", "gelu", "gelu_tanh")

# a drawn case costs at most what the largest listed one does
_MAX_FLOPS = 2.2e12
_MAX_BYTES = 0.8e9


def _quantize(dtype, T, C, block_rows, pad=0, name=None):
    case = {"op": "quantize", "dtype": dtype, "T": T, "C": C, "block_rows": block_rows, "pad": pad}
    return case if name is None else {**case, "name": name}


def _matmul(out, T, C, K, pad=0, name=None):
    case = {"op": "matmul", "dtype": "e4m3", "out": out, "T": T, "C": C, "K": K, "pad": pad}
    return case if name is None else {**case, "name": name}


def _forward(dtype, T, C, F, activation, keep=False, pad=0, name=None):
    case = {"op": "forward", "dtype": dtype, "T": T, "C": C, "F": F, "activation": activation, "keep": keep, "pad": pad}
    return case if name is None else {**case, "name": name}


def _backward(dtype, T, C, F, activation, keep, pad=0, name=None):
    case = {"op": "backward", "dtype": dtype, "T": T, "C": C, "F": F, "activation": activation, "keep": keep, "pad": pad}
    return case if name is None else {**case, "name": name}


def listed():
    return [
        # one token's activations before a product in 8 bits: latency and nothing else
        _quantize("bf16", 1, 4096, 1, name="quantize_b1"),
        # a master weight to 8 bits, blocks of 128 x 128
        _quantize("f32", 8192, 4096, 128, name="quantize_weight"),
        # a decoding step of one sequence: the weight is read once, that is all
        _matmul("bf16", 1, 4096, 8192, name="matmul_b1"),
        # a decoding step of a batch of sequences
        _matmul("bf16", 64, 8192, 4096, name="matmul_b64"),
        # nothing divides anything, and 32-bit results
        _matmul("f32", 517, 1000, 1111, name="matmul_ragged"),
        # a long prompt
        _matmul("bf16", 8192, 8192, 4096, name="matmul_prompt"),
        # a decoding step of one sequence with weights in bf16, and of sixteen with weights in 8 bits
        _forward("bf16", 1, 4096, 8192, "silu", name="forward_b1"),
        _forward("e4m3", 16, 4096, 8192, "silu", name="forward_e4m3_b16"),
        # a small model in full precision with sizes that nothing divides
        _forward("f32", 301, 515, 1031, "gelu", pad=3, name="forward_f32_ragged"),
        # the forward pass of a training step, which keeps both projections
        _forward("bf16", 8192, 4096, 8192, "silu", keep=True, name="forward_train"),
        # a backward pass that computes the projections again, sizes that nothing divides
        _backward("bf16", 777, 1001, 1515, "gelu_tanh", False, name="backward_ragged"),
        # the backward pass of a training step
        _backward("bf16", 8192, 4096, 8192, "silu", True, name="backward_train"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _size(rng, lo, hi):
    """Half of the sizes are multiples of 128, a quarter of 16, the others any number."""
    n, kind = _log_int(rng, lo, hi), rng.random()
    step = 128 if kind < 0.5 else 16 if kind < 0.75 else 1
    return max(step, (n + step // 2) // step * step)


def draw(rng):
    while True:
        op = rng.choice(("quantize", "matmul", "matmul", "forward", "forward", "forward", "backward", "backward"))
        T = 2 ** rng.randint(0, 13) if rng.random() < 0.4 else _log_int(rng, 1, 8192)
        C, F = _size(rng, 64, 8192), _size(rng, 64, 16384)
        pad = 0 if rng.random() < 0.8 else rng.choice((1, 8, 64, 129))
        if op == "quantize":
            block_rows = rng.choice((1, 1, 128))
            case = _quantize(rng.choice(("f32", "bf16", "bf16")), F if block_rows == 128 else T, C, block_rows, pad)
        elif op == "matmul":
            case = _matmul(rng.choice(("bf16", "bf16", "f32")), T, C, F, pad)
        elif op == "forward":
            dtype = rng.choice(("bf16", "bf16", "e4m3", "e4m3", "f32"))
            case = _forward(dtype, T, C, F, rng.choice(_ACTIVATIONS), dtype != "e4m3" and rng.random() < 0.5, pad)
        else:
            case = _backward(rng.choice(("bf16", "bf16", "f32")), T, C, F, rng.choice(_ACTIVATIONS), rng.random() < 0.5, pad)
        w = work(case)
        if w["flops"] <= _MAX_FLOPS and w["bytes"] <= _MAX_BYTES:
            return case


def _columns(t, pad):
    """`t` as the first columns of an array that has `pad` more."""
    if not pad:
        return t
    wide = torch.zeros((t.shape[0], t.shape[1] + pad), dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def _scaled(t, block_rows):
    """An operand as a file of weights in 8 bits has it: every block's largest value is 448 times its scale."""
    rows, cols = t.shape
    blocks = torch.nn.functional.pad(t, (0, -cols % _BLOCK, 0, -rows % block_rows))
    blocks = blocks.view(-1, block_rows, blocks.shape[1] // _BLOCK, _BLOCK)
    scale = blocks.abs().amax((1, 3)) / _E4M3_MAX
    scale = torch.where(scale > 0, scale, torch.ones_like(scale))
    q = (blocks / scale[:, None, :, None]).clamp(-_E4M3_MAX, _E4M3_MAX).view(-1, blocks.shape[2] * _BLOCK)
    return q[:rows, :cols].to(torch.float8_e4m3fn).contiguous(), scale.contiguous()


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    T, C, typ = case["T"], case["C"], _TORCH[case["dtype"]]
    # activations: some channels are larger than others, and every eleventh token is padding
    x = normal(T, C) * (normal(C) * 0.5).exp()
    if T > 1 and case.get("block_rows", 1) == 1:
        x[10::11] = 0
    if case["op"] == "quantize":
        return {"x": _columns(x.to(typ), case["pad"])}
    if case["op"] == "matmul":
        xq, xs = _scaled(x, 1)
        wq, ws = _scaled(normal(case["K"], C) / math.sqrt(C), _BLOCK)
        return {"x": _columns(xq, case["pad"]), "x_scale": xs, "w": wq, "w_scale": ws}
    F = case["F"]
    wg, wu = normal(F, C) / math.sqrt(C), normal(F, C) / math.sqrt(C)
    if case["dtype"] == "e4m3":
        xq, xs = _scaled(x, 1)
        (gq, gs), (uq, us) = _scaled(wg, _BLOCK), _scaled(wu, _BLOCK)
        return {"x": _columns(xq, case["pad"]), "x_scale": xs, "w_gate": gq, "w_gate_scale": gs, "w_up": uq, "w_up_scale": us}
    data = {"x": _columns(x.to(typ), case["pad"]), "w_gate": wg.to(typ), "w_up": wu.to(typ)}
    if case["op"] == "backward":
        data["grad_out"] = (normal(T, F) * 1e-3).to(typ)
        if case["keep"]:
            x32 = data["x"].float()
            data["gate"] = (x32 @ data["w_gate"].float().t()).to(typ)
            data["up"] = (x32 @ data["w_up"].float().t()).to(typ)
    return data


def prepare(case, seed):
    state = {"case": dict(case), **_inputs(case, seed)}

    def empty(*shape, dtype):
        return torch.empty(shape, device="cuda", dtype=dtype)

    T, C, typ = case["T"], case["C"], _TORCH[case["dtype"]]
    if case["op"] == "quantize":
        rows = -(-T // case["block_rows"])
        state["q"] = empty(T, C, dtype=torch.float8_e4m3fn)
        state["scale"] = empty(rows, -(-C // _BLOCK), dtype=torch.float32)
    elif case["op"] == "matmul":
        state["y"] = empty(T, case["K"], dtype=_TORCH[case["out"]])
    elif case["op"] == "forward":
        state["y"] = empty(T, case["F"], dtype=torch.bfloat16 if case["dtype"] == "e4m3" else typ)
        if case["keep"]:
            state["gate"], state["up"] = empty(T, case["F"], dtype=typ), empty(T, case["F"], dtype=typ)
    else:
        state["grad_x"] = empty(T, C, dtype=typ)
        state["grad_w_gate"], state["grad_w_up"] = empty(case["F"], C, dtype=typ), empty(case["F"], C, dtype=typ)
    return state


def _run_own(state):
    import paper_1802_06905_amd as cc
    case = state["case"]
    T, C = case["T"], case["C"]
    code = {"f32": cc.CACNN_F32, "bf16": cc.CACNN_BF16_F32ACC}
    if case["op"] == "quantize":
        cc.cacnn_quantize((T, C, case["block_rows"]), code[case["dtype"]], state["x"], state["q"], state["scale"])
        return [state["q"], state["scale"]]
    if case["op"] == "matmul":
        cc.cacnn_matmul_scaled((T, C, case["K"]), state["x"], state["x_scale"], state["w"], state["w_scale"], code[case["out"]], state["y"])
        return [state["y"]]
    activation = {"silu": cc.CACNN_GATE_SILU, "gelu": cc.CACNN_GATE_GELU, "gelu_tanh": cc.CACNN_GATE_GELU_TANH}[case["activation"]]
    problem = (T, C, case["F"], activation)
    if case["op"] == "forward":
        if case["dtype"] == "e4m3":
            cc.cacnn_gated_forward_scaled(problem, state["x"], state["x_scale"], state["w_gate"], state["w_gate_scale"], state["w_up"],
                                          state["w_up_scale"], cc.CACNN_BF16_F32ACC, state["y"])
            return [state["y"]]
        cc.cacnn_gated_forward(problem, code[case["dtype"]], state["x"], state["w_gate"], state["w_up"], state["y"],
                               gate=state.get("gate"), up=state.get("up"))
        return [state["y"], state["gate"], state["up"]] if case["keep"] else [state["y"]]
    workspace = torch.empty(cc.cacnn_gated_workspace(problem, code[case["dtype"]]), dtype=torch.uint8, device="cuda")
    cc.cacnn_gated_backward(problem, code[case["dtype"]], state["x"], state["w_gate"], state["w_up"], state["grad_out"], state["grad_x"],
                            state["grad_w_gate"], state["grad_w_up"], workspace, gate=state.get("gate"), up=state.get("up"))
    return [state["grad_x"], state["grad_w_gate"], state["grad_w_up"]]


def _values(q, scale, block_rows):
    """What an operand in 8 bits stands for, in 32 bits."""
    rows, cols = q.shape
    by_value = scale.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(_BLOCK, 1)[:, :cols]
    return q.float() * by_value


def _activate(name, g):
    """The activation and its derivative at g."""
    if name == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    if name == "gelu":
        p = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * p, p + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    k = math.sqrt(2 / math.pi)
    t = torch.tanh(k * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * k * (1 + 3 * 0.044715 * g * g)


def _run_plain(state):
    case = state["case"]
    x = state["x"]
    if case["op"] == "quantize":
        T, C, rows = case["T"], case["C"], case["block_rows"]
        blocks = torch.nn.functional.pad(x.float(), (0, -C % _BLOCK, 0, -T % rows))
        blocks = blocks.view(-1, rows, blocks.shape[1] // _BLOCK, _BLOCK)
        largest = blocks.abs().amax((1, 3))
        # largest = mantissa * 2^exponent with the mantissa in [0.5, 1), and 448 = 0.875 * 2^9
        mantissa, exponent = torch.frexp(largest)
        exponent = torch.where(largest > 0, torch.clamp(exponent - 9 + (mantissa > 0.875), min=-126), 0)
        scale = torch.ldexp(torch.ones_like(largest), exponent)
        q = (blocks / scale[:, None, :, None]).view(-1, blocks.shape[2] * _BLOCK)[:T, :C].to(torch.float8_e4m3fn)
        return [q, scale]
    if case["op"] == "matmul":
        y = _values(x, state["x_scale"], 1) @ _values(state["w"], state["w_scale"], _BLOCK).t()
        return [y.to(_TORCH[case["out"]])]
    if case["dtype"] == "e4m3":
        x32 = _values(x, state["x_scale"], 1)
        wg, wu = _values(state["w_gate"], state["w_gate_scale"], _BLOCK), _values(state["w_up"], state["w_up_scale"], _BLOCK)
        return [(_activate(case["activation"], x32 @ wg.t())[0] * (x32 @ wu.t())).to(torch.bfloat16)]
    typ = x.dtype
    x32, wg, wu = x.float(), state["w_gate"].float(), state["w_up"].float()
    if case["op"] == "forward":
        g, u = x32 @ wg.t(), x32 @ wu.t()
        y = (_activate(case["activation"], g)[0] * u).to(typ)
        return [y, g.to(typ), u.to(typ)] if case["keep"] else [y]
    g, u = (state["gate"].float(), state["up"].float()) if case["keep"] else (x32 @ wg.t(), x32 @ wu.t())
    a, slope = _activate(case["activation"], g)
    dy = state["grad_out"].float()
    dg, du = dy * u * slope, dy * a
    return [(dg @ wg + du @ wu).to(typ), (dg.t() @ x32).to(typ), (du.t() @ x32).to(typ)]


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    """Every operand read once, every result written once; the products' and sums' operations."""
    T, C = case["T"], case["C"]
    esz, blocks = _SIZE[case["dtype"]], -(-C // _BLOCK)
    if case["op"] == "quantize":
        return {"bytes": T * C * (esz + 1) + 4 * blocks * -(-T // case["block_rows"]), "flops": 2 * T * C}
    if case["op"] == "matmul":
        K = case["K"]
        return {"bytes": T * C + K * C + 4 * blocks * (T + -(-K // _BLOCK)) + T * K * _SIZE[case["out"]], "flops": 2 * T * C * K}
    F = case["F"]
    operands = esz * (T * C + 2 * F * C)
    if case["op"] == "forward":
        if case["dtype"] == "e4m3":
            return {"bytes": operands + 4 * blocks * (T + 2 * -(-F // _BLOCK)) + 2 * T * F, "flops": 4 * T * C * F}
        return {"bytes": operands + esz * T * F * (3 if case["keep"] else 1), "flops": 4 * T * C * F}
    return {"bytes": 2 * operands + esz * T * F * (3 if case["keep"] else 1), "flops": (8 if case["keep"] else 12) * T * C * F}


def _exact_e4m3(y):
    """The nearest number of four exponent and three fraction bits, ties to even, of 64-bit values of at most 448."""
    _, exponent = torch.frexp(y)                       # y = m * 2^exponent, 0.5 <= |m| < 1: the leading bit is 2^(exponent - 1)
    step = torch.ldexp(torch.ones_like(y), torch.clamp(exponent - 1, min=-6) - 3)
    return torch.round(y / step) * step


def _exact_activation(name, g):
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s + g * s * (1 - s)
    if name == "gelu":
        p = 0.5 * torch.erfc(-g / math.sqrt(2))
        return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    # 0.5 (1 + tanh z) = 1 / (1 + exp(-2 z))
    k = math.sqrt(8 / math.pi)
    s = torch.sigmoid(k * g * (1 + 0.044715 * g * g))
    return g * s, s + g * s * (1 - s) * k * (1 + 0.134145 * g * g)


def exact(case, seed):
    data = _inputs(case, seed)
    x = data["x"].double()
    if case["op"] == "quantize":
        T, C, rows = case["T"], case["C"], case["block_rows"]
        q = torch.empty_like(x)
        scale = torch.empty((-(-T // rows), -(-C // _BLOCK)), dtype=torch.float64, device=x.device)
        padded = x if T % rows == 0 else torch.cat((x, x.new_zeros((-T % rows, C))))
        for b in range(scale.shape[1]):
            part = slice(b * _BLOCK, min(C, (b + 1) * _BLOCK))
            largest = padded[:, part].abs().amax(1).view(-1, rows).amax(1)
            power = torch.ceil(torch.log2(torch.where(largest > 0, largest, 448.0) / 448.0)).to(torch.int32)
            # (the logarithm is rounded: one down or up where that is what the definition says)
            one = torch.ones_like(largest)
            power = power - (largest <= 448.0 * torch.ldexp(one, power - 1)).to(torch.int32) * (largest > 0)
            power = power + (largest > 448.0 * torch.ldexp(one, power)).to(torch.int32)
            scale[:, b] = torch.ldexp(one, power)
            q[:, part] = _exact_e4m3(x[:, part] / scale[:, b].repeat_interleave(rows)[:T, None])
        return [q, scale]

    def stands_for(name, block_rows):
        q, s = data[name].double(), data[name + "_scale"].double()
        return q * s.repeat_interleave(block_rows, 0)[:q.shape[0]].repeat_interleave(_BLOCK, 1)[:, :q.shape[1]]

    if case["op"] == "matmul":
        return [torch.mm(stands_for("x", 1), stands_for("w", _BLOCK).t())]
    if case["dtype"] == "e4m3":
        x, wg, wu = stands_for("x", 1), stands_for("w_gate", _BLOCK), stands_for("w_up", _BLOCK)
        return [_exact_activation(case["activation"], torch.mm(x, wg.t()))[0] * torch.mm(x, wu.t())]
    wg, wu = data["w_gate"].double(), data["w_up"].double()
    if case["op"] == "backward" and case["keep"]:
        g, u = data["gate"].double(), data["up"].double()
    else:
        g, u = torch.mm(x, wg.t()), torch.mm(x, wu.t())
    a, slope = _exact_activation(case["activation"], g)
    if case["op"] == "forward":
        return [a * u, g, u] if case["keep"] else [a * u]
    dy = data["grad_out"].double()
    dg, du = dy * u * slope, dy * a
    return [torch.mm(dg, wg) + torch.mm(du, wu), torch.mm(dg.t(), x), torch.mm(du.t(), x)]
