"""The operators around the convolutions in a network that is quantized group-wise to 8 bits, as measurable cases.

* ``op = "norm"``    ``rms_norm_quantize`` (root-mean-square norm, the residual's addition in front of it, codes and
                     scales), and ``dequantize_rows`` of its codes
* ``op = "linear"``  ``Linear.forward``: rows quantized, int8 matrix product with bias, activation (plain or gated) and
                     residual in its epilogue
* ``op = "block"``   the two as a transformer's feed-forward block has them: norm, gated product on the norm's codes,
                     product back with the residual stream added

The quantizer is the convolution's: groups of ``gs`` consecutive channels (0: the whole row), scale = amax / 127,
code = round_half_even(fl32(v * fl32(127 / amax))), both zero where amax < 1e-30.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6


def _norm(rows, C, gs, dtype, residual):
    return dict(op="norm", rows=rows, C=C, gs=gs, dtype=dtype, residual=residual)


def _linear(rows, C, K, gs, dtype, act="none", bias=False, residual=False, gated=False):
    return dict(op="linear", rows=rows, C=C, K=K, gs=gs, dtype=dtype, act=act, bias=bias, residual=residual,
                gated=gated)


def _block(rows, C, K, gs, dtype, act):
    return dict(op="block", rows=rows, C=C, K=K, gs=gs, dtype=dtype, act=act)


def listed():
    named = {
        # one new token in front of a projection: latency of a call
        "norm_token": _norm(1, 4096, 128, "bf16", True),
        # the 64x64 positions of a UNet's latent, two images (classifier-free guidance), first norm of a block
        "norm_unet_f32": _norm(8192, 640, 64, "f32", False),
        # a long prompt, residual stream updated on the way
        "norm_prompt": _norm(16384, 4096, 128, "bf16", True),
        # an odd width: last group short, rows that start on no 16-byte boundary
        "norm_odd": _norm(3001, 1009, 32, "f16", True),
        # serving one token
        "linear_token": _linear(1, 4096, 4096, 128, "bf16", bias=True, residual=True),
        # a batch of 24 sequences that decode together, wide layer
        "linear_decode_24": _linear(24, 4096, 16384, 128, "bf16", act="silu", gated=True),
        # 2 x 77 text tokens into the keys of a UNet's cross attention: odd rows, small groups
        "linear_text_154": _linear(154, 768, 1280, 32, "f16", bias=True),
        # feed-forward product of a UNet block at 64x64: GELU-gated, bias
        "linear_unet_geglu": _linear(4096, 640, 2560, 64, "f16", act="gelu", bias=True, gated=True),
        # a long prompt through a wide product with one scale per row and channel
        "linear_prompt_rowscale": _linear(8192, 4096, 8192, 0, "bf16"),
        # the same with groups of 128, fp32 results for the caller's own code
        "linear_prompt_f32": _linear(4096, 4096, 4096, 128, "f32", bias=True, residual=True),
        # feed-forward block while four sequences decode
        "block_decode_4": _block(4, 2048, 8192, 128, "bf16", "silu"),
        # the same block over a prompt of 2000 tokens
        "block_prompt": _block(2000, 2048, 8192, 128, "bf16", "silu"),
    }
    return [dict(name=name, **case) for name, case in named.items()]


def _effort(case):
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / 5e13


def draw(rng):
    limit = {}
    for c in listed():
        limit[c["op"]] = max(limit.get(c["op"], 0.0), _effort(c))

    def spread(lo, hi, step=1):
        return max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5 * step))) / step)) * step)

    while True:
        op = rng.choice(["norm", "linear", "linear", "block"])
        dtype = rng.choice(["f16", "bf16", "bf16", "f32"])
        gs = rng.choice([32, 64, 128, 128, 256, 96, 0])
        step = rng.choice([64, 64, 8, 1])
        C = max(64, spread(64, 8192, step))
        rows = spread(1, 16384)
        if op == "norm":
            case = _norm(rows, C, gs, dtype, rng.random() < 0.6)
        else:
            K = max(64, spread(64, 16384, rng.choice([64, 64, 8, 1])))
            act = rng.choice(["none", "relu", "silu", "gelu"])
            if op == "linear":
                case = _linear(rows, C, K, gs, dtype, act, rng.random() < 0.5, rng.random() < 0.5,
                               act != "none" and rng.random() < 0.5)
            else:
                case = _block(rows, C, K, gs, dtype, rng.choice(["silu", "gelu"]))
        if _effort(case) <= limit[op]:
            return case


def _activations(gen, rows, C, dtype):
    """Normal values with a few channels that are much larger in every row, as residual streams have them."""
    x = torch.randn((rows, C), generator=gen, device="cuda")
    large = torch.rand((C,), generator=gen, device="cuda") < 0.01
    return (x * torch.where(large, 12.0, 1.0)).to(DTYPES[dtype])


def _weights(gen, K, C, dtype):
    size = torch.exp(0.3 * torch.randn((K, 1), generator=gen, device="cuda")) / math.sqrt(C)
    return (torch.randn((K, C), generator=gen, device="cuda") * size).to(DTYPES[dtype])


def _groups(v, gs, fill=0.0):
    """[rows][C] as [rows][groups][gs], the last group filled up."""
    rows, C = v.shape
    gs = min(gs, C) if gs else C
    G = -(-C // gs)
    if G * gs != C:
        v = torch.nn.functional.pad(v, (0, G * gs - C), value=fill)
    return v.reshape(rows, G, gs)


def _quantized(v, gs):
    """Codes (as fp32) [rows][groups][gs] and scales [rows][groups][1] of fp32 rows."""
    g = _groups(v, gs)
    amax = g.abs().amax(dim=2, keepdim=True)
    some, top = amax >= 1e-30, torch.full_like(amax, 127.0)      # tensors: a quotient with a number is not rounded once
    inv = torch.where(some, top / amax, torch.zeros_like(amax))
    scale = torch.where(some, amax / top, torch.zeros_like(amax))
    return torch.round(g * inv).clamp_(-127.0, 127.0), scale


def _values(codes, scale, C):
    return (codes * scale).reshape(codes.shape[0], -1)[:, :C]


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def _layer(gen, case, C, K, act, gated, bias):
    """One product's weights: as given, their quantized values for the plain form, and, with the framework, its plan."""
    w = _weights(gen, 2 * K if gated else K, C, case["dtype"])
    b = 0.1 * torch.randn((w.shape[0],), generator=gen, device="cuda") if bias else None
    codes, scale = _quantized(w.float(), case["gs"])
    layer = {"C": C, "K": K, "gs": case["gs"], "act": act, "gated": gated, "bias": b, "w": w}
    if own:
        from paper_2412_19867_b200 import binding
        acts = {"none": binding.WFQ_ACT_NONE, "relu": binding.WFQ_ACT_RELU, "silu": binding.WFQ_ACT_SILU,
                "gelu": binding.WFQ_ACT_GELU}
        layer["plan"] = binding.Linear(C, K, case["gs"], case["rows"], case["dtype"], gated=gated)
        layer["plan"].prepare(w)
        layer["plan"].set_epilogue(b, acts[act])
    else:
        layer["values"] = _values(codes, scale, C).contiguous()
    return layer


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows, C, dtype = case["rows"], case["C"], case["dtype"]
    state = {"case": dict(case), "x": _activations(gen, rows, C, dtype)}
    if case["op"] != "linear":
        state["gain"] = 1.0 + 0.2 * torch.randn((C,), generator=gen, device="cuda")
        state["residual"] = _activations(gen, rows, C, dtype) if case.get("residual", True) else None
    if case["op"] == "linear":
        state["layers"] = [_layer(gen, case, C, case["K"], case["act"], case["gated"], case["bias"])]
        state["residual"] = _activations(gen, rows, case["K"], dtype) if case["residual"] else None
    if case["op"] == "block":
        state["layers"] = [_layer(gen, case, C, case["K"], case["act"], True, False),
                           _layer(gen, case, case["K"], C, "none", False, False)]
    return state


def _plain_norm(x, residual, gain, gs):
    """The residual stream (in x's type), codes and scales of the norm's output."""
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    hf = h.float()
    rstd = torch.rsqrt((hf * hf).mean(dim=1, keepdim=True) + EPS)
    codes, scale = _quantized(hf * gain, gs)
    return h, codes, scale * rstd.unsqueeze(2)


def _plain_product(values, layer, residual, dtype):
    """`values`: quantized rows as fp32 values."""
    z = values @ layer["values"].t()
    if layer["bias"] is not None:
        z = z + layer["bias"]
    if layer["gated"]:
        z = _act(z[:, :layer["K"]], layer["act"]) * z[:, layer["K"]:]
    else:
        z = _act(z, layer["act"])
    if residual is not None:
        z = z + residual.float()
    return z.to(dtype)


def run(state):
    case = state["case"]
    op, C, gs, dtype = case["op"], case["C"], case["gs"], DTYPES[case["dtype"]]
    if own:
        from paper_2412_19867_b200 import binding
        if op == "norm":
            q, h = binding.rms_norm_quantize(state["x"], state["gain"], EPS, gs, residual=state["residual"])
            values = binding.dequantize_rows(q, case["dtype"])
            return {"values": values, "h": h} if case["residual"] else {"values": values}
        if op == "linear":
            return {"y": state["layers"][0]["plan"].forward(state["x"], residual=state["residual"])}
        q, h = binding.rms_norm_quantize(state["x"], state["gain"], EPS, gs, residual=state["residual"])
        inner = state["layers"][0]["plan"].forward_codes(q)
        return {"h": h, "y": state["layers"][1]["plan"].forward(inner, residual=h)}
    x = state["x"]
    if op == "norm":
        h, codes, scale = _plain_norm(x, state["residual"], state["gain"], gs)
        values = _values(codes, scale, C).to(dtype)
        return {"values": values, "h": h} if case["residual"] else {"values": values}
    if op == "linear":
        return {"y": _plain_product(_values(*_quantized(x.float(), gs), C), state["layers"][0], state["residual"],
                                    dtype)}
    h, codes, scale = _plain_norm(x, state["residual"], state["gain"], gs)
    inner = _plain_product(_values(codes, scale, C), state["layers"][0], None, dtype)
    return {"h": h, "y": _plain_product(_values(*_quantized(inner.float(), gs), case["K"]), state["layers"][1], h,
                                        dtype)}


def work(case):
    rows, C, gs, e = case["rows"], case["C"], case["gs"], BYTES[case["dtype"]]
    groups = lambda n: -(-n // gs) if gs else 1  # noqa: E731
    if case["op"] == "norm":
        # x and the residual in, the stream out, codes with their scales, and the values they stand for
        n = rows * C * e * (3 if case["residual"] else 1) + rows * (C + 4 * groups(C)) + rows * C * e + 4 * C
        return {"bytes": n, "flops": 6.0 * rows * C}
    if case["op"] == "linear":
        K = case["K"] * (2 if case["gated"] else 1)
        n = K * (C + 4 * groups(C) + (4 if case["bias"] else 0)) + rows * C * e
        n += rows * case["K"] * e * (2 if case["residual"] else 1)
        return {"bytes": n, "flops": 2.0 * rows * C * K}
    K = case["K"]
    n = 3 * K * C + 4 * (2 * K * groups(C) + C * groups(K)) + 4 * rows * C * e + 4 * C
    return {"bytes": n, "flops": 6.0 * rows * C * K}


def _exact_quantizer(v, gs):
    """The definition on 64-bit values that 32 bits hold: its two quotients and its product rounded to 32 bits."""
    to32 = lambda t: t.float().double()  # noqa: E731
    rows, C = v.shape
    width = C if gs == 0 or gs > C else gs
    edges = list(range(0, C, width))
    codes, scales = torch.empty_like(v), torch.empty((rows, len(edges)), dtype=torch.float64, device=v.device)
    for i, lo in enumerate(edges):
        part = v[:, lo:lo + width]
        top = torch.maximum(part.max(dim=1).values, -part.min(dim=1).values)
        live = top >= 1e-30
        safe = torch.where(live, top, torch.ones_like(top))
        codes[:, lo:lo + width] = torch.round(to32(part * to32(127.0 / safe)[:, None])) * live[:, None]
        scales[:, i] = torch.where(live, to32(top / 127.0), torch.zeros_like(top))
    return codes, scales.repeat_interleave(width, dim=1)[:, :C]


def _exact_product(xv, layer, residual, narrow):
    wq, ws = _exact_quantizer(layer["w"].double(), layer["gs"])
    z = torch.einsum("rc,kc->rk", xv, wq * ws)
    if layer["bias"] is not None:
        z += layer["bias"].double()
    f = {"none": lambda t: t, "relu": lambda t: t.clamp(min=0.0), "silu": lambda t: t * torch.sigmoid(t),
         "gelu": lambda t: t * torch.special.ndtr(t)}[layer["act"]]
    z = f(z) if not layer["gated"] else f(z[:, :layer["K"]]) * z[:, layer["K"]:]
    if residual is not None:
        z += residual.double()
    return z if narrow is None else z.to(narrow).double()


def exact(case, seed):
    state = prepare(case, seed)
    dtype, gs, x = DTYPES[case["dtype"]], case["gs"], state["x"].double()
    if case["op"] == "linear":
        xq, xs = _exact_quantizer(x, gs)
        return {"y": _exact_product(xq * xs, state["layers"][0], state["residual"], None)}
    stream = x if state["residual"] is None else (x + state["residual"].double()).to(dtype).double()
    rms = torch.sqrt(stream.square().mean(dim=1, keepdim=True) + EPS)
    codes, scale = _exact_quantizer((stream * state["gain"].double()).float().double(), gs)
    values = codes * scale / rms
    if case["op"] == "norm":
        return {"values": values, "h": stream} if case["residual"] else {"values": values}
    inner = _exact_product(values, state["layers"][0], None, dtype)
    iq, isc = _exact_quantizer(inner, gs)
    return {"h": stream, "y": _exact_product(iq * isc, state["layers"][1], stream, None)}
