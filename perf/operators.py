"""The language-model operators whose speed is measured, with their plain forms.

  quantize   8-bit codes and a factor for each token of an activation tensor (`q8_quantize_tokens`) and the way back
             (`q8_dequantize_tokens`)
  linear     the matrix product of 8-bit codes with a factor per token and per output channel (`q8_linear`), given codes
             or given floating-point activations, which the call quantizes token by token
  moe        a mixture-of-experts layer for a few tokens (`q8_moe`): router, top k, gated experts with 8-bit weights, sum

Sizes: widths that language models of a few billion weights have in serving; ragged ones beside them.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2, "s8": 1}


# ------------------------------------------------------------------------------------------------ the cases
def _quantize(name, T, C, x):
    return {"name": name, "kind": "quantize", "T": T, "C": C, "x": x}


def _linear(name, T, C, K, x, y, pad=0, bias=False):
    """x: "s8" (codes and factors are at hand) or the type of the activations; pad: values between the end of one row of x
    and the start of the next."""
    return {"name": name, "kind": "linear", "T": T, "C": C, "K": K, "x": x, "y": y, "pad": pad, "bias": bias}


def _moe(name, T, C, I, E, k, x, renorm=True):
    return {"name": name, "kind": "moe", "T": T, "C": C, "I": I, "E": E, "k": k, "x": x, "renorm": renorm}


def listed():
    return [
        # the activations of one decoded token: latency of two small calls
        _quantize("quantize_1x4096_bf16", 1, 4096, "bf16"),
        # those of a long prompt: memory bandwidth
        _quantize("quantize_8192x4096_bf16", 8192, 4096, "bf16"),
        # fp32 activations of a ragged batch, rows off the 16-byte grid
        _quantize("quantize_1000x2051_f32", 1000, 2051, "f32"),
        # a projection of one decoded token: the weights' bytes
        _linear("linear_1x4096x4096", 1, 4096, 4096, "bf16", "bf16"),
        # a decoding batch, codes shared by several projections
        _linear("linear_24x2048x5632", 24, 2048, 5632, "s8", "f16"),
        # a short ragged prompt, sizes off the tiles, fp32 results with a bias, x a slice of a wider tensor
        _linear("linear_777x1032x1000", 777, 1032, 1000, "s8", "f32", pad=24, bias=True),
        # prompts: bound by the tensor cores; with the quantization of the activations, and the widest product
        _linear("linear_4096x4096x4096", 4096, 4096, 4096, "bf16", "bf16"),
        _linear("linear_8192x4096x11008", 8192, 4096, 11008, "s8", "bf16"),
        # one token through many small experts, as decoding meets them
        _moe("moe_t1_2048x768_e64k8", 1, 2048, 768, 64, 8, "bf16"),
        # few large experts, two tokens (a drafted token and its successor)
        _moe("moe_t2_4096x2048_e8k2", 2, 4096, 2048, 8, 2, "bf16"),
        # odd sizes in fp32, weights of the softmax over all experts
        _moe("moe_t5_1000x520_e17k2", 5, 1000, 520, 17, 2, "f32", renorm=False),
        # a decoding batch that reaches most experts
        _moe("moe_t16_2048x1024_e64k8", 16, 2048, 1024, 64, 8, "bf16"),
    ]


def _log(rng, lo, hi):
    """A whole number spread over its logarithm; half of them multiples of a power of two, the others as they fall."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5:
        step = 2 ** max(0, int(math.log2(v)) - 3)
        v = v // step * step
    return min(max(v, lo), hi)


def draw(rng):
    kind = rng.choice(["quantize", "linear", "linear", "moe", "moe"])
    if kind == "quantize":
        T = _log(rng, 1, 16384)
        c = {"T": T, "C": _log(rng, 64, min(16384, max(64, 8192 * 4096 // T))), "x": rng.choice(["f32", "f16", "bf16"])}
    elif kind == "linear":
        T, C = _log(rng, 1, 8192), _log(rng, 64, 8192)
        c = {"T": T, "C": C, "K": _log(rng, 64, max(64, min(16384, 8192 * 4096 * 11008 // (T * C)))),
             "x": rng.choice(["s8", "f32", "f16", "bf16"]), "y": rng.choice(["f32", "f16", "bf16"]),
             "pad": rng.choice([0, 0, 0, 16, 5]), "bias": rng.random() < 0.5}
    else:
        E = _log(rng, 2, 128)
        T, k = _log(rng, 1, 16), rng.randint(1, min(8, E))
        C = _log(rng, 128, 4096)
        most = min(64 * 1024 * 2048 // (E * C), 16 * 8 * 1024 * 2048 // (T * k * C), 2048)
        c = {"T": T, "C": C, "I": _log(rng, 32, max(32, most)), "E": E, "k": k, "x": rng.choice(["f32", "f16", "bf16"]),
             "renorm": rng.random() < 0.5}
    return {"kind": kind, **c}


# ------------------------------------------------------------------------------------------------ inputs
def _activations(g, T, C, dtype):
    """Normal values, one channel in a hundred or so twenty times as large, as trained networks have them."""
    x = torch.randn(T, C, generator=g, device="cuda")
    loud = torch.rand(C, generator=g, device="cuda") < 0.01
    return torch.where(loud, 20 * x, x).to(dtype)


def _weights(g, *shape):
    """Codes of normal weights whose largest, about four deviations out, is at 127, and a factor per output channel that
    makes products of the order of their inputs."""
    w = torch.randn(*shape, generator=g, device="cuda").mul_(32).round_().clamp_(-127, 127).to(torch.int8)
    s = (0.5 + torch.rand(*shape[:-1], generator=g, device="cuda")) / (32 * math.sqrt(shape[-1]))
    return w, s


def _codes(x):
    """Codes and factors by the definition of `q8_quantize_tokens`: maximum over 127, one fp32 division, ties to even."""
    x = x.float()
    m = x.abs().amax(-1, keepdim=True)
    s = torch.where(m == 0, torch.ones_like(m), (m / 127).clamp_min(2.0 ** -126))
    return (x / s).round().clamp(-128, 127), s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = dict(case)
    kind = c["kind"]
    if kind == "quantize":
        return {**c, "in": _activations(g, c["T"], c["C"], TYPES[c["x"]])}
    if kind == "linear":
        T, C, K = c["T"], c["C"], c["K"]
        x = _activations(g, T, C, torch.float32 if c["x"] == "s8" else TYPES[c["x"]])
        scale = None
        if c["x"] == "s8":
            z, s = _codes(x)
            x, scale = z.to(torch.int8), s[:, 0].contiguous()
        if c["pad"]:
            wide = torch.zeros(T, C + c["pad"], dtype=x.dtype, device="cuda")
            wide[:, :C] = x
            x = wide[:, :C]
        w, ws = _weights(g, K, C)
        bias = torch.randn(K, generator=g, device="cuda") if c["bias"] else None
        return {**c, "in": x, "scale": scale, "w": w, "ws": ws, "b": bias}
    T, C, I, E = c["T"], c["C"], c["I"], c["E"]
    x = _activations(g, T, C, TYPES[c["x"]])
    router = torch.randn(E, C, generator=g, device="cuda") / math.sqrt(C)
    wgu, sgu = _weights(g, E, 2 * I, C)
    wd, sd = _weights(g, E, C, I)
    return {**c, "in": x, "router": router, "wgu": wgu, "sgu": sgu, "wd": wd, "sd": sd}


# ------------------------------------------------------------------------------------------------ one pass
def _run_plain(s):
    kind, x = s["kind"], s["in"]
    if kind == "quantize":
        z, f = _codes(x)
        return {"values": (z * f).to(x.dtype), "factors": f[:, 0]}
    if kind == "linear":
        z, f = (x.float(), s["scale"][:, None]) if s["x"] == "s8" else _codes(x)
        y = (z @ s["w"].float().t()) * f * s["ws"]
        if s["b"] is not None:
            y = y + s["b"]
        return y.to(TYPES[s["y"]])
    I, k = s["I"], s["k"]
    logits = x.double() @ s["router"].double().t()            # 64 bits: the choice of experts is a border
    order = logits.sort(dim=-1, descending=True, stable=True)
    ids, top = order.indices[:, :k], order.values[:, :k]
    p = (torch.softmax(top, -1) if s["renorm"] else torch.softmax(logits, -1).gather(-1, ids)).float()
    xf = x.float()[:, None, :, None]
    gu = torch.matmul(s["wgu"][ids].float(), xf)[..., 0] * s["sgu"][ids]
    gate, up = gu[..., :I], gu[..., I:]
    h = gate / (1 + torch.exp(-gate)) * up
    d = torch.matmul(s["wd"][ids].float(), h[..., None])[..., 0] * s["sd"][ids]
    return {"y": (p[..., None] * d).sum(1).to(x.dtype), "experts": ids.to(torch.int32), "weights": p}


def _run_own(s):
    from paper_1805_08691_b200 import binding as q8
    out = {"f32": q8.Q8_F32, "f16": q8.Q8_F16, "bf16": q8.Q8_BF16}
    kind, x = s["kind"], s["in"]
    if kind == "quantize":
        z, f = q8.q8_quantize_tokens(x)
        return {"values": q8.q8_dequantize_tokens(z, f, out[s["x"]]), "factors": f}
    if kind == "linear":
        return q8.q8_linear(x, s["w"], s["ws"], x_scale=s["scale"], bias=s["b"], out_type=out[s["y"]])
    y, ids, p = q8.q8_moe(x, s["router"], s["wgu"], s["sgu"], s["wd"], s["sd"], s["k"], renormalize=s["renorm"])
    return {"y": y, "experts": ids, "weights": p}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    if c["kind"] == "quantize":
        n, e = c["T"] * c["C"], BYTES[c["x"]]
        return {"bytes": n * 2 * e + 4 * c["T"], "flops": 4 * n}
    if c["kind"] == "linear":
        T, C, K = c["T"], c["C"], c["K"]
        return {"bytes": T * C * BYTES[c["x"]] + K * C + 4 * (T + K) + T * K * BYTES[c["y"]], "flops": 2 * T * C * K}
    T, C, I, E, k = (c[n] for n in ("T", "C", "I", "E", "k"))
    reached = E * (1 - (1 - k / E) ** T)                      # experts that some token chooses, on average
    return {"bytes": reached * (3 * I * C + 4 * (2 * I + C)) + 4 * E * C + 2 * T * C * BYTES[c["x"]] + 8 * T * k,
            "flops": 2 * T * (3 * k * I * C + E * C)}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    x = s["in"]
    f64 = torch.float64

    def codes():
        # the factor and the quotient are fp32 divisions by definition, everything after them is exact
        v = x.to(torch.float32)
        m = torch.max(torch.abs(v), dim=1).values
        f = torch.maximum(torch.div(m, 127.0), torch.full_like(m, 2.0 ** -126))
        f[m == 0] = 1.0
        return torch.clamp(torch.round(torch.div(v, f.unsqueeze(1))), -128, 127).to(f64), f.to(f64)

    if s["kind"] == "quantize":
        z, f = codes()
        return {"values": z * f.unsqueeze(1), "factors": f}
    if s["kind"] == "linear":
        z, f = (x.to(f64), s["scale"].to(f64)) if s["x"] == "s8" else codes()
        y = torch.einsum("tc,kc->tk", z, s["w"].to(f64))
        y *= torch.outer(f, s["ws"].to(f64))
        return y if s["b"] is None else y.add_(s["b"].to(f64))
    I, E, k = s["I"], s["E"], s["k"]
    v = x.to(f64)
    logits = torch.einsum("tc,ec->te", v, s["router"].to(f64))
    y = torch.zeros_like(v)
    ids = torch.zeros(s["T"], k, dtype=torch.int32, device="cuda")
    p = torch.zeros(s["T"], k, dtype=f64, device="cuda")
    for t, row in enumerate(logits.tolist()):
        chosen = sorted(range(E), key=lambda e: (-row[e], e))[:k]
        top = max(row)
        total = sum(math.exp(row[e] - top) for e in (chosen if s["renorm"] else range(E)))
        for j, e in enumerate(chosen):
            weight = math.exp(row[e] - top) / total
            gu = (s["wgu"][e].to(f64) @ v[t]) * s["sgu"][e].to(f64)
            h = gu[:I] * torch.sigmoid(gu[:I]) * gu[I:]
            y[t] += weight * ((s["wd"][e].to(f64) @ h) * s["sd"][e].to(f64))
            ids[t, j], p[t, j] = e, weight
    return {"y": y, "experts": ids, "weights": p}
