"""The microscaled operators, as cases that can be timed and compared: conversion of tensors to 4- or 8-bit elements with one power-of-two scale
for 32 values and back, the inner product on such tensors with its result in floating point or converted again, and the root-mean-square norm with the
residual's addition whose result is converted on the way out.

Elements: 4 is E2M1 (two to a byte, the even one in the low half), 8 is E4M3.  A scale byte s stands for 2^(s-127)."""
import math

import torch

own = False
DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
WIDTH = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # a layer's float weights are converted once and looked at as what they now stand for
        dict(name="weights_4bit_8192", kind="roundtrip", rows=8192, K=8192, dtype="f32", elem=4, rule="cover", out="bf16"),
        # activations of a long prompt in front of a product
        dict(name="activations_8bit_4096x8192", kind="quantize", rows=4096, K=8192, dtype="bf16", elem=8, rule="floor"),
        # one token, where a call's latency is all there is
        dict(name="one_token_8bit_4096", kind="roundtrip", rows=1, K=4096, dtype="bf16", elem=8, rule="cover", out="f32"),
        # one token through a wide layer of 4-bit weights: the weights' bytes
        dict(name="linear_1x8192x8192", kind="linear", M=1, N=8192, K=8192, ex=8, ew=4, bias=False, relu=False, out="bf16"),
        # sixteen answers at once, a long reduction
        dict(name="linear_16x4096x16384", kind="linear", M=16, N=4096, K=16384, ex=4, ew=4, bias=False, relu=False, out="bf16"),
        # the classifier behind the benchmark's network at its batch
        dict(name="linear_256x1000x2048", kind="linear", M=256, N=1000, K=2048, ex=8, ew=8, bias=True, relu=False, out="f32"),
        # bulk work on 4-bit operands: the largest
        dict(name="linear_8192", kind="linear", M=8192, N=8192, K=8192, ex=4, ew=4, bias=False, relu=False, out="bf16"),
        # sizes that are multiples of nothing, a bias and a ReLU
        dict(name="linear_777x1357x2999", kind="linear", M=777, N=1357, K=2999, ex=8, ew=4, bias=True, relu=True, out="f16"),
        # the first product of a feed-forward block, its result converted for the second
        dict(name="linear_q_4096x8192x4096", kind="linear_q", M=4096, N=8192, K=4096, ex=8, ew=8, bias=False, relu=True, elem=8, rule="cover"),
        # the norm in front of a product, for one token and for a long prompt
        dict(name="norm_1x4096", kind="norm", rows=1, K=4096, dtype="bf16", add=True, rule="cover"),
        dict(name="norm_8192x8192", kind="norm", rows=8192, K=8192, dtype="bf16", add=True, rule="floor"),
        # a feed-forward block as it is used: norm, product with ReLU, product
        dict(name="block_512x4096x10240", kind="block", M=512, d=4096, hidden=10240, ex=8, eh=4, ew=4, dtype="bf16", rule="cover"),
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _length(rng, lo, hi):
    """A length: one of whole blocks as often as any other."""
    n = _spread(rng, lo, hi)
    return n if rng.random() < 0.5 else max(32, n // 32 * 32)


def draw(rng):
    kind = rng.choices(["roundtrip", "quantize", "linear", "linear_q", "norm", "block"], [14, 14, 32, 12, 18, 10])[0]
    rule = rng.choice(["cover", "floor"])
    if kind in ("roundtrip", "quantize", "norm"):
        K = _length(rng, 20, 16384)
        rows = _spread(rng, 1, max(1, min(16384, (1 << 26) // K)))
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        if kind == "norm":
            return dict(kind=kind, rows=rows, K=K, dtype=dtype, add=rng.random() < 0.7, rule=rule)
        if kind == "quantize":
            return dict(kind=kind, rows=rows, K=K, dtype=dtype, elem=8, rule=rule)
        return dict(kind=kind, rows=rows, K=K, dtype=dtype, elem=rng.choice([4, 8]), rule=rule, out=rng.choice(["f32", "bf16", "f16"]))
    if kind == "block":
        d, hidden, eh = _length(rng, 256, 8192), _length(rng, 256, 16384), rng.choice([4, 8])
        return dict(kind=kind, M=_spread(rng, 1, 2048), d=d, hidden=hidden, ex=8, eh=eh, ew=rng.choice([4, 4, 8]), dtype=rng.choice(["bf16", "f16"]), rule=rule)
    N, K = _length(rng, 24, 16384), _length(rng, 40, 16384)
    M = _spread(rng, 1, max(1, min(16384, (1 << 38) // (N * K))))
    ex, ew = rng.choice([(4, 4), (8, 4), (8, 8), (4, 8)])
    if kind == "linear_q":
        return dict(kind=kind, M=M, N=N, K=K, ex=ex, ew=ew, bias=rng.random() < 0.5, relu=rng.random() < 0.5, elem=8, rule=rule)
    return dict(kind=kind, M=M, N=N, K=K, ex=ex, ew=ew, bias=rng.random() < 0.5, relu=rng.random() < 0.3, out=rng.choice(["bf16", "bf16", "f16", "f32"]))


# ---- the plain form: elementary operations in 32 bits ---------------------------------------- #
def _blocks(v):
    """float32 [rows, K] -> [rows, blocks, 32], the last block filled up with zeros."""
    rows, K = v.shape
    return torch.nn.functional.pad(v, (0, -K % 32)).view(rows, -1, 32)


def _convert(v, elem, rule):
    """float32 [rows, K] -> (element values [rows, blocks, 32], exponents of the scales [rows, blocks])."""
    v = _blocks(v)
    amax = v.abs().amax(2)
    m, ex = torch.frexp(amax)                                     # amax = m * 2^ex, m in [1/2, 1)
    e = ex - (3 if elem == 4 else 9)                              # floor(log2 amax) - 2, - 8: the exponent of the largest element
    if rule == "cover":
        e = e + (m > (0.75 if elem == 4 else 0.875)).int()        # 6 = 0.75 * 2^3, 448 = 0.875 * 2^9
    e = torch.where(amax > 0, e, torch.full_like(e, -127)).clamp(min=-127)
    t = torch.ldexp(v, -e[:, :, None])                            # exact
    mag = t.abs().clamp(max=6.0 if elem == 4 else 448.0)
    _, k = torch.frexp(mag)
    step = torch.ldexp(torch.ones_like(mag), (k - 1).clamp(min=0 if elem == 4 else -6) - (1 if elem == 4 else 3))
    q = torch.round(mag / step) * step                            # ties to even
    return torch.where(t < 0, -q, q) + 0.0, e


def _pack(q, e, elem):
    """What the framework's tensors hold: code bytes, and scale bytes in rows of a multiple of four."""
    rows, nb, _ = q.shape
    scales = torch.zeros(rows, -(-nb // 4) * 4, dtype=torch.uint8, device=q.device)
    scales[:, :nb] = (e + 127).to(torch.uint8)
    if elem == 8:
        return q.to(torch.float8_e4m3fn).view(torch.uint8).view(rows, -1), scales
    index = torch.tensor([0, 1, 2, 3, 4, 0, 5, 0, 6, 0, 0, 0, 7], dtype=torch.uint8, device=q.device)     # twice the magnitude -> code
    c = index[(q.abs() * 2).int()] | (q < 0).to(torch.uint8) << 3
    c = c.view(rows, -1, 2)
    return (c[:, :, 0] | c[:, :, 1] << 4).contiguous(), scales


def _values(codes, scales, elem, K):
    """Code and scale bytes -> float32 [rows, K]."""
    rows = codes.shape[0]
    if elem == 8:
        v = codes.view(torch.float8_e4m3fn).float()
    else:
        table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
        v = table[torch.stack((codes & 15, codes >> 4), 2).int()].view(rows, -1)
    nb = v.shape[1] // 32
    e = scales[:, :nb].int() - 127
    return torch.ldexp(v.view(rows, nb, 32), e[:, :, None]).view(rows, -1)[:, :K]


def _linear(x, w, bias, relu):
    y = x @ w.t()
    if bias is not None:
        y = y + bias
    return y.clamp(min=0) if relu else y


def _norm(x, add, weight, eps):
    s = x.float() if add is None else x.float() + add.float()
    return s, s * torch.rsqrt(s.square().mean(1, keepdim=True) + eps) * weight.float()


def _seen(q, e):
    """A converted 8-bit tensor as what its elements and scales stand for."""
    return q.view(q.shape[0], -1).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


# ---- what a user has in hand ------------------------------------------------------------------ #
def _activations(g, rows, K, dtype):
    """Normal values with a few channels that stand out, as hidden states have them."""
    v = torch.randn(rows, K, generator=g, device=DEV)
    v *= torch.where(torch.rand(K, generator=g, device=DEV) < 0.005, 20.0, 1.0)
    return v.to(DTYPES[dtype])


def _weights(g, N, K, elem):
    return _pack(*_convert(torch.randn(N, K, generator=g, device=DEV) * K ** -0.5, elem, "cover"), elem)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed * 1009 + 17)
    kind, s = case["kind"], dict(case)
    if kind in ("roundtrip", "quantize", "norm"):
        s["x"] = _activations(g, case["rows"], case["K"], case["dtype"])
        if kind == "norm":
            s["add"] = _activations(g, case["rows"], case["K"], case["dtype"]) if case["add"] else None
            s["weight"] = (1 + 0.2 * torch.randn(case["K"], generator=g, device=DEV)).to(DTYPES[case["dtype"]])
    elif kind == "block":
        s["x"], s["add"] = (_activations(g, case["M"], case["d"], case["dtype"]) for _ in range(2))
        s["weight"] = (1 + 0.2 * torch.randn(case["d"], generator=g, device=DEV)).to(DTYPES[case["dtype"]])
        s["w1"], s["w2"] = _weights(g, case["hidden"], case["d"], case["ew"]), _weights(g, case["d"], case["hidden"], case["ew"])
    else:
        s["x"] = _pack(*_convert(_activations(g, case["M"], case["K"], "f32"), case["ex"], "cover"), case["ex"])
        s["w"] = _weights(g, case["N"], case["K"], case["ew"])
        s["b"] = 0.1 * torch.randn(case["N"], generator=g, device=DEV) if case["bias"] else None
    return s


EPS = 1e-5


def run(s):
    return _own(s) if own else _plain(s)


def _plain(s):
    kind = s["kind"]
    if kind == "quantize":
        return _seen(*_convert(s["x"].float(), s["elem"], s["rule"]))
    if kind == "roundtrip":
        q, e = _convert(s["x"].float(), s["elem"], s["rule"])
        return torch.ldexp(q, e[:, :, None]).view(s["rows"], -1)[:, :s["K"]].to(DTYPES[s["out"]])
    if kind == "norm":
        total, v = _norm(s["x"], s["add"], s["weight"], EPS)
        return *_seen(*_convert(v, 8, s["rule"])), total.to(DTYPES[s["dtype"]]) if s["add"] is not None else None
    if kind == "block":
        total, v = _norm(s["x"], s["add"], s["weight"], EPS)
        q, e = _convert(v, s["ex"], s["rule"])
        h = _linear(torch.ldexp(q, e[:, :, None]).view(s["M"], -1)[:, :s["d"]], _values(*s["w1"], s["ew"], s["d"]), None, True)
        q, e = _convert(h, s["eh"], s["rule"])
        y = _linear(torch.ldexp(q, e[:, :, None]).view(s["M"], -1)[:, :s["hidden"]], _values(*s["w2"], s["ew"], s["hidden"]), None, False)
        return total.to(DTYPES[s["dtype"]]), y.to(DTYPES[s["dtype"]])
    y = _linear(_values(*s["x"], s["ex"], s["K"]), _values(*s["w"], s["ew"], s["K"]), s["b"], s["relu"])
    return _seen(*_convert(y, s["elem"], s["rule"])) if kind == "linear_q" else y.to(DTYPES[s["out"]])


def _own(s):
    from paper_1805_07941_amd import binding as B
    kind, elem, rule = s["kind"], {4: B.MX4, 8: B.MX8}, {"cover": B.MX_COVER, "floor": B.MX_FLOOR}

    def seen(q):
        return q.codes.view(torch.float8_e4m3fn), q.scales[:, :-(-q.k // 32)].view(torch.float8_e8m0fnu)

    if kind == "quantize":
        return seen(B.quantize_mx(s["x"], elem[s["elem"]], rule[s["rule"]]))
    if kind == "roundtrip":
        return B.dequantize_mx(B.quantize_mx(s["x"], elem[s["elem"]], rule[s["rule"]]), DTYPES[s["out"]])
    if kind == "norm":
        q, _, total = B.rms_norm_mx(s["x"], s["weight"], EPS, add=s["add"], elem=B.MX8, rule=rule[s["rule"]])
        return *seen(q), total
    if kind == "block":
        q, _, total = B.rms_norm_mx(s["x"], s["weight"], EPS, add=s["add"], elem=elem[s["ex"]], rule=rule[s["rule"]])
        h = B.linear_mx_q(q, B.MxTensor(*s["w1"], elem[s["ew"]], s["d"]), elem=elem[s["eh"]], rule=rule[s["rule"]], relu=True)
        return total, B.linear_mx(h, B.MxTensor(*s["w2"], elem[s["ew"]], s["hidden"]), dtype=DTYPES[s["dtype"]])
    x, w = B.MxTensor(*s["x"], elem[s["ex"]], s["K"]), B.MxTensor(*s["w"], elem[s["ew"]], s["K"])
    if kind == "linear_q":
        return seen(B.linear_mx_q(x, w, s["b"], elem=elem[s["elem"]], rule=rule[s["rule"]], relu=s["relu"]))
    return B.linear_mx(x, w, s["b"], relu=s["relu"], dtype=DTYPES[s["out"]])


# ---- what a pass cannot do without ------------------------------------------------------------ #
def _held(rows, K, elem):
    """Bytes of a converted tensor: its codes and its scales."""
    return rows * (K * elem / 8 + -(-K // 32))


def work(case):
    c, kind = case, case["kind"]
    if kind in ("quantize", "roundtrip"):
        n, held = c["rows"] * c["K"], _held(c["rows"], c["K"], c["elem"])
        return {"bytes": n * WIDTH[c["dtype"]] + (held if kind == "quantize" else 2 * held + n * WIDTH[c["out"]]), "flops": 3 * n}
    if kind == "norm":
        n = c["rows"] * c["K"]
        return {"bytes": n * WIDTH[c["dtype"]] * (3 if c["add"] else 1) + _held(c["rows"], c["K"], 8) + c["K"] * WIDTH[c["dtype"]], "flops": 8 * n}
    if kind == "block":
        n, width = c["M"] * c["d"], WIDTH[c["dtype"]]
        held = 2 * _held(c["M"], c["d"], c["ex"]) + 2 * _held(c["M"], c["hidden"], c["eh"]) + _held(c["hidden"], c["d"], c["ew"]) + _held(c["d"], c["hidden"], c["ew"])
        return {"bytes": 4 * n * width + held, "flops": 4 * n * c["hidden"] + 8 * n}
    out = _held(c["M"], c["N"], 8) if kind == "linear_q" else c["M"] * c["N"] * WIDTH[c["out"]]
    return {"bytes": _held(c["M"], c["K"], c["ex"]) + _held(c["N"], c["K"], c["ew"]) + out + 4 * c["N"] * c["bias"], "flops": 2 * c["M"] * c["N"] * c["K"]}


# ---- the definition in 64 bits ---------------------------------------------------------------- #
def _magnitudes(elem):
    """The non-negative elements in the order of their codes."""
    bits, low, codes = (1, 0, 8) if elem == 4 else (3, -6, 127)
    fields = [(c >> bits, c & (1 << bits) - 1) for c in range(codes)]
    return [math.ldexp(m, low - bits) if f == 0 else math.ldexp((1 << bits) + m, low - bits + f - 1) for f, m in fields]


def _nearest(v, elem, rule):
    """float64 [rows, K] -> (elements [rows, 32 * blocks], scales [rows, blocks]) as numbers."""
    rows, K = v.shape
    table = torch.tensor(_magnitudes(elem), dtype=torch.float64, device=v.device)
    full = torch.zeros(rows, -(-K // 32) * 32, dtype=torch.float64, device=v.device)
    full[:, :K] = v
    full = full.view(rows, -1, 32)
    amax = full.abs().amax(2)
    powers = torch.exp2(torch.arange(-127, 128, dtype=torch.float64, device=v.device))
    if rule == "cover":
        at = torch.searchsorted(powers * table[-1], amax)                                        # the first that covers amax
    else:
        at = torch.searchsorted(powers * 2.0 ** (2 if elem == 4 else 8), amax, right=True) - 1   # the last that is not above it
    scale = powers[at.clamp(0, 254)]
    mag = (full.abs() / scale[:, :, None]).contiguous()
    between = (table[1:] + table[:-1]) / 2
    below = torch.searchsorted(between, mag)
    code = torch.where(below % 2 == 0, below, torch.searchsorted(between, mag, right=True))     # a tie goes to the even code
    q = table[code]
    return (torch.where(full < 0, -q, q) + 0.0).view(rows, -1), scale


def _times(q, scale, K):
    return (q.view(*scale.shape, 32) * scale[:, :, None]).view(q.shape)[:, :K]


def _stands_for(held, elem, K):
    codes, scales = held
    table = _magnitudes(elem)
    table = torch.tensor(table + [-v for v in table] if elem == 4 else table + [math.nan] + [-v for v in table] + [math.nan], dtype=torch.float64, device=codes.device)
    at = codes.long()
    if elem == 4:
        at = torch.stack((at % 16, at // 16), 2).view(codes.shape[0], -1)
    v = table[at]
    return _times(v, torch.exp2(scales[:, :v.shape[1] // 32].double() - 127), K)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("quantize", "roundtrip"):
        q, scale = _nearest(s["x"].double(), case["elem"], case["rule"])
        return (q, scale) if kind == "quantize" else _times(q, scale, case["K"])
    if kind in ("norm", "block"):
        total = s["x"].double() + (s["add"].double() if s["add"] is not None else 0)
        v = total / torch.sqrt((total * total).sum(1, keepdim=True) / total.shape[1] + EPS) * s["weight"].double()
        if kind == "norm":
            return *_nearest(v, 8, case["rule"]), total if s["add"] is not None else None
        x = _times(*_nearest(v, case["ex"], case["rule"]), case["d"])
        h = torch.matmul(x, _stands_for(s["w1"], case["ew"], case["d"]).t()).clamp(min=0)
        h = _times(*_nearest(h, case["eh"], case["rule"]), case["hidden"])
        return total, torch.matmul(h, _stands_for(s["w2"], case["ew"], case["hidden"]).t())
    y = torch.matmul(_stands_for(s["x"], case["ex"], case["K"]), _stands_for(s["w"], case["ew"], case["K"]).t())
    if s["b"] is not None:
        y = y + s["b"].double()
    if case["relu"]:
        y = torch.relu(y)
    return _nearest(y, case["elem"], case["rule"]) if kind == "linear_q" else y
