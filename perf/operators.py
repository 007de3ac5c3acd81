"""Operators for decoding: the MoE layer for a few tokens, and experts with 4-bit weights.

Four operators and what each computes:

``layer``    the whole MoE layer (router, top-K, SwiGLU experts, weighted sum) for 1 to 16 tokens, weights in bf16 or fp32
``layer_w4`` the same with the experts' weights in 4 bits
``matvec``   products of a few rows with a matrix of 4-bit weights, or with one matrix of several per row
``pack``     weights into the 4-bit form and back (what makes the form that the others read, and what a prefill on it starts from)

The 4-bit form of a matrix [N, C] with groups of g columns: codes, uint8 [N, C / 2], and scales, bf16 [C / g, N];
W[n, c] = scales[c / g, n] * (code - 8).  Eight columns are one little-endian 32-bit word, whose nibbles hold, from the least
significant one on, the columns 0, 2, 4, 6, 1, 3, 5, 7 of the eight.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

# H, E, K, F, renormalised weights: the layers that the package's workloads name
SHAPES = {
    "mixtral": dict(H=4096, E=8, K=2, F=14336, renorm=1),
    "phi35": dict(H=4096, E=16, K=2, F=6400, renorm=1),
    "qwen": dict(H=2048, E=60, K=4, F=1408, renorm=0),
    "deepseek": dict(H=7168, E=256, K=8, F=2048, renorm=1),
}
TOKENS = 16   # most tokens of a layer call
LARGEST = 9e9  # bytes that a drawn layer reads at most


def _layer(dtype, T, H, E, K, F, renorm=0, bias=0):
    return dict(op="layer", dtype=dtype, T=T, H=H, E=E, K=K, F=F, renorm=renorm, bias=bias)


def _layer_w4(g, T, H, E, K, F, renorm=0, bias=0):
    return dict(op="layer_w4", g=g, T=T, H=H, E=E, K=K, F=F, renorm=renorm, bias=bias)


def _matvec(g, M, N, C, E=1):
    return dict(op="matvec", g=g, M=M, N=N, C=C, E=E)


def _pack(dtype, g, E, N, C):
    return dict(op="pack", dtype=dtype, g=g, E=E, N=N, C=C)


def listed():
    S = SHAPES
    cases = {
        # decoding one sequence, four small experts: launches and latencies count as much as the bytes
        "layer_qwen_1": _layer("bf16", 1, **S["qwen"]),
        # a small batch over a few large experts: nearly every expert is read
        "layer_mixtral_5": _layer("bf16", 5, **S["mixtral"]),
        # a batch over many experts, with a bias on the router: the most bytes
        "layer_deepseek_16": _layer("bf16", 16, bias=1, **S["deepseek"]),
        # a small model kept in fp32, odd sizes
        "layer_fp32_3": _layer("fp32", 3, H=1020, E=16, K=2, F=2044),
        # the same layers with 4-bit experts
        "layer_w4_qwen_1": _layer_w4(64, 1, **S["qwen"]),
        "layer_w4_mixtral_7": _layer_w4(128, 7, **S["mixtral"]),
        "layer_w4_deepseek_16": _layer_w4(128, 16, **S["deepseek"]),
        # one projection of one token: the smallest call
        "matvec_1": _matvec(128, 1, 1408, 2048),
        # a projection of a small batch of tokens
        "matvec_8": _matvec(128, 8, 7168, 7168),
        # rows of a routed batch, each with its expert's matrix, more rows than one pass takes, small groups
        "matvec_experts_24": _matvec(32, 24, 2817, 2048, E=60),
        # a layer's gate matrices loaded in bf16, and small fp32 ones with a ragged number of rows
        "pack_bf16": _pack("bf16", 128, 8, 14336, 4096),
        "pack_fp32": _pack("fp32", 32, 3, 1001, 2048),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["layer", "layer", "layer_w4", "layer_w4", "matvec", "matvec", "pack"])
        g = rng.choice([32, 64, 128])
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        T = rng.randint(1, TOKENS)
        if op in ("layer", "layer_w4"):
            unit = g if op == "layer_w4" else 8 if dtype == "bf16" else 4
            c = dict(rng.choice([S for S in SHAPES.values()])) if rng.random() < 0.5 else dict(
                H=unit * _log_int(rng, -(-256 // unit), 8192 // unit), E=_log_int(rng, 4, 256), K=rng.randint(1, 4),
                F=unit * _log_int(rng, -(-128 // unit), 8192 // unit), renorm=rng.randint(0, 1))
            c["bias"] = rng.randint(0, 1)
            if 3.0 * c["E"] * c["H"] * c["F"] > (12e9 if op == "layer_w4" or dtype == "bf16" else 3e9):
                continue  # (the weights have to fit the card several times over)
            c = _layer_w4(g, T, **c) if op == "layer_w4" else _layer(dtype, T, **c)
            if work(c)["bytes"] > LARGEST:
                continue
        elif op == "matvec":
            E = rng.choice([1, 1, _log_int(rng, 2, 64)])
            c = _matvec(g, _log_int(rng, 1, 48), _log_int(rng, 1, 16384), g * _log_int(rng, 1, 14336 // g), E)
            if max(E, c["M"] if E > 1 else 1) * c["N"] * c["C"] > 4e9:  # (the plain form holds a matrix per row)
                continue
        else:
            c = _pack(dtype, g, _log_int(rng, 1, 16), _log_int(rng, 16, 8192), g * _log_int(rng, 2, 8192 // g))
            if c["E"] * c["N"] * c["C"] > 4.7e8:
                continue
        return c


def _type(c):
    return torch.float32 if c.get("dtype") == "fp32" else torch.bfloat16


def _normal(g, std, dtype, *shape):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def _w4(g, std, E, N, C, group):
    """Codes and scales as the quantisation of normal weights gives them: the largest of a group's codes is 1 or 15."""
    spread = {32: 3.4, 64: 3.0, 128: 2.7}[group]  # 7 over the largest of as many normal numbers
    codes = torch.empty(E, N, C // 2, dtype=torch.uint8, device="cuda")
    step = max(1, int(2e8 // (N * C)))
    for e in range(0, E, step):
        at = codes[e: e + step]
        low, high = (torch.empty(at.shape, dtype=torch.float16, device="cuda").normal_(0.0, spread, generator=g).round_().clamp_(-7, 7).add_(8).to(torch.uint8)
                     for _ in range(2))
        torch.add(low, high.mul_(16), out=at)
    scales = torch.empty(E, C // group, N, dtype=torch.bfloat16, device="cuda").normal_(1.0, 0.15, generator=g).mul_(std / spread)
    return codes, scales


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if c["op"] in ("layer", "layer_w4"):
        T, H, E, F, dt = c["T"], c["H"], c["E"], c["F"], _type(c)
        s["x"] = _normal(g, 1.0, dt, T, H)
        s["wr"] = _normal(g, 0.02, dt, E, H)
        s["bias"] = _normal(g, 0.5, torch.float32, E) if c["bias"] else None
        s["y"] = torch.empty(T, H, dtype=dt, device="cuda")
        if c["op"] == "layer":
            s["wg"], s["wu"], s["wd"] = _normal(g, 0.02, dt, E, F, H), _normal(g, 0.02, dt, E, F, H), _normal(g, 0.02, dt, E, H, F)
        else:
            s["wg"], s["wu"], s["wd"] = _w4(g, 0.02, E, F, H, c["g"]), _w4(g, 0.02, E, F, H, c["g"]), _w4(g, 0.02, E, H, F, c["g"])
    elif c["op"] == "matvec":
        s["w"] = _w4(g, 0.02, c["E"], c["N"], c["C"], c["g"])
        s["x"] = _normal(g, 1.0, torch.bfloat16, c["M"], c["C"])
        s["expert"] = torch.randint(c["E"], (c["M"],), generator=g, device="cuda", dtype=torch.int32) if c["E"] > 1 else None
        s["y"] = torch.empty(c["M"], c["N"], dtype=torch.bfloat16, device="cuda")
    else:
        shape = c["E"], c["N"], c["C"]
        s["w"] = _normal(g, 0.02, _type(c), *shape)
        s["codes"] = torch.empty(c["E"], c["N"], c["C"] // 2, dtype=torch.uint8, device="cuda")
        s["scales"] = torch.empty(c["E"], c["C"] // c["g"], c["N"], dtype=torch.bfloat16, device="cuda")
        s["values"] = torch.empty(shape, dtype=_type(c), device="cuda")
    if own:
        from paper_2605_05888_b200 import binding as B
        if c["op"] in ("layer", "layer_w4"):
            s["plan"] = B.Plan(B.make_config(T, H, E, 1, c["K"], F, B.DTYPE_FP32 if dt == torch.float32 else B.DTYPE_BF16, renormalize=c["renorm"]))
            if c["op"] == "layer_w4":
                for name in ("wg", "wu", "wd"):
                    s[name] = B.W4(*s[name])
        elif c["op"] == "matvec":
            s["w"] = B.W4(*s["w"])
        else:
            s["out"] = B.W4(s["codes"], s["scales"])
    return s


# ---- the plain forms: elementary torch operations in 32 bits, rounded once at the end ----------------------------------------

COLUMN_OF_NIBBLE = [0, 2, 4, 6, 1, 3, 5, 7]
NIBBLE_OF_COLUMN = [0, 4, 1, 5, 2, 6, 3, 7]


def _unpack(codes, scales):
    """[..., N, C/2] codes and [..., C/g, N] scales as fp32 weights [..., N, C]."""
    q = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).unflatten(-1, (-1, 8))[..., NIBBLE_OF_COLUMN].flatten(-2)
    w = q.to(torch.float32) - 8.0
    w.unflatten(-1, (scales.shape[-2], -1)).mul_(scales.to(torch.float32).transpose(-1, -2).unsqueeze(-1))
    return w


def _picked(w, idx):
    """The weights of the picked experts as fp32 [T, K, rows, columns]."""
    return _unpack(w[0][idx], w[1][idx]) if isinstance(w, tuple) else w[idx].to(torch.float32)


def _route(s):
    c = s["case"]
    logits = s["x"].to(torch.float64) @ s["wr"].to(torch.float64).T  # in 64 bits: the picks hang on near ties
    if s["bias"] is not None:
        logits = logits + s["bias"]
    order = torch.sort(logits, dim=1, descending=True, stable=True)
    p = torch.softmax(logits, 1).gather(1, order.indices)[:, : c["K"]]
    return order.indices[:, : c["K"]], (p / p.sum(1, keepdim=True) if c["renorm"] else p).to(torch.float32)


def _plain_layer(s):
    idx, w = _route(s)
    x = s["x"].to(torch.float32)[:, None, :, None]
    gate = torch.matmul(_picked(s["wg"], idx), x)
    inter = gate * torch.sigmoid(gate) * torch.matmul(_picked(s["wu"], idx), x)
    out = torch.matmul(_picked(s["wd"], idx), inter)[..., 0]
    return (out * w[..., None]).sum(1).to(s["x"].dtype)


def _plain_matvec(s):
    codes, scales = s["w"]
    x = s["x"].to(torch.float32)
    if s["expert"] is None:
        return (x @ _unpack(codes[0], scales[0]).T).to(torch.bfloat16)
    e = s["expert"].long()
    return torch.matmul(_unpack(codes[e], scales[e]), x[..., None])[..., 0].to(torch.bfloat16)


def _plain_pack(s):
    g = s["case"]["g"]
    w = s["w"].unflatten(-1, (-1, g))
    scales = (w.abs().amax(-1).to(torch.float64) / 7.0).to(torch.float32).to(torch.bfloat16)  # [E, N, C/g], the fp32 quotient
    some = torch.where(scales > 0, scales, 1.0).unsqueeze(-1)
    q = torch.where(scales.unsqueeze(-1) > 0, torch.round(w.to(torch.float64) / some.to(torch.float64)), 0.0).clamp(-8, 7).to(torch.float32)
    values = (q * scales.unsqueeze(-1).to(torch.float32)).flatten(-2).to(s["w"].dtype)
    return {"scales": scales.transpose(-1, -2).contiguous(), "values": values}


def run(s):
    op = s["case"]["op"]
    if not own:
        return _plain_pack(s) if op == "pack" else _plain_matvec(s) if op == "matvec" else _plain_layer(s)
    from paper_2605_05888_b200 import binding as B
    if op == "layer":
        s["plan"].moe_layer_few(s["x"], s["wr"], s["bias"], s["wg"], s["wu"], s["wd"], s["y"])
    elif op == "layer_w4":
        s["plan"].moe_layer_few_w4(s["x"], s["wr"], s["bias"], s["wg"], s["wu"], s["wd"], s["y"])
    elif op == "matvec":
        B.moe_w4_matvec(s["w"], s["x"], s["expert"], s["y"])
    else:
        B.moe_w4_pack(s["w"], s["out"])
        B.moe_w4_unpack(s["out"], s["values"])  # the codes as the values they stand for
        return {"scales": s["scales"], "values": s["values"]}
    return s["y"]


# ---- what a pass cannot do without -------------------------------------------------------------------------------------------

def _experts_used(c):
    """Experts that at least one token picks: simulated, as the logits are normal."""
    rng = np.random.default_rng(1)
    used = 0
    for _ in range(16):
        logits = rng.standard_normal((c["T"], c["E"])) * (0.02 * math.sqrt(c["H"]))
        if c["bias"]:
            logits = logits + 0.5 * rng.standard_normal(c["E"])
        used += len(np.unique(np.argpartition(-logits, c["K"] - 1, axis=1)[:, : c["K"]]))
    return used / 16


def work(case):
    c = case
    b = 4 if c.get("dtype") == "fp32" else 2
    packed = 0.5 + 2.0 / c.get("g", 1)
    if c["op"] == "pack":
        n = c["E"] * c["N"] * c["C"]
        return {"bytes": float(n * (2 * b + packed)), "flops": float(3 * n)}
    if c["op"] == "matvec":
        used = c["E"] * (1 - (1 - 1 / c["E"]) ** c["M"])  # distinct ids among M
        return {"bytes": float(used * c["N"] * c["C"] * packed + 2 * c["M"] * (c["N"] + c["C"])), "flops": float(2 * c["M"] * c["N"] * c["C"])}
    T, H, E, K, F = c["T"], c["H"], c["E"], c["K"], c["F"]
    weight = packed if c["op"] == "layer_w4" else b
    return {"bytes": float(3 * _experts_used(c) * F * H * weight + E * H * b + 2 * T * H * b), "flops": float(2 * T * H * E + 6 * T * K * H * F)}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------------

def _exact_matrix(w, e):
    """Expert e's matrix in 64 bits."""
    if not isinstance(w, tuple):
        return w[e].double()
    codes, scales = w[0][e], w[1][e].double()
    N, C = codes.shape[0], 2 * codes.shape[1]
    out = torch.empty(N, C, dtype=torch.float64, device=codes.device)
    for nibble, column in enumerate(COLUMN_OF_NIBBLE):
        out[:, column::8] = torch.bitwise_right_shift(codes[:, nibble // 2:: 4], 4 * (nibble % 2)).bitwise_and(15).double() - 8.0
    return out * scales.T.repeat_interleave(C // scales.shape[0], dim=1)


def _exact_layer(s):
    c = s["case"]
    x = s["x"].double()
    logits = torch.einsum("th,eh->te", x, s["wr"].double())
    if s["bias"] is not None:
        logits += s["bias"].double()
    logits = logits.cpu().numpy()
    y = torch.zeros_like(x)
    picks = np.argsort(-logits, axis=1, kind="stable")[:, : c["K"]]
    p = np.exp(logits - logits.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    w = np.take_along_axis(p, picks, 1)
    if c["renorm"]:
        w /= w.sum(1, keepdims=True)
    for e in np.unique(picks):
        t, k = (torch.from_numpy(i).to(x.device) for i in np.nonzero(picks == e))
        weight = torch.from_numpy(w).to(x.device)[t, k]
        a = x[t]
        gate, up = a @ _exact_matrix(s["wg"], e).T, a @ _exact_matrix(s["wu"], e).T
        o = (gate / (1.0 + torch.exp(-gate)) * up) @ _exact_matrix(s["wd"], e).T
        y[t] += weight[:, None] * o
    return y


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("layer", "layer_w4"):
        return _exact_layer(s)
    if case["op"] == "matvec":
        x = s["x"].double()
        e = np.zeros(case["M"], dtype=np.int64) if s["expert"] is None else s["expert"].cpu().numpy()
        y = torch.empty(case["M"], case["N"], dtype=torch.float64, device=x.device)
        for i in np.unique(e):
            rows = torch.from_numpy(np.nonzero(e == i)[0]).to(x.device)
            y[rows] = x[rows] @ _exact_matrix(s["w"], i).T
        return y
    E, N, C, g = case["E"], case["N"], case["C"], case["g"]
    scales = torch.empty(E, C // g, N, dtype=torch.float64, device="cuda")
    values = torch.empty(E, N, C, dtype=torch.float64, device="cuda")
    for e in range(E):
        w = s["w"][e].double().view(N, C // g, g)
        largest = torch.maximum(w.max(-1).values, -w.min(-1).values)
        scale = (largest / 7.0).float().bfloat16().double()  # by definition a bf16 number: the quotient rounded to fp32, then to bf16
        q = torch.round(w / torch.where(scale > 0, scale, torch.ones_like(scale))[..., None]).clamp(-8, 7) * (scale > 0)[..., None]
        scales[e], values[e] = scale.T, (q * scale[..., None]).view(N, C)
    return {"scales": scales, "values": values}
