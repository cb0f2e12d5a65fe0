"""Microscaled weights and activations, as cases that can be timed.

A matrix of rows of K values is held as codes of 8 bits (e4m3) or 4 bits (e2m1,
two a byte, the lower nibble first) with one power of two for each 32 codes of a
row (an e8m0 byte, its exponent plus 127).  Every case is one pass through an
operator on device-resident data:

  gemm      wq4_mx_gemm: activations of 8 or 4 bits through a projection whose
            weights have 4 bits, from one token to a long prompt
  norm      wq4_mx_norm: the residual's addition, the root-mean-square norm with
            its gain, and the normalised rows in 8 or 4 bits with scales
  silu      wq4_mx_silu: silu(gate) * up of fused gate_up rows, in 8 or 4 bits
  quantize  wq4_mx_quantize: rows of fp16 in 8 or 4 bits

What is held in 8 bits comes back as its codes and its scales; what is held in 4
bits as fp16 values, by wq4_mx_dequantize.  Scales lie in blocks of 128 rows by
four groups: row r, group g at byte ((r / 128) * (K / 128) + g / 4) * 512 +
(r % 32) * 16 + (r % 128) / 32 * 4 + g % 4, the order in which the tensor cores
take them.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5


def listed():
    return [
        # one token through the fused QKV projection of the 8B-shaped model: a call's latency
        {"name": "gemm-8b-qkv-1", "kind": "gemm", "M": 1, "N": 6144, "K": 4096, "bits": 8},
        # a serving batch's tokens through its down projection: a long sum, few rows
        {"name": "gemm-8b-down-16", "kind": "gemm", "M": 16, "N": 4096, "K": 14336, "bits": 8},
        # one token through its LM head: the longest stream of weights
        {"name": "gemm-8b-head-1", "kind": "gemm", "M": 1, "N": 128256, "K": 4096, "bits": 4},
        # a short prompt of odd length through a matrix of odd height
        {"name": "gemm-odd-77", "kind": "gemm", "M": 77, "N": 5003, "K": 2176, "bits": 8},
        # a prompt through the fused gate_up projection
        {"name": "gemm-8b-gate-up-2048", "kind": "gemm", "M": 2048, "N": 28672, "K": 4096, "bits": 8},
        # the largest product: prompts laid end to end, activations in 4 bits as well
        {"name": "gemm-8b-gate-up-8192-4", "kind": "gemm", "M": 8192, "N": 28672, "K": 4096, "bits": 4},
        # one token's norm: a call's latency
        {"name": "norm-8b-1", "kind": "norm", "M": 1, "K": 4096, "bits": 8, "pad": 0},
        # the norm of a long prompt
        {"name": "norm-8b-8192", "kind": "norm", "M": 8192, "K": 4096, "bits": 8, "pad": 0},
        # a serving batch between its projections
        {"name": "silu-8b-33", "kind": "silu", "M": 33, "K": 14336, "bits": 8, "pad": 8},
        # a prompt's fused gate_up rows
        {"name": "silu-8b-4096", "kind": "silu", "M": 4096, "K": 14336, "bits": 8, "pad": 0},
        # a prompt's attention outputs, read out of wider rows
        {"name": "quantize-odd-1001", "kind": "quantize", "M": 1001, "K": 4096, "bits": 8, "pad": 40},
        # a weight matrix on its way into the model
        {"name": "quantize-8b-down-4", "kind": "quantize", "M": 4096, "K": 14336, "bits": 4, "pad": 0},
    ]


def _log(rng, lo, hi):
    """A whole number spread over [lo, hi] by its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["gemm", "gemm", "gemm", "norm", "silu", "quantize"])
    bits = rng.choice([8, 8, 4])
    K = 128 * _log(rng, 1, 112)
    if kind == "gemm":
        M, N = _log(rng, 1, 8192), _log(rng, 1, 128256)
        while M * N * K > 8192 * 28672 * 4096:
            M, N = (M // 2, N) if M > 1024 else (M, N // 2)
        return {"kind": kind, "M": M, "N": N, "K": K, "bits": bits}
    M = _log(rng, 1, 16384)
    while M * K > 4096 * 14336:
        M = (M + 1) // 2
    return {"kind": kind, "M": M, "K": K, "bits": bits, "pad": rng.choice([0, 0, 8 * rng.randint(1, 64)])}


# ------------------------------------------------------------------ inputs --

def _tiled(scales, rows, K):
    """Scales [rows][K / 32] in blocks of 128 rows by four groups; rows behind the last are zero bytes."""
    full = torch.zeros(((rows + 127) // 128 * 128, K // 32), dtype=torch.uint8, device=scales.device)
    full[:rows] = scales
    return full.view(-1, 4, 32, K // 128, 4).permute(0, 3, 2, 1, 4).contiguous().view(-1)


def _untiled(scales, rows, K):
    return scales.view(-1, K // 128, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(-1, K // 32)[:rows]


# largest value, exponent of its power of two, bits of the mantissa, exponent of the smallest normal value
FORM = {8: (448.0, 8, 3, -6), 4: (6.0, 2, 1, 0)}


def _quantized(v, bits):
    """fp32 [rows][K] -> (values / scale, exponent of the scale) by group: the least power of two with which no
    value is over the type's largest, values to the nearest (ties to even).  A group of zeros has the scale 1, one
    with a value that is not finite the scale NaN (exponent 128)."""
    top, emax, mant, emin = FORM[bits]
    g = v.view(v.shape[0], -1, 32)
    amax = g.abs().amax(2)
    m, e = torch.frexp(amax)                                     # amax = m 2^e, m in [1/2, 1)
    e = e - 1 - emax + (2 * m * 2.0 ** emax > top).to(e.dtype)
    e = torch.where(amax > 0, e, torch.zeros_like(e)).clamp_min(-127)
    s = torch.ldexp(g, -e[..., None])
    _, ev = torch.frexp(s)
    step = torch.ldexp(torch.ones_like(s), (ev - 1).clamp_min(emin) - mant)
    q = torch.round(s / step) * step
    bad = ~torch.isfinite(amax)
    q = torch.where(bad[..., None], torch.zeros_like(q), q)
    return q, torch.where(bad, torch.full_like(e, 128), e)


def _values4():
    return torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device="cuda")


def _packed(q, bits):
    """Values over their scales [rows][K / 32][32] as code bytes [rows][K or K / 2]."""
    q = q.view(q.shape[0], -1)
    if bits == 8:
        return q.to(torch.float8_e4m3fn).view(torch.uint8)
    a = q.abs()
    code = (2 * a).clamp_max(4) + (a - 2).clamp(0, 2) + ((a - 4) / 2).clamp_min(0)      # 0 .5 1 1.5 2 3 4 6 -> 0 .. 7
    code = code.to(torch.uint8) + 8 * torch.signbit(q).to(torch.uint8)
    return code[:, 0::2] + 16 * code[:, 1::2]


def _operand(g, rows, K, bits, scale):
    """Codes and scales of normal values, their columns of different sizes as a model's channels are."""
    codes = torch.empty((rows, K * bits // 8), dtype=torch.uint8, device="cuda")
    exps = torch.empty((rows, K // 32), dtype=torch.uint8, device="cuda")
    channel = scale * torch.exp(0.5 * torch.randn(K, generator=g, device="cuda"))
    for r in range(0, rows, 16384):
        v = channel * torch.randn((min(16384, rows - r), K), generator=g, device="cuda")
        q, e = _quantized(v, bits)
        codes[r:r + 16384], exps[r:r + 16384] = _packed(q, bits), (e + 127).to(torch.uint8)
    return codes, _tiled(exps, rows, K)


def _half(g, rows, width, pad, scale=1.0):
    """fp16 [rows][width] read out of rows of width + pad."""
    return (scale * torch.randn((rows, width + pad), generator=g, device="cuda")).half()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    kind, M, K, bits = case["kind"], case["M"], case["K"], case["bits"]
    s = {"case": case, "kind": kind, "M": M, "K": K, "bits": bits}
    if kind == "gemm":
        N = s["N"] = case["N"]
        s["W"], s["W_scales"] = _operand(g, N, K, 4, 1 / math.sqrt(K))
        s["x"], s["x_scales"] = _operand(g, M, K, bits, 1.0)
        s["y"] = torch.zeros((M, N), dtype=torch.float16, device="cuda")
        return s
    s["stride"] = (2 * K if kind == "silu" else K) + case["pad"]
    s["x"] = _half(g, M, 2 * K if kind == "silu" else K, case["pad"], 1.5 if kind == "silu" else 1.0)
    if kind == "norm":
        s["residual"] = _half(g, M, K, 0, 3.0)
        s["gain"] = (1 + 0.3 * torch.randn(K, generator=g, device="cuda")).half()
        s["sum"] = torch.zeros((M, K), dtype=torch.float16, device="cuda")
    s["codes"] = torch.zeros((M, K * bits // 8), dtype=torch.uint8, device="cuda")
    s["scales"] = torch.zeros((M + 127) // 128 * 128 * (K // 32), dtype=torch.uint8, device="cuda")
    if bits == 4:
        s["values"] = torch.zeros((M, K), dtype=torch.float16, device="cuda")
    return s


# --------------------------------------------------------------- the calls --

def run(s):
    if own:
        return _own(s)
    return _plain(s)


def _own(s):
    from paper_2412_15803_gb300 import wq4
    kind, M, K, bits = s["kind"], s["M"], s["K"], s["bits"]
    if kind == "gemm":
        wq4.wq4_mx_gemm(s["W"], s["W_scales"], s["x"], s["x_scales"], s["y"], s["N"], K, M, bits)
        return s["y"]
    if kind == "norm":
        wq4.wq4_mx_norm(s["x"], s["stride"], s["residual"], K, s["gain"], EPS, s["sum"], K, s["codes"], s["scales"], M, K, bits)
    elif kind == "silu":
        wq4.wq4_mx_silu(s["x"], s["stride"], s["codes"], s["scales"], M, K, bits)
    else:
        wq4.wq4_mx_quantize(s["x"], s["stride"], s["codes"], s["scales"], M, K, bits)
    if bits == 8:
        out = {"codes": s["codes"].view(torch.float8_e4m3fn), "scales": s["scales"].view(torch.float8_e8m0fnu)}
    else:
        wq4.wq4_mx_dequantize(s["codes"], s["scales"], s["values"], K, M, K, bits)
        out = {"values": s["values"]}
    if kind == "norm":
        out["sum"] = s["sum"]
    return out


def _dequantized(codes, scales, rows, K, bits):
    """The fp32 values that codes and scales stand for."""
    if bits == 8:
        v = codes.view(torch.float8_e4m3fn).float()
    else:
        table = _values4()
        v = torch.stack((table[(codes & 15).int()], table[(codes >> 4).int()]), 2)
    return (v.view(rows, -1, 32) * torch.exp2(_untiled(scales, rows, K).float() - 127)[..., None]).view(rows, K)


def _plain(s):
    kind, M, K, bits = s["kind"], s["M"], s["K"], s["bits"]
    if kind == "gemm":
        x = _dequantized(s["x"], s["x_scales"], M, K, bits)
        return (x @ _dequantized(s["W"], s["W_scales"], s["N"], K, 4).T).half()
    out = {}
    if kind == "silu":
        gate, up = s["x"][:, :K].float(), s["x"][:, K:2 * K].float()
        v = gate / (1 + torch.exp(-gate)) * up
    elif kind == "norm":
        out["sum"] = (s["x"][:, :K].float() + s["residual"].float()).half()
        h = out["sum"].float()
        v = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["gain"].float()
    else:
        v = s["x"][:, :K].float()
    q, e = _quantized(v, bits)
    if bits == 8:
        out["codes"] = q.view(M, K).to(torch.float8_e4m3fn)
        out["scales"] = _tiled((e + 127).to(torch.uint8), M, K).view(torch.float8_e8m0fnu)
    else:
        out["values"] = torch.ldexp(q, e[..., None]).view(M, K).half()
    return out


def work(case):
    M, K, bits = case["M"], case["K"], case["bits"]
    held = M * K * bits // 8 + M * K // 32
    if case["kind"] == "gemm":
        N = case["N"]
        return {"bytes": N * K // 2 + N * K // 32 + held + 2 * M * N, "flops": 2 * M * N * K}
    if bits == 4:                                    # the codes are written, read again and come back as fp16
        held = 2 * held + 2 * M * K
    if case["kind"] == "norm":
        return {"bytes": 6 * M * K + 2 * K + held, "flops": 6 * M * K}
    return {"bytes": (4 if case["kind"] == "silu" else 2) * M * K + held, "flops": (8 if case["kind"] == "silu" else 2) * M * K}


# ------------------------------------------------------------ in 64 bits ----

def _magnitudes(bits):
    """Every magnitude of the type, in the order of its codes."""
    if bits == 4:
        return [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    return [(c & 7) * 2.0 ** -9 if c < 8 else (8 + (c & 7)) * 2.0 ** ((c >> 3) - 10) for c in range(127)]


def _exact_held(v, bits):
    """fp64 [rows][K] -> (the nearest value of the type over the group's scale, the scale [rows][K / 32])."""
    mags = torch.tensor(_magnitudes(bits), dtype=torch.float64, device=v.device)
    g = v.reshape(v.shape[0], -1, 32)
    amax = g.abs().amax(2)
    scale = torch.exp2(torch.ceil(torch.log2(torch.where(amax > 0, amax, torch.ones_like(amax)) / mags[-1])))
    scale = torch.where(amax > scale * mags[-1], 2 * scale, scale)          # the logarithm's own rounding
    scale = torch.where(amax <= scale / 2 * mags[-1], scale / 2, scale)
    scale = torch.where(amax > 0, scale, torch.ones_like(scale))
    a = g.abs() / scale[..., None]
    mids = (mags[1:] + mags[:-1]) / 2
    code = torch.bucketize(a, mids)
    tie = (a == mids[code.clamp_max(len(mids) - 1)]) & (code % 2 == 1)
    return torch.copysign(mags[code + tie.long()], g).view(v.shape), scale


def exact(case, seed):
    s = prepare(case, seed)
    kind, M, K, bits = s["kind"], s["M"], s["K"], s["bits"]
    if kind == "gemm":
        def full(codes, scales, rows, b):
            if b == 8:
                code = codes.long()
                table = torch.tensor(_magnitudes(8) + [math.nan], dtype=torch.float64, device="cuda")
                v = table[code & 127] * (1 - 2 * (code >> 7))
            else:
                code = torch.stack((codes & 15, codes >> 4), 2).view(rows, K).long()
                v = torch.tensor(_magnitudes(4), dtype=torch.float64, device="cuda")[code & 7] * (1 - 2 * (code >> 3))
            r = torch.arange(rows, device="cuda")[:, None]
            at = torch.arange(K // 32, device="cuda")[None]
            at = ((r // 128) * (K // 128) + at // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + at % 4
            return v * torch.exp2(scales[at].double() - 127).repeat_interleave(32, 1)
        x = full(s["x"], s["x_scales"], M, bits)
        return torch.cat([x @ full(s["W"][r:r + 16384].contiguous(), s["W_scales"][r * (K // 32):], min(16384, s["N"] - r), 4).T
                          for r in range(0, s["N"], 16384)], 1)
    out = {}
    x = s["x"].double()
    if kind == "silu":
        v = x[:, :K] * torch.sigmoid(x[:, :K]) * x[:, K:2 * K]
    elif kind == "norm":
        out["sum"] = (x[:, :K] + s["residual"].double())
        h = out["sum"].half().double()
        v = h * s["gain"].double() / torch.sqrt(h.square().sum(1, keepdim=True) / K + EPS)
    else:
        v = x[:, :K]
    q, scale = _exact_held(v, bits)
    if bits == 4:
        out["values"] = q * scale.repeat_interleave(32, 1)
        return out
    full = torch.full(((M + 127) // 128 * 128, K // 32), 2.0 ** -127, dtype=torch.float64, device="cuda")
    full[:M] = scale
    out["codes"] = q
    out["scales"] = full.view(-1, 4, 32, K // 128, 4).permute(0, 3, 2, 1, 4).reshape(-1)
    return out
