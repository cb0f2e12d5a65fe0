"""Microscaled matrices on the GPU against oracle/mx.py (64 bits).

quantize and dequantize are exact arithmetic and compared bit for bit.  The gate's values
are off by at most (8 + 1.2 |gate|) 2^-23 of themselves in fp32 (the exponential 2 +
1.173 |gate| ulp, the quotient 2, a sum and a product half an ulp each) or 2^-100 (gates
below -87, where the quotient becomes 0), the norm's by 2^-18 (at most 64
sums of squares a thread and ten of threads, half of 74 * 2^-24 after the root, rsqrtf 2
ulp, a quotient and two products): a code is then the nearest of a value within that of the
exact one.  Products are exact and their sums in fp32: K / 32 additions of at most 2^-22
of sum |w x| each, under 2^-12 of it to K = 16384, and one rounding to fp16.
"""
import numpy as np
import pytest
import torch

import oracle
from oracle import mx
from paper_2412_15803_gb300 import wq4

pytestmark = pytest.mark.gpu


def dev(a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view(np.int16) if a.dtype == np.float16 else a).cuda()


def padded(rows, stride, value=np.nan):
    """fp16 rows laid `stride` apart, what lies between filled with `value`."""
    out = np.full((len(rows), stride), value, np.float16)
    out[:, :rows.shape[1]] = rows
    return out


def held(M, K, bits):
    """Buffers for codes and scales, filled with a mark."""
    return (torch.full((M + 1, K * bits // 8), 0xA5, dtype=torch.uint8, device="cuda"),
            torch.full((wq4.wq4_mx_scale_bytes(M, K) + 64,), 0xA5, dtype=torch.uint8, device="cuda"))


def taken(codes, scales, M, K):
    """Host codes and scale bytes; what lies beside them keeps its mark."""
    torch.cuda.synchronize()
    c, s = codes.cpu().numpy(), scales.cpu().numpy()
    at = mx.scale_index(M, K)
    rest = np.ones(len(s), bool)
    rest[at] = False
    assert np.all(c[M] == 0xA5) and np.all(s[rest] == 0xA5)
    return c[:M], s[at]


def special_rows(rng, M, K):
    """Normal values with rows and groups where a scale can go wrong."""
    x = (rng.standard_normal((M, K)) * np.exp2(rng.integers(-12, 12, (M, K // 32)).repeat(32, 1))).astype(np.float16)
    rows = [lambda r: 0 * r, lambda r: np.where(np.arange(K) % 32 == 5, -np.inf, r), lambda r: np.where(np.arange(K) % 64 == 7, np.nan, r),
            lambda r: np.float16(2.0 ** -24) * np.sign(r), lambda r: 448 * np.sign(r), lambda r: 6 * np.sign(r) * np.exp2(np.arange(K) // 32 % 5),
            lambda r: np.where(np.arange(K) % 32 == 0, 448, 17), lambda r: np.where(np.arange(K) % 32 == 0, 6, 2.5),
            lambda r: np.where(np.arange(K) % 32 == 0, 449, 17.5), lambda r: np.full(K, -65504.0), lambda r: -0.0 * np.abs(r)]
    for i, f in enumerate(rows[:M]):
        x[i] = f(x[i].astype(np.float64))
    return x


SHAPES = [(1, 128), (3, 384), (11, 256), (33, 4096), (130, 1152), (300, 2176), (5, 14336)]
MANY = [(700, 128), (9001, 384), (1001, 2048), (1250, 2176), (640, 14336)]       # rows that a thread or a block takes several of


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,K", SHAPES + MANY)
def test_quantize_and_back(M, K, bits):
    rng = np.random.default_rng(M + K)
    x, stride = special_rows(rng, M, K), K + 24
    codes, scales = held(M, K, bits)
    wq4.wq4_mx_quantize(dev(padded(x, stride)), stride, codes, scales, M, K, bits)
    c, s = taken(codes, scales, M, K)
    c_ref, s_ref = mx.quantize(x.astype(np.float64), bits)
    assert np.array_equal(s, s_ref)
    assert np.array_equal(c, c_ref)
    y = torch.full((M, K + 16), 0x1234, dtype=torch.int16, device="cuda")
    wq4.wq4_mx_dequantize(codes, scales, y, K + 16, M, K, bits)
    torch.cuda.synchronize()
    y = y.cpu().numpy()
    assert np.all(y[:, K:] == 0x1234)
    ref = mx.half(mx.values(c_ref, s_ref, bits))
    assert np.array_equal(y[:, :K].copy().view(np.float16), ref, equal_nan=True)


@pytest.mark.parametrize("bits", [8, 4])
def test_dequantize_any_bytes(bits):
    """Every code under every scale."""
    M, K = 256, 8192 // bits
    codes = np.tile(np.arange(256, dtype=np.uint8), (M, K * bits // 8 // 256))
    exps = np.tile(np.arange(M, dtype=np.uint8)[:, None], (1, K // 32))
    y = torch.zeros((M, K), dtype=torch.int16, device="cuda")
    wq4.wq4_mx_dequantize(dev(codes), dev(mx.tiled(exps, K)), y, K, M, K, bits)
    torch.cuda.synchronize()
    assert np.array_equal(y.cpu().numpy().view(np.float16), mx.half(mx.values(codes, exps, bits)), equal_nan=True)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,K", SHAPES + MANY)
def test_silu(M, K, bits):
    rng = np.random.default_rng(2 * M + K)
    gu = (1.5 * rng.standard_normal((M, 2 * K))).astype(np.float16)
    if M > 2:
        gu[1, :K] = np.linspace(-120, 20, K)
        gu[2, 100:110] = [np.inf, -np.inf, np.nan, 0, -0.0, 65504, -65504, 1e-7, -1e-7, 88]
    stride = 2 * K + 8
    codes, scales = held(M, K, bits)
    wq4.wq4_mx_silu(dev(padded(gu, stride)), stride, codes, scales, M, K, bits)
    c, s = taken(codes, scales, M, K)
    with np.errstate(invalid="ignore"):
        v = mx.silu(gu)
    delta = (8 + 1.2 * np.abs(np.nan_to_num(gu[:, :K].astype(np.float64), posinf=0, neginf=0))) * 2.0 ** -23
    assert not mx.wrong_groups(c, s, v, bits, delta, 2.0 ** -100).any()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("residual,gain,summed", [(True, True, "new"), (True, True, "residual"), (True, False, "x"), (False, True, None),
                                                  (False, False, "new"), (True, True, None)])
@pytest.mark.parametrize("M,K", SHAPES + MANY + [(2, 16384), (2, 33024)])
def test_norm(M, K, residual, gain, summed, bits):
    rng = np.random.default_rng(3 * M + K)
    x = rng.standard_normal((M, K)).astype(np.float16)
    res = (3 * rng.standard_normal((M, K))).astype(np.float16) if residual else None
    g = (1 + 0.3 * rng.standard_normal(K)).astype(np.float16) if gain else None
    if M > 2:
        x[1], x[2] = 0, 60000
        if residual:
            res[1] = 0
    xs, rs, ss = K + 8, K + 16, K + 24
    xd, rd, sd = dev(padded(x, xs)), dev(padded(res, rs)) if residual else None, None
    if summed == "new":
        sd = torch.full((M, ss), 0x1234, dtype=torch.int16, device="cuda")
    elif summed:
        sd, ss = (xd, xs) if summed == "x" else (rd, rs)
    before = sd.clone() if sd is not None else None
    codes, scales = held(M, K, bits)
    wq4.wq4_mx_norm(xd, xs, rd, rs, dev(g) if gain else None, 1e-5, sd, ss, codes, scales, M, K, bits)
    c, s = taken(codes, scales, M, K)
    with np.errstate(invalid="ignore"):
        h, v = mx.norm(x, res, g, 1e-5)
    assert not mx.wrong_groups(c, s, v, bits, 2.0 ** -18).any()
    if sd is not None:
        assert np.array_equal(sd.cpu().numpy()[:, :K].copy().view(np.float16), h)
        assert torch.equal(sd[:, K:], before[:, K:])


def operand(rng, rows, K, bits, scale):
    """Codes and scale bytes of normal values of different sizes by channel."""
    v = scale * rng.standard_normal((rows, K)) * np.exp(0.5 * rng.standard_normal(K))
    return mx.quantize(v, bits)


def any_operand(rng, rows, K, bits):
    """Codes of every finite value and scales of a few binades."""
    c = rng.integers(0, 256, (rows, K * bits // 8), dtype=np.uint8)
    if bits == 8:
        c[(c & 127) == 127] = 0x3A
    return c, rng.integers(124, 130, (rows, K // 32), dtype=np.uint8)


def gemm(W, ws, x, xs, M, N, K, bits, fill=0xFF):
    y = torch.full((M + 1, N), -1, dtype=torch.int16, device="cuda")
    wq4.wq4_mx_gemm(dev(W), dev(mx.tiled(ws, K, fill)), dev(x), dev(mx.tiled(xs, K, fill)), y, N, K, M, bits)
    torch.cuda.synchronize()
    assert wq4.wq4_device_status() == 0
    assert torch.all(y[M] == -1)
    return y[:M].cpu().numpy().view(np.uint16)


def check_product(y16, W, ws, x, xs, bits):
    ref, A = mx.product(mx.values(x, xs, bits), mx.values(W, ws, 4))
    err = np.abs(oracle.half_to_double(y16) - ref)
    bad = np.argwhere(~(err <= 2.0 ** -12 * A + oracle.ulp16_array(ref)))
    assert bad.size == 0, f"{len(bad)} out of tolerance, first {bad[:3]}"


GEMMS = [(1, 1, 128), (1, 128, 128), (1, 300, 4096), (2, 130, 256), (5, 257, 384), (16, 1003, 640), (17, 129, 1152), (31, 64, 128),
         (33, 1000, 2176), (64, 128, 1024), (65, 257, 384), (77, 503, 2176), (128, 128, 512), (129, 5, 128), (200, 1003, 896),
         (257, 260, 256), (300, 640, 14336), (513, 384, 1280), (700, 1300, 384)]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,N,K", GEMMS)
def test_gemm(M, N, K, bits):
    """Scales of rows behind the last are NaN here: they are of no effect."""
    rng = np.random.default_rng(M * N + K)
    W, ws = operand(rng, N, K, 4, 1.0)
    x, xs = operand(rng, M, K, bits, K ** -0.5)
    check_product(gemm(W, ws, x, xs, M, N, K, bits), W, ws, x, xs, bits)


# pairs of blocks: tiles of 256 rows by 256 tokens, one and several a pair, ragged in each direction, rows that a
# tensor copy can write and rows that it cannot
PAIRS = [(129, 19464, 128), (200, 20003, 384), (513, 6600, 1280), (256, 40000, 256), (1000, 9728, 640), (700, 25001, 128), (2000, 5128, 2176)]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,N,K", PAIRS)
def test_gemm_pairs(M, N, K, bits):
    rng = np.random.default_rng(M * N + K)
    W, ws = any_operand(rng, N, K, 4)
    x, xs = any_operand(rng, M, K, bits)
    xs -= 6 if bits == 8 else 0
    y = gemm(W, ws, x, xs, M, N, K, bits)
    check_product(y, W, ws, x, xs, bits)
    assert np.array_equal(gemm(W, ws, x, xs, M, N, K, bits, 0x00), y)


# K split over a cluster, one tile a cluster and several; tokens in tiles of every size
SPLITS = [(1, 40000, 1024), (3, 20001, 1152), (16, 29000, 640), (20, 6144, 4096), (40, 12000, 896), (77, 5003, 2176), (100, 9000, 1024),
          (128, 8200, 3200), (150, 3000, 4096), (270, 2100, 2304)]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,N,K", SPLITS)
def test_gemm_split(M, N, K, bits):
    rng = np.random.default_rng(M * N + K)
    W, ws = any_operand(rng, N, K, 4)
    x, xs = any_operand(rng, M, K, bits)
    xs -= 6 if bits == 8 else 0
    y = gemm(W, ws, x, xs, M, N, K, bits)
    check_product(y, W, ws, x, xs, bits)
    assert np.array_equal(gemm(W, ws, x, xs, M, N, K, bits, 0x00), y)
