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
import time

import numpy as np
import pytest
import torch

import oracle
from oracle import mx
from paper_2412_15803_gb300 import wq4
from test_dependent_launch_gpu import late_copy  # noqa: F401  (a fixture)

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


def sampled(N, rng, n=400):
    """Weight rows whose outputs are checked: the edges of the first, some and the last tiles, others at random."""
    if N <= n:
        return np.arange(N)
    edges = np.concatenate([np.arange(0, 3), np.arange(125, 131), np.arange(253, 259), np.arange(N - 300, N)])
    return np.unique(np.concatenate([edges, rng.integers(0, N, n - 315)]))


def check_any(M, N, K, bits):
    """Every output finite and repeated to the bit, sampled rows against the oracle."""
    rng = np.random.default_rng(M * N + K)
    W, ws = any_operand(rng, N, K, 4)
    x, xs = any_operand(rng, M, K, bits)
    xs -= 6 if bits == 8 else 0
    y = gemm(W, ws, x, xs, M, N, K, bits)
    assert np.all((y & 0x7C00) != 0x7C00)
    n = sampled(N, rng)
    check_product(y[:, n], W[n], ws[n], x, xs, bits)
    assert np.array_equal(gemm(W, ws, x, xs, M, N, K, bits, 0x00), y)


# pairs of blocks: tiles of 256 rows by 256 tokens, one and several a pair, ragged in each direction, rows that a
# tensor copy can write and rows that it cannot
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,N,K", [(200, 30003, 384), (513, 6600, 1280), (1000, 9728, 640), (1500, 10001, 128), (2000, 5128, 2176),
                                   (1030, 40000, 256)])
def test_gemm_pairs(M, N, K, bits):
    check_any(M, N, K, bits)


# K split over a cluster, one or two blocks an SM; tokens in tiles of every size
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,N,K", [(1, 6144, 4096), (3, 2001, 8192), (16, 4096, 14336), (20, 6144, 4096), (40, 300, 14208), (77, 5003, 2176),
                                   (100, 1000, 8064), (128, 4100, 14336), (150, 1003, 4096), (270, 1100, 14336), (90, 200, 1152), (1, 40000, 1024)])
def test_gemm_split(M, N, K, bits):
    check_any(M, N, K, bits)


@pytest.mark.parametrize("M,N,K", [(3, 264, 256), (600, 9728, 256)])
def test_gemm_into_odd_addresses(M, N, K):
    """y two bytes behind a multiple of 16: no tensor copy can write it, and what lies around it stays."""
    rng = np.random.default_rng(12)
    W, ws = any_operand(rng, N, K, 4)
    x, xs = any_operand(rng, M, K, 8)
    xs -= 6
    ref = gemm(W, ws, x, xs, M, N, K, 8)
    buf = torch.full((M * N + 20,), 0x1234, dtype=torch.int16, device="cuda")
    wq4.wq4_mx_gemm(dev(W), dev(mx.tiled(ws, K)), dev(x), dev(mx.tiled(xs, K)), buf[9:], N, K, M, 8)
    torch.cuda.synchronize()
    out = buf.cpu().numpy().view(np.uint16)
    assert np.array_equal(out[9:9 + M * N].reshape(M, N), ref) and np.all(out[:9] == 0x1234) and np.all(out[9 + M * N:] == 0x1234)


@pytest.mark.parametrize("bits", [8, 4])
def test_gemm_over_drawn_sizes(bits):
    """Sizes spread by their logarithm over what the call is for."""
    rng = np.random.default_rng(bits)
    for _ in range(12):
        K = 128 * int(np.exp(rng.uniform(0, np.log(112))) + 0.5)
        M, N = (int(np.exp(rng.uniform(0, np.log(hi))) + 0.5) for hi in (2000, 20000))
        if M * N * K < 1.5e10:
            check_any(M, N, K, bits)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,N,K", [(5, 400, 512), (100, 300, 2048), (600, 9728, 256)])
def test_gemm_scales_and_codes_that_are_not_numbers(M, N, K, bits):
    """A NaN of one token or weight row is that token's or row's alone; scales from 2^-127 to 2^127."""
    rng = np.random.default_rng(5)
    W, ws = any_operand(rng, N, K, 4)
    x, xs = any_operand(rng, M, K, bits)
    xs -= 6 if bits == 8 else 0
    ref = gemm(W, ws, x, xs, M, N, K, bits)
    ws2, xs2, x2 = ws.copy(), xs.copy(), x.copy()
    ws2[7, 1], xs2[3, K // 32 - 1] = 255, 255
    bad = [3]
    if bits == 8:
        x2[M - 1, 40] = 0x7F
        bad.append(M - 1)
    y = gemm(W, ws2, x2, xs2, M, N, K, bits)
    nan = (y & 0x7FFF) > 0x7C00
    assert np.all(nan[:, 7]) and np.all(nan[bad])
    keep = np.delete(np.arange(M), bad)
    cols = np.delete(np.arange(N), 7)
    assert np.array_equal(y[np.ix_(keep, cols)], ref[np.ix_(keep, cols)])
    # far exponents that cancel: the same products
    far = gemm(W, (ws.astype(int) - 120).astype(np.uint8), x, (xs.astype(int) + 120).astype(np.uint8), M, N, K, bits)
    assert np.array_equal(far, ref)


# ------------------------------------------------------------- a run of them --

class Layer:
    """A decoder layer's projections and what stands between, in microscaled form: tokens x [M][H], residual h."""

    def __init__(self, M, bits, seed, H=512, F=1152, nq=768):
        rng = np.random.default_rng(seed)
        self.M, self.bits, self.H, self.F, self.nq = M, bits, H, F, nq
        self.host = [(rng.standard_normal(s) * s[1] ** -0.5).astype(np.float16) for s in ((nq, H), (H, H), (2 * F, H), (H, F))]
        self.mats = []
        for w in self.host:
            N, K = w.shape
            c, s = torch.zeros((N, K // 2), dtype=torch.uint8, device="cuda"), torch.zeros(wq4.wq4_mx_scale_bytes(N, K), dtype=torch.uint8, device="cuda")
            wq4.wq4_mx_quantize(dev(w), K, c, s, N, K, 4)
            self.mats.append((c, s))
        self.gains = [(1 + 0.3 * rng.standard_normal(H)).astype(np.float16) for _ in range(2)]
        self.dgains = [dev(g) for g in self.gains]
        self.x0, self.h0 = rng.standard_normal((M, H)).astype(np.float16), (2 * rng.standard_normal((M, H))).astype(np.float16)
        self.x, self.h = dev(self.x0), dev(self.h0)
        half = lambda n: torch.zeros((M, n), dtype=torch.int16, device="cuda")
        self.qkv, self.o, self.gu, self.y = half(nq), half(H), half(2 * F), half(H)
        self.held = [(torch.zeros((M, n * bits // 8), dtype=torch.uint8, device="cuda"),
                      torch.zeros(wq4.wq4_mx_scale_bytes(M, n), dtype=torch.uint8, device="cuda")) for n in (H, H, H, F)]

    def calls(self):
        M, H, F, nq, b = self.M, self.H, self.F, self.nq, self.bits
        (wq, sq), (wo, so), (wg, sg), (wd, sd) = self.mats
        (c0, s0), (c1, s1), (c2, s2), (c3, s3) = self.held
        return [lambda: wq4.wq4_mx_norm(self.x, H, self.h, H, self.dgains[0], 1e-5, self.h, H, c0, s0, M, H, b),
                lambda: wq4.wq4_mx_gemm(wq, sq, c0, s0, self.qkv, nq, H, M, b),
                lambda: wq4.wq4_mx_quantize(self.qkv, nq, c1, s1, M, H, b),
                lambda: wq4.wq4_mx_gemm(wo, so, c1, s1, self.o, H, H, M, b),
                lambda: wq4.wq4_mx_norm(self.o, H, self.h, H, self.dgains[1], 1e-5, self.h, H, c2, s2, M, H, b),
                lambda: wq4.wq4_mx_gemm(wg, sg, c2, s2, self.gu, 2 * F, H, M, b),
                lambda: wq4.wq4_mx_silu(self.gu, 2 * F, c3, s3, M, F, b),
                lambda: wq4.wq4_mx_gemm(wd, sd, c3, s3, self.y, H, F, M, b)]

    def run(self, sync=False):
        for c in self.calls():
            c()
            if sync:
                torch.cuda.synchronize()

    def state(self):
        torch.cuda.synchronize()
        return [t.clone() for t in (self.h, self.qkv, self.o, self.gu, self.y, *(t for p in self.held for t in p))]

    def reset(self):
        self.x.copy_(dev(self.x0))
        self.h.copy_(dev(self.h0))
        torch.cuda.synchronize()


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M", [1, 5, 150])
def test_layer_stage_by_stage(M, bits):
    """Each stage on the GPU's own input to it."""
    L = Layer(M, bits, 3)
    L.run()
    h1, qkv, o, gu, y, *held = [t.cpu().numpy() for t in L.state()]
    codes = [(held[2 * i], held[2 * i + 1][mx.scale_index(M, n)]) for i, n in enumerate((L.H, L.H, L.H, L.F))]
    f16 = lambda a: a.view(np.float16)
    hmid, v = mx.norm(L.x0, L.h0, L.gains[0], 1e-5)
    assert not mx.wrong_groups(*codes[0], v, bits, 2.0 ** -18).any()
    assert np.array_equal(codes[1][0], mx.quantize(f16(qkv)[:, :L.H].astype(np.float64), bits)[0])
    h, v = mx.norm(f16(o), hmid, L.gains[1], 1e-5)
    assert np.array_equal(f16(h1), h) and not mx.wrong_groups(*codes[2], v, bits, 2.0 ** -18).any()
    delta = (8 + 1.2 * np.abs(f16(gu)[:, :L.F].astype(np.float64))) * 2.0 ** -23
    assert not mx.wrong_groups(*codes[3], mx.silu(f16(gu)), bits, delta, 2.0 ** -100).any()
    for i, out in enumerate((qkv, o, gu, y)):
        N, K = L.host[i].shape
        wc, ws = L.mats[i][0].cpu().numpy(), L.mats[i][1].cpu().numpy()[mx.scale_index(N, K)]
        c_ref, s_ref = mx.quantize(L.host[i].astype(np.float64), 4)
        assert np.array_equal(wc, c_ref) and np.array_equal(ws, s_ref)
        check_product(out.view(np.uint16), wc, ws, *codes[i], bits)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M", [1, 40, 600])
def test_layer_back_to_back(late_copy, M, bits):  # noqa: F811
    """Nothing waited for between the calls, the first input written late by a kernel that lets its dependents launch."""
    L = Layer(M, bits, 4, H=1024, F=2048, nq=1536)
    L.run(sync=True)
    want = L.state()
    for _ in range(4):
        L.reset()
        src = L.x.clone()
        L.x.zero_()
        torch.cuda.synchronize()
        late_copy(L.x, src, 100_000)
        L.run()
        assert same(L.state(), want)
    assert wq4.wq4_device_status() == 0


# forms whose blocks of one call and of the next are resident together, and the others
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,N,K", [(1, 6144, 4096), (16, 4096, 14336), (1, 20000, 512), (77, 5003, 2176), (1000, 9728, 512)])
def test_products_back_to_back(M, N, K, bits):
    rng = np.random.default_rng(13)
    calls, want = [], []
    for _ in range(3):
        W, ws = any_operand(rng, N, K, 4)
        x, xs = any_operand(rng, M, K, bits)
        xs -= 6 if bits == 8 else 0
        want.append(gemm(W, ws, x, xs, M, N, K, bits))
        calls.append([dev(W), dev(mx.tiled(ws, K)), dev(x), dev(mx.tiled(xs, K)), torch.zeros((M, N), dtype=torch.int16, device="cuda"), N, K, M, bits])
    for _ in range(20):
        for c in calls:
            wq4.wq4_mx_gemm(*c)
    torch.cuda.synchronize()
    for c, w in zip(calls, want):
        assert np.array_equal(c[4].cpu().numpy().view(np.uint16), w)
    assert wq4.wq4_device_status() == 0


# one size of each form of the product: two blocks an SM, K split, one block an SM, pairs
@pytest.mark.parametrize("M,N,K", [(1, 20000, 512), (1, 2048, 4096), (100, 2048, 1024), (1000, 9728, 512)])
@pytest.mark.parametrize("bits", [8, 4])
def test_gemm_reads_weights_that_a_running_kernel_writes(late_copy, M, N, K, bits):  # noqa: F811
    rng = np.random.default_rng(6)
    W, ws = (dev(a) for a in any_operand(rng, N, K, 4))
    x, xs = (dev(a) for a in any_operand(rng, M, K, bits))
    ws, xs = (dev(mx.tiled(a.cpu().numpy(), K)) for a in (ws, xs))
    y = torch.zeros((M, N), dtype=torch.int16, device="cuda")
    wq4.wq4_mx_gemm(W, ws, x, xs, y, N, K, M, bits)
    torch.cuda.synchronize()
    ref = y.clone()
    for t in (W, ws, x, xs):
        src = t.clone()
        t.zero_()
        y.zero_()
        torch.cuda.synchronize()
        late_copy(t, src)
        wq4.wq4_mx_gemm(W, ws, x, xs, y, N, K, M, bits)
        torch.cuda.synchronize()
        assert torch.equal(y, ref)


@pytest.mark.parametrize("M", [1, 200])
def test_layer_in_a_graph(M):
    """Captured, and replayed with other inputs in the same buffers."""
    L, other = Layer(M, 8, 7), Layer(M, 8, 8)
    L.run()                                    # attributes are set outside the capture
    g = torch.cuda.CUDAGraph()
    L.reset()
    with torch.cuda.graph(g):
        L.run()
    L.reset()
    g.replay()
    got = L.state()
    L.reset()
    L.run()
    assert same(got, L.state())
    for (c, s), (c2, s2) in zip(L.mats, other.mats):
        c.copy_(c2)
        s.copy_(s2)
    for a, b in zip(L.dgains, other.dgains):
        a.copy_(b)
    L.x.copy_(other.x)
    L.h.copy_(other.h)
    g.replay()
    got = L.state()
    other.run()
    assert same(got, other.state())


def test_layers_on_two_streams_at_once():
    a, b = Layer(30, 8, 9), Layer(300, 4, 10)
    a.run()
    b.run()
    want = [a.state(), b.state()]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        a.reset()
        b.reset()
        for ca, cb in zip(a.calls(), b.calls()):
            with torch.cuda.stream(streams[0]):
                ca()
            with torch.cuda.stream(streams[1]):
                cb()
        assert same(a.state(), want[0]) and same(b.state(), want[1])
    assert wq4.wq4_device_status() == 0


# every form of the product, one tile a block and several
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,N,K", [(1, 6144, 4096), (3, 60000, 512), (100, 2048, 1024), (200, 1024, 4096), (1500, 28672, 512)])
def test_gemm_without_its_copies_ends(M, N, K, bits):
    """The waits for copies that never come run out, are flagged, and the next call is clean."""
    rng = np.random.default_rng(11)
    W, ws = any_operand(rng, N, K, 4)
    x, xs = any_operand(rng, M, K, bits)
    args = [dev(W), dev(mx.tiled(ws, K)), dev(x), dev(mx.tiled(xs, K)), torch.zeros((M, N), dtype=torch.int16, device="cuda"), N, K, M, bits]
    wq4.wq4_mx_gemm(*args)
    torch.cuda.synchronize()
    ref = args[4].clone()
    assert wq4.wq4_device_status() == 0
    try:
        wq4.wq4_test_copy_stall(2)
        t0 = time.perf_counter()
        wq4.wq4_mx_gemm(*args)
        torch.cuda.synchronize()
        took = time.perf_counter() - t0
        flags = wq4.wq4_device_status()
    finally:
        wq4.wq4_test_copy_stall()
    assert flags == 1 and 0.4 < took < 4.0
    args[4].zero_()
    wq4.wq4_mx_gemm(*args)
    torch.cuda.synchronize()
    assert wq4.wq4_device_status() == 0 and torch.equal(args[4], ref)
