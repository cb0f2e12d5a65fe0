"""Every form of the microscaled product, set by a test hook, so that no estimate decides which of them runs.

Sizes, NaN, scales at the ends of their range, late writers, copies that never come and forms one after another,
against oracle/mx.py with the tolerance of tests/test_mx_gpu.py: products are exact, their sums K / 32 additions in
fp32 of at most 2^-22 of sum |w x| each, then one rounding to fp16.
"""
import contextlib
import time

import numpy as np
import pytest
import torch

import oracle
from oracle import mx
from paper_2412_15803_gb300 import wq4
from test_dependent_launch_gpu import late_copy  # noqa: F401  (a fixture)
from test_mx_gpu import any_operand, check_product, dev, gemm, sampled

pytestmark = pytest.mark.gpu

HALF, WHOLE, PAIRS = 1, 2, 3


@contextlib.contextmanager
def form_of(form, split=0):
    wq4.wq4_test_mx_form(form, split)
    try:
        yield
    finally:
        wq4.wq4_test_mx_form()


def operands(seed, M, N, K, bits):
    """(W, its scales, x, its scales) whose products stay well inside fp16."""
    rng = np.random.default_rng(seed)
    W, ws = any_operand(rng, N, K, 4)
    x, xs = any_operand(rng, M, K, bits)
    return W, ws, x, xs - np.uint8(6 if bits == 8 else 0)


def on_gpu(ops, K):
    W, ws, x, xs = ops
    return [dev(W), dev(mx.tiled(ws, K)), dev(x), dev(mx.tiled(xs, K))]


def check(form, split, M, N, K, bits):
    """Every output finite and repeated to the bit, sampled rows against the oracle; rows behind the last have NaN scales."""
    ops = operands(M * N + K, M, N, K, bits)
    with form_of(form, split):
        y = gemm(*ops, M, N, K, bits)
        assert np.array_equal(gemm(*ops, M, N, K, bits, 0x00), y)
    assert np.all((y & 0x7C00) != 0x7C00)
    n = sampled(N, np.random.default_rng(1))
    check_product(y[:, n], ops[0][n], ops[1][n], *ops[2:], bits)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("split", range(1, 9))
@pytest.mark.parametrize("form,M", [(HALF, 1), (HALF, 37), (HALF, 80), (WHOLE, 2), (WHOLE, 80), (WHOLE, 128), (WHOLE, 150)])
def test_split(form, M, split, bits):
    check(form, split, M, 1003, 2176, bits)


# several tiles a block, and ragged ones
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("form,M,N,K", [(HALF, 1, 90000, 256), (HALF, 33, 45001, 384), (HALF, 80, 40000, 128), (HALF, 79, 1, 128),
                                        (WHOLE, 1, 45000, 384), (WHOLE, 90, 20001, 256), (WHOLE, 300, 9000, 640), (WHOLE, 513, 130, 1152)])
def test_many_tiles(form, M, N, K, bits):
    check(form, 1, M, N, K, bits)


# rows that tensor copies can write and rows that they cannot, one tile a pair and several
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,N,K", [(1, 8, 128), (1, 257, 384), (70, 1003, 2176), (256, 256, 128), (257, 513, 640), (300, 5000, 1152),
                                   (777, 5003, 896), (2000, 5003, 384), (2048, 6600, 256), (600, 20001, 128), (130, 41000, 256)])
def test_pairs(M, N, K, bits):
    check(PAIRS, 0, M, N, K, bits)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("form,M,N,K", [(HALF, 5, 1000, 256), (WHOLE, 200, 1000, 384), (PAIRS, 70, 1000, 384), (PAIRS, 600, 9728, 256)])
def test_odd_addresses(form, M, N, K, bits):
    """y two bytes behind a multiple of 16: the same outputs, and what lies around them stays."""
    ops = operands(12, M, N, K, bits)
    with form_of(form):
        ref = gemm(*ops, M, N, K, bits)
        buf = torch.full((M * N + 20,), 0x1234, dtype=torch.int16, device="cuda")
        wq4.wq4_mx_gemm(*on_gpu(ops, K), buf[9:], N, K, M, bits)
        torch.cuda.synchronize()
    out = buf.cpu().numpy().view(np.uint16)
    assert np.array_equal(out[9:9 + M * N].reshape(M, N), ref) and np.all(out[:9] == 0x1234) and np.all(out[9 + M * N:] == 0x1234)


FORMS = [(HALF, 1, 5, 40000, 256), (HALF, 3, 5, 1000, 1152), (WHOLE, 1, 100, 20000, 256), (WHOLE, 4, 100, 1000, 2176),
         (PAIRS, 0, 300, 1003, 640), (PAIRS, 0, 2000, 5003, 256), (PAIRS, 0, 2000, 5000, 256)]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("form,split,M,N,K", FORMS)
def test_not_a_number(form, split, M, N, K, bits):
    """A NaN of one token or weight row is that token's or row's alone."""
    W, ws, x, xs = operands(5, M, N, K, bits)
    with form_of(form, split):
        ref = gemm(W, ws, x, xs, M, N, K, bits)
        bad = [3]
        ws[7, 1], xs[3, K // 32 - 1] = 255, 255
        if bits == 8:
            x[M - 1, 40] = 0x7F
            bad.append(M - 1)
        y = gemm(W, ws, x, xs, M, N, K, bits)
    nan = (y & 0x7FFF) > 0x7C00
    assert np.all(nan[:, 7]) and np.all(nan[bad])
    at = np.ix_(np.delete(np.arange(M), bad), np.delete(np.arange(N), 7))
    assert np.array_equal(y[at], ref[at])


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("form,split,M,N,K", FORMS)
def test_scales_at_the_ends_of_their_range(form, split, M, N, K, bits):
    """2^-127 (byte 0) and 2^127 (254): the products are those of scales near 1 that differ by as much."""
    rng = np.random.default_rng(9)
    W, _ = any_operand(rng, N, K, 4)
    x, _ = any_operand(rng, M, K, bits)
    low, high = rng.integers(0, 3, (N, K // 32), dtype=np.uint8), rng.integers(244, 247, (M, K // 32), dtype=np.uint8)
    low2, high2 = rng.integers(0, 3, (M, K // 32), dtype=np.uint8), rng.integers(244, 247, (N, K // 32), dtype=np.uint8)
    with form_of(form, split):
        for shift in (0, 8):          # 8: scales up to 254, codes' products small
            for ws, xs in ((low, high + np.uint8(shift)), (high2 + np.uint8(shift), low2)):
                near = gemm(W, (ws.astype(int) + (100 if ws.max() < 9 else -100)).astype(np.uint8), x,
                            (xs.astype(int) + (100 if xs.max() < 9 else -100)).astype(np.uint8), M, N, K, bits)
                y = gemm(W, ws, x, xs, M, N, K, bits)
                assert np.array_equal(y, near)
                n = sampled(N, rng)
                if shift == 0:
                    check_product(y[:, n], W[n], ws[n], x, xs, bits)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("form,split,M,N", [(HALF, 1, 3, 40), (HALF, 8, 3, 40), (WHOLE, 1, 100, 40), (WHOLE, 7, 100, 40), (PAIRS, 0, 70, 40)])
def test_long_sums_of_one_sign(form, split, M, N, bits):
    """K / 32 additions: 2^-12 of sum |w x| up to 32768 of K, K 2^-27 behind it.  What an addition drops adds up here."""
    K = 131200
    rng = np.random.default_rng(10)
    W = rng.integers(0, 256, (N, K // 2), dtype=np.uint8) & 0x77
    x = rng.integers(0, 127, (M, K), dtype=np.uint8) if bits == 8 else rng.integers(0, 256, (M, K // 2), dtype=np.uint8) & 0x77
    ws = rng.integers(111, 116, (N, K // 32), dtype=np.uint8)
    xs = rng.integers(124, 129, (M, K // 32), dtype=np.uint8) if bits == 8 else rng.integers(128, 133, (M, K // 32), dtype=np.uint8)
    with form_of(form, split):
        y = gemm(W, ws, x, xs, M, N, K, bits)
    ref, A = mx.product(mx.values(x, xs, bits), mx.values(W, ws, 4))
    assert 50 < ref.min() and ref.max() < 60000
    err = np.abs(oracle.half_to_double(y) - ref)
    assert np.all(err <= max(2.0 ** -12, K * 2.0 ** -27) * A + oracle.ulp16_array(ref))


@pytest.mark.parametrize("form,split", [(0, 0), (HALF, 1), (WHOLE, 1), (PAIRS, 0)])
def test_the_longest_sum(form, split):
    """K of 2^24 in one block or pair: no wait runs out.  Every product is 1/2, -1/2 or 0 and the sum below 2^23, so exact."""
    K, M, N = 1 << 24, 2, 3
    W = torch.zeros((N, K // 2), dtype=torch.uint8, device="cuda")          # 1 (0x2) and -1 (0xA) at some k
    at = torch.from_numpy(np.random.default_rng(3).permutation(K // 2)[:20000]).cuda()
    for n in range(N):
        W[n, at[:5000 + 4000 * n]] = 0x02
        W[n, at[15000:15000 + 1000 * n]] = 0xA0
    ws = torch.full((wq4.wq4_mx_scale_bytes(N, K),), 127, dtype=torch.uint8, device="cuda")
    x = torch.full((M, K), 0x38, dtype=torch.uint8, device="cuda")          # 1
    x[1, ::2] = 0xB8                                                        # -1 and 1 in turn
    xs = torch.full((wq4.wq4_mx_scale_bytes(M, K),), 126, dtype=torch.uint8, device="cuda")
    y = torch.zeros((M, N), dtype=torch.float16, device="cuda")
    with form_of(form, split):
        wq4.wq4_mx_gemm(W, ws, x, xs, y, N, K, M, 8)
        torch.cuda.synchronize()
    assert wq4.wq4_device_status() == 0
    lower, upper = np.array([5000, 9000, 13000]), np.array([0, 1000, 2000])
    assert np.array_equal(y.cpu().numpy(), np.stack([lower - upper, -lower - upper]).astype(np.float64) / 2)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("form,split,M,N,K", FORMS)
def test_operands_written_late(late_copy, form, split, M, N, K, bits):  # noqa: F811
    ops = on_gpu(operands(6, M, N, K, bits), K)
    y = torch.zeros((M, N), dtype=torch.int16, device="cuda")
    with form_of(form, split):
        wq4.wq4_mx_gemm(*ops, y, N, K, M, bits)
        torch.cuda.synchronize()
        ref = y.clone()
        assert not torch.any((ref & 0x7C00) == 0x7C00)
        for t in ops:
            src = t.clone()
            t.zero_()
            y.zero_()
            torch.cuda.synchronize()
            late_copy(t, src)
            wq4.wq4_mx_gemm(*ops, y, N, K, M, bits)
            torch.cuda.synchronize()
            assert torch.equal(y, ref)


@pytest.mark.parametrize("bits", [8, 4])
def test_forms_one_after_another(bits):
    """Every form behind every other, nothing waited for between: what a block leaves when it ends is the next one's."""
    rng = np.random.default_rng(13)
    calls = []
    for i, (form, split, M, N, K) in enumerate(FORMS + [(PAIRS, 0, 1, 8, 128), (HALF, 1, 1, 6144, 512), (PAIRS, 0, 256, 20000, 128)]):
        ops = on_gpu(operands(20 + i, M, N, K, bits), K)
        y = torch.zeros((M, N), dtype=torch.int16, device="cuda")
        calls.append((form, split, [*ops, y, N, K, M, bits]))

    def once(i):
        form, split, args = calls[i]
        with form_of(form, split):
            wq4.wq4_mx_gemm(*args)

    for i in range(len(calls)):
        once(i)
        torch.cuda.synchronize()
    want = [c[2][4].clone() for c in calls]
    for _ in range(30):
        for c in calls:
            c[2][4].zero_()
        torch.cuda.synchronize()
        order = [int(i) for i in np.concatenate([rng.permutation(len(calls)) for _ in range(4)])]
        for i in order:
            once(i)
        torch.cuda.synchronize()
        assert all(torch.equal(c[2][4], w) for c, w in zip(calls, want))
    assert wq4.wq4_device_status() == 0


def test_forms_on_two_streams_at_once():
    """Blocks of one form on SMs that another form's have not left."""
    calls = []
    for i, (form, split, M, N, K) in enumerate(FORMS):
        for bits in (8, 4):
            y = torch.zeros((M, N), dtype=torch.int16, device="cuda")
            calls.append((form, split, [*on_gpu(operands(40 + i, M, N, K, bits), K), y, N, K, M, bits]))
    for form, split, args in calls:
        with form_of(form, split):
            wq4.wq4_mx_gemm(*args)
    torch.cuda.synchronize()
    want = [c[2][4].clone() for c in calls]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    rng = np.random.default_rng(14)
    for _ in range(10):
        for c in calls:
            c[2][4].zero_()
        torch.cuda.synchronize()
        for i in rng.permutation(len(calls)):
            form, split, args = calls[i]
            with torch.cuda.stream(streams[int(i) % 2]), form_of(form, split):
                wq4.wq4_mx_gemm(*args)
        torch.cuda.synchronize()
        assert all(torch.equal(c[2][4], w) for c, w in zip(calls, want))
    assert wq4.wq4_device_status() == 0


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("form,split,M,N,K", FORMS)
def test_without_its_copies_it_ends(form, split, M, N, K, bits):
    """The waits for copies that never come run out, are flagged, and the next call is clean."""
    args = [*on_gpu(operands(11, M, N, K, bits), K), torch.zeros((M, N), dtype=torch.int16, device="cuda"), N, K, M, bits]
    with form_of(form, split):
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


def test_what_a_form_does_not_take_is_refused():
    ops = on_gpu(operands(15, 100, 300, 256, 8), 256)
    y = torch.zeros((100, 300), dtype=torch.int16, device="cuda")
    for form, split in ((HALF, 0), (HALF, 1), (WHOLE, 2)):
        with form_of(form, split):
            assert wq4.wq4_mx_gemm(*ops, y, 300, 256, 100, 8, check=False) == wq4.WQ4_ERR_UNSUPPORTED
    assert not torch.any(y)
