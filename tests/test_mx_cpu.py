"""Microscaled matrices without a GPU: the oracle's pins, the calls' refusals, and their launches on several devices.

Addresses are made up and never read: an argument error returns before anything is enqueued.
"""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import mx
from paper_2412_15803_gb300 import wq4

HERE = os.path.dirname(os.path.abspath(__file__))
A = 1 << 40
INVALID, ALIGN, UNSUPPORTED = wq4.WQ4_ERR_INVALID, wq4.WQ4_ERR_ALIGN, wq4.WQ4_ERR_UNSUPPORTED
NAN, INF = float("nan"), float("inf")


# ------------------------------------------------------------- the oracle --

def test_e4m3_is_torchs():
    codes = np.arange(256, dtype=np.uint8)
    t = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    v = mx.values(np.tile(codes, (1, 1)), np.full((1, 8), 127, np.uint8), 8)[0]
    assert np.array_equal(v, t, equal_nan=True)


def test_codes_are_the_nearest():
    """Against a search over every code, ties to the even one."""
    rng = np.random.default_rng(0)
    for bits in (8, 4):
        mags = mx.magnitudes(bits)
        a = np.concatenate([rng.uniform(0, 1.2 * mags[-1], 3000), (mags[1:] + mags[:-1]) / 2, mags, np.exp2(rng.uniform(-14, 9, 3000))])
        got = mx.nearest(a, bits)
        for x, c in zip(a, got):
            d = np.abs(mags - x)
            best = np.flatnonzero(d == d.min())
            assert c == (best[0] if len(best) == 1 else best[best % 2 == 0][0])


@pytest.mark.parametrize("bits", [8, 4])
def test_scales_are_the_least_that_fit(bits):
    rng = np.random.default_rng(1)
    v = rng.standard_normal((40, 128)) * np.exp2(rng.integers(-40, 40, (40, 4)).repeat(32, 1))
    top = mx.magnitudes(bits)[-1]
    v[0, 0], v[1, 32], v[2, 64] = 2.0 ** 50 * top, 2.0 ** 50 * top * (1 + 2.0 ** -40), 0
    v[2, 64:96], v[3, 5], v[4, 40] = 0, INF, NAN
    codes, exps = mx.quantize(v, bits)
    amax = np.abs(v.reshape(40, 4, 32)).max(2)
    bad = ~np.isfinite(amax)
    assert np.array_equal(exps == 255, bad) and exps[0, 0] == 127 + 50 and exps[1, 1] == 127 + 51 and exps[2, 2] == 127
    s = np.where(bad, 1.0, np.ldexp(1.0, exps.astype(int) - 127))
    ok = ~bad & (amax > 0)
    assert np.all(amax[ok] <= top * s[ok]) and np.all(amax[ok] > top * s[ok] / 2)
    q = mx.values(codes, exps, bits)
    assert np.all(np.isnan(q.reshape(40, 4, 32)[bad])) and np.all(q[2, 64:96] == 0)
    good = np.repeat(~bad, 32, 1)
    assert np.all(np.abs(q - v)[good] <= (np.abs(v) * (2.0 ** -4 if bits == 8 else 0.25) + np.repeat(s, 32, 1) * (2.0 ** -10 if bits == 8 else 0.25))[good])
    assert not mx.wrong_groups(codes, exps, v, bits, 0.0).any()


@pytest.mark.parametrize("bits", [8, 4])
def test_wrong_groups_sees_wrong_groups(bits):
    v = np.random.default_rng(2).standard_normal((3, 256))
    codes, exps = mx.quantize(v, bits)
    c = codes.copy()
    c[1, 3] ^= 1
    assert mx.wrong_groups(c, exps, v, bits, 1e-6).sum() == 1
    for d in (-1, 1, 100):
        e = exps.copy()
        e[2, 4] = int(e[2, 4]) + d
        assert mx.wrong_groups(codes, e, v, bits, 1e-6)[2, 4]


def test_scale_places():
    """The layout in words: blocks of 128 rows by 128 columns; in one, 32 rows of four words, a byte a group."""
    K, rows = 384, 300
    at = mx.scale_index(rows, K)
    assert len(np.unique(at)) == at.size and at.max() < mx.scale_bytes(rows, K) == 384 * 12
    want = [(0, 0, 0), (0, 3, 3), (0, 4, 512), (1, 0, 16), (31, 0, 31 * 16), (32, 0, 4), (64, 1, 9), (127, 11, 1024 + 31 * 16 + 12 + 3),
            (128, 0, 1536), (299, 5, 2 * 1536 + 512 + (299 - 288) * 16 + 4 + 1)]
    for r, g, b in want:
        assert at[r, g] == b, (r, g)
    assert wq4.wq4_mx_scale_bytes(rows, K) == mx.scale_bytes(rows, K)
    assert [wq4.wq4_mx_scale_bytes(*a) for a in ((0, 128), (-1, 128), (4, 0), (4, 100), (4, 64))] == [0] * 5


def test_nibbles_lower_first():
    v = np.zeros((1, 128))
    v[0, :4] = [6, -0.5, 1.5, 4]
    codes, exps = mx.quantize(v, 4)
    assert codes[0, 0] == 0x97 and codes[0, 1] == 0x63 and exps[0, 0] == 127


def test_norm_and_silu_closed_forms():
    x = np.full((1, 128), 2, np.float16)
    h, v = mx.norm(x, x, None, 16.0 * 3)
    assert np.all(h == 4) and np.allclose(v, 4 / 8)
    _, v = mx.norm(x, None, np.full(128, 3, np.float16), 0.0)
    assert np.allclose(v, 3)
    gu = np.array([[0, np.log(3), -np.log(3), 100] + [0] * 124 + [5, 4, 4, 2] + [0] * 124], np.float64)
    assert np.allclose(mx.silu(gu)[0, :4], [0, 3 * np.log(3), -np.log(3), 200])


# --------------------------------------------------------------- refusals --

@pytest.mark.parametrize("changes,want", [
    (dict(W=0), INVALID), (dict(ws=None), INVALID), (dict(x=0), INVALID), (dict(xs=0), INVALID), (dict(y=0), INVALID),
    (dict(N=0), INVALID), (dict(M=0), INVALID), (dict(M=-5), INVALID), (dict(K=0), INVALID), (dict(K=192), INVALID), (dict(K=-128), INVALID),
    (dict(bits=6), INVALID), (dict(bits=0), INVALID), (dict(N=1 << 30, K=4096), INVALID), (dict(M=1 << 30, K=4096), INVALID),
    (dict(W=A + 16), ALIGN), (dict(ws=2 * A + 8), ALIGN), (dict(x=4 * A + 8), ALIGN), (dict(xs=5 * A + 4), ALIGN), (dict(y=6 * A + 1), ALIGN),
    (dict(y=A + 64), INVALID), (dict(y=2 * A + 512), INVALID), (dict(y=4 * A), INVALID), (dict(y=5 * A + 2), INVALID),
    (dict(N=1 << 28, M=1 << 20, K=128, W=1 << 50, ws=1 << 52, x=1 << 54, xs=1 << 56, y=1 << 58), UNSUPPORTED)])
def test_gemm_refuses(changes, want):
    a = dict(W=A, ws=2 * A, x=4 * A, xs=5 * A, y=6 * A, N=640, K=512, M=300, bits=8)
    a.update(changes)
    assert wq4.load().wq4_mx_gemm(a["W"], a["ws"], a["x"], a["xs"], a["y"], a["N"], a["K"], a["M"], a["bits"], None) == want


ROWS = [(dict(M=0), INVALID), (dict(M=-1), INVALID), (dict(K=0), INVALID), (dict(K=160), INVALID), (dict(bits=5), INVALID),
        (dict(M=1 << 30, K=4096, stride=8192), INVALID), (dict(codes=0), INVALID), (dict(scales=None), INVALID), (dict(x=0), INVALID),
        (dict(codes=A + 16), ALIGN), (dict(scales=2 * A + 8), ALIGN), (dict(x=4 * A + 8), ALIGN), (dict(stride=1036), ALIGN),
        (dict(scales=A + 1024), INVALID), (dict(codes=4 * A + 1024), INVALID), (dict(scales=4 * A + 32), INVALID), (dict(stride=248), INVALID)]


@pytest.mark.parametrize("changes,want", ROWS)
def test_row_calls_refuse(changes, want):
    a = dict(x=4 * A, stride=1032, codes=A, scales=2 * A, M=300, K=512, bits=8)
    a.update(changes)
    L = wq4.load()
    for f in (L.wq4_mx_quantize, L.wq4_mx_silu):
        assert f(a["x"], a["stride"], a["codes"], a["scales"], a["M"], a["K"], a["bits"], None) == want
    assert L.wq4_mx_dequantize(a["codes"], a["scales"], a["x"], a["stride"], a["M"], a["K"], a["bits"], None) == want


def test_silu_refuses_rows_without_room_for_both():
    assert wq4.load().wq4_mx_silu(4 * A, 1016, A, 2 * A, 3, 512, 8, None) == INVALID


@pytest.mark.parametrize("changes,want", [c for c in ROWS] + [
    (dict(eps=0.0), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=NAN), INVALID), (dict(eps=INF), INVALID),
    (dict(rs=504), INVALID), (dict(rs=1028), ALIGN), (dict(res=6 * A + 2), ALIGN), (dict(gain=7 * A + 8), ALIGN),
    (dict(ss=504), INVALID), (dict(ss=1028), ALIGN), (dict(sum=8 * A + 8), ALIGN),
    (dict(sum=4 * A), INVALID), (dict(sum=6 * A, ss=1024), INVALID), (dict(sum=4 * A + 1024, ss=1032), INVALID), (dict(sum=7 * A), INVALID),
    (dict(sum=A), INVALID), (dict(sum=2 * A), INVALID), (dict(codes=6 * A), INVALID), (dict(codes=7 * A), INVALID), (dict(scales=7 * A), INVALID),
    (dict(res=4 * A + 2064, sum=4 * A, ss=1032), INVALID)])
def test_norm_refuses(changes, want):
    a = dict(x=4 * A, stride=1032, res=6 * A, rs=1040, gain=7 * A, eps=1e-5, sum=8 * A, ss=1048, codes=A, scales=2 * A, M=300, K=512, bits=8)
    a.update(changes)
    assert wq4.load().wq4_mx_norm(a["x"], a["stride"], a["res"], a["rs"], a["gain"], a["eps"], a["sum"], a["ss"], a["codes"], a["scales"],
                                  a["M"], a["K"], a["bits"], None) == want


# --------------------------------------------------------------- launches --

CHILD = r"""
import ctypes, sys
fake = ctypes.CDLL(sys.argv[1])
from paper_2412_15803_gb300 import wq4
L = wq4.load(build_if_missing=False)
A = 1 << 40
for device in (0, 1, 0, 3):
    fake.fake_set_device(device)
    n = fake.fake_launches()
    def once(rc):
        global n
        n += 1
        assert rc == 0 and fake.fake_launches() == n, (device, rc, fake.fake_launches(), n)
    for bits in (8, 4):
        for M, N, K in ((1, 1, 128), (1, 6144, 4096), (1, 128256, 4096), (16, 4096, 14336), (77, 5003, 2176), (128, 1024, 8192), (300, 640, 14336),
                        (2048, 28672, 4096), (3, 1 << 24, 128), (1 << 24, 3, 128), (2147483647, 1, 128)):
            once(L.wq4_mx_gemm(A, 4 * A, 8 * A, 16 * A, 32 * A, N, K, M, bits, None))
        for M, K in ((1, 128), (1, 512), (1, 4096), (3, 16384), (2, 33024), (8192, 4096), (5000, 11008), (1 << 20, 128), (2147483647, 128)):
            once(L.wq4_mx_quantize(A, 2 * K, 16 * A, 64 * A, M, K, bits, None))
            once(L.wq4_mx_silu(A, 2 * K, 16 * A, 64 * A, M, K, bits, None))
            once(L.wq4_mx_dequantize(16 * A, 64 * A, A, 2 * K, M, K, bits, None))
            once(L.wq4_mx_norm(A, 2 * K, 4 * A, K, 128 * A, 1e-5, A, 2 * K, 16 * A, 64 * A, M, K, bits, None))
            once(L.wq4_mx_norm(A, 2 * K, None, 0, None, 1e-5, None, 0, 16 * A, 64 * A, M, K, bits, None))
"""


def test_launches_on_every_device(fake_cudart):
    env = dict(os.environ, LD_PRELOAD=fake_cudart, PYTHONPATH=os.path.dirname(HERE))
    r = subprocess.run([sys.executable, "-c", CHILD, fake_cudart], env=env, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
