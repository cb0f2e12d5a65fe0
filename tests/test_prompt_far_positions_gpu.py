"""Rotations of a prompt's rows at the largest positions that a page table can name.

The bar is the call's own at every position: half an fp16 ulp + 2^-22 of the pair's larger element.  An angle
that is off by d shows there only where the rotated element is small, and most (sqrt(2) d) where the pair's
elements are alike in size.  So the positions are those at which one frequency's angle is nearest to an odd
eighth of a turn, and the pairs are chosen such that one of the rotated elements nearly vanishes.  (A
frequency rounded to a double is 2^-54 or more off, an angle at 2^30 then 2^-24 or more, and a product of two
such frequencies up to 2^-22.4: the bases are those at which that is worst, with its pair, and common ones.)
"""
from decimal import Decimal, localcontext

import numpy as np
import pytest

import oracle
from oracle import cache as oc
from paper_2412_15803_gb300 import wq4
from test_prompt_gpu import D, run_append

pytestmark = pytest.mark.gpu

HQ, HKV, P, STRIDE, BATCH = 14, 2, 1 << 16, (1 << 14) - 1, 96
PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459")


def turns(theta):
    """theta^(-i / 64) in turns, times 2^96, from 60 digits."""
    with localcontext() as c:
        c.prec = 60
        ln = Decimal(theta).ln()
        return [int((ln * -i / 64).exp() / (2 * PI) * 2 ** 96) for i in range(D // 2)]


def angles(w, positions):
    return np.array([[(int(p) * x % 2 ** 96) / 2 ** 96 * 2 * np.pi for x in w] for p in positions])


@pytest.mark.parametrize("theta,pair", [(500000.0, 2), (10000.0, 1), (2.0, 23), (1.0000021117363704, 42), (1.0245430083734806, 33),
                                        (1.000000142667479, 31), (1e300, 0)])
@pytest.mark.parametrize("end", [STRIDE * P, 1 << 28])
def test_within_half_an_ulp_and_2_to_the_minus_22(theta, pair, end):
    w = turns(theta)
    near = np.abs(angles(w[pair:pair + 1], range(end - P, end))[:, 0] * 4 / np.pi % 2 - 1)
    pos = end - P + np.sort(np.argsort(near, kind="stable")[:BATCH])
    a = angles(w, pos)
    c, s = np.cos(a)[:, None], np.sin(a)[:, None]                                   # [rows][1][64]
    first = np.linspace(1, 2, 1024, endpoint=False).astype(np.float16)[None, :, None]
    x = np.zeros((BATCH, HQ + HKV, D // 2, 2), np.float16)
    with np.errstate(over="ignore", divide="ignore", invalid="ignore"):
        for half, ratio in ((0, c / s), (1, -s / c)):                               # the first or the second element vanishes
            second = (first * ratio).astype(np.float16)
            left = np.abs(first * c - second * s if half == 0 else first * s + second.astype(np.float64) * c)
            left = np.where(np.abs(second) < 8, left, np.inf)
            heads = np.argsort(left, axis=1)[:, :8]                                 # [rows][8][64]
            at = slice(8 * half, 8 * half + 8)
            x[:, at, :, 0] = np.take_along_axis(np.broadcast_to(first, left.shape), heads, 1)
            x[:, at, :, 1] = np.clip(np.nan_to_num(np.take_along_axis(second, heads, 1)), -8, 8)
    qkv = np.zeros((BATCH, (HQ + 2 * HKV) * D), np.float16)
    qkv[:, :(HQ + HKV) * D] = x.reshape(BATCH, -1)
    table = np.full((BATCH, STRIDE), -1, np.int32)
    table[:, (end - 1) // P] = 0                                                    # all rows in one page, a place each
    k = np.zeros((1, HKV, P, D), np.uint16)
    got, keys, _ = run_append(qkv.view(np.uint16), k, k, table, list(range(BATCH + 1)), pos + 1, HQ, HKV, theta)
    assert wq4.wq4_device_status() == 0
    mine = np.concatenate([got[:, :HQ * D], keys[0][:, pos % P].transpose(1, 0, 2).reshape(BATCH, -1)], 1)
    mine = oracle.half_to_double(np.ascontiguousarray(mine)).reshape(x.shape)
    x = x.astype(np.float64)
    ref = np.stack([x[..., 0] * c - x[..., 1] * s, x[..., 0] * s + x[..., 1] * c], -1)
    assert np.median(np.abs(ref).min(-1)) < 2.0 ** -12                              # the pairs do what they are for
    bar = oc.ulp16(ref) / 2 + 2.0 ** -22 * np.abs(x).max(-1, keepdims=True)
    assert np.all(np.abs(mine - ref) <= bar), f"{(np.abs(mine - ref) / bar).max()} of the bar"
