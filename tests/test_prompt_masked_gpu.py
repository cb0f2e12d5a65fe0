"""Rows computed again because a value beside theirs, which they do not see, is not finite.

Such a row is as if that value were not there: the bar is that of every other row, and what a row
does see of it reaches it: NaN as NaN, an infinity as an infinity, or as NaN where its weight is
below half of the smallest fp16 in the units that the kernel keeps weights in (0 * infinity = NaN).
"""
import numpy as np
import pytest

import oracle
from oracle import cache as oc
from paper_2412_15803_gb300 import wq4
from test_prompt_gpu import D, NAN16, SCALE, Call, make

pytestmark = pytest.mark.gpu


def poison(k, v, table, where):
    """NaN in a key of the first head, an infinity and a NaN in a value of the last, at the tokens (sequence, t)."""
    P = k.shape[2]
    for b, t in where:
        k[table[b, t // P], 0, t % P, 5] = NAN16
        v[table[b, t // P], -1, t % P, 7] = 0x7C00
        v[table[b, t // P], -1, t % P, 100] = NAN16


def check(got, q, k, v, table, starts, lens, Hq, window, sinks, scale):
    o, A, _ = oc.attention(q, k, v, table, starts, lens, scale, Hq, window, sinks)
    g = oracle.half_to_double(got).reshape(o.shape)
    fine = np.isfinite(o)
    assert fine.any() and not fine.all()
    assert np.all(np.isnan(g[np.isnan(o)]))
    assert np.all(np.isnan(g[np.isinf(o)]) | (g[np.isinf(o)] == o[np.isinf(o)]))
    bad = np.argwhere(fine & ~(np.abs(g - np.where(fine, o, 0)) <= oc.attention_tolerance(np.where(fine, o, 0), np.where(fine, A, 0))))
    assert bad.size == 0, f"{len(bad)} out of tolerance, first (row, head, dim) {bad[0]}"


def run(new, ctx, Hq, Hkv, P, where, window=0, sinks=0, scale=SCALE, seed=22):
    q, k, v, table, given, starts, lens = make(seed, new, ctx, Hq, Hkv, P, window, sinks)
    poison(k, v, table, where)
    call = Call(q, k, v, given, starts, lens, Hq)
    call(window, sinks, scale)
    got = call.result()
    assert wq4.wq4_device_status() == 0
    check(got, q, k, v, table, starts, lens, Hq, window, sinks, scale)


@pytest.mark.parametrize("scale", [-SCALE, -0.3, 0.3])
@pytest.mark.parametrize("window,sinks,tokens", [(0, 0, (150, 260)), (40, 2, (150,)), (64, 0, (30, 200))])
def test_scales_of_either_sign(window, sinks, tokens, scale):
    run([300], [20], 8, 2, 16, [(0, t) for t in tokens], window, sinks, scale)


@pytest.mark.parametrize("scale", [SCALE, -SCALE])
@pytest.mark.parametrize("window,sinks,where", [(0, 0, (9005, 9011)), (5000, 40, (9003,)), (5000, 40, (4006,)), (6000, 0, (3010, 9014))])
def test_a_few_rows_cut_into_many_parts(window, sinks, where, scale):
    """16 tokens over 9000: 71 key tiles of each of two heads in shares of four, so every item is joined
    from many parts.  The value is in the first, the last or both: of some rows' future or just behind
    their window."""
    run([16], [9000], 8, 2, 16, [(0, t) for t in where], window, sinks, scale)


@pytest.mark.parametrize("scale", [SCALE, -SCALE])
@pytest.mark.parametrize("window,sinks", [(0, 0), (150, 20)])
@pytest.mark.parametrize("new,ctx", [([200] * 26, [600] * 26), ([120] * 90 + [40], [20] * 90 + [900])])
def test_several_items_a_block(new, ctx, window, sinks, scale):
    """182 items of up to seven key tiles, and 362 of one or two (one of eight): more items than blocks,
    a block's share holds parts of two or three and many are joined from two.  In every third sequence
    a value in the middle of the new tokens, in every seventh one more at their end."""
    where = [(b, ctx[b] + new[b] // 2) for b in range(0, len(new), 3)] + [(b, ctx[b] + new[b] - 2) for b in range(0, len(new), 7)]
    run(new, ctx, 8, 1, 16, where, window, sinks, scale, seed=23)
