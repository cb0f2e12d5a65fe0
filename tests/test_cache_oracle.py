"""The reference of the cache operators, pinned by closed forms and by the C oracle (no GPU)."""
import numpy as np
import pytest

import oracle
from oracle import cache as oc
from paper_2412_15803_gb300 import synth

D = 128


def _cache(seed, pages, n_kv=2, P=16):
    return synth.kv_cache(seed, pages, n_kv, P, D)


def test_ulp16():
    v = np.array([0.0, 1e-9, 6.1e-5, 0.999, 1.0, 1.5, 2.0, 65504.0])
    assert np.allclose(oc.ulp16(v), oracle.ulp16_array(v), rtol=0, atol=0)


@pytest.mark.parametrize("pos,window,sinks,want", [
    (5, 0, 0, [0, 1, 2, 3, 4, 5]), (5, 1, 0, [5]), (5, 2, 1, [0, 4, 5]), (5, 3, 4, [0, 1, 2, 3, 4, 5]),
    (2, 100, 0, [0, 1, 2]), (0, 1, 7, [0]), (-1, 4, 2, []), (7, 2, 9, list(range(8)))])
def test_what_a_row_sees(pos, window, sinks, want):
    assert np.flatnonzero(oc.seen(pos, 10, window, sinks)).tolist() == want


def test_one_row_a_sequence_without_a_window_is_decode_attention():
    lens = np.array([1, 17, 40, 0], np.int32)
    k, v = _cache(1, 8)
    table = synth.page_table(1, lens, 16, 8)
    q = synth.queries(1, 4, 4, D)
    o, A, owned = oc.attention(q, k, v, table, [0, 1, 2, 3, 4], lens, 0.1, 4)
    ref, ref_A, _ = oracle.paged_attention(q, k, v, table, lens, 0.1, 4)
    assert owned.all()
    assert np.abs(o - ref).max() < 1e-12 and np.abs(A - ref_A).max() < 1e-12


def test_equal_scores_average_the_values_seen():
    k, v = _cache(2, 3)
    k[:] = 0
    table = np.array([[2, 0, 1]], np.int32)
    q = synth.queries(2, 3, 2, D)
    o, _, _ = oc.attention(q, k, v, table, [0, 3], [40], 1.0, 2, window=5, sinks=2)
    vals = oracle.half_to_double(np.concatenate([v[p, 0] for p in (2, 0, 1)]))
    for r, pos in enumerate((37, 38, 39)):
        want = vals[[0, 1] + list(range(pos - 4, pos + 1))].mean(0)
        assert np.abs(o[r, 0] - want).max() < 1e-12


def test_append_rotates_by_position_and_leaves_the_rest():
    k, v = _cache(3, 4)
    table = np.array([[3, -1, 1], [0, -1, -1]], np.int32)
    qkv = synth.sum4_fp16(3, 9, 0, 4 * 6 * D).reshape(4, 6 * D)
    q, k64, v64 = oc.append(qkv, k, v, table, [0, 3, 4], [35, 1], 2, 500000.0)
    x = oracle.half_to_double(np.ascontiguousarray(qkv[1, 2 * D:2 * D + 2]))
    z = complex(x[0], x[1]) * np.exp(1j * 33.0)       # the first pair turns by the position
    assert abs(k64[1, 0, 1, 0] - z.real) < 1e-9 and abs(k64[1, 0, 1, 1] - z.imag) < 1e-9
    assert np.array_equal(v64[1, 1, 1], oracle.half_to_double(np.ascontiguousarray(qkv[1, 5 * D:])))
    assert np.array_equal(q[3], oracle.half_to_double(np.ascontiguousarray(qkv[3, :2 * D])))     # position 0
    changed = np.argwhere((v64 != oracle.half_to_double(v)).any((1, 3)))
    assert {tuple(c) for c in changed} <= {(1, 0), (1, 1), (1, 2), (0, 0)}


def _check(pool):
    """What the calls keep true."""
    want = np.zeros_like(pool.refs)
    for s, T in enumerate(pool.lens):
        n = pool.pages(int(T))
        assert np.all(pool.table[s, n:] == -1)
        for e in pool.table[s, :n]:
            if e >= 0:
                want[e] += 1
    assert np.array_equal(want, pool.refs)


def test_pool_life():
    kv = np.arange(10 * 2 * 16 * 4, dtype=np.float64).reshape(10, 2, 16, 4)
    pool = oc.Pool(10, 4, 6, 16, [kv])
    pool.reserve([1, 0], [33, 16])
    assert pool.table[1, :3].tolist() == [0, 1, 2] and pool.table[0, 0] == 3
    before = kv.copy()
    pool.fork([1, 1], [2, 3])
    assert pool.table[2, :3].tolist() == [0, 1, 4] and pool.table[3, :3].tolist() == [0, 1, 5]
    assert np.array_equal(kv[4, :, 0], before[2, :, 0]) and np.array_equal(kv[4, :, 1:], before[4, :, 1:])
    _check(pool)
    pool.free([1])
    assert pool.refs.tolist() == [2, 2, 0, 1, 1, 1, 0, 0, 0, 0]
    seen = kv[pool.table[3, 2]].copy()
    pool.compact()
    assert pool.refs.tolist() == [2, 2, 1, 1, 1, 0, 0, 0, 0, 0] and pool.table[3, 2] == 2
    assert np.array_equal(kv[2], seen)
    pool.trim([3], 2, 0)
    assert pool.table[3, :3].tolist() == [-1, -1, 2] and pool.refs[:2].tolist() == [1, 1]    # token 33 sees 32 and itself
    _check(pool)


def test_trim_keeps_what_the_next_token_sees():
    for T in range(0, 70):
        for window in (1, 2, 16, 17, 40):
            for sinks in (0, 1, 17):
                pool = oc.Pool(8, 1, 5, 16)
                pool.reserve([0], [T])
                pool.trim([0], window, sinks)
                visible = np.flatnonzero(oc.seen(T, T + 1, window, sinks))
                for t in visible[visible < T]:
                    assert pool.table[0, t // 16] >= 0
                _check(pool)


def test_pool_refusals():
    pool = oc.Pool(4, 3, 4, 16)
    pool.reserve([0, 0, 7, 1], [16, 32, 1, 65])
    assert pool.refused == 3 and pool.lens.tolist() == [16, 0, 0]
    pool.reserve([1, 2, 0], [64, 1, 16])       # 4 pages wanted of 3: neither it nor a later one that needs any
    assert pool.lens.tolist() == [16, 0, 0] and pool.refused == 5
    pool.fork([0, 1, 0, 0], [1, 2, 2, 9])      # 1 is a parent, 2 is listed before
    assert pool.refused == 5 + 3 and pool.lens.tolist() == [16, 0, 0]
    pool.copy_pages([0, 1, 2, 3, 9], [1, 3, 3, 0, 2])
    assert pool.refused == 8 + 5
    _check(pool)
