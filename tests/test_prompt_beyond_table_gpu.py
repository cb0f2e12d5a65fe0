"""Rows at positions beyond the page table's end: flagged, and they see of the table's tokens what their
position shows them, whatever the window's size."""
import numpy as np
import pytest

import oracle
from oracle import cache as oc
from paper_2412_15803_gb300 import wq4
from test_prompt_gpu import D, SCALE, Call, make

pytestmark = pytest.mark.gpu

MOST = 2 ** 31 - 1                                          # the largest length that the array can hold


def run(cap, Hq, Hkv, T, window, sinks, new=90, P=16, nan=()):
    q, k, v, table, _, starts, lens = make(24, [new], [cap - new], Hq, Hkv, P, hide=False)
    for t in nan:
        v[table[0, t // P], :, t % P, 3] = 0x7E00
    call = Call(q, k, v, table, starts, np.array([T], np.int32), Hq)
    call(window, sinks)
    got = oracle.half_to_double(call.result()).reshape(new, Hq, D)
    assert wq4.wq4_device_status() == 8
    K, V = (oracle.half_to_double(x[table[0]]).transpose(1, 0, 2, 3).reshape(Hkv, cap, D).repeat(Hq // Hkv, 0) for x in (k, v))
    Q = oracle.half_to_double(q).reshape(new, Hq, D)
    for r in range(new):
        t = np.flatnonzero(oc.seen(T - new + r, cap, window, sinks))
        if not t.size:
            assert np.all(got[r] == 0)
            continue
        s = SCALE * np.einsum("hd,htd->ht", Q[r], K[:, t])
        p = np.exp(s - s.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        o, A = np.einsum("ht,htd->hd", p, V[:, t]), np.einsum("ht,htd->hd", p, np.abs(V[:, t]))
        assert np.array_equal(np.isnan(got[r]), np.isnan(o))
        o, A, got[r] = np.nan_to_num(o), np.nan_to_num(A), np.nan_to_num(got[r])
        assert np.all(np.abs(got[r] - o) <= oc.attention_tolerance(o, A)), f"row {r}"


@pytest.mark.parametrize("cap,Hq,Hkv", [(320, 8, 2), (1600, 6, 2)])
@pytest.mark.parametrize("beyond", [1, 30, 1000, None])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 0), (100, 37), (-1, 5)])
def test_beyond_the_end(cap, Hq, Hkv, beyond, window, sinks):
    """Of the table's tokens (its capacity less one is the largest window here) or none."""
    run(cap, Hq, Hkv, cap + beyond if beyond else MOST, window if window >= 0 else cap + window, sinks)


@pytest.mark.parametrize("cap,Hq,Hkv", [(320, 8, 2), (1600, 6, 2)])
@pytest.mark.parametrize("sinks", [0, 5])
def test_what_only_rows_beyond_the_end_do_not_see(cap, Hq, Hkv, sinks):
    """A NaN that the rows on the table's tokens see and those behind the end, past their window, do not."""
    run(cap, Hq, Hkv, cap + 30, 100, sinks, nan=(cap - 90, cap - 75))


@pytest.mark.parametrize("cap,Hq,Hkv", [(320, 8, 2), (1600, 6, 2)])
@pytest.mark.parametrize("beyond", [1, 30, 1000, None])
@pytest.mark.parametrize("more,sinks", [(0, 0), (0, 5), (1, 0), (25, 7), (None, 3)])
def test_windows_of_the_capacity_and_more(cap, Hq, Hkv, beyond, more, sinks):
    """Rows behind the end outgrow them too."""
    run(cap, Hq, Hkv, cap + beyond if beyond else MOST, MOST if more is None else cap + more, sinks)
