"""Window attention of one token and its refusals against the fp64 reference.

The bar is that of the paged attention: |o - o_ref| <= 2e-3 * sum_t p_t |V_t| + ulp16(|o_ref|).
"""
import math

import numpy as np
import pytest
import torch

import oracle
from oracle import cache as oc
from paper_2412_15803_gb300 import synth, wq4

pytestmark = pytest.mark.gpu

D = 128
NAN16 = np.uint16(0x7E00)
SCALE = 1.0 / math.sqrt(D)


def dev(a, dtype=np.int16):
    return torch.from_numpy(np.ascontiguousarray(a).view(dtype)).cuda()


def make(seed, lens, Hq, Hkv, P, window, sinks):
    """A cache whose every row that no new token sees holds NaN, and whose table entries of pages
    without a visible token lie outside the pool."""
    lens = np.asarray(lens, np.int32)
    pages = int(((lens.astype(np.int64) + P - 1) // P).sum()) + 2
    k, v = synth.kv_cache(seed, pages, Hkv, P, D)
    table = synth.page_table(seed, lens, P, pages)
    q = synth.queries(seed, len(lens), Hq, D)
    bad, full = table.copy(), np.zeros((pages, P), bool)
    for b, T in enumerate(lens):
        t = np.flatnonzero(oc.seen(T - 1, T, window, sinks))
        full[table[b][t // P], t % P] = True
        hidden = np.setdiff1d(np.arange(table.shape[1]), t // P)
        bad[b][hidden] = 1_000_000 if b % 2 else -1
    for a in (k, v):
        a.transpose(0, 2, 1, 3)[~full] = NAN16
    return q, k, v, table, bad, lens


def run(q, k, v, table, lens, Hq, window, sinks, scale=SCALE, q_stride=None, out_stride=None):
    batch, Hkv, P = len(lens), k.shape[1], k.shape[2]
    out_stride = out_stride or Hq * D
    kd, vd, td, ld, qd = dev(k), dev(v), dev(table, np.int32), dev(lens, np.int32), dev(q)
    out = torch.full((batch, out_stride), -1, dtype=torch.int16, device="cuda")
    ws = torch.zeros(wq4.wq4_paged_attention_workspace_bytes(batch, Hq, Hkv, D), dtype=torch.uint8, device="cuda")
    cache = wq4.kv_cache_desc(kd, vd, td, P)
    wq4.wq4_window_attention(cache, qd, q_stride or Hq * D, ld, out, out_stride, batch, Hq, scale, window, sinks, ws, ws.numel())
    torch.cuda.synchronize()
    return out.cpu().numpy().view(np.uint16)


def check(got, q, k, v, table, lens, Hq, window, sinks, scale=SCALE):
    o, A, _ = oc.attention(q, k, v, table, list(range(len(lens) + 1)), lens, scale, Hq, window, sinks)
    g = oracle.half_to_double(got[:, :Hq * D]).reshape(o.shape)
    bad = np.argwhere(~(np.abs(g - o) <= oc.attention_tolerance(o, A)))
    assert bad.size == 0, f"{len(bad)} out of tolerance, first {bad[0]}"


LENS = [0, 1, 2, 16, 17, 40, 129, 333, 1000]


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 16), (15, 0), (16, 1), (17, 4), (100, 17), (128, 33),
                                          (300, 700), (999, 1), (4096, 4)])
@pytest.mark.parametrize("Hq,Hkv,P", [(32, 8, 16), (24, 8, 32), (8, 1, 64), (5, 5, 16), (14, 2, 256)])
def test_parity(Hq, Hkv, P, window, sinks):
    q, k, v, table, bad, lens = make(window + sinks, LENS, Hq, Hkv, P, window, sinks)
    got = run(q, k, v, bad, lens, Hq, window, sinks)
    assert wq4.wq4_device_status() == 0
    check(got, q, k, v, table, lens, Hq, window, sinks)
    assert np.all(got[0] == 0)


def test_long_sequences_are_split_and_joined():
    lens = [20000, 9000, 3]
    q, k, v, table, bad, lens = make(5, lens, 16, 2, 16, 7777, 100)
    got = run(q, k, v, bad, lens, 16, 7777, 100)
    assert wq4.wq4_device_status() == 0
    check(got, q, k, v, table, lens, 16, 7777, 100)
    assert np.array_equal(got, run(q, k, v, bad, lens, 16, 7777, 100))


def test_a_window_that_hides_nothing_gives_the_paged_attention():
    q, k, v, table, _, lens = make(6, [100, 1, 300], 8, 2, 16, 0, 0)
    want = run(q, k, v, table, lens, 8, 0, 5)
    check(want, q, k, v, table, lens, 8, 0, 0)
    for window in (300, 10 ** 9, 2 ** 31 - 1):
        assert np.array_equal(run(q, k, v, table, lens, 8, window, 0), want)
    assert np.array_equal(run(q, k, v, table, lens, 8, 2, 2 ** 31 - 1), want)


def test_strided_rows():
    q, k, v, table, bad, lens = make(7, [50, 129], 8, 2, 16, 20, 3)
    wide = np.concatenate([q, np.full((2, 512), NAN16)], 1)
    got = run(wide, k, v, bad, lens, 8, 20, 3, scale=1.0, q_stride=8 * D + 512, out_stride=8 * D + 64)
    check(got, q, k, v, table, lens, 8, 20, 3, scale=1.0)
    assert np.all(got[:, 8 * D:] == 0xFFFF)


def test_a_visible_page_outside_the_pool_is_flagged():
    q, k, v, table, _, lens = make(8, [100], 8, 2, 16, 0, 0)
    table[0, 5] = 10 ** 6
    run(q, k, v, table, lens, 8, 40, 0)
    assert wq4.wq4_device_status() == 16
    run(q, k, v, table, lens, 8, 4, 16)       # the page is not looked at
    assert wq4.wq4_device_status() == 0
