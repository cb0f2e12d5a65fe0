"""Prompt append and prompt attention against the fp64 reference.

Append: rotated elements within half an fp16 ulp + 2^-22 of the pair's larger element, values bit for bit.
Attention: |o - o_ref| <= 2e-3 * sum_t p_t |V_t| + ulp16(|o_ref|), the bar of the decode attention.
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
THETA = 500000.0


def dev(a, dtype=np.int16):
    return torch.from_numpy(np.ascontiguousarray(a).view(dtype)).cuda()


def starts_of(new):
    return [0] + np.cumsum(new).tolist()


def make(seed, new, ctx, Hq, Hkv, P, window=0, sinks=0, pad=0, hide=True):
    """New tokens `new` behind `ctx` cached ones.  Rows of the cache that no row of the call sees hold
    NaN, and so do rows that no sequence owns; pages without a seen token are outside the pool."""
    new, ctx = np.asarray(new), np.asarray(ctx)
    lens = (new + ctx).astype(np.int32)
    pages = int(((lens.astype(np.int64) + P - 1) // P).sum()) + 2
    k, v = synth.kv_cache(seed, pages, Hkv, P, D)
    table = synth.page_table(seed, lens, P, pages)
    rows = int(new.sum()) + pad
    q = synth.queries(seed, rows, Hq, D)
    q[rows - pad:] = NAN16
    given = table.copy()
    if hide:
        full = np.zeros((pages, P), bool)
        for b, T in enumerate(lens):
            t = np.arange(T)
            if new[b]:
                first = T - new[b]
                t = t if not window else t[(t > first - window) | (t < sinks)]
            else:
                t = t[:0]
            full[table[b][t // P], t % P] = True
            given[b][np.setdiff1d(np.arange(table.shape[1]), t // P)] = 10 ** 6 if b % 2 else -1
        for a in (k, v):
            a.transpose(0, 2, 1, 3)[~full] = NAN16
    return q, k, v, table, given, starts_of(new), lens


class Call:
    """Device copies of one call's arrays."""

    def __init__(self, q, k, v, table, starts, lens, Hq, q_stride=None, out_stride=None, batch=None):
        self.Hq, self.rows, self.batch = Hq, q.shape[0], batch or len(lens)
        self.q_stride, self.out_stride = q_stride or q.shape[1], out_stride or Hq * D
        self.q, self.k, self.v = dev(q), dev(k), dev(v)
        self.table, self.lens = dev(table, np.int32), dev(np.asarray(lens, np.int32), np.int32)
        self.starts = dev(np.asarray(starts, np.int32), np.int32)
        self.out = torch.full((self.rows, self.out_stride), -1, dtype=torch.int16, device="cuda")
        n = wq4.wq4_prompt_attention_workspace_bytes(self.batch, self.rows, Hq, k.shape[1], D)
        assert n > 0
        self.ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")     # of any contents
        self.cache = wq4.kv_cache_desc(self.k, self.v, self.table, k.shape[2])

    def __call__(self, window=0, sinks=0, scale=SCALE, stream=None):
        return wq4.wq4_prompt_attention(self.cache, self.q, self.q_stride, self.starts, self.lens, self.out, self.out_stride,
                                        self.batch, self.rows, self.Hq, scale, window, sinks, self.ws, self.ws.numel(), stream)

    def result(self):
        torch.cuda.synchronize()
        return self.out.cpu().numpy().view(np.uint16)


def check(got, q, k, v, table, starts, lens, Hq, window=0, sinks=0, scale=SCALE):
    o, A, owned = oc.attention(q, k, v, table, starts, lens, scale, Hq, window, sinks)
    g = oracle.half_to_double(np.ascontiguousarray(got[:, :Hq * D])).reshape(o.shape)
    assert np.all(got[~owned] == 0xFFFF), "a row of no sequence was written"
    with np.errstate(invalid="ignore"):
        ok = np.where(np.isnan(o), np.isnan(g), np.abs(g - o) <= oc.attention_tolerance(o, np.nan_to_num(A)))
    ok[~owned] = True
    bad = np.argwhere(~ok)
    assert bad.size == 0, f"{len(bad)} out of tolerance, first (row, head, dim) {bad[0]}: {g[tuple(bad[0])]} for {o[tuple(bad[0])]}"


def both(new, ctx, Hq, Hkv, P, window=0, sinks=0, pad=0, seed=1):
    q, k, v, table, given, starts, lens = make(seed, new, ctx, Hq, Hkv, P, window, sinks, pad)
    call = Call(q, k, v, given, starts, lens, Hq)
    call(window, sinks)
    got = call.result()
    assert wq4.wq4_device_status() == 0
    check(got, q, k, v, table, starts, lens, Hq, window, sinks)


HEADS = [(8, 2), (6, 2), (2, 2), (8, 1), (5, 1), (14, 2)]


@pytest.mark.parametrize("Hq,Hkv", HEADS)
@pytest.mark.parametrize("new,ctx,P", [([1], [0], 16), ([77], [0], 16), ([128], [0], 32), ([129, 1, 0, 40], [0, 63, 5, 1], 16),
                                       ([3, 31, 64, 65], [1000, 127, 128, 129], 64), ([300], [257], 256)])
def test_causal(Hq, Hkv, new, ctx, P):
    both(new, ctx, Hq, Hkv, P, pad=3)


@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (3, 1), (2, 2)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 3), (16, 16), (100, 4), (128, 0), (129, 130), (300, 1000), (5000, 4)])
def test_window(Hq, Hkv, window, sinks):
    both([150, 1, 33, 0], [700, 900, 0, 10], Hq, Hkv, 16, window, sinks, pad=1)


@pytest.mark.parametrize("window,sinks", [(0, 0), (600, 40)])
@pytest.mark.parametrize("new,ctx", [([700], [0]), ([600, 5, 530], [100, 4000, 0]), ([16], [9000]), ([1, 2, 1], [5000, 6000, 7]),
                                     ([70], [3000])])
def test_longer(new, ctx, window, sinks):
    both(new, ctx, 8, 2, 32, window, sinks, seed=3)


@pytest.mark.parametrize("P", [48, 80, 144, 384])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 20)])
def test_pages_that_end_inside_a_tile(P, window, sinks):
    both([90, 200], [170, 31], 8, 2, P, window, sinks, seed=14)


@pytest.mark.parametrize("Hq,Hkv", [(7, 1), (12, 2), (16, 2), (9, 3)])
def test_groups(Hq, Hkv):
    both([140, 37], [100, 0], Hq, Hkv, 32, 70, 9, seed=15)
    both([140, 37], [100, 0], Hq, Hkv, 32, seed=15)


@pytest.mark.parametrize("scale", [-0.07, 0.0, 1e-30, 0.5])
def test_scales(scale):
    """Of either sign and none: with 0 every row is the mean of the values it sees."""
    q, k, v, table, given, starts, lens = make(16, [150, 3], [20, 300], 8, 2, 16)
    call = Call(q, k, v, given, starts, lens, 8)
    call(scale=scale)
    check(call.result(), q, k, v, table, starts, lens, 8, scale=scale)


def test_a_long_prompt_of_few_heads():
    """More key tiles than blocks a head: every item cut, some into many parts."""
    both([2500], [300], 2, 1, 64, seed=17)


def test_beyond_32_bits():
    """The sequence's pages lie behind 4 GiB of the pool, in bytes and in elements."""
    Hq, Hkv, P, pages = 4, 2, 64, 140_000
    k = torch.zeros((pages, Hkv, P, D), dtype=torch.int16, device="cuda")       # 4.6 GB each, 2.3e9 elements
    v = torch.zeros_like(k)
    q, ks, vs, table, _, starts, lens = make(18, [40], [60], Hq, Hkv, P, hide=False)
    n = ks.shape[0]
    k[pages - n:], v[pages - n:] = dev(ks), dev(vs)
    small = Call(q, ks, vs, table, starts, lens, Hq)
    small()
    big = Call(q, ks, vs, table + (pages - n), starts, lens, Hq)
    big.cache = wq4.kv_cache_desc(k, v, big.table, P)
    big()
    assert np.array_equal(small.result(), big.result())
    ws = torch.zeros(wq4.wq4_paged_attention_workspace_bytes(1, Hq, Hkv, D), dtype=torch.uint8, device="cuda")
    for c in (small, big):
        wq4.wq4_window_attention(c.cache, c.q, Hq * D, c.lens, c.out, Hq * D, 1, Hq, SCALE, 50, 3, ws, ws.numel())
    assert np.array_equal(small.result()[:1], big.result()[:1])
    x = dev(synth.sum4_fp16(18, 5, 0, 40 * (Hq + 2 * Hkv) * D).reshape(40, -1))
    for c in (small, big):
        wq4.wq4_prompt_append(c.cache, x, (Hq + 2 * Hkv) * D, c.q, Hq * D, c.starts, c.lens, 1, 40, Hq, THETA)
    torch.cuda.synchronize()
    assert torch.equal(k[pages - n:], small.k) and torch.equal(v[pages - n:], small.v) and not k[:1000].any()
    ints = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")   # noqa: E731
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    pool_ws = torch.empty(wq4.wq4_kv_pool_workspace_bytes(pages, 1), dtype=torch.uint8, device="cuda")
    pool = wq4.kv_pool_desc([big.cache], big.table, big.lens, refs, pool_ws)
    wq4.wq4_kv_copy_pages(pool, ints([pages - n]), ints([pages - n - 3]), 1)
    torch.cuda.synchronize()
    assert torch.equal(k[pages - n - 3], k[pages - n]) and torch.equal(v[pages - n - 3], v[pages - n])
    assert wq4.wq4_device_status() == 0


def test_without_its_copies_it_ends():
    """Waits for copies that never come run out: the kernel ends, flags it, and the next call is clean."""
    for new, ctx in (([300, 20], [500, 0]), ([10], [3000])):
        q, k, v, table, given, starts, lens = make(19, new, ctx, 8, 2, 16)
        call = Call(q, k, v, given, starts, lens, 8)
        call()
        want = call.result()
        assert wq4.wq4_device_status() == 0
        try:
            wq4.wq4_test_copy_stall(3)
            call()
            torch.cuda.synchronize()
        finally:
            wq4.wq4_test_copy_stall()
        assert wq4.wq4_device_status() & 1
        call.out.fill_(-1)
        call()
        assert np.array_equal(call.result(), want) and wq4.wq4_device_status() == 0


def test_many_sequences():
    rng = np.random.default_rng(0)
    new = rng.integers(0, 5, 1024)
    new[5] = 1
    both(new, rng.integers(0, 40, 1024), 4, 1, 16, seed=4)


def test_strides_and_untouched_columns():
    q, k, v, table, given, starts, lens = make(5, [50, 20], [3, 90], 8, 2, 16, pad=2)
    wide = np.concatenate([q, np.full((q.shape[0], 4 * D), NAN16)], 1)
    call = Call(wide, k, v, given, starts, lens, 8, out_stride=8 * D + 8)
    call()
    got = call.result()
    assert np.all(got[:, 8 * D:] == 0xFFFF)
    check(got, q, k, v, table, starts, lens, 8)


def test_what_a_row_does_not_see_does_not_reach_it():
    """NaN and infinities among the keys and values of tokens that later rows of the same tile see,
    and of tokens that earlier rows still saw: every other row as if they were not there."""
    for window, sinks, tokens in ((0, 0, (150, 260)), (40, 2, (150,)), (64, 0, (30, 200))):
        q, k, v, table, given, starts, lens = make(6, [300], [20], 8, 2, 16, window, sinks)
        for t in tokens:
            k[table[0, t // 16], 0, t % 16, 5] = NAN16
            v[table[0, t // 16], 1, t % 16, 7] = 0x7C00          # infinity
            v[table[0, t // 16], 1, t % 16, 100] = NAN16
        call = Call(q, k, v, given, starts, lens, 8)
        call(window, sinks)
        o, A, _ = oc.attention(q, k, v, table, starts, lens, SCALE, 8, window, sinks)
        g = oracle.half_to_double(call.result()).reshape(o.shape)
        fine = np.isfinite(o)
        assert fine.any() and not fine.all()
        assert np.array_equal(np.isnan(g), np.isnan(o)) and np.array_equal(g[~fine & ~np.isnan(o)], o[~fine & ~np.isnan(o)])
        assert np.all(np.abs(g[fine] - o[fine]) <= oc.attention_tolerance(o, A)[fine])


def test_lowest_and_infinite_scores():
    """Scores of the lowest finite size, and keys whose scores are -infinity: weight 0 beside any other."""
    q, k, v, table, given, starts, lens = make(7, [40], [0], 2, 1, 16)
    q[:, :], k[:, :] = 0x3C00, 0x3C00                             # all ones: every score is the same
    k[table[0, 0], 0, 3] = 0xFBFF                                 # -65504 in every dimension
    k[table[0, 1], 0, 2, 9] = 0xFC00                              # a -infinity
    call = Call(q, k, v, given, starts, lens, 2)
    call(scale=1.0)
    check(call.result(), q, k, v, table, starts, lens, 2, scale=1.0)


@pytest.mark.parametrize("first", [-30.0, 30.0])
def test_a_running_maximum_that_jumps(first):
    """Scores that rise or fall by far more than fp16's range between one key tile and another."""
    q, k, v, table, given, starts, lens = make(8, [200], [500], 4, 1, 16)
    step = np.linspace(first, -first, 700)
    q[:] = 0
    q[:, ::D] = 0x3C00                                            # 1 in the first dimension
    for t in range(700):
        k[table[0, t // 16], :, t % 16, 0] = np.float16(step[t]).view(np.uint16)
    call = Call(q, k, v, given, starts, lens, 4)
    call(scale=1.0)
    check(call.result(), q, k, v, table, starts, lens, 4, scale=1.0)


def test_rows_before_the_first_token_get_zeros():
    q, k, v, table, given, starts, lens = make(9, [40], [0], 8, 2, 16)
    lens = np.array([25], np.int32)                               # 15 rows more than tokens
    call = Call(q, k, v, given, starts, lens, 8)
    call()
    got = call.result()
    assert np.all(got[:15] == 0)
    check(got, q, k, v, table, starts, lens, 8)


def test_bad_pages_and_lengths_are_flagged():
    q, k, v, table, _, starts, lens = make(10, [40], [60], 8, 2, 16, hide=False)
    bad = table.copy()
    bad[0, 2] = k.shape[0]
    Call(q, k, v, bad, starts, lens, 8)()
    assert wq4.wq4_device_status() == 16
    bad[0, 2] = -2 ** 31
    Call(q, k, v, bad, starts, lens, 8)()
    assert wq4.wq4_device_status() == 16
    Call(q, k, v, table, starts, lens + 50, 8)()
    assert wq4.wq4_device_status() == 8


@pytest.mark.parametrize("starts", [[0, 500, 40], [30, 10, 40], [-5, 20, 10 ** 9], [2 ** 31 - 1, 0, 0]])
def test_row_starts_of_any_contents_stay_within_the_buffers(starts):
    q, k, v, table, _, _, lens = make(11, [20, 20], [16, 16], 8, 2, 16, hide=False)
    call = Call(q, k, v, table, starts, lens, 8)
    guard = call.out.clone()
    call()
    assert call.result().shape == guard.shape
    wq4.wq4_device_status()


def test_row_starts_that_give_more_tiles_than_an_int_counts():
    batch, rows, Hkv, cap = 1024, 65536, 8, 1 << 20
    k = torch.zeros((1, Hkv, 16, D), dtype=torch.int16, device="cuda")
    table = torch.zeros((batch, cap // 16), dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, rows] * (batch // 2) + [0], dtype=torch.int32, device="cuda")     # every other one owns all rows
    lens = torch.full((batch,), cap, dtype=torch.int32, device="cuda")
    q = torch.zeros((rows, Hkv * D), dtype=torch.int16, device="cuda")
    out = torch.full_like(q, -1)
    ws = torch.zeros(wq4.wq4_prompt_attention_workspace_bytes(batch, rows, Hkv, Hkv, D), dtype=torch.uint8, device="cuda")
    wq4.wq4_prompt_attention(wq4.kv_cache_desc(k, k.clone(), table, 16), q, Hkv * D, starts, lens, out, Hkv * D, batch, rows, Hkv, SCALE,
                             0, 0, ws, ws.numel())
    torch.cuda.synchronize()
    assert torch.all(out == -1)
    assert wq4.wq4_device_status() == 8


def test_same_bits_again_captured_and_on_other_streams():
    q, k, v, table, given, starts, lens = make(12, [130, 9], [500, 2000], 8, 2, 16)
    a, b = Call(q, k, v, given, starts, lens, 8), Call(q, k, v, given, starts, lens, 8)
    a()
    want = a.result()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):                                            # two calls at once, a workspace each
        a(stream=s)
        b(stream=t)
    assert np.array_equal(a.result(), want) and np.array_equal(b.result(), want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        a(stream=s)
        b(stream=s)
    for _ in range(3):
        a.out.fill_(-1)
        b.out.fill_(-1)
        g.replay()
        assert np.array_equal(a.result(), want) and np.array_equal(b.result(), want)
    assert wq4.wq4_device_status() == 0


def test_a_captured_call_follows_its_arrays():
    """Lengths, row starts and the table are read on the device: a graph's replay takes their new contents."""
    q, k, v, table, _, starts, lens = make(20, [60, 200], [900, 30], 8, 2, 16, hide=False)
    call = Call(q, k, v, table, starts, lens, 8)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        call(100, 20, stream=s)
    for new, T in (([60, 200], [960, 230]), ([1, 0], [17, 3]), ([130, 130], [130, 200]), ([0, 0], [5, 6]), ([0, 260], [1, 230])):
        starts, lens = starts_of(new), np.asarray(T, np.int32)
        flipped = table.copy()
        flipped[:, :1] = table[::-1, :1]                          # another page in front
        call.table.copy_(dev(flipped, np.int32))
        call.starts.copy_(dev(np.asarray(starts, np.int32), np.int32))
        call.lens.copy_(dev(lens, np.int32))
        call.out.fill_(-1)
        g.replay()
        check(call.result(), q, k, v, flipped, starts, lens, 8, 100, 20)
    assert wq4.wq4_device_status() == 0


def test_a_row_of_nothing_but_minus_infinity_gets_zeros():
    q, k, v, table, given, starts, lens = make(21, [20], [0], 2, 1, 16)
    q[:] = 0x3C00                                                 # ones
    k[table[0, 0], 0, :4, 0] = 0xFC00                             # the first four tokens score -infinity
    call = Call(q, k, v, given, starts, lens, 2)
    call()
    got = call.result()
    assert np.all(got[:4] == 0)
    o, A, _ = oc.attention(q[4:], k, v, table, [0, 16], [20], SCALE, 2)
    g = oracle.half_to_double(np.ascontiguousarray(got[4:])).reshape(o.shape)
    assert np.all(np.abs(g - o) <= oc.attention_tolerance(o, A))


# ------------------------------------------------------------------ append --

def run_append(qkv, k, v, table, starts, lens, Hq, Hkv, theta, in_place=False, want_q=True):
    rows, w = qkv.shape
    x, kd, vd = dev(qkv), dev(k), dev(v)
    td, ld, sd = dev(table, np.int32), dev(np.asarray(lens, np.int32), np.int32), dev(np.asarray(starts, np.int32), np.int32)
    out = x if in_place else torch.full((rows, Hq * D + 8), -1, dtype=torch.int16, device="cuda")
    wq4.wq4_prompt_append(wq4.kv_cache_desc(kd, vd, td, k.shape[2]), x, w, out if want_q else None, out.shape[1], sd, ld,
                          len(lens), rows, Hq, theta)
    torch.cuda.synchronize()
    return tuple(t.cpu().numpy().view(np.uint16) for t in (out, kd, vd))


def check_append(got, qkv, k, v, table, starts, lens, Hq, Hkv, theta):
    q_ref, k_ref, v_ref = oc.append(qkv, k, v, table, starts, lens, Hq, theta)
    q16, k16, v16 = got
    owned = slice(starts[0], starts[-1])
    x = oracle.half_to_double(qkv)
    pair = np.abs(x).reshape(x.shape[0], -1, 2).max(2).repeat(2, 1)
    for g, ref, big in ((q16[owned, :Hq * D], q_ref[owned], pair[owned, :Hq * D]), (k16, k_ref, np.abs(x).max())):
        err = np.abs(oracle.half_to_double(np.ascontiguousarray(g)) - ref)
        assert np.all(err <= oc.ulp16(ref) / 2 + 2.0 ** -22 * big)
    assert np.array_equal(oracle.half_to_double(v16), v_ref)


@pytest.mark.parametrize("Hq,Hkv,P,new,ctx", [(32, 8, 16, [1], [0]), (6, 2, 32, [9, 0, 100, 1], [5, 3, 60, 31]),
                                              (8, 1, 64, [40], [130000]), (14, 2, 16, [17, 23], [0, 1000]), (3, 3, 16, [8, 8, 8], [1, 2, 3])])
@pytest.mark.parametrize("theta", [THETA, 10000.0, 0.0])
def test_append(Hq, Hkv, P, new, ctx, theta):
    lens = np.asarray(new) + np.asarray(ctx)
    pages = int(((np.asarray(lens) + P - 1) // P).sum()) + 1
    k, v = synth.kv_cache(2, pages, Hkv, P, D)
    table = synth.page_table(2, lens, P, pages)
    starts = starts_of(new)
    qkv = synth.sum4_fp16(2, 77, 0, (starts[-1] + 2) * (Hq + 2 * Hkv) * D).reshape(starts[-1] + 2, -1)
    got = run_append(qkv, k, v, table, starts, lens, Hq, Hkv, theta)
    check_append(got, qkv, k, v, table, starts, lens, Hq, Hkv, theta)
    assert np.all(got[0][starts[-1]:] == 0xFFFF) and np.all(got[0][:, Hq * D:] == 0xFFFF)
    place = run_append(qkv, k, v, table, starts, lens, Hq, Hkv, theta, in_place=True)
    assert np.array_equal(place[0][:starts[-1], :Hq * D], got[0][:starts[-1], :Hq * D])
    assert np.array_equal(place[0][:, Hq * D:], qkv[:, Hq * D:]) and np.array_equal(place[1], got[1]) and np.array_equal(place[2], got[2])
    assert wq4.wq4_device_status() == 0


@pytest.mark.parametrize("Hq,Hkv,new", [(5, 1, [1501, 0, 602]), (16, 2, [2001]), (3, 3, [7] * 300)])
def test_append_of_many_rows(Hq, Hkv, new):
    P, lens = 16, np.asarray(new) + 5
    pages = int(((lens + P - 1) // P).sum()) + 1
    k, v = synth.kv_cache(4, pages, Hkv, P, D)
    table = synth.page_table(4, lens, P, pages)
    starts = starts_of(new)
    qkv = synth.sum4_fp16(4, 78, 0, (starts[-1] + 3) * (Hq + 2 * Hkv) * D).reshape(starts[-1] + 3, -1)
    for theta in (THETA, 0.0):
        got = run_append(qkv, k, v, table, starts, lens, Hq, Hkv, theta)
        check_append(got, qkv, k, v, table, starts, lens, Hq, Hkv, theta)
        assert np.all(got[0][starts[-1]:] == 0xFFFF) and np.all(got[0][:, Hq * D:] == 0xFFFF)
        place = run_append(qkv, k, v, table, starts, lens, Hq, Hkv, theta, in_place=True)
        assert np.array_equal(place[0][:starts[-1], :Hq * D], got[0][:starts[-1], :Hq * D])
        assert np.array_equal(place[0][:, Hq * D:], qkv[:, Hq * D:]) and np.array_equal(place[1], got[1]) and np.array_equal(place[2], got[2])
    assert wq4.wq4_device_status() == 0
    bad = table.copy()
    bad[0, -1 if len(new) < 4 else 0] = pages                                # a page outside the pool
    run_append(qkv, k, v, bad, starts, lens, Hq, Hkv, THETA)
    assert wq4.wq4_device_status() == 32


def test_append_without_a_place_is_flagged():
    k, v = synth.kv_cache(3, 3, 2, 16, D)
    table = np.array([[0, -1], [5, 1]], np.int32)
    qkv = synth.sum4_fp16(3, 77, 0, 44 * 8 * D).reshape(44, -1)
    lens = [20, 40]                                               # a missing page; beyond the table and outside the pool
    got = run_append(qkv, k, v, table, [0, 20, 44], lens, 4, 2, THETA)
    assert wq4.wq4_device_status() == 32
    check_append(got, qkv, k, v, table, [0, 20, 44], lens, 4, 2, THETA)


def test_append_of_values_alone():
    """No rotation, no query output: the cache alone is written."""
    k, v = synth.kv_cache(4, 4, 2, 16, D)
    table = np.array([[2, 0, 1]], np.int32)
    qkv = synth.sum4_fp16(4, 77, 0, 33 * 8 * D).reshape(33, -1)
    got = run_append(qkv, k, v, table, [0, 33], [40], 4, 2, 0.0, want_q=False)
    assert np.all(got[0] == 0xFFFF)
    check_append((np.ascontiguousarray(qkv[:, :4 * D]), got[1], got[2]), qkv, k, v, table, [0, 33], [40], 4, 2, 0.0)
