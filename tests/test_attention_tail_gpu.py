"""Attention where one token of zero values holds nearly all the weight, as a sink does: what is left of
the output is the tail's, whose weights are many powers of two below the largest.

A weight is kept in fp16 in units in which the largest is at least 2^lift: from 2^-(14 + lift) of the
largest up it is within 2^-11 of itself, below that within 2^-(25 + lift) of the largest.  So the bar is
2e-3 * sum_t p_t |V_t| + 2^-(25 + lift) * sum_t |V_t| + ulp16(|o|), the second sum over what is seen; for
weights that are not below 2^-(14 + lift) it is met without the second term.
"""
import numpy as np
import pytest
import torch

import oracle
from oracle import cache as oc
from paper_2412_15803_gb300 import synth, wq4

pytestmark = pytest.mark.gpu

D, HQ, HKV, P = 128, 8, 2, 16
DECODE_LIFT = 15


def dev(a, dtype=np.int16):
    return torch.from_numpy(np.ascontiguousarray(a).view(dtype)).cuda()


def make(seed, T, nats, spread, heavy, rows):
    """One sequence of T tokens: scores of 0 at token `heavy`, whose values are 0, and of -nats (plus a normal
    deviation) elsewhere, where values are positive and of the order of 100."""
    rng = np.random.default_rng(seed)
    pages = (T + P - 1) // P
    k, v = (np.zeros((pages, HKV, P, D), np.float16) for _ in range(2))
    s = -nats + spread * np.clip(rng.standard_normal((pages * P, HKV)), -3, 3)
    s[heavy] = 0
    k[..., 0] = s.reshape(pages, P, HKV).transpose(0, 2, 1)
    v[:] = np.abs(100 * rng.standard_normal(v.shape))
    v[heavy // P, :, heavy % P] = 0
    q = np.zeros((rows, HQ, D), np.float16)
    q[:, :, 0] = 1
    table = synth.page_table(seed, np.array([T], np.int32), P, pages)
    kk, vv = np.empty_like(k), np.empty_like(v)
    kk[table[0]], vv[table[0]] = k, v                        # the sequence's pages at random places of the pool
    return q.reshape(rows, -1).view(np.uint16), kk.view(np.uint16), vv.view(np.uint16), table


def check(got, q, k, v, table, T, rows, window, sinks, second):
    o, A, _ = oc.attention(q, k, v, table, [0, rows], [T], 1.0, HQ, window, sinks)
    assert np.abs(o).min() > 0
    V = np.abs(oracle.half_to_double(v[table[0]])).transpose(1, 0, 2, 3).reshape(HKV, -1, D)[:, :T]
    total = np.stack([V[:, oc.seen(T - rows + r, T, window, sinks)].sum(1) for r in range(rows)])
    err = np.abs(oracle.half_to_double(got).reshape(o.shape) - o)
    bar = oc.attention_tolerance(o, A) + second * total.repeat(HQ // HKV, 1)
    assert np.all(err <= bar), f"{(err / bar).max()} of the bar"


TAILS = [(12.3, 0.0), (16.0, 0.0), (16.0, 1.0), (18.0, 1.0), (20.0, 0.0), (25.0, 1.0), (30.0, 0.0)]


@pytest.mark.parametrize("nats,spread", TAILS)
@pytest.mark.parametrize("T,heavy,window,sinks", [(4000, 0, 0, 0), (4000, 0, 3000, 1), (4000, 3999, 0, 0), (300, 150, 200, 4),
                                                  (30000, 2, 20000, 4)])
def test_one_token(nats, spread, T, heavy, window, sinks):
    q, k, v, table = make(T + window, T, nats, spread, heavy, 1)
    kd, vd, td, qd, ld = dev(k), dev(v), dev(table, np.int32), dev(q), dev(np.array([T], np.int32), np.int32)
    out = torch.full((1, HQ * D), -1, dtype=torch.int16, device="cuda")
    ws = torch.zeros(wq4.wq4_paged_attention_workspace_bytes(1, HQ, HKV, D), dtype=torch.uint8, device="cuda")
    cache = wq4.kv_cache_desc(kd, vd, td, P)
    if window:
        wq4.wq4_window_attention(cache, qd, HQ * D, ld, out, HQ * D, 1, HQ, 1.0, window, sinks, ws, ws.numel())
    else:
        wq4.wq4_paged_attention(cache, qd, HQ * D, ld, out, HQ * D, 1, HQ, 1.0, ws, ws.numel())
    torch.cuda.synchronize()
    assert wq4.wq4_device_status() == 0
    deepest = (nats + 3 * spread) / np.log(2)
    check(out.cpu().numpy().view(np.uint16), q, k, v, table, T, 1, window, sinks,
          0.0 if deepest <= 14 + DECODE_LIFT else 2.0 ** -(25 + DECODE_LIFT))


PROMPT_LIFT = 6


@pytest.mark.parametrize("nats,spread", TAILS)
@pytest.mark.parametrize("T,heavy,window,sinks", [(4000, 0, 0, 0), (4000, 0, 3000, 1), (4000, 2000, 0, 0), (500, 300, 400, 4),
                                                  (9000, 2, 5000, 4)])
def test_a_prompt(nats, spread, T, heavy, window, sinks):
    rows = 20
    q, k, v, table = make(T + window, T, nats, spread, heavy, rows)
    kd, vd, td, qd, ld = dev(k), dev(v), dev(table, np.int32), dev(q), dev(np.array([T], np.int32), np.int32)
    out = torch.full((rows, HQ * D), -1, dtype=torch.int16, device="cuda")
    ws = torch.zeros(wq4.wq4_prompt_attention_workspace_bytes(1, rows, HQ, HKV, D), dtype=torch.uint8, device="cuda")
    starts = dev(np.array([0, rows], np.int32), np.int32)
    wq4.wq4_prompt_attention(wq4.kv_cache_desc(kd, vd, td, P), qd, HQ * D, starts, ld, out, HQ * D, 1, rows, HQ, 1.0, window, sinks,
                             ws, ws.numel())
    torch.cuda.synchronize()
    assert wq4.wq4_device_status() == 0
    deepest = (nats + 3 * spread) / np.log(2)
    check(out.cpu().numpy().view(np.uint16), q, k, v, table, T, rows, window, sinks,
          0.0 if deepest <= 14 + PROMPT_LIFT else 2.0 ** -(25 + PROMPT_LIFT))
