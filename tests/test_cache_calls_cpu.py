"""Refusals of the cache calls and their launches on every device, without a GPU.

Addresses are made up and never read: an argument error returns before anything is enqueued.
"""
import ctypes
import os
import subprocess
import sys

import pytest

from paper_2412_15803_gb300 import wq4

HERE = os.path.dirname(os.path.abspath(__file__))
A = 1 << 40
INVALID, ALIGN, UNSUPPORTED = wq4.WQ4_ERR_INVALID, wq4.WQ4_ERR_ALIGN, wq4.WQ4_ERR_UNSUPPORTED
NAN, INF = float("nan"), float("inf")


def cache(**kw):
    d = dict(k=A, v=2 * A, num_pages=64, n_kv_heads=8, page_size=16, head_dim=128, page_table=3 * A, page_table_stride=32)
    d.update(kw)
    return wq4.wq4_kv_cache(**d)


CACHE = [
    (dict(k=None), INVALID), (dict(v=0), INVALID), (dict(page_table=0), INVALID), (dict(num_pages=0), INVALID),
    (dict(n_kv_heads=0), INVALID), (dict(page_size=8), INVALID), (dict(page_size=24), INVALID),
    (dict(page_table_stride=0), INVALID), (dict(head_dim=64), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED),
    (dict(k=A + 8), ALIGN), (dict(v=2 * A + 2), ALIGN), (dict(page_table=3 * A + 2), ALIGN),
    (dict(num_pages=1 << 24), UNSUPPORTED), (dict(page_table_stride=1 << 26), UNSUPPORTED)]


def _both(defaults, changes):
    c = dict(changes.pop("cache", {}))
    return cache(**c), {**defaults, **changes}


@pytest.mark.parametrize("changes,want", [
    (dict(window=-1), INVALID), (dict(sinks=-1), INVALID), (dict(q=None), INVALID), (dict(out=0), INVALID), (dict(batch=0), INVALID),
    (dict(batch=1025), INVALID), (dict(heads=12), INVALID), (dict(heads=128), UNSUPPORTED), (dict(scale=NAN), INVALID),
    (dict(scale=INF), INVALID), (dict(q_stride=4095), INVALID), (dict(q=4 * A + 4), ALIGN)]
    + [(dict(cache=c), w) for c, w in CACHE[:13]])
def test_window_attention_refuses(changes, want):
    c, a = _both(dict(q=4 * A, q_stride=4096, lens=5 * A, out=6 * A, batch=4, heads=32, scale=0.1, window=100, sinks=4), dict(changes))
    rc = wq4.load().wq4_window_attention(ctypes.byref(c), a["q"], a["q_stride"], a["lens"], a["out"], 4096, a["batch"], a["heads"],
                                         a["scale"], a["window"], a["sinks"], 7 * A, 1 << 30, None)
    assert rc == want


@pytest.mark.parametrize("changes,want", [
    (dict(window=-1), INVALID), (dict(sinks=-5), INVALID), (dict(q=None), INVALID), (dict(out=0), INVALID), (dict(ws=None), INVALID),
    (dict(starts=0), INVALID), (dict(lens=None), INVALID), (dict(batch=0), INVALID), (dict(batch=1025), INVALID),
    (dict(rows=0), INVALID), (dict(rows=-3), INVALID), (dict(heads=12), INVALID), (dict(heads=4), INVALID),
    (dict(heads=72), UNSUPPORTED), (dict(scale=NAN), INVALID), (dict(scale=-INF), INVALID), (dict(q_stride=4088), INVALID),
    (dict(out_stride=4095), INVALID), (dict(q=4 * A + 8), ALIGN), (dict(q_stride=4100), ALIGN), (dict(out=6 * A + 8), ALIGN),
    (dict(out_stride=4100), ALIGN), (dict(ws=7 * A + 128), ALIGN), (dict(starts=8 * A + 2), ALIGN), (dict(lens=5 * A + 1), ALIGN)]
    + [(dict(cache=c), w) for c, w in CACHE])
def test_prompt_attention_refuses(changes, want):
    c, a = _both(dict(q=4 * A, q_stride=4096, starts=8 * A, lens=5 * A, out=6 * A, out_stride=4096, batch=4, rows=100, heads=32,
                      scale=0.1, window=0, sinks=0, ws=7 * A), dict(changes))
    rc = wq4.load().wq4_prompt_attention(ctypes.byref(c), a["q"], a["q_stride"], a["starts"], a["lens"], a["out"], a["out_stride"],
                                         a["batch"], a["rows"], a["heads"], a["scale"], a["window"], a["sinks"], a["ws"], 1 << 40, None)
    assert rc == want


@pytest.mark.parametrize("changes,want", [
    (dict(qkv=None), INVALID), (dict(q_out=None), INVALID), (dict(starts=0), INVALID), (dict(batch=0), INVALID), (dict(rows=0), INVALID),
    (dict(heads=12), INVALID), (dict(theta=1.0), INVALID), (dict(theta=-2.0), INVALID), (dict(theta=INF), INVALID),
    (dict(theta=NAN), INVALID), (dict(stride=6136), INVALID), (dict(stride=6148), ALIGN), (dict(q_stride=4088), INVALID),
    (dict(q_stride=4100), ALIGN), (dict(qkv=4 * A + 8), ALIGN), (dict(q_out=6 * A + 4), ALIGN), (dict(q_out=4 * A + 16), INVALID),
    (dict(q_out=4 * A), INVALID), (dict(q_out=A + 4096), INVALID), (dict(qkv=2 * A), INVALID), (dict(cache=dict(v=A + 4096)), INVALID)]
    + [(dict(cache=c), w) for c, w in CACHE])
def test_prompt_append_refuses(changes, want):
    c, a = _both(dict(qkv=4 * A, stride=6144, q_out=6 * A, q_stride=4096, starts=8 * A, lens=5 * A, batch=4, rows=100, heads=32,
                      theta=10000.0), dict(changes))
    rc = wq4.load().wq4_prompt_append(ctypes.byref(c), a["qkv"], a["stride"], a["q_out"], a["q_stride"], a["starts"], a["lens"],
                                      a["batch"], a["rows"], a["heads"], a["theta"], None)
    assert rc == want


def pool(layers=2, caches=None, **kw):
    arr = (wq4.wq4_kv_cache * layers)(*(caches or [cache(k=(4 * l + 1) * A, v=(4 * l + 2) * A) for l in range(layers)]))
    d = dict(layers=arr, num_layers=layers, max_seqs=10, page_table=3 * A, seq_lens=20 * A, page_refs=21 * A, workspace=22 * A,
             workspace_bytes=1 << 30)
    d.update(kw)
    p = wq4.wq4_kv_pool(**d)
    p._keep = arr
    return p


POOLS = [
    (dict(num_layers=0), INVALID), (dict(num_layers=129), UNSUPPORTED), (dict(max_seqs=0), INVALID), (dict(max_seqs=1025), UNSUPPORTED),
    (dict(page_table=None), INVALID), (dict(page_table=9 * A), INVALID), (dict(seq_lens=0), INVALID), (dict(page_refs=None), INVALID),
    (dict(workspace=0), INVALID), (dict(workspace_bytes=1000), INVALID), (dict(workspace=22 * A + 8), ALIGN),
    (dict(seq_lens=20 * A + 2), ALIGN), (dict(caches=[cache(), cache(page_size=32)]), INVALID),
    (dict(caches=[cache(), cache(num_pages=65)]), INVALID), (dict(caches=[cache(), cache(k=A + 4)]), ALIGN),
    (dict(layers=1, caches=[cache(head_dim=64)]), UNSUPPORTED), (dict(layers=1, caches=[cache(page_size=20)]), INVALID)]


@pytest.mark.parametrize("changes,want", POOLS)
def test_pool_calls_refuse_a_bad_pool(changes, want):
    L, p = wq4.load(), pool(**dict(changes))
    r = ctypes.byref(p)
    assert [L.wq4_kv_reserve(r, A, A, 1, None), L.wq4_kv_fork(r, A, A, 1, None), L.wq4_kv_free(r, A, 1, None),
            L.wq4_kv_trim(r, A, 1, 5, 0, None), L.wq4_kv_compact(r, None), L.wq4_kv_copy_pages(r, A, A, 1, None)] == [want] * 6


def test_sizes_that_an_int_does_not_count_are_refused():
    L = wq4.load()
    for caches, seqs in (([cache(num_pages=1, n_kv_heads=1 << 10, page_size=1 << 16)], 10), ([cache(page_table_stride=1 << 25)], 64)):
        p = pool(layers=1, caches=caches, max_seqs=seqs)
        r = ctypes.byref(p)
        assert [L.wq4_kv_reserve(r, A, A, 1, None), L.wq4_kv_fork(r, A, A, 1, None), L.wq4_kv_free(r, A, 1, None),
                L.wq4_kv_trim(r, A, 1, 5, 0, None), L.wq4_kv_compact(r, None), L.wq4_kv_copy_pages(r, A, A, 1, None)] == [UNSUPPORTED] * 6
    long = cache(num_pages=1 << 16, page_table_stride=1 << 16)              # room for 2^20 tokens
    assert L.wq4_prompt_attention(ctypes.byref(long), 4 * A, 4096, 8 * A, 5 * A, 6 * A, 4096, 1, 1 << 20, 32, 0.1, 0, 0, 7 * A,
                                  1 << 40, None) == UNSUPPORTED
    assert L.wq4_prompt_attention(ctypes.byref(long), 4 * A, 4096, 8 * A, 5 * A, 6 * A, 4096, 1, 1 << 20, 32, 0.1, 4096, 16, 7 * A,
                                  1 << 40, None) != UNSUPPORTED         # a window's tiles are few
    many, wide = cache(num_pages=1, n_kv_heads=1 << 25), 1 << 30
    for heads in (1 << 25, 1 << 27):
        assert L.wq4_prompt_append(ctypes.byref(many), 4 * A, wide, 6 * A, wide, 8 * A, 5 * A, 1, 1, heads, 1e4, None) == UNSUPPORTED
        assert L.wq4_prompt_attention(ctypes.byref(many), 4 * A, wide, 8 * A, 5 * A, 6 * A, wide, 1, 1, heads, 0.1, 0, 0, 7 * A,
                                      1 << 40, None) == UNSUPPORTED


def test_pool_calls_refuse_bad_lists():
    L, p = wq4.load(), pool()
    r = ctypes.byref(p)
    assert L.wq4_kv_reserve(None, A, A, 1, None) == INVALID
    for lst, n, want in ((None, 1, INVALID), (A, -1, INVALID), (A, 1025, INVALID), (A + 2, 1, ALIGN)):
        assert L.wq4_kv_free(r, lst, n, None) == want
        assert L.wq4_kv_trim(r, lst, n, 5, 0, None) == want
        assert L.wq4_kv_reserve(r, lst, A, n, None) == want
        assert L.wq4_kv_fork(r, A, lst, n, None) == want
        assert L.wq4_kv_copy_pages(r, lst, A, n, None) == want
    assert L.wq4_kv_copy_pages(r, A, A, 65, None) == INVALID                # more pairs than pages
    assert L.wq4_kv_trim(r, A, 1, 0, 0, None) == INVALID and L.wq4_kv_trim(r, A, 1, 3, -1, None) == INVALID


def test_workspace_sizes():
    assert wq4.wq4_kv_pool_workspace_bytes(0, 4) == 0 and wq4.wq4_kv_pool_workspace_bytes(10, 1025) == 0
    assert wq4.wq4_kv_pool_workspace_bytes(10, 4) >= 4 * 4 * 1024
    for bad in ((0, 1, 8, 8, 128), (1, 0, 8, 8, 128), (1, 1, 8, 3, 128), (1, 1, 72, 8, 128), (1, 1, 8, 8, 64)):
        assert wq4.wq4_prompt_attention_workspace_bytes(*bad) == 0


CHILD = r"""
import ctypes, sys
fake = ctypes.CDLL(sys.argv[1])
sys.path.insert(0, sys.argv[2])
from test_cache_calls_cpu import A, cache, pool
from paper_2412_15803_gb300 import wq4
L = wq4.load(build_if_missing=False)
for device in (0, 1, 0, 3):
    fake.fake_set_device(device)
    def counted(want, rc):
        global before
        assert rc == 0, f"device {device}: {rc}"
        assert fake.fake_launches() == before + want, (fake.fake_launches(), before, want)
        before = fake.fake_launches()
    before = fake.fake_launches()
    c, p = cache(num_pages=4096, page_table_stride=256), pool()
    r = ctypes.byref(p)
    n = L.wq4_paged_attention_workspace_bytes(3, 32, 8, 128)
    counted(1, L.wq4_window_attention(ctypes.byref(c), 4 * A, 4096, 5 * A, 6 * A, 4096, 3, 32, 0.1, 100, 4, 7 * A, n, None))
    for batch, rows in ((1, 1), (3, 900), (1024, 5000)):
        n = L.wq4_prompt_attention_workspace_bytes(batch, rows, 32, 8, 128)
        assert n > 0
        counted(2, L.wq4_prompt_attention(ctypes.byref(c), 4 * A, 4096, 8 * A, 5 * A, 6 * A, 4096, batch, rows, 32, 0.1, 100, 4,
                                          7 * A, n, None))
        assert L.wq4_prompt_attention(ctypes.byref(c), 4 * A, 4096, 8 * A, 5 * A, 6 * A, 4096, batch, rows, 32, 0.1, 100, 4,
                                      7 * A, n - 1, None) == wq4.WQ4_ERR_INVALID
        counted(1, L.wq4_prompt_append(ctypes.byref(c), 4 * A, 6144, 6 * A, 4096, 8 * A, 5 * A, batch, rows, 32, 10000.0, None))
        counted(1, L.wq4_prompt_append(ctypes.byref(c), 4 * A, 6144, 4 * A, 6144, 8 * A, 5 * A, batch, rows, 32, 10000.0, None))
    short = cache(page_table_stride=20)         # contexts of few key tiles: nothing is cut, nothing joined
    counted(1, L.wq4_prompt_attention(ctypes.byref(short), 4 * A, 4096, 8 * A, 5 * A, 6 * A, 4096, 3, 900, 32, 0.1, 0, 0, 7 * A,
                                      1 << 30, None))
    counted(1, L.wq4_kv_reserve(r, A, A, 3, None))
    counted(2, L.wq4_kv_fork(r, A, A, 3, None))
    counted(2, L.wq4_kv_free(r, A, 3, None))
    counted(1, L.wq4_kv_trim(r, A, 3, 5, 0, None))
    counted(2, L.wq4_kv_compact(r, None))
    counted(2, L.wq4_kv_copy_pages(r, A, A, 3, None))
    counted(0, L.wq4_kv_free(r, None, 0, None))
"""


def test_launches_on_every_device(fake_cudart):
    env = dict(os.environ, LD_PRELOAD=fake_cudart, PYTHONPATH=os.path.dirname(HERE))
    r = subprocess.run([sys.executable, "-c", CHILD, fake_cudart, HERE], env=env, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
