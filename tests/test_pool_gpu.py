"""The page pool against its reference, bit for bit, and the operators of a cache used together."""
import math

import numpy as np
import pytest
import torch

import oracle
from oracle import cache as oc
from paper_2412_15803_gb300 import synth, wq4

pytestmark = pytest.mark.gpu

D = 128
REFUSED = 128


def ints(a):
    return torch.tensor(np.asarray(a, np.int32), dtype=torch.int32, device="cuda")


class Twin:
    """A pool on the device and its reference, put through the same calls."""

    def __init__(self, pages, seqs, stride, P=16, layers=2, Hkv=2, seed=0, wild=True):
        self.P, self.Hkv = P, Hkv
        kv = [synth.kv_cache(seed, pages, Hkv, P, D, layer=l) for l in range(layers)]
        self.ref = oc.Pool(pages, seqs, stride, P, [a for pair in kv for a in pair])
        self.caches = [torch.from_numpy(a.copy().view(np.int16)).cuda() for a in self.ref.caches]
        self.table, self.lens, self.refs = ints(self.ref.table), ints(self.ref.lens), ints(self.ref.refs)
        n = wq4.wq4_kv_pool_workspace_bytes(pages, seqs)
        self.ws = torch.full((n,), 0xAB if wild else 0, dtype=torch.uint8, device="cuda")
        self.layers = [wq4.kv_cache_desc(self.caches[2 * l], self.caches[2 * l + 1], self.table, P) for l in range(layers)]
        self.pool = wq4.kv_pool_desc(self.layers, self.table, self.lens, self.refs, self.ws)

    def call(self, name, *lists, more=(), stream=None):
        before = self.ref.refused
        getattr(self.ref, name)(*[list(map(int, x)) for x in lists], *more)
        dev = [ints(x) for x in lists]
        n = (len(lists[0]),) if lists else ()
        getattr(wq4, "wq4_kv_" + name)(self.pool, *dev, *n, *more, stream=stream)
        torch.cuda.synchronize()
        assert (wq4.wq4_device_status() != 0) == (self.ref.refused != before)
        self.check()

    def check(self):
        assert np.array_equal(self.table.cpu().numpy(), self.ref.table)
        assert np.array_equal(self.lens.cpu().numpy(), self.ref.lens)
        assert np.array_equal(self.refs.cpu().numpy(), self.ref.refs)
        for got, want in zip(self.caches, self.ref.caches):
            assert np.array_equal(got.cpu().numpy().view(np.uint16), want)


def test_reserve_fork_free_trim_compact():
    t = Twin(40, 6, 10)
    t.call("reserve", [2, 0, 5], [33, 16, 0])
    t.call("reserve", [0, 2], [17, 40])
    t.call("fork", [2, 2, 0], [1, 3, 4])
    t.call("free", [2, 2])                                # listed twice: freed once
    t.call("reserve", [3, 5], [100, 31])
    t.call("trim", [3, 1], more=(20, 3))
    t.call("fork", [3, 3], [1, 2])                        # a trimmed parent; a child that held pages
    t.call("compact")
    t.call("compact")                                     # nothing left to move
    t.call("free", list(range(6)))
    assert int(t.refs.sum()) == 0


def test_refusals_leave_the_rest():
    t = Twin(6, 3, 4)
    t.call("reserve", [0, 0, 7, 1, -1], [16, 32, 1, 65, 3])
    t.call("reserve", [0], [15])                          # shorter than it is
    t.call("reserve", [1, 2, 0], [64, 48, 17])            # 4 + 3 wanted of 5
    t.call("fork", [0, 1, 0, 0, -3], [1, 2, 2, 9, 0])
    t.call("free", [5, 1, -1])
    t.call("trim", [3, 0], more=(1, 0))
    t.call("copy_pages", [0, 1, 2, 3, 9], [1, 3, 3, 0, 2])
    t.call("copy_pages", [5, 5, 0], [2, 4, 0])


def test_fork_without_a_free_page():
    t = Twin(4, 5, 4)
    t.call("reserve", [0], [40])
    t.call("fork", [0, 0, 0], [1, 2, 3])                  # one page left: the first child gets it
    assert t.lens.tolist() == [40, 40, 0, 0, 0]


def test_empty_lists_and_a_fork_longer_than_the_pool():
    t = Twin(1, 9, 1)
    t.call("reserve", [], [])
    t.call("free", [])
    t.call("fork", [], [])
    t.call("copy_pages", [], [])
    t.call("reserve", [0], [16])
    t.call("fork", [0] * 8, list(range(1, 9)))            # a full page: shared by all
    assert t.refs.tolist() == [9]
    t.call("compact")


@pytest.mark.parametrize("P,Hkv,layers", [(16, 1, 1), (32, 3, 3), (64, 2, 2)])
def test_random_life(P, Hkv, layers):
    rng = np.random.default_rng(P)
    S, stride = 12, 7
    t = Twin(50, S, stride, P=P, layers=layers, Hkv=Hkv, seed=P)
    for _ in range(60):
        op = rng.integers(0, 6)
        n = int(rng.integers(1, 6))
        seqs = rng.integers(-1, S + 1, n)
        if op == 0:
            t.call("reserve", seqs, [int(t.ref.lens[s]) + int(rng.integers(0, 3 * P)) if 0 <= s < S else 5 for s in seqs])
        elif op == 1:
            t.call("fork", seqs, rng.integers(0, S, n))
        elif op == 2:
            t.call("free", seqs[:2])
        elif op == 3:
            t.call("trim", seqs, more=(int(rng.integers(1, 3 * P)), int(rng.integers(0, P + 2))))
        elif op == 4:
            t.call("compact")
        else:
            t.call("copy_pages", rng.integers(-1, 51, n), rng.integers(-1, 51, n))


def test_a_pool_of_many_pages():
    """More pages than one scan looks at, all low ones taken."""
    pages = 70_001
    t = Twin.__new__(Twin)
    ref = oc.Pool(pages, 1024, 80, 16)
    t.ref, t.caches = ref, []
    k = torch.zeros((pages, 1, 16, D), dtype=torch.int16, device="cuda")
    v = torch.zeros_like(k)
    k[:, 0, 0, 0] = (torch.arange(pages, device="cuda") % 30011).to(torch.int16)
    t.table, t.lens, t.refs = ints(ref.table), ints(ref.lens), ints(ref.refs)
    t.ws = torch.zeros(wq4.wq4_kv_pool_workspace_bytes(pages, 1024), dtype=torch.uint8, device="cuda")
    t.layers = [wq4.kv_cache_desc(k, v, t.table, 16)]
    t.pool = wq4.kv_pool_desc(t.layers, t.table, t.lens, t.refs, t.ws)
    lens = np.random.default_rng(1).integers(0, 1100, 1024)

    def fast_reserve(seqs, new_lens):                     # the reference's rule, all pages free from `at` on
        at = int(ref.refs.sum())
        for s, L in zip(seqs, new_lens):
            old, new = ref.pages(int(ref.lens[s])), ref.pages(L)
            ref.table[s, old:new] = np.arange(at, at + new - old)
            ref.refs[at:at + new - old] = 1
            at += new - old
            ref.lens[s] = L
    ref.reserve = fast_reserve
    t.call("reserve", list(range(1024)), lens)
    t.call("reserve", [3, 1000], [1280, 1270])
    t.call("free", list(range(0, 1024, 2)))
    t.call("compact")
    page = t.table[1, 0]
    assert int(k[page, 0, 0, 0]) >= 0


def test_captured_and_replayed():
    """A decode iteration's housekeeping as a graph: trimmed and grown by 5 tokens at every replay."""
    t = Twin(40, 2, 30)
    t.call("reserve", [0, 1], [64, 30])
    seqs = ints([0, 1])
    grown = torch.empty_like(t.lens)
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        torch.add(t.lens, 5, out=grown)
        wq4.wq4_kv_trim(t.pool, seqs, 2, 33, 1, stream=s)
        wq4.wq4_kv_reserve(t.pool, seqs, grown, 2, stream=s)
    t.check()
    for _ in range(60):
        g.replay()
        t.ref.trim([0, 1], 33, 1)
        t.ref.reserve([0, 1], [int(x) + 5 for x in t.ref.lens])
    torch.cuda.synchronize()
    assert wq4.wq4_device_status() == 0
    t.check()


@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 3)])
def test_together(window, sinks):
    """Two prompts in chunks, a sample forked, decoded and trimmed, the pool compacted: every
    attention against the reference on the whole history of its sequence."""
    Hq, Hkv, P, W = 8, 2, 16, 12
    G = (Hq + 2 * Hkv) * D
    scale = 1 / math.sqrt(D)
    t = Twin(40, 4, W, layers=1, seed=5)
    hist = {s: (np.zeros((0, Hkv, D), np.uint16), np.zeros((0, Hkv, D), np.uint16)) for s in range(4)}
    ws = torch.zeros(max(wq4.wq4_prompt_attention_workspace_bytes(4, 200, Hq, Hkv, D),
                         wq4.wq4_paged_attention_workspace_bytes(4, Hq, Hkv, D)), dtype=torch.uint8, device="cuda")
    draws = 0

    def step(grow):
        """The sequences' new tokens: pages, rotation and append, attention; grow[s] tokens each."""
        nonlocal draws
        live = [int(x) for x in t.lens]
        t.call("reserve", list(range(4)), [a + b for a, b in zip(live, grow)])
        t.ref.caches = [c.cpu().numpy().view(np.uint16) for c in t.caches]
        rows = sum(grow)
        draws += 1
        qkv = synth.sum4_fp16(9, 300 + draws, 0, rows * G).reshape(rows, G)
        starts = [0] + np.cumsum(grow).tolist()
        x, q = torch.from_numpy(qkv.view(np.int16)).cuda(), torch.zeros((rows, Hq * D), dtype=torch.int16, device="cuda")
        wq4.wq4_prompt_append(t.layers[0], x, G, q, Hq * D, ints(starts), t.lens, 4, rows, Hq, 10000.0)
        out = torch.zeros_like(q)
        if max(grow) == 1 and min(grow) == 1:
            wq4.wq4_window_attention(t.layers[0], q, Hq * D, t.lens, out, Hq * D, 4, Hq, scale, window, sinks, ws, ws.numel())
        else:
            ws.random_(0, 256)
            wq4.wq4_prompt_attention(t.layers[0], q, Hq * D, ints(starts), t.lens, out, Hq * D, 4, rows, Hq, scale, window, sinks,
                                     ws, ws.numel())
            ws.zero_()
        torch.cuda.synchronize()
        assert wq4.wq4_device_status() == 0
        t.ref.caches = [c.cpu().numpy().view(np.uint16) for c in t.caches]
        q16, o16 = q.cpu().numpy().view(np.uint16), out.cpu().numpy().view(np.uint16)
        for s in range(4):
            if not grow[s]:
                continue
            mine = qkv[starts[s]:starts[s + 1]]
            _, keys = oracle.rope(np.ascontiguousarray(mine[:, Hq * D:(Hq + Hkv) * D]), [live[s] + i for i in range(grow[s])], D, 10000.0)
            k = np.concatenate([hist[s][0], keys.reshape(-1, Hkv, D)])
            v = np.concatenate([hist[s][1], mine[:, (Hq + Hkv) * D:].reshape(-1, Hkv, D)])
            hist[s] = (k, v)
            one = k.shape[0]                              # the history as one page of its own
            o, A, _ = oc.attention(q16[starts[s]:starts[s + 1]], k.transpose(1, 0, 2)[None].copy(), v.transpose(1, 0, 2)[None].copy(),
                                   np.zeros((1, 1), np.int32), [0, grow[s]], [one], scale, Hq, window, sinks)
            err = np.abs(oracle.half_to_double(np.ascontiguousarray(o16[starts[s]:starts[s + 1]])).reshape(o.shape) - o)
            # a cached key may be one fp16 step from the reference's rotation: 2^-10 of a score's terms
            assert np.all(err <= oc.attention_tolerance(o, A) + 2.0 ** -10 * A)

    step([70, 0, 33, 0])
    step([20, 0, 1, 0])
    t.call("fork", [0, 2], [1, 3])
    hist[1], hist[3] = hist[0], hist[2]
    for i in range(20):
        step([1, 1, 1, 1])
        if window and i % 3 == 0:
            t.call("trim", [0, 1, 2, 3], more=(window, sinks))
        if i == 7:
            t.call("free", [2])
            hist[2] = (np.zeros((0, Hkv, D), np.uint16),) * 2
            t.call("compact")
            step([3, 1, 40, 2])
