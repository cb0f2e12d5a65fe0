"""The calls around a cache one after another, nothing waited for between: each reads what the
kernel before it writes late (a writer that lets its dependents launch at its start)."""
import math

import pytest
import torch

from paper_2412_15803_gb300 import synth, wq4
from test_dependent_launch_gpu import late_copy  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu

HQ, HKV, D, P, PAGES, N = 8, 2, 128, 16, 64, 300
WIDTH, SCALE, THETA = (HQ + 2 * HKV) * D, 1.0 / math.sqrt(D), 10000.0


def ints(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


class Step:
    """A prompt of N tokens into an empty pool, a fork, and a token of both under a window."""

    def __init__(self):
        self.k = torch.zeros((PAGES, HKV, P, D), dtype=torch.int16, device="cuda")
        self.v = torch.zeros_like(self.k)
        self.table, self.lens, self.refs = torch.full((2, 24), -1, dtype=torch.int32, device="cuda"), ints([0, 0]), ints([0] * PAGES)
        self.cache = wq4.kv_cache_desc(self.k, self.v, self.table, P)
        self.pool_ws = torch.zeros(wq4.wq4_kv_pool_workspace_bytes(PAGES, 2), dtype=torch.uint8, device="cuda")
        self.pool = wq4.kv_pool_desc([self.cache], self.table, self.lens, self.refs, self.pool_ws)
        self.ws = torch.zeros(max(wq4.wq4_prompt_attention_workspace_bytes(2, N, HQ, HKV, D),
                                  wq4.wq4_paged_attention_workspace_bytes(2, HQ, HKV, D)), dtype=torch.uint8, device="cuda")
        self.win_ws = torch.zeros(wq4.wq4_paged_attention_workspace_bytes(2, HQ, HKV, D), dtype=torch.uint8, device="cuda")
        x = synth.sum4_fp16(5, 1, 0, (N + 2) * WIDTH).reshape(N + 2, WIDTH)
        self.x = torch.from_numpy(x.view("int16")).cuda()
        self.q, self.out = (torch.zeros((N + 2, HQ * D), dtype=torch.int16, device="cuda") for _ in range(2))
        self.starts, self.one = ints([0, N, N]), ints([0, 1, 2])
        self.lists = [ints(a) for a in ([0], [N], [1], [0, 1], [N + 1, N + 1])]

    def calls(self):
        zero, n, one, both, more = self.lists
        p, c = self.pool, self.cache
        return [lambda: wq4.wq4_kv_reserve(p, zero, n, 1),
                lambda: wq4.wq4_prompt_append(c, self.x, WIDTH, self.q, HQ * D, self.starts, self.lens, 2, N, HQ, THETA),
                lambda: wq4.wq4_prompt_attention(c, self.q, HQ * D, self.starts, self.lens, self.out, HQ * D, 2, N, HQ, SCALE, 0, 0,
                                                 self.ws, self.ws.numel()),
                lambda: wq4.wq4_kv_fork(p, zero, one, 1),
                lambda: wq4.wq4_kv_reserve(p, both, more, 2),
                lambda: wq4.wq4_prompt_append(c, self.x[N:], WIDTH, self.q[N:], HQ * D, self.one, self.lens, 2, 2, HQ, THETA),
                lambda: wq4.wq4_window_attention(c, self.q[N:], HQ * D, self.lens, self.out[N:], HQ * D, 2, HQ, SCALE, 40, 3,
                                                 self.win_ws, self.win_ws.numel()),
                lambda: wq4.wq4_kv_trim(p, both, 2, 64, 4),
                lambda: wq4.wq4_kv_compact(p)]

    def state(self):
        torch.cuda.synchronize()
        return [t.clone() for t in (self.k, self.v, self.table, self.lens, self.refs, self.q, self.out)]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_a_step_back_to_back(late_copy):  # noqa: F811
    ref = Step()
    for call in ref.calls():
        call()
        torch.cuda.synchronize()
    want = ref.state()
    for _ in range(5):
        s = Step()
        src = s.x.clone()
        s.x.zero_()
        torch.cuda.synchronize()
        late_copy(s.x, src, 100_000)
        for call in s.calls():
            call()
        assert same(s.state(), want)
    assert wq4.wq4_device_status() == 0


NAMES = ["reserve", "append", "attention", "fork", "reserve2", "append2", "window", "trim", "compact"]
READS = {"reserve": ("table", "lens", "refs"), "append": ("x", "starts", "lens", "table"), "attention": ("q", "k", "v", "table", "starts", "lens"),
         "fork": ("table", "lens", "refs", "k", "v"), "window": ("q", "k", "v", "table", "lens"), "trim": ("table", "lens", "refs"),
         "compact": ("table", "lens", "refs", "k", "v")}


@pytest.mark.parametrize("name,array", [(n, a) for n, arrays in READS.items() for a in arrays])
def test_each_array_written_right_before(late_copy, name, array):  # noqa: F811
    i = NAMES.index(name)
    results = []
    for late in (False, True):
        s = Step()
        calls = s.calls()
        for call in calls[:i]:
            call()
        torch.cuda.synchronize()
        t = getattr(s, array)
        if late:
            src = t.clone()
            t.zero_()
            torch.cuda.synchronize()
            late_copy(t, src, 100_000)
        calls[i]()
        results.append(s.state())
    assert same(*results)
    assert wq4.wq4_device_status() == 0
