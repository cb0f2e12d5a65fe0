"""Row starts of any contents: nothing outside the rows is written, and what the header says of them holds."""
import numpy as np
import pytest
import torch

from paper_2412_15803_gb300 import synth, wq4
from test_prompt_gpu import D, SCALE, THETA, Call, check, dev, make

pytestmark = pytest.mark.gpu

HQ, HKV, P, ROWS, MARGIN = 8, 2, 16, 40, 64


class Guarded:
    """A device array inside a larger one whose margins keep a pattern."""

    def __init__(self, inner):
        rows, cols = inner.shape
        self.whole = torch.full((rows + 2 * MARGIN, cols), 0x5A5A, dtype=torch.int16, device="cuda")
        self.inner = self.whole[MARGIN:MARGIN + rows]
        self.inner.copy_(inner)
        self.was = self.inner.clone()

    def margins_kept(self):
        return bool(torch.all(self.whole[:MARGIN] == 0x5A5A) and torch.all(self.whole[-MARGIN:] == 0x5A5A))

    def kept(self):
        return self.margins_kept() and torch.equal(self.inner, self.was)


DECREASING = [[0, 500, 40], [30, 10, 40], [2 ** 31 - 1, 0, 0], [0, 40, 39], [0, 0, -1]]
OUTSIDE = [[-5, 20, 10 ** 9], [0, 20, 2 ** 31 - 1], [-2 ** 31, 0, 40], [50, 60, 70], [-9, -5, -1]]


@pytest.mark.parametrize("window,sinks", [(0, 0), (12, 3)])
@pytest.mark.parametrize("starts", DECREASING + OUTSIDE)
def test_attention(starts, window, sinks):
    q, k, v, table, _, _, lens = make(11, [20, 20], [16, 16], HQ, HKV, P, hide=False)
    call = Call(q, k, v, table, starts, lens, HQ)
    out = Guarded(torch.full((ROWS, HQ * D), -1, dtype=torch.int16, device="cuda"))
    call.out = out.inner
    call(window, sinks)
    torch.cuda.synchronize()
    status = wq4.wq4_device_status()
    if starts in DECREASING:
        assert out.kept() and status == 8
        return
    assert out.margins_kept() and status == 0
    inside = [min(max(s, 0), ROWS) for s in starts]               # rows of the buffer that a sequence owns
    if inside[0] == inside[-1]:
        assert out.kept()
    else:
        check(call.result(), q, k, v, table, inside, lens, HQ, window, sinks)


@pytest.mark.parametrize("theta", [THETA, 0.0])
@pytest.mark.parametrize("starts", DECREASING + OUTSIDE + [[0, 20, 40]])
def test_append(starts, theta):
    width = (HQ + 2 * HKV) * D
    k0, v0 = synth.kv_cache(11, 6, HKV, P, D)
    table = np.array([[0, 2, 4], [1, 3, 5]], np.int32)
    k, v = (Guarded(dev(a).reshape(-1, D)) for a in (k0, v0))
    qkv = dev(synth.sum4_fp16(11, 77, 0, ROWS * width).reshape(ROWS, width))
    q = Guarded(torch.full((ROWS, HQ * D), -1, dtype=torch.int16, device="cuda"))
    given = qkv.clone()
    cache = wq4.wq4_kv_cache(k.inner.data_ptr(), v.inner.data_ptr(), 6, HKV, P, D, None, 3)
    td, sd, ld = dev(table, np.int32), dev(np.asarray(starts, np.int32), np.int32), dev(np.array([36, 36], np.int32), np.int32)
    cache.page_table = td.data_ptr()
    wq4.wq4_prompt_append(cache, qkv, width, q.inner, HQ * D, sd, ld, 2, ROWS, HQ, theta)
    torch.cuda.synchronize()
    status = wq4.wq4_device_status()
    assert status in (0, 32) and torch.equal(qkv, given)
    assert q.margins_kept() and k.margins_kept() and v.margins_kept()
    if starts in ([50, 60, 70], [-9, -5, -1]):                     # no row has an owner
        assert q.kept() and k.kept() and v.kept() and status == 0
    if starts == [0, 20, 40]:
        assert status == 0 and not q.kept() and not k.kept() and not v.kept()
