"""Microscaled calls right behind a kernel that is still writing what they read.

The writer lets its dependents launch at its start and writes late; before it the buffers
hold something else, so that a call which reads before the writer is through shows.
"""
import numpy as np
import pytest
import torch

from paper_2412_15803_gb300 import wq4
from test_dependent_launch_gpu import late_copy  # noqa: F401  (a fixture)
from test_mx_gpu import Layer, same

pytestmark = pytest.mark.gpu

# one row a thread, four rows a thread; the norm's rows by a warp, by a block, by bulk copies
FEW, MANY = [(1, 4096), (33, 1152)], [(700, 33024), (5000, 4096)]


def rows(M, width, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((M, width), generator=g, device="cuda").half().view(torch.int16)


def held(M, K, bits):
    return (torch.zeros((M, K * bits // 8), dtype=torch.uint8, device="cuda"),
            torch.zeros(wq4.wq4_mx_scale_bytes(M, K), dtype=torch.uint8, device="cuda"))


def check_late(late_copy, inputs, outputs, call):
    """Each input in turn written late, everything else as it was, outputs cleared."""
    call()
    torch.cuda.synchronize()
    want = [t.clone() for t in outputs]
    kept = [t.clone() for t in inputs]
    for i, t in enumerate(inputs):
        for a, b in zip(inputs, kept):
            a.copy_(b)
        for o in outputs:
            if all(o is not a for a in inputs):
                o.zero_()
        t.zero_()
        torch.cuda.synchronize()
        late_copy(t, kept[i])
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outputs, want)), f"input {i} read before it was written"
        assert any(torch.any(w != 0) for w in want)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,K", FEW + MANY)
def test_quantize(late_copy, M, K, bits):  # noqa: F811
    x, (c, s) = rows(M, K, 1), held(M, K, bits)
    check_late(late_copy, [x], [c, s], lambda: wq4.wq4_mx_quantize(x, K, c, s, M, K, bits))


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,K", FEW + MANY)
def test_silu(late_copy, M, K, bits):  # noqa: F811
    gu, (c, s) = rows(M, 2 * K, 2), held(M, K, bits)
    check_late(late_copy, [gu], [c, s], lambda: wq4.wq4_mx_silu(gu, 2 * K, c, s, M, K, bits))


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,K", FEW + MANY)
def test_dequantize(late_copy, M, K, bits):  # noqa: F811
    (c, s), y = held(M, K, bits), torch.zeros((M, K), dtype=torch.int16, device="cuda")
    wq4.wq4_mx_quantize(rows(M, K, 3), K, c, s, M, K, bits)
    check_late(late_copy, [c, s], [y], lambda: wq4.wq4_mx_dequantize(c, s, y, K, M, K, bits))


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,K", FEW + MANY + [(40, 512), (700, 8192)])
def test_norm(late_copy, M, K, bits):  # noqa: F811
    x, r, g, (c, s) = rows(M, K, 4), rows(M, K, 5), rows(1, K, 6), held(M, K, bits)
    h = torch.zeros((M, K), dtype=torch.int16, device="cuda")
    check_late(late_copy, [x, r, g], [h, c, s], lambda: wq4.wq4_mx_norm(x, K, r, K, g, 1e-5, h, K, c, s, M, K, bits))

@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M", [1, 40, 600])
def test_layer_back_to_back_into_cleared_buffers(late_copy, M, bits):  # noqa: F811
    """Nothing of the run before is left for a call that reads too early."""
    L = Layer(M, bits, 4, H=1024, F=2048, nq=1536)
    L.run(sync=True)
    want = L.state()
    for _ in range(4):
        L.reset()
        for t in (L.qkv, L.o, L.gu, L.y, *(t for p in L.held for t in p)):
            t.zero_()
        src = L.x.clone()
        L.x.zero_()
        torch.cuda.synchronize()
        late_copy(L.x, src, 100_000)
        L.run()
        assert same(L.state(), want)
    assert all(np.any(t.cpu().numpy()) for t in want)
    assert wq4.wq4_device_status() == 0
