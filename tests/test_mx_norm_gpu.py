"""The norm of many long rows, several of them a block: each width's own copies, against oracle/mx.py.

Rows repeat after 97 others, so that every row is compared: those of one kind have the same
codes, and one of each is held to the 64-bit norm (tolerance: tests/test_mx_gpu.py).
"""
import numpy as np
import pytest
import torch

from oracle import mx
from paper_2412_15803_gb300 import wq4
from test_mx_gpu import dev, held, padded, taken

pytestmark = pytest.mark.gpu

KINDS = 97


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("residual,summed", [(True, "new"), (True, "residual"), (True, None), (False, "x"), (False, None)])
@pytest.mark.parametrize("M,K", [(609, 6272), (5003, 6272), (4000, 8192), (4000, 11008), (3000, 12416), (2700, 16384)])
def test_many_long_rows(M, K, residual, summed, bits):
    rng = np.random.default_rng(M + K)
    x = rng.standard_normal((KINDS, K)).astype(np.float16)
    res = (3 * rng.standard_normal((KINDS, K))).astype(np.float16) if residual else None
    g = (1 + 0.3 * rng.standard_normal(K)).astype(np.float16)
    kind = np.arange(M) % KINDS
    xs, rs, ss = K + 8, K + 16, K + 24
    xd = dev(padded(x, xs))[torch.from_numpy(kind).cuda()]
    rd = dev(padded(res, rs))[torch.from_numpy(kind).cuda()] if residual else None
    sd = torch.full((M, ss), 0x1234, dtype=torch.int16, device="cuda") if summed == "new" else None
    if summed in ("x", "residual"):
        sd, ss = (xd, xs) if summed == "x" else (rd, rs)
    codes, scales = held(M, K, bits)
    wq4.wq4_mx_norm(xd, xs, rd, rs, dev(g), 1e-5, sd, ss, codes, scales, M, K, bits)
    c, s = taken(codes, scales, M, K)
    assert wq4.wq4_device_status() == 0
    assert np.array_equal(c, c[:KINDS][kind]) and np.array_equal(s, s[:KINDS][kind])
    h, v = mx.norm(x, res, g, 1e-5)
    assert not mx.wrong_groups(c[:KINDS], s[:KINDS], v, bits, 2.0 ** -18).any()
    if sd is not None:
        got = sd.cpu().numpy()[:, :K].view(np.uint16)
        assert np.array_equal(got, h.view(np.uint16)[kind])
