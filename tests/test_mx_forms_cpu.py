"""Which form of the microscaled product a call takes, and how the norm's launches fill the SMs.

Run without a GPU over a stand-in for the CUDA runtime (fake_cudart.c), which tells the kernel,
the grid and the shared memory of the last launch.
"""
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))

HEAD = r"""
import ctypes, sys
fake = ctypes.CDLL(sys.argv[1])
fake.fake_last_shape.restype = ctypes.c_size_t
from paper_2412_15803_gb300 import wq4
L = wq4.load(build_if_missing=False)
A = 1 << 40

def product(M, N, K, bits, off=0):
    '(kernel, grid, shared memory)'
    assert L.wq4_mx_gemm(A, 4 * A, 8 * A, 16 * A, 32 * A + off, N, K, M, bits, None) == 0
    s = fake.fake_last_shape()
    return fake.fake_last_kernel(), s >> 32, s & 0xffffffff
"""


def run(fake_cudart, child):
    env = dict(os.environ, LD_PRELOAD=fake_cudart, PYTHONPATH=os.path.dirname(HERE))
    r = subprocess.run([sys.executable, "-c", HEAD + child, fake_cudart], env=env, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]


def test_rows_that_tensor_copies_cannot_write_by_address(fake_cudart):
    """y off a multiple of 16 bytes costs what rows that 16 bytes do not divide cost: the same form for both."""
    run(fake_cudart, r"""
other = 0
for bits in (8, 4):
    for M, N, K in ((4000, 16384, 512), (600, 9728, 256), (2048, 28672, 4096), (730, 71064, 256), (1500, 10000, 128), (3, 264, 256),
                    (300, 30000, 384), (8192, 28672, 4096)):
        odd = product(M, N - 1, K, bits)[0]
        assert product(M, N, K, bits, 2)[0] == product(M, N, K, bits, 8)[0] == odd, (bits, M, N, K)
        other += product(M, N, K, bits)[0] != odd
assert other >= 3       # sizes where it decides
""")


def test_form_hook(fake_cudart):
    """Each form by its blocks' shared memory and its grid; what it does not take is refused."""
    run(fake_cudart, r"""
HALF, WHOLE = 113 * 1024, 227 * 1024
f = L.wq4_test_mx_form
refused = lambda *a: L.wq4_mx_gemm(A, 4 * A, 8 * A, 16 * A, 32 * A, a[1], a[2], a[0], a[3], None) == wq4.WQ4_ERR_UNSUPPORTED
sizes = [(1, 1, 128, 8), (1, 6144, 4096, 8), (77, 5003, 2176, 4), (300, 640, 14336, 8), (2048, 28672, 4096, 4)]
before = [product(*c) for c in sizes]
pairs = {}
for M, N, K, bits in ((1, 1, 128, 8), (33, 1003, 2176, 8), (80, 1003, 2176, 4), (300, 640, 14336, 8), (2048, 28672, 4096, 4)):
    tiles = -(-N // 128) * -(-M // min(128, -(-M // 16) * 16))
    for form, smem in ((1, HALF), (2, WHOLE)):
        for split in range(9):
            assert f(form, split) == 0
            slots = -(-K // (128 if bits == 8 and form == 1 else 256))
            if (form == 1 and M > 80) or split > slots:
                assert refused(M, N, K, bits), (M, N, K, bits, form, split)
            else:
                k, grid, s = product(M, N, K, bits)
                assert s == smem and (split == 0 or grid == (min(tiles, 304 if form == 1 else 152) if split == 1 else tiles * split))
    assert f(3, 0) == 0
    k, grid, s = product(M, N, K, bits)
    assert s not in (HALF, WHOLE) and grid == 2 * min(76, -(-N // 256) * -(-M // 256))
    assert pairs.setdefault(bits, k) == k
for bad in ((-1, 0), (4, 0), (0, 1), (3, 2), (1, 9), (2, -1)):
    assert f(*bad) == wq4.WQ4_ERR_INVALID
assert f(0, 0) == 0 and [product(*c) for c in sizes] == before
""")


def test_norm_of_many_long_rows(fake_cudart):
    """A block holds one row of each input in shared memory, whatever the width: more were of no use, and mostly not there."""
    run(fake_cudart, r"""
for K in range(6272, 16385, 128):
    for residual in (4 * A, None):
        for bits in (8, 4):
            assert L.wq4_mx_norm(A, K, residual, K, 128 * A, 1e-5, None, 0, 16 * A, 64 * A, 8000, K, bits, None) == 0
            s = fake.fake_last_shape()
            assert s & 0xffffffff == (4 if residual else 2) * K and 152 <= s >> 32 <= 8000
""")


def test_longest_sums(fake_cudart):
    """A tile's sum ends well within the limit of a wait for it, and its error stays below the sum: K to 2^24."""
    run(fake_cudart, r"""
for bits in (8, 4):
    for M, N in ((1, 1), (1, 128), (256, 256)):
        product(M, N, 1 << 24, bits)
        for K in ((1 << 24) + 128, (1 << 31) - 128):
            assert L.wq4_mx_gemm(A, 4 * A, 8 * A, 16 * A, 32 * A, N, K, M, bits, None) == wq4.WQ4_ERR_UNSUPPORTED
""")
