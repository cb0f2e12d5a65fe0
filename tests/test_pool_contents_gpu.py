"""What a pool of more pages than one scan looks at holds, page by page, after its pages have moved."""
import numpy as np
import pytest
import torch

from paper_2412_15803_gb300 import wq4

pytestmark = pytest.mark.gpu

PAGES, SEQS, STRIDE, P, D = 70_001, 1024, 80, 16, 128       # 16384 pages a scan: five of them


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


@pytest.fixture()
def pool():
    """Two layers; every page's keys and values carry its number, in the page's first and last elements."""
    class Made:
        pass
    m = Made()
    number = torch.arange(PAGES, device="cuda")
    m.caches = []
    for i in range(4):
        c = torch.zeros((PAGES, 1, P, D), dtype=torch.int16, device="cuda")
        c[:, 0, 0, 0] = c[:, 0, P - 1, D - 1] = (number & 0x7FFF).to(torch.int16)
        c[:, 0, 0, 1] = (number >> 15).to(torch.int16)
        c[:, 0, 0, 2] = i                                    # and which array it is
        m.caches.append(c)
    m.table = torch.full((SEQS, STRIDE), -1, dtype=torch.int32, device="cuda")
    m.lens, m.refs = ints(np.zeros(SEQS)), ints(np.zeros(PAGES))
    m.ws = torch.empty(wq4.wq4_kv_pool_workspace_bytes(PAGES, SEQS), dtype=torch.uint8, device="cuda").fill_(0x77)
    m.layers = [wq4.kv_cache_desc(m.caches[2 * l], m.caches[2 * l + 1], m.table, P) for l in range(2)]
    m.pool = wq4.kv_pool_desc(m.layers, m.table, m.lens, m.refs, m.ws)

    def numbers(c, pages):
        pages = pages.long()
        assert torch.equal(c[pages, 0, 0, 0], c[pages, 0, P - 1, D - 1])
        return c[pages, 0, 0, 0].long() + (c[pages, 0, 0, 1].long() << 15)
    m.numbers = numbers
    return m


def test_compaction_moves_every_page_with_its_contents(pool):
    rng = np.random.default_rng(1)
    wq4.wq4_kv_reserve(pool.pool, ints(np.arange(SEQS)), ints(rng.integers(600, STRIDE * P + 1, SEQS)), SEQS)
    wq4.wq4_kv_free(pool.pool, ints(np.arange(0, SEQS, 3)), len(range(0, SEQS, 3)))
    wq4.wq4_kv_trim(pool.pool, ints(np.arange(1, SEQS, 3)), len(range(1, SEQS, 3)), 200, 17)
    torch.cuda.synchronize()
    named = pool.table >= 0
    before, live = pool.table[named].clone(), int((pool.refs > 0).sum())
    assert int(before.max()) > 3 * 16384 and live > 16384 and int((pool.refs[:live] == 0).sum()) > 16384 // 2
    refs = pool.refs[before.long()].clone()
    wq4.wq4_kv_compact(pool.pool)
    torch.cuda.synchronize()
    assert wq4.wq4_device_status() == 0
    assert torch.equal(pool.table >= 0, named) and int(pool.refs[live:].abs().sum()) == 0 and int((pool.refs[:live] > 0).sum()) == live
    after = pool.table[named]
    assert torch.equal(pool.refs[after.long()], refs)
    for i, c in enumerate(pool.caches):
        assert torch.equal(pool.numbers(c, after), before.long())
        assert torch.all(c[after.long(), 0, 0, 2] == i)


def test_copies_of_many_pages(pool):
    """More pairs than one pass of the planning block, among them pairs that are refused."""
    order = torch.randperm(PAGES, generator=torch.Generator().manual_seed(3)).to(torch.int32).cuda()
    n = PAGES // 2
    src, dst = order[:n].clone(), order[n:2 * n].clone()
    dst[100], dst[20_000], src[30_000], src[5] = dst[101], PAGES, -1, dst[7]    # twice a destination, outside, outside, read and written
    wq4.wq4_kv_copy_pages(pool.pool, src, dst, n)
    torch.cuda.synchronize()
    assert wq4.wq4_device_status() == 128
    good = (src >= 0) & (src < PAGES) & (dst >= 0) & (dst < PAGES)
    written = torch.bincount(dst[good].long(), minlength=PAGES)
    ok = good.clone()                                        # its page written once, its source not at all
    ok[good] = (written[dst[good].long()] == 1) & (written[src[good].long()] == 0)
    assert torch.nonzero(~ok)[:, 0].tolist() == [5, 100, 101, 20_000, 30_000]
    want = torch.arange(PAGES, device="cuda")
    want[dst[ok].long()] = src[ok].long()
    for i, c in enumerate(pool.caches):
        assert torch.equal(pool.numbers(c, torch.arange(PAGES, device="cuda")), want)
        assert torch.all(c[:, 0, 0, 2] == i)


@pytest.mark.parametrize("length", [STRIDE * P + 1, 2 ** 31 - 17, 2 ** 31 - 1])
def test_a_length_beyond_the_table_still_frees_its_pages(pool, length):
    wq4.wq4_kv_reserve(pool.pool, ints([4, 9]), ints([STRIDE * P, 100]), 2)
    pool.lens[4] = length
    wq4.wq4_kv_free(pool.pool, ints([4]), 1)
    torch.cuda.synchronize()
    assert wq4.wq4_device_status() == 0
    assert pool.lens[[4, 9]].tolist() == [0, 100] and torch.all(pool.table[4] == -1)
    assert int(pool.refs.sum()) == 7 and pool.refs[pool.table[9, :7].long()].tolist() == [1] * 7
