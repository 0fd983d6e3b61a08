"""GPU: the cache's page operators against a cache kept row by row in Python. Everything is
compared exactly: tables, lengths, reference counts, statuses and the bytes of every page."""

import numpy as np
import pytest
import torch

from gpu_util import dev_i32
from oracle import history as oracle
from paper_2607_27744_amd import ops

pytestmark = pytest.mark.gpu


class Pair:
    """The same cache on the device and in the oracle; rows are distinct whole numbers."""

    def __init__(self, layers, pages, page, slots, width, heads=1, dim=4, dtype=torch.bfloat16):
        self.dev = ops.cache_pool(layers, pages, page, heads, dim, slots=slots, table_width=width,
                                  dtype=dtype)
        self.ref = oracle.Cache(layers, pages, page, slots, width)
        self.page, self.layers, self.width, self.dtype = page, layers, 2 * heads * dim, dtype
        self.next = 1

    def state(self):
        return self.dev[1:]

    def append(self, slots, counts):
        pool, table, lens, refs = self.dev
        total = int(sum(counts))
        off = dev_i32(np.concatenate([[0], np.cumsum(counts)]))
        rows, status = ops.cache_reserve(dev_i32(slots), off, total, table, lens, refs, self.page)
        want, code = self.ref.reserve(list(slots), list(counts))
        assert tuple(status.tolist()) == code and rows.tolist() == want
        for layer in range(self.layers):
            ids = (torch.arange(total) + self.next) % 251
            self.next += total
            x = ids[:, None].expand(total, self.width).to(self.dtype).cuda().contiguous()
            ops.cache_write(x, rows, pool[layer])
            self.ref.write(layer, want, ids.tolist())
        return code[0]

    def fork(self, parents, children):
        status = ops.cache_fork(dev_i32(parents), dev_i32(children), *self.state(), self.dev[0])
        code = self.ref.fork(list(parents), list(children))
        assert tuple(status.tolist()) == code
        return code[0]

    def free(self, slots):
        ops.cache_free(dev_i32(slots), *self.state(), self.page)
        self.ref.free(list(slots))

    def compact(self):
        status = ops.cache_compact(*self.state(), self.dev[0])
        assert tuple(status.tolist()) == self.ref.compact()

    def check(self):
        pool, table, lens, refs = self.dev
        assert table.tolist() == self.ref.table
        assert lens.tolist() == self.ref.lens and refs.tolist() == self.ref.refs
        got = pool.flatten(3).float().cpu()
        assert bool((got == got[..., :1]).all())                # a row is one number throughout
        want = [[[0 if x is None else x for x in p] for p in layer] for layer in self.ref.pool]
        assert torch.equal(got[..., 0], torch.tensor(want, dtype=torch.float32))


@pytest.mark.parametrize("page, heads, dim, dtype", [
    (1, 1, 4, torch.bfloat16), (7, 1, 3, torch.bfloat16), (16, 2, 64, torch.bfloat16),
    (64, 4, 128, torch.bfloat16), (5, 1, 1, torch.float32)])
@pytest.mark.parametrize("layers", [1, 3])
def test_a_life_of_a_cache(gpu_lib, page, heads, dim, dtype, layers):
    rng = np.random.default_rng(page)
    c = Pair(layers, 90, page, 24, 12, heads, dim, dtype)
    seen = set()
    for step in range(60):
        kind = rng.choice(["append", "append", "append", "fork", "free", "compact"])
        live = [s for s, n in enumerate(c.ref.lens) if n]
        if kind == "append":
            slots = rng.choice(24, rng.integers(1, 12), replace=False)
            code = c.append(slots, rng.integers(0, 2 * page + 2, slots.size))
        elif kind == "fork" and live:
            empty = [s for s, n in enumerate(c.ref.lens) if not n][:int(rng.integers(1, 6))]
            code = c.fork(rng.choice(live, len(empty)), empty) if empty else 0
        elif kind == "free" and live:
            c.free(rng.choice(live, min(len(live), int(rng.integers(1, 6)))))   # may repeat one
            code = 0
        else:
            c.compact()
            code = 0
        seen.add((kind, code))
        c.check()
    assert {k for k, _ in seen} == {"append", "fork", "free", "compact"}


def test_all_or_nothing(gpu_lib):
    c = Pair(1, 6, 4, 6, 3)
    assert c.append([0, 1], [9, 6]) == 0                        # 3 + 2 pages of 6
    for slots, counts, code in (([2], [5], 1), ([2, 3], [4, 1], 1), ([0], [4], 2), ([2, 2], [1, 1], 3),
                                ([6], [1], 3), ([-1], [1], 3), ([0, 2, 2], [9, 1, 1], 3)):
        assert c.append(slots, counts) == code
        c.check()
    for parents, children, code in (([0, 1], [2, 3], 1), ([0], [1], 3), ([0, 1], [2, 2], 3),
                                    ([0, 2], [2, 3], 3), ([7], [2], 3), ([0], [-1], 3), ([2], [2], 3)):
        assert c.fork(parents, children) == code
        c.check()
    assert c.fork([0], [4]) == 0 and c.append([4, 1], [3, 2]) == 0
    c.check()
    c.free([0, 0, 9, -3, 5])                                    # twice, out of range, empty
    c.check()
    assert c.fork([5], [0]) == 0                                # an empty parent: an empty child
    c.check()


def test_lengths_that_cannot_be(gpu_lib):
    # Device data that the operators did not write: refused, with nothing read or changed.
    c = Pair(1, 6, 4, 4, 2)
    assert c.append([0, 3], [7, 6]) == 0
    for length, code in ((-1, 3), (-100, 3), (9, 2), (2 ** 31 - 1, 2)):
        c.ref.lens[3] = length
        c.dev[2][3] = length
        assert c.append([3], [1]) == code and c.fork([3], [1]) == 3
        c.check()
    c.ref.lens[3] = 6
    c.dev[2][3] = 6
    assert c.fork([3], [1]) == 0
    c.check()


def test_empty_calls(gpu_lib):
    c = Pair(2, 4, 4, 3, 2)
    assert c.append([], []) == 0 and c.append([1], [0]) == 0 and c.fork([], []) == 0
    c.free([])
    c.compact()
    c.check()


@pytest.mark.parametrize("pages, slots", [(4096, 40), (4097, 40), (20000, 700)])
def test_many_pages(gpu_lib, pages, slots):
    # More pages than one round of the scans takes, in one and in many blocks.
    rng = np.random.default_rng(pages)
    c = Pair(1, pages, 2, slots, 2 * pages // slots, dim=1)
    assert c.append(np.arange(slots), rng.integers(1, 3 * pages // slots, slots)) == 0
    for _ in range(3):
        c.free(rng.choice(slots, slots // 3, replace=False))
        c.check()
        c.compact()
        c.check()
        c.append(rng.permutation(slots)[:slots // 4], rng.integers(0, 30, slots // 4))
        c.check()
    c.free(np.arange(slots))
    c.compact()
    c.check()


def test_full_cache_compacts(gpu_lib):
    for pages in (8, 4096, 8192):
        c = Pair(1, pages, 1, 4, pages, dim=1)
        assert c.append([0, 1], [pages // 2, pages // 2]) == 0
        c.compact()
        c.check()
        c.free([0])
        c.compact()
        c.check()


def test_many_entries(gpu_lib):
    # More entries than one segment of the reserve kernel, more rows than it places itself.
    n = 9001
    rng = np.random.default_rng(1)
    c = Pair(1, 30000, 3, n, 4, dim=1)
    assert c.append(rng.permutation(n), rng.integers(0, 4, n)) == 0
    c.check()
    assert c.append(rng.permutation(n)[:5000], rng.integers(0, 2, 5000)) == 0
    c.check()


@pytest.mark.parametrize("entries, padded", [(3, 10), (5, 9000)])
def test_a_padded_batch(gpu_lib, entries, padded):
    # A fixed number of rows of which the last belong to no entry: they go nowhere.
    pool, table, lens, refs = ops.cache_pool(1, 40, 4, 1, 8, slots=entries, table_width=8)
    off = dev_i32(np.arange(entries + 1) + (np.arange(entries + 1) > 1))      # one has two rows
    rows = torch.full((padded,), 7, dtype=torch.int32, device="cuda")
    got, status = ops.cache_reserve(dev_i32(np.arange(entries)), off, padded, table, lens, refs, 4,
                                    rows=rows)
    assert got is rows and status.tolist() == [0, 0]
    n = entries + 1
    assert rows[:n].min() >= 0 and bool((rows[n:] == -1).all()) and int(lens.sum()) == n
    ops.cache_write(torch.ones((padded, 16), dtype=torch.bfloat16, device="cuda"), rows, pool[0])
    assert float(pool.float().sum()) == 16 * n


def test_write_strided_and_missing_rows(gpu_lib):
    pool = torch.zeros((4, 8, 2, 1, 8), dtype=torch.bfloat16, device="cuda")
    for at, width in ((0, 40), (1, 19), (8, 24)):
        x = torch.randn(5, width, device="cuda").bfloat16()[:, at:at + 16]
        rows = dev_i32([3, -1, 31, 32, 1 << 30])
        pool.zero_()
        ops.cache_write(x, rows, pool)
        want = torch.zeros(32, 16, dtype=torch.bfloat16, device="cuda")
        want[3], want[31] = x[0], x[2]
        assert torch.equal(pool.view(32, 16), want)
    ops.cache_write(x[:0], rows[:0], pool)
    assert torch.equal(pool.view(32, 16), want)


def test_copy_between_pools(gpu_lib):
    for dtype, row in ((torch.bfloat16, 24), (torch.bfloat16, 3), (torch.uint8, 5), (torch.float32, 2048)):
        a = torch.arange(2 * 6 * 4 * row, device="cuda").view(2, 6, 4, row).remainder(97).to(dtype)
        b = torch.zeros((2, 9, 4, row), dtype=dtype, device="cuda")
        ops.cache_copy(dev_i32([5, 0, 6, -1, 2]), dev_i32([8, 1, 2, 3, 9]), a, b)
        want = torch.zeros_like(b)
        want[:, 8], want[:, 1] = a[:, 5], a[:, 0]
        assert torch.equal(b, want)
        ops.cache_copy(dev_i32([0, 1]), dev_i32([4, 5]), a)
        assert torch.equal(a[:, 4], a[:, 0]) and torch.equal(a[:, 5], a[:, 1])


def test_compact_past_32_bits(gpu_lib):
    pool, table, lens, refs = ops.cache_pool(2, 40000, 64, 4, 128, slots=2, table_width=4,
                                             dtype=torch.uint8)   # 2.6 GB a layer
    assert pool.numel() > 1 << 32
    table[0, :2] = dev_i32([39999, 20000])
    lens[0] = 100
    refs[39999] = refs[20000] = 1
    pool[:, 39999], pool[:, 20000] = 3, 4
    pool[1, 39999] = 5
    assert ops.cache_check(ops.cache_compact(table, lens, refs, pool)) == 2
    assert table[0].tolist() == [1, 0, -1, -1] and refs.sum().item() == 2
    assert bool((pool[0, 1] == 3).all()) and bool((pool[1, 1] == 5).all())
    assert bool((pool[:, 0] == 4).all())


def test_captured_steps(gpu_lib):
    # A captured append (fixed slots, one row each) replayed: the cache grows as with eager calls.
    a, b = (ops.cache_pool(1, 64, 4, 1, 8, slots=8, table_width=8) for _ in range(2))
    slots, off = dev_i32([3, 0, 6]), dev_i32([0, 1, 2, 3])
    x = torch.randn(3, 16, device="cuda").bfloat16()

    def step(c):
        pool, table, lens, refs = c
        rows, status = ops.cache_reserve(slots, off, 3, table, lens, refs, 4)
        ops.cache_write(x, rows, pool[0])
        return status

    step(a), step(b)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(a)
    for _ in range(9):
        g.replay()
        ops.cache_check(step(b))
        assert all(torch.equal(s, t) for s, t in zip(a, b))


def test_python_path_gives_the_same(gpu_lib, monkeypatch):
    one, two = Pair(2, 30, 4, 8, 6), Pair(2, 30, 4, 8, 6)

    def life(c):
        c.append([1, 4], [9, 6])
        c.fork([1, 4], [0, 5])
        c.free([1])
        c.compact()
        c.check()
    life(one)
    monkeypatch.setattr(ops, "_binding", ops._PythonPath())
    life(two)
    assert all(torch.equal(s, t) for s, t in zip(one.dev, two.dev))
