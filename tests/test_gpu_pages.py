"""Pages of a cache against a model in plain Python, state for state and byte for byte."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _ralm():
    import paper_2401_14021_b200 as ralm
    return ralm


class Model:
    """The contract of the page calls, row by row. pages[l][p] is the content of a page."""

    def __init__(self, layers, pages, rows, max_pages, page_size):
        self.ps, self.max_pages = page_size, max_pages
        self.table = [[] for _ in range(rows)]
        self.lengths = [0] * rows
        self.refs = [0] * pages
        self.pages = [[bytes()] * pages for _ in range(layers)]

    def need(self, length):
        return -(-length // self.ps)

    def resize(self, new):
        if any(not 0 <= n <= self.max_pages * self.ps for n in new):
            return 1
        refs = list(self.refs)
        for row, n in enumerate(new):
            for p in self.table[row][self.need(n):]:
                refs[p] -= 1
        writers = {}
        for row, n in enumerate(new):
            if n > self.lengths[row] and self.lengths[row] % self.ps:
                writers.setdefault(self.table[row][self.lengths[row] // self.ps], []).append(row)
        cow = set()
        for page, rows in writers.items():
            if refs[page] > 1:
                cow.update(rows[1:] if len(rows) == refs[page] else rows)
        free = [p for p, r in enumerate(refs) if r == 0]
        demand = sum(max(self.need(n) - self.need(self.lengths[r]), 0) + (r in cow) for r, n in enumerate(new))
        if demand > len(free):
            return 2
        take = iter(free)
        moves = []
        for row, n in enumerate(new):
            t = self.table[row] = self.table[row][:self.need(n)] if n < self.lengths[row] else self.table[row]
            if row in cow:
                at = self.lengths[row] // self.ps
                page = next(take)
                moves.append((t[at], page))
                refs[page] = 1
                t[at] = page
            while len(t) < self.need(n):
                page = next(take)
                refs[page] = 1
                t.append(page)
        for old, page in moves:
            refs[old] -= 1
            for layer in self.pages:
                layer[page] = layer[old]
        self.refs, self.lengths = refs, list(new)
        return 0

    def fork(self, src, dst):
        rows = len(self.table)
        if len(set(dst)) < len(dst) or set(src) & set(dst) or any(not 0 <= r < rows for r in src + dst):
            return 1
        for d in dst:
            for p in self.table[d]:
                self.refs[p] -= 1
        for s, d in zip(src, dst):
            self.table[d], self.lengths[d] = list(self.table[s]), self.lengths[s]
            for p in self.table[d]:
                self.refs[p] += 1
        return 0

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        movers = [p for p, r in enumerate(self.refs) if r > 0 and p >= live]
        holes = [p for p, r in enumerate(self.refs) if r == 0 and p < live]
        to = dict(zip(movers, holes))
        for a, b in to.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
            for layer in self.pages:
                layer[b] = layer[a]
        self.table = [[to.get(p, p) for p in row] for row in self.table]
        return live


def make(layers, pages, rows, max_pages, page_size, page_bytes=48, seed=0):
    ralm = _ralm()
    cache = ralm.Pages.allocate(layers, pages, page_bytes, rows, max_pages, page_size, device=DEV)
    g = torch.Generator(DEV).manual_seed(seed)
    cache.pool.copy_(torch.randint(0, 256, cache.pool.shape, generator=g, device=DEV, dtype=torch.uint8))
    model = Model(layers, pages, rows, max_pages, page_size)
    host = cache.pool.cpu().numpy()
    model.pages = [[host[l, p].tobytes() for p in range(pages)] for l in range(layers)]
    return cache, model


def same(cache, model):
    table = cache.table.tolist()
    assert [[p for p in row if p >= 0] for row in table] == model.table
    assert all(p == -1 for row, t in zip(table, model.table) for p in row[len(t):])
    assert cache.lengths.tolist() == model.lengths
    assert cache.refs.tolist() == model.refs
    host = cache.pool.cpu().numpy()
    assert all(host[l, p].tobytes() == b for l, layer in enumerate(model.pages) for p, b in enumerate(layer))


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("seed,layers,pages,rows,max_pages,page_size", [(1, 2, 40, 6, 10, 4), (2, 1, 9, 5, 4, 3), (3, 3, 64, 17, 8, 1),
                                                                        (4, 1, 5000, 40, 200, 16), (5, 1, 3000, 1500, 4, 2)])
def test_random_calls(seed, layers, pages, rows, max_pages, page_size):
    rng = random.Random(seed)
    cache, model = make(layers, pages, rows, max_pages, page_size, seed=seed)
    cap = max_pages * page_size
    refused = 0
    for step in range(40 if rows < 1000 else 12):
        kind = rng.random()
        if kind < 0.6:
            new = [max(0, min(cap, n + rng.randint(-page_size * 2, page_size * 3))) if rng.random() < 0.7 else n for n in model.lengths]
            want = model.resize(new)
            cache.resize(i32(new))
        elif kind < 0.85:
            some = rng.sample(range(rows), rng.randint(1, rows // 2) * 2)
            src, dst = some[::2], some[1::2]
            if rng.random() < 0.3:
                src = [src[0]] * len(dst)          # one row forked many times
            want = model.fork(src, dst)
            cache.fork(i32(src), i32(dst))
        else:
            want = 0
            live = model.compact()
            assert cache.compact().item() == live
        assert cache.device_status() == want
        refused += want != 0
        same(cache, model)
    assert refused < 40


def test_all_holders_of_a_page_grow():
    cache, model = make(1, 12, 4, 4, 4)
    for new in ([6, 0, 0, 0],):
        assert model.resize(new) == 0
        cache.resize(i32(new))
    model.fork([0, 0, 0], [1, 2, 3])
    cache.fork(i32([0, 0, 0]), i32([1, 2, 3]))
    same(cache, model)
    model.resize([7, 7, 7, 7])                     # the lowest row keeps the page
    cache.resize(i32([7, 7, 7, 7]))
    same(cache, model)
    assert model.table[0][1] == 1 and cache.refs[1].item() == 1
    # rolled back into the shared first page, then grown again: it is copied, not written
    model.resize([3, 3, 0, 8])
    cache.resize(i32([3, 3, 0, 8]))
    model.resize([5, 3, 0, 8])
    cache.resize(i32([5, 3, 0, 8]))
    same(cache, model)
    assert model.table[0][0] != 0


def test_too_few_pages_change_nothing():
    cache, model = make(1, 6, 3, 8, 2)
    assert model.resize([4, 4, 0]) == 0
    cache.resize(i32([4, 4, 0]))
    assert model.resize([2, 4, 12]) == 2           # the page that row 0 would give back does not suffice
    cache.resize(i32([2, 4, 12]))
    assert cache.device_status() == 2 and cache.device_status() == 0
    same(cache, model)
    assert model.resize([0, 4, 8]) == 0            # pages given back in the call are taken in the call
    cache.resize(i32([0, 4, 8]))
    assert cache.device_status() == 0
    same(cache, model)


def test_lengths_and_rows_that_are_refused_on_the_device():
    cache, model = make(1, 6, 3, 2, 4)
    for new in ([-1, 0, 0], [0, 9, 0], [0, 0, 2 ** 31 - 1]):
        cache.resize(i32(new))
        assert cache.device_status() == 1
        same(cache, model)
    cache.resize(i32([5, 0, 0]))
    model.resize([5, 0, 0])
    for src, dst in (([0], [3]), ([-1], [1]), ([0, 0], [1, 1]), ([0, 1], [1, 2]), ([0], [0])):
        cache.fork(i32(src), i32(dst))
        assert cache.device_status() == 1
        same(cache, model)


def test_copy_between_pools():
    ralm = _ralm()
    a, _ = make(3, 9, 2, 4, 4, page_bytes=16 * 1030, seed=1)
    b, _ = make(3, 5, 2, 4, 4, page_bytes=16 * 1030, seed=2)
    want = b.pool.clone()
    want[:, [4, 0, 2]] = a.pool[:, [1, 8, 3]]
    b.copy_from(a, i32([1, 8, 3]), i32([4, 0, 2]))
    assert torch.equal(b.pool, want) and b.device_status() == 0
    b.copy_from(a, i32([9, 1, -1, 2]), i32([1, 5, 3, 3]))          # pairs outside the pools are left out
    want[:, 3] = a.pool[:, 2]
    assert torch.equal(b.pool, want) and b.device_status() == 1
    c, _ = make(2, 5, 2, 4, 4, page_bytes=16 * 1030)
    with pytest.raises(ralm.RalmError):
        c.copy_from(a, i32([0]), i32([0]))                          # other layers


def test_bookkeeping_without_a_pool():
    ralm = _ralm()
    _, table, lengths, refs = ralm.Pages.tensors(1, 8, 16, 2, 4, DEV)
    pages = ralm.Pages(None, table, lengths, refs, page_size=4)
    pages.resize(i32([9, 4]))
    assert table.tolist() == [[0, 1, 2, -1], [3, -1, -1, -1]]
    pages.resize(i32([0, 4]))
    assert pages.compact().item() == 1 and table[1, 0].item() == 0


def test_offsets_beyond_32_bits():
    cache, _ = make(2, 70, 2, 40, 4, page_bytes=64)
    del cache
    ralm = _ralm()
    page_bytes = 1 << 26
    big = ralm.Pages.allocate(1, 70, page_bytes, 1, 70, 4, device=DEV)          # 4.7 GB
    big.resize(i32([70 * 4]))
    big.pool[0, 69, -16:] = 123
    big.pool[0, 0] = 0
    big.copy_from(big, i32([69]), i32([0]))
    assert (big.pool[0, 0, -16:] == 123).all() and big.device_status() == 0


def test_refusals():
    ralm = _ralm()
    cache, _ = make(1, 6, 3, 2, 4)
    with pytest.raises(TypeError):
        cache.resize(i32([1, 2]))
    with pytest.raises(TypeError):
        cache.resize(torch.tensor([1, 2, 3], device=DEV))
    with pytest.raises(TypeError):
        cache.fork(i32([0]), i32([1, 2]))
    with pytest.raises(ralm.RalmError):
        cache.fork(i32([0, 0, 0, 0]), i32([1, 2, 1, 2]))            # more pairs than rows
    with pytest.raises(TypeError):
        ralm.Pages(cache.pool, cache.table.long(), cache.lengths, cache.refs, 4)
    with pytest.raises(TypeError):
        ralm.Pages(cache.pool[0], cache.table, cache.lengths, cache.refs, 4)
    odd = torch.zeros((1, 6, 24), dtype=torch.uint8, device=DEV)
    with pytest.raises(ralm.RalmError):                              # page bytes are multiples of 16
        ralm.Pages(odd, cache.table, cache.lengths, cache.refs, 4).resize(i32([1, 0, 0]))
