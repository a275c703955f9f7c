"""The plan of a paged 8-bit cache's step, where many pages change hands and long slot maps are filled: equal to the oracle's book, entry by
entry.  (Pages alone, no tokens.)"""
import numpy as np
import pytest

from oracle import cache_oracle as co

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    import paper_2502_18137_amd as sp
    return sp


class Pair:
    """a cache's book and the oracle's"""

    def __init__(self, sp, rows, n_pages, max_blocks, seed):
        import torch
        self.sp, self.torch, self.rng = sp, torch, np.random.default_rng(seed)
        self.cache = sp.SpargeCache(rows, 1, 64, n_pages, max_blocks)
        free = self.rng.permutation(n_pages).astype(np.int32)
        self.cache.free_pages.copy_(torch.from_numpy(free))
        self.book = co.Book(rows, n_pages, max_blocks, free.tolist())

    def step(self, new, release=None, pad=0):
        n = int(np.sum(new)) + pad
        t = lambda x, dt: self.torch.tensor(np.asarray(x), dtype=dt, device="cuda")
        plan = self.sp.sparge_cache_plan(self.cache, t(new, self.torch.int32), n,
                                         None if release is None else t(release, self.torch.uint8))
        want = self.book.plan([int(x) for x in new], None if release is None else [int(x) for x in release], n)
        for name, w in zip(("cu", "slots", "req", "status"), want):
            assert np.array_equal(getattr(plan, name).cpu().numpy(), np.asarray(w)), name
        assert self.cache.length.tolist() == self.book.length
        n_free = int(self.cache.n_free)
        assert n_free == len(self.book.free) and self.cache.free_pages[:n_free].tolist() == self.book.free
        table = self.cache.table.cpu().numpy()
        for r, length in enumerate(self.book.length):
            blocks = -(-length // 64)
            assert np.array_equal(table[r, :blocks], self.book.table[r, :blocks]), r
        return want[3]


@pytest.mark.parametrize("rows", [300, 1000])
def test_thousands_of_pages_change_hands(sp, rows):
    """more than 8192 taken at once; given up and taken in one step, more of the one, more of the other, rows over the joints"""
    each = 9500 * 64 // rows                                     # tokens of a row for about 9500 pages
    some = lambda: m.rng.integers(each - 60, each + 60, rows)
    m = Pair(sp, rows, 22000, -(-(3 * each) // 64), rows)
    assert m.step(some())[0] == 0                                # 9500 taken
    assert m.step(some(), np.ones(rows))[0] == 0                 # 9500 given up, 9500 taken: those just given up
    assert m.step(some(), m.rng.random(rows) < 0.3)[0] == 0      # 2850 given up, 9500 taken
    assert m.step(np.ones(rows, int), np.ones(rows))[0] == 0     # 15000 given up, one page a row taken
    assert m.step(some() * (m.rng.random(rows) < 0.9))[0] == 0
    assert m.step(np.zeros(rows, int), np.ones(rows))[0] == 0    # everything given up
    assert int(m.cache.n_free) == 22000


def test_long_slot_maps_onto_rows_in_use(sp):
    """more than 4096 slots, which a launch of its own fills: rows that hold tokens, rows given up in this step, rows that add nothing"""
    m = Pair(sp, 50, 1200, 40, 3)
    m.step(m.rng.integers(0, 200, 50))
    for k in range(3):
        new = m.rng.integers(60, 300, 50) * (m.rng.random(50) < 0.8)
        assert new.sum() > 4096
        assert m.step(new, m.rng.random(50) < 0.3, pad=(0, 1, 700)[k])[0] == 0


@pytest.mark.parametrize("n_slots", [4096, 4097, 5000, 20000])
def test_a_long_step_that_does_not_fit(sp, n_slots):
    """slots and rows of -1, nothing changed, whoever fills the slot map"""
    m = Pair(sp, 40, 100, 80, n_slots)
    assert m.step([60] * 40)[0] == 0
    fits = [n_slots // 40] * 40
    assert m.step(fits, pad=n_slots - sum(fits))[0] & sp.CACHE_NO_PAGES
    assert m.step([0] * 39 + [n_slots], pad=0)[0] & (sp.CACHE_NO_PAGES | sp.CACHE_ROW_FULL)
    assert m.step([1] * 40, pad=n_slots - 40)[0] == 0
