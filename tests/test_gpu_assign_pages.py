"""Page tables, the pool and slot maps from request lengths, against a plain list form; whole numbers, bit for bit."""
import random

import pytest
import torch

import round_ops
from paper_2607_27735_b200 import binding

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Server:
    """Lengths, tables and pool of a batch on both sides."""

    def __init__(self, batch, ps, max_pages, n_pages, seed=0):
        self.ps, self.n_pages, self.rng = ps, n_pages, random.Random(seed)
        pages = list(range(n_pages))
        self.rng.shuffle(pages)
        self.table = [[-7] * max_pages for _ in range(batch)]
        self.held, self.pool, self.n_free, self.length = [0] * batch, pages, n_pages, [0] * batch
        self.d_table, self.d_held = _i32(self.table).view(batch, max_pages), _i32(self.held)
        self.d_pool, self.d_free = _i32(self.pool), _i32([n_pages])
        self.ws = binding.alloc_workspace(binding.pages_workspace_bytes(), "cuda")

    def step(self, first, new, max_rows, want=0):
        got = binding.spec_assign_pages(_i32(first), _i32(new), self.ps, self.d_table, self.d_held, self.d_pool, self.d_free,
                                        max_rows=max_rows, workspace=self.ws)
        ref = round_ops.assign_pages(first, new, self.ps, self.table, self.held, self.pool, self.n_free, max_rows, self.n_pages)
        assert binding.read_status(self.ws) == want
        if ref is None:
            assert want != 0
            assert got[0].tolist() == [0] * (len(new) + 1) and got[1].tolist() == [0] * max_rows and got[2].tolist() == [-1] * max_rows
        else:
            cu, positions, slots, self.table, self.held, self.pool, self.n_free = ref
            assert got[0].tolist() == cu and got[1].tolist() == positions and got[2].tolist() == slots
        assert self.d_table.tolist() == self.table and self.d_held.tolist() == self.held
        assert self.d_pool.tolist() == self.pool and self.d_free.tolist() == [self.n_free]
        return got


@pytest.mark.parametrize("batch,ps,max_pages", [(1, 16, 40), (1, 1, 50), (7, 24, 9), (33, 64, 5), (300, 8, 12), (2048, 16, 3)])
def test_many_steps_match_the_plain_form(batch, ps, max_pages):
    s = Server(batch, ps, max_pages, n_pages=batch * max_pages, seed=batch + ps)
    cap = max_pages * ps
    for step in range(12):
        first, new = [], []
        for b in range(batch):
            what = s.rng.random()
            t = s.length[b]
            if what < 0.1:
                f, n = 0, 0                                    # ended
            elif what < 0.2:
                f, n = 0, s.rng.randint(0, cap)                # another request in its place
            elif what < 0.3:
                f = n = t                                      # nothing new
            elif what < 0.4:
                f, n = min(t, cap), s.rng.randint(0, t)        # rolled back: no rows
            else:
                f, n = t, min(cap, t + s.rng.randint(1, 2 * ps))
            first.append(f), new.append(n)
            s.length[b] = n
        rows = sum(max(n - f, 0) for f, n in zip(first, new))
        s.step(first, new, rows + (step % 3) * 5)


def test_a_page_given_back_is_taken_again_in_the_same_call():
    s = Server(3, 4, 6, n_pages=8)
    s.step([0, 0, 0], [24, 8, 0], 32)            # the pool is empty now
    s.step([24, 8, 0], [9, 8, 11], 20)           # three pages come back, three are taken
    s.step([9, 8, 11], [9, 24, 11], 20, want=-7)  # none come back, four are wanted
    s.step([9, 8, 11], [0, 24, 0], 20)           # six come back


def test_errors_change_nothing():
    s = Server(3, 4, 6, n_pages=8)
    s.step([0, 0, 0], [13, 5, 1], 19)
    s.step([13, 5, 1], [13, 5, 24], 23, want=-7)       # one page is left, five wanted
    s.step([13, 5, 1], [13, 5, 25], 40, want=-6)       # beyond the table
    s.step([13, -1, 1], [13, 5, 2], 40, want=-6)
    s.step([13, 5, 1], [13, -5, 2], 40, want=-6)
    s.step([13, 5, 1], [16, 5, 2], 3, want=-6)         # four rows, room for three
    s.d_held[1] = 9                                    # more pages than a table has
    s.held[1] = 9
    s.step([13, 5, 1], [13, 5, 2], 4, want=-6)
    s.d_held[1] = s.held[1] = 2
    s.step([13, 5, 1], [0, 5, 24], 23)                 # with the first one gone it fits


def test_numbers_that_are_no_pages_are_reported_and_give_no_slot():
    s = Server(2, 4, 6, n_pages=8)
    s.pool[7] = 8
    s.d_pool[7] = 8
    s.step([0, 0], [4, 3], 7, want=-6)
    s.pool[5] = -3
    s.d_pool[5] = -3
    s.step([4, 3], [4, 5], 2, want=-6)


def test_no_sequences_and_no_rows():
    ws = binding.alloc_workspace(binding.pages_workspace_bytes(), "cuda")
    empty = torch.empty(0, dtype=torch.int32, device="cuda")
    pool, n_free = _i32([2, 1, 0]), _i32([3])
    cu, pos, slots, _ = binding.spec_assign_pages(empty, empty, 16, torch.empty(0, 4, dtype=torch.int32, device="cuda"), empty, pool,
                                                  n_free, max_rows=5, workspace=ws)
    assert cu.tolist() == [0] and slots.tolist() == [-1] * 5 and pos.tolist() == [0] * 5 and n_free.tolist() == [3]
    s = Server(2, 16, 4, 8)
    s.step([5, 7], [5, 7], 0)


def test_replayed_graph_goes_on_from_the_state_it_finds():
    s = Server(5, 8, 30, 150)
    first, new = _i32([0] * 5), _i32([3] * 5)
    cu = torch.empty(6, dtype=torch.int32, device="cuda")
    pos, slots = (torch.empty(64, dtype=torch.int32, device="cuda") for _ in range(2))

    def call():
        binding.spec_assign_pages(first, new, 8, s.d_table, s.d_held, s.d_pool, s.d_free, cu_rows=cu, positions=pos, slots=slots,
                                  workspace=s.ws)

    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    f, n = [0] * 5, [3, 17, 8, 9, 1]
    for _ in range(6):
        first.copy_(_i32(f))
        new.copy_(_i32(n))
        g.replay()
        ref = round_ops.assign_pages(f, n, 8, s.table, s.held, s.pool, s.n_free, 64, 150)
        assert cu.tolist() == ref[0] and pos.tolist() == ref[1] and slots.tolist() == ref[2]
        _, _, _, s.table, s.held, s.pool, s.n_free = ref
        f, n = n, [t + i + 2 for i, t in enumerate(n)]
    assert s.d_table.tolist() == s.table and s.d_free.tolist() == [s.n_free]


def test_shapes_and_types_are_checked():
    s = Server(2, 16, 4, 8)
    with pytest.raises(ValueError):
        binding.spec_assign_pages(_i32([0]), _i32([1, 2]), 16, s.d_table, s.d_held, s.d_pool, s.d_free, max_rows=4)
    with pytest.raises(ValueError):
        binding.spec_assign_pages(_i32([0, 0]).long(), _i32([1, 2]), 16, s.d_table, s.d_held, s.d_pool, s.d_free, max_rows=4)
    with pytest.raises(ValueError):
        binding.spec_assign_pages(_i32([0, 0]), _i32([1, 2]), 16, s.d_table, s.d_held, s.d_pool, s.d_free)
    with pytest.raises(binding.SpecError):
        binding.spec_assign_pages(_i32([0, 0]), _i32([1, 2]), 0, s.d_table, s.d_held, s.d_pool, s.d_free, max_rows=4)
    with pytest.raises(binding.SpecError):  # more sequences than a call takes
        big = Server(2049, 16, 1, 1)
        binding.spec_assign_pages(_i32([0] * 2049), _i32([0] * 2049), 16, big.d_table, big.d_held, big.d_pool, big.d_free, max_rows=4)
