"""GPU: page tables, lengths and maps of a step's tokens made on the device, against the same written out entry by entry."""
import pytest
import torch

from tests.tree_util import Pool

pytestmark = pytest.mark.gpu


def _mp():
    from paper_2506_13059_amd import binding as mp
    return mp


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda").reshape(len(x), *([-1] if x and isinstance(x[0], list) else []))


class OnDevice:
    def __init__(self, p):
        self.table, self.kv_len, self.q_start, self.stack, self.n_free = _i32(p.table), _i32(p.kv_len), _i32(p.q_start), _i32(p.stack), _i32([p.n_free])
        self.pool = _mp().MpPagePool(self.table, self.kv_len, self.q_start, self.stack, self.n_free, p.page)

    def same_as(self, p):
        assert self.n_free.tolist() == [p.n_free]
        assert self.kv_len.tolist() == p.kv_len and self.q_start.tolist() == p.q_start
        assert self.stack.tolist() == p.stack
        assert self.table.tolist() == p.table

    def step(self, p, come, keep, rows):
        granted, sequence, positions = (torch.full((n,), 77, dtype=torch.int32, device="cuda") for n in (len(come), rows, rows))
        slots = torch.full((rows,), 77, dtype=torch.int64, device="cuda")
        self.pool.mp_paged_reserve(_i32(come), None if keep is None else _i32(keep), granted, sequence, positions, slots)
        torch.cuda.synchronize()
        want = p.step(come, keep, rows)
        self.same_as(p)
        assert (granted.tolist(), sequence.tolist(), positions.tolist(), slots.tolist()) == tuple(list(w) for w in want)


@pytest.mark.parametrize("page,columns,n_pages,seqs,most,rows", [
    (16, 4, 9, 1, 30, 40), (1, 50, 100, 3, 20, 64), (16, 40, 130, 9, 200, 700), (64, 16, 500, 70, 90, 3000), (16, 60, 3000, 65, 500, 6000), (1024, 3, 20, 12, 1500, 5000),
    (32, 40, 5000, 1300, 60, 20000), (16, 200, 40000, 300, 3000, 100), (8, 3, 2000, 1024, 9, 4097), (16, 700, 12000, 17, 11000, 90000),
])
def test_steps(page, columns, n_pages, seqs, most, rows):
    print(f"case page={page} columns={columns} n_pages={n_pages} seqs={seqs} most={most} rows={rows}", flush=True)
    g = torch.Generator().manual_seed(page * 1000 + seqs)
    draw = lambda hi: torch.randint(0, hi, (seqs,), generator=g).tolist()      # noqa: E731
    p = Pool(page, columns, n_pages, seqs, seed=seqs)
    d = OnDevice(p)
    for step in range(6):
        # new ones, some of none, some of more than a table has room for; then some go, some lose their newest tokens
        come = [n - 2 if step % 3 else n for n in draw(most + 2)] if step % 2 == 0 else [n % 5 for n in draw(most + 2)]
        keep = None if step in (0, 3) else [k + 3 - (5 * r) % 17 if r % 4 else 0 for k, r in zip(p.kv_len, draw(1000))]
        d.step(p, come, keep, rows)


def test_entries_that_name_no_page_have_none_to_give():
    p = Pool(16, 12, 40, 4, seed=1, have=[100, 20, 0, 64])
    p.table[0][2], p.table[0][5], p.table[3][3], p.table[1][9] = -1, 40, -7, 3
    d = OnDevice(p)
    d.step(p, [5, 1, 3, 0], [17, 20, 0, 0], 20)
    # ... and lengths past the table's room count as that much, those below zero as none
    p.kv_len[1], p.kv_len[2] = 10 ** 6, -5
    d.kv_len.copy_(_i32(p.kv_len))
    d.step(p, [-3, 4, 2, 2 ** 31 - 1], [-1, 30, 9, 50], 20)


def test_pages_that_come_twice_stay_within_the_stack():
    p = Pool(4, 6, 6, 3, seed=1, have=[24, 0, 0])
    p.table[1], p.kv_len[1] = list(p.table[0]), 24
    d = OnDevice(p)
    d.step(p, [0, 0, 3], [0, 0, 0], 5)
    p.n_free, d.n_free[0] = 6, 900                 # (a count past the stack's end)
    p.stack = [3, 1, 0, 2, 4, 5]
    d.stack.copy_(_i32(p.stack))
    d.step(p, [1, 1, 1], [0, 0, 0], 5)


def test_no_sequences_and_results_left_out():
    mp = _mp()
    p = Pool(16, 4, 5, 2, seed=3)
    d = OnDevice(p)
    d.pool.mp_paged_reserve(_i32([20, 40]))
    p.step([20, 40])
    d.same_as(p)
    pos = torch.zeros(9, dtype=torch.int32, device="cuda")
    d.pool.mp_paged_reserve(_i32([3, 1]), positions=pos)
    _, _, want, _ = p.step([3, 1], None, 9)
    d.same_as(p)
    assert pos.tolist() == want
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    start, slots = torch.full((1,), 9, dtype=torch.int32, device="cuda"), torch.zeros(5000, dtype=torch.int64, device="cuda")
    mp.MpPagePool(none.view(0, 4), none, start, d.stack, d.n_free, 16).mp_paged_reserve(none, slots=slots)
    assert start.tolist() == [0] and (slots == -1).all()
    d.same_as(p)


def test_captured_steps():
    """A step captured once and replayed while the host changes what comes and goes."""
    seqs, rows = 33, 4500
    p = Pool(16, 30, 700, seqs, seed=5)
    d = OnDevice(p)
    come, keep, granted = (torch.zeros(seqs, dtype=torch.int32, device="cuda") for _ in range(3))
    sequence, positions = (torch.zeros(rows, dtype=torch.int32, device="cuda") for _ in range(2))
    slots = torch.zeros(rows, dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        d.pool.mp_paged_reserve(come, keep, granted, sequence, positions, slots)
    g = torch.Generator().manual_seed(2)
    for _ in range(5):
        n, k = torch.randint(0, 140, (seqs,), generator=g).tolist(), [max(0, x - int(torch.randint(0, 60, (1,), generator=g))) for x in p.kv_len]
        come.copy_(_i32(n))
        keep.copy_(_i32(k))
        graph.replay()
        torch.cuda.synchronize()
        want = p.step(n, k, rows)
        d.same_as(p)
        assert (granted.tolist(), sequence.tolist(), positions.tolist(), slots.tolist()) == tuple(list(w) for w in want)
