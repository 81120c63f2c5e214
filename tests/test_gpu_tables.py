"""Block tables brought up to date on the GPU against the same on lists (q4_reference.assign), and the rows that new tokens go to."""
import random

import pytest
import torch

import q4_reference as Q

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def sqa():
    from paper_2404_04793_amd import binding
    return binding


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Pool:
    """A table and its free list on the device, and the same on lists."""

    def __init__(self, B, Hkv, capacity, n_blocks, rng):
        self.B, self.Hkv, self.capacity, per = B, Hkv, capacity, -(-capacity // 16)
        self.free = rng.sample(range(n_blocks), n_blocks)
        self.rows, self.has = [[-1] * per for _ in range(B * Hkv)], [0] * B
        self.table, self.held = ints(self.rows), ints(self.has)
        self.free_ids, self.count, self.status = ints(self.free), ints([n_blocks]), ints([0])

    def step(self, sqa, tokens):
        self.status.zero_()
        sqa.block_assign(self.table, ints(tokens), self.held, self.free_ids, self.count, self.capacity, self.status)
        short = Q.assign(self.rows, tokens, self.has, self.free, self.capacity, self.Hkv)
        assert int(self.count) == len(self.free) and self.free_ids[:len(self.free)].tolist() == self.free
        assert self.held.tolist() == self.has and self.table.tolist() == self.rows
        assert int(self.status) == (6 if short else 0)
        return short


@pytest.mark.parametrize("B,Hkv,capacity,share", [(1, 1, 16, 1.0), (1, 8, 500, 1.0), (5, 3, 100, 0.6), (64, 8, 4096, 0.5), (300, 2, 333, 0.4), (1500, 1, 64, 0.7),
                                                  (2049, 1, 30, 1.0)])
def test_a_loop_of_joining_growing_and_leaving(sqa, B, Hkv, capacity, share):
    """As a serving loop goes: some leave, some join, the others grow, now and then the list is too short."""
    rng = random.Random(B * 7 + Hkv)
    per = -(-capacity // 16)
    pool = Pool(B, Hkv, capacity, max(1, int(B * Hkv * per * share)), rng)
    now = [0] * B
    for step in range(12):
        for b in range(B):
            r = rng.random()
            now[b] = 0 if r < 0.15 else (rng.randrange(capacity + 40) if r < 0.3 else now[b] + rng.choice([1, 1, 1, 17, 40]))
        pool.step(sqa, [-1 if rng.random() < 0.05 else n for n in now])
    pool.step(sqa, [0] * B)
    assert len(pool.free) == pool.free_ids.numel() and sorted(pool.free) == list(range(len(pool.free)))


def test_a_list_that_is_too_short(sqa):
    """Those in front get theirs, the first that does not fit gets nothing and none behind it does, until blocks come back."""
    pool = Pool(5, 2, 160, 30, random.Random(1))
    assert not pool.step(sqa, [64, 0, 33, 16, 0])     # 8 + 6 + 2 of 30
    assert pool.step(sqa, [64, 150, 80, 17, 1])       # 20 for the second: more than 14
    assert pool.has == [4, 0, 3, 1, 0]
    assert pool.step(sqa, [64, 80, 80, 17, 1])        # 10 for the second, 4 for the third, then nothing is left
    assert pool.has == [4, 5, 5, 1, 0] and not pool.free
    assert pool.step(sqa, [0, 80, -1, 17, 160])       # 8 come back: 2 for the fourth, 20 are too many for the last
    assert pool.has == [0, 5, 5, 2, 0]
    assert pool.step(sqa, [160, 160, 160, 160, 160])


def test_most_sequences(sqa):
    rng = random.Random(3)
    pool = Pool(8192, 1, 32, 12000, rng)
    for _ in range(3):
        pool.step(sqa, [rng.randrange(40) for _ in range(8192)])


def test_lists_that_contradict_themselves(sqa):
    """A count that is none, one that leaves no room for what comes back, and blocks that a row cannot hold: reported, nothing moved."""
    rng = random.Random(5)
    for count, held in ((-1, [2, 1]), (9, [2, 1]), (10, [2, 1])):
        p = Pool(2, 2, 64, 9, rng)
        p.count.fill_(count)
        p.held.copy_(ints(held))
        before = [x.clone() for x in (p.table, p.held, p.free_ids, p.count)]
        sqa.block_assign(p.table, ints([0, 0]), p.held, p.free_ids, p.count, 64, p.status)
        assert int(p.status) == 8 and all(torch.equal(a, b) for a, b in zip(before, (p.table, p.held, p.free_ids, p.count)))
    p = Pool(3, 2, 64, 20, rng)
    p.held.copy_(ints([5, 0, -1]))
    sqa.block_assign(p.table, ints([64, 20, 64]), p.held, p.free_ids, p.count, 64, p.status)
    assert int(p.status) == 8 and p.held.tolist() == [5, 2, -1] and int(p.count) == 16
    assert bool((p.table[:2] == -1).all()) and bool((p.table[4:] == -1).all()) and bool((p.table[2:4, :2] >= 0).all())


@pytest.mark.parametrize("capacity,sink", [(100, 0), (33, 0), (33, 4), (16, 15)])
@pytest.mark.parametrize("blocked", [False, True])
def test_map(sqa, capacity, sink, blocked):
    rng = random.Random(8)
    B, Hkv, per = 6, 3, -(-capacity // 16) + 1
    table = [[rng.randrange(1000) for _ in range(per)] for _ in range(B * Hkv)]
    table[4][0] = -1
    for T in (1, 5, 16, 70):
        new, before = [T, T, 0, max(1, T // 2), 1, T + 1], [0, 31, 5, 90, -1, 3]
        status = ints([0])
        out = torch.full((B, Hkv, T), 77, dtype=torch.int32, device=DEV)
        got = sqa.slot_map(ints(table) if blocked else None, capacity, T, 0, sink, out=out,
                           opts=sqa.batch_opts(prompt_len=ints(new), new_pos_seq=ints(before), status=status)).tolist()
        seen = 0
        for b in range(B):
            many = new[b] <= T and before[b] >= 0 and new[b] > capacity - sink and before[b] + new[b] > capacity
            n = 0 if new[b] > T or before[b] < 0 or many else new[b]
            seen |= (2 if new[b] > T else 0) | (6 if many else 0)
            for h in range(Hkv):
                u = b * Hkv + h
                for t in range(T):
                    want = -1
                    if t < n:
                        s = Q.slot_of(before[b] + t, capacity, sink)
                        want = u * capacity + s if not blocked else (-1 if table[u][s // 16] < 0 else table[u][s // 16] * 16 + s % 16)
                    assert got[b][h][t] == want, (T, b, h, t)
        assert int(status) in ((2,) if seen == 2 else (2, 6))


def test_rows_beyond_32_bits(sqa):
    status = ints([0])
    opts = sqa.batch_opts(status=status)
    got = sqa.slot_map(ints([[2 ** 27, 2 ** 27 - 1]]), 32, 32, out=torch.zeros(1, 1, 32, dtype=torch.int32, device=DEV), opts=opts)
    assert int(status) == 2 and bool((got[0, 0, :16] == -1).all()) and got[0, 0, 16:].tolist() == list(range(2 ** 31 - 16, 2 ** 31))
    status.zero_()
    got = sqa.slot_map(None, 1 << 30, 2, new_pos=(1 << 30) - 1, out=torch.zeros(1, 3, 2, dtype=torch.int32, device=DEV), opts=opts)
    assert got.tolist() == [[[(1 << 30) - 1, 0], [(1 << 31) - 1, 1 << 30], [-1, -1]]] and int(status) == 2


def test_in_a_graph(sqa):
    """Captured once, replayed as lengths change, on a stream of its own, with the program's own work in between."""
    rng = random.Random(11)
    p = Pool(7, 2, 200, 120, rng)
    tokens, rows = ints([0] * 7), torch.zeros(7, 2, 1, dtype=torch.int32, device=DEV)
    first = ints([0] * 7)
    opts = sqa.batch_opts(new_pos_seq=first)
    side = torch.cuda.Stream()

    def calls():
        sqa.block_assign(p.table, tokens, p.held, p.free_ids, p.count, 200, p.status)
        sqa.slot_map(p.table, 200, 1, out=rows, opts=opts)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            calls()
    torch.cuda.current_stream().wait_stream(side)
    now = [0] * 7
    for step in range(9):
        now = [0 if rng.random() < 0.2 else n + rng.choice([1, 16, 30]) for n in now]
        tokens.copy_(ints(now))
        first.copy_(ints([n - 1 for n in now]))
        torch.randn(1000, device=DEV).sum()
        graph.replay()
        Q.assign(p.rows, now, p.has, p.free, 200, 2)
        assert p.table.tolist() == p.rows and p.held.tolist() == p.has and p.free_ids[:int(p.count)].tolist() == p.free, step
        for b, n in enumerate(now):
            for h in range(2):
                s = Q.slot_of(n - 1, 200, 0) if n else 0
                block = p.rows[b * 2 + h][s // 16] if n else -1
                assert int(rows[b, h, 0]) == (block * 16 + s % 16 if block >= 0 else -1)
