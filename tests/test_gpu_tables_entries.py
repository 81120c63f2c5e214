"""Entries of tables and free lists that are no block's number: reported when they change hands, by tables of one workgroup and of many."""
import random

import pytest
import torch

import q4_reference as Q
from test_gpu_tables import Pool, ints, sqa  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu
SIZES = [(3, 2, 100), (64, 8, 4096)]                 # one workgroup's work, and a launch of many before one


def settled(sqa, B, Hkv, capacity, rng):
    p = Pool(B, Hkv, capacity, B * Hkv * -(-capacity // 16) + 5, rng)
    p.step(sqa, [capacity // 2] * B)
    return p


def call(sqa, p, tokens):
    """One call on both sides; -> the status."""
    p.status.zero_()
    sqa.block_assign(p.table, ints(tokens), p.held, p.free_ids, p.count, p.capacity, p.status)
    Q.assign(p.rows, tokens, p.has, p.free, p.capacity, p.Hkv)
    assert p.table.tolist() == p.rows and p.held.tolist() == p.has and p.free_ids[:int(p.count)].tolist() == p.free
    return int(p.status)


@pytest.mark.parametrize("bad", [-1, "n_blocks", 2 ** 31 - 1, -2 ** 31])
@pytest.mark.parametrize("B,Hkv,capacity", SIZES)
def test_entries_that_come_back(sqa, B, Hkv, capacity, bad):  # noqa: F811
    p = settled(sqa, B, Hkv, capacity, random.Random(3))
    bad = p.free_ids.numel() if bad == "n_blocks" else bad
    p.table[Hkv, 1] = bad                            # (of sequence 1)
    p.rows[Hkv][1] = bad
    same = [capacity // 2] * B
    assert call(sqa, p, same) == 0                   # it stays where it is
    assert call(sqa, p, [same[0], 0] + same[2:]) == 8
    assert bad in p.free
    assert call(sqa, p, [capacity] * B) == 8 and bad not in p.free           # and is reported again when it is dealt out


@pytest.mark.parametrize("bad", [-1, "n_blocks"])
@pytest.mark.parametrize("B,Hkv,capacity", SIZES)
def test_entries_of_the_list(sqa, B, Hkv, capacity, bad):  # noqa: F811
    p = settled(sqa, B, Hkv, capacity, random.Random(4))
    bad = p.free_ids.numel() if bad == "n_blocks" else bad
    p.free_ids[len(p.free) - 1] = bad
    p.free[-1] = bad
    same = [capacity // 2] * B
    assert call(sqa, p, same) == 0                   # (nothing is taken)
    assert call(sqa, p, [capacity // 2 + 16] + same[1:]) == 8
    assert p.rows[0][p.has[0] - 1] == bad


def test_without_a_status(sqa):  # noqa: F811
    p = settled(sqa, 3, 2, 100, random.Random(5))
    p.table[2, 1] = -7
    p.rows[2][1] = -7
    sqa.block_assign(p.table, ints([48, 0, 48]), p.held, p.free_ids, p.count, 100)
    Q.assign(p.rows, [48, 0, 48], p.has, p.free, 100, 2)
    assert p.table.tolist() == p.rows and p.free_ids[:int(p.count)].tolist() == p.free
