"""The forms of the chunk kernels that only many rows reach (chunk_forms.py), against the definitions in 64 bits with the bounds of chunk_reference.py:
128 and 64 rows of a workgroup, units' row tiles in turn, slots shared out, several row tiles of a score workgroup; values behind the mask that are
not finite, and units that do not hold the chunk, in those forms."""
import math

import pytest
import torch

import chunk_forms as F
import chunk_reference as R
from test_gpu_chunk import DEV, LAYOUTS, setup, sqa  # noqa: F401

pytestmark = pytest.mark.gpu


def name(case):
    return "%dx%d+%d-%dh%d%s" % (case[0], case[1], case[2][0], case[3], case[4], "r" if case[5] else "")


@pytest.mark.parametrize("case", F.ATTENTION, ids=name)
@pytest.mark.parametrize("dtype,D", F.TYPES)
def test_attention(sqa, dtype, D, case):  # noqa: F811
    B, T, first, Hq, Hkv, n = case
    g = Hq // Hkv
    for layout in LAYOUTS:
        dt, m, c, q, opts, status = setup(sqa, dtype, D, layout, B, T, first, Hq, Hkv, n, 500 + T)
        before = R.snapshot(c)
        out = torch.full((B, T, Hq, D), 3.0, dtype=dt, device=DEV)
        lse = torch.full((B, Hq, T), 3.0, device=DEV)
        ws = sqa.chunk_workspace(c, Hq, T)
        sqa.chunk_attention(q, first[0], c, out=out, lse=lse, workspace=ws, opts=opts)
        kept = out.clone(), lse.clone()
        sqa.chunk_attention(q, first[0], c, out=out, lse=lse, workspace=ws, opts=opts)
        assert R.same(kept, (out, lse)) and R.same(before, R.snapshot(c)) and int(status) == 0 and bool((ws[:4096] == 0).all())
        for b in range(B):
            assert bool((out[b, m[b]:] == 3).all()) and bool((lse[b, :, m[b]:] == 3).all()), (layout, b)
            for h in range(Hkv):
                K, V = R.rows_of(c, b, h, first[b] + m[b])
                heads = slice(h * g, (h + 1) * g)
                want, want_lse, tol, tol_lse = R.attention(q[b, heads, :m[b]], K, V, first[b], dt)
                off = (out[b, :m[b], heads].transpose(0, 1).double() - want).abs()
                assert bool((off <= tol).all()), (layout, b, h, float((off / tol).max()))
                off = (lse[b, heads, :m[b]].double() - want_lse).abs()
                assert bool((off <= tol_lse).all()), (layout, b, h, float((off / tol_lse).max()))


@pytest.mark.parametrize("case", F.SCORES, ids=name)
@pytest.mark.parametrize("dtype,D", F.TYPES)
def test_scores(sqa, dtype, D, case):  # noqa: F811
    B, T, first, Hq, Hkv, n = case
    g = Hq // Hkv
    for layout in LAYOUTS if max(first) < 8000 else ("dense", "packed"):        # (a blocked unit has 16384 slots at most)
        dt, m, c, q, opts, status = setup(sqa, dtype, D, layout, B, T, first, Hq, Hkv, n, 700 + T)
        lse = torch.full((B, Hq, T), math.nan, device=DEV)                       # (padding holds anything)
        held, units = [f + x for f, x in zip(first, m)], {}
        for b in range(B):
            for h in range(Hkv):
                K, _ = R.rows_of(c, b, h, held[b])
                heads = slice(h * g, (h + 1) * g)
                s, _, _ = R.logits(q[b, heads, :m[b]], K, first[b])
                lse[b, heads, :m[b]] = torch.logsumexp(s, -1).float()
                units[b, h] = K, c.unit(0, b, h)[2][:held[b]].clone()
        before = R.snapshot(c)
        sqa.chunk_scores(q, lse, first[0], c, opts=opts)
        after = R.snapshot(c)
        assert R.same(before[:2] + before[3:], after[:2] + after[3:]) and int(status) == 0
        for (b, h), (K, old) in units.items():
            heads = slice(h * g, (h + 1) * g)
            want, tol = R.scores(q[b, heads, :m[b]], K, lse[b, heads, :m[b]], first[b], old)
            score = c.unit(0, b, h)[2]
            off = (score[:held[b]].double() - want).abs()
            assert bool((off <= tol).all()), (layout, b, h, float((off / tol).max()))
            assert bool(score[held[b]:].isnan().all())


# 128 rows alone and shared out, 64 rows; an end inside a tile of slots
@pytest.mark.parametrize("B,T,first,Hq,Hkv", [(8, 150, 90, 64, 32), (4, 300, 3000, 8, 2), (40, 64, 200, 16, 16)])
@pytest.mark.parametrize("dtype,D", F.TYPES)
def test_values_that_are_not_finite_and_not_seen(sqa, dtype, D, B, T, first, Hq, Hkv):  # noqa: F811
    for layout in LAYOUTS:
        dt, _, c, q, _, _ = setup(sqa, dtype, D, layout, B, T, [first] * B, Hq, Hkv, None, 61)
        out, lse = sqa.chunk_attention(q, first, c)
        hit = torch.zeros(D, dtype=torch.bool, device=DEV)
        hit[2::5] = True
        for t in (1, T // 2, T - 1):
            rows = torch.stack([c.unit_kv_rows(0, b, h)[2][first + t] for b in range(B) for h in range(Hkv)])
            mem = c.V[0].view(-1, D)
            old = mem[rows].clone()
            for bad in (math.nan, math.inf, -math.inf):
                new = old.clone()
                new[:, hit] = bad
                mem[rows] = new
                got, got_lse = sqa.chunk_attention(q, first, c)
                assert R.same([out[:, :t].contiguous(), lse], [got[:, :t].contiguous(), got_lse]), (layout, t, bad)
                assert R.same([out[..., ~hit].contiguous()], [got[..., ~hit].contiguous()]), (layout, t, bad)
                late = got[:, t:][..., hit]
                # (a probability of 0 makes 0 x inf of it)
                assert bool(late.isnan().all() if math.isnan(bad) else (late.isnan() | (late == bad)).all() and (late == bad).any()), (layout, t, bad)
            mem[rows] = old


@pytest.mark.parametrize("B,T,first,Hq,Hkv", [(8, 150, 90, 64, 32), (4, 300, 3000, 8, 2), (40, 64, 200, 16, 16)])
@pytest.mark.parametrize("dtype,D", F.TYPES)
def test_units_that_do_not_hold_the_chunk(sqa, dtype, D, B, T, first, Hq, Hkv):  # noqa: F811
    _, _, c, q, opts, status = setup(sqa, dtype, D, "blocked", B, T, [first] * B, Hq, Hkv, [T] * B, 62)
    g = Hq // Hkv
    good, good_lse = sqa.chunk_attention(q, 0, c, opts=opts)
    b, h = B - 1, Hkv - 1
    heads = slice(h * g, (h + 1) * g)

    def short(): c.lens[0][b, h] = first + T - 1
    def outside(): c.block_table[0].view(B, Hkv, -1)[b, h, (first + T - 1) // 16] = 1 << 29
    for change, code in ((short, 8), (outside, 2)):
        keep = [x.clone() for x in (c.state[0], c.block_table[0])]
        change()
        status.zero_()
        out, lse = sqa.chunk_attention(q, 0, c, opts=opts)
        score0 = c.score[0].clone()
        sqa.chunk_scores(q, good_lse, 0, c, opts=opts)
        assert int(status) == code
        assert bool((out[b, :, heads] == 0).all()) and bool((lse[b, heads] == -math.inf).all()) and R.same([score0[b, h]], [c.score[0][b, h]])
        out[b, :, heads], lse[b, heads] = good[b, :, heads], good_lse[b, heads]
        assert R.same([good, good_lse], [out, lse]) and not R.same([score0[0, 0]], [c.score[0][0, 0]])
        for x, y in zip((c.state[0], c.block_table[0]), keep):
            x.copy_(y)
