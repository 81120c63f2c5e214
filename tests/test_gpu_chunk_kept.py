"""What the chunk calls leave alone, and what compression then keeps of a prompt that came in chunks."""
import math

import pytest
import torch

import chunk_reference as R
from test_gpu_chunk import DEV, LAYOUTS, generator, ints, sqa  # noqa: F401
from test_gpu_chunk_session import mods  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name,kw,ragged", [("tiny", dict(P=272), False), ("llama2_70b", dict(L=2, B=2, P=333, S=3, Hq=16, Hkv=2, hidden=256), False),
                                            ("llama2_7b", dict(L=2, B=3, P=200, S=3, Hq=4, Hkv=4, hidden=256), True)])
def test_heavy_hitters_of_a_prompt_in_chunks(mods, name, kw, ragged):  # noqa: F811
    """The two ways' scores differ by rounding, e at most in a unit.  A position that only one of them keeps has, by either's scores, at most 2 e
    more or less than one that only the other keeps; where both keep the same ones, their keys, values and scores (to e) are the same too."""
    _, session, W = mods
    wl = W.scaled(W.WORKLOADS[name], policy="h2o", **kw)
    lens = [wl.P - 37 * b for b in range(wl.B)] if ragged else [wl.P] * wl.B
    whole, parts = [session.Session(wl, DEV, prompt_len=lens if ragged else None, prompt_chunk=c) for c in (None, 64)]
    for s in (whole, parts):
        s.probe_and_allocate()
        s.compress_prompt()
    assert whole.budgets == parts.budgets and any(b < wl.P for b in whole.budgets)
    same = 0
    for l in range(wl.L):
        for b in range(wl.B):
            for h in range(wl.Hkv):
                n = int(whole.caches.lens[l][b, h])
                assert n == int(parts.caches.lens[l][b, h])
                kept = [s.caches.unit(l, b, h)[3][:n].long() for s in (whole, parts)]
                scores = [s.scores[l][b, h, :lens[b]].double() for s in (whole, parts)]
                e = float((scores[0] - scores[1]).abs().max())
                mine, theirs = (set(k.tolist()) for k in kept)
                assert len(mine) == len(theirs) == n
                a, c = sorted(mine - theirs), sorted(theirs - mine)
                if a:
                    assert float(scores[0][a].max() - scores[0][c].min()) <= 2 * e, (l, b, h, a, c)
                else:
                    same += 1
                    assert torch.equal(*kept)
                    for x, y in zip(whole.caches.unit(l, b, h)[:2], parts.caches.unit(l, b, h)[:2]):
                        assert torch.equal(x[:n], y[:n])
                    x, y = (s.caches.unit(l, b, h)[2][:n].double() for s in (whole, parts))
                    assert float((x - y).abs().max()) <= e
    assert same > 0


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
def test_append_writes_nothing_but_its_slots(sqa, dtype, D, layout):  # noqa: F811
    """Scores and positions (and keys, values, records of units that take no part) outside the chunk's slots, bit for bit."""
    dt, gen = R.DT[dtype], generator(19)
    for B, T, Hkv, first, n in ((1, 1, 1, [0], [1]), (3, 5, 5, [14, 0, 31], [5, 4, 0]), (2, 700, 4, [3, 900], [700, 611]), (4, 33, 3, [7, 16, 31, 2], [33, 1, 16, 33])):
        c = R.fill(R.make_cache(sqa, layout, B, Hkv, D, dt, [f + m + 3 for f, m in zip(first, n)]), first, gen, value=math.nan)
        before = R.snapshot(c)
        x = torch.randn(B, T, Hkv, D, generator=gen, device=DEV).to(dt)
        status = ints([0])
        sqa.chunk_append(x, x, 0, c, opts=sqa.batch_opts(prompt_len=ints(n), new_pos_seq=ints(first), status=status))
        assert int(status) == 0
        for b in range(B):
            for h in range(Hkv):
                lo = slice(first[b], first[b] + n[b])
                idx = c.unit_kv_rows(0, b, h)[2][lo]
                for now, old in ((c.K[0], before[0]), (c.V[0], before[1])):
                    assert torch.equal(now.view(-1, D)[idx], x[b, :n[b], h])
                    now.view(-1, D)[idx] = old.view(-1, D)[idx]
                start = (b * Hkv + h) * c.score[0].shape[-1] if c.offsets_host[0] is None else int(c.offsets_host[0][b * Hkv + h])
                at = slice(start + first[b], start + first[b] + n[b])
                assert bool((c.score[0].view(-1)[at] == 0).all())
                assert torch.equal(c.pos[0].view(-1)[at], torch.arange(lo.start, lo.stop, dtype=torch.int32, device=DEV))
                for now, old in ((c.score[0], before[2]), (c.pos[0], before[3])):
                    now.view(-1)[at] = old.view(-1)[at]
                if n[b]:
                    assert c.state[0][b, h].tolist() == [first[b] + n[b], 0, -2, 0]
                    c.state[0][b, h] = before[4][b, h]
        assert R.same(before, R.snapshot(c)), (B, T)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_a_draft_is_scored_by_what_stays_of_it(sqa, dtype, D):  # noqa: F811
    """Five drafted tokens, two of which are accepted: scored with prompt_len = 2 and written over by the next append, the layer is the one to which only
    those two were ever appended."""
    dt, gen, B, Hq, Hkv, T, first = R.DT[dtype], generator(23), 2, 8, 2, 5, [600, 37]
    layers = [R.fill(R.make_cache(sqa, "blocked", B, Hkv, D, dt, [620, 620]), first, generator(24)) for _ in range(2)]
    x = torch.randn(B, T, Hq + 2 * Hkv, D, generator=gen, device=DEV).to(dt)
    y = torch.randn(B, T, Hq + 2 * Hkv, D, generator=gen, device=DEV).to(dt)
    y[:, :2] = x[:, :2]
    two, three = ints([2, 2]), ints([3, 3])
    for drafted, c in zip((True, False), layers):
        opts = sqa.batch_opts(prompt_len=ints([T, T]) if drafted else two, new_pos_seq=ints(first))
        q = sqa.chunk_append(x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], 0, c, q=x[:, :, :Hq], opts=opts)
        _, lse = sqa.chunk_attention(q, 0, c, opts=opts)
        sqa.chunk_scores(q, lse, 0, c, opts=sqa.batch_opts(prompt_len=two, new_pos_seq=ints(first)))
        z = y[:, 2:].contiguous()
        later = sqa.batch_opts(prompt_len=three, new_pos_seq=ints([f + 2 for f in first]))
        q = sqa.chunk_append(z[:, :, Hq:Hq + Hkv], z[:, :, Hq + Hkv:], 0, c, q=z[:, :, :Hq], opts=later)
        _, lse = sqa.chunk_attention(q, 0, c, opts=later)
        sqa.chunk_scores(q, lse, 0, c, opts=later)
    for b in range(B):
        n = first[b] + 5
        for h in range(Hkv):
            a, c = (l.unit(0, b, h) for l in layers)
            assert all(torch.equal(p, q) for p, q in zip(R.rows_of(layers[0], b, h, n), R.rows_of(layers[1], b, h, n)))
            assert torch.equal(a[2][:n], c[2][:n]) and torch.equal(a[3][:n], c[3][:n])
    assert torch.equal(layers[0].state[0], layers[1].state[0])
