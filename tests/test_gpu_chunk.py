"""The calls on chunks of tokens against their definitions in 64 bits (chunk_reference.py: formulas and derived bounds), over
types, head layouts, lengths from one token on, cache layouts, strides, ragged batches, and caches that do not take a chunk."""
import math

import pytest
import torch

import chunk_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LAYOUTS = ["dense", "blocked", "packed"]


@pytest.fixture(scope="module")
def sqa():
    from paper_2404_04793_amd import binding
    return binding


def generator(seed):
    return torch.Generator(DEV).manual_seed(seed)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# ---- norm, rotation, append --------------------------------------------------------------------------------
PREPS = [("none", None, None, False), ("norm", 1e-6, None, False), ("rope", None, 1.0, False), ("both", 1e-5, 1.0, False), ("half", 1e-6, 0.5, False),
         ("pairs", 1e-6, 1.0, True), ("16", None, 16, False), ("16 pairs", None, 16, True)]


def make_prep(sqa, kind, D, dt, gen, n_pos=4000):
    _, eps, rot, pairs = kind
    w = [None, None] if eps is None else [(1 + 0.2 * torch.randn(D, generator=gen, device=DEV)).to(dt) for _ in range(2)]
    rope = None if rot is None else sqa.rope_table(n_pos, int(rot * D) if rot <= 1 else rot, device=DEV)
    return w, eps or 0.0, rope, pairs, sqa.head_prep(w[0], w[1], eps or 0.0, rope, pairs)


def close(got, want, bound, dt, what):
    assert got.dtype == dt
    off = (got.double() - want).abs()
    limit = bound + R.HALF[dt] * want.abs() * 1.0001 + 1e-30
    assert bool((off <= limit).all()), (what, float((off / limit).max()))


@pytest.mark.parametrize("kind", PREPS, ids=lambda k: k[0])
@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
def test_norm_and_rotation(sqa, dtype, D, kind):
    dt, gen = R.DT[dtype], generator(11)
    w, eps, rope, pairs, prep = make_prep(sqa, kind, D, dt, gen)
    for B, T, Hq, Hkv, first in ((1, 1, 1, 1, 0), (3, 1, 5, 1, 3999), (2, 7, 6, 3, 1234), (1, 130, 9, 3, 77), (2, 1024, 16, 16, 5)):
        packed = torch.randn(B, T + 2, (Hq + 2 * Hkv) * D + 16, generator=gen, device=DEV).to(dt)       # a part of a longer prompt's projection
        x = packed[:, 1:T + 1, :(Hq + 2 * Hkv) * D].view(B, T, Hq + 2 * Hkv, D) if B == 1 else packed[:, 1:T + 1, 16:].unflatten(2, (-1, D))
        q, k = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv]
        q_out, k_out = sqa.qk_norm_rope(q, k, first, prep)
        pos = torch.arange(first, first + T, device=DEV)
        for b in range(B):
            for got, src, weight in ((q_out, q, w[0]), (k_out, k, w[1])):
                want, bound = R.norm_rope(src[b], weight, eps, rope, pairs, pos)
                close(got[b].transpose(0, 1), want, bound, dt, (B, T, b))
        only_k = sqa.qk_norm_rope(None, k, first, prep)[1]
        only_q = sqa.qk_norm_rope(q, None, first, prep)[0]
        assert torch.equal(only_k, k_out) and torch.equal(only_q, q_out)


def test_norm_of_zero_rows_infinities_and_large_numbers(sqa):
    dt, D = torch.float32, 64
    prep = sqa.head_prep(torch.ones(D, device=DEV), torch.ones(D, device=DEV), 1e-6)
    x = torch.zeros(1, 4, 2, D, device=DEV)
    x[0, 1] = 1e18
    x[0, 2, 0, 5] = math.inf
    x[0, 3, 1, 7] = math.nan
    y, _ = sqa.qk_norm_rope(x, None, 0, prep)
    assert bool((y[0, :, 0] == 0).all())
    torch.testing.assert_close(y[0, :, 1], torch.ones(2, D, device=DEV), rtol=1e-5, atol=0)
    assert bool(y[0, 0, 2, 5].isnan()) and bool((y[0, 0, 2, :5] == 0).all()) and bool(y[0, 1, 3].isnan().all()) and bool((y[0, 0, 3] == 0).all())


def test_ragged_rows_are_left_alone(sqa):
    """Padding is neither read nor written, sequences that sit out neither; positions beyond the table are reported."""
    B, T, Hq, Hkv, D, dt = 5, 9, 4, 2, 128, torch.bfloat16
    gen = generator(5)
    n, first = [9, 0, 4, 9, 5], [0, 3, 91, -1, 96]           # the last: positions 96 .. 100 of a table of 100
    x = torch.randn(B, T, Hq + Hkv, D, generator=gen, device=DEV).to(dt)
    for b in range(B):
        x[b, n[b] if first[b] >= 0 else 0:] = math.nan
    rope = sqa.rope_table(100, D, device=DEV)
    q_out, k_out = (torch.full((B, H, T, D), 7.0, dtype=dt, device=DEV) for H in (Hq, Hkv))
    status = ints([0])
    opts = sqa.batch_opts(prompt_len=ints(n), new_pos_seq=ints(first), status=status)
    sqa.qk_norm_rope(x[:, :, :Hq], x[:, :, Hq:], 12345, sqa.head_prep(rope=rope), q_out, k_out, opts)
    assert int(status) == 2
    for b in range(B):
        m = n[b] if 0 <= first[b] and first[b] + n[b] <= 100 else 0
        assert bool((q_out[b, :, m:] == 7).all()) and bool((k_out[b, :, m:] == 7).all())
        if m:
            want, bound = R.norm_rope(x[b, :m, :Hq], None, 0.0, rope, False, torch.arange(first[b], first[b] + m, device=DEV))
            close(q_out[b, :, :m].transpose(0, 1), want, bound, dt, b)
    status.zero_()
    keep = q_out.clone()
    for bad in (-1, T + 1):
        sqa.qk_norm_rope(x[:, :, :Hq], None, 0, None, q_out, opts=sqa.batch_opts(prompt_len=ints([0, bad, 0, 0, 0]), status=status))
        assert int(status) == 2 and torch.equal(keep, q_out)
        status.zero_()


def appended(sqa, caches, before, n, first, x, Hq, prep_parts, dt):
    """Every unit after the call against its definition; returns whether all else is as it was."""
    w, eps, rope, pairs, _ = prep_parts
    B, Hkv, D = caches.B, caches.Hkv, caches.D
    K0, V0, sc0, pos0, st0 = before
    for b in range(B):
        pos = torch.arange(first[b], first[b] + n[b], device=DEV)
        kw, bound = R.norm_rope(x[b, :n[b], Hq:Hq + Hkv], w[1], eps, rope, pairs, pos)
        for h in range(Hkv):
            K, V = R.rows_of(caches, b, h, first[b] + n[b])
            close(K[first[b]:], kw[:, h], bound[:, h], dt, ("k", b, h))
            assert torch.equal(V[first[b]:], x[b, :n[b], Hq + Hkv + h])
            _, _, score, p = caches.unit(0, b, h)
            assert torch.equal(p[first[b]:first[b] + n[b]], pos.to(torch.int32)) and bool((score[first[b]:first[b] + n[b]] == 0).all())
            assert caches.state[0][b, h].tolist() == ([first[b] + n[b], 0, -2, 0] if n[b] else st0[b, h].tolist())
            # undo, so that what is left must be what was there
            idx = caches.unit_kv_rows(0, b, h)[2][first[b]:first[b] + n[b]]
            for now, old in ((caches.K[0], K0), (caches.V[0], V0)):
                now.view(-1, D)[idx] = old.view(-1, D)[idx]
    return R.same([K0, V0], [caches.K[0], caches.V[0]])


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("kind", [PREPS[0], PREPS[3], PREPS[5]], ids=lambda k: k[0])
@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
def test_append(sqa, dtype, D, kind, layout):
    dt, gen = R.DT[dtype], generator(7)
    parts = make_prep(sqa, kind, D, dt, gen)
    for B, T, Hq, Hkv, first, n in ((1, 1, 1, 1, [0], None), (2, 1, 6, 3, [15, 16], [1, 1]), (3, 5, 10, 5, [14, 0, 31], [5, 4, 0]),
                                    (1, 33, 8, 8, [61], None), (2, 700, 32, 16, [3, 900], [700, 611])):
        ragged = n is not None
        n = n or [T] * B
        room = [f + m + 2 for f, m in zip(first, n)]
        c = R.fill(R.make_cache(sqa, layout, B, Hkv, D, dt, room), first, gen, value=math.nan)
        before = R.snapshot(c)
        x = torch.randn(B, T, Hq + 2 * Hkv, D, generator=gen, device=DEV).to(dt)
        for b in range(B):
            x[b, n[b]:] = math.nan
        q_out = torch.full((B, Hq, T, D), 5.0, dtype=dt, device=DEV)
        status = ints([0])
        opts = sqa.batch_opts(prompt_len=ints(n), new_pos_seq=ints(first), status=status) if ragged else None
        sqa.chunk_append(x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], first[0], c, prep=parts[4], q=x[:, :, :Hq], q_out=q_out, opts=opts)
        assert int(status) == 0
        want = torch.full_like(q_out, 5.0)
        sqa.qk_norm_rope(x[:, :, :Hq], None, first[0], parts[4], want, opts=opts)
        assert torch.equal(q_out, want)                                      # the two calls' queries, padding among them
        assert appended(sqa, c, before, n, first, x, Hq, parts, dt)
        # without queries: the same cache
        d = R.make_cache(sqa, layout, B, Hkv, D, dt, room)
        for mine, theirs in zip(before, (d.K[0], d.V[0], d.score[0], d.pos[0], d.state[0])):
            theirs.copy_(mine)
        sqa.chunk_append(x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], first[0], d, prep=parts[4], opts=opts)
        assert R.same([c.score[0], c.pos[0], c.state[0]], [d.score[0], d.pos[0], d.state[0]])


@pytest.mark.parametrize("layout", LAYOUTS)
def test_append_takes_back_a_draft(sqa, layout):
    """A later append at a smaller position drops what lies behind it; up to the cache's last slot, and from it."""
    B, Hkv, D, dt, gen = 2, 2, 64, torch.float32, generator(9)
    c = R.fill(R.make_cache(sqa, layout, B, Hkv, D, dt, [40, 40]), [20, 20], gen)
    mk = lambda T: torch.randn(B, T, Hkv, D, generator=gen, device=DEV)
    a, b, status = mk(20), mk(7), ints([0])
    sqa.chunk_append(a, a, 20, c)
    assert c.lens[0].tolist() == [[40, 40]] * 2
    sqa.chunk_append(b, b, 23, c, opts=sqa.batch_opts(new_pos_seq=ints([23, 38 - 5]), status=status))
    assert int(status) == 0 and c.lens[0].tolist() == [[30, 30], [40, 40]]
    for s, first in ((0, 23), (1, 33)):
        for h in range(Hkv):
            K, V = R.rows_of(c, s, h, first + 7)
            assert torch.equal(K[20:first], a[s, :first - 20, h]) and torch.equal(V[first:], b[s, :, h])


@pytest.mark.parametrize("layout", LAYOUTS)
def test_append_leaves_units_that_take_no_chunk(sqa, layout):
    """Each unit's reason alone, the others of the batch appended to; the refused ones bit for bit as they were."""
    B, Hkv, D, T, dt, gen = 4, 2, 128, 6, torch.bfloat16, generator(13)
    x = torch.randn(B, T, Hkv, D, generator=gen, device=DEV).to(dt)

    def check(code, change, first=(10, 10, 10, 10), bad=(1,), heads=(0, 1), budget_seq=None):
        c = R.fill(R.make_cache(sqa, layout, B, Hkv, D, dt, [24] * B), [10] * B, gen)
        change(c)
        before, status = R.snapshot(c), ints([0])
        sqa.chunk_append(x, x, 0, c, opts=sqa.batch_opts(new_pos_seq=ints(first), budget_seq=budget_seq, status=status))
        assert int(status) == code, int(status)
        d = R.make_cache(sqa, layout, B, Hkv, D, dt, [24] * B)
        for b in range(B):
            for h in range(Hkv):
                refused = b in bad and h in heads
                assert int(c.lens[0][b, h]) == (int(before[4][b, h, 0]) if refused else first[b] + T), (b, h)
                for now, old in ((c.K[0], before[0]), (c.V[0], before[1])):
                    idx = d.unit_kv_rows(0, b, h)[2] if layout != "blocked" else c.unit_kv_rows(0, b, h)[2][:16]
                    if refused and int(idx.max()) < now.view(-1, D).shape[0] and int(idx.min()) >= 0:
                        assert torch.equal(now.view(-1, D)[idx], old.view(-1, D)[idx]), (b, h)
                if refused:
                    assert all(torch.equal(y, z) for y, z in zip(c.unit(0, b, h)[2:], R_unit(before, c, b, h)))

    def R_unit(before, c, b, h):
        if c.offsets_host[0] is None:
            return before[2][b, h], before[3][b, h]
        lo, hi = c.offsets_host[0][b * Hkv + h], c.offsets_host[0][b * Hkv + h + 1]
        return before[2][lo:hi], before[3][lo:hi]

    nothing = lambda c: None
    check(8, nothing, first=(10, 11, 10, 10))                                        # a gap
    check(8, lambda c: c.head[0][1].fill_(1))                                        # the ring has moved
    check(8, lambda c: c.lens[0][1].fill_(9))
    check(8, lambda c: c.unit(0, 1, 1)[3][9:10].fill_(12), heads=(1,))               # the last token is another one
    check(6, lambda c: (c.lens[0][1].fill_(20), [c.unit(0, 1, h)[3][:20].copy_(torch.arange(20)) for h in range(2)]), first=(10, 20, 10, 10))   # 26 > 24
    check(5, nothing, budget_seq=ints([24, 25, 24, 24]))
    check(5, nothing, budget_seq=ints([24, 0, 24, 24]))
    check(6, nothing, budget_seq=ints([24, 15, 24, 16]))
    # a full unit that has evicted: slot 7 holds a later token, slot 9 its own
    def evicted(c):
        c.lens[0][1].fill_(24)
        for h in range(2):
            p = c.unit(0, 1, h)[3]
            p[:24] = torch.arange(24, dtype=torch.int32)
            p[7] = 500
    check(8, evicted)
    if layout == "blocked":
        for bad in (-1, 1 << 30):
            check(2, lambda c: c.block_table[0].view(B, Hkv, -1)[1, 1, 0].fill_(bad), heads=(1,))


def test_append_of_a_unit_that_evicted_in_decode(sqa):
    """After real evictions an append is refused, whatever position it asks for."""
    B, Hkv, D, dt, gen = 1, 2, 64, torch.float32, generator(17)
    c = sqa.LayerCaches([16], [16], B, Hkv, D, dt, DEV, True)
    mk = lambda *s: torch.randn(*s, generator=gen, device=DEV)
    x = mk(B, 16, Hkv, D)
    sqa.chunk_append(x, x, 0, c)
    ws, out = sqa.decode_workspace(c, Hkv, "h2o"), torch.empty(1, B, Hkv, D, device=DEV)
    for t in range(16, 16 + 9):
        sqa.decode_step(mk(1, B, Hkv, D), mk(1, B, Hkv, D), mk(1, B, Hkv, D), t, "h2o", 4, c, out, ws)
    assert sqa.read_device_status(ws) == 0
    before = R.snapshot(c)
    for first in range(1, 17):
        status = ints([0])
        y = mk(B, 1, Hkv, D)
        sqa.chunk_append(y, y, 0, c, opts=sqa.batch_opts(new_pos_seq=ints([first]), status=status))
        held = [all(int(p) == s for s, p in enumerate(c.pos[0][0, h, :first])) and int(c.head[0][0, h]) == 0 for h in range(Hkv)]
        assert not any(held) and int(status) == 8 and R.same(before, R.snapshot(c)), first


# ---- attention and scores ----------------------------------------------------------------------------------
SHAPES = [  # B, T, first, Hq, Hkv, n (None: all T)
    (1, 1, [0], 1, 1, None), (1, 1, [63], 8, 1, None), (2, 1, [64, 200], 6, 2, [1, 1]), (1, 2, [30], 3, 1, None), (1, 33, [0], 1, 1, None),
    (2, 5, [127, 11], 8, 2, [5, 3]), (1, 31, [96], 2, 2, None), (1, 65, [1], 3, 1, None), (3, 20, [300, 0, 129], 10, 2, [20, 0, 7]),
    (1, 130, [70], 4, 4, None), (1, 257, [0], 2, 1, None), (2, 100, [5, 1000], 15, 3, [100, 99]), (1, 4, [3500], 4, 1, None), (1, 300, [1800], 2, 2, None)]


def setup(sqa, dtype, D, layout, B, T, first, Hq, Hkv, n, seed, room=1):
    dt, gen = R.DT[dtype], generator(seed)
    m = n or [T] * B
    held = [f + x for f, x in zip(first, m)]
    c = R.fill(R.make_cache(sqa, layout, B, Hkv, D, dt, [h + room for h in held]), held, gen, value=math.nan)
    q = (torch.randn(B, Hq, T, D, generator=gen, device=DEV) * 1.5).to(dt)
    for b in range(B):
        q[b, :, m[b]:] = math.nan
    status = ints([0])
    opts = sqa.batch_opts(prompt_len=ints(m), new_pos_seq=ints(first), status=status) if n is not None else None
    return dt, m, c, q, opts, status


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
def test_attention_and_scores(sqa, dtype, D, layout):
    for at, (B, T, first, Hq, Hkv, n) in enumerate(SHAPES):
        dt, m, c, q, opts, status = setup(sqa, dtype, D, layout, B, T, first, Hq, Hkv, n, 100 + at)
        g, before = Hq // Hkv, R.snapshot(c)
        out = torch.full((B, T, Hq, D), 3.0, dtype=dt, device=DEV)
        lse = torch.full((B, Hq, T), 3.0, device=DEV)
        ws = sqa.chunk_workspace(c, Hq, T)
        for again in range(2):
            sqa.chunk_attention(q, first[0], c, out=out, lse=lse, workspace=ws, opts=opts)
            if not again:
                kept = out.clone(), lse.clone()
        assert R.same(kept, (out, lse)) and R.same(before, R.snapshot(c)) and int(status) == 0
        for b in range(B):
            assert bool((out[b, m[b]:] == 3).all()) and bool((lse[b, :, m[b]:] == 3).all()), (at, b)
            for h in range(Hkv if m[b] else 0):
                K, V = R.rows_of(c, b, h, first[b] + m[b])
                heads = slice(h * g, (h + 1) * g)
                want, want_lse, tol, tol_lse = R.attention(q[b, heads, :m[b]], K, V, first[b], dt)
                off = (out[b, :m[b], heads].transpose(0, 1).double() - want).abs()
                assert bool((off <= tol).all()), (at, b, h, float((off / tol).max()))
                off = (lse[b, heads, :m[b]].double() - want_lse).abs()
                assert bool((off <= tol_lse).all()), (at, b, h, float((off / tol_lse).max()))
        # ---- scores by these normalisers (rows of padding hold anything)
        for b in range(B):
            lse[b, :, m[b]:] = math.nan
        sqa.chunk_scores(q, lse, first[0], c, workspace=ws, opts=opts)
        after = R.snapshot(c)
        assert R.same(before[:2] + before[3:], after[:2] + after[3:]) and int(status) == 0
        for b in range(B):
            for h in range(Hkv):
                score = c.unit(0, b, h)[2]
                old = before[2][b, h] if c.offsets_host[0] is None else before[2][c.offsets_host[0][b * Hkv + h]:][:score.numel()]
                held = first[b] + m[b]
                assert R.same([old[held:]], [score[held:]])
                if m[b]:
                    K, _ = R.rows_of(c, b, h, held)
                    want, tol = R.scores(q[b, h * g:(h + 1) * g, :m[b]], K, lse[b, h * g:(h + 1) * g, :m[b]], first[b], old[:held])
                    off = (score[:held].double() - want).abs()
                    assert bool((off <= tol).all()), (at, b, h, float((off / tol).max()))
                else:
                    assert R.same([old[:held]], [score[:held]])


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
def test_what_a_row_does_not_see_does_not_matter(sqa, dtype, D):
    """Keys and values of later tokens that are NaN or infinite: rows before them bit for bit as with ordinary ones, rows from
    them on as the definition says."""
    for T, first, g in ((5, 0, 4), (70, 30, 1), (200, 65, 2), (3, 1000, 2)):
        dt, _, c, q, _, _ = setup(sqa, dtype, D, "blocked", 1, T, [first], 2 * g, 2, None, T)
        ws = sqa.chunk_workspace(c, 2 * g, T)
        out, lse = sqa.chunk_attention(q, first, c, workspace=ws)
        for bad, what in ((math.nan, "V"), (math.inf, "V"), (-math.inf, "V"), (math.nan, "K"), (math.inf, "K"), (-math.inf, "K")):
            t = T // 2
            rows = [c.unit_kv_rows(0, 0, h)[2][first + t] for h in range(2)]
            mem = (c.V[0] if what == "V" else c.K[0]).view(-1, D)
            old = [mem[r].clone() for r in rows]
            for r in rows:
                mem[r, 3::5] = bad
            score0 = c.score[0].clone()
            out2, lse2 = sqa.chunk_attention(q, first, c, workspace=ws)
            assert R.same([out[:, :t], lse[..., :t]], [out2[:, :t].contiguous(), lse2[..., :t]]), (T, bad, what)
            late = out2[:, t:].float()
            if what == "V":
                assert R.same([lse], [lse2])
                hit = torch.zeros(D, dtype=torch.bool, device=DEV)
                hit[3::5] = True
                got = late[..., hit]
                # (a probability of 0 makes 0 x inf of it)
                assert bool((got.isnan() | (got == bad)).all()) and bool(torch.isfinite(late[..., ~hit]).all()), (T, bad)
                assert bool((got.isnan() if math.isnan(bad) else got == bad).any())
                assert R.same([out[:, t:][..., ~hit].contiguous()], [out2[:, t:][..., ~hit].contiguous()])
            else:
                s = q.double() @ torch.where(torch.isfinite(mem[rows[0]]), 0.0, mem[rows[0]].double())
                assert not bool(torch.isfinite(late).all()) or bool((s == -math.inf).all()) or bad == -math.inf or math.isinf(bad)
            # scores with these keys: slots that the odd one is not are as with ordinary ones
            if what == "K":
                sqa.chunk_scores(q, lse, first, c, workspace=ws)
                sc_odd = [c.unit(0, 0, h)[2].clone() for h in range(2)]
                c.score[0].copy_(score0)
                for r, o in zip(rows, old):
                    mem[r] = o
                sqa.chunk_scores(q, lse, first, c, workspace=ws)
                for h in range(2):
                    a, b = sc_odd[h].clone(), c.unit(0, 0, h)[2].clone()
                    a[first + t] = b[first + t] = 0
                    assert R.same([a], [b])
                c.score[0].copy_(score0)
            for r, o in zip(rows, old):
                mem[r] = o


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
def test_a_row_without_a_normaliser_spoils_only_what_it_sees(sqa, dtype, D):
    """A row whose log-sum-exp is NaN or -inf (its query or its keys were): the scores of later slots are what they are without it."""
    for B, T, first, Hq, Hkv, t in ((1, 70, 30, 4, 2, 20), (2, 200, 0, 2, 2, 63), (1, 5, 300, 8, 1, 0), (1, 130, 500, 3, 3, 129)):
        dt, _, c, q, _, _ = setup(sqa, dtype, D, "dense", B, T, [first] * B, Hq, Hkv, None, 31)
        _, lse = sqa.chunk_attention(q, first, c)
        score0, got = c.score[0].clone(), []
        for value in (math.inf, math.nan, -math.inf):                   # (infinite: the row gives nothing)
            lse[0, 0, t] = value
            c.score[0].copy_(score0)
            sqa.chunk_scores(q, lse, first, c)
            got.append(c.score[0][..., :first + T].clone())
        without, seen = got[0], first + t + 1
        assert bool(torch.isfinite(without).all())
        for other in got[1:]:
            assert not bool(torch.isfinite(other[0, 0, :seen]).any())
            assert R.same([without[0, 0, seen:], without[:, 1:]], [other[0, 0, seen:], other[:, 1:]]), (B, T, first, t)


def test_logits_of_every_size(sqa):
    """Rows whose logits are all very low, very high or far apart; one slot that takes all; a chunk whose logits are -inf but for its own."""
    D, T, first = 64, 40, 90
    for dtype in ("f32", "bf16"):
        dt, _, c, q, _, _ = setup(sqa, dtype, D, "dense", 1, T, [first], 2, 1, None, 3)
        K, V, idx = c.unit_kv_rows(0, 0, 0)
        ws = sqa.chunk_workspace(c, 2, T)
        for scale in (1e-30, 30.0, 1e4):
            q2 = (q.float() * scale).to(dt)
            out, lse = sqa.chunk_attention(q2, first, c, workspace=ws)
            want, want_lse, tol, tol_lse = R.attention(q2[0], K[idx[:first + T]], V[idx[:first + T]], first, dt)
            assert bool(((out[0].transpose(0, 1).double() - want).abs() <= tol).all()), scale
            assert bool(((lse[0].double() - want_lse).abs() <= tol_lse).all()), scale
        # every logit near the type's lowest value: the softmax is what it is without the offset
        q3, K3 = torch.zeros_like(q), K.clone()
        q3[..., 0] = 1e18
        K[idx[:first + T], 0] = -1e18
        out, lse = sqa.chunk_attention(q3, first, c, workspace=ws)
        want = torch.stack([V[idx[:first + 1 + t]].double().mean(0) for t in range(T)])
        assert bool(((out[0].transpose(0, 1).double() - want).abs() <= 2.0 ** -7 * V[idx[:first + T]].double().abs().mean() * 3).all())
        # -inf everywhere but in the chunk's own slots
        K.copy_(K3)
        K[idx[:first], 0] = -math.inf
        q3 = q.abs()
        q3[..., 1:] = 0
        own, _ = sqa.chunk_attention(q3, first, c, workspace=ws)
        want, _, tol, _ = R.attention(q3[0], K[idx[first:first + T]], V[idx[first:first + T]], 0, dt)
        assert bool(((own[0].transpose(0, 1).double() - want).abs() <= tol).all())
        K.copy_(K3)


def test_units_that_do_not_hold_the_chunk(sqa):
    """Their rows are zeros and lse -inf, their scores as they were; the other units' results as ever."""
    B, T, first, Hq, Hkv, D = 2, 20, [50, 50], 4, 2, 128
    dt, m, c, q, opts, status = setup(sqa, "bf16", D, "blocked", B, T, first, Hq, Hkv, [20, 20], 1)
    good, good_lse = sqa.chunk_attention(q, 0, c, opts=opts)
    u = (1, 1)

    def short(): c.lens[0][u] = 69
    def moved(): c.head[0][u] = 3
    def other(): c.pos[0][1, 1, 69] = 70
    def outside(): c.block_table[0][3, 2] = -5
    def outside2(): c.block_table[0][3, 0] = c.K[0].shape[0]
    for change, code in ((short, 8), (moved, 8), (other, 8), (outside, 2), (outside2, 2)):
        keep = [x.clone() for x in (c.state[0], c.pos[0], c.block_table[0])]
        change()
        status.zero_()
        out, lse = sqa.chunk_attention(q, 0, c, opts=opts)
        assert int(status) == code
        assert bool((out[1, :, 2:] == 0).all()) and bool((lse[1, 2:] == -math.inf).all())
        assert R.same([good[0], good[1, :, :2].contiguous(), good_lse[0], good_lse[1, :2]], [out[0], out[1, :, :2].contiguous(), lse[0], lse[1, :2]])
        score0 = c.score[0].clone()
        status.zero_()
        sqa.chunk_scores(q, good_lse, 0, c, opts=opts)
        assert int(status) == code and R.same([score0[1, 1]], [c.score[0][1, 1]]) and not R.same([score0[1, 0]], [c.score[0][1, 0]])
        for x, y in zip((c.state[0], c.pos[0], c.block_table[0]), keep):
            x.copy_(y)
        c.score[0].copy_(score0)
    # a position beyond the unit's slots
    status.zero_()
    out, lse = sqa.chunk_attention(q, 0, c, opts=sqa.batch_opts(new_pos_seq=ints([50, 2 ** 31 - 30]), status=status))
    assert int(status) == 8 and bool((out[1] == 0).all()) and R.same([good[0]], [out[0]])


def test_one_workspace_for_chunks_of_many_lengths(sqa):
    """Counters and partial results of one shape are not in the way of the next."""
    dt, _, c, q, _, _ = setup(sqa, "bf16", 128, "dense", 2, 200, [2000, 2000], 8, 2, None, 4)
    ws = sqa.chunk_workspace(c, 8, 200)
    for T in (1, 200, 3, 17, 64, 5, 130, 1):
        x = q[:, :, :T].contiguous()
        one = sqa.chunk_attention(x, 2000, c, workspace=ws)
        two = sqa.chunk_attention(x, 2000, c)
        assert R.same(one, two), T
        score0 = c.score[0].clone()
        sqa.chunk_scores(x, one[1], 2000, c, workspace=ws)
        a = c.score[0].clone()
        c.score[0].copy_(score0)
        sqa.chunk_scores(x, one[1], 2000, c)
        assert R.same([a], [c.score[0]])
        c.score[0].copy_(score0)
    assert bool((ws[:4096] == 0).all())


def test_from_another_stream(sqa):
    dt, _, c, q, _, _ = setup(sqa, "bf16", 64, "packed", 1, 50, [400], 4, 2, None, 6)
    want = sqa.chunk_attention(q, 400, c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = sqa.chunk_attention(q, 400, c)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert R.same(want, got)


def test_new_pos_is_not_looked_at_where_each_sequence_has_its_own(sqa):
    dt, _, c, q, opts, status = setup(sqa, "bf16", 64, "dense", 2, 5, [30, 7], 4, 2, [5, 3], 9)
    k = torch.randn(2, 5, 2, 64, device=DEV, generator=generator(9)).to(dt)
    got = []
    for new_pos in (0, -5, 2 ** 31 - 1, -2 ** 31):
        x = torch.zeros(2, 4, 5, 64, dtype=dt, device=DEV)
        sqa.chunk_append(k, k, new_pos, c, q=q.transpose(1, 2).contiguous(), q_out=x, opts=opts)
        out, lse = torch.zeros(2, 5, 4, 64, dtype=dt, device=DEV), torch.zeros(2, 4, 5, device=DEV)
        sqa.chunk_attention(x, new_pos, c, out=out, lse=lse, opts=opts)
        c.score[0].zero_()
        sqa.chunk_scores(x, lse, new_pos, c, opts=opts)
        got.append([x, out, lse, c.score[0].clone()])
    assert int(status) == 0 and all(R.same(got[0], other) for other in got[1:])


def test_sequences_that_take_no_part(sqa):
    """All of them out, by position or by length: nothing is read or written."""
    dt, _, c, q, _, _ = setup(sqa, "bf16", 128, "blocked", 2, 70, [30, 7], 4, 2, [0, 0], 9)
    k = torch.full((2, 70, 2, 128), math.nan, dtype=dt, device=DEV)
    ws = sqa.chunk_workspace(c, 4, 70)
    for pos, n in ((ints([-1, -7]), None), (None, ints([0, 0])), (ints([-1, 3]), ints([70, 0]))):
        status = ints([0])
        opts = sqa.batch_opts(prompt_len=n, new_pos_seq=pos, status=status)
        outs = [torch.full((2, 4, 70, 128), 3.0, dtype=dt, device=DEV), torch.full((2, 70, 4, 128), 3.0, dtype=dt, device=DEV),
                torch.full((2, 4, 70), 3.0, device=DEV)]
        before = [t.clone() for t in outs] + R.snapshot(c)
        sqa.chunk_append(k, k, 0, c, q=q.transpose(1, 2).contiguous(), q_out=outs[0], opts=opts)
        sqa.chunk_attention(q, 0, c, out=outs[1], lse=outs[2], workspace=ws, opts=opts)
        sqa.chunk_scores(q, outs[2], 0, c, workspace=ws, opts=opts)
        assert int(status) == 0 and R.same(before, outs + R.snapshot(c))
    assert bool((ws[:4096] == 0).all())


def test_two_calls_at_once(sqa):
    """Two layers' calls on two streams, a workspace each: what each gives alone."""
    sides = [torch.cuda.Stream() for _ in range(2)]
    made = [setup(sqa, "bf16", 128, layout, 4, T, [3000] * 4, 8, 2, None, 20 + T) for layout, T in (("dense", 4), ("blocked", 300))]
    wss = [sqa.chunk_workspace(m[2], 8, m[3].shape[2]) for m in made]

    def run(i):
        c, q = made[i][2], made[i][3]
        out, lse = sqa.chunk_attention(q, 3000, c, workspace=wss[i])
        sqa.chunk_scores(q, lse, 3000, c, workspace=wss[i])
        return [out, lse]

    alone, score0 = [], [m[2].score[0].clone() for m in made]
    for i in range(2):
        alone.append(run(i) + [made[i][2].score[0].clone()])
    torch.cuda.synchronize()
    for _ in range(4):
        for i in range(2):
            made[i][2].score[0].copy_(score0[i])
        torch.cuda.synchronize()
        got = [None, None]
        for i in range(2):
            with torch.cuda.stream(sides[i]):
                got[i] = run(i)
        torch.cuda.synchronize()
        for i in range(2):
            assert R.same(alone[i], got[i] + [made[i][2].score[0]])


def test_captured_and_replayed(sqa):
    """A chunk's three calls in a HIP graph, positions and inputs changing between the replays, two graphs on one workspace."""
    B, T, Hq, Hkv, D, dt, gen = 2, 4, 8, 2, 128, torch.bfloat16, generator(8)
    start = [700, 333]
    c = R.fill(R.make_cache(sqa, "blocked", B, Hkv, D, dt, [800, 800]), start, gen)
    prep = sqa.head_prep(rope=sqa.rope_table(800, D, device=DEV))
    ws = sqa.chunk_workspace(c, Hq, T)
    x, pos, n = torch.empty(B, T, Hq + 2 * Hkv, D, dtype=dt, device=DEV), ints(start), ints([T, T])
    opts = sqa.batch_opts(prompt_len=n, new_pos_seq=pos)
    bufs = [(torch.zeros(B, Hq, T, D, dtype=dt, device=DEV), torch.zeros(B, T, Hq, D, dtype=dt, device=DEV), torch.zeros(B, Hq, T, device=DEV)) for _ in range(2)]

    def step(q, out, lse):
        sqa.chunk_append(x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], 0, c, prep=prep, q=x[:, :, :Hq], q_out=q, opts=opts)
        sqa.chunk_attention(q, 0, c, out=out, lse=lse, workspace=ws, opts=opts)
        sqa.chunk_scores(q, lse, 0, c, workspace=ws, opts=opts)

    x.normal_(generator=gen)
    step(*bufs[0])
    torch.cuda.synchronize()
    graphs = []
    for b in bufs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            step(*b)
    torch.cuda.synchronize()
    for i in range(6):
        x.normal_(generator=gen)
        n.copy_(ints([T, 1 + i % T]))
        state = R.snapshot(c)
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in bufs[i % 2]] + R.snapshot(c)
        for t, s in zip((c.K[0], c.V[0], c.score[0], c.pos[0], c.state[0]), state):
            t.copy_(s)
        eager = [t.clone() for t in bufs[i % 2]]
        step(*eager)
        torch.cuda.synchronize()
        assert R.same(got, eager + R.snapshot(c)), i
        pos += n


@pytest.mark.parametrize("dtype,D,g", [("bf16", 128, 4), ("f32", 64, 1), ("bf16", 64, 2)])
def test_a_prompt_in_chunks_is_the_prompt(sqa, dtype, D, g):
    """Together, as they are used: a prompt in chunks of many lengths, then compression by the scores gathered on the way and decode
    steps, against the calls that take the prompt whole."""
    B, P, Hkv, b = 2, 307, 2, 90
    Hq, dt, gen = Hkv * g, R.DT[dtype], generator(21)
    qkv = torch.randn(B, P, Hq + 2 * Hkv, D, generator=gen, device=DEV).to(dt)
    w = [(1 + 0.1 * torch.randn(D, generator=gen, device=DEV)).to(dt) for _ in range(2)]
    prep = sqa.head_prep(w[0], w[1], 1e-6, sqa.rope_table(400, D, device=DEV))
    Q, K = sqa.qk_norm_rope(qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], 0, prep)
    V = qkv[:, :, Hq + Hkv:].transpose(1, 2).contiguous()
    whole = sqa.prefill_scores(Q, K)
    for layout in LAYOUTS:
        c = R.make_cache(sqa, layout, B, Hkv, D, dt, [P, P])
        ws, at, outs, lses, qs = sqa.chunk_workspace(c, Hq, 150), 0, [], [], []
        for T in (1, 31, 2, 150, 64, 59):
            x = qkv[:, at:at + T]
            q = sqa.chunk_append(x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], at, c, prep=prep, q=x[:, :, :Hq])
            out, lse = sqa.chunk_attention(q, at, c, workspace=ws)
            sqa.chunk_scores(q, lse, at, c, workspace=ws)
            outs.append(out); lses.append(lse); qs.append(q)
            at += T
        assert at == P and torch.equal(torch.cat(qs, 2), Q)
        out, lse = torch.cat(outs, 1), torch.cat(lses, 2)
        for s in range(B):
            for h in range(Hkv):
                Ku, Vu = R.rows_of(c, s, h, P)
                assert torch.equal(Ku, K[s, h]) and torch.equal(Vu, V[s, h])
                hs = slice(h * g, (h + 1) * g)
                want, want_lse, tol, tol_lse = R.attention(Q[s, hs], Ku, Vu, 0, dt)
                assert bool(((out[s, :, hs].transpose(0, 1).double() - want).abs() <= tol).all())
                assert bool(((lse[s, hs].double() - want_lse).abs() <= tol_lse).all())
                zero = torch.zeros(P, device=DEV)
                want, tol = R.scores(Q[s, hs], Ku, want_lse, 0, zero)
                # the chunks' normalisers are off by tol_lse, six chunks are added
                tol = tol + want * (tol_lse.max() + 8 * R.U)
                assert bool(((c.unit(0, s, h)[2].double() - want).abs() <= tol).all())
        torch.testing.assert_close(sqa.prefill_scores(Q, K, row_lse=lse), whole, rtol=1e-4, atol=1e-6)
        if layout != "dense":
            continue
        # the filled layer is the prompt that compression takes
        kept, ref = (sqa.LayerCaches([b], [b], B, Hkv, D, dt, DEV, True) for _ in range(2))
        sqa.prefill_compress(c.K[0], c.V[0], c.score[0], "h2o", 4, kept, 0)
        sqa.prefill_compress(K, V, c.score[0], "h2o", 4, ref, 0)
        assert R.same(R.snapshot(kept), R.snapshot(ref))
        w2 = sqa.decode_workspace(kept, Hq, "h2o")
        o, x = torch.empty(1, B, Hq, D, dtype=dt, device=DEV), torch.randn(B, 1, Hq + 2 * Hkv, D, generator=gen, device=DEV).to(dt)
        q1, k1 = sqa.qk_norm_rope(x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], P, prep)
        sqa.decode_step(q1.view(1, B, Hq, D), k1.view(1, B, Hkv, D), x[:, 0, Hq + Hkv:].contiguous()[None], P, "h2o", 4, kept, o, w2)
        assert sqa.read_device_status(w2) == 0 and bool(torch.isfinite(o.float()).all())
        # and a decode step over the layer with room is a chunk of one token
        full = [R.make_cache(sqa, "dense", B, Hkv, D, dt, [P + 1] * B) for _ in range(2)]
        for f in full:
            sqa.chunk_append(qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:], 0, f, prep=prep)
        q2 = sqa.chunk_append(x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], P, full[0], prep=prep, q=x[:, :, :Hq])
        one, _ = sqa.chunk_attention(q2, P, full[0])
        w3 = sqa.decode_workspace(full[1], Hq, "sliding")
        sqa.decode_step(q1.view(1, B, Hq, D), k1.view(1, B, Hkv, D), x[:, 0, Hq + Hkv:].contiguous()[None], P, "sliding", 4, full[1], o, w3)
        assert sqa.read_device_status(w3) == 0
        for s in range(B):
            for h in range(Hkv):
                Ku, Vu = R.rows_of(full[0], s, h, P + 1)
                want, _, tol, _ = R.attention(q2[s, h * g:(h + 1) * g], Ku, Vu, P, dt)
                for got in (one[s, :, h * g:(h + 1) * g].transpose(0, 1), o[0, s, h * g:(h + 1) * g][:, None]):
                    assert bool(((got.double() - want).abs() <= tol).all())


def test_rows_beyond_32_bits(sqa):
    """A cache whose rows lie beyond 2^31 elements: the last unit's tokens arrive there and are read there."""
    B, Hkv, D, cap, T, dt = 9, 8, 128, 250000, 3, torch.bfloat16
    c = sqa.LayerCaches([cap], [cap], B, Hkv, D, dt, DEV, True)
    assert B * Hkv * cap * D > 2 ** 31
    gen = generator(2)
    first = [0] * (B - 1) + [100]
    x = torch.randn(B, 100, 3 * Hkv, D, generator=gen, device=DEV).to(dt)
    sqa.chunk_append(x[:, :, Hkv:2 * Hkv], x[:, :, 2 * Hkv:], 0, c)
    y = x[:, :T]
    opts = sqa.batch_opts(new_pos_seq=ints(first))
    q = sqa.chunk_append(y[:, :, Hkv:2 * Hkv], y[:, :, 2 * Hkv:], 0, c, q=y[:, :, :Hkv], opts=opts)
    out, lse = sqa.chunk_attention(q, 0, c, opts=opts)
    sqa.chunk_scores(q, lse, 0, c, opts=opts)
    K, V = c.K[0][B - 1, Hkv - 1, :103], c.V[0][B - 1, Hkv - 1, :103]
    assert torch.equal(K[100:], x[B - 1, :T, 2 * Hkv - 1]) and torch.equal(V[:100], x[B - 1, :100, 3 * Hkv - 1])
    want, want_lse, tol, tol_lse = R.attention(q[B - 1, -1:], K, V, 100, dt)
    assert bool(((out[B - 1, :, -1:].transpose(0, 1).double() - want).abs() <= tol).all())
    want, tol = R.scores(q[B - 1, -1:], K, lse[B - 1, -1:], 100, torch.zeros(103, device=DEV))
    assert bool(((c.score[0][B - 1, Hkv - 1, :103].double() - want).abs() <= tol).all())
