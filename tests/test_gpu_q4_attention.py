"""Attention over a cache in 4 bits against its definition in 64 bits (q4_reference.py: formulas and derived bounds): types, head layouts, one
slot to long units, rings, ragged batches, numbers that are not finite, blocks that are not there, graphs, streams, and a serving
loop with tables made on the GPU."""
import math
import random

import pytest
import torch

import chunk_reference as R
import q4_reference as Q

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def sqa():
    from paper_2404_04793_amd import binding
    return binding


def generator(seed):
    return torch.Generator(DEV).manual_seed(seed)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def filled(sqa, B, Hkv, D, cap, sink, blocked, gen, **kw):
    """A cache whose every slot holds something: normal numbers with a power of their own per group."""
    c = sqa.Q4Caches([cap], B, Hkv, D, DEV, n_sink=sink, blocked=blocked, **kw)
    for x in (c.K[0], c.V[0]):
        x.copy_(torch.randint(0, 256, x.shape, generator=gen, device=DEV))
    for x in (c.K_scale[0], c.V_scale[0]):
        x.copy_(torch.randint(123, 128, x.shape, generator=gen, device=DEV))
    return c


def unit(c, name, u):
    x = getattr(c, name)[0]
    cap = c.capacities[0]
    return x[c.block_table[0][u].long()].flatten(0, 1)[:cap] if c.blocked else x.view(-1, cap, x.shape[-1])[u]


def hp_of(sqa, c, q, ragged, before=0):
    """How far probabilities may be off for the product with V: by the form that the call takes."""
    B, Hq, T, D = q.shape
    if q.dtype == torch.float32:
        return 0.0
    return 2.0 ** -8 if sqa.q4_plan(c.capacities[0], B, T, Hq, c.Hkv, D, "bf16", before, ragged)["rounded_probs"] else 2.0 ** -15


def check(hp, c, q, out, lse, before, new, cap, sink, what):
    """Every unit against the definition; before and new per sequence, cap their slots."""
    B, Hq, T, D = q.shape
    g = Hq // c.Hkv
    for b in range(B):
        n, end = new[b], before[b] + new[b]
        if n == 0:
            continue
        at = Q.held(end, cap[b], sink)[:min(end, cap[b])]
        at = torch.tensor(at, device=DEV)
        seen = at <= before[b] + torch.arange(n, device=DEV)[:, None]
        for h in range(c.Hkv):
            u = b * c.Hkv + h
            K, V = (Q.values(unit(c, x, u)[:len(at)], unit(c, x + "_scale", u)[:len(at)]) for x in ("K", "V"))
            want, want_lse, bound, lse_bound = Q.attention(q[b, h * g:(h + 1) * g, :n], K, V, seen, q.dtype, hp)
            got = out[b, :n, h * g:(h + 1) * g].transpose(0, 1).double()
            assert bool(((got - want).abs() <= bound).all()), (what, b, h, float(((got - want).abs() / bound).max()))
            off = (lse[b, h * g:(h + 1) * g, :n].double() - want_lse).abs()
            assert bool((off <= lse_bound).all()), (what, b, h, "lse", float((off / lse_bound).max()))


SHAPES = [  # B, T, before, Hq, Hkv
    (1, 1, 0, 1, 1), (2, 1, 14, 2, 1), (1, 1, 15, 3, 3), (3, 1, 30, 8, 2), (1, 1, 31, 1, 1), (2, 1, 32, 16, 1), (1, 1, 33, 17, 1),
    (2, 1, 1000, 8, 1), (1, 1, 5000, 12, 4), (40, 1, 200, 8, 8), (1, 1, 16000, 8, 2), (1, 5, 0, 4, 2), (2, 16, 0, 1, 1), (1, 17, 3, 2, 2),
    (2, 4, 500, 24, 2), (1, 33, 70, 3, 1), (1, 64, 0, 4, 4), (3, 40, 300, 5, 1), (1, 130, 1, 8, 2), (2, 257, 90, 4, 1), (1, 200, 3000, 2, 2)]


@pytest.mark.parametrize("blocked", [False, True])
@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
def test_attention(sqa, dtype, D, blocked):
    dt = R.DT[dtype]
    for i, (B, T, before, Hq, Hkv) in enumerate(SHAPES):
        gen = generator(100 + i)
        cap = before + T + 2
        c = filled(sqa, B, Hkv, D, cap, 0, blocked, gen)
        q = (torch.randn(B, Hq, T, D, generator=gen, device=DEV) * 1.5).to(dt)
        out, lse = sqa.q4_attention(q, before, c)
        check(hp_of(sqa, c, q, False, before), c, q, out, lse, [before] * B, [T] * B, [cap] * B, 0, (B, T, before, Hq, Hkv))
        again = sqa.q4_attention(q, before, c)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


WIDE = [  # B, T, before, Hq, Hkv, capacity (0: room for all), sinks -> slot splits: chunks whose workgroups have 128 rows
    (4, 520, 70, 16, 8, 0, 0, 1), (8, 300, 0, 32, 8, 0, 0, 1), (16, 129, 63, 16, 16, 0, 0, 1), (32, 96, 63, 16, 16, 0, 0, 1), (1, 128, 8000, 64, 8, 0, 0, 7), (2, 257, 7000, 16, 8, 0, 0, 6),
    (8, 130, 400, 32, 8, 200, 4, 1), (4, 900, 1500, 16, 4, 1000, 4, 1), (3, 1000, 600, 12, 12, 1000, 0, 1), (16, 128, 190, 16, 16, 300, 7, 1),
    (260, 1, 500, 128, 1, 0, 0, 1), (300, 1, 900, 96, 1, 333, 4, 1), (1, 3, 0, 200, 1, 0, 0, 0)]


@pytest.mark.parametrize("blocked", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_many_rows(sqa, D, blocked):
    """Sums joined over workgroups, tiles of slots that end inside a block, rows behind the last, chunks that turn a ring."""
    for i, (B, T, before, Hq, Hkv, cap, sink, splits) in enumerate(WIDE):
        gen = generator(200 + i)
        cap = cap or before + T + 2
        c = filled(sqa, B, Hkv, D, cap, sink, blocked, gen)
        q = (torch.randn(B, Hq, T, D, generator=gen, device=DEV) * 1.5).bfloat16()
        plan = sqa.q4_plan(cap, B, T, Hq, Hkv, D, "bf16", before)
        assert splits == 0 or plan["rows"] == 128 and plan["slot_splits"] == splits          # (0: one query head group of many, whatever the plan)
        out, lse = sqa.q4_attention(q, before, c)
        check(2.0 ** -8, c, q, out, lse, [before] * B, [T] * B, [cap] * B, sink, (B, T, before, Hq, Hkv))
        again = sqa.q4_attention(q, before, c)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


MIDDLE = [  # B, T, before, Hq, Hkv, capacity (0: room for all), sinks -> waves, slot splits: chunks whose workgroups have 32 rows
    (8, 9, 3200, 32, 16, 0, 0, 8, 2), (2, 127, 7000, 8, 8, 0, 0, 8, 4), (16, 20, 2500, 32, 16, 900, 4, 4, 1), (32, 9, 500, 64, 32, 0, 0, 2, 1),
    (1, 33, 13000, 16, 16, 0, 0, 8, 8), (16, 31, 1650, 16, 16, 1600, 0, 8, 1)]


@pytest.mark.parametrize("blocked", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_two_tiles_of_rows(sqa, D, blocked):
    """32 rows a workgroup: every number of waves, sums joined, a second tile with one row or none but the first's last again, rings that turn."""
    for i, (B, T, before, Hq, Hkv, cap, sink, waves, splits) in enumerate(MIDDLE):
        gen = generator(250 + i)
        cap = cap or before + T + 2
        c = filled(sqa, B, Hkv, D, cap, sink, blocked, gen)
        q = (torch.randn(B, Hq, T, D, generator=gen, device=DEV) * 1.5).bfloat16()
        plan = sqa.q4_plan(cap, B, T, Hq, Hkv, D, "bf16", before)
        assert (plan["rows"], plan["waves"], plan["slot_splits"]) == (32, waves, splits)
        out, lse = sqa.q4_attention(q, before, c)
        check(2.0 ** -15, c, q, out, lse, [before] * B, [T] * B, [cap] * B, sink, (B, T, before, Hq, Hkv))
        again = sqa.q4_attention(q, before, c)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


RINGS = [  # capacity, sinks, T, before
    (40, 0, 1, 39), (40, 0, 1, 40), (40, 4, 1, 41), (571, 4, 1, 1500), (16, 15, 1, 90), (1, 0, 1, 7), (33, 1, 5, 31), (100, 4, 96, 400), (64, 0, 64, 64),
    (70, 6, 20, 55), (300, 2, 130, 250), (2000, 4, 3, 100000), (5000, 0, 1, 2 ** 31 - 3),
    # (chunks that hide whole tiles of the ring from their first rows: in the middle, at both ends, behind sinks)
    (300, 0, 300, 400), (300, 0, 250, 640), (320, 40, 280, 330), (520, 3, 400, 1500), (520, 100, 420, 700), (257, 0, 200, 315)]


@pytest.mark.parametrize("blocked", [False, True])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_rings(sqa, dtype, D, blocked):
    """The sinks and the newest tokens, of a chunk's tokens each those that are not behind it."""
    dt = R.DT[dtype]
    for i, (cap, sink, T, before) in enumerate(RINGS):
        for B, Hq, Hkv in ((2, 8, 2), (1, 3, 3)):
            gen = generator(300 + i)
            c = filled(sqa, B, Hkv, D, cap, sink, blocked, gen)
            q = (torch.randn(B, Hq, T, D, generator=gen, device=DEV) * 1.5).to(dt)
            out, lse = sqa.q4_attention(q, before, c)
            # (what a slot holds depends on the position modulo the ring: long histories by a shorter one that ends the same way)
            ring = cap - sink
            short = before if before < 4 * cap + 200 else sink + ring + (before - sink) % ring + ring
            check(hp_of(sqa, c, q, False, before), c, q, out, lse, [short] * B, [T] * B, [cap] * B, sink, (cap, sink, T, before))


def test_ragged(sqa):
    """Own lengths, positions and budgets; padding and sequences that take no part stay as they were."""
    for dtype, D, T in (("bf16", 128, 9), ("f32", 64, 9), ("bf16", 64, 70), ("bf16", 128, 300), ("bf16", 64, 12), ("bf16", 128, 12)):
        dt, gen = R.DT[dtype], generator(17)
        B, cap, sink = 6, 700, 4
        Hq, Hkv = {300: (24, 8), 12: (192, 64)}.get(T, (6, 2))             # (128, 32 and 16 rows a workgroup)
        new = [T, 1, 0, T // 2, T, 1]
        before = [0, 650, 5, 100, -1, 3000]
        budget = [700, 300, 700, 505, 700, 64]
        for blocked in (False, True):
            c = filled(sqa, B, Hkv, D, cap, sink, blocked, gen)
            q = torch.randn(B, Hq, T, D, generator=gen, device=DEV).to(dt)
            out, lse = torch.full((B, T, Hq, D), 5.0, dtype=dt, device=DEV), torch.full((B, Hq, T), 6.0, device=DEV)
            status = ints([0])
            opts = sqa.batch_opts(prompt_len=ints(new), new_pos_seq=ints(before), budget_seq=ints(budget), status=status)
            sqa.q4_attention(q, 0, c, out=out, lse=lse, opts=opts)
            part = [n if p >= 0 else 0 for n, p in zip(new, before)]
            check(hp_of(sqa, c, q, True), c, q, out, lse, before, part, budget, sink, (dtype, D, T))
            assert int(status) == 0
            for b, n in enumerate(part):
                assert bool((out[b, n:] == 5).all()) and bool((lse[b, :, n:] == 6).all())


def test_what_is_not_seen_changes_nothing(sqa):
    """Unwritten slots, later tokens of the chunk and other units' rows hold anything: not a bit changes."""
    for dtype, D in (("bf16", 128), ("bf16", 64), ("f32", 128)):
        dt = R.DT[dtype]
        for B, T, before, Hq, Hkv, cap, sink in ((2, 1, 45, 4, 2, 100, 0), (1, 7, 20, 6, 2, 60, 0), (1, 40, 200, 8, 4, 1000, 0), (1, 20, 95, 4, 2, 64, 4),
                                                 (1, 300, 10, 8, 2, 400, 0), (16, 9, 850, 64, 32, 1000, 0), (16, 9, 900, 64, 32, 850, 4),
                                                 (8, 300, 50, 32, 8, 400, 0), (8, 130, 400, 32, 8, 200, 4)):
            if dt == torch.float32 and B * T > 1000:
                continue
            gen = generator(23)
            c = filled(sqa, B, Hkv, D, cap, sink, False, gen)
            q = torch.randn(B, Hq, T, D, generator=gen, device=DEV).to(dt)
            clean = [x.clone() for x in sqa.q4_attention(q, before, c)]
            end = before + T
            for u in range(B * Hkv):
                for x in (c.K[0], c.V[0], c.K_scale[0], c.V_scale[0]):
                    x.view(B * Hkv, cap, -1)[u, min(end, cap):] = 255
            assert all(torch.equal(a, b) for a, b in zip(clean, sqa.q4_attention(q, before, c)))
            # the last token: NaN for the rows that see it, not a bit for the others
            slot = Q.slot_of(end - 1, cap, sink)
            for name in ("K_scale", "V_scale"):
                keep = getattr(c, name)[0].clone()
                getattr(c, name)[0].view(B * Hkv, cap, -1)[:, slot, 0] = 255
                out, lse = sqa.q4_attention(q, before, c)
                assert torch.equal(out[:, :T - 1], clean[0][:, :T - 1]) and torch.equal(lse[:, :, :T - 1], clean[1][:, :, :T - 1]), (dtype, D, T, name)
                if name == "K_scale":
                    assert bool(out[:, T - 1].isnan().all()) and bool(lse[:, :, T - 1].isnan().all())
                else:
                    assert bool(out[:, T - 1, :, :32].isnan().all()) and torch.equal(out[:, T - 1, :, 32:], clean[0][:, T - 1, :, 32:])
                    assert torch.equal(lse, clean[1])
                getattr(c, name)[0].copy_(keep)


def test_extreme_logits_and_queries(sqa):
    """Logits far from 0, all of them equal, one that outweighs the others; a query that is not finite gives its own row alone NaN."""
    for dtype, D in (("bf16", 128), ("f32", 64)):
        dt, gen = R.DT[dtype], generator(29)
        c = filled(sqa, 1, 1, D, 300, 0, False, gen)
        q = torch.randn(1, 6, 1, D, generator=gen, device=DEV)
        q[0, 1] *= 60
        q[0, 2] = 0
        q[0, 3] = Q.values(c.K[0][0, 0, 77], c.K_scale[0][0, 0, 77]).float() * 40
        q[0, 4] = -Q.values(c.K[0][0, 0, 299], c.K_scale[0][0, 0, 299]).float() * 30
        q = q.to(dt)
        out, lse = sqa.q4_attention(q, 299, c)
        check(hp_of(sqa, c, q, False, 299), c, q, out, lse, [299], [1], [300], 0, dtype)
        q2 = q.clone()
        q2[0, 5, 0, 3], q2[0, 2, 0, 0] = math.nan, math.inf
        got = sqa.q4_attention(q2, 299, c)
        keep = [0, 1, 3, 4]
        assert torch.equal(got[0][:, :, keep], out[:, :, keep]) and torch.equal(got[1][:, keep], lse[:, keep])
        assert bool(got[0][0, 0, 5].isnan().all()) and bool(got[0][0, 0, 2].isnan().all())


def test_blocks_that_are_not_there(sqa):
    """A unit with a block outside the pools, and a sequence that overwrote its own tokens: zeros, -inf, reported; the others as they were."""
    for T, before, cap, Hq, Hkv in ((1, 40, 100, 4, 2), (1, 5000, 6000, 4, 2), (30, 60, 100, 4, 2), (200, 50, 300, 4, 2), (300, 20, 400, 64, 32), (9, 1700, 1800, 256, 64), (128, 7900, 8100, 32, 4)):
        gen = generator(31)
        B, D, g = 2, 128, Hq // Hkv
        c = filled(sqa, B, Hkv, D, cap, 0, True, gen)
        q = torch.randn(B, Hq, T, D, generator=gen, device=DEV).bfloat16()
        clean = sqa.q4_attention(q, before, c)
        for entry in sorted({0, (before + T - 1) // 16, (before + T) // 32}):
            for value in (-1, c.K[0].shape[0], 2 ** 31 - 1):
                was = c.block_table[0].clone()
                c.block_table[0][1, entry] = value
                status = ints([0])
                out, lse = sqa.q4_attention(q, before, c, opts=sqa.batch_opts(status=status))
                assert int(status) == 2
                # (rows that see no slot of the block may be there all the same: a chunk's first ones)
                sees = torch.arange(before, before + T, device=DEV) >= entry * 16
                assert bool((out[0, sees, g:2 * g] == 0).all()) and bool((lse[0, g:2 * g, sees] == -math.inf).all())
                assert torch.equal(out[0, :, :g], clean[0][0, :, :g]) and torch.equal(out[0, :, 2 * g:], clean[0][0, :, 2 * g:]) and torch.equal(out[1], clean[0][1]) and torch.equal(lse[1], clean[1][1])
                c.block_table[0].copy_(was)
        c.block_table[0][:, (before + T + 15) // 16:] = -1                   # (entries behind the last token are not read)
        assert all(torch.equal(a, b) for a, b in zip(clean, sqa.q4_attention(q, before, c)))
    c = filled(sqa, 2, 1, 64, 50, 40, False, generator(1))
    status, q = ints([0]), torch.randn(2, 2, 12, 64, device=DEV)
    out, lse = sqa.q4_attention(q, 0, c, opts=sqa.batch_opts(new_pos_seq=ints([45, 30]), status=status))
    assert int(status) == 6 and bool((out[0] == 0).all()) and bool((lse[0] == -math.inf).all()) and bool(lse[1].isfinite().all())


def test_far_into_large_pools(sqa):
    """Rows beyond 4 GiB of codes."""
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("less than 24 GiB free")
    D, Hkv, cap, gen = 128, 8, 9_500_000, generator(2)
    c = sqa.Q4Caches([cap], 1, Hkv, D, DEV)
    n = 3000
    for x in (c.K[0], c.V[0]):
        x[0, :, :n].copy_(torch.randint(0, 256, (Hkv, n, D // 2), generator=gen, device=DEV))
    for x in (c.K_scale[0], c.V_scale[0]):
        x[0, :, :n].copy_(torch.randint(123, 128, (Hkv, n, D // 32), generator=gen, device=DEV))
    q = torch.randn(1, 16, 1, D, generator=gen, device=DEV).bfloat16()
    out, lse = sqa.q4_attention(q, n - 1, c)
    small = sqa.Q4Caches([n], 1, Hkv, D, DEV)
    for a, b in ((small.K, c.K), (small.V, c.V), (small.K_scale, c.K_scale), (small.V_scale, c.V_scale)):
        a[0].copy_(b[0][:, :, :n])
    assert all(torch.equal(x, y) for x, y in zip((out, lse), sqa.q4_attention(q, n - 1, small)))


def test_graphs_and_streams(sqa):
    """Append and attention of a decode step in two graphs that share a workspace, replayed in turn as positions move on."""
    B, Hq, Hkv, D, cap, sink, dt = 3, 8, 2, 128, 90, 4, torch.bfloat16
    gen = generator(41)
    c = [sqa.Q4Caches([cap], B, Hkv, D, DEV, n_sink=sink, blocked=True, block_seed=s) for s in (1, 2)]
    mirror = [sqa.Q4Caches([cap], B, Hkv, D, DEV, n_sink=sink, blocked=True, block_seed=s) for s in (1, 2)]
    ws = sqa.q4_workspace(c[0], Hq, 1)
    x = torch.zeros(B, 1, Hq + 2 * Hkv, D, dtype=dt, device=DEV)
    first, q = ints([0] * B), torch.zeros(B, Hq, 1, D, dtype=dt, device=DEV)
    prep = sqa.head_prep(rope=sqa.rope_table(300, D, device=DEV))
    opts = sqa.batch_opts(new_pos_seq=first)
    outs = [(torch.zeros(B, 1, Hq, D, dtype=dt, device=DEV), torch.zeros(B, Hq, 1, device=DEV)) for _ in c]

    def step(cache, out, workspace):
        sqa.q4_append(x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], 0, cache, prep=prep, q=x[:, :, :Hq], q_out=q, opts=opts)
        return sqa.q4_attention(q, 0, cache, out=out[0], lse=out[1], workspace=workspace, opts=opts)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    first.fill_(-1)
    with torch.cuda.stream(side):
        step(c[0], outs[0], ws)
        for cache, out in zip(c, outs):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=side):
                step(cache, out, ws)
    torch.cuda.current_stream().wait_stream(side)
    for p in range(130):
        x.copy_(torch.randn(x.shape, generator=gen, device=DEV))
        first.copy_(ints([p, p // 2, p if p % 3 else -1]))
        for k in (0, 1):
            graphs[k].replay()
        if p % 13 == 0 or p > 125:
            torch.cuda.synchronize()
        for k in (0, 1):
            got = [t.clone() for t in outs[k]]
            want = step(mirror[k], [t.clone() for t in outs[k]], None)
            assert all(torch.equal(a, b) for a, b in zip(got, want)), p


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_serving_loop(sqa, dtype):
    """Sequences join with prompts in chunks, grow token by token, turn their rings and leave; tables and maps made on the GPU, several axes; every
    step's attention against 64 bits over the tokens that a list per sequence says are held."""
    B, Hq, Hkv, D, cap, sink, dt = 5, 6, 2, 64, 72, 4, R.DT[dtype]
    rng, gen = random.Random(7), generator(51)
    per = -(-cap // 16)
    c = sqa.Q4Caches([cap], B, Hkv, D, DEV, n_sink=sink, blocked=True, n_blocks=B * Hkv * per - 6)
    n_blocks = c.K[0].shape[0]
    held, free, count, status = ints([0] * B), torch.arange(n_blocks, dtype=torch.int32, device=DEV), ints([n_blocks]), ints([0])
    prep = sqa.head_prep((1 + 0.1 * torch.randn(D, generator=gen, device=DEV)).to(dt), (1 + 0.1 * torch.randn(D, generator=gen, device=DEV)).to(dt), 1e-6,
                         sqa.rope_table(400, D, device=DEV))
    T = 24
    ws = sqa.q4_workspace(c, Hq, T)
    length = [0] * B
    for step in range(40):
        new = []
        for b in range(B):
            if length[b] and rng.random() < 0.06:
                length[b] = 0                          # (it leaves; another takes its place)
                new.append(0)
            else:
                new.append(rng.randrange(5, T + 1) if length[b] < 30 and rng.random() < 0.5 else 1)
        tokens = ints([p + n for p, n in zip(length, new)])
        status.zero_()
        sqa.block_assign(c.block_table[0], tokens, held, free, count, cap, status)
        has = held.tolist()
        # a sequence without room waits
        new = [n if has[b] * 16 >= min(length[b] + n, cap) else 0 for b, n in enumerate(new)]
        opts = sqa.batch_opts(prompt_len=ints(new), new_pos_seq=ints(length), status=status)
        status.zero_()
        rows = sqa.slot_map(c.block_table[0], cap, T, 0, sink, out=torch.empty(B, Hkv, T, dtype=torch.int32, device=DEV), opts=opts)
        x = torch.randn(B, T, Hq + 2 * Hkv, D, generator=gen, device=DEV).to(dt)
        pos = torch.randint(0, 400, (3, B, T), generator=gen, device=DEV).to(torch.int32)
        q = sqa.q4_append(x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], 0, c, prep=prep, q=x[:, :, :Hq], opts=opts, axes=sqa.rope_axes(pos, [8, 12, 12]), slot_map=rows)
        out, lse = sqa.q4_attention(q, 0, c, workspace=ws, opts=opts)
        assert int(status) == 0
        safe = [n if n else 0 for n in new]
        # (units of sequences without blocks have -1 in their tables: looked at only where there are tokens)
        table = c.block_table[0].clone()
        c.block_table[0].clamp_(min=0)
        check(hp_of(sqa, c, q, True), c, q, out, lse, length, safe, [cap] * B, sink, step)
        c.block_table[0].copy_(table)
        got = sqa.q4_read(c, 0, cap, torch.float32, opts=sqa.batch_opts(prompt_len=ints([min(p + n, cap) if n else 0 for p, n in zip(length, new)])))
        for b, n in enumerate(new):
            if n:
                last = Q.slot_of(length[b] + n - 1, cap, sink)
                assert torch.equal(got[1][b, :, last].double(), Q.pack(x[b, n - 1, Hq + Hkv:])[0])
        length = [p + n for p, n in zip(length, new)]
