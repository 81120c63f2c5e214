"""The forms of the row kernels that take several groups of heads in a wave (large chunks): rotation on axes (sqa_qk_norm_rope_ex,
sqa_chunk_append_ex) with four or five groups and rows into a cache in 4 bits with four, in either type and head size; waves that hold queries and
keys, last runs that are not full, head counts that are no multiple of what a wave's lanes hold.  Against q4_reference.py's definitions and bounds."""
import math

import pytest
import torch

import chunk_reference as R
import q4_reference as Q
import test_gpu_q4_rows as rows_test

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)]
HEADS = {8: [(33, 11, 4), (60, 12, 5), (54, 9, 5)], 4: [(18, 6, 4), (27, 9, 5), (28, 7, 5), (26, 13, 4)], 2: [(9, 3, 4), (15, 3, 5), (15, 1, 5)]}
B, T, NEW, FIRST = 3, 401, [401, 7, 333], [0, 12, 3]


@pytest.fixture(scope="module")
def sqa():
    from paper_2404_04793_amd import binding
    return binding


def generator(seed):
    return torch.Generator(DEV).manual_seed(seed)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def heads_of_a_wave(dtype, D):
    return 64 * (8 if dtype == "bf16" else 4) // D


def groups(Hq, Hkv, hpw):
    return -(-Hq // hpw) + -(-Hkv // hpw)


def axis_groups(n):
    """Groups of heads that a wave takes of n, by the rule of sqa_chunk_rows.hip, for chunks of this file's size."""
    U = 5 if -(-n // 5) * 5 < -(-n // 4) * 4 else 4
    assert B * T * -(-n // U) >= 2048
    return U


def cases(dtype, D):
    hpw = heads_of_a_wave(dtype, D)
    for i, (Hq, Hkv, U) in enumerate(HEADS[hpw]):
        n = groups(Hq, Hkv, hpw)
        assert axis_groups(n) == U and B * T * -(-n // 4) >= 2048
        assert any(lo < -(-Hq // hpw) < lo + U for lo in range(0, n, U)) or n % U                  # (a wave with both kinds, or a run that is not full)
        yield i, Hq, Hkv


def projection(Hq, Hkv, D, dt, gen):
    x = torch.randn(B, T + 1, (Hq + 2 * Hkv) * D, generator=gen, device=DEV).to(dt)[:, 1:].unflatten(2, (-1, D))
    for b in range(B):
        x[b, NEW[b]:] = math.nan                     # (padding is not read)
    return x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]


def on_axes(sqa, i, D, dt, gen):
    """norm weights, table, prep, positions, axes, the axis of each pair"""
    turns, interleaved = bool(i % 2), i % 3 == 1
    half = D // 2
    pairs = [half - 2 * (half // 3), half // 3, half // 3]
    w = [(1 + 0.2 * torch.randn(D, generator=gen, device=DEV)).to(dt) for _ in range(2)]
    rope = sqa.rope_table(2000, D, device=DEV)
    pos = torch.randint(0, 2000, (3, B, T), generator=gen, device=DEV).to(torch.int32)
    for b in range(B):
        pos[:, b, NEW[b]:] = 1 << 30                 # (nor are these)
    return w, rope, interleaved, sqa.head_prep(w[0], w[1], 1e-6, rope, interleaved), pos, sqa.rope_axes(pos, pairs, turns), Q.axis_of(pairs, turns)


def close(got, want, bound, dt):
    return bool(((got.double() - want).abs() <= bound + R.HALF[dt] * want.abs() * 1.0001 + 1e-30).all())


@pytest.mark.parametrize("dtype,D", TYPES)
def test_rotation_on_axes(sqa, dtype, D):
    dt = R.DT[dtype]
    for i, Hq, Hkv in cases(dtype, D):
        gen = generator(500 + i)
        q, k, _ = projection(Hq, Hkv, D, dt, gen)
        w, rope, interleaved, prep, pos, axes, axis = on_axes(sqa, i, D, dt, gen)
        status = ints([0])
        opts = sqa.batch_opts(prompt_len=ints(NEW), status=status)
        outs = [torch.full((B, H, T, D), 7.0, dtype=dt, device=DEV) for H in (Hq, Hkv)]
        sqa.qk_norm_rope(q, k, 0, prep, *outs, opts=opts, axes=axes)
        assert int(status) == 0
        for out, src, weight in zip(outs, (q, k), w):
            for b, n in enumerate(NEW):
                want, bound = Q.norm_rope(src[b, :n], weight, 1e-6, rope, interleaved, pos[:, b, :n], axis)
                assert close(out[b, :, :n].transpose(0, 1), want, bound, dt), (Hq, Hkv, b)
                assert bool((out[b, :, n:] == 7).all())
        for which in (0, 1):                         # queries alone, keys alone
            alone = [torch.full_like(o, 7.0) if j == which else None for j, o in enumerate(outs)]
            sqa.qk_norm_rope(q if which == 0 else None, k if which == 1 else None, 0, prep, *alone, opts=opts, axes=axes)
            assert torch.equal(alone[which], outs[which])


@pytest.mark.parametrize("layout", ["dense", "blocked", "packed"])
@pytest.mark.parametrize("dtype,D", TYPES)
def test_append_on_axes(sqa, dtype, D, layout):
    """Into a cache that is not in 4 bits; one unit does not take the chunk, the others of its wave do."""
    dt = R.DT[dtype]
    for i, Hq, Hkv in cases(dtype, D):
        gen = generator(600 + i)
        q, k, v = projection(Hq, Hkv, D, dt, gen)
        w, rope, interleaved, prep, pos, axes, axis = on_axes(sqa, i, D, dt, gen)
        c = R.fill(R.make_cache(sqa, layout, B, Hkv, D, dt, [f + n + 2 for f, n in zip(FIRST, NEW)]), FIRST, gen, value=5.0)
        left = (2, Hkv // 2)
        c.head[0][left] = 1                          # (its ring has moved)
        K0, V0, score0, pos0, state0 = R.snapshot(c)
        status = ints([0])
        opts = sqa.batch_opts(prompt_len=ints(NEW), new_pos_seq=ints(FIRST), status=status)
        q_out = torch.full((B, Hq, T, D), 7.0, dtype=dt, device=DEV)
        sqa.chunk_append(k, v, 0, c, prep=prep, q=q, q_out=q_out, opts=opts, axes=axes)
        assert int(status) == 8
        want_q = torch.full_like(q_out, 7.0)
        sqa.qk_norm_rope(q, None, 0, prep, want_q, opts=opts, axes=axes)
        assert torch.equal(q_out, want_q)
        for b, (n, first) in enumerate(zip(NEW, FIRST)):
            want, bound = Q.norm_rope(k[b, :n], w[1], 1e-6, rope, interleaved, pos[:, b, :n], axis)
            for h in range(Hkv):
                if (b, h) == left:
                    continue
                K, V = R.rows_of(c, b, h, first + n)
                assert close(K[first:], want[:, h], bound[:, h], dt) and torch.equal(V[first:], v[b, :n, h]), (Hq, Hkv, b, h)
                _, _, score, at = c.unit(0, b, h)
                assert torch.equal(at[:first + n], torch.arange(first + n, dtype=torch.int32, device=DEV)) and bool((score[first:first + n] == 0).all())
                assert c.state[0][b, h].tolist() == [first + n, 0, -2, 0]
                # what was written as it was before: then nothing else may differ
                idx = c.unit_kv_rows(0, b, h)[2][first:first + n]
                for now, old in ((c.K[0], K0), (c.V[0], V0)):
                    now.view(-1, D)[idx] = old.view(-1, D)[idx]
                lo = c.offsets_host[0][b * Hkv + h] if c.offsets_host[0] is not None else None
                for now, old in ((c.score[0], score0), (c.pos[0], pos0)):
                    if lo is None:
                        now[b, h, first:first + n] = old[b, h, first:first + n]
                    else:
                        now[lo + first:lo + first + n] = old[lo + first:lo + first + n]
                c.state[0][b, h] = state0[b, h]
        assert R.same([K0, V0, score0, pos0, state0], R.snapshot(c))


@pytest.mark.parametrize("ring", [None, (440, 4)])
@pytest.mark.parametrize("blocked", [False, True])
@pytest.mark.parametrize("dtype,D", TYPES)
def test_rows_into_4_bits(sqa, dtype, D, blocked, ring):
    """Every row in its slot and no other byte changed, with a map of the slots and without."""
    dt = R.DT[dtype]
    for i, Hq, Hkv in cases(dtype, D):
        gen = generator(700 + i)
        q, k, v = projection(Hq, Hkv, D, dt, gen)
        first = FIRST if ring is None else [39, 900, 2 ** 20 + 7]
        cap, sink = ring or (max(f + n for f, n in zip(FIRST, NEW)) + 3, 0)
        status = ints([0])
        opts = sqa.batch_opts(prompt_len=ints(NEW), new_pos_seq=ints(first), status=status)
        results = []
        for mapped in (False, True):
            c = rows_test.caches(sqa, B, Hkv, D, cap, sink, blocked, fill=0x5a)
            rows = sqa.slot_map(c.block_table[0], cap, T, 0, sink, out=torch.zeros(B, Hkv, T, dtype=torch.int32, device=DEV), opts=opts) if mapped else None
            q_out = torch.full((B, Hq, T, D), 7.0, dtype=dt, device=DEV)
            sqa.q4_append(k, v, 0, c, q=q, q_out=q_out, opts=opts, slot_map=rows)
            results.append(rows_test.snapshot(c) + [q_out])
        assert int(status) == 0 and R.same(*results)
        touched = torch.zeros(c.K[0].view(-1, D // 2).shape[0], dtype=torch.bool, device=DEV)
        for b, n in enumerate(NEW):
            assert torch.equal(q_out[b, :, :n], q[b, :n].transpose(0, 1)) and bool((q_out[b, :, n:] == 7).all())
            slots = torch.tensor([Q.slot_of(p, cap, sink) for p in range(first[b], first[b] + n)], device=DEV)
            for name, src in (("K", k), ("V", v)):
                _, code, power = Q.pack(src[b, :n].transpose(0, 1))
                for h in range(Hkv):
                    u = b * Hkv + h
                    assert torch.equal(Q.codes(rows_test.unit(c, name, u)[slots]), code[h]), (Hq, Hkv, name, u)
                    assert torch.equal(rows_test.unit(c, name + "_scale", u)[slots], power[h])
                    touched[c.block_table[0][u].long()[slots // 16] * 16 + slots % 16 if blocked else u * cap + slots] = True
        for x in (c.K, c.V, c.K_scale, c.V_scale):
            assert bool((x[0].view(touched.shape[0], -1)[~touched] == 0x5a).all())


@pytest.mark.parametrize("plain", [False, True])
@pytest.mark.parametrize("dtype,D", TYPES)
def test_prepared_keys_into_4_bits(sqa, dtype, D, plain):
    """Norm and rotation (by the token's position, or on axes) in fp32, then one rounding; one sequence's keys have no room, its queries are there."""
    dt = R.DT[dtype]
    for i, Hq, Hkv in cases(dtype, D):
        gen = generator(800 + i)
        q, k, v = projection(Hq, Hkv, D, dt, gen)
        w, rope, interleaved, prep, pos, axes, axis = on_axes(sqa, i, D, dt, gen)
        if plain:
            pos, axes, axis = (ints(FIRST)[:, None] + torch.arange(T, dtype=torch.int32, device=DEV))[None], None, [0] * 64
        cap = 404
        c, status = rows_test.caches(sqa, B, Hkv, D, cap, 100), ints([0])
        first, new = [0, 12, 90], NEW                # (90 + 333 tokens past 404 slots, 304 of them a ring)
        if plain:
            pos = (ints(first)[:, None] + torch.arange(T, dtype=torch.int32, device=DEV))[None]
        q_out = torch.full((B, Hq, T, D), 7.0, dtype=dt, device=DEV)
        sqa.q4_append(k, v, 0, c, prep=prep, q=q, q_out=q_out, axes=axes, opts=sqa.batch_opts(prompt_len=ints(new), new_pos_seq=ints(first), status=status))
        assert int(status) == 6
        for b, n in enumerate(new):
            want, bound = Q.norm_rope(q[b, :n], w[0], 1e-6, rope, interleaved, pos[:, b, :n], axis)
            assert close(q_out[b, :, :n].transpose(0, 1), want, bound, dt) and bool((q_out[b, :, n:] == 7).all())
            if b == 2:
                assert all(not bool(x[0][b].any()) for x in (c.K, c.V, c.K_scale, c.V_scale))
                continue
            want, bound = (t.transpose(0, 1) for t in Q.norm_rope(k[b, :n], w[1], 1e-6, rope, interleaved, pos[:, b, :n], axis))
            at = slice(first[b], first[b] + n)
            mine = c.K_scale[0][b, :, at]
            _, _, power = Q.pack(want)
            # (another power only where the largest is as near to 7 times one as the arithmetic is exact)
            top, slack = want.abs().unflatten(-1, (-1, 32)).amax(-1), bound.unflatten(-1, (-1, 32)).amax(-1)
            edge = 7 * Q.two_to(torch.minimum(power, mine).long() - 127)
            assert bool(((power == mine) | ((top - edge).abs() <= slack)).all())
            scale = Q.two_to(mine.long() - 127).repeat_interleave(32, -1)
            grid = torch.tensor(Q.GRID, dtype=torch.float64, device=DEV)
            nearest = ((want.abs() / scale)[..., None] - grid).abs().amin(-1) * scale
            assert bool(((Q.values(c.K[0][b, :, at], mine) - want).abs() <= nearest + 2 * bound).all())
            assert torch.equal(Q.values(c.V[0][b, :, at], c.V_scale[0][b, :, at]), Q.pack(v[b, :n].transpose(0, 1))[0])
