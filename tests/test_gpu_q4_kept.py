"""What a cache in 4 bits holds, against a list of every token kept beside it: a serving loop, layers with budgets of their own, chunks that
fill a ring to its last slot; and the precision of calls with many heads and few rows."""
import random

import pytest
import torch

import chunk_reference as R
import q4_reference as Q
import test_gpu_q4_attention as attention_test

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


def rows_of(c, layer, u, slots):
    """(values of K, of V, bytes of K's groups) of unit u's slots."""
    cap, slots = c.capacities[layer], torch.as_tensor(slots, device=DEV)
    at = c.block_table[layer][u].long()[slots // 16] * 16 + slots % 16 if c.blocked else u * cap + slots
    pick = lambda x: x[layer].view(-1, x[layer].shape[-1])[at]
    return Q.values(pick(c.K), pick(c.K_scale)), Q.values(pick(c.V), pick(c.V_scale)), pick(c.K_scale)


def near(value, power, want, bound):
    """Keys that were rounded once from what the arithmetic's bound allows."""
    _, _, exact = Q.pack(want)
    top, slack = want.abs().unflatten(-1, (-1, 32)).amax(-1), bound.unflatten(-1, (-1, 32)).amax(-1)
    edge = 7 * Q.two_to(torch.minimum(exact, power).long() - 127)
    scale = Q.two_to(power.long() - 127).repeat_interleave(32, -1)
    grid = torch.tensor(Q.GRID, dtype=torch.float64, device=DEV)
    nearest = ((want.abs() / scale)[..., None] - grid).abs().amin(-1) * scale
    return bool(((exact == power) | ((top - edge).abs() <= slack)).all()) and bool(((value - want).abs() <= nearest + 2 * bound).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_serving_loop(sqa, dtype):
    """Sequences join with prompts in chunks, grow token by token, turn their rings, wait while the list is too short, and leave.  Every key is
    compared with its definition when it comes, and after every step all tokens that a sequence holds with the list; attention's keys and values are the list's."""
    B, Hq, Hkv, D, cap, sink, dt = 5, 6, 2, 64, 72, 4, R.DT[dtype]
    rng, gen, g = random.Random(19), generator(61), Hq // Hkv
    per = -(-cap // 16)
    c = sqa.Q4Caches([cap], B, Hkv, D, DEV, n_sink=sink, blocked=True, n_blocks=B * Hkv * per - 13)
    n_blocks = c.K[0].shape[0]
    held, free, count, status = ints([0] * B), torch.arange(n_blocks, dtype=torch.int32, device=DEV), ints([n_blocks]), ints([0])
    table, has, unused = c.block_table[0].tolist(), [0] * B, list(range(n_blocks))
    w = [(1 + 0.1 * torch.randn(D, generator=gen, device=DEV)).to(dt) for _ in range(2)]
    rope = sqa.rope_table(400, D, device=DEV)
    prep, pairs, axis = sqa.head_prep(w[0], w[1], 1e-6, rope), [8, 12, 12], Q.axis_of([8, 12, 12], False)
    T = 24
    ws = sqa.q4_workspace(c, Hq, T)
    kept = [[] for _ in range(B)]                    # of each sequence: (K, V) of every token, [Hkv, D] in 64 bits
    was_short = turned = waited = left = 0
    for step in range(60):
        new = []
        for b in range(B):
            if kept[b] and rng.random() < 0.05:
                kept[b], left = [], left + 1
                new.append(0)
            else:
                new.append(rng.randrange(5, T + 1) if len(kept[b]) < 30 and rng.random() < 0.5 else 1)
        tokens = [len(x) + n for x, n in zip(kept, new)]
        status.zero_()
        sqa.block_assign(c.block_table[0], ints(tokens), held, free, count, cap, status)
        short = Q.assign(table, tokens, has, unused, cap, Hkv)
        assert int(status) == (6 if short else 0) and held.tolist() == has and c.block_table[0].tolist() == table
        assert int(count) == len(unused) and free[:len(unused)].tolist() == unused
        was_short += short
        room = [n if has[b] * 16 >= min(len(kept[b]) + n, cap) else 0 for b, n in enumerate(new)]
        waited, new = waited + (room != new), room
        before = [len(x) for x in kept]
        opts = sqa.batch_opts(prompt_len=ints(new), new_pos_seq=ints(before), status=status)
        status.zero_()
        rows = sqa.slot_map(c.block_table[0], cap, T, 0, sink, out=torch.empty(B, Hkv, T, dtype=torch.int32, device=DEV), opts=opts) if step % 2 else None
        x = torch.randn(B, T, Hq + 2 * Hkv, D, generator=gen, device=DEV).to(dt)
        pos = torch.randint(0, 400, (3, B, T), generator=gen, device=DEV).to(torch.int32)
        q = sqa.q4_append(x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], 0, c, prep=prep, q=x[:, :, :Hq], opts=opts, axes=sqa.rope_axes(pos, pairs), slot_map=rows)
        out, lse = sqa.q4_attention(q, 0, c, workspace=ws, opts=opts)
        assert int(status) == 0
        hp = attention_test.hp_of(sqa, c, q, True)
        for b, n in enumerate(new):
            if n:
                slots = [Q.slot_of(p, cap, sink) for p in range(before[b], before[b] + n)]
                want, bound = Q.norm_rope(x[b, :n, Hq:Hq + Hkv], w[1], 1e-6, rope, False, pos[:, b, :n], axis)
                K, V = torch.empty(2, n, Hkv, D, dtype=torch.float64, device=DEV)
                for h in range(Hkv):
                    K[:, h], got_v, power = rows_of(c, 0, b * Hkv + h, slots)
                    assert near(K[:, h], power, want[:, h], bound[:, h])
                    V[:, h] = Q.pack(x[b, :n, Hq + Hkv + h])[0]
                    assert torch.equal(got_v, V[:, h])
                kept[b] += list(zip(K, V))
            if not kept[b]:
                continue
            at = Q.held(len(kept[b]), cap, sink)[:min(len(kept[b]), cap)]
            turned += len(kept[b]) > cap
            K, V = (torch.stack([kept[b][p][i] for p in at]) for i in (0, 1))                    # [slots, Hkv, D]
            for h in range(Hkv):
                got_k, got_v, _ = rows_of(c, 0, b * Hkv + h, list(range(len(at))))
                assert torch.equal(got_k, K[:, h]) and torch.equal(got_v, V[:, h]), (step, b, h)
                if n:
                    seen = torch.tensor(at, device=DEV) <= before[b] + torch.arange(n, device=DEV)[:, None]
                    heads = slice(h * g, (h + 1) * g)
                    want, want_lse, bound, lse_bound = Q.attention(q[b, heads, :n], K[:, h], V[:, h], seen, dt, hp)
                    assert bool(((out[b, :n, heads].transpose(0, 1).double() - want).abs() <= bound).all()), (step, b, h)
                    assert bool(((lse[b, heads, :n].double() - want_lse).abs() <= lse_bound).all()), (step, b, h)
    assert was_short and turned and waited and left


@pytest.mark.parametrize("blocked", [False, True])
def test_layers_with_budgets_of_their_own(sqa, blocked):
    """Three layers of one set, each with its budget: a call touches its layer alone, and its ring is its own."""
    B, Hq, Hkv, D, sink, dt, gen = 2, 6, 3, 128, 4, torch.bfloat16, generator(71)
    caps = [40, 101, 17]
    c = sqa.Q4Caches(caps, B, Hkv, D, DEV, n_sink=sink, blocked=blocked)
    kept = [[] for _ in caps]                        # of each layer: (K, V) [B, Hkv, D] of every token
    whole = lambda: [x[i].clone() for i in range(3) for x in (c.K, c.V, c.K_scale, c.V_scale)]
    for step in range(45):
        for layer, cap in enumerate(caps):
            T = 1 + (7 * step + layer) % 5
            before, others = len(kept[layer]), whole()
            x = torch.randn(B, T, Hq + 2 * Hkv, D, generator=gen, device=DEV).to(dt)
            q = sqa.q4_append(x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], before, c, layer=layer, q=x[:, :, :Hq])
            out, lse = sqa.q4_attention(q, before, c, layer=layer)
            kept[layer] += [tuple(Q.pack(x[:, t, lo:lo + Hkv])[0] for lo in (Hq, Hq + Hkv)) for t in range(T)]
            now = whole()
            assert all(torch.equal(a, b) for i, (a, b) in enumerate(zip(others, now)) if i // 4 != layer)
            if step % 11 and step < 43:
                continue
            n = before + T
            at = Q.held(n, cap, sink)[:min(n, cap)]
            K, V = (torch.stack([kept[layer][p][i] for p in at], 2) for i in (0, 1))              # [B, Hkv, slots, D]
            read = sqa.q4_read(c, 0, len(at), torch.float32, layer=layer)
            assert torch.equal(read[0].double(), K) and torch.equal(read[1].double(), V), (step, layer)
            seen = torch.tensor(at, device=DEV) <= before + torch.arange(T, device=DEV)[:, None]
            for b in range(B):
                for h in range(Hkv):
                    want, want_lse, bound, lse_bound = Q.attention(q[b, 2 * h:2 * h + 2], K[b, h], V[b, h], seen, dt, 2.0 ** -15)
                    assert bool(((out[b, :, 2 * h:2 * h + 2].transpose(0, 1).double() - want).abs() <= bound).all()), (step, layer, b, h)
                    assert bool(((lse[b, 2 * h:2 * h + 2].double() - want_lse).abs() <= lse_bound).all())


@pytest.mark.parametrize("cap,sink,T,before", [(13, 0, 4, 10), (13, 0, 13, 13), (13, 4, 9, 5), (13, 4, 9, 300), (64, 63, 1, 64), (300, 44, 256, 100)])
def test_chunks_that_fill_a_ring(sqa, cap, sink, T, before):
    """As many tokens past the capacity as the ring has slots are taken; one more is not, whether the host sees it or the GPU."""
    D, dt, gen = 64, torch.float32, generator(81)
    k, v = (torch.randn(1, T + 1, 1, D, generator=gen, device=DEV) for _ in range(2))
    q = torch.randn(1, 1, T + 1, D, generator=gen, device=DEV)
    for opts in (None, sqa.batch_opts(new_pos_seq=ints([before]), status=ints([0]))):
        c = sqa.Q4Caches([cap], 1, 1, D, DEV, n_sink=sink)
        first = torch.randn(1, sink, 1, D, generator=gen, device=DEV)
        if sink:
            sqa.q4_append(first, first, 0, c)
        sqa.q4_append(k[:, :T], v[:, :T], before, c, opts=opts)
        slots = [Q.slot_of(p, cap, sink) for p in range(before, before + T)]
        assert len(set(slots)) == T
        got = sqa.q4_read(c, 0, cap, dt)
        assert torch.equal(got[0][0, 0, slots].double(), Q.pack(k[0, :T, 0])[0]) and torch.equal(got[1][0, 0, slots].double(), Q.pack(v[0, :T, 0])[0])
        sqa.q4_attention(q[:, :, :T].contiguous(), before, c, opts=opts)
        rows = sqa.slot_map(None, cap, T, before, sink, out=torch.zeros(1, 1, T, dtype=torch.int32, device=DEV), opts=opts)
        assert rows[0, 0].tolist() == slots
    if T == cap - sink:
        for call in (lambda: sqa.q4_append(k, v, before, c), lambda: sqa.q4_attention(q, before, c)):
            with pytest.raises(sqa.SqaError) as e:
                call()
            assert e.value.code == 6
        keep = [x[0].clone() for x in (c.K, c.V, c.K_scale, c.V_scale)]
        status = ints([0])
        opts = sqa.batch_opts(new_pos_seq=ints([before]), status=status)
        sqa.q4_append(k, v, 0, c, opts=opts)
        assert int(status) == 6 and all(torch.equal(a, x[0]) for a, x in zip(keep, (c.K, c.V, c.K_scale, c.V_scale)))
        status.zero_()
        out, lse = sqa.q4_attention(q, 0, c, opts=opts)
        assert int(status) == 6 and not bool(out.any()) and bool((lse == -float("inf")).all())


def test_many_heads_and_few_rows_keep_their_probabilities(sqa):
    """Many query heads per KV head where the plan does not take the form that rounds probabilities: within the bound of two parts."""
    for D in (64, 128):
        for i, (B, T, before, Hq, Hkv) in enumerate(((1, 3, 0, 200, 1), (1, 1, 900, 128, 1), (2, 2, 333, 96, 2), (1, 40, 2000, 12, 2))):
            gen, cap = generator(90 + i), before + T + 2
            assert not sqa.q4_plan(cap, B, T, Hq, Hkv, D, "bf16", before)["rounded_probs"]
            c = attention_test.filled(sqa, B, Hkv, D, cap, 0, bool(i % 2), gen)
            q = (torch.randn(B, Hq, T, D, generator=gen, device=DEV) * 1.5).bfloat16()
            out, lse = sqa.q4_attention(q, before, c)
            attention_test.check(2.0 ** -15, c, q, out, lse, [before] * B, [T] * B, [cap] * B, 0, (B, T, before, Hq, Hkv))


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_how_much_a_chunk_sees_of_a_turned_ring(sqa, dtype, D):
    """Keys of zeros: ln(slots seen) is what a row's normaliser says.  A chunk's k-th token from its end sees k slots fewer than the ring and the sinks
    hold, a single token all of them."""
    dt, cap, sink = R.DT[dtype], 64, 4
    for T, before in ((1, 200), (10, 200), (60, 300), (7, 57), (7, 55)):
        for B, g, Hkv in ((1, 3, 1), (2, 8, 4)):
            c = sqa.Q4Caches([cap], B, Hkv, D, DEV, n_sink=sink)
            out, lse = sqa.q4_attention(torch.randn(B, g * Hkv, T, D, device=DEV).to(dt), before, c)
            turned = before + T > cap
            seen = torch.tensor([cap - (T - 1 - t) if turned else before + t + 1 for t in range(T)], dtype=torch.float64, device=DEV)
            want = seen.log().expand(lse.shape)
            # (chunk_reference.py's bound with logits of 0: sums of `cap` terms, the exponential's and the logarithm's roundings)
            assert bool(((lse.double() - want).abs() <= 4 * R.U + cap * R.U + 4 * R.U * (want + 1)).all()) and not bool(out.any()), (T, before)
