"""A layer's cache in 4 bits and what goes with it: the operators as a serving program calls them, and the same in elementary
torch operations.

A case is a dict of plain values.  Five kinds ("op"):
  rope       queries and keys as the projection leaves them, [B][T] rows of one packed tensor: each head normalised (root mean
             square) and rotated by its token's positions on several axes (time, height, width), laid out as [B][H][T][D]
  tables     block tables brought up to date on the GPU from the sequences' lengths (blocks of a free list taken and given
             back), and from them the row of the pools that each new token of each unit goes to
  append     a chunk's keys and values written into a cache of 4 bits, and read back as the values that it then stands for
  attention  causal attention of a chunk's queries (one token: a decode step) over a cache of 4 bits
  step       a projection's output to attention in two calls: queries and keys normalised and rotated, keys and values into
             the cache of 4 bits, attention over it

The 4 bits: 32 neighbouring elements of a row share a power of two 2^(byte - 127), the smallest with max |x| <= 7 * 2^e
(byte 2 .. 252); each is the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 times it, ties to the even code, larger ones 6; code =
sign * 8 + index, two of them in a byte, the element with the even number in its low half.

A unit (sequence, KV head) has `capacity` slots: the token of position p lies in slot p, and once p >= capacity the first
`sink` slots stay and the others are a ring, slot sink + (p - sink) % (capacity - sink).  `past` is the number of tokens that
the longest sequence of the batch had before the chunk, `chunk` the most tokens that one of them brings.  Shapes are those of
workloads.py (1 to 8 query heads per KV head, head size 64 or 128, prompts up to 8192, budgets of a few hundred tokens), with
contexts up to 32 k, chunks of one token to 2048, and sizes in between and odd ones.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 16             # slots of a block
GROUP = 32             # elements that share a power of two
EPS = 1e-6
BASE = 10000.0


# ---- the cases ------------------------------------------------------------------------------------------------
def _case(name, op, B, chunk, past, Hq, Hkv, D, dtype="bf16", capacity=0, sink=0, blocked=True, ragged=False, axes=3, turns=False,
          interleaved=False, norm=True):
    """capacity 0: room for every token."""
    return dict(name=name, op=op, batch=B, chunk=chunk, past=past, heads=Hq, kv_heads=Hkv, dim=D, dtype=dtype, capacity=capacity or past + chunk,
                sink=sink, blocked=blocked, ragged=ragged, axes=axes, turns=turns, interleaved=interleaved, norm=norm)


def listed():
    return [
        # one decode step of a model that has seen images: the smallest call
        _case("rope_axes_step", "rope", 8, 1, 2300, 32, 8, 128),
        # prompts with video frames, the three axes taking turns over the pairs
        _case("rope_axes_prompt", "rope", 2, 4500, 0, 32, 8, 128, turns=True, ragged=True),
        # a decode step of 64 sequences: some of them need a block more, some have left
        _case("tables_step", "tables", 64, 1, 4000, 32, 8, 128, ragged=True),
        # a chunk of 512 for each of 256 sequences, their tables taken from the free list
        _case("tables_chunk", "tables", 256, 512, 1500, 32, 8, 128, ragged=True),
        # five drafted tokens for each of 16 sequences
        _case("append_draft", "append", 16, 5, 4090, 64, 8, 128, ragged=True),
        # a batch of prompts, 512 tokens further
        _case("append_chunk", "append", 8, 512, 2048, 32, 8, 128),
        # a decode step of 16 sequences of 2000 to 4000 tokens
        _case("attention_step", "attention", 16, 1, 4090, 32, 8, 128, ragged=True),
        # a decode step against budgets of 571 slots with 4 sinks, rings long since turned, one query head per KV head
        _case("attention_ring", "attention", 64, 1, 1500, 32, 32, 128, capacity=571, sink=4, blocked=False),
        # one token far into a long context, 8 query heads per KV head
        _case("attention_long", "attention", 1, 1, 30000, 64, 8, 128, blocked=False),
        # the last quarter of a prompt of 8192 at once: the largest, bound by arithmetic
        _case("attention_chunk", "attention", 1, 2048, 6144, 64, 8, 128),
        # fp32, three query heads per KV head, a draft, odd lengths
        _case("attention_f32_odd", "attention", 3, 7, 1111, 12, 4, 64, dtype="f32", ragged=True),
        # a whole decode step of one layer
        _case("step", "step", 16, 1, 2300, 32, 8, 128),
    ]


def draw(rng):
    op = rng.choice(["rope", "tables", "append", "attention", "attention", "attention", "step"])
    spread = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    dtype = "bf16" if op == "step" else rng.choice(["bf16", "bf16", "bf16", "f32"])
    D = rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 3, 4, 6, 8, 16, 32])
    g = rng.choice([1, 2, 3, 4, 5, 8])
    chunk = rng.choice([1, 1, spread(1, 16), spread(1, 2048), spread(16, 2048)])
    past = rng.choice([spread(1, 30000), spread(16, 8192), 0])
    B = spread(1, 64)
    if op == "tables":
        B, chunk, past = spread(1, 400), min(chunk, 600), min(past, 8192)
        B = max(1, min(B, (1 << 22) // (Hkv * chunk), (1 << 23) // (Hkv * (past + chunk))))
    elif op == "step":
        chunk, past = rng.choice([1, 1, spread(1, 8)]), max(past, 300)
    # bytes of rope / append, logits of the others: no more than the largest listed cases have
    most = {"rope": 9000 * 32 * 128, "append": 4096 * 16 * 128}.get(op, 1 << 30 if dtype == "bf16" else 1 << 25)
    if op != "tables":
        each = lambda: chunk * Hkv * g * D if op in ("rope", "append") else chunk * Hkv * g * (past + chunk)
        B = max(1, min(B, most // each(), (1 << 30) // (2 * Hkv * D * (past + chunk))))
        while each() > most:
            chunk = chunk // 2 + 1
            past //= 2
    capacity, sink = 0, 0
    if op in ("append", "attention", "step") and rng.random() < 0.35:
        sink = rng.choice([0, 4])
        capacity = max(chunk + sink, spread(16, past + chunk + 16))
    c = _case("", op, B, chunk, past, g * Hkv, Hkv, D, dtype, capacity=capacity, sink=sink, blocked=op == "tables" or rng.random() < 0.5,
              ragged=rng.random() < 0.5, axes=rng.choice([2, 3, 3, 4]), turns=rng.random() < 0.4, interleaved=rng.random() < 0.3,
              norm=rng.random() < 0.6)
    if c["capacity"] > 16000:
        c["blocked"] = False
    del c["name"]
    return c


# ---- 4 bits ---------------------------------------------------------------------------------------------------
def _pack(x):
    """[.., D] in 32 bits -> codes [.., D / 2], powers [.., D / 32], both uint8."""
    g = x.unflatten(-1, (-1, GROUP))
    power = ((g.abs().amax(-1).view(torch.int32) + 0x1fffff >> 23) - 2).clamp(2, 252)
    y = g * (254 - power << 23).view(torch.float32)[..., None]          # (by 2^(127 - power): exact)
    a = y.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)
            + torch.signbit(y) * 8).to(torch.uint8).flatten(-2)
    return code[..., 0::2] | code[..., 1::2] << 4, power.to(torch.uint8)


def _unpack(code, power):
    """The values that they stand for, in 32 bits."""
    value = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=code.device)
    x = torch.stack([value[(code & 15).int()], value[(code >> 4).int()]], -1).flatten(-2)
    return (x.unflatten(-1, (-1, GROUP)) * (power.to(torch.int32) << 23).view(torch.float32)[..., None]).flatten(-2)


# ---- what a user's program has in hand ------------------------------------------------------------------------
def _lengths(case, seed):
    """(tokens before the chunk, tokens of the chunk) of every sequence; the first has the most of both."""
    B, T, past = case["batch"], case["chunk"], case["past"]
    if not case["ragged"]:
        return [past] * B, [T] * B
    g = torch.Generator().manual_seed(seed * 97 + B * 31 + T)
    before = torch.randint(past // 2, past + 1, (B - 1,), generator=g)
    new = torch.randint(max(1, T // 2), T + 1, (B - 1,), generator=g)
    return [past] + before.tolist(), [T] + new.tolist()


def _sections(case):
    """How many of the pairs go by each axis."""
    half, n = case["dim"] // 2, case["axes"]
    first = max(half // 4, 1) if n > 2 else half // n
    rest = [(half - first) // (n - 1)] * (n - 1)
    return [half - sum(rest)] + rest


def _axis_of(case):
    """The axis of each pair: one axis after the other, or in turns while an axis has pairs left."""
    left, order, at = _sections(case), [], 0
    if not case["turns"]:
        return [a for a, n in enumerate(left) for _ in range(n)]
    while len(order) < case["dim"] // 2:
        if left[at]:
            left[at] -= 1
            order.append(at)
        at = (at + 1) % len(left)
    return order


def _cache(case, s, rows, dev, gen, heavy):
    D = case["dim"]
    K = torch.randn(*rows, D, generator=gen, device=dev)
    K += (torch.rand(*rows, 1, generator=gen, device=dev) < 0.02) * heavy
    s["K"], s["K_scale"] = _pack(K)
    del K
    s["V"], s["V_scale"] = _pack(torch.randn(*rows, D, generator=gen, device=dev))


def _inputs(case, seed):
    """Every tensor of a case from its seed: projections, weights, table, and the cache as it lies in memory."""
    dev, dt = "cuda", DTYPES[case["dtype"]]
    B, T, Hq, Hkv, D, cap = (case[k] for k in ("batch", "chunk", "heads", "kv_heads", "dim", "capacity"))
    gen = torch.Generator(device=dev).manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device=dev)
    before, new = _lengths(case, seed)
    s = {"case": case, "before": torch.tensor(before, dtype=torch.int32, device=dev), "new": torch.tensor(new, dtype=torch.int32, device=dev)}
    per = -(-cap // BLOCK)
    if case["op"] == "tables":
        # every sequence holds blocks for what it had; of eight sequences one leaves, and one that comes new had none
        n_blocks = B * Hkv * per + 64
        ids = torch.randperm(n_blocks, generator=host).to(torch.int32)
        fate = torch.rand(B, generator=host)
        tokens = torch.tensor([b + n for b, n in zip(before, new)], dtype=torch.int32)
        had = (torch.tensor(before, dtype=torch.int32) + BLOCK - 1) // BLOCK
        had[(fate >= 0.125) & (fate < 0.25)] = 0
        tokens[fate < 0.125] = 0
        first = torch.tensor(before, dtype=torch.int32)
        first[fate < 0.125] = -1
        use = (had[:, None, None] > torch.arange(per)).expand(B, Hkv, per)
        table = torch.full((B, Hkv, per), -1, dtype=torch.int32)
        used = int(use.sum())
        table[use] = ids[:used]
        free = torch.full((n_blocks,), -1, dtype=torch.int32)
        free[:n_blocks - used] = ids[used:]
        # (one buffer: a pass starts from the same state each time)
        s["start"] = torch.cat([table.flatten(), had, free, torch.tensor([n_blocks - used], dtype=torch.int32)]).to(dev)
        s["now"] = s["start"].clone()
        s["table"], s["held"], s["free"], s["count"] = s["now"].split([B * Hkv * per, B, n_blocks, 1])
        s["table"] = s["table"].view(B * Hkv, per)
        s["tokens"], s["first"] = tokens.to(dev), first.to(dev)
        s["map"] = torch.zeros(B, Hkv, T, dtype=torch.int32, device=dev)
        return s
    heavy = normal(D)
    heavy *= 3.0 / heavy.norm()
    if case["op"] != "attention":
        s["qkv"] = (normal(B, T, (Hq + 2 * Hkv) * D) * 1.5).to(dt)
    if case["op"] in ("rope", "step"):
        s["wq"], s["wk"] = ((1 + 0.1 * normal(D)).to(dt) for _ in range(2)) if case["norm"] else (None, None)
        # a token's position on the first axis is its place in time, on the others a place in an image
        n_pos = case["past"] + T
        angle = torch.arange(n_pos, dtype=torch.float64)[:, None] * BASE ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
        s["rope"] = torch.cat([angle.cos(), angle.sin()], 1).to(torch.float32).to(dev)
        time = s["before"][:, None] + torch.arange(T, device=dev)
        place = [torch.randint(0, min(n_pos, 64), (B, T), generator=gen, device=dev) for _ in range(case["axes"] - 1)]
        s["pos"] = torch.stack([time.clamp(max=n_pos - 1)] + place).to(torch.int32)
    if case["op"] == "rope":
        s["q_out"] = torch.zeros(B, Hq, T, D, dtype=dt, device=dev)
        s["k_out"] = torch.zeros(B, Hkv, T, D, dtype=dt, device=dev)
        return s
    if case["op"] != "append":
        s["q"] = (normal(B, Hq, T, D) + heavy).to(dt)
        s["out"] = torch.zeros(B, T, Hq, D, dtype=dt, device=dev)
        s["lse"] = torch.zeros(B, Hq, T, dtype=torch.float32, device=dev)
    else:
        s["k_out"], s["v_out"] = (torch.zeros(B, Hkv, T, D, dtype=dt, device=dev) for _ in range(2))
    if case["blocked"]:
        n_blocks = B * Hkv * per + 3
        s["table"] = torch.randperm(n_blocks, generator=host)[:B * Hkv * per].to(torch.int32).view(B * Hkv, per).to(dev)
        _cache(case, s, (n_blocks, BLOCK), dev, gen, heavy)
    else:
        _cache(case, s, (B, Hkv, cap), dev, gen, heavy)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2404_04793_amd import binding as sqa
        B, Hkv, D, op = case["batch"], case["kv_heads"], case["dim"], case["op"]
        s["sqa"] = sqa
        s["opts"] = sqa.batch_opts(prompt_len=s["new"], new_pos_seq=s["before"]) if case["ragged"] else None
        if op in ("rope", "step"):
            s["prep"] = sqa.head_prep(s["wq"], s["wk"], EPS, s["rope"], case["interleaved"])
            s["axes"] = sqa.rope_axes(s["pos"], _sections(case), case["turns"])
        if op == "tables":
            s["opts"] = sqa.batch_opts(prompt_len=s["new"], new_pos_seq=s["first"])
        elif op != "rope":
            c = sqa.Q4Caches([case["capacity"]], B, Hkv, D, "cuda", n_sink=case["sink"], blocked=case["blocked"])
            for mine, theirs in (("K", c.K), ("V", c.V), ("K_scale", c.K_scale), ("V_scale", c.V_scale), ("table", c.block_table)):
                if mine in s:
                    theirs[0].copy_(s[mine])
                    s[mine] = theirs[0]
            s["caches"] = c
            if op != "append":
                s["workspace"] = sqa.q4_workspace(c, case["heads"], case["chunk"])
            else:
                # what is read back lies in the slots from the first new token's on (a ring that turns within the chunk: from slot 0 on)
                s["read"] = sqa.batch_opts(new_pos_seq=_read_from(s))
    return s


def _read_from(s):
    c = s["case"]
    first = s["before"]
    return torch.where(first + c["chunk"] > c["capacity"], c["capacity"] - c["chunk"], first).to(torch.int32)


# ---- one pass -------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if own:
        return _call(s, case["op"], s["sqa"], case["past"])
    return {"rope": _rope, "tables": _tables, "append": _append, "attention": _attention, "step": _step}[case["op"]](s)


def _projections(s):
    """Views of the packed projection: queries, keys, values, [B][T][H][D] each."""
    c = s["case"]
    Hq, Hkv, D = c["heads"], c["kv_heads"], c["dim"]
    x = s["qkv"].view(c["batch"], c["chunk"], Hq + 2 * Hkv, D)
    return x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]


def _call(s, op, sqa, past):
    case = s["case"]
    if op == "rope":
        q, k, _ = _projections(s)
        return sqa.qk_norm_rope(q, k, past, s["prep"], q_out=s["q_out"], k_out=s["k_out"], opts=s["opts"], axes=s["axes"])
    if op == "tables":
        s["now"].copy_(s["start"])
        sqa.block_assign(s["table"], s["tokens"], s["held"], s["free"], s["count"], case["capacity"])
        sqa.slot_map(s["table"], case["capacity"], case["chunk"], out=s["map"], opts=s["opts"])
        return [s[x] for x in ("table", "held", "free", "count", "map")]
    if op == "append":
        _, k, v = _projections(s)
        sqa.q4_append(k, v, past, s["caches"], opts=s["opts"])
        return sqa.q4_read(s["caches"], 0, case["chunk"], DTYPES[case["dtype"]], k_out=s["k_out"], v_out=s["v_out"], opts=s["read"])
    if op == "attention":
        return sqa.q4_attention(s["q"], past, s["caches"], out=s["out"], lse=s["lse"], workspace=s["workspace"], opts=s["opts"])
    q, k, v = _projections(s)
    sqa.q4_append(k, v, past, s["caches"], prep=s["prep"], q=q, q_out=s["q"], opts=s["opts"], axes=s["axes"])
    return sqa.q4_attention(s["q"], past, s["caches"], out=s["out"], workspace=s["workspace"], opts=s["opts"])[0]


def _valid(s):
    """[B][T]: which rows of the chunk are tokens."""
    return torch.arange(s["case"]["chunk"], device="cuda") < s["new"][:, None]


def _slot(s, p):
    """Slots of positions p."""
    c = s["case"]
    return torch.where(p < c["capacity"], p, c["sink"] + (p - c["sink"]) % (c["capacity"] - c["sink"]))


def _rows(s, slot):
    """Row of the cache (as one list of rows) for slots [B][1 or Hkv][n] of each unit."""
    c = s["case"]
    unit = torch.arange(c["batch"] * c["kv_heads"], device="cuda").view(c["batch"], c["kv_heads"], 1)
    if c["blocked"]:
        return s["table"][unit, slot // BLOCK].long() * BLOCK + slot % BLOCK
    return unit * c["capacity"] + slot


def _prepared(s, x, weight):
    """[B][T][H][D] -> [B][H][T][D] in 32 bits, normalised and rotated."""
    c = s["case"]
    x = x.float().transpose(1, 2)
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    half = c["dim"] // 2
    at = s["pos"][torch.tensor(_axis_of(c), device="cuda")].permute(1, 2, 0).long()        # [B][T][pairs]
    pair = torch.arange(half, device="cuda")
    cos, sin = s["rope"][at, pair][:, None], s["rope"][at, half + pair][:, None]
    if c["interleaved"]:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _put(out, value, valid):
    out.copy_(torch.where(valid[:, None, :, None], value.to(out.dtype), out))


def _rope(s):
    q, k, _ = _projections(s)
    _put(s["q_out"], _prepared(s, q, s["wq"]), _valid(s))
    _put(s["k_out"], _prepared(s, k, s["wk"]), _valid(s))
    return s["q_out"], s["k_out"]


def _tables(s):
    c = s["case"]
    Hkv, per = c["kv_heads"], s["table"].shape[1]
    s["now"].copy_(s["start"])
    need = (s["tokens"].clamp(max=c["capacity"]) + BLOCK - 1) // BLOCK
    entry = torch.arange(per, device="cuda")
    table = s["table"].view(-1, Hkv, per)
    # sequences that hold more than they need give blocks back, in order
    gives = ((entry >= need[:, None]) & (entry < s["held"][:, None]))[:, None].expand_as(table)
    back = table[gives]
    s["free"][s["count"] + torch.arange(len(back), device="cuda")] = back
    s["count"] += len(back)
    table[gives] = -1
    s["held"].copy_(torch.minimum(s["held"], need))
    # the others take theirs from the end of the list, in order, as far as it goes
    wants = (need - s["held"]) * Hkv
    fits = wants.cumsum(0) <= s["count"]
    takes = ((entry >= s["held"][:, None]) & (entry < need[:, None]) & fits[:, None])[:, None].expand_as(table)
    n = int(takes.sum())
    table[takes] = s["free"][s["count"] - 1 - torch.arange(n, device="cuda")]
    s["count"] -= n
    s["held"].copy_(torch.where(fits, need, s["held"]))
    # rows of the new tokens
    slot = _slot(s, s["first"][:, None] + torch.arange(c["chunk"], device="cuda"))[:, None].expand(-1, Hkv, -1)
    there = (_valid(s) & (s["first"] >= 0)[:, None])[:, None]
    block = table.gather(2, torch.where(there, slot // BLOCK, 0).long())
    s["map"].copy_(torch.where(there & (block >= 0), block * BLOCK + slot % BLOCK, -1))
    return [s[x] for x in ("table", "held", "free", "count", "map")]


def _store(s, name, x):
    """A chunk's rows [B][Hkv][T][D] in 32 bits into the cache."""
    c = s["case"]
    code, power = _pack(x)
    # rows behind a sequence's last token: that token once more, in its own slot
    t = torch.minimum(torch.arange(c["chunk"], device="cuda"), s["new"][:, None].long() - 1)
    slot = _slot(s, s["before"][:, None] + t)[:, None].expand(-1, c["kv_heads"], -1)
    rows = _rows(s, slot)
    pick = t[:, None, :, None].expand(-1, c["kv_heads"], -1, -1)
    s[name].view(-1, code.shape[-1])[rows] = code.gather(2, pick.expand(-1, -1, -1, code.shape[-1]))
    s[name + "_scale"].view(-1, power.shape[-1])[rows] = power.gather(2, pick.expand(-1, -1, -1, power.shape[-1]))


def _values(s, name, slot):
    """What the cache holds in slots [B][1][n], [B][Hkv][n][D] in 32 bits."""
    c = s["case"]
    rows = _rows(s, slot)
    return _unpack(s[name].view(-1, c["dim"] // 2)[rows], s[name + "_scale"].view(-1, c["dim"] // GROUP)[rows])


def _append(s):
    c = s["case"]
    _, k, v = _projections(s)
    _store(s, "K", k.float().transpose(1, 2))
    _store(s, "V", v.float().transpose(1, 2))
    slot = (_read_from(s)[:, None] + torch.arange(c["chunk"], device="cuda"))[:, None]
    s["k_out"].copy_(_values(s, "K", slot))
    s["v_out"].copy_(_values(s, "V", slot))
    return s["k_out"], s["v_out"]


def _attend(s, q):
    """[B][Hq][T][D] -> (out [B][T][Hq][D], lse) in 32 bits, of the chunk's tokens."""
    c = s["case"]
    B, Hkv, T, D, cap, sink = (c[k] for k in ("batch", "kv_heads", "chunk", "dim", "capacity", "sink"))
    end = (s["before"] + s["new"]).long()[:, None]                       # positions 0 .. end - 1 have been appended
    n = min(cap, c["past"] + T)
    slot = torch.arange(n, device="cuda")[None]
    turned = end - 1 - (end - 1 - slot) % (cap - sink)                   # the newest position that goes to a slot of the ring
    held = torch.where((end <= cap) | (slot < sink), slot, turned)
    held = torch.where(slot < end, held, c["past"] + T)                  # (nothing lies there yet)
    seen = held[:, None] <= (s["before"][:, None] + torch.arange(T, device="cuda"))[..., None]      # [B][T][n]
    seen &= (slot < end)[:, None]
    at = torch.minimum(slot, end - 1)[:, None]
    logits = q.float().reshape(B, Hkv, -1, D) @ _values(s, "K", at).transpose(2, 3) / math.sqrt(D)
    logits.masked_fill_(~seen[:, None].repeat(1, 1, c["heads"] // Hkv, 1), -math.inf)
    top = logits.amax(-1, keepdim=True).clamp(min=-1e30)
    p = logits.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = ((p @ _values(s, "V", at)) / total).view(B, c["heads"], T, D).transpose(1, 2)
    return out, (top + total.log()).view(B, c["heads"], T)


def _attention(s):
    out, lse = _attend(s, s["q"])
    valid = _valid(s)
    s["out"].copy_(torch.where(valid[:, :, None, None], out.to(s["out"].dtype), s["out"]))
    s["lse"].copy_(torch.where(valid[:, None], lse, s["lse"]))
    return s["out"], s["lse"]


def _step(s):
    q, k, v = _projections(s)
    _put(s["q"], _prepared(s, q, s["wq"]), _valid(s))
    _store(s, "K", _prepared(s, k, s["wk"]))
    _store(s, "V", v.float().transpose(1, 2))
    out, _ = _attend(s, s["q"])
    s["out"].copy_(torch.where(_valid(s)[:, :, None, None], out.to(s["out"].dtype), s["out"]))
    return s["out"]


# ---- what a pass cannot do without ------------------------------------------------------------------------------
def work(case):
    B, T, past, Hq, Hkv, D, cap = (case[k] for k in ("batch", "chunk", "past", "heads", "kv_heads", "dim", "capacity"))
    e, op = 2 if case["dtype"] == "bf16" else 4, case["op"]
    share = 0.75 if case["ragged"] else 1.0          # (sequences between half and all of the longest)
    tokens, held = B * T * share, B * min((past + T) * share, cap)
    row = D / 2 + D / GROUP                          # a row of the cache in bytes
    pairs = tokens * (min(past * share, cap) + (T * share + 1) / 2 if past + T <= cap else cap)
    if op == "rope":
        return {"bytes": 2 * tokens * (Hq + Hkv) * D * e + tokens * case["axes"] * 4 + T * D * 4, "flops": 6 * tokens * (Hq + Hkv) * D}
    if op == "tables":
        # the map, the tables' entries behind it, and what changes hands (a quarter of all blocks at most)
        moved = B * Hkv * ((past + T) * share / BLOCK * 0.25 + T * share / BLOCK)
        return {"bytes": 4 * (B * Hkv * T + B * Hkv * (1 + T * share / BLOCK) + 3 * moved + 4 * B), "flops": B * Hkv * T}
    if op == "append":
        return {"bytes": 2 * tokens * Hkv * (D * e + row) + 2 * B * T * Hkv * (row + D * e), "flops": 8 * tokens * Hkv * D}
    step = 2 * tokens * (Hq + Hkv) * D * e if op == "step" else 0
    return {"bytes": 2 * held * Hkv * row + tokens * Hq * (2 * D * e + 4) + step, "flops": 4 * pairs * Hq * D}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------
def exact(case, seed):
    """From the formulas, one sequence after the other, apart from the plain form above."""
    if case["op"] == "tables":
        return None
    s = _inputs(case, seed)
    B, T, Hq, Hkv, D, cap, sink = (case[k] for k in ("batch", "chunk", "heads", "kv_heads", "dim", "capacity", "sink"))
    g = Hq // Hkv
    before, new = _lengths(case, seed)
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")

    def rounded(x):
        """[.., D] in 64 bits -> the values that 4 bits stand for."""
        x = x.unflatten(-1, (-1, GROUP))
        m, e = torch.frexp(x.abs().amax(-1, keepdim=True) / 7)          # (the smallest power of two with max |x| <= 7 of it)
        unit = torch.where(m == 0, 0.0, torch.pow(2.0, torch.where(m == 0.5, e - 1, e).double())).clamp(2.0 ** -125, 2.0 ** 125)
        away = ((x / unit).abs()[..., None] - grid).abs()
        best = away.amin(-1, keepdim=True)
        near = (away == best).to(torch.int8)
        even = near * torch.tensor([2, 1, 2, 1, 2, 1, 2, 1], dtype=torch.int8, device="cuda")
        return (torch.sign(x) * grid[even.argmax(-1)] * unit).flatten(-2)

    def turned(x, weight, b, n):
        """[n][H][D], tokens 0 .. n - 1 of sequence b."""
        x = x.double()
        if weight is not None:
            x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / D + EPS) * weight.double()
        y = x.clone()
        for i, axis in enumerate(_axis_of(case)):
            angle = s["rope"][s["pos"][axis, b, :n].long()].double()
            at = (2 * i, 2 * i + 1) if case["interleaved"] else (i, D // 2 + i)
            z = torch.complex(x[..., at[0]], x[..., at[1]]) * torch.complex(angle[:, i], angle[:, D // 2 + i])[:, None]
            y[..., at[0]], y[..., at[1]] = z.real, z.imag
        return y

    def held(name, b, h):
        """Unit (b, h)'s slots as the cache stands, [cap][D]."""
        u = b * Hkv + h
        if case["blocked"]:
            pick = lambda x: x[s["table"][u].long()].flatten(0, 1)[:cap]
        else:
            pick = lambda x: x[b, h]
        code, power = pick(s[name]), pick(s[name + "_scale"])
        digits = torch.stack([code % 16, code // 16], -1).flatten(-2).long()
        value = grid[digits % 8] * torch.where(digits < 8, 1.0, -1.0)
        return value * torch.pow(2.0, power.double() - 127).repeat_interleave(GROUP, -1)

    place = lambda p: p if p < cap else sink + (p - sink) % (cap - sink)
    wide = {k: s[k].double() for k in ("q_out", "k_out", "v_out", "q", "out", "lse") if k in s}
    if case["op"] != "attention":
        x = s["qkv"].double().view(B, T, Hq + 2 * Hkv, D)
    if case["op"] == "rope":
        for b in range(B):
            n = new[b]
            wide["q_out"][b, :, :n] = turned(x[b, :n, :Hq], s["wq"], b, n).transpose(0, 1)
            wide["k_out"][b, :, :n] = turned(x[b, :n, Hq:Hq + Hkv], s["wk"], b, n).transpose(0, 1)
        return wide["q_out"], wide["k_out"]
    for b in range(B):
        n, end = new[b], before[b] + new[b]
        slots = torch.tensor([place(p) for p in range(before[b], end)], device="cuda")
        at = [-1] * cap                              # the position in each slot
        for p in range(max(0, end - cap) if end > cap else 0, end):
            at[place(p)] = p
        for p in range(min(sink, end)):
            at[p] = p
        at = torch.tensor(at, device="cuda")
        sees = (at >= 0) & (at <= before[b] + torch.arange(n, device="cuda")[:, None])
        if case["op"] != "attention":
            keys, values = x[b, :n, Hq:Hq + Hkv], x[b, :n, Hq + Hkv:]
            if case["op"] == "step":
                wide["q"][b, :, :n] = turned(x[b, :n, :Hq], s["wq"], b, n).transpose(0, 1).to(DTYPES[case["dtype"]]).double()
                keys = turned(keys, s["wk"], b, n)
        for h in range(Hkv):
            K, V = held("K", b, h), held("V", b, h)
            if case["op"] != "attention":
                K[slots], V[slots] = rounded(keys[:, h]), rounded(values[:, h])
            if case["op"] == "append":
                first = int(_read_from(s)[b])
                wide["k_out"][b, h], wide["v_out"][b, h] = K[first:first + T], V[first:first + T]
                continue
            for i in range(h * g, (h + 1) * g):
                logits = torch.where(sees, (wide["q"][b, i, :n] @ K.T) * D ** -0.5, -math.inf)
                wide["lse"][b, i, :n] = torch.logsumexp(logits, -1)
                wide["out"][b, :n, i] = torch.softmax(logits, -1) @ V
    return (wide["k_out"], wide["v_out"]) if case["op"] == "append" else wide["out"] if case["op"] == "step" else (wide["out"], wide["lse"])
