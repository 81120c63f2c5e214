"""A prompt, a chunk of one, or a few drafted tokens at a time: the operators between a model's projections and the
layer caches, as a serving program calls them, and the same in elementary torch operations.

A case is a dict of plain values.  Four kinds ("op"):
  rope       queries and keys as the projection leaves them, [B][T] rows of one packed tensor: each head normalised
             (root mean square) and rotated by its position, laid out head by head as [B][H][T][D]
  append     a chunk's keys (normalised and rotated) and values written into a layer's cache behind its tokens, and
             the chunk's queries prepared in the same call
  attention  causal attention of a chunk's queries over all that the cache holds up to each of them, with the
             logarithms of the softmax normalisers
  scores     the attention that a chunk gives to every slot of the cache, added to the accumulated scores

Shapes are those of workloads.py (1 to 8 query heads per KV head, head size 64 or 128, prompts up to 8192), with
contexts up to 32 k, chunks of one token to 2048, and sizes in between and odd ones.  `past` is the number of tokens the
longest sequence of the batch has in its cache before the chunk, `chunk` the most tokens one of them brings.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 16             # slots of a block, layout "blocked"
EPS = 1e-6
BASE = 10000.0


# ---- the cases ------------------------------------------------------------------------------------------------
def _case(name, op, B, chunk, past, Hq, Hkv, D, dtype, layout="dense", rot=None, interleaved=False, norm=True, ragged=False):
    return dict(name=name, op=op, batch=B, chunk=chunk, past=past, heads=Hq, kv_heads=Hkv, dim=D, dtype=dtype, layout=layout,
                rot=D if rot is None else rot, interleaved=interleaved, norm=norm, ragged=ragged)


def listed():
    return [
        # one decode step of the Llama-2-7B shape at batch 8: the smallest call, before sqa_decode_step
        _case("rope_step_b8", "rope", 8, 1, 2300, 32, 32, 128, "bf16", norm=False),
        # whole prompts of 2048 at once, grouped queries, before the prompt's scores
        _case("rope_prompt", "rope", 4, 2048, 0, 32, 8, 128, "bf16"),
        # five drafted tokens for each of 16 sequences in blocks: the smallest append
        _case("append_draft", "append", 16, 5, 4090, 64, 8, 128, "bf16", layout="blocked", ragged=True),
        # a batch of prompts, 512 tokens further
        _case("append_chunk", "append", 8, 512, 2048, 32, 8, 128, "bf16", layout="blocked"),
        # fp32, packed units, half of each head rotated in neighbouring pairs, sequences of different lengths
        _case("append_f32_packed", "append", 3, 333, 700, 12, 6, 64, "f32", layout="packed", rot=32, interleaved=True, ragged=True),
        # five drafted tokens against caches of about 4000: bound by reading the cache
        _case("attention_draft", "attention", 16, 5, 4090, 32, 8, 128, "bf16", layout="blocked", ragged=True),
        # prompts of 2048 from an empty cache, the Llama-2-7B shape
        _case("attention_prompt", "attention", 8, 2048, 0, 32, 32, 128, "bf16"),
        # the last chunk of a prompt of 8192, 8 query heads per KV head
        _case("attention_chunk", "attention", 1, 512, 7680, 64, 8, 128, "bf16", layout="blocked"),
        # a chunk far into a long context, one sequence: the largest
        _case("attention_long", "attention", 1, 2048, 30000, 32, 8, 128, "bf16"),
        # fp32, three query heads per KV head, odd lengths, packed units
        _case("attention_f32_odd", "attention", 3, 77, 1111, 12, 4, 64, "f32", layout="packed", ragged=True),
        # scores of the last chunk of a prompt of 8192
        _case("scores_chunk", "scores", 1, 512, 7680, 64, 8, 128, "bf16", layout="blocked"),
        # scores of an odd chunk in sequences of different lengths
        _case("scores_ragged", "scores", 4, 333, 1700, 32, 32, 128, "bf16", ragged=True),
    ]


def draw(rng):
    op = rng.choice(["rope", "append", "attention", "attention", "scores"])
    spread = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    D = rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 3, 4, 6, 8, 16, 32])
    g = rng.choice([1, 2, 3, 4, 5, 8])
    chunk = rng.choice([1, spread(1, 2048), spread(1, 2048), spread(16, 2048)])
    past = rng.choice([0, spread(1, 30000), spread(16, 8192)])
    B = spread(1, 32)
    # bytes of rope / append, logits of the others: no more than the largest listed cases have
    most = 4096 * 32 * 128 if op in ("rope", "append") else (1 << 30 if dtype == "bf16" else 1 << 26)
    each = chunk * Hkv * g * D if op in ("rope", "append") else chunk * Hkv * g * (past + chunk)
    B = max(1, min(B, most // each, (1 << 30) // (Hkv * D * (past + chunk))))
    while each > most:
        chunk = chunk // 2 + 1
        past //= 2
        each = chunk * Hkv * g * D if op in ("rope", "append") else chunk * Hkv * g * (past + chunk)
    layout = rng.choice(["dense", "blocked", "packed"])
    if layout == "blocked" and past + chunk > 16000:
        layout = "dense"
    c = _case("", op, B, chunk, past, g * Hkv, Hkv, D, dtype, layout=layout, rot=rng.choice([D, D, D // 2, 16]),
              interleaved=rng.random() < 0.3, norm=rng.random() < 0.6, ragged=rng.random() < 0.4)
    del c["name"]
    return c


# ---- what a user's program has in hand ------------------------------------------------------------------------
def _lengths(case, seed):
    """(tokens in the cache before the chunk, tokens of the chunk) of every sequence; the first has the most of both."""
    B, T, past = case["batch"], case["chunk"], case["past"]
    if not case["ragged"]:
        return [past] * B, [T] * B
    # (the same lengths in another order with another seed: packed units then fill the same memory)
    g = torch.Generator().manual_seed(B * 31 + T)
    before = torch.randint(past // 2, past + 1, (B - 1,), generator=g)
    new = torch.randint(max(1, T // 2), T + 1, (B - 1,), generator=g)
    order = torch.randperm(B - 1, generator=torch.Generator().manual_seed(seed))
    before, new = [past] + before[order].tolist(), [T] + new[order].tolist()
    return before, new


def _inputs(case, seed):
    """Every tensor of a case from its seed: projections, weights, table, and the cache as it lies in memory."""
    dev, dt = "cuda", DTYPES[case["dtype"]]
    B, T, Hq, Hkv, D, rot = (case[k] for k in ("batch", "chunk", "heads", "kv_heads", "dim", "rot"))
    gen = torch.Generator(device=dev).manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device=dev)
    before, new = _lengths(case, seed)
    s = {"case": case, "before": torch.tensor(before, dtype=torch.int32, device=dev), "new": torch.tensor(new, dtype=torch.int32, device=dev)}
    heavy = normal(D)
    heavy *= 3.0 / heavy.norm()
    if case["op"] in ("rope", "append"):
        s["qkv"] = (normal(B, T, (Hq + 2 * Hkv) * D) * 1.5).to(dt)
        s["wq"], s["wk"] = ((1 + 0.1 * normal(D)).to(dt) for _ in range(2)) if case["norm"] else (None, None)
        # one row of cosines and sines per position, as a program makes it once for its longest context
        inv = BASE ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
        angle = torch.arange(case["past"] + T, dtype=torch.float64)[:, None] * inv
        s["rope"] = torch.cat([angle.cos(), angle.sin()], 1).to(torch.float32).to(dev)
        s["q_out"] = torch.zeros(B, Hq, T, D, dtype=dt, device=dev)
        s["k_out"] = torch.zeros(B, Hkv, T, D, dtype=dt, device=dev)
    else:
        s["q"] = (normal(B, Hq, T, D) + heavy).to(dt)
        s["out"] = torch.zeros(B, T, Hq, D, dtype=dt, device=dev)
        s["lse"] = torch.zeros(B, Hq, T, dtype=torch.float32, device=dev)
    if case["op"] == "rope":
        return s
    # the cache: slots of a unit hold its tokens in order; the chunk is still to come (append) or already there
    full = [b + n for b, n in zip(before, new)]
    cap = case["past"] + T
    held = before if case["op"] == "append" else full
    if case["layout"] == "blocked":
        per = -(-cap // BLOCK)
        n_blocks = B * Hkv * per + 3
        s["table"] = torch.randperm(n_blocks, generator=torch.Generator().manual_seed(seed))[:B * Hkv * per].to(torch.int32).view(B * Hkv, per).to(dev)
        rows, flat = (n_blocks, BLOCK, D), (B, Hkv, cap)
    elif case["layout"] == "packed":
        s["unit_capacities"] = [full[u // Hkv] for u in range(B * Hkv)]
        s["offsets"] = torch.tensor([0] + s["unit_capacities"], dtype=torch.int64).cumsum(0).to(dev)
        rows, flat = (sum(s["unit_capacities"]), D), (sum(s["unit_capacities"]),)
    else:
        rows, flat = (B, Hkv, cap, D), (B, Hkv, cap)
    K = normal(*rows)
    K += (torch.rand(*rows[:-1], 1, generator=gen, device=dev) < 0.02) * heavy
    s["K"], s["V"] = K.to(dt), normal(*rows).to(dt)
    units = torch.arange(B * Hkv, device=dev).view(B, Hkv)
    held = torch.tensor(held, dtype=torch.int32, device=dev)
    if case["layout"] == "packed":
        unit = torch.repeat_interleave(units.flatten(), s["offsets"].diff())
        slot, of = torch.arange(flat[0], device=dev) - s["offsets"][unit], held[unit // Hkv]
    else:
        slot, of = torch.arange(cap, device=dev).expand(flat), held[:, None, None]
    there = slot < of
    s["pos"] = torch.where(there, slot, -1).to(torch.int32)
    s["score"] = torch.rand(*flat, generator=gen, device=dev) * 4 * there
    s["state"] = torch.zeros(B, Hkv, 4, dtype=torch.int32, device=dev)
    s["state"][..., 0] = held[:, None]
    s["state"][..., 2] = -2
    if case["op"] == "scores":
        s["score0"] = s["score"].clone()
        logits, seen = _logits(s, torch.float64)
        lse = torch.logsumexp(logits.masked_fill_(~seen, -math.inf), -1).view(B, Hq, T)
        s["lse"] = torch.where(_valid(s)[:, None], lse, 0.0).to(torch.float32)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2404_04793_amd import binding as sqa
        B, Hkv, D, cap = case["batch"], case["kv_heads"], case["dim"], case["past"] + case["chunk"]
        s["sqa"] = sqa
        s["opts"] = sqa.batch_opts(prompt_len=s["new"], new_pos_seq=s["before"]) if case["ragged"] else None
        if case["op"] in ("rope", "append"):
            s["prep"] = sqa.head_prep(s["wq"], s["wk"], EPS, s["rope"], case["interleaved"])
        if case["op"] != "rope":
            c = sqa.LayerCaches([cap], [cap], B, Hkv, D, DTYPES[case["dtype"]], "cuda", True, blocked=case["layout"] == "blocked",
                                unit_capacities=[s["unit_capacities"]] if case["layout"] == "packed" else None)
            for mine, theirs in (("K", c.K), ("V", c.V), ("pos", c.pos), ("score", c.score), ("state", c.state), ("table", c.block_table)):
                if mine in s:
                    theirs[0].copy_(s[mine])
                    s[mine] = theirs[0]
            s["caches"] = c
            s["workspace"] = sqa.chunk_workspace(c, case["heads"], case["chunk"])
    return s


# ---- one pass -------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if own:
        return _call(s, case["op"], s["sqa"], case["past"])
    return {"rope": _rope, "append": _append, "attention": _attention, "scores": _scores}[case["op"]](s)


def _projections(s):
    """Views of the packed projection: queries, keys, values, [B][T][H][D] each."""
    c = s["case"]
    Hq, Hkv, D = c["heads"], c["kv_heads"], c["dim"]
    x = s["qkv"].view(c["batch"], c["chunk"], Hq + 2 * Hkv, D)
    return x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]


def _call(s, op, sqa, past):
    if op == "rope":
        q, k, _ = _projections(s)
        return sqa.qk_norm_rope(q, k, past, s["prep"], q_out=s["q_out"], k_out=s["k_out"], opts=s["opts"])
    if op == "append":
        q, k, v = _projections(s)
        sqa.chunk_append(k, v, past, s["caches"], prep=s["prep"], q=q, q_out=s["q_out"], opts=s["opts"])
        return [s[x] for x in ("q_out", "K", "V", "pos", "score", "state")]
    if op == "attention":
        return sqa.chunk_attention(s["q"], past, s["caches"], out=s["out"], lse=s["lse"], workspace=s["workspace"], opts=s["opts"])
    s["score"].copy_(s["score0"])        # (the call adds to the scores: the pass starts from the same ones each time)
    sqa.chunk_scores(s["q"], s["lse"], past, s["caches"], workspace=s["workspace"], opts=s["opts"])
    return s["score"]


def _valid(s):
    """[B][T]: which rows of the chunk are tokens."""
    return torch.arange(s["case"]["chunk"], device="cuda") < s["new"][:, None]


def _positions(s):
    return s["before"][:, None] + torch.arange(s["case"]["chunk"], device="cuda")


def _rows(s, slot):
    """Row of K and V (as one list of rows) for slots [B][1 or Hkv][n] of each unit."""
    c = s["case"]
    unit = torch.arange(c["batch"] * c["kv_heads"], device="cuda").view(c["batch"], c["kv_heads"], 1)
    if c["layout"] == "blocked":
        return s["table"][unit, slot // BLOCK].long() * BLOCK + slot % BLOCK
    if c["layout"] == "packed":
        return s["offsets"][unit] + slot
    return unit * (c["past"] + c["chunk"]) + slot


def _prepared(s, x, weight):
    """[B][T][H][D] -> [B][H][T][D] in 32 bits, normalised and rotated."""
    c = s["case"]
    x = x.float().transpose(1, 2)
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    half = c["rot"] // 2
    angle = s["rope"][torch.clamp(_positions(s), max=s["rope"].shape[0] - 1)][:, None]
    cos, sin, turned = angle[..., :half], angle[..., half:], x[..., :c["rot"]]
    if c["interleaved"]:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = turned[..., :half], turned[..., half:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., c["rot"]:]], -1)


def _put(out, value, valid):
    out.copy_(torch.where(valid[:, None, :, None], value.to(out.dtype), out))


def _rope(s):
    q, k, _ = _projections(s)
    _put(s["q_out"], _prepared(s, q, s["wq"]), _valid(s))
    _put(s["k_out"], _prepared(s, k, s["wk"]), _valid(s))
    return s["q_out"], s["k_out"]


def _append(s):
    c = s["case"]
    q, k, v = _projections(s)
    _put(s["q_out"], _prepared(s, q, s["wq"]), _valid(s))
    # rows behind a sequence's last token: that token once more, in its own slot
    t = torch.minimum(torch.arange(c["chunk"], device="cuda"), s["new"][:, None].long() - 1)
    pick = t[:, None, :, None].expand(-1, c["kv_heads"], -1, c["dim"])
    slot = (s["before"][:, None] + t)[:, None].expand(-1, c["kv_heads"], -1)
    rows = _rows(s, slot)
    s["K"].view(-1, c["dim"])[rows] = _prepared(s, k, s["wk"]).to(s["K"].dtype).gather(2, pick)
    s["V"].view(-1, c["dim"])[rows] = v.transpose(1, 2).gather(2, pick)
    if c["layout"] != "packed":
        unit = torch.arange(c["batch"] * c["kv_heads"], device="cuda").view(c["batch"], c["kv_heads"], 1)
        rows = unit * (c["past"] + c["chunk"]) + slot
    s["pos"].view(-1)[rows] = slot.to(torch.int32)
    s["score"].view(-1)[rows] = 0.0
    s["state"][..., 0] = (s["before"] + s["new"])[:, None]
    s["state"][..., 1], s["state"][..., 2], s["state"][..., 3] = 0, -2, 0
    return [s[x] for x in ("q_out", "K", "V", "pos", "score", "state")]


def _held(s, x):
    """Rows of K or V of every unit by slot, [B][Hkv][slots][D]; slots behind a sequence's last token hold that one again."""
    c = s["case"]
    slot = torch.minimum(torch.arange(c["past"] + c["chunk"], device="cuda"), (s["before"] + s["new"])[:, None].long() - 1)
    return s[x].view(-1, c["dim"])[_rows(s, slot[:, None])]


def _logits(s, dtype):
    """q.k / sqrt(D) of a unit's query rows (head by head) and slots, [B][Hkv][g T][slots], and which of them count."""
    c = s["case"]
    q = s["q"].to(dtype).view(c["batch"], c["kv_heads"], -1, c["dim"])
    logits = q @ _held(s, "K").to(dtype).transpose(2, 3) / math.sqrt(c["dim"])
    seen = torch.arange(c["past"] + c["chunk"], device="cuda") <= _positions(s)[..., None]
    return logits, seen[:, None].repeat(1, 1, c["heads"] // c["kv_heads"], 1)


def _attention(s):
    c = s["case"]
    logits, seen = _logits(s, torch.float32)
    logits.masked_fill_(~seen, -math.inf)
    top = logits.amax(-1, keepdim=True)
    p = logits.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = ((p @ _held(s, "V").float()) / total).view(c["batch"], c["heads"], c["chunk"], c["dim"])
    valid = _valid(s)
    s["out"].copy_(torch.where(valid[:, :, None, None], out.transpose(1, 2).to(s["out"].dtype), s["out"]))
    lse = (top + total.log()).view(c["batch"], c["heads"], c["chunk"])
    s["lse"].copy_(torch.where(valid[:, None], lse, s["lse"]))
    return s["out"], s["lse"]


def _scores(s):
    c = s["case"]
    s["score"].copy_(s["score0"])
    logits, seen = _logits(s, torch.float32)
    seen &= _valid(s)[:, None].repeat(1, 1, c["heads"] // c["kv_heads"])[..., None]
    p = logits.sub_(s["lse"].view(c["batch"], c["kv_heads"], -1, 1)).exp_().masked_fill_(~seen, 0.0)
    added = p.sum(2)
    if c["layout"] == "packed":
        slot = torch.arange(added.shape[-1], device="cuda")
        there = (slot < (s["before"] + s["new"])[:, None])[:, None].expand_as(added)
        s["score"].add_(added[there])
    else:
        s["score"].add_(added)
    return s["score"]


# ---- what a pass cannot do without ------------------------------------------------------------------------------
def work(case):
    B, T, past, Hq, Hkv, D = (case[k] for k in ("batch", "chunk", "past", "heads", "kv_heads", "dim"))
    e = 2 if case["dtype"] == "bf16" else 4
    share = 0.75 if case["ragged"] else 1.0          # (sequences between half and all of the longest)
    tokens, held = B * T * share, B * (past + T) * share
    pairs = tokens * (past * share + (T * share + 1) / 2)
    if case["op"] == "rope":
        return {"bytes": 2 * tokens * (Hq + Hkv) * D * e + T * case["rot"] * 4, "flops": 6 * tokens * (Hq + Hkv) * D}
    if case["op"] == "append":
        return {"bytes": tokens * (2 * (Hq + 2 * Hkv) * D * e + 8 * Hkv) + T * case["rot"] * 4, "flops": 6 * tokens * (Hq + Hkv) * D}
    if case["op"] == "attention":
        return {"bytes": 2 * held * Hkv * D * e + tokens * Hq * (2 * D * e + 4), "flops": 4 * pairs * Hq * D}
    return {"bytes": held * Hkv * (D * e + 8) + tokens * Hq * (D * e + 4), "flops": 2 * pairs * Hq * D}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------
def exact(case, seed):
    """From the formulas, one sequence after the other, apart from the plain form above."""
    s = _inputs(case, seed)
    B, T, Hq, Hkv, D, R = (case[k] for k in ("batch", "chunk", "heads", "kv_heads", "dim", "rot"))
    g, cap = Hq // Hkv, case["past"] + T
    before, new = _lengths(case, seed)
    wide = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}

    def turned(x, weight, first):
        """[n][H][D] at positions first, first + 1, ..."""
        if weight is not None:
            x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / D + EPS) * weight.double()
        angle = torch.complex(wide["rope"][first:first + len(x), :R // 2], wide["rope"][first:first + len(x), R // 2:])[:, None]
        y = x.clone()
        at = (slice(0, R, 2), slice(1, R, 2)) if case["interleaved"] else (slice(0, R // 2), slice(R // 2, R))
        z = torch.complex(x[..., at[0]], x[..., at[1]]) * angle
        y[..., at[0]], y[..., at[1]] = z.real, z.imag
        return y

    def place(b, h):
        """Rows of unit (b, h)'s slots in K and V as lists of rows, and the unit's part of the arrays by slot."""
        u, slot = b * Hkv + h, torch.arange(before[b] + new[b], device="cuda")
        if case["layout"] == "blocked":
            return s["table"][u].long().repeat_interleave(BLOCK)[slot] * BLOCK + slot % BLOCK, u * cap + slot
        start = int(s["offsets"][u]) if case["layout"] == "packed" else u * cap
        return start + slot, start + slot

    if case["op"] in ("rope", "append"):
        x = wide["qkv"].view(B, T, Hq + 2 * Hkv, D)
        for b in range(B):
            n = new[b]
            wide["q_out"][b, :, :n] = turned(x[b, :n, :Hq], s["wq"], before[b]).transpose(0, 1)
            wide["k_out"][b, :, :n] = turned(x[b, :n, Hq:Hq + Hkv], s["wk"], before[b]).transpose(0, 1)
        if case["op"] == "rope":
            return wide["q_out"], wide["k_out"]
        for b in range(B):
            for h in range(Hkv):
                rows, flat = place(b, h)
                rows, flat = rows[before[b]:], flat[before[b]:]
                wide["K"].view(-1, D)[rows] = wide["k_out"][b, h, :new[b]]
                wide["V"].view(-1, D)[rows] = x[b, :new[b], Hq + Hkv + h]
                s["pos"].view(-1)[flat] = torch.arange(before[b], before[b] + new[b], dtype=torch.int32, device="cuda")
                wide["score"].view(-1)[flat] = 0.0
                s["state"][b, h] = torch.tensor([before[b] + new[b], 0, -2, 0], dtype=torch.int32)
        return [wide["q_out"], wide["K"], wide["V"], s["pos"], wide["score"], s["state"]]

    for b in range(B):
        later = torch.arange(before[b] + new[b], device="cuda") > before[b] + torch.arange(new[b], device="cuda")[:, None]
        for h in range(Hkv):
            rows, flat = place(b, h)
            k, v = s["K"].view(-1, D)[rows].double(), s["V"].view(-1, D)[rows].double()
            for i in range(h * g, (h + 1) * g):
                logits = (s["q"][b, i, :new[b]].double() @ k.T) * D ** -0.5
                if case["op"] == "attention":
                    logits[later] = -math.inf
                    wide["lse"][b, i, :new[b]] = torch.logsumexp(logits, -1)
                    wide["out"][b, :new[b], i] = torch.softmax(logits, -1) @ v
                else:
                    p = torch.exp(logits - wide["lse"][b, i, :new[b], None])
                    p[later] = 0.0
                    wide["score"].view(-1)[flat] += p.sum(0)
    return (wide["out"], wide["lse"]) if case["op"] == "attention" else wide["score"]
