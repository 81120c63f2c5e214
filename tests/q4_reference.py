"""A cache in 4 bits, positions on several axes and block tables in 64 bits or by hand, one unit at a time (plain torch and lists, no
library code), for their tests.  Test infrastructure only.

Tolerances: those of chunk_reference.py with u = 2^-24, h half a step of the storage type.  Keys and values are exact in bf16 (one
significand bit behind the first, powers within its range), and so are queries in bf16 and fp32 as three parts of 8 bits each.  The
product with V takes probabilities as two parts of bf16 in bf16 calls: the first is cut off to 8 bits (what is left is below 2^-7 of p), the
second rounded (half a step, 2^-8 of that): hp = 2^-15; three parts hold fp32's 24 bits: hp = 0.  Where the probabilities are rounded to
one bf16 hp = 2^-8."""
import math

import torch

import chunk_reference as R

GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
BLOCK = 16


def two_to(e):
    """2^e for whole e, by its bits (a power function may be off in its last bit)."""
    return (e.long() + 1023 << 52).view(torch.float64)


def pack(x):
    """[.., D] -> (values in 64 bits, codes 0..15, bytes of the groups)."""
    x = x.double()
    g = x.unflatten(-1, (-1, 32))
    top = g.abs().amax(-1, keepdim=True)
    finite = torch.isfinite(g).all(-1, keepdim=True)
    m, e = torch.frexp(torch.where(finite, top, 1.0))                            # top = m 2^e, 1/2 <= m < 1: top <= 7 2^p where m 2^e <= 7/8 2^(p + 3)
    e = torch.where(top == 0, -125.0, torch.where(m <= 0.875, e - 3, e - 2).double()).clamp(-125, 125)
    unit = two_to(e)
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    away = ((torch.where(finite, g, 0.0) / unit).abs()[..., None] - grid).abs()
    near = away == away.amin(-1, keepdim=True)
    even = torch.tensor([2, 1] * 4, device=x.device)
    code = (near * even).argmax(-1)
    sign = torch.signbit(g).long()
    value = torch.where(finite, grid[code] * unit * (1 - 2 * sign), math.nan)
    return value.flatten(-2), (code + 8 * sign).flatten(-2), torch.where(finite, e + 127, 255.0)[..., 0].to(torch.uint8)


def codes(packed):
    """uint8 [.., D / 2] -> 0..15, [.., D]."""
    return torch.stack([packed & 15, packed >> 4], -1).flatten(-2).long()


def values(packed, power):
    grid = torch.tensor(GRID + [-v for v in GRID], dtype=torch.float64, device=packed.device)
    scale = torch.where(power == 255, math.nan, two_to(power.long() - 127))
    return grid[codes(packed)] * scale.repeat_interleave(32, -1)


def slot_of(p, capacity, sink):
    return p if p < capacity else sink + (p - sink) % (capacity - sink)


def held(end, capacity, sink):
    """The position in each slot after tokens 0 .. end - 1, None where there is none."""
    at = [None] * capacity
    for p in range(end):
        at[slot_of(p, capacity, sink)] = p
    return at


def attention(q, K, V, seen, dtype, hp):
    """q [g, n, D], K and V [slots, D] in 64 bits, seen [n, slots] -> (out [g, n, D], lse [g, n], bounds of both, the last rounding among them)."""
    q, D = q.double(), q.shape[-1]
    V = torch.where(seen.any(0)[:, None], V, 0.0)
    K = torch.where(seen.any(0)[:, None], K, 0.0)
    s = torch.where(seen, q @ K.T / math.sqrt(D), -math.inf)
    ds = torch.where(seen, (D + 2) * R.U * (q.abs() @ K.abs().T) / math.sqrt(D), 0.0).amax(-1, keepdim=True)
    big = torch.where(seen, s, 0.0).abs().amax(-1, keepdim=True)
    dp = ds + 4 * R.U * big + 4 * R.U
    n = int(seen.sum(-1).max())
    lse = torch.logsumexp(s, -1)
    p = torch.softmax(s, -1)
    out = p @ V
    return out, lse, (2 * dp + 2 * n * R.U + hp) * (p @ V.abs()) + R.HALF[dtype] * out.abs() + 1e-30, dp[..., 0] + n * R.U + 4 * R.U * (lse.abs() + 1)


def axis_of(pairs, turns):
    """The axis of each pair."""
    if not turns:
        return [a for a, n in enumerate(pairs) for _ in range(n)]
    left, order = list(pairs), []
    while any(left):
        for a in range(len(left)):
            if left[a]:
                left[a] -= 1
                order.append(a)
    return order


def norm_rope(x, weight, eps, rope, interleaved, pos, axis):
    """chunk_reference.norm_rope with positions pos [n_axes, n] and pair i by axis[i]; -> (values, the bound on the error before the last
    rounding)."""
    y, bound = R.norm_rope(x, weight, eps, None, False, None)
    z, limit = y.clone(), bound.clone()
    size, half = (x.shape[-1] / 2 + 12) * R.U, rope.shape[1] // 2
    pair = torch.arange(half, device=x.device)
    a, b = (2 * pair, 2 * pair + 1) if interleaved else (pair, pair + half)
    row = pos[torch.tensor(axis[:half], device=x.device)].long()                  # [pairs, n]
    c, s = (rope.double()[row, (pair + k)[:, None]].T[:, None] for k in (0, half))
    z[..., a], z[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
    limit[..., a] = ((y[..., a] * c).abs() + (y[..., b] * s).abs()) * size
    limit[..., b] = ((y[..., b] * c).abs() + (y[..., a] * s).abs()) * size
    return z, limit


def assign(table, tokens, held_blocks, free, capacity, Hkv):
    """sqa_block_assign on lists, in place; free: the list's blocks.  -> whether the list was too short."""
    need = [h if t < 0 else -(-min(t, capacity) // BLOCK) for t, h in zip(tokens, held_blocks)]
    for b, n in enumerate(need):
        for u in range(b * Hkv, (b + 1) * Hkv):
            for e in range(n, held_blocks[b]):
                free.append(table[u][e])
                table[u][e] = -1
        held_blocks[b] = min(held_blocks[b], n)
    short = False
    for b, n in enumerate(need):
        lacks = (n - held_blocks[b]) * Hkv
        if lacks and (short or lacks > len(free)):
            short = True
            continue
        for u in range(b * Hkv, (b + 1) * Hkv):
            for e in range(held_blocks[b], n):
                table[u][e] = free.pop()
        held_blocks[b] = n
    return short
