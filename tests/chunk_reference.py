"""The calls on chunks of tokens in 64 bits, one unit at a time (plain torch, no library code), caches of every layout for
their tests, and how far fp32 arithmetic may be off.  Test infrastructure only.

Tolerances.  u = 2^-24 is half a step of fp32, h half a step of the storage type (2^-8 bf16, 2^-24 fp32).
  logits     a sum of D products: at most (D + 2) u (sum_d |q_d k_d|) / sqrt(D) off -- ds
  exp        of an argument that is off by ds and, in powers of two, by a rounding of its own size (s and the reference it
             is taken against, each below S = max |s|): relative error dp = ds + 4 u S + 4 u (v_exp_f32: one step)
  sums       of n terms: n u, relative to the sum of their absolute values
  out        sum p v / sum p: (2 dp + 2 n u + hp) sum p |v|, and h |out| for the last rounding; hp: probabilities are rounded to
             the storage type for the product (bf16 only)
  lse        dp + n u + 4 u (|lse| + 1)
  scores     sum over rows of p (dp + 4 u (|s| + |lse|)) + n u, and u for each number that is added
  norm+rope  a sum of D squares, a root, a quotient, three products and a sum: (D / 2 + 12) u (|a cos| + |b sin|), and h |y|
"""
import math

import torch

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def norm_rope(x, weight, eps, rope, interleaved, pos):
    """x [n, H, D], pos [n] -> ([n, H, D] in 64 bits, the bound on the error before the last rounding)."""
    x = x.double()
    D = x.shape[-1]
    size = (D / 2 + 12) * U
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    y, bound = x.clone(), x.abs() * size
    if rope is not None:
        R = rope.shape[1]
        for i in range(R // 2):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
            c, s = rope[pos, i].double()[:, None], rope[pos, R // 2 + i].double()[:, None]
            y[..., a] = x[..., a] * c - x[..., b] * s
            y[..., b] = x[..., b] * c + x[..., a] * s
            bound[..., a] = ((x[..., a] * c).abs() + (x[..., b] * s).abs()) * size
            bound[..., b] = ((x[..., b] * c).abs() + (x[..., a] * s).abs()) * size
    return y, bound


def logits(q, K, first):
    """q [g, n, D] at positions first .., K [slots, D] -> (s [g, n, slots] with -inf where not seen, bound ds, seen)."""
    q, K = q.double(), K.double()
    s = q @ K.T / math.sqrt(q.shape[-1])
    ds = (q.shape[-1] + 2) * U * (q.abs() @ K.abs().T) / math.sqrt(q.shape[-1])
    seen = torch.arange(K.shape[0], device=K.device) <= first + torch.arange(q.shape[1], device=K.device)[:, None]
    return torch.where(seen, s, -math.inf), torch.where(seen, ds, 0.0), seen


def attention(q, K, V, first, dtype):
    """-> (out [g, n, D], lse [g, n], bounds of both, the last rounding among them)."""
    s, ds, seen = logits(q, K, first)
    V = torch.where(torch.isfinite(V.double()), V.double(), 0.0)            # (what no row sees may be anything)
    big = torch.where(seen, s, 0.0).abs().amax(-1, keepdim=True)
    dp = ds.amax(-1, keepdim=True) + 4 * U * big + 4 * U
    n = K.shape[0]
    lse = torch.logsumexp(s, -1)
    p = torch.softmax(s, -1)
    out, spread = p @ V, p @ V.abs()
    hp = HALF[dtype] if dtype == torch.bfloat16 else 0.0
    return out, lse, (2 * dp + 2 * n * U + hp) * spread + HALF[dtype] * out.abs() + 1e-30, dp[..., 0] + n * U + 4 * U * (lse.abs() + 1)


def scores(q, K, lse, first, before):
    """What the rows add to `before` [slots] -> (scores, bound)."""
    s, ds, seen = logits(q, K, first)
    p = torch.where(seen, torch.exp(s - lse.double()[..., None]), 0.0)
    dp = ds + 4 * U * (torch.where(seen, s, 0.0).abs() + lse.double().abs()[..., None]) + 4 * U
    rows = q.shape[0] * q.shape[1]
    added = p.sum((0, 1))
    return before.double() + added, (p * dp).sum((0, 1)) + (rows + 2) * U * added + 2 * U * before.double().abs() + 1e-30


def make_cache(sqa, layout, B, Hkv, D, dtype, room, device="cuda:0", budget=None):
    """One layer of `layout`; room[b]: slots of sequence b's units ("packed"), the largest otherwise."""
    cap = max(room)
    return sqa.LayerCaches([cap if budget is None else budget], [cap], B, Hkv, D, dtype, device, True, blocked=layout == "blocked",
                           unit_capacities=[[room[b] for b in range(B) for _ in range(Hkv)]] if layout == "packed" else None)


def fill(caches, held, gen, value=None):
    """Tokens 0 .. held[b]-1 in every unit, random keys, values and scores; `value` in every other slot."""
    for x in (caches.K[0], caches.V[0]):
        x.copy_(torch.randn(x.shape, generator=gen, device=x.device).to(x.dtype))
        if value is not None:
            keep = x.clone()
            x.fill_(value)
            for b in range(caches.B):
                for h in range(caches.Hkv):
                    rows = caches.unit_kv_rows(0, b, h)[2][:held[b]]
                    x.view(-1, caches.D)[rows] = keep.view(-1, caches.D)[rows]
    if value is not None:
        caches.score[0].fill_(value)
    for b in range(caches.B):
        for h in range(caches.Hkv):
            _, _, score, pos = caches.unit(0, b, h)
            pos[:held[b]] = torch.arange(held[b], dtype=torch.int32, device=pos.device)
            score[:held[b]] = torch.rand(held[b], generator=gen, device=pos.device)
        caches.lens[0][b] = held[b]
    caches.head[0].zero_()
    caches.hint[0].fill_(-2)
    return caches


def rows_of(caches, b, h, n):
    """K and V of unit (b, h)'s first n slots."""
    K, V, idx = caches.unit_kv_rows(0, b, h)
    return K[idx[:n]], V[idx[:n]]


def snapshot(caches):
    return [x.clone() for x in (caches.K[0], caches.V[0], caches.score[0], caches.pos[0], caches.state[0])]


def same(before, after):
    """Bit for bit (NaN included)."""
    return all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(before, after))
