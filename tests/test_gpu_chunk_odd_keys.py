"""Keys that are not finite, row by row.  One element of a key is NaN or infinite, so that a row's logit with it is NaN, +inf or -inf by the sign of its
query's element.  The definition then says
  rows that do not see it   what they are without it, to the bit
  NaN, +inf                 softmax is NaN (inf - inf): a row of NaN, a log-sum-exp that is NaN or +inf
  -inf                      probability 0: the softmax over the other slots, within the usual bounds"""
import math

import pytest
import torch

import chunk_reference as R
from test_gpu_chunk import LAYOUTS, setup, sqa  # noqa: F401

pytestmark = pytest.mark.gpu


# few rows, alone and shared out; 64 rows; 128 rows alone and shared out
@pytest.mark.parametrize("B,T,first,Hq,Hkv", [(1, 5, 0, 8, 2), (1, 3, 1000, 4, 2), (3, 70, 30, 3, 3), (40, 64, 200, 16, 16), (8, 150, 90, 64, 32), (4, 300, 3000, 8, 2)])
@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
def test_one_element_of_a_key(sqa, dtype, D, B, T, first, Hq, Hkv):  # noqa: F811
    layout = LAYOUTS[(T + D) % 3]
    dt, _, c, q, _, _ = setup(sqa, dtype, D, layout, B, T, [first] * B, Hq, Hkv, None, 71)
    g, d = Hq // Hkv, 37
    ws = sqa.chunk_workspace(c, Hq, T)
    out, lse = sqa.chunk_attention(q, first, c, workspace=ws)
    assert bool((q[..., d] != 0).all())
    for at in ([first // 2] if first else []) + [first + T // 2, first + T - 1]:
        t = max(at - first, 0)                                       # the first token that sees it
        rows = torch.stack([c.unit_kv_rows(0, b, h)[2][at] for b in range(B) for h in range(Hkv)])
        mem = c.K[0].view(-1, D)
        old = mem[rows].clone()
        for bad in (math.nan, math.inf, -math.inf):
            new = old.clone()
            new[:, d] = bad
            mem[rows] = new
            got, got_lse = sqa.chunk_attention(q, first, c, workspace=ws)
            mem[rows] = old
            assert R.same([out[:, :t].contiguous(), lse[..., :t].contiguous()], [got[:, :t].contiguous(), got_lse[..., :t].contiguous()]), (at, bad)
            late, late_lse = got[:, t:].transpose(1, 2), got_lse[..., t:]                       # [B, Hq, T - t, D]
            logit = q[:, :, t:, d].double() * bad
            spoilt = logit != -math.inf
            assert bool(late[spoilt].isnan().all()) and bool((late_lse[spoilt].isnan() | (late_lse[spoilt] == math.inf)).all()), (at, bad)
            assert bool(torch.isfinite(late[~spoilt]).all()) if first else True, (at, bad)
            for b in range(0, B, 3):
                for h in range(0, Hkv, 5):
                    K, V = R.rows_of(c, b, h, first + T)
                    heads = slice(h * g, (h + 1) * g)
                    s, ds, seen = R.logits(q[b, heads], K, first)
                    seen = seen & (torch.arange(first + T, device=q.device) != at)
                    s = torch.where(seen, s, -math.inf)[:, t:]
                    big = torch.where(seen[t:], s, 0.0).abs().amax(-1, keepdim=True)
                    dp = torch.where(seen, ds, 0.0).amax(-1, keepdim=True)[:, t:] + 4 * R.U * big + 4 * R.U
                    p, n = torch.softmax(s, -1), first + T
                    want, spread, want_lse = p @ V.double(), p @ V.double().abs(), torch.logsumexp(s, -1)
                    tol = (2 * dp + 2 * n * R.U + (R.HALF[dt] if dt == torch.bfloat16 else 0.0)) * spread + R.HALF[dt] * want.abs() + 1e-30
                    tol_lse = dp[..., 0] + n * R.U + 4 * R.U * (want_lse.abs() + 1)
                    keep = ~spoilt[b, heads] & torch.isfinite(want_lse)                      # (a row that sees nothing else has no softmax)
                    assert bool(((late[b, heads].double() - want).abs() <= tol)[keep].all()), (at, bad, b, h)
                    assert bool(((late_lse[b, heads].double() - want_lse).abs() <= tol_lse)[keep].all()), (at, bad, b, h)
