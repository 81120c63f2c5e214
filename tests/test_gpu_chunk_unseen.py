"""Slots that a token may not see do not change its row, to the bit: large finite keys in them (a rejected draft's, say) move the softmax reference
and the way it is subtracted for the rows that see them, and for no other row of the same wave."""
import pytest
import torch

import chunk_reference as R
from test_gpu_chunk import setup, sqa  # noqa: F401

pytestmark = pytest.mark.gpu


# B, T, first, Hq, Hkv: few rows; 64 rows of a workgroup; 128 (many units, or many slots)
@pytest.mark.parametrize("B,T,first,Hq,Hkv", [(1, 5, 300, 8, 2), (2, 40, 0, 2, 2), (40, 64, 200, 16, 16), (4, 300, 3000, 8, 2), (8, 150, 90, 64, 32), (2, 130, 20, 160, 80)])
@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
def test_large_keys_in_slots_that_a_row_does_not_see(sqa, dtype, D, B, T, first, Hq, Hkv):  # noqa: F811
    dt, _, c, q, _, _ = setup(sqa, dtype, D, "dense", B, T, [first] * B, Hq, Hkv, None, 41)
    g = Hq // Hkv
    ws = sqa.chunk_workspace(c, Hq, T)
    out, lse = sqa.chunk_attention(q, first, c, workspace=ws)
    keys = c.K[0]
    for t in (T // 3, T // 2 + 1, T - 1):
        old = keys[:, :, first + t].clone()
        for size in (0.3, 1.0, 4.0, 40.0, -40.0):            # logits of about 8 to 1000: q.q is 2.25 D
            keys[:, :, first + t] = (q[:, ::g, t].float() * size).to(dt)
            got, got_lse = sqa.chunk_attention(q, first, c, workspace=ws)
            assert R.same([out[:, :t].contiguous(), lse[..., :t].contiguous()], [got[:, :t].contiguous(), got_lse[..., :t].contiguous()]), (t, size)
            assert not torch.equal(lse[..., t], got_lse[..., t])
        keys[:, :, first + t] = old


@pytest.mark.parametrize("B,T,Hq,Hkv", [(3, 5, 8, 2), (40, 64, 16, 16), (8, 150, 64, 32), (4, 300, 8, 2)])
def test_positions_up_to_the_last(sqa, B, T, Hq, Hkv):  # noqa: F811
    """A sequence whose position lies far beyond its unit's slots, up to 2^31 - 1: rows of zeros, whatever the form; the others as ever."""
    dt, _, c, q, _, status = setup(sqa, "bf16", 64, "dense", B, T, [100] * B, Hq, Hkv, [T] * B, 43)
    good, good_lse = sqa.chunk_attention(q, 0, c, opts=sqa.batch_opts(new_pos_seq=torch.full((B,), 100, dtype=torch.int32, device=q.device)))
    for far in (2 ** 31 - 1, 2 ** 31 - T, 2 ** 31 - 63, 2 ** 30, 101 + T):
        pos = torch.full((B,), 100, dtype=torch.int32, device=q.device)
        pos[B - 1] = far
        status.zero_()
        opts = sqa.batch_opts(new_pos_seq=pos, status=status)
        out, lse = sqa.chunk_attention(q, 0, c, opts=opts)
        assert int(status) == 8 and bool((out[B - 1] == 0).all()) and bool((lse[B - 1] == -float("inf")).all()), far
        assert R.same([good[:B - 1], good_lse[:B - 1]], [out[:B - 1], lse[:B - 1]])
        score0 = c.score[0].clone()
        status.zero_()
        sqa.chunk_scores(q, good_lse, 0, c, opts=opts)
        assert int(status) == 8 and R.same([score0[B - 1]], [c.score[0][B - 1]])
