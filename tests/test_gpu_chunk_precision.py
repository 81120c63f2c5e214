"""How exact the attention of few rows is in bf16: drafts, single tokens, short chunks.  Its probabilities reach the product with V in two parts,
p = high + low, so that what is left is the output's own rounding and not one of the probabilities.

Bound: that of chunk_reference.attention with 2^-15 in place of a rounding of the probabilities.  high is p cut off to 8 bits, so low < 2^-7 p, rounded to
bf16: 2^-7 2^-8 p; the 2^-126 that low is at least is far below 2 u of a row's sum."""
import math

import pytest
import torch

import chunk_reference as R
from test_gpu_chunk import DEV, LAYOUTS, setup, sqa  # noqa: F401

pytestmark = pytest.mark.gpu


def bound(want, p_bound, spread):
    return p_bound * spread + R.HALF[torch.bfloat16] * want.abs() + 1e-30


# B, T, first, Hq, Hkv, n (None: all T): one token, drafts, short chunks; one workgroup and shared-out slots; 32 and 64 rows of a workgroup
FEW = [(1, 1, [0], 1, 1, None), (1, 1, [700], 8, 1, None), (3, 5, [1500, 40, 4000], 10, 2, [5, 1, 4]), (1, 16, [3000], 3, 3, None),
       (16, 5, [1200] * 16, 32, 8, None), (1, 64, [100], 2, 2, None), (40, 64, [200] * 40, 16, 16, None)]


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("D", [64, 128])
def test_few_rows_are_as_exact_as_their_output(sqa, D, layout):  # noqa: F811
    for at, (B, T, first, Hq, Hkv, n) in enumerate(FEW):
        dt, m, c, q, opts, status = setup(sqa, "bf16", D, layout, B, T, first, Hq, Hkv, n, 300 + at)
        out, _ = sqa.chunk_attention(q, first[0], c, opts=opts)
        assert int(status) == 0
        g = Hq // Hkv
        for b in range(0, B, 5):
            for h in range(0, Hkv, 3):
                K, V = R.rows_of(c, b, h, first[b] + m[b])
                heads = slice(h * g, (h + 1) * g)
                s, ds, seen = R.logits(q[b, heads, :m[b]], K, first[b])
                big = torch.where(seen, s, 0.0).abs().amax(-1, keepdim=True)
                dp = ds.amax(-1, keepdim=True) + 4 * R.U * big + 4 * R.U
                p = torch.softmax(s, -1)
                want, spread = p @ V.double(), p @ V.double().abs()
                tol = bound(want, 2 * dp + (2 * K.shape[0] + 2) * R.U + 2.0 ** -15, spread)
                off = (out[b, :m[b], heads].transpose(0, 1).double() - want).abs()
                assert bool((off <= tol).all()), (at, b, h, float((off / tol).max()))


def test_infinite_values_that_a_row_sees_stay_infinite(sqa):  # noqa: F811
    """A value in a slot that takes part with any probability: its column is that infinity, not NaN, and the others are as before."""
    for T, first, g, D in ((1, 300, 8, 128), (5, 1000, 2, 64), (64, 70, 1, 128)):
        _, _, c, q, _, _ = setup(sqa, "bf16", D, "dense", 1, T, [first], 2 * g, 2, None, T)
        q.mul_(0.1)                                        # (probabilities far from 0)
        out, lse = sqa.chunk_attention(q, first, c)
        for slot in (0, first // 2):
            for bad in (math.inf, -math.inf):
                old = c.V[0][0, :, slot].clone()
                c.V[0][0, :, slot, 1::7] = bad
                got, lse2 = sqa.chunk_attention(q, first, c)
                c.V[0][0, :, slot] = old
                hit = torch.zeros(D, dtype=torch.bool, device=DEV)
                hit[1::7] = True
                assert bool((got[..., hit] == bad).all()), (T, slot, bad)
                assert R.same([out[..., ~hit].contiguous(), lse], [got[..., ~hit].contiguous(), lse2])


def test_infinite_values_at_the_smallest_probabilities(sqa):  # noqa: F811
    """exp(-d) for d up to 87 is not 0 in fp32, and times an infinite value it is that infinity.  64 slots of as many probabilities, each with an
    infinite value in a column of its own."""
    D, T, first = 64, 3, 500
    for d in (0.0, 0.5, 10.0, 70.0, 78.0, 82.0, 85.0, 86.0):
        _, _, c, q, _, _ = setup(sqa, "bf16", D, "dense", 1, T, [first], 4, 2, None, 9)
        q.zero_()
        q[..., :2] = 8.0                                   # s = K[0] + K[1] in every row: 8 / sqrt(64)
        c.K[0][:, :, :first + T, :2] = 0.0
        for j in range(D):
            c.K[0][:, :, 3 * j, 0] = -d
            c.K[0][:, :, 3 * j, 1] = -j / 64.0
            c.V[0][:, :, 3 * j, j] = math.inf
        out, _ = sqa.chunk_attention(q, first, c)
        assert bool((out == math.inf).all()), (d, (out != math.inf).nonzero()[:5].tolist())
