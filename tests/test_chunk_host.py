"""Calls on chunks of tokens, what can be seen without a GPU: the reference's formulas against the oracle's, struct layouts, and
every argument that is refused before any GPU call."""
import ctypes as C

import numpy as np
import pytest
import torch

import chunk_reference as R
from oracle import sqa_oracle as O
from paper_2404_04793_amd import binding as sqa

lib = sqa._lib
P = C.c_void_p


def test_reference_formulas_agree_with_the_oracle():
    g, n, D = 3, 21, 64
    gen = torch.Generator().manual_seed(3)
    q, K, V = (torch.randn(*s, generator=gen, dtype=torch.float64) for s in ((g, n, D), (n, D), (n, D)))
    out, lse, _, _ = R.attention(q, K, V, 0, torch.float32)
    np.testing.assert_allclose(lse.numpy(), O.prefill_row_lse(q.numpy(), K.numpy()), rtol=1e-13)
    added, _ = R.scores(q, K, lse, 0, torch.zeros(n))
    np.testing.assert_allclose(added.numpy(), O.prefill_scores(q.numpy(), K.numpy()), rtol=1e-12)
    for t in range(n):
        want, _ = O.attend(q[:, t].numpy(), K[:t + 1].numpy(), V[:t + 1].numpy())
        np.testing.assert_allclose(out[:, t].numpy(), want, rtol=1e-11, atol=1e-13)
    # a chunk at the end of the same cache
    late, _, _, _ = R.attention(q[:, 15:], K, V, 15, torch.float32)
    np.testing.assert_allclose(late.numpy(), out[:, 15:].numpy(), rtol=1e-13, atol=1e-15)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_rotation_and_norm_gives_unit_rows(interleaved):
    gen = torch.Generator().manual_seed(5)
    x = torch.randn(7, 2, 64, generator=gen, dtype=torch.float64)
    rope = sqa.rope_table(100, 32, device="cpu").double()
    pos = torch.arange(40, 47)
    y, _ = R.norm_rope(x, None, 0.0, rope, interleaved, pos)
    torch.testing.assert_close(y.norm(dim=-1), x.norm(dim=-1), rtol=1e-7, atol=0)     # (cos^2 + sin^2 of fp32 numbers)
    assert torch.equal(y[..., 32:], x[..., 32:])
    z, _ = R.norm_rope(x * 17, torch.ones(64), 0.0, None, False, pos)
    torch.testing.assert_close(z.square().mean(-1), torch.ones(7, 2, dtype=torch.float64), rtol=1e-12, atol=0)
    # what attention sees depends on the distance alone
    a, _ = R.norm_rope(x[:1], None, 0.0, rope, interleaved, torch.tensor([3]))
    b, _ = R.norm_rope(x[1:2], None, 0.0, rope, interleaved, torch.tensor([9]))
    c, _ = R.norm_rope(x[:1], None, 0.0, rope, interleaved, torch.tensor([53]))
    d, _ = R.norm_rope(x[1:2], None, 0.0, rope, interleaved, torch.tensor([59]))
    torch.testing.assert_close((a * b).sum(-1), (c * d).sum(-1), rtol=1e-5, atol=1e-5)


def test_rope_table_in_64_bits():
    t = sqa.rope_table(100001, 128, 10000.0, "cpu")
    assert t.shape == (100001, 128) and t.dtype == torch.float32
    import math
    for p, i in ((0, 0), (1, 0), (100000, 0), (99999, 3), (77777, 63)):
        a = p / 10000.0 ** (2 * i / 128)
        assert abs(float(t[p, i]) - math.cos(a)) < 1e-7 and abs(float(t[p, 64 + i]) - math.sin(a)) < 1e-7


def test_struct_layouts():
    assert C.sizeof(sqa.TokenRowsStruct) == 24 and sqa.TokenRowsStruct.row_stride.offset == 16
    assert C.sizeof(sqa.HeadPrepStruct) == 40 and sqa.HeadPrepStruct.eps.offset == 24 and sqa.HeadPrepStruct.interleaved.offset == 36


def rows(ptr=0x100000, seq=4096, row=512):
    return C.byref(sqa.TokenRowsStruct(ptr, seq, row))


def layer(cap=64, budget=64, K=0x4000000, score=0x3000, table=None, bpu=0, nb=0, offset=None):
    return sqa.LayerCacheStruct(K, 0x8000000, score, 0x4000, 0x5000, offset, table, cap, budget, bpu, nb)


def prep(**kw):
    base = dict(q_weight=None, k_weight=None, rope=0x7000, eps=1e-6, n_pos=100, rot_dim=64, interleaved=0)
    base.update(kw)
    return C.byref(sqa.HeadPrepStruct(*[base[f] for f, _ in sqa.HeadPrepStruct._fields_]))


NULL, SHAPE, DTYPE, BUDGET, CAP = 1, 2, 3, 5, 6


@pytest.mark.parametrize("change,code", [
    (dict(q=None, k=None), NULL), (dict(q_out=None), NULL), (dict(k_out=None), NULL), (dict(q=None), NULL), (dict(q=rows(None)), NULL),
    (dict(dt=2), DTYPE), (dict(dt=-1), DTYPE), (dict(B=0), SHAPE), (dict(T=0), SHAPE), (dict(Hq=5), SHAPE), (dict(Hkv=0), SHAPE),
    (dict(D=96), SHAPE), (dict(D=256), SHAPE), (dict(new_pos=-1), SHAPE), (dict(T=1 << 30, Hq=4), SHAPE), (dict(new_pos=2 ** 31 - 2), SHAPE),
    (dict(q=rows(0x100008)), SHAPE), (dict(q=rows(row=-8)), SHAPE), (dict(q=rows(row=12)), SHAPE), (dict(k=rows(seq=4)), SHAPE),
    (dict(q_out=P(0x2000008)), SHAPE), (dict(q_out=P(0x100000)), SHAPE), (dict(q_out=P(0x3000000)), SHAPE), (dict(k_out=P(0x100100)), SHAPE),
    (dict(prep=prep(rot_dim=24)), SHAPE), (dict(prep=prep(rot_dim=80)), SHAPE), (dict(prep=prep(rot_dim=0)), SHAPE),
    (dict(prep=prep(n_pos=0)), SHAPE), (dict(prep=prep(interleaved=2)), SHAPE), (dict(prep=prep(rope=0x7004)), SHAPE),
    (dict(prep=prep(q_weight=0x8008)), SHAPE), (dict(prep=prep(q_weight=0x8000, eps=float("nan"))), SHAPE),
    (dict(prep=prep(k_weight=0x8000, eps=-1.0)), SHAPE), (dict(new_pos=97), SHAPE), (dict(prep=prep(n_pos=13)), SHAPE)])
def test_qk_norm_rope_refusals(change, code):
    a = dict(q=rows(), k=rows(0x200000), dt=1, B=2, T=4, Hq=4, Hkv=2, D=64, prep=prep(), new_pos=10, q_out=P(0x3000000), k_out=P(0x3000000 + (2 << 20)),
             stream=None, opts=None)
    if "q_out" in change and change["q_out"] is not None and change["q_out"].value == 0x3000000:
        change = dict(change, k_out=P(0x3000100))                       # the two outputs overlap
    a.update(change)
    assert lib.sqa_qk_norm_rope(*a.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(layer=None), NULL), (dict(v=rows(None)), NULL), (dict(q_out=None), NULL), (dict(q=None), NULL),
    (dict(layer=layer(K=None)), NULL), (dict(layer=layer(K=0x4000004)), SHAPE), (dict(layer=layer(budget=0)), BUDGET), (dict(layer=layer(cap=0)), CAP),
    (dict(dt=5), DTYPE), (dict(D=32), SHAPE), (dict(v=rows(0x300004)), SHAPE),
    (dict(new_pos=61), CAP), (dict(layer=layer(budget=13)), CAP), (dict(layer=layer(cap=13)), CAP),
    (dict(layer=layer(table=0x9000, bpu=3, nb=9)), SHAPE), (dict(layer=layer(table=0x9000, bpu=4, nb=0)), SHAPE),
    (dict(layer=layer(table=0x9000, bpu=4, nb=9, offset=0xa000)), SHAPE), (dict(layer=layer(table=0x9000, bpu=1025, nb=9)), SHAPE),
    (dict(k=rows(0x4000100)), SHAPE), (dict(v=rows(0x8000000)), SHAPE), (dict(new_pos=-1), SHAPE), (dict(prep=prep(n_pos=12)), SHAPE)])
def test_chunk_append_refusals(change, code):
    a = dict(q=rows(), k=rows(0x200000), v=rows(0x300000), dt=1, B=2, T=4, Hq=4, Hkv=2, D=64, prep=prep(), new_pos=10, q_out=P(0x2000000),
             layer=layer(), stream=None, opts=None)
    a.update(change)
    ref = a["layer"]
    a["layer"] = None if ref is None else C.addressof(ref)
    assert lib.sqa_chunk_append(*a.values()) == code


COMMON = [(dict(q=None), NULL), (dict(layer=None), NULL), (dict(ws=None), NULL), (dict(layer=layer(K=None)), NULL), (dict(dt=2), DTYPE),
          (dict(B=0), SHAPE), (dict(T=0), SHAPE), (dict(Hq=3), SHAPE), (dict(D=80), SHAPE), (dict(new_pos=-1), SHAPE), (dict(q=P(0x100008)), SHAPE),
          (dict(ws=P(0x10)), SHAPE), (dict(ws_bytes=4096), CAP), (dict(new_pos=61), CAP), (dict(layer=layer(table=0x9000, bpu=3, nb=9)), SHAPE)]


@pytest.mark.parametrize("change,code", COMMON + [(dict(out=None), NULL), (dict(out=P(0x2000008)), SHAPE), (dict(out=P(0x100000)), SHAPE),
                                                  (dict(lse=P(0x2000100)), SHAPE), (dict(lse=P(0x600002)), SHAPE)])
def test_chunk_attention_refusals(change, code):
    a = dict(q=P(0x100000), dt=1, B=2, T=4, Hq=4, Hkv=2, D=64, new_pos=10, layer=layer(), out=P(0x2000000), lse=P(0x600000), ws=P(0x10000000),
             ws_bytes=1 << 30, stream=None, opts=None)
    a.update(change)
    ref = a["layer"]
    a["layer"] = None if ref is None else C.addressof(ref)
    assert lib.sqa_chunk_attention(*a.values()) == code


@pytest.mark.parametrize("change,code", COMMON + [(dict(lse=None), NULL), (dict(lse=P(0x600001)), SHAPE), (dict(layer=layer(score=None)), NULL)])
def test_chunk_scores_refusals(change, code):
    a = dict(q=P(0x100000), lse=P(0x600000), dt=1, B=2, T=4, Hq=4, Hkv=2, D=64, new_pos=10, layer=layer(), ws=P(0x10000000), ws_bytes=1 << 30,
             stream=None, opts=None)
    a.update(change)
    ref = a["layer"]
    a["layer"] = None if ref is None else C.addressof(ref)
    assert lib.sqa_chunk_scores(*a.values()) == code


def test_workspace_holds_for_every_shorter_chunk():
    """One workspace serves chunks of every length up to the one it was made for."""
    need = lambda B, T, Hq, Hkv, D: lib.sqa_chunk_workspace_bytes(C.addressof(keep), B, T, Hq, Hkv, D)
    keep = layer(cap=5000, budget=5000)
    for B, Hq, Hkv, D in ((1, 8, 8, 128), (3, 24, 8, 64), (16, 64, 8, 128), (2, 5, 1, 128)):
        sizes = [need(B, T, Hq, Hkv, D) for T in (1, 2, 3, 7, 8, 16, 17, 33, 64, 65, 129, 1000)]
        assert sizes == sorted(sizes) and sizes[0] > 4096 and all(s % 256 == 0 for s in sizes)
    assert need(0, 1, 8, 8, 128) == 0 and need(1, 1, 8, 3, 128) == 0 and need(1, 1, 8, 8, 96) == 0 and need(1, 0, 8, 8, 64) == 0
    assert lib.sqa_chunk_workspace_bytes(None, 1, 1, 8, 8, 64) == 0


def test_binding_refuses_what_it_cannot_describe():
    x = torch.zeros(2, 3, 4, 64)
    c = sqa.LayerCaches([8], [8], 2, 4, 64, torch.float32, "cpu", True)
    q, ws = torch.zeros(2, 4, 3, 64), torch.zeros(1 << 20, dtype=torch.uint8)
    refused = [
        ("queries or keys", lambda: sqa.qk_norm_rope(None, None, 0)),
        ("one after the other", lambda: sqa.qk_norm_rope(x.transpose(1, 2), None, 0)),
        ("one after the other", lambda: sqa.chunk_append(x, x.flip(0).transpose(2, 3).contiguous().transpose(2, 3), 0, c)),
        ("same tokens", lambda: sqa.qk_norm_rope(x, torch.zeros(2, 2, 4, 64), 0)),
        ("contiguous", lambda: sqa.qk_norm_rope(x, None, 0, q_out=torch.zeros(2, 4, 3, 32))),
        ("without its input", lambda: sqa.qk_norm_rope(x, None, 0, k_out=torch.zeros(2, 4, 3, 64))),
        ("call's dtype", lambda: sqa.qk_norm_rope(x, None, 0, prep=sqa.head_prep(torch.ones(64, dtype=torch.bfloat16)))),
        ("call's dtype", lambda: sqa.qk_norm_rope(x, None, 0, prep=sqa.head_prep(torch.ones(32)))),
        ("fp32", lambda: sqa.head_prep(rope=torch.zeros(4, 64, dtype=torch.float64))),
        ("norm weights", lambda: sqa.head_prep(torch.ones(2, 64))),
        ("one shape", lambda: sqa.chunk_append(x, x[:, :2], 0, c)),
        ("another dtype", lambda: sqa.chunk_append(x.bfloat16(), x.bfloat16(), 0, c)),
        ("another dtype", lambda: sqa.chunk_append(x[:1], x[:1], 0, c)),
        ("without its input", lambda: sqa.chunk_append(x, x, 0, c, q_out=x)),
        ("contiguous", lambda: sqa.chunk_attention(q.transpose(1, 2), 0, c)),
        ("contiguous", lambda: sqa.chunk_attention(q, 0, c, out=torch.zeros(2, 4, 3, 64), workspace=ws)),
        ("lse", lambda: sqa.chunk_scores(q, torch.zeros(2, 4, 4), 0, c))]
    for what, call in refused:
        with pytest.raises(TypeError, match=what):
            call()
    with pytest.raises(IndexError):
        sqa.chunk_append(x, x, 0, c, layer=1)
    # tensors of the host never reach a kernel
    for call in (lambda: sqa.qk_norm_rope(x, x, 0), lambda: sqa.chunk_append(x, x, 0, c), lambda: sqa.chunk_attention(q, 0, c, workspace=ws),
                 lambda: sqa.chunk_scores(q, torch.zeros(2, 4, 3), 0, c, workspace=ws)):
        with pytest.raises(ValueError, match="current device"):
            call()
