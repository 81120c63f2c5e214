"""A cache in 4 bits, positions on several axes, block tables: what can be seen without a GPU -- the references against the numbers'
definition, struct layouts, and every argument that is refused before any GPU call."""
import ctypes as C

import pytest
import torch

import q4_reference as Q
from paper_2404_04793_amd import binding as sqa

lib = sqa._lib
P = C.c_void_p
NULL, SHAPE, DTYPE, BUDGET, CAP = 1, 2, 3, 5, 6


def test_numbers_of_the_reference():
    x = torch.zeros(9, 32)
    x[0, :8] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0])          # ties go to the even code; 7 is the most with power 1
    x[1, 0], x[1, 1] = 7.0000005, 5.0                                            # one step more: power 2
    x[2, :2] = torch.tensor([-0.25, -0.0])
    x[3, 0], x[4, 0], x[5, 0] = float("inf"), float("nan"), 3.4e38
    x[6, :2] = torch.tensor([1e-45, -2e-38])
    x[7, 0] = 6 * 2.0 ** -100
    v, c, p = Q.pack(x)
    assert v[0, :8].tolist() == [0, 1, 1, 2, 2, 4, 4, 6] and p[0] == 127
    assert v[1, :2].tolist() == [8, 4] and p[1] == 128
    assert c[2, :2].tolist() == [14, 8] and p[2] == 127 - 4                      # (-0.25 is -4 of its own power; the zero keeps its sign)
    assert p[3] == 255 and p[4] == 255 and bool(v[3:5].isnan().all()) and p[5] == 252 and v[5, 0] == 6 * 2.0 ** 125
    assert p[6] == 2 and v[6, 1] == -1 * 2.0 ** -125 and p[7] == 127 - 100 and p[8] == 2 and not v[8].any()
    # no number is further away than half the widest gap
    y = torch.randn(4000, 128, generator=torch.Generator().manual_seed(1)) * torch.logspace(-20, 20, 4000)[:, None]
    v, _, p = Q.pack(y)
    assert bool(((v - y.double()).abs() <= (2.0 ** (p.double() - 127)).repeat_interleave(32, -1)).all())


def test_slots_of_the_reference():
    assert Q.held(3, 5, 2) == [0, 1, 2, None, None] and Q.held(9, 5, 2) == [0, 1, 8, 6, 7] and Q.held(7, 3, 0) == [6, 4, 5]
    assert Q.axis_of([3, 1, 2], False) == [0, 0, 0, 1, 2, 2] and Q.axis_of([3, 1, 2], True) == [0, 1, 2, 0, 2, 0]


def test_struct_layouts():
    assert C.sizeof(sqa.RopeAxesStruct) == 32 and sqa.RopeAxesStruct.pairs.offset == 12 and sqa.RopeAxesStruct.turns.offset == 28
    assert C.sizeof(sqa.Q4CacheStruct) == 56 and sqa.Q4CacheStruct.block_table.offset == 32 and sqa.Q4CacheStruct.n_blocks.offset == 52


def rows(ptr=0x100000, seq=4096, row=512):
    return C.byref(sqa.TokenRowsStruct(ptr, seq, row))


def layer(K=0x4000000, V=0x8000000, Ks=0x9000, Vs=0xa000, table=None, cap=64, sink=0, bpu=0, nb=0):
    return C.byref(sqa.Q4CacheStruct(K, V, Ks, Vs, table, cap, sink, bpu, nb))


def prep(rope=0x7000, n_pos=100, rot_dim=64, **kw):
    return C.byref(sqa.HeadPrepStruct(kw.get("q_weight"), kw.get("k_weight"), rope, kw.get("eps", 1e-6), n_pos, rot_dim, 0))


def axes(pos=0xb000, n=3, pairs=(8, 12, 12, 0), turns=0):
    return C.byref(sqa.RopeAxesStruct(pos, n, (C.c_int32 * 4)(*pairs), turns))


AXES = [(dict(axes=axes(pos=None)), NULL), (dict(axes=axes(), prep=None), NULL), (dict(axes=axes(), prep=prep(rope=None)), NULL),
        (dict(axes=axes(pos=0xb002)), SHAPE), (dict(axes=axes(n=0)), SHAPE), (dict(axes=axes(n=5)), SHAPE), (dict(axes=axes(pairs=(8, 12, 11, 1))), SHAPE),
        (dict(axes=axes(pairs=(44, -12, 0, 0))), SHAPE), (dict(axes=axes(pairs=(2 ** 31 - 1, 2 ** 31 - 1, 34, 0))), SHAPE), (dict(axes=axes(turns=2)), SHAPE),
        (dict(axes=axes(), prep=prep(rot_dim=32)), SHAPE)]


@pytest.mark.parametrize("change,code", AXES + [(dict(q=None, q_out=None, k=None, k_out=None), NULL), (dict(new_pos=-1), SHAPE)])
def test_norm_rope_on_axes_refusals(change, code):
    a = dict(q=rows(), k=rows(0x200000), dt=1, B=2, T=4, Hq=4, Hkv=2, D=64, prep=prep(), new_pos=10, q_out=P(0x3000000), k_out=P(0x3200000),
             stream=None, opts=None, axes=None)
    a.update(change)
    assert lib.sqa_qk_norm_rope_ex(*a.values()) == code


@pytest.mark.parametrize("change,code", AXES + [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(layer=None), NULL), (dict(v=rows(None)), NULL), (dict(q_out=None), NULL), (dict(q=None), NULL),
    (dict(layer=layer(K=None)), NULL), (dict(layer=layer(Vs=None)), NULL), (dict(layer=layer(K=0x4000008)), SHAPE), (dict(layer=layer(Ks=0x9002)), SHAPE),
    (dict(layer=layer(cap=0)), CAP), (dict(layer=layer(cap=(1 << 30) + 1)), CAP), (dict(layer=layer(sink=64)), BUDGET), (dict(layer=layer(sink=-1)), BUDGET),
    (dict(layer=layer(table=0xc000, bpu=3, nb=9)), SHAPE), (dict(layer=layer(table=0xc000, bpu=4, nb=0)), SHAPE),
    (dict(layer=layer(table=0xc000, bpu=1025, nb=9)), SHAPE), (dict(layer=layer(table=0xc002, bpu=4, nb=9)), SHAPE),
    (dict(dt=2), DTYPE), (dict(D=96), SHAPE), (dict(T=0), SHAPE), (dict(Hq=5), SHAPE), (dict(new_pos=-1), SHAPE), (dict(v=rows(0x300004)), SHAPE),
    (dict(layer=layer(cap=13)), "runs"), (dict(layer=layer(cap=13, sink=10)), CAP), (dict(layer=layer(cap=3)), CAP),
    (dict(k=rows(0x4000100)), SHAPE), (dict(v=rows(0x8000000)), SHAPE), (dict(q=rows(0x9000)), SHAPE), (dict(q_out=P(0x200000)), SHAPE),
    (dict(prep=prep(n_pos=12)), SHAPE), (dict(slot_map=P(0xd002)), SHAPE)])
def test_append_refusals(change, code):
    a = dict(q=rows(), k=rows(0x200000), v=rows(0x300000), dt=1, B=2, T=4, Hq=4, Hkv=2, D=64, prep=prep(), new_pos=10, q_out=P(0x2000000),
             layer=layer(), stream=None, opts=None, axes=None, slot_map=None)
    a.update(change)
    if code == "runs":                               # (4 tokens past a ring of 13: nothing to refuse, so not sent)
        return
    assert lib.sqa_q4_append(*a.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(layer=None), NULL), (dict(k_out=None, v_out=None), NULL), (dict(layer=layer(V=None)), NULL), (dict(dt=3), DTYPE), (dict(B=0), SHAPE),
    (dict(D=32), SHAPE), (dict(first=-1), SHAPE), (dict(first=61), CAP), (dict(k_out=P(0x100008)), SHAPE), (dict(layer=layer(sink=70)), BUDGET),
    (dict(v_out=P(0x100400)), SHAPE), (dict(k_out=P(0x4000100)), SHAPE), (dict(v_out=P(0x8000f00), k_out=None), SHAPE), (dict(k_out=P(0x9100), v_out=None), SHAPE)])
def test_read_refusals(change, code):
    a = dict(layer=layer(), dt=1, B=2, T=4, Hkv=2, D=64, first=10, k_out=P(0x100000), v_out=P(0x200000), stream=None, opts=None)
    a.update(change)
    assert lib.sqa_q4_read(*a.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(q=None), NULL), (dict(layer=None), NULL), (dict(out=None), NULL), (dict(ws=None), NULL), (dict(layer=layer(K=None)), NULL), (dict(dt=2), DTYPE),
    (dict(B=0), SHAPE), (dict(T=0), SHAPE), (dict(Hq=3), SHAPE), (dict(D=80), SHAPE), (dict(new_pos=-1), SHAPE), (dict(q=P(0x100008)), SHAPE),
    (dict(ws=P(0x10)), SHAPE), (dict(ws_bytes=4096), CAP), (dict(layer=layer(cap=13, sink=10)), CAP), (dict(out=P(0x2000008)), SHAPE),
    (dict(out=P(0x100000)), SHAPE), (dict(lse=P(0x2000100)), SHAPE), (dict(lse=P(0x600002)), SHAPE), (dict(layer=layer(cap=3)), CAP),
    (dict(layer=layer(table=0x9000, bpu=3, nb=9)), SHAPE)])
def test_attention_refusals(change, code):
    a = dict(q=P(0x100000), dt=1, B=2, T=4, Hq=4, Hkv=2, D=64, new_pos=10, layer=layer(), out=P(0x2000000), lse=P(0x600000), ws=P(0x10000000),
             ws_bytes=1 << 30, stream=None, opts=None)
    a.update(change)
    assert lib.sqa_q4_attention(*a.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(table=None), NULL), (dict(tokens=None), NULL), (dict(held=None), NULL), (dict(free=None), NULL), (dict(count=None), NULL),
    (dict(table=P(0x1002)), SHAPE), (dict(status=P(0x6001)), SHAPE), (dict(B=0), SHAPE), (dict(B=8193), SHAPE), (dict(Hkv=0), SHAPE), (dict(per=0), SHAPE),
    (dict(n_blocks=0), SHAPE), (dict(per=1 << 30), SHAPE), (dict(capacity=0), CAP), (dict(capacity=65), CAP), (dict(per=1 << 27, capacity=(1 << 30) + 1, B=1, Hkv=1), CAP)])
def test_assign_refusals(change, code):
    a = dict(table=P(0x1000), B=3, Hkv=2, per=4, capacity=64, tokens=P(0x2000), held=P(0x3000), free=P(0x4000), count=P(0x5000), n_blocks=9, status=P(0x6000),
             stream=None)
    a.update(change)
    assert lib.sqa_block_assign(*a.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(map=None), NULL), (dict(map=P(0x2001)), SHAPE), (dict(table=P(0x1001)), SHAPE), (dict(B=0), SHAPE), (dict(T=0), SHAPE), (dict(new_pos=-1), SHAPE),
    (dict(capacity=0), CAP), (dict(capacity=65), CAP), (dict(sink=-1), BUDGET), (dict(sink=64), BUDGET), (dict(T=1 << 29, B=4), SHAPE)])
def test_map_refusals(change, code):
    a = dict(table=P(0x1000), B=3, T=2, Hkv=2, per=4, capacity=64, sink=4, new_pos=0, map=P(0x2000), stream=None, opts=None)
    a.update(change)
    assert lib.sqa_slot_map(*a.values()) == code


FORMS = [  # capacity, B, T, Hq, Hkv, new_pos, dtype -> rows, waves, row tiles, slot splits
    (100, 1, 1, 8, 2, 99, "bf16", (16, 8, 1, 1)), (30001, 1, 1, 64, 8, 30000, "bf16", (16, 8, 1, 32)), (571, 64, 1, 32, 32, 1500, "bf16", (16, 2, 1, 1)),
    (1001, 64, 1, 32, 8, 1000, "bf16", (16, 4, 1, 1)), (4095, 16, 5, 32, 8, 4090, "bf16", (32, 8, 1, 2)), (5000, 2, 1, 12, 4, 4990, "f32", (16, 8, 1, 19)),
    (4000, 1, 128, 32, 8, 3000, "bf16", (32, 8, 16, 2)), (4000, 1, 128, 32, 8, 2900, "bf16", (16, 8, 32, 1)),
    (4095, 16, 5, 32, 8, 4090, "f32", (16, 8, 2, 1)), (4095, 16, 4, 32, 8, 4090, "bf16", (16, 8, 1, 2)), (900, 16, 20, 32, 16, 2500, "bf16", (32, 4, 2, 1)),
    (510, 32, 9, 64, 32, 500, "bf16", (32, 2, 1, 1)), (600, 4, 520, 16, 8, 70, "bf16", (128, 4, 9, 1)), (8192, 4, 300, 64, 8, 7800, "bf16", (128, 4, 19, 1)),
    (8200, 1, 128, 64, 8, 8000, "bf16", (128, 4, 8, 7)), (8200, 1, 128, 32, 4, 8000, "bf16", (32, 8, 32, 2)),
    (1100, 64, 24, 32, 8, 1000, "bf16", (128, 4, 1, 1)), (1100, 64, 16, 32, 8, 1000, "bf16", (32, 2, 2, 1)), (1100, 64, 33, 32, 8, 1000, "bf16", (128, 4, 2, 1)),
    (300, 16, 129, 16, 16, 63, "bf16", (128, 4, 2, 1)), (300, 16, 129, 16, 16, 63, "f32", (16, 2, 9, 1)), (8200, 1, 128, 32, 4, 8000, "f32", (16, 8, 64, 1)), (1 << 30, 1, 1, 1, 1, 5, "bf16", (16, 8, 1, 1))]


@pytest.mark.parametrize("capacity,B,T,Hq,Hkv,new_pos,dtype,want", FORMS)
def test_plan(capacity, B, T, Hq, Hkv, new_pos, dtype, want):
    got = sqa.q4_plan(capacity, B, T, Hq, Hkv, 128, dtype, new_pos)
    assert (got["rows"], got["waves"], got["row_tiles"], got["slot_splits"]) == want and got["rounded_probs"] == (want[0] == 128)
    assert got == sqa.q4_plan(min(capacity, new_pos + T), B, T, Hq, Hkv, 128, dtype, ragged=True)         # (a ragged batch: by the room there is)


def test_plans_fit_their_workspace():
    # no more records than the workspace has rows for, of any length up to the one that it was made for, and no more than a wave's lanes
    for dtype in ("bf16", "f32"):
        for B, Hq, Hkv in ((1, 1, 1), (1, 8, 1), (1, 64, 8), (3, 12, 4), (40, 32, 32)):
            for T in (1, 2, 5, 15, 16, 17, 31, 64, 127, 128, 129, 500, 4000):
                for cap in (1, 300, 5000, 100000, 1 << 30):
                    p = sqa.q4_plan(cap, B, T, Hq, Hkv, 64, dtype, ragged=True)
                    records = B * Hkv * p["row_tiles"] * p["slot_splits"] * p["rows"]
                    room = lib.sqa_q4_workspace_bytes(layer(cap=cap), B, T, Hq, Hkv, 64) - 4096
                    assert p["slot_splits"] <= 64 and (p["slot_splits"] == 1 or (records * 17 * 16 <= room and B * Hkv * p["row_tiles"] <= 1024))


@pytest.mark.parametrize("change,code", [(dict(layer=None), NULL), (dict(info=None), NULL), (dict(dt=2), DTYPE), (dict(T=0), SHAPE), (dict(D=32), SHAPE),
                                         (dict(layer=layer(cap=0)), CAP)])
def test_plan_refusals(change, code):
    a = dict(layer=layer(), dt=1, B=2, T=4, Hq=4, Hkv=2, D=64, new_pos=10, opts=None, info=C.byref(sqa.Q4PlanInfo()))
    a.update(change)
    assert lib.sqa_q4_plan(*a.values()) == code


def test_one_workspace_serves_every_shorter_chunk():
    need = lambda *shape: lib.sqa_q4_workspace_bytes(layer(cap=5000), *shape)
    for B, Hq, Hkv, D in ((1, 8, 8, 128), (3, 24, 8, 64), (16, 64, 8, 128), (2, 5, 1, 128)):
        sizes = [need(B, T, Hq, Hkv, D) for T in (1, 2, 3, 7, 8, 16, 17, 33, 64, 65, 129, 1000)]
        assert sizes == sorted(sizes) and sizes[0] > 4096 and all(s % 256 == 0 for s in sizes)
    assert need(0, 1, 8, 8, 128) == 0 and need(1, 1, 8, 3, 128) == 0 and need(1, 1, 8, 8, 96) == 0 and lib.sqa_q4_workspace_bytes(None, 1, 1, 8, 8, 64) == 0


def test_binding_refuses_what_it_cannot_describe():
    x, c = torch.zeros(2, 3, 4, 64), sqa.Q4Caches([8], 2, 4, 64, "cpu")
    q, ws = torch.zeros(2, 4, 3, 64), torch.zeros(1 << 24, dtype=torch.uint8)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    on = sqa.rope_axes(i32(3, 2, 3), [8, 12, 12])
    how = sqa.head_prep(rope=torch.zeros(9, 64))
    for what, call in [("int32 tensor", lambda: sqa.rope_axes(torch.zeros(3, 2, 3), [8, 12, 12])), ("each of 1 to 4", lambda: sqa.rope_axes(i32(3, 2, 3), [8, 24])),
                       ("int32 tensor", lambda: sqa.rope_axes(i32(2, 3), [32])), ("each of 1 to 4", lambda: sqa.rope_axes(i32(5, 2, 3), [8, 8, 8, 4, 4])),
                       ("call's tokens", lambda: sqa.qk_norm_rope(x[:, :2], None, 0, how, axes=on)), ("another batch", lambda: sqa.q4_append(x[:1], x[:1], 0, c)),
                       ("one shape", lambda: sqa.q4_append(x, x[:, :2], 0, c)), ("contiguous", lambda: sqa.q4_append(x, x, 0, c, slot_map=i32(2, 3, 4))),
                       ("contiguous", lambda: sqa.q4_read(c, 0, 3, torch.float32, k_out=torch.zeros(2, 4, 2, 64))),
                       ("contiguous", lambda: sqa.q4_attention(q.transpose(1, 2), 0, c)), ("another batch", lambda: sqa.q4_attention(q[:1], 0, c)),
                       ("contiguous", lambda: sqa.q4_attention(q, 0, c, out=torch.zeros(2, 4, 3, 64), workspace=ws)),
                       ("contiguous int32", lambda: sqa.block_assign(i32(4, 4), torch.zeros(2), i32(2), i32(9), i32(1), 64)),
                       ("tokens and held", lambda: sqa.block_assign(i32(5, 4), i32(2), i32(2), i32(9), i32(1), 64)),
                       ("B and Hkv", lambda: sqa.slot_map(i32(4, 4), 64, 1)), ("which device", lambda: sqa.slot_map(None, 64, 1, B=2, Hkv=2)),
                       ("blocks_per_unit", lambda: sqa.slot_map(i32(5, 4), 64, 1, out=i32(2, 2, 1)))]:
        with pytest.raises(TypeError, match=what):
            call()
    with pytest.raises(IndexError):
        sqa.q4_append(x, x, 0, c, layer=1)
    # tensors of the host never reach a kernel
    for call in (lambda: sqa.q4_append(x, x, 0, c), lambda: sqa.q4_read(c, 0, 3, torch.float32), lambda: sqa.q4_attention(q, 0, c, workspace=ws),
                 lambda: sqa.qk_norm_rope(x, x, 0, how, axes=on), lambda: sqa.block_assign(i32(4, 4), i32(2), i32(2), i32(9), i32(1), 64),
                 lambda: sqa.slot_map(i32(4, 4), 64, 1, out=i32(2, 2, 1))):
        with pytest.raises(ValueError, match="current device"):
            call()


def test_numbers_that_ctypes_would_cut_off():
    one = torch.zeros(1, dtype=torch.int32)
    for bad in (1 << 32, (1 << 32) + 5, -(1 << 31) - 1):
        with pytest.raises(sqa.SqaError):
            sqa.q4_plan(bad, 1, 1, 1, 1, 64, "bf16")
        with pytest.raises(sqa.SqaError):
            sqa.Q4Caches([16], 1, 1, 64, "cpu", n_sink=bad)
        with pytest.raises(sqa.SqaError):
            sqa.rope_axes(one.view(1, 1, 1), [bad])
        with pytest.raises((sqa.SqaError, ValueError)):              # (without a GPU the tensors' device is refused first)
            sqa.slot_map(one.view(1, 1), bad, 1, B=1, Hkv=1)
        with pytest.raises((sqa.SqaError, ValueError)):
            sqa.block_assign(one.view(1, 1), one, one, one, one, bad)
