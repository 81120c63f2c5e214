"""Calls on a cache in 4 bits as include/sqa.h allows them and a binding seldom makes them: outputs that are not wanted, positions at the end of 32 bits,
batches in which nobody takes part, one workspace for calls of every form."""
import ctypes as C

import pytest
import torch

import chunk_reference as R
import q4_reference as Q
from test_gpu_q4_attention import filled, generator, ints, sqa  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FORMS = [  # dtype, D, B, T, before, Hq, Hkv -> rows, waves, slot splits
    ("bf16", 128, 1, 1, 100, 8, 2, (16, 8, 1)), ("bf16", 64, 1, 1, 900, 8, 2, (16, 8, 3)), ("bf16", 128, 1, 1, 9000, 8, 2, (16, 8, 35)),
    ("f32", 64, 1, 1, 5000, 6, 2, (16, 8, 19)), ("f32", 128, 8, 2, 300, 64, 64, (16, 4, 1)), ("bf16", 128, 8, 9, 3200, 32, 16, (32, 8, 2)),
    ("bf16", 64, 1, 33, 13000, 16, 16, (32, 8, 8)), ("bf16", 128, 8, 300, 0, 32, 8, (128, 4, 1)), ("bf16", 64, 2, 257, 7000, 16, 8, (128, 4, 6))]


def case(sqa, form, blocked=False, room=3):
    dtype, D, B, T, before, Hq, Hkv, want = form
    gen = generator(T + before)
    c = filled(sqa, B, Hkv, D, before + T + room, 0, blocked, gen)
    plan = sqa.q4_plan(before + T + room, B, T, Hq, Hkv, D, dtype, before)
    assert (plan["rows"], plan["waves"], plan["slot_splits"]) == want
    return c, torch.randn(B, Hq, T, D, generator=gen, device=DEV).to(R.DT[dtype]), before


def test_outputs_that_are_not_wanted(sqa):  # noqa: F811
    """Rows without their normalisers: the same rows, of every form; refused units too."""
    for form in FORMS:
        for broken in (False, True):
            c, q, before = case(sqa, form, blocked=broken)
            if broken:
                c.block_table[0][1, 0] = -1
            B, Hq, T, D = q.shape
            ws, status = sqa.q4_workspace(c, Hq, T), ints([0])
            want, _ = sqa.q4_attention(q, before, c, workspace=ws, opts=sqa.batch_opts(status=status))
            assert int(status) == (2 if broken else 0)
            out = torch.full_like(want, 7.0)
            assert sqa._lib.sqa_q4_attention(q.data_ptr(), sqa._DT[q.dtype], B, T, Hq, c.Hkv, D, before, C.addressof(c.table), out.data_ptr(), None, ws.data_ptr(),
                                             ws.nbytes, torch.cuda.current_stream().cuda_stream, None) == 0
            assert torch.equal(out, want), form


def test_reading_one_of_the_two(sqa):  # noqa: F811
    for dtype, D in (("bf16", 128), ("f32", 64)):
        c = filled(sqa, 2, 3, D, 50, 0, True, generator(3))
        both = sqa.q4_read(c, 7, 20, R.DT[dtype])
        for which in (0, 1):
            out = torch.full_like(both[0], 7.0)
            to = [out.data_ptr() if i == which else None for i in (0, 1)]
            assert sqa._lib.sqa_q4_read(C.addressof(c.table), sqa._DT[R.DT[dtype]], 2, 20, 3, D, 7, *to, torch.cuda.current_stream().cuda_stream, None) == 0
            assert torch.equal(out, both[which])


def test_one_workspace_for_every_form(sqa):  # noqa: F811
    """Forms in turn on one workspace, as large as the largest needs, give what each gives with its own."""
    cases = [case(sqa, f) for f in FORMS]
    ws = max((sqa.q4_workspace(c, q.shape[1], q.shape[2]) for c, q, _ in cases), key=lambda w: w.nbytes)
    own = [sqa.q4_attention(q, before, c) for c, q, before in cases]
    for _ in range(2):
        for (c, q, before), want in zip(cases, own):
            assert R.same(want, sqa.q4_attention(q, before, c, workspace=ws))


def test_a_batch_in_which_nobody_takes_part(sqa):  # noqa: F811
    for form in FORMS:
        c, q, _ = case(sqa, form)
        B, Hq, T, D = q.shape
        status = ints([0])
        keep = [x[0].clone() for x in (c.K, c.V, c.K_scale, c.V_scale)]
        for n, first in ((0, 5), (T, -1)):
            opts = sqa.batch_opts(prompt_len=ints([n] * B), new_pos_seq=ints([first] * B), status=status)
            out, lse, q_out = torch.full((B, T, Hq, D), 7.0, dtype=q.dtype, device=DEV), torch.full((B, Hq, T), 7.0, device=DEV), torch.full_like(q, 7.0)
            sqa.q4_attention(q, 0, c, out=out, lse=lse, opts=opts)
            x = torch.randn(B, T, Hq + 2 * c.Hkv, D, device=DEV).to(q.dtype)
            sqa.q4_append(x[:, :, Hq:Hq + c.Hkv], x[:, :, Hq + c.Hkv:], 0, c, q=x[:, :, :Hq], q_out=q_out, opts=opts)
            rows = sqa.slot_map(None, c.capacities[0], T, out=torch.zeros(B, c.Hkv, T, dtype=torch.int32, device=DEV), opts=opts)
            assert all(bool((y == 7).all()) for y in (out, lse, q_out)) and bool((rows == -1).all()) and int(status) == 0
            assert all(torch.equal(a, b[0]) for a, b in zip(keep, (c.K, c.V, c.K_scale, c.V_scale)))


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_positions_at_the_end_of_32_bits(sqa, dtype, D):  # noqa: F811
    """The last position that a chunk may end at is taken; beyond it the sequence is left out and reported, the others not."""
    dt, gen, cap, sink, T, Hkv, Hq = R.DT[dtype], generator(5), 50, 4, 3, 2, 4
    last = 2 ** 31 - 1
    first = [last - T, last - T + 1, last, 20]       # (positions up to 2^31 - 2; one and three too many; an ordinary one)
    good = [0, 3]
    B = len(first)
    c = filled(sqa, B, Hkv, D, cap, sink, False, gen)
    keep = [x[0].clone() for x in (c.K, c.V, c.K_scale, c.V_scale)]
    x = torch.randn(B, T, Hq + 2 * Hkv, D, generator=gen, device=DEV).to(dt)
    status = ints([0])
    opts = sqa.batch_opts(new_pos_seq=ints(first), status=status)
    q = sqa.q4_append(x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], 0, c, q=x[:, :, :Hq], opts=opts)
    assert int(status) == 2 and torch.equal(q, x[:, :, :Hq].transpose(1, 2))
    for b in range(B):
        slots = [Q.slot_of(p, cap, sink) for p in range(first[b], first[b] + T)] if b in good else []
        others = torch.ones(cap, dtype=torch.bool, device=DEV)
        others[slots] = False
        for h in range(Hkv):
            assert torch.equal(Q.codes(c.K[0][b, h, slots]), Q.pack(x[b, :len(slots), Hq + h])[1])
            assert all(torch.equal(a[b, h, others], y[0][b, h, others]) for a, y in zip(keep, (c.K, c.V, c.K_scale, c.V_scale)))
    status.zero_()
    rows = sqa.slot_map(None, cap, T, n_sink=sink, out=torch.zeros(B, Hkv, T, dtype=torch.int32, device=DEV), opts=opts)
    assert int(status) == 2 and bool((rows[[1, 2]] == -1).all())
    assert rows[0, 0].tolist() == [Q.slot_of(p, cap, sink) for p in range(first[0], first[0] + T)]
    status.zero_()
    out, lse = sqa.q4_attention(q, 0, c, opts=opts)
    assert int(status) == 2 and not bool(out[[1, 2]].any()) and bool((lse[[1, 2]] == -float("inf")).all()) and bool(lse[good].isfinite().all())
    # the far sequence sees what one with the same slots sees
    ring = cap - sink
    near = sink + ring + (first[0] - sink) % ring
    small = sqa.q4_attention(q[:1].contiguous(), near, one(sqa, c, D, Hkv, cap, sink))
    assert torch.equal(small[0], out[:1]) and torch.equal(small[1], lse[:1])


def one(sqa, c, D, Hkv, cap, sink):  # noqa: F811
    """The first sequence's cache alone."""
    x = sqa.Q4Caches([cap], 1, Hkv, D, DEV, n_sink=sink)
    for a, b in ((x.K, c.K), (x.V, c.V), (x.K_scale, c.K_scale), (x.V_scale, c.V_scale)):
        a[0].copy_(b[0][:1])
    return x
