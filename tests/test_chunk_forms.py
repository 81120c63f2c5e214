"""Which forms of the chunk kernels the shapes of the tests reach (sqa_chunk_plan: host arithmetic), so that a change of the rules that choose a form
cannot leave one without a comparison; and what that call refuses."""
import ctypes as C

import pytest

import chunk_forms as F
from paper_2404_04793_amd import binding as sqa


def plans(cases, dtype, D):
    return [sqa.chunk_plan(F.capacity(c), c[0], c[1], c[3], c[4], D, dtype, c[2][0], c[5] is not None) for c in cases]


@pytest.mark.parametrize("dtype,D", F.TYPES)
def test_every_form_of_attention_is_reached(dtype, D):
    got = plans(F.ATTENTION, dtype, D)
    wide = [p for p in got if p["rows"] == 128]
    assert {p["slot_splits"] for p in wide} >= {1, 2, 3, 6} and {p["units_in_turn"] for p in wide} == {1, 2, 4, 8}
    assert any(p["units_in_turn"] == 1 and p["slot_splits"] == 1 and p["row_tiles"] >= 8 for p in wide)
    assert all(p["rounded_probs"] == (dtype == "bf16" and p["rows"] == 128) for p in got)
    middle = [p for p in got if p["rows"] == 64]
    assert any(p["slot_splits"] == 1 for p in middle) and any(p["slot_splits"] > 1 for p in middle) and any(p["units_in_turn"] > 1 for p in middle)
    ragged = [p for p, c in zip(got, F.ATTENTION) if c[5] is not None]
    assert {128, 64} <= {p["rows"] for p in ragged}
    few = [p for p in got if p["rows"] == 32]                      # (fp32 heads of 128 have no form for 32 rows)
    assert (not few) if (dtype, D) == ("f32", 128) else any(p["slot_splits"] > 1 for p in few)


@pytest.mark.parametrize("dtype,D", F.TYPES)
def test_score_workgroups_go_through_several_row_tiles(dtype, D):
    per = []
    for p, c in zip(plans(F.SCORES, dtype, D), F.SCORES):
        assert p["score_slots"] == (256 if (dtype, D) == ("bf16", 128) else 128)
        tiles = -(-c[1] * (c[3] // c[4]) // 64)                    # of 64 rows, at the unit's first slots
        per.append((p["score_row_splits"], tiles / p["score_row_splits"]))
    assert any(s == 1 and n >= 30 for s, n in per) and any(s > 1 and n >= 4 for s, n in per) and any(s == 1 and n == 5 for s, n in per)


def test_chunk_plan_of_known_calls():
    p = sqa.chunk_plan(8192, 1, 512, 64, 8, 128, "bf16", 7680)
    assert p == dict(rows=128, row_tiles=32, slot_splits=2, units_in_turn=1, rounded_probs=1, score_slots=256, score_slot_tiles=32, score_row_splits=2)
    p = sqa.chunk_plan(4095, 16, 5, 32, 8, 128, "bf16", 0, ragged=True)
    assert (p["rows"], p["row_tiles"], p["slot_splits"], p["rounded_probs"]) == (32, 1, 4, 0)
    assert sqa.chunk_plan(2048, 8, 2048, 32, 32, 128, "bf16")["units_in_turn"] == 8


def test_chunk_plan_refusals():
    info, layer = sqa.ChunkPlanInfo(), sqa.LayerCacheStruct(capacity=100)
    good = dict(layer=C.byref(layer), dt=1, B=1, T=4, Hq=8, Hkv=2, D=64, new_pos=10, opts=None, info=C.byref(info))
    assert sqa._lib.sqa_chunk_plan(*good.values()) == 0
    for change, code in ((dict(layer=None), 1), (dict(info=None), 1), (dict(dt=2), 3), (dict(B=0), 2), (dict(Hq=7), 2), (dict(D=96), 2), (dict(new_pos=-1), 2),
                         (dict(new_pos=97), 6), (dict(layer=C.byref(sqa.LayerCacheStruct(capacity=0))), 6)):
        assert sqa._lib.sqa_chunk_plan(*{**good, **change}.values()) == code, change
