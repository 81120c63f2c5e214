"""Memory that the chunk calls write may not be memory that they still read, or write something else to: refused on the host."""
import ctypes as C

import pytest

import test_chunk_host as host
from paper_2404_04793_amd import binding as sqa

P, SHAPE = C.c_void_p, 2
POOL = 2 * 2 * 64 * 64 * 2                           # bytes of K: 2 sequences, 2 heads, 64 slots of 64 bf16
BLOCKED = dict(table=0x20000, bpu=4, nb=20)
LAYER = lambda **kw: C.byref(host.layer(**kw))
NEED = sqa._lib.sqa_chunk_workspace_bytes(LAYER(), 2, 4, 4, 2, 64)
PLACES = [0x4000000, 0x4000000 + POOL - 16, 0x8000000, 0x8000000 + POOL - 16, 0x3000, 0x4000, 0x43f0, 0x5000, 0x5030]         # K, V, scores, positions, states


@pytest.mark.parametrize("change", [dict(out=P(x)) for x in PLACES] + [dict(lse=P(x)) for x in PLACES] + [
    dict(ws=P(0x4000000)), dict(ws=P(0x8000000)), dict(ws=P(0x100000)), dict(ws=P(0x600000)), dict(ws=P(0x2000000)), dict(out=P(0x10000000 + NEED - 16)),
    dict(lse=P(0x10000000 + NEED - 4)), dict(q=P(0x10000000 + NEED - 16)), dict(layer=LAYER(**BLOCKED), out=P(0x20030)),
    dict(layer=LAYER(**BLOCKED), out=P(0x4000000 + 20 * 16 * 128 - 16)), dict(layer=LAYER(offset=0x30000), out=P(0x30010)), dict(layer=LAYER(offset=0x30000), lse=P(0x5000))])
def test_attention(change):
    a = dict(q=P(0x100000), dt=1, B=2, T=4, Hq=4, Hkv=2, D=64, new_pos=10, layer=LAYER(), out=P(0x2000000), lse=P(0x600000), ws=P(0x10000000), ws_bytes=1 << 30,
             stream=None, opts=None)
    a.update(change)
    assert sqa._lib.sqa_chunk_attention(*a.values()) == SHAPE


@pytest.mark.parametrize("change", [dict(ws=P(0x4000000)), dict(ws=P(0x8000000)), dict(ws=P(0x100000)), dict(ws=P(0x600000)), dict(lse=P(0x3000)), dict(q=P(0x33f0)),
                                    dict(lse=P(0x10000000 + NEED - 4)), dict(q=P(0x10000000 + NEED - 16))])
def test_scores(change):
    a = dict(q=P(0x100000), lse=P(0x600000), dt=1, B=2, T=4, Hq=4, Hkv=2, D=64, new_pos=10, layer=LAYER(), ws=P(0x10000000), ws_bytes=1 << 30, stream=None,
             opts=None)
    a.update(change)
    assert sqa._lib.sqa_chunk_scores(*a.values()) == SHAPE


@pytest.mark.parametrize("change", [dict(q_out=P(x)) for x in PLACES] + [dict(layer=LAYER(K=0x8000000)), dict(layer=LAYER(K=0x8000000 - POOL + 16)),
                                                                       dict(layer=LAYER(**BLOCKED), q_out=P(0x20000))])
def test_append(change):
    a = dict(q=host.rows(), k=host.rows(0x200000), v=host.rows(0x300000), dt=1, B=2, T=4, Hq=4, Hkv=2, D=64, prep=host.prep(), new_pos=10, q_out=P(0x2000000),
             layer=LAYER(), stream=None, opts=None)
    a.update(change)
    assert sqa._lib.sqa_chunk_append(*a.values()) == SHAPE
