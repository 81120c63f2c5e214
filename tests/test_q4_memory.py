"""Memory that calls on a cache in 4 bits write may not be memory that they still read, or write something else to: refused on the host."""
import ctypes as C

import pytest

import test_q4_host as host
from paper_2404_04793_amd import binding as sqa

P, SHAPE = C.c_void_p, 2
ROWS = 2 * 2 * 64                                    # of the cache: 2 sequences, 2 heads, 64 slots; rows of 32 bytes of codes and 2 of powers
NEED = sqa._lib.sqa_q4_workspace_bytes(host.layer(), 2, 4, 4, 2, 64)
TABLE = dict(table=0x20000, bpu=4, nb=16)            # (16 blocks: as many rows)


@pytest.mark.parametrize("change", [
    dict(out=P(0x4000000)), dict(out=P(0x4000000 + ROWS * 32 - 16)), dict(out=P(0x8000100)), dict(out=P(0x9000)), dict(out=P(0xa000 + ROWS * 2 - 16)),
    dict(lse=P(0x4000000)), dict(lse=P(0x8000000 + ROWS * 32 - 4)), dict(lse=P(0x91fc)), dict(lse=P(0xa000)), dict(ws=P(0x4000000)), dict(ws=P(0x8001000)),
    dict(ws=P(0x100000)), dict(ws=P(0x2000000)), dict(ws=P(0x600000)), dict(out=P(0x10000000 + NEED - 16)), dict(lse=P(0x10000000 + NEED - 4)),
    dict(q=P(0x10000000 + NEED - 16)), dict(layer=host.layer(**TABLE), out=P(0x20000)), dict(layer=host.layer(**TABLE), lse=P(0x20000 + 60)),
    dict(layer=host.layer(**TABLE), out=P(0x4000000 + 16 * 16 * 32 - 16))])
def test_attention(change):
    a = dict(q=P(0x100000), dt=1, B=2, T=4, Hq=4, Hkv=2, D=64, new_pos=10, layer=host.layer(), out=P(0x2000000), lse=P(0x600000), ws=P(0x10000000),
             ws_bytes=1 << 30, stream=None, opts=None)
    a.update(change)
    assert sqa._lib.sqa_q4_attention(*a.values()) == SHAPE


@pytest.mark.parametrize("change", [
    dict(q_out=P(0x4000000)), dict(q_out=P(0x8000000 + ROWS * 32 - 16)), dict(q_out=P(0x9000)), dict(q_out=P(0xa000)), dict(layer=host.layer(V=0x4000000)),
    dict(layer=host.layer(V=0x4000000 + ROWS * 32 - 16)), dict(layer=host.layer(Vs=0x9000)), dict(layer=host.layer(Vs=0x9000 + ROWS * 2 - 4)),
    dict(layer=host.layer(Ks=0x4000000)), dict(layer=host.layer(Vs=0x8000000)), dict(layer=host.layer(Vs=0x4000010)),
    dict(layer=host.layer(**TABLE), q_out=P(0x20000)), dict(slot_map=P(0x4000000)), dict(slot_map=P(0xa000)), dict(slot_map=P(0x2000010))])
def test_append(change):
    a = dict(q=host.rows(), k=host.rows(0x200000), v=host.rows(0x300000), dt=1, B=2, T=4, Hq=4, Hkv=2, D=64, prep=host.prep(), new_pos=10, q_out=P(0x2000000),
             layer=host.layer(), stream=None, opts=None, axes=None, slot_map=None)
    a.update(change)
    assert sqa._lib.sqa_q4_append(*a.values()) == SHAPE


@pytest.mark.parametrize("change", [dict(k_out=P(0x20000)), dict(v_out=P(0x20000 + 48)), dict(k_out=P(0x4000000 + 16 * 16 * 32 - 16))])
def test_read(change):
    a = dict(layer=host.layer(**TABLE), dt=1, B=2, T=4, Hkv=2, D=64, first=10, k_out=P(0x100000), v_out=P(0x200000), stream=None, opts=None)
    a.update(change)
    assert sqa._lib.sqa_q4_read(*a.values()) == SHAPE


@pytest.mark.parametrize("B,Hkv,per", [(1, 1, 2 ** 31 - 1), (1, 1, 2 ** 31 - 65536), (2, 4, 2 ** 28 - 8191)])
def test_tables_whose_entries_a_thread_could_not_count(B, Hkv, per):
    """Threads step through what changes hands by 65536 at a time: past the last entry the number has to stay within 32 bits."""
    at = [P(x << 34) for x in range(1, 7)]
    assert sqa._lib.sqa_block_assign(at[0], B, Hkv, per, 64, at[1], at[2], at[3], at[4], 2 ** 31 - 1, at[5], None) == SHAPE
