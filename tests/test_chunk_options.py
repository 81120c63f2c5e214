"""Per-sequence arrays of the chunk calls: on the call's device, an entry for each sequence.  (Without a GPU: arrays that are too short are refused before
anything else is, and what looks at devices is asked itself; tests/test_gpu_chunk_options.py makes the calls.)"""
import pytest
import torch

from paper_2404_04793_amd import binding as sqa


def ints(n):
    return torch.zeros(n, dtype=torch.int32)


def calls(opts, B=2, T=3):
    x, q = torch.zeros(B, T, 4, 64), torch.zeros(B, 4, T, 64)
    c = sqa.LayerCaches([8], [8], B, 4, 64, torch.float32, "cpu", True)
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    return [lambda: sqa.qk_norm_rope(x, x, 0, opts=opts), lambda: sqa.chunk_append(x, x, 0, c, opts=opts),
            lambda: sqa.chunk_attention(q, 0, c, workspace=ws, opts=opts), lambda: sqa.chunk_scores(q, torch.zeros(B, 4, T), 0, c, workspace=ws, opts=opts)]


@pytest.mark.parametrize("field", ["prompt_len", "new_pos_seq", "budget_seq"])
@pytest.mark.parametrize("n", [0, 1])
def test_arrays_shorter_than_the_batch(field, n):
    for call in calls(sqa.batch_opts(**{field: ints(n)})):
        with pytest.raises(TypeError, match="each sequence"):
            call()


def test_arrays_of_another_device():
    for field in ("prompt_len", "new_pos_seq", "budget_seq", "status"):
        with pytest.raises(ValueError, match="current device"):
            sqa._opts_at(sqa.batch_opts(**{field: ints(2)}), 2, 0)
    assert sqa._opts_at(None, 2, 0) is None
    opts = sqa.batch_opts()
    assert sqa._opts_at(opts, 2, 0) == sqa.C.addressof(opts)
    opts = sqa.batch_opts(prompt_len=ints(2), budget_seq=torch.zeros(3, 2, dtype=torch.int32), status=ints(1))
    assert sqa._opts_at(opts, 2, -1) == sqa.C.addressof(opts)


def test_positions_beyond_32_bits(monkeypatch):
    """Refused, not cut off to another position.  (Before the library is called: its symbols are replaced.)"""
    class Library:
        def __getattr__(self, name):
            if name == "sqa_status_str":
                return lib.sqa_status_str
            return lambda *args: 0 if name != "sqa_chunk_workspace_bytes" else 1 << 20
    lib = sqa._lib
    monkeypatch.setattr(sqa, "_lib", Library())
    monkeypatch.setattr(sqa, "_check_device", lambda devices: None)
    monkeypatch.setattr(sqa, "_stream", lambda: None)
    for new_pos in (1 << 31, 1 << 32, (1 << 32) + 5, -(1 << 31) - 1):
        for call in (lambda c, x, q, ws: sqa.qk_norm_rope(x, x, new_pos), lambda c, x, q, ws: sqa.chunk_append(x, x, new_pos, c),
                     lambda c, x, q, ws: sqa.chunk_attention(q, new_pos, c, workspace=ws),
                     lambda c, x, q, ws: sqa.chunk_scores(q, torch.zeros(2, 4, 3), new_pos, c, workspace=ws),
                     lambda c, x, q, ws: sqa.chunk_plan(8, 2, 3, 4, 4, 64, "f32", new_pos)):
            with pytest.raises(sqa.SqaError) as e:
                call(sqa.LayerCaches([8], [8], 2, 4, 64, torch.float32, "cpu", True), torch.zeros(2, 3, 4, 64), torch.zeros(2, 4, 3, 64),
                     torch.zeros(1 << 20, dtype=torch.uint8))
            assert e.value.code == 2
