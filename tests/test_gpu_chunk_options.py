"""Host arrays in the options of the chunk calls never reach a kernel (test_chunk_options.py has the rest)."""
import pytest
import torch

from test_gpu_chunk import DEV, sqa  # noqa: F401

pytestmark = pytest.mark.gpu


def test_host_arrays_are_refused(sqa):  # noqa: F811
    x, q = torch.zeros(2, 3, 4, 64, device=DEV), torch.zeros(2, 4, 3, 64, device=DEV)
    c = sqa.LayerCaches([8], [8], 2, 4, 64, torch.float32, DEV, True)
    lse, there = torch.zeros(2, 4, 3, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    for field in ("prompt_len", "new_pos_seq", "budget_seq", "status"):
        other = "new_pos_seq" if field == "prompt_len" else "prompt_len"
        opts = sqa.batch_opts(**{field: torch.zeros(2, dtype=torch.int32), other: there})
        for call in (lambda: sqa.qk_norm_rope(x, x, 0, opts=opts), lambda: sqa.chunk_append(x, x, 0, c, opts=opts),
                     lambda: sqa.chunk_attention(q, 0, c, opts=opts), lambda: sqa.chunk_scores(q, lse, 0, c, opts=opts)):
            with pytest.raises(ValueError, match="current device"):
                call()
    torch.cuda.synchronize()
    assert int(c.lens[0].sum()) == 0
