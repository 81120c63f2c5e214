"""Registers of the kernels for chunks of tokens as the compiler reports them: none spills, and those that are made for two workgroups
per CU (two waves per SIMD) have room for them."""
import json
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PATH = os.path.join(ROOT, "paper_2404_04793_amd", "_build", "kernel_resources.json")


@pytest.mark.parametrize("name,forms,waves", [("chunk_rows_kernel", 8, 6), ("chunk_attention_kernel", 9, 1), ("chunk_attention_wide_kernel", 2, 2),
                                              ("chunk_scores_kernel", 4, 2)])
def test_chunk_kernels_keep_their_registers(name, forms, waves):
    if not os.path.exists(PATH):
        pytest.skip("the library has not been built in this tree (python -m paper_2404_04793_amd.build)")
    with open(PATH) as fh:
        hits = {k: v for k, v in json.load(fh).items() if name in k}
    assert len(hits) == forms, sorted(hits)
    for k, v in hits.items():
        assert v["ScratchSize"] == 0 and v["VGPRs Spill"] == 0 and v["Occupancy"] >= waves, (k, v)


def test_forms_made_for_two_workgroups_per_cu_have_room():
    """Every attention form runs two waves per SIMD but fp32 heads of 128 in 64 rows, whose tiles fill the LDS; scores of heads of 64 in bf16 run three."""
    if not os.path.exists(PATH):
        pytest.skip("the library has not been built in this tree (python -m paper_2404_04793_amd.build)")
    with open(PATH) as fh:
        res = {k: v["Occupancy"] for k, v in json.load(fh).items()}
    for k, waves in res.items():
        if "chunk_attention_kernel" in k:
            assert waves >= (1 if "IfLi128ELi2ELi64E" in k else 2), (k, waves)
        if "chunk_scores_kernel" in k:
            assert waves >= (3 if "bf16_tELi64E" in k else 2), (k, waves)
    assert any("chunk_attention_kernelIfLi128ELi2ELi64E" in k for k in res) and any("chunk_scores_kernelINS_6bf16_tELi64E" in k for k in res)
