"""Registers of the kernels for a cache in 4 bits, rotary positions on several axes and block tables as the compiler reports them: none
spills, and each has room for the waves that it is made for."""
import json
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PATH = os.path.join(ROOT, "paper_2404_04793_amd", "_build", "kernel_resources.json")


@pytest.mark.parametrize("name,forms,waves", [
    ("axis_rows_kernel", 12, 4), ("q4_rows_kernel", 16, 6), ("q4_read_kernel", 4, 8), ("q4_attention_kernel", 18, 2), ("q4_attention_wide_kernel", 2, 2),
    ("block_assign_kernel", 3, 8), ("slot_map_kernel", 1, 8)])
def test_kernels_keep_their_registers(name, forms, waves):
    if not os.path.exists(PATH):
        pytest.skip("the library has not been built in this tree (python -m paper_2404_04793_amd.build)")
    with open(PATH) as fh:
        hits = {k: v for k, v in json.load(fh).items() if name in k}
    assert len(hits) == forms, sorted(hits)
    for k, v in hits.items():
        assert v["ScratchSize"] == 0 and v["VGPRs Spill"] == 0 and v["Occupancy"] >= waves, (k, v)


def test_single_tokens_have_two_workgroups_per_cu():
    """16 rows in bf16, 8 waves: four waves per SIMD."""
    if not os.path.exists(PATH):
        pytest.skip("the library has not been built in this tree (python -m paper_2404_04793_amd.build)")
    with open(PATH) as fh:
        hits = {k: v["Occupancy"] for k, v in json.load(fh).items() if "q4_attention_kernelINS_6bf16" in k and k.split("EEEv")[0].endswith("Li1")}
    assert len(hits) == 6 and all(v >= 4 for v in hits.values()), hits
