"""An assignment under a condition of lanes that the compiler leaves out: `if (!(a && (b || c))) s[0] = -INFINITY` for the first register of a
matrix product's result became -inf for the lanes where !a, and for those where only !(b || c) holds a region without an instruction
(exec saved and masked, then restored at once): these lanes kept a logit that they may not see.  Seen in the 4-bit attention while it was
being written, in no kernel that was committed; so no kernel may hold such a region."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2404_04793_amd", "libsqa.so")
OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


def empty_regions(text):
    """(kernel, line) of each mask that is taken back before anything was done under it."""
    hits, kernel, saved = [], None, None
    for n, line in enumerate(text.splitlines()):
        name = re.match(r"[0-9a-f]+ <(\S+)>:", line)
        kernel = name.group(1) if name else kernel
        code = line.split("//")[0].strip()
        if not code or code.startswith("s_cbranch_execz") or code.endswith(":"):
            continue
        if saved and re.match(r"s_or_b64 exec, exec, " + re.escape(saved) + "$", code):
            hits.append((kernel, n))
        m = re.match(r"s_and_saveexec_b64 (s\[\d+:\d+\]),", code)
        saved = m.group(1) if m else None
    return hits


def test_what_the_scan_finds():
    kept = ["0000 <kernel>:", "s_and_saveexec_b64 s[0:1], vcc // 00", "s_cbranch_execz 3", "v_mov_b32_e32 v30, s82", "s_or_b64 exec, exec, s[0:1]"]
    assert empty_regions("\n".join(kept)) == []
    assert empty_regions("\n".join(kept[:3] + kept[4:])) == [("kernel", 3)]


def test_no_kernel_has_one(tmp_path):
    if not (os.path.exists(LIB) and os.path.exists(OBJDUMP)):
        pytest.skip("the library has not been built in this tree (python -m paper_2404_04793_amd.build)")
    copy = tmp_path / "libsqa.so"
    copy.write_bytes(open(LIB, "rb").read())
    subprocess.run([OBJDUMP, "--offloading", str(copy)], cwd=tmp_path, check=True, capture_output=True)
    objects = sorted(tmp_path.glob("*gfx950"))
    assert len(objects) == len([f for f in os.listdir(os.path.join(ROOT, "paper_2404_04793_amd", "csrc")) if f.endswith(".hip")])
    for code in objects:
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(code)], check=True, capture_output=True, text=True).stdout
        assert "s_endpgm" in text and "s_and_saveexec_b64" in text
        assert empty_regions(text) == [], code.name
