"""The compiled kernels whose DMA takes its base from a vector instruction: gfx950 wants five wait states between a vector
instruction that writes a scalar register and a memory instruction that reads it, and the compiler does not see into the
inline assembly that holds the memory instruction."""
import os
import re
import subprocess

import pytest

from paper_2609_31551_amd import build


def reads_too_early(lines):
    """(instruction, wait states) of memory instructions that read a scalar register less than five wait states after a
    vector instruction wrote it."""
    found, recent = [], []
    for line in lines:
        op = line.split(";")[0].strip()
        if not op or op.startswith(".") or op.endswith(":"):
            continue
        name, _, rest = op.partition(" ") if " " in op else op.partition("\t")
        scalars = set()
        for a, b in re.findall(r"\bs\[(\d+):(\d+)\]", rest):
            scalars |= set(range(int(a), int(b) + 1))
        scalars |= {int(a) for a in re.findall(r"\bs(\d+)\b", rest)}
        if name.startswith(("global_", "buffer_", "flat_", "scratch_")):
            waited = 0
            for states, written in reversed(recent):
                if written & scalars and waited < 5:
                    found.append((op, waited))
                waited += states
        written = set()
        if name.startswith(("v_readlane", "v_readfirstlane", "v_cmp")):
            first = rest.split(",")[0]
            m = re.match(r"\s*s\[(\d+):(\d+)\]", first) or re.match(r"\s*s(\d+)()", first)
            if m:
                written = set(range(int(m.group(1)), int(m.group(2) or m.group(1)) + 1))
        recent = (recent + [(int(rest, 0) + 1 if name == "s_nop" else 1, written)])[-8:]
    return found


def test_the_check_finds_what_it_looks_for():
    early = ["v_readlane_b32 s5, v1, 0", "s_mov_b32 m0, s9", "s_nop 0", "global_load_lds_dwordx4 v2, s[4:5]"]
    assert reads_too_early(early) == [(early[3], 2)]
    assert not reads_too_early(early[:2] + ["s_nop 3"] + early[3:])
    assert not reads_too_early(["v_readlane_b32 s6, v1, 0"] + early[1:])


@pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="needs hipcc")
@pytest.mark.parametrize("name", ["kv16_attention.hip", "prompt_attention.hip"])
def test_bases_from_vector_instructions_are_waited_for(name, tmp_path):
    out = str(tmp_path / "kernels.s")
    cmd = [build.HIPCC] + build.FLAGS + build.FILE_FLAGS.get(name, []) + ["--cuda-device-only", "-S", "-x", "hip",
                                                                            os.path.join(build.CSRC, name), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    with open(out) as f:
        lines = f.read().split("\n")
    assert sum("global_load_lds_dwordx4" in l for l in lines) > 100
    assert reads_too_early(lines) == []
