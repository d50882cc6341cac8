"""The compiled kernels' inline-assembly DMA: gfx950 wants five wait states between a vector instruction that writes a scalar
register (a lane read back, also one that the compiler itself makes to restore a register that it had put aside) and a
memory instruction whose address is in it.  The compiler keeps that for its own instructions and does not see into inline
assembly.  Here every way that leads to such an instruction is followed, over branches too, in every source that has one."""
import os
import re
import subprocess

import pytest

from paper_2609_31551_amd import build

WANTED = 5


def scalars(text):
    found = {int(a) for a in re.findall(r"\bs(\d+)\b", text)}
    for a, b in re.findall(r"\bs\[(\d+):(\d+)\]", text):
        found |= set(range(int(a), int(b) + 1))
    return found


def read_too_early(lines):
    """(memory instruction, vector instruction, wait states between them) wherever they are too few."""
    code, labels = [], {}
    for line in lines:
        text = line.split(";")[0].strip().replace("\t", " ")
        label = re.match(r"([\w.$]+):", text)
        if label:
            labels[label.group(1)] = len(code)
        elif text and not text.startswith("."):
            name, _, rest = text.partition(" ")
            code.append((name, rest.strip()))
    before = [[] for _ in code]
    for i, (name, rest) in enumerate(code):
        if i + 1 < len(code) and name not in ("s_branch", "s_endpgm", "s_setpc_b64"):
            before[i + 1].append(i)
        if name.startswith(("s_branch", "s_cbranch")) and labels.get(rest, len(code)) < len(code):
            before[labels[rest]].append(i)
    found = []
    for i, (name, rest) in enumerate(code):
        read = scalars(rest) if name.startswith(("global_", "buffer_", "flat_", "scratch_")) else ()
        ways, seen = [(j, 0) for j in before[i]] if read else [], set()
        while ways:
            way = ways.pop()
            if way[1] >= WANTED or way in seen:
                continue
            seen.add(way)
            j, waited = way
            op, args = code[j]
            if op.startswith(("v_readlane", "v_readfirstlane", "v_cmp")) and scalars(args.split(",")[0]) & read:
                found.append((name + " " + rest, op + " " + args, waited))
            waited += int(args, 0) + 1 if op == "s_nop" else 1
            ways += [(k, waited) for k in before[j]]
    return found


def test_the_check_finds_what_it_looks_for():
    dma = ["s_mov_b32 m0, s9", "s_nop 0", "global_load_lds_dwordx4 v2, s[4:5]"]
    assert read_too_early(["v_readlane_b32 s5, v1, 0"] + dma) == [(dma[2], "v_readlane_b32 s5, v1, 0", 2)]
    four = ["v_readlane_b32 s5, v1, 0", "s_add_u32 s0, s0, 1", "s_add_u32 s1, s1, 1"]
    assert read_too_early(four + dma)[0][2] == 4
    assert not read_too_early(four + ["s_add_u32 s2, s2, 1"] + dma)
    assert not read_too_early(four[:1] + [dma[0], "s_nop 3", dma[2]])
    assert not read_too_early(["v_readlane_b32 s6, v1, 0"] + dma)
    # over a loop's end, and over a jump forwards
    assert read_too_early([".L0:"] + dma + ["s_nop 7", "v_readlane_b32 s4, v1, 0", "s_cbranch_scc1 .L0"])[0][2] == 3
    assert read_too_early(["v_readlane_b32 s4, v1, 0", "s_branch .L1", "s_nop 7", ".L1:"] + dma)[0][2] == 3
    assert not read_too_early(["v_readlane_b32 s4, v1, 0", "s_endpgm", ".L1:"] + dma)


def with_dma():
    """Sources whose inline assembly is in them, or in a header that they include."""
    text = {f: open(os.path.join(build.CSRC, f)).read() for f in sorted(os.listdir(build.CSRC))}

    def has(name):
        return "global_load_lds" in text[name] or any(has(h) for h in re.findall(r'#include "(\w+\.h)"', text[name]))
    return [f for f in text if f.endswith(".hip") and has(f)]


def test_sources_with_dma_are_known():
    assert {"attention_dma.hip", "gemm_bf16.hip", "kv16_attention.hip", "prompt_attention.hip"} <= set(with_dma())


@pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="needs hipcc")
@pytest.mark.parametrize("name", with_dma())
def test_addresses_are_waited_for(name, tmp_path):
    out = str(tmp_path / "kernels.s")
    cmd = [build.HIPCC] + build.FLAGS + build.FILE_FLAGS.get(name, []) + ["--cuda-device-only", "-S", "-x", "hip",
                                                                            os.path.join(build.CSRC, name), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    with open(out) as f:
        assert read_too_early(f.read().split("\n")) == []
