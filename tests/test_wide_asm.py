"""The assembly of the wide paged attention's written-out instructions, whose operands the compiler's own hazard rules
do not watch: wait states between a vector instruction and a matrix product that reads what it wrote (two), and
between one that writes a scalar and a copy whose base it is (five); and no register is spilled to memory."""
import os
import re
import subprocess

import pytest

from paper_2607_17644_amd import build


def registers(text):
    out = set()
    for kind, lo, hi, one in re.findall(r"\b([sva])(?:\[(\d+):(\d+)\]|(\d+)\b)", text):
        out |= {kind + one} if one else {kind + str(i) for i in range(int(lo), int(hi) + 1)}
    return out


def hazards(lines):
    """(what is read too early, written-out products, copies with a scalar base) of a function's instructions."""
    found, products, copies, written, before = [], 0, 0, False, []
    for line in lines:
        text = line.split(";")[0].strip()
        if "ASMSTART" in line or "ASMEND" in line:
            written = "ASMSTART" in line
            continue
        if not text or text.startswith(".") or text.endswith(":"):
            continue
        op, _, args = text.partition(" ")
        args = args.strip()
        states = 0
        if op.startswith("v_mfma") and written:
            products += 1
            need, reads = 2, registers(args.split(",", 1)[1])
        elif op.startswith("global_load_lds") and "s[" in args:
            copies += 1
            need, reads = 5, {r for r in registers(args) if r[0] == "s"}
        else:
            need, reads = 0, set()
        for was in reversed(before[-need:] if need else []):
            if states >= need:
                break
            name, _, rest = was.partition(" ")
            vector = name.startswith("v_") and not name.startswith("v_mfma")
            if vector and registers(rest.split(",")[0]) & reads:
                found.append((states, was, text))
            states += 1 + (int(rest) if name == "s_nop" else 0)
        before.append(text)
    return found, products, copies


def test_the_check_finds_what_it_looks_for():
    early = ["v_mov_b32_e32 v4, v9", "s_nop 0", "; #ASMSTART", "v_mfma_f32_32x32x16_bf16 v[18:33], v[4:7], a[0:3], v[18:33]", "; #ASMEND"]
    late = early[:1] + ["s_nop 1"] + early[2:]
    assert hazards(early)[0] and not hazards(late)[0] and hazards(late)[1] == 1
    base = ["v_readlane_b32 s9, v4, 3", "s_add_u32 m0, s4, 8", "s_nop 2", "global_load_lds_dwordx4 v1, s[8:9]"]
    assert hazards(base)[0] and not hazards(base[:2] + ["s_nop 3"] + base[3:])[0]


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("asm") / "wide.s")
    cmd = [build.HIPCC, *build.FLAGS, *build.EXTRA.get("paged_wide.hip", []), "-S", "--offload-device-only",
           os.path.join(build.CSRC, "paged_wide.hip"), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    with open(out) as f:
        return f.read()


@pytest.mark.parametrize("groups", [1, 2])
def test_written_out_instructions(assembly, groups):
    name = re.search(rf"^(\S*wide_kernelILi{groups}E\S*):", assembly, re.M).group(1)
    body = assembly[assembly.index(f"\n{name}:"):]
    body = body[:body.index(".Lfunc_end")]
    found, products, copies = hazards(body.split("\n"))
    assert not found, found[:3]
    assert products > 0 and copies > 0
    kernel = assembly[assembly.index(f".amdhsa_kernel {name}"):]
    assert re.search(r"\.amdhsa_private_segment_fixed_size (\d+)", kernel).group(1) == "0"
