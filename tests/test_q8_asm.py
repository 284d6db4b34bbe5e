"""The assembly of the 8-bit paged attention's written-out products, whose operands the compiler's own hazard rules do not
watch: two wait states between a vector instruction and a product that reads what it wrote, and eight (16 x 16) or twelve
(32 x 32) between a chain's product and anything but the chain's next that reads or writes its result; and no register is
spilled to memory up to d_c = 512."""
import os
import re
import subprocess

import pytest

from paper_2607_17644_amd import build
from test_wide_asm import registers


def early_reads(lines):
    """(what is read too early, written-out products) of a function's instructions, block after block."""
    found, products, written, before, running = [], 0, False, [], []
    for line in lines:
        text = line.split(";")[0].strip()
        if "ASMSTART" in line or "ASMEND" in line:
            written = "ASMSTART" in line
            continue
        if not text or text.startswith(".") or text.endswith(":"):
            continue
        op, _, args = text.partition(" ")
        states = 1 + (int(args) if op == "s_nop" else 0)
        if op.startswith("v_mfma") and written:
            products += 1
            to, _, rest = args.partition(",")
            reads, ago = registers(rest), 0
            for was, cost in reversed(before):
                name, _, wrote = was.partition(" ")
                if ago >= 2:
                    break
                if name.startswith("v_") and not name.startswith("v_mfma") and registers(wrote.split(",")[0]) & reads:
                    found.append((ago, was, text))
                ago += cost
            source = registers(",".join(rest.split(",")[:2]))
            for result, need, since, by in running:
                if since < need and result & source:
                    found.append((since, by, text))
            running = [r for r in running if r[0] != registers(to)] + [[registers(to), 8 if "16x16" in op else 12, 0, text]]
        else:
            if op != "s_nop":
                touched = registers(args)
                for result, need, since, by in running:
                    if since < need and result & touched:
                        found.append((since, by, text))
            for r in running:
                r[2] += states
            running = [r for r in running if r[2] < r[1]]
        before = before[-3:] + [(text, states)]
    return found, products


def test_the_check_finds_what_it_looks_for():
    product = ["; #ASMSTART", "v_mfma_f32_16x16x32_f16 v[18:21], v[4:7], a[0:3], v[18:21]", "; #ASMEND"]
    assert early_reads(["v_mov_b32_e32 v4, v9", "s_nop 0"] + product)[0]
    assert early_reads(["v_mov_b32_e32 v4, v9", "s_nop 1"] + product) == ([], 1)
    assert early_reads(product + ["s_nop 6", "v_add_f32_e32 v1, v18, v2"])[0]
    assert not early_reads(product + ["s_nop 7", "v_add_f32_e32 v1, v18, v2"])[0]
    assert early_reads(product + ["v_accvgpr_write_b32 a9, v21"])[0] and not early_reads(product + product)[0]


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("asm") / "q8.s")
    cmd = [build.HIPCC, *build.FLAGS, *build.EXTRA.get("paged_q8.hip", []), "-S", "--offload-device-only",
           os.path.join(build.CSRC, "paged_q8.hip"), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    with open(out) as f:
        return f.read()


@pytest.mark.parametrize("nk,heads", [(2, 16), (2, 32), (2, 64), (4, 16), (4, 32), (4, 64), (8, 16), (8, 32), (8, 64), (16, 16)])
@pytest.mark.parametrize("fine", [0, 1])
def test_written_out_products(assembly, nk, heads, fine):
    name = re.search(rf"^(\S*q8_kernelILi{nk}ELi{heads}ELb{fine}E\S*):", assembly, re.M).group(1)
    body = assembly[assembly.index(f"\n{name}:"):]
    body = body[:body.index(".Lfunc_end")]
    found, products = early_reads(body.split("\n"))
    assert not found, found[:3]
    assert products > 0
    kernel = assembly[assembly.index(f".amdhsa_kernel {name}"):]
    memory = int(re.search(r"\.amdhsa_private_segment_fixed_size (\d+)", kernel).group(1))
    assert memory == 0 or nk > 8
