"""Registers, scratch and instruction distances of the kernels that train a layer, from the compiler's output (no GPU)."""
import os
import re
import subprocess

import pytest

from tests.test_kernel_resources import CSRC, HIPCC, ROOT, _registers

SOURCES = ["product.hip", "product_dw.hip", "gate.hip", "combine_backward.hip", "clip.hip"]


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    jobs = []
    for src in SOURCES:
        out = tmp_path_factory.mktemp("dev") / (src + ".s")
        jobs.append((out, subprocess.Popen(
            [HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-x", "hip", "--cuda-device-only", "-S", os.path.join(CSRC, src),
             f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}", "-o", str(out), "-Xclang", "-target-feature", "-Xclang",
             "-packed-fp32-ops"], stderr=subprocess.DEVNULL)))
    found = {}
    for out, job in jobs:
        assert job.wait() == 0
        text = out.read_text()
        for block in re.split(r"\n  - ", text.split("amdhsa.kernels:", 1)[1])[1:]:
            fields = dict(re.findall(r"^\s*\.(\w+):\s+(\S+)", block, re.M))
            if "name" in fields:
                fields["body"] = text.split("\n" + fields["name"] + ":", 1)[1].split(".Lfunc_end", 1)[0]
                found[fields["name"]] = fields
    return found


def test_no_kernel_spills(kernels):
    assert len(kernels) >= 20
    for name, f in kernels.items():
        assert int(f["private_segment_fixed_size"]) == 0, name
        assert int(f["vgpr_spill_count"]) == 0, name
        assert "v_pk_fma_f32" not in f["body"] and "v_pk_mul_f32" not in f["body"] and "v_pk_add_f32" not in f["body"], name


def instructions(body):
    """The emitted instructions, the wait states each takes to issue, and whether it is an assembly statement's."""
    ins, states, mine, inside = [], [], [], False
    for line in body.split("\n"):
        text = line.strip()
        if text.startswith(";;#ASM"):
            inside = text.startswith(";;#ASMSTART")
        op = text.split(";")[0].strip()
        if not line.startswith("\t") or not op or op.startswith("."):
            continue
        ins.append(op)
        states.append(int(op.split()[1]) + 1 if op.startswith("s_nop") else 1)
        mine.append(inside)
    return ins, states, mine


@pytest.mark.parametrize("kind,count", [("product_tile_kernel", 2), ("dw_tile_kernel", 2), ("product_small_kernel", 7), ("dw_small_kernel", 4),
                                        ("product_thin_kernel", 1)])
def test_assembly_statements_keep_their_distances(kernels, kind, count):
    """Matrix instructions and LDS DMAs that are assembly statements: no vector instruction writes an operand within two
    wait states before a matrix instruction reads it, none but a matrix instruction touches an accumulator within 11 of
    its product, and no lane read writes a DMA's scalar base within 5.  (The compiler sees to its own.)"""
    chosen = {n: f for n, f in kernels.items() if kind in n}
    assert len(chosen) == count
    for name, f in chosen.items():
        ins, states, mine = instructions(f["body"])

        def before(i, limit):
            ws = 0
            while i > 0 and ws < limit:
                i -= 1
                yield ins[i]
                ws += states[i]

        products = loads = 0
        for i, op in enumerate(ins):
            if op.startswith("v_mfma") and mine[i]:
                products += 1
                reads = {r for r in _registers(op) if r[0] in "va"}
                for p in before(i, 2):
                    if p.startswith("v_") and not p.startswith(("v_mfma", "v_cmp")):
                        assert not _registers(p.split(None, 1)[1].split(",")[0]) & reads, (name, p, op)
                acc, ws = {r for r in _registers(op) if r[0] == "a"}, 0
                for k in range(i + 1, len(ins)):
                    if ws >= 11 or ins[k].startswith(("s_cbranch", "s_branch", "s_endpgm")) and not mine[k]:
                        break
                    assert ins[k].startswith("v_mfma") or not _registers(ins[k]) & acc, (name, op, ins[k])
                    ws += 4 if ins[k].startswith("v_mfma") else states[k]
            elif op.startswith("global_load_lds"):
                loads += 1
                base = {r for r in _registers(op) if r[0] == "s"}
                for p in before(i, 5):
                    if p.startswith(("v_readlane", "v_readfirstlane")):
                        assert not _registers(p.split(None, 1)[1].split(",")[0]) & base, (name, p, op)
        assert loads >= 8 and (products >= 16 or kind == "product_thin_kernel"), (name, products, loads)
