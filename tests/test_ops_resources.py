"""Registers, scratch and instruction distances of the operators' kernels, from the compiler's output (no GPU)."""
import os
import re
import subprocess

import pytest

from tests.test_kernel_resources import CSRC, HIPCC, ROOT, _registers

SOURCES = ["norm.hip", "route.hip", "group.hip", "q8_product.hip"]


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    found = {}
    for src in SOURCES:
        out = tmp_path_factory.mktemp("dev") / (src + ".s")
        subprocess.run([HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-x", "hip", "--cuda-device-only",
                        "-S", os.path.join(CSRC, src), f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}", "-o", str(out),
                        "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"],
                       check=True, capture_output=True)
        text = out.read_text()
        for block in re.split(r"\n  - ", text.split("amdhsa.kernels:", 1)[1])[1:]:
            fields = dict(re.findall(r"^\s*\.(\w+):\s+(\S+)", block, re.M))
            if "name" in fields:
                fields["body"] = text.split("\n" + fields["name"] + ":", 1)[1].split(".Lfunc_end", 1)[0]
                found[fields["name"]] = fields
    return found


def test_no_kernel_spills(kernels):
    assert len(kernels) >= 8
    for name, f in kernels.items():
        assert int(f["private_segment_fixed_size"]) == 0, name
        assert int(f["vgpr_spill_count"]) == 0, name
        assert "v_pk_fma_f32" not in f["body"] and "v_pk_mul_f32" not in f["body"] and "v_pk_add_f32" not in f["body"], name


def test_assembly_products_keep_their_distances(kernels):
    """The tile kernels' matrix instructions and LDS DMAs are assembly statements: in the emitted order no vector
    instruction writes an operand within two wait states before a matrix instruction reads it, none but a matrix
    instruction touches an accumulator within 11 of its product, and no lane read writes a DMA's scalar base
    within 5."""
    tiles = {n: f for n, f in kernels.items() if "q8_tile_kernel" in n}
    assert tiles
    for name, f in tiles.items():
        ins = [line.split(";")[0].strip() for line in f["body"].split("\n")
               if line.startswith("\t") and not line.strip().startswith((".", ";"))]
        states = [int(i.split()[1]) + 1 if i.startswith("s_nop") else 1 for i in ins]

        def before(i, limit):
            ws = 0
            while i > 0 and ws < limit:
                i -= 1
                yield ins[i]
                ws += states[i]

        products = 0
        for i, op in enumerate(ins):
            if op.startswith("v_mfma"):
                products += 1
                reads = {r for r in _registers(op) if r[0] in "va"}
                for p in before(i, 2):
                    if p.startswith("v_") and not p.startswith(("v_mfma", "v_cmp")):
                        assert not _registers(p.split(None, 1)[1].split(",")[0]) & reads, (name, p, op)
                acc, ws = {r for r in _registers(op) if r[0] == "a"}, 0
                for k in range(i + 1, len(ins)):
                    if ws >= 11 or ins[k].startswith(("s_cbranch", "s_branch", "s_endpgm")):
                        break
                    assert ins[k].startswith("v_mfma") or not _registers(ins[k]) & acc, (name, op, ins[k])
                    ws += 4 if ins[k].startswith("v_mfma") else states[k]
            elif op.startswith("global_load_lds"):
                base = {r for r in _registers(op) if r[0] == "s"}
                for p in before(i, 5):
                    if p.startswith(("v_readlane", "v_readfirstlane")):
                        assert not _registers(p.split(None, 1)[1].split(",")[0]) & base, (name, p, op)
        assert products > 100, name


def instructions(body):
    """The emitted instructions, and the wait states each takes to issue."""
    ins = [line.split(";")[0].strip() for line in body.split("\n")
           if line.startswith("\t") and not line.strip().startswith((".", ";"))]
    return ins, [int(i.split()[1]) + 1 if i.startswith("s_nop") else 1 for i in ins]


def test_small_tiles_keep_the_distances_too(kernels):
    """The smaller tiles' kernels, gated and not, are made of the same assembly statements."""
    small = {n: f for n, f in kernels.items() if "q8_small_kernel" in n}
    assert len(small) == 4
    for name, f in small.items():
        ins, states = instructions(f["body"])

        def before(i, limit):
            ws = 0
            while i > 0 and ws < limit:
                i -= 1
                yield ins[i]
                ws += states[i]

        products = loads = 0
        for i, op in enumerate(ins):
            if op.startswith("v_mfma"):
                products += 1
                reads = {r for r in _registers(op) if r[0] in "va"}
                for p in before(i, 2):
                    if p.startswith("v_") and not p.startswith(("v_mfma", "v_cmp")):
                        assert not _registers(p.split(None, 1)[1].split(",")[0]) & reads, (name, p, op)
                acc, ws = {r for r in _registers(op) if r[0] == "a"}, 0
                for k in range(i + 1, len(ins)):
                    if ws >= 11 or ins[k].startswith(("s_cbranch", "s_branch", "s_endpgm")):
                        break
                    assert ins[k].startswith("v_mfma") or not _registers(ins[k]) & acc, (name, op, ins[k])
                    ws += 4 if ins[k].startswith("v_mfma") else states[k]
            elif op.startswith("global_load_lds"):
                loads += 1
                base = {r for r in _registers(op) if r[0] == "s"}
                for p in before(i, 5):
                    if p.startswith(("v_readlane", "v_readfirstlane")):
                        assert not _registers(p.split(None, 1)[1].split(",")[0]) & base, (name, p, op)
        # Four fragments by four (or two by two) in each half of five unrolled K steps at least, and their loads.
        side = 4 if "Li128E" in name else 2
        assert products >= 10 * side * side and loads >= 2 * side, (name, products, loads)
