"""What the compiler made of the 8-bit kernels: registers, and the distance of matrix instructions from the vector instructions they depend on.

The large product kernel keeps its accumulators in 256 registers of one kind and everything else in the other 256; a spill there would sit in the
k-loop.  Its matrix instructions are assembly, which the compiler knows nothing about: one must not follow a vector instruction that
writes one of its operands within two instructions.  CPU only: the device code is compiled with the library's own flags and read.
"""

import os
import re
import subprocess
import tempfile

import pytest

from paper_2403_11204_amd import build


def assembly(unit):
    with tempfile.TemporaryDirectory() as tmp:
        out = os.path.join(tmp, "unit.s")
        cmd = [build.hipcc()] + [a for a in build.COMMON if a != "-fPIC"] + build.UNITS[unit] + ["--cuda-device-only", "-S", os.path.join(build.CSRC, unit), "-o", out]
        r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        assert r.returncode == 0, r.stdout[-2000:]
        return open(out).read()


def kernels(text):
    found = {}
    for entry in text[text.index("amdhsa.kernels"):].split("- .agpr_count")[1:]:
        name = re.search(r"\.name:\s+(\S+)", entry).group(1)
        found[name] = {k: int(re.search(r"\.%s:\s+(\d+)" % k, entry).group(1)) for k in ("vgpr_count", "vgpr_spill_count", "private_segment_fixed_size")}
    return found


@pytest.fixture(scope="module")
def product():
    return assembly("product.hip")


@pytest.mark.parametrize("unit", ["norm.hip", "quantize.hip", "clip.hip"])
def test_no_kernel_spills(unit):
    for name, v in kernels(assembly(unit)).items():
        assert v["vgpr_spill_count"] == 0 and v["private_segment_fixed_size"] == 0, (name, v)


def test_no_product_spills(product):
    found = kernels(product)
    assert sum("product_long_kernel" in n for n in found) == 2 and sum("product_tile_kernel" in n for n in found) == 18 and sum("product_rows_kernel" in n for n in found) == 2
    for name, v in found.items():
        assert v["vgpr_spill_count"] == 0 and v["private_segment_fixed_size"] == 0, (name, v)
        if "product_tile_kernel" in name:
            assert v["vgpr_count"] <= 256, (name, v)      # two workgroups of 4 wavefronts on a compute unit


def registers(operands):
    found = set()
    for m in re.finditer(r"\bv\[(\d+):(\d+)\]|\bv(\d+)\b", operands):
        found |= {int(m.group(3))} if m.group(3) else set(range(int(m.group(1)), int(m.group(2)) + 1))
    return found


def test_matrix_instructions_in_assembly_keep_their_distance(product):
    names = re.findall(r"^(_ZN\S*product_long_kernel\S*):", product, re.M)
    assert len(names) == 2
    for name in names:
        body = product[product.index("\n" + name + ":"):]
        body = body[:body.index("s_endpgm")]
        written, matrix = [], 0
        for line in body.split("\n"):
            op, _, args = line.split(";")[0].strip().partition(" ")
            if not op or op.startswith(".") or op.endswith(":"):
                continue
            first, _, rest = args.partition("]," if args.startswith(("v[", "a[")) else ",")
            if op.startswith("v_mfma"):
                matrix += 1
                for back in written[-2:]:
                    assert not (back & registers(rest)), (name, line)
                written.append(set())
            elif op == "s_nop":
                written += [set()] * (int(args) + 1)
            else:
                written.append(registers(first + "]" if first.startswith("v[") else first) if op.startswith("v_") else set())
        assert matrix >= 64, (name, matrix)
