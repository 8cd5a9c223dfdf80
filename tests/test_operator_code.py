"""What the compiler made of the operators' kernels, by the notes of the built library: none of them, of any layer or row format, puts vector registers away,
and those that need most of the registers have no masked code behind their first product.

Where a kernel's values fill the registers the compiler (ROCm 7.2) has put four away and back as three, and has copied some to accumulation registers at
the end of masked code, before the mask was restored: results of single rows were lost, with no error.  (Scalar registers are put into lanes of a vector register, whatever the mask; that is another matter.)"""
import os
import re
import subprocess

import pytest

import paper_2305_03152_amd as spp
from test_hidden_code import READELF, _code_objects

# the layers in 4 and 8 bits, the weight gradients, rows to few bits and back, the optimiser
KERNELS = {"mx4_rows_kernel": 30, "mx4_product_kernel": 6, "hidden_held_kernel": 60, "hidden_wide_kernel": 60, "hidden_tile_kernel": 9, "weight_grad_kernel": 40,
           "weight_grad_sum_kernel": 1, "quantize_rows_kernel": 6, "dequantize_rows_kernel": 12, "adamw": 3}


def _built():
    if not os.path.exists(spp.LIB_PATH):
        from paper_2305_03152_amd import build
        build.build()


OBJDUMP = os.path.join(os.path.dirname(READELF), "llvm-objdump")
MANY = 300                       # registers, of 512


@pytest.mark.skipif(not os.path.exists(READELF), reason="no llvm-readelf")
def test_no_kernel_of_the_operators_spills(tmp_path):
    _built()
    seen, spilled = dict.fromkeys(KERNELS, 0), {}
    for k, obj in enumerate(_code_objects(open(spp.LIB_PATH, "rb").read())):
        path = tmp_path / f"{k}.o"
        path.write_bytes(obj)
        text = subprocess.run([READELF, "--notes", str(path)], check=True, capture_output=True, text=True).stdout
        for block in re.split(r"\n  - ", text):
            name, spill, scratch = (re.search(p, block) for p in (r"\.name:\s+(_Z\S+)\n", r"\.vgpr_spill_count:\s+(\d+)", r"\.private_segment_fixed_size:\s+(\d+)"))
            kind = name and next((kind for kind in KERNELS if re.search(r"\d" + kind, name.group(1))), None)
            if kind:
                seen[kind] += 1
                if (spill.group(1), scratch.group(1)) != ("0", "0"):
                    spilled[name.group(1)] = spill.group(1), scratch.group(1)
    assert all(seen[kind] >= least for kind, least in KERNELS.items()), seen
    assert spilled == {}


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no llvm-objdump")
def test_kernels_of_many_registers_are_not_masked_behind_their_products(tmp_path):
    _built()
    looked, masked = 0, {}
    for k, obj in enumerate(_code_objects(open(spp.LIB_PATH, "rb").read())):
        path = tmp_path / f"{k}.o"
        path.write_bytes(obj)
        notes = subprocess.run([READELF, "--notes", str(path)], check=True, capture_output=True, text=True).stdout
        many = set()
        for block in re.split(r"\n  - ", notes):
            name, count = (re.search(p, block) for p in (r"\.name:\s+(_Z\S+)\n", r"\.vgpr_count:\s+(\d+)"))
            if name and count and int(count.group(1)) > MANY and any(re.search(r"\d" + kind, name.group(1)) for kind in KERNELS):
                many.add(name.group(1))
        if not many:
            continue
        code = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", str(path)], check=True, capture_output=True, text=True).stdout
        for part in re.split(r"\n(?=[0-9a-f]* ?<_Z)", code):
            head = re.match(r"[0-9a-f]* ?<(_Z\S+)>:", part)
            if head and head.group(1) in many:
                looked += 1
                behind = part[part.index("v_mfma"):]
                if "saveexec" in behind:
                    masked[head.group(1)] = behind.count("saveexec")
    assert looked > 40
    assert masked == {}
