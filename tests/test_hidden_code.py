"""What the compiler made of the layers on hidden rows, by the notes of the built library: no kernel of them puts registers away.

Where a kernel's values fill the registers the compiler (ROCm 7.2) has copied some to accumulation registers at the end of a masked piece
of code, before the mask was restored, and has put four back as three: results of single rows were lost, with no error."""
import os
import re
import struct
import subprocess

import pytest

import paper_2305_03152_amd as spp

READELF = "/opt/rocm/llvm/bin/llvm-readelf"


def _code_objects(data):
    """The GPU's ELF files inside the library, by their header (machine 224)."""
    at = data.find(b"\x7fELF", 1)
    while at >= 0:
        if data[at + 4] == 2 and struct.unpack_from("<H", data, at + 18)[0] == 224:
            shoff, = struct.unpack_from("<Q", data, at + 40)
            size, count = struct.unpack_from("<HH", data, at + 58)
            yield data[at:at + shoff + size * count]
        at = data.find(b"\x7fELF", at + 1)


@pytest.mark.skipif(not os.path.exists(READELF), reason="no llvm-readelf")
def test_no_kernel_of_the_hidden_layers_spills(tmp_path):
    if not os.path.exists(spp.LIB_PATH):
        from paper_2305_03152_amd import build
        build.build()
    kernels = {}
    for k, obj in enumerate(_code_objects(open(spp.LIB_PATH, "rb").read())):
        path = tmp_path / f"{k}.o"
        path.write_bytes(obj)
        text = subprocess.run([READELF, "--notes", str(path)], check=True, capture_output=True, text=True).stdout
        for block in re.split(r"\n  - ", text):
            name, spill, scratch = (re.search(p, block) for p in (r"\.name:\s+(_Z\S*(?:hidden|Fp8)\S*)\n", r"\.vgpr_spill_count:\s+(\d+)", r"\.private_segment_fixed_size:\s+(\d+)"))
            if name and spill and scratch:
                kernels[name.group(1)] = int(spill.group(1)), int(scratch.group(1))
    assert len(kernels) > 100, len(kernels)
    assert {k: v for k, v in kernels.items() if v != (0, 0)} == {}
