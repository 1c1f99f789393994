"""What the compiler gives the attention kernels, read from the code objects of the built library: a wave more or less per SIMD is a step that
no result shows.  A SIMD has 512 registers of 64 lanes, given out by eight: three waves have up to 168 each."""
import os
import re
import struct
import subprocess

import pytest

import paper_1801_00829_amd as F
from paper_1801_00829_amd.build import ARCH

READELF = "/opt/rocm/llvm/bin/llvm-readelf"
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"
THREE_WAVES = 168


def _code_objects(data):
    """Of every bundle in the library, the part for the GPU: a count, then offset, size and target of each part."""
    at = data.find(MAGIC)
    while at >= 0:
        (count,), place = struct.unpack_from("<Q", data, at + len(MAGIC)), at + len(MAGIC) + 8
        for _ in range(count):
            offset, size, length = struct.unpack_from("<QQQ", data, place)
            target = data[place + 24:place + 24 + length]
            place += 24 + length
            if target.endswith(ARCH.encode()) and size:
                yield data[at + offset:at + offset + size]
        at = data.find(MAGIC, at + len(MAGIC))


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{mangled name: (registers, bytes of scratch memory per lane)}"""
    if not os.path.exists(F.lib_path()) or not os.path.exists(READELF):
        pytest.skip("needs the built library and %s" % READELF)
    with open(F.lib_path(), "rb") as f:
        data = f.read()
    elf, found = str(tmp_path_factory.mktemp("code") / "code.elf"), {}
    for code in _code_objects(data):
        with open(elf, "wb") as f:
            f.write(code)
        notes = subprocess.run([READELF, "--notes", elf], capture_output=True, text=True, check=True).stdout
        for kernel in re.split(r"\n  - ", notes)[1:]:
            name, registers, scratch = (re.search(r"^ *\.%s: +(\S+)" % key, kernel, re.M) for key in
                                        ("name", "vgpr_count", "private_segment_fixed_size"))
            if name and registers:
                found[name[1].strip("'")] = int(registers[1]), int(scratch[1])
    assert found
    return found


@pytest.mark.parametrize("type_", ["DF16b", "DF16_"])
@pytest.mark.parametrize("shape", [0, 1, 3])
@pytest.mark.parametrize("even", [0, 1])
def test_gradients_of_keys_of_64_dims_have_three_waves(kernels, type_, shape, even):
    """Plain scores, a prefix alone, and a cap: bf16 and fp16 alike."""
    got = [v for k, v in kernels.items() if "attention_key_grad_kernelI%sLi64ELb%dELi%dE" % (type_, even, shape) in k]
    assert len(got) == 1
    assert got[0][0] <= THREE_WAVES and got[0][1] == 0, got
