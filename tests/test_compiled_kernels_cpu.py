"""What the compiler made of the kernels, read from the built library's own metadata (no GPU here)."""
import functools
import os
import re
import struct
import subprocess

import pytest

READELF = "/opt/rocm/llvm/bin/llvm-readelf"


@functools.lru_cache(maxsize=None)
def kernels(tmp):
    """{demangled name: {key: number}} of the gfx950 kernels in the library."""
    from paper_2301_06284_amd import build
    data = open(build.LIB, "rb").read()
    found, at = {}, data.find(b"__CLANG_OFFLOAD_BUNDLE__")
    assert at >= 0
    while at >= 0:
        entries, pos = struct.unpack_from("<Q", data, at + 24)[0], at + 32
        for i in range(entries):
            offset, size, length = struct.unpack_from("<3Q", data, pos)
            target = data[pos + 24:pos + 24 + length]
            pos += 24 + length
            if b"gfx950" not in target:
                continue
            path = os.path.join(tmp, f"{at}_{i}.elf")
            with open(path, "wb") as f:
                f.write(data[at + offset:at + offset + size])
            notes = subprocess.run([READELF, "--notes", path], capture_output=True, text=True, check=True).stdout
            for part in re.split(r"\n  - ", notes)[1:]:
                name = re.search(r"^    \.name: +'?([^\s']+)", part, re.M)
                if name:
                    found[name.group(1)] = {k: int(v) for k, v in re.findall(r"^    \.(\w+): +(\d+)$", part, re.M)}
        at = data.find(b"__CLANG_OFFLOAD_BUNDLE__", at + 1)
    return found


@pytest.fixture(scope="module")
def compiled(tmp_path_factory):
    if not os.path.exists(READELF):
        pytest.skip("needs llvm-readelf")
    return kernels(str(tmp_path_factory.mktemp("code")))


def test_integer_tiles_keep_their_sums_in_registers(compiled):
    """The tiles of the typed linear in 8-bit integers, below the 256 x 256 one, spill nothing."""
    tiles = {n: k for n, k in compiled.items() if "typed_linear_kernelINS_2I8E" in n}
    assert len(tiles) >= 6
    for name, k in tiles.items():
        assert k["vgpr_spill_count"] == 0 and k["private_segment_fixed_size"] == 0, name


@pytest.mark.parametrize("pattern", [
    r"rms_norm_kernelI.*LNS_3FitE1ELi1ELi1E",                 # one lane a row, rows that end inside a vector: those have nine columns or more
    r"rms_norm_backward_kernelI.*LNS_3FitE1ELb[01]ELi1ELi1E",
    r"dropout_kernelIDF16_Lb1ELb1E",                          # all of fp32, compiled for a second 16-bit type
    r"typed_linear_kernelI.*(BF16|F16|F8|I8)ELi(32|64)ELi64E.*Lb0ELi1EEE",      # four-stage tiles where k is one step
])
def test_nothing_is_compiled_that_no_call_reaches(compiled, pattern):
    kept = re.sub(r"LNS_3FitE1", "LNS_3FitE0", pattern).replace("Lb1ELb1E", "Lb1ELb0E").replace("Lb0ELi1EEE", "Lb0ELi4EEE")
    assert any(re.search(kept, n) for n in compiled), "the names have changed"
    assert [n for n in compiled if re.search(pattern, n)] == []
