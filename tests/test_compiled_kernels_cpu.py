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
