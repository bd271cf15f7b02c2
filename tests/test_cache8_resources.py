"""Registers of the kernels of a cache held in 8 bits, by the built library's own metadata (written
by the compiler): no vector register in scratch memory, and how many waves of a SIMD the registers
leave.  Runs without a GPU."""
import re
import shutil
import subprocess

import pytest

from paper_2405_19888_amd import binding as B
from test_kernel_resources import code_objects

WAVES = {"k_cache8_fill": 3, "k_cache8_fill_tokens": 3, "k_cache8_plan": 4, "k_cache8_attend": 2, "k_cache8_direct": 2,
         "k_cache8_join": 4, "k_copy_blocks": 8}


def test_registers(parrot_lib, tmp_path):
    readelf = shutil.which("llvm-readelf", path="/opt/rocm/llvm/bin") or shutil.which("llvm-readelf")
    if readelf is None:
        pytest.skip("llvm-readelf is not installed")
    found = {}
    for i, image in enumerate(code_objects(open(B.LIB_PATH, "rb").read())):
        f = tmp_path / f"{i}.elf"
        f.write_bytes(image)
        notes = subprocess.run([readelf, "--notes", str(f)], capture_output=True, text=True, check=True).stdout
        for entry in re.split(r"\n\s+- \.a", notes)[1:]:
            value = lambda field: int(re.search(rf"\.{field}:\s+(\d+)", entry).group(1))
            name = re.search(r"\.name:\s+_ZN6parrot\d+(k_(?:cache8|copy)_[a-z]+(?:_[a-z]+)?)(I\S+?E)?E?v?N?S?_?", entry)
            if not name:
                continue
            kernel = name.group(1)
            assert value("vgpr_spill_count") == 0 and value("private_segment_fixed_size") == 0, (kernel, name.group(2))
            waves = 512 // (-(-value("vgpr_count") // 8) * 8)
            found[kernel] = min(found.get(kernel, 8), waves)
    assert set(found) == set(WAVES)
    for kernel, waves in found.items():
        assert waves >= WAVES[kernel], kernel
