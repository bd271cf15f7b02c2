"""Registers of a drafting step's kernels, by the built library's own metadata (written by the
compiler): vector registers spilled to scratch memory, and how many waves of a SIMD the
registers leave.  Runs without a GPU."""
import re
import shutil
import subprocess

import pytest

from paper_2405_19888_amd import binding as B
from test_kernel_resources import code_objects

# the 16-bit tiles of 128-element heads, at three waves a SIMD: outside their stage loops
SPILLS = {"k_tree_partials<16, 128, 0>": 32, "k_tree_decode<16, 128>": 2}
WAVES = {"k_rotary_fill": 8, "k_tree_decode": 3, "k_tree_small": 2, "k_tree_partials": 2, "k_tree_join": 8,
         "k_tree_accept": 8, "k_tree_commit": 8}


def test_registers(parrot_lib, tmp_path):
    readelf = shutil.which("llvm-readelf", path="/opt/rocm/llvm/bin") or shutil.which("llvm-readelf")
    if readelf is None:
        pytest.skip("llvm-readelf is not installed")
    found = set()
    for i, image in enumerate(code_objects(open(B.LIB_PATH, "rb").read())):
        f = tmp_path / f"{i}.elf"
        f.write_bytes(image)
        notes = subprocess.run([readelf, "--notes", str(f)], capture_output=True, text=True, check=True).stdout
        for entry in re.split(r"\n\s+- \.a", notes)[1:]:
            value = lambda field: int(re.search(rf"\.{field}:\s+(\d+)", entry).group(1))
            name = re.search(r"\.name:\s+_ZN6parrot\d+(k_(?:tree|rotary)_[a-z]+)(I(?:Li\d+E)+E)?", entry)
            if not name:
                continue
            kernel, numbers = name.group(1), re.findall(r"Li(\d+)E", name.group(2) or "")
            found.add(kernel)
            full = kernel + "<" + ", ".join(["32" if numbers[0] == "0" else "16", *numbers[1:]]) + ">" if numbers else kernel
            assert value("vgpr_spill_count") <= SPILLS.get(full, 0), full
            # (element-wise partners are read at half the waves)
            least = 4 if kernel == "k_rotary_fill" and numbers[2] == "3" else WAVES[kernel]
            if kernel == "k_tree_partials" and numbers[2] == "0":
                least = 3
            assert 512 // (-(-value("vgpr_count") // 8) * 8) >= least, full
    assert found == set(WAVES)
