"""Registers of the products' kernels as they were compiled: a compute unit has 128 vector registers a lane for each of four waves on a SIMD, so a workgroup of
eight waves that takes more of them has the compute unit to itself.  (Tiles of 128 x 128 need two workgroups there: with one, a product's dx took 1.3 times as long.)"""
import os
import re
import subprocess

import pytest

from paper_2506_00812_amd import build

LLVM = "/opt/rocm/llvm/bin"
OBJECTS = [os.path.join(build.CSRC, "_build", name) for name in ("vf_linear.o", "vf_gated.o")]


def kernels(obj, tmp):
    """(mangled name, vector registers, bytes of scratch memory) of each kernel in an object of this library."""
    fat, code = os.path.join(tmp, "fat"), os.path.join(tmp, "code")
    subprocess.run([f"{LLVM}/llvm-objcopy", "--dump-section", f".hip_fatbin={fat}", obj, os.path.join(tmp, "copy")], check=True)
    subprocess.run([f"{LLVM}/clang-offload-bundler", "--unbundle", "--type=o", f"--input={fat}", f"--output={code}",
                    "--targets=hipv4-amdgcn-amd-amdhsa--gfx950"], check=True)
    notes = subprocess.run([f"{LLVM}/llvm-readelf", "--notes", code], check=True, capture_output=True, text=True).stdout
    for part in notes.split("- .agpr_count")[1:]:
        value = lambda key: re.search(rf"\.{key}:\s+(\S+)", part).group(1)   # noqa: E731
        yield value("name"), int(value("vgpr_count")), int(value("private_segment_fixed_size"))


@pytest.mark.parametrize("obj", OBJECTS, ids=os.path.basename)
def test_two_workgroups_of_eight_waves_fit(obj, tmp_path):
    if not os.path.exists(obj) or not os.path.exists(f"{LLVM}/clang-offload-bundler"):
        pytest.skip("no compiled object, or no tools to look into it")
    tiles = [k for k in kernels(obj, str(tmp_path)) if "11tile_kernelI" in k[0] and "ELi128ELi128ELi2ELi4E" in k[0]]
    assert len(tiles) == (9 if "linear" in obj else 3)
    for name, registers, scratch in tiles:
        assert registers <= 128 and scratch == 0, (name, registers, scratch)
