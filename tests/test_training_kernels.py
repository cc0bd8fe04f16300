"""CPU test of what the training operators' kernels were compiled to, from the
metadata of the built library: none spills or uses scratch memory, and those
whose workgroups must fit the GPU together have the registers for it."""
from __future__ import annotations

import os
import re
import shutil
import subprocess

LLVM = "/opt/rocm/llvm/bin"


def kernels(tmp_path):
    from paper_2301_08897_amd import LIB_PATH
    lib = shutil.copy(LIB_PATH, tmp_path)
    subprocess.run([f"{LLVM}/llvm-objdump", "--offloading", lib], cwd=tmp_path, check=True, capture_output=True)
    found = {}
    for f in os.listdir(tmp_path):
        if "gfx950" not in f:
            continue
        notes = subprocess.run([f"{LLVM}/llvm-readelf", "--notes", f], cwd=tmp_path, check=True, capture_output=True, text=True).stdout
        name = None
        for key, value in re.findall(r"^\s+\.(\w+):\s+(\S+)$", notes, re.M):
            if key == "name" and re.search(r"k_(adamw|grad_norm|route)", value):
                name = value
                found[name] = {}
            elif name and key in ("vgpr_count", "vgpr_spill_count", "private_segment_fixed_size"):
                found[name].setdefault(key, int(value))
    return found


def test_no_spills(tmp_path):
    found = kernels(tmp_path)
    assert len(found) > 40, sorted(found)
    for name, r in found.items():
        assert r["vgpr_spill_count"] == 0 and r["private_segment_fixed_size"] == 0, (name, r)
        if "k_adamwI" in name:
            assert r["vgpr_count"] <= 64, (name, r)         # eight waves per SIMD hide the loads
        elif "k_routeI" in name and name.split("k_routeI")[1].split("EvNS")[0].endswith("Lb0E"):
            assert r["vgpr_count"] <= 128, (name, r)        # four workgroups per compute unit
        elif "k_route_back" in name:
            assert r["vgpr_count"] <= 96, (name, r)         # five
