"""CPU test of what the kernels between tokens and logits were compiled to, from the metadata
of the built library: none spills or uses scratch memory, and the products' workgroups
have a compute unit's LDS to themselves and two waves of registers to a SIMD."""
from __future__ import annotations

import re
import os
import shutil
import subprocess

LLVM = "/opt/rocm/llvm/bin"
KERNELS = r"k_(order|sort_scan|dispatch|combine|ids|embed|norm|logits|loss|gradients|join|turn|planes|align|column_top|clear)"


def test_resources(tmp_path):
    from paper_2301_08897_amd import LIB_PATH
    lib = shutil.copy(LIB_PATH, tmp_path)
    subprocess.run([f"{LLVM}/llvm-objdump", "--offloading", lib], cwd=tmp_path, check=True, capture_output=True)
    found = {}
    for f in os.listdir(tmp_path):
        if "gfx950" not in f:
            continue
        notes = subprocess.run([f"{LLVM}/llvm-readelf", "--notes", f], cwd=tmp_path, check=True, capture_output=True, text=True).stdout
        for block in re.split(r"^\s+- \.agpr_count", notes, flags=re.M)[1:]:
            at = dict(re.findall(r"^\s+\.(name|vgpr_count|vgpr_spill_count|private_segment_fixed_size|group_segment_fixed_size):\s+(\S+)$", block, re.M))
            if "name" in at and re.search(KERNELS, at["name"]):
                found[at["name"]] = at
    assert len(found) > 90, sorted(found)
    for name, r in found.items():
        assert int(r["vgpr_spill_count"]) == 0 and int(r["private_segment_fixed_size"]) == 0, (name, r)
        if re.search(r"k_(logits|gradients)", name):
            assert int(r["vgpr_count"]) <= 256 and int(r["group_segment_fixed_size"]) == 160 * 1024, (name, r)
