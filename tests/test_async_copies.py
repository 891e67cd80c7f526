"""Kernels that may be on the SMs while the one ahead of them still writes (launch() in conef_internal.h), and that bring its results by asynchronous copies, order
those behind its ordinary stores: copies go through another proxy, which a wait for the grid ahead is not said to cover."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2312_08538_b200", "csrc")


def test_a_proxy_fence_follows_the_wait():
    found = []
    for name in sorted(os.listdir(CSRC)):
        if not name.endswith((".cu", ".cuh")):
            continue
        with open(os.path.join(CSRC, name)) as f:
            text = re.sub(r"//.*", "", f.read())
        if not re.search(r"tc::(tile_load|bulk_load)", text):
            continue
        for kernel in re.split(r"__global__", text)[1:]:
            if re.search(r"tc::(tile_load|bulk_load)", kernel):
                found.append((name, bool(re.search(r"grid_wait\(\);\s*asm volatile\(\"fence\.proxy\.async;\" ::: \"memory\"\);", kernel))))
    assert len(found) >= 2 and all(ok for _, ok in found), found
