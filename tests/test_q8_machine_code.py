"""What the compiler made of the 8-bit cache's kernels: no scratch memory, and the kernel that merges its pieces waits for its stores
before it counts itself in."""
import os
import subprocess

import pytest

import paper_2405_03917_amd as cq
from test_arrival_waits import OBJDUMP, kernels, unwaited
from test_kernel_scratch import _code_objects, _kernels

pytestmark = pytest.mark.skipif(not os.path.exists(cq.LIB_PATH), reason="library not built")
FAMILIES = {"append_token_q8_kernel": 2, "append_q8_kernel": 2, "dequantize_q8_kernel": 2, "rows_q8_kernel": 4, "chunk_q8_kernel": 4, "merge_q8_kernel": 1}


@pytest.fixture(scope="module")
def objects():
    """(code object, metadata of its kernels), of those that hold kernels of the 8-bit cache"""
    with open(cq.LIB_PATH, "rb") as f:
        found = [(elf, list(_kernels(elf))) for elf in _code_objects(f.read())]
    return [(elf, ks) for elf, ks in found if any(family in k[".name"] for k in ks for family in FAMILIES)]


def test_no_scratch_memory(objects):
    ours = {k[".name"]: k[".private_segment_fixed_size"] for _, ks in objects for k in ks if any(f in k[".name"] for f in FAMILIES)}
    assert {f: sum(f in name for name in ours) for f in FAMILIES} == FAMILIES
    assert not any(ours.values()), ours


@pytest.mark.skipif(OBJDUMP is None, reason="no llvm-objdump")
def test_stores_are_waited_for_before_the_count(objects, tmp_path):
    counted = 0
    for i, (elf, ks) in enumerate(objects):
        if not any("rows_q8_kernel" in k[".name"] for k in ks):
            continue
        path = tmp_path / f"{i}.elf"
        path.write_bytes(elf)
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(path)], check=True, capture_output=True, text=True).stdout
        for name, code in kernels(text).items():
            if "rows_q8_kernel" in name:
                n, faults = unwaited(code)
                assert n == 1 and not faults, (name, n, faults)
                counted += 1
    assert counted == FAMILIES["rows_q8_kernel"]
