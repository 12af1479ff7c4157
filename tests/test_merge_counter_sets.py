"""Which streams get arrival counters for a merge inside their kernels: the library's own choice, compiled for the host with stand-ins for
the runtime's calls.  Two launches that can overlap must never share a set."""
import os
import re
import subprocess

import pytest

import paper_2405_03917_amd as cq

SOURCE = os.path.join(os.path.dirname(cq.__file__), "csrc", "cq_decode.hip")

STAND_INS = r"""
#include <cstddef>
#include <cstdint>
#include <mutex>
#include <set>
typedef struct stream_t* hipStream_t;
enum hipError_t { hipSuccess, hipErrorUnknown };
enum hipStreamCaptureStatus { hipStreamCaptureStatusNone, hipStreamCaptureStatusActive };
#define hipStreamPerThread ((hipStream_t)2)
#define HIP_SYMBOL(x) (&x)
constexpr int kMergeRows = 64, kMergeSets = 4;
unsigned merge_counters[kMergeRows * kMergeSets];
bool capturing = false;
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s) { *s = capturing ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone; return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipGetSymbolAddress(void** p, unsigned (*x)[kMergeRows * kMergeSets]) { *p = x; return hipSuccess; }
"""

CHECKS = r"""
int main()
{
    MergeCounters c;
    const auto stream = [](uintptr_t x) { return reinterpret_cast<hipStream_t>(x); };
    if (c.for_stream(hipStreamPerThread, 1)) return 1;                  // another stream in every host thread
    if (c.for_stream(stream(0x100), kMergeRows + 1)) return 2;
    capturing = true;
    if (c.for_stream(stream(0x100), 1)) return 3;
    capturing = false;
    std::set<unsigned*> sets;
    for (uintptr_t s : {0x0, 0x100, 0x200, 0x300}) {
        unsigned* p = c.for_stream(stream(s), kMergeRows);
        if (!p || p < merge_counters || p + kMergeRows > merge_counters + kMergeRows * kMergeSets || c.for_stream(stream(s), 1) != p) return 4;
        sets.insert(p);
    }
    if (sets.size() != 4) return 5;
    if (c.for_stream(stream(0x400), 1)) return 6;                       // no set left
    return c.for_stream(hipStreamPerThread, 1) ? 7 : 0;
}
"""


def test_no_two_streams_share_a_set(tmp_path):
    with open(SOURCE) as f:
        struct = re.search(r"^struct MergeCounters \{.*?^\};$", f.read(), re.S | re.M).group(0)
    src, exe = tmp_path / "sets.cpp", tmp_path / "sets"
    src.write_text(STAND_INS + struct + CHECKS)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-pthread", "-o", str(exe), str(src)], check=True)
    assert subprocess.run([str(exe)], timeout=60).returncode == 0


@pytest.mark.parametrize("name", sorted(x for x in os.listdir(os.path.dirname(SOURCE)) if x.endswith((".hip", ".hpp"))))
def test_sets_are_handed_out_in_one_place(name):
    with open(os.path.join(os.path.dirname(SOURCE), name)) as f:
        text = f.read()
    assert name == "cq_decode.hip" or "for_stream" not in text
