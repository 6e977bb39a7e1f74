"""Transfers to LDS that are written in assembly leave the wait states that the compiler does not see there."""
import os
import subprocess

import pytest

import __graft_entry__ as entry
from tests import machine_code

pytestmark = pytest.mark.skipif(not os.path.exists(machine_code.OBJDUMP), reason="no disassembler")

# A scalar operand that comes from a vector register in the instruction before.
KERNELS = """
#include "paged_keys.hpp"
using namespace zc;
__device__ inline uint32_t scalar(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__global__ void k_shared_base(const uint32_t* at, uint32_t lds) {
  const uint32_t lo = at[threadIdx.x], hi = at[threadIdx.x + 64];
  gdma16(lds, (const void*)((uint64_t)scalar(hi) << 32 | scalar(lo)), threadIdx.x * 16);
}
__global__ void k_keys(const uint32_t* at, uint32_t lds) {
  const uint32_t lo = at[threadIdx.x], hi = at[threadIdx.x + 64], n = at[threadIdx.x + 128];
  const int v[2] = {(int)threadIdx.x * 16, (int)threadIdx.x * 16 + 1024};
  move_keys<2>(lds, __builtin_amdgcn_make_buffer_rsrc((void*)((uint64_t)scalar(hi) << 32 | scalar(lo)), 0, scalar(n), kBufFlags), v);
}
"""


def test_transfers_wait_for_their_scalar_operands(tmp_path):
    src, lib = tmp_path / "k.hip", tmp_path / "k.so"
    src.write_text(KERNELS)
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *entry.HIPCC_FLAGS, "-I", os.path.join(entry.ROOT, "include"), "-I", os.path.join(entry.PKG, "csrc"),
                    str(src), "-o", str(lib)], check=True, capture_output=True)
    seen = set()
    for (_, name), code in machine_code.kernels(str(lib)).items():
        if "k_shared_base" in name or "k_keys" in name:
            seen.add(name)
            assert any("readfirstlane" in c[1] for c in code) and any("lds" in c[1] + c[2] for c in code)
            assert not machine_code.too_soon(code)[1], name
    assert len(seen) == 2


@pytest.mark.skipif(not os.path.exists(entry.LIB), reason="not built")
def test_no_memory_instruction_of_the_library_reads_a_scalar_too_soon():
    n = 0
    for name, code in machine_code.kernels(entry.LIB).items():
        some, found = machine_code.too_soon(code)
        n += some
        assert not found, (name, found[:4])
    assert n > 10000
