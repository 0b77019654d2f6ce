"""The copies from memory into LDS write the register M0 in assembly.  What the compiler keeps in M0 for itself must not be taken
to live across them, which shows in the code that it makes: no GPU is needed."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2411_19379_amd import build as b

PROBE = """
#include <hip/hip_runtime.h>
#include "attn_common.h"
typedef const __attribute__((address_space(1))) void *global_ptr;
typedef __attribute__((address_space(3))) void *lds_ptr;
__device__ __forceinline__ void compilers_own(const void *from, void *to) { __builtin_amdgcn_global_load_lds((global_ptr)from, (lds_ptr)to, 4, 0, 0); }
__global__ void probe(const unsigned char *p, const unsigned char *q, uint4 *out)
{
    extern __shared__ __align__(16) unsigned char lds_raw[];
    compilers_own(q + threadIdx.x * 4, lds_raw + 4096);
    copy16_to_lds(p, threadIdx.x * 16, lds_address(lds_raw));
    compilers_own(q + 1024 + threadIdx.x * 4, lds_raw + 4096);
    copy16_to_lds(p + threadIdx.x * 16, lds_address(lds_raw) + 1024);
    compilers_own(q + 2048 + threadIdx.x * 4, lds_raw + 4096);
    memory_wait();
    __syncthreads();
    out[threadIdx.x] = reinterpret_cast<uint4 *>(lds_raw)[threadIdx.x];
}
"""


def test_the_compiler_knows_that_the_copies_write_m0(tmp_path):
    if not shutil.which("hipcc"):
        pytest.skip("no hipcc")
    src, asm = str(tmp_path / "probe.hip"), str(tmp_path / "probe.s")
    open(src, "w").write(PROBE)
    flags = [f for f in b.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run(["hipcc", *flags, "-I", os.path.join(b._ROOT, "include"), "-I", b.CSRC, "--offload-device-only", "-S", "-o", asm, src],
                   check=True, stderr=subprocess.DEVNULL)
    by_hand, writer, own, copies = False, None, 0, 0
    for line in open(asm):
        by_hand = "#ASMSTART" in line or by_hand and "#ASMEND" not in line
        if re.match(r"\s*s_\w+ m0,", line):
            writer = "copy" if by_hand else "compiler"
        elif re.match(r"\s*global_load_lds_dwordx4 ", line):
            copies += 1
            assert writer == "copy"
        elif re.match(r"\s*global_load_lds_dword ", line):
            own += 1
            assert writer == "compiler", "a load of the compiler's goes where the copy in front of it went"
    assert own == 3 and copies == 2
