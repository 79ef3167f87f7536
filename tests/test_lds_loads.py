"""The loads that go past the registers to LDS (gemm_stage.h) are assembly that writes m0: a load to LDS of the compiler's own behind one
must set m0 anew.  Shown in the code that the compiler makes of both (no GPU is needed)."""
import os
import re
import subprocess

from paper_2410_05911_amd import build

SOURCE = """#include "gemm_stage.h"
__global__ void k(const void *p, const uint32_t *q, float *out) {
  __shared__ char lds[8192];
  const aecct::BufferOf buffer(p, 4096);
  auto own = [&](int at) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t *)q + at + threadIdx.x,
                                     (__attribute__((address_space(3))) uint32_t *)(lds + 4096), 4, 0, 0);
  };
  own(0);
  buffer.to_lds(lds, threadIdx.x * 16);
  own(64);
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  out[threadIdx.x] = ((float *)lds)[threadIdx.x] + ((float *)lds)[1024 + threadIdx.x];
}
"""


def test_loads_to_lds_leave_no_stale_m0(tmp_path):
    (tmp_path / "two.hip").write_text(SOURCE)
    out = str(tmp_path / "two.s")
    subprocess.run([build.HIPCC, *build.COMMON, *build.DEVICE, "-I", build.CSRC, "--cuda-device-only", "-S",
                    str(tmp_path / "two.hip"), "-o", out], check=True, capture_output=True)
    with open(out) as f:
        steps = [m.group(0) for m in re.finditer(r"\bm0\b(?=,)|buffer_load_dwordx4 .* lds|global_load_lds_dword", f.read())]
    assert steps == ["m0", "global_load_lds_dword", "m0", steps[3], "m0", "global_load_lds_dword"], steps
