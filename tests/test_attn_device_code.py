"""Properties of the serving operators' device code that show in the compiled
text alone (no GPU)."""
import os
import re
import subprocess

import pytest

from paper_2606_17787_amd import build

HIPCC = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "bin", "hipcc")

# Loads into the same LDS through the compiler, with one of the library's own
# between them.
PROBE = """
#include "lumen_attn_common.h"
__global__ void probe(const char *from, char *out) {
  __shared__ char lds[2048];
  auto *at = LDS_PTR(char, lds);
  const auto *p =
      (__attribute__((address_space(1))) char *)(from + threadIdx.x * 16);
  __builtin_amdgcn_global_load_lds(p, at, 16, 0, 0);
  lumen_attn_detail::%s;
  __builtin_amdgcn_global_load_lds(p + 4096, at, 16, 0, 0);
  __syncthreads();
  out[threadIdx.x] = lds[threadIdx.x];
}
"""


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="no hipcc")
@pytest.mark.parametrize("call", ["load_to_lds(from, 1024)",
                                  "load_to_lds(from, threadIdx.x * 16, 1024)"])
def test_the_compiler_knows_that_a_load_into_lds_takes_m0(tmp_path, call):
    src = tmp_path / "probe.hip"
    src.write_text(PROBE % call)
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-Werror")]
    text = subprocess.run(
        [HIPCC, *flags, "-I", build.INCLUDE, "-I",
         os.path.join(build.PKG, "csrc"), "--cuda-device-only", "-S",
         str(src), "-o", "-"], capture_output=True, text=True, check=True).stdout
    lines = [l.strip() for l in text.splitlines()
             if re.search(r"\bm0\b|global_load_lds", l)]
    assert sum("global_load_lds" in l for l in lines) == 3, lines
    # each load has its own write of m0 before it
    for i, l in enumerate(lines):
        if "global_load_lds" in l:
            assert re.match(r"s_\w+ m0,", lines[i - 1]), lines
