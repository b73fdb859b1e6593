"""Loads from memory to LDS in the device code the compiler makes (no GPU needed).

They take their LDS address from m0.  On gfx950 a scalar write of m0 needs one wait state before a load that reads it;
the compiler puts it in where it makes both instructions, but not inside an asm text."""
import os
import re
import subprocess

import pytest

from paper_2607_28633_amd.build import ARCH, INCLUDE, PKG, hipcc

CSRC = os.path.join(PKG, "csrc")
KERNEL = """
#include "attention_mfma.h"
extern "C" __global__ void loads(const char* from, float* to, int n) {
  __shared__ __attribute__((aligned(16))) char s[4][1024];
  topkv_attend::%s(s[n & 1], from + threadIdx.x * 16);
  topkv_attend::%s(s[2 + (n & 1)], from + 4096 + threadIdx.x * 16);
  topkv_attend::wait_loads();
  to[threadIdx.x] = reinterpret_cast<float*>(s[3])[threadIdx.x];
}
"""


@pytest.mark.parametrize("name", ["load_to_lds", "load_once_to_lds"])
def test_m0_has_its_wait_state(tmp_path, name):
    source, out = tmp_path / "loads.hip", tmp_path / "loads.s"
    source.write_text(KERNEL % (name, name))
    r = subprocess.run([hipcc(), f"--offload-arch={ARCH}", "--offload-device-only", "-O3", "-std=c++17", "-S", f"-I{INCLUDE}",
                        f"-I{CSRC}", "-o", str(out), str(source)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    code = [ln.split(";")[0].strip() for ln in out.read_text().splitlines()]
    code = [ln for ln in code if re.match(r"[a-z]\w*(\s|$)", ln)]      # instructions: no labels, directives, comments
    at = [i for i, ln in enumerate(code) if ln.startswith("global_load_lds")]
    assert len(at) == 2
    for i in at:
        assert not re.match(r"s_\w+ m0\b", code[i - 1]), code[i - 1:i + 1]


def test_no_other_loads_to_lds():
    """Every load of this kind goes through the two functions above."""
    for name in sorted(os.listdir(CSRC)):
        with open(os.path.join(CSRC, name)) as f:
            found = len(re.findall(r"(?:global|buffer)_load\w*_lds|raw_ptr_buffer_load_lds", f.read()))
        assert found == (2 if name == "attention_mfma.h" else 0), name
