"""The lowest reference of a softmax (``lowest_reference`` in ``csrc/wave_ops.h``), on the CPU: over all
scales it is about as low as a float32 can be, and its product with the scale is finite."""

import shutil
import subprocess

import pytest

from paper_2608_14624_amd import build as _build

SOURCE = r"""
#include "wave_ops.h"
#include <cfloat>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>

int main() {
  // every 61st positive float32, denormal ones and the largest included
  for (uint32_t bits = 1; bits <= 0x7f7fffffu; bits += 61) {
    float c;
    memcpy(&c, &bits, 4);
    const float m = cs::lowest_reference(c);
    const float mc = m * c;
    const bool low = c <= 1.f ? m < -0.999f * FLT_MAX : mc < -0.999f * FLT_MAX;
    if (!std::isfinite(m) || !std::isfinite(mc) || !low) {
      printf("c = %a: m = %a, m c = %a\n", c, m, mc);
      return 1;
    }
  }
  return 0;
}
"""


def test_its_product_with_any_scale_is_finite(tmp_path):
    if shutil.which("hipcc") is None and not shutil.which("/opt/rocm/bin/hipcc"):
        pytest.skip("hipcc not available")
    src, exe = tmp_path / "scan.hip", tmp_path / "scan"
    src.write_text(SOURCE)
    subprocess.run([_build.hipcc(), "--offload-host-only", "-O2", "-std=c++17", "-I", f"{_build.PKG_DIR}/csrc", str(src),
                    "-o", str(exe)], check=True, capture_output=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True, timeout=100)
    assert res.returncode == 0, res.stdout
