"""The weights that sampling adds up (csrc/kd_weight.hpp, compiled for the host), by rows' largest entries from the smallest to the largest magnitudes:
each against exp in extended precision, and none above what a chunk's sum has room for."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include "%s/paper_2603_01875_amd/csrc/kd_weight.hpp"
#include <stdio.h>
#include <float.h>
using namespace kd;
static int bad(const char* what, float top, float tau, float z, double w) {
  printf("%%s: top %%a tau %%a z %%a w %%a\n", what, top, tau, z, w);
  return 1;
}
int main() {
  const float bf16_most = 0x1.fep127f;
  const float tops[] = {0.f, 1e-30f, -1e-30f, 3.f, -3.f, 255.9f, 256.f, -256.1f, 500.f, -1000.f, 12345.f, -1e6f, 1e7f, 1e10f, -1e13f, 1e16f, -1e18f, 1e20f, -1e20f,
                        1e30f, -1e30f, FLT_MAX, -FLT_MAX, bf16_most, -bf16_most};
  const float taus[] = {1e-6f, 1e-3f, 0.7f, 1.f, 3.f, 1e3f, 1e6f};
  for (float top : tops)
    for (float tau : taus) {
      const double scale = kLog2e / (double)tau;
      const Exponents e = exponents_of(top, scale);
      uint64_t sum = 0;
      auto check = [&](float z) {
        const double w = weight(exponent(e, z));
        const long double want = exp2l(((long double)z - top) * 1.44269504088896340735992468100189214L / tau);
        // the polynomial 2^-39.7, the exponent's own roundings (scale and product, of at most 80) 3 80 2^-53, zero's 2^-46; what is below 2^-80 counts as that
        if (!(w >= 0 && w <= 1 + 0x1p-44)) return bad("range", top, tau, z, w);
        if (!(fabsl((long double)w - want) <= 0x1p-39L * want + 0x1p-79L)) return bad("value", top, tau, z, w);
        sum += whole_one(w, 0x1p48);
        return 0;
      };
      if (weight(exponent(e, top)) < 1 - 0x1p-44) return bad("largest", top, tau, top, 0);
      float z = top;
      for (int i = 0; i < 300 && z >= -FLT_MAX; ++i, z = nextafterf(z, -INFINITY))      // the next floats below
        if (check(z)) return 1;
      for (int i = 0; i < 3000; ++i) {                                                     // and what lies up to 100 units below
        const float y = (float)((double)top - 100. / 3000 * i * tau);
        if (y <= top && y >= -FLT_MAX && check(y)) return 1;
      }
      if (check(-FLT_MAX)) return 1;
      const double none = weight(exponent(e, -INFINITY));
      if (!(none >= 0 && none <= 0x1p-79)) return bad("minus infinity", top, tau, 0, none);
      if (sum < (uint64_t)1 << 47) return bad("sum", top, tau, top, (double)sum);
      // a chunk's sum at the row's largest entry: that entry's own is what it was
      if (rescale(top, top, scale) != 1) return bad("rescale", top, tau, top, 0);
      if (!(rescale(-FLT_MAX, top, scale) >= 0 && rescale(-FLT_MAX, top, scale) <= 1)) return bad("rescale", top, tau, -FLT_MAX, 0);
    }
  return 0;
}
"""


def test_weights(tmp_path):
    src, exe = tmp_path / "w.cpp", tmp_path / "w"
    src.write_text(PROGRAM % ROOT)
    subprocess.run(["g++", "-std=c++17", "-O2", "-ffp-contract=off", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout
