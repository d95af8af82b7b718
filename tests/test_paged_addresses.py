"""Offsets that the paged attention's transfers are given, by the functions that the kernels use, compiled for the host."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

PROGRAM = r'''
#include "paged_attention.h"
#include <cstdio>
using namespace sdllm;

// Every stride (a multiple of 16 bytes, as the entry point demands) for which the kernels take the offset: it has to be the distance
// itself, less the j KiB that the transfer's instruction adds back, in 32 bits.
template <int D> static bool check(long long& taken) {
  using S = Slab<D>;
  for (long long stride = 0; stride <= 2LL << 27; stride += stride < 8192 ? 16 : (stride >> 3) / 16 * 16) {
    if (!S::strided(stride)) continue;
    ++taken;
    for (int v = 0; v < 2; ++v)
      for (int j = 0; j < S::IPT; ++j)
        for (int lane = 0; lane < 64; ++lane) {
          const int r = S::RPI * j + lane / S::CPR, c = S::at(v, r, lane % S::CPR);
          const long long want = r * stride + 16 * c - 1024LL * j;
          if (c < 0 || c >= S::CPR || want < 0 || want + 1024LL * j + 16 > 15 * stride + S::ROWB ||
              (long long)S::strided_offset(v, lane, j, (unsigned)stride) != want) {
            printf("D %d, rows %lld bytes apart, transfer %d, lane %d: %lld, offset %u\n", D, stride, j, lane, want,
                   S::strided_offset(v, lane, j, (unsigned)stride));
            return false;
          }
        }
  }
  return S::strided(S::ROWB) && S::strided(28 * S::ROWB) && S::strided((1 << 27) - 16);
}

int main() {
  long long taken = 0;
  const bool ok = check<64>(taken) && check<128>(taken);
  printf("%lld strides\n", taken);
  return ok && taken > 500 ? 0 : 1;
}
'''


def test_strided_block_rows_stay_within_the_tensor(tmp_path):
    if shutil.which(HIPCC) is None:
        pytest.skip("no hipcc")
    src, exe = tmp_path / "offsets.hip", str(tmp_path / "offsets")
    src.write_text(PROGRAM)
    csrc = os.path.join(ROOT, "paper_2601_17917_amd", "csrc")
    r = subprocess.run([HIPCC, "--offload-host-only", "--offload-arch=gfx950", "-std=c++17", "-I", csrc, "-I", os.path.join(ROOT, "include"),
                        str(src), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout
