"""Strides inside the attention kernels' workspace (csrc/attention_seq.h), compiled for the CPU: the copy of
dO that a backward with fp32 gradients of bf16 operands keeps is read by the same tile loads as the
caller's tensors, and has to stay within the row strides those count in 32 bits."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

MAIN = r'''
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "attention_seq.h"
using namespace opfuse;
#define CHECK(c) do { if (!(c)) { printf("line %d: %s\n", __LINE__, #c); exit(1); } } while (0)

int main() {
  // every head count, row count and width that a call can have: H T <= 2^31 - 1024
  for (int D : {1, 7, 64, 72, 128, 256})
    for (int64_t H = 1; H <= (1LL << 30); H *= 2)
      for (int64_t T : {int64_t(1), int64_t(64), int64_t(((1LL << 31) - 1024) / H)}) {
        if (T < 1 || H * T > (1LL << 31) - 1024) continue;
        int64_t ld, hs;
        copy_strides(T, D, ld, hs);
        CHECK(ld >= D && ld <= kRowStrideMax);
        for (int rows : {32, 64}) {      // bytes to a tile's last element, in the kernels' types
          const int64_t last = ((rows - 1) * ld + D) * (rows == 32 ? 4 : 2);
          CHECK(last < (1LL << 31) && (int)last == last && (uint32_t)((rows - 1) * ld * 4) == (rows - 1) * ld * 4);
        }
        CHECK((T - 1) * ld + (H - 1) * hs + D == T * H * D);     // inside the copy, to its end
      }
  for (int64_t H = 1; H < 5; ++H)         // no two elements at one place
    for (int64_t T = 1; T < 6; ++T) {
      const int D = 3;
      int64_t ld, hs;
      copy_strides(T, D, ld, hs);
      std::vector<int> seen(H * T * D, 0);
      for (int64_t t = 0; t < T; ++t)
        for (int64_t h = 0; h < H; ++h)
          for (int d = 0; d < D; ++d) CHECK(!seen[t * ld + h * hs + d]++);
    }
  printf("ok\n");
}
'''


def test_copy_of_dout(tmp_path):
    src, exe = tmp_path / "copy.cpp", tmp_path / "copy"
    src.write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", os.path.join(ROOT, "paper_2104_00237_amd", "csrc"), str(src),
                    "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout + out.stderr
