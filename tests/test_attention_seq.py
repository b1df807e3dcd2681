"""The attention kernels' row bookkeeping (csrc/attention_seq.h), compiled for the CPU and walked tile by
tile: valid offsets give every row exactly once, whatever else they hold nothing leaves the tensors, and
the mask ranges are the definition's."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

MAIN = r'''
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>
#include "attention_seq.h"
using namespace opfuse;
#define CHECK(c) do { if (!(c)) { printf("line %d: %s\n", __LINE__, #c); exit(1); } } while (0)

int main() {
  std::mt19937 r(7);
  auto pick = [&](int a, int b) { return (int)(a + r() % (unsigned)(b - a + 1)); };
  for (int it = 0; it < 20000; ++it) {
    const int nseq = pick(1, 9), per = pick(1, 9), B = 1 << pick(2, 7);
    const bool offs = pick(0, 3) > 0, lens = pick(0, 1), bad = it % 4 == 3;
    std::vector<int32_t> off(nseq + 1), len(nseq);
    int64_t T = 0;
    if (offs) {
      off[0] = pick(0, 1) ? pick(0, 300) : 0;
      for (int s = 0; s < nseq; ++s) off[s + 1] = off[s] + (pick(0, 2) ? pick(0, 200) : 0);
      T = off[nseq] + pick(0, 50);
      if (T == 0) T = 1;
    } else {
      T = (int64_t)pick(1, 200) * nseq;
    }
    for (auto& n : len) n = pick(0, 250);
    if (bad) {
      for (auto& o : off) if (pick(0, 1)) o = (int32_t)r();
      for (auto& n : len) if (pick(0, 1)) n = (int32_t)r();
    }
    const int32_t* po = offs ? off.data() : nullptr;
    const int32_t* pl = lens ? len.data() : nullptr;
    std::vector<int> seen(T * per, 0), mine(T * per, 0);
    for (int s = 0; s < nseq; ++s) {
      const SeqRows q = seq_rows(po, pl, T, nseq, s);
      CHECK(q.beg >= 0 && q.len >= 0 && q.beg + q.len <= T);
      for (int64_t i = 0; i < (int64_t)q.len * per; ++i) ++mine[q.beg * per + i];
    }
    const int64_t n = attn_tiles(T, nseq, offs, per, B);
    for (int64_t w = 0; w < n; ++w) {
      int s;
      int64_t tile;
      find_tile(po, T, nseq, per, B, w, s, tile);
      CHECK(s >= 0 && s < nseq);
      const SeqRows q = seq_rows(po, pl, T, nseq, s);
      const int64_t R = (int64_t)q.len * per;
      if (tile < 0 || tile >= (R + B - 1) / B) continue;
      for (int64_t x = tile * B; x < R && x < tile * B + B; ++x) ++seen[q.beg * per + x];
    }
    if (!bad) for (size_t x = 0; x < seen.size(); ++x) CHECK(seen[x] == mine[x] && mine[x] <= 1);
  }
  for (int it = 0; it < 3000; ++it) {
    const int nq = pick(0, 40), nk = pick(0, 40), causal = pick(0, 1), window = pick(0, 2) ? 0 : pick(1, 50);
    const int shift = nk - nq;
    for (int i = 0; i < nq; ++i) {
      int lo, hi, lo1, hi1;
      keys_of(causal, window, i, shift, nk, lo, hi);
      CHECK(lo >= 0 && hi >= 0 && lo <= nk && hi <= nk);
      if (i) {
        keys_of(causal, window, i - 1, shift, nk, lo1, hi1);
        CHECK(lo1 <= lo && hi1 <= hi);
      }
      for (int j = 0; j < nk; ++j) {
        const int p = i + shift;
        const bool sees = (!causal || j <= p) && (!window || (j > p - window && (causal || j < p + window)));
        CHECK(sees == (j >= lo && j < hi));
        int ql, qh;
        queries_of(causal, window, j, shift, nq, ql, qh);
        CHECK(sees == (i >= ql && i < qh));
        if (j) {
          int ql1, qh1;
          queries_of(causal, window, j - 1, shift, nq, ql1, qh1);
          CHECK(ql1 <= ql && qh1 <= qh);
        }
      }
    }
  }
  for (int it = 0; it < 2000; ++it) {      // an order takes every number once
    const int n = pick(1, 700), first = pick(1, 300);
    std::vector<int> seen(n, 0);
    for (int b = 0; b < n; ++b) {
      const int64_t x = paired(b, n, first);
      CHECK(x >= 0 && x < n && !seen[x]);
      seen[x] = 1;
    }
  }
  // the largest window and the longest rows stay in range
  int lo, hi;
  keys_of(1, 0x7fffffff, 0x7ffffff0, 0, 0x7fffffff, lo, hi);
  CHECK(lo == 0 && hi == 0x7ffffff1);
  queries_of(0, 0x7fffffff, 0x7ffffff0, -100, 0x7fffffff, lo, hi);
  CHECK(hi == 0x7fffffff);
  printf("ok\n");
}
'''


def test_rows_tiles_and_masks(tmp_path):
    src, exe = tmp_path / "walk.cpp", tmp_path / "walk"
    src.write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-O2", "-fsanitize=undefined", "-fno-sanitize-recover",
                    "-I", os.path.join(ROOT, "paper_2104_00237_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout + out.stderr
