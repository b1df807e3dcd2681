// Which rows an attention workgroup works on: the sequences behind offsets and lengths in device
// memory, their tiles, and the masks as ranges.  Host and device: the host counts tiles, and a test
// walks all of them on the CPU.
#pragma once

#include <stdint.h>

#ifdef __HIP__
#include <hip/hip_runtime.h>
#define OF_HD __host__ __device__ __forceinline__
#else
#define OF_HD inline
#endif

namespace opfuse {

OF_HD int64_t clamp64(int64_t x, int64_t lo, int64_t hi) { return x < lo ? lo : x > hi ? hi : x; }

// Row strides are at most this many elements: a tile's loads count bytes from its first row in 32 bits
// (64 rows of 2-byte or 32 of 4-byte elements: below 2^30), and columns behind the width are sent to
// offset 2^31, which has to lie behind the tile's last row.
constexpr int64_t kRowStrideMax = 1LL << 22;

// Strides of dO's rounded copy in a backward's workspace: head after head, so that the row stride does
// not grow with the heads (with rows of all heads, H D = 2^26 would wrap the loads' 32 bits at row 32).
// Row t of head h is row h T + t, as in the row statistics.
OF_HD void copy_strides(int64_t T, int D, int64_t& ld, int64_t& hs) {
  ld = D;
  hs = T * D;
}

// Rows [beg, beg + len) of a sequence.  Offsets and lengths come from device memory the host has
// not seen: whatever they hold, the result lies inside [0, T).
struct SeqRows {
  int64_t beg;
  int len;
};
OF_HD SeqRows seq_rows(const int32_t* off, const int32_t* len, int64_t T, int nseq, int s) {
  int64_t b, e;
  if (off) {
    b = clamp64(off[s], 0, T);
    e = clamp64(off[s + 1], b, T);
  } else {
    const uint32_t slot = (uint32_t)T / (uint32_t)nseq;   // T < 2^31
    b = (int64_t)s * slot;
    e = b + slot;
  }
  return SeqRows{b, (int)(len ? clamp64(len[s], 0, e - b) : e - b)};
}

// Tiles of B rows (each row counted `per` times) of all sequences, numbered so that a tile's
// sequence is found from the offsets alone: sequence s begins at tile floor(off[s] per / B) + s,
// which leaves every sequence at least ceil(len per / B) numbers.  The host launches attn_tiles() of
// them; a number past a sequence's rows has nothing to do.
OF_HD int64_t attn_tiles(int64_t T, int nseq, bool offsets, int per, int B) {
  return offsets ? T * per / B + nseq : (T / nseq * per + B - 1) / B * nseq;
}
OF_HD void find_tile(const int32_t* off, int64_t T, int nseq, int per, int B, int64_t w, int& s, int64_t& tile) {
  if (!off) {   // equal slots: tile by tile, so that tiles of one length lie together
    const uint32_t t = (uint32_t)w / (uint32_t)nseq;   // (a grid has fewer than 2^31 workgroups)
    tile = t;
    s = (int)((uint32_t)w - t * (uint32_t)nseq);
    return;
  }
  int lo = 0, hi = nseq;   // the last s whose first tile is <= w
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (clamp64(off[mid], 0, T) * per / B + mid <= w) lo = mid; else hi = mid;
  }
  s = lo;
  tile = w - (clamp64(off[lo], 0, T) * per / B + lo);
}

// Order of n workgroups of different lengths.  Two of them run on a CU at a time, the second wave's b + 256
// beside b: where no more than that many are launched, the second half is taken from its end, so that
// with the longest first the shortest joins the longest.
OF_HD int64_t paired(int64_t b, int64_t n, int64_t first) {
  return n <= 2 * first && b >= first ? n - 1 - (b - first) : b;
}

// Keys [lo, hi) that query i of a sequence sees (none where hi <= lo); nk keys, shift = nk - nq.  Both
// ends grow with i, so of queries i .. i' the keys lo(i) .. hi(i') hold every pair and lo(i') .. hi(i)
// have no masked one.
OF_HD void keys_of(int causal, int window, int i, int shift, int nk, int& lo, int& hi) {
  const int64_t p = (int64_t)i + shift;
  hi = (int)clamp64(causal ? p + 1 : window ? p + window : nk, 0, nk);
  lo = (int)clamp64(window ? p - window + 1 : 0, 0, nk);
}
// Queries [lo, hi) that see key j: the same relation from the other side.
OF_HD void queries_of(int causal, int window, int j, int shift, int nq, int& lo, int& hi) {
  const int64_t p = (int64_t)j - shift;
  lo = (int)clamp64(causal ? p : window ? p - window + 1 : 0, 0, nq);
  hi = (int)clamp64(window ? p + window : nq, 0, nq);
}

}  // namespace opfuse
