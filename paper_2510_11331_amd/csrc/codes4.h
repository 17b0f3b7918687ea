// 4-bit format of the cached keys and values, shared by the kernels that write
// the cache (kv4.hip) and the attention that reads it (attention4.hip).
//
// e2m1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6 with signs) with a power-of-two scale
// 2^(E - 127) per block of 32 dimensions of one token and head.  E is the
// smallest E >= 1 with amax <= 6 2^(E - 127): scaling and rounding to a code
// are then functions of the value alone, without a division.  A block with a
// NaN or an infinity, or a value that would be rounded to one (from 1.75 2^127
// on, to 4 2^126), has E = 255, whose scale is an infinity: the conversion
// instruction makes NaN of all 32 codes.
//
// A page holds 16 tokens of one kv head in 17 hd bytes:
//   keys    [16 tokens][hd / 2]: lane (token, g) of a wave reads its hd / 4
//           dimensions (whole or half a scale's block) as one load, and the
//           wave's loads are the page's keys in order;
//   values  [token / 4][16][token % 4][hd / 32 bytes]: lane (r, g) reads
//           dimensions (hd / 16) r .. of tokens 4 g .. 4 g + 3 as one load;
//   scales  of the keys [16 tokens][hd / 32], of the values [hd / 32][16].
// The even dimension of a pair is the low half of its byte.
#pragma once

#include "sd_internal.h"

namespace sd {

typedef float f32x2 __attribute__((ext_vector_type(2)));

template <int HD> struct Page4 {
  static constexpr int KROW = HD / 2;            // bytes of a key
  static constexpr int UNIT = HD / 32;           // bytes of a token in one of its 16 value units
  static constexpr int BLOCKS = HD / 32;         // scales of a token
  static constexpr int V = 8 * HD, KS = 16 * HD, VS = 16 * HD + HD / 2, BYTES = 17 * HD;
  __device__ __forceinline__ static int key(int t, int d) { return t * KROW + d / 2; }
  __device__ __forceinline__ static int value(int t, int r) { return V + ((t / 4 * 16 + r) * 4 + t % 4) * UNIT; }
  __device__ __forceinline__ static int key_scale(int t, int b) { return KS + t * BLOCKS + b; }
  __device__ __forceinline__ static int value_scale(int t, int b) { return VS + b * 16 + t; }
};

// E of a block whose largest magnitude has the given bits (255 from 1.75 2^127 on)
__device__ __forceinline__ uint32_t block_exp4(uint32_t amax) {
  if (amax >= 0x7f600000u) return 255u;
  const int e = (int)((amax + 0x3fffffu) >> 23) - 2;   // the fraction past 1.5 carries
  return (uint32_t)(e < 1 ? 1 : e);
}
__device__ __forceinline__ float scale4(uint32_t E) { return __uint_as_float(E << 23); }

// codes of 8 values, the scale being that of E (v_cvt_scalef32_pk_fp4_f32 divides by it and rounds to nearest even)
__device__ __forceinline__ uint32_t encode4(const float (&x)[8], uint32_t E) {
  if (E == 255u) return 0u;
  const float s = scale4(E);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], s, 3);
  return c;
}
__device__ __forceinline__ void decode4(uint32_t c, float s, float (&x)[8]) {
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 1);
  const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 3);
  x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1];
  x[4] = d[0]; x[5] = d[1]; x[6] = e[0]; x[7] = e[1];
}

// Where the sequences start and end, and their lengths: in LDS for up to PLACES of them, so that looking a row up costs
// one round of memory latency; past that from memory.
constexpr int PLACES = 1024;
struct Places {
  int cu[PLACES + 1], len[PLACES];
  __device__ __forceinline__ void load(const KvRows& s) {
    if (s.B > PLACES) return;
    for (int i = threadIdx.x; i <= s.B; i += blockDim.x) {
      cu[i] = s.cu[i];
      if (i < s.B) len[i] = s.len[i];
    }
  }
};
// Sequence of row r (the last one that starts at or before it) and its
// position; false where r belongs to none.  cu is read within [0, B] whatever
// it holds.
__device__ __forceinline__ bool row_place(const KvRows& s, const Places& at, int r, int& b, int& pos) {
  const bool near = s.B <= PLACES;
  auto cu = [&](int i) { return near ? at.cu[i] : s.cu[i]; };
  if (cu(0) > r || cu(s.B) <= r) return false;
  int lo = 0, hi = s.B;                          // cu[lo] <= r < cu[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu(mid) <= r) lo = mid;
    else hi = mid;
  }
  b = lo;
  const int len = near ? at.len[b] : s.len[b];
  pos = len > 0 ? len - (cu(lo + 1) - r) : -1;   // cu[lo + 1] > r
  return true;
}
// page of a position, or -1
__device__ __forceinline__ int row_page(const KvRows& s, int b, int pos, int n_blocks) {
  if (pos < 0 || pos / 16 >= s.W) return -1;
  const int p = s.table[(size_t)b * s.W + pos / 16];
  return (unsigned)p < (unsigned)n_blocks ? p : -1;
}

}  // namespace sd
