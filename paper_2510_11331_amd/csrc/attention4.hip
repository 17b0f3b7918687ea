// Attention over a paged KV cache held in 4 bits (format: codes4.h):
//   o = sum_j softmax_j(scale q . k_j) v_j
// over the positions j that a row sees: up to its own (causal), or all of its
// sequence's.
//
// A query vector is one head of one row; the G = H / KV heads of a kv head and
// all rows of a sequence are one run of vectors that share its keys.  A
// workgroup takes up to 16 QT vectors of such a run and a range of its keys.
//
// S^T = K Q^T and O^T += V^T P^T on v_mfma_f32_16x16x32_bf16.  A code times its
// scale is a bf16 number (two significant bits; scales of 2^-126 to 2^126), so
// v_cvt_scalef32_pk_bf16_fp4 loses nothing, and neither do the products with
// bf16 queries.  fp32 queries enter as three bf16 parts (all 24 bits).  Weights
// enter as two for bf16 outputs, off by at most 2^-15 of themselves where the
// output's own rounding is 2^-8, and as three (exact) for fp32 ones (the prefill
// kernel's: below).  Scores, the running maximum, the weights' sum and the output
// are fp32.
//
// Why matrix instructions for one row of keys: 16 query vectors cost as much as
// one, and there the conversion of the codes, which everything needs, is the
// larger part; the vector unit's own products would add to it.
//
// A wave takes 32 keys (two pages) at a time.  Lane (r, g) = (lane % 16, lane /
// 16) loads key r's dimensions (hd / 4) g .. as they lie in the page: they are
// whole or half a scale's block, and the order in which the k-steps of the
// matrix instruction take dimensions is free as long as the queries follow it.
// S^T leaves query r's scores of keys 4 g .. 4 g + 3 of both pages in the lane,
// which is the order in which P^T enters the second product if V^T's k index
// runs over the same keys: so a lane loads the values of these eight, and
// nothing crosses lanes.  Of the values it takes dimensions (hd / 16) r .., one
// scale per key; output tile t has the dimensions t of each such group.  What the
// conversion leaves in pairs of dimensions of a key becomes pairs of keys of a
// dimension by byte permutes.
//
// The running maximum moves only when a score passes it by 2^8: the weights stay
// far inside fp32, and the usual step needs neither a reduction over lanes nor
// a rescaling of the output.
//
// Measured (a call in a replayed graph; the plain read rate of this memory is 6.8
// TB/s, a large bf16 product runs at 1.57 PFLOP/s):
//   64 sequences of 8192 keys, a row of 32 heads on 8, hd 128, bf16: 95 us, 6.0 TB/s
//   8 sequences of 1044 keys, 5 rows of 32 heads on 32, bf16: 11.4 us, 3.3 TB/s
//   32 ragged ones up to 2176 keys, 5 rows of 32 heads on 32, fp32: 29.1 us
//   1 of 32763 keys, 5 rows of 32 heads on 8, bf16: 21.9 us (16.5 and the join 5)
//   1 of 520 keys, a row of 32 heads on 8, hd 64: 6.3 us
//   2048 rows on 4095 keys, 32 heads on 32, bf16: 111 us, 0.93 PFLOP/s
// Short calls are bound by the chain of latencies (the sequence, its page ids,
// the pages, the waves' join): 5 us whatever their size.  fp32 ones of few rows by
// the instructions of three parts of queries and of weights (vector units 0.57,
// matrix units 0.24 of the cycles).  Decoding at length by memory.  Prefill by no
// unit alone (below).
#include "codes4.h"

#include <float.h>
#include <limits.h>
#include <math.h>

#include <algorithm>
#include <utility>

namespace sd {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x4 mfma_bf16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma_f16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <int E, bool F16 = false> __device__ __forceinline__ uint32_t cvt4(uint32_t c, float s) {   // byte E
  if constexpr (F16) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, s, E));
  else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, E));
}
__device__ __forceinline__ u32x4 cvt4_all(uint32_t c, float s) {
  return u32x4{cvt4<0>(c, s), cvt4<1>(c, s), cvt4<2>(c, s), cvt4<3>(c, s)};
}
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
}

// over the four lanes that share lane % 16
__device__ __forceinline__ float quad_max(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const uint32_t w = __float_as_uint(v);
  const auto b = __builtin_amdgcn_permlane16_swap(w, w, false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float quad_sum(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const uint32_t w = __float_as_uint(v);
  const auto b = __builtin_amdgcn_permlane16_swap(w, w, false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// 8 floats as PARTS bf16 operands whose sum they are: all but the last are cut, the last is rounded
template <int PARTS> __device__ __forceinline__ void parts8(const float (&x)[8], u32x4 (&o)[PARTS]) {
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = x[e];
#pragma unroll
  for (int k = 0; k < PARTS; ++k)
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      if (k < PARTS - 1) {
        o[k][e / 2] = high_halves(__float_as_uint(r[e]), __float_as_uint(r[e + 1]));
        r[e] -= __uint_as_float(__float_as_uint(r[e]) & 0xffff0000u);
        r[e + 1] -= __uint_as_float(__float_as_uint(r[e + 1]) & 0xffff0000u);
      } else {
        o[k][e / 2] = pack_bf16(r[e], r[e + 1]);
      }
    }
}

// The vectors of workgroup `block`: sequence b, its first row, its rows n and the first of its vectors.
struct Block4 { int b, row0, n, v0, len; };
// Up to 64 sequences: sequence b has ceil(n G / cap) workgroups, which every wave adds up by itself, in the order of the
// sequences or, sorted, the longest first.
// More (a sum of all of them in each workgroup would cost as much as the attention does: 64 keys of 512 sequences 32 us,
// of 4096 sequences 786 us; so 25 and 198): with u = gcd(G, cap) and C = cap / u, sequence b's workgroups are those from S(b) =
// floor((cu[b] G / u + (C - 1) min(b, cu[b])) / C) on.  Where n >= 1 the minimum grows by at least one, so that S(b + 1) - S(b) >=
// floor((n G / u - 1) / C) + 1 = ceil(n G / cap): they suffice, the few between its last and S(b + 1) have nothing to do, and
// sequences without rows cost none but those.  A wave looks at 64 values of S at a time.
constexpr int SUMMED = 64;
__host__ __device__ constexpr int common4(int a, int b) {
  while (b) {
    const int r = a % b;
    a = b;
    b = r;
  }
  return a;
}
__device__ __forceinline__ bool find_block(const KvRows& s, int M, int G, int cap, int block, bool sorted, Block4& o) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = 0, len = 0;                   // of a lane's sequence
  int at, before;                                // the lane that has the workgroup's, and that one's workgroups before this
  if (s.B <= SUMMED) {
    if (lane < s.B) {
      lo = min(max(s.cu[lane], 0), M);
      hi = min(max(s.cu[lane + 1], lo), M);
      len = s.len[lane];                         // (of all of them: not a second round of latency)
    }
    int b = lane;
    if (sorted) {
      const int keys = min(max(len, 0), 1 << 24), near = __builtin_amdgcn_readfirstlane(keys);
      if (__any(lane < s.B && abs(keys - near) > near / 4)) {         // lane k takes the sequence that k longer ones go before
        const int key = lane < s.B ? keys * 64 + 63 - lane : -1 - lane;
        int rank = 0;
#pragma unroll 16
        for (int j = 0; j < 64; ++j) rank += __builtin_amdgcn_readlane(key, j) > key;
        lo = __builtin_amdgcn_ds_permute(4 * rank, lo);
        hi = __builtin_amdgcn_ds_permute(4 * rank, hi);
        len = __builtin_amdgcn_ds_permute(4 * rank, len);
        b = __builtin_amdgcn_ds_permute(4 * rank, lane);
      }
    }
    const int mine = ((hi - lo) * G + cap - 1) / cap;
    int sum = mine;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
      const int up = __shfl_up(sum, k);
      if (lane >= k) sum += up;
    }
    const uint64_t past = __ballot(sum > block);
    if (!past) return false;
    at = __builtin_ctzll(past);
    before = block - (__builtin_amdgcn_readlane(sum, at) - __builtin_amdgcn_readlane(mine, at));
    o.b = __builtin_amdgcn_readlane(b, at);
  } else {
    const int u = common4(cap, G), C = cap / u;
    int b0 = 0, b1 = s.B, step, start;           // S(b0) <= block < S(b1), where the workgroup is any sequence's
    do {
      step = (b1 - b0 + 63) / 64;
      const int b = b0 + step * lane;
      start = INT_MAX;
      if (b < b1) {
        lo = min(max(s.cu[b], 0), M);
        hi = min(max(s.cu[b + 1], lo), M);
        len = s.len[b];
        start = (int)(((int64_t)lo * (G / u) + (int64_t)(C - 1) * min(b, lo)) / C);
      }
      const uint64_t past = __ballot(start > block);
      at = past ? __builtin_ctzll(past) - 1 : 63;
      if (at < 0) return false;
      b0 += step * at;
      b1 = min(b1, b0 + step);
    } while (step > 1);
    before = block - __builtin_amdgcn_readlane(start, at);
    o.b = b0;
  }
  o.row0 = __builtin_amdgcn_readlane(lo, at);
  o.n = __builtin_amdgcn_readlane(hi, at) - o.row0;
  o.len = __builtin_amdgcn_readlane(len, at);
  o.v0 = before * cap;
  return before < (o.n * G + cap - 1) / cap;
}

// keys that vector v of a sequence sees
__device__ __forceinline__ int sees(const Attn4Params& p, int len, int n, int v, int G) {
  return len <= 0 ? 0 : p.causal ? len - n + v / G + 1 : len;     // (not positive: none)
}
// keys of one of p.splits ranges, of n in all, in a workgroup that takes `unit` at a time
__device__ __forceinline__ int range_keys(int n, int splits, int unit) {
  const int k = (int)(((int64_t)n + splits - 1) / splits);
  return (k + unit - 1) / unit * unit;
}
// positions behind the table have no page: the first of them makes NaN of what sees it
__device__ __forceinline__ int loop_keys(const Attn4Params& p, int n) { return min(n, 16 * p.rows.W + 16); }

template <typename T> __device__ __forceinline__ void store4(T* p, f32x4 x) {
  if constexpr (sizeof(T) == 2) *(u32x2*)p = u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
  else *(f32x4*)p = x;
}

template <int HD> struct Load4;            // what a lane has of a page's keys or values
template <> struct Load4<128> { typedef u32x4 type; };
template <> struct Load4<64> { typedef u32x2 type; };

// A page of one head as a buffer: its address is the wave's, a lane's offset within it does not change from page to
// page, so that a load costs no vector arithmetic.
template <int HD> __device__ __forceinline__ __amdgpu_buffer_rsrc_t page_buffer(const uint8_t* pg) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(pg), (short)0, Page4<HD>::BYTES, 0x00020000);
}
template <typename V, bool NT = false> __device__ __forceinline__ V page_load(__amdgpu_buffer_rsrc_t b, uint32_t off) {
  constexpr int AUX = NT ? 2 : 0;                // 2: non-temporal
  if constexpr (sizeof(V) == 16) return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b128(b, off, 0, AUX));
  else if constexpr (sizeof(V) == 8) return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b64(b, off, 0, AUX));
  else if constexpr (sizeof(V) == 4) return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b32(b, off, 0, 0));
  else return __builtin_amdgcn_raw_buffer_load_b8(b, off, 0, 0);
}
// every wave's LDS accesses are done; loads from memory stay in flight
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// parts of a query, and of a weight that meets bf16 values
template <typename T> constexpr int QUERY_PARTS = sizeof(T) == 2 ? 1 : 3;
template <typename T> constexpr int WEIGHT_PARTS = sizeof(T) == 2 ? 2 : 3;

// a vector's query as operands: lane (r, g) has dimensions (hd / 4) g + 8 s .. in k-step s
template <typename T, int HD>
__device__ __forceinline__ void load_query(const T* src, bool negative, u32x4 (&q)[HD / 32][QUERY_PARTS<T>]) {
#pragma unroll
  for (int s = 0; s < HD / 32; ++s) {
    if constexpr (sizeof(T) == 2) {
      q[s][0] = ((const u32x4*)src)[s];
      if (negative) q[s][0] ^= 0x80008000u;
    } else {
      const f32x4 a = ((const f32x4*)src)[2 * s], b = ((const f32x4*)src)[2 * s + 1];
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = negative ? -(e < 4 ? a[e] : b[e - 4]) : e < 4 ? a[e] : b[e - 4];
      parts8<QUERY_PARTS<T>>(x, q[s]);
    }
  }
}

// A weight's logarithm is z c - m of one rounding, m the rounded z c of a maximum (less UP).  m's own rounding is the same for
// all weights; up to |m| = FAR it is at most 4, small against their range.  Past 2^32 it would take the largest weight out of
// fp32's, past 2^29 out of fp16's: from FAR on the product is rounded as m's was, and the largest key's weight is 1 again.
// (There neighbouring floats z lie 8 apart in z c, so that this is the scores' own rounding; from 2^20 on, tried first, it
// took bits from scores that are close.)
constexpr float FAR = 134217728.f;
// What a step's largest logarithm may be before the maximum moves: 8 more than the maximum's own, UP, and with a far m in the
// wave nothing.  (As the bits of a float: 8, 15.)
constexpr int FAR_LIMIT = -1;
template <int UP> constexpr int NEAR_LIMIT = UP ? 0x41700000 : 0x41000000;
// Scores z of keys key .. key + 3 and key + 16 .. key + 19 -> the logarithms x of their weights, with the running maxima
// m, and what goes with these: the weights' sums l and the outputs o.  edge: vector t sees the keys below vis[t] only.
// UP: m is so much below the maximum, 0 or 7.
template <int UP, int QT, int DT, typename L>
__device__ __forceinline__ void weigh(bool edge, const f32x4 (&z)[QT][2], float c, int key, const int (&vis)[QT], float (&m)[QT],
                                      int& limit, L (&l)[QT], f32x4 (&o)[QT][DT], float (&x)[QT][8]) {
  auto over = [&](int t, bool far) {             // in powers of two over the maximum
#pragma clang fp contract(off)
#pragma unroll
    for (int e = 0; e < 8; ++e) x[t][e] = far ? z[t][e / 4][e % 4] * c - m[t] : fmaf(z[t][e / 4][e % 4], c, -m[t]);
    if (edge) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (key + 16 * (e / 4) + e % 4 >= vis[t]) x[t][e] = -INFINITY;
    }
  };
  // (as integers: negative numbers below all others, NaN above)
  int top = 0;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    over(t, false);
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_int(x[t][e]));
  }
  if (__any(top > limit)) {
    bool any_far = false;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      float most = -FLT_MAX;
#pragma unroll
      for (int e = 0; e < 8; ++e) most = fmaxf(most, x[t][e] == -INFINITY ? -FLT_MAX : z[t][e / 4][e % 4] * c);
      const float to = fmaxf(m[t], quad_max(most) - UP), old = __builtin_amdgcn_exp2f(m[t] - to);
      m[t] = to;
      l[t] *= old;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[t][d] *= old;
      const bool far = fabsf(to) >= FAR;
      over(t, far);
      any_far |= far && to > -FLT_MAX;           // (the maximum of nothing yet)
    }
    limit = __any(any_far) ? FAR_LIMIT : NEAR_LIMIT<UP>;
  }
}
__device__ __forceinline__ void exp8(float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = __builtin_amdgcn_exp2f(x[e]);
}
__device__ __forceinline__ float sum8(const float (&x)[8]) {
  return ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
}

// Two pages' values as a lane loads them (codes c, scales E) -> operands of tiles 2 B and 2 B + 1.  Byte B of a key holds
// dimensions 2 B and 2 B + 1 of the lane's: pairs of dimensions of a key become pairs of keys of a dimension.
template <int HD, int B, int PAGES, bool F16 = false>
__device__ __forceinline__ void value_tiles(const typename Load4<HD>::type (&c)[PAGES], const float (&s)[PAGES][4],
                                            uint32_t (&even)[2 * PAGES], uint32_t (&odd)[2 * PAGES]) {
#pragma unroll
  for (int e = 0; e < 2 * PAGES; ++e) {
    const int t = e / 2, k = 2 * (e % 2);
    uint32_t a, b;
    if constexpr (HD == 128) {
      a = cvt4<B, F16>(c[t][k], s[t][k]);
      b = cvt4<B, F16>(c[t][k + 1], s[t][k + 1]);
    } else {
      a = cvt4<B, F16>(c[t][k / 2], s[t][k]);
      b = cvt4<B + 2, F16>(c[t][k / 2], s[t][k + 1]);
    }
    even[e] = low_halves(a, b);
    odd[e] = high_halves(a, b);
  }
}
template <int PAGES> __device__ __forceinline__ void value_scales(const uint32_t (&E)[PAGES], float (&s)[PAGES][4]) {
#pragma unroll
  for (int t = 0; t < PAGES; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) s[t][e] = scale4(__builtin_amdgcn_ubfe(E[t], 8 * e, 8));
}

// o += the step's values, of two pages in registers, times the weights
template <int HD, int QT, int PP>
__device__ __forceinline__ void add_values(const typename Load4<HD>::type (&c)[2], const uint32_t (&E)[2],
                                           const u32x4 (&w)[QT][PP], f32x4 (&o)[QT][HD / 16]) {
  float s[2][4];
  value_scales(E, s);
  [&]<int... B>(std::integer_sequence<int, B...>) {
    (([&] {
       uint32_t even[4], odd[4];
       value_tiles<HD, B>(c, s, even, odd);
       const u32x4 a{even[0], even[1], even[2], even[3]}, b{odd[0], odd[1], odd[2], odd[3]};
#pragma unroll
       for (int u = 0; u < QT; ++u)
#pragma unroll
         for (int part = PP - 1; part >= 0; --part) {
           o[u][2 * B] = mfma_bf16(a, w[u][part], o[u][2 * B]);
           o[u][2 * B + 1] = mfma_bf16(b, w[u][part], o[u][2 * B + 1]);
         }
     }()),
     ...);
  }(std::make_integer_sequence<int, HD / 32>{});
}

// Values that not every vector sees must be finite: their weights are zero where they are not seen.  Scales of keys behind
// the last (key: the lane's first) and of pages that are none (no) become 1; whether there is one of 253 or more among the
// others, whose codes may be infinities or NaN.
__device__ __forceinline__ bool clean_scales(uint32_t (&E)[2], int key, int n_max, uint32_t no) {
  uint32_t large = 0;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (key + 16 * t + e >= n_max || (no >> t & 1)) E[t] = (E[t] & ~(255u << (8 * e))) | 127u << (8 * e);
    large |= ((E[t] & 0x7f7f7f7fu) + 0x03030303u) & E[t] & 0x80808080u;      // (four bytes at once)
  }
  return large != 0;
}
// Of these, NaN (255) becomes a number; put_nan puts it into the outputs of the vectors that see it.  Codes whose numbers are
// infinities (4 and 6 with E = 253, 2 to 6 with E = 254; nothing writes them) become the largest number that is none: 3 or
// 1.5, both the odd code below the first.  Whether there was a NaN.
template <int HD> __device__ __forceinline__ bool clean_codes(typename Load4<HD>::type (&c)[2], uint32_t (&E)[2]) {
  bool nan = false;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t E8 = E[t] >> (8 * e) & 255u;
      const uint32_t w = c[t][HD == 128 ? e : e / 2];
      const uint32_t mine = HD == 128 ? 0x11111111u : 0x1111u << (16 * (e % 2));
      const uint32_t inf = (E8 == 253u ? w >> 2 & w >> 1 : E8 == 254u ? w >> 2 : 0u) & mine;
      c[t][HD == 128 ? e : e / 2] = (w & ~(7u * inf)) | inf * (E8 == 253u ? 5u : 3u);
      if (E8 == 255u) E[t] ^= 128u << (8 * e);
      nan |= E8 == 255u;
    }
  return nan;
}
// the value blocks of NaN among the step's keys; all of a lane's outputs are of scale block (hd / 4) g / 32
template <int HD, int QT>
__device__ __forceinline__ void put_nan(const uint8_t* const (&pages)[2], uint32_t no, int key0, int n_max, int g,
                                        const int (&vis)[QT], f32x4 (&o)[QT][HD / 16]) {
  for (int key = key0; key < min(key0 + 32, n_max); ++key) {
    const int t = key - key0 >= 16;
    if ((no >> t & 1) || pages[t][Page4<HD>::value_scale(key & 15, g * (HD / 4) / 32)] != 255) continue;
#pragma unroll
    for (int u = 0; u < QT; ++u)
      if (key < vis[u])
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) o[u][d] = f32x4{NAN, NAN, NAN, NAN};
  }
}

// A joined vector's four dimensions: the output itself, or a range's part of it
template <typename T, int HD>
__device__ __forceinline__ void emit(const Attn4Params& p, int split, int row, int h, int d, bool sees_any, float M, float L, f32x4 O) {
  if (p.splits == 1) {
    if (!sees_any) O = f32x4{0.f, 0.f, 0.f, 0.f};
    else O *= 1.f / L;
    store4((T*)p.out + (size_t)row * p.ldo + h * HD + d, O);
  } else {
    const size_t at = ((size_t)split * p.M + row) * p.H + h;
    *(f32x4*)(p.part_o + at * HD + d) = O;
    // (a sum of -1: of nothing to see, which the joined output is zero for)
    if (d == 0) *(float2*)(p.part_ml + 2 * at) = sees_any ? make_float2(M, L) : make_float2(0.f, -1.f);
  }
}
// a range without keys
__device__ __forceinline__ void emit_nothing(const Attn4Params& p, int split, int row, int h, bool sees_any) {
  *(float2*)(p.part_ml + 2 * (((size_t)split * p.M + row) * p.H + h)) = sees_any ? make_float2(-FLT_MAX, 0.f) : make_float2(0.f, -1.f);
}

// A wave's keys first .. first + 31, from there on each `stride` further, up to `end`: the scores of its vectors q (of
// which all see n_min keys, vector r of tile t vis[t], and none more than n_max), their weights, and the values times these.
// FULL: steps that all vectors see whole are taken by code without masks.  guessed: guess_id is the lane's first page id.
template <typename T, int HD, int QT, bool FULL, bool NT>
__device__ __forceinline__ void take_keys(const Attn4Params& p, int kvh, int b, int first, int stride, int end, int n_min, int n_max,
                                          const u32x4 (&q)[QT][HD / 32][QUERY_PARTS<T>], float c, const int (&vis)[QT],
                                          float (&m)[QT], float (&l)[QT], f32x4 (&o)[QT][HD / 16], bool guessed, int guess_id) {
  using P = Page4<HD>;
  using L4 = typename Load4<HD>::type;
  constexpr int KS = HD / 32, DT = HD / 16, QP = QUERY_PARTS<T>, PP = WEIGHT_PARTS<T>;
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const uint8_t* const head = p.pool + (size_t)kvh * P::BYTES;
  const size_t page_bytes = (size_t)p.KV * P::BYTES;
  const int32_t* const table = p.rows.table + (size_t)b * p.rows.W;
  const uint32_t off_k = P::key(r, g * (HD / 4)), off_v = P::value(4 * g, r);
  const uint32_t off_ks = P::key_scale(r, g * (HD / 4) / 32), off_vs = P::value_scale(4 * g, r * DT / 32);

  // lane l of ids holds page l % 2 of step 32 j + l / 2, and of ids_next that of 32 steps later
  const int steps = end > first ? (end - first + stride - 1) / stride : 0;
  auto page_id = [&](int i0, bool& no, bool known) {
    const int i = i0 + lane / 2, pg = (first + stride * i) / 16 + (lane & 1);
    int id = 0;
    no = false;
    if (i < steps && 16 * pg < end) {
      id = known ? guess_id : pg < p.rows.W ? table[pg] : -1;
      no = (unsigned)id >= (unsigned)p.n_blocks;
    }
    return no ? 0 : id;
  };
  bool no_next;
  int ids = page_id(0, no_next, guessed);
  uint64_t no_ids = __ballot(no_next);
  int ids_next = page_id(32, no_next, false);

  // keys are loaded a step ahead when those of the step have been used, values likewise
  L4 kc[2], vc[2];
  uint32_t kE[2], vE[2];
  const uint8_t *pg0, *pg1;                      // the pages being loaded, and which of them are none
  uint32_t no = 0;
  auto pages = [&](int i) {
    pg0 = head + (size_t)(uint32_t)__builtin_amdgcn_readlane(ids, 2 * i) * page_bytes;
    pg1 = head + (size_t)(uint32_t)__builtin_amdgcn_readlane(ids, 2 * i + 1) * page_bytes;
    no = (uint32_t)(no_ids >> (2 * i)) & 3u;
  };
  auto load_k = [&]() {
    const auto b0 = page_buffer<HD>(pg0), b1 = page_buffer<HD>(pg1);
    kc[0] = page_load<L4, NT>(b0, off_k);
    kE[0] = page_load<uint8_t>(b0, off_ks);
    kc[1] = page_load<L4, NT>(b1, off_k);
    kE[1] = page_load<uint8_t>(b1, off_ks);
  };
  auto load_v = [&]() {
    const auto b0 = page_buffer<HD>(pg0), b1 = page_buffer<HD>(pg1);
    vc[0] = page_load<L4, NT>(b0, off_v);
    vE[0] = page_load<uint32_t>(b0, off_vs);
    vc[1] = page_load<L4, NT>(b1, off_v);
    vE[1] = page_load<uint32_t>(b1, off_vs);
  };

  int limit = FAR_LIMIT;
  int key0 = first, left = steps, at = 0;       // at: of the step after this one, within ids
  // EDGE: some key of the step is not seen by all vectors, or a page is none
  auto step = [&]<bool EDGE>() {
    const uint8_t* const here[2] = {pg0, pg1};
    const uint32_t no_here = no;
    f32x4 z[QT][2];
#pragma unroll
    for (int t = 0; t < QT; ++t) z[t][0] = z[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float ks = scale4(EDGE && (no_here >> t & 1) ? 255u : kE[t]);
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const u32x4 k = cvt4_all(kc[t][s], ks);
#pragma unroll
        for (int u = 0; u < QT; ++u)
#pragma unroll
          for (int part = QP - 1; part >= 0; --part) z[u][t] = mfma_bf16(k, q[u][s][part], z[u][t]);
      }
    }

    // the next step's keys (behind the last step its own again, which nothing uses)
    if (left > 1) {
      if (++at == 32) {
        at = 0;
        ids = ids_next;
        no_ids = __ballot(no_next);
        ids_next = page_id(steps - left + 1 + 32, no_next, false);
      }
      pages(at);
    }
    load_k();

    u32x4 w8[QT][PP];
    float x[QT][8];
    weigh<0>(EDGE, z, c, key0 + 4 * g, vis, m, limit, l, o, x);
#pragma unroll
    for (int u = 0; u < QT; ++u) {
      exp8(x[u]);
      l[u] += sum8(x[u]);
      parts8<PP>(x[u], w8[u]);
    }

    bool nan = false;
    if (EDGE && __any(clean_scales(vE, key0 + 4 * g, n_max, no_here))) nan = __any(clean_codes<HD>(vc, vE));
    add_values<HD>(vc, vE, w8, o);
    load_v();
    if (nan) put_nan<HD>(here, no_here, key0, n_max, g, vis, o);
  };

  if (left > 0) {
    pages(0);
    load_k();
    load_v();
  }
  if constexpr (FULL)
    for (; left > 0 && key0 + 32 <= n_min && !no; --left, key0 += stride) step.template operator()<false>();
  for (; left > 0; --left, key0 += stride) step.template operator()<true>();
}

// waves that a SIMD is to hold at once, for which the compiler keeps to so many registers
template <typename T, int QT> constexpr int MIN_WAVES = QT == 2 ? 2 : sizeof(T) == 2 ? 4 : 3;

template <typename T, int HD, int QT, int WAVES, bool NT>
__global__ __launch_bounds__(64 * WAVES, (MIN_WAVES<T, QT>)) void attention4_stream_kernel(Attn4Params p) {
  constexpr int KS = HD / 32, DT = HD / 16, QP = QUERY_PARTS<T>;
  constexpr int ROWS = 64 / WAVES;               // vectors that are joined at a time
  __shared__ __attribute__((aligned(16))) float s_o[WAVES][ROWS][HD + 4];
  __shared__ float s_m[WAVES][16], s_l[WAVES][16];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int G = p.H / p.KV;
  const int kvh = blockIdx.x % p.KV, split = blockIdx.x / p.KV % p.splits, block = blockIdx.x / p.KV / p.splits;
  // one block a sequence is the usual case: its first pages' ids are on their way while the sequence is looked up
  const int guess = min(block, p.rows.B - 1), guess_page = 2 * wave + 2 * WAVES * (lane / 2) + (lane & 1);
  const int guess_id = p.splits == 1 && guess_page < p.rows.W ? p.rows.table[(size_t)guess * p.rows.W + guess_page] : -1;
  Block4 w;
  if (!find_block(p.rows, p.M, G, 16 * QT, block, p.sorted, w)) return;
  const int len = w.len;
  const int nv = min(16 * QT, w.n * G - w.v0);   // vectors of this workgroup
  const int n_max = loop_keys(p, max(0, sees(p, len, w.n, w.v0 + nv - 1, G)));
  const int n_min = sees(p, len, w.n, w.v0, G);  // what all of them see
  const int kps = range_keys(n_max, p.splits, 32 * WAVES);
  const int k0 = split * kps, k1 = min(k0 + kps, n_max);
  if (split > 0 && k0 >= k1) {
    const int vec = w.v0 + tid;
    if (tid < nv) emit_nothing(p, split, w.row0 + vec / G, kvh * G + vec % G, sees(p, len, w.n, vec, G) > 0);
    return;
  }

  u32x4 q[QT][KS][QP];
  int vis[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int v = w.v0 + 16 * t + r;
    const bool on = 16 * t + r < nv;
    vis[t] = on ? sees(p, len, w.n, v, G) : 0;
    load_query<T, HD>((const T*)p.q + (size_t)(w.row0 + (on ? v / G : 0)) * p.ldq + (kvh * G + (on ? v % G : 0)) * HD + g * (HD / 4),
                      p.scale < 0.f, q[t]);                // the sign of the scale goes into the queries
  }
  const float c = fabsf(p.scale) * 1.4426950408889634f;

  float m[QT], l[QT];
  f32x4 o[QT][DT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m[t] = -FLT_MAX;
    l[t] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  take_keys<T, HD, QT, true, NT>(p, kvh, w.b, k0 + 32 * wave, 32 * WAVES, k1, n_min, n_max, q, c, vis, m, l, o,
                                 p.splits == 1 && w.b == guess, guess_id);

  // the waves' outputs are joined in their order
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    if (16 * t >= nv) break;
    const float sum = quad_sum(l[t]);
    for (int v0 = 0; v0 < min(16, nv - 16 * t); v0 += ROWS) {
      if (t || v0) __syncthreads();
      if (v0 == 0 && g == 0) {
        s_m[wave][r] = m[t];
        s_l[wave][r] = sum;
      }
      if ((unsigned)(r - v0) < (unsigned)ROWS) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int d = 0; d < DT; d += 4)
            *(f32x4*)&s_o[wave][r - v0][(4 * g + i) * DT + d] = f32x4{o[t][d][i], o[t][d + 1][i], o[t][d + 2][i], o[t][d + 3][i]};
      }
      __syncthreads();
      for (int idx = tid; idx < ROWS * (HD / 4); idx += 64 * WAVES) {
        const int v = v0 + idx / (HD / 4), d = idx % (HD / 4) * 4;
        if (16 * t + v >= nv) continue;
        float M = s_m[0][v], L = 0.f;
#pragma unroll
        for (int k = 1; k < WAVES; ++k) M = fmaxf(M, s_m[k][v]);
        f32x4 O{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < WAVES; ++k) {
          const float e = __builtin_amdgcn_exp2f(s_m[k][v] - M);
          L += s_l[k][v] * e;
          O += *(const f32x4*)&s_o[k][v - v0][d] * e;
        }
        const int vec = w.v0 + 16 * t + v;
        emit<T, HD>(p, split, w.row0 + vec / G, kvh * G + vec % G, d, sees(p, len, w.n, vec, G) > 0, M, L, O);
      }
    }
  }
}

// Prefill: 128 vectors a workgroup, 32 a wave, and the keys in LDS: each wave converts a quarter of a step's 32 keys for all
// four, while they take the step before it.  Without sharing, a wave's conversions cost as much as its products: 2048 rows
// on 4095 keys of 32 heads take 157 us that way and 111 us this way.
//
// bf16 only.  The values are held as fp16, which their codes times scales of 2^-23 to 2^8 are exactly, so that a weight is
// one fp16 part and half the products of the second matrix are saved.  It is off by 2^-11 of itself, where the output's own
// rounding is 2^-8.  Weights reach 2^15, and the largest so far is 2^7 at least: so they are that exact down to 2^-21 of the
// largest, and what is left out is below 2^-32 of it (with 1 for the largest, thousands of keys of 2^-25 each were).
// A workgroup that meets a value outside that range, NaN or a missing page leaves the loop and takes the rest of its keys as
// above.  (fp32 vectors would need three parts of either operand here too: 63 to 74 us against 49 for 3 sequences of 600
// rows.)
//
// Counters: of the SIMDs' cycles the products take 42 % and vector instructions 51 %; the waves, two to a SIMD, wait to issue
// for 32 % of theirs and for loads, LDS and barriers for 22 %.  Taken out of the loop one at a time (of 133 us, at an earlier step), the conversions are worth 24, the maximum test 9,
// the exponentials 8, the barrier 8.  The rare paths lie outside the loop because their code there kept the accumulators from
// staying in place.  Tried and worse: waves' priorities raised around the products (146), eight waves of 16 vectors, two
// waves of 64 (registers spill).
template <int HD> __global__ __launch_bounds__(256, 2) void attention4_tile_kernel(Attn4Params p) {
  using T = bf16_t;
  using P = Page4<HD>;
  using L4 = typename Load4<HD>::type;
  constexpr int QT = 2, KS = HD / 32, DT = HD / 16;
  constexpr int UP = 7;                          // weights of up to 2^15
  __shared__ u32x4 s_k[2][2][KS][64];            // [buffer][page][k-step][lane]
  __shared__ u32x4 s_v[3][DT][64];               // [buffer][tile][lane]: four keys of either page
  __shared__ int s_leave[3];                     // step + 1 that is not for the loop over LDS

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int G = p.H / p.KV;
  const int kvh = blockIdx.x % p.KV, order = blockIdx.x / p.KV, part = (p.blocks + 1) / 2;
  // the rows that see most go first; where all workgroups run at once, two to a CU, a long one meets a short one there
  const int block = order >= part && (int64_t)p.blocks * p.KV <= 512 ? order - part : p.blocks - 1 - order;
  Block4 w;
  if (!find_block(p.rows, p.M, G, 64 * QT, block, false, w)) return;
  const int len = w.len;
  const int nv = min(64 * QT, w.n * G - w.v0);
  const int n_max = loop_keys(p, max(0, sees(p, len, w.n, w.v0 + nv - 1, G)));
  const int n_min = sees(p, len, w.n, w.v0, G);

  // this wave's vectors
  const int first = w.v0 + 16 * QT * wave, on = min(16 * QT, nv - 16 * QT * wave);
  const int mine_min = on > 0 ? sees(p, len, w.n, first, G) : 0;
  const int mine_max = on > 0 ? loop_keys(p, sees(p, len, w.n, first + on - 1, G)) : 0;
  u32x4 q[QT][KS][1];
  int vis[QT];
  float m[QT];
  f32x4 o[QT][DT], l[QT];                        // l: the weights' sum, four times, as the product with a tile of ones
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int v = first + 16 * t + r;
    const bool is = 16 * t + r < on;
    vis[t] = is ? sees(p, len, w.n, v, G) : 0;
    load_query<T, HD>((const T*)p.q + (size_t)(w.row0 + (is ? v / G : 0)) * p.ldq + (kvh * G + (is ? v % G : 0)) * HD + g * (HD / 4),
                      p.scale < 0.f, q[t]);
    m[t] = -FLT_MAX;
    l[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int d = 0; d < DT; ++d) o[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float c = fabsf(p.scale) * 1.4426950408889634f;

  // Conversion: wave 2 a + b takes half a of page b of a step: k-steps KS / 2 a .., and tiles DT / 2 a .. of all 16 keys.
  // Lane l of ids holds its page of step 64 j + l.
  const int half = wave >> 1, mypage = wave & 1;
  const uint8_t* const head = p.pool + (size_t)kvh * P::BYTES;
  const size_t page_bytes = (size_t)p.KV * P::BYTES;
  const int32_t* const table = p.rows.table + (size_t)w.b * p.rows.W;
  const uint32_t off_k = P::key(r, g * (HD / 4) + half * (HD / 8)), off_v = P::value(4 * g, r);
  const uint32_t off_ks = P::key_scale(r, g * (HD / 4) / 32), off_vs = P::value_scale(4 * g, r * DT / 32);
  auto page_id = [&](int i0, bool& no) {
    const int pg = 2 * (i0 + lane) + mypage;
    int id = 0;
    no = false;
    if (16 * pg < n_max) {
      id = pg < p.rows.W ? table[pg] : -1;
      no = (unsigned)id >= (unsigned)p.n_blocks;
    }
    return no ? 0 : id;
  };
  int ids = 0;
  uint64_t no_ids = 0;
  // what is loaded of a step, four steps ahead of its use
  struct Raw {
    u32x2 kc;                                    // codes of keys (HD 64: one of them)
    uint32_t kE, vE;                             // scales
    L4 vc;                                       // codes of values
    bool none;                                   // no page
  } raw[2];
  auto load = [&](Raw& a, int i) {               // step i, in order (behind the last: any page)
    if (i % 64 == 0) {
      bool no;
      ids = page_id(i, no);
      no_ids = __ballot(no);
    }
    const auto pg = page_buffer<HD>(head + (size_t)(uint32_t)__builtin_amdgcn_readlane(ids, i % 64) * page_bytes);
    a.none = no_ids >> (i % 64) & 1;
    if constexpr (KS == 4) a.kc = page_load<u32x2>(pg, off_k);
    else a.kc[0] = page_load<uint32_t>(pg, off_k);
    a.kE = page_load<uint8_t>(pg, off_ks);
    a.vc = page_load<L4>(pg, off_v);
    a.vE = page_load<uint32_t>(pg, off_vs);
  };
  auto put_keys = [&](const Raw& a, int kb) {
#pragma unroll
    for (int s = 0; s < KS / 2; ++s) s_k[kb][mypage][half * (KS / 2) + s][lane] = cvt4_all(a.kc[s], scale4(a.kE));
  };
  auto put_values = [&](const Raw& a, int vb) {
    float s[1][4];
    const uint32_t Es[1] = {a.vE};
    value_scales(Es, s);
    // the half's bytes of every key, by a shift that does not depend on it
    L4 mine = a.vc;
#pragma unroll
    for (int e = 0; e < HD / 32; ++e) mine[e] = a.vc[e] >> (8 * (HD / 64) * half);
    const L4 cs[1] = {mine};
    [&]<int... B>(std::integer_sequence<int, B...>) {
      (([&] {
         uint32_t even[2], odd[2];
         value_tiles<HD, B, 1, true>(cs, s, even, odd);
         u32x2* const to = (u32x2*)&s_v[vb][half * (DT / 2) + 2 * B][lane] + mypage;
         to[0] = u32x2{even[0], even[1]};
         to[2 * 64] = u32x2{odd[0], odd[1]};
       }()),
       ...);
    }(std::make_integer_sequence<int, HD / 64>{});
  };
  // what load left of step i, into its buffers
  auto convert = [&](const Raw& a, int i, int kb, int vb) {
    put_keys(a, kb);
    put_values(a, vb);
    // the four scales at once, E + 24 of 128 to 159 (a carry from a byte is of one that is outside)
    const bool outside = ((a.vE + 0x18181818u) & 0xe0e0e0e0u) != 0x80808080u;
    if (a.none || __any(outside)) {
      bool leave = a.none;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t E = a.vE >> (8 * e) & 255u;
        uint32_t codes;
        if constexpr (HD == 128) codes = a.vc[e];
        else codes = e & 1 ? a.vc[e / 2] >> 16 : a.vc[e / 2] & 0xffffu;
        leave |= E == 255u || (E - 104u > 31u && (codes & 0x77777777u) != 0);      // (zeros have E = 1)
      }
      if (__any(leave) && lane == 0) s_leave[vb] = i + 1;
    }
  };

  f32x4 z[QT][2];
  u32x4 kf[KS][2];
  auto read_keys = [&](int kb) {
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int t = 0; t < 2; ++t) kf[s][t] = s_k[kb][t][s][lane];
  };
  auto scores = [&]() {
#pragma unroll
    for (int u = 0; u < QT; ++u) z[u][0] = z[u][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int u = 0; u < QT; ++u) z[u][t] = mfma_bf16(kf[s][t], q[u][s][0], z[u][t]);
  };
  // Steps that all vectors see whole, while the workgroup meets no value outside fp16, no NaN and no page that is none.
  // Step i: its weights; the scores of step i + 1; its values; the conversion of step i + 2; the loads of step i + 4
  const int full = max(0, min(n_max, n_min)) / 32;
  int i = 0;
  if (full > 0) {
    if (tid < 3) s_leave[tid] = 0;
    lds_barrier();
    load(raw[0], 0);
    load(raw[1], 1);
    convert(raw[0], 0, 0, 0);
    load(raw[0], 2);
    convert(raw[1], 1, 1, 1);
    load(raw[1], 3);
    lds_barrier();
    read_keys(0);
    scores();
    int vb = 0, leave = s_leave[0], limit = NEAR_LIMIT<UP>;
    lds_barrier();
    auto next = [&]<int S>() {                   // step i, S = i % 2
      if (i >= full || __builtin_amdgcn_readfirstlane(leave) == i + 1) return false;
      const int after = vb == 2 ? 0 : vb + 1;
      read_keys(1 - S);
      leave = s_leave[after];
      float x[QT][8];
      weigh<UP>(false, z, c, 0, vis, m, limit, l, o, x);
      u32x4 vf[DT];
#pragma unroll
      for (int d = 0; d < DT; ++d) vf[d] = s_v[vb][d][lane];
      scores();
#pragma unroll
      for (int u = 0; u < QT; ++u) exp8(x[u]);
      u32x4 w8[QT];
#pragma unroll
      for (int u = 0; u < QT; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) w8[u][e] = __builtin_bit_cast(uint32_t, f16x2{(f16_t)x[u][2 * e], (f16_t)x[u][2 * e + 1]});
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int u = 0; u < QT; ++u) o[u][d] = mfma_f16(vf[d], w8[u], o[u][d]);
#pragma unroll
      for (int u = 0; u < QT; ++u) l[u] = mfma_f16(u32x4{} + 0x3c003c00u, w8[u], l[u]);
      convert(raw[S], i + 2, S, vb == 0 ? 2 : vb - 1);     // (the buffers of steps i and i - 1)
      load(raw[S], i + 4);
      lds_barrier();
      vb = after;
      ++i;
      return true;
    };
    while (next.template operator()<0>() && next.template operator()<1>()) {}
  }

  // the others (behind the first keys that some vector does not see, 128 at most per head of a row): each wave by itself
  float sums[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const float to = m[t] + UP, by = __builtin_amdgcn_exp2f(m[t] - to);       // (of m as it is rounded)
    m[t] = to;
    sums[t] = g == 0 ? l[t][0] * by : 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[t][d] *= by;
  }
  take_keys<T, HD, QT, false, false>(p, kvh, w.b, 32 * i, 32, mine_max, mine_min, mine_max, q, c, vis, m, sums, o, false, 0);

#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const float sum = quad_sum(sums[t]);
    const int vec = first + 16 * t + r;
    if (16 * t + r >= on) continue;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int d = 0; d < DT; d += 4)
        emit<T, HD>(p, 0, w.row0 + vec / G, kvh * G + vec % G, (4 * g + e) * DT + d, vis[t] > 0, m[t], sum,
                    f32x4{o[t][d][e], o[t][d + 1][e], o[t][d + 2][e], o[t][d + 3][e]});
  }
}

// Joins the ranges of a vector in their order: hd / 4 lanes of four dimensions for each of PARTS runs of 8 ranges, then
// the runs.  No load waits for another, so that it is a launch and one round of latency: 5 us for 160 vectors of 32 ranges.
template <typename T, int HD, int PARTS> __global__ __launch_bounds__(256) void attention4_join_kernel(Attn4Params p) {
  constexpr int LANES = HD / 4, EACH = 256 / (LANES * PARTS);       // vectors of a workgroup
  __shared__ __attribute__((aligned(16))) float s_o[PARTS > 1 ? 256 : 1][4];
  __shared__ float s_m[PARTS > 1 ? 256 : 1], s_l[PARTS > 1 ? 256 : 1];
  const int tid = threadIdx.x, d = tid % LANES * 4, part = tid / LANES % PARTS;
  const int64_t vec = (int64_t)blockIdx.x * EACH + tid / (LANES * PARTS);
  const bool on = vec < (int64_t)p.M * p.H;
  const size_t at = on ? (size_t)vec : 0, step = (size_t)p.M * p.H;
  const int first = p.rows.cu[0], last = p.rows.cu[p.rows.B];
  float2 ml[8];
  f32x4 o[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int range = 8 * part + k;
    ml[k] = make_float2(-FLT_MAX, 0.f);
    o[k] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (range < p.splits) {
      ml[k] = *(const float2*)(p.part_ml + 2 * (at + range * step));
      o[k] = *(const f32x4*)(p.part_o + (at + range * step) * HD + d);
    }
  }
  float M = -FLT_MAX, L = 0.f;
  f32x4 O{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < 8; ++k) M = fmaxf(M, ml[k].x);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float e = __builtin_amdgcn_exp2f(ml[k].x - M);
    if (ml[k].y == 0.f && ml[k].x == -FLT_MAX) continue;            // without keys: its outputs were not written
    L += ml[k].y * e;
    O += o[k] * e;
  }
  if constexpr (PARTS > 1) {
    *(f32x4*)s_o[tid] = O;
    s_m[tid] = M;
    s_l[tid] = L;
    __syncthreads();
    if (part) return;
    const float M0 = M;
#pragma unroll
    for (int k = 1; k < PARTS; ++k) M = fmaxf(M, s_m[tid + k * LANES]);
    const float e0 = __builtin_amdgcn_exp2f(M0 - M);
    L *= e0;
    O *= e0;
#pragma unroll
    for (int k = 1; k < PARTS; ++k) {
      const float e = __builtin_amdgcn_exp2f(s_m[tid + k * LANES] - M);
      L += s_l[tid + k * LANES] * e;
      O += *(const f32x4*)s_o[tid + k * LANES] * e;
    }
  }
  const int row = (int)(vec / p.H), h = (int)(vec % p.H);
  if (!on || row < first || row >= last) return;
  if (L < 0.f) O = f32x4{0.f, 0.f, 0.f, 0.f};
  else O *= 1.f / L;
  store4((T*)p.out + (size_t)row * p.ldo + h * HD + d, O);
}

// Every rule with what was measured on both sides of it (us, in a replayed graph; hd 128 and bf16 unless said).
Attn4Plan plan_attention4(int dtype, int hd, int M, int H, int KV, int n_seqs, int max_len) {
  Attn4Plan a{};
  const int64_t G = H / KV, nz = std::min(n_seqs, M);
  const int64_t vectors = (M + nz - 1) / nz * G;             // of an average sequence
  // workgroups at most: the sum of ceil(n G / cap) over nz sequences of M rows, or what find_block numbers
  auto blocks = [&](int64_t cap) {
    if (n_seqs <= SUMMED) return (M * G - nz) / cap + nz;
    const int64_t u = common4((int)cap, (int)G), C = cap / u;
    return (M * (G / u) + (C - 1) * nz) / C;
  };
  auto typical = [&](int64_t cap) { return nz * ((vectors + cap - 1) / cap) * KV; };    // ... of alike sequences, and heads
  const int64_t steps = ((int64_t)max_len + 31) / 32;

  // Keys shared in LDS pay where a workgroup's 128 vectors are there and every CU has one: 2048 rows of 32 heads on 32,
  // 4095 keys, 111 shared and 157 not; 512 rows of 4 vectors each, 8192 keys, 99 and 100; 128 rows, 30 and 16; with 128 such
  // workgroups (2 sequences of 974 rows, 8 heads on 4, 1156 keys) 47.5 and 22.2.
  a.tile_kernel = dtype == 0 && vectors >= 128 && typical(128) >= 256;
  // Two tiles read and convert the keys once for 32 vectors, and leave half the workgroups: 32 sequences of 20 vectors and
  // 4000 keys, 40 with two tiles and 44 with one; 8 of 8192 keys, 25.7 and 26.5; but 4 of 8192 keys, 25.1 and 20.4; 32 of
  // 1000 keys on average, hd 64, 15.5 and 12.5.
  a.tiles = a.tile_kernel ? 8 : vectors > 16 && dtype == 0 && typical(16) * steps >= 28 * 1024 ? 2 : 1;
  a.blocks = (int)blocks(16 * a.tiles);
  const int64_t items = typical(16 * a.tiles);
  // Eight waves shorten a workgroup's loop over its keys; four leave less to join, and a CU takes twice as many of them (two
  // of eight waves, 512 on the card; of fp32, whose waves need a third of a SIMD's registers, one and 256), so that what does
  // not fit at once as eight and does as four takes one round instead of two.  256 workgroups of 1044 keys: 12.1 with eight
  // and 13.2 with four; 576 of 1024 keys 21.9 and 19.1, of 2048 keys 41.0 and 37.1, of ragged 4096 keys 40.0 and 43.1; 1024 of
  // 1000 keys 33.4 and 30.7; 2560 of 1024 keys 76 and 82, of 600 keys 58.6 and 55.3; 864 of 489 keys, fp32, hd 64, 19.6 and
  // 12.6; fp32, 384 of 1024 keys 22.1 and 18.0, 1024 of 1100 keys 42.8 and 34.7.
  const bool wide = dtype == 1 && hd == 128;
  const bool four = (wide && items >= 512) || (items > (wide ? 256 : 512) && items <= 1024 && steps < 128) || (items >= 1024 && steps < 24);
  a.waves = a.tile_kernel || a.tiles == 2 || four ? 4 : 8;
  // Ranges of keys fill the card where there are few workgroups; the join's launch costs 4 to 5.  8 workgroups: of 4000 keys
  // 12.0 with 16 ranges and 20 with one, of 2000 keys 11.1 with 7 and 11.7 to 12.5 with one, of 32768 keys 16.7 with 64 and 17.2
  // with 32; of 131072 keys 36 and 44.  128 workgroups of 4096 keys 18.1 with two ranges and 22.1 with one, of two tiles and
  // 8192 keys 40.2 with four and 66.2 with one; but 160 of 4096 keys 25.7 and 23.8, 256 of 8192 keys 57.2 and 54.6.  A little
  // over one workgroup to a CU leaves most CUs idle for the last: 288 of 16384 keys 124 and 140, 384 of 8192 keys 83 and 86
  // (320 of 4096 keys 44.5 and 44.3).
  a.splits = 1;
  if (items <= 64 && max_len >= 1536) {
    a.waves = 4;
    a.splits = (int)std::max<int64_t>(1, std::min<int64_t>({512 / items, max_len / 256, 64}));
  } else if (items <= 128 && max_len >= 2560) {
    a.splits = a.waves == 8 ? 2 : 4;
  } else if (a.waves == 8 && items > 256 && items <= 384 && max_len >= 8192) {
    a.splits = 2;
  }
  // Pages that one workgroup reads once, of a cache that does not fit the last-level cache (256 MiB) twice over, are loaded
  // past it: 64 sequences of 8192 keys 99.7 and 108.9 without; what does fit loses by it (36 MB: 14.1 and 12.8).
  // Where a workgroup's keys take long and not all workgroups run at once, the longest sequences go first, if some is over a
  // quarter longer or shorter than the first (finding the order costs each of them about 0.5): up to 8192 keys, lengths
  // evenly spread, 64 sequences on 8 heads 57.3 and 62.3 as they come; up to 4096 keys 36.0 and 39.9, 48 of them 30.5 and 36.7;
  // fp32, 32 of 5 rows on 32 heads, up to 2176 keys 50.8 and 53.4; alike ones 91.4 and 90.9, 56.0 and 55.0.  Up to 1024 keys, 64
  // sequences on 32 heads: 48.4 and 45.4.
  a.sorted = !a.tile_kernel && n_seqs > 1 && n_seqs <= SUMMED && items > 256 && steps * (dtype == 1 ? 2 : 1) >= 128;
  a.stream = !a.tile_kernel && vectors <= 16 * a.tiles && (double)nz * max_len * KV * 17 * hd / 16 > 536870912.0;
  return a;
}

size_t attention4_part_floats(const Attn4Plan& a, int M, int H, int hd) {
  return a.splits > 1 ? (size_t)a.splits * M * H * (hd + 2) : 0;
}

template <typename T, int HD, int QT, int WAVES> static void launch_stream(const Attn4Plan& a, const Attn4Params& p, hipStream_t s) {
  const dim3 grid((unsigned)a.blocks * p.KV * a.splits);
  if (a.stream) attention4_stream_kernel<T, HD, QT, WAVES, true><<<grid, 64 * WAVES, 0, s>>>(p);
  else attention4_stream_kernel<T, HD, QT, WAVES, false><<<grid, 64 * WAVES, 0, s>>>(p);
}

template <typename T, int HD> static void launch_hd(const Attn4Plan& a, Attn4Params p, hipStream_t s) {
  p.blocks = a.blocks;
  p.splits = a.splits;
  p.sorted = a.sorted;
  if constexpr (sizeof(T) == 2) {
    if (a.tile_kernel) {
      attention4_tile_kernel<HD><<<dim3((unsigned)a.blocks * p.KV), 256, 0, s>>>(p);
      return;
    }
    if (a.tiles == 2) launch_stream<T, HD, 2, 4>(a, p, s);
  }
  if (a.tiles == 1) {
    if (a.waves == 8) launch_stream<T, HD, 1, 8>(a, p, s);
    else launch_stream<T, HD, 1, 4>(a, p, s);
  }
  if (a.splits > 1) {
    const int64_t n = (int64_t)p.M * p.H;
    constexpr int each = 1024 / HD;              // hd / 4 lanes a vector
    if (a.splits <= 8) attention4_join_kernel<T, HD, 1><<<dim3((unsigned)((n + each - 1) / each)), 256, 0, s>>>(p);
    else attention4_join_kernel<T, HD, 8><<<dim3((unsigned)((n * 8 + each - 1) / each)), 256, 0, s>>>(p);
  }
}

hipError_t launch_attention4(int dtype, int hd, const Attn4Plan& a, const Attn4Params& p, hipStream_t s) {
  if (dtype == 1) {
    if (hd == 128) launch_hd<float, 128>(a, p, s);
    else launch_hd<float, 64>(a, p, s);
  } else {
    if (hd == 128) launch_hd<bf16_t, 128>(a, p, s);
    else launch_hd<bf16_t, 64>(a, p, s);
  }
  return hipGetLastError();
}

}  // namespace sd
