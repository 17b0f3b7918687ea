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
// bf16 queries.  fp32 queries enter as three bf16 parts (24 bits), weights as two
// for bf16 outputs (16 bits or more: an error of a quarter of a percent of the output's own
// rounding) and as three for fp32 ones.  Scores, the running maximum, the
// weights' sum and the output are fp32.
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
#include "codes4.h"

#include <float.h>
#include <math.h>

#include <algorithm>

namespace sd {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x4 mfma_bf16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <int E> __device__ __forceinline__ uint32_t cvt4(uint32_t c, float s) {   // byte E
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, E));
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

// The vectors of workgroup `block`: sequence b, its first row, its rows n and the first of its vectors.  Sequence b has
// ceil(n G / cap) workgroups; every wave adds them up by itself, 64 sequences at a time.
struct Block4 { int b, row0, n, v0; };
__device__ __forceinline__ bool find_block(const KvRows& s, int M, int G, int cap, int block, Block4& o) {
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < s.B; b0 += 64) {
    const int b = b0 + lane;
    int lo = 0, hi = 0;
    if (b < s.B) {
      lo = min(max(s.cu[b], 0), M);
      hi = min(max(s.cu[b + 1], lo), M);
    }
    const int mine = ((hi - lo) * G + cap - 1) / cap;
    int sum = mine;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
      const int up = __shfl_up(sum, k);
      if (lane >= k) sum += up;
    }
    const int total = __builtin_amdgcn_readlane(sum, 63);
    if (block < total) {
      const int at = __builtin_ctzll(__ballot(sum > block));
      o.b = b0 + at;
      o.row0 = __builtin_amdgcn_readlane(lo, at);
      o.n = __builtin_amdgcn_readlane(hi, at) - o.row0;
      o.v0 = (block - (__builtin_amdgcn_readlane(sum, at) - __builtin_amdgcn_readlane(mine, at))) * cap;
      return (unsigned)o.v0 < (unsigned)(o.n * G);           // (row counts that overflow, of no valid cu)
    }
    block -= total;
  }
  return false;
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

template <typename T, int HD, int QT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void attention4_stream_kernel(Attn4Params p) {
  using P = Page4<HD>;
  using L4 = typename Load4<HD>::type;
  constexpr int KS = HD / 32;                    // k-steps of a score
  constexpr int DT = HD / 16;                    // output tiles, dimensions of a lane's values
  constexpr int QP = sizeof(T) == 2 ? 1 : 3;     // parts of a query
  constexpr int PP = sizeof(T) == 2 ? 2 : 3;     // parts of a weight
  __shared__ __attribute__((aligned(16))) float s_o[WAVES][16][HD + 4];
  __shared__ float s_m[WAVES][16], s_l[WAVES][16];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int G = p.H / p.KV;
  const int kvh = blockIdx.x % p.KV, split = blockIdx.x / p.KV % p.splits, block = blockIdx.x / p.KV / p.splits;
  Block4 w;
  if (!find_block(p.rows, p.M, G, 16 * QT, block, w)) return;
  const int len = p.rows.len[w.b];
  const int nv = min(16 * QT, w.n * G - w.v0);   // vectors of this workgroup
  const int n_max = loop_keys(p, max(0, sees(p, len, w.n, w.v0 + nv - 1, G)));
  const int n_min = sees(p, len, w.n, w.v0, G);  // what all of them see
  const int kps = range_keys(n_max, p.splits, 32 * WAVES);
  const int k0 = split * kps, k1 = min(k0 + kps, n_max);
  if (split > 0 && k0 >= k1) return;

  // queries, as operands: lane (r, g) has dimensions (hd / 4) g + 8 s .. of vector r in k-step s
  u32x4 q[QT][KS][QP];
  int vis[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int v = w.v0 + 16 * t + r;
    const bool on = 16 * t + r < nv;
    vis[t] = on ? sees(p, len, w.n, v, G) : 0;
    const T* const src = (const T*)p.q + (size_t)(w.row0 + (on ? v / G : 0)) * p.ldq + (kvh * G + (on ? v % G : 0)) * HD + g * (HD / 4);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      if constexpr (sizeof(T) == 2) {
        q[t][s][0] = ((const u32x4*)src)[s];
        if (p.scale < 0.f) q[t][s][0] ^= 0x80008000u;      // the sign of the scale goes into the queries
      } else {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = p.scale < 0.f ? -src[8 * s + e] : src[8 * s + e];
        parts8<QP>(x, q[t][s]);
      }
    }
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

  const uint8_t* const head = p.pool + (size_t)kvh * P::BYTES;
  const size_t page_bytes = (size_t)p.KV * P::BYTES;
  const int32_t* const table = p.rows.table + (size_t)w.b * p.rows.W;
  const int off_k = P::key(r, g * (HD / 4)), off_v = P::value(4 * g, r);
  const int off_ks = P::key_scale(r, g * (HD / 4) / 32), off_vs = P::value_scale(4 * g, r * DT / 32);

  // the wave's steps are 32 (wave + WAVES i) keys into the range; lane l holds page l % 2 of step i0 + l / 2
  const int steps = k1 > k0 ? ((k1 - k0 + 31) / 32 - wave + WAVES - 1) / WAVES : 0;
  int ids = 0;
  uint64_t bad = 0;
  auto load_ids = [&](int i0) {
    const int i = i0 + lane / 2;
    const int pg = (k0 + 32 * (wave + WAVES * i)) / 16 + (lane & 1);
    int id = 0;
    bool no = false;
    if (i < steps && 16 * pg < k1) {
      id = pg < p.rows.W ? table[pg] : -1;
      no = (unsigned)id >= (unsigned)p.n_blocks;
      if (no) id = 0;
    }
    ids = id;
    bad = __ballot(no);
  };

  struct Stage { L4 k[2], v[2]; uint32_t ks[2], vs[2]; };
  auto load = [&](Stage& st, int i) {            // i: step within the ids held
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint8_t* const pg = head + (size_t)(uint32_t)__builtin_amdgcn_readlane(ids, 2 * i + t) * page_bytes;
      st.k[t] = *(const L4*)(pg + off_k);
      st.ks[t] = pg[off_ks];
      st.v[t] = *(const L4*)(pg + off_v);
      st.vs[t] = *(const uint32_t*)(pg + off_vs);
    }
  };

  // edge: some key of the step is not seen by all vectors, or a page is none
  auto step = [&](const Stage& st, int i, int key0) {
    const uint32_t no = (uint32_t)(bad >> (2 * i)) & 3u;
    const bool edge = key0 + 32 > n_min || no;
    uint32_t vs[2] = {st.vs[0], st.vs[1]};
    float ks[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) ks[t] = scale4(no >> t & 1 ? 255u : st.ks[t]);
    bool nan_v = false;
    if (edge) {
      // values that not every vector sees must be finite: their weights are zero where they are not seen, and NaN
      // that a vector does see is put into its output below
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
          const int key = key0 + 16 * t + 4 * g + i4;
          const bool is_nan = (vs[t] >> (8 * i4) & 255u) == 255u, none = key >= n_max || (no >> t & 1);
          nan_v |= is_nan && !none;
          if (is_nan || none) vs[t] = (vs[t] & ~(255u << (8 * i4))) | 127u << (8 * i4);
        }
    }

    f32x4 z[QT][2];
#pragma unroll
    for (int t = 0; t < QT; ++t) z[t][0] = z[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const u32x4 k = cvt4_all(st.k[t][s], ks[t]);
#pragma unroll
        for (int u = 0; u < QT; ++u)
#pragma unroll
          for (int part = QP - 1; part >= 0; --part) z[u][t] = mfma_bf16(k, q[u][s][part], z[u][t]);
      }

    u32x4 w8[QT][PP];
#pragma unroll
    for (int u = 0; u < QT; ++u) {
      if (edge) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (key0 + 16 * t + 4 * g + e >= vis[u]) z[u][t][e] = -FLT_MAX;
      }
      float top = fmaxf(fmaxf(z[u][0][0], z[u][0][1]), fmaxf(z[u][0][2], z[u][0][3]));
      top = fmaxf(top, fmaxf(fmaxf(z[u][1][0], z[u][1][1]), fmaxf(z[u][1][2], z[u][1][3]))) * c;
      if (__any(top > m[u] + 8.f)) {
        const float m_new = fmaxf(m[u], quad_max(top));
        const float old = __builtin_amdgcn_exp2f(m[u] - m_new);
        m[u] = m_new;
        l[u] *= old;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[u][d] *= old;
      }
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] = __builtin_amdgcn_exp2f(fmaf(z[u][e / 4][e % 4], c, -m[u]));
        if (edge && key0 + 16 * (e / 4) + 4 * g + e % 4 >= vis[u]) x[e] = 0.f;
      }
      l[u] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
      parts8<PP>(x, w8[u]);
    }

    // pairs of dimensions of a key -> pairs of keys of a dimension
    constexpr int NB = HD / 32;                  // bytes of a key
    uint32_t cv[2][4][NB];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float s = scale4(vs[t] >> (8 * e) & 255u);
        if constexpr (HD == 128) {
          const u32x4 x = cvt4_all(st.v[t][e], s);
#pragma unroll
          for (int b = 0; b < NB; ++b) cv[t][e][b] = x[b];
        } else {
          cv[t][e][0] = e & 1 ? cvt4<2>(st.v[t][e / 2], s) : cvt4<0>(st.v[t][e / 2], s);
          cv[t][e][1] = e & 1 ? cvt4<3>(st.v[t][e / 2], s) : cvt4<1>(st.v[t][e / 2], s);
        }
      }
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      u32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t a = cv[e / 2][2 * (e % 2)][d / 2], b = cv[e / 2][2 * (e % 2) + 1][d / 2];
        v[e] = d & 1 ? high_halves(a, b) : low_halves(a, b);
      }
#pragma unroll
      for (int u = 0; u < QT; ++u)
#pragma unroll
        for (int part = PP - 1; part >= 0; --part) o[u][d] = mfma_bf16(v, w8[u][part], o[u][d]);
    }

    if (edge && __any(nan_v)) {                  // rare: a value block of NaN that some vector sees
      // all of a lane's outputs are of scale block (hd / 4) g / 32
      for (int key = key0; key < min(key0 + 32, n_max); ++key) {
        const int t = key - key0 >= 16;
        const uint8_t* const pg = head + (size_t)(uint32_t)__builtin_amdgcn_readlane(ids, 2 * i + t) * page_bytes;
        if (!(no >> t & 1) && pg[P::value_scale(key & 15, g * (HD / 4) / 32)] == 255) {
#pragma unroll
          for (int u = 0; u < QT; ++u)
            if (key < vis[u])
#pragma unroll
              for (int d = 0; d < DT; ++d) o[u][d] = f32x4{NAN, NAN, NAN, NAN};
        }
      }
    }
  };

  for (int i0 = 0; i0 < steps; i0 += 32) {
    load_ids(i0);
    const int n = min(32, steps - i0);
    const int first = k0 + 32 * (wave + WAVES * i0);
    Stage a, b;
    load(a, 0);
    for (int i = 0; i < n; i += 2) {
      if (i + 1 < n) load(b, i + 1);
      step(a, i, first + 32 * WAVES * i);
      if (i + 1 >= n) break;
      if (i + 2 < n) load(a, i + 2);
      step(b, i + 1, first + 32 * WAVES * (i + 1));
    }
  }

  // the waves' outputs are joined in their order, a tile of vectors at a time
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const float sum = quad_sum(l[t]);
    if (t) __syncthreads();
    if (16 * t >= nv) break;
    if (g == 0) {
      s_m[wave][r] = m[t];
      s_l[wave][r] = sum;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int d = 0; d < DT; d += 4)
        *(f32x4*)&s_o[wave][r][(4 * g + i) * DT + d] = f32x4{o[t][d][i], o[t][d + 1][i], o[t][d + 2][i], o[t][d + 3][i]};
    __syncthreads();
    for (int idx = tid; idx < 16 * (HD / 4); idx += 64 * WAVES) {
      const int v = idx / (HD / 4), d = idx % (HD / 4) * 4;
      if (16 * t + v >= nv) continue;
      float M = s_m[0][v], L = 0.f;
#pragma unroll
      for (int k = 1; k < WAVES; ++k) M = fmaxf(M, s_m[k][v]);
      f32x4 O{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < WAVES; ++k) {
        const float e = __builtin_amdgcn_exp2f(s_m[k][v] - M);
        L += s_l[k][v] * e;
        O += *(const f32x4*)&s_o[k][v][d] * e;
      }
      const int vec = w.v0 + 16 * t + v;
      if (p.splits == 1) {
        if (sees(p, len, w.n, vec, G) <= 0) O = f32x4{0.f, 0.f, 0.f, 0.f};
        else O *= 1.f / L;
        store4((T*)p.out + (size_t)(w.row0 + vec / G) * p.ldo + (kvh * G + vec % G) * HD + d, O);
      } else {
        const size_t at = (((size_t)block * p.KV + kvh) * p.splits + split) * (16 * QT) + 16 * t + v;
        *(f32x4*)(p.part_o + at * HD + d) = O;
        if (d == 0) *(float2*)(p.part_ml + 2 * at) = make_float2(M, L);
      }
    }
  }
}

// joins the ranges of a workgroup's vectors, in their order
template <typename T, int HD> __global__ __launch_bounds__(256) void attention4_join_kernel(Attn4Params p, int cap, int unit) {
  const int G = p.H / p.KV, kvh = blockIdx.x % p.KV, block = blockIdx.x / p.KV;
  Block4 w;
  if (!find_block(p.rows, p.M, G, cap, block, w)) return;
  const int len = p.rows.len[w.b], nv = min(cap, w.n * G - w.v0);
  const int n_max = loop_keys(p, max(0, sees(p, len, w.n, w.v0 + nv - 1, G)));
  const int kps = range_keys(n_max, p.splits, unit);
  const int used = n_max > 0 ? (n_max + kps - 1) / kps : 1;
  for (int idx = threadIdx.x; idx < nv * (HD / 4); idx += 256) {
    const int v = idx / (HD / 4), d = idx % (HD / 4) * 4;
    const size_t at = ((size_t)block * p.KV + kvh) * p.splits * cap + v;
    float M = -FLT_MAX, L = 0.f;
    for (int k = 0; k < used; ++k) M = fmaxf(M, p.part_ml[2 * (at + (size_t)k * cap)]);
    f32x4 O{0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < used; ++k) {
      const size_t i = at + (size_t)k * cap;
      const float e = __builtin_amdgcn_exp2f(p.part_ml[2 * i] - M);
      L += p.part_ml[2 * i + 1] * e;
      O += *(const f32x4*)(p.part_o + i * HD + d) * e;
    }
    const int vec = w.v0 + v;
    if (sees(p, len, w.n, vec, G) <= 0) O = f32x4{0.f, 0.f, 0.f, 0.f};
    else O *= 1.f / L;
    store4((T*)p.out + (size_t)(w.row0 + vec / G) * p.ldo + (kvh * G + vec % G) * HD + d, O);
  }
}

constexpr int WAVES4 = 4;

Attn4Plan plan_attention4(int dtype, int M, int H, int KV, int n_seqs, int max_len) {
  Attn4Plan a{};
  const int64_t G = H / KV, nz = std::min(n_seqs, M);
  const int64_t vectors = (M + nz - 1) / nz * G;             // of an average sequence
  a.tiles = vectors <= 16 ? 1 : vectors <= 32 || dtype == 1 ? 2 : 4;
  const int64_t cap = 16 * a.tiles;
  a.blocks = (int)((M * G - nz) / cap + nz);                 // sum of ceil(n G / cap) over nz sequences of M rows
  const int64_t items = (int64_t)a.blocks * KV, want = (1024 + items - 1) / items;
  a.splits = (int)std::max<int64_t>(1, std::min<int64_t>({want, (max_len + 255) / 256, 64}));
  return a;
}

size_t attention4_part_floats(const Attn4Plan& a, int KV, int hd) {
  return a.splits > 1 ? (size_t)a.blocks * KV * a.splits * 16 * a.tiles * (hd + 2) : 0;
}

template <typename T, int HD> static void launch_hd(const Attn4Plan& a, Attn4Params p, hipStream_t s) {
  const dim3 grid((unsigned)a.blocks * p.KV * a.splits);
  switch (a.tiles) {
    case 1: attention4_stream_kernel<T, HD, 1, WAVES4><<<grid, 64 * WAVES4, 0, s>>>(p); break;
    case 2: attention4_stream_kernel<T, HD, 2, WAVES4><<<grid, 64 * WAVES4, 0, s>>>(p); break;
    case 4:
      if constexpr (sizeof(T) == 2) attention4_stream_kernel<T, HD, 4, WAVES4><<<grid, 64 * WAVES4, 0, s>>>(p);
      break;
  }
  if (a.splits > 1)
    attention4_join_kernel<T, HD><<<dim3((unsigned)a.blocks * p.KV), 256, 0, s>>>(p, 16 * a.tiles, 32 * WAVES4);
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
