// What lies between a layer's QKV product and its attention over a 4-bit cache
// (format: codes4.h): the RMS norm of every query and key head and the rotary
// embedding, the quantisation of keys and values into their pages, and the
// reverse.
//
//   y = x / sqrt(mean(x^2) + eps) gain      over the hd entries of a head
//   (y_i, y_{i + hd/2}) -> (y_i c - y_{i + hd/2} s, y_{i + hd/2} c + y_i s)
//
// Everything is bound by memory (a value is read once and written once; about
// seven operations on it), or in small calls by its latency.  hd / 16 lanes
// take a head, a lane 8 entries of either half of it, from 8 i and from hd / 2 +
// 8 i: the two entries that a rotation mixes are in one lane, a scale's block
// of 32 in four neighbouring ones, and every access to a row is of 16 bytes.
// Where nothing is quantised, fp32 heads are taken as two groups of four a half,
// hd / 4 apart, so that neighbouring lanes' 16 bytes are neighbours in memory
// (2048 rows of 80 heads of 128: 41.7 -> 37.5 us).
//
// The norm and the rotation are in 64 bits, which the vector unit does at the
// rate of 32: a result is then a function of the input, whatever the order of a
// sum (but for one in about 2^28).  What is stored is rounded to fp32, off by
// 2^-24, and from there to its type or its code.
//
// Measured (times of a call in a replayed graph): norms and rotation of 2048
// fp32 rows of 80 heads of 128, 168 MB, 37.5 us, 4.5 TB/s (a copy of 1 GiB runs at
// 5.1); of one bf16 row of 40 heads of 64, 3.2 us, a launch and two rounds of
// memory latency.  40 bf16 rows of 96 heads of 128 (32 of them queries, returned)
// into the cache and the same rows back, 8.3 us; 2048 fp32 rows of 16 heads of
// 128 into the cache and back, 38 MB in 14.3 us, of which the two launches are
// half.  Up to 4096 cached positions of each of 8 sequences, 8 heads of 128, into
// bf16: 83 MB in 19.9 us, 4.2 TB/s.
#include "codes4.h"

namespace sd {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// 8 entries of a row; of fp32, two groups of four that lie APART entries apart
template <typename T, int APART = 4> __device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    const u32x4 u = *(const u32x4*)p;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(e & 1 ? u[e / 2] & 0xffff0000u : u[e / 2] << 16);
  } else {
    const u32x4 u = *(const u32x4*)p, w = *(const u32x4*)(p + APART);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = __uint_as_float(u[e]);
      x[4 + e] = __uint_as_float(w[e]);
    }
  }
}
template <typename T, int APART = 4> __device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    u32x4 u;
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x[2 * e], (__bf16)x[2 * e + 1]});
    *(u32x4*)p = u;
  } else {
    *(u32x4*)p = u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
    *(u32x4*)(p + APART) = u32x4{__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7])};
  }
}

// 8 entries of a gain in the same two groups; it is aligned to its entries only (the memory unit takes wide loads of any
// address)
template <int APART> __device__ __forceinline__ void gain8(const void* g, int bf16, int i, float (&x)[8]) {
  typedef uint16_t halves4 __attribute__((ext_vector_type(4), aligned(2)));
  typedef float floats4 __attribute__((ext_vector_type(4), aligned(4)));
  if (bf16) {
    const halves4 a = *(const halves4*)((const bf16_t*)g + i), b = *(const halves4*)((const bf16_t*)g + i + APART);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = bf2f(a[e]), x[4 + e] = bf2f(b[e]);
  } else {
    const floats4 a = *(const floats4*)((const float*)g + i), b = *(const floats4*)((const float*)g + i + APART);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = a[e], x[4 + e] = b[e];
  }
}

// x^-1/2 for x > 0: the hardware's estimate (24 bits) and two steps of Newton's iteration, each of which squares the error
__device__ __forceinline__ double rsqrt64(double x) {
  if (x == INFINITY) return 0.0;
  double y = __builtin_amdgcn_rsq(x);
  y = y * fma(-0.5 * x * y, y, 1.5);
  return y * fma(-0.5 * x * y, y, 1.5);
}

template <typename T, int HD, Kv4Mode MODE> __global__ __launch_bounds__(256) void kv4_kernel(Kv4Params p) {
  using P = Page4<HD>;
  constexpr int LANES = HD / 16;
  constexpr bool WIDE = MODE == KV4_HEADS && sizeof(T) == 4;
  constexpr int APART = WIDE ? HD / 4 : 4;
  const int per_row = (MODE == KV4_HEADS || MODE == KV4_BOTH ? p.H : 0) + (MODE == KV4_HEADS ? 1 : 2) * p.KV;
  const int64_t item = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  const int i = threadIdx.x % LANES, i8 = WIDE ? 4 * i : 8 * i;
  __shared__ Places s_places;
  if constexpr (MODE != KV4_HEADS) {
    s_places.load(p.rows);
    __syncthreads();
  }
  if (item >= (int64_t)p.M * per_row) return;    // whole heads: the shuffles below stay within one
  const int row = (int)(item / per_row), h0 = (int)(item % per_row);
  const int nq = MODE == KV4_HEADS || MODE == KV4_BOTH ? p.H : 0;
  const int what = h0 < nq ? 0 : h0 < nq + p.KV ? 1 : 2;      // query, key, value
  const int h = what == 0 ? h0 : what == 1 ? h0 - nq : h0 - nq - p.KV;

  float x[2][8];
  if constexpr (MODE != KV4_READ) {              // (rows of no sequence are read all the same)
    const T* const src = what == 0   ? (const T*)p.q + (size_t)row * p.ldq
                         : what == 1 ? (const T*)p.k + (size_t)row * p.ldk
                                     : (const T*)p.v + (size_t)row * p.ldv;
#pragma unroll
    for (int half = 0; half < 2; ++half) load8<T, APART>(src + h * HD + half * (HD / 2) + i8, x[half]);
  }

  int b = 0, pos = 0, page = -1;
  if constexpr (MODE == KV4_HEADS) {
    if (p.positions) pos = p.positions[row];
  } else {
    if (!row_place(p.rows, s_places, row, b, pos)) return;
    page = what ? row_page(p.rows, b, pos, p.n_blocks) : -1;
  }
  const int t = pos & 15;
  uint8_t* const pg = p.pool + ((size_t)max(page, 0) * p.KV + h) * P::BYTES;

  if constexpr (MODE == KV4_READ) {
    T* const out = (T*)(what == 1 ? p.k_out : p.v_out) + (size_t)row * (what == 1 ? p.ldko : p.ldvo) + h * HD;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int d = half * (HD / 2) + 8 * i;
      uint32_t c = 0, E = 255;
      if (page >= 0) {
        if (what == 1) {
          c = *(const uint32_t*)(pg + P::key(t, d));
          E = pg[P::key_scale(t, d / 32)];
        } else {
          if constexpr (HD == 128) {
            c = *(const uint32_t*)(pg + P::value(t, d / 8));
          } else {
            c = *(const uint16_t*)(pg + P::value(t, d / 4)) | (uint32_t)*(const uint16_t*)(pg + P::value(t, d / 4 + 1)) << 16;
          }
          E = pg[P::value_scale(t, d / 32)];
        }
      }
      decode4(c, scale4(E), x[half]);
      store8(out + d, x[half]);
    }
    return;
  }

  if (MODE != KV4_APPEND && what != 2) {
    // The gain and the rotation are read before the sum that they wait for.
    const void* const gain = what == 0 ? p.q_gain : p.k_gain;
    float g[2][8];
    if (gain) {
      gain8<APART>(gain, p.gain_bf16, i8, g[0]);
      gain8<APART>(gain, p.gain_bf16, HD / 2 + i8, g[1]);
    }
    float4 w[4] = {};
    if (p.rope) {
      const bool in = (unsigned)pos < (unsigned)p.n_pos;
      const float4* const cs = (const float4*)(p.rope + ((size_t)(in ? pos : 0) * (HD / 2) + i8) * 2);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = in ? cs[e < 2 ? e : e - 2 + APART / 2] : make_float4(NAN, NAN, NAN, NAN);
    }
    double r = 1.0;
    if (gain) {
      double sum = 0.0;
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fma((double)x[half][e], (double)x[half][e], sum);
#pragma unroll
      for (int o = LANES / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
      r = rsqrt64(sum / HD + p.eps);
    } else {
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int e = 0; e < 8; ++e) g[half][e] = 1.0f;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const double y0 = x[0][e] * r * g[0][e], y1 = x[1][e] * r * g[1][e];
      const double c = e % 2 ? w[e / 2].z : w[e / 2].x, sn = e % 2 ? w[e / 2].w : w[e / 2].y;
      x[0][e] = (float)(p.rope ? y0 * c - y1 * sn : y0);
      x[1][e] = (float)(p.rope ? y1 * c + y0 * sn : y1);
    }
    if (MODE == KV4_HEADS || what == 0) {
      T* const out = what == 0 ? (T*)p.q_out + (size_t)row * p.ldqo : (T*)p.k_out + (size_t)row * p.ldko;
#pragma unroll
      for (int half = 0; half < 2; ++half) store8<T, APART>(out + h * HD + half * (HD / 2) + i8, x[half]);
    }
  }
  if (MODE == KV4_HEADS || what == 0) return;

#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int d = half * (HD / 2) + 8 * i;
    uint32_t amax = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) amax = max(amax, __float_as_uint(x[half][e]) & 0x7fffffffu);   // NaN is past infinity
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 1));
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 2));
    const uint32_t E = block_exp4(amax), c = encode4(x[half], E);
    if (page < 0) continue;
    if (what == 1) {
      *(uint32_t*)(pg + P::key(t, d)) = c;
      if (i % 4 == 0) pg[P::key_scale(t, d / 32)] = (uint8_t)E;
    } else {
      if constexpr (HD == 128) {
        *(uint32_t*)(pg + P::value(t, d / 8)) = c;
      } else {
        *(uint16_t*)(pg + P::value(t, d / 4)) = (uint16_t)c;
        *(uint16_t*)(pg + P::value(t, d / 4 + 1)) = (uint16_t)(c >> 16);
      }
      if (i % 4 == 0) pg[P::value_scale(t, d / 32)] = (uint8_t)E;
    }
  }
}

template <typename T, int HD> static void launch_mode(Kv4Mode mode, const Kv4Params& p, hipStream_t s) {
  const int per_row = (mode == KV4_HEADS || mode == KV4_BOTH ? p.H : 0) + (mode == KV4_HEADS ? 1 : 2) * p.KV;
  const int64_t items = (int64_t)p.M * per_row;
  constexpr int each = 256 / (HD / 16);
  const dim3 grid((unsigned)((items + each - 1) / each));
  switch (mode) {
    case KV4_HEADS: kv4_kernel<T, HD, KV4_HEADS><<<grid, 256, 0, s>>>(p); break;
    case KV4_APPEND: kv4_kernel<T, HD, KV4_APPEND><<<grid, 256, 0, s>>>(p); break;
    case KV4_BOTH: kv4_kernel<T, HD, KV4_BOTH><<<grid, 256, 0, s>>>(p); break;
    case KV4_READ: kv4_kernel<T, HD, KV4_READ><<<grid, 256, 0, s>>>(p); break;
  }
}

hipError_t launch_kv4(Kv4Mode mode, int dtype, int hd, const Kv4Params& p, hipStream_t s) {
  if (dtype == 1) {
    if (hd == 128) launch_mode<float, 128>(mode, p, s);
    else launch_mode<float, 64>(mode, p, s);
  } else {
    if (hd == 128) launch_mode<bf16_t, 128>(mode, p, s);
    else launch_mode<bf16_t, 64>(mode, p, s);
  }
  return hipGetLastError();
}

}  // namespace sd
