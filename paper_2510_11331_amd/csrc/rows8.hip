// 8-bit operands of the feed-forward network: RMSNorm with an 8-bit output,
// quantisation of fp32 rows, and the packing of weight matrices (format: codes8.h).
#include "sd_internal.h"
#include "codes8.h"

namespace sd {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// maximum over the N lanes that hold a block
template <int N> __device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
  for (int o = N / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}

// entries 8 i .. 8 i + 7 of a row of n entries, zero past the end; VEC: rows are whole units, 16-byte aligned
struct Eight { float v[8]; };
template <typename T, bool VEC> __device__ __forceinline__ Eight load8(const T* row, int i, int n) {
  Eight r;
  if constexpr (VEC) {
    constexpr int U = sizeof(T) / 2;                   // 16-byte loads
    u32x4 u[U];
#pragma unroll
    for (int k = 0; k < U; ++k) u[k] = 8 * i < n ? ((const u32x4*)row)[U * i + k] : u32x4{0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (sizeof(T) == 4) r.v[e] = __uint_as_float(u[e / 4][e % 4]);
      else r.v[e] = __uint_as_float(e & 1 ? u[0][e / 2] & 0xffff0000u : u[0][e / 2] << 16);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) r.v[e] = 8 * i + e < n ? Store<T>::load(row, 8 * i + e) : 0.f;
  }
  return r;
}
template <typename T, bool VEC> __device__ __forceinline__ void store8(T* row, int i, int n, const Eight& x) {
  if constexpr (VEC) {
    if (8 * i >= n) return;
    constexpr int U = sizeof(T) / 2;
    u32x4 u[U];
#pragma unroll
    for (int k = 0; k < 4 * U; ++k) {
      if constexpr (sizeof(T) == 4) u[k / 4][k % 4] = __float_as_uint(x.v[k]);
      else u[0][k] = bf16_bits(x.v[2 * k]) | bf16_bits(x.v[2 * k + 1]) << 16;
    }
#pragma unroll
    for (int k = 0; k < U; ++k) ((u32x4*)row)[U * i + k] = u[k];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (8 * i + e >= n) continue;
      if constexpr (sizeof(T) == 4) row[8 * i + e] = x.v[e];
      else row[8 * i + e] = (bf16_t)bf16_bits(x.v[e]);
    }
  }
}

// Residual addition, RMSNorm and 8-bit output of one row per workgroup (R units
// of eight entries a thread, a block's 128 entries in 16 neighbouring lanes):
//   s = x + add_0 + ... + add_{n-1}         summed in 64 bits, stored in x's type (by way of fp32)
//   y = s / sqrt(mean(s^2) + eps) * gain    in 64 bits, rounded to fp32
//   q, E = codes and exponents of y
// 64-bit sums and norm: codes are a function of the input alone, not of the
// order of a sum (in 32 bits the kernel would be 0.2 us faster at one row and 1.5
// us at 2048).  Bound by memory: 2048 x 8192 fp32 with two addends 59 us, 4.8
// TB/s of the 5.2 that a copy reaches; 2048 x 5120 bf16 with one 20.0 us; 40 x
// 4096 fp32 with four 5.2 us and one row 3.3 us, a launch and three memory round
// trips.  Sixteen bytes a load (eight before: 24.2 us at 2048 x 5120).  All
// addends are loaded before the first is added (NS of them, those past n_add as
// zeros).
// Two addends take the code of six, and no time by it: 2048 x 8192 fp32 with six
// 112 us, 5.0 TB/s.  What 128 registers do not hold goes to scratch: six addends of
// four units (d past 8192, two or more addends) 70 to 300 registers, 2048 x
// 16384 fp32 with two 379 us, 1.5 TB/s; and rows that are read entry by entry (d no
// multiple of 8, or off 16 bytes) with two or more addends 270 to 800 of them from
// d = 2049 on, 2048 x 4096 fp32 with two 214 us against 32.
template <typename TX, typename TG, int R, int NS, bool VEC>
__global__ __launch_bounds__(R == 1 ? 256 : 512, 4) void add_rmsnorm8_kernel(Norm8Params p) {
  __shared__ double red[8];
  const size_t r = blockIdx.x;
  const int d = p.d, tid = threadIdx.x, th = blockDim.x;
  const TX* x = (const TX*)p.x + r * d;
  Eight v[R], a[NS > 0 ? NS : 1][R], g[R];
#pragma unroll
  for (int k = 0; k < R; ++k) v[k] = load8<TX, VEC>(x, tid + th * k, d);
#pragma unroll
  for (int j = 0; j < NS; ++j)
#pragma unroll
    for (int k = 0; k < R; ++k)
      a[j][k] = load8<TX, VEC>((const TX*)p.add + ((size_t)(j < p.n_add ? j : 0) * p.M + r) * d, tid + th * k, j < p.n_add ? d : 0);
#pragma unroll
  for (int k = 0; k < R; ++k) g[k] = load8<TG, VEC>((const TG*)p.gain, tid + th * k, d);
  if constexpr (NS > 0) {
#pragma unroll
    for (int k = 0; k < R; ++k) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        double s = (double)v[k].v[e];
#pragma unroll
        for (int j = 0; j < NS; ++j) s += (double)a[j][k].v[e];
        v[k].v[e] = sizeof(TX) == 4 ? (float)s : bf2f((bf16_t)bf16_bits((float)s));
      }
      store8<TX, VEC>((TX*)p.x_out + r * d, tid + th * k, d, v[k]);
    }
  }
  double ss = 0;
#pragma unroll
  for (int k = 0; k < R; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) ss += (double)v[k].v[e] * (double)v[k].v[e];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) ss += __shfl_xor(ss, o);
  if ((tid & 63) == 0) red[tid >> 6] = ss;
  __syncthreads();
  ss = 0;
  for (int w = 0; w < th >> 6; ++w) ss += red[w];
  const double inv = 1.0 / sqrt(ss / d + (double)p.eps);
  const int kb = blocks8(d), ke = ke8(d);
#pragma unroll
  for (int k = 0; k < R; ++k) {
    const int i = tid + th * k;
    float y[8], m = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      y[e] = (float)((double)v[k].v[e] * inv * (double)g[k].v[e]);
      if (8 * i + e >= d) y[e] = 0.f;     // a NaN of the row stays out of the padding
      m = fmaxf(m, finite_abs(y[e]));
    }
    m = lanes_max<16>(m);
    if (i < 16 * kb) {
      const int E = block_exp(m);
      const float sc = inv_scale(E);
      ((uint2*)(p.q + r * 128 * kb))[i] = make_uint2(codes4(y[0], y[1], y[2], y[3], sc), codes4(y[4], y[5], y[6], y[7], sc));
      if ((i & 15) == 0) p.exps[r * ke + i / 16] = (uint8_t)E;
    }
  }
  if (tid < ke - kb) p.exps[r * ke + kb + tid] = 0;
}

// fp32 rows [M, F] (F a multiple of 16) -> codes and exponents; 32 lanes per block
__global__ __launch_bounds__(256) void quantise_rows8_kernel(const float* h, uint8_t* q, uint8_t* exps, int M, int F) {
  const int kb = (F + 127) / 128, ke = (kb + 3) & ~3;
  const size_t blk = (size_t)blockIdx.x * 8 + threadIdx.x / 32;
  if (blk >= (size_t)M * ke) return;
  const size_t r = blk / ke;
  const int b = (int)(blk % ke), l = threadIdx.x & 31;
  if (b >= kb) {
    if (l == 0) exps[r * ke + b] = 0;
    return;
  }
  const int c = 128 * b + 4 * l;
  const f32x4 y = c < F ? *(const f32x4*)(h + r * F + c) : f32x4{0.f, 0.f, 0.f, 0.f};
  const float m = lanes_max<32>(fmaxf(fmaxf(finite_abs(y.x), finite_abs(y.y)), fmaxf(finite_abs(y.z), finite_abs(y.w))));
  const int E = block_exp(m);
  *(uint32_t*)(q + r * 128 * kb + c) = codes4(y.x, y.y, y.z, y.w, inv_scale(E));
  if (l == 0) exps[r * ke + b] = (uint8_t)E;
}

// One 128 x 128 block per workgroup: 16 lanes read the 128 entries of a row
// (lanes across rows, as the packed order has them, would touch a line each),
// the codes are put in order in LDS and leave as the block's eight 2 KB tiles.
// 22016 x 4096 bf16: 54.3 us, 5.0 TB/s (78 us with lanes across rows); fp32 84 us, 5.35.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void pack_linear8_kernel(const T* src, uint8_t* dst, int N, int K) {
  __shared__ __attribute__((aligned(16))) uint8_t out[8 * 2048];
  __shared__ float red[4];
  const int kbn = blocks8(K), ke = ke8(K), tiles = (N + 15) / 16;
  const int kb = blockIdx.x % kbn, nb = blockIdx.x / kbn, tid = threadIdx.x;
  const int r = tid >> 4, c = tid & 15;                // row of a tile, unit of eight entries
  Eight v[8];
  float m = 0.f;
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    const int n = 128 * nb + 16 * t + r;
    v[t] = load8<T, VEC>(src + (size_t)min(n, N - 1) * K, 16 * kb + c, n < N ? K : 0);
  }
#pragma unroll
  for (int t = 0; t < 8; ++t)
#pragma unroll
    for (int e = 0; e < 8; ++e) m = fmaxf(m, finite_abs(v[t].v[e]));
  m = lanes_max<64>(m);
  if ((tid & 63) == 0) red[tid >> 6] = m;
  __syncthreads();
  const int E = block_exp(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
  const float sc = inv_scale(E);
#pragma unroll
  for (int t = 0; t < 8; ++t)
    *(uint2*)(out + t * 2048 + (c >> 3) * 1024 + (((c & 7) >> 1) * 16 + r) * 16 + (c & 1) * 8) =
        make_uint2(codes4(v[t].v[0], v[t].v[1], v[t].v[2], v[t].v[3], sc), codes4(v[t].v[4], v[t].v[5], v[t].v[6], v[t].v[7], sc));
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int u = j * 256 + tid, t = 8 * nb + (u >> 7);
    if (t < tiles) *(u32x4*)(dst + ((size_t)t * kbn + kb) * 2048 + (u & 127) * 16) = *(const u32x4*)(out + u * 16);
  }
  uint8_t* exps = dst + (size_t)tiles * kbn * 2048 + (size_t)nb * ke;
  if (tid == 0) exps[kb] = (uint8_t)E;
  if (kb == kbn - 1 && tid < ke - kbn) exps[kbn + tid] = 0;
}

template <typename TX, typename TG, int R, int NS>
static void norm8_v(const Norm8Params& p, int th, bool vec, hipStream_t s) {
  if (vec) hipLaunchKernelGGL((add_rmsnorm8_kernel<TX, TG, R, NS, true>), dim3(p.M), dim3(th), 0, s, p);
  else hipLaunchKernelGGL((add_rmsnorm8_kernel<TX, TG, R, NS, false>), dim3(p.M), dim3(th), 0, s, p);
}
template <typename TX, typename TG, int R> static void norm8_n(const Norm8Params& p, int th, bool vec, hipStream_t s) {
  if (p.n_add == 0) norm8_v<TX, TG, R, 0>(p, th, vec, s);
  else if (p.n_add == 1) norm8_v<TX, TG, R, 1>(p, th, vec, s);
  else norm8_v<TX, TG, R, NORM8_MAX_ADD>(p, th, vec, s);
}
template <typename TX, typename TG> static void norm8_r(const Norm8Params& p, bool vec, hipStream_t s) {
  const int units = 16 * blocks8(p.d), r = units <= 256 ? 1 : units <= 1024 ? 2 : 4, th = (units + 64 * r - 1) / (64 * r) * 64;
  if (r == 1) norm8_n<TX, TG, 1>(p, th, vec, s);
  else if (r == 2) norm8_n<TX, TG, 2>(p, th, vec, s);
  else norm8_n<TX, TG, 4>(p, th, vec, s);
}

hipError_t launch_add_rmsnorm8(int x_dtype, int gain_dtype, const Norm8Params& p, hipStream_t s) {
  if (p.M <= 0) return hipSuccess;
  if (p.d < 1 || p.d > NORM8_MAX_D || p.n_add < 0 || p.n_add > NORM8_MAX_ADD) return hipErrorInvalidValue;
  // whole aligned units in every row of every operand
  const uintptr_t all = (uintptr_t)p.x | (uintptr_t)p.gain | (p.n_add ? (uintptr_t)p.add | (uintptr_t)p.x_out : 0);
  const bool vec = p.d % 8 == 0 && all % 16 == 0;
  if (x_dtype == 0) {
    if (gain_dtype == 0) norm8_r<bf16_t, bf16_t>(p, vec, s);
    else norm8_r<bf16_t, float>(p, vec, s);
  } else {
    if (gain_dtype == 0) norm8_r<float, bf16_t>(p, vec, s);
    else norm8_r<float, float>(p, vec, s);
  }
  return hipGetLastError();
}

hipError_t launch_quantise_rows8(const float* h, uint8_t* q, uint8_t* exps, int M, int F, hipStream_t s) {
  if (M <= 0) return hipSuccess;
  const int ke = ((F + 127) / 128 + 3) & ~3;
  const size_t blocks = ((size_t)M * ke + 7) / 8;
  hipLaunchKernelGGL(quantise_rows8_kernel, dim3((uint32_t)blocks), dim3(256), 0, s, h, q, exps, M, F);
  return hipGetLastError();
}

hipError_t launch_pack_linear8(int dtype, const void* src, void* dst, int N, int K, hipStream_t s) {
  if (N < 1 || K < 1) return hipErrorInvalidValue;
  const size_t blocks = (size_t)((N + 127) / 128) * ((K + 127) / 128);
  if (blocks > 0x7fffffff) return hipErrorInvalidValue;
  const dim3 grid((uint32_t)blocks), th(256);
  const bool vec = K % 8 == 0 && (uintptr_t)src % 16 == 0;
  uint8_t* d = (uint8_t*)dst;
  if (dtype == 0) {
    if (vec) hipLaunchKernelGGL((pack_linear8_kernel<bf16_t, true>), grid, th, 0, s, (const bf16_t*)src, d, N, K);
    else hipLaunchKernelGGL((pack_linear8_kernel<bf16_t, false>), grid, th, 0, s, (const bf16_t*)src, d, N, K);
  } else {
    if (vec) hipLaunchKernelGGL((pack_linear8_kernel<float, true>), grid, th, 0, s, (const float*)src, d, N, K);
    else hipLaunchKernelGGL((pack_linear8_kernel<float, false>), grid, th, 0, s, (const float*)src, d, N, K);
  }
  return hipGetLastError();
}

}  // namespace sd
