// 8-bit operands of the feed-forward network: RMSNorm with an 8-bit output,
// quantisation of fp32 rows, and the packing of weight matrices (format: codes8.h).
#include "sd_internal.h"
#include "codes8.h"

namespace sd {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// maximum over the 32 lanes that hold a block (4 entries each)
__device__ __forceinline__ float half_wave_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}

// entries 4 i .. 4 i + 3 of a row of n entries, zero past the end; VEC: rows are whole aligned units of four
template <typename T, bool VEC> __device__ __forceinline__ f32x4 load4(const T* row, int i, int n) {
  if constexpr (VEC) {
    if (4 * i >= n) return f32x4{0.f, 0.f, 0.f, 0.f};
    if constexpr (sizeof(T) == 4) {
      return ((const f32x4*)row)[i];
    } else {
      const uint2 u = ((const uint2*)row)[i];
      return f32x4{__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16),
                   __uint_as_float(u.y & 0xffff0000u)};
    }
  } else {
    f32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = 4 * i + e < n ? Store<T>::load(row, 4 * i + e) : 0.f;
    return v;
  }
}
template <typename T, bool VEC> __device__ __forceinline__ void store4(T* row, int i, int n, f32x4 v) {
  if constexpr (VEC) {
    if (4 * i >= n) return;
    if constexpr (sizeof(T) == 4) ((f32x4*)row)[i] = v;
    else
      ((uint2*)row)[i] = make_uint2(bf16_bits(v.x) | bf16_bits(v.y) << 16, bf16_bits(v.z) | bf16_bits(v.w) << 16);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (4 * i + e >= n) continue;
      if constexpr (sizeof(T) == 4) row[4 * i + e] = v[e];
      else row[4 * i + e] = (bf16_t)bf16_bits(v[e]);
    }
  }
}

// Residual addition, RMSNorm and 8-bit output of one row per workgroup of TH
// threads (R units of four entries each):
//   s = x + add_0 + ... + add_{n-1}         summed in 64 bits, stored in x's type
//   y = s / sqrt(mean(s^2) + eps) * gain    in 64 bits, rounded to fp32
//   q, E = codes and exponents of y
// 64-bit sums and norm: codes are a function of the input alone, not of the
// order of a sum (the arithmetic hides behind the memory latency).
// The addends are loaded before the first is added (NS of them, those past n_add
// as zeros), or for the longest rows, which fill the registers, one at a time (NS < 0).
template <typename TX, typename TG, int TH, int R, int NS, bool VEC>
__global__ __launch_bounds__(TH) void add_rmsnorm8_kernel(Norm8Params p) {
  __shared__ double red[TH / 64];
  const size_t r = blockIdx.x;
  const int d = p.d, tid = threadIdx.x;
  const TX* x = (const TX*)p.x + r * d;
  f32x4 v[R], a[NS > 0 ? NS : 1][R], g[R];
#pragma unroll
  for (int k = 0; k < R; ++k) v[k] = load4<TX, VEC>(x, tid + TH * k, d);
#pragma unroll
  for (int j = 0; j < NS; ++j)
#pragma unroll
    for (int k = 0; k < R; ++k)
      a[j][k] = j < p.n_add ? load4<TX, VEC>((const TX*)p.add + ((size_t)j * p.M + r) * d, tid + TH * k, d)
                            : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < R; ++k) g[k] = load4<TG, VEC>((const TG*)p.gain, tid + TH * k, d);
  if constexpr (NS != 0) {
    double s[R][4];
#pragma unroll
    for (int k = 0; k < R; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[k][e] = (double)v[k][e];
#pragma unroll
        for (int j = 0; j < NS; ++j) s[k][e] += (double)a[j][k][e];
      }
    if constexpr (NS < 0) {
#pragma unroll 1
      for (int j = 0; j < p.n_add; ++j)
#pragma unroll
        for (int k = 0; k < R; ++k) {
          const f32x4 t = load4<TX, VEC>((const TX*)p.add + ((size_t)j * p.M + r) * d, tid + TH * k, d);
#pragma unroll
          for (int e = 0; e < 4; ++e) s[k][e] += (double)t[e];
        }
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        v[k][e] = sizeof(TX) == 4 ? (float)s[k][e] : bf2f((bf16_t)bf16_bits((float)s[k][e]));
      store4<TX, VEC>((TX*)p.x_out + r * d, tid + TH * k, d, v[k]);
    }
  }
  double ss = 0;
#pragma unroll
  for (int k = 0; k < R; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) ss += (double)v[k][e] * (double)v[k][e];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) ss += __shfl_xor(ss, o);
  if ((tid & 63) == 0) red[tid >> 6] = ss;
  __syncthreads();
  ss = 0;
#pragma unroll
  for (int w = 0; w < TH / 64; ++w) ss += red[w];
  const double inv = 1.0 / sqrt(ss / d + (double)p.eps);
  const int kb = (d + 127) / 128, ke = (kb + 3) & ~3;
#pragma unroll
  for (int k = 0; k < R; ++k) {
    const int i = tid + TH * k;
    f32x4 y;
    float m = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      y[e] = (float)((double)v[k][e] * inv * (double)g[k][e]);
      if (4 * i + e >= d) y[e] = 0.f;     // a NaN of the row stays out of the padding
      m = fmaxf(m, finite_abs(y[e]));
    }
    m = half_wave_max(m);
    if (i < 32 * kb) {
      const int E = block_exp(m);
      ((uint32_t*)(p.q + r * 128 * kb))[i] = codes4(y.x, y.y, y.z, y.w, inv_scale(E));
      if ((i & 31) == 0) p.exps[r * ke + i / 32] = (uint8_t)E;
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
  const float m = half_wave_max(fmaxf(fmaxf(finite_abs(y.x), finite_abs(y.y)), fmaxf(finite_abs(y.z), finite_abs(y.w))));
  const int E = block_exp(m);
  *(uint32_t*)(q + r * 128 * kb + c) = codes4(y.x, y.y, y.z, y.w, inv_scale(E));
  if (l == 0) exps[r * ke + b] = (uint8_t)E;
}

// One 128 x 128 block per workgroup: unit u (16 codes of a row) of the block's
// eight 2 KB tiles is row 16 (u / 128) + u % 16, columns 64 ((u / 64) % 2) +
// 16 ((u / 16) % 4) ..; each thread takes 4 units, so a wave reads 64 or 128
// bytes of 16 rows and writes 1 KB runs.  Bound by the copy.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void pack_linear8_kernel(const T* src, uint8_t* dst, int N, int K) {
  __shared__ float red[4];
  const int kbn = (K + 127) / 128, ke = (kbn + 3) & ~3, tiles = (N + 15) / 16;
  const int kb = blockIdx.x % kbn, nb = blockIdx.x / kbn, tid = threadIdx.x;
  f32x4 v[4][4];
  float m = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int u = j * 256 + tid;
    const int n = 128 * nb + 16 * (u >> 7) + (u & 15), k = 128 * kb + 64 * ((u >> 6) & 1) + 16 * ((u >> 4) & 3);
    const T* row = src + (size_t)min(n, N - 1) * K;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      v[j][c] = n < N ? load4<T, VEC>(row, k / 4 + c, K) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 4; ++e) m = fmaxf(m, finite_abs(v[j][c][e]));
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  if ((tid & 63) == 0) red[tid >> 6] = m;
  __syncthreads();
  const int E = block_exp(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
  const float inv = inv_scale(E);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int u = j * 256 + tid, t = 8 * nb + (u >> 7);
    if (t >= tiles) continue;
    u32x4 o;
#pragma unroll
    for (int c = 0; c < 4; ++c) o[c] = codes4(v[j][c].x, v[j][c].y, v[j][c].z, v[j][c].w, inv);
    *(u32x4*)(dst + ((size_t)t * kbn + kb) * 2048 + (u & 127) * 16) = o;
  }
  uint8_t* exps = dst + (size_t)tiles * kbn * 2048 + (size_t)nb * ke;
  if (tid == 0) exps[kb] = (uint8_t)E;
  if (kb == kbn - 1 && tid < ke - kbn) exps[kbn + tid] = 0;
}

template <typename TX, typename TG, int TH, int R, int NS>
static void norm8_v(const Norm8Params& p, bool vec, hipStream_t s) {
  if (vec) hipLaunchKernelGGL((add_rmsnorm8_kernel<TX, TG, TH, R, NS, true>), dim3(p.M), dim3(TH), 0, s, p);
  else hipLaunchKernelGGL((add_rmsnorm8_kernel<TX, TG, TH, R, NS, false>), dim3(p.M), dim3(TH), 0, s, p);
}
template <typename TX, typename TG, int TH, int R>
static void norm8_n(const Norm8Params& p, bool vec, hipStream_t s) {
  if (p.n_add == 0) norm8_v<TX, TG, TH, R, 0>(p, vec, s);
  else if (p.n_add == 1) norm8_v<TX, TG, TH, R, 1>(p, vec, s);
  else norm8_v<TX, TG, TH, R, TH == 1024 ? -1 : NORM8_MAX_ADD>(p, vec, s);
}
template <typename TX, typename TG> static void norm8_r(const Norm8Params& p, bool vec, hipStream_t s) {
  const int units = (p.d + 127) / 128 * 32;
  if (units <= 256) norm8_n<TX, TG, 256, 1>(p, vec, s);
  else if (units <= 512) norm8_n<TX, TG, 256, 2>(p, vec, s);
  else if (units <= 1024) norm8_n<TX, TG, 256, 4>(p, vec, s);
  else if (units <= 2048) norm8_n<TX, TG, 512, 4>(p, vec, s);
  else norm8_n<TX, TG, 1024, 4>(p, vec, s);
}

hipError_t launch_add_rmsnorm8(int x_dtype, int gain_dtype, const Norm8Params& p, hipStream_t s) {
  if (p.M <= 0) return hipSuccess;
  if (p.d < 1 || p.d > NORM8_MAX_D || p.n_add < 0 || p.n_add > NORM8_MAX_ADD) return hipErrorInvalidValue;
  // whole units of four at their alignment in every row of every operand
  const uintptr_t fx = (uintptr_t)p.x | (p.n_add ? (uintptr_t)p.add | (uintptr_t)p.x_out : 0);
  const bool vec = p.d % 4 == 0 && fx % (x_dtype == 0 ? 8 : 16) == 0 && (uintptr_t)p.gain % (gain_dtype == 0 ? 8 : 16) == 0;
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
  const bool vec = K % 4 == 0 && (uintptr_t)src % (dtype == 0 ? 8 : 16) == 0;
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
