// Products of 8-bit operands (format: rows8.hip):
//   out[m, n] = sum_b 2^(E_mb + F_nb - 254) sum_{k in block b} q[m, k] w[n, k]
// over the 128-entry blocks b of K, accumulated in fp32.
//
// The weight is the matrix instruction's first operand, so a lane's four
// results are four consecutive columns n of one row m: stores are 16 bytes
// wide and one row scale serves them all.
#include "sd_internal.h"

#include <algorithm>

namespace sd {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr uint32_t OOB8 = 0x80000000u;   // a load there returns zero and reads nothing
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc8(const void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, (int)bytes, 0x00020000);
}
template <bool NT> __device__ __forceinline__ u32x4 load16(__amdgpu_buffer_rsrc_t r, uint32_t off) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, NT ? 2 : 0));
}

// The 32 codes that a lane holds of a 16 x 128 operand tile (two 16-byte units)
// as fp16, exactly: e4m3's values are a subset.
struct Frag16 { f16x8 v[4]; };
__device__ __forceinline__ Frag16 widen(const u32x4 (&c)[2]) {
  Frag16 r;
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)c[h][e], 1.0f, false);
      const f16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)c[h][e], 1.0f, true);
      f16x8& d = r.v[2 * h + e / 2];
      d[4 * (e & 1)] = lo.x;
      d[4 * (e & 1) + 1] = lo.y;
      d[4 * (e & 1) + 2] = hi.x;
      d[4 * (e & 1) + 3] = hi.y;
    }
  return r;
}

__device__ __forceinline__ float silu8(float g) { return g / (1.0f + expf(-g)); }

// One workgroup: 16 NT columns x up to 16 MT rows; its KW waves take the
// 128-entry blocks of K in turn and add their sums through LDS in wave order.
// Every wave keeps the next block's loads in flight while it multiplies one.
//
// The products run on fp16 operands: a block's sum of exact fp32 products is
// scaled and added in fp32.  The 8-bit matrix instruction drops low bits of
// the products it adds (1.3e-5 of the sums for normal data, at any K, against
// 1e-7 here), which fp32 outputs would show.
template <int MT, int NT, int EPI, int KW>
__global__ __launch_bounds__(64 * KW) void gemm8_kernel(Gemm8Params p) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, g = lane >> 4;
  const int kb = blocks8(p.K), ke = ke8(p.K), K8 = 128 * kb;
  const int tiles = (p.N + 15) / 16, gx = (tiles + NT - 1) / NT;
  const int bx = blockIdx.x % gx, bz = blockIdx.x / gx;
  const int tile0 = bx * NT, ntile = min(NT, tiles - tile0);
  const int m0 = bz * 16 * MT, mrows = min(16 * MT, p.M - m0);
  const uint32_t tile_bytes = (uint32_t)kb * 2048u;
  const __amdgpu_buffer_rsrc_t wr = rsrc8(p.w + (size_t)tile0 * tile_bytes, ntile * tile_bytes);
  const __amdgpu_buffer_rsrc_t ar = rsrc8(p.q + (size_t)m0 * K8, (uint32_t)mrows * K8);
  const __amdgpu_buffer_rsrc_t er = rsrc8(p.exps + (size_t)m0 * ke, (uint32_t)mrows * ke);
  const __amdgpu_buffer_rsrc_t fr = rsrc8(p.wexps + (size_t)(tile0 / 8) * ke, ke);   // NT divides 8

  f32x4 acc[NT][MT];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};

  u32x4 ws[2][NT][2], as[2][MT][2];
  int we[2], ae[2][MT];
  auto load = [&]<int S>(int b) {
    const bool ok = b < kb;
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        ws[S][j][h] = load16<true>(wr, ok ? j * tile_bytes + (uint32_t)b * 2048u + 1024u * h + lane * 16u : OOB8);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int m = 16 * i + r16;
      const bool row = ok && m < mrows;
#pragma unroll
      for (int h = 0; h < 2; ++h)
        as[S][i][h] = load16<false>(ar, row ? (uint32_t)m * K8 + 128u * b + 64u * h + 16u * g : OOB8);
      ae[S][i] = __builtin_amdgcn_raw_buffer_load_b8(er, row ? (uint32_t)m * ke + b : OOB8, 0, 0);
    }
    we[S] = __builtin_amdgcn_raw_buffer_load_b8(fr, ok ? (uint32_t)b : OOB8, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  auto compute = [&]<int S>() {
    Frag16 a[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) a[i] = widen(as[S][i]);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const Frag16 w = widen(ws[S][j]);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < 4; ++u) s = __builtin_amdgcn_mfma_f32_16x16x32_f16(w.v[u], a[i].v[u], s, 0, 0, 0);
        const int e = (ae[S][i] & 255) + (we[S] & 255) - 254;
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[j][i][v] += ldexpf(s[v], e);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  load.template operator()<0>(wave);
  for (int b = wave; b < kb; b += 2 * KW) {
    load.template operator()<1>(b + KW);
    compute.template operator()<0>();
    load.template operator()<0>(b + 2 * KW);
    compute.template operator()<1>();
  }

  // sums over the waves, in wave order; unit u (a tile, or a gate tile and its
  // up tile) is finished by wave u % KW
  __shared__ f32x4 red[KW][NT * MT][64];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < MT; ++i) red[wave][j * MT + i][lane] = acc[j][i];
  __syncthreads();
  auto total = [&](int j, int i) {
    f32x4 t = red[0][j * MT + i][lane];
#pragma unroll
    for (int w = 1; w < KW; ++w) t += red[w][j * MT + i][lane];
    return t;
  };
  constexpr int TPU = EPI == EPI8_SWIGLU ? 2 : 1;
#pragma unroll
  for (int j = 0; j < NT; j += TPU)
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int m = 16 * i + r16;
      if ((j / TPU * MT + i) % KW != wave || j >= ntile || m >= mrows) continue;
      const size_t row = m0 + m;
      if constexpr (EPI == EPI8_SWIGLU) {
        const f32x4 gt = total(j, i), up = total(j + 1, i);
        f32x4 h;
#pragma unroll
        for (int v = 0; v < 4; ++v) h[v] = silu8(gt[v]) * up[v];
        *(f32x4*)((float*)p.out + row * (p.N / 2) + 8 * (tile0 + j) + 4 * g) = h;
      } else {
        const f32x4 o = total(j, i);
        const int n = 16 * (tile0 + j) + 4 * g;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          if (n + v >= p.N) continue;
          const size_t at = row * p.ldo + n + v;
          const float y = p.add ? p.add[at] + o[v] : o[v];
          if (p.bf16) ((__bf16*)p.out)[at] = (__bf16)y;
          else ((float*)p.out)[at] = y;
        }
      }
    }
}

template <int MT, int NT, int EPI, int KW>
static hipError_t gemm8_t(const Gemm8Params& p, hipStream_t s) {
  const size_t gx = ((p.N + 15) / 16 + NT - 1) / NT, gz = (p.M + 16 * MT - 1) / (16 * MT);
  if (gx * gz > 0x7fffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL((gemm8_kernel<MT, NT, EPI, KW>), dim3((uint32_t)(gx * gz)), dim3(64 * KW), 0, s, p);
  return hipGetLastError();
}
template <int EPI> static hipError_t gemm8_m(const Gemm8Params& p, hipStream_t s) {
  switch (std::min(4, (p.M + 15) / 16)) {
    case 1: return gemm8_t<1, 2, EPI, 4>(p, s);
    case 2: return gemm8_t<2, 2, EPI, 4>(p, s);
    case 3: return gemm8_t<3, 2, EPI, 4>(p, s);
    default: return gemm8_t<4, 2, EPI, 4>(p, s);
  }
}

hipError_t launch_gemm8(int epi, const Gemm8Params& p, hipStream_t s) {
  if (p.M <= 0) return hipSuccess;
  if (p.N < 1 || p.K < 1 || p.K > LINEAR8_MAX_K || p.M > LINEAR8_MAX_MN || p.N > LINEAR8_MAX_MN)
    return hipErrorInvalidValue;
  if (epi == EPI8_STORE) return gemm8_m<EPI8_STORE>(p, s);
  if (epi == EPI8_SWIGLU && p.N % 32 == 0) return gemm8_m<EPI8_SWIGLU>(p, s);
  return hipErrorInvalidValue;
}

}  // namespace sd
