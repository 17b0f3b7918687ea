// Attention over a paged KV cache held in 4 bits (format: codes4.h):
//   o = sum_j softmax_j(scale q . k_j) v_j
// over the positions j that a row sees: up to its own (causal), or all of its
// sequence's.
//
// One workgroup takes a row and a query head: each thread scores a key, and
// the weighted values are summed with a thread per dimension and group of keys.
#include "codes4.h"

#include <math.h>

namespace sd {

template <typename T, int HD> __global__ __launch_bounds__(256) void attention4_kernel(Attn4Params p) {
  using P = Page4<HD>;
  constexpr int GROUPS = 256 / HD;
  __shared__ float s_q[HD], s_p[256], s_red[4], s_o[256];
  __shared__ int s_page[16];
  const int row = blockIdx.x, h = blockIdx.y, kvh = h / (p.H / p.KV);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int b, pos;
  if (!row_place(p.rows, row, b, pos)) return;
  int n = p.causal ? pos + 1 : p.rows.len[b];           // keys
  const bool past = n > 16 * p.rows.W;                  // ... the table has no pages for
  if (past) n = 16 * p.rows.W;
  const T* const q = (const T*)p.q + (size_t)row * p.ldq + h * HD;
  if (tid < HD) s_q[tid] = Store<T>::load(q, tid) * p.scale;
  float m = -INFINITY, l = 0.f, o = 0.f;
  const int d = tid % HD, grp = tid / HD;
  for (int j0 = 0; j0 < n; j0 += 256) {
    __syncthreads();
    if (tid < 16) s_page[tid] = j0 + 16 * tid < n ? row_page(p.rows, b, j0 + 16 * tid, p.n_blocks) : -1;
    __syncthreads();
    const int j = j0 + tid, page = s_page[tid / 16], t = tid % 16;
    float z = -INFINITY;
    if (j < n) {
      z = 0.f;
      const uint8_t* const pg = p.pool + ((size_t)max(page, 0) * p.KV + kvh) * P::BYTES;
      for (int c = 0; c < HD / 8; ++c) {
        float x[8];
        decode4(page < 0 ? 0u : *(const uint32_t*)(pg + P::key(t, 8 * c)), scale4(page < 0 ? 255u : pg[P::key_scale(t, c / 4)]), x);
#pragma unroll
        for (int e = 0; e < 8; ++e) z += s_q[8 * c + e] * x[e];
      }
    }
    float top = z;
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor(top, k));
    if (lane == 0) s_red[wave] = top;
    __syncthreads();
    const float m_new = fmaxf(m, fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3])));
    const float old = m == m_new ? 1.f : expf(m - m_new);
    const float w = j < n ? expf(z - m_new) : 0.f;
    float sum = w;
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) sum += __shfl_xor(sum, k);
    __syncthreads();
    if (lane == 0) s_red[wave] = sum;
    s_p[tid] = w;
    __syncthreads();
    l = l * old + (s_red[0] + s_red[1] + s_red[2] + s_red[3]);
    o *= old;
    m = m_new;
    for (int k = grp; k < min(256, n - j0); k += GROUPS) {
      const int pk = s_page[k / 16];
      const uint8_t* const pg = p.pool + ((size_t)max(pk, 0) * p.KV + kvh) * P::BYTES;
      const int r = d / (HD / 16), e = d % (HD / 16);
      const uint32_t c = pk < 0 ? 0u : pg[P::value(k % 16, r) + e / 2];
      const f32x2 v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale4(pk < 0 ? 255u : pg[P::value_scale(k % 16, d / 32)]), 0);
      o += s_p[k] * (e & 1 ? v[1] : v[0]);
    }
  }
  s_o[tid] = o;
  __syncthreads();
  if (tid < HD) {
    float sum = 0.f;
    for (int k = 0; k < GROUPS; ++k) sum += s_o[k * HD + tid];
    const float out = past ? NAN : n > 0 ? sum / l : 0.f;
    T* const dst = (T*)p.out + (size_t)row * p.ldo + h * HD;
    if constexpr (sizeof(T) == 2) dst[tid] = __builtin_bit_cast(bf16_t, (__bf16)out);
    else dst[tid] = out;
  }
}

hipError_t launch_attention4(int dtype, int hd, const Attn4Params& p, hipStream_t s) {
  const dim3 grid(p.M, p.H);
  if (dtype == 1) {
    if (hd == 128) attention4_kernel<float, 128><<<grid, 256, 0, s>>>(p);
    else attention4_kernel<float, 64><<<grid, 256, 0, s>>>(p);
  } else {
    if (hd == 128) attention4_kernel<bf16_t, 128><<<grid, 256, 0, s>>>(p);
    else attention4_kernel<bf16_t, 64><<<grid, 256, 0, s>>>(p);
  }
  return hipGetLastError();
}

}  // namespace sd
