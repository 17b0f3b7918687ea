// Products of 8-bit operands (format: codes8.h):
//   out[m, n] = sum_b 2^(E_mb + F_nb - 254) sum_{k in block b} q[m, k] w[n, k]
// over the 128-entry blocks b of K, accumulated in fp32.
//
// The weight is the matrix instruction's first operand, so a lane's four
// results are four consecutive columns n of one row m: stores are 16 bytes
// wide and one row scale serves them all.
#include "sd_internal.h"
#include "codes8.h"

#include <algorithm>
#include <cmath>
#include <utility>

namespace sd {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr uint32_t OOB8 = 0x80000000u;   // a load there returns zero and reads nothing
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc8(const void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, (int)bytes, 0x00020000);
}
template <bool NT> __device__ __forceinline__ u32x4 load16(__amdgpu_buffer_rsrc_t r, uint32_t off) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, NT ? 2 : 0));
}

struct Pair16 { u32x4 lo, hi; };   // the two 16-byte units of a lane's operand

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

// out[row, n .. n + 3] (those below N) of a STORE epilogue
__device__ __forceinline__ void store_out(const Gemm8Params& p, size_t row, int n, f32x4 o) {
  const size_t at = row * p.ldo + n;
  if (p.wide && n + 3 < p.N) {
    if (p.add) o += *(const f32x4*)(p.add + at);
    if (p.bf16) {
      *(uint2*)((uint16_t*)p.out + at) = make_uint2(bf16_bits(o.x) | bf16_bits(o.y) << 16, bf16_bits(o.z) | bf16_bits(o.w) << 16);
    } else {
      *(f32x4*)((float*)p.out + at) = o;
    }
    return;
  }
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    if (n + v >= p.N) continue;
    const float y = p.add ? p.add[at + v] + o[v] : o[v];
    if (p.bf16) ((uint16_t*)p.out)[at + v] = (uint16_t)bf16_bits(y);
    else ((float*)p.out)[at + v] = y;
  }
}

__device__ __forceinline__ float silu8(float g) { return g / (1.0f + expf(-g)); }

// Waits for all but N of this wave's loads and for its LDS reads.
template <int N> __device__ __forceinline__ void wait_loads() {
  static_assert(N >= 0 && N < 64, "vmcnt is 6 bits");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));
}

// 2^(E + F - 254) of two scale exponents, as a float: from 2^-126 to 2^127 (a
// smaller one counts as zero: the sums that it would scale are below 2^-101; a
// larger one as 2^127); 255, which no kernel here writes, is NaN
__device__ __forceinline__ float scale_of(int E, int F) {
  return __uint_as_float(max(E, F) == 255 ? 0x7fc00000u : (uint32_t)min(max(E + F - 127, 0), 254) << 23);
}
__device__ __forceinline__ void add_scaled(f32x4& acc, f32x4 s, float f) {
#pragma unroll
  for (int v = 0; v < 4; ++v) acc[v] = fmaf(s[v], f, acc[v]);
}

// K ranges: ksplit of them, whole groups of four blocks (which share a load of
// scales), none empty if the launch has checked range8(kb, ksplit) (ksplit - 1) < kb
__host__ __device__ __forceinline__ int range8(int kb, int ksplit) { return ((kb + ksplit - 1) / ksplit + 3) & ~3; }

// Product for few rows (up to 64), bound by streaming the weights: a workgroup
// takes up to NT tiles of 16 columns and all rows (MT tiles), its KW waves the
// 128-entry blocks of its K range in turn, and their sums are added through LDS
// in wave order.  A wave loads its weight tiles into registers and its rows
// into a part of LDS of its own, D - 1 blocks ahead, and waits for nothing but
// its own loads.  (The rows go through LDS because a load straight into the
// operand's layout touches 16 rows' lines: four times the address work of one
// that reads whole lines.)
//
// The products run on fp16 operands: a block's sum of exact fp32 products is
// scaled and added in fp32.  The 8-bit matrix instruction drops low bits of
// the products it adds (1.5e-5 of the sums for normal data, at any K, up to 5.1e-5
// for rows with a few large entries, against 1e-7 here; with 32 entries of K
// or 128 an instruction alike), which fp32 outputs would show.
//
// 4096 x 11008: 8 rows 10.5 us (4.3 TB/s), 40 rows 15.7, 64 rows 18.8; gate/up
// 22016 x 4096 without the codes' pass (3 to 5 us): 8 rows 17.5 us (5.2 TB/s), 40
// rows 19.3.  A plain read of the bytes reaches 6.3 to 6.8 TB/s; what grows with
// the rows is their reads from L2, once per workgroup.
constexpr int STREAM8_KE = 128;          // bytes of a row's scales: K up to 16384
template <int MT, int NT, int KW, int D, int EPI>
__global__ __launch_bounds__(64 * KW) void gemm8_kernel(Gemm8Params p) {
  constexpr int TPU = EPI == EPI8_SWIGLU ? 2 : 1;            // tiles of a finishing unit
  constexpr int STAGE = MT * 2048;                           // bytes of a block's rows
  constexpr int PS = 2 * MT + 2 * NT;                        // loads of a block
  constexpr int RED = KW * NT * MT * 1024, BUF = KW * D * STAGE > RED ? KW * D * STAGE : RED;
  constexpr int SCALES = (16 * MT + 2) * STREAM8_KE;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[BUF + SCALES];
  static_assert(BUF + SCALES <= 160 * 1024 && (D - 1) * PS < 64, "LDS of a CU, loads in flight");

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, g = lane >> 4;
  const int kb = blocks8(p.K), ke = ke8(p.K), K8 = 128 * kb;
  // the columns' tiles (SwiGLU: pairs of a gate tile and its up tile) are dealt
  // to the workgroups of a K range evenly, a contiguous run of at most NT tiles each
  const int tiles = (p.N + 15) / 16, gx = gridDim.x / p.ksplit;
  const int bx = blockIdx.x % gx, split = blockIdx.x / gx;
  const int units = tiles / TPU, base = units / gx, extra = units % gx;
  const int tile0 = (bx * base + min(bx, extra)) * TPU, ntile = (base + (bx < extra ? 1 : 0)) * TPU;
  const int sps = range8(kb, p.ksplit), s_lo = split * sps, s_hi = min(s_lo + sps, kb);   // blocks of this K range
  const int mrows = p.M;
  const uint32_t tile_bytes = (uint32_t)kb * 2048u;
  const uint8_t* Wp = p.w + (size_t)tile0 * tile_bytes;
  const uint8_t* Ap = p.q;
  uint8_t* const own = smem + wave * D * STAGE;

  // the scales of the rows, then of the columns (one or two rows of them) are copied to LDS:
  // 256 bytes a load (a load of one block's scales would touch a line per row)
  uint8_t* const sc = smem + BUF;
  const uint8_t* const wsc = sc + mrows * ke;
  {
    const __amdgpu_buffer_rsrc_t er = rsrc8(p.exps, (uint32_t)mrows * ke);
    const int wn = ((tile0 + ntile - 1) / 8 - tile0 / 8 + 1) * ke;
    const __amdgpu_buffer_rsrc_t fr = rsrc8(p.wexps + (size_t)(tile0 / 8) * ke, wn);
    const int n = mrows * ke;
    for (int o = wave * 256; o < n + wn; o += KW * 256) {
      const uint32_t at = o + 4 * lane;
      const bool rows = (int)at < n;
      // (the part in which the rows' scales end, and the columns', go through registers)
      if (o < n && o + 256 <= n) {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(er, (__attribute__((address_space(3))) void*)(sc + o), 4, at, 0, 0, 0);
      } else {
        const uint32_t x = rows ? __builtin_amdgcn_raw_buffer_load_b32(er, at, 0, 0)
                                : __builtin_amdgcn_raw_buffer_load_b32(fr, at - n, 0, 0);
        if ((int)at < n + wn) *(uint32_t*)(sc + at) = x;
      }
    }
  }

  f32x4 acc[NT][MT];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};

  // eight rows a load, eight lanes to a row's 128 bytes: slot lane % 8 takes unit (lane % 8) ^ (row % 8)
  uint32_t aoff[2 * MT];
#pragma unroll
  for (int k = 0; k < 2 * MT; ++k) {
    const int m = 8 * k + (lane >> 3);
    aoff[k] = m < mrows ? (uint32_t)m * K8 + 16u * ((lane ^ (lane >> 3)) & 7) : OOB8;
  }
  uint32_t woff[NT][2];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int h = 0; h < 2; ++h) woff[j][h] = j < ntile ? j * tile_bytes + 1024u * h + 16u * lane : OOB8;
  const int aswz = r16 * 128 + ((g ^ r16) & 7) * 16;

  const int step8 = tile0 % 8 + ntile > 8 ? 1 : 0;     // tiles from the next multiple of 8 on have the second row of scales
  const uint8_t* srow[MT];                             // this lane's rows' scales
#pragma unroll
  for (int t = 0; t < MT; ++t) srow[t] = sc + min(16 * t + r16, mrows - 1) * ke;

  // block number i of this wave is block KW i + wave of the K range; past the last the
  // buffers are empty: zeros, nothing read
  u32x4 wf[D][NT][2];
  auto load = [&]<int S>(int i) {
    const int b = s_lo + KW * i + wave;
    const bool ok = b < s_hi;
    const __amdgpu_buffer_rsrc_t ar = rsrc8(Ap, ok ? (uint32_t)mrows * K8 : 0u);
    const __amdgpu_buffer_rsrc_t wr = rsrc8(Wp, ok ? ntile * tile_bytes : 0u);
#pragma unroll
    for (int k = 0; k < 2 * MT; ++k) {
      const uint32_t off = aoff[k];
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ar, (__attribute__((address_space(3))) void*)(own + S * STAGE + k * 1024), 16,
                                               off, 128 * b, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        wf[S][j][h] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(wr, woff[j][h], 2048 * b, 2));
    __builtin_amdgcn_sched_barrier(0);
  };
  auto compute = [&]<int S>(int i) {
    wait_loads<(D - 1) * PS>();
    asm volatile("" ::: "memory");
    const uint8_t* st = own + S * STAGE;
    const int b = min(s_lo + KW * i + wave, s_hi - 1);  // (past the last block: its products are zero)
    const int we[2] = {wsc[b], wsc[(NT > 1 ? step8 * ke : 0) + b]};
    u32x4 c[MT][2];
    int e[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      c[t][0] = *(const u32x4*)(st + t * 2048 + aswz);
      c[t][1] = *(const u32x4*)(st + t * 2048 + (aswz ^ 64));
      e[t] = srow[t][b];
    }
    Frag16 a[MT];
    float f[2][MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      a[t] = widen(c[t]);
#pragma unroll
      for (int r = 0; r < (NT > 1 ? 2 : 1); ++r) f[r][t] = scale_of(e[t], we[r]);
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const Frag16 w = widen(wf[S][j]);
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < 4; ++u) s = __builtin_amdgcn_mfma_f32_16x16x32_f16(w.v[u], a[t].v[u], s, 0, 0, 0);
        add_scaled(acc[j][t], s, NT > 1 && tile0 % 8 + j >= 8 ? f[1][t] : f[0][t]);
      }
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  const int n = (s_hi - s_lo - wave + KW - 1) / KW;    // this wave's blocks (maybe none)
  [&]<int... S>(std::integer_sequence<int, S...>) {
    (load.template operator()<S>(S), ...);
  }(std::make_integer_sequence<int, D - 1>());
  wait_loads<(D - 1) * PS>();                          // the scales
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  for (int i = 0; i < n; i += D) {
    [&]<int... S>(std::integer_sequence<int, S...>) {
      ((load.template operator()<(S + D - 1) % D>(i + S + D - 1), compute.template operator()<S>(i + S)), ...);
    }(std::make_integer_sequence<int, D>());
  }
  wait_loads<0>();                                     // the loads past the last block

  // sums over the waves, in wave order; unit u (a tile, or a gate tile and its
  // up tile) is finished by wave u % KW
  __syncthreads();                                     // the waves' buffers have been read
  f32x4(*red)[NT * MT][64] = (f32x4(*)[NT * MT][64])smem;
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
#pragma unroll
  for (int j = 0; j < NT; j += TPU)
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int m = 16 * i + r16;
      if ((j / TPU * MT + i) % KW != wave || j >= ntile || m >= mrows) continue;
      const size_t row = m;
      if constexpr (EPI == EPI8_SWIGLU) {
        const f32x4 gt = total(j, i), up = total(j + 1, i);
        f32x4 h;
#pragma unroll
        for (int v = 0; v < 4; ++v) h[v] = silu8(gt[v]) * up[v];
        *(f32x4*)((float*)p.out + row * (p.N / 2) + 8 * (tile0 + j) + 4 * g) = h;
      } else if constexpr (EPI == EPI8_PART) {
        const int n = 16 * (tile0 + j) + 4 * g;         // ldo is N rounded up to 4
        if (n < p.N) *(f32x4*)((float*)p.out + ((size_t)split * p.M + row) * p.ldo + n) = total(j, i);
      } else {
        store_out(p, row, 16 * (tile0 + j) + 4 * g, total(j, i));
      }
    }
}

// Row-tiled product for more rows: a workgroup of WM x WN waves owns BM rows x
// BN columns, wave (wm, wn) 16 MF rows x 16 NF columns of them.  K advances one
// 128-entry block a stage; a stage's operands and scales are loaded straight
// into one of NB LDS buffers (lane i's bytes land at the fragment's base + 16 i,
// in the order the matrix instruction reads them), NB - 1 stages ahead.  At the
// top of a stage a wave waits for its own loads of it, a barrier makes every
// wave's visible and frees the buffer of the stage before, which the loads of
// stage + NB - 1 then fill.  Every wave issues the same number of loads in every
// stage; those past the operands have an empty buffer range or an offset outside
// it: zeros, nothing read.
//
// With two buffers (tiles of 192 and 256 rows) the rows' loads of the next stage
// go out in the first half of a stage; a second barrier in its middle, when every
// wave has the stage's weights in registers, frees their part of the buffer for
// the weights' loads of the stage after next.  All of them then have at least
// half a stage to arrive (gate/up of 8192 rows on sixteen waves: 755 -> 695 us).
// Eight waves of 128 x 64 read three quarters of what sixteen of 64 x 64 read
// from LDS, whose reads take as long as the products (8192 rows 645 us, 2048 rows
// 220 -> 184 in the same graph).
//
// On the 8-bit instruction 2048 x 4096 x 11008, bf16 out: 82 us, 2.26 PFLOP/s of the
// 2.64 of a large library product (in a graph of such calls 91, of which its loads
// alone would take 78 and its LDS reads and products alone 80); gate/up 2048 x
// 22016 x 4096: 178 us, 2.08 PFLOP/s.
//
// On fp16 operands 155 us and 359 us, 1.2 and 1.03 PFLOP/s of the 1.56 of a large
// library product: the matrix units are busy 0.48 of the cycles (of the first), the
// other vector instructions (3.7 for each matrix instruction: widening, scaling,
// addresses) issue in 0.44, and the waves wait a quarter of theirs for loads.
template <int MF_, int NF_, int WM_, int WN_, int NB_, bool EXACT_> struct Tile8 {
  static constexpr int MF = MF_, NF = NF_, WM = WM_, WN = WN_, NB = NB_;
  static constexpr bool EXACT = EXACT_;
  static constexpr int WAVES = WM * WN, BM = 16 * MF * WM, BN = 16 * NF * WN;
  static constexpr int FA = BM / 16 * 2, FW = BN / 16 * 2;             // 1 KB fragments of a stage
  static constexpr int LA = FA / WAVES, LW = FW / WAVES;
  static constexpr int LE = (BM / 64 + 1 + WAVES - 1) / WAVES;         // 256-byte scale loads of a wave
  static constexpr int STAGE = (FA + FW) * 1024;                       // bytes
  static constexpr int SCALES = LE * WAVES * 256;                      // of four stages
  static constexpr int LDS = NB * STAGE + 2 * SCALES;
  static_assert(FA % WAVES == 0 && FW % WAVES == 0 && BM % 64 == 0, "whole fragments per wave");
  static_assert((NB - 2) * (LA + LW) < 64 && LDS <= 160 * 1024, "loads in flight, LDS of a CU");
};

template <typename C, int EPI>
__global__ __launch_bounds__(64 * C::WAVES, C::WAVES / 4) void gemm8_rows_kernel(Gemm8Params p) {
  constexpr int MF = C::MF, NF = C::NF, NB = C::NB, WAVES = C::WAVES, BM = C::BM, BN = C::BN;
  constexpr int FA = C::FA, FW = C::FW, LA = C::LA, LW = C::LW, LE = C::LE, L = LA + LW;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[C::LDS];
  uint8_t* const lds = smem;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % C::WM, wn = wave / C::WM;
  const int r16 = lane & 15, g = lane >> 4;
  const int kb = blocks8(p.K), ke = ke8(p.K), K8 = 128 * kb;
  const int tiles = (p.N + 15) / 16;
  const int gz = (p.M + BM - 1) / BM;
  // Workgroup w runs on XCD w % 8, which takes one contiguous run of tiles in this
  // order: groups of up to 8 row tiles (of even size); in a group its column tiles;
  // of a column tile the row tiles of each K range.  The 32 workgroups that an XCD
  // runs at a time then share about as many bytes of rows as of weights (8192 x
  // 4096 x 11008, bf16 out: 333 us, 355 with all row tiles of a column tile first).
  int bx, bz, split;
  {
    const int w = blockIdx.x, T8 = gridDim.x >> 3, rem = gridDim.x & 7, x = w & 7;
    const int gx = (tiles + BN / 16 - 1) / (BN / 16), col = gx * p.ksplit;
    const int groups = (gz + 7) / 8, lo = gz / groups, more = gz % groups;   // the first `more` groups have lo + 1 rows
    int tile = x * T8 + min(x, rem) + (w >> 3), rows = lo + 1, z0;
    if (tile < more * rows * col) {
      z0 = tile / (rows * col) * rows;
      tile %= rows * col;
    } else {
      tile -= more * rows * col;
      rows = lo;
      z0 = more + tile / (rows * col) * rows + more * lo;
      tile %= rows * col;
    }
    const int r = tile % (rows * p.ksplit);
    bx = tile / (rows * p.ksplit);
    bz = z0 + r % rows;
    split = r / rows;
  }
  const int sps = range8(kb, p.ksplit), s_lo = split * sps, s_hi = min(s_lo + sps, kb);   // blocks of this K range
  const uint32_t tile_bytes = (uint32_t)kb * 2048u;
  const int mrows = min(BM, p.M - bz * BM), ntile = min(BN / 16, tiles - bx * (BN / 16));
  const uint8_t* Wp = p.w + (size_t)bx * (BN / 16) * tile_bytes;
  const uint8_t* Ap = p.q + (size_t)bz * BM * K8;
  const uint8_t* Ep = p.exps + (size_t)bz * BM * ke;
  const uint8_t* Fp = p.wexps + (size_t)(bx * BN / 128) * ke;
  const int nblk = (16 * ntile + 127) / 128;           // weight scale rows of the tile

  uint32_t aoff[LA], woff[LW], eoff[LE];
#pragma unroll
  for (int k = 0; k < LA; ++k) {
    // eight rows a load, eight lanes to a row's 128 bytes: slot lane % 8 takes unit (lane % 8) ^ (row % 8)
    const int m = 8 * (WAVES * k + wave) + (lane >> 3);
    aoff[k] = m < mrows ? (uint32_t)m * K8 + 16u * ((lane ^ (lane >> 3)) & 7) : OOB8;
  }
#pragma unroll
  for (int k = 0; k < LW; ++k) {
    const int f = WAVES * k + wave;
    woff[k] = (f >> 1) < ntile ? (uint32_t)(f >> 1) * tile_bytes + 1024u * (f & 1) + 16u * lane : OOB8;
  }
#pragma unroll
  for (int k = 0; k < LE; ++k) {
    const int e = WAVES * k + wave, m = 64 * e + lane;
    if (e < BM / 64) eoff[k] = m < mrows ? (uint32_t)m * ke : OOB8;
    else eoff[k] = e == BM / 64 && lane < nblk ? (uint32_t)lane * ke : OOB8;
  }
  // loads from .. to - 1 of stage st (the rows', then the weights')
  auto gload = [&](int st, int from, int to) {
    const bool ok = st < s_hi;
    const __amdgpu_buffer_rsrc_t ar = rsrc8(Ap, ok ? (uint32_t)mrows * K8 : 0u);
    const __amdgpu_buffer_rsrc_t wr = rsrc8(Wp, ok ? (uint32_t)ntile * tile_bytes : 0u);
    uint8_t* base = lds + (st % NB) * C::STAGE;
#pragma unroll
    for (int q = 0; q < L; ++q) {
      if (q < from || q >= to) continue;
      if (q < LA) {
        const uint32_t off = aoff[q];
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            ar, (__attribute__((address_space(3))) void*)(base + (WAVES * q + wave) * 1024), 16, off, 128 * st, 0, 0);
      } else {
        const int k = q - LA;
        const uint32_t off = woff[k];
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            wr, (__attribute__((address_space(3))) void*)(base + (FA + WAVES * k + wave) * 1024), 16, off, 2048 * st, 0, 0);
      }
    }
  };
  // the scales of the four stages from 4 sg on (a line per row: four stages share it)
  auto load_scales = [&](int sg) {
    uint8_t* base = lds + NB * C::STAGE + (sg & 1) * C::SCALES;
#pragma unroll
    for (int k = 0; k < LE; ++k) {
      const int e = WAVES * k + wave;
      const bool rows = e < BM / 64;
      const uint32_t off = eoff[k];
      const __amdgpu_buffer_rsrc_t er = rsrc8(rows ? Ep : Fp, 4 * sg < s_hi ? (uint32_t)(rows ? mrows : nblk) * ke : 0u);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(er, (__attribute__((address_space(3))) void*)(base + e * 256), 4, off, 4 * sg,
                                               0, 0);
    }
  };
  // this lane's 16 bytes g of row r16 in a tile of 16 rows; the other half's lie 4 units away
  const int aswz = r16 * 128 + ((g ^ r16) & 7) * 16;

  f32x4 acc[MF][NF];
#pragma unroll
  for (int i = 0; i < MF; ++i)
#pragma unroll
    for (int j = 0; j < NF; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

#pragma unroll
  for (int st = 0; st < NB - 1; ++st) {
    if (st == 0) load_scales(s_lo / 4);
    gload(s_lo + st, 0, L);
  }
  if constexpr (NB == 2) gload(s_lo + 1, LA, L);
  f32x4 last[C::EXACT ? NF : 1] = {};                  // sums not added yet, and their scale
  float flast = 0.f;
  for (int st = s_lo; st < s_hi; ++st) {
    wait_loads<NB == 2 ? LW : (NB - 2) * L>();
    asm volatile("s_barrier" ::: "memory");
    if ((st & 3) == 0) load_scales(st / 4 + 1);
    const uint8_t* base = lds + (st % NB) * C::STAGE;
    const uint32_t* ex = (const uint32_t*)(lds + NB * C::STAGE + (st / 4 & 1) * C::SCALES);
    const int sh = 8 * (st & 3);
    const int we = (int)(ex[BM + wn * NF * 16 / 128] >> sh);
    u32x4 wf[NF][2], af[2][2];
    int ae[2];
    auto read_a = [&](int i) {
      ae[i & 1] = (int)(ex[(wm * MF + i) * 16 + r16] >> sh);
      af[i & 1][0] = *(const u32x4*)(base + (wm * MF + i) * 2048 + aswz);
      af[i & 1][1] = *(const u32x4*)(base + (wm * MF + i) * 2048 + (aswz ^ 64));
    };
#pragma unroll
    for (int j = 0; j < NF; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        wf[j][h] = *(const u32x4*)(base + (FA / 2 + wn * NF + j) * 2048 + 1024 * h + lane * 16);
    read_a(0);
    __builtin_amdgcn_sched_barrier(0);
    // the loads of stage st + NB - 1 go out between the rows' products: issued
    // together they would hold up every wave behind the address unit
    if constexpr (!C::EXACT) {
#pragma unroll
      for (int i = 0; i < MF; ++i) {
        if (i + 1 < MF) read_a(i + 1);
        if constexpr (NB > 2) {
          gload(st + NB - 1, L * i / MF, L * (i + 1) / MF);
        } else if (i < MF / 2) {                        // two buffers
          gload(st + 1, LA * i / (MF / 2), LA * (i + 1) / (MF / 2));
        } else {
          if (i == MF / 2) asm volatile("s_barrier" ::: "memory");
          gload(st + 2, LA + LW * (i - MF / 2) / (MF - MF / 2), LA + LW * (i - MF / 2 + 1) / (MF - MF / 2));
        }
        __builtin_amdgcn_sched_barrier(0);
        const i32x8 a = __builtin_bit_cast(i32x8, Pair16{af[i & 1][0], af[i & 1][1]});
#pragma unroll
        for (int j = 0; j < NF; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
              __builtin_bit_cast(i32x8, Pair16{wf[j][0], wf[j][1]}), a, acc[i][j], 0, 0, 0, we, 0, ae[i & 1]);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      // while a row tile's products run, the next is widened and the sums of the
      // one before (the last stage's last, first) are scaled and added (2048 x
      // 4096 x 4096: 71.5 -> 67.6 us against doing the three in turn)
      Frag16 w16[NF], a[2];
      float f[2];
      a[0] = widen(af[0]);
      f[0] = scale_of(ae[0] & 255, we & 255);
      if (MF > 1) read_a(1);
#pragma unroll
      for (int i = 0; i < MF; ++i) {
        if (i + 2 < MF) read_a(i + 2);
        gload(st + NB - 1, L * i / MF, L * (i + 1) / MF);
        __builtin_amdgcn_sched_barrier(0);
        f32x4 sum[NF];
#pragma unroll
        for (int j = 0; j < NF; ++j) {
          if (i == 0) w16[j] = widen(wf[j]);
          sum[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int u = 0; u < 4; ++u) sum[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w16[j].v[u], a[i & 1].v[u], sum[j], 0, 0, 0);
        }
        if (i + 1 < MF) {
          a[(i + 1) & 1] = widen(af[(i + 1) & 1]);
          f[(i + 1) & 1] = scale_of(ae[(i + 1) & 1] & 255, we & 255);
        }
#pragma unroll
        for (int j = 0; j < NF; ++j) {
          add_scaled(acc[(i + MF - 1) % MF][j], last[j], flast);
          last[j] = sum[j];
        }
        flast = f[i & 1];
        if (i > 0) {
#pragma unroll
          for (int k = 0; k < 4 * NF; ++k) {
            __builtin_amdgcn_sched_group_barrier(8, 1, 0);                       // a product, then
            __builtin_amdgcn_sched_group_barrier(2, (20 + 4 * NF) / (4 * NF), 0);  // vector instructions
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  if constexpr (C::EXACT) {
#pragma unroll
    for (int j = 0; j < NF; ++j) add_scaled(acc[MF - 1][j], last[j], flast);
  }
  wait_loads<0>();                                    // the trailing empty loads

  // element v of acc[i][j] is row m0 + 16 i, column n0 + 16 j + v of this lane
  const int m0 = wm * MF * 16 + r16, n0 = bx * BN + wn * NF * 16 + 4 * g;
  if constexpr (EPI == EPI8_SWIGLU_Q) {
    // the tile's 256 gate and up columns are one block of 128 outputs: its
    // maximum per row is taken over the WN waves through LDS
    static_assert(BN == 256 && NF % 2 == 0, "one block of outputs per workgroup");
    asm volatile("s_barrier" ::: "memory");           // the stage buffers have been read
    float* red = (float*)lds;                         // [WN][BM]
#pragma unroll
    for (int i = 0; i < MF; ++i) {
      float m = 0.f;
#pragma unroll
      for (int j = 0; j < NF; j += 2)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          acc[i][j][v] = silu8(acc[i][j][v]) * acc[i][j + 1][v];
          m = fmaxf(m, finite_abs(acc[i][j][v]));
        }
      m = fmaxf(m, __shfl_xor(m, 16));
      m = fmaxf(m, __shfl_xor(m, 32));
      if (g == 0) red[wn * BM + m0 + 16 * i] = m;
    }
    __syncthreads();
    const int fb = blocks8(p.N / 2), fe = ke8(p.N / 2);
#pragma unroll
    for (int i = 0; i < MF; ++i) {
      float m = red[m0 + 16 * i];
#pragma unroll
      for (int w = 1; w < C::WN; ++w) m = fmaxf(m, red[w * BM + m0 + 16 * i]);
      if (m0 + 16 * i >= mrows) continue;
      const size_t row = (size_t)bz * BM + m0 + 16 * i;
      const int E = block_exp(m);
      const float inv = inv_scale(E);
#pragma unroll
      for (int j = 0; j < NF; j += 2)                  // (padding is zero in rows of NaN too)
        *(uint32_t*)(p.q_out + row * 128 * fb + 128 * bx + (wn * NF + j) * 8 + 4 * g) =
            wn * NF + j < ntile ? codes4(acc[i][j].x, acc[i][j].y, acc[i][j].z, acc[i][j].w, inv) : 0u;
      if (wn == 0 && g == 0) p.exps_out[row * fe + bx] = (uint8_t)E;
      if (bx == fb - 1 && wn == 1 && g < fe - fb) p.exps_out[row * fe + fb + g] = 0;   // padding (at most 3)
    }
  } else if constexpr (EPI == EPI8_PART) {
    float* part = (float*)p.out + (size_t)split * p.M * p.ldo;
#pragma unroll
    for (int i = 0; i < MF; ++i) {
      if (m0 + 16 * i >= mrows) continue;
      float* row = part + ((size_t)bz * BM + m0 + 16 * i) * p.ldo;
#pragma unroll
      for (int j = 0; j < NF; ++j) {                   // ldo is N rounded up to 4
        if (n0 + 16 * j < p.N) *(f32x4*)(row + n0 + 16 * j) = acc[i][j];
      }
    }
  } else {
    static_assert(EPI == EPI8_STORE, "");
#pragma unroll
    for (int i = 0; i < MF; ++i) {
      if (m0 + 16 * i >= mrows) continue;
      const size_t row = (size_t)bz * BM + m0 + 16 * i;
#pragma unroll
      for (int j = 0; j < NF; ++j) store_out(p, row, n0 + 16 * j, acc[i][j]);
    }
  }
}

// out = [add +] the sum of the K ranges' products, in their order
__global__ __launch_bounds__(256) void gemm8_reduce_kernel(Gemm8Params p, const float* part, int ldp) {
  const int units = ldp / 4;
  const size_t u = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (u >= (size_t)p.M * units) return;
  const size_t m = u / units;
  const int n = (int)(u % units) * 4;
  const float* src = part + m * ldp + n;
  f32x4 s = *(const f32x4*)src;
  for (int k = 1; k < p.ksplit; ++k) s += *(const f32x4*)(src + (size_t)k * p.M * ldp);
  store_out(p, m, n, s);
}

template <typename C, int EPI> static hipError_t gemm8_rows_t(const Gemm8Params& p, hipStream_t s) {
  const size_t gx = ((p.N + 15) / 16 + C::BN / 16 - 1) / (C::BN / 16), gz = ((size_t)p.M + C::BM - 1) / C::BM;
  if (gx * gz * p.ksplit > 0x7fffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL((gemm8_rows_kernel<C, EPI>), dim3((uint32_t)(gx * gz * p.ksplit)), dim3(64 * C::WAVES), 0, s, p);
  return hipGetLastError();
}

static bool ranges8_ok(int kb, int ksplit) { return range8(kb, ksplit) * (ksplit - 1) < kb; }

// grid: workgroups of a K range, if the tiles are enough for them and fit them
template <int MT, int NT, int D, int EPI> static hipError_t gemm8_t(const Gemm8Params& p, int grid, hipStream_t s) {
  constexpr int TPU = EPI == EPI8_SWIGLU ? 2 : 1;
  const int units = (p.N + 15) / 16 / TPU;
  const int gx = std::min(units, std::max(grid, (units + NT / TPU - 1) / (NT / TPU)));
  hipLaunchKernelGGL((gemm8_kernel<MT, NT, 4, D, EPI>), dim3((uint32_t)gx * p.ksplit), dim3(256), 0, s, p);
  return hipGetLastError();
}

// Tiles of a workgroup, and K ranges, of a product of up to 64 rows.  What
// differs is how often the rows are read from L2 (once per workgroup, which from
// 30 rows on takes as long as the weights) against how many workgroups there are:
//   * up to 256 tiles one a workgroup, until the rows' share grows (steps: K / 512
//     times row tiles): from 20 steps on up to 64 tiles, whose grid leaves most
//     CUs idle, K in four ranges; from 40 on two tiles a workgroup and K in two
//     ranges, up to 128 tiles four (4096 x 11008: 16 rows 11.6 us with one tile
//     and 12.8 so, 40 rows 17.1 and 16.0; 512 x 11008, 64 rows: 18.1 -> 10.5);
//   * beyond, two tiles a workgroup, four from 1000 tiles and 17 rows on (16384
//     x 8192, 64 rows: 34.9 -> 31.7).
// Over 448 measured calls (1 to 64 rows) on average 2 % slower than the fastest
// of fifteen choices; one tile up to 256, two beyond: 6 %.
static Gemm8Plan plan_stream8(int M, int N, int K, int most) {
  const int tiles = (N + 15) / 16, kb = blocks8(K), steps4 = kb * ((M + 15) / 16);   // four times the steps
  Gemm8Plan r{false, tiles <= 256 ? 1 : tiles >= 1000 && M > 16 ? 4 : 2, 1};
  if (tiles <= 64 && steps4 >= 4 * 20) {
    r.ksplit = 4;
  } else if (tiles <= 256 && steps4 >= 4 * 40) {
    r.tile = 2;
    r.ksplit = tiles <= 128 ? 4 : 2;
  }
  r.ksplit = std::min(r.ksplit, most);
  while (r.ksplit > 1 && !ranges8_ok(kb, r.ksplit)) r.ksplit /= 2;
  return r;
}

template <int MT, int EPI> static hipError_t gemm8_n(int nt, const Gemm8Params& p, hipStream_t s) {
  if constexpr (EPI == EPI8_SWIGLU) {
    switch (nt) {
      case 2: return gemm8_t<MT, 2, 2, EPI>(p, 256, s);
      case 4: return gemm8_t<MT, 4, 2, EPI>(p, 256, s);
      case 6: return gemm8_t<MT, 6, 2, EPI>(p, 256, s);
      case 8: return gemm8_t<MT, 8, 2, EPI>(p, 256, s);
      default: return hipErrorInvalidValue;
    }
  } else {
    if (nt == 1) return gemm8_t<MT, 1, 3, EPI>(p, 0, s);
    if constexpr (EPI == EPI8_STORE || MT > 1) {         // (two tiles in K ranges: 17 rows and more, at K up to 16384)
      if (nt == 2) return gemm8_t<MT, 2, 2, EPI>(p, 0, s);
    }
    if constexpr (EPI == EPI8_STORE && MT > 1) {
      if (nt == 4) return gemm8_t<MT, 4, 2, EPI>(p, 0, s);
    }
    return hipErrorInvalidValue;
  }
}
template <int EPI> static hipError_t gemm8_m(int nt, const Gemm8Params& p, hipStream_t s) {
  switch ((p.M + 15) / 16) {
    case 1: return gemm8_n<1, EPI>(nt, p, s);
    case 2: return gemm8_n<2, EPI>(nt, p, s);
    case 3: return gemm8_n<3, EPI>(nt, p, s);
    case 4: return gemm8_n<4, EPI>(nt, p, s);
    default: return hipErrorInvalidValue;
  }
}

// The row tiles and the model that picks one of a list, and a number of K
// ranges: a round of workgroups takes e for its start and epilogue, and a + c w for
// every stage, w the workgroups per CU (up to per_cu; less than one in a last
// round that does not fill the card).  K ranges add the pass that sums them.  The
// coefficients are about microseconds, but set for the right choice, not the right
// time: with fp16 operands a measured time is up to 1.9 times the model's (2048 x
// 4096 x 2816), and one of them changed alone ranks its tile wrongly.  Fitted to
// 65 to 8192 rows, N of 512 to 11008 and K of 1024 to 11008 (weights from HBM);
// against the fastest of all tiles and of 1, 2 and 4 K ranges the choice is on
// average 0.4 % slower for the 8-bit instruction (360 shapes with bf16 outputs, the
// worst 31 %), 0.8 % for fp16 operands (304 with fp32 ones, the worst 14 %) and
// 0.03 % for gate/up on the 8-bit instruction (405, the worst 5 %).  One K range
// for all would cost 5 % and 17 %.
struct Tile8Model {
  int mf, nf, wm, wn, nb;   // Tile8
  bool exact;
  int per_cu;
  float e, a, c;
  constexpr int bm() const { return 16 * mf * wm; }
  constexpr int bn() const { return 16 * nf * wn; }
};
static constexpr Tile8Model TILES8[] = {
    // on the 8-bit matrix instruction, for callers that chose it (2048 x 4096 x
    // 11008, bf16 out: 82 us)
    {4, 4, 2, 4, 3, false, 1, 6.8f, 0.756f, 0.207f},    // 128 x 256
    {4, 2, 2, 4, 3, false, 1, 5.3f, 0.399f, 0.156f},    // 128 x 128
    {2, 2, 4, 2, 4, false, 1, 3.4f, 0.346f, 0.050f},    // 128 x 64
    {2, 2, 2, 2, 4, false, 2, 3.1f, 0.227f, 0.138f},    // 64 x 64
    {8, 4, 2, 4, 2, false, 1, 10.3f, 1.111f, 0.446f},   // 256 x 256
    // on fp16 operands (2048 x 4096 x 11008, bf16 out: 155 us)
    {4, 4, 2, 4, 3, true, 1, 4.5f, 0.968f, 0.223f},     // 128 x 256
    {2, 2, 2, 4, 3, true, 2, 4.3f, 0.554f, 0.174f},     // 64 x 128
    {2, 2, 2, 2, 4, true, 2, 3.8f, 0.513f, 0.145f},     // 64 x 64
    // gate/up: 256 columns, the block of 128 outputs.  On the 8-bit matrix
    // instruction, for callers that chose it: its outputs are rounded to four
    // significant bits, and what it is off by moves under one code in a
    // thousand across a border (2^-3 of its value; 1.8e-3 of all outputs' norm at
    // 2048 x 22016 x 4096, of which the rounding to codes takes 2.5e-2)
    {8, 4, 2, 4, 2, false, 1, 11.6f, 1.264f, 0.378f},   // 256 x 256
    {6, 4, 2, 4, 2, false, 1, 7.2f, 1.072f, 0.356f},   // 192 x 256
    {4, 4, 2, 4, 3, false, 1, 8.8f, 0.731f, 0.161f},    // 128 x 256
    {2, 4, 2, 4, 3, false, 1, 6.1f, 0.550f, 0.054f},    // 64 x 256
    // gate/up on fp16 operands (2048 x 22016 x 4096 359 us against 178; 446 measured
    // calls of 65 to 4096 rows: the choice is on average 0.06 % slower than the
    // faster of the two, the worst 4 %)
    {4, 4, 2, 4, 3, true, 1, 9.2f, 1.530f, 0.242f},     // 128 x 256
    {2, 4, 2, 4, 3, true, 1, 6.4f, 1.061f, 0.015f},     // 64 x 256
};
constexpr int TILES8_FAST = 0, TILES8_EXACT = 5, TILES8_GATE_UP = 8, TILES8_GATE_UP_EXACT = 12, TILES8_END = 14;
template <int T>
using Tile8At = Tile8<TILES8[T].mf, TILES8[T].nf, TILES8[T].wm, TILES8[T].wn, TILES8[T].nb, TILES8[T].exact>;

static Gemm8Plan pick_tile8(int lo, int hi, int M, int N, int K, int max_ksplit) {
  const int kb = blocks8(K);
  Gemm8Plan best{true, lo, 1};
  double best_t = 1e30;
  for (int t = lo; t < hi; ++t) {
    const Tile8Model& m = TILES8[t];
    for (int ks = 1; ks <= max_ksplit; ks *= 2) {
      if (!ranges8_ok(kb, ks)) continue;
      const double grid = std::ceil((double)M / m.bm()) * std::ceil((double)N / m.bn()) * ks;
      const int stages = std::min(range8(kb, ks), kb);
      const double slots = 256.0 * m.per_cu, full = std::floor(grid / slots), part = grid - full * slots;
      double us = full * (m.e + stages * (m.a + m.c * m.per_cu));
      if (part > 0) us += m.e + stages * (m.a + m.c * part / 256);
      if (ks > 1) us += 4.0 + 0.29e-6 * ks * M * N * 4;
      if (us < best_t) {
        best_t = us;
        best = Gemm8Plan{true, t, ks};
      }
    }
  }
  return best;
}

// Up to 64 rows the streaming kernel, above (and past the scales it holds in LDS) row tiles.
// Up to 64 rows sums are exact on both.  (Past K = 16384 the row tiles compute 64 rows
// for one: 4096 columns, 8 rows, K = 16384 14.1 us, 28672 49.3)
constexpr int FEW8 = 64;
static bool streams8(int M, int K) { return M <= FEW8 && ke8(K) <= STREAM8_KE; }
bool gate_up8_fused(int M, int K) { return !streams8(M, K); }
Gemm8Plan plan_gate_up8(int M, int N, int K, bool exact) {
  if (streams8(M, K)) {
    // one workgroup per CU and round, which holds all the tiles it is dealt (of 224
    // measured calls 1 % slower than the fastest; two tiles throughout 3 %, 27 % at
    // 27648 x 5120 and 64 rows)
    return Gemm8Plan{false, std::min(8, (N / 16 + 511) / 512 * 2), 1};
  }
  return exact || M <= FEW8 ? pick_tile8(TILES8_GATE_UP_EXACT, TILES8_END, M, N, K, 1)
                            : pick_tile8(TILES8_GATE_UP, TILES8_GATE_UP_EXACT, M, N, K, 1);
}
Gemm8Plan plan_gemm8(int M, int N, int K, bool exact, size_t part_cap) {
  const size_t one = (size_t)M * part8_ld(N);
  const int most = part_cap >= 4 * one ? 4 : part_cap >= 2 * one ? 2 : 1;
  if (streams8(M, K)) return plan_stream8(M, N, K, most);
  return exact || M <= FEW8 ? pick_tile8(TILES8_EXACT, TILES8_GATE_UP, M, N, K, most)
                            : pick_tile8(TILES8_FAST, TILES8_EXACT, M, N, K, most);
}

Gemm8Tile tile_of(const Gemm8Plan& plan, int M) {
  if (!plan.rows) return Gemm8Tile{true, (M + 15) / 16 * 16, 16 * plan.tile};
  const Tile8Model& t = TILES8[plan.tile];
  return Gemm8Tile{t.exact, t.bm(), t.bn()};
}

template <int EPI, int LO, int HI> static hipError_t gemm8_rows_at(int tile, const Gemm8Params& p, hipStream_t s) {
  hipError_t r = hipErrorInvalidValue;
  auto at = [&]<int T>() {
    if (tile == LO + T) r = gemm8_rows_t<Tile8At<LO + T>, EPI>(p, s);
    return tile == LO + T;
  };
  [&]<int... T>(std::integer_sequence<int, T...>) {
    (at.template operator()<T>() || ...);
  }(std::make_integer_sequence<int, HI - LO>());
  return r;
}

hipError_t launch_gemm8(int epi, const Gemm8Plan& plan, const Gemm8Params& p0, hipStream_t s) {
  Gemm8Params p = p0;
  if (p.M <= 0) return hipSuccess;
  if (p.N < 1 || p.K < 1 || p.K > LINEAR8_MAX_K || p.M > LINEAR8_MAX_MN || p.N > LINEAR8_MAX_MN)
    return hipErrorInvalidValue;
  p.wide = p.ldo % 4 == 0 && (uintptr_t)p.out % (p.bf16 ? 8 : 16) == 0 && (uintptr_t)p.add % 16 == 0;
  p.ksplit = 1;
  if (epi == EPI8_SWIGLU_Q) {
    if (p.N % 32 || !plan.rows) return hipErrorInvalidValue;
    return gemm8_rows_at<EPI8_SWIGLU_Q, TILES8_GATE_UP, TILES8_END>(plan.tile, p, s);
  }
  if (epi == EPI8_SWIGLU) {
    if (p.N % 32 || plan.rows || !streams8(p.M, p.K)) return hipErrorInvalidValue;
    return gemm8_m<EPI8_SWIGLU>(plan.tile, p, s);
  }
  if (epi != EPI8_STORE && epi != EPI8_PART) return hipErrorInvalidValue;
  if (!plan.rows && !streams8(p.M, p.K)) return hipErrorInvalidValue;
  if (plan.ksplit == 1) {
    if (epi == EPI8_PART) return hipErrorInvalidValue;
    return plan.rows ? gemm8_rows_at<EPI8_STORE, 0, TILES8_GATE_UP>(plan.tile, p, s) : gemm8_m<EPI8_STORE>(plan.tile, p, s);
  }
  if (!p.part || plan.ksplit < 1 || !ranges8_ok(blocks8(p.K), plan.ksplit)) return hipErrorInvalidValue;
  p.ksplit = plan.ksplit;
  Gemm8Params q = p;
  q.out = p.part;
  q.ldo = part8_ld(p.N);
  const hipError_t r = plan.rows ? gemm8_rows_at<EPI8_PART, 0, TILES8_GATE_UP>(plan.tile, q, s)
                                 : gemm8_m<EPI8_PART>(plan.tile, q, s);
  if (r != hipSuccess || epi == EPI8_PART) return r;
  const size_t blocks = ((size_t)p.M * (q.ldo / 4) + 255) / 256;
  if (blocks > 0x7fffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL(gemm8_reduce_kernel, dim3((uint32_t)blocks), dim3(256), 0, s, p, (const float*)p.part, q.ldo);
  return hipGetLastError();
}

hipError_t launch_gate_up8(const Gemm8Params& p, float* h, bool exact, hipStream_t s) {
  const Gemm8Plan plan = plan_gate_up8(p.M, p.N, p.K, exact);
  if (plan.rows) return launch_gemm8(EPI8_SWIGLU_Q, plan, p, s);
  Gemm8Params q = p;
  q.out = h;
  const hipError_t r = launch_gemm8(EPI8_SWIGLU, plan, q, s);
  return r != hipSuccess ? r : launch_quantise_rows8(h, p.q_out, p.exps_out, p.M, p.N / 2, s);
}

}  // namespace sd
