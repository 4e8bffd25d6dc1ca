// 8-bit rows and their products for gfx950.
//
// k_quantize_rows: x [R, K] in bf16 or fp32 -> e4m3 with a power of two 2^e for each 128 columns of a row:
// e is the least exponent with which 448, e4m3's largest number, reaches the largest finite magnitude of
// the block, so that x 2^-e is exact and the one rounding is that to e4m3 (nearest, ties to even; half a
// step is 2^-4 of the value).
//
// Products: v_mfma_scale_f32_16x16x128_f8f6f4 takes the 128 columns of a block with both scales and adds in
// fp32.  It adds a block's products with the bits below 2^-13 of the largest one left out (1.6e-5 of the
// result in the mean where all are of a size, 5e-5 where they are not: an eightieth of bf16's half step), so results
// that leave in fp32 to the caller are made by the bf16 instruction, which keeps 32 bits (4e-8), at half
// its rate.  The weights are its first operand, so that a lane holds one row of the result and four columns.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "rows8.hpp"
#include "tiles.hpp"

namespace cora {

namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));
// 16 bytes at any alignment of two
struct __attribute__((packed, aligned(2))) bf16x8_any { uint16_t v[8]; };
struct __attribute__((packed, aligned(4))) f32x4_any { float v[4]; };
// Stores at any alignment of the elements, one instruction each (3579 x 24990 x 2241 180 us, element by element 302).
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_out __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ void unpack16(const uint16_t* p, float (&x)[16]) {  // aligned to 16 bytes
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const u32x4_t v = *reinterpret_cast<const u32x4_t*>(p + 8 * t);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[8 * t + 2 * i] = __uint_as_float(v[i] << 16);
      x[8 * t + 2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
  }
}

// columns c0 .. c0 + 15 of a row, zeros from column K on
template <R8Source FROM>
__device__ __forceinline__ void load_chunk(const QuantizeArgs& a, int64_t row, int c0, float (&x)[16]) {
  if constexpr (FROM == R8_F32) {
    const float* p = static_cast<const float*>(a.x) + row * a.ld + c0;
    if (c0 + 16 <= a.cols) {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const f32x4_any v = *reinterpret_cast<const f32x4_any*>(p + 4 * t);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[4 * t + i] = v.v[i];
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = c0 + i < a.cols ? p[i] : 0.f;
  } else if constexpr (FROM == R8_BF16) {
    const uint16_t* p = static_cast<const uint16_t*>(a.x) + row * a.ld + c0;
    if (c0 + 16 <= a.cols) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const bf16x8_any v = *reinterpret_cast<const bf16x8_any*>(p + 8 * t);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[8 * t + i] = bf16_bits_to_f32(v.v[i]);
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = c0 + i < a.cols ? bf16_bits_to_f32(p[i]) : 0.f;
  } else {
    const uint16_t* p = static_cast<const uint16_t*>(a.x);
    if (c0 >= a.cols) {  // cols % 16 == 0
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = 0.f;
    } else if constexpr (FROM == R8_BLOCKS) {
      unpack16(p + ((row >> 6) * (a.cols >> 5) + (c0 >> 5)) * 2048 + (row & 63) * 32 + (c0 & 31), x);
    } else if constexpr (FROM == R8_PANELS) {
      unpack16(p + ((int64_t)(c0 >> 5) * a.rows + row) * 32 + (c0 & 31), x);
    } else {
      float up[16];
      unpack16(p + row * a.ld + 2 * c0, x);
      unpack16(p + row * a.ld + 2 * c0 + 16, up);
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = x[i] / (1.0f + __expf(-x[i])) * up[i];
    }
  }
}

// 16 values to e4m3: what is not finite becomes NaN
__device__ __forceinline__ u32x4_t pack_e4m3(const float (&x)[16], float by) {
  u32x4_t q;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    q[t] = r8_pack(x[4 * t] * by, x[4 * t + 1] * by, x[4 * t + 2] * by, x[4 * t + 3] * by);
  }
  return q;
}

}  // namespace

// A thread has 16 columns of one row, eight neighbouring threads a block's row, two wavefronts a block: a block's scale takes
// three lane exchanges, its values leave as 16 bytes a thread in the products' order.  Bound by memory: 4096 x 18944
// bf16 in 36.6 us (6.3 TB/s), 2048 x 18944 fp32 in 31.6 (6.1); rows of any alignment within a tenth of that.
template <R8Source FROM>
__global__ __launch_bounds__(512) void k_quantize_rows(QuantizeArgs a) {
  const int tid = threadIdx.x, c = tid & 7, r = (tid >> 3) & 15;
  const int nk = r8_blocks(a.cols), nq = r8_quads(a.cols), quad = blockIdx.x % nq, kb = quad * 4 + (tid >> 7);
  const int64_t group = blockIdx.x / nq, row = group * 16 + r;
  float x[16];
  uint32_t most = 0;
  if (row < a.rows && kb < nk) {
    load_chunk<FROM>(a, row, kb * 128 + c * 16, x);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 0.f;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint32_t b = __float_as_uint(x[i]) & 0x7fffffffu;
    if (b >= 0x7f800000u) x[i] = __uint_as_float(0x7fc00000u);
    else most = max(most, b);
  }
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o, 64));
  const int e = r8_scale_byte(most);  // 127 + exponent
  if (kb < nk) {
    const u32x4_t q = pack_e4m3(x, r8_inverse(e));
    *reinterpret_cast<u32x4_t*>(a.data + (group * nk + kb) * R8_BLOCK + c * 256 + r * 16) = q;
  }
  if (c == 0) a.scale[(group * nq + quad) * 64 + r * 4 + (tid >> 7)] = (uint8_t)e;
}

hipError_t launch_quantize_rows(const QuantizeArgs& a, R8Source from, hipStream_t s) {
  const dim3 grid((unsigned)(r8_groups(a.rows) * r8_quads(a.cols)));  // below 2^23: 2^32 threads
  switch (from) {
    case R8_BF16: hipLaunchKernelGGL(k_quantize_rows<R8_BF16>, grid, dim3(512), 0, s, a); break;
    case R8_F32: hipLaunchKernelGGL(k_quantize_rows<R8_F32>, grid, dim3(512), 0, s, a); break;
    case R8_BLOCKS: hipLaunchKernelGGL(k_quantize_rows<R8_BLOCKS>, grid, dim3(512), 0, s, a); break;
    case R8_PANELS: hipLaunchKernelGGL(k_quantize_rows<R8_PANELS>, grid, dim3(512), 0, s, a); break;
    case R8_SWIGLU: hipLaunchKernelGGL(k_quantize_rows<R8_SWIGLU>, grid, dim3(512), 0, s, a); break;
  }
  return hipGetLastError();
}

// ---- products ---------------------------------------------------------------------------------------
namespace {

template <int POLICY>
__device__ __forceinline__ u32x4_t load16(__amdgpu_buffer_rsrc_t rs, int off, int soff) {
  return __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rs, off, soff, POLICY));
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const void* p, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, (int)(bytes > 0x7fffffffLL ? 0x7fffffff : bytes), 0x00020000);
}
__device__ __forceinline__ i32x8_t both(u32x4_t lo, u32x4_t hi) {
  return i32x8_t{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}
// acc += w . a of one block; byte U of the scales' dwords
template <int U>
__device__ __forceinline__ f32x4_t mfma(i32x8_t w, i32x8_t a, f32x4_t acc, uint32_t ws, uint32_t as) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, a, acc, 0, 0, U, (int)ws, U, (int)as);
}

// eight e4m3 numbers times a power of two as bf16, which holds them exactly
__device__ __forceinline__ bf16x8_t widened(uint32_t lo, uint32_t hi, float by) {
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, by, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, by, true);
  const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, by, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, by, true);
  return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// The same by the bf16 instruction, whose sums keep 32 bits: sum first, then the scales.  ws: the scales
// of the lane's four weight rows.
struct Wide { bf16x8_t k[4]; };
__device__ __forceinline__ Wide widened(i32x8_t x, float by = 1.0f) {
  return Wide{{widened(x[0], x[1], by), widened(x[2], x[3], by), widened(x[4], x[5], by), widened(x[6], x[7], by)}};
}
__device__ __forceinline__ f32x4_t mfma_wide(const Wide& w, const Wide& a, f32x4_t acc, u32x4_t ws, uint32_t as, int byte) {
  f32x4_t p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int t = 0; t < 4; ++t) p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.k[t], a.k[t], p, 0, 0, 0);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t bw = ws[e] >> 8 * byte & 255, ba = as >> 8 * byte & 255;
    acc[e] += max(bw, ba) == 255 ? __builtin_nanf("") : ldexpf(p[e], (int)(bw + ba) - 254);
  }
  return acc;
}

__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }
// The value is there now: what made it is not moved past a branch to where it is used (no instruction).
template <class T>
__device__ __forceinline__ void pin(T& x) { asm volatile("" : "+v"(x)); }

template <int... U, class F>
__device__ __forceinline__ void each(std::integer_sequence<int, U...>, F&& f) {
  (f(std::integral_constant<int, U>{}), ...);
}

// a scale's byte outside 2^-50 .. 2^50
__device__ __forceinline__ uint32_t is_far(uint32_t byte) { return byte - 77 > 100 ? 1 : 0; }

constexpr int OOB = 0x7fffffff;  // an offset past every buffer: zeros, no traffic
constexpr int STREAM = 2;        // cache policy of weights that are read once a call: nontemporal
enum { OUT_BF16 = 0, OUT_F32 = 1 };

// bias, rounding and store of columns col .. col + 3 of a row
template <int OUT>
__device__ __forceinline__ void store4(const Rows8ProductArgs& g, int64_t row, int col, f32x4_t x) {
  if (g.bias) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (col + e < g.N) x[e] += g.bias[col + e];
  }
  if constexpr (OUT == OUT_F32) {
    float* dst = static_cast<float*>(g.out) + row * g.ld + col;
    if (col + 3 < g.N) {
      *reinterpret_cast<f32x4_out*>(dst) = x;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (col + e < g.N) dst[e] = x[e];
    }
  } else {
    uint16_t* dst = static_cast<uint16_t*>(g.out) + row * g.ld + col;
    if (col + 3 < g.N) {
      *reinterpret_cast<u32x2_any*>(dst) = u32x2_t{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (col + e < g.N) dst[e] = (uint16_t)f32_to_bf16_bits(x[e]);
    }
  }
}

}  // namespace

// Few rows.  A workgroup's eight wavefronts are KW neighbours along the columns for each of 8 / KW sets of NB
// groups of 16 weight rows.  A wavefront keeps its 512 SQ columns of all the activations in registers and goes
// through sets of weight rows, a set's four next blocks in flight while the ones before are multiplied;
// neighbours add their sums through LDS in their order.  Columns beyond 512 SQ KW go to other workgroups
// (blockIdx.y), whose sums a second kernel adds.  Bound by the stream of weights: 32 x 24576 x 4096 in 18.9 us a call
// (5.4 TB/s; 16.3 the kernel at its best), 64 x 24577 x 4096 in 21.2; 16 x 688 x 256 in 4.1.  Loads that pass the end read zeros
// without traffic, so that the loop has no branch.
template <int MB, int NB, int SQ, int OUT, bool WIDE>
__global__ __launch_bounds__(512, 2) void k_rows8_few(Rows8ProductArgs g, Rows8Few f) {
  extern __shared__ __attribute__((aligned(16))) char stages[];
  constexpr int BL = MB * NB, S = 4 * SQ;
  f32x4_t(*part)[BL][64] = reinterpret_cast<f32x4_t(*)[BL][64]>(stages);  // [2 x 8]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kw = wave & (f.kw - 1), nw = wave / f.kw, sets_wg = 8 / f.kw;
  const int nk = r8_blocks(g.K), nq = r8_quads(g.K);
  // this wavefront's quads of blocks [q0, q0 + SQ), up to the end of the workgroup's columns
  const int range0 = (int)((int64_t)nq * blockIdx.y / gridDim.y), range1 = (int)((int64_t)nq * (blockIdx.y + 1) / gridDim.y);
  const int q0 = range0 + kw * SQ, s_end = min(4 * range1, nk) - 4 * q0;  // blocks there are from 4 q0 on
  const int w_groups = (int)((g.N + 15) / 16), a_groups = (g.M + 15) / 16;
  const auto a_rs = rsrc(g.a, (int64_t)a_groups * nk * R8_BLOCK);
  const auto as_rs = rsrc(g.a_scale, (int64_t)a_groups * nq * 64);

  i32x8_t a[MB][S], w[NB][4];
  typedef std::conditional_t<WIDE, u32x4_t, uint32_t> w_scale_t;
  uint32_t as[MB][SQ];
  w_scale_t ws[NB][SQ], next_ws[NB][SQ];
  auto load_w = [&](int64_t set, int u) {  // block u of the wavefront's, of a set, into its place of four
    const int64_t grp = set * NB;
    const int there = (int)max((int64_t)0, min((int64_t)NB, w_groups - grp));
    const auto rs = rsrc(g.w + (there ? grp : 0) * nk * R8_BLOCK, (int64_t)there * nk * R8_BLOCK);
    const int at = u < s_end ? (4 * q0 + u) * R8_BLOCK + lane * 16 : -1;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const int o = at < 0 ? OOB : at + n * nk * R8_BLOCK;
      w[n][u & 3] = both(load16<STREAM>(rs, o, 0), load16<STREAM>(rs, o, 1024));
    }
  };
  auto load_scales = [&](int64_t set, w_scale_t(&x)[NB][SQ]) {
    const int64_t grp = set * NB;
    const int there = (int)max((int64_t)0, min((int64_t)NB, w_groups - grp));
    const auto rs = rsrc(g.w_scale + (there ? grp : 0) * nq * 64, (int64_t)there * nq * 64);
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int q = 0; q < SQ; ++q) {
        const int at = 4 * q < s_end ? (n * nq + q0 + q) * 64 : -1;
        if constexpr (WIDE) x[n][q] = load16<0>(rs, at < 0 ? OOB : at + (lane >> 4) * 16, 0);
        else x[n][q] = __builtin_amdgcn_raw_buffer_load_b32(rs, at < 0 ? OOB : at + (lane & 15) * 4, 0, 0);
      }
  };
  int64_t set = (int64_t)blockIdx.x * sets_wg + nw;
  const int64_t step = (int64_t)gridDim.x * sets_wg;
  const int64_t sets = (w_groups + NB - 1) / NB, rounds = (sets - (int64_t)blockIdx.x * sets_wg + step - 1) / step;
  load_scales(set, ws);
#pragma unroll
  for (int u = 0; u < 4; ++u) load_w(set, u);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int q = 0; q < SQ; ++q)
#pragma unroll
    for (int m = 0; m < MB; ++m) {
      as[m][q] = __builtin_amdgcn_raw_buffer_load_b32(as_rs, 4 * q < s_end ? (m * nq + q0 + q) * 64 + (lane & 15) * 4 : OOB, 0, 0);
#pragma unroll
      for (int u = 4 * q; u < 4 * q + 4; ++u) {
        const int o = u < s_end ? (m * nk + 4 * q0 + u) * R8_BLOCK + lane * 16 : OOB;
        a[m][u] = both(load16<0>(a_rs, o, 0), load16<0>(a_rs, o, 1024));
      }
    }
  for (int64_t r = 0; r < rounds; ++r, set += step) {
    f32x4_t acc[MB][NB] = {};
    load_scales(set + step, next_ws);  // past the last set: zeros, no traffic, and no branch in the loop
    auto block = [&](auto u_c) {
      constexpr int U = decltype(u_c)::value;
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          if constexpr (WIDE) acc[m][n] = mfma_wide(widened(w[n][U & 3]), widened(a[m][U]), acc[m][n], ws[n][U / 4], as[m][U / 4], U & 3);
          else acc[m][n] = mfma<U & 3>(w[n][U & 3], a[m][U], acc[m][n], ws[n][U / 4], as[m][U / 4]);
        }
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (U + 4 < S) load_w(set, U + 4);
      else load_w(set + step, U + 4 - S);
    };
    each(std::make_integer_sequence<int, S>{}, block);
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int q = 0; q < SQ; ++q) ws[n][q] = next_ws[n][q];
    f32x4_t(*mine)[BL][64] = part + (r & 1) * 8;
    if (f.kw > 1) {
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int n = 0; n < NB; ++n) mine[wave][m * NB + n][lane] = acc[m][n];
      __syncthreads();
    }
#pragma unroll
    for (int t = 0; t < BL; ++t) {
      if ((t & (f.kw - 1)) != kw) continue;
      f32x4_t x = acc[t / NB][t % NB];
      if (f.kw > 1) {
        x = mine[wave - kw][t][lane];
        for (int v = 1; v < f.kw; ++v) x += mine[wave - kw + v][t][lane];
      }
      const int row = (t / NB) * 16 + (lane & 15);
      const int64_t col = (set * NB + t % NB) * 16 + 4 * (lane >> 4);
      if (row < g.M && col < g.N) store4<OUT>(g, (int64_t)blockIdx.y * g.M + row, (int)col, x);
    }
  }
}

// Tiles of many rows.  A workgroup of WM x WN wavefronts goes through tiles of BM x BN; a wavefront owns TM x TN
// blocks of 16 x 16.
//
// A ring of ST stages in LDS, a section's 128 columns and the rows' scales each as they lie in memory, is filled by
// loads that write LDS directly, ST sections ahead and across the tiles' borders.  The MFMAs of a section work from
// registers; a fragment is reloaded with the next section's right after its last MFMA, half a section before it is
// needed: the first half of the rows with all columns, then the others, while the columns become free one by one.
// The section's one barrier stands before the first reload: past it the next section's stage is whole and the
// stage of the section at hand, all in registers, takes new loads.  What it waits for is then long done.
//
// A tile's results pass through LDS of the wavefront's own and leave as runs of CB x 32 bytes, 16 a lane, behind the
// next tile's first loads (4096 x 37888 bf16 written alone in runs of 32 bytes 81 us, of 64 58 us, of 256 56 us).
// Bound by the matrix cores: 8192^3 bf16 in 400 us (2.75 PFLOP/s; on zeros 357, so that the power that they draw costs a tenth),
// 4096 x 37888 x 3584 in 475 (2.34: the cores busy for 66 % of the cycles; a tenth round on a quarter of the CUs and 310 MB
// of results account for part of the rest), 2048 x 24576 x 4096 in 148 (2.8).
// WIDE (sums of 32 bits): a section's fragments are widened to bf16 first, times their scales, the activations all, a group
// of weight rows at a time; they are free at once, and the barrier stands between.  Bound by the conversions beside the
// matrix cores: 2048 x 12288 x 4096 in 182 us (1.13 PFLOP/s; 227 with the scales applied to each block's sums).  The results of
// rows with a scale outside 2^-50 .. 2^50, whose products may leave the normal numbers, are made again that way, from memory.
template <int WM, int WN, int TM, int TN, int ST, int CB, int OUT, bool WIDE>
__global__ __launch_bounds__(WM * WN * 64, 2) void k_rows8_tiles(Rows8ProductArgs g, int splits) {
  constexpr int NW = WM * WN, BM = WM * TM * 16, BN = WN * TN * 16, GA = BM / 16, GB = BN / 16;
  constexpr int ROWS = BM + BN, STAGE = ROWS * 132;       // 128 columns and a dword of scales a row
  // loads of 1 KB (half a block) and of 64 rows' scales of a wavefront (where the scales do not divide evenly some
  // load the same to the same place, so that every wavefront counts alike)
  constexpr int LPW = (GA + GB) * 2 / NW, SCALES = ROWS / 64, SPW = (SCALES + NW - 1) / NW, ALL = LPW + SPW;
  static_assert((GA + GB) % NW == 0 && BM % 64 == 0 && BN % 64 == 0 && ST >= 2 && TM % 2 == 0, "every wavefront loads alike");
  extern __shared__ __attribute__((aligned(1024))) char stages[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN, r16 = lane & 15, g4 = lane >> 4;
  const int nk_all = r8_blocks(g.K), nq = r8_quads(g.K);
  const int num_m = (g.M + BM - 1) / BM, tiles = num_m * ((g.N + BN - 1) / BN), items = tiles * splits;
  const int first = xcd_remap(blockIdx.x, gridDim.x);
  if (first >= items) return;  // grids have no more workgroups than items
  auto k_range = [&](int item, int& k0, int& k1) {  // blocks of columns; splits <= blocks, so it is never empty
    const int split = item / tiles;
    k0 = scalar((int)((int64_t)nk_all * split / splits));
    k1 = scalar((int)((int64_t)nk_all * (split + 1) / splits));
  };

  // ---- the stream of loads: the item, and the block of its columns, of the next section to load
  constexpr int GPW = LPW / 2;
  int l_item = first, l_k = 0, l_end = 0;
  u32x4_t rs[GPW], ss[SPW];
  int so[GPW], vs[SPW];
  auto open_item = [&]() {
    int tm, tn;
    tile_of(l_item % tiles, num_m, tiles, tm, tn);
    k_range(l_item, l_k, l_end);
    const int64_t a0 = (int64_t)scalar(tm) * GA, b0 = (int64_t)scalar(tn) * GB;  // divisions leave them in vector registers
    const int a_last = (int)((g.M + 15) / 16 - 1 - a0), b_last = (int)((g.N + 15) / 16 - 1 - b0);
    const u32x4_t a_rs = buffer_rsrc(g.a + a0 * nk_all * R8_BLOCK, (int64_t)(a_last + 1) * nk_all * R8_BLOCK);
    const u32x4_t b_rs = buffer_rsrc(g.w + b0 * nk_all * R8_BLOCK, (int64_t)(b_last + 1) * nk_all * R8_BLOCK);
    const u32x4_t as_rs = buffer_rsrc(g.a_scale + a0 * nq * 64, (int64_t)(a_last + 1) * nq * 64);
    const u32x4_t bs_rs = buffer_rsrc(g.w_scale + b0 * nq * 64, (int64_t)(b_last + 1) * nq * 64);
#pragma unroll
    for (int t = 0; t < GPW; ++t) {
      const int grp = wave * GPW + t;
      const bool is_a = grp < GA;
      rs[t] = is_a ? a_rs : b_rs;
      so[t] = (is_a ? min(grp, a_last) : min(grp - GA, b_last)) * nk_all * R8_BLOCK;  // past the last group: it again
    }
#pragma unroll
    for (int t = 0; t < SPW; ++t) {
      const int row0 = (wave * SPW + t) % SCALES * 64;
      const bool is_a = row0 < BM;
      const int row = (is_a ? row0 : row0 - BM) + lane;
      ss[t] = is_a ? as_rs : bs_rs;
      vs[t] = min(row >> 4, is_a ? a_last : b_last) * nq * 64 + (row & 15) * 4;
    }
  };
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)stages;
  const int lane16 = lane * 16;
  auto issue = [&](uint32_t st, int t) {  // load t of the section into the stage at st
    if (t < LPW) load_lds(lds0 + st + (wave * LPW + t) * 1024, lane16, rs[t < LPW ? t / 2 : 0], so[t < LPW ? t / 2 : 0] + l_k * R8_BLOCK + (t & 1) * 1024);
    else load_lds_dword(lds0 + st + ROWS * 128 + (wave * SPW + t - LPW) % SCALES * 256, vs[t < LPW ? 0 : t - LPW], ss[t < LPW ? 0 : t - LPW], (l_k >> 2) * 64);
  };
  auto advance = [&]() {  // past the last item: its last section again, never read
    if (l_k + 1 < l_end) ++l_k;
    else if (l_item + (int)gridDim.x < items) {
      l_item += gridDim.x;
      open_item();
    }
  };

  // ---- the products
  f32x4_t acc[TM][TN];
  i32x8_t fa[TM], fb[TN];
  uint32_t sb[TN];  // scales: the section's byte; WIDE: the dword
  uint32_t sa[TM];
  const int a_at = wm * TM * R8_BLOCK + lane * 16, b_at = (GA + wn * TN) * R8_BLOCK + lane * 16;
  const int as_at = ROWS * 128 + (wm * TM * 16 + r16) * 4, bs_at = ROWS * 128 + (BM + wn * TN * 16 + r16) * 4;
  auto frag = [&](int at) {
    return both(*reinterpret_cast<const u32x4_t*>(stages + at), *reinterpret_cast<const u32x4_t*>(stages + at + 1024));
  };
  auto read_a = [&](int st, int by, int i) {
    fa[i] = frag(st + a_at + i * R8_BLOCK);
    if constexpr (WIDE) sa[i] = *reinterpret_cast<const uint32_t*>(stages + st + as_at + i * 64);
    else sa[i] = *reinterpret_cast<const uint8_t*>(stages + st + as_at + by + i * 64);
  };
  auto read_b = [&](int st, int by, int j) {
    fb[j] = frag(st + b_at + j * R8_BLOCK);
    if constexpr (WIDE) sb[j] = *reinterpret_cast<const uint32_t*>(stages + st + bs_at + j * 64);
    else sb[j] = *reinterpret_cast<const uint8_t*>(stages + st + bs_at + by + j * 64);
  };
  constexpr int NM = TM * TN, HALF = TM / 2, BAR = NM / 2 >= 2 ? NM / 2 - 2 : 0;
  constexpr int RUNS = 16 * CB * 2 / 64, STORES = OUT == OUT_BF16 ? TM * (TN / CB) * RUNS : 0;
  int st = 0;           // stage of the section at hand
  int this_by = 0;      // WIDE: byte of its scales
  uint32_t far = 0;     // WIDE: a scale of the tile's lies outside 2^-50 .. 2^50
  bool late = false;    // a tile's stores, STORES of them or more, were issued since the loads that a barrier waits for
  // FIRST: of a tile; by: byte of the next section's scales
  auto section = [&](auto first_c, int by) {
    constexpr bool FIRST = decltype(first_c)::value;
    const int nx = st + STAGE == ST * STAGE ? 0 : st + STAGE;
    if constexpr (WIDE) {
      auto scale_of = [&](uint32_t dword) {
        const uint32_t e = dword >> 8 * this_by & 255;
        far |= is_far(e);
        return __uint_as_float(e << 23);
      };
      Wide a[TM];
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        a[i] = widened(fa[i], scale_of(sa[i]));
        if constexpr (FIRST) {
#pragma unroll
          for (int j = 0; j < TN; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
      }
      wait_vm<(ST - 2) * ALL>();
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < TM; ++i) read_a(nx, by, i);
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const Wide w = widened(fb[j], scale_of(sb[j]));
        read_b(nx, by, j);
#pragma unroll
        for (int t = 0; t < ALL; ++t)
          if (t * TN / ALL == j) issue((uint32_t)st, t);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < TM; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.k[t], a[i].k[t], acc[i][j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      this_by = by;
    } else {
#pragma unroll
    for (int q = 0; q < NM; ++q) {
      const int half = q / (HALF * TN), j = q % (HALF * TN) / HALF, i = half * HALF + q % HALF;
      if (q == BAR) {
        if (FIRST && STORES > 0 && ST == 2 && late) wait_vm<STORES>();
        else wait_vm<(ST - 2) * ALL>();
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
      }
      acc[i][j] = mfma<0>(fb[j], fa[i], FIRST ? f32x4_t{0.f, 0.f, 0.f, 0.f} : acc[i][j], sb[j], sa[i]);
      if (j == TN - 1) read_a(nx, by, i);
      if (i == TM - 1) read_b(nx, by, j);
#pragma unroll
      for (int t = 0; t < ALL; ++t)
        if (BAR + t * (NM - BAR) / ALL == q) issue((uint32_t)st, t);
      __builtin_amdgcn_sched_barrier(0);
    }
    }
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) pin(acc[i][j]);
    advance();
    st = nx;
  };
  open_item();
#pragma unroll
  for (int u = 0; u < ST; ++u) {
#pragma unroll
    for (int t = 0; t < ALL; ++t) issue(u * STAGE, t);
    advance();
  }
  wait_vm<(ST - 1) * ALL>();
  __syncthreads();
  int k0, k1;
  k_range(first, k0, k1);
  this_by = k0 & 3;
#pragma unroll
  for (int i = 0; i < TM; ++i) read_a(0, k0 & 3, i);
#pragma unroll
  for (int j = 0; j < TN; ++j) read_b(0, k0 & 3, j);
  for (int item = first; item < items; item += gridDim.x) {
    k_range(item, k0, k1);
    int n0 = 0, n1;
    if (item + (int)gridDim.x < items) k_range(item + gridDim.x, n0, n1);
    section(std::true_type{}, (k0 + 1 < k1 ? k0 + 1 : n0) & 3);
    for (int k = k0 + 1; k < k1; ++k) section(std::false_type{}, (k + 1 < k1 ? k + 1 : n0) & 3);

    // a lane holds row lane % 16 and columns 4 (lane / 16) .. + 3 of each block
    int tm, tn;
    tile_of(item % tiles, num_m, tiles, tm, tn);
    const int64_t row0 = (int64_t)scalar(tm) * BM + wm * TM * 16, slab = (int64_t)scalar(item / tiles) * g.M;
    const int col0 = scalar(tn) * BN + wn * TN * 16;
    late = OUT == OUT_BF16 && row0 + TM * 16 <= g.M && col0 + TN * 16 <= g.N;
    if (late) {
      constexpr int PITCH = CB * 32 + 16;
      char* scr = stages + ST * STAGE + wave * 16 * PITCH;
      uint16_t* dst = static_cast<uint16_t*>(g.out) + (row0 + lane / (CB * 2)) * g.ld + col0 + lane % (CB * 2) * 8;
      if (g.bias) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float b = g.bias[col0 + j * 16 + 4 * g4 + e];
#pragma unroll
            for (int i = 0; i < TM; ++i) acc[i][j][e] += b;
          }
      }
#pragma unroll
      for (int j0 = 0; j0 < TN; j0 += CB) {
#pragma unroll
        for (int i = 0; i < TM; ++i) {
#pragma unroll
          for (int j = 0; j < CB; ++j) {
            const f32x4_t x = acc[i][j0 + j];
            *reinterpret_cast<u32x2_t*>(scr + r16 * PITCH + j * 32 + g4 * 8) = u32x2_t{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
          }
          wave_lds_sync();
#pragma unroll
          for (int u = 0; u < RUNS; ++u) {
            constexpr int RPR = 16 / RUNS;  // rows of a run of 64 lanes
            *reinterpret_cast<u32x4_any*>(dst + (int64_t)(i * 16 + u * RPR) * g.ld + j0 * 16) =
                *reinterpret_cast<const u32x4_t*>(scr + (u * RPR + lane / (CB * 2)) * PITCH + lane % (CB * 2) * 16);
          }
          wave_lds_sync();
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          const int64_t r = row0 + i * 16 + r16;
          const int c = col0 + j * 16 + 4 * g4;
          if (r < g.M && c < g.N) store4<OUT>(g, slab + r, c, acc[i][j]);
        }
    }
    if constexpr (WIDE) {
      // Products of such scales' numbers may leave the normal ones: the tile again, its blocks' sums first, then the scales, over the
      // results of rows that have such a scale.  The others keep theirs, so that no row's bits depend on another's numbers.
      if (__builtin_expect(__ballot(far != 0) != 0, 0)) {
        const int64_t ga = row0 / 16, gb = col0 / 16, a_end = (g.M + 15) / 16 - 1, b_end = (g.N + 15) / 16 - 1;
#pragma unroll 1
        for (int t = 0; t < TM * TN; ++t) {
          const int64_t ra = min(ga + t / TN, a_end), rb = min(gb + t % TN, b_end);  // past the last group: it again, not stored
          f32x4_t x = {0.f, 0.f, 0.f, 0.f};
          uint32_t again = 0;  // bit e: column e's
#pragma unroll 1
          for (int k = k0; k < k1; ++k) {
            const uint8_t *pa = g.a + (ra * nk_all + k) * R8_BLOCK + lane * 16, *pw = g.w + (rb * nk_all + k) * R8_BLOCK + lane * 16;
            const i32x8_t a = both(*reinterpret_cast<const u32x4_t*>(pa), *reinterpret_cast<const u32x4_t*>(pa + 1024));
            const i32x8_t w = both(*reinterpret_cast<const u32x4_t*>(pw), *reinterpret_cast<const u32x4_t*>(pw + 1024));
            const uint8_t *qa = g.a_scale + (ra * nq + (k >> 2)) * 64, *qw = g.w_scale + (rb * nq + (k >> 2)) * 64;
            const uint32_t as = qa[r16 * 4 + (k & 3)];
            u32x4_t ws;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              ws[e] = qw[(4 * g4 + e) * 4 + (k & 3)];
              again |= (is_far(ws[e]) | is_far(as)) << e;
            }
            x = mfma_wide(widened(w), widened(a), x, ws, as, 0);
          }
          const int64_t r = row0 + t / TN * 16 + r16;
          const int c = col0 + t % TN * 16 + 4 * g4;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (again >> e & 1 && r < g.M && c + e < g.N)
              static_cast<float*>(g.out)[(slab + r) * g.ld + c + e] = x[e] + (g.bias ? g.bias[c + e] : 0.f);
        }
      }
      far = 0;
    }
  }
  wait_vm<0>();
}

// ---- sums of several workgroups' columns -----------------------------------------------------------------
// parts [splits][M][ld], added in their order, four columns a thread; bound by memory, 4.6 us for two splits of 32 x 4096
// (most of it the launch)
template <int OUT>
__global__ __launch_bounds__(256) void k_rows8_fold(Rows8ProductArgs g, const float* parts, int splits, int ld) {
  const int64_t per_row = ld / 4, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= per_row * g.M) return;
  const int64_t row = i / per_row;
  const int col = (int)(i - row * per_row) * 4;
  const float* p = parts + row * ld + col;
  f32x4_t x = *reinterpret_cast<const f32x4_t*>(p);
  for (int s = 1; s < splits; ++s) x += *reinterpret_cast<const f32x4_t*>(p + (int64_t)s * g.M * ld);
  store4<OUT>(g, row, col, x);
}

// ---- plans ---------------------------------------------------------------------------------------------
// X(config, wavefronts along M and N, blocks of a wavefront, stages, blocks side by side on their way out,
//   workgroups a CU; a lone tile's us a section, a section's us a CU in use, us a tile)
#define R8_TILES(X)                               \
  X(0, 4, 2, 4, 8, 2, 4, 1, 1.412, 1.198, 4.89)   \
  X(1, 4, 2, 4, 4, 3, 2, 1, 0.709, 0.843, 2.60)   \
  X(2, 2, 4, 4, 4, 3, 2, 1, 0.856, 0.861, 2.65)   \
  X(3, 2, 2, 4, 4, 2, 4, 2, 0.841, 0.563, 1.31)   \
  X(4, 2, 2, 2, 4, 3, 2, 2, 0.389, 0.351, 1.45)   \
  X(5, 2, 2, 2, 2, 4, 2, 2, 0.242, 0.213, 1.05)
constexpr int R8_CONFIGS = 6;
struct R8Shape {
  int bm, bn, per_cu;
  double section_us, cu_us, tile_us;
};
static R8Shape r8_shape(int cfg) {
  switch (cfg) {
#define X(C, WM, WN, TM, TN, ST, CB, PER, SEC, CU, TILE) case C: return {WM * TM * 16, WN * TN * 16, PER, SEC, CU, TILE};
    R8_TILES(X)
#undef X
  }
  return {};
}

// Estimated time of a product by tiles in microseconds: rounds of resident tiles, each the larger of a tile's own
// latency a section and the chip's throughput, plus what a tile takes besides; the stream of weights, a fifth of which
// goes beside it; the sums of split columns.  Fitted to all configs and splits of 209 shapes (80 to 4096 rows, 688 to
// 37888 weight rows, 1000 to 12288 columns; 12 % off in the mean).  What it picks is on average 1 %, at most 15 % slower
// than the fastest of these.  Sections of 32-bit sums count 1.95 times (their measured 1.7 picks
// plans that are 1 % slower).
static double tiles_us(int M, int N, int K, int cfg, int splits, bool wide, int num_cus) {
  R8Shape sh = r8_shape(cfg);
  if (wide) {
    sh.section_us *= 1.95;
    sh.cu_us *= 1.95;
  }
  const double sections = (double)r8_blocks(K) / splits;
  const int64_t items = (int64_t)((M + sh.bm - 1) / sh.bm) * ((N + sh.bn - 1) / sh.bn) * splits, slots = (int64_t)num_cus * sh.per_cu;
  auto round_us = [&](int64_t n) {
    const double per_cu = (double)std::min<int64_t>(sh.per_cu, (n + num_cus - 1) / num_cus), busy = std::min(1.0, (double)n / num_cus);
    return sections * std::max(sh.section_us, per_cu * sh.cu_us * (0.843 + 0.157 * busy)) + sh.tile_us;
  };
  double us = 1.15 + (double)(items / slots) * round_us(slots);
  if (items % slots) us += round_us(items % slots);
  const double stream_us = 1.15 + (double)N * K / 8.67e6;
  us = std::max(us, stream_us) + 0.8 * std::min(us, stream_us);
  if (splits > 1) us += 0.34 * (double)splits * M * N * 4.0 / (1 << 20) + 3.4;
  return us;
}

// What fits a wavefront's 256 registers: groups of 16 activation rows MB, of weight rows NB, quads of blocks SQ.
// X(MB, NB, SQ), for results of 8-bit sums and of 32-bit ones
#define R8_FEW(X) X(1, 1, 1) X(1, 1, 2) X(1, 1, 3) X(1, 2, 1) X(2, 1, 1) X(2, 1, 2) X(2, 2, 1) X(4, 1, 1)
#define R8_FEW_WIDE(X) X(1, 1, 1) X(1, 1, 2) X(1, 2, 1) X(2, 1, 1)

static int few_groups(int M, bool wide) { return M <= 16 ? 1 : (M <= 32 || wide ? 2 : 4); }  // MB
int rows8_few_rows(bool wide) { return wide ? 32 : 64; }

Rows8Plan rows8_plan_few(int M, int N, int K, int nb, int sq, int ranges, bool wide, int num_cus) {
  Rows8Plan p{};
  p.few = true;
  p.mb = few_groups(M, wide);
  p.nb = nb;
  p.sq = sq;
  p.splits = ranges;
  const int nq = r8_quads(K), per = (nq + ranges - 1) / ranges;
  p.kw = 1;
  while (p.kw * sq < per) p.kw *= 2;
  if (p.kw > 8) p.splits = 0;  // no such plan
  const int64_t sets = (r8_groups(N) + nb - 1) / nb, wgs = (sets * p.kw + 7) / 8;
  p.grid = (int)std::min<int64_t>(wgs, std::max(1, num_cus / ranges));
  p.ws_floats = ranges > 1 ? (size_t)ranges * M * ((N + 3) / 4 * 4) : 0;
  return p;
}
Rows8Plan rows8_plan_tiles(int M, int N, int K, int cfg, int splits, int num_cus) {
  Rows8Plan p{};
  p.cfg = cfg;
  p.splits = splits;
  p.ws_floats = splits > 1 ? (size_t)splits * M * ((N + 3) / 4 * 4) : 0;
  const R8Shape sh = r8_shape(cfg);
  const int64_t items = (int64_t)((M + sh.bm - 1) / sh.bm) * ((N + sh.bn - 1) / sh.bn) * splits;
  p.grid = (int)std::min<int64_t>(items, (int64_t)num_cus * sh.per_cu);
  return p;
}

// A second launch's own time, and what two launches have to promise: what the estimate gives them is 4 % more than they keep.
constexpr double R8_REST_US = 1.5, R8_REST_GAIN = 0.92;
// Splits of a product by tiles leave no more than this in the workspace.
constexpr int64_t R8_MOST_PARTS = 1 << 26;

Rows8Plan rows8_plan(int M, int N, int K, bool wide, int num_cus) {
  if (M <= rows8_few_rows(wide)) {
    // as many columns as a wavefront's registers hold, then more workgroups along them; two groups of weight
    // rows where there are enough for all CUs (32 x 24576 x 4096 19.4 us, with one 19.9)
    const int nq = r8_quads(K), mb = few_groups(M, wide), most = mb == 4 || (wide && mb == 2) ? 1 : (wide || mb == 2 ? 2 : 3);
    int sq = 1, ranges = 1;
    while (8 * sq * ranges < nq) {
      if (sq < most) ++sq;
      else ++ranges;
    }
    const int nb = mb < 4 && sq == 1 && !(wide && mb == 2) && r8_groups(N) >= 2 * num_cus ? 2 : 1;
    return rows8_plan_few(M, N, K, nb, sq, ranges, wide, num_cus);
  }
  int best_cfg = 0, best_splits = 1;
  double best_us = -1;
  for (int splits = 1; splits <= 8; splits *= 2) {
    if (splits > 1 && (r8_blocks(K) < 4 * splits || (int64_t)splits * M * ((N + 3) / 4 * 4) > R8_MOST_PARTS)) continue;
    for (int c = 0; c < R8_CONFIGS; ++c) {
      if (wide && c != 3 && c != 5) continue;
      const R8Shape sh = r8_shape(c);
      // the smallest tiles read too much from L2 for more of them than CUs (with them the picks are 2.4 % slower in the mean)
      if (c == 5 && !wide && (int64_t)((M + sh.bm - 1) / sh.bm) * ((N + sh.bn - 1) / sh.bn) * splits > num_cus) continue;
      const double us = tiles_us(M, N, K, c, splits, wide, num_cus);
      if (best_us < 0 || us < best_us) { best_cfg = c; best_splits = splits; best_us = us; }
    }
  }
  // The last round of tiles may leave most CUs idle: whole rounds of one config, then the other weight rows as a product
  // of their own (3804 x 4493 x 11519, 1.05 rounds of 256 x 256 tiles: 162 us, as 256 x 128 tiles alone 240).
  int n_first = N, rest_cfg = 0;
  double rest_us = 0;
  for (int c = 0; c < R8_CONFIGS; ++c) {
    if (wide && c != 3 && c != 5) continue;
    const R8Shape sh = r8_shape(c);
    const int64_t num_m = (M + sh.bm - 1) / sh.bm, slots = (int64_t)num_cus * sh.per_cu, items = num_m * ((N + sh.bn - 1) / sh.bn);
    const int64_t first = items / slots * slots / num_m * sh.bn;
    if (first < 1 || first >= N) continue;
    const double us = tiles_us(M, (int)first, K, c, 1, wide, num_cus);
    if (us + R8_REST_US >= R8_REST_GAIN * best_us) continue;
    for (int d = 0; d < R8_CONFIGS; ++d) {
      if (wide && d != 3 && d != 5) continue;
      const double both = us + R8_REST_US + tiles_us(M, N - (int)first, K, d, 1, wide, num_cus);
      if (both < R8_REST_GAIN * best_us && (n_first == N || both < rest_us)) { best_cfg = c; best_splits = 1; n_first = (int)first; rest_cfg = d; rest_us = both; }
    }
  }
  Rows8Plan p = rows8_plan_tiles(M, n_first, K, best_cfg, best_splits, num_cus);
  if (n_first < N) {
    p.rest = N - n_first;
    p.rest_cfg = rest_cfg;
    p.rest_grid = rows8_plan_tiles(M, p.rest, K, rest_cfg, 1, num_cus).grid;
  }
  return p;
}

static hipError_t fold(const Rows8ProductArgs& a, const float* parts, int splits, int ld, bool f32, hipStream_t s) {
  const unsigned grid = (unsigned)(((int64_t)ld / 4 * a.M + 255) / 256);
  if (f32) hipLaunchKernelGGL(k_rows8_fold<OUT_F32>, dim3(grid), dim3(256), 0, s, a, parts, splits, ld);
  else hipLaunchKernelGGL(k_rows8_fold<OUT_BF16>, dim3(grid), dim3(256), 0, s, a, parts, splits, ld);
  return hipGetLastError();
}

template <int OUT, bool WIDE>
static hipError_t run_few(const Rows8ProductArgs& a, const Rows8Plan& p, hipStream_t s) {
  const unsigned lds = p.kw > 1 ? 16 * p.mb * p.nb * 1024 : 0;
#define X(MB, NB, SQ)                                                                                                  \
  if (p.mb == MB && p.nb == NB && p.sq == SQ) {                                                                        \
    hipLaunchKernelGGL((k_rows8_few<MB, NB, SQ, OUT, WIDE>), dim3(p.grid, p.splits), dim3(512), lds, s, a, Rows8Few{p.kw}); \
    return hipGetLastError();                                                                                          \
  }
  if constexpr (WIDE) {
    R8_FEW_WIDE(X)
  } else {
    R8_FEW(X)
  }
#undef X
  return hipErrorInvalidValue;
}
// those of 32-bit sums, which need more registers
#define R8_TILES_WIDE(X)     \
  X(3, 2, 2, 4, 4, 2, 4, 2)  \
  X(5, 2, 2, 2, 2, 4, 2, 2)

template <int OUT, bool WIDE>
static hipError_t run_tiles(const Rows8ProductArgs& a, const Rows8Plan& p, hipStream_t s) {
#define X(C, WM, WN, TM, TN, ST, CB, PER, ...)                                                                           \
  if (p.cfg == C) {                                                                                                      \
    constexpr unsigned LDS = ST * (WM * TM + WN * TN) * 16 * 132 + WM * WN * 16 * (CB * 32 + 16);                        \
    static_assert(LDS * PER <= 160 * 1024, "LDS of a CU");                                                               \
    hipLaunchKernelGGL((k_rows8_tiles<WM, WN, TM, TN, ST, CB, OUT, WIDE>), dim3(p.grid), dim3(WM * WN * 64), LDS, s, a, p.splits); \
    return hipGetLastError();                                                                                            \
  }
  if constexpr (WIDE) {
    R8_TILES_WIDE(X)
  } else {
    R8_TILES(X)
  }
#undef X
  return hipErrorInvalidValue;
}

static hipError_t run(const Rows8ProductArgs& a, const Rows8Plan& p, bool f32, bool wide, hipStream_t s) {
  if (p.few && a.M > rows8_few_rows(wide)) return hipErrorInvalidValue;
  if (p.few) return wide ? run_few<OUT_F32, true>(a, p, s) : (f32 ? run_few<OUT_F32, false>(a, p, s) : run_few<OUT_BF16, false>(a, p, s));
  return wide ? run_tiles<OUT_F32, true>(a, p, s) : (f32 ? run_tiles<OUT_F32, false>(a, p, s) : run_tiles<OUT_BF16, false>(a, p, s));
}

static Rows8ProductArgs into_parts(const Rows8ProductArgs& in, float* ws) {
  Rows8ProductArgs a = in;
  a.out = ws;
  a.ld = (in.N + 3) / 4 * 4;
  a.bias = nullptr;
  return a;
}

hipError_t launch_rows8_product(const Rows8ProductArgs& a, const Rows8Plan& p, bool f32, bool wide, float* ws, hipStream_t s) {
  if (p.rest) {
    Rows8ProductArgs g = a;
    g.N = a.N - p.rest;
    if (hipError_t e = run(g, p, f32, wide, s)) return e;
    const int nk = r8_blocks(a.K), nq = r8_quads(a.K);
    g.w += (int64_t)(g.N / 16) * nk * R8_BLOCK;  // g.N: whole tiles
    g.w_scale += (int64_t)(g.N / 16) * nq * 64;
    if (g.bias) g.bias += g.N;
    g.out = static_cast<char*>(g.out) + (int64_t)g.N * (f32 ? 4 : 2);
    g.N = p.rest;
    Rows8Plan rest{};
    rest.cfg = p.rest_cfg;
    rest.grid = p.rest_grid;
    rest.splits = 1;
    return run(g, rest, f32, wide, s);
  }
  if (p.splits == 1) return run(a, p, f32, wide, s);
  const Rows8ProductArgs parts = into_parts(a, ws);
  if (hipError_t e = run(parts, p, true, wide, s)) return e;
  return fold(a, ws, p.splits, (int)parts.ld, f32, s);
}

hipError_t launch_rows8_parts(const Rows8ProductArgs& a, const Rows8Plan& p, float* ws, hipStream_t s) {
  if (p.splits < 2 || a.N % 4 != 0) return hipErrorInvalidValue;
  return run(into_parts(a, ws), p, true, false, s);
}

}  // namespace cora
