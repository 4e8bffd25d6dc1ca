// 8-bit rows and their products for gfx950.
//
// k_quantize_rows: x [R, K] in bf16 or fp32 -> e4m3 with a power of two 2^e for each 128 columns of a row:
// e is the least exponent with which 448, e4m3's largest number, reaches the largest finite magnitude of
// the block, so that x 2^-e is exact and the one rounding is that to e4m3 (nearest, ties to even; half a
// step is 2^-4 of the value).
//
// k_rows8_stream: few rows of activations times many rows of weights.  v_mfma_scale_f32_16x16x128_f8f6f4
// takes the 128 columns of a block with both scales and adds in fp32.
#include <algorithm>

#include "rows8.hpp"
#include "tiles.hpp"

namespace cora {

namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));
// 16 bytes at any alignment of two
struct __attribute__((packed, aligned(2))) bf16x8_any { uint16_t v[8]; };
struct __attribute__((packed, aligned(4))) f32x4_any { float v[4]; };

// columns c0 .. c0 + 15 of a row, zeros from column K on
template <bool F32>
__device__ __forceinline__ void load_chunk(const QuantizeArgs& a, int64_t row, int c0, float (&x)[16]) {
  if constexpr (F32) {
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
  } else {
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
  }
}

// The scale's byte of a block whose largest finite magnitude has these bits: with most = m 2^p, 1 <= m < 2,
// the exponent is p - 8 for m <= 1.75 (448 = 1.75 2^8), else p - 7; no less than -127.
__device__ __forceinline__ int scale_byte(uint32_t most) {
  const int e = (int)(most >> 23) - 8 + ((most & 0x7fffffu) > 0x600000u ? 1 : 0);
  return most == 0 ? 127 : max(e, 0);
}

// 16 values to e4m3: what is not finite becomes NaN
__device__ __forceinline__ u32x4_t pack_e4m3(const float (&x)[16], float by) {
  u32x4_t q;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    int w = 0;
    w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * t] * by, x[4 * t + 1] * by, w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * t + 2] * by, x[4 * t + 3] * by, w, true);
    q[t] = (uint32_t)w;
  }
  return q;
}

}  // namespace

// A thread has 16 columns of one row, eight neighbouring threads a block's row, two wavefronts a block.
template <bool F32>
__global__ __launch_bounds__(512) void k_quantize_rows(QuantizeArgs a) {
  const int tid = threadIdx.x, c = tid & 7, r = (tid >> 3) & 15;
  const int nk = r8_blocks(a.cols), nq = r8_quads(a.cols), quad = blockIdx.x % nq, kb = quad * 4 + (tid >> 7);
  const int64_t group = blockIdx.x / nq, row = group * 16 + r;
  float x[16];
  uint32_t most = 0;
  if (row < a.rows && kb < nk) {
    load_chunk<F32>(a, row, kb * 128 + c * 16, x);
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
  const int e = scale_byte(most);  // 127 + exponent
  if (kb < nk) {
    const u32x4_t q = pack_e4m3(x, __uint_as_float((uint32_t)(254 - e) << 23));
    *reinterpret_cast<u32x4_t*>(a.data + (group * nk + kb) * R8_BLOCK + c * 256 + r * 16) = q;
  }
  if (c == 0) a.scale[(group * nq + quad) * 64 + r * 4 + (tid >> 7)] = (uint8_t)e;
}

hipError_t launch_quantize_rows(const QuantizeArgs& a, bool f32, hipStream_t s) {
  const dim3 grid((unsigned)(r8_groups(a.rows) * r8_quads(a.cols)));  // below 2^23
  if (f32) hipLaunchKernelGGL((k_quantize_rows<true>), grid, dim3(512), 0, s, a);
  else hipLaunchKernelGGL((k_quantize_rows<false>), grid, dim3(512), 0, s, a);
  return hipGetLastError();
}

// ---- products ---------------------------------------------------------------------------------------
namespace {

__device__ __forceinline__ u32x4_t load16(__amdgpu_buffer_rsrc_t rs, int off) {
  return __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, 0));
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

// eight e4m3 numbers as bf16, which holds them exactly
__device__ __forceinline__ bf16x8_t widened(uint32_t lo, uint32_t hi) {
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
  const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// The same by the bf16 instruction, whose sums keep 32 bits: sum first, then the scales.  ws: the scales
// of the lane's four weight rows.
template <int U>
__device__ __forceinline__ f32x4_t mfma_wide(const u32x4_t (&w)[2], const u32x4_t (&a)[2], f32x4_t acc, u32x4_t ws, uint32_t as) {
  f32x4_t p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int t = 0; t < 2; ++t)
      p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widened(w[h][2 * t], w[h][2 * t + 1]), widened(a[h][2 * t], a[h][2 * t + 1]), p, 0, 0, 0);
#pragma unroll
  for (int e = 0; e < 4; ++e) acc[e] += ldexpf(p[e], (int)(ws[e] >> 8 * U & 255) + (int)(as >> 8 * U & 255) - 254);
  return acc;
}

constexpr int OOB = 0x7fffffff;  // an offset past every buffer: zeros, no traffic

// bias, rounding and store of columns col .. col + 3 of a row
template <bool F32>
__device__ __forceinline__ void store4(const Rows8ProductArgs& g, int64_t row, int col, f32x4_t x) {
  if (g.bias) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (col + e < g.N) x[e] += g.bias[col + e];
  }
  if constexpr (F32) {
    float* dst = static_cast<float*>(g.out) + row * g.ld + col;
    if (col + 3 < g.N && (g.ld & 3) == 0 && ((uintptr_t)g.out & 15) == 0) {
      *reinterpret_cast<f32x4_t*>(dst) = x;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (col + e < g.N) dst[e] = x[e];
    }
  } else {
    uint16_t* dst = static_cast<uint16_t*>(g.out) + row * g.ld + col;
    if (col + 3 < g.N && (g.ld & 3) == 0 && ((uintptr_t)g.out & 7) == 0) {
      *reinterpret_cast<u32x2_t*>(dst) = u32x2_t{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (col + e < g.N) dst[e] = (uint16_t)f32_to_bf16_bits(x[e]);
    }
  }
}

}  // namespace

// A workgroup has NB groups of 16 weight rows and MB of activations over all of K; its wavefronts share K
// in runs of four blocks and add their sums through LDS in their order.
template <int MB, int NB, int WAVES, bool F32, bool WIDE>
__global__ __launch_bounds__(WAVES * 64) void k_rows8_stream(Rows8ProductArgs g) {
  __shared__ f32x4_t part[WAVES][MB * NB][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nk = r8_blocks(g.K), nq = r8_quads(g.K);
  const int64_t wg0 = (int64_t)blockIdx.x * NB, ag0 = (int64_t)blockIdx.y * MB;
  const int wn = (int)min((int64_t)NB, (g.N + 15) / 16 - wg0), an = (int)min((int64_t)MB, (g.M + 15) / 16 - ag0);
  const auto w_rs = rsrc(g.w + wg0 * nk * R8_BLOCK, (int64_t)wn * nk * R8_BLOCK);
  const auto a_rs = rsrc(g.a + ag0 * nk * R8_BLOCK, (int64_t)an * nk * R8_BLOCK);
  const auto ws_rs = rsrc(g.w_scale + wg0 * nq * 64, (int64_t)wn * nq * 64);
  const auto as_rs = rsrc(g.a_scale + ag0 * nq * 64, (int64_t)an * nq * 64);
  const int per = (nq + WAVES - 1) / WAVES, q0 = wave * per, q1 = min(q0 + per, nq);

  struct Slice { u32x4_t w[NB][2], a[MB][2]; };
  Slice ring[4];
  typedef std::conditional_t<WIDE, u32x4_t, uint32_t> w_scale_t;
  w_scale_t ws[2][NB];
  uint32_t as[2][MB];
  auto issue = [&](int s, Slice& x) {
    const int at = s < nk && s < 4 * q1 ? s * R8_BLOCK + lane * 16 : -1;
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h) x.w[n][h] = load16(w_rs, at < 0 ? OOB : at + n * nk * R8_BLOCK + h * 1024);
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
      for (int h = 0; h < 2; ++h) x.a[m][h] = load16(a_rs, at < 0 ? OOB : at + m * nk * R8_BLOCK + h * 1024);
  };
  auto scales = [&](int q, w_scale_t (&w)[NB], uint32_t (&a)[MB]) {
    const int at = (lane & 15) * 4 + q * 64;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      if constexpr (WIDE) w[n] = load16(ws_rs, q < q1 ? (lane >> 4) * 16 + q * 64 + n * nq * 64 : OOB);
      else w[n] = __builtin_amdgcn_raw_buffer_load_b32(ws_rs, q < q1 ? at + n * nq * 64 : OOB, 0, 0);
    }
#pragma unroll
    for (int m = 0; m < MB; ++m) a[m] = __builtin_amdgcn_raw_buffer_load_b32(as_rs, q < q1 ? at + m * nq * 64 : OOB, 0, 0);
  };
  f32x4_t acc[MB][NB] = {};
  if (q0 < q1) {
    scales(q0, ws[0], as[0]);
#pragma unroll
    for (int u = 0; u < 4; ++u) issue(4 * q0 + u, ring[u]);
    for (int q = q0; q < q1; ++q) {
      scales(q + 1, ws[1], as[1]);
      auto step = [&](auto u_c) {
        constexpr int U = decltype(u_c)::value;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int m = 0; m < MB; ++m)
#pragma unroll
          for (int n = 0; n < NB; ++n) {
            if constexpr (WIDE) acc[m][n] = mfma_wide<U>(ring[U].w[n], ring[U].a[m], acc[m][n], ws[0][n], as[0][m]);
            else acc[m][n] = mfma<U>(both(ring[U].w[n][0], ring[U].w[n][1]), both(ring[U].a[m][0], ring[U].a[m][1]), acc[m][n],
                                     ws[0][n], as[0][m]);
          }
        __builtin_amdgcn_sched_barrier(0);
        issue(4 * (q + 1) + U, ring[U]);
      };
      step(std::integral_constant<int, 0>{});
      step(std::integral_constant<int, 1>{});
      step(std::integral_constant<int, 2>{});
      step(std::integral_constant<int, 3>{});
#pragma unroll
      for (int n = 0; n < NB; ++n) ws[0][n] = ws[1][n];
#pragma unroll
      for (int m = 0; m < MB; ++m) as[0][m] = as[1][m];
    }
  }
#pragma unroll
  for (int m = 0; m < MB; ++m)
#pragma unroll
    for (int n = 0; n < NB; ++n) part[wave][m * NB + n][lane] = acc[m][n];
  __syncthreads();
  for (int t = wave; t < MB * NB; t += WAVES) {
    f32x4_t x = part[0][t][lane];
#pragma unroll
    for (int v = 1; v < WAVES; ++v) x += part[v][t][lane];
    const int64_t row = (ag0 + t / NB) * 16 + (lane & 15);
    const int64_t col = (wg0 + t % NB) * 16 + 4 * (lane >> 4);
    if (row < g.M && col < g.N) store4<F32>(g, row, (int)col, x);
  }
}

// Tiles of many rows.  A workgroup of WM x WN wavefronts owns a tile, a wavefront TM x TN blocks of
// 16 x 16.  Two stages of 128 columns in LDS, filled by loads that write LDS directly, hold operands and
// scales as they lie in memory.  The MFMAs of a section work from registers; each fragment is reloaded with the
// next section's as soon as its last MFMA is issued, half the section before it is needed: the first
// TM / 2 rows with all columns, then the others, so that columns are free one by one in the second half.
// The section's one barrier stands before the first reload: what it waits for (the next stage's loads, this
// wavefront's reads of the stage that is overwritten from then on) is long done.
template <int WM, int WN, int TM, int TN>
__global__ __launch_bounds__(WM * WN * 64, 2) void k_rows8_tiles(Rows8ProductArgs g, float* parts, int splits, int f32) {
  constexpr int NW = WM * WN, BM = WM * TM * 16, BN = WN * TN * 16, GA = BM / 16, GB = BN / 16;
  constexpr int STAGE = (BM + BN) * 132;                 // 128 columns and a dword of scales a row
  constexpr int LPW = (GA + GB) * 2 / NW;                // loads of 1 KB a wavefront
  static_assert((GA + GB) % NW == 0 && (BM + BN) % (NW * 64) == 0, "every wavefront loads alike");
  constexpr int SPW = (BM + BN) / (NW * 64);             // loads of 64 scales a wavefront
  static_assert(TM % 2 == 0, "two halves");
  extern __shared__ __attribute__((aligned(1024))) char stages[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;
  const int li = xcd_remap(blockIdx.x, gridDim.x), n_tiles = gridDim.x / splits, split = li / n_tiles;
  int tile_m, tile_n;
  tile_of(li - split * n_tiles, (g.M + BM - 1) / BM, n_tiles, tile_m, tile_n);
  const int nk_all = r8_blocks(g.K), nq = r8_quads(g.K);
  const int k0 = (int)((int64_t)nk_all * split / splits), nk = (int)((int64_t)nk_all * (split + 1) / splits) - k0;
  const int ga0 = tile_m * GA, gb0 = tile_n * GB;        // first row groups
  const int a_last = (g.M + 15) / 16 - 1 - ga0, b_last = (g.N + 15) / 16 - 1 - gb0;

  // this wavefront's loads: LPW / 2 row groups of A or W, clamped to the last one, and 64 scales SPW times
  u32x4_t rs[LPW / 2], ss[SPW];
  int vo[LPW / 2], vs[SPW];
  const u32x4_t a_rs = buffer_rsrc(g.a + (int64_t)ga0 * nk_all * R8_BLOCK, (int64_t)(a_last + 1) * nk_all * R8_BLOCK);
  const u32x4_t b_rs = buffer_rsrc(g.w + (int64_t)gb0 * nk_all * R8_BLOCK, (int64_t)(b_last + 1) * nk_all * R8_BLOCK);
  const u32x4_t as_rs = buffer_rsrc(g.a_scale + (int64_t)ga0 * nq * 64, (int64_t)(a_last + 1) * nq * 64);
  const u32x4_t bs_rs = buffer_rsrc(g.w_scale + (int64_t)gb0 * nq * 64, (int64_t)(b_last + 1) * nq * 64);
#pragma unroll
  for (int t = 0; t < LPW / 2; ++t) {
    const int grp = wave * (LPW / 2) + t;
    const bool is_a = grp < GA;
    rs[t] = is_a ? a_rs : b_rs;
    vo[t] = (is_a ? min(grp, a_last) : min(grp - GA, b_last)) * nk_all * R8_BLOCK + lane * 16;
  }
#pragma unroll
  for (int t = 0; t < SPW; ++t) {
    const int row0 = (wave * SPW + t) * 64;
    const bool is_a = row0 < BM;
    const int row = (is_a ? row0 : row0 - BM) + lane;
    ss[t] = is_a ? as_rs : bs_rs;
    vs[t] = min(row >> 4, is_a ? a_last : b_last) * nq * 64 + (row & 15) * 4;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)stages;
  auto issue = [&](int kt, uint32_t st, int t) {  // load t of slice kt into the stage at st
    const int k = k0 + kt;
    if (t < LPW) load_lds(lds0 + st + (wave * LPW + t) * 1024, vo[t / 2], rs[t / 2], k * R8_BLOCK + (t & 1) * 1024);
    else load_lds_dword(lds0 + st + (BM + BN) * 128 + (wave * SPW + t - LPW) * 256, vs[t - LPW < 0 ? 0 : t - LPW], ss[t - LPW < 0 ? 0 : t - LPW], (k >> 2) * 64);
  };

  f32x4_t acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  i32x8_t fa[TM], fb[TN];
  uint32_t sa[TM], sb[TN];
  const int a_at = wm * TM * R8_BLOCK + lane * 16, b_at = (GA + wn * TN) * R8_BLOCK + lane * 16;
  const int as_at = (BM + BN) * 128 + (wm * TM * 16 + (lane & 15)) * 4, bs_at = (BM + BN) * 128 + (BM + wn * TN * 16 + (lane & 15)) * 4;
  auto frag = [&](int at) {
    return both(*reinterpret_cast<const u32x4_t*>(stages + at), *reinterpret_cast<const u32x4_t*>(stages + at + 1024));
  };
  auto read_a = [&](int st, int by, int i) {
    fa[i] = frag(st + a_at + i * R8_BLOCK);
    sa[i] = *reinterpret_cast<const uint8_t*>(stages + st + as_at + by + i * 64);
  };
  auto read_b = [&](int st, int by, int j) {
    fb[j] = frag(st + b_at + j * R8_BLOCK);
    sb[j] = *reinterpret_cast<const uint8_t*>(stages + st + bs_at + by + j * 64);
  };
  constexpr int NM = TM * TN, HALF = TM / 2, BAR = NM / 2 - 2 < 0 ? 0 : NM / 2 - 2, ALL = LPW + SPW;
  auto section = [&](auto more_c, int kt, int st, int nx) {
    constexpr bool MORE = decltype(more_c)::value;
    const int by = (k0 + kt + 1) & 3;
#pragma unroll
    for (int q = 0; q < NM; ++q) {
      const int half = q / (HALF * TN), j = q % (HALF * TN) / HALF, i = half * HALF + q % HALF;
      if (MORE && q == BAR) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
      }
      acc[i][j] = mfma<0>(fb[j], fa[i], acc[i][j], sb[j], sa[i]);
      if constexpr (MORE) {
        if (j == TN - 1) read_a(nx, by, i);
        if (half == 1 && i == TM - 1) read_b(nx, by, j);
#pragma unroll
        for (int t = 0; t < ALL; ++t)
          if (BAR + t * (NM - BAR) / ALL == q) issue(min(kt + 2, nk - 1), (uint32_t)st, t);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  if (nk > 0) {
#pragma unroll
    for (int t = 0; t < ALL; ++t) issue(0, 0, t);
#pragma unroll
    for (int t = 0; t < ALL; ++t) issue(min(1, nk - 1), STAGE, t);
    wait_vm<ALL>();
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TM; ++i) read_a(0, k0 & 3, i);
#pragma unroll
    for (int j = 0; j < TN; ++j) read_b(0, k0 & 3, j);
    int st = 0;
    for (int kt = 0; kt + 1 < nk; ++kt) {
      section(std::true_type{}, kt, st, STAGE - st);
      st = STAGE - st;
    }
    section(std::false_type{}, nk - 1, 0, 0);
    wait_vm<0>();
  }

  // a lane holds row lane % 16 and columns 4 (lane / 16) .. + 3 of each block
  const int row0 = tile_m * BM + wm * TM * 16 + (lane & 15), col0 = tile_n * BN + wn * TN * 16 + 4 * (lane >> 4);
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int row = row0 + i * 16;
    if (row >= g.M) continue;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int col = col0 + j * 16;
      if (col >= g.N) continue;
      store4<false>(g, row, col, acc[i][j]);
    }
  }
}

Rows8Plan rows8_plan(int, int, int, int) { return Rows8Plan{0}; }

template <int MB, int NB, int WAVES>
static hipError_t run_stream(const Rows8ProductArgs& a, bool f32, hipStream_t s) {
  const dim3 grid((unsigned)((r8_groups(a.N) + NB - 1) / NB), (unsigned)((r8_groups(a.M) + MB - 1) / MB));
  if (grid.y > 65535) return hipErrorInvalidValue;
  if (f32) hipLaunchKernelGGL((k_rows8_stream<MB, NB, WAVES, true, true>), grid, dim3(WAVES * 64), 0, s, a);
  else hipLaunchKernelGGL((k_rows8_stream<MB, NB, WAVES, false, false>), grid, dim3(WAVES * 64), 0, s, a);
  return hipGetLastError();
}

template <int WM, int WN, int TM, int TN>
static hipError_t run_tiles(const Rows8ProductArgs& a, hipStream_t s) {
  constexpr int BM = WM * TM * 16, BN = WN * TN * 16;
  constexpr unsigned LDS = 2 * (BM + BN) * 132;
  static_assert(LDS <= 160 * 1024, "LDS of a CU");
  const int grid = ((a.M + BM - 1) / BM) * ((a.N + BN - 1) / BN);
  hipLaunchKernelGGL((k_rows8_tiles<WM, WN, TM, TN>), dim3(grid), dim3(WM * WN * 64), LDS, s, a, nullptr, 1, 0);
  return hipGetLastError();
}

hipError_t launch_rows8_product(const Rows8ProductArgs& a, const Rows8Plan&, bool f32, float*, hipStream_t s) {
  if (!f32 && a.M > 64) return run_tiles<4, 2, 4, 8>(a, s);
  if (a.M <= 16) return run_stream<1, 2, 4>(a, f32, s);
  if (a.M <= 32) return run_stream<2, 2, 4>(a, f32, s);
  return run_stream<4, 2, 4>(a, f32, s);
}

}  // namespace cora
