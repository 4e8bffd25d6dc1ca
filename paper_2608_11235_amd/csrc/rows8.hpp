// Rows of 8-bit floating point (e4m3) with a power of two as the scale of each 128 columns: their
// layout, the arguments of the kernels that make and multiply them.
#pragma once
#include "common.hpp"
#include "cora.h"
#include "internal.hpp"

namespace cora {

// Values of 16 rows and 128 columns are a block of 2 KB, the blocks of a row group one after another:
// byte (k / 64) 1024 + (k / 16 % 4) 256 + r 16 + k % 16 holds row r, column k, so that each half is one
// wavefront's load of 1 KB and its lane r + 16 g gets 16 columns of row r.  Scales (exponent + 127) of 16
// rows and four blocks are 64 bytes, byte 4 r + block: one dword a row.  Rows and columns up to multiples
// of 16 and 128 are zero, scales of blocks past the last one are 1.
constexpr int R8_BLOCK = 2048;
inline int64_t r8_groups(int64_t rows) { return (rows + 15) / 16; }
__host__ __device__ inline int r8_blocks(int cols) { return (cols + 127) / 128; }
__host__ __device__ inline int r8_quads(int cols) { return (cols + 511) / 512; }
constexpr int R8_MAX_COLS = 1 << 20, R8_MAX_ROWS = 1 << 27;
constexpr int R8_MAX_PRODUCT_ROWS = 1 << 21, R8_MAX_PRODUCT_COLS = 1 << 25;  // a launch's workgroups
constexpr int64_t R8_MAX_PRODUCT = 1LL << 40;  // tiles are counted in 31 bits, the smallest is 64 x 64

// The scale's byte of a block whose largest finite magnitude has these bits: with most = m 2^p, 1 <= m < 2,
// the exponent is p - 8 for m <= 1.75 (448 = 1.75 2^8), else p - 7; no less than -127.
__device__ __forceinline__ int r8_scale_byte(uint32_t most) {
  const int e = (int)(most >> 23) - 8 + ((most & 0x7fffffu) > 0x600000u ? 1 : 0);
  return most == 0 ? 127 : max(e, 0);
}
// one over that scale
__device__ __forceinline__ float r8_inverse(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }
__device__ __forceinline__ uint32_t r8_pack(float x0, float x1, float x2, float x3) {
  int w = 0;
  w = __builtin_amdgcn_cvt_pk_fp8_f32(x0, x1, w, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x2, x3, w, true);
}

// Where the quantized rows come from: bf16 or fp32 rows of stride ld; a layer's weights in 64 x 32 blocks; K panels
// [cols / 32][rows][32] (cols % 32 == 0 in both); or silu(gate) * up of bf16 rows that hold 16 gate and 16 up
// columns in turn.
enum R8Source { R8_BF16, R8_F32, R8_BLOCKS, R8_PANELS, R8_SWIGLU };
struct QuantizeArgs {
  const void* x; int64_t ld;
  int rows, cols;
  uint8_t *data, *scale;
};
hipError_t launch_quantize_rows(const QuantizeArgs& a, R8Source from, hipStream_t s);
inline size_t r8_data_bytes(int64_t rows, int cols) { return (size_t)r8_groups(rows) * r8_blocks(cols) * R8_BLOCK; }
inline size_t r8_scale_bytes(int64_t rows, int cols) { return (size_t)r8_groups(rows) * r8_quads(cols) * 64; }

// out[m, n] = sum over blocks b of 2^(a's and w's scales of b) times the products' sum, + bias[n]
struct Rows8ProductArgs {
  const uint8_t *a, *a_scale, *w, *w_scale;
  int M, N, K;
  const float* bias;
  void* out; int64_t ld;
};
// How a product runs, made from its sizes alone.
struct Rows8Plan {
  bool few;              // activations kept in registers (k_rows8_few), or tiles
  int cfg;               // tiles: their config
  int mb, nb, sq, kw, grid;  // few: groups of activation and weight rows and quads of blocks a wavefront, wavefronts along the columns
  int splits;            // workgroups along the columns, whose sums a second kernel adds
  size_t ws_floats;
  int rest, rest_cfg, rest_grid;  // tiles: the last weight rows that go to a launch of other tiles, or 0
};
struct Rows8Few { int kw; };
// wide: results in fp32 with sums of 32 bits (else those of the 8-bit instruction)
Rows8Plan rows8_plan(int M, int N, int K, bool wide, int num_cus);
Rows8Plan rows8_plan_few(int M, int N, int K, int nb, int sq, int ranges, bool wide, int num_cus);
int rows8_few_rows(bool wide);  // of a launch
Rows8Plan rows8_plan_tiles(int M, int N, int K, int cfg, int splits, int num_cus);
hipError_t launch_rows8_product(const Rows8ProductArgs& a, const Rows8Plan& p, bool f32, bool wide, float* ws, hipStream_t s);
// the same without bias, the splits' fp32 sums [splits][M][N] left in the workspace (splits > 1, N % 4 == 0)
hipError_t launch_rows8_parts(const Rows8ProductArgs& a, const Rows8Plan& p, float* ws, hipStream_t s);

// launch_residual_norm (internal.hpp) with its bf16 rows in 8 bits
hipError_t launch_residual_norm_rows8(float* h, const float* part, int splits, int rows, int d, const float* w,
                                      uint8_t* data, uint8_t* scale, float eps, hipStream_t s);

}  // namespace cora
