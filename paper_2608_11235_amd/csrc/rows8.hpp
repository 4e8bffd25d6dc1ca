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

struct QuantizeArgs {
  const void* x; int64_t ld;  // bf16, or fp32
  int rows, cols;
  uint8_t *data, *scale;
};
hipError_t launch_quantize_rows(const QuantizeArgs& a, bool f32, hipStream_t s);

// out[m, n] = sum over blocks b of 2^(a's and w's scales of b) times the products' sum, + bias[n]
struct Rows8ProductArgs {
  const uint8_t *a, *a_scale, *w, *w_scale;
  int M, N, K;
  const float* bias;
  void* out; int64_t ld;
};
struct Rows8Plan {
  size_t ws_floats;
};
Rows8Plan rows8_plan(int M, int N, int K, int num_cus);
hipError_t launch_rows8_product(const Rows8ProductArgs& a, const Rows8Plan& p, bool f32, float* ws, hipStream_t s);

}  // namespace cora
