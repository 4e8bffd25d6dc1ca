// What sampling and the paged K/V cache share: their launches' arguments, the pages' layout and the
// sums over a wavefront.
#pragma once
#include "common.hpp"
#include "cora.h"
#include "internal.hpp"

namespace cora {

// Workgroups of a launch, whose threads are counted in 32 bits.
constexpr int64_t most_workgroups(int threads) { return 0xffffffffLL / threads; }

// ---- sampling -----------------------------------------------------------------------------
// Row r of the logits starts at logits + r * ld.  top_k, top_p, min_p may be null (off).
struct SampleArgs {
  const uint16_t* logits;
  int rows, V;
  int64_t ld;
  int mask_id;  // -1: none
  const float* temperature; const int32_t* top_k; const float* top_p; const float* min_p; const float* u;
  int32_t* token; float* conf;
};
constexpr int64_t SAMPLE_MAX_ROWS = most_workgroups(512);  // a workgroup a row, of 1024 threads up to 256 rows
hipError_t launch_vocab_sample(const SampleArgs& a, hipStream_t s);

// ---- paged K/V cache -----------------------------------------------------------------------
// A page of one kv head holds K and V of its positions as 32-key groups of 1 KB blocks, each the
// operand of one 16x16x32 MFMA in lane order (lane r + 16 g, 8 elements a lane).
// K: two halves (key bit 2) of head_dim / 32 blocks of 16 keys x 32 dimensions.  Key 8 (r / 4) + 4 half
// + r % 4 of the group is row r, so that the scores of a lane group are 8 neighbouring keys.
__host__ __device__ inline int cache_k_index(int p, int d, int hd) {
  const int k = p & 31;
  return (p >> 5) * 32 * hd + ((k >> 2) & 1) * 16 * hd + (d >> 5) * 512 + ((d >> 3) & 3) * 128 +
         (4 * (k >> 3) + (k & 3)) * 8 + (d & 7);
}
// V: head_dim / 16 blocks of 16 dimensions x 32 keys.
__host__ __device__ inline int cache_v_index(int p, int d, int hd) {
  return (p >> 5) * 32 * hd + (d >> 4) * 512 + ((p >> 3) & 3) * 128 + (d & 15) * 8 + (p & 7);
}
constexpr int CACHE_MAX_BATCH = CORA_CACHE_MAX_BATCH;
struct CachePlanArgs {
  int32_t *table, *len, *free, *n_free;
  const int32_t *start, *count;
  int32_t *cu, *positions, *slots, *status;
  int B, max_pages, n_pages, shift, rows, reset;  // page size 1 << shift
  int rows_apart;                                 // set by the launcher
};
hipError_t launch_cache_plan(CachePlanArgs a, hipStream_t s);
// Rows [0, cu_end[0]) of x = [q | k | v], bf16 (xb) or the sum of `splits` fp32 slabs and the bias
// (xf), row stride ld.  q may be null.
struct CacheStoreArgs {
  const uint16_t* xb; const float* xf; int64_t ld, slab; int splits; const float* bias;
  int rows, H, Hkv, shift, n_slots;
  const int32_t *positions, *slots, *cu_end;
  const float* rope; int n_pos;  // (cos, sin) [n_pos][hd / 2], null: no rotation
  int rope_by_row;               // `rope` holds the rows' own angles, [rows][hd / 2]
  uint16_t *k, *v, *q;
};
// out [rows][half]: (cos, sin) of the rows' positions times freq [half], from the table of n_pos
// positions where that has them.  Rows from cu_end[0] on and those without a position are left alone.
hipError_t launch_rope_rows(const int32_t* positions, const int32_t* cu_end, const float* table, int n_pos,
                            const double* freq, int rows, int half, float* out, hipStream_t s);
// paired: a head's dimensions come pair-interleaved (ROW_ROPE_PAIR) and stay so
int64_t cache_store_workgroups(int rows, int H, int Hkv, int hd);
hipError_t launch_cache_store(const CacheStoreArgs& a, int hd, bool paired, hipStream_t s);
struct CacheAttnArgs {
  const uint16_t *q, *k, *v;
  uint16_t* out;
  const int32_t *table, *len, *start, *cu;
  float *part_o, *part_ml;  // of each range: [rows][H][splits][hd], (max, sum) [rows][H][splits][2]
  int B, rows, H, Hkv, shift, n_pages, max_pages, causal, panels;
  float scale_log2;
  int G, tiles, per_request, splits, chunk;  // set from the plan
};
// tile_rows (token, head) rows a workgroup; a request in ranges of about `chunk` keys, no more than
// `splits` of them.  Made from sizes a caller keeps from call to call, never from the lengths on the device,
// so that a row's sums do not depend on what else is in the batch.
struct CacheAttnPlan {
  int tile_rows, tiles, splits, chunk;
  int per_request;  // tiles of each request where they have about as many rows, or 0
  int workgroups;
  size_t ws_floats;
};
CacheAttnPlan cache_attention_plan(int B, int rows, int H, int Hkv, int hd, int max_count, int max_len,
                                   int num_cus, size_t most_ws_floats);
hipError_t launch_cache_attention(CacheAttnArgs a, const CacheAttnPlan& p, int hd, float* ws, hipStream_t s);

}  // namespace cora

// ---- wavefront sums by lane moves (DPP) -----------------------------------------------------
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t moved(uint32_t v) {  // 0 where a lane has no source
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = moved<CTRL, ROWS>((uint32_t)b), hi = moved<CTRL, ROWS>((uint32_t)(b >> 32));
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// inclusive sums over the lanes: inside rows of 16, then the rows before
template <class T>
__device__ __forceinline__ T wave_scan(T v) {
  v += moved<0x111, 0xf>(v);  // row_shr 1, 2, 4, 8
  v += moved<0x112, 0xf>(v);
  v += moved<0x114, 0xf>(v);
  v += moved<0x118, 0xf>(v);
  v += moved<0x142, 0xa>(v);  // row_bcast 15, 31
  v += moved<0x143, 0xc>(v);
  return v;
}
