// The paged K/V cache's bookkeeping and its writes.
//
// k_cache_plan: block tables and slot maps from request lengths.  With have_b = ceil(len_b / P),
// need_b = max(0, ceil((start_b + count_b) / P) - have_b) and exclusive prefix sums over the
// requests, page i of request b's new ones is free[n_free - 1 - (prefix(need)_b + i)] and row r of
// the chunk rows belongs to the request with cu_b <= r < cu_(b+1).  One workgroup does the prefix
// sums in LDS and the pages, four a thread at a time; the rows follow in the same launch when there
// are few of them and in a second one when there are many.
//
// k_cache_store: rotate-half RoPE on the q and k of the chunk's rows, q row-major, k and v into
// the pages in the order of the attention's matrix operands (cache_k_index, cache_v_index).
#include <limits.h>

#include <algorithm>

#include "cached.hpp"

namespace cora {

namespace {

constexpr int PT = 1024;  // threads of the plan's workgroup

// sums that stay at 2^32 - 1: 4096 requests may ask for more than that between them, what is granted
// fits the pool and the chunk, which are smaller
__device__ __forceinline__ uint32_t add_sat(uint32_t x, uint32_t y) { return __builtin_elementwise_add_sat(x, y); }

// inclusive saturating sums over the lanes of each row of 16
__device__ __forceinline__ uint32_t row_scan(uint32_t v) {
  v = add_sat(v, moved<0x111, 0xf>(v));
  v = add_sat(v, moved<0x112, 0xf>(v));
  v = add_sat(v, moved<0x114, 0xf>(v));
  return add_sat(v, moved<0x118, 0xf>(v));
}

// inclusive sums of two values over the workgroup, `carry` added and advanced by the totals
__device__ __forceinline__ void block_scan(uint32_t (&v)[2], uint32_t (&carry)[2], uint32_t (*part)[PT / 64]) {
  static_assert(PT / 64 == 16, "a row of lanes holds the wavefronts' totals");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    v[k] = row_scan(v[k]);
    v[k] = add_sat(v[k], moved<0x142, 0xa>(v[k]));  // row_bcast 15, 31
    v[k] = add_sat(v[k], moved<0x143, 0xc>(v[k]));
    if (lane == 63) part[k][wave] = v[k];
  }
  __syncthreads();
  const int totals = (int)row_scan(lane < 32 ? part[lane >> 4][lane & 15] : 0u);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const uint32_t before = wave > 0 ? (uint32_t)__builtin_amdgcn_readlane(totals, 16 * k + wave - 1) : 0u;
    v[k] = add_sat(add_sat(v[k], before), carry[k]);
    carry[k] = add_sat(carry[k], (uint32_t)__builtin_amdgcn_readlane(totals, 16 * k + 15));
  }
  __syncthreads();
}

// the greatest b in [0, B) with first[b] <= i  (first[0] = 0, ascending)
__device__ __forceinline__ int owner(const uint32_t* first, int B, uint32_t i) {
  int b = 0;
  for (int step = 1 << (31 - __clz(B)); step > 0; step >>= 1)
    if (b + step < B && first[b + step] <= i) b += step;
  return b;
}
// of i and the three after it, which mostly have the same; first[B] is the end
__device__ __forceinline__ void owners(const uint32_t* first, int B, uint32_t i, int (&b)[4]) {
  b[0] = owner(first, B, i);
#pragma unroll
  for (int u = 1; u < 4; ++u) {
    b[u] = b[u - 1];
    if (first[b[u] + 1] > i + u || i + u >= first[B]) continue;
    ++b[u];  // the next one, unless that is empty
    if (first[b[u] + 1] <= i + u) b[u] = owner(first, B, i + u);
  }
}

__device__ __forceinline__ int pages_of(int len, int shift) { return (int)(((int64_t)len + (1 << shift) - 1) >> shift); }

// Positions and slots of rows r .. r + 3.  `top` != null: the pages that the call takes are read from
// where they come from, since the table may not hold them yet.
__device__ __forceinline__ void place_rows(const CachePlanArgs& a, const uint32_t* first_row, uint32_t r,
                                           const uint32_t* first_page, const uint32_t* have, const int32_t* top) {
  const uint32_t total = first_row[a.B];
  int b[4] = {}, pos[4], page[4];
  if (r < total) owners(first_row, a.B, r, b);
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    page[u] = pos[u] = -1;
    if (r + u < total) {
      pos[u] = a.start[b[u]] + (int)(r + u - first_row[b[u]]);
      const int j = pos[u] >> a.shift;
      if (first_page && j >= (int)have[b[u]]) {
        const int i = (int)first_page[b[u]] + j - (int)have[b[u]];
        page[u] = top ? top[-i] : i;
      } else {
        page[u] = a.table[(int64_t)b[u] * a.max_pages + j];
      }
    }
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    if (r + u >= (uint32_t)a.rows) continue;
    a.positions[r + u] = pos[u];
    const bool known = pos[u] >= 0 && (uint32_t)page[u] < (uint32_t)a.n_pages;  // a table's nonsense stays outside
    a.slots[r + u] = known ? (page[u] << a.shift) + (pos[u] & ((1 << a.shift) - 1)) : -1;
  }
}

}  // namespace

// Bound by latency: a chain of loads, scans and stores of one workgroup.  Requests' sums are made once
// where none is refused, and after a reset, which leaves page i at the stack's i'th place, no page is
// read back.  64 requests of one token 4.8 us (a search of
// its own for every page and row, scans by lane exchanges through LDS: 6.0); 512 prompts of 545
// thousand rows 7.9 us (13.0) and 5.9 for the rows (7.2).
__global__ __launch_bounds__(PT) void k_cache_plan(CachePlanArgs a) {
  extern __shared__ uint32_t lds[];
  const int tid = threadIdx.x, B = a.B;
  uint32_t* first_page = lds;           // exclusive prefix of the granted pages (first: of those given back)
  uint32_t* first_row = lds + B + 1;    // exclusive prefix of the granted rows
  uint32_t* have = lds + 2 * (B + 1);   // pages a request holds already
  __shared__ uint32_t part[2][PT / 64];
  const int most = a.max_pages << a.shift;
  int n_free = a.reset ? a.n_pages : min(max(a.n_free[0], 0), a.n_pages);
  auto length = [&](int b) { return a.reset ? 0 : min(max(a.len[b], 0), most); };
  // the first requests' numbers, one a thread, are read once
  const int own_count = tid < B ? a.count[tid] : 0, own_start = tid < B ? a.start[tid] : 0, own_len = tid < B ? length(tid) : 0;

  // what each request asks for, and whether it gets it; pages that finished requests give back first
  uint32_t sum[2] = {0, 0};  // pages, rows
  uint32_t back[2] = {0, 0};
  bool returns = own_count < 0, refused = false;
  for (int b = tid + PT; b < B; b += PT) returns |= a.count[b] < 0;
  if (a.reset) {
    for (int i = tid; i < a.n_pages; i += PT) a.free[i] = a.n_pages - 1 - i;
  } else if (__syncthreads_or(returns)) {
    for (int b0 = 0; b0 < B; b0 += PT) {
      const int b = b0 + tid;
      const uint32_t n = b < B && a.count[b] < 0 ? (uint32_t)pages_of(length(b), a.shift) : 0u;
      uint32_t v[2] = {n, 0};
      block_scan(v, back, part);
      if (b < B) first_page[b] = v[0] - n;
    }
    if (tid == 0) first_page[B] = back[0];
    __syncthreads();  // first_page is whole
    const uint32_t given = min(back[0], (uint32_t)(a.n_pages - n_free));  // more only if a table holds a page twice
    for (uint32_t i = 4 * tid; i < given; i += 4 * PT) {
      int b[4];
      owners(first_page, B, i, b);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (i + u < given) a.free[n_free + i + u] = a.table[(int64_t)b[u] * a.max_pages + (i + u - first_page[b[u]])];
    }
    n_free += (int)given;
    __syncthreads();  // first_page is used anew, and the pages below are taken from the stack
  }

  for (int b0 = 0; b0 < B; b0 += PT) {
    const int b = b0 + tid;
    int status = 0;
    uint32_t need = 0, count = 0, held = 0;
    if (b < B) {
      const int start = b0 ? a.start[b] : own_start, len = b0 ? length(b) : own_len, n = max(b0 ? a.count[b] : own_count, 0);
      held = (uint32_t)pages_of(len, a.shift);
      if (n > 0) {
        if (start < 0 || start > len || (int64_t)start + n > most) status = CORA_ERR_INVALID_ARG;
        else {
          need = (uint32_t)max(0, pages_of(start + n, a.shift) - (int)held);
          count = (uint32_t)n;
        }
      }
    }
    uint32_t v[2] = {need, count};
    block_scan(v, sum, part);
    if (need > 0 && v[0] > (uint32_t)n_free) status = CORA_ERR_OOM;
    else if (count > 0 && v[1] > (uint32_t)a.rows) status = CORA_ERR_UNSUPPORTED;
    refused |= status == CORA_ERR_OOM || status == CORA_ERR_UNSUPPORTED;
    if (b < B) {
      first_page[b] = v[0] - need;
      first_row[b] = v[1] - count;
      have[b] = held;
      a.status[b] = status;
    }
  }
  if (__syncthreads_or(refused)) {  // the others' sums, without those
    sum[0] = sum[1] = 0;
    for (int b0 = 0; b0 < B; b0 += PT) {
      const int b = b0 + tid;
      uint32_t v[2] = {0, 0};
      if (b < B && a.status[b] == 0) {  // written by this thread
        const int n = max(a.count[b], 0);
        v[0] = n > 0 ? (uint32_t)max(0, pages_of(a.start[b] + n, a.shift) - (int)have[b]) : 0u;
        v[1] = (uint32_t)n;
      }
      const uint32_t need = v[0], count = v[1];
      block_scan(v, sum, part);
      if (b < B) {
        first_page[b] = v[0] - need;
        first_row[b] = v[1] - count;
      }
    }
  }
  const uint32_t pages = sum[0], rows = sum[1];
  if (tid == 0) {
    first_page[B] = pages;
    first_row[B] = rows;
    a.n_free[0] = n_free - (int)pages;
  }
  __syncthreads();

  const int32_t* top = a.reset ? nullptr : a.free + n_free - 1;
  // the pages from the last thread on, the rows from the first, so that few of both go side by side
  for (uint32_t i = 4 * (PT - 1 - tid); i < pages; i += 4 * PT) {
    int b[4], page[4];
    owners(first_page, B, i, b);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i + u < pages) page[u] = top ? top[-(int)(i + u)] : (int)(i + u);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i + u < pages) a.table[(int64_t)b[u] * a.max_pages + have[b[u]] + (i + u - first_page[b[u]])] = page[u];
  }
  if (!a.rows_apart)
    for (uint32_t r = 4 * tid; r < (uint32_t)a.rows; r += 4 * PT) place_rows(a, first_row, r, first_page, have, top);
  for (int b = tid; b <= B; b += PT) {
    a.cu[b] = (int)first_row[b];
    if (b == B) continue;
    const int n = (int)(first_row[b + 1] - first_row[b]);
    const bool own = b == tid;
    const int count = own ? own_count : a.count[b], start = own ? own_start : a.start[b], len = own ? own_len : length(b);
    a.len[b] = count < 0 ? 0 : (n > 0 ? max(len, start + n) : len);
  }
}

// the rows' positions and slots of a large chunk
__global__ __launch_bounds__(256) void k_cache_rows(CachePlanArgs a) {
  extern __shared__ uint32_t lds[];
  for (int b = threadIdx.x; b <= a.B; b += 256) lds[b] = (uint32_t)a.cu[b];
  __syncthreads();
  place_rows(a, lds, (blockIdx.x * 256 + threadIdx.x) * 4, nullptr, nullptr, nullptr);
}

hipError_t launch_cache_plan(CachePlanArgs a, hipStream_t s) {
  if (a.B > CACHE_MAX_BATCH) return hipErrorInvalidValue;
  a.rows_apart = a.rows > 8192;
  hipLaunchKernelGGL(k_cache_plan, dim3(1), dim3(PT), (size_t)(3 * (a.B + 1)) * 4, s, a);
  if (hipError_t e = hipGetLastError()) return e;
  if (a.rows_apart) hipLaunchKernelGGL(k_cache_rows, dim3(((unsigned)a.rows + 1023) / 1024), dim3(256),
                                       (size_t)(a.B + 1) * 4, s, a);
  return hipGetLastError();
}

// ---- rotary positions and the write into the pages -----------------------------------------------
namespace {

// x[n] = the sum over the partials' slabs, in their order, of what stands at `at + offset(n)` of each:
// four slabs' loads at a time (one number after the other, a store of 64 rows out of four slabs took
// 13 us, not 8.9)
template <int N, class T, class F>
__device__ __forceinline__ void add_slabs(const CacheStoreArgs& a, const float* at, F&& offset, T (&x)[N]) {
#pragma unroll
  for (int n = 0; n < N; ++n) x[n] = *reinterpret_cast<const T*>(at + offset(n));
  for (int sp = 1; sp < a.splits; sp += 4) {
    T t[4][N];
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int n = 0; n < N; ++n)
        t[u][n] = *reinterpret_cast<const T*>(at + min(sp + u, a.splits - 1) * a.slab + offset(n));
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int n = 0; n < N; ++n)
        if (sp + u < a.splits) x[n] += t[u][n];
  }
}

// 8 values each of the input row (bf16, or the sum of fp32 partials and the bias) from columns c0 and c1 on
template <bool F32>
__device__ __forceinline__ void load16(const CacheStoreArgs& a, int64_t row, int c0, int c1, float (&x0)[8], float (&x1)[8]) {
  if constexpr (F32) {
    f32x4_t x[4];
    add_slabs<4>(a, a.xf + row * a.ld, [&](int n) { return (n < 2 ? c0 : c1) + (n & 1) * 4; }, x);
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      if (a.bias) x[n] += *reinterpret_cast<const f32x4_t*>(a.bias + (n < 2 ? c0 : c1) + (n & 1) * 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) (n < 2 ? x0 : x1)[(n & 1) * 4 + i] = x[n][i];
    }
  } else {
    const u32x4_t w0 = *reinterpret_cast<const u32x4_t*>(a.xb + row * a.ld + c0);
    const u32x4_t w1 = *reinterpret_cast<const u32x4_t*>(a.xb + row * a.ld + c1);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x0[2 * i] = bf16_bits_to_f32(w0[i] & 0xffff); x0[2 * i + 1] = bf16_bits_to_f32(w0[i] >> 16);
      x1[2 * i] = bf16_bits_to_f32(w1[i] & 0xffff); x1[2 * i + 1] = bf16_bits_to_f32(w1[i] >> 16);
    }
  }
}

__device__ __forceinline__ u32x4_t pack8(const float (&v)[8]) {
  return u32x4_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
}

// whether row r is stored, and the slot it goes to
__device__ __forceinline__ bool slot_of(const CacheStoreArgs& a, int r, int& slot) {
  slot = a.slots[r];
  const int pos = a.positions[r];
  return slot >= 0 && slot < a.n_slots && pos >= 0 && (!a.rope || a.rope_by_row || pos < a.n_pos);
}

// q and k of 32 rows and NH x HPW heads from h0 on: hd / 16 threads per row and head, 16 dimensions
// each: j .. j + 7 and their partners j + hd / 2 .. (or, PAIRED, 16 neighbouring ones that hold 8
// pairs).  The NH heads of a thread share the row's angles.
template <int HD, bool F32, bool PAIRED, int NH>
__device__ __forceinline__ void store_qk(const CacheStoreArgs& a, int r, int h0) {
  constexpr int TPH = HD / 16, HPW = 8 / TPH;
  const int heads = a.H + a.Hkv, j = threadIdx.x % TPH;
  const int d0 = PAIRED ? j * 16 : j * 8, d1 = PAIRED ? d0 + 8 : d0 + HD / 2;
  h0 += threadIdx.x / TPH % HPW;
  float x0[NH][8], x1[NH][8];
#pragma unroll
  for (int n = 0; n < NH; ++n) {
    const int h = min(h0 + n * HPW, heads - 1);
    load16<F32>(a, r, h * HD + d0, h * HD + d1, x0[n], x1[n]);
  }
  int slot;
  const bool live = slot_of(a, r, slot);
  if (!live) {
#pragma unroll
    for (int n = 0; n < NH; ++n)
#pragma unroll
      for (int e = 0; e < 8; ++e) x0[n][e] = x1[n][e] = 0.f;
  } else if (a.rope) {
    // (cos, sin) of the 8 pairs: pair p of the head turns by pos theta^(-2 p / HD)
    const int at = a.rope_by_row ? r : a.positions[r];
    const f32x4_t* cs = reinterpret_cast<const f32x4_t*>(a.rope + ((int64_t)at * (HD / 2) + j * 8) * 2);
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const f32x4_t c = cs[p];
#pragma unroll
      for (int n = 0; n < NH; ++n)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const int e = 2 * p + q;
          float& u = PAIRED ? (e < 4 ? x0[n][2 * e] : x1[n][2 * e - 8]) : x0[n][e];
          float& w = PAIRED ? (e < 4 ? x0[n][2 * e + 1] : x1[n][2 * e - 7]) : x1[n][e];
          const float u0 = u, w0 = w;
          u = u0 * c[2 * q] - w0 * c[2 * q + 1];
          w = w0 * c[2 * q] + u0 * c[2 * q + 1];
        }
    }
  }
#pragma unroll
  for (int n = 0; n < NH; ++n) {
    const int h = h0 + n * HPW;
    if (h < a.H) {
      if (!a.q) continue;
      uint16_t* q = a.q + ((int64_t)r * a.H + h) * HD;
      *reinterpret_cast<u32x4_t*>(q + d0) = pack8(x0[n]);
      *reinterpret_cast<u32x4_t*>(q + d1) = pack8(x1[n]);
    } else if (h < heads && live) {
      const int page = slot >> a.shift, p = slot & ((1 << a.shift) - 1);
      uint16_t* k = a.k + ((((int64_t)page * a.Hkv + h - a.H) << a.shift) * HD);
      *reinterpret_cast<u32x4_t*>(k + cache_k_index(p, d0, HD)) = pack8(x0[n]);
      *reinterpret_cast<u32x4_t*>(k + cache_k_index(p, d1, HD)) = pack8(x1[n]);
    }
  }
}

// v of the 8 rows from r0 on by a wavefront, two dimensions a lane, one head of 128 or two of 64.
// Eight rows whose slots are an aligned run of 8 leave as one 16-byte store per dimension, by the
// wavefront in whose window the run begins; the other rows leave by themselves.
template <int HD, bool F32>
__device__ __forceinline__ void store_v(const CacheStoreArgs& a, int rows, int r0, int h) {
  constexpr int LPH = HD / 2;  // lanes per head
  const int lane = threadIdx.x & 63;
  h += lane / LPH;
  const int d = (lane % LPH) * 2;
  const bool on = h < a.Hkv;
  const int col = (a.H + a.Hkv + (on ? h : 0)) * HD + d;
  // two dimensions of rows r .. r + 7, behind the last one of that row
  auto load = [&](int r, uint32_t (&x)[8]) {
    if constexpr (F32) {
      f32x2_t v[8];
      add_slabs<8>(a, a.xf + col, [&](int e) { return (int64_t)min(r + e, rows - 1) * a.ld; }, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (a.bias) v[e] += *reinterpret_cast<const f32x2_t*>(a.bias + col);
        x[e] = pack_bf16x2(v[e][0], v[e][1]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = *reinterpret_cast<const uint32_t*>(a.xb + (int64_t)min(r + e, rows - 1) * a.ld + col);
    }
  };
  uint32_t x[8];
  load(r0, x);
  // lane t: the slot of row r0 - 7 + t, -1 where it is not stored
  int slot = -1;
  {
    const int r = r0 - 7 + lane;
    int s;
    if (lane < 22 && r >= 0 && r < rows && slot_of(a, r, s)) slot = s;
  }
  const uint64_t stored = __ballot(slot >= 0);
  uint64_t starts = __ballot(slot >= 0 && (slot & 7) == 0);
  const uint64_t follows = __ballot(slot >= 0 && __shfl_down(slot, 1, 64) == slot + 1);
#pragma unroll
  for (int e = 0; e < 7; ++e) starts &= follows >> e;
  uint64_t covered = starts;
#pragma unroll
  for (int e = 1; e < 8; ++e) covered |= starts << e;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int s = __builtin_amdgcn_readlane(slot, 7 + e);
    const int page = s >> a.shift, p = s & ((1 << a.shift) - 1);
    uint16_t* v = a.v + (((int64_t)page * a.Hkv + h) << a.shift) * HD;
    if (starts >> (7 + e) & 1) {
      uint32_t y[8];
      if (e == 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[i];
      } else {
        load(r0 + e, y);
      }
      u32x4_t lo, hi;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        lo[i] = (y[2 * i] & 0xffffu) | (y[2 * i + 1] << 16);
        hi[i] = (y[2 * i] >> 16) | (y[2 * i + 1] & 0xffff0000u);
      }
      if (on) {
        *reinterpret_cast<u32x4_t*>(v + cache_v_index(p, d, HD)) = lo;
        *reinterpret_cast<u32x4_t*>(v + cache_v_index(p, d + 1, HD)) = hi;
      }
    } else if ((stored & ~covered) >> (7 + e) & 1) {
      if (on) {
        v[cache_v_index(p, d, HD)] = (uint16_t)x[e];
        v[cache_v_index(p, d + 1, HD)] = (uint16_t)(x[e] >> 16);
      }
    }
  }
}

}  // namespace

// A workgroup takes 32 rows of NH (q and k) or one (v) head of 128, or twice as many of 64, so that
// the 16-byte pieces of a 32-key group's blocks come from one XCD and meet in its L2.  Bound by memory:
// 4096 rows of 32 + 32 + 32 heads of 128 42.7 us, 4.7 TB/s read and written, which a large copy reaches
// too (84 us in two launches that spread a row's heads over the card); 64 single tokens 4.4 us.
template <int HD, bool F32, bool PAIRED, int NH>
__global__ __launch_bounds__(256) void k_cache_store(CacheStoreArgs a) {
  constexpr int HPW = 128 / HD;
  const int qk = (a.H + a.Hkv + HPW * NH - 1) / (HPW * NH), groups = qk + (a.Hkv + HPW - 1) / HPW;
  const int group = blockIdx.x % groups, r0 = blockIdx.x / groups * 32, rows = min(a.rows, a.cu_end[0]);
  if (group < qk) {
    const int r = r0 + threadIdx.x / 8;
    if (r < rows) store_qk<HD, F32, PAIRED, NH>(a, r, group * HPW * NH);
  } else {
    const int r = r0 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 8;
    if (r < rows) store_v<HD, F32>(a, rows, r, (group - qk) * HPW);
  }
}

// The angles of a chunk's rows in a pass whose cache goes beyond the table of angles: once a pass, one
// thread a pair, in 64 bits (an angle of 2^30 in 32 bits is off by whole turns).
__global__ __launch_bounds__(256) void k_rope_rows(const int32_t* positions, const int32_t* cu_end, const float* table,
                                                   int n_pos, const double* freq, int rows, int half, float* out) {
  const int64_t i = blockIdx.x * 256ll + threadIdx.x;
  const int r = (int)(i / half), j = (int)(i % half);
  if (r >= min(rows, cu_end[0])) return;
  const int pos = positions[r];
  if (pos < 0) return;
  f32x2_t cs;
  if (pos < n_pos) {
    cs = *reinterpret_cast<const f32x2_t*>(table + ((int64_t)pos * half + j) * 2);
  } else {
    double sn, c;
    sincos(pos * freq[j], &sn, &c);
    cs = f32x2_t{(float)c, (float)sn};
  }
  *reinterpret_cast<f32x2_t*>(out + i * 2) = cs;
}

hipError_t launch_rope_rows(const int32_t* positions, const int32_t* cu_end, const float* table, int n_pos,
                            const double* freq, int rows, int half, float* out, hipStream_t s) {
  if (rows == 0) return hipSuccess;
  const int64_t wgs = ((int64_t)rows * half + 255) / 256;
  if (wgs > 0xffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL(k_rope_rows, dim3((unsigned)wgs), dim3(256), 0, s, positions, cu_end, table, n_pos, freq, rows,
                     half, out);
  return hipGetLastError();
}

// Windows x heads of 128 from which a thread takes four: 43.3 against 46.6 us at 8192 and 20.4 against
// 20.9 at 4096, but 15.2 against 14.0 at 2048; of 64, 14.8 against 14.2 at 5120.
constexpr int64_t MANY_HEADS = 4096;

namespace {

struct StoreGrid {
  bool many;
  int64_t workgroups;
};
StoreGrid store_grid(int rows, int H, int Hkv, int hd) {
  const int64_t windows = ((int64_t)rows + 31) / 32;
  const int hpw = hd == 128 ? 1 : 2;
  const bool many = hd == 128 && windows * (H + Hkv) >= MANY_HEADS;
  const int nh = hpw * (many ? 4 : 1);
  return {many, windows * ((H + Hkv + nh - 1) / nh + (Hkv + hpw - 1) / hpw)};
}

}  // namespace

int64_t cache_store_workgroups(int rows, int H, int Hkv, int hd) { return store_grid(rows, H, Hkv, hd).workgroups; }

hipError_t launch_cache_store(const CacheStoreArgs& a, int hd, bool paired, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  const bool f32 = a.xf != nullptr;
  if (paired && !f32) return hipErrorInvalidValue;
  const StoreGrid g = store_grid(a.rows, a.H, a.Hkv, hd);
  if (g.workgroups > most_workgroups(256)) return hipErrorInvalidValue;
  const dim3 grid((unsigned)g.workgroups);
#define STORE(HD_, NH_)                                                                                     \
  do {                                                                                                      \
    if (paired) hipLaunchKernelGGL((k_cache_store<HD_, true, true, NH_>), grid, dim3(256), 0, s, a);        \
    else if (f32) hipLaunchKernelGGL((k_cache_store<HD_, true, false, NH_>), grid, dim3(256), 0, s, a);     \
    else hipLaunchKernelGGL((k_cache_store<HD_, false, false, NH_>), grid, dim3(256), 0, s, a);             \
  } while (0)
  if (g.many) STORE(128, 4);
  else if (hd == 128) STORE(128, 1);
  else if (hd == 64) STORE(64, 1);
  else return hipErrorInvalidValue;
#undef STORE
  return hipGetLastError();
}

}  // namespace cora
