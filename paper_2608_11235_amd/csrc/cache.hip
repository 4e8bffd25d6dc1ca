// The paged K/V cache's bookkeeping and its writes.
//
// k_cache_plan: block tables and slot maps from request lengths.  With have_b = ceil(len_b / P),
// need_b = max(0, ceil((start_b + count_b) / P) - have_b) and exclusive prefix sums over the
// requests, page i of request b's new ones is free[n_free - 1 - (prefix(need)_b + i)] and row r of
// the chunk rows belongs to the request with cu_b <= r < cu_(b+1).  One workgroup does the prefix
// sums in LDS and, a thread per page, the pages; the rows follow in the same launch when there
// are few of them and in a second one, a thread per four rows, when there are many.
//
// k_cache_store: rotate-half RoPE on the q and k of the chunk's rows, q row-major, k and v into
// the pages in the order of the attention's matrix operands (cache_k_index, cache_v_index).
#include <limits.h>

#include <algorithm>

#include "common.hpp"
#include "internal.hpp"

namespace cora {

namespace {

constexpr int PT = 1024;  // threads of the plan's workgroup

// inclusive sum over the workgroup, `carry` added and advanced by the total
template <class T>
__device__ __forceinline__ T block_scan(T v, T& carry, T* part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const T u = __shfl_up(v, o, 64);
    if (lane >= o) v += u;
  }
  if (lane == 63) part[wave] = v;
  __syncthreads();
  T before = carry, total = 0;
#pragma unroll
  for (int w = 0; w < PT / 64; ++w) {
    const T p = part[w];
    if (w < wave) before += p;
    total += p;
  }
  carry += total;
  __syncthreads();
  return v + before;
}

// greatest b in [0, B) with first[b] <= i  (first[0] = 0, ascending)
__device__ __forceinline__ int owner(const uint32_t* first, int B, uint32_t i) {
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int m = (lo + hi) >> 1;
    if (first[m] <= i) lo = m;
    else hi = m;
  }
  return lo;
}

__device__ __forceinline__ int pages_of(int len, int shift) { return (int)(((int64_t)len + (1 << shift) - 1) >> shift); }

}  // namespace

// What is asked for is summed in 64 bits (4096 requests may ask for more than 2^32 rows between
// them), what is granted fits the pool and the chunk.
__global__ __launch_bounds__(PT) void k_cache_plan(CachePlanArgs a) {
  extern __shared__ uint32_t lds[];
  uint32_t* first_page = lds;                // exclusive prefix of the pages needed (or given back)
  uint32_t* first_row = lds + a.B + 1;       // exclusive prefix of the granted rows
  __shared__ uint32_t part[PT / 64];
  __shared__ unsigned long long part64[PT / 64];
  const int tid = threadIdx.x, B = a.B;
  const int most = a.max_pages << a.shift;
  int n_free = a.reset ? a.n_pages : min(max(a.n_free[0], 0), a.n_pages);
  if (a.reset)
    for (int i = tid; i < a.n_pages; i += PT) a.free[i] = a.n_pages - 1 - i;
  auto length = [&](int b) { return a.reset ? 0 : min(max(a.len[b], 0), most); };

  // pages that finished requests give back, on top of the stack in the requests' order
  uint32_t carry = 0;
  for (int b0 = 0; b0 < B; b0 += PT) {
    const int b = b0 + tid;
    const uint32_t back = b < B && a.count[b] < 0 ? (uint32_t)pages_of(length(b), a.shift) : 0u;
    const uint32_t inc = block_scan<uint32_t>(back, carry, part);
    if (b < B) first_page[b] = inc - back;
  }
  __syncthreads();  // first_page is whole
  const uint32_t room = (uint32_t)(a.n_pages - n_free);
  const uint32_t back = min(carry, room);  // more only if the tables hold a page twice
  for (uint32_t i = tid; i < back; i += PT) {
    const int b = owner(first_page, B, i);
    a.free[n_free + i] = a.table[(int64_t)b * a.max_pages + (i - first_page[b])];
  }
  n_free += (int)back;
  __syncthreads();  // first_page is used anew, and the pages below are taken from the stack

  // what each request asks for, and whether it gets it
  unsigned long long pages = 0, rows = 0;
  uint32_t granted_pages = 0, granted_rows = 0;
  for (int b0 = 0; b0 < B; b0 += PT) {
    const int b = b0 + tid;
    int status = 0, count = 0;
    uint32_t need = 0;
    if (b < B) {
      count = max(a.count[b], 0);
      const int start = a.start[b], len = length(b);
      if (count > 0) {
        if (start < 0 || start > len || (int64_t)start + count > most) status = CORA_ERR_INVALID_ARG;
        else need = (uint32_t)max(0, pages_of(start + count, a.shift) - pages_of(len, a.shift));
      }
      if (status) count = 0;
    }
    const auto pi = block_scan<unsigned long long>(need, pages, part64);
    const auto ri = block_scan<unsigned long long>((uint32_t)count, rows, part64);
    if (!status && need > 0 && pi > (uint32_t)n_free) status = CORA_ERR_OOM;
    else if (!status && count > 0 && ri > (uint32_t)a.rows) status = CORA_ERR_UNSUPPORTED;
    if (status) { need = 0; count = 0; }
    const uint32_t gp = block_scan<uint32_t>(need, granted_pages, part), gr = block_scan<uint32_t>((uint32_t)count, granted_rows, part);
    if (b < B) {
      first_page[b] = gp - need;
      first_row[b] = gr - count;
      a.cu[b] = (int)(gr - count);
      a.status[b] = status;
    }
  }
  if (tid == 0) {
    first_row[B] = granted_rows;
    a.cu[B] = (int)granted_rows;
  }
  __syncthreads();

  for (uint32_t i = tid; i < granted_pages; i += PT) {
    const int b = owner(first_page, B, i);
    const int j = pages_of(length(b), a.shift) + (int)(i - first_page[b]);
    a.table[(int64_t)b * a.max_pages + j] = a.free[n_free - 1 - (int)i];
  }
  __syncthreads();
  if (tid == 0) a.n_free[0] = n_free - (int)granted_pages;
  for (int b = tid; b < B; b += PT) {
    const int rows_b = (int)(first_row[b + 1] - first_row[b]);
    a.len[b] = a.count[b] < 0 ? 0 : (rows_b > 0 ? max(length(b), a.start[b] + rows_b) : length(b));
  }
  if (a.rows_apart) return;
  for (int r = tid; r < a.rows; r += PT) {
    int pos = -1, slot = -1;
    if ((uint32_t)r < granted_rows) {
      const int b = owner(first_row, B, (uint32_t)r);
      pos = a.start[b] + r - (int)first_row[b];
      slot = (a.table[(int64_t)b * a.max_pages + (pos >> a.shift)] << a.shift) + (pos & ((1 << a.shift) - 1));
    }
    a.positions[r] = pos;
    a.slots[r] = slot;
  }
}

// positions and slots of the rows, four to a thread, after cu and the tables are written
__global__ __launch_bounds__(256) void k_cache_rows(CachePlanArgs a) {
  const int r0 = (blockIdx.x * 256 + threadIdx.x) * 4;
  if (r0 >= a.rows) return;
  const int total = a.cu[a.B];
  int b = owner(reinterpret_cast<const uint32_t*>(a.cu), a.B, (uint32_t)r0);
  for (int r = r0; r < min(r0 + 4, a.rows); ++r) {
    int pos = -1, slot = -1;
    if (r < total) {
      while (b + 1 < a.B && a.cu[b + 1] <= r) ++b;
      pos = a.start[b] + r - a.cu[b];
      slot = (a.table[(int64_t)b * a.max_pages + (pos >> a.shift)] << a.shift) + (pos & ((1 << a.shift) - 1));
    }
    a.positions[r] = pos;
    a.slots[r] = slot;
  }
}

hipError_t launch_cache_plan(CachePlanArgs a, hipStream_t s) {
  if (a.B > CACHE_MAX_BATCH) return hipErrorInvalidValue;
  a.rows_apart = a.rows > 8192;
  hipLaunchKernelGGL(k_cache_plan, dim3(1), dim3(PT), (size_t)(2 * a.B + 2) * 4, s, a);
  if (hipError_t e = hipGetLastError()) return e;
  if (a.rows_apart) hipLaunchKernelGGL(k_cache_rows, dim3((a.rows + 1023) / 1024), dim3(256), 0, s, a);
  return hipGetLastError();
}

// ---- rotary positions and the write into the pages -----------------------------------------------
namespace {

// 8 values of the input row (bf16, or the sum of fp32 partials and the bias) from column c on
template <bool F32>
__device__ __forceinline__ void load8(const CacheStoreArgs& a, int64_t row, int c, float (&v)[8]) {
  if constexpr (F32) {
    const float* p = a.xf + row * a.ld + c;
    f32x4_t x0 = *reinterpret_cast<const f32x4_t*>(p), x1 = *reinterpret_cast<const f32x4_t*>(p + 4);
    for (int sp = 1; sp < a.splits; ++sp) {
      p += a.slab;
      x0 += *reinterpret_cast<const f32x4_t*>(p);
      x1 += *reinterpret_cast<const f32x4_t*>(p + 4);
    }
    if (a.bias) {
      x0 += *reinterpret_cast<const f32x4_t*>(a.bias + c);
      x1 += *reinterpret_cast<const f32x4_t*>(a.bias + c + 4);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = x0[i]; v[4 + i] = x1[i]; }
  } else {
    const u32x4_t w = *reinterpret_cast<const u32x4_t*>(a.xb + row * a.ld + c);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = bf16_bits_to_f32(w[i] & 0xffff); v[2 * i + 1] = bf16_bits_to_f32(w[i] >> 16); }
  }
}

__device__ __forceinline__ u32x4_t pack8(const float (&v)[8]) {
  return u32x4_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
}

// whether row r is stored, and the slot it goes to
__device__ __forceinline__ bool slot_of(const CacheStoreArgs& a, int r, int& slot) {
  slot = a.slots[r];
  const int pos = a.positions[r];
  return slot >= 0 && slot < a.n_slots && pos >= 0 && (!a.rope || pos < a.n_pos);
}

}  // namespace

// q and k: hd / 16 threads per row and head, 16 dimensions each: j .. j + 7 and their partners
// j + hd / 2 .. (or, PAIRED, 16 neighbouring ones that hold 8 pairs).
template <int HD, bool F32, bool PAIRED>
__global__ __launch_bounds__(256) void k_cache_store_qk(CacheStoreArgs a) {
  constexpr int TPH = HD / 16;
  const int heads = a.H + a.Hkv;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int j = (int)(i % TPH);
  const int64_t rh = i / TPH;
  const int r = (int)(rh / heads), h = (int)(rh % heads);
  if (r >= min(a.rows, a.cu_end[0])) return;
  const int d0 = PAIRED ? j * 16 : j * 8, d1 = PAIRED ? d0 + 8 : d0 + HD / 2;
  int slot;
  const bool live = slot_of(a, r, slot);
  if (h >= a.H && !live) return;
  float x0[8], x1[8];
  load8<F32>(a, r, h * HD + d0, x0);
  load8<F32>(a, r, h * HD + d1, x1);
  if (!live) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x0[e] = x1[e] = 0.f;
  } else if (a.rope) {
    // (cos, sin) of the 8 pairs: pair p of the head turns by pos theta^(-2 p / HD)
    const f32x4_t* cs = reinterpret_cast<const f32x4_t*>(a.rope + ((int64_t)a.positions[r] * (HD / 2) + j * 8) * 2);
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const f32x4_t c = cs[p];
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int e = 2 * p + q;
        float& u = PAIRED ? (e < 4 ? x0[2 * e] : x1[2 * e - 8]) : x0[e];
        float& w = PAIRED ? (e < 4 ? x0[2 * e + 1] : x1[2 * e - 7]) : x1[e];
        const float u0 = u, w0 = w;
        u = u0 * c[2 * q] - w0 * c[2 * q + 1];
        w = w0 * c[2 * q] + u0 * c[2 * q + 1];
      }
    }
  }
  if (h < a.H) {
    if (!a.q) return;
    uint16_t* q = a.q + ((int64_t)r * a.H + h) * HD;
    *reinterpret_cast<u32x4_t*>(q + d0) = pack8(x0);
    *reinterpret_cast<u32x4_t*>(q + d1) = pack8(x1);
  } else {
    const int page = slot >> a.shift, p = slot & ((1 << a.shift) - 1);
    uint16_t* k = a.k + ((((int64_t)page * a.Hkv + h - a.H) << a.shift) * HD);
    *reinterpret_cast<u32x4_t*>(k + cache_k_index(p, d0, HD)) = pack8(x0);
    *reinterpret_cast<u32x4_t*>(k + cache_k_index(p, d1, HD)) = pack8(x1);
  }
}

// v: a wavefront takes a window of 8 rows and, two dimensions a lane, one head of 128 or two of 64.
// Rows whose slots follow one another inside an aligned run of 8 leave as one 16-byte store per
// dimension.  A run belongs to the window in which it begins.
template <int HD, bool F32>
__global__ __launch_bounds__(256) void k_cache_store_v(CacheStoreArgs a) {
  constexpr int LPH = HD / 2, HPW = 64 / LPH;  // lanes per head, heads per wavefront
  const int lane = threadIdx.x & 63;
  const int rows = min(a.rows, a.cu_end[0]);
  const int hgroups = (a.Hkv + HPW - 1) / HPW;
  const int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r0 = (int)(unit / hgroups) * 8, h = (int)(unit % hgroups) * HPW + lane / LPH;
  if (r0 >= rows) return;
  const int d = (lane % LPH) * 2;
  const bool on = h < a.Hkv;
  const int col = (a.H + a.Hkv + h) * HD + d;
  auto load2 = [&](int r) -> uint32_t {
    if (!on) return 0;
    if constexpr (F32) {
      const float* p = a.xf + (int64_t)r * a.ld + col;
      float x = p[0], y = p[1];
      for (int sp = 1; sp < a.splits; ++sp) {
        p += a.slab;
        x += p[0];
        y += p[1];
      }
      if (a.bias) {
        x += a.bias[col];
        y += a.bias[col + 1];
      }
      return pack_bf16x2(x, y);
    } else {
      return *reinterpret_cast<const uint32_t*>(a.xb + (int64_t)r * a.ld + col);
    }
  };
  auto slot_or = [&](int r) {  // -1 where the row is not stored
    int s;
    return r < rows && slot_of(a, r, s) ? s : -1;
  };
  int prev = r0 > 0 ? slot_or(r0 - 1) : -1;
  for (int r = r0; r < min(r0 + 8, rows);) {
    const int s = slot_or(r);
    const bool begins = s >= 0 && !(prev >= 0 && s == prev + 1 && (s & 7));
    if (!begins) {
      prev = s;
      ++r;
      continue;
    }
    int n = 1, last = s;
    while (((s + n) & 7) && slot_or(r + n) == s + n) last = s + n++;
    const int page = s >> a.shift, p = s & ((1 << a.shift) - 1);
    uint16_t* v = a.v + (((int64_t)page * a.Hkv + h) << a.shift) * HD;
    if (n == 8) {
      uint32_t x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = load2(r + e);
      u32x4_t lo, hi;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        lo[e] = (x[2 * e] & 0xffffu) | (x[2 * e + 1] << 16);
        hi[e] = (x[2 * e] >> 16) | (x[2 * e + 1] & 0xffff0000u);
      }
      if (on) {
        *reinterpret_cast<u32x4_t*>(v + cache_v_index(p, d, HD)) = lo;
        *reinterpret_cast<u32x4_t*>(v + cache_v_index(p, d + 1, HD)) = hi;
      }
    } else {
      for (int e = 0; e < n; ++e) {
        const uint32_t x = load2(r + e);
        if (on) {
          v[cache_v_index(p + e, d, HD)] = (uint16_t)x;
          v[cache_v_index(p + e, d + 1, HD)] = (uint16_t)(x >> 16);
        }
      }
    }
    prev = last;
    r += n;
  }
}

hipError_t launch_cache_store(const CacheStoreArgs& a, int hd, bool paired, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  const bool f32 = a.xf != nullptr;
  if (paired && !f32) return hipErrorInvalidValue;
  const int64_t nqk = (int64_t)a.rows * (a.H + a.Hkv) * (hd / 16);
  const int64_t nv = (int64_t)((a.rows + 7) / 8) * (hd == 128 ? a.Hkv : (a.Hkv + 1) / 2);
  const dim3 gqk((unsigned)((nqk + 255) / 256)), gv((unsigned)((nv + 3) / 4));
#define STORE(HD_)                                                                                         \
  do {                                                                                                     \
    if (paired) hipLaunchKernelGGL((k_cache_store_qk<HD_, true, true>), gqk, dim3(256), 0, s, a);          \
    else if (f32) hipLaunchKernelGGL((k_cache_store_qk<HD_, true, false>), gqk, dim3(256), 0, s, a);       \
    else hipLaunchKernelGGL((k_cache_store_qk<HD_, false, false>), gqk, dim3(256), 0, s, a);               \
    if (f32) hipLaunchKernelGGL((k_cache_store_v<HD_, true>), gv, dim3(256), 0, s, a);                     \
    else hipLaunchKernelGGL((k_cache_store_v<HD_, false>), gv, dim3(256), 0, s, a);                        \
  } while (0)
  if (hd == 128) STORE(128);
  else if (hd == 64) STORE(64);
  else return hipErrorInvalidValue;
#undef STORE
  return hipGetLastError();
}

}  // namespace cora
