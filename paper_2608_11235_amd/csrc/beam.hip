// The best continuations of beams over beams and vocabulary.
//
// Beam k of a request has a running score; its candidates are score + log softmax(l)_v over the allowed
// ids of its row (not the mask id, not NaN, not -inf), and the W best of all beams of a request go on.
// Since a row's log sum is the same for all its ids, a row's own order is that of its logits (equal ones
// by id): k_beam_rows reads a range of a row once, adds up exp and keeps the range's W largest logits;
// k_beam_merge adds the ranges' sums, and puts the W best of a request's candidates in order.
//
// Sums of exp: the 16 terms of a thread and tile in fp32 relative to a power of two of the thread's own, all further sums
// and the scores in 64 bits.  Each term is off by its exponent's rounding (1.65e-7 at the most near the reference), the
// hardware's exponential (1.2e-7) and four additions: candidates of different beams are told apart to about 1e-7, to 7e-7 at the
// worst (2^18 ids; a row of 2^30 has so many small terms that it is 1.5e-6).
#include <limits.h>

#include <algorithm>

#include "cached.hpp"

namespace cora {

namespace {

constexpr int BT = 256;         // threads of a range
constexpr int BE = 16;          // logits of a thread and tile
constexpr int TILE = BT * BE;
constexpr int CAP = 512;       // held candidates of a range
constexpr int RANK = 8;          // compared at a time
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
constexpr float LOWEST = -3.3895313892515355e38f;  // bf16's lowest finite number
// LOG2E's own error, relative: a sum of 2^(v LOG2E) is that of exp(v (1 + this)), which for the terms that count,
// those near the largest, is a factor 1 + this times v
constexpr double LOG2E_OFF = -1.3349e-8;

// order of a logit: larger for larger numbers, equal for both zeros, 0 for what is no candidate
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t b = __float_as_uint(v + 0.f) >> 16;
  return v > -INFINITY ? ((b & 0x8000u) ? 0xffffu - b : b | 0x8000u) : 0u;
}
__device__ __forceinline__ float of_ordered(uint32_t o) {
  return bf16_bits_to_f32((o & 0x8000u) ? o & 0x7fffu : 0xffffu - o);
}
// a candidate: its order, then lower ids first; 0 is none
__device__ __forceinline__ uint64_t candidate(uint32_t o, int id) { return (uint64_t)o << 32 | (0xffffffffu - (uint32_t)id); }
__device__ __forceinline__ int id_of(uint64_t c) { return (int)(0xffffffffu - (uint32_t)c); }

// The W largest of list[0 .. n) in falling order at its front; their number.  The list's rest is undefined; it has
// room for RANK more.  RANK are compared at a time (one after the other, each waits for its own load from LDS).
__device__ __forceinline__ int keep_best(uint64_t* list, int n, int W, uint64_t* least) {
  const int tid = threadIdx.x;
  if (tid < RANK) list[n + tid] = 0;
  __syncthreads();
  uint64_t own[CAP / BT];
  int rank[CAP / BT];
#pragma unroll
  for (int e = 0; e < CAP / BT; ++e) {
    own[e] = 0;
    rank[e] = W;
    if (tid + e * BT < n) {
      own[e] = list[tid + e * BT];
      int r = 0;
      for (int i = 0; i < n; i += RANK) {
        uint64_t x[RANK];
#pragma unroll
        for (int u = 0; u < RANK; ++u) x[u] = list[i + u];
#pragma unroll
        for (int u = 0; u < RANK; ++u) r += x[u] > own[e] ? 1 : 0;
      }
      rank[e] = r;
    }
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < CAP / BT; ++e)
    if (rank[e] < W) {
      list[rank[e]] = own[e];
      if (rank[e] == W - 1 && own[e]) *least = own[e];
    }
  __syncthreads();
  return min(n, W);
}

}  // namespace

// 1024 x 152064 in 69 us (4.5 TB/s) with four workgroups of 256 threads a CU; of these (when all sums were fp32) without the
// candidates 59, without the exponentials 63,
// without both 57.  Slower were two workgroups of 512 (80), 32 logits a thread (105, in scratch memory), lists of the wavefronts' own
// in place of the workgroup's barriers (94: four times the candidates) and a cut at 64 or 128 held candidates (72, 79).
// A row's logits are loaded eight at a time, a tile ahead, whatever its alignment, so that equal rows have equal sums wherever
// they lie; the up to seven behind are one each of the first threads', before the first tile.
__global__ __launch_bounds__(BT, 4) void k_beam_rows(BeamArgs a) {
  __shared__ __attribute__((aligned(16))) uint64_t list[CAP + RANK];
  __shared__ uint64_t least;      // candidates below it are out
  __shared__ int held;
  __shared__ uint64_t group_best[64];  // of BT / 64 threads each
  __shared__ double sums[BT / 64], tops[BT / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = blockIdx.x / a.parts;
  const int part = blockIdx.x % a.parts;
  const bool none = !(a.score[row] > -INFINITY) || (a.done && a.done[row]);  // no candidates, or the one without logits
  const int W = a.W, trim = max(32, 2 * W);  // held candidates beyond which they are cut down to the W best
  const uint16_t* x = a.logits + row * a.ld;
  const int blocks = a.V / 8;
  const int tiles = (blocks + TILE / 8 - 1) / (TILE / 8);
  const int b0 = tiles * part / a.parts * (TILE / 8), b1 = min(tiles * (part + 1) / a.parts * (TILE / 8), blocks);  // blocks of this range
  const u32x4_any* body = reinterpret_cast<const u32x4_any*>(x);
  u32x4_t next[BE / 8] = {};
  auto load = [&](int at, bool any) {
    if (!any) return;
#pragma unroll
    for (int h = 0; h < BE / 8; ++h) next[h] = body[min(at + h * BT + tid, b1 - 1)];
  };
  load(b0, b0 < b1);  // on its way while the score is looked at
  if (none) return;
  if (tid == 0) {
    least = 0x80ull << 32;  // LOWEST
    held = 0;
  }

  float ref = 0.f, k = LOG2E, o = 0.f;
  double s = 0;
  auto refer = [&](float m) {  // what the thread's terms are relative to: a power of two
    ref = fminf(fmaxf(m, LOWEST), -LOWEST);
    k = fabsf(ref) >= 16384.f ? 1.f : LOG2E;  // from there on different bf16 numbers are 64 and more apart: 1 is as good
    o = k == 1.f ? -ref : -rintf(ref * LOG2E);
  };
  auto follow = [&](float m) {
    if (!(m > ref + 5.f)) return;  // terms beyond 2^8 would round their exponents coarser; from 2 on: 1024 x 152064 72.6 us a call, from 5 on 70.8
    const float was_k = k, was_o = o, was = ref;
    refer(m);
    s = was_k == LOG2E && k == LOG2E ? ldexp(s, (int)(o - was_o)) : s * fast_exp2((was - ref) * LOG2E);
  };

  // the logit behind the blocks that this thread has, if any
  int side = part == a.parts - 1 && tid < a.V - 8 * blocks ? 8 * blocks + tid : -1;
  if (side == a.mask_id) side = -1;
  const float sv = side >= 0 ? bf16_bits_to_f32(x[side]) : -INFINITY;

  uint64_t bound = 0x80ull << 32;
  float bound_v = LOWEST;
  for (int base = b0; base == b0 || base < b1; base += BT * BE / 8) {
    u32x4_t cur[BE / 8];
    float m8[BE / 8];
    const bool first = base == b0, any = b0 < b1;
    const int id0 = 8 * (base + tid);  // of the first logit; those of cur[h] are BT * 8 h behind
#pragma unroll
    for (int h = 0; h < BE / 8; ++h) cur[h] = next[h];
    load(min(base + BT * BE / 8, max(b1 - 1, 0)), any);  // past the last tile: not used
    if (base + BT * BE / 8 > b1 || (uint32_t)(a.mask_id - 8 * base) < (uint32_t)TILE) {  // the last tile, or the mask's
#pragma unroll
      for (int h = 0; h < BE / 8; ++h) {
        int at = base + h * BT + tid >= b1 ? INT_MIN : a.mask_id - id0 - h * BT * 8;  // which of the eight is out; INT_MIN: all
        asm volatile("" : "+v"(at));
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (at == e || at == INT_MIN)
            cur[h][e >> 1] = e & 1 ? (cur[h][e >> 1] & 0xffffu) | 0xff800000u : (cur[h][e >> 1] & 0xffff0000u) | 0xff80u;
      }
    }
    auto logit = [&](int h, int e) { return __uint_as_float(e & 1 ? cur[h][e >> 1] & 0xffff0000u : cur[h][e >> 1] << 16); };
#pragma unroll
    for (int h = 0; h < BE / 8; ++h) {
      m8[h] = logit(h, 0);
#pragma unroll
      for (int e = 1; e < 8; ++e) m8[h] = fmaxf(m8[h], logit(h, e));
    }
    float m = m8[0];
#pragma unroll
    for (int h = 1; h < BE / 8; ++h) m = fmaxf(m, m8[h]);
    if (first) {
      refer(fmaxf(m, sv));
      s = fast_exp2(fmaf(sv, k, o));
    } else {
      follow(m);
    }
    float t[BE / 4];  // in four steps: one after the other into the thread's sum, 600 equal ones would round the same way
#pragma unroll
    for (int q = 0; q < BE / 4; ++q) {
      auto term = [&](int e) { return fast_exp2(fmaf(logit(e >> 3, e & 7), k, o)); };
      t[q] = (term(4 * q) + term(4 * q + 1)) + (term(4 * q + 2) + term(4 * q + 3));
    }
    s += (t[0] + t[1]) + (t[2] + t[3]);

    if (first) {
      // W of 64 groups of threads hold a logit no smaller than the W'th of the groups' largest
      int at_m = 0;  // the lowest place of the thread's largest
#pragma unroll
      for (int e = BE - 1; e >= 0; --e) at_m = logit(e >> 3, e & 7) == m ? (e >> 3) * BT * 8 + (e & 7) : at_m;
      uint64_t best = candidate(ordered(m), id0 + at_m);
      if (side >= 0) {
        const uint64_t c = candidate(ordered(sv), side);
        best = c > best ? c : best;
      }
#pragma unroll
      for (int d = 1; d < BT / 64; d <<= 1) {
        const uint64_t c = __shfl_xor((unsigned long long)best, d, 64);
        best = c > best ? c : best;
      }
      if (tid % (BT / 64) == 0) group_best[tid / (BT / 64)] = best;
      __syncthreads();
      const uint64_t mine = group_best[lane];
      int rank = 0;
#pragma unroll 8
      for (int j = 0; j < 64; ++j) rank += group_best[j] > mine || (group_best[j] == mine && j < lane) ? 1 : 0;
      const uint64_t at = __ballot(rank == W - 1);
      const uint64_t t = __shfl((unsigned long long)mine, __ffsll((unsigned long long)at) - 1, 64);
      bound = t > bound ? t : bound;
      bound_v = of_ordered((uint32_t)(bound >> 32));
      if (tid == 0) least = bound;
      if (side >= 0 && candidate(ordered(sv), side) >= bound) list[atomicAdd(&held, 1)] = candidate(ordered(sv), side);  // 7 at the most
    }
    auto offer = [&]() {
#pragma unroll
      for (int h = 0; h < BE / 8; ++h) {
        if (!(m8[h] >= bound_v)) continue;
        int id = id0 + h * BT * 8;
        asm volatile("" : "+v"(id));  // made here: eight ids made before the branch cost a workgroup its place on the CU
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float v = logit(h, e);
          if (!(v >= bound_v)) continue;
          const uint64_t c = candidate(ordered(v), id + e);
          if (c >= bound) {
            const int at = atomicAdd(&held, 1);
            if (at < CAP) list[at] = c;
          }
        }
      }
    };
    auto cut = [&](int n) {
      n = keep_best(list, n, W, &least);
      bound = least;
      bound_v = of_ordered((uint32_t)(bound >> 32));
      return n;
    };
    offer();
    __syncthreads();
    int n = held;
    while (n > CAP) {  // more than fit: the bound of those that do, then this tile's again
      cut(CAP);
      for (int i = tid; i < W; i += BT) {
        const int id = id_of(list[i]);
        if (id >= 8 * base && id < 8 * b1) list[i] = 0;
      }
      if (tid == 0) held = W;
      __syncthreads();
      offer();
      __syncthreads();
      n = held;
    }
    if (n > trim) {
      n = cut(n);
      if (tid == 0) held = n;
    }
    __syncthreads();
  }
  // a wavefront's sum, relative to the largest of its threads' references
  double top = warp_max(ref), sum = s * (k == 1.f ? 1.0 : 1.0 - LOG2E_OFF * ref) * exp((k == 1.f ? (double)ref : -(double)o * 0.6931471805599453) - top);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 64);
  if (lane == 0) {
    tops[wave] = top;
    sums[wave] = sum;
  }
  const int n = keep_best(list, held, W, &least);  // its barriers come before what follows
  uint64_t* out = a.best + (row * a.parts + part) * W;
  for (int i = tid; i < W; i += BT) out[i] = i < n ? list[i] : 0;
  if (wave == BT / 64 - 1) {
    const double t = tops[lane & (BT / 64 - 1)];
    top = t;
#pragma unroll
    for (int d = BT / 128; d > 0; d >>= 1) top = fmax(top, __shfl_xor(top, d, 64));
    sum = sums[lane & (BT / 64 - 1)] * exp(t - top);
#pragma unroll
    for (int d = BT / 128; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 64);
    if (lane == 0) {
      a.stats[2 * (row * a.parts + part)] = top;
      a.stats[2 * (row * a.parts + part) + 1] = sum;
    }
  }
}

namespace {

// A candidate in order: its score's, then lower beams first, then its order in the row; 0 is none.
typedef uint64_t key_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ key_t key_of(double score, int beam, uint64_t which) {
  const uint64_t b = __builtin_bit_cast(uint64_t, score + 0.0);
  return key_t{b >> 63 ? ~b : b | 1ull << 63, (uint64_t)(63 - beam) << 48 | which};
}
__device__ __forceinline__ double score_of(key_t k) {
  return __builtin_bit_cast(double, k[0] >> 63 ? k[0] ^ 1ull << 63 : ~k[0]);
}
__device__ __forceinline__ bool before(key_t x, key_t y) { return x[0] > y[0] || (x[0] == y[0] && x[1] > y[1]); }
// how many of n keys come before that of four lanes, which go over a quarter each; the list has room for 4 RANK more,
// which are none
__device__ __forceinline__ int rank_of(const key_t* keys, int n, key_t mine) {
  int r = 0;
  for (int i = threadIdx.x & 3; i < n; i += 4 * RANK) {
    key_t x[RANK];
#pragma unroll
    for (int u = 0; u < RANK; ++u) x[u] = keys[i + 4 * u];
#pragma unroll
    for (int u = 0; u < RANK; ++u) r += before(x[u], mine) ? 1 : 0;
  }
  r += __shfl_xor(r, 1, 64);
  return r + __shfl_xor(r, 2, 64);
}

}  // namespace

static_assert(BEAM_MAX <= 64, "a beam's number in six bits above a candidate's 48");

// Bound by latency: the ranges' numbers, a logarithm a beam, and ranks by comparing all with all, four lanes a candidate.
// 128 requests of 8 x 16 candidates 5.3 us (a lane a candidate: 6.8).
__global__ __launch_bounds__(512) void k_beam_merge(BeamArgs a) {
  extern __shared__ __attribute__((aligned(16))) char mem[];
  const int tid = threadIdx.x, K = a.K, P = a.parts, W = a.W, lists = K * P;
  const int64_t row0 = (int64_t)blockIdx.x * K;
  key_t* keys = reinterpret_cast<key_t*>(mem);          // [max(W W, lists) + 4 RANK]
  double* base = reinterpret_cast<double*>(keys + max(W * W, lists) + 4 * RANK);  // [K] score minus the log of the row's sum; NaN: no candidate
  double* origin = base + K;                            // [K] which is relative to this (logits of 1e38 keep the score's bits)
  __shared__ int n_in;
  __shared__ key_t least;
  if (tid == 0) {
    n_in = 0;
    least = key_t{0, 0};
  }
  auto is_done = [&](int k) { return a.done && a.done[row0 + k]; };
  // the first candidate of a thread is on its way while the sums are made
  const uint64_t early = tid < lists * W ? a.best[row0 * P * W + tid] : 0;
  for (int k = tid >> 6; k < K; k += 8) {  // a wavefront a beam
    const int lane = tid & 63;
    const double s = a.score[row0 + k];
    double b = __builtin_nan(""), top = -INFINITY, sum = 0;
    if (s > -INFINITY && s < INFINITY) {
      if (is_done(k)) {
        b = s;
        top = 0;
      } else {
        const double* st = a.stats + 2 * (row0 + k) * P;
        for (int p = lane; p < P; p += 64) {
          const double t = st[2 * p], u = st[2 * p + 1], was = top;
          top = fmax(top, t);
          sum = sum * exp(was - top) + u * exp(t - top);
        }
        double all = top;
        for (int d = 1; d < min(P, 64); d <<= 1) all = fmax(all, __shfl_xor(all, d, 64));
        if (P > 1) sum *= exp(top - all);
        for (int d = 1; d < min(P, 64); d <<= 1) sum += __shfl_xor(sum, d, 64);
        top = all;
        if (sum > 0 && sum < INFINITY) b = s - log(sum);
      }
    }
    if (lane == 0) {
      base[k] = b;
      origin[k] = top;
    }
  }
  __syncthreads();
  // candidate i of list l (a beam's range), in the list's falling order
  auto get = [&](int l, int i) {
    const int k = l / P, c = l * W + i;
    const double b = base[k];
    if (!(b == b)) return key_t{0, 0};
    if (is_done(k)) return l % P == 0 && i == 0 ? key_of(b, k, 1) : key_t{0, 0};
    const uint64_t w = c == tid ? early : a.best[row0 * P * W + c];
    return w ? key_of(b + ((double)of_ordered((uint32_t)(w >> 32)) - origin[k]), k, w) : key_t{0, 0};
  };
  // the W'th of the lists' heads: a candidate behind it has that many others before it
  if (lists > W) {
    for (int l = tid; l < lists + 4 * RANK; l += 512) keys[l] = l < lists ? get(l, 0) : key_t{0, 0};
    __syncthreads();
    for (int l = tid >> 2; l < lists; l += 128) {
      const key_t mine = keys[l];
      const int rank = rank_of(keys, lists, mine);
      if (mine[0] && rank == W - 1) least = mine;
    }
    __syncthreads();
  }
  const key_t bound = least;
  __syncthreads();
  for (int c = tid; c < lists * W; c += 512) {
    const key_t mine = get(c / W, c % W);
    if (mine[0] && !before(bound, mine)) keys[atomicAdd(&n_in, 1)] = mine;  // W lists of W at the most
  }
  __syncthreads();
  const int n = n_in;
  if (tid < 4 * RANK) keys[n + tid] = key_t{0, 0};
  __syncthreads();
  const int64_t out = (int64_t)blockIdx.x * W;
  for (int c = tid >> 2; c < n; c += 128) {
    const key_t mine = keys[c];
    const int rank = rank_of(keys, n, mine), k = 63 - (int)(mine[1] >> 48);
    if (rank < W && (tid & 3) == 0) {
      a.token[out + rank] = is_done(k) ? a.done_token : id_of(mine[1]);
      a.parent[out + rank] = (int)(row0 + k);
      a.next[out + rank] = (float)score_of(mine);
    }
  }
  for (int c = n + tid; c < W; c += 512) {
    a.token[out + c] = -1;
    a.parent[out + c] = -1;
    a.next[out + c] = -INFINITY;
  }
}

// Ranges of a row: enough workgroups for the chip, of whole tiles.
BeamPlan beam_plan(int B, int K, int V, int W, int num_cus) {
  const int64_t rows = (int64_t)B * K;
  const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(4 * num_cus / std::max<int64_t>(rows, 1), (V + TILE - 1) / TILE));
  BeamPlan p;
  p.parts = (int)parts;
  p.bytes = (size_t)rows * p.parts * (16 + 8 * (size_t)W);
  return p;
}

hipError_t launch_vocab_beam(BeamArgs a, const BeamPlan& p, void* ws, hipStream_t s) {
  a.parts = p.parts;
  a.stats = static_cast<double*>(ws);
  a.best = reinterpret_cast<uint64_t*>(a.stats + 2 * (size_t)a.B * a.K * a.parts);
  hipLaunchKernelGGL(k_beam_rows, dim3((unsigned)((int64_t)a.B * a.K * a.parts)), dim3(BT), 0, s, a);
  if (hipError_t e = hipGetLastError()) return e;
  const size_t lds = 16 * ((size_t)std::max(a.W * a.W, a.K * a.parts) + 4 * RANK + a.K);
  hipLaunchKernelGGL(k_beam_merge, dim3((unsigned)a.B), dim3(512), lds, s, a);
  return hipGetLastError();
}

}  // namespace cora
