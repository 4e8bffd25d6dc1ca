// The best continuations of beams over beams and vocabulary.
//
// Beam k of a request has a running score; its candidates are score + log softmax(l)_v over the allowed
// ids of its row (not the mask id, not NaN, not -inf), and the W best of all beams of a request go on.
// Since a row's log sum is the same for all its ids, a row's own order is that of its logits (equal ones
// by id): k_beam_rows reads a range of a row once, adds up exp and keeps the range's W largest logits;
// k_beam_merge adds the ranges' sums, and puts the W best of a request's candidates in order.
//
// Sums of exp: a thread's terms in fp32 relative to a power of two of its own, all further sums and the
// scores in 64 bits, so that candidates of different beams are told apart to about 1e-7.
#include <limits.h>

#include <algorithm>

#include "cached.hpp"

namespace cora {

namespace {

constexpr int BT = 512;         // threads of a range
constexpr int BE = 16;          // logits of a thread and tile
constexpr int TILE = BT * BE;
constexpr int CAP = 1024;       // held candidates of a range
constexpr int TRIM = 512;       // cut down to the W best beyond that
constexpr float LOWEST = -3.3895313892515355e38f;  // bf16's lowest finite number
// LOG2E's own error, relative: a sum of 2^(v LOG2E) is that of exp(v (1 + this)), which for the terms that count,
// those near the largest, is a factor 1 + this times v
constexpr double LOG2E_OFF = -1.3349e-8;

struct __attribute__((packed, aligned(2))) bf16x8_any { uint16_t v[8]; };

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

// The W largest of list[0 .. n) in falling order at its front; their number.  The list's rest is undefined.
__device__ __forceinline__ int keep_best(uint64_t* list, int n, int W, uint64_t* least) {
  uint64_t own[CAP / BT];
  int rank[CAP / BT];
#pragma unroll
  for (int e = 0; e < CAP / BT; ++e) {
    const int at = threadIdx.x + e * BT;
    own[e] = at < n ? list[at] : 0;
    rank[e] = 0;
  }
  for (int i = 0; i < n; ++i) {
    const uint64_t x = list[i];
#pragma unroll
    for (int e = 0; e < CAP / BT; ++e) rank[e] += x > own[e] ? 1 : 0;
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < CAP / BT; ++e)
    if (threadIdx.x + e * BT < n && rank[e] < W) {
      list[rank[e]] = own[e];
      if (rank[e] == W - 1 && own[e]) *least = own[e];
    }
  __syncthreads();
  return min(n, W);
}

}  // namespace

__global__ __launch_bounds__(BT) void k_beam_rows(BeamArgs a) {
  __shared__ uint64_t list[CAP];
  __shared__ uint64_t least;      // candidates below it are out
  __shared__ int held;
  __shared__ uint64_t group_best[64];
  __shared__ double sums[BT / 64], tops[BT / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = blockIdx.x / a.parts;
  const int part = blockIdx.x % a.parts;
  const float score = a.score[row];
  if (!(score > -INFINITY) || (a.done && a.done[row])) return;  // no candidates, or the one without logits
  const int lo = part * a.chunk, hi = min(a.V, lo + a.chunk), W = a.W;
  const uint16_t* x = a.logits + row * a.ld;
  if (tid == 0) {
    least = 0x80ull << 32;  // LOWEST
    held = 0;
  }
  __syncthreads();

  float ref = 0.f, k = LOG2E, o = 0.f, s = 0.f;
  auto refer = [&](float m) {  // the power of two that the thread's terms are relative to
    ref = fminf(fmaxf(m, LOWEST), -LOWEST);
    k = fabsf(ref) >= 16384.f ? 1.f : LOG2E;  // from there on different bf16 numbers are 64 and more apart
    o = k == 1.f ? -ref : -rintf(ref * LOG2E);
  };
  for (int base = lo; base < hi; base += TILE) {
    float v[BE];
    float m8[BE / 8];
#pragma unroll
    for (int h = 0; h < BE / 8; ++h) {
      const int i = base + h * BT * 8 + tid * 8;
      if (i + 8 <= hi) {
        const bf16x8_any w = *reinterpret_cast<const bf16x8_any*>(x + i);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[8 * h + e] = bf16_bits_to_f32(w.v[e]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[8 * h + e] = i + e < hi ? bf16_bits_to_f32(x[i + e]) : -INFINITY;
      }
      const uint32_t at = (uint32_t)(a.mask_id - i);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (at == (uint32_t)e) v[8 * h + e] = -INFINITY;
      m8[h] = v[8 * h];
#pragma unroll
      for (int e = 1; e < 8; ++e) m8[h] = fmaxf(m8[h], v[8 * h + e]);
    }
    const float m = fmaxf(m8[0], m8[1]);
    if (base == lo) refer(m);
    else if (m > ref + 60.f) {
      const float was_k = k, was_o = o, was = ref;
      refer(m);
      s = was_k == LOG2E && k == LOG2E ? s * fast_exp2(o - was_o) : s * fast_exp2((was - ref) * LOG2E);
    }
#pragma unroll
    for (int e = 0; e < BE; ++e) s += fast_exp2(fmaf(v[e], k, o));

    if (base == lo) {
      // W of 64 groups of eight threads hold a logit no smaller than the W'th of the groups' largest
      uint64_t best = 0;
#pragma unroll
      for (int h = 0; h < BE / 8; ++h)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint64_t c = candidate(ordered(v[8 * h + e]), base + h * BT * 8 + tid * 8 + e);
          best = c > best ? c : best;
        }
#pragma unroll
      for (int d = 1; d < 8; d <<= 1) {
        const uint64_t c = __shfl_xor((unsigned long long)best, d, 64);
        best = c > best ? c : best;
      }
      if ((lane & 7) == 0) group_best[tid >> 3] = best;
      __syncthreads();
      if (wave == 0) {
        const uint64_t mine = group_best[lane];
        int rank = 0;
        for (int j = 0; j < 64; ++j) rank += group_best[j] > mine || (group_best[j] == mine && j < lane) ? 1 : 0;
        if (rank == W - 1 && mine > least) least = mine;
      }
      __syncthreads();
    }
    auto offer = [&]() {
      const uint64_t t = least;
      const float tv = of_ordered((uint32_t)(t >> 32));
#pragma unroll
      for (int h = 0; h < BE / 8; ++h) {
        if (!(m8[h] >= tv)) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint64_t c = candidate(ordered(v[8 * h + e]), base + h * BT * 8 + tid * 8 + e);
          if (c >= t) {
            const int at = atomicAdd(&held, 1);
            if (at < CAP) list[at] = c;
          }
        }
      }
    };
    offer();
    __syncthreads();
    int n = held;
    while (n > CAP) {  // more than fit: the bound of those that do, then this tile's again
      uint64_t mine[CAP / BT];
      keep_best(list, CAP, W, &least);
#pragma unroll
      for (int e = 0; e < CAP / BT; ++e) {
        const int at = tid + e * BT;
        mine[e] = at < W ? list[at] : 0;
        if (at < W && id_of(mine[e]) >= base) list[at] = 0;
      }
      if (tid == 0) held = W;
      __syncthreads();
      offer();
      __syncthreads();
      n = held;
    }
    if (n > TRIM) {
      n = keep_best(list, n, W, &least);
      if (tid == 0) held = n;
    }
    __syncthreads();
  }
  const int n = keep_best(list, held, W, &least);
  uint64_t* out = a.best + (row * a.parts + part) * W;
  for (int i = tid; i < W; i += BT) out[i] = i < n ? list[i] : 0;

  // the range's sum, relative to the largest thread's reference
  double at = k == 1.f ? (double)ref : -(double)o * 0.6931471805599453, top = at;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = fmax(top, __shfl_xor(top, d, 64));
  if (lane == 0) tops[wave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < BT / 64; ++w) top = fmax(top, tops[w]);
  double sum = (double)s * (k == 1.f ? 1.0 : 1.0 - LOG2E_OFF * ref) * exp(at - top);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 64);
  if (lane == 0) sums[wave] = sum;
  __syncthreads();
  if (tid == 0) {
    sum = 0;
    for (int w = 0; w < BT / 64; ++w) sum += sums[w];
    a.stats[2 * (row * a.parts + part)] = top;
    a.stats[2 * (row * a.parts + part) + 1] = sum;
  }
}

namespace {

struct Scored {
  double score;
  uint64_t which;
  int row;
};
__device__ __forceinline__ bool before(double s, int row, uint64_t which, double t, int row2, uint64_t which2) {
  return s > t || (s == t && (row < row2 || (row == row2 && which > which2)));
}

}  // namespace

constexpr int MT = 512;

__global__ __launch_bounds__(MT) void k_beam_merge(BeamArgs a) {
  extern __shared__ char mem[];
  const int tid = threadIdx.x, K = a.K, P = a.parts, W = a.W, lists = K * P;
  const int64_t row0 = (int64_t)blockIdx.x * K;
  double* base = reinterpret_cast<double*>(mem);               // [K] score minus the log of the row's sum; NaN: no candidate
  double* origin = base + K;                                   // [K] which is relative to this (logits of 1e38 keep the score's bits)
  double* score = origin + K;                                    // [W W] of the candidates that may be in
  uint64_t* which = reinterpret_cast<uint64_t*>(score + W * W);
  int* row = reinterpret_cast<int*>(which + W * W);
  double* head = reinterpret_cast<double*>(row + W * W + (W * W & 1));  // [lists]
  __shared__ int n_in;
  __shared__ Scored least;
  if (tid == 0) {
    n_in = 0;
    least = Scored{-INFINITY, 0, INT_MAX};
  }
  for (int k = tid; k < K; k += MT) {
    const double s = a.score[row0 + k];
    double b = __builtin_nan(""), top = 0;
    if (s > -INFINITY) {
      if (a.done && a.done[row0 + k]) {
        b = s;
      } else {
        const double* st = a.stats + 2 * (row0 + k) * P;
        double sum = 0;
        top = st[0];
        for (int p = 1; p < P; ++p) top = fmax(top, st[2 * p]);
        for (int p = 0; p < P; ++p) sum += st[2 * p + 1] * exp(st[2 * p] - top);
        if (sum > 0 && sum < INFINITY) b = s - log(sum);
      }
    }
    base[k] = b;
    origin[k] = top;
  }
  __syncthreads();
  auto is_done = [&](int k) { return a.done && a.done[row0 + k]; };
  // candidate i of list l (a beam's range), in the list's falling order
  auto get = [&](int l, int i, double& s, uint64_t& w) {
    const int k = l / P;
    if (!(base[k] == base[k]) || !(base[k] < INFINITY)) return false;
    if (is_done(k)) {
      s = base[k];
      w = 1;
      return l % P == 0 && i == 0;
    }
    w = a.best[((row0 + k) * P + l % P) * W + i];
    s = base[k] + ((double)of_ordered((uint32_t)(w >> 32)) - origin[k]);
    return w != 0;
  };
  // the W'th largest head of the lists: a candidate before that many others at least
  if (lists > W) {
    for (int l = tid; l < lists; l += MT) {
      double s;
      uint64_t w;
      head[l] = get(l, 0, s, w) ? s : -INFINITY;
    }
    __syncthreads();
    for (int l = tid; l < lists; l += MT) {
      double s;
      uint64_t w;
      if (!get(l, 0, s, w)) continue;
      int rank = 0;
      for (int j = 0; j < lists; ++j) {
        if (head[j] > s) ++rank;
        else if (head[j] == s && j != l) {
          double t;
          uint64_t u;
          if (get(j, 0, t, u) && before(t, j / P, u, s, l / P, w)) ++rank;
        }
      }
      if (rank == W - 1) least = Scored{s, w, l / P};
    }
  }
  __syncthreads();
  const Scored lim = least;
  for (int c = tid; c < lists * W; c += MT) {
    const int l = c / W;
    double s;
    uint64_t w;
    if (!get(l, c % W, s, w) || !(s > -INFINITY)) continue;
    if (lim.row != INT_MAX && before(lim.score, lim.row, lim.which, s, l / P, w)) continue;
    const int at = atomicAdd(&n_in, 1);
    if (at < W * W) {
      score[at] = s;
      which[at] = w;
      row[at] = l / P;
    }
  }
  __syncthreads();
  const int n = min(n_in, W * W);
  const int64_t out = (int64_t)blockIdx.x * W;
  for (int c = tid; c < n; c += MT) {
    const double s = score[c];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += before(score[j], row[j], which[j], s, row[c], which[c]) ? 1 : 0;
    if (rank < W) {
      a.token[out + rank] = is_done(row[c]) ? a.done_token : id_of(which[c]);
      a.parent[out + rank] = (int)(row0 + row[c]);
      a.next[out + rank] = (float)s;
    }
  }
  for (int c = n + tid; c < W; c += MT) {
    a.token[out + c] = -1;
    a.parent[out + c] = -1;
    a.next[out + c] = -INFINITY;
  }
}

// Ranges of a row: enough workgroups for the chip, ranges of a tile at the least.
BeamPlan beam_plan(int B, int K, int V, int W, int num_cus) {
  const int64_t rows = (int64_t)B * K;
  int64_t parts = std::max<int64_t>(1, std::min<int64_t>(4 * num_cus / std::max<int64_t>(rows, 1), (V + TILE - 1) / TILE));
  BeamPlan p;
  p.chunk = (int)(((V + parts - 1) / parts + 7) / 8 * 8);
  p.parts = (V + p.chunk - 1) / p.chunk;
  p.bytes = (size_t)rows * p.parts * (16 + 8 * (size_t)W);
  return p;
}

hipError_t launch_vocab_beam(BeamArgs a, const BeamPlan& p, void* ws, hipStream_t s) {
  a.parts = p.parts;
  a.chunk = p.chunk;
  a.stats = static_cast<double*>(ws);
  a.best = reinterpret_cast<uint64_t*>(a.stats + 2 * (size_t)a.B * a.K * a.parts);
  hipLaunchKernelGGL(k_beam_rows, dim3((unsigned)((int64_t)a.B * a.K * a.parts)), dim3(BT), 0, s, a);
  if (hipError_t e = hipGetLastError()) return e;
  const size_t lds = 16 * (size_t)a.K + 20 * (size_t)a.W * a.W + 8 + 8 * (size_t)a.K * a.parts;
  hipLaunchKernelGGL(k_beam_merge, dim3((unsigned)a.B), dim3(MT), lds, s, a);
  return hipGetLastError();
}

}  // namespace cora
