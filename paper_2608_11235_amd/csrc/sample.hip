// A token per logits row by temperature, top-k, top-p and min-p, from a given random number.
//
// Over the allowed ids of a row (not the mask id, not NaN, not -inf), ordered by logit downwards
// and by id upwards among equal ones, with w_j = exp((l_j - l_0) / T):
//   n1 = top_k > 0 ? min(top_k, n) : n,   n2 = least m with sum_{j<m} w_j >= top_p sum_{j<n1} w_j,
//   n3 = #{w_j >= min_p},   N = min(n1, n2, n3) >= 1,
//   token = id of the least m with sum_{j<=m} w_j > u sum_{j<N} w_j,
//   conf = exp(l_token - l_0) / sum_j exp(l_j - l_0), Eq. (1)'s softmax at temperature 1.
//
// A token is decided where a running sum of up to 152064 terms passes a number, so sums in 32
// bits would pick another token of every few hundred rows.  bf16 logits take few distinct
// values (about 3500 in a row of 126464 drawn from N(0, 1)), and the order is by value: the row
// is counted into a histogram with one bin per value (integers: exact in any order), and every
// sum runs over bins in 64 bits.  No exponential is taken per logit at all.
//
// One workgroup per row:
//   1 count: one pass over the row, an LDS add per logit;
//   2 sum:   count, sum of w and sum of exp of each entry of 256 bins;
//   3 pick:  the borders n1, n2, n3 and the token's bin and rank in it, by wavefront 0: a scan of
//            the entries, then of the 256 bins of the one that holds the border;
//   4 find:  the rank-th id that holds the value, in a second reading of the row, from the end
//            that is nearer by rank, up to that id.
// The bins of step 1 are the bf16 numbers of magnitude 2^-44 to 2^19 of either sign and zero, in
// 16-bit counts, a number and its negative to a word: 32 KB, so that three workgroups share a CU and
// one counts while another scans.  A row with any other finite number (a maximum beyond 2^19, a
// logit below 2^-44), +inf, NaN or more than 65535 equal logits is done by the same steps over all
// 65536 bf16 numbers in eight windows of 32-bit counts, at one reading of the row each; finite
// numbers far below the maximum (a ban by bf16's lowest one), whose terms are 0 in 64 bits, do not
// count.
//
// 4096 rows of 126464 take 226 us, 4.6 TB/s.  Three things of like size share that time: the rows'
// bytes (150 us at the 6.9 TB/s of a plain reading, and 22 % more for step 4), the LDS adds (117 us: 3.7 ns a wavefront's 64
// on a CU when they fall on some 500 words, 1.8 without bank conflicts) and about 7 instructions a
// logit (95 us).  Steps 2 to 4 are 13 of a row's 32 us, beside two other rows' counting.  A single
// row is bound by latency: 2048 logits 8 us in the kernel, 126464 17 us, 9 of them counting.
#include <limits.h>

#include <algorithm>

#include "cached.hpp"

namespace cora {

namespace {

constexpr int ENT = 256;             // bins per entry
constexpr int BEFORE = -1, BEHIND = -2;  // instead of a chunk: a logit outside the whole ones
constexpr uint32_t LO = 83u << 7, SPAN = 63u << 7;         // magnitudes 2^-44 <= |l| < 2^19
constexpr uint32_t FAR_BELOW = 1, OTHER = 2;               // finite numbers <= -2^19; the rest without a bin

typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
typedef short s16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u16x2_t halves(uint32_t w) { return __builtin_bit_cast(u16x2_t, w); }
__device__ __forceinline__ s16x2_t signed_halves(uint32_t w) { return __builtin_bit_cast(s16x2_t, w); }
__device__ __forceinline__ uint32_t word(u16x2_t h) { return __builtin_bit_cast(uint32_t, h); }

// A scheme of bins, numbered in the order of falling value; a window of BINS of them is in LDS.
// Narrow, one window: place 1 + magnitude - LO, 0 for zero, so that a place is a subtraction away.
// PAIRED: positive numbers in the low half of the place's word, negative ones in the high half;
// else negative numbers HALF words further.
template <bool PAIRED>
struct Narrow {
  static constexpr int HALF = 8192, WORDS = PAIRED ? HALF : 2 * HALF;
  static constexpr int WINDOWS = 1, BINS = 2 * HALF, LAST = BINS - 1, ENTRIES = BINS / ENT;
  static __device__ __forceinline__ int place(uint32_t b) {  // -1: none
    const uint32_t mag = b & 0x7fff, t = mag - LO;
    return t < SPAN ? 1 + (int)t : (mag == 0 ? 0 : -1);
  }
  // words from a number's place to the one that counts it, and n as it counts there; zero is counted
  // as a positive number
  static __device__ __forceinline__ int further(uint32_t b) { return !PAIRED && b > 0x8000u ? HALF : 0; }
  static __device__ __forceinline__ uint32_t count(uint32_t b, uint32_t n) { return PAIRED && b > 0x8000u ? n << 16 : n; }
  static __device__ __forceinline__ int bin(uint32_t b, int place) {
    return b > 0x8000u ? HALF + place : HALF - 1 - place;
  }
  static __device__ __forceinline__ uint32_t bits(int i) {
    const uint32_t s = (uint32_t)(i < HALF ? HALF - 1 - i : i - HALF);
    return (i < HALF ? 0u : 0x8000u) | (s == 0 ? 0u : LO + s - 1);
  }
  // The step to the next smaller number below bin i is that of octave(i): 1 + the exponent's offset
  // for a step inside it, 0 for the one between zero and 2^-44.
  static __device__ __forceinline__ int octave(int i) {
    return i < HALF ? ((HALF - 2 - i) + 127) >> 7 : ((i - HALF) + 127) >> 7;
  }
  // the counts of bins i .. i + 3, i a multiple of 4
  static __device__ __forceinline__ u32x4_t four(const uint32_t* hist, int i) {
    if (i >= HALF) {
      const u32x4_t c = *reinterpret_cast<const u32x4_t*>(hist + (PAIRED ? i - HALF : i));
      return PAIRED ? c >> 16 : c;
    }
    const u32x4_t c = *reinterpret_cast<const u32x4_t*>(hist + HALF - 4 - i);
    const u32x4_t r = {c[3], c[2], c[1], c[0]};
    return PAIRED ? r & 0xffffu : r;
  }
};
// Wide, all bf16 numbers, a word each.
template <int WORDS_>
struct Wide {
  static constexpr int WORDS = WORDS_, BINS = WORDS, WINDOWS = 65536 / BINS, ENTRIES = BINS / ENT;
  static constexpr int LAST = 0xff7f;  // the bin of the lowest finite number
  static __device__ __forceinline__ int bin(uint32_t b) {
    const uint32_t mag = b & 0x7fff;
    if (mag > 0x7f80 || b == 0xff80) return -1;  // NaN, -inf
    return (b & 0x8000) && mag ? 0x8000 + (int)mag : 0x7fff - (int)mag;
  }
  static __device__ __forceinline__ uint32_t bits(int i) {
    return i < 0x8000 ? 0x7fffu - (uint32_t)i : 0x8000u | (uint32_t)(i - 0x8000);
  }
  static __device__ __forceinline__ u32x4_t four(const uint32_t* hist, int i) {
    return *reinterpret_cast<const u32x4_t*>(hist + (i & (BINS - 1)));
  }
};

template <int WORDS>
struct Shared {
  uint32_t hist[WORDS];
  uint32_t cnt[256];
  double wt[256], w1[256];            // of each entry: sum of w, sum of exp
  double step[2][64];                 // Narrow: exp of minus an octave's step, over T and over 1
  double root[64];                    // 2^(i / 64)
  uint32_t tot[2][64];
  uint32_t first[16], special;        // least bin in use of each wavefront; FAR_BELOW, OTHER numbers without a bin
  uint32_t uncounted;                 // logits without a bin
  int top[16];                        // of each wavefront
  int window;                         // that the histogram holds
  // the pick: value, its ids, the token's rank among them
  uint32_t value, count, rank;
  float conf;
  int id;
  uint32_t first_id;
};

__device__ __forceinline__ uint32_t lane_value(uint32_t v, int l) { return (uint32_t)__builtin_amdgcn_readlane((int)v, l); }
__device__ __forceinline__ double lane_value(double v, int l) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  return __builtin_bit_cast(double, (uint64_t)lane_value((uint32_t)(b >> 32), l) << 32 | lane_value((uint32_t)b, l));
}

// exp(x), x <= 0, to about 2^-52 of it: x = n ln 2 / 64 + r, |r| <= ln 2 / 128, exp(x) = 2^(n / 64) exp(r)
// with the series of exp(r) up to r^5 (the next term is below 2^-54).  12 operations in 64 bits
// where the library's, good for any x, takes twice as many.
template <class Sh>
__device__ __forceinline__ double exp_down(const Sh& sh, double x) {
  x = fmax(x, -800.0);  // 0 from -746 on
  const double n = rint(x * 92.332482616893656877);
  double r = fma(n, -0x1.62e42fefa0000p-7, x);  // ln 2 / 64 in two parts, the first of 36 bits
  r = fma(n, -0x1.cf79abc9e3b3ap-46, r);
  double p = fma(r, 1.0 / 120.0, 1.0 / 24.0);
  p = fma(p, r, 1.0 / 6.0);
  p = fma(p, r, 0.5);
  p = fma(p * r, r, r);
  const int k = (int)n;
  const double e = sh.root[k & 63];
  return ldexp(fma(e, p, e), k >> 6);
}

// Calls f(logit bits, id) for every logit of the row.
template <int NT, class F>
__device__ __forceinline__ void each_logit(const uint16_t* x, int V, F&& f) {
  const int tid = threadIdx.x;
  const int v0 = min((int)((0 - (uintptr_t)x) & 15) / 2, V);
  const int nch = (V - v0) >> 3, v1 = v0 + nch * 8;
  const u32x4_t* xv = reinterpret_cast<const u32x4_t*>(x + v0);
  for (int c = tid; c < nch; c += NT) {
    const u32x4_t w = xv[c];
#pragma unroll
    for (int j = 0; j < 8; ++j) f((j & 1) ? w[j >> 1] >> 16 : w[j >> 1] & 0xffffu, v0 + c * 8 + j);
  }
  if (tid < v0) f(x[tid], tid);
  if (tid < V - v1) f(x[v1 + tid], v1 + tid);
}

// Step 1, Narrow.  Eight logits a load, four loads ahead; their words by 16-bit pairs, one test for
// all eight.  The mask id is counted like the others: its bin starts one below zero.  Returns
// FAR_BELOW / OTHER; `uncounted` logits had no bin; `top` is the largest of this thread's logits' bits
// as signed numbers (the maximum where that is not below zero), first seen in its chunk `top_at`.
template <int NT, bool PAIRED, class Sh>
__device__ __forceinline__ uint32_t count_row(Sh& sh, const uint16_t* x, int V, int mask_id, double inv_t,
                                              uint32_t& uncounted, int& top, int& top_at) {
  using Bins = Narrow<PAIRED>;
  const int tid = threadIdx.x;
  uint32_t special = 0;
  uncounted = 0;
  top = -32768;
  top_at = 0;
  auto one = [&](uint32_t b) {
    const int w = Bins::place(b);
    if (w >= 0) {
      atomicAdd(&sh.hist[w + Bins::further(b)], Bins::count(b, 1));
    } else {
      ++uncounted;
      if (b != 0xff80u) special |= b > 0x8000u + LO && b < 0xff80u ? FAR_BELOW : OTHER;
    }
  };
  const int v0 = min((int)((0 - (uintptr_t)x) & 15) / 2, V);
  const int nch = (V - v0) >> 3, v1 = v0 + nch * 8;
  const u32x4_t* xv = reinterpret_cast<const u32x4_t*>(x + v0) + tid;
  const int mine = (nch - tid + NT - 1) / NT;  // this thread's chunks: xv[i NT], i < mine
  u32x4_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < mine) w[i] = xv[i * NT];
  // meanwhile the histogram is cleared and the tables of factors are made
  if (tid < 192) {
    const int o = tid & 63;
    const double d = o ? ldexp(1.0, 83 + o - 1 - 127 - 7) : 0x1p-44;
    const double y = exp(tid < 64 ? -d * inv_t : (tid < 128 ? -d : o * (0.6931471805599453094 / 64)));
    if (tid < 128) sh.step[tid >> 6][o] = y;
    else sh.root[o] = y;
  }
  u32x4_t* h = reinterpret_cast<u32x4_t*>(sh.hist);
#pragma unroll
  for (int i = 0; i < Bins::WORDS / 4 / NT; ++i) h[tid + i * NT] = u32x4_t{0, 0, 0, 0};
  if (mask_id >= 0) {
    const uint32_t b = x[mask_id];
    const int w = Bins::place(b), at = w < 0 ? -1 : w + Bins::further(b);
    if (at >= 0 && (at >> 2) % NT == tid) sh.hist[at] = Bins::count(b, ~0u);
    if (tid == 0 && w >= 0) uncounted = 1;
  }
  __syncthreads();
  auto eight = [&](const u32x4_t& q, int i) {
    s16x2_t high = signed_halves(q[0]);
#pragma unroll
    for (int j = 1; j < 4; ++j) high = __builtin_elementwise_max(high, signed_halves(q[j]));
    const int m = max((int)high[0], (int)high[1]);
    if (m > top) {
      top = m;
      top_at = i;
    }
    uint32_t t[4];  // places less one, by pairs
    u16x2_t most = {0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      t[j] = word(halves(q[j]) - (unsigned short)LO) & 0x7fff7fffu;
      most = __builtin_elementwise_max(most, halves(t[j]));
    }
    if (most[0] < SPAN && most[1] < SPAN) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t at = word(halves(t[j]) << (unsigned short)2);  // byte address of the word before the place's
        if (!PAIRED) at |= q[j] & 0x80008000u;
        auto add = [&](uint32_t o, uint32_t neg) {
          atomicAdd(reinterpret_cast<uint32_t*>(reinterpret_cast<char*>(sh.hist) + o) + 1,
                    PAIRED ? __umul24(neg, 0xffffu) + 1u : 1u);
        };
        add(at & 0xffffu, (q[j] >> 15) & 1);
        add(at >> 16, q[j] >> 31);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        one(q[j] & 0xffffu);
        one(q[j] >> 16);
      }
    }
  };
  // the up to seven logits before the first whole chunk are a thread's each, and so are those behind
  // the last one
  auto edge = [&](int id, int at) {
    one(x[id]);
    if ((int)(short)x[id] > top) {
      top = (int)(short)x[id];
      top_at = at;
    }
  };
  if (tid < v0) edge(tid, BEFORE);
  int i = 0;
  for (; i + 8 <= mine; i += 4) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      eight(w[k], i + k);
      w[k] = xv[(i + 4 + k) * NT];
    }
  }
  for (; i < mine; i += 4) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k < mine) {
        eight(w[k], i + k);
        if (i + 4 + k < mine) w[k] = xv[(i + 4 + k) * NT];
      }
  }
  if (tid < V - v1) edge(v1 + tid, BEHIND);
  return special;
}

// what the terms of a row are measured against
struct Terms {
  float max;
  double inv_t;  // 1 / T, -1 for a greedy row
  int first;     // the maximum's bin
  // l - max of a bin's number; 0 for the maximum also where that is +inf
  template <class Scheme>
  __device__ __forceinline__ double below(int bin) const {
    const float v = bf16_bits_to_f32(Scheme::bits(bin));
    return v == max ? 0.0 : (double)v - (double)max;
  }
  __device__ __forceinline__ double weight(double d) const {
    return d == 0.0 ? 1.0 : (d == -INFINITY ? 0.0 : exp(d * inv_t));
  }
  // w over T (OVER_T) or over 1 of bins i .. i + 3, i a multiple of 4; at least 0 and finite for bins
  // above the maximum too.  Narrow: neighbouring numbers of an octave are a step apart, so one
  // exponential and three products (four exponentials each took step 2 from 3.1 to 4.5 us).
  template <class Scheme, bool OVER_T, class Sh>
  __device__ __forceinline__ void weights(const Sh& sh, int i, double (&w)[4]) const {
    if constexpr (Scheme::WINDOWS == 1) {
      const double d = below<Scheme>(i), k = OVER_T ? inv_t : 1.0;
      w[0] = i <= first ? 1.0 : exp_down(sh, d * k);
#pragma unroll
      for (int j = 1; j < 4; ++j)
        w[j] = i + j <= first ? 1.0 : w[j - 1] * sh.step[OVER_T ? 0 : 1][min(Scheme::octave(i + j - 1), 63)];
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const double d = below<Scheme>(i + j);
        w[j] = i + j <= first ? 1.0 : (OVER_T ? weight(d) : exp(d));
      }
    }
  }
};

// A place in the order of falling logits: `before` terms of sum `mass` come before the bin, whose
// terms weigh `w` each and are `count` in number.
struct Place {
  int bin;
  uint32_t before, count;
  double mass, w;
};

// The histogram of one row and the searches in it.  Narrow: one wavefront may search.  Wide: the
// whole workgroup does, since a search may have to count another window.
template <class Scheme, int NT, class Sh>
struct Row {
  Sh& sh;
  const uint16_t* x;
  int V, mask_id;
  Terms t;
  static constexpr int NW = NT / 64, NENT = Scheme::ENTRIES, BINS = Scheme::BINS;
  static constexpr int EPL = Scheme::WINDOWS * NENT / 64;  // entries of a lane
  uint32_t n, ni;  // terms in this lane's entries, in those and all before
  double s, si;    // their sums of w

  __device__ __forceinline__ void count_window(int win) {
    if constexpr (Scheme::WINDOWS > 1) {
    __syncthreads();  // everyone is done with the window before
    u32x4_t* h = reinterpret_cast<u32x4_t*>(sh.hist);
    for (int i = threadIdx.x; i < Scheme::WORDS / 4; i += NT) h[i] = u32x4_t{0, 0, 0, 0};
    __syncthreads();
    each_logit<NT>(x, V, [&](uint32_t b, int id) {
      const int i = Scheme::bin(b) - win * BINS;
      if (id != mask_id && (uint32_t)i < (uint32_t)BINS) atomicAdd(&sh.hist[i], 1u);
    });
    if (threadIdx.x == 0) sh.window = win;
    __syncthreads();
    }
  }

  // Step 2 on the window that the histogram holds: the entries in use, dealt to the wavefronts.
  // Their counts are there already.
  __device__ void sum_window(int win) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    unsigned long long used = __ballot(lane < NENT && sh.cnt[win * NENT + lane] != 0);
    if (wave == 0 && lane < NENT && !((used >> lane) & 1)) sh.wt[win * NENT + lane] = sh.w1[win * NENT + lane] = 0.0;
    for (int k = 0; used; ++k) {
      const int e = __ffsll(used) - 1;
      used &= used - 1;
      if (k % NW != wave) continue;
      const int i0 = win * BINS + e * ENT + lane * 4;
      const u32x4_t c = Scheme::four(sh.hist, i0);
      double w[4], st = 0.0, s1 = 0.0;
      t.template weights<Scheme, false>(sh, i0, w);
#pragma unroll
      for (int j = 0; j < 4; ++j) s1 += c[j] ? c[j] * w[j] : 0.0;
      st = s1;
      if (t.inv_t != 1.0 && t.inv_t >= 0.0) {
        st = 0.0;
        t.template weights<Scheme, true>(sh, i0, w);
#pragma unroll
        for (int j = 0; j < 4; ++j) st += c[j] ? c[j] * w[j] : 0.0;
      }
      st = lane_value(wave_scan(st), 63);
      s1 = lane_value(wave_scan(s1), 63);
      if (lane == 0) {
        sh.wt[win * NENT + e] = st;
        sh.w1[win * NENT + e] = s1;
      }
    }
  }

  // Step 2, Narrow: 16 lanes to an entry, 16 bins a lane in a row: an exponential, and from bin to
  // bin a product with the octave's factor.  The first or the last of the 15 steps may be another
  // octave's.  A wavefront's four entries are neighbours, so that the few in use keep few wavefronts
  // busy: 1.7 us against 2.8 with entries dealt out one by one, alone in a CU.
  __device__ __forceinline__ void sum_all() {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), sub = lane & 15;
#pragma unroll 1
    for (int k = 0; k < NENT / NW / 4; ++k) {
      const int e = 4 * (wave + NW * k) + (lane >> 4), i0 = e * ENT + sub * 16;
      u32x4_t c[4];
      uint32_t cn = 0;
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        c[v] = Scheme::four(sh.hist, i0 + 4 * v);
        cn += c[v][0] + c[v][1] + c[v][2] + c[v][3];
      }
      double st = 0.0, s1 = 0.0;
      if (__any(cn != 0)) {
        const double d = t.template below<Scheme>(i0);
        const int a = min(Scheme::octave(i0), 63), b = min(Scheme::octave(i0 + 1), 63), z = min(Scheme::octave(i0 + 14), 63);
        auto total = [&](double k1, const double* step) {
          const double qa = step[a], qb = step[b], qz = step[z];
          double w = i0 <= t.first ? 1.0 : exp_down(sh, d * k1), sum = c[0][0] ? w * c[0][0] : 0.0;
#pragma unroll
          for (int j = 1; j < 16; ++j) {
            w = i0 + j <= t.first ? 1.0 : w * (j == 1 ? qa : (j == 15 ? qz : qb));
            sum += w * c[j >> 2][j & 3];
          }
          return sum;
        };
        s1 = total(1.0, sh.step[1]);
        st = t.inv_t == 1.0 || t.inv_t < 0.0 ? s1 : total(t.inv_t, sh.step[0]);
      }
      // over the entry's lanes: the last one holds the sums
      cn += moved<0x111, 0xf>(cn); s1 += moved<0x111, 0xf>(s1); st += moved<0x111, 0xf>(st);
      cn += moved<0x112, 0xf>(cn); s1 += moved<0x112, 0xf>(s1); st += moved<0x112, 0xf>(st);
      cn += moved<0x114, 0xf>(cn); s1 += moved<0x114, 0xf>(s1); st += moved<0x114, 0xf>(st);
      cn += moved<0x118, 0xf>(cn); s1 += moved<0x118, 0xf>(s1); st += moved<0x118, 0xf>(st);
      if (sub == 15) {
        sh.cnt[e] = cn;
        sh.wt[e] = st;
        sh.w1[e] = s1;
      }
    }
  }

  // this lane's entries, after step 2; returns the row's sum of exp
  __device__ double gather() {
    const int lane = threadIdx.x & 63;
    double s1 = 0.0;
    n = 0;
    s = 0.0;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      n += sh.cnt[lane * EPL + i];
      s += sh.wt[lane * EPL + i];
      s1 += sh.w1[lane * EPL + i];
    }
    ni = wave_scan(n);
    si = wave_scan(s);
    return lane_value(wave_scan(s1), 63);
  }

  // the first lane of a border, or, where rounding left the last sum short of it, the last lane in use
  static __device__ __forceinline__ int border(bool hit, bool in_use) {
    const unsigned long long h = __ballot(hit), u = __ballot(in_use);
    return h ? __ffsll(h) - 1 : (u ? 63 - __clzll((long long)u) : 0);
  }

  __device__ __forceinline__ void hold(int e) {
    if constexpr (Scheme::WINDOWS > 1)
      if (sh.window != e / NENT) count_window(e / NENT);
  }

  // this lane's four bins of entry e: their counts, w of those in use, the sums
  __device__ __forceinline__ u32x4_t four(int e, double (&w)[4], uint32_t& cn, double& cs) const {
    const int i0 = e * ENT + (threadIdx.x & 63) * 4;
    const u32x4_t c = Scheme::four(sh.hist, i0);
    t.template weights<Scheme, true>(sh, i0, w);
    cn = 0;
    cs = 0.0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (!c[j]) w[j] = 0.0;
      cn += c[j];
      cs += c[j] * w[j];
    }
    return c;
  }

  // The bin that holds term k of the row's order (BY_COUNT), or in which the running sum of w passes
  // m (strict) or reaches it.
  template <bool BY_COUNT>
  __device__ Place find(uint32_t k, double m, bool strict) {
    auto past = [&](uint32_t terms, double sum) { return BY_COUNT ? terms > k : (strict ? sum > m : sum >= m); };
    // the entry, with what comes before it
    int l = border(n > 0 && past(ni, si), n > 0);
    uint32_t before = l > 0 ? lane_value(ni, l - 1) : 0;
    double mass = l > 0 ? lane_value(si, l - 1) : 0.0;
    int e = l * EPL;
    if constexpr (EPL > 1) {
      int last = e;  // of the lane's entries in use
#pragma unroll
      for (int i = 1; i < EPL; ++i)
        if (sh.cnt[l * EPL + i]) last = l * EPL + i;
      for (; e < last; ++e) {
        const uint32_t c = sh.cnt[e];
        const double w = sh.wt[e];
        if (c && past(before + c, mass + w)) break;
        before += c;
        mass += w;
      }
    }
    hold(e);
    // its bins
    uint32_t cn;
    double cs, w[4];
    const u32x4_t c = four(e, w, cn, cs);
    const uint32_t bi = wave_scan(cn) + before;
    const double mi = wave_scan(cs) + mass;
    l = border(cn > 0 && past(bi, mi), cn > 0);
    Place p{0, bi - cn, 0, mi - cs, 0.0};
    bool found = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (!c[j] || found) continue;
      if (p.count) {  // the bin before is not the one
        p.before += p.count;
        p.mass += p.count * p.w;
      }
      p.bin = e * ENT + (int)(threadIdx.x & 63) * 4 + j;
      p.count = c[j];
      p.w = w[j];
      found = past(p.before + c[j], p.mass + c[j] * w[j]);
    }
    return Place{(int)lane_value((uint32_t)p.bin, l), lane_value(p.before, l), lane_value(p.count, l),
                 lane_value(p.mass, l), lane_value(p.w, l)};
  }

  // terms in bins up to `bin` and their sum
  __device__ uint32_t up_to(int bin, double& mass) {
    const int lane = threadIdx.x & 63, e = bin / ENT;
    uint32_t cn = 0;
    double cs = 0.0;
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (lane * EPL + i < e) {
        cn += sh.cnt[lane * EPL + i];
        cs += sh.wt[lane * EPL + i];
      }
    hold(e);
    uint32_t en;
    double es, w[4];
    const u32x4_t c = four(e, w, en, es);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (e * ENT + lane * 4 + j <= bin) {
        cn += c[j];
        cs += c[j] * w[j];
      }
    mass = lane_value(wave_scan(cs), 63);
    return lane_value(wave_scan(cn), 63);
  }
};

// A row's settings.
struct Settings {
  float T;
  int top_k;
  float top_p, min_p, u;
};

// Step 3: the bin of the token and its rank among that bin's ids.
template <class Scheme, int NT, class Sh>
__device__ __forceinline__ void pick(Row<Scheme, NT, Sh>& row, int first, const Settings& g, Place& p, uint32_t& rank) {
  rank = 0;
  if (!(g.T > 0.f)) {
    p = row.template find<true>(0, 0.0, false);
    return;
  }
  uint32_t N = lane_value(row.ni, 63);
  double mass = lane_value(row.si, 63);  // of the first N terms
  if (g.top_k > 0 && (uint32_t)g.top_k < N) {
    N = (uint32_t)g.top_k;
    p = row.template find<true>(N - 1, 0.0, false);
    mass = p.mass + (N - p.before) * p.w;
  }
  if (g.top_p < 1.f) {
    const double m = (double)g.top_p * mass;
    p = row.template find<false>(0, m, false);
    const double r = p.w > 0.0 ? ceil((m - p.mass) / p.w) : 1.0;
    const uint32_t in = r < 1.0 ? 1u : (r > (double)p.count ? p.count : (uint32_t)r);
    if (p.before + in < N) {
      N = p.before + in;
      mass = p.mass + in * p.w;
    }
  }
  if (g.min_p > 0.f) {
    // the last bin of w >= min_p (w falls from bin to bin), by halving; `first` where none is
    int lo = first, hi = Scheme::LAST;
    while (lo < hi) {
      const int c = (lo + hi + 1) >> 1;
      const bool in = row.t.weight(row.t.template below<Scheme>(c)) >= (double)g.min_p;
      lo = in ? c : lo;
      hi = in ? hi : c - 1;
    }
    uint32_t n3 = 1;
    double m3 = 1.0;
    if (g.min_p <= 1.f) n3 = row.up_to(lo, m3);
    if (n3 < N) {
      N = n3;
      mass = m3;
    }
  }
  const double m = (double)g.u * mass;
  p = row.template find<false>(0, m, true);
  const double r = p.w > 0.0 ? floor((m - p.mass) / p.w) : 0.0;
  rank = r < 0.0 ? 0u : (r >= (double)p.count ? p.count - 1 : (uint32_t)r);
  if (p.before + rank >= N) {  // rounding: never past the last kept term
    p = row.template find<true>(N - 1, 0.0, false);
    rank = N - 1 - p.before;
  }
}

// Step 4: the rank-th id that holds the value, in blocks of CH NT chunks of eight ids, from the front
// or from the back.
template <int NT, class Sh>
__device__ __forceinline__ void find_id(Sh& sh, const uint16_t* x, int V, int mask_id) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  constexpr int NW = NT / 64, CH = 2;  // chunks a thread and block (4: the tiny vocabulary's rows 0.5 us more, 32 rows of 126464 0.4 less)
  const uint32_t want = __builtin_amdgcn_readfirstlane(sh.value), even = want | want << 16;
  const uint32_t care = want == 0 ? 0x7fffu : 0xffffu;
  const bool back = sh.rank >= sh.count - sh.rank;  // fewer of its ids behind than before
  const uint32_t left = back ? sh.count - 1 - sh.rank : sh.rank;
  const int shift = (int)((uintptr_t)x & 15) / 2;  // chunk c holds ids 8 c - shift ..
  const u32x4_t* xv = reinterpret_cast<const u32x4_t*>(x - shift);
  const int nch = (V + shift + 7) >> 3, blocks = (nch + CH * NT - 1) / (CH * NT);
  auto whole = [&](int c) { return c * 8 >= shift && c * 8 - shift + 8 <= V; };
  auto first_chunk = [&](int i) { return (back ? blocks - 1 - i : i) * CH * NT + tid; };
  u32x4_t w[CH];
  auto load = [&](int i) {
#pragma unroll
    for (int k = 0; k < CH; ++k)
      if (whole(first_chunk(i) + k * NT)) w[k] = xv[first_chunk(i) + k * NT];
  };
  load(0);
  uint32_t seen = 0;
  for (int i = 0; i < blocks; ++i) {
    const int c0 = first_chunk(i);
    uint32_t hits[CH];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int c = c0 + k * NT, id = c * 8 - shift;
      hits[k] = 0;
      if (whole(c)) {
        u16x2_t least = {0xffff, 0xffff};
        u16x2_t d[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          d[j] = halves(w[k][j] ^ even);
          if (want == 0) d[j] = halves(word(d[j]) & 0x7fff7fffu);  // zeros of either sign are equal
          least = __builtin_elementwise_min(least, d[j]);
        }
        if (least[0] == 0 || least[1] == 0)
#pragma unroll
          for (int j = 0; j < 8; ++j) hits[k] |= (uint32_t)(d[j >> 1][j & 1] == 0) << j;
      } else if (id < V) {
        for (int j = 0; j < 8; ++j)
          if (id + j >= 0 && id + j < V) hits[k] |= (uint32_t)(((x[id + j] ^ want) & care) == 0) << j;
      }
      if ((uint32_t)(mask_id - id) < 8u) hits[k] &= ~(1u << (mask_id - id));
    }
    // ahead where the id is likely to be further on: blocks read for nothing, always, took 235 us for 4096
    // rows and not 228
    const bool ahead = i + 1 < blocks && (uint64_t)(left - seen) * blocks > sh.count;
    if (ahead) load(i + 1);
    uint32_t own[CH], inc[CH];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      own[k] = __popc(hits[k]);
      inc[k] = 0;
      if (__any(hits[k] != 0)) inc[k] = wave_scan(own[k]);
      if (lane == 63) sh.tot[i & 1][k * NW + wave] = inc[k];
    }
    __syncthreads();
    static_assert(CH * NW <= 64, "a total of each wavefront and chunk to a lane");
    const uint32_t all = wave_scan(lane < CH * NW ? sh.tot[i & 1][lane] : 0u), total = lane_value(all, 63);
    if (left < seen + total) {
      const uint32_t at = back ? total - 1 - (left - seen) : left - seen;
#pragma unroll
      for (int k = 0; k < CH; ++k) {
        const int o = k * NW + wave;
        const uint32_t before = (o > 0 ? lane_value(all, o - 1) : 0) + inc[k] - own[k];
        if (before <= at && at < before + own[k]) {
          uint32_t h = hits[k];
          for (uint32_t j = before; j < at; ++j) h &= h - 1;
          sh.id = (c0 + k * NT) * 8 - shift + __ffs(h) - 1;
        }
      }
      break;
    }
    seen += total;
    if (!ahead && i + 1 < blocks) load(i + 1);
  }
  __syncthreads();
}

// The counts of the window's entries and its least bin in use, dealt to the wavefronts.  A barrier
// follows.  sh.first holds each wavefront's least bin.
template <class Scheme, int NT, class Sh>
__device__ __forceinline__ void count_entries(Sh& sh, int win) {
  constexpr int NW = NT / 64, NENT = Scheme::ENTRIES, BINS = Scheme::BINS;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t least = INT_MAX;
#pragma unroll
  for (int k = 0; k < NENT / NW; ++k) {
    const int e = wave * (NENT / NW) + k, i0 = win * BINS + e * ENT + lane * 4;
    const u32x4_t c = Scheme::four(sh.hist, i0);
    const uint32_t cn = c[0] + c[1] + c[2] + c[3];
    const unsigned long long used = __ballot(cn != 0);
    if (used && least == INT_MAX) {
      const int in = c[0] ? 0 : (c[1] ? 1 : (c[2] ? 2 : 3));
      least = lane_value((uint32_t)(i0 + in), __ffsll(used) - 1);
    }
    const uint32_t total = used ? lane_value(wave_scan(cn), 63) : 0;
    if (lane == 0) sh.cnt[win * NENT + e] = total;
  }
  if (lane == 0) sh.first[wave] = least;
}

template <int NT, class Sh>
__device__ __forceinline__ uint32_t least_first(const Sh& sh) {
  uint32_t f = INT_MAX;
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) f = min(f, sh.first[i]);
  return f;
}

// Steps 3 and 4.  own_top: the row's maximum as its bits, where it is no less than zero and not the
// mask id's too; top, top_at: of this thread, as count_row gives them.
constexpr int NO_TOP = -1;
template <class Scheme, int NT, class Sh>
__device__ __forceinline__ void draw(Sh& sh, Row<Scheme, NT, Sh>& row, int first, const Settings& g, bool nan,
                                     int own_top = NO_TOP, int top = 0, int top_at = 0) {
  if (Scheme::WINDOWS > 1 || threadIdx.x < 64) {
    const double s1 = row.gather();
    Place p;
    uint32_t rank;
    pick<Scheme, NT>(row, first, g, p, rank);
    if (threadIdx.x == 0) {
      sh.value = Scheme::bits(p.bin);
      sh.count = p.count;
      sh.rank = rank;
      const double d = row.t.template below<Scheme>(p.bin);
      sh.conf = nan ? __builtin_nanf("") : (float)(exp_down(sh, d) / s1);
      sh.id = -1;
      sh.first_id = ~0u;
    }
  }
  __syncthreads();
  if (own_top != NO_TOP && sh.rank == 0 && sh.value == (uint32_t)own_top) {
    // the first id of the maximum, which the threads met while counting
    if (top == own_top) {
      const int tid = threadIdx.x, V = row.V;
      const int v0 = min((int)((0 - (uintptr_t)row.x) & 15) / 2, V), v1 = V - ((V - v0) & 7);
      int id = top_at == BEFORE ? tid : v1 + tid;
      if (top_at >= 0) {
        id = v0 + (top_at * NT + tid) * 8;
        while ((int)(short)row.x[id] != top) ++id;
      }
      atomicMin(&sh.first_id, (uint32_t)id);
    }
    __syncthreads();
    if (threadIdx.x == 0) sh.id = (int)sh.first_id;
    return;
  }
  find_id<NT>(sh, row.x, row.V, row.mask_id);
}

// A row with numbers beyond the narrow bins: maximum and NaNs of the allowed ids, then all bins.
template <int NT, int WORDS>
__device__ __forceinline__ void wide_row(Shared<WORDS>& sh, const uint16_t* x, int V, int mask_id, const Settings& g, double inv_t) {
  __syncthreads();
  if (threadIdx.x < NT / 64) sh.first[threadIdx.x] = INT_MAX;
  if (threadIdx.x == 0) { sh.special = 0; sh.window = -1; sh.id = -1; }
  __syncthreads();
  uint32_t first = INT_MAX;
  bool nan = false;
  each_logit<NT>(x, V, [&](uint32_t b, int id) {
    if (id == mask_id) return;
    const int i = Wide<WORDS>::bin(b);
    if (i >= 0) first = min(first, (uint32_t)i);
    else nan |= b != 0xff80u;
  });
  atomicMin(&sh.first[threadIdx.x >> 6], first);
  if (nan) atomicOr(&sh.special, 1u);
  __syncthreads();
  first = least_first<NT>(sh);
  nan = sh.special != 0;
  if (first < 65536u) {
    using Bins = Wide<WORDS>;
    Row<Bins, NT, Shared<WORDS>> row{sh, x, V, mask_id, Terms{bf16_bits_to_f32(Bins::bits((int)first)), inv_t, (int)first}};
    for (int w = 0; w < Bins::WINDOWS; ++w) {
      row.count_window(w);
      count_entries<Bins, NT>(sh, w);
      __syncthreads();
      row.sum_window(w);
    }
    __syncthreads();
    draw<Bins, NT>(sh, row, (int)first, g, nan);
  } else if (threadIdx.x == 0) sh.conf = nan ? __builtin_nanf("") : 0.f;
}

}  // namespace

template <int NT, bool PAIRED>
__global__ __launch_bounds__(NT, NT == 512 ? 6 : 4) void k_vocab_sample(SampleArgs a) {
  using Bins = Narrow<PAIRED>;
  __shared__ Shared<Bins::WORDS> sh;
  const int tid = threadIdx.x;
  const int64_t r = blockIdx.x;
  const uint16_t* x = a.logits + r * a.ld;
  const Settings g{a.temperature[r], a.top_k ? a.top_k[r] : 0, a.top_p ? a.top_p[r] : 1.f,
                   a.min_p ? a.min_p[r] : 0.f, a.u[r]};
  if (tid == 0) { sh.special = sh.uncounted = 0; sh.window = 0; sh.id = -1; sh.conf = 0.f; }
  const double inv_t = g.T > 0.f ? 1.0 / (double)g.T : -1.0;  // -1: a greedy row
  uint32_t uncounted;
  int top, top_at;
  uint32_t special = count_row<NT, PAIRED>(sh, x, a.V, a.mask_id, inv_t, uncounted, top, top_at);  // a barrier before it counts
  if (special) atomicOr(&sh.special, special);
  if (uncounted) atomicAdd(&sh.uncounted, uncounted);
  int most = top;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) most = max(most, __shfl_xor(most, o, 64));
  if ((tid & 63) == 0) sh.top[tid >> 6] = most;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) most = max(most, sh.top[i]);
  special = sh.special;
  const int place = most >= 0 ? Bins::place((uint32_t)most) : -1;
  uint32_t first = place < 0 ? INT_MAX : (uint32_t)Bins::bin((uint32_t)most, place);
  if (first == INT_MAX || Bins::four(sh.hist, first & ~3u)[first & 3] == 0) {
    // no logit above -0, or the mask id alone holds the maximum
    count_entries<Bins, NT>(sh, 0);
    __syncthreads();
    first = least_first<NT>(sh);
    // a multiple of 65536 equal negative logits and no other leave no count at all
    if (PAIRED && first == INT_MAX && sh.uncounted != (uint32_t)a.V) special = OTHER;
  }
  // Numbers of -2^19 and below beside a maximum of at least -2^18 weigh exp(-2^18 / T), which is
  // 0 in 64 bits for T up to 350, and can then be left out.
  if (special == FAR_BELOW && g.T < 350.f && first < (uint32_t)Bins::BINS &&
      bf16_bits_to_f32(Bins::bits((int)first)) >= -262144.f)
    special = 0;
  if (!special && first < (uint32_t)Bins::BINS) {
    Row<Bins, NT, Shared<Bins::WORDS>> row{sh, x, a.V, a.mask_id,
                                           Terms{bf16_bits_to_f32(Bins::bits((int)first)), inv_t, (int)first}};
    row.sum_all();
    __syncthreads();
    if (PAIRED) {  // a count that passed 65535 took 65535 or 65536 off the sum
      static_assert(Bins::ENTRIES == 64, "an entry to a lane");
      const uint32_t n = lane_value(wave_scan(sh.cnt[tid & 63]), 63);
      if (n + sh.uncounted != (uint32_t)a.V) special = OTHER;
    }
    if (!special) {
      const bool known = most > 0 && (a.mask_id < 0 || (int)(short)x[a.mask_id] != most);
      draw<Bins, NT>(sh, row, (int)first, g, false, known ? most : NO_TOP, top, top_at);
    }
  }
  if (special) wide_row<NT>(sh, x, a.V, a.mask_id, g, inv_t);
  if (tid == 0) {
    a.token[r] = sh.id;
    a.conf[r] = sh.conf;
  }
}

hipError_t launch_vocab_sample(const SampleArgs& a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  // Up to a row per CU: 1024 threads, 32 x 126464 in 21.9 us against 25.0 with 512.  More: 512, three
  // rows to a CU, 4096 x 126464 in 253 us against 378 with 1024 and one, 303 with 1024 in 64 registers
  // and two, 310 with 512 in 64 registers and four (both spill); 777 x 50257 in 41.5 against 57, 54, 47
  // (225 and 38 us since).
  const bool many = a.rows > 256;
  if (many) hipLaunchKernelGGL((k_vocab_sample<512, true>), dim3(a.rows), dim3(512), 0, s, a);
  else hipLaunchKernelGGL((k_vocab_sample<1024, false>), dim3(a.rows), dim3(1024), 0, s, a);
  return hipGetLastError();
}

}  // namespace cora
