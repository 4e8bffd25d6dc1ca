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
// One workgroup of 1024 threads per row:
//   1 count: one pass over the row, an LDS add per logit;
//   2 sum:   (count, sum of w, sum of exp) of each 256-bin entry;
//   3 pick:  the borders n1, n2, n3 and the token's bin and rank in it, by wavefront 0: a scan of
//            the entries, then of the 256 bins of the one that holds the border;
//   4 find:  the rank-th id that holds the value, in a second reading of the row up to that id.
// The bins of step 1 are the bf16 numbers of magnitude 2^-44 to 2^19 of either sign and zero, 64
// KB, so that two workgroups share a CU and one counts while the other scans.  A row with any
// other finite number (a ban by bf16's lowest one, a maximum beyond 2^19), +inf or NaN is done by
// the same steps over all 65536 bf16 numbers in four windows, at one reading of the row each.
#include <limits.h>

#include <algorithm>

#include "common.hpp"
#include "internal.hpp"

namespace cora {

namespace {

constexpr int NT = 1024, NW = NT / 64;
constexpr int BINS = 16384, ENT = 256, NENT = BINS / ENT;  // bins in LDS, bins per entry
constexpr uint32_t LO = 83u << 7, SPAN = 63u << 7;         // magnitudes 2^-44 <= |l| < 2^19
constexpr int MID = (int)SPAN;                             // the bin of zero
constexpr uint32_t FAR_BELOW = 1, OTHER = 2;               // finite numbers <= -2^19; the rest without a bin

// A scheme of bins in the order of falling value.  Narrow: one window as above.
// Wide: all bf16 numbers, window w holds bins [w BINS, (w + 1) BINS).
struct Narrow {
  static constexpr int WINDOWS = 1, LAST = 2 * MID;
  // bin of a number, or -1 when it has none
  static __device__ __forceinline__ int bin(uint32_t b) {
    const uint32_t mag = b & 0x7fff, t = mag - LO;
    const int i = (b & 0x8000) ? MID + 1 + (int)t : MID - 1 - (int)t;
    return t < SPAN ? i : (mag == 0 ? MID : -1);
  }
  static __device__ __forceinline__ uint32_t bits(int i) {
    return i == MID ? 0u : (i < MID ? LO + (uint32_t)(MID - 1 - i) : 0x8000u | (LO + (uint32_t)(i - MID - 1)));
  }
};
struct Wide {
  static constexpr int WINDOWS = 4, LAST = 0xff7f;  // the bin of the lowest finite number
  static __device__ __forceinline__ int bin(uint32_t b) {
    const uint32_t mag = b & 0x7fff;
    if (mag > 0x7f80 || b == 0xff80) return -1;  // NaN, -inf
    return (b & 0x8000) && mag ? 0x8000 + (int)mag : 0x7fff - (int)mag;
  }
  static __device__ __forceinline__ uint32_t bits(int i) {
    return i < 0x8000 ? 0x7fffu - (uint32_t)i : 0x8000u | (uint32_t)(i - 0x8000);
  }
};

struct Shared {
  uint32_t hist[BINS];
  uint32_t cnt[4 * NENT];
  double wt[4 * NENT], w1[4 * NENT];  // of each entry: sum of w, sum of exp
  uint32_t first, special;            // least bin in use; FAR_BELOW, OTHER numbers without a bin
  int window;                         // that the histogram holds
  uint32_t tot[2][4][NW];
  // the pick: value, rank among its equals
  uint32_t value, rank;
  float conf;
  int id;
};

// Calls f(logit bits, id) for every logit of the row.
template <class F>
__device__ __forceinline__ void each_logit(const uint16_t* x, int V, F&& f) {
  const int tid = threadIdx.x;
  const int v0 = min((int)((0 - (uintptr_t)x) & 15) / 2, V);
  const int nch = (V - v0) >> 3, v1 = v0 + nch * 8;
  const u32x4_t* xv = reinterpret_cast<const u32x4_t*>(x + v0);
  auto eight = [&](u32x4_t w, int c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) f((j & 1) ? w[j >> 1] >> 16 : w[j >> 1] & 0xffffu, v0 + c * 8 + j);
  };
  int c = tid;
  for (; c + 3 * NT < nch; c += 4 * NT) {
    u32x4_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = xv[c + i * NT];
#pragma unroll
    for (int i = 0; i < 4; ++i) eight(w[i], c + i * NT);
  }
  for (; c < nch; c += NT) eight(xv[c], c);
  if (tid < v0) f(x[tid], tid);
  if (tid < V - v1) f(x[v1 + tid], v1 + tid);
}

__device__ __forceinline__ double shfl_up_f64(double v, int o) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __shfl_up((uint32_t)b, o, 64), hi = __shfl_up((uint32_t)(b >> 32), o, 64);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

__device__ __forceinline__ double shfl_f64(double v, int lane) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __shfl((uint32_t)b, lane, 64), hi = __shfl((uint32_t)(b >> 32), lane, 64);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// inclusive sums over the lanes of a wavefront
__device__ __forceinline__ double scan_f64(double v, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double u = shfl_up_f64(v, o);
    if (lane >= o) v += u;
  }
  return v;
}

__device__ __forceinline__ uint32_t scan_u32(uint32_t v, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t u = __shfl_up(v, o, 64);
    if (lane >= o) v += u;
  }
  return v;
}

// what the terms of a row are measured against
struct Terms {
  float max;
  double inv_t;  // 1 / T, 0 for a greedy row
  // l - max of a bin's number; 0 for the maximum also where that is +inf
  template <class Scheme>
  __device__ __forceinline__ double below(int bin) const {
    const float v = bf16_bits_to_f32(Scheme::bits(bin));
    return v == max ? 0.0 : (double)v - (double)max;
  }
  __device__ __forceinline__ double weight(double d) const {
    return d == 0.0 ? 1.0 : (d == -INFINITY ? 0.0 : exp(d * inv_t));
  }
};

// A place in the order of falling logits: `before` terms of sum `mass` come before the bin, whose
// terms weigh `w` each and are `count` in number.
struct Place {
  int bin;
  uint32_t before, count;
  double mass, w;
};

// The histogram of one row: windows of it counted on demand, and the searches in it.  Every
// method is called by the whole workgroup; the searches' results are wavefront 0's.
template <class Scheme>
struct Row {
  Shared& sh;
  const uint16_t* x;
  int V, mask_id;
  Terms t;
  static constexpr int EPL = Scheme::WINDOWS * NENT / 64;  // entries of a lane

  __device__ void clear() {
    u32x4_t* h = reinterpret_cast<u32x4_t*>(sh.hist);
    for (int i = threadIdx.x; i < BINS / 4; i += NT) h[i] = u32x4_t{0, 0, 0, 0};
  }

  // counts window `win`
  __device__ void count_window(int win) {
    __syncthreads();  // everyone is done with the window before
    clear();
    __syncthreads();
    each_logit(x, V, [&](uint32_t b, int id) {
      const int i = Scheme::bin(b) - win * BINS;
      if (id != mask_id && (uint32_t)i < (uint32_t)BINS) atomicAdd(&sh.hist[i], 1u);
    });
    if (threadIdx.x == 0) sh.window = win;
    __syncthreads();
  }

  // the entries of the window that the histogram holds
  __device__ void sum_window(int win) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int e = wave; e < NENT; e += NW) {
      const u32x4_t c = *reinterpret_cast<const u32x4_t*>(&sh.hist[e * ENT + lane * 4]);
      uint32_t n = 0;
      double st = 0.0, s1 = 0.0;
      if (__any((c[0] | c[1] | c[2] | c[3]) != 0)) {
#pragma unroll 1
        for (int j = 0; j < 4; ++j) {
          const uint32_t cj = j == 0 ? c[0] : (j == 1 ? c[1] : (j == 2 ? c[2] : c[3]));
          if (cj) {
            const double d = t.template below<Scheme>(win * BINS + e * ENT + lane * 4 + j);
            const double e1 = exp(d);
            n += cj;
            s1 += cj * e1;
            st += t.inv_t == 1.0 ? cj * e1 : cj * t.weight(d);
          }
        }
        n = scan_u32(n, lane);
        st = scan_f64(st, lane);
        s1 = scan_f64(s1, lane);
      }
      if (lane == 63) {
        sh.cnt[win * NENT + e] = n;
        sh.wt[win * NENT + e] = st;
        sh.w1[win * NENT + e] = s1;
      }
    }
  }

  // The entry that holds term k of the row's order (BY_COUNT), or at which the running sum of w
  // passes m (strict) or reaches it; and the terms and their sum before it.
  template <bool BY_COUNT>
  __device__ int entry_of(uint32_t k, double m, bool strict, uint32_t& before, double& mass) const {
    const int lane = threadIdx.x & 63;
    uint32_t n = 0;
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      n += sh.cnt[lane * EPL + i];
      s += sh.wt[lane * EPL + i];
    }
    const uint32_t ni = scan_u32(n, lane);
    const double si = scan_f64(s, lane);
    const int l = border(n > 0 && (BY_COUNT ? ni > k : (strict ? si > m : si >= m)), n > 0);
    before = __shfl(ni - n, l, 64);
    mass = l > 0 ? shfl_f64(si, l - 1) : 0.0;
    int e = l * EPL, last = e;  // last: of the lane's entries in use
#pragma unroll
    for (int i = 1; i < EPL; ++i)
      if (sh.cnt[l * EPL + i]) last = l * EPL + i;
    for (; e < last; ++e) {
      const uint32_t c = sh.cnt[e];
      const double w = sh.wt[e];
      if (c && (BY_COUNT ? before + c > k : (strict ? mass + w > m : mass + w >= m))) break;
      before += c;
      mass += w;
    }
    return e;
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
  __device__ __forceinline__ u32x4_t four(int e, double (&w)[4], uint32_t& n, double& s) const {
    const int lane = threadIdx.x & 63;
    const u32x4_t c = *reinterpret_cast<const u32x4_t*>(&sh.hist[(e % NENT) * ENT + lane * 4]);
    n = 0;
    s = 0.0;
#pragma unroll 1
    for (int j = 0; j < 4; ++j) {
      const uint32_t cj = j == 0 ? c[0] : (j == 1 ? c[1] : (j == 2 ? c[2] : c[3]));
      double v = 0.0;
      if (cj) v = t.weight(t.template below<Scheme>(e * ENT + lane * 4 + j));
      if (j == 0) w[0] = v; else if (j == 1) w[1] = v; else if (j == 2) w[2] = v; else w[3] = v;
      n += cj;
      s += cj * v;
    }
    return c;
  }

  // The bin that holds term k (BY_COUNT), or in which the running sum passes / reaches m.
  template <bool BY_COUNT>
  __device__ Place find(uint32_t k, double m, bool strict) {
    uint32_t before = 0, n;
    double mass = 0.0, s, w[4];
    const int lane = threadIdx.x & 63;
    const int e = entry_of<BY_COUNT>(k, m, strict, before, mass);
    hold(e);
    const u32x4_t c = four(e, w, n, s);
    const uint32_t ni = scan_u32(n, lane) + before;
    const double si = scan_f64(s, lane) + mass;
    const int l = border(n > 0 && (BY_COUNT ? ni > k : (strict ? si > m : si >= m)), n > 0);
    Place p{0, ni - n, 0, si - s, 0.0};
    bool found = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (!c[j] || found) continue;
      if (p.count) {  // the bin before is not the one
        p.before += p.count;
        p.mass += p.count * p.w;
      }
      p.bin = e * ENT + lane * 4 + j;
      p.count = c[j];
      p.w = w[j];
      found = BY_COUNT ? p.before + c[j] > k : (strict ? p.mass + c[j] * w[j] > m : p.mass + c[j] * w[j] >= m);
    }
    p.bin = __shfl(p.bin, l, 64);
    p.before = __shfl(p.before, l, 64);
    p.count = __shfl(p.count, l, 64);
    p.mass = shfl_f64(p.mass, l);
    p.w = shfl_f64(p.w, l);
    return p;
  }

  // terms in bins up to `bin` and their sum
  __device__ uint32_t up_to(int bin, double& mass) {
    const int lane = threadIdx.x & 63, e = bin / ENT;
    uint32_t n = 0;
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (lane * EPL + i < e) {
        n += sh.cnt[lane * EPL + i];
        s += sh.wt[lane * EPL + i];
      }
    hold(e);
    uint32_t ne;
    double se, w[4];
    const u32x4_t c = four(e, w, ne, se);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (e * ENT + lane * 4 + j <= bin) {
        n += c[j];
        s += c[j] * w[j];
      }
    mass = shfl_f64(scan_f64(s, lane), 63);
    return __shfl(scan_u32(n, lane), 63, 64);
  }
};

// A row's settings.
struct Settings {
  float T;
  int top_k;
  float top_p, min_p, u;
};

// Step 3, by wavefront 0 (by every wavefront where windows are counted on the way): the bin of
// the token and its rank among that bin's ids.
template <class Scheme>
__device__ void pick(Row<Scheme>& row, int first, const Settings& g, uint32_t n, Place& p, uint32_t& rank) {
  p = Place{first, 0, 1, 0.0, 1.0};
  rank = 0;
  if (!(g.T > 0.f)) return;
  uint32_t N = g.top_k > 0 ? min((uint32_t)g.top_k, n) : n;
  p = row.template find<true>(N - 1, 0.0, false);
  double mass = p.mass + (N - p.before) * p.w;  // of the first N terms
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
    double m3;
    const uint32_t n3 = g.min_p > 1.f ? 1u : row.up_to(lo, m3);
    if (g.min_p > 1.f) m3 = 1.0;
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

// Step 4: the rank-th id that holds the value, FIND * 8 * NT ids at a time in order.
constexpr int FIND = 4;
__device__ void find_id(Shared& sh, const uint16_t* x, int V, int mask_id) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t want = sh.value, left = sh.rank;
  const int shift = (int)((uintptr_t)x & 15) / 2;  // chunk c holds ids 8 c - shift ..
  const u32x4_t* xv = reinterpret_cast<const u32x4_t*>(x - shift);
  const int nch = (V + shift + 7) >> 3;
  uint32_t seen = 0;
  for (int c0 = 0, it = 0; c0 < nch; c0 += FIND * NT, it ^= 1) {
    uint32_t hits[FIND], inc[FIND];
    u32x4_t w[FIND];
    bool whole[FIND];
#pragma unroll
    for (int k = 0; k < FIND; ++k) {
      const int id = (c0 + k * NT + tid) * 8 - shift;
      whole[k] = id >= 0 && id + 8 <= V;
      if (whole[k]) w[k] = xv[c0 + k * NT + tid];
    }
#pragma unroll
    for (int k = 0; k < FIND; ++k) {
      const int id = (c0 + k * NT + tid) * 8 - shift;
      hits[k] = 0;
      if (whole[k]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint32_t b = (j & 1) ? w[k][j >> 1] >> 16 : w[k][j >> 1] & 0xffffu;
          hits[k] |= (uint32_t)(b == want || (want == 0 && b == 0x8000u)) << j;
        }
      } else if (id < V) {
        for (int j = 0; j < 8; ++j)
          if (id + j >= 0 && id + j < V) {
            const uint32_t b = x[id + j];
            hits[k] |= (uint32_t)(b == want || (want == 0 && b == 0x8000u)) << j;
          }
      }
      if ((uint32_t)(mask_id - id) < 8u) hits[k] &= ~(1u << (mask_id - id));
    }
#pragma unroll
    for (int k = 0; k < FIND; ++k) {
      inc[k] = 0;
      if (__any(hits[k])) inc[k] = scan_u32(__popc(hits[k]), lane);
      if (lane == 63) sh.tot[it][k][wave] = inc[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < FIND; ++k) {
      uint32_t before = seen;
#pragma unroll
      for (int i = 0; i < NW; ++i) {
        const uint32_t c = sh.tot[it][k][i];
        if (i < wave) before += c;
        seen += c;
      }
      const uint32_t own = __popc(hits[k]);
      before += inc[k] - own;
      if (before <= left && left < before + own) {
        uint32_t h = hits[k];
        for (uint32_t j = before; j < left; ++j) h &= h - 1;
        sh.id = (c0 + k * NT + tid) * 8 - shift + __ffs(h) - 1;
      }
    }
    if (seen > left) break;
  }
  __syncthreads();
}

// Steps 2 to 4 of a row that holds an allowed number; its window is counted (Narrow) or none is.
template <class Scheme>
__device__ void draw(Shared& sh, const uint16_t* x, int V, int mask_id, int first, const Settings& g, bool nan) {
  const int tid = threadIdx.x, lane = tid & 63;
  Row<Scheme> row{sh, x, V, mask_id,
                  Terms{bf16_bits_to_f32(Scheme::bits(first)), g.T > 0.f ? 1.0 / (double)g.T : 0.0}};
  for (int w = 0; w < Scheme::WINDOWS; ++w) {
    if (Scheme::WINDOWS > 1) row.count_window(w);
    row.sum_window(w);
  }
  __syncthreads();
  if (Scheme::WINDOWS > 1 || tid < 64) {
    uint32_t n = 0, rank;
    double s1 = 0.0;
#pragma unroll
    for (int i = 0; i < Row<Scheme>::EPL; ++i) {
      n += sh.cnt[lane * Row<Scheme>::EPL + i];
      s1 += sh.w1[lane * Row<Scheme>::EPL + i];
    }
    n = __shfl(scan_u32(n, lane), 63, 64);
    s1 = shfl_f64(scan_f64(s1, lane), 63);
    Place p;
    pick<Scheme>(row, first, g, n, p, rank);
    if (tid == 0) {
      sh.value = Scheme::bits(p.bin);
      sh.rank = rank;
      sh.conf = nan ? __builtin_nanf("") : (float)(exp(row.t.template below<Scheme>(p.bin)) / s1);
      sh.id = -1;
    }
  }
  __syncthreads();
  find_id(sh, x, V, mask_id);
}

}  // namespace

__global__ __launch_bounds__(NT, 8) void k_vocab_sample(SampleArgs a) {
  __shared__ Shared sh;
  const int tid = threadIdx.x;
  const int64_t r = blockIdx.x;
  const uint16_t* x = a.logits + r * a.ld;
  const Settings g{a.temperature[r], a.top_k ? a.top_k[r] : 0, a.top_p ? a.top_p[r] : 1.f,
                   a.min_p ? a.min_p[r] : 0.f, a.u[r]};

  {
    u32x4_t* h = reinterpret_cast<u32x4_t*>(sh.hist);
    for (int i = tid; i < BINS / 4; i += NT) h[i] = u32x4_t{0, 0, 0, 0};
  }
  if (tid == 0) { sh.first = INT_MAX; sh.special = 0; sh.window = 0; }
  __syncthreads();
  uint32_t first = INT_MAX, special = 0;
  each_logit(x, a.V, [&](uint32_t b, int) {
    const int i = Narrow::bin(b);
    if (i >= 0) {
      atomicAdd(&sh.hist[i], 1u);
      first = min(first, (uint32_t)i);
    } else if (b != 0xff80u) {
      special |= b > 0x8000u + LO && b < 0xff80u ? FAR_BELOW : OTHER;
    }
  });
  atomicMin(&sh.first, first);
  if (special) atomicOr(&sh.special, special);
  __syncthreads();
  if (tid == 0 && a.mask_id >= 0) {  // the mask id was counted like the others: taken back
    const int i = Narrow::bin(x[a.mask_id]);
    if (i >= 0) sh.hist[i] -= 1;
  }
  __syncthreads();
  first = sh.first;
  special = sh.special;
  if (first < (uint32_t)BINS && sh.hist[first] == 0) {  // the mask id alone held the maximum
    __syncthreads();
    if (tid == 0) sh.first = INT_MAX;
    __syncthreads();
    uint32_t f = INT_MAX;
    for (int i = tid; i < BINS; i += NT)
      if (sh.hist[i]) f = min(f, (uint32_t)i);
    atomicMin(&sh.first, f);
    __syncthreads();
    first = sh.first;
  }
  // Numbers of -2^19 and below beside a maximum of at least -2^18 weigh exp(-2^18 / T), which is
  // 0 in 64 bits for T up to 350, and can then be left out.
  if (special == FAR_BELOW && g.T < 350.f && first < (uint32_t)BINS &&
      bf16_bits_to_f32(Narrow::bits((int)first)) >= -262144.f)
    special = 0;
  if (special) {
    // numbers beyond the narrow bins: maximum and NaNs of the allowed ids, then all bins
    __syncthreads();
    if (tid == 0) { sh.first = INT_MAX; sh.special = 0; sh.window = -1; }
    __syncthreads();
    first = INT_MAX;
    bool nan = false;
    each_logit(x, a.V, [&](uint32_t b, int id) {
      if (id == a.mask_id) return;
      const int i = Wide::bin(b);
      if (i >= 0) first = min(first, (uint32_t)i);
      else nan |= b != 0xff80u;
    });
    atomicMin(&sh.first, first);
    if (nan) atomicOr(&sh.special, 1u);
    __syncthreads();
    first = sh.first;
    nan = sh.special != 0;
    if (first < 4u * BINS) draw<Wide>(sh, x, a.V, a.mask_id, (int)first, g, nan);
    else if (tid == 0) { sh.id = -1; sh.conf = nan ? __builtin_nanf("") : 0.f; }
  } else if (first < (uint32_t)BINS) {
    draw<Narrow>(sh, x, a.V, a.mask_id, (int)first, g, false);
  } else if (tid == 0) {
    sh.id = -1;
    sh.conf = 0.f;
  }
  if (tid == 0) {
    a.token[r] = sh.id;
    a.conf[r] = sh.conf;
  }
}

hipError_t launch_vocab_sample(const SampleArgs& a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  hipLaunchKernelGGL(k_vocab_sample, dim3(a.rows), dim3(NT), 0, s, a);
  return hipGetLastError();
}

}  // namespace cora
