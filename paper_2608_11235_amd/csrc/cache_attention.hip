// Attention of a chunk of new tokens over a paged K/V cache, online softmax in fp32.
//
// For row i of request b's chunk and query head h (kv head h / G, G = H / Hkv):
//   o = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q . k_j),  j < len_b and, causal, j <= start_b + i.
// A row without a key is zero.  Both products run transposed on v_mfma_f32_16x16x32_bf16, like the
// dense pass's attention: S^T = K Q^T, O^T = V^T P^T, so that a query's statistics stay in its lanes
// and the S^T registers are the P^T operand.  The pages hold K and V in the lane order of these
// operands (cache_k_index, cache_v_index): 32 keys are HD / 16 blocks of 1 KB each, one wavefront
// load a block, and the eight P^T slots of a lane group are eight neighbouring keys.
//
// The G query heads of a kv head share its K and V: the rows of a tile are (token, head) pairs,
// token-major.  Tile t of RT rows belongs to the request b with base_b <= t < base_(b+1),
// base_b = cu_b G / RT + b, which leaves each request at least as many tiles as it fills and needs
// no pass over the lengths; a workgroup whose tile holds no row returns.
//
// Two kernels.  k_cache_attend_rows (16 or 32 rows a tile): bound by the stream of K and V, each of
// whose blocks is used by one wavefront, so they go from memory into the operand registers and the
// four wavefronts take every fourth group of 32 keys; their states merge through LDS.
// k_cache_attend_tile (64 or 128 rows): 64-key tiles through two LDS stages, loaded directly.
// Either runs over key ranges of `chunk` keys where the rows alone would not fill the card; the
// ranges' (max, sum, O) go to the workspace and k_cache_attend_merge folds them in order.
#include <algorithm>

#include "common.hpp"
#include "internal.hpp"

namespace cora {

namespace {

constexpr float SLACK = 8.f;  // a reference maximum moves when a score passes it by 2^SLACK

__device__ __forceinline__ int clamped_cu(const CacheAttnArgs& a, int b) { return min(max(a.cu[b], 0), a.rows); }

// The greatest b in [0, B) with first(b) <= t, for an ascending first with first(0) <= t, by the
// lanes of a wavefront together.
template <class F>
__device__ __forceinline__ int owner_by_lanes(int B, int t, F first) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = B;
  while (hi - lo > 64) {
    const int step = (hi - lo + 63) / 64, i = lo + lane * step;
    const int n = __popcll(__ballot(i < hi && first(i) <= t));
    lo += (max(n, 1) - 1) * step;
    hi = min(hi, lo + step);
  }
  const int n = __popcll(__ballot(lo + lane < hi && first(lo + lane) <= t));
  return lo + max(n, 1) - 1;
}

// What a workgroup works on: rows [row0, row0 + RT) of the (token, head) rows of request b and kv
// head kvh, keys [k0, k1) of its `len`.
struct Work {
  int b, kvh, split, row0, n_rows, cu, start, len, k0, k1;
};

template <int RT>
__device__ __forceinline__ bool work_of(const CacheAttnArgs& a, Work& w) {
  const int li = xcd_remap(blockIdx.x, gridDim.x);
  // later tiles see more keys under the causal mask: they start first
  const int t = a.tiles - 1 - li % a.tiles, rest = li / a.tiles;
  w.split = rest % a.splits;
  w.kvh = rest / a.splits;
  const int G = a.G;
  w.b = __builtin_amdgcn_readfirstlane(
      owner_by_lanes(a.B, t, [&](int b) { return (int)((int64_t)clamped_cu(a, b) * G / RT) + b; }));
  w.cu = clamped_cu(a, w.b);
  const int n = clamped_cu(a, w.b + 1) - w.cu;
  w.n_rows = n * G;
  w.row0 = (t - (int)((int64_t)w.cu * G / RT) - w.b) * RT;
  if (w.row0 >= w.n_rows) return false;
  w.start = a.start[w.b];
  w.len = min(max(a.len[w.b], 0), a.max_pages << a.shift);
  w.k0 = w.split * a.chunk;
  if (w.split > 0 && w.k0 >= w.len) return false;
  w.k1 = w.split == a.splits - 1 ? w.len : min(w.len, w.k0 + a.chunk);
  return true;
}

// keys that row `row` sees; rows behind the last one, whose results nobody reads, as many as it
__device__ __forceinline__ int limit_of(const CacheAttnArgs& a, const Work& w, int row) {
  row = min(row, w.n_rows - 1);
  if (!a.causal) return w.len;
  return min((int64_t)w.len, max((int64_t)w.start + row / a.G + 1, (int64_t)0));
}

// The page of 32-key group `grp` of the request, 64 table entries held in the lanes.
struct PageList {
  const int32_t* table;
  int shift5, n_pages, max_pages, base, mine;  // shift5: log2 of 32-key groups a page
  __device__ __forceinline__ void load(int page) {
    base = page;
    const int p = page + (int)(threadIdx.x & 63);
    mine = p < max_pages ? table[p] : 0;
  }
  __device__ __forceinline__ int page(int grp) {
    const int p = grp >> shift5;
    if (p - base >= 64) load(p);
    const int e = __builtin_amdgcn_readlane(mine, p - base);
    return (unsigned)e < (unsigned)n_pages ? e : 0;  // a bad entry reads page 0, never past the pool
  }
};

template <int HD>
__device__ __forceinline__ void load_q(const CacheAttnArgs& a, const Work& w, int row, bf16x8_t (&qf)[HD / 32]) {
  const int g = (threadIdx.x & 63) >> 4;
  const uint16_t* q = a.q + ((int64_t)(w.cu + row / a.G) * a.H + w.kvh * a.G + row % a.G) * HD + g * 8;
#pragma unroll
  for (int kk = 0; kk < HD / 32; ++kk)
    qf[kk] = as_bf16x8(row < w.n_rows ? *reinterpret_cast<const u32x4_t*>(q + kk * 32) : u32x4_t{0, 0, 0, 0});
}

// Moves the reference of the scores st[NB] of one query (max over its four lane groups) and
// rescales, then turns the scores into terms.
template <int NB, int ND>
__device__ __forceinline__ void soften(f32x4_t (&st)[NB], float scale_log2, float& m_ref, float& m_use, float& l,
                                       f32x4_t (&o)[ND]) {
  float lmax = -INFINITY;
#pragma unroll
  for (int kb = 0; kb < NB; ++kb)
#pragma unroll
    for (int i = 0; i < 4; ++i) lmax = fmaxf(lmax, st[kb][i]);
  if (__any(lmax * scale_log2 > m_ref + SLACK)) {
    float tmax = fmaxf(lmax, __shfl_xor(lmax, 16, 64));
    tmax = fmaxf(tmax, __shfl_xor(tmax, 32, 64));
    const float tm = tmax * scale_log2;
    if (tm > m_ref + SLACK) {  // never while no key was seen and none is
      const float alpha = fast_exp2(m_ref - tm);
      m_ref = m_use = tm;
      l *= alpha;
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d] *= alpha;
    }
  }
#pragma unroll
  for (int kb = 0; kb < NB; ++kb)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p = fast_exp2(fmaf(st[kb][i], scale_log2, -m_use));  // m_use 0 until a key is seen
      st[kb][i] = p;
      l += p;
    }
}

__device__ __forceinline__ bf16x8_t terms_operand(const f32x4_t& x, const f32x4_t& y) {
  return as_bf16x8(u32x4_t{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(y[0], y[1]),
                           pack_bf16x2(y[2], y[3])});
}

// the first n of a lane's eight keys, zeros for the others
__device__ __forceinline__ u32x4_t keep_keys(u32x4_t v, int n) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t m = n >= 2 * i + 2 ? 0xffffffffu : (n == 2 * i + 1 ? 0xffffu : 0u);
    v[i] &= m;
  }
  return v;
}

// Where the mask cuts rows of one group at different keys, a row must not see the others' V even
// as 0 * NaN: V that is inf or NaN goes into the product as 0 ...
__device__ __forceinline__ u32x4_t finite_only(u32x4_t v, bool& bad) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool lo = (v[i] & 0x7f80u) == 0x7f80u, hi = (v[i] & 0x7f800000u) == 0x7f800000u;
    bad |= lo | hi;
    v[i] &= (lo ? 0xffff0000u : 0xffffffffu) & (hi ? 0xffffu : 0xffffffffu);
  }
  return v;
}

// ... and is added by hand to the rows that see its key: `v` the 32-key group's V, p0 and p1 its terms,
// n the keys of the group that the lane's row sees.
template <int ND>
__device__ __forceinline__ void add_non_finite(const uint16_t* v, const f32x4_t& p0, const f32x4_t& p1, int n,
                                               f32x4_t (&o)[ND]) {
  const int lane = threadIdx.x & 63, g = lane >> 4, r16 = lane & 15;
#pragma unroll 1
  for (int key = 0; key < 32; ++key) {
    const int e = key & 7, gk = key >> 3;
    float p = e < 4 ? p0[0] : p1[0];
    p = (e & 3) == 1 ? (e < 4 ? p0[1] : p1[1]) : p;
    p = (e & 3) == 2 ? (e < 4 ? p0[2] : p1[2]) : p;
    p = (e & 3) == 3 ? (e < 4 ? p0[3] : p1[3]) : p;
    p = __shfl(p, gk * 16 + r16, 64);
    if (key >= n) continue;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t x = v[d * 512 + gk * 128 + (4 * g + i) * 8 + e];
        if ((x & 0x7f80u) == 0x7f80u) o[d][i] += p * bf16_bits_to_f32(x);
      }
  }
}

__device__ __forceinline__ int64_t out_index(const CacheAttnArgs& a, int token, int head, int d, int HD) {
  if (!a.panels) return ((int64_t)token * a.H + head) * HD + d;
  const int c = head * HD + d;  // K panels [H HD / 32][rows][32]
  return ((int64_t)(c >> 5) * a.rows + token) * 32 + (c & 31);
}

}  // namespace

template <int HD, int RB>
__global__ __launch_bounds__(256) void k_cache_attend_rows(CacheAttnArgs a) {
  constexpr int RT = RB * 16, NK = HD / 32, ND = HD / 16, LDO = HD + 4;
  __shared__ float so[4][RT][LDO];
  __shared__ float sm[4][RT], sl[4][RT];
  Work w;
  if (!work_of<RT>(a, w)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, r16 = lane & 15;

  bf16x8_t qf[RB][NK];
  int lim[RB], most = 0;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = w.row0 + rb * 16 + r16;
    load_q<HD>(a, w, row, qf[rb]);
    lim[rb] = limit_of(a, w, row);
    most = max(most, lim[rb]);
  }
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) most = max(most, __shfl_xor(most, o, 64));
  const int end = __builtin_amdgcn_readfirstlane(min(w.k1, most));  // keys that some row sees
  const int g0 = w.k0 >> 5, g1 = (end + 31) >> 5;

  f32x4_t o[RB][ND];
  float m_ref[RB], m_use[RB], l[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    m_ref[rb] = -INFINITY;
    m_use[rb] = l[rb] = 0.f;
#pragma unroll
    for (int d = 0; d < ND; ++d) o[rb][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  const int64_t head_elems = (int64_t)HD << a.shift;
  PageList pl{a.table + (int64_t)w.b * a.max_pages, a.shift - 5, a.n_pages, a.max_pages, 0, 0};
  const int gmask = (1 << (a.shift - 5)) - 1;
  auto at = [&](int grp) -> int64_t {  // element offset of a 32-key group in the pool
    return ((int64_t)pl.page(grp) * a.Hkv + w.kvh) * head_elems + (int64_t)(grp & gmask) * (32 * HD) + lane * 8;
  };
  u32x4_t kf[2 * NK], vf[ND];
  int grp = g0 + wave;
  if (grp < g1) {
    pl.load(grp >> pl.shift5);
    const u32x4_t* p = reinterpret_cast<const u32x4_t*>(a.k + at(grp));
#pragma unroll
    for (int i = 0; i < 2 * NK; ++i) kf[i] = p[i * 64];
  }
  for (; grp < g1; grp += 4) {
    {
      const u32x4_t* p = reinterpret_cast<const u32x4_t*>(a.v + at(grp));
#pragma unroll
      for (int i = 0; i < ND; ++i) vf[i] = p[i * 64];
    }
    f32x4_t st[RB][2];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        st[rb][kb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < NK; ++kk)
          st[rb][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kf[kb * NK + kk]), qf[rb][kk], st[rb][kb], 0, 0, 0);
      }
    if (grp + 4 < g1) {
      const u32x4_t* p = reinterpret_cast<const u32x4_t*>(a.k + at(grp + 4));
#pragma unroll
      for (int i = 0; i < 2 * NK; ++i) kf[i] = p[i * 64];
    }
    const int key = grp * 32 + 8 * g;  // of the lane's first term
    bool cut = false;                  // some row's last key lies in the group
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int n = min(lim[rb], w.k1) - key;
      if (__any(n < 8)) {
        cut = true;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (4 * kb + i >= n) st[rb][kb][i] = -INFINITY;
      }
      soften<2, ND>(st[rb], a.scale_log2, m_ref[rb], m_use[rb], l[rb], o[rb]);
    }
    if (grp * 32 + 32 > w.len) {  // slots behind the last key may hold anything
#pragma unroll
      for (int d = 0; d < ND; ++d) vf[d] = keep_keys(vf[d], w.len - key);
    }
    bool bad = false;
    if (cut && a.causal) {
#pragma unroll
      for (int d = 0; d < ND; ++d) vf[d] = finite_only(vf[d], bad);
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const bf16x8_t p = terms_operand(st[rb][0], st[rb][1]);
#pragma unroll
      for (int d = 0; d < ND; ++d)
        o[rb][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(vf[d]), p, o[rb][d], 0, 0, 0);
    }
    if (__any(bad)) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
        add_non_finite<ND>(a.v + at(grp) - lane * 8, st[rb][0], st[rb][1], min(lim[rb], w.k1) - grp * 32, o[rb]);
    }
  }

#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    float s = l[rb];
    s += __shfl_xor(s, 16, 64);
    s += __shfl_xor(s, 32, 64);
    const int row = rb * 16 + r16;
    if (g == 0) {
      sm[wave][row] = m_ref[rb];
      sl[wave][row] = s;
    }
#pragma unroll
    for (int d = 0; d < ND; ++d) *reinterpret_cast<f32x4_t*>(&so[wave][row][d * 16 + g * 4]) = o[rb][d];
  }
  __syncthreads();
  // thread: 4 dimensions of a row at a time
  constexpr int TPR = HD / 4;
  for (int i = threadIdx.x; i < RT * TPR; i += 256) {
    const int r = i / TPR, d = (i % TPR) * 4, row = w.row0 + r;
    if (row >= w.n_rows) continue;
    const float m = fmaxf(fmaxf(sm[0][r], sm[1][r]), fmaxf(sm[2][r], sm[3][r]));
    float sum = 0.f;
    f32x4_t x{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const float c = sm[v][r] == -INFINITY ? 0.f : fast_exp2(sm[v][r] - m);
      // a wavefront that saw no key, unlike one that saw a NaN, adds nothing
      if (sm[v][r] == -INFINITY && sl[v][r] == 0.f) continue;
      sum += sl[v][r] * (sm[v][r] == -INFINITY ? 1.f : c);
      x += *reinterpret_cast<const f32x4_t*>(&so[v][r][d]) * (sm[v][r] == -INFINITY ? 1.f : c);
    }
    const int token = w.cu + row / a.G, head = w.kvh * a.G + row % a.G;
    if (a.splits == 1) {
      const float inv = sum == 0.f ? 0.f : 1.0f / sum;
      *reinterpret_cast<u32x2_t*>(a.out + out_index(a, token, head, d, HD)) =
          u32x2_t{pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv)};
    } else {
      const int64_t p = ((int64_t)token * a.H + head) * a.splits + w.split;
      if (d == 0) {
        a.part_ml[2 * p] = m;
        a.part_ml[2 * p + 1] = sum;
      }
      *reinterpret_cast<f32x4_t*>(a.part_o + p * HD + d) = x;
    }
  }
}

template <int HD, int RB>
__global__ __launch_bounds__(256, 2) void k_cache_attend_tile(CacheAttnArgs a) {
  constexpr int RT = 64 * RB, NK = HD / 32, ND = HD / 16, KT = 64;
  constexpr int GB = 32 * HD * 2;             // bytes of K (or V) of a 32-key group
  constexpr int STAGE = 4 * GB;               // two groups of K, then two of V
  __shared__ __attribute__((aligned(16))) unsigned char lds[2 * STAGE];
  typedef __attribute__((address_space(3))) void* lds_ptr_t;
  typedef const __attribute__((address_space(1))) void* global_ptr_t;
  Work w;
  if (!work_of<RT>(a, w)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, r16 = lane & 15;

  bf16x8_t qf[RB][NK];
  int lim[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = w.row0 + (wave * RB + rb) * 16 + r16;
    load_q<HD>(a, w, row, qf[rb]);
    lim[rb] = min(limit_of(a, w, row), w.k1);
  }
  // keys that some row of the wavefront sees, and that some row of the workgroup does
  const int last = min(w.row0 + (wave + 1) * RB * 16, w.n_rows) - 1;
  const int wave_end = w.row0 + wave * RB * 16 < w.n_rows ? min(w.k1, limit_of(a, w, last)) : 0;
  const int end = min(w.k1, limit_of(a, w, min(w.row0 + RT, w.n_rows) - 1));
  const int t0 = w.k0 / KT, t1 = (end + KT - 1) / KT;

  f32x4_t o[RB][ND];
  float m_ref[RB], m_use[RB], l[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    m_ref[rb] = -INFINITY;
    m_use[rb] = l[rb] = 0.f;
#pragma unroll
    for (int d = 0; d < ND; ++d) o[rb][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  const int64_t head_elems = (int64_t)HD << a.shift;
  PageList pl{a.table + (int64_t)w.b * a.max_pages, a.shift - 5, a.n_pages, a.max_pages, 0, 0};
  const int gmask = (1 << (a.shift - 5)) - 1;
  // wavefront w loads half (w & 1) of group (w >> 1) of the tile, K and V: HD / 32 blocks each
  auto fetch = [&](int t, int buf) {
    const int grp = 2 * t + (wave >> 1);
    if (grp * 32 >= w.len) return;
    const int64_t e = ((int64_t)pl.page(grp) * a.Hkv + w.kvh) * head_elems + (int64_t)(grp & gmask) * (32 * HD) +
                      (wave & 1) * (16 * HD) + lane * 8;
    unsigned char* dst = lds + buf * STAGE + wave * (GB / 2);
#pragma unroll
    for (int i = 0; i < NK; ++i)
      __builtin_amdgcn_global_load_lds((global_ptr_t)(a.k + e + i * 512), (lds_ptr_t)(dst + i * 1024), 16, 0, 0);
#pragma unroll
    for (int i = 0; i < NK; ++i)
      __builtin_amdgcn_global_load_lds((global_ptr_t)(a.v + e + i * 512), (lds_ptr_t)(dst + 2 * GB + i * 1024), 16, 0, 0);
  };
  if (t0 < t1) {
    pl.load((2 * t0) >> pl.shift5);
    fetch(t0, 0);
  }
  for (int t = t0; t < t1; ++t) {
    const int buf = (t - t0) & 1, key0 = t * KT;
    // tile t has landed, and every wavefront is done with the stage that tile t + 1 goes to
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (t + 1 < t1) fetch(t + 1, buf ^ 1);
    if (key0 >= wave_end) continue;
    const unsigned char* kl = lds + buf * STAGE + lane * 16;
    const unsigned char* vl = kl + 2 * GB;
    f32x4_t st[RB][4];
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      bf16x8_t kf[NK];
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) kf[kk] = as_bf16x8(*reinterpret_cast<const u32x4_t*>(kl + (kb * NK + kk) * 1024));
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        st[rb][kb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < NK; ++kk)
          st[rb][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[kk], qf[rb][kk], st[rb][kb], 0, 0, 0);
      }
    }
    bool cut = false;  // some row's last key lies in the tile
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int n = lim[rb] - key0 - 8 * g;  // the lane's terms are keys 32 (kb / 2) + 4 (kb % 2) + i
      if (__any(n < 40)) {
        cut = true;
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (32 * (kb >> 1) + 4 * (kb & 1) + i >= n) st[rb][kb][i] = -INFINITY;
      }
      soften<4, ND>(st[rb], a.scale_log2, m_ref[rb], m_use[rb], l[rb], o[rb]);
    }
    const bool ragged = key0 + KT > w.len;  // slots behind the last key may hold anything
    cut = cut && a.causal;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      bool bad = false;
      bf16x8_t p[RB];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) p[rb] = terms_operand(st[rb][2 * ks], st[rb][2 * ks + 1]);
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        u32x4_t v = *reinterpret_cast<const u32x4_t*>(vl + (ks * ND + d) * 1024);
        if (ragged) v = keep_keys(v, w.len - key0 - 32 * ks - 8 * g);
        if (cut) v = finite_only(v, bad);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
          o[rb][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(v), p[rb], o[rb][d], 0, 0, 0);
      }
      if (__any(bad)) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
          add_non_finite<ND>(reinterpret_cast<const uint16_t*>(lds + buf * STAGE + 2 * GB + ks * GB), st[rb][2 * ks],
                             st[rb][2 * ks + 1], lim[rb] - key0 - 32 * ks, o[rb]);
      }
    }
  }

#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    float s = l[rb];
    s += __shfl_xor(s, 16, 64);
    s += __shfl_xor(s, 32, 64);
    const int row = w.row0 + (wave * RB + rb) * 16 + r16;
    if (row >= w.n_rows) continue;
    const int token = w.cu + row / a.G, head = w.kvh * a.G + row % a.G;
    if (a.splits == 1) {
      const float inv = s == 0.f ? 0.f : 1.0f / s;
#pragma unroll
      for (int d = 0; d < ND; ++d)
        *reinterpret_cast<u32x2_t*>(a.out + out_index(a, token, head, d * 16 + g * 4, HD)) =
            u32x2_t{pack_bf16x2(o[rb][d][0] * inv, o[rb][d][1] * inv), pack_bf16x2(o[rb][d][2] * inv, o[rb][d][3] * inv)};
    } else {
      const int64_t p = ((int64_t)token * a.H + head) * a.splits + w.split;
      if (g == 0) {
        a.part_ml[2 * p] = m_ref[rb];
        a.part_ml[2 * p + 1] = s;
      }
#pragma unroll
      for (int d = 0; d < ND; ++d) *reinterpret_cast<f32x4_t*>(a.part_o + p * HD + d * 16 + g * 4) = o[rb][d];
    }
  }
}

// One wavefront per (row, head): the key ranges' partial results, in their order.
template <int HD>
__global__ __launch_bounds__(256) void k_cache_attend_merge(CacheAttnArgs a) {
  constexpr int E = HD / 64;
  const int lane = threadIdx.x & 63;
  const int64_t i = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int token = (int)(i / a.H), head = (int)(i % a.H);
  if (token >= clamped_cu(a, a.B)) return;
  const int b = owner_by_lanes(a.B, token, [&](int x) { return clamped_cu(a, x); });
  const int len = min(max(a.len[b], 0), a.max_pages << a.shift);
  const int used = min(a.splits, max(1, (len + a.chunk - 1) / a.chunk));
  const int64_t p = i * a.splits;
  float m = -INFINITY;
  for (int s = 0; s < used; ++s) m = fmaxf(m, a.part_ml[2 * (p + s)]);
  float sum = 0.f, x[E] = {};
  for (int s = 0; s < used; ++s) {
    const float ms = a.part_ml[2 * (p + s)], ls = a.part_ml[2 * (p + s) + 1];
    if (ms == -INFINITY && ls == 0.f) continue;  // no key of this range was seen
    const float c = ms == -INFINITY ? 1.f : fast_exp2(ms - m);
    sum += ls * c;
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] += a.part_o[(p + s) * HD + lane * E + e] * c;
  }
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  uint16_t* out = a.out + out_index(a, token, head, lane * E, HD);
  if constexpr (E == 2) *reinterpret_cast<uint32_t*>(out) = pack_bf16x2(x[0] * inv, x[1] * inv);
  else out[0] = (uint16_t)f32_to_bf16_bits(x[0] * inv);
}

CacheAttnPlan cache_attention_plan(int B, int rows, int H, int Hkv, int hd, int max_count, int max_len,
                                   int num_cus, size_t most_ws_floats) {
  const int G = H / Hkv;
  const int64_t most_rows = (int64_t)std::max(1, max_count) * G;
  CacheAttnPlan p{};
  p.tile_rows = most_rows <= 16 ? 16 : (most_rows <= 32 ? 32 : (most_rows <= 64 ? 64 : 128));
  p.tiles = (int)((int64_t)rows * G / p.tile_rows) + B;
  const int64_t units = (int64_t)p.tiles * Hkv;
  const int64_t want = p.tile_rows <= 32 ? 8 * (int64_t)num_cus : 2 * (int64_t)num_cus;
  const int64_t by_fill = std::max<int64_t>(1, want / std::max<int64_t>(1, units));
  const int64_t by_len = std::max(1, max_len / 256);
  const size_t per_split = (size_t)std::max(1, rows) * H * (2 + hd);
  p.splits = (int)std::min<int64_t>(std::min(by_fill, by_len), 64);
  p.splits = (int)std::max<size_t>(1, std::min<size_t>(p.splits, most_ws_floats / per_split));
  p.chunk = ((max_len + p.splits - 1) / p.splits + 63) / 64 * 64;
  if (p.chunk < 64) p.chunk = 64;
  p.ws_floats = p.splits > 1 ? per_split * p.splits : 0;
  return p;
}

hipError_t launch_cache_attention(CacheAttnArgs a, const CacheAttnPlan& p, int hd, float* ws, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  a.G = a.H / a.Hkv;
  a.tiles = p.tiles;
  a.splits = p.splits;
  a.chunk = p.chunk;
  if (p.splits > 1 && !ws) return hipErrorInvalidValue;
  a.part_o = ws;
  a.part_ml = ws ? ws + (size_t)a.rows * a.H * p.splits * hd : nullptr;
  const int64_t wgs = (int64_t)p.tiles * p.splits * a.Hkv;
  if (wgs > 0x7fffffffLL) return hipErrorInvalidValue;
  const dim3 grid((unsigned)wgs);
#define ATTEND(HD_)                                                                                              \
  do {                                                                                                           \
    if (p.tile_rows == 16) hipLaunchKernelGGL((k_cache_attend_rows<HD_, 1>), grid, dim3(256), 0, s, a);          \
    else if (p.tile_rows == 32) hipLaunchKernelGGL((k_cache_attend_rows<HD_, 2>), grid, dim3(256), 0, s, a);     \
    else if (p.tile_rows == 64) hipLaunchKernelGGL((k_cache_attend_tile<HD_, 1>), grid, dim3(256), 0, s, a);     \
    else hipLaunchKernelGGL((k_cache_attend_tile<HD_, 2>), grid, dim3(256), 0, s, a);                            \
    if (p.splits > 1) {                                                                                          \
      if (hipError_t e = hipGetLastError()) return e;                                                            \
      hipLaunchKernelGGL((k_cache_attend_merge<HD_>), dim3((unsigned)(((int64_t)a.rows * a.H + 3) / 4)),         \
                         dim3(256), 0, s, a);                                                                    \
    }                                                                                                            \
  } while (0)
  if (hd == 128) ATTEND(128);
  else if (hd == 64) ATTEND(64);
  else return hipErrorInvalidValue;
#undef ATTEND
  return hipGetLastError();
}

}  // namespace cora
