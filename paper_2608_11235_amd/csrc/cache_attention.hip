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
// token-major.
//
// Two kernels.  k_cache_attend_rows (16 or 32 rows a tile): bound by the stream of K and V, each of
// whose blocks is used by one wavefront, so they go from memory into the operand registers and the
// four wavefronts take every fourth group of 32 keys; their states merge through LDS.  The queries
// stay in LDS, which leaves registers for three workgroups a CU at 16 rows of 128.
// k_cache_attend_tile (64 or 128 rows): 64-key tiles through two LDS stages, loaded directly.
// Either runs over key ranges where the rows alone would not fill the card; the ranges' (max, sum, O)
// go to the workspace and k_cache_attend_merge folds them in order.
#include <algorithm>
#include <type_traits>

#include "cached.hpp"

namespace cora {

namespace {

constexpr float SLACK = 8.f;  // a reference maximum moves when a score passes it by 2^SLACK

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

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

__device__ __forceinline__ int clamped_len(const CacheAttnArgs& a, int b) { return min(max(a.len[b], 0), a.max_pages << a.shift); }

// Key ranges that a request is attended in, and the keys of each (the last has what is left): they
// follow from its own length, never from the others in the batch.
__device__ __forceinline__ int pieces(const CacheAttnArgs& a, int len) {
  return min(a.splits, max(1, (int)(((uint32_t)len + a.chunk - 1) / (uint32_t)a.chunk)));  // neither beyond 2^30
}
__device__ __forceinline__ int piece_keys(int len, int n) { return (int)(((uint32_t)(len + 31) / 32 + n - 1) / (uint32_t)n * 32); }

// What a workgroup works on: rows [row0, row0 + RT) of the (token, head) rows of request b and kv
// head kvh, keys [k0, k1) of its `len`.
struct Work {
  int b, kvh, split, row0, n_rows, cu, start, len, k0, k1;
};

// The first tile of a workgroup of k_cache_attend_tile; false when it has none.  Workgroups are
// numbered with the key range slowest and from the last one on: what only long requests have starts
// first, and the first range, which holds the short ones whole, fills the gaps at the end.  With
// `per_request` tiles a request (every request has about as many rows) a workgroup's place follows from
// its number, the kv head the fastest and the later tiles, which see more keys under the causal mask,
// before the earlier ones (4 x 2048 tokens, the kernel's case below: 351 us in either order).  Else (a prompt beside single tokens) tile t belongs to
// the request b with base_b <= t < base_(b+1), base_b = cu_b G / RT + b, which leaves each request at
// least as many tiles as it fills and needs no pass over the lengths, and an XCD takes a range of kv
// heads and tiles, whose keys its L2 then holds.
template <int RT>
__device__ __forceinline__ bool first_tile(const CacheAttnArgs& a, Work& w) {
  int li = blockIdx.x;
  if (a.per_request > 0) {
    w.kvh = li % a.Hkv;
    li /= a.Hkv;
    w.b = li % a.B;
    li /= a.B;
    w.row0 = (a.per_request - 1 - li % a.per_request) * RT;
    w.split = a.splits - 1 - li / a.per_request;
  } else {
    const int n = a.tiles * a.Hkv;
    w.split = a.splits - 1 - li / n;
    li = xcd_remap(li % n, n);
    const int t = a.tiles - 1 - li % a.tiles;  // later tiles first here too
    w.kvh = li / a.tiles;
    w.b = uniform(owner_by_lanes(a.B, t, [&](int b) { return (int)((int64_t)clamped_cu(a, b) * a.G / RT) + b; }));
    w.row0 = (t - (int)((int64_t)uniform(clamped_cu(a, w.b)) * a.G / RT) - w.b) * RT;
  }
  w.cu = uniform(clamped_cu(a, w.b));
  w.n_rows = (uniform(clamped_cu(a, w.b + 1)) - w.cu) * a.G;
  if (w.row0 < 0 || w.row0 >= w.n_rows) return false;  // below 0: a cu that starts late or does not ascend
  w.start = uniform(a.start[w.b]);
  w.len = uniform(clamped_len(a, w.b));
  const int n = pieces(a, w.len);
  if (w.split >= n) return false;
  const int each = (piece_keys(w.len, n) + 63) / 64 * 64;
  w.k0 = w.split * each;
  w.k1 = min(w.len, w.k0 + each);
  return true;
}

// The next one: a request with more rows than its tiles were made for takes several turns.
template <int RT>
__device__ __forceinline__ bool next_tile(const CacheAttnArgs& a, Work& w) {
  if (a.per_request == 0) return false;
  w.row0 += a.per_request * RT;
  return w.row0 < w.n_rows;
}

// keys that row `row` sees; rows behind the last one, whose results nobody reads, as many as it
__device__ __forceinline__ int limit_of(const CacheAttnArgs& a, const Work& w, int row) {
  row = min(row, w.n_rows - 1);
  if (!a.causal) return w.len;
  return min((int64_t)w.len, max((int64_t)w.start + row / a.G + 1, (int64_t)0));
}

// Where the 32-key groups of one request and kv head lie.  The block table is read by scalar loads:
// they are counted apart from the vector loads in flight, so that a page can be looked up between
// those of K and V without waiting for them, and an entry is read a group before its use.
template <int HD>
struct Groups {
  const __attribute__((address_space(4))) int32_t* table;
  int shift5, mask5, n_pages;  // log2 of 32-key groups a page, that less one
  int64_t page_bytes, head_bytes;
  __device__ __forceinline__ Groups(const CacheAttnArgs& a, const Work& w)
      : table((const __attribute__((address_space(4))) int32_t*)(uintptr_t)(a.table + (int64_t)w.b * a.max_pages)),
        shift5(a.shift - 5), mask5((1 << (a.shift - 5)) - 1), n_pages(a.n_pages),
        page_bytes((int64_t)a.Hkv * HD * 2 << a.shift), head_bytes((int64_t)w.kvh * HD * 2 << a.shift) {}
  __device__ __forceinline__ int entry(int grp) const { return table[uniform(grp >> shift5)]; }
  // byte offset in the pool of a group of that entry; a bad entry reads page 0, never past the pool
  __device__ __forceinline__ int64_t offset(int entry, int grp) const {
    const int page = (unsigned)entry < (unsigned)n_pages ? entry : 0;
    return page * page_bytes + head_bytes + (int64_t)(grp & mask5) * (32 * HD * 2);
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

// Moves the reference of the scores st[rb] of a query (the maximum over its four lane groups) and
// rescales, where one of them needs it, then turns the scores into terms.
template <int RB, int NB, int ND>
__device__ __forceinline__ void soften(f32x4_t (&st)[RB][NB], float scale_log2, float (&m_ref)[RB], float (&m_use)[RB],
                                       float (&l)[RB], f32x4_t (&o)[RB][ND]) {
  float lmax[RB];
  bool moves = false;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    lmax[rb] = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
      for (int i = 0; i < 4; ++i) lmax[rb] = fmaxf(lmax[rb], st[rb][kb][i]);
    moves |= lmax[rb] * scale_log2 > m_ref[rb] + SLACK;
  }
  if (__any(moves)) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float tmax = fmaxf(lmax[rb], __shfl_xor(lmax[rb], 16, 64));
      tmax = fmaxf(tmax, __shfl_xor(tmax, 32, 64));
      const float tm = tmax * scale_log2;
      if (tm > m_ref[rb] + SLACK) {  // never while no key was seen and none is
        const float alpha = fast_exp2(m_ref[rb] - tm);
        m_ref[rb] = m_use[rb] = tm;
        l[rb] *= alpha;
#pragma unroll
        for (int d = 0; d < ND; ++d) o[rb][d] *= alpha;
      }
    }
  }
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p = fast_exp2(fmaf(st[rb][kb][i], scale_log2, -m_use[rb]));  // m_use 0 until a key is seen
        st[rb][kb][i] = p;
        l[rb] += p;
      }
}

// The terms of eight keys as the second product's operand.  V is bf16 and the matrix instruction takes
// both operands in one type, so a term is rounded by up to 2^-8 of it, while its sum l adds the fp32
// value.  Outputs are off from 64 bits by 2.0e-3 to 2.3e-3 of their norm, 1.7e-3 of which is their own
// rounding (what fp32 terms leave).  Terms in two bf16 parts would double the second product.
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

// The result of RB x 16 rows from row `first` of the workgroup on, or their part of it.
template <int HD, int RB>
__device__ __forceinline__ void store_rows(const CacheAttnArgs& a, const Work& w, int first, const float (&m_ref)[RB],
                                           const float (&l)[RB], const f32x4_t (&o)[RB][HD / 16]) {
  constexpr int ND = HD / 16;
  const int lane = threadIdx.x & 63, g = lane >> 4, r16 = lane & 15;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    float s = l[rb];
    s += __shfl_xor(s, 16, 64);
    s += __shfl_xor(s, 32, 64);
    const int row = w.row0 + first + rb * 16 + r16;
    if (row >= w.n_rows) continue;
    const int token = w.cu + row / a.G, head = w.kvh * a.G + row % a.G;
    if (pieces(a, w.len) == 1) {  // the whole of the request's keys
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

}  // namespace

template <int HD, int RB>
struct RowsShared {
  u32x4_t q[RB * (HD / 32)][64];
  f32x4_t o[2][RB * (HD / 16)][64];
  float m[2][RB][64], l[2][RB][64];
};

template <int HD, int RB>
__device__ __forceinline__ void attend_rows(const CacheAttnArgs& a, const Work& w, RowsShared<HD, RB>& sh) {
  constexpr int NK = HD / 32, ND = HD / 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, r16 = lane & 15;

  int lim[RB], most = 0;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = w.row0 + rb * 16 + r16;
    if (wave == rb) {
      bf16x8_t qf[NK];
      load_q<HD>(a, w, row, qf);
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) sh.q[rb * NK + kk][lane] = __builtin_bit_cast(u32x4_t, qf[kk]);
    }
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
  __syncthreads();
  const Groups<HD> groups(a, w);
  // K and V are read once, past the caches' regular places (non-temporal): 46 us against 55 for the
  // ragged tokens, 22.6 against 25.2 for the blocks.
  // Per group: V's loads go out first, S^T waits for K's, which were sent a group ago; then the next
  // K's loads take the registers that S^T has read, and O^T waits for V's.
  u32x4_t kf[2 * NK], vf[ND];
  auto load_k = [&](int64_t at) {
    const u32x4_t* p = reinterpret_cast<const u32x4_t*>(reinterpret_cast<const char*>(a.k) + at) + lane;
#pragma unroll
    for (int i = 0; i < 2 * NK; ++i) kf[i] = __builtin_nontemporal_load(p + i * 64);
  };
  int grp = g0 + wave;
  int64_t here = 0;
  int entry = 0;
  if (grp < g1) {
    here = groups.offset(groups.entry(grp), grp);
    load_k(here);
    entry = groups.entry(min(grp + 4, g1 - 1));
  }
  for (; grp < g1; grp += 4) {
    // the last time once more the same: no branch, so that V's waits count on K's loads
    const int next = grp + 4 < g1 ? grp + 4 : grp;
    const int64_t ahead = groups.offset(entry, next);
    entry = groups.entry(min(grp + 8, g1 - 1));
    {
      const u32x4_t* p = reinterpret_cast<const u32x4_t*>(reinterpret_cast<const char*>(a.v) + here) + lane;
#pragma unroll
      for (int i = 0; i < ND; ++i) vf[i] = __builtin_nontemporal_load(p + i * 64);
    }
    __builtin_amdgcn_sched_barrier(0);
    f32x4_t st[RB][2];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        st[rb][kb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < NK; ++kk)
          st[rb][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kf[kb * NK + kk]), as_bf16x8(sh.q[rb * NK + kk][lane]), st[rb][kb], 0, 0, 0);
      }
    __builtin_amdgcn_sched_barrier(0);
    load_k(ahead);
    __builtin_amdgcn_sched_barrier(0);
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
    }
    soften<RB, 2, ND>(st, a.scale_log2, m_ref, m_use, l, o);
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
        add_non_finite<ND>(reinterpret_cast<const uint16_t*>(reinterpret_cast<const char*>(a.v) + here), st[rb][0], st[rb][1], min(lim[rb], w.k1) - grp * 32, o[rb]);
    }
    here = ahead;
  }

  // wavefronts 2 and 3 hand their states to 0 and 1, and 1 to 0, lane by lane
#pragma unroll
  for (int from = 2; from > 0; from >>= 1) {
    if (wave >= from && wave < 2 * from) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        sh.m[wave - from][rb][lane] = m_ref[rb];
        sh.l[wave - from][rb][lane] = l[rb];
#pragma unroll
        for (int d = 0; d < ND; ++d) sh.o[wave - from][rb * ND + d][lane] = o[rb][d];
      }
    }
    __syncthreads();
    if (wave < from) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const float m1 = sh.m[wave][rb][lane], m = fmaxf(m_ref[rb], m1);
        // a state that saw no key is (-inf, 0, 0), or holds a NaN that has to stay one
        const float c0 = m_ref[rb] == m ? 1.f : fast_exp2(m_ref[rb] - m), c1 = m1 == m ? 1.f : fast_exp2(m1 - m);
        m_ref[rb] = m;
        l[rb] = l[rb] * c0 + sh.l[wave][rb][lane] * c1;
#pragma unroll
        for (int d = 0; d < ND; ++d) o[rb][d] = o[rb][d] * c0 + sh.o[wave][rb * ND + d][lane] * c1;
      }
    }
    __syncthreads();  // the LDS is free again
  }
  if (wave == 0) store_rows<HD, RB>(a, w, 0, m_ref, l, o);
}

// The work is a list of (request, key range, tile, kv head).  Every workgroup adds up the requests'
// counts and takes every gridDim'th entry: the list holds no empty ones, where a grid over the ranges
// of the longest request took 27 us to start for 64 ragged tokens, half of it for nothing.
template <int HD, int RB>
__global__ __launch_bounds__(256, 2) void k_cache_attend_rows(CacheAttnArgs a) {
  constexpr int RT = RB * 16;
  extern __shared__ uint32_t first[];  // [B + 1]: pieces of the requests before
  __shared__ uint32_t part[4];
  __shared__ int near[4][256];  // cu, rows, start and len of the first requests, read once
  __shared__ RowsShared<HD, RB> sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  uint32_t carry = 0;
  for (int b0 = 0; b0 < a.B; b0 += 256) {
    const int b = b0 + tid;
    uint32_t n = 0;
    if (b < a.B) {
      const int cu = clamped_cu(a, b), rows = (clamped_cu(a, b + 1) - cu) * a.G, len = clamped_len(a, b);
      if (b0 == 0) {
        near[0][tid] = cu;
        near[1][tid] = rows;
        near[2][tid] = a.start[b];
        near[3][tid] = len;
      }
      if (rows > 0)
        n = (uint32_t)((rows + RT - 1) / RT) * (uint32_t)a.Hkv * (uint32_t)pieces(a, len);
    }
    uint32_t s = wave_scan(n);
    if (lane == 63) part[wave] = s;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i < wave) s += part[i];
    }
    if (b < a.B) first[b] = carry + s - n;
    carry += part[0] + part[1] + part[2] + part[3];
    __syncthreads();
  }
  const uint32_t total = uniform(carry);
  for (uint32_t i = blockIdx.x; i < total; i += gridDim.x) {
    Work w;
    w.b = uniform(owner_by_lanes(a.B, (int)i, [&](int b) { return (int)first[b]; }));
    if (w.b < 256) {
      w.cu = uniform(near[0][w.b]);
      w.n_rows = uniform(near[1][w.b]);
      w.start = uniform(near[2][w.b]);
      w.len = uniform(near[3][w.b]);
    } else {
      w.cu = uniform(clamped_cu(a, w.b));
      w.n_rows = (uniform(clamped_cu(a, w.b + 1)) - w.cu) * a.G;
      w.start = uniform(a.start[w.b]);
      w.len = uniform(clamped_len(a, w.b));
    }
    uint32_t k = i - uniform(first[w.b]);
    w.kvh = k % a.Hkv;
    k /= a.Hkv;
    const int n = pieces(a, w.len);
    const uint32_t tiles = max(1, (w.n_rows + RT - 1) / RT);
    w.row0 = k % tiles * RT;
    w.split = k / tiles;
    if (w.n_rows <= 0 || (unsigned)w.split >= (unsigned)n) continue;  // cu that does not ascend
    const int each = piece_keys(w.len, n);
    w.k0 = w.split * each;
    w.k1 = min(w.len, w.k0 + each);
    attend_rows<HD, RB>(a, w, sh);
  }
}

// Bound by the products and, nearly as much, by the LDS reads that feed them (a fragment of K or V
// serves RB x 16 rows) and the exponentials: 4 x 2048 tokens of 28 heads of 128 behind 2048 others,
// causal, 345 to 362 us from card to card, 1.00 to 1.05 PFLOP/s.  Tiles that no row's limit cuts take a path without masks or branches
// but one, for a moved reference.  Tried at RB = 2: 32-key tiles in 2 to 4 stages, two or three
// workgroups a CU (366 us); RB = 3 (348 us, and 54 against 44 us where 2 x 1024 tokens of 32 heads
// leave fewer workgroups than places); RB = 4 on one wavefront a SIMD (544 us).
constexpr int TILE_KEYS = 64, TILE_STAGES = 2;

template <int HD, int RB>
__device__ __forceinline__ void attend_tile(const CacheAttnArgs& a, const Work& w, unsigned char* lds) {
  constexpr int RT = 64 * RB, NK = HD / 32, ND = HD / 16, KT = TILE_KEYS, NS = TILE_STAGES;
  constexpr int GB = 32 * HD * 2;           // bytes of K (or V) of a 32-key group
  constexpr int NG = KT / 32, VAT = NG * GB, STAGE = 2 * NG * GB;  // a stage: groups of K, then of V
  constexpr int NL = NG * ND / 4;           // blocks of K (and of V) that a wavefront loads
  typedef __attribute__((address_space(3))) void* lds_ptr_t;
  typedef const __attribute__((address_space(1))) void* global_ptr_t;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int g = lane >> 4, r16 = lane & 15;

  bf16x8_t qf[RB][NK];
  int lim[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = w.row0 + (wave * RB + rb) * 16 + r16;
    load_q<HD>(a, w, row, qf[rb]);
    lim[rb] = min(limit_of(a, w, row), w.k1);
  }
  // keys that every row of the wavefront sees, that some row of it does, and that some row of the
  // workgroup does
  const int first = w.row0 + wave * RB * 16, last = min(first + RB * 16, w.n_rows) - 1;
  const int wave_full = first < w.n_rows ? min(w.k1, limit_of(a, w, first)) : 0;
  const int wave_end = first < w.n_rows ? min(w.k1, limit_of(a, w, last)) : 0;
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
  const Groups<HD> groups(a, w);
  // A wavefront loads its share of a tile's blocks; the entry of the tile after is read meanwhile.
  // Behind the last key the last group is loaded once more, so that each tile counts the same loads.
  const int last_grp = max((w.len + 31) / 32 - 1, 0), sub = wave * NG / 4, part = wave - sub * (4 / NG);
  int entry = t0 < t1 ? groups.entry(min(NG * t0 + sub, last_grp)) : 0;
  auto fetch = [&](int t, int buf) {
    const int grp = min(NG * t + sub, last_grp);
    const int64_t at = groups.offset(entry, grp) + part * (NL * 1024);
    entry = groups.entry(min(NG * (t + 1) + sub, last_grp));
    const char* k = reinterpret_cast<const char*>(a.k) + at + lane * 16;
    const char* v = reinterpret_cast<const char*>(a.v) + at + lane * 16;
    unsigned char* dst = lds + buf * STAGE + wave * (NL * 1024);
#pragma unroll
    for (int i = 0; i < NL; ++i)
      __builtin_amdgcn_global_load_lds((global_ptr_t)(k + i * 1024), (lds_ptr_t)(dst + i * 1024), 16, 0, 0);
#pragma unroll
    for (int i = 0; i < NL; ++i)
      __builtin_amdgcn_global_load_lds((global_ptr_t)(v + i * 1024), (lds_ptr_t)(dst + VAT + i * 1024), 16, 0, 0);
  };
  auto fold = [&](const unsigned char* stage, int key0, auto edge) {
    constexpr bool EDGE = decltype(edge)::value;
    const unsigned char *kl = stage + lane * 16, *vl = kl + VAT;
    // the scheduler's strategy 1 mixes LDS reads and products best: 344 us against 354 (0 and 2: 348, 357)
    __builtin_amdgcn_iglp_opt(1);
    f32x4_t st[RB][2 * NG];
#pragma unroll
    for (int kb = 0; kb < 2 * NG; ++kb) {
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
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      if constexpr (EDGE) {
        const int n = lim[rb] - key0 - 8 * g;  // the lane's terms are keys 32 (kb / 2) + 4 (kb % 2) + i
#pragma unroll
        for (int kb = 0; kb < 2 * NG; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (32 * (kb >> 1) + 4 * (kb & 1) + i >= n) st[rb][kb][i] = -INFINITY;
      }
    }
    soften<RB, 2 * NG, ND>(st, a.scale_log2, m_ref, m_use, l, o);
#pragma unroll
    for (int ks = 0; ks < NG; ++ks) {
      bool bad = false;
      bf16x8_t p[RB];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) p[rb] = terms_operand(st[rb][2 * ks], st[rb][2 * ks + 1]);
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        u32x4_t v = *reinterpret_cast<const u32x4_t*>(vl + (ks * ND + d) * 1024);
        if constexpr (EDGE) {  // slots behind the last key may hold anything
          v = keep_keys(v, w.len - key0 - 32 * ks - 8 * g);
          if (a.causal) v = finite_only(v, bad);
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
          o[rb][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(v), p[rb], o[rb][d], 0, 0, 0);
      }
      if constexpr (EDGE) {
        if (__any(bad)) {
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
            add_non_finite<ND>(reinterpret_cast<const uint16_t*>(stage + VAT + ks * GB), st[rb][2 * ks],
                               st[rb][2 * ks + 1], min(lim[rb], w.k1) - key0 - 32 * ks, o[rb]);
        }
      }
    }
  };
  if (t0 < t1) {
#pragma unroll
    for (int i = 0; i < NS - 1; ++i) fetch(t0 + i, i);
  }
  int buf = 0;
  for (int t = t0; t < t1; ++t) {
    // tile t has landed, and every wavefront is done with the stage that tile t + NS - 1 goes to
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NS - 2) * 2 * NL) : "memory");
    __syncthreads();
    fetch(t + NS - 1, buf ? buf - 1 : NS - 1);
    if (t * KT < wave_end) {
      if (t * KT + KT <= wave_full) fold(lds + buf * STAGE, t * KT, std::false_type{});
      else fold(lds + buf * STAGE, t * KT, std::true_type{});
    }
    buf = buf + 1 < NS ? buf + 1 : 0;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // loads behind the last tile

  store_rows<HD, RB>(a, w, wave * RB * 16, m_ref, l, o);
}

template <int HD, int RB>
__global__ __launch_bounds__(256, 2) void k_cache_attend_tile(CacheAttnArgs a) {
  __shared__ __attribute__((aligned(16))) unsigned char lds[TILE_STAGES * TILE_KEYS * HD * 4];
  Work w;
  if (!first_tile<64 * RB>(a, w)) return;
  do {
    attend_tile<HD, RB>(a, w, lds);
    __syncthreads();  // the LDS is free again
  } while (next_tile<64 * RB>(a, w));
}

// One wavefront per (row, head): the key ranges' partial results, in their order.
template <int HD>
__global__ __launch_bounds__(256) void k_cache_attend_merge(CacheAttnArgs a) {
  constexpr int E = HD / 64;
  const int lane = threadIdx.x & 63;
  const uint32_t i = blockIdx.x * 4 + uniform(threadIdx.x >> 6);  // rows H is no more than 2^30
  const int token = (int)(i / (uint32_t)a.H), head = (int)(i % (uint32_t)a.H);
  if (token >= clamped_cu(a, a.B)) return;
  const int b = owner_by_lanes(a.B, token, [&](int x) { return clamped_cu(a, x); });
  if (token < clamped_cu(a, b) || token >= clamped_cu(a, b + 1)) return;  // no request's
  const int len = clamped_len(a, b);
  const int used = pieces(a, len);
  if (used == 1) return;  // written already
  const int64_t p = (int64_t)i * a.splits;
  float t[8][E];  // eight ranges' loads at a time
  auto load = [&](int s0) {
#pragma unroll
    for (int u = 0; u < 8; ++u)
#pragma unroll
      for (int e = 0; e < E; ++e) t[u][e] = a.part_o[(p + min(s0 + u, used - 1)) * HD + lane * E + e];
  };
  load(0);
  // a lane holds one range's maximum and sum; E x 4 B of a lane's O a range
  const bool has = lane < used;  // no more than 64
  const float ml = has ? a.part_ml[2 * (p + lane)] : -INFINITY, l = has ? a.part_ml[2 * (p + lane) + 1] : 0.f;
  float m = ml;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  const float c = ml == m ? 1.f : fast_exp2(ml - m);  // a range without a key is (-inf, 0, 0)
  float sum = l * c, x[E] = {};
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o, 64);
  for (int s0 = 0; s0 < used; s0 += 8) {
    if (s0 > 0) load(s0);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (s0 + u >= used) continue;
      const float cs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(c), s0 + u));
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] += t[u][e] * cs;
    }
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
  p.tiles = (int)((int64_t)rows * G / p.tile_rows) + B;  // no fewer than there are
  const int64_t each = (most_rows + p.tile_rows - 1) / p.tile_rows;
  if (p.tile_rows > 32 && each * B <= p.tiles) {
    p.per_request = (int)each;
    p.tiles = (int)each * B;
  }
  const int64_t units = (int64_t)p.tiles * Hkv;
  if (p.tile_rows <= 32) {
    // Requests of up to 1.25 ranges stay whole.  1280 keys where the units (tiles and kv heads) could
    // fill the card whole, 640 where they could not, 320 where they are very few (heads of 128):
    //   64 ragged tokens of 4 kv heads up to 8192 long     44 us at 1280, 47 at 640, 50 at 320
    //   32 blocks of 8 kv heads up to 1280 long            22 us whole, 28 in two
    //   256 tokens of 8 kv heads up to 1024 long           68 us whole, 72 in two
    //   16 tokens of 8 kv heads up to 4096 long            21 us at 1280, 18 at 640, 19 at 320
    //   one token of 4 kv heads, 8192 long                 19 us at 1280, 15 at 640, 14 at 320
    //   one block of 32 kv heads, 1280 long                18 us whole, 15.6 at 640, 14 at 320
    // No more than 32 ranges unless the units are very few, since each is written and read once more
    // (one token of 8 kv heads, 32768 long: 28 us in 32 ranges, 31 in 64).
    const int keys = units >= num_cus ? 1280 : (8 * units > num_cus ? 640 : 320);
    const int64_t cap = std::min<int64_t>(64, std::max<int64_t>(32, num_cus / units));
    const int64_t n = max_len <= keys + keys / 4 ? 1 : (max_len + (int64_t)keys - 1) / keys;
    p.splits = (int)std::min(n, cap);
  } else {
    const int64_t want = std::max<int64_t>(1, 2 * (int64_t)num_cus / units), by_len = std::max(1, max_len / 256);
    p.splits = (int)std::min<int64_t>(std::min(want, by_len), 64);
  }
  const size_t per_split = (size_t)std::max(1, rows) * H * (2 + hd);
  // the list of work is counted in 31 bits, a grid over all tiles and the merge's over all rows and
  // heads in workgroups
  const int64_t list = p.tile_rows <= 32 ? 0x7fffffffLL : most_workgroups(256);
  int64_t most = std::min<int64_t>(most_ws_floats / per_split, list / units);
  if (((int64_t)rows * H + 3) / 4 > most_workgroups(256)) most = 1;
  p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(p.splits, most));
  p.chunk = std::max(64, ((max_len + p.splits - 1) / p.splits + 63) / 64 * 64);
  p.workgroups = (int)std::min<int64_t>(p.tile_rows <= 32 ? 6 * num_cus : 0x7fffffffLL, units * p.splits);
  p.ws_floats = p.splits > 1 ? per_split * p.splits : 0;
  return p;
}

hipError_t launch_cache_attention(CacheAttnArgs a, const CacheAttnPlan& p, int hd, float* ws, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  a.G = a.H / a.Hkv;
  a.tiles = p.tiles;
  a.per_request = p.per_request;
  a.splits = p.splits;
  a.chunk = p.chunk;
  if (p.splits > 1 && !ws) return hipErrorInvalidValue;
  a.part_o = ws;
  a.part_ml = ws ? ws + (size_t)a.rows * a.H * p.splits * hd : nullptr;
  if (p.workgroups > most_workgroups(256)) return hipErrorInvalidValue;
  const dim3 grid((unsigned)p.workgroups);
  const size_t lds = (size_t)(a.B + 1) * 4;
#define ATTEND(HD_)                                                                                              \
  do {                                                                                                           \
    if (p.tile_rows == 16) hipLaunchKernelGGL((k_cache_attend_rows<HD_, 1>), grid, dim3(256), lds, s, a);        \
    else if (p.tile_rows == 32) hipLaunchKernelGGL((k_cache_attend_rows<HD_, 2>), grid, dim3(256), lds, s, a);   \
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
