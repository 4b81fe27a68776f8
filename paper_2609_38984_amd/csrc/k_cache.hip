// Attention of a chunk of new tokens to a paged cache: grouped K/V heads, causal, with a
// window, or over the whole chunk.
//
// The rows of a tile are (query token, head of the group) pairs of one sequence and one
// K/V head.  bf16: S^T = K Q^T and O^T = V^T P^T on 32x32x16 MFMAs, one row per lane
// (lane & 31) and the keys in the accumulator registers; softmax in one pass with a running
// maximum (base 2, float32).  K and V tiles of 64 keys go global -> LDS by buffer loads of 8
// keys each: a page holds a multiple of 8, so each such slab has one base and its descriptor
// ends with the sequence's last key; what lies behind it, and what has no page, stores
// zeros.  Which keys a row sees is a 64-bit mask per lane, formed only for tiles that
// some row sees in part.
#include "gemm_common.h"
#include "paged.h"

#include <algorithm>
#include <cfloat>

namespace swam {

typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16;

constexpr int CA_BK = 64;                      // keys per tile
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// How the keys are split and where partial results go: slot i holds slot_rows rows of
// [head_dim] sums, and (maximum, sum) for each.
struct Split {
  float* o;
  float* ml;
  int* plan;          // [0]: tiles of a slice, written by workgroup 0 for the joining pass
  int budget;         // slices beyond the first of every tile, 0: keys are not split
  int slot_rows;
};

// Sequence s as the kernels see it.
struct Seq {
  int a, n;           // first row, tokens of its chunk
  int old, total;     // tokens before the chunk, keys
  int qt, nk;         // row tiles, key tiles that a row tile reads at most
};
template <int BQ, int BK>
__device__ __forceinline__ Seq seq_at(const CacheArgs& c, int group, int s) {
  Seq q{};
  if (s >= c.pg.n_seqs) return q;
  int e;
  chunk_of(c.pg, s, c.n_q, q.a, e);
  q.n = e - q.a;
  q.old = held(c.pg, s);
  q.total = (int)min((int64_t)q.old + q.n, (int64_t)c.pg.max_pages << c.pg.lg_page);
  q.qt = (q.n * group + BQ - 1) / BQ;
  q.nk = (q.total + BK - 1) / BK;
  // a causal window bounds what a row tile reads: its own tokens and the window before them
  if (c.window && c.causal) q.nk = min(q.nk, (min(c.window, 1 << 30) + BQ / group + 1) / BK + 2);
  return q;
}

template <typename T>
__device__ __forceinline__ T wave_scan(T v) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const T u = __shfl_up(v, s);
    if ((int)(threadIdx.x & 63) >= s) v += u;
  }
  return v;
}

// Tiles of a slice, from the key tiles of all row tiles (`all`, over all K/V heads) and the most of
// one: modelled time of a workgroup by itself (`lone` ns a tile) and of several that
// share a CU, and of the pass that joins the slices.
template <int D>
__device__ __forceinline__ int slice_tiles(int64_t all, int most, const Split& sp) {
  if (sp.budget == 0) return max(most, 1);
  const float lone = D == 64 ? 1.2f : 1.6f, share = (D == 64 ? 0.64f : 1.0f) / 256.0f * (float)all;
  const int least = max((int)((all + sp.budget - 1) / sp.budget), 2);
  int best = max(most, 1);
  float best_us = fmaxf(lone * (float)most, share);
  for (int k = 1; k < 16; ++k) {
    const int t = (most + (1 << k) - 1) >> k;
    if (t < least) break;
    const float us = fmaxf(lone * (float)t, share) + 4.5f +
                     2.0f * (float)all / (float)t * (float)sp.slot_rows * (D + 2) * (4.0f / 3.0e6f);
    if (us < best_us) { best_us = us; best = t; }
  }
  return best;
}

// What a workgroup does: slice y of ch of the keys of row tile qi of sequence s, its
// partial results in `slot` (units before it in split sequences).
struct Work {
  Seq q;
  int s, qi, y, ch, slot;
};
// The lanes hold the sequences in order, `per` to a lane; three passes over them find the
// slices' length, the units in front of each, and the one that holds `unit`.
template <int D, int BQ, int BK>
__device__ __forceinline__ bool work_at(const CacheArgs& c, const Split& sp, int unit, Work& w) {
  const int lane = threadIdx.x & 63, group = c.heads / c.pg.kv_heads;
  const int per = (c.pg.n_seqs + 63) >> 6;
  const Seq first = seq_at<BQ, BK>(c, group, lane * per);
  int64_t all = 0;
  int most = 0;
  for (int i = 0; i < per; ++i) {
    const Seq q = i == 0 ? first : seq_at<BQ, BK>(c, group, lane * per + i);
    all += (int64_t)q.qt * q.nk;
    most = max(most, q.nk);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    all += __shfl_xor(all, o);
    most = max(most, __shfl_xor(most, o));
  }
  const int tiles = slice_tiles<D>(all * c.pg.kv_heads, most, sp);
  if (blockIdx.x == 0 && threadIdx.x == 0 && sp.budget) sp.plan[0] = tiles < most ? tiles : 0;
  int units = 0, split = 0;
  for (int i = 0; i < per; ++i) {
    const Seq q = i == 0 ? first : seq_at<BQ, BK>(c, group, lane * per + i);
    const int ch = max((q.nk + tiles - 1) / tiles, 1);
    units += q.qt * ch;
    split += ch > 1 ? q.qt * ch : 0;
  }
  int at = wave_scan(units), slot = wave_scan(split);
  const uint64_t past = __ballot(at > unit);
  if (past == 0) return false;
  at -= units;
  slot -= split;
  w = Work{};
  for (int i = 0; i < per; ++i) {
    const Seq q = i == 0 ? first : seq_at<BQ, BK>(c, group, lane * per + i);
    const int ch = max((q.nk + tiles - 1) / tiles, 1), n = q.qt * ch;
    if (unit >= at && unit < at + n) {
      w.q = q;
      w.s = lane * per + i;
      w.ch = ch;
      // the last rows of a causal chunk see most: they come first
      w.qi = q.qt - 1 - (unit - at) / ch;
      w.y = (unit - at) % ch;
      w.slot = slot + unit - at;
    }
    at += n;
    slot += ch > 1 ? n : 0;
  }
  const int b = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)past) - 1);
  auto bcast = [&](int& v) { v = __builtin_amdgcn_readlane(v, b); };
  bcast(w.q.a); bcast(w.q.n); bcast(w.q.old); bcast(w.q.total); bcast(w.q.qt); bcast(w.q.nk);
  bcast(w.s); bcast(w.qi); bcast(w.y); bcast(w.ch); bcast(w.slot);
  return true;
}

// the keys [lo, hi) that rows [r0, r1] of a sequence see, as far as one range holds them
__device__ __forceinline__ void key_range(const CacheArgs& c, const Seq& q, int group, int r0, int r1, int& lo, int& hi) {
  hi = c.causal ? min(q.old + r1 / group + 1, q.total) : q.total;
  lo = c.window ? min(max(q.old + r0 / group - c.window + 1, 0), hi) : 0;
}

// tiles [t0, t1) of slice y of ch
__device__ __forceinline__ void slice_of(int lo, int hi, int bk, int y, int ch, int& t0, int& t1) {
  const int a = lo / bk, n = (hi + bk - 1) / bk - a;
  t0 = a + (int)((int64_t)n * y / ch);
  t1 = a + (int)((int64_t)n * (y + 1) / ch);
}

template <int D>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 64 ? 4 : 2, 8)))
cache_bf16(const CacheArgs c, const Split sp, int unit0) {
  constexpr int H2 = D / 64;                     // 128-byte halves of a head's row
  constexpr int NW = 4, BQ = 32 * NW;
  constexpr int TILE = CA_BK * 8 * H2;           // uint4 of a K or V tile
  __shared__ uint4 kv[2][2][TILE];               // [stage][K | V][half][key][8 chunks]
  const int group = c.heads / c.pg.kv_heads;
  // neighbouring workgroups take the K/V heads in turn: with a multiple of 8 of them a
  // head stays on one XCD
  const int hk = blockIdx.x % c.pg.kv_heads;
  Work w;
  if (!work_at<D, BQ, CA_BK>(c, sp, unit0 + blockIdx.x / c.pg.kv_heads, w)) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 5, r31 = lane & 31;
  const int rows = w.q.n * group, r0 = w.qi * BQ, total = w.q.total;
  int lo, hi, t0, t1;
  key_range(c, w.q, group, r0, min(r0 + BQ, rows) - 1, lo, hi);
  slice_of(lo, hi, CA_BK, w.y, w.ch, t0, t1);
  // the keys that all rows of this wave see lie in [low_last, lim_first], those that any
  // sees in [low_first, lim_last]; a wave behind the last row sees none
  const int wr = r0 + wave * 32;
  int lim_first = total - 1, lim_last = wr < rows ? total - 1 : -1, low_first = 0, low_last = 0;
  const int tok_first = min(wr, rows - 1) / group, tok_last = min(wr + 31, rows - 1) / group;
  if (c.causal) {
    lim_first = min(lim_first, w.q.old + tok_first);
    lim_last = min(lim_last, w.q.old + tok_last);
  }
  if (c.window) {
    low_first = max(w.q.old + tok_first - c.window + 1, 0);
    low_last = max(w.q.old + tok_last - c.window + 1, 0);
  }
  bf16x8 qf[D / 16];
  int lim = total - 1, low = 0;                  // of this lane's row
  {
    const int rr = min(wr + r31, rows - 1);
    const int64_t tok = w.q.a + rr / group;
    const int head = hk * group + rr % group;
    if (c.causal) lim = min(lim, w.q.old + rr / group);
    if (c.window) low = max(w.q.old + rr / group - c.window + 1, 0);
    const bf16_t* qp = (const bf16_t*)c.q + tok * c.q_ld + head * D;
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
      qf[s] = __builtin_bit_cast(bf16x8, *(const uint4*)(qp + 8 * (2 * s + g)));
  }
  const int32_t* table = c.pg.table + w.s * c.pg.table_ld;

  // the page of this lane's key of tile t, -1: none
  auto page_at = [&](int t) -> int {
    const int key = t * CA_BK + (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
    if (t >= t1 || key >= total) return -1;
    const int p = table[key >> c.pg.lg_page];
    return p >= 0 && p < c.pg.n_pages ? p : -1;
  };
  const int lrow = lane >> 3;
  constexpr int SL = 8 * H2 / NW;                // 8-key slabs of a tile that a wave stages
  int off_k[2], off_v[2];                        // of even and odd slabs
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int r = j * 8 + lrow, col = 8 * ((lane & 7) ^ lds_swz(r));
    off_k[j] = (lrow * (int)c.pg.k_token + col) * 2;
    off_v[j] = (lrow * (int)c.pg.v_token + col) * 2;
  }
  // K and V of tile t into LDS, `pages` of its keys in the lanes
  auto issue = [&](uint4 (&to)[2][TILE], int t, int pages) {
#pragma unroll
    for (int j = 0; j < SL; ++j) {
      const int slab = wave * SL + j, r = (slab & 7) * 8, half = slab >> 3;
      const int page = __builtin_amdgcn_readlane(pages, r);
      const int key = t * CA_BK + r, n = page < 0 ? 0 : min(total - key, 8);
      const int64_t p = max(page, 0), at = key & ((1 << c.pg.lg_page) - 1);
      const bf16_t* kb = (const bf16_t*)c.pg.k + p * c.pg.k_page + at * c.pg.k_token + hk * c.pg.k_head + 64 * half;
      const bf16_t* vb = (const bf16_t*)c.pg.v + p * c.pg.v_page + at * c.pg.v_token + hk * c.pg.v_head + 64 * half;
      const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc(
          (void*)kb, (short)0, n ? ((n - 1) * (int)c.pg.k_token + 64) * 2 : 0, SWAM_BUF_DWORD3);
      const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc(
          (void*)vb, (short)0, n ? ((n - 1) * (int)c.pg.v_token + 64) * 2 : 0, SWAM_BUF_DWORD3);
      dma_slab(rk, &to[0][slab * 64], off_k[j & 1]);
      dma_slab(rv, &to[1][slab * 64], off_v[j & 1]);
    }
  };
  // V^T operand by transposed LDS reads: in each 16-lane group lane a addresses
  // V[key0 + (a >> 2)][col0 + 4 (a & 3)] and lane i receives keys key0..key0+3 of
  // column col0 + i, the order in which the P^T accumulators hold the keys
  const int a16 = lane & 15, G = lane >> 4, rlo = 4 * g + (a16 >> 2);
  int vofs[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int hd = 32 * x + 16 * (G & 1) + 4 * (a16 & 3);
    vofs[x] = rlo * 64 + 8 * ((hd >> 3) ^ lds_swz(rlo)) + (hd & 7);
  }
  int kofs[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) kofs[s] = r31 * 8 + ((2 * s + g) ^ lds_swz(r31));

  f32x16 o[D / 32];
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[t][r] = 0.0f;
  // the lowest finite value: a row whose keys so far are all hidden adds nothing
  float m_run = -FLT_MAX, l_run = 0.0f;
  const float sc = LOG2E * c.scale;

  // the keys of tile t that this lane's row sees, one bit each
  auto seen = [&](int t, uint64_t vis) -> uint64_t {
    const int h = lim - t * CA_BK, l = low - t * CA_BK;
    uint64_t m = h < 0 ? 0 : h >= 63 ? vis : vis & ((2ull << h) - 1);
    return l > 63 ? 0 : l > 0 ? m & (~0ull << l) : m;
  };
  auto v_operand = [&](const unsigned short* vs, int ht, int t, int u) -> bf16x8 {
    const int base = (ht >> 1) * CA_BK * 64 + (32 * t + 16 * u) * 64;
    const v4i16 x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(vs + vofs[ht & 1] + base));
    const v4i16 x2 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(vs + vofs[(ht & 1) ^ 1] + 8 * 64 + base));
    const uint2 w1 = __builtin_bit_cast(uint2, x1), w2 = __builtin_bit_cast(uint2, x2);
    return __builtin_bit_cast(bf16x8, make_uint4(w1.x, w1.y, w2.x, w2.y));
  };

  // one tile of keys; `part`: some row sees some of its keys only; `mixed`: of those that
  // another row sees; `fresh`: the first of this wave
  auto tile = [&](const uint4 (&from)[2][TILE], int at, uint64_t vis, bool part, bool mixed, bool fresh) {
    const uint4* Kt = from[0];
    auto scores = [&](f32x16 (&st)[2], uint64_t vis) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int r = 0; r < 16; ++r) st[t][r] = 0.0f;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
          const bf16x8 kf = __builtin_bit_cast(bf16x8, Kt[(s >> 2) * CA_BK * 8 + kofs[s & 3] + t * 32 * 8]);
          st[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[s], st[t], 0, 0, 0);
        }
      }
      if (part) {
        // register r holds key 8 (r >> 2) + 4 g + (r & 3) of its half
        const uint64_t m = seen(at, vis) >> (4 * g);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const uint32_t bits = (uint32_t)(m >> (32 * t));
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const uint32_t keep = (uint32_t)__builtin_amdgcn_sbfe((int)bits, 8 * (r >> 2) + (r & 3), 1);
            st[t][r] = __uint_as_float((__float_as_uint(st[t][r]) & keep) | (0xff800000u & ~keep));
          }
        }
      }
    };
    bf16x8 pf[2][2];
    float ps0 = 0.0f, ps1 = 0.0f;
    auto probs = [&](const f32x16 (&st)[2]) {
      ps0 = 0.0f; ps1 = 0.0f;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int mm = 0; mm < 8; mm += 2) {
            const float p0 = __builtin_amdgcn_exp2f(fmaf(st[t][8 * u + mm], sc, -m_run));
            const float p1 = __builtin_amdgcn_exp2f(fmaf(st[t][8 * u + mm + 1], sc, -m_run));
            ps0 += p0; ps1 += p1;
            // P in bf16, the other operand's type; the sum keeps float32
            pf[t][u][mm] = (__bf16)p0; pf[t][u][mm + 1] = (__bf16)p1;
          }
    };
    if (!fresh) {
      f32x16 st[2];
      scores(st, vis);
      probs(st);
    }
    // the running maximum moves only when a row sum shows that some weight passed
    // 2^8 (or is NaN): the scores are then formed again against the new one
    if (fresh || __any(!(ps0 + ps1 <= 256.0f))) {
      uint64_t again = vis;
      asm volatile("" : "+s"(again) : : "memory");
      f32x16 st[2];
      scores(st, again);
      float mx = st[0][0];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, st[t][r]);
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float m_new = fmaxf(m_run, mx * sc);
      const float corr = __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= corr;
#pragma unroll
      for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] *= corr;
      probs(st);
    }
    l_run += ps0 + ps1;
    const unsigned short* vs = reinterpret_cast<const unsigned short*>(from[1]);
    bool odd = false;
    if (mixed) {
      // a weight of zero does not hide a value that is not finite
      u16x2 top = {0, 0};
#pragma unroll
      for (int i = 0; i < TILE / 64; ++i) {
        const uint4 x = from[1][i * 64 + lane];
        const uint32_t x4[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
          top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, x4[e] & 0x7fff7fffu));
      }
      odd = __any(top[0] >= 0x7f80 || top[1] >= 0x7f80);
    }
    if (odd) {
      // key by key: every product keeps one, and only the rows that see it take it
      const uint64_t m = seen(at, vis);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll 1
          for (int key = 0; key < 16; ++key) {
            const int e = 4 * (key >> 3) + (key & 3);
            const bool mine = ((key >> 2) & 1) == g, sees = (m >> (32 * t + 16 * u + key)) & 1;
            uint32_t keep[4];
#pragma unroll
            for (int d = 0; d < 4; ++d)
              keep[d] = mine && (e >> 1) == d ? ((e & 1) ? 0xffff0000u : 0xffffu) : 0u;
            auto only = [&](bf16x8 x) -> bf16x8 {
              const uint4 y = __builtin_bit_cast(uint4, x);
              return __builtin_bit_cast(bf16x8, make_uint4(y.x & keep[0], y.y & keep[1], y.z & keep[2], y.w & keep[3]));
            };
            const bf16x8 pk = only(pf[t][u]);
#pragma unroll
            for (int ht = 0; ht < D / 32; ++ht) {
              const f32x16 x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(only(v_operand(vs, ht, t, u)), pk, o[ht], 0, 0, 0);
#pragma unroll
              for (int r = 0; r < 16; ++r) o[ht][r] = sees ? x[r] : o[ht][r];
            }
          }
      return;
    }
#pragma unroll
    for (int ht = 0; ht < D / 32; ++ht)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int u = 0; u < 2; ++u)
          o[ht] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_operand(vs, ht, t, u), pf[t][u], o[ht], 0, 0, 0);
  };

  // All waves form the same mask words: that of the tile at hand, of the next, whose loads
  // run meanwhile, and the pages of the one after it.
  int pages = page_at(t0), next = page_at(t0 + 1);
  uint64_t vis = __ballot(pages >= 0);
  if (vis) issue(kv[0], t0, pages);
  bool fresh = true;
  int buf = 0;
  for (int t = t0; t < t1; ++t) {
    const uint64_t ahead = __ballot(next >= 0);
    if (vis | ahead) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
    }
    if (ahead) issue(kv[buf ^ 1], t + 1, next);
    next = page_at(t + 2);
    const int k0 = t * CA_BK, k1 = k0 + CA_BK - 1;
    if (vis && k0 <= lim_last && k1 >= low_first) {
      const bool cut = k1 > lim_first, early = k0 < low_last;
      tile(kv[buf], t, vis, cut || early || vis != ~0ull, (cut && lim_first < total - 1) || early, fresh);
      fresh = false;
    }
    vis = ahead;
    buf ^= 1;
  }
  const float l = l_run + __shfl_xor(l_run, 32);
  int me = tid;
  asm volatile("" : "+v"(me));
  const int in_tile = (me >> 6) * 32 + (me & 31), want = r0 + in_tile, rr = min(want, rows - 1);
  const int64_t tok = w.q.a + rr / group;
  const int head = hk * group + rr % group;
  if (w.ch > 1) {
    if (want >= rows) return;
    const int64_t row = ((int64_t)w.slot * c.pg.kv_heads + hk) * sp.slot_rows + in_tile;
    float* po = sp.o + row * D;
#pragma unroll
    for (int ht = 0; ht < D / 32; ++ht)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
        *reinterpret_cast<float4*>(po + 32 * ht + 8 * q4 + 4 * g) =
            make_float4(o[ht][4 * q4], o[ht][4 * q4 + 1], o[ht][4 * q4 + 2], o[ht][4 * q4 + 3]);
    if (g == 0) {
      float* pm = sp.ml + row * 2;
      pm[0] = m_run;
      pm[1] = l;
    }
    return;
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  bf16_t* op = (bf16_t*)c.o + tok * c.o_ld + head * D;
  // a lane holds 4 of every 8 columns, its partner (lane ^ 32) the others: two runs are
  // exchanged into one whole run of 8 each
#pragma unroll
  for (int ht = 0; ht < D / 32; ++ht)
#pragma unroll
    for (int q4 = 0; q4 < 4; q4 += 2) {
      uint32_t v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        v[e] = pack_bf16x2(o[ht][4 * q4 + 2 * e] * inv, o[ht][4 * q4 + 2 * e + 1] * inv);
      const auto x = __builtin_amdgcn_permlane32_swap(v[0], v[2], false, false);
      const auto y = __builtin_amdgcn_permlane32_swap(v[1], v[3], false, false);
      if (want < rows) *(uint4*)(op + 32 * ht + 8 * (q4 + g)) = make_uint4(x[0], y[0], x[1], y[1]);
    }
  if (want >= rows) return;
  if (c.lse != nullptr && g == 0) c.lse[tok * c.heads + head] = l == 0.0f ? -INFINITY : (m_run + log2f(l)) * LN2;
}

// float32: the same products on 32x32x2 MFMAs with operands straight from global memory.
// Four waves take every fourth tile of 32 keys of the same 32 rows and meet in LDS.
template <int D>
__global__ void __launch_bounds__(256)
cache_f32(const CacheArgs c, const Split sp, int unit0) {
  constexpr int LD = D + 4, BQ = 32, BK = 32;
  __shared__ float os[4][32][LD];
  __shared__ float ms[4][32], ls[4][32];
  const int group = c.heads / c.pg.kv_heads;
  const int hk = blockIdx.x % c.pg.kv_heads;
  Work w;
  if (!work_at<D, BQ, BK>(c, sp, unit0 + blockIdx.x / c.pg.kv_heads, w)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 5, r31 = lane & 31;
  const int rows = w.q.n * group, r0 = w.qi * BQ, total = w.q.total;
  const int rl = min(r0 + BQ, rows) - 1;         // the tile's last row
  int lo, hi, t0, t1;
  key_range(c, w.q, group, r0, rl, lo, hi);
  slice_of(lo, hi, BK, w.y, w.ch, t0, t1);
  const int rr = min(r0 + r31, rl);
  int lim = total - 1, low = 0, lim_first = total - 1, low_last = 0;
  if (c.causal) {
    lim = min(lim, w.q.old + rr / group);
    lim_first = min(lim_first, w.q.old + r0 / group);
  }
  if (c.window) {
    low = max(w.q.old + rr / group - c.window + 1, 0);
    low_last = max(w.q.old + rl / group - c.window + 1, 0);
  }
  f32x4 qf[D / 8];
  {
    const float* qp = (const float*)c.q + (int64_t)(w.q.a + rr / group) * c.q_ld + (hk * group + rr % group) * D;
#pragma unroll
    for (int s = 0; s < D / 8; ++s) qf[s] = *reinterpret_cast<const f32x4*>(qp + 4 * (2 * s + g));
  }
  const int32_t* table = c.pg.table + w.s * c.pg.table_ld;
  const int slot_mask = (1 << c.pg.lg_page) - 1;
  f32x16 o[D / 32];
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[t][r] = 0.0f;
  const float sc = LOG2E * c.scale;
  float m = -FLT_MAX, l = 0.0f;
  for (int t = t0 + wave; t < t1; t += 4) {
    const int kb = t * BK, key = kb + r31;
    int page = key < total ? table[key >> c.pg.lg_page] : -1;
    if (page >= c.pg.n_pages) page = -1;
    const uint32_t vis = (uint32_t)__ballot(page >= 0);
    if (vis == 0) continue;
    page = max(page, 0);                         // (a tile with a visible key has a page 0)
    // all operands of the tile are requested before the first product
    const float* kp = (const float*)c.pg.k + page * c.pg.k_page + (key & slot_mask) * c.pg.k_token + hk * c.pg.k_head;
    f32x4 kf[D / 8];
#pragma unroll
    for (int s = 0; s < D / 8; ++s) kf[s] = *reinterpret_cast<const f32x4*>(kp + 4 * (2 * s + g));
    float vf[D / 32][16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int kr = 8 * (r >> 2) + 4 * g + (r & 3);
      const float* vp = (const float*)c.pg.v + __shfl(page, kr) * c.pg.v_page + ((kb + kr) & slot_mask) * c.pg.v_token +
                        hk * c.pg.v_head + r31;
#pragma unroll
      for (int h = 0; h < D / 32; ++h) vf[h][r] = vp[32 * h];
    }
    f32x16 st;
#pragma unroll
    for (int r = 0; r < 16; ++r) st[r] = 0.0f;
#pragma unroll
    for (int s = 0; s < D / 8; ++s) {
#pragma unroll
      for (int e = 0; e < 4; ++e) st = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[s][e], qf[s][e], st, 0, 0, 0);
    }
    // the keys that this lane's row sees
    const int h = lim - kb, u = low - kb;
    uint32_t row_sees = h < 0 ? 0u : h >= 31 ? vis : vis & ((2u << h) - 1);
    row_sees = u > 31 ? 0u : u > 0 ? row_sees & (~0u << u) : row_sees;
    const uint32_t mine = row_sees >> (4 * g), any = vis >> (4 * g);
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      st[r] = ((mine >> (8 * (r >> 2) + (r & 3))) & 1u) ? st[r] * sc : -INFINITY;
      mx = fmaxf(mx, st[r]);
    }
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    const float m_new = fmaxf(m, mx), corr = exp2f(m - m_new);
    m = m_new;
    l *= corr;
#pragma unroll
    for (int h = 0; h < D / 32; ++h)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[h][r] *= corr;
    // a weight of zero does not hide a value that is not finite: where rows see different keys
    // such a tile is summed key by key
    bool odd = false;
    if (kb + BK - 1 > lim_first || kb < low_last) {
#pragma unroll
      for (int h = 0; h < D / 32; ++h)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          odd |= ((any >> (8 * (r >> 2) + (r & 3))) & 1u) && !(fabsf(vf[h][r]) <= FLT_MAX);
      odd = __any(odd);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int b = 8 * (r >> 2) + (r & 3);
      const bool see = (any >> b) & 1u;
      const float p = exp2f(st[r] - m_new);
      l += p;
      if (!odd) {
#pragma unroll
        for (int h = 0; h < D / 32; ++h)
          o[h] = __builtin_amdgcn_mfma_f32_32x32x2f32(see ? vf[h][r] : 0.0f, p, o[h], 0, 0, 0);
        continue;
      }
#pragma unroll
      for (int gg = 0; gg < 2; ++gg) {
        const bool sees = (row_sees >> (b + 4 * gg)) & 1u;
#pragma unroll
        for (int h = 0; h < D / 32; ++h) {
          const f32x16 x = __builtin_amdgcn_mfma_f32_32x32x2f32(g == gg ? vf[h][r] : 0.0f, g == gg ? p : 0.0f, o[h], 0, 0, 0);
#pragma unroll
          for (int e = 0; e < 16; ++e) o[h][e] = sees ? x[e] : o[h][e];
        }
      }
    }
  }
  l += __shfl_xor(l, 32);
  if (g == 0) { ms[wave][r31] = m; ls[wave][r31] = l; }
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4)
      *reinterpret_cast<float4*>(&os[wave][r31][32 * t + 8 * q4 + 4 * g]) =
          make_float4(o[t][4 * q4], o[t][4 * q4 + 1], o[t][4 * q4 + 2], o[t][4 * q4 + 3]);
  __syncthreads();
  const int q = tid >> 3;
  if (r0 + q > rl) return;
  const int64_t tok = w.q.a + (r0 + q) / group;
  const int head = hk * group + (r0 + q) % group;
  const float mt = fmaxf(fmaxf(ms[0][q], ms[1][q]), fmaxf(ms[2][q], ms[3][q]));
  float f[4], lt = 0.0f;
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    f[v] = exp2f(ms[v][q] - mt);
    lt = fmaf(ls[v][q], f[v], lt);
  }
  const bool whole = w.ch <= 1;
  const int64_t row = ((int64_t)w.slot * c.pg.kv_heads + hk) * sp.slot_rows + q;
  const float inv = !whole ? 1.0f : lt == 0.0f ? 0.0f : 1.0f / lt;
  float* dst = whole ? (float*)c.o + tok * c.o_ld + head * D : sp.o + row * D;
#pragma unroll
  for (int h = 0; h < D / 64; ++h) {
    const int col = 64 * h + (tid & 7) * 8;
    float acc[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      acc[e] = 0.0f;
#pragma unroll
      for (int v = 0; v < 4; ++v) acc[e] = fmaf(os[v][q][col + e], f[v], acc[e]);
      acc[e] *= inv;
    }
    store8(dst + col, acc);
  }
  if ((tid & 7) == 0) {
    if (!whole) {
      sp.ml[row * 2] = mt;
      sp.ml[row * 2 + 1] = lt;
    } else if (c.lse != nullptr) {
      c.lse[tok * c.heads + head] = lt == 0.0f ? -INFINITY : (mt + log2f(lt)) * LN2;
    }
  }
}

// One wave per token and head of a split sequence adds up its slices, in their order.
template <typename T, int D, int BQ, int BK>
__global__ void __launch_bounds__(256)
cache_join(const CacheArgs c, const Split sp) {
  const int tiles = sp.plan[0];
  if (tiles == 0) return;                       // nothing was split
  const int lane = threadIdx.x & 63, kvh = c.pg.kv_heads, group = c.heads / kvh;
  const int64_t n = (int64_t)c.n_q * c.heads;
  const int per = (c.pg.n_seqs + 63) >> 6;
  for (int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); id < n; id += (int64_t)gridDim.x * 4) {
    const int tok = (int)(id / c.heads), head = (int)(id % c.heads);
    const int s = seq_of(c.pg, tok);
    const Seq q = seq_at<BQ, BK>(c, group, s);
    const int ch = max((q.nk + tiles - 1) / tiles, 1);
    if (tok < q.a || tok >= q.a + q.n || ch == 1) continue;
    // units of the split sequences in front of it
    int units = 0;
    for (int i = 0; i < per; ++i) {
      const int b = lane * per + i;
      if (b >= s) break;
      const Seq f = seq_at<BQ, BK>(c, group, b);
      const int fc = max((f.nk + tiles - 1) / tiles, 1);
      units += fc > 1 ? f.qt * fc : 0;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) units += __shfl_xor(units, o);
    const int r = (tok - q.a) * group + head % group, qi = r / BQ;
    // (the workgroups count the row tiles from the last)
    const int64_t slot = ((int64_t)(units + (q.qt - 1 - qi) * ch) * kvh + head / group) * sp.slot_rows + r % BQ;
    const int64_t pitch = (int64_t)kvh * sp.slot_rows;
    float m = -FLT_MAX;
    for (int y = lane; y < ch; y += 64) m = fmaxf(m, sp.ml[(slot + y * pitch) * 2]);
    m = warp_max(m);
    float l = 0.0f, acc[D / 64];
#pragma unroll
    for (int e = 0; e < D / 64; ++e) acc[e] = 0.0f;
    for (int y = 0; y < ch; ++y) {
      const float f = exp2f(sp.ml[(slot + y * pitch) * 2] - m);
      l = fmaf(sp.ml[(slot + y * pitch) * 2 + 1], f, l);
#pragma unroll
      for (int e = 0; e < D / 64; ++e) acc[e] = fmaf(sp.o[(slot + y * pitch) * D + 64 * e + lane], f, acc[e]);
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int e = 0; e < D / 64; ++e)
      Elem<T>::store((T*)c.o + tok * c.o_ld + head * D + 64 * e + lane, acc[e] * inv);
    if (c.lse != nullptr && lane == 0) c.lse[id] = l == 0.0f ? -INFINITY : (m + log2f(l)) * LN2;
  }
}

template <typename T, int D>
static void run_cache(const CacheArgs& c, float* ws, int64_t ws_floats, hipStream_t st) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int BQ = F32 ? 32 : 128, BK = F32 ? 32 : CA_BK;
  const int kvh = c.pg.kv_heads, group = c.heads / kvh;
  // row tiles at most and at least: the chunks' lengths are on the device
  const int64_t rows = (int64_t)c.n_q * group;
  const int64_t most = std::min((rows + (int64_t)(BQ - 1) * c.pg.n_seqs) / BQ, rows), least = (rows + BQ - 1) / BQ;
  Split sp{};
  sp.slot_rows = (int)std::min<int64_t>(BQ, rows);
  // keys are split where the row tiles do not fill the card twice, as far as the
  // workspace holds the partial results: at most two per slice of the budget
  if (least * kvh < 2048) {
    const int64_t fit = (ws_floats - 64) / (2 * (int64_t)sp.slot_rows * (D + 2));
    sp.budget = (int)std::min<int64_t>(1024, std::max<int64_t>(fit, 0));
    sp.plan = (int*)ws;
    sp.o = ws + 64;
    sp.ml = sp.o + 2 * (int64_t)sp.budget * sp.slot_rows * D;
  }
  const int64_t units = most + sp.budget / kvh;
  // a grid holds less than 2^32 threads: more take another launch
  const int64_t step = ((1 << 24) - 1) / kvh;
  for (int64_t u = 0; u < units; u += step) {
    const dim3 grid((unsigned)(std::min(units - u, step) * kvh));
    if constexpr (F32) hipLaunchKernelGGL((cache_f32<D>), grid, dim3(256), 0, st, c, sp, (int)u);
    else hipLaunchKernelGGL((cache_bf16<D>), grid, dim3(256), 0, st, c, sp, (int)u);
  }
  if (sp.budget) {
    const unsigned n = (unsigned)std::min<int64_t>(((int64_t)c.n_q * c.heads + 3) / 4, 2048);
    hipLaunchKernelGGL((cache_join<T, D, BQ, BK>), dim3(n), dim3(256), 0, st, c, sp);
  }
}

hipError_t launch_cache_attention(int dtype, const CacheArgs& c, float* ws, int64_t ws_floats, hipStream_t st) {
  if (c.n_q <= 0) return hipSuccess;
  if (dtype == 1) {
    if (c.dim == 64) run_cache<bf16_t, 64>(c, ws, ws_floats, st);
    else run_cache<bf16_t, 128>(c, ws, ws_floats, st);
  } else {
    if (c.dim == 64) run_cache<float, 64>(c, ws, ws_floats, st);
    else run_cache<float, 128>(c, ws, ws_floats, st);
  }
  return hipGetLastError();
}

}  // namespace swam
