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
//
// What bounds it (kernels alone, on keys from memory): for chunks the instructions of a score (causal 10,160 x 24
// heads of 64 373 to 388 us by the clock, 820 to 850 TFLOP/s: vector operations 65% of the time, MFMAs 40%, hardly
// side by side); for single
// tokens the bytes of K and V (8 x 10,160 keys of 24 heads 92 us, 5.4 TB/s); in float32 the matrix unit
// (causal 4,096 x 24 heads 443 us with the joining pass, 1.2 times its products at a large product's rate).
#include "gemm_common.h"
#include "paged.h"

#include <algorithm>
#include <cfloat>
#include <type_traits>

namespace swam {

typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16;

constexpr int CA_BK = 64;                      // keys per tile
constexpr int FEW_BQ = 32;                     // rows of a tile of the line below
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// How the keys are split and where partial results go: slot i holds slot_rows rows of
// [head_dim] sums, and (maximum, sum) for each.
struct Split {
  float* o;
  float* ml;
  int* plan;          // [0]: tiles of a slice, written by workgroup 0 for the joining pass
  int budget;         // slices beyond the first of every row tile, 0: keys are not split
  int slot_rows;
};
constexpr int NO_SPLIT = 1 << 30;              // more tiles than any sequence has

// Sequence s as the kernels see it.
struct Seq {
  int a, n;           // first row, tokens of its chunk
  int old, total;     // tokens before the chunk, keys
  int qt, nk;         // row tiles, key tiles that a row tile reads at most
};
template <int BQ, int BK>
__device__ __forceinline__ Seq seq_at(const CacheArgs& c, int s) {
  Seq q{};
  if (s >= c.pg.n_seqs) return q;
  int e;
  chunk_of(c.pg, s, c.n_q, q.a, e);
  q.n = e - q.a;
  q.old = held(c.pg, s);
  q.total = (int)min((int64_t)q.old + q.n, (int64_t)c.pg.max_pages << c.pg.lg_page);
  q.qt = (q.n * c.group + BQ - 1) / BQ;
  q.nk = (q.total + BK - 1) / BK;
  // a causal window bounds what a row tile reads: its own tokens (BQ + 1 at most) and the
  // window before them
  if (c.window && c.causal) q.nk = min(q.nk, (min(c.window, 1 << 30) + BQ + 1) / BK + 2);
  return q;
}

// inclusive sums over the first `n` lanes
template <typename T>
__device__ __forceinline__ T wave_scan(T v, int n) {
  for (int s = 1; s < n; s <<= 1) {
    const T u = __shfl_up(v, s);
    if ((int)(threadIdx.x & 63) >= s) v += u;
  }
  return v;
}

// Tiles of a slice, from the key tiles of all row tiles (`all`, over all K/V heads) and the most of
// one: modelled time (us) of the workgroups, by how many share a CU (`tile`: the time that each
// takes for a tile then), of what they write, and of the pass that joins the slices.  all / t
// slices beyond the first are within the budget; a row tile of more than t tiles has
// fewer than 2 all / t.
// Measured on 313 tiles out of the caches, us a tile.  head_dim 64, groups of waves: 0.6 for one workgroup to a CU,
// then in whole rounds (1.2, 1.8); one group: 1.14, 1.37, 1.90 and 2.42 for one to four, 3.0 as soon as there are more.
// head_dim 128: groups 1.0 and 2.1; one group 1.55, 2.13, 3.50, 4.36.  Keys from memory take longer where little
// else runs (one group, one workgroup to a CU 1.77, two 1.89): the constants are theirs.
template <int D, int KG>
__device__ __forceinline__ int slice_tiles(float all, int most, const Split& sp) {
  if (sp.budget == 0) return NO_SPLIT;
  const float bytes = all * (float)sp.slot_rows * (D + 2) * 4.0f;     // of one tile to a slice
  auto time_of = [&](float t) {
    const float n = all * __builtin_amdgcn_rcpf(t) * (1.0f / 256.0f);   // workgroups to a CU
    if (KG > 1) return t * (D == 64 ? 0.68f : 1.0f) * fmaxf(n, 1.0f);
    if (D == 64) return t * (n <= 1.0f ? 1.77f : n <= 2.0f ? 1.89f : n <= 3.0f ? 2.07f : 0.675f * fmaxf(n, 4.0f));
    return t * (n <= 1.0f ? 1.8f : 1.1f * fmaxf(n, 2.0f));
  };
  int best = NO_SPLIT;
  float best_us = time_of((float)most);
  constexpr int PARTS[] = {2, 3, 4, 5, 6, 8, 10, 12, 16, 24, 32, 64};
#pragma unroll
  for (int k = 0; k < (int)(sizeof(PARTS) / sizeof(int)); ++k) {
    const int n = (most + PARTS[k] - 1) / PARTS[k];
    const float t = (float)n;
    const float us = time_of(t) + 6.0f + bytes * (1.0f / 1.6e6f) * __builtin_amdgcn_rcpf(t);
    if (n > 1 && t * (float)sp.budget >= all * 1.0001f + 1.0f && us < best_us) { best_us = us; best = n; }
  }
  return best;
}
__device__ __forceinline__ int slices(int nk, int tiles) { return nk <= tiles ? 1 : (nk + tiles - 1) / tiles; }

// What a workgroup does: slice y of ch of the keys of row tile qi of sequence s, its
// partial results in `slot` (units before it in split sequences).
struct Work {
  Seq q;
  int s, qi, y, ch, slot;
};
// The lanes hold the sequences in order, `per` to a lane; passes over them find the
// slices' length, the units in front of each, and the one that holds `unit`.
template <int D, int KG, int BQ, int BK>
__device__ __forceinline__ bool work_at(const CacheArgs& c, const Split& sp, int unit, Work& w) {
  const int lane = threadIdx.x & 63;
  const int per = (c.pg.n_seqs + 63) >> 6, lanes = min(c.pg.n_seqs, 64);
  const Seq first = seq_at<BQ, BK>(c, lane * per);
  int tiles = NO_SPLIT;
  if (sp.budget) {
    float all = (float)first.qt * (float)first.nk;
    int most = first.nk;
    for (int i = 1; i < per; ++i) {
      const Seq q = seq_at<BQ, BK>(c, lane * per + i);
      all += (float)q.qt * (float)q.nk;
      most = max(most, q.nk);
    }
    for (int o = 1; o < lanes; o <<= 1) {
      all += __shfl_xor(all, o);
      most = max(most, __shfl_xor(most, o));
    }
    all = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, all)));
    tiles = __builtin_amdgcn_readfirstlane(
        slice_tiles<D, KG>(all * (float)c.pg.kv_heads, __builtin_amdgcn_readfirstlane(most), sp));
    if (blockIdx.x == 0 && threadIdx.x == 0) sp.plan[0] = tiles;
  }
  int units = 0, split = 0;
  for (int i = 0; i < per; ++i) {
    const Seq q = i == 0 ? first : seq_at<BQ, BK>(c, lane * per + i);
    const int ch = slices(q.nk, tiles);
    units += q.qt * ch;
    split += ch > 1 ? q.qt * ch : 0;
  }
  int at = wave_scan(units, lanes), slot = sp.budget ? wave_scan(split, lanes) : 0;
  const uint64_t past = __ballot(at > unit);
  if (past == 0) return false;
  at -= units;
  slot -= split;
  w = Work{};
  int r = 0;
  for (int i = 0; i < per; ++i) {
    const Seq q = i == 0 ? first : seq_at<BQ, BK>(c, lane * per + i);
    const int ch = slices(q.nk, tiles), n = q.qt * ch;
    if (unit >= at && unit < at + n) {
      w.q = q;
      w.s = lane * per + i;
      w.ch = ch;
      w.slot = slot + unit - at;
      r = unit - at;
    }
    at += n;
    slot += ch > 1 ? n : 0;
  }
  const int b = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)past) - 1);
  auto bcast = [&](int& v) { v = __builtin_amdgcn_readlane(v, b); };
  bcast(w.q.a); bcast(w.q.n); bcast(w.q.old); bcast(w.q.total); bcast(w.q.qt); bcast(w.q.nk);
  bcast(w.s); bcast(w.ch); bcast(w.slot); bcast(r);
  // (sequences that overlap against the contract can pass what 32 bits count: nothing is done then)
  if (w.ch == 0 || (w.ch > 1 && (uint32_t)w.slot >= (uint32_t)(2 * sp.budget / c.pg.kv_heads))) return false;
  // the last rows of a causal chunk see most: they come first
  const int qi = w.ch == 1 ? r : r / w.ch;
  w.qi = w.q.qt - 1 - qi;
  w.y = r - qi * w.ch;
  return true;
}

// Row r of a sequence is head r % group of token r / group: for rows near the tile's first,
// whose token and remainder are known (x below group + BQ).
struct Rows {
  int tok, rem, group;
  uint32_t magic;                              // ceil(2^32 / group), exact for x (group - 1) < 2^32
  __device__ __forceinline__ Rows(int r0, const CacheArgs& c) : group(c.group), magic(c.group_magic) {
    tok = group == 1 ? r0 : r0 / group;
    rem = r0 - tok * group;
  }
  __device__ __forceinline__ int token(int i) const { return tok + (group == 1 ? i : (int)__umulhi(rem + i, magic)); }
  __device__ __forceinline__ int head(int i) const {
    return group == 1 ? 0 : rem + i - (int)__umulhi(rem + i, magic) * group;
  }
};

// the keys [lo, hi) that tokens [t0, t1] of a sequence see, as far as one range holds them
__device__ __forceinline__ void key_range(const CacheArgs& c, const Seq& q, int t0, int t1, int& lo, int& hi) {
  hi = c.causal ? min(q.old + t1 + 1, q.total) : q.total;
  lo = c.window ? min(max(q.old + t0 - c.window + 1, 0), hi) : 0;
}

// tiles [t0, t1) of slice y of ch
__device__ __forceinline__ void slice_of(int lo, int hi, int bk, int y, int ch, int& t0, int& t1) {
  const int a = lo / bk, n = (hi + bk - 1) / bk - a;
  if (ch == 1) { t0 = a; t1 = a + n; return; }
  const int each = n / ch, more = n - each * ch;
  t0 = a + each * y + min(y, more);
  t1 = t0 + each + (y < more);
}

// Pages of the runs of RUN 8-key slabs of a tile, -1: none; and which of its keys there are.
template <int N, int RUN>
__device__ __forceinline__ void pages_of(const Paged& pg, const_i32* table, int key0, int total, int (&pages)[N]) {
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int key = key0 + 8 * RUN * j;
    const int p = key < total ? table[key >> pg.lg_page] : -1;
    pages[j] = p < pg.n_pages ? p : -1;
  }
}
template <int N, int RUN>
__device__ __forceinline__ uint64_t keys_of(int key0, int total, const int (&pages)[N]) {
  uint64_t m = 0;
#pragma unroll
  for (int j = 0; j < N; ++j) m |= pages[j] >= 0 ? (~0ull >> (64 - 8 * RUN)) << (8 * RUN * j) : 0ull;
  const int n = total - key0;
  return n >= 8 * RUN * N ? m : n <= 0 ? 0ull : m & ((1ull << n) - 1);
}

// A sum over its weights' (inv: 1 / them, or 0 where no key with a weight was seen: its values then do not
// matter, whatever they are).
__device__ __forceinline__ float norm(float o, float inv) { return inv == 0.0f ? 0.0f : o * inv; }

// Loads into LDS that this wave has read: its reads have arrived.
__device__ __forceinline__ void reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Values that are not finite (bf16, exponent all ones): a weight of zero does not hide them, so
// where rows see different keys they are left out of the products and added by hand.
__device__ __forceinline__ uint4 without_odd(uint4 x) {
  auto f = [](uint32_t y) {
    if ((y & 0x7f80u) == 0x7f80u) y &= 0xffff0000u;
    return (y & 0x7f800000u) == 0x7f800000u ? y & 0xffffu : y;
  };
  return make_uint4(f(x.x), f(x.y), f(x.z), f(x.w));
}
__device__ __forceinline__ void add_odd(f32x16& o, int q4, bool sees, uint2 x) {
  const float f[4] = {__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xffff0000u),
                      __uint_as_float(x.y << 16), __uint_as_float(x.y & 0xffff0000u)};
#pragma unroll
  for (int e = 0; e < 4; ++e) o[4 * q4 + e] += sees && !(fabsf(f[e]) <= FLT_MAX) ? f[e] : 0.0f;
}

// RUN: 8-key slabs that share a page for certain
// KG: groups of four waves.  Each takes every KG-th tile of the same rows; they meet in LDS.
// FINE: sequences of up to FEW_BQ rows, which stand beside longer ones here or in a padded call, keep 16 bits of
// each weight as they do on the line: their rows are one wave's, and the second wave, which has none, takes the
// same rows with what bf16 leaves of the weights (three single tokens of 24 heads beside 1,248 behind 3,000 keys:
// 88 us, with bf16's 8 bits alone 71; calls without such a sequence within 0.5%)
template <int D, int RUN, int KG, bool FINE>
__global__ void __launch_bounds__(256 * KG) __attribute__((amdgpu_waves_per_eu(D == 64 ? 4 : 2, 8)))
cache_bf16(const CacheArgs c, const Split sp, int unit0) {
  constexpr int H2 = D / 64;                     // 128-byte halves of a head's row
  constexpr int NW = 4, BQ = 32 * NW;
  constexpr int TILE = CA_BK * 8 * H2;           // uint4 of a K or V tile
  constexpr int RUNS = CA_BK / 8 / RUN;
  __shared__ uint4 kv[KG][2][2][TILE];           // [group][stage][K | V][half][key][8 chunks]
  const int group = c.group;
  // neighbouring workgroups take the K/V heads in turn: with a multiple of 8 of them a
  // head stays on one XCD
  const int hk = blockIdx.x % c.pg.kv_heads;
  Work w;
  if (!work_at<D, KG, BQ, CA_BK>(c, sp, unit0 + blockIdx.x / c.pg.kv_heads, w)) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int kg = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid >> 8);
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6) & 3;     // of its group
  const int g = lane >> 5, r31 = lane & 31;
  const int r0 = w.qi * BQ, left = w.q.n * group - r0, total = w.q.total;   // rows of the sequence from r0 on
  const Rows row_of(r0, c);
  int lo, hi, t0, t1;
  key_range(c, w.q, row_of.tok, row_of.token(min(BQ, left) - 1), lo, hi);
  slice_of(lo, hi, CA_BK, w.y, w.ch, t0, t1);
  [[maybe_unused]] const bool fine = FINE && w.q.n * group <= FEW_BQ, rest = fine && wave == 1;
  // the keys that all rows of this wave see lie in [low_last, lim_first], those that any
  // sees in [low_first, lim_last]; a wave behind the last row sees none
  const int wr = FINE && rest ? 0 : wave * 32;
  int lim_first = total - 1, lim_last = wr < left ? total - 1 : -1, low_first = 0, low_last = 0;
  const int p_first = w.q.old + row_of.token(min(wr, left - 1)), p_last = w.q.old + row_of.token(min(wr + 31, left - 1));
  if (c.causal) {
    lim_first = min(lim_first, p_first);
    lim_last = min(lim_last, p_last);
  }
  if (c.window) {
    low_first = max(p_first - c.window + 1, 0);
    low_last = max(p_last - c.window + 1, 0);
  }
  bf16x8 qf[D / 16];
  int lim = total - 1, low = 0;                  // of this lane's row
  {
    const int i = min(wr + r31, left - 1), tok = row_of.token(i);
    if (c.causal) lim = min(lim, w.q.old + tok);
    if (c.window) low = max(w.q.old + tok - c.window + 1, 0);
    const bf16_t* qp = (const bf16_t*)c.q + (int64_t)(w.q.a + tok) * c.q_ld + (hk * group + row_of.head(i)) * D;
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
      qf[s] = __builtin_bit_cast(bf16x8, *(const uint4*)(qp + 8 * (2 * s + g)));
  }
  const_i32* table = (const_i32*)(c.pg.table + w.s * c.pg.table_ld);

  const int lrow = lane >> 3;
  constexpr int SL = 8 * H2 / NW;                // 8-key slabs of a tile that a wave stages
  const int slab0 = wave * SL, key0 = (slab0 & 7) * 8, half = slab0 >> 3;
  int off_k[2], off_v[2];                        // of even and odd slabs
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int r = j * 8 + lrow, col = 8 * ((lane & 7) ^ lds_swz(r));
    off_k[j] = (r * (int)c.pg.k_token + col) * 2;
    off_v[j] = (r * (int)c.pg.v_token + col) * 2;
  }
  const bf16_t* k_head = (const bf16_t*)c.pg.k + hk * c.pg.k_head + 64 * half;
  const bf16_t* v_head = (const bf16_t*)c.pg.v + hk * c.pg.v_head + 64 * half;
  // K and V of tile t into LDS, `pages` those of this wave's slabs (always as many loads: what has
  // no page stores zeros)
  constexpr int MINE = RUN < SL ? RUN : SL;      // slabs of this wave that share a page
  auto issue = [&](uint4 (&to)[2][TILE], int t, const int (&pages)[SL / MINE]) {
#pragma unroll
    for (int j = 0; j < SL; j += MINE) {
      const int page = pages[j / MINE];
      const int key = t * CA_BK + key0 + 8 * j, n = page < 0 ? 0 : max(min(total - key, 8 * MINE), 0);
      const int64_t p = max(page, 0);
      const int64_t at = key & ((1 << c.pg.lg_page) - 1);
      const bf16_t* kb = k_head + p * c.pg.k_page + at * c.pg.k_token;
      const bf16_t* vb = v_head + p * c.pg.v_page + at * c.pg.v_token;
      const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc(
          (void*)kb, (short)0, n ? ((n - 1) * (int)c.pg.k_token + 64) * 2 : 0, SWAM_BUF_DWORD3);
      const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc(
          (void*)vb, (short)0, n ? ((n - 1) * (int)c.pg.v_token + 64) * 2 : 0, SWAM_BUF_DWORD3);
#pragma unroll
      for (int i = 0; i < MINE; ++i) {
        // (off_* has 8 rows in front of odd slabs')
        const int slab = slab0 + j + i, rows = MINE == 1 ? -8 * ((j + i) & 1) : 16 * (i >> 1);
        dma_slab(rk, &to[0][slab * 64], rows ? vadd_sgpr(off_k[(j + i) & 1], rows * (int)c.pg.k_token * 2) : off_k[(j + i) & 1]);
        dma_slab(rv, &to[1][slab * 64], rows ? vadd_sgpr(off_v[(j + i) & 1], rows * (int)c.pg.v_token * 2) : off_v[(j + i) & 1]);
      }
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
  auto v_operand = [&](const unsigned short* vs, int ht, int t, int u) -> uint4 {
    const int base = (ht >> 1) * CA_BK * 64 + (32 * t + 16 * u) * 64;
    const v4i16 x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(vs + vofs[ht & 1] + base));
    const v4i16 x2 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(vs + vofs[(ht & 1) ^ 1] + 8 * 64 + base));
    const uint2 w1 = __builtin_bit_cast(uint2, x1), w2 = __builtin_bit_cast(uint2, x2);
    return make_uint4(w1.x, w1.y, w2.x, w2.y);
  };

  // one tile of keys; `part`: some row sees some of its keys only; `mixed`: of those that
  // another row sees; `fresh`: the first of this wave
  auto tile = [&](const uint4 (&from)[2][TILE], int at, uint64_t vis, bool part, bool mixed, bool fresh) {
    const uint4* Kt = from[0];
    auto scores = [&](f32x16 (&st)[2], uint64_t vis) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) st[t][r] = 0.0f;
#pragma unroll
      for (int s = 0; s < D / 16; ++s)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const bf16x8 kf = __builtin_bit_cast(bf16x8, Kt[(s >> 2) * CA_BK * 8 + kofs[s & 3] + t * 32 * 8]);
          st[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[s], st[t], 0, 0, 0);
        }
      if (part) {
        // register r holds key 8 (r >> 2) + 4 g + (r & 3) of its half.  (A branch: no tile
        // but the first and last of a row needs these)
        const uint64_t m = seen(at, vis) >> (4 * g);
        uint32_t bits[2] = {(uint32_t)m, (uint32_t)(m >> 32)};
        asm volatile("" : "+v"(bits[0]), "+v"(bits[1]));
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const uint32_t keep = (uint32_t)__builtin_amdgcn_sbfe((int)bits[t], 8 * (r >> 2) + (r & 3), 1);
            st[t][r] = __uint_as_float((__float_as_uint(st[t][r]) & keep) | (0xff800000u & ~keep));
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
      uint32_t w0 = __builtin_amdgcn_readfirstlane((uint32_t)vis), w1 = __builtin_amdgcn_readfirstlane((uint32_t)(vis >> 32));
      asm volatile("" : "+s"(w0), "+s"(w1) : : "memory");
      const uint64_t again = (uint64_t)w1 << 32 | w0;
      f32x16 st[2];
      scores(st, again);
      float mx = st[0][0];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, st[t][r]);
      if constexpr (FINE) {                        // (without the register of an index)
        const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        mx = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
      } else {
        mx = fmaxf(mx, __shfl_xor(mx, 32));
      }
      const float m_new = fmaxf(m_run, mx * sc);
      const float corr = __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= corr;
#pragma unroll
      for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] *= corr;
      if (!FINE || !rest) {
        probs(st);
      } else {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float p = __builtin_amdgcn_exp2f(fmaf(st[t][r], sc, -m_run));
            pf[t][r >> 3][r & 7] = (__bf16)(p - (float)(__bf16)p);
          }
      }
    }
    l_run += ps0 + ps1;
    const unsigned short* vs = reinterpret_cast<const unsigned short*>(from[1]);
    bool odd = false;
    // (what is left of a weight may be zero or negative: nor is an infinite value multiplied by it)
    if (FINE ? mixed || rest : mixed) {
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
      // such values are left out of the products, and the rows that see them add them
      const uint64_t m = seen(at, vis);
#pragma unroll 1
      for (int key = 0; key < CA_BK; ++key) {
        const bool sees = (m >> key) & 1;
#pragma unroll
        for (int ht = 0; ht < D / 32; ++ht)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            const int chunk = (4 * (ht & 1) + q4) ^ lds_swz(key);
            add_odd(o[ht], q4, sees, *reinterpret_cast<const uint2*>(vs + (ht >> 1) * CA_BK * 64 + key * 64 + 8 * chunk + 4 * g));
          }
      }
    }
    auto products = [&](auto clean) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int ht = 0; ht < D / 32; ++ht) {
            const uint4 x = clean(v_operand(vs, ht, t, u));
            o[ht] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), pf[t][u], o[ht], 0, 0, 0);
          }
    };
    if (odd) products([](uint4 x) { return without_odd(x); });
    else products([](uint4 x) { return x; });
  };

  // The next tile is on its way, with its keys in `ahead`; the pages of the one after it are read
  // meanwhile.
  const int stop = min(total, t1 * CA_BK);       // (behind the last tile there are no pages)
  uint4 (&ring)[2][2][TILE] = kv[kg];
  int all[RUNS], own[SL / MINE];
  auto pages_for = [&](int t) {
    pages_of<RUNS, RUN>(c.pg, table, t * CA_BK, stop, all);
    pages_of<SL / MINE, MINE>(c.pg, table, t * CA_BK + key0, stop, own);
  };
  pages_for(t0 + kg);
  uint64_t vis = keys_of<RUNS, RUN>((t0 + kg) * CA_BK, total, all);
  issue(ring[0], t0 + kg, own);
  pages_for(t0 + kg + KG);
  bool fresh = true;
  int buf = 0;
#pragma unroll 1
  for (int tg = t0; tg < t1; tg += KG) {
    const int t = tg + kg;
    // the tile at hand has arrived, and every wave is done with the one before it
    wait_stage<0>();
    reads_done();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const uint64_t ahead = keys_of<RUNS, RUN>((t + KG) * CA_BK, total, all);
    issue(ring[buf ^ 1], t + KG, own);
    pages_for(t + 2 * KG);
    const int k0 = t * CA_BK, k1 = k0 + CA_BK - 1;
    if (vis && k0 <= lim_last && k1 >= low_first) {
      const bool cut = k1 > lim_first, early = k0 < low_last;
      tile(ring[buf], t, vis, cut || early || vis != ~0ull, (cut && lim_first < total - 1) || early, fresh);
      // (both parts of the weights have to go by the same maximum: it moves in every tile)
      fresh = FINE && fine;
    }
    vis = ahead;
    buf ^= 1;
  }
  wait_stage<0>();
  if (FINE && fine) {
    // both parts of the weights meet in the first wave
    float* meet = reinterpret_cast<float*>(&ring[0][0][0]);
    static_assert(D / 2 * 64 * 4 <= (int)sizeof(kv[0]), "they fit in the tiles' place");
    __syncthreads();
    if (rest) {
#pragma unroll
      for (int ht = 0; ht < D / 32; ++ht)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
          *reinterpret_cast<float4*>(meet + ((4 * ht + q4) * 64 + lane) * 4) =
              make_float4(o[ht][4 * q4], o[ht][4 * q4 + 1], o[ht][4 * q4 + 2], o[ht][4 * q4 + 3]);
    }
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int ht = 0; ht < D / 32; ++ht)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const float4 x = *reinterpret_cast<const float4*>(meet + ((4 * ht + q4) * 64 + lane) * 4);
          o[ht][4 * q4] += x.x;
          o[ht][4 * q4 + 1] += x.y;
          o[ht][4 * q4 + 2] += x.z;
          o[ht][4 * q4 + 3] += x.w;
        }
    }
  }
  if constexpr (KG > 1) {
    // what the other groups have, register by register: the same lanes hold the same rows
    float* meet = reinterpret_cast<float*>(&kv[0][0][0][0]);
    constexpr int EACH = (D / 2 + 2) * 64;       // floats of a wave
    static_assert((KG - 1) * 4 * EACH * 4 <= (int)sizeof(kv), "they fit in the tiles' place");
    __syncthreads();
    if (kg > 0) {
      float* to = meet + ((kg - 1) * 4 + wave) * EACH;
#pragma unroll
      for (int ht = 0; ht < D / 32; ++ht)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
          *reinterpret_cast<float4*>(to + ((4 * ht + q4) * 64 + lane) * 4) =
              make_float4(o[ht][4 * q4], o[ht][4 * q4 + 1], o[ht][4 * q4 + 2], o[ht][4 * q4 + 3]);
      *reinterpret_cast<float2*>(to + D / 2 * 64 + 2 * lane) = make_float2(m_run, l_run);
    }
    __syncthreads();
    if (kg > 0) return;
#pragma unroll 1
    for (int k = 0; k < KG - 1; ++k) {
      const float* from = meet + (k * 4 + wave) * EACH;
      const float2 ml = *reinterpret_cast<const float2*>(from + D / 2 * 64 + 2 * lane);
      const float m_new = fmaxf(m_run, ml.x), mine = __builtin_amdgcn_exp2f(m_run - m_new), theirs = __builtin_amdgcn_exp2f(ml.x - m_new);
      m_run = m_new;
      l_run = l_run * mine + ml.y * theirs;
#pragma unroll
      for (int ht = 0; ht < D / 32; ++ht)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const float4 x = *reinterpret_cast<const float4*>(from + ((4 * ht + q4) * 64 + lane) * 4);
          o[ht][4 * q4] = fmaf(x.x, theirs, o[ht][4 * q4] * mine);
          o[ht][4 * q4 + 1] = fmaf(x.y, theirs, o[ht][4 * q4 + 1] * mine);
          o[ht][4 * q4 + 2] = fmaf(x.z, theirs, o[ht][4 * q4 + 2] * mine);
          o[ht][4 * q4 + 3] = fmaf(x.w, theirs, o[ht][4 * q4 + 3] * mine);
        }
    }
  }
  const float l = l_run + __shfl_xor(l_run, 32);
  int me = tid;
  asm volatile("" : "+v"(me));
  const int in_tile = (me >> 6) * 32 + (me & 31), have = min(in_tile, left - 1);
  const int64_t tok = w.q.a + row_of.token(have);
  const int head = hk * group + row_of.head(have);
  if (w.ch > 1) {
    if (in_tile >= left) return;
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
        v[e] = pack_bf16x2(norm(o[ht][4 * q4 + 2 * e], inv), norm(o[ht][4 * q4 + 2 * e + 1], inv));
      const auto x = __builtin_amdgcn_permlane32_swap(v[0], v[2], false, false);
      const auto y = __builtin_amdgcn_permlane32_swap(v[1], v[3], false, false);
      if (in_tile < left) *(uint4*)(op + 32 * ht + 8 * (q4 + g)) = make_uint4(x[0], y[0], x[1], y[1]);
    }
  if (in_tile >= left) return;
  if (c.lse != nullptr && g == 0) c.lse[tok * c.heads + head] = l == 0.0f ? -INFINITY : (m_run + log2f(l)) * LN2;
}

// Adds up the `ch` partial results of rows [r0, r1) of a row tile, slot_at(y) the slot of the
// y-th, in their order.  A wave takes 256 / D rows at a time, AHEAD slices on their way.
template <typename T, int D, int AHEAD, typename SlotAt>
__device__ __forceinline__ void join_rows(const CacheArgs& c, const float* po, const float* pml, int slot_rows, int ch,
                                          int a, int hk, const Rows& row_of, int r0, int r1, SlotAt slot_at) {
  constexpr int PER = D / 4, SETS = 64 / PER;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane % PER * 4;
  for (int rb = r0 + wave * SETS; rb < r1; rb += 4 * SETS) {
    const int r = min(rb + lane / PER, r1 - 1);
    float m = -FLT_MAX, l = 0.0f;
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int y0 = 0; y0 < ch; y0 += AHEAD) {
      float4 v[AHEAD];
      float2 w[AHEAD];
#pragma unroll
      for (int x = 0; x < AHEAD; ++x) {
        const int64_t at = (int64_t)slot_at(min(y0 + x, ch - 1)) * slot_rows + r;
        w[x] = *reinterpret_cast<const float2*>(pml + at * 2);
        v[x] = *reinterpret_cast<const float4*>(po + at * D + col);
        if (y0 + x >= ch) w[x] = make_float2(-FLT_MAX, 0.0f);
      }
      float m_new = m;
#pragma unroll
      for (int x = 0; x < AHEAD; ++x) m_new = fmaxf(m_new, w[x].x);
      const float corr = exp2f(m - m_new);
      m = m_new;
      l *= corr;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] *= corr;
#pragma unroll
      for (int x = 0; x < AHEAD; ++x) {
        if (y0 + x < ch) {
          const float e = exp2f(w[x].x - m);
          l = fmaf(w[x].y, e, l);
          acc[0] = fmaf(v[x].x, e, acc[0]);
          acc[1] = fmaf(v[x].y, e, acc[1]);
          acc[2] = fmaf(v[x].z, e, acc[2]);
          acc[3] = fmaf(v[x].w, e, acc[3]);
        }
      }
    }
    if (rb + lane / PER >= r1) continue;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const int64_t tok = a + row_of.token(r);
    const int head = hk * c.group + row_of.head(r);
    T* op = (T*)c.o + tok * c.o_ld + head * D + col;
    if constexpr (sizeof(T) == 2)
      *reinterpret_cast<uint2*>(op) = make_uint2(pack_bf16x2(norm(acc[0], inv), norm(acc[1], inv)), pack_bf16x2(norm(acc[2], inv), norm(acc[3], inv)));
    else
      *reinterpret_cast<float4*>(op) = make_float4(norm(acc[0], inv), norm(acc[1], inv), norm(acc[2], inv), norm(acc[3], inv));
    if (c.lse != nullptr && col == 0) c.lse[tok * c.heads + head] = l == 0.0f ? -INFINITY : (m + log2f(l)) * LN2;
  }
}

// The slices of a chunk's row tiles: workgroup (x, y) adds up rows [32 y, 32 y + 32) of the x-th
// (row tile, K/V head).
template <int D>
__global__ void __launch_bounds__(256)
cache_join(const CacheArgs c, const Split sp) {
  constexpr int BQ = 128, BK = CA_BK;
  const int tiles = sp.plan[0];
  if (tiles == NO_SPLIT) return;                // nothing was split
  const int lane = threadIdx.x & 63, kvh = c.pg.kv_heads;
  const int per = (c.pg.n_seqs + 63) >> 6, lanes = min(c.pg.n_seqs, 64);
  const int hk = blockIdx.x % kvh, tile = blockIdx.x / kvh;
  int own = 0, split = 0;
  for (int i = 0; i < per; ++i) {
    const Seq q = seq_at<BQ, BK>(c, lane * per + i);
    const int ch = slices(q.nk, tiles);
    own += q.qt;
    split += ch > 1 ? q.qt * ch : 0;
  }
  int at = wave_scan(own, lanes), units = wave_scan(split, lanes);
  const uint64_t past = __ballot(at > tile);
  if (past == 0) return;
  const int b = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)past) - 1);
  at = __builtin_amdgcn_readlane(at - own, b);
  units = __builtin_amdgcn_readlane(units - split, b);
  Seq q = seq_at<BQ, BK>(c, b * per);
  int ch = slices(q.nk, tiles);
  for (int s = b * per; tile >= at + q.qt;) {
    at += q.qt;
    units += ch > 1 ? q.qt * ch : 0;
    q = seq_at<BQ, BK>(c, ++s);
    ch = slices(q.nk, tiles);
  }
  if (ch == 1) return;
  const int qi = tile - at, left = min(q.n * c.group - qi * BQ, BQ);
  const Rows row_of(qi * BQ, c);
  // (the workgroups count the row tiles from the last)
  const int first = units + (q.qt - 1 - qi) * ch;
  if (first < 0 || first + ch > 2 * sp.budget / kvh) return;
  join_rows<bf16_t, D, 8>(c, sp.o, sp.ml, sp.slot_rows, ch, q.a, hk, row_of, (int)blockIdx.y * 32,
                       min(left, (int)blockIdx.y * 32 + 32), [&](int y) { return (first + y) * kvh + hk; });
}

// ---------------------------------------------------------------------------
// one line of key tiles
// ---------------------------------------------------------------------------
// Single tokens and short chunks read K and V once and their bytes are the time; in float32 the
// matrix unit is slow enough for small row tiles.  There all key tiles of all (sequence, K/V
// head, row tile) segments stand in one line that is cut evenly over the workgroups, so
// single tokens of unequal contexts have equal shares (a segment counts a few more for its start and end); a
// segment cut by a border leaves partial results, at most two to a workgroup.  Every row tile of a sequence
// counts the most keys that one of them reads, so shares of chunks whose masks let row tiles see unequal numbers
// of keys are less equal: eight float32 chunks with windows of 1,000 count 29,112 tiles (and the segments' ends)
// where 24,720 are read, and the fullest workgroup reads 65 of them, the mean 48.
struct Few {
  float* o;           // [2 wgs][slot_rows][head_dim] sums
  float* ml;          // [2 wgs][slot_rows] (maximum, sum)
  int wgs;            // of the launch
  int cut;            // workgroups that tiles may be cut over, 0: segments stay whole
  int slot_rows;
  int extra;          // tiles that a segment's start and end are worth
};

// a sequence with the units of its segments for key tiles
template <int BK>
__device__ __forceinline__ Seq line_seq(const CacheArgs& c, const Few& f, int s) {
  Seq q = seq_at<FEW_BQ, BK>(c, s);
  if (q.nk) q.nk += f.extra;
  return q;
}

// The line of tiles (or of whole segments) as the lanes hold it, `per` sequences to a lane.
struct Line {
  int per, mine, upto;                         // this lane's units, and all up to its last
  int all;                                     // units
  int wgs;                                     // that share them
  bool cut;                                    // units are tiles
  Seq first;                                   // the lane's first sequence
  __device__ __forceinline__ static int count(const Seq& q, int kvh, bool cut) {
    return q.qt * kvh * (cut ? q.nk : 1);
  }
  // the units [begin(w), begin(w + 1)) are workgroup w's
  __device__ __forceinline__ int begin(int w) const {
    const int each = all / wgs;
    return w * each + min(w, all - each * wgs);
  }
  // the workgroup of unit x
  __device__ __forceinline__ int wg_of(int x) const {
    const int each = all / wgs, more = all - each * wgs;
    return x < more * (each + 1) ? x / (each + 1) : more + (x - more * (each + 1)) / each;
  }
};
template <int BK>
__device__ __forceinline__ Line line_of(const CacheArgs& c, const Few& f) {
  const int lane = threadIdx.x & 63, lanes = min(c.pg.n_seqs, 64), kvh = c.pg.kv_heads;
  Line l;
  l.per = (c.pg.n_seqs + 63) >> 6;
  // (in 64 bits: sequences that overlap against the contract can pass what 32 bits count, and
  // nothing is done then)
  int64_t tiles = 0, segs = 0;
  int most = 0;
  l.first = line_seq<BK>(c, f, lane * l.per);
  for (int i = 0; i < l.per; ++i) {
    const Seq q = i == 0 ? l.first : line_seq<BK>(c, f, lane * l.per + i);
    if (f.cut) tiles += (int64_t)q.qt * kvh * q.nk;
    segs += (int64_t)q.qt * kvh;
    most = max(most, q.nk);
  }
  const int64_t tiles_upto = wave_scan(tiles, lanes), segs_upto = wave_scan(segs, lanes);
  for (int o = 1; o < lanes; o <<= 1) most = max(most, __shfl_xor(most, o));
  auto last = [&](int64_t v) {
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)v, lanes - 1), hi = __builtin_amdgcn_readlane((uint32_t)(v >> 32), lanes - 1);
    return (int64_t)((uint64_t)hi << 32 | lo);
  };
  constexpr int64_t MOST = 1 << 30;
  const int n_segs = last(segs_upto) < MOST ? (int)last(segs_upto) : 0;
  const int n_tiles = last(tiles_upto) < MOST ? (int)last(tiles_upto) : 0;
  most = __builtin_amdgcn_readfirstlane(most);
  // cut where that saves the time of more tiles than the joining pass adds
  const int cut_wgs = n_segs > 0 ? min(f.cut, (n_tiles + 1) / 2) : 0;
  l.cut = false;
  if (cut_wgs > 0) {
    const int whole = (n_segs + f.wgs - 1) / f.wgs * most, each = (n_tiles + cut_wgs - 1) / cut_wgs;
    l.cut = whole > each + 2;
  }
  l.mine = (int)(l.cut ? tiles : segs);
  l.upto = (int)(l.cut ? tiles_upto : segs_upto);
  l.all = l.cut ? n_tiles : n_segs;
  l.wgs = l.cut ? cut_wgs : min(f.wgs, max(n_segs, 1));
  return l;
}

// Row tiles stand in the line as first, last, second, last but one ...: of a causal chunk the later
// ones see more, and the line counts the most for each.
__device__ __forceinline__ int folded(int i, int n) { return i & 1 ? n - 1 - (i >> 1) : i >> 1; }
__device__ __forceinline__ int fold_index(int tile, int n) { return 2 * tile < n ? 2 * tile : 2 * (n - 1 - tile) + 1; }

// The part of the line that starts at `unit`: units [from, upto) of one segment, the first `extra` of
// which hold no tile.
struct Part {
  Seq q;
  int seq, hk, r0;    // sequence, K/V head, first row
  int from, upto;
  bool whole;
};
template <int BK>
__device__ __forceinline__ Part part_at(const CacheArgs& c, const Few& f, const Line& line, int unit, int end) {
  const int kvh = c.pg.kv_heads;
  Part p;
  const int b = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)__ballot(line.upto > unit)) - 1);
  int at = __builtin_amdgcn_readlane(line.upto, b) - __builtin_amdgcn_readlane(line.mine, b), seq = b * line.per;
  auto held = [&](int v) { return __builtin_amdgcn_readlane(v, b); };
  Seq q{held(line.first.a), held(line.first.n), held(line.first.old), held(line.first.total), held(line.first.qt),
        held(line.first.nk)};
  for (int n = Line::count(q, kvh, line.cut); unit >= at + n; n = Line::count(q, kvh, line.cut)) {
    at += n;
    q = line_seq<BK>(c, f, ++seq);
  }
  auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  p.seq = uniform(seq);
  p.q = Seq{uniform(q.a), uniform(q.n), uniform(q.old), uniform(q.total), uniform(q.qt), uniform(q.nk)};
  const int rel = uniform(unit - at);
  const int seg = line.cut ? rel / p.q.nk : rel;
  p.from = line.cut ? rel - seg * p.q.nk : 0;
  p.upto = line.cut ? min(p.q.nk, p.from + end - unit) : p.q.nk;
  p.whole = p.from == 0 && p.upto == p.q.nk;
  // row tiles of a K/V head side by side: they read the same keys
  p.hk = seg / p.q.qt;
  p.r0 = folded(seg - p.hk * p.q.qt, p.q.qt) * FEW_BQ;
  return p;
}
// Neighbouring workgroups run on different XCDs: each XCD gets a stretch of the line.
__device__ __forceinline__ int place_of(int wg, int wgs) {
  const int xcd = wg & 7;
  return xcd * (wgs >> 3) + min(xcd, wgs & 7) + (wg >> 3);
}

// bf16, few rows: a workgroup is one wave with a ring of its own in LDS: nothing waits for
// another wave, and a tile of 16 KB is always in flight.
constexpr int FEW_STAGES = 2;
template <int D> constexpr int FEW_BK = D == 64 ? 64 : 32;     // 16 KB of K and V either way
// RUN: 8-key slabs that share a page for certain
template <int D, int RUN>
__global__ void __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(2, 8)))
cache_few(const CacheArgs c, const Few f) {
  constexpr int H2 = D / 64, BK = FEW_BK<D>, KT = BK / 32, SLABS = BK / 8;
  constexpr int TILE = BK * 8 * H2;              // uint4 of a K or V tile
  constexpr int NI = 2 * SLABS * H2;             // loads of a stage
  __shared__ uint4 kv[FEW_STAGES][2][TILE];      // [stage][K | V][half][key][8 chunks]
  const int lane = threadIdx.x, g = lane >> 5, r31 = lane & 31, kvh = c.pg.kv_heads;
  const Line line = line_of<BK>(c, f);
  if ((int)blockIdx.x >= line.wgs) return;
  const int wid = place_of(blockIdx.x, line.wgs);
  const int first = line.begin(wid), end = line.begin(wid + 1);

  const int lrow = lane >> 3;
  int off_k[2], off_v[2];                        // of even and odd 8-key slabs
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int col = 8 * ((lane & 7) ^ lds_swz(j * 8 + lrow));
    off_k[j] = (lrow * (int)c.pg.k_token + col) * 2;
    off_v[j] = (lrow * (int)c.pg.v_token + col) * 2;
  }
  // (operand layouts as in the kernel above)
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
  const float sc = LOG2E * c.scale;

  // What bf16 leaves of a weight may be zero or negative, and infinity times that is NaN: a part whose sums are
  // not finite is done again, with a look at every tile's values.
  bool look = false;
  for (int unit = first; unit < end;) {
    const Part p = part_at<BK>(c, f, line, unit, end);
    const Seq& q = p.q;
    // the segment starts this wave's units, or ends them behind others
    const int slot = 2 * wid + (unit != first), here = unit;
    unit += line.cut ? p.upto - p.from : 1;

    const int hk = p.hk, r0 = p.r0, left = min(q.n * c.group - r0, FEW_BQ), total = q.total;
    const Rows row_of(r0, c);
    const int t_last = row_of.token(left - 1);
    int lo, hi;
    key_range(c, q, row_of.tok, t_last, lo, hi);
    const int base = lo / BK, t0 = base + max(p.from - f.extra, 0), t1 = min(base + max(p.upto - f.extra, 0), (hi + BK - 1) / BK);
    const int mine = min(r31, left - 1), my_tok = row_of.token(mine);
    int lim = total - 1, low = 0, lim_first = total - 1, low_last = 0;
    if (c.causal) {
      lim = min(lim, q.old + my_tok);
      lim_first = min(lim_first, q.old + row_of.tok);
    }
    if (c.window) {
      low = max(q.old + my_tok - c.window + 1, 0);
      low_last = max(q.old + t_last - c.window + 1, 0);
    }
    const_i32* table = (const_i32*)(c.pg.table + p.seq * c.pg.table_ld);
    const bf16_t* k_head = (const bf16_t*)c.pg.k + hk * c.pg.k_head;
    const bf16_t* v_head = (const bf16_t*)c.pg.v + hk * c.pg.v_head;

    constexpr int RUNS = SLABS / RUN;
    // (always as many loads: what has no page stores zeros)
    auto issue = [&](int stage, int t, const int (&pages)[RUNS]) {
#pragma unroll
      for (int j = 0; j < RUNS; ++j) {
        const int key = t * BK + 8 * RUN * j, n = pages[j] < 0 ? 0 : min(total - key, 8 * RUN);
        const int64_t pg = max(pages[j], 0), slot = key & ((1 << c.pg.lg_page) - 1);
        const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc(
            (void*)(k_head + pg * c.pg.k_page + slot * c.pg.k_token), (short)0, n ? ((n - 1) * (int)c.pg.k_token + D) * 2 : 0,
            SWAM_BUF_DWORD3);
        const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc(
            (void*)(v_head + pg * c.pg.v_page + slot * c.pg.v_token), (short)0, n ? ((n - 1) * (int)c.pg.v_token + D) * 2 : 0,
            SWAM_BUF_DWORD3);
#pragma unroll
        for (int i = 0; i < RUN; ++i)
#pragma unroll
          for (int h = 0; h < H2; ++h) {
            const int slab = j * RUN + i;
            dma_slab(rk, &kv[stage][0][(h * SLABS + slab) * 64], vadd_sgpr(off_k[slab & 1], 128 * h + 16 * i * (int)c.pg.k_token));
            dma_slab(rv, &kv[stage][1][(h * SLABS + slab) * 64], vadd_sgpr(off_v[slab & 1], 128 * h + 16 * i * (int)c.pg.v_token));
          }
      }
    };

    f32x16 o[D / 32];
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[t][r] = 0.0f;
    float m_run = -FLT_MAX, l_run = 0.0f;

    // (behind the last tile there are no pages)
    const int stop = min(total, t1 * BK);
    int pages[RUNS];
    pages_of<RUNS, RUN>(c.pg, table, t0 * BK, stop, pages);
    uint64_t keys = keys_of<RUNS, RUN>(t0 * BK, total, pages), ahead;   // of the tile at hand and the next
    issue(0, t0, pages);
    pages_of<RUNS, RUN>(c.pg, table, (t0 + 1) * BK, stop, pages);
    bf16x8 qf[D / 16];
    {
      const bf16_t* qp = (const bf16_t*)c.q + (int64_t)(q.a + my_tok) * c.q_ld + (hk * c.group + row_of.head(mine)) * D;
#pragma unroll
      for (int s = 0; s < D / 16; ++s)
        qf[s] = __builtin_bit_cast(bf16x8, *(const uint4*)(qp + 8 * (2 * s + g)));
    }
    int buf = 0;
#pragma unroll 1
    for (int t = t0; t < t1; ++t, keys = ahead, buf ^= 1) {
        ahead = keys_of<RUNS, RUN>((t + 1) * BK, total, pages);
        reads_done();
        issue(buf ^ 1, t + 1, pages);
        pages_of<RUNS, RUN>(c.pg, table, (t + 2) * BK, stop, pages);
        wait_stage<NI>();
        if (keys == 0) continue;
        const uint4* Kt = kv[buf][0];
        const unsigned short* vs = reinterpret_cast<const unsigned short*>(kv[buf][1]);
        f32x16 st[KT];
#pragma unroll
        for (int x = 0; x < KT; ++x) {
#pragma unroll
          for (int r = 0; r < 16; ++r) st[x][r] = 0.0f;
#pragma unroll
          for (int s = 0; s < D / 16; ++s) {
            const bf16x8 kf = __builtin_bit_cast(bf16x8, Kt[(s >> 2) * BK * 8 + kofs[s & 3] + x * 32 * 8]);
            st[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[s], st[x], 0, 0, 0);
          }
        }
        const int k0 = t * BK, h = lim - k0, u = low - k0;
        constexpr uint64_t ALL = ~0ull >> (64 - BK);
        uint64_t sees = h < 0 ? 0 : h >= BK - 1 ? keys : keys & ((2ull << h) - 1);
        sees = u >= BK ? 0 : u > 0 ? sees & (~0ull << u) : sees;
        if (__any(sees != ALL)) {
          const uint64_t m = sees >> (4 * g);
          uint32_t bits[2] = {(uint32_t)m, (uint32_t)(m >> 32)};
          asm volatile("" : "+v"(bits[0]), "+v"(bits[1]));
#pragma unroll
          for (int x = 0; x < KT; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const uint32_t keep = (uint32_t)__builtin_amdgcn_sbfe((int)bits[x], 8 * (r >> 2) + (r & 3), 1);
              st[x][r] = __uint_as_float((__float_as_uint(st[x][r]) & keep) | (0xff800000u & ~keep));
            }
        }
        float mx = st[0][0];
#pragma unroll
        for (int x = 0; x < KT; ++x)
#pragma unroll
          for (int r = 0; r < 16; ++r) mx = fmaxf(mx, st[x][r]);
        // the running maximum moves only when some weight would pass 2^8
        if (__any(mx * sc > m_run + 8.0f)) {
          mx = fmaxf(mx, __shfl_xor(mx, 32));
          const float m_new = fmaxf(m_run, mx * sc), corr = __builtin_amdgcn_exp2f(m_run - m_new);
          m_run = m_new;
          l_run *= corr;
#pragma unroll
          for (int x = 0; x < D / 32; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[x][r] *= corr;
        }
        // P in bf16, the other operand's type, and what that leaves out as a second operand: the
        // bytes of K and V hide most of it (8 x 10,160 keys of 24 heads 97.8 us, with one product 96.1; 64 x 300
        // 40.7 and 39.1), and outputs are off by bf16's own 0.0017 of their size instead of 0.0024
        bf16x8 pf[KT][2], pl[KT][2];
        float ps0 = 0.0f, ps1 = 0.0f;
#pragma unroll
        for (int x = 0; x < KT; ++x)
#pragma unroll
          for (int r = 0; r < 16; r += 2) {
            const float p0 = __builtin_amdgcn_exp2f(fmaf(st[x][r], sc, -m_run));
            const float p1 = __builtin_amdgcn_exp2f(fmaf(st[x][r + 1], sc, -m_run));
            ps0 += p0; ps1 += p1;
            const __bf16 h0 = (__bf16)p0, h1 = (__bf16)p1;
            pf[x][r >> 3][r & 7] = h0; pf[x][r >> 3][(r & 7) + 1] = h1;
            pl[x][r >> 3][r & 7] = (__bf16)(p0 - (float)h0); pl[x][r >> 3][(r & 7) + 1] = (__bf16)(p1 - (float)h1);
          }
        l_run += ps0 + ps1;
        bool odd = false;
        if (look || (k0 + BK - 1 > lim_first && lim_first < total - 1) || k0 < low_last) {
          u16x2 top = {0, 0};
#pragma unroll
          for (int i = 0; i < TILE / 64; ++i) {
            const uint4 x = kv[buf][1][i * 64 + lane];
            const uint32_t x4[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
              top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, x4[e] & 0x7fff7fffu));
          }
          odd = __any(top[0] >= 0x7f80 || top[1] >= 0x7f80);
        }
        if (odd) {
#pragma unroll 1
          for (int key = 0; key < BK; ++key) {
            const bool see = (sees >> key) & 1u;
#pragma unroll
            for (int ht = 0; ht < D / 32; ++ht)
#pragma unroll
              for (int q4 = 0; q4 < 4; ++q4) {
                const int chunk = (4 * (ht & 1) + q4) ^ lds_swz(key);
                add_odd(o[ht], q4, see, *reinterpret_cast<const uint2*>(vs + (ht >> 1) * BK * 64 + key * 64 + 8 * chunk + 4 * g));
              }
          }
        }
        auto products = [&](auto clean) {
#pragma unroll
          for (int ht = 0; ht < D / 32; ++ht)
#pragma unroll
            for (int x = 0; x < KT; ++x)
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                const int at = (ht >> 1) * BK * 64 + (32 * x + 16 * u) * 64;
                const v4i16 x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(vs + vofs[ht & 1] + at));
                const v4i16 x2 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(vs + vofs[(ht & 1) ^ 1] + 8 * 64 + at));
                const uint2 w1 = __builtin_bit_cast(uint2, x1), w2 = __builtin_bit_cast(uint2, x2);
                const uint4 vf = clean(make_uint4(w1.x, w1.y, w2.x, w2.y));
                o[ht] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf), pf[x][u], o[ht], 0, 0, 0);
                o[ht] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf), pl[x][u], o[ht], 0, 0, 0);
              }
        };
        // (head_dim 128: the reads of V stay behind the softmax, or 256 registers do not hold them)
        if constexpr (D == 128) asm volatile("" ::: "memory");
        if (odd) products([](uint4 x) { return without_odd(x); });
        else products([](uint4 x) { return x; });
    }
    wait_stage<0>();                             // (the ring is free again)
    float odd4[4] = {0.0f, 0.0f, 0.0f, 0.0f};    // NaN where a sum is not finite
#pragma unroll
    for (int x = 0; x < D / 32; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) odd4[r & 3] = fmaf(o[x][r], 0.0f, odd4[r & 3]);
    look = !look && __any((odd4[0] + odd4[1]) + (odd4[2] + odd4[3]) != 0.0f);
    if (look) {
      unit = here;
      continue;
    }
    const float l = l_run + __shfl_xor(l_run, 32);
    const int64_t tok = q.a + my_tok;
    const int head = hk * c.group + row_of.head(mine);
    if (!p.whole) {
      if (r31 < left) {
        const int64_t row = (int64_t)slot * f.slot_rows + r31;
        float* po = f.o + row * D;
#pragma unroll
        for (int ht = 0; ht < D / 32; ++ht)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4)
            *reinterpret_cast<float4*>(po + 32 * ht + 8 * q4 + 4 * g) =
                make_float4(o[ht][4 * q4], o[ht][4 * q4 + 1], o[ht][4 * q4 + 2], o[ht][4 * q4 + 3]);
        if (g == 0) *reinterpret_cast<float2*>(f.ml + row * 2) = make_float2(m_run, l);
      }
      continue;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    bf16_t* op = (bf16_t*)c.o + tok * c.o_ld + head * D;
#pragma unroll
    for (int ht = 0; ht < D / 32; ++ht)
#pragma unroll
      for (int q4 = 0; q4 < 4; q4 += 2) {
        uint32_t v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          v[e] = pack_bf16x2(norm(o[ht][4 * q4 + 2 * e], inv), norm(o[ht][4 * q4 + 2 * e + 1], inv));
        const auto x = __builtin_amdgcn_permlane32_swap(v[0], v[2], false, false);
        const auto y = __builtin_amdgcn_permlane32_swap(v[1], v[3], false, false);
        if (r31 < left) *(uint4*)(op + 32 * ht + 8 * (q4 + g)) = make_uint4(x[0], y[0], x[1], y[1]);
      }
    if (c.lse != nullptr && g == 0 && r31 < left)
      c.lse[tok * c.heads + head] = l == 0.0f ? -INFINITY : (m_run + log2f(l)) * LN2;
  }
}

// float32: 32x32x2 MFMAs.  Four waves take every fourth tile of 32 keys of the same 32 rows and
// meet in LDS.  Each has room for one tile of K and one of V there: V is on its way during the
// scores, the next K during the products with V, so a wave never waits for both, and two
// waves share a SIMD.  What a part has at its start
// (its place in the line, pages, queries, first keys) is asked for before the sums of the part before it
// meet: 1,024 rows of 192 heads on 24 heads of 1,024 keys take a tenth less (now 462 us).
// Bound by the fp32 MFMA over long parts (8,192 x 8,192 keys, 24 heads: 3,320 us, 124 TFLOP/s) and by the parts'
// ends over short ones.  Operands read ahead of the products and weights formed between them made windowed
// chunks 4% slower.
template <int D, int RUN>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 64 ? 2 : 1, 8)))
cache_f32(const CacheArgs c, const Few f) {
  constexpr int H2 = D / 64, BK = 32, SLABS = BK / 8, RUNS = SLABS / RUN;
  constexpr int TILE = BK * 16 * H2;             // float4 of a K or V tile
  constexpr int NI = 8 * H2;                     // loads of one
  constexpr int NW = 4;
  __shared__ float4 kv[NW][2][TILE];             // [wave][K | V][half][key][16 chunks]
  __shared__ float ms[NW][32], ls[NW][32];
  // a part's sums meet in the places of V while the next part's first K is on its way: row r's chunk x
  // in place x ^ (r & 15)
  static_assert(TILE == 32 * D / 4, "a wave's sums fill its V tile");
  auto sum_at = [&](int w, int row, int x) -> float4& { return kv[w][1][(x >> 4) * 512 + row * 16 + ((x ^ row) & 15)]; };
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, r31 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Line line = line_of<BK>(c, f);
  if ((int)blockIdx.x >= line.wgs) return;
  const int wid = place_of(blockIdx.x, line.wgs);
  const int first = line.begin(wid), end = line.begin(wid + 1);

  // A load brings 4 keys of 256 bytes.  Chunk x of K's key r stands in place x ^ (r & 15), so that
  // 16 keys at one chunk (the scores' operand) hit every bank once; V's in x ^ 8 for every second
  // four keys, so that two rows 4 keys apart at 32 columns do.
  const int lrow = lane >> 4, lcol = 16 * (lane & 15), lcol_k = lcol ^ (16 * lrow);
  const int vofs[2] = {4 * g * 64 + r31 + 32 * g, 4 * g * 64 + r31 + 32 * (g ^ 1)};
  const float sc = LOG2E * c.scale;

  // the part whose sums wait in LDS
  struct { int a, hk, left, slot; bool whole; Rows rows; } last{0, 0, 0, 0, false, Rows(0, c)};
  int unit = first;
  auto join = [&]() {
    __syncthreads();                             // the waves' sums are there
    for (int row = tid >> 3; row < last.left; row += 8 * NW) {
      const int64_t tok = last.a + last.rows.token(row);
      const int head = last.hk * c.group + last.rows.head(row);
      float mt = ms[0][row];
#pragma unroll
      for (int v = 1; v < NW; ++v) mt = fmaxf(mt, ms[v][row]);
      float e4[NW], lt = 0.0f;
#pragma unroll
      for (int v = 0; v < NW; ++v) {
        e4[v] = exp2f(ms[v][row] - mt);
        lt = fmaf(ls[v][row], e4[v], lt);
      }
      const int64_t at = (int64_t)last.slot * f.slot_rows + row;
      const float inv = !last.whole ? 1.0f : lt == 0.0f ? 0.0f : 1.0f / lt;
      float* dst = last.whole ? (float*)c.o + tok * c.o_ld + head * D : f.o + at * D;
#pragma unroll
      for (int x = tid & 7; x < D / 4; x += 8) {
        float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int v = 0; v < NW; ++v) {
          const float4 y = sum_at(v, row, x);
          acc[0] = fmaf(y.x, e4[v], acc[0]);
          acc[1] = fmaf(y.y, e4[v], acc[1]);
          acc[2] = fmaf(y.z, e4[v], acc[2]);
          acc[3] = fmaf(y.w, e4[v], acc[3]);
        }
        *reinterpret_cast<float4*>(dst + 4 * x) = make_float4(norm(acc[0], inv), norm(acc[1], inv), norm(acc[2], inv), norm(acc[3], inv));
      }
      if ((tid & 7) == 0) {
        if (!last.whole) *reinterpret_cast<float2*>(f.ml + at * 2) = make_float2(mt, lt);
        else if (c.lse != nullptr) c.lse[tok * c.heads + head] = lt == 0.0f ? -INFINITY : (mt + log2f(lt)) * LN2;
      }
    }
    __syncthreads();                             // V's places are free again
  };
  while (unit < end) {
    const Part p = part_at<BK>(c, f, line, unit, end);
    const Seq& q = p.q;
    const int slot = 2 * wid + (unit != first);
    unit += line.cut ? p.upto - p.from : 1;

    const int hk = p.hk, r0 = p.r0, left = min(q.n * c.group - r0, FEW_BQ), total = q.total;
    const Rows row_of(r0, c);
    const int t_last = row_of.token(left - 1);
    int lo, hi;
    key_range(c, q, row_of.tok, t_last, lo, hi);
    const int base = lo / BK, t0 = base + max(p.from - f.extra, 0), t1 = min(base + max(p.upto - f.extra, 0), (hi + BK - 1) / BK);
    const int mine = min(r31, left - 1), my_tok = row_of.token(mine);
    int lim = total - 1, low = 0, lim_first = total - 1, low_last = 0;
    if (c.causal) {
      lim = min(lim, q.old + my_tok);
      lim_first = min(lim_first, q.old + row_of.tok);
    }
    if (c.window) {
      low = max(q.old + my_tok - c.window + 1, 0);
      low_last = max(q.old + t_last - c.window + 1, 0);
    }
    const_i32* table = (const_i32*)(c.pg.table + p.seq * c.pg.table_ld);
    const float* k_head = (const float*)c.pg.k + hk * c.pg.k_head;
    const float* v_head = (const float*)c.pg.v + hk * c.pg.v_head;
    // (always as many loads: what has no page stores zeros)
    auto issue = [&](bool is_v, int t, const int (&pages)[RUNS]) {
      float4* to = kv[wave][is_v];
      const float* head = is_v ? v_head : k_head;
      const int64_t page_ld = is_v ? c.pg.v_page : c.pg.k_page, token_ld = is_v ? c.pg.v_token : c.pg.k_token;
      const int row = lrow * (int)token_ld * 4;
#pragma unroll
      for (int j = 0; j < RUNS; ++j) {
        const int key = t * BK + 8 * RUN * j, n = pages[j] < 0 ? 0 : min(total - key, 8 * RUN);
        const int64_t pg = max(pages[j], 0), at = key & ((1 << c.pg.lg_page) - 1);
        const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
            (void*)(head + pg * page_ld + at * token_ld), (short)0, n ? ((n - 1) * (int)token_ld + D) * 4 : 0, SWAM_BUF_DWORD3);
#pragma unroll
        for (int i = 0; i < 2 * RUN; ++i)
#pragma unroll
          for (int h = 0; h < H2; ++h) {
            const int four = 2 * RUN * j + i;    // 4 keys
            dma_slab(r, (uint4*)&to[(h * 2 * SLABS + four) * 64],
                     vadd_sgpr(row + (is_v ? lcol ^ ((four & 1) << 7) : lcol_k ^ ((four & 3) << 6)), 256 * h + 16 * i * (int)token_ld));
          }
      }
    };
    f32x4 qf[D / 8];
    {
      const float* qp = (const float*)c.q + (int64_t)(q.a + my_tok) * c.q_ld + (hk * c.group + row_of.head(mine)) * D;
#pragma unroll
      for (int s = 0; s < D / 8; ++s) qf[s] = *reinterpret_cast<const f32x4*>(qp + 4 * (2 * s + g));
    }
    const float4* Kt = kv[wave][0];
    const float4* Vt = kv[wave][1];
    const int stop = min(total, t1 * BK);
    int pages[RUNS], ahead[RUNS];
    pages_of<RUNS, RUN>(c.pg, table, (t0 + wave) * BK, stop, pages);
    issue(false, t0 + wave, pages);
    if (slot != 2 * wid) join();
    f32x16 o[D / 32];
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[t][r] = 0.0f;
    float m = -FLT_MAX, l = 0.0f;
#pragma unroll 1
    for (int t = t0 + wave; t < t1; t += NW) {
      const int k0 = t * BK;
      reads_done();
      issue(true, t, pages);
      pages_of<RUNS, RUN>(c.pg, table, k0 + NW * BK, stop, ahead);
      const uint32_t vis = (uint32_t)keys_of<RUNS, RUN>(k0, total, pages);
      wait_stage<NI>();
      f32x16 st;
#pragma unroll
      for (int r = 0; r < 16; ++r) st[r] = 0.0f;
#pragma unroll
      for (int s = 0; s < D / 8; ++s) {
        const float4 kf = Kt[(s >> 3) * BK * 16 + r31 * 16 + ((2 * (s & 7) + g) ^ (r31 & 15))];
        st = __builtin_amdgcn_mfma_f32_32x32x2f32(kf.x, qf[s][0], st, 0, 0, 0);
        st = __builtin_amdgcn_mfma_f32_32x32x2f32(kf.y, qf[s][1], st, 0, 0, 0);
        st = __builtin_amdgcn_mfma_f32_32x32x2f32(kf.z, qf[s][2], st, 0, 0, 0);
        st = __builtin_amdgcn_mfma_f32_32x32x2f32(kf.w, qf[s][3], st, 0, 0, 0);
      }
      reads_done();
      issue(false, t + NW, ahead);
#pragma unroll
      for (int j = 0; j < RUNS; ++j) pages[j] = ahead[j];
      // the keys that this lane's row sees
      const int h = lim - k0, u = low - k0;
      uint32_t sees = h < 0 ? 0u : h >= BK - 1 ? vis : vis & ((2u << h) - 1);
      sees = u > 31 ? 0u : u > 0 ? sees & (~0u << u) : sees;
      if (__any(sees != ~0u)) {
        uint32_t bits = sees >> (4 * g);
        asm volatile("" : "+v"(bits));
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const uint32_t keep = (uint32_t)__builtin_amdgcn_sbfe((int)bits, 8 * (r >> 2) + (r & 3), 1);
          st[r] = __uint_as_float((__float_as_uint(st[r]) & keep) | (0xff800000u & ~keep));
        }
      }
      float mx = st[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) mx = fmaxf(mx, st[r]);
      // the running maximum moves only when some weight would pass 2^8
      if (__any(mx * sc > m + 8.0f)) {
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float m_new = fmaxf(m, mx * sc), corr = __builtin_amdgcn_exp2f(m - m_new);
        m = m_new;
        l *= corr;
#pragma unroll
        for (int x = 0; x < D / 32; ++x)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[x][r] *= corr;
      }
      wait_stage<NI>();
      // a weight of zero does not hide a value that is not finite: where rows see different keys
      // such values are left out of the products and added by hand
      bool odd = false;
      if ((k0 + BK - 1 > lim_first && lim_first < total - 1) || k0 < low_last) {
#pragma unroll
        for (int i = 0; i < TILE / 64; ++i) {
          const float4 x = Vt[i * 64 + lane];
          odd |= !(fmaxf(fmaxf(fabsf(x.x), fabsf(x.y)), fmaxf(fabsf(x.z), fabsf(x.w))) <= FLT_MAX) || x.x != x.x ||
                 x.y != x.y || x.z != x.z || x.w != x.w;
        }
        odd = __any(odd);
      }
      if (odd) {
#pragma unroll 1
        for (int key = 0; key < BK; ++key) {
          const bool see = (sees >> key) & 1u;
#pragma unroll
          for (int x = 0; x < D / 32; ++x)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
              const float4 v = Vt[(x >> 1) * BK * 16 + key * 16 + ((8 * (x & 1) + 2 * q4 + g) ^ (2 * (key & 4)))];
              const float e4[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
              for (int e = 0; e < 4; ++e)
                o[x][4 * q4 + e] += see && !(fabsf(e4[e]) <= FLT_MAX) ? e4[e] : 0.0f;
            }
        }
      }
      float w[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        w[r] = __builtin_amdgcn_exp2f(fmaf(st[r], sc, -m));
        l += w[r];
      }
      auto products = [&](auto clean) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
#pragma unroll
          for (int x = 0; x < D / 32; ++x) {
            const float v = reinterpret_cast<const float*>(Vt)[vofs[x & 1] + (x >> 1) * BK * 64 + (8 * (r >> 2) + (r & 3)) * 64];
            o[x] = __builtin_amdgcn_mfma_f32_32x32x2f32(clean(v), w[r], o[x], 0, 0, 0);
          }
      };
      if (odd) products([](float v) { return fabsf(v) <= FLT_MAX ? v : 0.0f; });
      else products([](float v) { return v; });
    }
    wait_stage<0>();
    l += __shfl_xor(l, 32);
    if (g == 0) { ms[wave][r31] = m; ls[wave][r31] = l; }
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
        sum_at(wave, r31, 8 * t + 2 * q4 + g) = make_float4(o[t][4 * q4], o[t][4 * q4 + 1], o[t][4 * q4 + 2], o[t][4 * q4 + 3]);
    last = {q.a, hk, left, slot, p.whole, row_of};
  }
  join();
}

// The segment that the border behind workgroup j's units cuts, where j has its start: a
// workgroup for each border.
template <typename T, int D, int BK>
__global__ void __launch_bounds__(256)
line_join(const CacheArgs c, const Few f) {
  const Line line = line_of<BK>(c, f);
  const int j = blockIdx.x;
  if (!line.cut || j + 1 >= line.wgs) return;
  const int begin = line.begin(j), end = line.begin(j + 1);
  const Part p = part_at<BK>(c, f, line, end - 1, end);
  const int start = end - 1 - p.from;
  if (start < begin || start + p.q.nk <= end) return;
  const int ch = line.wg_of(start + p.q.nk - 1) - j + 1, left = min(p.q.n * c.group - p.r0, FEW_BQ);
  const Rows row_of(p.r0, c);
  // j's may be the end of its units, the others' start theirs
  auto slot_at = [&](int y) { return 2 * (j + y) + (y == 0 && start != begin); };
  if (ch > 8) join_rows<T, D, 16>(c, f.o, f.ml, f.slot_rows, ch, p.q.a, p.hk, row_of, 0, left, slot_at);
  else join_rows<T, D, 8>(c, f.o, f.ml, f.slot_rows, ch, p.q.a, p.hk, row_of, 0, left, slot_at);
}
// The same for few rows, which have many partial results each: a workgroup of NW waves per
// token and head, each wave every NW-th group of them.
template <typename T, int D, int BK, int NW>
__global__ void __launch_bounds__(64 * NW)
line_join_row(const CacheArgs c, const Few f) {
  constexpr int PER = D / 4, SETS = 64 / PER, AHEAD = 8;
  __shared__ float4 os[NW][PER];
  __shared__ float2 mls[NW];
  const Line line = line_of<BK>(c, f);
  if (!line.cut) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, kvh = c.pg.kv_heads;
  const int set = lane / PER, col = lane % PER * 4;
  const int n = c.n_q * c.heads;
  for (int id = blockIdx.x; id < n; id += gridDim.x) {
    const int tok = id / c.heads, head = id % c.heads;
    int s = seq_of(c.pg, tok);
    Seq q = line_seq<BK>(c, f, s);
    if (tok < q.a || tok >= q.a + q.n) {         // offsets that fall, or nobody's
      s = seq_that_holds(c.pg, tok);
      if (s < 0) continue;
      q = line_seq<BK>(c, f, s);
    }
    if (q.nk == 0) continue;
    // tiles in front of the sequence
    int before = __shfl(line.upto, s / line.per) - __shfl(line.mine, s / line.per);
    for (int i = s / line.per * line.per; i < s; ++i) before += Line::count(line_seq<BK>(c, f, i), kvh, true);
    const int r = (tok - q.a) * c.group + head % c.group, qi = r / FEW_BQ;
    const int a = before + (head / c.group * q.qt + fold_index(qi, q.qt)) * q.nk;
    const int w0 = line.wg_of(a), ch = line.wg_of(a + q.nk - 1) - w0 + 1;
    if (ch == 1) continue;
    // the first one's may be the end of its units, the others' start theirs
    const int begins = line.begin(w0) == a;
    auto row_at = [&](int y) -> int64_t {
      return (int64_t)(2 * (w0 + y) + (y == 0 && !begins)) * f.slot_rows + r % FEW_BQ;
    };
    // each group of lanes with a maximum of its own
    float m = -FLT_MAX, l = 0.0f;
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int y0 = wave * SETS * AHEAD; y0 < ch; y0 += NW * SETS * AHEAD) {
      float4 v[AHEAD];
      float2 w[AHEAD];
#pragma unroll
      for (int x = 0; x < AHEAD; ++x) {
        const int y = y0 + SETS * x + set;
        const int64_t at = row_at(min(y, ch - 1));
        w[x] = *reinterpret_cast<const float2*>(f.ml + at * 2);
        v[x] = *reinterpret_cast<const float4*>(f.o + at * D + col);
        if (y >= ch) w[x] = make_float2(-FLT_MAX, 0.0f);
      }
      float m_new = m;
#pragma unroll
      for (int x = 0; x < AHEAD; ++x) m_new = fmaxf(m_new, w[x].x);
      const float corr = exp2f(m - m_new);
      m = m_new;
      l *= corr;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] *= corr;
#pragma unroll
      for (int x = 0; x < AHEAD; ++x) {
        if (y0 + SETS * x + set < ch) {
          const float e = exp2f(w[x].x - m);
          l = fmaf(w[x].y, e, l);
          acc[0] = fmaf(v[x].x, e, acc[0]);
          acc[1] = fmaf(v[x].y, e, acc[1]);
          acc[2] = fmaf(v[x].z, e, acc[2]);
          acc[3] = fmaf(v[x].w, e, acc[3]);
        }
      }
    }
    float mt = m;
#pragma unroll
    for (int x = PER; x < 64; x <<= 1) mt = fmaxf(mt, __shfl_xor(mt, x));
    const float e0 = exp2f(m - mt);
    l *= e0;
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] *= e0;
#pragma unroll
    for (int x = PER; x < 64; x <<= 1) {
      l += __shfl_xor(l, x);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], x);
    }
    __syncthreads();                             // (the last row's are read)
    if (set == 0) os[wave][lane] = make_float4(acc[0], acc[1], acc[2], acc[3]);
    if (lane == 0) mls[wave] = make_float2(mt, l);
    __syncthreads();
    if (wave == 0 && set == 0) {
      float top = -FLT_MAX, sum = 0.0f;
#pragma unroll
      for (int v = 0; v < NW; ++v) top = fmaxf(top, mls[v].x);
      float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int v = 0; v < NW; ++v) {
        const float e = exp2f(mls[v].x - top);
        const float4 p = os[v][lane];
        sum = fmaf(mls[v].y, e, sum);
        x[0] = fmaf(p.x, e, x[0]);
        x[1] = fmaf(p.y, e, x[1]);
        x[2] = fmaf(p.z, e, x[2]);
        x[3] = fmaf(p.w, e, x[3]);
      }
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
      T* op = (T*)c.o + tok * c.o_ld + head * D + col;
      if constexpr (sizeof(T) == 2)
        *reinterpret_cast<uint2*>(op) = make_uint2(pack_bf16x2(norm(x[0], inv), norm(x[1], inv)), pack_bf16x2(norm(x[2], inv), norm(x[3], inv)));
      else
        *reinterpret_cast<float4*>(op) = make_float4(norm(x[0], inv), norm(x[1], inv), norm(x[2], inv), norm(x[3], inv));
      if (c.lse != nullptr && lane == 0) c.lse[id] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * LN2;
    }
  }
}

template <typename T, int D>
static void run_line(const CacheArgs& c, float* ws, int64_t ws_floats, hipStream_t st) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int BK = F32 ? 32 : FEW_BK<D>, SLABS = BK / 8;
  const int64_t rows = (int64_t)c.n_q * c.group;
  Few f{};
  f.slot_rows = (int)std::min<int64_t>(FEW_BQ, rows);
  // A segment's start and end take about as long as this many tiles (passes with the joining one): 64 x 1 token of
  // 20 to 10,161 keys without them 55.5 us, with one, two, four 50.2, 50.5, 51.7; eight float32 chunks of 100 to
  // 326 rows behind 6 to 3,000 keys 97.2 us with none, 92.2 with four, 96.2 with eight, 107.5 with sixteen.
  f.extra = F32 ? 4 : 1;
  // bf16: one wave to a SIMD, 64 KB in flight on a CU: 8 x 10,160 keys of 24 heads 97.8 us, 1 x 139,776
  // of 4 heads of 128 64.1, 64 x 300 of 24 heads 40.7; with three to a CU 98.8, 65.8 and 42.8, with five (a SIMD
  // then has two) 128, 80 and 56.
  // float32: as many workgroups as the LDS holds.
  f.wgs = 256 * (!F32 ? 4 : D == 64 ? 2 : 1);
  f.cut = (int)std::max<int64_t>(0, std::min<int64_t>(f.wgs, ws_floats / (2 * (int64_t)f.slot_rows * (D + 2))));
  // nothing to cut, and no pass to join it, where a table holds two tiles
  if ((int64_t)c.pg.max_pages << c.pg.lg_page <= 2 * BK) f.cut = 0;
  f.o = ws;
  f.ml = ws + 2 * (int64_t)f.cut * f.slot_rows * D;
  auto launch = [&](auto run) {
    constexpr int RUN = decltype(run)::value;
    if constexpr (F32) hipLaunchKernelGGL((cache_f32<D, RUN>), dim3(f.wgs), dim3(256), 0, st, c, f);
    else hipLaunchKernelGGL((cache_few<D, RUN>), dim3(f.wgs), dim3(64), 0, st, c, f);
  };
  const int run = std::min(1 << c.pg.lg_page >> 3, SLABS);
  if (run == 1) launch(std::integral_constant<int, 1>{});
  else if (run == 2) launch(std::integral_constant<int, 2>{});
  else if (run == 4) launch(std::integral_constant<int, 4>{});
  else launch(std::integral_constant<int, SLABS>{});
  if (f.cut) {
    const int64_t n = (int64_t)c.n_q * c.heads;
    if (n <= 64) hipLaunchKernelGGL((line_join_row<T, D, BK, 16>), dim3((unsigned)n), dim3(1024), 0, st, c, f);
    else if (n <= 512) hipLaunchKernelGGL((line_join_row<T, D, BK, 4>), dim3((unsigned)n), dim3(256), 0, st, c, f);
    else hipLaunchKernelGGL((line_join<T, D, BK>), dim3(f.cut), dim3(256), 0, st, c, f);
  }
}

// bf16 chunks
template <int D>
static void run_chunk(const CacheArgs& c, float* ws, int64_t ws_floats, hipStream_t st) {
  constexpr int BQ = 128;
  const int kvh = c.pg.kv_heads;
  // row tiles at most and at least: the chunks' lengths are on the device
  const int64_t rows = (int64_t)c.n_q * c.group;
  const int64_t most = std::min((rows + (int64_t)(BQ - 1) * c.pg.n_seqs) / BQ, rows), least = (rows + BQ - 1) / BQ;
  Split sp{};
  sp.slot_rows = (int)std::min<int64_t>(BQ, rows);
  // Keys are split, as far as the workspace holds the partial results (at most two per slice of
  // the budget), unless the row tiles fill the card: those of one sequence are as long
  // as each other, those of several may not be.  Split and whole, us: one sequence of 24 heads behind 20,000 keys,
  // 48 row tiles 85 and 177, 96 146 and 179, 144 207 and 183, 192 211 and 189, 240 212 and 204; several, 576 tiles
  // of unequal contexts 43 and 84, 1,536 of equal ones 97 and 92, 3,072 163 and 153.  1,024 slices: with 256
  // the unequal contexts take 86 us, though the first two of one sequence 59 and 108.
  if (least * kvh < (c.pg.n_seqs == 1 ? 192 : 2048)) {
    const int64_t fit = (ws_floats - 64) / (2 * (int64_t)sp.slot_rows * (D + 2));
    sp.budget = (int)std::min<int64_t>(1024, std::max<int64_t>(fit, 0));
    sp.plan = (int*)ws;
    sp.o = ws + 64;
    sp.ml = sp.o + 2 * (int64_t)sp.budget * sp.slot_rows * D;
  }
  const int64_t units = most + sp.budget / kvh;
  // a grid holds less than 2^32 threads: more take another launch
  const int64_t step = ((1 << 24) - 1) / kvh;
  auto launch_with = [&](auto run, auto groups) {
    constexpr int RUN = decltype(run)::value, KG = decltype(groups)::value;
    // (a sequence of few rows is here only beside others, or where offsets leave rows out)
    const auto kernel = c.pg.cu != nullptr ? cache_bf16<D, RUN, KG, true> : cache_bf16<D, RUN, KG, false>;
    for (int64_t u = 0; u < units; u += step)
      hipLaunchKernelGGL(kernel, dim3((unsigned)(std::min(units - u, step) * kvh)), dim3(256 * KG), 0, st, c, sp, (int)u);
  };
  // Few row tiles: one workgroup to a CU that takes several key tiles at once, as many as the LDS
  // holds.  With groups and without, us: chunks of 24 heads of 64 behind 2,000 keys, 192 row tiles 34 and 55, 240 38
  // and 61, 384 66 and 75, 528 105 and 92, 648 124 and 114; of 4 K/V heads of 128, 252 73 and 103, 512 154 and 178,
  // 752 both 285.
  auto launch = [&](auto run) {
    if (most * kvh <= 640) launch_with(run, std::integral_constant<int, D == 64 ? 4 : 2>{});
    else launch_with(run, std::integral_constant<int, 1>{});
  };
  switch (std::min(c.pg.lg_page, 6)) {
    case 3: launch(std::integral_constant<int, 1>{}); break;
    case 4: launch(std::integral_constant<int, 2>{}); break;
    case 5: launch(std::integral_constant<int, 4>{}); break;
    default: launch(std::integral_constant<int, 8>{});
  }
  if (sp.budget)                                // (row tiles below 2,048 + n_seqs here)
    hipLaunchKernelGGL((cache_join<D>), dim3((unsigned)(most * kvh), (unsigned)((sp.slot_rows + 31) / 32)), dim3(256), 0, st, c, sp);
}

template <int D>
static void run_cache(int dtype, const CacheArgs& c, float* ws, int64_t ws_floats, hipStream_t st) {
  // Few rows to a sequence, by the mean that the host knows; also twice as many where there are few
  // row tiles in all, which the line cuts finer: one chunk of 64 rows behind 10,000 keys, 3 heads of 128,
  // 27 us on the line and 53 in slices, 24 heads of 64 43 and 47; eight such of 24 heads behind
  // 2,000 55 and 42.  (The mean goes wrong where one long chunk stands among many sequences that are idle: 20,000
  // tokens of 12 heads among 1,024 take 2,040 us, alone 690.)
  const int64_t rows = (int64_t)c.n_q * c.group;
  const bool few = rows <= (int64_t)FEW_BQ * c.pg.n_seqs ||
                   (rows <= 2 * (int64_t)FEW_BQ * c.pg.n_seqs && rows * c.pg.kv_heads <= FEW_BQ * 128);
  if (dtype != 1) run_line<float, D>(c, ws, ws_floats, st);
  else if (few) run_line<bf16_t, D>(c, ws, ws_floats, st);
  else run_chunk<D>(c, ws, ws_floats, st);
}

hipError_t launch_cache_attention(int dtype, const CacheArgs& c, float* ws, int64_t ws_floats, hipStream_t st) {
  if (c.n_q <= 0) return hipSuccess;
  if (c.dim == 64) run_cache<64>(dtype, c, ws, ws_floats, st);
  else run_cache<128>(dtype, c, ws, ws_floats, st);
  return hipGetLastError();
}

}  // namespace swam
