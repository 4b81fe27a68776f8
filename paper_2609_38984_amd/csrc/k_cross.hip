// Attention of query tokens to the states of an encoder: another length than the
// queries', grouped K/V heads, padding masks, prompts shared by sequences.
//
// The rows of a tile are (query token, head of the group) pairs of one sequence
// and one K/V head, so that every head that reads a K/V head reads it from the
// same tile.  bf16: S^T = K Q^T and O^T = V^T P^T on 32x32x16 MFMAs, one row per
// lane (lane & 31) and the keys in the accumulator registers, as in the block's
// self attention: row maxima and sums need one exchange, and P^T is the next
// operand as it stands.  K and V tiles of 64 keys go global -> LDS by buffer
// loads; a hidden key's lanes get an offset past the descriptor's end and store
// zeros, so what padding holds never reaches a product.
// Softmax in one pass with a running maximum (base 2, float32).
//
// What bounds it: for many rows the instructions of a score (head_dim 64, per wave and
// tile: 16 MFMAs of 32 cycles, 32 exponentials of 8, 81 other vector operations, which
// overlap with other waves' MFMAs in part: two waves of each take 83 cycles (exponentials,
// products) to 113 (fused, conversions) where either kind alone takes 64 to 69; additions,
// 35 alone, come on top in full)
// and, on few keys, the queries and outputs (10,160 rows of 24 heads on one tile 20 us for
// 62 MB, 4 us more for each further tile); for single queries the bytes of K and V (8 x
// 10,160 keys of 24 heads 100 us, 499 MB at 5.0 TB/s).  4,096 x 4,096 at head_dim 128 and
// 16 heads 138 us: 1,000 TFLOP/s.
#include "gemm_common.h"

#include <algorithm>
#include <cfloat>

namespace swam {

typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16;

constexpr int CR_BK = 64;                      // keys per tile: one bit of a mask word each
constexpr int CR_PAST_END = 0x7fffff00;        // an offset that no tile reaches
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// The sequence that holds tile t of `bq` rows (rows are tokens x group): lane b
// looks at sequence b and its keys, a scan over the lanes finds the one.
struct TileAt {
  int a, rows;        // first token, token x group rows of the sequence
  int r0;             // first row of the tile
  int s0, s1;         // its keys
};
__device__ __forceinline__ bool tile_at(const CrossArgs& c, int group, int bq, int t, TileAt& o) {
  const int lane = threadIdx.x & 63;
  int a = 0, e = 0, s0 = 0, s1 = 0;
  if (lane < c.n_seqs) {
    const int kb = c.kv_seq ? c.kv_seq[lane] : lane;
    e = c.cu_q ? min(max(c.cu_q[lane + 1], 0), c.n_q) : c.n_q;
    a = c.cu_q ? min(max(c.cu_q[lane], 0), e) : 0;
    if (kb >= 0 && kb < c.n_kv_seqs) {
      s1 = c.cu_k ? min(max(c.cu_k[kb + 1], 0), c.n_k) : c.n_k;
      s0 = c.cu_k ? min(max(c.cu_k[kb], 0), s1) : 0;
    }
  }
  const int nt = ((e - a) * group + bq - 1) / bq;
  int upto = nt;
  for (int s = 1; s < c.n_seqs; s <<= 1) {
    const int v = __shfl_up(upto, s);
    if (lane >= s) upto += v;
  }
  const uint64_t past = __ballot(upto > t);
  if (past == 0) return false;
  const int b = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)past) - 1);
  o.a = __builtin_amdgcn_readlane(a, b);
  o.rows = (__builtin_amdgcn_readlane(e, b) - o.a) * group;
  o.r0 = (t - (__builtin_amdgcn_readlane(upto, b) - __builtin_amdgcn_readlane(nt, b))) * bq;
  o.s0 = __builtin_amdgcn_readlane(s0, b);
  o.s1 = __builtin_amdgcn_readlane(s1, b);
  return true;
}

// tiles [t0, t1) of the keys of slice y of 2^lg
__device__ __forceinline__ void slice_of(int s0, int s1, int bk, int y, int lg, int& t0, int& t1) {
  const int64_t n = (s1 - s0 + bk - 1) / bk;
  t0 = (int)(n * y >> lg);
  t1 = (int)(n * (y + 1) >> lg);
}

// partial results of slice y: [y][token][head][head_dim] sums, then [y][token][head][2]
// (maximum, sum)
struct Partial {
  float* o;
  float* ml;
  int splits, lg;     // splits = 2^lg
};

// Four waves of 32 rows each.  The registers decide at head_dim 64: with 128 of them four
// waves share a SIMD, and what one waits for (LDS, its own chain from scores to weights
// to products) the others hide.  So a tile has one body, masked behind a branch (a second
// one for whole tiles keeps more alive: 154 registers, three waves), and what only the
// end needs is formed there.  Four waves | three, 24 heads: 10,160 rows on 512 keys 47 us
// | 56, on 2,048 156 | 183; 4,096 rows on 10,160 295 | 338 (870 TFLOP/s).
template <int D>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 64 ? 4 : 2, 8)))
cross_bf16(const CrossArgs c, const Partial part) {
  constexpr int H2 = D / 64;                     // 128-byte halves of a head's row
  constexpr int NW = 4, BQ = 32 * NW;
  constexpr int TILE = CR_BK * 8 * H2;           // uint4 of a K or V tile
  __shared__ uint4 kv[2][2][TILE];               // [stage][K | V][half][key][8 chunks]
  const int group = c.heads / c.kv_heads;
  // neighbouring workgroups take the K/V heads in turn: with a multiple of 8 of them a
  // head stays on one XCD, and every XCD gets a share of every sequence, long or empty
  const int hk = blockIdx.x % c.kv_heads;
  TileAt ta;
  if (!tile_at(c, group, BQ, blockIdx.x / c.kv_heads, ta)) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 5, r31 = lane & 31;
  bf16x8 qf[D / 16];
  {
    const int rr = min(ta.r0 + wave * 32 + r31, ta.rows - 1);
    const int64_t tok = ta.a + rr / group;
    const int head = hk * group + rr % group;
    const bf16_t* qp = (const bf16_t*)c.q + tok * c.q_ld + head * D;
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
      qf[s] = __builtin_bit_cast(bf16x8, *(const uint4*)(qp + 8 * (2 * s + g)));
  }
  int t0, t1;
  slice_of(ta.s0, ta.s1, CR_BK, blockIdx.y, part.lg, t0, t1);

  // whether this lane's key of tile t is visible
  auto mask_byte = [&](int t) -> int {
    const int key = ta.s0 + t * CR_BK + __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
    return t < t1 && key < ta.s1 && (c.mask == nullptr || c.mask[key] != 0);
  };
  const int lrow = lane >> 3;
  constexpr int SLABS = 8 * H2;                  // 8-row slabs of a tile
  static_assert(SLABS % NW == 0, "every wave stages whole slabs");
  int off_k[SLABS / NW], off_v[SLABS / NW];
#pragma unroll
  for (int j = 0; j < SLABS / NW; ++j) {
    const int slab = wave * (SLABS / NW) + j, half = slab >> 3;
    const int r = (slab & 7) * 8 + lrow, col = 64 * half + 8 * ((lane & 7) ^ lds_swz(r));
    off_k[j] = (r * (int)c.k_ld + col) * 2;
    off_v[j] = (r * (int)c.v_ld + col) * 2;
  }
  // K and V of tile t into LDS; hidden keys are zeros
  auto issue = [&](uint4 (&to)[2][TILE], int t, uint64_t vis) {
    const int64_t row = ta.s0 + (int64_t)t * CR_BK;
    const int rows = min(ta.s1 - (int)row, CR_BK);
    const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc(
        (void*)((const bf16_t*)c.k + row * c.k_ld + hk * D), (short)0, ((rows - 1) * (int)c.k_ld + D) * 2, SWAM_BUF_DWORD3);
    const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc(
        (void*)((const bf16_t*)c.v + row * c.v_ld + hk * D), (short)0, ((rows - 1) * (int)c.v_ld + D) * 2, SWAM_BUF_DWORD3);
    const int at = wave * (SLABS / NW) * 64;
    if (vis == ~(uint64_t)0) {
#pragma unroll
      for (int j = 0; j < SLABS / NW; ++j) {
        dma_slab(rk, &to[0][at + j * 64], off_k[j]);
        dma_slab(rv, &to[1][at + j * 64], off_v[j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < SLABS / NW; ++j) {
        const bool see = (vis >> (8 * ((wave * (SLABS / NW) + j) & 7) + lrow)) & 1;
        dma_slab(rk, &to[0][at + j * 64], see ? off_k[j] : CR_PAST_END);
        dma_slab(rv, &to[1][at + j * 64], see ? off_v[j] : CR_PAST_END);
      }
    }
  };
  // V^T operand by transposed LDS reads: in each 16-lane group lane a addresses
  // V[key0 + (a >> 2)][col0 + 4 (a & 3)] and lane i receives keys key0..key0+3 of
  // column col0 + i, the order in which the P^T accumulators hold the keys
  const int a16 = lane & 15, G = lane >> 4, rlo = 4 * g + (a16 >> 2);
  // (8 rows or 32 columns further the swizzle flips the same bit of the chunk)
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

  // one tile of keys; `fresh`: the first visible one
  auto tile = [&](const uint4 (&from)[2][TILE], uint64_t vis, bool fresh) {
    const uint4* Kt = from[0];
    auto scores = [&](f32x16 (&st)[2], uint64_t vis) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int r = 0; r < 16; ++r) st[t][r] = 0.0f;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
          const bf16x8 kf = __builtin_bit_cast(bf16x8, Kt[(s >> 2) * CR_BK * 8 + kofs[s & 3] + t * 32 * 8]);
          st[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[s], st[t], 0, 0, 0);
        }
        if (vis != ~(uint64_t)0) {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            // register r holds key b of the lower 32 lanes and key b + 4 of the upper: the
            // select's mask is two scalar bits spread
            const int b = 32 * t + 8 * (r >> 2) + (r & 3);
            const uint64_t see = ((vis >> b) & 1 ? 0xffffffffull : 0) | ((vis >> (b + 4)) & 1 ? 0xffffffffull << 32 : 0);
            if (!__builtin_amdgcn_inverse_ballot_w64(see)) st[t][r] = -INFINITY;
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
            // P in bf16, the other operand's type; the sum keeps float32.  Outputs are off by
            // 0.0023 of their size where bf16 itself makes 0.0017; the rest of P as a second
            // operand gives the 0.0017 and takes 80 us for 71 (8 sequences of up to 3,360, 12
            // heads of 128), 61 for 45 (10,160 x 24 heads on 512), 133 for 106 (8 x 1 on 10,160)
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
      // formed anew: neither operands nor masks of the first time are kept for this
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
#pragma unroll
    for (int ht = 0; ht < D / 32; ++ht)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int base = (ht >> 1) * CR_BK * 64 + (32 * t + 16 * u) * 64;
          const v4i16 x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(vs + vofs[ht & 1] + base));
          const v4i16 x2 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(vs + vofs[(ht & 1) ^ 1] + 8 * 64 + base));
          const uint2 w1 = __builtin_bit_cast(uint2, x1), w2 = __builtin_bit_cast(uint2, x2);
          const bf16x8 vf = __builtin_bit_cast(bf16x8, make_uint4(w1.x, w1.y, w2.x, w2.y));
          o[ht] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[t][u], o[ht], 0, 0, 0);
        }
  };

  // All waves of the workgroup form the same mask words: that of the tile at hand, of the
  // next, whose loads run meanwhile, and the bytes of the one after it.  A tile without a
  // visible key is neither loaded nor multiplied.
  uint64_t vis = __ballot(mask_byte(t0));
  int next = mask_byte(t0 + 1);
  if (vis) issue(kv[0], t0, vis);
  bool fresh = true;
  int buf = 0;
  for (int t = t0; t < t1; ++t) {
    const uint64_t ahead = __ballot(next);
    if (vis | ahead) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
    }
    if (ahead) issue(kv[buf ^ 1], t + 1, ahead);
    next = mask_byte(t + 2);
    if (vis) tile(kv[buf], vis, fresh);
    fresh = fresh && vis == 0;
    vis = ahead;
    buf ^= 1;
  }
  const float l = l_run + __shfl_xor(l_run, 32);
  int me = tid;
  asm volatile("" : "+v"(me));
  const int want = ta.r0 + (me >> 6) * 32 + (me & 31), rr = min(want, ta.rows - 1);
  const int64_t tok = ta.a + rr / group;
  const int head = hk * group + rr % group;
  const int64_t row = tok * c.heads + head;
  if (part.splits > 1) {
    if (want >= ta.rows) return;
    float* po = part.o + ((int64_t)blockIdx.y * c.n_q * c.heads + row) * D;
#pragma unroll
    for (int ht = 0; ht < D / 32; ++ht)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
        *reinterpret_cast<float4*>(po + 32 * ht + 8 * q4 + 4 * g) =
            make_float4(o[ht][4 * q4], o[ht][4 * q4 + 1], o[ht][4 * q4 + 2], o[ht][4 * q4 + 3]);
    if (g == 0) {
      float* pm = part.ml + ((int64_t)blockIdx.y * c.n_q * c.heads + row) * 2;
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
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        w[e] = pack_bf16x2(o[ht][4 * q4 + 2 * e] * inv, o[ht][4 * q4 + 2 * e + 1] * inv);
      const auto x = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
      const auto y = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
      if (want < ta.rows) *(uint4*)(op + 32 * ht + 8 * (q4 + g)) = make_uint4(x[0], y[0], x[1], y[1]);
    }
  if (want >= ta.rows) return;
  if (c.lse != nullptr && g == 0) c.lse[row] = l == 0.0f ? -INFINITY : (m_run + log2f(l)) * LN2;
}

// float32: the same products on 32x32x2 MFMAs with operands straight from global
// memory (an MFMA takes 64 cycles for 4 to 16 bytes per lane).  Four waves take
// every fourth tile of 32 keys of the same 32 rows and meet in LDS.  326 rows of 24
// heads on 77 keys 9.3 us: one tile to a wave, the chain of its loads (offsets, mask,
// K and V, merge) around 2 us of MFMAs.  3,000 x 12 heads of 128 on 512 keys 110 us for
// 62 of MFMAs (requesting K and V before the mask is known: a third more, hidden tiles are
// loaded too); 8 x 1 query of 24 heads on 10,160 keys 250 us (998 MB), 1 x 1 47.
template <int D>
__global__ void __launch_bounds__(256)
cross_f32(const CrossArgs c, const Partial part, int tile0) {
  constexpr int LD = D + 4;
  __shared__ float os[4][32][LD];
  __shared__ float ms[4][32], ls[4][32];
  const int group = c.heads / c.kv_heads;
  const int hk = blockIdx.x % c.kv_heads;
  TileAt ta;
  if (!tile_at(c, group, 32, tile0 + blockIdx.x / c.kv_heads, ta)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 5, r31 = lane & 31;
  const int rr = min(ta.r0 + r31, ta.rows - 1);
  f32x4 qf[D / 8];
  {
    const float* qp = (const float*)c.q + (int64_t)(ta.a + rr / group) * c.q_ld + (hk * group + rr % group) * D;
#pragma unroll
    for (int s = 0; s < D / 8; ++s) qf[s] = *reinterpret_cast<const f32x4*>(qp + 4 * (2 * s + g));
  }
  int t0, t1;
  slice_of(ta.s0, ta.s1, 32, blockIdx.y, part.lg, t0, t1);
  f32x16 o[D / 32];
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[t][r] = 0.0f;
  const float sc = LOG2E * c.scale;
  float m = -FLT_MAX, l = 0.0f;
  for (int t = t0 + wave; t < t1; t += 4) {
    const int kb = ta.s0 + t * 32;
    const int key = kb + r31;
    const uint32_t vis = (uint32_t)__ballot(key < ta.s1 && (c.mask == nullptr || c.mask[min(key, ta.s1 - 1)] != 0));
    if (vis == 0) continue;
    // all operands of the tile are requested before the first product
    const float* kp = (const float*)c.k + (int64_t)min(key, ta.s1 - 1) * c.k_ld + hk * D;
    const float* vb = (const float*)c.v + hk * D + r31;
    f32x4 kf[D / 8];
#pragma unroll
    for (int s = 0; s < D / 8; ++s) kf[s] = *reinterpret_cast<const f32x4*>(kp + 4 * (2 * s + g));
    float vf[D / 32][16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int kr = 8 * (r >> 2) + 4 * g + (r & 3);
      const float* vp = vb + (int64_t)min(kb + kr, ta.s1 - 1) * c.v_ld;
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
    const uint32_t w = vis >> (4 * g);
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      st[r] = ((w >> (8 * (r >> 2) + (r & 3))) & 1u) ? st[r] * sc : -INFINITY;
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
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const bool see = (w >> (8 * (r >> 2) + (r & 3))) & 1u;
      const float p = exp2f(st[r] - m_new);
      l += p;
#pragma unroll
      for (int h = 0; h < D / 32; ++h)
        o[h] = __builtin_amdgcn_mfma_f32_32x32x2f32(see ? vf[h][r] : 0.0f, p, o[h], 0, 0, 0);
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
  if (ta.r0 + q >= ta.rows) return;
  const int64_t tok = ta.a + (ta.r0 + q) / group;
  const int head = hk * group + (ta.r0 + q) % group;
  const int64_t row = tok * c.heads + head;
  const float mt = fmaxf(fmaxf(ms[0][q], ms[1][q]), fmaxf(ms[2][q], ms[3][q]));
  float f[4], lt = 0.0f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    f[w] = exp2f(ms[w][q] - mt);
    lt = fmaf(ls[w][q], f[w], lt);
  }
  const bool whole = part.splits <= 1;
  const float inv = !whole ? 1.0f : lt == 0.0f ? 0.0f : 1.0f / lt;
  float* dst = whole ? (float*)c.o + tok * c.o_ld + head * D
                     : part.o + ((int64_t)blockIdx.y * c.n_q * c.heads + row) * D;
#pragma unroll
  for (int h = 0; h < D / 64; ++h) {
    const int col = 64 * h + (tid & 7) * 8;
    float acc[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      acc[e] = 0.0f;
#pragma unroll
      for (int w = 0; w < 4; ++w) acc[e] = fmaf(os[w][q][col + e], f[w], acc[e]);
      acc[e] *= inv;
    }
    store8(dst + col, acc);
  }
  if ((tid & 7) == 0) {
    if (!whole) {
      float* pm = part.ml + ((int64_t)blockIdx.y * c.n_q * c.heads + row) * 2;
      pm[0] = mt;
      pm[1] = lt;
    } else if (c.lse != nullptr) {
      c.lse[row] = lt == 0.0f ? -INFINITY : (mt + log2f(lt)) * LN2;
    }
  }
}

// One wave per token and head adds up the slices, in a fixed order.  Lane s weighs slice
// s; D / 4 lanes hold a slice's row, so a wave reads several at once and eight such
// loads are in flight (32 slices of 32 rows 4 us; one slice after the other 12).  Rows
// outside every sequence have none and are left as they are.
template <typename T, int D>
__global__ void __launch_bounds__(256)
cross_join(const CrossArgs c, const Partial part) {
  constexpr int PER = D / 4, SETS = 64 / PER, AHEAD = 8;
  const int64_t n = (int64_t)c.n_q * c.heads;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= n) return;
  const int lane = threadIdx.x & 63;
  const int tok = (int)(row / c.heads), head = (int)(row % c.heads);
  bool in = c.cu_q == nullptr;
  if (c.cu_q != nullptr && lane < c.n_seqs) in = tok >= c.cu_q[lane] && tok < c.cu_q[lane + 1];
  float m = -FLT_MAX, l = 0.0f;
  if (lane < part.splits) {
    const float2 ml = *reinterpret_cast<const float2*>(part.ml + (lane * n + row) * 2);
    m = ml.x;
    l = ml.y;
  }
  if (!__any(in)) return;
  const float mt = warp_max(m);
  const float f = lane < part.splits ? exp2f(m - mt) : 0.0f;
  l = warp_sum(l * f);
  const int set = lane / PER, col = lane % PER * 4;
  float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s0 = 0; s0 < part.splits; s0 += SETS * AHEAD) {
    float4 v[AHEAD];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const int s = min(s0 + SETS * a + set, part.splits - 1);
      v[a] = *reinterpret_cast<const float4*>(part.o + (s * n + row) * D + col);
    }
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const int s = s0 + SETS * a + set;
      if (s0 + SETS * a >= part.splits) break;
      const float w = __shfl(f, min(s, 63));
      if (s < part.splits) {
        acc[0] = fmaf(v[a].x, w, acc[0]);
        acc[1] = fmaf(v[a].y, w, acc[1]);
        acc[2] = fmaf(v[a].z, w, acc[2]);
        acc[3] = fmaf(v[a].w, w, acc[3]);
      }
    }
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
#pragma unroll
    for (int o = PER; o < 64; o <<= 1) acc[e] += __shfl_xor(acc[e], o);
    if (set == 0) Elem<T>::store((T*)c.o + tok * c.o_ld + head * D + col + e, acc[e] * inv);
  }
  if (c.lse != nullptr && lane == 0) c.lse[row] = l == 0.0f ? -INFINITY : (mt + log2f(l)) * LN2;
}

// workgroups of `bq` rows at most, the lengths being on the device
static int64_t cross_slots(const CrossArgs& c, int64_t bq) {
  return ((int64_t)c.n_q * (c.heads / c.kv_heads) + (bq - 1) * c.n_seqs) / bq;
}

// Few rows leave CUs idle and a workgroup alone on its CU waits out the latency of every
// tile, so the keys are split, as far as the workspace holds the partial results.  Chosen
// by modelled time (us): tiles per slice, each `lone` for a workgroup by itself and
// `share` per workgroup where several share a CU, plus the pass that joins the
// slices and what they write and read.  bf16, us without | with the chosen split: 8 x 1
// query of 24 heads on 10,160 keys 245 | 100 (4 slices), 1 query of 32 heads of 128 on 8 on
// 10,160 233 | 19 (64), 32 x 24 on 2,048 40 | 13 (16), 300 x 16 on 4,096 69 | 25 (8), 326 x
// 24 on 2,048 37 | 24 (4); 512 x 24 on 512 11 | 19 (2, not chosen), 4,096 x 12 of 128 on 512
// 23 | 54 (2, not chosen).
// The constants are the bf16 kernel's.  For float32 they are within 4% of the best split for
// single queries (the same three 379 | 250, 458 | 31, 61 | 18) and up to a quarter off for
// many rows: 300 x 16 114 | 80 (4; 8: 70), 326 x 24 92 | 80 (2; 8: 71), 1,000 x 12 of 128 on
// 4,096 330 (none; 4: 262).
// The lengths are on the device, so the mean one counts: beside 63 prompts of 16 states one
// of 10,160 is not split (64 x 1 query of 24 heads 186 us, with 8 slices 60), beside 7 of 512
// into 4 (57, with 16 slices 34).
static int cross_splits(int64_t wgs, int64_t tiles, int64_t rows, int D, int64_t ws_floats) {
  const double lone = D == 64 ? 1.2 : 1.6, share = D == 64 ? 0.64 : 1.0;
  int best = 1;
  double best_us = 1e300;
  for (int s = 1; s <= 64 && (s == 1 || s * 2 <= tiles); s *= 2) {
    if (s > 1 && (int64_t)s * rows * (D + 2) > ws_floats) break;
    double us = (double)((tiles + s - 1) / s) * std::max(lone, share * (double)(wgs * s) / 256.0);
    if (s > 1) us += 4.5 + 0.05 * s + 2.0 * s * (double)rows * (D + 2) * 4.0 / 3.0e6;
    if (us < best_us) { best_us = us; best = s; }
  }
  return best;
}

template <int D>
static void run_cross(int dtype, const CrossArgs& c, float* ws, int64_t ws_floats, hipStream_t st) {
  const int64_t wgs = cross_slots(c, dtype == 1 ? 128 : 32) * c.kv_heads;
  const int64_t tiles = (c.n_k / c.n_kv_seqs + CR_BK - 1) / CR_BK;
  const int64_t rows = (int64_t)c.n_q * c.heads;
  const int splits = cross_splits(wgs, tiles, rows, D, ws_floats);
  const Partial p{ws, ws + splits * rows * D, splits, __builtin_ctz(splits)};
  if (dtype == 1) {                             // (fewer than 2^32 threads at n_q * heads = 2^30)
    hipLaunchKernelGGL((cross_bf16<D>), dim3((unsigned)wgs, splits), dim3(256), 0, st, c, p);
  } else {
    // a grid holds less than 2^32 threads: more tiles than that (2^29 rows) take another launch
    const int64_t most = ((1 << 24) - 1) / c.kv_heads, tiles = wgs / c.kv_heads;
    for (int64_t t = 0; t < tiles; t += most)
      hipLaunchKernelGGL((cross_f32<D>), dim3((unsigned)(std::min(tiles - t, most) * c.kv_heads), splits), dim3(256),
                         0, st, c, p, (int)t);
  }
  if (splits > 1) {
    const unsigned n = (unsigned)((rows + 3) / 4);
    if (dtype == 1) hipLaunchKernelGGL((cross_join<bf16_t, D>), dim3(n), dim3(256), 0, st, c, p);
    else hipLaunchKernelGGL((cross_join<float, D>), dim3(n), dim3(256), 0, st, c, p);
  }
}

hipError_t launch_cross(int dtype, const CrossArgs& c, float* ws, int64_t ws_floats, hipStream_t st) {
  if (c.n_q <= 0) return hipSuccess;
  if (c.head_dim == 64) run_cross<64>(dtype, c, ws, ws_floats, st);
  else run_cross<128>(dtype, c, ws, ws_floats, st);
  return hipGetLastError();
}

}  // namespace swam
