// Norm and rotation of query and key heads, to rows or straight into a paged cache.
//
// A head vector of D elements takes LPH lanes of 8 (D / 8 rounded up to a power of two), so
// a wave holds 64 / LPH heads of q, of k or of v at a time and their sums of squares are
// log2(LPH) exchanges.  A wave takes a row and walks over its heads: the angles of the row are
// formed once (one pair per lane, in float64 up to the fraction of a turn) while the first
// heads are on their way, and stay in the registers of the lanes for every head.
//   y = x / sqrt(mean(x^2) + eps) * gain,  a' = m (a cos t - b sin t), b' = m (a sin t + b cos t)
// What bounds it: HBM, each element read and written once: 10,160 rows of 48 heads of 64 in bf16 26 us
// (125 MB, 4.8 TB/s), 17,472 of 20 heads of 128 40 (179 MB), an append of 10,160 x 72 heads 43 (187 MB),
// of 18 float32 heads of 128 to 15,390 rows 71 (365 MB, 5.1 TB/s).  What counted: the loads in front of
// the angles and always some on their way (44 us without, for the first), steps of heads of one kind, so that
// pointers and gains are scalar choices, and few registers (72 for the first: seven waves to a SIMD).
#include "paged.h"

#include <algorithm>

namespace swam {

// 8 elements as they are loaded
template <typename T> struct Raw;
template <> struct Raw<bf16_t> { uint4 a; };
template <> struct Raw<float> { float4 a, b; };
__device__ __forceinline__ Raw<bf16_t> raw8(const bf16_t* p) { return {*(const uint4*)p}; }
__device__ __forceinline__ Raw<float> raw8(const float* p) { return {((const float4*)p)[0], ((const float4*)p)[1]}; }
__device__ __forceinline__ void raw_store(bf16_t* p, const Raw<bf16_t>& r) { *(uint4*)p = r.a; }
__device__ __forceinline__ void raw_store(float* p, const Raw<float>& r) {
  ((float4*)p)[0] = r.a;
  ((float4*)p)[1] = r.b;
}
__device__ __forceinline__ void widen(const Raw<bf16_t>& r, float (&o)[8]) {
  const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    o[2 * e] = __uint_as_float(w[e] << 16);
    o[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void widen(const Raw<float>& r, float (&o)[8]) {
  o[0] = r.a.x; o[1] = r.a.y; o[2] = r.a.z; o[3] = r.a.w; o[4] = r.b.x; o[5] = r.b.y; o[6] = r.b.z; o[7] = r.b.w;
}

// v plus the v of lane ^ O, for O up to 8 on data that the smaller exchanges have made equal
template <int O>
__device__ __forceinline__ float add_across(float v) {
  // quads by their own permutes, 8 and 16 lanes mirrored, further by the LDS's
  constexpr int CTRL = O == 1 ? 0xB1 : O == 2 ? 0x4E : O == 4 ? 0x141 : 0x140;
  if constexpr (O <= 8)
    return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, true));
  else
    return v + __shfl_xor(v, O);
}

// 1 / sqrt(mean + eps) of each head.  Where squares would pass float32's range at either end
// the vector is lifted by a power of two first (lift, 1 else).
template <int LPH>
__device__ __forceinline__ float head_scale(float (&x)[8], float inv_dim, float eps, float& lift) {
  auto mean_plus = [&](float add) {
    float ss = x[0] * x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
    if constexpr (LPH > 1) ss = add_across<1>(ss);
    if constexpr (LPH > 2) ss = add_across<2>(ss);
    if constexpr (LPH > 4) ss = add_across<4>(ss);
    if constexpr (LPH > 8) ss = add_across<8>(ss);
    if constexpr (LPH > 16) ss = add_across<16>(ss);
    if constexpr (LPH > 32) ss = add_across<32>(ss);
    return fmaf(ss, inv_dim, add);
  };
  lift = 1.0f;
  float t = mean_plus(eps);
  const bool odd = !(t >= 0x1p-100f && t <= 0x1p100f);
  if (__any(odd)) {
    if (odd) lift = t < 1.0f ? 0x1p100f : 0x1p-70f;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= lift;
    t = mean_plus(eps * lift * lift);
  }
  return t == 0.0f ? 0.0f : __builtin_amdgcn_rsqf(t);
}

// where an element's partner is
enum Pairs {
  PAIRS_NEXT,         // beside it
  PAIRS_LANES,        // whole lanes away (half layout, rotated elements a multiple of 16)
  PAIRS_ANY           // at any distance
};

template <typename T, int LPH, Pairs PAIRS, bool CACHE>
__global__ void __launch_bounds__(256)
head_post(const HeadPost a, const Paged pg, int lg_parts) {
  constexpr int HPI = 64 / LPH;                 // heads at a time
  // of these on their way, each replaced when it is used (bf16: six, reloaded as a group, 28 and 50 us
  // for the first two sizes above)
  constexpr int U = PAIRS == PAIRS_ANY ? 1 : sizeof(T) == 2 ? 4 : 2;
  constexpr bool HALF = PAIRS != PAIRS_NEXT;
  __shared__ float2 tab[4][4 * LPH];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int c8 = lane % LPH * 8, hs = lane / LPH, mine = hs * a.dim + c8;
  const bool has = c8 < a.dim;
  const int pairs = a.rot >> 1, parts = 1 << lg_parts;
  const int nq = (a.heads + HPI - 1) / HPI, nk = nq + (a.kv_heads + HPI - 1) / HPI;
  const int steps = CACHE ? 2 * nk - nq : nk;   // of q, then k, then v heads
  Raw<T> gq{}, gk{};
  if (a.q_gain != nullptr && has) gq = raw8((const T*)a.q_gain + c8);
  if (a.k_gain != nullptr && has) gk = raw8((const T*)a.k_gain + c8);

  const int64_t waves = (int64_t)gridDim.x * 4;
  for (int64_t w = (int64_t)blockIdx.x * 4 + wave; w < a.rows << lg_parts; w += waves) {
    const int64_t row = w >> lg_parts;
    const int part = (int)w & (parts - 1);
    const T* q_row = (const T*)a.q + row * a.q_ld;
    const T* k_row = (const T*)a.k + row * a.k_ld;
    const T* v_row = (const T*)a.v + row * a.v_ld;
    auto src_of = [&](int step) {
      return step < nq ? q_row + (int64_t)step * HPI * a.dim
           : CACHE && step >= nk ? v_row + (int64_t)(step - nk) * HPI * a.dim
                                 : k_row + (int64_t)(step - nq) * HPI * a.dim;
    };
    // heads of a step and behind it
    auto left_of = [&](int step) {
      return step < nq ? a.heads - step * HPI : a.kv_heads - (CACHE && step >= nk ? step - nk : step - nq) * HPI;
    };
    Raw<T> x[U];
    auto load = [&](int step) {
      Raw<T> r{};
      if (step < steps && has && hs < left_of(step)) r = raw8(src_of(step) + mine);
      return r;
    };
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = load(part + u * parts);

    int pos = (int)row;
    int64_t k_at = -1, v_at = -1;               // where the token's first head goes
    if constexpr (CACHE) {
      int s = seq_of(pg, row);
      int b, e;
      chunk_of(pg, s, (int)a.rows, b, e);
      if (__builtin_expect(row < b || row >= e, 0)) {   // offsets that fall, or nobody's
        s = seq_that_holds(pg, row);
        if (s < 0) continue;
        chunk_of(pg, s, (int)a.rows, b, e);
      }
      const int64_t slot = held(pg, s) + (row - b);
      pos = (int)slot;
      const int64_t pi = slot >> pg.lg_page;
      const int page = pi < pg.max_pages ? pg.table[s * pg.table_ld + pi] : -1;
      if (page >= 0 && page < pg.n_pages) {
        const int t = (int)slot & ((1 << pg.lg_page) - 1);
        k_at = page * pg.k_page + t * pg.k_token;
        v_at = page * pg.v_page + t * pg.v_token;
      }
    }
    if (a.pos != nullptr) pos = a.pos[row];
    // the angle's whole turns are taken off in float64; (cos, sin) of every pair, times m
    for (int p = lane; p < pairs; p += 64) {
      const double t = (double)pos * (a.freq[p] * 0.15915494309189533577);
      float sn, cs;
      sincospif(2.0f * (float)(t - rint(t)), &sn, &cs);
      tab[wave][p] = make_float2(a.mag * cs, a.mag * sn);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    // (cos, sin) of this lane's elements: interleaved, one for two of them; half, the sign of
    // the partner's term in the sine
    constexpr int NC = HALF ? 8 : 4;
    float c[NC], sg[NC];
#pragma unroll
    for (int e = 0; e < NC; ++e) {
      const int j = HALF ? c8 + e : c8 + 2 * e;
      c[e] = sg[e] = 0.0f;
      if (j < a.rot) {
        const float2 cs = tab[wave][HALF ? (j < pairs ? j : j - pairs) : j >> 1];
        c[e] = cs.x;
        sg[e] = HALF && j < pairs ? -cs.y : cs.y;
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    // the lane of the partners (PAIRS_LANES)
    [[maybe_unused]] const int from = c8 < a.rot ? lane + (c8 < pairs ? pairs >> 3 : -(pairs >> 3)) : lane;

#pragma unroll 1
    for (int step0 = part; step0 < steps; step0 += U * parts) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int step = step0 + u * parts;
        if (step >= steps) break;
        const bool is_q = step < nq, is_v = CACHE && step >= nk;
        const bool live = has && hs < left_of(step);
        const Raw<T> raw = x[u];
        x[u] = load(step + U * parts);
        if (is_v) {
          if (live && v_at >= 0) raw_store((T*)pg.v + v_at + ((step - nk) * HPI + hs) * pg.v_head + c8, raw);
          continue;
        }
        float y[8];
        widen(raw, y);
        float lift = 1.0f, r = 1.0f;
        if (a.norm) {
          r = head_scale<LPH>(y, a.inv_dim, a.eps, lift);
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] *= r;
          if ((is_q ? a.q_gain : a.k_gain) != nullptr) {
            float g[8];
            widen(is_q ? gq : gk, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] *= g[e];
          }
        }
        if (a.rot) {
          if constexpr (PAIRS == PAIRS_NEXT) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float p = fmaf(y[2 * e + 1], -sg[e], y[2 * e] * c[e]), n = fmaf(y[2 * e], sg[e], y[2 * e + 1] * c[e]);
              const bool in = c8 + 2 * e < a.rot;
              y[2 * e] = in ? p : y[2 * e];
              y[2 * e + 1] = in ? n : y[2 * e + 1];
            }
          } else {
            float z[8];
            if constexpr (PAIRS == PAIRS_LANES) {
#pragma unroll
              for (int e = 0; e < 8; ++e) z[e] = __shfl(y[e], from);
            } else {
              // they are read and formed again
              const T* src = src_of(step) + hs * a.dim;
              const T* gain = (const T*)(is_q ? a.q_gain : a.k_gain);
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const int j = c8 + e;
                z[e] = 0.0f;
                if (live && j < a.rot) {
                  const int m = j < pairs ? j + pairs : j - pairs;
                  z[e] = Elem<T>::load(src + m);
                  if (a.norm) z[e] = z[e] * lift * r * (gain != nullptr ? Elem<T>::load(gain + m) : 1.0f);
                }
              }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float t = fmaf(z[e], sg[e], y[e] * c[e]);
              y[e] = (PAIRS == PAIRS_LANES ? c8 < a.rot : c8 + e < a.rot) ? t : y[e];
            }
          }
        }
        if (is_q) {
          if (live) store8((T*)a.q_out + row * a.qo_ld + (int64_t)step * HPI * a.dim + mine, y);
        } else if constexpr (CACHE) {
          if (live && k_at >= 0) store8((T*)pg.k + k_at + ((step - nq) * HPI + hs) * pg.k_head + c8, y);
        } else {
          if (live) store8((T*)a.k_out + row * a.ko_ld + (int64_t)(step - nq) * HPI * a.dim + mine, y);
        }
      }
    }
  }
}

template <typename T, int LPH, Pairs PAIRS>
static void run_head_post(const HeadPost& a, const Paged* cache, hipStream_t st) {
  constexpr int HPI = 64 / LPH;
  const int steps = (a.heads + HPI - 1) / HPI + (a.kv_heads + HPI - 1) / HPI * (cache ? 2 : 1);
  // few rows: the heads of a row go to several waves (one row of 48 heads in float32 4.2 us)
  int lg = 0;
  while (a.rows << lg < 4096 && 1 << lg < steps) ++lg;
  const int64_t wgs = std::min(((a.rows << lg) + 3) / 4, (int64_t)8192);
  if constexpr (LPH == 8 || LPH == 16)          // a cache has heads of 64 or 128
    if (cache) {
      hipLaunchKernelGGL((head_post<T, LPH, PAIRS, true>), dim3((unsigned)wgs), dim3(256), 0, st, a, *cache, lg);
      return;
    }
  hipLaunchKernelGGL((head_post<T, LPH, PAIRS, false>), dim3((unsigned)wgs), dim3(256), 0, st, a, Paged{}, lg);
}

template <typename T, Pairs PAIRS>
static void run_head_post(const HeadPost& a, const Paged* cache, hipStream_t st) {
  const int n = a.dim / 8;
  if (n <= 1) run_head_post<T, 1, PAIRS>(a, cache, st);
  else if (n <= 2) run_head_post<T, 2, PAIRS>(a, cache, st);
  else if (n <= 4) run_head_post<T, 4, PAIRS>(a, cache, st);
  else if (n <= 8) run_head_post<T, 8, PAIRS>(a, cache, st);
  else if (n <= 16) run_head_post<T, 16, PAIRS>(a, cache, st);
  else if (n <= 32) run_head_post<T, 32, PAIRS>(a, cache, st);
  else run_head_post<T, 64, PAIRS>(a, cache, st);
}

template <typename T>
static void run_head_post(const HeadPost& a, const Paged* cache, hipStream_t st) {
  if (!a.half || a.rot == 0) run_head_post<T, PAIRS_NEXT>(a, cache, st);
  else if (a.rot % 16 == 0) run_head_post<T, PAIRS_LANES>(a, cache, st);
  else run_head_post<T, PAIRS_ANY>(a, cache, st);
}

hipError_t launch_head_post(int dtype, const HeadPost& a, const Paged* cache, hipStream_t st) {
  if (a.rows <= 0) return hipSuccess;
  if (dtype == 1) run_head_post<bf16_t>(a, cache, st);
  else run_head_post<float>(a, cache, st);
  return hipGetLastError();
}

}  // namespace swam
