// Norm and rotation of query and key heads, to rows or straight into a paged cache.
//
// A head vector of D elements takes LPH lanes of 8 (D / 8 rounded up to a power of two), so
// a wave holds 64 / LPH heads at a time and their sums of squares are log2(LPH) exchanges.
// A wave takes a row and walks over its heads: the angles of the row are formed once (one
// pair per lane, in float64 up to the fraction of a turn), and stay in the registers of the
// lanes for every head.
//   y = x / sqrt(mean(x^2) + eps) * gain,  a' = m (a cos t - b sin t), b' = m (a sin t + b cos t)
// What bounds it: HBM, each element read and written once.
#include "paged.h"

#include <algorithm>

namespace swam {

// 1 / sqrt(mean + eps) of each head as two factors, a power of two and the rest.  Squares
// that would pass float32's range at either end are formed of the lifted vector.
template <int LPH>
__device__ __forceinline__ void head_scale(const float (&x)[8], int dim, float eps, float& lift, float& r) {
  auto mean_of = [&](float f) {
    float ss = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(x[e] * f, x[e] * f, ss);
#pragma unroll
    for (int o = LPH / 2; o > 0; o >>= 1) ss += __shfl_xor(ss, o);
    return ss / (float)dim;
  };
  lift = 1.0f;
  float t = mean_of(1.0f) + eps;
  const bool odd = !(t >= 0x1p-100f && t <= 0x1p100f);
  if (__any(odd)) {
    if (odd) lift = t < 1.0f ? 0x1p100f : 0x1p-70f;
    t = mean_of(lift) + eps * lift * lift;
  }
  r = t == 0.0f ? 0.0f : rsqrtf(t);
}

template <typename T, int LPH, bool CACHE>
__global__ void __launch_bounds__(256)
head_post(const HeadPost a, const Paged pg, int lg_parts) {
  constexpr int HPI = 64 / LPH;                 // heads at a time
  constexpr int U = 4;                          // of these in flight
  __shared__ float2 tab[4][4 * LPH];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int c8 = lane % LPH * 8, hs = lane / LPH;
  const bool has = c8 < a.dim;
  const int pairs = a.rot >> 1;
  const int n_heads = a.heads + a.kv_heads * (CACHE ? 2 : 1);
  float gq[8], gk[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) gq[e] = gk[e] = 1.0f;
  if (a.q_gain != nullptr && has) load8((const T*)a.q_gain + c8, gq);
  if (a.k_gain != nullptr && has) load8((const T*)a.k_gain + c8, gk);

  const int64_t waves = (int64_t)gridDim.x * 4;
  for (int64_t w = (int64_t)blockIdx.x * 4 + wave; w < a.rows << lg_parts; w += waves) {
    const int64_t row = w >> lg_parts;
    int pos = (int)row;
    int64_t k_at = -1, v_at = -1;               // where the token's first head goes
    if constexpr (CACHE) {
      const int s = seq_of(pg, row);
      int b, e;
      chunk_of(pg, s, (int)a.rows, b, e);
      if (row < b || row >= e) continue;        // behind the last sequence
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
    // this lane's elements: x' = c x + s (partner of x)
    float c[8], sg[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int j = c8 + e;
      const bool first = a.half ? j < pairs : !(e & 1);
      const int p = a.half ? (first ? j : j - pairs) : j >> 1;
      c[e] = sg[e] = 0.0f;
      if (j < a.rot) {
        const float2 cs = tab[wave][p];
        c[e] = cs.x;
        sg[e] = first ? -cs.y : cs.y;
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int across = c8 < pairs ? pairs >> 3 : -(pairs >> 3);   // lanes to the partners (half layout)
    const int from = c8 < a.rot ? lane + across : lane;

    const int step = HPI << lg_parts;
    for (int h0 = ((int)w & ((1 << lg_parts) - 1)) * HPI; h0 < n_heads; h0 += U * step) {
      float x[U][8];
      const T* src[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = h0 + u * step + hs;
        src[u] = nullptr;
        if (has && h < n_heads)
          src[u] = h < a.heads ? (const T*)a.q + row * a.q_ld + (int64_t)h * a.dim
                 : !CACHE || h < a.heads + a.kv_heads
                     ? (const T*)a.k + row * a.k_ld + (int64_t)(h - a.heads) * a.dim
                     : (const T*)a.v + row * a.v_ld + (int64_t)(h - a.heads - a.kv_heads) * a.dim;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[u][e] = 0.0f;
        if (src[u] != nullptr) load8(src[u] + c8, x[u]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (h0 + u * step >= n_heads) break;
        const int h = h0 + u * step + hs;
        const bool is_q = h < a.heads, is_v = CACHE && h >= a.heads + a.kv_heads;
        float lift = 1.0f, r = 1.0f;
        if (a.norm) head_scale<LPH>(x[u], a.dim, a.eps, lift, r);
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = a.norm ? x[u][e] * lift * r * (is_q ? gq[e] : gk[e]) : x[u][e];
        if (a.rot) {
          float z[8];
          if (!a.half) {
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = y[e ^ 1];
          } else if (pairs % 8 == 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = __shfl(y[e], from);
          } else {
            // partners at any distance are read and formed again
            const void* gain = is_q ? a.q_gain : a.k_gain;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int j = c8 + e;
              z[e] = 0.0f;
              if (src[u] == nullptr || j >= a.rot) continue;
              const int m = j < pairs ? j + pairs : j - pairs;
              z[e] = Elem<T>::load(src[u] + m);
              if (a.norm) z[e] = z[e] * lift * r * (gain != nullptr ? Elem<T>::load((const T*)gain + m) : 1.0f);
            }
          }
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (c8 + e < a.rot) y[e] = fmaf(z[e], sg[e], y[e] * c[e]);
        }
        T* dst = nullptr;
        if (is_q) {
          dst = (T*)a.q_out + row * a.qo_ld + (int64_t)h * a.dim;
        } else if (!CACHE) {
          dst = (T*)a.k_out + row * a.ko_ld + (int64_t)(h - a.heads) * a.dim;
        } else if (k_at >= 0) {
          dst = is_v ? (T*)pg.v + v_at + (h - a.heads - a.kv_heads) * pg.v_head
                     : (T*)pg.k + k_at + (h - a.heads) * pg.k_head;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (is_v) y[e] = x[u][e];
        if (src[u] != nullptr && dst != nullptr) store8(dst + c8, y);
      }
    }
  }
}

template <typename T, int LPH>
static void run_head_post(const HeadPost& a, const Paged* cache, hipStream_t st) {
  constexpr int HPI = 64 / LPH;
  const int n_heads = a.heads + a.kv_heads * (cache ? 2 : 1);
  // few rows: the heads of a row go to several waves
  int lg = 0;
  while (a.rows << lg < 4096 && HPI << lg < n_heads) ++lg;
  const int64_t wgs = std::min(((a.rows << lg) + 3) / 4, (int64_t)4096);
  if constexpr (LPH == 8 || LPH == 16)          // a cache has heads of 64 or 128
    if (cache) {
      hipLaunchKernelGGL((head_post<T, LPH, true>), dim3((unsigned)wgs), dim3(256), 0, st, a, *cache, lg);
      return;
    }
  hipLaunchKernelGGL((head_post<T, LPH, false>), dim3((unsigned)wgs), dim3(256), 0, st, a, Paged{}, lg);
}

template <typename T>
static void run_head_post(const HeadPost& a, const Paged* cache, hipStream_t st) {
  const int n = a.dim / 8;
  if (n <= 1) run_head_post<T, 1>(a, cache, st);
  else if (n <= 2) run_head_post<T, 2>(a, cache, st);
  else if (n <= 4) run_head_post<T, 4>(a, cache, st);
  else if (n <= 8) run_head_post<T, 8>(a, cache, st);
  else if (n <= 16) run_head_post<T, 16>(a, cache, st);
  else if (n <= 32) run_head_post<T, 32>(a, cache, st);
  else run_head_post<T, 64>(a, cache, st);
}

hipError_t launch_head_post(int dtype, const HeadPost& a, const Paged* cache, hipStream_t st) {
  if (a.rows <= 0) return hipSuccess;
  if (dtype == 1) run_head_post<bf16_t>(a, cache, st);
  else run_head_post<float>(a, cache, st);
  return hipGetLastError();
}

}  // namespace swam
