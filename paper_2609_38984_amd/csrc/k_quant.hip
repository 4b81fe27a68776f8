// Rows to 8-bit codes with a scale each: the residual addition and RMS norm in
// front of an 8-bit projection, and the plain quantiser of activations and
// weights.
//
//   t = x + r;  y = t / sqrt(mean t^2 + eps) * gain * (1 + scale) + shift
//   s = max|y| / 127;  code = round(y / s)
// Two numbers of the whole row (the mean square and the largest magnitude) stand
// between reading x and writing the codes.  The row stays on chip in float32
// between them, so every byte moves once: memory bounds it (rows * d * (x + r +
// sum + 1) bytes): bf16 with residual, sum, gain and modulation 10,160 x 1,536 23.6 us
// (4.6 TB/s), 17,472 x 8,192 192 us (5.2); plain 76 us (5.6).  A large copy reaches 5.1.
#include "launchers.h"

#include <algorithm>
#include <type_traits>

namespace swam {

// Bits of |v|: as unsigned integers they order like the magnitudes, with
// infinities and then NaN above every finite value, so one integer maximum
// finds the largest magnitude and any non-finite value.
__device__ __forceinline__ uint32_t mag_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }
constexpr uint32_t INF_BITS = 0x7f800000u;

__device__ __forceinline__ uint32_t warp_umax(uint32_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o));
  return v;
}

// What a row's largest magnitude makes of it: the stored scale, and the factors
// pre, inv with code = round((y pre) inv).  pre lifts rows whose 127 / max would
// overflow.
struct RowScale {
  float s, pre, inv, top;
};
__device__ __forceinline__ RowScale row_scale(uint32_t bits) {
  RowScale r;
  r.top = __uint_as_float(bits);
  r.pre = r.top < 0x1p-100f ? 0x1p100f : 1.0f;
  r.inv = bits == 0u ? 0.0f : 127.0f / (r.top * r.pre);
  r.s = r.top / 127.0f;
  if (bits >= INF_BITS) {
    r.s = __uint_as_float(0x7fc00000u);
    r.pre = r.inv = 0.0f;
  }
  return r;
}

// The code of y.  EXACT: within 1e-4 of a border (the product above is off by at
// most 2^-16 there) the side is decided on 254 |y| against (2 b + 1) max, both
// exact in float64.
template <bool EXACT>
__device__ __forceinline__ int code_of(float y, const RowScale& r) {
  if (r.inv == 0.0f) return 0;
  const float f = (y * r.pre) * r.inv;
  float c = rintf(f);
  if constexpr (EXACT) {
    if (fabsf(fabsf(f - c) - 0.5f) < 1e-4f) {
      const float b = floorf(fabsf(f));
      const double lhs = 254.0 * (double)fabsf(y), rhs = (2.0 * (double)b + 1.0) * (double)r.top;
      const float even = ((int)b & 1) ? b + 1.0f : b;
      const float m = lhs > rhs ? b + 1.0f : lhs < rhs ? b : even;
      c = copysignf(m, y);
    }
  }
  return (int)c;
}

// 1 / sqrt(ms), ms = mean square + eps; NaN for a sum of squares ss that is NaN or
// overflowed, so that every y and with it the scale is NaN; 0 for a row of zeros without eps
__device__ __forceinline__ float inv_rms(float ss, float ms) {
  return !(ss < INFINITY) ? __uint_as_float(0x7fc00000u) : ms > 0.0f ? 1.0f / sqrtf(ms) : 0.0f;
}

// Below this ms a row is lifted by 2^100 (and eps by its square) before its squares are
// summed again, which leaves y as it is: a square loses at most 2^-150 to float32's end of
// range, 2^-30 of a mean that is not below.  Lifted, elements are below 2^48 and the smallest
// one that a row can hold is 2^-49, its square far inside the range.
constexpr float TINY_MS = 0x1p-120f, LIFT = 0x1p100f;

__device__ __forceinline__ uint32_t pack4(int a, int b, int c, int d) {
  return (uint32_t)(a & 255) | ((uint32_t)(b & 255) << 8) | ((uint32_t)(c & 255) << 16) | ((uint32_t)d << 24);
}

// Sum / maximum over the NW waves that share a row; one wave needs no LDS.
template <int NW>
__device__ __forceinline__ float row_sum(float v, float* red) {
  v = warp_sum(v);
  if constexpr (NW > 1) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) v += red[w];
  }
  return v;
}
// A second sum of the row, once every wave has read the parts of the first; one part after
// the other, for it is rare and the registers of the common path are counted.
template <int NW>
__device__ __forceinline__ float row_sum_again(float v, float* red) {
  v = warp_sum(v);
  if constexpr (NW > 1) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll 1
    for (int w = 0; w < NW; ++w) v += red[w];
  }
  return v;
}
template <int NW>
__device__ __forceinline__ uint32_t row_umax(uint32_t v, uint32_t* red) {
  v = warp_umax(v);
  if constexpr (NW > 1) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) v = max(v, red[w]);
  }
  return v;
}

// 8 neighbouring elements as they lie in memory, moved in one access at any alignment
// of the element type (the hardware takes unaligned vectors; with scalar accesses 17,472
// x 8,192 bf16 with rows 10 bytes off take 200 us, with vectors 83, aligned 75: 5.7 TB/s).
template <typename T> struct Raw8 { uint32_t w[2 * sizeof(T)]; };
template <typename T>
__device__ __forceinline__ void raw_to_f32(const Raw8<T>& r, float (&o)[8]) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      o[2 * e] = __uint_as_float(r.w[e] << 16);
      o[2 * e + 1] = __uint_as_float(r.w[e] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = __uint_as_float(r.w[e]);
  }
}
template <typename T>
__device__ __forceinline__ void raw_store(T* p, const float (&v)[8]) {
  Raw8<T> r;
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int e = 0; e < 4; ++e) r.w[e] = pack_bf16x2(v[2 * e], v[2 * e + 1]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) r.w[e] = __float_as_uint(v[e]);
  }
  __builtin_memcpy(p, &r, sizeof(r));
}

// How a row divides into vectors of 8.  WHOLE: evenly.  TAIL: the last lane with any
// elements reads the last 8 of the row and owns those that no other lane has; lanes past
// the end read them too and own none, so no read is behind a branch (with the odd
// elements read one by one there, 10,038 x 2,402 with the norm over eight waves took 64 us
// instead of 54, and the plain quantiser on aligned rows of 8,192 85 instead of 75).
// SHORT: fewer than 8 elements, one by one.
enum { WHOLE, TAIL, SHORT };

// Waves of the norm per CU, all resident at once: what the registers of the form allow in
// whole workgroups, and no more than 24 (10,160 x 1,536 23.6 us, with 30 25.5, with 16
// 25.2) except where 16 waves share a row (17,472 x 8,192 192 us with 32, with 16 210).
constexpr int norm_waves(int esz, int fit, int nw, int nv) {
  if (nv > 1) return 16;
  if (nw == 16) return fit == WHOLE && esz == 2 ? 32 : 16;
  return fit == WHOLE ? 24 : nw == 8 ? 16 : 20;
}

// Rows of up to NW * 64 * 8 * NV elements in registers: NW waves to a row, lane t
// holding the 8-element vectors t, t + 64 NW, ...  NW = 1 puts four rows on a workgroup
// and needs no barrier.  With the norm a workgroup takes every gridDim-th row: gain and
// modulation (more bytes than a bf16 row itself) are read once where they fit the
// registers, and the next row is requested before this one's sums.
template <typename T, bool NORM, int FIT, int NW, int NV>
__global__ void __launch_bounds__(NW == 1 ? 256 : NW * 64) __attribute__((amdgpu_waves_per_eu(
    NORM ? norm_waves(sizeof(T), FIT, NW, NV) / 4 : 1, 8)))
quant_rows(const RowQuant a) {
  constexpr int TPR = NW * 64, RPW = NW == 1 ? 4 : 1;
  constexpr bool KEEP = NORM && NV == 1, TURNS = NORM && NV <= 2;
  __shared__ float red[NW];
  __shared__ uint32_t redu[NW];
  int64_t row = (int64_t)blockIdx.x * RPW + (NW == 1 ? threadIdx.x / TPR : 0);
  if (row >= a.rows) return;                    // whole waves
  const int t = threadIdx.x % TPR, d = a.d;
  auto first = [&](int i) { return (i * TPR + t) * 8; };                 // first own element
  auto from = [&](int i) { return FIT == SHORT ? first(i) : min(first(i), d - 8); };
  // whether element j of vector i is this lane's (a vector starts at from())
  auto own = [&](int i, int j) {
    return FIT == WHOLE ? first(i) < d : FIT == TAIL ? from(i) + j >= first(i) : first(i) + j < d;
  };
  // An element's place beside the row's scalar pointer.  With 16 waves it is added anew each
  // time: a 64-bit pointer per lane and tensor is more than their 64 registers hold (17,472 x
  // 8,192 203 us with 4 of them spilled); with fewer waves the additions cost 1-5%.
  auto offset = [&](int at) {
    if constexpr (NW == 16) asm volatile("" : "+v"(at));
    return (uint32_t)at;
  };
  auto read = [&](const auto* p, int i, auto& o) {
    if constexpr (FIT != SHORT) {
      __builtin_memcpy(&o, p + offset(from(i)), sizeof(o));
    } else {
      o = {};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (!own(i, j)) continue;
        if constexpr (sizeof(*p) == 2) o.w[j / 2] |= (uint32_t)p[first(i) + j] << (16 * (j & 1));
        else o.w[j] = __float_as_uint(p[first(i) + j]);
      }
    }
  };
  // y = (t / rms) fac + add
  auto factors = [&](int i, float (&fac)[8], float (&add)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) { fac[j] = 1.0f; add[j] = 0.0f; }
    if (a.gain != nullptr) {
      Raw8<T> g;
      read((const T*)a.gain, i, g);
      raw_to_f32(g, fac);
    }
    if (a.shift != nullptr) {
      Raw8<float> sc, sh;
      read(a.scale, i, sc);
      read(a.shift, i, sh);
      raw_to_f32(sh, add);
#pragma unroll
      for (int j = 0; j < 8; ++j) fac[j] *= 1.0f + __uint_as_float(sc.w[j]);
    }
  };
  Raw8<T> x[NV], r[NV];
  auto fetch = [&](int64_t at) {
#pragma unroll
    for (int i = 0; i < NV; ++i) read((const T*)a.x + at * a.x_ld, i, x[i]);
    if (NORM && a.res != nullptr) {
#pragma unroll
      for (int i = 0; i < NV; ++i) read((const T*)a.res + at * a.res_ld, i, r[i]);
    }
  };
  fetch(row);
  float kfac[8], kadd[8];
  if constexpr (KEEP) factors(0, kfac, kadd);
  for (;;) {
    float v[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      raw_to_f32(x[i], v[i]);
      if (NORM && a.res != nullptr) {
        float o[8];
        raw_to_f32(r[i], o);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] += o[j];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (!own(i, j)) v[i][j] = 0.0f;
    }
    const int64_t next = row + (int64_t)gridDim.x * RPW;
    const bool more = TURNS && next < a.rows;
    if constexpr (NORM) {
      if (more) fetch(next);
      if (a.sum != nullptr) {
        T* sp = (T*)a.sum + row * a.sum_ld;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          if (first(i) + 8 <= d) {
            raw_store(sp + offset(first(i)), v[i]);
          } else if (FIT != WHOLE) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (first(i) < d && own(i, j)) Elem<T>::store(sp + from(i) + j, v[i][j]);
          }
        }
      }
      auto squares = [&] {
        float ss = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) ss = fmaf(v[i][j], v[i][j], ss);
        return ss;
      };
      float ss = row_sum<NW>(squares(), red), ms = ss / (float)d + a.eps;
      if (__any(ms < TINY_MS)) {                // one answer for all waves of the row
        float eps = a.eps;
        asm volatile("" : "+s"(eps));           // formed here: no register holds it for every row
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) v[i][j] *= LIFT;
        ss = row_sum_again<NW>(squares(), red);
        ms = ss / (float)d + eps * LIFT * LIFT;
      }
      const float inv = inv_rms(ss, ms);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        float fac[8], add[8];
        if constexpr (!KEEP) factors(i, fac, add);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          v[i][j] = KEEP ? fmaf(v[i][j] * inv, kfac[j], kadd[j]) : fmaf(v[i][j] * inv, fac[j], add[j]);
          if (!own(i, j)) v[i][j] = 0.0f;
        }
      }
    }
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) top = max(top, mag_bits(v[i][j]));
    const RowScale rs = row_scale(row_umax<NW>(top, redu));
    int8_t* qp = a.q + row * a.q_ld;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (first(i) >= d) continue;
      int c[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) c[j] = code_of<!NORM>(v[i][j], rs);
      if (FIT == WHOLE || first(i) + 8 <= d) {
        const uint32_t w[2] = {pack4(c[0], c[1], c[2], c[3]), pack4(c[4], c[5], c[6], c[7])};
        __builtin_memcpy(qp + offset(first(i)), w, 8);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (own(i, j)) qp[from(i) + j] = (int8_t)c[j];
      }
    }
    if (t == 0) a.q_scale[row] = rs.s;
    if (!more) return;
    row = next;
  }
}

template <typename T, bool NORM, int FIT, int NW, int NV>
static void run_rows(RowQuant a, hipStream_t st) {
  constexpr int RPW = NW == 1 ? 4 : 1, WAVES = NW == 1 ? 4 : NW;
  constexpr bool TURNS = NORM && NV <= 2;
  // a grid holds less than 2^32 threads: more rows than that take another launch
  constexpr int64_t MOST = TURNS ? (int64_t)1 << 31 : (int64_t)RPW << 20;
  for (int64_t left = a.rows;; left -= MOST) {
    a.rows = std::min(left, MOST);
    const int64_t sets = (a.rows + RPW - 1) / RPW;
    const unsigned n = (unsigned)(TURNS ? std::min<int64_t>(sets, 256 * (norm_waves(sizeof(T), FIT, NW, NV) / WAVES)) : sets);
    hipLaunchKernelGGL((quant_rows<T, NORM, FIT, NW, NV>), dim3(n), dim3(WAVES * 64), 0, st, a);
    if (left <= MOST) return;
    a.x = (const T*)a.x + MOST * a.x_ld;
    if (a.res != nullptr) a.res = (const T*)a.res + MOST * a.res_ld;
    if (a.sum != nullptr) a.sum = (T*)a.sum + MOST * a.sum_ld;
    a.q += MOST * a.q_ld;
    a.q_scale += MOST;
  }
}

// One wave to a row up to 512 elements.  Beyond, the norm adds waves, so that a lane's one
// vector of factors stays in registers (17,472 x 8,192 bf16 over 16 waves 192 us; over 4
// with the factors read anew for every row 227), five of them to 2,560 elements
// (10,038 x 2,402 38.7 us, over eight 54, 10,160 x 2,560 38 | 41.5; six or seven gain less,
// and lose with float32's odd widths).  The plain quantiser has no factors and adds
// vectors first (17,472 x 1,001 float32 15.6 us with one wave, 17.1 with two).
template <typename T, bool NORM, int FIT>
static void run_quant(const RowQuant& a, hipStream_t st) {
  const int vecs = (a.d + 7) / 8;
  if (vecs <= 64) return run_rows<T, NORM, FIT, 1, 1>(a, st);
  if constexpr (FIT != SHORT) {
    if (vecs <= 128) return run_rows<T, NORM, FIT, NORM ? 2 : 1, NORM ? 1 : 2>(a, st);
    if (vecs <= 192) return run_rows<T, NORM, FIT, 3, 1>(a, st);
    if (vecs <= 256) return run_rows<T, NORM, FIT, 4, 1>(a, st);
    if constexpr (NORM) {
      if (vecs <= 320) return run_rows<T, NORM, FIT, 5, 1>(a, st);
    }
    if (vecs <= 512) return run_rows<T, NORM, FIT, NORM ? 8 : 4, NORM ? 1 : 2>(a, st);
    if (vecs <= 1024) return run_rows<T, NORM, FIT, NORM ? 16 : 4, NORM ? 1 : 4>(a, st);
    if (vecs <= 2048) return run_rows<T, NORM, FIT, 16, 2>(a, st);
    return run_rows<T, NORM, FIT, 16, 4>(a, st);
  }
}

hipError_t launch_quant_rows(int dtype, bool norm, const RowQuant& a, hipStream_t st) {
  if (a.rows <= 0) return hipSuccess;
  auto run = [&](auto type, auto with_norm) {
    using T = decltype(type);
    constexpr bool N = decltype(with_norm)::value;
    if (a.d % 8 == 0) run_quant<T, N, WHOLE>(a, st);
    else if (a.d > 8) run_quant<T, N, TAIL>(a, st);
    else run_quant<T, N, SHORT>(a, st);
  };
  if (dtype == 1) {
    if (norm) run(bf16_t{}, std::true_type{});
    else run(bf16_t{}, std::false_type{});
  } else {
    if (norm) run(float{}, std::true_type{});
    else run(float{}, std::false_type{});
  }
  return hipGetLastError();
}

}  // namespace swam
