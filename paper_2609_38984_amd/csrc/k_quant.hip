// Rows to 8-bit codes with a scale each: the residual addition and RMS norm in
// front of an 8-bit projection, and the plain quantiser of activations and
// weights.
//
//   t = x + r;  y = t / sqrt(mean t^2 + eps) * gain * (1 + scale) + shift
//   s = max|y| / 127;  code = round(y / s)
// Two numbers of the whole row (the mean square and the largest magnitude) stand
// between reading x and writing the codes.  The row stays on chip in float32
// between them, so every byte moves once: memory bounds it (rows * d * (x + r +
// sum + 1) bytes).
#include "launchers.h"

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

// 1 / sqrt(mean square + eps); NaN for a sum that is NaN or overflowed, so that every
// y and with it the scale is NaN; 0 for a row of zeros without eps
__device__ __forceinline__ float inv_rms(float ss, int d, float eps) {
  const float ms = ss / (float)d + eps;
  return !(ss < INFINITY) ? __uint_as_float(0x7fc00000u) : ms > 0.0f ? 1.0f / sqrtf(ms) : 0.0f;
}

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

// 8 elements at p, of which the first n are inside the row (n <= 0: none), as float32,
// and back; WHOLE: rows of whole vectors, n is never 1..7.  A vector moves in one
// access at any alignment of the element type (the hardware takes unaligned vectors;
// with scalar accesses 17,472 x 8,192 bf16 with rows 10 bytes off take 200 us, with
// vectors 90, aligned 88: 4.9 TB/s).
template <typename T> struct Raw8 { uint32_t w[2 * sizeof(T)]; };
template <bool WHOLE, typename T>
__device__ __forceinline__ void row_load8(const T* p, int n, float (&o)[8]) {
  if (n >= 8) {
    Raw8<T> r;
    __builtin_memcpy(&r, p, sizeof(r));
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
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = !WHOLE && e < n ? Elem<T>::load(p + e) : 0.0f;
  }
}
template <bool WHOLE, typename T>
__device__ __forceinline__ void row_store8(T* p, int n, const float (&v)[8]) {
  if (n >= 8) {
    Raw8<T> r;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int e = 0; e < 4; ++e) r.w[e] = pack_bf16x2(v[2 * e], v[2 * e + 1]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) r.w[e] = __float_as_uint(v[e]);
    }
    __builtin_memcpy(p, &r, sizeof(r));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (!WHOLE && e < n) Elem<T>::store(p + e, v[e]);
  }
}

// Rows of up to NW * 64 * 8 * NV elements in registers: NW waves to a row, lane t
// holding the 8-element vectors t, t + 64 NW, ...  NW = 1 puts four rows on a workgroup
// and needs no barrier; it pays to 1,024 elements (17,472 x 1,001 with the norm 41.7 us,
// two waves to a row 43.3).  From there on more, shorter waves leave less of a last round
// half empty (17,472 x 2,048 56 us, with one wave to a row 60; 10,160 x 1,536 28.1 | 29.4,
// 3.9 TB/s), and rows of more than 2,048 need the registers of several.
template <typename T, bool NORM, bool WHOLE, int NW, int NV>
__global__ void __launch_bounds__(NW == 1 ? 256 : NW * 64)
quant_rows(const RowQuant a) {
  constexpr int TPR = NW * 64, RPW = NW == 1 ? 4 : 1;
  __shared__ float red[NW];
  __shared__ uint32_t redu[NW];
  const int64_t row = (int64_t)blockIdx.x * RPW + (NW == 1 ? threadIdx.x / TPR : 0);
  if (row >= a.rows) return;                    // whole waves
  const int t = threadIdx.x % TPR, d = a.d;
  const T* xp = (const T*)a.x + row * a.x_ld;
  float v[NV][8];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int e = (i * TPR + t) * 8;
    row_load8<WHOLE>(xp + e, d - e, v[i]);
  }
  if constexpr (NORM) {
    float ss = 0.0f;
    if (a.res != nullptr) {
      const T* rp = (const T*)a.res + row * a.res_ld;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int e = (i * TPR + t) * 8;
        float r[8];
        row_load8<WHOLE>(rp + e, d - e, r);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] += r[j];
      }
    }
    if (a.sum != nullptr) {
      T* sp = (T*)a.sum + row * a.sum_ld;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int e = (i * TPR + t) * 8;
        row_store8<WHOLE>(sp + e, d - e, v[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) ss = fmaf(v[i][j], v[i][j], ss);
    ss = row_sum<NW>(ss, red);
    const float r = inv_rms(ss, d, a.eps);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int e = (i * TPR + t) * 8;
      if (e < d) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] *= r;
        if (a.gain != nullptr) {
          float g[8];
          row_load8<WHOLE>((const T*)a.gain + e, d - e, g);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[i][j] *= g[j];
        }
        if (a.shift != nullptr) {
          float sc[8], sh[8];
          row_load8<WHOLE>(a.scale + e, d - e, sc);
          row_load8<WHOLE>(a.shift + e, d - e, sh);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[i][j] = fmaf(v[i][j], 1.0f + sc[j], sh[j]);
        }
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
    const int e = (i * TPR + t) * 8;
    if (e < d) {
      int c[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) c[j] = code_of<!NORM>(v[i][j], rs);
      if (WHOLE || d - e >= 8) {
        const uint32_t w[2] = {pack4(c[0], c[1], c[2], c[3]), pack4(c[4], c[5], c[6], c[7])};
        __builtin_memcpy(qp + e, w, 8);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (e + j < d) qp[e + j] = (int8_t)c[j];
      }
    }
  }
  if (t == 0) a.q_scale[row] = rs.s;
}

template <typename T, bool NORM, bool WHOLE>
static void run_quant(const RowQuant& a, hipStream_t st) {
  const int vecs = (a.d + 7) / 8;
#define SWAM_Q(NW_, NV_)                                                                                   \
  hipLaunchKernelGGL((quant_rows<T, NORM, WHOLE, NW_, NV_>), dim3((unsigned)(NW_ == 1 ? (a.rows + 3) / 4 : a.rows)), \
                     dim3(NW_ == 1 ? 256 : NW_ * 64), 0, st, a)
  if (vecs <= 64) SWAM_Q(1, 1);
  else if (vecs <= 128) SWAM_Q(1, 2);
  else if (vecs <= 192) SWAM_Q(3, 1);
  else if (vecs <= 256) SWAM_Q(4, 1);
  else if (vecs <= 512) SWAM_Q(4, 2);
  else if (vecs <= 1024) SWAM_Q(4, 4);
  else if (vecs <= 2048) SWAM_Q(16, 2);
  else SWAM_Q(16, 4);
#undef SWAM_Q
}

hipError_t launch_quant_rows(int dtype, bool norm, const RowQuant& a, hipStream_t st) {
  if (a.rows <= 0) return hipSuccess;
  auto run = [&](auto type, auto with_norm) {
    using T = decltype(type);
    constexpr bool N = decltype(with_norm)::value;
    if (a.d % 8 == 0) run_quant<T, N, true>(a, st);
    else run_quant<T, N, false>(a, st);
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
