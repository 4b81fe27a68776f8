// 8-bit projections: C = epi(a_scale b_scale (A . B^T) + bias), A [M][K] and
// B [N][K] int8 codes with a scale per row, the sum exact in int32.
//
// A 128-byte row of an LDS tile holds 128 codes of K: the tiles have the layout
// of the bf16 projections (16-byte chunk ^ lds_swz(row)) at twice the depth, and
// a 32x32x32 MFMA takes one 16-byte chunk per lane and operand.  Global -> LDS
// by buffer loads whose descriptors end with the operand, so rows past M or N
// and, by an offset past the end, chunks past K read as zeros.
#include "gemm_common.h"

namespace swam {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

constexpr int I8_BK = 128;            // codes of K per stage: one 128-byte row
constexpr int PAST_END = 0x7fffff00;  // a buffer offset that no operand reaches

// The operand's bytes from its tile's first row on; rows * ld stays below
// 2^31 for the rows of a tile, so a clamped size hides none of them.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t i8_rows(const int8_t* p, int64_t ld, int r0, int rows, int64_t K) {
  const int64_t bytes = (int64_t)(rows - r0 - 1) * ld + K;
  return __builtin_amdgcn_make_buffer_rsrc((void*)(p + r0 * ld), (short)0,
                                           (int)min(bytes, (int64_t)0x7fff0000), SWAM_BUF_DWORD3);
}

// 8 columns of a row: scale, bias, GELU or gated residual, rounded once
template <typename T>
struct I8Epilogue {
  const GemmI8 g;
  int vec;       // whole, 16-byte aligned runs of 8 columns in c, residual, bias
  __device__ __forceinline__ void run(const int (&acc)[8], int64_t row, int col) const {
    if (row >= g.M || col >= g.N) return;
    const float sa = g.a_scale[row];
    T* cp = (T*)g.c + row * g.ldc + col;
    const T* rp = g.res ? (const T*)g.res + row * g.ldr + col : nullptr;
    const T* bp = g.bias ? (const T*)g.bias + col : nullptr;
    if (vec && col + 8 <= g.N) {
      float z[8], b[8], r[8];
      if (bp) load8(bp, b);
      if (rp) load8(rp, r);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        z[e] = (float)acc[e] * (sa * g.b_scale[col + e]) + (bp ? b[e] : 0.0f);
        if (g.gelu) z[e] = gelu_tanh(z[e]);
        if (rp) z[e] = fmaf(g.gate ? g.gate[col + e] : 1.0f, z[e], r[e]);
      }
      store8(cp, z);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (col + e >= g.N) return;
        float z = (float)acc[e] * (sa * g.b_scale[col + e]) + (bp ? Elem<T>::load(bp + e) : 0.0f);
        if (g.gelu) z = gelu_tanh(z);
        if (rp) z = fmaf(g.gate ? g.gate[col + e] : 1.0f, z, Elem<T>::load(rp + e));
        Elem<T>::store(cp + e, z);
      }
    }
  }
};

template <typename T, int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(WM * WN * 64)
gemm_i8(const I8Epilogue<T> ep, int tiles_m, int tiles_n) {
  constexpr int NW = WM * WN, TM = BM / WM, TN = BN / WN, FM = TM / 32, FN = TN / 32;
  constexpr int A_INS = BM / 8 / NW, B_INS = BN / 8 / NW;
  constexpr int STAGE = (BM + BN) * 8;
  __shared__ uint4 lds[2 * STAGE];
  const GemmI8& g = ep.g;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int tm, tn;
  tile_of(blockIdx.x, tiles_m * tiles_n, tiles_m, tiles_n, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN, wm = wave / WN, wn = wave % WN;
  const int lrow = lane >> 3, K = (int)g.K;
  const __amdgpu_buffer_rsrc_t ra = i8_rows(g.a, g.lda, m0, (int)g.M, g.K);
  const __amdgpu_buffer_rsrc_t rb = i8_rows(g.b, g.ldb, n0, (int)g.N, g.K);
  auto issue = [&](uint4* as, uint4* bs, int k0) {
#pragma unroll
    for (int j = 0; j < A_INS; ++j) {
      const int r = (wave * A_INS + j) * 8 + lrow, kc = k0 + 16 * ((lane & 7) ^ lds_swz(r));
      const int off = kc < K ? r * (int)g.lda + kc : PAST_END;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_void_t*)(as + (wave * A_INS + j) * 64), 16, off, 0, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < B_INS; ++j) {
      const int r = (wave * B_INS + j) * 8 + lrow, kc = k0 + 16 * ((lane & 7) ^ lds_swz(r));
      const int off = kc < K ? r * (int)g.ldb + kc : PAST_END;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_void_t*)(bs + (wave * B_INS + j) * 64), 16, off, 0, 0, 0);
    }
  };
  i32x16 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;
  const int KT = (K + I8_BK - 1) / I8_BK, half = lane >> 5, r31 = lane & 31, sw = lds_swz(r31);
  issue(lds, lds + BM * 8, 0);
  for (int kt = 0; kt < KT; ++kt) {
    uint4* cur = lds + (kt & 1) * STAGE;
    uint4* nxt = lds + ((kt + 1) & 1) * STAGE;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (kt + 1 < KT) issue(nxt, nxt + BM * 8, (kt + 1) * I8_BK);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      i32x4 af[FM], bf[FN];
      const int ch = (2 * s + half) ^ sw;
#pragma unroll
      for (int i = 0; i < FM; ++i) af[i] = __builtin_bit_cast(i32x4, cur[(wm * TM + i * 32 + r31) * 8 + ch]);
#pragma unroll
      for (int j = 0; j < FN; ++j)
        bf[j] = __builtin_bit_cast(i32x4, cur[(BM + wn * TN + j * 32 + r31) * 8 + ch]);
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(af[i], bf[j], acc[i][j], 0, 0, 0);
    }
  }
  __syncthreads();
  constexpr int EP_LD = TN + 4;
  static_assert(NW * 32 * EP_LD * 4 <= (int)sizeof(lds), "epilogue staging exceeds LDS");
  int* park = reinterpret_cast<int*>(lds) + wave * 32 * EP_LD;
#pragma unroll
  for (int i = 0; i < FM; ++i) {
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        park[(8 * (r >> 2) + 4 * half + (r & 3)) * EP_LD + j * 32 + r31] = acc[i][j][r];
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_s_waitcnt(0xc07f);
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int it = 0; it < 32 * TN / 8 / 64; ++it) {
      const int rl = (lane + 64 * it) / (TN / 8), cl = (lane + 64 * it) % (TN / 8) * 8;
      int v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = park[rl * EP_LD + cl + e];
      ep.run(v, m0 + wm * TM + i * 32 + rl, n0 + wn * TN + cl);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

template <typename T>
static void run_gemm_i8(const GemmI8& g, hipStream_t st) {
  const int esz = sizeof(T);
  auto row16 = [&](const void* p, int64_t ld) { return (((uintptr_t)p | (uintptr_t)(ld * esz)) & 15) == 0; };
  const I8Epilogue<T> ep{g, row16(g.c, g.ldc) && row16(g.res, g.res ? g.ldr : 0) && row16(g.bias, 0)};
  const int tm = (int)((g.M + 127) / 128), tn = (int)((g.N + 127) / 128);
  hipLaunchKernelGGL((gemm_i8<T, 128, 128, 2, 2>), dim3(tm * tn), dim3(256), 0, st, ep, tm, tn);
}

hipError_t launch_gemm_i8(int dtype, const GemmI8& g, int32_t* ws, int64_t ws_words, hipStream_t st) {
  if (g.M <= 0 || g.N <= 0) return hipSuccess;
  (void)ws; (void)ws_words;
  if (dtype == 1) run_gemm_i8<bf16_t>(g, st);
  else run_gemm_i8<float>(g, st);
  return hipGetLastError();
}

}  // namespace swam
