// Tiled MFMA product of e4m3 matrices with block scales (gfx950); instantiated
// by k_gemm_fp8.hip.
//
//   out[m][n] = act(sum_j sa[m][j] sw[n/128][j] sum_{k in block j} A[m][k] W[n][k] + bias[n])
//
// A scale block is 128 values of K, which is the K of one
// v_mfma_f32_16x16x128_f8f6f4: each block product is one MFMA onto zero, and its
// four results per lane join the float32 sum with one multiply-add each by the
// product of the two scales.  (The scales of the scaled MFMA are powers of two
// per 32 values; float32 scales need the multiply-add.)  The weight tile is the
// first operand, as in gemm_tile.h, so a lane owns four consecutive columns of
// one row.
//
// The 8-bit matrix instruction does not add all products in float32: in each
// group of 8 consecutive values of K it cuts every product, toward zero, below
// 2^-13 of the power of two of the group's largest one (measured; 16x16x32 the
// same), and only the groups' sums add in float32.  That is under the rounding
// of a bf16 result.  For float32 results (EXACT) the operands are converted to
// bf16, which holds every e4m3 value, and go through v_mfma_f32_16x16x32_bf16,
// whose products add in float32, at half the matrix rate.
//
// K advances one block (128 bytes of a row) per LDS stage; stages, swizzle and
// direct-to-LDS loads are those of gemm_tile.h, in bytes.  A lane's 32-byte
// operand is the chunks lg and lg + 4 of its row: which values of K a lane holds
// does not matter as long as both operands hold the same ones.  The scales of a
// stage's rows (a weight row's being its block's) travel with it, one float per
// row, by 4-byte loads straight into LDS.
#pragma once

#include "fp8.h"
#include "gemm_tile.h"

namespace wam {
namespace gemm {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

struct Fp8Operands {
  const uint8_t *a, *w;
  const float *sa, *sw;
  int64_t lda, ldw, ldsa, ldsw;  // row strides, in elements
  int M, N, K;
};

struct Fp8Out {
  const float* bias;  // or null
  void* out;
  int64_t ld;
  int bf16_out, gelu;
  int vec;  // rows and base allow stores of four elements
};

__device__ __forceinline__ void store_out(const Fp8Out& o, int m, int n, int N, f32x4 v) {
  if (o.gelu) v = gelu4(v);
  const int64_t off = (int64_t)m * o.ld + n;
  if (o.vec && n + 3 < N) {
    if (o.bf16_out) store4(static_cast<bf16*>(o.out) + off, v);
    else store4(static_cast<float*>(o.out) + off, v);
    return;
  }
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (n + r < N) {
      if (o.bf16_out) static_cast<bf16*>(o.out)[off + r] = static_cast<bf16>(v[r]);
      else static_cast<float*>(o.out)[off + r] = v[r];
    }
}

__device__ __forceinline__ f32x4 bias4(const float* bias, int n, int N) {
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (bias)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (n + r < N) v[r] = bias[n + r];
  return v;
}

// bf16 values of the bytes 8 t .. 8 t + 7 of a lane's operand
__device__ __forceinline__ bf16x8 to_bf16(const i32x8& v, int t) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  bf16x8 r;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * t + w], 1.0f, false);
    const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * t + w], 1.0f, true);
    r[4 * w] = lo[0], r[4 * w + 1] = lo[1], r[4 * w + 2] = hi[0], r[4 * w + 3] = hi[1];
  }
  return r;
}

template <int BM, int BN, int WGM, int WGN, int ST, bool EXACT>
__global__ __launch_bounds__(WGM* WGN * 64) void gemm_fp8_kernel(Fp8Operands p, Fp8Out o) {
  constexpr int BK = kScaleBlock;              // bytes of a row per stage
  constexpr int NW = WGM * WGN;
  constexpr int WM = BM / WGM, WN = BN / WGN;  // wave tile
  constexpr int TM = WM / 16, TN = WN / 16;
  constexpr int ROWS = BM + BN;
  constexpr int IPW = ROWS / 8 / NW;                       // 1 KiB loads per wave and stage (8 rows each)
  constexpr int SPW = (ROWS + 64 * NW - 1) / (64 * NW);    // loads of 64 scales per wave and stage
  static_assert(IPW * NW * 8 == ROWS, "stage rows / wave mismatch");
  static_assert(128 % WN == 0 && BN % WN == 0, "a wave's columns share a weight scale");
  static_assert(ST >= 2 && (ST - 2) * (IPW + SPW) < 64, "stage count");

  __shared__ __attribute__((aligned(1024))) uint8_t sm[ST][ROWS * BK];
  __shared__ __attribute__((aligned(256))) float sc[ST][SPW * NW * 64];

  const int tiles_m = (p.M + BM - 1) / BM, tiles_n = (p.N + BN - 1) / BN;
  int tm, tn;
  tile_coords(blockIdx.x, gridDim.x, tiles_m, tiles_n, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  const int tid = threadIdx.x, lane = tid % 64, wid = tid / 64;
  const int wm = wid / WGN, wn = wid % WGN;
  const int nk = (p.K + BK - 1) / BK;
  const int last = (p.K - 1) / 16 * 16;  // first byte of a row's last 16-byte chunk

  // Load j of this wave fills LDS rows 8 (wid + NW j) .. + 7 of the stage, lane l
  // the chunk l % 8 of row l / 8, i.e. global chunk (l % 8) ^ swizzle.  Rows past
  // M or N read the last one (never stored); chunks past K read the row's last
  // one and are cleared in LDS before use.
  const uint8_t* src[IPW];
  int col[IPW];
#pragma unroll
  for (int j = 0; j < IPW; ++j) {
    const int row = 8 * (wid + NW * j) + lane / 8;
    col[j] = ((lane % 8) ^ chunk_swizzle(row)) * 16;
    src[j] = row < BM ? p.a + (int64_t)min(m0 + row, p.M - 1) * p.lda
                      : p.w + (int64_t)min(n0 + row - BM, p.N - 1) * p.ldw;
  }
  const float* ssrc[SPW];
#pragma unroll
  for (int j = 0; j < SPW; ++j) {
    const int row = min(64 * (wid + NW * j) + lane, ROWS - 1);
    ssrc[j] = row < BM ? p.sa + (int64_t)min(m0 + row, p.M - 1) * p.ldsa
                       : p.sw + (int64_t)(min(n0 + row - BM, p.N - 1) / kScaleBlock) * p.ldsw;
  }
  auto issue = [&](auto S, int kt) __attribute__((always_inline)) {
    constexpr int s = decltype(S)::value;
#pragma unroll
    for (int j = 0; j < IPW; ++j)
      __builtin_amdgcn_global_load_lds((const global_void*)(src[j] + min(kt * BK + col[j], last)),
                                       (lds_void*)(&sm[s][(wid + NW * j) * 8 * BK]), 16, 0, 0);
#pragma unroll
    for (int j = 0; j < SPW; ++j)
      __builtin_amdgcn_global_load_lds((const global_void*)(ssrc[j] + kt), (lds_void*)(&sc[s][(wid + NW * j) * 64]), 4,
                                       0, 0);
  };

  f32x4 acc[TN][TM];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int i = 0; i < TM; ++i) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int lr = lane % 16, lg = lane / 16;
  const int ch0 = (lg ^ chunk_swizzle(lr)) * 16, ch1 = ((lg + 4) ^ chunk_swizzle(lr)) * 16;
  const int arow = (wm * WM + lr) * BK, wrow = (BM + wn * WN + lr) * BK;
  auto operand = [&](const uint8_t* row) __attribute__((always_inline)) {
    const i32x4 x = *reinterpret_cast<const i32x4*>(row + ch0), y = *reinterpret_cast<const i32x4*>(row + ch1);
    return i32x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
  };
  auto compute = [&](auto S) __attribute__((always_inline)) {
    constexpr int s = decltype(S)::value;
    const float sw = sc[s][BM + wn * WN];
    i32x8 wf[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) wf[j] = operand(&sm[s][wrow + j * 16 * BK]);
    bf16x8 wb[EXACT ? TN : 1][4];
    if constexpr (EXACT) {
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int t = 0; t < 4; ++t) wb[j][t] = to_bf16(wf[j], t);
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const i32x8 af = operand(&sm[s][arow + i * 16 * BK]);
      const float f = sc[s][wm * WM + i * 16 + lr] * sw;
      bf16x8 ab[4];
      if constexpr (EXACT) {
#pragma unroll
        for (int t = 0; t < 4; ++t) ab[t] = to_bf16(af, t);
      }
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        if constexpr (EXACT) {
#pragma unroll
          for (int t = 0; t < 4; ++t) v = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb[j][t], ab[t], v, 0, 0, 0);
        } else {
          v = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wf[j], af, v, 0, 0, 0, 0, 0, 0);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[j][i][r] = fmaf(v[r], f, acc[j][i][r]);
      }
    }
  };
  // clears the bytes past K of the last stage, in both operands (either may hold
  // a NaN there)
  auto clear_tail = [&](auto S) __attribute__((always_inline)) {
    constexpr int s = decltype(S)::value;
    const int used = p.K - (nk - 1) * BK;
    for (int c = tid; c < ROWS * 8; c += NW * 64) {
      const int row = c / 8, at = ((c % 8) ^ chunk_swizzle(row)) * 16;  // first byte of K in this chunk
      if (at + 16 <= used) continue;
      i32x4* q = reinterpret_cast<i32x4*>(&sm[s][row * BK + (c % 8) * 16]);
      i32x4 v = *q;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int keep = min(max(used - at - 4 * r, 0), 4);  // bytes of this word
        v[r] = keep == 4 ? v[r] : keep == 0 ? 0 : v[r] & ((1 << (8 * keep)) - 1);
      }
      *q = v;
    }
    __syncthreads();
  };
  // one K step on stage slot J, as in gemm_tile.h
  auto step = [&](auto J, int kt) __attribute__((always_inline)) {
    constexpr int j = decltype(J)::value;
    __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0((ST - 2) * (IPW + SPW)));
    compiler_fence();
    __builtin_amdgcn_s_barrier();
    compiler_fence();
    issue(std::integral_constant<int, (j + ST - 1) % ST>{}, min(kt + ST - 1, nk - 1));
    __builtin_amdgcn_sched_barrier(0);
    if (kt == nk - 1 && p.K % BK) clear_tail(J);
    compute(J);
  };

  static_for<ST - 1>([&](auto P) __attribute__((always_inline)) { issue(P, min((int)decltype(P)::value, nk - 1)); });
  const int nfull = nk / ST * ST;
  for (int kt0 = 0; kt0 < nfull; kt0 += ST)
    static_for<ST>([&](auto J) __attribute__((always_inline)) { step(J, kt0 + decltype(J)::value); });
  static_for<ST - 1>([&](auto J) __attribute__((always_inline)) {
    const int kt = nfull + decltype(J)::value;
    if (kt < nk) step(J, kt);
  });
  // no load may still be writing this block's LDS when the block retires
  __builtin_amdgcn_s_waitcnt(0);

#pragma unroll
  for (int j = 0; j < TN; ++j) {
    const int n = n0 + wn * WN + j * 16 + lg * 4;
    if (n >= p.N) continue;
    const f32x4 bias = bias4(o.bias, n, p.N);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int m = m0 + wm * WM + i * 16 + lr;
      if (m < p.M) store_out(o, m, n, p.N, acc[j][i] + bias);
    }
  }
}

}  // namespace gemm
}  // namespace wam
