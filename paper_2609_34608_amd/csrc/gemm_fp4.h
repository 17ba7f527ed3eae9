// Tiled MFMA product of matrices in 4-bit blocks (gfx950); instantiated by
// k_gemm_fp4.hip.
//
//   out[m][n] = act(sum_j 2^(sa[m][j] + sw[n][j] - 254) sum_{k in block j} A[m][k] W[n][k] + bias[n])
//
// v_mfma_scale_f32_16x16x128_f8f6f4 takes a scale byte per lane, i.e. per row and 32
// values of K: a block.  All accumulation stays in its float32 registers, so one
// kernel serves every type of result.  The weight tile is the first operand, as in
// gemm_tile.h, so a lane owns four consecutive columns of one row.
//
// K advances 128 bytes of a row (256 values, two MFMA steps) per LDS stage; stages,
// swizzle and direct-to-LDS loads are those of gemm_fp8.h.  Which values of K a lane
// holds does not matter as long as both operands hold the same ones: lane group g takes
// the chunks (16 bytes, one block) 2 g and 2 g + 1 of a stage, so that its two scale bytes
// are neighbours and come in one 16-bit read, the second step naming the second byte.
// The eight scale bytes of each row of a stage travel with it, by 4-byte loads
// straight into LDS.
//
// What bounds it: 10176 x 6144 x 1536 takes 64 us (3.0 PFLOP/s; the instruction alone
// reaches 9.5), 71 with the GELU, once the card has done such work for 40 ms (the clock moves: up
// to 95 before).  A 256x256 tile's six stages are 9.3 us of it each, at
// 55% of the matrix rate, and what it costs beside them 5.3: its first loads, the
// activation, and a result whose 125 MB alone take 20 us of memory.
#pragma once

#include "fp4.h"
#include "gemm_fp8.h"

namespace wam {
namespace gemm {

struct Fp4Operands {
  const uint8_t *a, *w, *sa, *sw;
  int64_t lda, ldw, ldsa, ldsw;  // row strides, in bytes
  int M, N, K;                   // K in values, even
};

// The product of one block's tile; epilogue(acc, m, n, lane, lds) takes a wave's
// accumulators, whose rows start at m and columns at n (lds: the stages, which no
// load writes any more but other waves may still read).  WIDE: rows further apart
// than 32-bit offsets inside a tile reach.
template <int BM, int BN, int WGM, int WGN, int ST, bool WIDE, typename EPILOGUE>
__device__ __forceinline__ void gemm_fp4_body(const Fp4Operands& p, EPILOGUE epilogue) {
  constexpr int BK = 128;                      // bytes of a row per stage
  constexpr int SB = BK / 16;                  // and scale bytes
  constexpr int NW = WGM * WGN;
  constexpr int WM = BM / WGM, WN = BN / WGN;  // wave tile
  constexpr int TM = WM / 16, TN = WN / 16;
  constexpr int ROWS = BM + BN;
  constexpr int IPW = ROWS / 8 / NW;                           // 1 KiB loads per wave and stage (8 rows each)
  constexpr int SPW = (ROWS * SB / 4 + 64 * NW - 1) / (64 * NW);  // loads of 64 words of scales
  static_assert(IPW * NW * 8 == ROWS, "stage rows / wave mismatch");
  static_assert(BN % WN == 0, "whole waves");
  static_assert(ST >= 2 && (ST - 2) * (IPW + SPW) < 64, "stage count");
  typedef typename std::conditional<WIDE, int64_t, uint32_t>::type offset;

  // a stage: operand rows, then their scales, in one object (gemm_fp8.h)
  constexpr int SCALES = ROWS * BK;
  constexpr int STAGE = SCALES + SPW * NW * 64 * 4;
  __shared__ __attribute__((aligned(1024))) uint8_t sm[ST][STAGE];

  const int tiles_m = (p.M + BM - 1) / BM, tiles_n = (p.N + BN - 1) / BN;
  int tm, tn;
  tile_coords(blockIdx.x, gridDim.x, tiles_m, tiles_n, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  const int tid = threadIdx.x, lane = tid % 64, wid = __builtin_amdgcn_readfirstlane(tid / 64);
  const int wm = wid / WGN, wn = wid % WGN;
  const int bytes = p.K / 2, nk = (bytes + BK - 1) / BK;
  const uint32_t last = (bytes - 1) / 16 * 16;                       // first byte of a row's last 16-byte chunk
  const uint32_t last_scale = ((p.K - 1) / kFp4Block) / 4 * 4;       // and of its last word of scales

  // Load j of this wave fills LDS rows 8 (wid + NW j) .. + 7 of the stage, lane l
  // the chunk l % 8 of row l / 8, i.e. global chunk (l % 8) ^ swizzle.  Rows past M or
  // N read the last one (never stored); chunks past K read the row's last one and are
  // cleared on their way into the MFMAs, like the words of scales past the last.
  const uint8_t* abase = p.a + (int64_t)m0 * p.lda;
  const uint8_t* wbase = p.w + (int64_t)n0 * p.ldw;
  const uint32_t col = ((lane % 8) ^ chunk_swizzle(lane / 8)) * 16;
  auto wcol = [&](int j) {  // of a load of weight rows: the swizzle's bits from the lane and from the load
    return (uint32_t)((lane % 8) ^ weight_swizzle<TN>(8 * (wid + NW * j) - BM + lane / 8)) * 16;
  };
  offset roff[IPW];
  const uint8_t* ssrc[SPW];
#pragma unroll
  for (int j = 0; j < IPW; ++j) {
    const int row = 8 * (wid + NW * j) + lane / 8;
    roff[j] = 8 * (wid + NW * j) < BM ? (offset)min(row, p.M - 1 - m0) * (offset)p.lda
                                      : (offset)min(row - BM, p.N - 1 - n0) * (offset)p.ldw;
  }
#pragma unroll
  for (int j = 0; j < SPW; ++j) {  // two words of a row
    const int row = min((64 * (wid + NW * j) + lane) / 2, ROWS - 1);
    ssrc[j] = row < BM ? p.sa + (int64_t)min(m0 + row, p.M - 1) * p.ldsa
                       : p.sw + (int64_t)min(n0 + row - BM, p.N - 1) * p.ldsw;
  }
  // loads lo .. hi - 1 of this wave's LPS for stage kt, the scales' last
  constexpr int LPS = IPW + SPW;
  auto issue = [&](auto S, int kt, int lo, int hi) __attribute__((always_inline)) {
    constexpr int s = decltype(S)::value;
    const uint32_t at = min(kt * BK + col, last);
#pragma unroll
    for (int j = 0; j < IPW; ++j) {
      if (j < lo || j >= hi) continue;
      const bool act = 8 * (wid + NW * j) < BM;
      const uint32_t c = act ? at : min(kt * BK + wcol(j), last);
      __builtin_amdgcn_global_load_lds((const global_void*)((act ? abase : wbase) + (offset)(roff[j] + c)),
                                       (lds_void*)(&sm[s][(wid + NW * j) * 8 * BK]), 16, 0, 0);
    }
    const uint32_t sat = min((uint32_t)(kt * SB + (lane % 2) * 4), last_scale);
#pragma unroll
    for (int j = 0; j < SPW; ++j)
      if (lo <= IPW + j && IPW + j < hi)
        __builtin_amdgcn_global_load_lds((const global_void*)(ssrc[j] + sat),
                                         (lds_void*)(&sm[s][SCALES + (wid + NW * j) * 64 * 4]), 4, 0, 0);
  };

  // loads per row tile, spread over about 5/8 of them
  constexpr int LPT = (8 * LPS + 5 * TM - 1) / (5 * TM);

  f32x4 acc[TN][TM];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int i = 0; i < TM; ++i) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int lr = lane % 16, lg = lane / 16;
  const int ch[2] = {((2 * lg) ^ chunk_swizzle(lr)) * 16, ((2 * lg + 1) ^ chunk_swizzle(lr)) * 16};
  const int arow = (wm * WM + lr) * BK, wrow = (BM + wn * WN + tile_row<kPaired<TN>>(0, lr)) * BK;
  const int ascale = SCALES + (wm * WM + lr) * SB + 2 * lg;
  const int wscale = SCALES + (BM + wn * WN + tile_row<kPaired<TN>>(0, lr)) * SB + 2 * lg;
  // TAIL: chunks past K of the last stage count as zero with a scale of one, in both
  // operands (either may hold anything there); the bytes past K of a chunk that it ends
  // in are cleared in LDS (clear_chunk).
  const int used = bytes - (nk - 1) * BK;
  auto operand = [&](const uint8_t* row, int t, auto TAIL) __attribute__((always_inline)) {
    i32x4 x = *reinterpret_cast<const i32x4*>(row + ch[t]);
    if constexpr (decltype(TAIL)::value) x &= 32 * lg + 16 * t < used ? -1 : 0;
    return i32x8{x[0], x[1], x[2], x[3], 0, 0, 0, 0};
  };
  auto scales = [&](const uint8_t* at, auto TAIL) __attribute__((always_inline)) {
    int s = *reinterpret_cast<const uint16_t*>(at);
    if constexpr (decltype(TAIL)::value) {
      if (32 * lg >= used) s = 0x7f7f;
      else if (32 * lg + 16 >= used) s = (s & 0xff) | 0x7f00;
    }
    return s;
  };
  auto clear_chunk = [&](int s) __attribute__((always_inline)) {
    for (int row = tid; row < ROWS; row += NW * 64) {
      const int sw = row < BM ? chunk_swizzle(row) : weight_swizzle<TN>(row - BM);
      i32x4* q = reinterpret_cast<i32x4*>(&sm[s][row * BK + ((used / 16) ^ sw) * 16]);
      i32x4 v = *q;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int keep = min(max(used % 16 - 4 * r, 0), 4);  // bytes of this word
        v[r] &= (int)(0xffffffffull >> (32 - 8 * keep));
      }
      *q = v;
    }
    __syncthreads();
  };
  // load(i) requests part of a later stage before the MFMAs of row tile i
  auto compute = [&](int s, auto TAIL, auto load) __attribute__((always_inline)) {
    i32x8 wf[TN][2];
    int ws[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      ws[j] = scales(&sm[s][wscale + tile_row<kPaired<TN>>(j, 0) * SB], TAIL);
#pragma unroll
      for (int t = 0; t < 2; ++t) wf[j][t] = operand(&sm[s][wrow + tile_row<kPaired<TN>>(j, 0) * BK], t, TAIL);
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      load(i);
      const int as = scales(&sm[s][ascale + i * 16 * SB], TAIL);
      i32x8 af[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) af[t] = operand(&sm[s][arow + i * 16 * BK], t, TAIL);
#pragma unroll
      for (int j = 0; j < TN; ++j)
        acc[j][i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wf[j][0], af[0], acc[j][i], 4, 4, 0, ws[j], 0, as);
#pragma unroll
      for (int j = 0; j < TN; ++j)
        acc[j][i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wf[j][1], af[1], acc[j][i], 4, 4, 1, ws[j], 1, as);
    }
  };
  // One K step on stage slot J (gemm_fp8.h): this wave's loads of stage kt have landed
  // (the ST - 2 newer stages may still be in flight) and its LDS reads are done; after
  // the barrier everyone's are, and the slot read in the previous step is free for
  // stage kt + ST - 1.  Past the last stage the loads repeat it into slots nobody reads
  // again.
  auto enter = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0((ST - 2) * LPS));
    compiler_fence();
    __builtin_amdgcn_s_barrier();
    compiler_fence();
    __builtin_amdgcn_s_setprio(1);
  };
  auto step = [&](auto J, int kt) __attribute__((always_inline)) {
    constexpr int j = decltype(J)::value;
    enter();
    compute(j, std::false_type{}, [&](int i) __attribute__((always_inline)) {
      issue(std::integral_constant<int, (j + ST - 1) % ST>{}, min(kt + ST - 1, nk - 1), i * LPT,
            i < TM - 1 ? (i + 1) * LPT : LPS);
    });
  };

  static_for<ST - 1>([&](auto P) __attribute__((always_inline)) { issue(P, min((int)decltype(P)::value, nk - 1), 0, LPS); });
  // whole rounds of the slots, what is left, and a last stage that K cuts off
  const int whole = nk - (bytes % BK != 0);
  const int rounds = whole / ST * ST;
  for (int kt0 = 0; kt0 < rounds; kt0 += ST)
    static_for<ST>([&](auto J) __attribute__((always_inline)) { step(J, kt0 + decltype(J)::value); });
  static_for<ST - 1>([&](auto J) __attribute__((always_inline)) {
    const int kt = rounds + decltype(J)::value;
    if (kt < whole) step(J, kt);
  });
  if (whole < nk) {
    enter();
    const int s = whole % ST;
    if (used % 16) clear_chunk(s);
    compute(s, std::true_type{}, [](int) {});
  }
  // no load may still be writing this block's LDS when the block retires
  __builtin_amdgcn_s_waitcnt(0);

  epilogue(acc, m0 + wm * WM, n0 + wn * WN, lane, &sm[0][0]);
}

// Bias, activation and 4-bit blocks of the result.  Two neighbouring tiles give a lane
// eight consecutive columns and the four lanes of a row 32: a block, whose maximum
// takes two exchanges.  The values never leave the registers unrounded.
template <int TN, int TM, bool GELU>
__device__ __forceinline__ void store_fp4_blocks(const Fp4Operands& p, const Fp8Out& o, uint8_t* scale,
                                                 const f32x4 (&acc)[TN][TM], int mb, int nb, int lane) {
  static_assert(TN % 2 == 0, "blocks of two tiles");
  const int lr = lane % 16, lg = lane / 16;
  float bias[TN / 2][8];
  load_bias<TN>(bias, o.bias, nb, lg, p.N);
  uint8_t* out = static_cast<uint8_t*>(o.out);
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int m = mb + i * 16 + lr;
#pragma unroll
    for (int j = 0; j < TN / 2; ++j) {
      const int n = nb + tile_col<true>(2 * j, lg);
      float x[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        const float v = acc[2 * j + r / 4][i][r % 4] + bias[j][r];
        x[r] = n + r < p.N ? (GELU ? gelu_tanh_f(v) : v) : 0.f;  // columns past N are no part of their block
      }
      uint32_t most = 0;
#pragma unroll
      for (int r = 0; r < 8; ++r) most = max(most, abs_bits(x[r]));
      most = max(most, (uint32_t)__shfl_xor((int)most, 16, 64));
      most = max(most, (uint32_t)__shfl_xor((int)most, 32, 64));
      const uint32_t byte = fp4_scale(most);
      const uint32_t w = pack_fp4(x, byte);
      if (m >= p.M || n >= p.N) continue;
      store_fp4(out + m * o.ld + n / 2, w, p.N - n);
      if (lg == 0) scale[m * o.ldscale + n / kFp4Block] = (uint8_t)byte;
    }
  }
}

template <int BM, int BN, int WGM, int WGN, int ST, bool FLOAT, bool GELU, bool WIDE>
__global__ __launch_bounds__(WGM* WGN * 64) void gemm_fp4_kernel(Fp4Operands p, Fp8Out o) {
  constexpr int TM = BM / WGM / 16, TN = BN / WGN / 16;
  gemm_fp4_body<BM, BN, WGM, WGN, ST, WIDE>(
      p, [&](const f32x4(&acc)[TN][TM], int m, int n, int lane, uint8_t* lds) __attribute__((always_inline)) {
        store_product<TN, TM, FLOAT, GELU>(p, o, acc, m, n, lane, lds);
      });
}

template <int BM, int BN, int WGM, int WGN, int ST, bool GELU, bool WIDE>
__global__ __launch_bounds__(WGM* WGN * 64) void gemm_fp4_blocks_kernel(Fp4Operands p, Fp8Out o, uint8_t* scale) {
  constexpr int TM = BM / WGM / 16, TN = BN / WGN / 16;
  gemm_fp4_body<BM, BN, WGM, WGN, ST, WIDE>(
      p, [&](const f32x4(&acc)[TN][TM], int m, int n, int lane, uint8_t*) __attribute__((always_inline)) {
        store_fp4_blocks<TN, TM, GELU>(p, o, scale, acc, m, n, lane);
      });
}

}  // namespace gemm
}  // namespace wam
