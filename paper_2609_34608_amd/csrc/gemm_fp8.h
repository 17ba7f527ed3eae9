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
// same), and only the groups' sums add in float32.  Against those products that is
// finer than a bf16 result's rounding (2^-8); against a sum in which they cancel it
// need not be.  bf16 and e4m3 results take it, and so do the gated residuals of the
// 8-bit layers, whose operands are rounded to 2^-4 anyway.  For the operator's float32
// results (EXACT) the operands are converted to bf16, which holds every e4m3 value,
// and go through v_mfma_f32_16x16x32_bf16, whose products add in float32, at half the
// matrix rate.
//
// The two scales of a block are multiplied first, so a block whose product of scales is
// subnormal or infinite is not what float64 makes of it.  A check of every stage's scales, with a second pass over the tile
// that splits far ones into a power of two and a rest, was right at any scale and
// cost every product its registers and issue slots (10176 x 6144 x 1536 102 -> 128 us, 9224
// x 1024 x 4096 44.7 -> 47.4, 864 x 2304 x 768 7.5 -> 7.9).
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

// Weight rows are dealt to the MFMA tiles in pairs (tile_row) where a wave has an
// even number of them.
template <int TN>
constexpr bool kPaired = TN % 2 == 0;
// XOR swizzle of a weight row's chunks: index i of every tile gets i & 7, as an
// activation row does
template <int TN>
__host__ __device__ constexpr int weight_swizzle(int row) {
  return kPaired<TN> ? (row & 3) | ((row >> 3) & 1) << 2 : row & 7;
}

struct Fp8Operands {
  const uint8_t *a, *w;
  const float *sa, *sw;
  int64_t lda, ldw, ldsa, ldsw;  // row strides, in elements
  int M, N, K;
};

struct Fp8Out {
  const float* bias;  // or null
  void* out;          // bf16, float32 of an EXACT product, or e4m3 with
  int64_t ld;
  float* scale;       // a scale per row and 128 columns
  int64_t ldscale;
};

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

// The product of one block's tile; epilogue(acc, m, n, lane, lds) takes a wave's
// accumulators, whose rows start at m and columns at n (lds: the stages, which no
// load writes any more but other waves may still read).  WIDE: rows further apart
// than 32-bit offsets inside a tile reach.
template <int BM, int BN, int WGM, int WGN, int ST, bool EXACT, bool WIDE, typename EPILOGUE>
__device__ __forceinline__ void gemm_fp8_body(const Fp8Operands& p, EPILOGUE epilogue) {
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
  typedef typename std::conditional<WIDE, int64_t, uint32_t>::type offset;

  // a stage: operand rows, then their scales.  One object: with the scales in a
  // second one the compiler takes every LDS read to depend on the loads in flight
  // and waits for all of them, which serialises loads and MFMAs.
  constexpr int SCALES = ROWS * BK;
  constexpr int STAGE = SCALES + SPW * NW * 64 * 4;
  __shared__ __attribute__((aligned(1024))) uint8_t sm[ST][STAGE];

  const int tiles_m = (p.M + BM - 1) / BM, tiles_n = (p.N + BN - 1) / BN;
  int tm, tn;
  tile_coords(blockIdx.x, gridDim.x, tiles_m, tiles_n, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  const int tid = threadIdx.x, lane = tid % 64, wid = __builtin_amdgcn_readfirstlane(tid / 64);
  const int wm = wid / WGN, wn = wid % WGN;
  const int nk = (p.K + BK - 1) / BK;
  const uint32_t last = (p.K - 1) / 16 * 16;  // first byte of a row's last 16-byte chunk

  // Load j of this wave fills LDS rows 8 (wid + NW j) .. + 7 of the stage, lane l
  // the chunk l % 8 of row l / 8, i.e. global chunk (l % 8) ^ swizzle (the same
  // for every j).  Rows past M or N read the last one (never stored); chunks past
  // K read the row's last one and are cleared on their way into the MFMAs.
  const uint8_t* abase = p.a + (int64_t)m0 * p.lda;
  const uint8_t* wbase = p.w + (int64_t)n0 * p.ldw;
  const uint32_t col = ((lane % 8) ^ chunk_swizzle(lane / 8)) * 16;
  auto wcol = [&](int j) {  // of a load of weight rows: the swizzle's bits from the lane and from the load
    return (uint32_t)((lane % 8) ^ weight_swizzle<TN>(8 * (wid + NW * j) - BM + lane / 8)) * 16;
  };
  offset roff[IPW];
  const float* ssrc[SPW];
#pragma unroll
  for (int j = 0; j < IPW; ++j) {
    const int row = 8 * (wid + NW * j) + lane / 8;
    roff[j] = 8 * (wid + NW * j) < BM ? (offset)min(row, p.M - 1 - m0) * (offset)p.lda
                                      : (offset)min(row - BM, p.N - 1 - n0) * (offset)p.ldw;
  }
#pragma unroll
  for (int j = 0; j < SPW; ++j) {
    const int row = min(64 * (wid + NW * j) + lane, ROWS - 1);
    ssrc[j] = row < BM ? p.sa + (int64_t)min(m0 + row, p.M - 1) * p.ldsa
                       : p.sw + (int64_t)(min(n0 + row - BM, p.N - 1) / kScaleBlock) * p.ldsw;
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
#pragma unroll
    for (int j = 0; j < SPW; ++j)
      if (lo <= IPW + j && IPW + j < hi)
        __builtin_amdgcn_global_load_lds((const global_void*)(ssrc[j] + kt),
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
  const int ch0 = (lg ^ chunk_swizzle(lr)) * 16, ch1 = ((lg + 4) ^ chunk_swizzle(lr)) * 16;
  const int arow = (wm * WM + lr) * BK, wrow = (BM + wn * WN + tile_row<kPaired<TN>>(0, lr)) * BK;
  // TAIL: chunks past K of the last stage count as zero, in both operands (either may
  // hold a NaN there); the bytes past K of a chunk that it ends in are cleared in
  // LDS (clear_chunk).
  const int used = p.K - (nk - 1) * BK;
  auto operand = [&](const uint8_t* row, auto TAIL) __attribute__((always_inline)) {
    i32x4 x = *reinterpret_cast<const i32x4*>(row + ch0), y = *reinterpret_cast<const i32x4*>(row + ch1);
    if constexpr (decltype(TAIL)::value) {
      x &= 16 * lg < used ? -1 : 0;
      y &= 64 + 16 * lg < used ? -1 : 0;
    }
    return i32x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
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
  // The multiply-adds of row tile i run behind the MFMAs of row tile i + 1, one
  // MFMA and four multiply-adds in turn, so that neither unit waits for the other.
  // load(i) requests part of a later stage before the MFMAs of row tile i.
  auto compute = [&](int s, auto TAIL, auto load) __attribute__((always_inline)) {
    const float* sc = reinterpret_cast<const float*>(&sm[s][SCALES]);
    const float sw = sc[BM + wn * WN];
    float f[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) f[i] = sc[wm * WM + i * 16 + lr] * sw;
    i32x8 wf[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) wf[j] = operand(&sm[s][wrow + tile_row<kPaired<TN>>(j, 0) * BK], TAIL);
    if constexpr (EXACT) {
      bf16x8 wb[TN][4];
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int t = 0; t < 4; ++t) wb[j][t] = to_bf16(wf[j], t);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        load(i);
        const i32x8 af = operand(&sm[s][arow + i * 16 * BK], TAIL);
        bf16x8 ab[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) ab[t] = to_bf16(af, t);
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int t = 0; t < 4; ++t) v = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb[j][t], ab[t], v, 0, 0, 0);
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[j][i][r] = fmaf(v[r], f[i], acc[j][i][r]);
        }
      }
    } else {
      const f32x4 z = {0.f, 0.f, 0.f, 0.f};
      f32x4 v[2][TN];
      i32x8 af[2];
      af[0] = operand(&sm[s][arow], TAIL);
#pragma unroll
      for (int i = 0; i <= TM; ++i) {
        if (i + 1 < TM) af[(i + 1) & 1] = operand(&sm[s][arow + (i + 1) * 16 * BK], TAIL);
        if (i < TM) load(i);
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          if (i < TM)
            v[i & 1][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wf[j], af[i & 1], z, 0, 0, 0, 0, 0, 0);
          if (i > 0)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[j][i - 1][r] = fmaf(v[(i - 1) & 1][j][r], f[i - 1], acc[j][i - 1][r]);
          if (i > 0 && i < TM) {
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);  // one MFMA
            __builtin_amdgcn_sched_group_barrier(0x2, 4, 0);  // four VALU
            if (j == 0) __builtin_amdgcn_sched_group_barrier(0x10, LPT, 0);  // the loads
          }
        }
      }
    }
  };
  // One K step on stage slot J: this wave's loads of stage kt have landed (the ST - 2
  // newer stages may still be in flight) and its LDS reads are done; after the
  // barrier everyone's are, and the slot read in the previous step is free for
  // stage kt + ST - 1.  Its loads go out a few at a time between the MFMAs of the
  // first row tiles: all at once they fill the load path and every wave waits for
  // its turn before its first MFMA (M = 10176, N = 1536, K = 6144: 100 -> 90 us).
  // Waves that have passed the barrier go before those that have not (90 -> 87 us).
  // Past the last stage the loads repeat it into slots nobody reads again.
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
  const int whole = nk - (p.K % BK != 0);
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

// bias of a lane's columns (zeros without one; columns past N take the last)
template <int TN, int J, int W>
__device__ __forceinline__ void load_bias(float (&bias)[J][W], const float* from, int nb, int lg, int N) {
#pragma unroll
  for (int j = 0; j < J; ++j)
#pragma unroll
    for (int r = 0; r < W; ++r) bias[j][r] = 0.f;
  if (from)
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int r = 0; r < W; ++r) bias[j][r] = from[min(nb + tile_col<kPaired<TN>>(j * (TN / J), lg) + r, N - 1)];
}

// Bias, activation and 8-bit blocks of the result.  A block's 128 columns are those
// of two neighbouring waves (64 each), which meet in LDS: the largest magnitude of
// a row's columns over the lane's values, the row's four lanes, the two waves.  The
// values themselves never leave the registers unrounded.
template <int TN, int TM, bool GELU>
__device__ __forceinline__ void store_blocks(const Fp8Operands& p, const Fp8Out& o, f32x4 (&acc)[TN][TM], int mb,
                                             int nb, int lane, uint8_t* lds) {
  static_assert(TN == 4, "two waves to a block");
  const int lr = lane % 16, lg = lane / 16, wid = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  uint32_t(*top)[TM * 16] = reinterpret_cast<uint32_t(*)[TM * 16]>(lds);
  constexpr int W = 8;
  const bool ragged = nb + TN * 16 > p.N;
  float bias[TN / 2][W];
  load_bias<TN>(bias, o.bias, nb, lg, p.N);
  __syncthreads();  // the stages have been read
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float v = acc[j][i][r] + bias[j / 2][j % 2 * 4 + r];
        if (GELU) v = gelu_tanh_f(v);
        acc[j][i][r] = v;
        most = max(most, abs_bits(v));
      }
    if (ragged) {  // columns past N are no part of their block
      most = 0;
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (nb + tile_col<true>(j, lg) + r < p.N) most = max(most, abs_bits(acc[j][i][r]));
    }
    most = max(most, (uint32_t)__shfl_xor((int)most, 16, 64));
    most = max(most, (uint32_t)__shfl_xor((int)most, 32, 64));
    if (lg == 0) top[wid][i * 16 + lr] = most;
  }
  __syncthreads();
  struct __attribute__((packed, aligned(1))) Row {
    uint32_t v[2];
  };
  uint8_t* out = static_cast<uint8_t*>(o.out);
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int m = mb + i * 16 + lr;
    const float s = block_scale(max(top[wid][i * 16 + lr], top[wid ^ 1][i * 16 + lr]));
    const Divisor by = divisor(s);
    if (m >= p.M) continue;
    if (lg == 0 && wid % 2 == 0 && nb < p.N) o.scale[m * o.ldscale + nb / kScaleBlock] = s;
    uint8_t* row = out + m * o.ld + nb;
#pragma unroll
    for (int j = 0; j < TN; j += 2) {
      const int c = tile_col<true>(j, lg);
      Row x;
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const f32x4 v = acc[j + w][i];
        x.v[w] = pack_e4m3(divide_by(v[0], by), divide_by(v[1], by), divide_by(v[2], by), divide_by(v[3], by));
      }
      if (nb + c + W <= p.N) *reinterpret_cast<Row*>(row + c) = x;
    }
  }
  if (!ragged || p.N % W == 0) return;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int m = mb + i * 16 + lr;
    const float s = block_scale(max(top[wid][i * 16 + lr], top[wid ^ 1][i * 16 + lr]));
#pragma unroll
    for (int j = 0; j < TN; j += 2) {
      const int n = nb + tile_col<true>(j, lg);
      if (m >= p.M || n >= p.N || n + W <= p.N) continue;
#pragma unroll
      for (int c = 0; c < W; ++c)
        if (n + c < p.N) out[m * o.ld + n + c] = to_e4m3(acc[j + c / 4][i][c % 4] / s);
    }
  }
}

// Bias, activation and rounding of a wave's accumulators into an M x N result (p.M, p.N)
// of any row stride.
template <int TN, int TM, bool EXACT, bool GELU, typename SIZES>
__device__ __forceinline__ void store_product(const SIZES& p, const Fp8Out& o, const f32x4 (&acc)[TN][TM],
                                              int mb, int nb, int lane, uint8_t* lds) {
  const int lr = lane % 16, lg = lane / 16;
  // G tiles side by side hold W consecutive columns of a lane.  Global memory takes
  // wide stores at any address, so rows of any stride do; only columns that N cuts
  // off go one by one, in a pass of their own that most blocks skip.
  constexpr int G = TN % 2 ? 1 : 2, W = 4 * G;
  typedef typename std::conditional<EXACT, float, bf16>::type T;
  struct __attribute__((packed, aligned(sizeof(T)))) Row {
    T v[W];
  };
  float bias[TN / G][W];
  load_bias<TN>(bias, o.bias, nb, lg, p.N);
  auto value = [&](int j, int i, int r) __attribute__((always_inline)) {
    const float v = acc[j * G + r / 4][i][r % 4] + bias[j][r];
    return static_cast<T>(GELU ? gelu_tanh_f(v) : v);
  };
  T* out = static_cast<T*>(o.out);
  // Rows of bf16 that start inside a word: stores there leave a word to two lanes,
  // which do not meet in one request (10176 x 6144 x 1536 with rows of 6145: 147 us, 107
  // with the same stores on words).  Such a row is shifted by one column, the next
  // lanes' first one coming in, so that only the first and the last column of a
  // wave are stored by themselves (115 us).
  const bool shift = !EXACT && ((reinterpret_cast<uintptr_t>(out) | (uintptr_t)o.ld * 2) & 2);
  if constexpr (!EXACT && TN == 4) {
    // A wave has 128 bytes of a row: they go out through LDS, so that eight lanes side
    // by side store them, and past kStreamBytes as streaming stores where rows
    // start on lines (10176 x 6144 x 1536 106 -> 100 us, with the GELU 115 -> 109; rows of
    // 6152, whose lines two waves share, 106 -> 119).
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    __syncthreads();  // the stages have been read
    if (!shift && nb + TN * 16 <= p.N) {
      const bool stream = (int64_t)p.M * p.N * 2 > kStreamBytes &&
                          (reinterpret_cast<uintptr_t>(out) | (uintptr_t)o.ld * 2) % 128 == 0;
      uint8_t* st = lds + __builtin_amdgcn_readfirstlane(threadIdx.x / 64) * 2048;
      const int sr = lane / 8, sc = lane % 8;
#pragma unroll
      for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          Row x;
#pragma unroll
          for (int r = 0; r < W; ++r) x.v[r] = value(j, i, r);
          words v;
          __builtin_memcpy(&v, &x, 16);
          *reinterpret_cast<words*>(st + lr * 128 + (((j * 4 + lg) ^ (lr & 7)) * 16)) = v;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int row = h * 8 + sr, m = mb + i * 16 + row;
          const words v = *reinterpret_cast<const words*>(st + row * 128 + ((sc ^ sr) * 16));
          if (m < p.M) put(out + (int64_t)m * o.ld + nb + sc * 8, v, stream);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
      return;
    }
  }
  if (shift) {
    constexpr int NJ = TN / G, V = W / 2;
    struct __attribute__((packed, aligned(2))) Words {
      uint32_t v[V];
    };
    struct __attribute__((packed, aligned(2))) Cut {
      uint32_t v[V - 1];
    };
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int m = mb + i * 16 + lr;
      T* row = out + (int64_t)m * o.ld + nb;
      const int odd = reinterpret_cast<uintptr_t>(row) & 2 ? 1 : 0;
      uint32_t w[NJ][V], next[NJ];
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const bf16 x[2] = {static_cast<bf16>(value(j, i, 2 * k)), static_cast<bf16>(value(j, i, 2 * k + 1))};
          w[j][k] = __builtin_bit_cast(uint32_t, x);
        }
        next[j] = (uint32_t)__shfl((int)w[j][0], (lane + 16) % 64, 64);
      }
      if (m >= p.M) continue;
      if (odd && lg == 0 && nb < p.N) row[0] = value(0, i, 0);
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const uint32_t after = lg < 3 || j + 1 == NJ ? next[j] : next[(j + 1) % NJ];
        Words x;
#pragma unroll
        for (int k = 0; k < V; ++k)
          x.v[k] = odd ? w[j][k] >> 16 | (k + 1 < V ? w[j][(k + 1) % V] : after) << 16 : w[j][k];
        const int c = tile_col<kPaired<TN>>(j * G, lg) + odd;
        if (c + W <= min(p.N - nb, TN * 16)) {
          *reinterpret_cast<Words*>(row + c) = x;
        } else if (c + W > TN * 16 && c + W - 1 <= p.N - nb) {
          Cut y;
#pragma unroll
          for (int k = 0; k < V - 1; ++k) y.v[k] = x.v[k];
          *reinterpret_cast<Cut*>(row + c) = y;
          row[c + W - 2] = value(j, i, W - 1);
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int m = mb + i * 16 + lr;
      if (m >= p.M) continue;
#pragma unroll
      for (int j = 0; j < TN / G; ++j) {
        const int n = nb + tile_col<kPaired<TN>>(j * G, lg);
        Row x;
#pragma unroll
        for (int r = 0; r < W; ++r) x.v[r] = value(j, i, r);
        if (n + W <= p.N) *reinterpret_cast<Row*>(out + (int64_t)m * o.ld + n) = x;
      }
    }
  }
  if ((p.N % W || shift) && nb + TN * 16 > p.N) {
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int m = mb + i * 16 + lr;
      T* row = out + (int64_t)m * o.ld;
      const int odd = shift && (reinterpret_cast<uintptr_t>(row + nb) & 2) ? 1 : 0;
#pragma unroll
      for (int j = 0; j < TN / G; ++j) {
        const int n = nb + tile_col<kPaired<TN>>(j * G, lg);
        if (m >= p.M || n >= p.N || n + odd + W <= p.N) continue;
#pragma unroll
        for (int r = 0; r < W; ++r)
          if (n + r < p.N) row[n + r] = value(j, i, r);
      }
    }
  }
}

template <int BM, int BN, int WGM, int WGN, int ST, bool EXACT, bool GELU, bool WIDE>
__global__ __launch_bounds__(WGM* WGN * 64) void gemm_fp8_kernel(Fp8Operands p, Fp8Out o) {
  constexpr int TM = BM / WGM / 16, TN = BN / WGN / 16;
  gemm_fp8_body<BM, BN, WGM, WGN, ST, EXACT, WIDE>(
      p, [&](const f32x4(&acc)[TN][TM], int m, int n, int lane, uint8_t* lds) __attribute__((always_inline)) {
        store_product<TN, TM, EXACT, GELU>(p, o, acc, m, n, lane, lds);
      });
}

template <int BM, int BN, int WGM, int WGN, int ST, bool GELU>
__global__ __launch_bounds__(WGM* WGN * 64) void gemm_fp8_blocks_kernel(Fp8Operands p, Fp8Out o, const int* skip) {
  constexpr int TM = BM / WGM / 16, TN = BN / WGN / 16;
  if (skip && *skip) return;
  gemm_fp8_body<BM, BN, WGM, WGN, ST, false, false>(
      p, [&](f32x4(&acc)[TN][TM], int m, int n, int lane, uint8_t* lds) __attribute__((always_inline)) {
        store_blocks<TN, TM, GELU>(p, o, acc, m, n, lane, lds);
      });
}

// A projection of the DiT block (store_tile's epilogues, N a multiple of 64).
template <int BM, int BN, int WGM, int WGN, int ST, int EPI>
__global__ __launch_bounds__(WGM* WGN * 64) void gemm_fp8_layer_kernel(Fp8Operands p, GemmArgs g) {
  constexpr int TM = BM / WGM / 16, TN = BN / WGN / 16;
  static_assert(EPI != EPI_QKV || TN == 4, "QKV epilogue needs whole heads per wave");
  if (g.skip && *g.skip) return;
  gemm_fp8_body<BM, BN, WGM, WGN, ST, false, false>(
      p, [&](const f32x4(&acc)[TN][TM], int m, int n, int lane, uint8_t*) __attribute__((always_inline)) {
        if (n < p.N) store_tile<bf16, EPI, 64, TN, TM, kPaired<TN>>(g, acc, m, n, lane);
      });
}

}  // namespace gemm
}  // namespace wam
