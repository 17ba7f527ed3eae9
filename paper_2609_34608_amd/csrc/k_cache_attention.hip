// Attention over a paged cache of 4-bit blocks (gfx950).
//
// Per key head, the query rows (t, head of the group) of a sequence are tiled by 16 and
// the tokens by 64.  As in k_attention.hip, S^T = K Q^T and O^T = V^T P^T on
// v_mfma_f32_16x16x32_bf16, so a lane's scores all belong to one query and feed the
// second product without leaving the lane.
//
// Codes go from memory straight into registers.  A code times its power of two has two
// significant bits and is exact in bf16, so both products are those of bf16 operands:
//  * K: lane (r, g) holds the dh / 4 values of token r from dh / 4 * g on, whole words of
//    codes, which the conversions turn into the chunks of 8 that the MFMA takes.  Which
//    dims a lane holds does not matter as long as q's chunks are the same.
//  * V: the second product runs over tokens, which lie in different rows of codes.  A
//    wave puts its converted tile (token rows) into LDS and reads it back with
//    ds_read_b64_tr_b16, four tokens of a dim a lane, at the tokens whose scores the
//    lane group holds.
// The softmax has a running maximum m (in units of log2) that moves when a tile passes it
// by more than 8, so most tiles have no rescale; its denominator is one more MFMA
// against ones, which sums exactly the rounded probabilities that multiply V.  Under bf16 q
// they are rounded to bf16, the instruction's type (results are then 0.0023 off the definition,
// 0.0017 by their own rounding alone); float32 q and its probabilities go in three bf16
// parts, at 2.4 times the time.
// A probability's exponent is one multiply-add of score, scale and -m.  m is a rounded
// product, which from 2^22 on is no longer near the exact one that the multiply-add takes (from
// 2^32 on by more than the exponent's range), so from there the scores are scaled and
// rounded first, as m was: the largest is then m.
//
// A block's four waves share the tokens of its rows, taking tiles in turn, and join through
// LDS; where blocks are few, a sequence's tokens are split over blocks too, whose parts go
// to the workspace for a second launch to join in order.  Over few tokens the waves take
// rows of their own.
//
// What bounds it, on one MI355X: single rows the bytes of the cache (16 streams of 16384 to
// 32768 tokens, 8 heads of 128: 91 us, 4.8 TB/s; a 1 GiB copy reaches 5.0); many rows the
// instructions: 10176 rows of 24 heads of 64 over 20352 tokens take 1440 us, 884 TFLOP/s
// (a bf16 product of 8192^3 reaches 1213), the matrix cores 40% busy, at 2.1 GHz, to which
// the power of this mix brings the clock down.  A form for many rows that converts tokens
// once for four waves of 64 rows, with 32x32x16 products between the exponentials and
// without the maximum, has half the matrix instructions and 30% fewer others, and took as
// long (1340 to 1410 us, this one 1416 then; shorter sequences longer), so this one stays.
#include <float.h>
#include <math.h>

#include <algorithm>

#include "cache.h"
#include "fp4.h"
#include "layer_util.h"

namespace wam {

int check_cache(const wam_cache& c, const wam_page_table& t, bool written, bool empty, const char* what);

namespace {

constexpr int kKeys = 64;      // tokens of a tile
constexpr int kWaves = 4;
constexpr float kNone = -FLT_MAX;  // running maximum of a row that has seen nothing
constexpr float kSlack = 8.f;    // a probability reaches 2^8 before the maximum moves
constexpr float kSteep = 0x1p22f;  // a maximum from here on takes rounded scores
constexpr uint32_t kFar = 253;   // scales from here on may pass the bf16 range
constexpr float kLn2 = 0.6931471805599453f;

struct AttendParams {
  wam_cache_attention_args a;
  int shift;       // of a page
  int group;       // query heads of a key head
  int row_blocks;  // blocks of rows of a (sequence, key head)
  int splits;      // blocks that share the tokens of a row block
  int by_rows;     // a block's waves take rows of their own instead of tokens
  float log2_scale;
};

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// Which block of rows, part of the tokens, key head and sequence a workgroup takes.
// Workgroups go to the 8 XCDs round-robin.  Where several blocks read the tokens of a
// (sequence, key head), that pair's blocks go to one XCD, whose L2 they share, and the
// pairs round; the pairs that 8 does not divide go to ranges of blocks.  Otherwise
// neighbours in the grid are the parts of one pair, so that long sequences burden all
// XCDs alike.
struct BlockAt {
  int rb, split, pair;
};
__device__ __forceinline__ BlockAt block_at(int i, int pairs, int row_blocks, int splits) {
  const int each = row_blocks * splits;
  int pair, k;
  if (row_blocks == 1) {
    pair = i / each, k = i % each;
  } else {
    const int x = i % 8, j = i / 8, whole = pairs / 8 * each;
    if (j < whole) {
      pair = j / each * 8 + x, k = j % each;
    } else {
      const int n = pairs % 8 * each, per = n / 8, rem = n % 8;
      const int at = x * per + min(x, rem) + j - whole;
      pair = pairs / 8 * 8 + at / each, k = at % each;
    }
  }
  return {k / splits, k % splits, pair};
}

// bf16 parts of a float32: the first alone, or three that add up to it
template <int NS>
__device__ __forceinline__ void split(float x, bf16 (&part)[NS]) {
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    part[s] = static_cast<bf16>(x);
    x -= static_cast<float>(part[s]);
  }
}

// The same of q, which may lie past the bf16 range: the first part stays finite where q is.
template <int NS>
__device__ __forceinline__ void split_q(float x, bf16 (&part)[NS]) {
  part[0] = static_cast<bf16>(x);
  if constexpr (NS > 1) {
    const bool finite = fabsf(x) < INFINITY;
    if (finite && !(fabsf((float)part[0]) < INFINITY)) part[0] = (bf16)copysignf(0x1.fep127f, x);
    x = finite ? x - (float)part[0] : 0.f;
#pragma unroll
    for (int s = 1; s < NS; ++s) {
      part[s] = static_cast<bf16>(x);
      x -= (float)part[s];
    }
  }
}

typedef __attribute__((address_space(1))) const uint8_t global_byte;

// Codes and scales of 16 tokens: lane (r, g) has the words g DB .. + DB - 1 of token r
template <int DB>
struct Codes {
  uint32_t w[DB];
  uint8_t s[DB];
};

// q, scale: the first of the tokens (uniform); at, sat: the lane's place from there
template <int DB>
__device__ __forceinline__ void load_codes(Codes<DB>& c, const global_byte* q, const global_byte* scale, uint32_t at,
                                           uint32_t sat, int lg) {
  typedef uint32_t words __attribute__((ext_vector_type(DB), aligned(4)));
  typedef __attribute__((address_space(1))) const words global_words;
  if constexpr (DB == 1) {
    c.w[0] = *reinterpret_cast<__attribute__((address_space(1))) const uint32_t*>(q + at);
  } else {
    const words v = *reinterpret_cast<global_words*>(q + at);
#pragma unroll
    for (int i = 0; i < DB; ++i) c.w[i] = v[i];
  }
  if constexpr (DB == 3) {  // a lane's words lie in two blocks
#pragma unroll
    for (int i = 0; i < DB; ++i) c.s[i] = scale[sat + (uint32_t)(lg * DB + i) / 4];
  } else {
    c.s[0] = scale[sat + (uint32_t)(lg * DB) / 4];
  }
}
template <int DB>
__device__ __forceinline__ uint32_t scale_of(const Codes<DB>& c, int i) { return DB == 3 ? c.s[i] : c.s[0]; }

// A probability of zero does not keep a NaN or an infinity of a token that a row does not
// see out of its sums.  As rows see the first tokens, it is enough to know of each dim the first
// token with such a value, for the rows that see it, and to put zeros in their place.  Rare:
// called where a scale may pass the bf16 range.
template <int DB>
__device__ __forceinline__ void drop_far(Codes<DB>& v, int token, int lg, int* first) {
#pragma unroll
  for (int s = 0; s < DB; ++s) {
    const bf16x8 x = fp4_to_bf16(v.w[s], fp4_scale_operand(scale_of(v, s)));
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (!(fabsf((float)x[e]) < INFINITY)) {
        atomicMin(first + (lg * DB + s) * 8 + e, token);
        v.w[s] &= ~(0xfu << (4 * e));
      }
  }
#pragma unroll
  for (int s = 0; s < DB; ++s)
    if (v.s[s] == kFp4NaN) v.s[s] = 0;
}

// A value of a row from its sum and the probabilities' (inv: 1 / total): 0 where the row saw
// nothing, and NaN where a value of v past the bf16 range, an infinity in the product, came in
// without a mask (under one drop_far keeps it out).
__device__ __forceinline__ float value_of(float sum, float total, float inv) {
  return total == 0.f ? 0.f : fmaf(sum, inv, sum * 0.f);  // infinity * 0: NaN
}

// DB: blocks of a head; QT: tiles of 16 rows; NS: bf16 parts of q and of a probability
template <int DB, int QT, int NS>
__global__ __launch_bounds__(kWaves* kWave, 2) void attend_kernel(AttendParams p) {
  typedef typename std::conditional<NS == 1, bf16, float>::type T;
  constexpr int DH = DB * 32, DT = DH / 16;
  constexpr int VROW = DH * 2 + 32;  // bytes of a token in LDS: the reads of 16 rows meet no bank twice
  __shared__ __attribute__((aligned(64))) uint8_t vt[kWaves][kKeys * VROW];
  __shared__ float part_m[kWaves][QT * 16], part_l[kWaves][QT * 16];
  __shared__ int odd[DH];  // token that is the first without a finite value, by dim

  const wam_cache_attention_args& a = p.a;
  const wam_cache& ca = a.cache;
  const int lane = threadIdx.x % kWave, wid = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int lr = lane % 16, lg = lane / 16;
  const BlockAt id = block_at(blockIdx.x, a.B * ca.H, p.row_blocks, p.splits);
  // causal: the rows that see most first (3000 rows of 2 x 8 heads over 4000 tokens 70 -> 55 us)
  const int rb = a.causal ? p.row_blocks - 1 - id.rb : id.rb;
  const int split_at = id.split, hk = id.pair % ca.H, b = id.pair / ca.H;

  const int R = p.group * a.T, r0 = (p.by_rows ? rb * kWaves + wid : rb) * QT * 16;
  const int stride = p.by_rows ? 1 : kWaves;  // from tile to tile
  const int rows = a.rows ? min(max(a.rows[b], 0), a.T) : a.T;
  const int length = a.lengths[b], held = tokens_held(length, a.table.width, p.shift);
  // what the rows of this block see at least and at most (row r is t = r / group, in order)
  // rows past the last are never stored and hinder nothing
  int most = 0, least = INT32_MAX;
  int vis[QT];
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    const int r = r0 + i * 16 + lr;
    vis[i] = r < R ? tokens_seen(held, length, a.causal, rows, r / p.group) : INT32_MAX;
    int hi = r < R ? vis[i] : 0, lo = vis[i];
#pragma unroll
    for (int o = 1; o < 16; o *= 2) hi = max(hi, __shfl_xor(hi, o, 64)), lo = min(lo, __shfl_xor(lo, o, 64));
    most = max(most, hi), least = min(least, lo);
  }
  most = __builtin_amdgcn_readfirstlane(most), least = __builtin_amdgcn_readfirstlane(least);
  const int tiles = (most + kKeys - 1) / kKeys;
  const int t_lo = (int)((int64_t)tiles * split_at / p.splits), t_hi = (int)((int64_t)tiles * (split_at + 1) / p.splits);

  // q, in chunks of the dims that the K operand has
  bf16x8 qf[QT][DB][NS];
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    const int r = min(r0 + i * 16 + lr, R - 1);
    const T* q = static_cast<const T*>(a.q) + b * a.q_stride[0] + r / p.group * a.q_stride[1] +
                 (hk * p.group + r % p.group) * a.q_stride[2];
#pragma unroll
    for (int s = 0; s < DB; ++s) {
      float x[8];
      load_n(x, q + (lg * DB + s) * 8, 8);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        bf16 part[NS];
        split_q<NS>(x[e], part);
#pragma unroll
        for (int n = 0; n < NS; ++n) qf[i][s][n][e] = part[n];
      }
    }
  }

  // Where the groups of 16 tokens of the wave's next 16 tiles lie, one a lane: a table that
  // is read when its pages are needed costs a tile the latency of one more load, and
  // addresses that every tile works out anew cost it 200 scalar instructions.
  const int32_t* table = a.table.entry + b * a.table.stride;
  auto token_of = [&](int tile) { return ((int64_t)tile + lane / 4 * stride) * kKeys + lane % 4 * 16; };
  auto pages_from = [&](int tile) __attribute__((always_inline)) {
    const int64_t t = token_of(tile);
    return t < held ? page_of(table, a.table.width, p.shift, ca.pages, (int)t) : -1;
  };
  const uint8_t *group_k, *group_ks, *group_v, *group_vs;
  uint64_t have = 0;  // lanes whose tokens have a page
  auto place_groups = [&](int tile, int page) __attribute__((always_inline)) {
    have = __ballot(page >= 0);
    const int64_t pg = max(page, 0), place = token_of(tile) & ((1 << p.shift) - 1);
    group_k = ca.k + (pg * ca.k_stride[0] + place * ca.k_stride[1] + hk * ca.k_stride[2]);
    group_ks = ca.k_scale + (pg * ca.k_scale_stride[0] + place * ca.k_scale_stride[1] + hk * ca.k_scale_stride[2]);
    group_v = ca.v + (pg * ca.v_stride[0] + place * ca.v_stride[1] + hk * ca.v_stride[2]);
    group_vs = ca.v_scale + (pg * ca.v_scale_stride[0] + place * ca.v_scale_stride[1] + hk * ca.v_scale_stride[2]);
  };
  const uint32_t at_k = lr * (uint32_t)ca.k_stride[1] + lg * DB * 4, at_v = lr * (uint32_t)ca.v_stride[1] + lg * DB * 4;
  const uint32_t at_ks = lr * (uint32_t)ca.k_scale_stride[1], at_vs = lr * (uint32_t)ca.v_scale_stride[1];
  Codes<DB> kc[4], vc[4];
  uint32_t there = 0;  // bit g: the 16 tokens have a page
  auto request = [&](int turn) __attribute__((always_inline)) {
    auto of = [&](const uint8_t* x, int g) __attribute__((always_inline)) {
      const uint64_t u = reinterpret_cast<uint64_t>(x);
      const uint32_t lo = __builtin_amdgcn_readlane((int)u, turn * 4 + g);
      const uint32_t hi = __builtin_amdgcn_readlane((int)(u >> 32), turn * 4 + g);
      return reinterpret_cast<const global_byte*>((uint64_t)hi << 32 | lo);
    };
    there = (uint32_t)(have >> (turn * 4)) & 15;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      load_codes(kc[g], of(group_k, g), of(group_ks, g), at_k, at_ks, lg);
      load_codes(vc[g], of(group_v, g), of(group_vs, g), at_v, at_vs, lg);
    }
  };

  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  bf16x8 ones;
#pragma unroll
  for (int e = 0; e < 8; ++e) ones[e] = (bf16)1.0f;
  f32x4 o[QT][DT], l[QT];
  float m[QT];
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    m[i] = kNone, l[i] = zero;
#pragma unroll
    for (int j = 0; j < DT; ++j) o[i][j] = zero;
  }
  uint8_t* own = vt[wid];
  // V^T of dims 16 J .. + 15 and the tokens of score tiles 2 C, 2 C + 1; lane s of a group
  // reads dims 4 (s % 4) .. + 3 of token s / 4 of its four
  const uint8_t* from = own + (4 * lg + lr / 4) * VROW + lr % 4 * 8;
  auto values = [&](auto J, auto C) __attribute__((always_inline)) {
    const uint8_t* at = from + 2 * decltype(C)::value * 16 * VROW + decltype(J)::value * 32;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 16 * VROW));
    bf16x8 vf;
    __builtin_memcpy(&vf, &lo, 8);
    __builtin_memcpy(reinterpret_cast<char*>(&vf) + 8, &hi, 8);
    return vf;
  };

  if (a.causal) {
    if (threadIdx.x < DH) odd[threadIdx.x] = INT32_MAX;
    __syncthreads();
  }
  int unit = 0;  // whether scores are scaled before their exponents
  const int first = t_lo + (p.by_rows ? 0 : wid);
  int more = -1, turn = 0;
  if (first < t_hi) {
    place_groups(first, pages_from(first));
    more = pages_from(first + 16 * stride);
    request(0);
  }
  for (int tile = first; tile < t_hi; tile += stride) {
    const int k0 = tile * kKeys;
    const uint32_t has = there;
    const bool whole = k0 + kKeys <= least && has == 15;
    if (!whole) {
      // tokens that the sequence does not hold count as zeros, whatever lies there
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const bool live = (has >> g & 1) && k0 + g * 16 + lr < held;
#pragma unroll
        for (int s = 0; s < DB; ++s)
          if (!live) vc[g].w[s] = 0, vc[g].s[s] = 0;
      }
    }
    if (a.causal) {
      bool far = false;
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int s = 0; s < DB; ++s) far |= scale_of(vc[g], s) >= kFar;
      if (__any(far)) {
#pragma unroll
        for (int g = 0; g < 4; ++g) drop_far(vc[g], k0 + g * 16 + lr, lg, odd);
      }
    }
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
      for (int s = 0; s < DB; ++s)
        *reinterpret_cast<bf16x8*>(own + (g * 16 + lr) * VROW + (lg * DB + s) * 16) =
            fp4_to_bf16(vc[g].w[s], fp4_scale_operand(scale_of(vc[g], s)));
    f32x4 st[QT][4];
    auto scores = [&](auto FAR) __attribute__((always_inline)) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
#pragma unroll
        for (int i = 0; i < QT; ++i) st[i][g] = zero;
#pragma unroll
        for (int s = 0; s < DB; ++s) {
          const bf16x8 kf = fp4_to_bf16(kc[g].w[s], fp4_scale_operand(scale_of(kc[g], s)));
          bf16x8 rest = kf;  // for the later parts of q
          if constexpr (decltype(FAR)::value) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (!(fabsf((float)rest[e]) < INFINITY)) rest[e] = (bf16)0.f;
          }
#pragma unroll
          for (int i = 0; i < QT; ++i)
#pragma unroll
            for (int n = 0; n < NS; ++n)
              st[i][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(n ? rest : kf, qf[i][s][n], st[i][g], 0, 0, 0);
        }
      }
    };
    scores(std::false_type{});
    if constexpr (NS > 1) {
      // a key past the bf16 range, an infinity, meets the first part of q alone: the others may be
      // zero, and add nothing to an infinite score
      uint32_t far = 0;
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int s = 0; s < DB; ++s) far = max(far, scale_of(kc[g], s));
      if (__any(far >= kFar)) scores(std::true_type{});
    }
    if (tile + stride < t_hi) {
      if (++turn == 16) {
        turn = 0;
        place_groups(tile + stride, more);
        more = pages_from(tile + 17 * stride);
      }
      request(turn);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();

    if (!whole) {
#pragma unroll
      for (int i = 0; i < QT; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (!((has >> g & 1) && k0 + g * 16 + 4 * lg + r < vis[i])) st[i][g][r] = -INFINITY;
    }
    float top[QT];
    bool grown = false;
#pragma unroll
    for (int i = 0; i < QT; ++i) {
      top[i] = st[i][0][0];
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int r = 0; r < 4; ++r) top[i] = fmaxf(top[i], st[i][g][r]);
      top[i] *= p.log2_scale;
      grown |= top[i] > m[i] + kSlack;
    }
    if (__any(grown)) {
      bool steep = false;
#pragma unroll
      for (int i = 0; i < QT; ++i) {
        top[i] = fmaxf(top[i], __shfl_xor(top[i], 16, 64));
        top[i] = fmaxf(top[i], __shfl_xor(top[i], 32, 64));
        const float to = top[i] > m[i] + kSlack ? top[i] : m[i], f = __builtin_amdgcn_exp2f(m[i] - to);
        m[i] = to;
        l[i] *= f;
#pragma unroll
        for (int j = 0; j < DT; ++j) o[i][j] *= f;
        steep |= fabsf(to) >= kSteep && to != kNone;
      }
      unit |= __builtin_amdgcn_readfirstlane(__any(steep));
    }
    const float mul = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(unit ? 1.f : p.log2_scale)));
    if (unit) {
#pragma unroll
      for (int i = 0; i < QT; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) st[i][g] *= p.log2_scale;
    }
    // Half of the tile's tokens at a time, so that V^T of that half stays in registers for
    // all row tiles; the exponentials of the next row tile run between the matrix
    // instructions of this one.
    bf16x8 pf[2][NS], vf[DT];
    auto exponentials = [&](auto N) __attribute__((always_inline)) {
      constexpr int c = decltype(N)::value / QT, i = decltype(N)::value % QT;
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          bf16 part[NS];
          split<NS>(__builtin_amdgcn_exp2f(fmaf(st[i][2 * c + g][r], mul, -m[i])), part);
#pragma unroll
          for (int n = 0; n < NS; ++n) pf[decltype(N)::value & 1][n][g * 4 + r] = part[n];
        }
    };
    exponentials(std::integral_constant<int, 0>{});
    static_for<2 * QT>([&](auto N) __attribute__((always_inline)) {
      constexpr int n = decltype(N)::value, c = n / QT, i = n % QT;
      if constexpr (i == 0)
        static_for<DT>([&](auto J) __attribute__((always_inline)) { vf[decltype(J)::value] = values(J, std::integral_constant<int, c>{}); });
      if constexpr (n + 1 < 2 * QT) exponentials(std::integral_constant<int, n + 1>{});
#pragma unroll
      for (int k = 0; k < NS; ++k) {
        l[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[n & 1][k], l[i], 0, 0, 0);
#pragma unroll
        for (int j = 0; j < DT; ++j)
          o[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[j], pf[n & 1][k], o[i][j], 0, 0, 0);
      }
      if constexpr (NS == 1 && n + 1 < 2 * QT) {
#pragma unroll
        for (int k = 0; k <= DT; ++k) {
          __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);              // one MFMA
          __builtin_amdgcn_sched_group_barrier(0x2, 20 / (DT + 1), 0);  // and its share of the VALU
        }
      }
    });
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }

  if (p.by_rows) {
#pragma unroll
    for (int i = 0; i < QT; ++i) {
      const int r = r0 + i * 16 + lr, t = r / p.group, h = hk * p.group + r % p.group;
      if (r >= R) continue;
      const float total = l[i][0], inv = 1.0f / total;
      const int sees = a.causal ? tokens_seen(held, length, true, rows, t) : 0;
      T* out = static_cast<T*>(a.out) + b * a.out_stride[0] + t * a.out_stride[1] + h * a.out_stride[2];
#pragma unroll
      for (int j = 0; j < DT; ++j) {
        const int d = j * 16 + 4 * lg;
        Pack<T, 4> w;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float x = sees > odd[d + k] && a.causal ? NAN : o[i][j][k];
          w.v[k] = static_cast<T>(value_of(x, total, inv));
        }
        *reinterpret_cast<Pack<T, 4>*>(out + d) = w;
      }
      if (a.lse && lg == 0)
        a.lse[b * a.lse_stride[0] + t * a.lse_stride[1] + h * a.lse_stride[2]] =
            total == 0.f ? -INFINITY : (m[i] + __builtin_amdgcn_logf(total)) * kLn2;
    }
    return;
  }
  // The waves' parts join in LDS, in the order of the waves: maximum, then the sums at
  // that maximum.
#pragma unroll
  for (int i = 0; i < QT; ++i)
    if (lg == 0) part_m[wid][i * 16 + lr] = m[i];
  __syncthreads();
  float f[QT];
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    float to = part_m[0][i * 16 + lr];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) to = fmaxf(to, part_m[w][i * 16 + lr]);
    f[i] = __builtin_amdgcn_exp2f(m[i] - to);
    m[i] = to;
    if (lg == 0) part_l[wid][i * 16 + lr] = l[i][0] * f[i];
  }
  // a slice of the dims at a time, so that the waves' slices fit where V was
  constexpr int kRow = DT * 16 + 4;  // floats of a row, apart from the banks of the next
  static_assert(16 * kRow * 4 <= kKeys * VROW, "a tile of rows fits a wave's V");
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    float* mine = reinterpret_cast<float*>(vt[wid]);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < DT; ++j)
      *reinterpret_cast<f32x4*>(mine + lr * kRow + j * 16 + 4 * lg) = o[i][j] * f[i];
    __syncthreads();
    for (int e = threadIdx.x; e < 16 * DH / 4; e += kWaves * kWave) {
      const int row = e / (DH / 4), d = e % (DH / 4) * 4, r = r0 + i * 16 + row;
      f32x4 sum = zero;
      float total = 0.f, top = kNone;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        sum += *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(vt[w]) + row * kRow + d);
        total += part_l[w][i * 16 + row];
        top = fmaxf(top, part_m[w][i * 16 + row]);
      }
      if (r >= R) continue;
      if (a.causal) {
        const int sees = tokens_seen(held, length, true, rows, r / p.group);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (sees > odd[d + k]) sum[k] = NAN;
      }
      if (p.splits > 1) {
        const int64_t at = (((int64_t)b * ca.H + hk) * p.splits + split_at) * R + r;
        float* ws = static_cast<float*>(a.workspace);
        *reinterpret_cast<f32x4*>(ws + at * DH + d) = sum;
        if (d == 0) {
          float* ml = ws + (int64_t)a.B * ca.H * p.splits * R * DH + at * 2;
          ml[0] = top, ml[1] = total;
        }
        continue;
      }
      const int t = r / p.group, h = hk * p.group + r % p.group;
      const float inv = 1.0f / total;
      T* out = static_cast<T*>(a.out) + b * a.out_stride[0] + t * a.out_stride[1] + h * a.out_stride[2];
      Pack<T, 4> w;
#pragma unroll
      for (int k = 0; k < 4; ++k) w.v[k] = static_cast<T>(value_of(sum[k], total, inv));
      *reinterpret_cast<Pack<T, 4>*>(out + d) = w;
      if (a.lse && d == 0)
        a.lse[b * a.lse_stride[0] + t * a.lse_stride[1] + h * a.lse_stride[2]] =
            total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * kLn2;
    }
  }
}

// Joins the parts of a row, W waves a row: a lane takes four values of dh in every G-th part
// of its wave's, so that the loads of several parts go out together, and the sums of a
// value add up in a fixed order.  Bound by latency (1536 rows of 64 values in 21 parts 7.3 us
// with a wave a row, 5.6 with four; 64 rows in 192 parts 9.5 with four, 38 -> 23 the call).
template <typename T, int W>
__global__ __launch_bounds__(256) void join_kernel(AttendParams p) {
  __shared__ float shared[W][kWave * 5];
  const wam_cache_attention_args& a = p.a;
  const int R = p.group * a.T, DH = a.cache.dh, lane = threadIdx.x % kWave, wid = threadIdx.x / kWave % W;
  const int64_t i = (int64_t)blockIdx.x * (4 / W) + threadIdx.x / (kWave * W);  // (b, hk, r)
  if (i >= (int64_t)a.B * a.cache.H * R) return;                               // (W = 4: all of the block's or none)
  const int64_t bh = i / R;
  const int r = (int)(i % R), b = (int)(bh / a.cache.H), hk = (int)(bh % a.cache.H);
  const float* ws = static_cast<const float*>(a.workspace) + (bh * p.splits * R + r) * DH;
  const float* ml = static_cast<const float*>(a.workspace) + (int64_t)a.B * a.cache.H * p.splits * R * DH +
                    (bh * p.splits * R + r) * 2;
  float top = kNone;
  for (int s = lane; s < p.splits; s += kWave) top = fmaxf(top, ml[(int64_t)s * R * 2]);
#pragma unroll
  for (int o = 1; o < kWave; o *= 2) top = fmaxf(top, __shfl_xor(top, o, 64));
  const int lanes = DH <= 64 ? DH / 4 <= 8 ? 8 : 16 : 32;  // of a row's values, a power of two
  const int at = lane % lanes, G = kWave / lanes;
  const bool mine = 4 * at < DH;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  float total = 0.f;
#pragma unroll 8
  for (int s = wid * G + lane / lanes; s < p.splits; s += W * G) {
    const int64_t row = (int64_t)s * R;
    const float f = __builtin_amdgcn_exp2f(ml[row * 2] - top);
    total += ml[row * 2 + 1] * f;
    if (mine) x += *reinterpret_cast<const f32x4*>(ws + row * DH + 4 * at) * f;
  }
  for (int o = lanes; o < kWave; o *= 2) {
    total += __shfl_xor(total, o, 64);
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] += __shfl_xor(x[k], o, 64);
  }
  if constexpr (W > 1) {
    shared[wid][lane] = total;
#pragma unroll
    for (int k = 0; k < 4; ++k) shared[wid][(k + 1) * kWave + lane] = x[k];
    __syncthreads();
    if (wid) return;
#pragma unroll
    for (int w = 1; w < W; ++w) {
      total += shared[w][lane];
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] += shared[w][(k + 1) * kWave + lane];
    }
  }
  if (lane >= lanes) return;
  const int t = r / p.group, h = hk * p.group + r % p.group;
  const float inv = 1.0f / total;
  T* out = static_cast<T*>(a.out) + b * a.out_stride[0] + t * a.out_stride[1] + h * a.out_stride[2];
  Pack<T, 4> w;
#pragma unroll
  for (int k = 0; k < 4; ++k) w.v[k] = static_cast<T>(value_of(x[k], total, inv));
  if (mine) *reinterpret_cast<Pack<T, 4>*>(out + 4 * at) = w;
  if (a.lse && lane == 0)
    a.lse[b * a.lse_stride[0] + t * a.lse_stride[1] + h * a.lse_stride[2]] =
        total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * kLn2;
}

// Tiles of 16 rows a wave takes, whether the waves of a block share tokens or rows, and over
// how many blocks a sequence's tokens go.
constexpr int kShort = 32;      // tiles of a sequence
constexpr int kPartTiles = 24;  // what a block costs beside its tiles, in tiles
constexpr int kJoinTiles = 24;  // and the launch that joins parts
struct AttendPlan {
  int qt, row_blocks, splits;
  bool by_rows;
};
AttendPlan plan_attend(const wam_cache_attention_args& a) {
  AttendPlan pl;
  const int64_t R = (int64_t)(a.Hq / a.cache.H) * a.T, pairs = (int64_t)a.B * a.cache.H;
  const int64_t tiles = ((int64_t)a.table.width * a.cache.page + kKeys - 1) / kKeys;
  const bool narrow = a.cache.dh <= 64;
  // As many rows as registers hold: a tile's conversions serve all of them.  In float32 that
  // takes many blocks of long sequences (2 x 16 rows against 16: 10176 rows of 24 heads over
  // as many tokens 2022 -> 1768 us, 4 x 864 of 12 over 864 47 -> 52).
  int most = narrow ? 4 : 2;
  if (a.dtype == WAM_FP32) most = narrow && tiles > kShort && pairs * ((R + 15) / 16) >= 4096 ? 2 : 1;
  pl.qt = 1;
  while (pl.qt < most && pl.qt * 16 < R) pl.qt *= 2;
  pl.row_blocks = (int)((R + pl.qt * 16 - 1) / (pl.qt * 16));
  const int64_t blocks = pairs * pl.row_blocks;
  // Blocks counted as a round: what 256 CUs hold at once, by registers and LDS, of most forms
  // (two a CU, three of 16 rows of 64).  Heads of 32 hold others: five of 16 bf16 rows and three
  // of 16 float32 rows a CU, where four are counted, and three of 32 bf16 rows, where two are.
  const int64_t slots = pl.qt == 1 && narrow ? a.cache.dh == 32 ? 1024 : 768 : 512;
  // Few tiles leave waves that share them without work, or with less of it than joining
  // costs (9 x 4924 rows of 9 heads over 60 tokens 143 -> 44 us, 8 x 1000 of 16 over 700
  // 53 -> 37, 8 x 4000 of 24 over 4000 940 -> 845); rows of their own take more blocks to
  // fill the chip, and many of them where the rounds are long (10176 rows of 24 heads over
  // as many tokens, 3816 blocks that share tokens: 742 -> 772).
  pl.by_rows = pl.row_blocks > 1 && (tiles <= kWaves || blocks >= (tiles <= kShort ? 2048 : 8192));
  pl.splits = 1;
  if (pl.by_rows) {
    pl.row_blocks = (pl.row_blocks + kWaves - 1) / kWaves;
  } else if (blocks < 4 * slots) {
    // As many parts as fill one round of blocks or two, whichever ends first, each wave with
    // two tiles at least (64 rows of 24 heads over 101760 tokens in 1032 blocks, three
    // rounds: 88 us; in 504, one: 71).
    auto cost = [&](int64_t parts) {
      return (double)((blocks * parts + slots - 1) / slots) * ((double)tiles / (double)parts + kPartTiles) +
             (parts > 1 ? kJoinTiles : 0);
    };
    for (int rounds = 1; rounds <= 2; ++rounds) {
      const int64_t parts = std::min(tiles / (2 * kWaves), rounds * slots / blocks);
      if (parts > 1 && cost(parts) < cost(pl.splits)) pl.splits = (int)parts;
    }
  }
  return pl;
}

size_t workspace_of(const wam_cache_attention_args& a, const AttendPlan& pl) {
  if (pl.splits == 1) return 0;
  const size_t rows = (size_t)a.B * a.Hq * a.T * pl.splits;
  return rows * (a.cache.dh + 2) * sizeof(float);
}

template <int DB, int NS>
hipError_t launch_blocks_of(const AttendParams& p, const AttendPlan& pl, dim3 grid, hipStream_t s) {
  if (pl.qt == 1) launch_k(attend_kernel<DB, 1, NS>, grid, kWaves * kWave, 0, s, p);
  else if constexpr (NS == 1 || DB <= 2) {
    if (pl.qt == 2) launch_k(attend_kernel<DB, 2, NS>, grid, kWaves * kWave, 0, s, p);
    else if constexpr (NS == 1 && DB <= 2) launch_k(attend_kernel<DB, 4, NS>, grid, kWaves * kWave, 0, s, p);
  }
  return hipGetLastError();
}
template <int NS>
hipError_t launch_attend(const AttendParams& p, const AttendPlan& pl, hipStream_t s) {
  const int64_t blocks = (int64_t)p.a.B * p.a.cache.H * pl.row_blocks * pl.splits;
  if (blocks * kWaves * kWave > 0xffffffffll) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)blocks);
  hipError_t e;
  switch (p.a.cache.dh) {
    case 32: e = launch_blocks_of<1, NS>(p, pl, grid, s); break;
    case 64: e = launch_blocks_of<2, NS>(p, pl, grid, s); break;
    case 96: e = launch_blocks_of<3, NS>(p, pl, grid, s); break;
    default: e = launch_blocks_of<4, NS>(p, pl, grid, s); break;
  }
  if (e != hipSuccess || pl.splits == 1) return e;
  typedef typename std::conditional<NS == 1, bf16, float>::type T;
  const int64_t rows = (int64_t)p.a.B * p.a.Hq * p.a.T;
  // a wave a row, four where a row has many parts
  if (pl.splits > 16) launch_k(join_kernel<T, 4>, dim3((unsigned)rows), 256, 0, s, p);
  else launch_k(join_kernel<T, 1>, dim3((unsigned)((rows + 3) / 4)), 256, 0, s, p);
  return hipGetLastError();
}

int check_attention(const wam_cache_attention_args* a) {
  if (!a) return noalloc_fail(WAM_E_ARG, "wam_cache_attention: null argument");
  if (a->B < 0 || a->T < 0) return noalloc_fail(WAM_E_ARG, "wam_cache_attention: sizes must be >= 0");
  if (!float_type(a->dtype)) return noalloc_fail(WAM_E_ARG, "wam_cache_attention: q must be WAM_FP32 or WAM_BF16");
  const int st = check_cache(a->cache, a->table, false, a->B == 0 || a->T == 0, "wam_cache_attention");
  if (st) return st;
  if (a->Hq < 1 || a->Hq % a->cache.H)
    return noalloc_fail(WAM_E_SHAPE, "wam_cache_attention: Hq must be a multiple of the cache's heads");
  if (!(a->scale > 0.0) || !(a->scale < 1e30)) return noalloc_fail(WAM_E_ARG, "wam_cache_attention: scale must be > 0");
  if ((int64_t)a->B * a->T > WAM_MAX_ROWS || (int64_t)a->B * a->T * a->Hq > INT32_MAX - 65536)
    return noalloc_fail(WAM_E_SHAPE, "wam_cache_attention: too many rows");
  return WAM_OK;
}

}  // namespace

}  // namespace wam

using namespace wam;

extern "C" {

size_t wam_cache_attention_workspace(const wam_cache_attention_args* a) {
  if (check_attention(a) || a->B == 0 || a->T == 0) return 0;
  return workspace_of(*a, plan_attend(*a));
}

int wam_cache_attention(const wam_cache_attention_args* a, void* hip_stream) {
  const int st = check_attention(a);
  if (st) return st;
  if (a->B == 0 || a->T == 0) return WAM_OK;
  if (!a->q || !a->out || !a->lengths) return noalloc_fail(WAM_E_ARG, "wam_cache_attention: null q, out or lengths");
  const int64_t unit = type_size(a->dtype), size[3] = {a->B, a->T, a->Hq};
  if (!aligned_to(a->q, unit) || !aligned_to(a->out, unit) || !aligned_to(a->lse, 4) || !aligned_to(a->lengths, 4) ||
      !aligned_to(a->rows, 4))
    return noalloc_fail(WAM_E_ARG, "wam_cache_attention: buffers must be aligned to their elements");
  if (!strides_ok(a->q_stride, 3)) return noalloc_fail(WAM_E_ARG, "wam_cache_attention: strides must be >= 0");
  if (!strides_ok(a->out_stride, 3) || !distinct(a->out_stride, size, 3, a->cache.dh) ||
      (a->lse && (!strides_ok(a->lse_stride, 3) || !distinct(a->lse_stride, size, 3, 1))))
    return noalloc_fail(WAM_E_ARG, "wam_cache_attention: the elements of a result must be distinct");
  if (a->q == a->out) return noalloc_fail(WAM_E_ARG, "wam_cache_attention: out must not be q");
  const void* lse = a->lse;
  if (lse && (lse == a->q || lse == a->out))
    return noalloc_fail(WAM_E_ARG, "wam_cache_attention: lse must be a buffer of its own");
  const AttendPlan pl = plan_attend(*a);
  if (const size_t need = workspace_of(*a, pl)) {
    if (!a->workspace || !aligned_to(a->workspace, 16) || a->workspace_bytes < need)
      return noalloc_fail(WAM_E_WORKSPACE, "wam_cache_attention: workspace too small or not on 16 bytes");
  }
  AttendParams p;
  p.a = *a;
  if (a->cache.pages == 0) p.a.table.width = 0;  // no token has a page
  p.shift = 0;
  while ((1 << p.shift) < a->cache.page) ++p.shift;
  p.group = a->Hq / a->cache.H;
  p.row_blocks = pl.row_blocks;
  p.splits = pl.splits;
  p.by_rows = pl.by_rows;
  // not zero: the -infinity of a token that a row does not see has to stay one
  p.log2_scale = std::max((float)(a->scale * 1.4426950408889634), FLT_TRUE_MIN);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const hipError_t e = a->dtype == WAM_BF16 ? launch_attend<1>(p, pl, s) : launch_attend<3>(p, pl, s);
  if (e == hipErrorInvalidConfiguration) return noalloc_fail(WAM_E_SHAPE, "wam_cache_attention: too many blocks for one launch");
  if (e != hipSuccess) return noalloc_fail(WAM_E_HIP, "wam_cache_attention: kernel launch failed");
  return WAM_OK;
}

}  // extern "C"
