// Layer operators behind the handle-free entry points of wam.h (gfx950): rotary
// positions over several axes, the norms around a block with its gate and
// residual, and the quantisation into e4m3 blocks.  All are bound by memory:
// each reads its inputs once and writes its results once.
#include <math.h>

#include <algorithm>

#include "fp8.h"
#include "wam_internal.h"

namespace wam {

namespace {

// ------------------------------------------------------------- elements
// Element i of a row of float32 or bf16 values (type uniform over the launch).
__device__ __forceinline__ float load1(const void* p, int64_t i, int dtype) {
  return dtype == WAM_BF16 ? to_f32(static_cast<const bf16*>(p)[i]) : static_cast<const float*>(p)[i];
}
__device__ __forceinline__ void store1(void* p, int64_t i, int dtype, float v) {
  if (dtype == WAM_BF16) static_cast<bf16*>(p)[i] = static_cast<bf16>(v);
  else static_cast<float*>(p)[i] = v;
}

// N consecutive elements at p, which needs only the alignment of an element:
// global memory takes wide loads and stores at any address.  Elements from n on
// are zero (not loaded) or left alone (not stored).
template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Pack {
  T v[N];
};
template <int N, typename T>
__device__ __forceinline__ void load_n(float (&x)[N], const T* p, int n) {
  if (n >= N) {
    const Pack<T, N> w = *reinterpret_cast<const Pack<T, N>*>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = to_f32(w.v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = i < n ? to_f32(p[i]) : 0.f;
  }
}

template <int N, typename T>
__device__ __forceinline__ void store_n(T* p, const float (&x)[N], int n, bool stream) {
  Pack<T, N> w;
#pragma unroll
  for (int i = 0; i < N; ++i) w.v[i] = static_cast<T>(x[i]);
  if (n >= N) {
    put(p, w, stream);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) p[i] = w.v[i];
  }
}

// ------------------------------------------------------------- rotary positions
constexpr int kMaxPairs = WAM_MAX_HEAD / 2;
// P: room for that many pairs.  Arguments travel with every launch, so heads of up to
// 32 pairs have a form of their own (a call on one row 8.3 -> 7.9 us).
constexpr int kFewPairs = 32;
template <int P>
struct RopeParams {
  wam_rope_args a;
  int pairs, end0, end1;     // pairs of axis 0 end at end0, of axis 1 at end1
  const int* skip;
  double turns[P];           // revolutions per unit of position
};

// cos and sin of pos * freq.  The product is taken in revolutions and in
// float64, so that dropping the whole ones is exact and far positions lose
// nothing (a float32 angle of position 1e5 is off by 4e-3); what is left lies
// within half a turn and float32 does for it.
template <int P>
__device__ __forceinline__ void axis_turn(const RopeParams<P>& p, const float* pos, int i, float& c, float& s) {
  const int axis = i < p.end0 ? 0 : i < p.end1 ? 1 : 2;
  double t = (double)pos[axis] * p.turns[i];
  t -= rint(t);
  sincospif((float)(2.0 * t), &s, &c);
}

// Sum over aligned groups of n lanes (a power of two up to 16), in every lane.
__device__ __forceinline__ float lanes_sum(float v, int n) {
  auto add = [&](auto CTRL) __attribute__((always_inline)) {
    v += __uint_as_float(dpp<decltype(CTRL)::value>(__float_as_uint(v)));
  };
  if (n >= 2) add(std::integral_constant<int, 0xb1>{});
  if (n >= 4) add(std::integral_constant<int, 0x4e>{});
  if (n >= 8) add(std::integral_constant<int, 0x141>{});
  if (n >= 16) add(std::integral_constant<int, 0x140>{});
  return v;
}

// Which rows and heads a block and its waves take (rope_units_kernel).
struct RopeTiling {
  int lanes;        // lanes per head vector, a power of two >= dh / 16
  int heads_wave;   // head vectors of one row side by side in a wave
  int wave_rows;    // waves side by side along the rows (the others along the heads)
  int heads_block;  // heads of a block
  int stream;       // streaming stores
};
constexpr int kRopeTable = 1024;  // most (row, pair) angles of a block

// Head vectors of whole units of 16 elements: eight pairs, or 16 elements past the
// rotated ones.  A lane takes one unit with two 8-element loads (the two halves
// of the pairs, or 16 neighbours), so that a pair never leaves its lane and only
// the norm needs the other lanes of its vector.  The block's angles are computed
// once, in LDS, while the first loads are in flight, and a lane keeps those of
// its unit in registers for all the heads it visits.  Results go out through LDS,
// where a wave keeps its vectors side by side, so that 16 bytes a lane make whole
// lines.  10176 rows of 24 + 24 heads take 21-22 us in either layout, with any
// number of pairs, and as 48 + 48 heads of 32 (125 MB, 5.8 TB/s); streamed as a lane
// holds them, lines in pieces, 26 to 36, and 5088 rows of neighbours in float32 78.
template <typename T, bool PAIRS, bool NORM, int P>
__global__ __launch_bounds__(256) void rope_units_kernel(RopeParams<P> p, RopeTiling tl) {
  constexpr int kPieces = sizeof(T);  // 16-byte pieces of a lane
  __shared__ float2 turn[kRopeTable];
  __shared__ __attribute__((aligned(16))) uint8_t stage[4][kWave * kPieces * 16];
  if (p.skip && *p.skip) return;
  const wam_rope_args& a = p.a;
  const bool isq = blockIdx.z == 0 && a.Hq > 0;
  const int H = isq ? a.Hq : a.Hk;
  const int64_t* si = isq ? a.q_stride : a.k_stride;
  const int64_t* so = isq ? a.q_out_stride : a.k_out_stride;
  const int h_end = min(((int)blockIdx.y + 1) * tl.heads_block, H);

  const int lane = threadIdx.x % kWave, wid = threadIdx.x / kWave;
  const int unit = lane % tl.lanes, slot = lane / tl.lanes;
  const int rows_wave = kWave / tl.lanes / tl.heads_wave;
  const int row_in_block = (wid % tl.wave_rows) * rows_wave + slot / tl.heads_wave;
  const int rows_block = rows_wave * tl.wave_rows;
  const int head_step = tl.heads_wave * (4 / tl.wave_rows);
  int h = (int)blockIdx.y * tl.heads_block + (wid / tl.wave_rows) * tl.heads_wave + slot % tl.heads_wave;

  const uint32_t Tn = a.T, rows = a.B * Tn, row0 = blockIdx.x * (uint32_t)rows_block;  // rows < 2^24
  const uint32_t row = row0 + row_in_block, b = row / Tn, t = row % Tn;
  const bool live = row < rows && 16 * unit < a.dh;
  const int turned = p.pairs / 8;  // units that turn
  const int e1 = PAIRS || unit >= turned ? 16 * unit : 8 * unit;
  const int e2 = PAIRS || unit >= turned ? e1 + 8 : e1 + p.pairs;
  const T* x = static_cast<const T*>(isq ? a.q : a.k) + (live ? b * si[0] + t * si[1] : 0);

  // where the wave's vectors, one after the other in LDS, go in pieces of 16 bytes
  const uint32_t vec = a.dh * (uint32_t)sizeof(T);
  uint8_t* own = stage[wid] + slot * vec;
  uint8_t* to[kPieces];
  int to_head[kPieces];
#pragma unroll
  for (int k = 0; k < kPieces; ++k) {
    const uint32_t at = (k * kWave + lane) * 16, s = at / vec;
    const uint32_t r = row0 + (wid % tl.wave_rows) * rows_wave + s / tl.heads_wave;
    const int head = h + (int)(s % tl.heads_wave) - slot % tl.heads_wave;
    const bool some = s < (uint32_t)(kWave / tl.lanes) && r < rows;
    to_head[k] = some ? head : H;
    to[k] = static_cast<uint8_t*>(isq ? a.q_out : a.k_out) + at % vec +
            (some ? (r / Tn * so[0] + r % Tn * so[1] + head * so[2]) * (int64_t)sizeof(T) : 0);
  }

  Pack<T, 8> x1{}, x2{};  // as loaded: converted only when their turn comes
  auto load = [&](int hh) __attribute__((always_inline)) {
    if (live && hh < h_end) {
      x1 = *reinterpret_cast<const Pack<T, 8>*>(x + hh * si[2] + e1);
      x2 = *reinterpret_cast<const Pack<T, 8>*>(x + hh * si[2] + e2);
    }
  };
  load(h);
  for (uint32_t i = threadIdx.x; i < (uint32_t)(rows_block * p.pairs); i += 256) {
    const uint32_t r = i / (uint32_t)p.pairs;
    const uint32_t rr = min(row0 + r, rows - 1);
    const float* pos = a.pos + rr / Tn * a.pos_stride + rr % Tn * 3;
    float c, s;
    axis_turn(p, pos, (int)(i % (uint32_t)p.pairs), c, s);
    turn[i] = make_float2(c, s);
  }
  float g1[8], g2[8];
  if constexpr (NORM) {
    const float* gain = isq ? a.q_gain : a.k_gain;
    if (live && gain) {
      load_n(g1, gain + e1, 8);
      load_n(g2, gain + e2, 8);
    }
  }
  __syncthreads();
  float c[8], s[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float2 cs = unit < turned ? turn[row_in_block * p.pairs + 8 * unit + j] : make_float2(1.f, 0.f);
    c[j] = cs.x, s[j] = cs.y;
  }
  const bool normed = NORM && (isq ? a.q_gain : a.k_gain);
  for (int h0 = 0; h0 < tl.heads_block; h0 += head_step, h += head_step) {
    float y1[8], y2[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) y1[j] = to_f32(x1.v[j]), y2[j] = to_f32(x2.v[j]);
    load(h + head_step);  // the next head's while this one is turned
    if constexpr (NORM) {
      if (normed) {
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) ss += y1[j] * y1[j] + y2[j] * y2[j];
        const float rs = rsqrt_newton(lanes_sum(live && h < h_end ? ss : 0.f, tl.lanes) / (float)a.dh + a.eps);
#pragma unroll
        for (int j = 0; j < 8; ++j) y1[j] *= rs * g1[j], y2[j] *= rs * g2[j];
      }
    }
    Pack<T, 8> o1, o2;
    if (unit < turned) {
      if constexpr (PAIRS) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          o1.v[2 * j] = static_cast<T>(y1[2 * j] * c[j] - y1[2 * j + 1] * s[j]);
          o1.v[2 * j + 1] = static_cast<T>(y1[2 * j] * s[j] + y1[2 * j + 1] * c[j]);
          o2.v[2 * j] = static_cast<T>(y2[2 * j] * c[4 + j] - y2[2 * j + 1] * s[4 + j]);
          o2.v[2 * j + 1] = static_cast<T>(y2[2 * j] * s[4 + j] + y2[2 * j + 1] * c[4 + j]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          o1.v[j] = static_cast<T>(y1[j] * c[j] - y2[j] * s[j]);
          o2.v[j] = static_cast<T>(y1[j] * s[j] + y2[j] * c[j]);
        }
      }
    } else {  // past the pairs: not by 1 and 0, which would spread a NaN or an infinity
#pragma unroll
      for (int j = 0; j < 8; ++j) o1.v[j] = static_cast<T>(y1[j]), o2.v[j] = static_cast<T>(y2[j]);
    }
    if (16 * unit < a.dh) {
      __builtin_memcpy(__builtin_assume_aligned(own + e1 * sizeof(T), 16), &o1, sizeof(o1));
      __builtin_memcpy(__builtin_assume_aligned(own + e2 * sizeof(T), 16), &o2, sizeof(o2));
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      typedef uint32_t words __attribute__((ext_vector_type(4)));
      const words v = *reinterpret_cast<const words*>(stage[wid] + (k * kWave + lane) * 16);
      if (to_head[k] < h_end) put(to[k], v, tl.stream);
      to_head[k] += head_step;
      to[k] += head_step * so[2] * (int64_t)sizeof(T);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// Any other head size or sections: one wave per head vector, element e = lane +
// 64 j; blocks of four vectors, each taking several where a grid ends.
template <int P>
__global__ __launch_bounds__(256) void rope_kernel(RopeParams<P> p) {
  if (p.skip && *p.skip) return;
  const wam_rope_args& a = p.a;
  const int heads = a.Hq + a.Hk;
  const int64_t items = (int64_t)a.B * a.T * heads;
  const int lane = threadIdx.x % kWave;
  for (int64_t item = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave; item < items; item += (int64_t)gridDim.x * 4) {
    const int hd = (int)(item % heads);
    const int64_t row = item / heads;
    const int t = (int)(row % a.T), b = (int)(row / a.T);
    const bool isq = hd < a.Hq;
    const int h = isq ? hd : hd - a.Hq;
    const int64_t* si = isq ? a.q_stride : a.k_stride;
    const int64_t* so = isq ? a.q_out_stride : a.k_out_stride;
    const int64_t in = b * si[0] + t * si[1] + h * si[2], out = b * so[0] + t * so[1] + h * so[2];
    const void* x = isq ? a.q : a.k;
    void* o = isq ? a.q_out : a.k_out;
    const float* gain = isq ? a.q_gain : a.k_gain;
    const float* pos = a.pos + b * a.pos_stride + (int64_t)t * 3;

    constexpr int J = WAM_MAX_HEAD / kWave;
    float own[J], other[J];
    float ss = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int e = lane + kWave * j;
      own[j] = other[j] = 0.f;
      if (e >= a.dh) continue;
      own[j] = load1(x, in + e, a.dtype);
      ss += own[j] * own[j];
      if (e < 2 * p.pairs) {
        const int partner = a.layout == WAM_ROPE_PAIRS ? e ^ 1 : e < p.pairs ? e + p.pairs : e - p.pairs;
        other[j] = load1(x, in + partner, a.dtype);
        if (gain) other[j] *= gain[partner];
      }
      if (gain) own[j] *= gain[e];
    }
    __builtin_amdgcn_wave_barrier();  // in place: every lane has read its partner before any lane stores
    const float rs = gain ? rsqrt_newton(wave_sum(ss) / (float)a.dh + a.eps) : 1.0f;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int e = lane + kWave * j;
      if (e >= a.dh) continue;
      float v = own[j] * rs;
      if (e < 2 * p.pairs) {
        const bool first = a.layout == WAM_ROPE_PAIRS ? e % 2 == 0 : e < p.pairs;
        const int i = a.layout == WAM_ROPE_PAIRS ? e / 2 : first ? e : e - p.pairs;
        float c, s;
        axis_turn(p, pos, i, c, s);
        v = v * c + other[j] * rs * (first ? -s : s);
      }
      store1(o, out + e, a.dtype, v);
    }
  }
}

// ------------------------------------------------------------- 8-bit blocks
template <int N>
__device__ __forceinline__ uint32_t most_of(const float (&x)[N]) {
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) most = max(most, abs_bits(x[i]));
  return most;
}

// e4m3 of x / s into the first n bytes at q
template <int N>
__device__ __forceinline__ void store_e4m3(uint8_t* q, const float (&x)[N], float s, int n, bool stream) {
  struct __attribute__((packed, aligned(1))) Bytes {
    uint32_t v[N / 4];
  };
  const Divisor by = divisor(s);
  Bytes w;
#pragma unroll
  for (int i = 0; i < N / 4; ++i)
    w.v[i] = pack_e4m3(divide_by(x[4 * i], by), divide_by(x[4 * i + 1], by), divide_by(x[4 * i + 2], by),
                       divide_by(x[4 * i + 3], by));
  if (n >= N) {
    put(q, w, stream);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) q[i] = (uint8_t)(w.v[i / 4] >> (8 * (i % 4)));
  }
}

// ------------------------------------------------------------- norms around a block
// Sum over a wave, in every lane: sixteen lanes on the data-parallel crossbar,
// then the four groups.
__device__ __forceinline__ float wave_sum_fast(float v) {
  v = lanes_sum(v, 16);
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

constexpr int kNormCols = 4;  // columns of a lane and chunk

// A row belongs to W waves (one up to 256 CH = 2048 columns, else four) and stays
// in registers between its loads and stores: lane i holds the columns
// 4 (i + 64 W c) .. + 3 of chunk c < CH = ceil(D / 256 W), 16-byte loads and
// stores in float32 that a wave makes without a gap, 8-byte ones in bf16, at any
// alignment (with eight columns a lane, 16 bytes of bf16 but two strided loads of
// float32: 4 x 2306 rows of 1024 31.7 against 29.7 us).  Sums are over lanes, and over
// the waves in LDS.  32 lanes of a chunk are one block of 128 columns, which is
// what 8-bit results need.  HBM bound: 10176 rows of 1536 into 8-bit blocks move
// 172 MB in 37 us (4.6 TB/s), 4 x 2306 rows of 1024 with modulation per row 227 MB in
// 42.5 (5.3); requesting gate and modulation ahead of the sums was 3-5% slower
// (registers).
template <int CH, int W, typename TH, typename TY>
__global__ __launch_bounds__(256) void norm_residual_kernel(wam_norm_args a, bool stream_h, bool stream_u, const int* skip) {
  __shared__ float part[2][4];
  if (skip && *skip) return;
  const int lane = threadIdx.x % kWave, wid = threadIdx.x / kWave;
  const int64_t row = W == 1 ? (int64_t)blockIdx.x * (blockDim.x / kWave) + wid : blockIdx.x;
  if (W == 1 && row >= (int64_t)a.B * a.T) return;
  const int b = __builtin_amdgcn_readfirstlane((int)(row / a.T)), t = __builtin_amdgcn_readfirstlane((int)(row % a.T));
  const int D = a.D;
  auto col = [&](int c) { return kNormCols * ((W == 1 ? lane : (int)threadIdx.x) + kWave * W * c); };
  // columns of chunk c that the row has (all four but in the last chunk)
  auto have = [&](int c) { return c < CH - 1 ? kNormCols : D - col(c); };
  int turn = 0;
  auto row_sum = [&](float v) __attribute__((always_inline)) {
    v = wave_sum_fast(v);
    if constexpr (W > 1) {
      if (lane == 0) part[turn][wid] = v;
      __syncthreads();
      v = (part[turn][0] + part[turn][1]) + (part[turn][2] + part[turn][3]);
      turn ^= 1;
    }
    return v;
  };
  // x <- (x - mean) / spread, as kind says
  auto standardise = [&](float (&x)[CH][kNormCols], int kind) __attribute__((always_inline)) {
    if (kind == WAM_NORM_NONE) return;
    if (kind == WAM_NORM_LAYER) {
      float s = 0.f;
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int j = 0; j < kNormCols; ++j) s += x[c][j];  // zero past the row
      const float mean = row_sum(s) / (float)D;
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int j = 0; j < kNormCols; ++j) x[c][j] = c < CH - 1 || j < have(c) ? x[c][j] - mean : 0.f;
    }
    float q = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int j = 0; j < kNormCols; ++j) q += x[c][j] * x[c][j];
    const float rs = rsqrt_newton(row_sum(q) / (float)D + a.eps);
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int j = 0; j < kNormCols; ++j) x[c][j] *= rs;
  };

  float x[CH][kNormCols], y[CH][kNormCols];
  const TH* h = static_cast<const TH*>(a.h) + b * a.h_stride[0] + t * a.h_stride[1];
#pragma unroll
  for (int c = 0; c < CH; ++c) load_n(x[c], h + col(c), have(c));
  if (a.y) {
    const TY* yr = static_cast<const TY*>(a.y) + b * a.y_stride[0] + t * a.y_stride[1];
#pragma unroll
    for (int c = 0; c < CH; ++c) load_n(y[c], yr + col(c), have(c));
    standardise(y, a.post);
    auto times = [&](const float* f) __attribute__((always_inline)) {
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        float v[kNormCols];
        load_n(v, f + col(c), have(c));
#pragma unroll
        for (int j = 0; j < kNormCols; ++j) y[c][j] *= v[j];
      }
    };
    if (a.post_gain) times(a.post_gain);
    if (a.gate) times(a.gate + b * a.gate_stride[0] + t * a.gate_stride[1]);
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int j = 0; j < kNormCols; ++j) x[c][j] = a.res_scale * x[c][j] + y[c][j];
  } else {
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int j = 0; j < kNormCols; ++j) x[c][j] *= a.res_scale;
  }
  if (a.h_out) {
    TH* o = static_cast<TH*>(a.h_out) + b * a.h_out_stride[0] + t * a.h_out_stride[1];
#pragma unroll
    for (int c = 0; c < CH; ++c) store_n(o + col(c), x[c], have(c), stream_h);
  }
  if (!a.u) return;
  standardise(x, a.pre);
  auto each = [&](const float* f, auto OP) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float v[kNormCols];
      load_n(v, f + col(c), have(c));
#pragma unroll
      for (int j = 0; j < kNormCols; ++j) x[c][j] = OP(x[c][j], v[j]);
    }
  };
  if (a.pre_gain) each(a.pre_gain, [](float p, float q) { return p * q; });
  if (a.scale) each(a.scale + b * a.scale_stride[0] + t * a.scale_stride[1], [](float p, float q) { return p * (1.0f + q); });
  if (a.shift) each(a.shift + b * a.shift_stride[0] + t * a.shift_stride[1], [](float p, float q) { return p + q; });
  const int64_t u0 = b * a.u_stride[0] + t * a.u_stride[1];
  if (a.u_dtype == WAM_BF16) {
#pragma unroll
    for (int c = 0; c < CH; ++c) store_n(static_cast<bf16*>(a.u) + u0 + col(c), x[c], have(c), stream_u);
  } else if (a.u_dtype == WAM_FP32) {
#pragma unroll
    for (int c = 0; c < CH; ++c) store_n(static_cast<float*>(a.u) + u0 + col(c), x[c], have(c), stream_u);
  } else {
    float* us = a.u_scale + b * a.u_scale_stride[0] + t * a.u_scale_stride[1];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int n = have(c);
      uint32_t most = group_max<16>(most_of(x[c]));
      most = max(most, (uint32_t)__shfl_xor((int)most, 16, 64));
      const float s = block_scale(most);
      store_e4m3(static_cast<uint8_t*>(a.u) + u0 + col(c), x[c], s, n, stream_u);
      if (lane % 32 == 0 && n > 0) us[col(c) / kScaleBlock] = s;
    }
  }
}

template <int W, typename TH, typename TY>
hipError_t launch_norm_rows(const wam_norm_args& a, hipStream_t s, const int* skip) {
  const int64_t rows = (int64_t)a.B * a.T;
  // one wave per row: blocks of four rows, or of one while the chip has room
  const int block = W > 1 || rows >= 1024 ? 256 : kWave;
  const dim3 grid((unsigned)(W > 1 ? rows : (rows + block / kWave - 1) / (block / kWave)));
  const bool stream_h = rows * a.D * (int64_t)sizeof(TH) > kStreamBytes;
  const bool stream_u = rows * a.D * (a.u_dtype == WAM_FP32 ? 4 : a.u_dtype == WAM_BF16 ? 2 : 1) > kStreamBytes;
  const int chunks = (a.D + kNormCols * kWave * W - 1) / (kNormCols * kWave * W);
  auto launch = [&](auto CH) {
    constexpr int c = decltype(CH)::value;
    if constexpr (W == 1 || c > 2) {  // four waves: past 2048 columns
      if (chunks == c) launch_k(norm_residual_kernel<c, W, TH, TY>, grid, block, 0, s, a, stream_h, stream_u, skip);
    }
  };
  launch(std::integral_constant<int, 1>{});
  launch(std::integral_constant<int, 2>{});
  launch(std::integral_constant<int, 3>{});
  launch(std::integral_constant<int, 4>{});
  launch(std::integral_constant<int, 5>{});
  launch(std::integral_constant<int, 6>{});
  launch(std::integral_constant<int, 7>{});
  launch(std::integral_constant<int, 8>{});
  return hipGetLastError();
}
template <typename TH, typename TY>
hipError_t launch_norm(const wam_norm_args& a, hipStream_t s, const int* skip) {
  return a.D <= 8 * kNormCols * kWave ? launch_norm_rows<1, TH, TY>(a, s, skip) : launch_norm_rows<4, TH, TY>(a, s, skip);
}

// ------------------------------------------------------------- quantisation
// A thread takes 16 columns of a row (two 16-byte loads of bf16, one 16-byte
// store), eight neighbouring threads a scale block of the row, whose maximum
// they share without LDS; the row is read once, from registers.
constexpr int kQuantCols = 16, kQuantGroup = kScaleBlock / kQuantCols;

// blocks of 1 x 128
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(wam_quantize_args a, int kb, bool stream, const int* skip) {
  if (skip && *skip) return;
  const uint32_t i = blockIdx.x * 32u + threadIdx.x / kQuantGroup;  // scale block
  const int m = (int)(i / (uint32_t)kb), bk = (int)(i % (uint32_t)kb);
  if (m >= a.M) return;
  const int col = bk * kScaleBlock + (threadIdx.x % kQuantGroup) * kQuantCols;
  float x[kQuantCols];
  load_n(x, static_cast<const T*>(a.x) + m * a.x_stride + col, a.K - col);
  const float s = block_scale(group_max<kQuantGroup>(most_of(x)));
  if (threadIdx.x % kQuantGroup == 0) a.scale[m * a.scale_stride + bk] = s;
  store_e4m3(static_cast<uint8_t*>(a.q) + m * a.q_stride + col, x, s, a.K - col, stream);
}

// blocks of 128 x 128: one per thread block, four rows per thread in registers
template <typename T>
__global__ __launch_bounds__(256) void quantize_tiles_kernel(wam_quantize_args a, int kb) {
  __shared__ uint32_t top[4];
  constexpr int kRows = kScaleBlock * kQuantGroup / 256;
  const int bk = blockIdx.x % kb, bm = blockIdx.x / kb;
  const int col = bk * kScaleBlock + (threadIdx.x % kQuantGroup) * kQuantCols;
  const int64_t m0 = (int64_t)bm * kScaleBlock + threadIdx.x / kQuantGroup;
  float x[kRows][kQuantCols];
  uint32_t most = 0;
#pragma unroll
  for (int j = 0; j < kRows; ++j) {
    const int64_t m = m0 + j * (256 / kQuantGroup);
    load_n(x[j], static_cast<const T*>(a.x) + m * a.x_stride + col, m < a.M ? a.K - col : 0);
    most = max(most, most_of(x[j]));
  }
  most = wave_max(most);
  if (threadIdx.x % kWave == 0) top[threadIdx.x / kWave] = most;
  __syncthreads();
  const float s = block_scale(max(max(top[0], top[1]), max(top[2], top[3])));
  if (threadIdx.x == 0) a.scale[bm * a.scale_stride + bk] = s;
#pragma unroll
  for (int j = 0; j < kRows; ++j) {
    const int64_t m = m0 + j * (256 / kQuantGroup);
    if (m < a.M) store_e4m3(static_cast<uint8_t*>(a.q) + m * a.q_stride + col, x[j], s, a.K - col, false);
  }
}

template <typename T>
hipError_t launch_blocks(const wam_quantize_args& a, hipStream_t s, const int* skip) {
  const int kb = (a.K + kScaleBlock - 1) / kScaleBlock;
  const int64_t n = (int64_t)kb * ((a.M + a.block_rows - 1) / a.block_rows);
  if (a.block_rows == 1) launch_k(quantize_rows_kernel<T>, dim3((unsigned)((n + 31) / 32)), 256, 0, s, a, kb,
                                    (int64_t)a.M * a.K > kStreamBytes, skip);
  else launch_k(quantize_tiles_kernel<T>, dim3((unsigned)n), 256, 0, s, a, kb);
  return hipGetLastError();
}

// ------------------------------------------------------------- argument checks
constexpr int64_t kMaxStride = (int64_t)1 << 40;  // a larger one is no buffer of this machine

// Elements of a strided result are distinct: by stride, each dimension of more
// than one index steps over the whole of the smaller ones (the last, contiguous
// one has `inner` elements).
bool distinct(const int64_t* stride, const int64_t* size, int n, int64_t inner) {
  bool used[3] = {false, false, false};
  int64_t extent = inner;
  for (int step = 0; step < n; ++step) {
    int at = -1;
    for (int i = 0; i < n; ++i)
      if (!used[i] && size[i] > 1 && (at < 0 || stride[i] < stride[at])) at = i;
    if (at < 0) return true;
    if (stride[at] < extent) return false;
    extent = stride[at] * (size[at] - 1) + extent;
    used[at] = true;
  }
  return true;
}
// strides of at most 2^40 elements, so that no offset or extent passes 64 bits
bool strides_ok(const int64_t* stride, int n) {
  for (int i = 0; i < n; ++i)
    if (stride[i] < 0 || stride[i] > kMaxStride) return false;
  return true;
}
bool same(const int64_t* a, const int64_t* b, int n) {
  for (int i = 0; i < n; ++i)
    if (a[i] != b[i]) return false;
  return true;
}
bool float_type(int t) { return t == WAM_FP32 || t == WAM_BF16; }
int64_t type_size(int t) { return t == WAM_FP32 ? 4 : t == WAM_BF16 ? 2 : 1; }
bool aligned_to(const void* p, int64_t n) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)n == 0; }

// blocks of 256 threads along one dimension of a grid, whose threads count in 32 bits
constexpr int64_t kMaxGrid = (1 << 24) - 1;

int check_heads(int H, const wam_rope_args* a, const void* x, const void* out, const int64_t* si,
                const int64_t* so) {
  if (H == 0) return WAM_OK;
  if (!x || !out) return noalloc_fail(WAM_E_ARG, "wam_rope: null q, k or result");
  if (!aligned_to(x, type_size(a->dtype)) || !aligned_to(out, type_size(a->dtype)))
    return noalloc_fail(WAM_E_ARG, "wam_rope: buffers must be aligned to their elements");
  if (!strides_ok(si, 3)) return noalloc_fail(WAM_E_ARG, "wam_rope: strides must be >= 0");
  const int64_t size[3] = {a->B, a->T, H};
  if (!strides_ok(so, 3) || !distinct(so, size, 3, a->dh))
    return noalloc_fail(WAM_E_ARG, "wam_rope: the elements of a result must be distinct");
  if (x == out && !same(si, so, 3))
    return noalloc_fail(WAM_E_ARG, "wam_rope: a result in place needs the strides of its input");
  return WAM_OK;
}

template <typename T, bool PAIRS, int P>
void launch_rope_units(const RopeParams<P>& p, const RopeTiling& tl, dim3 grid, hipStream_t s) {
  if (p.a.q_gain || p.a.k_gain) launch_k(rope_units_kernel<T, PAIRS, true, P>, grid, 256, 0, s, p, tl);
  else launch_k(rope_units_kernel<T, PAIRS, false, P>, grid, 256, 0, s, p, tl);
}

template <int P>
hipError_t launch_rope_params(const RopeParams<P>& p, hipStream_t s) {
  const wam_rope_args& a = p.a;
  const int64_t rows = (int64_t)a.B * a.T;
  const int H = a.Hq > a.Hk ? a.Hq : a.Hk;
  if (a.dh % 16 || p.pairs % 8) {
    const int64_t blocks = (rows * (a.Hq + a.Hk) + 3) / 4;
    launch_k(rope_kernel<P>, dim3((unsigned)std::min(blocks, kMaxGrid)), 256, 0, s, p);
    return hipGetLastError();
  }
  RopeTiling tl{};
  tl.lanes = 1;
  while (tl.lanes * 16 < a.dh) tl.lanes *= 2;
  // Four heads side by side, two waves along the rows, up to three steps over the
  // heads: within 2% of the fastest of six tilings at 10176 rows of 24 heads of 64 (21.2 us;
  // the slowest 26), of 48 of 32, 2 x 2877 rows of 19 with the norm (13.0; 18), 4 x 2306 of
  // 16 and 5088 float32 rows, rows or heads innermost in memory alike; of 12 heads of
  // 128 within 6% (23.4; 30).  Few rows: one step, so that
  // more blocks share them.
  const int slots = kWave / tl.lanes;
  tl.heads_wave = 1;
  while (tl.heads_wave < 4 && tl.heads_wave < H) tl.heads_wave *= 2;
  tl.wave_rows = 2;
  const int rows_block = slots / tl.heads_wave * tl.wave_rows, head_step = tl.heads_wave * 4 / tl.wave_rows;
  const int64_t row_blocks = (rows + rows_block - 1) / rows_block;
  constexpr int kMaxHeadBlocks = 65535;  // of a grid's second dimension
  const int all_steps = (H + head_step - 1) / head_step;
  const int steps = std::max(row_blocks < 256 ? 1 : std::min(3, all_steps), all_steps / kMaxHeadBlocks + 1);
  tl.heads_block = head_step * steps;
  // in place too, as in the model's layers: no difference there (28.0 us either way, the
  // layers of 9224 and 10176 rows within 1%)
  tl.stream = rows * ((int64_t)a.Hq + a.Hk) * a.dh * (a.dtype == WAM_BF16 ? 2 : 4) > kStreamBytes;
  const int head_blocks = (all_steps + steps - 1) / steps;
  const dim3 grid((unsigned)row_blocks, (unsigned)head_blocks, a.Hq > 0 && a.Hk > 0 ? 2 : 1);
  if (a.dtype == WAM_BF16) {
    if (a.layout == WAM_ROPE_PAIRS) launch_rope_units<bf16, true>(p, tl, grid, s);
    else launch_rope_units<bf16, false>(p, tl, grid, s);
  } else {
    if (a.layout == WAM_ROPE_PAIRS) launch_rope_units<float, true>(p, tl, grid, s);
    else launch_rope_units<float, false>(p, tl, grid, s);
  }
  return hipGetLastError();
}

template <int P>
hipError_t launch_rope_room(const wam_rope_args& a, hipStream_t s, const int* skip) {
  RopeParams<P> p;
  p.a = a;
  p.skip = skip;
  p.end0 = a.sections[0];
  p.end1 = p.end0 + a.sections[1];
  p.pairs = p.end1 + a.sections[2];
  for (int i = 0; i < p.pairs; ++i) p.turns[i] = a.freq[i] * (0.5 / M_PI);
  return launch_rope_params(p, s);
}

}  // namespace

hipError_t launch_rope(const wam_rope_args& a, hipStream_t s, const int* skip) {
  return a.sections[0] + a.sections[1] + a.sections[2] <= kFewPairs ? launch_rope_room<kFewPairs>(a, s, skip)
                                                                    : launch_rope_room<kMaxPairs>(a, s, skip);
}

hipError_t launch_norm_residual(const wam_norm_args& a, hipStream_t s, const int* skip) {
  const bool yf = a.y && a.y_dtype == WAM_FP32;
  if (a.h_dtype == WAM_FP32) return yf ? launch_norm<float, float>(a, s, skip) : launch_norm<float, bf16>(a, s, skip);
  return yf ? launch_norm<bf16, float>(a, s, skip) : launch_norm<bf16, bf16>(a, s, skip);
}

hipError_t launch_quantize(const wam_quantize_args& a, hipStream_t s, const int* skip) {
  return a.dtype == WAM_BF16 ? launch_blocks<bf16>(a, s, skip) : launch_blocks<float>(a, s, skip);
}

}  // namespace wam

using namespace wam;

extern "C" {

int wam_rope_frequencies(const int32_t* sections, double theta, int32_t shared, double* freq) {
  if (!sections || !freq) return noalloc_fail(WAM_E_ARG, "wam_rope_frequencies: null argument");
  if (!(theta > 0.0) || !(theta < INFINITY))
    return noalloc_fail(WAM_E_ARG, "wam_rope_frequencies: theta must be positive and finite");
  int64_t pairs = 0;
  for (int a = 0; a < 3; ++a) {
    if (sections[a] < 0) return noalloc_fail(WAM_E_ARG, "wam_rope_frequencies: sections must be >= 0");
    pairs += sections[a];
  }
  if (pairs > kMaxPairs) return noalloc_fail(WAM_E_SHAPE, "wam_rope_frequencies: at most WAM_MAX_HEAD / 2 pairs");
  int i = 0;
  for (int a = 0; a < 3; ++a)
    for (int j = 0; j < sections[a]; ++j, ++i)
      freq[i] = shared ? pow(theta, -(double)i / (double)pairs) : pow(theta, -(double)j / (double)sections[a]);
  return WAM_OK;
}

int wam_rope(const wam_rope_args* a, void* hip_stream) {
  if (!a) return noalloc_fail(WAM_E_ARG, "wam_rope: null argument");
  if (a->B < 0 || a->T < 0 || a->Hq < 0 || a->Hk < 0) return noalloc_fail(WAM_E_ARG, "wam_rope: sizes must be >= 0");
  if (a->dh < 1 || a->dh > WAM_MAX_HEAD) return noalloc_fail(WAM_E_SHAPE, "wam_rope: head size must be 1..WAM_MAX_HEAD");
  if (!float_type(a->dtype)) return noalloc_fail(WAM_E_ARG, "wam_rope: dtype must be WAM_FP32 or WAM_BF16");
  if (a->layout != WAM_ROPE_HALVES && a->layout != WAM_ROPE_PAIRS)
    return noalloc_fail(WAM_E_ARG, "wam_rope: unknown layout");
  int64_t pairs = 0;
  for (int i = 0; i < 3; ++i) {
    if (a->sections[i] < 0) return noalloc_fail(WAM_E_ARG, "wam_rope: sections must be >= 0");
    pairs += a->sections[i];
  }
  if (2 * pairs > a->dh) return noalloc_fail(WAM_E_SHAPE, "wam_rope: the sections' pairs must fit the head (2 P <= dh)");
  if (pairs > 0 && !a->freq) return noalloc_fail(WAM_E_ARG, "wam_rope: null freq");
  if ((a->q_gain || a->k_gain) && !(a->eps >= 0.f)) return noalloc_fail(WAM_E_ARG, "wam_rope: eps must be >= 0");
  if ((int64_t)a->Hq + a->Hk > WAM_MAX_ROWS) return noalloc_fail(WAM_E_SHAPE, "wam_rope: too many heads");
  if (a->B == 0 || a->T == 0 || a->Hq + a->Hk == 0) return WAM_OK;
  if (!a->pos || !aligned_to(a->pos, 4)) return noalloc_fail(WAM_E_ARG, "wam_rope: null or unaligned pos");
  if (!strides_ok(&a->pos_stride, 1)) return noalloc_fail(WAM_E_ARG, "wam_rope: strides must be >= 0");
  int st = check_heads(a->Hq, a, a->q, a->q_out, a->q_stride, a->q_out_stride);
  if (!st) st = check_heads(a->Hk, a, a->k, a->k_out, a->k_stride, a->k_out_stride);
  if (st) return st;
  if ((int64_t)a->B * a->T > WAM_MAX_ROWS) return noalloc_fail(WAM_E_SHAPE, "wam_rope: too many rows");
  if (a->Hq > 0 && a->Hk > 0 && (a->q_out == a->k_out || a->q_out == a->k || a->k_out == a->q))
    return noalloc_fail(WAM_E_ARG, "wam_rope: a result must not be the other one or its input");
  if (launch_rope(*a, static_cast<hipStream_t>(hip_stream)) != hipSuccess)
    return noalloc_fail(WAM_E_HIP, "wam_rope: kernel launch failed");
  return WAM_OK;
}

int wam_norm_residual(const wam_norm_args* a, void* hip_stream) {
  if (!a) return noalloc_fail(WAM_E_ARG, "wam_norm_residual: null argument");
  if (a->B < 0 || a->T < 0) return noalloc_fail(WAM_E_ARG, "wam_norm_residual: sizes must be >= 0");
  if (a->D < 1 || a->D > WAM_MAX_NORM_D)
    return noalloc_fail(WAM_E_SHAPE, "wam_norm_residual: D must be 1..WAM_MAX_NORM_D");
  if (!float_type(a->h_dtype)) return noalloc_fail(WAM_E_ARG, "wam_norm_residual: h must be WAM_FP32 or WAM_BF16");
  if (!(a->eps >= 0.f)) return noalloc_fail(WAM_E_ARG, "wam_norm_residual: eps must be >= 0");
  auto kind = [](int k) { return k == WAM_NORM_NONE || k == WAM_NORM_RMS || k == WAM_NORM_LAYER; };
  if (!kind(a->post) || !kind(a->pre)) return noalloc_fail(WAM_E_ARG, "wam_norm_residual: unknown norm");
  if ((int64_t)a->B * a->T > WAM_MAX_ROWS) return noalloc_fail(WAM_E_SHAPE, "wam_norm_residual: too many rows");
  if (a->B == 0 || a->T == 0) return WAM_OK;
  const int64_t size[2] = {a->B, a->T};
  if (!a->h) return noalloc_fail(WAM_E_ARG, "wam_norm_residual: null h");
  if (!a->h_out && !a->u) return noalloc_fail(WAM_E_ARG, "wam_norm_residual: no result asked for");
  auto in_ok = [&](const void* p, int64_t n, const int64_t* st) { return !p || (aligned_to(p, n) && strides_ok(st, 2)); };
  auto out_ok = [&](const void* p, int64_t n, const int64_t* st, int64_t inner) {
    return !p || (aligned_to(p, n) && strides_ok(st, 2) && distinct(st, size, 2, inner));
  };
  if (a->y && !float_type(a->y_dtype)) return noalloc_fail(WAM_E_ARG, "wam_norm_residual: y must be WAM_FP32 or WAM_BF16");
  if (a->u && !float_type(a->u_dtype) && a->u_dtype != WAM_FP8)
    return noalloc_fail(WAM_E_ARG, "wam_norm_residual: u must be WAM_FP32, WAM_BF16 or WAM_FP8");
  if (!in_ok(a->h, type_size(a->h_dtype), a->h_stride) || !in_ok(a->y, type_size(a->y_dtype), a->y_stride) ||
      !in_ok(a->gate, 4, a->gate_stride) || !in_ok(a->scale, 4, a->scale_stride) ||
      !in_ok(a->shift, 4, a->shift_stride) || !aligned_to(a->post_gain, 4) || !aligned_to(a->pre_gain, 4))
    return noalloc_fail(WAM_E_ARG, "wam_norm_residual: strides must be >= 0 and buffers aligned to their elements");
  if (!out_ok(a->h_out, type_size(a->h_dtype), a->h_out_stride, a->D) ||
      !out_ok(a->u, type_size(a->u_dtype), a->u_stride, a->D))
    return noalloc_fail(WAM_E_ARG, "wam_norm_residual: the elements of a result must be distinct and aligned");
  if (a->u && a->u_dtype == WAM_FP8 &&
      (!a->u_scale || !out_ok(a->u_scale, 4, a->u_scale_stride, (a->D + kScaleBlock - 1) / kScaleBlock)))
    return noalloc_fail(WAM_E_ARG, "wam_norm_residual: u of WAM_FP8 needs u_scale with distinct elements");
  if (a->h_out == a->h && !same(a->h_out_stride, a->h_stride, 2))
    return noalloc_fail(WAM_E_ARG, "wam_norm_residual: h_out in place needs the strides of h");
  if (a->u && (a->u == a->h || a->u == a->h_out))
    return noalloc_fail(WAM_E_ARG, "wam_norm_residual: u must not be h or h_out");
  if (a->y && (a->h_out == a->y || (a->u == a->y && (a->u_dtype != a->y_dtype || !same(a->u_stride, a->y_stride, 2)))))
    return noalloc_fail(WAM_E_ARG, "wam_norm_residual: h_out must not be y, and u only with its type and strides");
  if (launch_norm_residual(*a, static_cast<hipStream_t>(hip_stream)) != hipSuccess)
    return noalloc_fail(WAM_E_HIP, "wam_norm_residual: kernel launch failed");
  return WAM_OK;
}

int wam_quantize_fp8(const wam_quantize_args* a, void* hip_stream) {
  if (!a) return noalloc_fail(WAM_E_ARG, "wam_quantize_fp8: null argument");
  if (a->M < 0 || a->K < 0) return noalloc_fail(WAM_E_ARG, "wam_quantize_fp8: sizes must be >= 0");
  if (!float_type(a->dtype)) return noalloc_fail(WAM_E_ARG, "wam_quantize_fp8: x must be WAM_FP32 or WAM_BF16");
  if (a->block_rows != 1 && a->block_rows != kScaleBlock)
    return noalloc_fail(WAM_E_ARG, "wam_quantize_fp8: block_rows must be 1 or 128");
  if (a->M == 0 || a->K == 0) return WAM_OK;
  if (!a->x || !a->q || !a->scale) return noalloc_fail(WAM_E_ARG, "wam_quantize_fp8: null buffer");
  if (!aligned_to(a->x, type_size(a->dtype)) || !aligned_to(a->scale, 4))
    return noalloc_fail(WAM_E_ARG, "wam_quantize_fp8: buffers must be aligned to their elements");
  if (a->x == a->q) return noalloc_fail(WAM_E_ARG, "wam_quantize_fp8: q must not be x");
  const int64_t kb = ((int64_t)a->K + kScaleBlock - 1) / kScaleBlock;
  const int64_t mb = ((int64_t)a->M + a->block_rows - 1) / a->block_rows;
  if (!strides_ok(&a->x_stride, 1) || (a->M > 1 && a->q_stride < a->K) || (mb > 1 && a->scale_stride < kb))
    return noalloc_fail(WAM_E_ARG, "wam_quantize_fp8: x_stride must be >= 0, and rows of the results distinct");
  // 32 blocks of one row to a thread block; columns of the last scale block stay in 31 bits
  if (mb * kb > (a->block_rows == 1 ? 32 * kMaxGrid : kMaxGrid) || a->K > INT32_MAX - kScaleBlock)
    return noalloc_fail(WAM_E_SHAPE, "wam_quantize_fp8: too many blocks for one launch");
  if (launch_quantize(*a, static_cast<hipStream_t>(hip_stream)) != hipSuccess)
    return noalloc_fail(WAM_E_HIP, "wam_quantize_fp8: kernel launch failed");
  return WAM_OK;
}

}  // extern "C"
