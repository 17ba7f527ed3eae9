// 4-bit blocks: into them, back to values, and new keys and values into a paged cache
// of them (gfx950).  All are bound by memory.
#include <math.h>

#include <algorithm>

#include "cache.h"
#include "fp4.h"
#include "layer_util.h"

namespace wam {

namespace {

// ------------------------------------------------------------- blocks of a matrix
// A lane takes eight neighbouring columns (16 bytes of bf16), four lanes a block, whose
// maximum they share without LDS; a wave stores its codes as 256 bytes side by side
// (10176 x 6144 of bf16 30 us, 5.3 TB/s; back to values 23 us, 6.9 TB/s).
template <typename T>
__global__ __launch_bounds__(256) void quantize_fp4_kernel(wam_quantize_fp4_args a, int kb) {
  const uint32_t i = blockIdx.x * 64u + threadIdx.x / 4;  // block
  const int m = (int)(i / (uint32_t)kb), bk = (int)(i % (uint32_t)kb);
  if (m >= a.M) return;
  const int col = bk * kFp4Block + (threadIdx.x % 4) * 8;
  float x[8];
  load_n(x, static_cast<const T*>(a.x) + m * a.x_stride + col, a.K - col);
  const uint32_t byte = fp4_scale(quad_max(most_of(x)));
  if (threadIdx.x % 4 == 0) a.scale[m * a.scale_stride + bk] = (uint8_t)byte;
  store_fp4(a.q + m * a.q_stride + col / 2, pack_fp4(x, byte), a.K - col);
}

template <typename T>
__global__ __launch_bounds__(256) void dequantize_fp4_kernel(wam_dequantize_fp4_args a, int kb, bool stream) {
  const uint32_t i = blockIdx.x * 64u + threadIdx.x / 4;
  const int m = (int)(i / (uint32_t)kb), bk = (int)(i % (uint32_t)kb);
  if (m >= a.M) return;
  const int col = bk * kFp4Block + (threadIdx.x % 4) * 8, n = a.K - col;
  if (n <= 0) return;
  const uint8_t* q = a.q + m * a.q_stride + col / 2;
  uint32_t w = 0;
  if (n >= 7) {
    struct __attribute__((packed, aligned(1))) Word {
      uint32_t v;
    };
    w = reinterpret_cast<const Word*>(q)->v;
  } else {
#pragma unroll
    for (int b = 0; b < 3; ++b)
      if (2 * b < n) w |= (uint32_t)q[b] << (8 * b);
  }
  float x[8];
  fp4_to_f32(x, w, fp4_scale_operand(a.scale[m * a.scale_stride + bk]));
  store_n(static_cast<T*>(a.x) + m * a.x_stride + col, x, n, stream);
}

// ------------------------------------------------------------- appending to a cache
constexpr int kAppendMaxPairs = 64;  // heads of at most 128
constexpr int kAppendFewPairs = 32;  // arguments travel with every launch: a form for heads of up to 64
template <int P>
struct AppendParams {
  wam_cache_append_args a;
  int pairs, end0, end1, shift;
  int lanes;        // lanes of a head vector, a power of two >= dh / 8
  int rows_block;   // rows of a thread block
  double inverse;   // 1 / dh
  double turns[P];  // revolutions per unit of position
};

// Sum over aligned groups of n lanes (4, 8 or 16), in every lane.
template <int CTRL>
__device__ __forceinline__ double dpp_d(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  return __builtin_bit_cast(double, (uint64_t)dpp<CTRL>((uint32_t)(u >> 32)) << 32 | dpp<CTRL>((uint32_t)u));
}
__device__ __forceinline__ double lanes_sum_d(double v, int n) {
  v += dpp_d<0xb1>(v);
  v += dpp_d<0x4e>(v);
  if (n >= 8) v += dpp_d<0x141>(v);
  if (n >= 16) v += dpp_d<0x140>(v);
  return v;
}

// cos and sin of the angles of a block's rows, [row][pair], into LDS.  The product with the
// position is taken in revolutions, so that dropping the whole ones is exact.
template <int P>
__device__ __forceinline__ void append_turns(const AppendParams<P>& p, int row0, int rows, double2* turn) {
  for (int i = threadIdx.x; i < rows * p.pairs; i += 256) {
    const int row = row0 + i / p.pairs, j = i % p.pairs;
    const float* pos = p.a.pos + row / p.a.T * p.a.pos_stride + row % p.a.T * 3;
    double t = (double)pos[j < p.end0 ? 0 : j < p.end1 ? 1 : 2] * p.turns[j];
    t -= rint(t);
    double c, s;
    sincospi(2.0 * t, &s, &c);
    turn[i] = make_double2(c, s);
  }
}

// Place of a row's token in its page, and the page: -1 where the row is dropped.
template <int P>
__device__ __forceinline__ int append_page(const AppendParams<P>& p, int b, int t, int& place) {
  const wam_cache_append_args& a = p.a;
  if (a.rows && t >= a.rows[b]) return -1;
  const int64_t token = (int64_t)a.start[b] + t;
  place = (int)(token & ((1 << p.shift) - 1));
  if (token > INT32_MAX) return -1;
  return page_of(a.table.entry + b * a.table.stride, a.table.width, p.shift, a.cache.pages, (int)token);
}

// A lane takes eight neighbouring values of a head vector, four lanes a block of it.
// Keys are normed and turned in float64 and rounded to float32 once: a value next to a
// border between two codes moves by a whole step, so with float32 arithmetic the codes
// would hang on the order of its roundings.  The vector pipe does float64 at the rate of
// float32, so that costs little beside the loads.  A block's angles are computed once, in
// LDS; a thread keeps one row for all the heads it visits, with the products of its
// cosines, sines and gains in registers.  The other values of its pairs are a load of
// their own (a lane's eight are neighbours, so that a block of 32 lies in four lanes).
// The values' heads go along with the keys'; both are loaded one ahead of the arithmetic,
// the first before the row's page is known (10176 rows of 24 heads of 64 with the RMS norm,
// from HBM: 36 us with keys and values in blocks of their own, 31 so; 26 without its stores).
template <typename T, bool PAIRS, int P>
__global__ __launch_bounds__(256) void cache_append_units_kernel(AppendParams<P> p) {
  extern __shared__ double2 turn[];
  const wam_cache_append_args& a = p.a;
  const wam_cache& ca = a.cache;
  const int rows = a.B * a.T, row0 = blockIdx.x * p.rows_block, live_rows = min(p.rows_block, rows - row0);
  const int slot = threadIdx.x / p.lanes, unit = threadIdx.x % p.lanes, col = 8 * unit;
  const int heads_par = 256 / p.lanes / p.rows_block;
  const int row = row0 + slot / heads_par, b = row / a.T, t = row % a.T;
  int h = blockIdx.y * heads_par + slot % heads_par;
  const int step = gridDim.y * heads_par;
  const bool mine = row < rows && col < ca.dh;  // idle lanes of 96 values take part in the exchanges
  int place = 0;
  const int page = row < rows ? append_page(p, b, t, place) : -1;

  const T *xk = static_cast<const T*>(a.k) + col, *xv = static_cast<const T*>(a.v) + col;
  if (mine) {
    xk += b * a.k_stride[0] + t * a.k_stride[1];
    xv += b * a.v_stride[0] + t * a.v_stride[1];
  }
  const bool turned = col < 2 * p.pairs;
  const int other = PAIRS || !turned ? 0 : col < p.pairs ? p.pairs : -p.pairs;  // from the lane's own values
  Pack<T, 8> own{}, far{}, val{};
  auto load = [&](int hh) __attribute__((always_inline)) {
    if (mine && hh < ca.H) {
      own = *reinterpret_cast<const Pack<T, 8>*>(xk + hh * a.k_stride[2]);
      if (!PAIRS && turned) far = *reinterpret_cast<const Pack<T, 8>*>(xk + hh * a.k_stride[2] + other);
      val = *reinterpret_cast<const Pack<T, 8>*>(xv + hh * a.v_stride[2]);
    }
  };
  load(h);
  double gc[8], gs[8];  // factors of the lane's own values and of the others
  const bool normed = a.k_gain;
  append_turns(p, row0, live_rows, turn);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int j = PAIRS ? 4 * unit + i / 2 : (col < p.pairs ? col : col + other) + i;
    const bool first = PAIRS ? i % 2 == 0 : col < p.pairs;
    const double2 cs = turned && mine ? turn[slot / heads_par * p.pairs + j] : make_double2(1.0, 0.0);
    gc[i] = cs.x, gs[i] = first ? -cs.y : cs.y;
    if (normed && mine) {
      gc[i] *= (double)a.k_gain[col + i];
      gs[i] *= (double)a.k_gain[PAIRS ? col + (i ^ 1) : col + other + i];
    }
  }
  uint8_t* qk = ca.k + page * ca.k_stride[0] + place * ca.k_stride[1] + col / 2;
  uint8_t* qv = ca.v + page * ca.v_stride[0] + place * ca.v_stride[1] + col / 2;
  uint8_t* sk = ca.k_scale + page * ca.k_scale_stride[0] + place * ca.k_scale_stride[1] + col / kFp4Block;
  uint8_t* sv = ca.v_scale + page * ca.v_scale_stride[0] + place * ca.v_scale_stride[1] + col / kFp4Block;
  for (int h0 = blockIdx.y * heads_par; h0 < ca.H; h0 += step, h += step) {
    float y[8], v[8];
    double z[8], w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = to_f32(own.v[i]), v[i] = to_f32(val.v[i]);
    if (p.pairs || normed) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        z[i] = (double)y[i];
        w[i] = (double)to_f32(PAIRS ? own.v[i ^ 1] : far.v[i]);
      }
    }
    load(h + step);  // while this head is turned
    if (p.pairs || normed) {
      double rs = 1.0;
      if (normed) {
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += z[i] * z[i];
        rs = rsqrt(lanes_sum_d(mine ? sum : 0.0, p.lanes) * p.inverse + a.eps);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)  // past the pairs: not plus 0, which would spread a NaN or an infinity
        y[i] = (float)((turned ? z[i] * gc[i] + w[i] * gs[i] : z[i] * gc[i]) * rs);
    }
    const uint32_t bk = fp4_scale(quad_max(mine ? most_of(y) : 0)), bv = fp4_scale(quad_max(mine ? most_of(v) : 0));
    if (!mine || page < 0 || h >= ca.H) continue;
    *reinterpret_cast<uint32_t*>(qk + h * ca.k_stride[2]) = pack_fp4(y, bk);
    *reinterpret_cast<uint32_t*>(qv + h * ca.v_stride[2]) = pack_fp4(v, bv);
    if (unit % 4 == 0) {
      sk[h * ca.k_scale_stride[2]] = (uint8_t)bk;
      sv[h * ca.v_scale_stride[2]] = (uint8_t)bv;
    }
  }
}

// Sections of any number of pairs: value by value.
template <typename T, int P>
__global__ __launch_bounds__(256) void cache_append_kernel(AppendParams<P> p) {
  extern __shared__ double2 turn[];
  const wam_cache_append_args& a = p.a;
  const wam_cache& ca = a.cache;
  const bool isk = blockIdx.z == 0;
  const int rows = a.B * a.T, row0 = blockIdx.x * p.rows_block, live_rows = min(p.rows_block, rows - row0);
  const int vectors = 256 / p.lanes;  // of the block at a time
  const int slot = threadIdx.x / p.lanes, unit = threadIdx.x % p.lanes, col = 8 * unit;
  if (isk) {
    append_turns(p, row0, live_rows, turn);
    __syncthreads();
  }
  for (int v = slot; v < live_rows * ca.H; v += vectors) {
    const int r = v / ca.H, h = v % ca.H, row = row0 + r, b = row / a.T, t = row % a.T;
    int place = 0;
    const int page = append_page(p, b, t, place);
    if (page < 0) continue;
    float y[8];
    const int64_t* si = isk ? a.k_stride : a.v_stride;
    const T* x = static_cast<const T*>(isk ? a.k : a.v) + b * si[0] + t * si[1] + h * si[2];
    const int n = col < ca.dh ? 8 : 0;
    load_n(y, x + col, n);
    if (isk) {
      double d[8], rs = 1.0;
      if (a.k_gain) {
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += (double)y[i] * (double)y[i];
        rs = rsqrt(lanes_sum_d(sum, p.lanes) * p.inverse + a.eps);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) d[i] = (double)y[i] * rs * (a.k_gain && n ? (double)a.k_gain[col + i] : 1.0);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int e = col + i;
        y[i] = (float)d[i];
        if (e >= 2 * p.pairs || !n) continue;
        const bool pairs = a.layout == WAM_ROPE_PAIRS;
        const bool first = pairs ? e % 2 == 0 : e < p.pairs;
        const int partner = pairs ? e ^ 1 : first ? e + p.pairs : e - p.pairs;
        double o = (double)to_f32(x[partner]) * rs;
        if (a.k_gain) o *= (double)a.k_gain[partner];
        const double2 cs = turn[r * p.pairs + (pairs ? e / 2 : first ? e : partner)];
        y[i] = (float)(d[i] * cs.x + (first ? -o : o) * cs.y);
      }
    }
    const uint32_t byte = fp4_scale(quad_max(most_of(y)));
    if (!n) continue;
    const int64_t* so = isk ? ca.k_stride : ca.v_stride;
    const int64_t* ss = isk ? ca.k_scale_stride : ca.v_scale_stride;
    uint8_t* q = (isk ? ca.k : ca.v) + page * so[0] + place * so[1] + h * so[2];
    *reinterpret_cast<uint32_t*>(q + col / 2) = pack_fp4(y, byte);
    if (unit % 4 == 0)
      ((isk ? ca.k_scale : ca.v_scale) + page * ss[0] + place * ss[1] + h * ss[2])[col / kFp4Block] = (uint8_t)byte;
  }
}

template <typename T, int P>
void launch_append_type(const AppendParams<P>& p, dim3 grid, size_t lds, hipStream_t s) {
  if (p.pairs % 8) launch_k(cache_append_kernel<T, P>, dim3(grid.x, 1, 2), 256, lds, s, p);
  else if (p.a.layout == WAM_ROPE_PAIRS) launch_k(cache_append_units_kernel<T, true, P>, grid, 256, lds, s, p);
  else launch_k(cache_append_units_kernel<T, false, P>, grid, 256, lds, s, p);
}

template <int P>
hipError_t launch_append(const wam_cache_append_args& a, int shift, hipStream_t s) {
  AppendParams<P> p;
  p.a = a;
  p.shift = shift;
  p.end0 = a.sections[0];
  p.end1 = p.end0 + a.sections[1];
  p.pairs = p.end1 + a.sections[2];
  for (int i = 0; i < p.pairs; ++i) p.turns[i] = a.freq[i] * (0.5 / M_PI);
  p.inverse = 1.0 / a.cache.dh;
  p.lanes = 4;
  while (p.lanes * 8 < a.cache.dh) p.lanes *= 2;
  const int rows = a.B * a.T, H = a.cache.H, slots = 256 / p.lanes;
  // 16 rows a block, whose codes of a head lie side by side in its page; fewer where
  // that leaves CUs without a block
  p.rows_block = 16;
  while (p.rows_block > 1 && (rows + p.rows_block - 1) / p.rows_block < 512) p.rows_block /= 2;
  const int heads_par = slots / p.rows_block, head_blocks = (H + heads_par - 1) / heads_par;
  const int row_blocks = (rows + p.rows_block - 1) / p.rows_block;
  const dim3 grid(row_blocks, row_blocks >= 512 ? 1 : std::min(head_blocks, 65535));
  const size_t lds = sizeof(double2) * p.rows_block * p.pairs;
  if (a.dtype == WAM_BF16) launch_append_type<bf16>(p, grid, lds, s);
  else launch_append_type<float>(p, grid, lds, s);
  return hipGetLastError();
}

int page_shift(int page) {
  int s = 0;
  while ((1 << s) < page) ++s;
  return s;
}

}  // namespace

// Status of a cache and its table; `what` is the call's name.  empty: the call has no
// rows, so that nothing needs to be there.
int check_cache(const wam_cache& c, const wam_page_table& t, bool written, bool empty, const char* what) {
  static thread_local char msg[160];
  auto fail = [&](int code, const char* text) {
    snprintf(msg, sizeof(msg), "%s: %s", what, text);
    return noalloc_fail(code, msg);
  };
  if (c.pages < 0 || c.H < 1 || t.width < 0) return fail(WAM_E_ARG, "a cache needs heads, and pages and table >= 0");
  if (c.dh < 32 || c.dh > 128 || c.dh % kFp4Block) return fail(WAM_E_SHAPE, "head size must be 32, 64, 96 or 128");
  if (c.page < 16 || c.page > 4096 || (c.page & (c.page - 1)))
    return fail(WAM_E_SHAPE, "pages must hold a power of two of tokens, 16 to 4096");
  if ((int64_t)t.width * c.page > INT32_MAX - 4096) return fail(WAM_E_SHAPE, "a sequence must stay below 2^31 - 4096 tokens");
  if (c.H > WAM_MAX_ROWS) return fail(WAM_E_SHAPE, "too many heads");
  if (empty || c.pages == 0 || t.width == 0) return WAM_OK;
  if (!c.k || !c.v || !c.k_scale || !c.v_scale || !t.entry) return fail(WAM_E_ARG, "null cache or table");
  if (written && (c.k == c.v || c.k_scale == c.v_scale || c.k == c.k_scale || c.k == c.v_scale || c.v == c.k_scale ||
                  c.v == c.v_scale))
    return fail(WAM_E_ARG, "the cache's arrays must be different buffers");
  if (!aligned_to(c.k, 4) || !aligned_to(c.v, 4) || !aligned_to(t.entry, 4))
    return fail(WAM_E_ARG, "codes and table must start on 4 bytes");
  if (!strides_ok(c.k_stride, 3) || !strides_ok(c.v_stride, 3) || !strides_ok(c.k_scale_stride, 3) ||
      !strides_ok(c.v_scale_stride, 3) || !strides_ok(&t.stride, 1))
    return fail(WAM_E_ARG, "strides must be >= 0");
  for (int i = 0; i < 3; ++i)
    if (c.k_stride[i] % 4 || c.v_stride[i] % 4) return fail(WAM_E_ARG, "strides of codes must be multiples of 4");
  const int64_t near = (int64_t)1 << 26;  // offsets of 16 tokens in 32 bits
  if (c.k_stride[1] > near || c.v_stride[1] > near || c.k_scale_stride[1] > near || c.v_scale_stride[1] > near)
    return fail(WAM_E_SHAPE, "tokens of a page must be at most 2^26 bytes apart");
  const int64_t size[3] = {c.pages, c.page, c.H};
  if (written && (!distinct(c.k_stride, size, 3, c.dh / 2) || !distinct(c.v_stride, size, 3, c.dh / 2) ||
                  !distinct(c.k_scale_stride, size, 3, c.dh / kFp4Block) ||
                  !distinct(c.v_scale_stride, size, 3, c.dh / kFp4Block)))
    return fail(WAM_E_ARG, "the bytes of the cache must be distinct");
  return WAM_OK;
}

}  // namespace wam

using namespace wam;

extern "C" {

int wam_quantize_fp4(const wam_quantize_fp4_args* a, void* hip_stream) {
  if (!a) return noalloc_fail(WAM_E_ARG, "wam_quantize_fp4: null argument");
  if (a->M < 0 || a->K < 0) return noalloc_fail(WAM_E_ARG, "wam_quantize_fp4: sizes must be >= 0");
  if (!float_type(a->dtype)) return noalloc_fail(WAM_E_ARG, "wam_quantize_fp4: x must be WAM_FP32 or WAM_BF16");
  if (a->M == 0 || a->K == 0) return WAM_OK;
  if (!a->x || !a->q || !a->scale) return noalloc_fail(WAM_E_ARG, "wam_quantize_fp4: null buffer");
  if (!aligned_to(a->x, type_size(a->dtype)))
    return noalloc_fail(WAM_E_ARG, "wam_quantize_fp4: x must be aligned to its elements");
  if (a->x == a->q || a->x == a->scale || a->q == a->scale)
    return noalloc_fail(WAM_E_ARG, "wam_quantize_fp4: x, q and scale must be different buffers");
  const int64_t kb = ((int64_t)a->K + kFp4Block - 1) / kFp4Block;
  if (!strides_ok(&a->x_stride, 1) || !strides_ok(&a->q_stride, 1) || !strides_ok(&a->scale_stride, 1) ||
      (a->M > 1 && (a->q_stride < ((int64_t)a->K + 1) / 2 || a->scale_stride < kb)))
    return noalloc_fail(WAM_E_ARG, "wam_quantize_fp4: strides must be >= 0, and rows of the results distinct");
  if (a->M * kb > 32 * kMaxGrid || a->K > INT32_MAX - kFp4Block)
    return noalloc_fail(WAM_E_SHAPE, "wam_quantize_fp4: too many blocks for one launch");
  const dim3 grid((unsigned)((a->M * kb + 63) / 64));
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (a->dtype == WAM_BF16) launch_k(quantize_fp4_kernel<bf16>, grid, 256, 0, s, *a, (int)kb);
  else launch_k(quantize_fp4_kernel<float>, grid, 256, 0, s, *a, (int)kb);
  if (hipGetLastError() != hipSuccess) return noalloc_fail(WAM_E_HIP, "wam_quantize_fp4: kernel launch failed");
  return WAM_OK;
}

int wam_dequantize_fp4(const wam_dequantize_fp4_args* a, void* hip_stream) {
  if (!a) return noalloc_fail(WAM_E_ARG, "wam_dequantize_fp4: null argument");
  if (a->M < 0 || a->K < 0) return noalloc_fail(WAM_E_ARG, "wam_dequantize_fp4: sizes must be >= 0");
  if (!float_type(a->dtype)) return noalloc_fail(WAM_E_ARG, "wam_dequantize_fp4: x must be WAM_FP32 or WAM_BF16");
  if (a->M == 0 || a->K == 0) return WAM_OK;
  if (!a->x || !a->q || !a->scale) return noalloc_fail(WAM_E_ARG, "wam_dequantize_fp4: null buffer");
  if (!aligned_to(a->x, type_size(a->dtype)))
    return noalloc_fail(WAM_E_ARG, "wam_dequantize_fp4: x must be aligned to its elements");
  if (a->x == a->q || a->x == a->scale) return noalloc_fail(WAM_E_ARG, "wam_dequantize_fp4: x must not be q or scale");
  const int64_t kb = ((int64_t)a->K + kFp4Block - 1) / kFp4Block;
  if (!strides_ok(&a->x_stride, 1) || !strides_ok(&a->q_stride, 1) || !strides_ok(&a->scale_stride, 1) ||
      (a->M > 1 && a->x_stride < a->K))
    return noalloc_fail(WAM_E_ARG, "wam_dequantize_fp4: strides must be >= 0, and rows of x distinct");
  if (a->M * kb > 32 * kMaxGrid || a->K > INT32_MAX - kFp4Block)
    return noalloc_fail(WAM_E_SHAPE, "wam_dequantize_fp4: too many blocks for one launch");
  const dim3 grid((unsigned)((a->M * kb + 63) / 64));
  const bool stream = (int64_t)a->M * a->K * type_size(a->dtype) > kStreamBytes;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (a->dtype == WAM_BF16) launch_k(dequantize_fp4_kernel<bf16>, grid, 256, 0, s, *a, (int)kb, stream);
  else launch_k(dequantize_fp4_kernel<float>, grid, 256, 0, s, *a, (int)kb, stream);
  if (hipGetLastError() != hipSuccess) return noalloc_fail(WAM_E_HIP, "wam_dequantize_fp4: kernel launch failed");
  return WAM_OK;
}

int wam_cache_append(const wam_cache_append_args* a, void* hip_stream) {
  if (!a) return noalloc_fail(WAM_E_ARG, "wam_cache_append: null argument");
  if (a->B < 0 || a->T < 0) return noalloc_fail(WAM_E_ARG, "wam_cache_append: sizes must be >= 0");
  if (!float_type(a->dtype)) return noalloc_fail(WAM_E_ARG, "wam_cache_append: k and v must be WAM_FP32 or WAM_BF16");
  if (a->layout != WAM_ROPE_HALVES && a->layout != WAM_ROPE_PAIRS)
    return noalloc_fail(WAM_E_ARG, "wam_cache_append: unknown layout");
  int st = check_cache(a->cache, a->table, true, a->B == 0 || a->T == 0, "wam_cache_append");
  if (st) return st;
  int64_t pairs = 0;
  for (int i = 0; i < 3; ++i) {
    if (a->sections[i] < 0) return noalloc_fail(WAM_E_ARG, "wam_cache_append: sections must be >= 0");
    pairs += a->sections[i];
  }
  if (2 * pairs > a->cache.dh)
    return noalloc_fail(WAM_E_SHAPE, "wam_cache_append: the sections' pairs must fit the head (2 P <= dh)");
  if (pairs > 0 && !a->freq) return noalloc_fail(WAM_E_ARG, "wam_cache_append: null freq");
  if (a->k_gain && (!(a->eps >= 0.0) || !aligned_to(a->k_gain, 4)))
    return noalloc_fail(WAM_E_ARG, "wam_cache_append: eps must be >= 0");
  if ((int64_t)a->B * a->T > WAM_MAX_ROWS) return noalloc_fail(WAM_E_SHAPE, "wam_cache_append: too many rows");
  if (a->B == 0 || a->T == 0) return WAM_OK;
  if (pairs > 0 && (!a->pos || !aligned_to(a->pos, 4) || !strides_ok(&a->pos_stride, 1)))
    return noalloc_fail(WAM_E_ARG, "wam_cache_append: pairs need pos, aligned, with a stride >= 0");
  if (!a->k || !a->v || !a->start) return noalloc_fail(WAM_E_ARG, "wam_cache_append: null k, v or start");
  if (!aligned_to(a->k, type_size(a->dtype)) || !aligned_to(a->v, type_size(a->dtype)) || !aligned_to(a->start, 4) ||
      !aligned_to(a->rows, 4) || !strides_ok(a->k_stride, 3) || !strides_ok(a->v_stride, 3))
    return noalloc_fail(WAM_E_ARG, "wam_cache_append: strides must be >= 0 and buffers aligned to their elements");
  if (a->cache.pages == 0 || a->table.width == 0) return WAM_OK;  // no token has a page
  const int shift = page_shift(a->cache.page);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const hipError_t e = pairs <= kAppendFewPairs ? launch_append<kAppendFewPairs>(*a, shift, s)
                                                : launch_append<kAppendMaxPairs>(*a, shift, s);
  if (e != hipSuccess)
    return noalloc_fail(WAM_E_HIP, "wam_cache_append: kernel launch failed");
  return WAM_OK;
}

}  // extern "C"
