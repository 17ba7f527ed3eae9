// Product of e4m3 matrices with block scales: checks and dispatch of
// wam_matmul_fp8, and the projections of the 8-bit mode, for the kernels of
// gemm_fp8.h.
#include <utility>

#include "gemm_fp8.h"
#include "layer_util.h"

namespace wam {

namespace {

using gemm::Fp8Operands;
using gemm::Fp8Out;

// Blocks of `threads` for the tiles of an M x N result, 0 where a grid, whose
// threads count in 32 bits, ends before them.
unsigned tile_grid(const Fp8Operands& p, int bm, int bn, int threads) {
  const int64_t blocks = (int64_t)((p.M + bm - 1) / bm) * ((p.N + bn - 1) / bn);
  return blocks * threads > 0xffffffffll ? 0 : (unsigned)blocks;
}

template <int BM, int BN, int WGM, int WGN, int ST, bool EXACT, bool WIDE>
hipError_t launch_tile(const Fp8Operands& p, const Fp8Out& o, bool gelu, hipStream_t s) {
  const dim3 block(WGM * WGN * 64), grid(tile_grid(p, BM, BN, block.x));
  if (!grid.x) return hipErrorInvalidConfiguration;
  if (gelu) launch_k(gemm::gemm_fp8_kernel<BM, BN, WGM, WGN, ST, EXACT, true, WIDE>, grid, block, 0, s, p, o);
  else launch_k(gemm::gemm_fp8_kernel<BM, BN, WGM, WGN, ST, EXACT, false, WIDE>, grid, block, 0, s, p, o);
  return hipGetLastError();
}

template <bool EXACT, int C>
hipError_t launch_cfg(const Fp8Operands& p, const Fp8Out& o, bool gelu, hipStream_t s) {
  constexpr TileCfg t = EXACT ? kFp8ExactCfgs[EXACT ? C : 0] : kFp8Cfgs[C];
  return launch_tile<t.bm, t.bn, t.wgm, t.wgn, t.st, EXACT, false>(p, o, gelu, s);
}

template <bool EXACT, int... C>
hipError_t launch_any(const Fp8Operands& p, const Fp8Out& o, int cfg, bool gelu, hipStream_t s,
                      std::integer_sequence<int, C...>) {
  hipError_t e = hipErrorInvalidValue;
  ((cfg == C ? (void)(e = launch_cfg<EXACT, C>(p, o, gelu, s)) : (void)0), ...);
  return e;
}

constexpr int64_t kNear = (int64_t)1 << 23;  // rows further apart need 64-bit offsets inside a tile

constexpr int kCfgCount = sizeof(kFp8Cfgs) / sizeof(kFp8Cfgs[0]);
constexpr int kExactCfgCount = sizeof(kFp8ExactCfgs) / sizeof(kFp8ExactCfgs[0]);

// 8-bit results
template <int C>
hipError_t launch_blocks_cfg(const Fp8Operands& p, const Fp8Out& o, bool gelu, hipStream_t s, const int* skip) {
  constexpr TileCfg t = kFp8Cfgs[C];
  if constexpr (t.bn % 128 == 0) {
    const dim3 block(t.wgm * t.wgn * 64), grid(tile_grid(p, t.bm, t.bn, block.x));
    if (!grid.x) return hipErrorInvalidConfiguration;
    if (gelu) launch_k(gemm::gemm_fp8_blocks_kernel<t.bm, t.bn, t.wgm, t.wgn, t.st, true>, grid, block, 0, s, p, o, skip);
    else launch_k(gemm::gemm_fp8_blocks_kernel<t.bm, t.bn, t.wgm, t.wgn, t.st, false>, grid, block, 0, s, p, o, skip);
    return hipGetLastError();
  }
  return hipErrorInvalidValue;
}

template <int... C>
hipError_t launch_blocks(const Fp8Operands& p, const Fp8Out& o, bool gelu, hipStream_t s, const int* skip,
                         std::integer_sequence<int, C...>) {
  const int cfg = plan_fp8(kFp8Cfgs, p.M, p.N, p.K, FP8_BLOCKS);
  hipError_t e = hipErrorInvalidValue;
  ((cfg == C ? (void)(e = launch_blocks_cfg<C>(p, o, gelu, s, skip)) : (void)0), ...);
  return e;
}

// out_dtype WAM_FP32 (exact), WAM_BF16 or WAM_FP8
hipError_t launch_fp8(const Fp8Operands& p, const Fp8Out& o, int out_dtype, bool gelu, hipStream_t s) {
  const bool exact = out_dtype == WAM_FP32;
  // offsets of up to 256 rows inside a tile in 32 bits, else rows by 64-bit offsets
  const bool wide = p.lda > kNear || p.ldw > kNear || p.K > kNear;
  if (out_dtype == WAM_FP8)
    return wide ? hipErrorInvalidValue
                : launch_blocks(p, o, gelu, s, nullptr, std::make_integer_sequence<int, kCfgCount>{});
  if (wide)
    return exact ? launch_tile<64, 64, 2, 2, 2, true, true>(p, o, gelu, s)
                 : launch_tile<64, 64, 2, 2, 2, false, true>(p, o, gelu, s);
  if (exact)
    return launch_any<true>(p, o, plan_fp8(kFp8ExactCfgs, p.M, p.N, p.K), gelu, s,
                            std::make_integer_sequence<int, kExactCfgCount>{});
  return launch_any<false>(p, o, plan_fp8(kFp8Cfgs, p.M, p.N, p.K), gelu, s,
                           std::make_integer_sequence<int, kCfgCount>{});
}

template <int C>
hipError_t launch_layer_cfg(const Fp8Operands& p, const GemmArgs& g, hipStream_t s) {
  constexpr TileCfg t = kFp8Cfgs[C];
  const dim3 block(t.wgm * t.wgn * 64), grid(tile_grid(p, t.bm, t.bn, block.x));
  if (!grid.x) return hipErrorInvalidConfiguration;
  auto go = [&](auto EPI) {
    launch_k(gemm::gemm_fp8_layer_kernel<t.bm, t.bn, t.wgm, t.wgn, t.st, decltype(EPI)::value>, grid, block, 0, s, p, g);
    return hipGetLastError();
  };
  switch (g.epi) {
    case EPI_BIAS: return go(std::integral_constant<int, EPI_BIAS>{});
    case EPI_GATED_RES: return go(std::integral_constant<int, EPI_GATED_RES>{});
    case EPI_QKV:
      if constexpr (t.bn / t.wgn == 64) return go(std::integral_constant<int, EPI_QKV>{});
  }
  return hipErrorInvalidValue;
}

template <int... C>
hipError_t launch_layer_any(const Fp8Operands& p, const GemmArgs& g, int cfg, hipStream_t s,
                            std::integer_sequence<int, C...>) {
  hipError_t e = hipErrorInvalidValue;
  ((cfg == C ? (void)(e = launch_layer_cfg<C>(p, g, s)) : (void)0), ...);
  return e;
}

}  // namespace

hipError_t launch_gemm_fp8(const GemmArgs& a, const float* a_scale, const float* w_scale, float* out_scale,
                           hipStream_t s) {
  if (a.M <= 0) return hipSuccess;
  if (a.N % 64 || a.K % 16) return hipErrorInvalidValue;
  const int kb = (a.K + kScaleBlock - 1) / kScaleBlock;
  const Fp8Operands p{static_cast<const uint8_t*>(a.A), static_cast<const uint8_t*>(a.W), a_scale, w_scale, a.K, a.K,
                      kb, kb, a.M, a.N, a.K};
  if (a.epi == EPI_BIAS_GELU) {
    const Fp8Out o{a.bias, a.out, a.N, out_scale, (a.N + kScaleBlock - 1) / kScaleBlock};
    return launch_blocks(p, o, true, s, a.skip, std::make_integer_sequence<int, kCfgCount>{});
  }
  return launch_layer_any(p, a, plan_fp8(kFp8Cfgs, a.M, a.N, a.K, a.epi == EPI_QKV ? FP8_QKV : FP8_PLAIN), s,
                          std::make_integer_sequence<int, kCfgCount>{});
}

}  // namespace wam

using namespace wam;

extern "C" int wam_matmul_fp8(const wam_matmul_args* a, void* hip_stream) {
  if (!a) return noalloc_fail(WAM_E_ARG, "wam_matmul_fp8: null argument");
  if (a->M < 0 || a->N < 0 || a->K < 0) return noalloc_fail(WAM_E_ARG, "wam_matmul_fp8: sizes must be >= 0");
  if (a->out_dtype != WAM_FP32 && a->out_dtype != WAM_BF16 && a->out_dtype != WAM_FP8)
    return noalloc_fail(WAM_E_ARG, "wam_matmul_fp8: out must be WAM_FP32, WAM_BF16 or WAM_FP8");
  if (a->act != WAM_ACT_NONE && a->act != WAM_ACT_GELU)
    return noalloc_fail(WAM_E_ARG, "wam_matmul_fp8: unknown activation");
  if (a->M == 0 || a->N == 0) return WAM_OK;
  if (a->K == 0) return noalloc_fail(WAM_E_SHAPE, "wam_matmul_fp8: K must be >= 1");
  constexpr int kMaxDim = 0x7fffffff - 1024;  // tile arithmetic stays in 31 bits
  if (a->M > kMaxDim || a->N > kMaxDim || a->K > kMaxDim)
    return noalloc_fail(WAM_E_SHAPE, "wam_matmul_fp8: a size is too large");
  if (!a->a || !a->a_scale || !a->w || !a->w_scale || !a->out)
    return noalloc_fail(WAM_E_ARG, "wam_matmul_fp8: null buffer");
  if (!aligned_to(a->a, 16) || !aligned_to(a->w, 16) || (a->M > 1 && a->a_stride % 16) ||
      (a->N > 1 && a->w_stride % 16))
    return noalloc_fail(WAM_E_ARG, "wam_matmul_fp8: a and w must start on 16 bytes, their rows a multiple of 16 apart");
  if ((a->M > 1 && a->a_stride < a->K) || (a->N > 1 && a->w_stride < a->K))
    return noalloc_fail(WAM_E_ARG, "wam_matmul_fp8: rows of a and w must not overlap");
  if (a->a_scale_stride < 0 || a->w_scale_stride < 0 || !aligned_to(a->a_scale, 4) || !aligned_to(a->w_scale, 4) ||
      !aligned_to(a->bias, 4))
    return noalloc_fail(WAM_E_ARG, "wam_matmul_fp8: scales must be aligned, their strides >= 0");
  const int64_t esize = a->out_dtype == WAM_FP32 ? 4 : a->out_dtype == WAM_BF16 ? 2 : 1;
  if (a->out_dtype == WAM_FP8) {
    const int64_t nb = ((int64_t)a->N + kScaleBlock - 1) / kScaleBlock;
    if (!a->out_scale || !aligned_to(a->out_scale, 4) || (a->M > 1 && a->out_scale_stride < nb))
      return noalloc_fail(WAM_E_ARG, "wam_matmul_fp8: out of WAM_FP8 needs out_scale with distinct rows");
    if ((a->M > 1 && a->a_stride > kNear) || (a->N > 1 && a->w_stride > kNear) || a->K > kNear)
      return noalloc_fail(WAM_E_UNSUPPORTED, "wam_matmul_fp8: out of WAM_FP8 needs rows of at most 2^23 bytes");
  }
  if ((a->M > 1 && a->out_stride < a->N) || !aligned_to(a->out, esize))
    return noalloc_fail(WAM_E_ARG, "wam_matmul_fp8: rows of out must be distinct and aligned to their elements");
  if (a->out == a->a || a->out == a->w) return noalloc_fail(WAM_E_ARG, "wam_matmul_fp8: out must not be a or w");
  gemm::Fp8Operands p{static_cast<const uint8_t*>(a->a), static_cast<const uint8_t*>(a->w), a->a_scale, a->w_scale,
                      a->M > 1 ? a->a_stride : 0, a->N > 1 ? a->w_stride : 0, a->a_scale_stride, a->w_scale_stride,
                      a->M, a->N, a->K};
  gemm::Fp8Out o{a->bias, a->out, a->out_stride, a->out_scale, a->out_scale_stride};
  const hipError_t e = launch_fp8(p, o, a->out_dtype, a->act == WAM_ACT_GELU, static_cast<hipStream_t>(hip_stream));
  if (e == hipErrorInvalidConfiguration) return noalloc_fail(WAM_E_SHAPE, "wam_matmul_fp8: too many tiles for one launch");
  if (e != hipSuccess) return noalloc_fail(WAM_E_HIP, "wam_matmul_fp8: kernel launch failed");
  return WAM_OK;
}
