// Product of matrices in 4-bit blocks: checks and dispatch of wam_matmul_fp4, for the
// kernels of gemm_fp4.h.
#include <utility>

#include "gemm_fp4.h"
#include "layer_util.h"

namespace wam {

namespace {

using gemm::Fp4Operands;
using gemm::Fp8Out;

constexpr int64_t kNear = (int64_t)1 << 23;  // rows further apart need 64-bit offsets inside a tile
constexpr int kCfgCount = sizeof(kFp4Cfgs) / sizeof(kFp4Cfgs[0]);

template <int BM, int BN, int WGM, int WGN, int ST, bool WIDE>
hipError_t launch_tile(const Fp4Operands& p, const Fp8Out& o, uint8_t* scale, int out_dtype, bool gelu, hipStream_t s) {
  const dim3 block(WGM * WGN * 64);
  const int64_t blocks = (int64_t)((p.M + BM - 1) / BM) * ((p.N + BN - 1) / BN);
  if (blocks * block.x > 0xffffffffll) return hipErrorInvalidConfiguration;  // a grid's threads count in 32 bits
  const dim3 grid((unsigned)blocks);
  auto go = [&](auto GELU) {
    constexpr bool g = decltype(GELU)::value;
    if (out_dtype == WAM_FP4) {
      if constexpr (BN / WGN % 32 == 0)
        launch_k(gemm::gemm_fp4_blocks_kernel<BM, BN, WGM, WGN, ST, g, WIDE>, grid, block, 0, s, p, o, scale);
      else return hipErrorInvalidValue;
    } else if (out_dtype == WAM_FP32) {
      launch_k(gemm::gemm_fp4_kernel<BM, BN, WGM, WGN, ST, true, g, WIDE>, grid, block, 0, s, p, o);
    } else {
      launch_k(gemm::gemm_fp4_kernel<BM, BN, WGM, WGN, ST, false, g, WIDE>, grid, block, 0, s, p, o);
    }
    return hipGetLastError();
  };
  return gelu ? go(std::true_type{}) : go(std::false_type{});
}

template <int C>
hipError_t launch_cfg(const Fp4Operands& p, const Fp8Out& o, uint8_t* scale, int out_dtype, bool gelu, hipStream_t s) {
  constexpr TileCfg t = kFp4Cfgs[C];
  return launch_tile<t.bm, t.bn, t.wgm, t.wgn, t.st, false>(p, o, scale, out_dtype, gelu, s);
}

template <int... C>
hipError_t launch_any(const Fp4Operands& p, const Fp8Out& o, uint8_t* scale, int out_dtype, bool gelu, int cfg,
                      hipStream_t s, std::integer_sequence<int, C...>) {
  hipError_t e = hipErrorInvalidValue;
  ((cfg == C ? (void)(e = launch_cfg<C>(p, o, scale, out_dtype, gelu, s)) : (void)0), ...);
  return e;
}

hipError_t launch_fp4(const Fp4Operands& p, const Fp8Out& o, uint8_t* scale, int out_dtype, bool gelu, hipStream_t s) {
  if (p.lda > kNear || p.ldw > kNear || p.K > kNear)
    return launch_tile<64, 64, 2, 2, 2, true>(p, o, scale, out_dtype, gelu, s);
  const int cfg = plan_fp4(kFp4Cfgs, p.M, p.N, p.K, out_dtype == WAM_FP4);
  return launch_any(p, o, scale, out_dtype, gelu, cfg, s, std::make_integer_sequence<int, kCfgCount>{});
}

}  // namespace

}  // namespace wam

using namespace wam;

extern "C" int wam_matmul_fp4(const wam_matmul_fp4_args* a, void* hip_stream) {
  if (!a) return noalloc_fail(WAM_E_ARG, "wam_matmul_fp4: null argument");
  if (a->M < 0 || a->N < 0 || a->K < 0) return noalloc_fail(WAM_E_ARG, "wam_matmul_fp4: sizes must be >= 0");
  if (a->out_dtype != WAM_FP32 && a->out_dtype != WAM_BF16 && a->out_dtype != WAM_FP4)
    return noalloc_fail(WAM_E_ARG, "wam_matmul_fp4: out must be WAM_FP32, WAM_BF16 or WAM_FP4");
  if (a->act != WAM_ACT_NONE && a->act != WAM_ACT_GELU)
    return noalloc_fail(WAM_E_ARG, "wam_matmul_fp4: unknown activation");
  if (a->M == 0 || a->N == 0) return WAM_OK;
  if (a->K == 0) return noalloc_fail(WAM_E_SHAPE, "wam_matmul_fp4: K must be >= 2");
  if (a->K % 2) return noalloc_fail(WAM_E_SHAPE, "wam_matmul_fp4: K must be even (whole bytes)");
  constexpr int kMaxDim = 0x7fffffff - 1024;  // tile arithmetic stays in 31 bits
  if (a->M > kMaxDim || a->N > kMaxDim || a->K > kMaxDim)
    return noalloc_fail(WAM_E_SHAPE, "wam_matmul_fp4: a size is too large");
  if (!a->a || !a->a_scale || !a->w || !a->w_scale || !a->out)
    return noalloc_fail(WAM_E_ARG, "wam_matmul_fp4: null buffer");
  auto rows_ok = [](const void* p, int64_t stride, int rows, int64_t unit, int64_t n) {
    return aligned_to(p, unit) && (rows == 1 || (stride >= n && stride % unit == 0 && stride <= kMaxStride));
  };
  const int64_t kb = ((int64_t)a->K + kFp4Block - 1) / kFp4Block;
  if (!rows_ok(a->a, a->a_stride, a->M, 16, a->K / 2) || !rows_ok(a->w, a->w_stride, a->N, 16, a->K / 2))
    return noalloc_fail(WAM_E_ARG, "wam_matmul_fp4: a and w must start on 16 bytes, their rows apart and a multiple of 16 bytes");
  if (!rows_ok(a->a_scale, a->a_scale_stride, a->M, 4, kb) || !rows_ok(a->w_scale, a->w_scale_stride, a->N, 4, kb))
    return noalloc_fail(WAM_E_ARG, "wam_matmul_fp4: scales must start on 4 bytes, their rows apart and a multiple of 4 bytes");
  if (!aligned_to(a->bias, 4)) return noalloc_fail(WAM_E_ARG, "wam_matmul_fp4: bias must be aligned");
  const bool blocks = a->out_dtype == WAM_FP4;
  const int64_t esize = a->out_dtype == WAM_FP32 ? 4 : blocks ? 1 : 2;
  const int64_t row = blocks ? ((int64_t)a->N + 1) / 2 : a->N;
  if (!aligned_to(a->out, esize) || (a->M > 1 && (a->out_stride < row || a->out_stride > kMaxStride)))
    return noalloc_fail(WAM_E_ARG, "wam_matmul_fp4: rows of out must be distinct and aligned to their elements");
  if (blocks && (!a->out_scale || (a->M > 1 && (a->out_scale_stride < ((int64_t)a->N + kFp4Block - 1) / kFp4Block ||
                                                a->out_scale_stride > kMaxStride))))
    return noalloc_fail(WAM_E_ARG, "wam_matmul_fp4: out of WAM_FP4 needs out_scale with distinct rows");
  if (a->out == a->a || a->out == a->w || a->out == a->a_scale || a->out == a->w_scale)
    return noalloc_fail(WAM_E_ARG, "wam_matmul_fp4: out must not be an operand");
  if (blocks && (a->out_scale == a->a || a->out_scale == a->w || a->out_scale == a->a_scale ||
                 a->out_scale == a->w_scale || a->out_scale == a->out))
    return noalloc_fail(WAM_E_ARG, "wam_matmul_fp4: out_scale must be a buffer of its own");
  const gemm::Fp4Operands p{a->a, a->w, a->a_scale, a->w_scale, a->M > 1 ? a->a_stride : 0, a->N > 1 ? a->w_stride : 0,
                            a->M > 1 ? a->a_scale_stride : 0, a->N > 1 ? a->w_scale_stride : 0, a->M, a->N, a->K};
  const gemm::Fp8Out o{a->bias, a->out, a->M > 1 ? a->out_stride : 0, nullptr, a->M > 1 ? a->out_scale_stride : 0};
  const hipError_t e = launch_fp4(p, o, a->out_scale, a->out_dtype, a->act == WAM_ACT_GELU,
                                  static_cast<hipStream_t>(hip_stream));
  if (e == hipErrorInvalidConfiguration) return noalloc_fail(WAM_E_SHAPE, "wam_matmul_fp4: too many tiles for one launch");
  if (e != hipSuccess) return noalloc_fail(WAM_E_HIP, "wam_matmul_fp4: kernel launch failed");
  return WAM_OK;
}
