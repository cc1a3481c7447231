// gemm_experts.hip -- dispatch of the products of experts over the operand
// formats, and the choice of their kernel and tile (kernels: gemm_mx.h,
// gemm_direct.h with SEG).
#include "gemm_direct.h"
#include "gemm_mx.h"

namespace fastbfp {

FASTBFP_MX_EXPERTS_ALL(FASTBFP_MX_EXPERTS_DECLARE, 1, 1)
FASTBFP_MX_EXPERTS_ALL(FASTBFP_MX_EXPERTS_DECLARE, 1, 2)
FASTBFP_MX_EXPERTS_ALL(FASTBFP_MX_EXPERTS_DECLARE, 2, 1)
FASTBFP_MX_EXPERTS_ALL(FASTBFP_MX_EXPERTS_DECLARE, 2, 2)
FASTBFP_DIRECT_EXPERTS_ALL(FASTBFP_DIRECT_EXPERTS_DECLARE, 1, 1)
FASTBFP_DIRECT_EXPERTS_ALL(FASTBFP_DIRECT_EXPERTS_DECLARE, 1, 2)
FASTBFP_DIRECT_EXPERTS_ALL(FASTBFP_DIRECT_EXPERTS_DECLARE, 2, 1)
FASTBFP_DIRECT_EXPERTS_ALL(FASTBFP_DIRECT_EXPERTS_DECLARE, 2, 2)

namespace {

struct Operands {
  const uint8_t *a_mant, *a_exp;
  int64_t a_ps;
  const uint8_t *b_mant, *b_exp;
  int64_t b_ps;
  int M, N, ng;
  int na, nb, fa, fb;
  float scale;
};

int fmt_flag(int m, int planes) { return planes == 1 ? plane0_fp4(m) : m <= 6; }

// Calls f(ic<FA>{}, ic<FB>{}) for the operands' formats.
template <class F>
hipError_t with_formats(const Operands& p, F f) {
  if (!p.fa && !p.fb) return f(ic<0>{}, ic<0>{});
  if (!p.fa) return f(ic<0>{}, ic<1>{});
  if (!p.fb) return f(ic<1>{}, ic<0>{});
  return f(ic<1>{}, ic<1>{});
}
template <class F>
hipError_t with_operands(const Operands& p, F f) {
  return with_formats(p, [&](auto fa, auto fb) {
    if (p.na == 1 && p.nb == 1) return f(ic<1>{}, ic<1>{}, fa, fb);
    if (p.na == 1) return f(ic<1>{}, ic<2>{}, fa, fb);
    if (p.nb == 1) return f(ic<2>{}, ic<1>{}, fa, fb);
    return f(ic<2>{}, ic<2>{}, fa, fb);
  });
}

hipError_t run_tiled(const Operands& p, bool small, bool k_segments, float* C, int64_t ldc, const Segments& seg,
                     hipStream_t s) {
  return with_operands(p, [&](auto na, auto nb, auto fa, auto fb) {
    return launch_mx_experts_t<decltype(na)::value, decltype(nb)::value, decltype(fa)::value, decltype(fb)::value>(
        small, k_segments, p.a_mant, p.a_exp, p.a_ps, p.b_mant, p.b_exp, p.b_ps, p.M, p.N, p.ng, p.scale, C, ldc, seg, s);
  });
}

hipError_t run_direct(const Operands& p, int rm, int kw, int each, float* C, int64_t ldc, const Segments& seg, hipStream_t s) {
  return with_operands(p, [&](auto na, auto nb, auto fa, auto fb) {
    return launch_direct_experts_t<decltype(na)::value, decltype(nb)::value, decltype(fa)::value, decltype(fb)::value>(
        rm, kw, each, p.a_mant, p.a_exp, p.a_ps, p.b_mant, p.b_exp, p.b_ps, p.N, p.ng, p.scale, C, ldc, seg, s);
  });
}

}  // namespace

hipError_t launch_gemm_experts(const uint8_t* a_mant, const uint8_t* a_exp, int a_m, int na, const uint8_t* b_mant,
                               const uint8_t* b_exp, int b_m, int nb, const int32_t* offsets, int experts,
                               int64_t slots, int64_t N, int64_t K, int scale_log2, float* C, int64_t ldc,
                               hipStream_t s) {
  if (slots == 0 || N == 0) return hipSuccess;
  const Operands p{a_mant, a_exp, slots * (K / 16) * plane_group_bytes(16, a_m, 0), b_mant, b_exp,
                   experts * N * (K / 16) * plane_group_bytes(16, b_m, 0), (int)slots, (int)N, (int)(K / 16), na, nb,
                   fmt_flag(a_m, na), fmt_flag(b_m, nb), ldexpf(1.0f, scale_log2)};
  const Segments seg{offsets, experts, (int)slots};
  const int64_t mean = slots / experts;
  for (int rm = 1; rm <= (na == 1 ? 2 : 1); ++rm) {
    const int64_t rows = most_segment_tiles(seg, 16 * rm);
    if (mean > 16 * rm || rows > direct::kMaxRowTiles) continue;
    const int wide = direct_experts_cols(na, nb, rm);
    const int64_t cols = (N + wide - 1) / wide, pairs = (K / 16 + 31) / 32;
    // waves for a tile: until every CU has eight
    int kw = 1;
    while (kw < direct::kExpertWaves && rows * cols * kw < 2048 && 2 * kw <= pairs) kw *= 2;
    const int64_t each = rows * cols * kw / (512 * direct::kExpertWaves);
    return run_direct(p, rm, kw, each < 1 ? 1 : each > 8 ? 8 : (int)each, C, ldc, seg, s);
  }
  return run_tiled(p, mean < 512, false, C, ldc, seg, s);
}

hipError_t launch_gemm_experts_grad(const uint8_t* a_mant, const uint8_t* a_exp, int a_m, int na, const uint8_t* b_mant,
                                    const uint8_t* b_exp, int b_m, int nb, const int32_t* k_offsets, int experts,
                                    int64_t M, int64_t N, int64_t klen, int scale_log2, float* C, hipStream_t s) {
  if (M == 0 || N == 0) return hipSuccess;
  const Operands p{a_mant, a_exp, M * (klen / 16) * plane_group_bytes(16, a_m, 0), b_mant, b_exp,
                   N * (klen / 16) * plane_group_bytes(16, b_m, 0), (int)M, (int)N, (int)(klen / 16), na, nb,
                   fmt_flag(a_m, na), fmt_flag(b_m, nb), ldexpf(1.0f, scale_log2)};
  const Segments seg{k_offsets, experts, (int)klen};
  const int64_t tiles = (M + 255) / 256 * ((N + 255) / 256) * experts;
  return run_tiled(p, tiles < 256, true, C, N, seg, s);
}

}  // namespace fastbfp
