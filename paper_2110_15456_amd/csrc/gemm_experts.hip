// gemm_experts.hip -- dispatch of the products of experts over the operand
// formats, and the choice of their kernel and tile (kernels: gemm_mx.h,
// gemm_direct.h with SEG).
#include <math.h>

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

// What a product takes, in us, on the tiles there are.  The routing is device data,
// so the tiles of rows are those that slots spread over all experts would have, each
// expert's last one half full.  Fitted to graph replays of ten calls at 1 to 1024
// slots an expert, 4 to 128 experts of 256 x 256 to 4096 x 4096: over 288 products of up
// to 160 slots an expert the kernel taken is 4% slower than the fastest in the mean and
// 50% at worst, over 92 of more slots 1% and 32%.  What decided, us (few tokens on 16 and
// 32 rows, tiles of 128 x 128, large tiles):
//   8 x 2048 x 2048 (4,4)    4 slots   7.2   9.0   18   32     (6,6)  12     -   31  37
//                           24        11.4   9.6   19   31            18     -   31  37
//                           64        22    22     19   32            40     -   34  38
//                          512       170   142     46   41             -     -   97  84
//   64 x 1024 x 1024 (4,4)  64        60    50     18   25            79     -   42  47
//                          128       122    90     33   27             -     -   60  50
//                          256       186   140     47   53             -     -   96  80
struct Price {
  double few[2], small, big;  // few[0]: 16 rows, few[1]: 32
};
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Rounds of 128 x 128 tiles, and of the formats' large ones.
void price_tiles(const Operands& p, double rows128, double rows256, double slabs, Price& out) {
  const bool one = p.na == 1 && p.nb == 1, both4 = one && p.fa && p.fb, split2 = p.na == 2 && p.nb == 2;
  const double n128 = (double)ceil_div(p.N, 128), n256 = (double)ceil_div(p.N, 256);
  if (one) {
    // two workgroups of 128 x 128 share a CU, and take a quarter longer than alone
    const double w = rows128 * n128, full = floor(w / 512.0), rest = w - 512.0 * full;
    const double two = 1.25 * (4.7 + 1.19 * slabs), alone = 1.25 * (2.4 + 0.93 * slabs);
    out.small = (both4 ? 0.76 : 1.0) * (full * two + (rest <= 0.5 ? 0.0 : rest <= 256.0 ? alone : two));
    out.big = (both4 ? 0.92 : 1.0) * ceil(rows256 * n256 / 256.0) * (10.9 + 1.97 * slabs);
    return;
  }
  // the large tile of two planes on one side: 256 rows of the other
  const double wide = p.na == 1 ? rows256 * n128 : split2 && p.fa && p.fb ? rows256 * n128 : split2 ? rows128 * n128
                                                                                             : rows128 * n256;
  out.small = ceil(rows128 * n128 / 256.0) * (split2 ? 4.0 + 2.0 * slabs : 5.0 + 1.45 * slabs);
  out.big = ceil(wide / 256.0) * (split2 ? 7.0 + 2.2 * slabs : 8.0 + 1.8 * slabs);
}

// Tiles of T rows that `slots` slots of `experts` experts have.
double tiles_of_rows(double slots, double experts, int T) {
  const double busy = slots < experts ? slots : experts;
  return busy * (slots / busy / T < 0.5 ? 1.0 : slots / busy / T + 0.5);
}

Price price(const Operands& p, int experts, int64_t slots, int64_t K) {
  Price out{};
  const double s = (double)slots, slabs = (double)ceil_div(K / 16, mx::KG) * (K % 128 ? 1.15 : 1.0);
  price_tiles(p, tiles_of_rows(s, experts, 128), tiles_of_rows(s, experts, 256), slabs, out);
  // the few-token kernels: the weights, once for every tile of rows, and from the caches
  // the rows, once for every 16 columns, at rates in bytes per us
  auto bytes_of = [](int planes, bool narrow) {
    return (planes == 1 ? (narrow ? 4.0 : 6.0) : narrow ? 10.0 : 12.0) / 8.0 + 1.0 / 16.0;
  };
  const double values = (double)p.N * (double)K;
  const double weights = values * bytes_of(p.nb, p.fb), rows = s / 16.0 * values * bytes_of(p.na, p.fa);
  constexpr double rate = 5.5e6, rows_rate = 8.3e6;
  out.few[0] = 3.0 + tiles_of_rows(s, experts, 16) * weights / rate + rows / rows_rate;
  out.few[1] = p.na == 1 ? 3.0 + 1.3 * (tiles_of_rows(s, experts, 32) * weights / rate + rows / rows_rate) : 1e30;
  return out;
}

Operands operands(const uint8_t* a_mant, const uint8_t* a_exp, int a_m, int na, const uint8_t* b_mant,
                  const uint8_t* b_exp, int b_m, int nb, int64_t a_rows, int64_t b_rows, int64_t M, int64_t N, int64_t K,
                  int scale_log2) {
  return Operands{a_mant, a_exp, a_rows * (K / 16) * plane_group_bytes(16, a_m, 0), b_mant, b_exp,
                  b_rows * (K / 16) * plane_group_bytes(16, b_m, 0), (int)M, (int)N, (int)(K / 16), na, nb,
                  fmt_flag(a_m, na), fmt_flag(b_m, nb), ldexpf(1.0f, scale_log2)};
}

ExpertsRoute route_rows(const Operands& p, int experts, int64_t slots, int64_t K) {
  const Segments seg{nullptr, experts, (int)slots};
  const Price us = price(p, experts, slots, K);
  const double tiled = us.small < us.big ? us.small : us.big;
  for (int rm = 1; rm <= 2; ++rm) {
    const int64_t rows = most_segment_tiles(seg, 16 * rm);
    if (us.few[rm - 1] > tiled || us.few[rm - 1] > us.few[2 - rm] || rows > direct::kMaxRowTiles) continue;
    const int64_t cols = ceil_div(p.N, direct_experts_cols(p.na, p.nb, rm)), pairs = ceil_div(K / 16, 32);
    // waves for a tile: until every CU has eight
    int kw = 1;
    while (kw < direct::kExpertWaves && rows * cols * kw < 2048 && 2 * kw <= pairs) kw *= 2;
    const int64_t each = rows * cols * kw / (512 * direct::kExpertWaves);
    return ExpertsRoute{16 * rm, kw, each < 1 ? 1 : each > 4 ? 4 : (int)each};
  }
  return ExpertsRoute{us.small <= us.big ? 128 : 0, 0, 0};
}

ExpertsRoute route_grad(const Operands& p, int experts, int64_t M, int64_t klen) {
  // (the tiles of every expert, at the mean length of K)
  Price us{};
  price_tiles(p, (double)(experts * ceil_div(M, 128)), (double)(experts * ceil_div(M, 256)),
              (double)klen / 128.0 / experts, us);
  return ExpertsRoute{us.small <= us.big ? 128 : 0, 0, 0};
}

}  // namespace

ExpertsRoute experts_route(int a_m, int na, int b_m, int nb, int experts, int64_t slots, int64_t N, int64_t K) {
  return route_rows(operands(nullptr, nullptr, a_m, na, nullptr, nullptr, b_m, nb, slots, experts * N, slots, N, K, 0),
                    experts, slots, K);
}

ExpertsRoute experts_grad_route(int a_m, int na, int b_m, int nb, int experts, int64_t M, int64_t N, int64_t klen) {
  return route_grad(operands(nullptr, nullptr, a_m, na, nullptr, nullptr, b_m, nb, M, N, M, N, klen, 0), experts, M,
                    klen);
}

hipError_t launch_gemm_experts(const uint8_t* a_mant, const uint8_t* a_exp, int a_m, int na, const uint8_t* b_mant,
                               const uint8_t* b_exp, int b_m, int nb, const int32_t* offsets, int experts,
                               int64_t slots, int64_t N, int64_t K, int scale_log2, float* C, int64_t ldc,
                               hipStream_t s) {
  if (slots == 0 || N == 0) return hipSuccess;
  const Operands p = operands(a_mant, a_exp, a_m, na, b_mant, b_exp, b_m, nb, slots, experts * N, slots, N, K, scale_log2);
  const Segments seg{offsets, experts, (int)slots};
  const ExpertsRoute r = route_rows(p, experts, slots, K);
  if (r.waves > 0) return run_direct(p, r.rows / 16, r.waves, r.each, C, ldc, seg, s);
  return run_tiled(p, r.rows == 128, false, C, ldc, seg, s);
}

hipError_t launch_gemm_experts_grad(const uint8_t* a_mant, const uint8_t* a_exp, int a_m, int na, const uint8_t* b_mant,
                                    const uint8_t* b_exp, int b_m, int nb, const int32_t* k_offsets, int experts,
                                    int64_t M, int64_t N, int64_t klen, int scale_log2, float* C, hipStream_t s) {
  if (M == 0 || N == 0) return hipSuccess;
  const Operands p = operands(a_mant, a_exp, a_m, na, b_mant, b_exp, b_m, nb, M, N, M, N, klen, scale_log2);
  const Segments seg{k_offsets, experts, (int)klen};
  return run_tiled(p, route_grad(p, experts, M, klen).rows == 128, true, C, N, seg, s);
}

}  // namespace fastbfp
