// api_layer.cpp -- the C ABI of the 8-bit blocks, the norm and the gradients' scaling
// (include/fastbfp.h): argument validation on the host, then launches on the caller's
// stream.
#include <hip/hip_runtime.h>

#include <math.h>

#include <algorithm>
#include <new>

#include "checks.h"
#include "fp8.h"
#include "launch.h"

using fastbfp::aligned;
using fastbfp::overlap;
using fastbfp::status_of;

namespace {

using fastbfp::fp8::code_pitch;
using fastbfp::fp8::exp_pitch;

constexpr int64_t kMost = int64_t(1) << 23;  // of a row's values: 256 rows of codes within 2^31 bytes
constexpr int64_t kGrid = 0x7fffffff;
using fastbfp::kMostThreads;

bool type_ok(int t) { return t == BFP_F32 || t == BFP_BF16; }
uint64_t bytes_of(int t) { return t == BFP_F32 ? 4 : 2; }

bool format_ok(int f) { return f == BFP_FP8_E4M3 || f == BFP_FP8_E5M2; }

int check_fp8(int64_t rows, int64_t len, int format) {
  if (rows < 0 || len < 0 || !format_ok(format)) return BFP_E_ARG;
  if (len > kMost || rows > (int64_t(1) << 40)) return BFP_E_UNSUPPORTED;
  return BFP_OK;
}

// The tensors of a conversion: x [R][C] and up to two outputs.
uint64_t code_bytes(int64_t rows, int64_t len) { return (uint64_t)rows * (uint64_t)code_pitch(len); }
uint64_t exp_bytes(int64_t rows, int64_t len) { return (uint64_t)rows * (uint64_t)exp_pitch(len); }

bool codes_ok(const uint8_t* codes, const uint8_t* exps) {
  return codes && exps && aligned(codes, 16) && aligned(exps, 4);
}

int check_product(int64_t M, int64_t N, int64_t K) {
  if (M < 0 || N < 0 || K < 0) return BFP_E_ARG;
  if (K > kMost || M > kGrid || N > kGrid) return BFP_E_UNSUPPORTED;
  if (((M + 63) / 64) * ((N + 63) / 64) > kGrid / 64 || (K == 0 && N > 0 && M > kMostThreads / N)) return BFP_E_UNSUPPORTED;
  return BFP_OK;
}

int check_norm(int64_t rows, int64_t d) {
  if (rows < 0 || d < 0) return BFP_E_ARG;
  if (d > fastbfp::kMaxNorm || rows > kMostThreads / fastbfp::rms_norm_threads(d)) return BFP_E_UNSUPPORTED;
  return BFP_OK;
}

// The arguments that the norms share; BFP_OK also where there is nothing to do.
int check_norm_args(const void* x, int x_type, const float* residual, const float* w, int64_t rows, int64_t d, double eps,
                    const float* h, const float* rstd) {
  const int st = check_norm(rows, d);
  if (st != BFP_OK) return st;
  if (!type_ok(x_type) || !(eps >= 0.0) || isinf(eps)) return BFP_E_ARG;
  if (rows == 0 || d == 0) return BFP_OK;
  if (!x || !w || !aligned(x, bytes_of(x_type)) || !aligned(residual, 4) || !aligned(w, 4) || !aligned(h, 4) || !aligned(rstd, 4))
    return BFP_E_ARG;
  // h may be x or the residual itself (a row's values are read before any is written)
  const uint64_t n = (uint64_t)rows * d * 4, xn = (uint64_t)rows * d * bytes_of(x_type);
  if (((h != x || x_type != BFP_F32) && overlap(h, n, x, xn)) || (h != residual && overlap(h, n, residual, n)) || overlap(h, n, w, d * 4) ||
      overlap(h, n, rstd, rows * 4) || overlap(rstd, rows * 4, x, xn) || overlap(rstd, rows * 4, residual, n) ||
      overlap(rstd, rows * 4, w, d * 4))
    return BFP_E_ARG;
  return BFP_OK;
}

// Whether an output shares bytes with what a norm reads or also writes.
bool norm_overlap(const void* o, uint64_t bytes, const void* x, int x_type, const float* residual, const float* w, int64_t rows,
                  int64_t d, const float* h, const float* rstd) {
  const uint64_t n = (uint64_t)rows * d * 4;
  return overlap(o, bytes, x, (uint64_t)rows * d * bytes_of(x_type)) || overlap(o, bytes, residual, n) || overlap(o, bytes, w, d * 4) ||
         overlap(o, bytes, h, n) || overlap(o, bytes, rstd, rows * 4);
}

int check_sizes(const int64_t* sizes, int64_t count) {
  if (count < 0 || (count > 0 && !sizes)) return BFP_E_ARG;
  if (count > (int64_t(1) << 24)) return BFP_E_UNSUPPORTED;
  int64_t total = 0;
  for (int64_t i = 0; i < count; ++i) {
    if (sizes[i] < 0) return BFP_E_ARG;
    if (sizes[i] > (int64_t(1) << 42) || (total += sizes[i]) > (int64_t(1) << 42)) return BFP_E_UNSUPPORTED;
  }
  return BFP_OK;
}

int check_list(const void* const* tensors, int type, const int64_t* sizes, int64_t count) {
  if (!type_ok(type) || count < 0 || (count > 0 && (!tensors || !sizes))) return BFP_E_ARG;
  for (int64_t i = 0; i < count; ++i)
    if (sizes[i] > 0 && (!tensors[i] || !aligned(tensors[i], bytes_of(type)))) return BFP_E_ARG;
  return check_sizes(sizes, count);
}

struct Span {
  uintptr_t begin, end;
};
bool before(const Span& a, const Span& b) { return a.begin < b.begin; }

// Whether no output of a list shares bytes with another one, or with an input that is not
// that output itself (pieces of a launch run in any order).  BFP_OK if so.
int check_apart(const void* const* in, void* const* out, uint64_t bytes, const int64_t* sizes, int64_t count) {
  // (outputs one behind another, as in a bucket, all apart from all inputs: no sort)
  uintptr_t last = 0, in_lo = UINTPTR_MAX, in_hi = 0, out_lo = UINTPTR_MAX;
  bool ordered = true;
  int64_t n = 0;
  for (int64_t i = 0; i < count; ++i) {
    if (sizes[i] == 0) continue;
    const uintptr_t p = reinterpret_cast<uintptr_t>(in[i]), q = reinterpret_cast<uintptr_t>(out[i]), b = sizes[i] * bytes;
    ordered = ordered && q >= last;
    last = q + b;
    in_lo = std::min(in_lo, p), in_hi = std::max(in_hi, p + b), out_lo = std::min(out_lo, q);
    ++n;
  }
  if (n == 0 || (ordered && (in_hi <= out_lo || last <= in_lo))) return BFP_OK;
  Span* spans = new (std::nothrow) Span[n];
  if (!spans) return BFP_E_UNSUPPORTED;
  int64_t k = 0;
  for (int64_t i = 0; i < count; ++i)
    if (sizes[i] > 0) spans[k] = {reinterpret_cast<uintptr_t>(out[i]), 0}, spans[k].end = spans[k].begin + sizes[i] * bytes, ++k;
  if (!ordered) std::sort(spans, spans + n, before);
  bool apart = true;
  for (int64_t i = 1; i < n; ++i) apart = apart && spans[i - 1].end <= spans[i].begin;
  for (int64_t i = 0; apart && i < count; ++i) {
    if (sizes[i] == 0 || in[i] == out[i]) continue;  // (its own output, which meets no other)
    const uintptr_t p = reinterpret_cast<uintptr_t>(in[i]);
    const Span s{p, p + sizes[i] * bytes};
    const Span* at = std::lower_bound(spans, spans + n, s, before);  // the first output from s.begin on
    if ((at < spans + n && at->begin < s.end) || (at > spans && (at - 1)->end > s.begin)) apart = false;
  }
  delete[] spans;
  return apart ? BFP_OK : BFP_E_ARG;
}

}  // namespace

extern "C" {

int bfp_fp8_sizes(int64_t rows, int64_t len, size_t* code_bytes_out, size_t* exp_bytes_out) {
  const int st = check_fp8(rows, len, BFP_FP8_E4M3);
  if (st != BFP_OK) return st;
  if (!code_bytes_out || !exp_bytes_out) return BFP_E_ARG;
  *code_bytes_out = code_bytes(rows, len);
  *exp_bytes_out = exp_bytes(rows, len);
  return BFP_OK;
}

int bfp_quantize_fp8(const void* x, int x_type, int64_t R, int64_t C, int group_axis, int format, uint8_t* codes, uint8_t* exp,
                     uint32_t* status_word, void* stream) {
  if ((group_axis != 0 && group_axis != 1) || !type_ok(x_type)) return BFP_E_ARG;
  const int64_t rows = group_axis == 1 ? R : C, len = group_axis == 1 ? C : R;
  const int st = check_fp8(rows, len, format);
  if (st != BFP_OK) return st;
  if (rows == 0 || len == 0) return BFP_OK;
  if (!x || !aligned(x, bytes_of(x_type)) || !codes_ok(codes, exp) || !aligned(status_word, 4)) return BFP_E_ARG;
  const int64_t quads = (fastbfp::fp8::blocks_of(len) + 3) / 4;
  if (group_axis == 1 ? R > kMostThreads / 32 / quads
                      : fastbfp::fp8::blocks_of(C) > kMostThreads / 256 / fastbfp::fp8::blocks_of(R))
    return BFP_E_UNSUPPORTED;
  const uint64_t n = (uint64_t)R * C * bytes_of(x_type), cb = code_bytes(rows, len), eb = exp_bytes(rows, len);
  if (overlap(codes, cb, x, n) || overlap(exp, eb, x, n) || overlap(codes, cb, exp, eb)) return BFP_E_ARG;
  return status_of(fastbfp::launch_quantize_fp8(x, x_type == BFP_BF16, R, C, group_axis, format, codes, exp, status_word,
                                                static_cast<hipStream_t>(stream)));
}

int bfp_quantize_fp8_dual(const void* x, int x_type, int64_t R, int64_t C, int format, uint8_t* codes_r, uint8_t* exp_r,
                          uint8_t* codes_c, uint8_t* exp_c, uint32_t* status_word, void* stream) {
  if (!type_ok(x_type)) return BFP_E_ARG;
  int st = check_fp8(R, C, format);
  if (st == BFP_OK) st = check_fp8(C, R, format);
  if (st != BFP_OK) return st;
  if (R == 0 || C == 0) return BFP_OK;
  if (!x || !aligned(x, bytes_of(x_type)) || !codes_ok(codes_r, exp_r) || !codes_ok(codes_c, exp_c) || !aligned(status_word, 4))
    return BFP_E_ARG;
  if (fastbfp::fp8::blocks_of(C) > kMostThreads / 256 / fastbfp::fp8::blocks_of(R)) return BFP_E_UNSUPPORTED;
  const uint64_t n = (uint64_t)R * C * bytes_of(x_type);
  const void* o[4] = {codes_r, exp_r, codes_c, exp_c};
  const uint64_t b[4] = {code_bytes(R, C), exp_bytes(R, C), code_bytes(C, R), exp_bytes(C, R)};
  for (int i = 0; i < 4; ++i) {
    if (overlap(o[i], b[i], x, n)) return BFP_E_ARG;
    for (int j = 0; j < i; ++j)
      if (overlap(o[i], b[i], o[j], b[j])) return BFP_E_ARG;
  }
  return status_of(fastbfp::launch_quantize_fp8_dual(x, x_type == BFP_BF16, R, C, format, codes_r, exp_r, codes_c, exp_c, status_word,
                                                     static_cast<hipStream_t>(stream)));
}

int bfp_dequantize_fp8(const uint8_t* codes, const uint8_t* exp, int64_t rows, int64_t len, int format, float* y,
                       void* stream) {
  const int st = check_fp8(rows, len, format);
  if (st != BFP_OK) return st;
  if (rows == 0 || len == 0) return BFP_OK;
  if (!codes_ok(codes, exp) || !y || !aligned(y, 4)) return BFP_E_ARG;
  if (rows > kMostThreads / ((len + 3) / 4)) return BFP_E_UNSUPPORTED;
  const uint64_t n = (uint64_t)rows * len * 4;
  if (overlap(y, n, codes, code_bytes(rows, len)) || overlap(y, n, exp, exp_bytes(rows, len))) return BFP_E_ARG;
  return status_of(
      fastbfp::launch_dequantize_fp8(codes, exp, rows, len, format, y, static_cast<hipStream_t>(stream)));
}

int bfp_gemm_fp8_ws_size(int64_t M, int64_t N, int64_t K, size_t* workspace_bytes) {
  const int st = check_product(M, N, K);
  if (st != BFP_OK) return st;
  if (!workspace_bytes) return BFP_E_ARG;
  *workspace_bytes = M && N && K ? (size_t)fastbfp::fp8_plan_ws(fastbfp::fp8_plan(M, N, K, true), M, N) : 0;
  return BFP_OK;
}

int bfp_gemm_fp8_route(int64_t M, int64_t N, int64_t K, size_t workspace_bytes, int* rows, int* cols, int* waves,
                       int* parts) {
  const int st = check_product(M, N, K);
  if (st != BFP_OK) return st;
  if (!rows || !cols || !waves || !parts || M == 0 || N == 0 || K == 0) return BFP_E_ARG;
  fastbfp::Fp8Plan plan = fastbfp::fp8_plan(M, N, K, true);
  if ((int64_t)workspace_bytes < fastbfp::fp8_plan_ws(plan, M, N)) plan = fastbfp::fp8_plan(M, N, K, false);
  *rows = plan.rows, *cols = plan.cols;
  *waves = plan.waves;
  *parts = plan.parts;
  return BFP_OK;
}

int bfp_gemm_fp8(const uint8_t* a_codes, const uint8_t* a_exp, int a_format, const uint8_t* b_codes,
                 const uint8_t* b_exp, int b_format, int64_t M, int64_t N, int64_t K, void* C, int c_type,
                 int64_t ldc, void* workspace, size_t workspace_bytes, void* stream) {
  if (!format_ok(a_format) || !format_ok(b_format) || !type_ok(c_type)) return BFP_E_ARG;
  const int st = check_product(M, N, K);
  if (st != BFP_OK) return st;
  if (ldc < N) return BFP_E_SHAPE;
  if (M == 0 || N == 0) return BFP_OK;
  if (!C || !aligned(C, bytes_of(c_type)) || (K > 0 && (!codes_ok(a_codes, a_exp) || !codes_ok(b_codes, b_exp)))) return BFP_E_ARG;
  const uint64_t cb = ((uint64_t)(M - 1) * ldc + N) * bytes_of(c_type);
  const void* in[4] = {a_codes, a_exp, b_codes, b_exp};
  const uint64_t n[4] = {code_bytes(M, K), exp_bytes(M, K), code_bytes(N, K), exp_bytes(N, K)};
  for (int i = 0; i < 4; ++i)
    if (overlap(C, cb, in[i], n[i])) return BFP_E_ARG;
  fastbfp::Fp8Plan plan = fastbfp::fp8_plan(M, N, K, true);
  const uint64_t need = (uint64_t)fastbfp::fp8_plan_ws(plan, M, N);
  if (need > 0) {
    if (!workspace || workspace_bytes < need) {
      plan = fastbfp::fp8_plan(M, N, K, false);
    } else {
      if (!aligned(workspace, 16) || overlap(workspace, need, C, cb)) return BFP_E_ARG;
      for (int i = 0; i < 4; ++i)
        if (overlap(workspace, need, in[i], n[i])) return BFP_E_ARG;
    }
  }
  return status_of(fastbfp::launch_gemm_fp8(plan, a_codes, a_exp, a_format, b_codes, b_exp, b_format, M, N, K, C,
                                            c_type == BFP_BF16, ldc, static_cast<float*>(workspace), static_cast<hipStream_t>(stream)));
}

int bfp_rms_norm(const void* x, int x_type, const float* residual, const float* weight, int64_t rows, int64_t d, double eps,
                 float* h, float* rstd, float* y, void* stream) {
  const int st = check_norm_args(x, x_type, residual, weight, rows, d, eps, h, rstd);
  if (st != BFP_OK || rows == 0 || d == 0) return st;
  if (!y || !aligned(y, 4)) return BFP_E_ARG;
  // (y may be x or the residual, where h is not: a row is read before it is written)
  const uint64_t n = (uint64_t)rows * d * 4;
  if (((y != x || x_type != BFP_F32) && overlap(y, n, x, (uint64_t)rows * d * bytes_of(x_type))) || (y != residual && overlap(y, n, residual, n)) || overlap(y, n, weight, d * 4) ||
      overlap(y, n, h, n) || overlap(y, n, rstd, rows * 4))
    return BFP_E_ARG;
  return status_of(fastbfp::launch_rms_norm(x, x_type == BFP_BF16, residual, weight, rows, d, eps, h, rstd, y,
                                            static_cast<hipStream_t>(stream)));
}

int bfp_rms_norm_fp8(const void* x, int x_type, const float* residual, const float* weight, int64_t rows, int64_t d, double eps,
                     float* h, float* rstd, int format, uint8_t* codes, uint8_t* exp, uint32_t* status_word,
                     void* stream) {
  if (!format_ok(format)) return BFP_E_ARG;
  const int st = check_norm_args(x, x_type, residual, weight, rows, d, eps, h, rstd);
  if (st != BFP_OK || rows == 0 || d == 0) return st;
  if (!codes_ok(codes, exp) || !aligned(status_word, 4)) return BFP_E_ARG;
  const uint64_t cb = code_bytes(rows, d), eb = exp_bytes(rows, d);
  if (norm_overlap(codes, cb, x, x_type, residual, weight, rows, d, h, rstd) ||
      norm_overlap(exp, eb, x, x_type, residual, weight, rows, d, h, rstd) || overlap(codes, cb, exp, eb))
    return BFP_E_ARG;
  return status_of(fastbfp::launch_rms_norm_fp8(x, x_type == BFP_BF16, residual, weight, rows, d, eps, h, rstd, format, codes, exp,
                                                status_word, static_cast<hipStream_t>(stream)));
}

int bfp_rms_norm_bfp(const void* x, int x_type, const float* residual, const float* weight, int64_t rows, int64_t d, double eps,
                     float* h, float* rstd, int m_bits, int round_mode, uint64_t seed, uint8_t* mant, uint8_t* exp,
                     uint32_t* status_word, void* stream) {
  if (round_mode < BFP_ROUND_NEAREST || round_mode > BFP_ROUND_TRUNCATE) return BFP_E_ARG;
  const int st = check_norm_args(x, x_type, residual, weight, rows, d, eps, h, rstd);
  if (st != BFP_OK) return st;
  if (m_bits < 1 || m_bits > 8) return BFP_E_PRECISION;
  if (d % 16 != 0) return BFP_E_SHAPE;
  if (rows == 0 || d == 0) return BFP_OK;
  if (!mant || !exp || !aligned(mant, 4) || !aligned(status_word, 4)) return BFP_E_ARG;
  const uint64_t groups = (uint64_t)rows * (d / 16), eb = groups;
  uint64_t mb = groups * fastbfp::plane_group_bytes(16, m_bits, 0);
  if (m_bits > 4) mb += groups * fastbfp::plane_group_bytes(16, m_bits, 1);
  if (norm_overlap(mant, mb, x, x_type, residual, weight, rows, d, h, rstd) ||
      norm_overlap(exp, eb, x, x_type, residual, weight, rows, d, h, rstd) || overlap(mant, mb, exp, eb))
    return BFP_E_ARG;
  return status_of(fastbfp::launch_rms_norm_bfp(x, x_type == BFP_BF16, residual, weight, rows, d, eps, h, rstd, m_bits, round_mode, seed,
                                                mant, exp, status_word, static_cast<hipStream_t>(stream)));
}

int bfp_rms_norm_grad_ws_size(int64_t rows, int64_t d, size_t* workspace_bytes) {
  const int st = check_norm(rows, d);
  if (st != BFP_OK) return st;
  if (!workspace_bytes) return BFP_E_ARG;
  *workspace_bytes = (size_t)fastbfp::rms_norm_grad_parts(rows, d) * d * 4;
  return BFP_OK;
}

int bfp_rms_norm_grad(const void* dy, int dy_type, const float* h, const float* rstd, const float* weight, const float* dresidual,
                      int64_t rows, int64_t d, float* dx, float* dweight, void* workspace, size_t workspace_bytes,
                      void* stream) {
  const int st = check_norm(rows, d);
  if (st != BFP_OK || d == 0) return st;
  if (!type_ok(dy_type) || !dweight || !aligned(dweight, 4)) return BFP_E_ARG;
  const uint64_t n = (uint64_t)rows * d * 4, need = (uint64_t)fastbfp::rms_norm_grad_parts(rows, d) * d * 4;
  if (rows > 0) {
    if (!dy || !h || !rstd || !weight || !dx || !workspace || workspace_bytes < need) return BFP_E_ARG;
    if (!aligned(dy, bytes_of(dy_type)) || !aligned(h, 4) || !aligned(rstd, 4) || !aligned(weight, 4) || !aligned(dresidual, 4) ||
        !aligned(dx, 4) || !aligned(workspace, 4))
      return BFP_E_ARG;
    // dx may be dy or dresidual itself (a row's values are read before any is written)
    const uint64_t yn = (uint64_t)rows * d * bytes_of(dy_type);
    if (((dx != dy || dy_type != BFP_F32) && overlap(dx, n, dy, yn)) || (dx != dresidual && overlap(dx, n, dresidual, n))) return BFP_E_ARG;
    const void* in[6] = {dy, h, rstd, weight, dresidual, dx};
    const uint64_t b[6] = {yn, n, (uint64_t)rows * 4, (uint64_t)d * 4, n, n};
    for (int i = 0; i < 6; ++i)
      if (overlap(dweight, d * 4, in[i], b[i]) || overlap(workspace, need, in[i], b[i]) ||
          (i >= 1 && i <= 3 && overlap(dx, n, in[i], b[i])))
        return BFP_E_ARG;
    if (overlap(workspace, need, dweight, d * 4)) return BFP_E_ARG;
  }
  return status_of(fastbfp::launch_rms_norm_grad(dy, dy_type == BFP_BF16, h, rstd, weight, dresidual, rows, d, dx, dweight,
                                                 static_cast<float*>(workspace), static_cast<hipStream_t>(stream)));
}

int bfp_sum_squares_ws_size(const int64_t* sizes, int64_t count, size_t* workspace_bytes) {
  const int st = check_sizes(sizes, count);
  if (st != BFP_OK) return st;
  if (!workspace_bytes) return BFP_E_ARG;
  *workspace_bytes = (size_t)fastbfp::gradient_pieces(sizes, count) * sizeof(double);
  return BFP_OK;
}

int bfp_sum_squares(const void* const* tensors, int type, const int64_t* sizes, int64_t count, double* sumsq, void* workspace,
                    size_t workspace_bytes, void* stream) {
  const int st = check_list(tensors, type, sizes, count);
  if (st != BFP_OK) return st;
  if (!aligned(sumsq, 8)) return BFP_E_ARG;
  const uint64_t need = (uint64_t)fastbfp::gradient_pieces(sizes, count) * sizeof(double);
  if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 8))) return BFP_E_ARG;
  if (overlap(sumsq, 8, workspace, need)) return BFP_E_ARG;
  for (int64_t i = 0; i < count; ++i)
    if (overlap(sumsq, 8, tensors[i], sizes[i] * bytes_of(type)) ||
        overlap(workspace, need, tensors[i], sizes[i] * bytes_of(type)))
      return BFP_E_ARG;
  return status_of(fastbfp::launch_sum_squares(tensors, type == BFP_BF16, sizes, count, sumsq, static_cast<double*>(workspace),
                                               static_cast<hipStream_t>(stream)));
}

int bfp_clip_gradients(const void* const* tensors, void* const* out, int type, const int64_t* sizes, int64_t count,
                       double max_norm, const double* sumsq, int64_t sums, double* norm, void* stream) {
  int st = check_list(tensors, type, sizes, count);
  if (st == BFP_OK) st = check_list(const_cast<const void* const*>(out), type, sizes, count);
  if (st != BFP_OK) return st;
  if (!(max_norm >= 0.0) || !sumsq || !norm || !aligned(sumsq, 8) || !aligned(norm, 8)) return BFP_E_ARG;
  if (sums < 1) return BFP_E_ARG;
  if (sums > fastbfp::kMostSums) return BFP_E_UNSUPPORTED;
  const uint64_t sb = (uint64_t)sums * 8;
  if (overlap(sumsq, sb, norm, 8)) return BFP_E_ARG;
  for (int64_t i = 0; i < count; ++i) {
    const uint64_t n = sizes[i] * bytes_of(type);
    if (overlap(out[i], n, sumsq, sb) || overlap(out[i], n, norm, 8) || overlap(norm, 8, tensors[i], n)) return BFP_E_ARG;
  }
  st = check_apart(tensors, out, bytes_of(type), sizes, count);
  if (st != BFP_OK) return st;
  return status_of(fastbfp::launch_scale_gradients(tensors, out, type == BFP_BF16, sizes, count, max_norm, sumsq,
                                                   (int)sums, norm, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
