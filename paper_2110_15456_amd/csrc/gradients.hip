// gradients.hip -- the sum of squares over a list of FP32 or BF16 tensors and their scaling down
// to a largest norm.  Squares and sums are 64 bits (a square of FP32 is exact there, and
// none is out of range), so the norm is right for any values and any number of them.
// HBM-bound: every value read once for the norm, and read and written once for the scaling.
//
// A launch takes up to kTensors tensors from its arguments (no table to copy to the
// card).  Work is pieces of kPiece values; a workgroup finds its piece's tensor in the
// list of their first pieces.
#include "launch.h"

#include "fp8.h"

namespace fastbfp {

namespace grads {

using fp8::load4;
using fp8::store4;
using fp8::u4;

constexpr int kTensors = 120, kPiece = 16384;

struct List {
  const void* in[kTensors];
  void* out[kTensors];
  int64_t size[kTensors];
  uint32_t first[kTensors + 1];  // piece of each tensor's start
  int count;
};

__device__ __forceinline__ int find(const List& l, uint32_t piece) {
  int lo = 0, hi = l.count;  // first[lo] <= piece < first[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (l.first[mid] <= piece) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Sum over 256 threads, in a fixed order, in all of them.
__device__ __forceinline__ double block_sum(double v) {
  __shared__ double red[4];
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

// part[piece] = the sum of squares of a piece.
template <class T>
__global__ __launch_bounds__(256) void k_squares(List l, double* __restrict__ part) {
  const int i = find(l, blockIdx.x);
  const int64_t at = (int64_t)(blockIdx.x - l.first[i]) * kPiece, n = l.size[i] - at;
  const T* x = static_cast<const T*>(l.in[i]) + at;
  double sum = 0.0;
#pragma unroll 4
  for (int k = 0; k < kPiece / 1024; ++k) {
    const int64_t c = 4 * (threadIdx.x + 256 * k);
    const u4 v = load4(x + c, n - c);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const double a = (double)__uint_as_float(v[t]);
      sum = __builtin_fma(a, a, sum);
    }
  }
  sum = block_sum(sum);
  if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

// out = the sum of part[0 .. n), in a fixed order.
__global__ __launch_bounds__(256) void k_squares_join(const double* __restrict__ part, int64_t n,
                                                      double* __restrict__ out) {
  double sum = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += 256) sum += part[i];
  sum = block_sum(sum);
  if (threadIdx.x == 0) *out = sum;
}

// out = in * min(1, max_norm / sqrt(sumsq)): factor and product in 64 bits, rounded to FP32
// and, for BF16, from there (its own half step is 2^15 times FP32's).  With a factor of 1
// and in place nothing moves.  A norm that is not finite scales nothing.
template <class T>
__global__ __launch_bounds__(256) void k_scale(List l, double max_norm, const double* __restrict__ sumsq, double* norm) {
  const double n2 = sqrt(*sumsq);
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = n2;
  const bool scale = n2 > max_norm && n2 < __builtin_inf();
  const double f = scale ? max_norm / n2 : 1.0;
  const int i = find(l, blockIdx.x);
  const int64_t at = (int64_t)(blockIdx.x - l.first[i]) * kPiece, n = l.size[i] - at;
  const T* x = static_cast<const T*>(l.in[i]) + at;
  T* y = static_cast<T*>(l.out[i]) + at;
  if (!scale && x == y) return;
#pragma unroll 4
  for (int k = 0; k < kPiece / 1024; ++k) {
    const int64_t c = 4 * (threadIdx.x + 256 * k);
    if (c >= n) break;
    u4 v = load4(x + c, n - c);
    if (scale)
#pragma unroll
      for (int t = 0; t < 4; ++t) v[t] = __float_as_uint((float)((double)__uint_as_float(v[t]) * f));
    store4(y + c, v, n - c);
  }
}

__global__ void k_norm(const double* __restrict__ sumsq, double* norm) { *norm = sqrt(*sumsq); }

// Calls f(list, pieces) for the tensors in runs of kTensors.
template <class F>
hipError_t each_run(const void* const* in, void* const* out, const int64_t* sizes, int64_t count, F&& f) {
  List l;
  l.count = 0;
  l.first[0] = 0;
  auto flush = [&]() -> hipError_t {
    if (l.count == 0) return hipSuccess;
    const hipError_t e = f(l, l.first[l.count]);
    l.count = 0;
    return e;
  };
  for (int64_t i = 0; i < count; ++i) {
    if (sizes[i] == 0) continue;
    l.in[l.count] = in[i];
    l.out[l.count] = out ? out[i] : nullptr;
    l.size[l.count] = sizes[i];
    l.first[l.count + 1] = l.first[l.count] + (uint32_t)((sizes[i] + kPiece - 1) / kPiece);
    if (++l.count == kTensors) {
      const hipError_t e = flush();
      if (e != hipSuccess) return e;
    }
  }
  return flush();
}

}  // namespace grads

int64_t gradient_pieces(const int64_t* sizes, int64_t count) {
  int64_t n = 0;
  for (int64_t i = 0; i < count; ++i) n += (sizes[i] + grads::kPiece - 1) / grads::kPiece;
  return n;
}

hipError_t launch_sum_squares(const void* const* in, bool bf16, const int64_t* sizes, int64_t count, double* sumsq, double* ws,
                              hipStream_t s) {
  int64_t done = 0;
  const hipError_t e = grads::each_run(in, nullptr, sizes, count, [&](const grads::List& l, uint32_t pieces) {
    hipLaunchKernelGGL(bf16 ? grads::k_squares<fp8::bf16_t> : grads::k_squares<float>, dim3(pieces), dim3(256), 0, s, l,
                       ws + done);
    done += pieces;
    return hipGetLastError();
  });
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(grads::k_squares_join, dim3(1), dim3(256), 0, s, ws, done, sumsq);
  return hipGetLastError();
}

hipError_t launch_scale_gradients(const void* const* in, void* const* out, bool bf16, const int64_t* sizes, int64_t count,
                                  double max_norm, const double* sumsq, double* norm, hipStream_t s) {
  bool first = true;
  const hipError_t e = grads::each_run(in, out, sizes, count, [&](const grads::List& l, uint32_t pieces) {
    hipLaunchKernelGGL(bf16 ? grads::k_scale<fp8::bf16_t> : grads::k_scale<float>, dim3(pieces), dim3(256), 0, s, l,
                       max_norm, sumsq, first ? norm : nullptr);
    first = false;
    return hipGetLastError();
  });
  if (e != hipSuccess || !first) return e;
  hipLaunchKernelGGL(grads::k_norm, dim3(1), dim3(1), 0, s, sumsq, norm);  // (no values)
  return hipGetLastError();
}

}  // namespace fastbfp
