// gradients.hip -- the sum of squares over a list of FP32 or BF16 tensors and their scaling
// down to a largest norm.  Squares and sums are 64 bits (a square of FP32 is exact there,
// and none is out of range), so the norm is right for any values and any number of them.
// HBM-bound: every value read once for the norm, and read and written once for the scaling.
//
// A launch takes its tensors' addresses from its arguments (no table to copy to the
// card).  Work is pieces of 4096 << shift values, at most about 8192 of them; a workgroup
// finds its piece's tensor in the list of their first pieces.
//
// Measured, 4e8 FP32 values in 24 tensors: norm 255 us (6.3 TB/s) and 5 for the join, scaling
// 600 (5.3 TB/s); 150 BF16 tensors of 4e7 values in all: 15, 4 and 31 us.
#include "launch.h"

#include "fp8.h"

namespace fastbfp {

namespace grads {

using fp8::u2;
using fp8::u4;

constexpr int kUnit = 4096, kPieces = 8192;
constexpr int kSums = (int)kMostSums;  // that the scaling adds up itself

// N tensors (that many fit in the 4 KB of a launch's arguments): piece of each one's start,
// and the values of its last piece.
template <int N> struct List {
  const void* in[N];
  uint32_t first[N + 1], tail[N];
  int count, shift;
};
constexpr int kRead = 240, kWrite = 160;
struct Outs {
  void* out[kWrite];
};

template <int N>
__device__ __forceinline__ int find(const List<N>& l, uint32_t piece) {
  int lo = 0, hi = l.count;  // first[lo] <= piece < first[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (l.first[mid] <= piece) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Sum over NT threads, in a fixed order, in all of them.
template <int NT>
__device__ __forceinline__ double block_sum(double v) {
  __shared__ double red[NT / 64];
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) v += red[i];
  return v;
}

// 16 bytes at any value.
template <class T> struct Any16;
template <> struct Any16<float> { typedef u4 __attribute__((aligned(4))) type; };
template <> struct Any16<fp8::bf16_t> { typedef u4 __attribute__((aligned(2))) type; };

// 16 bytes, four FP32 or eight BF16 values, of which `left` are there (the others zeros).
template <class T>
__device__ __forceinline__ u4 load16(const T* p, int left) {
  constexpr int V = 16 / sizeof(T);
  if (left >= V) return *reinterpret_cast<const typename Any16<T>::type*>(p);
  u4 v = u4{0u, 0u, 0u, 0u};
#pragma unroll
  for (int t = 0; t < V - 1; ++t)
    if (t < left) {
      if constexpr (V == 4) v[t] = __float_as_uint(p[t]);
      else v[t / 2] |= (uint32_t)p[t] << (16 * (t & 1));
    }
  return v;
}
template <class T>
__device__ __forceinline__ float value(const u4& v, int t) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(v[t]);
  else return __uint_as_float(t & 1 ? v[t / 2] & 0xFFFF0000u : v[t / 2] << 16);
}

// part[piece] = the sum of squares of a piece.
template <class T>
__global__ __launch_bounds__(256) void k_squares(List<kRead> l, double* __restrict__ part) {
  constexpr int V = 16 / sizeof(T), AT_ONCE = sizeof(T) == 4 ? 4 : 2;  // a unit of values: 4096
  const int i = find(l, blockIdx.x);
  const int64_t at = (int64_t)(blockIdx.x - l.first[i]) * ((int64_t)kUnit << l.shift);
  const int n = blockIdx.x + 1 == l.first[i + 1] ? (int)l.tail[i] : kUnit << l.shift;
  const T* x = static_cast<const T*>(l.in[i]) + at;
  double sum = 0.0;
  for (int u = 0; u < n; u += 2 * kUnit) {
    u4 v[2 * AT_ONCE];
#pragma unroll
    for (int k = 0; k < 2 * AT_ONCE; ++k) {
      const int c = u + V * (threadIdx.x + 256 * k);
      v[k] = load16(x + c, n - c);
    }
#pragma unroll
    for (int k = 0; k < 2 * AT_ONCE; ++k)
#pragma unroll
      for (int t = 0; t < V; ++t) {
        const double a = (double)value<T>(v[k], t);
        sum = __builtin_fma(a, a, sum);
      }
  }
  sum = block_sum<256>(sum);
  if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

// A thread's share of the sum of v[0 .. n), n up to kSums, on the first 256 threads.
__device__ __forceinline__ double few_of(const double* v, int n) {
  double s = 0.0;
#pragma unroll
  for (int k = 0; k < kSums / 256; ++k) s += (int)threadIdx.x + 256 * k < n ? v[threadIdx.x + 256 * k] : 0.0;
  return s;
}

// out = the sum of part[0 .. n), in a fixed order, of few that of the scaling.
__global__ __launch_bounds__(1024) void k_squares_join(const double* __restrict__ part, int64_t n,
                                                       double* __restrict__ out) {
  double sum = n <= kSums && threadIdx.x < 256 ? few_of(part, (int)n) : 0.0;
  for (int64_t i = n <= kSums ? n : threadIdx.x; i < n; i += 8 * 1024) {
    double v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = i + 1024 * k < n ? part[i + 1024 * k] : 0.0;
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += v[k];
  }
  sum = block_sum<1024>(sum);
  if (threadIdx.x == 0) *out = sum;
}

// Values from the last whole line in front of p on.
template <class T>
__host__ __device__ __forceinline__ int ahead(const void* p) {
  return (int)(reinterpret_cast<uintptr_t>(p) % 128 / sizeof(T));
}

// out = in * min(1, max_norm / sqrt(sumsq)): factor and product in 64 bits, rounded to FP32
// and, for BF16, from there (its own half step is 2^16 times FP32's).  With a factor of 1
// and in place nothing moves.  A norm that is not finite scales nothing.  Pieces begin at
// whole lines of the output, which leaves past the caches, and are taken from the last one
// on: what the norm read last is still in the caches behind HBM.
template <class T>
__global__ __launch_bounds__(256) void k_scale(List<kWrite> l, Outs o, double max_norm, const double* __restrict__ sumsq,
                                               int sums, double* norm) {
  constexpr int V = 16 / sizeof(T), AT_ONCE = sizeof(T) == 4 ? 4 : 2;
  const double n2 = sqrt(sums == 1 ? *sumsq : block_sum<256>(few_of(sumsq, sums)));
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = n2;
  const bool scale = n2 > max_norm && n2 < __builtin_inf();
  const double f = scale ? max_norm / n2 : 1.0;
  const uint32_t piece = gridDim.x - 1 - blockIdx.x;
  const int i = find(l, piece);
  if (!scale && l.in[i] == o.out[i]) return;
  const int h = ahead<T>(o.out[i]);
  const int64_t at = (int64_t)(piece - l.first[i]) * ((int64_t)kUnit << l.shift) - h;
  const int begin = at < 0 ? h : 0, n = piece + 1 == l.first[i + 1] ? (int)l.tail[i] : kUnit << l.shift;
  const T* x = static_cast<const T*>(l.in[i]) + at;
  T* y = static_cast<T*>(o.out[i]) + at;
  for (int u = 0; u < n; u += 2 * kUnit) {
    u4 v[2 * AT_ONCE];
#pragma unroll
    for (int k = 0; k < 2 * AT_ONCE; ++k) {
      const int c = u + V * (threadIdx.x + 256 * k);
      v[k] = c >= begin ? load16(x + c, n - c) : u4{0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int k = 0; k < 2 * AT_ONCE; ++k) {
      const int c = u + V * (threadIdx.x + 256 * k);
      if (scale) {
        u4 lo, hi;
#pragma unroll
        for (int t = 0; t < V; ++t) {
          const uint32_t b = __float_as_uint((float)((double)value<T>(v[k], t) * f));
          if (t < 4) lo[t] = b;
          else hi[t - 4] = b;
        }
        if constexpr (V == 4) {
          v[k] = lo;
        } else {
          const u2 p = fp8::to_bf16(lo), q = fp8::to_bf16(hi);
          v[k] = u4{p[0], p[1], q[0], q[1]};
        }
      }
      if (c >= begin && c + V <= n) {
        __builtin_nontemporal_store(v[k], reinterpret_cast<u4*>(y + c));
      } else {
        // (values in front of the tensor were not read: those of its first 16 bytes one by one)
#pragma unroll
        for (int t = 0; t < V; ++t)
          if (c + t >= begin && c + t < n) {
            if (c < begin) {
              const float w = sizeof(T) == 4 ? (float)x[c + t] : __uint_as_float((uint32_t)x[c + t] << 16);
              const uint32_t b = __float_as_uint(scale ? (float)((double)w * f) : w);
              if constexpr (V == 4) y[c + t] = __uint_as_float(b);
              else y[c + t] = (T)fp8::to_bf16(u4{b, 0u, 0u, 0u})[0];
            } else if constexpr (V == 4) {
              y[c + t] = __uint_as_float(v[k][t]);
            } else {
              y[c + t] = (T)(v[k][t / 2] >> (16 * (t & 1)));
            }
          }
      }
    }
  }
}

__global__ __launch_bounds__(256) void k_norm(const double* __restrict__ sumsq, int sums, double* norm) {
  const double s = block_sum<256>(few_of(sumsq, sums));
  if (threadIdx.x == 0) *norm = sqrt(s);
}

// Values of a piece: 4096 << shift, for at most about kPieces of them.
int shift_of(const int64_t* sizes, int64_t count) {
  int64_t total = 0;
  for (int64_t i = 0; i < count; ++i) total += sizes[i];
  int shift = 0;
  while ((total >> shift) > (int64_t)kUnit * kPieces && shift < 18) ++shift;
  return shift;
}

// Fills the lists of N tensors from the first one on, and calls f(list, first tensor's
// number, pieces before, pieces) for each.  ahead(i): values by which tensor i's first piece
// begins in front of it.
template <int N, class A, class F>
hipError_t each_list(const void* const* in, const int64_t* sizes, int64_t count, A&& ahead, F&& f) {
  List<N> l;
  l.shift = shift_of(sizes, count);
  const int64_t piece = (int64_t)kUnit << l.shift;
  int64_t done = 0, from = 0;
  l.count = 0;
  l.first[0] = 0;
  for (int64_t i = 0; i < count; ++i) {
    // (a tensor without values takes a place, and no piece)
    const int64_t n = sizes[i] > 0 ? sizes[i] + ahead(i) : 0, pieces = (n + piece - 1) / piece;
    l.in[l.count] = in[i];
    l.first[l.count + 1] = l.first[l.count] + (uint32_t)pieces;
    l.tail[l.count] = (uint32_t)(n - (pieces > 0 ? pieces - 1 : 0) * piece);
    if (++l.count < N && i + 1 < count) continue;
    const int64_t all = l.first[l.count];
    if (all > 0) {
      const hipError_t e = f(l, from, done, all);
      if (e != hipSuccess) return e;
    }
    done += all;
    from = i + 1;
    l.count = 0;
  }
  return hipSuccess;
}

}  // namespace grads

int64_t gradient_pieces(const int64_t* sizes, int64_t count) {
  const int64_t piece = (int64_t)grads::kUnit << grads::shift_of(sizes, count);
  int64_t n = 0;
  for (int64_t i = 0; i < count; ++i) n += (sizes[i] + piece - 1) / piece;
  return n;
}

hipError_t launch_sum_squares(const void* const* in, bool bf16, const int64_t* sizes, int64_t count, double* sumsq,
                              double* ws, hipStream_t s) {
  using namespace grads;
  int64_t all = 0;
  const hipError_t e = each_list<kRead>(in, sizes, count, [](int64_t) { return 0; },
                                        [&](const List<kRead>& l, int64_t, int64_t done, int64_t pieces) {
    hipLaunchKernelGGL(bf16 ? k_squares<fp8::bf16_t> : k_squares<float>, dim3((unsigned)pieces), dim3(256), 0, s, l,
                       ws + done);
    all = done + pieces;
    return hipGetLastError();
  });
  if (e != hipSuccess || !sumsq) return e;
  hipLaunchKernelGGL(k_squares_join, dim3(1), dim3(1024), 0, s, ws, all, sumsq);
  return hipGetLastError();
}

hipError_t launch_scale_gradients(const void* const* in, void* const* out, bool bf16, const int64_t* sizes,
                                  int64_t count, double max_norm, const double* sumsq, int sums, double* norm,
                                  hipStream_t s) {
  using namespace grads;
  bool first = true;
  auto before = [&](int64_t i) { return bf16 ? ahead<fp8::bf16_t>(out[i]) : ahead<float>(out[i]); };
  const hipError_t e = each_list<kWrite>(in, sizes, count, before,
                                         [&](const List<kWrite>& l, int64_t from, int64_t, int64_t pieces) {
    Outs o;
    for (int i = 0; i < l.count; ++i) o.out[i] = out[from + i];
    hipLaunchKernelGGL(bf16 ? k_scale<fp8::bf16_t> : k_scale<float>, dim3((unsigned)pieces), dim3(256), 0, s, l, o,
                       max_norm, sumsq, sums, first ? norm : nullptr);
    first = false;
    return hipGetLastError();
  });
  if (e != hipSuccess || !first) return e;
  hipLaunchKernelGGL(k_norm, dim3(1), dim3(256), 0, s, sumsq, sums, norm);  // (no values)
  return hipGetLastError();
}

}  // namespace fastbfp
