// rms_norm.hip -- a residual's addition and the root-mean-square norm of the sum, with
// the output left in FP32 or converted on the way (8-bit blocks or BFP groups of 16), and
// the norm's gradients.
//
//   h = x + residual (FP32),  r = (mean(h^2) + eps)^(-1/2),  y = h r w
// The mean, r and the product are 64 bits and y is rounded once to FP32: y is the formula's
// value whatever the launch, and the converted output the conversion of that y.  (64-bit
// multiplies and adds run at FP32's rate here, and the kernel waits for HBM.)
// HBM-bound: x and the residual read once, h and the output written once.
//
// Measured, 8192 x 4096: BF16 x + residual -> h and e4m3 blocks 66 us, 5.6 TB/s; FP32 x +
// residual -> h and BFP of width 4 77 us (120 when 16 lanes of a wave converted), -> h and FP32
// 92; the gradient from a BF16 dy 86 us, 5.6 TB/s, and 5.4 for the join of dw.  One row: 4.0
// us, a launch.
#include "fp8.h"
#include "gemm_direct.h"
#include "launch.h"

namespace fastbfp {

namespace norm {

using fp8::load4;
using fp8::store4;
using fp8::u4;

// Sum over the workgroup of NT threads, in all of them; the order depends on NT alone.
template <int NT>
__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) v += red[i];
  }
  return v;
}

enum { kToF32 = 0, kToFp8 = 1, kToBfp = 2 };

struct Args {
  const void* x;  // FP32 or BF16
  const float *residual, *w;
  int64_t rows, d;
  double eps;
  float *h, *rstd, *y;  // (h and rstd may be null)
  uint8_t *codes, *exps;
  int fmt;
  uint32_t* status;
  direct::Out bfp;
};

// A workgroup of NT threads takes a row, thread t its values 4 (t + NT k) .. + 3.
// Rows of 8193 to 12288 values are kept to 64 registers, and so two of them on a CU, at the
// price of weights that are not on the way with the values (2781 x 9408 FP32 -> e4m3 34 us, with
// 16384's registers 55).
template <int NT, int NV, bool RES, int TO, class T>
__global__ __launch_bounds__(NT, NV == 3 ? 8 : 1) void k_rms_norm(Args p) {
  constexpr bool EARLY = NV != 3;
  __shared__ double red[NT > 64 ? NT / 64 : 1];
  __shared__ __attribute__((aligned(16))) float stage[TO == kToBfp ? 4 * NT * NV : 4];
  const int64_t row = blockIdx.x, d = p.d;
  const int t = threadIdx.x;
  const T* x = static_cast<const T*>(p.x) + row * d;
  u4 v[NV], w[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) v[k] = load4(x + 4 * (t + NT * k), d - 4 * (t + NT * k));
  if constexpr (EARLY) {
#pragma unroll
    for (int k = 0; k < NV; ++k) w[k] = load4(p.w + 4 * (t + NT * k), d - 4 * (t + NT * k));
  }
  if constexpr (RES) {
    u4 z[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) z[k] = load4(p.residual + row * d + 4 * (t + NT * k), d - 4 * (t + NT * k));
#pragma unroll
    for (int k = 0; k < NV; ++k) {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[k][i] = __float_as_uint(__uint_as_float(v[k][i]) + __uint_as_float(z[k][i]));
    }
  }
  double sum = 0.0;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    if (p.h) store4(p.h + row * d + 4 * (t + NT * k), v[k], d - 4 * (t + NT * k));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const double a = (double)__uint_as_float(v[k][i]);
      sum = __builtin_fma(a, a, sum);
    }
  }
  sum = block_sum<NT>(sum, red);
  const double r = 1.0 / sqrt(sum / (double)d + p.eps);
  if (p.rstd && t == 0) p.rstd[row] = (float)r;
  uint32_t bad = 0;
  float* mine = stage + (TO == kToBfp ? 256 * NV * (t >> 6) : 0);
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int64_t c = 4 * (t + NT * k);
    if constexpr (!EARLY) w[k] = load4(p.w + c, d - c);
    u4 y;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      y[i] = __float_as_uint((float)((double)__uint_as_float(v[k][i]) * r * (double)__uint_as_float(w[k][i])));
    if constexpr (TO == kToF32) {
      store4(p.y + row * d + c, y, d - c);
    } else if constexpr (TO == kToFp8) {
      if (c >= d)  // (past the end, where 0 r w may be NaN)
        y = u4{0u, 0u, 0u, 0u};
      else if (d - c < 4)
#pragma unroll
        for (int i = 1; i < 4; ++i) y[i] = c + i < d ? y[i] : 0u;
      uint32_t s;
      bool b;
      const uint32_t q = p.fmt == fp8::kE4M3 ? fp8::convert_block<fp8::kE4M3>(y, s, b) : fp8::convert_block<fp8::kE5M2>(y, s, b);
      bad |= b ? 1u : 0u;
      const int64_t block = c / fp8::kBlock;
      if (block * fp8::kBlock < d) *reinterpret_cast<uint32_t*>(p.codes + row * fp8::code_pitch(d) + c) = q;
      if ((t & 31) == 0 && block < fp8::exp_pitch(d)) p.exps[row * fp8::exp_pitch(d) + block] = (uint8_t)s;
    } else {
      const int q = 64 * k + (t & 63);
      *reinterpret_cast<u4*>(mine + 4 * (q ^ ((q >> 4) & 3))) = y;
    }
  }
  if constexpr (TO == kToBfp) {
    // A wave's 256 consecutive values for each k, 16 groups, are in its part of LDS; a lane
    // converts a group.  (Quad q sits at q ^ ((q >> 4) & 3): 16 lanes that read a quad of
    // 16 groups hit all banks.)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
    const int lane = t & 63;
    const int64_t g = 16 * (int64_t)((t >> 6) + NT / 64 * (lane >> 4)) + (lane & 15);
    if (lane < 16 * NV && 16 * g < d) {
      uint32_t b[16];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int q = 4 * lane + i;
        const u4 x = *reinterpret_cast<const u4*>(mine + 4 * (q ^ ((q >> 4) & 3)));
#pragma unroll
        for (int e = 0; e < 4; ++e) b[4 * i + e] = x[e];
      }
      bad |= direct::convert(b, row * (d / 16) + g, p.bfp) ? 1u : 0u;
    }
  }
  if constexpr (TO != kToF32) {
    if (TO == kToFp8 && t == 0 && NT * NV * 4 / fp8::kBlock < fp8::exp_pitch(d)) {
      // (scales behind the last block that no thread's values reach)
      for (int64_t b = NT * NV * 4 / fp8::kBlock; b < fp8::exp_pitch(d); ++b) p.exps[row * fp8::exp_pitch(d) + b] = 0;
    }
    if (p.status && bad) atomicOr(p.status, 1u);
  }
}

// The gradients, for u = w dy, h and r of the forward pass and n = h r (at most sqrt(d),
// so that nothing leaves FP32's range on the way while r is in it):
//   dx = r (u - n mean(u n)) (+ dresidual),  dw = sum over rows of dy n
// u and n are rounded to FP32; their products, dy n and the sums of both are 64 bits (FP32
// products, and sums of four of them, took as long: 8192 x 4096 with a residual 91.5 us
// and 91.6).  NT threads take a row, W rows side by side in a workgroup, and then every
// gridDim W-th one; their share of dw stays in registers, in 64 bits, and goes to part[b]
// in FP32 (in 64 bits the shares would move 8 MB more each way at d = 4096).  (The next
// row's loads ahead of this one's sum changed nothing up to 8192 values, where the workgroups
// on a CU cover each other's.)  W is 8 for rows of one wave: with one of them to a workgroup
// 16384 x 512 took 40.6 us.  Rows of more than 8192 values leave no registers for their share:
// it is in LDS (2000 x 9698: 162 us with spills).
struct GradArgs {
  const void* dy;  // FP32 or BF16
  const float *h, *rstd, *w, *dresidual;
  int64_t rows, d;
  float *dx, *part;
};
constexpr int rows_of(int nt) { return nt == 64 ? 8 : 1; }  // W
template <int NT, int NV, bool RES, class T>
__global__ __launch_bounds__(NT * rows_of(NT)) void k_rms_norm_grad(GradArgs p) {
  constexpr int W = rows_of(NT);
  static_assert(W == 1 || NT == 64, "waves that take rows of their own meet nowhere in the loop");
  constexpr bool LDS = NT * NV >= 4096;
  __shared__ double red[2][NT > 64 ? NT / 64 : 1];
  const int64_t d = p.d;
  const int t = threadIdx.x % NT, slot = threadIdx.x / NT;
  u4 w[NV];
  double mine[LDS ? 1 : NV][4];
  __shared__ double share[LDS ? NV * 4 * NT : 1];  // (a thread's own places: nothing to wait for)
  auto dw = [&](int k, int i) __attribute__((always_inline)) -> double& {
    return LDS ? share[(4 * k + i) * NT + t] : mine[LDS ? 0 : k][i];
  };
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    w[k] = load4(p.w + 4 * (t + NT * k), d - 4 * (t + NT * k));
#pragma unroll
    for (int i = 0; i < 4; ++i) dw(k, i) = 0.0;
  }
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * W + slot; row < p.rows; row += (int64_t)gridDim.x * W, turn ^= 1) {
    const float r = p.rstd[row];
    u4 g[NV], h[NV], z[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int64_t c = 4 * (t + NT * k);
      g[k] = load4(static_cast<const T*>(p.dy) + row * d + c, d - c);
      h[k] = load4(p.h + row * d + c, d - c);
      if constexpr (RES) z[k] = load4(p.dresidual + row * d + c, d - c);
    }
    double sum = 0.0;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float dy = __uint_as_float(g[k][i]);
        const double n = (double)(__uint_as_float(h[k][i]) * r);
        sum = __builtin_fma((double)(dy * __uint_as_float(w[k][i])), n, sum);
        dw(k, i) = __builtin_fma((double)dy, n, dw(k, i));
      }
    }
    // (two places for the waves' sums: a wave may be a row ahead of one that still reads)
    sum = block_sum<NT>(sum, red[turn]);
    const float a = (float)((double)r * (sum / (double)d));
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int64_t c = 4 * (t + NT * k);
      u4 o;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float u = __uint_as_float(g[k][i]) * __uint_as_float(w[k][i]);
        float v = __builtin_fmaf(-(__uint_as_float(h[k][i]) * r), a, u * r);
        if constexpr (RES) v += __uint_as_float(z[k][i]);
        o[i] = __float_as_uint(v);
      }
      store4(p.dx + row * d + c, o, d - c);
    }
  }
  float* part = p.part + (int64_t)blockIdx.x * d;
  if constexpr (W == 1) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int64_t c = 4 * (t + NT * k);
      u4 o;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = __float_as_uint((float)dw(k, i));
      store4(part + c, o, d - c);
    }
  } else {
    __shared__ double rows[W][4 * NT];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      if (k > 0) __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i) rows[slot][4 * t + i] = dw(k, i);
      __syncthreads();
      const int64_t c = 4 * NT * k + threadIdx.x;
      if (threadIdx.x < 4 * NT && c < d) {
        double sum = 0.0;
#pragma unroll
        for (int s = 0; s < W; ++s) sum += rows[s][threadIdx.x];
        part[c] = (float)sum;
      }
    }
  }
}

// dw[c] = the sum of part[b][c] over b, in 64 bits and a fixed order: 64 columns a
// workgroup, in 16 runs of rows.
__global__ __launch_bounds__(256) void k_rms_norm_join(const float* __restrict__ part, int parts, int64_t d,
                                                       float* __restrict__ dw) {
  __shared__ double red[16][64];
  const int run = threadIdx.x >> 4;
  const int64_t col = (int64_t)blockIdx.x * 64 + 4 * (threadIdx.x & 15), left = d - col;
  double v[4] = {0.0, 0.0, 0.0, 0.0};
  for (int b = run; b < parts; b += 16 * 8) {
    u4 x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      x[k] = b + 16 * k < parts ? load4(part + (int64_t)(b + 16 * k) * d + col, left) : u4{0u, 0u, 0u, 0u};
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] += (double)__uint_as_float(x[k][i]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) red[run][4 * (threadIdx.x & 15) + i] = v[i];
  __syncthreads();
  const int64_t c = (int64_t)blockIdx.x * 64 + threadIdx.x;
  if (threadIdx.x < 64 && c < d) {
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < 16; ++i) sum += red[i][threadIdx.x];
    dw[c] = (float)sum;
  }
}

// Threads to a row and vectors to a thread.
struct Shape {
  int nt, nv;
};
Shape shape_of(int64_t d) {
  const int nt = d <= 1024 ? 64 : d <= 4096 ? 256 : 1024;
  const int64_t v = (d + 4 * nt - 1) / (4 * nt);
  return {nt, v <= 1 ? 1 : v <= 2 ? 2 : v <= 3 && nt == 1024 ? 3 : 4};
}

template <int NT, int NV, class T>
hipError_t launch_norm(const Args& a, int to, hipStream_t s) {
  const dim3 grid((unsigned)a.rows);
#define FASTBFP_NORM(RES, TO) hipLaunchKernelGGL((k_rms_norm<NT, NV, RES, TO, T>), grid, dim3(NT), 0, s, a)
  if (a.residual) {
    if (to == kToF32) FASTBFP_NORM(true, kToF32);
    else if (to == kToFp8) FASTBFP_NORM(true, kToFp8);
    else FASTBFP_NORM(true, kToBfp);
  } else {
    if (to == kToF32) FASTBFP_NORM(false, kToF32);
    else if (to == kToFp8) FASTBFP_NORM(false, kToFp8);
    else FASTBFP_NORM(false, kToBfp);
  }
#undef FASTBFP_NORM
  return hipGetLastError();
}
template <int NT, class T>
hipError_t launch_norm_nv(const Args& a, int nv, int to, hipStream_t s) {
  return nv == 1   ? launch_norm<NT, 1, T>(a, to, s)
         : nv == 2 ? launch_norm<NT, 2, T>(a, to, s)
         : nv == 3 ? launch_norm<1024, 3, T>(a, to, s)
                   : launch_norm<NT, 4, T>(a, to, s);
}
template <class T>
hipError_t launch_t(const Args& a, int to, hipStream_t s) {
  const Shape f = shape_of(a.d);
  return f.nt == 64    ? launch_norm_nv<64, T>(a, f.nv, to, s)
         : f.nt == 256 ? launch_norm_nv<256, T>(a, f.nv, to, s)
                       : launch_norm_nv<1024, T>(a, f.nv, to, s);
}
hipError_t launch(const Args& a, bool bf16, int to, hipStream_t s) {
  return bf16 ? launch_t<fp8::bf16_t>(a, to, s) : launch_t<float>(a, to, s);
}

template <int NT, class T>
void launch_grad(const GradArgs& a, int nv, int parts, hipStream_t s) {
  const dim3 grid((unsigned)parts), block(NT * rows_of(NT));
#define FASTBFP_GRAD(NV)                                                                    \
  if (a.dresidual) hipLaunchKernelGGL((k_rms_norm_grad<NT, NV, true, T>), grid, block, 0, s, a); \
  else hipLaunchKernelGGL((k_rms_norm_grad<NT, NV, false, T>), grid, block, 0, s, a)
  if (nv == 1) {
    FASTBFP_GRAD(1);
  } else if (nv == 2) {
    FASTBFP_GRAD(2);
  } else {
    FASTBFP_GRAD(4);
  }
#undef FASTBFP_GRAD
}

template <class T>
void launch_grad_t(const GradArgs& a, int parts, hipStream_t s) {
  const Shape f = shape_of(a.d);
  if (f.nt == 64) launch_grad<64, T>(a, f.nv, parts, s);
  else if (f.nt == 256) launch_grad<256, T>(a, f.nv, parts, s);
  else launch_grad<1024, T>(a, f.nv, parts, s);
}

}  // namespace norm

hipError_t launch_rms_norm(const void* x, bool bf16, const float* residual, const float* w, int64_t rows, int64_t d, double eps,
                           float* h, float* rstd, float* y, hipStream_t s) {
  norm::Args a{};
  a.x = x, a.residual = residual, a.w = w, a.rows = rows, a.d = d, a.eps = eps, a.h = h, a.rstd = rstd, a.y = y;
  return norm::launch(a, bf16, norm::kToF32, s);
}

hipError_t launch_rms_norm_fp8(const void* x, bool bf16, const float* residual, const float* w, int64_t rows, int64_t d,
                               double eps, float* h, float* rstd, int fmt, uint8_t* codes, uint8_t* exps,
                               uint32_t* status, hipStream_t s) {
  norm::Args a{};
  a.x = x, a.residual = residual, a.w = w, a.rows = rows, a.d = d, a.eps = eps, a.h = h, a.rstd = rstd;
  a.fmt = fmt, a.codes = codes, a.exps = exps, a.status = status;
  return norm::launch(a, bf16, norm::kToFp8, s);
}

hipError_t launch_rms_norm_bfp(const void* x, bool bf16, const float* residual, const float* w, int64_t rows, int64_t d,
                               double eps, float* h, float* rstd, int m, int mode, uint64_t seed, uint8_t* mant,
                               uint8_t* exps, uint32_t* status, hipStream_t s) {
  norm::Args a{};
  a.x = x, a.residual = residual, a.w = w, a.rows = rows, a.d = d, a.eps = eps, a.h = h, a.rstd = rstd;
  a.status = status;
  a.bfp = {mant, mant + rows * (d / 16) * plane_group_bytes(16, m, 0), exps, status, m, mode, (uint32_t)seed,
           (uint32_t)(seed >> 32)};
  return norm::launch(a, bf16, norm::kToBfp, s);
}

int64_t rms_norm_threads(int64_t d) { return norm::shape_of(d).nt; }

// Workgroups of the gradient, up to 512: enough for all rows at once where a wave takes one,
// else one for each row up to 256 and for every fourth row from there on.  One takes up to
// three rows alone, whose share is dw: a second launch would take longer than the rows.
int64_t rms_norm_grad_parts(int64_t rows, int64_t d) {
  const int64_t w = norm::rows_of(norm::shape_of(d).nt), all = (rows + w - 1) / w;
  if (w == 1 && rows <= 3) return rows < 1 ? 0 : 1;
  if (w > 1 || all <= 256) return all < 512 ? all : 512;
  const int64_t n = (rows + 3) / 4;
  return n < 256 ? 256 : n < 512 ? n : 512;
}

hipError_t launch_rms_norm_grad(const void* dy, bool bf16, const float* h, const float* rstd, const float* w,
                                const float* dresidual, int64_t rows, int64_t d, float* dx, float* dw, float* ws,
                                hipStream_t s) {
  const int parts = (int)rms_norm_grad_parts(rows, d);
  if (rows > 0) {
    const norm::GradArgs a{dy, h, rstd, w, dresidual, rows, d, dx, parts == 1 ? dw : ws};
    if (bf16) norm::launch_grad_t<fp8::bf16_t>(a, parts, s);
    else norm::launch_grad_t<float>(a, parts, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || parts == 1) return e;
  }
  hipLaunchKernelGGL(norm::k_rms_norm_join, dim3((unsigned)((d + 63) / 64)), dim3(256), 0, s, ws, parts, d, dw);
  return hipGetLastError();
}

}  // namespace fastbfp
