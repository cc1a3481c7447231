// quantize_fp8.hip -- FP32 or BF16 -> 8-bit floating-point blocks (fp8.h) along either axis,
// or both from one read, and the inverse.  HBM-bound: 4 or 2 bytes read and 1 + 1/128
// written a value (2 + 1/64 with both).
//
// Measured, 8192 x 4096 of BF16: rows 16.7 us (6.1 TB/s read and written), columns 19, both
// 26.6 (5.1); with a wave to a block and FP32 arithmetic for scale and rounding they took 30,
// 60 and 79.  Small ones take as long as their code's way through the instruction caches
// (both conversions of 16 x 4096 5.8).  Zeros, and what lies past the tensor's ends,
// decide no branch: while they did, both conversions of 1531 x 1050 FP32 took 11.3 us and
// those along its rows 5.1, now 7.6 and 3.5; with zeros in every seventh row of 8192 x 4096
// both took 33, now 26.
// The inverse of 8192 x 4096 takes 26 us (6.4 TB/s).
#include "fp8.h"
#include "launch.h"

namespace fastbfp {

namespace fp8 {

// Blocks along the rows.  Half a wave takes four blocks of a row, a lane four values of
// each: every load reads 512 contiguous bytes (256 of BF16), every store writes a block's
// 128, and the four scales leave as one dword.
template <int FMT, class T>
__global__ __launch_bounds__(256) void k_fp8_rows(const T* __restrict__ x, int64_t len, uint32_t quads_row,
                                                  int64_t quads, uint8_t* __restrict__ codes,
                                                  uint8_t* __restrict__ exps, uint32_t* status) {
  const int64_t q = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (q >= quads) return;
  const int lane = threadIdx.x & 31;
  const int64_t row = q / quads_row;
  const int64_t c0 = (q - row * quads_row) * (4 * kBlock) + 4 * lane;
  const T* src = x + row * len;
  typename Raw<T>::type v[4];
#pragma unroll
  for (int b = 0; b < 4; ++b) v[b] = raw4(src + c0 + b * kBlock, len - (c0 + b * kBlock));
  uint32_t scales = 0, w[4], s[4];
  bool any;
  uint8_t* out = codes + row * code_pitch(len);
  convert_blocks<FMT>(v, w, s, any);
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    scales |= s[b] << (8 * b);
    if (c0 - 4 * lane + b * kBlock < len) *reinterpret_cast<uint32_t*>(out + c0 + b * kBlock) = w[b];
  }
  if (lane == 0) *reinterpret_cast<uint32_t*>(exps + row * exp_pitch(len) + (c0 / kBlock)) = scales;
  if (status && any) atomicOr(status, 1u);
}

// Blocks down the columns (transposed: output row c is column c), and with ROWS also
// along the rows, by tiles of 128 x 128: a tile holds a block of each of its rows and of
// each of its columns.  Half a wave loads 16 rows, all on the way at once, converts them
// where asked to and leaves them in LDS as they are; then a thread takes 64 values down
// the columns (FP32: half of one; BF16: a quarter of two beside each other, a dword a row),
// and the codes leave through LDS as whole lines.
constexpr int kCodeStride = kBlock + 16;  // of a column's codes in LDS, bytes

template <int FMT, bool ROWS, class T>
__global__ __launch_bounds__(256) void k_fp8_tiles(const T* __restrict__ x, int64_t R, int64_t C, uint32_t tiles_c,
                                                   uint8_t* __restrict__ codes_r, uint8_t* __restrict__ exps_r,
                                                   uint8_t* __restrict__ codes_c, uint8_t* __restrict__ exps_c,
                                                   uint32_t* status) {
  constexpr bool B = sizeof(T) == 2;
  constexpr int RUNS = B ? 4 : 2;  // threads to a column
  __shared__ __attribute__((aligned(16))) T tile[kBlock * kBlock];
  __shared__ uint32_t top[RUNS][kBlock];
  static_assert(sizeof(tile) >= kBlock * kCodeStride, "the codes fit where the tile was");
  const int tr = blockIdx.x / tiles_c, tc = blockIdx.x % tiles_c;
  const int64_t r0 = (int64_t)tr * kBlock, c0 = (int64_t)tc * kBlock;
  {
    const int half = threadIdx.x >> 5, lane = threadIdx.x & 31;
    typedef typename Raw<T>::type V;
    const int rows = (int)min((int64_t)kBlock, R - r0);
    const T* src = x + (r0 + half) * C + c0 + 4 * lane;
    T* mine = tile + half * kBlock + 4 * lane;
    uint8_t* codes = codes_r + (r0 + half) * code_pitch(C) + c0 + 4 * lane;
    uint8_t* exps = exps_r + (r0 + half) * exp_pitch(C) + tc + lane;
    // (a row's scale, and in its last tile the zeros behind it)
    const bool scales = lane < (tc + 1 == (int)tiles_c ? (int)(exp_pitch(C) - tc) : 1);
    bool any = false, done = false;
    if (C >= 4) {
      // (of a lane that the rows' end leaves some of its four, the row's last four, moved
      // down: no branch among the loads)
      const int left = (int)max(min(C - (c0 + 4 * lane), (int64_t)4), (int64_t)0), past = left > 0 ? 4 - left : 0;
      V v[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = 8 * i + half < rows && left > 0 ? raw4(src - past + 8 * i * C, 4) : V{};
      if (c0 + kBlock > C && C % 4 != 0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = down(v[i], past);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) *reinterpret_cast<V*>(mine + 8 * i * kBlock) = v[i];
      if constexpr (ROWS) {
        uint32_t key[16];
        done = true;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          key[i] = max_half_wave(key4(v[i]));
          done &= quick(key[i], scale_of(key[i] >> 1, FMT));
        }
        if (done) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const uint32_t s = scale_of(key[i] >> 1, FMT);
            if (8 * i + half < rows) {
              *reinterpret_cast<uint32_t*>(codes + 8 * i * code_pitch(C)) = quick4<FMT>(v[i], s);
              if (scales) exps[8 * i * exp_pitch(C)] = lane == 0 ? (uint8_t)s : 0;
            }
          }
        }
      }
    } else {
#pragma unroll 4
      for (int i = 0; i < 16; ++i)
        *reinterpret_cast<V*>(mine + 8 * i * kBlock) = 8 * i + half < rows ? raw4(src + 8 * i * C, C - (c0 + 4 * lane)) : V{};
    }
    if (ROWS && !done) {
      // (not unrolled, from LDS: in the quick way's path its code would be fetched too)
#pragma unroll 1
      for (int i = 0; 8 * i + half < rows; ++i) {
        uint32_t s;
        bool bad;
        const uint32_t w = convert_block<FMT>(*reinterpret_cast<const V*>(mine + 8 * i * kBlock), s, bad);
        any |= bad;
        *reinterpret_cast<uint32_t*>(codes + 8 * i * code_pitch(C)) = w;
        if (scales) exps[8 * i * exp_pitch(C)] = lane == 0 ? (uint8_t)s : 0;
      }
      if (status && any) atomicOr(status, 1u);
    }
  }
  __syncthreads();
  // Column c (with BF16 c and c + 1) from row run * 128 / RUNS on.
  const int c = B ? 2 * (threadIdx.x & 63) : threadIdx.x & 127, run = threadIdx.x / (B ? 64 : 128);
  constexpr int Q = B ? 8 : 16, COLS = B ? 2 : 1;  // quads of rows, columns
  typename Raw<T>::type v[COLS][Q];
  uint32_t key[COLS];
#pragma unroll
  for (int j = 0; j < COLS; ++j) key[j] = 0;
#pragma unroll
  for (int i = 0; i < Q; ++i) {
    const int r = run * (kBlock / RUNS) + 4 * i;
    if constexpr (B) {
      uint32_t w[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) w[t] = *reinterpret_cast<const uint32_t*>(&tile[(r + t) * kBlock + c]);
      v[0][i] = u2{__builtin_amdgcn_perm(w[1], w[0], 0x05040100u), __builtin_amdgcn_perm(w[3], w[2], 0x05040100u)};
      v[COLS - 1][i] = u2{__builtin_amdgcn_perm(w[1], w[0], 0x07060302u), __builtin_amdgcn_perm(w[3], w[2], 0x07060302u)};
    } else {
#pragma unroll
      for (int t = 0; t < 4; ++t) v[0][i][t] = __float_as_uint(tile[(r + t) * kBlock + c]);
    }
#pragma unroll
    for (int j = 0; j < COLS; ++j) key[j] = max(key[j], key4(v[j][i]));
  }
#pragma unroll
  for (int j = 0; j < COLS; ++j) top[run][c + j] = key[j];
  bool odd = false;
#pragma unroll
  for (int j = 0; j < COLS; ++j) odd |= !key_finite(key[j]);
  // (also: the tile is read)
  if (__syncthreads_or(odd)) {
    // a tile with infinities or NaN: the maxima without them
    if (odd && status) atomicOr(status, 1u);
#pragma unroll
    for (int j = 0; j < COLS; ++j) {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < Q; ++i) m = max(m, max4(wide(v[j][i])));
      top[run][c + j] = m << 1;
    }
    __syncthreads();
  }
  uint8_t* out = reinterpret_cast<uint8_t*>(tile);
#pragma unroll
  for (int j = 0; j < COLS; ++j) {
    uint32_t m = top[0][c + j];
#pragma unroll
    for (int k = 1; k < RUNS; ++k) m = max(m, top[k][c + j]);
    const uint32_t s = scale_of(m >> 1, FMT);
    uint32_t w[Q];
    if (!odd && quick(m, s)) {
#pragma unroll
      for (int i = 0; i < Q; ++i) w[i] = quick4<FMT>(v[j][i], s);
    } else {
      const float inv = inverse(s);
#pragma unroll
      for (int i = 0; i < Q; ++i) w[i] = convert4(wide(v[j][i]), inv, FMT);
    }
#pragma unroll
    for (int i = 0; i < Q / 4; ++i)
      *reinterpret_cast<u4*>(out + (c + j) * kCodeStride + run * (kBlock / RUNS) + 16 * i) =
          u4{w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
    if (c0 + c + j < C) {
      uint8_t* e = exps_c + (c0 + c + j) * exp_pitch(R) + tr;
      if (run == 0) *e = (uint8_t)s;
      else if (run == 1 && r0 + kBlock >= R)
        for (int k = 1; k < (int)(exp_pitch(R) - tr); ++k) e[k] = 0;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int cc = i * 32 + (threadIdx.x >> 3), at = (threadIdx.x & 7) * 16;
    if (c0 + cc < C)
      *reinterpret_cast<u4*>(codes_c + (c0 + cc) * code_pitch(R) + r0 + at) =
          *reinterpret_cast<const u4*>(out + cc * kCodeStride + at);
  }
}

// The values: codes times their block's scale (exact unless below FP32's range).
template <int FMT>
__global__ __launch_bounds__(256) void k_fp8_values(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ exps,
                                                    int64_t len, int64_t words_row, int64_t words,
                                                    float* __restrict__ y) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= words) return;
  const int64_t row = i / words_row, k = (i - row * words_row) * 4;
  const int w = *reinterpret_cast<const int*>(codes + row * code_pitch(len) + k);
  const int e = (int)exps[row * exp_pitch(len) + k / kBlock] - 127;
  float f[4];
  if constexpr (FMT == kE4M3) {
    f[0] = __builtin_amdgcn_cvt_f32_fp8(w, 0), f[1] = __builtin_amdgcn_cvt_f32_fp8(w, 1);
    f[2] = __builtin_amdgcn_cvt_f32_fp8(w, 2), f[3] = __builtin_amdgcn_cvt_f32_fp8(w, 3);
  } else {
    f[0] = __builtin_amdgcn_cvt_f32_bf8(w, 0), f[1] = __builtin_amdgcn_cvt_f32_bf8(w, 1);
    f[2] = __builtin_amdgcn_cvt_f32_bf8(w, 2), f[3] = __builtin_amdgcn_cvt_f32_bf8(w, 3);
  }
  u4 v;
#pragma unroll
  for (int t = 0; t < 4; ++t) v[t] = __float_as_uint(__builtin_ldexpf(f[t], e));
  store4(y + row * len + k, v, len - k);
}

}  // namespace fp8

namespace fp8 {

template <int FMT, class T>
hipError_t launch_rows(const T* x, int64_t R, int64_t C, uint8_t* codes, uint8_t* exps, uint32_t* status,
                       hipStream_t s) {
  const int64_t quads_row = (blocks_of(C) + 3) / 4, quads = R * quads_row;
  hipLaunchKernelGGL((k_fp8_rows<FMT, T>), dim3((unsigned)((quads + 7) / 8)), dim3(256), 0, s, x, C,
                     (uint32_t)quads_row, quads, codes, exps, status);
  return hipGetLastError();
}

template <int FMT, class T>
hipError_t launch_tiles(const T* x, int64_t R, int64_t C, uint8_t* codes_r, uint8_t* exps_r, uint8_t* codes_c,
                        uint8_t* exps_c, uint32_t* status, hipStream_t s) {
  const uint32_t tiles_c = (uint32_t)blocks_of(C);
  const dim3 grid((unsigned)(blocks_of(R) * tiles_c));
  if (codes_r)
    hipLaunchKernelGGL((k_fp8_tiles<FMT, true, T>), grid, dim3(256), 0, s, x, R, C, tiles_c, codes_r, exps_r, codes_c,
                       exps_c, status);
  else
    hipLaunchKernelGGL((k_fp8_tiles<FMT, false, T>), grid, dim3(256), 0, s, x, R, C, tiles_c, codes_r, exps_r, codes_c,
                       exps_c, status);
  return hipGetLastError();
}

}  // namespace fp8

hipError_t launch_quantize_fp8(const void* x, bool bf16, int64_t R, int64_t C, int group_axis, int fmt, uint8_t* codes,
                               uint8_t* exps, uint32_t* status, hipStream_t s) {
  using namespace fp8;
  if (group_axis == 0) return launch_quantize_fp8_dual(x, bf16, R, C, fmt, nullptr, nullptr, codes, exps, status, s);
  const float* f = static_cast<const float*>(x);
  const bf16_t* b = static_cast<const bf16_t*>(x);
  if (fmt == kE4M3)
    return bf16 ? launch_rows<kE4M3>(b, R, C, codes, exps, status, s) : launch_rows<kE4M3>(f, R, C, codes, exps, status, s);
  return bf16 ? launch_rows<kE5M2>(b, R, C, codes, exps, status, s) : launch_rows<kE5M2>(f, R, C, codes, exps, status, s);
}

hipError_t launch_quantize_fp8_dual(const void* x, bool bf16, int64_t R, int64_t C, int fmt, uint8_t* codes_r,
                                    uint8_t* exps_r, uint8_t* codes_c, uint8_t* exps_c, uint32_t* status,
                                    hipStream_t s) {
  using namespace fp8;
  const float* f = static_cast<const float*>(x);
  const bf16_t* b = static_cast<const bf16_t*>(x);
  if (fmt == kE4M3)
    return bf16 ? launch_tiles<kE4M3>(b, R, C, codes_r, exps_r, codes_c, exps_c, status, s)
                : launch_tiles<kE4M3>(f, R, C, codes_r, exps_r, codes_c, exps_c, status, s);
  return bf16 ? launch_tiles<kE5M2>(b, R, C, codes_r, exps_r, codes_c, exps_c, status, s)
              : launch_tiles<kE5M2>(f, R, C, codes_r, exps_r, codes_c, exps_c, status, s);
}

hipError_t launch_dequantize_fp8(const uint8_t* codes, const uint8_t* exps, int64_t rows, int64_t len, int fmt,
                                 float* y, hipStream_t s) {
  using namespace fp8;
  const int64_t words_row = (len + 3) / 4, words = rows * words_row;
  const dim3 grid((unsigned)((words + 255) / 256));
  if (fmt == kE4M3)
    hipLaunchKernelGGL(k_fp8_values<kE4M3>, grid, dim3(256), 0, s, codes, exps, len, words_row, words, y);
  else
    hipLaunchKernelGGL(k_fp8_values<kE5M2>, grid, dim3(256), 0, s, codes, exps, len, words_row, words, y);
  return hipGetLastError();
}

}  // namespace fastbfp
