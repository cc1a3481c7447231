// fp8.h -- 8-bit floating-point blocks: e4m3 or e5m2 codes (OCP 8-bit floating point)
// with one power-of-two scale for each 128 consecutive values of a row, the E8M0 block
// scale of gfx950's MFMA of K = 128 (shared by its four blocks of 32).
//
// The scale of a block is the least power of two by which its largest value is at most
// the format's, 448 = 1.75 * 2^8 (57344 = 1.75 * 2^15): with the FP32 exponent field E of
// the largest magnitude, 2^(E - 127 - 8), or twice that where its fraction is above 0.75.
// So no value is beyond the format, and codes are the hardware converter's nearest-even
// ones of x / scale, an exact power-of-two scaling.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fastbfp {

namespace fp8 {

enum { kE4M3 = 0, kE5M2 = 1 };  // (the MFMA's format codes; bfp_fp8_t)

constexpr int kBlock = 128;

__host__ __device__ constexpr int64_t blocks_of(int64_t len) { return (len + kBlock - 1) / kBlock; }
// Bytes from one row's codes, or scales, to the next one's.
__host__ __device__ constexpr int64_t code_pitch(int64_t len) { return blocks_of(len) * kBlock; }
__host__ __device__ constexpr int64_t exp_pitch(int64_t len) { return (blocks_of(len) + 3) / 4 * 4; }

typedef float v4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint16_t h2 __attribute__((ext_vector_type(2)));
typedef short s2 __attribute__((ext_vector_type(2)));
typedef __bf16 b4 __attribute__((ext_vector_type(4)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef uint16_t bf16_t;  // a BF16 value's bits, the upper half of an FP32's

// Four values as they are in memory.
template <class T> struct Raw;
template <> struct Raw<float> { typedef u4 type; };
template <> struct Raw<bf16_t> { typedef u2 type; };
// Their FP32 bits.
__device__ __forceinline__ u4 wide(const u4& v) { return v; }
__device__ __forceinline__ u4 wide(const u2& v) { return u4{v[0] << 16, v[0] & 0xFFFF0000u, v[1] << 16, v[1] & 0xFFFF0000u}; }

// Magnitude bits of a value as the block's maximum takes them: subnormals, infinities
// and NaN do not count.
__device__ __forceinline__ uint32_t counted(uint32_t bits) {
  const uint32_t a = bits & 0x7FFFFFFFu;
  return a - 0x00800000u < 0x7F000000u ? a : 0u;
}
__device__ __forceinline__ bool finite(uint32_t bits) { return (bits & 0x7FFFFFFFu) < 0x7F800000u; }

// The scale's byte (2^(byte - 127)) for the largest magnitude's bits.
__device__ __forceinline__ uint32_t scale_of(uint32_t amax, int fmt) {
  const int e = (int)(amax >> 23) + ((amax & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return (uint32_t)max(e - (fmt == kE4M3 ? 8 : 15), 0);
}
// 1 / scale, a power of two in FP32's range (the byte is at most 247).
__device__ __forceinline__ float inverse(uint32_t scale) { return __uint_as_float((254u - scale) << 23); }

// What the converter takes for x: subnormals as zero, infinities as NaN.
__device__ __forceinline__ float ready(uint32_t bits, float inv) {
  const uint32_t a = bits & 0x7FFFFFFFu;
  if (a < 0x00800000u) bits &= 0x80000000u;
  if (a >= 0x7F800000u) bits |= 0x7FC00000u;
  return __uint_as_float(bits) * inv;
}

// Codes of four values.
__device__ __forceinline__ uint32_t convert4(const u4& b, float inv, int fmt) {
  const float x0 = ready(b[0], inv), x1 = ready(b[1], inv), x2 = ready(b[2], inv), x3 = ready(b[3], inv);
  if (fmt == kE4M3) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x0, x1, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x2, x3, lo, true);
  }
  const int lo = __builtin_amdgcn_cvt_pk_bf8_f32(x0, x1, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(x2, x3, lo, true);
}

// The quick way through a conversion: `key`, twice the bits of a block's largest magnitude
// as they are, and the hardware's scaled conversion.  It does not hold for blocks with
// infinities or NaN, or whose scale would show FP32 subnormals as more than zero
// (a subnormal over 2^(18 - 127) is below half of e5m2's least value, 2^-17).  It does for
// blocks of zeros, and of rows or blocks that are not there, whose scale byte is 0: their
// codes are the zeros' signs by any scale (kQuickLeast's in quick4).
constexpr uint32_t kQuickLeast = 19;
__device__ __forceinline__ uint32_t key4(const u4& b) {
  return max(max(b[0] << 1, b[1] << 1), max(b[2] << 1, b[3] << 1));
}
__device__ __forceinline__ uint32_t key4(const u2& b) {
  const h2 x = __builtin_bit_cast(h2, b[0] & 0x7FFF7FFFu), y = __builtin_bit_cast(h2, b[1] & 0x7FFF7FFFu);
  const h2 m = __builtin_elementwise_max(x, y);
  return (uint32_t)max(m[0], m[1]) << 17;
}
__device__ __forceinline__ bool key_finite(uint32_t key) { return key < 0xFF000000u; }
__device__ __forceinline__ bool quick(uint32_t key, uint32_t scale) {
  return key == 0u || (key_finite(key) && scale >= kQuickLeast);
}

template <int FMT>
__device__ __forceinline__ uint32_t quick4(const u4& b, uint32_t scale) {
  const float f = __uint_as_float(max(scale, kQuickLeast) << 23);
  const float x0 = __uint_as_float(b[0]), x1 = __uint_as_float(b[1]), x2 = __uint_as_float(b[2]), x3 = __uint_as_float(b[3]);
  s2 r{};
  if constexpr (FMT == kE4M3) {
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, x0, x1, f, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, x2, x3, f, true);
  } else {
    r = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(r, x0, x1, f, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(r, x2, x3, f, true);
  }
  return __builtin_bit_cast(uint32_t, r);
}
template <int FMT>
__device__ __forceinline__ uint32_t quick4(const u2& b, uint32_t scale) {
  const float f = __uint_as_float(max(scale, kQuickLeast) << 23);
  const uint32_t lo = b[0], hi = b[1];  // (of b[1] itself the compiler's bit cast takes b[0])
  const b2 x = __builtin_bit_cast(b2, lo), y = __builtin_bit_cast(b2, hi);
  s2 r{};
  if constexpr (FMT == kE4M3) {
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, x, f, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, y, f, true);
  } else {
    r = __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(r, x, f, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(r, y, f, true);
  }
  return __builtin_bit_cast(uint32_t, r);
}

template <int CTRL>
__device__ __forceinline__ uint32_t max_dpp(uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false));
}
// The maximum over the 32 lanes of a half wave, in all of them.
__device__ __forceinline__ uint32_t max_half_wave(uint32_t v) {
  v = max_dpp<0xB1>(v);   // quad_perm 1 0 3 2
  v = max_dpp<0x4E>(v);   // quad_perm 2 3 0 1
  v = max_dpp<0x141>(v);  // mirrored within eight lanes
  v = max_dpp<0x140>(v);  // mirrored within sixteen
  // (rows of 16 lanes: of each pair the first one's in both, and the second one's)
  typedef uint32_t pair __attribute__((ext_vector_type(2)));
  const pair p = __builtin_bit_cast(pair, __builtin_amdgcn_permlane16_swap(v, v, false, false));
  return max(p[0], p[1]);
}
__device__ __forceinline__ uint32_t max4(const u4& b) {
  return max(max(counted(b[0]), counted(b[1])), max(counted(b[2]), counted(b[3])));
}


// A block along a row, four values a lane of half a wave: its codes, and in `scale` its
// scale's byte; bad: whether the lane has an infinity or NaN.
template <int FMT, class V>
__device__ __forceinline__ uint32_t convert_block(const V& v, uint32_t& scale, bool& bad) {
  const uint32_t key = max_half_wave(key4(v));
  scale = scale_of(key >> 1, FMT);
  bad = false;
  if (quick(key, scale)) return quick4<FMT>(v, scale);
  const u4 b = wide(v);
  scale = scale_of(max_half_wave(max4(b)), FMT);
#pragma unroll
  for (int t = 0; t < 4; ++t) bad |= !finite(b[t]);
  return convert4(b, inverse(scale), FMT);
}

// N blocks at once, with one branch for all of them.
template <int FMT, int N, class V>
__device__ __forceinline__ void convert_blocks(const V (&v)[N], uint32_t (&code)[N], uint32_t (&scale)[N], bool& bad) {
  bool all = true;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t key = max_half_wave(key4(v[i]));
    scale[i] = scale_of(key >> 1, FMT);
    all &= quick(key, scale[i]);
  }
  bad = false;
  if (all) {
#pragma unroll
    for (int i = 0; i < N; ++i) code[i] = quick4<FMT>(v[i], scale[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      bool b;
      code[i] = convert_block<FMT>(v[i], scale[i], b);
      bad |= b;
    }
  }
}

// Four values from `left` (of a row) on, as they are: those past the row's end are zeros.
// Rows of any length begin at any multiple of a value's bytes.
__device__ __forceinline__ u4 raw4(const float* p, int64_t left) {
  typedef u4 __attribute__((aligned(4))) u4_any;
  if (left >= 4) return *reinterpret_cast<const u4_any*>(p);
  u4 v = u4{0u, 0u, 0u, 0u};
#pragma unroll
  for (int t = 0; t < 3; ++t)
    if (t < left) v[t] = __float_as_uint(p[t]);
  return v;
}
__device__ __forceinline__ u2 raw4(const bf16_t* p, int64_t left) {
  typedef u2 __attribute__((aligned(2))) u2_any;
  if (left >= 4) return *reinterpret_cast<const u2_any*>(p);
  u2 v = u2{0u, 0u};
#pragma unroll
  for (int t = 0; t < 3; ++t)
    if (t < left) v[t / 2] |= (uint32_t)p[t] << (16 * (t & 1));
  return v;
}
// Four values moved down by `n` places (0 to 3), zeros behind them.
__device__ __forceinline__ u4 down(u4 v, int n) {
  if (n & 1) v = u4{v[1], v[2], v[3], 0u};
  if (n & 2) v = u4{v[2], v[3], 0u, 0u};
  return v;
}
__device__ __forceinline__ u2 down(const u2& v, int n) {
  return __builtin_bit_cast(u2, __builtin_bit_cast(uint64_t, v) >> (16 * n));
}
// Their FP32 bits.
template <class T>
__device__ __forceinline__ u4 load4(const T* p, int64_t left) { return wide(raw4(p, left)); }
// Stores four values, rounded to the nearest (ties to even) for BF16.
__device__ __forceinline__ void store4(float* p, const u4& v, int64_t left) {
  typedef u4 __attribute__((aligned(4))) u4_any;
  if (left >= 4) {
    *reinterpret_cast<u4_any*>(p) = v;
    return;
  }
#pragma unroll
  for (int t = 0; t < 3; ++t)
    if (t < left) p[t] = __uint_as_float(v[t]);
}
__device__ __forceinline__ u2 to_bf16(const u4& v) {
  b4 b;
#pragma unroll
  for (int t = 0; t < 4; ++t) b[t] = (__bf16)__uint_as_float(v[t]);
  return __builtin_bit_cast(u2, b);
}
__device__ __forceinline__ void store4(bf16_t* p, const u4& v, int64_t left) {
  typedef u2 __attribute__((aligned(2))) u2_any;
  const u2 b = to_bf16(v);
  if (left >= 4) {
    *reinterpret_cast<u2_any*>(p) = b;
    return;
  }
#pragma unroll
  for (int t = 0; t < 3; ++t)
    if (t < left) p[t] = (bf16_t)(b[t / 2] >> (16 * (t & 1)));
}

// Eight of them.
__device__ __forceinline__ void store8(bf16_t* p, const u4& x, const u4& y, int64_t left) {
  typedef u4 __attribute__((aligned(2))) u4_any;
  if (left >= 8) {
    const u2 a = to_bf16(x), b = to_bf16(y);
    *reinterpret_cast<u4_any*>(p) = u4{a[0], a[1], b[0], b[1]};
    return;
  }
  store4(p, x, left);
  store4(p + 4, y, left - 4);
}

}  // namespace fp8

}  // namespace fastbfp
