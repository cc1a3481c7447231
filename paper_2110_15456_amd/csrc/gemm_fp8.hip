// gemm_fp8.hip -- C = A . B^T on 8-bit floating-point blocks (fp8.h):
//   C[i][j] = sum over blocks b of 2^(ea[i][b] + eb[j][b] - 254) sum over k in b of a[i][k] b[j][k]
// on v_mfma_scale_f32_32x32x64_f8f6f4, whose E8M0 scales are the blocks' own.
//
// Accuracy.  Products are exact.  The MFMA aligns the products of eight consecutive k to the
// largest of them and drops what lies below 2^-13 of it (measured with two products: the
// smaller one is kept whole down to 2^-13 of the larger among eight, and down to 2^-23
// beside another eight or the running sum); the eights' sums and C are FP32.  So C is off
// by about 2^-14 of the products' size at random, whatever K: a fraction of BF16's
// rounding, and 1/500 of what e4m3's rounding of a value does.
#include "fp8.h"
#include "launch.h"

namespace fastbfp {

namespace fp8 {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v16 __attribute__((ext_vector_type(16)));
typedef __amdgpu_buffer_rsrc_t rsrc_t;
typedef __attribute__((address_space(3))) void lds_void;

struct Gemm {
  const uint8_t *a, *ea, *b, *eb;
  int M, N, slabs;         // slabs: blocks of K
  uint32_t pitch, epitch;  // of a row's codes and scales
  void* c;                 // FP32, or BF16 (a part's sums: FP32)
  int64_t ldc;
  int tiles_m, tiles_n;
  int part_slabs;          // slabs of a part of K; part p goes to c + p * part_stride
  int64_t part_stride;
};

__device__ __forceinline__ rsrc_t make_rsrc(const uint8_t* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), (short)0, (int)bytes, 0x00020000);
}

// Workgroup -> item: contiguous runs of items on each XCD.
__device__ __forceinline__ int xcd_order(int bid, int n) {
  const int xcd = bid % 8;
  return xcd * (n / 8) + min(xcd, n % 8) + bid / 8;
}

// BM x BN tiles, WGM x WGN waves; a slab is one block of K, 128 bytes of every row,
// brought by direct buffer -> LDS loads of 1 KB into one of two stages while the other
// is computed on.  16-byte chunk c of row r sits at chunk c ^ ((r >> 1) & 7): 16 lanes
// that read one chunk of 16 rows hit all 64 banks.  Rows past the end read zeros (the
// buffer resources end at the last row).  A lane's scales are those of its rows, four
// slabs in a dword.
template <int BM, int BN, int WGM, int WGN, int FA, int FB, class T>
__global__ __launch_bounds__(64 * WGM * WGN, 2) void k_gemm_fp8(Gemm p) {
  constexpr int NW = WGM * WGN, WM = BM / WGM, WN = BN / WGN, TM = WM / 32, TN = WN / 32;
  constexpr int OFF_B = BM * kBlock, STAGE = OFF_B + BN * kBlock;
  static_assert((BM / 8) % NW == 0 && (BN / 8) % NW == 0 && NW % 2 == 0, "loads split evenly over the waves");
  __shared__ __attribute__((aligned(128))) uint8_t stage0[STAGE];
  __shared__ __attribute__((aligned(128))) uint8_t stage1[STAGE];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int wr = wave / WGN, wc = wave % WGN;

  const int tiles = p.tiles_m * p.tiles_n, id = xcd_order(blockIdx.x, gridDim.x), part = id / tiles, t = id % tiles;
  // bands of four tile rows, down each band's column first: the tiles that an XCD runs
  // at once share rows of A and of B
  const int band = t / (4 * p.tiles_n), in = t % (4 * p.tiles_n), rows = min(4, p.tiles_m - 4 * band);
  const int row0 = (4 * band + in % rows) * BM, col0 = in / rows * BN;
  const int slab0 = part * p.part_slabs, nslabs = min(p.part_slabs, p.slabs - slab0);

  const int arows = min(BM, p.M - row0), brows = min(BN, p.N - col0);
  const rsrc_t ra = make_rsrc(p.a + (int64_t)row0 * p.pitch, (uint32_t)arows * p.pitch);
  const rsrc_t rb = make_rsrc(p.b + (int64_t)col0 * p.pitch, (uint32_t)brows * p.pitch);
  const rsrc_t rea = make_rsrc(p.ea + (int64_t)row0 * p.epitch, (uint32_t)arows * p.epitch);
  const rsrc_t reb = make_rsrc(p.eb + (int64_t)col0 * p.epitch, (uint32_t)brows * p.epitch);

  v16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = v16{};

  const uint32_t chunk = (uint32_t)((lane & 7) ^ ((4 * (wave & 1) + (lane >> 4)) & 7)) * 16;
  auto issue = [&](uint8_t* stage, int s) __attribute__((always_inline)) {
    const uint32_t k0 = (uint32_t)(slab0 + s) * kBlock + chunk;
#pragma unroll
    for (int u = 0; u < BM / 8 / NW; ++u) {
      const int blk = wave + NW * u;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_void*)(stage + blk * 1024), 16,
                                               (uint32_t)(8 * blk + (lane >> 3)) * p.pitch + k0, 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < BN / 8 / NW; ++u) {
      const int blk = wave + NW * u;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_void*)(stage + OFF_B + blk * 1024), 16,
                                               (uint32_t)(8 * blk + (lane >> 3)) * p.pitch + k0, 0, 0, 0);
    }
  };
  const int fr = lane & 31, fk = lane >> 5, fsw = (fr >> 1) & 7;
  auto frag = [&](const uint8_t* tile, int r, int h) __attribute__((always_inline)) -> v8i {
    const uint8_t* at = tile + (r + fr) * kBlock;
    const u4 x = *reinterpret_cast<const u4*>(at + (((4 * h + 2 * fk) ^ fsw) * 16));
    const u4 y = *reinterpret_cast<const u4*>(at + (((4 * h + 2 * fk + 1) ^ fsw) * 16));
    return v8i{(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)y[0], (int)y[1], (int)y[2], (int)y[3]};
  };
  // the scales of slab s, one byte for each of the lane's rows
  auto scales = [&](int s, int (&sa)[TM], int (&sb)[TN]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
      sa[i] = (int)__builtin_amdgcn_raw_buffer_load_b8(rea, (uint32_t)(wr * WM + 32 * i + fr) * p.epitch + slab0 + s, 0, 0);
#pragma unroll
    for (int j = 0; j < TN; ++j)
      sb[j] = (int)__builtin_amdgcn_raw_buffer_load_b8(reb, (uint32_t)(wc * WN + 32 * j + fr) * p.epitch + slab0 + s, 0, 0);
  };
  int sa[TM], sb[TN], na[TM], nb[TN];
  auto step = [&](const uint8_t* cur, uint8_t* nxt, int s) __attribute__((always_inline)) {
    // this wave's loads of slab s have landed and its reads of slab s - 1 are done
    __builtin_amdgcn_s_waitcnt(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int i = 0; i < TM; ++i) sa[i] = na[i];
#pragma unroll
    for (int j = 0; j < TN; ++j) sb[j] = nb[j];
    if (s + 1 < nslabs) {
      scales(s + 1, na, nb);
      issue(nxt, s + 1);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      v8i b[TN];
#pragma unroll
      for (int j = 0; j < TN; ++j) b[j] = frag(cur + OFF_B, wc * WN + 32 * j, h);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const v8i a = frag(cur, wr * WM + 32 * i, h);
#pragma unroll
        for (int j = 0; j < TN; ++j)  // (B first: a lane's quads are columns of a row)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b[j], a, acc[i][j], FB, FA, 0, sb[j], 0, sa[i]);
      }
    }
  };
  scales(0, na, nb);
  issue(stage0, 0);
  int s = 0;
  for (; s + 2 <= nslabs; s += 2) {
    step(stage0, stage1, s);
    step(stage1, stage0, s + 1);
  }
  if (s < nslabs) step(stage0, stage1, s);

  // A lane holds columns 8 q + 4 fk .. + 3 of row fr of each 32 x 32 tile.
  T* C = static_cast<T*>(p.c) + part * p.part_stride;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int r = row0 + wr * WM + 32 * i + fr;
    if (r >= p.M) continue;
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = col0 + wc * WN + 32 * j + 8 * q + 4 * fk;
        u4 v;
#pragma unroll
        for (int t = 0; t < 4; ++t) v[t] = __float_as_uint(acc[i][j][4 * q + t]);
        store4(C + r * p.ldc + c, v, p.N - c);
      }
  }
}

// C of a product without K.
template <class T>
__global__ __launch_bounds__(256) void k_zero_rows(T* c, int64_t ldc, int N, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) c[i / N * ldc + i % N] = T(0);
}

// C = the sum of the parts' matrices, in order; four columns a thread.
template <class T>
__global__ __launch_bounds__(256) void k_join(const float* __restrict__ src, int parts, int64_t part_stride, int quads,
                                              int64_t n, int N, T* __restrict__ c, int64_t ldc) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  v4 v = *reinterpret_cast<const v4*>(src + 4 * i);
  for (int p = 1; p < parts; ++p) v += *reinterpret_cast<const v4*>(src + p * part_stride + 4 * i);
  const int64_t row = i / quads, col = (i - row * quads) * 4;
  store4(c + row * ldc + col, __builtin_bit_cast(u4, v), N - col);
}

template <int BM, int BN, int WGM, int WGN, class T>
hipError_t launch_tiles(const Gemm& g, int fa, int fb, int parts, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)g.tiles_m * g.tiles_n * parts)), block(64 * WGM * WGN);
  if (fa == kE4M3 && fb == kE4M3) hipLaunchKernelGGL((k_gemm_fp8<BM, BN, WGM, WGN, 0, 0, T>), grid, block, 0, s, g);
  else if (fa == kE4M3) hipLaunchKernelGGL((k_gemm_fp8<BM, BN, WGM, WGN, 0, 1, T>), grid, block, 0, s, g);
  else if (fb == kE4M3) hipLaunchKernelGGL((k_gemm_fp8<BM, BN, WGM, WGN, 1, 0, T>), grid, block, 0, s, g);
  else hipLaunchKernelGGL((k_gemm_fp8<BM, BN, WGM, WGN, 1, 1, T>), grid, block, 0, s, g);
  return hipGetLastError();
}

template <class T>
hipError_t launch_plan(const Fp8Plan& plan, Gemm g, int fa, int fb, T* C, int64_t ldc, float* ws, hipStream_t s) {
  if (g.slabs == 0) {
    const int64_t n = (int64_t)g.M * g.N;
    hipLaunchKernelGGL(k_zero_rows<T>, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, C, ldc, g.N, n);
    return hipGetLastError();
  }
  g.part_slabs = plan.part_slabs;
  g.tiles_m = (g.M + plan.tile - 1) / plan.tile;
  g.tiles_n = (g.N + plan.tile - 1) / plan.tile;
  if (plan.parts == 1) {
    g.c = C, g.ldc = ldc, g.part_stride = 0;
    return plan.tile == 128 ? launch_tiles<128, 128, 2, 2, T>(g, fa, fb, 1, s)
                            : launch_tiles<64, 64, 2, 2, T>(g, fa, fb, 1, s);
  }
  g.c = ws, g.ldc = gemm_plan_ld(g.N), g.part_stride = g.M * g.ldc;
  const hipError_t e = plan.tile == 128 ? launch_tiles<128, 128, 2, 2, float>(g, fa, fb, plan.parts, s)
                                        : launch_tiles<64, 64, 2, 2, float>(g, fa, fb, plan.parts, s);
  if (e != hipSuccess) return e;
  const int64_t n = g.part_stride / 4;
  hipLaunchKernelGGL(k_join<T>, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, ws, plan.parts, g.part_stride,
                     (int)(g.ldc / 4), n, g.N, C, ldc);
  return hipGetLastError();
}

}  // namespace fp8

Fp8Plan fp8_plan(int64_t M, int64_t N, int64_t K, bool room) {
  (void)room;
  const int64_t big = ((M + 127) / 128) * ((N + 127) / 128);
  const int slabs = (int)fp8::blocks_of(K);
  return {big >= 256 ? 128 : 64, slabs, 1};
}

int64_t fp8_plan_ws(const Fp8Plan& plan, int64_t M, int64_t N) {
  return plan.parts > 1 ? plan.parts * M * gemm_plan_ld(N) * 4 : 0;
}

hipError_t launch_gemm_fp8(const Fp8Plan& plan, const uint8_t* a, const uint8_t* ea, int fa, const uint8_t* b,
                           const uint8_t* eb, int fb, int64_t M, int64_t N, int64_t K, void* C, bool bf16, int64_t ldc,
                           float* ws, hipStream_t s) {
  using namespace fp8;
  Gemm g{};
  g.a = a, g.ea = ea, g.b = b, g.eb = eb;
  g.M = (int)M, g.N = (int)N, g.slabs = (int)blocks_of(K);
  g.pitch = (uint32_t)code_pitch(K), g.epitch = (uint32_t)exp_pitch(K);
  return bf16 ? launch_plan(plan, g, fa, fb, static_cast<bf16_t*>(C), ldc, ws, s)
              : launch_plan(plan, g, fa, fb, static_cast<float*>(C), ldc, ws, s);
}

}  // namespace fastbfp
