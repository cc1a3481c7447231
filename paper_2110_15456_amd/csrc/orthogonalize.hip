// orthogonalize.hip -- a step of momentum whose result is orthogonalised by the
// quintic Newton-Schulz iteration:
//   M' = beta M + G,  U = G + beta M' (Nesterov) or M',  X = U / (|U|_F + eps),
//   repeated:  S = X X^T,  X <- (a I + b S + c S^2) X
// with (a, b, c) = (3.4445, -4.7750, 2.0315), which takes every singular value
// of X in (0, 1] towards 1 (into about 0.7 .. 1.2) and leaves the vectors.  (Form and
// coefficients of the Muon optimiser: K. Jordan and others, "Muon: An optimizer for
// hidden layers in neural networks", 2024.)
//
// X is kept with no more rows than columns (n <= k; the transpose of U where it
// has more), so the products are n x n x k, n x n x n and n x k x n.
//
// Steps are taken two at a time.  With P = a I + b S + c S^2 the second step's S is
// P S P, so X is needed twice for both, for S = X X^T and X <- P' P X, and in between
// there are products of symmetric n x n matrices that commute (all are polynomials
// of S), of which one triangle is computed.  In units of n^2 multiply-adds two
// steps alone take 6 k + 2 n and a pair 3 k + 5 n: five steps of k = 4 n, in two
// pairs and one, 47 n instead of 65; the same at k = n.  Rounding allows no more:
// what P S P misses of the next X X^T grows by a^2 in each step of a group.  Over
// noise, strong directions over noise, power laws, six decades of singular values
// and two levels of them 1 to 10^5 apart, pairs had 0.7 to 2.4 times the error of
// evaluating the formula in FP32 (single steps 0.6 to 2.5), groups of three up to
// 12 times and five in one 40 times and more.
//
// Arithmetic.  The iteration grows small singular values by up to a^5 = 485,
// and the errors of the products with them, so they are computed to FP32
// accuracy: every matrix is two FP16 planes, hi = fp16(x 2^s) and lo = fp16(x 2^s
// - hi), which hold 22 bits, and a product is the three MFMAs hi hi + hi lo + lo hi
// (lo lo is below 2^-22 of it) accumulated in FP32.  Three passes at the FP16 rate
// (2.5 PFLOP/s) take a fifth of the time of FP32 MFMAs (157 TFLOP/s).  The scales
// 2^s put the largest entry a matrix can have just below FP16's end, since X's
// singular values stay below 1.21 (the polynomial's maximum on [0, 1], and again
// on [0, 1.21]): |X| < 1.21 and |S| < 1.47 at 2^15, |P| < 3.5 at 2^14.
// FP16 ends at 2^-24, though, so an entry is held to 2^-23 of itself or (of X) 2^-40 at
// least: rows or columns 2^-20 and more below the rest lose what FP32 would keep of
// them (rows at 10^-6 of the others, 1024 x 4096: 8e-4 of themselves after five steps,
// FP32 5e-7; of the matrix 1.1e-6, FP32 4.2e-6).  That is this layout's price: planes
// with an exponent range of their own would be three of BF16 and six MFMAs.
//
// Layout ("planes"): rows of blocks of 32 columns, a block 128 bytes, 32 hi then
// 32 lo: one line holds what a K slab of 32 needs of a row.
#include <hip/hip_runtime.h>

#include <utility>

#include "launch.h"

namespace fastbfp {

namespace ns {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr int kXScale = 15, kSScale = 15, kPScale = 14, kQScale = 12;

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef float v4 __attribute__((ext_vector_type(4)));
typedef float v16 __attribute__((ext_vector_type(16)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef __amdgpu_buffer_rsrc_t rsrc_t;
typedef __attribute__((address_space(3))) void lds_void;

constexpr int KS = 32;      // columns of a block, and of a K slab
constexpr int BLOCK = 128;  // its bytes

__host__ __device__ constexpr int64_t blocks_of(int64_t cols) { return (cols + KS - 1) / KS; }

__device__ __forceinline__ rsrc_t make_rsrc(const uint8_t* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), (short)0, (int)bytes, 0x00020000);
}

template <int I> struct ic { static constexpr int value = I; };
template <int N, int I = 0, class F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (I < N) {
    f(ic<I>{});
    static_for<N, I + 1>(f);
  }
}

// What a product writes: planes of a symmetric matrix, alpha sum + beta m + gamma I,
// of the lower triangle's tiles and mirrored; planes; FP32; FP32 transposed.
enum { kSym, kPlanes, kF32, kF32T };

struct Gemm {
  const uint8_t* a;  // planes, rows x blocks_k
  int64_t a_batch;
  const uint8_t* b;  // planes: rows of the product's columns (TR: X itself, rows of its K)
  int64_t b_batch;
  int M, N, K;       // C is M x N
  int tiles_m, tiles_n;  // (kSym: tiles_m alone, the lower triangle's tiles)
  float alpha;
  uint8_t* c;        // planes, or FP32; rows of ldc values
  int64_t c_batch;
  int ldc;
  // kSym
  const uint8_t* m;  // planes as c's, or null
  float beta, gamma;
  int whole;         // tiles (of all matrices) from here on are summed in parts of K
  int parts, part_slabs;
  float* sums;       // [tile - whole][part][BM][BN]
};

// 16 bytes of a plane: hi or lo of eight values.
__device__ __forceinline__ void store_chunk(uint8_t* o, const float (&x)[8], bool lo) {
  h8 v;
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    const _Float16 h = (_Float16)x[t];
    v[t] = lo ? (_Float16)(x[t] - (float)h) : h;
  }
  *reinterpret_cast<h8*>(o) = v;
}

// Tile t of a lower triangle, row by row.
__device__ __forceinline__ void triangle_tile(int t, int& tm, int& tn) {
  tm = (int)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
  while (tm * (tm + 1) / 2 > t) --tm;
  while ((tm + 1) * (tm + 2) / 2 <= t) ++tm;
  tn = t - tm * (tm + 1) / 2;
}

// Workgroup -> item: contiguous runs of items on each XCD.
__device__ __forceinline__ int xcd_order(int bid, int n) {
  const int xcd = bid % 8;
  return xcd * (n / 8) + min(xcd, n % 8) + bid / 8;
}

// C = A B^T (or A X with TR: B's tile is rows of K, read transposed from LDS) on
// BM x BN tiles, WGM x WGN waves.
//
// A slab is 32 of K: 128 bytes of every row of A and B (of 32 rows of X with TR),
// brought by direct buffer -> LDS loads of 1 KB each into one of two stages while
// the other is computed on.  16-byte chunk c of row r sits at chunk c ^ ((r >> 1) & 7):
// 16 lanes that read one chunk of 16 rows hit all 64 banks.  With TR a tile row
// holds BN columns, and 32-byte unit u of row r sits at u ^ (2 (r & 3)), so that
// the four rows x 32 columns of two lane groups of a transposed read do.  Rows past
// the end read zeros (the buffer resources end at the last row).
//
// A wave's tile is 128 x 64, 64 x 64 or, on the 64 tile, 32 x 32: per slab 24 (16, 8)
// KB of fragments for 48 (24, 6) MFMAs of 32x32x16, i.e. the LDS is busy a half (two
// thirds, four thirds) of the time that the matrix cores are.
//
// ST stages: two, or four for few 64 tiles of few slabs, where the loads' latency is
// what a slab takes (0.5 us) and nearly all of them can be on the way at once: the
// update of 256 x 256 went from 135 to 126 us, of 384 x 1536 from 190 to 177; with 16
// and more slabs, and on the 128 tile, it gained nothing.
//
// Large products are bound by power: the clock falls to 1.7 .. 1.85 GHz (of 2.4) with
// the matrix cores busy 60 to 65 % of the cycles.  Q X of 4096 x 16384 takes 1.36 to
// 1.47 ms, i.e. 1.12 to 1.21 PFLOP/s of FP16; a library's FP16 product of 8192^3
// reached 1.15 on the same card.  Reading a slab's first fragments before the last one's
// barrier changed nothing.
template <int BM, int BN, int WGM, int WGN, bool TR, int OUT, int ST>
__global__ __launch_bounds__(64 * WGM * WGN, BM == 64 && ST == 2 ? 4 : 2) void k_ns_gemm(Gemm p) {
  constexpr int NW = WGM * WGN, WM = BM / WGM, WN = BN / WGN, TM = WM / 32, TN = WN / 32;
  constexpr int OFF_B = BM * BLOCK, STAGE = OFF_B + BN * BLOCK;
  static_assert((BM / 8) % NW == 0 && (BN / 8) % NW == 0 && NW % 2 == 0, "loads split evenly over the waves");
  __shared__ __attribute__((aligned(128))) uint8_t stage0[STAGE];
  __shared__ __attribute__((aligned(128))) uint8_t stage1[STAGE];
  __shared__ __attribute__((aligned(128))) uint8_t stage2[ST == 4 ? STAGE : 16];
  __shared__ __attribute__((aligned(128))) uint8_t stage3[ST == 4 ? STAGE : 16];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int wr = wave / WGN, wc = wave % WGN;

  int tm, tn, slab0 = 0, nslabs = (int)blocks_of(p.K);
  int64_t batch;
  float* sums = nullptr;  // where the sums of a part go
  if constexpr (OUT == kSym) {
    const int bid = blockIdx.x, tiles = p.tiles_m * (p.tiles_m + 1) / 2;
    int t = bid;
    if (bid < p.whole) {
      t = xcd_order(bid, p.whole);
    } else {
      const int part = (bid - p.whole) % p.parts;
      t = p.whole + (bid - p.whole) / p.parts;
      slab0 = part * p.part_slabs;
      nslabs = min(p.part_slabs, nslabs - slab0);
      sums = p.sums + (int64_t)(bid - p.whole) * (BM * BN);
    }
    triangle_tile(t % tiles, tm, tn);
    batch = t / tiles;
  } else {
    // bands of four tile rows, down each band's column first: the tiles that an
    // XCD runs at once share rows of A and columns of X
    const int id = xcd_order(blockIdx.x, gridDim.x), tiles = p.tiles_m * p.tiles_n, t = id % tiles;
    batch = id / tiles;
    const int band = t / (4 * p.tiles_n), in = t % (4 * p.tiles_n), rows = min(4, p.tiles_m - 4 * band);
    tm = 4 * band + in % rows;
    tn = in / rows;
  }
  const int row0 = tm * BM, col0 = tn * BN;
  const uint32_t a_row = (uint32_t)blocks_of(p.K) * BLOCK;
  const uint32_t b_row = TR ? (uint32_t)blocks_of(p.N) * BLOCK : a_row;
  const uint8_t* A = p.a + batch * p.a_batch + (int64_t)row0 * a_row;
  const rsrc_t ra = make_rsrc(A, (uint32_t)min(BM, p.M - row0) * a_row);
  const uint8_t* B = p.b + batch * p.b_batch + (TR ? (int64_t)col0 * 4 : (int64_t)col0 * b_row);
  const rsrc_t rb = make_rsrc(B, TR ? (uint32_t)p.K * b_row - (uint32_t)col0 * 4 : (uint32_t)min(BN, p.N - col0) * b_row);

  // The sums of hi hi and, on the 64 tile, those of hi lo + lo hi beside them, which then
  // are rounded at their own size, 2^-11 of the other (all of it in one: 30% more error on
  // 256 x 512 to 2048 x 2048, and no faster; larger tiles have no registers left).
  constexpr bool APART = BM == 64;
  v16 acc[TM][TN], cross[APART ? TM : 1][APART ? TN : 1];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      acc[i][j] = v16{};
      if constexpr (APART) cross[i][j] = v16{};
    }

  const uint32_t chunk = (uint32_t)((lane & 7) ^ ((4 * (wave & 1) + (lane >> 4)) & 7));
  const uint32_t ab_lane = chunk * 16;  // (rows of A, and of B without TR)
  auto issue = [&](uint8_t* stage, int s) __attribute__((always_inline)) {
    const uint32_t k0 = (uint32_t)(slab0 + s) * BLOCK;
#pragma unroll
    for (int u = 0; u < BM / 8 / NW; ++u) {
      const int blk = wave + NW * u;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_void*)(stage + blk * 1024), 16,
                                               (uint32_t)(8 * blk + (lane >> 3)) * a_row + ab_lane + k0, 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < BN / 8 / NW; ++u) {
      const int blk = wave + NW * u;
      uint32_t off;
      if constexpr (TR) {
        constexpr int LR = BN / 4;  // lanes of a tile row (4 BN bytes)
        const int r = blk * (64 / LR) + lane / LR, q = lane % LR;
        off = (uint32_t)((slab0 + s) * KS + r) * b_row + (uint32_t)(((q >> 1) ^ (2 * (r & 3))) * 32 + (q & 1) * 16);
      } else {
        off = (uint32_t)(8 * blk + (lane >> 3)) * b_row + ab_lane + k0;
      }
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_void*)(stage + OFF_B + blk * 1024), 16, off, 0, 0, 0);
    }
  };
  const int fr = lane & 31, fk = lane >> 5, fsw = (fr >> 1) & 7;
  auto frag = [&](const uint8_t* tile, int r, int h, int pl) __attribute__((always_inline)) -> h8 {
    return *reinterpret_cast<const h8*>(tile + (r + fr) * BLOCK + (((pl * 4 + 2 * h + fk) ^ fsw) * 16));
  };
  const int tr_k = 8 * fk + ((lane >> 2) & 3), tr_sw = 2 * ((lane >> 2) & 3), tr_u = (lane >> 4) & 1;
  auto frag_tr = [&](const uint8_t* tile, int c, int h, int pl) __attribute__((always_inline)) -> h8 {
    const uint8_t* at = tile + (16 * h + tr_k) * (BN * 4) + ((((c / 32) * 4 + pl * 2 + tr_u) ^ tr_sw) * 32) + (lane & 3) * 8;
    const s4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)(at));
    const s4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)(at + 4 * BN * 4));
    return __builtin_bit_cast(h8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  auto mma = [&](v16& c, const h8& a, const h8& b) __attribute__((always_inline)) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_f16(b, a, c, 0, 0, 0);  // (B first: a lane's quads are columns of a row)
  };
  auto step = [&](const uint8_t* cur, uint8_t* nxt, int s) __attribute__((always_inline)) {
    // this wave's loads of slab s have landed (those of the ST - 2 after it may be on
    // the way) and its reads of slab s - 1 are done
    constexpr int YOUNGER = (ST - 2) * ((BM + BN) / 8 / NW);
    if (ST > 2 && s + ST - 1 <= nslabs)
      __builtin_amdgcn_s_waitcnt((YOUNGER & 15) | ((YOUNGER >> 4) << 14) | (7 << 4));  // vmcnt(YOUNGER) lgkmcnt(0)
    else
      __builtin_amdgcn_s_waitcnt(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (s + ST - 1 < nslabs) issue(nxt, s + ST - 1);
    static_for<2>([&](auto hc) __attribute__((always_inline)) {
      constexpr int h = decltype(hc)::value;
      h8 b[TN][2];
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int pl = 0; pl < 2; ++pl)
          b[j][pl] = TR ? frag_tr(cur + OFF_B, wc * WN + 32 * j, h, pl) : frag(cur + OFF_B, wc * WN + 32 * j, h, pl);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const h8 hi = frag(cur, wr * WM + 32 * i, h, 0), lo = frag(cur, wr * WM + 32 * i, h, 1);
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          if constexpr (APART) mma(cross[i][j], lo, b[j][0]);
          else mma(acc[i][j], lo, b[j][0]);
        }
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          if constexpr (APART) mma(cross[i][j], hi, b[j][1]);
          else mma(acc[i][j], hi, b[j][1]);
        }
#pragma unroll
        for (int j = 0; j < TN; ++j) mma(acc[i][j], hi, b[j][0]);
      }
    });
  };
  issue(stage0, 0);
  int s = 0;
  if constexpr (ST == 2) {
    for (; s + 2 <= nslabs; s += 2) {
      step(stage0, stage1, s);
      step(stage1, stage0, s + 1);
    }
    if (s < nslabs) step(stage0, stage1, s);
  } else {
    if (nslabs > 1) issue(stage1, 1);
    if (nslabs > 2) issue(stage2, 2);
    for (; s + 4 <= nslabs; s += 4) {
      step(stage0, stage3, s);
      step(stage1, stage0, s + 1);
      step(stage2, stage1, s + 2);
      step(stage3, stage2, s + 3);
    }
    if (s < nslabs) step(stage0, stage3, s);
    if (s + 1 < nslabs) step(stage1, stage0, s + 1);
    if (s + 2 < nslabs) step(stage2, stage1, s + 2);
  }

  // Epilogue.  A lane holds columns 8 q + 4 fk .. + 3 of row fr of each 32 x 32
  // tile.  64 x 64 values at a time go through the wave's 16 KB of the stages, so
  // that rows and, mirrored, columns leave as whole lines.  16-byte granule g of row r
  // sits at g ^ swz(r): 16 rows of one granule, and 8 rows 8 apart, on all banks.
  // (On the 64 tile the four waves' 32 x 32 are one such piece, of which each
  // writes a quarter.)
  if constexpr (APART) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] += cross[i][j];
  }
  __syncthreads();
  constexpr bool JOIN = BM == 64;
  static_assert(JOIN ? BN == 64 && NW == 4 && STAGE == 16384
                     : WN == 64 && TM % 2 == 0 && NW * 16384 <= 2 * STAGE, "the sums fit in the stages");
  constexpr int HI = JOIN ? 1 : 2, ITS = JOIN ? 4 : 16;  // 32-row pieces of a wave's share, its lines / 4
  float* tile = reinterpret_cast<float*>(JOIN ? stage0
                                              : (wave < NW / 2 ? stage0 : stage1) + (wave % (NW / 2)) * 16384);
  const int pr = JOIN ? wr * 32 : 0, pg = JOIN ? wc * 8 : 0, it0 = JOIN ? wave * ITS : 0;
  auto at = [](int r, int g) __attribute__((always_inline)) -> int { return r * 64 + ((g ^ ((r ^ (r >> 3)) & 15)) * 4); };
  uint8_t* C = p.c + batch * p.c_batch;
  const float alpha = OUT == kSym && sums ? 1.0f : p.alpha;
#pragma unroll
  for (int half = 0; half < (JOIN ? 1 : TM / 2); ++half) {
#pragma unroll
    for (int i = 0; i < HI; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          v4 v;
#pragma unroll
          for (int t = 0; t < 4; ++t) v[t] = acc[HI * half + i][j][4 * q + t] * alpha;
          *reinterpret_cast<v4*>(&tile[at(pr + 32 * i + fr, pg + 8 * j + 2 * q + fk)]) = v;
        }
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): the wave reads back what it wrote
    if constexpr (JOIN) __syncthreads();
    else __builtin_amdgcn_wave_barrier();
    const int r0 = JOIN ? row0 : row0 + wr * WM + 64 * half, c0 = JOIN ? col0 : col0 + wc * WN;
    auto row8 = [&](int r, int c, float (&x)[8]) __attribute__((always_inline)) {
      const v4 a = *reinterpret_cast<const v4*>(&tile[at(r, c / 4)]), b = *reinterpret_cast<const v4*>(&tile[at(r, c / 4 + 1)]);
#pragma unroll
      for (int t = 0; t < 4; ++t) x[t] = a[t], x[4 + t] = b[t];
    };
    auto col8 = [&](int r, int c, float (&x)[8]) __attribute__((always_inline)) {  // rows r .. r + 7 of column c
#pragma unroll
      for (int t = 0; t < 8; ++t) x[t] = tile[at(r + t, c / 4) + (c & 3)];
    };
    if (OUT == kSym && sums) {
      float* o = sums + (r0 - row0) * BN + (c0 - col0);
#pragma unroll 4
      for (int it = it0; it < it0 + ITS; ++it) {
        const int r = 4 * it + (lane >> 4), c = 4 * (lane & 15);
        *reinterpret_cast<v4*>(o + r * BN + c) = *reinterpret_cast<const v4*>(&tile[at(r, c / 4)]);
      }
    } else if constexpr (OUT == kSym || OUT == kPlanes) {
      const int64_t line = (int64_t)(p.ldc / KS) * BLOCK;
      const uint8_t* m = OUT == kSym && p.m ? p.m + batch * p.c_batch : nullptr;
      for (int mirror = 0; mirror < (OUT == kSym && tm != tn ? 2 : 1); ++mirror) {
        const int ro = mirror ? c0 : r0, co = mirror ? r0 : c0, rows = mirror ? p.N : p.M;
#pragma unroll 4
        for (int it = it0; it < it0 + ITS; ++it) {
          const int r = 4 * it + (lane >> 4), blk = (lane >> 3) & 1, lo = (lane >> 2) & 1, k = lane & 3;
          const int c = blk * KS + 8 * k;
          if (ro + r >= rows || co + c >= p.ldc) continue;
          float x[8];
          if (mirror) col8(c, r, x);
          else row8(r, c, x);
          const int64_t o = (int64_t)(ro + r) * line + (co + c) / KS * BLOCK + k * 16;
          if constexpr (OUT == kSym) {
            if (m) {
              const h8 h = *reinterpret_cast<const h8*>(m + o), l = *reinterpret_cast<const h8*>(m + o + 64);
#pragma unroll
              for (int t = 0; t < 8; ++t) x[t] += p.beta * ((float)h[t] + (float)l[t]);
            }
#pragma unroll
            for (int t = 0; t < 8; ++t)
              if (ro + r == co + c + t) x[t] += p.gamma;
          }
          store_chunk(C + o + lo * 64, x, lo);
        }
      }
    } else {
      float* o = reinterpret_cast<float*>(C);
      const int ro = OUT == kF32T ? c0 : r0, co = OUT == kF32T ? r0 : c0;
      const int rows = OUT == kF32T ? p.N : p.M, cols = OUT == kF32T ? p.M : p.N;
      const bool vec = (p.ldc & 3) == 0 && (reinterpret_cast<uintptr_t>(C) & 15) == 0;
#pragma unroll 4
      for (int it = it0; it < it0 + ITS; ++it) {
        const int r = 4 * it + (lane >> 4), c = 4 * (lane & 15);
        v4 v;
        if constexpr (OUT == kF32T) {
#pragma unroll
          for (int t = 0; t < 4; ++t) v[t] = tile[at(c + t, r / 4) + (r & 3)];
        } else {
          v = *reinterpret_cast<const v4*>(&tile[at(r, c / 4)]);
        }
        if (ro + r >= rows) continue;
        float* d = o + (int64_t)(ro + r) * p.ldc + co + c;
        if (vec && co + c + 3 < cols) {
          *reinterpret_cast<v4*>(d) = v;
        } else {
#pragma unroll
          for (int t = 0; t < 4; ++t)
            if (co + c + t < cols) d[t] = v[t];
        }
      }
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);  // read before the next half overwrites it
    __builtin_amdgcn_wave_barrier();
  }
}

// What kSym writes of the tiles that were summed in parts of K: a 32 x 32 piece of
// one per workgroup, four values per thread (bound by the latency of the parts'
// loads: 64 x 64 pieces took 22 us for 16 tiles in 16 parts).
template <int BT>
__global__ __launch_bounds__(256) void k_ns_finish(Gemm p) {
  constexpr int T = 32, PIECES = (BT / T) * (BT / T);
  __shared__ float tile[T][T + 1];
  const int tiles = p.tiles_m * (p.tiles_m + 1) / 2, split = blockIdx.x / PIECES, piece = blockIdx.x % PIECES;
  const int t = p.whole + split;
  const int64_t batch = t / tiles;
  int tm, tn;
  triangle_tile(t % tiles, tm, tn);
  const int pr = piece / (BT / T) * T, pc = piece % (BT / T) * T, r0 = tm * BT + pr, c0 = tn * BT + pc;
  if (r0 >= p.M || c0 >= p.ldc) return;
  const uint8_t* m = p.m ? p.m + batch * p.c_batch : nullptr;
  const int64_t line = (int64_t)(p.ldc / KS) * BLOCK;
  const float* sums = p.sums + (int64_t)split * p.parts * (BT * BT) + pr * BT + pc;
  {
    const int r = threadIdx.x / (T / 4), c = 4 * (threadIdx.x % (T / 4)), row = r0 + r, col = c0 + c;
    v4 v = {};
#pragma unroll 8
    for (int i = 0; i < p.parts; ++i) v += *reinterpret_cast<const v4*>(sums + (int64_t)i * (BT * BT) + r * BT + c);
    v *= p.alpha;
    if (m && row < p.M) {
      const uint8_t* o = m + row * line + col / KS * BLOCK + (col % KS) * 2;
      const h4 hi = *reinterpret_cast<const h4*>(o), lo = *reinterpret_cast<const h4*>(o + 64);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] += p.beta * ((float)hi[k] + (float)lo[k]);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) tile[r][c + k] = v[k] + (row == col + k ? p.gamma : 0.0f);
  }
  __syncthreads();
  uint8_t* out = p.c + batch * p.c_batch;
  for (int mirror = 0; mirror < (tm == tn ? 1 : 2); ++mirror) {
    const int ro = mirror ? c0 : r0, co = mirror ? r0 : c0;
    const int r = threadIdx.x / 8, lo = (threadIdx.x & 4) / 4, k = threadIdx.x & 3;  // 8 chunks of 16 bytes a row
    if (ro + r >= p.M || co >= p.ldc) continue;
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = mirror ? tile[8 * k + i][r] : tile[r][8 * k + i];
    store_chunk(out + (ro + r) * line + co / KS * BLOCK + lo * 64 + k * 16, x, lo);
  }
}

// The products of symmetric matrices of n <= 128 in one launch, a workgroup for each
// matrix with a wave for each 32 x 32 tile: S from the sums of X X^T's parts, P, and
// for a pair of steps S P, P S P, P' and P' P; the planes of P or P' P leave.
// Everything stays in LDS, in two matrices (128 KB at n = 128), as each product takes
// the place of an operand that it is the last to read: a launch for each product
// takes 6.9 us at n = 64 where its 12 MFMAs a wave take 0.3.
//
// A's diagonal takes its own way: it is zero in A's fragments, and a_rr b_rc, with a_rr
// (and b_rr) in FP32, is added to what the MFMAs give.  The matrix cores add eight
// products after aligning them to the largest and dropping what lies below its last
// place; these matrices are near-diagonal, and next to a product of two diagonal values
// the others lost their last bits (update of 64 x 576 of noise: 2.7e-6 off, FP32 1.7e-6;
// now 0.6e-6, for 1.2 us more in a launch of 7.0; the diagonal's products in MFMAs of
// their own, at 22 bits: 1.0e-6, 0.7 us).
struct Chain {
  const float* sums;  // [matrix][tile of the lower triangle][part][64][64]
  int parts, n, pair;
  uint8_t* out;       // planes
  int64_t out_batch;
};
template <int NB>
__global__ __launch_bounds__(64 * NB * NB) void k_ns_chain(Chain p) {
  constexpr int R = KS * NB, ROW = BLOCK * NB, NT = 64 * NB * NB, T = 64;
  __shared__ __attribute__((aligned(128))) uint8_t mem[2][R * ROW];
  __shared__ __attribute__((aligned(16))) float diag[2][R];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int wr = wave / NB, wc = wave % NB, fr = lane & 31, fk = lane >> 5;
  // chunk c (16 bytes) of row r, spread over the banks within its block
  auto at = [](int r, int c) { return r * ROW + (c & ~7) * 16 + ((c & 7) ^ (NB % 2 ? (r >> 1) & 7 : r & 7)) * 16; };
  // four values of a row of matrix m
  auto put4 = [&](int m, int r, int c, const v4& v) {
    h4 hi, lo;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      hi[t] = (_Float16)v[t];
      lo[t] = (_Float16)(v[t] - (float)hi[t]);
    }
    const int chunk = c / KS * 8 + (c % KS) / 8;
    *reinterpret_cast<h4*>(mem[m] + at(r, chunk) + (c & 4) * 2) = hi;
    *reinterpret_cast<h4*>(mem[m] + at(r, chunk + 4) + (c & 4) * 2) = lo;
  };
  // this lane's four values, of row r of the wave's tile, with d on the diagonal
  auto get4 = [&](int m, int r, int c, float d) -> v4 {
    const int chunk = c / KS * 8 + (c % KS) / 8;
    const h4 hi = *reinterpret_cast<const h4*>(mem[m] + at(r, chunk) + (c & 4) * 2);
    const h4 lo = *reinterpret_cast<const h4*>(mem[m] + at(r, chunk + 4) + (c & 4) * 2);
    v4 v;
#pragma unroll
    for (int t = 0; t < 4; ++t) v[t] = r == c + t ? d : (float)hi[t] + (float)lo[t];
    return v;
  };
  // zero where the diagonal lies in this lane's eight columns of either half of a block
  u4 off[2];
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int i = fr - 16 * k - 8 * fk - 2 * t;
      off[k][t] = i == 0 ? 0xFFFF0000u : i == 1 ? 0x0000FFFFu : 0xFFFFFFFFu;
    }
  // dst = alpha a b^T + beta m + gamma I for symmetric b; dst may be any of the others,
  // m -1: none
  auto product = [&](int dst, int ia, int ib, float alpha, int im, float beta, float gamma) {
    const uint8_t *a = mem[ia], *b = mem[ib];
    const int r = 32 * wr + fr;
    const float da = diag[ia][r], db = diag[ib][r], dm = im >= 0 ? diag[im][r] : 0.0f;
    v16 acc = {}, cross = {};
#pragma unroll
    for (int h = 0; h < 2 * NB; ++h) {
      h8 f[2][2];
#pragma unroll
      for (int pl = 0; pl < 2; ++pl) {
        const int chunk = h / 2 * 8 + pl * 4 + 2 * (h & 1) + fk;
        f[0][pl] = *reinterpret_cast<const h8*>(a + at(r, chunk));
        f[1][pl] = *reinterpret_cast<const h8*>(b + at(32 * wc + fr, chunk));
      }
      if (h / 2 == wr) {  // (the whole wave: A's diagonal lies in these columns)
#pragma unroll
        for (int pl = 0; pl < 2; ++pl) f[0][pl] = __builtin_bit_cast(h8, __builtin_bit_cast(u4, f[0][pl]) & off[h & 1]);
      }
      cross = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[1][0], f[0][1], cross, 0, 0, 0);
      cross = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[1][1], f[0][0], cross, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[1][0], f[0][0], acc, 0, 0, 0);
    }
    acc += cross;
    v4 out[4];
    float d = 0.0f;  // the lane's value on the diagonal, if it has one
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int c = 32 * wc + 8 * q + 4 * fk;
      const v4 vb = get4(ib, r, c, db);
      v4& v = out[q];
#pragma unroll
      for (int t = 0; t < 4; ++t) v[t] = __builtin_fmaf(da, vb[t], acc[4 * q + t]) * alpha;
      if (im >= 0) {
        const v4 vm = im == ib ? vb : get4(im, r, c, dm);
#pragma unroll
        for (int t = 0; t < 4; ++t) v[t] += beta * vm[t];
      }
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        v[t] += r == c + t && r < p.n ? gamma : 0.0f;
        d = r == c + t ? v[t] : d;
      }
    }
    __syncthreads();  // every wave has read
#pragma unroll
    for (int q = 0; q < 4; ++q) put4(dst, r, 32 * wc + 8 * q + 4 * fk, out[q]);
    if (wr == wc && ((fr >> 2) & 1) == fk) diag[dst][r] = d;
    __syncthreads();
  };
  constexpr int S = 0, P = 1;
  // the triangle's tiles, four values of a row at a time; those below the diagonal mirrored
  constexpr int QUADS = (NB <= 2 ? 1 : 3) * T * T / 4, EACH = (QUADS + NT - 1) / NT;
  const float* sums = p.sums + (int64_t)blockIdx.x * (QUADS * 4) * p.parts;
  v4 sum[EACH] = {};
#pragma unroll 4
  for (int i = 0; i < p.parts; ++i)
#pragma unroll
    for (int u = 0; u < EACH; ++u) {
      const int q = min(tid + u * NT, QUADS - 1), t = q / (T * T / 4);
      sum[u] += *reinterpret_cast<const v4*>(sums + ((int64_t)t * p.parts + i) * (T * T) + 4 * (q % (T * T / 4)));
    }
#pragma unroll
  for (int u = 0; u < EACH; ++u) {
    const int q = tid + u * NT, t = q / (T * T / 4), in = q % (T * T / 4);
    const int r = in / (T / 4) + (t > 0 ? T : 0), c = 4 * (in % (T / 4)) + (t == 2 ? T : 0);
    if (q >= QUADS || r >= R || c >= R) continue;
    const v4 v = sum[u] * ldexpf(1.0f, kSScale - 2 * kXScale);
    put4(S, r, c, v);
    if (r / 4 == c / 4) diag[S][r] = v[r % 4];
    if (t != 1) continue;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const _Float16 hi = (_Float16)v[j];
      uint8_t* o = mem[S] + (r & 7) * 2;
      *reinterpret_cast<_Float16*>(o + at(c + j, r / KS * 8 + (r % KS) / 8)) = hi;
      *reinterpret_cast<_Float16*>(o + at(c + j, r / KS * 8 + (r % KS) / 8 + 4)) = (_Float16)(v[j] - (float)hi);
    }
  }
  __syncthreads();
  const float one = ldexpf(1.0f, -kPScale), sq = ldexpf(kC, kPScale - 2 * kSScale), li = ldexpf(kB, kPScale - kSScale);
  const float id = ldexpf(kA, kPScale);
  product(P, S, S, sq, S, li, id);
  int Q = P;
  if (p.pair) {
    product(S, S, P, one, -1, 0.0f, 0.0f);  // S P
    product(S, S, P, one, -1, 0.0f, 0.0f);  // P S P
    product(S, S, S, sq, S, li, id);        // P'
    product(S, S, P, ldexpf(1.0f, kQScale - 2 * kPScale), -1, 0.0f, 0.0f);
    Q = S;
  }
  uint8_t* out = p.out + blockIdx.x * p.out_batch;
  for (int q = tid; q < p.n * NB * 8; q += NT) {
    const int r = q / (NB * 8), c = q % (NB * 8);
    *reinterpret_cast<h8*>(out + (int64_t)r * ROW + c * 16) = *reinterpret_cast<const h8*>(mem[Q] + at(r, c));
  }
}

// U of one value: the new momentum (written where there is one) and what is
// orthogonalised.
__device__ __forceinline__ float update_of(float g, float m_new, float beta, int mode) {
  return mode == 0 ? g : mode == 1 ? m_new : g + beta * m_new;
}

// M' = beta M + G, and the sums of squares of U in 64 bits: part[matrix][block].
// mode 0: U = G (no momentum); 1: U = M'; 2: U = G + beta M'.
template <int V>
__global__ __launch_bounds__(256) void k_ns_momentum(const float* __restrict__ g, const float* m, float* m_out,
                                                     float beta, int mode, int64_t count, int blocks,
                                                     double* __restrict__ part) {
  typedef float v_t __attribute__((ext_vector_type(V)));
  __shared__ double red[4];
  const int64_t matrix = blockIdx.x / blocks, block = blockIdx.x % blocks, base = matrix * count;
  double sum = 0.0;
  for (int64_t i = (block * 256 + threadIdx.x) * V; i < count; i += (int64_t)blocks * 256 * V) {
    const v_t x = *reinterpret_cast<const v_t*>(g + base + i);
    v_t n = {};
    if (mode) {
      n = beta * *reinterpret_cast<const v_t*>(m + base + i) + x;
      *reinterpret_cast<v_t*>(m_out + base + i) = n;
    }
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const double u = update_of(x[k], n[k], beta, mode);
      sum += u * u;
    }
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

// X = U / (|U| + eps) in planes, transposed where U has more rows than columns:
// one 64 x 64 tile of X per workgroup.
template <bool FLIP>
__global__ __launch_bounds__(256) void k_ns_split(const float* __restrict__ g, const float* __restrict__ m_new,
                                                  float beta, int mode, int n, int k, int tiles_n, int64_t per_matrix,
                                                  int blocks, const double* __restrict__ part, float eps,
                                                  uint8_t* __restrict__ x) {
  constexpr int T = 64;
  __shared__ float tile[T][T + 1];
  __shared__ double red[4];
  const int64_t matrix = blockIdx.x / per_matrix, t = blockIdx.x % per_matrix, base = matrix * ((int64_t)n * k);
  const int r0 = (int)(t / tiles_n) * T, c0 = (int)(t % tiles_n) * T;
  // the tile of U: rows of U are X's columns where it is transposed
  const int rows = FLIP ? k : n, cols = FLIP ? n : k, ur = FLIP ? c0 : r0, uc = FLIP ? r0 : c0;
  // (every load before the first is waited for: values past the edge are read at it)
  constexpr int EACH = T * T / 256;
  const int ic = threadIdx.x % T, ir = threadIdx.x / T;
  float gv[EACH], mv[EACH];
  const int64_t from = base + min(uc + ic, cols - 1);
#pragma unroll
  for (int i = 0; i < EACH; ++i) gv[i] = g[from + (int64_t)min(ur + ir + 4 * i, rows - 1) * cols];
  if (mode) {
#pragma unroll
    for (int i = 0; i < EACH; ++i) mv[i] = m_new[from + (int64_t)min(ur + ir + 4 * i, rows - 1) * cols];
  } else {
#pragma unroll
    for (int i = 0; i < EACH; ++i) mv[i] = 0.0f;
  }
  double sum = 0.0;
  for (int i = threadIdx.x; i < blocks; i += 256) sum += part[matrix * blocks + i];
#pragma unroll
  for (int i = 0; i < EACH; ++i)
    tile[ir + 4 * i][ic] = ur + ir + 4 * i < rows && uc + ic < cols ? update_of(gv[i], mv[i], beta, mode) : 0.0f;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
  __syncthreads();
  const double norm = sqrt((red[0] + red[1]) + (red[2] + red[3]));
  // the factor as a fraction and a power of two, which may lie outside FP32's range
  int power;
  const float part_of = (float)frexp((double)(1 << kXScale) / (norm + (double)eps), &power);
  const int64_t ld = blocks_of(k);
  uint8_t* out = x + matrix * (n * ld * BLOCK);
  for (int q = threadIdx.x; q < T * 16; q += 256) {
    const int r = q / 16, blk = (q % 16) / 8, lo = (q % 8) / 4, kk = q % 4, col = blk * KS + 8 * kk;
    if (r0 + r >= n || c0 + col >= ld * KS) continue;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = part_of * ldexpf(FLIP ? tile[col + i][r] : tile[r][col + i], power);
    store_chunk(out + ((int64_t)(r0 + r) * ld + (c0 + col) / KS) * BLOCK + lo * 64 + kk * 16, v, lo);
  }
}

constexpr int kNormBlocks = 2048;
constexpr int kChainMost = 128;  // rows of the matrices that k_ns_chain takes

}  // namespace ns

namespace {

using namespace ns;

int64_t up(int64_t n, int64_t m) { return (n + m - 1) / m * m; }

// Tiles of 256, 128 or 64 squared, of which a CU takes one, two or four at once.
// Whole rounds of tiles run as they are; those left over, where the product may be
// split, are summed in parts of K that share out the last round.  Priced in us: a slab
// of a tile that has its CU for itself, what each further tile there adds, the start
// and end of a tile, and a split's second launch and its sums' way to memory and back.
// (S S^T of n = 256: 14.8 us on 128 tiles, 8.3 on 64; n = 4096: 290 on 64, 206 on 128
// with the last 16 of 528 tiles in parts, 251 without; Q X of 4096 x 16384: 1940, 1600
// and 1450 on 64, 128 and 256.)
struct Tiling {
  int tile, parts;
  int64_t whole;
};
Tiling tiling(const int64_t (&count)[3], int64_t slabs, bool split) {
  struct Price {
    int tile, per_cu;
    double slab, more, ends, part_ends, sums;
  };
  constexpr Price prices[3] = {{256, 1, 2.8, 0.0, 10.0, 8.0, 0.045},
                               {128, 2, 1.0, 0.45, 6.5, 2.0, 0.0125},
                               {64, 4, 0.5, 0.14, 4.5, 2.3, 0.003}};
  Tiling best{128, 1, count[1]};
  double least = 1e30;
  for (int i = 0; i < 3; ++i) {
    const Price& p = prices[i];
    const int64_t tiles = count[i], room = 256 * p.per_cu, whole = tiles / room * room, rest = tiles - whole;
    // workgroups of so many slabs, in rounds
    auto rounds = [&](int64_t wgs, int64_t s) {
      const int64_t left = wgs % room, deep = (left + 255) / 256;
      return (double)(wgs / room) * (s * (p.slab + (p.per_cu - 1) * p.more) + p.ends / 2) +
             (left ? s * (p.slab + (deep - 1) * p.more) : 0.0);
    };
    for (int64_t parts = 1; parts == 1 || (split && rest > 0 && parts <= 64 && slabs / parts >= 4); ++parts) {
      const int64_t ps = (slabs + parts - 1) / parts, wgs = rest * parts;
      const double cost = parts == 1 ? rounds(tiles, slabs) + p.ends
                                     : rounds(whole, slabs) + rounds(wgs, ps) + p.part_ends + 6.5 + p.sums * wgs;
      if (cost < least) least = cost, best = Tiling{p.tile, (int)parts, parts > 1 ? whole : tiles};
    }
  }
  return best;
}

// The iteration of one call: sizes of its matrices and where they lie in the
// workspace.
struct NsPlan {
  int64_t n, k, x_bytes, s_bytes, ld;  // one matrix: X, S (planes), values in a row of S
  Tiling gram, square, apply;
  int norm_blocks;
  int64_t off_x[2], off_s[2], off_p[3], off_sum, off_norm, bytes;
};

NsPlan ns_plan(int64_t batch, int64_t rows, int64_t cols) {
  NsPlan p;
  p.n = rows < cols ? rows : cols;
  p.k = rows < cols ? cols : rows;
  p.ld = blocks_of(p.n) * KS;
  p.x_bytes = p.n * blocks_of(p.k) * BLOCK;
  p.s_bytes = p.n * blocks_of(p.n) * BLOCK;
  // tiles of edge t in a matrix, and in the lower triangles of all
  auto count = [&](int64_t t) { return (p.n + t - 1) / t * ((p.k + t - 1) / t) * batch; };
  auto tri = [&](int64_t t) { return batch * ((p.n + t - 1) / t) * ((p.n + t - 1) / t + 1) / 2; };
  p.gram = tiling({tri(256), tri(128), tri(64)}, blocks_of(p.k), true);
  p.square = tiling({tri(256), tri(128), tri(64)}, blocks_of(p.n), true);
  if (p.n <= kChainMost) {  // tiles of 64, their sums left to the chain
    const int64_t slabs = blocks_of(p.k), fill = 512 / tri(64), most = slabs / 4 < 16 ? slabs / 4 : 16;
    p.gram = Tiling{64, (int)(fill < 1 || most < 1 ? 1 : fill < most ? fill : most), 0};
    p.square = Tiling{64, 1, tri(64)};
  }
  p.apply = tiling({count(256), count(128), count(64)}, blocks_of(p.n), false);
  const int64_t per = (p.n * p.k + 4095) / 4096;
  p.norm_blocks = (int)(per < kNormBlocks ? per : kNormBlocks);
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t o = at;
    at += up(bytes, 256);
    return o;
  };
  for (auto& o : p.off_x) o = take(batch * p.x_bytes);
  for (auto& o : p.off_s) o = take(batch * p.s_bytes);
  for (auto& o : p.off_p) o = take(batch * p.s_bytes);
  int64_t sums = 0;
  for (const Tiling& t : {p.gram, p.square}) {
    const int64_t bytes = (tri(t.tile) - t.whole) * t.parts * t.tile * t.tile * 4;
    sums = bytes > sums ? bytes : sums;
  }
  p.off_sum = take(sums);
  p.off_norm = take(batch * p.norm_blocks * 8);
  p.bytes = at;
  return p;
}

// Stages of a product's slabs in LDS (k_ns_gemm).
int stages_of(int tile, int64_t wgs, int64_t slabs) { return tile == 64 && wgs <= 512 && slabs <= 12 ? 4 : 2; }

template <bool TR, int OUT>
hipError_t run_gemm(const Gemm& g, int tile, int64_t wgs, hipStream_t s) {
  if (tile == 256)
    hipLaunchKernelGGL((k_ns_gemm<256, 256, 2, 4, TR, OUT, 2>), dim3((unsigned)wgs), dim3(512), 0, s, g);
  else if (tile == 128)
    hipLaunchKernelGGL((k_ns_gemm<128, 128, 2, 2, TR, OUT, 2>), dim3((unsigned)wgs), dim3(256), 0, s, g);
  else if (stages_of(tile, wgs, g.parts > 1 ? g.part_slabs : blocks_of(g.K)) == 4)
    hipLaunchKernelGGL((k_ns_gemm<64, 64, 2, 2, TR, OUT, 4>), dim3((unsigned)wgs), dim3(256), 0, s, g);
  else
    hipLaunchKernelGGL((k_ns_gemm<64, 64, 2, 2, TR, OUT, 2>), dim3((unsigned)wgs), dim3(256), 0, s, g);
  return hipGetLastError();
}

// A symmetric product's launch: slabs in a part of K, parts, workgroups.
struct SymLaunch {
  int part_slabs, parts;
  int64_t tiles, wgs;
};
SymLaunch sym_launch(const Tiling& how, int64_t batch, int64_t n, int64_t K) {
  const int64_t t = (n + how.tile - 1) / how.tile, tri = batch * t * (t + 1) / 2;
  const int slabs = (int)blocks_of(K), ps = (slabs + how.parts - 1) / how.parts, parts = (slabs + ps - 1) / ps;
  return SymLaunch{ps, parts, tri, how.whole + (tri - how.whole) * parts};
}

}  // namespace

int64_t orthogonalize_ws(int64_t batch, int64_t rows, int64_t cols) { return ns_plan(batch, rows, cols).bytes; }

OrthoRoute orthogonalize_route(int64_t batch, int64_t rows, int64_t cols) {
  const NsPlan p = ns_plan(batch, rows, cols);
  OrthoRoute r{};
  auto sym = [&](int i, const Tiling& how, int64_t K) {
    const SymLaunch l = sym_launch(how, batch, p.n, K);
    r.tile[i] = how.tile;
    r.stages[i] = stages_of(how.tile, l.wgs, l.parts > 1 ? l.part_slabs : blocks_of(K));
    r.parts[i] = l.parts;
    r.whole[i] = how.whole;
  };
  sym(0, p.gram, p.k);
  sym(1, p.square, p.n);
  const int64_t t = p.apply.tile;
  r.tile[2] = p.apply.tile;
  r.stages[2] = stages_of(p.apply.tile, batch * ((p.n + t - 1) / t) * ((p.k + t - 1) / t), blocks_of(p.n));
  return r;
}

hipError_t launch_orthogonalize(const float* grad, const float* momentum, float* momentum_out, float beta,
                                bool nesterov, int64_t batch, int64_t rows, int64_t cols, int steps, float eps,
                                float* out, uint8_t* ws, hipStream_t s) {
  if (batch == 0 || rows == 0 || cols == 0) return hipSuccess;
  const NsPlan p = ns_plan(batch, rows, cols);
  const int n = (int)p.n, k = (int)p.k, mode = !momentum ? 0 : nesterov ? 2 : 1;
  uint8_t* X[2] = {ws + p.off_x[0], ws + p.off_x[1]};
  float* sum = reinterpret_cast<float*>(ws + p.off_sum);
  double* norm = reinterpret_cast<double*>(ws + p.off_norm);
  const int64_t count = rows * cols;
  auto al = [](const void* q) { return reinterpret_cast<uintptr_t>(q) % 16 == 0; };
  if (count % 4 == 0 && al(grad) && al(momentum) && al(momentum_out))
    hipLaunchKernelGGL((k_ns_momentum<4>), dim3((unsigned)(batch * p.norm_blocks)), dim3(256), 0, s, grad, momentum,
                       momentum_out, beta, mode, count, p.norm_blocks, norm);
  else
    hipLaunchKernelGGL((k_ns_momentum<1>), dim3((unsigned)(batch * p.norm_blocks)), dim3(256), 0, s, grad, momentum,
                       momentum_out, beta, mode, count, p.norm_blocks, norm);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int tiles_k = (k + 63) / 64;
  const int64_t split = (int64_t)((n + 63) / 64) * tiles_k;
  const bool flip = rows > cols;
  if (flip)
    hipLaunchKernelGGL((k_ns_split<true>), dim3((unsigned)(batch * split)), dim3(256), 0, s, grad, momentum_out, beta,
                       mode, n, k, tiles_k, split, p.norm_blocks, norm, eps, X[0]);
  else
    hipLaunchKernelGGL((k_ns_split<false>), dim3((unsigned)(batch * split)), dim3(256), 0, s, grad, momentum_out, beta,
                       mode, n, k, tiles_k, split, p.norm_blocks, norm, eps, X[0]);
  e = hipGetLastError();
  if (e != hipSuccess) return e;

  // out = alpha a b^T + beta m + gamma I of symmetric n x n matrices
  auto product = [&](const uint8_t* a, const uint8_t* b, int64_t batch_bytes, int K, const Tiling& how, uint8_t* o,
                     float alpha, const uint8_t* m, float beta_m, float gamma) {
    const SymLaunch l = sym_launch(how, batch, n, K);
    const int t = (n + how.tile - 1) / how.tile;
    const Gemm g{a, batch_bytes, b, batch_bytes, n, n, K, t, t, alpha, o, p.s_bytes, (int)p.ld, m, beta_m, gamma,
                 (int)how.whole, l.parts, l.part_slabs, sum};
    const hipError_t err = run_gemm<false, kSym>(g, how.tile, l.wgs, s);
    if (err != hipSuccess || how.whole == l.tiles) return err;
    const int64_t pieces = (l.tiles - how.whole) * (how.tile / 32) * (how.tile / 32);
    if (how.tile == 256) hipLaunchKernelGGL(k_ns_finish<256>, dim3((unsigned)pieces), dim3(256), 0, s, g);
    else if (how.tile == 64) hipLaunchKernelGGL(k_ns_finish<64>, dim3((unsigned)pieces), dim3(256), 0, s, g);
    else hipLaunchKernelGGL(k_ns_finish<128>, dim3((unsigned)pieces), dim3(256), 0, s, g);
    return hipGetLastError();
  };
  uint8_t *S = ws + p.off_s[0], *T = ws + p.off_s[1];
  uint8_t* poly[3] = {ws + p.off_p[0], ws + p.off_p[1], ws + p.off_p[2]};
  for (int done = 0, at = 0; done < steps; at ^= 1) {
    // a pair pays from k = n on; near it its launches decide, which the chain does not have
    const int group = (p.k < p.n + p.n / 8 && n > kChainMost) || steps - done < 2 ? 1 : 2;
    const uint8_t* Q = nullptr;
    int q_scale = 0;
    if (n <= kChainMost) {
      const SymLaunch l = sym_launch(p.gram, batch, n, k);
      const int t = (n + 63) / 64;
      e = run_gemm<false, kSym>(Gemm{X[at], p.x_bytes, X[at], p.x_bytes, n, n, k, t, t, 1.0f, nullptr, 0, (int)p.ld,
                                     nullptr, 0.0f, 0.0f, 0, l.parts, l.part_slabs, sum},
                                64, l.wgs, s);
      if (e != hipSuccess) return e;
      const Chain c{sum, l.parts, n, group == 2, poly[0], p.s_bytes};
      if (n <= 32) hipLaunchKernelGGL(k_ns_chain<1>, dim3((unsigned)batch), dim3(64), 0, s, c);
      else if (n <= 64) hipLaunchKernelGGL(k_ns_chain<2>, dim3((unsigned)batch), dim3(256), 0, s, c);
      else if (n <= 96) hipLaunchKernelGGL(k_ns_chain<3>, dim3((unsigned)batch), dim3(576), 0, s, c);
      else hipLaunchKernelGGL(k_ns_chain<4>, dim3((unsigned)batch), dim3(1024), 0, s, c);
      Q = poly[0], q_scale = group == 2 ? kQScale : kPScale;
    } else {
      e = product(X[at], X[at], p.x_bytes, k, p.gram, S, ldexpf(1.0f, kSScale - 2 * kXScale), nullptr, 0.0f, 0.0f);
    }
    if (e == hipSuccess) e = hipGetLastError();
    if (e != hipSuccess) return e;
    for (int i = 0; i < group && n > kChainMost; ++i) {
      uint8_t* P = poly[i & 1];
      if (i > 0) {  // S <- P S P of the last step's P
        const float one = ldexpf(1.0f, -kPScale);
        e = product(S, poly[(i - 1) & 1], p.s_bytes, n, p.square, T, one, nullptr, 0.0f, 0.0f);
        if (e != hipSuccess) return e;
        e = product(T, poly[(i - 1) & 1], p.s_bytes, n, p.square, S, one, nullptr, 0.0f, 0.0f);
        if (e != hipSuccess) return e;
      }
      e = product(S, S, p.s_bytes, n, p.square, P, ldexpf(kC, kPScale - 2 * kSScale), S, ldexpf(kB, kPScale - kSScale),
                  ldexpf(kA, kPScale));
      if (e != hipSuccess) return e;
      if (i == 0) {
        Q = P, q_scale = kPScale;
      } else {  // |P' P| < 3.45^2: 2^12 of it stays below FP16's end
        e = product(P, Q, p.s_bytes, n, p.square, poly[2], ldexpf(1.0f, kQScale - 2 * kPScale), nullptr, 0.0f, 0.0f);
        if (e != hipSuccess) return e;
        Q = poly[2], q_scale = kQScale;
      }
    }
    done += group;
    const bool last = done == steps;
    const int tile = p.apply.tile;
    const Gemm g{Q, p.s_bytes, X[at], p.x_bytes, n, k, n, (n + tile - 1) / tile, (k + tile - 1) / tile,
                 ldexpf(1.0f, last ? -q_scale - kXScale : -q_scale), last ? reinterpret_cast<uint8_t*>(out) : X[at ^ 1],
                 last ? count * 4 : p.x_bytes, last ? (int)cols : (int)(blocks_of(k) * KS), nullptr, 0.0f, 0.0f, 0, 1, 0,
                 nullptr};
    const int64_t wgs = batch * g.tiles_m * g.tiles_n;
    e = !last ? run_gemm<true, kPlanes>(g, tile, wgs, s) : flip ? run_gemm<true, kF32T>(g, tile, wgs, s)
                                                                : run_gemm<true, kF32>(g, tile, wgs, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace fastbfp
