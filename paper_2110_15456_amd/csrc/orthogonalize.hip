// orthogonalize.hip -- a step of momentum whose result is orthogonalised by the
// quintic Newton-Schulz iteration:
//   M' = beta M + G,  U = G + beta M' (Nesterov) or M',  X = U / (|U|_F + eps),
//   repeated:  S = X X^T,  X <- (a I + b S + c S^2) X
// with (a, b, c) = (3.4445, -4.7750, 2.0315), which takes every singular value
// of X in (0, 1] towards 1 (into about 0.7 .. 1.2) and leaves the vectors.
//
// X is kept with no more rows than columns (n <= k; the transpose of U where it
// has more), so the products are n x n x k, n x n x n and n x k x n.
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
//
// Layout ("planes"): rows of blocks of 32 columns, a block 128 bytes, 32 hi then
// 32 lo: one line holds what a K slab of 32 needs of a row.
#include <hip/hip_runtime.h>

#include <utility>

#include "launch.h"

namespace fastbfp {

namespace ns {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr int kXScale = 15, kSScale = 15, kPScale = 14;

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

// What a product writes.
enum { kParts, kPlanes, kF32, kF32T };

struct Gemm {
  const uint8_t* a;  // planes, rows x blocks_k
  int64_t a_batch;
  const uint8_t* b;  // planes: rows of the product's columns (TR: X itself, rows of its K)
  int64_t b_batch;
  int M, N, K;       // C is M x N
  int tiles_m, tiles_n;  // (kParts: tiles_m alone, the lower triangle's tiles)
  int part_slabs, parts;
  float scale;
  uint8_t* c;        // planes, or FP32 rows of ldc
  int64_t c_batch, c_part;
  int ldc;
};

// Workgroup -> (item, tile): contiguous runs of workgroups on each XCD.
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
// A wave's tile is 128 x 64 (64 x 64 on the small tile): per slab 24 (16) KB of
// fragments for 96 (48) MFMAs of 32x32x16, i.e. the LDS is busy half of the time
// that the matrix cores are.
template <int BM, int BN, int WGM, int WGN, bool TR, int OUT>
__global__ __launch_bounds__(64 * WGM * WGN, 2) void k_ns_gemm(Gemm p) {
  constexpr int NW = WGM * WGN, WM = BM / WGM, WN = BN / WGN, TM = WM / 32, TN = WN / 32;
  constexpr int OFF_B = BM * BLOCK, STAGE = OFF_B + BN * BLOCK;
  constexpr bool SWAP = OUT != kF32T;  // a lane's quads: columns of one row, or rows of one column
  static_assert((BM / 8) % NW == 0 && (BN / 8) % NW == 0 && NW % 2 == 0, "loads split evenly over the waves");
  __shared__ __attribute__((aligned(128))) uint8_t stage0[STAGE];
  __shared__ __attribute__((aligned(128))) uint8_t stage1[STAGE];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int wr = wave / WGN, wc = wave % WGN;

  int id = xcd_order(blockIdx.x, gridDim.x), tm, tn, part = 0;
  int64_t batch;
  if constexpr (OUT == kParts) {
    const int tiles = p.tiles_m * (p.tiles_m + 1) / 2;
    const int t = id % tiles;
    id /= tiles;
    part = id % p.parts;
    batch = id / p.parts;
    tm = (int)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
    while (tm * (tm + 1) / 2 > t) --tm;
    while ((tm + 1) * (tm + 2) / 2 <= t) ++tm;
    tn = t - tm * (tm + 1) / 2;
  } else {
    // bands of four tile rows, down each band's column first: the tiles that an
    // XCD runs at once share rows of A and columns of X
    const int tiles = p.tiles_m * p.tiles_n, t = id % tiles;
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
  const int all = (int)blocks_of(p.K), slab0 = part * p.part_slabs;
  const int nslabs = OUT == kParts ? min(p.part_slabs, all - slab0) : all;

  v16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = v16{};

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
    c = SWAP ? __builtin_amdgcn_mfma_f32_32x32x16_f16(b, a, c, 0, 0, 0)
             : __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  };
  auto step = [&](const uint8_t* cur, uint8_t* nxt, int s) __attribute__((always_inline)) {
    // this wave's loads of slab s have landed and its reads of slab s - 1 are done
    __builtin_amdgcn_s_waitcnt(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (s + 1 < nslabs) issue(nxt, s + 1);
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
        for (int j = 0; j < TN; ++j) mma(acc[i][j], lo, b[j][0]);
#pragma unroll
        for (int j = 0; j < TN; ++j) mma(acc[i][j], hi, b[j][1]);
#pragma unroll
        for (int j = 0; j < TN; ++j) mma(acc[i][j], hi, b[j][0]);
      }
    });
  };
  issue(stage0, 0);
  int s = 0;
  for (; s + 2 <= nslabs; s += 2) {
    step(stage0, stage1, s);
    step(stage1, stage0, s + 1);
  }
  if (s < nslabs) step(stage0, stage1, s);

  // Epilogue.  SWAP: lane holds columns 8 q + 4 fk .. + 3 of row fr of each 32 x 32
  // tile; otherwise rows of column fr.
  uint8_t* C = p.c + batch * p.c_batch + part * p.c_part;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int j = 0; j < TN; ++j) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        v4 v;
#pragma unroll
        for (int t = 0; t < 4; ++t) v[t] = acc[i][j][4 * q + t] * p.scale;
        const int quad = 8 * q + 4 * fk;
        if constexpr (OUT == kF32T) {
          // C^T: columns row .. row + 3 of row col
          const int row = row0 + wr * WM + 32 * i + quad, col = col0 + wc * WN + 32 * j + fr;
          float* o = reinterpret_cast<float*>(C) + (int64_t)col * p.ldc + row;
          if (col < p.N) {
            if ((p.ldc & 3) == 0 && row + 3 < p.M) *reinterpret_cast<v4*>(o) = v;
            else
#pragma unroll
              for (int t = 0; t < 4; ++t)
                if (row + t < p.M) o[t] = v[t];
          }
        } else {
          const int row = row0 + wr * WM + 32 * i + fr, col = col0 + wc * WN + 32 * j + quad;
          if (row >= p.M) continue;
          if constexpr (OUT == kParts) {
            if (col < p.ldc) *reinterpret_cast<v4*>(reinterpret_cast<float*>(C) + (int64_t)row * p.ldc + col) = v;
          } else if constexpr (OUT == kPlanes) {
            if (col < p.ldc) {
              h4 hi, lo;
#pragma unroll
              for (int t = 0; t < 4; ++t) {
                hi[t] = (_Float16)v[t];
                lo[t] = (_Float16)(v[t] - (float)hi[t]);
              }
              uint8_t* o = C + ((int64_t)row * (p.ldc / KS) + col / KS) * BLOCK + (col % KS) * 2;
              *reinterpret_cast<h4*>(o) = hi;
              *reinterpret_cast<h4*>(o + 64) = lo;
            }
          } else {
            float* o = reinterpret_cast<float*>(C) + (int64_t)row * p.ldc + col;
            if ((p.ldc & 3) == 0 && col + 3 < p.N) *reinterpret_cast<v4*>(o) = v;
            else
#pragma unroll
              for (int t = 0; t < 4; ++t)
                if (col + t < p.N) o[t] = v[t];
          }
        }
      }
    }
  }
}

// out = alpha sum_parts + beta m + gamma I of symmetric n x n matrices, of whose
// parts (FP32, rows of ld = blocks_of(n) * 32) the lower triangle's tiles are
// there: one 64 x 64 tile per workgroup, written twice, as it is and mirrored.
// Columns from n to ld become zeros.
struct Finish {
  const float* sum;
  int64_t part, batch;  // strides, values
  int parts;
  const uint8_t* m;     // planes, or null
  uint8_t* out;         // planes
  int64_t m_batch, out_batch;
  int n, ld, tiles;
  float alpha, beta, gamma;
};
__device__ __forceinline__ void store_chunk(uint8_t* o, const float (&x)[8], bool lo) {
  h8 v;
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    const _Float16 h = (_Float16)x[t];
    v[t] = lo ? (_Float16)(x[t] - (float)h) : h;
  }
  *reinterpret_cast<h8*>(o) = v;
}
__global__ __launch_bounds__(256) void k_ns_finish(Finish p) {
  constexpr int T = 64;
  __shared__ float tile[T][T + 1];
  const int tiles = p.tiles * (p.tiles + 1) / 2, t = blockIdx.x % tiles;
  const int64_t batch = blockIdx.x / tiles;
  int tm = (int)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
  while (tm * (tm + 1) / 2 > t) --tm;
  while ((tm + 1) * (tm + 2) / 2 <= t) ++tm;
  const int tn = t - tm * (tm + 1) / 2, r0 = tm * T, c0 = tn * T;
  const uint8_t* m = p.m ? p.m + batch * p.m_batch : nullptr;
  for (int q = threadIdx.x; q < T * T / 4; q += 256) {
    const int r = q / (T / 4), c = 4 * (q % (T / 4)), row = r0 + r, col = c0 + c;
    v4 v = {};
    if (row < p.n && col < p.n) {
      const float* at = p.sum + batch * p.batch + (int64_t)row * p.ld + col;
      for (int i = 0; i < p.parts; ++i) v += *reinterpret_cast<const v4*>(at + i * p.part);
      v *= p.alpha;
      if (m) {
        const uint8_t* o = m + ((int64_t)row * (p.ld / KS) + col / KS) * BLOCK + (col % KS) * 2;
        const h4 hi = *reinterpret_cast<const h4*>(o), lo = *reinterpret_cast<const h4*>(o + 64);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] += p.beta * ((float)hi[k] + (float)lo[k]);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (row == col + k) v[k] += p.gamma;
        if (col + k >= p.n) v[k] = 0.0f;
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) tile[r][c + k] = v[k];
  }
  __syncthreads();
  uint8_t* out = p.out + batch * p.out_batch;
  for (int mirror = 0; mirror < (tm == tn ? 1 : 2); ++mirror) {
    const int ro = mirror ? c0 : r0, co = mirror ? r0 : c0;
    for (int q = threadIdx.x; q < T * 16; q += 256) {  // 16 chunks of 16 bytes a row
      const int r = q / 16, blk = (q % 16) / 8, lo = (q % 8) / 4, k = q % 4, col = blk * KS + 8 * k;
      if (ro + r >= p.n || co + col >= p.ld) continue;
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = mirror ? tile[col + i][r] : tile[r][col + i];
      store_chunk(out + ((int64_t)(ro + r) * (p.ld / KS) + (co + col) / KS) * BLOCK + lo * 64 + k * 16, x, lo);
    }
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
  double sum = (int)threadIdx.x < blocks ? part[matrix * blocks + threadIdx.x] : 0.0;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
  // the tile of U: rows of U are X's columns where it is transposed
  const int rows = FLIP ? k : n, cols = FLIP ? n : k, ur = FLIP ? c0 : r0, uc = FLIP ? r0 : c0;
#pragma unroll 4
  for (int q = threadIdx.x; q < T * T; q += 256) {
    const int r = q / T, c = q % T;
    float u = 0.0f;
    if (ur + r < rows && uc + c < cols) {
      const int64_t i = base + (int64_t)(ur + r) * cols + uc + c;
      u = update_of(g[i], mode ? m_new[i] : 0.0f, beta, mode);
    }
    tile[r][c] = u;
  }
  __syncthreads();
  const double norm = sqrt((red[0] + red[1]) + (red[2] + red[3]));
  const float inv = (float)((double)(1 << kXScale) / (norm + (double)eps));
  const int64_t ld = blocks_of(k);
  uint8_t* out = x + matrix * (n * ld * BLOCK);
  for (int q = threadIdx.x; q < T * 16; q += 256) {
    const int r = q / 16, blk = (q % 16) / 8, lo = (q % 8) / 4, kk = q % 4, col = blk * KS + 8 * kk;
    if (r0 + r >= n || c0 + col >= ld * KS) continue;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = inv * (FLIP ? tile[col + i][r] : tile[r][col + i]);
    store_chunk(out + ((int64_t)(r0 + r) * ld + (c0 + col) / KS) * BLOCK + lo * 64 + kk * 16, v, lo);
  }
}

constexpr int kNormBlocks = 256;

}  // namespace ns

namespace {

using namespace ns;

int64_t up(int64_t n, int64_t m) { return (n + m - 1) / m * m; }

// The iteration of one call: sizes of its matrices and where they lie in the
// workspace.
struct NsPlan {
  int64_t n, k, x_bytes, s_bytes, ld, part;  // one matrix: X, S (planes), row and part of sums (values)
  int tile, gram_parts, square_parts, norm_blocks;
  int64_t off_x[2], off_s, off_p, off_sum, off_norm, bytes;
};

// Parts of K so that the lower triangle's tiles fill the card (256 workgroups of
// 256 x 256, 512 of 128 x 128), with at least eight slabs in each.
int parts_of(int64_t tiles, int64_t slabs, int64_t room) {
  int64_t best = 1;
  double best_cost = 1e30;
  for (int64_t p = 1; p <= 16 && (p == 1 || slabs / p >= 8); ++p) {
    const int64_t rounds = (tiles * p + room - 1) / room;
    const double cost = (double)rounds * ((slabs + p - 1) / p + 4) + 2.0 * p;
    if (cost < best_cost) best_cost = cost, best = p;
  }
  return (int)best;
}

NsPlan ns_plan(int64_t batch, int64_t rows, int64_t cols) {
  NsPlan p;
  p.n = rows < cols ? rows : cols;
  p.k = rows < cols ? cols : rows;
  p.ld = blocks_of(p.n) * KS;
  p.x_bytes = p.n * blocks_of(p.k) * BLOCK;
  p.s_bytes = p.n * blocks_of(p.n) * BLOCK;
  p.part = p.n * p.ld;
  const int64_t t256 = (p.n + 255) / 256;
  p.tile = batch * t256 * (t256 + 1) / 2 >= 200 ? 256 : 128;
  const int64_t t = (p.n + p.tile - 1) / p.tile, tiles = batch * t * (t + 1) / 2, room = p.tile == 256 ? 256 : 512;
  p.gram_parts = parts_of(tiles, blocks_of(p.k), room);
  p.square_parts = parts_of(tiles, blocks_of(p.n), room);
  const int64_t per = (p.n * p.k + 4095) / 4096;
  p.norm_blocks = (int)(per < kNormBlocks ? per : kNormBlocks);
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t o = at;
    at += up(bytes, 256);
    return o;
  };
  p.off_x[0] = take(batch * p.x_bytes);
  p.off_x[1] = take(batch * p.x_bytes);
  p.off_s = take(batch * p.s_bytes);
  p.off_p = take(batch * p.s_bytes);
  const int64_t parts = p.gram_parts > p.square_parts ? p.gram_parts : p.square_parts;
  p.off_sum = take(batch * parts * p.part * 4);
  p.off_norm = take(batch * p.norm_blocks * 8);
  p.bytes = at;
  return p;
}

template <bool TR, int OUT>
hipError_t run_gemm(const Gemm& g, int tile, int64_t wgs, hipStream_t s) {
  if (tile == 256)
    hipLaunchKernelGGL((k_ns_gemm<256, 256, 2, 4, TR, OUT>), dim3((unsigned)wgs), dim3(512), 0, s, g);
  else
    hipLaunchKernelGGL((k_ns_gemm<128, 128, 2, 2, TR, OUT>), dim3((unsigned)wgs), dim3(256), 0, s, g);
  return hipGetLastError();
}

}  // namespace

int64_t orthogonalize_ws(int64_t batch, int64_t rows, int64_t cols) { return ns_plan(batch, rows, cols).bytes; }

hipError_t launch_orthogonalize(const float* grad, const float* momentum, float* momentum_out, float beta,
                                bool nesterov, int64_t batch, int64_t rows, int64_t cols, int steps, float eps,
                                float* out, uint8_t* ws, hipStream_t s) {
  if (batch == 0 || rows == 0 || cols == 0) return hipSuccess;
  const NsPlan p = ns_plan(batch, rows, cols);
  const int n = (int)p.n, k = (int)p.k, mode = !momentum ? 0 : nesterov ? 2 : 1;
  uint8_t* X[2] = {ws + p.off_x[0], ws + p.off_x[1]};
  uint8_t *S = ws + p.off_s, *P = ws + p.off_p;
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

  const int t = (n + p.tile - 1) / p.tile;
  const int64_t tri = batch * t * (t + 1) / 2;
  // sums of a symmetric product a b^T, its K in parts
  auto product = [&](const uint8_t* a, int64_t a_batch, const uint8_t* b, int64_t b_batch, int K, int parts) {
    const int slabs = (int)blocks_of(K), ps = (slabs + parts - 1) / parts;
    Gemm g{a, a_batch, b, b_batch, n, n, K, t, t, ps, (slabs + ps - 1) / ps, 1.0f, reinterpret_cast<uint8_t*>(sum),
           p.part * 4, batch * p.part * 4, (int)p.ld};
    return std::pair<hipError_t, int>(run_gemm<false, kParts>(g, p.tile, tri * g.parts, s), g.parts);
  };
  auto finish = [&](int parts, const uint8_t* m, uint8_t* o, float alpha, float b, float gamma) {
    const int tiles = (n + 63) / 64;
    hipLaunchKernelGGL(k_ns_finish, dim3((unsigned)(batch * tiles * (tiles + 1) / 2)), dim3(256), 0, s,
                       Finish{sum, batch * p.part, p.part, parts, m, o, p.s_bytes, p.s_bytes, n, (int)p.ld, tiles, alpha,
                              b, gamma});
    return hipGetLastError();
  };
  const int at = (p.n + 255) / 256 * ((p.k + 255) / 256) * batch >= 200 ? 256 : 128;
  for (int i = 0; i < steps; ++i) {
    auto [e1, parts] = product(X[i & 1], p.x_bytes, X[i & 1], p.x_bytes, k, p.gram_parts);
    if (e1 != hipSuccess) return e1;
    e = finish(parts, nullptr, S, ldexpf(1.0f, kSScale - 2 * kXScale), 0.0f, 0.0f);
    if (e != hipSuccess) return e;
    auto [e2, parts2] = product(S, p.s_bytes, S, p.s_bytes, n, p.square_parts);
    if (e2 != hipSuccess) return e2;
    e = finish(parts2, S, P, ldexpf(kC, kPScale - 2 * kSScale), ldexpf(kB, kPScale - kSScale), ldexpf(kA, kPScale));
    if (e != hipSuccess) return e;
    const bool last = i + 1 == steps;
    Gemm g{P, p.s_bytes, X[i & 1], p.x_bytes, n, k, n, (n + at - 1) / at, (k + at - 1) / at, 0, 1,
           ldexpf(1.0f, last ? -kPScale - kXScale : -kPScale), last ? reinterpret_cast<uint8_t*>(out) : X[(i + 1) & 1],
           last ? count * 4 : p.x_bytes, 0, last ? (int)cols : (int)(blocks_of(k) * KS)};
    const int64_t wgs = batch * g.tiles_m * g.tiles_n;
    e = !last ? run_gemm<true, kPlanes>(g, at, wgs, s) : flip ? run_gemm<true, kF32T>(g, at, wgs, s)
                                                              : run_gemm<true, kF32>(g, at, wgs, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace fastbfp
