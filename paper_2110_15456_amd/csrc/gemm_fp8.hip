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
#include <math.h>

#include <type_traits>

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

// s_waitcnt's operand: vmcnt(n), and lgkmcnt(0) with `lds`.
constexpr int wait_loads(int n, bool lds = false) { return (n & 15) | (n >> 4) << 14 | 7 << 4 | (lds ? 0 : 15) << 8; }

// Asks for a step's LDS reads and LOADS loads evenly among its MFMAs: a wave's loads in one
// run hold it up for as long as the L1 takes them, 64 cycles a KB.
template <int TM, int TN, int LOADS>
__device__ __forceinline__ void spread() {
  if constexpr (TM * TN >= 4) {
    constexpr int READS = (2 * (TM + TN) + TM * TN - 1) / (TM * TN), EACH = (LOADS + TM * TN - 1) / (TM * TN);
#pragma unroll
    for (int u = 0; u < TM * TN; ++u) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, LOADS ? 1 : 0);  // MFMA
      if constexpr (LOADS > 0) __builtin_amdgcn_sched_group_barrier(0x010, EACH, 1);  // loads
      __builtin_amdgcn_sched_group_barrier(0x100, READS, LOADS ? 1 : 0);  // LDS reads
    }
  }
}

// BM x BN tiles, 2 x 2 waves; a slab is one block of K, 128 bytes of every row, brought by
// direct buffer -> LDS loads of 1 KB into one of two stages while the other is computed
// on.  16-byte chunk c of row r sits at chunk c ^ ((r >> 1) & 7): 16 lanes that read one
// chunk of 16 rows hit all 64 banks.  Rows past the end read zeros (the buffer resources
// end at the last row).
//
// A slab is two steps of 64.  A step's fragments are read while the one before is
// multiplied; between a slab's steps, when all of the slab is in registers, the waves
// meet: the next slab has landed, and the loads of the one after it go to the stage that
// was just read, a whole slab ahead of their use.
//
// Two stages, and on the 64 tile four: it serves products of so few tiles that a slab
// takes as long as its loads do (1024 x 1024 x 8192 with two 34.8 us, with four 15.6).
//
// Measured (BF16 out, 200 launches in a row): 8192^3 378 us, 2.91 PFLOP/s; 4096 x 4096 x 8192
// 96 us, 2.87; 8192 x 16384 x 4096 404 us, 2.72; 8192 x 4096 x 4096 102 us, 2.69; with FP32 out
// 398, 101, 436 and 111.  After a rest the clock takes some 20 ms to rise (8192 x 16384 x 4096:
// 480 us each of ten launches, 416 of forty).  A library's FP8 product of the same codes,
// without scales, takes 337, 86, 364 and 93 us: 0.89 to 0.91 of this kernel's.  The matrix
// units are busy for 73 to 79% of the cycles, and the clock is at 1.75 GHz of 2.4; a round of
// tiles ends with 5.5 us of writing C.  The 128 tile, two workgroups on a CU, reaches 2.2 and
// moves 1.5 bytes through the LDS for each of the 256 tile's; the 64 tile 1.3.
template <int BM, int BN, int FA, int FB, class T>
__global__ __launch_bounds__(256, BM == 256 ? 1 : 2) void k_gemm_fp8(Gemm p) {
  constexpr int ST = BM == 64 ? 4 : 2;
  constexpr int NW = 4, WM = BM / 2, WN = BN / 2, TM = WM / 32, TN = WN / 32;
  constexpr int OFF_B = BM * kBlock, STAGE = OFF_B + BN * kBlock;
  constexpr int LA = BM / 8 / NW, LB = BN / 8 / NW;  // loads of a wave
  __shared__ __attribute__((aligned(128))) uint8_t stage0[STAGE];
  __shared__ __attribute__((aligned(128))) uint8_t stage1[STAGE];
  __shared__ __attribute__((aligned(128))) uint8_t stage2[ST == 4 ? STAGE : 16];
  __shared__ __attribute__((aligned(128))) uint8_t stage3[ST == 4 ? STAGE : 16];
  __shared__ int scale_stage[2 * (BM + BN)];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int wr = wave >> 1, wc = wave & 1;

  const int tiles = p.tiles_m * p.tiles_n, id = xcd_order(blockIdx.x, gridDim.x), part = id / tiles, t = id % tiles;
  // bands of four tile rows, down each band's column first: the tiles that an XCD runs
  // at once share rows of A and of B
  const int band = t / (4 * p.tiles_n), in = t % (4 * p.tiles_n), rows = min(4, p.tiles_m - 4 * band);
  const int row0 = (4 * band + in % rows) * BM, col0 = in / rows * BN;
  const int slab0 = part * p.part_slabs, nslabs = min(p.part_slabs, p.slabs - slab0);

  const int arows = min(BM, p.M - row0), brows = min(BN, p.N - col0);
  const uint8_t *pa = p.a + (int64_t)row0 * p.pitch, *pb = p.b + (int64_t)col0 * p.pitch;
  const uint8_t *pea = p.ea + (int64_t)row0 * p.epitch, *peb = p.eb + (int64_t)col0 * p.epitch;
  const uint32_t size_a = (uint32_t)arows * p.pitch, size_b = (uint32_t)brows * p.pitch;
  v16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = v16{};

  const uint32_t lane_off =
      (uint32_t)(8 * wave + (lane >> 3)) * p.pitch + (uint32_t)((lane & 7) ^ ((4 * (wave & 1) + (lane >> 4)) & 7)) * 16;
  const uint32_t step_off = 8 * NW * p.pitch;  // from one of a wave's loads to the next
  // (All of an offset is the lane's: the buffer's bound does not count a scalar one.  Slabs
  // behind the last one: the loads find an empty buffer and write zeros, so that the loop
  // has no branch around them.)
  auto issue = [&](uint8_t* stage, int s) __attribute__((always_inline)) {
    const uint32_t k0 = (uint32_t)(slab0 + s) * kBlock;
    const rsrc_t sa = make_rsrc(pa, s < nslabs ? size_a : 0u), sb = make_rsrc(pb, s < nslabs ? size_b : 0u);
#pragma unroll
    for (int u = 0; u < LA; ++u)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(sa, (lds_void*)(stage + (wave + NW * u) * 1024), 16,
                                               lane_off + (k0 + u * step_off), 0, 0, 0);
#pragma unroll
    for (int u = 0; u < LB; ++u)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(sb, (lds_void*)(stage + OFF_B + (wave + NW * u) * 1024), 16,
                                               lane_off + (k0 + u * step_off), 0, 0, 0);
  };
  const int fr = lane & 31, fk = lane >> 5, fsw = (fr >> 1) & 7;
  // (the chunks of a lane's 32 bytes of step h: 4 h + 2 fk and the one beside it)
  const int at0 = fr * kBlock + (((2 * fk) ^ fsw) * 16), at1 = fr * kBlock + (((2 * fk + 1) ^ fsw) * 16);
  auto frag = [&](const uint8_t* tile, int r, int h) __attribute__((always_inline)) -> v8i {
    const uint8_t* at = tile + r * kBlock;
    const u4 x = *reinterpret_cast<const u4*>(at + (at0 ^ (64 * h)));
    const u4 y = *reinterpret_cast<const u4*>(at + (at1 ^ (64 * h)));
    return v8i{(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)y[0], (int)y[1], (int)y[2], (int)y[3]};
  };
  // The scales of slab s and its neighbours of a dword, for each row of A and then of B, to
  // LDS: 64 rows at a time, which of them goes by the wave.  (A lane's
  // own loads of its rows' dwords, each in a line of its own, took as long as half of the
  // codes' loads: 8192 x 16384 x 4096 445 us with them, 404 so.)
  constexpr int RUNS = (BM + BN) / 64, LS = RUNS < NW ? 1 : RUNS / NW;  // loads of a wave
  auto issue_scales = [&](int s) __attribute__((always_inline)) {
    const int first = s & ~3, quad = (s >> 2) & 1;
#pragma unroll
    for (int u = 0; u < LS; ++u) {
      const int run = RUNS < NW ? wave % RUNS : wave + NW * u;
      const bool of_b = run >= BM / 64;
      const rsrc_t rs = make_rsrc(of_b ? peb : pea, first < nslabs ? (uint32_t)(of_b ? brows : arows) * p.epitch : 0u);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)(scale_stage + quad * (BM + BN) + run * 64), 4,
                                               (uint32_t)((of_b ? run - BM / 64 : run) * 64 + lane) * p.epitch +
                                                   (uint32_t)(slab0 + first), 0, 0, 0);
    }
  };
  auto read_scales = [&](int s, int (&sa)[TM], int (&sb)[TN]) __attribute__((always_inline)) {
    const int* at = scale_stage + ((s >> 2) & 1) * (BM + BN) + fr;
    const int down = 8 * (s & 3);  // (slab s's byte lowest)
#pragma unroll
    for (int i = 0; i < TM; ++i) sa[i] = (int)((uint32_t)at[wr * WM + 32 * i] >> down);
#pragma unroll
    for (int j = 0; j < TN; ++j) sb[j] = (int)((uint32_t)at[BM + wc * WN + 32 * j] >> down);
  };
  v8i a[2][TM], b[2][TN];
  int sa[TM], sb[TN], na[TM], nb[TN];
  auto read = [&](const uint8_t* tile, int h, v8i (&fa)[TM], v8i (&fb)[TN]) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < TN; ++j) fb[j] = frag(tile + OFF_B, wc * WN + 32 * j, h);
#pragma unroll
    for (int i = 0; i < TM; ++i) fa[i] = frag(tile, wr * WM + 32 * i, h);
  };
  auto multiply = [&](const v8i (&fa)[TM], const v8i (&fb)[TN]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)  // (B first: a lane's quads are columns of a row)
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[j], fa[i], acc[i][j], FB, FA, 0, sb[j], 0, sa[i]);
  };
  // all but `younger` of this wave's loads have landed and its LDS reads are done, as are
  // the other waves'
  auto meet = [&](auto younger) __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(wait_loads(decltype(younger)::value, true));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  constexpr std::integral_constant<int, 0> all{};
  // Slab s, the k-th of a run of ST.  When its second step's fragments are read, slab s + 1
  // has to have landed, while those of s + 2 .. s + ST - 1 (and the next scales, until they
  // are older than slab s + 1) may be on the way.  The run's first slab asks for the scales
  // of the slab four from it (with ST = 2 every second time for those that are there
  // already, which does no harm), its last reads the next run's.
  auto slab = [&](uint8_t* cur, uint8_t* nxt, auto kc, int s) __attribute__((always_inline)) {
    constexpr int k = decltype(kc)::value;
    constexpr int YOUNGER = (ST - 2) * (LA + LB) + (ST == 4 && (k == 1 || k == 2) ? LS : 0);
    __builtin_amdgcn_sched_barrier(0);
    read(cur, 1, a[1], b[1]);
    multiply(a[0], b[0]);
    spread<TM, TN, 0>();
    __builtin_amdgcn_sched_barrier(0);
    meet(std::integral_constant<int, YOUNGER>{});
    if constexpr (k == 0) issue_scales(s + 4);
    issue(cur, s + ST);
    read(nxt, 0, a[0], b[0]);  // (behind the last slab: what lies there, unused)
    if constexpr (k == ST - 1) read_scales(s + 1, na, nb);
    multiply(a[1], b[1]);
    spread<TM, TN, LA + LB>();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < TM; ++i) sa[i] = k == ST - 1 ? na[i] : (int)((uint32_t)sa[i] >> 8);
#pragma unroll
    for (int j = 0; j < TN; ++j) sb[j] = k == ST - 1 ? nb[j] : (int)((uint32_t)sb[j] >> 8);
  };
  issue_scales(0);
  issue(stage0, 0);
  issue(stage1, 1);
  if constexpr (ST == 4) {
    issue(stage2, 2);
    issue(stage3, 3);
  }
  meet(std::integral_constant<int, (ST - 1) * (LA + LB)>{});
  read_scales(0, sa, sb);
  read(stage0, 0, a[0], b[0]);
  // Whole runs of ST slabs have no branch among them, and the slabs that are left, all of which
  // are on the way by then, run behind the loop: the compiler waits by itself for loads to a
  // stage that some path leaves on the way, and on a path from a run's first slab back to
  // the loop's head that is all of them (with branches in one loop 64 tiles waited for
  // all they had on the way once in four slabs, 128 tiles half a slab early in every second).
  constexpr std::integral_constant<int, 0> k0{};
  constexpr std::integral_constant<int, 1> k1{};
  // The j-th slab behind the loop, its `next` one's loads older than those of ST - 2 - j more.
  auto last = [&](const uint8_t* cur, const uint8_t* nxt, auto jc, bool next) __attribute__((always_inline)) {
    read(cur, 1, a[1], b[1]);
    multiply(a[0], b[0]);
    if (next) {
      meet(std::integral_constant<int, (ST - 2 - decltype(jc)::value) * (LA + LB)>{});
      read(nxt, 0, a[0], b[0]);
    }
    multiply(a[1], b[1]);
#pragma unroll
    for (int i = 0; i < TM; ++i) sa[i] = (int)((uint32_t)sa[i] >> 8);
#pragma unroll
    for (int j = 0; j < TN; ++j) sb[j] = (int)((uint32_t)sb[j] >> 8);
  };
  int s = 0;
  if constexpr (BM == 256) {
    // (an odd slab's partner runs on zeros: with another slab behind the loop the fragments
    // would not stay in registers)
    for (; s < nslabs; s += 2) {
      slab(stage0, stage1, k0, s);
      slab(stage1, stage0, k1, s + 1);
    }
  } else if constexpr (ST == 2) {
    for (; s + 1 < nslabs; s += 2) {
      slab(stage0, stage1, k0, s);
      slab(stage1, stage0, k1, s + 1);
    }
    if (s < nslabs) last(stage0, stage1, k0, false);
  } else {
    constexpr std::integral_constant<int, 2> k2{};
    constexpr std::integral_constant<int, 3> k3{};
    for (; s + 3 < nslabs; s += 4) {
      slab(stage0, stage1, k0, s);
      slab(stage1, stage2, k1, s + 1);
      slab(stage2, stage3, k2, s + 2);
      slab(stage3, stage0, k3, s + 3);
    }
    if (s < nslabs) {
      last(stage0, stage1, k0, s + 1 < nslabs);
      if (s + 1 < nslabs) {
        last(stage1, stage2, k1, s + 2 < nslabs);
        if (s + 2 < nslabs) last(stage2, stage3, k2, false);
      }
    }
  }

  // A lane holds columns 8 q + 4 fk .. + 3 of row fr of each 32 x 32 tile.  32 rows of
  // the wave's columns at a time go through its part of the first stage, so that rows
  // leave as whole lines; 16-byte granule g of row r sits at g ^ swz(r), which spreads 16
  // rows of one granule over all banks.
  meet(all);
  constexpr int G = WN / 4;  // granules of a row
  float* tile = reinterpret_cast<float*>(stage0) + wave * (32 * WN);
  auto swz = [](int r) __attribute__((always_inline)) -> int { return G == 8 ? (r >> 1) & 7 : r & 15; };
  T* C = static_cast<T*>(p.c) + part * p.part_stride;
  // C past the caches where its rows are whole lines (8192 x 16384 x 4096: 475 -> 445 us),
  // but for sums that are read again
  const bool lines = p.part_stride == 0 && ((p.ldc * sizeof(T)) | reinterpret_cast<uintptr_t>(C)) % 128 == 0;
  constexpr int V = 16 / sizeof(T), LR = WN / V, RI = 64 / LR;  // a lane's values, lanes of a row, rows at a time
  const int c = col0 + wc * WN + lane % LR * V;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        v4 v;
#pragma unroll
        for (int t = 0; t < 4; ++t) v[t] = acc[i][j][4 * q + t];
        *reinterpret_cast<v4*>(tile + fr * WN + ((8 * j + 2 * q + fk) ^ swz(fr)) * 4) = v;
      }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int it = 0; it < 32 / RI; ++it) {
      const int r = it * RI + lane / LR, g = lane % LR * (V / 4), row = row0 + wr * WM + 32 * i + r;
      const u4 x = *reinterpret_cast<const u4*>(tile + r * WN + (g ^ swz(r)) * 4);
      u4 y = u4{0u, 0u, 0u, 0u};
      if constexpr (V == 8) y = *reinterpret_cast<const u4*>(tile + r * WN + ((g + 1) ^ swz(r)) * 4);
      if (row >= p.M) continue;
      T* o = C + row * p.ldc + c;
      if (lines && c + V <= p.N) {
        if constexpr (V == 4) {
          __builtin_nontemporal_store(x, reinterpret_cast<u4*>(o));
        } else {
          const u2 lo = to_bf16(x), hi = to_bf16(y);
          __builtin_nontemporal_store(u4{lo[0], lo[1], hi[0], hi[1]}, reinterpret_cast<u4*>(o));
        }
      } else if constexpr (V == 4) {
        store4(o, x, p.N - c);
      } else {
        store8(o, x, y, p.N - c);
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Few rows of A: a workgroup takes 16 RM rows x 16 RN columns, and its waves split K: a wave
// takes every waves-th run of four slabs.  Each keeps four slabs of its own on the way to
// its own part of LDS, so that the waves never meet before their sums are added, in their
// order.  What bounds these products is the bytes of B on the way: direct buffer -> LDS
// loads of whole lines (8 rows x 128 bytes each) move them; loads straight into the
// registers' layout touch 16 rows at once and were held to 4 TB/s by the L1's lookups
// (16 x 16384 x 4096: 18.1 us with them, 12.4 so, 5.5 TB/s of B).
template <int RM, int RN, int WAVES, int FA, int FB, class T>
__global__ __launch_bounds__(64 * WAVES) void k_gemm_fp8_few(Gemm p) {
  constexpr int ROWS = 16 * (RM + RN), PART = ROWS * kBlock;  // a wave's slab
  constexpr int LOADS = 2 * (RM + RN), SCALES = RM + RN;
  __shared__ __attribute__((aligned(128))) uint8_t stage0[WAVES * PART];
  __shared__ __attribute__((aligned(128))) uint8_t stage1[WAVES * PART];
  __shared__ __attribute__((aligned(128))) uint8_t stage2[WAVES * PART];
  __shared__ __attribute__((aligned(128))) uint8_t stage3[WAVES * PART];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int id = xcd_order(blockIdx.x, gridDim.x), row0 = id / p.tiles_n * (16 * RM), col0 = id % p.tiles_n * (16 * RN);
  const uint32_t arows = (uint32_t)min(16 * RM, p.M - row0), brows = (uint32_t)min(16 * RN, p.N - col0);
  const uint8_t *pa = p.a + (int64_t)row0 * p.pitch, *pb = p.b + (int64_t)col0 * p.pitch;
  const uint8_t *pea = p.ea + (int64_t)row0 * p.epitch, *peb = p.eb + (int64_t)col0 * p.epitch;
  const int supers = (p.slabs + 3) / 4;
  v4 acc[RM][RN];
#pragma unroll
  for (int i = 0; i < RM; ++i)
#pragma unroll
    for (int j = 0; j < RN; ++j) acc[i][j] = v4{0.f, 0.f, 0.f, 0.f};
  // (the swizzle of k_gemm_fp8: chunk c of row r at c ^ ((r >> 1) & 7))
  uint32_t load_off[2];
#pragma unroll
  for (int u = 0; u < 2; ++u)
    load_off[u] = (uint32_t)(8 * u + (lane >> 3)) * p.pitch + (uint32_t)((lane & 7) ^ ((4 * u + (lane >> 4)) & 7)) * 16;
  auto issue = [&](uint8_t* stage, int slab) __attribute__((always_inline)) {
    const rsrc_t ra = make_rsrc(pa, slab < p.slabs ? arows * p.pitch : 0u);
    const rsrc_t rb = make_rsrc(pb, slab < p.slabs ? brows * p.pitch : 0u);
    uint8_t* mine = stage + wave * PART;
#pragma unroll
    for (int i = 0; i < RM; ++i)
#pragma unroll
      for (int u = 0; u < 2; ++u)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_void*)(mine + (2 * i + u) * 1024), 16,
                                                 load_off[u] + ((uint32_t)slab * kBlock + 16 * i * p.pitch), 0, 0, 0);
#pragma unroll
    for (int j = 0; j < RN; ++j)
#pragma unroll
      for (int u = 0; u < 2; ++u)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_void*)(mine + (2 * (RM + j) + u) * 1024), 16,
                                                 load_off[u] + ((uint32_t)slab * kBlock + 16 * j * p.pitch), 0, 0, 0);
  };
  const int r = lane & 15, q = lane >> 4, rsw = (r >> 1) & 7;
  int sa[RM], sb[RN], na[RM], nb[RN];
  auto scales = [&](int super) __attribute__((always_inline)) {
    const rsrc_t ra = make_rsrc(pea, super < supers ? arows * p.epitch : 0u);
    const rsrc_t rb = make_rsrc(peb, super < supers ? brows * p.epitch : 0u);
#pragma unroll
    for (int i = 0; i < RM; ++i)
      na[i] = (int)__builtin_amdgcn_raw_buffer_load_b32(ra, (uint32_t)(16 * i + r) * p.epitch + 4 * super, 0, 0);
#pragma unroll
    for (int j = 0; j < RN; ++j)
      nb[j] = (int)__builtin_amdgcn_raw_buffer_load_b32(rb, (uint32_t)(16 * j + r) * p.epitch + 4 * super, 0, 0);
  };
  auto frag = [&](const uint8_t* at) __attribute__((always_inline)) -> v8i {
    const u4 x = *reinterpret_cast<const u4*>(at + r * kBlock + ((2 * q) ^ rsw) * 16);
    const u4 y = *reinterpret_cast<const u4*>(at + r * kBlock + ((2 * q + 1) ^ rsw) * 16);
    return v8i{(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)y[0], (int)y[1], (int)y[2], (int)y[3]};
  };
  // slab k of a run of four: its loads have landed when only the three younger slabs'
  // (and, for slabs 1 to 3, the next run's scales) may be on the way
  auto slab = [&](uint8_t* stage, auto kc, int next) __attribute__((always_inline)) {
    constexpr int k = decltype(kc)::value;
    __builtin_amdgcn_s_waitcnt(wait_loads(3 * LOADS + (k > 0 ? SCALES : 0)));
    asm volatile("" ::: "memory");
    const uint8_t* mine = stage + wave * PART;
    v8i a[RM], b[RN];
#pragma unroll
    for (int i = 0; i < RM; ++i) a[i] = frag(mine + i * 16 * kBlock);
#pragma unroll
    for (int j = 0; j < RN; ++j) b[j] = frag(mine + (RM + j) * 16 * kBlock);
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): the stage is read
    asm volatile("" ::: "memory");
    if constexpr (k == 0) {
#pragma unroll
      for (int i = 0; i < RM; ++i) sa[i] = na[i];
#pragma unroll
      for (int j = 0; j < RN; ++j) sb[j] = nb[j];
      scales(next);
    }
    issue(stage, 4 * next + k);
#pragma unroll
    for (int i = 0; i < RM; ++i)
#pragma unroll
      for (int j = 0; j < RN; ++j)  // (B first: a lane's four are columns of a row)
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b[j], a[i], acc[i][j], FB, FA, k, sb[j], k, sa[i]);
  };
  // (the first run's scales go in front of all slabs but the first: behind them, the wait for
  // them in the loop would be one for all but the youngest slab, in every run)
  issue(stage0, 4 * wave);
  __builtin_amdgcn_sched_barrier(0);
  scales(wave);
  __builtin_amdgcn_sched_barrier(0);
  issue(stage1, 4 * wave + 1);
  issue(stage2, 4 * wave + 2);
  issue(stage3, 4 * wave + 3);
  for (int s = wave; s < supers; s += WAVES) {
    slab(stage0, std::integral_constant<int, 0>{}, s + WAVES);
    slab(stage1, std::integral_constant<int, 1>{}, s + WAVES);
    slab(stage2, std::integral_constant<int, 2>{}, s + WAVES);
    slab(stage3, std::integral_constant<int, 3>{}, s + WAVES);
  }
  // A lane holds columns 4 q .. + 3 of row r of each 16 x 16 tile.
  constexpr int QUADS = 64 * RM * RN;
  static_assert(QUADS * 16 <= PART, "the sums fit in a stage");
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  float* sums = reinterpret_cast<float*>(stage0);
#pragma unroll
  for (int i = 0; i < RM; ++i)
#pragma unroll
    for (int j = 0; j < RN; ++j)
      *reinterpret_cast<v4*>(sums + (wave * QUADS + ((16 * i + r) * RN + j) * 4 + q) * 4) = acc[i][j];
  __syncthreads();
  T* C = static_cast<T*>(p.c);
  for (int o = threadIdx.x; o < QUADS; o += 64 * WAVES) {
    v4 v = *reinterpret_cast<const v4*>(sums + 4 * o);
    for (int w = 1; w < WAVES; ++w) v += *reinterpret_cast<const v4*>(sums + (w * QUADS + o) * 4);
    const int row = row0 + o / (4 * RN), c = col0 + o % (4 * RN) * 4;
    if (row < p.M) store4(C + row * p.ldc + c, __builtin_bit_cast(u4, v), p.N - c);
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

template <int FA, int FB, class T>
void launch_kernel(const Fp8Plan& plan, const Gemm& g, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)g.tiles_m * g.tiles_n * plan.parts));
#define FASTBFP_FEW(RM, RN, WAVES) \
  hipLaunchKernelGGL((k_gemm_fp8_few<RM, RN, WAVES, FA, FB, T>), grid, dim3(64 * WAVES), 0, s, g)
#define FASTBFP_TILE(EDGE) hipLaunchKernelGGL((k_gemm_fp8<EDGE, EDGE, FA, FB, T>), grid, dim3(256), 0, s, g)
  if (plan.waves == 0) {
    if (plan.rows == 256) FASTBFP_TILE(256);
    else if (plan.rows == 128) FASTBFP_TILE(128);
    else FASTBFP_TILE(64);
  } else if (plan.rows == 16 && plan.cols == 16) {
    FASTBFP_FEW(1, 1, 4);
  } else if (plan.rows == 16) {
    FASTBFP_FEW(1, 4, 2);
  } else {
    FASTBFP_FEW(2, 2, 2);
  }
#undef FASTBFP_FEW
#undef FASTBFP_TILE
}

template <class T>
hipError_t launch_formats(const Fp8Plan& plan, const Gemm& g, int fa, int fb, hipStream_t s) {
  if (fa == kE4M3 && fb == kE4M3) launch_kernel<0, 0, T>(plan, g, s);
  else if (fa == kE4M3) launch_kernel<0, 1, T>(plan, g, s);
  else if (fb == kE4M3) launch_kernel<1, 0, T>(plan, g, s);
  else launch_kernel<1, 1, T>(plan, g, s);
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
  g.tiles_m = (g.M + plan.rows - 1) / plan.rows;
  g.tiles_n = (g.N + plan.cols - 1) / plan.cols;
  if (plan.parts == 1) {
    g.c = C, g.ldc = ldc, g.part_stride = 0;
    return launch_formats<T>(plan, g, fa, fb, s);
  }
  g.c = ws, g.ldc = gemm_plan_ld(g.N), g.part_stride = g.M * g.ldc;
  const hipError_t e = launch_formats<float>(plan, g, fa, fb, s);
  if (e != hipSuccess) return e;
  const int64_t n = g.part_stride / 4;
  hipLaunchKernelGGL(k_join<T>, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, ws, plan.parts, g.part_stride,
                     (int)(g.ldc / 4), n, g.N, C, ldc);
  return hipGetLastError();
}

// The kernels, and their price in us, of a form that was fitted to the times of 900 drawn
// products (1 .. 8192 rows, 64 .. 16384 columns and K, either way round): `start` once, then for
// each round of workgroups on the 256 CUs the larger of one's latency, `open` + slabs * `slab`,
// and of what those on a CU together need of it, each `each_open` + slabs * `each`.  They
// order the kernels and are no times: launches in a graph take 0.75 of the price of an
// unsplit 64 tile or a few-row kernel, 0.9 of a 128 tile's, and large products on 256 tiles up
// to 1.3 of it.  Of 1600 drawn products the kernel and parts taken are 1.4% slower than the
// fastest ones in the mean, 2.3% of the products lose more than 20%, and one 49% at worst (5 us).
struct Kernel {
  int rows, cols, waves, on_cu;
  float start, open, slab, each_open, each;
};
constexpr Kernel kKernels[] = {
    {64, 64, 0, 2, 2.95f, 1.61f, 0.148f, 0.99f, 0.207f},  {128, 128, 0, 2, 3.32f, 0.0f, 0.540f, 2.24f, 0.418f},
    {256, 256, 0, 1, 0.0f, 12.17f, 1.04f, 0.66f, 0.254f}, {16, 16, 4, 2, 3.67f, 0.225f, 0.121f, 0.075f, 0.226f},
    {16, 64, 2, 2, 3.87f, 0.264f, 0.223f, 0.400f, 0.323f},  {32, 32, 2, 2, 3.64f, 0.603f, 0.158f, 0.425f, 0.266f},
};
constexpr float kJoin = 2.5f, kJoinValue = 1.1e-6f;  // us, and for a value of a part

float price(const Kernel& k, int64_t tiles, int slabs) {
  if (k.waves > 0) {
    // (a wave takes runs of four slabs)
    const float run = 4.0f * (float)(((slabs + 3) / 4 + k.waves - 1) / k.waves);
    const int64_t rounds = (tiles + 256 * k.on_cu - 1) / (256 * k.on_cu);
    return k.start + fmaxf((float)rounds * (k.open + run * k.slab), (float)tiles / 256.0f * (k.each_open + run * k.each));
  }
  const float run = (float)(k.rows == 256 ? (slabs + 1) / 2 * 2 : slabs);
  const int64_t on = (tiles + 255) / 256, rounds = on / k.on_cu, last = on % k.on_cu;
  auto round = [&](int64_t n) { return fmaxf(k.open + run * k.slab, (float)n * (k.each_open + run * k.each)); };
  return k.start + (float)rounds * round(k.on_cu) + (last ? round(last) : 0.0f);
}

}  // namespace fp8

Fp8Plan fp8_plan(int64_t M, int64_t N, int64_t K, bool room) {
  using namespace fp8;
  const int slabs = (int)blocks_of(K);
  Fp8Plan best{64, 64, 0, slabs, 1};
  float least = INFINITY;
  if (slabs == 0) return best;
  for (const Kernel& k : kKernels) {
    const int64_t tiles = ((M + k.rows - 1) / k.rows) * ((N + k.cols - 1) / k.cols);
    for (const int want : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
      if (want > 1 && (!room || k.waves > 0 || tiles > 1024 || 4 * (want - 1) >= slabs)) break;
      // (a part's scales begin at a whole dword)
      const int each = want == 1 ? slabs : ((slabs + want - 1) / want + 3) / 4 * 4, parts = (slabs + each - 1) / each;
      if (parts != want || (parts > 1 && parts * M * gemm_plan_ld(N) > (int64_t(1) << 26))) continue;
      if (tiles * parts * (k.waves ? 64 * k.waves : 256) > kMostThreads) continue;
      float t = price(k, tiles * parts, each);
      if (parts > 1) t += kJoin + kJoinValue * (float)parts * (float)M * (float)N;
      if (t < least) {
        least = t;
        best = {k.rows, k.cols, k.waves, each, parts};
      }
    }
  }
  return best;
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
