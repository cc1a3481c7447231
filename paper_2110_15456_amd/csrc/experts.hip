// experts.hip -- what surrounds the products of an expert layer: the plan of a
// routing (the slots in the order of their experts) and the weighted sum of the
// experts' outputs with its gradients.
//
// A slot is one choice of one token, slot = token * top + j; ids[slot] is its
// expert, and any value outside [0, experts) a choice that was dropped.
#include <hip/hip_runtime.h>

#include "launch.h"
#include "segments.h"

namespace fastbfp {

// ---- the plan -----------------------------------------------------------
//
// A stable counting sort by expert: a slot's place is the number of slots of
// lower experts, plus those of its own before it.  Ranks come from ballots (the
// lanes of a wave with the same id, one ballot for each bit of the ids), counts
// of the waves from LDS, counts of the workgroups from a first launch that is
// left out where one workgroup takes all slots.  Order and places depend on the
// ids alone: no atomics.
//
// Every workgroup adds up the counts of all of them, so there are at most
// kPlanMost: beyond 2^20 slots a wave goes over its share in several rounds, first
// counting, then (the ids read again) placing, and the time stays linear (8 million
// slots of 128 experts 172 us, 64 million 1.43 ms).
//
// Bound by the latency of its one or two launches: 32 slots of 8 experts take 4.7
// us, 16384 5.9 and 6.2 (in one workgroup, 16 slots a lane, 17.6).
namespace {

constexpr int kPlanWaves = 16;
constexpr int kPlanIter = kPlanBlock / (64 * kPlanWaves);  // slots that a lane takes

// The lanes of this wave whose id equals this lane's; ids of `bits` bits.
__device__ __forceinline__ uint64_t same_id(int id, int bits) {
  uint64_t same = ~uint64_t(0);
  for (int k = 0; k < bits; ++k) {
    const uint64_t set = __ballot((id >> k) & 1);
    same &= (id >> k) & 1 ? set : ~set;
  }
  return same;
}

// This lane's ids, `experts` for dropped slots and experts + 1 past the end.
template <class ID, int ITER>
__device__ __forceinline__ void load_ids(const ID* ids, int64_t slots, int experts, int64_t first, int (&id)[ITER]) {
#pragma unroll
  for (int it = 0; it < ITER; ++it) {
    const int64_t i = first + 64 * it;
    id[it] = experts + 1;
    if (i < slots) {
      const ID v = ids[i];
      id[it] = v >= 0 && v < (ID)experts ? (int)v : experts;
    }
  }
}

// The lanes of this wave that have the same id as this one, for each of its slots.
template <int ITER>
__device__ __forceinline__ void match_ids(const int (&id)[ITER], int bits, uint64_t (&same)[ITER]) {
#pragma unroll
  for (int it = 0; it < ITER; ++it) same[it] = same_id(id[it], bits);
}

// Counts of this workgroup's slots by wave and id into cnt[wave][experts + 2]; the
// wave's slots begin at first - lane, `rounds` times 64 ITER of them.  id and same
// are left as of the last round.
template <class ID, int ITER>
__device__ __forceinline__ void count_ids(const ID* ids, int64_t slots, int experts, int bits, int rounds,
                                          int64_t first, int* cnt, int (&id)[ITER], uint64_t (&same)[ITER]) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, cols = experts + 2;
  load_ids(ids, slots, experts, first, id);
  for (int i = threadIdx.x; i < kPlanWaves * cols; i += blockDim.x) cnt[i] = 0;
  __syncthreads();
  for (int r = 0; r < rounds; ++r) {
    if (r > 0) load_ids(ids, slots, experts, first + (int64_t)r * (64 * ITER), id);
    match_ids(id, bits, same);
#pragma unroll
    for (int it = 0; it < ITER; ++it) {
      if ((same[it] & ((uint64_t(1) << lane) - 1)) == 0) cnt[wave * cols + id[it]] += __popcll(same[it]);
      __builtin_amdgcn_wave_barrier();
    }
  }
  __syncthreads();
}

// This lane's first slot.
template <int ITER>
__device__ __forceinline__ int64_t first_slot(int rounds) {
  return ((int64_t)blockIdx.x * kPlanWaves + (threadIdx.x >> 6)) * (int64_t)(64 * ITER) * rounds + (threadIdx.x & 63);
}

// hist[workgroup][id] for ids 0 .. experts.
template <class ID>
__global__ __launch_bounds__(64 * kPlanWaves) void k_plan_count(const ID* ids, int64_t slots, int experts, int bits,
                                                                int rounds, int32_t* hist) {
  extern __shared__ int cnt[];
  int id[kPlanIter];
  uint64_t same[kPlanIter];
  count_ids(ids, slots, experts, bits, rounds, first_slot<kPlanIter>(rounds), cnt, id, same);
  for (int e = threadIdx.x; e <= experts; e += blockDim.x) {
    int n = 0;
    for (int w = 0; w < kPlanWaves; ++w) n += cnt[w * (experts + 2) + e];
    hist[(int64_t)blockIdx.x * (experts + 1) + e] = n;
  }
}

template <class ID, int ITER>
__global__ __launch_bounds__(64 * kPlanWaves) void k_plan_place(const ID* ids, int64_t slots, int experts, int bits,
                                                                int rounds, const int32_t* hist, int32_t* offsets,
                                                                int32_t* k_offsets, int32_t* order, int32_t* place) {
  extern __shared__ int cnt[];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, cols = experts + 2;
  int* total = cnt + kPlanWaves * cols;  // slots of each id, then where they begin
  int id[ITER];
  uint64_t same[ITER];
  const int64_t i0 = first_slot<ITER>(rounds);
  count_ids(ids, slots, experts, bits, rounds, i0, cnt, id, same);
  // counts of the waves before each wave, after those of the workgroups before this one
  for (int e = threadIdx.x; e <= experts; e += blockDim.x) {
    int before = 0, all = 0;
    for (int b = 0; hist && b < (int)gridDim.x; ++b) {
      const int n = hist[(int64_t)b * (experts + 1) + e];
      before += b < (int)blockIdx.x ? n : 0;
      all += n;
    }
    int run = before;
    for (int w = 0; w < kPlanWaves; ++w) {
      const int n = cnt[w * cols + e];
      cnt[w * cols + e] = run;
      run += n;
    }
    total[e] = hist ? all : run;
  }
  __syncthreads();
  if (wave == 0) {
    int first = 0, k_first = 0;
    for (int c = 0; c <= experts; c += 64) {
      const int e = c + lane, n = e <= experts ? total[e] : 0;
      const int places = e < experts ? (n + 127) / 128 * 128 : 0;
      const int upto = first + wave_scan(n), k_upto = k_first + wave_scan(places);
      if (e <= experts) {
        total[e] = upto - n;
        if (blockIdx.x == 0) {
          offsets[e] = upto - n;
          k_offsets[e] = k_upto - places;
        }
      }
      first = __builtin_amdgcn_readlane(upto, 63);
      k_first = __builtin_amdgcn_readlane(k_upto, 63);
    }
  }
  __syncthreads();
  for (int r = 0; r < rounds; ++r) {
    const int64_t i1 = i0 + (int64_t)r * (64 * ITER);
    if (rounds > 1) {
      load_ids(ids, slots, experts, i1, id);
      match_ids(id, bits, same);
    }
#pragma unroll
    for (int it = 0; it < ITER; ++it) {
      const int rank = __popcll(same[it] & ((uint64_t(1) << lane) - 1));
      const int64_t i = i1 + 64 * it;
      int* run = &cnt[wave * cols + id[it]];
      const int before = *run;
      __builtin_amdgcn_wave_barrier();  // every lane has read before the first of each id adds
      if (rank == 0) *run = before + __popcll(same[it]);
      __builtin_amdgcn_wave_barrier();
      if (i < slots) {
        const int p = total[id[it]] + before + rank;
        order[p] = (int32_t)i;
        place[i] = p;
      }
    }
  }
}

// Rounds of kPlanBlock slots that a workgroup takes, and workgroups.
int plan_rounds(int64_t slots) {
  const int64_t most = (int64_t)kPlanMost * kPlanBlock;
  return slots > most ? (int)((slots + most - 1) / most) : 1;
}
int64_t plan_blocks(int64_t slots) {
  const int64_t each = (int64_t)kPlanBlock * plan_rounds(slots);
  return slots > 0 ? (slots + each - 1) / each : 1;
}

template <class ID>
hipError_t plan_t(const ID* ids, int64_t slots, int experts, int32_t* offsets, int32_t* k_offsets, int32_t* order,
                  int32_t* place, int32_t* ws, hipStream_t s) {
  const int64_t blocks = plan_blocks(slots);
  const int rounds = plan_rounds(slots);
  int bits = 1;
  while ((experts + 1) >> bits) ++bits;
  const size_t lds = (size_t)((kPlanWaves + 1) * (experts + 2)) * 4;
  if (blocks > 1) {
    hipLaunchKernelGGL((k_plan_count<ID>), dim3((unsigned)blocks), dim3(64 * kPlanWaves), lds, s, ids, slots, experts,
                       bits, rounds, ws);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
#define FASTBFP_PLACE(ITER)                                                                                       \
  hipLaunchKernelGGL((k_plan_place<ID, ITER>), dim3((unsigned)blocks), dim3(64 * kPlanWaves), lds, s, ids, slots, \
                     experts, bits, rounds, blocks > 1 ? ws : nullptr, offsets, k_offsets, order, place)
  if (slots <= 64 * kPlanWaves) FASTBFP_PLACE(1);
  else FASTBFP_PLACE(kPlanIter);
#undef FASTBFP_PLACE
  return hipGetLastError();
}

}  // namespace

int64_t expert_places(int64_t slots, int experts) {
  const int64_t busy = slots < experts ? slots : experts;  // each ends at most 127 places after its last slot
  return (slots + 127 * busy) / 128 * 128;
}

int64_t expert_plan_ws(int64_t slots, int experts) {
  const int64_t blocks = plan_blocks(slots);
  return blocks > 1 ? blocks * (experts + 1) : 0;
}

hipError_t launch_expert_plan(const void* ids, bool ids64, int64_t slots, int experts, int32_t* offsets,
                              int32_t* k_offsets, int32_t* order, int32_t* place, int32_t* ws, hipStream_t s) {
  if (ids64) return plan_t(static_cast<const int64_t*>(ids), slots, experts, offsets, k_offsets, order, place, ws, s);
  return plan_t(static_cast<const int32_t*>(ids), slots, experts, offsets, k_offsets, order, place, ws, s);
}

// ---- the weighted sum of the experts' outputs ----------------------------
//
// out[t] = sum over j of gates[t][j] y[place[t top + j]], added in the order of
// j in FP32; slots whose place is not before offsets[experts] were dropped and
// add nothing.  Every row of y is read once and every row of out written once:
// bound by HBM.  A thread takes four columns of a token (V = 4), so that a wave
// reads 1 KB of a row at a time; rows that are not 16-byte aligned go value by
// value (V = 1).  8192 tokens of 4 slots, 4096 columns: 106 us, 5.8 TB/s (a copy of
// 1 GB reaches 5.1); 16 tokens of 2: 2.9 us, a launch.
namespace {

template <int V> struct vec;
template <> struct vec<4> { typedef float type __attribute__((ext_vector_type(4))); };
template <> struct vec<1> { typedef float type __attribute__((ext_vector_type(1))); };

template <int V, bool GATES>
__global__ __launch_bounds__(256) void k_combine(const float* __restrict__ y, const float* __restrict__ gates,
                                                 const int32_t* __restrict__ place, const int32_t* __restrict__ offsets,
                                                 int experts, int64_t tokens, int top, int64_t N, int64_t per_row,
                                                 int64_t slots, float* __restrict__ out) {
  typedef typename vec<V>::type v_t;
  const int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x, t = q / per_row, c = (q - t * per_row) * V;
  if (t >= tokens) return;
  const int kept = min(max(offsets[experts], 0), (int)slots);
  v_t sum = {};
#pragma unroll 4
  for (int j = 0; j < top; ++j) {
    const int p = place[t * top + j];
    if (p < 0 || p >= kept) continue;
    const v_t v = __builtin_nontemporal_load(reinterpret_cast<const v_t*>(y + (int64_t)p * N + c));
    sum += GATES ? gates[t * top + j] * v : v;
  }
  __builtin_nontemporal_store(sum, reinterpret_cast<v_t*>(out + t * N + c));
}

// dy[place[slot]] = gates[slot] dout[token], dgates[slot] = dout[token] .
// y[place[slot]]; zeros for dropped slots.  WPS waves take a slot: one where
// there are enough slots to fill the card, so that the slots of a token, which
// follow one another, read its row of dout from the same L1; four otherwise.
// Four products at a time are added in FP32 and those sums in 64 bits (lane by lane in
// the order of the columns, then over the lanes and waves in a fixed tree), rounded
// once.  (A chain of N / 64 FP32 sums a lane, which this replaces, was as fast and the
// largest part of the error; 64 bits from the products on took 4% longer.)  Bound by
// HBM: y read and dy written once, 211 us or 5.5 TB/s for 8192 tokens of 4 slots and
// 4096 columns.
template <int V, int WPS>
__global__ __launch_bounds__(256) void k_combine_grad(const float* __restrict__ dout, const float* __restrict__ y,
                                                      const float* __restrict__ gates,
                                                      const int32_t* __restrict__ place,
                                                      const int32_t* __restrict__ offsets, int experts, int top,
                                                      int64_t N, int64_t slots, float* __restrict__ dy,
                                                      float* __restrict__ dgates) {
  typedef typename vec<V>::type v_t;
  __shared__ double part[4];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t slot = (int64_t)blockIdx.x * (4 / WPS) + wave / WPS;
  const bool live = slot < slots;
  double dot = 0.0;
  if (live) {
    const int p = place[slot], kept = min(max(offsets[experts], 0), (int)slots);
    const bool in = p >= 0 && p < kept;
    if (p >= 0 && p < slots) {
      const float g = gates ? gates[slot] : 1.0f;
      const float *d = dout + slot / top * N, *src = y + (int64_t)p * N;
      float* dst = dy + (int64_t)p * N;
#pragma unroll 4
      for (int64_t c = ((wave % WPS) * 64 + lane) * V; c < N; c += 64 * WPS * V) {
        v_t r = {};
        if (in) {
          const v_t a = *reinterpret_cast<const v_t*>(d + c);
          const v_t b = __builtin_nontemporal_load(reinterpret_cast<const v_t*>(src + c));
          r = g * a;
          float sum = a[0] * b[0];
#pragma unroll
          for (int k = 1; k < V; ++k) sum = __builtin_fmaf(a[k], b[k], sum);
          dot += (double)sum;
        }
        __builtin_nontemporal_store(r, reinterpret_cast<v_t*>(dst + c));
      }
    }
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) dot += __shfl_xor(dot, off);
  if constexpr (WPS > 1) {
    if (lane == 0) part[wave] = dot;
    __syncthreads();
    dot = (part[0] + part[1]) + (part[2] + part[3]);
  }
  if (live && dgates && lane == 0 && wave % WPS == 0) dgates[slot] = (float)dot;
}

bool rows_aligned(int64_t N, const void* a, const void* b, const void* c) {
  auto al = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
  return N % 4 == 0 && al(a) && al(b) && al(c);
}

}  // namespace

hipError_t launch_combine_experts(const float* y, const float* gates, const int32_t* place, const int32_t* offsets,
                                  int experts, int64_t tokens, int top, int64_t N, float* out, hipStream_t s) {
  if (tokens == 0 || N == 0) return hipSuccess;
  const int V = rows_aligned(N, y, out, nullptr) ? 4 : 1;
  const int64_t per_row = N / V, blocks = (tokens * per_row + 255) / 256, slots = tokens * top;
  if (blocks > 0x7fffffff) return hipErrorInvalidValue;  // (the caller checks)
#define FASTBFP_COMBINE(V, GATES)                                                                                    \
  hipLaunchKernelGGL((k_combine<V, GATES>), dim3((unsigned)blocks), dim3(256), 0, s, y, gates, place, offsets, experts, \
                     tokens, top, N, per_row, slots, out)
  if (V == 4 && gates) FASTBFP_COMBINE(4, true);
  else if (V == 4) FASTBFP_COMBINE(4, false);
  else if (gates) FASTBFP_COMBINE(1, true);
  else FASTBFP_COMBINE(1, false);
#undef FASTBFP_COMBINE
  return hipGetLastError();
}

hipError_t launch_combine_experts_grad(const float* dout, const float* y, const float* gates, const int32_t* place,
                                       const int32_t* offsets, int experts, int64_t tokens, int top, int64_t N,
                                       float* dy, float* dgates, hipStream_t s) {
  const int64_t slots = tokens * top;
  if (slots == 0) return hipSuccess;
  const int V = rows_aligned(N, dout, y, dy) ? 4 : 1;
  const int wps = slots >= 4096 ? 1 : 4;
  const int64_t blocks = wps == 1 ? (slots + 3) / 4 : slots;
#define FASTBFP_COMBINE(V, WPS)                                                                                   \
  hipLaunchKernelGGL((k_combine_grad<V, WPS>), dim3((unsigned)blocks), dim3(256), 0, s, dout, y, gates, place,    \
                     offsets, experts, top, N, slots, dy, dgates)
  if (V == 4 && wps == 1) FASTBFP_COMBINE(4, 1);
  else if (V == 4) FASTBFP_COMBINE(4, 4);
  else if (wps == 1) FASTBFP_COMBINE(1, 1);
  else FASTBFP_COMBINE(1, 4);
#undef FASTBFP_COMBINE
  return hipGetLastError();
}

}  // namespace fastbfp
