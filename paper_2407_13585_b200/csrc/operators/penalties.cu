// Penalties for tokens seen before, biases and a mask on rows of logits (ACC_PENALIZE).
#include "operators/common.cuh"

namespace acc {
namespace ops {
namespace {

constexpr int kVectors = 4, kHeld = 8;      // 16-byte vectors, tokens in registers per thread
constexpr uint16_t kNoBias = 0xFFFF;

struct PenaltyArgs {
  Report report;
  const void* logits;
  const int* tokens;
  const float* params;
  const int* ids;
  const float* bias;
  const uint32_t* mask;
  void* out;
  float* sums;         // [B, K]: of the biases of a column, at the number of its first one
  int V, L, K, M;
  int cols, blocks;    // columns of a block, blocks of a row
  int table_bits;      // k_penalize_marked: log2 of the places of a block's table
};

// A logit that occurs c times (the top bit: also among the first `prompt` tokens) and the sum of its biases, -0 if it has
// none: x + -0 is x for every x.
__device__ __forceinline__ float changed(float x, uint32_t c, float bias, const float4& p) {
  if (c) {
    x = x > 0 ? __fdiv_rn(x, p.x) : __fmul_rn(x, p.x);
    const uint32_t times = c & 0x7FFFFFFFu;
    if (times) x = __fsub_rn(__fsub_rn(x, __fmul_rn(p.y, (float)times)), p.z);
  }
  return __fadd_rn(x, bias);
}

// By a whole warp: bias number k of a row goes to a column, if it is `mine`.  The first bias of a column leaves its number in
// the column's link, and the column's sum is kept at that number; a lane adds up for all lanes of its column, in their order.
// So every bias is looked at once, however often a column occurs (searched for in the rest of the list instead, 65535 biases
// of a row take 38 ms with one column twice; so 0.9).
__device__ __forceinline__ void add_bias(bool mine, int column, uint16_t* link, int k, float bias, float* sums) {
  const int lane = threadIdx.x & 31;
  const uint32_t same = __match_any_sync(~0u, mine ? column : -1 - lane);
  const bool adds = mine && lane == __ffs(same) - 1;
  const int had = adds ? *link : kNoBias;
  uint32_t left = adds ? same : 0;
  float sum = bias;
  if (__any_sync(~0u, had != kNoBias || (left & (left - 1)))) {
    sum = had != kNoBias ? sums[had] : -0.0f;
    while (__any_sync(~0u, left)) {
      const float next = __shfl_sync(~0u, bias, left ? __ffs(left) - 1 : 0);
      if (left) sum = __fadd_rn(sum, next);
      left &= left - 1;
    }
  }
  if (adds) {
    if (had == kNoBias) *link = (uint16_t)k;
    sums[had == kNoBias ? k : had] = sum;
  }
  __syncwarp();
}

// A block takes `cols` columns of one row.  They are read, masked and written as they come; meanwhile it goes through the
// row's tokens: words of shared memory for the columns that occur (and only those) are cleared, then counted up, integer
// atomics whose order does not matter; who finds a column unmarked puts it on a list.  One warp adds up the biases in list
// order.  At last the columns of the list are read back, changed and written again.  (Done for every element of a vector in
// turn instead, the code is so long that a block waits for instructions: 256 rows of 131072 bf16 logits and 4096 tokens 151
// us.)  Bound: reading and writing the logits; the tokens are read once per block, from L2.
template <class T, int THREADS, bool MARKS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) k_penalize(PenaltyArgs a) {
  constexpr int E = 16 / sizeof(T), kCols = THREADS * kVectors * E;
  extern __shared__ __align__(16) uint32_t count[];      // [kCols]: later occurrences; the top bit: occurs among the first `prompt` tokens
  uint32_t* touched = count + (a.L > 0 ? kCols : 0);                        // [kCols / 32]
  uint16_t* link = reinterpret_cast<uint16_t*>(touched + kCols / 32);       // [kCols]: the first bias of a column
  uint16_t* list = link + (a.K > 0 ? kCols : 0);                            // the marked columns: no more than L + K, or kCols
  __shared__ int listed;
  const int b = blockIdx.x / a.blocks;
  const int v0 = (blockIdx.x - b * a.blocks) * a.cols, v1 = min(v0 + a.cols, a.V);
  // vectors lie on 16 bytes of the whole array, a row may start between two of them: column v is word v - origin
  const long long row = (long long)b * a.V;
  const int origin = (int)((row + v0) / E * E - row);
  union Vector { uint4 raw; T x[E]; };
  cudaGridDependencySynchronize();
  cudaTriggerProgrammaticLaunchCompletion();       // (only now: k_penalize_marked reads tokens before it waits for this kernel)
  const T* from = static_cast<const T*>(a.logits) + row;
  T* to = static_cast<T*>(a.out) + row;
  const int* tokens = a.tokens + (size_t)b * a.L;
  const int* ids = a.ids + (size_t)b * a.K;
  const float* biases = a.bias + (size_t)b * a.K;
  float* sums = a.sums + (size_t)b * a.K;
  const uint32_t* mask = a.mask + (size_t)b * a.M;
  Vector in[kVectors];
  uint32_t bits[kVectors][2];                      // the words that hold a vector's bits
  int held[kHeld];                                 // a thread's first tokens: they are gone through twice
#pragma unroll
  for (int k = 0; k < kVectors; ++k) {
    const int v = origin + (k * THREADS + (int)threadIdx.x) * E, at = max(v, 0);
    if (v >= v0 && v + E <= v1) in[k].raw = *reinterpret_cast<const uint4*>(from + v);
    bits[k][0] = a.M > 0 && v < v1 ? mask[at >> 5] : ~0u;
    bits[k][1] = a.M > 0 && v < v1 && (at & 31) + E > 32 && (at >> 5) + 1 < a.M ? mask[(at >> 5) + 1] : ~0u;
  }
  if constexpr (MARKS)
#pragma unroll
    for (int k = 0; k < kHeld; ++k) held[k] = k * THREADS + (int)threadIdx.x < a.L ? tokens[k * THREADS + threadIdx.x] : -1;
  // the warp that goes through the biases has the first of them at hand
  const int bias_lane = (int)threadIdx.x - (THREADS - 32);
  const bool has_bias = MARKS && bias_lane >= 0 && bias_lane < a.K;
  int id = has_bias ? ids[bias_lane] : -1;
  float bias = has_bias ? biases[bias_lane] : 0.0f;
  const uint32_t width = v1 - v0;
  if constexpr (MARKS) {
    for (int i = threadIdx.x; i < kCols / 32; i += THREADS) touched[i] = 0;
    if (threadIdx.x == 0) listed = 0;
    bool bad = false;
    const auto clear = [&](int v) {
      if ((uint32_t)(v - v0) < width) {
        if (a.L > 0) count[v - origin] = 0;
        if (a.K > 0) link[v - origin] = kNoBias;
      }
      bad = bad || v >= a.V;
    };
#pragma unroll
    for (int k = 0; k < kHeld; ++k) clear(held[k]);
#pragma unroll 4
    for (int i = kHeld * THREADS + threadIdx.x; i < a.L; i += THREADS) clear(tokens[i]);
#pragma unroll 1
    for (int k = threadIdx.x; k < a.K; k += THREADS) clear(ids[k]);
    if (bad) raise_index(a.report);
  }
  const T least = narrow<T>(-INFINITY);
#pragma unroll
  for (int k = 0; k < kVectors; ++k) {
    const int v = origin + (k * THREADS + (int)threadIdx.x) * E;
    if (v >= v1) break;
    const int at = max(v, 0);                                  // (a vector that starts before its row: the bits from column 0 on)
    const uint32_t allowed = __funnelshift_r(bits[k][0], bits[k][1], at & 31) << (at - v);
    if (v >= v0 && v + E <= v1) {
      if (a.M > 0) {
#pragma unroll
        for (int i = 0; i < E; ++i)
          if (!(allowed >> i & 1)) in[k].x[i] = least;
      }
      *reinterpret_cast<uint4*>(to + v) = in[k].raw;
    } else {
#pragma unroll 1
      for (int i = 0; i < E; ++i)
        if (v + i >= v0 && v + i < v1) to[v + i] = allowed >> i & 1 ? from[v + i] : least;
    }
  }
  if constexpr (!MARKS) return;
  const float4 p = *reinterpret_cast<const float4*>(a.params + 4 * (size_t)b);
  __syncthreads();
  const int prompt = (int)fminf(fmaxf(p.w, 0.0f), 2147483520.0f);
  const auto put_on_list = [&](int w) {
    const uint32_t bit = 1u << (w & 31);
    if (!(touched[w >> 5] & bit) && !(atomicOr(touched + (w >> 5), bit) & bit)) list[atomicAdd(&listed, 1)] = (uint16_t)w;
  };
  const auto note = [&](int v, int i) {
    if ((uint32_t)(v - v0) >= width) return;
    const int w = v - origin;
    if (i >= prompt) atomicAdd(count + w, 1u);
    else atomicOr(count + w, 0x80000000u);
    put_on_list(w);
  };
#pragma unroll
  for (int k = 0; k < kHeld; ++k) note(held[k], k * THREADS + threadIdx.x);
#pragma unroll 4
  for (int i = kHeld * THREADS + threadIdx.x; i < a.L; i += THREADS) note(tokens[i], i);
  if (bias_lane >= 0) {                                        // 32 at a time
    for (int k = bias_lane; k < a.K + bias_lane; k += 32) {
      const bool more = k + 32 < a.K;
      const int next_id = more ? ids[k + 32] : -1;
      const float next_bias = more ? biases[k + 32] : 0.0f;
      const bool mine = (uint32_t)(id - v0) < width;
      if (mine) put_on_list(id - origin);
      if (__any_sync(~0u, mine)) add_bias(mine, id, link + (mine ? id - origin : 0), k, bias, sums);
      id = next_id, bias = next_bias;
    }
  }
  __syncthreads();
  const int n = listed;
#pragma unroll 1
  for (int i = threadIdx.x; i < n; i += THREADS) {
    const int w = list[i], v = origin + w;
    if (a.M > 0 && !(mask[v >> 5] >> (v & 31) & 1)) continue;
    const int bias = a.K > 0 ? link[w] : kNoBias;
    to[v] = narrow<T>(changed(widen<T>(to[v]), a.L > 0 ? count[w] : 0, bias != kNoBias ? sums[bias] : -0.0f, p));
  }
}

// Large batches: the rows are copied and masked by k_penalize without tokens, at the rate of a copy, and this kernel changes
// the columns that occur, behind it.  A block takes a range of the columns of one row (all of them, if rows are many), and
// counts the row's tokens that lie there in a hash table of at least half as many places again as tokens and biases:
// shared memory goes by the tokens, not by the columns.  It does that before it waits for the copy; then it goes through the
// table.  Which place a column gets depends on the order of the threads, what is written to it does not.
constexpr int kMarkedThreads = 512, kMaxTableBits = 14, kMaxTableBytes = (10 << kMaxTableBits) + (4 << kMaxTableBits) / 3;
constexpr int kEmptyPlace = -1;
constexpr size_t kThirdOfAnSM = 77 << 10;   // shared memory that three blocks of an SM cannot have
template <class T>
__global__ void __launch_bounds__(kMarkedThreads, 2) k_penalize_marked(PenaltyArgs a) {
  extern __shared__ __align__(16) uint32_t count[];                         // [places]
  const int places = 1 << a.table_bits;
  int* key = reinterpret_cast<int*>(count + places);                        // [places]: the column
  uint16_t* link = reinterpret_cast<uint16_t*>(key + places);               // [places]: the first bias of a column
  uint16_t* list = link + (a.K > 0 ? places : 0);                           // the places that were taken: no more than L + K
  __shared__ int listed;
  const int b = blockIdx.x / a.blocks;
  const int v0 = (blockIdx.x - b * a.blocks) * a.cols, v1 = min(v0 + a.cols, a.V);
  const uint32_t width = v1 - v0;
  const int* tokens = a.tokens + (size_t)b * a.L;
  const int* ids = a.ids + (size_t)b * a.K;
  const float* biases = a.bias + (size_t)b * a.K;
  float* sums = a.sums + (size_t)b * a.K;
  const uint32_t* mask = a.mask + (size_t)b * a.M;
  int held[kHeld];
#pragma unroll
  for (int k = 0; k < kHeld; ++k) held[k] = k * kMarkedThreads + (int)threadIdx.x < a.L ? tokens[k * kMarkedThreads + threadIdx.x] : -1;
  const int bias_lane = (int)threadIdx.x - (kMarkedThreads - 32);
  const bool has_bias = bias_lane >= 0 && bias_lane < a.K;
  int id = has_bias ? ids[bias_lane] : -1;
  float bias = has_bias ? biases[bias_lane] : 0.0f;
  const float4 p = *reinterpret_cast<const float4*>(a.params + 4 * (size_t)b);
  // (64 places at least: every array is a multiple of 16 bytes)
  for (int i = threadIdx.x; i < places / 4; i += kMarkedThreads) {
    reinterpret_cast<uint4*>(count)[i] = make_uint4(0, 0, 0, 0);
    reinterpret_cast<int4*>(key)[i] = make_int4(kEmptyPlace, kEmptyPlace, kEmptyPlace, kEmptyPlace);
  }
  if (a.K > 0)
    for (int i = threadIdx.x; i < places / 8; i += kMarkedThreads) reinterpret_cast<uint4*>(link)[i] = make_uint4(~0u, ~0u, ~0u, ~0u);
  if (threadIdx.x == 0) listed = 0;
  __syncthreads();
  const int prompt = (int)fminf(fmaxf(p.w, 0.0f), 2147483520.0f);
  bool bad = false;
  const auto place_of = [&](int v, bool& taken) {  // (the table is never full: every probe ends)
    uint32_t i = (uint32_t)v * 2654435769u >> (32 - a.table_bits);
    for (;; i = (i + 1) & (places - 1)) {
      int found = key[i];
      if (found == kEmptyPlace) {
        found = atomicCAS(key + i, kEmptyPlace, v);
        taken = found == kEmptyPlace;
      }
      if (taken || found == v) return i;
    }
  };
  const auto put_on_list = [&](bool taken, uint32_t place) {      // by a whole warp, one addition for all of it
    const uint32_t all = __ballot_sync(~0u, taken);
    if (all == 0) return;
    const int lane = threadIdx.x & 31;
    int first = lane == 0 ? atomicAdd(&listed, __popc(all)) : 0;
    first = __shfl_sync(~0u, first, 0);
    if (taken) list[first + __popc(all & ((1u << lane) - 1))] = (uint16_t)place;
  };
  const auto note = [&](int v, int i) {
    bad = bad || v >= a.V;
    bool taken = false;
    uint32_t place = 0;
    if ((uint32_t)(v - v0) < width) {
      place = place_of(v, taken);
      if (i >= prompt) atomicAdd(count + place, 1u);
      else atomicOr(count + place, 0x80000000u);
    }
    put_on_list(taken, place);
  };
#pragma unroll
  for (int k = 0; k < kHeld; ++k)
    if (k * kMarkedThreads < a.L) note(held[k], k * kMarkedThreads + threadIdx.x);
#pragma unroll 1
  for (int i0 = kHeld * kMarkedThreads; i0 < a.L; i0 += kMarkedThreads) {
    const int i = i0 + threadIdx.x;
    note(i < a.L ? tokens[i] : -1, i);
  }
  if (bias_lane >= 0) {                            // 32 at a time
    for (int k = bias_lane; k < a.K + bias_lane; k += 32) {
      const bool more = k + 32 < a.K;
      const int next_id = more ? ids[k + 32] : -1;
      const float next_bias = more ? biases[k + 32] : 0.0f;
      bad = bad || id >= a.V;
      const bool mine = (uint32_t)(id - v0) < width;
      bool taken = false;
      const uint32_t place = mine ? place_of(id, taken) : 0;
      put_on_list(taken, place);
      if (__any_sync(~0u, mine)) add_bias(mine, id, link + place, k, bias, sums);
      id = next_id, bias = next_bias;
    }
  }
  if (bad) raise_index(a.report);
  __syncthreads();
  cudaTriggerProgrammaticLaunchCompletion();
  cudaGridDependencySynchronize();
  T* to = static_cast<T*>(a.out) + (long long)b * a.V;
  const int n = listed;
  constexpr int kAhead = 4;
#pragma unroll 1
  for (int i0 = threadIdx.x; i0 < n; i0 += kAhead * kMarkedThreads) {
    int v[kAhead], first[kAhead];
    float x[kAhead], bias[kAhead];
    uint32_t c[kAhead], word[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int i = i0 + k * kMarkedThreads, place = i < n ? list[i] : 0;
      v[k] = i < n ? key[place] : kEmptyPlace;
      x[k] = v[k] >= 0 ? widen<T>(to[v[k]]) : 0.0f;
      word[k] = v[k] < 0 ? 0 : a.M > 0 ? mask[v[k] >> 5] : ~0u;
      c[k] = count[place];
      first[k] = a.K > 0 ? link[place] : kNoBias;
      bias[k] = first[k] != kNoBias ? sums[first[k]] : -0.0f;
    }
#pragma unroll 1
    for (int k = 0; k < kAhead; ++k) {
      if (word[0] >> (v[0] & 31) & 1) to[v[0]] = narrow<T>(changed(x[0], c[0], bias[0], p));
#pragma unroll
      for (int u = 0; u + 1 < kAhead; ++u) v[u] = v[u + 1], x[u] = x[u + 1], c[u] = c[u + 1], word[u] = word[u + 1], bias[u] = bias[u + 1];
    }
  }
}

PenaltyArgs arguments(const ClusterLaunch& L) {
  return {report_of(L), slot(L, 0).ptr, slot_ptr<int>(L, 1), slot_ptr<float>(L, 2), slot_ptr<int>(L, 3), slot_ptr<float>(L, 4),
          slot_ptr<uint32_t>(L, 5), result_ptr<void>(L), reinterpret_cast<float*>(L.scratch), (int)L.op.shape[1], slot(L, 1).C, slot(L, 3).C, slot(L, 5).C, 0, 0, 0};
}

template <class T, int THREADS, bool MARKS>
int launch(const ClusterLaunch& L, PenaltyArgs a) {
  constexpr int E = 16 / sizeof(T), kCols = THREADS * kVectors * E;
  a.cols = a.V % E == 0 ? kCols : kCols - E;
  a.blocks = (a.V + a.cols - 1) / a.cols;
  const size_t shared = !MARKS ? 0 : (size_t)kCols * ((a.L > 0 ? 4 : 0) + (a.K > 0 ? 2 : 0)) + kCols / 8 + 2 * std::min<size_t>((size_t)a.L + a.K, kCols);
  if (MARKS) {
    static std::atomic<uint64_t> allowed{0};
    const int rc = allow_shared(k_penalize<T, THREADS, MARKS>, (size_t)kCols * 8 + kCols / 8, allowed);
    if (rc != ACC_OK) return rc;
  }
  return launch_following(k_penalize<T, THREADS, MARKS>, dim3((unsigned)L.op.shape[0] * (unsigned)a.blocks), THREADS, shared, L.stream, a);
}

template <class T>
int launch_marked(const ClusterLaunch& L, PenaltyArgs a) {
  a.table_bits = 6;
  while ((2ll << a.table_bits) < 3ll * (a.L + a.K)) ++a.table_bits;
  // two blocks to an SM, none with fewer than 4096 columns
  const int B = (int)L.op.shape[0];
  a.blocks = std::max(1, std::min(2 * sm_count() / B, a.V / 4096));
  a.cols = (a.V + a.blocks - 1) / a.blocks;
  const auto bytes = [&](int bits) { return ((size_t)(a.K > 0 ? 10 : 8) << bits) + 2 * ((size_t)a.L + a.K); };
  static std::atomic<uint64_t> allowed{0};
  const int rc = allow_shared(k_penalize_marked<T>, (size_t)kMaxTableBytes, allowed);
  if (rc != ACC_OK) return rc;
  ++L.extra_launches;
  // (blocks that two to an SM hold are not put three to those SMs that the copy leaves first: 256 rows, 4096 tokens 70 us, so 43)
  const unsigned grid = (unsigned)B * (unsigned)a.blocks;
  const size_t shared = std::max(bytes(a.table_bits), grid <= 2u * sm_count() ? kThirdOfAnSM : 0);
  return launch_following(k_penalize_marked<T>, dim3(grid), kMarkedThreads, shared, L.stream, a);
}

// From this many logits on, two kernels (with a mask; one kernel, two, in us).  Rows of 131072: 256 of bf16 with 4096 tokens 54, 48,
// with 256 tokens 43, 28; 32 of fp32 with 4096 20, 15, of bf16 with 2000 11, 10; 16 of bf16 9.2, 9.5.  Shorter rows, with 20
// to 64 biases: 256 of 32000 and 2000 tokens 17.4, 18.6; 256 of 16384 and 2000 13.8, 15.7; 1000 of 8000 and 500 18, 20; 2000
// of 4000 and 500 30, 30; 4000 of 1000 and 300 50, 45, and 4000 76, 95.
constexpr int64_t kTwoKernels = 1 << 22;
template <class T>
int launch(const ClusterLaunch& L) {
  PenaltyArgs a = arguments(L);
  if (L.op.shape[0] == 0 || L.op.shape[1] == 0) {
    no_launch(L);
    const int rc = report_beyond(L, a.tokens, L.op.shape[0] * a.L, a.V);
    return rc == ACC_OK ? report_beyond(L, a.ids, L.op.shape[0] * a.K, a.V) : rc;
  }
  const int64_t marks = (int64_t)a.L + a.K;
  if (marks == 0) return launch<T, 256, false>(L, a);
  if (L.op.shape[0] * L.op.shape[1] >= kTwoKernels && 3 * marks <= 2 << kMaxTableBits) {
    const int rc = launch<T, 256, false>(L, a);
    return rc == ACC_OK ? launch_marked<T>(L, a) : rc;
  }
  // large blocks where they still leave each SM a few: a row's tokens are then gone through fewer times
  constexpr int64_t kLarge = 512 * kVectors * (16 / sizeof(T));
  const int64_t blocks = L.op.shape[0] * ((L.op.shape[1] + kLarge - 1) / kLarge);
  return blocks >= 4 * sm_count() ? launch<T, 512, true>(L, a) : launch<T, 256, true>(L, a);
}

int launch_penalize(const ClusterLaunch& L) {
  return L.op.dtype == ACC_F32 ? launch<float>(L) : L.op.dtype == ACC_F16 ? launch<__half>(L) : launch<__nv_bfloat16>(L);
}

int64_t penalties_scratch(const ClusterLaunch& L) { return L.op.shape[1] > 0 ? 4 * L.op.shape[0] * slot(L, 3).C : 0; }

const Register penalize(ACC_PENALIZE, "k_penalize", penalties_scratch, launch_penalize);

}  // namespace
}  // namespace ops
}  // namespace acc
