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
  int V, L, K, M;
  int cols, blocks;    // columns of a block, blocks of a row
};

// A block takes `cols` columns of one row.  They are read, masked and written as they come; meanwhile it goes through the
// row's tokens: words of shared memory for the columns that occur (and only those) are cleared, then counted up, integer
// atomics whose order does not matter; who finds a column unmarked puts it on a list.  Of several biases of a column the
// first one's number is kept; the others, if there are any, are looked for in list order.  At last the columns of the list
// are read back, changed and written again.  (Done for every element of a vector in turn instead, the code is so long that
// a block waits for instructions: 256 rows of 131072 bf16 logits and 4096 tokens 151 us.)  Bound: reading and writing the
// logits; the tokens are read once per block, from L2.
template <class T, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) k_penalize(PenaltyArgs a) {
  constexpr int E = 16 / sizeof(T), kCols = THREADS * kVectors * E;
  extern __shared__ uint32_t count[];              // [kCols]: later occurrences; the top bit: occurs among the first `prompt` tokens
  uint32_t* touched = count + (a.L > 0 ? kCols : 0);                        // [kCols / 32]
  uint16_t* link = reinterpret_cast<uint16_t*>(touched + kCols / 32);       // [kCols]: the first bias of a column
  uint16_t* list = link + (a.K > 0 ? kCols : 0);                            // the marked columns: no more than L + K, or kCols
  __shared__ int listed, repeated;
  const int b = blockIdx.x / a.blocks;
  const int v0 = (blockIdx.x - b * a.blocks) * a.cols, v1 = min(v0 + a.cols, a.V);
  // vectors lie on 16 bytes of the whole array, a row may start between two of them: column v is word v - origin
  const long long row = (long long)b * a.V;
  const int origin = (int)((row + v0) / E * E - row);
  union Vector { uint4 raw; T x[E]; };
  follow();
  const T* from = static_cast<const T*>(a.logits) + row;
  T* to = static_cast<T*>(a.out) + row;
  const bool marks = a.L > 0 || a.K > 0;
  const int* tokens = a.tokens + (size_t)b * a.L;
  const int* ids = a.ids + (size_t)b * a.K;
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
#pragma unroll
  for (int k = 0; k < kHeld; ++k) held[k] = k * THREADS + (int)threadIdx.x < a.L ? tokens[k * THREADS + threadIdx.x] : -1;
  // the warp that goes through the biases has the last of them at hand
  const int bias_lane = (int)threadIdx.x - (THREADS - 32), last_bias = (a.K - 1) / 32 * 32 + bias_lane;
  const int last_id = a.K > 0 && bias_lane >= 0 && last_bias < a.K ? ids[last_bias] : -1;
  const uint32_t width = v1 - v0;
  if (marks) {
    for (int i = threadIdx.x; i < kCols / 32; i += THREADS) touched[i] = 0;
    if (threadIdx.x == 0) listed = repeated = 0;
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
  if (!marks) return;
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
  if (bias_lane >= 0 && a.K > 0) {                             // from the last bias to the first, 32 at a time
    const int lane = bias_lane;
    int v = last_id;
    for (int k = last_bias; k >= lane; k -= 32) {
      const int before = k >= 32 + lane ? ids[k - 32] : -1;
      const bool mine = (uint32_t)(v - v0) < width;
      const uint32_t same = __match_any_sync(~0u, mine ? v : -1 - lane);
      if (mine && ((same & (same - 1)) || link[v - origin] != kNoBias)) repeated = 1;
      __syncwarp();
      if (mine && lane == __ffs(same) - 1) link[v - origin] = (uint16_t)k;
      if (mine) put_on_list(v - origin);
      __syncwarp();
      v = before;
    }
  }
  __syncthreads();
  const int n = listed;
#pragma unroll 1
  for (int i = threadIdx.x; i < n; i += THREADS) {
    const int w = list[i], v = origin + w;
    if (a.M > 0 && !(mask[v >> 5] >> (v & 31) & 1)) continue;
    float x = widen<T>(to[v]);
    const uint32_t c = a.L > 0 ? count[w] : 0;
    if (c) {
      x = x > 0 ? __fdiv_rn(x, p.x) : __fmul_rn(x, p.x);
      const uint32_t times = c & 0x7FFFFFFFu;
      if (times) x = __fsub_rn(__fsub_rn(x, __fmul_rn(p.y, (float)times)), p.z);
    }
    const int first = a.K > 0 ? link[w] : kNoBias;
    if (first != kNoBias) {
      const float* bias = a.bias + (size_t)b * a.K;
      float sum = bias[first];
      if (repeated)
#pragma unroll 1
        for (int j = first + 1; j < a.K; ++j)
          if (ids[j] == v) sum = __fadd_rn(sum, bias[j]);
      x = __fadd_rn(x, sum);
    }
    to[v] = narrow<T>(x);
  }
}

template <class T, int THREADS>
int launch(const ClusterLaunch& L) {
  constexpr int E = 16 / sizeof(T), kCols = THREADS * kVectors * E;
  const int B = (int)L.op.shape[0], V = (int)L.op.shape[1];
  PenaltyArgs a{report_of(L), slot(L, 0).ptr, slot_ptr<int>(L, 1), slot_ptr<float>(L, 2), slot_ptr<int>(L, 3), slot_ptr<float>(L, 4),
                slot_ptr<uint32_t>(L, 5), result_ptr<void>(L),
                V, slot(L, 1).C, slot(L, 3).C, slot(L, 5).C, V % E == 0 ? kCols : kCols - E, 0};
  a.blocks = (V + a.cols - 1) / a.cols;
  const size_t shared = a.L + a.K == 0 ? 0 : (size_t)kCols * ((a.L > 0 ? 4 : 0) + (a.K > 0 ? 2 : 0)) + kCols / 8 + 2 * std::min<size_t>((size_t)a.L + a.K, kCols);
  static std::atomic<uint64_t> allowed{0};
  const int rc = allow_shared(k_penalize<T, THREADS>, (size_t)kCols * 8 + kCols / 8, allowed);
  if (rc != ACC_OK) return rc;
  return launch_following(k_penalize<T, THREADS>, dim3((unsigned)B * (unsigned)a.blocks), THREADS, shared, L.stream, a);
}

// Large blocks where they still leave each SM a few: a row's tokens are then gone through fewer times.
template <class T>
int launch(const ClusterLaunch& L) {
  if (L.op.shape[0] == 0 || L.op.shape[1] == 0) return ACC_OK;
  constexpr int64_t kLarge = 512 * kVectors * (16 / sizeof(T));
  const int64_t blocks = L.op.shape[0] * ((L.op.shape[1] + kLarge - 1) / kLarge);
  return blocks >= 4 * sm_count() ? launch<T, 512>(L) : launch<T, 256>(L);
}

int launch_penalize(const ClusterLaunch& L) {
  return L.op.dtype == ACC_F32 ? launch<float>(L) : L.op.dtype == ACC_F16 ? launch<__half>(L) : launch<__nv_bfloat16>(L);
}

const Register penalize(ACC_PENALIZE, "k_penalize", no_scratch, launch_penalize);

}  // namespace
}  // namespace ops
}  // namespace acc
