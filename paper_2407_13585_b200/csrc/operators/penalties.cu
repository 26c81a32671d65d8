// Penalties for tokens seen before, biases and a mask on rows of logits (ACC_PENALIZE).
#include "operators/common.cuh"

namespace acc {
namespace ops {
namespace {

constexpr int kThreads = 256, kVectors = 4;      // 16-byte vectors per thread

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

// A block takes `cols` columns of one row, whose logits it asks for before anything else.  Meanwhile it goes through the
// row's tokens: words of shared memory for the columns that occur (and only those) are cleared, then counted up, integer
// atomics whose order does not matter; a bitmap says which columns to look at.  Of several biases of a column the first
// one's number is kept; the others, if there are any, are looked for in list order.  Bound: reading and writing the
// logits; the tokens are read once per block, from L2.
template <class T>
__global__ void __launch_bounds__(kThreads) k_penalize(PenaltyArgs a) {
  constexpr int E = 16 / sizeof(T), kCols = kThreads * kVectors * E;
  __shared__ uint32_t touched[kCols / 32];
  extern __shared__ uint32_t words[];
  uint32_t* count = words;                         // [kCols]: later occurrences; the top bit: occurs among the first `prompt` tokens
  int* link = reinterpret_cast<int*>(words) + (a.L > 0 ? kCols : 0);   // [kCols]: the first bias of a column
  __shared__ int repeated;
  const int b = blockIdx.x / a.blocks;
  const int v0 = (blockIdx.x - b * a.blocks) * a.cols, v1 = min(v0 + a.cols, a.V);
  // vectors lie on 16 bytes of the whole array, a row may start between two of them: column v is word v - origin
  const long long row = (long long)b * a.V;
  const int origin = (int)((row + v0) / E * E - row);
  union Vector { uint4 raw; T x[E]; };
  Vector in[kVectors];
  const T* from = static_cast<const T*>(a.logits) + row;
#pragma unroll
  for (int k = 0; k < kVectors; ++k) {
    const int v = origin + (k * kThreads + (int)threadIdx.x) * E;
    if (v >= v0 && v + E <= v1) in[k].raw = *reinterpret_cast<const uint4*>(from + v);
    else
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (v + i >= v0 && v + i < v1) in[k].x[i] = from[v + i];
  }
  const bool marks = a.L > 0 || a.K > 0;
  float rep = 1, freq = 0, pres = 0;
  if (marks) {
    const int* tokens = a.tokens + (size_t)b * a.L;
    const int* ids = a.ids + (size_t)b * a.K;
    const float4 p = *reinterpret_cast<const float4*>(a.params + 4 * (size_t)b);
    rep = p.x, freq = p.y, pres = p.z;
    const int prompt = (int)fminf(fmaxf(p.w, 0.0f), 2147483520.0f);
    for (int i = threadIdx.x; i < kCols / 32; i += kThreads) touched[i] = 0;
    if (threadIdx.x == 0) repeated = 0;
    bool bad = false;
    for (int i = threadIdx.x; i < a.L; i += kThreads) {
      const int v = tokens[i];
      if (v >= v0 && v < v1) {
        count[v - origin] = 0;
        if (a.K > 0) link[v - origin] = 0x7FFFFFFF;
      }
      bad = bad || v >= a.V;
    }
    for (int k = threadIdx.x; k < a.K; k += kThreads) {
      const int v = ids[k];
      if (v >= v0 && v < v1) {
        if (a.L > 0) count[v - origin] = 0;
        link[v - origin] = 0x7FFFFFFF;
      }
      bad = bad || v >= a.V;
    }
    if (bad) raise_index(a.report);
    __syncthreads();
    for (int i = threadIdx.x; i < a.L; i += kThreads) {
      const int v = tokens[i];
      if (v < v0 || v >= v1) continue;
      const int w = v - origin;
      if (i >= prompt) atomicAdd(count + w, 1u);
      else atomicOr(count + w, 0x80000000u);
      atomicOr(touched + (w >> 5), 1u << (w & 31));
    }
    for (int k = threadIdx.x; k < a.K; k += kThreads) {
      const int v = ids[k];
      if (v < v0 || v >= v1) continue;
      const int w = v - origin;
      atomicMin(link + w, k);
      atomicOr(touched + (w >> 5), 1u << (w & 31));
    }
    __syncthreads();
    if (a.K > 0) {
      for (int k = threadIdx.x; k < a.K; k += kThreads) {
        const int v = ids[k];
        if (v >= v0 && v < v1 && link[v - origin] != k) repeated = 1;
      }
      __syncthreads();
    }
  }
  T* to = static_cast<T*>(a.out) + row;
#pragma unroll
  for (int k = 0; k < kVectors; ++k) {
    const int w = (k * kThreads + (int)threadIdx.x) * E, v = origin + w;
    if (v >= v1) break;
    const uint32_t look = marks ? touched[w >> 5] >> (w & 31) & ((1u << E) - 1) : 0;
    if (look) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        if (!(look >> i & 1)) continue;
        float x = widen<T>(in[k].x[i]);
        const uint32_t c = a.L > 0 ? count[w + i] : 0;
        if (c) {
          x = x > 0 ? __fdiv_rn(x, rep) : __fmul_rn(x, rep);
          const uint32_t times = c & 0x7FFFFFFFu;
          if (times) x = __fsub_rn(__fsub_rn(x, __fmul_rn(freq, (float)times)), pres);
        }
        const int first = a.K > 0 ? link[w + i] : 0x7FFFFFFF;
        if (first != 0x7FFFFFFF) {
          const int* ids = a.ids + (size_t)b * a.K;
          const float* bias = a.bias + (size_t)b * a.K;
          float sum = bias[first];
          if (repeated)
            for (int j = first + 1; j < a.K; ++j)
              if (ids[j] == v + i) sum = __fadd_rn(sum, bias[j]);
          x = __fadd_rn(x, sum);
        }
        in[k].x[i] = narrow<T>(x);
      }
    }
    if (a.M > 0) {
      const uint32_t* mask = a.mask + (size_t)b * a.M;
      const int at = max(v, 0), word = at >> 5;                  // (a vector that starts before its row: the bits from column 0 on)
      uint32_t bits = mask[word] >> (at & 31);
      if ((at & 31) + E > 32 && word + 1 < a.M) bits |= mask[word + 1] << (32 - (at & 31));
      bits <<= at - v;
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (!(bits >> i & 1)) in[k].x[i] = narrow<T>(-INFINITY);
    }
    if (v >= v0 && v + E <= v1) *reinterpret_cast<uint4*>(to + v) = in[k].raw;
    else
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (v + i >= v0 && v + i < v1) to[v + i] = in[k].x[i];
  }
}

template <class T>
int launch(const ClusterLaunch& L) {
  constexpr int E = 16 / sizeof(T), kCols = kThreads * kVectors * E;
  const int B = (int)L.op.shape[0], V = (int)L.op.shape[1];
  if (B == 0 || V == 0) return ACC_OK;
  PenaltyArgs a{report_of(L), slot(L, 0).ptr, slot_ptr<int>(L, 1), slot_ptr<float>(L, 2), slot_ptr<int>(L, 3), slot_ptr<float>(L, 4),
                slot_ptr<uint32_t>(L, 5), result_ptr<void>(L),
                V, slot(L, 1).C, slot(L, 3).C, slot(L, 5).C, V % E == 0 ? kCols : kCols - E, 0};
  a.blocks = (V + a.cols - 1) / a.cols;
  const size_t shared = (size_t)((a.L > 0) + (a.K > 0)) * kCols * 4;
  static std::atomic<uint64_t> allowed{0};
  const int rc = allow_shared(k_penalize<T>, 2 * kCols * 4, allowed);
  if (rc != ACC_OK) return rc;
  k_penalize<T><<<(unsigned)B * (unsigned)a.blocks, kThreads, shared, L.stream>>>(a);
  return launched();
}

int launch_penalize(const ClusterLaunch& L) {
  return L.op.dtype == ACC_F32 ? launch<float>(L) : L.op.dtype == ACC_F16 ? launch<__half>(L) : launch<__nv_bfloat16>(L);
}

const Register penalize(ACC_PENALIZE, "k_penalize", no_scratch, launch_penalize);

}  // namespace
}  // namespace ops
}  // namespace acc
