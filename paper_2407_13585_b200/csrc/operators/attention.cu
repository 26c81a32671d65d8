// Attention of one new token per request over its paged keys and values (ACC_PAGED_ATTENTION).
#include "operators/common.cuh"

namespace acc {
namespace ops {
namespace {

struct AttentionArgs {
  Report report;
  const void *q, *keys, *values;
  const int *table, *lens;
  void* out;
  int B, W, S, Hq, Hk, D, window;
  float scale;
  Divisor block;
};

// out = sum_t exp(s_t - m) v_t / sum_t exp(s_t - m), s_t = scale q.k_t, with the running maximum m.  A block per request and
// head; its four warps take every fourth token, lanes share the dimensions, and the warps' sums are joined at the end.
template <class T>
__global__ void __launch_bounds__(128) k_attention_simple(AttentionArgs a) {
  const int b = blockIdx.x, h = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = h / (a.Hq / a.Hk);
  float q[8], acc[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int d = lane + 32 * i;
    q[i] = d < a.D ? widen<T>(static_cast<const T*>(a.q)[((size_t)b * a.Hq + h) * a.D + d]) : 0.0f;
    acc[i] = 0;
  }
  const int length = a.lens[b];
  const long long room = (long long)a.W * a.block.d;
  const int n = (int)min((long long)max(length, 0), room);
  bool bad = length < 0 || length > room;
  float m = -INFINITY, l = 0;
  bool any = false;                                        // (no score but -infinity is not the same as no token)
  for (int t = (a.window > 0 ? max(n - a.window, 0) : 0) + warp; t < n; t += 4) {
    const int p = (int)((uint32_t)t / a.block);
    const int page = a.table[(size_t)b * a.W + p];
    const long long at = (long long)page * a.block.d + (t - p * (int)a.block.d);
    if (page < 0 || at >= a.S) {
      bad = true;
      continue;
    }
    any = true;
    const size_t base = ((size_t)at * a.Hk + g) * a.D;
    float s = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (lane + 32 * i < a.D) s = fmaf(q[i], widen<T>(static_cast<const T*>(a.keys)[base + lane + 32 * i]), s);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
    s *= a.scale;
    const float top = fmaxf(m, s);
    const float fall = top == -INFINITY ? 1.0f : expf(m - top), p_t = top == -INFINITY ? 0.0f : expf(s - top);
    l = l * fall + p_t;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (lane + 32 * i < a.D) acc[i] = fmaf(p_t, widen<T>(static_cast<const T*>(a.values)[base + lane + 32 * i]), acc[i] * fall);
    m = top;
  }
  if (bad && lane == 0) raise_index(a.report);
  __shared__ float ms[4], ls[4], sums[4][256];
#pragma unroll
  for (int i = 0; i < 8; ++i) sums[warp][lane + 32 * i] = acc[i];
  if (lane == 0) ms[warp] = m, ls[warp] = l;
  any = __syncthreads_or(any);
  const float top = fmaxf(fmaxf(ms[0], ms[1]), fmaxf(ms[2], ms[3]));
  float all = 0;
  for (int w = 0; w < 4; ++w) all += top == -INFINITY ? 0.0f : ls[w] * expf(ms[w] - top);
  for (int d = threadIdx.x; d < a.D; d += 128) {
    float x = 0;
    for (int w = 0; w < 4; ++w) x += top == -INFINITY ? 0.0f : sums[w][d] * expf(ms[w] - top);
    static_cast<T*>(a.out)[((size_t)b * a.Hq + h) * a.D + d] = narrow<T>(any ? x / all : 0.0f);
  }
}

int launch_attention(const ClusterLaunch& L) {
  const int D = (int)L.op.iparam[1];
  AttentionArgs a{report_of(L), slot(L, 0).ptr, slot(L, 1).ptr, slot(L, 2).ptr, slot_ptr<int>(L, 3), slot_ptr<int>(L, 4), result_ptr<void>(L),
                  (int)L.op.shape[0], slot(L, 3).C, slot(L, 1).R, (int)L.op.shape[1] / D, slot(L, 1).C / D, D,
                  (int)std::min<int64_t>(L.op.iparam[2], 0x7FFFFFFF), (float)L.op.fparam[0], divisor((uint32_t)L.op.iparam[0])};
  if (a.B == 0 || a.Hq == 0) return ACC_OK;
  const dim3 grid(a.B, a.Hq);
  if (L.op.dtype == ACC_F32) k_attention_simple<float><<<grid, 128, 0, L.stream>>>(a);
  else if (L.op.dtype == ACC_F16) k_attention_simple<__half><<<grid, 128, 0, L.stream>>>(a);
  else k_attention_simple<__nv_bfloat16><<<grid, 128, 0, L.stream>>>(a);
  return launched();
}

const Register attention(ACC_PAGED_ATTENTION, "k_attention", no_scratch, launch_attention);

}  // namespace
}  // namespace ops
}  // namespace acc
