// What the operators (foreign functions, Section 3.4) share: how a launch finds its slots, element types, status words.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>

#include "acc.h"
#include "device/eval.cuh"
#include "division.h"
#include "graph.h"
#include "registry.h"

namespace acc {
namespace ops {

// Where a kernel reports to (see raise_status in device/eval.cuh); the first member of every operator's parameters.
struct Report {
  uint32_t* status;
  uint32_t run_id;
};
inline Report report_of(const ClusterLaunch& L) { return {L.status, L.run_id}; }
__device__ __forceinline__ void raise_index(const Report& r) { *reinterpret_cast<volatile uint32_t*>(r.status + dev::kStatusIndex) = r.run_id; }

inline const dev::NodeArg& slot(const ClusterLaunch& L, int s) { return L.nodes[L.slot[s]]; }
template <class T>
const T* slot_ptr(const ClusterLaunch& L, int s) { return static_cast<const T*>(slot(L, s).ptr); }
template <class T>
T* result_ptr(const ClusterLaunch& L) { return static_cast<T*>(const_cast<void*>(L.nodes[L.result].ptr)); }

__device__ __forceinline__ uint32_t operator/(uint32_t v, const Divisor& p) {
  const uint32_t t = __umulhi(v, p.mul);
  return (t + ((v - t) >> p.sh1)) >> p.sh2;
}

// The blocks that `length` tokens take up.
__device__ __forceinline__ int blocks_of(int length, const Divisor& block) { return length <= 0 ? 0 : (int)((uint32_t)(length - 1) / block) + 1; }

// Launches a kernel so that it may be set up while the one before it in the stream still runs.  Most begin with follow():
// nothing is read or written before everything that was launched earlier has finished and its results are visible.  (A
// kernel that begins so may follow another one: each of them ends only after it has waited.)  Two read inputs before they
// wait, each behind a kernel of its own operator that cannot have begun before all inputs were complete: k_put_rows behind
// k_settle_owners, which is launched plainly, and k_penalize_marked (which also writes its scratch) behind k_penalize, which
// has waited before it lets the next one start.
template <class... P, class... A>
int launch_following(void (*kernel)(P...), dim3 grid, int threads, size_t shared, cudaStream_t stream, const A&... args) {
  cudaLaunchConfig_t config{};
  config.gridDim = grid;
  config.blockDim = dim3(threads);
  config.dynamicSmemBytes = shared;
  config.stream = stream;
  cudaLaunchAttribute early{};
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  config.attrs = &early;
  config.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&config, kernel, args...);
  return e == cudaSuccess ? ACC_OK : set_error(ACC_ERR_CUDA, "kernel launch failed: %s", cudaGetErrorString((cudaGetLastError(), e)));
}
__device__ __forceinline__ void follow() {
  cudaTriggerProgrammaticLaunchCompletion();
  cudaGridDependencySynchronize();
}

inline int launched() {
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? ACC_OK : set_error(ACC_ERR_CUDA, "kernel launch failed: %s", cudaGetErrorString(e));
}

// Lets a kernel have `bytes` of dynamic shared memory on the current device (asked for once per device and kernel).
template <class K>
int allow_shared(K kernel, size_t bytes, std::atomic<uint64_t>& devices) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return set_error(ACC_ERR_CUDA, "no current device: %s", cudaGetErrorString(cudaGetLastError()));
  const uint64_t bit = 1ull << (dev & 63);
  if (dev < 64 && (devices.load(std::memory_order_relaxed) & bit)) return ACC_OK;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e != cudaSuccess) return set_error(ACC_ERR_CUDA, "%zu bytes of shared memory: %s", bytes, cudaGetErrorString(cudaGetLastError()));
  devices.fetch_or(bit, std::memory_order_relaxed);
  return ACC_OK;
}

// An operator's entry counts one launch: for a run without any.
inline int no_launch(const ClusterLaunch& L) {
  L.extra_launches = -1;
  return ACC_OK;
}

// Reports the numbers x[0 .. n) from `bound` on, for operators whose result has no elements: one launch, if n > 0, counted
// in extra_launches.
int report_beyond(const ClusterLaunch& L, const int* x, int64_t n, int bound);

inline int64_t no_scratch(const ClusterLaunch&) { return 0; }

struct Register {
  Register(int kind, const char* name, int64_t (*scratch)(const ClusterLaunch&), int (*launch)(const ClusterLaunch&)) {
    register_kernel(KernelEntry{operator_signature(kind), name, scratch, no_scratch, launch, 1});
  }
};

template <class T> __device__ __forceinline__ float widen(T x);
template <> __device__ __forceinline__ float widen<float>(float x) { return x; }
template <> __device__ __forceinline__ float widen<__half>(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float widen<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
// One rounding, to nearest even; beyond the type's range an infinity.
template <class T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ float narrow<float>(float x) { return x; }
template <> __device__ __forceinline__ __half narrow<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

}  // namespace ops
}  // namespace acc
