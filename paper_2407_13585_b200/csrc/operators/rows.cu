// Rows put into an array at given slots (ACC_PUT_ROWS): the paper's scatter (Section 2, "destructive update") with whole
// rows in place of elements and the last row in place of a combine operator.
#include <algorithm>

#include "operators/common.cuh"

namespace acc {
namespace ops {
namespace {

struct RowArgs {
  Report report;
  const int* slots;
  const void* rows[2];  // of one array, or of two of one shape (the grid's second dimension)
  void* out[2];
  int* owner;          // the last row of every slot that a row is put into; null: the rows look for a later one themselves
  int T, S, units;     // units of the vector type per row
  int pieces;          // warps per row
};

template <int BYTES> struct Unit;
template <> struct Unit<16> { using type = uint4; };
template <> struct Unit<4> { using type = uint32_t; };
template <> struct Unit<2> { using type = uint16_t; };

constexpr int kUnitsPerLane = 8;

// A warp moves 32 x 8 units of a row (4 KB of 16-byte units; 12000 rows of 4 KB, twice: 38 us, with 4 units to a lane 42).
// Bound: memory, rows read in order and written at random places.  Rows for one slot: the last one stays, whatever the order
// the warps run in, because every warp looks for a later row of its slot before it stores (its row is on the way
// meanwhile), or finds the slot's last row in `owner`.
template <int BYTES>
__global__ void __launch_bounds__(128) k_put_rows(RowArgs a) {
  using U = typename Unit<BYTES>::type;
  // behind the kernel that settles owners it is waited for only once the row is on its way: that kernel did not begin
  // before all that slots and rows come from had finished
  if (a.owner) cudaTriggerProgrammaticLaunchCompletion();
  else follow();
  const int lane = threadIdx.x & 31;
  const long long w = (long long)blockIdx.x * (blockDim.x / 32) + (threadIdx.x >> 5);
  const int t = (int)(w / a.pieces), piece = (int)(w % a.pieces);
  const int at = t < a.T ? a.slots[t] : -1;
  if (at >= a.S && lane == 0) raise_index(a.report);
  if (at < 0 || at >= a.S) {
    if (a.owner) cudaGridDependencySynchronize();
    return;
  }
  const int first = piece * 32 * kUnitsPerLane + lane;
  const U* from = static_cast<const U*>(a.rows[blockIdx.y]) + (size_t)t * a.units;
  U v[kUnitsPerLane];
#pragma unroll
  for (int k = 0; k < kUnitsPerLane; ++k)
    if (first + 32 * k < a.units) v[k] = from[first + 32 * k];
  bool later = false;
  if (a.owner) {
    cudaGridDependencySynchronize();
    later = a.owner[at] != t;
  } else {
#pragma unroll 4
    for (int i = t + 1 + lane; i < a.T; i += 32) later = later || a.slots[i] == at;
    later = __any_sync(~0u, later);
  }
  if (later) return;
  U* to = static_cast<U*>(a.out[blockIdx.y]) + (size_t)at * a.units;
#pragma unroll
  for (int k = 0; k < kUnitsPerLane; ++k)
    if (first + 32 * k < a.units) to[first + 32 * k] = v[k];
}

// owner[s] = the last row for slot s, without clearing the array first: a number that is no row for this slot is nobody's,
// and one that is a row for it is an owner like any other, wherever it comes from.
__global__ void __launch_bounds__(256) k_settle_owners(const int* slots, int* owner, int T, int S) {
  cudaTriggerProgrammaticLaunchCompletion();
  const int t = blockIdx.x * 256 + threadIdx.x;
  const int slot = t < T ? slots[t] : -1;
  if (slot < 0 || slot >= S) return;
  int old = *reinterpret_cast<volatile int*>(owner + slot);
  while (!((uint32_t)old < (uint32_t)T && old >= t && slots[old] == slot)) {
    const int seen = atomicCAS(owner + slot, old, t);
    if (seen == old) break;
    old = seen;
  }
}

__global__ void __launch_bounds__(256) k_copy_array(const uint4* from, uint4* to, size_t vectors, size_t bytes) {
  follow();
  const size_t stride = (size_t)gridDim.x * 256;
#pragma unroll 4
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < vectors; i += stride) to[i] = from[i];
  if (blockIdx.x == 0)
    for (size_t i = vectors * 16 + 2 * threadIdx.x; i < bytes; i += 512)
      *reinterpret_cast<uint16_t*>(reinterpret_cast<char*>(to) + i) = *reinterpret_cast<const uint16_t*>(reinterpret_cast<const char*>(from) + i);
}

// Up to this many rows every row looks at the slots behind it (4 T^2 / 2 bytes, from L1 and L2), one launch; beyond, the
// slots' owners are settled first, two launches (rows of 2 KB, twice: 200 10.2 us looked, 12.3 settled; 500 14.3 and 12.3;
// 8000 47 and 19).
constexpr int kRowsThatLook = 256;

int64_t put_rows_scratch(const ClusterLaunch& L) { return slot(L, 1).C > kRowsThatLook ? 4 * L.op.shape[0] : 0; }

int launch_put_rows(const ClusterLaunch& L) {
  const size_t e = element_bytes(L.op.dtype);
  const size_t row_bytes = (size_t)L.op.shape[1] * e, bytes = row_bytes * L.op.shape[0];
  if (bytes == 0) return no_launch(L), report_beyond(L, slot_ptr<int>(L, 1), slot(L, 1).C, (int)L.op.shape[0]);
  int launches = 0, rc = ACC_OK;
  const ClusterLaunch* both[2] = {&L, L.also};
  for (int k = 0; k < (L.also ? 2 : 1) && rc == ACC_OK; ++k) {
    const void* dest = slot(*both[k], 0).ptr;
    void* out = result_ptr<void>(*both[k]);
    if (dest == out) continue;
    const size_t vectors = bytes / 16;
    const int grid = (int)std::min<size_t>(std::max<size_t>((vectors + 1023) / 1024, 1), (size_t)sm_count() * 8);
    rc = launch_following(k_copy_array, dim3(grid), 256, 0, L.stream, static_cast<const uint4*>(dest), static_cast<uint4*>(out), vectors, bytes);
    ++launches;
  }
  RowArgs a{report_of(L), slot_ptr<int>(L, 1), {slot(L, 2).ptr, L.also ? slot(*L.also, 2).ptr : nullptr},
            {result_ptr<void>(L), L.also ? result_ptr<void>(*L.also) : nullptr}, nullptr, (int)slot(L, 1).C, (int)L.op.shape[0], 0, 1};
  if (a.T > 0 && rc == ACC_OK) {
    if (a.T > kRowsThatLook) {
      a.owner = reinterpret_cast<int*>(L.scratch);
      // launched plainly, and it has to be: it begins when everything before it has finished, so that k_put_rows, which may start
      // as soon as this one has, finds slots and rows complete without waiting
      k_settle_owners<<<(a.T + 255) / 256, 256, 0, L.stream>>>(a.slots, a.owner, a.T, a.S);
      rc = launched();
      ++launches;
    }
    const int unit = row_bytes % 16 == 0 ? 16 : row_bytes % 4 == 0 ? 4 : 2;
    a.units = (int)(row_bytes / unit);
    a.pieces = (a.units + 32 * kUnitsPerLane - 1) / (32 * kUnitsPerLane);
    const dim3 grid((unsigned)(((long long)a.T * a.pieces + 3) / 4), L.also ? 2 : 1);
    if (rc == ACC_OK) rc = launch_following(unit == 16 ? k_put_rows<16> : unit == 4 ? k_put_rows<4> : k_put_rows<2>, grid, 128, 0, L.stream, a);
    ++launches;
  }
  L.extra_launches = launches - 1;
  return rc;
}

const Register put_rows(ACC_PUT_ROWS, "k_put_rows", put_rows_scratch, launch_put_rows);

}  // namespace
}  // namespace ops
}  // namespace acc
