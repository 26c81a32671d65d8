// Block tables and slot maps from request lengths (ACC_BLOCK_TABLE, ACC_SLOT_MAP).
#include "operators/common.cuh"

namespace acc {
namespace ops {
namespace {

constexpr int kThreads = 256;

struct TableArgs {
  Report report;
  const int *lens, *free, *old_lens, *old;   // old_lens, old: null if every block comes from `free`
  int* out;
  int R, W, N;
  Divisor block, width;
};

__device__ __forceinline__ int blocks_taken(const TableArgs& a, int r) {
  return max(blocks_of(a.lens[r], a.block) - (a.old_lens ? blocks_of(a.old_lens[r], a.block) : 0), 0);
}

// Sum over the block, and over the threads before this one (kThreads threads; `warp_sums` of kThreads / 32 words).
__device__ __forceinline__ long long block_scan(long long v, long long* warp_sums, long long* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long incl = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long below = __shfl_up_sync(~0u, incl, d);
    if (lane >= d) incl += below;
  }
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  long long before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) before += warp_sums[w];
    all += warp_sums[w];
  }
  __syncthreads();
  *total = all;
  return before + incl - v;
}

// table[r, j] = old[r, j] | free[base_r + j - had_r] | -1 with base_r the blocks that earlier requests took.  A block
// writes a run of kTableTile elements of the table, whatever rows they belong to, and adds up for itself what the
// requests before its first one take: one launch and no waiting on other blocks.  Bound: writing the table.  The lengths
// that are read over again (4 R bytes for a block, from L2) are the smaller part as long as R < kTableTile.
constexpr int kTableTile = 2048;
__global__ void __launch_bounds__(kThreads) k_block_table(TableArgs a) {
  __shared__ long long warp_sums[kThreads / 32];
  __shared__ int first_free[kTableTile + 2], had[kTableTile + 2], has[kTableTile + 2];
  const int f0 = blockIdx.x * kTableTile, f1 = min(f0 + kTableTile, (int)((long long)a.R * a.W));
  const int r0 = (uint32_t)f0 / a.width, r1 = (uint32_t)(f1 - 1) / a.width + 1;
  long long base = 0;
  {
    long long mine = 0;
#pragma unroll 4
    for (int r = threadIdx.x; r < r0; r += kThreads) mine += blocks_taken(a, r);
    block_scan(mine, warp_sums, &base);
  }
  for (int r = r0; r < r1; r += kThreads) {
    const int row = r + threadIdx.x;
    const int len = row < r1 ? a.lens[row] : 0, old_len = row < r1 && a.old_lens ? a.old_lens[row] : 0;
    const int need = blocks_of(len, a.block), kept = blocks_of(old_len, a.block);
    long long total;
    const long long start = base + block_scan(max(need - kept, 0), warp_sums, &total);
    if (row < r1) {
      first_free[row - r0] = (int)min(start, (long long)a.N);
      had[row - r0] = kept;
      has[row - r0] = need;
      if (len < 0 || old_len < 0 || need > a.W || start + max(need - kept, 0) > a.N) raise_index(a.report);
    }
    base += total;
  }
  __syncthreads();
  const auto entry = [&](int f, int r, int j) {
    const int need = has[r - r0], kept = had[r - r0];
    if (j >= need) return -1;
    if (j < kept) return a.old ? a.old[f] : -1;
    const long long at = (long long)first_free[r - r0] + (j - kept);
    return at < a.N ? a.free[at] : -1;
  };
  for (int f = f0 + 4 * threadIdx.x; f < f1; f += 4 * kThreads) {
    int r = (uint32_t)f / a.width, j = f - r * a.W;
    int v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[k] = f + k < f1 ? entry(f + k, r, j) : 0;
      if (++j == a.W) { j = 0; ++r; }
    }
    if (f + 4 <= f1) *reinterpret_cast<int4*>(a.out + f) = make_int4(v[0], v[1], v[2], v[3]);
    else for (int k = 0; f + k < f1; ++k) a.out[f + k] = v[k];
  }
}

int launch_block_table(const ClusterLaunch& L) {
  const dev::NodeArg& t = L.nodes[L.result];
  const long long count = (long long)L.op.shape[0] * L.op.shape[1];
  if (L.op.shape[0] == 0) return ACC_OK;
  const bool grow = L.op.n_inputs == 4;
  TableArgs a{report_of(L), slot_ptr<int>(L, 0), slot_ptr<int>(L, 1), grow ? slot_ptr<int>(L, 2) : nullptr, grow ? slot_ptr<int>(L, 3) : nullptr,
              result_ptr<int>(L), t.R, t.C, (int)slot(L, 1).C, divisor((uint32_t)L.op.iparam[0]), divisor((uint32_t)std::max<int64_t>(L.op.shape[1], 1))};
  if (count == 0) return ACC_OK;
  k_block_table<<<(unsigned)((count + kTableTile - 1) / kTableTile), kThreads, 0, L.stream>>>(a);
  return launched();
}

struct SlotArgs {
  Report report;
  const int *table, *lens, *off;
  int* out;
  int R, W, T;
  Divisor block;
};

// The number of requests whose tokens all lie before t (off does not decrease): 32 probes at a time, by a whole warp.
__device__ __forceinline__ int requests_before(const int* off, int lo, int hi, int t) {
  const int lane = threadIdx.x & 31;
  while (lo < hi) {
    const int step = (hi - lo + 31) / 32;
    const long long at = (long long)lo + (long long)(lane + 1) * step - 1;
    const int passed = __popc(__ballot_sync(~0u, at < hi && off[at + 1] <= t));
    const int next = (int)min((long long)lo + (long long)passed * step, (long long)hi);
    hi = (int)min((long long)hi, (long long)next + step - 1);
    lo = next;
  }
  return lo;
}

// A block maps a run of kSlotTile tokens.  Its first warp finds the requests of the first and the last of them; when those
// are few (they are, unless many are empty), their offsets and lengths are brought into shared memory, and every thread
// finds the request of its tokens there.  Bound: latency, a chain of five dependent reads; then writing the slots.
constexpr int kSlotTile = 4 * kThreads, kSlotRows = 1024;
__global__ void __launch_bounds__(kThreads) k_slot_map(SlotArgs a) {
  __shared__ int ends[kSlotRows + 1], length[kSlotRows];
  __shared__ int range[2];
  const int t0 = blockIdx.x * kSlotTile, t1 = min(t0 + kSlotTile, a.T);
  if (threadIdx.x < 64) {
    const int which = threadIdx.x >> 5;
    const int r = requests_before(a.off, 0, a.R, which ? t1 - 1 : t0);
    if ((threadIdx.x & 31) == 0) range[which] = r;
  }
  __syncthreads();
  const int r0 = range[0], n = min(range[1], a.R - 1) - r0 + 1;        // (off decreases against the rule: n may be anything)
  const bool staged = n >= 1 && n <= kSlotRows;
  if (staged) {
    for (int i = threadIdx.x; i <= n; i += kThreads) ends[i] = a.off[r0 + i];
    for (int i = threadIdx.x; i < n; i += kThreads) length[i] = a.lens[r0 + i];
  }
  __syncthreads();
  const int* off = staged ? ends : a.off;                              // off[i + 1]: where the tokens of request i of these end
  const int* lens = staged ? length : a.lens;
  const int rows = staged ? n : a.R, first = staged ? r0 : 0;
  const int t = t0 + 4 * threadIdx.x;
  if (t >= t1) return;
  int lo = 0, hi = rows;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (off[mid + 1] <= t) lo = mid + 1;
    else hi = mid;
  }
  int v[4];
  bool bad = false;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v[k] = -1;
    while (lo < rows && off[lo + 1] <= t + k) ++lo;
    if (t + k >= t1 || lo >= rows || t + k < off[lo]) continue;
    const long long p = (long long)lens[lo] - ((long long)off[lo + 1] - (t + k));
    int page = -1;
    uint32_t q = 0;
    if (p >= 0) {
      q = (uint32_t)p / a.block;
      if (q < (uint32_t)a.W) page = a.table[(size_t)(first + lo) * a.W + q];
    }
    const long long at = (long long)page * a.block.d + (p - (long long)q * a.block.d);
    if (page < 0 || at > 0x7FFFFFFFll) bad = true;
    else v[k] = (int)at;
  }
  if (bad) raise_index(a.report);
  if (t + 4 <= t1) *reinterpret_cast<int4*>(a.out + t) = make_int4(v[0], v[1], v[2], v[3]);
  else for (int k = 0; t + k < t1; ++k) a.out[t + k] = v[k];
}

int launch_slot_map(const ClusterLaunch& L) {
  const dev::NodeArg& table = slot(L, 0);
  SlotArgs a{report_of(L), slot_ptr<int>(L, 0), slot_ptr<int>(L, 1), slot_ptr<int>(L, 2), result_ptr<int>(L),
             table.R, table.C, (int)L.op.shape[0], divisor((uint32_t)L.op.iparam[0])};
  if (a.T == 0) return ACC_OK;
  k_slot_map<<<(unsigned)((a.T + kSlotTile - 1) / kSlotTile), kThreads, 0, L.stream>>>(a);
  return launched();
}

const Register block_table(ACC_BLOCK_TABLE, "k_block_table", no_scratch, launch_block_table);
const Register slot_map(ACC_SLOT_MAP, "k_slot_map", no_scratch, launch_slot_map);

}  // namespace
}  // namespace ops
}  // namespace acc
