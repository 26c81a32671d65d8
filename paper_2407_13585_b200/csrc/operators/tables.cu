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
  int R, W, N, tile;
  Divisor block, width;
};

// Sums that stay at 2^31 - 1 once they get there: more than any list is long.
__device__ __forceinline__ uint32_t add_up_to(uint32_t a, uint32_t b) { return min(a + b, 0x7FFFFFFFu); }

// Of v: the sum over the threads before this one, and over all; of w the sum over all.  (kThreads threads.)
struct Scan {
  uint32_t before, all, all_w;
};
__device__ __forceinline__ Scan block_scan(uint32_t v, uint32_t w, uint32_t (*warp_sums)[2]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t incl = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t below = __shfl_up_sync(~0u, incl, d);
    w = add_up_to(w, __shfl_xor_sync(~0u, w, d));
    if (lane >= d) incl = add_up_to(incl, below);
  }
  const uint32_t above = __shfl_up_sync(~0u, incl, 1);
  if (lane == 31) warp_sums[warp][0] = incl, warp_sums[warp][1] = w;
  __syncthreads();
  Scan r{lane == 0 ? 0 : above, 0, 0};
  uint32_t ahead = 0;
#pragma unroll
  for (int k = 0; k < kThreads / 32; ++k) {
    if (k == warp) ahead = r.all;
    r.all = add_up_to(r.all, warp_sums[k][0]);
    r.all_w = add_up_to(r.all_w, warp_sums[k][1]);
  }
  r.before = add_up_to(r.before, ahead);
  __syncthreads();
  return r;
}

// An entry of a row {kept, end, from}: its first `kept` entries are the old row's, entry j in kept <= j < end is
// free[from + j], the others are -1.
__device__ __noinline__ int table_entry(const TableArgs& a, int f, int j, int4 row) {
  return j < row.x ? (a.old ? a.old[f] : -1) : j < row.y ? a.free[row.z + j] : -1;
}

// table[r, j] = old[r, j] | free[base_r + j - had_r] | -1 with base_r the blocks that earlier requests took.  A block
// writes a run of a.tile elements of the table, whatever rows they belong to, and adds up for itself what the requests
// before its first one take: one launch and no waiting on other blocks.  Bound: latency for small tables, then the sums and
// searches ahead of a block's first entry: the lengths that are read over again (4 R bytes for a block, from L2) are the
// smaller part of the bytes as long as R < a.tile, but not of the instructions (1000 rows of 3750 entries: 11 us with the
// caches flushed, 59 % of the issue slots taken).  kTableRows rows at most: where they are shorter than four elements a block
// takes fewer elements.
constexpr int kTableTile = 4096, kTableRows = 1024;
__global__ void __launch_bounds__(kThreads) k_block_table(TableArgs a) {
  __shared__ uint32_t warp_sums[kThreads / 32][2];
  __shared__ int4 rows[kTableRows + 2];                       // kept, end, from (see table_entry)
  follow();
  const int f0 = blockIdx.x * a.tile, f1 = (int)min((long long)f0 + a.tile, (long long)a.R * a.W);
  // (rows of no entries: one block that only looks for what there is to report)
  const int r0 = (uint32_t)f0 / a.width, r1 = a.W == 0 ? a.R : (int)((uint32_t)(f1 - 1) / a.width) + 1;
  const auto length = [&](int row) { return row < r1 ? a.lens[row] : 0; };
  const auto old_length = [&](int row) { return row < r1 && a.old_lens ? a.old_lens[row] : 0; };
  int len = length(r0 + threadIdx.x), old_len = old_length(r0 + threadIdx.x);
  uint32_t earlier = 0;
#pragma unroll 4
  for (int r = threadIdx.x; r < r0; r += kThreads)
    earlier = add_up_to(earlier, max(blocks_of(a.lens[r], a.block) - (a.old_lens ? blocks_of(a.old_lens[r], a.block) : 0), 0));
  uint32_t base = 0;
  for (int r = r0; r < r1; r += kThreads) {
    const int row = r + threadIdx.x;
    if (r > r0) len = length(row), old_len = old_length(row);
    const int need = blocks_of(len, a.block), had = blocks_of(old_len, a.block), taken = max(need - had, 0);
    const Scan s = block_scan(taken, r == r0 ? earlier : 0, warp_sums);
    base = add_up_to(base, s.all_w);
    if (row < r1) {
      const uint32_t start = add_up_to(base, s.before);
      // the list may end inside the row, or before it; from + j < N for all j < end
      const int from = (int)min(start, (uint32_t)a.N) - had;
      if (a.W > 0) rows[row - r0] = make_int4(min(had, need), (int)min((long long)need, (long long)a.N - from), from, 0);
      if (len < 0 || old_len < 0 || need > a.W || add_up_to(start, taken) > (uint32_t)a.N) raise_index(a.report);
    }
    base = add_up_to(base, s.all);
  }
  __syncthreads();
  int f = f0 + 4 * threadIdx.x, r = (uint32_t)f / a.width, j = f - r * a.W;
#pragma unroll 4
  for (; f < f1; f += 4 * kThreads) {
    const int4 row = rows[min(r - r0, kTableRows + 1)];
    if (f + 4 <= f1 && j + 4 <= a.W) {                         // four of one row
      int4 v = make_int4(-1, -1, -1, -1);
      if (j < row.x && a.old) v = *reinterpret_cast<const int4*>(a.old + f);
      if (j + 4 > row.x) {
        if (j >= row.x) v.x = j < row.y ? a.free[row.z + j] : -1;
        if (j + 1 >= row.x) v.y = j + 1 < row.y ? a.free[row.z + j + 1] : -1;
        if (j + 2 >= row.x) v.z = j + 2 < row.y ? a.free[row.z + j + 2] : -1;
        v.w = j + 3 < row.y ? a.free[row.z + j + 3] : -1;
      }
      *reinterpret_cast<int4*>(a.out + f) = v;
    } else {
      for (int k = 0, at = j, of = r - r0; k < 4 && f + k < f1; ++k) {
        a.out[f + k] = table_entry(a, f + k, at, rows[of]);
        if (++at == a.W) { at = 0; ++of; }
      }
    }
    j += 4 * kThreads;
    if (j >= a.W) r = (uint32_t)(f + 4 * kThreads) / a.width, j = f + 4 * kThreads - r * a.W;
  }
}

int launch_block_table(const ClusterLaunch& L) {
  const dev::NodeArg& t = L.nodes[L.result];
  const long long count = (long long)L.op.shape[0] * L.op.shape[1];
  if (L.op.shape[0] == 0) return no_launch(L);
  const bool grow = L.op.n_inputs == 4;
  TableArgs a{report_of(L), slot_ptr<int>(L, 0), slot_ptr<int>(L, 1), grow ? slot_ptr<int>(L, 2) : nullptr, grow ? slot_ptr<int>(L, 3) : nullptr,
              result_ptr<int>(L), t.R, t.C, (int)slot(L, 1).C, 0, divisor((uint32_t)L.op.iparam[0]), divisor((uint32_t)std::max<int64_t>(L.op.shape[1], 1))};
  // six blocks to an SM, if that leaves each at least four elements a thread
  const long long even = (count + 6 * sm_count() - 1) / (6 * sm_count());
  a.tile = (int)std::min<long long>(kTableTile, (even + 4 * kThreads - 1) / (4 * kThreads) * (4 * kThreads));
  a.tile = (int)std::min<int64_t>(a.tile, kTableRows * (int64_t)a.W);
  return launch_following(k_block_table, dim3((unsigned)std::max<long long>((count + a.tile - 1) / std::max(a.tile, 1), 1)), kThreads, 0, L.stream, a);
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

// Slot of token t, which request `lo` (of those from `first` on) holds or none; -1, and bad, where there is none.
__device__ __forceinline__ int slot_of(const SlotArgs& a, const int* off, const int* lens, int first, int rows, int lo, int t, bool& bad) {
  if (lo >= rows || t < off[lo]) return -1;
  const long long p = (long long)lens[lo] - ((long long)off[lo + 1] - t);
  int page = -1;
  uint32_t q = 0;
  if (p >= 0) {
    q = (uint32_t)p / a.block;
    if (q < (uint32_t)a.W) page = a.table[(size_t)(first + lo) * a.W + q];
  }
  const long long at = (long long)page * a.block.d + (p - (long long)q * a.block.d);
  if (page < 0 || at > 0x7FFFFFFFll) {
    bad = true;
    return -1;
  }
  return (int)at;
}

// Slots of tokens t .. t+3, of which the first is held by request lo or a later one.
__device__ __forceinline__ int4 four_slots(const SlotArgs& a, const int* off, const int* lens, int first, int rows, int lo, int t, int t1, bool& bad) {
  if (lo < rows && t + 4 <= t1 && off[lo] <= t && t + 4 <= off[lo + 1] && a.block.d >= 4 && lens[lo] >= 0) {
    // all of one request, in one block or in two
    const uint32_t left = (uint32_t)off[lo + 1] - (uint32_t)t, p = (uint32_t)lens[lo] - left;
    const uint32_t q = p / a.block, inside = p - q * a.block.d, here = a.block.d - inside;         // tokens of the first block
    const bool two = here < 4;
    if ((uint32_t)lens[lo] >= left && q + two < (uint32_t)a.W) {
      const int* row = a.table + (size_t)(first + lo) * a.W + q;
      const int page = row[0], behind = two ? row[1] : page;
      const long long at = (long long)page * a.block.d + inside, next = two ? (long long)behind * a.block.d - here : at;
      if (page >= 0 && behind >= 0 && at + 4 <= 0x7FFFFFFFll && next + 4 <= 0x7FFFFFFFll)
        return make_int4((int)at, (1 < here ? (int)at : (int)next) + 1, (2 < here ? (int)at : (int)next) + 2, (3 < here ? (int)at : (int)next) + 3);
    }
  }
  int v[4] = {-1, -1, -1, -1};
#pragma unroll 1
  for (int k = 0; k < 4 && t + k < t1; ++k) {
    while (lo < rows && off[lo + 1] <= t + k) ++lo;
    const int x = slot_of(a, off, lens, first, rows, lo, t + k, bad);
    if (k == 0) v[0] = x;
    else if (k == 1) v[1] = x;
    else if (k == 2) v[2] = x;
    else v[3] = x;
  }
  return make_int4(v[0], v[1], v[2], v[3]);
}

// A block maps a run of tokens, a thread one, or a warp 512 in rows of four to a lane (for prompts mostly one request's:
// then it is looked for once).  The offsets and lengths of their requests are brought into shared memory, those of all
// requests where that is few, else those from the first to the last token's, which the first warps look for; every thread
// finds the request of its tokens there.  (Between two tokens may lie more empty requests than there is room for: then the
// offsets are searched where they are.)  Bound: latency, a chain of three to five dependent reads; for prompts writing
// the slots.
constexpr int kSlotRows = 1024;
template <int PER>
__global__ void __launch_bounds__(kThreads) k_slot_map(SlotArgs a) {
  constexpr int kTile = PER * kThreads;
  __shared__ int ends[kSlotRows + 1], length[kSlotRows];
  __shared__ int range[2];
  follow();
  const int t0 = blockIdx.x * kTile, t1 = (int)min((long long)t0 + kTile, (long long)a.T);
  const auto find_range = [&](const int* off, int rows) {              // requests of the tile's first and last token
    if (threadIdx.x < 64) {
      const int which = threadIdx.x >> 5;
      const int r = requests_before(off, 0, rows, which ? t1 - 1 : t0);
      if ((threadIdx.x & 31) == 0) range[which] = r;
    }
    __syncthreads();
  };
  int r0 = 0, n = a.R;
  if (a.R > kSlotRows) {
    find_range(a.off, a.R);
    r0 = range[0];
    n = min(range[1], a.R - 1) - r0 + 1;                               // (off decreases against the rule: n may be anything)
  }
  const bool staged = n >= 1 && n <= kSlotRows;
  if (staged) {
#pragma unroll
    for (int k = 0; k <= kSlotRows / kThreads; ++k)
      if (const int i = k * kThreads + threadIdx.x; i <= n) ends[i] = a.off[r0 + i];
#pragma unroll
    for (int k = 0; k < kSlotRows / kThreads; ++k)
      if (const int i = k * kThreads + threadIdx.x; i < n) length[i] = a.lens[r0 + i];
  }
  __syncthreads();
  const int* off = staged ? ends : a.off;                              // off[i + 1]: where the tokens of request i of these end
  const int* lens = staged ? length : a.lens;
  const int rows = staged ? n : a.R, first = staged ? r0 : 0;
  int low = 0, high = rows;
  if (PER > 1 && staged && a.R <= kSlotRows) {
    find_range(ends, rows);
    low = min(range[0], rows), high = max(min(range[1], rows), low);
  }
  bool bad = false;
  const auto holder = [&](int t, int from) {                           // (the request of the last token is found by elimination)
    int lo = from, hi = high;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (off[mid + 1] <= t) lo = mid + 1;
      else hi = mid;
    }
    return lo;
  };
  if constexpr (PER == 1) {
    const int t = t0 + threadIdx.x;
    if (t < t1) a.out[t] = slot_of(a, off, lens, first, rows, holder(t, low), t, bad);
  } else {
    const int from = t0 + (threadIdx.x & ~31) * PER;                   // the warp's first token
    if (from >= t1) return;
    const int request = holder(from, low);
    const bool one = request < rows && off[request] <= from && min((long long)from + 32 * PER, (long long)t1) <= off[request + 1];
#pragma unroll 1
    for (int g = 0; g < PER / 4; ++g) {
      const int t = from + (g * 32 + (threadIdx.x & 31)) * 4;
      if (t >= t1) break;
      const int4 v = four_slots(a, off, lens, first, rows, one ? request : holder(t, request), t, t1, bad);
      if (t + 4 <= t1) *reinterpret_cast<int4*>(a.out + t) = v;
      else {
        a.out[t] = v.x;
        if (t + 1 < t1) a.out[t + 1] = v.y;
        if (t + 2 < t1) a.out[t + 2] = v.z;
      }
    }
  }
  if (bad) raise_index(a.report);
}

// Tokens up to which every thread takes one: a step's tokens are of a request each, so that four side by side would read
// the table one after the other.
constexpr int kSingleTokens = 1 << 16;
int launch_slot_map(const ClusterLaunch& L) {
  const dev::NodeArg& table = slot(L, 0);
  SlotArgs a{report_of(L), slot_ptr<int>(L, 0), slot_ptr<int>(L, 1), slot_ptr<int>(L, 2), result_ptr<int>(L),
             table.R, table.C, (int)L.op.shape[0], divisor((uint32_t)L.op.iparam[0])};
  if (a.T == 0) return no_launch(L);
  const bool single = a.T <= kSingleTokens;
  const int tile = single ? kThreads : 16 * kThreads;
  return launch_following(single ? k_slot_map<1> : k_slot_map<16>, dim3((unsigned)(((long long)a.T + tile - 1) / tile)), kThreads, 0, L.stream, a);
}

const Register block_table(ACC_BLOCK_TABLE, "k_block_table", no_scratch, launch_block_table);
const Register slot_map(ACC_SLOT_MAP, "k_slot_map", no_scratch, launch_slot_map);

}  // namespace
}  // namespace ops
}  // namespace acc
