// Attention of one new token per request over its paged keys and values (ACC_PAGED_ATTENTION).
//
//   out[b, h] = sum_t w_t v_t / sum_t w_t,   w_t = 2^(s_t - m),   s_t = log2(e) scale q[b, h].k_t,   m = max_t s_t
//
// in one pass over keys and values: with a running maximum m, sums and products so far are multiplied by 2^(m - m') when a
// larger m' turns up, and two runs over different tokens join the same way.  Reading keys and values is what bounds it (2 e D
// bytes per token and key head for 4 D (Hq / Hk) operations), so the query heads of a key head are worked on together: up to
// eight or sixteen in 16-bit types, two, four or eight in fp32.  Where a key head has more, they are several units, and each of
// them goes through the tokens again.
//
// Splitting.  The work is the list of all tiles (four warps x 16 or 8 tokens) of all requests and key heads, one unit
// (request, block of heads) after the other; every block of a grid that fills the GPU once takes an equal run of that
// list, whatever the lengths are.  It finds its place by adding up the lengths itself.  A unit that ends inside one block
// is finished there; of one that does not, every block leaves its sums in scratch and k_join adds them up in the order of
// the blocks: no atomics, the same bits every time.
//
// Inside a block every warp takes its 16 (8) tokens of a tile through a ring of stages of its own in shared memory, filled
// by 16-byte asynchronous copies across units, two tiles ahead, or one where there is room for two stages only (16-bit heads of
// 65 to 96 elements, fp32 heads of 65 to 128); the block numbers are read one tile further ahead.
#include <cfloat>

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
  int group, units;       // query heads of a key head, units of a request
  float scale_log2;       // log2(e) scale
  Divisor block;
  float* parts;           // two records of sums per block of the grid; null: no unit is split
  int grid, join_rows;    // blocks of the grid; heads that a block of the joining kernel takes
  // {request, unit, first block, last block} of split units, -1 for none: by unit (request * units + unit) where there are no
  // more units than blocks, else by the block that a unit starts in
  int4* joins;
  bool by_unit;
};

// 2^x to 2^-22; results below 2^-126, which no sum would notice, are zeros.
__device__ __forceinline__ float power2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

constexpr int kWarps = 4, kThreads = kWarps * 32;

// The tokens [first, end) that request b attends to.
struct Span {
  int first, end;
};
__device__ __forceinline__ Span span_of(const AttentionArgs& a, int b) {
  const int length = a.lens[b];
  const int end = (int)min((long long)max(length, 0), (long long)a.W * a.block.d);
  return {a.window > 0 ? max(end - a.window, 0) : 0, end};
}
template <int TILE>
__device__ __forceinline__ int tiles_of(Span s) { return (int)(((uint32_t)(s.end - s.first) + TILE - 1) / TILE); }

// A place in the list of tiles.
template <int TILE>
struct Cursor {
  int b, unit, tile, tiles;
  Span span;
  long long left;          // tiles of this block's run, this one included

  __device__ __forceinline__ void enter(const AttentionArgs& a) {
    span = span_of(a, b);
    tiles = tiles_of<TILE>(span);
  }
  __device__ __forceinline__ void advance(const AttentionArgs& a) {
    if (--left <= 0) return;
    if (++tile < tiles) return;
    tile = 0;
    if (++unit < a.units) return;
    unit = 0;
    do {                                       // (left > 0: there is a request with tokens behind)
      ++b;
      enter(a);
    } while (tiles == 0 && b + 1 < a.B);
  }
};

struct Place {
  long long total;           // tiles of all requests
  int blocks;                // blocks that have any: each has at least one
  int b;                     // the request that the run starts in
  long long b_start;         // tiles before that request
};
__device__ __forceinline__ long long run_start(int block, long long total, int blocks) {
  if (total < 1 << 20) return (uint32_t)block * (uint32_t)total / (uint32_t)blocks;     // (at most 2^10 blocks)
  return (long long)block * total / blocks;
}

// What the joining kernel needs of the unit whose start this block has and whose end it has not.
template <int TILE>
__device__ __forceinline__ int4 join_of(const AttentionArgs& a, const Cursor<TILE>& c, const Place& place) {
  const long long unit_end = run_start(blockIdx.x + 1, place.total, place.blocks) - 1 - c.tile + c.tiles;     // in tiles of the list
  return make_int4(c.b, c.unit, blockIdx.x, (int)((unit_end * place.blocks - 1) / place.total));
}

// Where this block's run of the list starts.  Every thread adds up a share of the requests; requests without tokens get
// their zeros here, spread over the grid.
template <class T, int TILE>
__device__ Cursor<TILE> find_place(const AttentionArgs& a, Place* shared, long long* sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int share = (a.B + kThreads - 1) / kThreads;
  const int r0 = min((int)threadIdx.x * share, a.B), r1 = min(r0 + share, a.B);
  long long mine = 0;
  bool bad = false;
  for (int r = r0; r < r1; ++r) {
    const int length = a.lens[r];
    bad = bad || length < 0 || length > (long long)a.W * a.block.d;
    mine += tiles_of<TILE>(span_of(a, r));
  }
  if (bad) raise_index(a.report);
  mine *= a.units;
  long long upto = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long below = __shfl_up_sync(~0u, upto, d);
    if (lane >= d) upto += below;
  }
  if (lane == 31) sums[warp] = upto;
  __syncthreads();
  long long total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) upto += sums[w];
    total += sums[w];
  }
  const int blocks = (int)min((long long)gridDim.x, total);
  const bool any = (int)blockIdx.x < blocks;
  const long long start = any ? run_start(blockIdx.x, total, blocks) : 0, end = any ? run_start(blockIdx.x + 1, total, blocks) : 0;
  if (any && upto - mine <= start && start < upto) {
    long long at = upto - mine;
    int r = r0;
    for (; r + 1 < r1; ++r) {
      const long long n = (long long)tiles_of<TILE>(span_of(a, r)) * a.units;
      if (at + n > start) break;
      at += n;
    }
    *shared = {total, blocks, r, at};
  }
  for (int r = blockIdx.x; r < a.B; r += gridDim.x) {
    const Span s = span_of(a, r);
    if (s.first < s.end) continue;
    for (int d = threadIdx.x; d < a.Hq * a.D; d += kThreads) static_cast<T*>(a.out)[(size_t)r * a.Hq * a.D + d] = narrow<T>(0.0f);
    if (a.parts && a.by_unit)
      for (int u = threadIdx.x; u < a.units; u += kThreads) a.joins[(size_t)r * a.units + u] = make_int4(-1, 0, 0, 0);
  }
  __syncthreads();
  Cursor<TILE> c{};
  if (!any) return c;
  c.b = shared->b;
  c.enter(a);
  const long long inside = start - shared->b_start;
  c.unit = inside <= 0x7FFFFFFF ? (int)((uint32_t)inside / (uint32_t)c.tiles) : (int)(inside / c.tiles);
  c.tile = (int)(inside - (long long)c.unit * c.tiles);
  c.left = end - start;
  return c;
}

// Where the sums of block `block` go that does not finish a unit: record 1 if it started the unit, record 0 if it goes on
// with it.  A record is one row of sums for every head of the unit (WAYS x ROWS x DP), its maxima and weights apart.
template <int DP, int HEADS>
struct Records {
  float *sums, *tops, *weights;
  __host__ __device__ static constexpr size_t bytes(int blocks) { return (size_t)blocks * 2 * HEADS * (DP + 2) * 4; }
  __device__ __forceinline__ Records(const AttentionArgs& a)
      : sums(a.parts), tops(a.parts + (size_t)a.grid * 2 * HEADS * DP), weights(tops + (size_t)a.grid * 2 * HEADS) {}
  __device__ __forceinline__ static size_t row(int block, bool started, int head) { return ((size_t)block * 2 + (started ? 1 : 0)) * HEADS + head; }
};

// In the shared sums of a warp, dimension d of row r lies at d ^ spread(r): the eight dimensions that a matrix
// instruction's result has in a column go to banks of their own for each of the four columns written together.
__device__ __forceinline__ int spread(int row) { return (row >> 1 & 3) << 3; }

// The four warps' sums over the tokens of one unit, sums[warp * stride + row * DP + ...], their maxima and weights in
// ml[0][warp][row], ml[1][warp][row].  Written out if they are the whole unit, else to scratch.  A row without any token
// has the maximum -infinity; with tokens it is at least -FLT_MAX.
template <class T, int DP, int ROWS, bool SPREAD>
__device__ __forceinline__ void finish_unit(const AttentionArgs& a, int b, int kv, int head0, bool from_start, bool to_end, const float* sums, int stride,
                                            const float* ml) {
  const int rows = min(ROWS, a.group - head0);
  const bool whole = from_start && to_end;
  for (int i = threadIdx.x; i < rows * (DP / 4); i += kThreads) {
    const int row = i / (DP / 4), d = i % (DP / 4) * 4;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) top = fmaxf(top, ml[w * ROWS + row]);
    const float ref = top == -INFINITY ? 0.0f : top;
    float l = 0, x[4] = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float weight = power2(ml[w * ROWS + row] - ref);
      const float4 s = *reinterpret_cast<const float4*>(sums + (size_t)w * stride + row * DP + (SPREAD ? d ^ spread(row) : d));
      l = fmaf(ml[(kWarps + w) * ROWS + row], weight, l);
      x[0] = fmaf(s.x, weight, x[0]), x[1] = fmaf(s.y, weight, x[1]), x[2] = fmaf(s.z, weight, x[2]), x[3] = fmaf(s.w, weight, x[3]);
    }
    if (whole) {
      if (d >= a.D) continue;
      T* out = static_cast<T*>(a.out) + ((size_t)b * a.Hq + (size_t)kv * a.group + head0 + row) * a.D + d;
#pragma unroll
      for (int k = 0; k < 4; ++k) out[k] = narrow<T>(top == -INFINITY ? 0.0f : __fdiv_rn(x[k], l));
    } else {
      const Records<DP, ROWS> to(a);
      const size_t at = to.row(blockIdx.x, from_start, row);
      *reinterpret_cast<float4*>(to.sums + at * DP + d) = make_float4(x[0], x[1], x[2], x[3]);
      if (d == 0) {
        to.tops[at] = top;
        to.weights[at] = l;
      }
    }
  }
}

// Adds up the records of a split unit.  Few units (a.join_rows = 1), so many records each: a block to 32 dimensions of a
// head, whose records its warps share, a lane in eight four dimensions of one.  Else a block to eight heads, a warp to each,
// a lane to four dimensions, eight records on their way at a time: lengths differ, and so one unit may have many records
// where most have few (4 requests of up to 6000 tokens, all of a block's warps on one head after the other: 26 us, so 4).
constexpr int kJoinThreads = 256, kJoinWarps = kJoinThreads / 32, kMaxGrid = 1024, kPiece = 32;
template <class T, int DP, int ROWS, int WAYS>
__global__ void __launch_bounds__(kJoinThreads) k_join(AttentionArgs a) {
  constexpr int HEADS = ROWS * WAYS, VECS = (DP / 4 + 31) / 32;
  __shared__ float weight[kMaxGrid];
  __shared__ float tops[kJoinWarps], shares[kJoinWarps];
  __shared__ float4 sums[kJoinWarps][kPiece / 4];
  follow();
  const int4 join = a.joins[blockIdx.x];
  if (join.x < 0) return;
  const int per = a.units / (a.Hk / WAYS), head0 = join.y % per * ROWS;
  const int n = join.w - join.z + 1;
  const Records<DP, HEADS> from(a);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int r0 = blockIdx.y * a.join_rows;
  const auto at = [&](int i, int h) { return from.row(join.z + i, i == 0, h); };
  const auto add = [&](float4& y, float w, const float4& s) { y.x = fmaf(s.x, w, y.x), y.y = fmaf(s.y, w, y.y), y.z = fmaf(s.z, w, y.z), y.w = fmaf(s.w, w, y.w); };
  const auto write = [&](int h, int d, const float4& y, float l, float top) {
    if (d >= a.D) return;
    const int kv = join.y / per * WAYS + h / ROWS;
    T* out = static_cast<T*>(a.out) + ((size_t)join.x * a.Hq + (size_t)kv * a.group + head0 + h % ROWS) * a.D + d;
    const float z[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) out[k] = narrow<T>(top == -INFINITY ? 0.0f : __fdiv_rn(z[k], l));
  };
  constexpr int BATCH = 8;
  if (a.join_rows > 1) {
    for (int h = r0 + warp; h < r0 + a.join_rows; h += kJoinWarps) {
      if (h % ROWS >= a.group - head0) continue;
      float top = -INFINITY;
      for (int i = lane; i < n; i += 32) top = fmaxf(top, from.tops[at(i, h)]);
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
      const float ref = top == -INFINITY ? 0.0f : top;
      float4 y[VECS] = {};
      float l = 0;
#pragma unroll 1
      for (int i0 = 0; i0 < n; i0 += BATCH) {
        float4 x[BATCH][VECS];
        float w[BATCH], share[BATCH];
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
          const bool is = i0 + k < n;
          const size_t row = at(is ? i0 + k : 0, h);
          w[k] = is ? from.tops[row] : -INFINITY;
          share[k] = is ? from.weights[row] : 0.0f;
#pragma unroll
          for (int v = 0; v < VECS; ++v)
            x[k][v] = is && (lane + 32 * v) * 4 < DP ? *reinterpret_cast<const float4*>(from.sums + row * DP + (lane + 32 * v) * 4) : make_float4(0, 0, 0, 0);
        }
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
          const float wk = power2(w[k] - ref);
          l = fmaf(wk, share[k], l);
#pragma unroll
          for (int v = 0; v < VECS; ++v) add(y[v], wk, x[k][v]);
        }
      }
#pragma unroll
      for (int v = 0; v < VECS; ++v) write(h, (lane + 32 * v) * 4, y[v], l, top);
    }
    return;
  }
  constexpr int STEP = 4 * kJoinWarps;                     // four records to a warp at a time
  const int mine = warp * 4 + (lane >> 3);
  const int h = r0;
  if (h % ROWS >= a.group - head0) return;
  const int d = blockIdx.z * kPiece + (lane & 7) * 4;
  const auto load = [&](int i) { return i < n ? *reinterpret_cast<const float4*>(from.sums + at(i, h) * DP + d) : make_float4(0, 0, 0, 0); };
  float4 ahead[BATCH];                                 // on their way while the maxima are compared
#pragma unroll
  for (int k = 0; k < BATCH; ++k) ahead[k] = load(mine + k * STEP);
  float top = -INFINITY;
  for (int i = threadIdx.x; i < n; i += kJoinThreads) {
    weight[i] = from.tops[at(i, h)];
    top = fmaxf(top, weight[i]);
  }
#pragma unroll
  for (int k = 16; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, k));
  if (lane == 0) tops[warp] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kJoinWarps; ++w) top = fmaxf(top, tops[w]);
  const float ref = top == -INFINITY ? 0.0f : top;
  float l = 0;
  for (int i = threadIdx.x; i < n; i += kJoinThreads) {
    weight[i] = power2(weight[i] - ref);
    l = fmaf(weight[i], from.weights[at(i, h)], l);
  }
#pragma unroll
  for (int k = 16; k > 0; k >>= 1) l += __shfl_xor_sync(~0u, l, k);
  if (lane == 0) shares[warp] = l;
  __syncthreads();
  float4 y = make_float4(0, 0, 0, 0);
  for (int i0 = mine; i0 < n; i0 += BATCH * STEP) {
    if (i0 != mine)
#pragma unroll
      for (int k = 0; k < BATCH; ++k) ahead[k] = load(i0 + k * STEP);
#pragma unroll
    for (int k = 0; k < BATCH; ++k)
      if (i0 + k * STEP < n) add(y, weight[i0 + k * STEP], ahead[k]);
  }
#pragma unroll
  for (int k = 8; k < 32; k <<= 1) {
    y.x += __shfl_xor_sync(~0u, y.x, k), y.y += __shfl_xor_sync(~0u, y.y, k);
    y.z += __shfl_xor_sync(~0u, y.z, k), y.w += __shfl_xor_sync(~0u, y.w, k);
  }
  if (lane < kPiece / 4) sums[warp][lane] = y;
  __syncthreads();
  if (threadIdx.x < kPiece / 4) {
    l = 0;
    y = make_float4(0, 0, 0, 0);
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) {
      l += shares[w];
      add(y, 1.0f, sums[w][lane]);
    }
    write(h, d, y, l, top);
  }
}

__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// 16 bytes to shared memory, or 16 zeros
__device__ __forceinline__ void copy16(uint32_t to, const void* from, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// The block number of a token and its slot's place in the block, read ahead of the copies.
struct Ahead {
  int page;
  uint32_t inside;
};
template <int TILE, int TOKENS>
__device__ __forceinline__ Ahead look_ahead(const AttentionArgs& a, const Cursor<TILE>& c, int first, int lane) {
  Ahead r{-2, 0};                              // -2: no token
  if (c.left <= 0 || lane >= TOKENS) return r;
  const uint32_t p = (uint32_t)c.span.first + (uint32_t)c.tile * TILE + first + lane;
  if (p >= (uint32_t)c.span.end) return r;
  const uint32_t page = p / a.block;
  r.page = a.table[(size_t)c.b * a.W + page];
  if (r.page < 0) r.page = -1;                 // (no block: reported when its turn comes)
  r.inside = p - page * a.block.d;
  return r;
}

// Asks for the keys and values of a warp's tokens of a tile; returns which of them there are.  A row of DP elements is
// kept as CHUNKS chunks of 16 bytes, chunk c of row r at c ^ swizzle(r).
template <class T, int DP, int CHUNKS, int TOKENS, int TILE, class SwizzleK, class SwizzleV>
__device__ __forceinline__ uint32_t ask_for(const AttentionArgs& a, const Cursor<TILE>& c, Ahead ahead, uint32_t stage, int lane, int kv, SwizzleK sk, SwizzleV sv) {
  constexpr int PER = 16 / sizeof(T), ACROSS = CHUNKS < 32 ? CHUNKS : 32, ROWS = 32 / ACROSS;
  const long long slot = (long long)ahead.page * a.block.d + ahead.inside;
  const bool there = ahead.page >= 0 && slot < a.S;
  if (ahead.page != -2 && !there) raise_index(a.report);
  const uint32_t have = __ballot_sync(~0u, there);
  // in chunks: an array of 2^31 elements has fewer than 2^30
  const uint32_t offset = there ? (uint32_t)((slot * a.Hk + kv) * a.D / PER) : 0;
  const uint4 *keys = static_cast<const uint4*>(a.keys), *values = static_cast<const uint4*>(a.values);
  const bool all = have == (TOKENS == 32 ? ~0u : (1u << TOKENS) - 1);
#pragma unroll
  for (int r = 0; r < TOKENS; r += ROWS) {
    const int row = r + lane / ACROSS;
    const uint32_t from = __shfl_sync(~0u, offset, row);
#pragma unroll
    for (int k = 0; k < CHUNKS; k += ACROSS) {
      const int chunk = k + lane % ACROSS;
      const uint32_t k_at = stage + (row * CHUNKS + (chunk ^ sk(row))) * 16, v_at = stage + ((TOKENS + row) * CHUNKS + (chunk ^ sv(row))) * 16;
      if (CHUNKS > DP / PER && chunk >= DP / PER) continue;
      const bool inside = chunk * PER < a.D;               // (the same for every row: a lane's chunk)
      if (all) {
        const uint32_t at = from + (inside ? chunk : 0);
        copy16(k_at, keys + at, inside);
        copy16(v_at, values + at, inside);
      } else {
        const bool want = (have >> row & 1) && inside;
        const uint32_t at = want ? from + chunk : 0;
        copy16(k_at, keys + at, want);
        copy16(v_at, values + at, want);
      }
    }
  }
  return have;
}

// ---- 16-bit types: matrix instructions ------------------------------------------------------------------------------

template <class T> struct Half;
template <> struct Half<__half> {
  // The type ends at 2^16 and its steps at 2^-24.  Weights are raised by 2^15: two parts hold one of 2^-18 of the maximum or
  // more to 2^-22.  Those below (kSmall) are raised by another 2^18 and have products of their own, in tiles that have any:
  // down to 2^-36 they are held to 2^-22 as well, and what is lost of smaller ones is 2^-58 of the maximum at most.  (Raised
  // by 2^12 and without products of their own, weights of 2^-30 were off by 2^-8 and those of 2^-38 were nothing.  Where every
  // tile has small ones, 31 windows of 20 heads of 80 take 110 us in place of 97, 2 GB under sixteen heads of 256 673 in place of 515.)
  static constexpr int kParts = 2;
  static constexpr float kRaise = 32768.0f, kSmall = 0x1p-3f, kRaiseSmall = 0x1p18f, kNothing = 0x1p-43f;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
  static __device__ __forceinline__ float2 unpack(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
  // the product alone, and added to c
  static __device__ __forceinline__ void product(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
  }
  static __device__ __forceinline__ void mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};
template <> struct Half<__nv_bfloat16> {
  // eight bits each: all of a 32-bit weight, if it is above 2^-110 of the maximum
  static constexpr int kParts = 3;
  static constexpr float kRaise = 1.0f, kSmall = 0.0f;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
  static __device__ __forceinline__ float2 unpack(uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u)); }
  static __device__ __forceinline__ void product(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
  }
  static __device__ __forceinline__ void mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};

__device__ __forceinline__ void load_matrices(uint32_t* r, uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void load_matrices_transposed(uint32_t* r, uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ uint32_t transpose_matrix(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}

template <int DP, int NT, int WAYS>
struct HalfShape {
  static constexpr int kMats = DP == 64 ? 2 : 1;               // 16-token matrices of a warp's tile
  static constexpr int kTokens = 16 * kMats, kTile = kWarps / WAYS * kTokens, kRows = 8 * NT, kWays = WAYS;
  static constexpr int kChunks = DP == 96 ? 16 : DP / 8, kRowBytes = kChunks * 16;      // (a power of two, for the swizzle)
  static constexpr int kStageBytes = 2 * kTokens * kRowBytes;
  // stages and resident blocks per SM: as many as 227 KB hold
  static constexpr int kStages = DP == 96 ? 2 : 3;
  static constexpr int kResident = DP == 256 ? 1 : DP == 96 ? 3 : 2;
  // sixteen heads of 256: a lane's queries lie in shared memory, 16 bytes for every sixteen dimensions, because sums and queries
  // together do not fit its registers beside products that do not wait for one another (2 GB of bf16 660 us, so 501)
  static constexpr bool kAside = DP == 256 && NT == 2;
  static constexpr int kRingBytes = kWarps * kStages * kStageBytes, kShared = kRingBytes + (kAside ? kThreads * DP : 0);
  static_assert(WAYS > 1 || kRows * DP * 4 <= kStageBytes, "a warp's sums go through a stage");
};

// Scores as keys x queries (16 tokens x 8 heads, products of 16-bit values exact, sums in 32 bits), weighted values as
// values^T x weights (16 dimensions x 8 heads): the heads are the eight columns of a matrix instruction both times, and a
// lane's scores, maxima and sums belong to the same two heads, so that nothing is exchanged to rescale them.  The weights
// go from one shape to the other by transposing 8 x 8 matrices, as 16-bit parts that add up to them: three in bf16, all their
// bits, two in fp16, to 2^-22 (see Half).  Fewer would cost 2^-17 (bf16) of sum w |v|, more than the rounding of the result where
// values cancel.  A matrix instruction cuts off what it adds up, always to the same side, so that a sum that went through
// thousands of them would drift (128 requests of up to 24000 tokens: 0.65 % of the results in bf16 one step off, 0.03 % as it
// is): a tile's products start from zero and are added to the sums before them by rounding additions.  With up to eight
// query heads a key head the third part and the additions are hidden behind the loads (2 GB of bf16 heads of 256 331 us without
// both, 360 with; of 128 and 64 no difference); with sixteen they take their time (of 256 470 and 501, of 128 355 and 376, of 64
// 357 and 376).
template <class T, int DP, int NT, int WAYS>
__global__ void __launch_bounds__(kThreads, HalfShape<DP, NT, WAYS>::kResident) k_attention_half(AttentionArgs a) {
  using H = Half<T>;
  using S = HalfShape<DP, NT, WAYS>;
  constexpr int MT = S::kMats;
  constexpr int KS = S::kAside ? 4 : 2;        // steps of sixteen dimensions at a time: products that do not wait for one another
  extern __shared__ __align__(128) unsigned char shared[];
  __shared__ long long scan[kWarps];
  __shared__ Place place;
  __shared__ float ml[2 * kWarps * S::kRows];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  cudaTriggerProgrammaticLaunchCompletion();
  Cursor<S::kTile> c = find_place<T, S::kTile>(a, &place, scan);
  int4 join = make_int4(-1, 0, 0, 0);          // (by block)
  if (c.left <= 0) {
    if (a.parts && !a.by_unit && threadIdx.x == 0) a.joins[blockIdx.x] = join;
    return;
  }
  const uint32_t ring = shared_address(shared) + warp * S::kStages * S::kStageBytes;
  const auto swizzle = [](int row) { return row & 7; };
  // where this lane's rows of the 8 x 8 matrices start: tokens 0-7 | 8-15 by dimensions 0-7 | 8-15
  const int k_row = (lane & 7) + (lane >> 3 & 1) * 8, k_half = lane >> 4;
  const int v_row = (lane & 7) + (lane >> 4) * 8, v_half = lane >> 3 & 1;

  const int per = a.units / (a.Hk / WAYS);     // units of WAYS key heads
  const auto kv_of = [&](int unit) { return (per == 1 ? unit : unit / per) * WAYS + (WAYS > 1 ? warp : 0); };
  const int first = WAYS > 1 ? 0 : warp * S::kTokens;
  Cursor<S::kTile> next = c;
  Ahead ahead = look_ahead<S::kTile, S::kTokens>(a, next, first, lane);
  uint32_t have[S::kStages];
#pragma unroll
  for (int s = 0; s < S::kStages - 1; ++s) {
    have[s] = 0;
    if (next.left > 0) {
      have[s] = ask_for<T, DP, S::kChunks, S::kTokens>(a, next, ahead, ring + s * S::kStageBytes, lane, kv_of(next.unit), swizzle, swizzle);
      next.advance(a);
      ahead = look_ahead<S::kTile, S::kTokens>(a, next, first, lane);
    }
    commit_copies();
  }
  uint32_t q[NT][S::kAside ? 1 : DP / 16][2];
  uint4* aside = reinterpret_cast<uint4*>(shared + S::kRingBytes) + threadIdx.x;      // kAside: [DP / 16][kThreads]
  float o[NT][DP / 16][4], m[NT][2], l[NT][2];
  bool fresh = true, from_start = c.tile == 0;
  int stage = 0;
  while (c.left > 0) {
    if (fresh) {                               // a unit's queries: column n of B is head n, its rows are dimensions
      fresh = false;
      const int head0 = c.unit % per * S::kRows, kv = kv_of(c.unit);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int head = head0 + n * 8 + (lane >> 2);
        const uint32_t* from = reinterpret_cast<const uint32_t*>(static_cast<const T*>(a.q) + ((size_t)c.b * a.Hq + (size_t)kv * a.group + head) * a.D) + (lane & 3);
#pragma unroll
        for (int k = 0; k < DP / 16; ++k) {
          const uint32_t x = head < a.group && k * 16 < a.D ? from[k * 8] : 0, y = head < a.group && k * 16 + 8 < a.D ? from[k * 8 + 4] : 0;
          if constexpr (S::kAside) reinterpret_cast<uint2*>(aside + k * kThreads)[n] = make_uint2(x, y);
          else q[n][k][0] = x, q[n][k][1] = y;
#pragma unroll
          for (int i = 0; i < 4; ++i) o[n][k][i] = 0;
        }
        m[n][0] = m[n][1] = -INFINITY;
        l[n][0] = l[n][1] = 0;
      }
    }
    // the tile S::kStages - 1 further on
    uint32_t got = 0;
    {
      int to = stage + S::kStages - 1;
      if (to >= S::kStages) to -= S::kStages;
      if (next.left > 0) {
        got = ask_for<T, DP, S::kChunks, S::kTokens>(a, next, ahead, ring + to * S::kStageBytes, lane, kv_of(next.unit), swizzle, swizzle);
        next.advance(a);
        ahead = look_ahead<S::kTile, S::kTokens>(a, next, first, lane);
      }
      commit_copies();
    }
    wait_copies<S::kStages - 1>();
    __syncwarp();
    const uint32_t valid = have[0];
#pragma unroll
    for (int s = 0; s + 1 < S::kStages - 1; ++s) have[s] = have[s + 1];
    have[S::kStages - 2] = got;
    if (valid) {
      const uint32_t keys = ring + stage * S::kStageBytes, values = keys + S::kTokens * S::kRowBytes;
      // two sums each, over the even and the odd steps: half the chain of dependent instructions
      float s[MT][NT][4], odd[MT][NT][4];
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[t][n][i] = odd[t][n][i] = 0;
#pragma unroll
      for (int k = 0; k < DP / 16; ++k) {
        const int at = S::kAside ? 0 : k;
        if constexpr (S::kAside) {
          const uint4 x = aside[k * kThreads];
          q[0][0][0] = x.x, q[0][0][1] = x.y, q[NT - 1][0][0] = x.z, q[NT - 1][0][1] = x.w;
        }
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          uint32_t f[4];
          load_matrices(f, keys + (t * 16 + k_row) * S::kRowBytes + (((k * 2 + k_half) ^ (k_row & 7)) << 4));
#pragma unroll
          for (int n = 0; n < NT; ++n) H::mma(k & 1 ? odd[t][n] : s[t][n], f, q[n][at][0], q[n][at][1]);
        }
      }
      uint32_t parts[H::kParts][MT][NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const bool is = valid >> (t * 16 + (lane >> 2) + (i & 2) * 4) & 1;
            const float x = (s[t][n][i] + odd[t][n][i]) * a.scale_log2;
            s[t][n][i] = is ? x : -INFINITY;
            top[i & 1] = fmaxf(top[i & 1], is ? fmaxf(x, -FLT_MAX) : -INFINITY);
          }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) top[i] = fmaxf(top[i], __shfl_xor_sync(~0u, top[i], d));
          top[i] = fmaxf(top[i], m[n][i]);
        }
        if (__any_sync(~0u, top[0] > m[n][0] || top[1] > m[n][1])) {
          const float f0 = power2(m[n][0] - top[0]), f1 = power2(m[n][1] - top[1]);     // (valid: the new maxima are finite, or above)
#pragma unroll
          for (int k = 0; k < DP / 16; ++k) o[n][k][0] *= f0, o[n][k][1] *= f1, o[n][k][2] *= f0, o[n][k][3] *= f1;
          l[n][0] *= f0, l[n][1] *= f1;
          m[n][0] = top[0], m[n][1] = top[1];
        }
        // a weight as the sum of 16-bit parts, each transposed to what the second product takes
        const auto split = [](const float* w, auto&& part) {
          float rest[4] = {w[0], w[1], w[2], w[3]};
#pragma unroll
          for (int p = 0; p < H::kParts; ++p)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const uint32_t x = H::pack(rest[2 * i], rest[2 * i + 1]);
              const float2 back = H::unpack(x);
              rest[2 * i] -= back.x, rest[2 * i + 1] -= back.y;
              part(p, i) = transpose_matrix(x);
            }
        };
        float w[MT][4];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
#pragma unroll
          for (int i = 0; i < 4; ++i) w[t][i] = power2(s[t][n][i] - m[n][i & 1]) * H::kRaise;
          l[n][0] += w[t][0] + w[t][2];
          l[n][1] += w[t][1] + w[t][3];
        }
        if constexpr (H::kSmall > 0) {
          // (of numbers that are not negative, in the order of their patterns)
          const uint32_t least = __float_as_uint(H::kNothing);
          uint32_t above = ~0u;
#pragma unroll
          for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) above = min(above, __float_as_uint(w[t][i]) - least);
          if (__any_sync(~0u, above < __float_as_uint(H::kSmall) - least)) {
            uint32_t small[H::kParts][MT][2];
#pragma unroll
            for (int t = 0; t < MT; ++t) {
              float x[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const bool is = w[t][i] < H::kSmall;
                x[i] = is ? w[t][i] * H::kRaiseSmall : 0.0f;
                w[t][i] = is ? 0.0f : w[t][i];
              }
              split(x, [&](int p, int i) -> uint32_t& { return small[p][t][i]; });
            }
#pragma unroll
            for (int k = 0; k < DP / 16; ++k) {
              float c[4] = {0, 0, 0, 0};
#pragma unroll
              for (int t = 0; t < MT; ++t) {
                uint32_t f[4];
                load_matrices_transposed(f, values + (t * 16 + v_row) * S::kRowBytes + (((k * 2 + v_half) ^ (v_row & 7)) << 4));
#pragma unroll
                for (int p = 0; p < H::kParts; ++p) H::mma(c, f, small[p][t][0], small[p][t][1]);
              }
#pragma unroll
              for (int i = 0; i < 4; ++i) o[n][k][i] = fmaf(c[i], 1 / H::kRaiseSmall, o[n][k][i]);
            }
          }
        }
#pragma unroll
        for (int t = 0; t < MT; ++t) split(w[t], [&](int p, int i) -> uint32_t& { return parts[p][t][n][i]; });
      }
#pragma unroll
      for (int k = 0; k < DP / 16; k += KS) {
        float c[KS][NT][4];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          uint32_t f[KS][4];
#pragma unroll
          for (int i = 0; i < KS; ++i)
            load_matrices_transposed(f[i], values + (t * 16 + v_row) * S::kRowBytes + ((((k + i) * 2 + v_half) ^ (v_row & 7)) << 4));
#pragma unroll
          for (int p = 0; p < H::kParts; ++p)
#pragma unroll
            for (int i = 0; i < KS; ++i)
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                if (t == 0 && p == 0) H::product(c[i][n], f[i], parts[p][t][n][0], parts[p][t][n][1]);
                else H::mma(c[i][n], f[i], parts[p][t][n][0], parts[p][t][n][1]);
              }
        }
#pragma unroll
        for (int i = 0; i < KS; ++i)
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[n][k + i][j] += c[i][n][j];
      }
    }
    __syncwarp();                              // the stage may be filled again
    if (++stage == S::kStages) stage = 0;
    const bool to_end = c.tile + 1 == c.tiles;
    if (to_end || c.left == 1) {
      const int head0 = c.unit % per * S::kRows, kv = kv_of(c.unit);
      const bool whole = from_start && to_end;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) l[n][i] += __shfl_xor_sync(~0u, l[n][i], d);
      }
      if constexpr (WAYS > 1) {                // a warp has the unit's tokens for its own key head
        const Records<DP, S::kRows * WAYS> to(a);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int row = n * 8 + (lane & 3) * 2 + i;
            if (head0 + row >= a.group) continue;
            if (whole) {
              T* out = static_cast<T*>(a.out) + ((size_t)c.b * a.Hq + (size_t)kv * a.group + head0 + row) * a.D + (lane >> 2);
              const bool none = m[n][i] == -INFINITY;
#pragma unroll
              for (int k = 0; k < DP / 16; ++k) {
                if (k * 16 < a.D) out[k * 16] = narrow<T>(none ? 0.0f : __fdiv_rn(o[n][k][i], l[n][i]));
                if (k * 16 + 8 < a.D) out[k * 16 + 8] = narrow<T>(none ? 0.0f : __fdiv_rn(o[n][k][i + 2], l[n][i]));
              }
            } else {
              const size_t at = to.row(blockIdx.x, from_start, warp * S::kRows + row);
              float* sum = to.sums + at * DP + (lane >> 2);
#pragma unroll
              for (int k = 0; k < DP / 16; ++k) sum[k * 16] = o[n][k][i], sum[k * 16 + 8] = o[n][k][i + 2];
              if (lane < 4) to.tops[at] = m[n][i], to.weights[at] = l[n][i];
            }
          }
      } else {                                 // through the stage just read, which is filled again only behind this
        const int used = (stage == 0 ? S::kStages : stage) - 1;
        float* sums = reinterpret_cast<float*>(shared + used * S::kStageBytes);
        constexpr int kStride = S::kStages * S::kStageBytes / 4;
        __syncwarp();
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int row = n * 8 + (lane & 3) * 2 + i;
            if (lane < 4) {
              ml[warp * S::kRows + row] = m[n][i];
              ml[(kWarps + warp) * S::kRows + row] = l[n][i];
            }
            float* to = sums + warp * kStride + row * DP;
#pragma unroll
            for (int k = 0; k < DP / 16; ++k) {
              to[(k * 16 + (lane >> 2)) ^ spread(row)] = o[n][k][i];
              to[(k * 16 + 8 + (lane >> 2)) ^ spread(row)] = o[n][k][i + 2];
            }
          }
        __syncthreads();
        finish_unit<T, DP, S::kRows, true>(a, c.b, kv, head0, from_start, to_end, sums, kStride, ml);
        __syncthreads();
      }
      if (a.parts && from_start) {
        const int4 of = to_end ? make_int4(-1, 0, 0, 0) : join_of(a, c, place);
        if (!to_end) join = of;
        if (a.by_unit && threadIdx.x == 0) a.joins[(size_t)c.b * a.units + c.unit] = of;
      }
      fresh = from_start = true;
    }
    c.advance(a);
  }
  wait_copies<0>();
  if (a.parts && !a.by_unit && threadIdx.x == 0) a.joins[blockIdx.x] = join;
}

// ---- fp32 --------------------------------------------------------------------------------------------------------------

template <int DP, int HEADS>
struct FloatShape {
  static constexpr int kTokens = 8, kTile = kWarps * kTokens, kRows = HEADS, kWays = 1;
  static constexpr int kStageBytes = 2 * kTokens * DP * 4;
  static constexpr int kStages = DP == 128 ? 2 : 3;
  static constexpr int kResident = DP == 256 ? 1 : DP == 64 && HEADS < 8 ? 4 : 3;
  static constexpr int kShared = kWarps * kStages * kStageBytes;
};

// Two 32-bit numbers in one register pair, worked on by one instruction each.
using Pair = unsigned long long;
__device__ __forceinline__ Pair pair_of(float lo, float hi) {
  Pair p;
  asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(lo), "f"(hi));
  return p;
}
__device__ __forceinline__ float2 both_of(Pair p) {
  float2 v;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(p));
  return v;
}
__device__ __forceinline__ Pair fma_pair(Pair a, Pair b, Pair c) {
  Pair d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ Pair mul_pair(Pair a, Pair b) {
  Pair d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

// The same walk with 32-bit multiplications and additions, two, four or eight heads at a time.  Scores: DP / 8 lanes share
// a token, eight dimensions of all heads' queries in a lane's registers; the heads' sums are scattered over those lanes,
// so that a lane ends up with one head's scores.  (With the queries in shared memory, read for every key, the block waits
// for shared memory: eight heads of 128, 2 GB of keys and values 459 us.)  Values: a lane has four dimensions of all heads.
template <int DP, int HEADS>
__global__ void __launch_bounds__(kThreads, FloatShape<DP, HEADS>::kResident) k_attention_float(AttentionArgs a) {
  using S = FloatShape<DP, HEADS>;
  constexpr int LANES = DP / 8, AT_ONCE = 32 / LANES, PASSES = S::kTokens / AT_ONCE;        // lanes of a token, tokens of a pass
  constexpr int CHUNKS = DP / 4, SPLIT = CHUNKS < 32 ? 32 / CHUNKS : 1, VECS = CHUNKS / 32 > 1 ? CHUNKS / 32 : 1;
  extern __shared__ __align__(128) unsigned char shared[];
  __shared__ long long scan[kWarps];
  __shared__ Place place;
  __shared__ float ml[2 * kWarps * S::kRows];
  __shared__ __align__(16) float2 weights[kWarps][HEADS][8];       // each twice, for pairs of dimensions
  __shared__ float falls[kWarps][HEADS];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  cudaTriggerProgrammaticLaunchCompletion();
  Cursor<S::kTile> c = find_place<float, S::kTile>(a, &place, scan);
  int4 join = make_int4(-1, 0, 0, 0);          // (by block)
  if (c.left <= 0) {
    if (a.parts && !a.by_unit && threadIdx.x == 0) a.joins[blockIdx.x] = join;
    return;
  }
  const unsigned char* ring = shared + warp * S::kStages * S::kStageBytes;
  const uint32_t ring_at = shared_address(ring);
  const auto plain = [](int) { return 0; };
  const int part = lane % LANES, token = lane / LANES;        // of a pass
  int head = 0;                                               // this lane's
#pragma unroll
  for (int b = 0, left = HEADS / 2; left > 0; ++b, left /= 2) head += (lane >> b & 1) * left;
  const int chunk = lane % (CHUNKS < 32 ? CHUNKS : 32), half = lane / (CHUNKS < 32 ? CHUNKS : 32);

  Cursor<S::kTile> next = c;
  Ahead ahead = look_ahead<S::kTile, S::kTokens>(a, next, warp * S::kTokens, lane);
  uint32_t have[S::kStages];
#pragma unroll
  for (int s = 0; s < S::kStages - 1; ++s) {
    have[s] = 0;
    if (next.left > 0) {
      have[s] = ask_for<float, DP, CHUNKS, S::kTokens>(a, next, ahead, ring_at + s * S::kStageBytes, lane, next.unit / (a.units / a.Hk), plain, plain);
      next.advance(a);
      ahead = look_ahead<S::kTile, S::kTokens>(a, next, warp * S::kTokens, lane);
    }
    commit_copies();
  }
  Pair o[HEADS][VECS][2];
  Pair q[HEADS][4];
  float m, l;
  bool fresh = true, from_start = c.tile == 0;
  int stage = 0;
  while (c.left > 0) {
    if (fresh) {
      fresh = false;
      const int per = a.units / a.Hk, head0 = c.unit % per * S::kRows, kv = c.unit / per;
#pragma unroll
      for (int h = 0; h < HEADS; ++h) {
        const float4* from = reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + ((size_t)c.b * a.Hq + (size_t)kv * a.group + head0 + h) * a.D);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int at = part + i * LANES;
          const float4 x = head0 + h < a.group && at * 4 < a.D ? from[at] : make_float4(0, 0, 0, 0);
          q[h][2 * i] = pair_of(x.x, x.y), q[h][2 * i + 1] = pair_of(x.z, x.w);
        }
#pragma unroll
        for (int v = 0; v < VECS; ++v) o[h][v][0] = o[h][v][1] = 0;
      }
      m = -INFINITY, l = 0;
    }
    uint32_t got = 0;
    {
      int to = stage + S::kStages - 1;
      if (to >= S::kStages) to -= S::kStages;
      if (next.left > 0) {
        got = ask_for<float, DP, CHUNKS, S::kTokens>(a, next, ahead, ring_at + to * S::kStageBytes, lane, next.unit / (a.units / a.Hk), plain, plain);
        next.advance(a);
        ahead = look_ahead<S::kTile, S::kTokens>(a, next, warp * S::kTokens, lane);
      }
      commit_copies();
    }
    wait_copies<S::kStages - 1>();
    __syncwarp();
    const uint32_t valid = have[0];
#pragma unroll
    for (int s = 0; s + 1 < S::kStages - 1; ++s) have[s] = have[s + 1];
    have[S::kStages - 2] = got;
    if (valid) {
      const ulonglong2* keys = reinterpret_cast<const ulonglong2*>(ring + stage * S::kStageBytes);
      const ulonglong2* values = keys + S::kTokens * CHUNKS;
      float s[PASSES], top = -INFINITY;
#pragma unroll
      for (int j = 0; j < PASSES; ++j) {
        const int t = j * AT_ONCE + token;
        const ulonglong2 k0 = keys[t * CHUNKS + part], k1 = keys[t * CHUNKS + part + LANES];
        float x[HEADS];
#pragma unroll
        for (int h = 0; h < HEADS; ++h) {
          const float2 y = both_of(fma_pair(k1.y, q[h][3], fma_pair(k1.x, q[h][2], fma_pair(k0.y, q[h][1], mul_pair(k0.x, q[h][0])))));
          x[h] = y.x + y.y;
        }
        int left = HEADS;                      // heads halved between the lanes of pairs, then sums alone
#pragma unroll
        for (int b = 1; b < LANES; b <<= 1) {
          if (left > 1) {
            left /= 2;
#pragma unroll
            for (int i = 0; i < left; ++i) {
              const float other = __shfl_xor_sync(~0u, lane & b ? x[i] : x[i + left], b);
              x[i] = (lane & b ? x[i + left] : x[i]) + other;
            }
          } else x[0] += __shfl_xor_sync(~0u, x[0], b);
        }
        const bool is = valid >> t & 1;
        s[j] = is ? x[0] * a.scale_log2 : -INFINITY;
        top = fmaxf(top, is ? fmaxf(s[j], -FLT_MAX) : -INFINITY);
      }
#pragma unroll
      for (int d = LANES; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
      top = fmaxf(top, m);
      const bool rises = __any_sync(~0u, top > m);
      const float fall = power2(m - top);
      m = top;
      l *= fall;
      const bool writes = part < HEADS;                       // (further lanes of a token hold the same again)
#pragma unroll
      for (int j = 0; j < PASSES; ++j) {
        const float w = power2(s[j] - top);
        l += w;
        if (writes) weights[warp][head][j * AT_ONCE + token] = make_float2(w, w);
      }
      if (lane < HEADS) falls[warp][head] = fall;
      __syncwarp();
#pragma unroll
      for (int h = 0; h < HEADS; ++h) {
        if (rises) {
          const Pair fall = pair_of(falls[warp][h], falls[warp][h]);
#pragma unroll
          for (int v = 0; v < VECS; ++v) o[h][v][0] = mul_pair(o[h][v][0], fall), o[h][v][1] = mul_pair(o[h][v][1], fall);
        }
      }
#pragma unroll
      for (int f = 0; f < 4 / SPLIT; ++f) {                  // tokens two by two
        const int t0 = ((SPLIT == 2 ? half * 2 : 0) + f) * 2;
        ulonglong2 w[HEADS];
#pragma unroll
        for (int h = 0; h < HEADS; ++h) w[h] = *reinterpret_cast<const ulonglong2*>(&weights[warp][h][t0]);
#pragma unroll
        for (int v = 0; v < VECS; ++v) {
          const ulonglong2 x = values[t0 * CHUNKS + chunk + v * 32], y = values[(t0 + 1) * CHUNKS + chunk + v * 32];
#pragma unroll
          for (int h = 0; h < HEADS; ++h) {
            o[h][v][0] = fma_pair(w[h].y, y.x, fma_pair(w[h].x, x.x, o[h][v][0]));
            o[h][v][1] = fma_pair(w[h].y, y.y, fma_pair(w[h].x, x.y, o[h][v][1]));
          }
        }
      }
    }
    __syncwarp();
    if (++stage == S::kStages) stage = 0;
    const bool to_end = c.tile + 1 == c.tiles;
    if (to_end || c.left == 1) {
      const int per = a.units / a.Hk, used = (stage == 0 ? S::kStages : stage) - 1;
      float* sums = reinterpret_cast<float*>(shared + used * S::kStageBytes);      // through the stage just read
      constexpr int kStride = S::kStages * S::kStageBytes / 4;
#pragma unroll
      for (int d = LANES; d < 32; d <<= 1) l += __shfl_xor_sync(~0u, l, d);
      if (lane < HEADS) {
        ml[warp * S::kRows + head] = m;
        ml[(kWarps + warp) * S::kRows + head] = l;
      }
#pragma unroll
      for (int h = 0; h < HEADS; ++h)
#pragma unroll
        for (int v = 0; v < VECS; ++v) {
          const float2 lo = both_of(o[h][v][0]), hi = both_of(o[h][v][1]);
          float x[4] = {lo.x, lo.y, hi.x, hi.y};
          if constexpr (SPLIT == 2)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] += __shfl_xor_sync(~0u, x[i], 16);
          if (half == 0) *reinterpret_cast<float4*>(sums + warp * kStride + h * DP + (chunk + v * 32) * 4) = make_float4(x[0], x[1], x[2], x[3]);
        }
      __syncthreads();
      finish_unit<float, DP, S::kRows, false>(a, c.b, c.unit / per, c.unit % per * S::kRows, from_start, to_end, sums, kStride, ml);
      if (a.parts && from_start) {
        const int4 of = to_end ? make_int4(-1, 0, 0, 0) : join_of(a, c, place);
        if (!to_end) join = of;
        if (a.by_unit && threadIdx.x == 0) a.joins[(size_t)c.b * a.units + c.unit] = of;
      }
      __syncthreads();
      fresh = from_start = true;
    }
    c.advance(a);
  }
  wait_copies<0>();
  if (a.parts && !a.by_unit && threadIdx.x == 0) a.joins[blockIdx.x] = join;
}

// No query heads, and so no result: only the lengths and the blocks of the tokens attended to are looked at.  A block of the
// grid to a request.
__global__ void __launch_bounds__(kThreads) k_attended_blocks(AttentionArgs a) {
  follow();
  bool bad = false;
  for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
    const int length = a.lens[b];
    bad = bad || length < 0 || length > (long long)a.W * a.block.d;
    const Span s = span_of(a, b);
    if (s.first == s.end) continue;
    const uint32_t last = (uint32_t)(s.end - 1) / a.block;
    for (uint32_t p = (uint32_t)s.first / a.block + threadIdx.x; p <= last; p += kThreads) {
      const int page = a.table[(size_t)b * a.W + p];
      const uint32_t inside = p < last ? a.block.d - 1 : (uint32_t)(s.end - 1) - last * a.block.d;      // the block's last token
      bad = bad || page < 0 || (long long)page * a.block.d + inside >= a.S;
    }
  }
  if (bad) raise_index(a.report);
}

// ---- launches ------------------------------------------------------------------------------------------------------------

AttentionArgs arguments(const ClusterLaunch& L) {
  const int D = (int)L.op.iparam[1];
  const int Hq = (int)L.op.shape[1] / D, Hk = slot(L, 1).C / D;
  const bool empty = slot(L, 1).R == 0;                       // (a copy of no bytes still names an address)
  return {report_of(L), slot(L, 0).ptr, slot(L, empty ? 0 : 1).ptr, slot(L, empty ? 0 : 2).ptr, slot_ptr<int>(L, 3), slot_ptr<int>(L, 4), result_ptr<void>(L),
          (int)L.op.shape[0], slot(L, 3).C, slot(L, 1).R, Hq, Hk, D, (int)std::min<int64_t>(L.op.iparam[2], 0x7FFFFFFF),
          Hk > 0 ? Hq / Hk : 0, 0, (float)(L.op.fparam[0] * 1.4426950408889634), divisor((uint32_t)L.op.iparam[0]), nullptr, 0, 0, nullptr, false};
}

// Blocks of the grid, and whether a unit may be split: never if no request can have more than a tile.
template <class S>
int grid_of(AttentionArgs& a, bool& splits) {
  a.units = a.Hk / S::kWays * ((a.group + S::kRows - 1) / S::kRows);
  const long long room = std::min<long long>((long long)a.W * a.block.d, 0x7FFFFFFF);       // (lengths are 32-bit numbers)
  const long long tiles = std::max<long long>((room + S::kTile - 1) / S::kTile, 1) * a.B * a.units;
  splits = room > S::kTile;
  return a.grid = (int)std::min<long long>(tiles, std::min((long long)sm_count() * S::kResident, (long long)kMaxGrid));
}

// Entries of AttentionArgs::joins.
long long joins_of(const AttentionArgs& a) { return std::min<long long>(a.grid, (long long)a.B * a.units); }

template <class S, int DP>
int64_t scratch_of(AttentionArgs a) {
  bool splits;
  const int64_t grid = grid_of<S>(a, splits);
  return splits ? joins_of(a) * 16 + (int64_t)Records<DP, S::kRows * S::kWays>::bytes((int)grid) : 0;
}

template <class T, int DP, class S, class K>
int run(const ClusterLaunch& L, K kernel, std::atomic<uint64_t>& allowed) {
  AttentionArgs a = arguments(L);
  bool splits;
  const int grid = grid_of<S>(a, splits);
  if (splits) {
    a.joins = reinterpret_cast<int4*>(L.scratch);
    a.by_unit = (long long)a.B * a.units <= grid;
    a.parts = reinterpret_cast<float*>(a.joins + joins_of(a));
  }
  const int rc = allow_shared(kernel, S::kShared, allowed);
  if (rc != ACC_OK) return rc;
  const int heads = S::kRows * S::kWays, pieces = DP / kPiece;
  a.join_rows = joins_of(a) * heads * pieces <= 8 * sm_count() ? 1 : std::min(8, heads);
  // (not launched early: beside the kernel before it an SM is divided for less shared memory, and keeps to that while the
  // blocks that did fit run; 31 windows of 4096 tokens, back to back: 101 us, launched early 154)
  kernel<<<grid, kThreads, S::kShared, L.stream>>>(a);
  const int first = launched();
  if (first != ACC_OK || !splits) return first;
  ++L.extra_launches;
  return launch_following(k_join<T, DP, S::kRows, S::kWays>, dim3((unsigned)joins_of(a), heads / a.join_rows, a.join_rows == 1 ? pieces : 1),
                          kJoinThreads, 0, L.stream, a);
}

// Calls f(type, DP, shape, kernel) for the kernel that a launch takes: heads padded to 64, 96, 128 or 256 elements; for
// 16-bit types sixteen heads at a time where a key head has more than eight; and the four warps on four key heads where
// there are many requests: their rows lie side by side, so that what is read together is four times as long (2 GB of keys
// and values of 20 heads of 80: 443 us with four warps on one head, 302 so; of 8 heads of 128 no difference).  With few
// requests it would leave more records to join: one of 8000 tokens 21 us, so 30.
constexpr int kManyHeads = 128;
template <class T, int DP, int NT, class F>
auto choose_ways(const ClusterLaunch& L, F f) {
  const std::integral_constant<int, DP> dp{};
  const int Hk = slot(L, 1).C / (int)L.op.iparam[1];
  if (Hk % kWarps == 0 && L.op.shape[0] * Hk >= kManyHeads) return f(T{}, dp, HalfShape<DP, NT, kWarps>{}, k_attention_half<T, DP, NT, kWarps>);
  return f(T{}, dp, HalfShape<DP, NT, 1>{}, k_attention_half<T, DP, NT, 1>);
}
template <class T, class F>
auto choose_half(const ClusterLaunch& L, F f) {
  const int D = (int)L.op.iparam[1];
  const bool wide = (int)L.op.shape[1] > 8 * slot(L, 1).C;
  if (D <= 64) return wide ? choose_ways<T, 64, 2>(L, f) : choose_ways<T, 64, 1>(L, f);
  if (D <= 96) return wide ? choose_ways<T, 96, 2>(L, f) : choose_ways<T, 96, 1>(L, f);
  if (D <= 128) return wide ? choose_ways<T, 128, 2>(L, f) : choose_ways<T, 128, 1>(L, f);
  return wide ? choose_ways<T, 256, 2>(L, f) : choose_ways<T, 256, 1>(L, f);
}
template <class F>
auto choose(const ClusterLaunch& L, F f) {
  const int D = (int)L.op.iparam[1];
  if (L.op.dtype == ACC_F32) {
    const auto heads = [&](auto dp) {
      constexpr int DP = decltype(dp)::value;
      const int group = (int)(L.op.shape[1] / std::max(slot(L, 1).C, 1));
      if (group <= 2) return f(float{}, dp, FloatShape<DP, 2>{}, k_attention_float<DP, 2>);
      if (group <= 4) return f(float{}, dp, FloatShape<DP, 4>{}, k_attention_float<DP, 4>);
      return f(float{}, dp, FloatShape<DP, 8>{}, k_attention_float<DP, 8>);
    };
    if (D <= 64) return heads(std::integral_constant<int, 64>{});
    if (D <= 128) return heads(std::integral_constant<int, 128>{});
    return heads(std::integral_constant<int, 256>{});
  }
  return L.op.dtype == ACC_F16 ? choose_half<__half>(L, f) : choose_half<__nv_bfloat16>(L, f);
}

bool nothing(const ClusterLaunch& L) { return L.op.shape[0] == 0 || L.op.shape[1] == 0; }

int launch_checks(const ClusterLaunch& L) {
  const AttentionArgs a = arguments(L);
  if (a.B == 0) return no_launch(L);
  return launch_following(k_attended_blocks, dim3((unsigned)std::min(a.B, sm_count() * 8)), kThreads, 0, L.stream, a);
}

int64_t attention_scratch(const ClusterLaunch& L) {
  if (nothing(L)) return 0;
  return choose(L, [&](auto, auto dp, auto shape, auto) { return scratch_of<decltype(shape), decltype(dp)::value>(arguments(L)); });
}

int launch_attention(const ClusterLaunch& L) {
  if (nothing(L)) return launch_checks(L);
  return choose(L, [&](auto t, auto dp, auto shape, auto kernel) {
    static std::atomic<uint64_t> allowed{0};
    return run<decltype(t), decltype(dp)::value, decltype(shape)>(L, kernel, allowed);
  });
}

const Register attention(ACC_PAGED_ATTENTION, "k_attention", attention_scratch, launch_attention);

}  // namespace
}  // namespace ops
}  // namespace acc
