// Embedding of packed tokens: the lookup, and the table's gradient by tokens sorted by id.
//
//   x_k = scale table[id_k]          dtable_v = scale sum_{k : id_k = v} dx_k
//
// Both are bound by HBM: the lookup reads the rows that occur and writes one a token, the gradient reads
// one a token and writes the whole table in 32 bits.  For the gradient the pairs (id, k) are sorted by a stable radix
// sort, so that the tokens of a table row stand together in ascending order, and every row of the table is written
// once, by the threads that add up its tokens.  Nothing is added by atomics: the order of the sums is fixed.
#include <atomic>
#include <initializer_list>

#include "nat_common.cuh"
#include "nat_rows.cuh"

namespace nat {
namespace embed {
namespace {

using rows::kChunk;
using rows::kPairs;
using rows::Raw;

constexpr int kThreads = 256;
// Pairs a block sorts at a time: 166,001 tokens of 1024 columns 219, 209, 212 us with 2048, 1024, 512; 20,000 of 512 93, 89,
// 88; 1,000,000 of 64 217, 226, 245.
constexpr int kTile = 1024;
constexpr int kWarps = kThreads / 32;
constexpr int kRounds = kTile / kThreads;
constexpr int kMaxDigits = 512;
// Sorted tokens of a piece; a table row with more is added up in pieces.  us with 128, 64, 32: 20,000 tokens of 512 columns
// 100, 93, 89; 166,001 of 4096 687, 677, 701; 5,000 of 512 with two ids 27, 21, 20; 166,001 of 1024 with 512 ids 93, 99, 113.
constexpr uint32_t kPiece = 64;

struct Rows {
  const int32_t *ids, *sel_idx, *n_rows;
  int64_t cap;
  int32_t V;
};

// Positions are unsigned: a tile's end may lie behind 2^31.
__device__ __forceinline__ uint32_t row_count(const Rows& r) {
  return (uint32_t)(r.n_rows ? min((int64_t)max(*r.n_rows, 0), r.cap) : r.cap);
}
// The id of row k, V where it lies outside the table.
__device__ __forceinline__ uint32_t row_id(const Rows& r, uint32_t k) {
  const int32_t id = r.ids[r.sel_idx ? r.sel_idx[k] : k];
  return (uint32_t)id < (uint32_t)r.V ? (uint32_t)id : (uint32_t)r.V;
}

// ------------------------------------------------------------------------- lookup
// A warp a row, or several short rows a warp (`tpr` lanes each, a power of two), each lane with kAhead chunks on their
// way.  Every warp has one turn and the blocks come in the rows' order, so that the rows written at any time lie
// together: 166,001 rows of 4096 take 303 us, and 340 where persistent warps stride over them.
template <typename T>
constexpr int kAhead = sizeof(T) == 2 ? 4 : 2;

// Rows of the table are read again and again: they stay in L2 (the output, written once, does not).
__device__ __forceinline__ Raw<__nv_bfloat16> load_kept(const __nv_bfloat16* p) {
  return {__ldg(reinterpret_cast<const uint4*>(p))};
}
__device__ __forceinline__ Raw<float> load_kept(const float* p) {
  return {__ldg(reinterpret_cast<const float4*>(p)), __ldg(reinterpret_cast<const float4*>(p) + 1)};
}

// PLAIN: a scale of one; the rows are moved as they are (at the board's power limit the arithmetic would cost time).
template <typename T, bool PLAIN>
__global__ void __launch_bounds__(kThreads, 6)
lookup_kernel(const T* __restrict__ table, Rows r, T* __restrict__ x, int d, int tpr_log2, float scale) {
  constexpr int A = kAhead<T>;
  const int64_t k = (int64_t)blockIdx.x * (kThreads >> tpr_log2) + (threadIdx.x >> tpr_log2);
  if (k >= row_count(r)) return;
  const uint32_t id = row_id(r, (uint32_t)k);
  const bool known = id < (uint32_t)r.V;
  const T* from = table + (int64_t)(known ? id : 0u) * d;
  T* to = x + k * d;
  const int stride = kChunk << tpr_log2;
  for (int c = (threadIdx.x & ((1 << tpr_log2) - 1)) * kChunk; c < d; c += A * stride) {
    Raw<T> raw[A];
#pragma unroll
    for (int u = 0; u < A; ++u)
      if (c + u * stride < d) raw[u] = load_kept(from + c + u * stride);
#pragma unroll
    for (int u = 0; u < A; ++u) {
      if (c + u * stride >= d) break;
      if (!PLAIN || !known) {
        float2 v[kPairs];
        rows::widen(raw[u], v);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) v[i] = known ? mul2(v[i], both(scale)) : both(__uint_as_float(0x7FC00000u));
        rows::narrow(v, raw[u]);
      }
      rows::store_raw(to + c + u * stride, raw[u]);
    }
  }
}

// --------------------------------------------------------------------------- sort
// Stable sort by digits from the lowest up.  A block owns up to kTile consecutive pairs and a warp of it a run of
// them, in rounds of 32, so that a pair's rank among those of its digit is: what earlier warps counted, what this
// warp counted in earlier rounds, and the lanes below.  Rounds are dealt evenly, so that few pairs take few.
struct Digit {
  int shift, bits;
  __device__ __forceinline__ int of(uint32_t key) const { return (int)(key >> shift) & ((1 << bits) - 1); }
  __device__ __forceinline__ int count() const { return 1 << bits; }
};

template <int THREADS = kThreads>
__device__ __forceinline__ int rounds_for(uint32_t valid) {
  return (int)((min(valid, (uint32_t)(THREADS * kRounds)) + THREADS - 1) / THREADS);
}
__device__ __forceinline__ uint32_t slot_of(int round, int rounds) {
  return (threadIdx.x >> 5) * rounds * 32 + round * 32 + (threadIdx.x & 31);
}

// rank[j] of the thread's pairs among their digit within the warp; `counts` [warps][digits] holds the warps' totals
// afterwards.
template <int THREADS = kThreads>
__device__ __forceinline__ void warp_ranks(const uint32_t (&key)[kRounds], uint32_t valid, int rounds, Digit digit,
                                           uint32_t* counts, uint32_t (&rank)[kRounds]) {
  const int lane = threadIdx.x & 31;
  uint32_t* mine = counts + (threadIdx.x >> 5) * digit.count();
  for (int i = threadIdx.x; i < THREADS / 32 * digit.count(); i += THREADS) counts[i] = 0u;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kRounds; ++j) {
    if (j >= rounds) break;
    const bool in = slot_of(j, rounds) < valid;
    const int g = digit.of(key[j]);
    // the lanes with the same digit, bit by bit (__match_any_sync takes longer)
    unsigned same = __ballot_sync(0xFFFFFFFFu, in);
    for (int b = 0; b < digit.bits; ++b) {
      const unsigned set = __ballot_sync(0xFFFFFFFFu, (g >> b) & 1);
      same &= (g >> b) & 1 ? set : ~set;
    }
    const unsigned below = same & ((1u << lane) - 1u);
    uint32_t before = 0u;
    if (in) before = mine[g];
    __syncwarp();
    if (in && below == 0u) mine[g] = before + (uint32_t)__popc(same);
    __syncwarp();
    rank[j] = before + (uint32_t)__popc(below);
  }
  __syncthreads();
}

// counts[w][g] -> how many of digit g the warps before w hold; returns nothing, leaves the block's total of digit g
// in total[g].
template <int THREADS>
__device__ __forceinline__ void across_warps(uint32_t* counts, uint32_t* total, int digits) {
  for (int g = threadIdx.x; g < digits; g += THREADS) {
    uint32_t run = 0u;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
      const uint32_t c = counts[w * digits + g];
      counts[w * digits + g] = run;
      run += c;
    }
    total[g] = run;
  }
  __syncthreads();
}

// total[0..digits) -> its exclusive prefix sums (digits <= kMaxDigits = 2 kThreads: two of each thread).
template <int THREADS = kThreads>
__device__ __forceinline__ void prefix_digits(uint32_t* total, int digits) {
  __shared__ uint32_t sums[THREADS / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t a = 2 * threadIdx.x < digits ? total[2 * threadIdx.x] : 0u;
  uint32_t b = 2 * threadIdx.x + 1 < digits ? total[2 * threadIdx.x + 1] : 0u;
  uint32_t run = a + b;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t left = __shfl_up_sync(0xFFFFFFFFu, run, o);
    if (lane >= o) run += left;
  }
  if (lane == 31) sums[warp] = run;
  __syncthreads();
  uint32_t before = run - (a + b);
  for (int w = 0; w < min(warp, kWarps); ++w) before += sums[w];
  if (2 * threadIdx.x < digits) total[2 * threadIdx.x] = before;
  if (2 * threadIdx.x + 1 < digits) total[2 * threadIdx.x + 1] = before + a;
  __syncthreads();
}

// A block's pairs (id, row), in registers before anything else is done with them: one round trip to memory.  `pairs`
// NULL: the rows in their order.
__device__ __forceinline__ void load_pairs(const Rows& r, const uint2* pairs, uint32_t base, uint32_t n, int rounds,
                                           uint32_t (&key)[kRounds], uint32_t (&val)[kRounds]) {
#pragma unroll
  for (int j = 0; j < kRounds; ++j) {
    const uint32_t i = base + slot_of(j, rounds);
    const bool in = j < rounds && i < n;
    const uint2 p = !in ? make_uint2(0u, 0u) : pairs ? pairs[i] : make_uint2(row_id(r, i), i);
    key[j] = p.x;
    val[j] = p.y;
  }
}

// Up to kRounds pairs a thread: all passes in one block, the pairs in shared memory between them.
template <int THREADS>
struct Small {
  static constexpr int kMost = THREADS * kRounds;
  static constexpr size_t kSmem = (kMost + (THREADS / 32 + 1) * kMaxDigits) * sizeof(uint32_t) + kMost * sizeof(uint16_t);
};
constexpr int kSmallThreads = 1024;  // beyond kTile pairs (a gradient of 3000 tokens of 256 columns 49 us, 56 with the kernels below)

template <int THREADS>
__global__ void __launch_bounds__(THREADS, 1)
sort_small_kernel(Rows r, int passes, int bits, uint2* pairs) {
  extern __shared__ uint32_t smem[];
  uint32_t *skey = smem, *counts = smem + Small<THREADS>::kMost, *total = counts + THREADS / 32 * kMaxDigits;
  uint16_t* sval = reinterpret_cast<uint16_t*>(total + kMaxDigits);
  release_secondary();
  const uint32_t n = row_count(r);
  const int rounds = rounds_for<THREADS>(n);
  uint32_t key[kRounds], val[kRounds], rank[kRounds];
  load_pairs(r, nullptr, 0u, n, rounds, key, val);
  for (int p = 0; p < passes; ++p) {
    const Digit digit{p * bits, bits};
    warp_ranks<THREADS>(key, n, rounds, digit, counts, rank);
    across_warps<THREADS>(counts, total, digit.count());
    prefix_digits<THREADS>(total, digit.count());
    const bool last = p == passes - 1;
#pragma unroll
    for (int j = 0; j < kRounds; ++j) {
      if (j < rounds && slot_of(j, rounds) < n) {
        const int g = digit.of(key[j]);
        const uint32_t to = total[g] + counts[(threadIdx.x >> 5) * digit.count() + g] + rank[j];
        if (last) {
          pairs[to] = make_uint2(key[j], val[j]);
        } else {
          skey[to] = key[j];
          sval[to] = (uint16_t)val[j];
        }
      }
    }
    if (last) return;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kRounds; ++j) {
      const uint32_t i = slot_of(j, rounds);
      if (j < rounds && i < n) {
        key[j] = skey[i];
        val[j] = sval[i];
      }
    }
    __syncthreads();
  }
}

// How many pairs of each digit a block holds: hist [digits][blocks].
__global__ void __launch_bounds__(kThreads)
count_kernel(Rows r, const uint2* pairs, Digit digit, uint32_t* hist) {
  release_secondary();
  __shared__ uint32_t c[kMaxDigits];
  for (int g = threadIdx.x; g < digit.count(); g += kThreads) c[g] = 0u;
  __syncthreads();
  wait_for_primary();
  const uint32_t n = row_count(r), base = blockIdx.x * kTile;
  const int rounds = base < n ? rounds_for(n - base) : 0;
  uint32_t key[kRounds], val[kRounds];
  load_pairs(r, pairs, base, n, rounds, key, val);
#pragma unroll
  for (int j = 0; j < kRounds; ++j)
    if (j < rounds && base + slot_of(j, rounds) < n) atomicAdd(&c[digit.of(key[j])], 1u);
  __syncthreads();
  for (int g = threadIdx.x; g < digit.count(); g += kThreads) hist[(int64_t)g * gridDim.x + blockIdx.x] = c[g];
}

// hist[g][.] -> its exclusive prefix sums, total[g]; a warp a digit.
__global__ void __launch_bounds__(kThreads)
prefix_kernel(uint32_t* hist, int blocks, int digits, uint32_t* total) {
  release_secondary();
  wait_for_primary();
  const int g = blockIdx.x * kWarps + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (g >= digits) return;
  uint32_t before = 0u;
  for (int base = 0; base < blocks; base += 32) {
    const int i = base + lane;
    const uint32_t c = i < blocks ? hist[(int64_t)g * blocks + i] : 0u;
    uint32_t run = c;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t left = __shfl_up_sync(0xFFFFFFFFu, run, o);
      if (lane >= o) run += left;
    }
    if (i < blocks) hist[(int64_t)g * blocks + i] = before + run - c;
    before += __shfl_sync(0xFFFFFFFFu, run, 31);
  }
  if (lane == 0) total[g] = before;
}

__global__ void __launch_bounds__(kThreads)
scatter_kernel(Rows r, const uint2* pairs, Digit digit, const uint32_t* hist, const uint32_t* totals, uint2* out) {
  release_secondary();
  wait_for_primary();
  __shared__ uint32_t counts[kWarps * kMaxDigits], total[kMaxDigits];
  const uint32_t n = row_count(r), base = blockIdx.x * kTile;
  const int digits = digit.count();
  if (base >= n) return;
  const int rounds = rounds_for(n - base);
  uint32_t key[kRounds], val[kRounds], rank[kRounds];
  load_pairs(r, pairs, base, n, rounds, key, val);
  for (int g = threadIdx.x; g < digits; g += kThreads) total[g] = totals[g];
  warp_ranks(key, n - base, rounds, digit, counts, rank);
  prefix_digits(total, digits);
  // where the block's pairs of each digit, and those of each warp of it, begin
  for (int g = threadIdx.x; g < digits; g += kThreads) {
    uint32_t run = total[g] + hist[(int64_t)g * gridDim.x + blockIdx.x];
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const uint32_t c = counts[w * digits + g];
      counts[w * digits + g] = run;
      run += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kRounds; ++j) {
    if (j < rounds && base + slot_of(j, rounds) < n) {
      const uint32_t to = counts[(threadIdx.x >> 5) * digits + digit.of(key[j])] + rank[j];
      out[to] = make_uint2(key[j], val[j]);
    }
  }
}

// -------------------------------------------------------------------------- sums
struct SumArgs {
  Rows r;
  const uint2* pairs;           // (id, row), sorted
  const void* dx;
  float *dtable, *partial;      // partial [2 tiles][d]
  uint32_t* status;
  int d, tpr_log2, rows_per_block;
  int tiles;                    // blocks that add up pieces, before those that write rows of the table
  float scale;
  bool accumulate;
};

// First sorted position in [lo, hi) whose key is not below `key`, hi if there is none.
__device__ __forceinline__ uint32_t lower_bound(const uint2* pairs, uint32_t lo, uint32_t hi, uint32_t key) {
  while (lo < hi) {
    const uint32_t mid = (lo + hi) >> 1;
    if (pairs[mid].x < key) lo = mid + 1; else hi = mid;
  }
  return lo;
}
// The same by a whole warp, 32 probes at a time: four dependent loads where one lane would take eighteen.
__device__ __forceinline__ uint32_t warp_lower_bound(const uint2* pairs, uint32_t lo, uint32_t hi, uint32_t key) {
  while (lo < hi) {  // the answer is in [lo, hi]
    const uint32_t step = (hi - lo + 31) / 32, at = lo + ((threadIdx.x & 31) + 1) * step - 1;
    const unsigned not_below = __ballot_sync(0xFFFFFFFFu, at >= hi || pairs[at].x >= key);
    // lane f is the first not below: the answer is in its step; lanes past hi count as not below
    const uint32_t f = not_below ? __ffs(not_below) - 1 : 32;
    const uint32_t from = lo + f * step;
    hi = f == 32 ? hi : min(hi, from + step - 1);
    lo = min(from, hi);
  }
  return lo;
}

// Sum over the rows row_of(lo) .. row_of(hi - 1) of eight columns, in order, with several loads on their way at a time
// (the usual row of the table has a few tokens, and one after the other each would cost a round trip).  As many as four
// blocks a multiprocessor leave registers for: 166,001 bfloat16 rows of 4096, 732 us with four loads and four blocks, 677
// with six, 692 with four loads and five blocks, 781 with twelve and three.
template <typename T>
constexpr int kFlight = sizeof(T) == 2 ? 6 : 4;
constexpr int kSumBlocks = 4;

template <typename T, typename R>
__device__ __forceinline__ void add_tokens(const SumArgs& a, R row_of, uint32_t lo, uint32_t hi, int c, float2 (&sum)[kPairs]) {
  constexpr int F = kFlight<T>;
  const T* dx = (const T*)a.dx + c;
#pragma unroll
  for (int i = 0; i < kPairs; ++i) sum[i] = both(0.f);
  for (uint32_t i = lo; i < hi; i += F) {
    Raw<T> raw[F];
#pragma unroll
    for (int u = 0; u < F; ++u)
      if (i + u < hi) raw[u] = rows::load_raw(dx + (int64_t)row_of(i + u) * a.d);
#pragma unroll
    for (int u = 0; u < F; ++u) {
      if (i + u >= hi) break;
      float2 v[kPairs];
      rows::widen(raw[u], v);
#pragma unroll
      for (int j = 0; j < kPairs; ++j) sum[j] = add2(sum[j], v[j]);
    }
  }
}

// Rows of the table a block writes: 96 KB of them, between 24 and 128 (74,003 tokens, 1024 columns: 175 us with 16, 172 with
// 24 or 32; 166,001, 4096: 678, 680, 696; 40,000 tokens, 128 columns, V 152,000: 76 us with 24, 65 with 128; 9,000 tokens,
// 64 columns, V 1,000,000: 155, 90).
constexpr int kRowsPerBlock = 128, kFewestRows = 24, kBlockBytes = 96 * 1024;

// Blocks [0, tiles): the piece of a table row with more than kPiece tokens that lies in a tile of kPiece sorted
// positions.  A tile meets at most two such rows, one that began before it (slot 0) and one that begins in it and
// goes on behind it (slot 1).  The blocks behind: rows of the table with up to kPiece tokens, or, where there are no
// blocks for pieces, all.
template <typename T, bool PIECES>
__global__ void __launch_bounds__(kThreads, kSumBlocks) sum_kernel(SumArgs a) {
  release_secondary();
  wait_for_primary();
  __shared__ uint32_t start[kRowsPerBlock + 1];
  const uint32_t n = row_count(a.r);
  const int tpr = 1 << a.tpr_log2, group = threadIdx.x >> a.tpr_log2, groups = kThreads >> a.tpr_log2;
  const int first = (threadIdx.x & (tpr - 1)) * kChunk, stride = kChunk << a.tpr_log2;
  if (PIECES && blockIdx.x < (unsigned)a.tiles) {
    const uint32_t t0 = blockIdx.x * kPiece, t1 = min(t0 + kPiece, n);
    if (t0 >= n) return;
    // a row that goes on over an end of the tile has the same id on both sides of it; most tiles have none
    const uint32_t k0 = a.pairs[t0].x, k1 = a.pairs[t1 - 1].x;
    const bool from_before = t0 > 0 && k0 != (uint32_t)a.r.V && a.pairs[t0 - 1].x == k0;
    const bool goes_on = t1 < n && k1 != (uint32_t)a.r.V && a.pairs[t1].x == k1;
    if (!from_before && !goes_on) return;
    if (threadIdx.x < 128) {  // where the first and the last token's rows begin and end, a warp each
      const int warp = threadIdx.x >> 5;
      const uint32_t key = (warp < 2 ? k0 : k1) + (warp & 1);
      const uint32_t at = warp == 0 ? warp_lower_bound(a.pairs, 0u, t0, key)
                                    : warp_lower_bound(a.pairs, warp == 2 ? 0u : warp == 1 ? t0 : t1, warp == 2 ? t1 : n, key);
      if ((threadIdx.x & 31) == 0) start[warp] = at;
    }
    __syncthreads();
    auto row_of = [&](uint32_t i) { return a.pairs[i].y; };
    for (int s = group; s < 2; s += groups) {
      const uint32_t b = start[2 * s], e = start[2 * s + 1];
      if (e - b <= kPiece || !(s == 0 ? from_before : goes_on && b >= t0)) continue;
      for (int c = first; c < a.d; c += stride) {
        float2 sum[kPairs];
        add_tokens<T>(a, row_of, max(b, t0), min(e, t1), c, sum);
        Raw<float> out;
        rows::narrow(sum, out);
        rows::store_raw(a.partial + (2 * (int64_t)blockIdx.x + s) * a.d + c, out);
      }
    }
    return;
  }
  const int v0 = (blockIdx.x - a.tiles) * a.rows_per_block, count = min(a.rows_per_block, a.r.V - v0);
  // where the block's rows begin among the sorted tokens: its first and last by two warps, those between from the
  // tokens themselves where they are few
  __shared__ uint32_t ends[2], row_at[kThreads];
  if (threadIdx.x < 64) {
    const uint32_t at = warp_lower_bound(a.pairs, 0u, n, (uint32_t)(v0 + (threadIdx.x < 32 ? 0 : count)));
    if ((threadIdx.x & 31) == 0) ends[threadIdx.x >> 5] = at;
  }
  __syncthreads();
  const uint32_t lo0 = ends[0], hi0 = ends[1];
  const bool few = hi0 - lo0 <= kThreads;  // their tokens' rows fit into shared memory
  if (!few) {
    if (threadIdx.x <= count) start[threadIdx.x] = lower_bound(a.pairs, lo0, hi0, (uint32_t)(v0 + threadIdx.x));
  } else {
    // token i tells where the rows after its predecessor's, up to its own, begin; the end tells of the rest
    const uint32_t i = lo0 + threadIdx.x;
    if (i <= hi0) {
      const uint2 own = i < hi0 ? a.pairs[i] : make_uint2((uint32_t)(v0 + count), 0u);
      const int from = i == lo0 ? 0 : (int)a.pairs[i - 1].x - v0 + 1, to = (int)own.x - v0;
      row_at[threadIdx.x] = own.y;
      for (int v = from; v <= to; ++v) start[v] = i;
    }
    if (hi0 - lo0 == kThreads && threadIdx.x == 0)  // one more than there are threads
      for (int v = (int)a.pairs[hi0 - 1].x - v0 + 1; v <= count; ++v) start[v] = hi0;
  }
  if (v0 == 0 && threadIdx.x == 0) *a.status = n > 0 && a.pairs[n - 1].x == (uint32_t)a.r.V ? NAT_DEV_BAD_TARGET : 0u;
  __syncthreads();
  auto write_rows = [&](auto row_of) {
    for (int i = group; i < count; i += groups) {
      const uint32_t lo = start[i], hi = start[i + 1];
      if (hi - lo > kPiece || (a.accumulate && hi == lo)) continue;
      float* row = a.dtable + (int64_t)(v0 + i) * a.d;
      for (int c = first; c < a.d; c += stride) {
        float2 sum[kPairs];
        add_tokens<T>(a, row_of, lo, hi, c, sum);
        Raw<float> out;
        float2 old[kPairs];
        if (a.accumulate) rows::widen(rows::load_raw(row + c), old);
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
          sum[j] = mul2(sum[j], both(a.scale));
          if (a.accumulate) sum[j] = add2(old[j], sum[j]);
        }
        rows::narrow(sum, out);
        rows::store_raw(row + c, out);
      }
    }
  };
  if (few) write_rows([&](uint32_t i) { return row_at[i - lo0]; });
  else write_rows([&](uint32_t i) { return a.pairs[i].y; });
  if (PIECES || hi0 - lo0 <= kPiece) return;
  // without blocks for pieces: a row with more than kPiece tokens by the whole block, a run of them a group
  __shared__ float2 sums[PIECES ? 1 : kThreads][kPairs];
  for (int i = 0; i < count; ++i) {
    const uint32_t lo = start[i], hi = start[i + 1];
    if (hi - lo <= kPiece) continue;  // the same for all threads
    const uint32_t per = (hi - lo + groups - 1) / groups, from = min(lo + group * per, hi), to = min(from + per, hi);
    float* row = a.dtable + (int64_t)(v0 + i) * a.d;
    for (int base = 0; base < a.d; base += stride) {
      const int c = base + first;
      float2 sum[kPairs];
      if (c < a.d) add_tokens<T>(a, [&](uint32_t k) { return a.pairs[k].y; }, from, to, c, sum);
#pragma unroll
      for (int j = 0; j < kPairs; ++j) sums[threadIdx.x][j] = sum[j];
      __syncthreads();
      if (group == 0 && c < a.d) {
        float2 old[kPairs];
        if (a.accumulate) rows::widen(rows::load_raw(row + c), old);
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
          for (int g = 1; g < groups; ++g) sum[j] = add2(sum[j], sums[g * tpr + threadIdx.x][j]);
          sum[j] = mul2(sum[j], both(a.scale));
          if (a.accumulate) sum[j] = add2(old[j], sum[j]);
        }
        Raw<float> out;
        rows::narrow(sum, out);
        rows::store_raw(row + c, out);
      }
      __syncthreads();
    }
  }
}

// Joins the pieces of the rows that begin in one of the block's tiles and go on behind it: the warps take runs of
// pieces, 256 columns at a time, and their sums are added in the runs' order.
constexpr int kJoinTiles = kWarps;

__global__ void __launch_bounds__(kThreads) join_kernel(SumArgs a) {
  release_secondary();
  wait_for_primary();
  __shared__ float2 sums[kWarps][32][kPairs];
  __shared__ uint32_t bounds[kJoinTiles][2];
  const uint32_t n = row_count(a.r);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = (blockIdx.y * 32 + lane) * kChunk;
  {  // a tile a warp
    const uint32_t t0 = (blockIdx.x * kJoinTiles + warp) * kPiece, t1 = t0 + kPiece;
    uint32_t b = 0u, e = 0u;
    if (t1 < n) {
      const uint32_t key = a.pairs[t1 - 1].x, next = a.pairs[t1].x, before = t0 > 0 ? a.pairs[t0 - 1].x : (uint32_t)a.r.V;
      if (key != (uint32_t)a.r.V && next == key && before != key) {
        b = warp_lower_bound(a.pairs, t0, t1, key);
        e = warp_lower_bound(a.pairs, t1, n, key + 1);
      }
    }
    if (lane == 0) {
      bounds[warp][0] = b;
      bounds[warp][1] = e;
    }
  }
  __syncthreads();
  for (int i = 0; i < kJoinTiles; ++i) {
    const uint32_t b = bounds[i][0], e = bounds[i][1];
    if (e - b <= kPiece) continue;  // the same for all threads
    const uint32_t tile = blockIdx.x * kJoinTiles + i;
    const int pieces = (int)((e - 1) / kPiece - tile + 1);
    const int per = (pieces + kWarps - 1) / kWarps, lo = warp * per, hi = min(lo + per, pieces);
    float2 sum[kPairs];
#pragma unroll
    for (int j = 0; j < kPairs; ++j) sum[j] = both(0.f);
    if (c < a.d) {
#pragma unroll 4
      for (int p = lo; p < hi; ++p) {
        // the row's first piece is the second slot of its tile, the others the first slots of theirs
        const int64_t slot = 2 * ((int64_t)tile + p) + (p == 0 ? 1 : 0);
        float2 v[kPairs];
        rows::widen(rows::load_raw(a.partial + slot * a.d + c), v);
#pragma unroll
        for (int j = 0; j < kPairs; ++j) sum[j] = add2(sum[j], v[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < kPairs; ++j) sums[warp][lane][j] = sum[j];
    __syncthreads();
    if (warp == 0 && c < a.d) {
      float* at = a.dtable + (int64_t)a.pairs[b].x * a.d + c;
      float2 old[kPairs];
      if (a.accumulate) rows::widen(rows::load_raw(at), old);
      Raw<float> out;
#pragma unroll
      for (int j = 0; j < kPairs; ++j) {
        for (int w = 1; w < kWarps; ++w) sum[j] = add2(sum[j], sums[w][lane][j]);
        sum[j] = mul2(sum[j], both(a.scale));
        if (a.accumulate) sum[j] = add2(old[j], sum[j]);
      }
      rows::narrow(sum, out);
      rows::store_raw(at, out);
    }
    __syncthreads();
  }
}

// --------------------------------------------------------------------------- host
// Threads that share a row of d elements, as a power of two.
int threads_log2(int d) {
  int t = 0;
  while ((kChunk << t) < d && (1 << t) < kThreads) ++t;
  return t;
}

struct Layout {
  int passes, bits, blocks, tiles;
  size_t pairs[2], hist, total, partial, bytes;
};

Layout layout(const nat_embed_params& p, int64_t cap) {
  Layout l;
  int b = 1;
  while ((p.V >> b) != 0) ++b;  // ids 0..V, V for those outside
  l.passes = (b + 8) / 9;
  l.bits = (b + l.passes - 1) / l.passes;
  l.blocks = (int)((cap + kTile - 1) / kTile);
  // none where the groups of threads of a block that writes rows can share any row among them, kPiece tokens each at most:
  // 290 tokens of 64 columns 12.8 us with blocks for pieces, 10.2 without (a kernel of its own: in one with the other it
  // would cost the large ones 2 to 6 %)
  l.tiles = cap > kPiece * (kThreads >> threads_log2(p.d)) ? (int)((cap + kPiece - 1) / kPiece) : 0;
  size_t at = 256;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at = align_up(at + bytes, 256);
    return o;
  };
  for (int i = 0; i < 2; ++i) l.pairs[i] = take(sizeof(uint2) * (size_t)cap);
  l.hist = take(4 * (size_t)kMaxDigits * l.blocks);
  l.total = take(4 * kMaxDigits);
  l.partial = take(2 * (size_t)l.tiles * p.d * sizeof(float));
  l.bytes = at;
  return l;
}

int check(const char* who, const nat_embed_params* p, int64_t cap) {
  if (!p) return fail(NAT_ERR_INVALID_ARG, "%s: params is null", who);
  if (p->dtype != NAT_F32 && p->dtype != NAT_BF16)
    return fail(NAT_ERR_UNSUPPORTED, "%s: unknown dtype %d", who, p->dtype);
  if (p->V <= 0 || p->d <= 0 || cap < 0 || cap > 0x7FFFFFFFll)
    return fail(NAT_ERR_INVALID_ARG, "%s: V and d must be positive, cap in [0, 2^31)", who);
  if (p->d % kChunk != 0 || p->d > 65536 || p->V > (1 << 30))
    return fail(NAT_ERR_UNSUPPORTED, "%s: d must be a multiple of 8, at most 65536, and V at most 2^30 (d = %d, V = %d)",
                who, p->d, p->V);
  if (!(p->scale - p->scale == 0.f)) return fail(NAT_ERR_INVALID_ARG, "%s: scale must be finite", who);
  return NAT_OK;
}

int check_pointers(const char* who, std::initializer_list<const void*> needed, std::initializer_list<const void*> wide,
                   std::initializer_list<const void*> words) {
  for (const void* q : needed)
    if (!q) return fail(NAT_ERR_INVALID_ARG, "%s: null pointer", who);
  for (const void* q : wide)
    if ((uintptr_t)q & 15u) return fail(NAT_ERR_INVALID_ARG, "%s: matrices must be 16-byte aligned", who);
  for (const void* q : words)
    if ((uintptr_t)q & 3u) return fail(NAT_ERR_INVALID_ARG, "%s: ids, sel_idx and n_rows must be 4-byte aligned", who);
  return NAT_OK;
}

template <typename T>
int fwd(const nat_embed_params& p, const void* table, const Rows& r, void* x, cudaStream_t stream) {
  const int tpr_log2 = min(threads_log2(p.d), 5), rpb = kThreads >> tpr_log2;
  const unsigned blocks = (unsigned)((r.cap + rpb - 1) / rpb);
  if (p.scale == 1.f)
    lookup_kernel<T, true><<<blocks, kThreads, 0, stream>>>((const T*)table, r, (T*)x, p.d, tpr_log2, p.scale);
  else
    lookup_kernel<T, false><<<blocks, kThreads, 0, stream>>>((const T*)table, r, (T*)x, p.d, tpr_log2, p.scale);
  NAT_LAUNCH_CHECK("embed_lookup");
  return NAT_OK;
}

// Raises the larger small sort's shared-memory limit, once for each device.
int allow_smem() {
  static std::atomic<uint64_t> allowed{0};
  int dev = 0;
  NAT_CUDA(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return fail(NAT_ERR_UNSUPPORTED, "device index %d is beyond the 64 this library tracks", dev);
  if (!(allowed.load(std::memory_order_relaxed) >> dev & 1u)) {
    NAT_CUDA(cudaFuncSetAttribute(sort_small_kernel<kSmallThreads>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                  (int)Small<kSmallThreads>::kSmem));
    allowed.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  return NAT_OK;
}
static_assert(Small<kThreads>::kSmem <= 48 * 1024, "within the limit that needs no raising");

template <typename T>
int bwd(const nat_embed_params& p, const Rows& r, const void* dx, float* dtable, void* workspace, const Layout& l,
        cudaStream_t stream) {
  char* ws = (char*)workspace;
  auto at = [&](size_t o) { return reinterpret_cast<uint32_t*>(ws + o); };
  uint2* pairs[2] = {reinterpret_cast<uint2*>(ws + l.pairs[0]), reinterpret_cast<uint2*>(ws + l.pairs[1])};
  int src = 0, s;
  if (r.cap <= kTile) {
    sort_small_kernel<kThreads><<<1, kThreads, Small<kThreads>::kSmem, stream>>>(r, l.passes, l.bits, pairs[0]);
    NAT_LAUNCH_CHECK("embed_sort_small");
  } else if (r.cap <= Small<kSmallThreads>::kMost) {
    s = allow_smem();
    if (s != NAT_OK) return s;
    sort_small_kernel<kSmallThreads><<<1, kSmallThreads, Small<kSmallThreads>::kSmem, stream>>>(r, l.passes, l.bits, pairs[0]);
    NAT_LAUNCH_CHECK("embed_sort_small");
  } else {
    for (int pass = 0; pass < l.passes; ++pass) {
      const Digit digit{pass * l.bits, l.bits};
      const uint2* from = pass ? pairs[src] : nullptr;
      const int dst = pass ? src ^ 1 : 0;
      if (pass == 0) {  // behind whatever wrote the ids: not before that has ended
        count_kernel<<<l.blocks, kThreads, 0, stream>>>(r, from, digit, at(l.hist));
        NAT_LAUNCH_CHECK("embed_count");
      } else {
        s = launch_after(count_kernel, dim3(l.blocks), kThreads, 0, stream, "embed_count", r, from, digit, at(l.hist));
        if (s != NAT_OK) return s;
      }
      s = launch_after(prefix_kernel, dim3(((1 << l.bits) + kWarps - 1) / kWarps), kThreads, 0, stream, "embed_prefix",
                       at(l.hist), l.blocks, 1 << l.bits, at(l.total));
      if (s != NAT_OK) return s;
      s = launch_after(scatter_kernel, dim3(l.blocks), kThreads, 0, stream, "embed_scatter", r, from, digit,
                       (const uint32_t*)at(l.hist), (const uint32_t*)at(l.total), pairs[dst]);
      if (s != NAT_OK) return s;
      src = dst;
    }
  }
  SumArgs a{r, pairs[src], dx, dtable, (float*)(ws + l.partial), at(0), p.d, threads_log2(p.d), max(kFewestRows, min(kRowsPerBlock, kBlockBytes / (4 * p.d))),
            l.tiles, p.scale, p.accumulate != 0};
  while (a.rows_per_block > 1 && p.V / a.rows_per_block < 148 * 8) a.rows_per_block >>= 1;
  s = launch_after(l.tiles > 0 ? sum_kernel<T, true> : sum_kernel<T, false>, dim3((unsigned)(l.tiles + (p.V + a.rows_per_block - 1) / a.rows_per_block)), kThreads, 0,
                   stream, "embed_sum", a);
  if (s != NAT_OK) return s;
  if (l.tiles > 0) {
    s = launch_after(join_kernel, dim3((unsigned)((l.tiles + kJoinTiles - 1) / kJoinTiles), (unsigned)((p.d + 255) / 256)),
                     kThreads, 0, stream, "embed_join", a);
    if (s != NAT_OK) return s;
  }
  return NAT_OK;
}

}  // namespace
}  // namespace embed
}  // namespace nat

extern "C" {

size_t nat_embed_workspace_bytes(const nat_embed_params* p, int64_t cap) {
  if (nat::embed::check("nat_embed_workspace_bytes", p, cap) != NAT_OK) return 0;
  return nat::embed::layout(*p, cap).bytes;
}

int nat_embed_fwd(const nat_embed_params* p, const void* table, const int32_t* ids, const int32_t* sel_idx,
                  const int32_t* n_rows, int64_t cap, void* x, void* stream) {
  const char* who = "nat_embed_fwd";
  int s = nat::embed::check(who, p, cap);
  if (s != NAT_OK || cap == 0) return s;
  s = nat::embed::check_pointers(who, {table, ids, x}, {table, x}, {ids, sel_idx, n_rows});
  if (s != NAT_OK) return s;
  const nat::embed::Rows r{ids, sel_idx, n_rows, cap, p->V};
  return p->dtype == NAT_F32 ? nat::embed::fwd<float>(*p, table, r, x, (cudaStream_t)stream)
                             : nat::embed::fwd<__nv_bfloat16>(*p, table, r, x, (cudaStream_t)stream);
}

int nat_embed_bwd(const nat_embed_params* p, const int32_t* ids, const int32_t* sel_idx, const int32_t* n_rows,
                  int64_t cap, const void* dx, float* dtable, void* workspace, size_t workspace_bytes, void* stream) {
  const char* who = "nat_embed_bwd";
  int s = nat::embed::check(who, p, cap);
  if (s != NAT_OK) return s;
  s = cap > 0 ? nat::embed::check_pointers(who, {ids, dx, dtable}, {dx, dtable}, {ids, sel_idx, n_rows})
              : nat::embed::check_pointers(who, {dtable}, {dtable}, {n_rows});
  if (s != NAT_OK) return s;
  const nat::embed::Layout l = nat::embed::layout(*p, cap);
  if (!workspace || workspace_bytes < l.bytes)
    return nat::fail(NAT_ERR_CAPACITY, "%s: workspace too small (%zu < %zu)", who, workspace_bytes, l.bytes);
  if ((uintptr_t)workspace & 255u)
    return nat::fail(NAT_ERR_INVALID_ARG, "%s: workspace must be 256-byte aligned", who);
  const nat::embed::Rows r{ids, sel_idx, n_rows, cap, p->V};
  return p->dtype == NAT_F32 ? nat::embed::bwd<float>(*p, r, dx, dtable, workspace, l, (cudaStream_t)stream)
                             : nat::embed::bwd<__nv_bfloat16>(*p, r, dx, dtable, workspace, l, (cudaStream_t)stream);
}

}  // extern "C"
