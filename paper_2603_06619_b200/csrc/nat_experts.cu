// Entry points of the products grouped by expert: argument checks, workspace, the list of row tiles, and the sum of
// the parts of a weights' gradient.
#include "nat_experts.cuh"

#include "nat_rows.cuh"

namespace nat {
namespace experts {
namespace {

constexpr int kMaxExperts = 1024;
constexpr int kPlanThreads = 1024;
// The kernels' row numbers are of 32 bits, and they look up to a tile and some slices of the contraction past an expert's
// last row: with more rows than this the next tile's first would lie past 2^31, and the expert be taken to have none.
constexpr int64_t kMostRows = 0x7FFFFFFFll - 1023;

// The row tiles of all experts in their order, and the experts' order by falling number of rows (equal ones by
// number): the weights' gradient takes its tiles in that order, so that those in flight together are of about the
// same length and the shortest come last.
__global__ void __launch_bounds__(kPlanThreads)
plan_kernel(const int32_t* offsets, int E, int64_t cap, int tile_rows, Head* head, Tile* by_rows, Tile* tiles) {
  release_secondary();
  __shared__ int rows[kMaxExperts];
  __shared__ int sums[kPlanThreads / 32];
  const int e = threadIdx.x, lane = e & 31, warp = e >> 5;
  int lo = 0, hi = 0, fault = 0;
  if (e < E) {
    expert_rows(offsets, e, cap, lo, hi);
    fault = (int)offsets_fault(offsets, e, cap);
    rows[e] = hi - lo;
  }
  const bool broken = __syncthreads_or(fault & kBroken), any = __syncthreads_or(fault);
  const int count = (hi - lo + tile_rows - 1) / tile_rows;
  int run = count;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int left = __shfl_up_sync(0xFFFFFFFFu, run, o);
    if (lane >= o) run += left;
  }
  if (lane == 31) sums[warp] = run;
  __syncthreads();
  int first = run - count;
  for (int w = 0; w < warp; ++w) first += sums[w];
  if (e == kPlanThreads - 1) {
    head->tiles = broken ? 0u : (uint32_t)(first + count);
    head->broken = broken;
    head->status = any ? NAT_DEV_CAPACITY : 0u;
  }
  if (broken) return;
  for (int i = 0; i < count; ++i)
    tiles[first + i] = {e, lo + i * tile_rows, min(lo + (i + 1) * tile_rows, hi), 0};
  if (e < E) {
    int before = 0;
    for (int f = 0; f < E; ++f) before += rows[f] > rows[e] || (rows[f] == rows[e] && f < e);
    by_rows[before] = {e, lo, hi, 0};
  }
}

// dw (+)= the parts' sums: the warps take runs of parts, 256 elements at a time, and their sums are added in the runs' order
// (a thread for all parts of an element: 37,106 rows, 40 x 16, 289 parts, both gradients 92 us, 38 like this).
constexpr int kJoinWarps = 8;

__global__ void __launch_bounds__(kJoinWarps * 32)
join_kernel(const float* partial, int parts, int64_t size, const Head* head, bool accumulate, float* dw) {
  __shared__ float2 sums[kJoinWarps][32][rows::kPairs];
  if (head->broken) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int per = (parts + kJoinWarps - 1) / kJoinWarps, lo = min(warp * per, parts), hi = min(lo + per, parts);
  const int64_t step = (int64_t)gridDim.x * 32 * rows::kChunk;
  for (int64_t first = (int64_t)blockIdx.x * 32 * rows::kChunk; first < size; first += step) {
    const int64_t i = first + lane * rows::kChunk;
    float2 sum[rows::kPairs], v[rows::kPairs];
#pragma unroll
    for (int j = 0; j < rows::kPairs; ++j) sum[j] = both(0.f);
    if (i < size) {
#pragma unroll 4
      for (int p = lo; p < hi; ++p) {
        rows::widen(rows::load_raw(partial + p * size + i), v);
#pragma unroll
        for (int j = 0; j < rows::kPairs; ++j) sum[j] = add2(sum[j], v[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < rows::kPairs; ++j) sums[warp][lane][j] = sum[j];
    __syncthreads();
    if (warp == 0 && i < size) {
      if (accumulate) rows::widen(rows::load_raw(dw + i), v);
#pragma unroll
      for (int j = 0; j < rows::kPairs; ++j) {
        for (int w = 1; w < kJoinWarps; ++w) sum[j] = add2(sum[j], sums[w][lane][j]);
        if (accumulate) sum[j] = add2(v[j], sum[j]);
      }
      rows::Raw<float> out;
      rows::narrow(sum, out);
      rows::store_raw(dw + i, out);
    }
    __syncthreads();
  }
}

int check(const char* who, const nat_experts_params* p, int64_t cap) {
  if (!p) return fail(NAT_ERR_INVALID_ARG, "%s: params is null", who);
  if (p->dtype != NAT_F32 && p->dtype != NAT_BF16)
    return fail(NAT_ERR_UNSUPPORTED, "%s: unknown dtype %d", who, p->dtype);
  if (p->n_experts <= 0 || p->n_in <= 0 || p->n_out <= 0 || cap < 0 || cap > kMostRows)
    return fail(NAT_ERR_INVALID_ARG, "%s: n_experts, n_in and n_out must be positive, cap in [0, 2^31 - 1024]", who);
  if (p->n_experts > kMaxExperts || p->n_in % 8 != 0 || p->n_out % 8 != 0 || p->n_in > (1 << 20) ||
      p->n_out > (1 << 20) || (int64_t)p->n_in * p->n_out > (1ll << 31))
    return fail(NAT_ERR_UNSUPPORTED,
                "%s: at most 1024 experts; n_in and n_out multiples of 8, at most 2^20 and their product 2^31", who);
  const int64_t strides[2] = {p->x_stride, p->y_stride};
  for (int i = 0; i < 2; ++i) {
    if (strides[i] < (i == 0 ? p->n_in : p->n_out))
      return fail(NAT_ERR_INVALID_ARG, "%s: a row's stride (%lld) is shorter than the row", who, (long long)strides[i]);
    if (strides[i] % 8 != 0 || strides[i] >= (1ll << 31))
      return fail(NAT_ERR_UNSUPPORTED, "%s: strides must be multiples of 8 elements, below 2^31", who);
  }
  return NAT_OK;
}

int check_call(const char* who, const Args& a, size_t workspace_bytes, bool bwd, Layout* l) {
  if (!a.offsets) return fail(NAT_ERR_INVALID_ARG, "%s: offsets is null", who);
  // without rows the row matrices are not looked at
  if (a.cap > 0 && (((!bwd || a.dw) && !a.x) || ((!bwd || a.dx) && !a.w) || (bwd ? !a.dy : !a.y)))
    return fail(NAT_ERR_INVALID_ARG, "%s: null pointer", who);
  if (bwd && !a.dx && !a.dw) return fail(NAT_ERR_INVALID_ARG, "%s: neither dx nor dw", who);
  if (((uintptr_t)a.x | (uintptr_t)a.w | (uintptr_t)a.dy | (uintptr_t)a.y | (uintptr_t)a.dx | (uintptr_t)a.dw) & 15u)
    return fail(NAT_ERR_INVALID_ARG, "%s: matrices must be 16-byte aligned", who);
  if ((uintptr_t)a.offsets & 3u) return fail(NAT_ERR_INVALID_ARG, "%s: offsets must be 4-byte aligned", who);
  *l = layout(a.p, a.cap);
  if (!a.workspace || workspace_bytes < l->total)
    return fail(NAT_ERR_CAPACITY, "%s: workspace too small (%zu < %zu)", who, workspace_bytes, l->total);
  if ((uintptr_t)a.workspace & 255u)
    return fail(NAT_ERR_INVALID_ARG, "%s: workspace must be 256-byte aligned", who);
  return NAT_OK;
}

int product(const Args& a, const Layout& l, Product which) {
  return a.p.dtype == NAT_F32 ? f32_product(a, l, which) : bf16_product(a, l, which);
}

// Not for float32, nor for few experts, with rows: the blocks find their tiles and write the status word themselves.
int launch_plan(const Args& a, const Layout& l, int tile_rows) {
  if ((a.p.dtype == NAT_F32 || a.p.n_experts <= kOwnExperts) && a.cap > 0) return NAT_OK;
  plan_kernel<<<1, kPlanThreads, 0, a.stream>>>(a.offsets, a.p.n_experts, a.cap, tile_rows, head(a), by_rows(a, l),
                                                tiles(a, l));
  NAT_LAUNCH_CHECK("experts_plan");
  return NAT_OK;
}

}  // namespace

Layout layout(const nat_experts_params& p, int64_t cap) {
  Layout l;
  const bool f32 = p.dtype == NAT_F32;
  for (int i = 0; i < 3; ++i) l.tile_rows[i] = f32 ? f32_tile(p, (Product)i, cap) : bf16_tile_rows(p, (Product)i, cap);
  // Few tiles of the weights' gradient: their rows are cut into parts, of 512 rows (float32: 64) of an average expert at
  // least, whose sums take up to 40 MB.  One expert's parts are of one length, and as many as are held at a time; of
  // several experts one may have most of the rows, so there are up to four times as many.  us, as many as held / twice / four
  // times (float32: as many, of 128 rows at least / four times, of 64):
  //   one expert's 300,000 rows, 256 x 256          156, 171, 191
  //   4 experts, 245,491 rows, 560 x 16, uneven     369, 274, 236     6, 85,068, 432 x 16, uneven   152, 106, 96
  //   4, 100,000, 256 x 512, nearly even             92, 103, 103     15, 66,802, 24 x 912, even     74, 77, 82
  //   float32: 10, 61,655, 104 x 296                618, 325          80, 32,601, 48 x 136, uneven  450, 164
  //            2, 178,829, 8 x 16, even               82, 97
  const bool lone = p.n_experts == 1;
  const int64_t rows = l.tile_rows[kDw], cols = f32 ? rows : kBf16Cols;
  const int64_t units = p.n_experts * ((p.n_out + rows - 1) / rows) * ((p.n_in + cols - 1) / cols);
  const int64_t fit = (f32 ? (lone ? 296 : 1184) : (lone ? 74 : 296)) / units;
  const int64_t worth = cap / p.n_experts / (f32 ? (lone ? 128 : 64) : 512);
  const int64_t room = 40000000 / ((int64_t)p.n_experts * p.n_out * p.n_in * 4);
  l.parts = (int)max((int64_t)1, min(min(fit, worth), room));
  size_t at = 256;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at = align_up(at + bytes, 256);
    return o;
  };
  l.by_rows_off = take(sizeof(Tile) * p.n_experts);
  // room for as many tiles as the smallest ones would be, so that it grows with cap whatever the tiles' size; none where the
  // blocks find their tiles themselves
  l.tiles_off = take(f32 || p.n_experts <= kOwnExperts ? 0 : sizeof(Tile) * (size_t)most_tiles(p, cap, kFewestRows));
  l.partial_off = take(l.parts > 1 ? sizeof(float) * (size_t)l.parts * p.n_experts * p.n_out * p.n_in : 0);
  l.total = at;
  return l;
}

}  // namespace experts
}  // namespace nat

extern "C" {

size_t nat_experts_workspace_bytes(const nat_experts_params* p, int64_t cap) {
  if (nat::experts::check("nat_experts_workspace_bytes", p, cap) != NAT_OK) return 0;
  return nat::experts::layout(*p, cap).total;
}

int nat_experts_fwd(const nat_experts_params* p, const int32_t* offsets, int64_t cap, const void* x, const void* w,
                    void* y, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace nat::experts;
  const char* who = "nat_experts_fwd";
  int s = check(who, p, cap);
  if (s != NAT_OK) return s;
  Args a{};
  a.p = *p; a.offsets = offsets; a.cap = cap; a.x = x; a.w = w; a.y = y; a.workspace = workspace;
  a.stream = (cudaStream_t)stream;
  Layout l;
  s = check_call(who, a, workspace_bytes, false, &l);
  if (s != NAT_OK) return s;
  s = launch_plan(a, l, l.tile_rows[kFwd]);
  return s != NAT_OK || cap == 0 ? s : product(a, l, kFwd);
}

int nat_experts_bwd(const nat_experts_params* p, const int32_t* offsets, int64_t cap, const void* x, const void* w,
                    const void* dy, void* dx, float* dw, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace nat::experts;
  const char* who = "nat_experts_bwd";
  int s = check(who, p, cap);
  if (s != NAT_OK) return s;
  Args a{};
  a.p = *p; a.offsets = offsets; a.cap = cap; a.x = x; a.w = w; a.dy = dy; a.dx = dx; a.dw = dw;
  a.workspace = workspace; a.stream = (cudaStream_t)stream;
  Layout l;
  s = check_call(who, a, workspace_bytes, true, &l);
  if (s != NAT_OK) return s;
  s = launch_plan(a, l, l.tile_rows[kDx]);
  if (s == NAT_OK && dx && cap > 0) s = product(a, l, kDx);
  if (s != NAT_OK || !dw) return s;
  const int64_t size = (int64_t)p->n_experts * p->n_out * p->n_in;
  if (cap == 0) {
    if (!p->accumulate) NAT_CUDA(cudaMemsetAsync(dw, 0, size * sizeof(float), a.stream));
    return NAT_OK;
  }
  s = product(a, l, kDw);
  if (s != NAT_OK || l.parts == 1) return s;
  const int64_t want = (size / nat::rows::kChunk + 31) / 32;
  join_kernel<<<(unsigned)min(want, (int64_t)148 * 8), kJoinWarps * 32, 0, a.stream>>>(partial(a, l), l.parts, size, head(a),
                                                                          p->accumulate != 0, dw);
  NAT_LAUNCH_CHECK("experts_join");
  return NAT_OK;
}

}  // extern "C"
