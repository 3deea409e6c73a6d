// Entry points of the packed causal attention: argument checks, workspace, the plan kernel.
#include "nat_attn.cuh"

namespace nat {
namespace attn {
namespace {

constexpr int kBuckets = 1024;

struct PlanArgs {
  Batch batch;
  int span;     // tokens of a step
  int by_rest;  // the steps run from the tile to the sequence's end, not from its start to the tile
  int heads;    // key heads, which multiply the work
  int which;
  bool split;
  int64_t max_entries;
  Entry* list;
  Head* head;
};

constexpr int kMinPiece = 8;  // steps: a piece's start, its partial result and their join cost about two

// Lists the tiles of all sequences, longest work first: under a causal mask the tiles of a
// sequence cost 1, 2, ... tiles of keys (queries' plans) or as much in the opposite order (keys'
// plan), and blocks that take the list in turn finish together when the short ones come last.  Where
// tiles are few (`split`) the long ones are cut into equal pieces, so that the work of all heads makes about
// kSplitBlocks pieces.  A counting sort by steps; the order inside a bucket and the numbering of the slots
// are not fixed, which no result depends on.  Sequence bounds are clamped to [0, cap], so no list
// entry points outside the buffers whatever cu_seqlens holds.
__device__ __forceinline__ void plan(const PlanArgs& a) {
  const int32_t* cu = a.batch.cu;
  const int32_t B = a.batch.B;
  const int64_t cap = a.batch.cap;
  const int tile = a.batch.tile;
  __shared__ uint32_t bucket[kBuckets], warp_sum[32], next_slot;
  __shared__ unsigned long long work;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  bucket[threadIdx.x] = 0u;
  if (threadIdx.x == 0) {
    work = 0ull;
    next_slot = 0u;
  }
  int faults = 0;
  for (int i = threadIdx.x; i < B; i += blockDim.x) faults |= sequence_fault(cu, i, cap);
  const bool broken = __syncthreads_or(faults & kBroken), any = __syncthreads_or(faults);
  if (broken) {
    if (threadIdx.x == 0) {
      a.head->count[a.which] = 0u;
      a.head->status = NAT_DEV_CAPACITY;  // a call's plans find the same
    }
    return;
  }
  auto steps_of = [&](int lo, int hi, int t) {
    const int first = lo + t * tile;
    return a.by_rest ? (hi - first + a.span - 1) / a.span : (min(first + tile, hi) - lo + a.span - 1) / a.span;
  };
  // visit(lo, hi, t) for every tile t of every sequence
  auto for_tiles = [&](auto visit) {
    // all threads together where the sequences are few, a warp each where they are many
    const bool few = B <= 32;
    for (int i = few ? 0 : warp; i < B; i += few ? 1 : 32) {
      int lo, hi;
      sequence_bounds(cu, i, cap, lo, hi);
      const int tiles = (hi - lo + tile - 1) / tile;
      for (int t = few ? threadIdx.x : lane; t < tiles; t += few ? 1024 : 32) visit(lo, hi, t);
    }
  };
  int chunk = kAllSteps;
  if (a.split) {
    unsigned long long mine = 0ull;
    for_tiles([&](int lo, int hi, int t) { mine += steps_of(lo, hi, t); });
    if (mine) atomicAdd(&work, mine);
    __syncthreads();
    chunk = (int)max((unsigned long long)kMinPiece, (work * a.heads + kSplitBlocks - 1) / kSplitBlocks);
  }
  int shift = 0;
  while ((min((int)((cap + a.span - 1) / a.span), chunk) >> shift) >= kBuckets) ++shift;
  for (int pass = 0; pass < 2; ++pass) {
    for_tiles([&](int lo, int hi, int t) {
      const int steps = steps_of(lo, hi, t);
      int pieces = (steps - 1) / chunk + 1;
      const int per = (steps + pieces - 1) / pieces;
      pieces = (steps + per - 1) / per;
      uint32_t slot = 0u;
      if (pass == 1 && pieces > 1) slot = atomicAdd(&next_slot, (uint32_t)pieces);
      for (int p = 0; p < pieces; ++p) {
        const int begin = p * per, end = min(steps, begin + per);
        const uint32_t at = atomicAdd(&bucket[kBuckets - 1 - ((end - begin) >> shift)], 1u);
        if (pass == 1 && at < a.max_entries)  // always, as the bounds ascend
          a.list[at] = Entry{lo, hi, lo + t * tile, begin, end, (int32_t)slot, p, pieces};
      }
    });
    __syncthreads();
    if (pass == 0) {  // exclusive scan of the counts, costliest bucket first
      const uint32_t mine = bucket[threadIdx.x];
      uint32_t run = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t left = __shfl_up_sync(0xFFFFFFFFu, run, o);
        if (lane >= o) run += left;
      }
      if (lane == 31) warp_sum[warp] = run;
      __syncthreads();
      uint32_t before = 0u;
      for (int w = 0; w < warp; ++w) before += warp_sum[w];
      bucket[threadIdx.x] = before + run - mine;
      if (threadIdx.x == kBuckets - 1) {
        const uint32_t total = before + run;
        a.head->count[a.which] = total;
        a.head->status = any ? NAT_DEV_CAPACITY : 0u;
      }
      __syncthreads();
    }
  }
}

__global__ void __launch_bounds__(1024) plan_kernel(PlanArgs a) {
  release_secondary();
  plan(a);
}

// What the bfloat16 backward pass reads, in one launch: its plans (blocks 0 and 1, where it needs them)
// and, for every row of out, delta = dout . out and lse in units of log 2.  Bound by the read of
// out and dout.  (out is bfloat16: the sum of P dP would be free of its rounding, which dq and dk of the first few
// tokens of a sequence show, but takes the products S and dP of every tile once more.)  Half a warp takes a row's 16-byte pieces.
struct StatsArgs {
  const __nv_bfloat16 *out, *dout;
  const float* lse;
  float *lse2, *delta;
  int64_t o_stride;
  int n_heads, head_dim;
};

__global__ void __launch_bounds__(1024) bwd_prologue_kernel(PlanArgs a, PlanArgs b, StatsArgs s, unsigned plans) {
  release_secondary();
  if (blockIdx.x < plans) {
    plan(blockIdx.x == 0 ? a : b);
    return;
  }
  const int64_t rows = min((int64_t)max(a.batch.cu[a.batch.B], 0), a.batch.cap) * s.n_heads;
  const int lane = threadIdx.x & 15;
  const int64_t step = (int64_t)(gridDim.x - plans) * 64;
  // the bound is the block's: both halves of a warp take the same turns
  for (int64_t base = (int64_t)(blockIdx.x - plans) * 64; base < rows; base += step) {
    const int64_t row = base + (threadIdx.x >> 4);
    float dot = 0.f;
    if (row < rows && lane * 8 < s.head_dim) {
      const uint32_t token = (uint32_t)(row / s.n_heads), h = (uint32_t)(row - (int64_t)token * s.n_heads);
      const int64_t at = (int64_t)token * s.o_stride + (int64_t)h * s.head_dim + lane * 8;
      const uint4 x = __ldg(reinterpret_cast<const uint4*>(s.out + at));
      const uint4 y = __ldg(reinterpret_cast<const uint4*>(s.dout + at));
      const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        dot = fmaf(__uint_as_float(xs[i] << 16), __uint_as_float(ys[i] << 16), dot);
        dot = fmaf(__uint_as_float(xs[i] & 0xFFFF0000u), __uint_as_float(ys[i] & 0xFFFF0000u), dot);
      }
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) dot += __shfl_xor_sync(0xFFFFFFFFu, dot, o, 16);
    if (row < rows && lane == 0) {
      s.delta[row] = dot;
      s.lse2[row] = s.lse[row] * 1.4426950408889634f;
    }
  }
}

int check(const char* who, const nat_attn_params* p, int32_t B, int64_t cap) {
  if (!p) return fail(NAT_ERR_INVALID_ARG, "%s: params is null", who);
  if (p->dtype != NAT_F32 && p->dtype != NAT_BF16)
    return fail(NAT_ERR_UNSUPPORTED, "%s: unknown dtype %d", who, p->dtype);
  if (p->n_heads <= 0 || p->n_kv_heads <= 0 || p->head_dim <= 0 || B < 0 || cap < 0 ||
      cap > 0x7FFFFFFFll)
    return fail(NAT_ERR_INVALID_ARG, "%s: head counts and head_dim must be positive, B >= 0, cap in [0, 2^31)", who);
  if (p->n_heads % p->n_kv_heads != 0)
    return fail(NAT_ERR_INVALID_ARG, "%s: n_heads must be a multiple of n_kv_heads", who);
  if (p->head_dim % 8 != 0 || p->head_dim > 128)
    return fail(NAT_ERR_UNSUPPORTED, "%s: head_dim must be a multiple of 8, at most 128 (head_dim = %d)",
                who, p->head_dim);
  if (p->n_heads / p->n_kv_heads > 64 || p->n_heads > 65535)
    return fail(NAT_ERR_UNSUPPORTED, "%s: at most 64 query heads share a key head, and 65535 in all", who);
  if (!(p->scale - p->scale == 0.f)) return fail(NAT_ERR_INVALID_ARG, "%s: scale must be finite", who);
  const int64_t strides[4] = {p->q_stride, p->k_stride, p->v_stride, p->o_stride};
  for (int i = 0; i < 4; ++i) {
    const int64_t width = (int64_t)(i == 0 || i == 3 ? p->n_heads : p->n_kv_heads) * p->head_dim;
    if (strides[i] < width)
      return fail(NAT_ERR_INVALID_ARG, "%s: a token's row (stride %lld) is shorter than its heads (%lld)",
                  who, (long long)strides[i], (long long)width);
    if (strides[i] % 8 != 0 || strides[i] >= (1ll << 31))
      return fail(NAT_ERR_UNSUPPORTED, "%s: strides must be multiples of 8 elements, below 2^31", who);
  }
  return NAT_OK;
}

// Chooses the workspace's layout: tiles are cut into pieces where it has room for them.
int check_buffers(const char* who, const Args& a, size_t workspace_bytes, bool bwd, Layout* l) {
  if (!a.cu_seqlens || !a.q || !a.k || !a.v || !a.out || !a.lse)
    return fail(NAT_ERR_INVALID_ARG, "%s: null pointer", who);
  if (bwd && (!a.dout || !a.dq || !a.dk || !a.dv))
    return fail(NAT_ERR_INVALID_ARG, "%s: null gradient", who);
  const uintptr_t all = (uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v | (uintptr_t)a.out |
                        (uintptr_t)a.dout | (uintptr_t)a.dq | (uintptr_t)a.dk | (uintptr_t)a.dv;
  if (all & 15u) return fail(NAT_ERR_INVALID_ARG, "%s: rows must be 16-byte aligned", who);
  *l = layout(a.p, a.B, a.cap, true);
  if (workspace_bytes < l->total) *l = layout(a.p, a.B, a.cap, false);
  if (!a.workspace || workspace_bytes < l->total)
    return fail(NAT_ERR_CAPACITY, "%s: workspace too small (%zu < %zu)", who, workspace_bytes, l->total);
  if ((uintptr_t)a.workspace & 255u)
    return fail(NAT_ERR_INVALID_ARG, "%s: workspace must be 256-byte aligned", who);
  return NAT_OK;
}

}  // namespace

int plan_tile(const nat_attn_params& p, Plan which) {
  if (p.dtype == NAT_F32) return 64;
  const int tq = 128 / (p.n_heads / p.n_kv_heads);  // tokens of a tile with the group's heads folded in
  return which == kPlanFwd ? 2 * tq : which == kPlanDq ? tq : 128;
}

Layout layout(const nat_attn_params& p, int32_t B, int64_t cap, bool cut) {
  Layout l;
  size_t at = 256;
  int64_t pieces[3];
  for (int w = 0; w < 3; ++w) {
    // a sequence's last tile may be part full: at most one extra tile for each sequence
    const int64_t tiles = cap / plan_tile(p, (Plan)w) + B;
    // Few tiles (under two for each multiprocessor), each with many steps: cut into pieces.
    l.split[w] = cut && p.dtype == NAT_BF16 && cap > 1024 && tiles * p.n_kv_heads <= 2 * 148;
    pieces[w] = l.split[w] ? tiles + (kSplitBlocks + p.n_kv_heads - 1) / p.n_kv_heads : 0;
    l.entries[w] = l.split[w] ? pieces[w] : tiles;
    l.plan_off[w] = at;
    if (p.dtype == NAT_BF16) at = align_up(at + (size_t)l.entries[w] * sizeof(Entry), 256);
  }
  l.listed = p.dtype == NAT_F32 && (int64_t)B * p.n_heads > kSearchMost;
  if (l.listed) at = align_up(at + (size_t)l.entries[kPlanFwd] * sizeof(Entry), 256);
  l.delta_off = at;
  l.lse2_off = at = align_up(at + (size_t)cap * p.n_heads * sizeof(float), 256);
  if (p.dtype == NAT_BF16) at = align_up(at + (size_t)cap * p.n_heads * sizeof(float), 256);
  // the forward pass and the backward pass do not run together
  auto bytes = [&](Plan w) {
    return align_up((size_t)pieces[w] * p.n_kv_heads * partial_floats(p, w) * sizeof(float), 256);
  };
  l.partial_off[kPlanFwd] = l.partial_off[kPlanDq] = at;
  l.partial_off[kPlanDkv] = at + bytes(kPlanDq);
  l.total = at + max(bytes(kPlanFwd), bytes(kPlanDq) + bytes(kPlanDkv));
  return l;
}

Batch batch(const Args& a, const Layout& l, Plan which) {
  return {a.cu_seqlens, a.B, plan_tile(a.p, which), a.cap};
}

namespace {
PlanArgs plan_args(const Args& a, const Layout& l, Plan which) {
  return {batch(a, l, which),
          which == kPlanDkv ? plan_tile(a.p, kPlanDq) : 128,
          which == kPlanDkv ? 1 : 0,
          a.p.n_kv_heads,
          (int)which,
          l.split[which],
          l.entries[which],
          entries(a, l, which),
          head(a)};
}
}  // namespace

int launch_plan(const Args& a, const Layout& l, Plan which) {
  plan_kernel<<<1, 1024, 0, a.stream>>>(plan_args(a, l, which));
  NAT_LAUNCH_CHECK("plan_kernel");
  return NAT_OK;
}

int launch_bwd_prologue(const Args& a, const Layout& l, bool plans) {
  const StatsArgs s{(const __nv_bfloat16*)a.out, (const __nv_bfloat16*)a.dout, a.lse, lse2(a, l),
                    delta(a, l), a.p.o_stride, a.p.n_heads, a.p.head_dim};
  const int64_t want = (a.cap * a.p.n_heads + 63) / 64;
  const unsigned first = plans ? 2 : 0, blocks = first + (unsigned)min(want, (int64_t)148 * 2 * 4);
  bwd_prologue_kernel<<<blocks, 1024, 0, a.stream>>>(plan_args(a, l, kPlanDq), plan_args(a, l, kPlanDkv), s, first);
  NAT_LAUNCH_CHECK("bwd_prologue_kernel");
  return NAT_OK;
}

int device(Device* d) {
  static std::atomic<int> sms[64];  // 0: not asked yet
  NAT_CUDA(cudaGetDevice(&d->index));
  if (d->index < 0 || d->index >= 64)
    return fail(NAT_ERR_UNSUPPORTED, "device index %d is beyond the 64 this library tracks", d->index);
  d->sms = sms[d->index].load(std::memory_order_relaxed);
  if (d->sms == 0) {
    const int s = require_sm100();
    if (s != NAT_OK) return s;
    NAT_CUDA(cudaDeviceGetAttribute(&d->sms, cudaDevAttrMultiProcessorCount, d->index));
    sms[d->index].store(d->sms, std::memory_order_relaxed);
  }
  return NAT_OK;
}

}  // namespace attn
}  // namespace nat

extern "C" {

size_t nat_attn_workspace_bytes(const nat_attn_params* p, int32_t B, int64_t cap) {
  if (nat::attn::check("nat_attn_workspace_bytes", p, B, cap) != NAT_OK) return 0;
  return nat::attn::layout(*p, B, cap, true).total;
}

int nat_attn_fwd(const nat_attn_params* p, int32_t B, const int32_t* cu_seqlens, int64_t cap,
                 const void* q, const void* k, const void* v, void* out, float* lse,
                 void* workspace, size_t workspace_bytes, void* stream) {
  int s = nat::attn::check("nat_attn_fwd", p, B, cap);
  if (s != NAT_OK || B == 0 || cap == 0) return s;
  nat::attn::Args a{};
  a.p = *p; a.B = B; a.cu_seqlens = cu_seqlens; a.cap = cap; a.q = q; a.k = k; a.v = v;
  a.out = out; a.lse = lse; a.workspace = workspace; a.stream = (cudaStream_t)stream;
  nat::attn::Layout l;
  s = nat::attn::check_buffers("nat_attn_fwd", a, workspace_bytes, false, &l);
  if (s != NAT_OK) return s;
  return p->dtype == NAT_F32 ? nat::attn::f32_fwd(a, l) : nat::attn::bf16_fwd(a, l);
}

int nat_attn_bwd(const nat_attn_params* p, int32_t B, const int32_t* cu_seqlens, int64_t cap,
                 const void* q, const void* k, const void* v, const void* out, const float* lse,
                 const void* dout, void* dq, void* dk, void* dv, void* workspace,
                 size_t workspace_bytes, void* stream) {
  int s = nat::attn::check("nat_attn_bwd", p, B, cap);
  if (s != NAT_OK || B == 0 || cap == 0) return s;
  nat::attn::Args a{};
  a.p = *p; a.B = B; a.cu_seqlens = cu_seqlens; a.cap = cap; a.q = q; a.k = k; a.v = v;
  a.out = const_cast<void*>(out); a.lse = const_cast<float*>(lse); a.dout = dout; a.dq = dq;
  a.dk = dk; a.dv = dv; a.workspace = workspace; a.stream = (cudaStream_t)stream;
  nat::attn::Layout l;
  s = nat::attn::check_buffers("nat_attn_bwd", a, workspace_bytes, true, &l);
  if (s != NAT_OK) return s;
  return p->dtype == NAT_F32 ? nat::attn::f32_bwd(a, l) : nat::attn::bf16_bwd(a, l);
}

}  // extern "C"
