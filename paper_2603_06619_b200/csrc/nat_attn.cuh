// Shared parts of the packed causal attention: arguments, workspace layout and the plan that
// deals the tiles of the packed sequences to the blocks.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <atomic>
#include <cstdint>

#include "nat_common.cuh"

namespace nat {
namespace attn {

struct Args {
  nat_attn_params p;
  int32_t B;
  const int32_t* cu_seqlens;
  int64_t cap;
  const void *q, *k, *v;
  void* out;
  float* lse;
  const void* dout;
  void *dq, *dk, *dv;
  void* workspace;
  cudaStream_t stream;
};

// Sequence i of a batch, clamped to [0, cap] whatever cu_seqlens holds.
__device__ __forceinline__ void sequence_bounds(const int32_t* cu, int i, int64_t cap, int& lo, int& hi) {
  lo = (int)min((int64_t)max(__ldg(cu + i), 0), cap);
  hi = (int)min((int64_t)max(__ldg(cu + i + 1), 0), cap);
  if (hi < lo) hi = lo;
}

// Head of the workspace.  `status` is first, where nat_poll_status reads it.
struct Head {
  uint32_t status;
  uint32_t count[3];  // entries of the forward, dq and dkv plans
};

// One tile of tokens starting at `lo`, of the sequence that holds rows [seq_lo, seq_hi), and the steps
// [begin, end) of its long axis (keys, or queries in the keys' part).  A tile in several pieces leaves
// partial results in slots [slot, slot + pieces), which a kernel behind joins in that order.
struct Entry {
  int32_t seq_lo, seq_hi, lo, begin, end, slot, piece, pieces;
};
constexpr int32_t kAllSteps = 0x7FFFFFFF;

// The batch itself, for kernels that find their tile without a list.
struct Batch {
  const int32_t* cu;
  int32_t B;
  int tile;
  int64_t cap;
};

// What a call finds wrong with sequence i: kTooLong, more rows than the buffers hold (the surplus is left
// out), or kBroken, bounds that do not ascend (nothing is computed).
enum { kTooLong = 1, kBroken = 2 };
__device__ __forceinline__ int sequence_fault(const int32_t* cu, int i, int64_t cap) {
  const int lo = __ldg(cu + i), hi = __ldg(cu + i + 1);
  return (lo < 0 || hi < lo ? kBroken : 0) | ((int64_t)hi > cap ? kTooLong : 0);
}

// Tile number `index` of all tiles in the sequences' order (for one warp; the same in every lane), and how
// many there are.  Where there are no more tiles than blocks their order does not matter, and the
// search, a few hundred cycles for every 32 sequences, is cheaper than a kernel that sorts them.
__device__ __forceinline__ Entry find_entry(const Batch& b, uint32_t index, uint32_t* total, uint32_t* status) {
  const int lane = threadIdx.x & 31;
  uint32_t before = 0u;
  Entry found{0, 0, 0, 0, kAllSteps, 0, 0, 1};
  unsigned faults = 0u;
  for (int base = 0; base < b.B; base += 32) {
    int lo = 0, hi = 0;
    int fault = 0;
    if (base + lane < b.B) {
      sequence_bounds(b.cu, base + lane, b.cap, lo, hi);
      fault = sequence_fault(b.cu, base + lane, b.cap);
    }
    faults |= __reduce_or_sync(0xFFFFFFFFu, (unsigned)fault);
    const uint32_t tiles = (uint32_t)((hi - lo + b.tile - 1) / b.tile);
    uint32_t run = tiles;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t left = __shfl_up_sync(0xFFFFFFFFu, run, o);
      if (lane >= o) run += left;
    }
    const uint32_t first = before + run - tiles;
    const bool mine = index >= first && index < first + tiles;
    const uint32_t who = __ballot_sync(0xFFFFFFFFu, mine);
    if (who) {
      const int from = __ffs(who) - 1;
      found.seq_lo = __shfl_sync(0xFFFFFFFFu, lo, from);
      found.seq_hi = __shfl_sync(0xFFFFFFFFu, hi, from);
      found.lo = found.seq_lo + (int)(index - __shfl_sync(0xFFFFFFFFu, first, from)) * b.tile;
    }
    before += __shfl_sync(0xFFFFFFFFu, run, 31);
  }
  *status = faults ? NAT_DEV_CAPACITY : 0u;
  *total = (faults & kBroken) ? 0u : before;
  return found;
}

enum Plan { kPlanFwd = 0, kPlanDq = 1, kPlanDkv = 2 };

// Tokens of a tile of each plan, for the head layout and type of `p`.
int plan_tile(const nat_attn_params& p, Plan which);

struct Layout {
  size_t plan_off[3], delta_off, lse2_off, partial_off[3], total;
  int64_t entries[3];  // of the list
  bool split[3];       // tiles may be cut into pieces
  bool listed;         // float32: the tiles come from a list
};

// Sequences times heads up to which every block of a float32 call searches cu_seqlens for its tile.  The search
// takes 32 sequences a turn in every block, so its cost grows with their square; beyond this a list is made
// first, in a launch of its own.  Forward, searching / listed: 2 heads of 64 columns, 4 tokens a sequence: 512
// sequences 59 / 79 us, 1024 141 / 145, 65,536 310,000 / 8,600; 8 heads of 128 columns, 64 tokens: 128 sequences
// 94 / 93, 256 217 / 182, 512 550 / 356; 16 heads of 128 columns, 4 tokens: 64 sequences 73 / 79, 256 327 / 288.
constexpr int64_t kSearchMost = 2048;

// Floats of one piece's partial result for one key head.
inline size_t partial_floats(const nat_attn_params& p, Plan which) {
  const size_t dp = p.head_dim <= 64 ? 64 : 128;
  return which == kPlanFwd ? 256 * (dp + 2) : which == kPlanDq ? 128 * dp : 128 * 2 * dp;
}
// The workspace of a call.  `cut`: with room for the pieces, where the tiles of this B and cap are worth cutting;
// without it the size grows with B and cap, so a workspace for some batch holds every smaller one uncut.
Layout layout(const nat_attn_params& p, int32_t B, int64_t cap, bool cut);

// Pieces that the splitting of tiles aims at: one and a half for each of the 148 multiprocessors, so that the
// shorter ones fill the gaps behind the longer (7013 tokens, 4 heads over 2: forward 89 us with 148
// pieces, 76 with 222, 84 with 296; backward 173, 169, 185).
constexpr int kSplitBlocks = 222;

inline Entry* entries(const Args& a, const Layout& l, Plan which) {
  return reinterpret_cast<Entry*>((char*)a.workspace + l.plan_off[which]);
}
inline Head* head(const Args& a) { return reinterpret_cast<Head*>(a.workspace); }
inline float* delta(const Args& a, const Layout& l) {
  return reinterpret_cast<float*>((char*)a.workspace + l.delta_off);
}

inline float* lse2(const Args& a, const Layout& l) {
  return reinterpret_cast<float*>((char*)a.workspace + l.lse2_off);
}

inline float* partials(const Args& a, const Layout& l, Plan which) {
  return reinterpret_cast<float*>((char*)a.workspace + l.partial_off[which]);
}

// Writes the plan of `which` and the status word.
int launch_plan(const Args& a, const Layout& l, Plan which);
// delta and lse2 of the bfloat16 backward pass, and (with `plans`) both its plans.
int launch_bwd_prologue(const Args& a, const Layout& l, bool plans);

Batch batch(const Args& a, const Layout& l, Plan which);

// Facts of the current device, asked for once.
struct Device {
  int index, sms;
};
int device(Device* d);

// Raises a kernel's shared-memory limit, once for each device.
template <typename K>
int allow_smem(K kernel, size_t smem, const Device& d, std::atomic<uint64_t>* devices) {
  if (devices->load(std::memory_order_relaxed) >> d.index & 1u) return NAT_OK;
  NAT_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  devices->fetch_or(1ull << d.index, std::memory_order_relaxed);
  return NAT_OK;
}

int f32_fwd(const Args& a, const Layout& l);
int f32_bwd(const Args& a, const Layout& l);
int bf16_fwd(const Args& a, const Layout& l);
int bf16_bwd(const Args& a, const Layout& l);

}  // namespace attn
}  // namespace nat
