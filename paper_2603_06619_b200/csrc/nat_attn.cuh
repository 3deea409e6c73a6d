// Shared parts of the packed causal attention: arguments, workspace layout and the plan that
// deals the tiles of the packed sequences to the blocks.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
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

// Head of the workspace.  `status` is first, where nat_poll_status reads it.
struct Head {
  uint32_t status;
  uint32_t count[3];  // entries of the forward, dq and dkv plans
};

// One tile of `tile` tokens starting at `lo`, of the sequence that holds rows [seq_lo, seq_hi).
struct Entry {
  int32_t seq_lo, seq_hi, lo, pad;
};

enum Plan { kPlanFwd = 0, kPlanDq = 1, kPlanDkv = 2 };

// Tokens of a tile of each plan, for the head layout and type of `p`.
int plan_tile(const nat_attn_params& p, Plan which);

struct Layout {
  size_t plan_off[3], delta_off, lse2_off, total;
  int64_t entries[3];
};
Layout layout(const nat_attn_params& p, int32_t B, int64_t cap);

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

// Writes the plan of `which` and the status word.
int launch_plan(const Args& a, const Layout& l, Plan which);
// Both plans of the bfloat16 backward pass, delta and lse2.
int launch_bwd_prologue(const Args& a, const Layout& l);

int f32_fwd(const Args& a, const Layout& l);
int f32_bwd(const Args& a, const Layout& l);
int bf16_fwd(const Args& a, const Layout& l);
int bf16_bwd(const Args& a, const Layout& l);

}  // namespace attn
}  // namespace nat
