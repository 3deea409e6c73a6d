// Shared parts of the products grouped by expert: arguments, workspace layout, the list of row tiles.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "nat_common.cuh"

namespace nat {
namespace experts {

struct Args {
  nat_experts_params p;
  const int32_t* offsets;
  int64_t cap;
  const void *x, *w, *dy;
  void *y, *dx;
  float* dw;
  void* workspace;
  cudaStream_t stream;
};

enum Product { kFwd = 0, kDx = 1, kDw = 2 };

// Head of the workspace.  `status` is first, where nat_poll_status reads it.
struct Head {
  uint32_t status;
  uint32_t tiles;   // entries of the list
  uint32_t broken;  // offsets that do not ascend: nothing is computed
};

// Rows [lo, hi) of one expert, at most a tile's number.
struct Tile {
  int32_t expert, lo, hi, spare;
};

// Rows of expert e, clamped to [0, cap] whatever the offsets hold.
__device__ __forceinline__ void expert_rows(const int32_t* offsets, int e, int64_t cap, int& lo, int& hi) {
  lo = (int)min((int64_t)max(offsets[e], 0), cap);
  hi = (int)min((int64_t)max(offsets[e + 1], 0), cap);
  if (hi < lo) hi = lo;
}

// What a call finds wrong with the offsets of expert e: kTooMany, more rows than the matrices hold (the surplus is left
// out), or kBroken, offsets that do not ascend (nothing is computed).
enum { kTooMany = 1, kBroken = 2 };
__device__ __forceinline__ unsigned offsets_fault(const int32_t* offsets, int e, int64_t cap) {
  const int a = offsets[e], b = offsets[e + 1];
  return (a < 0 || b < a ? kBroken : 0) | ((int64_t)b > cap ? kTooMany : 0);
}

struct Layout {
  int tile_rows[3];           // of a tile, for each product: the rows' tiles (kFwd, kDx), or the weights' (kDw)
  int parts;                  // into which the rows are cut for the weights' gradient
  size_t by_rows_off, tiles_off, partial_off, total;
};
Layout layout(const nat_experts_params& p, int64_t cap);

inline Head* head(const Args& a) { return reinterpret_cast<Head*>(a.workspace); }
// All rows of each expert, by falling number.
inline Tile* by_rows(const Args& a, const Layout& l) {
  return reinterpret_cast<Tile*>((char*)a.workspace + l.by_rows_off);
}
inline Tile* tiles(const Args& a, const Layout& l) { return reinterpret_cast<Tile*>((char*)a.workspace + l.tiles_off); }
inline float* partial(const Args& a, const Layout& l) {
  return reinterpret_cast<float*>((char*)a.workspace + l.partial_off);
}

// Experts up to which the blocks (bfloat16) find their tiles themselves, in place of a kernel in front that lists them: 300
// rows over 4 experts forward 10.2 -> 7.3 us, 9,400 rows of one 21.5 -> 17.9, 200 over 32 (4096 x 1536) 68.6 -> 66.6.
constexpr int kOwnExperts = 64;
constexpr int kBf16Cols = 256;  // columns of a tile (float32: as many as rows)

// Rows of the k-blocks [lo, hi) that part `part` of `parts` takes of `blocks`.
__host__ __device__ inline void part_range(int blocks, int part, int parts, int& lo, int& hi) {
  const int per = (blocks + parts - 1) / parts;
  lo = part * per < blocks ? part * per : blocks;
  hi = lo + per < blocks ? lo + per : blocks;
}

// Row tiles of a call at most: an expert's last one may be part full.
inline int64_t most_tiles(const nat_experts_params& p, int64_t cap, int tile_rows) { return cap / tile_rows + p.n_experts; }
constexpr int kFewestRows = 64;  // of a row tile

// Rows of a tile of the kernel that `which` of a call takes.
int bf16_tile_rows(const nat_experts_params& p, Product which, int64_t cap);
int f32_tile(const nat_experts_params& p, Product which, int64_t cap);
int bf16_product(const Args& a, const Layout& l, Product which);
int f32_product(const Args& a, const Layout& l, Product which);

}  // namespace experts
}  // namespace nat
