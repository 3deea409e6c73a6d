// Products grouped by expert on the tensor cores (tcgen05 + TMEM + TMA).
//
//   kFwd  y  = x w_e^T     (rows x n_out,  contraction n_in)    x and w_e contiguous along it
//   kDx   dx = dy w_e      (rows x n_in,   contraction n_out)   w_e contiguous across it
//   kDw   dw_e = dy^T x    (n_out x n_in,  contraction rows)    both contiguous across it
//
// Persistent CTA pairs: the even CTA issues MMAs of M = 256, N = 256 (cta_group::2), each CTA loads its half of A and of B
// for each stage and drains its own rows of the two accumulators.  Warp 0 loads by TMA, warp 1 issues, four warps (eight
// where sums go to registers: kDw, and long contractions) write out.  Every wait is bounded and raises NAT_DEV_TIMEOUT.
//
// Ragged ends.  A tile's rows behind its expert's last belong to another expert or to none: they give rows of the
// accumulator that nobody writes out.  Columns behind n_in or n_out, and another expert's weights, lie outside the
// tensor maps (the weights' has a dimension for the expert) and are read as zeros.  For kDw the rows are the
// contraction, and a row too many would be added in: where an expert's last block of 64 rows is not full, the loading
// warp of each CTA waits for its own part of it, writes zeros over the rows behind (both operands': a weight of zero
// would not hide an infinity), and the odd CTA tells the even one before the MMA warp is let on.
#include <atomic>
#include <type_traits>

#include "nat_elect.cuh"
#include "nat_experts.cuh"
#include "nat_rows.cuh"
#include "nat_tc.cuh"

namespace nat {
namespace experts {
namespace {

constexpr int BM = 128, BK = 64, BN = kBf16Cols;
constexpr int kBox = 64 * 64 * 2;  // bytes of a 64 x 64 box of an operand that is contiguous across the contraction
constexpr int kTmemCols = 512;
// Blocks of the contraction (64 terms each) that an accumulator takes at most (kDw; kFwd and kDx where LONG): the tensor
// cores cut off what they add (toward zero, about half a step of 2^-23 each time), so after that many the sum goes to
// registers, where it is added to those before, rounded to nearest, and is begun anew in the other accumulator.  Relative
// error of a gradient of up to 17,389 rows an expert: 4.6e-7 with 8, 9.0e-7 with 16, 8.2e-6 with whole sums (plain float32
// 3.8e-7).  300,013 rows take the same time with 8 and 16, 2 % less with 32.  kFwd and kDx, whose result is rounded to
// bfloat16 anyway, take less with 16 (200 rows over 32 experts, 4096 terms, 67 us; with 8 75).
template <int WHICH>
constexpr int kSegment = WHICH == kDw ? 8 : 16;
constexpr int kGroup = 8;  // row tiles that go through the columns together

// ROWS: of a tile.  LONG (kFwd, kDx): a contraction whose sum goes to registers every kSegment blocks.  Shared memory:
// stages of A and half of B, and a piece of finished rows for each warp that writes out, from which it leaves by TMA.
template <int WHICH, int ROWS, bool LONG>
struct Ring {
  static constexpr int kABytes = ROWS / 2 * BK * 2, kBBytes = (BN / 2) * BK * 2;
  static constexpr int kPer = ROWS < 2 * BM ? 2 : 1;  // blocks of the contraction in a stage
  static constexpr int kBlock = kABytes + kBBytes, kStage = kPer * kBlock;
  static constexpr bool kSums = WHICH == kDw || LONG;    // in registers
  static constexpr int kWriters = kSums ? 8 : 4;         // warps that write out
  // of finished rows: 32 x 64 of bfloat16 or 32 x 32 of float; 32 x 32 of bfloat16 where all tiles are turned
  static constexpr int kPiece = LONG && ROWS < 2 * BM ? 2048 : 4096;
  static constexpr int kStaging = kWriters * kPiece;
  static constexpr int kBarriers = 512;
  static constexpr int kNum = (226 * 1024 - 1024 - kBarriers - kStaging) / kStage;
  static_assert((3 * kNum + 5) * 8 + 8 <= kBarriers, "barriers, tensor memory's address and the abort flag");
  static constexpr int kThreads = 64 + 32 * kWriters;
  static constexpr size_t kSmem = (size_t)kNum * kStage + kStaging + 1024 /*alignment*/ + kBarriers;
};

struct TcArgs {
  Head* head;
  const Tile* tiles;           // row tiles (kFwd, kDx), or the experts by falling number of rows (kDw)
  int E, n_cols, k_blocks;     // columns of the result; blocks of the contraction (kFwd, kDx)
  int m_tiles;                 // kDw: tiles along n_out
  int parts;
  bool accumulate;
  bool merged;                 // kDw: both operands' columns are whole blocks of 64, loaded two at a time
  __nv_bfloat16* rows_out;     // kFwd, kDx
  int64_t rows_stride;
  const int32_t* offsets;      // with few experts: the blocks find the tiles themselves
  int64_t cap;
  bool tells;                  // the first product of a call, whose block 0 writes the status word then
};

// Where each expert's row tiles begin, and its rows; the experts by falling number of rows, equal ones by number (kDw).
struct Own {
  int first[kOwnExperts + 1], lo[kOwnExperts], hi[kOwnExperts], order[kOwnExperts];
  bool broken;
};
// By one warp.
template <int WHICH, int ROWS>
__device__ __forceinline__ void find_tiles(const TcArgs& a, Own& own) {
  const int lane = threadIdx.x & 31;
  int before = 0;
  unsigned faults = 0u;
  for (int base = 0; base < a.E; base += 32) {
    const int e = base + lane;
    int lo = 0, hi = 0;
    unsigned fault = 0u;
    if (e < a.E) {
      expert_rows(a.offsets, e, a.cap, lo, hi);
      fault = offsets_fault(a.offsets, e, a.cap);
      own.lo[e] = lo;
      own.hi[e] = hi;
    }
    faults |= __reduce_or_sync(0xFFFFFFFFu, fault);
    const int count = (hi - lo + ROWS - 1) / ROWS;
    int run = count;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int left = __shfl_up_sync(0xFFFFFFFFu, run, o);
      if (lane >= o) run += left;
    }
    if (e < a.E) own.first[e] = before + run - count;
    before += __shfl_sync(0xFFFFFFFFu, run, 31);
  }
  if (lane == 0) {
    own.first[a.E] = (faults & kBroken) ? 0 : before;
    own.broken = (faults & kBroken) != 0;
    if (a.tells && blockIdx.x == 0) {
      a.head->status = faults ? NAT_DEV_CAPACITY : 0u;
      a.head->broken = own.broken;
    }
  }
  if (WHICH == kDw) {
    __syncwarp();
    for (int e = lane; e < a.E; e += 32) {
      const int rows = own.hi[e] - own.lo[e];
      int before_it = 0;
      for (int f = 0; f < a.E; ++f) {
        const int other = own.hi[f] - own.lo[f];
        before_it += other > rows || (other == rows && f < e);
      }
      own.order[before_it] = e;
    }
  }
}

struct Unit {
  int expert, lo, hi;  // rows of the tile, or of the expert (kDw)
  int m0, n0;          // kDw: first row of the result; first column
  int kb_lo, kb_hi, slice;
};

// kFwd, kDx: groups of kGroup row tiles go through the columns, the row tile varying fastest, so that the pairs at
// work share few row tiles and few column tiles through L2.  kDw: the experts in the list's order.
template <int WHICH, int ROWS>
__device__ __forceinline__ Unit decode(const TcArgs& a, const Own& own, int rows, int u) {
  const int n_tiles = (a.n_cols + BN - 1) / BN;
  Unit w;
  if (WHICH == kDw) {
    const int per = a.m_tiles * n_tiles, rank = u / (per * a.parts), in = u - rank * per * a.parts;
    const int part = in / per, tile = in - part * per;
    Tile t;
    if (a.offsets) {
      t.expert = own.order[rank];
      t.lo = own.lo[t.expert];
      t.hi = own.hi[t.expert];
    } else {
      t = a.tiles[rank];
    }
    w.expert = tc::uniform(t.expert);
    w.lo = tc::uniform(t.lo);
    w.hi = tc::uniform(t.hi);
    w.m0 = tile / n_tiles * ROWS;
    w.n0 = (tile - tile / n_tiles * n_tiles) * BN;
    part_range((w.hi - w.lo + BK - 1) / BK, part, a.parts, w.kb_lo, w.kb_hi);
    w.slice = part * a.E + w.expert;
    return w;
  }
  const int grp = u / (kGroup * n_tiles), in = u - grp * kGroup * n_tiles;
  const int left = max(1, min(kGroup, rows - grp * kGroup));
  const int n = in / left;
  const int index = grp * kGroup + in - n * left;
  Tile t;
  if (a.offsets) {  // the last expert whose tiles begin at or before it, by the whole warp
    static_assert(kOwnExperts == 64, "two a lane");
    const int e = threadIdx.x & 31;
    t.expert = __popc(__ballot_sync(0xFFFFFFFFu, e < a.E && own.first[e] <= index)) +
               __popc(__ballot_sync(0xFFFFFFFFu, e + 32 < a.E && own.first[e + 32] <= index)) - 1;
    t.lo = own.lo[t.expert] + (index - own.first[t.expert]) * ROWS;
    t.hi = min(t.lo + ROWS, own.hi[t.expert]);
  } else {
    t = a.tiles[index];
  }
  w.expert = tc::uniform(t.expert);
  w.lo = tc::uniform(t.lo);
  w.hi = tc::uniform(t.hi);
  w.m0 = 0;
  w.n0 = n * BN;
  w.kb_lo = 0;
  w.kb_hi = a.k_blocks;
  w.slice = 0;
  return w;
}

__device__ __forceinline__ uint32_t pack_bf16(uint32_t lo, uint32_t hi) {
  return rows::pack_bf16(make_float2(__uint_as_float(lo), __uint_as_float(hi)));
}

// kFwd, kDx: a tile of up to 128 rows is turned: the weights' columns go along M and its rows along N, whose length an
// MMA's time follows in steps of 32 (16 rows of each CTA), with the same loads into the same places.  Its N, 0 for a tile
// that is not turned.  us, without / with this: 62 rows an expert (32 experts, 4096 x 1536) 112 / 91, 1875 (64, 2048 x
// 1024) 457 / 452.  Tiles of up to 224 rows turned as well take the same within 2 %: they wait for their operands, which
// are no fewer.
__device__ __forceinline__ int turned_rows(const Unit& w) {
  const int n = (w.hi - w.lo + 31) / 32 * 32;
  return n <= BM ? n : 0;
}

// The operand of the MMA step kk (16 elements of the contraction) in a stage.  Contiguous along it: 32 bytes of the swizzled
// 128-byte row, groups of eight rows 1024 bytes apart; across it: 16 rows are two such groups, blocks of 64 columns
// whole boxes apart.
template <bool ACROSS>
__device__ __forceinline__ uint64_t step_desc(uint32_t base, int kk) {
  return ACROSS ? tc::smem_desc_sw128(base + kk * 2048, kBox, 1024) : tc::smem_desc_sw128(base + kk * 32, 16, 1024);
}

__device__ __forceinline__ void load_3d(void* dst, const CUtensorMap* map, uint64_t* bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(tc::smem_u32(dst)),
      "l"(map), "r"(tc::smem_u32(bar)), "r"(x), "r"(y), "r"(z)
      : "memory");
}
__device__ __forceinline__ void load_3d_pair(void* dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(tc::smem_u32(dst)),
      "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
      : "memory");
}
// A wait for what the other CTA of the pair has written.
__device__ __forceinline__ bool peer_wait(uint64_t* bar, uint32_t parity, volatile uint32_t* abort_flag) {
  const uint64_t t0 = tc::global_timer_ns();
  for (uint32_t it = 1;; ++it) {
    uint32_t ok;
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
        "selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(ok)
        : "r"(tc::smem_u32(bar)), "r"(parity)
        : "memory");
    if (ok) return true;
    if ((it & 127u) == 0u) {
      if (*abort_flag != 0u) return false;
      if (tc::global_timer_ns() - t0 > tc::kWaitLimitNs) {
        *abort_flag = 1u;
        return false;
      }
    }
  }
}

template <bool ADD>
__device__ __forceinline__ void put_3d(const CUtensorMap* map, const void* src, int x, int y, int z) {
  if (ADD)
    asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map),
                 "r"(tc::smem_u32(src)), "r"(x), "r"(y), "r"(z)
                 : "memory");
  else
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map),
                 "r"(tc::smem_u32(src)), "r"(x), "r"(y), "r"(z)
                 : "memory");
}

template <int WHICH, int ROWS, bool LONG>
__global__ void __launch_bounds__(Ring<WHICH, ROWS, LONG>::kThreads, 1)
experts_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_a32,
               const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_c, const TcArgs a) {
  using R = Ring<WHICH, ROWS, LONG>;
  constexpr int kNS = R::kNum;
  constexpr bool kAcross = WHICH == kDw;                    // A is contiguous across the contraction
  constexpr bool kBcross = WHICH == kDw || WHICH == kDx;
  constexpr uint32_t kIdesc = tc::instr_desc_bf16(2 * BM, BN, kAcross ? 1 : 0, kBcross ? 1 : 0);

  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* staging = smem + (size_t)kNS * R::kStage;
  uint64_t* full_bar = reinterpret_cast<uint64_t*>(staging + R::kStaging);  // [kNS], the even CTA's are used
  uint64_t* empty_bar = full_bar + kNS;                                     // [kNS]
  uint64_t* tfull_bar = empty_bar + kNS;                                    // [2]
  uint64_t* tempty_bar = tfull_bar + 2;                                     // [2], the even CTA's are used
  uint64_t* tail_bar = tempty_bar + 2;                                      // kDw: this CTA's part of a last block
  uint64_t* peer_bar = tail_bar + 1;                                        // [kNS] the odd CTA's is done
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(peer_bar + kNS);
  volatile uint32_t* abort_flag = tmem_slot + 1;

  const int warp = tc::uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int rank = (int)(tc::cluster_ctarank() & 1u);
  const int unit0 = blockIdx.x / 2, stride = gridDim.x / 2;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kNS; ++s) {
      tc::mbar_init(&full_bar[s], 1);
      tc::mbar_init(&empty_bar[s], 1);
      tc::mbar_init(&peer_bar[s], 1);
    }
    tc::mbar_init(tail_bar, 1);
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(&tfull_bar[i], 1);
      tc::mbar_init(&tempty_bar[i], R::kWriters * 2);
    }
    *abort_flag = 0u;
    tc::fence_barrier_init();
    tc::fence_proxy_async();
    tc::prefetch_tensormap(&map_a);
    tc::prefetch_tensormap(&map_b);
    if (WHICH != kDw) tc::prefetch_tensormap(&map_a32);
    tc::prefetch_tensormap(&map_c);
  }
  if (warp == 1) {
    tc::tmem_alloc_pair(tmem_slot, kTmemCols);
    tc::tmem_relinquish_pair();
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::cluster_sync_all();  // the peer's barriers exist before anyone signals them
  tc::fence_after_sync();
  const uint32_t tmem_base = tc::uniform(*tmem_slot);
  wait_for_primary();  // the list of tiles, or what it is made from, is there
  __shared__ Own own;
  if (a.offsets) {
    if (warp == 0) find_tiles<WHICH, ROWS>(a, own);
    __syncthreads();
  }
  const int row_tiles = a.offsets ? tc::uniform(own.first[a.E]) : (int)a.head->tiles;
  const bool broken = a.offsets ? own.broken : a.head->broken != 0;
  const int units = (a.n_cols + BN - 1) / BN * (WHICH == kDw ? (broken ? 0 : a.E * a.m_tiles * a.parts) : row_tiles);

  auto all = [](bool x) { return __all_sync(0xFFFFFFFFu, x ? 1 : 0) != 0; };
  // The entry of the unit after `u` is asked for before u is worked on: it costs a round trip to L2.
  auto first_unit = [&]() { return decode<WHICH, ROWS>(a, own, row_tiles, units > 0 ? min(unit0, units - 1) : 0); };
  auto unit_after = [&](int u) { return decode<WHICH, ROWS>(a, own, row_tiles, u + stride < units ? u + stride : u); };
  auto segments_of = [&](const Unit& w) {
    return R::kSums ? max(1, (w.kb_hi - w.kb_lo + kSegment<WHICH> - 1) / kSegment<WHICH>) : 1;
  };
  // A gradient that is added to takes nothing from an expert without rows.
  auto skipped = [&](const Unit& w) {
    return WHICH == kDw && a.accumulate && a.parts == 1 && w.kb_lo == w.kb_hi;
  };

  if (warp == 0) {
    // ------------------------------------------------ TMA producer (lane 0; all lanes for the last rows)
    uint32_t it = 0, tail_phase = 0u, peer_phase = 0u;  // peer_phase: a bit a stage
    bool ok = true;
    Unit next = first_unit();
    for (int u = unit0; ok && u < units; u += stride) {
      const Unit w = next;
      next = unit_after(u);
      if (skipped(w)) continue;
      const int n0 = w.n0 + rank * (BN / 2);
      // the tile's row slots of each CTA, and the pieces of 32 of them that have rows
      const int turned = turned_rows(w), each = turned ? turned / 2 : BM, first = rank * each;
      auto pieces_from = [&](int r) { return max(0, (min(w.hi - w.lo - r, each) + 31) / 32); };
      const int pieces = pieces_from(first), all_pieces = pieces + pieces_from(each - first);
      for (int kb = w.kb_lo; kb < w.kb_hi; kb += R::kPer, ++it) {
        const int s = it % kNS;
        ok = all(tc::mbar_wait(&empty_bar[s], ((it / kNS) & 1u) ^ 1u, abort_flag));
        if (!ok) break;
        uint8_t* a_dst = smem + (size_t)s * R::kStage;
        uint8_t* b_dst = a_dst + R::kABytes;
        // both CTAs' loads count on the even CTA's barrier, which its producer arms with the bytes of the pair
        const uint32_t bar = tc::map_to_cta(tc::smem_u32(&full_bar[s]), 0);
        if (WHICH == kDw) {
          // from the last block to the first: the one that is not full, whose way takes longest, is then asked for while
          // the tile before is still at work
          const int t = w.lo + (w.kb_hi - 1 - (kb - w.kb_lo)) * BK, len = min(BK, w.hi - t);
          if (tc::elect_one()) {
            if (len < BK) tc::mbar_arrive_expect_tx(tail_bar, R::kStage);
            else if (rank == 0) tc::mbar_arrive_expect_tx(&full_bar[s], 2 * R::kStage);
            if (a.merged) {
              const int ax = (w.m0 + rank * BM) / 64, bx = n0 / 64;
              if (len < BK) {
                load_3d(a_dst, &map_a, tail_bar, 0, t, ax);
                load_3d(b_dst, &map_b, tail_bar, 0, t, bx);
              } else {
                load_3d_pair(a_dst, &map_a, bar, 0, t, ax);
                load_3d_pair(b_dst, &map_b, bar, 0, t, bx);
              }
            } else {
#pragma unroll
              for (int j = 0; j < 4; ++j) {  // boxes of A, then of B
                const CUtensorMap* map = j < 2 ? &map_a : &map_b;
                const int x = j < 2 ? w.m0 + rank * BM + j * 64 : n0 + (j - 2) * 64;
                if (len < BK) tc::tma_load_2d(a_dst + j * kBox, map, tail_bar, x, t);
                else tc::tma_load_2d_pair(a_dst + j * kBox, map, bar, x, t);
              }
            }
          }
          __syncwarp();
          if (len < BK) {
            ok = all(tc::mbar_wait(tail_bar, tail_phase, abort_flag));
            if (!ok) break;
            tail_phase ^= 1u;
#pragma unroll
            for (int j = 0; j < 4; ++j)
              for (int i = len * 8 + lane; i < BK * 8; i += 32)
                *reinterpret_cast<uint4*>(a_dst + j * kBox + i * 16) = make_uint4(0u, 0u, 0u, 0u);
            tc::fence_proxy_async();
            __syncwarp();
            if (rank == 1) {
              if (lane == 0) tc::mbar_arrive_cluster(tc::map_to_cta(tc::smem_u32(&peer_bar[s]), 0));
            } else {
              ok = all(peer_wait(&peer_bar[s], (peer_phase >> s) & 1u, abort_flag));
              if (!ok) break;
              peer_phase ^= 1u << s;
              if (lane == 0) tc::mbar_arrive(&full_bar[s]);
            }
          }
        } else if (tc::elect_one()) {
          // of A only what has rows of the tile: 128 of them, or fewer in pieces of 32 (the rest of the stage is what it
          // was: rows of the accumulator that nobody writes out)
          const int here = min(R::kPer, w.kb_hi - kb);
          if (rank == 0) tc::mbar_arrive_expect_tx(&full_bar[s], here * (2 * R::kBBytes + all_pieces * 32 * BK * 2));
#pragma unroll
          for (int h = 0; h < R::kPer; ++h) {
            if (h >= here) break;
            const int at = h * R::kBlock, k0 = (kb + h) * BK;
            if (pieces == 4) {
              tc::tma_load_2d_pair(a_dst + at, &map_a, bar, k0, w.lo + first);
            } else {
              for (int i = 0; i < pieces; ++i)
                tc::tma_load_2d_pair(a_dst + at + i * 32 * BK * 2, &map_a32, bar, k0, w.lo + first + i * 32);
            }
            if (WHICH == kFwd) {
              load_3d_pair(b_dst + at, &map_b, bar, k0, n0, w.expert);
            } else {
#pragma unroll
              for (int j = 0; j < 2; ++j) load_3d_pair(b_dst + at + j * kBox, &map_b, bar, n0 + j * 64, k0, w.expert);
            }
          }
        }
      }
    }
    // Wait until every stage this warp filled has been released, so that no arrival targets this CTA after it has
    // left and no load is still writing its shared memory.  Bounded like every wait.
    const uint32_t pending = it < (uint32_t)kNS ? it : (uint32_t)kNS;
    for (uint32_t j = 0; ok && j < pending; ++j) {
      const uint32_t jt = it - 1 - j;
      ok = all(tc::mbar_wait(&empty_bar[jt % kNS], (jt / kNS) & 1u, abort_flag));
    }
    if (!ok) {  // given up: time for the copies in flight to land
      const uint64_t t0 = tc::global_timer_ns();
      while (tc::global_timer_ns() - t0 < 20000000ull) __nanosleep(1000);
    }
  } else if (warp == 1) {
    // ------------------------------------------------ MMA issuer (even CTA)
    if (rank == 0) {
      // The whole warp goes through the loops and one elected lane issues: what the instructions need has to be in uniform
      // registers, and what one lane alone has worked out is moved there value by value.
      uint32_t it = 0, tcount = 0;
      bool ok = true;
      Unit next = first_unit();
      for (int u = unit0; ok && u < units; u += stride) {
        const Unit w = next;
        next = unit_after(u);
        if (skipped(w)) continue;
        // of about the same length, whole stages each; none is empty, as none has more than kSegment blocks
        static_assert(kSegment<WHICH> % R::kPer == 0, "whole stages");
        const int blocks = w.kb_hi - w.kb_lo, segments = segments_of(w);
        const int per = R::kSums ? ((blocks + segments - 1) / segments + R::kPer - 1) / R::kPer * R::kPer : blocks;
        const int turned = WHICH == kDw ? 0 : turned_rows(w);
        const uint32_t turned_idesc = tc::instr_desc_bf16(2 * BM, turned, kBcross ? 1 : 0, 0);
        for (int seg = 0; ok && seg < segments; ++seg, ++tcount) {
          const uint32_t acc = tcount & 1u, aph = (tcount >> 1) & 1u;
          const int kb_lo = seg * per, kb_hi = min(kb_lo + per, blocks);
          ok = all(tc::mbar_wait(&tempty_bar[acc], aph ^ 1u, abort_flag));
          if (!ok) break;
          tc::fence_after_sync();
          const uint32_t d_tmem = tmem_base + acc * BN;
          for (int kb = kb_lo; kb < kb_hi; kb += R::kPer, ++it) {
            const int s = it % kNS;
            ok = all(tc::mbar_wait(&full_bar[s], (it / kNS) & 1u, abort_flag));
            if (!ok) break;
            tc::fence_after_sync();
            const uint32_t stage = tc::smem_u32(smem + (size_t)s * R::kStage);
            if (tc::elect_one()) {
#pragma unroll
              for (int h = 0; h < R::kPer; ++h) {
                if (kb + h >= kb_hi) break;
                const uint32_t a_base = stage + h * R::kBlock, b_base = a_base + R::kABytes;
                if (WHICH != kDw && turned) {
#pragma unroll
                  for (int kk = 0; kk < BK / 16; ++kk)
                    tc::umma_bf16_pair(d_tmem, step_desc<kBcross>(b_base, kk), step_desc<kAcross>(a_base, kk), turned_idesc,
                                       (kb + h > kb_lo || kk > 0) ? 1u : 0u);
                } else {
#pragma unroll
                  for (int kk = 0; kk < BK / 16; ++kk)
                    tc::umma_bf16_pair(d_tmem, step_desc<kAcross>(a_base, kk), step_desc<kBcross>(b_base, kk), kIdesc,
                                       (kb + h > kb_lo || kk > 0) ? 1u : 0u);
                }
              }
              tc::umma_commit_pair(&empty_bar[s], 3);
            }
            __syncwarp();
          }
          if (ok && tc::elect_one()) tc::umma_commit_pair(&tfull_bar[acc], 3);
          __syncwarp();
        }
      }
    }
    __syncwarp();
  } else {
    // ------------------------------------------------ epilogue
    const int q = warp & 3;                     // tensor-memory lanes that this warp may read
    uint8_t* const stage = staging + (warp - 2) * R::kPiece;
    const int in_tile = rank * BM + q * 32;     // first of the warp's rows
    uint32_t tcount = 0;
    bool ok = true;
    Unit next = first_unit();
    for (int u = unit0; ok && u < units; u += stride) {
      const Unit w = next;
      next = unit_after(u);
      if (skipped(w)) continue;
      const int turned_n = WHICH == kDw ? 0 : turned_rows(w);
      const bool turned = WHICH != kDw && (ROWS <= BM || turned_n > 0);
      const int valid = WHICH == kDw ? 32 : min(32, w.hi - w.lo - in_tile);  // of the warp's rows, where not turned
      // Columns [col, col + 64) of the warp's rows, two to a register.
      auto put_rows = [&](int col, const uint32_t (&packed)[32]) {
        if (valid == 32) {
          // through the warp's block of shared memory, whole lines at a time
          if (lane == 0) tc::bulk_wait_read_all();
          __syncwarp();
#pragma unroll
          for (int j = 0; j < 8; ++j)
            *reinterpret_cast<uint4*>(stage + lane * 128 + ((j ^ (lane & 7)) << 4)) =
                make_uint4(packed[4 * j], packed[4 * j + 1], packed[4 * j + 2], packed[4 * j + 3]);
          tc::fence_proxy_async();
          __syncwarp();
          if (lane == 0) {
            tc::tma_store_2d(&map_c, stage, col, w.lo + in_tile);
            tc::bulk_commit();
          }
        } else if (lane < valid) {
          // the expert's last rows: those behind are another's
          __nv_bfloat16* dst = a.rows_out + (int64_t)(w.lo + in_tile + lane) * a.rows_stride + col;
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (col + 8 * j < a.n_cols)
              *reinterpret_cast<uint4*>(dst + 8 * j) =
                  make_uint4(packed[4 * j], packed[4 * j + 1], packed[4 * j + 2], packed[4 * j + 3]);
        }
        __syncwarp();
      };
      // Rows [first, first + 32) of a turned tile, element(j) of each lane, which has a column of the result: 32 rows of 64
      // bytes through the warp's block of shared memory, then 16 bytes a lane (single elements straight to memory: 8 us
      // for a tile of 184 rows).  Before the first, what left the block by TMA has to have been read.
      auto put_turned = [&](int first, auto element) {
        const int rows = w.hi - w.lo, col = w.n0 + in_tile + lane % 4 * 8;
        __nv_bfloat16* rows32 = reinterpret_cast<__nv_bfloat16*>(stage);
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 32; ++j) rows32[j * 32 + lane] = __float2bfloat16_rn(element(j));
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int row = first + j * 8 + lane / 4;
          if (row < rows && col < a.n_cols)
            *reinterpret_cast<uint4*>(a.rows_out + (int64_t)(w.lo + row) * a.rows_stride + col) =
                *reinterpret_cast<const uint4*>(rows32 + (j * 8 + lane / 4) * 32 + lane % 4 * 8);
        }
      };
      if constexpr (R::kSums) {
        // Two warps for 32 lanes of tensor memory, with 32 columns at a time of their half, or, of a turned tile, every
        // other 32: the segments' sums are added up in registers.
        constexpr int kRuns = WHICH != kDw && ROWS <= BM ? ROWS / 64 : BN / 64;
        const int segments = segments_of(w), half = (warp - 2) >> 2;
        auto run_at = [&](int c) { return turned ? (2 * c + half) * 32 : half * (BN / 2) + c * 32; };
        auto run_has = [&](int c) { return turned ? run_at(c) < turned_n : valid > 0; };
        float2 sum[kRuns * 16];
#pragma unroll
        for (int j = 0; j < kRuns * 16; ++j) sum[j] = both(0.f);
        for (int seg = 0; seg < segments; ++seg, ++tcount) {
          const uint32_t acc = tcount & 1u, aph = (tcount >> 1) & 1u;
          ok = all(tc::mbar_wait(&tfull_bar[acc], aph, abort_flag));
          if (!ok) break;
          tc::fence_after_sync();
          const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + acc * BN;
#pragma unroll
          for (int c = 0; c < kRuns; ++c) {
            if (!run_has(c)) break;
            uint32_t v[32];
            tc::tmem_ld32_issue(taddr + run_at(c), v);
            tc::tmem_ld_wait(v);
#pragma unroll
            for (int j = 0; j < 16; ++j)
              sum[c * 16 + j] = add2(sum[c * 16 + j], make_float2(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1])));
          }
          tc::fence_before_sync();
          __syncwarp();
          if (lane == 0) tc::mbar_arrive_cluster(tc::map_to_cta(tc::smem_u32(&tempty_bar[acc]), 0));
        }
        if (!ok) break;
        if (WHICH != kDw && turned) {
          if (lane == 0) tc::bulk_wait_read_all();
#pragma unroll
          for (int c = 0; c < min(kRuns, BM / 64); ++c) {
            if (!run_has(c)) break;
            put_turned(run_at(c), [&](int j) { return j & 1 ? sum[c * 16 + j / 2].y : sum[c * 16 + j / 2].x; });
          }
          __syncwarp();
        } else if constexpr (WHICH != kDw && ROWS > BM) {
#pragma unroll
          for (int c = 0; c < kRuns; c += 2) {
            const int col = w.n0 + run_at(c);
            if (valid <= 0 || col >= a.n_cols) break;
            uint32_t packed[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) packed[j] = rows::pack_bf16(sum[c * 16 + j]);
            put_rows(col, packed);
          }
        } else if constexpr (WHICH == kDw) {
          const bool none = w.kb_lo == w.kb_hi;  // no rows: zeros, not what tensor memory held
          const bool add = a.accumulate && a.parts == 1;
#pragma unroll
          for (int c = 0; c < kRuns; ++c) {
            const int col = w.n0 + run_at(c);
            if (col >= a.n_cols) break;
            if (lane == 0) tc::bulk_wait_read_all();  // the piece before has left
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float2 x = sum[c * 16 + 2 * j], y = sum[c * 16 + 2 * j + 1];
              *reinterpret_cast<float4*>(stage + lane * 128 + ((j ^ (lane & 7)) << 4)) =
                  none ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(x.x, x.y, y.x, y.y);
            }
            tc::fence_proxy_async();
            __syncwarp();
            if (lane == 0) {
              // rows behind n_out are outside the map
              if (add) put_3d<true>(&map_c, stage, col, w.m0 + in_tile, w.slice);
              else put_3d<false>(&map_c, stage, col, w.m0 + in_tile, w.slice);
              tc::bulk_commit();
            }
          }
        }
      } else {
        const uint32_t acc = tcount & 1u, aph = (tcount >> 1) & 1u;
        ++tcount;
        ok = all(tc::mbar_wait(&tfull_bar[acc], aph, abort_flag));
        if (!ok) break;
        tc::fence_after_sync();
        const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + acc * BN;
        if (turned) {
          if (lane == 0) tc::bulk_wait_read_all();
#pragma unroll 1
          for (int c = 0; c < turned_n; c += 32) {
            uint32_t v[32];
            tc::tmem_ld32_issue(taddr + c, v);
            tc::tmem_ld_wait(v);
            put_turned(c, [&](int j) { return __uint_as_float(v[j]); });
          }
          __syncwarp();
        } else {
#pragma unroll 1
          for (int c = 0; c < BN / 64 && valid > 0; ++c) {
            const int col = w.n0 + c * 64;
            if (col >= a.n_cols) break;
            uint32_t ra[32], rb[32], packed[32];
            tc::tmem_ld32_issue(taddr + c * 64, ra);
            tc::tmem_ld32_issue(taddr + c * 64 + 32, rb);
            tc::tmem_ld_wait(ra);
            tc::tmem_ld_pin(rb);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              packed[j] = pack_bf16(ra[2 * j], ra[2 * j + 1]);
              packed[16 + j] = pack_bf16(rb[2 * j], rb[2 * j + 1]);
            }
            put_rows(col, packed);
          }
        }
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive_cluster(tc::map_to_cta(tc::smem_u32(&tempty_bar[acc]), 0));
      }
    }
    if (lane == 0) tc::bulk_wait_all();  // this warp's stores are done
  }
  tc::fence_before_sync();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag != 0u) atomicOr(&a.head->status, NAT_DEV_TIMEOUT);
  tc::cluster_sync_all();  // the pair leaves together
  if (warp == 1) {
    tc::fence_after_sync();
    tc::tmem_dealloc_pair(tmem_base, kTmemCols);
  }
}

// --------------------------------------------------------------------------- host
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

int encode(CUtensorMap* map, CUtensorMapDataType type, int dims, uintptr_t base, const cuuint64_t* size,
           const cuuint64_t* pitch, const cuuint32_t* box) {
  static std::atomic<EncodeTiledFn> cached{nullptr};
  EncodeTiledFn fn = cached.load(std::memory_order_relaxed);
  if (!fn) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    NAT_CUDA(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found));
    if (found != cudaDriverEntryPointSuccess || !p)
      return fail(NAT_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
    fn = reinterpret_cast<EncodeTiledFn>(p);
    cached.store(fn, std::memory_order_relaxed);
  }
  const cuuint32_t one[3] = {1, 1, 1};
  const CUresult r = fn(map, type, (cuuint32_t)dims, reinterpret_cast<void*>(base), size, pitch, box, one,
                        CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return fail(NAT_ERR_CUDA, "cuTensorMapEncodeTiled failed with code %d", (int)r);
  return NAT_OK;
}

// Rows of a matrix [rows, cols] of bfloat16: boxes of 64 columns.
int map_rows(CUtensorMap* map, const void* base, int cols, int64_t rows, int64_t stride, int box_rows) {
  const cuuint64_t size[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, pitch[1] = {(cuuint64_t)stride * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, (uintptr_t)base, size, pitch, box);
}
// The same with the columns in blocks of 64: boxes of two blocks by BK rows (one load in place of two: the weights' gradient
// takes 5 to 7 % less).  cols a multiple of 64.
int map_blocks(CUtensorMap* map, const void* base, int cols, int64_t rows, int64_t stride) {
  const cuuint64_t size[3] = {64, (cuuint64_t)rows, (cuuint64_t)(cols / 64)}, pitch[2] = {(cuuint64_t)stride * 2, 128};
  const cuuint32_t box[3] = {64, (cuuint32_t)BK, 2};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, (uintptr_t)base, size, pitch, box);
}
// The experts' weights [E, n_out, n_in]: boxes of 64 columns by box_rows of one expert.
int map_weights(CUtensorMap* map, const nat_experts_params& p, const void* w, int box_rows) {
  const cuuint64_t size[3] = {(cuuint64_t)p.n_in, (cuuint64_t)p.n_out, (cuuint64_t)p.n_experts};
  const cuuint64_t pitch[2] = {(cuuint64_t)p.n_in * 2, (cuuint64_t)p.n_in * p.n_out * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, (uintptr_t)w, size, pitch, box);
}
// Their gradient, or the parts' [slices, n_out, n_in] in float32: pieces of 32 x 32.
int map_gradient(CUtensorMap* map, const nat_experts_params& p, const float* dw, int64_t slices) {
  const cuuint64_t size[3] = {(cuuint64_t)p.n_in, (cuuint64_t)p.n_out, (cuuint64_t)slices};
  const cuuint64_t pitch[2] = {(cuuint64_t)p.n_in * 4, (cuuint64_t)p.n_in * p.n_out * 4};
  const cuuint32_t box[3] = {32, 32, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, (uintptr_t)dw, size, pitch, box);
}

// Of the current device, below 64.
int device_index(int* dev) {
  static std::atomic<bool> fits[64];
  NAT_CUDA(cudaGetDevice(dev));
  if (*dev < 0 || *dev >= 64)
    return fail(NAT_ERR_UNSUPPORTED, "device index %d is beyond the 64 this library tracks", *dev);
  if (!fits[*dev].load(std::memory_order_relaxed)) {
    const int s = require_sm100();
    if (s != NAT_OK) return s;
    fits[*dev].store(true, std::memory_order_relaxed);
  }
  return NAT_OK;
}

// CTA pairs that the current device holds at a time, found once for each device.
template <int WHICH, int ROWS, bool LONG>
int pairs(int* out) {
  static std::atomic<int> cached[64];
  int dev = 0;
  int s = device_index(&dev);
  if (s != NAT_OK) return s;
  int n = cached[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    NAT_CUDA(cudaFuncSetAttribute(experts_kernel<WHICH, ROWS, LONG>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                  (int)Ring<WHICH, ROWS, LONG>::kSmem));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(148);
    cfg.blockDim = dim3(Ring<WHICH, ROWS, LONG>::kThreads);
    cfg.dynamicSmemBytes = Ring<WHICH, ROWS, LONG>::kSmem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    NAT_CUDA(cudaOccupancyMaxActiveClusters(&n, experts_kernel<WHICH, ROWS, LONG>, &cfg));
    if (n <= 0) return fail(NAT_ERR_UNSUPPORTED, "the device does not hold the experts' CTA pairs");
    cached[dev].store(n, std::memory_order_relaxed);
  }
  *out = n;
  return NAT_OK;
}

template <int WHICH, int ROWS, bool LONG>
int launch(const CUtensorMap& ma, const CUtensorMap& ma32, const CUtensorMap& mb, const CUtensorMap& mc, const TcArgs& t,
           int64_t most_units, cudaStream_t stream) {
  int slots = 0;
  int s = pairs<WHICH, ROWS, LONG>(&slots);
  if (s != NAT_OK) return s;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(2 * min(most_units, (int64_t)slots)));
  cfg.blockDim = dim3(Ring<WHICH, ROWS, LONG>::kThreads);
  cfg.dynamicSmemBytes = Ring<WHICH, ROWS, LONG>::kSmem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  NAT_CUDA(cudaLaunchKernelEx(&cfg, experts_kernel<WHICH, ROWS, LONG>, ma, ma32, mb, mc, t));
  return NAT_OK;
}

}  // namespace

// Terms of a contraction up to which one accumulator takes them all (kFwd, kDx).  Where the terms have one sign, what the
// tensor cores cut off adds up to 6e-9 of the sum a term: 2.4e-5 at 4096, a hundredth of bfloat16's half step, but 1.5e-3
// at 262,144, where a quarter of the results was not the nearest.  Sums in registers, us without / with: 20,000 rows over 8
// experts, 14,336 x 2048, 953 / 961; 1500 over 32, 8192 x 1536, 132 / 134; up to 4096 terms they would cost as much and
// gain nothing: 120,007 over 64, 2048 x 1024, 432 / 438, rows' gradient 441 / 453.
constexpr int kWhole = 4096;

// Average rows of an expert (by the capacity, which is what the host knows) up to which a row tile has 64 or 128 rows in
// place of 256.  All are turned then, a stage holds two blocks of the contraction (a block with few rows is done with
// sooner than its barriers are), and what is left to bound it is the reading of the weights.  us, tiles of 256, 128 and 64
// rows, forward:
//   rows an expert                  31             47             62             94             125
//   32 experts, 4096 x 1536     83, 77, 75     86, 79, 76     90, 83, 85     94, 87, 106    98, 100, -
//   128 experts, 2048 x 768         -          85, 80, 78     89, 83, 84     96, 88, 105    104, 103, -
//   8 experts, 4096 x 4096          -          59, 55, 53     60, 56, 62         -          66, 74, -
constexpr int64_t kFew = 48, kSome = 96;
static_assert(BM / 2 == kFewestRows, "the list of tiles has room for the smallest");
int bf16_tile_rows(const nat_experts_params& p, Product which, int64_t cap) {
  const int64_t rows = cap / p.n_experts;
  if (which != kDw) return rows <= kFew ? BM / 2 : rows <= kSome ? BM : 2 * BM;
  return 2 * BM;
}

int bf16_product(const Args& a, const Layout& l, Product which) {
  const nat_experts_params& p = a.p;
  CUtensorMap ma, ma32, mb, mc;
  int s;
  TcArgs t{};
  t.head = head(a);
  t.tiles = which == kDw ? by_rows(a, l) : tiles(a, l);
  t.E = p.n_experts;
  t.parts = which == kDw ? l.parts : 1;
  t.accumulate = p.accumulate != 0;
  t.offsets = p.n_experts <= kOwnExperts ? a.offsets : nullptr;
  t.cap = a.cap;
  t.tells = which != kDw || !a.dx;
  if (which == kDw) {
    t.merged = p.n_out % 64 == 0 && p.n_in % 64 == 0;
    if ((s = t.merged ? map_blocks(&ma, a.dy, p.n_out, a.cap, p.y_stride)
                      : map_rows(&ma, a.dy, p.n_out, a.cap, p.y_stride, BK)) != NAT_OK)
      return s;
    if ((s = t.merged ? map_blocks(&mb, a.x, p.n_in, a.cap, p.x_stride)
                      : map_rows(&mb, a.x, p.n_in, a.cap, p.x_stride, BK)) != NAT_OK)
      return s;
    if ((s = l.parts > 1 ? map_gradient(&mc, p, partial(a, l), (int64_t)l.parts * p.n_experts)
                         : map_gradient(&mc, p, a.dw, p.n_experts)) != NAT_OK)
      return s;
    t.n_cols = p.n_in;
    t.m_tiles = (p.n_out + l.tile_rows[kDw] - 1) / l.tile_rows[kDw];
    const int64_t units = (int64_t)t.E * t.m_tiles * ((p.n_in + BN - 1) / BN) * t.parts;
    return launch<kDw, 2 * BM, false>(ma, ma, mb, mc, t, units, a.stream);
  }
  const bool fwd = which == kFwd;
  const void *in = fwd ? a.x : a.dy;
  void* out = fwd ? a.y : a.dx;
  const int k = fwd ? p.n_in : p.n_out, n = fwd ? p.n_out : p.n_in;
  const int64_t in_stride = fwd ? p.x_stride : p.y_stride;
  t.n_cols = n;
  t.k_blocks = (k + BK - 1) / BK;
  t.rows_out = (__nv_bfloat16*)out;
  t.rows_stride = fwd ? p.y_stride : p.x_stride;
  if ((s = map_rows(&ma, in, k, a.cap, in_stride, BM)) != NAT_OK) return s;
  if ((s = map_rows(&ma32, in, k, a.cap, in_stride, 32)) != NAT_OK) return s;
  if ((s = map_weights(&mb, p, a.w, fwd ? BN / 2 : BK)) != NAT_OK) return s;
  if ((s = map_rows(&mc, out, n, a.cap, t.rows_stride, 32)) != NAT_OK) return s;
  const int64_t units = most_tiles(p, a.cap, l.tile_rows[which]) * ((n + BN - 1) / BN);
  auto product = [&](auto tile_rows) {
    constexpr int kRows = decltype(tile_rows)::value;
    if (k > kWhole)
      return fwd ? launch<kFwd, kRows, true>(ma, ma32, mb, mc, t, units, a.stream)
                 : launch<kDx, kRows, true>(ma, ma32, mb, mc, t, units, a.stream);
    return fwd ? launch<kFwd, kRows, false>(ma, ma32, mb, mc, t, units, a.stream)
               : launch<kDx, kRows, false>(ma, ma32, mb, mc, t, units, a.stream);
  };
  switch (l.tile_rows[which]) {
    case BM / 2: return product(std::integral_constant<int, BM / 2>());
    case BM: return product(std::integral_constant<int, BM>());
    default: return product(std::integral_constant<int, 2 * BM>());
  }
}

}  // namespace experts
}  // namespace nat
