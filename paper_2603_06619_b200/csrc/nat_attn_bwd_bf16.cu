// Backward pass of the packed causal attention on the tensor cores, bfloat16.
//
// Two parts, both persistent with one block per multiprocessor, each forming P = exp(S - lse) anew; one
// launch holds the blocks of the first part and, behind them, those of the second:
//   dq   a row tile of queries (heads of a group folded in) against its keys: S = Q K^T,
//        dP = dO V^T, dS = P (dP - delta), dQ += dS K                      (three products)
//   dkv  a tile of 128 keys against all later queries of its group, transposed: S' = K Q^T,
//        dP' = V dO^T, dV += P' dO, dK += dS' Q                            (four products)
// Seven products where one part for both would do five, but every sum stays in tensor memory and
// in a fixed order: no atomics on dQ, no fp32 scratch for it, and results that repeat bit for bit.
//
// Warps: 0-3 and 4-7 take the two column halves of the score tile (a thread has 64 columns of one
// row), 9 loads tiles by TMA, 11 (dkv) loads lse and delta of the query rows, and 8 and 10 issue the MMAs:
// the tensor pipe holds about one MMA beyond the running one, so with one issuing warp every wait and
// every commit between two products leaves it idle.  In dkv the warps have a chain each, S' and dV, dP'
// and dK, which share no tensor memory; in dq one has S, the other dP and dQ.
//
// 16 sequences of up to 8192 tokens, 32 heads over 8, 128 columns: 4.8 ms, 700 TFLOP/s counted (980 executed), at the
// 1000 W cap (1450 MHz).  A step of 128 x 128 takes 2640 cycles in dq (products alone 1536) and 2930 in dkv
// (2048); of either about 1200-1450 are the exponentials, which both halves of the threads take at once.
#include <cuda.h>

#include "nat_attn.cuh"
#include "nat_attn_masked.cuh"
#include "nat_attn_tc.cuh"

namespace nat {
namespace attn {
namespace {

struct BwdParams {
  const Entry* list;  // null where every block has one unit at most and finds it itself
  Batch batch;
  const uint32_t* count;
  float* partial;
  uint32_t* status;
  const float *lse2, *delta;  // [cap, n_heads]
  __nv_bfloat16 *dq, *dk, *dv;
  int64_t q_stride, k_stride, v_stride;
  int n_heads, n_kv_heads, group, tq, head_dim;
  float scale;
  Rows q, k, v, dout;  // for mend_dq and mend_dkv
};

template <int DP>
struct BwdShape {
  static constexpr int kNP = DP / 64;
  static constexpr uint32_t kTile = kNP * kPanel;
  // Beside the two resident tiles two rings: A holds the tiles that live long (K in dq, Q in dkv: used
  // by the first and the last product of a step), B the others.  In one common ring a B tile would
  // wait for the slot of an A tile that is still in use.
  static constexpr int kA = DP == 128 ? 3 : 4, kB = DP == 128 ? 2 : 4;
  static constexpr uint32_t kTiles = (2 + kA + kB) * kTile;
  static constexpr uint32_t kStats = 2 * 2 * kRows * 4;   // lse2 and delta of two row tiles
  static constexpr uint32_t kSlack = 768;                 // room to round the base up to 1024 bytes
  static constexpr uint32_t kBars = DP == 128 ? 256 : 384;  // barriers, then what Found describes
  static constexpr uint32_t kSmem = kTiles + kStats + kBars + kSlack;
};

// Behind the barriers: the address of the block's tensor memory, its abort flag, whether a result was not finite and,
// without a list, its tile and their number.
struct Found {
  uint32_t tmem, abort, total, odd;
  Entry entry;
};
__device__ __forceinline__ void find(const BwdParams& p, uint32_t block, Found* f, bool report) {
  uint32_t total, status;
  const Entry e = find_entry(p.batch, block / p.n_kv_heads, &total, &status);
  if ((threadIdx.x & 31) == 0) {
    f->entry = e;
    f->total = total;
    if (report && block == 0) *p.status = status;
  }
}

// The tiles need a 1024-byte aligned base.  Dynamic shared memory starts on such a boundary where a
// kernel has no static shared memory; should it not, the block reports it and does nothing.
__device__ __forceinline__ uint8_t* tile_base(uint8_t* raw, uint32_t slack, bool* fits) {
  const uint32_t at = tc::smem_u32(raw), up = (at + 1023u) & ~1023u;
  *fits = up - at <= slack;
  return raw + (up - at);
}

// 64 values as bf16 pairs into the first 32 of the 64 columns that they came from: each half of
// the threads stays in its own columns.
__device__ __forceinline__ void store64(uint32_t addr, const float (&x)[64]) {
  uint32_t r[32];
#pragma unroll
  for (int c = 0; c < 32; ++c) r[c] = bf16_pair(x[2 * c], x[2 * c + 1]);
  tmem_st32(addr, r);
  tmem_st_wait();
}

// Where step kk (16 of the contraction) of such an operand lies.
constexpr __device__ uint32_t half_cols(int kk) { return (uint32_t)(kk < 4 ? kk * 8 : 64 + (kk - 4) * 8); }

// D columns [half * DP/2, ...) of an accumulator row, times f, to global memory.  Returns zero, or NaN where one
// is not finite.
template <int DP>
__device__ __forceinline__ float2 store_acc(uint32_t addr, int half, __nv_bfloat16* dst, int D, float f, bool valid,
                                            bool wide) {
  float2 odd = {0.f, 0.f};
#pragma unroll
  for (int c = 0; c < DP / 64; ++c) {
    const int col = half * (DP / 2) + c * 32;
    float o[32];
    tc::tmem_ld32(addr + col, o);
    odd = finite32(o, odd);
    if (valid) store_row32(dst + col, o, f, D - col, wide);
  }
  return odd;
}

// Where a piece's N accumulators go for one row: [accumulator column][row].
template <int DP, int N>
__device__ __forceinline__ float* piece_slot(const BwdParams& p, const Entry& e, int head, int row) {
  return p.partial + ((int64_t)(e.slot + e.piece) * p.n_kv_heads + head) * (128 * N * DP) + row;
}
// One of them, from tensor-memory column `addr` on.  Returns as store_acc.
template <int DP>
__device__ __forceinline__ float2 store_piece(float* slot, uint32_t addr, int half) {
  float2 odd = {0.f, 0.f};
#pragma unroll
  for (int c = 0; c < DP / 64; ++c) {
    const int col = half * (DP / 2) + c * 32;
    float o[32];
    tc::tmem_ld32(addr + col, o);
    odd = finite32(o, odd);
#pragma unroll
    for (int i = 0; i < 32; ++i) __stcg(slot + (col + i) * 128, o[i]);
  }
  return odd;
}

// A thread's half of a row of gradients that was added up again: to the piece's slot or, times f, to the result.
template <int DP>
__device__ __forceinline__ void store_again(const float (&o)[DP / 2], int half, float* slot, __nv_bfloat16* dst, float f, int D) {
#pragma unroll
  for (int c = 0; c < DP / 2; c += 8) {
    const int col = half * (DP / 2) + c;
    if (slot) {
#pragma unroll
      for (int i = 0; i < 8; ++i) __stcg(slot + (col + i) * 128, o[c + i]);
    } else if (col < D) {
      *reinterpret_cast<uint4*>(dst + col) = make_uint4(bf16_pair(o[c] * f, o[c + 1] * f), bf16_pair(o[c + 2] * f, o[c + 3] * f),
                                                        bf16_pair(o[c + 4] * f, o[c + 5] * f), bf16_pair(o[c + 6] * f, o[c + 7] * f));
    }
  }
}

// P and P (dP - delta) of one query and key.
__device__ __forceinline__ float2 weight_and_slope(const BwdParams& p, int token, int head, int key, int kv_head) {
  const int D = p.head_dim;
  const int64_t at = (int64_t)token * p.n_heads + head;
  const float s = row_dot(p.q.at(token, head, D), p.k.at(key, kv_head, D), D);
  const float w = ex2(fmaf(s, p.scale * kLog2e, -__ldcg(p.lse2 + at)));
  return make_float2(w, w * (row_dot(p.dout.at(token, head, D), p.v.at(key, kv_head, D), D) - __ldcg(p.delta + at)));
}

// The rows of dq of this block's units that masked values of k have spoilt, over the keys [first, token] of their
// piece.  Each thread takes the half row that it had.
template <int DP>
__device__ __noinline__ void mend_dq(const BwdParams& p, const Entry* found, uint32_t units, uint32_t block, uint32_t blocks) {
  const int half = threadIdx.x >> 7, row = threadIdx.x & 127, D = p.head_dim, lo = half * (DP / 2), hi = min(lo + DP / 2, D);
  for (uint32_t u = block; u < units; u += blocks) {
    const Entry e = p.list ? p.list[u / p.n_kv_heads] : *found;
    const int kv_head = (int)(u % p.n_kv_heads), token = e.lo + row / p.group, head = kv_head * p.group + row % p.group;
    if (row >= p.group * p.tq || token >= e.seq_hi) continue;
    float* slot = e.pieces == 1 ? nullptr : piece_slot<DP, 1>(p, e, kv_head, row);
    __nv_bfloat16* dst = p.dq + (int64_t)token * p.q_stride + (int64_t)head * D;
    if (slot ? finite_piece<128>(slot, lo, hi) : finite_row(dst, lo, hi)) continue;
    const int64_t at = (int64_t)token * p.n_heads + head;
    if (!(fabsf(__ldcg(p.lse2 + at)) < INFINITY && fabsf(__ldcg(p.delta + at)) < INFINITY)) continue;
    const int first = e.seq_lo + e.begin * kRows, end = min(min(e.lo + p.tq, e.seq_hi), e.end == kAllSteps ? e.seq_hi : e.seq_lo + e.end * kRows);
    if (!hidden_only(p.k, kv_head, 1, D, token + 1, end, max(first, token - (kRows - 1)), token + 1)) continue;
    float o[DP / 2];
#pragma unroll
    for (int c = 0; c < DP / 2; ++c) o[c] = 0.f;
    for (int j = first; j <= token && j < end; ++j)
      row_add<DP / 2>(o, as_bf16(weight_and_slope(p, token, head, j, kv_head).y), p.k.at(j, kv_head, D), half * (DP / 16), D);
    store_again<DP>(o, half, slot, dst, p.scale, D);
  }
}

// The same for the rows of dv (of_k false) or dk, spoilt by masked values of dout or q, over the queries from the key on.
template <int DP>
__device__ __noinline__ void mend_dkv(const BwdParams& p, bool of_k, const Entry* found, uint32_t units, uint32_t block,
                                      uint32_t blocks) {
  const int half = threadIdx.x >> 7, row = threadIdx.x & 127, D = p.head_dim, lo = half * (DP / 2), hi = min(lo + DP / 2, D);
  const Rows& rows = of_k ? p.q : p.dout;
  for (uint32_t u = block; u < units; u += blocks) {
    const Entry e = p.list ? p.list[u / p.n_kv_heads] : *found;
    const int kv_head = (int)(u % p.n_kv_heads), key = e.lo + row, head = kv_head * p.group;
    if (key >= e.seq_hi) continue;
    float* slot = e.pieces == 1 ? nullptr : piece_slot<DP, 2>(p, e, kv_head, row) + (of_k ? DP * 128 : 0);
    __nv_bfloat16* dst = (of_k ? p.dk + (int64_t)key * p.k_stride : p.dv + (int64_t)key * p.v_stride) + (int64_t)kv_head * D;
    if (slot ? finite_piece<128>(slot, lo, hi) : finite_row(dst, lo, hi)) continue;
    const int first = e.lo + e.begin * p.tq, end = e.end == kAllSteps ? e.seq_hi : (int)min((int64_t)e.lo + (int64_t)e.end * p.tq, (int64_t)e.seq_hi);
    const int seen = max(first, key);
    if (!hidden_only(rows, head, p.group, D, first, min(key, end), seen, min(seen + kRows, end))) continue;
    float o[DP / 2];
#pragma unroll
    for (int c = 0; c < DP / 2; ++c) o[c] = 0.f;
    for (int i = seen; i < end; ++i)
      for (int h = head; h < head + p.group; ++h) {
        const float2 w = weight_and_slope(p, i, h, key, kv_head);
        row_add<DP / 2>(o, as_bf16(of_k ? w.y : w.x), rows.at(i, h, D), half * (DP / 16), D);
      }
    store_again<DP>(o, half, slot, dst, of_k ? p.scale : 1.f, D);
  }
}

// A ring of N tiles: `item` numbers the loads of a block, stage item % N.
template <int N>
struct Ring {
  uint32_t tiles;  // shared-memory address
  uint64_t *full, *empty;
  uint32_t tile_bytes;
  __device__ __forceinline__ uint32_t tile(uint32_t item) const { return tiles + (item % N) * tile_bytes; }
  __device__ __forceinline__ uint64_t* full_of(uint32_t item) const { return &full[item % N]; }
  __device__ __forceinline__ uint64_t* empty_of(uint32_t item) const { return &empty[item % N]; }
  __device__ __forceinline__ static uint32_t parity(uint32_t item) { return (item / N) & 1; }
};

template <int DP>
struct Loader {
  using R = BwdShape<DP>;
  uint64_t* raw;
  volatile uint32_t* abort_flag;
  int lane;
  uint32_t raw_turns = 0;
  bool ok = true;

  // Load number `item` of a ring: a box of `rows` rows of heads from `head` on, tokens from `row` on; rows
  // [valid, rows) belong to nobody and are zeroed.
  template <int N>
  __device__ __forceinline__ void load(const Ring<N>& ring, uint32_t item, uint8_t* tiles, const CUtensorMap* map,
                                       int head, int row, int rows, int valid) {
    ok = ok && warp_wait(ring.empty_of(item), ring.parity(item) ^ 1, abort_flag);
    if (!ok) return;
    const bool fix = valid < rows;
    uint64_t* bar = fix ? raw : ring.full_of(item);
    uint8_t* dst = tiles + (item % N) * R::kTile;
    if (lane == 0) {
      tc::mbar_arrive_expect_tx(bar, (uint32_t)rows * 128u * R::kNP);
      for (int c = 0; c < R::kNP; ++c)
        tma_load_3d(tc::smem_u32(dst + c * kPanel), map, bar, c * 64, head, row);
    }
    if (fix) {
      ok = warp_wait(raw, raw_turns & 1, abort_flag);
      ++raw_turns;
      if (!ok) return;
      zero_rows<R::kNP>(dst, valid, lane);
      if (lane == 0) tc::mbar_arrive(ring.full_of(item));
    }
  }

  // After a wait that gave up: the block must not leave with a copy in flight.
  template <int N>
  __device__ __forceinline__ void land(const Ring<N>& ring, uint32_t items) {
    uint32_t never = 0u;
    for (uint32_t i = items > (uint32_t)N ? items - N : 0; i < items; ++i)
      tc::mbar_wait(ring.full_of(i), ring.parity(i), &never, 1000000000ull), never = 0u;
  }
  __device__ __forceinline__ void land(uint64_t* bar, uint32_t turns) {
    uint32_t never = 0u;
    if (turns) tc::mbar_wait(bar, (turns - 1) & 1, &never, 1000000000ull);
  }
};

// 32 score columns of one thread: P = exp(scale S - lse), the subtrahends one for the row or one a column.
__device__ __forceinline__ float2 weight(float2 s, float2 scale, float2 minus_lse2) {
  const float2 x = fma2(s, scale, minus_lse2);
  return make_float2(ex2(x.x), ex2(x.y));
}

template <int DP>
__device__ __forceinline__ void dq_part(const CUtensorMap& map_q, const CUtensorMap& map_k, const CUtensorMap& map_v,
                                        const CUtensorMap& map_do, const BwdParams& p, uint32_t block,
                                        uint32_t blocks) {
  using R = BwdShape<DP>;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  bool fits;
  uint8_t* smem = tile_base(smem_raw, R::kSlack, &fits);
  if (!fits) {
    if (threadIdx.x == 0) atomicOr(p.status, NAT_DEV_TIMEOUT);
    return;
  }
  uint8_t *tiles_a = smem + 2 * R::kTile, *tiles_b = tiles_a + R::kA * R::kTile;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + R::kTiles + R::kStats);
  uint64_t *qdo_full = bars, *qdo_empty = bars + 1, *s_full = bars + 2, *dp_full = bars + 4, *ds_full = bars + 5;
  uint64_t *dq_done = bars + 6, *raw = bars + 7, *drain = bars + 8;
  const Ring<R::kA> ring_k{tc::smem_u32(tiles_a), bars + 10, bars + 10 + R::kA, R::kTile};
  const Ring<R::kB> ring_v{tc::smem_u32(tiles_b), bars + 10 + 2 * R::kA, bars + 10 + 2 * R::kA + R::kB, R::kTile};
  Found* const found = reinterpret_cast<Found*>(bars + 10 + 2 * (R::kA + R::kB));
  volatile uint32_t *abort_flag = &found->abort, *odd_flag = &found->odd;
  const int warp = uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    tc::mbar_init(qdo_full, 1);
    tc::mbar_init(qdo_empty, 2);  // by both MMA warps
    tc::mbar_init(&s_full[0], 1);
    tc::mbar_init(&s_full[1], 1);
    tc::mbar_init(dp_full, 1);
    tc::mbar_init(ds_full, 256);
    tc::mbar_init(dq_done, 1);
    tc::mbar_init(raw, 1);
    tc::mbar_init(drain, 2);
    for (int s = 0; s < 2 * (R::kA + R::kB); ++s) tc::mbar_init(&bars[10 + s], 1);
    *abort_flag = *odd_flag = 0u;
    tc::fence_barrier_init();
  }
  if (warp == 8) {
    tc::tmem_alloc(&found->tmem, 512);
    tc::tmem_relinquish();
  }
  if (warp == 9 && !p.list) find(p, block, found, true);
  wait_for_primary();
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = uniform(found->tmem);  // S/dS in two buffers, dP, dQ: 128 columns each
  const uint32_t units = (p.list ? *p.count : found->total) * (uint32_t)p.n_kv_heads;
  auto entry_of = [&](uint32_t u) { return p.list ? p.list[u / p.n_kv_heads] : found->entry; };
  // tiles of keys of a list entry
  auto tiles_of = [&](const Entry& e) {
    return min((min(e.lo + p.tq, e.seq_hi) - e.seq_lo + kRows - 1) / kRows, e.end) - e.begin;
  };

  if (warp == 9) {
    Loader<DP> ld{raw, abort_flag, lane};
    uint32_t turns = 0, item = 0;
    const int q_rows = p.group * p.tq;
    for (uint32_t u = block; ld.ok && u < units; u += blocks) {
      const Entry e = entry_of(u);
      const int head = (int)(u % p.n_kv_heads), n = tiles_of(e);
      ld.ok = warp_wait(qdo_empty, (turns & 1) ^ 1, abort_flag);
      if (!ld.ok) break;
      ++turns;
      if (lane == 0) {
        tc::mbar_arrive_expect_tx(qdo_full, 2u * (uint32_t)q_rows * 128u * R::kNP);
        for (int c = 0; c < R::kNP; ++c) {
          tma_load_3d(tc::smem_u32(smem + c * kPanel), &map_q, qdo_full, c * 64, head * p.group, e.lo);
          tma_load_3d(tc::smem_u32(smem + R::kTile + c * kPanel), &map_do, qdo_full, c * 64, head * p.group, e.lo);
        }
      }
      const int end = min(e.lo + p.tq, e.seq_hi);
      for (int j = 0; ld.ok && j < n; ++j, ++item) {
        const int row = e.seq_lo + (e.begin + j) * kRows;
        // K is also the second factor of dS K, where rows past the end must not count; V only
        // meets the mask of dS
        ld.load(ring_k, item, tiles_a, &map_k, head, row, kRows, min(end - row, kRows));
        if (ld.ok) ld.load(ring_v, item, tiles_b, &map_v, head, row, kRows, kRows);
      }
    }
    if (!ld.ok) {
      ld.land(raw, ld.raw_turns);
      ld.land(ring_k, item + 1);
      ld.land(ring_v, item + 1);
      ld.land(qdo_full, turns);
    }
  } else if (warp == 8 || warp == 10) {
    constexpr uint32_t kIdescD = tc::instr_desc_bf16(128, DP, 0, 1);
    const int ksteps = (p.head_dim + 15) / 16;
    const uint32_t q_addr = tc::smem_u32(smem), do_addr = q_addr + R::kTile;
    uint32_t turns = 0, tile = 0;  // `tile` numbers the key tiles of the block, and the items of both rings
    bool ok = true;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      ok = ok && warp_wait(bar, parity & 1, abort_flag);
      tc::fence_after_sync();
    };
    for (uint32_t u = block; ok && u < units; u += blocks) {
      const Entry e = entry_of(u);
      const int n = tiles_of(e);
      wait(qdo_full, turns);
      ++turns;
      if (warp == 10) {
        for (int j = 0; ok && j < n; ++j, ++tile) {  // S = Q K^T
          wait(ring_k.full_of(tile), ring_k.parity(tile));
          // the buffer's dS of two tiles before has been read when the K tile beside it is released
          if (tile >= 2) wait(ring_k.empty_of(tile - 2), ring_k.parity(tile - 2));
          if (ok && elect_one()) {
            product_kk<DP>(tmem + (tile & 1) * 128, q_addr, ring_k.tile(tile), ksteps);
            tc::umma_commit(&s_full[tile & 1]);
            if (j + 1 == n) tc::umma_commit(qdo_empty);
          }
          __syncwarp();
        }
      } else {
        auto slopes = [&](uint32_t i, bool last) {  // dP = dO V^T
          wait(ring_v.full_of(i), ring_v.parity(i));
          if (ok && elect_one()) {
            product_kk<DP>(tmem + 256, do_addr, ring_v.tile(i), ksteps);
            tc::umma_commit(dp_full);
            tc::umma_commit(ring_v.empty_of(i));
            if (last) tc::umma_commit(qdo_empty);
          }
          __syncwarp();
        };
        slopes(tile, n == 1);
        for (int j = 0; ok && j < n; ++j, ++tile) {
          wait(ds_full, tile);
          if (ok && elect_one()) {  // dQ += dS K, before dP of the next tile: S of the one after waits for it
            const uint32_t b = desc_mnmajor(ring_k.tile(tile)), a = tmem + (tile & 1) * 128;
#pragma unroll
            for (int kk = 0; kk < 8; ++kk)
              umma_ts(tmem + 384, a + half_cols(kk), b + step_mnmajor(kk), kIdescD, j > 0 || kk > 0);
            tc::umma_commit(ring_k.empty_of(tile));
            if (j + 1 == n) tc::umma_commit(dq_done);
          }
          __syncwarp();
          if (j + 1 < n) slopes(tile + 1, j + 2 == n);
        }
      }
    }
    if (elect_one()) tc::umma_commit(drain);
    uint32_t never = 0u;
    tc::mbar_wait(drain, 0, &never);
  } else if (warp < 8) {
    const int half = warp >> 2, row = threadIdx.x & 127;
    const uint32_t lane_base = (uint32_t)(warp & 3) * 32u << 16, mine = lane_base + half * 64;
    const int token_in = row / p.group, head_in = row % p.group;
    const float sc = p.scale * kLog2e;
    const bool wide = wide_rows(p.dq, p.q_stride, p.head_dim);
    uint32_t tile = 0, turns = 0;
    bool ok = true;
    for (uint32_t u = block; ok && u < units; u += blocks) {
      const Entry e = entry_of(u);
      const int n = tiles_of(e), token = e.lo + token_in;
      const int head = (int)(u % p.n_kv_heads) * p.group + head_in;
      const bool valid = row < p.group * p.tq && token < e.seq_hi;
      const int64_t at = (int64_t)token * p.n_heads + head;
      const float2 minus_lse2 = both(valid ? -__ldcg(p.lse2 + at) : 0.f);
      const float2 minus_delta = both(valid ? -__ldcg(p.delta + at) : 0.f);
      for (int j = 0; j < n; ++j, ++tile) {
        ok = warp_wait(&s_full[tile & 1], (tile >> 1) & 1, abort_flag);
        if (!ok) break;
        tc::fence_after_sync();
        const uint32_t s_addr = tmem + (tile & 1) * 128 + mine;
        float x[64], d[64];
        tmem_ld64(s_addr, x);
#pragma unroll
        for (int c = 0; c < 64; c += 2) {
          const float2 w = weight(make_float2(x[c], x[c + 1]), both(sc), minus_lse2);
          x[c] = w.x;
          x[c + 1] = w.y;
        }
        ok = warp_wait(dp_full, tile & 1, abort_flag);
        if (!ok) break;
        tc::fence_after_sync();
        tmem_ld64(tmem + 256 + mine, d);
#pragma unroll
        for (int c = 0; c < 64; c += 2) {
          const float2 g = mul2(make_float2(x[c], x[c + 1]), add2(make_float2(d[c], d[c + 1]), minus_delta));
          x[c] = g.x;
          x[c + 1] = g.y;
        }
        const int kv0 = e.seq_lo + (e.begin + j) * kRows;
        if (kv0 + kRows - 1 > e.lo) {  // the tile touches the diagonal
          const int last = token - kv0 - half * 64;
#pragma unroll
          for (int c = 0; c < 64; ++c)
            if (c > last) x[c] = 0.f;
        }
        store64(s_addr, x);
        tc::fence_before_sync();
        tc::mbar_arrive(ds_full);
      }
      if (!ok) break;
      ok = warp_wait(dq_done, turns & 1, abort_flag);
      if (!ok) break;
      ++turns;
      tc::fence_after_sync();
      __nv_bfloat16* dst = p.dq + (int64_t)token * p.q_stride + (int64_t)head * p.head_dim;
      float* slot = e.pieces == 1 ? nullptr : piece_slot<DP, 1>(p, e, (int)(u % p.n_kv_heads), row);
      const float2 odd = e.pieces == 1 ? store_acc<DP>(tmem + 384 + lane_base, half, dst, p.head_dim, p.scale, valid, wide)
                                       : store_piece<DP>(slot, tmem + 384 + lane_base, half);
      if (valid && !is_finite(odd)) *odd_flag = 1u;
      tc::fence_before_sync();
    }
  }

  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  if (threadIdx.x == 0 && *abort_flag) atomicOr(p.status, NAT_DEV_TIMEOUT);
  if (warp == 8) tc::tmem_dealloc(tmem, 512);
  if (warp < 8 && *odd_flag && !*abort_flag) mend_dq<DP>(p, &found->entry, units, block, blocks);
}

template <int DP>
__device__ __forceinline__ void dkv_part(const CUtensorMap& map_q, const CUtensorMap& map_k, const CUtensorMap& map_v,
                                        const CUtensorMap& map_do, const BwdParams& p, uint32_t block,
                                        uint32_t blocks) {
  using R = BwdShape<DP>;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  bool fits;
  uint8_t* smem = tile_base(smem_raw, R::kSlack, &fits);
  if (!fits) {
    if (threadIdx.x == 0) atomicOr(p.status, NAT_DEV_TIMEOUT);
    return;
  }
  uint8_t *tiles_a = smem + 2 * R::kTile, *tiles_b = tiles_a + R::kA * R::kTile;
  float* stats = reinterpret_cast<float*>(smem + R::kTiles);  // [2][-lse2 | -delta][128]
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + R::kTiles + R::kStats);
  // p_early: the first half of each thread's columns of P' is there
  uint64_t *kv_full = bars, *kv_empty = bars + 1, *s_full = bars + 2, *dp_full = bars + 3, *done = bars + 4;
  uint64_t *raw = bars + 5, *drain = bars + 6, *p_full = bars + 7, *ds_full = bars + 8, *p_early = bars + 9;
  uint64_t *st_full = bars + 10, *st_empty = bars + 12;
  const Ring<R::kA> ring_q{tc::smem_u32(tiles_a), bars + 14, bars + 14 + R::kA, R::kTile};
  const Ring<R::kB> ring_do{tc::smem_u32(tiles_b), bars + 14 + 2 * R::kA, bars + 14 + 2 * R::kA + R::kB, R::kTile};
  Found* const found = reinterpret_cast<Found*>(bars + 14 + 2 * (R::kA + R::kB));
  volatile uint32_t *abort_flag = &found->abort, *odd_flag = &found->odd;
  const int warp = uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int q_rows = p.group * p.tq;

  if (threadIdx.x == 0) {
    tc::mbar_init(kv_full, 1);
    tc::mbar_init(kv_empty, 2);  // by both MMA warps, like done and the slots of dO
    tc::mbar_init(s_full, 1);
    tc::mbar_init(p_full, 256);
    tc::mbar_init(dp_full, 1);
    tc::mbar_init(ds_full, 256);
    tc::mbar_init(done, 2);
    tc::mbar_init(raw, 1);
    tc::mbar_init(drain, 2);
    for (int s = 0; s < 2; ++s) {
      tc::mbar_init(&st_full[s], 1);
      tc::mbar_init(&st_empty[s], 8);
    }
    tc::mbar_init(p_early, 256);
    for (int s = 0; s < 2 * (R::kA + R::kB); ++s) tc::mbar_init(&bars[14 + s], s < 2 * R::kA + R::kB ? 1 : 2);
    *abort_flag = *odd_flag = 0u;
    tc::fence_barrier_init();
  }
  if (warp == 8) {
    tc::tmem_alloc(&found->tmem, 512);
    tc::tmem_relinquish();
  }
  if (q_rows < kRows) {
    // rows that no load reaches are part of every contraction over queries: zero, once
    for (uint32_t i = threadIdx.x; i < (R::kA + R::kB) * R::kTile / 16; i += blockDim.x)
      reinterpret_cast<uint4*>(tiles_a)[i] = make_uint4(0u, 0u, 0u, 0u);
    tc::fence_proxy_async();
  }
  if (warp == 9 && !p.list) find(p, block, found, false);
  wait_for_primary();
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = uniform(found->tmem);  // S'/P', dP'/dS', dV, dK: 128 columns each
  const uint32_t units = (p.list ? *p.count : found->total) * (uint32_t)p.n_kv_heads;
  auto entry_of = [&](uint32_t u) { return p.list ? p.list[u / p.n_kv_heads] : found->entry; };
  // tiles of queries of a list entry: they start at the key tile's first token
  auto tiles_of = [&](const Entry& e) { return min((e.seq_hi - e.lo + p.tq - 1) / p.tq, e.end) - e.begin; };

  if (warp == 9) {
    Loader<DP> ld{raw, abort_flag, lane};
    uint32_t turns = 0, item = 0;
    for (uint32_t u = block; ld.ok && u < units; u += blocks) {
      const Entry e = entry_of(u);
      const int head = (int)(u % p.n_kv_heads), n = tiles_of(e);
      auto load_q = [&](int j) {
        const int row = e.lo + (e.begin + j) * p.tq, valid = min((e.seq_hi - row) * p.group, q_rows);
        ld.load(ring_q, item, tiles_a, &map_q, head * p.group, row, q_rows, valid);
      };
      // the unit's first query tile does not wait for the end of the unit before
      load_q(0);
      if (!ld.ok) break;
      ld.ok = warp_wait(kv_empty, (turns & 1) ^ 1, abort_flag);
      if (!ld.ok) break;
      ++turns;
      if (lane == 0) {
        tc::mbar_arrive_expect_tx(kv_full, 2u * R::kTile);
        for (int c = 0; c < R::kNP; ++c) {
          tma_load_3d(tc::smem_u32(smem + c * kPanel), &map_k, kv_full, c * 64, head, e.lo);
          tma_load_3d(tc::smem_u32(smem + R::kTile + c * kPanel), &map_v, kv_full, c * 64, head, e.lo);
        }
      }
      for (int j = 0; ld.ok && j < n; ++j, ++item) {
        if (j > 0) load_q(j);
        const int row = e.lo + (e.begin + j) * p.tq, valid = min((e.seq_hi - row) * p.group, q_rows);
        if (ld.ok) ld.load(ring_do, item, tiles_b, &map_do, head * p.group, row, q_rows, valid);
      }
    }
    if (!ld.ok) {
      ld.land(raw, ld.raw_turns);
      ld.land(ring_q, item + 1);
      ld.land(ring_do, item + 1);
      ld.land(kv_full, turns);
    }
  } else if (warp == 11) {
    // lse and delta of the query rows, up to two tiles ahead
    uint32_t tile = 0;
    bool ok = true;
    for (uint32_t u = block; ok && u < units; u += blocks) {
      const Entry e = entry_of(u);
      const int head = (int)(u % p.n_kv_heads) * p.group, n = tiles_of(e);
      for (int j = 0; j < n; ++j, ++tile) {
        const int first = e.lo + (e.begin + j) * p.tq, valid = min((e.seq_hi - first) * p.group, q_rows);
        float a[4], b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = lane + 32 * i, token = first + r / p.group;
          const int64_t at = (int64_t)token * p.n_heads + head + r % p.group;
          a[i] = r < valid ? -__ldcg(p.lse2 + at) : 0.f;
          b[i] = r < valid ? -__ldcg(p.delta + at) : 0.f;
        }
        ok = warp_wait(&st_empty[tile & 1], ((tile >> 1) & 1) ^ 1, abort_flag);
        if (!ok) break;
        float* slot = stats + (tile & 1) * 2 * kRows;
#pragma unroll
        for (int i = 0; i < 4; ++i) slot[lane + 32 * i] = a[i], slot[kRows + lane + 32 * i] = b[i];
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&st_full[tile & 1]);
      }
    }
  } else if (warp == 8 || warp == 10) {
    constexpr uint32_t kIdescD = tc::instr_desc_bf16(128, DP, 0, 1);
    const int ksteps = (p.head_dim + 15) / 16;
    const uint32_t k_addr = tc::smem_u32(smem), v_addr = k_addr + R::kTile;
    uint32_t turns = 0, tile = 0;  // `tile` numbers the query tiles of the block, and the items of both rings
    bool ok = true;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      ok = ok && warp_wait(bar, parity & 1, abort_flag);
      tc::fence_after_sync();
    };
    // steps first, first + 1 and first + 4, first + 5 of a product with P' or dS': a half of each thread's columns
    auto half_steps = [&](uint32_t d, uint32_t a, uint32_t b, int first, bool add) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int kk = first + (k & 1) + (k >> 1) * 4;
        umma_ts(d, a + half_cols(kk), b + step_mnmajor(kk), kIdescD, add || k > 0);
      }
    };
    for (uint32_t u = block; ok && u < units; u += blocks) {
      const Entry e = entry_of(u);
      const int n = tiles_of(e);
      wait(kv_full, turns);
      ++turns;
      if (warp == 8) {
        auto scores = [&](uint32_t i) {  // S' = K Q^T
          wait(ring_q.full_of(i), ring_q.parity(i));
          if (ok && elect_one()) {
            product_kk<DP>(tmem, k_addr, ring_q.tile(i), ksteps);
            tc::umma_commit(s_full);
          }
          __syncwarp();
        };
        scores(tile);
        for (int j = 0; ok && j < n; ++j, ++tile) {  // dV += P' dO
          const uint32_t b = desc_mnmajor(ring_do.tile(tile));
          wait(ring_do.full_of(tile), ring_do.parity(tile));
          wait(p_early, tile);
          if (ok && elect_one()) half_steps(tmem + 256, tmem, b, 0, j > 0);
          __syncwarp();
          wait(p_full, tile);
          if (ok && elect_one()) {
            half_steps(tmem + 256, tmem, b, 2, true);
            tc::umma_commit(ring_do.empty_of(tile));
          }
          __syncwarp();
          if (j + 1 < n) scores(tile + 1);
        }
      } else {
        auto slopes = [&](uint32_t i) {  // dP' = V dO^T
          wait(ring_do.full_of(i), ring_do.parity(i));
          if (ok && elect_one()) {
            product_kk<DP>(tmem + 128, v_addr, ring_do.tile(i), ksteps);
            tc::umma_commit(dp_full);
            tc::umma_commit(ring_do.empty_of(i));
          }
          __syncwarp();
        };
        slopes(tile);
        for (int j = 0; ok && j < n; ++j, ++tile) {  // dK += dS' Q; S' of this tile was done before dS'
          const uint32_t b = desc_mnmajor(ring_q.tile(tile));
          wait(ds_full, tile);
          if (ok && elect_one()) {
            half_steps(tmem + 384, tmem + 128, b, 0, j > 0);
            half_steps(tmem + 384, tmem + 128, b, 2, true);
            tc::umma_commit(ring_q.empty_of(tile));
          }
          __syncwarp();
          if (j + 1 < n) slopes(tile + 1);
        }
      }
      if (ok && elect_one()) {
        tc::umma_commit(done);
        tc::umma_commit(kv_empty);
      }
      __syncwarp();
    }
    if (elect_one()) tc::umma_commit(drain);
    uint32_t never = 0u;
    tc::mbar_wait(drain, 0, &never);
  } else if (warp < 8) {
    const int half = warp >> 2, row = threadIdx.x & 127;
    const uint32_t lane_base = (uint32_t)(warp & 3) * 32u << 16, mine = lane_base + half * 64;
    const float sc = p.scale * kLog2e;
    const bool wide = wide_rows(p.dk, p.k_stride, p.head_dim) && wide_rows(p.dv, p.v_stride, p.head_dim);
    uint32_t tile = 0, turns = 0;
    bool ok = true;
    for (uint32_t u = block; ok && u < units; u += blocks) {
      const Entry e = entry_of(u);
      const int n = tiles_of(e), key = e.lo + row;
      for (int j = 0; j < n; ++j, ++tile) {
        const int first = e.lo + (e.begin + j) * p.tq, rows = min((e.seq_hi - first) * p.group, q_rows);
        const float4* slot = reinterpret_cast<const float4*>(stats + (tile & 1) * 2 * kRows + half * 64);
        ok = warp_wait(&st_full[tile & 1], (tile >> 1) & 1, abort_flag) && warp_wait(s_full, tile & 1, abort_flag);
        if (!ok) break;
        tc::fence_after_sync();
        float x[64], d[64];
        tmem_ld64(tmem + mine, x);
        // columns of queries before the key, and of rows that are not there
        const bool edge = first < e.lo + kRows || rows < kRows;
        const int c_lo = (key - first) * p.group - half * 64, c_hi = rows - half * 64;
        uint32_t packed[16];
#pragma unroll
        for (int part = 0; part < 2; ++part) {  // dV's first half runs during the second half's exponentials
#pragma unroll
          for (int c = part * 32; c < part * 32 + 32; c += 4) {
            const float4 l = slot[c / 4];
            const float2 v = weight(make_float2(x[c], x[c + 1]), both(sc), make_float2(l.x, l.y));
            const float2 w = weight(make_float2(x[c + 2], x[c + 3]), both(sc), make_float2(l.z, l.w));
            x[c] = v.x;
            x[c + 1] = v.y;
            x[c + 2] = w.x;
            x[c + 3] = w.y;
          }
          if (edge) {
#pragma unroll
            for (int c = part * 32; c < part * 32 + 32; ++c)
              if (c < c_lo || c >= c_hi) x[c] = 0.f;
          }
#pragma unroll
          for (int c = 0; c < 16; ++c) packed[c] = bf16_pair(x[part * 32 + 2 * c], x[part * 32 + 2 * c + 1]);
          tmem_st16(tmem + mine + part * 16, packed);
          tmem_st_wait();
          tc::fence_before_sync();
          tc::mbar_arrive(part == 0 ? p_early : p_full);
        }
        ok = warp_wait(dp_full, tile & 1, abort_flag);
        if (!ok) break;
        tc::fence_after_sync();
        tmem_ld64(tmem + 128 + mine, d);
#pragma unroll
        for (int c = 0; c < 64; c += 4) {
          const float4 l = slot[kRows / 4 + c / 4];
          const float2 v = mul2(make_float2(x[c], x[c + 1]), add2(make_float2(d[c], d[c + 1]), make_float2(l.x, l.y)));
          const float2 w = mul2(make_float2(x[c + 2], x[c + 3]), add2(make_float2(d[c + 2], d[c + 3]), make_float2(l.z, l.w)));
          x[c] = v.x;
          x[c + 1] = v.y;
          x[c + 2] = w.x;
          x[c + 3] = w.y;
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&st_empty[tile & 1]);
        if (edge) {  // zero times an infinity that another row left
#pragma unroll
          for (int c = 0; c < 64; ++c)
            if (c < c_lo || c >= c_hi) x[c] = 0.f;
        }
        store64(tmem + 128 + mine, x);
        tc::fence_before_sync();
        tc::mbar_arrive(ds_full);
      }
      if (!ok) break;
      ok = warp_wait(done, turns & 1, abort_flag);
      if (!ok) break;
      ++turns;
      tc::fence_after_sync();
      const bool valid = key < e.seq_hi;
      const int64_t col = (int64_t)(u % p.n_kv_heads) * p.head_dim;
      __nv_bfloat16 *dv = p.dv + (int64_t)key * p.v_stride + col, *dk = p.dk + (int64_t)key * p.k_stride + col;
      float* slot = e.pieces == 1 ? nullptr : piece_slot<DP, 2>(p, e, (int)(u % p.n_kv_heads), row);
      const float2 odd_v = e.pieces == 1 ? store_acc<DP>(tmem + 256 + lane_base, half, dv, p.head_dim, 1.f, valid, wide)
                                         : store_piece<DP>(slot, tmem + 256 + lane_base, half);
      const float2 odd_k = e.pieces == 1 ? store_acc<DP>(tmem + 384 + lane_base, half, dk, p.head_dim, p.scale, valid, wide)
                                         : store_piece<DP>(slot + DP * 128, tmem + 384 + lane_base, half);
      if (valid && !(is_finite(odd_v) && is_finite(odd_k))) *odd_flag = 1u;
      tc::fence_before_sync();
    }
  }

  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  if (threadIdx.x == 0 && *abort_flag) atomicOr(p.status, NAT_DEV_TIMEOUT);
  if (warp == 8) tc::tmem_dealloc(tmem, 512);
  if (warp < 8 && *odd_flag && !*abort_flag) {
    mend_dkv<DP>(p, false, &found->entry, units, block, blocks);
    mend_dkv<DP>(p, true, &found->entry, units, block, blocks);
  }
}

template <int DP>
__global__ void __launch_bounds__(384, 1)
attn_bwd_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_do,
                const __grid_constant__ BwdParams dq, const __grid_constant__ BwdParams dkv, unsigned dq_blocks) {
  if (blockIdx.x < dq_blocks)
    dq_part<DP>(map_q, map_k, map_v, map_do, dq, blockIdx.x, dq_blocks);
  else
    dkv_part<DP>(map_q, map_k, map_v, map_do, dkv, blockIdx.x - dq_blocks, gridDim.x - dq_blocks);
}

// Adds up the pieces of a tile, in their order: a block takes 16 columns of the 128 rows of a list entry (of
// dQ, or of dV and dK), a thread a row.
template <int DP>
__global__ void __launch_bounds__(128) attn_bwd_join_kernel(const BwdParams dq, const BwdParams dkv, unsigned dq_units) {
  wait_for_primary();
  const bool keys = blockIdx.x >= dq_units;
  const BwdParams& p = keys ? dkv : dq;
  const unsigned unit = keys ? blockIdx.x - dq_units : blockIdx.x;
  if (!p.partial || unit / p.n_kv_heads >= *p.count) return;
  const Entry e = p.list[unit / p.n_kv_heads];
  if (e.piece != 0 || e.pieces == 1) return;
  const int kv_head = (int)(unit % p.n_kv_heads), columns = keys ? 2 * DP : DP, row = threadIdx.x;
  if ((int)blockIdx.y * 16 >= columns) return;
  const int of = blockIdx.y * 16 / DP, col = blockIdx.y * 16 % DP;  // of keys: dV first, then dK
  const int token = keys ? e.lo + row : e.lo + row / p.group;
  if (token >= e.seq_hi || col >= p.head_dim || (!keys && row >= p.group * p.tq)) return;
  const int64_t size = 128 * columns, step = (int64_t)p.n_kv_heads * size;
  const float* slot = p.partial + ((int64_t)e.slot * p.n_kv_heads + kv_head) * size + blockIdx.y * 16 * 128 + row;
  float o[16];
#pragma unroll
  for (int k = 0; k < 16; ++k) o[k] = 0.f;
#pragma unroll 2
  for (int i = 0; i < e.pieces; ++i)
#pragma unroll
    for (int k = 0; k < 16; ++k) o[k] += slot[i * step + k * 128];
  __nv_bfloat16* dst =
      !keys ? p.dq + (int64_t)token * p.q_stride + (int64_t)(kv_head * p.group + row % p.group) * p.head_dim
            : (of == 0 ? p.dv + (int64_t)token * p.v_stride : p.dk + (int64_t)token * p.k_stride) +
                  (int64_t)kv_head * p.head_dim;
  const float f = keys && of == 0 ? 1.f : p.scale;
#pragma unroll
  for (int k = 0; k < 2; ++k)
    if (col + 8 * k < p.head_dim)
      *reinterpret_cast<uint4*>(dst + col + 8 * k) =
          make_uint4(bf16_pair(o[8 * k] * f, o[8 * k + 1] * f), bf16_pair(o[8 * k + 2] * f, o[8 * k + 3] * f),
                     bf16_pair(o[8 * k + 4] * f, o[8 * k + 5] * f), bf16_pair(o[8 * k + 6] * f, o[8 * k + 7] * f));
}

template <int DP>
int bwd(const Args& a, const Layout& l) {
  const nat_attn_params& p = a.p;
  const int group = p.n_heads / p.n_kv_heads, tq = kRows / group;
  Device dev;
  int s = device(&dev);
  CUtensorMap mq, mk, mv, mdo;
  if (s == NAT_OK) s = make_map(&mq, a.q, p.head_dim, p.n_heads, a.cap, p.q_stride, group, tq);
  if (s == NAT_OK) s = make_map(&mdo, a.dout, p.head_dim, p.n_heads, a.cap, p.o_stride, group, tq);
  if (s == NAT_OK) s = make_map(&mk, a.k, p.head_dim, p.n_kv_heads, a.cap, p.k_stride, 1, kRows);
  if (s == NAT_OK) s = make_map(&mv, a.v, p.head_dim, p.n_kv_heads, a.cap, p.v_stride, 1, kRows);
  static std::atomic<uint64_t> allowed;
  const size_t smem = BwdShape<DP>::kSmem;
  if (s == NAT_OK) s = allow_smem(attn_bwd_kernel<DP>, smem, dev, &allowed);
  if (s != NAT_OK) return s;
  const int64_t units_q = l.entries[kPlanDq] * p.n_kv_heads, units_k = l.entries[kPlanDkv] * p.n_kv_heads;
  const bool plan = units_q > dev.sms || units_k > dev.sms || l.split[kPlanDq] || l.split[kPlanDkv];
  s = launch_bwd_prologue(a, l, plan);
  if (s != NAT_OK) return s;
  BwdParams bp{};
  bp.status = &head(a)->status;
  bp.lse2 = lse2(a, l);
  bp.delta = delta(a, l);
  bp.dq = (__nv_bfloat16*)a.dq;
  bp.dk = (__nv_bfloat16*)a.dk;
  bp.dv = (__nv_bfloat16*)a.dv;
  bp.q_stride = p.q_stride;
  bp.k_stride = p.k_stride;
  bp.v_stride = p.v_stride;
  bp.n_heads = p.n_heads;
  bp.n_kv_heads = p.n_kv_heads;
  bp.group = group;
  bp.tq = tq;
  bp.head_dim = p.head_dim;
  bp.scale = p.scale;
  bp.q = {(const __nv_bfloat16*)a.q, p.q_stride};
  bp.k = {(const __nv_bfloat16*)a.k, p.k_stride};
  bp.v = {(const __nv_bfloat16*)a.v, p.v_stride};
  bp.dout = {(const __nv_bfloat16*)a.dout, p.o_stride};
  auto part = [&](Plan which) {
    BwdParams w = bp;
    w.list = plan ? entries(a, l, which) : nullptr;
    w.count = &head(a)->count[which];
    w.partial = l.split[which] ? partials(a, l, which) : nullptr;
    w.batch = batch(a, l, which);
    return w;
  };
  const unsigned blocks_q = (unsigned)min((int64_t)dev.sms, units_q), blocks_k = (unsigned)min((int64_t)dev.sms, units_k);
  const BwdParams dq = part(kPlanDq), dkv = part(kPlanDkv);
  s = launch_after(attn_bwd_kernel<DP>, dim3(blocks_q + blocks_k), 384, smem, a.stream, "attn_bwd_kernel", mq, mk, mv,
                   mdo, dq, dkv, blocks_q);
  if (s == NAT_OK && (l.split[kPlanDq] || l.split[kPlanDkv]))
    s = launch_after(attn_bwd_join_kernel<DP>, dim3((unsigned)(units_q + units_k), 2 * DP / 16), 128, 0, a.stream,
                     "attn_bwd_join_kernel", dq, dkv, (unsigned)units_q);
  return s;
}

}  // namespace

int bf16_bwd(const Args& a, const Layout& l) {
  return a.p.head_dim <= 64 ? bwd<64>(a, l) : bwd<128>(a, l);
}

}  // namespace attn
}  // namespace nat
