// Packed causal attention on the tensor cores (tcgen05 + TMEM + TMA), bfloat16.
//
// The query heads of a group are folded into the rows of a tile: a tile holds TQ = 128 / g tokens
// times the g heads that share a key head, row r = token (r / g), head (r % g), which one 3-D TMA
// box loads.  Grouped heads then share every key tile, and the diagonal of the causal mask
// wastes TQ tokens instead of 128.
//
// Forward, one persistent block per multiprocessor, twelve warps:
//   warps 0-3, 4-7  softmax of row tile 0 and 1: one thread a row, all 128 scores in registers
//   warp 8          issues the MMAs: S = Q K^T (both in shared memory), O += P V (P in tensor memory)
//   warp 9          TMA loads of Q, K, V through a ring (warps 10, 11 only lend their registers)
// Two row tiles alternate, so the tensor cores work on one while the other is in its softmax; they
// share K and V, which halves the operand feed.  Tensor memory: S0 S1 O0 O1, 128 columns each; P
// (bf16 pairs) overwrites the first half of its S.  O is rescaled only when a row's maximum has
// grown by more than 2^8 since the last time: P stays below 2^8 and the sums in fp32 lose nothing.
//
// 33,777 tokens in three sequences, 32 heads over 8, 128 columns: 3.08 ms, 1020 TFLOP/s counted, at the 1000 W
// cap (1580 MHz; 0.61 of the measured burst rate of a plain product, 0.74 of its sustained rate).
#include <cuda.h>

#include "nat_attn.cuh"
#include "nat_attn_masked.cuh"
#include "nat_attn_tc.cuh"

namespace nat {
namespace attn {
namespace {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kFar = 16777216.f;  // a shift above this (2^24) is off by more than half a unit
constexpr float kRescale = 8.f;  // growth of a row's maximum (log2) that is left in P

struct FwdParams {
  const Entry* list;  // null where every block has one unit at most and finds it itself
  Batch batch;
  const uint32_t* count;
  float* partial;
  uint32_t* status;
  __nv_bfloat16* out;
  float* lse;
  int64_t o_stride;
  int n_heads, n_kv_heads, group, tq, head_dim;
  float scale;
  Rows q, k, v;  // for mend_rows
};

template <int DP>
struct FwdShape {
  static constexpr int kNP = DP / 64;                       // 64-column panels of a tile
  static constexpr uint32_t kTile = kNP * kPanel;
  static constexpr int kStages = DP == 128 ? 4 : 8;
  static constexpr uint32_t kSmem = 1024 + (2 + kStages) * kTile + 512;
};

template <int DP>
constexpr __host__ __device__ int fwd_slot() {
  return 256 * (DP + 2);
}

// What all roles derive from a list entry.
struct Unit {
  int seq_lo, seq_hi, lo, head, kv_hi;
  int begin, nk[2];  // this piece's first key tile and, of each row tile, how many it has
  int slot, pieces;  // where its partial result goes, if it is not all
};
template <bool SPLIT>
__device__ __forceinline__ Unit unit_of(const FwdParams& p, const Entry* found, uint32_t u) {
  const Entry e = p.list ? p.list[u / p.n_kv_heads] : *found;
  Unit w;
  w.seq_lo = e.seq_lo;
  w.seq_hi = e.seq_hi;
  w.lo = e.lo;
  w.head = (int)(u % p.n_kv_heads);
  w.begin = SPLIT ? e.begin : 0;
  w.slot = SPLIT ? e.slot + e.piece : 0;
  w.pieces = SPLIT ? e.pieces : 1;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int first = e.lo + t * p.tq, end = min(first + p.tq, e.seq_hi);
    const int all = first < e.seq_hi ? (end - e.seq_lo + kRows - 1) / kRows : 0;
    w.nk[t] = SPLIT ? max(min(all, e.end) - e.begin, 0) : all;
  }
  w.kv_hi = min(e.lo + 2 * p.tq, e.seq_hi);
  return w;
}

// The rows of this block's units that masked values of v have spoilt, over the keys [first, token] of their piece; to
// the piece's slot or to out.  For the softmax's threads, each the row that it had.
template <int DP, bool SPLIT>
__device__ __noinline__ void mend_rows(const FwdParams& p, const Entry* found, uint32_t units) {
  const int t = threadIdx.x >> 7, row = threadIdx.x & 127, D = p.head_dim;
  const float sign = p.scale > 0.f ? 1.f : p.scale < 0.f ? -1.f : 0.f, sc = p.scale == 0.f ? 1.f : fabsf(p.scale) * kLog2e;
  for (uint32_t u = blockIdx.x; u < units; u += gridDim.x) {
    const Unit w = unit_of<SPLIT>(p, found, u);
    const int token = w.lo + t * p.tq + row / p.group, head = w.head * p.group + row % p.group;
    if (row >= p.group * p.tq || token >= w.seq_hi || w.nk[t] == 0) continue;
    float* piece = w.pieces == 1 ? nullptr : p.partial + ((int64_t)w.slot * p.n_kv_heads + w.head) * fwd_slot<DP>() + t * 128 + row;
    __nv_bfloat16* dst = p.out + (int64_t)token * p.o_stride + (int64_t)head * D;
    // the piece's maximum, or the row's log-sum: neither is finite where the softmax itself was not
    const float top = piece ? __ldcg(piece + DP * 256) : __ldcg(p.lse + (int64_t)token * p.n_heads + head);
    if (!(fabsf(top) < INFINITY) || (piece ? finite_piece<256>(piece, 0, D) : finite_row(dst, 0, D))) continue;
    const int first = w.seq_lo + w.begin * kRows, end = min(first + w.nk[t] * kRows, w.kv_hi);
    if (!hidden_only(p.v, w.head, 1, D, token + 1, end, max(first, token - (kRows - 1)), token + 1)) continue;
    float o[DP], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int c = 0; c < DP; ++c) o[c] = 0.f;
    for (int j = first; j <= token; ++j) {
      const float s = sign * row_dot(p.q.at(token, head, D), p.k.at(j, w.head, D), D);
      if (s == -INFINITY) continue;
      if (s > m) {
        const float f = ex2((m - s) * sc);
#pragma unroll
        for (int c = 0; c < DP; ++c) o[c] *= f;
        l *= f;
        m = s;
      }
      const float weight = ex2((s - m) * sc);
      l += weight;
      row_add<DP>(o, as_bf16(weight), p.v.at(j, w.head, D), 0, D);
    }
    const float inv = 1.f / l;
    if (piece) {
      __stcg(piece + DP * 256, m);
      __stcg(piece + (DP + 1) * 256, l);
    }
#pragma unroll
    for (int c = 0; c < DP; c += 8) {
      if (piece) {
#pragma unroll
        for (int i = 0; i < 8; ++i) __stcg(piece + (c + i) * 256, o[c + i]);
      } else if (c < D) {
        *reinterpret_cast<uint4*>(dst + c) = make_uint4(bf16_pair(o[c] * inv, o[c + 1] * inv), bf16_pair(o[c + 2] * inv, o[c + 3] * inv),
                                                        bf16_pair(o[c + 4] * inv, o[c + 5] * inv), bf16_pair(o[c + 6] * inv, o[c + 7] * inv));
      }
    }
  }
}

template <int DP, bool SPLIT>  // SPLIT: some tiles come in pieces
__global__ void __launch_bounds__(384, 1)
attn_fwd_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                const __grid_constant__ CUtensorMap map_v, const __grid_constant__ FwdParams p) {
  using R = FwdShape<DP>;
  constexpr int kNS = R::kStages;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* ring = smem + 2 * R::kTile;
  uint64_t* bars = reinterpret_cast<uint64_t*>(ring + kNS * R::kTile);
  uint64_t *q_full = bars, *q_empty = bars + 2, *s_full = bars + 4, *o_done = bars + 6, *raw = bars + 8;
  uint64_t *drain = bars + 9, *p_full = bars + 10;  // p_full [row tile][half of the keys]
  uint64_t *full = bars + 14, *empty = bars + 14 + kNS;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 14 + 2 * kNS);  // address, abort flag, total, odd flag
  volatile uint32_t *abort_flag = tmem_slot + 1, *odd_flag = tmem_slot + 3;
  Entry* found = reinterpret_cast<Entry*>(tmem_slot + 4);
  const int warp = uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int t = 0; t < 2; ++t) {
      tc::mbar_init(&q_full[t], 1);
      tc::mbar_init(&q_empty[t], 1);
      tc::mbar_init(&s_full[t], 1);
      tc::mbar_init(&p_full[2 * t], 128);
      tc::mbar_init(&p_full[2 * t + 1], 128);
      tc::mbar_init(&o_done[t], 1);
    }
    tc::mbar_init(raw, 1);
    tc::mbar_init(drain, 1);
    for (int s = 0; s < kNS; ++s) {
      tc::mbar_init(&full[s], 1);
      tc::mbar_init(&empty[s], 1);
    }
    *abort_flag = *odd_flag = 0u;
    tc::fence_barrier_init();
  }
  if (warp == 8) {
    tc::tmem_alloc(tmem_slot, 512);
    tc::tmem_relinquish();
  }
  if (warp == 9 && !p.list) {
    uint32_t total, status;
    const Entry e = find_entry(p.batch, blockIdx.x / p.n_kv_heads, &total, &status);
    if (lane == 0) {
      *found = e;
      tmem_slot[2] = total;
      if (blockIdx.x == 0) *p.status = status;
    }
  }
  wait_for_primary();
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = uniform(*tmem_slot);
  const uint32_t units = (p.list ? *p.count : tmem_slot[2]) * (uint32_t)p.n_kv_heads;

  // 168 registers a thread at launch: the softmax warpgroups, which hold a row of scores, take
  // some of the third's (2 x 192 + 120 = 3 x 168)
  if (warp >= 8) {
    regs_dec<120>();
    if (warp == 9) {
      // ---------------------------------------------------------------- loads
      uint32_t item = 0, raw_turns = 0, q_turns[2] = {0, 0};
      bool ok = true;
      const uint32_t q_bytes = (uint32_t)(p.group * p.tq) * 128u * R::kNP;
      auto load_q = [&](const Unit& w, int t) {
        if (w.nk[t] == 0) return;
        ok = ok && warp_wait(&q_empty[t], (q_turns[t] & 1) ^ 1, abort_flag);
        if (!ok) return;
        ++q_turns[t];
        if (lane == 0) {
          tc::mbar_arrive_expect_tx(&q_full[t], q_bytes);
          for (int c = 0; c < R::kNP; ++c)
            tma_load_3d(tc::smem_u32(smem + t * R::kTile + c * kPanel), &map_q, &q_full[t], c * 64,
                        w.head * p.group, w.lo + t * p.tq);
        }
      };
      auto load_kv = [&](const CUtensorMap* map, const Unit& w, int j, bool is_v) {
        const int s = item % kNS;
        ok = ok && warp_wait(&empty[s], ((item / kNS) & 1) ^ 1, abort_flag);
        if (!ok) return;
        ++item;
        const int row = w.seq_lo + (w.begin + j) * kRows, valid = w.kv_hi - row;
        const bool fix = is_v && valid < kRows;
        uint64_t* bar = fix ? raw : &full[s];
        uint8_t* dst = ring + s * R::kTile;
        if (lane == 0) {
          tc::mbar_arrive_expect_tx(bar, R::kTile);
          for (int c = 0; c < R::kNP; ++c)
            tma_load_3d(tc::smem_u32(dst + c * kPanel), map, bar, c * 64, w.head, row);
        }
        if (fix) {
          ok = warp_wait(raw, raw_turns & 1, abort_flag);
          ++raw_turns;
          if (!ok) return;
          zero_rows<R::kNP>(dst, valid, lane);
          if (lane == 0) tc::mbar_arrive(&full[s]);
        }
      };
      for (uint32_t u = blockIdx.x; ok && u < units; u += gridDim.x) {
        const Unit w = unit_of<SPLIT>(p, found, u);
        const int n = max(w.nk[0], w.nk[1]);
        for (int j = 0; ok && j < n; ++j) {
          if (j == 0) load_q(w, 0);
          load_kv(&map_k, w, j, false);
          if (j == 0) load_q(w, 1);
          load_kv(&map_v, w, j, true);
        }
      }
      // the block must not leave with a copy in flight: every tile that was loaded has to have landed
      if (!ok) {
        uint32_t never = 0u;
        if (raw_turns) tc::mbar_wait(raw, (raw_turns - 1) & 1, &never, 1000000000ull), never = 0u;
        for (uint32_t i = item > (uint32_t)kNS ? item - kNS : 0; i < item; ++i)
          tc::mbar_wait(&full[i % kNS], (i / kNS) & 1, &never, 1000000000ull), never = 0u;
        for (int t = 0; t < 2; ++t)
          if (q_turns[t]) tc::mbar_wait(&q_full[t], (q_turns[t] - 1) & 1, &never, 1000000000ull), never = 0u;
      }
    } else if (warp == 8) {
      // ---------------------------------------------------------------- MMAs
      constexpr uint32_t kIdescO = tc::instr_desc_bf16(128, DP, 0, 1);
      const int ksteps = (p.head_dim + 15) / 16;
      const uint32_t q_addr = tc::smem_u32(smem), ring_addr = tc::smem_u32(ring);
      uint32_t item = 0, q_turns = 0, p_turns = 0;  // bit t of q_turns, p_turns: the next phase of row tile t
      bool ok = true;
      auto wait = [&](uint64_t* bar, uint32_t parity) {
        ok = ok && warp_wait(bar, parity & 1, abort_flag);
        tc::fence_after_sync();
      };
      auto scores = [&](int t, uint32_t k_item, bool last) {
        if (elect_one()) {
          product_kk<DP>(tmem + t * 128, q_addr + t * R::kTile, ring_addr + (k_item % kNS) * R::kTile, ksteps);
          tc::umma_commit(&s_full[t]);  // which also says that O += P V of the step before is complete
          if (last) tc::umma_commit(&q_empty[t]);
        }
        __syncwarp();
      };
      auto release = [&](uint32_t i) {
        if (elect_one()) tc::umma_commit(&empty[i % kNS]);
        __syncwarp();
      };
      for (uint32_t u = blockIdx.x; ok && u < units; u += gridDim.x) {
        const Unit w = unit_of<SPLIT>(p, found, u);
        const int n = max(w.nk[0], w.nk[1]);
        // the unit's items are K_0 V_0 K_1 V_1 ...: K_j is item + 2 j, V_j the next
        wait(&full[item % kNS], item / kNS);
#pragma unroll
        for (int t = 0; t < 2; ++t)
          if (w.nk[t]) {
            wait(&q_full[t], q_turns >> t);
            q_turns ^= 1u << t;
            if (!ok) break;
            scores(t, item, w.nk[t] == 1);
          }
        if (!ok) break;
        release(item);
        for (int j = 0; ok && j < n; ++j) {
          const uint32_t v_item = item + 2 * j + 1, k_next = v_item + 1;
          wait(&full[v_item % kNS], v_item / kNS);
          if (j + 1 < n) wait(&full[k_next % kNS], k_next / kNS);
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (j >= w.nk[t] || !ok) continue;
            const uint32_t b = desc_mnmajor(ring_addr + (v_item % kNS) * R::kTile);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              wait(&p_full[2 * t + half], p_turns >> t);
              if (!ok) break;
              if (elect_one()) {
#pragma unroll
                for (int kk = half * 4; kk < half * 4 + 4; ++kk)
                  umma_ts(tmem + 256 + t * 128, tmem + t * 128 + kk * 8, b + step_mnmajor(kk), kIdescO, j > 0 || kk > 0);
                if (half == 1 && j + 1 == w.nk[t]) tc::umma_commit(&o_done[t]);
              }
              __syncwarp();
            }
            p_turns ^= 1u << t;
            if (ok && j + 1 < w.nk[t]) scores(t, k_next, j + 2 == w.nk[t]);
          }
          if (!ok) break;
          release(v_item);
          if (j + 1 < n) release(k_next);
        }
        item += 2 * n;
      }
      // every MMA has to have finished before the tensor memory is given back
      if (elect_one()) tc::umma_commit(drain);
      uint32_t never = 0u;
      tc::mbar_wait(drain, 0, &never);
    }
  } else {
    // ------------------------------------------------------------- softmax
    regs_inc<192>();
    const int t = warp >> 2, row = threadIdx.x & 127;
    const uint32_t lane_base = (uint32_t)(warp & 3) * 32u << 16;
    const uint32_t s_addr = tmem + t * 128 + lane_base, o_addr = tmem + 256 + t * 128 + lane_base;
    const int token_in = row / p.group, head_in = row % p.group;
    // the maximum is taken before the scale, which therefore has to be positive: a negative one
    // gives its sign, and zero itself, to the scores
    const float sign = p.scale > 0.f ? 1.f : p.scale < 0.f ? -1.f : 0.f;
    const bool wide = wide_rows(p.out, p.o_stride, p.head_dim);
    const float sc = p.scale == 0.f ? 1.f : fabsf(p.scale) * kLog2e;
    uint32_t s_turns = 0, o_turns = 0;
    bool ok = true;
    for (uint32_t u = blockIdx.x; ok && u < units; u += gridDim.x) {
      const Unit w = unit_of<SPLIT>(p, found, u);
      const int nk = w.nk[t], first = w.lo + t * p.tq, token = first + token_in;
      const bool valid = row < p.group * p.tq && token < w.seq_hi;
      float m = -INFINITY, l = 0.f;
      for (int j = 0; j < nk; ++j) {
        ok = warp_wait(&s_full[t], s_turns & 1, abort_flag);
        ++s_turns;
        if (!ok) break;
        tc::fence_after_sync();
        uint32_t sr[128];
#pragma unroll
        for (int c = 0; c < 4; ++c) tc::tmem_ld32_issue(s_addr + c * 32, sr + c * 32);
        tc::tmem_ld_wait(sr);
#pragma unroll
        for (int c = 1; c < 4; ++c) tc::tmem_ld_pin(sr + c * 32);
        float s[128];
#pragma unroll
        for (int c = 0; c < 128; ++c) s[c] = __uint_as_float(sr[c]);
        if (sign != 1.f) {
#pragma unroll
          for (int c = 0; c < 128; ++c) s[c] *= sign;
        }
        const int kv0 = w.seq_lo + (w.begin + j) * kRows;
        if (kv0 + kRows - 1 > first) {  // the tile touches the diagonal
          const int last = token - kv0;
#pragma unroll
          for (int c = 0; c < 128; ++c)
            if (c > last) s[c] = -INFINITY;
        }
        float top[4] = {m, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int c = 0; c < 128; c += 8)
#pragma unroll
          for (int i = 0; i < 4; ++i) top[i] = max3(top[i], s[c + 2 * i], s[c + 2 * i + 1]);
        const float now = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
        float base = m;
        if (j == 0) {
          m = base = now;
        } else {
          const bool grow = valid && (now - m) * sc > kRescale;
          if (__any_sync(0xFFFFFFFFu, grow)) {  // O is at rest: s_full came after the step before
            const float f = grow ? ex2((m - now) * sc) : 1.f;
            if (grow) m = now;
            l *= f;
#pragma unroll
            for (int c = 0; c < DP / 16; ++c) {  // few columns at a time: the scores stay in registers
              uint32_t o[16];
              tmem_ld16(o_addr + c * 16, o);
#pragma unroll
              for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
              tmem_st16(o_addr + c * 16, o);
            }
            base = m;
          }
        }
        // a row whose scores are all minus infinity so far has no maximum to subtract
        float shift = base == -INFINITY ? 0.f : base * sc;
        // The fused subtraction below leaves the rounding of the shift in every exponent.  It cancels in out, but of scores
        // beyond 2^30 it would take the weights out of range: there the maximum is subtracted first.
        if (__any_sync(0xFFFFFFFFu, fabsf(shift) > kFar)) {
          const float far = fabsf(shift) > kFar ? base : 0.f;
          if (far != 0.f) shift = 0.f;
#pragma unroll
          for (int c = 0; c < 128; ++c) s[c] -= far;
        }
        const float2 scale2 = {sc, sc}, shift2 = {-shift, -shift};
        float2 sum[2] = {{0.f, 0.f}, {0.f, 0.f}};
        // P goes out in halves: the first one's product runs during the second one's exponentials
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t pk[32];
#pragma unroll
          for (int c = 0; c < 32; ++c) {
            float2 e = fma2({s[half * 64 + 2 * c], s[half * 64 + 2 * c + 1]}, scale2, shift2);
            e.x = ex2(e.x);
            e.y = ex2(e.y);
            sum[c & 1] = add2(sum[c & 1], e);
            pk[c] = bf16_pair(e.x, e.y);
          }
          tmem_st32(s_addr + half * 32, pk);
          tmem_st_wait();
          tc::fence_before_sync();
          tc::mbar_arrive(&p_full[2 * t + half]);
        }
        sum[0] = add2(sum[0], sum[1]);
        l += sum[0].x + sum[0].y;
      }
      if (!ok) break;
      if (nk == 0 && w.pieces == 1) continue;
      if (nk > 0) {
        ok = warp_wait(&o_done[t], o_turns & 1, abort_flag);
        if (!ok) break;
        ++o_turns;
        tc::fence_after_sync();
      }
      const int head = w.head * p.group + head_in;
      __nv_bfloat16* dst = p.out + (int64_t)token * p.o_stride + (int64_t)head * p.head_dim;
      float* lse = p.lse + (int64_t)token * p.n_heads + head;
      float2 odd = {0.f, 0.f};
      if (w.pieces == 1) {
        const float inv = 1.f / l;
#pragma unroll
        for (int c = 0; c < DP / 32; ++c) {
          float o[32];
          tc::tmem_ld32(o_addr + c * 32, o);
          odd = finite32(o, odd);
          if (valid) store_row32(dst + c * 32, o, inv, p.head_dim - c * 32, wide);
        }
        if (valid) *lse = fmaf(m, sc * kLn2, logf(l));
      } else {
        // this piece's O, maximum and sum, [column][row]
        float* own = p.partial + ((int64_t)w.slot * p.n_kv_heads + w.head) * fwd_slot<DP>() + t * 128 + row;
        if (nk > 0) {
#pragma unroll
          for (int c = 0; c < DP / 32; ++c) {
            float o[32];
            tc::tmem_ld32(o_addr + c * 32, o);
            odd = finite32(o, odd);
#pragma unroll
            for (int i = 0; i < 32; ++i) __stcg(own + (c * 32 + i) * 256, o[i]);
          }
        }
        __stcg(own + DP * 256, nk > 0 ? m : -INFINITY);
        __stcg(own + (DP + 1) * 256, nk > 0 ? l : 0.f);
      }
      if (valid && !is_finite(odd)) *odd_flag = 1u;
      tc::fence_before_sync();
    }
  }

  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  if (threadIdx.x == 0 && *abort_flag) atomicOr(p.status, NAT_DEV_TIMEOUT);
  if (warp == 8) tc::tmem_dealloc(tmem, 512);
  if (warp < 8 && *odd_flag && !*abort_flag) mend_rows<DP, SPLIT>(p, found, units);
}

// Joins the pieces of a tile, in their order: a block takes 16 columns of the 256 rows of a list entry, a
// thread a row.  out = sum_i w_i O_i / sum_i w_i l_i with w_i = exp(m_i - max m).
template <int DP>
__global__ void __launch_bounds__(256) attn_fwd_join_kernel(const FwdParams p) {
  wait_for_primary();
  if (blockIdx.x / p.n_kv_heads >= *p.count) return;
  const Entry e = p.list[blockIdx.x / p.n_kv_heads];
  if (e.piece != 0 || e.pieces == 1) return;
  const int kv_head = (int)(blockIdx.x % p.n_kv_heads), col = blockIdx.y * 16, row = threadIdx.x & 127;
  const int token = e.lo + (threadIdx.x >> 7) * p.tq + row / p.group, head = kv_head * p.group + row % p.group;
  if (row >= p.group * p.tq || token >= e.seq_hi || col >= p.head_dim) return;
  const float sign_scale = p.scale == 0.f ? 1.f : fabsf(p.scale) * kLog2e;
  const int64_t step = (int64_t)p.n_kv_heads * fwd_slot<DP>();
  const float* slot = p.partial + ((int64_t)e.slot * p.n_kv_heads + kv_head) * fwd_slot<DP>() + threadIdx.x;
  float top = -INFINITY;
#pragma unroll 4
  for (int i = 0; i < e.pieces; ++i) top = fmaxf(top, slot[i * step + DP * 256]);
  const float base = top == -INFINITY ? 0.f : top;
  float sum = 0.f, o[16];
#pragma unroll
  for (int k = 0; k < 16; ++k) o[k] = 0.f;
#pragma unroll 2
  for (int i = 0; i < e.pieces; ++i) {
    const float* from = slot + i * step;
    const float m = from[DP * 256], f = ex2((m - base) * sign_scale);
    sum = fmaf(f, from[(DP + 1) * 256], sum);
    if (m == -INFINITY) continue;  // a piece without keys for this row, whose O may not be there
#pragma unroll
    for (int k = 0; k < 16; ++k) o[k] = fmaf(f, from[(col + k) * 256], o[k]);
  }
  const float inv = 1.f / sum;
  __nv_bfloat16* dst = p.out + (int64_t)token * p.o_stride + (int64_t)head * p.head_dim + col;
#pragma unroll
  for (int k = 0; k < 2; ++k)
    if (col + 8 * k < p.head_dim)
      *reinterpret_cast<uint4*>(dst + 8 * k) =
          make_uint4(bf16_pair(o[8 * k] * inv, o[8 * k + 1] * inv), bf16_pair(o[8 * k + 2] * inv, o[8 * k + 3] * inv),
                     bf16_pair(o[8 * k + 4] * inv, o[8 * k + 5] * inv), bf16_pair(o[8 * k + 6] * inv, o[8 * k + 7] * inv));
  if (col == 0) p.lse[(int64_t)token * p.n_heads + head] = fmaf(base, sign_scale * kLn2, logf(sum));
}

// ------------------------------------------------------------------------- host side
using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                                   const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                   const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                   CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

int get_encoder(EncodeTiledFn* out) {
  static EncodeTiledFn cached = nullptr;
  if (!cached) {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult qres;
    NAT_CUDA(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres));
    if (qres != cudaDriverEntryPointSuccess || !fn)
      return fail(NAT_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
    cached = reinterpret_cast<EncodeTiledFn>(fn);
  }
  *out = cached;
  return NAT_OK;
}

}  // namespace

// [cap, heads, D] with a token stride; a box of 64 columns x box_heads x box_tokens, zero outside.
int make_map(CUtensorMap* map, const void* base, int D, int heads, int64_t cap, int64_t stride,
             int box_heads, int box_tokens) {
  EncodeTiledFn enc;
  int s = get_encoder(&enc);
  if (s != NAT_OK) return s;
  const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)heads, (cuuint64_t)cap};
  const cuuint64_t strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)stride * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_tokens};
  const cuuint32_t estr[3] = {1, 1, 1};
  const CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides,
                         box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                         CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return fail(NAT_ERR_CUDA, "cuTensorMapEncodeTiled failed with code %d", (int)r);
  return NAT_OK;
}

namespace {

template <int DP>
int fwd(const Args& a, const Layout& l) {
  const nat_attn_params& p = a.p;
  const int group = p.n_heads / p.n_kv_heads, tq = kRows / group;
  Device dev;
  int s = device(&dev);
  CUtensorMap mq, mk, mv;
  if (s == NAT_OK) s = make_map(&mq, a.q, p.head_dim, p.n_heads, a.cap, p.q_stride, group, tq);
  if (s == NAT_OK) s = make_map(&mk, a.k, p.head_dim, p.n_kv_heads, a.cap, p.k_stride, 1, kRows);
  if (s == NAT_OK) s = make_map(&mv, a.v, p.head_dim, p.n_kv_heads, a.cap, p.v_stride, 1, kRows);
  if (s != NAT_OK) return s;
  const bool split = l.split[kPlanFwd];
  const auto kernel = split ? attn_fwd_kernel<DP, true> : attn_fwd_kernel<DP, false>;
  static std::atomic<uint64_t> allowed[2];
  s = allow_smem(kernel, FwdShape<DP>::kSmem, dev, &allowed[split ? 1 : 0]);
  if (s != NAT_OK) return s;
  const int64_t units = l.entries[kPlanFwd] * p.n_kv_heads;
  const bool plan = units > dev.sms || split;
  if (plan) s = launch_plan(a, l, kPlanFwd);
  if (s != NAT_OK) return s;
  FwdParams fp{};
  fp.list = plan ? entries(a, l, kPlanFwd) : nullptr;
  fp.batch = batch(a, l, kPlanFwd);
  fp.count = &head(a)->count[kPlanFwd];
  fp.partial = partials(a, l, kPlanFwd);
  fp.status = &head(a)->status;
  fp.out = (__nv_bfloat16*)a.out;
  fp.lse = a.lse;
  fp.o_stride = p.o_stride;
  fp.n_heads = p.n_heads;
  fp.n_kv_heads = p.n_kv_heads;
  fp.group = group;
  fp.tq = tq;
  fp.head_dim = p.head_dim;
  fp.scale = p.scale;
  fp.q = {(const __nv_bfloat16*)a.q, p.q_stride};
  fp.k = {(const __nv_bfloat16*)a.k, p.k_stride};
  fp.v = {(const __nv_bfloat16*)a.v, p.v_stride};
  const unsigned grid = (unsigned)min((int64_t)dev.sms, units);
  const size_t smem = FwdShape<DP>::kSmem;
  if (plan) {
    s = launch_after(kernel, dim3(grid), 384, smem, a.stream, "attn_fwd_kernel", mq, mk, mv, fp);
    if (s == NAT_OK && split)
      s = launch_after(attn_fwd_join_kernel<DP>, dim3((unsigned)units, DP / 16), 256, 0, a.stream,
                       "attn_fwd_join_kernel", fp);
    return s;
  }
  kernel<<<grid, 384, smem, a.stream>>>(mq, mk, mv, fp);
  NAT_LAUNCH_CHECK("attn_fwd_kernel");
  return NAT_OK;
}

}  // namespace

int bf16_fwd(const Args& a, const Layout& l) {
  return a.p.head_dim <= 64 ? fwd<64>(a, l) : fwd<128>(a, l);
}

}  // namespace attn
}  // namespace nat
