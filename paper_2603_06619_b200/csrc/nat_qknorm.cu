// The heads' norms of queries and keys with the rotation by position, forward and backward.
//
//   n = x rstd w,  out = rot_p(n)          g = rot_{-p}(dout),  dx = rstd (g w - xhat mean(g w xhat)),  dw = sum g xhat
//
// Bound by HBM: one pass over the rows.  LANES lanes share a head's row, two chunks of eight elements each, chosen so
// that both members of a rotated pair are in one lane; a warp owns a token and walks its heads, so that the angles'
// sines and cosines are found once a token, each by one of the warp's groups of lanes, and dealt to the others.  A warp
// takes a run of consecutive tokens and finds its first token's sequence once; its rows are on their way into
// shared memory three steps ahead.  156,000 tokens of 32 and 8 heads of 128 in bfloat16 forward, one call after the other:
// 532 us, 0.92 of the copy rate at the board's power limit (a lone call 480 us, 1.02), 160,000 backward 800 us, 0.94.
// At that limit instructions count: weights and rotation in one (forward), one exchange of two sums for a row (backward)
// and packed arithmetic took these from 576 and 914 us.
#include <atomic>
#include <initializer_list>

#include "nat_common.cuh"
#include "nat_rows.cuh"

namespace nat {
namespace qknorm {
namespace {

using rows::kChunk;
using rows::kPairs;
using rows::Raw;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxDim = 128;

struct Args {
  nat_qknorm_params p;
  int32_t B;
  const int32_t *cu, *positions, *n_rows;
  int64_t cap;
  const void *q, *k;
  const float *w_q, *w_k;
  const double* inv_freq;
  const void *dq_out, *dk_out;   // backward
  void *q_to, *k_to;             // q_out and k_out, or dq and dk
  float* partial;                // backward with norms: [blocks][2][head_dim]
};

// Rows [first, end) of the call: those of the sequences, where there are any, whether or not the positions are given.
__device__ __forceinline__ void row_range(const Args& a, int64_t& first, int64_t& end) {
  end = a.n_rows ? min((int64_t)max(__ldg(a.n_rows), 0), a.cap) : a.cap;
  first = 0;
  if (a.cu) {
    first = max(__ldg(a.cu), 0);
    end = max(first, min(end, (int64_t)max(__ldg(a.cu + a.B), 0)));
  }
}

// The last sequence that begins at or before row n (0 where none does).
__device__ __forceinline__ int owner(const int32_t* cu, int B, int64_t n) {
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if ((int64_t)__ldg(cu + mid) <= n) lo = mid; else hi = mid;
  }
  return lo;
}

// A lane's two chunks of a head's row and the pairs that they hold.  First chunks of neighbouring lanes lie side by side,
// and second ones: whole sectors at a time (a lane's two side by side instead, for the elements that do not turn: 160,000
// tokens of 32 and 8 heads of 128 of which 64 turn forward 657 us, 564 like this; backward 1004, 839).
struct Slot {
  int a, b;        // first elements; b < 0: none
  bool turns, in;  // the lane has a part of the row at all
};
__device__ __forceinline__ Slot slot_of(const nat_qknorm_params& p, int lane) {
  const int r16 = p.rot_dim / 16, rest = (p.head_dim - p.rot_dim) / kChunk;
  if (lane < r16) return {lane * kChunk, (lane + r16) * kChunk, true, true};
  const int j = lane - r16, half = (rest + 1) / 2;
  if (j >= half) return {0, -1, false, false};
  return {p.rot_dim + j * kChunk, j + half < rest ? p.rot_dim + (j + half) * kChunk : -1, false, true};
}
// Number i of the angle of the lane's e-th pair.
template <bool INTER>
__device__ __forceinline__ int angle_of(const Slot& s, int e) {
  if (!INTER) return s.a + e;
  return e < 4 ? s.a / 2 + e : s.b / 2 + e - 4;
}

__device__ __forceinline__ float2 swapped(float2 x) { return make_float2(x.y, x.x); }

__device__ __forceinline__ void read8(const float* w, float2 (&x)[kPairs]) {
#pragma unroll
  for (int i = 0; i < kPairs; i += 2) {
    const float4 v = *reinterpret_cast<const float4*>(w + 2 * i);
    x[i] = make_float2(v.x, v.y);
    x[i + 1] = make_float2(v.z, v.w);
  }
}

// Forward, the weights and the rotation of a lane's two chunks in one: each pair of elements becomes
//   pair own + other across,
// other being the same pair of the other chunk, or, with INTER, the pair itself the other way round.
struct Turn {
  float2 own[2][kPairs], across[2][kPairs];
};
template <bool INTER, bool NORM>
__device__ __forceinline__ void make_turn(Turn& t, const Slot& slot, const float* w, const float (&c)[8], const float (&s)[8]) {
  float2 wt[2][kPairs];
  if (NORM) {
    read8(w + slot.a, wt[0]);
    read8(w + max(slot.b, 0), wt[1]);
  }
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      const float2 cs = INTER ? both(c[4 * k + i]) : make_float2(c[2 * i], c[2 * i + 1]);
      const float2 sn = INTER ? both(s[4 * k + i]) : make_float2(s[2 * i], s[2 * i + 1]);
      const float2 self = NORM ? wt[k][i] : both(1.f), over = NORM ? (INTER ? swapped(wt[k][i]) : wt[1 - k][i]) : both(1.f);
      t.own[k][i] = slot.turns ? (NORM ? mul2(self, cs) : cs) : self;
      const float2 x = NORM ? mul2(over, sn) : sn;
      t.across[k][i] = INTER ? make_float2(-x.x, x.y) : k == 0 ? make_float2(-x.x, -x.y) : x;
    }
}
template <bool INTER>
__device__ __forceinline__ void apply_turn(const Turn& t, bool turns, float2 (&a)[kPairs], float2 (&b)[kPairs]) {
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    const float2 x = mul2(a[i], t.own[0][i]), y = mul2(b[i], t.own[1][i]);
    if (turns) {  // not a product with zero: an infinity of the other element stays out
      const float2 oa = INTER ? swapped(a[i]) : b[i], ob = INTER ? swapped(b[i]) : a[i];
      a[i] = fma2(oa, t.across[0][i], x);
      b[i] = fma2(ob, t.across[1][i], y);
    } else {
      a[i] = x;
      b[i] = y;
    }
  }
}

// Backward, the rotation the other way.
struct Back {
  float2 c[kPairs], s[kPairs], minus_s[kPairs];  // with INTER: cosines and sines of chunk a's pairs, then of b's
};
template <bool INTER>
__device__ __forceinline__ void turn_back(const Back& t, float2 (&a)[kPairs], float2 (&b)[kPairs]) {
  auto one = [](float2& x, float cs, float sn) {
    x = make_float2(fmaf(x.x, cs, x.y * sn), fmaf(x.y, cs, -(x.x * sn)));
  };
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    if (INTER) {  // c[i] and s[i] hold those of pair i of chunk a and of chunk b
      one(a[i], t.c[i].x, t.s[i].x);
      one(b[i], t.c[i].y, t.s[i].y);
    } else {
      const float2 x = fma2(b[i], t.s[i], mul2(a[i], t.c[i]));
      b[i] = fma2(a[i], t.minus_s[i], mul2(b[i], t.c[i]));
      a[i] = x;
    }
  }
}

template <typename T>
__device__ __forceinline__ void store(T* row, const Slot& s, bool on, const float2 (&a)[kPairs], const float2 (&b)[kPairs]) {
  Raw<T> r;
  if (on && s.in) {
    rows::narrow(a, r);
    rows::store_raw(row + s.a, r);
  }
  if (on && s.in && s.b >= 0) {
    rows::narrow(b, r);
    rows::store_raw(row + s.b, r);
  }
}

__device__ __forceinline__ float products(const float2 (&a)[kPairs], const float2 (&x)[kPairs], const float2 (&b)[kPairs],
                                          const float2 (&y)[kPairs]) {
  float2 sum = mul2(a[0], x[0]);
#pragma unroll
  for (int i = 1; i < kPairs; ++i) sum = fma2(a[i], x[i], sum);
#pragma unroll
  for (int i = 0; i < kPairs; ++i) sum = fma2(b[i], y[i], sum);
  return sum.x + sum.y;
}

// Stages of rows on their way into shared memory, and blocks a multiprocessor (see qknorm_kernel).
template <typename T, bool BWD>
struct Pipe {
  static constexpr int kTensors = BWD ? 2 : 1, kPieces = sizeof(Raw<T>) / 16;
  static constexpr int kStages = BWD && sizeof(T) == 4 ? 3 : 4;
  static constexpr int kBlocks = 2;
  static constexpr int kSlot = kTensors * 2 * kPieces * 32;  // 16-byte pieces of a warp and stage
  static constexpr size_t kBytes = (size_t)kWarps * kStages * kSlot * 16;
};

template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// A lane's own slots of one stage: [tensor][chunk][piece][lane], so that a warp's accesses fall on consecutive
// addresses.
template <typename T>
__device__ __forceinline__ void copy_chunks(uint4* slot, const T* row, const Slot& s) {
  constexpr int kPieces = sizeof(Raw<T>) / 16;
#pragma unroll
  for (int k = 0; k < kPieces; ++k) {
    rows::copy_async<16>(slot + k * 32, reinterpret_cast<const uint4*>(row + s.a) + k);
    if (s.b >= 0) rows::copy_async<16>(slot + (kPieces + k) * 32, reinterpret_cast<const uint4*>(row + s.b) + k);
  }
}
template <typename T>
__device__ __forceinline__ void read_chunks(const uint4* slot, bool in_a, bool in_b, float2 (&a)[kPairs], float2 (&b)[kPairs]) {
  constexpr int kPieces = sizeof(Raw<T>) / 16;
  Raw<T> ra = rows::zero_raw<T>(), rb = rows::zero_raw<T>();
#pragma unroll
  for (int k = 0; k < kPieces; ++k) {
    if (in_a) reinterpret_cast<uint4*>(&ra)[k] = slot[k * 32];
    if (in_b) reinterpret_cast<uint4*>(&rb)[k] = slot[(kPieces + k) * 32];
  }
  rows::widen(ra, a);
  rows::widen(rb, b);
}

// One step: a head for each group of lanes, from its slots to memory.  Forward: x rstd, then weights and rotation.
template <typename T, int LANES, bool INTER, bool NORM>
__device__ __forceinline__ void forward_step(float eps, float inv_d, const Slot& slot, const uint4* from, bool on, T* to,
                                             const Turn& turn) {
  const bool in_a = on && slot.in, in_b = in_a && slot.b >= 0;
  float2 a[kPairs], b[kPairs];
  read_chunks<T>(from, in_a, in_b, a, b);
  if (NORM) {
    float sum = products(a, a, b, b);
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    const float2 rstd = both(rsqrtf(fmaf(sum, inv_d, eps)));
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      a[i] = mul2(a[i], rstd);
      b[i] = mul2(b[i], rstd);
    }
  }
  apply_turn<INTER>(turn, slot.turns, a, b);
  store<T>(to, slot, on, a, b);
}

// Backward: g turned back, u = g w, and with one exchange of two sums, of x^2 and of u x:
//   dx = rstd u - x (mean(u x) rstd) rstd rstd,   dw += g (x rstd)
template <typename T, int LANES, bool INTER, bool NORM>
__device__ __forceinline__ void backward_step(float eps, float inv_d, const Slot& slot, const uint4* from, bool on, T* to,
                                              const Back& back, const float* w, float2 (&dwq)[2][kPairs],
                                              float2 (&dwk)[2][kPairs], bool key) {
  constexpr int kTensor = 2 * (sizeof(Raw<T>) / 16) * 32;
  const bool in_a = on && slot.in, in_b = in_a && slot.b >= 0;
  float2 a[kPairs], b[kPairs];
  read_chunks<T>(from + kTensor, in_a, in_b, a, b);
  if (slot.turns) turn_back<INTER>(back, a, b);
  if (NORM) {
    float2 x[kPairs], y[kPairs], ua[kPairs], ub[kPairs];
    read_chunks<T>(from, in_a, in_b, x, y);
    read8(w + slot.a, ua);
    read8(w + max(slot.b, 0), ub);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      ua[i] = mul2(ua[i], a[i]);
      ub[i] = mul2(ub[i], b[i]);
    }
    float square = products(x, x, y, y), dot = products(ua, x, ub, y);
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) {
      square += __shfl_xor_sync(0xFFFFFFFFu, square, o);
      dot += __shfl_xor_sync(0xFFFFFFFFu, dot, o);
    }
    const float rstd = rsqrtf(fmaf(square, inv_d, eps));
    const float along = -(dot * inv_d * rstd) * rstd * rstd;  // in this order nothing leaves the range before the result
    // query and key heads have sums of their own
    if (key) {
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        dwk[0][i] = fma2(a[i], mul2(x[i], both(rstd)), dwk[0][i]);
        dwk[1][i] = fma2(b[i], mul2(y[i], both(rstd)), dwk[1][i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        dwq[0][i] = fma2(a[i], mul2(x[i], both(rstd)), dwq[0][i]);
        dwq[1][i] = fma2(b[i], mul2(y[i], both(rstd)), dwq[1][i]);
      }
    }
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      a[i] = fma2(x[i], both(along), mul2(ua[i], both(rstd)));
      b[i] = fma2(y[i], both(along), mul2(ub[i], both(rstd)));
    }
  }
  store<T>(to, slot, on, a, b);
}

template <typename T, int LANES, bool BWD, bool INTER, bool NORM>
__global__ void __launch_bounds__(kThreads, (Pipe<T, BWD>::kBlocks)) qknorm_kernel(const Args args) {
  using P = Pipe<T, BWD>;
  constexpr int kGroups = 32 / LANES, kStages = P::kStages;
  constexpr int kAngles = kGroups >= 8 ? 1 : 8 / kGroups;  // that a lane finds
  constexpr bool kReadsX = !BWD || NORM;
  extern __shared__ __align__(16) uint4 slots[];
  __shared__ __align__(16) float weights[2][kMaxDim];
  const nat_qknorm_params& p = args.p;
  const int D = p.head_dim, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = lane / LANES;
  const Slot slot = slot_of(p, lane & (LANES - 1));
  const float inv_d = 1.f / (float)D;
  if (NORM) {
    for (int i = threadIdx.x; i < 2 * kMaxDim; i += kThreads)
      weights[i / kMaxDim][i % kMaxDim] = i % kMaxDim < D ? (i < kMaxDim ? args.w_q : args.w_k)[i % kMaxDim] : 0.f;
    __syncthreads();
  }
  int64_t first_row, end_row;
  row_range(args, first_row, end_row);
  const int64_t n = end_row - first_row;
  const int64_t total = (int64_t)gridDim.x * kWarps, mine = (int64_t)blockIdx.x * kWarps + warp;
  const int64_t each = n / total, more = n % total;
  const uint32_t begin = (uint32_t)(first_row + mine * each + min(mine, more)),
                 end = begin + (uint32_t)each + (mine < more ? 1u : 0u);

  // Steps of a token: its query heads and right behind them its key heads, kGroups at a time (one with both kinds in
  // place of two: 230,000 tokens of 2 and 1 heads forward 227 -> 182 us).
  const int heads = p.n_heads + p.n_kv_heads, steps = (heads + kGroups - 1) / kGroups;
  struct Head {
    bool key, in;
    uint32_t at;  // its first element in a token's row
  };
  auto element = [](uint32_t t, int64_t stride, uint32_t at) { return (int64_t)((uint64_t)t * (uint32_t)stride + at); };
  auto head_of = [&](int i) -> Head {
    const int h = i * kGroups + group;
    const bool key = h >= p.n_heads;
    return {key, h < heads, (uint32_t)((key ? h - p.n_heads : h) * D)};
  };
  uint4* own = slots + (size_t)warp * kStages * P::kSlot + lane;
  uint32_t ahead_t = begin;
  int ahead_step = 0, ahead_stage = 0;
  auto fetch = [&]() {  // the next step that is not on its way yet
    if (ahead_t < end) {
      const Head h = head_of(ahead_step);
      if (slot.in && h.in) {
        uint4* to = own + ahead_stage * P::kSlot;
        if (kReadsX)
          copy_chunks<T>(to, (const T*)(h.key ? args.k : args.q) + element(ahead_t, h.key ? p.k_stride : p.q_stride, h.at), slot);
        if (BWD)
          copy_chunks<T>(to + P::kSlot / 2,
                         (const T*)(h.key ? args.dk_out : args.dq_out) +
                             element(ahead_t, h.key ? p.k_out_stride : p.q_out_stride, h.at),
                         slot);
      }
      if (++ahead_step == steps) {
        ahead_step = 0;
        ++ahead_t;
      }
    }
    ahead_stage = ahead_stage + 1 == kStages ? 0 : ahead_stage + 1;
    rows::copies_commit();
  };
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) fetch();

  float2 dwq[2][kPairs], dwk[2][kPairs];
  if (BWD && NORM) {
#pragma unroll
    for (int i = 0; i < 2 * kPairs; ++i) dwq[i / kPairs][i % kPairs] = dwk[i / kPairs][i % kPairs] = both(0.f);
  }
  // turns of a full circle a position, of the angles that this lane finds
  double freq[kAngles];
#pragma unroll
  for (int j = 0; j < kAngles; ++j) {
    const int e = j * kGroups + group;
    freq[j] = slot.turns && e < 8 ? __ldg(args.inv_freq + angle_of<INTER>(slot, e)) * 0.15915494309189533577 : 0.0;
  }
  int seq = 0;
  int64_t seq_lo = 0, seq_hi = 0;
  if (!args.positions && begin < end) {
    seq = owner(args.cu, args.B, begin);
    seq_lo = __ldg(args.cu + seq);
    seq_hi = __ldg(args.cu + seq + 1);
  }
  int stage = 0;
  const int first_key = p.n_heads / kGroups;  // the step in which the key heads begin
  for (uint32_t t = begin; t < end; ++t) {
    int64_t pos;
    if (args.positions) {
      pos = __ldg(args.positions + t);
    } else {
      while (t >= seq_hi && seq + 1 < args.B) {
        ++seq;
        seq_lo = seq_hi;
        seq_hi = __ldg(args.cu + seq + 1);
      }
      pos = t - seq_lo;
    }
    float cj[kAngles], sj[kAngles];
#pragma unroll
    for (int j = 0; j < kAngles; ++j) {
      const double x = freq[j] * (double)pos;
      sincospif((float)(2.0 * (x - rint(x))), &sj[j], &cj[j]);
    }
    auto deal = [&](float (&c)[8], float (&s)[8]) {  // for all lanes
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int from = (e % kGroups) * LANES + (lane & (LANES - 1));
        c[e] = __shfl_sync(0xFFFFFFFFu, cj[e / kGroups], from);
        s[e] = __shfl_sync(0xFFFFFFFFu, sj[e / kGroups], from);
      }
    };
    Turn turn;
    Back back;
    if (BWD) {
      float c[8], s[8];
      deal(c, s);
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        back.c[i] = INTER ? make_float2(c[i], c[4 + i]) : make_float2(c[2 * i], c[2 * i + 1]);
        back.s[i] = INTER ? make_float2(s[i], s[4 + i]) : make_float2(s[2 * i], s[2 * i + 1]);
        back.minus_s[i] = make_float2(-back.s[i].x, -back.s[i].y);
      }
    }
    // a stage is fetched anew only after the step that read it has used, and stored, what it read
    for (int i = 0; i < steps; ++i) {
      fetch();
      copies_wait<kStages - 1>();
      const uint4* from = own + stage * P::kSlot;
      stage = stage + 1 == kStages ? 0 : stage + 1;
      const Head h = head_of(i);
      T* to = (T*)(h.key ? args.k_to : args.q_to) +
              element(t, BWD ? (h.key ? p.k_stride : p.q_stride) : (h.key ? p.k_out_stride : p.q_out_stride), h.at);
      const float* w = weights[h.key ? 1 : 0];
      if (BWD) {
        backward_step<T, LANES, INTER, NORM>(p.eps, inv_d, slot, from, h.in, to, back, w, dwq, dwk, h.key);
      } else {
        // the weights change with the kind of head: in the first step, in that of the first key heads, and, where that one
        // has both kinds, in the one behind
        if (i == 0 || (NORM && (i == first_key || i == first_key + 1))) {
          float c[8], s[8];
          deal(c, s);
          make_turn<INTER, NORM>(turn, slot, w, c, s);
        }
        forward_step<T, LANES, INTER, NORM>(p.eps, inv_d, slot, from, h.in, to, turn);
      }
    }
  }
  if (BWD && NORM) {
    // over the groups of the warp, over the warps of the block (in the slots, which nothing is on its way to now)
    copies_wait<0>();
    __syncthreads();
    float* sums = reinterpret_cast<float*>(slots);  // [warp][kind][column]
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
      float2(&dw)[2][kPairs] = kind == 0 ? dwq : dwk;
#pragma unroll
      for (int i = 0; i < 2 * kPairs; ++i) {
        float2& v = dw[i / kPairs][i % kPairs];
#pragma unroll
        for (int o = LANES; o < 32; o <<= 1) {
          v.x += __shfl_xor_sync(0xFFFFFFFFu, v.x, o);
          v.y += __shfl_xor_sync(0xFFFFFFFFu, v.y, o);
        }
        const int at = i < kPairs ? slot.a + 2 * i : slot.b + 2 * (i - kPairs);
        if (group == 0 && slot.in && (i < kPairs || slot.b >= 0))
          *reinterpret_cast<float2*>(sums + (warp * 2 + kind) * kMaxDim + at) = v;
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) v += sums[(w * 2 + i / D) * kMaxDim + i % D];
      args.partial[(int64_t)blockIdx.x * 2 * D + i] = v;
    }
  }
}

// Adds the blocks' sums: 32 columns a block, each warp a run of blocks in their order, then the warps in theirs.
constexpr int kSumThreads = 1024;
__global__ void __launch_bounds__(kSumThreads)
weights_kernel(const float* partial, int blocks, int D, float* dw_q, float* dw_k) {
  __shared__ float sums[32][33];
  wait_for_primary();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, i = blockIdx.x * 32 + lane;
  const int per = (blocks + 31) / 32, end = min((warp + 1) * per, blocks);
  float v = 0.f;
  if (i < 2 * D) {
#pragma unroll 8
    for (int b = warp * per; b < end; ++b) v += partial[(int64_t)b * 2 * D + i];
  }
  sums[warp][lane] = v;
  __syncthreads();
  if (warp == 0 && i < 2 * D) {
    v = sums[0][lane];
    for (int w = 1; w < 32; ++w) v += sums[w][lane];
    (i < D ? dw_q : dw_k)[i % D] = v;
  }
}

// --------------------------------------------------------------------------- host
// Lanes of a head's row: two chunks each.
int lanes_of(const nat_qknorm_params& p) {
  const int slots = p.rot_dim / 16 + ((p.head_dim - p.rot_dim) / kChunk + 1) / 2;
  return slots > 4 ? 8 : slots > 2 ? 4 : 2;
}

// Blocks, and with them the tokens of a warp.  Many short runs in the blocks' order keep what is read and written at any
// time together, where persistent warps with long runs of their own drift over all of it: 160,000 tokens of 32 and 8
// heads of 128, forward 582 us persistent, 531, 509, 496, 488, 479 with runs of 16, 8, 4, 2, 1; backward 850 us
// persistent, 776, 772, 756, 798 with runs of 12, 8, 4, 2 (74,000 of 16 and 8 heads: 255, 250, 261, 255, 271), where every
// block leaves sums behind.  So a run is about 8 KB of queries and keys forward and 32 KB backward; few tokens are
// dealt to all that the multiprocessors hold.
int blocks_of(const nat_qknorm_params& p, int64_t cap, bool bwd) {
  const int64_t row = (int64_t)(p.n_heads + p.n_kv_heads) * p.head_dim * (p.dtype == NAT_F32 ? 4 : 2);
  const int64_t run = ((bwd ? 32768 : 8192) + row - 1) / row;
  const int64_t most = (cap + kWarps - 1) / kWarps, held = 148 * 2;
  return (int)min(most, max(held, (cap + kWarps * run - 1) / (kWarps * run)));
}

int check(const char* who, const nat_qknorm_params* p, int64_t cap) {
  if (!p) return fail(NAT_ERR_INVALID_ARG, "%s: params is null", who);
  if (p->dtype != NAT_F32 && p->dtype != NAT_BF16)
    return fail(NAT_ERR_UNSUPPORTED, "%s: unknown dtype %d", who, p->dtype);
  if (p->n_heads <= 0 || p->n_kv_heads <= 0 || p->head_dim <= 0 || p->rot_dim < 0 || cap < 0 || cap > 0x7FFFFFFFll)
    return fail(NAT_ERR_INVALID_ARG,
                "%s: head counts and head_dim must be positive, rot_dim >= 0, cap in [0, 2^31)", who);
  if (p->head_dim % kChunk != 0 || p->head_dim > kMaxDim)
    return fail(NAT_ERR_UNSUPPORTED, "%s: head_dim must be a multiple of 8, at most 128 (head_dim = %d)", who,
                p->head_dim);
  if (p->rot_dim > p->head_dim)
    return fail(NAT_ERR_INVALID_ARG, "%s: rot_dim exceeds head_dim", who);
  if (p->rot_dim % 16 != 0)
    return fail(NAT_ERR_UNSUPPORTED, "%s: rot_dim must be a multiple of 16 (rot_dim = %d)", who, p->rot_dim);
  if (p->interleaved != 0 && p->interleaved != 1)
    return fail(NAT_ERR_INVALID_ARG, "%s: interleaved must be 0 or 1", who);
  if (!(p->eps >= 0.f) || p->eps - p->eps != 0.f)
    return fail(NAT_ERR_INVALID_ARG, "%s: eps must be finite and >= 0", who);
  const int64_t strides[4] = {p->q_stride, p->q_out_stride, p->k_stride, p->k_out_stride};
  for (int i = 0; i < 4; ++i) {
    const int64_t width = (int64_t)(i < 2 ? p->n_heads : p->n_kv_heads) * p->head_dim;
    if (strides[i] < width)
      return fail(NAT_ERR_INVALID_ARG, "%s: a token's row (stride %lld) is shorter than its heads (%lld)", who,
                  (long long)strides[i], (long long)width);
    if (strides[i] % kChunk != 0 || strides[i] >= (1ll << 31))
      return fail(NAT_ERR_UNSUPPORTED, "%s: strides must be multiples of 8 elements, below 2^31", who);
  }
  return NAT_OK;
}

int check_call(const char* who, const Args& a, std::initializer_list<const void*> matrices) {
  if (!a.positions && (!a.cu || a.B <= 0))
    return fail(NAT_ERR_INVALID_ARG, "%s: needs positions, or cu_seqlens of B > 0 sequences", who);
  if ((a.w_q == nullptr) != (a.w_k == nullptr))
    return fail(NAT_ERR_INVALID_ARG, "%s: w_q and w_k come together", who);
  if (a.p.rot_dim > 0 && !a.inv_freq) return fail(NAT_ERR_INVALID_ARG, "%s: inv_freq is null", who);
  for (const void* m : matrices) {
    if (!m) return fail(NAT_ERR_INVALID_ARG, "%s: null pointer", who);
    if ((uintptr_t)m & 15u) return fail(NAT_ERR_INVALID_ARG, "%s: rows must be 16-byte aligned", who);
  }
  if (((uintptr_t)a.cu | (uintptr_t)a.positions | (uintptr_t)a.n_rows | (uintptr_t)a.w_q | (uintptr_t)a.w_k) & 3u ||
      (uintptr_t)a.inv_freq & 7u)
    return fail(NAT_ERR_INVALID_ARG, "%s: a vector is not aligned to its type", who);
  return NAT_OK;
}

template <typename T, int LANES, bool BWD, bool INTER, bool NORM>
int launch_kernel(const Args& a, cudaStream_t stream) {
  static std::atomic<uint64_t> allowed{0};  // a bit for each device whose shared-memory limit is raised
  constexpr size_t smem = Pipe<T, BWD>::kBytes;
  int dev = 0;
  NAT_CUDA(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return fail(NAT_ERR_UNSUPPORTED, "device index %d is beyond the 64 this library tracks", dev);
  if (!(allowed.load(std::memory_order_relaxed) >> dev & 1u)) {
    NAT_CUDA(cudaFuncSetAttribute(qknorm_kernel<T, LANES, BWD, INTER, NORM>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                  (int)smem));
    allowed.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  qknorm_kernel<T, LANES, BWD, INTER, NORM><<<blocks_of(a.p, a.cap, BWD), kThreads, smem, stream>>>(a);
  NAT_LAUNCH_CHECK("qknorm");
  return NAT_OK;
}

template <typename T, int LANES, bool BWD>
int launch_lanes(const Args& a, cudaStream_t stream) {
  if (a.p.interleaved)
    return a.w_q ? launch_kernel<T, LANES, BWD, true, true>(a, stream) : launch_kernel<T, LANES, BWD, true, false>(a, stream);
  return a.w_q ? launch_kernel<T, LANES, BWD, false, true>(a, stream) : launch_kernel<T, LANES, BWD, false, false>(a, stream);
}

template <typename T, bool BWD>
int launch(const Args& a, cudaStream_t stream) {
  const int lanes = lanes_of(a.p);
  return lanes == 8 ? launch_lanes<T, 8, BWD>(a, stream) : lanes == 4 ? launch_lanes<T, 4, BWD>(a, stream)
                                                                      : launch_lanes<T, 2, BWD>(a, stream);
}

size_t workspace_bytes_of(const nat_qknorm_params& p, int64_t cap) {
  return 256 + align_up((size_t)blocks_of(p, cap, true) * 2 * p.head_dim * sizeof(float), 256);
}

}  // namespace
}  // namespace qknorm
}  // namespace nat

extern "C" {

size_t nat_qknorm_workspace_bytes(const nat_qknorm_params* p, int64_t cap) {
  if (nat::qknorm::check("nat_qknorm_workspace_bytes", p, cap) != NAT_OK) return 0;
  return nat::qknorm::workspace_bytes_of(*p, cap);
}

int nat_qknorm_fwd(const nat_qknorm_params* p, int32_t B, const int32_t* cu_seqlens, const int32_t* positions,
                   const int32_t* n_rows, int64_t cap, const void* q, const void* k, const float* w_q,
                   const float* w_k, const double* inv_freq, void* q_out, void* k_out, void* stream) {
  const char* who = "nat_qknorm_fwd";
  int s = nat::qknorm::check(who, p, cap);
  if (s != NAT_OK || cap == 0) return s;
  nat::qknorm::Args a{};
  a.p = *p; a.B = B; a.cu = B >= 0 ? cu_seqlens : nullptr; a.positions = positions; a.n_rows = n_rows; a.cap = cap; a.q = q; a.k = k;
  a.w_q = w_q; a.w_k = w_k; a.inv_freq = inv_freq; a.q_to = q_out; a.k_to = k_out;
  s = nat::qknorm::check_call(who, a, {q, k, q_out, k_out});
  if (s != NAT_OK) return s;
  return p->dtype == NAT_F32 ? nat::qknorm::launch<float, false>(a, (cudaStream_t)stream)
                             : nat::qknorm::launch<__nv_bfloat16, false>(a, (cudaStream_t)stream);
}

int nat_qknorm_bwd(const nat_qknorm_params* p, int32_t B, const int32_t* cu_seqlens, const int32_t* positions,
                   const int32_t* n_rows, int64_t cap, const void* q, const void* k, const float* w_q,
                   const float* w_k, const double* inv_freq, const void* dq_out, const void* dk_out, void* dq,
                   void* dk, float* dw_q, float* dw_k, void* workspace, size_t workspace_bytes, void* stream) {
  const char* who = "nat_qknorm_bwd";
  int s = nat::qknorm::check(who, p, cap);
  if (s != NAT_OK) return s;
  nat::qknorm::Args a{};
  a.p = *p; a.B = B; a.cu = B >= 0 ? cu_seqlens : nullptr; a.positions = positions; a.n_rows = n_rows; a.cap = cap; a.q = q; a.k = k;
  a.w_q = w_q; a.w_k = w_k; a.inv_freq = inv_freq; a.dq_out = dq_out; a.dk_out = dk_out; a.q_to = dq; a.k_to = dk;
  if (cap > 0)
    s = w_q ? nat::qknorm::check_call(who, a, {q, k, dq_out, dk_out, dq, dk})
            : nat::qknorm::check_call(who, a, {dq_out, dk_out, dq, dk});
  if (s != NAT_OK) return s;
  if (w_q) {
    if (!dw_q || !dw_k) return nat::fail(NAT_ERR_INVALID_ARG, "%s: null gradient", who);
    if (((uintptr_t)dw_q | (uintptr_t)dw_k) & 3u)
      return nat::fail(NAT_ERR_INVALID_ARG, "%s: a vector is not aligned to its type", who);
    const size_t need = nat::qknorm::workspace_bytes_of(*p, cap);
    if (!workspace || workspace_bytes < need)
      return nat::fail(NAT_ERR_CAPACITY, "%s: workspace too small (%zu < %zu)", who, workspace_bytes, need);
    if ((uintptr_t)workspace & 255u)
      return nat::fail(NAT_ERR_INVALID_ARG, "%s: workspace must be 256-byte aligned", who);
    a.partial = (float*)((char*)workspace + 256);
  }
  cudaStream_t st = (cudaStream_t)stream;
  if (cap > 0) {
    s = p->dtype == NAT_F32 ? nat::qknorm::launch<float, true>(a, st) : nat::qknorm::launch<__nv_bfloat16, true>(a, st);
    if (s != NAT_OK) return s;
  }
  if (w_q) {
    s = nat::launch_after(nat::qknorm::weights_kernel, dim3((2 * p->head_dim + 31) / 32), nat::qknorm::kSumThreads, 0, st,
                          "qknorm_weights", (const float*)a.partial, nat::qknorm::blocks_of(*p, cap, true), p->head_dim, dw_q,
                          dw_k);
    if (s != NAT_OK) return s;
  }
  return NAT_OK;
}

}  // extern "C"
