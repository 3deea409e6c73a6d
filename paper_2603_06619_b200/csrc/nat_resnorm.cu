// The join of two blocks on packed rows, forward and backward: post-norm of a block's output,
// gate and residual scale, and the next block's pre-norm, in one pass over the rows.
//
//   n = y rstd_y w_post,  r = alpha x + gate n,  h = r rstd_r w_pre,  rstd = (mean(.^2) + eps)^-1/2
//
// Bound by HBM.  NT threads own a row, each with CH chunks of eight elements in registers, and
// persistent blocks walk the rows, with the next rows on their way into shared memory by asynchronous
// copies.  What the threads of a row have to agree on is found in ONE sum over the row, because its
// barrier, not the arithmetic, is what a row waits for: with z = y (w_post gate)
//   sum r^2 = alpha^2 sum x^2 + 2 alpha rstd_y sum x z + rstd_y^2 sum z^2
// gives the second norm before r is formed.  Where the terms cancel (below 1/16 of their
// magnitudes), or one of the sums has lost its squares to underflow, the row is summed again from r
// itself.  The weights, multiplied together, are kept in shared memory; from L1 they were half evicted by
// the rows.  60,000 rows of 4096 bfloat16: 302 us, 0.99 of the measured copy bandwidth; with checkpoints
// 495 us (0.76; issue slots 72 % busy with the quantisation).
//
// Backward, with u = dh w_pre, rhat = r rstd_r, yhat = y rstd_y, e = dr_in + rstd_r u, z = yhat w_post gate:
//   dr = e - rstd_r rhat mean(u rhat),   dx = alpha dr,   v = dr w_post gate,
//   dy = rstd_y (v - yhat mean(v yhat)),   sum v yhat = sum e z - rstd_r mean(u rhat) sum rhat z
//   dw_pre = sum dh rhat,  dw_post = sum gate dr yhat,  dgate = sum dr yhat w_post  (over rows, or over a row),
// again with one sum over the row, of three products.  (The difference in sum v yhat loses no more
// than the elements of dr, formed by the same difference, have lost.)
// A gate per column factors out of its sum: dw_post = gate A, dgate = w_post A with one
// A = sum dr yhat, so a thread keeps two sums per column.  Every block leaves its sums in the
// workspace and a second kernel adds them in block order: the gradients of the weights repeat
// bit for bit.  74,003 rows of 1024: 162 us with the second kernel, 0.86 of the copy bandwidth; 60,000 rows of
// 4096 from checkpoints: 530 us, 0.71, two blocks a multiprocessor waiting for their rows' sums in turn.
#include <initializer_list>

#include "nat_common.cuh"
#include "nat_rows.cuh"

namespace nat {
namespace {

using rows::kChunk;

struct FwdArgs {
  const void *x, *y;
  const float *w_post, *gate, *w_pre;
  void *r, *h;
  float *rstd_y, *rstd_r;
  int8_t *y8, *r8;
  float *y8s, *r8s;
  const int32_t* n_rows;
  int64_t cap;
  int d, groups, gate_mode, stages;
  float eps, alpha, inv_d;
};

struct BwdArgs {
  const void *y, *r, *dr_in, *dh;
  const int8_t *y8, *r8;
  const float *y8s, *r8s;
  const float *w_post, *gate, *w_pre, *rstd_y, *rstd_r;
  void *dx, *dy;
  float *dgate_row, *partial;  // partial [blocks][2][d]: A, then dw_pre
  const int32_t* n_rows;
  int64_t cap;
  int d, groups, gate_mode, stages;
  float alpha, inv_d;
  bool has_y;
};

// N sums over the NT threads of a row, the same in every thread: within the warps, then of the warps'
// sums, which every warp adds up with the same shuffles.  `buf` alternates between calls, so one
// barrier a call is enough: a buffer is written again only after the next call's barrier.
template <int NT, int N>
struct RowSum {
  float4* buf;  // [2][NT / 32], where a row has more than a warp
  uint32_t turn = 0;
  __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
    for (int o = NT < 32 ? NT / 2 : 16; o > 0; o >>= 1)
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
    if (NT > 32) {
      constexpr int W = NT / 32;
      float4* b = buf + (turn & 1) * W;
      ++turn;
      if ((threadIdx.x & 31) == 0)
        b[threadIdx.x >> 5] = make_float4(v[0], N > 1 ? v[N > 1 ? 1 : 0] : 0.f, N > 2 ? v[N > 2 ? 2 : 0] : 0.f,
                                          N > 3 ? v[N > 3 ? 3 : 0] : 0.f);
      __syncthreads();
      const float4 w = b[threadIdx.x & (W - 1)];
      const float ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] = ws[k];
#pragma unroll
      for (int o = W / 2; o > 0; o >>= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
    }
  }
};

__device__ __forceinline__ float sum_pairs(const float2& s) { return s.x + s.y; }

// Threads and rows of a block: short rows have a warp or less of their own.  (The rows of a warp take
// the same turns, the ones past the end idly, for the shuffles' sake.)
constexpr __host__ __device__ int block_threads(int nt) { return nt <= 32 ? 128 : nt; }
constexpr __host__ __device__ int block_rows(int nt) { return nt <= 32 ? 128 / nt : 1; }

// Threads a multiprocessor, which set the registers a thread may have.  Few threads with their rows on the way
// beat many that spill (60,000 rows of 4096): forward 302 us with 512, 348 with 768, 335 with 1024; leaving
// checkpoints, which takes twice the instructions, 546, 495, 595; backward, where a thread also keeps the sums
// of its columns, 530 with 512, 867 with 768.  With one chunk a thread the backward has its best between
// (120e6 bfloat16 elements in rows of 128, plain and from checkpoints: 255 and 251 us with 512, 239 and 238
// with 640, 270 and 280 with 768, 544 and 434 with 1024).
constexpr __host__ __device__ int fwd_threads(bool c8, int nt) { return nt <= 32 || c8 ? 768 : 512; }
constexpr __host__ __device__ int bwd_threads(int ch) { return ch == 1 ? 640 : 512; }
constexpr __host__ __device__ int blocks_per_sm(int threads, int nt) {
  return threads / block_threads(nt) > 0 ? threads / block_threads(nt) : 1;
}

// Shared memory of a block: [stage][piece of the slot][thread], 16-byte pieces, so that the copies and
// reads of a warp fall on consecutive addresses.
template <typename T>
struct Pieces {
  static constexpr int kRaw = sizeof(rows::Raw<T>) / 16;
};

template <typename T, int NT>
__device__ __forceinline__ void copy_piece(uint4* slot, const T* src) {
  // a Raw<float> is two pieces, a row of threads apart
#pragma unroll
  for (int k = 0; k < Pieces<T>::kRaw; ++k)
    rows::copy_async<16>(slot + k * block_threads(NT), reinterpret_cast<const uint4*>(src) + k);
}
template <typename T, int NT>
__device__ __forceinline__ rows::Raw<T> read_piece(const uint4* slot) {
  rows::Raw<T> r;
#pragma unroll
  for (int k = 0; k < Pieces<T>::kRaw; ++k) reinterpret_cast<uint4*>(&r)[k] = slot[k * block_threads(NT)];
  return r;
}

using rows::kPairs;

// Weights in shared memory: w_post times a gate per column (ones where there is neither), and w_pre.
// For a row of NT threads with CH chunks each they are laid out like the pieces: the two float4 of a
// chunk a row of threads apart.
template <int NT, int CH>
struct Weights {
  float4* at;  // [2][CH][2][NT]
  __device__ __forceinline__ void fill(int d, const float* w_post, const float* gate, const float* w_pre) {
    for (int i = threadIdx.x; i < 2 * CH * NT; i += blockDim.x) {
      // i numbers float4s of a row: chunk i / 2, its half i % 2
      const int col = i * 4, t = (i >> 1) % NT, c = (i >> 1) / NT, half = i & 1;
      float a[4], b[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool in = col + j < d;
        a[j] = (in && w_post ? w_post[col + j] : 1.f) * (in && gate ? gate[col + j] : 1.f);
        b[j] = in && w_pre ? w_pre[col + j] : 0.f;
      }
      at[(c * 2 + half) * NT + t] = make_float4(a[0], a[1], a[2], a[3]);
      at[((CH + c) * 2 + half) * NT + t] = make_float4(b[0], b[1], b[2], b[3]);
    }
    __syncthreads();
  }
  __device__ __forceinline__ void get(int which, int c, int t, float2 (&w)[kPairs]) const {
    const float4 a = at[((which * CH + c) * 2) * NT + t], b = at[((which * CH + c) * 2 + 1) * NT + t];
    w[0] = make_float2(a.x, a.y);
    w[1] = make_float2(a.z, a.w);
    w[2] = make_float2(b.x, b.y);
    w[3] = make_float2(b.z, b.w);
  }
};

constexpr float kTiny = 1e-28f;  // of 8192 squares: the larger ones are above 2^-107, normal with all their bits

template <typename T, int NT, int CH, bool C8>
__global__ void __launch_bounds__(block_threads(NT), blocks_per_sm(fwd_threads(C8, NT), NT))
resnorm_fwd_kernel(FwdArgs a) {
  constexpr int RPB = block_rows(NT), P = Pieces<T>::kRaw, BT = block_threads(NT);
  extern __shared__ uint4 ring[];  // [stages][x, y][CH][P][BT], then the weights
  __shared__ float4 red[NT > 32 ? 2 * (NT / 32) : 1];
  RowSum<NT, 4> row_sums{red};
  const int t = threadIdx.x % NT, sub = threadIdx.x / NT, in_warp = NT < 32 ? (threadIdx.x & 31) / NT : 0;
  const int64_t n = a.n_rows ? min((int64_t)max(*a.n_rows, 0), a.cap) : a.cap;
  const int64_t step = (int64_t)gridDim.x * RPB;
  const T* x = (const T*)a.x;
  const T* y = (const T*)a.y;
  auto slot = [&](int stage, int of, int i) { return ring + (((stage * 2 + of) * CH + i) * P) * BT + threadIdx.x; };
  auto fetch = [&](int64_t row, int stage) {
    if (row < n) {
      const int64_t at = row * a.d + t * kChunk;
#pragma unroll
      for (int i = 0; i < CH; ++i)
        if ((t + i * NT) * kChunk < a.d) {
          copy_piece<T, NT>(slot(stage, 0, i), x + at + i * NT * kChunk);
          if (y) copy_piece<T, NT>(slot(stage, 1, i), y + at + i * NT * kChunk);
        }
    }
    rows::copies_commit();
  };
  auto checkpoint = [&](const rows::Raw<T>& raw, int64_t row, int col, int8_t* codes, float* scales) {
    const rows::GroupScale gs = rows::group_scale(rows::group_top<(NT < rows::kGroupLanes ? NT : rows::kGroupLanes)>(raw));
    if (row < n && col < a.d) {
      float2 v[kPairs];
      rows::widen(raw, v);
      __stcs(reinterpret_cast<uint2*>(codes + row * a.d + col), rows::group_codes(v, gs.inv));
      if ((t & 15) == 0) scales[row * a.groups + (col >> 7)] = gs.scale;
    }
  };
  int64_t row = (int64_t)blockIdx.x * RPB + sub;
  for (int k = 0; k < a.stages; ++k) fetch(row + k * step, k);
  Weights<NT, CH> weights{reinterpret_cast<float4*>(ring + a.stages * 2 * CH * P * BT)};
  weights.fill(a.d, a.w_post, a.gate_mode == NAT_GATE_CHANNEL ? a.gate : nullptr, a.w_pre);
  for (int stage = 0; row - in_warp < n; row += step, stage = stage + 1 == a.stages ? 0 : stage + 1) {
    const bool live = row < n;
    const float gate_row = live && a.gate_mode == NAT_GATE_ROW ? __ldg(a.gate + row) : 1.f;
    rows::copies_wait(a.stages - 1);
    float2 r[CH][kPairs], z[CH][kPairs];  // x, then r; y w_post gate
    float2 yy = both(0.f), xx = both(0.f), xz = both(0.f), zz = both(0.f);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int col = (t + i * NT) * kChunk;
      const bool in = live && col < a.d;
      rows::widen(in ? read_piece<T, NT>(slot(stage, 0, i)) : rows::zero_raw<T>(), r[i]);
      const rows::Raw<T> qy = (in && y) ? read_piece<T, NT>(slot(stage, 1, i)) : rows::zero_raw<T>();
      rows::widen(qy, z[i]);
      float2 w[kPairs];
      weights.get(0, i, t, w);
#pragma unroll
      for (int j = 0; j < kPairs; ++j) {
        yy = fma2(z[i][j], z[i][j], yy);
        z[i][j] = mul2(z[i][j], w[j]);
        xx = fma2(r[i][j], r[i][j], xx);
        xz = fma2(r[i][j], z[i][j], xz);
        zz = fma2(z[i][j], z[i][j], zz);
      }
      if (C8 && y) checkpoint(qy, row, col, a.y8, a.y8s);
    }
    fetch(row + a.stages * step, stage);
    float sums[4] = {sum_pairs(yy), sum_pairs(xx), sum_pairs(xz), sum_pairs(zz)};
    row_sums(sums);
    float inv_y = 1.f;
    if (a.w_post) {
      inv_y = __frsqrt_rn(fmaf(sums[0], a.inv_d, a.eps));
      if (live && t == 0) a.rstd_y[row] = inv_y;
    }
    const float f = inv_y * gate_row;
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int j = 0; j < kPairs; ++j) r[i][j] = fma2(z[i][j], both(f), mul2(r[i][j], both(a.alpha)));
    float inv_r = 1.f;
    if (a.w_pre) {
      // h is formed from r before its rounding: the norm then adds no error of its own
      const float own = a.alpha * a.alpha * sums[1] + f * f * sums[3];
      float square = fmaf(2.f * a.alpha * f, sums[2], own);
      // the same in all threads of the row; squares that small have left the normal range, or sums of them may have
      const bool cancels = !(square > 0.0625f * own) || sums[1] < kTiny || (y && sums[3] < kTiny);
      if (__any_sync(0xFFFFFFFFu, live && cancels)) {
        float2 rr = both(0.f);
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
          for (int j = 0; j < kPairs; ++j) rr = fma2(r[i][j], r[i][j], rr);
        float again[4] = {sum_pairs(rr), 0.f, 0.f, 0.f};
        row_sums(again);
        if (cancels) square = again[0];
      }
      inv_r = __frsqrt_rn(fmaf(square, a.inv_d, a.eps));
      if (live && t == 0) a.rstd_r[row] = inv_r;
    }
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int col = (t + i * NT) * kChunk;
      const bool in = live && col < a.d;
      rows::Raw<T> out;
      rows::narrow(r[i], out);
      if (in) rows::store_raw((T*)a.r + row * a.d + col, out);
      if (C8) checkpoint(out, row, col, a.r8, a.r8s);  // of the row as it is stored
      if (a.w_pre && in) {
        float2 w[kPairs];
        weights.get(1, i, t, w);
#pragma unroll
        for (int j = 0; j < kPairs; ++j) w[j] = mul2(mul2(r[i][j], both(inv_r)), w[j]);
        rows::narrow(w, out);
        rows::store_raw((T*)a.h + row * a.d + col, out);
      }
    }
  }
}

template <typename T, int NT, int CH, bool C8>
__global__ void __launch_bounds__(block_threads(NT), blocks_per_sm(bwd_threads(CH), NT))
resnorm_bwd_kernel(BwdArgs a) {
  constexpr int RPB = block_rows(NT), P = Pieces<T>::kRaw, BT = block_threads(NT);
  // [stages][CH][dr, dh: P pieces each; y, r: P pieces each, or one of codes (8 bytes y, 8 bytes r)][BT],
  // then the weights
  constexpr int kPieces = C8 ? 2 * P + 1 : 4 * P;
  extern __shared__ uint4 ring[];
  __shared__ float4 red[NT > 32 ? 2 * (NT / 32) : 1];
  RowSum<NT, 3> row_sums{red};
  const int t = threadIdx.x % NT, sub = threadIdx.x / NT, in_warp = NT < 32 ? (threadIdx.x & 31) / NT : 0;
  const int64_t n = a.n_rows ? min((int64_t)max(*a.n_rows, 0), a.cap) : a.cap;
  const int64_t step = (int64_t)gridDim.x * RPB;
  const bool row_gate = a.gate_mode == NAT_GATE_ROW;
  float2 acc[CH][kPairs], acc_pre[CH][kPairs];
#pragma unroll
  for (int i = 0; i < CH; ++i)
#pragma unroll
    for (int j = 0; j < kPairs; ++j) acc[i][j] = acc_pre[i][j] = both(0.f);

  auto col_of = [&](int i) { return (t + i * NT) * kChunk; };
  auto slot = [&](int stage, int i, int piece) { return ring + ((stage * CH + i) * kPieces + piece) * BT + threadIdx.x; };
  // A chunk's address as the row's, the same in the block, and the thread's column in it, or as one sum: the
  // first leaves the compiler registers in long rows (120e6 bfloat16 elements in rows of 2048, 4096, 8192: 240,
  // 236, 241 us against 262, 272, 305), the second is faster in short ones (of 1024: 239 against 254).
  constexpr bool kRowBase = NT >= 128;
  auto fetch = [&](int64_t row, int stage) {
    if (row < n) {
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int own = kRowBase ? t * kChunk : 0, left = a.d - i * NT * kChunk;
        if (!kRowBase && t * kChunk >= left) continue;
        const int64_t at = row * a.d + (kRowBase ? i * NT * kChunk : col_of(i));
        auto copy = [&](int piece, const void* src) {
          if (!kRowBase || own < left) copy_piece<T, NT>(slot(stage, i, piece), (const T*)src + at + own);
        };
        if (a.dr_in) copy(0, a.dr_in);
        if (a.w_pre) copy(P, a.dh);
        if (C8) {
          if (kRowBase && own >= left) continue;
          uint2* codes = reinterpret_cast<uint2*>(slot(stage, i, 2 * P));
          if (a.has_y) rows::copy_async<8>(codes, a.y8 + at + own);
          if (a.w_pre) rows::copy_async<8>(codes + 1, a.r8 + at + own);
        } else {
          if (a.has_y) copy(2 * P, a.y);
          if (a.w_pre) copy(3 * P, a.r);
        }
      }
    }
    rows::copies_commit();
  };
  // the row's scalars, one row ahead in registers
  float inv_y_next = 1.f, inv_r_next = 0.f, gate_next = 1.f, sy_next[CH], sr_next[CH];
#pragma unroll
  for (int i = 0; i < CH; ++i) sy_next[i] = sr_next[i] = 0.f;
  auto fetch_scalars = [&](int64_t row) {
    if (row >= n) {  // a row that only keeps its warp company adds nothing, whatever the one before it held
      inv_y_next = inv_r_next = 0.f;
#pragma unroll
      for (int i = 0; i < CH; ++i) sy_next[i] = sr_next[i] = 0.f;
      return;
    }
    if (a.w_post) inv_y_next = __ldg(a.rstd_y + row);
    if (a.w_pre) inv_r_next = __ldg(a.rstd_r + row);
    if (row_gate) gate_next = __ldg(a.gate + row);
    if (C8) {
#pragma unroll
      for (int i = 0; i < CH; ++i)
        if (col_of(i) < a.d) {
          const int64_t at = row * a.groups + (col_of(i) >> 7);
          if (a.has_y) sy_next[i] = __ldg(a.y8s + at);
          if (a.w_pre) sr_next[i] = __ldg(a.r8s + at);
        }
    }
  };
  int64_t row = (int64_t)blockIdx.x * RPB + sub;
  for (int k = 0; k < a.stages; ++k) fetch(row + k * step, k);
  fetch_scalars(row);
  Weights<NT, CH> weights{reinterpret_cast<float4*>(ring + a.stages * CH * kPieces * BT)};
  weights.fill(a.d, a.w_post, a.gate_mode == NAT_GATE_CHANNEL ? a.gate : nullptr, a.w_pre);
  for (int stage = 0; row - in_warp < n; row += step, stage = stage + 1 == a.stages ? 0 : stage + 1) {
    const bool live = row < n;
    const float inv_y = inv_y_next, inv_r = inv_r_next, gate_row = gate_next;
    float2 e[CH][kPairs], yv[CH][kPairs], rv[CH][kPairs];
    float2 s_ur = both(0.f), s_ez = both(0.f), s_rz = both(0.f);
    rows::copies_wait(a.stages - 1);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const bool in = live && col_of(i) < a.d;
      float2 u[kPairs], w[kPairs];
      if (C8) {
        const uint4 c = in ? *slot(stage, i, 2 * P) : make_uint4(0u, 0u, 0u, 0u);
        // a piece that was never copied holds old bytes, and its scale is zero
        rows::widen_codes(make_uint2(c.x, c.y), sy_next[i], yv[i]);
        rows::widen_codes(make_uint2(c.z, c.w), sr_next[i], rv[i]);
      } else {
        rows::widen((in && a.has_y) ? read_piece<T, NT>(slot(stage, i, 2 * P)) : rows::zero_raw<T>(), yv[i]);
        rows::widen((in && a.w_pre) ? read_piece<T, NT>(slot(stage, i, 3 * P)) : rows::zero_raw<T>(), rv[i]);
      }
      rows::widen((in && a.dr_in) ? read_piece<T, NT>(slot(stage, i, 0)) : rows::zero_raw<T>(), e[i]);
      rows::widen((in && a.w_pre) ? read_piece<T, NT>(slot(stage, i, P)) : rows::zero_raw<T>(), u);
      weights.get(1, i, t, w);
#pragma unroll
      for (int j = 0; j < kPairs; ++j) {
        rv[i][j] = mul2(rv[i][j], both(inv_r));  // rhat
        acc_pre[i][j] = fma2(u[j], rv[i][j], acc_pre[i][j]);
        u[j] = mul2(u[j], w[j]);
        s_ur = fma2(u[j], rv[i][j], s_ur);
        e[i][j] = fma2(both(inv_r), u[j], e[i][j]);
      }
      weights.get(0, i, t, w);
#pragma unroll
      for (int j = 0; j < kPairs; ++j) {
        yv[i][j] = mul2(yv[i][j], both(inv_y));  // yhat
        w[j] = mul2(w[j], yv[i][j]);             // z
        s_ez = fma2(e[i][j], w[j], s_ez);
        s_rz = fma2(rv[i][j], w[j], s_rz);
      }
    }
    fetch(row + a.stages * step, stage);
    fetch_scalars(row + step);
    float sums[3] = {sum_pairs(s_ur), sum_pairs(s_ez), sum_pairs(s_rz)};
    row_sums(sums);
    const float m1 = inv_r * sums[0] * a.inv_d, s_vy = fmaf(-m1, sums[2], sums[1]);
    if (row_gate && live && t == 0) a.dgate_row[row] = s_vy;  // of dr yhat w_post, without the gate itself
    const float2 m2 = both(a.w_post ? -gate_row * s_vy * a.inv_d : 0.f);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      if (!live || col_of(i) >= a.d) continue;
      float2 dx[kPairs], w[kPairs];
#pragma unroll
      for (int j = 0; j < kPairs; ++j) {
        e[i][j] = fma2(rv[i][j], both(-m1), e[i][j]);  // dr
        dx[j] = mul2(both(a.alpha), e[i][j]);
      }
      rows::Raw<T> out;
      rows::narrow(dx, out);
      rows::store_raw((T*)a.dx + row * a.d + col_of(i), out);
      if (!a.has_y) continue;
      weights.get(0, i, t, w);
#pragma unroll
      for (int j = 0; j < kPairs; ++j) {
        e[i][j] = mul2(e[i][j], both(gate_row));
        acc[i][j] = fma2(e[i][j], yv[i][j], acc[i][j]);
        w[j] = mul2(e[i][j], w[j]);  // v
      }
      if (a.w_post) {
#pragma unroll
        for (int j = 0; j < kPairs; ++j) w[j] = mul2(both(inv_y), fma2(yv[i][j], m2, w[j]));
      }
      rows::narrow(w, out);
      rows::store_raw((T*)a.dy + row * a.d + col_of(i), out);
    }
  }

  // the block's sums; those of the rows that it holds side by side are added in their order first
  float* p = a.partial + (int64_t)blockIdx.x * 2 * a.d;
  if (RPB == 1) {
#pragma unroll
    for (int i = 0; i < CH; ++i)
      if (col_of(i) < a.d)
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
          *reinterpret_cast<float2*>(p + col_of(i) + 2 * j) = acc[i][j];
          *reinterpret_cast<float2*>(p + a.d + col_of(i) + 2 * j) = acc_pre[i][j];
        }
  } else {
    __shared__ float2 part[2][RPB][RPB > 1 ? CH * NT * kPairs : 1];
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int j = 0; j < kPairs; ++j) {
        part[0][sub][(t + i * NT) * kPairs + j] = acc[i][j];
        part[1][sub][(t + i * NT) * kPairs + j] = acc_pre[i][j];
      }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * a.d; c += blockDim.x) {
      const int which = c >= a.d;
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < RPB; ++w) s += reinterpret_cast<const float*>(part[which][w])[c - which * a.d];
      p[c] = s;
    }
  }
}

// Adds the blocks' sums in block order (eight strided runs, joined in order) and applies the
// factors that were kept out of them.
__global__ void __launch_bounds__(256)
resnorm_columns_kernel(const float* partial, int blocks, int d, int gate_channel, const float* w_post,
                       const float* gate, float* dw_post, float* dgate, float* dw_pre) {
  wait_for_primary();
  __shared__ float part[8][33];
  const int lane = threadIdx.x & 31, run = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;  // over 2 d columns
  float s = 0.f;
  if (c < 2 * d)
    for (int b = run; b < blocks; b += 8) s += __ldcg(partial + (int64_t)b * 2 * d + c);
  part[run][lane] = s;
  __syncthreads();
  if (run != 0 || c >= 2 * d) return;
  s = 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) s += part[k][lane];
  if (c >= d) {
    if (dw_pre) dw_pre[c - d] = s;
    return;
  }
  if (dw_post) dw_post[c] = gate_channel ? s * gate[c] : s;
  if (gate_channel) dgate[c] = w_post ? s * w_post[c] : s;
}

// ---- launch shapes ----------------------------------------------------------------------
// Threads of a row and chunks of a thread, by the row's length: rows of up to 128 columns share a warp (two
// of 128, four of 64), up to 256 (forward 512) they have one, beyond that a block.  What bounds a short row is
// its chain of load, sums and store, so a warp that holds more of them is faster: against a warp a row of two
// chunks a thread, 55,164 bf16 rows of 64 take 8.3 instead of 26.9 us forward.  Rows of 257 to 512 backward: one
// chunk in each of 64 threads against two in 32 (120e6 elements in rows of 512): bfloat16 258 against 298 us, from
// checkpoints 249 against 234; float32 (60e6) 400 against 376 and 277 against 326.
constexpr int kMaxD = 8192;
struct Cut {
  int nt, ch;
};
Cut cut_of(int d, bool bwd) {
  if (d <= 64) return {8, 1};
  if (d <= 128) return {16, 1};
  if (d <= 256) return {32, 1};
  if (bwd && d <= 512) return {64, 1};
  int nt = 32;
  while (nt * 2 * kChunk < d) nt *= 2;
  return {nt, 2};
}

// Persistent blocks, all resident, fewer of them where the rows on their way would not fit into a
// multiprocessor's shared memory.
constexpr int kSmemPerSm = 216 * 1024;  // of 228 KB, less 1 KB and the static part a block

struct Shape {
  int64_t blocks;
  int stages;
  size_t smem;
};
Shape shape_of(int nt, int chunks, int threads_per_sm, size_t stage_bytes, int64_t cap) {
  const size_t weights = (size_t)2 * chunks * 2 * nt * sizeof(float4);
  int per_sm = blocks_per_sm(threads_per_sm, nt);
  const int fit = (int)(kSmemPerSm / (stage_bytes + weights));
  if (per_sm > fit) per_sm = fit > 0 ? fit : 1;
  Shape s;
  const int64_t want = (cap + block_rows(nt) - 1) / block_rows(nt);
  s.blocks = max((int64_t)1, min((int64_t)148 * per_sm, want));
  s.stages = (int)min((size_t)3, max((size_t)1, (kSmemPerSm / per_sm - weights) / stage_bytes));
  s.smem = s.stages * stage_bytes + weights;
  return s;
}

// Blocks of a backward pass at most: its workspace holds their column sums.
int64_t max_blocks(Cut c, int64_t cap) {
  return max((int64_t)1, min((int64_t)148 * blocks_per_sm(bwd_threads(c.ch), c.nt),
                             (cap + block_rows(c.nt) - 1) / block_rows(c.nt)));
}

template <typename K, typename A>
int launch(K kernel, A& a, int nt, int chunks, int threads_per_sm, size_t stage_bytes, cudaStream_t stream, int64_t* blocks,
           const char* name) {
  const Shape s = shape_of(nt, chunks, threads_per_sm, stage_bytes, a.cap);
  a.stages = s.stages;
  *blocks = s.blocks;
  if (s.smem > 32 * 1024)  // with the static part past the 48 KB of a plain launch
    NAT_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)s.smem));
  kernel<<<(unsigned)s.blocks, block_threads(nt), s.smem, stream>>>(a);
  NAT_LAUNCH_CHECK(name);
  return NAT_OK;
}

template <typename T, int NT, int CH>
int launch_fwd(FwdArgs& a, cudaStream_t stream) {
  constexpr size_t stage = 2 * CH * sizeof(rows::Raw<T>) * block_threads(NT);
  int64_t blocks;
  return a.r8 ? launch(resnorm_fwd_kernel<T, NT, CH, true>, a, NT, CH, fwd_threads(true, NT), stage, stream, &blocks,
                       "resnorm_fwd_kernel")
              : launch(resnorm_fwd_kernel<T, NT, CH, false>, a, NT, CH, fwd_threads(false, NT), stage, stream, &blocks,
                       "resnorm_fwd_kernel");
}

template <typename T, int NT, int CH>
int launch_bwd(BwdArgs& a, bool c8, cudaStream_t stream, int64_t* blocks) {
  constexpr size_t raw = sizeof(rows::Raw<T>), per = CH * block_threads(NT);
  return c8 ? launch(resnorm_bwd_kernel<T, NT, CH, true>, a, NT, CH, bwd_threads(CH), (2 * raw + 16) * per, stream,
                     blocks, "resnorm_bwd_kernel")
            : launch(resnorm_bwd_kernel<T, NT, CH, false>, a, NT, CH, bwd_threads(CH), 4 * raw * per, stream, blocks,
                     "resnorm_bwd_kernel");
}

template <typename T>
int dispatch_fwd(FwdArgs& a, cudaStream_t stream) {
  const Cut c = cut_of(a.d, false);
  switch (c.nt) {
    case 8: return launch_fwd<T, 8, 1>(a, stream);
    case 16: return launch_fwd<T, 16, 1>(a, stream);
    case 32: return c.ch == 1 ? launch_fwd<T, 32, 1>(a, stream) : launch_fwd<T, 32, 2>(a, stream);
    case 64: return launch_fwd<T, 64, 2>(a, stream);
    case 128: return launch_fwd<T, 128, 2>(a, stream);
    case 256: return launch_fwd<T, 256, 2>(a, stream);
    default: return launch_fwd<T, 512, 2>(a, stream);
  }
}

template <typename T>
int dispatch_bwd(BwdArgs& a, bool c8, cudaStream_t stream, int64_t* blocks) {
  const Cut c = cut_of(a.d, true);
  switch (c.nt) {
    case 8: return launch_bwd<T, 8, 1>(a, c8, stream, blocks);
    case 16: return launch_bwd<T, 16, 1>(a, c8, stream, blocks);
    case 32: return launch_bwd<T, 32, 1>(a, c8, stream, blocks);
    case 64: return c.ch == 1 ? launch_bwd<T, 64, 1>(a, c8, stream, blocks) : launch_bwd<T, 64, 2>(a, c8, stream, blocks);
    case 128: return launch_bwd<T, 128, 2>(a, c8, stream, blocks);
    case 256: return launch_bwd<T, 256, 2>(a, c8, stream, blocks);
    default: return launch_bwd<T, 512, 2>(a, c8, stream, blocks);
  }
}

int check_params(const char* who, const nat_resnorm_params* p, int64_t cap) {
  if (!p) return fail(NAT_ERR_INVALID_ARG, "%s: params is null", who);
  if (p->dtype != NAT_F32 && p->dtype != NAT_BF16)
    return fail(NAT_ERR_UNSUPPORTED, "%s: unknown dtype %d", who, p->dtype);
  if (p->d <= 0 || cap < 0 || cap > 0x7FFFFFFFll)
    return fail(NAT_ERR_INVALID_ARG, "%s: d must be positive and cap in [0, 2^31)", who);
  if (p->d % kChunk != 0 || p->d > kMaxD)
    return fail(NAT_ERR_UNSUPPORTED, "%s: d must be a multiple of 8, at most %d (d = %d)", who, kMaxD,
                p->d);
  if (!(p->eps >= 0.f) || !(p->alpha - p->alpha == 0.f))
    return fail(NAT_ERR_INVALID_ARG, "%s: eps must be >= 0 and alpha finite", who);
  if (p->gate_mode != NAT_GATE_NONE && p->gate_mode != NAT_GATE_CHANNEL && p->gate_mode != NAT_GATE_ROW)
    return fail(NAT_ERR_INVALID_ARG, "%s: unknown gate mode %d", who, p->gate_mode);
  return NAT_OK;
}

bool misaligned(std::initializer_list<const void*> ptrs, uintptr_t mask) {
  for (const void* q : ptrs)
    if ((uintptr_t)q & mask) return true;
  return false;
}

}  // namespace
}  // namespace nat

extern "C" {

size_t nat_resnorm_workspace_bytes(const nat_resnorm_params* p, int64_t cap) {
  if (nat::check_params("nat_resnorm_workspace_bytes", p, cap) != NAT_OK) return 0;
  const int64_t blocks = nat::max_blocks(nat::cut_of(p->d, true), cap);
  return nat::align_up((size_t)blocks * 2 * p->d * sizeof(float), 256);
}

int nat_resnorm_fwd(const nat_resnorm_params* p, const void* x, const void* y, const float* w_post,
                    const float* gate, const float* w_pre, const int32_t* n_rows, int64_t cap,
                    void* r, void* h, float* rstd_y, float* rstd_r, int8_t* y8, float* y8_scales,
                    int8_t* r8, float* r8_scales, void* stream) {
  const char* who = "nat_resnorm_fwd";
  int s = nat::check_params(who, p, cap);
  if (s != NAT_OK) return s;
  if (!y && (w_post || p->gate_mode != NAT_GATE_NONE))
    return nat::fail(NAT_ERR_INVALID_ARG, "%s: w_post and gate need y", who);
  if ((p->gate_mode != NAT_GATE_NONE) != (gate != nullptr))
    return nat::fail(NAT_ERR_INVALID_ARG, "%s: gate and gate_mode disagree", who);
  if (!r8 != !r8_scales || !y8 != !y8_scales || (y ? !y8 != !r8 : y8 != nullptr))
    return nat::fail(NAT_ERR_INVALID_ARG, "%s: checkpoints come whole (codes and scales, of y and r)",
                     who);
  if (cap == 0) return NAT_OK;
  if (!x || !r || (w_pre && (!h || !rstd_r)) || (w_post && !rstd_y))
    return nat::fail(NAT_ERR_INVALID_ARG, "%s: null pointer", who);
  if (nat::misaligned({x, y, r, h, w_post, w_pre, p->gate_mode == NAT_GATE_CHANNEL ? gate : nullptr, y8, r8}, 15u))
    return nat::fail(NAT_ERR_INVALID_ARG, "%s: rows, weights and codes must be 16-byte aligned", who);
  nat::FwdArgs a{};
  a.x = x; a.y = y; a.w_post = w_post; a.gate = gate; a.w_pre = w_pre; a.r = r; a.h = h;
  a.rstd_y = rstd_y; a.rstd_r = rstd_r; a.y8 = y8; a.r8 = r8; a.y8s = y8_scales; a.r8s = r8_scales;
  a.n_rows = n_rows; a.cap = cap; a.d = p->d; a.groups = (p->d + nat::rows::kGroup - 1) / nat::rows::kGroup;
  a.gate_mode = p->gate_mode; a.eps = p->eps; a.alpha = p->alpha; a.inv_d = 1.f / (float)p->d;
  return p->dtype == NAT_F32 ? nat::dispatch_fwd<float>(a, (cudaStream_t)stream)
                             : nat::dispatch_fwd<__nv_bfloat16>(a, (cudaStream_t)stream);
}

int nat_resnorm_bwd(const nat_resnorm_params* p, const void* y, const void* r, const int8_t* y8,
                    const float* y8_scales, const int8_t* r8, const float* r8_scales,
                    const float* w_post, const float* gate, const float* w_pre, const float* rstd_y,
                    const float* rstd_r, const int32_t* n_rows, int64_t cap, const void* dr,
                    const void* dh, void* dx, void* dy, float* dw_post, float* dgate, float* dw_pre,
                    void* workspace, size_t workspace_bytes, void* stream) {
  const char* who = "nat_resnorm_bwd";
  int s = nat::check_params(who, p, cap);
  if (s != NAT_OK) return s;
  if (!y8 != !y8_scales || !r8 != !r8_scales)
    return nat::fail(NAT_ERR_INVALID_ARG, "%s: checkpoints come whole (codes and scales)", who);
  if ((y && y8) || (r && r8) || (y && r8) || (r && y8))
    return nat::fail(NAT_ERR_INVALID_ARG, "%s: y and r come both as rows or both as checkpoints", who);
  const bool c8 = y8 || r8, has_y = y || y8;
  if (!has_y && (w_post || p->gate_mode != NAT_GATE_NONE || dy))
    return nat::fail(NAT_ERR_INVALID_ARG, "%s: w_post, gate and dy need y", who);
  if ((p->gate_mode != NAT_GATE_NONE) != (gate != nullptr))
    return nat::fail(NAT_ERR_INVALID_ARG, "%s: gate and gate_mode disagree", who);
  if (cap > 0 && (!dx || (w_pre && (!dh || !rstd_r || !(r || r8))) || (has_y && !dy) ||
                  (w_post && !rstd_y) || (!w_pre && !dr)))
    return nat::fail(NAT_ERR_INVALID_ARG, "%s: null pointer", who);
  if ((w_post && !dw_post) || (w_pre && !dw_pre) || (gate && !dgate))
    return nat::fail(NAT_ERR_INVALID_ARG, "%s: null gradient", who);
  if (nat::misaligned({y, r, dr, dh, dx, dy, w_post, w_pre, y8, r8,
                       p->gate_mode == NAT_GATE_CHANNEL ? gate : nullptr}, 15u))
    return nat::fail(NAT_ERR_INVALID_ARG, "%s: rows, weights and codes must be 16-byte aligned", who);
  const size_t need = nat_resnorm_workspace_bytes(p, cap);
  if (!workspace || workspace_bytes < need)
    return nat::fail(NAT_ERR_CAPACITY, "%s: workspace too small (%zu < %zu)", who, workspace_bytes, need);
  if ((uintptr_t)workspace & 255u)
    return nat::fail(NAT_ERR_INVALID_ARG, "%s: workspace must be 256-byte aligned", who);
  nat::BwdArgs a{};
  a.y = y; a.r = r; a.dr_in = dr; a.dh = dh; a.y8 = y8; a.r8 = r8; a.y8s = y8_scales; a.r8s = r8_scales;
  a.w_post = w_post; a.gate = gate; a.w_pre = w_pre; a.rstd_y = rstd_y; a.rstd_r = rstd_r;
  a.dx = dx; a.dy = dy; a.dgate_row = dgate; a.partial = (float*)workspace; a.n_rows = n_rows;
  a.cap = cap; a.d = p->d; a.groups = (p->d + nat::rows::kGroup - 1) / nat::rows::kGroup;
  a.gate_mode = p->gate_mode; a.alpha = p->alpha; a.inv_d = 1.f / (float)p->d; a.has_y = has_y;
  int64_t blocks = 0;
  s = p->dtype == NAT_F32 ? nat::dispatch_bwd<float>(a, c8, (cudaStream_t)stream, &blocks)
                          : nat::dispatch_bwd<__nv_bfloat16>(a, c8, (cudaStream_t)stream, &blocks);
  if (s != NAT_OK) return s;
  const bool channel = p->gate_mode == NAT_GATE_CHANNEL;
  if (w_post || w_pre || channel) {
    return nat::launch_after(nat::resnorm_columns_kernel, dim3((2 * p->d + 31) / 32), 256, 0, (cudaStream_t)stream,
                             "resnorm_columns_kernel", (const float*)a.partial, (int)blocks, (int)p->d,
                             channel ? 1 : 0, w_post, gate, w_post ? dw_post : nullptr, dgate,
                             w_pre ? dw_pre : nullptr);
  }
  return NAT_OK;
}

}  // extern "C"
