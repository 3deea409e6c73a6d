// The join of two blocks on packed rows, forward and backward: post-norm of a block's output,
// gate and residual scale, and the next block's pre-norm, in one pass over the rows.
//
//   n = y rstd_y w_post,  r = alpha x + gate n,  h = r rstd_r w_pre,  rstd = (mean(.^2) + eps)^-1/2
//
// Bound by HBM.  NT threads own a row, each with CH chunks of eight elements in registers, so
// that a row is read once although its two means follow one another; persistent blocks walk the rows,
// with the next rows (up to three) on their way into shared memory by asynchronous copies: the loads
// in flight, 60 KB and more a multiprocessor, are what the bandwidth needs, and registers would not
// hold them beside the column sums.  Weights stay in L1.
//
// Backward, with u = dh w_pre, rhat = r rstd_r, yhat = y rstd_y:
//   dr = dr_in + rstd_r (u - rhat mean(u rhat)),   dx = alpha dr,   dn = gate dr,
//   v = dn w_post,  dy = rstd_y (v - yhat mean(v yhat)),
//   dw_pre = sum dh rhat,  dw_post = sum dn yhat,  dgate = sum dr n  (over rows, or over a row).
// A gate per column factors out of its sum: dw_post = gate A, dgate = w_post A with one
// A = sum dr yhat, so a thread keeps two sums per column.  Every block leaves its sums in the
// workspace and a second kernel adds them in block order: the gradients of the weights repeat
// bit for bit.
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

// Sum over the NT threads of a row, the same in every thread.  `buf` alternates between calls,
// so one barrier a call is enough: a buffer is written again only after the next call's barrier.
template <int NT, int N>
struct RowSum {
  float (*buf)[N * 32];
  uint32_t turn = 0;
  __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
    if (NT > 32) {
      constexpr int W = NT / 32;
      float* b = buf[turn & 1];
      ++turn;
      if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int k = 0; k < N; ++k) b[k * W + (threadIdx.x >> 5)] = v[k];
      __syncthreads();
#pragma unroll
      for (int k = 0; k < N; ++k) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) s += b[k * W + w];
        v[k] = s;
      }
    }
  }
};

// Threads and rows of a block: below 256 columns a warp has a row to itself, four to a block.
constexpr __host__ __device__ int block_threads(int nt) { return nt == 32 ? 128 : nt; }
constexpr __host__ __device__ int block_rows(int nt) { return nt == 32 ? 4 : 1; }

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

template <typename T, int NT, int CH, bool C8>
__global__ void __launch_bounds__(block_threads(NT), 1024 / block_threads(NT))
resnorm_fwd_kernel(FwdArgs a) {
  constexpr int RPB = block_rows(NT), P = Pieces<T>::kRaw, BT = block_threads(NT);
  extern __shared__ uint4 ring[];  // [stages][x, y][CH][P][BT]
  __shared__ float red[2][32];
  RowSum<NT, 1> row_sum{red};
  const int t = threadIdx.x % NT, sub = threadIdx.x / NT;
  const int64_t n = a.n_rows ? min((int64_t)max(*a.n_rows, 0), a.cap) : a.cap;
  const int64_t step = (int64_t)gridDim.x * RPB;
  const T* x = (const T*)a.x;
  const T* y = (const T*)a.y;
  auto slot = [&](int stage, int of, int i) { return ring + (((stage * 2 + of) * CH + i) * P) * BT + threadIdx.x; };
  auto fetch = [&](int64_t row, int stage) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int col = (t + i * NT) * kChunk;
      if (row < n && col < a.d) {
        copy_piece<T, NT>(slot(stage, 0, i), x + row * a.d + col);
        if (y) copy_piece<T, NT>(slot(stage, 1, i), y + row * a.d + col);
      }
    }
    rows::copies_commit();
  };
  int64_t row = (int64_t)blockIdx.x * RPB + sub;
  for (int k = 0; k < a.stages; ++k) fetch(row + k * step, k);
  for (int stage = 0; row < n; row += step, stage = stage + 1 == a.stages ? 0 : stage + 1) {
    const float gate_row = a.gate_mode == NAT_GATE_ROW ? __ldg(a.gate + row) : 1.f;
    rows::copies_wait(a.stages - 1);
    rows::Raw<T> qy[CH];
    float r[CH][kChunk], yv[CH][kChunk];
    float ss[1] = {0.f};
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const bool in = (t + i * NT) * kChunk < a.d;
      rows::widen(in ? read_piece<T, NT>(slot(stage, 0, i)) : rows::zero_raw<T>(), r[i]);
      qy[i] = (in && y) ? read_piece<T, NT>(slot(stage, 1, i)) : rows::zero_raw<T>();
      rows::widen(qy[i], yv[i]);
#pragma unroll
      for (int j = 0; j < kChunk; ++j) ss[0] = fmaf(yv[i][j], yv[i][j], ss[0]);
    }
    fetch(row + a.stages * step, stage);
    if (C8 && y) {  // while the copies are issued and the sum is on its way
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int col = (t + i * NT) * kChunk;
        const rows::GroupScale gs = rows::group_scale(rows::group_top(qy[i]));
        if (col < a.d) {
          __stcs(reinterpret_cast<uint2*>(a.y8 + row * a.d + col), rows::group_codes(yv[i], gs.inv));
          if ((t & 15) == 0) a.y8s[row * a.groups + (col >> 7)] = gs.scale;
        }
      }
    }
    float inv_y = 1.f;
    if (a.w_post) {
      row_sum(ss);
      inv_y = __frsqrt_rn(fmaf(ss[0], a.inv_d, a.eps));
      if (t == 0) a.rstd_y[row] = inv_y;
    }
    ss[0] = 0.f;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int col = (t + i * NT) * kChunk;
      const bool in = col < a.d;
      if (in) {
        float w[kChunk], g[kChunk];
#pragma unroll
        for (int j = 0; j < kChunk; ++j) w[j] = 1.f, g[j] = gate_row;
        if (a.w_post) rows::load_weights(a.w_post + col, w);
        if (a.gate_mode == NAT_GATE_CHANNEL) rows::load_weights(a.gate + col, g);
#pragma unroll
        for (int j = 0; j < kChunk; ++j) {
          r[i][j] *= a.alpha;
          if (y) r[i][j] = fmaf(g[j], yv[i][j] * inv_y * w[j], r[i][j]);
        }
      }
      // h is formed from r before its rounding: the norm then adds no error of its own
#pragma unroll
      for (int j = 0; j < kChunk; ++j) ss[0] = fmaf(r[i][j], r[i][j], ss[0]);
      rows::Raw<T> out;
      rows::narrow(r[i], out);
      if (in) rows::store_raw((T*)a.r + row * a.d + col, out);
      if (C8) {
        float rounded[kChunk];  // the checkpoint is of the row as it is stored
        rows::widen(out, rounded);
        const rows::GroupScale gs = rows::group_scale(rows::group_top(out));
        if (in) {
          __stcs(reinterpret_cast<uint2*>(a.r8 + row * a.d + col), rows::group_codes(rounded, gs.inv));
          if ((t & 15) == 0) a.r8s[row * a.groups + (col >> 7)] = gs.scale;
        }
      }
    }
    if (a.w_pre) {
      row_sum(ss);
      const float inv_r = __frsqrt_rn(fmaf(ss[0], a.inv_d, a.eps));
      if (t == 0) a.rstd_r[row] = inv_r;
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int col = (t + i * NT) * kChunk;
        if (col < a.d) {
          float w[kChunk];
          rows::load_weights(a.w_pre + col, w);
#pragma unroll
          for (int j = 0; j < kChunk; ++j) w[j] *= r[i][j] * inv_r;
          rows::Raw<T> out;
          rows::narrow(w, out);
          rows::store_raw((T*)a.h + row * a.d + col, out);
        }
      }
    }
  }
}

// A thread has one chunk of a row.
template <typename T, int NT, bool C8>
__global__ void __launch_bounds__(block_threads(NT), 1024 / block_threads(NT))
resnorm_bwd_kernel(BwdArgs a) {
  constexpr int RPB = block_rows(NT), P = Pieces<T>::kRaw, BT = block_threads(NT);
  // [stages][dr, dh: P pieces each][y, r: P pieces each, or one of codes (8 bytes y, 8 bytes r)][BT]
  constexpr int kPieces = C8 ? 2 * P + 1 : 4 * P;
  extern __shared__ uint4 ring[];
  __shared__ float red1[2][32], red2[2][64];
  RowSum<NT, 1> sum1{red1};
  RowSum<NT, 2> sum2{red2};
  const int t = threadIdx.x % NT, sub = threadIdx.x / NT, col = t * kChunk;
  const bool in_row = col < a.d;
  const int64_t n = a.n_rows ? min((int64_t)max(*a.n_rows, 0), a.cap) : a.cap;
  const int64_t step = (int64_t)gridDim.x * RPB;
  float acc[kChunk], acc_pre[kChunk];
#pragma unroll
  for (int j = 0; j < kChunk; ++j) acc[j] = acc_pre[j] = 0.f;

  auto slot = [&](int stage, int piece) { return ring + (stage * kPieces + piece) * BT + threadIdx.x; };
  auto fetch = [&](int64_t row, int stage) {
    if (row < n && in_row) {
      const int64_t at = row * a.d + col;
      if (a.dr_in) copy_piece<T, NT>(slot(stage, 0), (const T*)a.dr_in + at);
      if (a.w_pre) copy_piece<T, NT>(slot(stage, P), (const T*)a.dh + at);
      if (C8) {
        uint2* codes = reinterpret_cast<uint2*>(slot(stage, 2 * P));
        if (a.has_y) rows::copy_async<8>(codes, a.y8 + at);
        if (a.w_pre) rows::copy_async<8>(codes + 1, a.r8 + at);
      } else {
        if (a.has_y) copy_piece<T, NT>(slot(stage, 2 * P), (const T*)a.y + at);
        if (a.w_pre) copy_piece<T, NT>(slot(stage, 3 * P), (const T*)a.r + at);
      }
    }
    rows::copies_commit();
  };
  // the row's scalars, one row ahead in registers
  float inv_y_next = 1.f, inv_r_next = 1.f, gate_next = 1.f, sy_next = 0.f, sr_next = 0.f;
  auto fetch_scalars = [&](int64_t row) {
    if (row >= n) return;
    if (a.w_post) inv_y_next = __ldg(a.rstd_y + row);
    if (a.w_pre) inv_r_next = __ldg(a.rstd_r + row);
    if (a.gate_mode == NAT_GATE_ROW) gate_next = __ldg(a.gate + row);
    if (C8 && in_row) {
      if (a.has_y) sy_next = __ldg(a.y8s + row * a.groups + (col >> 7));
      if (a.w_pre) sr_next = __ldg(a.r8s + row * a.groups + (col >> 7));
    }
  };
  int64_t row = (int64_t)blockIdx.x * RPB + sub;
  for (int k = 0; k < a.stages; ++k) fetch(row + k * step, k);
  fetch_scalars(row);
  for (int stage = 0; row < n; row += step, stage = stage + 1 == a.stages ? 0 : stage + 1) {
    const float inv_y = inv_y_next, inv_r = inv_r_next, gate_row = gate_next, sy = sy_next, sr = sr_next;
    float dr[kChunk], yv[kChunk];
    rows::copies_wait(a.stages - 1);
    if (C8) {
      const uint4 c = (in_row && a.has_y) ? *slot(stage, 2 * P) : make_uint4(0u, 0u, 0u, 0u);
      rows::widen_codes(make_uint2(c.x, c.y), sy, yv);
    } else {
      rows::widen((in_row && a.has_y) ? read_piece<T, NT>(slot(stage, 2 * P)) : rows::zero_raw<T>(), yv);
    }
    rows::widen((in_row && a.dr_in) ? read_piece<T, NT>(slot(stage, 0)) : rows::zero_raw<T>(), dr);
    if (a.w_pre) {
      float rv[kChunk], u[kChunk];
      float s1[1] = {0.f};
#pragma unroll
      for (int j = 0; j < kChunk; ++j) rv[j] = u[j] = 0.f;
      if (in_row) {
        if (C8) {
          const uint4 c = *slot(stage, 2 * P);
          rows::widen_codes(make_uint2(c.z, c.w), sr, rv);
        } else {
          rows::widen(read_piece<T, NT>(slot(stage, 3 * P)), rv);
        }
        rows::widen(read_piece<T, NT>(slot(stage, P)), u);
        float w[kChunk];
        rows::load_weights(a.w_pre + col, w);
#pragma unroll
        for (int j = 0; j < kChunk; ++j) {
          rv[j] *= inv_r;
          acc_pre[j] = fmaf(u[j], rv[j], acc_pre[j]);
          u[j] *= w[j];
          s1[0] = fmaf(u[j], rv[j], s1[0]);
        }
      }
      fetch(row + a.stages * step, stage);
      fetch_scalars(row + step);
      sum1(s1);
      const float m = s1[0] * a.inv_d;
#pragma unroll
      for (int j = 0; j < kChunk; ++j) dr[j] = fmaf(inv_r, fmaf(-rv[j], m, u[j]), dr[j]);
    } else {
      fetch(row + a.stages * step, stage);
      fetch_scalars(row + step);
    }
    if (in_row) {
      float dx[kChunk];
#pragma unroll
      for (int j = 0; j < kChunk; ++j) dx[j] = a.alpha * dr[j];
      rows::Raw<T> out;
      rows::narrow(dx, out);
      rows::store_raw((T*)a.dx + row * a.d + col, out);
    }
    if (a.has_y) {
      float s2[2] = {0.f, 0.f};
      if (in_row) {
        float w[kChunk], g[kChunk];
#pragma unroll
        for (int j = 0; j < kChunk; ++j) w[j] = 1.f, g[j] = gate_row;
        if (a.w_post) rows::load_weights(a.w_post + col, w);
        if (a.gate_mode == NAT_GATE_CHANNEL) rows::load_weights(a.gate + col, g);
#pragma unroll
        for (int j = 0; j < kChunk; ++j) {
          yv[j] *= inv_y;  // yhat
          acc[j] = fmaf(dr[j] * gate_row, yv[j], acc[j]);
          s2[1] = fmaf(dr[j] * yv[j], w[j], s2[1]);
          dr[j] *= g[j] * w[j];  // v
          s2[0] = fmaf(dr[j], yv[j], s2[0]);
        }
      }
      if (a.w_post || a.gate_mode == NAT_GATE_ROW) sum2(s2);
      if (a.gate_mode == NAT_GATE_ROW && t == 0) a.dgate_row[row] = s2[1];
      if (in_row) {
        const float m = s2[0] * a.inv_d;
        float dy[kChunk];
#pragma unroll
        for (int j = 0; j < kChunk; ++j) dy[j] = a.w_post ? inv_y * fmaf(-yv[j], m, dr[j]) : dr[j];
        rows::Raw<T> out;
        rows::narrow(dy, out);
        rows::store_raw((T*)a.dy + row * a.d + col, out);
      }
    }
  }

  // the block's sums; four warps with rows of their own are added in warp order first
  float* p = a.partial + (int64_t)blockIdx.x * 2 * a.d;
  if (RPB == 1) {
    if (in_row)
#pragma unroll
      for (int j = 0; j < kChunk; ++j) p[col + j] = acc[j], p[a.d + col + j] = acc_pre[j];
  } else {
    __shared__ float part[2][RPB][RPB > 1 ? 32 * kChunk : 1];
#pragma unroll
    for (int j = 0; j < kChunk; ++j) part[0][sub][col + j] = acc[j], part[1][sub][col + j] = acc_pre[j];
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * a.d; c += blockDim.x) {
      const int which = c >= a.d;
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < RPB; ++w) s += part[which][w][c - which * a.d];
      p[c] = s;
    }
  }
}

// Adds the blocks' sums in block order (eight strided runs, joined in order) and applies the
// factors that were kept out of them.
__global__ void __launch_bounds__(256)
resnorm_columns_kernel(const float* __restrict__ partial, int blocks, int d, int gate_channel,
                       const float* __restrict__ w_post, const float* __restrict__ gate,
                       float* __restrict__ dw_post, float* __restrict__ dgate,
                       float* __restrict__ dw_pre) {
  __shared__ float part[8][33];
  const int lane = threadIdx.x & 31, run = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;  // over 2 d columns
  float s = 0.f;
  if (c < 2 * d)
    for (int b = run; b < blocks; b += 8) s += partial[(int64_t)b * 2 * d + c];
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
// Threads of a row by its length: two chunks a thread forward, one backward (whose column sums
// take the registers).
constexpr int kMaxD = 8192;

int threads_of(int d, int chunks) {
  int nt = 32;
  while (nt * chunks * kChunk < d) nt *= 2;
  return nt;
}

// Persistent blocks, all resident: 1024 threads a multiprocessor (64 registers each), fewer where
// the rows on their way would not fit into its shared memory.
constexpr int kSmemPerSm = 216 * 1024;  // of 228 KB, less 1 KB and the static part a block

struct Shape {
  int64_t blocks;
  int stages;
  size_t smem;
};
Shape shape_of(int nt, size_t stage_bytes, int64_t cap) {
  int per_sm = 1024 / block_threads(nt);
  const int fit = (int)(kSmemPerSm / stage_bytes);
  if (per_sm > fit) per_sm = fit > 0 ? fit : 1;
  Shape s;
  const int64_t want = (cap + block_rows(nt) - 1) / block_rows(nt);
  s.blocks = max((int64_t)1, min((int64_t)148 * per_sm, want));
  s.stages = (int)min((size_t)3, max((size_t)1, kSmemPerSm / per_sm / stage_bytes));
  s.smem = s.stages * stage_bytes;
  return s;
}

// Blocks of a backward pass at most: its workspace holds their column sums.
int64_t max_blocks(int nt, int64_t cap) {
  return max((int64_t)1, min((int64_t)148 * (1024 / block_threads(nt)), (cap + block_rows(nt) - 1) / block_rows(nt)));
}

template <typename K, typename A>
int launch(K kernel, A& a, int nt, size_t stage_bytes, cudaStream_t stream, int64_t* blocks, const char* name) {
  const Shape s = shape_of(nt, stage_bytes, a.cap);
  a.stages = s.stages;
  *blocks = s.blocks;
  if (s.smem > 32 * 1024)  // with the static part past the 48 KB of a plain launch
    NAT_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)s.smem));
  kernel<<<(unsigned)s.blocks, block_threads(nt), s.smem, stream>>>(a);
  NAT_LAUNCH_CHECK(name);
  return NAT_OK;
}

template <typename T, int NT>
int launch_fwd(FwdArgs& a, cudaStream_t stream) {
  constexpr size_t stage = (size_t)2 * 2 * sizeof(rows::Raw<T>) * block_threads(NT);
  int64_t blocks;
  return a.r8 ? launch(resnorm_fwd_kernel<T, NT, 2, true>, a, NT, stage, stream, &blocks, "resnorm_fwd_kernel")
              : launch(resnorm_fwd_kernel<T, NT, 2, false>, a, NT, stage, stream, &blocks, "resnorm_fwd_kernel");
}

template <typename T>
int dispatch_fwd(FwdArgs& a, cudaStream_t stream) {
  switch (threads_of(a.d, 2)) {
    case 32: return launch_fwd<T, 32>(a, stream);
    case 64: return launch_fwd<T, 64>(a, stream);
    case 128: return launch_fwd<T, 128>(a, stream);
    case 256: return launch_fwd<T, 256>(a, stream);
    default: return launch_fwd<T, 512>(a, stream);
  }
}

template <typename T, int NT>
int launch_bwd(BwdArgs& a, bool c8, cudaStream_t stream, int64_t* blocks) {
  constexpr size_t raw = sizeof(rows::Raw<T>), bt = block_threads(NT);
  return c8 ? launch(resnorm_bwd_kernel<T, NT, true>, a, NT, (2 * raw + 16) * bt, stream, blocks, "resnorm_bwd_kernel")
            : launch(resnorm_bwd_kernel<T, NT, false>, a, NT, 4 * raw * bt, stream, blocks, "resnorm_bwd_kernel");
}

template <typename T>
int dispatch_bwd(BwdArgs& a, bool c8, cudaStream_t stream, int64_t* blocks) {
  switch (threads_of(a.d, 1)) {
    case 32: return launch_bwd<T, 32>(a, c8, stream, blocks);
    case 64: return launch_bwd<T, 64>(a, c8, stream, blocks);
    case 128: return launch_bwd<T, 128>(a, c8, stream, blocks);
    case 256: return launch_bwd<T, 256>(a, c8, stream, blocks);
    case 512: return launch_bwd<T, 512>(a, c8, stream, blocks);
    default: return launch_bwd<T, 1024>(a, c8, stream, blocks);
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
  const int64_t blocks = nat::max_blocks(nat::threads_of(p->d, 1), cap);
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
    nat::resnorm_columns_kernel<<<(2 * p->d + 31) / 32, 256, 0, (cudaStream_t)stream>>>(
        a.partial, (int)blocks, p->d, channel ? 1 : 0, w_post, gate, w_post ? dw_post : nullptr, dgate,
        w_pre ? dw_pre : nullptr);
    NAT_LAUNCH_CHECK("resnorm_columns_kernel");
  }
  return NAT_OK;
}

}  // extern "C"
