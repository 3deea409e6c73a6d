// The join of two blocks on packed rows, forward and backward: post-norm of a block's output,
// gate and residual scale, and the next block's pre-norm, in one pass over the rows.
//
//   n = y rstd_y w_post,  r = alpha x + gate n,  h = r rstd_r w_pre,  rstd = (mean(.^2) + eps)^-1/2
//
// Bound by HBM.  NT threads own a row, each with CH chunks of eight elements in registers, so
// that a row is read once although its two means follow one another; persistent blocks walk the rows and
// issue a row's loads while the row before it is reduced.  Weights stay in L1.
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
  int d, groups, gate_mode;
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
  int d, groups, gate_mode;
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

template <typename T, int NT, int CH, bool C8>
__global__ void __launch_bounds__(NT == 32 ? 128 : NT)
resnorm_fwd_kernel(FwdArgs a) {
  constexpr int RPB = NT == 32 ? 4 : 1;
  __shared__ float red[2][32];
  RowSum<NT, 1> row_sum{red};
  const int t = threadIdx.x % NT, sub = threadIdx.x / NT;
  const int64_t n = a.n_rows ? min((int64_t)max(*a.n_rows, 0), a.cap) : a.cap;
  const int64_t step = (int64_t)gridDim.x * RPB;
  const T* x = (const T*)a.x;
  const T* y = (const T*)a.y;
  rows::Raw<T> rx[CH], ry[CH];
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int col = (t + i * NT) * kChunk;
      const bool in = row < n && col < a.d;
      rx[i] = in ? rows::load_raw(x + row * a.d + col) : rows::zero_raw<T>();
      ry[i] = (in && y) ? rows::load_raw(y + row * a.d + col) : rows::zero_raw<T>();
    }
  };
  int64_t row = (int64_t)blockIdx.x * RPB + sub;
  fetch(row);
  for (; row < n; row += step) {
    float r[CH][kChunk], yv[CH][kChunk];
    float ss[1] = {0.f};
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      rows::widen(rx[i], r[i]);
      rows::widen(ry[i], yv[i]);
#pragma unroll
      for (int j = 0; j < kChunk; ++j) ss[0] = fmaf(yv[i][j], yv[i][j], ss[0]);
    }
    fetch(row + step);
    float inv_y = 1.f;
    if (a.w_post) {
      row_sum(ss);
      inv_y = __frsqrt_rn(fmaf(ss[0], a.inv_d, a.eps));
      if (t == 0) a.rstd_y[row] = inv_y;
    }
    const float gate_row = a.gate_mode == NAT_GATE_ROW ? a.gate[row] : 1.f;
    ss[0] = 0.f;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int col = (t + i * NT) * kChunk;
      const bool in = col < a.d;
      if (C8 && y) {
        const rows::GroupScale gs = rows::group_scale(rows::group_top(yv[i]));
        if (in) {
          __stcs(reinterpret_cast<uint2*>(a.y8 + row * a.d + col), rows::group_codes(yv[i], gs.inv));
          if ((t & 15) == 0) a.y8s[row * a.groups + (col >> 7)] = gs.scale;
        }
      }
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
        const rows::GroupScale gs = rows::group_scale(rows::group_top(rounded));
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

template <typename T, int NT, int CH, bool C8>
__global__ void __launch_bounds__(NT == 32 ? 128 : NT)
resnorm_bwd_kernel(BwdArgs a) {
  constexpr int RPB = NT == 32 ? 4 : 1;
  __shared__ float red1[2][32], red2[2][64];
  RowSum<NT, 1> sum1{red1};
  RowSum<NT, 2> sum2{red2};
  const int t = threadIdx.x % NT, sub = threadIdx.x / NT;
  const int64_t n = a.n_rows ? min((int64_t)max(*a.n_rows, 0), a.cap) : a.cap;
  const int64_t step = (int64_t)gridDim.x * RPB;
  float acc[CH][kChunk], acc_pre[CH][kChunk];
#pragma unroll
  for (int i = 0; i < CH; ++i)
#pragma unroll
    for (int j = 0; j < kChunk; ++j) acc[i][j] = acc_pre[i][j] = 0.f;

  rows::Raw<T> qy[CH], qr[CH], qdr[CH], qdh[CH];
  uint2 cy[CH], cr[CH];
  float sy[CH], sr[CH], inv_y_next = 1.f, inv_r_next = 1.f;
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int col = (t + i * NT) * kChunk;
      const bool in = row < n && col < a.d;
      const int64_t at = row * a.d + col;
      if (C8) {
        cy[i] = (in && a.has_y) ? __ldcs(reinterpret_cast<const uint2*>(a.y8 + at)) : make_uint2(0u, 0u);
        sy[i] = (in && a.has_y) ? __ldg(a.y8s + row * a.groups + (col >> 7)) : 0.f;
        cr[i] = (in && a.w_pre) ? __ldcs(reinterpret_cast<const uint2*>(a.r8 + at)) : make_uint2(0u, 0u);
        sr[i] = (in && a.w_pre) ? __ldg(a.r8s + row * a.groups + (col >> 7)) : 0.f;
      } else {
        qy[i] = (in && a.has_y) ? rows::load_raw((const T*)a.y + at) : rows::zero_raw<T>();
        qr[i] = (in && a.w_pre) ? rows::load_raw((const T*)a.r + at) : rows::zero_raw<T>();
      }
      qdr[i] = (in && a.dr_in) ? rows::load_raw((const T*)a.dr_in + at) : rows::zero_raw<T>();
      qdh[i] = (in && a.w_pre) ? rows::load_raw((const T*)a.dh + at) : rows::zero_raw<T>();
    }
    if (a.w_post && row < n) inv_y_next = __ldg(a.rstd_y + row);
    if (a.w_pre && row < n) inv_r_next = __ldg(a.rstd_r + row);
  };
  int64_t row = (int64_t)blockIdx.x * RPB + sub;
  fetch(row);
  for (; row < n; row += step) {
    float dr[CH][kChunk], rv[CH][kChunk], yv[CH][kChunk], u[CH][kChunk];
    const float inv_y = inv_y_next, inv_r = inv_r_next;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      if (C8) {
        rows::widen_codes(cr[i], sr[i], rv[i]);
        rows::widen_codes(cy[i], sy[i], yv[i]);
      } else {
        rows::widen(qr[i], rv[i]);
        rows::widen(qy[i], yv[i]);
      }
      rows::widen(qdr[i], dr[i]);
      rows::widen(qdh[i], u[i]);
    }
    fetch(row + step);
    if (a.w_pre) {
      float s1[1] = {0.f};
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int col = (t + i * NT) * kChunk;
        if (col < a.d) {
          float w[kChunk];
          rows::load_weights(a.w_pre + col, w);
#pragma unroll
          for (int j = 0; j < kChunk; ++j) {
            rv[i][j] *= inv_r;
            acc_pre[i][j] = fmaf(u[i][j], rv[i][j], acc_pre[i][j]);
            u[i][j] *= w[j];
            s1[0] = fmaf(u[i][j], rv[i][j], s1[0]);
          }
        }
      }
      sum1(s1);
      const float m = s1[0] * a.inv_d;
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int j = 0; j < kChunk; ++j)
          dr[i][j] = fmaf(inv_r, fmaf(-rv[i][j], m, u[i][j]), dr[i][j]);
    }
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int col = (t + i * NT) * kChunk;
      if (col < a.d) {
        float dx[kChunk];
#pragma unroll
        for (int j = 0; j < kChunk; ++j) dx[j] = a.alpha * dr[i][j];
        rows::Raw<T> out;
        rows::narrow(dx, out);
        rows::store_raw((T*)a.dx + row * a.d + col, out);
      }
    }
    if (a.has_y) {
      const float gate_row = a.gate_mode == NAT_GATE_ROW ? __ldg(a.gate + row) : 1.f;
      float s2[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int col = (t + i * NT) * kChunk;
        if (col < a.d) {
          float w[kChunk], g[kChunk];
#pragma unroll
          for (int j = 0; j < kChunk; ++j) w[j] = 1.f, g[j] = gate_row;
          if (a.w_post) rows::load_weights(a.w_post + col, w);
          if (a.gate_mode == NAT_GATE_CHANNEL) rows::load_weights(a.gate + col, g);
#pragma unroll
          for (int j = 0; j < kChunk; ++j) {
            yv[i][j] *= inv_y;  // yhat
            acc[i][j] = fmaf(dr[i][j] * gate_row, yv[i][j], acc[i][j]);
            s2[1] = fmaf(dr[i][j] * yv[i][j], w[j], s2[1]);
            dr[i][j] *= g[j] * w[j];  // v
            s2[0] = fmaf(dr[i][j], yv[i][j], s2[0]);
          }
        }
      }
      if (a.w_post || a.gate_mode == NAT_GATE_ROW) sum2(s2);
      if (a.gate_mode == NAT_GATE_ROW && t == 0) a.dgate_row[row] = s2[1];
      const float m = a.w_post ? s2[0] * a.inv_d : 0.f;
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int col = (t + i * NT) * kChunk;
        if (col < a.d) {
          float dy[kChunk];
#pragma unroll
          for (int j = 0; j < kChunk; ++j)
            dy[j] = a.w_post ? inv_y * fmaf(-yv[i][j], m, dr[i][j]) : dr[i][j];
          rows::Raw<T> out;
          rows::narrow(dy, out);
          rows::store_raw((T*)a.dy + row * a.d + col, out);
        }
      }
    }
  }

  // the block's sums; four warps with rows of their own are added in warp order first
  if (RPB == 1) {
    float* p = a.partial + (int64_t)blockIdx.x * 2 * a.d;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int col = (t + i * NT) * kChunk;
      if (col < a.d)
#pragma unroll
        for (int j = 0; j < kChunk; ++j) p[col + j] = acc[i][j], p[a.d + col + j] = acc_pre[i][j];
    }
  } else {
    constexpr int kCols = RPB > 1 ? 32 * CH * kChunk : 1;
    __shared__ float part[2][RPB][kCols];
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int j = 0; j < kChunk; ++j) {
        part[0][sub][(t + i * 32) * kChunk + j] = acc[i][j];
        part[1][sub][(t + i * 32) * kChunk + j] = acc_pre[i][j];
      }
    __syncthreads();
    float* p = a.partial + (int64_t)blockIdx.x * 2 * a.d;
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
// and four inputs take the registers); below 256 columns a warp has a row to itself.
constexpr int kMaxD = 8192;

int threads_of(int d, int chunks) {
  int nt = 32;
  while (nt * chunks * kChunk < d) nt *= 2;
  return nt;
}

// Persistent blocks: about 1024 resident threads a multiprocessor, each with one row in flight
// and one being loaded.
int64_t blocks_of(int nt, int64_t cap) {
  const int per_block = nt == 32 ? 4 : 1, threads = nt == 32 ? 128 : nt;
  const int64_t most = 148ll * max(1, 1024 / threads);
  const int64_t want = (cap + per_block - 1) / per_block;
  return max((int64_t)1, min(most, want));
}

template <typename T, int NT, int CH>
int launch_fwd(const FwdArgs& a, cudaStream_t stream) {
  const int64_t blocks = blocks_of(NT, a.cap);
  const int threads = NT == 32 ? 128 : NT;
  if (a.r8) resnorm_fwd_kernel<T, NT, CH, true><<<(unsigned)blocks, threads, 0, stream>>>(a);
  else resnorm_fwd_kernel<T, NT, CH, false><<<(unsigned)blocks, threads, 0, stream>>>(a);
  NAT_LAUNCH_CHECK("resnorm_fwd_kernel");
  return NAT_OK;
}

template <typename T>
int dispatch_fwd(const FwdArgs& a, cudaStream_t stream) {
  switch (threads_of(a.d, 2)) {
    case 32: return launch_fwd<T, 32, 2>(a, stream);
    case 64: return launch_fwd<T, 64, 2>(a, stream);
    case 128: return launch_fwd<T, 128, 2>(a, stream);
    case 256: return launch_fwd<T, 256, 2>(a, stream);
    default: return launch_fwd<T, 512, 2>(a, stream);
  }
}

template <typename T, int NT, int CH>
int launch_bwd(const BwdArgs& a, bool c8, cudaStream_t stream) {
  const int64_t blocks = blocks_of(NT, a.cap);
  const int threads = NT == 32 ? 128 : NT;
  if (c8) resnorm_bwd_kernel<T, NT, CH, true><<<(unsigned)blocks, threads, 0, stream>>>(a);
  else resnorm_bwd_kernel<T, NT, CH, false><<<(unsigned)blocks, threads, 0, stream>>>(a);
  NAT_LAUNCH_CHECK("resnorm_bwd_kernel");
  return NAT_OK;
}

template <typename T>
int dispatch_bwd(const BwdArgs& a, bool c8, cudaStream_t stream) {
  switch (threads_of(a.d, 1)) {
    case 32: return launch_bwd<T, 32, 1>(a, c8, stream);
    case 64: return launch_bwd<T, 64, 1>(a, c8, stream);
    case 128: return launch_bwd<T, 128, 1>(a, c8, stream);
    case 256: return launch_bwd<T, 256, 1>(a, c8, stream);
    case 512: return launch_bwd<T, 512, 1>(a, c8, stream);
    default: return launch_bwd<T, 1024, 1>(a, c8, stream);
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
  const int64_t blocks = nat::blocks_of(nat::threads_of(p->d, 1), cap);
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
  s = p->dtype == NAT_F32 ? nat::dispatch_bwd<float>(a, c8, (cudaStream_t)stream)
                          : nat::dispatch_bwd<__nv_bfloat16>(a, c8, (cudaStream_t)stream);
  if (s != NAT_OK) return s;
  const int blocks = (int)nat::blocks_of(nat::threads_of(p->d, 1), cap);
  const bool channel = p->gate_mode == NAT_GATE_CHANNEL;
  if (w_post || w_pre || channel) {
    nat::resnorm_columns_kernel<<<(2 * p->d + 31) / 32, 256, 0, (cudaStream_t)stream>>>(
        a.partial, blocks, p->d, channel ? 1 : 0, w_post, gate, w_post ? dw_post : nullptr, dgate,
        w_pre ? dw_pre : nullptr);
    NAT_LAUNCH_CHECK("resnorm_columns_kernel");
  }
  return NAT_OK;
}

}  // extern "C"
