// Products grouped by expert on the tensor cores where the experts have few rows: y = x w_e^T and dx = dy w_e.
//
// What bounds them then is the reading of the weights, and an MMA's time is that of its slots, filled or not: with the
// rows along M (256 slots of a CTA pair) it would take as long as the weights.  So the weights lie along M, 128 of
// their rows (or columns) a tile, and up to 128 rows of x along N, which an MMA takes in steps of 16:
//   D[c, r] = sum_k w[c, k] x[r, k]
// One CTA a multiprocessor with 32 KB stages of weights and rows; warp 0 loads by TMA, warp 1 issues, four warps write
// D out, a row's 32 columns at a time.  Rows behind a tile's last are another expert's: they fill columns of D that
// nobody writes out.  Every wait is bounded and raises NAT_DEV_TIMEOUT.
#include "nat_experts_tc.cuh"

namespace nat {
namespace experts {
namespace {

constexpr int kABytes = BM * BK * 2, kBBytes = kFewRows * BK * 2, kStage = kABytes + kBBytes;
constexpr int kNS = 227 * 1024 / kStage - (227 * 1024 % kStage < 1280 ? 1 : 0), kThreads = 192;
constexpr int kTmemCols = kFewRows < 32 ? 64 : 2 * kFewRows;  // two tiles
constexpr size_t kSmem = (size_t)kNS * kStage + 1024 /*alignment*/ + 256 /*barriers*/;
constexpr int kPiece = 16;               // rows that are loaded together

struct FewArgs {
  Head* head;
  const Tile* tiles;
  int n_cols, k_blocks;
  __nv_bfloat16* out;
  int64_t out_stride;
};

__device__ __forceinline__ void load_3d(void* dst, const CUtensorMap* map, uint64_t* bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(tc::smem_u32(dst)),
      "l"(map), "r"(tc::smem_u32(bar)), "r"(x), "r"(y), "r"(z)
      : "memory");
}

template <int WHICH>
__global__ void __launch_bounds__(kThreads, 1)
few_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
           const __grid_constant__ CUtensorMap map_x16, const FewArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint64_t* full_bar = reinterpret_cast<uint64_t*>(smem + (size_t)kNS * kStage);
  uint64_t* empty_bar = full_bar + kNS;
  uint64_t* tfull_bar = empty_bar + kNS;   // [2]
  uint64_t* tempty_bar = tfull_bar + 2;    // [2]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tempty_bar + 2);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kNS; ++s) {
      tc::mbar_init(&full_bar[s], 1);
      tc::mbar_init(&empty_bar[s], 1);
    }
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(&tfull_bar[i], 1);
      tc::mbar_init(&tempty_bar[i], 4);
    }
    *abort_flag = 0u;
    tc::fence_barrier_init();
    tc::fence_proxy_async();
    tc::prefetch_tensormap(&map_w);
    tc::prefetch_tensormap(&map_x);
    tc::prefetch_tensormap(&map_x16);
  }
  if (warp == 1) {
    tc::tmem_alloc(tmem_slot, kTmemCols);
    tc::tmem_relinquish();
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;
  wait_for_primary();  // the list of tiles is there

  // a tile's columns one after the other, so that the CTAs at work read an expert's weights in their order
  const int m_tiles = (a.n_cols + BM - 1) / BM;
  const int units = (int)a.head->tiles * m_tiles, stride = gridDim.x;
  auto tile_of = [&](int u) { return a.tiles[min(u, max(units - 1, 0)) / m_tiles]; };

  if (warp == 0) {
    // ------------------------------------------------ TMA producer
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      Tile next = tile_of(blockIdx.x);
      for (int u = blockIdx.x; ok && u < units; u += stride) {
        const Tile t = next;
        next = tile_of(u + stride);
        const int m0 = u % m_tiles * BM, pieces = (t.hi - t.lo + kPiece - 1) / kPiece;
        for (int kb = 0; kb < a.k_blocks; ++kb, ++it) {
          const int s = it % kNS;
          if (!tc::mbar_wait(&empty_bar[s], ((it / kNS) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
          uint8_t* w_dst = smem + (size_t)s * kStage;
          uint8_t* x_dst = w_dst + kABytes;
          tc::mbar_arrive_expect_tx(&full_bar[s], kABytes + pieces * kPiece * BK * 2);
          if (WHICH == kFwd) {
            load_3d(w_dst, &map_w, &full_bar[s], kb * BK, m0, t.expert);
          } else {
#pragma unroll
            for (int j = 0; j < 2; ++j) load_3d(w_dst + j * kBox, &map_w, &full_bar[s], m0 + j * 64, kb * BK, t.expert);
          }
          if (pieces == kFewRows / kPiece) {
            tc::tma_load_2d(x_dst, &map_x, &full_bar[s], kb * BK, t.lo);
          } else {
            for (int i = 0; i < pieces; ++i)
              tc::tma_load_2d(x_dst + i * kPiece * BK * 2, &map_x16, &full_bar[s], kb * BK, t.lo + i * kPiece);
          }
        }
      }
      // every stage is released before the CTA leaves: no load is still writing its shared memory
      const uint32_t pending = it < (uint32_t)kNS ? it : (uint32_t)kNS;
      for (uint32_t j = 0; j < pending; ++j) {
        const uint32_t jt = it - 1 - j;
        if (ok) ok = tc::mbar_wait(&empty_bar[jt % kNS], (jt / kNS) & 1u, abort_flag);
        if (!ok) {  // given up: the loads' own end, again with a limit
          const uint64_t t0 = tc::global_timer_ns();
          while (!tc::mbar_try_wait(&full_bar[jt % kNS], (jt / kNS) & 1u))
            if (tc::global_timer_ns() - t0 > 100000000ull) break;
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------------------------ MMA issuer
    if (lane == 0) {
      uint32_t it = 0, tcount = 0;
      bool ok = true;
      Tile next = tile_of(blockIdx.x);
      for (int u = blockIdx.x; ok && u < units; u += stride, ++tcount) {
        const Tile t = next;
        next = tile_of(u + stride);
        const uint32_t acc = tcount & 1u;
        const uint32_t idesc = tc::instr_desc_bf16(BM, (t.hi - t.lo + 15) / 16 * 16, WHICH == kDx ? 1 : 0, 0);
        if (!tc::mbar_wait(&tempty_bar[acc], ((tcount >> 1) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
        tc::fence_after_sync();
        for (int kb = 0; kb < a.k_blocks; ++kb, ++it) {
          const int s = it % kNS;
          if (!tc::mbar_wait(&full_bar[s], (it / kNS) & 1u, abort_flag)) { ok = false; break; }
          tc::fence_after_sync();
          const uint32_t w_base = tc::smem_u32(smem + (size_t)s * kStage), x_base = w_base + kABytes;
#pragma unroll
          for (int kk = 0; kk < BK / 16; ++kk) {
            const uint64_t wdesc = WHICH == kDx ? tc::smem_desc_sw128(w_base + kk * 2048, kBox, 1024)
                                                : tc::smem_desc_sw128(w_base + kk * 32, 16, 1024);
            const uint64_t xdesc = tc::smem_desc_sw128(x_base + kk * 32, 16, 1024);
            tc::umma_bf16(tmem_base + acc * kFewRows, wdesc, xdesc, idesc, (kb > 0 || kk > 0) ? 1u : 0u);
          }
          tc::umma_commit(&empty_bar[s]);
        }
        if (ok) tc::umma_commit(&tfull_bar[acc]);
      }
    }
    __syncwarp();
  } else {
    // ------------------------------------------------ epilogue
    const int q = warp & 3;  // tensor-memory lanes that this warp may read: columns of the result
    uint32_t tcount = 0;
    bool ok = true;
    Tile next = tile_of(blockIdx.x);
    for (int u = blockIdx.x; ok && u < units; u += stride, ++tcount) {
      const Tile t = next;
      next = tile_of(u + stride);
      const uint32_t acc = tcount & 1u;
      ok = __all_sync(0xFFFFFFFFu, tc::mbar_wait(&tfull_bar[acc], (tcount >> 1) & 1u, abort_flag) ? 1 : 0) != 0;
      if (!ok) break;
      tc::fence_after_sync();
      const int col = u % m_tiles * BM + q * 32 + lane, rows = t.hi - t.lo;
      __nv_bfloat16* out = a.out + (int64_t)t.lo * a.out_stride + col;
#pragma unroll 1
      for (int c = 0; c < rows; c += 32) {
        uint32_t v[32];
        tc::tmem_ld32_issue(tmem_base + ((uint32_t)(q * 32) << 16) + acc * kFewRows + c, v);
        tc::tmem_ld_wait(v);
        if (col < a.n_cols) {
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if (c + j < rows) out[(int64_t)(c + j) * a.out_stride] = __float2bfloat16_rn(__uint_as_float(v[j]));
        }
        __syncwarp();
      }
      tc::fence_before_sync();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&tempty_bar[acc]);
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag != 0u) atomicOr(&a.head->status, NAT_DEV_TIMEOUT);
  if (warp == 1) {
    tc::fence_after_sync();
    tc::tmem_dealloc(tmem_base, kTmemCols);
  }
}

template <int WHICH>
int launch(const CUtensorMap& mw, const CUtensorMap& mx, const CUtensorMap& mx16, const FewArgs& f, int64_t most_units,
           cudaStream_t stream) {
  static std::atomic<int> multiprocessors[64];
  int dev = 0;
  int s = device_index(&dev);
  if (s != NAT_OK) return s;
  int sms = multiprocessors[dev].load(std::memory_order_relaxed);
  if (sms == 0) {
    NAT_CUDA(cudaFuncSetAttribute(few_kernel<WHICH>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem));
    NAT_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    multiprocessors[dev].store(sms, std::memory_order_relaxed);
  }
  return launch_after(few_kernel<WHICH>, dim3((unsigned)min(most_units, (int64_t)sms)), kThreads, kSmem, stream, "experts_few",
                      mw, mx, mx16, f);
}

}  // namespace

int few_product(const Args& a, const Layout& l, Product which) {
  const nat_experts_params& p = a.p;
  const bool fwd = which == kFwd;
  const void* in = fwd ? a.x : a.dy;
  const int k = fwd ? p.n_in : p.n_out;
  const int64_t in_stride = fwd ? p.x_stride : p.y_stride;
  FewArgs f{head(a), tiles(a, l), fwd ? p.n_out : p.n_in, (k + BK - 1) / BK, (__nv_bfloat16*)(fwd ? a.y : a.dx),
            fwd ? p.y_stride : p.x_stride};
  CUtensorMap mw, mx, mx16;
  int s;
  if ((s = map_weights(&mw, p, a.w, fwd ? BM : BK)) != NAT_OK) return s;
  if ((s = map_rows(&mx, in, k, a.cap, in_stride, kFewRows)) != NAT_OK) return s;
  if ((s = map_rows(&mx16, in, k, a.cap, in_stride, kPiece)) != NAT_OK) return s;
  const int64_t units = l.most_tiles * ((f.n_cols + BM - 1) / BM);
  return fwd ? launch<kFwd>(mw, mx, mx16, f, units, a.stream) : launch<kDx>(mw, mx, mx16, f, units, a.stream);
}

}  // namespace experts
}  // namespace nat
