// Product of E4M3 operands with a power-of-two scale per block of 128 along k, on the tensor cores' own block scaling:
//
//   y[m, n] = act( sum_b 2^(ea[m, b] + ew[n / 128, b]) sum_{k in block b} Aq(m, k) Wq(n, k) + bias[n] )
//
// dense, or over rows sorted by expert with a weight matrix per expert (rows seg_start[e] .. seg_start[e + 1] use matrix e; an
// expert's tiles begin at its first row, and what a tile's last rows hold of the next expert is never stored).
//
// tcgen05.mma kind::mxf8f6f4 multiplies each 32 values of k by one scale a row of A and one a row of W, read from tensor memory as
// the byte e + 127 that the scales are held in.  A word of tensor memory has four such bytes, and an instruction says which one it
// means: so a word is the scales of four slabs of 128 values, and the four instructions of a slab use the same byte.  Scales
// cost one copy of 512 bytes a 128 rows and four slabs.  (Scaling the partial sums of every slab in registers instead would read the
// accumulators once a slab.)
//
// Persistent, one CTA per SM, tiles of 128 rows and 64, 128 or 192 columns (two accumulators of 192 leave tensor memory for
// the scales; two of 256 would not):
//   warp 0      : TMA producer (one lane)
//   warp 1      : tensor-memory allocation, copies of scales to tensor memory, MMA issue (one lane)
//   warp 2      : scales from global to shared memory, in the order in which tensor memory takes them
//   warps 3..10 : epilogue, as in gemm_tc.cu
// Every wait is bounded as in gemm_tc.cu.
#include <cuda.h>

#include "common.cuh"
#include "kernels.h"
#include "tc_epilogue.cuh"
#include "tc_ptx.cuh"

namespace bsr {
namespace tcb {
using namespace tc;

constexpr int BM = 128, BK = 128, UMMA_K = 32;             // a slab is a block of scales: 128 bytes of every row
constexpr int A_BYTES = BM * BK;
constexpr int RING_BYTES = 168 * 1024;
constexpr int stages_for(int bn) { return RING_BYTES / (A_BYTES + bn * BK) < 8 ? RING_BYTES / (A_BYTES + bn * BK) : 8; }
constexpr int SF_STAGES = 4, SF_BYTES = 3 * 512;           // words of 128 rows of A, of up to 256 rows of W
constexpr int EPI_WARPS = 8, STAGING_BYTES = 32 * 128;
constexpr int THREADS = 96 + EPI_WARPS * 32;
constexpr int MAX_E = 1024;
constexpr int SMEM_BYTES = RING_BYTES + EPI_WARPS * STAGING_BYTES + SF_STAGES * SF_BYTES + 1024;
constexpr uint32_t TMEM_COLS = 512, SF_COL = 384;          // four columns of A's scales and eight of W's per stage, 16 apart

// D = f32, A = W = E4M3 (format code 0), both along k, scales of type E8M0; sf is the byte of the scale words.
__host__ __device__ constexpr uint32_t make_idesc_scaled(int m, int n) {
  return ((uint32_t)(n >> 3) << 17) | (1u << 23) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ uint32_t sf_id(uint32_t byte) { return byte << 4 | byte << 29; }
__device__ __forceinline__ void umma_scaled(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
      : "memory");
}
// 32 rows of 16 bytes to four columns of tensor memory, the same in each of its four lane quarters.
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
// Shared-memory descriptor without swizzle: rows of 16 bytes, groups of eight rows 128 bytes apart.
__device__ __forceinline__ uint64_t make_desc_scales(uint32_t saddr) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
}

struct Problem {
  int M, N, K;                       // M: rows of A in all
  int tiles_n, experts;
  const int* seg_start;              // null: dense
  const uint32_t* a_scale;           // [M][groups] words
  const uint32_t* w_scale;           // [experts][ceil(N / 128)][groups]
};

// One tile.  r0 .. r1 - 1 are the rows that it stores.
struct Tile { int r0, r1, nt, e; };
__device__ __forceinline__ Tile decode_tile(int w, const Problem& p, const int* tile_start, const int* seg) {
  Tile t;
  const int mt = w / p.tiles_n;
  t.nt = w - mt * p.tiles_n;
  if (p.seg_start == nullptr) {
    t.e = 0;
    t.r0 = mt * BM;
    t.r1 = min(p.M, t.r0 + BM);
  } else {
    int lo = 0, hi = p.experts;      // the last expert whose first tile is not behind mt
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (tile_start[mid] <= mt) lo = mid; else hi = mid;
    }
    t.e = lo;
    t.r0 = seg[lo] + (mt - tile_start[lo]) * BM;
    t.r1 = min(seg[lo + 1], t.r0 + BM);
  }
  return t;
}

template <int BN>
__global__ void __launch_bounds__(THREADS, 1)
gemm_block128_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_a32, const __grid_constant__ CUtensorMap map_w,
                     bf16* __restrict__ C, Problem p, Epi ep, int* status) {
  constexpr int W_BYTES = BN * BK, STAGE_BYTES = A_BYTES + W_BYTES, STAGES = stages_for(BN), HALF_CHUNKS = BN / 64;
  extern __shared__ unsigned char smem_dyn[];
  __shared__ __align__(8) unsigned long long bar_mem[2 * STAGES + 2 * SF_STAGES + 4];
  __shared__ int tile_start[MAX_E + 1], seg[MAX_E + 1];
  __shared__ int warp_total[THREADS / 32];
  __shared__ uint32_t tmem_base_slot;
  __shared__ int abort_flag;
  const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  const uint32_t staging0 = base + STAGES * STAGE_BYTES, sf0 = staging0 + EPI_WARPS * STAGING_BYTES;
  const uint32_t bars = smem_u32(bar_mem);
  auto full_bar = [&](int s) { return bars + 8u * s; };
  auto empty_bar = [&](int s) { return bars + 8u * (STAGES + s); };
  auto sfull_bar = [&](int s) { return bars + 8u * (2 * STAGES + s); };
  auto sempty_bar = [&](int s) { return bars + 8u * (2 * STAGES + SF_STAGES + s); };
  auto tfull_bar = [&](int b) { return bars + 8u * (2 * STAGES + 2 * SF_STAGES + b); };
  auto tempty_bar = [&](int b) { return bars + 8u * (2 * STAGES + 2 * SF_STAGES + 2 + b); };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int total_kb = (p.K + BK - 1) / BK, groups = (total_kb + 3) / 4;

  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int s = 0; s < STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int s = 0; s < SF_STAGES; ++s) { mbar_init(sfull_bar(s), 1); mbar_init(sempty_bar(s), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(tfull_bar(b), 1); mbar_init(tempty_bar(b), EPI_WARPS); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_map(&map_a);
    prefetch_map(&map_a32);
    prefetch_map(&map_w);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(&tmem_base_slot), TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = tmem_base_slot;
  if (ep.release) release_dependents();
  await_inputs();
  volatile int* abortp = &abort_flag;

  // first tile of every expert: a scan over their row counts (segments are cut to the rows there are, and one that reaches into a later
  // one to what is before that, so that no row has two)
  int tiles_m = (p.M + BM - 1) / BM;
  if (p.seg_start != nullptr) {
    for (int i = threadIdx.x; i <= p.experts; i += THREADS) seg[i] = min(max(p.seg_start[i], 0), p.M);
    __syncthreads();
    int falls = 0;
    for (int i = threadIdx.x; i < p.experts; i += THREADS) falls |= seg[i + 1] < seg[i];
    if (__syncthreads_or(falls)) {
      if (threadIdx.x == 0)
        for (int i = p.experts - 1; i >= 0; --i) seg[i] = min(seg[i], seg[i + 1]);
      __syncthreads();
    }
    int below = 0;
    for (int e0 = 0; e0 < p.experts; e0 += THREADS) {
      const int e = e0 + threadIdx.x;
      const int n = e < p.experts ? (seg[e + 1] - seg[e] + BM - 1) / BM : 0;
      int scan = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, scan, o);
        if (lane >= o) scan += v;
      }
      if (lane == 31) warp_total[warp] = scan;
      __syncthreads();
      int prior = below;
      for (int w = 0; w < THREADS / 32; ++w) {
        const int v = warp_total[w];
        if (w < warp) prior += v;
        below += v;
      }
      if (e < p.experts) tile_start[e] = prior + scan - n;
      __syncthreads();
    }
    tiles_m = below;
  }
  const int work_items = tiles_m * p.tiles_n;

  if (warp == 0) {
    // ------------------------------- TMA producer -------------------------------
    if (lane == 0) {
      int stage = 0, armed = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int w = blockIdx.x; w < work_items && ok; w += gridDim.x) {
        const Tile t = decode_tile(w, p, tile_start, seg);
        // a tile of few rows takes those alone, 32 at a time; what the ring holds below them enters rows that nobody reads
        const int boxes = (t.r1 - t.r0 + 31) / 32;
        const uint32_t bytes = (uint32_t)(boxes * 32 * BK + W_BYTES);
        for (int kb = 0; kb < total_kb; ++kb) {
          if (!mbar_wait(empty_bar(stage), phase ^ 1u, abortp)) { ok = false; break; }
          mbar_expect_tx(full_bar(stage), bytes);
          const uint32_t sa = base + stage * STAGE_BYTES;
          if (boxes == 4) tma_load_2d(sa, &map_a, full_bar(stage), kb * BK, t.r0);
          else
            for (int j = 0; j < boxes; ++j) tma_load_2d(sa + j * 32 * BK, &map_a32, full_bar(stage), kb * BK, t.r0 + j * 32);
          tma_load_2d(sa + A_BYTES, &map_w, full_bar(stage), kb * BK, t.e * p.N + t.nt * BN);
          ++armed;
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        }
      }
      if (!ok && armed > 0) {
        unsigned long long t0 = global_ns();       // copies already issued still land in shared memory
        while (global_ns() - t0 < 1000000ull) {}
      }
    }
  } else if (warp == 1) {
    // ------------------------------- MMA issuer ---------------------------------
    if (lane == 0) {
      constexpr uint32_t idesc0 = make_idesc_scaled(BM, BN), KSTEP = UMMA_K >> 4;
      const uint64_t desc_a0 = make_desc(base, 16, 1024), desc_w0 = make_desc(base + A_BYTES, 16, 1024), desc_s0 = make_desc_scales(sf0);
      int stage = 0, sf = 0, local = 0;
      uint32_t phase = 0, sphase = 0;
      bool ok = true;
      for (int w = blockIdx.x; w < work_items && ok; w += gridDim.x, ++local) {
        const int buf = local & 1;
        if (!mbar_wait(tempty_bar(buf), ((local >> 1) & 1) ^ 1u, abortp)) { ok = false; break; }
        tc_fence_after();
        const uint32_t d_tmem = tmem_base + buf * BN;
        for (int kb = 0; kb < total_kb; ++kb) {
          const uint32_t sfa = tmem_base + SF_COL + sf * 16, sfb = sfa + 4;
          if ((kb & 3) == 0) {
            if (!mbar_wait(sfull_bar(sf), sphase, abortp)) { ok = false; break; }
            tc_fence_after();
            const uint64_t ds = desc_s0 + (uint64_t)((sf * SF_BYTES) >> 4);
            copy_scales(sfa, ds);
            copy_scales(sfb, ds + (512 >> 4));
            if (BN > 128) copy_scales(sfb + 4, ds + (1024 >> 4));
          }
          if (!mbar_wait(full_bar(stage), phase, abortp)) { ok = false; break; }
          tc_fence_after();
          const uint64_t off = (uint64_t)((stage * STAGE_BYTES) >> 4);
          const uint32_t idesc = idesc0 | sf_id(kb & 3);
#pragma unroll
          for (int k = 0; k < BK / UMMA_K; ++k)
            umma_scaled(d_tmem, desc_a0 + off + (uint64_t)(k * KSTEP), desc_w0 + off + (uint64_t)(k * KSTEP), idesc, sfa, sfb, (kb > 0 || k > 0) ? 1u : 0u);
          umma_commit(empty_bar(stage));
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
          if ((kb & 3) == 3 || kb == total_kb - 1) {
            umma_commit(sempty_bar(sf));
            if (++sf == SF_STAGES) { sf = 0; sphase ^= 1u; }
          }
        }
        if (ok) umma_commit(tfull_bar(buf));
      }
    }
  } else if (warp == 2) {
    // ------------------------------- scales --------------------------------------
    // Row l of a copy's 32 holds the words of rows l, l + 32, l + 64 and l + 96.  A word of the next group is fetched while this
    // one's stage is waited for.
    int sf = 0;
    uint32_t sphase = 0;
    const int nblocks = (p.N + 127) / 128;
    bool ok = true;
    for (int w = blockIdx.x; w < work_items && ok; w += gridDim.x) {
      const Tile t = decode_tile(w, p, tile_start, seg);
      const uint32_t* ws = p.w_scale + (size_t)t.e * nblocks * groups;
      uint4 a, b[2];
      auto fetch = [&](int g) {
        uint32_t x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = __ldg(p.a_scale + (size_t)min(t.r0 + j * 32 + lane, p.M - 1) * groups + g);
        a = make_uint4(x[0], x[1], x[2], x[3]);
#pragma unroll
        for (int h = 0; h < (BN > 128 ? 2 : 1); ++h) {
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] = __ldg(ws + (size_t)min((t.nt * BN + h * 128 + j * 32) >> 7, nblocks - 1) * groups + g);
          b[h] = make_uint4(x[0], x[1], x[2], x[3]);
        }
      };
      fetch(0);
      for (int g = 0; g < groups; ++g) {
        ok = __all_sync(0xffffffffu, mbar_wait(sempty_bar(sf), sphase ^ 1u, abortp));
        if (!ok) break;
        unsigned char* at = smem_dyn + (sf0 - smem_u32(smem_dyn)) + sf * SF_BYTES + lane * 16;
        *reinterpret_cast<uint4*>(at) = a;
        *reinterpret_cast<uint4*>(at + 512) = b[0];
        if (BN > 128) *reinterpret_cast<uint4*>(at + 1024) = b[1];
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(sfull_bar(sf));
        if (++sf == SF_STAGES) { sf = 0; sphase ^= 1u; }
        if (g + 1 < groups) fetch(g + 1);
      }
    }
  } else {
    // ------------------------------- epilogue -----------------------------------
    const int ew = warp - 3, quarter = warp & 3, chalf = ew >> 2;     // (a warp reads the lanes of tensor memory that its number names)
    unsigned char* st = smem_dyn + (staging0 - smem_u32(smem_dyn)) + ew * STAGING_BYTES;
    int local = 0;
    for (int w = blockIdx.x; w < work_items; w += gridDim.x, ++local) {
      const Tile t = decode_tile(w, p, tile_start, seg);
      const int buf = local & 1;
      auto ready = [&]() {
        const bool r = __all_sync(0xffffffffu, mbar_wait(tfull_bar(buf), (local >> 1) & 1, abortp));
        tc_fence_after();
        return r;
      };
      if (!epilogue_tile<bf16, false, true>(ready, ep, t.e * p.N, C, t.r1, p.N, t.r0 + quarter * 32, t.nt * BN + chalf * HALF_CHUNKS * 32, HALF_CHUNKS,
                                            tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * BN + chalf * HALF_CHUNKS * 32), st, lane))
        break;
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(tempty_bar(buf));
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, TMEM_COLS);
  }
  if (threadIdx.x == 0 && abort_flag && status != nullptr) atomicOr(status, STATUS_TIMEOUT);
}

template <int BN>
static int launch(const Ctx& c, const CUtensorMap& ma, const CUtensorMap& ma32, const CUtensorMap& mw, void* C, const Problem& p, const Epi& ep, long tiles) {
  auto kern = gemm_block128_kernel<BN>;
  static SmemLimit lim;
  if (!ensure_smem(lim, kern, SMEM_BYTES)) return -3;
  const int sms = c.sm_count > 0 ? c.sm_count : B200_SMS, grid = (int)(tiles < sms ? tiles : sms);
  Epi epi = ep;
  epi.release = 2 * grid <= sms;
  note_launch(1);
  launch_k(kern, grid, THREADS, SMEM_BYTES, c.stream, ma, ma32, mw, (bf16*)C, p, epi, c.status);
  return 0;
}

}  // namespace tcb

// y [m, n] bf16 = epilogue(A W^T); see kernels.h.
int gemm_block128(const Ctx& c, const void* Aq, const void* a_scale, const void* Wq, const void* w_scale, const int* seg_start, int experts, void* C, int m, int n, int k,
                  const GemmEpilogue& e) {
  using namespace tcb;
  const int sms = c.sm_count > 0 ? c.sm_count : B200_SMS;
  const long tiles_m = seg_start != nullptr ? ceil_div(m, BM) + (long)(experts < m ? experts : m) - 1 : ceil_div(m, BM);      // at most
  const int bn = tiles_m * ceil_div(n, 64) <= sms ? 64 : tiles_m * ceil_div(n, 128) <= sms ? 128 : 192;
  CUtensorMap ma, ma32, mw;
  if (!make_map_u8(&ma, Aq, (uint64_t)k, (uint64_t)m, (uint64_t)k, BM) || !make_map_u8(&ma32, Aq, (uint64_t)k, (uint64_t)m, (uint64_t)k, 32) ||
      !make_map_u8(&mw, Wq, (uint64_t)k, (uint64_t)experts * n, (uint64_t)k, bn))
    return -2;
  Problem p;
  p.M = m; p.N = n; p.K = k; p.tiles_n = ceil_div(n, bn); p.experts = experts; p.seg_start = seg_start;
  p.a_scale = (const uint32_t*)a_scale; p.w_scale = (const uint32_t*)w_scale;
  Epi ep;
  ep.bias = e.bias; ep.act = e.act; ep.aux_out = e.aux_out; ep.aux_in = e.aux_in;
  const long tiles = tiles_m * p.tiles_n;
  return bn == 64 ? launch<64>(c, ma, ma32, mw, C, p, ep, tiles) : bn == 128 ? launch<128>(c, ma, ma32, mw, C, p, ep, tiles) : launch<192>(c, ma, ma32, mw, C, p, ep, tiles);
}

}  // namespace bsr
