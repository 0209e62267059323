// Product of E4M3 operands with a power-of-two scale per block of 128 along k, on the tensor cores' own block scaling:
//
//   y[m, n] = act( sum_b 2^(ea[m, b] + ew[n / 128, b]) sum_{k in block b} Aq(m, k) Wq(n, k) + bias[n] )
//
// dense, or over rows sorted by expert with a weight matrix per expert (rows seg_start[e] .. seg_start[e + 1] use matrix e; an
// expert's tiles begin at its first row, and what a tile's last rows hold of the next expert is never stored).  Over
// sorted rows a row's sums do not depend on the others: k is never cut there, as it is for a dense product of few rows.
//
// tcgen05.mma kind::mxf8f6f4 multiplies each 32 values of k by one scale a row of A and one a row of W, read from tensor memory as
// the byte e + 127 that the scales are held in.  A word of tensor memory has four such bytes, and an instruction says which one it
// means: so a word is the scales of four slabs of 128 values, and the four instructions of a slab use the same byte.  Scales
// cost one copy of 512 bytes a 128 rows and four slabs.  (Scaling the partial sums of every slab in registers instead would read the
// accumulators once a slab.)
//
// Three kernels:
//   gemm_block128_kernel        persistent, one CTA a tile of 128 rows and 64, 128 or 192 columns (two accumulators of 192 leave tensor memory
//                               for the scales; two of 256 would not)
//   gemm_block128_pair_kernel   persistent, two CTAs (cta_group::2) a tile of 256 rows and up to 240 columns: long k, many rows
//   gemm_block128_small_kernel  a tile's k over the CTAs of a cluster: few tiles
// What bounds them: the tensor pipe where k is long (8192 x 4096 x 7168: 177 us, 2.72 PFLOP/s; under the power limit 216 us); at k = 768 and below what operand
// loads, output stores and the tensor core's reads share inside an SM (25216 x 2304 x 768 on single CTAs 53.7 us, without stores 38.2, without an
// epilogue 36.9; on pairs 51.5, 42.7 and 39.9).  A warp waits for a whole tile's sums: k is limited so that they are there long before it gives up.
// The persistent kernels' warps:
//   warp 0      : TMA producer (one lane)
//   warp 1      : tensor-memory allocation, copies of scales to tensor memory, MMA issue (one lane)
//   warp 2      : scales from global to shared memory, in the order in which tensor memory takes them
//   warps 3..14 : epilogue, three warps per TMEM lane quarter
// Every wait is bounded as in gemm_tc.cu.
#include <cuda.h>

#include <type_traits>

#include "common.cuh"
#include "kernels.h"
#include "tc_epilogue.cuh"
#include "tc_ptx.cuh"
#include "tc_pair.cuh"

namespace bsr {
namespace tcb {
using namespace tc;

constexpr int BM = 128, BK = 128, UMMA_K = 32;             // a slab is a block of scales: 128 bytes of every row
constexpr int A_BYTES = BM * BK;
constexpr int SF_BYTES = 3 * 512;                          // words of 128 rows of A, of up to 256 rows of W
constexpr int EPI_WARPS = 12, EPI_SHARE = EPI_WARPS / 4;   // warps that share a quarter's chunks of columns
// Scales wait in SF_STAGES stages of shared memory: their way there is long beside a group of few slabs.
constexpr int SF_STAGES = 4;
constexpr int STAGING_BYTES = 4096;                        // a warp's 32 rows x 64 columns of bf16
constexpr int THREADS = 96 + EPI_WARPS * 32;
constexpr int MAX_E = 1024;
constexpr uint32_t TMEM_COLS = 512;

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

// One lane of a converged warp, the same one every time.  What it issues to the tensor cores takes its operands from uniform registers only
// where the compiler knows that a single lane runs: behind a comparison of the lane's number an MMA took 180 clocks to issue (whatever
// its width), behind this none that shows.
__device__ __forceinline__ bool elected() {
  uint32_t is;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
  return is != 0;
}

// Whether a phase is over, without waiting.
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// The whole warp waits; false where any lane gave up.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abortp) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, abortp)); }

struct Problem {
  int M, N, K;                       // M: rows of A in all
  int tiles_n, experts;
  const int* seg_start;              // null: dense
  const uint32_t* a_scale;           // [M][groups] words
  const uint32_t* w_scale;           // [experts][ceil(N / 128)][groups]
};

// What one tile covers: rows r0 .. r1 - 1 of expert e, columns from n0.
struct Tile { int r0, r1, n0, e; };
constexpr int LISTED = 32;
struct Tables {
  int tile_start[MAX_E + 1], seg[MAX_E + 1];
  int warp_total[THREADS / 32];
  Tile list[LISTED];                 // this worker's first tiles
};
__device__ __forceinline__ Tile find_tile(int w, const Problem& p, int rows, int width, const Tables& tab) {
  Tile t;
  const int mt = w / p.tiles_n;
  t.n0 = (w - mt * p.tiles_n) * width;
  if (p.seg_start == nullptr) {
    t.e = 0;
    t.r0 = mt * rows;
    t.r1 = min(p.M, t.r0 + rows);
  } else {
    int lo = 0, hi = p.experts;      // the last expert whose first tile is not behind mt
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (tab.tile_start[mid] <= mt) lo = mid; else hi = mid;
    }
    t.e = lo;
    t.r0 = tab.seg[lo] + (mt - tab.tile_start[lo]) * rows;
    t.r1 = min(tab.seg[lo + 1], t.r0 + rows);
  }
  return t;
}
// The tiles of one worker, ascending, columns fastest.  Four roles walk them: the first ones come from a list that the CTA's threads make
// side by side.
struct Walk {
  int i, w, workers, items;
  __device__ __forceinline__ Walk(int worker, int workers_, int items_) : i(0), w(worker), workers(workers_), items(items_) {}
  __device__ __forceinline__ bool next(Tile& t, const Problem& p, int rows, int width, const Tables& tab) {
    if (w >= items) return false;
    t = i < LISTED ? tab.list[i] : find_tile(w, p, rows, width, tab);
    ++i;
    w += workers;
    return true;
  }
};
// All threads: segments, the first tile of every expert (tiles of `rows` rows) and the worker's list to shared memory; returns the number
// of tiles.  Segments are cut to the rows there are, and one that reaches into a later one to what is before that, so that no row has two.
__device__ __forceinline__ int make_tables(const Problem& p, int rows, int width, int worker, int workers, Tables& tab) {
  int tiles_m = (p.M + rows - 1) / rows;
  if (p.seg_start != nullptr) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int i = threadIdx.x; i <= p.experts; i += THREADS) tab.seg[i] = min(max(p.seg_start[i], 0), p.M);
    __syncthreads();
    int falls = 0;
    for (int i = threadIdx.x; i < p.experts; i += THREADS) falls |= tab.seg[i + 1] < tab.seg[i];
    if (__syncthreads_or(falls)) {
      if (threadIdx.x == 0)
        for (int i = p.experts - 1; i >= 0; --i) tab.seg[i] = min(tab.seg[i], tab.seg[i + 1]);
      __syncthreads();
    }
    int below = 0;
    for (int e0 = 0; e0 < p.experts; e0 += THREADS) {
      const int e = e0 + threadIdx.x;
      const int n = e < p.experts ? (tab.seg[e + 1] - tab.seg[e] + rows - 1) / rows : 0;
      int scan = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, scan, o);
        if (lane >= o) scan += v;
      }
      if (lane == 31) tab.warp_total[warp] = scan;
      __syncthreads();
      int prior = lane < THREADS / 32 ? tab.warp_total[lane] : 0;
      const int sum = warp_sum_int(prior);
      prior = below + warp_sum_int(lane < warp ? prior : 0);
      below += sum;
      if (e < p.experts) tab.tile_start[e] = prior + scan - n;
      __syncthreads();
    }
    tiles_m = below;
  }
  const int items = tiles_m * p.tiles_n, mine = worker + (int)threadIdx.x * workers;
  if (threadIdx.x < LISTED && mine < items) tab.list[threadIdx.x] = find_tile(mine, p, rows, width, tab);
  __syncthreads();
  return items;
}

// Scales of one group of four slabs, as this lane stores them: row l of a copy's 32 holds the words of rows l, l + 32, l + 64, l + 96.
struct Scales {
  uint4 a, b[2];
  __device__ __forceinline__ void fetch(const Problem& p, const Tile& t, int row0, int g, int groups, int nblocks, bool wide) {
    const int lane = threadIdx.x & 31;
    uint32_t x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = __ldg(p.a_scale + (size_t)min(row0 + j * 32 + lane, p.M - 1) * groups + g);
    a = make_uint4(x[0], x[1], x[2], x[3]);
    const uint32_t* ws = p.w_scale + (size_t)t.e * nblocks * groups;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (h == 1 && !wide) break;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = __ldg(ws + (size_t)min((t.n0 + h * 128 + j * 32 + lane) >> 7, nblocks - 1) * groups + g);
      b[h] = make_uint4(x[0], x[1], x[2], x[3]);
    }
  }
  __device__ __forceinline__ void store(unsigned char* stage, bool wide) const {
    unsigned char* at = stage + (threadIdx.x & 31) * 16;
    *reinterpret_cast<uint4*>(at) = a;
    *reinterpret_cast<uint4*>(at + 512) = b[0];
    if (wide) *reinterpret_cast<uint4*>(at + 1024) = b[1];
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
};

// ---- epilogue ----------------------------------------------------------------------------------------------------------
// A lane has a row of accumulators.  Chunks of 32 rows x 64 columns leave through a swizzled buffer in shared memory and a bulk
// tensor store, which needs one lane (stores of the lanes' own rows, 32 bytes each, keep the load-store unit busy for 64 clocks per
// 32 columns).
//
// GELU(z) = max(z, 0) - |z| Phi(-|z|) and GELU'(z) = Phi(z) + z phi(z), with Phi(-t) = exp(-t^2 / 2) R(t).  R falls from 1/2 and goes as
// 1 / t: it is c0 + c1 u + .. + c5 u^5 in u = 1 / (1 + 0.36015 t), fitted to erfcx in double precision by relative error, 1.1e-5 over
// 0 <= t <= 13.3, beyond which the exponential is zero: a 350th of the rounding to bf16, and of every value, where a polynomial
// for Phi itself is off by a fixed amount.  (Without c0, u times as many terms is one operation more for 4.0e-6: 25216 x 1536 x 384 45.0 -> 46.2 us.)
// s = -min(|z|, 16): beyond, the exponential is zero, and so are its products with s, for infinities too.
// Two values at a time, packed wherever an instruction takes pairs (618 -> 541 instructions for 32 rows x 32 columns with the rest: 25216 x 1536 x 384 41.9 -> 37.5 us).
__device__ __forceinline__ void phi_tail2(uint64_t z, float z0, float z1, uint64_t& s, uint64_t& p, float& e0, float& e1) {
  float h0, h1, d0, d1, u0, u1;
  unpack2(mul2(mul2(z, z), dup2(-0.72134752044448170f)), h0, h1);      // exp(-z^2 / 2) = 2^(-log2(e) / 2 z^2)
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(h0));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(h1));
  s = pack2(fmaxf(-fabsf(z0), -16.f), fmaxf(-fabsf(z1), -16.f));
  unpack2(fma2(s, dup2(-0.3601517975330353f), dup2(1.0f)), d0, d1);
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(u0) : "f"(d0));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(u1) : "f"(d1));
  const uint64_t u = pack2(u0, u1);
  uint64_t r = dup2(-0.099203065f);
  r = fma2(r, u, dup2(0.2558196f));
  r = fma2(r, u, dup2(0.03368386f));
  r = fma2(r, u, dup2(0.16946077f));
  r = fma2(r, u, dup2(0.1400296f));
  r = fma2(r, u, dup2(0.00020378547f));
  p = mul2(r, pack2(e0, e1));
}
__device__ __forceinline__ void gelu2(float& z0, float& z1) {
  uint64_t s, p;
  float e0, e1;
  phi_tail2(pack2(z0, z1), z0, z1, s, p, e0, e1);
  unpack2(fma2(s, p, pack2(fmaxf(z0, 0.f), fmaxf(z1, 0.f))), z0, z1);
}
__device__ __forceinline__ void gelu_grad_mul(float& g0, float& g1, float z0, float z1) {
  uint64_t s, p;
  float e0, e1, p0, p1, s0, s1;
  phi_tail2(pack2(z0, z1), z0, z1, s, p, e0, e1);
  unpack2(p, p0, p1);
  unpack2(mul2(s, dup2(0.39894228040143268f)), s0, s1);
  const uint64_t phi = pack2(z0 < 0.f ? p0 : 1.f - p0, z1 < 0.f ? p1 : 1.f - p1);
  unpack2(mul2(pack2(g0, g1), fma2(pack2(copysignf(s0, z0), copysignf(s1, z1)), pack2(e0, e1), phi)), g0, g1);
}

struct Out {
  bf16* y;
  bf16* z;                           // the pre-activation, written (act 1, optional) or read (act 2)
  const float* bias;                 // [experts][N], optional
  bool release;                      // the next kernel may be scheduled while this one runs
};

__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, uint32_t src, int c0, int c1) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(src), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void stores_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void stores_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }

// A warp's staging buffer and what goes through it: 32 rows x 64 columns (one buffer), or 32 x 32 (two: the output's and the
// pre-activation's, on its way out or in).  16-byte units are swizzled as the tensor maps say.
template <int CH>
struct Exit {
  unsigned char* st;
  int N;
  static constexpr int UNITS = CH / 8;
  __device__ __forceinline__ static uint32_t slot(int r, int u) { return (uint32_t)(r * CH * 2 + ((CH == 64 ? u ^ (r & 7) : u ^ ((r >> 1) & 3)) << 4)); }

  // 32 columns of this lane's row, from unit u0 of buffer b on.
  __device__ __forceinline__ void stage(const float* v, int b, int u0) const {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[u * 8 + 2 * j], v[u * 8 + 2 * j + 1]);
        w[j] = *reinterpret_cast<const uint32_t*>(&h);
      }
      *reinterpret_cast<uint4*>(st + b * 2048 + slot(threadIdx.x & 31, u0 + u)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  // The staged rows row0 .. row0 + 31 of CH columns from col (cols of them wanted) on their way: buffer 0 to out, and where there is
  // out1 too, buffer 1 to that.  full: no row or column has to be left out that the tensor maps do not leave out by themselves.
  __device__ __forceinline__ void send(const CUtensorMap* map, bf16* out, const CUtensorMap* map1, bf16* out1, int row0, int r1, int col, int cols, bool full) const {
    const int lane = threadIdx.x & 31;
    if (full) {
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (elected()) {
        tma_store_2d(map, smem_u32(st), col, row0);
        if (out1 != nullptr) tma_store_2d(map1, smem_u32(st + 2048), col, row0);
        stores_commit();
      }
    } else {
      __syncwarp();
#pragma unroll
      for (int i = 0; i < UNITS; ++i) {
        const int r = i * (32 / UNITS) + lane / UNITS, u = lane % UNITS;
        if (row0 + r < r1 && u * 8 < cols) {
          const size_t at = (size_t)(row0 + r) * N + col + u * 8;
          *reinterpret_cast<uint4*>(out + at) = *reinterpret_cast<const uint4*>(st + slot(r, u));
          if (out1 != nullptr) *reinterpret_cast<uint4*>(out1 + at) = *reinterpret_cast<const uint4*>(st + 2048 + slot(r, u));
        }
      }
    }
  }
  // The last store has read its buffers.
  __device__ __forceinline__ void free_buffers() const {
    if (elected()) stores_read();
    __syncwarp();
  }
  // The stored pre-activation of a chunk on its way to the second buffer, and this lane's row of it once it is there.
  __device__ __forceinline__ void ask(const bf16* z, int row0, int r1, int col, int cols) const {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      const int r = i * (32 / UNITS) + lane / UNITS, u = lane % UNITS;
      const bool in = row0 + r < r1 && u * 8 < cols;
      copy16_async(st + 2048 + slot(r, u), in ? z + (size_t)(row0 + r) * N + col + u * 8 : z, in ? 16 : 0);
    }
    copies_commit();
  }
  __device__ __forceinline__ void got(uint4* w) const {
    copies_wait<0>();
    __syncwarp();
#pragma unroll
    for (int u = 0; u < UNITS; ++u) w[u] = *reinterpret_cast<const uint4*>(st + 2048 + slot(threadIdx.x & 31, u));
    __syncwarp();
  }
};

__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
// 32 columns of this lane's row of accumulators, with the bias.
__device__ __forceinline__ void load_sums(uint32_t taddr, const float* sbias, bool bias, float* v) {
  uint32_t r[32];
  tmem_ld32(taddr, r);
  tmem_ld_wait();
#pragma unroll
  for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]);
  if (bias) {
#pragma unroll
    for (int j = 0; j < 32; j += 4) {
      const float4 b = *reinterpret_cast<const float4*>(sbias + j);
      unpack2(add2(pack2(v[j], v[j + 1]), pack2(b.x, b.y)), v[j], v[j + 1]);
      unpack2(add2(pack2(v[j + 2], v[j + 3]), pack2(b.z, b.w)), v[j + 2], v[j + 3]);
    }
  }
}

// An epilogue warp's way through the tiles.  Of each it has every EPI_SHARE-th chunk of CH columns from its `first` on, rows row0 .. row0 + 31
// (those below r1; row0 is t.r0 + row_off), columns n0 .. n0 + width - 1 (those below N).  next(t) gives the tiles; ready(i) waits for tile i's sums, which lie at
// taddr(i); release(i) says that this warp has read them.  What does not depend on the sums -- the bias, the first chunk of the
// pre-activation -- is asked for a tile ahead.  clipped: the tensor maps end where the rows do (no other expert's rows follow).
constexpr int chunk_of(int act) { return act == 0 ? 64 : 32; }
template <int ACT, int BIAS, typename Next, typename Ready, typename Addr, typename Release>
__device__ __forceinline__ void epilogue(Next next, Ready ready, Addr taddr, Release release, const Out& o, const CUtensorMap* map_y, const CUtensorMap* map_z,
                                         const Exit<chunk_of(ACT)>& x, int N, int row_off, int width, int first, float* sbias, bool clipped) {
  constexpr int CH = chunk_of(ACT), STEP = EPI_SHARE * CH, NB = BIAS / 128;
  const int lane = threadIdx.x & 31;
  const bool bias = o.bias != nullptr;
  Tile t, after;
  float ahead[NB];
  auto ask_ahead = [&](const Tile& q) {
    if (bias) {
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int c = first * CH + i * 32 % CH + i * 32 / CH * STEP + lane;
        ahead[i] = c < width && q.n0 + c < N ? __ldg(o.bias + (size_t)q.e * N + q.n0 + c) : 0.f;
      }
    }
  };
  auto any_of = [&](const Tile& q) { return q.r0 + row_off < q.r1 && first * CH < min(width, N - q.n0); };
  auto ask_z = [&](const Tile& q) {
    if (ACT == 2 && any_of(q)) x.ask(o.z, q.r0 + row_off, q.r1, q.n0 + first * CH, min(width, N - q.n0) - first * CH);
  };
  bool more = next(t);
  if (more) {
    ask_ahead(t);
    ask_z(t);
  }
  for (int local = 0; more; ++local) {
    if (bias) {
#pragma unroll
      for (int i = 0; i < NB; ++i) sbias[i * 32 + lane] = ahead[i];
    }
    more = next(after);
    if (more) ask_ahead(after);
    if (!ready(local)) return;
    __syncwarp();
    const uint32_t sums = taddr(local);
    const int row0 = t.r0 + row_off, r1 = t.r1, n0 = t.n0, end = min(n0 + width, N);
    if (any_of(t)) {
      const bool rows_full = clipped || row0 + 32 <= r1;
#pragma unroll 1
      for (int i = 0, c = first * CH; n0 + c < end; ++i, c += STEP) {
        const int col = n0 + c, cols = end - col;                         // cols: what is left of the tile
        const bool full = rows_full && (c + CH <= width || end == N);     // (a tile's last columns leave by themselves)
        const bool last = cols <= STEP;
        float v[32];
        if constexpr (ACT == 0) {
          load_sums(sums + c, sbias + i * CH, bias, v);
          x.free_buffers();
          x.stage(v, 0, 0);
          if (cols > 32) {
            load_sums(sums + c + 32, sbias + i * CH + 32, bias, v);
            x.stage(v, 0, 4);
          }
          if (last) release(local);
          x.send(map_y, o.y, nullptr, nullptr, row0, r1, col, cols, full);
        } else if constexpr (ACT == 1) {
          load_sums(sums + c, sbias + i * CH, bias, v);
          if (last) release(local);
          x.free_buffers();
          if (o.z != nullptr) x.stage(v, 1, 0);
#pragma unroll
          for (int j = 0; j < 32; j += 2) gelu2(v[j], v[j + 1]);
          x.stage(v, 0, 0);
          x.send(map_y, o.y, map_z, o.z, row0, r1, col, cols, full);
        } else {
          uint4 zw[4];
          x.got(zw);
          if (!last) x.ask(o.z, row0, r1, col + STEP, cols - STEP);
          else if (more) ask_z(after);
          load_sums(sums + c, sbias + i * CH, bias, v);
          if (last) release(local);
          const uint32_t w[16] = {zw[0].x, zw[0].y, zw[0].z, zw[0].w, zw[1].x, zw[1].y, zw[1].z, zw[1].w, zw[2].x, zw[2].y, zw[2].z, zw[2].w, zw[3].x, zw[3].y, zw[3].z, zw[3].w};
#pragma unroll
          for (int j = 0; j < 32; j += 2) gelu_grad_mul(v[j], v[j + 1], __uint_as_float(w[j / 2] << 16), __uint_as_float(w[j / 2] & 0xffff0000u));
          x.free_buffers();
          x.stage(v, 0, 0);
          x.send(map_y, o.y, nullptr, nullptr, row0, r1, col, cols, full);
        }
      }
    } else {
      if (more) ask_z(after);
      release(local);
    }
    __syncwarp();                    // (the bias is read before the next tile's replaces it)
    t = after;
  }
  if (elected()) stores_read();      // shared memory stays until the last stores have read it
}

// ---- one CTA a tile ------------------------------------------------------------------------------------------------------
constexpr int RING_BYTES = 160 * 1024;
constexpr int stages_for(int bn) { return RING_BYTES / (A_BYTES + bn * BK) < 8 ? RING_BYTES / (A_BYTES + bn * BK) : 8; }
constexpr int BIAS_BYTES = 64 * 4;   // bias of a warp's columns of a tile: 192 among three
constexpr int SMEM_BYTES = RING_BYTES + EPI_WARPS * (STAGING_BYTES + BIAS_BYTES) + SF_STAGES * SF_BYTES + 1024;
constexpr uint32_t SF_COL = 384;     // four columns of A's scales and eight of W's per stage, 16 apart

template <int BN, int ACT>
__global__ void __launch_bounds__(THREADS, 1)
gemm_block128_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_a32, const __grid_constant__ CUtensorMap map_w,
                     const __grid_constant__ CUtensorMap map_y, const __grid_constant__ CUtensorMap map_z, Problem p, Out out, int* status) {
  constexpr int W_BYTES = BN * BK, STAGE_BYTES = A_BYTES + W_BYTES, STAGES = stages_for(BN);
  extern __shared__ unsigned char smem_dyn[];
  __shared__ __align__(8) unsigned long long bar_mem[2 * STAGES + 2 * SF_STAGES + 4];
  __shared__ __align__(16) Tables tab;
  __shared__ uint32_t tmem_base_slot;
  __shared__ int abort_flag;
  const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  const uint32_t staging0 = base + STAGES * STAGE_BYTES, sf0 = staging0 + EPI_WARPS * STAGING_BYTES, bias0 = sf0 + SF_STAGES * SF_BYTES;
  auto ptr = [&](uint32_t a) { return smem_dyn + (a - smem_u32(smem_dyn)); };
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
    prefetch_map(&map_y);
    prefetch_map(&map_z);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(&tmem_base_slot), TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = tmem_base_slot;
  if (out.release) release_dependents();
  await_inputs();
  volatile int* abortp = &abort_flag;
  Walk walk(blockIdx.x, gridDim.x, make_tables(p, BM, BN, blockIdx.x, gridDim.x, tab));
  Tile t;
  auto next = [&]() { return walk.next(t, p, BM, BN, tab); };

  if (warp == 0) {
    // ------------------------------- TMA producer -------------------------------
    if (elected()) {
      int stage = 0, armed = 0;
      uint32_t phase = 0;
      bool ok = true;
      while (ok && next()) {
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
          tma_load_2d(sa + A_BYTES, &map_w, full_bar(stage), kb * BK, t.e * p.N + t.n0);
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
    if (elected()) {
      const uint32_t idesc0 = make_idesc_scaled(BM, BN);
      constexpr uint32_t KSTEP = UMMA_K >> 4;
      const uint64_t desc_a0 = make_desc(base, 16, 1024), desc_w0 = make_desc(base + A_BYTES, 16, 1024), desc_s0 = make_desc_scales(sf0);
      int stage = 0, sf = 0, local = 0;
      uint32_t phase = 0, sphase = 0;
      bool ok = true, here = false;           // here: this slab's operands were seen to be there
      for (; ok && next(); ++local) {
        const int buf = local & 1;
        if (!mbar_wait(tempty_bar(buf), ((local >> 1) & 1) ^ 1u, abortp)) break;
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
          if (!here && !mbar_wait(full_bar(stage), phase, abortp)) { ok = false; break; }
          tc_fence_after();
          const int after = stage + 1 == STAGES ? 0 : stage + 1;
          const uint32_t phase_after = after == 0 ? phase ^ 1u : phase;
          here = mbar_test(full_bar(after), phase_after);      // (its answer arrives while this slab's instructions are issued)
          const uint64_t off = (uint64_t)((stage * STAGE_BYTES) >> 4);
          const uint32_t idesc = idesc0 | sf_id(kb & 3);
#pragma unroll
          for (int k = 0; k < BK / UMMA_K; ++k)
            umma_scaled(d_tmem, desc_a0 + off + (uint64_t)(k * KSTEP), desc_w0 + off + (uint64_t)(k * KSTEP), idesc, sfa, sfb, (kb > 0 || k > 0) ? 1u : 0u);
          umma_commit(empty_bar(stage));
          stage = after;
          phase = phase_after;
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
    // (words are fetched two groups ahead, across tiles: a group's come from L2, and there may be one group a tile)
    const int nblocks = (p.N + 127) / 128;
    bool more = next();
    int g = 0, sf = 0;
    uint32_t sphase = 0;
    auto fetch = [&](Scales& s) {
      if (!more) return false;
      s.fetch(p, t, t.r0, g, groups, nblocks, BN > 128);
      if (++g == groups) { g = 0; more = next(); }
      return true;
    };
    auto hand = [&](const Scales& s) {
      if (!warp_wait(sempty_bar(sf), sphase ^ 1u, abortp)) return false;
      s.store(ptr(sf0 + sf * SF_BYTES), BN > 128);
      __syncwarp();
      if (lane == 0) mbar_arrive(sfull_bar(sf));
      if (++sf == SF_STAGES) { sf = 0; sphase ^= 1u; }
      return true;
    };
    Scales s0, s1;
    bool h0 = fetch(s0), h1 = fetch(s1);
    while (h0) {
      if (!hand(s0)) break;
      h0 = fetch(s0);
      if (!h1) break;
      if (!hand(s1)) break;
      h1 = fetch(s1);
    }
  } else {
    // ------------------------------- epilogue -----------------------------------
    const int ew = warp - 3, quarter = warp & 3, first = ew >> 2;    // (a warp reads the lanes of tensor memory that its number names)
    float* sbias = reinterpret_cast<float*>(ptr(bias0 + ew * BIAS_BYTES));
    const Exit<chunk_of(ACT)> way = {ptr(staging0 + ew * STAGING_BYTES), p.N};
    epilogue<ACT, BIAS_BYTES>([&](Tile& q) { return walk.next(q, p, BM, BN, tab); },
                              [&](int i) {
                                const bool r = warp_wait(tfull_bar(i & 1), (i >> 1) & 1, abortp);
                                tc_fence_after();
                                return r;
                              },
                              [&](int i) { return tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)((i & 1) * BN); },
                              [&](int i) {
                                tc_fence_before();
                                __syncwarp();
                                if (lane == 0) mbar_arrive(tempty_bar(i & 1));
                              },
                              out, &map_y, &map_z, way, p.N, quarter * 32, BN, first, sbias, p.seg_start == nullptr);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, TMEM_COLS);
  }
  if (threadIdx.x == 0 && abort_flag && status != nullptr) atomicOr(status, STATUS_TIMEOUT);
}

// ---- two CTAs a tile -------------------------------------------------------------------------------------------------------
// As gemm_tc2.cu: each SM stages its own 128 rows of A and half of the columns of W, 31 KB a slab for 256 x 240 sums where one CTA
// takes 40 KB for 128 x 192.  Both CTAs hold the scales of their own rows and of all columns.  `width` columns a tile, a multiple of 16, is chosen
// for each product: up to 240, so that two accumulators and the scales of two groups fit tensor memory; a group's are copied into the place of those
// before the last once the products that read these are done.  Four, five or six stages: within 3 %.
constexpr int P_WIDTH = 240, P_STAGES = 5, P_BIAS_BYTES = 128 * 4;
constexpr int P_STAGE_BYTES = A_BYTES + P_WIDTH / 2 * BK;
constexpr int P_SMEM_BYTES = P_STAGES * P_STAGE_BYTES + EPI_WARPS * (STAGING_BYTES + P_BIAS_BYTES) + SF_STAGES * SF_BYTES + 1024;
constexpr uint32_t P_SF_COL = 2 * P_WIDTH;
static_assert(P_SF_COL + 16 + 12 <= TMEM_COLS && P_STAGE_BYTES % 1024 == 0, "the scales fit behind the accumulators");

__device__ __forceinline__ void umma_scaled_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void copy_scales_pair(uint32_t taddr, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait_cluster(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}

template <int ACT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1)
gemm_block128_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_a32, const __grid_constant__ CUtensorMap map_w,
                          const __grid_constant__ CUtensorMap map_y, const __grid_constant__ CUtensorMap map_z, Problem p, Out out, int width, int* status) {
  extern __shared__ unsigned char smem_dyn[];
  __shared__ __align__(8) unsigned long long bar_mem[2 * P_STAGES + 2 * SF_STAGES + 4];
  __shared__ __align__(16) Tables tab;
  __shared__ uint32_t tmem_base_slot;
  __shared__ int abort_flag;
  const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  const uint32_t staging0 = base + P_STAGES * P_STAGE_BYTES, sf0 = staging0 + EPI_WARPS * STAGING_BYTES, bias0 = sf0 + SF_STAGES * SF_BYTES;
  auto ptr = [&](uint32_t a) { return smem_dyn + (a - smem_u32(smem_dyn)); };
  const uint32_t bars = smem_u32(bar_mem);
  auto full_bar = [&](int s) { return bars + 8u * s; };
  auto empty_bar = [&](int s) { return bars + 8u * (P_STAGES + s); };
  auto sfull_bar = [&](int s) { return bars + 8u * (2 * P_STAGES + s); };
  auto sempty_bar = [&](int s) { return bars + 8u * (2 * P_STAGES + SF_STAGES + s); };
  auto tfull_bar = [&](int b) { return bars + 8u * (2 * P_STAGES + 2 * SF_STAGES + b); };
  auto tempty_bar = [&](int b) { return bars + 8u * (2 * P_STAGES + 2 * SF_STAGES + 2 + b); };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int total_kb = (p.K + BK - 1) / BK, groups = (total_kb + 3) / 4;
  const int rank = (int)cluster_rank();
  const bool leader = rank == 0;

  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int s = 0; s < P_STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int s = 0; s < SF_STAGES; ++s) { mbar_init(sfull_bar(s), 2); mbar_init(sempty_bar(s), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(tfull_bar(b), 1); mbar_init(tempty_bar(b), 2 * EPI_WARPS); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_map(&map_a);
    prefetch_map(&map_a32);
    prefetch_map(&map_w);
    prefetch_map(&map_y);
    prefetch_map(&map_z);
  }
  if (warp == 1) {
    tmem_alloc_pair(smem_u32(&tmem_base_slot), TMEM_COLS);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  cluster_sync_all();                       // barriers of both CTAs exist before anyone signals them
  tc_fence_after();
  const uint32_t tmem_base = tmem_base_slot;
  await_inputs();                           // (fills the SMs: see release_dependents)
  volatile int* abortp = &abort_flag;
  Walk walk(blockIdx.x >> 1, gridDim.x >> 1, make_tables(p, 2 * BM, width, blockIdx.x >> 1, gridDim.x >> 1, tab));
  Tile t;
  auto next = [&]() { return walk.next(t, p, 2 * BM, width, tab); };
  auto rows_of = [&](int r) { return min(max(t.r1 - t.r0 - r * BM, 0), BM); };

  if (warp == 0) {
    // ------------------------------- TMA producer (both CTAs) -------------------------------
    if (elected()) {
      int stage = 0, armed = 0;
      uint32_t phase = 0;
      bool ok = true;
      const int cols = width >> 1;
      while (ok && next()) {
        const int boxes = (rows_of(rank) + 31) / 32, row0 = t.r0 + rank * BM;
        const uint32_t bytes = (uint32_t)(((rows_of(0) + 31) / 32 + (rows_of(1) + 31) / 32) * 32 * BK + width * BK);
        for (int kb = 0; kb < total_kb; ++kb) {
          if (!mbar_wait(empty_bar(stage), phase ^ 1u, abortp)) { ok = false; break; }
          const uint32_t fb = full_bar(stage) & PEER_MASK;      // the leader's barrier collects both CTAs' bytes
          if (leader) mbar_expect_tx(full_bar(stage), bytes);
          const uint32_t sa = base + stage * P_STAGE_BYTES;
          if (boxes == 4) tma_load_2d_pair(sa, &map_a, fb, kb * BK, row0);
          else
            for (int j = 0; j < boxes; ++j) tma_load_2d_pair(sa + j * 32 * BK, &map_a32, fb, kb * BK, row0 + j * 32);
          tma_load_2d_pair(sa + A_BYTES, &map_w, fb, kb * BK, t.e * p.N + t.n0 + rank * cols);
          ++armed;
          if (++stage == P_STAGES) { stage = 0; phase ^= 1u; }
        }
      }
      if (!ok && armed > 0) {
        unsigned long long t0 = global_ns();
        while (global_ns() - t0 < 1000000ull) {}
      }
    }
  } else if (warp == 1) {
    // ------------------------------- MMA issuer (leader CTA only) ---------------------------
    if (leader && elected()) {
      const uint32_t idesc0 = make_idesc_scaled(2 * BM, width);
      constexpr uint32_t KSTEP = UMMA_K >> 4;
      const uint64_t desc_a0 = make_desc(base, 16, 1024), desc_w0 = make_desc(base + A_BYTES, 16, 1024), desc_s0 = make_desc_scales(sf0);
      int stage = 0, sf = 0, local = 0;
      uint32_t phase = 0, sphase = 0;
      bool ok = true, here = false;           // here: this slab's operands were seen to be there
      for (; ok && next(); ++local) {
        const int buf = local & 1;
        if (!mbar_wait(tempty_bar(buf), ((local >> 1) & 1) ^ 1u, abortp)) break;
        tc_fence_after();
        const uint32_t d_tmem = tmem_base + buf * P_WIDTH;
        for (int kb = 0; kb < total_kb; ++kb) {
          const uint32_t sfa = tmem_base + P_SF_COL + (sf & 1) * 16, sfb = sfa + 4;
          if ((kb & 3) == 0) {
          // (the other CTA's scales were written by its own threads: the wait takes part in the cluster's order)
            if (!mbar_wait(sempty_bar(sf ^ 2), sf < 2 ? sphase ^ 1u : sphase, abortp) || !mbar_wait(sfull_bar(sf), sphase, abortp) || !mbar_try_wait_cluster(sfull_bar(sf), sphase)) {
              ok = false;
              break;
            }
            tc_fence_after();
            const uint64_t ds = desc_s0 + (uint64_t)((sf * SF_BYTES) >> 4);
            copy_scales_pair(sfa, ds);
            copy_scales_pair(sfb, ds + (512 >> 4));
            if (width > 128) copy_scales_pair(sfb + 4, ds + (1024 >> 4));
          }
          if (!here && !mbar_wait(full_bar(stage), phase, abortp)) { ok = false; break; }
          tc_fence_after();
          const int after = stage + 1 == P_STAGES ? 0 : stage + 1;
          const uint32_t phase_after = after == 0 ? phase ^ 1u : phase;
          here = mbar_test(full_bar(after), phase_after);      // (its answer arrives while this slab's instructions are issued)
          const uint64_t off = (uint64_t)((stage * P_STAGE_BYTES) >> 4);
          const uint32_t idesc = idesc0 | sf_id(kb & 3);
#pragma unroll
          for (int k = 0; k < BK / UMMA_K; ++k)
            umma_scaled_pair(d_tmem, desc_a0 + off + (uint64_t)(k * KSTEP), desc_w0 + off + (uint64_t)(k * KSTEP), idesc, sfa, sfb, (kb > 0 || k > 0) ? 1u : 0u);
          umma_commit_pair(empty_bar(stage));
          stage = after;
          phase = phase_after;
          if ((kb & 3) == 3 || kb == total_kb - 1) {
            umma_commit_pair(sempty_bar(sf));
            if (++sf == SF_STAGES) { sf = 0; sphase ^= 1u; }
          }
        }
        if (ok) umma_commit_pair(tfull_bar(buf));
      }
    }
  } else if (warp == 2) {
    // ------------------------------- scales (both CTAs) --------------------------------------
    // (words are fetched two groups ahead, across tiles: a group's come from L2, and there may be one group a tile)
    const int nblocks = (p.N + 127) / 128;
    bool more = next();
    int g = 0, sf = 0;
    uint32_t sphase = 0;
    auto fetch = [&](Scales& s) {
      if (!more) return false;
      s.fetch(p, t, t.r0 + rank * BM, g, groups, nblocks, width > 128);
      if (++g == groups) { g = 0; more = next(); }
      return true;
    };
    auto hand = [&](const Scales& s) {
      if (!warp_wait(sempty_bar(sf), sphase ^ 1u, abortp)) return false;
      s.store(ptr(sf0 + sf * SF_BYTES), width > 128);
      __syncwarp();
      if (lane == 0) mbar_arrive_leader(sfull_bar(sf));
      if (++sf == SF_STAGES) { sf = 0; sphase ^= 1u; }
      return true;
    };
    Scales s0, s1;
    bool h0 = fetch(s0), h1 = fetch(s1);
    while (h0) {
      if (!hand(s0)) break;
      h0 = fetch(s0);
      if (!h1) break;
      if (!hand(s1)) break;
      h1 = fetch(s1);
    }
  } else {
    // ------------------------------- epilogue (both CTAs, own rows) --------------------------
    const int ew = warp - 3, quarter = warp & 3, first = ew >> 2;
    float* sbias = reinterpret_cast<float*>(ptr(bias0 + ew * P_BIAS_BYTES));
    const Exit<chunk_of(ACT)> way = {ptr(staging0 + ew * STAGING_BYTES), p.N};
    epilogue<ACT, P_BIAS_BYTES>([&](Tile& q) { return walk.next(q, p, 2 * BM, width, tab); },
                                [&](int i) {
                                  const bool r = warp_wait(tfull_bar(i & 1), (i >> 1) & 1, abortp);
                                  tc_fence_after();
                                  return r;
                                },
                                [&](int i) { return tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)((i & 1) * P_WIDTH); },
                                [&](int i) {
                                  tc_fence_before();
                                  __syncwarp();
                                  if (lane == 0) mbar_arrive_leader_relaxed(tempty_bar(i & 1));
                                },
                                out, &map_y, &map_z, way, p.N, rank * BM + quarter * 32, width, first, sbias, p.seg_start == nullptr);
  }
  tc_fence_before();
  __syncwarp();
  cluster_sync_all();                       // neither CTA leaves while the other may still touch its memory
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem_base, TMEM_COLS);
  }
  if (threadIdx.x == 0 && abort_flag && status != nullptr) atomicOr(status, STATUS_TIMEOUT);
}

// ---- few tiles: a tile's k over a cluster -----------------------------------------------------------------------------------
// What bounds a product of few rows is latency: 16 x 4096 x 4096 is 64 tiles with 32 slabs one after the other.  As in gemm_tc_small.cu
// a tile's k is split over the CTAs of a cluster (in groups of four slabs, whole words of scales), which send each other their partial sums through
// distributed shared memory; each adds up and finishes an equal share of the rows, in the order of k.
constexpr int S_BN = 64, S_STAGES = 6, S_MAX_SPLITS = 8, S_THREADS = 256;
constexpr int S_STAGE_BYTES = A_BYTES + S_BN * BK;
constexpr int S_RECV_BYTES = (BM + S_MAX_SPLITS) * S_BN * 4;          // shares of the rows are rounded up
constexpr int S_SMEM_BYTES = S_STAGES * S_STAGE_BYTES + S_RECV_BYTES + SF_STAGES * SF_BYTES + 1024;
constexpr uint32_t S_TMEM_COLS = 128, S_SF_COL = S_BN;
constexpr int S_PASSES = BM / 2 / 16;                                  // a CTA finishes 16 rows a pass

template <int ACT>
__global__ void __launch_bounds__(S_THREADS, 1)
gemm_block128_small_kernel(const __grid_constant__ CUtensorMap map_a32, const __grid_constant__ CUtensorMap map_w, Problem p, Out out, int* status) {
  extern __shared__ unsigned char smem_dyn[];
  __shared__ __align__(8) unsigned long long bar_mem[2 * S_STAGES + 2 * SF_STAGES + 1];
  __shared__ uint32_t tmem_base_slot;
  __shared__ int abort_flag;
  const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  const uint32_t recv = base + S_STAGES * S_STAGE_BYTES, sf0 = recv + S_RECV_BYTES;
  auto ptr = [&](uint32_t a) { return smem_dyn + (a - smem_u32(smem_dyn)); };
  const uint32_t bars = smem_u32(bar_mem);
  auto full_bar = [&](int s) { return bars + 8u * s; };
  auto empty_bar = [&](int s) { return bars + 8u * (S_STAGES + s); };
  auto sfull_bar = [&](int s) { return bars + 8u * (2 * S_STAGES + s); };
  auto sempty_bar = [&](int s) { return bars + 8u * (2 * S_STAGES + SF_STAGES + s); };
  const uint32_t done_bar = bars + 8u * (2 * S_STAGES + 2 * SF_STAGES);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = blockIdx.z, splits = gridDim.z;
  const int total_kb = (p.K + BK - 1) / BK, groups = (total_kb + 3) / 4;
  const int g0 = rank * groups / splits, g1 = (rank + 1) * groups / splits, kb0 = g0 * 4, nkb = min(g1 * 4, total_kb) - kb0;
  Tile t;
  t.e = 0;
  t.r0 = blockIdx.y * BM;
  t.r1 = min(p.M, t.r0 + BM);
  t.n0 = blockIdx.x * S_BN;
  // an equal share of the tile's rows for every CTA of the cluster; this one's are q0 to q1 - 1
  const int rows = t.r1 - t.r0, share = (rows + splits - 1) / splits, q0 = min(rank * share, rows), q1 = min(rows, q0 + share);

  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int s = 0; s < S_STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int s = 0; s < SF_STAGES; ++s) { mbar_init(sfull_bar(s), 1); mbar_init(sempty_bar(s), 1); }
    mbar_init(done_bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_map(&map_a32);
    prefetch_map(&map_w);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(&tmem_base_slot), S_TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  cluster_arrive();                        // this CTA has started: the others may write to its shared memory
  const uint32_t tmem_base = tmem_base_slot;
  release_dependents();
  await_inputs();
  volatile int* abortp = &abort_flag;

  if (warp == 0) {
    if (elected()) {
      const int boxes = (rows + 31) / 32;
      int stage = 0;
      uint32_t phase = 0;
      for (int i = 0; i < nkb; ++i) {
        if (!mbar_wait(empty_bar(stage), phase ^ 1u, abortp)) break;
        mbar_expect_tx(full_bar(stage), (uint32_t)(boxes * 32 * BK + S_BN * BK));
        const uint32_t sa = base + stage * S_STAGE_BYTES;
        tma_load_2d(sa + A_BYTES, &map_w, full_bar(stage), (kb0 + i) * BK, t.n0);
        for (int j = 0; j < boxes; ++j) tma_load_2d(sa + j * 32 * BK, &map_a32, full_bar(stage), (kb0 + i) * BK, t.r0 + j * 32);
        if (++stage == S_STAGES) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp == 1) {
    if (elected()) {
      constexpr uint32_t idesc0 = make_idesc_scaled(BM, S_BN), KSTEP = UMMA_K >> 4;
      const uint64_t desc_a0 = make_desc(base, 16, 1024), desc_w0 = make_desc(base + A_BYTES, 16, 1024), desc_s0 = make_desc_scales(sf0);
      int stage = 0, sf = 0;
      uint32_t phase = 0, sphase = 0;
      for (int i = 0; i < nkb; ++i) {
        const uint32_t sfa = tmem_base + S_SF_COL + sf * 8, sfb = sfa + 4;           // (four columns each; as many turns as stages)
        if ((i & 3) == 0) {
          if (!mbar_wait(sfull_bar(sf), sphase, abortp)) break;
          tc_fence_after();
          const uint64_t ds = desc_s0 + (uint64_t)((sf * SF_BYTES) >> 4);
          copy_scales(sfa, ds);
          copy_scales(sfb, ds + (512 >> 4));
        }
        if (!mbar_wait(full_bar(stage), phase, abortp)) break;
        tc_fence_after();
        const uint64_t off = (uint64_t)((stage * S_STAGE_BYTES) >> 4);
        const uint32_t idesc = idesc0 | sf_id(i & 3);
#pragma unroll
        for (int k = 0; k < BK / UMMA_K; ++k)
          umma_scaled(tmem_base, desc_a0 + off + (uint64_t)(k * KSTEP), desc_w0 + off + (uint64_t)(k * KSTEP), idesc, sfa, sfb, (i > 0 || k > 0) ? 1u : 0u);
        umma_commit(empty_bar(stage));
        if (++stage == S_STAGES) { stage = 0; phase ^= 1u; }
        if ((i & 3) == 3) {
          umma_commit(sempty_bar(sf));
          if (++sf == SF_STAGES) { sf = 0; sphase ^= 1u; }
        }
      }
      umma_commit(done_bar);               // after a wait that gave up: of what was issued
    }
  } else if (warp == 2) {
    const int nblocks = (p.N + 127) / 128;
    int sf = 0;
    uint32_t sphase = 0;
    Scales s;
    s.fetch(p, t, t.r0, g0, groups, nblocks, false);
    for (int g = g0; g < g1; ++g) {
      if (!warp_wait(sempty_bar(sf), sphase ^ 1u, abortp)) break;
      s.store(ptr(sf0 + sf * SF_BYTES), false);
      __syncwarp();
      if (lane == 0) mbar_arrive(sfull_bar(sf));
      if (++sf == SF_STAGES) { sf = 0; sphase ^= 1u; }
      if (g + 1 < g1) s.fetch(p, t, t.r0, g + 1, groups, nblocks, false);
    }
  }
  __syncwarp();

  // what the epilogue of this CTA's rows reads, 16 rows a pass: a thread has four columns of a row
  const int unit = threadIdx.x & 15, sub = threadIdx.x >> 4, col = t.n0 + unit * 4;
  auto at = [&](int r) { return (size_t)(t.r0 + r) * p.N + col; };
  auto mine = [&](int i) { return q0 + i * 16 + sub < q1 && col < p.N; };
  float4 bias = make_float4(0.f, 0.f, 0.f, 0.f);
  float z[S_PASSES][4];
  if (out.bias != nullptr && col < p.N) bias = __ldg(reinterpret_cast<const float4*>(out.bias + col));
  if constexpr (ACT == 2) {
#pragma unroll
    for (int i = 0; i < S_PASSES; ++i)
      if (mine(i)) load4(out.z + at(q0 + i * 16 + sub), z[i]);
  }

  // accumulators -> their rows' owners: [splits][share][64], a row's 16-byte units permuted by the row (no bank conflicts)
  const bool ok = warp_wait(done_bar, 0, abortp);
  tc_fence_after();
  cluster_wait();
  if (ok) {
    const int quarter = warp & 3, half = warp >> 2, row = quarter * 32 + lane;
    uint32_t r[32];
    tmem_ld32(tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(half * 32), r);
    tmem_ld_wait();
    if (row < rows) {
      const int owner = row / share, local = row - owner * share;
      const uint32_t dst = peer_addr(recv + (uint32_t)(rank * share + local) * (S_BN * 4), owner);
#pragma unroll
      for (int u = 0; u < 8; ++u) send16(dst + (((half * 8 + u) ^ (local & 7)) << 4), r + 4 * u);
    }
  }
  __syncwarp();
  tc_fence_before();
  cluster_arrive();
  cluster_wait();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, S_TMEM_COLS);
  }

  const float* got = reinterpret_cast<const float*>(ptr(recv));
#pragma unroll
  for (int i = 0; i < S_PASSES; ++i) {
    if (!mine(i) || !ok) continue;
    const int local = i * 16 + sub;
    const float* src = got + local * S_BN + ((unit ^ (local & 7)) << 2);
    float v[4] = {bias.x, bias.y, bias.z, bias.w};
    float4 x[S_MAX_SPLITS];
#pragma unroll
    for (int q = 0; q < S_MAX_SPLITS; ++q)
      if (q < splits) x[q] = *reinterpret_cast<const float4*>(src + q * share * S_BN);
    float4 sum = x[0];
#pragma unroll
    for (int q = 1; q < S_MAX_SPLITS; ++q)
      if (q < splits) { sum.x += x[q].x; sum.y += x[q].y; sum.z += x[q].z; sum.w += x[q].w; }
    v[0] += sum.x; v[1] += sum.y; v[2] += sum.z; v[3] += sum.w;
    if constexpr (ACT == 1) {
      if (out.z != nullptr) store4(out.z + at(q0 + local), v);
      gelu2(v[0], v[1]);
      gelu2(v[2], v[3]);
    } else if constexpr (ACT == 2) {
      gelu_grad_mul(v[0], v[1], z[i][0], z[i][1]);
      gelu_grad_mul(v[2], v[3], z[i][2], z[i][3]);
    }
    store4(out.y + at(q0 + local), v);
  }
  if (threadIdx.x == 0 && abort_flag) {
    unsigned long long t0 = global_ns();   // copies already issued still land in shared memory
    while (global_ns() - t0 < 1000000ull) {}
    if (status != nullptr) atomicOr(status, STATUS_TIMEOUT);
  }
}

// Splits of a tile's k range, 0: not a product for this kernel.  As many as still fit the SMs in one wave, each with a group of slabs at least.
static int small_splits(int m, int n, int k, int sms) {
  const long tiles = (long)ceil_div(m, BM) * ceil_div(n, S_BN);
  const int groups = ceil_div(k, 4 * BK);
  int s = 1;
  while (s < S_MAX_SPLITS && tiles * s * 2 <= sms && groups >= s * 2) s *= 2;
  return s >= 2 ? s : 0;
}
template <int ACT>
static int launch_small(const Ctx& c, const CUtensorMap& ma32, const CUtensorMap& mw, const Problem& p, const Out& o, int splits) {
  auto kern = gemm_block128_small_kernel<ACT>;
  static SmemLimit lim;
  if (!ensure_smem(lim, kern, S_SMEM_BYTES)) return -3;
  note_launch(1);
  launch_cluster(kern, dim3(ceil_div(p.N, S_BN), ceil_div(p.M, BM), splits), S_THREADS, S_SMEM_BYTES, c.stream, dim3(1, 1, splits), ma32, mw, p, o, c.status);
  return 0;
}

template <int BN, int ACT>
static int launch(const Ctx& c, const CUtensorMap& ma, const CUtensorMap& ma32, const CUtensorMap& mw, const CUtensorMap& my, const CUtensorMap& mz, const Problem& p, const Out& o, long tiles) {
  auto kern = gemm_block128_kernel<BN, ACT>;
  static SmemLimit lim;
  if (!ensure_smem(lim, kern, SMEM_BYTES)) return -3;
  const int sms = c.sm_count > 0 ? c.sm_count : B200_SMS, grid = (int)(tiles < sms ? tiles : sms);
  Out out = o;
  out.release = 2 * grid <= sms;
  note_launch(1);
  launch_k(kern, grid, THREADS, SMEM_BYTES, c.stream, ma, ma32, mw, my, mz, p, out, c.status);
  return 0;
}
template <int ACT>
static int launch_pair(const Ctx& c, const CUtensorMap& ma, const CUtensorMap& ma32, const CUtensorMap& mw, const CUtensorMap& my, const CUtensorMap& mz, const Problem& p, const Out& o, int width, long tiles) {
  auto kern = gemm_block128_pair_kernel<ACT>;
  static SmemLimit lim;
  if (!ensure_smem(lim, kern, P_SMEM_BYTES)) return -3;
  const int pairs = (c.sm_count > 0 ? c.sm_count : B200_SMS) / 2;
  note_launch(1);
  launch_k(kern, 2 * (int)(tiles < pairs ? tiles : pairs), THREADS, P_SMEM_BYTES, c.stream, ma, ma32, mw, my, mz, p, o, width, c.status);
  return 0;
}

// Rows of bf16 outputs in boxes of 32 rows x `cols` columns (64 or 32), swizzled over a row of the box.
static bool make_out_map(CUtensorMap* map, const void* ptr, int n, int m, int cols) {
  EncodeFn fn = encode_fn();
  if (fn == nullptr) return false;
  cuuint64_t dims[2] = {(cuuint64_t)n, (cuuint64_t)m};
  cuuint64_t strides[1] = {(cuuint64_t)n * 2};
  cuuint32_t box[2] = {(cuuint32_t)cols, 32};
  cuuint32_t estr[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// How a product that is not of few tiles is cut: what fits the SMs in one wave takes the narrowest tiles that do; else one CTA or two a tile,
// and the pair's width, by waves times the time of one.  A wave takes 0.93 us and 0.367 a slab on single CTAs, 1.5 and 0.38 on pairs of 240 columns
// (narrower ones less: a slab of 160, 192, 240 columns 341, 370, 402 ns where nothing else waits), or, longer, its epilogue (by activation).
//   us of a launch (thirty in a row on cool clocks), one CTA a tile and two:
//   25216 x 2304 x 384    35.2 / 35.4      25216 x 2304 x 768    53.7 / 51.5      25216 x 2304 x 1536   85.4 / 80.4      6304 x 2304 x 768    16.7 / 17.8
//   25216 x 768 x 1536    31.2 / 34.9      2048 x 2048 x 4096    23.6 / 18.6      3000 x 1000 x 7168    22.1 / 25.1      4096 x 4096 x 4096   57.7 / 53.1
//   8192 x 4096 x 7168     196 / 177       8192 x 1024 x 1024    13.9 / 16.2      64 experts of 768 rows, 1408 x 2048: 152 / 135
//   16 experts, 25216 x 1536 x 768 with GELU: 50.3 / 55.9
// Of these the estimate takes the slower side three times: 25216 x 2304 x 768 on single CTAs, 6304 x 2304 x 768 on pairs of 224 and 3000 x 1000 x 7168 on
// pairs of 176 (it has one slope for all widths and no cost for a short last wave).
// Experts are taken to have equal shares of the rows (their counts are on the device).
struct Cut { bool pair; int bn; int splits; };       // splits: of a few-tile product's k; 0: one of the persistent kernels
static Cut choose_wide_cut(int m, int n, int k, int experts, int act, int sms) {
  const int share = ceil_div(m, experts), kb = ceil_div(k, BK);
  auto tiles = [&](int rows, int cols) { return (long)(experts < m ? experts : m) * ceil_div(share, rows) * ceil_div(n, cols); };
  if (n <= 64 || tiles(BM, 64) <= sms) return {false, 64, 0};
  if (n <= 128 || tiles(BM, 128) <= sms) return {false, 128, 0};
  auto longer = [](double x, double y) { return x > y ? x : y; };
  const double epi1[3] = {0.0, 3.3, 4.3}, epi2[3] = {0.0, 4.6, 5.3};
  Cut best = {false, 192, 0};
  double t_best = ceil_div(tiles(BM, 192), sms) * longer(0.93 + 0.367 * kb, epi1[act]);
  for (int w = P_WIDTH; w >= 128; w -= 16) {
    const double t = ceil_div(tiles(2 * BM, w), sms / 2) * longer(1.5 + 0.38 * kb * (152 + w / 2) / 272, epi2[act]);
    if (t < t_best) { t_best = t; best = {true, w, 0}; }
  }
  return best;
}
static Cut choose_cut(int m, int n, int k, bool grouped, int experts, int act, int sms) {
  const int splits = grouped ? 0 : small_splits(m, n, k, sms);
  return splits > 0 ? Cut{false, S_BN, splits} : choose_wide_cut(m, n, k, experts, act, sms);
}

}  // namespace tcb

void block128_cut(const Ctx& c, int m, int n, int k, bool grouped, int experts, int act, int* out) {
  const tcb::Cut cut = tcb::choose_cut(m, n, k, grouped, experts, act, c.sm_count > 0 ? c.sm_count : B200_SMS);
  out[0] = cut.splits > 0 ? 2 : cut.pair ? 1 : 0;
  out[1] = cut.bn;
  out[2] = cut.splits > 0 ? cut.splits : 1;
}

// y [m, n] bf16 = epilogue(A W^T); see kernels.h.
int gemm_block128(const Ctx& c, const void* Aq, const void* a_scale, const void* Wq, const void* w_scale, const int* seg_start, int experts, void* C, int m, int n, int k,
                  const GemmEpilogue& e) {
  using namespace tcb;
  const int sms = c.sm_count > 0 ? c.sm_count : B200_SMS;
  const long some = seg_start != nullptr ? (experts < m ? experts : m) - 1 : 0;      // at most so many tiles more than the rows alone would take
  const Cut cut = choose_cut(m, n, k, seg_start != nullptr, experts, e.act, sms);
  const bool pair = cut.pair;
  const int bn = cut.bn, splits = cut.splits;
  bf16* z = (bf16*)(e.act == 1 ? e.aux_out : const_cast<void*>(e.aux_in));
  CUtensorMap ma, ma32, mw, my, mz;
  if (!make_out_map(&my, C, n, m, chunk_of(e.act)) || !make_out_map(&mz, z != nullptr ? z : C, n, m, chunk_of(e.act))) return -2;
  if (!make_map_u8(&ma, Aq, (uint64_t)k, (uint64_t)m, (uint64_t)k, BM) || !make_map_u8(&ma32, Aq, (uint64_t)k, (uint64_t)m, (uint64_t)k, 32) ||
      !make_map_u8(&mw, Wq, (uint64_t)k, (uint64_t)experts * n, (uint64_t)k, pair ? bn / 2 : bn))
    return -2;
  Problem p;
  p.M = m; p.N = n; p.K = k; p.tiles_n = ceil_div(n, bn); p.experts = experts; p.seg_start = seg_start;
  p.a_scale = (const uint32_t*)a_scale; p.w_scale = (const uint32_t*)w_scale;
  Out o;
  o.y = (bf16*)C;
  o.z = z;
  o.bias = e.bias;
  o.release = false;
  const long tiles = (ceil_div(m, pair ? 2 * BM : BM) + some) * p.tiles_n;
  auto go = [&](auto act) {
    constexpr int A = decltype(act)::value;
    if (splits > 0) return launch_small<A>(c, ma32, mw, p, o, splits);
    if (pair) return launch_pair<A>(c, ma, ma32, mw, my, mz, p, o, bn, tiles);
    return bn == 64 ? launch<64, A>(c, ma, ma32, mw, my, mz, p, o, tiles) : bn == 128 ? launch<128, A>(c, ma, ma32, mw, my, mz, p, o, tiles) : launch<192, A>(c, ma, ma32, mw, my, mz, p, o, tiles);
  };
  return e.act == 0 ? go(std::integral_constant<int, 0>()) : e.act == 1 ? go(std::integral_constant<int, 1>()) : go(std::integral_constant<int, 2>());
}

}  // namespace bsr
