// Rows of an expert layer: the slots (token, s) that chose an expert in the order of (expert, token, s), the tokens' rows laid out in
// that order, and the experts' outputs back per token, each with its gradient.  Unlike the tables of the step's own expert
// layers (moe.cu) an expert's rows follow the ones before without padding, and a slot may have no expert (its position is -1).
// All sums run in slot order: results do not depend on scheduling.
#include <cooperative_groups.h>

#include <type_traits>

#include "common.cuh"
#include "kernels.h"

namespace bsr {

namespace cg = cooperative_groups;

// ---- positions ---------------------------------------------------------------------------------------------------------
// A stable counting sort in one launch: every warp has a run of consecutive slots.  It counts its run per expert in a row of
// shared memory of its own; the counts become starts, down the warps, over the CTAs of the cluster through distributed shared memory, and
// along the experts; then the warp walks its run again and hands out positions: lanes with equal experts find each other by
// a ballot for each bit of the expert's number (with the match instruction 262144 slots of 128 experts took 57 us, so 24, and 13.7 with
// sixteen CTAs instead of eight).  Bound by latency (the bytes are 8 a slot), so the experts' numbers of four steps are
// loaded at once.
constexpr int SORT_CLUSTER = 16, SORT_U = 4;

template <int THREADS, int BITS>
__global__ void __launch_bounds__(THREADS)
expert_sort_kernel(const int* __restrict__ expert, int slots, int E, int per_warp, int* __restrict__ pos, int* __restrict__ seg_start) {
  constexpr int W = THREADS / 32;
  extern __shared__ int sort_smem[];
  int* hist = sort_smem;                       // [W][E]
  int* total = hist + W * E;                   // [E], read by the cluster
  int* start = total + E;                      // [E]
  __shared__ int carry[W];
  cg::cluster_group cluster = cg::this_cluster();
  const int ranks = cluster.num_blocks(), rank = cluster.block_rank();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t lt = (1u << lane) - 1u;
  int* mine = hist + warp * E;
  for (int i = lane; i < E; i += 32) mine[i] = 0;
  __syncwarp();
  dependent_sync();
  const long first = (long)(rank * W + warp) * per_warp;
  const int begin = (int)min(first, (long)slots), end = (int)min(first + per_warp, (long)slots);
  auto load = [&](int i0, int* e) {            // -1: no expert
#pragma unroll
    for (int u = 0; u < SORT_U; ++u) {
      const int i = i0 + u * 32 + lane;
      e[u] = i < end ? expert[i] : -1;
    }
#pragma unroll
    for (int u = 0; u < SORT_U; ++u) e[u] = e[u] < E ? max(e[u], -1) : -1;
  };
  for (int i0 = begin; i0 < end; i0 += 32 * SORT_U) {
    int e[SORT_U];
    load(i0, e);
#pragma unroll
    for (int u = 0; u < SORT_U; ++u)
      if (e[u] >= 0) atomicAdd(&mine[e[u]], 1);         // integer counts: order-independent
  }
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += THREADS) {
    int s = 0;
#pragma unroll 8
    for (int w = 0; w < W; ++w) {
      const int n = hist[w * E + e];
      hist[w * E + e] = s;
      s += n;
    }
    total[e] = s;
  }
  if (ranks > 1) cluster.sync(); else __syncthreads();
  // starts of the experts' segments (an exclusive scan over all experts) and of this CTA's part of each
  int below = 0;
  for (int e0 = 0; e0 < E; e0 += THREADS) {
    const int e = e0 + threadIdx.x;
    int all = 0, before = 0;
    if (e < E) {
      if (ranks == 1) all = total[e];
      else {
#pragma unroll
        for (int r = 0; r < SORT_CLUSTER; ++r) {
          const int n = r < ranks ? *cluster.map_shared_rank(&total[e], r) : 0;
          all += n;
          if (r < rank) before += n;
        }
      }
    }
    int scan = all;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int n = __shfl_up_sync(0xffffffffu, scan, o);
      if (lane >= o) scan += n;
    }
    if (lane == 31) carry[warp] = scan;
    __syncthreads();
    int prior = lane < W ? carry[lane] : 0;            // (at most 32 warps)
    const int sum = warp_sum_int(prior);
    prior = below + warp_sum_int(lane < warp ? prior : 0);
    below += sum;
    if (e < E) {
      start[e] = prior + scan - all + before;
      if (rank == 0) seg_start[e] = prior + scan - all;
    }
    __syncthreads();
  }
  if (rank == 0 && threadIdx.x == 0) seg_start[E] = below;
  for (int i0 = begin; i0 < end; i0 += 32 * SORT_U) {
    int e[SORT_U];
    load(i0, e);
#pragma unroll
    for (int u = 0; u < SORT_U; ++u) {
      const int i = i0 + u * 32 + lane;
      uint32_t same = __ballot_sync(0xffffffffu, e[u] >= 0);
#pragma unroll
      for (int b = 0; b < BITS; ++b) {
        const bool bit = (e[u] >> b) & 1;
        same &= __ballot_sync(0xffffffffu, bit) ^ (bit ? 0u : 0xffffffffu);
      }
      int at = -1;
      if (e[u] >= 0) {
        at = start[e[u]] + mine[e[u]] + __popc(same & lt);
      }
      __syncwarp();
      if (e[u] >= 0 && (same & lt) == 0) mine[e[u]] += __popc(same);
      __syncwarp();
      if (i < end) pos[i] = at;
    }
  }
  if (ranks > 1) cluster.sync();               // no CTA leaves while another may still read its counts
}

// ---- rows --------------------------------------------------------------------------------------------------------------
// rows[pos[t, s]] = x[t], 16 bytes a thread: x is read once, whatever the number of slots.  A CTA has `cx` chunks of `ty` tokens beside
// one another, so that a row's bytes leave together (32768 tokens, 8 slots, 2048 wide: a warp walking a token's row 191 us, this
// 176, the loads of two tokens a thread 180).
__global__ void __launch_bounds__(512)
expert_scatter_kernel(const uint4* __restrict__ x, int tokens, int chunks, int cx, int ty, int top_k, const int* __restrict__ pos, unsigned rows, uint4* __restrict__ out) {
  dependent_sync();
  const int tl = threadIdx.x / cx, ch = blockIdx.y * cx + threadIdx.x - tl * cx, t = blockIdx.x * ty + tl;
  if (tl >= ty || ch >= chunks || t >= tokens) return;
  const uint4 v = x[(size_t)t * chunks + ch];
  const int* p = pos + (size_t)t * top_k;
#pragma unroll 4
  for (int s = 0; s < top_k; ++s) {
    const unsigned to = (unsigned)p[s];
    if (to < rows) out[(size_t)to * chunks + ch] = v;
  }
}

// 16 bytes of a row and the values in them (eight bf16, four floats).
template <typename T> struct Chunk { static constexpr int N = 16 / sizeof(T); };
template <typename T> __device__ __forceinline__ void chunk_values(const uint4& u, float* v);
template <> __device__ __forceinline__ void chunk_values<float>(const uint4& u, float* v) {
  v[0] = __uint_as_float(u.x); v[1] = __uint_as_float(u.y); v[2] = __uint_as_float(u.z); v[3] = __uint_as_float(u.w);
}
template <> __device__ __forceinline__ void chunk_values<bf16>(const uint4& u, float* v) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) { v[2 * j] = __uint_as_float(w[j] << 16); v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u); }
}
// As many values of the other tensor's row, whatever its type.
template <int N> __device__ __forceinline__ void load_vals(const float* p, float* f) { load_n<N>(p, f); }
template <int N> __device__ __forceinline__ void load_vals(const bf16* p, float* f) { if constexpr (N == 8) load16(p, f); else load4(p, f); }
template <int N> __device__ __forceinline__ void store_vals(float* p, const float* f) { store_n<N>(p, f); }
template <int N> __device__ __forceinline__ void store_vals(bf16* p, const float* f) { if constexpr (N == 8) store16(p, f); else store4(p, f); }

// out[t] = residual[t] + sum_s w[t, s] rows[pos[t, s]] (without w: the plain sum, the gradient of the scatter).
// Bytes bound it, and what moves them is loads in flight: rows lie anywhere, so a thread reads the positions of S slots, then has their
// S loads of 16 bytes on their way.  More a thread (eight slots, or several tokens) leaves fewer threads on an SM and is slower:
// 12608 tokens, 2 slots, 384 wide 14.5 us with four tokens a thread, 11.2 with one; 32768 tokens, 8 slots, 2048 wide 242 us with
// eight slots at once, 219 with four.
template <typename TR, typename TO, int S>
__global__ void __launch_bounds__(256)
expert_combine_kernel(const TR* __restrict__ rows, const int* __restrict__ pos, const float* __restrict__ w, const TO* __restrict__ residual,
                      TO* __restrict__ out, int tokens, int dim, int cx, int ty, int top_k, unsigned nrows) {
  constexpr int N = Chunk<TR>::N;
  dependent_sync();
  const int tl = threadIdx.x / cx, col = (blockIdx.y * cx + threadIdx.x - tl * cx) * N, t = blockIdx.x * ty + tl;
  if (tl >= ty || col >= dim || t >= tokens) return;
  float acc[N];
  if (residual != nullptr) load_vals<N>(residual + (size_t)t * dim + col, acc);
  else {
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j] = 0.f;
  }
  for (int s0 = 0; s0 < top_k; s0 += S) {
    unsigned from[S];
    uint4 v[S];
    float ws[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const size_t slot = (size_t)t * top_k + s0 + s;
      const bool is = s0 + s < top_k;
      from[s] = is ? (unsigned)pos[slot] : 0xffffffffu;
      ws[s] = is && w != nullptr ? w[slot] : 1.f;
    }
#pragma unroll
    for (int s = 0; s < S; ++s)
      if (from[s] < nrows) v[s] = *reinterpret_cast<const uint4*>(rows + (size_t)from[s] * dim + col);
#pragma unroll
    for (int s = 0; s < S; ++s)
      if (from[s] < nrows) {
        float f[N];
        chunk_values<TR>(v[s], f);
#pragma unroll
        for (int j = 0; j < N; ++j) acc[j] = fmaf(ws[s], f[j], acc[j]);
      }
  }
  store_vals<N>(out + (size_t)t * dim + col, acc);
}

// Sums of S values over the warp: each exchange halves the values that a lane still has, so that lanes s * 32 / S ... have the sum of
// value s (S - 1 + log2(32 / S) shuffles instead of 5 S).  Returns this lane's.
template <int S>
__device__ __forceinline__ float warp_sums(float* v) {
  const int lane = threadIdx.x & 31;
  int o = 16;
#pragma unroll
  for (int n = S / 2; n > 0; n >>= 1, o >>= 1)
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const bool up = (lane & o) != 0;
      const float give = up ? v[i] : v[i + n], keep = up ? v[i + n] : v[i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
    }
  float s = v[0];
  for (; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}

// drows[pos[t, s]] = w[t, s] dout[t];  dw[t, s] = <dout[t], rows[pos[t, s]]> (0 without an expert).  `wpt` warps a token, by the length of
// its row, S slots at a time with all their loads in flight; the warps' parts of a dot product meet in shared memory, in warp order.
template <typename TR, typename TO, int S>
__global__ void __launch_bounds__(256)
expert_combine_bwd_kernel(const TO* __restrict__ dout, const TR* __restrict__ rows, const int* __restrict__ pos, const float* __restrict__ w,
                          TR* __restrict__ drows, float* __restrict__ dw, int tokens, int dim, int wpt, int top_k, unsigned nrows) {
  constexpr int N = Chunk<TR>::N, PER = 32 / S;
  __shared__ float part[8][S];
  dependent_sync();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int tl = warp / wpt, wr = warp - tl * wpt;
  const int t = blockIdx.x * (8 / wpt) + tl;
  for (int s0 = 0; s0 < top_k; s0 += S) {
    float dot[S], ws[S];
    unsigned at[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const bool is = t < tokens && s0 + s < top_k;
      at[s] = is ? (unsigned)pos[(size_t)t * top_k + s0 + s] : 0xffffffffu;
      ws[s] = is ? w[(size_t)t * top_k + s0 + s] : 0.f;
      dot[s] = 0.f;
    }
    if (t < tokens)
      for (int col = (wr * 32 + lane) * N; col < dim; col += wpt * 32 * N) {
        float g[N];
        uint4 v[S];
        load_vals<N>(dout + (size_t)t * dim + col, g);
#pragma unroll
        for (int s = 0; s < S; ++s)
          if (at[s] < nrows) v[s] = *reinterpret_cast<const uint4*>(rows + (size_t)at[s] * dim + col);
#pragma unroll
        for (int s = 0; s < S; ++s)
          if (at[s] < nrows) {
            float d[N], f[N];
            chunk_values<TR>(v[s], f);
#pragma unroll
            for (int j = 0; j < N; ++j) {
              dot[s] = fmaf(g[j], f[j], dot[s]);
              d[j] = ws[s] * g[j];
            }
            store_vals<N>(drows + (size_t)at[s] * dim + col, d);
          }
      }
    const float sum = warp_sums<S>(dot);
    const int s = lane / PER;
    const bool writes = lane % PER == 0 && t < tokens && s0 + s < top_k;
    if (wpt == 1) {
      if (writes) dw[(size_t)t * top_k + s0 + s] = sum;
    } else {
      if (lane % PER == 0) part[warp][s] = sum;
      __syncthreads();
      if (wr == 0 && writes) {
        float all = sum;
        for (int q = 1; q < wpt; ++q) all += part[warp + q][s];
        dw[(size_t)t * top_k + s0 + s] = all;
      }
      __syncthreads();
    }
  }
}

// =================================================================================================
// launchers
// =================================================================================================
int expert_sort(const Ctx& c, const int* expert, int slots, int E, int* pos, int* seg_start) {
  // Few slots (decoding) leave most of a large CTA idle, and its start takes longer: 4 slots, 16 experts 3.2 -> 2.4 us.  Many go to a
  // cluster of sixteen CTAs, which the kernel has to be allowed once.
  auto go = [&](auto kern, int threads, int ranks, SmemLimit& lim) {
    const int warps = threads / 32, per_warp = ceil_div(ceil_div(slots, ranks * warps), 32) * 32;
    const size_t smem = (size_t)(warps + 2) * E * sizeof(int);
    if (!ensure_smem(lim, kern, smem)) return -3;
    if (ranks > 8 && cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return -3;
    note_launch(1);
    launch_cluster(kern, ranks, threads, smem, c.stream, ranks, expert, slots, E, per_warp, pos, seg_start);
    return 0;
  };
  auto size = [&](auto bits) {
    constexpr int B = decltype(bits)::value;
    static SmemLimit small, large;
    if (slots <= 2048) return go(expert_sort_kernel<256, B>, 256, 1, small);
    const int want = ceil_div(slots, 4096);           // 128 slots a warp (25216 slots, 16 experts: 5.2 us; 512 a warp 9.8)
    return go(expert_sort_kernel<1024, B>, 1024, want < SORT_CLUSTER ? want : SORT_CLUSTER, large);
  };
  return E <= 16 ? size(std::integral_constant<int, 4>()) : E <= 128 ? size(std::integral_constant<int, 7>()) : size(std::integral_constant<int, 10>());
}

// A row's chunks over up to `cap` threads of a CTA: `cx` of them, `ty` tokens beside one another, a row that is too long in `parts`.
struct Spread {
  int parts, cx, ty, threads;
  Spread(int chunks, int cap) : parts(ceil_div(chunks, cap)), cx(ceil_div(chunks, parts)), ty(cap / cx), threads(ceil_div(cx * ty, 32) * 32) {}
  bool fuller_than(const Spread& o) const { return (long)cx * ty * o.threads > (long)o.cx * o.ty * threads; }
};

void expert_scatter(const Ctx& c, const void* x, int tokens, int dim, int top_k, const int* pos, void* rows) {
  const int chunks = (int)(dim * dtype_size(c.dtype) / 16);
  // 256 threads, or 512 where that leaves fewer of them without a chunk (6305 tokens, 4 slots, 257 chunks: 129 of 160 threads 26.6 us, 257 of 288
  // 22.7; in the combination, whose registers then allow fewer CTAs, 32768 tokens, 8 slots, 2048 wide 218 -> 236)
  const Spread less(chunks, 256), more(chunks, 512), s = more.fuller_than(less) ? more : less;
  note_launch(1);
  launch_k(expert_scatter_kernel, dim3(ceil_div(tokens, s.ty), s.parts), s.threads, 0, c.stream, (const uint4*)x, tokens, chunks, s.cx, s.ty, top_k, pos,
           (unsigned)tokens * (unsigned)top_k, (uint4*)rows);
}

template <typename TR, typename TO>
static void combine(const Ctx& c, const void* rows, const int* pos, const float* w, const void* residual, void* out, int tokens, int dim, int top_k) {
  const Spread s(dim / Chunk<TR>::N, 256);
  auto go = [&](auto kern) {
    note_launch(1);
    launch_k(kern, dim3(ceil_div(tokens, s.ty), s.parts), s.threads, 0, c.stream, (const TR*)rows, pos, w, (const TO*)residual, (TO*)out, tokens, dim, s.cx, s.ty, top_k,
             (unsigned)tokens * (unsigned)top_k);
  };
  if (top_k <= 2) go(expert_combine_kernel<TR, TO, 2>);
  else go(expert_combine_kernel<TR, TO, 4>);
}

void expert_combine(const Ctx& c, const void* rows, int rows_dtype, const int* pos, const float* w, const void* residual, void* out, int tokens, int dim, int top_k) {
  if (rows_dtype == 0) c.dtype == 0 ? combine<float, float>(c, rows, pos, w, residual, out, tokens, dim, top_k) : combine<float, bf16>(c, rows, pos, w, residual, out, tokens, dim, top_k);
  else c.dtype == 0 ? combine<bf16, float>(c, rows, pos, w, residual, out, tokens, dim, top_k) : combine<bf16, bf16>(c, rows, pos, w, residual, out, tokens, dim, top_k);
}

template <typename TR, typename TO>
static void combine_bwd(const Ctx& c, const void* dout, const void* rows, const int* pos, const float* w, void* drows, float* dw, int tokens, int dim, int top_k) {
  // Warps a token: by the length of its row; fewer where there are tokens enough and the last round would leave most lanes without a
  // chunk (257 chunks: eight warps 44 us for 6305 tokens and 4 slots of floats, one 41).
  const int chunks = dim / Chunk<TR>::N;
  int wpt = chunks <= 64 ? 1 : chunks <= 128 ? 2 : chunks <= 256 ? 4 : 8;
  auto lanes = [&](int w) { return 32 * w * ceil_div(chunks, 32 * w); };
  while (wpt > 1 && (long)tokens * wpt >= 32 * B200_SMS && lanes(wpt) * 9 > lanes(1) * 10) wpt /= 2;
  auto go = [&](auto kern) {
    note_launch(1);
    launch_k(kern, ceil_div(tokens, 8 / wpt), 256, 0, c.stream, (const TO*)dout, (const TR*)rows, pos, w, (TR*)drows, dw, tokens, dim, wpt, top_k, (unsigned)tokens * (unsigned)top_k);
  };
  if (top_k <= 2) go(expert_combine_bwd_kernel<TR, TO, 2>);
  else go(expert_combine_bwd_kernel<TR, TO, 4>);         // (eight at once: 32768 tokens, 8 slots, 2048 wide 314 -> 354 us)
}

void expert_combine_bwd(const Ctx& c, const void* dout, const void* rows, int rows_dtype, const int* pos, const float* w, void* drows, float* dw, int tokens, int dim, int top_k) {
  if (rows_dtype == 0) c.dtype == 0 ? combine_bwd<float, float>(c, dout, rows, pos, w, drows, dw, tokens, dim, top_k) : combine_bwd<float, bf16>(c, dout, rows, pos, w, drows, dw, tokens, dim, top_k);
  else c.dtype == 0 ? combine_bwd<bf16, float>(c, dout, rows, pos, w, drows, dw, tokens, dim, top_k) : combine_bwd<bf16, bf16>(c, dout, rows, pos, w, drows, dw, tokens, dim, top_k);
}

}  // namespace bsr
