// Rows of an expert layer: the slots (token, s) that chose an expert in the order of (expert, token, s), the tokens' rows laid out in
// that order, and the experts' outputs back per token, each with its gradient.  Unlike the tables of the step's own expert
// layers (moe.cu) an expert's rows follow the ones before without padding, and a slot may have no expert (its position is -1).
// All sums run in slot order: results do not depend on scheduling.
#include <cooperative_groups.h>

#include "common.cuh"
#include "kernels.h"

namespace bsr {

namespace cg = cooperative_groups;

// ---- positions ---------------------------------------------------------------------------------------------------------
// A stable counting sort in one launch: every warp has a run of consecutive slots.  It counts its run per expert in a row of
// shared memory of its own (lanes with equal experts find each other by match, so one of them adds for all); the counts become
// starts, down the warps, over the CTAs of the cluster through distributed shared memory, and along the experts; then the warp walks its
// run again and hands out positions.  Bound by latency: the bytes are 8 a slot.
constexpr int SORT_CLUSTER = 8, SORT_MAX_E = 1024;

template <int THREADS>
__global__ void __launch_bounds__(THREADS)
expert_sort_kernel(const int* __restrict__ expert, int slots, int E, int per_warp, int* __restrict__ pos, int* __restrict__ seg_start) {
  constexpr int W = THREADS / 32;
  extern __shared__ int sort_smem[];
  int* hist = sort_smem;                       // [W][E]
  int* total = hist + W * E;                   // [E], read by the cluster
  int* start = total + E;                      // [E]
  __shared__ int carry[W + 1];
  cg::cluster_group cluster = cg::this_cluster();
  const int ranks = cluster.num_blocks(), rank = cluster.block_rank();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t lt = (1u << lane) - 1u;
  for (int i = threadIdx.x; i < W * E; i += THREADS) hist[i] = 0;
  dependent_sync();
  __syncthreads();
  int* mine = hist + warp * E;
  const long first = (long)(rank * W + warp) * per_warp;
  const int begin = (int)min(first, (long)slots), end = (int)min(first + per_warp, (long)slots);
  for (int i0 = begin; i0 < end; i0 += 32) {
    const int i = i0 + lane;
    const int e = i < end ? expert[i] : -1;
    const bool has = e >= 0 && e < E;
    const uint32_t same = __match_any_sync(0xffffffffu, has ? e : -1);
    if (has && (same & lt) == 0) mine[e] += __popc(same);
    __syncwarp();
  }
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += THREADS) {
    int s = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const int n = hist[w * E + e];
      hist[w * E + e] = s;
      s += n;
    }
    total[e] = s;
  }
  cluster.sync();
  // starts of the experts' segments (an exclusive scan over all experts) and of this CTA's part of each
  int below = 0;
  for (int e0 = 0; e0 < E; e0 += THREADS) {
    const int e = e0 + threadIdx.x;
    int all = 0, before = 0;
    if (e < E) {
      for (int r = 0; r < ranks; ++r) {
        const int n = *cluster.map_shared_rank(&total[e], r);
        all += n;
        if (r < rank) before += n;
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
    int prior = below;
    for (int w = 0; w < W; ++w) {
      const int n = carry[w];
      if (w < warp) prior += n;
      below += n;
    }
    if (e < E) {
      start[e] = prior + scan - all + before;
      if (rank == 0) seg_start[e] = prior + scan - all;
    }
    __syncthreads();
  }
  if (rank == 0 && threadIdx.x == 0) seg_start[E] = below;
  for (int i0 = begin; i0 < end; i0 += 32) {
    const int i = i0 + lane;
    const int e = i < end ? expert[i] : -1;
    const bool has = e >= 0 && e < E;
    const uint32_t same = __match_any_sync(0xffffffffu, has ? e : -1);
    const int at = has ? start[e] + mine[e] + __popc(same & lt) : -1;
    __syncwarp();
    if (has && (same & lt) == 0) mine[e] += __popc(same);
    __syncwarp();
    if (i < end) pos[i] = at;
  }
  cluster.sync();                              // no CTA leaves while another may still read its counts
}

// ---- rows --------------------------------------------------------------------------------------------------------------
// rows[pos[t, s]] = x[t], 16 bytes a lane: x is read once, whatever the number of slots.  A warp has `cols` chunks of a token.
__global__ void __launch_bounds__(256)
expert_scatter_kernel(const uint4* __restrict__ x, int tokens, int chunks, int parts, int top_k, const int* __restrict__ pos, unsigned rows,
                      uint4* __restrict__ out) {
  dependent_sync();
  const long unit = ((long)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
  const int lane = threadIdx.x & 31;
  if (unit >= (long)tokens * parts) return;
  const int t = (int)(unit / parts), part = (int)(unit - (long)t * parts);
  const int* p = pos + (size_t)t * top_k;
  for (int ch = part * 32 + lane; ch < chunks; ch += parts * 32) {
    const uint4 v = x[(size_t)t * chunks + ch];
    for (int s = 0; s < top_k; ++s) {
      const unsigned to = (unsigned)p[s];
      if (to < rows) out[(size_t)to * chunks + ch] = v;
    }
  }
}

// out[t] = residual[t] + sum_s w[t, s] rows[pos[t, s]] (without w: the plain sum, the gradient of the scatter).  N values a lane.
template <typename TR, typename TO, int N>
__global__ void __launch_bounds__(256)
expert_combine_kernel(const TR* __restrict__ rows, const int* __restrict__ pos, const float* __restrict__ w, const TO* __restrict__ residual,
                      TO* __restrict__ out, int tokens, int dim, int parts, int top_k, unsigned nrows) {
  dependent_sync();
  const long unit = ((long)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
  const int lane = threadIdx.x & 31;
  if (unit >= (long)tokens * parts) return;
  const int t = (int)(unit / parts), part = (int)(unit - (long)t * parts);
  const int* p = pos + (size_t)t * top_k;
  for (int col = (part * 32 + lane) * N; col < dim; col += parts * 32 * N) {
    float acc[N];
    if (residual != nullptr) load_n<N>(residual + (size_t)t * dim + col, acc);
    else {
#pragma unroll
      for (int j = 0; j < N; ++j) acc[j] = 0.f;
    }
    for (int s0 = 0; s0 < top_k; s0 += 4) {
      float v[4][N], ws[4];
      bool has[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const unsigned from = s0 + u < top_k ? (unsigned)p[s0 + u] : 0xffffffffu;
        has[u] = from < nrows;
        ws[u] = w != nullptr && has[u] ? w[(size_t)t * top_k + s0 + u] : 1.f;
        if (has[u]) load_n<N>(rows + (size_t)from * dim + col, v[u]);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (has[u])
#pragma unroll
          for (int j = 0; j < N; ++j) acc[j] = fmaf(ws[u], v[u][j], acc[j]);
    }
    store_n<N>(out + (size_t)t * dim + col, acc);
  }
}

// drows[pos[t, s]] = w[t, s] dout[t];  dw[t, s] = <dout[t], rows[pos[t, s]]> (0 without an expert).  A warp a token, S slots at a time.
template <typename TR, typename TO, int N, int S>
__global__ void __launch_bounds__(256)
expert_combine_bwd_kernel(const TO* __restrict__ dout, const TR* __restrict__ rows, const int* __restrict__ pos, const float* __restrict__ w,
                          TR* __restrict__ drows, float* __restrict__ dw, int tokens, int dim, int top_k, unsigned nrows) {
  dependent_sync();
  const int t = (int)(((long)blockIdx.x * blockDim.x + threadIdx.x) >> 5), lane = threadIdx.x & 31;
  if (t >= tokens) return;
  const int* p = pos + (size_t)t * top_k;
  for (int s0 = 0; s0 < top_k; s0 += S) {
    float dot[S], ws[S];
    unsigned at[S];
#pragma unroll
    for (int u = 0; u < S; ++u) {
      at[u] = s0 + u < top_k ? (unsigned)p[s0 + u] : 0xffffffffu;
      ws[u] = at[u] < nrows ? w[(size_t)t * top_k + s0 + u] : 0.f;
      dot[u] = 0.f;
    }
    for (int col = lane * N; col < dim; col += 32 * N) {
      float g[N], v[S][N];
      load_n<N>(dout + (size_t)t * dim + col, g);
#pragma unroll
      for (int u = 0; u < S; ++u)
        if (at[u] < nrows) load_n<N>(rows + (size_t)at[u] * dim + col, v[u]);
#pragma unroll
      for (int u = 0; u < S; ++u)
        if (at[u] < nrows) {
          float d[N];
#pragma unroll
          for (int j = 0; j < N; ++j) {
            dot[u] = fmaf(g[j], v[u][j], dot[u]);
            d[j] = ws[u] * g[j];
          }
          store_n<N>(drows + (size_t)at[u] * dim + col, d);
        }
    }
#pragma unroll
    for (int u = 0; u < S; ++u) {
      const float sum = warp_sum(dot[u]);
      if (lane == 0 && s0 + u < top_k) dw[(size_t)t * top_k + s0 + u] = at[u] < nrows ? sum : 0.f;
    }
  }
}

// =================================================================================================
// launchers
// =================================================================================================
int expert_sort(const Ctx& c, const int* expert, int slots, int E, int* pos, int* seg_start) {
  constexpr int THREADS = 1024, W = THREADS / 32;
  const int ranks = slots > W * 128 ? SORT_CLUSTER : 1;
  const int per_warp = ceil_div(ceil_div(slots, ranks * W), 32) * 32;
  const size_t smem = (size_t)(W + 2) * E * sizeof(int);
  static SmemLimit lim;
  if (!ensure_smem(lim, expert_sort_kernel<THREADS>, smem)) return -3;
  note_launch(1);
  launch_cluster(expert_sort_kernel<THREADS>, ranks, THREADS, smem, c.stream, ranks, expert, slots, E, per_warp, pos, seg_start);
  return 0;
}

// Warps a token: more than one where the tokens alone would leave SMs without work.
static int parts_for(int tokens, int per_warp, int dim) {
  const int most = ceil_div(dim, per_warp), want = ceil_div(B200_SMS * 16, tokens);
  return most < want ? most : want;
}

void expert_scatter(const Ctx& c, const void* x, int tokens, int dim, int top_k, const int* pos, void* rows) {
  const int chunks = (int)(dim * dtype_size(c.dtype) / 16), parts = parts_for(tokens, 32, chunks);
  note_launch(1);
  launch_k(expert_scatter_kernel, ceil_div((long)tokens * parts, 8), 256, 0, c.stream, (const uint4*)x, tokens, chunks, parts, top_k, pos, (unsigned)tokens * (unsigned)top_k, (uint4*)rows);
}

template <typename TR, typename TO>
static void combine(const Ctx& c, const void* rows, const int* pos, const float* w, const void* residual, void* out, int tokens, int dim, int top_k) {
  constexpr int N = sizeof(TR) + sizeof(TO) == 8 ? 4 : 8;
  const int parts = parts_for(tokens, 32 * N, dim);
  note_launch(1);
  launch_k(expert_combine_kernel<TR, TO, N>, ceil_div((long)tokens * parts, 8), 256, 0, c.stream, (const TR*)rows, pos, w, (const TO*)residual, (TO*)out, tokens, dim, parts, top_k,
           (unsigned)tokens * (unsigned)top_k);
}

void expert_combine(const Ctx& c, const void* rows, int rows_dtype, const int* pos, const float* w, const void* residual, void* out, int tokens, int dim, int top_k) {
  if (rows_dtype == 0) c.dtype == 0 ? combine<float, float>(c, rows, pos, w, residual, out, tokens, dim, top_k) : combine<float, bf16>(c, rows, pos, w, residual, out, tokens, dim, top_k);
  else c.dtype == 0 ? combine<bf16, float>(c, rows, pos, w, residual, out, tokens, dim, top_k) : combine<bf16, bf16>(c, rows, pos, w, residual, out, tokens, dim, top_k);
}

template <typename TR, typename TO>
static void combine_bwd(const Ctx& c, const void* dout, const void* rows, const int* pos, const float* w, void* drows, float* dw, int tokens, int dim, int top_k) {
  constexpr int N = sizeof(TR) + sizeof(TO) == 8 ? 4 : 8;
  auto go = [&](auto kern) {
    note_launch(1);
    launch_k(kern, ceil_div((long)tokens, 8), 256, 0, c.stream, (const TO*)dout, (const TR*)rows, pos, w, (TR*)drows, dw, tokens, dim, top_k, (unsigned)tokens * (unsigned)top_k);
  };
  if (top_k <= 2) go(expert_combine_bwd_kernel<TR, TO, N, 2>);
  else go(expert_combine_bwd_kernel<TR, TO, N, 4>);
}

void expert_combine_bwd(const Ctx& c, const void* dout, const void* rows, int rows_dtype, const int* pos, const float* w, void* drows, float* dw, int tokens, int dim, int top_k) {
  if (rows_dtype == 0) c.dtype == 0 ? combine_bwd<float, float>(c, dout, rows, pos, w, drows, dw, tokens, dim, top_k) : combine_bwd<float, bf16>(c, dout, rows, pos, w, drows, dw, tokens, dim, top_k);
  else c.dtype == 0 ? combine_bwd<bf16, float>(c, dout, rows, pos, w, drows, dw, tokens, dim, top_k) : combine_bwd<bf16, bf16>(c, dout, rows, pos, w, drows, dw, tokens, dim, top_k);
}

}  // namespace bsr
