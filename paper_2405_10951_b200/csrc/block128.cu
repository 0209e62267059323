// Quantisation to E4M3 with a power-of-two scale per block of 128 values (a row's) or 128 x 128 values (a weight's):
//
//   e = the least integer with max|x| <= 448 * 2^e over the block's finite values,   q = E4M3(x * 2^-e), to nearest and even
//
// A scale is held as the byte e + 127.  Being a power of two it costs no rounding: x * 2^-e is exact, so that every code is the one nearest
// to x / scale, and the tensor core's block scaling multiplies by it exactly.  (A scale of max / 448 itself would use up to one more
// bit of the largest exponent, which a floating-point code does not need.)  Values that are not finite become the NaN code and have no
// part in the scale: only their own rows and columns of a product are lost.  Bytes per value are what bounds both kernels.
#include "block128.cuh"
#include "common.cuh"
#include "kernels.h"

namespace bsr {

// Rows of x to codes and scales, eight lanes a block of 128, 16 values each.  A thread has the loads of U blocks on their way (loads in
// flight are what the bandwidth hangs on).  The group of a row's last block also writes the padding behind its scales.  With
// `pos`, token t's codes go to the rows pos[t, 0 .. top_k) (negative: none) of what is written, which has `rows` of them; without
// it to row t.
constexpr int QR_THREADS = 256, QR_UNITS = QR_THREADS / 8;
template <typename T, bool SCATTER, int U>
__global__ void __launch_bounds__(QR_THREADS)
quantize_rows128_kernel(const T* __restrict__ x, unsigned units, int k, unsigned kblocks, int stride, const int* __restrict__ pos, int top_k, unsigned rows,
                        uint8_t* __restrict__ q, uint8_t* __restrict__ scale) {
  dependent_sync();
  const unsigned u0 = blockIdx.x * (QR_UNITS * U) + (threadIdx.x >> 3);
  const int lane8 = threadIdx.x & 7;
  Values16<T> v[U];
  unsigned row[U], blk[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const unsigned u = u0 + i * QR_UNITS;
    row[i] = u / kblocks;
    blk[i] = u - row[i] * kblocks;
    const int col = (int)blk[i] * 128 + lane8 * 16;
    if (u < units && col < k) v[i].load(x + (size_t)row[i] * k + col);
    else v[i].zero();
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    uint32_t top = v[i].top();
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    const bool finite = top < F32_INF;
    if (!__all_sync(0xffffffffu, finite)) {
      uint32_t f = finite_top(v[i]);
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) f = max(f, __shfl_xor_sync(0xffffffffu, f, o));
      top = f;
    }
    const uint32_t byte = scale_byte(top);
    const uint4 c = codes16(v[i], byte, finite);
    const int col = (int)blk[i] * 128 + lane8 * 16;
    if (u0 + i * QR_UNITS >= units) continue;
    const int pad = blk[i] == kblocks - 1 ? stride - (int)kblocks : 0;           // lane 0 writes the scale, lanes 1 .. 3 the padding
    auto put = [&](size_t to) {
      if (col < k) *reinterpret_cast<uint4*>(q + to * k + col) = c;
      if (lane8 <= pad) scale[to * stride + blk[i] + lane8] = (uint8_t)(lane8 == 0 ? byte : 127u);
    };
    if constexpr (SCATTER) {
      for (int s = 0; s < top_k; ++s) {
        const unsigned to = (unsigned)pos[(size_t)row[i] * top_k + s];
        if (to < rows) put(to);
      }
    } else {
      put(row[i]);
    }
  }
}

// Stacked matrices w [count, n, k]: a CTA per block of 128 x 128, which it holds in registers (16 columns of four rows a thread).  With
// qt also the transposed copies [count, k, n] and their scales: a block's scale is the same either way, and its codes are turned in
// shared memory, four by four.
constexpr int QB_THREADS = 256;
template <typename T>
__global__ void __launch_bounds__(QB_THREADS)
quantize_blocks128_kernel(const T* __restrict__ w, int n, int k, uint8_t* __restrict__ q, uint8_t* __restrict__ scale, int stride,
                          uint8_t* __restrict__ qt, uint8_t* __restrict__ scale_t, int stride_t) {
  dependent_sync();
  __shared__ uint32_t tops[QB_THREADS / 32];
  __shared__ uint32_t tile[128 * 33];
  const int kb = blockIdx.x, nb = blockIdx.y;
  const size_t mat = blockIdx.z;
  const int r0 = threadIdx.x >> 3, c0 = (threadIdx.x & 7) * 16, col = kb * 128 + c0;
  w += mat * n * k;
  q += mat * n * k;
  Values16<T> v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = nb * 128 + r0 + 32 * i;
    if (row < n && col < k) v[i].load(w + (size_t)row * k + col);
    else v[i].zero();
  }
  uint32_t top = 0;
  auto reduce = [&]() {
    top = __reduce_max_sync(0xffffffffu, top);
    if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < QB_THREADS / 32; ++i) top = max(top, tops[i]);
  };
#pragma unroll
  for (int i = 0; i < 4; ++i) top = max(top, v[i].top());
  reduce();
  const bool finite = top < F32_INF;
  if (!finite) {                                 // (the same for all threads)
    __syncthreads();
    top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, finite_top(v[i]));
    reduce();
  }
  const uint32_t byte = scale_byte(top);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = r0 + 32 * i, row = nb * 128 + r;
    const uint4 c = codes16(v[i], byte, finite);
    if (row < n && col < k) *reinterpret_cast<uint4*>(q + (size_t)row * k + col) = c;
    if (qt != nullptr) {
      uint32_t* at = tile + r * 33 + c0 / 4;
      at[0] = c.x; at[1] = c.y; at[2] = c.z; at[3] = c.w;
    }
  }
  // scales: the thread of the block's first column writes its byte, the last block's threads the padding behind it
  const int kblocks = (k - 1) / 128 + 1, nblocks = (n - 1) / 128 + 1;       // (k may lie within 127 of 2^31)
  if (threadIdx.x == 0) scale[(mat * nblocks + nb) * stride + kb] = (uint8_t)byte;
  if (kb == kblocks - 1 && threadIdx.x < stride - kblocks) scale[(mat * nblocks + nb) * stride + kblocks + threadIdx.x] = 127;
  if (qt == nullptr) return;
  if (threadIdx.x == 0) scale_t[(mat * kblocks + kb) * stride_t + nb] = (uint8_t)byte;
  if (nb == nblocks - 1 && threadIdx.x < stride_t - nblocks) scale_t[(mat * kblocks + kb) * stride_t + nblocks + threadIdx.x] = 127;
  __syncthreads();
  // a thread turns four 4 x 4 squares of a word column (four values of k): rows n 16 a .. 16 a + 15, and writes 16 bytes a value of k
  const int kw = threadIdx.x & 31, a = threadIdx.x >> 5;
  uint32_t out[4][4];
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    uint32_t x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = tile[(a * 16 + s * 4 + j) * 33 + kw];
    const uint32_t p0 = __byte_perm(x[0], x[1], 0x5140), p1 = __byte_perm(x[2], x[3], 0x5140);
    const uint32_t p2 = __byte_perm(x[0], x[1], 0x7362), p3 = __byte_perm(x[2], x[3], 0x7362);
    out[0][s] = __byte_perm(p0, p1, 0x5410);
    out[1][s] = __byte_perm(p0, p1, 0x7632);
    out[2][s] = __byte_perm(p2, p3, 0x5410);
    out[3][s] = __byte_perm(p2, p3, 0x7632);
  }
  __syncthreads();
  // through shared memory once more, so that a row of the transposed copy leaves 128 bytes at a time
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int s = 0; s < 4; ++s) tile[(kw * 4 + j) * 33 + a * 4 + s] = out[j][s];
  __syncthreads();
  qt += mat * n * k;
  const int ncol = nb * 128 + c0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = r0 + 32 * i, krow = kb * 128 + r;
    if (krow < k && ncol < n) {
      uint4 u;
      u.x = tile[r * 33 + c0 / 4]; u.y = tile[r * 33 + c0 / 4 + 1]; u.z = tile[r * 33 + c0 / 4 + 2]; u.w = tile[r * 33 + c0 / 4 + 3];
      *reinterpret_cast<uint4*>(qt + (size_t)krow * n + ncol) = u;
    }
  }
}

int scale_stride128(int k) { return (k / 512 + (k % 512 != 0)) * 4; }

template <typename T>
static void quantize_rows(const Ctx& c, const void* x, int m, int k, const int* pos, int top_k, void* q, void* scale) {
  const unsigned kblocks = (unsigned)ceil_div(k, 128), units = (unsigned)m * kblocks;
  const int stride = scale_stride128(k);
  constexpr int U = sizeof(T) == 2 ? 2 : 1;
  const unsigned per = QR_UNITS * U, blocks = (units + per - 1) / per;
  note_launch(1);
  if (pos != nullptr)
    launch_k(quantize_rows128_kernel<T, true, U>, blocks, QR_THREADS, 0, c.stream, (const T*)x, units, k, kblocks, stride, pos, top_k, (unsigned)m * (unsigned)top_k, (uint8_t*)q, (uint8_t*)scale);
  else
    launch_k(quantize_rows128_kernel<T, false, U>, blocks, QR_THREADS, 0, c.stream, (const T*)x, units, k, kblocks, stride, pos, top_k, 0u, (uint8_t*)q, (uint8_t*)scale);
}

void quantize_rows128(const Ctx& c, const void* x, int m, int k, const int* pos, int top_k, void* q, void* scale) {
  if (c.dtype == 0) quantize_rows<float>(c, x, m, k, pos, top_k, q, scale);
  else quantize_rows<bf16>(c, x, m, k, pos, top_k, q, scale);
}

void quantize_blocks128(const Ctx& c, const void* w, int count, int n, int k, void* q, void* scale, void* qt, void* scale_t) {
  const dim3 grid(ceil_div(k, 128), ceil_div(n, 128), count);
  note_launch(1);
  if (c.dtype == 0)
    launch_k(quantize_blocks128_kernel<float>, grid, QB_THREADS, 0, c.stream, (const float*)w, n, k, (uint8_t*)q, (uint8_t*)scale, scale_stride128(k), (uint8_t*)qt, (uint8_t*)scale_t, scale_stride128(n));
  else
    launch_k(quantize_blocks128_kernel<bf16>, grid, QB_THREADS, 0, c.stream, (const bf16*)w, n, k, (uint8_t*)q, (uint8_t*)scale, scale_stride128(k), (uint8_t*)qt, (uint8_t*)scale_t, scale_stride128(n));
}

}  // namespace bsr
