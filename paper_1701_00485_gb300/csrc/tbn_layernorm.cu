// tbn_layernorm.cu -- layer norm over the last dimension, forward and
// backward, with the reduction of the gradients of gamma and beta.
//
//   mean = sum x / D,  var = sum (x - mean)^2 / D,  rstd = (var + eps)^-1/2
//   y = (x - mean) rstd gamma + beta
// and with w = gamma dy, xh = (x - mean) rstd:
//   dx = dres + rstd (w - sum w / D - xh sum (w xh) / D)
//   dgamma = sum over rows of dy xh,  dbeta = sum over rows of dy
//
// Both directions are bound by HBM: forward reads x and writes y, backward
// reads x, dy (and dres) and writes dx.  A row stays in registers between its
// statistics and its result, so each tensor is touched once; the variance is
// the sum of squared distances from the mean (no cancellation), and every sum
// is held in 32 bits and taken in an order that depends on the sizes alone.
#include <cuda_bf16.h>

#include "tbn_device.cuh"
#include "tbn_internal.h"

namespace tbn {
namespace {

constexpr int kVec = 8;   // consecutive elements of a thread

__device__ __forceinline__ float bf16_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }

// Element indexes of a row over `threads` threads: thread t's slot (j, k) is
// its k-th element of vector j where rows are 16-byte aligned, and element
// (8 j + k) threads + t where they are not (then each access of a warp still
// covers consecutive addresses).
template <bool kAligned>
__device__ __forceinline__ int slot(int j, int k, int t, int threads) {
  return kAligned ? (j * threads + t) * kVec + k : (j * kVec + k) * threads + t;
}

template <bool kAligned, typename T, int NV>
__device__ __forceinline__ void load_row(const T* p, int D, int t, int threads,
                                         float (&v)[NV][kVec]) {
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if constexpr (kAligned) {
      const int e = slot<true>(j, 0, t, threads);
      if (e < D) {
        if constexpr (sizeof(T) == 2) {
          const uint4 r = *reinterpret_cast<const uint4*>(p + e);
          v[j][0] = bf16_lo(r.x); v[j][1] = bf16_hi(r.x);
          v[j][2] = bf16_lo(r.y); v[j][3] = bf16_hi(r.y);
          v[j][4] = bf16_lo(r.z); v[j][5] = bf16_hi(r.z);
          v[j][6] = bf16_lo(r.w); v[j][7] = bf16_hi(r.w);
        } else {
          const float4 a = *reinterpret_cast<const float4*>(p + e);
          const float4 b = *reinterpret_cast<const float4*>(p + e + 4);
          v[j][0] = a.x; v[j][1] = a.y; v[j][2] = a.z; v[j][3] = a.w;
          v[j][4] = b.x; v[j][5] = b.y; v[j][6] = b.z; v[j][7] = b.w;
        }
      } else {
#pragma unroll
        for (int k = 0; k < kVec; ++k) v[j][k] = 0.0f;
      }
    } else {
#pragma unroll
      for (int k = 0; k < kVec; ++k) {
        const int e = slot<false>(j, k, t, threads);
        v[j][k] = e < D ? static_cast<float>(p[e]) : 0.0f;
      }
    }
  }
}

// gamma or beta (fp32 or bf16, any alignment that its type has), or `none`.
template <bool kAligned, int NV>
__device__ __forceinline__ void load_weight(const void* w, bool bf16, float none, int D, int t,
                                            int threads, float (&v)[NV][kVec]) {
  if (w == nullptr) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < kVec; ++k) v[j][k] = none;
  } else if (bf16) {
    load_row<kAligned>(static_cast<const __nv_bfloat16*>(w), D, t, threads, v);
  } else {
    load_row<kAligned>(static_cast<const float*>(w), D, t, threads, v);
  }
}

template <bool kAligned, int NV>
__device__ __forceinline__ void store_row(void* out, bool bf16, int64_t at, int D, int t,
                                          int threads, const float (&v)[NV][kVec]) {
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if constexpr (kAligned) {
      const int e = slot<true>(j, 0, t, threads);
      if (e < D) {
        if (bf16) {
          *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(out) + at + e) =
              make_uint4(pack_bf16x2(v[j][0], v[j][1]), pack_bf16x2(v[j][2], v[j][3]),
                         pack_bf16x2(v[j][4], v[j][5]), pack_bf16x2(v[j][6], v[j][7]));
        } else {
          float4* p = reinterpret_cast<float4*>(static_cast<float*>(out) + at + e);
          p[0] = make_float4(v[j][0], v[j][1], v[j][2], v[j][3]);
          p[1] = make_float4(v[j][4], v[j][5], v[j][6], v[j][7]);
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < kVec; ++k) {
        const int e = slot<false>(j, k, t, threads);
        if (e < D) {
          if (bf16)
            static_cast<__nv_bfloat16*>(out)[at + e] = __float2bfloat16_rn(v[j][k]);
          else
            static_cast<float*>(out)[at + e] = v[j][k];
        }
      }
    }
  }
}

// Sums of a and b over the lanes of a group of G (a power of two, <= 32).
template <int G>
__device__ __forceinline__ void group_sum(float& a, float& b) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) {
    a += __shfl_xor_sync(0xffffffffu, a, o);
    b += __shfl_xor_sync(0xffffffffu, b, o);
  }
}

// The same over a row's threads: a group of G <= 32 lanes, or (G = 0) the
// block, through `red`, which the next call may use again at once where the
// caller alternates between two of them.
template <int G>
__device__ __forceinline__ void row_sum(float& a, float& b, float2* red) {
  if constexpr (G != 0) {
    group_sum<G>(a, b);
  } else {
    group_sum<32>(a, b);
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) red[threadIdx.x >> 5] = make_float2(a, b);
    __syncthreads();
    const float2 v = lane < warps ? red[lane] : make_float2(0.0f, 0.0f);
    a = v.x;
    b = v.y;
    group_sum<32>(a, b);
  }
}

struct FwdArgs {
  const void* x;
  void* y;
  const void *gamma, *beta;
  float *mean, *rstd;
  int64_t rows, ldx, ldy;
  int D;
  float eps;
  int y_bf16, w_bf16;
};

// A row by G lanes (256 / G rows per block) or, G = 0, by the block.
template <typename T, bool kAligned, int G, int NV>
__global__ void __launch_bounds__(G != 0 ? 256 : 1024) layernorm_fwd_kernel(const FwdArgs a) {
  __shared__ float2 red[2][32];
  const int threads = G != 0 ? G : blockDim.x;
  const int t = G != 0 ? threadIdx.x % (G != 0 ? G : 1) : threadIdx.x;
  const int64_t row = G != 0 ? blockIdx.x * static_cast<int64_t>(256 / (G != 0 ? G : 1)) +
                                   threadIdx.x / (G != 0 ? G : 1)
                             : blockIdx.x;
  const bool there = G == 0 || row < a.rows;
  grid_dependency_wait();
  grid_dependents_launch();
  float v[NV][kVec];
  load_row<kAligned>(static_cast<const T*>(a.x) + (there ? row : 0) * a.ldx, there ? a.D : 0, t,
                     threads, v);
  float s = 0.0f, unused = 0.0f;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int k = 0; k < kVec; ++k) s += v[j][k];
  row_sum<G>(s, unused, red[0]);
  const float mean = s / static_cast<float>(a.D);
  float q = 0.0f;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      v[j][k] -= mean;
      if (slot<kAligned>(j, k, t, threads) < a.D) q = fmaf(v[j][k], v[j][k], q);
    }
  row_sum<G>(q, unused, red[1]);
  const float rstd = 1.0f / sqrtf(q / static_cast<float>(a.D) + a.eps);
  if (!there) return;
  if (t == 0) {
    if (a.mean != nullptr) a.mean[row] = mean;
    if (a.rstd != nullptr) a.rstd[row] = rstd;
  }
  float w[NV][kVec];
  load_weight<kAligned>(a.gamma, a.w_bf16, 1.0f, a.D, t, threads, w);
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int k = 0; k < kVec; ++k) v[j][k] *= rstd * w[j][k];
  if (a.beta != nullptr) {
    load_weight<kAligned>(a.beta, a.w_bf16, 0.0f, a.D, t, threads, w);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < kVec; ++k) v[j][k] += w[j][k];
  }
  store_row<kAligned>(a.y, a.y_bf16, row * a.ldy, a.D, t, threads, v);
}

// Rows too long for registers: the row is read three times, the second and
// third time from the caches.
template <typename T>
__global__ void __launch_bounds__(1024) layernorm_fwd_long_kernel(const FwdArgs a) {
  __shared__ float2 red[2][32];
  grid_dependency_wait();
  grid_dependents_launch();
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  float s = 0.0f, unused = 0.0f;
  for (int e = threadIdx.x; e < a.D; e += blockDim.x) s += static_cast<float>(x[e]);
  row_sum<0>(s, unused, red[0]);
  const float mean = s / static_cast<float>(a.D);
  float q = 0.0f;
  for (int e = threadIdx.x; e < a.D; e += blockDim.x) {
    const float d = static_cast<float>(x[e]) - mean;
    q = fmaf(d, d, q);
  }
  row_sum<0>(q, unused, red[1]);
  const float rstd = 1.0f / sqrtf(q / static_cast<float>(a.D) + a.eps);
  if (threadIdx.x == 0) {
    if (a.mean != nullptr) a.mean[row] = mean;
    if (a.rstd != nullptr) a.rstd[row] = rstd;
  }
  const auto weight = [&](const void* w, int e, float none) {
    return w == nullptr ? none
           : a.w_bf16   ? __bfloat162float(static_cast<const __nv_bfloat16*>(w)[e])
                        : static_cast<const float*>(w)[e];
  };
  for (int e = threadIdx.x; e < a.D; e += blockDim.x) {
    const float y = (static_cast<float>(x[e]) - mean) * (rstd * weight(a.gamma, e, 1.0f)) +
                    weight(a.beta, e, 0.0f);
    if (a.y_bf16)
      static_cast<__nv_bfloat16*>(a.y)[row * a.ldy + e] = __float2bfloat16_rn(y);
    else
      static_cast<float*>(a.y)[row * a.ldy + e] = y;
  }
}

struct BwdArgs {
  const void *x, *dy, *dres;
  void* dx;
  const void* gamma;
  const float *mean, *rstd;
  float* part;   // [gridDim.x][2][D]: sums of dy xh, then of dy
  int64_t rows, ldx, lddy, lddres, lddx;
  int D;
  int x_bf16, w_bf16;
};

// The rows blockIdx.x, blockIdx.x + gridDim.x, ... (times the groups of a
// block); a thread keeps the sums of its own columns over all of them.
template <typename T, typename DY, bool kAligned, int G, int NV>
__global__ void __launch_bounds__(G != 0 ? 256 : 512) layernorm_bwd_kernel(const BwdArgs a) {
  extern __shared__ float sums[];   // G != 0: [2][D]
  __shared__ float2 red[2][32];
  constexpr int kGroups = G != 0 ? 256 / (G != 0 ? G : 1) : 1;
  const int threads = G != 0 ? G : blockDim.x;
  const int t = G != 0 ? threadIdx.x % (G != 0 ? G : 1) : threadIdx.x;
  const int group = G != 0 ? threadIdx.x / (G != 0 ? G : 1) : 0;
  grid_dependency_wait();
  grid_dependents_launch();
  float gamma[NV][kVec], dg[NV][kVec], db[NV][kVec];
  load_weight<kAligned>(a.gamma, a.w_bf16, 1.0f, a.D, t, threads, gamma);
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int k = 0; k < kVec; ++k) dg[j][k] = db[j][k] = 0.0f;
  const float inv_d = 1.0f / static_cast<float>(a.D);
  int turn = 0;
  for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * kGroups; r0 < a.rows;
       r0 += static_cast<int64_t>(gridDim.x) * kGroups, turn ^= 1) {
    const int64_t row = r0 + group;
    const bool there = row < a.rows;
    const int64_t at = there ? row : 0;
    const int n = there ? a.D : 0;
    float xh[NV][kVec], dy[NV][kVec];
    load_row<kAligned>(static_cast<const T*>(a.x) + at * a.ldx, n, t, threads, xh);
    load_row<kAligned>(static_cast<const DY*>(a.dy) + at * a.lddy, n, t, threads, dy);
    const float mean = a.mean[at], rstd = a.rstd[at];
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < kVec; ++k) {
        // what lies past the row's end takes no part, whatever mean and rstd are
        const bool in = slot<kAligned>(j, k, t, threads) < n;
        xh[j][k] = in ? (xh[j][k] - mean) * rstd : 0.0f;
        dg[j][k] = fmaf(dy[j][k], xh[j][k], dg[j][k]);
        db[j][k] += dy[j][k];
        const float w = dy[j][k] * gamma[j][k];
        s1 += w;
        s2 = fmaf(w, xh[j][k], s2);
      }
    row_sum<G>(s1, s2, red[turn]);
    s1 *= inv_d;
    s2 *= inv_d;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < kVec; ++k)
        xh[j][k] = rstd * (dy[j][k] * gamma[j][k] - s1 - xh[j][k] * s2);
    if (a.dres != nullptr) {
      load_row<kAligned>(static_cast<const T*>(a.dres) + at * a.lddres, n, t, threads, dy);
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int k = 0; k < kVec; ++k) xh[j][k] += dy[j][k];
    }
    if (there) store_row<kAligned>(a.dx, a.x_bf16, row * a.lddx, a.D, t, threads, xh);
  }
  if (a.part == nullptr) return;
  float* part = a.part + static_cast<int64_t>(blockIdx.x) * 2 * a.D;
  if constexpr (G == 0) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < kVec; ++k) {
        const int e = slot<kAligned>(j, k, t, threads);
        if (e < a.D) {
          part[e] = dg[j][k];
          part[a.D + e] = db[j][k];
        }
      }
  } else {
    // the groups of the block one after another
    for (int g = 0; g < kGroups; ++g) {
      if (group == g) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int k = 0; k < kVec; ++k) {
            const int e = slot<kAligned>(j, k, t, threads);
            if (e < a.D) {
              sums[e] = g == 0 ? dg[j][k] : sums[e] + dg[j][k];
              sums[a.D + e] = g == 0 ? db[j][k] : sums[a.D + e] + db[j][k];
            }
          }
      }
      __syncthreads();
    }
    for (int e = threadIdx.x; e < 2 * a.D; e += blockDim.x) part[e] = sums[e];
  }
}

// Rows too long for registers: dx of one row per block, and the columns' sums
// over a slice of the rows in a kernel of their own.
template <typename T, typename DY>
__global__ void __launch_bounds__(1024) layernorm_bwd_long_kernel(const BwdArgs a) {
  __shared__ float2 red[32];
  grid_dependency_wait();
  grid_dependents_launch();
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  const DY* dy = static_cast<const DY*>(a.dy) + row * a.lddy;
  const float mean = a.mean[row], rstd = a.rstd[row];
  const auto gamma = [&](int e) {
    return a.gamma == nullptr ? 1.0f
           : a.w_bf16         ? __bfloat162float(static_cast<const __nv_bfloat16*>(a.gamma)[e])
                              : static_cast<const float*>(a.gamma)[e];
  };
  float s1 = 0.0f, s2 = 0.0f;
  for (int e = threadIdx.x; e < a.D; e += blockDim.x) {
    const float w = static_cast<float>(dy[e]) * gamma(e);
    s1 += w;
    s2 = fmaf(w, (static_cast<float>(x[e]) - mean) * rstd, s2);
  }
  row_sum<0>(s1, s2, red);
  s1 /= static_cast<float>(a.D);
  s2 /= static_cast<float>(a.D);
  for (int e = threadIdx.x; e < a.D; e += blockDim.x) {
    float d = rstd * (static_cast<float>(dy[e]) * gamma(e) - s1 -
                      (static_cast<float>(x[e]) - mean) * rstd * s2);
    if (a.dres != nullptr) d += static_cast<float>(static_cast<const T*>(a.dres)[row * a.lddres + e]);
    static_cast<T*>(a.dx)[row * a.lddx + e] = static_cast<T>(d);
  }
}

template <typename T, typename DY>
__global__ void __launch_bounds__(256) layernorm_bwd_columns_kernel(const BwdArgs a,
                                                                    int64_t rows_per_slice) {
  grid_dependency_wait();
  grid_dependents_launch();
  const int e = blockIdx.y * 256 + threadIdx.x;
  if (e >= a.D) return;
  const int64_t beg = blockIdx.x * rows_per_slice;
  const int64_t end = beg + rows_per_slice < a.rows ? beg + rows_per_slice : a.rows;
  float dg = 0.0f, db = 0.0f;
  for (int64_t r = beg; r < end; ++r) {
    const float dy = static_cast<float>(static_cast<const DY*>(a.dy)[r * a.lddy + e]);
    const float x = static_cast<float>(static_cast<const T*>(a.x)[r * a.ldx + e]);
    dg = fmaf(dy, (x - a.mean[r]) * a.rstd[r], dg);
    db += dy;
  }
  float* part = a.part + static_cast<int64_t>(blockIdx.x) * 2 * a.D;
  part[e] = dg;
  part[a.D + e] = db;
}

// dgamma, dbeta = the partial sums of `slices` blocks, added by eight threads
// a column (thread row q takes slices q, q + 8, ...) and then in order.
__global__ void __launch_bounds__(256) layernorm_bwd_reduce_kernel(const float* part, int slices,
                                                                   int D, float* dgamma,
                                                                   float* dbeta) {
  __shared__ float sum[8][33];
  grid_dependency_wait();
  grid_dependents_launch();
  const int c = threadIdx.x & 31, q = threadIdx.x >> 5;
  const int64_t col = static_cast<int64_t>(blockIdx.x) * 32 + c;
  float s = 0.0f;
  if (col < 2ll * D)
    for (int i = q; i < slices; i += 8) s += part[2ll * D * i + col];
  sum[q][c] = s;
  __syncthreads();
  if (q == 0 && col < 2ll * D) {
    for (int i = 1; i < 8; ++i) s += sum[i][c];
    float* out = col < D ? dgamma : dbeta;
    if (out != nullptr) out[col < D ? col : col - D] = s;
  }
}

// How a row is spread: lanes per row (0: the block), vectors and threads.
struct Spread {
  int G, NV, threads;
  bool fits;
};

Spread spread(int64_t D, int max_threads, int max_nv, bool wide) {
  const int64_t u = (D + kVec - 1) / kVec;
  if (u <= 8) return {8, 1, 256, true};
  if (u <= 16) return {16, 1, 256, true};
  if (u <= 32) return {32, 1, 256, true};
  if (u <= 64 && max_nv >= 2) return {32, 2, 256, true};
  int nv = wide ? 1 : max_nv;
  while (nv < max_nv && u > static_cast<int64_t>(nv) * max_threads) nv *= 2;
  while (nv > 1 && (u + nv - 1) / nv < 64) nv /= 2;
  const int64_t threads = ((u + nv - 1) / nv + 31) / 32 * 32;
  return {0, nv, static_cast<int>(threads < max_threads ? threads : max_threads),
          threads <= max_threads};
}

constexpr int64_t kFwdLongest = 1024 * 4 * kVec;
constexpr int64_t kBwdLongest = 512 * 2 * kVec;

template <typename T, bool kAligned>
cudaError_t launch_fwd(const FwdArgs& a, const Spread& sp, cudaStream_t s) {
  const auto go = [&](auto kernel, int64_t per_block) {
    const unsigned grid = static_cast<unsigned>((a.rows + per_block - 1) / per_block);
    return launch_dependent(kernel, dim3(grid), dim3(sp.threads), 0, s, a);
  };
  if (sp.G == 8) return go(layernorm_fwd_kernel<T, kAligned, 8, 1>, 32);
  if (sp.G == 16) return go(layernorm_fwd_kernel<T, kAligned, 16, 1>, 16);
  if (sp.G == 32 && sp.NV == 1) return go(layernorm_fwd_kernel<T, kAligned, 32, 1>, 8);
  if (sp.G == 32) return go(layernorm_fwd_kernel<T, kAligned, 32, 2>, 8);
  if (sp.NV == 1) return go(layernorm_fwd_kernel<T, kAligned, 0, 1>, 1);
  if (sp.NV == 2) return go(layernorm_fwd_kernel<T, kAligned, 0, 2>, 1);
  return go(layernorm_fwd_kernel<T, kAligned, 0, 4>, 1);
}

template <typename T, typename DY, bool kAligned>
cudaError_t launch_bwd(const BwdArgs& a, const Spread& sp, int grid, cudaStream_t s) {
  const auto go = [&](auto kernel) {
    const size_t smem = sp.G != 0 ? sizeof(float) * 2 * static_cast<size_t>(a.D) : 0;
    return launch_dependent(kernel, dim3(grid), dim3(sp.threads), smem, s, a);
  };
  if (sp.G == 8) return go(layernorm_bwd_kernel<T, DY, kAligned, 8, 1>);
  if (sp.G == 16) return go(layernorm_bwd_kernel<T, DY, kAligned, 16, 1>);
  if (sp.G == 32 && sp.NV == 1) return go(layernorm_bwd_kernel<T, DY, kAligned, 32, 1>);
  if (sp.G == 32) return go(layernorm_bwd_kernel<T, DY, kAligned, 32, 2>);
  if (sp.NV == 1) return go(layernorm_bwd_kernel<T, DY, kAligned, 0, 1>);
  return go(layernorm_bwd_kernel<T, DY, kAligned, 0, 2>);
}

// Blocks of the backward pass, which each leave one row of partial sums:
// several resident on every SM, and at least four rows for each of them.
int bwd_slices(int64_t rows, int64_t D) {
  const Spread sp = spread(D, 512, 2, false);
  const int64_t groups = !sp.fits ? 1 : sp.G != 0 ? 256 / sp.G : 1;
  const int per_sm = !sp.fits ? 4 : 1024 / sp.threads < 8 ? 1024 / sp.threads : 8;
  int64_t n = static_cast<int64_t>(device_sm_count()) * per_sm;
  const int64_t most = (rows + 4 * groups - 1) / (4 * groups);
  if (n > most) n = most;
  return static_cast<int>(n < 1 ? 1 : n);
}

bool aligned_rows(const void* p, int64_t ld, size_t elem) {
  return is_aligned(p, 16) && (static_cast<size_t>(ld) * elem) % 16 == 0;
}

}  // namespace

size_t layernorm_bwd_workspace_bytes(int64_t rows, int64_t D) {
  return sizeof(float) * 2 * static_cast<size_t>(D) * static_cast<size_t>(bwd_slices(rows, D));
}

tbn_status launch_layernorm_fwd(const LayerNormProblem& p, cudaStream_t s) {
  if (p.rows == 0) return TBN_OK;
  FwdArgs a{p.x, p.y, p.gamma, p.beta, p.mean_out, p.rstd_out, p.rows, p.ldx, p.ldy,
            static_cast<int>(p.D), p.eps, p.ydt == TBN_BF16, p.wdt == TBN_BF16};
  cudaError_t e;
  if (p.D > kFwdLongest) {
    auto* kernel = p.xdt == TBN_BF16 ? layernorm_fwd_long_kernel<__nv_bfloat16>
                                     : layernorm_fwd_long_kernel<float>;
    e = launch_dependent(kernel, dim3(static_cast<unsigned>(p.rows)), dim3(1024), 0, s, a);
  } else {
    const bool al = p.D % kVec == 0 && aligned_rows(p.x, p.ldx, dtype_size(p.xdt)) &&
                    aligned_rows(p.y, p.ldy, dtype_size(p.ydt)) && is_aligned(p.gamma, 16) &&
                    is_aligned(p.beta, 16);
    const Spread sp = spread(p.D, 1024, 4, p.rows < 2 * device_sm_count());
    if (p.xdt == TBN_BF16)
      e = al ? launch_fwd<__nv_bfloat16, true>(a, sp, s) : launch_fwd<__nv_bfloat16, false>(a, sp, s);
    else
      e = al ? launch_fwd<float, true>(a, sp, s) : launch_fwd<float, false>(a, sp, s);
  }
  return e == cudaSuccess ? TBN_OK : cuda_fail(e, "layernorm_fwd_kernel");
}

tbn_status launch_layernorm_bwd(const LayerNormProblem& p, cudaStream_t s) {
  const bool sums = p.dgamma != nullptr || p.dbeta != nullptr;
  const int slices = bwd_slices(p.rows, p.D);
  const bool x16 = p.xdt == TBN_BF16, dy16 = p.ydt == TBN_BF16;
  BwdArgs a{p.x, p.dy, p.dres, p.dx, p.gamma, p.mean, p.rstd, sums ? p.part : nullptr, p.rows,
            p.ldx, p.ldy, p.lddres, p.lddx, static_cast<int>(p.D), x16, p.wdt == TBN_BF16};
  cudaError_t e = cudaSuccess;
  using B = __nv_bfloat16;
  if (p.D > kBwdLongest) {
    auto* rows = x16 ? layernorm_bwd_long_kernel<B, B>
                     : dy16 ? layernorm_bwd_long_kernel<float, B> : layernorm_bwd_long_kernel<float, float>;
    auto* columns = x16 ? layernorm_bwd_columns_kernel<B, B>
                        : dy16 ? layernorm_bwd_columns_kernel<float, B>
                               : layernorm_bwd_columns_kernel<float, float>;
    // the columns first: dx may be written over x, dy or dres
    if (sums)
      e = launch_dependent(columns, dim3(slices, static_cast<unsigned>((p.D + 255) / 256)), dim3(256),
                           0, s, a, (p.rows + slices - 1) / slices);
    if (e == cudaSuccess && p.rows > 0)
      e = launch_dependent(rows, dim3(static_cast<unsigned>(p.rows)), dim3(1024), 0, s, a);
  } else {
    const bool al = p.D % kVec == 0 && aligned_rows(p.x, p.ldx, dtype_size(p.xdt)) &&
                    aligned_rows(p.dy, p.ldy, dtype_size(p.ydt)) &&
                    aligned_rows(p.dx, p.lddx, dtype_size(p.xdt)) &&
                    (p.dres == nullptr || aligned_rows(p.dres, p.lddres, dtype_size(p.xdt))) &&
                    is_aligned(p.gamma, 16);
    const Spread sp = spread(p.D, 512, 2, false);
    if (x16)
      e = al ? launch_bwd<B, B, true>(a, sp, slices, s) : launch_bwd<B, B, false>(a, sp, slices, s);
    else if (dy16)
      e = al ? launch_bwd<float, B, true>(a, sp, slices, s)
             : launch_bwd<float, B, false>(a, sp, slices, s);
    else
      e = al ? launch_bwd<float, float, true>(a, sp, slices, s)
             : launch_bwd<float, float, false>(a, sp, slices, s);
  }
  if (e != cudaSuccess) return cuda_fail(e, "layernorm_bwd_kernel");
  if (!sums) return TBN_OK;
  e = launch_dependent(layernorm_bwd_reduce_kernel, dim3(static_cast<unsigned>((2 * p.D + 31) / 32)),
                       dim3(256), 0, s, a.part, slices, static_cast<int>(p.D), p.dgamma, p.dbeta);
  return e == cudaSuccess ? TBN_OK : cuda_fail(e, "layernorm_bwd_reduce_kernel");
}

}  // namespace tbn
