// Linear cross entropy of small problems (heads of a few hundred classes, a few hundred rows): fp32 arithmetic on the CUDA
// cores, two launches for loss and gradients.  At these sizes the tensor-core path is all launch and pipeline latency
// (128 x 512 x 100 fp32, loss and gradients: 47 us on the device and 51 us a call there, 29 and 30 us here).
//
// Rows kernel: a block takes kR tokens from logits to dX: z = x W^T, softmax statistics, loss, dz (kept in shared memory,
// written out for dW), dX = dz W.  W is read from the L2 twice per block, and those reads
// (52 MB at that size) and their latency bound it.  Gradient kernel: dW = dz^T X, one 32 x 32 tile per
// block, the contraction over all tokens.
#pragma once

#include "hdqt_types.cuh"

namespace hdqt {

namespace {

constexpr int kSmallThreads = 1024;          // a block per SM: all of its latency hiding comes from its own warps
constexpr int kSmallWarps = kSmallThreads / 32;
constexpr int kGradThreads = 256;

struct SmallParams {
  const void* x;
  const void* w;
  const int64_t* labels;
  const float* g;             // gradient of the loss: [tokens] (g_rows) or one value; null = 1
  const float* lse_in;        // backward: statistics of the forward call; null = formed here
  float* lse;                 // null: not written
  float* loss_rows;           // null: not written
  float* dz;                  // [tokens, classes] workspace for dW; null = not needed
  void* dx;                   // null = not needed
  void* dw;
  float* loss;                // reduced loss, written by the gradient kernel; null = not written
  int32_t* dev_status;
  int64_t ignore, ld_x, ld_w, ld_dx, ld_dw;
  int32_t tokens, features, classes;
  int32_t w_is_cd, g_rows, mean;
};

template <typename T>
__device__ __forceinline__ float ldf(const T* p) { return to_f32(*p); }

// out(r, n) = sum_k in[r][k] M(n, k), M stored [k][n]: a lane per kV neighbouring n, the warps share n in tiles of 32 kV
// (and k in slices where there are fewer tiles than warps).  red: kSmallThreads * kR floats.  All threads take part.
template <typename T, int kR, int kV, typename F>
__device__ __forceinline__ void rows_by_columns(const float* in, const T* m, int64_t ld, int N, int K, float* red, F&& out) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int tiles = (N + 32 * kV - 1) / (32 * kV);
  const int slices = kV == 1 && tiles < kSmallWarps ? kSmallWarps / tiles : 1;
  const int per = (K + slices - 1) / slices;
  const int step = slices > 1 ? tiles : kSmallWarps;
  for (int t0 = 0; t0 < tiles; t0 += step) {         // (one round where the contraction is sliced)
    const int slice = slices > 1 ? warp / tiles : 0;
    const int tile = slices > 1 ? warp - slice * tiles : t0 + warp;
    const int n = (tile * 32 + lane) * kV;
    float acc[kR][kV];
#pragma unroll
    for (int r = 0; r < kR; ++r)
#pragma unroll
      for (int j = 0; j < kV; ++j) acc[r][j] = 0.0f;
    const int k1 = min(K, (slice + 1) * per);
    if (slice < slices && tile < tiles && n < N) {   // (kV > 1: N is a multiple of kV)
      const T* p = m + n;
#pragma unroll(kV == 1 ? 32 : 16)
      for (int k = slice * per; k < k1; ++k) {
        float v[kV];
        unpack(*reinterpret_cast<const Vec<T, kV>*>(p + k * ld), v);
#pragma unroll
        for (int r = 0; r < kR; ++r)
#pragma unroll
          for (int j = 0; j < kV; ++j) acc[r][j] = fmaf(in[r * K + k], v[j], acc[r][j]);
      }
      if (slices == 1) {
#pragma unroll
        for (int r = 0; r < kR; ++r)
#pragma unroll
          for (int j = 0; j < kV; ++j) out(r, n + j, acc[r][j]);
      }
    }
    if (slices > 1) {
#pragma unroll
      for (int r = 0; r < kR; ++r) red[r * kSmallThreads + threadIdx.x] = acc[r][0];
      __syncthreads();
      if (slice == 0 && n < N) {
#pragma unroll
        for (int r = 0; r < kR; ++r) {
          float s = red[r * kSmallThreads + threadIdx.x];
          for (int i = 1; i < slices; ++i) s += red[r * kSmallThreads + threadIdx.x + i * tiles * 32];
          out(r, n, s);
        }
      }
      __syncthreads();
    }
  }
}

// the same with M stored [n][k]: a warp per n (kN at a time), lanes along k, kV neighbouring k per access
template <typename T, int kR, int kV, int kN, typename F>
__device__ __forceinline__ void rows_by_rows(const float* in, const T* m, int64_t ld, int N, int K, F&& out) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int n0 = warp; n0 < N; n0 += kN * kSmallWarps) {
    const T* p[kN];
    float a[kN][kR];
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      p[i] = m + (int64_t)min(n0 + i * kSmallWarps, N - 1) * ld;
#pragma unroll
      for (int r = 0; r < kR; ++r) a[i][r] = 0.0f;
    }
#pragma unroll 4
    for (int k = lane * kV; k < K; k += 32 * kV) {   // (kV > 1: K is a multiple of kV)
      float v[kN][kV];
#pragma unroll
      for (int i = 0; i < kN; ++i) unpack(*reinterpret_cast<const Vec<T, kV>*>(p[i] + k), v[i]);
#pragma unroll
      for (int r = 0; r < kR; ++r)
#pragma unroll
        for (int j = 0; j < kV; ++j) {
          const float x = in[r * K + k + j];
#pragma unroll
          for (int i = 0; i < kN; ++i) a[i][r] = fmaf(x, v[i][j], a[i][r]);
        }
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1)
#pragma unroll
      for (int i = 0; i < kN; ++i)
#pragma unroll
        for (int r = 0; r < kR; ++r) a[i][r] += __shfl_xor_sync(0xFFFFFFFFu, a[i][r], d);
    // lane i * kR + r writes result (i, r)
#pragma unroll
    for (int i = 0; i < kN; ++i)
#pragma unroll
      for (int r = 0; r < kR; ++r)
        if (lane == i * kR + r && n0 + i * kSmallWarps < N) out(r, n0 + i * kSmallWarps, a[i][r]);
  }
}

// by sizes and alignment: as many n per warp as leave work for every warp, four elements per access where rows allow it
template <typename T, int kR, typename F>
__device__ __forceinline__ void by_rows(const float* in, const T* m, int64_t ld, int N, int K, F&& out) {
  const bool wide = ((reinterpret_cast<uintptr_t>(m) | (uintptr_t)(ld * sizeof(T)) | (uintptr_t)(K * sizeof(T))) & (4 * sizeof(T) - 1)) == 0;
  if (wide && N > 4 * kSmallWarps) rows_by_rows<T, kR, 4, kR == 1 ? 8 : 4>(in, m, ld, N, K, out);
  else if (wide) rows_by_rows<T, kR, 4, 2>(in, m, ld, N, K, out);
  else if (N > 4 * kSmallWarps) rows_by_rows<T, kR, 1, kR == 1 ? 8 : 4>(in, m, ld, N, K, out);
  else rows_by_rows<T, kR, 1, 2>(in, m, ld, N, K, out);
}
template <typename T, int kR, typename F>
__device__ __forceinline__ void by_columns(const float* in, const T* m, int64_t ld, int N, int K, float* red, F&& out) {
  const bool wide = ((reinterpret_cast<uintptr_t>(m) | (uintptr_t)(ld * sizeof(T)) | (uintptr_t)(N * sizeof(T))) & (4 * sizeof(T) - 1)) == 0;
  if (wide && N >= 64 * kSmallWarps) rows_by_columns<T, kR, 4>(in, m, ld, N, K, red, out);
  else rows_by_columns<T, kR, 1>(in, m, ld, N, K, red, out);
}

template <typename T, int kR>
__global__ void __launch_bounds__(kSmallThreads) xent_small_rows_kernel(const __grid_constant__ SmallParams p) {
  extern __shared__ float sm[];
  __shared__ int s_kept;
  chain_wait();
  float* xs = sm;                              // [kR][features]
  float* zs = xs + kR * p.features;            // [kR][classes]
  float* red = zs + kR * p.classes;            // [kR][kSmallThreads]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int t0 = blockIdx.x * kR;
  const int D = p.features, V = p.classes;
  const T* x = reinterpret_cast<const T*>(p.x);
  const T* w = reinterpret_cast<const T*>(p.w);
  if (threadIdx.x == 0) s_kept = 0;
  for (int i = threadIdx.x; i < kR * D; i += kSmallThreads) {
    const int r = i / D;
    xs[i] = t0 + r < p.tokens ? ldf(x + (int64_t)(t0 + r) * p.ld_x + (i - r * D)) : 0.0f;
  }
  int kept = 0;                                // every block counts the kept tokens for itself
  if (p.mean)
    for (int t = threadIdx.x; t < p.tokens; t += kSmallThreads) kept += p.labels[t] != p.ignore;
  __syncthreads();
  kept = __reduce_add_sync(0xFFFFFFFFu, kept);
  if (lane == 0 && kept) atomicAdd(&s_kept, kept);
  auto to_z = [&](int r, int n, float v) { zs[r * V + n] = v; };
  if (p.w_is_cd) by_rows<T, kR>(xs, w, p.ld_w, V, D, to_z);
  else by_columns<T, kR>(xs, w, p.ld_w, V, D, red, to_z);
  __syncthreads();
  const float scale = p.mean ? 1.0f / (float)s_kept : 1.0f;
  if (warp < kR && t0 + warp < p.tokens) {     // a warp per row
    const int t = t0 + warp;
    float* z = zs + warp * V;
    const int64_t l = p.labels[t];
    const bool ignored = l == p.ignore, valid = !ignored && l >= 0 && l < V;
    float lse;
    if (p.lse_in != nullptr) {
      lse = p.lse_in[t];
    } else {
      float m = -3.402823466e38f, s = 0.0f;
      for (int v = lane; v < V; v += 32) m = fmaxf(m, z[v]);
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
      for (int v = lane; v < V; v += 32) s += ex2((z[v] - m) * kLog2e);
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
      lse = m + logf(s);
    }
    if (lane == 0) {
      if (!ignored && !valid) report_status(p.dev_status, HDQT_ERR_INVALID_ARG);
      if (p.lse != nullptr) p.lse[t] = lse;
      if (p.loss_rows != nullptr) p.loss_rows[t] = valid ? lse - z[l] : ignored ? 0.0f : NAN;
    }
    if constexpr (kR > 1) return;              // (two tokens per block: the loss alone)
    __syncwarp();
    if (p.dz != nullptr || p.dx != nullptr) {
      const float g = (p.g != nullptr ? p.g[p.g_rows ? t : 0] : 1.0f) * scale;
      for (int v = lane; v < V; v += 32) {
        const float e = valid ? g * (ex2((z[v] - lse) * kLog2e) - (v == l ? 1.0f : 0.0f)) : 0.0f;
        z[v] = e;
        if (p.dz != nullptr) p.dz[(int64_t)t * V + v] = e;
      }
    }
  }
  if constexpr (kR > 1) return;
  if (p.dx == nullptr) return;
  __syncthreads();
  T* dx = reinterpret_cast<T*>(p.dx);
  auto to_dx = [&](int r, int n, float v) {
    if (t0 + r < p.tokens) dx[(int64_t)(t0 + r) * p.ld_dx + n] = from_f32<T>(v);
  };
  if (p.w_is_cd) by_columns<T, kR>(zs, w, p.ld_w, D, V, red, to_dx);
  else by_rows<T, kR>(zs, w, p.ld_w, D, V, to_dx);
}

// dW[v, d] = sum_t dz[t, v] x[t, d] (stored [classes, features] or transposed), 32 classes x 32 features per block; the
// blocks of the last blockIdx.x reduce the rows' losses instead
template <typename T>
__global__ void __launch_bounds__(kGradThreads) xent_small_grad_kernel(const __grid_constant__ SmallParams p) {
  constexpr int kT = 64;                       // tokens per step
  __shared__ float s_dz[kT][32], s_x[kT][32];
  __shared__ double s_sum[(kGradThreads / 32)];
  __shared__ int s_kept[(kGradThreads / 32)];
  chain_wait();
  const T* x = reinterpret_cast<const T*>(p.x);
  if (blockIdx.x == gridDim.x - 1) {
    if (blockIdx.y != 0 || p.loss == nullptr) return;
    double s = 0.0;
    int kept = 0;
    for (int t = threadIdx.x; t < p.tokens; t += kGradThreads) {
      s += (double)p.loss_rows[t];
      kept += p.labels[t] != p.ignore;
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    kept = __reduce_add_sync(0xFFFFFFFFu, kept);
    if ((threadIdx.x & 31) == 0) { s_sum[threadIdx.x >> 5] = s; s_kept[threadIdx.x >> 5] = kept; }
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 1; w < (kGradThreads / 32); ++w) { s += s_sum[w]; kept += s_kept[w]; }
      p.loss[0] = (float)(p.mean ? s * (double)(1.0f / (float)kept) : s);
    }
    return;
  }
  const int v0 = blockIdx.y * 32, d0 = blockIdx.x * 32;
  // 2 classes x 2 features per thread; the contiguous index of dW runs along the lanes
  const int tv = p.w_is_cd ? threadIdx.x >> 4 : threadIdx.x & 15, td = p.w_is_cd ? threadIdx.x & 15 : threadIdx.x >> 4;
  float acc[2][2] = {};
  for (int t0 = 0; t0 < p.tokens; t0 += kT) {
#pragma unroll
    for (int i = threadIdx.x; i < kT * 32; i += kGradThreads) {
      const int t = t0 + (i >> 5), v = v0 + (i & 31);
      s_dz[i >> 5][i & 31] = t < p.tokens && v < p.classes ? p.dz[(int64_t)t * p.classes + v] : 0.0f;
    }
#pragma unroll
    for (int i = threadIdx.x; i < kT * 32; i += kGradThreads) {
      const int t = t0 + (i >> 5), d = d0 + (i & 31);
      s_x[i >> 5][i & 31] = t < p.tokens && d < p.features ? ldf(x + (int64_t)t * p.ld_x + d) : 0.0f;
    }
    __syncthreads();
#pragma unroll 8
    for (int t = 0; t < kT; ++t) {
      const float a0 = s_dz[t][tv], a1 = s_dz[t][tv + 16];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float b = s_x[t][td + 16 * j];
        acc[0][j] = fmaf(a0, b, acc[0][j]);
        acc[1][j] = fmaf(a1, b, acc[1][j]);
      }
    }
    __syncthreads();
  }
  T* dw = reinterpret_cast<T*>(p.dw);
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int v = v0 + tv + 16 * i, d = d0 + td + 16 * j;
      if (v < p.classes && d < p.features)
        dw[p.w_is_cd ? (int64_t)v * p.ld_dw + d : (int64_t)d * p.ld_dw + v] = from_f32<T>(acc[i][j]);
    }
}

}  // namespace

}  // namespace hdqt
