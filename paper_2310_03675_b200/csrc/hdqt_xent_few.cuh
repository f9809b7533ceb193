// Linear cross entropy of a few tokens (loss only: scoring one token after the other): reading W once is all there is, so
// the products run on the CUDA cores in fp32 while W streams past, in two launches.
//
// W [classes, features]: a warp takes four classes at a time, lanes along the features.  W [features, classes]: eight lanes
// along 64 classes, 32 slices of the features.  Either way every thread has eight 16-byte loads in flight, and a block keeps a running
// (maximum, sum of exponentials) per token.  X lies in shared memory as fp32.
// 2048 x 32000 bf16, one token (131 MB): XXFEW us, XXFEWBW TB/s; the tensor-core path, whose 256-row blocks would be empty but
// for one row, takes 45 us.
#pragma once

#include "hdqt_types.cuh"

namespace hdqt {

namespace {

constexpr int kFewThreads = 256;
constexpr int kFewWarps = kFewThreads / 32;
constexpr int kFewTokens = 8;            // most tokens
constexpr int kFewSmem = 96 << 10;       // most bytes of X as fp32

struct FewParams {
  const void* x;
  const void* w;
  const int64_t* labels;
  float2* part;                // [tokens, blocks]: (maximum, sum of exponentials)
  float* label_logit;          // [tokens]
  int64_t ld_x, ld_w;
  int32_t tokens, features, classes;
};

struct Running {
  float m = -3.402823466e38f, s = 0.0f;
  __device__ __forceinline__ void add(float om, float os) {
    const float n = fmaxf(m, om);
    s = s * ex2((m - n) * kLog2e) + os * ex2((om - n) * kLog2e);
    m = n;
  }
};

// x[t][k] as fp32 in shared memory, zero for tokens past the end
template <typename T, int kT>
__device__ __forceinline__ void few_load_x(const FewParams& p, float* xs) {
  const T* x = reinterpret_cast<const T*>(p.x);
  for (int t = 0; t < kT; ++t)
    for (int k = threadIdx.x; k < p.features; k += kFewThreads)
      xs[t * p.features + k] = t < p.tokens ? to_f32(x[t * p.ld_x + k]) : 0.0f;
  __syncthreads();
}

// kV elements per access (16 bytes, or one element where rows do not start on 16 bytes)
template <typename T, int kT, int kV>
__global__ void __launch_bounds__(kFewThreads) xent_few_rows_kernel(const __grid_constant__ FewParams p) {
  extern __shared__ __align__(16) float xs[];
  __shared__ float2 s_part[kT][kFewWarps];
  constexpr int kN = 4;                                      // classes at a time
  chain_wait();
  few_load_x<T, kT>(p, xs);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const T* w = reinterpret_cast<const T*>(p.w);
  const int D = p.features;
  int label[kT];
#pragma unroll
  for (int t = 0; t < kT; ++t) {
    const int64_t l = t < p.tokens ? p.labels[t] : -1;
    label[t] = l >= 0 && l < p.classes ? (int)l : -1;
  }
  Running run[kT];
  for (int n0 = (blockIdx.x * kFewWarps + warp) * kN; n0 < p.classes; n0 += gridDim.x * kFewWarps * kN) {
    const T* row[kN];
    float acc[kN][kT];
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      row[i] = w + (int64_t)min(n0 + i, p.classes - 1) * p.ld_w;
#pragma unroll
      for (int t = 0; t < kT; ++t) acc[i][t] = 0.0f;
    }
#pragma unroll 2
    for (int k = lane * kV; k < D; k += 32 * kV) {
      Vec<T, kV> v[kN];
#pragma unroll
      for (int i = 0; i < kN; ++i) v[i] = *reinterpret_cast<const Vec<T, kV>*>(row[i] + k);
#pragma unroll
      for (int t = 0; t < kT; ++t) {
        float xv[kV];
        if constexpr (kV % 4 == 0) {
#pragma unroll
          for (int j = 0; j < kV; j += 4) *reinterpret_cast<float4*>(&xv[j]) = *reinterpret_cast<const float4*>(xs + t * D + k + j);
        } else {
#pragma unroll
          for (int j = 0; j < kV; ++j) xv[j] = xs[t * D + k + j];
        }
#pragma unroll
        for (int i = 0; i < kN; ++i) {
          float f[kV];
          unpack(v[i], f);
#pragma unroll
          for (int j = 0; j < kV; ++j) acc[i][t] = fmaf(f[j], xv[j], acc[i][t]);
        }
      }
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1)
#pragma unroll
      for (int i = 0; i < kN; ++i)
#pragma unroll
        for (int t = 0; t < kT; ++t) acc[i][t] += __shfl_xor_sync(0xFFFFFFFFu, acc[i][t], d);
#pragma unroll
    for (int t = 0; t < kT; ++t) {
      float m = run[t].m;
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        if (n0 + i >= p.classes) acc[i][t] = -INFINITY;
        m = fmaxf(m, acc[i][t]);
        if (lane == 0 && n0 + i == label[t]) p.label_logit[t] = acc[i][t];
      }
      float s = run[t].s * ex2((run[t].m - m) * kLog2e);
#pragma unroll
      for (int i = 0; i < kN; ++i) s += ex2((acc[i][t] - m) * kLog2e);
      run[t].m = m;
      run[t].s = s;
    }
  }
  if (lane == 0) {
#pragma unroll
    for (int t = 0; t < kT; ++t) s_part[t][warp] = make_float2(run[t].m, run[t].s);
  }
  __syncthreads();
  if (threadIdx.x < kT && threadIdx.x < p.tokens) {
    Running r;
    for (int i = 0; i < kFewWarps; ++i) r.add(s_part[threadIdx.x][i].x, s_part[threadIdx.x][i].y);
    p.part[threadIdx.x * gridDim.x + blockIdx.x] = make_float2(r.m, r.s);
  }
}

template <typename T, int kT, int kV>
__global__ void __launch_bounds__(kFewThreads) xent_few_columns_kernel(const __grid_constant__ FewParams p) {
  extern __shared__ __align__(16) float xs[];
  constexpr int kLanes = 8, kTile = kLanes * kV;             // classes of a tile
  constexpr int kSlices = kFewThreads / kLanes;
  __shared__ float s_z[kFewWarps][kT][kTile];
  chain_wait();
  few_load_x<T, kT>(p, xs);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int col = (threadIdx.x % kLanes) * kV, slice = threadIdx.x / kLanes;
  const T* w = reinterpret_cast<const T*>(p.w);
  const int64_t lab = warp < p.tokens ? p.labels[warp] : -1;   // warp t keeps the statistics of token t
  Running run;
  for (int n0 = blockIdx.x * kTile; n0 < p.classes; n0 += gridDim.x * kTile) {
    const int n = n0 + col;
    float acc[kT][kV];
#pragma unroll
    for (int t = 0; t < kT; ++t)
#pragma unroll
      for (int j = 0; j < kV; ++j) acc[t][j] = 0.0f;
    if (n < p.classes) {                                      // (kV > 1: classes is a multiple of kV)
#pragma unroll 8
      for (int k = slice; k < p.features; k += kSlices) {
        float f[kV];
        unpack(*reinterpret_cast<const Vec<T, kV>*>(w + k * p.ld_w + n), f);
#pragma unroll
        for (int t = 0; t < kT; ++t) {
          const float xv = xs[t * p.features + k];
#pragma unroll
          for (int j = 0; j < kV; ++j) acc[t][j] = fmaf(f[j], xv, acc[t][j]);
        }
      }
    }
#pragma unroll
    for (int t = 0; t < kT; ++t)
#pragma unroll
      for (int j = 0; j < kV; ++j) {
#pragma unroll
        for (int d = 16; d >= kLanes; d >>= 1) acc[t][j] += __shfl_xor_sync(0xFFFFFFFFu, acc[t][j], d);
        if (lane < kLanes) s_z[warp][t][col + j] = acc[t][j];
      }
    __syncthreads();
    if (warp < kT && warp < p.tokens) {
      float m = -3.402823466e38f, z[(kTile + 31) / 32];
#pragma unroll
      for (int c = 0; c < (kTile + 31) / 32; ++c) {
        const int i = c * 32 + lane;
        z[c] = -INFINITY;
        if (i < kTile && n0 + i < p.classes) {
          z[c] = 0.0f;
#pragma unroll
          for (int q = 0; q < kFewWarps; ++q) z[c] += s_z[q][warp][i];
          if (n0 + i == lab) p.label_logit[warp] = z[c];
        }
        m = fmaxf(m, z[c]);
      }
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
      float s = 0.0f;
#pragma unroll
      for (int c = 0; c < (kTile + 31) / 32; ++c) s += ex2((z[c] - m) * kLog2e);
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
      run.add(m, s);
    }
    __syncthreads();
  }
  if (warp < kT && warp < p.tokens && lane == 0) p.part[warp * gridDim.x + blockIdx.x] = make_float2(run.m, run.s);
}

// One block: lse and loss of every token (a warp each) and the reduced loss.
__global__ void __launch_bounds__(kFewThreads)
xent_few_join_kernel(const float2* __restrict__ part, int parts, const float* __restrict__ label_logit,
                     const int64_t* __restrict__ labels, int tokens, int classes, int64_t ignore, int reduction,
                     float* __restrict__ lse, float* __restrict__ loss, int32_t* dev_status) {
  __shared__ float s_loss[kFewTokens];
  __shared__ int s_kept[kFewTokens];
  chain_wait();
  const int t = threadIdx.x >> 5, lane = threadIdx.x & 31;
  static_assert(kFewTokens <= kFewWarps, "a warp per token");
  if (t < tokens) {
    Running r;
#pragma unroll 4
    for (int i = lane; i < parts; i += 32) r.add(part[t * parts + i].x, part[t * parts + i].y);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      const float m = __shfl_xor_sync(0xFFFFFFFFu, r.m, d), s = __shfl_xor_sync(0xFFFFFFFFu, r.s, d);
      r.add(m, s);
    }
    if (lane == 0) {
      const int64_t l = labels[t];
      const bool ignored = l == ignore, valid = !ignored && l >= 0 && l < classes;
      const float e = r.m + logf(r.s);
      const float v = valid ? e - label_logit[t] : ignored ? 0.0f : NAN;
      if (!ignored && !valid) report_status(dev_status, HDQT_ERR_INVALID_ARG);
      lse[t] = e;
      if (reduction == HDQT_REDUCE_NONE) loss[t] = v;
      s_loss[t] = v;
      s_kept[t] = !ignored;
    }
  }
  __syncthreads();
  if (threadIdx.x == 0 && reduction != HDQT_REDUCE_NONE) {
    double s = 0.0;
    int kept = 0;
    for (int i = 0; i < tokens; ++i) { s += (double)s_loss[i]; kept += s_kept[i]; }
    loss[0] = (float)(reduction == HDQT_REDUCE_MEAN ? s * (double)(1.0f / (float)kept) : s);
  }
}

}  // namespace

}  // namespace hdqt
