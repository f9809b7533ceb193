// Linear cross entropy of a few tokens: reading W (and writing dW) is all there is, so the products run on the CUDA cores in
// fp32 while W streams past.
//
// Loss only (scoring one token after the other), two launches:
// W [classes, features]: a warp takes four classes at a time, lanes along the features.  W [features, classes]: eight lanes
// along 64 classes, 32 slices of the features.  Either way every thread has eight 16-byte loads in flight, and a block keeps a running
// (maximum, sum of exponentials) per token.  X lies in shared memory as fp32.
// Bound by HBM.  2048 x 32000 bf16, one token (131 MB): 24.5 us, 5.3 TB/s; the tensor-core path, whose 256-row blocks would be
// empty but for one row, takes 45 us.
#pragma once

#include "hdqt_types.cuh"

namespace hdqt {

namespace {

constexpr int kFewThreads = 256;
constexpr int kFewWarps = kFewThreads / 32;
constexpr int kFewTokens = 8;            // most tokens
// Most bytes of X as fp32: four blocks per SM.  Beyond it the tensor-core path (fp32: the streamed products) takes over.  With 100 KB
// and two blocks per SM, 4 x 4096 x 32000 bf16: 90 us (W [classes, features]) and 133, 80 and 78 by the tensor-core path; 8 x 3000 x 32000
// fp32, W [classes, features]: 174, 197 by the streamed products.
constexpr int kFewSmem = 48 << 10;

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

// ---- gradients -----------------------------------------------------------------------------------------------
// logits -> xent_few_stats_kernel -> xent_few_softmax_kernel (lse, loss, dz in fp32) -> dX and dW.  Two kinds of kernel, by how W lies to the product:
//   rows    : out[t, n] = sum_k in[t, k] M[n, k], a warp per four n, lanes along k   (logits of W [classes, features],
//             dX of W [features, classes])
//   columns : out[t, n] = sum_k in[t, k] M[k, n], a thread per kC neighbouring n, walking down k   (the other two); with kOuter
//             it also writes dW[k, n] = sum_t in[t, k] b[t, n], so that dX and dW take one pass over W
// Both cut k into slices (blockIdx.y) with partial results, and take tokens in groups.

struct FewMatrix {
  const void* p;
  int64_t ld;
  int32_t f32;        // element type: fp32, else bf16
};
__device__ __forceinline__ float few_at(const FewMatrix& m, int64_t r, int64_t c) {
  return m.f32 ? reinterpret_cast<const float*>(m.p)[r * m.ld + c]
               : to_f32(reinterpret_cast<const __nv_bfloat16*>(m.p)[r * m.ld + c]);
}

struct FewProduct {
  FewMatrix in, b;             // in [tokens, K]; b [tokens, N] (kOuter)
  const void* m;               // the matrix: [N, K] (rows) or [K, N] (columns)
  int64_t ld_m;
  float* out;                  // [slices, tokens, N]; null: no product (kOuter alone)
  void* outer;                 // [K, N]
  int64_t ld_outer;
  int32_t tokens, N, K, per_slice;
};

constexpr int kFewChunk = 1024;      // k held in shared memory at a time
template <typename T, int kT, int kV>
__global__ void __launch_bounds__(kFewThreads) xent_few_product_rows_kernel(const __grid_constant__ FewProduct p) {
  constexpr int kN = 4;
  __shared__ __align__(16) float s_in[kT][kFewChunk];
  chain_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int groups = (p.tokens + kT - 1) / kT;
  const int t0 = (blockIdx.x % groups) * kT;               // groups of one tile run together: W comes from the L2 for all but one
  const int n0 = ((blockIdx.x / groups) * kFewWarps + warp) * kN;
  const int k0 = blockIdx.y * p.per_slice, k1 = min(p.K, k0 + p.per_slice);
  const T* row[kN];
  float acc[kN][kT];
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    row[i] = reinterpret_cast<const T*>(p.m) + (int64_t)min(n0 + i, p.N - 1) * p.ld_m;
#pragma unroll
    for (int t = 0; t < kT; ++t) acc[i][t] = 0.0f;
  }
  for (int c0 = k0; c0 < k1; c0 += kFewChunk) {
    const int len = min(kFewChunk, k1 - c0);
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kT; ++t)
      for (int k = threadIdx.x; k < len; k += kFewThreads) s_in[t][k] = t0 + t < p.tokens ? few_at(p.in, t0 + t, c0 + k) : 0.0f;
    __syncthreads();
    if (n0 >= p.N) continue;
#pragma unroll 4
    for (int k = lane * kV; k < len; k += 32 * kV) {
      Vec<T, kV> v[kN];
#pragma unroll
      for (int i = 0; i < kN; ++i) v[i] = *reinterpret_cast<const Vec<T, kV>*>(row[i] + c0 + k);
#pragma unroll
      for (int t = 0; t < kT; ++t) {
        float x[kV];
        if constexpr (kV % 4 == 0) {
#pragma unroll
          for (int j = 0; j < kV; j += 4) *reinterpret_cast<float4*>(&x[j]) = *reinterpret_cast<const float4*>(&s_in[t][k + j]);
        } else {
#pragma unroll
          for (int j = 0; j < kV; ++j) x[j] = s_in[t][k + j];
        }
#pragma unroll
        for (int i = 0; i < kN; ++i) {
          float w[kV];
          unpack(v[i], w);
#pragma unroll
          for (int j = 0; j < kV; ++j) acc[i][t] = fmaf(w[j], x[j], acc[i][t]);
        }
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
  for (int i = 0; i < kN; ++i)
#pragma unroll
    for (int t = 0; t < kT; ++t)
      if (lane == (i * kT + t) % 32 && n0 + i < p.N && t0 + t < p.tokens)
        p.out[((int64_t)blockIdx.y * p.tokens + t0 + t) * p.N + n0 + i] = acc[i][t];
}

// Most registers: kT * kC sums and, with kOuter, as many values of b.
template <typename T, int kT, int kC, bool kOuter>
__global__ void __launch_bounds__(kFewThreads) xent_few_columns_product_kernel(const __grid_constant__ FewProduct p) {
  constexpr int kRows = 64;                                 // rows of `in` held in shared memory at a time
  __shared__ __align__(16) float s_in[kRows][kT];
  chain_wait();
  const int groups = (p.tokens + kT - 1) / kT;              // (1 with kOuter)
  const int t0 = (blockIdx.x % groups) * kT;
  const int n = ((blockIdx.x / groups) * blockDim.x + threadIdx.x) * kC;
  const bool on = n < p.N;                                  // (kC > 1: N is a multiple of kC)
  const int k0 = blockIdx.y * p.per_slice, k1 = min(p.K, k0 + p.per_slice);
  const T* m = reinterpret_cast<const T*>(p.m) + n;
  float acc[kT][kC], b[kOuter ? kT : 1][kOuter ? kC : 1];
#pragma unroll
  for (int t = 0; t < kT; ++t)
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      acc[t][c] = 0.0f;
      if constexpr (kOuter) b[t][c] = on && t < p.tokens ? few_at(p.b, t, n + c) : 0.0f;
    }
  for (int r0 = k0; r0 < k1; r0 += kRows) {
    __syncthreads();
    for (int i = threadIdx.x; i < kRows * kT; i += blockDim.x) {
      const int t = i / kRows, r = i - t * kRows;           // neighbouring threads read neighbouring k
      s_in[r][t] = r0 + r < k1 && t0 + t < p.tokens ? few_at(p.in, t0 + t, r0 + r) : 0.0f;
    }
    __syncthreads();
    if (!on) continue;
    const int rows = min(kRows, k1 - r0);
    auto row = [&](int r, const Vec<T, kC>& v) {
      float w[kC], o[kC];
      unpack(v, w);
#pragma unroll
      for (int c = 0; c < kC; ++c) o[c] = 0.0f;
#pragma unroll
      for (int t = 0; t < kT; ++t) {
        const float a = s_in[r][t];
#pragma unroll
        for (int c = 0; c < kC; ++c) {
          acc[t][c] = fmaf(a, w[c], acc[t][c]);
          if constexpr (kOuter) o[c] = fmaf(a, b[t][c], o[c]);
        }
      }
      if constexpr (kOuter) *reinterpret_cast<Vec<T, kC>*>(reinterpret_cast<T*>(p.outer) + (int64_t)(r0 + r) * p.ld_outer + n) = pack<T>(o);
    };
    constexpr int kU = kT * kC >= 64 ? 4 : 8;
    if (kOuter && p.out == nullptr) {                       // dW alone: W is not read
      for (int r = 0; r < rows; ++r) row(r, Vec<T, kC>{});
      continue;
    }
    int r = 0;
    for (; r + kU <= rows; r += kU) {
      Vec<T, kC> v[kU];
#pragma unroll
      for (int u = 0; u < kU; ++u) v[u] = *reinterpret_cast<const Vec<T, kC>*>(m + (int64_t)(r0 + r + u) * p.ld_m);
#pragma unroll
      for (int u = 0; u < kU; ++u) row(r + u, v[u]);
    }
    for (; r < rows; ++r) row(r, *reinterpret_cast<const Vec<T, kC>*>(m + (int64_t)(r0 + r) * p.ld_m));
  }
  if (on && p.out != nullptr) {
#pragma unroll
    for (int t = 0; t < kT; ++t) {
      if (t0 + t >= p.tokens) break;
#pragma unroll
      for (int c = 0; c < kC; ++c) p.out[((int64_t)blockIdx.y * p.tokens + t0 + t) * p.N + n + c] = acc[t][c];
    }
  }
}

// Sums the slices of the logits z [slices, tokens, classes] into the first one; part[token, chunk] = (maximum, sum of
// exponentials) of a chunk of kFewSpan classes, label_logit[token] its label's logit.
constexpr int kFewSpan = 1024;
__global__ void __launch_bounds__(kFewThreads)
xent_few_stats_kernel(float* __restrict__ z, int slices, int tokens, int classes, const int32_t* __restrict__ label,
                      float2* __restrict__ part, float* __restrict__ label_logit) {
  __shared__ float2 s_part[kFewWarps];
  chain_wait();
  const int t = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float* row = z + (int64_t)t * classes;
  const int64_t step = (int64_t)tokens * classes;
  constexpr int kPer = kFewSpan / kFewThreads;
  const int j0 = blockIdx.x * kFewSpan + threadIdx.x;
  float v[kPer], m = -3.402823466e38f;
#pragma unroll
  for (int i = 0; i < kPer; ++i) v[i] = j0 + i * kFewThreads < classes ? row[j0 + i * kFewThreads] : -INFINITY;
#pragma unroll 4
  for (int s = 1; s < slices; ++s) {
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (j0 + i * kFewThreads < classes) v[i] += __ldcg(row + s * step + j0 + i * kFewThreads);
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    m = fmaxf(m, v[i]);
    if (slices > 1 && j0 + i * kFewThreads < classes) row[j0 + i * kFewThreads] = v[i];
    if (j0 + i * kFewThreads == label[t]) label_logit[t] = v[i];
  }
  Running r;
  r.m = m;
#pragma unroll
  for (int i = 0; i < kPer; ++i) r.s += ex2((v[i] - m) * kLog2e);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    const float om = __shfl_xor_sync(0xFFFFFFFFu, r.m, d), os = __shfl_xor_sync(0xFFFFFFFFu, r.s, d);
    r.add(om, os);
  }
  if (lane == 0) s_part[warp] = make_float2(r.m, r.s);
  __syncthreads();
  if (threadIdx.x == 0) {
    r = Running{};
    for (int w = 0; w < kFewWarps; ++w) r.add(s_part[w].x, s_part[w].y);
    part[t * gridDim.x + blockIdx.x] = make_float2(r.m, r.s);
  }
}

// lse (or lse_in) and the loss of a token from its parts, and dz (with its weight) in place of the logits; blocks as above
__global__ void __launch_bounds__(kFewThreads)
xent_few_softmax_kernel(float* __restrict__ z, int classes, const float2* __restrict__ part, const int32_t* __restrict__ label,
                        const float* __restrict__ label_logit, const float* __restrict__ row_weight,
                        const float* __restrict__ scale, const float* __restrict__ lse_in, float* __restrict__ lse,
                        float* __restrict__ loss, int gradients) {
  chain_wait();
  const int t = blockIdx.y, lane = threadIdx.x & 31;
  float* row = z + (int64_t)t * classes;
  const int32_t lab = label[t];
  float l;
  if (lse_in != nullptr) {
    l = lse_in[t];
  } else {                                    // every warp joins the parts for itself
    Running r;
    for (int i = lane; i < gridDim.x; i += 32) r.add(part[t * gridDim.x + i].x, part[t * gridDim.x + i].y);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      const float om = __shfl_xor_sync(0xFFFFFFFFu, r.m, d), os = __shfl_xor_sync(0xFFFFFFFFu, r.s, d);
      r.add(om, os);
    }
    l = r.m + logf(r.s);
    if (threadIdx.x == 0 && blockIdx.x == 0) {
      lse[t] = l;
      loss[t] = lab >= 0 ? l - label_logit[t] : lab == -1 ? 0.0f : NAN;
    }
  }
  if (!gradients) return;
  const bool keep = lab >= 0;
  const float w = !keep ? 0.0f : row_weight != nullptr ? row_weight[t] : *scale;
  const int j0 = blockIdx.x * kFewSpan + threadIdx.x;
  constexpr int kPer = kFewSpan / kFewThreads;
  float v[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) v[i] = j0 + i * kFewThreads < classes ? row[j0 + i * kFewThreads] : 0.0f;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int j = j0 + i * kFewThreads;
    if (j < classes) row[j] = keep ? w * (ex2((v[i] - l) * kLog2e) - (j == lab ? 1.0f : 0.0f)) : 0.0f;
  }
}

// out[t, n] = sum over the slices of [slices, tokens, N]: 16 outputs x 16 slices of threads
template <typename T>
__global__ void __launch_bounds__(256) xent_few_join_slices_kernel(const float* __restrict__ part, int slices, int64_t total,
                                                                   int N, T* __restrict__ out, int64_t ld) {
  __shared__ float s_sum[16][17];
  chain_wait();
  const int c = threadIdx.x & 15, q = threadIdx.x >> 4;
  const int64_t i = (int64_t)blockIdx.x * 16 + c;
  float s = 0.0f;
  if (i < total) {
#pragma unroll 8
    for (int k = q; k < slices; k += 16) s += part[k * total + i];
  }
  s_sum[q][c] = s;
  __syncthreads();
  if (q == 0 && i < total) {
    for (int k = 1; k < 16; ++k) s += s_sum[k][c];
    const int64_t t = i / N;
    out[t * ld + (i - t * N)] = from_f32<T>(s);
  }
}

}  // namespace

}  // namespace hdqt
