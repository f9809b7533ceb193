// Layer norm with an activation over the channels of a row, forward and backward, alone or fused with the dropout and the
// residual add in front of it.
//
//   z = gamma (x - mu) rs + beta,  y = act(z);  dz = dy act'(z)
//   dx = rs (gamma dz - mean(gamma dz) - xhat mean(gamma dz xhat)),  dgamma = sum dz xhat,  dbeta = sum dz
//
// A "team" of threads (part of a warp up to a whole block) holds a row in registers: one read of the inputs, one write of the
// outputs, the mean and then the sum of squared deviations over the same registers (no cancellation however large the mean).
// Bound by HBM.  Backward, teams walk over the rows with the next row's loads in flight and keep the sums of dgamma and dbeta of
// their columns in registers; a block's sums are joined in shared memory and written once, and a second launch adds the
// blocks' in a fixed order.  Rows too wide for registers are read again from the L2 (the "long" kernels).
#include <math.h>

#include "hdqt_dropout.cuh"

namespace hdqt {

namespace {

constexpr int kLongThreads = 1024;

struct RowParams {
  const void* x;                 // x, or h (fused backward)
  const void* residual;
  const void* dy;
  const void* dh;
  void* y;
  void* h;
  void* dx;
  void* dres;
  const void* gamma;
  const void* beta;
  int32_t param_dtype, act, channels;
  int32_t team;                  // threads of a row: a power of two up to 32, or a multiple of 32
  int32_t params_wide;           // gamma and beta start on 16-byte boundaries
  int32_t bits_stride;           // bytes of a team's dropout decisions in shared memory
  int64_t rows, x_rs, r_rs, y_rs;
  float eps;
  float* mean;
  float* rstd;
  float2* part;                  // [blocks, channels] sums of dbeta (x) and dgamma (y)
  DropParams d;
};

// V elements of gamma or beta from channel c on
template <int V>
__device__ __forceinline__ void load_params(const void* p, const RowParams& q, int c, float fill, float (&f)[V]) {
  if (p == nullptr) {
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] = fill;
  } else if (!q.params_wide || V == 1) {
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] = load_param(p, q.param_dtype, c + j);
  } else if (q.param_dtype == HDQT_DTYPE_F32) {
    constexpr int W = V < 4 ? V : 4;
#pragma unroll
    for (int j = 0; j < V; j += W) {
      const Vec<float, W> v = *reinterpret_cast<const Vec<float, W>*>(reinterpret_cast<const float*>(p) + c + j);
#pragma unroll
      for (int i = 0; i < W; ++i) f[j + i] = v.v[i];
    }
  } else if (q.param_dtype == HDQT_DTYPE_BF16) {
    unpack(*reinterpret_cast<const Vec<__nv_bfloat16, V>*>(reinterpret_cast<const __nv_bfloat16*>(p) + c), f);
  } else {
    unpack(*reinterpret_cast<const Vec<__half, V>*>(reinterpret_cast<const __half*>(p) + c), f);
  }
}

__device__ __forceinline__ void team_barrier(int team, int size) {
  if (size <= 32) __syncwarp();
  else if (size == (int)blockDim.x) __syncthreads();
  else asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(size) : "memory");
}

// Sums over the threads of a team; every thread gets them.  s: one slot of N per warp of the block, not in use since the barrier
// before the last one.
template <int N>
__device__ __forceinline__ void team_sum(float (&v)[N], int team, int t, int size, float* s) {
  for (int d = (size < 32 ? size : 32) >> 1; d > 0; d >>= 1) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xFFFFFFFFu, v[i], d);
  }
  if (size <= 32) return;
  const int warps = size >> 5, lane = t & 31;
  s += team * warps * N;
  if (lane == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) s[(t >> 5) * N + i] = v[i];
  }
  team_barrier(team, size);
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = lane < warps ? s[lane * N + i] : 0.0f;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xFFFFFFFFu, v[i], d);
  }
}

// Dropout decisions of a whole row for accesses narrower than a Philox group of eight: a byte per group in shared memory (visible
// after the team's next barrier), bit (o & 7) of byte o >> 3 for the element at o = (row * channels) % 8 + channel.
__device__ __forceinline__ void row_bits(const RowParams& p, int64_t row, int t, int size, uint8_t* bits) {
  const uint64_t first = (uint64_t)row * (uint64_t)p.channels;
  const int groups = ((int)(first & 7) + p.channels + 7) >> 3;
  const uint32_t offset = drop_offset(p.d);
  for (int k = t; k < groups; k += size) bits[k] = (uint8_t)drop_bits(p.d, offset, (first >> 3) + k);
}
// those of the V elements from channel c on
template <int V>
__device__ __forceinline__ uint32_t chunk_bits(const RowParams& p, int64_t row, int c, const uint8_t* bits) {
  if constexpr (V == 8) return drop_bits(p.d, drop_offset(p.d), ((uint64_t)row * (uint64_t)p.channels + c) >> 3);
  const int o = ((int)((uint64_t)row * (uint64_t)p.channels) & 7) + c;
  return bits[o >> 3] >> (o & 7);
}

// x scale where kept, else 0
__device__ __forceinline__ float dropped(float x, uint32_t bits, int j, float scale) {
  return (bits >> j) & 1 ? __fmul_rn(x, scale) : 0.0f;
}

template <typename T>
__device__ __forceinline__ float rounded(float v) { return to_f32(from_f32<T>(v)); }

// ---- rows in registers -------------------------------------------------------------------------------------

// Element i of thread t: channel ((i / V) * team + t) * V + i % V.
template <typename T, int V, int K, bool kFused>
__global__ void __launch_bounds__(1024) row_fwd_kernel(const RowParams p) {
  using A = Vec<T, V>;
  __shared__ float s_sum[2][32];
  extern __shared__ __align__(16) uint8_t s_dyn[];
  const int size = p.team, team = threadIdx.x / size, t = threadIdx.x - team * size;
  const int64_t row = (int64_t)blockIdx.x * (blockDim.x / size) + team;
  const bool live = row < p.rows;
  uint8_t* bits = s_dyn + team * p.bits_stride;

  A vx[K], vr[K];
  const T* src = reinterpret_cast<const T*>(p.x) + row * p.x_rs;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c = (k * size + t) * V;
    vx[k] = A{};
    if (live && c < p.channels) vx[k] = *reinterpret_cast<const A*>(src + c);
  }
  if constexpr (kFused) {
    const T* res = reinterpret_cast<const T*>(p.residual) + row * p.r_rs;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * size + t) * V;
      vr[k] = A{};
      if (p.residual && live && c < p.channels) vr[k] = *reinterpret_cast<const A*>(res + c);
    }
    if (V < 8 && p.d.on) {
      if (live) row_bits(p, row, t, size, bits);
      team_barrier(team, size);
    }
  }

  float x[K][V];
  float sum[1] = {0.0f};
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c = (k * size + t) * V;
    unpack(vx[k], x[k]);
    if constexpr (kFused) {
      float r[V];
      unpack(vr[k], r);
      if (p.d.on && live && c < p.channels) {
        const uint32_t b = chunk_bits<V>(p, row, c, bits);
#pragma unroll
        for (int j = 0; j < V; ++j) x[k][j] = dropped(x[k][j], b, j, p.d.scale);
      }
      if (p.residual) {
#pragma unroll
        for (int j = 0; j < V; ++j) x[k][j] = __fadd_rn(r[j], x[k][j]);
      }
      const A h = pack<T>(x[k]);
      if (live && c < p.channels) *reinterpret_cast<A*>(reinterpret_cast<T*>(p.h) + row * p.y_rs + c) = h;
      unpack(h, x[k]);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) sum[0] += x[k][j];
  }
  team_sum(sum, team, t, size, s_sum[0]);
  const float mu = sum[0] / (float)p.channels;
  float m2[1] = {0.0f};
#pragma unroll
  for (int k = 0; k < K; ++k) {
    if ((k * size + t) * V < p.channels) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float e = x[k][j] - mu;
        m2[0] = fmaf(e, e, m2[0]);
      }
    }
  }
  team_sum(m2, team, t, size, s_sum[1]);
  const float rs = __frsqrt_rn(m2[0] / (float)p.channels + p.eps);
  if (!live) return;
  if (t == 0) {
    p.mean[row] = mu;
    p.rstd[row] = rs;
  }
  T* dst = reinterpret_cast<T*>(p.y) + row * p.y_rs;
  with_act(p.act, [&]<int kAct>() {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * size + t) * V;
      if (c < p.channels) {
        float g[V], b[V], o[V];
        load_params(p.gamma, p, c, 1.0f, g);
        load_params(p.beta, p, c, 0.0f, b);
#pragma unroll
        for (int j = 0; j < V; ++j) o[j] = act_fwd<kAct>(fmaf((x[k][j] - mu) * rs, g[j], b[j]));
        *reinterpret_cast<A*>(dst + c) = pack<T>(o);
      }
    }
  });
}

template <typename T, int V, int K, bool kFused, int kMaxThreads>
__global__ void __launch_bounds__(kMaxThreads) row_bwd_kernel(const RowParams p) {
  using A = Vec<T, V>;
  __shared__ float s_sum[2][2 * kMaxThreads / 32];
  extern __shared__ __align__(16) uint8_t s_dyn[];
  const int size = p.team, teams = blockDim.x / size, team = threadIdx.x / size, t = threadIdx.x - team * size;
  const int64_t step = (int64_t)gridDim.x * teams;
  int64_t row = (int64_t)blockIdx.x * teams + team;
  const int ahead = size < 32 ? (threadIdx.x & 31) / size : 0;      // teams of this warp in front of this one

  A nx[K], nd[K];      // the next row
  float nmu = 0.0f, nrs = 0.0f;
  auto fetch = [&](int64_t r) {
    const bool live = r < p.rows;
    if (live) {
      nmu = p.mean[r];
      nrs = p.rstd[r];
    } else {
      nmu = nrs = 0.0f;
    }
    const T* src = reinterpret_cast<const T*>(p.x) + r * p.x_rs;
    const T* dys = reinterpret_cast<const T*>(p.dy) + r * p.y_rs;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * size + t) * V;
      nx[k] = A{};
      nd[k] = A{};
      if (live && c < p.channels) {
        nx[k] = *reinterpret_cast<const A*>(src + c);
        nd[k] = *reinterpret_cast<const A*>(dys + c);
      }
    }
  };

  float sum_g[K][V], sum_b[K][V];
#pragma unroll
  for (int k = 0; k < K; ++k) {
#pragma unroll
    for (int j = 0; j < V; ++j) sum_g[k][j] = sum_b[k][j] = 0.0f;
  }
  const float inv_c = 1.0f / (float)p.channels;
  int turn = 0;
  fetch(row);
  for (; row - ahead < p.rows; row += step, turn ^= 1) {            // (the same number of turns for all teams of a warp)
    const bool live = row < p.rows;
    A vx[K], vh[K];
    float d[K][V];
    const float mu = nmu, rs = nrs;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      vx[k] = nx[k];
      unpack(nd[k], d[k]);
    }
    fetch(row + step);
    uint8_t* bits = s_dyn + (turn * teams + team) * p.bits_stride;
    if constexpr (kFused) {
      if (p.dh) {
        const T* dhs = reinterpret_cast<const T*>(p.dh) + row * p.y_rs;
#pragma unroll
        for (int k = 0; k < K; ++k) {
          const int c = (k * size + t) * V;
          if (live && c < p.channels) vh[k] = *reinterpret_cast<const A*>(dhs + c);
        }
      }
      if (V < 8 && p.d.on && live) row_bits(p, row, t, size, bits);
    }
    float s[2] = {0.0f, 0.0f};
    with_act(p.act, [&]<int kAct>() {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int c = (k * size + t) * V;
        if (c < p.channels) {
          float x[V], g[V], b[V];
          unpack(vx[k], x);
          load_params(p.gamma, p, c, 1.0f, g);
          if constexpr (kAct != HDQT_ACT_NONE) load_params(p.beta, p, c, 0.0f, b);
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const float xh = (x[j] - mu) * rs;
            float dz = d[k][j];
            if constexpr (kAct != HDQT_ACT_NONE) dz = act_bwd<kAct>(dz, fmaf(xh, g[j], b[j]));
            sum_b[k][j] += dz;
            sum_g[k][j] = fmaf(dz, xh, sum_g[k][j]);
            d[k][j] = dz * g[j];
            s[0] += d[k][j];
            s[1] = fmaf(d[k][j], xh, s[1]);
          }
        }
      }
    });
    team_sum(s, team, t, size, s_sum[turn]);
    if (kFused && V < 8 && size <= 32) __syncwarp();
    const float m1 = s[0] * inv_c, m2 = s[1] * inv_c;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * size + t) * V;
      if (live && c < p.channels) {
        float x[V], o[V];
        unpack(vx[k], x);
#pragma unroll
        for (int j = 0; j < V; ++j) o[j] = rs * (d[k][j] - m1 - (x[j] - mu) * rs * m2);
        if constexpr (kFused) {
          if (p.dh) {
            float h[V];
            unpack(vh[k], h);
#pragma unroll
            for (int j = 0; j < V; ++j) o[j] += h[j];
          }
          if (p.dres) *reinterpret_cast<A*>(reinterpret_cast<T*>(p.dres) + row * p.y_rs + c) = pack<T>(o);
          if (p.d.on) {
            const uint32_t b = chunk_bits<V>(p, row, c, bits);
#pragma unroll
            for (int j = 0; j < V; ++j) o[j] = dropped(o[j], b, j, p.d.scale);
          }
        }
        if (p.dx) *reinterpret_cast<A*>(reinterpret_cast<T*>(p.dx) + row * p.y_rs + c) = pack<T>(o);
      }
    }
  }

  if (p.part == nullptr) return;
  float2* part = p.part + (int64_t)blockIdx.x * p.channels;
  // teams of a warp, then those of the block
  for (int o = size; o < 32; o <<= 1) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        sum_g[k][j] += __shfl_xor_sync(0xFFFFFFFFu, sum_g[k][j], o);
        sum_b[k][j] += __shfl_xor_sync(0xFFFFFFFFu, sum_b[k][j], o);
      }
    }
  }
  const int holders = size <= 32 ? (int)blockDim.x >> 5 : teams;
  const int holder = size <= 32 ? (int)threadIdx.x >> 5 : team;
  float2* mine = holders == 1 ? part : reinterpret_cast<float2*>(s_dyn) + holder * p.channels;
  if (holders > 1) __syncthreads();                                 // (the decisions are read, the sums take their place)
  if (ahead == 0) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * size + t) * V;
      if (c < p.channels) {
#pragma unroll
        for (int j = 0; j < V; ++j) mine[c + j] = make_float2(sum_b[k][j], sum_g[k][j]);
      }
    }
  }
  if (holders == 1) return;
  __syncthreads();
  for (int c = threadIdx.x; c < p.channels; c += blockDim.x) {
    float2 a = make_float2(0.0f, 0.0f);
    for (int i = 0; i < holders; ++i) {
      const float2 v = reinterpret_cast<const float2*>(s_dyn)[i * p.channels + c];
      a.x += v.x;
      a.y += v.y;
    }
    part[c] = a;
  }
}

// ---- rows of any length, read again from the L2 ------------------------------------------------------------

template <typename T, int V, bool kFused>
__global__ void __launch_bounds__(kLongThreads) long_fwd_kernel(const RowParams p) {
  using A = Vec<T, V>;
  __shared__ float s_sum[2][32];
  const int t = threadIdx.x;
  const uint32_t offset = kFused ? drop_offset(p.d) : 0;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const T* src = reinterpret_cast<const T*>(p.x) + row * p.x_rs;
    T* dst = reinterpret_cast<T*>(p.y) + row * p.y_rs;
    T* hs = kFused ? reinterpret_cast<T*>(p.h) + row * p.y_rs : nullptr;
    float sum[1] = {0.0f};
    for (int c = t * V; c < p.channels; c += kLongThreads * V) {
      float x[V];
      unpack(*reinterpret_cast<const A*>(src + c), x);
      if constexpr (kFused) {
        if (p.d.on) {
          const uint64_t i = (uint64_t)row * (uint64_t)p.channels + c;
          const uint32_t b = drop_bits(p.d, offset, i >> 3) >> (i & 7);
#pragma unroll
          for (int j = 0; j < V; ++j) x[j] = dropped(x[j], b, j, p.d.scale);
        }
        if (p.residual) {
          float r[V];
          unpack(*reinterpret_cast<const A*>(reinterpret_cast<const T*>(p.residual) + row * p.r_rs + c), r);
#pragma unroll
          for (int j = 0; j < V; ++j) x[j] = __fadd_rn(r[j], x[j]);
        }
        const A h = pack<T>(x);
        *reinterpret_cast<A*>(hs + c) = h;
        unpack(h, x);
      }
#pragma unroll
      for (int j = 0; j < V; ++j) sum[0] += x[j];
    }
    team_sum(sum, 0, t, kLongThreads, s_sum[0]);
    const float mu = sum[0] / (float)p.channels;
    const T* in = kFused ? hs : src;                                // (a thread reads back what it has written itself)
    float m2[1] = {0.0f};
    for (int c = t * V; c < p.channels; c += kLongThreads * V) {
      float x[V];
      unpack(*reinterpret_cast<const A*>(in + c), x);
#pragma unroll
      for (int j = 0; j < V; ++j) m2[0] = fmaf(x[j] - mu, x[j] - mu, m2[0]);
    }
    team_sum(m2, 0, t, kLongThreads, s_sum[1]);
    const float rs = __frsqrt_rn(m2[0] / (float)p.channels + p.eps);
    if (t == 0) {
      p.mean[row] = mu;
      p.rstd[row] = rs;
    }
    with_act(p.act, [&]<int kAct>() {
      for (int c = t * V; c < p.channels; c += kLongThreads * V) {
        float x[V], g[V], b[V];
        unpack(*reinterpret_cast<const A*>(in + c), x);
        load_params(p.gamma, p, c, 1.0f, g);
        load_params(p.beta, p, c, 0.0f, b);
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = act_fwd<kAct>(fmaf((x[j] - mu) * rs, g[j], b[j]));
        *reinterpret_cast<A*>(dst + c) = pack<T>(x);
      }
    });
  }
}

// gamma dz of V channels, and xhat
template <typename T, int V, int kAct>
__device__ __forceinline__ void long_terms(const RowParams& p, const T* xs, const T* dys, int c, float mu, float rs, float (&xh)[V],
                                           float (&dz)[V], float (&g)[V]) {
  unpack(*reinterpret_cast<const Vec<T, V>*>(xs + c), xh);
  unpack(*reinterpret_cast<const Vec<T, V>*>(dys + c), dz);
  load_params(p.gamma, p, c, 1.0f, g);
  float b[V];
  if constexpr (kAct != HDQT_ACT_NONE) load_params(p.beta, p, c, 0.0f, b);
#pragma unroll
  for (int j = 0; j < V; ++j) {
    xh[j] = (xh[j] - mu) * rs;
    if constexpr (kAct != HDQT_ACT_NONE) dz[j] = act_bwd<kAct>(dz[j], fmaf(xh[j], g[j], b[j]));
  }
}

template <typename T, int V, bool kFused>
__global__ void __launch_bounds__(kLongThreads) long_bwd_kernel(const RowParams p) {
  using A = Vec<T, V>;
  __shared__ float s_sum[2][64];
  const int t = threadIdx.x;
  const uint32_t offset = kFused ? drop_offset(p.d) : 0;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, turn ^= 1) {
    const T* xs = reinterpret_cast<const T*>(p.x) + row * p.x_rs;
    const T* dys = reinterpret_cast<const T*>(p.dy) + row * p.y_rs;
    const float mu = p.mean[row], rs = p.rstd[row];
    with_act(p.act, [&]<int kAct>() {
      float s[2] = {0.0f, 0.0f};
      for (int c = t * V; c < p.channels; c += kLongThreads * V) {
        float xh[V], dz[V], g[V];
        long_terms<T, V, kAct>(p, xs, dys, c, mu, rs, xh, dz, g);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          s[0] = fmaf(dz[j], g[j], s[0]);
          s[1] = fmaf(dz[j] * g[j], xh[j], s[1]);
        }
      }
      team_sum(s, 0, t, kLongThreads, s_sum[turn]);
      const float m1 = s[0] / (float)p.channels, m2 = s[1] / (float)p.channels;
      for (int c = t * V; c < p.channels; c += kLongThreads * V) {
        float xh[V], dz[V], g[V];
        long_terms<T, V, kAct>(p, xs, dys, c, mu, rs, xh, dz, g);
        float o[V];
#pragma unroll
        for (int j = 0; j < V; ++j) o[j] = rs * (dz[j] * g[j] - m1 - xh[j] * m2);
        if constexpr (kFused) {
          if (p.dh) {
            float h[V];
            unpack(*reinterpret_cast<const A*>(reinterpret_cast<const T*>(p.dh) + row * p.y_rs + c), h);
#pragma unroll
            for (int j = 0; j < V; ++j) o[j] += h[j];
          }
          if (p.dres) *reinterpret_cast<A*>(reinterpret_cast<T*>(p.dres) + row * p.y_rs + c) = pack<T>(o);
          if (p.d.on) {
            const uint64_t i = (uint64_t)row * (uint64_t)p.channels + c;
            const uint32_t b = drop_bits(p.d, offset, i >> 3) >> (i & 7);
#pragma unroll
            for (int j = 0; j < V; ++j) o[j] = dropped(o[j], b, j, p.d.scale);
          }
        }
        if (p.dx) *reinterpret_cast<A*>(reinterpret_cast<T*>(p.dx) + row * p.y_rs + c) = pack<T>(o);
      }
    });
  }
}

// sums of V columns over a share of the rows
template <typename T, int V>
__global__ void __launch_bounds__(256) long_param_kernel(const RowParams p) {
  const int c = (int)(blockIdx.x * 256 + threadIdx.x) * V;
  if (c >= p.channels) return;
  const int64_t first = p.rows * blockIdx.y / gridDim.y, last = p.rows * (blockIdx.y + 1) / gridDim.y;
  float sum_g[V], sum_b[V];
#pragma unroll
  for (int j = 0; j < V; ++j) sum_g[j] = sum_b[j] = 0.0f;
  with_act(p.act, [&]<int kAct>() {
#pragma unroll 4
    for (int64_t row = first; row < last; ++row) {
      float xh[V], dz[V], g[V];
      long_terms<T, V, kAct>(p, reinterpret_cast<const T*>(p.x) + row * p.x_rs, reinterpret_cast<const T*>(p.dy) + row * p.y_rs, c,
                             p.mean[row], p.rstd[row], xh, dz, g);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        sum_b[j] += dz[j];
        sum_g[j] = fmaf(dz[j], xh[j], sum_g[j]);
      }
    }
  });
#pragma unroll
  for (int j = 0; j < V; ++j) p.part[(int64_t)blockIdx.y * p.channels + c + j] = make_float2(sum_b[j], sum_g[j]);
}

// ---- host side ---------------------------------------------------------------------------------------------

constexpr int kMostParts = 4 * kNumSMsHint;      // blocks that leave parameter sums

hdqt_status_t check_desc(const hdqt_layer_norm_desc_t* d, bool fused) {
  if (!d) return HDQT_ERR_INVALID_ARG;
  if (d->rows < 0 || d->channels <= 0 || dtype_size(d->dtype) == 0) return HDQT_ERR_INVALID_ARG;
  if (d->param_dtype != HDQT_DTYPE_F32 && d->param_dtype != d->dtype) return HDQT_ERR_INVALID_ARG;
  if (d->act < HDQT_ACT_NONE || d->act > HDQT_ACT_SILU || !(d->eps >= 0.0f)) return HDQT_ERR_INVALID_ARG;
  if (d->rows > 1 && (d->x_row_stride < d->channels || d->y_row_stride < d->channels)) return HDQT_ERR_INVALID_ARG;
  if (fused && !valid_probability(d->p)) return HDQT_ERR_INVALID_ARG;
  if (d->channels > (1 << 20) || d->rows > 0x7FFFFFFFll) return HDQT_ERR_UNSUPPORTED;
  return HDQT_OK;
}

uintptr_t bits_of(const void* p) { return reinterpret_cast<uintptr_t>(p); }

RowParams make_params(const hdqt_layer_norm_desc_t& d, const void* gamma, const void* beta, float* mean, float* rstd) {
  RowParams p{};
  p.gamma = gamma;
  p.beta = beta;
  p.param_dtype = d.param_dtype;
  p.act = d.act;
  p.channels = (int32_t)d.channels;
  p.params_wide = ((bits_of(gamma) | bits_of(beta)) & 15) == 0;
  p.rows = d.rows;
  p.x_rs = d.x_row_stride;
  p.r_rs = d.r_row_stride;
  p.y_rs = d.y_row_stride;
  p.eps = d.eps;
  p.mean = mean;
  p.rstd = rstd;
  return p;
}

// threads of a row with E elements each
int team_size(int channels, int vec, int per_thread) {
  const int k = per_thread / vec, n = ((channels + vec - 1) / vec + k - 1) / k;
  if (n > 32) return (n + 31) / 32 * 32;
  int size = 1;
  while (size < n) size *= 2;
  return size;
}

template <auto kernel>
hdqt_status_t with_smem(size_t smem, const char* what) {
  if (smem <= 48 * 1024) return HDQT_OK;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  return e == cudaSuccess ? HDQT_OK : cuda_failure(e, what);
}

template <typename T, int V, bool kFused>
hdqt_status_t run_fwd(RowParams p, cudaStream_t s) {
  const int c = p.channels;
  int e = 8;
  if (p.rows * team_size(c, V, 8) > 148 * 2048 || team_size(c, V, 8) > 1024) e = 16;
  if (team_size(c, V, e) > 1024) e = 32;
  p.team = team_size(c, V, e);
  if (p.team > 1024) {
    const unsigned blocks = (unsigned)(p.rows < 2 * kNumSMsHint ? p.rows : 2 * kNumSMsHint);
    long_fwd_kernel<T, V, kFused><<<blocks, kLongThreads, 0, s>>>(p);
    return last_error("layer norm");
  }
  const int threads = p.team < 128 ? 128 / p.team * p.team : p.team;
  const int per_block = p.team <= 32 ? threads / p.team : 1;
  const int block = p.team <= 32 ? threads : p.team;
  p.bits_stride = V < 8 ? c / 8 + 2 : 0;
  const size_t smem = kFused ? (size_t)per_block * p.bits_stride : 0;
  const unsigned blocks = (unsigned)((p.rows + per_block - 1) / per_block);
  if (e == 8) row_fwd_kernel<T, V, 8 / V, kFused><<<blocks, block, smem, s>>>(p);
  else if (e == 16) row_fwd_kernel<T, V, 16 / V, kFused><<<blocks, block, smem, s>>>(p);
  else row_fwd_kernel<T, V, 32 / V, kFused><<<blocks, block, smem, s>>>(p);
  return last_error("layer norm");
}

template <typename T, int V, int E, bool kFused, int kMaxThreads>
hdqt_status_t launch_bwd(const RowParams& p, int block, int* parts, cudaStream_t s) {
  constexpr auto kernel = row_bwd_kernel<T, V, E / V, kFused, kMaxThreads>;
  const int teams = block / p.team;
  const int holders = p.team <= 32 ? block / 32 : teams;
  size_t smem = holders > 1 ? (size_t)holders * p.channels * sizeof(float2) : 0;
  const size_t bits = kFused ? (size_t)2 * teams * p.bits_stride : 0;
  if (bits > smem) smem = bits;
  const hdqt_status_t st = with_smem<kernel>(smem, "layer norm gradient");
  if (st != HDQT_OK) return st;
  int per_sm = 0;
  const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, block, smem);
  if (e != cudaSuccess) return cuda_failure(e, "layer norm gradient");
  if (per_sm > kMostParts / kNumSMsHint) per_sm = kMostParts / kNumSMsHint;
  const int64_t most = (p.rows + teams - 1) / teams;
  const int64_t blocks = most < (int64_t)per_sm * kNumSMsHint ? most : (int64_t)per_sm * kNumSMsHint;
  kernel<<<(unsigned)blocks, block, smem, s>>>(p);
  *parts = (int)blocks;
  return last_error("layer norm gradient");
}

template <typename T, int V, bool kFused>
hdqt_status_t run_bwd(RowParams p, int* parts, cudaStream_t s) {
  const int c = p.channels;
  constexpr int E = sizeof(T) == 2 ? 16 : 8;
  p.team = team_size(c, V, E);
  p.bits_stride = V < 8 ? c / 8 + 2 : 0;
  if (p.team <= 256) return launch_bwd<T, V, E, kFused, 256>(p, 256 / p.team * p.team, parts, s);
  if (p.team <= 512) return launch_bwd<T, V, E, kFused, 512>(p, p.team, parts, s);
  const unsigned blocks = (unsigned)(p.rows < 2 * kNumSMsHint ? p.rows : 2 * kNumSMsHint);
  if (p.dx || p.dres) long_bwd_kernel<T, V, kFused><<<blocks, kLongThreads, 0, s>>>(p);
  if (p.part) {
    const unsigned columns = (unsigned)((c / V + 255) / 256);
    const int64_t want = (8 * kNumSMsHint + columns - 1) / columns;
    const int64_t shares = want < p.rows ? want : p.rows;
    *parts = (int)(shares < kMostParts ? shares : kMostParts);
    long_param_kernel<T, V><<<dim3(columns, (unsigned)*parts), 256, 0, s>>>(p);
  }
  return last_error("layer norm gradient");
}

hdqt_status_t forward(const hdqt_layer_norm_desc_t* d, bool fused, const void* x, const void* residual, const void* gamma,
                      const void* beta, void* h, void* y, float* mean, float* rstd, void* stream) {
  const hdqt_status_t st = check_desc(d, fused);
  if (st != HDQT_OK) return st;
  if (d->rows == 0) return HDQT_OK;
  if (!x || !y || !mean || !rstd || (fused && !h)) return HDQT_ERR_INVALID_ARG;
  if (residual && d->rows > 1 && d->r_row_stride < d->channels) return HDQT_ERR_INVALID_ARG;
  const int elem = dtype_size(d->dtype), pelem = dtype_size(d->param_dtype);
  const uintptr_t bases = bits_of(x) | bits_of(residual) | bits_of(h) | bits_of(y);
  if ((bases & (uintptr_t)(elem - 1)) || ((bits_of(gamma) | bits_of(beta)) & (uintptr_t)(pelem - 1)) ||
      ((bits_of(mean) | bits_of(rstd)) & 3) || (fused && (bits_of(d->philox_offset) & 3)))
    return HDQT_ERR_ALIGNMENT;
  RowParams p = make_params(*d, gamma, beta, mean, rstd);
  p.x = x;
  p.residual = residual;
  p.h = h;
  p.y = y;
  if (fused) p.d = make_drop(d->p, d->seed, d->tag, d->philox_offset);
  const uintptr_t strides = d->rows > 1 ? (uintptr_t)((p.x_rs | p.y_rs | (residual ? p.r_rs : 0)) * elem) : 0;
  const int vec = vector_width(d->channels, elem, bases | strides);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  return with_type_and_width(d->dtype, vec, [&]<typename T, int V>() { return fused ? run_fwd<T, V, true>(p, s) : run_fwd<T, V, false>(p, s); });
}

hdqt_status_t backward(const hdqt_layer_norm_desc_t* d, bool fused, const void* dy, const void* dh, const void* x, const void* gamma,
                       const void* beta, const float* mean, const float* rstd, void* dx, void* dres, void* dgamma, void* dbeta,
                       void* workspace, size_t workspace_bytes, void* stream) {
  const hdqt_status_t st = check_desc(d, fused);
  if (st != HDQT_OK) return st;
  if (!workspace || (d->rows > 0 && (!x || !dy || !mean || !rstd))) return HDQT_ERR_INVALID_ARG;
  const int elem = dtype_size(d->dtype), pelem = dtype_size(d->param_dtype);
  const uintptr_t bases = bits_of(x) | bits_of(dy) | bits_of(dh) | bits_of(dx) | bits_of(dres);
  const uintptr_t params = bits_of(gamma) | bits_of(beta) | bits_of(dgamma) | bits_of(dbeta);
  if ((bases & (uintptr_t)(elem - 1)) || (params & (uintptr_t)(pelem - 1)) || ((bits_of(mean) | bits_of(rstd)) & 3) ||
      (bits_of(workspace) & 255) || (fused && (bits_of(d->philox_offset) & 3)))
    return HDQT_ERR_ALIGNMENT;
  if (workspace_bytes < hdqt_layer_norm_workspace_bytes(d)) return HDQT_ERR_WORKSPACE;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  float2* part = reinterpret_cast<float2*>(workspace);
  const bool want_params = dgamma || dbeta;
  int parts = 0;
  if (d->rows > 0 && (dx || dres || want_params)) {
    RowParams p = make_params(*d, gamma, beta, const_cast<float*>(mean), const_cast<float*>(rstd));
    p.x = x;
    p.dy = dy;
    p.dh = dh;
    p.dx = dx;
    p.dres = dres;
    p.part = want_params ? part : nullptr;
    if (fused) p.d = make_drop(d->p, d->seed, d->tag, d->philox_offset);
    const uintptr_t strides = d->rows > 1 ? (uintptr_t)((p.x_rs | p.y_rs) * elem) : 0;
    const int vec = vector_width(d->channels, elem, bases | strides);
    const hdqt_status_t e = with_type_and_width(d->dtype, vec, [&]<typename T, int V>() {
      return fused ? run_bwd<T, V, true>(p, &parts, s) : run_bwd<T, V, false>(p, &parts, s);
    });
    if (e != HDQT_OK) return e;
  }
  if (want_params) launch_param_grad(part, parts, (int)d->channels, dgamma, dbeta, d->param_dtype, parts > 0, s);
  return last_error("layer norm gradient");
}

}  // namespace

}  // namespace hdqt

using namespace hdqt;

extern "C" size_t hdqt_layer_norm_workspace_bytes(const hdqt_layer_norm_desc_t* d) {
  if (check_desc(d, false) != HDQT_OK) return 0;
  const int64_t parts = d->rows < kMostParts ? d->rows : kMostParts;
  return align256((size_t)parts * d->channels * sizeof(float2)) + 256;
}

extern "C" hdqt_status_t hdqt_layer_norm_fwd(const hdqt_layer_norm_desc_t* d, const void* x, const void* gamma, const void* beta,
                                             void* y, float* mean, float* rstd, void* stream) {
  return forward(d, false, x, nullptr, gamma, beta, nullptr, y, mean, rstd, stream);
}

extern "C" hdqt_status_t hdqt_layer_norm_bwd(const hdqt_layer_norm_desc_t* d, const void* dy, const void* x, const void* gamma,
                                             const void* beta, const float* mean, const float* rstd, void* dx, void* dgamma,
                                             void* dbeta, void* workspace, size_t workspace_bytes, void* stream) {
  return backward(d, false, dy, nullptr, x, gamma, beta, mean, rstd, dx, nullptr, dgamma, dbeta, workspace, workspace_bytes, stream);
}

extern "C" hdqt_status_t hdqt_dropout_add_layer_norm_fwd(const hdqt_layer_norm_desc_t* d, const void* x, const void* residual,
                                                         const void* gamma, const void* beta, void* h, void* y, float* mean,
                                                         float* rstd, void* stream) {
  return forward(d, true, x, residual, gamma, beta, h, y, mean, rstd, stream);
}

extern "C" hdqt_status_t hdqt_dropout_add_layer_norm_bwd(const hdqt_layer_norm_desc_t* d, const void* dy, const void* dh,
                                                         const void* h, const void* gamma, const void* beta, const float* mean,
                                                         const float* rstd, void* dx, void* dresidual, void* dgamma, void* dbeta,
                                                         void* workspace, size_t workspace_bytes, void* stream) {
  return backward(d, true, dy, dh, h, gamma, beta, mean, rstd, dx, dresidual, dgamma, dbeta, workspace, workspace_bytes, stream);
}
