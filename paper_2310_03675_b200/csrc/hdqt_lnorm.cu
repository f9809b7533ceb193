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

#include <atomic>

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
  int32_t classes;               // rows that are cut at different places (1 = all alike)
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
  // (constant names: a barrier named by a register makes the block reserve all sixteen, and four such blocks fill an SM)
  else if (team == 0) asm volatile("bar.sync 1, %0;" ::"r"(size) : "memory");
  else if (team == 1) asm volatile("bar.sync 2, %0;" ::"r"(size) : "memory");
  else if (team == 2) asm volatile("bar.sync 3, %0;" ::"r"(size) : "memory");
  else asm volatile("bar.sync 4, %0;" ::"r"(size) : "memory");
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

// ---- rows in registers, 16-byte accesses ---------------------------------------------------------------------
//
// A row is cut at the 16-byte boundaries of memory into chunks of V elements; thread t of a team holds the chunks t, t + team, ...
// (K of them).  Where the channels are not a multiple of V, rows of a dense tensor start `lead` elements behind a boundary, lead =
// (row * channels) mod V, which repeats every `classes` rows.  A block keeps to the rows of one class, so that all its rows
// are cut alike: element j of chunk q is channel q V - lead + j, and a chunk that is shared with a neighbouring row is masked.
// gamma and beta stand in shared memory in this order, in fp32.

template <int V>
struct Cut {
  int lead, chunks;        // elements in front of the row in its first chunk; chunks of the row
  uint32_t mask;           // V bits per chunk of this thread: elements that belong to the row
  __device__ __forceinline__ uint32_t of(int k) const { return (mask >> (k * V)) & ((1u << V) - 1); }
};
template <int V, int K>
__device__ __forceinline__ Cut<V> cut_row(const RowParams& p, int cls, int t, int size) {
  static_assert(V * K <= 32);
  Cut<V> u;
  u.lead = (int)(((int64_t)cls * p.channels) & (V - 1));
  u.chunks = (u.lead + p.channels + V - 1) / V;
  u.mask = 0;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int first = (k * size + t) * V - u.lead;          // channel of the chunk's first element
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (first + j >= 0 && first + j < p.channels) u.mask |= 1u << (k * V + j);
  }
  return u;
}

// The chunk at src, with a neighbouring row's elements in it where the mask has gaps.  `edge`: the row's end may be the tensor's, so
// that a shared chunk is read element by element.
template <typename T, int V, bool kShift>
__device__ __forceinline__ Words load_chunk(const T* src, uint32_t mask, bool edge) {
  Words v{};
  if (kShift && edge && mask != (1u << V) - 1) {
    if constexpr (kShift) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
          if ((mask >> i) & 1) v.w[i] = __float_as_uint(src[i]);
        } else {
          if ((mask >> (2 * i)) & 1) v.w[i] = reinterpret_cast<const uint16_t*>(src)[2 * i];
          if ((mask >> (2 * i)) & 2) v.w[i] |= (uint32_t) reinterpret_cast<const uint16_t*>(src)[2 * i + 1] << 16;
        }
      }
    }
  } else if (mask != 0) {
    v = *reinterpret_cast<const Words*>(src);
  }
  return v;
}
template <typename T, int V, bool kShift>
__device__ __forceinline__ void unpack_chunk(const Words& v, uint32_t mask, float (&f)[V]) {
  unpack<T>(v, f);
  if constexpr (kShift) {
    if (mask != (1u << V) - 1) {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (!((mask >> j) & 1)) f[j] = 0.0f;
    }
  }
}
template <typename T, int V, bool kShift>
__device__ __forceinline__ void store_chunk(T* dst, uint32_t mask, const Words& v) {
  if (mask == (1u << V) - 1) *reinterpret_cast<Words*>(dst) = v;
  if constexpr (kShift) {
    if (mask != (1u << V) - 1) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if ((mask >> j) & 1) {
          if constexpr (sizeof(T) == 4) reinterpret_cast<uint32_t*>(dst)[j] = v.w[j];
          else reinterpret_cast<uint16_t*>(dst)[j] = (uint16_t)(v.w[j / 2] >> (16 * (j & 1)));
        }
      }
    }
  }
}

// gamma or beta in the block's order: four elements of every chunk, then the next four
template <int V>
__device__ __forceinline__ void stage_params(const void* src, const RowParams& p, int lead, int slots, float fill, float* s) {
  for (int i = threadIdx.x; i < slots * V; i += blockDim.x) {
    const int c = i - lead;
    const bool in = c >= 0 && c < p.channels;
    const float v = !in ? 0.0f : src ? load_param(src, p.param_dtype, c) : fill;
    s[(((i & (V - 1)) >> 2) * slots + i / V) * 4 + (i & 3)] = v;
  }
}
template <int V>
__device__ __forceinline__ void staged(const float* s, int slots, int q, float (&f)[V]) {
#pragma unroll
  for (int i = 0; i < V / 4; ++i) {
    const float4 v = reinterpret_cast<const float4*>(s)[i * slots + q];
    f[4 * i] = v.x;
    f[4 * i + 1] = v.y;
    f[4 * i + 2] = v.z;
    f[4 * i + 3] = v.w;
  }
}

// random words of chunk number i (of the flattened tensor), its elements the first V
template <int V>
__device__ __forceinline__ Philox4 chunk_words(const DropParams& d, uint32_t offset, uint64_t i) {
  if constexpr (V == 8) return drop_words(d, offset, i);
  Philox4 w = drop_words(d, offset, i >> 1);
  if (i & 1) {
    w.w[0] = w.w[2];
    w.w[1] = w.w[3];
  }
  return w;
}
template <int V>
__device__ __forceinline__ void drop_chunk(const DropParams& d, uint32_t offset, uint64_t i, float (&x)[V]) {
  const Philox4 w = chunk_words<V>(d, offset, i);
#pragma unroll
  for (int j = 0; j < V; ++j) x[j] = drop_keeps(w, j, d.limit) ? __fmul_rn(x[j], d.scale) : 0.0f;
}

template <typename T, int K, bool kFused, bool kShift>
__global__ void __launch_bounds__(512) team_fwd_kernel(const RowParams p) {
  constexpr int V = 16 / sizeof(T);
  __shared__ float s_sum[2][2][16];
  extern __shared__ __align__(16) float s_params[];
  const int size = p.team, teams = blockDim.x / size, team = threadIdx.x / size, t = threadIdx.x - team * size;
  const int cls = kShift ? blockIdx.x % p.classes : 0;
  const int64_t step = (int64_t)(gridDim.x / p.classes) * teams * p.classes;
  int64_t row = (int64_t)(blockIdx.x / p.classes * teams + team) * p.classes + cls;
  const int64_t ahead = size < 32 ? (int64_t)((threadIdx.x & 31) / size) * p.classes : 0;   // to this warp's first team's row
  const Cut<V> cut = cut_row<V, K>(p, cls, t, size);
  const int slots = K * size;
  float* s_beta = s_params + slots * V;

  Words nx[K], nr[K];      // the next row
  auto fetch = [&](int64_t r) {
    const bool live = r < p.rows, edge = r == p.rows - 1;
    const T* src = reinterpret_cast<const T*>(p.x) + r * p.x_rs - cut.lead;
    const T* res = reinterpret_cast<const T*>(p.residual) + r * p.r_rs - cut.lead;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t m = live ? cut.of(k) : 0;
      nx[k] = load_chunk<T, V, kShift>(src + (k * size + t) * V, m, edge);
      if constexpr (kFused) nr[k] = load_chunk<T, V, kShift>(res + (k * size + t) * V, p.residual ? m : 0, edge);
    }
  };
  fetch(row);
  stage_params<V>(p.gamma, p, cut.lead, slots, 1.0f, s_params);
  stage_params<V>(p.beta, p, cut.lead, slots, 0.0f, s_beta);
  __syncthreads();
  const uint32_t offset = kFused ? drop_offset(p.d) : 0;
  const float inv_c = 1.0f / (float)p.channels;
  for (int turn = 0; row - ahead < p.rows; row += step, turn ^= 1) {      // (the same number of turns for all teams of a warp)
    const bool live = row < p.rows;
    float x[K][V];
    float sum[1] = {0.0f};
    const int64_t at = row * p.y_rs - cut.lead + t * V;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t m = live ? cut.of(k) : 0;
      unpack_chunk<T, V, kShift>(nx[k], m, x[k]);
      if constexpr (kFused) {
        if (p.d.on) drop_chunk<V>(p.d, offset, ((uint64_t)row * (uint64_t)p.channels - cut.lead) / V + k * size + t, x[k]);
        if (p.residual) {
          float r[V];
          unpack_chunk<T, V, kShift>(nr[k], m, r);
#pragma unroll
          for (int j = 0; j < V; ++j) x[k][j] = __fadd_rn(r[j], x[k][j]);
        }
        const Words h = pack_words<T>(x[k]);
        store_chunk<T, V, kShift>(reinterpret_cast<T*>(p.h) + at + k * size * V, m, h);
        unpack<T>(h, x[k]);
      }
#pragma unroll
      for (int j = 0; j < V; ++j) sum[0] += x[k][j];
    }
    fetch(row + step);
    team_sum(sum, team, t, size, s_sum[turn][0]);
    const float mu = sum[0] * inv_c;
    float m2[1] = {0.0f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t m = cut.of(k);
#pragma unroll
      for (int j = 0; j < V; ++j) x[k][j] -= mu;
      if (m != (1u << V) - 1) {
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (!((m >> j) & 1)) x[k][j] = 0.0f;
      }
#pragma unroll
      for (int j = 0; j < V; ++j) m2[0] = fmaf(x[k][j], x[k][j], m2[0]);
    }
    team_sum(m2, team, t, size, s_sum[turn][1]);
    const float rs = __frsqrt_rn(fmaf(m2[0], inv_c, p.eps));
    if (t == 0 && live) {
      p.mean[row] = mu;
      p.rstd[row] = rs;
    }
    with_act(p.act, [&]<int kAct>() {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        float g[V], b[V];
        staged<V>(s_params, slots, k * size + t, g);
        staged<V>(s_beta, slots, k * size + t, b);
#pragma unroll
        for (int j = 0; j < V; ++j) x[k][j] = act_fwd<kAct>(fmaf(x[k][j] * rs, g[j], b[j]));
        store_chunk<T, V, kShift>(reinterpret_cast<T*>(p.y) + at + k * size * V, live ? cut.of(k) : 0, pack_words<T>(x[k]));
      }
    });
  }
}

template <typename T, int K, bool kFused, bool kShift>
__global__ void __launch_bounds__(512) team_bwd_kernel(const RowParams p) {
  constexpr int V = 16 / sizeof(T);
  __shared__ float s_sum[2][32];
  extern __shared__ __align__(16) float s_params[];
  const int size = p.team, teams = blockDim.x / size, team = threadIdx.x / size, t = threadIdx.x - team * size;
  const int cls = kShift ? blockIdx.x % p.classes : 0;
  const int64_t step = (int64_t)(gridDim.x / p.classes) * teams * p.classes;
  int64_t row = (int64_t)(blockIdx.x / p.classes * teams + team) * p.classes + cls;
  const int64_t ahead = size < 32 ? (int64_t)((threadIdx.x & 31) / size) * p.classes : 0;
  const Cut<V> cut = cut_row<V, K>(p, cls, t, size);
  const int slots = K * size;
  float* s_beta = s_params + slots * V;

  Words nx[K], nd[K];      // the next row
  float nmu = 0.0f, nrs = 0.0f;
  auto fetch = [&](int64_t r) {
    const bool live = r < p.rows, edge = r == p.rows - 1;
    const T* src = reinterpret_cast<const T*>(p.x) + r * p.x_rs - cut.lead;
    const T* dys = reinterpret_cast<const T*>(p.dy) + r * p.y_rs - cut.lead;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t m = live ? cut.of(k) : 0;
      nx[k] = load_chunk<T, V, kShift>(src + (k * size + t) * V, m, edge);
      nd[k] = load_chunk<T, V, kShift>(dys + (k * size + t) * V, m, edge);
    }
    nmu = live ? p.mean[r] : 0.0f;
    nrs = live ? p.rstd[r] : 0.0f;
  };
  fetch(row);
  stage_params<V>(p.gamma, p, cut.lead, slots, 1.0f, s_params);
  if (p.act != HDQT_ACT_NONE) stage_params<V>(p.beta, p, cut.lead, slots, 0.0f, s_beta);
  __syncthreads();
  const uint32_t offset = kFused ? drop_offset(p.d) : 0;

  float sum_g[K][V], sum_b[K][V];
#pragma unroll
  for (int k = 0; k < K; ++k) {
#pragma unroll
    for (int j = 0; j < V; ++j) sum_g[k][j] = sum_b[k][j] = 0.0f;
  }
  const float inv_c = 1.0f / (float)p.channels;
  for (int turn = 0; row - ahead < p.rows; row += step, turn ^= 1) {
    const bool live = row < p.rows;
    const int64_t at = row * p.y_rs - cut.lead + t * V;
    Words vx[K], vh[K];
    float d[K][V];
    const float mu = nmu, rs = nrs;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      vx[k] = nx[k];
      unpack_chunk<T, V, kShift>(nd[k], live ? cut.of(k) : 0, d[k]);
    }
    fetch(row + step);
    if constexpr (kFused) {
      if (p.dh) {
#pragma unroll
        for (int k = 0; k < K; ++k)
          vh[k] = load_chunk<T, V, kShift>(reinterpret_cast<const T*>(p.dh) + at + k * size * V, live ? cut.of(k) : 0, row == p.rows - 1);
      }
    }
    float s[2] = {0.0f, 0.0f};
    with_act(p.act, [&]<int kAct>() {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        float x[V], g[V], b[V];
        unpack_chunk<T, V, kShift>(vx[k], cut.of(k), x);
        staged<V>(s_params, slots, k * size + t, g);
        if constexpr (kAct != HDQT_ACT_NONE) staged<V>(s_beta, slots, k * size + t, b);
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
    });
    team_sum(s, team, t, size, s_sum[turn]);
    const float m1 = s[0] * inv_c, m2 = s[1] * inv_c;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t m = live ? cut.of(k) : 0;
      float x[V], o[V];
      unpack<T>(vx[k], x);
#pragma unroll
      for (int j = 0; j < V; ++j) o[j] = rs * (d[k][j] - m1 - (x[j] - mu) * rs * m2);
      if constexpr (kFused) {
        if (p.dh) {
          float h[V];
          unpack<T>(vh[k], h);
#pragma unroll
          for (int j = 0; j < V; ++j) o[j] += h[j];
        }
        if (p.dres) store_chunk<T, V, kShift>(reinterpret_cast<T*>(p.dres) + at + k * size * V, m, pack_words<T>(o));
        if (p.d.on) drop_chunk<V>(p.d, offset, ((uint64_t)row * (uint64_t)p.channels - cut.lead) / V + k * size + t, o);
      }
      if (p.dx) store_chunk<T, V, kShift>(reinterpret_cast<T*>(p.dx) + at + k * size * V, m, pack_words<T>(o));
    }
  }

  if (p.part == nullptr) return;
  // sums of the teams of a warp, then of the block (in shared memory, in the place of gamma and beta), then to this block's part
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
  float2* part = p.part + (int64_t)blockIdx.x * p.channels;
  const int holders = size <= 32 ? (int)blockDim.x >> 5 : teams;
  const int holder = size <= 32 ? (int)threadIdx.x >> 5 : team;
  float2* mine = holders == 1 ? part : reinterpret_cast<float2*>(s_params) + holder * p.channels;
  if (holders > 1) __syncthreads();
  if (ahead == 0) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if ((cut.of(k) >> j) & 1) mine[(k * size + t) * V - cut.lead + j] = make_float2(sum_b[k][j], sum_g[k][j]);
    }
  }
  if (holders == 1) return;
  __syncthreads();
  for (int c = threadIdx.x; c < p.channels; c += blockDim.x) {
    float2 a = make_float2(0.0f, 0.0f);
    for (int i = 0; i < holders; ++i) {
      const float2 v = reinterpret_cast<const float2*>(s_params)[i * p.channels + c];
      a.x += v.x;
      a.y += v.y;
    }
    part[c] = a;
  }
}

// ---- rows in registers, any strides and addresses: one element per access -------------------------------------

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

constexpr int kMostTeam = 512;                   // threads of a row held in registers
constexpr size_t kMostSmem = 200 * 1024;

// Blocks of a kernel that fit an SM, by the threads of a row (which fix the block and its shared memory).  Looked up once per
// kernel and row width; the shared memory limit is raised at a kernel's first launch on a device.
template <auto kernel>
hdqt_status_t blocks_per_sm(int team, int block, size_t smem, int* out) {
  static std::atomic<uint64_t> ready{0};
  static std::atomic<int> known[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev > 63 || !((ready.load(std::memory_order_relaxed) >> dev) & 1))) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostSmem);
    if (e == cudaSuccess && dev <= 63) ready.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  if (e != cudaSuccess) return cuda_failure(e, "layer norm");
  const int slot = team > 32 ? 6 + team / 32 : __builtin_ctz(team);
  int n = known[slot].load(std::memory_order_relaxed);
  if (n == 0) {
    e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, block, smem);
    if (e != cudaSuccess) return cuda_failure(e, "layer norm");
    if (n < 1) n = 1;
    known[slot].store(n, std::memory_order_relaxed);
  }
  *out = n;
  return HDQT_OK;
}

// One launch of a kernel whose teams walk over the rows: as many blocks as the machine holds, at most `most` per SM.
template <auto kernel>
hdqt_status_t launch_teams(const RowParams& p, size_t smem, int most, int* blocks, cudaStream_t s) {
  const int block = p.team < 256 ? 256 / p.team * p.team : p.team, teams = block / p.team;
  int per_sm = 0;
  const hdqt_status_t st = blocks_per_sm<kernel>(p.team, block, smem, &per_sm);
  if (st != HDQT_OK) return st;
  if (per_sm > most) per_sm = most;
  const int64_t needed = ((p.rows + p.classes - 1) / p.classes + teams - 1) / teams;       // of each class
  const int64_t room = (int64_t)per_sm * kNumSMsHint / p.classes;
  const int64_t n = (needed < room ? needed : room) * p.classes;
  kernel<<<(unsigned)n, block, smem, s>>>(p);
  *blocks = (int)n;
  return last_error("layer norm");
}

// threads of a row whose chunks are divided K to a thread
int chunk_team(const RowParams& p, int vec, int k) { return team_size(p.channels + (p.classes > 1 ? vec - 1 : 0), vec, k * vec); }

template <typename T, int K, bool kFused>
hdqt_status_t fwd_teams(RowParams p, cudaStream_t s) {
  constexpr int V = 16 / sizeof(T);
  p.team = chunk_team(p, V, K);
  const size_t smem = (size_t)2 * K * p.team * V * sizeof(float);
  int blocks;
  if (p.classes > 1) return launch_teams<team_fwd_kernel<T, K, kFused, true>>(p, smem, 32, &blocks, s);
  return launch_teams<team_fwd_kernel<T, K, kFused, false>>(p, smem, 32, &blocks, s);
}

template <typename T, bool kFused>
hdqt_status_t run_fwd(RowParams p, bool wide, cudaStream_t s) {
  constexpr int V = 16 / sizeof(T), kMost = 32 / V;      // chunks of a thread
  if (wide && chunk_team(p, V, kMost) <= kMostTeam) {
    // wider teams where there are too few rows to fill the machine
    const int64_t chunks = p.rows * ((p.channels + V - 1) / V);
    if (chunks >= (int64_t)kMost * kNumSMsHint * 768 || chunk_team(p, V, kMost / 2) > kMostTeam) return fwd_teams<T, kMost, kFused>(p, s);
    if (chunks >= (int64_t)kMost / 2 * kNumSMsHint * 768 || chunk_team(p, V, kMost / 4) > kMostTeam)
      return fwd_teams<T, kMost / 2, kFused>(p, s);
    return fwd_teams<T, kMost / 4, kFused>(p, s);
  }
  p.classes = 1;
  p.team = team_size(p.channels, 1, 16);
  if (p.team <= 1024 && !wide) {
    const int per_block = p.team <= 32 ? 128 / p.team : 1, block = p.team <= 32 ? 128 : p.team;
    p.bits_stride = p.channels / 8 + 2;
    const size_t smem = kFused ? (size_t)per_block * p.bits_stride : 0;
    row_fwd_kernel<T, 1, 16, kFused><<<(unsigned)((p.rows + per_block - 1) / per_block), block, smem, s>>>(p);
    return last_error("layer norm");
  }
  const unsigned blocks = (unsigned)(p.rows < 2 * kNumSMsHint ? p.rows : 2 * kNumSMsHint);
  if (wide && p.channels % V == 0) long_fwd_kernel<T, V, kFused><<<blocks, kLongThreads, 0, s>>>(p);
  else long_fwd_kernel<T, 1, kFused><<<blocks, kLongThreads, 0, s>>>(p);
  return last_error("layer norm");
}

size_t sums_bytes(const RowParams& p) {
  const int block = p.team < 256 ? 256 / p.team * p.team : p.team, holders = p.team <= 32 ? block / 32 : block / p.team;
  return holders > 1 ? (size_t)holders * p.channels * sizeof(float2) : 0;
}

template <typename T, int K, bool kFused>
hdqt_status_t bwd_teams(RowParams p, int* parts, cudaStream_t s) {
  constexpr int V = 16 / sizeof(T);
  p.team = chunk_team(p, V, K);
  const size_t params = (size_t)2 * K * p.team * V * sizeof(float), sums = sums_bytes(p);
  const size_t smem = params > sums ? params : sums;
  if (p.classes > 1) return launch_teams<team_bwd_kernel<T, K, kFused, true>>(p, smem, kMostParts / kNumSMsHint, parts, s);
  return launch_teams<team_bwd_kernel<T, K, kFused, false>>(p, smem, kMostParts / kNumSMsHint, parts, s);
}

template <typename T, bool kFused>
hdqt_status_t run_bwd(RowParams p, bool wide, int* parts, cudaStream_t s) {
  constexpr int V = 16 / sizeof(T);
  if (wide && chunk_team(p, V, 2) <= kMostTeam) return bwd_teams<T, 2, kFused>(p, parts, s);
  p.classes = 1;
  p.team = team_size(p.channels, 1, 8);
  if (p.team <= 512 && !wide) {
    p.bits_stride = p.channels / 8 + 2;
    const int block = p.team < 256 ? 256 / p.team * p.team : p.team;
    const size_t bits = kFused ? (size_t)2 * (block / p.team) * p.bits_stride : 0, sums = sums_bytes(p);
    return launch_teams<row_bwd_kernel<T, 1, 8, kFused, 512>>(p, bits > sums ? bits : sums, kMostParts / kNumSMsHint, parts, s);
  }
  const unsigned blocks = (unsigned)(p.rows < 2 * kNumSMsHint ? p.rows : 2 * kNumSMsHint);
  const bool vector = wide && p.channels % V == 0;
  if (p.dx || p.dres) {
    if (vector) long_bwd_kernel<T, V, kFused><<<blocks, kLongThreads, 0, s>>>(p);
    else long_bwd_kernel<T, 1, kFused><<<blocks, kLongThreads, 0, s>>>(p);
  }
  if (p.part) {
    const unsigned columns = (unsigned)((p.channels / (vector ? V : 1) + 255) / 256);
    const int64_t want = (8 * kNumSMsHint + columns - 1) / columns;
    const int64_t shares = want < p.rows ? want : p.rows;
    *parts = (int)(shares < kMostParts ? shares : kMostParts);
    if (vector) long_param_kernel<T, V><<<dim3(columns, (unsigned)*parts), 256, 0, s>>>(p);
    else long_param_kernel<T, 1><<<dim3(columns, (unsigned)*parts), 256, 0, s>>>(p);
  }
  return last_error("layer norm gradient");
}

// 16-byte accesses: rows of whole chunks on 16-byte boundaries, or dense tensors that start on one (rows cut at the boundaries)
bool set_classes(RowParams* p, int elem, uintptr_t bases, bool dense, uintptr_t strides) {
  const int v = 16 / elem;
  p->classes = 1;
  if (bases & 15) return false;
  if (p->channels % v == 0 && (strides & 15) == 0) return true;
  if (!dense) return false;
  for (int c = p->channels; (int64_t)c * p->classes % v != 0;) p->classes *= 2;
  return true;
}

template <typename F>
hdqt_status_t with_type(int dtype, F&& f) {
  if (dtype == HDQT_DTYPE_F32) return f.template operator()<float>();
  if (dtype == HDQT_DTYPE_BF16) return f.template operator()<__nv_bfloat16>();
  return f.template operator()<__half>();
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
  const bool dense = d->rows == 1 || (p.x_rs == d->channels && p.y_rs == d->channels && (!residual || p.r_rs == d->channels));
  const bool wide = set_classes(&p, elem, bases, dense, strides);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  return with_type(d->dtype, [&]<typename T>() { return fused ? run_fwd<T, true>(p, wide, s) : run_fwd<T, false>(p, wide, s); });
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
    const bool dense = d->rows == 1 || (p.x_rs == d->channels && p.y_rs == d->channels);
    const bool wide = set_classes(&p, elem, bases, dense, strides);
    const hdqt_status_t e = with_type(d->dtype, [&]<typename T>() {
      return fused ? run_bwd<T, true>(p, wide, &parts, s) : run_bwd<T, false>(p, wide, &parts, s);
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
  const int64_t parts = d->rows < kMostParts - 7 ? d->rows + 7 : kMostParts;      // (a block of every class, rows or not)
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
