// Group norm with an activation on channels-last activations x[batch, pixels, channels].
//
//   z = gamma (x - mu) rs + beta,  y = act(z);  dz = dy act'(z)
//   dx = rs (gamma dz - mean(gamma dz) - xhat mean(gamma dz xhat)),  dgamma = sum dz xhat,  dbeta = sum dz
//
// In both directions a thread keeps one column of V channels and walks down the pixels, so gamma, beta and the
// statistics of its channels stay in registers.  Bound by HBM: x is read and y written once, dy, x read and dx written.
//
// Cluster kernels: a cluster of up to 16 thread blocks takes whole groups of one image (a "slab" of channels, its pixels
// divided over the blocks): one pass for the statistics, which are joined over the cluster's shared memories, and a second
// pass over the same data (from L1 and L2 up to about 100 MB in flight, from HBM above).  One launch, backward two.
//
// Streaming kernels, for groups wider than a block's columns: per-channel partial statistics of a piece of an image, a
// join per group, and an elementwise pass.  8 x 64 x 64 x 4160 in two groups, SiLU: bf16 (273 MB) forward 301 us, backward 555
// (2.7 and 2.5 TB/s of the three and five passes over the data), fp32 410 and 930 us.  The widest accesses spill (48 to 224 bytes).
//
// Variance: a thread sums d = x - p and d^2 with p its own first value, so that its M2 = sum d^2 - (sum d)^2 / n never
// cancels by more than a factor n (p is one of the n values), and thread results are joined by Chan's formula.  Means
// travel relative to the group's first value (the "anchor"), so that a mean far larger than the spread costs no digits of it.
#include <cooperative_groups.h>
#include <math.h>

#include <atomic>

#include "hdqt_types.cuh"

namespace cg = cooperative_groups;

namespace hdqt {

namespace {

constexpr int NT = 256;           // threads of every kernel here
constexpr int kCols = 32;         // columns (of V channels) of a streaming block
constexpr int kPixelsPerRow = 32; // pixels a thread of a streaming block walks

struct NormParams {
  const void* x;
  const void* dy;
  void* out;               // y or dx
  const void* gamma;
  const void* beta;
  int32_t param_dtype, act;
  int64_t batch, pixels;
  int64_t x_bs, x_ps, y_bs, y_ps;   // batch and pixel strides of x, and of y, dy, dx
  int32_t channels, groups, per_group;
  float eps;
  float* mean;             // [batch, groups]
  float* rstd;
  float2* chan;            // streaming: [batch, chunks, channels] partial results
  float2* group;           // backward: [batch, groups] means of gamma dz and gamma dz xhat
  int32_t chunks, chunk_pixels;   // cluster kernels: blocks of a cluster, pixels of a block
  int32_t slabs, slab_groups;     // cluster kernels: slabs of an image, groups of a slab
  double inv_total;               // 1 / values of a group
  FastDiv div_slabs, div_cols, div_group, div_width;   // by slabs, columns of a slab, channels of a group, of a slab
  int32_t cluster_shift;          // log2 of chunks (cluster kernels)
};

__device__ __forceinline__ float gamma_of(const NormParams& p, int c) { return p.gamma ? load_param(p.gamma, p.param_dtype, c) : 1.0f; }
__device__ __forceinline__ float beta_of(const NormParams& p, int c) { return p.beta ? load_param(p.beta, p.param_dtype, c) : 0.0f; }

// Walks i = first, first + step, ... < end in batches whose loads are all issued before the first of them is used:
// what keeps HBM busy is the number of bytes in flight.
template <int U, typename L, typename F>
__device__ __forceinline__ void batched(int first, int end, int step, L&& load, F&& use) {
  int i = first;
  for (; i + (U - 1) * step < end; i += U * step) {
    decltype(load(0)) v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = load(i + u * step);
#pragma unroll
    for (int u = 0; u < U; ++u) use(i + u * step, v[u]);
  }
  if (i < end) {
    decltype(load(0)) v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u * step < end) v[u] = load(i + u * step);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u * step < end) use(i + u * step, v[u]);
  }
}
template <typename A>
struct Two {
  A x, dy;
};

// ---- streaming kernels -------------------------------------------------------------------------------------

struct Column {
  int cols, rows, row, col;   // columns of this block, thread rows, this thread's place
  int c0;                     // first channel of this thread's column
  bool live;
};
template <int V>
__device__ __forceinline__ Column column_of(const NormParams& p) {
  Column k;
  const int first = blockIdx.y * kCols;
  k.cols = min(kCols, p.channels / V - first);
  k.rows = NT / k.cols;
  k.row = threadIdx.x / k.cols;
  k.col = threadIdx.x - k.row * k.cols;
  k.c0 = (first + k.col) * V;
  k.live = k.row < k.rows;
  return k;
}

// first value of group g of image b
template <typename T>
__device__ __forceinline__ float anchor(const NormParams& p, int64_t b, int g) {
  return to_f32(reinterpret_cast<const T*>(p.x)[b * p.x_bs + g * p.per_group]);
}

// chan[b, chunk, c] = (mean - anchor, M2) of the chunk's pixels
template <typename T, int V>
__global__ void __launch_bounds__(NT, 3) norm_stats_kernel(const NormParams p) {
  chain_wait();
  __shared__ float s_mean[NT * V], s_m2[NT * V];
  const Column k = column_of<V>(p);
  const int64_t p0 = (int64_t)blockIdx.x * p.chunk_pixels;
  const int n = (int)min((int64_t)p.chunk_pixels, p.pixels - p0);
  for (int64_t b = blockIdx.z; b < p.batch; b += gridDim.z) {
    const T* src = reinterpret_cast<const T*>(p.x) + b * p.x_bs + p0 * p.x_ps + k.c0;
    float pivot[V], s1[V], s2[V];
    const int n_row = n / k.rows, n_more = n - n_row * k.rows;      // rows below n_more hold one pixel more
    const int cnt = n_row + (k.row < n_more ? 1 : 0);
    if (k.live && cnt > 0) {
      unpack(*reinterpret_cast<const Vec<T, V>*>(src + (int64_t)k.row * p.x_ps), pivot);
#pragma unroll
      for (int j = 0; j < V; ++j) s1[j] = s2[j] = 0.0f;
      batched<8>(k.row, n, k.rows, [&](int i) { return *reinterpret_cast<const Vec<T, V>*>(src + (int64_t)i * p.x_ps); },
                 [&](int, const Vec<T, V>& v) {
                   float x[V];
                   unpack(v, x);
#pragma unroll
                   for (int j = 0; j < V; ++j) {
                     const float d = x[j] - pivot[j];
                     s1[j] += d;
                     s2[j] = fmaf(d, d, s2[j]);
                   }
                 });
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float md = s1[j] / (float)cnt;
        s_mean[(k.row * k.cols + k.col) * V + j] = (pivot[j] - anchor<T>(p, b, (k.c0 + j) / p.per_group)) + md;
        s_m2[(k.row * k.cols + k.col) * V + j] = fmaxf(s2[j] - s1[j] * md, s2[j] != s2[j] ? s2[j] : 0.0f);
      }
    }
    __syncthreads();
    const int width = k.cols * V;
    for (int c = threadIdx.x; c < width; c += NT) {
      const int used = min(k.rows, n);
      float mean = 0.0f, m2 = 0.0f;
      for (int r = 0; r < used; ++r) mean += s_mean[r * width + c] * (float)(n_row + (r < n_more ? 1 : 0));
      mean /= (float)n;
      for (int r = 0; r < used; ++r) {
        const float d = s_mean[r * width + c] - mean;
        m2 += fmaf(d * d, (float)(n_row + (r < n_more ? 1 : 0)), s_m2[r * width + c]);
      }
      p.chan[(b * p.chunks + blockIdx.x) * p.channels + blockIdx.y * kCols * V + c] = make_float2(mean, m2);
    }
    __syncthreads();
  }
}

// (fp64: thousands of partial results may cancel against the anchor)
__device__ __forceinline__ double block_sum(double v) {
  __shared__ double s_part[NT / 32];
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int w = 0; w < NT / 32; ++w) v += s_part[w];
  __syncthreads();
  return v;
}

// one block per (image, group): joins the chunks' channel statistics
template <typename T>
__global__ void __launch_bounds__(NT) norm_join_stats_kernel(const NormParams p) {
  chain_wait();
  const int64_t b = blockIdx.x / p.groups;
  const int g = (int)(blockIdx.x - b * p.groups);
  const float2* part = p.chan + b * p.chunks * p.channels + (int64_t)g * p.per_group;
  const int64_t items = (int64_t)p.chunks * p.per_group;
  const double total = (double)(p.pixels * p.per_group);
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < items; i += NT) {
    const int64_t chunk = i / p.per_group, c = i - chunk * p.per_group;
    const double n = (double)min((int64_t)p.chunk_pixels, p.pixels - chunk * p.chunk_pixels);
    s += (double)part[chunk * p.channels + c].x * n;
  }
  const double mean = block_sum(s) / total;
  s = 0.0;
  for (int64_t i = threadIdx.x; i < items; i += NT) {
    const int64_t chunk = i / p.per_group, c = i - chunk * p.per_group;
    const double n = (double)min((int64_t)p.chunk_pixels, p.pixels - chunk * p.chunk_pixels);
    const float2 v = part[chunk * p.channels + c];
    const double d = (double)v.x - mean;
    s += d * d * n + (double)v.y;
  }
  const double var = block_sum(s) / total;
  if (threadIdx.x == 0) {
    p.mean[blockIdx.x] = (float)((double)anchor<T>(p, b, g) + mean);
    p.rstd[blockIdx.x] = rsqrtf((float)var + p.eps);
  }
}

template <typename T, int V>
__global__ void __launch_bounds__(NT, 3) norm_apply_kernel(const NormParams p) {
  chain_wait();
  const Column k = column_of<V>(p);
  if (!k.live) return;
  const int64_t p0 = (int64_t)blockIdx.x * p.chunk_pixels;
  const int n = (int)min((int64_t)p.chunk_pixels, p.pixels - p0);
  for (int64_t b = blockIdx.z; b < p.batch; b += gridDim.z) {
    const int64_t base = b * p.y_bs + p0 * p.y_ps + k.c0;
    const T* src = reinterpret_cast<const T*>(p.x) + b * p.x_bs + p0 * p.x_ps + k.c0;
    T* dst = reinterpret_cast<T*>(p.out) + base;
    float mu[V], a[V], be[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int64_t bg = b * p.groups + (k.c0 + j) / p.per_group;
      mu[j] = p.mean[bg];
      a[j] = p.rstd[bg] * gamma_of(p, k.c0 + j);
      be[j] = beta_of(p, k.c0 + j);
    }
    with_act(p.act, [&]<int kAct>() {
      batched<8>(k.row, n, k.rows, [&](int i) { return *reinterpret_cast<const Vec<T, V>*>(src + (int64_t)i * p.x_ps); },
                 [&](int i, const Vec<T, V>& v) {
                   float x[V];
                   unpack(v, x);
#pragma unroll
                   for (int j = 0; j < V; ++j) x[j] = act_fwd<kAct>(fmaf(x[j] - mu[j], a[j], be[j]));
                   *reinterpret_cast<Vec<T, V>*>(dst + (int64_t)i * p.y_ps) = pack<T>(x);
                 });
    });
  }
}

// chan[b, chunk, c] = (sum dz, sum dz xhat) of the chunk's pixels
template <typename T, int V>
__global__ void __launch_bounds__(NT, 2) norm_bwd_sums_kernel(const NormParams p) {
  chain_wait();
  __shared__ float s_a[NT * V], s_b[NT * V];
  const Column k = column_of<V>(p);
  const int64_t p0 = (int64_t)blockIdx.x * p.chunk_pixels;
  const int n = (int)min((int64_t)p.chunk_pixels, p.pixels - p0);
  for (int64_t b = blockIdx.z; b < p.batch; b += gridDim.z) {
    if (k.live) {
      const T* src = reinterpret_cast<const T*>(p.x) + b * p.x_bs + p0 * p.x_ps + k.c0;
      const T* dys = reinterpret_cast<const T*>(p.dy) + b * p.y_bs + p0 * p.y_ps + k.c0;
      float mu[V], rs[V], ga[V], be[V], sa[V], sb[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int64_t bg = b * p.groups + (k.c0 + j) / p.per_group;
        mu[j] = p.mean[bg];
        rs[j] = p.rstd[bg];
        ga[j] = gamma_of(p, k.c0 + j);
        be[j] = beta_of(p, k.c0 + j);
        sa[j] = sb[j] = 0.0f;
      }
      with_act(p.act, [&]<int kAct>() {
        batched<4>(k.row, n, k.rows,
                   [&](int i) {
                     return Two<Vec<T, V>>{*reinterpret_cast<const Vec<T, V>*>(src + (int64_t)i * p.x_ps),
                                           *reinterpret_cast<const Vec<T, V>*>(dys + (int64_t)i * p.y_ps)};
                   },
                   [&](int, const Two<Vec<T, V>>& v) {
                     float x[V], d[V];
                     unpack(v.x, x);
                     unpack(v.dy, d);
#pragma unroll
                     for (int j = 0; j < V; ++j) {
                       const float xh = (x[j] - mu[j]) * rs[j];
                       const float dz = act_bwd<kAct>(d[j], fmaf(xh, ga[j], be[j]));
                       sa[j] += dz;
                       sb[j] = fmaf(dz, xh, sb[j]);
                     }
                   });
      });
#pragma unroll
      for (int j = 0; j < V; ++j) {
        s_a[(k.row * k.cols + k.col) * V + j] = sa[j];
        s_b[(k.row * k.cols + k.col) * V + j] = sb[j];
      }
    }
    __syncthreads();
    const int width = k.cols * V;
    for (int c = threadIdx.x; c < width; c += NT) {
      float ta = 0.0f, tb = 0.0f;
      for (int r = 0; r < k.rows; ++r) { ta += s_a[r * width + c]; tb += s_b[r * width + c]; }
      p.chan[(b * p.chunks + blockIdx.x) * p.channels + blockIdx.y * kCols * V + c] = make_float2(ta, tb);
    }
    __syncthreads();
  }
}

// one block per (image, group): group[b, g] = means of gamma dz and gamma dz xhat
__global__ void __launch_bounds__(NT) norm_join_sums_kernel(const NormParams p) {
  chain_wait();
  const int64_t b = blockIdx.x / p.groups;
  const int g = (int)(blockIdx.x - b * p.groups);
  const float2* part = p.chan + b * p.chunks * p.channels + (int64_t)g * p.per_group;
  const int64_t items = (int64_t)p.chunks * p.per_group;
  double s1 = 0.0, s2 = 0.0;
  for (int64_t i = threadIdx.x; i < items; i += NT) {
    const int64_t chunk = i / p.per_group, c = i - chunk * p.per_group;
    const float2 v = part[chunk * p.channels + c];
    const double ga = gamma_of(p, g * p.per_group + (int)c);
    s1 += v.x * ga;
    s2 += v.y * ga;
  }
  s1 = block_sum(s1);
  s2 = block_sum(s2);
  const double inv = 1.0 / (double)(p.pixels * p.per_group);
  if (threadIdx.x == 0) p.group[blockIdx.x] = make_float2((float)(s1 * inv), (float)(s2 * inv));
}

template <typename T, int V>
__global__ void __launch_bounds__(NT, 2) norm_bwd_apply_kernel(const NormParams p) {
  chain_wait();
  const Column k = column_of<V>(p);
  if (!k.live) return;
  const int64_t p0 = (int64_t)blockIdx.x * p.chunk_pixels;
  const int n = (int)min((int64_t)p.chunk_pixels, p.pixels - p0);
  for (int64_t b = blockIdx.z; b < p.batch; b += gridDim.z) {
    const int64_t base = b * p.y_bs + p0 * p.y_ps + k.c0;
    const T* src = reinterpret_cast<const T*>(p.x) + b * p.x_bs + p0 * p.x_ps + k.c0;
    const T* dys = reinterpret_cast<const T*>(p.dy) + base;
    T* dst = reinterpret_cast<T*>(p.out) + base;
    float mu[V], rs[V], ga[V], be[V], m1[V], m2[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int64_t bg = b * p.groups + (k.c0 + j) / p.per_group;
      mu[j] = p.mean[bg];
      rs[j] = p.rstd[bg];
      ga[j] = gamma_of(p, k.c0 + j);
      be[j] = beta_of(p, k.c0 + j);
      const float2 m = p.group[bg];
      m1[j] = m.x;
      m2[j] = m.y;
    }
    with_act(p.act, [&]<int kAct>() {
      batched<4>(k.row, n, k.rows,
                 [&](int i) {
                   return Two<Vec<T, V>>{*reinterpret_cast<const Vec<T, V>*>(src + (int64_t)i * p.x_ps),
                                         *reinterpret_cast<const Vec<T, V>*>(dys + (int64_t)i * p.y_ps)};
                 },
                 [&](int i, const Two<Vec<T, V>>& v) {
                   float x[V], d[V];
                   unpack(v.x, x);
                   unpack(v.dy, d);
#pragma unroll
                   for (int j = 0; j < V; ++j) {
                     const float xh = (x[j] - mu[j]) * rs[j];
                     const float dz = act_bwd<kAct>(d[j], fmaf(xh, ga[j], be[j]));
                     x[j] = rs[j] * (fmaf(dz, ga[j], -m1[j]) - xh * m2[j]);
                   }
                   *reinterpret_cast<Vec<T, V>*>(dst + (int64_t)i * p.y_ps) = pack<T>(x);
                 });
    });
  }
}

// ---- cluster kernels ---------------------------------------------------------------------------------------
// Block r of a cluster takes pixels [r chunk_pixels, ...) of one slab.

constexpr int kMaxCluster = 16;
constexpr int kMaxClusterSmem = 100 << 10;
constexpr int64_t kLongBlock = 256 << 10;      // bytes of x from which a forward block is worth dividing further

struct Slab {
  int64_t b;
  int rank, g0, c0, width, cols, rows, row, col, np;
  int64_t p0;
  bool live;
};
template <int V>
__device__ __forceinline__ Slab slab_of(const NormParams& p) {
  Slab k;
  k.rank = (int)(blockIdx.x & (unsigned)(p.chunks - 1));
  uint32_t b, slab, row, col;
  fastdivmod(blockIdx.x >> p.cluster_shift, p.div_slabs, b, slab);
  k.b = b;
  k.g0 = (int)slab * p.slab_groups;
  k.c0 = k.g0 * p.per_group;
  k.width = p.slab_groups * p.per_group;
  k.cols = k.width / V;
  k.rows = (int)fastdiv(NT, p.div_cols);
  fastdivmod(threadIdx.x, p.div_cols, row, col);
  k.row = (int)row;
  k.col = (int)col;
  k.live = k.row < k.rows;
  k.p0 = (int64_t)k.rank * p.chunk_pixels;
  const int64_t n = p.pixels - k.p0;
  k.np = n < 0 ? 0 : n < p.chunk_pixels ? (int)n : p.chunk_pixels;
  return k;
}

// lanes that share one group's (or channel's) entries: the largest power of two <= NT / n, at most a warp
__device__ __forceinline__ int lanes_for(int n) {
  int l = 32;
  while (l > 1 && l * n > NT) l >>= 1;
  return l;
}

// kOne: the V channels of a thread lie in one group.  Four blocks per SM (64 registers).
template <typename T, int V, bool kOne>
__global__ void __launch_bounds__(NT, 4) norm_fwd_cluster_kernel(const __grid_constant__ NormParams p) {
  extern __shared__ __align__(16) uint8_t smem[];
  const Slab k = slab_of<V>(p);
  using A = Vec<T, V>;
  float2* s_part = reinterpret_cast<float2*>(smem);
  double2* s_group = reinterpret_cast<double2*>(s_part + NT * V);   // this block's sum of n m, and of M2 + n m^2
  float2* s_stat = reinterpret_cast<float2*>(s_group + p.slab_groups);   // (mean, rstd)
  float* s_anchor = reinterpret_cast<float*>(s_stat + p.slab_groups);
  float* s_gamma = s_anchor + p.slab_groups;                              // [channel]
  float* s_beta = s_gamma + k.width;
  const T* src = reinterpret_cast<const T*>(p.x) + k.b * p.x_bs + k.p0 * p.x_ps + k.c0 + k.col * V;
  for (int g = threadIdx.x; g < p.slab_groups; g += NT) s_anchor[g] = anchor<T>(p, k.b, k.g0 + g);
  for (int c = threadIdx.x; c < k.width; c += NT) {
    s_gamma[c] = gamma_of(p, k.c0 + c);
    s_beta[c] = beta_of(p, k.c0 + c);
  }
  float pivot[V], s1[V], s2[V];
#pragma unroll
  for (int j = 0; j < V; ++j) pivot[j] = s1[j] = s2[j] = 0.0f;
  const int cnt = k.live && k.row < k.np ? (k.np - k.row + k.rows - 1) / k.rows : 0;    // pixels of this thread
  auto add = [&](const A& v) {
    float x[V];
    unpack(v, x);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float d = x[j] - pivot[j];
      s1[j] += d;
      s2[j] = fmaf(d, d, s2[j]);
    }
  };
  if (cnt > 0) {
    unpack(*reinterpret_cast<const A*>(src + (int64_t)k.row * p.x_ps), pivot);
    batched<sizeof(T) == 4 ? 8 : 4>(k.row, k.np, k.rows, [&](int i) { return *reinterpret_cast<const A*>(src + (int64_t)i * p.x_ps); },
               [&](int, const A& v) { add(v); });
  }
  __syncthreads();      // the anchors
  // one entry per thread and group where the thread's channels lie in one group, else one per channel
  constexpr int entries = kOne ? 1 : V;            // per thread
  const int my_group = k.live ? (int)fastdiv((uint32_t)(k.col * V), p.div_group) : 0;   // of the thread's first channel
  if (k.live && cnt > 0) {
    const float inv = __fdividef(1.0f, (float)cnt);
    float m[V], m2[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float md = s1[j] * inv;
      m[j] = (pivot[j] - s_anchor[kOne ? my_group : (int)fastdiv((uint32_t)(k.col * V + j), p.div_group)]) + md;
      m2[j] = s2[j] - s1[j] * md;
      if (m2[j] < 0.0f) m2[j] = 0.0f;
    }
    float2* e = s_part + (k.row * k.cols + k.col) * entries;
    if constexpr (kOne) {
      float mm = 0.0f, mm2 = 0.0f;
#pragma unroll
      for (int j = 0; j < V; ++j) mm += m[j];
      mm *= 1.0f / V;
#pragma unroll
      for (int j = 0; j < V; ++j) mm2 += fmaf((m[j] - mm) * (m[j] - mm), (float)cnt, m2[j]);
      e[0] = make_float2(mm, mm2);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) e[j] = make_float2(m[j], m2[j]);
    }
  }
  __syncthreads();
  // Groups: `lanes` threads each.  An entry stands for n values with mean m (relative to the anchor) and M2; in fp64
  // sum(M2 + n m^2) - (sum n m)^2 / N loses nothing, so one pass over the entries does.
  const int eg = p.per_group * entries / V;         // entries of a group in one row
  const int row_entries = k.cols * entries;
  const int used_rows = min(k.rows, k.np);
  const int n_row = k.np / k.rows, n_more = k.np - n_row * k.rows;    // rows below n_more hold one pixel more
  constexpr int weight = kOne ? V : 1;
  {
    const int lanes = lanes_for(p.slab_groups);
    const int sub = threadIdx.x & (lanes - 1);
    const int per_round = NT / lanes, dr = lanes / eg, de = lanes - dr * eg;
    for (int g0 = 0; g0 < p.slab_groups; g0 += per_round) {
      const int g = g0 + (int)threadIdx.x / lanes;
      double n1 = 0.0, n2 = 0.0;
      if (g < p.slab_groups) {
        int r = sub / eg, e = sub - r * eg;
        const float2* base = s_part + g * eg;
        while (r < used_rows) {
          const float2 v = base[r * row_entries + e];
          const double n = (double)((n_row + (r < n_more ? 1 : 0)) * weight), m = (double)v.x;
          n1 += n * m;
          n2 += n * m * m + (double)v.y;
          e += de;
          r += dr;
          if (e >= eg) { e -= eg; ++r; }
        }
      }
      for (int d = lanes >> 1; d > 0; d >>= 1) {
        n1 += __shfl_xor_sync(0xFFFFFFFFu, n1, d);
        n2 += __shfl_xor_sync(0xFFFFFFFFu, n2, d);
      }
      if (g < p.slab_groups && sub == 0) s_group[g] = make_double2(n1, n2);
    }
  }
  cg::cluster_group cluster = cg::this_cluster();
  if (p.chunks > 1) cluster.sync();
  else __syncthreads();
  for (int g = threadIdx.x; g < p.slab_groups; g += NT) {
    // joined in rank order: the same bits in every block
    const float first = s_anchor[g];
    double n1 = 0.0, n2 = 0.0;
    for (int r = 0; r < p.chunks; ++r) {
      const double2 v = p.chunks > 1 ? *cluster.map_shared_rank(s_group + g, r) : s_group[g];
      n1 += v.x;
      n2 += v.y;
    }
    const double mean = n1 * p.inv_total;
    const float mu = (float)((double)first + mean);
    const float var = (float)((n2 - n1 * mean) * p.inv_total);
    const float rs = rsqrtf((var < 0.0f ? 0.0f : var) + p.eps);      // (a NaN stays)
    s_stat[g] = make_float2(mu, rs);
    if (k.rank == 0) {
      p.mean[k.b * p.groups + k.g0 + g] = mu;
      p.rstd[k.b * p.groups + k.g0 + g] = rs;
    }
  }
  __syncthreads();
  if (k.live) {
    float mu[V], a[V], be[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float2 st = s_stat[kOne ? my_group : (int)fastdiv((uint32_t)(k.col * V + j), p.div_group)];
      mu[j] = st.x;
      a[j] = st.y * s_gamma[k.col * V + j];
      be[j] = s_beta[k.col * V + j];
    }
    T* dst = reinterpret_cast<T*>(p.out) + k.b * p.y_bs + k.p0 * p.y_ps + k.c0 + k.col * V;
    with_act(p.act, [&]<int kAct>() {
      batched<4>(
          k.row, k.np, k.rows, [&](int i) { return *reinterpret_cast<const A*>(src + (int64_t)i * p.x_ps); },
          [&](int i, const A& v) {
            float x[V];
            unpack(v, x);
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] = act_fwd<kAct>(fmaf(x[j] - (kOne ? mu[0] : mu[j]), a[j], be[j]));
            *reinterpret_cast<A*>(dst + (int64_t)i * p.y_ps) = pack<T>(x);
          });
    });
  }
  if (p.chunks > 1) cluster.sync();     // the other blocks may still be reading this one's statistics
}

// chan[b * chunks + rank, c] = (sum dz, sum dz xhat) of this block's pixels, and dx
template <typename T, int V, bool kOne>
__global__ void __launch_bounds__(NT, 2) norm_bwd_cluster_kernel(const __grid_constant__ NormParams p) {
  extern __shared__ __align__(16) uint8_t smem[];
  chain_wait();
  const Slab k = slab_of<V>(p);
  using A = Vec<T, V>;
  float2* s_part = reinterpret_cast<float2*>(smem);                // [j][row][column]
  float2* s_chan = s_part + NT * V;                                // [channel]
  float2* s_group = s_chan + k.width;
  float2* s_mean = s_group + p.slab_groups;
  float2* s_stat = s_mean + p.slab_groups;                         // (mean, rstd)
  float* s_gamma = reinterpret_cast<float*>(s_stat + p.slab_groups);   // [channel]
  float* s_beta = s_gamma + k.width;
  float2* s_slice = reinterpret_cast<float2*>(s_beta + k.width);       // [slice][channel], at least NT of them
  const T* src = reinterpret_cast<const T*>(p.x) + k.b * p.x_bs + k.p0 * p.x_ps + k.c0 + k.col * V;
  const T* dys = reinterpret_cast<const T*>(p.dy) + k.b * p.y_bs + k.p0 * p.y_ps + k.c0 + k.col * V;
  for (int g = threadIdx.x; g < p.slab_groups; g += NT) {
    const int64_t bg = k.b * p.groups + k.g0 + g;
    s_stat[g] = make_float2(p.mean[bg], p.rstd[bg]);
  }
  for (int c = threadIdx.x; c < k.width; c += NT) {
    s_gamma[c] = gamma_of(p, k.c0 + c);
    s_beta[c] = beta_of(p, k.c0 + c);
  }
  __syncthreads();
  // xhat = (x - mu) rs,  z = xhat ga + be (x - mu first: it cancels exactly where it cancels)
  float mu[V], rs[V], ga[V], be[V], sa[V], sb[V];
#pragma unroll
  for (int j = 0; j < V; ++j) sa[j] = sb[j] = 0.0f;
  const int my_group = k.live ? (int)fastdiv((uint32_t)(k.col * V), p.div_group) : 0;
  if (k.live) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float2 st = s_stat[kOne ? my_group : (int)fastdiv((uint32_t)(k.col * V + j), p.div_group)];
      rs[j] = st.y;
      mu[j] = st.x;
      ga[j] = s_gamma[k.col * V + j];
      be[j] = s_beta[k.col * V + j];
    }
  }
  with_act(p.act, [&]<int kAct>() {
    auto add = [&](const A& vx, const A& vd) {
      float x[V], d[V];
      unpack(vx, x);
      unpack(vd, d);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float xh = (x[j] - (kOne ? mu[0] : mu[j])) * (kOne ? rs[0] : rs[j]);
        const float dz = act_bwd<kAct>(d[j], fmaf(xh, ga[j], be[j]));
        sa[j] += dz;
        sb[j] = fmaf(dz, xh, sb[j]);
      }
    };
    if (k.live) {
      batched<4>(k.row, k.np, k.rows,
                 [&](int i) {
                   return Two<A>{*reinterpret_cast<const A*>(src + (int64_t)i * p.x_ps),
                                 *reinterpret_cast<const A*>(dys + (int64_t)i * p.y_ps)};
                 },
                 [&](int, const Two<A>& v) { add(v.x, v.dy); });
    }
  });
  // Channels: sums over the rows of threads.  Layout [j][row][column], so that neighbouring threads touch neighbouring
  // words both ways; with few channels, slices of the rows are summed first.
  if (k.live) {
#pragma unroll
    for (int j = 0; j < V; ++j) s_part[j * NT + k.row * k.cols + k.col] = make_float2(sa[j], sb[j]);
  }
  __syncthreads();
  const int slices = k.width >= NT ? 1 : NT / k.width;
  {
    uint32_t slice, first;
    fastdivmod(threadIdx.x, p.div_width, slice, first);
    if ((int)slice < slices) {
      for (int q = (int)first; q < k.width; q += NT) {
        uint32_t j, col;
        fastdivmod((uint32_t)q, p.div_cols, j, col);      // q-th channel in the order [j][column]
        float a = 0.0f, b = 0.0f;
        for (int r = (int)slice; r < k.rows; r += slices) {
          const float2 v = s_part[j * NT + r * k.cols + col];
          a += v.x;
          b += v.y;
        }
        s_slice[slice * k.width + q] = make_float2(a, b);
      }
    }
    __syncthreads();
    for (int q = threadIdx.x; q < k.width; q += NT) {
      uint32_t j, col;
      fastdivmod((uint32_t)q, p.div_cols, j, col);
      float2 t = s_slice[q];
      for (int i = 1; i < slices; ++i) {
        const float2 v = s_slice[i * k.width + q];
        t.x += v.x;
        t.y += v.y;
      }
      const int c = (int)col * V + (int)j;
      s_chan[c] = t;
      p.chan[(k.b * p.chunks + k.rank) * p.channels + k.c0 + c] = t;
    }
  }
  if (p.out == nullptr) return;      // (the whole grid)
  __syncthreads();
  {
    const int lanes = lanes_for(p.slab_groups);
    const int sub = threadIdx.x & (lanes - 1);
    const int rounds = (p.slab_groups * lanes + NT - 1) / NT;
    for (int round = 0; round < rounds; ++round) {
      const int g = (round * NT + (int)threadIdx.x) / lanes;
      float a = 0.0f, b = 0.0f;
      if (g < p.slab_groups)
        for (int i = sub; i < p.per_group; i += lanes) {
          const float2 v = s_chan[g * p.per_group + i];
          const float w = s_gamma[g * p.per_group + i];
          a = fmaf(v.x, w, a);
          b = fmaf(v.y, w, b);
        }
      for (int d = lanes >> 1; d > 0; d >>= 1) {
        a += __shfl_xor_sync(0xFFFFFFFFu, a, d);
        b += __shfl_xor_sync(0xFFFFFFFFu, b, d);
      }
      if (g < p.slab_groups && sub == 0) s_group[g] = make_float2(a, b);
    }
  }
  cg::cluster_group cluster = cg::this_cluster();
  if (p.chunks > 1) cluster.sync();
  else __syncthreads();
  for (int g = threadIdx.x; g < p.slab_groups; g += NT) {
    double a = 0.0, b = 0.0;
    for (int r = 0; r < p.chunks; ++r) {
      const float2 v = p.chunks > 1 ? *cluster.map_shared_rank(s_group + g, r) : s_group[g];
      a += v.x;
      b += v.y;
    }
    s_mean[g] = make_float2((float)(a * p.inv_total), (float)(b * p.inv_total));
  }
  __syncthreads();
  if (k.live) {
    float m1[V], m2[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float2 m = s_mean[kOne ? my_group : (int)fastdiv((uint32_t)(k.col * V + j), p.div_group)];
      m1[j] = m.x;
      m2[j] = m.y;
    }
    T* dst = reinterpret_cast<T*>(p.out) + k.b * p.y_bs + k.p0 * p.y_ps + k.c0 + k.col * V;
    with_act(p.act, [&]<int kAct>() {
      batched<4>(
          k.row, k.np, k.rows,
          [&](int i) {
            return Two<A>{*reinterpret_cast<const A*>(src + (int64_t)i * p.x_ps), *reinterpret_cast<const A*>(dys + (int64_t)i * p.y_ps)};
          },
          [&](int i, const Two<A>& v) {
            float x[V], d[V];
            unpack(v.x, x);
            unpack(v.dy, d);
#pragma unroll
            for (int j = 0; j < V; ++j) {
              const float r = kOne ? rs[0] : rs[j];
              const float xh = (x[j] - (kOne ? mu[0] : mu[j])) * r;
              const float dz = act_bwd<kAct>(d[j], fmaf(xh, ga[j], be[j]));
              x[j] = r * (fmaf(dz, ga[j], -(kOne ? m1[0] : m1[j])) - xh * (kOne ? m2[0] : m2[j]));
            }
            *reinterpret_cast<A*>(dst + (int64_t)i * p.y_ps) = pack<T>(x);
          });
    });
  }
  if (p.chunks > 1) cluster.sync();
}

// dgamma, dbeta: sum of the parts [parts, channels] of all images; 8 channels x 32 rows of threads per block, so that
// a few hundred parts are one or two rounds of loads
constexpr int kGradChannels = 8;
__global__ void __launch_bounds__(NT) norm_param_grad_kernel(const float2* __restrict__ part, int64_t parts, int channels,
                                                             void* dgamma, void* dbeta, int32_t param_dtype) {
  __shared__ float2 s[NT / 32][kGradChannels];
  chain_wait();
  const int lane = threadIdx.x & (kGradChannels - 1), row = threadIdx.x / kGradChannels;
  const int c = blockIdx.x * kGradChannels + lane;
  float a = 0.0f, b = 0.0f;
  if (c < channels) {
#pragma unroll 8
    for (int64_t i = row; i < parts; i += NT / kGradChannels) {
      const float2 v = part[i * channels + c];
      a += v.x;
      b += v.y;
    }
  }
#pragma unroll
  for (int d = 16; d >= kGradChannels; d >>= 1) {
    a += __shfl_xor_sync(0xFFFFFFFFu, a, d);
    b += __shfl_xor_sync(0xFFFFFFFFu, b, d);
  }
  if ((threadIdx.x & 31) < kGradChannels) s[threadIdx.x >> 5][lane] = make_float2(a, b);
  __syncthreads();
  if (threadIdx.x < kGradChannels && c < channels) {
    for (int w = 1; w < NT / 32; ++w) { a += s[w][lane].x; b += s[w][lane].y; }
    if (dbeta) store_param(dbeta, param_dtype, c, a);
    if (dgamma) store_param(dgamma, param_dtype, c, b);
  }
}

__global__ void fill_nan_kernel(float* a, float* b, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) {
    a[i] = NAN;
    b[i] = NAN;
  }
}

// ---- host side ---------------------------------------------------------------------------------------------

struct Plan {
  int vec;                 // channels per access
  int chunks, chunk_pixels;
};

Plan make_plan(const hdqt_group_norm_desc_t& d, int vec) {
  Plan pl;
  pl.vec = vec;
  const int64_t ncol = d.channels / vec;
  const int cols = (int)(ncol < kCols ? ncol : kCols);
  pl.chunk_pixels = (NT / cols) * kPixelsPerRow;
  pl.chunks = (int)((d.pixels + pl.chunk_pixels - 1) / pl.chunk_pixels);
  return pl;
}

// chunks for the narrowest access: an upper bound of the partial results whatever the alignment turns out to be
int64_t most_chunks(const hdqt_group_norm_desc_t& d) {
  const int64_t a = make_plan(d, 1).chunks;
  const int elem = dtype_size(d.dtype);
  int64_t most = a;
  for (int v = 16 / elem; v > 1; v >>= 1)
    if (d.channels % v == 0) {
      const int64_t b = make_plan(d, v).chunks;
      if (b > most) most = b;
    }
  return most > kMaxCluster ? most : kMaxCluster;     // (a cluster's blocks leave one each)
}

hdqt_status_t check_desc(const hdqt_group_norm_desc_t* d) {
  if (!d) return HDQT_ERR_INVALID_ARG;
  if (d->batch < 0 || d->pixels < 0 || d->channels <= 0 || d->groups <= 0 || d->channels % d->groups != 0) return HDQT_ERR_INVALID_ARG;
  if (dtype_size(d->dtype) == 0) return HDQT_ERR_INVALID_ARG;
  if (d->param_dtype != HDQT_DTYPE_F32 && d->param_dtype != d->dtype) return HDQT_ERR_INVALID_ARG;
  if (d->act < HDQT_ACT_NONE || d->act > HDQT_ACT_SILU || !(d->eps >= 0.0f)) return HDQT_ERR_INVALID_ARG;
  if (d->x_pixel_stride < d->channels || d->y_pixel_stride < d->channels) return HDQT_ERR_INVALID_ARG;
  if (d->batch > 1 && (d->x_batch_stride < d->pixels * d->x_pixel_stride || d->y_batch_stride < d->pixels * d->y_pixel_stride))
    return HDQT_ERR_INVALID_ARG;
  if (d->channels > (1 << 20) || d->pixels > (1ll << 31) || d->batch * d->groups > 0x7FFFFFFFll) return HDQT_ERR_UNSUPPORTED;
  return HDQT_OK;
}

NormParams make_params(const hdqt_group_norm_desc_t& d, const Plan& pl) {
  NormParams p{};
  p.param_dtype = d.param_dtype;
  p.act = d.act;
  p.batch = d.batch;
  p.pixels = d.pixels;
  p.x_bs = d.x_batch_stride;
  p.x_ps = d.x_pixel_stride;
  p.y_bs = d.y_batch_stride;
  p.y_ps = d.y_pixel_stride;
  p.channels = (int32_t)d.channels;
  p.groups = (int32_t)d.groups;
  p.per_group = (int32_t)(d.channels / d.groups);
  p.eps = d.eps;
  p.inv_total = 1.0 / ((double)d.pixels * (double)p.per_group);
  p.chunks = pl.chunks;
  p.chunk_pixels = pl.chunk_pixels;
  return p;
}

dim3 stream_grid(const hdqt_group_norm_desc_t& d, const Plan& pl) {
  const int64_t ncol = d.channels / pl.vec;
  return dim3((unsigned)pl.chunks, (unsigned)((ncol + kCols - 1) / kCols), (unsigned)(d.batch < 65535 ? d.batch : 65535));
}

uintptr_t stride_bits(const hdqt_group_norm_desc_t& d) {
  const int e = dtype_size(d.dtype);
  return (uintptr_t)((d.x_pixel_stride | d.y_pixel_stride) * e) |
         (d.batch > 1 ? (uintptr_t)((d.x_batch_stride | d.y_batch_stride) * e) : 0);
}

// How the cluster kernels divide a call; cluster == 0: not at all (streaming kernels).
struct Division {
  int cluster, slabs;
  size_t smem;
};

Division division(const hdqt_group_norm_desc_t& d, int vec, int cluster, int slabs, bool backward) {
  const int64_t width = d.channels / slabs, groups = d.groups / slabs;
  return Division{cluster, slabs,
                  (size_t)NT * vec * 8 + (size_t)groups * 28 + (size_t)width * (backward ? 16 : 8) +
                      (backward ? 8 * (size_t)(width > NT ? width : NT) : 0)};
}

// The fewest blocks that fill the machine, with rows of a slab as long as that allows; slabs before clusters (no exchange).
// One wave (two blocks per SM backward, up to four forward) was fastest at every size measured: 16 x 128 x 128 x 512 bf16
// forward 156 us with 512 blocks, 168 with 1024, 206 with 256; backward 288 with 256 blocks, 296 with 512, 311 with rows of
// 128 bytes; 128 x 32 x 32 x 64 fp32 forward 18 us with 256 or 512 blocks, 23 with 1024.
Division choose_division(const hdqt_group_norm_desc_t& d, int vec, bool backward) {
  const int elem = dtype_size(d.dtype);
  Division best{0, 0, 0};
  int64_t best_blocks = 0;
  for (int segment = 256; segment >= 32; segment /= 2) {
    for (int cluster = 1; cluster <= kMaxCluster; cluster *= 2) {
      if (cluster > 1 && d.pixels < 4 * cluster) break;
      for (int64_t slabs = 1; slabs <= d.groups; ++slabs) {
        if (d.groups % slabs != 0) continue;
        const int64_t width = d.channels / slabs;
        if (width % vec != 0 || width / vec > NT) continue;
        if (slabs > 1 && width * elem < segment) break;
        const int64_t blocks = d.batch * slabs * cluster;
        if (blocks > 0x7FFFFFFFll) continue;
        const Division now = division(d, vec, cluster, (int)slabs, backward);
        if (now.smem > (size_t)kMaxClusterSmem) continue;
        const int64_t bytes = (d.pixels + cluster - 1) / cluster * width * elem;
        if (blocks >= (!backward && bytes > kLongBlock ? 3 * 148 : 3 * 148 / 2)) return now;
        if (blocks > best_blocks) { best = now; best_blocks = blocks; }
      }
    }
  }
  return best;
}

template <auto kernel>
hdqt_status_t launch_cluster(const NormParams& p, const Division& dv, int64_t batch, cudaStream_t s) {
  // the attributes hold per device for as long as the library is loaded: set at a kernel's first launch there
  static std::atomic<uint64_t> ready{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev > 63 || !((ready.load(std::memory_order_relaxed) >> dev) & 1))) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxClusterSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess && dev <= 63) ready.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  if (e != cudaSuccess) return cuda_failure(e, "group norm");
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(batch * dv.slabs * dv.cluster));
  cfg.blockDim = dim3(NT);
  cfg.dynamicSmemBytes = dv.smem;
  cfg.stream = s;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)dv.cluster;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, kernel, p);
  return e == cudaSuccess ? HDQT_OK : cuda_failure(e, "group norm");
}

void set_division(NormParams* p, const hdqt_group_norm_desc_t& d, const Division& dv, int vec) {
  p->chunks = dv.cluster;
  p->chunk_pixels = (int32_t)((d.pixels + dv.cluster - 1) / dv.cluster);
  p->slabs = dv.slabs;
  p->slab_groups = (int32_t)(d.groups / dv.slabs);
  p->div_slabs = make_fastdiv((uint32_t)dv.slabs);
  p->div_cols = make_fastdiv((uint32_t)(d.channels / dv.slabs / vec));
  p->div_group = make_fastdiv((uint32_t)p->per_group);
  p->div_width = make_fastdiv((uint32_t)(d.channels / dv.slabs));
  p->cluster_shift = 0;
  while ((1 << p->cluster_shift) < dv.cluster) ++p->cluster_shift;
}

}  // namespace

void launch_param_grad(const float2* part, int64_t parts, int channels, void* dgamma, void* dbeta, int32_t param_dtype, bool chained,
                       cudaStream_t s) {
  const unsigned blocks = (unsigned)((channels + kGradChannels - 1) / kGradChannels);
  if (chained) launch_chained(norm_param_grad_kernel, blocks, NT, 0, s, part, parts, channels, dgamma, dbeta, param_dtype);
  else norm_param_grad_kernel<<<blocks, NT, 0, s>>>(part, parts, channels, dgamma, dbeta, param_dtype);
}

}  // namespace hdqt

using namespace hdqt;

extern "C" size_t hdqt_group_norm_workspace_bytes(const hdqt_group_norm_desc_t* d, int32_t backward) {
  if (check_desc(d) != HDQT_OK) return 0;
  const size_t chan = align256((size_t)d->batch * most_chunks(*d) * d->channels * sizeof(float2));
  const size_t group = backward ? align256((size_t)d->batch * d->groups * sizeof(float2)) : 0;
  return chan + group + 256;
}

extern "C" hdqt_status_t hdqt_group_norm_fwd(const hdqt_group_norm_desc_t* d, const void* x, const void* gamma,
                                             const void* beta, void* y, float* mean, float* rstd, void* workspace,
                                             size_t workspace_bytes, void* stream) {
  hdqt_status_t st = check_desc(d);
  if (st != HDQT_OK) return st;
  if (!workspace || (d->batch > 0 && (!mean || !rstd))) return HDQT_ERR_INVALID_ARG;
  const bool empty = d->batch == 0 || d->pixels == 0;
  if (!empty && (!x || !y)) return HDQT_ERR_INVALID_ARG;
  const int elem = dtype_size(d->dtype), pelem = dtype_size(d->param_dtype);
  const uintptr_t bases = reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(y);
  if ((bases & (uintptr_t)(elem - 1)) || ((reinterpret_cast<uintptr_t>(gamma) | reinterpret_cast<uintptr_t>(beta)) & (uintptr_t)(pelem - 1)) ||
      ((reinterpret_cast<uintptr_t>(mean) | reinterpret_cast<uintptr_t>(rstd)) & 3) || (reinterpret_cast<uintptr_t>(workspace) & 255))
    return HDQT_ERR_ALIGNMENT;
  if (workspace_bytes < hdqt_group_norm_workspace_bytes(d, 0)) return HDQT_ERR_WORKSPACE;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (empty) {
    if (d->batch > 0) fill_nan_kernel<<<64, NT, 0, s>>>(mean, rstd, d->batch * d->groups);
    return last_error("group norm");
  }
  const int vec = vector_width(d->channels, elem, bases | stride_bits(*d));
  const Plan pl = make_plan(*d, vec);
  NormParams p = make_params(*d, pl);
  p.x = x;
  p.gamma = gamma;
  p.beta = beta;
  p.out = y;
  p.mean = mean;
  p.rstd = rstd;
  p.chan = reinterpret_cast<float2*>(workspace);
  const Division dv = choose_division(*d, vec, false);
  if (dv.cluster > 0) {
    set_division(&p, *d, dv, vec);
    return with_type_and_width(d->dtype, vec, [&]<typename T, int V>() {
      return p.per_group % V == 0 ? launch_cluster<norm_fwd_cluster_kernel<T, V, true>>(p, dv, d->batch, s)
                                  : launch_cluster<norm_fwd_cluster_kernel<T, V, false>>(p, dv, d->batch, s);
    });
  }
  const dim3 grid = stream_grid(*d, pl);
  return with_type_and_width(d->dtype, vec, [&]<typename T, int V>() {
    norm_stats_kernel<T, V><<<grid, NT, 0, s>>>(p);
    launch_chained(norm_join_stats_kernel<T>, (unsigned)(d->batch * d->groups), NT, 0, s, p);
    launch_chained(norm_apply_kernel<T, V>, grid, NT, 0, s, p);
    return last_error("group norm");
  });
}

extern "C" hdqt_status_t hdqt_group_norm_bwd(const hdqt_group_norm_desc_t* d, const void* dy, const void* x,
                                             const void* gamma, const void* beta, const float* mean, const float* rstd,
                                             void* dx, void* dgamma, void* dbeta, void* workspace,
                                             size_t workspace_bytes, void* stream) {
  hdqt_status_t st = check_desc(d);
  if (st != HDQT_OK) return st;
  if (!workspace) return HDQT_ERR_INVALID_ARG;
  const bool empty = d->batch == 0 || d->pixels == 0;
  if (!empty && (!x || !dy || !mean || !rstd)) return HDQT_ERR_INVALID_ARG;
  const int elem = dtype_size(d->dtype), pelem = dtype_size(d->param_dtype);
  const uintptr_t bases = reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(dy) | reinterpret_cast<uintptr_t>(dx);
  const uintptr_t pbases = reinterpret_cast<uintptr_t>(gamma) | reinterpret_cast<uintptr_t>(beta) |
                           reinterpret_cast<uintptr_t>(dgamma) | reinterpret_cast<uintptr_t>(dbeta);
  if ((bases & (uintptr_t)(elem - 1)) || (pbases & (uintptr_t)(pelem - 1)) ||
      ((reinterpret_cast<uintptr_t>(mean) | reinterpret_cast<uintptr_t>(rstd)) & 3) || (reinterpret_cast<uintptr_t>(workspace) & 255))
    return HDQT_ERR_ALIGNMENT;
  if (workspace_bytes < hdqt_group_norm_workspace_bytes(d, 1)) return HDQT_ERR_WORKSPACE;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  float2* chan = reinterpret_cast<float2*>(workspace);
  if (empty) {
    if (dgamma || dbeta) launch_param_grad(chan, 0, (int)d->channels, dgamma, dbeta, d->param_dtype, false, s);
    return last_error("group norm gradient");
  }
  const int vec = vector_width(d->channels, elem, bases | stride_bits(*d));
  const Plan pl = make_plan(*d, vec);
  NormParams p = make_params(*d, pl);
  p.x = x;
  p.dy = dy;
  p.gamma = gamma;
  p.beta = beta;
  p.out = dx;
  p.mean = const_cast<float*>(mean);
  p.rstd = const_cast<float*>(rstd);
  p.chan = chan;
  p.group = reinterpret_cast<float2*>(reinterpret_cast<uint8_t*>(workspace) +
                                      align256((size_t)d->batch * most_chunks(*d) * d->channels * sizeof(float2)));
  const Division dv = choose_division(*d, vec, true);
  if (dv.cluster > 0) {
    set_division(&p, *d, dv, vec);
    return with_type_and_width(d->dtype, vec, [&]<typename T, int V>() {
      const hdqt_status_t e = p.per_group % V == 0 ? launch_cluster<norm_bwd_cluster_kernel<T, V, true>>(p, dv, d->batch, s)
                                                   : launch_cluster<norm_bwd_cluster_kernel<T, V, false>>(p, dv, d->batch, s);
      if (e != HDQT_OK) return e;
      if (dgamma || dbeta) launch_param_grad(chan, d->batch * dv.cluster, (int)d->channels, dgamma, dbeta, d->param_dtype, true, s);
      return last_error("group norm gradient");
    });
  }
  const dim3 grid = stream_grid(*d, pl);
  return with_type_and_width(d->dtype, vec, [&]<typename T, int V>() {
    norm_bwd_sums_kernel<T, V><<<grid, NT, 0, s>>>(p);
    if (dx) {
      launch_chained(norm_join_sums_kernel, (unsigned)(d->batch * d->groups), NT, 0, s, p);
      launch_chained(norm_bwd_apply_kernel<T, V>, grid, NT, 0, s, p);
    }
    if (dgamma || dbeta) launch_param_grad(chan, d->batch * pl.chunks, (int)d->channels, dgamma, dbeta, d->param_dtype, true, s);
    return last_error("group norm gradient");
  });
}
