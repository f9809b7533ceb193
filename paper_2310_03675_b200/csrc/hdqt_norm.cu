// Group norm with an activation on channels-last activations x[batch, pixels, channels].
//
//   z = gamma (x - mu) rs + beta,  y = act(z);  dz = dy act'(z)
//   dx = rs (gamma dz - mean(gamma dz) - xhat mean(gamma dz xhat)),  dgamma = sum dz xhat,  dbeta = sum dz
//
// Streaming kernels (this path serves every size): per-channel partial statistics of a piece of an image, a join per
// group, and an elementwise pass.  A thread keeps one column of V channels and walks down the pixels, so gamma, beta and
// the statistics of its channels stay in registers.
//
// Variance: a thread sums d = x - p and d^2 with p its own first value, so that its M2 = sum d^2 - (sum d)^2 / n never
// cancels by more than a factor n (p is one of the n values), and thread results are joined by Chan's formula.  Means
// travel relative to the group's first value (the "anchor"), so that a mean far larger than the spread costs no digits of it.
#include <math.h>

#include "hdqt_types.cuh"

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
  int32_t chunks, chunk_pixels;
};

__device__ __forceinline__ float gamma_of(const NormParams& p, int c) { return p.gamma ? load_param(p.gamma, p.param_dtype, c) : 1.0f; }
__device__ __forceinline__ float beta_of(const NormParams& p, int c) { return p.beta ? load_param(p.beta, p.param_dtype, c) : 0.0f; }

// 1 / (1 + exp(-z)); exp overflows to infinity for z < -88, where the quotient is the correct 0
__device__ __forceinline__ float sigmoid(float z) { return __fdividef(1.0f, 1.0f + __expf(-z)); }

__device__ __forceinline__ float act_fwd(float z, int act) {
  if (act == HDQT_ACT_RELU) return z > 0.0f ? z : (z != z ? z : 0.0f);
  if (act == HDQT_ACT_SILU) return z == -INFINITY ? 0.0f * z : z * sigmoid(z);
  return z;
}
// dy * act'(z)
__device__ __forceinline__ float act_bwd(float dy, float z, int act) {
  if (act == HDQT_ACT_RELU) return z > 0.0f ? dy : 0.0f;
  if (act == HDQT_ACT_SILU) {
    const float s = sigmoid(z);
    return dy * s * fmaf(z, 1.0f - s, 1.0f);
  }
  return dy;
}

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
__global__ void __launch_bounds__(NT) norm_stats_kernel(const NormParams p) {
  __shared__ float s_mean[NT * V], s_m2[NT * V];
  const Column k = column_of<V>(p);
  const int64_t p0 = (int64_t)blockIdx.x * p.chunk_pixels;
  const int n = (int)min((int64_t)p.chunk_pixels, p.pixels - p0);
  for (int64_t b = blockIdx.z; b < p.batch; b += gridDim.z) {
    const T* src = reinterpret_cast<const T*>(p.x) + b * p.x_bs + p0 * p.x_ps + k.c0;
    float pivot[V], s1[V], s2[V];
    int cnt = 0;
    if (k.live && k.row < n) {
      const Vec<T, V> f = *reinterpret_cast<const Vec<T, V>*>(src + (int64_t)k.row * p.x_ps);
#pragma unroll
      for (int j = 0; j < V; ++j) { pivot[j] = to_f32(f.v[j]); s1[j] = s2[j] = 0.0f; }
#pragma unroll 4
      for (int i = k.row; i < n; i += k.rows) {
        const Vec<T, V> v = *reinterpret_cast<const Vec<T, V>*>(src + (int64_t)i * p.x_ps);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float d = to_f32(v.v[j]) - pivot[j];
          s1[j] += d;
          s2[j] = fmaf(d, d, s2[j]);
        }
        ++cnt;
      }
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
      // row r holds ceil((n - r) / rows) pixels
      float mean = 0.0f, m2 = 0.0f;
      for (int r = 0; r < k.rows && r < n; ++r) mean += s_mean[r * width + c] * (float)((n - r + k.rows - 1) / k.rows);
      mean /= (float)n;
      for (int r = 0; r < k.rows && r < n; ++r) {
        const float d = s_mean[r * width + c] - mean;
        m2 += fmaf(d * d, (float)((n - r + k.rows - 1) / k.rows), s_m2[r * width + c]);
      }
      p.chan[(b * p.chunks + blockIdx.x) * p.channels + blockIdx.y * kCols * V + c] = make_float2(mean, m2);
    }
    __syncthreads();
  }
}

__device__ __forceinline__ float block_sum(float v) {
  __shared__ float s_part[NT / 32];
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.0f;
#pragma unroll
  for (int w = 0; w < NT / 32; ++w) v += s_part[w];
  __syncthreads();
  return v;
}

// one block per (image, group): joins the chunks' channel statistics
template <typename T>
__global__ void __launch_bounds__(NT) norm_join_stats_kernel(const NormParams p) {
  const int64_t b = blockIdx.x / p.groups;
  const int g = (int)(blockIdx.x - b * p.groups);
  const float2* part = p.chan + b * p.chunks * p.channels + (int64_t)g * p.per_group;
  const int64_t items = (int64_t)p.chunks * p.per_group;
  const float total = (float)(p.pixels * p.per_group);
  float s = 0.0f;
  for (int64_t i = threadIdx.x; i < items; i += NT) {
    const int64_t chunk = i / p.per_group, c = i - chunk * p.per_group;
    const float n = (float)min((int64_t)p.chunk_pixels, p.pixels - chunk * p.chunk_pixels);
    s = fmaf(part[chunk * p.channels + c].x, n, s);
  }
  const float mean = block_sum(s) / total;
  s = 0.0f;
  for (int64_t i = threadIdx.x; i < items; i += NT) {
    const int64_t chunk = i / p.per_group, c = i - chunk * p.per_group;
    const float n = (float)min((int64_t)p.chunk_pixels, p.pixels - chunk * p.chunk_pixels);
    const float2 v = part[chunk * p.channels + c];
    const float d = v.x - mean;
    s += fmaf(d * d, n, v.y);
  }
  const float var = block_sum(s) / total;
  if (threadIdx.x == 0) {
    p.mean[blockIdx.x] = anchor<T>(p, b, g) + mean;
    p.rstd[blockIdx.x] = rsqrtf(var + p.eps);
  }
}

template <typename T, int V>
__global__ void __launch_bounds__(NT) norm_apply_kernel(const NormParams p) {
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
#pragma unroll 4
    for (int i = k.row; i < n; i += k.rows) {
      Vec<T, V> v = *reinterpret_cast<const Vec<T, V>*>(src + (int64_t)i * p.x_ps);
#pragma unroll
      for (int j = 0; j < V; ++j) v.v[j] = from_f32<T>(act_fwd(fmaf(to_f32(v.v[j]) - mu[j], a[j], be[j]), p.act));
      *reinterpret_cast<Vec<T, V>*>(dst + (int64_t)i * p.y_ps) = v;
    }
  }
}

// chan[b, chunk, c] = (sum dz, sum dz xhat) of the chunk's pixels
template <typename T, int V>
__global__ void __launch_bounds__(NT) norm_bwd_sums_kernel(const NormParams p) {
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
#pragma unroll 2
      for (int i = k.row; i < n; i += k.rows) {
        const Vec<T, V> v = *reinterpret_cast<const Vec<T, V>*>(src + (int64_t)i * p.x_ps);
        const Vec<T, V> d = *reinterpret_cast<const Vec<T, V>*>(dys + (int64_t)i * p.y_ps);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float xh = (to_f32(v.v[j]) - mu[j]) * rs[j];
          const float dz = act_bwd(to_f32(d.v[j]), fmaf(xh, ga[j], be[j]), p.act);
          sa[j] += dz;
          sb[j] = fmaf(dz, xh, sb[j]);
        }
      }
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
  const int64_t b = blockIdx.x / p.groups;
  const int g = (int)(blockIdx.x - b * p.groups);
  const float2* part = p.chan + b * p.chunks * p.channels + (int64_t)g * p.per_group;
  const int64_t items = (int64_t)p.chunks * p.per_group;
  float s1 = 0.0f, s2 = 0.0f;
  for (int64_t i = threadIdx.x; i < items; i += NT) {
    const int64_t chunk = i / p.per_group, c = i - chunk * p.per_group;
    const float2 v = part[chunk * p.channels + c];
    const float ga = gamma_of(p, g * p.per_group + (int)c);
    s1 = fmaf(v.x, ga, s1);
    s2 = fmaf(v.y, ga, s2);
  }
  s1 = block_sum(s1);
  s2 = block_sum(s2);
  const float inv = 1.0f / (float)(p.pixels * p.per_group);
  if (threadIdx.x == 0) p.group[blockIdx.x] = make_float2(s1 * inv, s2 * inv);
}

template <typename T, int V>
__global__ void __launch_bounds__(NT) norm_bwd_apply_kernel(const NormParams p) {
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
#pragma unroll 2
    for (int i = k.row; i < n; i += k.rows) {
      Vec<T, V> v = *reinterpret_cast<const Vec<T, V>*>(src + (int64_t)i * p.x_ps);
      const Vec<T, V> d = *reinterpret_cast<const Vec<T, V>*>(dys + (int64_t)i * p.y_ps);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float xh = (to_f32(v.v[j]) - mu[j]) * rs[j];
        const float dz = act_bwd(to_f32(d.v[j]), fmaf(xh, ga[j], be[j]), p.act);
        v.v[j] = from_f32<T>(rs[j] * (fmaf(dz, ga[j], -m1[j]) - xh * m2[j]));
      }
      *reinterpret_cast<Vec<T, V>*>(dst + (int64_t)i * p.y_ps) = v;
    }
  }
}

// dgamma, dbeta: sum of the parts [parts, channels] of all images, 32 channels x 8 rows of threads per block
__global__ void __launch_bounds__(NT) norm_param_grad_kernel(const float2* __restrict__ part, int64_t parts, int channels,
                                                             void* dgamma, void* dbeta, int32_t param_dtype) {
  __shared__ float2 s[8][32];
  const int lane = threadIdx.x & 31, row = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;
  float2 t = make_float2(0.0f, 0.0f);
  if (c < channels) {
#pragma unroll 4
    for (int64_t i = row; i < parts; i += 8) {
      const float2 v = part[i * channels + c];
      t.x += v.x;
      t.y += v.y;
    }
  }
  s[row][lane] = t;
  __syncthreads();
  if (row == 0 && c < channels) {
    for (int r = 1; r < 8; ++r) { t.x += s[r][lane].x; t.y += s[r][lane].y; }
    if (dbeta) store_param(dbeta, param_dtype, c, t.x);
    if (dgamma) store_param(dgamma, param_dtype, c, t.y);
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

// widest access (16 bytes, or down to one element) that `align` (bases and strides in bytes, or-ed together) allows
int vector_width(int64_t channels, int elem, uintptr_t align) {
  int v = 16 / elem;
  while (v > 1 && (channels % v != 0 || (align & (uintptr_t)(v * elem - 1)) != 0)) v >>= 1;
  return v;
}

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
  return most;
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

template <typename F>
hdqt_status_t with_type_and_width(int dtype, int vec, F&& f) {
  if (dtype == HDQT_DTYPE_F32) {
    if (vec == 4) return f.template operator()<float, 4>();
    if (vec == 2) return f.template operator()<float, 2>();
    return f.template operator()<float, 1>();
  }
  if (dtype == HDQT_DTYPE_BF16) {
    if (vec == 8) return f.template operator()<__nv_bfloat16, 8>();
    if (vec == 4) return f.template operator()<__nv_bfloat16, 4>();
    if (vec == 2) return f.template operator()<__nv_bfloat16, 2>();
    return f.template operator()<__nv_bfloat16, 1>();
  }
  if (vec == 8) return f.template operator()<__half, 8>();
  if (vec == 4) return f.template operator()<__half, 4>();
  if (vec == 2) return f.template operator()<__half, 2>();
  return f.template operator()<__half, 1>();
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
  p.chunks = pl.chunks;
  p.chunk_pixels = pl.chunk_pixels;
  return p;
}

dim3 stream_grid(const hdqt_group_norm_desc_t& d, const Plan& pl) {
  const int64_t ncol = d.channels / pl.vec;
  return dim3((unsigned)pl.chunks, (unsigned)((ncol + kCols - 1) / kCols), (unsigned)(d.batch < 65535 ? d.batch : 65535));
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

uintptr_t stride_bits(const hdqt_group_norm_desc_t& d) {
  const int e = dtype_size(d.dtype);
  return (uintptr_t)((d.x_pixel_stride | d.y_pixel_stride) * e) |
         (d.batch > 1 ? (uintptr_t)((d.x_batch_stride | d.y_batch_stride) * e) : 0);
}

hdqt_status_t last_error(const char* what) {
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? HDQT_OK : cuda_failure(e, what);
}

}  // namespace

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
  const dim3 grid = stream_grid(*d, pl);
  return with_type_and_width(d->dtype, vec, [&]<typename T, int V>() {
    norm_stats_kernel<T, V><<<grid, NT, 0, s>>>(p);
    norm_join_stats_kernel<T><<<(unsigned)(d->batch * d->groups), NT, 0, s>>>(p);
    norm_apply_kernel<T, V><<<grid, NT, 0, s>>>(p);
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
  const unsigned param_blocks = (unsigned)((d->channels + 31) / 32);
  float2* chan = reinterpret_cast<float2*>(workspace);
  if (empty) {
    if (dgamma || dbeta) norm_param_grad_kernel<<<param_blocks, NT, 0, s>>>(chan, 0, (int)d->channels, dgamma, dbeta, d->param_dtype);
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
  const dim3 grid = stream_grid(*d, pl);
  return with_type_and_width(d->dtype, vec, [&]<typename T, int V>() {
    norm_bwd_sums_kernel<T, V><<<grid, NT, 0, s>>>(p);
    if (dx) {
      norm_join_sums_kernel<<<(unsigned)(d->batch * d->groups), NT, 0, s>>>(p);
      norm_bwd_apply_kernel<T, V><<<grid, NT, 0, s>>>(p);
    }
    if (dgamma || dbeta)
      norm_param_grad_kernel<<<param_blocks, NT, 0, s>>>(chan, d->batch * pl.chunks, (int)d->channels, dgamma, dbeta, d->param_dtype);
    return last_error("group norm gradient");
  });
}
