// Global norm over a list of tensors, and clipping by it.
//
//   norm = sqrt(sum x^2) or max |x|,   dst = src * min(1, max_norm / (norm + 1e-6))
//
// Two launches whatever the number of tensors (per kMaxTensors of them): a pass that leaves one partial result per
// block, and a pass in which every block joins the partials by itself (a few KB from L2) and scales its share.  The
// tensor table travels in the kernel parameters, so no copy to the device precedes the launch.
//
// Bound by HBM: every element is read twice (the factor is known after the last one only) and written once; the scaling pass
// walks backwards, so that what the first pass left in the L2 is read from there.  400 M elements of mixed types (1.35 GB): 225 us
// for the norm (6.0 TB/s), 427 us for scaling (6.3 TB/s).  62 tensors with 11 M elements: 26 us on the device, 53 us a call, which is
// the host's time for filling the table (and, 1 us of it, for looking for overlaps).
#include <math.h>
#include <stdlib.h>

#include <algorithm>

#include "hdqt_types.cuh"

namespace hdqt {

namespace {

constexpr int kThreads = 512;
constexpr int kChunkBytes = 32768;    // unit of work: consecutive bytes of one tensor
constexpr int kMaxBlocks = 148 * 4;   // partial results: one per block of the first pass
constexpr int kMaxTensors = 512;      // per launch

struct TableEntry {
  const void* src;
  void* dst;
  int64_t numel;
  uint32_t first_chunk;
  int32_t dtype;
};
template <int N>
struct Table {
  TableEntry e[N];
  uint32_t chunks;
  int32_t count;
};

// entry that chunk c belongs to: the last one whose first chunk is <= c (entries without elements are left out)
template <int N>
__device__ __forceinline__ int find_entry(const Table<N>& t, uint32_t c) {
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.e[mid].first_chunk <= c) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// |x| as its bit pattern: patterns order like the values, and a NaN is above everything
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

template <bool kInf>
struct Acc {
  float s = 0.0f;
  uint32_t m = 0u;
  __device__ __forceinline__ void add(float x) {
    if (kInf) m = max(m, abs_bits(x));
    else s = fmaf(x, x, s);
  }
};

template <typename T, bool kInf>
__device__ __forceinline__ void reduce_chunk(const T* __restrict__ src, int n, bool vec, Acc<kInf>& a) {
  constexpr int V = 16 / sizeof(T);
  int done = 0;
  if (vec) {
    const Vec<T, V>* p = reinterpret_cast<const Vec<T, V>*>(src);
    const int nv = n / V;
#pragma unroll 4
    for (int i = threadIdx.x; i < nv; i += kThreads) {
      const Vec<T, V> x = p[i];
#pragma unroll
      for (int k = 0; k < V; ++k) a.add(to_f32(x.v[k]));
    }
    done = nv * V;
  }
  for (int i = done + threadIdx.x; i < n; i += kThreads) a.add(to_f32(src[i]));
}

template <typename T>
__device__ __forceinline__ void scale_chunk(const T* src, T* dst, int n, bool vec, float f) {
  constexpr int V = 16 / sizeof(T);
  int done = 0;
  if (vec) {
    const Vec<T, V>* p = reinterpret_cast<const Vec<T, V>*>(src);
    Vec<T, V>* q = reinterpret_cast<Vec<T, V>*>(dst);
    const int nv = n / V;
#pragma unroll 4
    for (int i = threadIdx.x; i < nv; i += kThreads) {
      Vec<T, V> x = p[i];
#pragma unroll
      for (int k = 0; k < V; ++k) x.v[k] = from_f32<T>(to_f32(x.v[k]) * f);
      q[i] = x;
    }
    done = nv * V;
  }
  for (int i = done + threadIdx.x; i < n; i += kThreads) dst[i] = from_f32<T>(to_f32(src[i]) * f);
}

// what chunk c covers: a pointer, a number of elements and the type
struct Piece {
  int64_t at;
  int n;
};
__device__ __forceinline__ Piece piece_of(const TableEntry& e, uint32_t c, int elem) {
  const int64_t per = kChunkBytes / elem;
  Piece p;
  p.at = (int64_t)(c - e.first_chunk) * per;
  p.n = (int)min(per, e.numel - p.at);
  return p;
}

// block-wide join of fp64 sums (or bit-pattern maxima), valid in thread 0
template <bool kInf>
__device__ __forceinline__ double block_join(double v) {
  __shared__ double s_part[kThreads / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    const double o = __shfl_xor_sync(0xFFFFFFFFu, v, d);
    v = kInf ? fmax(v, o) : v + o;
  }
  if (lane == 0) s_part[warp] = v;
  __syncthreads();
  if (threadIdx.x == 0) {
    v = s_part[0];
    for (int w = 1; w < kThreads / 32; ++w) v = kInf ? fmax(v, s_part[w]) : v + s_part[w];
  }
  return v;
}

// partials[slot0 + block]: fp64 sum of squares, or the bit pattern of the maximum as a (whole) fp64 number
template <int N, bool kInf>
__global__ void __launch_bounds__(kThreads) grad_partial_kernel(const __grid_constant__ Table<N> t, double* __restrict__ partials) {
  chain_wait();
  Acc<kInf> a;
  for (uint32_t c = blockIdx.x; c < t.chunks; c += gridDim.x) {
    const TableEntry& e = t.e[find_entry(t, c)];
    const bool vec = (reinterpret_cast<uintptr_t>(e.src) & 15) == 0;
    const int elem = e.dtype == HDQT_DTYPE_F32 ? 4 : 2;
    const Piece p = piece_of(e, c, elem);
    if (e.dtype == HDQT_DTYPE_F32) reduce_chunk<float, kInf>(reinterpret_cast<const float*>(e.src) + p.at, p.n, vec, a);
    else if (e.dtype == HDQT_DTYPE_BF16) reduce_chunk<__nv_bfloat16, kInf>(reinterpret_cast<const __nv_bfloat16*>(e.src) + p.at, p.n, vec, a);
    else reduce_chunk<__half, kInf>(reinterpret_cast<const __half*>(e.src) + p.at, p.n, vec, a);
  }
  const double v = block_join<kInf>(kInf ? (double)a.m : (double)a.s);
  if (threadIdx.x == 0) partials[blockIdx.x] = v;
}

template <bool kInf>
__device__ __forceinline__ float join_partials(const double* __restrict__ partials, int n) {
  __shared__ float s_norm;
  double v = 0.0;
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const double o = partials[i];
    v = kInf ? fmax(v, o) : v + o;
  }
  v = block_join<kInf>(v);
  if (threadIdx.x == 0) s_norm = kInf ? __uint_as_float((uint32_t)v) : (float)sqrt(v);
  __syncthreads();
  return s_norm;
}

template <bool kInf>
__global__ void __launch_bounds__(kThreads) grad_norm_kernel(const double* __restrict__ partials, int n, float* __restrict__ norm_out) {
  chain_wait();
  const float norm = join_partials<kInf>(partials, n);
  if (threadIdx.x == 0) *norm_out = norm;
}

// this block's share of dst = src * f
template <int N>
__device__ __forceinline__ void scale_table(const Table<N>& t, float f) {
  // from the end: what a pass over the table read last is still in the L2
  for (uint32_t i = blockIdx.x; i < t.chunks; i += gridDim.x) {
    const uint32_t c = t.chunks - 1 - i;
    const TableEntry& e = t.e[find_entry(t, c)];
    if (f == 1.0f && e.src == e.dst) continue;
    const bool vec = ((reinterpret_cast<uintptr_t>(e.src) | reinterpret_cast<uintptr_t>(e.dst)) & 15) == 0;
    const int elem = e.dtype == HDQT_DTYPE_F32 ? 4 : 2;
    const Piece p = piece_of(e, c, elem);
    if (e.dtype == HDQT_DTYPE_F32)
      scale_chunk(reinterpret_cast<const float*>(e.src) + p.at, reinterpret_cast<float*>(e.dst) + p.at, p.n, vec, f);
    else if (e.dtype == HDQT_DTYPE_BF16)
      scale_chunk(reinterpret_cast<const __nv_bfloat16*>(e.src) + p.at, reinterpret_cast<__nv_bfloat16*>(e.dst) + p.at, p.n, vec, f);
    else
      scale_chunk(reinterpret_cast<const __half*>(e.src) + p.at, reinterpret_cast<__half*>(e.dst) + p.at, p.n, vec, f);
  }
}

template <int N, bool kInf>
__global__ void __launch_bounds__(kThreads)
grad_scale_kernel(const __grid_constant__ Table<N> t, const double* __restrict__ partials, int n, float max_norm,
                  float* __restrict__ norm_out) {
  chain_wait();
  const float norm = join_partials<kInf>(partials, n);
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm_out = norm;
  float f = max_norm / (norm + 1e-6f);
  if (f > 1.0f) f = 1.0f;      // (a NaN stays)
  scale_table(t, f);
}

template <int N>
__global__ void __launch_bounds__(kThreads) scale_by_kernel(const __grid_constant__ Table<N> t, const float* __restrict__ factor) {
  scale_table(t, *factor);
}

// Fills one launch's table from `tensors` starting at *next; returns the number of chunks (0 = nothing left).
template <int N>
uint32_t fill_table(const hdqt_tensor_t* tensors, int64_t count, int64_t* next, Table<N>* t) {
  t->count = 0;
  uint32_t chunks = 0;
  for (; *next < count && t->count < N; ++*next) {
    const hdqt_tensor_t& x = tensors[*next];
    if (x.numel == 0) continue;
    const int64_t per = kChunkBytes / dtype_size(x.dtype);
    const int64_t need = (x.numel + per - 1) / per;
    if ((int64_t)chunks + need > 0x7FFFFFFFll) break;     // (64 TB: one launch's worth)
    TableEntry& e = t->e[t->count++];
    e.src = x.src;
    e.dst = x.dst;
    e.numel = x.numel;
    e.first_chunk = chunks;
    e.dtype = (int32_t)x.dtype;
    chunks += (uint32_t)need;
  }
  t->chunks = chunks;
  return chunks;
}

template <int N, bool kInf>
hdqt_status_t run(const hdqt_tensor_t* tensors, int64_t count, bool clip, float max_norm, float* norm_out, double* partials,
                  cudaStream_t s) {
  const int sms = sm_count();
  if (sms <= 0) return HDQT_ERR_CUDA;
  const uint32_t most = (uint32_t)(sms * 4 < kMaxBlocks ? sms * 4 : kMaxBlocks);
  Table<N> t;
  int n_part = 0;
  for (int64_t next = 0; uint32_t chunks = fill_table(tensors, count, &next, &t);) {
    const uint32_t grid = chunks < most ? chunks : most;
    if (n_part == 0) grad_partial_kernel<N, kInf><<<grid, kThreads, 0, s>>>(t, partials);
    else launch_chained(grad_partial_kernel<N, kInf>, grid, kThreads, 0, s, t, partials + n_part);
    n_part += (int)grid;
  }
  if (!clip || n_part == 0) {
    if (n_part == 0) grad_norm_kernel<kInf><<<1, kThreads, 0, s>>>(partials, n_part, norm_out);
    else launch_chained(grad_norm_kernel<kInf>, 1, kThreads, 0, s, partials, n_part, norm_out);
  } else {
    for (int64_t next = 0; uint32_t chunks = fill_table(tensors, count, &next, &t);) {
      const uint32_t grid = chunks < most ? chunks : most;
      launch_chained(grad_scale_kernel<N, kInf>, grid, kThreads, 0, s, t, partials, n_part, max_norm, norm_out);
    }
  }
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? HDQT_OK : cuda_failure(e, "gradient norm");
}

template <int N>
hdqt_status_t run_scale(const hdqt_tensor_t* tensors, int64_t count, const float* factor, cudaStream_t s) {
  const int sms = sm_count();
  if (sms <= 0) return HDQT_ERR_CUDA;
  const uint32_t most = (uint32_t)(sms * 4 < kMaxBlocks ? sms * 4 : kMaxBlocks);
  Table<N> t;
  for (int64_t next = 0; uint32_t chunks = fill_table(tensors, count, &next, &t);)
    scale_by_kernel<N><<<chunks < most ? chunks : most, kThreads, 0, s>>>(t, factor);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? HDQT_OK : cuda_failure(e, "scaling");
}

struct Span {
  uintptr_t lo, hi;
};
Span span_of(const void* p, const hdqt_tensor_t& x) {
  const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
  return Span{lo, lo + (uintptr_t)x.numel * (uintptr_t)dtype_size(x.dtype)};
}

// No element that is written may be written twice, or read for another element: the blocks that do so run in no fixed order.
// n tensors with elements; their destinations sorted by address (1 us for 62 of them).
hdqt_status_t check_overlap(const hdqt_tensor_t* tensors, int64_t count, int64_t n) {
  if (n == 0) return HDQT_OK;
  Span few[kMaxTensors];
  Span* dst = n <= kMaxTensors ? few : static_cast<Span*>(malloc((size_t)n * sizeof(Span)));
  if (dst == nullptr) return HDQT_ERR_UNSUPPORTED;
  int64_t k = 0;
  for (int64_t i = 0; i < count; ++i)
    if (tensors[i].numel > 0) dst[k++] = span_of(tensors[i].dst, tensors[i]);
  std::sort(dst, dst + n, [](const Span& a, const Span& b) { return a.lo < b.lo; });
  bool ok = true;
  for (int64_t i = 1; i < n; ++i) ok = ok && dst[i - 1].hi <= dst[i].lo;
  for (int64_t i = 0; ok && i < count; ++i) {
    if (tensors[i].numel == 0 || tensors[i].src == tensors[i].dst) continue;
    const Span s = span_of(tensors[i].src, tensors[i]);
    const Span* after = std::lower_bound(dst, dst + n, s.hi, [](const Span& a, uintptr_t v) { return a.lo < v; });
    ok = after == dst || after[-1].hi <= s.lo;
  }
  if (dst != few) free(dst);
  return ok ? HDQT_OK : HDQT_ERR_INVALID_ARG;
}

// the list itself; *used = tensors with elements
hdqt_status_t check_list(const hdqt_tensor_t* tensors, int64_t count, bool write, int64_t* used) {
  if (count < 0 || (count > 0 && tensors == nullptr)) return HDQT_ERR_INVALID_ARG;
  *used = 0;
  for (int64_t i = 0; i < count; ++i) {
    const hdqt_tensor_t& x = tensors[i];
    const int size = dtype_size(x.dtype);
    if (size == 0 || x.numel < 0) return HDQT_ERR_INVALID_ARG;
    if (x.numel == 0) continue;
    if (x.numel > (1ll << 42)) return HDQT_ERR_UNSUPPORTED;
    if (!x.src || (write && !x.dst)) return HDQT_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(x.src) | (write ? reinterpret_cast<uintptr_t>(x.dst) : 0)) & (uintptr_t)(size - 1))
      return HDQT_ERR_ALIGNMENT;
    ++*used;
  }
  return write ? check_overlap(tensors, count, *used) : HDQT_OK;
}

hdqt_status_t check_and_run(const hdqt_tensor_t* tensors, int64_t count, int32_t norm_type, bool clip, float max_norm,
                            float* norm_out, void* workspace, size_t workspace_bytes, void* stream) {
  if (!norm_out || !workspace) return HDQT_ERR_INVALID_ARG;
  if (norm_type != HDQT_NORM_L2 && norm_type != HDQT_NORM_INF) return HDQT_ERR_INVALID_ARG;
  if (clip && !(max_norm >= 0.0f)) return HDQT_ERR_INVALID_ARG;
  int64_t used = 0;
  const hdqt_status_t st = check_list(tensors, count, clip, &used);
  if (st != HDQT_OK) return st;
  if (reinterpret_cast<uintptr_t>(norm_out) & 3) return HDQT_ERR_ALIGNMENT;
  if (reinterpret_cast<uintptr_t>(workspace) & 127) return HDQT_ERR_ALIGNMENT;
  if (workspace_bytes < hdqt_grad_norm_workspace_bytes(count)) return HDQT_ERR_WORKSPACE;
  double* partials = reinterpret_cast<double*>(workspace);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  // the smaller table keeps the parameter block of the usual call small
  if (used <= 64) {
    return norm_type == HDQT_NORM_INF ? run<64, true>(tensors, count, clip, max_norm, norm_out, partials, s)
                                      : run<64, false>(tensors, count, clip, max_norm, norm_out, partials, s);
  }
  return norm_type == HDQT_NORM_INF ? run<kMaxTensors, true>(tensors, count, clip, max_norm, norm_out, partials, s)
                                    : run<kMaxTensors, false>(tensors, count, clip, max_norm, norm_out, partials, s);
}

}  // namespace

}  // namespace hdqt

using namespace hdqt;

extern "C" size_t hdqt_grad_norm_workspace_bytes(int64_t count) {
  const int64_t launches = count <= 0 ? 1 : (count + kMaxTensors - 1) / kMaxTensors + 1;
  return (size_t)launches * kMaxBlocks * sizeof(double);
}

extern "C" hdqt_status_t hdqt_grad_norm(const hdqt_tensor_t* tensors, int64_t count, int32_t norm_type, float* norm_out,
                                        void* workspace, size_t workspace_bytes, void* stream) {
  return check_and_run(tensors, count, norm_type, false, 0.0f, norm_out, workspace, workspace_bytes, stream);
}

extern "C" hdqt_status_t hdqt_clip_grad_norm(const hdqt_tensor_t* tensors, int64_t count, int32_t norm_type,
                                             float max_norm, float* norm_out, void* workspace, size_t workspace_bytes,
                                             void* stream) {
  return check_and_run(tensors, count, norm_type, true, max_norm, norm_out, workspace, workspace_bytes, stream);
}

extern "C" hdqt_status_t hdqt_scale_tensors(const hdqt_tensor_t* tensors, int64_t count, const float* factor, void* stream) {
  if (!factor) return HDQT_ERR_INVALID_ARG;
  int64_t used = 0;
  const hdqt_status_t st = check_list(tensors, count, true, &used);
  if (st != HDQT_OK) return st;
  if (reinterpret_cast<uintptr_t>(factor) & 3) return HDQT_ERR_ALIGNMENT;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  return used <= 64 ? run_scale<64>(tensors, count, factor, s) : run_scale<kMaxTensors>(tensors, count, factor, s);
}
