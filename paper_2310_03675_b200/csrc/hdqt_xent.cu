// Linear layer + softmax cross entropy over a large vocabulary, without the fp32 logits of all tokens in memory.
//
//   z = X W^T,  lse = log sum exp z,  loss = lse - z[label],  dz = g (exp(z - lse) - [label]),  dX = dz W,  dW = dz^T X
//
// Everything large is a matrix product on the tensor cores (hdqt_xent_gemm.cuh); this file holds the row kernels between
// them and the host side.  The logits product's epilogue leaves, per row and 128 columns, the maximum and the sum of
// exponentials, so the softmax statistics never need the logits again; a row is joined from these parts.
//
//   forward  : logits product (statistics) -> rows
//   training : per piece of the tokens: logits product (statistics + 16-bit codes) -> rows, codes to dz in place ->
//              dX and dW products in one launch (fp32: fp32 logits -> three bf16 planes of dz)
//   backward : per piece of the vocabulary: logits product (dz from lse) -> dX (fp32 sums over the pieces) and dW
// A few output blocks or tokens: the logits as fp32 partial products of a split contraction (xent_softmax_kernel, hdqt_xent_few.cuh).
#include <math.h>

#include <atomic>
#include <utility>

#include "hdqt_xent_gemm.cuh"
#include "hdqt_xent_few.cuh"
#include "hdqt_xent_small.cuh"

namespace hdqt {

namespace {

constexpr int kRowThreads = 256;

// ---- labels ------------------------------------------------------------------------------------------------

// label[t] = class, -1 (ignored) or -2 (outside [0, classes)); scale[0] = 1 / kept rows (mean) or 1: factor of the reduced
// loss; scale[1] = scale[0] g (0 if no row is kept): factor of its gradients.  One block.
// weights (with unit): a weight per row of the loss.  scale[1] is then their largest finite magnitude (1 if there is none) and
// unit[t] = weights[t] / scale[1], so that equal weights reach dz as 1.
__global__ void __launch_bounds__(1024)
xent_labels_kernel(const int64_t* __restrict__ labels, int64_t tokens, int64_t classes, int64_t ignore, int32_t mean,
                   const float* __restrict__ g, int32_t* __restrict__ label, float* __restrict__ scale,
                   const float* __restrict__ weights, float* __restrict__ unit, int32_t* dev_status) {
  __shared__ int s_kept;
  __shared__ uint32_t s_most;
  chain_wait();
  if (threadIdx.x == 0) { s_kept = 0; s_most = 0u; }
  __syncthreads();
  int kept = 0;
  uint32_t most = 0u;          // magnitudes order like their bit patterns
  bool bad = false;
#pragma unroll 4
  for (int64_t t = threadIdx.x; t < tokens; t += blockDim.x) {
    const int64_t l = labels[t];
    int32_t v = -1;
    if (l != ignore) {
      ++kept;
      if (l >= 0 && l < classes) v = (int32_t)l;
      else { v = -2; bad = true; }
    }
    label[t] = v;
    if (unit != nullptr && v >= 0) {
      const uint32_t bits = __float_as_uint(weights[t]) & 0x7FFFFFFFu;
      if (bits < 0x7F800000u) most = max(most, bits);
    }
  }
  if (unit != nullptr) {
    most = __reduce_max_sync(0xFFFFFFFFu, most);
    if ((threadIdx.x & 31) == 0) atomicMax(&s_most, most);
    __syncthreads();
    const float s = s_most != 0u ? __uint_as_float(s_most) : 1.0f;
    for (int64_t t = threadIdx.x; t < tokens; t += blockDim.x) unit[t] = weights[t] / s;
    if (threadIdx.x == 0) { scale[0] = 1.0f; scale[1] = s; }
    if (bad) report_status(dev_status, HDQT_ERR_INVALID_ARG);
    return;
  }
  if (mean) {
    kept = __reduce_add_sync(0xFFFFFFFFu, kept);
    if ((threadIdx.x & 31) == 0) atomicAdd(&s_kept, kept);
  }
  if (bad) report_status(dev_status, HDQT_ERR_INVALID_ARG);
  __syncthreads();
  if (threadIdx.x == 0) {
    const float sc = mean ? 1.0f / (float)s_kept : 1.0f;
    scale[0] = sc;
    scale[1] = mean && s_kept == 0 ? 0.0f : sc * (g != nullptr ? *g : 1.0f);
  }
}

// ---- rows: joining the parts of the softmax statistics -------------------------------------------------------

struct MaxSum {
  float m, s;    // sum of exp(z - m)
};
__device__ __forceinline__ MaxSum join(const MaxSum& a, const MaxSum& b) {
  MaxSum r;
  r.m = fmaxf(a.m, b.m);
  r.s = a.s * ex2((a.m - r.m) * kLog2e) + b.s * ex2((b.m - r.m) * kLog2e);
  return r;
}
__device__ __forceinline__ MaxSum warp_join(MaxSum v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    MaxSum o;
    o.m = __shfl_xor_sync(0xFFFFFFFFu, v.m, d);
    o.s = __shfl_xor_sync(0xFFFFFFFFu, v.s, d);
    v = join(v, o);
  }
  return v;
}

__device__ __forceinline__ float row_loss(int32_t label, float lse, float label_logit) {
  return label >= 0 ? lse - label_logit : label == -1 ? 0.0f : NAN;
}

// one warp per row
__global__ void __launch_bounds__(kRowThreads) xent_rows_kernel(const float2* __restrict__ part, int parts, int64_t parts_ld,
                                                                const int32_t* __restrict__ label,
                                                                const float* __restrict__ label_logit, int64_t rows,
                                                                float* __restrict__ lse, float* __restrict__ loss) {
  chain_wait();
  const int64_t row = (int64_t)blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5);
  if (row >= rows) return;
  const int lane = threadIdx.x & 31;
  MaxSum v = {kLowest, 0.0f};
  for (int i = lane; i < parts; i += 32) {
    const float2 q = part[row * parts_ld + i];
    v = join(v, MaxSum{q.x, q.y});
  }
  v = warp_join(v);
  if (lane == 0) {
    const float l = v.m + logf(v.s);
    lse[row] = l;
    loss[row] = row_loss(label[row], l, label_logit[row]);
  }
}

// one block: loss = scale * sum of the rows' losses
__global__ void __launch_bounds__(1024) xent_loss_kernel(const float* __restrict__ rows, int64_t n, const float* __restrict__ scale,
                                                         float* __restrict__ loss) {
  __shared__ double s_part[32];
  chain_wait();
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += blockDim.x) s += (double)rows[i];
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
  if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0;
    for (int w = 0; w < 32; ++w) s += s_part[w];
    loss[0] = (float)(s * (double)scale[0]);
  }
}

// Training: the blocks of a row (blockIdx.y: slices of the classes) join the row's parts, write lse and the loss, and turn
// the row's codes (or fp32 logits) into dz = w (softmax - [label]): bf16 in place of the codes, or three bf16 planes.
template <int kPlanes>
__global__ void __launch_bounds__(kRowThreads)
xent_dz_kernel(const float2* __restrict__ part, int parts, int64_t parts_ld, const int32_t* __restrict__ label,
               const float* __restrict__ label_logit, const float* __restrict__ weight, int64_t classes, void* z, int64_t ld,
               uint16_t* planes, int64_t plane, float* __restrict__ lse, float* __restrict__ loss) {
  __shared__ float s_m[kRowThreads / 32], s_s[kRowThreads / 32];
  chain_wait();
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const float2* pr = part + row * parts_ld;
  MaxSum v = {kLowest, 0.0f};
  for (int i = threadIdx.x; i < parts; i += kRowThreads) {
    const float2 q = pr[i];
    v = join(v, MaxSum{q.x, q.y});
  }
  v = warp_join(v);
  if (lane == 0) { s_m[warp] = v.m; s_s[warp] = v.s; }
  __syncthreads();
  v = MaxSum{s_m[0], s_s[0]};
#pragma unroll
  for (int w = 1; w < kRowThreads / 32; ++w) v = join(v, MaxSum{s_m[w], s_s[w]});
  const int32_t lab = label[row];
  if (threadIdx.x == 0 && blockIdx.y == 0) {
    const float l = v.m + logf(v.s);
    lse[row] = l;
    loss[row] = row_loss(lab, l, label_logit[row]);
  }
  const bool keep = lab >= 0;
  const float w = !keep ? 0.0f : weight != nullptr ? weight[row] : 1.0f;
  const float scale = w / v.s;
  if (kPlanes == 1) {
    uint4* codes = reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(z) + row * ld);
#pragma unroll 2
    for (int j = blockIdx.y * kRowThreads + threadIdx.x; j * 8 < classes; j += kRowThreads * gridDim.y) {
      uint4 c = codes[j];
      uint32_t* cw = reinterpret_cast<uint32_t*>(&c);
      const float f = keep ? ex2((pr[j >> 4].x - v.m) * kLog2e) * scale : 0.0f;   // NaN where the row has one
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t ca = cw[k] & 0xFFFFu, cb = cw[k] >> 16;
        float a = (ca == kCodeZero ? 0.0f : ex2((float)ca * (-1.0f / kCodeScale))) * f;
        float b = (cb == kCodeZero ? 0.0f : ex2((float)cb * (-1.0f / kCodeScale))) * f;
        if (lab == j * 8 + 2 * k) a -= w;
        if (lab == j * 8 + 2 * k + 1) b -= w;
        cw[k] = pack_bf16(a, b);
      }
      codes[j] = c;
    }
  } else {
    const float4* logits = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(z) + row * ld);
    uint2* o = reinterpret_cast<uint2*>(planes + row * ld);
#pragma unroll 2
    for (int j = blockIdx.y * kRowThreads + threadIdx.x; j * 4 < classes; j += kRowThreads * gridDim.y) {
      const float4 q = logits[j];
      float a[4] = {q.x, q.y, q.z, q.w}, p0[4], p1[4], p2[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float e = keep ? ex2((a[k] - v.m) * kLog2e) * scale : 0.0f;
        if (lab == j * 4 + k) e -= w;
        split3(e, p0[k], p1[k], p2[k]);
      }
      o[j] = make_uint2(pack_bf16(p0[0], p0[1]), pack_bf16(p0[2], p0[3]));
      reinterpret_cast<uint2*>(planes + plane + row * ld)[j] = make_uint2(pack_bf16(p1[0], p1[1]), pack_bf16(p1[2], p1[3]));
      reinterpret_cast<uint2*>(planes + 2 * plane + row * ld)[j] = make_uint2(pack_bf16(p2[0], p2[1]), pack_bf16(p2[2], p2[3]));
    }
  }
}

// Few output blocks: the logits come as fp32 partial products [splits][rows][ld_part].  One block per row sums them in shared
// memory, forms lse (or takes lse_in) and the loss, and writes dz in 1 or 3 bf16 planes (planes 0: no gradient).
template <int kPlanes, int kThreads>
__global__ void __launch_bounds__(kThreads)
xent_softmax_kernel(const float* __restrict__ part, int splits, int64_t rows, int64_t ld_part, int classes,
                    const int32_t* __restrict__ label, const float* __restrict__ weight, const float* __restrict__ lse_in,
                    uint16_t* planes, int64_t ld, int64_t plane, float* __restrict__ lse, float* __restrict__ loss) {
  extern __shared__ float s_z[];
  __shared__ float s_m[kThreads / 32], s_s[kThreads / 32];
  chain_wait();
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const float* pr = part + row * ld_part;
  const int64_t step = rows * ld_part;
  float m = kLowest;
#pragma unroll 2
  for (int j = threadIdx.x; j < classes; j += kThreads) {
    float z = pr[j];
#pragma unroll 4
    for (int s = 1; s < splits; ++s) z += pr[s * step + j];
    s_z[j] = z;
    m = fmaxf(m, z);
  }
  const int32_t lab = label[row];
  float l;
  if (lse_in != nullptr) {
    l = lse_in[row];
  } else {
    float s = 0.0f;      // (a thread reads back what it wrote)
    for (int j = threadIdx.x; j < classes; j += kThreads) s += ex2((s_z[j] - m) * kLog2e);
    MaxSum v = warp_join(MaxSum{m, s});
    if (lane == 0) { s_m[warp] = v.m; s_s[warp] = v.s; }
    __syncthreads();
    v = MaxSum{s_m[0], s_s[0]};
#pragma unroll
    for (int w = 1; w < kThreads / 32; ++w) v = join(v, MaxSum{s_m[w], s_s[w]});
    l = v.m + logf(v.s);
    if (threadIdx.x == 0) {
      lse[row] = l;
      loss[row] = row_loss(lab, l, lab >= 0 ? s_z[lab] : 0.0f);
    }
  }
  if (kPlanes == 0) return;
  const bool keep = lab >= 0;
  const float w = !keep ? 0.0f : weight != nullptr ? weight[row] : 1.0f;
  for (int j = threadIdx.x; j < classes; j += kThreads) {
    const float e = keep ? w * (ex2((s_z[j] - l) * kLog2e) - (j == lab ? 1.0f : 0.0f)) : 0.0f;
    if (kPlanes == 1) {
      reinterpret_cast<__nv_bfloat16*>(planes)[row * ld + j] = __float2bfloat16_rn(e);
    } else {
      float p0, p1, p2;
      split3(e, p0, p1, p2);
      __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(planes) + row * ld + j;
      o[0] = __float2bfloat16_rn(p0);
      o[plane] = __float2bfloat16_rn(p1);
      o[2 * plane] = __float2bfloat16_rn(p2);
    }
  }
}

// ---- operands that cannot be read in place ---------------------------------------------------------------------

// fp32 -> three bf16 planes, or bf16 -> a copy with rows that start on 16 bytes; kV columns per thread (one access where the
// rows of the source allow it, else element by element), a block walks down the rows
template <typename T, int kV, bool kWide>
__global__ void __launch_bounds__(256) xent_stage_kernel(const T* __restrict__ src, int64_t ld, int64_t rows, int64_t cols,
                                                         uint16_t* __restrict__ dst, int64_t ld_dst, int64_t plane) {
  chain_wait();
  const int64_t c = kV * ((int64_t)blockIdx.x * 256 + threadIdx.x);
  if (c >= cols) return;
#pragma unroll 4
  for (int64_t r = blockIdx.y; r < rows; r += gridDim.y) {
    float x[kV];
    if constexpr (kWide) {
      unpack(*reinterpret_cast<const Vec<T, kV>*>(src + r * ld + c), x);
    } else {
#pragma unroll
      for (int j = 0; j < kV; ++j) x[j] = c + j < cols ? to_f32(src[r * ld + c + j]) : 0.0f;
    }
    uint16_t* d = dst + r * ld_dst + c;
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<Vec<__nv_bfloat16, kV>*>(d) = pack<__nv_bfloat16>(x);
    } else {
      float p0[kV], p1[kV], p2[kV];
#pragma unroll
      for (int j = 0; j < kV; ++j) split3(x[j], p0[j], p1[j], p2[j]);
      *reinterpret_cast<Vec<__nv_bfloat16, kV>*>(d) = pack<__nv_bfloat16>(p0);
      *reinterpret_cast<Vec<__nv_bfloat16, kV>*>(d + plane) = pack<__nv_bfloat16>(p1);
      *reinterpret_cast<Vec<__nv_bfloat16, kV>*>(d + 2 * plane) = pack<__nv_bfloat16>(p2);
    }
  }
}

// bf16 X times the weights of its rows' losses in two planes (16 significant bits), and the weights themselves; a row without a
// valid label weighs 0 whatever is given for it
__global__ void __launch_bounds__(256)
xent_weighted_rows_kernel(const __nv_bfloat16* __restrict__ x, int64_t ld, int64_t cols, const int32_t* __restrict__ label,
                          const float* __restrict__ g, uint16_t* __restrict__ dst, int64_t ld_dst, int64_t plane,
                          float* __restrict__ weight) {
  chain_wait();
  const int64_t r = blockIdx.y, c = 4 * ((int64_t)blockIdx.x * 256 + threadIdx.x);
  const float w = label[r] >= 0 ? g[r] : 0.0f;
  if (c == 0) weight[r] = w;
  if (c >= cols) return;
  float a[4], p0[4], p1[4], p2[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) a[j] = c + j < cols ? to_f32(x[r * ld + c + j]) : 0.0f;
#pragma unroll
  for (int j = 0; j < 4; ++j) split3(a[j] * w, p0[j], p1[j], p2[j]);
  uint16_t* d = dst + r * ld_dst + c;
  *reinterpret_cast<Vec<__nv_bfloat16, 4>*>(d) = pack<__nv_bfloat16>(p0);
  *reinterpret_cast<Vec<__nv_bfloat16, 4>*>(d + plane) = pack<__nv_bfloat16>(p1);
}

// sum of the splits' partial outputs, in order; four elements of the flat [rows, cols] at a time
template <typename T>
__global__ void __launch_bounds__(256) xent_join_splits_kernel(const float* __restrict__ part, int splits, int64_t rows,
                                                               int64_t cols, T* __restrict__ out, int64_t ld) {
  chain_wait();
  const int64_t n = rows * cols;
  const bool vec = n % 4 == 0 && cols % 4 == 0 && ld % 4 == 0 && (reinterpret_cast<uintptr_t>(out) & (4 * sizeof(T) - 1)) == 0;
  if (vec) {
    for (int64_t i = 4 * ((int64_t)blockIdx.x * 256 + threadIdx.x); i < n; i += 4 * (int64_t)gridDim.x * 256) {
      float4 s = *reinterpret_cast<const float4*>(part + i);
#pragma unroll 4
      for (int k = 1; k < splits; ++k) {
        const float4 v = *reinterpret_cast<const float4*>(part + k * n + i);
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
      }
      const float f[4] = {s.x, s.y, s.z, s.w};
      const int64_t r = i / cols;
      *reinterpret_cast<Vec<T, 4>*>(out + r * ld + (i - r * cols)) = pack<T>(f);
    }
    return;
  }
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    float s = part[i];
    for (int k = 1; k < splits; ++k) s += part[k * n + i];
    const int64_t r = i / cols;
    out[r * ld + (i - r * cols)] = from_f32<T>(s);
  }
}

template <typename T>
__global__ void __launch_bounds__(256) xent_zero_kernel(T* out, int64_t rows, int64_t cols, int64_t ld) {
  chain_wait();
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * cols; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / cols;
    out[r * ld + (i - r * cols)] = from_f32<T>(0.0f);
  }
}

// ---- host side ---------------------------------------------------------------------------------------------

size_t up256(size_t x) { return (x + 255) / 256 * 256; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// A bf16 operand (or its three planes) as the product kernels read it.
struct Operand {
  const void* base;
  int64_t inner, outer;     // contiguous extent, and the number of rows that far apart
  int64_t ld, plane;        // elements
  int planes;
};

bool make_map(CUtensorMap* map, const Operand& o, bool mn_major) {
  EncodeTiledFn enc = get_encode_fn();
  if (enc == nullptr) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)o.inner, (cuuint64_t)o.outer, (cuuint64_t)o.planes};
  const cuuint64_t strides[2] = {(cuuint64_t)o.ld * 2, (cuuint64_t)(o.planes > 1 ? o.plane : o.ld) * 2};
  const cuuint32_t box[3] = {64, mn_major ? 64u : 128u, 1};
  const cuuint32_t elem_strides[3] = {1, 1, 1};
  const CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(o.base), dims, strides, box,
                         elem_strides, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                         CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS;
}

struct Product {     // out[M, N] = A B^T with the operands stored as they are
  Operand a, b;
  bool a_mn, b_mn;
  int64_t M, N, K;
};

XProblem make_problem(const Product& g, int splits) {
  XProblem r{};
  r.M = (int32_t)g.M;
  r.N = (int32_t)g.N;
  r.tiles_m = (int32_t)ceil_div(g.M, XM);
  r.tiles_n = (int32_t)ceil_div(g.N, XN);
  r.group_m = 16;
  r.kblocks = (int32_t)ceil_div(g.K, XK);
  r.kblocks_split = (int32_t)ceil_div(r.kblocks, splits);
  r.splits = (int32_t)ceil_div(r.kblocks, r.kblocks_split);
  r.a_mn = g.a_mn;
  r.b_mn = g.b_mn;
  r.two = g.a.planes == 2 ? 1 : g.b.planes == 2 ? 2 : 0;
  r.products = g.a.planes == 3 ? 6 : r.two ? 2 : 1;
  r.items = r.tiles_m * r.tiles_n * r.splits;
  return r;
}

// attribute of a kernel, per device and for as long as the library is loaded: set at its first launch there
template <auto kernel>
cudaError_t allow_smem(int bytes) {
  static std::atomic<uint64_t> ready{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev > 63 || !((ready.load(std::memory_order_relaxed) >> dev) & 1))) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && dev <= 63) ready.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  return e;
}

template <int kEpi, typename C>
hdqt_status_t launch(XParams& p, const Product* g, int n, const C& c) {
  CUtensorMap maps[4];
  for (int i = 0; i < n; ++i) {
    if (!make_map(&maps[2 * i], g[i].a, g[i].a_mn) || !make_map(&maps[2 * i + 1], g[i].b, g[i].b_mn)) return HDQT_ERR_CUDA;
  }
  if (n == 1) { maps[2] = maps[0]; maps[3] = maps[1]; }
  p.num_problems = n;
  const int sms = sm_count();
  if (sms < 2) return HDQT_ERR_CUDA;
  const int items = p.pr[0].items + (n > 1 ? p.pr[1].items : 0);
  const int pairs = items < sms / 2 ? items : sms / 2;
  cudaError_t e = allow_smem<xent_gemm_kernel<kEpi>>(X_SMEM);
  if (e != cudaSuccess) return cuda_failure(e, "cross entropy product");
  c.run(xent_gemm_kernel<kEpi>, 2 * pairs, X_THREADS, X_SMEM, maps[0], maps[1], maps[2], maps[3], p);
  e = cudaGetLastError();
  return e == cudaSuccess ? HDQT_OK : cuda_failure(e, "cross entropy product");
}

// Sizes and workspace of a call.
struct Plan {
  int planes;
  int small_rows;                       // > 0: small problem (hdqt_xent_small.cuh), tokens per block
  size_t small_smem;
  int few_tokens;                       // > 0: loss of a few tokens (hdqt_xent_few.cuh), tokens a thread accumulates
  int few_grad;                         // > 0: a few tokens by streamed products, tokens a thread accumulates
  int few_z_slices, few_dx_slices;
  bool stage_x, stage_w;
  int64_t ld_xs, ld_ws;                 // of the staged copies
  int64_t w_rows, w_cols;
  int64_t rows_piece, cols_piece;       // tokens x classes of a piece
  int64_t ld_z;
  int64_t parts_ld;
  int splits_dx_alone;                  // of dX where dW is not asked for
  int splits_z, splits_dx, splits_dw;   // splits_z > 1: few output blocks, logits as partial products (xent_softmax_kernel)
  int64_t ld_part;
  bool acc_dx, acc_dw;                  // fp32 sums over several pieces
  // weights per row, bf16: in dX's epilogue and in two planes of X (few tokens), or in dz over their largest, which multiplies the sums
  bool plane_weights, unit_weights;
  // workspace offsets
  size_t label, scale, unit, xw, label_logit, loss_rows, part, xs, ws, z, dz, dx_f32, dw_f32, total;
};

constexpr int64_t kPieceBytes = 1ll << 30;
constexpr int64_t kSoftmaxClasses = 12000;      // xent_softmax_kernel holds a row of fp32 logits in 48 KB

// Small problems: most tokens, most elements of W and most products of the two launches of hdqt_xent_small.cuh.
struct SmallLimits {
  int64_t tokens, weights, work;
};
// The rows kernel reads W from the L2 once per token and product and the gradient kernel walks over all tokens, where the
// tensor-core path costs its launches and its pipelines' fill and drain whatever the size: 25 us on the device (30 us a
// call) for bf16 gradients, 47 (51) for fp32, 16 (23) and 33 (35) for the loss alone.  Measured (tokens, features, classes; device, both):
// bf16 gradients 32 x 128 x 64 10 and 20 us, 128 x 512 x 100 27 and 25, 128 x 512 x 300 41 and 27; fp32 gradients 128 x 512 x 100 29 and 47,
// 256 x 512 x 128 44 and 51, 512 x 512 x 128 63 and 49; bf16 loss from W [classes, features] 64 x 512 x 512 14 and 16, from
// [features, classes] 25 and 16; fp32 loss 512 x 512 x 128 26 and 33.  The limits are set by whole calls; on the device alone the
// bf16 loss could leave this path earlier (512 x 256 x 256 in a CUDA graph with a cold L2: 22 us here, 18 there).
SmallLimits small_limits(bool gradients, bool f32, bool w_is_cd) {
  if (!gradients) return f32 || w_is_cd ? SmallLimits{512, 1 << 18, 1 << 25} : SmallLimits{512, 1 << 16, 1 << 25};
  return f32 ? SmallLimits{256, 1 << 18, 1 << 24} : SmallLimits{128, 1 << 16, 1 << 23};
}

// ... and where the streamed products below would do: 2 x 512 x 512 fp32 loss 27 us here and 8 there, gradients 47 and 23.
constexpr int64_t kSmallFewWeights = 1 << 16;

// Streamed products: most tokens of a loss in two launches, and of the calls with products written out.  They cost
// tokens x |W| fp32 operations a product, the tensor-core path the same up to 256 tokens (fp32: six products, and three
// planes of W to be written first).  2048 x 32000, streamed and tensor-core path, us:
//   loss, bf16: 1 token 30 and 53, 4 tokens 47 and 47, 8 tokens 84 and 45 (512 x 4000: 14 and 16)
//   loss, fp32: 8 tokens 91 and 280; 16 tokens 165 and 263, from W [features, classes] 106 and 269
//   gradients, bf16: 4 tokens 127 and 147, 8 tokens 250 and 145; from W [features, classes] 2 tokens 118 and 149, 4 tokens 167 and 150
//   gradients, fp32: 8 tokens 215 and 510, 16 tokens 338 and 495, from W [features, classes] 431 and 505
int64_t few_loss_tokens(bool f32, bool w_is_cd, int64_t weights) {
  // (fp32 from W [features, classes]: beyond two tokens the products of the next function are faster)
  if (f32) return w_is_cd ? kFewTokens : 2;
  return weights <= (1 << 22) ? kFewTokens : 4;
}
int64_t few_product_tokens(bool gradients, bool f32, bool w_is_cd) {
  if (!gradients) return f32 ? (w_is_cd ? 24 : 32) : 0;
  return f32 ? 16 : w_is_cd ? 4 : 2;
}
constexpr size_t kSmallSmem = 100 << 10;
constexpr int kFewBlocks = 4 * kNumSMsHint;      // most blocks of the few-token kernels

// An item shorter than this many stages takes as long all the same: its epilogue (256 x 256 outputs) does.
constexpr int64_t kEpilogueStages = 16;
// So dW of a few tokens takes X in two planes at next to no cost: backward of 28 x 472 x 121432 bf16 154 us and 152 with the weights in
// dz, 100 x 2048 x 32000 152 and 148, 300 x 1024 x 50000 160 and 156, but 512 x 2048 x 32000 221 and 190.  Random weights in dz
// give 1.3 times the error of rounding the exact gradients from a few hundred tokens on, and 1.6 or 2 times with a few.
constexpr int64_t kPlaneTokens = 4 * XK;
int64_t item_cost(int64_t stages) { return stages > kEpilogueStages ? stages : kEpilogueStages; }

// Work items along the contraction of a product of `blocks` output blocks of `kblocks` x `products` stages, next to `other` stages of
// shorter items: the number with the shortest schedule on `pairs` CTA pairs.  A split adds one pass over fp32 partial
// outputs (8 bytes per element at about 6 TB/s against 0.3 us per stage).
int choose_splits(int64_t blocks, int64_t kblocks, int64_t products, int64_t elements, int64_t other, int64_t pairs) {
  int best = 1;
  double best_time = 0.0;
  for (int s = 1; s <= 16; ++s) {
    const int64_t len = item_cost(ceil_div(kblocks, s) * products), items = blocks * s;
    if (s > 1 && (ceil_div(kblocks, s) * products < 12 || ceil_div(kblocks, s) == ceil_div(kblocks, s - 1))) continue;
    const int64_t whole = items / pairs, more = items % pairs;
    const double mean = (double)(items * len + other) / (double)pairs;
    const double longest = (double)((whole + (more > 0)) * len);
    // the pairs with one item fewer fill up with the other product's items
    const bool filled = other >= (more > 0 ? (pairs - more) * len : 0);
    const double time = (filled && mean > len ? mean : longest > mean ? longest : mean) + (s > 1 ? (double)elements * s * 8 / 6e12 / 0.3e-6 + 10.0 : 0.0);
    if (s == 1 || time < best_time) { best = s; best_time = time; }
  }
  return best;
}

hdqt_status_t make_plan(const hdqt_xent_desc_t* d, int kind, Plan* pl) {
  if (!d || kind < HDQT_XENT_FWD || kind > HDQT_XENT_TRAIN) return HDQT_ERR_INVALID_ARG;
  if (d->tokens < 0 || d->features <= 0 || d->classes <= 0 || d->piece_bytes < 0) return HDQT_ERR_INVALID_ARG;
  if (d->dtype != HDQT_DTYPE_F32 && d->dtype != HDQT_DTYPE_BF16)
    return dtype_size(d->dtype) ? HDQT_ERR_UNSUPPORTED : HDQT_ERR_INVALID_ARG;
  if (d->reduction < HDQT_REDUCE_NONE || d->reduction > HDQT_REDUCE_SUM) return HDQT_ERR_INVALID_ARG;
  pl->w_rows = d->w_is_cd ? d->classes : d->features;
  pl->w_cols = d->w_is_cd ? d->features : d->classes;
  if (d->ld_x < d->features || d->ld_w < pl->w_cols) return HDQT_ERR_INVALID_ARG;
  if (kind != HDQT_XENT_FWD && (d->ld_dx < d->features || d->ld_dw < pl->w_cols)) return HDQT_ERR_INVALID_ARG;
  if (d->tokens > (1 << 30) || d->features > (1 << 24) || d->classes > (1 << 30)) return HDQT_ERR_UNSUPPORTED;
  if (ceil_div(d->tokens, XM) * ceil_div(d->classes, XN) > (1 << 26) ||
      ceil_div(d->tokens > d->classes ? d->tokens : d->classes, XM) * ceil_div(d->features, XN) > (1 << 26))
    return HDQT_ERR_UNSUPPORTED;
  const bool f32 = d->dtype == HDQT_DTYPE_F32;
  pl->planes = f32 ? 3 : 1;
  pl->plane_weights = pl->unit_weights = false;       // (tensor-core path: set below)
  pl->small_rows = 0;
  const bool gradients = kind != HDQT_XENT_FWD, cd = d->w_is_cd != 0;
  const int64_t weights = d->classes * d->features;
  const bool any = d->tokens > 0 && d->piece_bytes == 0;      // (a stated piece size selects the tensor-core path)
  const bool few_loss = any && !gradients && d->tokens <= few_loss_tokens(f32, cd, weights);
  const bool few_product = any && d->tokens <= few_product_tokens(gradients, f32, cd);
  const SmallLimits small = small_limits(gradients, f32, cd);
  const int64_t small_weights = few_loss || few_product ? kSmallFewWeights : small.weights;
  if (any && d->tokens <= small.tokens && weights <= small_weights && d->tokens * weights <= small.work) {
    int rows = gradients || d->tokens <= 2 * kNumSMsHint ? 1 : 2;
    auto smem = [&](int r) { return sizeof(float) * (size_t)r * (size_t)(d->features + d->classes + kSmallThreads); };
    if (smem(rows) > kSmallSmem) rows = 1;
    if (smem(rows) <= kSmallSmem) {
      pl->small_rows = rows;
      pl->small_smem = smem(rows);
    }
  }
  pl->few_tokens = 0;
  if (few_loss && pl->small_rows == 0) {
    int n = 1;
    while (n < d->tokens) n *= 2;
    if (4 * n * d->features <= kFewSmem) pl->few_tokens = n;
  }
  pl->few_grad = 0;
  if (few_product && pl->small_rows == 0 && pl->few_tokens == 0) {
    pl->few_grad = 1;
    while (pl->few_grad < d->tokens && pl->few_grad < 16) pl->few_grad *= 2;
  }
  pl->stage_x = f32 || d->ld_x % 8 != 0;
  pl->stage_w = f32 || d->ld_w % 8 != 0;
  pl->ld_xs = ceil_div(d->features, 8) * 8;
  pl->ld_ws = ceil_div(pl->w_cols, 8) * 8;
  const int64_t T = d->tokens > 0 ? d->tokens : 1, V = d->classes, D = d->features;
  // a piece: all classes of some tokens (forward, training) or all tokens of some classes (backward)
  const int64_t elem = f32 ? (kind == HDQT_XENT_TRAIN ? 10 : 6) : 2;
  int64_t budget = d->piece_bytes;
  if (budget == 0) {
    // a second piece needs fp32 sums of dW (dX): splitting below that size would save no memory
    const int64_t sums = 4 * D * (kind == HDQT_XENT_BWD ? T : V);
    budget = kPieceBytes > sums ? kPieceBytes : sums;
  }
  pl->rows_piece = T;
  pl->cols_piece = V;
  if (kind == HDQT_XENT_BWD) {
    const int64_t fit = budget / (T * elem) / 256 * 256;
    if (fit < V) pl->cols_piece = fit > 256 ? fit : 256;
  } else {
    const int64_t ldv = ceil_div(V, 256) * 256;
    // the forward call only holds the parts, 8 bytes per 128 columns
    const int64_t row = kind == HDQT_XENT_TRAIN ? ldv * elem : ldv / 128 * 8;
    const int64_t fit = budget / row / 256 * 256;
    if (fit < T) pl->rows_piece = fit > 256 ? fit : 256;
  }
  if (pl->cols_piece > V) pl->cols_piece = V;
  if (pl->rows_piece > T) pl->rows_piece = T;
  pl->ld_z = ceil_div(pl->cols_piece, 256) * 256;
  pl->parts_ld = ceil_div(V, XN) * 2;
  pl->acc_dw = kind == HDQT_XENT_TRAIN && pl->rows_piece < T;
  pl->acc_dx = kind == HDQT_XENT_BWD && pl->cols_piece < V;
  const int64_t pairs = kNumSMsHint / 2;
  const int64_t dx_blocks = ceil_div(pl->rows_piece, XM) * ceil_div(D, XN), dx_k = ceil_div(pl->cols_piece, XK);
  const int64_t dw_blocks = ceil_div(pl->cols_piece, XM) * ceil_div(D, XN), dw_k = ceil_div(pl->rows_piece, XK);
  const int64_t pieces = ceil_div(V, pl->cols_piece);
  const int64_t products = f32 ? 6 : 1;
  pl->splits_dx = choose_splits(dx_blocks, dx_k, products, pl->rows_piece * D, dw_blocks * item_cost(dw_k * products), pairs);
  pl->splits_dw = pl->acc_dw ? 1 : choose_splits(dw_blocks, dw_k, products, pl->cols_piece * D, dx_blocks * item_cost(dx_k * products), pairs);
  pl->splits_dx_alone = choose_splits(dx_blocks, dx_k, products, pl->rows_piece * D, 0, pairs);
  if (pl->acc_dx) {
    // the pieces leave the shares of their splits side by side where there is room for them, and add to one sum otherwise
    const int64_t most = budget / (4 * pieces * T * D);
    if (pl->splits_dx > most) pl->splits_dx = most > 1 ? (int)most : 1;
    if (pl->splits_dx_alone > most) pl->splits_dx_alone = most > 1 ? (int)most : 1;
  }
  pl->splits_z = 1;
  pl->ld_part = ceil_div(V, 8) * 8;
  if (pl->rows_piece == T && pl->cols_piece == V && V <= kSoftmaxClasses && d->piece_bytes == 0)
    pl->splits_z = choose_splits(ceil_div(T, XM) * ceil_div(V, XN), ceil_div(D, XK), products, T * V, 0, pairs);

  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t at = o; o += up256(bytes); return at; };
  if (pl->small_rows > 0) {
    pl->loss_rows = take(4 * T);
    pl->dz = kind == HDQT_XENT_FWD ? o : take(4 * T * V);
    pl->total = o;
    return HDQT_OK;
  }
  if (pl->few_tokens > 0) {
    pl->label_logit = take(4 * T);
    pl->part = take(sizeof(float2) * T * kFewBlocks);
    pl->total = o;
    return HDQT_OK;
  }
  if (pl->few_grad > 0) {
    // slices of the contraction: enough blocks to fill the machine, at least 64 rows or 512 columns each
    // (threads of four columns on average; a block of 256)
    const int64_t cols_blocks_v = ceil_div(V, 1024), cols_blocks_d = ceil_div(D, 1024);
    auto slices = [&](int64_t blocks, int64_t k, int64_t least) {
      int64_t s = ceil_div(6 * kNumSMsHint, blocks);
      const int64_t most = ceil_div(k, least);
      return (int)(s < most ? s : most);
    };
    pl->few_z_slices = d->w_is_cd ? slices(ceil_div(V, 16), D, 512) : slices(cols_blocks_v, D, 64);
    pl->few_dx_slices = d->w_is_cd ? slices(cols_blocks_d, V, 64) : slices(ceil_div(D, 16), V, 512);
    pl->label = take(4 * T);
    pl->scale = take(256);
    pl->loss_rows = take(4 * T);
    pl->label_logit = take(4 * T);
    pl->part = take(sizeof(float2) * T * ceil_div(V, kFewSpan));
    pl->z = take(4 * T * V * pl->few_z_slices);
    pl->dx_f32 = kind == HDQT_XENT_FWD ? o : take(4 * T * D * pl->few_dx_slices);
    pl->total = o;
    return HDQT_OK;
  }
  pl->label = take(4 * T);
  pl->scale = take(256);
  const bool row_weights = !f32 && gradients && d->reduction == HDQT_REDUCE_NONE;
  pl->plane_weights = row_weights && T <= kPlaneTokens;
  pl->unit_weights = row_weights && T > kPlaneTokens;
  pl->unit = row_weights ? take(4 * T) : o;
  pl->xw = pl->plane_weights ? take(2 * 2 * T * pl->ld_xs) : o;
  pl->label_logit = take(4 * T);
  pl->loss_rows = take(4 * T);
  pl->part = kind == HDQT_XENT_BWD ? o : take(8 * pl->rows_piece * pl->parts_ld);
  pl->xs = pl->stage_x ? take(2 * pl->planes * T * pl->ld_xs) : o;
  pl->ws = pl->stage_w ? take(2 * pl->planes * pl->w_rows * pl->ld_ws) : o;
  pl->z = pl->dz = o;
  if (pl->splits_z > 1) {
    pl->z = take(4 * pl->splits_z * T * pl->ld_part);
    pl->dz = kind == HDQT_XENT_FWD ? o : take(2 * pl->planes * T * pl->ld_z);
  } else if (kind == HDQT_XENT_TRAIN) {
    pl->z = take((f32 ? 4 : 2) * pl->rows_piece * pl->ld_z);
    pl->dz = f32 ? take(6 * pl->rows_piece * pl->ld_z) : pl->z;
  } else if (kind == HDQT_XENT_BWD) {
    pl->dz = take(2 * pl->planes * pl->rows_piece * pl->ld_z);
  }
  pl->dx_f32 = pl->dw_f32 = o;
  if (kind != HDQT_XENT_FWD) {
    const int64_t most_dx = pl->splits_dx > pl->splits_dx_alone ? pl->splits_dx : pl->splits_dx_alone;
    if (most_dx > 1) pl->dx_f32 = take(4 * pieces * most_dx * pl->rows_piece * D);
    else if (pl->acc_dx && !f32) pl->dx_f32 = take(4 * T * D);
    if (pl->splits_dw > 1) pl->dw_f32 = take(4 * pl->splits_dw * pl->cols_piece * D);
    else if (pl->acc_dw && !f32) pl->dw_f32 = take(4 * V * D);
  }
  pl->total = o;
  return HDQT_OK;
}

struct Call {
  const hdqt_xent_desc_t* d;
  Plan pl;
  uint8_t* ws;
  int32_t* dev_status;
  cudaStream_t s;
  Operand x, w;          // as stored: x [tokens, features], w [w_rows, w_cols]
  const float* row_weights = nullptr;   // [tokens]: weights of the rows' losses
  const float* alpha = nullptr;         // or one weight for all, applied to the gradient products
  const float* row_scale = nullptr;     // [tokens]: weights that dX's epilogue applies, dW's X being weighted X

  mutable bool started = false;
  mutable int dx_shares = 0;            // partial products of dX so far (backward call in pieces)

  template <typename T>
  T* at(size_t off) const { return reinterpret_cast<T*>(ws + off); }

  // the call's kernels, in order: the first behind everything on the stream, the others chained to it
  template <typename... P, typename... A>
  void run(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, A&&... args) const {
    if (started) launch_chained(kernel, grid, block, smem, s, args...);
    else kernel<<<grid, block, smem, s>>>(static_cast<P>(args)...);
    started = true;
  }

  Operand x_rows(int64_t t0, int64_t n) const {
    Operand o = x;
    o.base = reinterpret_cast<const uint16_t*>(x.base) + t0 * x.ld;
    o.outer = n;
    return o;
  }
  // X as dW reads it
  Operand x_rows_dw(int64_t t0, int64_t n) const {
    if (!pl.plane_weights) return x_rows(t0, n);
    return Operand{at<uint16_t>(pl.xw) + t0 * pl.ld_xs, d->features, n, pl.ld_xs, d->tokens * pl.ld_xs, 2};
  }
  // the columns [v0, v0 + n) of the vocabulary
  Operand w_classes(int64_t v0, int64_t n) const {
    Operand o = w;
    o.base = reinterpret_cast<const uint16_t*>(w.base) + (d->w_is_cd ? v0 * w.ld : v0);
    (d->w_is_cd ? o.outer : o.inner) = n;
    return o;
  }
  Operand dz(int64_t rows, int64_t cols) const {
    Operand o;
    o.base = at<uint16_t>(pl.dz);
    o.inner = cols;
    o.outer = rows;
    o.ld = pl.ld_z;
    o.plane = pl.rows_piece * pl.ld_z;
    o.planes = pl.planes;
    return o;
  }
};

void fill_common(const Call& c, XParams* p) {
  memset(p, 0, sizeof(*p));
  p->planes = c.pl.planes;
  // stages per part: 1024 additions of 16 products for bf16 results, 32 where fp32 precision is to be kept
  p->part_iters = c.pl.planes == 1 ? 256 : 8;
  p->dev_status = c.dev_status;
}

// checks, staged operands and labels: what all three calls begin with
hdqt_status_t begin(Call* c, const hdqt_xent_desc_t* d, int kind, const void* X, const void* W, const int64_t* labels,
                    void* workspace, size_t workspace_bytes, int32_t* dev_status, void* stream) {
  const hdqt_status_t st = make_plan(d, kind, &c->pl);
  if (st != HDQT_OK) return st;
  const bool empty = d->tokens == 0;
  if (!W || !workspace || (!empty && (!X || !labels))) return HDQT_ERR_INVALID_ARG;
  const uintptr_t need = d->dtype == HDQT_DTYPE_BF16 ? 15 : 3;
  if (((reinterpret_cast<uintptr_t>(X) | reinterpret_cast<uintptr_t>(W)) & need) || (reinterpret_cast<uintptr_t>(labels) & 7) ||
      (reinterpret_cast<uintptr_t>(workspace) & 255))
    return HDQT_ERR_ALIGNMENT;
  if (workspace_bytes < c->pl.total) return HDQT_ERR_WORKSPACE;
  c->d = d;
  c->ws = reinterpret_cast<uint8_t*>(workspace);
  c->dev_status = dev_status;
  c->s = reinterpret_cast<cudaStream_t>(stream);
  return HDQT_OK;
}

hdqt_status_t stage(const Call& c, const void* src, int64_t ld, int64_t rows, int64_t cols, size_t off, int64_t ld_dst,
                    Operand* o) {
  uint16_t* dst = c.at<uint16_t>(off);
  o->base = dst;
  o->ld = ld_dst;
  o->plane = rows * ld_dst;
  if (rows == 0) return HDQT_OK;
  // four rows per thread while that leaves enough blocks; fp32 in accesses of four, two or one element as the rows allow
  const uintptr_t bits = reinterpret_cast<uintptr_t>(src) | (uintptr_t)(ld * 4) | (uintptr_t)(cols * 4);
  const bool two = c.d->dtype == HDQT_DTYPE_F32 && (bits & 15) != 0 && (bits & 7) == 0;
  const int64_t bx = ceil_div(cols, two ? 512 : 1024);
  int64_t by = ceil_div(rows, 4);
  if (bx * by < 8 * kNumSMsHint) by = rows;
  const dim3 grid((unsigned)bx, (unsigned)(by < 65535 ? by : 65535));
  if (c.d->dtype == HDQT_DTYPE_F32) {
    c.run((bits & 15) == 0 ? xent_stage_kernel<float, 4, true> : two ? xent_stage_kernel<float, 2, true> : xent_stage_kernel<float, 4, false>,
          grid, 256, 0, reinterpret_cast<const float*>(src), ld, rows, cols, dst, ld_dst, rows * ld_dst);
  } else {
    c.run(xent_stage_kernel<__nv_bfloat16, 4, false>, grid, 256, 0, reinterpret_cast<const __nv_bfloat16*>(src), ld, rows, cols,
          dst, ld_dst, 0);
  }
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? HDQT_OK : cuda_failure(e, "cross entropy operands");
}

void label_rows(Call* c, const int64_t* labels, const float* g) {
  const hdqt_xent_desc_t& d = *c->d;
  const Plan& pl = c->pl;
  // a weight per row goes into dz; one weight for all multiplies the fp32 sums of the gradient products, so that rounding dz
  // to bf16 never rounds the weight (1 / rows would be off by the same 0.1 % in almost every element); of weights per row the
  // largest does, so that equal ones are as good as one
  const bool rows = d.reduction == HDQT_REDUCE_NONE;
  const bool unit = pl.unit_weights;
  c->row_weights = unit ? c->at<float>(pl.unit) : rows && !pl.plane_weights ? g : nullptr;
  c->row_scale = pl.plane_weights ? c->at<float>(pl.unit) : nullptr;
  c->alpha = rows && !unit ? nullptr : c->at<float>(pl.scale) + 1;
  c->run(xent_labels_kernel, 1, d.tokens > 512 ? 1024 : 256, 0, labels, d.tokens, d.classes, d.ignore_index,
         d.reduction == HDQT_REDUCE_MEAN, rows ? nullptr : g, c->at<int32_t>(pl.label), c->at<float>(pl.scale),
         unit ? g : nullptr, unit ? c->at<float>(pl.unit) : nullptr, c->dev_status);
}

hdqt_status_t prepare(Call* c, const void* X, const void* W, const int64_t* labels, const float* g) {
  const hdqt_xent_desc_t& d = *c->d;
  const Plan& pl = c->pl;
  c->x = Operand{X, d.features, d.tokens, d.ld_x, 0, pl.planes};
  c->w = Operand{W, pl.w_cols, pl.w_rows, d.ld_w, 0, pl.planes};
  hdqt_status_t st = HDQT_OK;
  if (pl.stage_x) st = stage(*c, X, d.ld_x, d.tokens, d.features, pl.xs, pl.ld_xs, &c->x);
  if (st == HDQT_OK && pl.stage_w) st = stage(*c, W, d.ld_w, pl.w_rows, pl.w_cols, pl.ws, pl.ld_ws, &c->w);
  if (st != HDQT_OK) return st;
  label_rows(c, labels, g);
  if (pl.plane_weights && d.tokens > 0)
    c->run(xent_weighted_rows_kernel, dim3((unsigned)ceil_div(d.features, 1024), (unsigned)d.tokens), 256, 0,
           reinterpret_cast<const __nv_bfloat16*>(c->x.base), c->x.ld, d.features, c->at<int32_t>(pl.label), g,
           c->at<uint16_t>(pl.xw), pl.ld_xs, d.tokens * pl.ld_xs, c->at<float>(pl.unit));
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? HDQT_OK : cuda_failure(e, "cross entropy labels");
}

Product logits_product(const Call& c, int64_t t0, int64_t nt, int64_t v0, int64_t nv) {
  return Product{c.x_rows(t0, nt), c.w_classes(v0, nv), false, c.d->w_is_cd == 0, nt, nv, c.d->features};
}

// dX and dW of a piece whose dz lies in the workspace: one launch
hdqt_status_t gradient_products(const Call& c, int64_t t0, int64_t nt, int64_t v0, int64_t nv, void* dX, void* dW,
                                bool first, bool last) {
  const hdqt_xent_desc_t& d = *c.d;
  const Plan& pl = c.pl;
  const bool bf16 = d.dtype == HDQT_DTYPE_BF16;
  const int64_t D = d.features;
  XParams p;
  fill_common(c, &p);
  p.alpha = c.alpha;
  Product g[2];
  int n = 0;
  const Operand dz = c.dz(nt, nv);
  void* dx_rows = dX ? reinterpret_cast<uint8_t*>(dX) + t0 * d.ld_dx * (bf16 ? 2 : 4) : nullptr;
  void* dw_out = dW ? reinterpret_cast<uint8_t*>(dW) + (d.w_is_cd ? v0 * d.ld_dw : v0) * (bf16 ? 2 : 4) : nullptr;
  int dx_total = 0;           // shares of dX to be joined
  // where a product goes: partial sums of its splits, the result itself, or fp32 sums over the pieces
  auto target = [&](XProblem& r, void* out, int64_t ld, bool acc, float* f32, int64_t f32_ld) {
    if (r.splits > 1) {
      r.out = f32;
      r.ld_out = f32_ld;
      r.split_stride = (int64_t)r.M * f32_ld;
    } else if (!acc || !bf16) {
      r.out = out;
      r.ld_out = ld;
      r.out_bf16 = bf16;
      if (acc && !first) { r.add = reinterpret_cast<const float*>(r.out); r.ld_add = ld; }
    } else {
      if (!first) { r.add = f32; r.ld_add = f32_ld; }
      r.out = last ? out : static_cast<void*>(f32);
      r.ld_out = last ? ld : f32_ld;
      r.out_bf16 = last;
    }
  };
  if (dX) {
    // dX[t, d] = sum_v dz[t, v] W[v, d]
    g[n] = Product{dz, c.w_classes(v0, nv), false, d.w_is_cd != 0, nt, D, nv};
    const int splits = dW ? pl.splits_dx : pl.splits_dx_alone;
    p.pr[n] = make_problem(g[n], splits);
    p.pr[n].row_scale = c.row_scale != nullptr ? c.row_scale + t0 : nullptr;
    if (splits > 1) {
      // (a last piece may be too short for two splits: its share is joined with the others all the same)
      XProblem& r = p.pr[n];
      r.out = c.at<float>(pl.dx_f32) + c.dx_shares * nt * D;
      r.ld_out = D;
      r.split_stride = nt * D;
      dx_total = c.dx_shares + r.splits;
      c.dx_shares = pl.acc_dx ? dx_total : 0;
    } else {
      target(p.pr[n], dx_rows, d.ld_dx, pl.acc_dx, c.at<float>(pl.dx_f32), D);
    }
    ++n;
  }
  if (dW) {
    // dW[v, d] = sum_t dz[t, v] X[t, d], or its transpose
    if (d.w_is_cd) {
      g[n] = Product{dz, c.x_rows_dw(t0, nt), true, true, nv, D, nt};
    } else {
      g[n] = Product{c.x_rows_dw(t0, nt), dz, true, true, D, nv, nt};
    }
    p.pr[n] = make_problem(g[n], pl.splits_dw);
    target(p.pr[n], dw_out, d.ld_dw, pl.acc_dw, c.at<float>(pl.dw_f32), d.w_is_cd ? D : nv);
    ++n;
  }
  if (n == 0) return HDQT_OK;
  auto join = [&](int shares, int64_t M, int64_t N, void* out, int64_t ld, size_t off) {
    const int64_t blocks = ceil_div(M * N, 1024);
    const unsigned grid = (unsigned)(blocks < 148 * 8 ? blocks : 148 * 8);
    if (bf16) c.run(xent_join_splits_kernel<__nv_bfloat16>, grid, 256, 0, c.at<float>(off), shares, M, N, reinterpret_cast<__nv_bfloat16*>(out), ld);
    else c.run(xent_join_splits_kernel<float>, grid, 256, 0, c.at<float>(off), shares, M, N, reinterpret_cast<float*>(out), ld);
  };
  const XProblem dw_problem = p.pr[n - 1];      // (if dW is asked for)
  if (n == 2) {
    auto length = [&](int i) { return (int64_t)p.pr[i].kblocks_split * p.pr[i].products; };
    if (length(1) > length(0)) {      // the longer items first
      std::swap(p.pr[0], p.pr[1]);
      std::swap(g[0], g[1]);
    }
    p.extra = (int32_t)(item_cost(length(0)) / item_cost(length(1)));
  }
  const hdqt_status_t st = launch<X_OUT>(p, g, n, c);
  if (st != HDQT_OK) return st;
  if (dx_total > 0 && (last || !pl.acc_dx)) join(dx_total, nt, D, dx_rows, d.ld_dx, pl.dx_f32);
  if (dW && dw_problem.splits > 1) join(dw_problem.splits, dw_problem.M, dw_problem.N, dw_out, d.ld_dw, pl.dw_f32);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? HDQT_OK : cuda_failure(e, "cross entropy gradients");
}

hdqt_status_t zero_out(const Call& c, void* out, int64_t rows, int64_t cols, int64_t ld) {
  if (c.d->dtype == HDQT_DTYPE_BF16) c.run(xent_zero_kernel<__nv_bfloat16>, 148 * 4, 256, 0, reinterpret_cast<__nv_bfloat16*>(out), rows, cols, ld);
  else c.run(xent_zero_kernel<float>, 148 * 4, 256, 0, reinterpret_cast<float*>(out), rows, cols, ld);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? HDQT_OK : cuda_failure(e, "cross entropy gradients");
}

// reduced loss from the rows' losses (which are the result themselves without a reduction)
hdqt_status_t reduce_loss(const Call& c, float* loss) {
  if (c.d->reduction != HDQT_REDUCE_NONE)
    c.run(xent_loss_kernel, 1, 1024, 0, c.at<float>(c.pl.loss_rows), c.d->tokens, c.at<float>(c.pl.scale), loss);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? HDQT_OK : cuda_failure(e, "cross entropy loss");
}

// A small problem in two launches.  kind as in the plan; lse_in for the backward call.
template <typename T>
hdqt_status_t run_small(const Call& c, int kind, const void* X, const void* W, const int64_t* labels, const float* lse_in,
                        const float* g, float* loss, float* lse, void* dX, void* dW) {
  const hdqt_xent_desc_t& d = *c.d;
  const bool none = d.reduction == HDQT_REDUCE_NONE;
  SmallParams p{};
  p.x = X;
  p.w = W;
  p.labels = labels;
  p.g = g;
  p.lse_in = lse_in;
  p.lse = lse;
  p.loss_rows = kind == HDQT_XENT_BWD ? nullptr : none ? loss : c.at<float>(c.pl.loss_rows);
  p.dz = dW ? c.at<float>(c.pl.dz) : nullptr;
  p.dx = dX;
  p.dw = dW;
  p.loss = kind == HDQT_XENT_BWD || none ? nullptr : loss;
  p.dev_status = c.dev_status;
  p.ignore = d.ignore_index;
  p.ld_x = d.ld_x;
  p.ld_w = d.ld_w;
  p.ld_dx = d.ld_dx;
  p.ld_dw = d.ld_dw;
  p.tokens = (int32_t)d.tokens;
  p.features = (int32_t)d.features;
  p.classes = (int32_t)d.classes;
  p.w_is_cd = d.w_is_cd != 0;
  p.g_rows = none;
  p.mean = d.reduction == HDQT_REDUCE_MEAN;
  const unsigned blocks = (unsigned)ceil_div(d.tokens, c.pl.small_rows);
  cudaError_t e = c.pl.small_rows == 1 ? allow_smem<xent_small_rows_kernel<T, 1>>((int)kSmallSmem)
                                       : allow_smem<xent_small_rows_kernel<T, 2>>((int)kSmallSmem);
  if (e != cudaSuccess) return cuda_failure(e, "cross entropy");
  if (c.pl.small_rows == 1) c.run(xent_small_rows_kernel<T, 1>, blocks, kSmallThreads, c.pl.small_smem, p);
  else c.run(xent_small_rows_kernel<T, 2>, blocks, kSmallThreads, c.pl.small_smem, p);
  if (dW || p.loss) {
    const dim3 grid((dW ? (unsigned)ceil_div(d.features, 32) : 0) + 1, dW ? (unsigned)ceil_div(d.classes, 32) : 1);
    c.run(xent_small_grad_kernel<T>, grid, kGradThreads, 0, p);
  }
  e = cudaGetLastError();
  return e == cudaSuccess ? HDQT_OK : cuda_failure(e, "cross entropy");
}

template <typename T, int kT, int kV>
cudaError_t run_few_kernel(const Call& c, const FewParams& p, int* blocks) {
  const size_t smem = sizeof(float) * kT * (size_t)p.features;
  constexpr int per_sm = 4;
  const int tile = c.d->w_is_cd ? 4 * kFewWarps : 8 * kV;
  int64_t n = ceil_div(p.classes, tile);
  *blocks = (int)(n < per_sm * kNumSMsHint ? n : per_sm * kNumSMsHint);
  // whole rounds: every block the same number of tiles, if that can be had with little fewer blocks
  const int64_t rounds = ceil_div(n, *blocks);
  *blocks = (int)ceil_div(n, rounds);
  cudaError_t e;
  if (c.d->w_is_cd) {
    e = allow_smem<xent_few_rows_kernel<T, kT, kV>>(kFewSmem);
    if (e == cudaSuccess) c.run(xent_few_rows_kernel<T, kT, kV>, *blocks, kFewThreads, smem, p);
  } else if constexpr (sizeof(T) == 2 || kT <= 2) {            // (few_loss_tokens)
    e = allow_smem<xent_few_columns_kernel<T, kT, kV>>(kFewSmem);
    if (e == cudaSuccess) c.run(xent_few_columns_kernel<T, kT, kV>, *blocks, kFewThreads, smem, p);
  } else {
    e = cudaErrorInvalidValue;
  }
  return e;
}

template <typename T, int kV>
cudaError_t run_few_tokens(const Call& c, const FewParams& p, int* blocks) {
  switch (c.pl.few_tokens) {
    case 1: return run_few_kernel<T, 1, kV>(c, p, blocks);
    case 2: return run_few_kernel<T, 2, kV>(c, p, blocks);
    case 4: return run_few_kernel<T, 4, kV>(c, p, blocks);
    default: return run_few_kernel<T, 8, kV>(c, p, blocks);
  }
}

// Loss of a few tokens in two launches.
hdqt_status_t few(const Call& c, const void* X, const void* W, const int64_t* labels, float* loss, float* lse) {
  const hdqt_xent_desc_t& d = *c.d;
  FewParams p{};
  p.x = X;
  p.w = W;
  p.labels = labels;
  p.part = c.at<float2>(c.pl.part);
  p.label_logit = c.at<float>(c.pl.label_logit);
  p.ld_x = d.ld_x;
  p.ld_w = d.ld_w;
  p.tokens = (int32_t)d.tokens;
  p.features = (int32_t)d.features;
  p.classes = (int32_t)d.classes;
  const int elem = dtype_size(d.dtype), vec = 16 / elem;
  const bool wide = (reinterpret_cast<uintptr_t>(W) & 15) == 0 && d.ld_w % vec == 0 && c.pl.w_cols % vec == 0;
  int blocks = 0;
  cudaError_t e;
  if (elem == 2) e = wide ? run_few_tokens<__nv_bfloat16, 8>(c, p, &blocks) : run_few_tokens<__nv_bfloat16, 1>(c, p, &blocks);
  else e = wide ? run_few_tokens<float, 4>(c, p, &blocks) : run_few_tokens<float, 1>(c, p, &blocks);
  if (e != cudaSuccess) return cuda_failure(e, "cross entropy of a few tokens");
  c.run(xent_few_join_kernel, 1, kFewThreads, 0, p.part, blocks, p.label_logit, labels, p.tokens, p.classes, d.ignore_index,
        d.reduction, lse, loss, c.dev_status);
  e = cudaGetLastError();
  return e == cudaSuccess ? HDQT_OK : cuda_failure(e, "cross entropy of a few tokens");
}

template <typename T, int kT, bool kOuter>
void run_few_columns(const Call& c, const FewProduct& p, int slices, bool wide) {
  // 16-byte accesses while the sums of so many columns fit into registers, then two elements, or one where rows are odd
  constexpr int kC = kT <= 8 ? 16 / (int)sizeof(T) : 2;
  const int groups = (int)ceil_div(p.tokens, kT);
  auto go = [&](auto kernel, int columns) {
    const int64_t per_row = ceil_div(p.N, columns);
    const int threads = per_row < kFewThreads ? (int)ceil_div(per_row, 32) * 32 : kFewThreads;
    c.run(kernel, dim3((unsigned)(ceil_div(per_row, threads) * groups), slices), threads, 0, p);
  };
  if (wide) go(xent_few_columns_product_kernel<T, kT, kC, kOuter>, kC);
  else go(xent_few_columns_product_kernel<T, kT, 1, kOuter>, 1);
}

template <typename T, bool kOuter>
void few_columns_product(const Call& c, FewProduct p, int slices) {
  p.per_slice = (int32_t)ceil_div(p.K, slices);
  const int n = c.pl.few_grad;
  const uintptr_t bits = reinterpret_cast<uintptr_t>(p.m) | (uintptr_t)(p.ld_m * sizeof(T)) | (uintptr_t)(p.N * sizeof(T)) |
                         (kOuter ? reinterpret_cast<uintptr_t>(p.outer) | (uintptr_t)(p.ld_outer * sizeof(T)) : 0);
  const bool wide = (bits & (n <= 8 ? 15 : 2 * sizeof(T) - 1)) == 0;
  if (n == 1) return run_few_columns<T, 1, kOuter>(c, p, slices, wide);
  if (n == 2) return run_few_columns<T, 2, kOuter>(c, p, slices, wide);
  if (sizeof(T) == 2 || n == 4) return run_few_columns<T, 4, kOuter>(c, p, slices, wide);
  if constexpr (sizeof(T) == 4) {                               // (few_product_tokens)
    if (n == 8) return run_few_columns<T, 8, kOuter>(c, p, slices, wide);
    return run_few_columns<T, 16, kOuter>(c, p, slices, wide);
  }
}

template <typename T, int kT>
void run_few_rows(const Call& c, const FewProduct& p, int slices) {
  constexpr int kV = 16 / (int)sizeof(T), kN = 4;
  const dim3 grid((unsigned)(ceil_div(p.N, kN * kFewWarps) * ceil_div(p.tokens, kT)), slices);
  const bool wide = ((reinterpret_cast<uintptr_t>(p.m) | (uintptr_t)(p.ld_m * sizeof(T)) | (uintptr_t)(p.K * sizeof(T))) & 15) == 0 &&
                    p.per_slice % kV == 0;
  if (wide) c.run(xent_few_product_rows_kernel<T, kT, kV>, grid, kFewThreads, 0, p);
  else c.run(xent_few_product_rows_kernel<T, kT, 1>, grid, kFewThreads, 0, p);
}

template <typename T>
void few_rows_product(const Call& c, FewProduct p, int slices) {
  p.per_slice = (int32_t)(ceil_div(ceil_div(p.K, slices), 8) * 8);
  const int n = c.pl.few_grad;
  if (n == 1) return run_few_rows<T, 1>(c, p, slices);
  if (n == 2) return run_few_rows<T, 2>(c, p, slices);
  if (sizeof(T) == 2 || n == 4) return run_few_rows<T, 4>(c, p, slices);
  if constexpr (sizeof(T) == 4) return run_few_rows<T, 8>(c, p, slices);
}

// A few tokens by streamed products: logits, softmax, dX and dW (and the reduced loss by the caller).
template <typename T>
hdqt_status_t run_few_grad(Call& c, int kind, const void* X, const void* W, const int64_t* labels, const float* lse_in,
                           const float* g, float* loss_rows, float* lse, void* dX, void* dW) {
  const hdqt_xent_desc_t& d = *c.d;
  const Plan& pl = c.pl;
  const int f32 = d.dtype == HDQT_DTYPE_F32;
  const int32_t tokens = (int32_t)d.tokens, D = (int32_t)d.features, V = (int32_t)d.classes;
  label_rows(&c, labels, g);
  float* z = c.at<float>(pl.z);
  FewProduct q{};
  q.in = FewMatrix{X, d.ld_x, f32};
  q.m = W;
  q.ld_m = d.ld_w;
  q.out = z;
  q.tokens = tokens;
  q.N = V;
  q.K = D;
  if (d.w_is_cd) few_rows_product<T>(c, q, pl.few_z_slices);
  else few_columns_product<T, false>(c, q, pl.few_z_slices);
  const bool grads = kind != HDQT_XENT_FWD;
  const dim3 spans((unsigned)ceil_div(V, kFewSpan), (unsigned)tokens);
  if (lse_in == nullptr || pl.few_z_slices > 1)
    c.run(xent_few_stats_kernel, spans, kFewThreads, 0, z, pl.few_z_slices, tokens, V, c.at<int32_t>(pl.label),
          c.at<float2>(pl.part), c.at<float>(pl.label_logit));
  c.run(xent_few_softmax_kernel, spans, kFewThreads, 0, z, V, c.at<float2>(pl.part),
        c.at<int32_t>(pl.label), c.at<float>(pl.label_logit), c.row_weights, c.at<float>(pl.scale) + 1, lse_in, lse, loss_rows,
        grads ? 1 : 0);
  if (grads && (dX || dW)) {
    FewProduct r{};
    r.in = FewMatrix{z, V, 1};
    r.b = FewMatrix{X, d.ld_x, f32};
    r.m = W;
    r.ld_m = d.ld_w;
    r.out = dX ? c.at<float>(pl.dx_f32) : nullptr;
    r.tokens = tokens;
    r.N = D;
    r.K = V;
    if (d.w_is_cd) {             // W [classes, features]: one pass for both
      r.outer = dW;
      r.ld_outer = d.ld_dw;
      if (dW) few_columns_product<T, true>(c, r, pl.few_dx_slices);
      else few_columns_product<T, false>(c, r, pl.few_dx_slices);
    } else {
      if (dX) few_rows_product<T>(c, r, pl.few_dx_slices);
      if (dW) {
        FewProduct o{};          // dW [features, classes]
        o.in = FewMatrix{X, d.ld_x, f32};
        o.b = FewMatrix{z, V, 1};
        o.outer = dW;
        o.ld_outer = d.ld_dw;
        o.tokens = tokens;
        o.N = V;
        o.K = D;
        few_columns_product<T, true>(c, o, pl.few_z_slices);
      }
    }
    if (dX) {
      const int64_t total = (int64_t)tokens * D;
      c.run(xent_few_join_slices_kernel<T>, (unsigned)ceil_div(total, 16), 256, 0, r.out, pl.few_dx_slices, total, D,
            reinterpret_cast<T*>(dX), d.ld_dx);
    }
  }
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? HDQT_OK : cuda_failure(e, "cross entropy of a few tokens");
}

hdqt_status_t few_grad(Call& c, int kind, const void* X, const void* W, const int64_t* labels, const float* lse_in,
                       const float* g, float* loss_rows, float* lse, void* dX, void* dW) {
  return c.d->dtype == HDQT_DTYPE_BF16 ? run_few_grad<__nv_bfloat16>(c, kind, X, W, labels, lse_in, g, loss_rows, lse, dX, dW)
                                       : run_few_grad<float>(c, kind, X, W, labels, lse_in, g, loss_rows, lse, dX, dW);
}

hdqt_status_t small(const Call& c, int kind, const void* X, const void* W, const int64_t* labels, const float* lse_in,
                    const float* g, float* loss, float* lse, void* dX, void* dW) {
  return c.d->dtype == HDQT_DTYPE_BF16 ? run_small<__nv_bfloat16>(c, kind, X, W, labels, lse_in, g, loss, lse, dX, dW)
                                       : run_small<float>(c, kind, X, W, labels, lse_in, g, loss, lse, dX, dW);
}

// Few output blocks: logits in partial products, then a block per row.  dz (kind != forward) is left for the gradient products.
hdqt_status_t split_logits(const Call& c, int kind, const float* lse_in, float* loss_rows, float* lse) {
  const hdqt_xent_desc_t& d = *c.d;
  const Plan& pl = c.pl;
  const Product g = logits_product(c, 0, d.tokens, 0, d.classes);
  XParams p;
  fill_common(c, &p);
  p.pr[0] = make_problem(g, pl.splits_z);
  p.pr[0].out = c.at<float>(pl.z);
  p.pr[0].ld_out = pl.ld_part;
  p.pr[0].split_stride = d.tokens * pl.ld_part;
  const hdqt_status_t st = launch<X_OUT>(p, &g, 1, c);
  if (st != HDQT_OK) return st;
  const size_t smem = sizeof(float) * (size_t)d.classes;
  auto go = [&](auto kernel, int threads) {
    c.run(kernel, (unsigned)d.tokens, threads, smem, c.at<float>(pl.z), p.pr[0].splits, d.tokens, pl.ld_part,
          (int)d.classes, c.at<int32_t>(pl.label), c.row_weights, lse_in, c.at<uint16_t>(pl.dz), pl.ld_z,
          d.tokens * pl.ld_z, lse, loss_rows);
  };
  if (d.tokens > 16 * kNumSMsHint && d.classes <= 128) {
    // many short rows: a warp for each (fp32 loss and gradients of 8000 x 512 x 100: 71 us, 80 with blocks of 256 threads; of
    // 1000 x 512 x 100 33 us backward with blocks, 35 with warps)
    if (kind == HDQT_XENT_FWD) go(xent_softmax_kernel<0, 32>, 32);
    else if (pl.planes == 1) go(xent_softmax_kernel<1, 32>, 32);
    else go(xent_softmax_kernel<3, 32>, 32);
  } else if (d.tokens > 2 * kNumSMsHint || d.classes <= 1024) {
    if (kind == HDQT_XENT_FWD) go(xent_softmax_kernel<0, kRowThreads>, kRowThreads);
    else if (pl.planes == 1) go(xent_softmax_kernel<1, kRowThreads>, kRowThreads);
    else go(xent_softmax_kernel<3, kRowThreads>, kRowThreads);
  } else {                    // few long rows: more threads for each
    if (kind == HDQT_XENT_FWD) go(xent_softmax_kernel<0, 1024>, 1024);
    else if (pl.planes == 1) go(xent_softmax_kernel<1, 1024>, 1024);
    else go(xent_softmax_kernel<3, 1024>, 1024);
  }
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? HDQT_OK : cuda_failure(e, "cross entropy rows");
}

bool outputs_misaligned(const hdqt_xent_desc_t* d, const void* a, const void* b) {
  return ((reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b)) & (uintptr_t)(dtype_size(d->dtype) - 1)) != 0;
}
bool floats_misaligned(const void* a, const void* b, const void* c) {
  return ((reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b) | reinterpret_cast<uintptr_t>(c)) & 3) != 0;
}

}  // namespace

}  // namespace hdqt

using namespace hdqt;

extern "C" size_t hdqt_linear_xent_workspace_bytes(const hdqt_xent_desc_t* d, int32_t kind) {
  Plan pl;
  return make_plan(d, kind, &pl) == HDQT_OK ? pl.total : 0;
}

extern "C" hdqt_status_t hdqt_linear_xent_fwd(const hdqt_xent_desc_t* d, const void* X, const void* W,
                                              const int64_t* labels, float* loss, float* lse, void* workspace,
                                              size_t workspace_bytes, int32_t* dev_status, void* stream) {
  Call c;
  hdqt_status_t st = begin(&c, d, HDQT_XENT_FWD, X, W, labels, workspace, workspace_bytes, dev_status, stream);
  if (st != HDQT_OK) return st;
  if ((d->tokens > 0 && !lse) || (!loss && (d->tokens > 0 || d->reduction != HDQT_REDUCE_NONE))) return HDQT_ERR_INVALID_ARG;
  if (floats_misaligned(loss, lse, nullptr)) return HDQT_ERR_ALIGNMENT;
  if (c.pl.small_rows > 0) return small(c, HDQT_XENT_FWD, X, W, labels, nullptr, nullptr, loss, lse, nullptr, nullptr);
  if (c.pl.few_grad > 0) {
    st = few_grad(c, HDQT_XENT_FWD, X, W, labels, nullptr, nullptr, d->reduction == HDQT_REDUCE_NONE ? loss : c.at<float>(c.pl.loss_rows),
                  lse, nullptr, nullptr);
    return st == HDQT_OK ? reduce_loss(c, loss) : st;
  }
  if (c.pl.few_tokens > 0) return few(c, X, W, labels, loss, lse);
  st = prepare(&c, X, W, labels, nullptr);
  if (st != HDQT_OK) return st;
  float* rows = d->reduction == HDQT_REDUCE_NONE ? loss : c.at<float>(c.pl.loss_rows);
  if (d->tokens > 0 && c.pl.splits_z > 1) {
    st = split_logits(c, HDQT_XENT_FWD, nullptr, rows, lse);
    return st == HDQT_OK ? reduce_loss(c, loss) : st;
  }
  for (int64_t t0 = 0; t0 < d->tokens; t0 += c.pl.rows_piece) {
    const int64_t nt = d->tokens - t0 < c.pl.rows_piece ? d->tokens - t0 : c.pl.rows_piece;
    const Product g = logits_product(c, t0, nt, 0, d->classes);
    XParams p;
    fill_common(c, &p);
    p.pr[0] = make_problem(g, 1);
    p.label = c.at<int32_t>(c.pl.label) + t0;
    p.part = c.at<float2>(c.pl.part);
    p.parts_ld = c.pl.parts_ld;
    p.label_logit = c.at<float>(c.pl.label_logit) + t0;
    st = launch<X_STATS>(p, &g, 1, c);
    if (st != HDQT_OK) return st;
    c.run(xent_rows_kernel, (unsigned)ceil_div(nt, kRowThreads / 32), kRowThreads, 0, p.part, (int)p.parts_ld, p.parts_ld, p.label, p.label_logit, nt, lse + t0, rows + t0);
  }
  return reduce_loss(c, loss);
}

extern "C" hdqt_status_t hdqt_linear_xent_bwd(const hdqt_xent_desc_t* d, const void* X, const void* W,
                                              const int64_t* labels, const float* lse, const float* gr, void* dX, void* dW,
                                              void* workspace, size_t workspace_bytes, int32_t* dev_status, void* stream) {
  Call c;
  hdqt_status_t st = begin(&c, d, HDQT_XENT_BWD, X, W, labels, workspace, workspace_bytes, dev_status, stream);
  if (st != HDQT_OK) return st;
  if (d->tokens > 0 && (!lse || (d->reduction == HDQT_REDUCE_NONE && !gr))) return HDQT_ERR_INVALID_ARG;
  if (floats_misaligned(lse, gr, nullptr) || outputs_misaligned(d, dX, dW)) return HDQT_ERR_ALIGNMENT;
  if (!dX && !dW) return HDQT_OK;
  if (d->tokens == 0) return dW ? zero_out(c, dW, c.pl.w_rows, c.pl.w_cols, d->ld_dw) : HDQT_OK;
  if (c.pl.small_rows > 0) return small(c, HDQT_XENT_BWD, X, W, labels, lse, gr, nullptr, nullptr, dX, dW);
  if (c.pl.few_grad > 0) return few_grad(c, HDQT_XENT_BWD, X, W, labels, lse, gr, nullptr, nullptr, dX, dW);
  st = prepare(&c, X, W, labels, gr);
  if (st != HDQT_OK) return st;
  if (c.pl.splits_z > 1) {
    st = split_logits(c, HDQT_XENT_BWD, lse, nullptr, nullptr);
    return st == HDQT_OK ? gradient_products(c, 0, d->tokens, 0, d->classes, dX, dW, true, true) : st;
  }
  for (int64_t v0 = 0; v0 < d->classes; v0 += c.pl.cols_piece) {
    const int64_t nv = d->classes - v0 < c.pl.cols_piece ? d->classes - v0 : c.pl.cols_piece;
    const Product g = logits_product(c, 0, d->tokens, v0, nv);
    XParams p;
    fill_common(c, &p);
    p.pr[0] = make_problem(g, 1);
    p.label = c.at<int32_t>(c.pl.label);
    p.n0 = (int32_t)v0;
    p.z = c.at<void>(c.pl.dz);
    p.ld_z = c.pl.ld_z;
    p.plane_z = c.pl.rows_piece * c.pl.ld_z;
    p.lse = lse;
    p.g = c.row_weights;
    st = launch<X_DZ>(p, &g, 1, c);
    if (st != HDQT_OK) return st;
    st = gradient_products(c, 0, d->tokens, v0, nv, dX, dW, v0 == 0, v0 + nv == d->classes);
    if (st != HDQT_OK) return st;
  }
  return HDQT_OK;
}

extern "C" hdqt_status_t hdqt_linear_xent_train(const hdqt_xent_desc_t* d, const void* X, const void* W,
                                                const int64_t* labels, const float* gr, float* loss, float* lse, void* dX,
                                                void* dW, void* workspace, size_t workspace_bytes, int32_t* dev_status,
                                                void* stream) {
  Call c;
  hdqt_status_t st = begin(&c, d, HDQT_XENT_TRAIN, X, W, labels, workspace, workspace_bytes, dev_status, stream);
  if (st != HDQT_OK) return st;
  if ((d->tokens > 0 && !lse) || (!loss && (d->tokens > 0 || d->reduction != HDQT_REDUCE_NONE))) return HDQT_ERR_INVALID_ARG;
  if (d->tokens > 0 && d->reduction == HDQT_REDUCE_NONE && !gr) return HDQT_ERR_INVALID_ARG;
  if (floats_misaligned(loss, lse, gr) || outputs_misaligned(d, dX, dW)) return HDQT_ERR_ALIGNMENT;
  if (c.pl.small_rows > 0) return small(c, HDQT_XENT_TRAIN, X, W, labels, nullptr, gr, loss, lse, dX, dW);
  if (c.pl.few_grad > 0) {
    st = few_grad(c, HDQT_XENT_TRAIN, X, W, labels, nullptr, gr, d->reduction == HDQT_REDUCE_NONE ? loss : c.at<float>(c.pl.loss_rows),
                  lse, dX, dW);
    return st == HDQT_OK ? reduce_loss(c, loss) : st;
  }
  st = prepare(&c, X, W, labels, gr);
  if (st != HDQT_OK) return st;
  if (d->tokens == 0) {
    if (dW) st = zero_out(c, dW, c.pl.w_rows, c.pl.w_cols, d->ld_dw);
    return st == HDQT_OK ? reduce_loss(c, loss) : st;
  }
  float* rows = d->reduction == HDQT_REDUCE_NONE ? loss : c.at<float>(c.pl.loss_rows);
  if (c.pl.splits_z > 1) {
    st = split_logits(c, HDQT_XENT_TRAIN, nullptr, rows, lse);
    if (st == HDQT_OK) st = gradient_products(c, 0, d->tokens, 0, d->classes, dX, dW, true, true);
    return st == HDQT_OK ? reduce_loss(c, loss) : st;
  }
  for (int64_t t0 = 0; t0 < d->tokens; t0 += c.pl.rows_piece) {
    const int64_t nt = d->tokens - t0 < c.pl.rows_piece ? d->tokens - t0 : c.pl.rows_piece;
    const Product g = logits_product(c, t0, nt, 0, d->classes);
    XParams p;
    fill_common(c, &p);
    p.pr[0] = make_problem(g, 1);
    p.label = c.at<int32_t>(c.pl.label) + t0;
    p.part = c.at<float2>(c.pl.part);
    p.parts_ld = c.pl.parts_ld;
    p.label_logit = c.at<float>(c.pl.label_logit) + t0;
    p.z = c.at<void>(c.pl.z);
    p.ld_z = c.pl.ld_z;
    st = c.pl.planes == 1 ? launch<X_CODES>(p, &g, 1, c) : launch<X_LOGITS>(p, &g, 1, c);
    if (st != HDQT_OK) return st;
    // few rows: slices of the classes fill the machine
    int64_t slices = ceil_div(4 * kNumSMsHint, nt);
    const int64_t most = ceil_div(d->classes, 8 * kRowThreads);
    const dim3 grid((unsigned)nt, (unsigned)(slices < most ? slices : most));
    if (c.pl.planes == 1)
      c.run(xent_dz_kernel<1>, grid, kRowThreads, 0, p.part, (int)p.parts_ld, p.parts_ld, p.label, p.label_logit,
                                                               c.row_weights ? c.row_weights + t0 : nullptr, d->classes, p.z, c.pl.ld_z,
            static_cast<uint16_t*>(nullptr), 0, lse + t0, rows + t0);
    else
      c.run(xent_dz_kernel<3>, grid, kRowThreads, 0, p.part, (int)p.parts_ld, p.parts_ld, p.label, p.label_logit,
                                                               c.row_weights ? c.row_weights + t0 : nullptr, d->classes, p.z, c.pl.ld_z,
                                                               c.at<uint16_t>(c.pl.dz), c.pl.rows_piece * c.pl.ld_z,
                                                               lse + t0, rows + t0);
    st = gradient_products(c, t0, nt, 0, d->classes, dX, dW, t0 == 0, t0 + nt == d->tokens);
    if (st != HDQT_OK) return st;
  }
  return reduce_loss(c, loss);
}
