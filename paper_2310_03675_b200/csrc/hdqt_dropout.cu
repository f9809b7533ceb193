// Dropout, added to a residual: y = residual + (u >= T ? x scale : 0), u 16 bits of Philox4x32-10 per element.
//
// One Philox call serves eight consecutive elements (of the flattened tensor), which is one 16-byte access of a 16-bit type and two
// of fp32.  Bound by HBM: x and residual read once, y written once.  32768 x 4096 bf16: 81 us (6.6 TB/s, what a copy reaches), with a
// residual 116 us (6.9); 14 instructions per element, six of them the generator's, fill 65 % of the issue slots.
#include "hdqt_dropout.cuh"

namespace hdqt {

namespace {

constexpr int NT = 256;

struct DropCall {
  DropParams d;
  const void* x;
  const void* residual;
  void* y;
  int64_t n, rows, cols;     // elements, and their division into rows
  int64_t x_rs, r_rs, y_rs;
};

// kGroups times eight elements per thread, 16-byte accesses, all loads ahead of the generator.  kLinear: dense tensors (one row of n
// elements); otherwise cols % 8 == 0.
template <typename T, bool kLinear, bool kResidual, int kGroups>
__global__ void __launch_bounds__(NT) dropout_vec_kernel(const DropCall p) {
  constexpr int V = 16 / sizeof(T), K = 8 / V;
  const uint32_t offset = drop_offset(p.d);
  uint64_t g[kGroups];
  int64_t yi[kGroups];
  Words vx[kGroups][K], vr[kGroups][K];
#pragma unroll
  for (int u = 0; u < kGroups; ++u) {
    g[u] = ((uint64_t)blockIdx.x * kGroups + u) * NT + threadIdx.x;
    const int64_t first = (int64_t)g[u] * 8;
    int64_t xi = first, ri = first;
    yi[u] = first;
    if constexpr (!kLinear) {
      const int64_t r = first / p.cols, c = first - r * p.cols;
      xi = r * p.x_rs + c;
      ri = r * p.r_rs + c;
      yi[u] = r * p.y_rs + c;
    }
    if (first + 8 <= p.n) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        vx[u][k] = *reinterpret_cast<const Words*>(reinterpret_cast<const T*>(p.x) + xi + k * V);
        if (kResidual) vr[u][k] = *reinterpret_cast<const Words*>(reinterpret_cast<const T*>(p.residual) + ri + k * V);
      }
    }
  }
  Philox4 words[kGroups];
  drop_words(p.d, offset, g, words);
  const uint32_t limit = p.d.limit;
  const bool all = !p.d.on;      // nothing is dropped
#pragma unroll
  for (int u = 0; u < kGroups; ++u) {
    const int64_t first = (int64_t)g[u] * 8;
    if (first >= p.n) return;
    const Philox4& w = words[u];
    T* y = reinterpret_cast<T*>(p.y) + yi[u];
    if (first + 8 <= p.n) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        float f[V], q[V];
        unpack<T>(vx[u][k], f);
        if (kResidual) unpack<T>(vr[u][k], q);
#pragma unroll
        for (int j = 0; j < V; j += 2) {
          mul2(f[j], f[j + 1], p.d.scale, p.d.scale);
          f[j] = drop_keeps(w, k * V + j, limit) || all ? f[j] : 0.0f;
          f[j + 1] = drop_keeps(w, k * V + j + 1, limit) || all ? f[j + 1] : 0.0f;
          if (kResidual) add2(f[j], f[j + 1], q[j], q[j + 1]);
        }
        *reinterpret_cast<Words*>(y + k * V) = pack_words<T>(f);
      }
    } else {      // the last elements of a dense tensor
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (first + j >= p.n) break;
        float f = to_f32(reinterpret_cast<const T*>(p.x)[first + j]);
        f = drop_keeps(w, j, limit) || all ? __fmul_rn(f, p.d.scale) : 0.0f;
        if (kResidual) f = __fadd_rn(to_f32(reinterpret_cast<const T*>(p.residual)[first + j]), f);
        y[j] = from_f32<T>(f);
      }
    }
  }
}

// any strides and addresses: a thread takes the same eight elements one by one
template <typename T>
__global__ void __launch_bounds__(NT) dropout_any_kernel(const DropCall p) {
  const int64_t g = (int64_t)blockIdx.x * NT + threadIdx.x, first = g * 8;
  if (first >= p.n) return;
  uint32_t bits = 0xFFu;
  if (p.d.on) bits = drop_bits(p.d, drop_offset(p.d), (uint64_t)g);
  int64_t r = first / p.cols, c = first - r * p.cols;
  const int m = (int)min((int64_t)8, p.n - first);
  for (int j = 0; j < m; ++j) {
    float f = to_f32(reinterpret_cast<const T*>(p.x)[r * p.x_rs + c]);
    if (p.d.on) f = (bits >> j) & 1 ? __fmul_rn(f, p.d.scale) : 0.0f;
    if (p.residual) f = __fadd_rn(to_f32(reinterpret_cast<const T*>(p.residual)[r * p.r_rs + c]), f);
    reinterpret_cast<T*>(p.y)[r * p.y_rs + c] = from_f32<T>(f);
    if (++c == p.cols) { c = 0; ++r; }
  }
}

template <typename T, bool kLinear>
void launch_vec(const DropCall& p, cudaStream_t s) {
  constexpr int kGroups = sizeof(T) == 2 ? 2 : 1;      // 32 bytes of every tensor per thread
  const unsigned blocks = (unsigned)(((p.n + 7) / 8 + kGroups * NT - 1) / (kGroups * NT));
  if (p.residual) dropout_vec_kernel<T, kLinear, true, kGroups><<<blocks, NT, 0, s>>>(p);
  else dropout_vec_kernel<T, kLinear, false, kGroups><<<blocks, NT, 0, s>>>(p);
}
template <typename T>
void launch_dropout(const DropCall& p, bool linear, bool wide, cudaStream_t s) {
  if (wide && linear) launch_vec<T, true>(p, s);
  else if (wide) launch_vec<T, false>(p, s);
  else dropout_any_kernel<T><<<(unsigned)(((p.n + 7) / 8 + NT - 1) / NT), NT, 0, s>>>(p);
}

}  // namespace

}  // namespace hdqt

using namespace hdqt;

extern "C" hdqt_status_t hdqt_dropout_add(const hdqt_dropout_desc_t* d, const void* x, const void* residual, void* y, void* stream) {
  if (!d || d->rows < 0 || d->cols < 0 || !valid_probability(d->p)) return HDQT_ERR_INVALID_ARG;
  const int elem = dtype_size(d->dtype);
  if (elem == 0) return HDQT_ERR_INVALID_ARG;
  if (d->rows == 0 || d->cols == 0) return HDQT_OK;
  if (!x || !y) return HDQT_ERR_INVALID_ARG;
  if (d->rows > 1 && (d->x_row_stride < d->cols || d->y_row_stride < d->cols || (residual && d->r_row_stride < d->cols)))
    return HDQT_ERR_INVALID_ARG;
  if (d->rows > (1ll << 40) / d->cols) return HDQT_ERR_UNSUPPORTED;
  const uintptr_t bases = reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(residual) | reinterpret_cast<uintptr_t>(y);
  if ((bases & (uintptr_t)(elem - 1)) || (reinterpret_cast<uintptr_t>(d->philox_offset) & 3)) return HDQT_ERR_ALIGNMENT;
  DropCall p{};
  p.d = make_drop(d->p, d->seed, d->tag, d->philox_offset);
  p.x = x;
  p.residual = residual;
  p.y = y;
  p.rows = d->rows;
  p.cols = d->cols;
  p.n = d->rows * d->cols;
  p.x_rs = d->x_row_stride;
  p.r_rs = residual ? d->r_row_stride : d->cols;
  p.y_rs = d->y_row_stride;
  const bool linear = d->rows == 1 || (p.x_rs == d->cols && p.r_rs == d->cols && p.y_rs == d->cols);
  const bool wide = (bases & 15) == 0 && (linear || (d->cols % 8 == 0 && ((p.x_rs | p.r_rs | p.y_rs) * elem & 15) == 0));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (d->dtype == HDQT_DTYPE_F32) launch_dropout<float>(p, linear, wide, s);
  else if (d->dtype == HDQT_DTYPE_BF16) launch_dropout<__nv_bfloat16>(p, linear, wide, s);
  else launch_dropout<__half>(p, linear, wide, s);
  return last_error("dropout");
}
