// Matrix products of the linear cross entropy on CTA pairs (tcgen05 cta_group::2, bf16 operands, fp32 accumulators).
//
//   out[m, n] = sum over plane pairs (i, j) and k of A_i[m, k] B_j[n, k]
//
// bf16 operands have one plane.  An fp32 operand is held as three bf16 planes x = x0 + x1 + x2 (8 significant bits each,
// 24 together); of the nine products the six above 2^-24 are summed, smallest first, so that an fp32 product costs six
// bf16 products on the tensor cores and keeps fp32 precision.
//
// Each operand may be stored with its contraction index contiguous ("K-major") or with its row index contiguous
// ("MN-major"): the logits, dX and dW products read X, W and dZ where they lie, no operand is ever transposed in memory.
//
// Cluster of two CTAs = one 256 x 256 output block: CTA rank r loads rows [128 r, 128 r + 128) of the A block and of the B
// block (32 KB per stage of 64 k), the leader issues M = 256 MMAs, each CTA's TMEM receives its 128 rows.  Two accumulators of 256
// columns alternate, so a block's epilogue overlaps the next block's main loop.
// Warps: 0 = TMA producer, 1 = MMA issuer (leader only), 2..9 = epilogue (lane quarter x 128 columns).
//
// The tensor core adds into its fp32 accumulator without rounding to nearest, an error that grows with the number of
// additions: a contraction is cut into parts of at most `part_iters` stages, whose sums the epilogue adds up in
// registers with ordinary fp32 additions.
//
// One bf16 operand may come as two planes (X times the rows' weights, 16 significant bits): its product then takes two passes.
//
// Bound by the tensor pipe.  4096 x 2048 x 32000 bf16: logits with codes 351 us (1.53 PFLOP/s, pipe 86 % active), dX and dW in
// one launch 693 us (1.55, 89 %).  2048 x 1024 x 32768 fp32, six products: logits 532 us (1.55, 86 %), dX and dW 1138 us (1.45,
// 85 %).
#pragma once

#include "hdqt_ptx.cuh"
#include "hdqt_types.cuh"

namespace hdqt {

namespace {

constexpr int XM = 256, XN = 256, XK = 64;          // output block and k per stage (128 bytes of bf16)
constexpr int X_STAGES = 6;
constexpr int X_OPERAND = 128 * 128;                // one operand's bytes per stage and CTA
constexpr int X_STAGE_BYTES = 2 * X_OPERAND;
constexpr int X_EPI_WARPS = 8;
constexpr int X_THREADS = 32 * (2 + X_EPI_WARPS);
constexpr int X_BOX = 32 * 33 * 4;                  // per epilogue warp: 32 rows x 32 columns fp32 for the store transpose
constexpr int X_BOX_OFF = X_STAGES * X_STAGE_BYTES + 256;
constexpr int X_SMEM = X_BOX_OFF + X_EPI_WARPS * X_BOX;
constexpr int X_TMEM_COLS = 512;
static_assert(X_SMEM <= 232448, "exceeds the 227 KB of shared memory a CTA may use");

constexpr float kLowest = -3.402823466e38f;
// Softmax codes: 16 bits of log2(max / value) with 2^-11 resolution.  The rounding is at most 2^-12 in log2, 1.7e-4
// relative, a twelfth of the bf16 rounding that follows.  A value below 2^-32 of the largest of its 128 columns is held as 0:
// a vocabulary of a million such values would together be 2^-12 of that one.
constexpr float kCodeScale = 2048.0f;
constexpr uint32_t kCodeZero = 65535u;

enum XEpilogue {
  X_STATS = 0,    // per row and 128 columns: (max, sum of exp(z - max)); the label's logit
  X_CODES = 1,    // X_STATS, and 16-bit softmax codes of the block
  X_LOGITS = 2,   // X_STATS, and the logits in fp32
  X_DZ = 3,       // dz = g (exp(z - lse) - [n = label]) in 1 or 3 bf16 planes
  X_OUT = 4       // plain output, bf16 or fp32, optionally added to earlier fp32 sums
};

struct XProblem {
  int32_t M, N;
  int32_t tiles_m, tiles_n, group_m;
  int32_t kblocks;                 // stages of 64 per plane pair
  int32_t splits, kblocks_split;   // work items per block along the contraction; kblocks each
  int32_t a_mn, b_mn;              // MN-major operand
  int32_t items;                   // tiles_m * tiles_n * splits
  // X_OUT
  void* out;
  int64_t ld_out;
  int64_t split_stride;            // elements between the partial outputs of two splits
  const float* add;                // fp32 sums of earlier pieces (may be out itself)
  int64_t ld_add;
  const float* row_scale;          // [M]: the output row is this times the product (null: XParams::alpha)
  int32_t out_bf16;
  int32_t products;                // plane pairs: 1, 6 (fp32) or 2 (one bf16 operand in two planes)
  int32_t two;                     // which one: 1 = A, 2 = B
};

struct XParams {
  XProblem pr[2];
  int32_t num_problems;
  int32_t extra;                   // see x_item
  int32_t planes;                  // 1 or 3
  int32_t part_iters;
  // statistics and dz epilogues
  const int32_t* label;            // [M]; < 0: no label (ignored)
  int32_t n0;                      // first column of this piece in the whole vocabulary
  float2* part;                    // [M, parts_ld]
  int64_t parts_ld;
  float* label_logit;              // [M]
  void* z;                         // codes (uint16), logits (fp32) or dz (bf16 planes)
  int64_t ld_z, plane_z;           // elements
  const float* lse;                // [M]
  const float* g;                  // weight of each row's loss, [M]; null: 1
  const float* alpha;              // X_OUT: the output is this times the product; null: 1
  int32_t* dev_status;
};

__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, int32_t z,
                                                 uint32_t bar_local) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar_local & kPeerBitMask)
      : "memory");
}

// Descriptors as their two words: along a contraction only the address field of the low word moves.
__device__ __forceinline__ void tc_mma_bf16_pair(uint32_t d_tmem, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi,
                                                 uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
      "mov.b64 a, {%1, %2};\n\t"
      "mov.b64 b, {%3, %4};\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %5, p;\n\t}"
      ::"r"(d_tmem), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
      : "memory");
}

// MN-major operand tile with 128-byte swizzle: 64 rows (MN) x 8 k form one 1024-byte atom; `lbo` = distance to the next
// 64 rows, `sbo` = distance to the next 8 k.
__device__ __forceinline__ uint64_t make_smem_desc_mn(uint32_t addr, uint32_t lbo, uint32_t sbo) {
  uint64_t d = 0;
  d |= (uint64_t)((addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(lbo >> 4) << 16;
  d |= (uint64_t)(sbo >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

// Arrival at the pair leader's barrier for an accumulator that has been read (tcgen05.wait::ld and the fence before it order
// that).  Not the cluster-scope release of mbar_arrive_cluster: it would also wait for every output store in flight, which
// made each 256 x 256 block's epilogue 4.7 us long.
__device__ __forceinline__ void mbar_arrive_read(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}

// 32 bytes in one access (the address is 32-byte aligned)
__device__ __forceinline__ void st256(void* p, const uint32_t (&v)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]),
               "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// x = p0 + p1 + p2 in bf16, each the rounding of what the ones before leave.  fp32 values above the largest bf16 value (a mask of
// the lowest fp32 value) would round to infinity and leave NaN: p0 stops at that value, and the other two still hold the rest.
constexpr float kBf16Max = 3.38953139e38f;      // 2^128 - 2^120
__device__ __forceinline__ void split3(float x, float& p0, float& p1, float& p2) {
  p0 = __bfloat162float(__float2bfloat16_rn(fminf(fmaxf(x, -kBf16Max), kBf16Max)));
  p1 = __bfloat162float(__float2bfloat16_rn(x - p0));
  p2 = x - p0 - p1;
}

// planes of the s-th product, smallest first; of an fp32 contraction (0,2) (2,0) (1,1) (0,1) (1,0) (0,0)
__device__ __forceinline__ void plane_pair(int planes, int two, int s, int& a, int& b) {
  a = planes > 1 ? (int)((0x118u >> (2 * s)) & 3u) : two == 1 ? 1 - s : 0;
  b = planes > 1 ? (int)((0x052u >> (2 * s)) & 3u) : two == 2 ? 1 - s : 0;
}

struct XItem {
  int m, n, split, kb0, nkb;     // block coordinates, split, first stage and stages per plane pair
  int q;                         // problem
};

// k-th work item of this pair, or false.  Items of problem 0 (the longer ones) go round the pairs first; the pairs that get one
// fewer of them take `extra` items of problem 1 in its place, and the rest go round all pairs.
__device__ __forceinline__ bool x_item(const XParams& p, int pair, int pairs, int k, XItem& t) {
  const int n0 = p.pr[0].items;
  const int whole = n0 / pairs, more = n0 - whole * pairs;       // pairs below `more` have one item more
  const int mine = whole + (pair < more ? 1 : 0);
  int i;
  if (k < mine) {
    t.q = 0;
    i = pair + k * pairs;
  } else {
    if (p.num_problems < 2) return false;
    t.q = 1;
    k -= mine;
    const int low = pairs - more, given = p.extra * low;
    if (pair >= more && k < p.extra) i = k * low + (pair - more);
    else i = given + (k - (pair >= more ? p.extra : 0)) * pairs + (pair >= more ? pair - more : low + pair);
    if (i >= p.pr[1].items) return false;
  }
  const XProblem& r = p.pr[t.q];
  const int blocks = r.tiles_m * r.tiles_n;
  t.split = i / blocks;
  i -= t.split * blocks;
  const int per_group = r.group_m * r.tiles_n;
  const int grp = i / per_group;
  const int first = grp * r.group_m;
  const int rows = min(r.group_m, r.tiles_m - first);
  i -= grp * per_group;
  t.m = first + i % rows;
  t.n = i / rows;
  t.kb0 = t.split * r.kblocks_split;
  t.nkb = min(r.kblocks_split, r.kblocks - t.kb0);
  return true;
}

// ---- epilogues: one thread holds 128 consecutive columns of one row ----------------------------------------

template <int kEpi>
__device__ __forceinline__ void x_stats(const XParams& p, const XProblem& r, const XItem& t, int row, int col0, int half,
                                        float (&acc)[128]) {
  const int ncols = r.N - col0;                     // columns that exist (may be <= 0)
  if (row >= r.M) return;
  float m = kLowest;
  if (ncols >= 128) {
#pragma unroll
    for (int j = 0; j < 128; ++j) m = fmaxf(m, acc[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 128; ++j) {
      if (j < ncols) m = fmaxf(m, acc[j]);
      else acc[j] = -INFINITY;
    }
  }
  const int lab = __ldg(p.label + row) - p.n0 - col0;
  if (lab >= 0 && lab < 128) {
    float zl = 0.0f;
#pragma unroll
    for (int j = 0; j < 128; ++j) zl = (j == lab) ? acc[j] : zl;
    p.label_logit[row] = zl;
  }
  if (kEpi == X_LOGITS) {
    float* dst = reinterpret_cast<float*>(p.z) + (int64_t)row * p.ld_z + col0;
#pragma unroll
    for (int j = 0; j < 128; j += 8) {
      if (j >= ncols) break;
      uint32_t v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = __float_as_uint(acc[j + k]);
      st256(dst + j, v);
    }
  }
  float s = 0.0f;
#pragma unroll
  for (int j = 0; j < 128; ++j) {
    const float d = m - acc[j];
    s += ex2(d * -kLog2e);
    acc[j] = d;
  }
  p.part[(int64_t)row * p.parts_ld + 2 * t.n + half] = make_float2(m, s);
  if (kEpi == X_CODES) {
    uint16_t* dst = reinterpret_cast<uint16_t*>(p.z) + (int64_t)row * p.ld_z + col0;
#pragma unroll
    for (int j = 0; j < 128; j += 16) {
      if (j >= ncols) break;
      uint32_t v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        // 2^23 + code: the code is the low half of the sum's bits
        const float lo = fminf(fmaf(acc[j + 2 * k], kCodeScale * kLog2e, 8388608.0f), 8388608.0f + 65535.0f);
        const float hi = fminf(fmaf(acc[j + 2 * k + 1], kCodeScale * kLog2e, 8388608.0f), 8388608.0f + 65535.0f);
        v[k] = __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x5410);
      }
      st256(dst + j, v);
    }
  }
}

// dz is an operand of the gradient products: bf16 beside bf16 X and W, rounded once (2^-8 at most), or three planes.  A second plane
// for what the rounding leaves would double both products (693 us at 4096 x 2048 x 32000).  A weight that all rows share is not in
// dz but multiplies the fp32 sums (XParams::alpha); a row's largest value, p - 1 at its label, is then close to a bf16 number, and the
// gradients are as exact as fp32 arithmetic rounded at the end (error against 64 bits 1.7e-3 both, at that size).  Of weights
// per row the largest is treated like that and the rest, g / largest, multiplied in before the rounding: equal weights cost
// nothing, random ones give 2.2e-3 against 1.7e-3 at 1531 x 1000 x 50257.  Few tokens, whose roundings do not average, keep them
// out of dz: dX's epilogue multiplies its rows by them, and dW's X is weighted X in two planes (hdqt_xent.cu, kPlaneTokens).
__device__ __forceinline__ void x_dz(const XParams& p, const XProblem& r, int row, int col0, float (&acc)[128]) {
  const int ncols = r.N - col0;
  if (row >= r.M || ncols <= 0) return;
  const int lab_row = __ldg(p.label + row);
  const bool keep = lab_row >= 0;
  const float lse = p.lse[row], g = p.g != nullptr ? p.g[row] : 1.0f;
  const int lab = lab_row - p.n0 - col0;
#pragma unroll
  for (int j = 0; j < 128; ++j) {
    float e = ex2((acc[j] - lse) * kLog2e) - (j == lab ? 1.0f : 0.0f);
    acc[j] = keep ? e * g : 0.0f;
  }
  uint16_t* dst = reinterpret_cast<uint16_t*>(p.z) + (int64_t)row * p.ld_z + col0;
#pragma unroll
  for (int j = 0; j < 128; j += 16) {
    if (j >= ncols) break;
    uint32_t v[8];
    if (p.planes == 1) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = pack_bf16(acc[j + 2 * k], acc[j + 2 * k + 1]);
      st256(dst + j, v);
    } else {
      uint32_t v1[8], v2[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        float a0, a1, a2, b0, b1, b2;
        split3(acc[j + 2 * k], a0, a1, a2);
        split3(acc[j + 2 * k + 1], b0, b1, b2);
        v[k] = pack_bf16(a0, b0);
        v1[k] = pack_bf16(a1, b1);
        v2[k] = pack_bf16(a2, b2);
      }
      st256(dst + j, v);
      st256(dst + p.plane_z + j, v1);
      st256(dst + 2 * p.plane_z + j, v2);
    }
  }
}

__device__ __forceinline__ void x_out(const XParams& p, const XProblem& r, const XItem& t, int row, int col0, float (&acc)[128]) {
  const int ncols = r.N - col0;
  if (row >= r.M || ncols <= 0) return;
  if (p.alpha != nullptr || r.row_scale != nullptr) {
    const float alpha = r.row_scale != nullptr ? r.row_scale[row] : *p.alpha;
#pragma unroll
    for (int j = 0; j < 128; ++j) acc[j] *= alpha;
  }
  const int64_t at = (int64_t)row * r.ld_out + col0 + t.split * r.split_stride;
  if (r.add != nullptr) {
    const float* a = r.add + (int64_t)row * r.ld_add + col0;
    const bool vec = ((reinterpret_cast<uintptr_t>(a) & 15) == 0);
#pragma unroll
    for (int j = 0; j < 128; j += 4) {
      if (vec && j + 4 <= ncols) {
        const float4 v = *reinterpret_cast<const float4*>(a + j);
        acc[j] += v.x; acc[j + 1] += v.y; acc[j + 2] += v.z; acc[j + 3] += v.w;
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (j + k < ncols) acc[j + k] += a[j + k];
      }
    }
  }
  if (r.out_bf16) {
    __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(r.out) + at;
    const bool high = (reinterpret_cast<uintptr_t>(o) & 16) != 0;      // rows of 16 bytes' multiples alternate between 0 and 16
#pragma unroll
    for (int j = 0; j < 128; j += 16) {
      if (j + 16 <= ncols) {
        uint32_t v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = pack_bf16(acc[j + 2 * k], acc[j + 2 * k + 1]);
        if (!high) {
          st256(o + j, v);
        } else {
          *reinterpret_cast<uint4*>(o + j) = make_uint4(v[0], v[1], v[2], v[3]);
          *reinterpret_cast<uint4*>(o + j + 8) = make_uint4(v[4], v[5], v[6], v[7]);
        }
      } else {
#pragma unroll
        for (int k = 0; k < 16; ++k)
          if (j + k < ncols) o[j + k] = __float2bfloat16_rn(acc[j + k]);
      }
    }
  } else {
    float* o = reinterpret_cast<float*>(r.out) + at;
    const bool high = (reinterpret_cast<uintptr_t>(o) & 16) != 0;
#pragma unroll
    for (int j = 0; j < 128; j += 8) {
      if (j + 8 <= ncols) {
        uint32_t v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = __float_as_uint(acc[j + k]);
        if (!high) {
          st256(o + j, v);
        } else {
          *reinterpret_cast<uint4*>(o + j) = make_uint4(v[0], v[1], v[2], v[3]);
          *reinterpret_cast<uint4*>(o + j + 4) = make_uint4(v[4], v[5], v[6], v[7]);
        }
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (j + k < ncols) o[j + k] = acc[j + k];
      }
    }
  }
}

// Output rows that do not all start on 16 bytes: 32 x 32 pieces are turned in shared memory, so that the 32 lanes of a store
// write neighbouring elements of one row (3 x 425 x 21344 bf16 loss and gradients: 96 us, and 201 with a store per element and
// row; loss and gradients of 35 x 2604 x 44400 with rows of 4-byte starts: 262 us, and 504).
__device__ __forceinline__ void x_out_odd(const XParams& p, const XProblem& r, const XItem& t, int row0, int col0, int lane,
                                          float* box, float (&acc)[128]) {
  const int rows = min(32, r.M - row0);
  const float alpha = r.row_scale != nullptr ? (lane < rows ? r.row_scale[row0 + lane] : 0.0f) : p.alpha != nullptr ? *p.alpha : 1.0f;
  if (r.out_bf16 && r.add == nullptr && ((reinterpret_cast<uintptr_t>(r.out) | (uintptr_t)(r.ld_out * 2)) & 3) == 0 && (r.N & 1) == 0) {
    // rows start on 4 bytes: two neighbouring bf16 per lane, 64 columns at a time
    uint32_t* pair = reinterpret_cast<uint32_t*>(box);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int col = col0 + 64 * c;
      if (col >= r.N) break;
      __syncwarp();
#pragma unroll
      for (int k = 0; k < 32; ++k) pair[lane * 33 + k] = pack_bf16(acc[64 * c + 2 * k] * alpha, acc[64 * c + 2 * k + 1] * alpha);
      __syncwarp();
      if (col + 2 * lane < r.N) {
        uint32_t* o = reinterpret_cast<uint32_t*>(reinterpret_cast<__nv_bfloat16*>(r.out) + (int64_t)row0 * r.ld_out + col + 2 * lane);
#pragma unroll 8
        for (int i = 0; i < rows; ++i) o[i * (r.ld_out >> 1)] = pair[i * 33 + lane];
      }
    }
    return;
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int col = col0 + 32 * c;
    if (col >= r.N) break;
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 32; ++k) box[lane * 33 + k] = acc[32 * c + k] * alpha;
    __syncwarp();
    if (col + lane < r.N) {
      const int64_t at = (int64_t)row0 * r.ld_out + col + lane + t.split * r.split_stride;
      const float* a = r.add != nullptr ? r.add + (int64_t)row0 * r.ld_add + col + lane : nullptr;
#pragma unroll 8
      for (int i = 0; i < rows; ++i) {
        float v = box[i * 33 + lane];
        if (a != nullptr) v += a[i * r.ld_add];
        if (r.out_bf16) reinterpret_cast<__nv_bfloat16*>(r.out)[at + i * r.ld_out] = __float2bfloat16_rn(v);
        else reinterpret_cast<float*>(r.out)[at + i * r.ld_out] = v;
      }
    }
  }
}

// whether every row of the output starts on 16 bytes
__device__ __forceinline__ bool x_out_even(const XProblem& r) {
  const int size = r.out_bf16 ? 2 : 4;
  return ((reinterpret_cast<uintptr_t>(r.out) | (uintptr_t)(r.ld_out * size) | (uintptr_t)(r.split_stride * size)) & 15) == 0;
}

// Tensor maps: K-major operand {k, rows, planes} with box {64, 128, 1}; MN-major {rows, k, planes} with box {64, 64, 1}
// (two boxes per stage).  Everything outside an operand reads as zero.
// Stages of the next part of an item with `left` stages to go, nkb a product.  The five smaller products of fp32 operands come first
// and are at most 2^-8 of the last one: 1024 of their stages lose less than half of what 8 of its stages do.  So they form one part,
// during which the item before has its epilogue (2048 x 1024 x 32768 fp32, loss and gradients: 1970 us, 2100 all in parts of 8).
constexpr int kHeadStages = 1024;
__device__ __forceinline__ int x_part(const XParams& p, int left, int nkb) {
  return p.planes > 1 && left > nkb ? min(left - nkb, kHeadStages) : min(left, p.part_iters);
}

template <int kEpi>
__global__ void __launch_bounds__(X_THREADS, 1) __cluster_dims__(2, 1, 1)
xent_gemm_kernel(const __grid_constant__ CUtensorMap map_a0, const __grid_constant__ CUtensorMap map_b0,
                 const __grid_constant__ CUtensorMap map_a1, const __grid_constant__ CUtensorMap map_b1,
                 const __grid_constant__ XParams p) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t smem_base = smem_u32(smem_raw);
  if (smem_base & 1023u) {   // (same outcome in both CTAs of a pair)
    if (threadIdx.x == 0) report_status(p.dev_status, HDQT_ERR_CUDA);
    return;
  }
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem_raw + X_STAGES * X_STAGE_BYTES);
  const uint32_t bar_full = smem_u32(bars);              // [X_STAGES] both CTAs' TMA -> leader's MMA issuer
  const uint32_t bar_empty = bar_full + 8 * X_STAGES;    // [X_STAGES] leader's MMA -> both producers
  const uint32_t bar_tfull = bar_empty + 8 * X_STAGES;   // [2] leader's MMA -> both CTAs' epilogue
  const uint32_t bar_tempty = bar_tfull + 16;            // [2] both CTAs' epilogue -> leader's MMA issuer
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * X_STAGES + 4);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t cta_rank = cluster_ctarank();
  const bool leader = (cta_rank == 0);
  const int pair_id = blockIdx.x >> 1, num_pairs = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < X_STAGES; ++s) {
      mbar_init(bar_full + 8 * s, 1);
      mbar_init(bar_empty + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(bar_tfull + 8 * b, 1);
      mbar_init(bar_tempty + 8 * b, 2 * X_EPI_WARPS);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                 "r"(X_TMEM_COLS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();     // the peer's barriers are initialised before anything is signalled across the pair
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  chain_wait();           // everything above overlaps the kernel before

  if (warp == 0) {
    // ------------------------------ TMA producer (both CTAs) ------------------
    if (lane == 0) {
      uint32_t it = 0;                // stages issued so far (for the drain after a timeout)
      uint32_t ps = 0, pe_par = 1u;   // stage slot and the parity its "empty" barrier is waited on with
      bool ok = true;
      XItem t;
      for (int i = 0; ok && x_item(p, pair_id, num_pairs, i, t); ++i) {
        const XProblem& r = p.pr[t.q];
        const CUtensorMap* ma = t.q ? &map_a1 : &map_a0;
        const CUtensorMap* mb = t.q ? &map_b1 : &map_b0;
        const int a0 = t.m * XM + (int)cta_rank * 128, b0 = t.n * XN + (int)cta_rank * 128;
        for (int s = 0; s < r.products && ok; ++s) {
          int pa, pb;
          plane_pair(p.planes, r.two, s, pa, pb);
          for (int kb = t.kb0; kb < t.kb0 + t.nkb; ++kb, ++it) {
            if (!mbar_try_wait(bar_empty + 8 * ps, pe_par) && !mbar_wait(bar_empty + 8 * ps, pe_par, abort_flag)) { ok = false; break; }
            if (leader) mbar_expect_tx(bar_full + 8 * ps, 2 * X_STAGE_BYTES);   // collects both CTAs' bytes
            const uint32_t dst = smem_base + ps * X_STAGE_BYTES;
            const uint32_t bar = bar_full + 8 * ps;
            if (r.a_mn) {
              tma_load_3d_pair(dst, ma, a0, kb * XK, pa, bar);
              tma_load_3d_pair(dst + X_OPERAND / 2, ma, a0 + 64, kb * XK, pa, bar);
            } else {
              tma_load_3d_pair(dst, ma, kb * XK, a0, pa, bar);
            }
            if (r.b_mn) {
              tma_load_3d_pair(dst + X_OPERAND, mb, b0, kb * XK, pb, bar);
              tma_load_3d_pair(dst + X_OPERAND + X_OPERAND / 2, mb, b0 + 64, kb * XK, pb, bar);
            } else {
              tma_load_3d_pair(dst + X_OPERAND, mb, kb * XK, b0, pb, bar);
            }
            if (++ps == X_STAGES) { ps = 0; pe_par ^= 1u; }
          }
        }
      }
      if (*abort_flag && leader) {
        for (uint32_t k = (it > X_STAGES ? it - X_STAGES : 0u); k < it; ++k) {
          const uint32_t bar = bar_full + 8 * (k % X_STAGES);
          for (int j = 0; j < (1 << 16) && !mbar_try_wait(bar, (k / X_STAGES) & 1u); ++j) __nanosleep(256);
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------------ MMA issuer (leader only) ------------------
    if (lane == 0 && leader) {
      // The tensor pipe takes one MMA while it works on another, so what this thread does between two MMAs must fit into
      // one MMA's time: low words of the descriptors by one addition each, one turn of the stage ring unrolled.
      uint32_t s = 0, full_par = 0u;
      int buf_i = 0;             // accumulators filled so far
      bool ok = true;
      XItem t;
      for (int i = 0; ok && x_item(p, pair_id, num_pairs, i, t); ++i) {
        const XProblem& r = p.pr[t.q];
        // instruction descriptor: D = f32, A = B = bf16, majors, N = 256, M = 256
        const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)r.a_mn << 15) | ((uint32_t)r.b_mn << 16) |
                               ((uint32_t)(XN >> 3) << 17) | ((uint32_t)(XM >> 4) << 24);
        const uint64_t da = r.a_mn ? make_smem_desc_mn(smem_base, X_OPERAND / 2, 1024) : make_smem_desc(smem_base);
        const uint64_t db = r.b_mn ? make_smem_desc_mn(smem_base + X_OPERAND, X_OPERAND / 2, 1024)
                                   : make_smem_desc(smem_base + X_OPERAND);
        const uint32_t ah = (uint32_t)(da >> 32), bh = (uint32_t)(db >> 32);
        const uint32_t ka = r.a_mn ? 2048 >> 4 : 32 >> 4, kb = r.b_mn ? 2048 >> 4 : 32 >> 4;   // per 16 k
        const uint32_t a0 = (uint32_t)da, a1 = a0 + ka, a2 = a1 + ka, a3 = a2 + ka;
        const uint32_t b0 = (uint32_t)db, b1 = b0 + kb, b2 = b1 + kb, b3 = b2 + kb;
        int left = t.nkb * r.products;
        while (left > 0 && ok) {
          const int n = x_part(p, left, t.nkb);
          left -= n;
          const int buf = buf_i & 1;
          if (!mbar_wait(bar_tempty + 8 * buf, (((uint32_t)buf_i >> 1) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const uint32_t d_tmem = tmem_base + buf * XN;
          uint32_t acc = 0u;
          for (int k = 0; k < n;) {
            if (s == 0 && k + X_STAGES <= n) {
#pragma unroll
              for (int j = 0; j < X_STAGES; ++j) {
                if (!mbar_try_wait(bar_full + 8 * j, full_par) && !mbar_wait(bar_full + 8 * j, full_par, abort_flag)) { ok = false; break; }
                tc_fence_after();
                const uint32_t o = (uint32_t)(j * (X_STAGE_BYTES >> 4));
                tc_mma_bf16_pair(d_tmem, a0 + o, ah, b0 + o, bh, idesc, acc);
                tc_mma_bf16_pair(d_tmem, a1 + o, ah, b1 + o, bh, idesc, 1u);
                tc_mma_bf16_pair(d_tmem, a2 + o, ah, b2 + o, bh, idesc, 1u);
                tc_mma_bf16_pair(d_tmem, a3 + o, ah, b3 + o, bh, idesc, 1u);
                acc = 1u;
                tc_commit_pair(bar_empty + 8 * j);
              }
              if (!ok) break;
              full_par ^= 1u;
              k += X_STAGES;
              continue;
            }
            if (!mbar_try_wait(bar_full + 8 * s, full_par) && !mbar_wait(bar_full + 8 * s, full_par, abort_flag)) { ok = false; break; }
            tc_fence_after();
            const uint32_t o = s * (uint32_t)(X_STAGE_BYTES >> 4);
            tc_mma_bf16_pair(d_tmem, a0 + o, ah, b0 + o, bh, idesc, acc);
            tc_mma_bf16_pair(d_tmem, a1 + o, ah, b1 + o, bh, idesc, 1u);
            tc_mma_bf16_pair(d_tmem, a2 + o, ah, b2 + o, bh, idesc, 1u);
            tc_mma_bf16_pair(d_tmem, a3 + o, ah, b3 + o, bh, idesc, 1u);
            acc = 1u;
            tc_commit_pair(bar_empty + 8 * s);
            if (++s == X_STAGES) { s = 0; full_par ^= 1u; }
            ++k;
          }
          if (ok) tc_commit_pair(bar_tfull + 8 * buf);
          ++buf_i;
        }
      }
    }
  } else {
    // ------------------------------ epilogue (both CTAs) ----------------------
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    const uint32_t lane_addr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(half * 128);
    const uint32_t tempty = map_to_cta(bar_tempty, 0);      // the leader's barriers, as cluster addresses
    int buf_i = 0;
    bool ok = true;
    XItem t;
    for (int i = 0; ok && x_item(p, pair_id, num_pairs, i, t); ++i) {
      const XProblem& r = p.pr[t.q];
      float acc[128];
      bool first = true;
      int left = t.nkb * r.products;
      while (left > 0) {
        left -= x_part(p, left, t.nkb);
        const int buf = buf_i & 1;
        if (!mbar_wait_yield<64>(bar_tfull + 8 * buf, ((uint32_t)buf_i >> 1) & 1u, abort_flag)) { ok = false; break; }
        ++buf_i;
        tc_fence_after();
        if (first) {                 // all four loads in flight
          uint32_t v[128];
#pragma unroll
          for (int c = 0; c < 4; ++c) HDQT_TMEM_LD32(lane_addr + buf * XN + c * 32, (v + c * 32));
#pragma unroll
          for (int c = 0; c < 4; ++c) HDQT_TMEM_WAIT32((v + c * 32));
#pragma unroll
          for (int k = 0; k < 128; ++k) acc[k] = __uint_as_float(v[k]);
        } else {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            uint32_t v[32];
            HDQT_TMEM_LD32(lane_addr + buf * XN + c * 32, v);
            HDQT_TMEM_WAIT32(v);
#pragma unroll
            for (int k = 0; k < 32; ++k) acc[c * 32 + k] += __uint_as_float(v[k]);
          }
        }
        first = false;
        // the accumulator is in registers: hand it back before anything else
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_read(tempty + 8 * buf);
      }
      if (!ok) break;
      const int row = t.m * XM + (int)cta_rank * 128 + quarter * 32 + lane;
      const int col0 = t.n * XN + half * 128;
      if constexpr (kEpi == X_STATS || kEpi == X_CODES || kEpi == X_LOGITS) x_stats<kEpi>(p, r, t, row, col0, half, acc);
      else if constexpr (kEpi == X_DZ) x_dz(p, r, row, col0, acc);
      else if (x_out_even(r)) x_out(p, r, t, row, col0, acc);
      else x_out_odd(p, r, t, row - lane, col0, lane, reinterpret_cast<float*>(smem_raw + X_BOX_OFF + (warp - 2) * X_BOX), acc);
    }
  }

  tc_fence_before();
  __syncthreads();
  cluster_sync_all();     // neither CTA leaves while the other may still read its operands or signal its barriers
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(X_TMEM_COLS)
                 : "memory");
  }
  if (threadIdx.x == 0 && *abort_flag) report_status(p.dev_status, HDQT_ERR_TIMEOUT);
}

}  // namespace

}  // namespace hdqt
