// Dense products on the matrix cores with fused epilogues: the core shared by
// the linear, gated and classifying layers (dense_kernels.h).
//
//   out[q][p] = sum_k P(p, k) Q(q, k),   p contiguous in memory
//
// Each operand is stored along k ([rows][k], "C") or across it ([k][rows],
// "S"): a forward pass is C x C, an input gradient S x C, a weight gradient
// S x S.  A workgroup computes BP x BQ outputs; k runs in steps of 128 bytes.
// Both tiles of a step go from memory straight to LDS (16 bytes per lane; fp32:
// through registers), two or four steps ahead, one barrier per step.
//
// A fragment is 16 bytes per lane: lane (g = lane / 16, i = lane % 16) holds
// row i and the k's 8 g .. 8 g + 7 of 32 (16-bit types, one MFMA 16x16x32) or
// 4 g .. 4 g + 3 of 16 (fp32, four MFMA 16x16x4, the n-th taking element n of
// every lane; both operands agree on the order of k, which is free).
//   C: one 128-bit LDS read.  Rows are 128 bytes; chunk c (16 bytes) of row r
//      lies at c ^ ((r >> 1) & 7), so that 16 rows' reads cover all banks.
//   S: transposed LDS reads (16-bit) or one dword per k (fp32).  Row k's
//      chunk c lies at c ^ swizzle(k), spreading the rows of one read.
// MFMA's first operand is P: a lane ends up with 4 consecutive p of one q.
//
// Bounds: an operand is read through a buffer descriptor whose extent ends
// with its last element, so rows past the end read as 0 (each of a load's four
// dwords is checked by itself; rows need to start at whole dwords only); the
// tail of k is cut off lane by lane (C; within 16 bytes, in LDS) or by the
// extent (S).  p and q past the end are not stored.
#pragma once

#include <type_traits>

#include "qcnn_internal.h"

namespace qcnn {
namespace dense {

typedef float f2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef __bf16 b4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void;

// Transposing LDS read: with 16 lanes' addresses on 4 rows of 16 elements (lane
// i: row i / 4, elements 4 (i % 4) ..), lane i receives element i of each row.
__device__ __forceinline__ s4 read_transposed(const char* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)p);
}

template <typename T>
struct Num;

template <>
struct Num<float> {
  typedef f4 Frag;
  typedef f4 Quad;
  static __device__ __forceinline__ f4 mma(Frag a, Frag b, f4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ float exp_(float x) { return expf(x); }
  static __device__ __forceinline__ float div_(float a, float b) { return a / b; }
  // The normal distribution function; density = exp(-z^2 / 2).  By erfc, which
  // keeps its digits where 1 + erf cancels (below z = -5.5 nothing is left of it).
  static __device__ __forceinline__ float phi(float z, float) { return 0.5f * erfcf(z * -0.70710678118654752f); }
};

// 16-bit results carry 8 or 11 bits: the hardware's exponential and reciprocal
// (about 2^-22) are far below their rounding.
struct Num16 {
  static __device__ __forceinline__ float exp_(float x) { return __expf(x); }
  static __device__ __forceinline__ float div_(float a, float b) { return a * __builtin_amdgcn_rcpf(b); }
  // Phi(-|z|) = exp(-z^2 / 2) t Q(t), t = 1 / (1 + c |z|), with Q the polynomial
  // of degree 6 that fits Phi(-|z|) exp(z^2 / 2) / t over |z| < 28 best in the
  // largest relative error, 2e-6: a sixth of erff's instructions, and the
  // slope's exponential with it (4096 x 4096 slopes: 45 us with erff).
  static __device__ __forceinline__ float phi(float z, float density) {
    const float t = __builtin_amdgcn_rcpf(1.f + 0.371231049f * fabsf(z));
    const float upper = 0.0494158827f + t * (0.139162809f + t * (-0.166493893f + t * 0.0475246012f));
    const float tail = density * t * (0.148124367f + t * (0.14742066f + t * (0.134845033f + t * upper)));
    return z > 0.f ? 1.f - tail : tail;
  }
};

template <>
struct Num<__bf16> : Num16 {
  typedef b8 Frag;
  typedef b4 Quad;
  static __device__ __forceinline__ f4 mma(Frag a, Frag b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ b4 read_tr(const char* p) {
    return __builtin_bit_cast(b4, read_transposed(p));
  }
};

template <>
struct Num<_Float16> : Num16 {
  typedef h8 Frag;
  typedef h4 Quad;
  static __device__ __forceinline__ f4 mma(Frag a, Frag b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ h4 read_tr(const char* p) {
    return __builtin_bit_cast(h4, read_transposed(p));
  }
};

// ------------------------------------------------------------- activations

template <typename T>
__device__ __forceinline__ float act_value(int act, float z) {
  switch (act) {
    case QCNN_ACT_RELU: return z > 0.f ? z : z != z ? z : 0.f;
    case QCNN_ACT_GELU: return z * Num<T>::phi(z, Num<T>::exp_(-0.5f * z * z));
    case QCNN_ACT_GELU_TANH: {  // 1 + tanh(u) = 2 / (1 + exp(-2 u))
      const float u2 = 1.5957691216057308f * (z + 0.044715f * z * z * z);
      return Num<T>::div_(z, 1.f + Num<T>::exp_(-u2));
    }
    case QCNN_ACT_SILU: return Num<T>::div_(z, 1.f + Num<T>::exp_(-z));
    default: return z;
  }
}

template <typename T>
__device__ __forceinline__ float act_slope(int act, float z) {
  switch (act) {
    case QCNN_ACT_RELU: return z > 0.f ? 1.f : z != z ? z : 0.f;
    case QCNN_ACT_GELU: {
      const float density = Num<T>::exp_(-0.5f * z * z);
      return Num<T>::phi(z, density) + 0.39894228040143268f * z * density;
    }
    case QCNN_ACT_GELU_TANH: {
      const float s = Num<T>::div_(1.f, 1.f + Num<T>::exp_(-1.5957691216057308f * (z + 0.044715f * z * z * z)));
      // z^2 overflows from 2^64 on, where s (1 - s) is 0.
      return s + z * s * (1.f - s) * 1.5957691216057308f * (1.f + 0.134145f * fminf(z * z, 0x1p100f));
    }
    case QCNN_ACT_SILU: {
      const float s = Num<T>::div_(1.f, 1.f + Num<T>::exp_(-z));
      return s * (1.f + z * (1.f - s));
    }
    default: return 1.f;
  }
}

// --------------------------------------------------------------- epilogues

enum EpiKind { kLinear = 0, kPartial = 1, kGated = 2, kStats = 3, kXgrad = 4 };

// What becomes of a sum.  Quads are 4 consecutive p.
struct Epi {
  void* y;          // T [nq][ldy]: the result (kXgrad: the logits' gradient)
  void* pre;        // T [nq][ldpre] or null: the sum with its bias
  const void* bias; // T [np] (kGated: [2 np]) or null
  const void* res;  // T [nq][ldr] or null: added last
  float* acc;       // fp32 [nq][ldacc]: running sums over pieces of k, or null
  const float* alpha;  // device scalar that the finished sum is multiplied by, or null
  long long ldy, ldpre, ldr, ldacc;
  int act;
  int acc_in, acc_out;  // add what is in acc; leave the sum there (no y)
  // kStats, kXgrad: classes class0 .. class0 + np - 1 of `classes`
  const long long* labels;
  const float* lse;
  const float* dloss;
  const float* dmax;  // device scalar: dmax_kernel's out[0]
  float gain;
  float2* stat;       // [slot][nq]: maximum and sum of exponentials of a slot's logits
  float* zlabel;      // [nq]: the label's logit
  float *loss, *lse_out;  // [nq]: for the kernel that finishes a split product
  int class0, classes;
};

// Four elements, or the n that are left.  Global memory takes them at any
// address: rows of odd length need no other path.
template <typename T>
__device__ __forceinline__ f4 load_quad(const T* p, int n) {
  typename Num<T>::Quad t;
  f4 v = {0.f, 0.f, 0.f, 0.f};
  if (n >= 4) {
    __builtin_memcpy(&t, p, sizeof(t));
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)t[i];
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < n) v[i] = (float)p[i];
  }
  return v;
}

template <typename T>
__device__ __forceinline__ void store_quad(T* p, f4 v, int n) {
  typename Num<T>::Quad t;
#pragma unroll
  for (int i = 0; i < 4; ++i) t[i] = (T)v[i];
  if (n >= 4) {
    __builtin_memcpy(p, &t, sizeof(t));
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < n) p[i] = t[i];
  }
}

// 16 bytes of elements, or the n that are left.
template <typename T, int Q>
__device__ __forceinline__ void load_wide(const T* p, int n, f4 (&v)[Q]) {
  if (n >= 4 * Q) {
    typename Num<T>::Frag t;
    __builtin_memcpy(&t, p, 16);
#pragma unroll
    for (int i = 0; i < 4 * Q; ++i) v[i / 4][i % 4] = (float)t[i];
  } else {
#pragma unroll
    for (int k = 0; k < Q; ++k) v[k] = load_quad(p + 4 * k, n - 4 * k);
  }
}

template <typename T, int Q>
__device__ __forceinline__ void store_wide(T* p, int n, const f4 (&v)[Q]) {
  if (n >= 4 * Q) {
    typename Num<T>::Frag t;
#pragma unroll
    for (int i = 0; i < 4 * Q; ++i) t[i] = (T)v[i / 4][i % 4];
    __builtin_memcpy(p, &t, 16);
  } else {
#pragma unroll
    for (int k = 0; k < Q; ++k) store_quad(p + 4 * k, v[k], n - 4 * k);
  }
}

// The bias of columns p .. p + 3 (zeros without one, and past the end).
template <typename T>
__device__ __forceinline__ f4 bias_quad(const Epi& e, int np, int p, int from = 0) {
  if (!e.bias || p >= np) return f4{0.f, 0.f, 0.f, 0.f};
  return load_quad(static_cast<const T*>(e.bias) + from + p, np - p);
}

// What becomes of U quads of columns p .. p + 3 in rows q, q + dq, ...: all
// their loads first, so that they are on their way together.
template <typename T, int U>
__device__ __forceinline__ void emit_linear(const Epi& e, int np, int nq, int q, int dq, int p, f4 (&v)[U], f4 bias) {
  const int n = np - p;
  if (n <= 0) return;
  if (e.acc_in) {
#pragma unroll
    for (int k = 0; k < U; ++k)
      if (q + k * dq < nq) v[k] += *reinterpret_cast<const f4*>(e.acc + (q + k * dq) * e.ldacc + p);
  }
  if (e.acc_out) {
#pragma unroll
    for (int k = 0; k < U; ++k)
      if (q + k * dq < nq) *reinterpret_cast<f4*>(e.acc + (q + k * dq) * e.ldacc + p) = v[k];
    return;
  }
  f4 r[U];
#pragma unroll
  for (int k = 0; k < U; ++k) {
    r[k] = f4{0.f, 0.f, 0.f, 0.f};
    if (e.res && q + k * dq < nq) r[k] = load_quad(static_cast<const T*>(e.res) + (q + k * dq) * e.ldr + p, n);
  }
  const float alpha = e.alpha ? *e.alpha : 1.f;
#pragma unroll
  for (int k = 0; k < U; ++k) {
    if (q + k * dq >= nq) break;
    f4 z = v[k] * alpha + bias;
    if (e.pre) store_quad(static_cast<T*>(e.pre) + (q + k * dq) * e.ldpre + p, z, n);
    if (e.act != QCNN_ACT_NONE) {
#pragma unroll
      for (int i = 0; i < 4; ++i) z[i] = act_value<T>(e.act, z[i]);
    }
    if (e.res) z += r[k];
    store_quad(static_cast<T*>(e.y) + (q + k * dq) * e.ldy + p, z, n);
  }
}

// np: columns of the result (half of the weight's rows).
template <typename T, int U>
__device__ __forceinline__ void emit_gated(const Epi& e, int np, int nq, int q, int dq, int p, f4 (&g)[U], f4 (&u)[U],
                                           f4 bias_g, f4 bias_u) {
  const int n = np - p;
  if (n <= 0) return;
#pragma unroll
  for (int k = 0; k < U; ++k) {
    if (q + k * dq >= nq) break;
    f4 z = g[k] + bias_g, w = u[k] + bias_u;
    if (e.pre) {
      T* pre = static_cast<T*>(e.pre) + (q + k * dq) * e.ldpre + p;
      store_quad(pre, z, n);
      store_quad(pre + np, w, n);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = act_value<T>(e.act, z[i]) * w[i];
    store_quad(static_cast<T*>(e.y) + (q + k * dq) * e.ldy + p, z, n);
  }
}

// Logits with their bias; classes past the end become -inf.
__device__ __forceinline__ f4 class_logits(int np, int p, f4 v, f4 bias) {
  v += bias;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i >= np - p) v[i] = -INFINITY;
  return v;
}

// d = dloss (softmax - onehot), divided by the largest |dloss| (the products
// that read d multiply it back) so that a mean's 1 / N neither leaves a 16-bit
// type's range nor rounds every label's entry the same way; times `gain`, a
// power of two that keeps fp16's small probabilities off its subnormals.
// Rounded to T, which is what the products take; its column sums are made from
// the rounded entries, too (the tiles of a column do not meet).
// y's rows are whole quads: what lies past np is written as 0.
template <typename T, int U>
__device__ __forceinline__ void emit_xgrad(const Epi& e, int np, int nq, int q, int dq, int p, f4 (&z)[U], f4 bias) {
  int at[U];  // the label's place from p on
  float lse[U], w[U];
  bool counted[U];
  const float scale = e.gain / *e.dmax;
#pragma unroll
  for (int k = 0; k < U; ++k) {
    const int row = min(q + k * dq, nq - 1);
    const long long label = e.labels[row];
    counted[k] = label >= 0;
    at[k] = label >= e.classes ? -1 : (int)label - e.class0 - p;
    lse[k] = e.lse[row];
    w[k] = label >= e.classes ? NAN : e.dloss[row] * scale;
  }
#pragma unroll
  for (int k = 0; k < U; ++k) {
    if (q + k * dq >= nq) break;
    const f4 l = z[k] + bias;
    f4 d = {0.f, 0.f, 0.f, 0.f};
    if (counted[k]) {
#pragma unroll
      for (int i = 0; i < 4; ++i) d[i] = w[k] * (Num<T>::exp_(l[i] - lse[k]) - (at[k] == i ? 1.f : 0.f));
    }
    if (np - p < 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i >= np - p) d[i] = 0.f;
    }
    store_quad(static_cast<T*>(e.y) + (q + k * dq) * e.ldy + p, d, 4);
  }
}

// (max, sum of exp(. - max)) of two disjoint sets.  fmaxf passes over NaN: the
// sum is what carries it.  A set whose maximum is -inf is empty or masked and
// has the sum 0, or NaN where a logit was that; either is added as it is.  The
// hardware's exponential in fp32 too: it is off by |x| 2^-24 of exp(x), that is
// a sum of C exponentials by log(C) 2^-24 of itself at most, and lse by as much.
__device__ __forceinline__ float2 join_stat(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x);
  const float sa = a.x == -INFINITY ? a.y : a.y * __expf(a.x - m);
  const float sb = b.x == -INFINITY ? b.y : b.y * __expf(b.x - m);
  return make_float2(m, sa + sb);
}

// ------------------------------------------------------------- the product

struct Prod {
  const char* p;
  const char* q;
  long long ldp, ldq;   // bytes
  int np, nq, nk;       // outputs and terms
  int kp, kq;           // rows that an S operand has (C: unused)
  int colsp, colsq;     // columns that an S operand stores, whole dwords (as nk of a C operand)
  int p2;               // kGated: rows between a gate row and its up row
  int p0, p1, q0, q1;   // the outputs of this launch; kStats: their first slot
  int slot0;
  int splits, steps;    // parts of k; steps of 128 bytes in each
  float* part;          // kPartial: fp32 [splits][nq][ldpart]
  long long ldpart;     // kGated's sums: gate at p, up at ldpart / 2 + p
};

__device__ __forceinline__ int bytes_of(long long bytes) {
  const int low = (int)bytes, high = (int)(bytes >> 32);  // scalar compares have 32 bits
  return high < 0 ? 0 : high > 0 || low < 0 ? 0x7fffffff : low;
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t resource(const char* base, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, bytes, 0x00020000);
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t descriptor(const char* base, long long bytes) {
  return resource(base, bytes_of(bytes));
}

// An operand's tile of ROWS rows: staging and fragments.
template <typename T, bool S, int ROWS, int NW>
struct Operand {
  static constexpr int kS = sizeof(T);
  static constexpr int kStep = 128 / kS;                   // k's of a step
  static constexpr int kRowBytes = S ? ROWS * kS : 128;    // LDS row
  static constexpr int kPerRow = kRowBytes / 16;           // chunks of an LDS row
  static constexpr int kRowsPer = 64 / kPerRow;            // LDS rows of one wave's load
  static constexpr int kLoads = ROWS * 128 / 1024 / NW;    // loads of one wave and step
  static constexpr int kBytes = ROWS * 128;
  static constexpr int kReads = S ? (kS == 2 ? 2 : 4) : 1;  // LDS reads of a fragment
  static_assert(kLoads >= 1 && kLoads * NW * 1024 == ROWS * 128, "whole loads");
  static_assert(!S || kRowBytes >= 256, "the swizzle of S tiles spans 256 bytes");
  static_assert(kPerRow <= 64, "a row per load at least");

  // XOR on the chunk index of LDS row r.
  static constexpr __host__ __device__ int swizzle(int r) {
    return !S ? (r >> 1) & 7 : kS == 2 ? 2 * ((r & 3) | (((r >> 3) & 1) << 2)) : 4 * ((r >> 2) & 3);
  }

  // Load j of a wave fills kRowsPer LDS rows from first(j); a lane's row among
  // them and its chunk there (in bytes; the first load's, the others differ by
  // a constant) do not depend on j.
  static __device__ __forceinline__ int first(int wave, int j) { return (wave + j * NW) * kRowsPer; }
  static __device__ __forceinline__ int lane_row(int lane) { return lane / kPerRow; }
  static __device__ __forceinline__ int lane_chunk(int wave, int lane) {
    return ((lane % kPerRow) ^ swizzle(first(wave, 0) + lane_row(lane))) * 16;
  }
  static constexpr __device__ int chunk_delta(int j) { return swizzle(j * NW * kRowsPer) * 16; }

  // Where a lane reads its part of the fragments of rows at, at + 1, ...
  static __device__ __forceinline__ int lane_base(int lane, int at) {
    const int g = lane >> 4, i = lane & 15;
    if (!S) return (at + i) * 128 + ((g ^ (i >> 1)) << 4);
    if (kS == 2)
      return (8 * g + (i >> 2)) * kRowBytes + (((at >> 3) + ((i & 3) >> 1)) ^ (2 * ((i >> 2) | ((g & 1) << 2)))) * 16 +
             (i & 1) * 8;
    return 4 * g * kRowBytes + (((at + i) >> 2) ^ (4 * g)) * 16 + (i & 3) * 4;
  }

  // Fragment f (16 rows further on each) of the kk-th part of a step.
  static __device__ __forceinline__ typename Num<T>::Frag frag(const char* lds, int base, int f, int kk) {
    if constexpr (!S) {
      return *reinterpret_cast<const typename Num<T>::Frag*>(lds + (base ^ (kk * 64)) + f * 2048);
    } else if constexpr (kS == 2) {
      const char* a = lds + (base ^ (f * 32)) + kk * 32 * kRowBytes;
      const auto lo = Num<T>::read_tr(a), hi = Num<T>::read_tr(a + 4 * kRowBytes);
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      const char* a = lds + (base ^ (f * 64)) + kk * 16 * kRowBytes;
      f4 v;
#pragma unroll
      for (int n = 0; n < 4; ++n) v[n] = *reinterpret_cast<const float*>(a + n * kRowBytes);
      return v;
    }
  }
};

// Four fp32 values as three bf16 parts each: the nearest 8 bits of the 24, the
// nearest 8 of what is left, and the rest, which is exact.  Of the nine products
// of two numbers' parts the three smallest are left out: the parts are at most
// 2^-8 and 2^-17 of a number in [1, 2), so these come to 2^-24 of the product,
// of either sign (upper bits cut off: 2^-21, always shrinking it).  The largest
// numbers round to an infinity; their tiles are computed again.
__device__ __forceinline__ void split_bf16(f4 x, uint2 (&out)[3]) {
#pragma unroll
  for (int n = 0; n < 3; ++n) {
    uint32_t u[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      u[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{x[2 * i], x[2 * i + 1]}, b2));
      x[2 * i] -= __uint_as_float(u[i] << 16);
      x[2 * i + 1] -= __uint_as_float(u[i] & 0xffff0000u);
    }
    out[n] = make_uint2(u[0], u[1]);
  }
}

// Whether any thread of the workgroup has `bad`; `word` is LDS that nobody uses.
__device__ __forceinline__ bool any_of_group(bool bad, int* word) {
  if (threadIdx.x == 0) *word = 0;
  __syncthreads();
  if (bad) *word = 1;
  __syncthreads();
  const bool any = *word != 0;
  __syncthreads();
  return any;
}

// This wave's loads but the last N have landed and its LDS reads are done;
// then everyone's.
template <int N>
__device__ __forceinline__ void wait_and_meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | (N >> 4) << 14);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// The waves' LDS accesses are done; loads to registers may be on their way.
__device__ __forceinline__ void meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Tile (tp, tq) and part of k of a workgroup.  Consecutive workgroups go to
// the 8 XCDs in turn, each with an L2 of its own: every XCD gets a contiguous
// run of tiles, and a run goes down groups of 8 q tiles, so that what is in
// flight on one XCD shares rows of both operands.
__device__ __forceinline__ void tile_of(int id, int total, int tps, int tqs, int* tp, int* tq, int* split) {
  const int per = total / 8, over = total % 8, x = id % 8;
  id = id / 8 + x * per + (x < over ? x : over);
  const int tiles = tps * tqs;
  *split = id / tiles;
  id -= *split * tiles;
  const int group = id / (8 * tps), first = group * 8;
  const int size = tqs - first < 8 ? tqs - first : 8;
  id -= group * 8 * tps;
  *tq = first + id % size;
  *tp = id / size;
}

// An operand's tile walked along k, 128 bytes a step: what a lane loads where.
template <typename T, bool S, int ROWS, int NW>
struct Walk {
  typedef Operand<T, S, ROWS, NW> O;
  const char* base;
  long long ld, kbytes, extent;  // extent: bytes from base to the operand's end
  int lane_off, chunk;           // of a lane: its row's offset, its bytes in the row

  // first: the tile's first row of `rows` (C) or column of `cols` stored (S);
  // krows: an S operand's rows.  swizzled: the lanes' chunks in the order that
  // LDS wants them, for loads that go there.
  __device__ __forceinline__ Walk(const char* p, long long ld_, int first, int rows, int cols, int nk, int krows,
                                  int wave, int lane, bool swizzled)
      : ld(ld_), kbytes((long long)nk * O::kS) {
    base = p + (S ? (long long)first * O::kS : first * ld);
    extent = S ? (krows - 1) * ld + (long long)(cols - first) * O::kS : (rows - 1 - first) * ld + kbytes;
    lane_off = (int)(O::lane_row(lane) * ld);
    chunk = swizzled ? O::lane_chunk(wave, lane) : lane % O::kPerRow * 16;
  }

  // The tile's first byte in a step, and from there to the operand's end.
  __device__ __forceinline__ long long before(int step) const {
    return S ? (long long)step * O::kStep * ld : (long long)step * 128;
  }
  // Bytes of k that a C operand has in this step.
  __device__ __forceinline__ int left(int step) const { return min((int)kbytes - step * 128, 128); }

  // Offset of load j's 16 bytes; row: the load's first in the tile.
  __device__ __forceinline__ int offset(int row, int delta, int left) const {
    const int v = lane_off + (chunk ^ delta) + (int)(row * ld);
    return !S && chunk >= left ? (int)0x80000000 : v;
  }
};

// A step's descriptor, `rows_on` rows further on; none: it holds nothing.
template <typename W>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t descriptor(const W& w, int step, bool none, long long rows_on = 0) {
  const long long before = w.before(step);
  return descriptor(w.base + before + rows_on * w.ld, none ? 0 : w.extent - before);
}

// The weight row of a gated tile's row: a wave's WP rows are WP / 2 gate rows
// and, from the same first one, their up rows, so that a lane has both sums.
template <int WP>
__device__ __forceinline__ int gated_row(int r) { return r / WP * (WP / 2) + r % (WP / 2); }
template <int WP>
__device__ __forceinline__ bool gated_up(int r) { return r % WP >= WP / 2; }

// Where a workgroup's tile lies.
struct Place {
  int tp, cp, cq, split, step0, nsteps;
  bool ragged;  // its last step ends within 16 bytes of k
};

template <int BC, int BQ, int S>
__device__ __forceinline__ Place place_of(const Prod& a) {
  Place t;
  int tq;
  tile_of(blockIdx.x, gridDim.x, (a.p1 - a.p0 + BC - 1) / BC, (a.q1 - a.q0 + BQ - 1) / BQ, &t.tp, &tq, &t.split);
  t.cp = a.p0 + t.tp * BC;
  t.cq = a.q0 + tq * BQ;
  t.step0 = t.split * a.steps;
  const int all = (int)(((long long)a.nk * S + 127) / 128);
  t.nsteps = min(a.steps, all - t.step0);
  t.ragged = (a.nk * S & 15) && t.step0 + t.nsteps == all;
  return t;
}

// The lane's number, counted anew: no register holds it through the loop.
__device__ __forceinline__ int fresh_lane() {
  int ones = -1;
  asm volatile("" : "+s"(ones));
  return __builtin_amdgcn_mbcnt_hi(ones, __builtin_amdgcn_mbcnt_lo(ones, 0));
}

// In the tiles of a ragged last step, zeros from its `left` bytes of k on to
// the next 16 (what lies behind the rows' ends was loaded there): a row per
// thread.  Between a barrier that the tiles are complete behind and another.
template <bool PS, bool QS, int BP, int BQ>
__device__ __forceinline__ void zero_tail(char* lp, char* lq, int left, int wave) {
  const int id = wave * 64 + fresh_lane();
  const bool is_p = id < BP;
  const int r = is_p ? id : id - BP;
  if (is_p ? PS : QS || r >= BQ) return;
  char* at = (is_p ? lp : lq) + r * 128 + (((left >> 4) ^ ((r >> 1) & 7)) << 4);
  for (int d = left & 15; d < 16; d += 4) *reinterpret_cast<uint32_t*>(at + d) = 0;
}

constexpr int kRoomBytes = 16384;

// What becomes of a wave's sums: acc[i][j] holds p = 16 i + 4 g + 0..3 of
// q = 16 j + lane % 16.  room: 16 KB of LDS for this wave alone.
template <typename T, int WP, int WQ, int NWP, int EPI, bool GATED>
__device__ __forceinline__ void finish_tile(const Prod& a, const Epi& e, const Place& at, f4 (&acc)[WP / 16][WQ / 16],
                                            f4* room, int lane, int wp, int wq) {
  constexpr int FP = WP / 16, FQ = WQ / 16;
  const int tp = at.tp, cp = at.cp, cq = at.cq, split = at.split;
  const int g = lane >> 4, c = lane & 15;
  if constexpr (EPI == kStats) {
    const int q_first = cq + wq * WQ + c, p_wave = cp + wp * WP, p_first = p_wave + 4 * g;
    if (e.bias || p_wave + WP > a.np) {  // else the sums are the logits
#pragma unroll
      for (int i = 0; i < FP; ++i) {
        const f4 bias = bias_quad<T>(e, a.np, p_first + 16 * i, e.class0);
#pragma unroll
        for (int j = 0; j < FQ; ++j) acc[i][j] = class_logits(a.np, p_first + 16 * i, acc[i][j], bias);
      }
    }
#pragma unroll
    for (int j = 0; j < FQ; ++j) {
      const int q = q_first + 16 * j;
      const long long label = q < a.nq ? e.labels[q] - e.class0 : -1;
      float m = -INFINITY;
#pragma unroll
      for (int i = 0; i < FP; ++i)
#pragma unroll
        for (int n = 0; n < 4; ++n) m = fmaxf(m, acc[i][j][n]);
      // The difference first: a mask of the type's lowest value must not overflow.
      const float top = m == -INFINITY ? 0.f : m;
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < FP; ++i)
#pragma unroll
        for (int n = 0; n < 4; ++n) sum += __expf(acc[i][j][n] - top);
      if (label >= p_wave && label < min(p_wave + WP, a.np)) {  // few waves have a row's label
        const int at = (int)label - p_first;
#pragma unroll
        for (int i = 0; i < FP; ++i)
#pragma unroll
          for (int n = 0; n < 4; ++n)
            if (at == 16 * i + n) e.zlabel[q] = acc[i][j][n];
      }
      float2 t = make_float2(m, sum);
#pragma unroll
      for (int o = 16; o < 64; o *= 2) t = join_stat(t, make_float2(__shfl_xor(t.x, o), __shfl_xor(t.y, o)));
      if (g == 0 && q < a.nq) e.stat[(long long)(a.slot0 + tp * NWP + wp) * a.nq + q] = t;
    }
  } else {
    // Through LDS, a wave's 16 KB of it: 64 lanes in the products' order hold
    // 16 rows' 32 bytes each, and memory wants whole lines (stored as they
    // are, 2.4 times the result's bytes were written to HBM).  Row q's quad p
    // lies at p ^ (q % 16), free of conflicts both ways.
    constexpr int kRows = kRoomBytes / (WP * 4) < WQ ? kRoomBytes / (WP * 4) : WQ;
    constexpr int kQuads = WP / 4, kOut = GATED ? kQuads / 2 : kQuads;  // of a row; that one emit covers
    static_assert(kQuads >= 16 && kRows % 16 == 0, "the XOR stays within a row");
    const int quad = lane % kOut, p = cp + wp * (GATED ? WP / 2 : WP) + 4 * quad;  // a lane keeps its columns
    f4 bias = {0.f, 0.f, 0.f, 0.f}, bias_up = bias;
    if constexpr (EPI != kPartial) {
      bias = bias_quad<T>(e, a.np, p, EPI == kXgrad ? e.class0 : 0);
      if (GATED) bias_up = bias_quad<T>(e, a.np, p, a.np);
    }
#pragma unroll
    for (int first = 0; first < WQ; first += kRows) {
#pragma unroll
      for (int j = 0; j < kRows / 16; ++j)
#pragma unroll
        for (int i = 0; i < FP; ++i) room[(16 * j + c) * kQuads + ((4 * i + g) ^ c)] = acc[i][first / 16 + j];
      constexpr int kAll = kRows * kOut / 64, U = kAll < 4 ? kAll : 4, kStep = 64 / kOut;
#pragma unroll 1
      for (int t = 0; t < kAll; t += U) {
        const int row = t * kStep + lane / kOut, q = cq + wq * WQ + first + row;
        f4 v[U], u[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
          const int r = row + k * kStep;
          v[k] = room[r * kQuads + (quad ^ (r & 15))];
          u[k] = GATED ? room[r * kQuads + ((quad + kOut) ^ (r & 15))] : v[k];
        }
        if constexpr (EPI == kPartial) {
          if (p >= a.np) continue;
          float* o = a.part + ((long long)split * a.nq + q) * a.ldpart + p;
#pragma unroll
          for (int k = 0; k < U; ++k) {
            if (q + k * kStep >= a.nq) break;
            *reinterpret_cast<f4*>(o + k * kStep * a.ldpart) = v[k];
            if (GATED) *reinterpret_cast<f4*>(o + k * kStep * a.ldpart + a.ldpart / 2) = u[k];
          }
        } else if constexpr (GATED) {
          emit_gated<T, U>(e, a.np, a.nq, q, kStep, p, v, u, bias, bias_up);
        } else if constexpr (EPI == kXgrad) {
          if (p < e.ldy) emit_xgrad<T, U>(e, a.np, a.nq, q, kStep, p, v, bias);
        } else {
          emit_linear<T, U>(e, a.np, a.nq, q, kStep, p, v, bias);
        }
      }
    }
  }
}

// 16-bit products.  WP x WQ outputs per wave, DEPTH steps in LDS.  Large tiles
// (256 x 256, 8 waves of 128 x 64): a step is 64 MFMA per wave for 24 LDS reads
// of 16 bytes and 8 loads; a larger tile than 128 x 128 halves the LDS and L2
// bytes per product, and 64 KB a step twice is what LDS holds.  Bound by the
// matrix cores and the chip's power: 8192 x 4096 -> 16384 in bf16 takes 901 us
// in 50 calls in a row (1220 TFLOP/s), its input gradient 866, its weight
// gradient 873; single calls 860 to 1130 as the clock, 1.4 to 1.9 GHz, has it.
// The way there, in short runs of one day, which end at 825 us: 128 x 128 tiles
// 1185; 256 x 256 1128; with the half-step prefetch 1060; with results through
// LDS, not stored in the products' order, 955, and other steps 865; with a
// step's scalar work and loads between the products, not in a block behind the
// barrier, 825.  Four waves of 128 x 128 spill their sums between the two
// register files (1140 us); 32 x 32 MFMA are 5 % slower.
// Bounded to 512 threads also where 256 run: with more than 256 registers to
// give, the compiler keeps the sums in the other file and moves them around in
// every turn of the loop (512 x 4096 -> 4096: 29.2 us, so 28.2).
template <typename T, bool PS, bool QS, int BP, int BQ, int WP, int WQ, int DEPTH, int EPI, bool GATED>
__global__ __launch_bounds__(512) void product_kernel(const Prod a, const Epi e) {
#ifdef __HIP_DEVICE_COMPILE__  // the host pass, which only needs the name, gives up on the body without a word
  constexpr int NWP = BP / WP, NW = NWP * (BQ / WQ), FP = WP / 16, FQ = WQ / 16;
  static_assert(!GATED || !PS, "the gated layer's weights are read along k");
  typedef Operand<T, PS, BP, NW> OP;
  typedef Operand<T, QS, BQ, NW> OQ;
  // One array per tile: the compiler then knows that a read of one does not
  // wait for the loads into another.
  static_assert(DEPTH == 2 || DEPTH == 4, "buffers");
  __shared__ __align__(16) char p0[OP::kBytes], p1[OP::kBytes], q0[OQ::kBytes], q1[OQ::kBytes];
  __shared__ __align__(16) char p2[DEPTH > 2 ? OP::kBytes : 16], p3[DEPTH > 2 ? OP::kBytes : 16];
  __shared__ __align__(16) char q2[DEPTH > 2 ? OQ::kBytes : 16], q3[DEPTH > 2 ? OQ::kBytes : 16];
  char* const ps[4] = {p0, p1, p2, p3};
  char* const qs[4] = {q0, q1, q2, q3};
  constexpr int kFlight = OP::kLoads + OQ::kLoads;  // loads of a wave and step

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wp = wave % NWP, wq = wave / NWP;
  const Place t = place_of<GATED ? BP / 2 : BP, BQ, sizeof(T)>(a);
  const int nsteps = t.nsteps;
  // Large tiles have no registers left for it: their rows end with 16 bytes.
  constexpr bool kCut = BP == 128 && (!PS || !QS);
  const bool ragged = kCut && t.ragged;
  const Walk<T, PS, BP, NW> walk_p(a.p, a.ldp, t.cp, a.np, a.colsp, a.nk, a.kp, wave, lane, true);
  const Walk<T, QS, BQ, NW> walk_q(a.q, a.ldq, t.cq, a.nq, a.colsq, a.nk, a.kq, wave, lane, true);

  // Where a step's bytes lie; made ahead of its loads, in scalar registers,
  // except where both operands are read transposed: the order that this needs
  // costs large tiles eight vector registers too many (their loop spills:
  // weight gradient of 8192 x 4096 -> 16384, 1690 us for 815).
  constexpr bool kAhead = !PS || !QS;
  struct Source {
    const char *p, *q;
    int np, nq, left;
  };
  auto locate = [&](int s) __attribute__((always_inline)) {
    const int step = t.step0 + s;
    const bool none = s >= nsteps;  // loads nothing: the loop runs ahead of its end
    const long long bp = walk_p.before(step), bq = walk_q.before(step);
    Source r;
    r.p = walk_p.base + bp;
    r.q = walk_q.base + bq;
    r.np = bytes_of(none ? 0 : walk_p.extent - bp);
    r.nq = bytes_of(none ? 0 : walk_q.extent - bq);
    r.left = walk_p.left(step);
    if (kAhead) asm volatile("" : "+s"(r.p), "+s"(r.q), "+s"(r.np), "+s"(r.nq), "+s"(r.left));
    return r;
  };
  auto stage = [&](const Source& r, char* lp, char* lq) __attribute__((always_inline)) {
    const __amdgpu_buffer_rsrc_t rq = resource(r.q, r.nq), rp = resource(r.p, r.np);
    const __amdgpu_buffer_rsrc_t rp2 = GATED ? resource(r.p + a.p2 * walk_p.ld, r.np) : rp;
#pragma unroll
    for (int j = 0; j < OP::kLoads; ++j) {
      const int row = OP::first(wave, j);
      const int v = walk_p.offset(GATED ? gated_row<WP>(row) : row, OP::chunk_delta(j), r.left);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(GATED && gated_up<WP>(row) ? rp2 : rp,
                                               (lds_void*)(lp + (wave + j * NW) * 1024), 16, v, 0, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < OQ::kLoads; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rq, (lds_void*)(lq + (wave + j * NW) * 1024), 16,
                                               walk_q.offset(OQ::first(wave, j), OQ::chunk_delta(j), r.left), 0, 0, 0);
  };

  f4 acc[FP][FQ];
#pragma unroll
  for (int i = 0; i < FP; ++i)
#pragma unroll
    for (int j = 0; j < FQ; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};

  struct Frags {
    typename Num<T>::Frag p[FP], q[FQ];
  };
  int rp_ = OP::lane_base(lane, wp * WP), rq_ = OQ::lane_base(lane, wq * WQ);
  auto read = [&](Frags& f, const char* lp, const char* lq, int kk) __attribute__((always_inline)) {
    // One register each: the fragments' addresses are made from it again
    // every time (the registers are for the sums and two sets of fragments).
    asm volatile("" : "+v"(rp_), "+v"(rq_));
#pragma unroll
    for (int j = 0; j < FQ; ++j) f.q[j] = OQ::frag(lq, rq_, j, kk);
#pragma unroll
    for (int i = 0; i < FP; ++i) f.p[i] = OP::frag(lp, rp_, i, kk);
  };
  auto multiply = [&](const Frags& f) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < FP; ++i)
#pragma unroll
      for (int j = 0; j < FQ; ++j) acc[i][j] = Num<T>::mma(f.p[i], f.q[j], acc[i][j]);
  };
  // LDS reads, and a step's loads, one by one between the products.
  auto interleave = [&](auto loads_) __attribute__((always_inline)) {
    constexpr int reads = FP * OP::kReads + FQ * OQ::kReads, mmas = FP * FQ;
    constexpr int loads = decltype(loads_)::value;
    constexpr int per = mmas / (reads + loads) > 0 ? mmas / (reads + loads) : 1;
#pragma unroll
    for (int i = 0; i < loads; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, per, 0);
    }
#pragma unroll
    for (int i = 0; i < reads; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, per, 0);
      if (kAhead && loads == 0) __builtin_amdgcn_sched_group_barrier(0x004, 3, 0);
    }
    constexpr int rest = mmas - per * (reads + loads);
    if (rest > 0) __builtin_amdgcn_sched_group_barrier(0x008, rest, 0);
  };
  // A step: the first half's fragments are in f0.  Reads its second half
  // under the first half's products; then everyone's reads of this buffer are
  // done and everyone's loads of the next have landed: the step that is DEPTH
  // further on is sent for, and the next step's first half is read under the
  // second half's products.
  Frags f0, f1;
  auto body = [&](auto cut, int s, char* lp, char* lq, char* next_p, char* next_q) __attribute__((always_inline)) {
    read(f1, lp, lq, 1);
    multiply(f0);
    const Source far = locate(s + DEPTH);
    interleave(std::integral_constant<int, 0>());
    __builtin_amdgcn_sched_barrier(0);
    wait_and_meet<(DEPTH - 2) * kFlight>();
    if (decltype(cut)::value && ragged && s + 2 == nsteps) {
      zero_tail<PS, QS, BP, BQ>(next_p, next_q, walk_p.left(t.step0 + s + 1), wave);
      meet();
    }
    stage(far, lp, lq);
    read(f0, next_p, next_q, 0);
    multiply(f1);
    interleave(std::integral_constant<int, kFlight>());
    __builtin_amdgcn_sched_barrier(0);
  };

#pragma unroll
  for (int b = 0; b < DEPTH; ++b) stage(locate(b), ps[b], qs[b]);
  wait_and_meet<(DEPTH - 1) * kFlight>();
  if (ragged && nsteps == 1) {
    zero_tail<PS, QS, BP, BQ>(p0, q0, walk_p.left(t.step0), wave);
    meet();
  }
  read(f0, p0, q0, 0);
  // A branch within the loop would part what is to be interleaved: the steps
  // that may have to cut are behind it.
  constexpr int kRest = kCut ? DEPTH + 1 : DEPTH - 1;
  int s = 0;
  for (; s + DEPTH + (kCut ? 2 : 0) <= nsteps; s += DEPTH) {
#pragma unroll
    for (int b = 0; b < DEPTH; ++b)
      body(std::false_type(), s + b, ps[b], qs[b], ps[(b + 1) % DEPTH], qs[(b + 1) % DEPTH]);
  }
#pragma unroll
  for (int b = 0; b < kRest; ++b)
    if (s + b < nsteps)
      body(std::integral_constant<bool, kCut>(), s + b, ps[b % DEPTH], qs[b % DEPTH], ps[(b + 1) % DEPTH],
           qs[(b + 1) % DEPTH]);
  wait_and_meet<0>();  // nothing is on its way to this LDS, or read from it, any more

  constexpr int kPer = OP::kBytes / kRoomBytes;  // waves' rooms in a tile
  static_assert(OP::kBytes == OQ::kBytes && kPer * 4 >= NW, "a room for each wave");
  char* room = p0;
#pragma unroll
  for (int b = 1; b < 4; ++b)
    if (wave / kPer == b) room = b == 1 ? p1 : b == 2 ? q0 : q1;
  finish_tile<T, WP, WQ, NWP, EPI, GATED>(a, e, t, acc, reinterpret_cast<f4*>(room + wave % kPer * kRoomBytes),
                                          fresh_lane(), wp, wq);
#endif
}

// ---- fp32 products: three bf16 parts of each number, six products of them,
// instead of fp32's own matrix instruction, which has 1/16 of bf16's rate.
// The parts are made once per workgroup, between memory and LDS (made where
// the fragments are read, every number is split by two to four waves, and
// splitting takes as long as multiplying): a step's 32 k's go to registers, a
// step ahead, then as three tiles of bf16 to LDS, double-buffered.
//   C: rows of 64 bytes, chunk c (16 bytes, 8 k's) of row r at c ^ spread(r): the
//      hardware serves 16 lanes of a 128-bit read at a time, 8 of one chunk and
//      8 of the next, from rows 0-3, 12-15 and 4-11 (or the other way round).
//   S: rows along p or q as for 16-bit types, read transposed.
template <bool S, int ROWS, int NW>
struct Planes {
  typedef Operand<float, S, ROWS, NW> O;             // of the loads
  typedef Operand<__bf16, S, ROWS, NW> R;            // of an S tile's rows in LDS
  static constexpr int kPlane = ROWS * 64, kBytes = 3 * kPlane, kLoads = O::kLoads;

  // Where a lane's four numbers of load j go in a plane.
  static __device__ __forceinline__ int lane_write(int wave, int lane) {
    const int r = O::first(wave, 0) + O::lane_row(lane), c = lane % O::kPerRow;  // c: four numbers
    if (!S) return r * 64 + (((c >> 1) ^ spread(r)) << 4) + (c & 1) * 8;
    return r * R::kRowBytes + (((c >> 1) ^ swizzle(r)) << 4) + (c & 1) * 8;
  }
  static constexpr __device__ int swizzle(int r) { return 2 * ((r & 3) | (((r >> 3) & 1) << 2)); }
  static constexpr __device__ int spread(int r) {  // 0, 2, 3, 1 for rows 0-3, 4-7, 8-11, 12-15
    const int x = (r >> 2) & 3;
    return ((x ^ (x >> 1)) & 1) << 1 | x >> 1;
  }
  static __device__ __forceinline__ int write_at(int base, int j) {
    constexpr int kRow = S ? ROWS * 2 : 64;
    return (S ? base ^ (swizzle(j * NW * O::kRowsPer) << 4) : base) + j * NW * O::kRowsPer * kRow;
  }

  static __device__ __forceinline__ int lane_read(int lane, int at) {
    const int g = lane >> 4, i = lane & 15;
    if constexpr (S) return R::lane_base(lane, at);
    else return (at + i) * 64 + ((g ^ spread(i)) << 4);
  }
  static __device__ __forceinline__ b8 frag(const char* plane, int base, int f) {
    if constexpr (S) return R::frag(plane, base, f, 0);
    else return *reinterpret_cast<const b8*>(plane + base + f * 1024);
  }
};

// Large tiles 256 x 128 (8 waves of 64 x 64), small ones 128 x 128 (of 64 x 32).
// Bound by the matrix cores and power: 4096 x 4096 -> 4096 takes 639 us forward
// in 50 calls in a row, 647 and 645 for the gradients (215 TFLOP/s, that is 1290
// of bf16 products); single calls 630 to 720.  The way there, in short runs:
// fp32's own instruction 970, split where the fragments are read 712 to 765,
// split in blocks before and after the products of a row 720 (gradients 625 and
// 617), between them one by one 670 (608 and 585).
template <bool PS, bool QS, int BP, int BQ, int WP, int WQ, int EPI, bool GATED>
__global__ __launch_bounds__(64 * (BP / WP) * (BQ / WQ)) void product_f32_kernel(const Prod a, const Epi e) {
#ifdef __HIP_DEVICE_COMPILE__
  constexpr int NWP = BP / WP, NW = NWP * (BQ / WQ), FP = WP / 16, FQ = WQ / 16;
  static_assert(!GATED || !PS, "the gated layer's weights are read along k");
  typedef Planes<PS, BP, NW> LP;
  typedef Planes<QS, BQ, NW> LQ;
  // Two arrays: the compiler then knows that reads of one may pass writes of
  // the other.
  __shared__ __align__(16) char lds[LP::kBytes + LQ::kBytes], other[LP::kBytes + LQ::kBytes];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wp = wave % NWP, wq = wave / NWP;
  const Place t = place_of<GATED ? BP / 2 : BP, BQ, 4>(a);
  const Walk<float, PS, BP, NW> walk_p(a.p, a.ldp, t.cp, a.np, a.colsp, a.nk, a.kp, wave, lane, false);
  const Walk<float, QS, BQ, NW> walk_q(a.q, a.ldq, t.cq, a.nq, a.colsq, a.nk, a.kq, wave, lane, false);

  f4 acc[FP][FQ];
#pragma unroll
  for (int i = 0; i < FP; ++i)
#pragma unroll
    for (int j = 0; j < FQ; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};

  // Numbers on their way: load j < LP::kLoads of P, then those of Q.
  constexpr int kLoads = LP::kLoads + LQ::kLoads;
  f4 ahead[kLoads];
  const int write_p = LP::lane_write(wave, lane), write_q = LQ::lane_write(wave, lane);
  const int read_p = LP::lane_read(lane, wp * WP), read_q = LQ::lane_read(lane, wq * WQ);
  auto load = [&](int s, int j) __attribute__((always_inline)) {
    const int step = t.step0 + s, left = walk_p.left(step);
    const bool none = s >= t.nsteps;
    if (j < LP::kLoads) {
      const int r = LP::O::first(wave, j);
      const __amdgpu_buffer_rsrc_t rsrc = descriptor(walk_p, step, none, GATED && gated_up<WP>(r) ? a.p2 : 0);
      const int v = walk_p.offset(GATED ? gated_row<WP>(r) : r, 0, left);
      ahead[j] = __builtin_bit_cast(f4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, v, 0, 0));
    } else {
      const int v = walk_q.offset(LQ::O::first(wave, j - LP::kLoads), 0, left);
      ahead[j] = __builtin_bit_cast(f4, __builtin_amdgcn_raw_buffer_load_b128(descriptor(walk_q, step, none), v, 0, 0));
    }
  };
  auto put = [&](char* buffer, int j) __attribute__((always_inline)) {
    const bool is_p = j < LP::kLoads;
    char* o = is_p ? buffer + LP::write_at(write_p, j) : buffer + LP::kBytes + LQ::write_at(write_q, j - LP::kLoads);
    uint2 w[3];
    split_bf16(ahead[j], w);
#pragma unroll
    for (int n = 0; n < 3; ++n) *reinterpret_cast<uint2*>(o + n * (is_p ? LP::kPlane : LQ::kPlane)) = w[n];
  };

  // What lies behind the rows' ends, and came with their last 16 bytes.
  auto cut_off = [&](char* buffer) __attribute__((always_inline)) {
    const int id = threadIdx.x;
    const bool is_p = id < BP;
    const int r = is_p ? id : id - BP;
    if (is_p ? PS : QS || r >= BQ) return;
    char* row = buffer + (is_p ? 0 : LP::kBytes) + r * 64;
    for (int k = walk_p.left(t.step0 + t.nsteps - 1) / 4; k & 3; ++k)
#pragma unroll
      for (int n = 0; n < 3; ++n)
        *reinterpret_cast<uint16_t*>(row + n * (is_p ? LP::kPlane : LQ::kPlane) + (((k >> 3) ^ LP::spread(r)) << 4) +
                                     (k & 7) * 2) = 0;
  };

#pragma unroll
  for (int j = 0; j < kLoads; ++j) load(0, j);
#pragma unroll
  for (int j = 0; j < kLoads; ++j) {
    put(lds, j);
    load(1, j);
  }
  meet();
  auto body = [&](auto last, int s, const char* now, char* next) __attribute__((always_inline)) {
    b8 fq[FQ][3], fp[2][3];
#pragma unroll
    for (int n = 0; n < 3; ++n) fp[0][n] = LP::frag(now + n * LP::kPlane, read_p, 0);
#pragma unroll
    for (int j = 0; j < FQ; ++j)
#pragma unroll
      for (int n = 0; n < 3; ++n) fq[j][n] = LQ::frag(now + LP::kBytes + n * LQ::kPlane, read_q, j);
    // The next step's numbers and the loads of the one after, between the
    // products, which leave three of four issue slots.
#pragma unroll
    for (int i = 0; i < FP; ++i) {
      if (i + 1 < FP) {
#pragma unroll
        for (int n = 0; n < 3; ++n) fp[(i + 1) & 1][n] = LP::frag(now + n * LP::kPlane, read_p, i + 1);
      }
#pragma unroll
      for (int n = 0; n < 6; ++n) {  // smallest first
        constexpr int kA[6] = {2, 0, 1, 1, 0, 0}, kB[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
        for (int j = 0; j < FQ; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp[i & 1][kA[n]], fq[j][kB[n]], acc[i][j], 0, 0, 0);
      }
      if constexpr (!decltype(last)::value) {
#pragma unroll
        for (int j = i * kLoads / FP; j < (i + 1) * kLoads / FP; ++j) {
          put(next, j);
          load(s + 2, j);
        }
      }
    }
    constexpr int kReadsP = 3 * (PS ? 2 : 1), kReadsQ = 3 * (QS ? 2 : 1), kRow = 6 * FQ, kMma = kRow * FP;
    constexpr int kEach = kMma / kLoads, kFill = (28 * kLoads + kMma - 1) / kMma;
    __builtin_amdgcn_sched_group_barrier(0x100, kReadsP + FQ * kReadsQ, 0);
#pragma unroll
    for (int m = 0; m < kMma; ++m) {
      if (m % kRow == 0 && m / kRow + 1 < FP) __builtin_amdgcn_sched_group_barrier(0x100, kReadsP, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      if (decltype(last)::value) continue;
      __builtin_amdgcn_sched_group_barrier(0x002, kFill, 0);
      if (m % kEach == kEach - 1) {
        __builtin_amdgcn_sched_group_barrier(0x200, 3, 0);
        __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    meet();
  };
  const std::false_type more;
  int s = 0;
  for (; s + 2 < t.nsteps; s += 2) {
    body(more, s, lds, other);
    body(more, s + 1, other, lds);
  }
  char* end = lds;
  if (s + 2 == t.nsteps) {
    body(more, s, lds, other);
    end = other;
  }
  if ((!PS || !QS) && t.ragged) {
    cut_off(end);
    meet();
  }
  body(std::true_type(), 0, end, nullptr);

  // An infinity's lower parts are NaN: a tile whose sums are not all finite is
  // computed again with fp32's own instruction, from fp32 tiles in LDS.  Past
  // the columns of an S operand is whatever lies between its rows: it decides
  // nothing.
  const int end_p = PS ? a.np - t.cp - wp * WP - 4 * (lane >> 4) : BP;
  const int end_q = QS ? a.nq - t.cq - wq * WQ - (lane & 15) : BQ;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < FP; ++i)
#pragma unroll
    for (int j = 0; j < FQ; ++j)
#pragma unroll
      for (int n = 0; n < 4; ++n) bad |= 16 * i + n < end_p && 16 * j < end_q && !(fabsf(acc[i][j][n]) < INFINITY);
  if (any_of_group(bad, reinterpret_cast<int*>(lds))) {
    typedef Operand<float, PS, BP, NW> OP;
    typedef Operand<float, QS, BQ, NW> OQ;
    const Walk<float, PS, BP, NW> again_p(a.p, a.ldp, t.cp, a.np, a.colsp, a.nk, a.kp, wave, lane, true);
    const Walk<float, QS, BQ, NW> again_q(a.q, a.ldq, t.cq, a.nq, a.colsq, a.nk, a.kq, wave, lane, true);
    const int base_p = OP::lane_base(lane, wp * WP), base_q = OQ::lane_base(lane, wq * WQ);
#pragma unroll
    for (int i = 0; i < FP; ++i)
#pragma unroll
      for (int j = 0; j < FQ; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < t.nsteps; ++s) {
      const int step = t.step0 + s, left = again_p.left(step);
#pragma unroll
      for (int j = 0; j < OP::kLoads; ++j) {
        const int r = OP::first(wave, j);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            descriptor(again_p, step, false, GATED && gated_up<WP>(r) ? a.p2 : 0), (lds_void*)(lds + (wave + j * NW) * 1024), 16,
            again_p.offset(GATED ? gated_row<WP>(r) : r, OP::chunk_delta(j), left), 0, 0, 0);
      }
#pragma unroll
      for (int j = 0; j < OQ::kLoads; ++j)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            descriptor(again_q, step, false), (lds_void*)(lds + OP::kBytes + (wave + j * NW) * 1024), 16,
            again_q.offset(OQ::first(wave, j), OQ::chunk_delta(j), left), 0, 0, 0);
      wait_and_meet<0>();
      if (t.ragged && s + 1 == t.nsteps) {
        zero_tail<PS, QS, BP, BQ>(lds, lds + OP::kBytes, left, wave);
        meet();
      }
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int i = 0; i < FP; ++i)
#pragma unroll
          for (int j = 0; j < FQ; ++j)
            acc[i][j] = Num<float>::mma(OP::frag(lds, base_p, i, kk), OQ::frag(lds + OP::kBytes, base_q, j, kk),
                                        acc[i][j]);
      wait_and_meet<0>();
    }
  }
  constexpr int kRoom = WP * WQ * 4 < kRoomBytes ? WP * WQ * 4 : kRoomBytes;
  static_assert(NW / 2 * kRoom <= LP::kBytes + LQ::kBytes, "half of the waves' rooms in an array");
  static_assert(BP * 128 + BQ * 128 <= LP::kBytes + LQ::kBytes, "fp32 tiles in an array");
  f4* const room = reinterpret_cast<f4*>((wave < NW / 2 ? lds : other) + wave % (NW / 2) * kRoom);
  finish_tile<float, WP, WQ, NWP, EPI, GATED>(a, e, t, acc, room, lane, wp, wq);
#endif
}

}  // namespace dense
}  // namespace qcnn
