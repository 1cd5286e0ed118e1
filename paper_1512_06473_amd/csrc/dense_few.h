// Forward products of few rows: y[q][p] = sum_k w[p][k] x[q][k], q < 16 (fp32: 32).
//
// Every weight is used for a handful of products only, so the time is that of
// reading w once, and what matters is how many bytes are on their way.  The
// MFMA operand layout (lane (g, i): row i, 16 bytes at k chunk g) is also a
// good order of reading a row-major matrix: a wave's 16-byte loads take 64
// bytes of 16 rows, kBatch loads in a row 64 kBatch bytes of each.  So w goes
// from memory to the matrix cores' registers, without LDS; x comes the same
// way, out of L2.  A workgroup's 8 waves share groups of 16 p and parts of k:
// with `ks` parts, 8 / ks groups; the parts meet in LDS.  Rows may start at any
// element: the loads are unaligned where they have to be.
//
// Bound by reading w, in bf16 with weights out of cache: 4096 -> 4096 at one
// row 9.5 us (3.5 TB/s; of that 4 us are any launch's), 4096 -> 22016 36.5 us
// (4.9 TB/s), -> 128000 194 us (5.4 TB/s; a read alone reaches 6.2); at 8 and 16
// rows, whose loads share the way out of L2 with the weights', 45 and 50 us.
#pragma once

#include "dense_core.h"

namespace qcnn {
namespace dense {

struct Few {
  const char* p;        // w
  const char* q;        // x
  long long ldp, ldq;   // bytes
  int np, nq, nk;       // nk: elements, any number
  int p2;               // gated: rows from a gate row to its up row
  int ks, units;        // parts of k in a workgroup; 64-byte units of k in each part
  int splits;           // workgroups along k
  float* part;
  long long ldpart;
};

constexpr int kFewWaves = 8, kBatch = 8;

template <typename T>
__device__ __forceinline__ typename Num<T>::Frag load_any(const char* p) {
  typename Num<T>::Frag v;
  __builtin_memcpy(&v, p, 16);
  return v;
}

// FP times 16 weight rows per wave (gated: half of them the gate's, the others
// their up projections).
template <typename T, int FP, int FQ, int EPI, bool GATED>
__global__ __launch_bounds__(64 * kFewWaves) void few_kernel(const Few a, const Epi e) {
  constexpr int kUnit = 64 / (int)sizeof(T), kPer = 16 / (int)sizeof(T);  // k's of a unit, of a lane's load
  __shared__ f4 parts[kFewWaves][FP * FQ][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, i = lane & 15;
  const int groups = kFewWaves / a.ks, kpart = wave % a.ks;
  constexpr int kCols = GATED ? 8 * FP : 16 * FP;  // result columns of a group
  const int tp = blockIdx.x / a.splits, split = blockIdx.x % a.splits;
  const int p_first = (tp * groups + wave / a.ks) * kCols;
  const int units = (a.nk + kUnit - 1) / kUnit;
  const int u0 = min(units, (split * a.ks + kpart) * a.units), u1 = min(units, u0 + a.units);

  f4 acc[FP][FQ];
#pragma unroll
  for (int f = 0; f < FP; ++f)
#pragma unroll
    for (int j = 0; j < FQ; ++j) acc[f][j] = f4{0.f, 0.f, 0.f, 0.f};

  if (p_first < a.np) {
    // Rows past the end read the last one's; what they add up to is not stored.
    const char *rp[FP], *rq[FQ];
#pragma unroll
    for (int f = 0; f < FP; ++f) {
      const long long row = min(p_first + 16 * (GATED ? f % (FP / 2) : f) + i, a.np - 1) + (GATED && f >= FP / 2 ? a.p2 : 0);
      rp[f] = a.p + row * a.ldp + g * 16;
    }
#pragma unroll
    for (int j = 0; j < FQ; ++j) rq[j] = a.q + (long long)min(16 * j + i, a.nq - 1) * a.ldq + g * 16;

    const int full = min(u1, a.nk / kUnit);  // units that end within the row
    int u = u0;
    for (; u + kBatch <= full; u += kBatch) {
      typename Num<T>::Frag vp[kBatch][FP], vq[kBatch][FQ];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const long long at = (long long)(u + b) * 64;
#pragma unroll
        for (int f = 0; f < FP; ++f) vp[b][f] = load_any<T>(rp[f] + at);
#pragma unroll
        for (int j = 0; j < FQ; ++j) vq[b][j] = load_any<T>(rq[j] + at);
      }
#pragma unroll
      for (int b = 0; b < kBatch; ++b)
#pragma unroll
        for (int f = 0; f < FP; ++f)
#pragma unroll
          for (int j = 0; j < FQ; ++j) acc[f][j] = Num<T>::mma(vp[b][f], vq[b][j], acc[f][j]);
    }
    for (; u < u1; ++u) {
      typename Num<T>::Frag vp[FP], vq[FQ];
      const int n = a.nk - u * kUnit - g * kPer;  // k's left for this lane
#pragma unroll
      for (int f = 0; f < FP + FQ; ++f) {
        const char* r = (f < FP ? rp[f < FP ? f : 0] : rq[f < FP ? 0 : f - FP]) + (long long)u * 64;
        typename Num<T>::Frag v;
        if (n >= kPer) {
          v = load_any<T>(r);
        } else {
#pragma unroll
          for (int k = 0; k < kPer; ++k) {
            T t = (T)0.f;
            if (k < n) t = reinterpret_cast<const T*>(r)[k];
            v[k] = t;
          }
        }
        if (f < FP) vp[f < FP ? f : 0] = v;
        else vq[f < FP ? 0 : f - FP] = v;
      }
#pragma unroll
      for (int f = 0; f < FP; ++f)
#pragma unroll
        for (int j = 0; j < FQ; ++j) acc[f][j] = Num<T>::mma(vp[f], vq[j], acc[f][j]);
    }
  }

  // Parts of k meet; the first wave of each group goes on.
  if (a.ks > 1) {
#pragma unroll
    for (int f = 0; f < FP; ++f)
#pragma unroll
      for (int j = 0; j < FQ; ++j) parts[wave][f * FQ + j][lane] = acc[f][j];
    __syncthreads();
    if (kpart == 0)
      for (int w = 1; w < a.ks; ++w)
#pragma unroll
        for (int f = 0; f < FP; ++f)
#pragma unroll
          for (int j = 0; j < FQ; ++j) acc[f][j] += parts[wave + w][f * FQ + j][lane];
  }
  if (kpart != 0 || p_first >= a.np) return;
  const int p = p_first + 4 * g;
#pragma unroll
  for (int j = 0; j < FQ; ++j) {
    const int q = 16 * j + i;
    if constexpr (EPI == kStats) {
      const long long label = q < a.nq ? e.labels[q] - e.class0 : -1;
      float2 t = make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int f = 0; f < FP; ++f) {
        const f4 z = class_logits(a.np, p + 16 * f, acc[f][j], bias_quad<T>(e, a.np, p + 16 * f, e.class0));
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          if (label == p + 16 * f + n && p + 16 * f + n < a.np) e.zlabel[q] = z[n];
          t = join_stat(t, make_float2(z[n], z[n] == -INFINITY ? 0.f : z[n] != z[n] ? z[n] : 1.f));
        }
      }
#pragma unroll
      for (int o = 16; o < 64; o *= 2) t = join_stat(t, make_float2(__shfl_xor(t.x, o), __shfl_xor(t.y, o)));
      if (g == 0 && q < a.nq) e.stat[(long long)(p_first / kCols) * a.nq + q] = t;
    } else {
      if (q >= a.nq) continue;
      if constexpr (GATED) {
#pragma unroll
        for (int f = 0; f < FP / 2; ++f) {
          const int pf = p + 16 * f;
          if constexpr (EPI == kPartial) {
            if (pf < a.np) {
              float* o = a.part + ((long long)split * a.nq + q) * a.ldpart + pf;
              *reinterpret_cast<f4*>(o) = acc[f][j];
              *reinterpret_cast<f4*>(o + a.ldpart / 2) = acc[f + FP / 2][j];
            }
          } else {
            f4 v[1] = {acc[f][j]}, u[1] = {acc[f + FP / 2][j]};
            emit_gated<T, 1>(e, a.np, a.nq, q, 1, pf, v, u, bias_quad<T>(e, a.np, pf), bias_quad<T>(e, a.np, pf, a.np));
          }
        }
      } else {
#pragma unroll
        for (int f = 0; f < FP; ++f) {
          const int pf = p + 16 * f;
          if constexpr (EPI == kPartial) {
            if (pf < a.np) *reinterpret_cast<f4*>(a.part + ((long long)split * a.nq + q) * a.ldpart + pf) = acc[f][j];
          } else if constexpr (EPI == kXgrad) {
            f4 v[1] = {acc[f][j]};
            if (pf < e.ldy) emit_xgrad<T, 1>(e, a.np, a.nq, q, 1, pf, v, bias_quad<T>(e, a.np, pf, e.class0));
          } else {
            f4 v[1] = {acc[f][j]};
            emit_linear<T, 1>(e, a.np, a.nq, q, 1, pf, v, bias_quad<T>(e, a.np, pf));
          }
        }
      }
    }
  }
}

// Weight gradients of few rows: out[t][c] = alpha sum_n d[n][t] x[n][c], at most 32 n.
// Bound by writing out, in fp32 past 16 rows by its own matrix instruction: 16 x
// 4096 -> 16384 in bf16 34 us (4.0 TB/s), in fp32 59 (4.5); 1 x 3968 -> 61184 in
// fp32 178 (5.4), with large tiles, whose epilogues nothing runs beside, 352.
// A wave keeps its 128 columns of x in the
// matrix cores' registers and goes down the rows t, 16 at a time; the columns
// are dealt to the matrix rows so that a lane ends up with 16 bytes in a row,
// and four lanes with 64.  Nothing is staged: d and x come element by element
// out of L2, from rows of any place.
struct Outer {
  const char* x;
  const char* d;
  char* out;               // [rows][cols]
  long long ldx, ldd;      // elements
  int n, cols, rows, per;  // per: rows of a wave, whole 16
  const float* alpha;      // or null
};

template <typename T>
__global__ __launch_bounds__(256) void outer_kernel(const Outer a) {
  typedef typename Num<T>::Frag Frag;
  constexpr int kV = 16 / (int)sizeof(T), kK = 4 * kV, kParts = 32 / kK, kQ = kV / 4, kTiles = 8;
  const int lane = threadIdx.x & 63, g = lane >> 4, i = lane & 15;
  const int c0 = (blockIdx.x * 4 + (threadIdx.x >> 6)) * 16 * kTiles;
  const int t1 = min(a.rows, (int)(blockIdx.y + 1) * a.per);
  if (c0 >= a.cols) return;
  // Elements n of one column, zeros past the last.
  auto column = [&](const char* p, long long ld, int c, int end, Frag (&f)[kParts]) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < kParts; ++k)
#pragma unroll
      for (int e = 0; e < kV; ++e) {
        const int n = k * kK + g * kV + e;
        T v = (T)0.f;
        if (n < a.n && c < end) v = reinterpret_cast<const T*>(p)[n * ld + c];
        f[k][e] = v;
      }
  };
  Frag x[kTiles][kParts], d[kParts];
#pragma unroll
  for (int j = 0; j < kTiles; ++j) {
    const int m = j / kQ;  // 16 kQ columns: 4 kQ of each lane group
    column(a.x, a.ldx, c0 + 16 * kQ * m + 4 * kQ * (i >> 2) + 4 * (j % kQ) + (i & 3), a.cols, x[j]);
  }
  const float alpha = a.alpha ? *a.alpha : 1.f;
  int t = blockIdx.y * a.per;
  column(a.d, a.ldd, t + i, t1, d);
  for (; t < t1; t += 16) {
    f4 acc[kTiles];
#pragma unroll
    for (int j = 0; j < kTiles; ++j) {
      acc[j] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < kParts; ++k)
        if (k == 0 || k * kK < a.n) acc[j] = Num<T>::mma(x[j][k], d[k], acc[j]);
    }
    column(a.d, a.ldd, t + 16 + i, t1, d);
    if (t + i >= t1) continue;
    T* o = reinterpret_cast<T*>(a.out) + (long long)(t + i) * a.cols;
#pragma unroll
    for (int m = 0; m < kTiles / kQ; ++m) {
      const int c = c0 + 16 * kQ * m + kV * g;
      f4 v[kQ];
#pragma unroll
      for (int k = 0; k < kQ; ++k) v[k] = acc[m * kQ + k] * alpha;
      if (c < a.cols) store_wide(o + c, a.cols - c, v);
    }
  }
}

// Input gradients of few rows in fp32: y[n][c] = sum_t d[n][t] w[t][c], n <= 32.
// Bound by reading w (1 x 3968 -> 61184: 179 us, 5.4 TB/s, with large tiles 289),
// past 16 rows by fp32's own matrix instruction (32 rows 268, tiles, at 33,
// 286; 4096 -> 16384 77 and 78).  A lane's 16 bytes of a row are four columns,
// each for a matrix instruction of its own, which therefore takes every fourth
// of 64 columns; 16 rows t are four loads.  A workgroup's waves have parts of
// t, which meet in LDS.
struct Thin {
  const float* w;
  const float* d;
  long long ldw, ldd;  // elements
  int rows, cols, n;   // rows: of w
  int units, splits;   // 16 rows each, of a wave; workgroups along t
  float* part;
  long long ldpart;
};

template <int FQ, int EPI>
static __global__ __launch_bounds__(64 * kFewWaves) void thin_kernel(const Thin a, const Epi e) {
  __shared__ f4 parts[kFewWaves][4 * FQ][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, i = lane & 15;
  const int tp = blockIdx.x / a.splits, split = blockIdx.x % a.splits, c0 = tp * 64, c = c0 + 4 * i;
  const int all = (a.rows + 15) / 16;
  const int u0 = min(all, (split * kFewWaves + wave) * a.units), u1 = min(all, u0 + a.units);
  f4 acc[4][FQ];
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int j = 0; j < FQ; ++j) acc[k][j] = f4{0.f, 0.f, 0.f, 0.f};
  auto multiply = [&](const f4 (&w)[4], const f4 (&d)[FQ]) __attribute__((always_inline)) {
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int j = 0; j < FQ; ++j)
          acc[k][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[m][k], d[j][m], acc[k][j], 0, 0, 0);
  };
  // Past the last n, column or row: zeros.
  auto load = [&](int u, bool whole, f4 (&w)[4], f4 (&d)[FQ]) __attribute__((always_inline)) {
    const int t = 16 * u + 4 * g;
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      w[m] = f4{0.f, 0.f, 0.f, 0.f};
      if (whole || t + m < a.rows) w[m] = load_quad(a.w + (t + m) * a.ldw + c, a.cols - c);
    }
#pragma unroll
    for (int j = 0; j < FQ; ++j) {
      const int n = 16 * j + i;
      d[j] = f4{0.f, 0.f, 0.f, 0.f};
      if (n < a.n) d[j] = load_quad(a.d + n * a.ldd + t, whole ? 4 : a.rows - t);
    }
  };
  const int full = min(u1, a.rows / 16);
  int u = u0;
  for (; u + 2 <= full; u += 2) {
    f4 w[2][4], d[2][FQ];
#pragma unroll
    for (int b = 0; b < 2; ++b) load(u + b, true, w[b], d[b]);
#pragma unroll
    for (int b = 0; b < 2; ++b) multiply(w[b], d[b]);
  }
  for (; u < u1; ++u) {
    f4 w[4], d[FQ];
    load(u, false, w, d);
    multiply(w, d);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int j = 0; j < FQ; ++j) parts[wave][k * FQ + j][lane] = acc[k][j];
  __syncthreads();
  if (wave > 0) return;
  for (int o = 1; o < kFewWaves; ++o)
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int j = 0; j < FQ; ++j) acc[k][j] += parts[o][k * FQ + j][lane];
#pragma unroll
  for (int j = 0; j < FQ; ++j) {
    const int n = 16 * j + i;
    if (n >= a.n) continue;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int p = c0 + 16 * g + 4 * r;
      const f4 v = {acc[0][j][r], acc[1][j][r], acc[2][j][r], acc[3][j][r]};
      if constexpr (EPI == kPartial) {
        if (p < a.cols) *reinterpret_cast<f4*>(a.part + ((long long)split * a.n + n) * a.ldpart + p) = v;
      } else {
        f4 v1[1] = {v};
        emit_linear<float, 1>(e, a.cols, a.n, n, 1, p, v1, f4{0.f, 0.f, 0.f, 0.f});
      }
    }
  }
}

}  // namespace dense
}  // namespace qcnn
