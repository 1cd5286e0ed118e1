// The dense layers for one element type: planning, the kernels around the
// products, and the calls of qcnn_internal.h.  Included once per type
// (dense_f32.hip, dense_bf16.hip, dense_f16.hip).
#pragma once

#include "dense_few.h"

namespace qcnn {
namespace dense {

inline size_t align256(size_t b) { return (b + 255) & ~(size_t)255; }

// Parts of one call's workspace.
struct Layout {
  size_t bytes = 0;
  size_t add(size_t b) {
    const size_t at = bytes;
    bytes += align256(b);
    return at;
  }
};

template <typename T>
constexpr int pad16(int n) {  // elements, to whole 16 bytes
  constexpr int u = 16 / (int)sizeof(T);
  return (n + u - 1) / u * u;
}

// Rows that the products read where they are: they start at whole dwords
// (always, in fp32).
template <typename T>
bool direct(const void* p, long long ld, int cols) {
  return ((uintptr_t)p & 3) == 0 && ld * sizeof(T) % 4 == 0 && cols * sizeof(T) % 4 == 0;
}

// ------------------------------------------------------ kernels around them

// [rows][cols] with row stride ld -> rows of ldo, zeros past cols: a thread
// writes 16 bytes.
template <typename T>
__global__ __launch_bounds__(256) void pad_kernel(const T* __restrict__ src, long long ld, int rows, int cols,
                                                  T* __restrict__ dst, int ldo) {
  constexpr int kV = 16 / (int)sizeof(T);
  const long long per = ldo / kV, all = rows * per;
  for (long long id = blockIdx.x * 256LL + threadIdx.x; id < all; id += gridDim.x * 256LL) {
    const long long r = id / per;
    const int c = (int)(id % per) * kV;
    const T* s = src + r * ld + c;
    struct alignas(16) { T v[kV]; } t;
    if (cols - c >= kV) {
      __builtin_memcpy(&t, s, 16);
    } else {
#pragma unroll
      for (int i = 0; i < kV; ++i) t.v[i] = c + i < cols ? s[i] : (T)0.f;
    }
    __builtin_memcpy(__builtin_assume_aligned(dst + r * ldo + c, 16), &t, 16);
  }
}

// dz = dy act'(pre) (gated: gate and up halves) and its sums over rows: bound by
// HBM (gated, 4096 x 11008 in bf16, 451 MB: 104 us, 4.3 TB/s).  A
// thread has 16 bytes of columns and goes down `chunk` rows, the loads of 4 at
// a time; the sums of a block's rows go to part[blockIdx.y][columns of dz],
// joined by colsum_kernel: the order of the additions is the same in every run.
// dz is rounded to T for the products, whose instructions take 16-bit operands
// (two parts of it would double their time); the sums are of dz unrounded.
struct Slope {
  const void* dy;
  const void* pre;
  void* dz;     // null: only the sums
  float* part;  // null: no sums
  void* sums;   // T: the finished sums, where one block row has all rows
  const float* alpha;
  long long lddy, ldpre, lddz;
  int rows, cols, chunk, act;  // cols: of dy
};

// With GROUPS, that many groups of a block's threads share its rows.
template <typename T, bool GATED, int GROUPS>
__global__ __launch_bounds__(256) void slope_kernel(const Slope a) {
  constexpr int kV = 16 / (int)sizeof(T), kQ = kV / 4, kWide = 256 / GROUPS, kSums = GATED ? 2 : 1;
  __shared__ f4 sums[GROUPS > 1 ? GROUPS - 1 : 1][kSums][kQ][kWide];
  const int lane = threadIdx.x % kWide, group = threadIdx.x / kWide;
  const int p = (blockIdx.x * kWide + lane) * kV;
  const long long width = GATED ? 2LL * a.cols : a.cols;
  const int r0 = blockIdx.y * a.chunk + group, r1 = min(a.rows, (int)(blockIdx.y + 1) * a.chunk);
  if (p >= a.cols) {
    // the zeros between the columns and the row's end, fewer than kV
    const long long col = width + (p - (a.cols + kV - 1) / kV * kV);
    if (a.dz && p < a.cols + kV)
      for (int r = r0; r < r1; r += GROUPS)
        for (int i = 0; i < kV; ++i)
          if (col + i < a.lddz) static_cast<T*>(a.dz)[r * a.lddz + col + i] = (T)0.f;
    if (GROUPS == 1) return;
  }
  f4 s0[kQ], s1[kQ];
#pragma unroll
  for (int k = 0; k < kQ; ++k) s0[k] = s1[k] = f4{0.f, 0.f, 0.f, 0.f};
  const int n = a.cols - p;
#pragma unroll 4
  for (int r = r0; r < (GROUPS > 1 && n <= 0 ? 0 : r1); r += GROUPS) {
    f4 dy[kQ], g[kQ], u[kQ];
    load_wide(static_cast<const T*>(a.dy) + r * a.lddy + p, n, dy);
    if constexpr (GATED) {
      const T* z = static_cast<const T*>(a.pre) + r * a.ldpre + p;
      load_wide(z, n, g);
      load_wide(z + a.cols, n, u);
#pragma unroll
      for (int k = 0; k < kQ; ++k) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float d = dy[k][i], z = g[k][i];
          g[k][i] = d * u[k][i] * act_slope<T>(a.act, z);
          u[k][i] = d * act_value<T>(a.act, z);
        }
        s0[k] += g[k];
        s1[k] += u[k];
      }
      if (a.dz) {
        T* o = static_cast<T*>(a.dz) + r * a.lddz + p;
        store_wide(o, n, g);
        store_wide(o + a.cols, n, u);
      }
    } else {
      if (a.act != QCNN_ACT_NONE) {
        load_wide(static_cast<const T*>(a.pre) + r * a.ldpre + p, n, g);
#pragma unroll
        for (int k = 0; k < kQ; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i) dy[k][i] *= act_slope<T>(a.act, g[k][i]);
      }
      if (a.dz) store_wide(static_cast<T*>(a.dz) + r * a.lddz + p, n, dy);
#pragma unroll
      for (int k = 0; k < kQ; ++k) s0[k] += dy[k];
    }
  }
  if constexpr (GROUPS > 1) {
    if (group > 0) {
#pragma unroll
      for (int k = 0; k < kQ; ++k) {
        sums[group - 1][0][k][lane] = s0[k];
        if (GATED) sums[group - 1][kSums - 1][k][lane] = s1[k];
      }
    }
    __syncthreads();
    if (group > 0 || n <= 0) return;
#pragma unroll
    for (int i = 0; i < GROUPS - 1; ++i)
#pragma unroll
      for (int k = 0; k < kQ; ++k) {
        s0[k] += sums[i][0][k][lane];
        if (GATED) s1[k] += sums[i][kSums - 1][k][lane];
      }
  }
  if (a.sums) {
    T* o = static_cast<T*>(a.sums) + p;
    const float alpha = a.alpha ? *a.alpha : 1.f;
#pragma unroll
    for (int k = 0; k < kQ; ++k) {
      store_quad(o + 4 * k, s0[k] * alpha, n - 4 * k);
      if (GATED) store_quad(o + a.cols + 4 * k, s1[k] * alpha, n - 4 * k);
    }
  } else if (a.part) {
    float* o = a.part + blockIdx.y * width + p;
#pragma unroll
    for (int k = 0; k < kQ; ++k) {
      store_quad(o + 4 * k, s0[k], n - 4 * k);
      if (GATED) store_quad(o + a.cols + 4 * k, s1[k], n - 4 * k);
    }
  }
}

// out[c] = alpha sum_r part[r][c]: 64 columns by 16 groups of rows (512 rows of
// 4096 sums: 7.0 us with 4 groups, 4.8 with 16).
template <typename T>
__global__ __launch_bounds__(1024) void colsum_kernel(const float* __restrict__ part, int rows, long long width,
                                                      const float* alpha, T* __restrict__ out) {
  constexpr int kGroups = 16;
  __shared__ float group[kGroups][64];
  const int lane = threadIdx.x & 63, g = threadIdx.x >> 6;
  const long long c = blockIdx.x * 64LL + lane;
  float s = 0.f;
  if (c < width) {
#pragma unroll 8
    for (int r = g; r < rows; r += kGroups) s += part[r * width + c];
  }
  group[g][lane] = s;
  for (int n = kGroups / 2; n > 0; n /= 2) {
    __syncthreads();
    if (g < n) group[g][lane] = s += group[g + n][lane];
  }
  if (g == 0 && c < width) out[c] = (T)(alpha ? s * *alpha : s);
}

// Rows of a block: all of a few, which saves the kernel that joins the sums,
// and which its groups of threads share (gated, 11 x 10624 in bf16: 37 us with
// one group, 9.7 with 8); else enough blocks for the chip, and at most 512 rows
// of sums.
constexpr int kFewSlopes = 32;
inline int slope_chunk(int rows) { return rows <= kFewSlopes ? rows : std::max(4, ceil_div(rows, 512)); }

// dz and, with dbias, alpha times its sums over rows.
template <typename T, bool GATED>
hipError_t run_slope(Slope a, void* dbias, const float* alpha, hipStream_t st) {
  const int chunks = ceil_div(a.rows, a.chunk), width = GATED ? 2 * a.cols : a.cols;
  const int threads = ceil_div(a.cols, 16 / (int)sizeof(T)) + (a.dz && a.lddz > width);
  if (chunks == 1) {
    a.sums = dbias;
    a.alpha = alpha;
  }
  if (a.rows <= kFewSlopes) slope_kernel<T, GATED, 8><<<dim3(ceil_div(threads, 32), chunks), 256, 0, st>>>(a);
  else slope_kernel<T, GATED, 1><<<dim3(ceil_div(threads, 256), chunks), 256, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !dbias || chunks == 1) return e;
  colsum_kernel<T><<<ceil_div(width, 64), 1024, 0, st>>>(a.part, chunks, width, alpha, static_cast<T*>(dbias));
  return hipGetLastError();
}

// Sums of the parts of k, then the epilogue: a thread per quad of a row, or,
// with many parts (few outputs, that is), G threads that take every G-th part
// (24 x 4096 -> 500 gated, 32 parts: 25 us with one, 11 with four).
template <typename T, int EPI, int G>
__global__ __launch_bounds__(256) void finish_kernel(const float* __restrict__ part, int splits, long long ldpart,
                                                     int np, int nq, int quads_of_row, const Epi e) {
  constexpr int kQuads = 256 / G, kSums = EPI == kGated ? 2 : 1;
  __shared__ f4 sums[G > 1 ? G - 1 : 1][kSums][kQuads];
  const int t = threadIdx.x % kQuads, group = threadIdx.x / kQuads;
  const long long id = blockIdx.x * (long long)kQuads + t;
  const int q = (int)(id / quads_of_row), p = (int)(id % quads_of_row) * 4;
  const long long each = (long long)nq * ldpart;
  const float* s = part + q * ldpart + p;
  f4 v = {0.f, 0.f, 0.f, 0.f}, u = v;
  if (q < nq && p < np) {
#pragma unroll 8
    for (int i = group; i < splits; i += G) {
      v += *reinterpret_cast<const f4*>(s + i * each);
      if (EPI == kGated) u += *reinterpret_cast<const f4*>(s + i * each + ldpart / 2);
    }
  }
  if constexpr (G > 1) {
    if (group > 0) {
      sums[group - 1][0][t] = v;
      if (EPI == kGated) sums[group - 1][kSums - 1][t] = u;
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int i = 0; i < G - 1; ++i) {
      v += sums[i][0][t];
      if (EPI == kGated) u += sums[i][kSums - 1][t];
    }
  }
  if (q >= nq) return;
  f4 v1[1] = {v}, u1[1] = {u};
  const f4 bias = bias_quad<T>(e, np, p, EPI == kXgrad ? e.class0 : 0);
  if constexpr (EPI == kGated) emit_gated<T, 1>(e, np, nq, q, 1, p, v1, u1, bias, bias_quad<T>(e, np, p, np));
  else if constexpr (EPI == kXgrad) emit_xgrad<T, 1>(e, np, nq, q, 1, p, v1, bias);
  else emit_linear<T, 1>(e, np, nq, q, 1, p, v1, bias);
}

__device__ __forceinline__ void write_loss(float2 t, float zlabel, long long label, int classes, float* loss,
                                           float* lse) {
  const float l = t.x + logf(t.y);
  *lse = l;
  *loss = label < 0 ? 0.f : label >= classes ? NAN : l - zlabel;
}

// The same for the loss: a workgroup per row and `width` classes, which
// finishes the row where that is all of them, else leaves a slot's statistics.
template <typename T>
__global__ __launch_bounds__(256) void finish_loss_kernel(const float* __restrict__ part, int splits,
                                                          long long ldpart, int np, int nq, int width, const Epi e) {
  __shared__ float2 stats[4];
  __shared__ float zlabel;
  const int q = blockIdx.x, end = min(np, (int)(blockIdx.y + 1) * width);
  const long long label = e.labels[q], each = (long long)nq * ldpart;
  float2 t = make_float2(-INFINITY, 0.f);
  for (int p = blockIdx.y * width + threadIdx.x * 4; p < end; p += 1024) {
    f4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int i = 0; i < splits; ++i) z += *reinterpret_cast<const f4*>(part + i * each + q * ldpart + p);
    z = class_logits(np, p, z, bias_quad<T>(e, np, p, e.class0));
    const float m = fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3]));
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (label == p + i && p + i < np) {
        zlabel = z[i];
        if (e.stat) e.zlabel[q] = z[i];
      }
      sum += z[i] == -INFINITY ? 0.f : __expf(z[i] - m);
    }
    t = join_stat(t, make_float2(m, sum));
  }
#pragma unroll
  for (int o = 1; o < 64; o *= 2) t = join_stat(t, make_float2(__shfl_xor(t.x, o), __shfl_xor(t.y, o)));
  if ((threadIdx.x & 63) == 0) stats[threadIdx.x >> 6] = t;
  __syncthreads();
  if (threadIdx.x) return;
  t = join_stat(join_stat(stats[0], stats[1]), join_stat(stats[2], stats[3]));
  if (e.stat) e.stat[(long long)blockIdx.y * nq + q] = t;
  else write_loss(t, zlabel, label, e.classes, e.loss + q, e.lse_out + q);
}

// Joins the slots' maxima and sums of each row: ROWS rows by THREADS / ROWS
// threads, each of which takes every so many-th slot.
template <int ROWS, int THREADS>
static __global__ __launch_bounds__(THREADS) void loss_kernel(const float2* __restrict__ stat,
                                                          const float* __restrict__ zlabel,
                                                          const long long* __restrict__ labels, int slots, int nq,
                                                          int classes, float* __restrict__ loss,
                                                          float* __restrict__ lse) {
  constexpr int kEach = THREADS / ROWS;
  __shared__ float2 part[kEach][ROWS];
  const int c = threadIdx.x % ROWS, r = threadIdx.x / ROWS, q = blockIdx.x * ROWS + c;
  float2 t = make_float2(-INFINITY, 0.f);
  if (q < nq) {
#pragma unroll 4
    for (int s = r; s < slots; s += kEach) t = join_stat(t, stat[(long long)s * nq + q]);
  }
  part[r][c] = t;
  for (int n = kEach / 2; n > 0; n /= 2) {
    __syncthreads();
    if (r < n) part[r][c] = join_stat(part[r][c], part[r + n][c]);
  }
  if (r != 0 || q >= nq) return;
  write_loss(part[0][c], zlabel[q], labels[q], classes, loss + q, lse + q);
}

// out[0] = the largest finite |dloss| of a counted row (1 if there is none or
// it is 0; 2^-110 at least, so that gain / out[0] is finite and out[1] a normal
// number), out[1] = out[0] / gain: what products with d are multiplied by.
static __global__ __launch_bounds__(1024) void dmax_kernel(const float* __restrict__ dloss,
                                                    const long long* __restrict__ labels, int n, float gain,
                                                    float* __restrict__ out) {
  __shared__ float part[16];
  float m = 0.f;
  for (int i = threadIdx.x; i < n; i += 1024) {
    const float v = fabsf(dloss[i]);
    if (labels[i] >= 0 && v < INFINITY) m = fmaxf(m, v);
  }
#pragma unroll
  for (int o = 1; o < 64; o *= 2) m = fmaxf(m, __shfl_xor(m, o));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
  __syncthreads();
  if (threadIdx.x) return;
  for (int i = 1; i < 16; ++i) m = fmaxf(m, part[i]);
  m = m == 0.f ? 1.f : fmaxf(m, 0x1p-110f);
  out[0] = m;
  out[1] = m / gain;
}

// ---------------------------------------------------------------- planning

// A product's tiles and parts of k.
struct Cut {
  int big;  // large tiles of 8 waves: 256 x 256, fp32 256 x 128; else 128 x 128
  int main_p, main_q;  // large tiles along one axis (0: all), the rest in small ones
  int splits, steps;
  size_t part_bytes;
  long long ldpart;
};

// Results of a tile along p and q.
template <typename T>
struct Edge {
  static constexpr int p(bool big, bool gated) { return (big ? 256 : 128) / (gated ? 2 : 1); }
  static constexpr int q(bool big) { return big && sizeof(T) == 2 ? 256 : 128; }
  static constexpr int slots(bool big) { return big && sizeof(T) == 4 ? 4 : 2; }  // waves along p
  static long long tiles(int np, int nq, bool gated, bool big) {
    return (long long)ceil_div(np, p(big, gated)) * ceil_div(nq, q(big));
  }
};

// The cut that should take the least time: the rounds of tiles that the busiest
// CU goes through, times what one takes: `step` for each step and `ends` for
// its first loads and its epilogue.  A CU holds one tile, or two small 16-bit
// ones, which hide each other's waits.  Measured in us on whole products (64 to
// 1024 tiles, k from 64 to 4096), step and ends: 16-bit types, a small tile
// alone 0.55 to 0.75 and 4, two 1.05 and 6, a large one (the work of four) 1.6
// and 10; fp32, a small tile 1.4 and 6, a large one (of two) 2.35 and 9.  Parts
// of k are written and read once in fp32 (5 TB/s) and take a second kernel.
// Against the best of all measured cuts of ten shapes the choice loses 0 to 12
// %; one fixed rule (256 workgroups) lost up to 1.4 times, and a model without
// the ends 1.2 times where k is short (774 x 100 -> 104192: 107 us).
// A last round of large tiles that would leave most CUs idle goes in small ones
// (1999 rows to 50001 classes: 6.1 rounds).  rows_alike: not along q.
template <typename T>
Cut cut_of(int np, int nq, int nk, bool gated, bool rows_alike = false) {
  constexpr bool f32 = sizeof(T) == 4;
  const int all = ceil_div(nk * (int)sizeof(T), 128);
  auto large_rounds = [&](long long groups, int steps) {
    return (groups + 255) / 256 * (f32 ? 2.35 * steps + 9. : 1.6 * steps + 10.);
  };
  auto small_rounds = [&](long long groups, int steps) {
    if (f32) return (groups + 255) / 256 * (1.4 * steps + 6.);
    const double one = 0.62 * steps + 4., two = 1.05 * steps + 6.;
    const long long rest = groups % 512;
    return groups / 512 * two + (rest > 256 ? two : rest ? one : 0.);
  };
  Cut best = {};
  double least = 1e300;
  for (int big = 0; big < 2; ++big) {
    const long long tiles = Edge<T>::tiles(np, nq, gated, big);
    for (int n = 1; n <= 32 && (n == 1 || (n <= all / 2 && tiles * n <= 1024)); ++n) {
      const int steps = ceil_div(all, n), splits = ceil_div(all, steps);
      const long long groups = tiles * splits;
      const double t = (big ? large_rounds(groups, steps) : small_rounds(groups, steps)) +
                       (splits > 1 ? 4. + 1.6e-6 * splits * nq * np * (gated ? 2 : 1) : 0.);
      if (t >= least) continue;
      least = t;
      best.big = big;
      best.splits = splits;
      best.steps = steps;
    }
  }
  const int wide = Edge<T>::p(true, gated), high = Edge<T>::q(true), tps = ceil_div(np, wide), tqs = ceil_div(nq, high);
  const long long rounds = (long long)tps * tqs / 256;
  for (int axis = 0; axis < (rows_alike ? 1 : 2) && rounds > 0; ++axis) {
    const int mine = axis ? tqs : tps, other = axis ? tps : tqs;
    const int main = (int)(rounds * 256 / other);
    if (main < 1 || main >= mine) continue;
    const long long tail = axis ? Edge<T>::tiles(np, nq - main * high, gated, false)
                                : Edge<T>::tiles(np - main * wide, nq, gated, false);
    const double t = large_rounds((long long)main * other, all) + small_rounds(tail, all) + 4.;
    if (t >= least) continue;
    least = t;
    best.big = best.splits = 1;
    best.steps = all;
    best.main_p = axis ? 0 : main;
    best.main_q = axis ? main : 0;
  }
  best.ldpart = (long long)ceil_div(np, 4) * 4 * (gated ? 2 : 1);
  best.part_bytes = best.splits > 1 ? (size_t)best.splits * nq * best.ldpart * 4 : 0;
  return best;
}

// The tiles of outputs [p0, p1) x [q0, q1).
template <typename T, bool PS, bool QS, int EPI, bool GATED>
hipError_t launch_tiles(Prod a, const Epi& e, bool big, int p0, int p1, int q0, int q1, hipStream_t st) {
  a.p0 = p0;
  a.p1 = p1;
  a.q0 = q0;
  a.q1 = q1;
  LaunchTimer timer;
  const dim3 grid((unsigned)(Edge<T>::tiles(p1 - p0, q1 - q0, GATED, big) * a.splits));
  if constexpr (sizeof(T) == 4) {
    if (big)
      return timed_launch(&timer, product_f32_kernel<PS, QS, 256, 128, 64, 64, EPI, GATED>, grid, dim3(512), 0u, st, a, e);
    return timed_launch(&timer, product_f32_kernel<PS, QS, 128, 128, 64, 32, EPI, GATED>, grid, dim3(512), 0u, st, a, e);
  } else {
    if (big)
      return timed_launch(&timer, product_kernel<T, PS, QS, 256, 256, 128, 64, 2, EPI, GATED>, grid, dim3(512), 0u, st, a, e);
    if (grid.x <= 256)  // one workgroup per CU: its LDS holds four steps (1024 x 4096 -> 1024 bf16: 45 us, with four 39)
      return timed_launch(&timer, product_kernel<T, PS, QS, 128, 128, 64, 64, 4, EPI, GATED>, grid, dim3(256), 0u, st, a, e);
    return timed_launch(&timer, product_kernel<T, PS, QS, 128, 128, 64, 64, 2, EPI, GATED>, grid, dim3(256), 0u, st, a, e);
  }
}

template <typename T, bool PS, bool QS, int EPI, bool GATED>
hipError_t launch_product(Prod a, const Epi& e, const Cut& c, hipStream_t st) {
  const int p = c.main_p * Edge<T>::p(true, GATED), q = c.main_q * Edge<T>::q(true);
  if (!p && !q) return launch_tiles<T, PS, QS, EPI, GATED>(a, e, c.big, 0, a.np, 0, a.nq, st);
  const hipError_t err = launch_tiles<T, PS, QS, EPI, GATED>(a, e, true, 0, p ? p : a.np, 0, q ? q : a.nq, st);
  if (err != hipSuccess) return err;
  if (p) a.slot0 = Edge<T>::slots(true) * c.main_p;
  return launch_tiles<T, PS, QS, EPI, GATED>(a, e, false, p, a.np, q, a.nq, st);
}

// Classes of a workgroup of finish_loss_kernel; slots of statistics that it
// leaves (none if it finishes the rows).
inline int loss_width(int np) { return np <= 4096 ? 4096 : 1024; }
inline int loss_slots(int np) { return np <= 4096 ? 0 : ceil_div(np, 1024); }

// After kPartial: the parts' sums and the epilogue.
template <typename T, int EPI>
hipError_t finish(int np, int nq, const Epi& e, const Cut& c, const float* part, hipStream_t st) {
  if constexpr (EPI == kStats) {
    const int width = loss_width(np);
    finish_loss_kernel<T><<<dim3(nq, ceil_div(np, width)), 256, 0, st>>>(part, c.splits, c.ldpart, np, nq, width, e);
  } else {
    const int per = EPI == kXgrad ? (int)(e.ldy / 4) : ceil_div(np, 4);
    const long long n = (long long)per * nq;
    if (c.splits >= 8)
      finish_kernel<T, EPI, 4><<<(unsigned)((n + 63) / 64), 256, 0, st>>>(part, c.splits, c.ldpart, np, nq, per, e);
    else
      finish_kernel<T, EPI, 1><<<(unsigned)((n + 255) / 256), 256, 0, st>>>(part, c.splits, c.ldpart, np, nq, per, e);
  }
  return hipGetLastError();
}

template <typename T, bool PS, bool QS, int EPI, bool GATED>
hipError_t run_product(Prod a, const Epi& e, const Cut& c, float* part, hipStream_t st) {
  a.splits = c.splits;
  a.steps = c.steps;
  a.part = part;
  a.ldpart = c.ldpart;
  if (c.splits == 1) return launch_product<T, PS, QS, EPI, GATED>(a, e, c, st);
  const hipError_t err = launch_product<T, PS, QS, kPartial, GATED>(a, e, c, st);
  return err != hipSuccess ? err : finish<T, EPI>(a.np, a.nq, e, c, part, st);
}

// Whether a product's operands along k have to end with whole 16 bytes.
template <typename T>
bool ends_whole(const Cut& c) { return sizeof(T) == 2 && c.big; }

// Slots of a product that is not split: one per wave along p (the same for
// every row, so none of its rows may go in tiles of another size).
template <typename T>
int stat_slots(const Cut& c, int np) {
  typedef Edge<T> E;
  if (c.main_p)
    return E::slots(true) * c.main_p + E::slots(false) * ceil_div(np - c.main_p * E::p(true, false), E::p(false, false));
  return E::slots(c.big) * ceil_div(np, E::p(c.big, false));
}

// A forward product: the tiles, or for few rows the kernel that streams the
// weights.  At 24 rows (4096 -> 4096, 9216 -> 4096, 4096 -> 22016) it takes 16,
// 29 and 58 us in bf16, the tiles 15, 23 and 49; in fp32 27, 50 and 109 against
// 34, 62 and 160 (at 33 rows 35, 68 and 152 against 34, 61 and 158).
template <typename T>
constexpr int kFewRows = sizeof(T) == 4 ? 32 : 16;

template <typename T>
struct Forward : Cut {
  bool few, wide_ = false;
  int ks, slots;  // slots: of kStats, 0 where the parts' sums go straight to the loss
  int np, nq, nk;
  bool gated;
  Forward(int np_, int nq_, int nk_, bool gated_, bool rows_alike = false)
      : np(np_), nq(nq_), nk(nk_), gated(gated_) {
    few = nq <= kFewRows<T>;
    if (!few) {
      static_cast<Cut&>(*this) = cut_of<T>(np, nq, pad16<T>(nk), gated, rows_alike);
      slots = splits > 1 ? loss_slots(np) : stat_slots<T>(*this, np);
      return;
    }
    // A wave's 16 rows (32 past 8 rows of x and where there are many, whose
    // loads of x then serve twice the weights: 50 against 55 us at 16 x 4096
    // -> 22016) by 8192 waves' worth of parts of k within the workgroups:
    // 4096 -> 22016 in bf16 took 53 us with 2048 waves, 38 with 4096, 37 with
    // 8192.  A second kernel that joins workgroups costs 2 us: only for layers
    // that would leave most CUs without a workgroup.
    wide_ = !gated && (nq > 16 || (nq > 8 && np >= 16384));
    const long long groups = ceil_div(np, cols());
    const int all = ceil_div(nk * (int)sizeof(T), 64);
    for (ks = 1; ks < kFewWaves && groups * ks < 8192 && all / (2 * ks) >= kBatch; ks *= 2) {}
    int parts = groups * ks >= 2048 ? 1 : (int)std::min<long long>(4096 / (groups * ks), all / (ks * kBatch));
    if (parts < 1) parts = 1;
    steps = ceil_div(all, ks * parts);
    splits = ceil_div(all, ks * steps);
    ldpart = (long long)ceil_div(np, 4) * 4 * (gated ? 2 : 1);
    part_bytes = splits > 1 ? (size_t)splits * nq * ldpart * 4 : 0;
    slots = splits > 1 ? loss_slots(np) : ceil_div(np, cols());
  }

  int cols() const { return wide_ ? 32 : 16; }  // result columns of a wave
  bool whole() const { return !few && ends_whole<T>(*this); }

  template <int EPI, bool GATED>
  hipError_t launch_few(const Few& a, const Epi& e, hipStream_t st) const {
    LaunchTimer timer;
    const dim3 grid((unsigned)(ceil_div(ceil_div(np, cols()), kFewWaves / ks) * splits)), block(64 * kFewWaves);
    if constexpr (kFewRows<T> > 16)
      if (nq > 16) return timed_launch(&timer, few_kernel<T, 2, 2, EPI, GATED>, grid, block, 0u, st, a, e);
    if constexpr (!GATED)
      if (!wide_) return timed_launch(&timer, few_kernel<T, 1, 1, EPI, GATED>, grid, block, 0u, st, a, e);
    return timed_launch(&timer, few_kernel<T, 2, 1, EPI, GATED>, grid, block, 0u, st, a, e);
  }

  // w and x: rows of ldw and ldx bytes; as the tiles read them unless `few`,
  // with `stored` columns in both.
  template <int EPI, bool GATED>
  hipError_t run(const char* w, long long ldw, const char* x, long long ldx, int stored, const Epi& e, float* part,
                 hipStream_t st) const {
    if (!few) {
      Prod a = {};
      a.p = w;
      a.q = x;
      a.ldp = ldw;
      a.ldq = ldx;
      a.np = a.p2 = np;
      a.nq = nq;
      a.nk = stored;
      return run_product<T, false, false, EPI, GATED>(a, e, *this, part, st);
    }
    Few a = {w, x, ldw, ldx, np, nq, nk, np, ks, steps, splits, part, ldpart};
    if (splits == 1) return launch_few<EPI, GATED>(a, e, st);
    const hipError_t err = launch_few<kPartial, GATED>(a, e, st);
    return err != hipSuccess ? err : finish<T, EPI>(np, nq, e, *this, part, st);
  }
};

// A matrix as the products read it: the caller's, or a copy with padded rows.
template <typename T>
struct Source {
  const T* p;
  long long ld;
  int rows, cols;
  bool copy;
  size_t at = 0;
  // tiles: the products read it; whole: and want the rows' ends, along k, to be
  // those of 16 bytes.
  Source(const void* ptr, long long ld_, int rows_, int cols_, Layout* l, bool tiles = true, bool whole = false)
      : p(static_cast<const T*>(ptr)), ld(ld_), rows(rows_), cols(cols_),
        copy(tiles && (!direct<T>(ptr, ld_, cols_) || (whole && cols_ * sizeof(T) % 16))) {
    if (copy) at = l->add((size_t)rows * pad16<T>(cols) * sizeof(T));
  }
  hipError_t place(char* ws, hipStream_t st) {
    if (!copy) return hipSuccess;
    T* o = reinterpret_cast<T*>(ws + at);
    const int ldo = pad16<T>(cols);
    const long long n = (long long)rows * (ldo / (16 / (int)sizeof(T)));
    pad_kernel<T><<<(unsigned)std::min<long long>((n + 255) / 256, 1 << 20), 256, 0, st>>>(p, ld, rows, cols, o, ldo);
    p = o;
    ld = ldo;
    return hipGetLastError();
  }
  long long bytes() const { return ld * (long long)sizeof(T); }
  const char* ptr() const { return reinterpret_cast<const char*>(p); }
  int stored() const { return copy ? pad16<T>(cols) : cols; }  // columns, whole dwords
};

// ------------------------------------------------------------------- calls

// The call's workspace: the caller's or the stream's.  `*asked`: the caller
// only wants its size.
inline hipError_t claim(Scratch* ws, const Layout& l, const Room& room, hipStream_t st, bool* asked) {
  *asked = room.bytes && !room.ptr;
  if (*asked) {
    *room.bytes = l.bytes;
    return hipSuccess;
  }
  if (l.bytes == 0) return hipSuccess;
  const Workspace own{static_cast<char*>(room.ptr), room.bytes ? *room.bytes : 0};
  return ws->take(st, l.bytes, room.ptr ? &own : nullptr);
}

template <typename T>
hipError_t linear_forward(const LinearShape& s, const void* x, const void* w, const void* bias, int act,
                          const void* res, void* pre, void* y, const Room& room, hipStream_t st) {
  Layout l;
  const Forward<T> c(s.Ct, s.N, s.Cs, false);
  Source<T> xs(x, s.ldx, s.N, s.Cs, &l, !c.few, c.whole()), wsrc(w, s.Cs, s.Ct, s.Cs, &l, !c.few, c.whole());
  const size_t part = l.add(c.part_bytes);
  Scratch ws;
  bool asked;
  hipError_t e = claim(&ws, l, room, st, &asked);
  if (asked) return e;
  if (e == hipSuccess) e = xs.place(ws.get(), st);
  if (e == hipSuccess) e = wsrc.place(ws.get(), st);
  if (e != hipSuccess) return e;
  Epi p = {};
  p.y = y;
  p.ldy = s.ldy;
  p.pre = pre;
  p.ldpre = s.Ct;
  p.bias = bias;
  p.res = res;
  p.ldr = s.ldr;
  p.act = act;
  return c.template run<kLinear, false>(wsrc.ptr(), wsrc.bytes(), xs.ptr(), xs.bytes(),
                   std::min(wsrc.stored(), xs.stored()), p, reinterpret_cast<float*>(ws.get() + part), st);
}

template <typename T>
hipError_t gated_forward(const LinearShape& s, const void* x, const void* w, const void* bias, int act, void* pre,
                         void* y, const Room& room, hipStream_t st) {
  Layout l;
  const Forward<T> c(s.Ct, s.N, s.Cs, true);
  Source<T> xs(x, s.ldx, s.N, s.Cs, &l, !c.few, c.whole()), wsrc(w, s.Cs, 2 * s.Ct, s.Cs, &l, !c.few, c.whole());
  const size_t part = l.add(c.part_bytes);
  Scratch ws;
  bool asked;
  hipError_t e = claim(&ws, l, room, st, &asked);
  if (asked) return e;
  if (e == hipSuccess) e = xs.place(ws.get(), st);
  if (e == hipSuccess) e = wsrc.place(ws.get(), st);
  if (e != hipSuccess) return e;
  Epi p = {};
  p.y = y;
  p.ldy = s.ldy;
  p.pre = pre;
  p.ldpre = 2LL * s.Ct;
  p.bias = bias;
  p.act = act;
  return c.template run<kGated, true>(wsrc.ptr(), wsrc.bytes(), xs.ptr(), xs.bytes(),
                   std::min(wsrc.stored(), xs.stored()), p, reinterpret_cast<float*>(ws.get() + part), st);
}

// dx = dz w, as fp32 running sums in `acc` or finished in y.
// stored: dz's columns, whole dwords (zeros past the weight's rows).
template <typename T>
Prod dx_prod(const Source<T>& w, const char* wp, int wrows, const char* dz, long long lddz, int stored, int N) {
  Prod a = {};
  a.p = wp;
  a.ldp = w.bytes();
  a.np = w.cols;
  a.colsp = w.stored();
  a.kp = wrows;
  a.q = dz;
  a.ldq = lddz * (long long)sizeof(T);
  a.nq = N;
  a.nk = stored;
  return a;
}

// An input gradient's cut: of at most 32 rows in fp32, that of their own kernel
// (splits and ldpart; steps: 16 rows each, of a wave).
template <typename T>
constexpr int kThinRows = sizeof(T) == 4 ? 32 : 0;

template <typename T>
Cut dx_cut(int cols, int N, int rows) {
  if (N > kThinRows<T>) return cut_of<T>(cols, N, pad16<T>(rows), false);
  Cut c = {};
  const int groups = ceil_div(cols, 64), all = ceil_div(rows, 16);
  c.splits = std::max(1, std::min(1024 / groups, all / (8 * kFewWaves)));
  c.steps = ceil_div(all, kFewWaves * c.splits);
  c.splits = ceil_div(all, kFewWaves * c.steps);
  c.ldpart = (long long)ceil_div(cols, 4) * 4;
  c.part_bytes = c.splits > 1 ? (size_t)c.splits * N * c.ldpart * 4 : 0;
  return c;
}

// dx = dz w: d's columns are `stored`, whole dwords, `rows` without its zeros.
template <typename T>
hipError_t run_dx(const Source<T>& w, const char* wp, int rows, const char* d, long long ldd, int stored, int N,
                  const Epi& e, const Cut& c, float* part, hipStream_t st) {
  if constexpr (kThinRows<T> > 0) {
    if (N <= kThinRows<T>) {
      const Thin a = {reinterpret_cast<const float*>(wp), reinterpret_cast<const float*>(d), w.ld, ldd, rows, w.cols, N,
                      c.steps, c.splits, part, c.ldpart};
      const dim3 grid((unsigned)(ceil_div(w.cols, 64) * c.splits)), block(64 * kFewWaves);
      auto launch = [&](auto kernel) {
        LaunchTimer timer;
        return timed_launch(&timer, kernel, grid, block, 0u, st, a, e);
      };
      if (c.splits == 1) return N <= 16 ? launch(thin_kernel<1, kLinear>) : launch(thin_kernel<2, kLinear>);
      const hipError_t err = N <= 16 ? launch(thin_kernel<1, kPartial>) : launch(thin_kernel<2, kPartial>);
      return err != hipSuccess ? err : finish<T, kLinear>(w.cols, N, e, c, part, st);
    }
  }
  return run_product<T, true, false, kLinear, false>(dx_prod(w, wp, rows, d, ldd, stored, N), e, c, part, st);
}

// dw = dz^T x
template <typename T>
Prod dw_prod(const Source<T>& x, const char* dz, long long lddz, int stored, int wrows) {
  Prod a = {};
  a.p = x.ptr();
  a.ldp = x.bytes();
  a.np = x.cols;
  a.colsp = x.stored();
  a.kp = x.rows;
  a.q = dz;
  a.ldq = lddz * (long long)sizeof(T);
  a.nq = wrows;
  a.colsq = stored;
  a.kq = x.rows;
  a.nk = x.rows;
  return a;
}

// Weight gradients of at most 32 rows, one k of the matrix instruction: their
// own kernel (4096 -> 16384 in us: 32 rows bf16 36, fp32 75; tiles, at 33 rows,
// 52 and 100; 512 -> 512 takes 11 to 12 either way).
inline bool few_outer(int N) { return N <= 32; }

template <typename T>
hipError_t run_outer(const Source<T>& x, const char* d, long long ldd, int rows, const Epi& e, hipStream_t st) {
  Outer a = {x.ptr(), d, static_cast<char*>(e.y), x.ld, ldd, x.rows, x.cols, rows, 0, e.alpha};
  // 8192 waves fill the chip; each reads its columns of x once.
  const int across = ceil_div(x.cols, 512), down = std::max(1, std::min(ceil_div(rows, 16), 2048 / across));
  a.per = ceil_div(ceil_div(rows, down), 16) * 16;
  LaunchTimer timer;
  return timed_launch(&timer, outer_kernel<T>, dim3(across, ceil_div(rows, a.per)), dim3(256), 0u, st, a);
}

// Both layers' gradients from dz: rows of the weight `rows` (2 C_t if gated).
template <typename T, bool GATED>
hipError_t layer_backward(const LinearShape& s, const void* dy, const void* x, const void* w, const void* pre, int act,
                          void* dx, void* dw, void* dbias, const Room& room, hipStream_t st) {
  const int rows = GATED ? 2 * s.Ct : s.Ct;
  Layout l;
  // With no activation dy is dz, where the products can read it in place; with
  // no products dz is only summed.
  const bool products = dx || dw;
  const Cut cx = dx_cut<T>(s.Cs, s.N, rows), cw = cut_of<T>(s.Cs, rows, s.N, false);
  const bool fits = direct<T>(dy, s.ldy, s.Ct) && !(dx && ends_whole<T>(cx) && s.Ct * sizeof(T) % 16);
  const bool in_place = !GATED && act == QCNN_ACT_NONE && (fits || !products);
  const long long lddz = in_place ? s.ldy : pad16<T>(rows);
  const int stored = in_place ? rows : pad16<T>(rows);
  const bool kept = products && !in_place;
  const size_t dz_at = !kept ? 0 : l.add((size_t)s.N * lddz * sizeof(T));
  const int chunk = slope_chunk(s.N), chunks = ceil_div(s.N, chunk);
  const size_t sums_at = dbias ? l.add((size_t)chunks * rows * 4) : 0;
  const bool outer = few_outer(s.N);
  Source<T> xs(dw ? x : nullptr, dw ? s.ldx : 0, s.N, s.Cs, &l, dw && !outer),
      wsrc(dx ? w : nullptr, s.Cs, rows, s.Cs, &l, dx != nullptr);
  const size_t part = l.add(std::max(dx ? cx.part_bytes : 0, dw && !outer ? cw.part_bytes : 0));
  Scratch ws;
  bool asked;
  hipError_t e = claim(&ws, l, room, st, &asked);
  if (asked) return e;
  if (e == hipSuccess && dw) e = xs.place(ws.get(), st);
  if (e == hipSuccess && dx) e = wsrc.place(ws.get(), st);
  if (e != hipSuccess) return e;
  const char* dz = in_place ? static_cast<const char*>(dy) : ws.get() + dz_at;
  if (!in_place || dbias) {
    Slope a = {};
    a.dy = dy;
    a.pre = pre;
    a.dz = kept ? ws.get() + dz_at : nullptr;
    a.part = dbias ? reinterpret_cast<float*>(ws.get() + sums_at) : nullptr;
    a.lddy = s.ldy;
    a.ldpre = rows;
    a.lddz = lddz;
    a.rows = s.N;
    a.cols = s.Ct;
    a.chunk = chunk;
    a.act = act;
    e = run_slope<T, GATED>(a, dbias, nullptr, st);
    if (e != hipSuccess) return e;
  }
  float* sums = reinterpret_cast<float*>(ws.get() + part);
  if (dx) {
    Epi p = {};
    p.y = dx;
    p.ldy = s.Cs;
    e = run_dx<T>(wsrc, wsrc.ptr(), rows, dz, lddz, stored, s.N, p, cx, sums, st);
    if (e != hipSuccess) return e;
  }
  if (dw) {
    Epi p = {};
    p.y = dw;
    p.ldy = s.Cs;
    e = outer ? run_outer<T>(xs, dz, lddz, rows, p, st)
              : run_product<T, true, true, kLinear, false>(dw_prod(xs, dz, lddz, stored, rows), p, cw, sums, st);
  }
  return e;
}

template <typename T>
hipError_t xent_forward(const LinearShape& s, const void* x, const void* w, const void* bias, const long long* labels,
                        float* loss, float* lse, const Room& room, hipStream_t st) {
  Layout l;
  const Forward<T> c(s.Ct, s.N, s.Cs, false, true);
  Source<T> xs(x, s.ldx, s.N, s.Cs, &l, !c.few, c.whole()), wsrc(w, s.Cs, s.Ct, s.Cs, &l, !c.few, c.whole());
  const int slots = c.slots;
  const size_t part = l.add(c.part_bytes), stat = l.add((size_t)slots * s.N * 8), zl = l.add((size_t)s.N * 4);
  Scratch ws;
  bool asked;
  hipError_t e = claim(&ws, l, room, st, &asked);
  if (asked) return e;
  if (e == hipSuccess) e = xs.place(ws.get(), st);
  if (e == hipSuccess) e = wsrc.place(ws.get(), st);
  if (e != hipSuccess) return e;
  Epi p = {};
  p.bias = bias;
  p.labels = labels;
  p.stat = slots ? reinterpret_cast<float2*>(ws.get() + stat) : nullptr;
  p.zlabel = reinterpret_cast<float*>(ws.get() + zl);
  p.classes = s.Ct;
  p.loss = loss;
  p.lse_out = lse;
  e = c.template run<kStats, false>(wsrc.ptr(), wsrc.bytes(), xs.ptr(), xs.bytes(),
                   std::min(wsrc.stored(), xs.stored()), p, reinterpret_cast<float*>(ws.get() + part), st);
  if (e != hipSuccess || slots == 0) return e;
  // 16 rows read whole 128-byte lines; fewer than 64 rows would leave most of
  // the chip idle and go down hundreds of slots one after another.
  if (s.N >= 64)
    loss_kernel<16, 1024><<<ceil_div(s.N, 16), 1024, 0, st>>>(p.stat, p.zlabel, labels, slots, s.N, s.Ct, loss, lse);
  else
    loss_kernel<1, 256><<<s.N, 256, 0, st>>>(p.stat, p.zlabel, labels, slots, s.N, s.Ct, loss, lse);
  return hipGetLastError();
}

// Bytes of the logits' gradient that are held at once.
constexpr size_t kPieceBytes = (size_t)256 << 20;

template <typename T>
hipError_t xent_backward(const LinearShape& s, const void* x, const void* w, const void* bias, const long long* labels,
                         const float* lse, const float* dloss, void* dx, void* dw, void* dbias, const Room& room,
                         hipStream_t st) {
  Layout l;
  long long fit = (long long)(kPieceBytes / ((size_t)s.N * sizeof(T))) / 256 * 256;
  if (fit < 256) fit = 256;
  const int piece = fit < s.Ct ? (int)fit : s.Ct, pieces = ceil_div(s.Ct, piece);
  bool tiles = false, whole = false;
  const bool outer = few_outer(s.N);
  for (int n : {piece, s.Ct - (pieces - 1) * piece}) {
    const Forward<T> f(n, s.N, s.Cs, false);
    tiles |= !f.few;
    whole |= f.whole();
  }
  Source<T> xs(x, s.ldx, s.N, s.Cs, &l, tiles || (dw && !outer), whole), wsrc(w, s.Cs, s.Ct, s.Cs, &l, tiles || dx, whole);
  const long long ldd = pad16<T>(piece), ldacc = (s.Cs + 3) / 4 * 4;
  const size_t d_at = l.add((size_t)s.N * ldd * sizeof(T)), scale_at = l.add(8);
  const size_t acc_at = dx && pieces > 1 ? l.add((size_t)s.N * ldacc * 4) : 0;
  const int chunk = slope_chunk(s.N), chunks = ceil_div(s.N, chunk);
  const size_t sums_at = dbias ? l.add((size_t)chunks * piece * 4) : 0;
  size_t part_bytes = 0;
  for (int n : {piece, s.Ct - (pieces - 1) * piece}) {
    part_bytes = std::max(part_bytes, Forward<T>(n, s.N, s.Cs, false).part_bytes);
    if (dx) part_bytes = std::max(part_bytes, dx_cut<T>(s.Cs, s.N, n).part_bytes);
    if (dw && !outer) part_bytes = std::max(part_bytes, cut_of<T>(s.Cs, n, s.N, false).part_bytes);
  }
  const size_t part = l.add(part_bytes);
  Scratch ws;
  bool asked;
  hipError_t e = claim(&ws, l, room, st, &asked);
  if (asked) return e;
  if (e == hipSuccess) e = xs.place(ws.get(), st);
  if (e == hipSuccess) e = wsrc.place(ws.get(), st);
  if (e != hipSuccess) return e;
  float* scale = reinterpret_cast<float*>(ws.get() + scale_at);
  float* sums = reinterpret_cast<float*>(ws.get() + part);
  char* d = ws.get() + d_at;
  constexpr float gain = std::is_same<T, _Float16>::value ? 1024.f : 1.f;
  dmax_kernel<<<1, 1024, 0, st>>>(dloss, labels, s.N, gain, scale);
  e = hipGetLastError();
  for (int k = 0; k < pieces && e == hipSuccess; ++k) {
    const int c0 = k * piece, n = std::min(piece, s.Ct - c0);
    const long long ld = pad16<T>(n);
    Epi p = {};
    p.y = d;
    p.ldy = ld;
    p.bias = bias;
    p.labels = labels;
    p.lse = lse;
    p.dloss = dloss;
    p.dmax = scale;
    p.gain = gain;
    p.class0 = c0;
    p.classes = s.Ct;
    e = Forward<T>(n, s.N, s.Cs, false).template run<kXgrad, false>(wsrc.ptr() + c0 * wsrc.bytes(), wsrc.bytes(),
                                                                    xs.ptr(), xs.bytes(),
                                                                    std::min(wsrc.stored(), xs.stored()), p, sums, st);
    if (e == hipSuccess && dbias) {
      Slope b = {};
      b.dy = d;
      b.lddy = ld;
      b.part = reinterpret_cast<float*>(ws.get() + sums_at);
      b.rows = s.N;
      b.cols = n;
      b.chunk = chunk;
      b.act = QCNN_ACT_NONE;
      e = run_slope<T, false>(b, static_cast<T*>(dbias) + c0, scale + 1, st);
    }
    if (e == hipSuccess && dx) {
      Epi o = {};
      o.y = dx;
      o.ldy = s.Cs;
      o.alpha = scale + 1;
      o.acc = reinterpret_cast<float*>(ws.get() + acc_at);
      o.ldacc = ldacc;
      o.acc_in = k > 0;
      o.acc_out = k + 1 < pieces;
      e = run_dx<T>(wsrc, wsrc.ptr() + c0 * wsrc.bytes(), n, d, ld, (int)ld, s.N, o, dx_cut<T>(s.Cs, s.N, n), sums, st);
    }
    if (e == hipSuccess && dw) {
      Epi o = {};
      o.y = static_cast<T*>(dw) + (long long)c0 * s.Cs;
      o.ldy = s.Cs;
      o.alpha = scale + 1;
      e = outer ? run_outer<T>(xs, d, ld, n, o, st)
                : run_product<T, true, true, kLinear, false>(dw_prod(xs, d, ld, (int)ld, n), o,
                                                             cut_of<T>(s.Cs, n, s.N, false), sums, st);
    }
  }
  return e;
}

template <typename T>
hipError_t dispatch(const DenseCall& c, hipStream_t st) {
  switch (c.op) {
    case kLinearForward: return linear_forward<T>(c.s, c.x, c.w, c.bias, c.act, c.res, const_cast<void*>(c.pre), c.y, c.room, st);
    case kGatedForward: return gated_forward<T>(c.s, c.x, c.w, c.bias, c.act, const_cast<void*>(c.pre), c.y, c.room, st);
    case kLinearBackward: return layer_backward<T, false>(c.s, c.dy, c.x, c.w, c.pre, c.act, c.dx, c.dw, c.dbias, c.room, st);
    case kGatedBackward: return layer_backward<T, true>(c.s, c.dy, c.x, c.w, c.pre, c.act, c.dx, c.dw, c.dbias, c.room, st);
    case kXentForward: return xent_forward<T>(c.s, c.x, c.w, c.bias, c.labels, c.loss, c.lse, c.room, st);
    case kXentBackward:
      return xent_backward<T>(c.s, c.x, c.w, c.bias, c.labels, c.lse, static_cast<const float*>(c.dy), c.dx, c.dw, c.dbias, c.room, st);
  }
  return hipErrorInvalidValue;
}

}  // namespace dense
}  // namespace qcnn
