// C ABI of the dense layers: host-side validation before the first HIP call,
// then the kernels of the call's element type on the caller's stream.
#include <initializer_list>

#include "qcnn_internal.h"

namespace {

using qcnn::dense::DenseCall;

constexpr int kMaxRows = 1 << 21;
constexpr int kMaxCols = 1 << 20;           // 256 rows of an operand lie within 2^31 bytes
constexpr long long kMaxTiles = 1LL << 22;  // times 512 threads, a launch stays below 2^32

struct Span {
  const void* p;
  size_t bytes;
};

bool meet(const Span& a, const Span& b) {
  const uintptr_t a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p;
  return a.p && b.p && (a0 <= b0 ? b0 - a0 < a.bytes : a0 - b0 < b.bytes);  // no sum that could wrap
}

// The caller's workspace, which is written as outputs are.
Span room(const void* workspace, const size_t* bytes) { return {workspace, workspace && bytes ? *bytes : 0}; }

// An output overlaps an input or another output.
bool aliased(std::initializer_list<Span> in, std::initializer_list<Span> out) {
  for (const Span* o = out.begin(); o != out.end(); ++o) {
    for (const Span& i : in)
      if (meet(*o, i)) return true;
    for (const Span* t = out.begin(); t != o; ++t)
      if (meet(*o, *t)) return true;
  }
  return false;
}

int size_of(int dtype) { return dtype == QCNN_F32 ? 4 : dtype == QCNN_BF16 || dtype == QCNN_F16 ? 2 : 0; }

long long tiles(long long a, long long b) { return ((a + 127) / 128) * ((b + 127) / 128); }

// Sizes, strides (0: not given) and the alignment of the arrays of T; rows:
// those of the weight, at most 2 C_t.
qcnn_status check(int dtype, int act, int N, int Cs, int Ct, int halves, std::initializer_list<long long> ld_cols,
                  std::initializer_list<const void*> arrays) {
  const int s = size_of(dtype);
  if (!s || act < QCNN_ACT_NONE || act > QCNN_ACT_SILU) return QCNN_ERR_UNSUPPORTED;
  if (N < 1 || Cs < 1 || Ct < 1) return QCNN_ERR_SHAPE;
  for (const long long* v = ld_cols.begin(); v != ld_cols.end(); v += 2) {
    if (v[0] < v[1]) return QCNN_ERR_SHAPE;
    if (v[0] > kMaxCols) return QCNN_ERR_UNSUPPORTED;
  }
  const long long rows = (long long)halves * Ct;
  if (N > kMaxRows || Cs > kMaxCols || rows > kMaxCols) return QCNN_ERR_UNSUPPORTED;
  if (tiles(N, rows) > kMaxTiles || tiles(N, Cs) > kMaxTiles || tiles(rows, Cs) > kMaxTiles)
    return QCNN_ERR_UNSUPPORTED;
  for (const void* p : arrays)
    if ((uintptr_t)p & (s - 1)) return QCNN_ERR_UNSUPPORTED;
  return QCNN_OK;
}

size_t span(int rows, long long ld, long long cols, int s) { return ((size_t)(rows - 1) * ld + cols) * s; }

qcnn_status run(int dtype, DenseCall& c, void* workspace, size_t* workspace_bytes, void* stream) {
  if (workspace && !workspace_bytes) return QCNN_ERR_NULL;
  if ((uintptr_t)workspace & 255) return QCNN_ERR_UNSUPPORTED;
  c.room = qcnn::dense::Room{workspace, workspace_bytes};
  const hipStream_t st = (hipStream_t)stream;
  try {
    const hipError_t e = dtype == QCNN_F32 ? qcnn::dense::run_f32(c, st)
                         : dtype == QCNN_BF16 ? qcnn::dense::run_bf16(c, st)
                                              : qcnn::dense::run_f16(c, st);
    if (e == hipSuccess) return QCNN_OK;
    return workspace && e == hipErrorOutOfMemory ? QCNN_ERR_WORKSPACE : QCNN_ERR_HIP;
  } catch (...) {
    return QCNN_ERR_HIP;
  }
}

qcnn_status backward(bool gated, int dtype, const void* dy, long long lddy, const void* x, long long ldx, int N,
                     int C_s, const void* w, int C_t, const void* pre, int act, void* dx, void* dw, void* dbias,
                     void* workspace, size_t* workspace_bytes, void* stream) {
  if (!dy || (!dx && !dw && !dbias) || (dx && !w) || (dw && !x) || (!pre && (gated || act != QCNN_ACT_NONE)))
    return QCNN_ERR_NULL;
  const int halves = gated ? 2 : 1, s = size_of(dtype);
  if (!dw) ldx = C_s;  // x is not read
  const qcnn_status st = check(dtype, act, N, C_s, C_t, halves, {lddy, C_t, ldx, C_s}, {dy, x, w, pre, dx, dw, dbias});
  if (st != QCNN_OK) return st;
  const size_t rows = (size_t)halves * C_t, nw = rows * C_s * s, nx = (size_t)N * C_s * s;
  if (aliased({{dy, span(N, lddy, C_t, s)}, {dw ? x : nullptr, span(N, ldx, C_s, s)}, {dx ? w : nullptr, nw},
               {pre, rows * N * s}},
              {{dx, nx}, {dw, nw}, {dbias, rows * s}, room(workspace, workspace_bytes)}))
    return QCNN_ERR_ALIAS;
  DenseCall c = {};
  c.op = gated ? qcnn::dense::kGatedBackward : qcnn::dense::kLinearBackward;
  c.s = {N, C_s, C_t, ldx, lddy, 0};
  c.act = act;
  c.x = x;
  c.w = w;
  c.dy = dy;
  c.pre = pre;
  c.dx = dx;
  c.dw = dw;
  c.dbias = dbias;
  return run(dtype, c, workspace, workspace_bytes, stream);
}

}  // namespace

extern "C" {

qcnn_status qcnn_linear_forward(int dtype, const void* x, long long ldx, int N, int C_s, const void* w, int C_t,
                                const void* bias, int act, const void* residual, long long ldr, void* pre, void* y,
                                long long ldy, void* workspace, size_t* workspace_bytes, void* stream) {
  if (!x || !w || !y) return QCNN_ERR_NULL;
  const int s = size_of(dtype);
  if (!residual) ldr = C_t;
  const qcnn_status st = check(dtype, act, N, C_s, C_t, 1, {ldx, C_s, ldy, C_t, ldr, C_t},
                               {x, w, bias, residual, pre, y});
  if (st != QCNN_OK) return st;
  if (aliased({{x, span(N, ldx, C_s, s)}, {w, (size_t)C_t * C_s * s}, {bias, (size_t)C_t * s},
               {residual, span(N, ldr, C_t, s)}},
              {{y, span(N, ldy, C_t, s)}, {pre, (size_t)N * C_t * s}, room(workspace, workspace_bytes)}))
    return QCNN_ERR_ALIAS;
  DenseCall c = {};
  c.op = qcnn::dense::kLinearForward;
  c.s = {N, C_s, C_t, ldx, ldy, ldr};
  c.act = act;
  c.x = x;
  c.w = w;
  c.bias = bias;
  c.res = residual;
  c.pre = pre;
  c.y = y;
  return run(dtype, c, workspace, workspace_bytes, stream);
}

qcnn_status qcnn_linear_backward(int dtype, const void* dy, long long lddy, const void* x, long long ldx, int N,
                                 int C_s, const void* w, int C_t, const void* pre, int act, void* dx, void* dw,
                                 void* dbias, void* workspace, size_t* workspace_bytes, void* stream) {
  return backward(false, dtype, dy, lddy, x, ldx, N, C_s, w, C_t, pre, act, dx, dw, dbias, workspace, workspace_bytes,
                  stream);
}

qcnn_status qcnn_gated_forward(int dtype, const void* x, long long ldx, int N, int C_s, const void* w, int C_t,
                               const void* bias, int act, void* pre, void* y, long long ldy, void* workspace,
                               size_t* workspace_bytes, void* stream) {
  if (!x || !w || !y) return QCNN_ERR_NULL;
  const int s = size_of(dtype);
  const qcnn_status st = check(dtype, act, N, C_s, C_t, 2, {ldx, C_s, ldy, C_t}, {x, w, bias, pre, y});
  if (st != QCNN_OK) return st;
  const size_t rows = 2 * (size_t)C_t;
  if (aliased({{x, span(N, ldx, C_s, s)}, {w, rows * C_s * s}, {bias, rows * s}},
              {{y, span(N, ldy, C_t, s)}, {pre, N * rows * s}, room(workspace, workspace_bytes)}))
    return QCNN_ERR_ALIAS;
  DenseCall c = {};
  c.op = qcnn::dense::kGatedForward;
  c.s = {N, C_s, C_t, ldx, ldy, 0};
  c.act = act;
  c.x = x;
  c.w = w;
  c.bias = bias;
  c.pre = pre;
  c.y = y;
  return run(dtype, c, workspace, workspace_bytes, stream);
}

qcnn_status qcnn_gated_backward(int dtype, const void* dy, long long lddy, const void* x, long long ldx, int N,
                                int C_s, const void* w, int C_t, const void* pre, int act, void* dx, void* dw,
                                void* dbias, void* workspace, size_t* workspace_bytes, void* stream) {
  return backward(true, dtype, dy, lddy, x, ldx, N, C_s, w, C_t, pre, act, dx, dw, dbias, workspace, workspace_bytes,
                  stream);
}

qcnn_status qcnn_linear_xent_forward(int dtype, const void* x, long long ldx, int N, int C_s, const void* w, int C_t,
                                     const void* bias, const int64_t* labels, float* loss, float* lse,
                                     void* workspace, size_t* workspace_bytes, void* stream) {
  if (!x || !w || !labels || !loss || !lse) return QCNN_ERR_NULL;
  const int s = size_of(dtype);
  const qcnn_status st = check(dtype, QCNN_ACT_NONE, N, C_s, C_t, 1, {ldx, C_s}, {x, w, bias});
  if (st != QCNN_OK) return st;
  if (((uintptr_t)labels & 7) || (((uintptr_t)loss | (uintptr_t)lse) & 3)) return QCNN_ERR_UNSUPPORTED;
  if (aliased({{x, span(N, ldx, C_s, s)}, {w, (size_t)C_t * C_s * s}, {bias, (size_t)C_t * s}, {labels, (size_t)N * 8}},
              {{loss, (size_t)N * 4}, {lse, (size_t)N * 4}, room(workspace, workspace_bytes)}))
    return QCNN_ERR_ALIAS;
  DenseCall c = {};
  c.op = qcnn::dense::kXentForward;
  c.s = {N, C_s, C_t, ldx, 0, 0};
  c.x = x;
  c.w = w;
  c.bias = bias;
  c.labels = reinterpret_cast<const long long*>(labels);
  c.loss = loss;
  c.lse = lse;
  return run(dtype, c, workspace, workspace_bytes, stream);
}

qcnn_status qcnn_linear_xent_backward(int dtype, const float* dloss, const float* lse, const void* x, long long ldx,
                                      int N, int C_s, const void* w, int C_t, const void* bias,
                                      const int64_t* labels, void* dx, void* dw, void* dbias, void* workspace,
                                      size_t* workspace_bytes, void* stream) {
  if (!x || !w || !labels || !dloss || !lse || (!dx && !dw && !dbias)) return QCNN_ERR_NULL;
  const int s = size_of(dtype);
  const qcnn_status st = check(dtype, QCNN_ACT_NONE, N, C_s, C_t, 1, {ldx, C_s}, {x, w, bias, dx, dw, dbias});
  if (st != QCNN_OK) return st;
  if (((uintptr_t)labels & 7) || (((uintptr_t)dloss | (uintptr_t)lse) & 3)) return QCNN_ERR_UNSUPPORTED;
  const size_t nw = (size_t)C_t * C_s * s;
  if (aliased({{x, span(N, ldx, C_s, s)}, {w, nw}, {bias, (size_t)C_t * s}, {labels, (size_t)N * 8},
               {dloss, (size_t)N * 4}, {lse, (size_t)N * 4}},
              {{dx, (size_t)N * C_s * s}, {dw, nw}, {dbias, (size_t)C_t * s}, room(workspace, workspace_bytes)}))
    return QCNN_ERR_ALIAS;
  DenseCall c = {};
  c.op = qcnn::dense::kXentBackward;
  c.s = {N, C_s, C_t, ldx, 0, 0};
  c.x = x;
  c.w = w;
  c.bias = bias;
  c.dy = dloss;
  c.lse = const_cast<float*>(lse);
  c.labels = reinterpret_cast<const long long*>(labels);
  c.dx = dx;
  c.dw = dw;
  c.dbias = dbias;
  return run(dtype, c, workspace, workspace_bytes, stream);
}

}  // extern "C"
