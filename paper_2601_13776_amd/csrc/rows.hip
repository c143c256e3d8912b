// Entry points of the row-grouped products: the application of a batch of
// dense matrices to their rows, the gradient with respect to the matrices,
// and the classification loss with its gradients.  No call copies a table or
// allocates, so every call here can be captured into a HIP graph.
//
// The loss: z = scale x W^T is never stored.  Its product's epilogue reduces
// each tile's columns to a maximum m and a sum of exp(z - m) per row, which the
// join turns into lse = m + log sum, loss = lse - z_target (all fp32).  The
// backward forms z again, a piece of the classes at a time, and from it dz =
// scale grad_loss (exp(z - lse) - [target]), the operand of dx = dz W and dW =
// dz^T x: in fp32, or for bf16 operands in two bf16 pieces, 16 bits, whose
// products are twice as many (8 N V d flop; with the loss and the second z 12).
// Against kept logits the second z costs 2 N V d for N V fewer values to hold.
// 4096 rows, 2048 features, 50003 classes in bf16: loss 0.71, backward 3.52 ms,
// together 1190 TFLOP/s of these, bound by the products (with dz in one bf16
// piece the backward took 2.27).  8 rows, 4096 features, 131072 classes: loss 171
// us, W read at 6.3 TB/s.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdio>

#include "rows.h"

namespace orth {

namespace {

constexpr size_t kAlign = 256;
size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }

int invalid(const char* msg) { return report_error(ORTH_EINVAL, msg); }
int hip_check(hipError_t e, const char* what) {
  if (e == hipSuccess) return ORTH_OK;
  char buf[256];
  snprintf(buf, sizeof buf, "%s: %s", what, hipGetErrorString(e));
  return report_error(ORTH_EHIP, buf);
}
int check_ws(const void* ws, size_t have, size_t need) {
  if (need == 0) return ORTH_OK;
  if (!ws) return report_error(ORTH_EWORKSPACE, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(ws) % kAlign)
    return report_error(ORTH_EWORKSPACE, "workspace must be 256-byte aligned");
  if (have < need) {
    char buf[128];
    snprintf(buf, sizeof buf, "workspace too small: %zu bytes given, %zu needed", have, need);
    return report_error(ORTH_EWORKSPACE, buf);
  }
  return ORTH_OK;
}
bool known(int dtype) { return dtype == ORTH_F32 || dtype == ORTH_BF16; }
int64_t esize(int dtype) { return dtype == ORTH_BF16 ? 2 : 4; }
constexpr int64_t kMaxBlocks = (1 << 23) - 1;   // of up to 512 threads: a grid holds less than 2^32
constexpr int kMaxRowBlocks = 1 << 20;          // of kernels that take rows in turn
constexpr int kMaxSize = 1 << 30;   // of every extent: sums of two stay within 32 bits
// Every workgroup reads all offsets, 64 at a time with 32-bit counters (which
// 2^31 groups overflow): 0.6 ms of 2^16 groups, 9 ms of the most.
constexpr int kMaxGroups = 1 << 20;

// Whether [a, a + n) and [b, b + m) share a byte.
bool overlap(const void* a, int64_t n, const void* b, int64_t m) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return n > 0 && m > 0 && x < y + (uintptr_t)m && y < x + (uintptr_t)n;
}
// The same of two matrices of one type; column slices of one buffer, with
// the buffer's leading dimension both, do not share.
bool overlap_rows(const void* a, int64_t ra, int64_t la, int64_t ca, const void* b, int64_t rb, int64_t lb, int64_t cb,
                  int dtype) {
  const int64_t es = esize(dtype);
  if (ra < 1 || rb < 1 || !overlap(a, ((ra - 1) * la + ca) * es, b, ((rb - 1) * lb + cb) * es)) return false;
  if (la != lb || ra == 1 || rb == 1) return true;
  const int64_t ld = la * es;
  const int64_t d = ((int64_t)(reinterpret_cast<uintptr_t>(b) - reinterpret_cast<uintptr_t>(a)) % ld + ld) % ld;
  return !(d >= ca * es && d + cb * es <= ld);
}
int64_t span(int64_t rows, int64_t ld, int64_t cols, int dtype) {
  return rows < 1 ? 0 : ((rows - 1) * ld + cols) * esize(dtype);
}

// Whether n rows (matrices) that far apart span more than any memory: their
// byte offsets would not fit 64 bits.
bool far(int64_t n, int64_t ld) { return (double)n * (double)ld > 0x1p48; }

constexpr int kOuter = 16;   // (in place of a tile edge: rows_few.hip)

// The tile edge of a product; 32: the kernel without staging, where its 32 x 32
// tiles run in one round of two workgroups per compute unit, and where groups
// hold so few rows that reading the matrices is what counts.  Measured (us,
// this / staged tiles) at 512 workgroups: bf16 512 x 1024 x 1024 7.0 / 11.9, 64
// x 4096 x 4096 10 / 32, fp32 13.6 / 20; at 1024 bf16 11 / 12, fp32 39 / 21.
// 64 rows over 64 matrices of 4096^2 342 / 376, 128 over 64 of 2048^2 101 / 134,
// 1024 over 64 of 2048^2 109 / 138.
int tile_of(const RowsProd& p, int dtype, bool at, bool bt) {
  if (!at && rows_blocks(p, false, 32) <= 512) return 32;
  if (!at && !bt && p.rows / p.groups <= 16 && (p.offsets || dtype == ORTH_F32 || !rows_bf16_dma(p, false, false)))
    return 32;
  return dtype == ORTH_BF16 ? rows_bf16_tile(p, at, bt) : rows_f32_tile(p, at);
}
hipError_t launch(const RowsProd& p, int dtype, bool at, bool bt, int epi, int tile, const char* name, hipStream_t s) {
  if (tile == 32) return launch_rows_direct(p, dtype, bt, epi, 1, name, s);
  if (tile == kOuter) return launch_rows_outer(p, dtype, name, s);
  return dtype == ORTH_BF16 ? launch_rows_bf16(p, at, bt, epi, tile, name, s)
                            : launch_rows_f32(p, at, bt, epi, tile, name, s);
}

// The gradient of the matrices (grouped along K), in one launch or, where its
// tiles fill half the chip at most and groups hold many rows, with the rows
// cut into slices whose sums a second launch joins.  Measured (us, whole /
// sliced), one group: bf16 256 x 256, 4096 rows 31 / 15, 16384 rows 112 / 22,
// 2048 x 1024, 16384 rows 115 / 86; fp32 256 x 256, 1024 rows 23 / 14, 16384
// rows 288 / 33.  With fewer rows the second launch costs what the first
// gains: bf16 256 x 256, 1024 rows 12.6 / 13.9; fp32, 256 rows 9.0 / 13.  Few
// rows per group (us, tiles / rows_outer, 50000 x 2048): bf16 8 rows 104 / 37, 32
// rows 94 / 46, 64 rows 89 / 92 and of operands that the direct loads cannot take
// (20001 x 1001) 43 / 24; fp32 8 rows 185 / 81, 32 rows 200 / 132, 64 rows 253 /
// 198, but 1000 x 2048 from 64 rows 9.9 / 12.8.
struct GradPlan {
  int tile = 0, kslice = 0;   // kslice 0: whole
  size_t bytes = 0;           // of the slices' sums
};
GradPlan grad_plan(const RowsProd& p, int dtype) {
  GradPlan g;
  const int few = dtype == ORTH_F32 || !rows_bf16_dma(p, true, true) ? 64 : 32;
  if (p.rows / p.groups <= few && p.groups <= 65535) {
    g.tile = kOuter;
    return g;
  }
  g.tile = tile_of(p, dtype, true, true);
  const int64_t tiles = (int64_t)((p.M + g.tile - 1) / g.tile) * ((p.N + g.tile - 1) / g.tile);
  const int least = dtype == ORTH_BF16 ? 512 : 256;
  if (tiles * p.groups > 128 || p.rows / p.groups < 4 * least) return g;
  const int64_t parts = 256 / tiles;   // slices that fill the chip once
  g.kslice = (int)std::max<int64_t>(least, (p.rows / parts + 63) / 64 * 64);
  g.bytes = (size_t)rows_parts(p, g.kslice) * p.M * p.N * 4;
  return g;
}
hipError_t launch_grad(RowsProd p, int dtype, const GradPlan& g, void* ws, const char* name, const char* join,
                       hipStream_t s) {
  if (!g.kslice) return launch(p, dtype, true, true, ROWS_STORE, g.tile, name, s);
  p.kslice = g.kslice;
  p.slices = static_cast<float*>(ws);
  const hipError_t e = launch(p, dtype, true, true, ROWS_SLICE, g.tile, name, s);
  return e == hipSuccess ? launch_rows_join_groups(p, join, s) : e;
}
int64_t grad_blocks(RowsProd p, int dtype, const GradPlan& g) {
  if (g.tile == kOuter) return rows_outer_blocks(p, dtype);
  p.kslice = g.kslice;
  return rows_launch_blocks(p, true, g.kslice ? ROWS_SLICE : ROWS_STORE, g.tile);
}

// ----------------------------------------------------- small kernels ------
// The rows' (maximum, sum of exponentials) of every column block joined: a
// wave per row, or a workgroup where rows have many blocks (8 rows of 2048
// blocks: 19 us with a wave each, 5 with 256 threads).
template <int W>
__global__ __launch_bounds__(256) void xent_join_kernel(const float2* part, int n_part, const float* ztarget,
                                                        const int64_t* targets, int rows, int classes, float* loss,
                                                        float* lse) {
  __shared__ float2 waves[4];
  const int lane = threadIdx.x & 63, first = W == 4 ? threadIdx.x : lane;
  const int step = W == 4 ? gridDim.x : gridDim.x * 4;
  for (int i = W == 4 ? blockIdx.x : blockIdx.x * 4 + (threadIdx.x >> 6); i < rows; i += step) {
    const float* q = reinterpret_cast<const float*>(part + (int64_t)i * n_part);
    float top = -INFINITY, sum = 0.f;
    // eight blocks in flight; an empty sum adds nothing, whatever its maximum
    for (int k = first; k < n_part; k += 8 * 64 * W) {
      orth_f32x2 v[8];
      float m = top;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int b = k + u * 64 * W;
        v[u] = orth_f32x2{-INFINITY, 0.f};
        if (b < n_part) v[u] = *(const ORTH_GLOBAL orth_f32x2*)(q + 2 * (int64_t)b);
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) m = fmaxf(m, v[u].x);
      const float from = lse_base(m);
      sum = sum == 0.f ? 0.f : sum * __expf(top - from);
#pragma unroll
      for (int u = 0; u < 8; ++u) sum += v[u].y == 0.f ? 0.f : v[u].y * __expf(v[u].x - from);
      top = m;
    }
    auto join = [](float& t, float& s, float ot, float os) {
      const float m = fmaxf(t, ot), from = lse_base(m);
      s = (s == 0.f ? 0.f : s * __expf(t - from)) + (os == 0.f ? 0.f : os * __expf(ot - from));
      t = m;
    };
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
      const float ot = __shfl_xor(top, d, 64), os = __shfl_xor(sum, d, 64);
      join(top, sum, ot, os);
    }
    if constexpr (W == 4) {
      if (lane == 0) waves[threadIdx.x >> 6] = make_float2(top, sum);
      __syncthreads();
      if (threadIdx.x == 0)
        for (int w = 1; w < 4; ++w) join(top, sum, waves[w].x, waves[w].y);
      __syncthreads();
    }
    if (first == 0) {
      const float l = top + __logf(sum);
      const int64_t t = targets[i];
      lse[i] = l;
      loss[i] = t >= 0 && t < classes ? l - ztarget[i] : 0.f;
    }
  }
}

// Rows of a matrix with zeros in the columns up to ldo; targets (may be
// NULL): zeros for rows without one.  twice: row i as rows 2 i and 2 i + 1.
// A thread moves 16 bytes from any alignment to an aligned place.
template <typename V>
__global__ __launch_bounds__(256) void pad_rows_kernel(const V* x, int64_t ld, V* out, int ldo, int rows,
                                                       int cols, const int64_t* targets, int classes, int twice) {
  constexpr int L = 16 / sizeof(V);
  for (int64_t i = blockIdx.x; i < rows; i += gridDim.x) {
    const int64_t t = targets ? targets[i] : 0;
    const bool has = t >= 0 && t < classes;
    for (int c = threadIdx.x * L; c < ldo; c += 256 * L) {   // (ldo is a multiple of 8)
      const V* at = x + i * ld + c;
      V w[L] = {};
      if (has && c + L <= cols) {
        const orth_u32x4_a2 v = *(const ORTH_GLOBAL orth_u32x4_a2*)at;
        __builtin_memcpy(w, &v, 16);
      } else if (has) {
#pragma unroll
        for (int e = 0; e < L; ++e)
          if (c + e < cols) w[e] = at[e];
      }
      orth_u32x4 v;
      __builtin_memcpy(&v, w, 16);
      V* to = out + (i << twice) * ldo + c;
      *(ORTH_GLOBAL orth_u32x4*)to = v;
      if (twice) *(ORTH_GLOBAL orth_u32x4*)(to + ldo) = v;
    }
  }
}

hipError_t launch_pad(const void* x, int64_t ld, void* out, int ldo, int rows, int cols, int dtype,
                      const int64_t* targets, int classes, int twice, const char* name, hipStream_t s) {
  timing_begin(name, s);
  if (dtype == ORTH_BF16)
    hipLaunchKernelGGL(pad_rows_kernel<uint16_t>, dim3((unsigned)std::min(rows, kMaxRowBlocks)), dim3(256), 0, s,
                       static_cast<const uint16_t*>(x), ld, static_cast<uint16_t*>(out), ldo, rows, cols, targets, classes, twice);
  else
    hipLaunchKernelGGL(pad_rows_kernel<float>, dim3((unsigned)std::min(rows, kMaxRowBlocks)), dim3(256), 0, s, static_cast<const float*>(x), ld,
                       static_cast<float*>(out), ldo, rows, cols, targets, classes, twice);
  const hipError_t e = hipGetLastError();
  timing_end(name, s);
  return e;
}

}  // namespace

// ------------------------------------------------------- application ------
namespace {
int validate_linear(const orth_linear_args* a, bool grad) {
  if (!a) return invalid("args is NULL");
  if (!a->w || (a->rows > 0 && (!a->x || !a->y))) return invalid("NULL data pointer");
  if (!known(a->dtype) || !known(a->grad_dtype)) return invalid("unknown dtype");
  if (a->rows < 0 || a->groups < 1 || a->in_features < 1 || a->out_features < 1)
    return invalid("rows must be >= 0, groups, in_features and out_features >= 1");
  if (a->rows > kMaxSize || a->in_features > kMaxSize || a->out_features > kMaxSize)
    return invalid("size too large");
  if (a->groups > kMaxGroups) return invalid("too many groups");
  if (!a->offsets && a->groups != 1) return invalid("offsets is NULL with several groups");
  const int64_t cx = grad || !a->transposed ? a->in_features : a->out_features;
  const int64_t cy = grad || !a->transposed ? a->out_features : a->in_features;
  if (a->ld_x < cx || a->ld_y < cy || a->ld_w < a->in_features) return invalid("leading dimension below the columns");
  if (a->groups > 1 && a->stride_w < (int64_t)(a->out_features - 1) * a->ld_w + a->in_features &&
      (grad || a->stride_w != 0))
    return invalid("stride_w below one matrix");
  if (far(a->rows, a->ld_x) || far(a->rows, a->ld_y) || far(a->out_features, a->ld_w) ||
      (a->groups > 1 && far(a->groups, a->stride_w)))
    return invalid("leading dimension or stride_w too large");
  return ORTH_OK;
}

RowsProd grad_product(const orth_linear_args* a) {
  RowsProd p{};
  p.A = a->y;
  p.B = a->x;
  p.C = a->w;
  p.lda = a->ld_y;
  p.ldb = a->ld_x;
  p.ldc = a->ld_w;
  p.gc = a->groups > 1 ? a->stride_w : 0;
  p.offsets = a->offsets;
  p.groups = a->groups;
  p.rows = p.K = p.kslice = a->rows;
  p.M = a->out_features;
  p.N = a->in_features;
  p.c_dtype = a->grad_dtype;
  return p;
}
}  // namespace

}  // namespace orth

using namespace orth;

extern "C" {

int orth_linear_apply(const orth_linear_args* a, void* stream) {
  const int rc = validate_linear(a, false);
  if (rc) return rc;
  if (a->transposed != 0 && a->transposed != 1) return invalid("transposed must be 0 or 1");
  const bool tr = a->transposed != 0;
  RowsProd p{};
  p.A = a->x;
  p.B = a->w;
  p.C = a->y;
  p.lda = a->ld_x;
  p.ldb = a->ld_w;
  p.ldc = a->ld_y;
  p.gb = a->groups > 1 ? a->stride_w : 0;
  p.offsets = a->offsets;
  p.groups = a->groups;
  p.rows = p.M = a->rows;
  p.N = tr ? a->in_features : a->out_features;
  p.K = tr ? a->out_features : a->in_features;
  p.c_dtype = a->dtype;
  p.kslice = p.K;
  const int64_t by = span(a->rows, a->ld_y, p.N, a->dtype);
  const int64_t bw = span(a->out_features, a->ld_w, a->in_features, a->dtype) + (a->groups - 1) * p.gb * esize(a->dtype);
  if (overlap_rows(a->x, a->rows, a->ld_x, p.K, a->y, a->rows, a->ld_y, p.N, a->dtype) || overlap(a->w, bw, a->y, by))
    return invalid("y must not overlap x or w");
  const int tile = tile_of(p, a->dtype, false, tr);
  if (rows_blocks(p, false, tile) > kMaxBlocks) return invalid("rows x columns too large");
  return hip_check(launch(p, a->dtype, false, tr, ROWS_STORE, tile, tr ? "linear_apply_t" : "linear_apply",
                          static_cast<hipStream_t>(stream)),
                   "orth_linear_apply");
}

int orth_linear_grad_weight_workspace_size(const orth_linear_args* a, size_t* bytes) {
  if (!bytes) return invalid("bytes is NULL");
  const int rc = validate_linear(a, true);
  if (rc) return rc;
  *bytes = grad_plan(grad_product(a), a->dtype).bytes;
  return ORTH_OK;
}

int orth_linear_grad_weight(const orth_linear_args* a, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = validate_linear(a, true);
  if (rc) return rc;
  const RowsProd p = grad_product(a);
  const int64_t bx = span(a->rows, a->ld_x, p.N, a->dtype), by = span(a->rows, a->ld_y, p.M, a->dtype);
  const int64_t bw = span(p.M, a->ld_w, p.N, a->grad_dtype) + (a->groups - 1) * p.gc * esize(a->grad_dtype);
  if (overlap(a->x, bx, a->w, bw) || overlap(a->y, by, a->w, bw)) return invalid("w must not overlap x or y");
  const GradPlan g = grad_plan(p, a->dtype);
  rc = check_ws(workspace, workspace_bytes, g.bytes);
  if (rc) return rc;
  if (grad_blocks(p, a->dtype, g) > kMaxBlocks) return invalid("groups x matrix too large");
  return hip_check(launch_grad(p, a->dtype, g, workspace, "linear_grad_weight", "linear_grad_weight_join",
                               static_cast<hipStream_t>(stream)),
                   "orth_linear_grad_weight");
}

}  // extern "C"

// --------------------------------------------------------------- loss -----
namespace orth {
namespace {

int validate_xent(const orth_linear_xent_args* a) {
  if (!a) return invalid("args is NULL");
  if (!a->w || (a->rows > 0 && (!a->x || !a->targets))) return invalid("NULL data pointer");
  if (!known(a->dtype)) return invalid("unknown dtype");
  if (a->rows < 0 || a->features < 1 || a->classes < 1) return invalid("rows must be >= 0, features and classes >= 1");
  if (a->rows > kMaxSize || a->features > kMaxSize || a->classes > kMaxSize)
    return invalid("size too large");
  if (a->ld_x < a->features || a->ld_w < a->features) return invalid("leading dimension below the columns");
  if (far(a->rows, a->ld_x) || far(a->classes, a->ld_w)) return invalid("leading dimension too large");
  if (!std::isfinite(a->scale)) return invalid("scale must be finite");
  if (a->piece < 0) return invalid("piece must be >= 0");
  return ORTH_OK;
}

// Leading dimension of the padded copy that a bf16 product of many rows takes
// of an operand whose rows the direct-to-LDS loads cannot (0: none): the copy
// costs one pass over it, the loads through registers twice the products' time
// (3272 rows, 1444 features, 54027 classes: logits 1230 us, with copies 620).
int padded(const orth_linear_xent_args* a, const void* w, int64_t ld) {
  const bool aligned = reinterpret_cast<uintptr_t>(w) % 16 == 0 && ld % 8 == 0 && ld <= (1 << 22);
  if (a->dtype != ORTH_BF16 || a->rows < 256 || (aligned && a->features % 8 == 0)) return 0;
  return (a->features + 7) / 8 * 8;
}

struct XentPlan {
  RowsProd logits{};   // x W^T over all classes
  int tile = 0, ldw = 0, ldx = 0;   // padded copies
  size_t off_part = 0, off_target = 0, off_w = 0, off_x = 0, total = 0;
};
int validate_xent_vjp(const orth_linear_xent_args* a) {
  const int rc = validate_xent(a);
  if (rc) return rc;
  // (bf16: dz takes two rows each)
  return a->dtype == ORTH_BF16 && a->rows > kMaxSize / 2 ? invalid("size too large") : (int)ORTH_OK;
}

// (ws: the workspace, or any aligned address to size it)
XentPlan xent_plan(const orth_linear_xent_args* a, unsigned char* ws) {
  XentPlan P;
  RowsProd& p = P.logits;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += align_up(bytes);
    return at;
  };
  P.ldw = padded(a, a->w, a->ld_w);
  P.ldx = padded(a, a->x, a->ld_x);
  if (P.ldw) P.off_w = take((size_t)a->classes * P.ldw * 2);
  if (P.ldx) P.off_x = take((size_t)a->rows * P.ldx * 2);
  p.A = P.ldx ? ws + P.off_x : a->x;
  p.B = P.ldw ? ws + P.off_w : a->w;
  p.lda = P.ldx ? P.ldx : a->ld_x;
  p.ldb = P.ldw ? P.ldw : a->ld_w;
  p.groups = 1;
  p.rows = p.M = a->rows;
  p.N = p.classes = a->classes;
  p.K = p.kslice = a->features;
  p.scale = a->scale;
  p.targets = a->targets;
  P.tile = tile_of(p, a->dtype, false, false);
  // one (maximum, sum) per wave's columns
  p.n_part = (p.N + P.tile - 1) / P.tile * (P.tile == 32 ? 1 : a->dtype == ORTH_BF16 ? 2 : P.tile / 32);
  P.off_part = take((size_t)a->rows * p.n_part * 8);
  P.off_target = take((size_t)a->rows * 4);
  P.total = off;
  p.part = reinterpret_cast<float2*>(ws + P.off_part);
  p.ztarget = reinterpret_cast<float*>(ws + P.off_target);
  return P;
}
unsigned char* stand_in() { return reinterpret_cast<unsigned char*>(uintptr_t(1) << 44); }

// us of a product M x N x K on staged tiles, by their rounds.
double rows_time(int dtype, int64_t M, int64_t N, int64_t K) {
  auto tiles = [&](int64_t e) { return (double)((M + e - 1) / e) * (double)((N + e - 1) / e); };
  if (dtype == ORTH_F32)
    return (double)K * std::min(0.053 * std::ceil(tiles(128) / 256), 0.033 * std::max(0.5, tiles(64) / 512));
  return std::min((14 + 0.0235 * K) * std::ceil(tiles(256) / 256), (8 + 0.0155 * K) * std::ceil(tiles(128) / 512));
}

// The backward: x' (the rows with a target, padded to a multiple of 8
// columns), dz of one piece of the classes, and with several pieces the sum
// of dx in fp32.  In bf16 dz takes two rows (RowsProd::pairs), x' too.
struct XentVjpPlan {
  int two = 0;                  // 1: of that
  int piece = 0, ldz = 0, ldx = 0, ldw = 0;   // ldw: W's padded copy, 0: none
  int slices = 1, kslice = 0, dx_tile = 0;   // of a piece's dx product
  GradPlan dw, dw_last;         // of a piece's dW and the last one's, which may be smaller
  size_t off_x = 0, off_dz = 0, off_w = 0, off_sum = 0, off_slices = 0, total = 0;   // (dx's and dW's slices take turns)
};
XentVjpPlan xent_vjp_plan(const orth_linear_xent_args* a) {
  XentVjpPlan P;
  P.two = a->dtype == ORTH_BF16 ? 1 : 0;
  const int64_t es = esize(a->dtype), rows = std::max(a->rows, 1), held = rows << P.two;
  // pieces whose dz takes 256 MB at most (bf16: each of its two pieces), but of
  // 4096 classes at least; of multiples of 256 down to half of that, the one
  // whose products take the fewest rounds of tiles.  (4096 rows, 2048 features,
  // 50003 classes: two pieces of 24576 are 6 whole rounds of dz's 256-tiles and 3
  // of dW's each, 851 classes are left: 3.52 ms; pieces of 12288 3.84, of 25088
  // 3.75, one of all 3.75)
  int64_t piece = a->piece;
  if (!piece) {
    const int64_t most = std::max<int64_t>(4096, (256ll << 20) / (rows * es) / 256 * 256);
    if (most >= a->classes && a->dtype == ORTH_F32) piece = a->classes;
    double best = 0;
    const int64_t step = std::max<int64_t>(256, most / 128 / 256 * 256);   // (64 of them at most)
    for (int64_t p = std::min<int64_t>(most, (a->classes + 255) / 256 * 256); !a->piece && p >= std::max<int64_t>(most / 2, 4096);
         p -= step) {
      const int64_t whole = a->classes / p, rest = a->classes % p;
      auto time = [&](int64_t n) {
        return n ? rows_time(a->dtype, rows, n, a->features) + rows_time(a->dtype, n, a->features, held) + 10 : 0.0;
      };
      const double t = whole * time(p) + time(rest);
      if (!piece || t < best) {
        best = t;
        piece = p;
      }
    }
    if (!piece) piece = a->classes;
  }
  piece = std::min<int64_t>(piece, a->classes);
  P.piece = (int)piece;
  P.ldz = (int)((piece + 7) / 8 * 8);
  P.ldx = (a->features + 7) / 8 * 8;
  P.off_dz = align_up((size_t)held * P.ldx * es);
  P.off_w = P.off_dz + align_up((size_t)held * P.ldz * es);
  P.ldw = padded(a, a->w, a->ld_w);
  P.off_sum = P.off_w + (P.ldw ? align_up((size_t)a->classes * P.ldw * es) : 0);
  const size_t sum = align_up((size_t)a->rows * a->features * 4);
  P.off_slices = P.off_sum + (piece < a->classes ? sum : 0);
  // dx has few tiles and a long k: whole, or its k in slices on staged tiles or,
  // from few rows, on the kernel without staging, by the times (us) that they
  // take per round of workgroups and k, and to join.  Measured (us, dz and dx of
  // 93718 classes and 1344 features, whole tiles or slices without staging / the
  // slices this chooses): fp32, 128 rows 579 / 458; bf16 with dz in one piece 128
  // rows 241 / 137, 512 rows 954 / 326, 2048 rows 1581 / 1200 (in two, with what
  // this chooses: 173, 463, 1855).
  RowsProd d{};
  d.groups = 1;
  d.rows = d.M = (int)held;
  d.N = a->features;
  d.lda = P.ldz;
  d.ldb = P.ldw ? P.ldw : a->ld_w;
  d.B = P.ldw ? nullptr : a->w;
  d.b_pad8 = P.ldw ? 1 : 0;
  const bool f32 = a->dtype == ORTH_F32, dma = !f32 && rows_bf16_dma(d, false, true);
  const double k = (double)piece;
  double best = INFINITY;
  auto consider = [&](int tile, int64_t n, double per_k, double start) {
    const int64_t slice = ((piece + n - 1) / n + 63) / 64 * 64;
    const double join = n > 1 ? 6 + (double)n * a->rows * a->features * 2e-6 : 0;
    const double t = start + per_k * (double)std::min(slice, piece) + join;
    if (t >= best) return;
    best = t;
    P.dx_tile = tile;
    P.kslice = (int)std::min(slice, piece);
    P.slices = (int)((piece + P.kslice - 1) / P.kslice);
  };
  // us per k of w workgroups
  auto rate = [&](int tile, double w) {
    if (f32) return tile == 128 ? std::ceil(w / 256) * 0.053 : std::max(0.018, w / 512 * 0.033);
    if (tile == 256) return std::ceil(w / 256) * 0.024;
    return (w <= 256 ? 0.0095 : std::ceil(w / 512) * 0.0155) * (dma ? 1 : 2);
  };
  for (const int tile : {64, 128, 256}) {
    if (tile == (f32 ? 256 : 64) || (tile == 256 && !dma)) continue;
    const double tiles = (double)rows_blocks(d, false, tile);
    const int64_t most = std::max<int64_t>(1, std::min((int64_t)((tile == 256 ? 256 : 512) / tiles), piece / 512));
    for (int64_t n = 1; n <= most; ++n) consider(tile, n, rate(tile, tiles * n), 8);
  }
  const double tiles = (double)rows_blocks(d, false, 32);
  const int least = f32 ? 1024 : 2048;
  const int64_t n = std::min<int64_t>((int64_t)std::ceil(1024 / tiles), (piece + least - 1) / least);
  consider(32, n, tiles * n / 512 * (f32 ? 0.01 : 0.0045), 12);
  RowsProd w{};
  w.groups = 1;
  w.rows = w.K = (int)held;
  w.M = P.piece;
  w.N = a->features;
  w.lda = P.ldz;
  w.ldb = P.ldx;
  w.a_pad8 = w.b_pad8 = 1;
  P.dw = grad_plan(w, a->dtype);
  w.M = (int)((a->classes - 1) % piece + 1);
  P.dw_last = grad_plan(w, a->dtype);
  P.total = P.off_slices + std::max({P.slices > 1 ? (size_t)P.slices * a->rows * a->features * 4 : 0, P.dw.bytes,
                                     P.dw_last.bytes});
  return P;
}

}  // namespace
}  // namespace orth

extern "C" {

int orth_linear_xent_workspace_size(const orth_linear_xent_args* a, size_t* bytes) {
  if (!bytes) return invalid("bytes is NULL");
  const int rc = validate_xent(a);
  if (rc) return rc;
  *bytes = a->rows == 0 ? 0 : xent_plan(a, stand_in()).total;
  return ORTH_OK;
}

int orth_linear_xent(const orth_linear_xent_args* a, float* loss, float* lse, void* workspace, size_t workspace_bytes,
                     void* stream) {
  int rc = validate_xent(a);
  if (rc) return rc;
  if (a->rows == 0) return ORTH_OK;
  if (!loss || !lse) return invalid("NULL data pointer");
  const int64_t bl = (int64_t)a->rows * 4;
  for (const float* out : {loss, lse})
    if (overlap(out, bl, a->x, span(a->rows, a->ld_x, a->features, a->dtype)) || overlap(out, bl, a->targets, 2 * bl) ||
        overlap(out, bl, a->w, span(a->classes, a->ld_w, a->features, a->dtype)))
      return invalid("loss and lse must not overlap x, w or targets");
  if (overlap(loss, bl, lse, bl)) return invalid("loss and lse must not overlap");
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  const XentPlan P = xent_plan(a, ws ? ws : stand_in());
  rc = check_ws(workspace, workspace_bytes, P.total);
  if (rc) return rc;
  if (rows_blocks(P.logits, false, P.tile) > kMaxBlocks) return invalid("rows x classes too large");
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t pe = hipSuccess;
  if (P.ldw)
    pe = launch_pad(a->w, a->ld_w, ws + P.off_w, P.ldw, a->classes, a->features, a->dtype, nullptr, 1, 0, "xent_pad", s);
  if (P.ldx && pe == hipSuccess)
    pe = launch_pad(a->x, a->ld_x, ws + P.off_x, P.ldx, a->rows, a->features, a->dtype, nullptr, 1, 0, "xent_pad", s);
  rc = hip_check(pe != hipSuccess ? pe : launch(P.logits, a->dtype, false, false, ROWS_LSE, P.tile, "xent_logits", s), "orth_linear_xent");
  if (rc) return rc;
  timing_begin("xent_join", s);
  if (P.logits.n_part > 256)
    hipLaunchKernelGGL(xent_join_kernel<4>, dim3(std::min(a->rows, kMaxRowBlocks)), dim3(256), 0, s, P.logits.part, P.logits.n_part,
                       P.logits.ztarget, a->targets, a->rows, a->classes, loss, lse);
  else
    hipLaunchKernelGGL(xent_join_kernel<1>, dim3(std::min((a->rows + 3) / 4, kMaxRowBlocks)), dim3(256), 0, s, P.logits.part,
                       P.logits.n_part, P.logits.ztarget, a->targets, a->rows, a->classes, loss, lse);
  const hipError_t e = hipGetLastError();
  timing_end("xent_join", s);
  return hip_check(e, "orth_linear_xent");
}

int orth_linear_xent_vjp_workspace_size(const orth_linear_xent_args* a, size_t* bytes) {
  if (!bytes) return invalid("bytes is NULL");
  const int rc = validate_xent_vjp(a);
  if (rc) return rc;
  *bytes = a->rows == 0 ? 0 : xent_vjp_plan(a).total;
  return ORTH_OK;
}

int orth_linear_xent_vjp(const orth_linear_xent_args* a, const float* lse, const float* grad_loss, void* grad_x,
                         int64_t ld_grad_x, void* grad_w, int64_t ld_grad_w, void* workspace, size_t workspace_bytes,
                         void* stream) {
  int rc = validate_xent_vjp(a);
  if (rc) return rc;
  if ((a->rows > 0 && (!lse || !grad_loss)) || (!grad_x && !grad_w)) return invalid("NULL data pointer");
  if ((grad_x && ld_grad_x < a->features) || (grad_w && ld_grad_w < a->features))
    return invalid("leading dimension below the columns");
  if ((grad_x && far(a->rows, ld_grad_x)) || (grad_w && far(a->classes, ld_grad_w)))
    return invalid("leading dimension too large");
  const int64_t bx = span(a->rows, a->ld_x, a->features, a->dtype), bw = span(a->classes, a->ld_w, a->features, a->dtype);
  const int64_t bgx = grad_x ? span(a->rows, ld_grad_x, a->features, a->dtype) : 0;
  const int64_t bgw = grad_w ? span(a->classes, ld_grad_w, a->features, a->dtype) : 0;
  if ((grad_x && (overlap(grad_x, bgx, a->x, bx) || overlap(grad_x, bgx, a->w, bw))) ||
      (grad_w && (overlap(grad_w, bgw, a->x, bx) || overlap(grad_w, bgw, a->w, bw))) ||
      (grad_x && grad_w && overlap(grad_x, bgx, grad_w, bgw)))
    return invalid("grad_x and grad_w must not overlap x, w or each other");
  const int64_t bl = (int64_t)a->rows * 4;
  auto hits = [&](const void* g, int64_t n) {
    return g && (overlap(g, n, lse, bl) || overlap(g, n, grad_loss, bl) || overlap(g, n, a->targets, 2 * bl));
  };
  if (hits(grad_x, bgx) || hits(grad_w, bgw)) return invalid("grad_x and grad_w must not overlap lse, grad_loss or targets");
  const XentVjpPlan P = a->rows > 0 ? xent_vjp_plan(a) : XentVjpPlan{};
  hipStream_t s = static_cast<hipStream_t>(stream);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  if (a->rows > 0) {
    rc = check_ws(workspace, workspace_bytes, P.total);
    if (rc) return rc;
  }
  const int es = (int)esize(a->dtype);
  auto product = [&](const void* A, int64_t lda, const void* B, int64_t ldb, int rows, int N, int K) {
    RowsProd p{};
    p.A = A;
    p.lda = lda;
    p.B = B;
    p.ldb = ldb;
    p.groups = 1;
    p.rows = p.M = rows;
    p.N = N;
    p.K = p.kslice = K;
    p.c_dtype = a->dtype;
    return p;
  };
  if (a->rows == 0) {
    // no row: dW = 0 (a product over no rows)
    if (!grad_w) return ORTH_OK;
    RowsProd p = product(a->x, a->ld_x, a->x, a->ld_x, 0, a->features, 0);
    p.M = a->classes;
    p.C = grad_w;
    p.ldc = ld_grad_w;
    const int tile = tile_of(p, a->dtype, true, true);
    if (rows_blocks(p, true, tile) > kMaxBlocks) return invalid("classes x features too large");
    return hip_check(launch(p, a->dtype, true, true, ROWS_STORE, tile, "xent_grad_w", s), "orth_linear_xent_vjp");
  }
  void* x = ws;
  void* dz = ws + P.off_dz;
  float* sum = reinterpret_cast<float*>(ws + P.off_sum);
  const int held = a->rows << P.two;
  struct Step {
    RowsProd p;
    bool at, bt;
    int epi, tile;
    const char* name;
    RowsJoin join;   // to launch behind it
  };
  // dW needs x with zeros for the rows without a target; dz's values of those
  // are zeros whatever x holds, so without dW the copy is made for its padding
  // only.  The kernel without staging takes the copy along.
  const bool copy = grad_w || padded(a, a->x, a->ld_x);
  const bool along = copy && tile_of(product(a->x, a->ld_x, P.ldw ? ws + P.off_w : a->w, P.ldw ? P.ldw : a->ld_w, a->rows,
                                             P.piece, a->features),
                                     a->dtype, false, false) == 32;
  // the products of the piece that starts at class c0
  auto steps_of = [&](int c0, Step* st) {
    const int n = std::min(P.piece, a->classes - c0);
    const int64_t ldw = P.ldw ? P.ldw : a->ld_w;
    const char* w = (P.ldw ? reinterpret_cast<const char*>(ws + P.off_w) : static_cast<const char*>(a->w)) + c0 * ldw * es;
    int k = 0;
    const bool first = along && c0 == 0, own = first || !copy;
    RowsProd z = product(own ? a->x : x, own ? a->ld_x : (int64_t)P.ldx << P.two, w, ldw, a->rows, n, a->features);
    z.copy = first ? x : nullptr;
    z.ld_copy = P.ldx;
    z.twice = P.two;
    z.C = dz;
    z.ldc = (int64_t)P.ldz << P.two;
    z.c_low = P.two ? P.ldz : 0;
    z.col0 = c0;
    z.classes = a->classes;
    z.scale = a->scale;
    z.targets = a->targets;
    z.lse = lse;
    z.grad_loss = grad_loss;
    st[k++] = {z, false, false, ROWS_DZ, first ? 32 : tile_of(z, a->dtype, false, false), "xent_dz"};
    RowsJoin join{};
    if (grad_x) {
      RowsProd d = product(dz, P.ldz, w, ldw, held, a->features, n);
      d.pairs = P.two;
      d.b_pad8 = P.ldw ? 1 : 0;
      d.C = grad_x;
      d.ldc = ld_grad_x;
      const bool one = P.piece >= a->classes;
      d.sum = one ? nullptr : sum;
      d.add = c0 > 0;
      d.last = c0 + n >= a->classes;
      d.kslice = P.kslice;
      d.slices = reinterpret_cast<float*>(ws + P.off_slices);
      if (P.slices > 1)
        join = {d.slices, d.sum, d.C, d.ldc, a->rows, d.N, (n + P.kslice - 1) / P.kslice, d.add, d.last, d.c_dtype};
      st[k++] = {d, false, true, P.slices > 1 ? (int)ROWS_SLICE : one ? (int)ROWS_STORE : (int)ROWS_SUM, P.dx_tile,
                 "xent_grad_x"};
    }
    if (grad_w) {
      RowsProd d = product(dz, P.ldz, x, P.ldx, held, a->features, held);
      d.M = n;
      d.a_pad8 = d.b_pad8 = 1;
      d.C = static_cast<char*>(grad_w) + (int64_t)c0 * ld_grad_w * es;
      d.ldc = ld_grad_w;
      const GradPlan& g = c0 + n >= a->classes ? P.dw_last : P.dw;
      // (dW's slices take the place of dx's.  A staged tile's launch holds one or
      // two workgroups per compute unit, of which a join keeps each for 2 us:
      // 8192 of them 65 us, where a launch of their own takes 17)
      if (!g.kslice && rows_join_blocks(join) <= (g.tile == kOuter ? 4096 : 512)) d.join = join;
      st[k++] = {d, true, true, ROWS_STORE, g.tile, "xent_grad_w"};
    }
    if (k > 1 && join.slices && !st[k - 1].p.join.slices) st[1].join = join;
    return k;
  };
  Step st[3];
  for (int i = 0, k = steps_of(0, st); i < k; ++i)   // (the first piece is a largest one)
    if ((st[i].at ? grad_blocks(st[i].p, a->dtype, P.piece >= a->classes ? P.dw_last : P.dw) : rows_blocks(st[i].p, false, st[i].tile)) > kMaxBlocks) return invalid("rows x piece too large");
  hipError_t e = hipSuccess;
  if (copy && !along)
    e = launch_pad(a->x, a->ld_x, x, P.ldx, a->rows, a->features, a->dtype, a->targets, a->classes, P.two, "xent_rows", s);
  if (P.ldw && e == hipSuccess)
    e = launch_pad(a->w, a->ld_w, ws + P.off_w, P.ldw, a->classes, a->features, a->dtype, nullptr, 1, 0, "xent_pad", s);
  for (int c0 = 0; c0 < a->classes && e == hipSuccess; c0 += P.piece) {
    const int k = steps_of(c0, st);
    for (int i = 0; i < k && e == hipSuccess; ++i) {
      const RowsProd& q = st[i].p;
      if (st[i].at) {
        e = launch_grad(q, a->dtype, c0 + q.M >= a->classes ? P.dw_last : P.dw, ws + P.off_slices, st[i].name, "xent_grad_w_join", s);
      } else if (st[i].epi == ROWS_SLICE) {
        e = st[i].tile == 32 ? launch_rows_direct(q, a->dtype, true, ROWS_SLICE, (q.K + q.kslice - 1) / q.kslice, st[i].name, s)
                         : launch(q, a->dtype, false, true, ROWS_SLICE, st[i].tile, st[i].name, s);
        if (e == hipSuccess && st[i].join.slices) e = launch_rows_join(st[i].join, "xent_grad_x_join", s);
      } else {
        e = launch(q, a->dtype, st[i].at, st[i].bt, st[i].epi, st[i].tile, st[i].name, s);
      }
    }
    if (a->classes - c0 <= P.piece) break;   // (c0 + piece may pass 2^31)
  }
  return hip_check(e, "orth_linear_xent_vjp");
}

}  // extern "C"
