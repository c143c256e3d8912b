// Global norm of a list of gradients, n = sqrt(sum of every value's square),
// and clipping by it: out = min(1, max_norm / (n + eps)) grad.
//
// Both kernels walk the list as one line of 16-byte vectors, dealt to a fixed
// number of workgroups in equal runs whatever the tensors' sizes; they are
// bound by HBM.  2 GB of bf16: the norm 315 us (6.8 TB/s; 405 with loads
// through the caches), the clipping 837 us (5.1 TB/s read and written).  Squares
// are summed in fp64 (fp32 squares overflow from 1.8e19 on), one partial sum
// per workgroup; the clipping kernel's workgroups each add all partial sums
// in the same order, so the result does not depend on timing.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdio>
#include <new>
#include <vector>

#include "rows.h"

namespace orth {

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 4 * kThreads;   // vectors per step of a workgroup
constexpr int kBlocks = 2048;          // eight workgroups per compute unit
constexpr int kSmallThreads = 1024;    // the one workgroup of a short list, which holds
constexpr int kSmallPer = 4;           // so many vectors per thread
constexpr int kInline = 56;            // tensors whose table fits the kernel arguments
constexpr int64_t kCached = 128 << 20; // lists up to this may be read a second time from the last-level cache

struct GradDesc {
  const void* in;
  void* out;
  int64_t ld_in, ld_out, cols;   // a contiguous tensor is one row
  int64_t first;                 // chunks before this tensor
  int32_t rows, dtype;
  int64_t last;                  // chunks up to its end
};
// The table in the kernel arguments, with a compact index of it: the arguments
// are host memory, of which every workgroup then reads a few lines only.
struct GradTable {
  GradDesc d[kInline];
  int32_t last[kInline];   // chunks up to each tensor's end (INT32_MAX: more, or no tensor)
};

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
  return v;
}
// the workgroup's sum, on every thread
__device__ __forceinline__ double group_sum(double v, double* lds) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) v += lds[w];
  return v;
}

__device__ __forceinline__ int find_tensor(const GradTable& t, int, int64_t c) {
  const int lane = threadIdx.x & 63;
  return __ffsll(__ballot(lane < kInline && c < t.last[lane < kInline ? lane : 0])) - 1;
}
__device__ __forceinline__ const GradDesc& desc_of(const GradTable& t, int i) { return t.d[i]; }
__device__ __forceinline__ const GradDesc& desc_of(const GradDesc* d, int i) { return d[i]; }

// The tensor that holds chunk c: the last one with first <= c that is not
// empty.  64 candidates at a time.
__device__ __forceinline__ int find_tensor(const GradDesc* d, int n, int64_t c) {
  const int lane = threadIdx.x & 63;
  int lo = 0, len = n;   // the answer is in [lo, lo + len)
  while (len > 1) {
    const int step = (len + 63) / 64, at = lo + lane * step;
    const unsigned long long le = __ballot(at < lo + len && d[at].first <= c);
    const int k = le ? 63 - __clzll(le) : 0;
    const int end = lo + len;
    lo += k * step;
    len = min(step, end - lo);
  }
  return lo;
}

// Vectors of a row of `cols` values.
__host__ __device__ __forceinline__ int64_t row_vectors(int64_t cols, int dtype) {
  return dtype == ORTH_BF16 ? (cols + 7) >> 3 : (cols + 3) >> 2;
}

// Vector v of a tensor: its place and its values that exist.
struct Place {
  int64_t row, col;
  int n;
};
__device__ __forceinline__ Place place(const GradDesc& d, int64_t v) {
  const int len = d.dtype == ORTH_BF16 ? 8 : 4;
  Place p{0, v * len, len};
  if (d.rows > 1) {
    const int64_t per = row_vectors(d.cols, d.dtype);
    p.row = ((v | per) >> 32) ? v / per : (int64_t)((uint32_t)v / (uint32_t)per);
    p.col = (v - p.row * per) * len;
  }
  p.n = (int)min((int64_t)len, d.cols - p.col);
  return p;
}
// NT: past the caches (lists that do not fit them anyway).
template <bool NT, typename V>
__device__ __forceinline__ V get(const void* p) {
  if constexpr (NT) return __builtin_nontemporal_load((const ORTH_GLOBAL V*)p);
  return *(const ORTH_GLOBAL V*)p;
}
template <bool NT, typename V>
__device__ __forceinline__ void put(void* p, V v) {
  if constexpr (NT)
    __builtin_nontemporal_store(v, (ORTH_GLOBAL V*)p);
  else
    *(ORTH_GLOBAL V*)p = v;
}
// A vector's values as fp32.
template <int DT>
__device__ __forceinline__ void values(orth_u32x4_a2 w, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (DT == ORTH_BF16) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    } else {
      x[i] = __uint_as_float(w[i]);
    }
  }
}
template <int DT>
__device__ __forceinline__ orth_u32x4_a2 packed(const float (&x)[8]) {
  if (DT == ORTH_BF16)
    return orth_u32x4_a2{cvt2_bf16(x[0], x[1]), cvt2_bf16(x[2], x[3]), cvt2_bf16(x[4], x[5]), cvt2_bf16(x[6], x[7])};
  return orth_u32x4_a2{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
}
// The same of n values of a tensor, whole vectors in one load or store.
__device__ __forceinline__ void load_some(const GradDesc& g, int64_t at, int n, float (&x)[8]) {
  if (g.dtype == ORTH_BF16 && n == 8) {
    values<ORTH_BF16>(get<false, orth_u32x4_a2>(static_cast<const uint16_t*>(g.in) + at), x);
  } else if (g.dtype == ORTH_F32 && n == 4) {
    values<ORTH_F32>(get<false, orth_u32x4_a2>(static_cast<const float*>(g.in) + at), x);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) x[e] = load_as_f32(g.in, at + e, g.dtype);
  }
}
__device__ __forceinline__ void store_some(const GradDesc& g, int64_t at, int n, const float (&x)[8]) {
  if (g.dtype == ORTH_BF16 && n == 8) {
    put<false>(static_cast<uint16_t*>(g.out) + at, packed<ORTH_BF16>(x));
  } else if (g.dtype == ORTH_F32 && n == 4) {
    put<false>(static_cast<float*>(g.out) + at, packed<ORTH_F32>(x));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) store_from_f32(g.out, at + e, g.dtype, x[e]);
  }
}

constexpr int kPer = kChunk / kThreads;   // vectors of a chunk per thread

// Whether every vector of the chunk at v0 is whole and they follow each other.
__device__ __forceinline__ bool whole_chunk(const GradDesc& g, int64_t v0) {
  return g.rows == 1 && (v0 + kChunk) * (g.dtype == ORTH_BF16 ? 8 : 4) <= g.cols;
}

// This workgroup's chunks, f(tensor, first vector, end vector) for each;
// backwards: the last first.
template <typename D, typename F>
__device__ __forceinline__ void walk(const D& d, int n, int64_t chunks, bool backwards, F&& f) {
  const int64_t lo = chunks * blockIdx.x / gridDim.x, hi = chunks * (blockIdx.x + 1) / gridDim.x;
  if (lo >= hi) return;
  int t = __builtin_amdgcn_readfirstlane(find_tensor(d, n, backwards ? hi - 1 : lo));
  GradDesc g = desc_of(d, t);
  int64_t nv = g.rows * row_vectors(g.cols, g.dtype);
  for (int64_t k = 0; k < hi - lo; ++k) {
    const int64_t c = backwards ? hi - 1 - k : lo + k;
    if (c >= g.last || c < g.first) {
      t += backwards ? -1 : 1;   // (no tensor of the table is empty)
      g = desc_of(d, t);
      nv = g.rows * row_vectors(g.cols, g.dtype);
    }
    const int64_t v0 = (c - g.first) * kChunk;
    f(g, v0, min(v0 + kChunk, nv));
  }
}

template <int DT, bool NT>
__device__ __forceinline__ void norm_whole(const GradDesc& g, int64_t v0, double& sum) {
  const char* at = static_cast<const char*>(g.in) + (v0 + threadIdx.x) * 16;
  orth_u32x4_a2 w[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) w[i] = get<NT, orth_u32x4_a2>(at + i * kThreads * 16);
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    float x[8];
    values<DT>(w[i], x);
#pragma unroll
    for (int e = 0; e < (DT == ORTH_BF16 ? 8 : 4); ++e) sum = fma((double)x[e], (double)x[e], sum);
  }
}
template <bool NT, typename D>
__device__ __forceinline__ void norm_part(const D& d, int n, int64_t chunks, double* partial) {
  __shared__ double lds[kThreads / 64];
  double sum = 0.0;
  walk(d, n, chunks, false, [&](const GradDesc& g, int64_t v0, int64_t end) {
    if (whole_chunk(g, v0)) {
      if (g.dtype == ORTH_BF16)
        norm_whole<ORTH_BF16, NT>(g, v0, sum);
      else
        norm_whole<ORTH_F32, NT>(g, v0, sum);
      return;
    }
    for (int64_t v = v0 + threadIdx.x; v < end; v += kThreads) {
      const Place p = place(g, v);
      float x[8] = {};
      load_some(g, p.row * g.ld_in + p.col, p.n, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fma((double)x[e], (double)x[e], sum);
    }
  });
  sum = group_sum(sum, lds);
  if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

// sqrt of the sum of all partial sums, on every thread
__device__ __forceinline__ double whole_norm(const double* partial, int n, double* lds) {
  double v = 0.0;
  for (int i = threadIdx.x; i < n; i += kThreads) v += gld_f64(partial, i);
  return sqrt(group_sum(v, lds));
}

// (a NaN norm makes every value NaN)
__device__ __forceinline__ float clip_factor(double norm, float max_norm, float eps) {
  const double ratio = (double)max_norm / (norm + (double)eps);
  return norm == 0.0 || ratio > 1.0 ? 1.f : (float)ratio;
}
template <int DT, bool NT>
__device__ __forceinline__ void clip_whole(const GradDesc& g, int64_t v0, float factor) {
  const int64_t off = (v0 + threadIdx.x) * 16;
  const char* in = static_cast<const char*>(g.in) + off;
  char* out = static_cast<char*>(g.out) + off;
  orth_u32x4_a2 w[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) w[i] = get<NT, orth_u32x4_a2>(in + i * kThreads * 16);
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    float x[8];
    values<DT>(w[i], x);
#pragma unroll
    for (int e = 0; e < (DT == ORTH_BF16 ? 8 : 4); ++e) x[e] *= factor;
    put<NT>(out + i * kThreads * 16, packed<DT>(x));
  }
}
template <bool NT, typename D>
__device__ __forceinline__ void clip_part(const D& d, int n, int64_t chunks, const double* partial, int n_partial,
                                          float* norm, float max_norm, float eps) {
  __shared__ double lds[kThreads / 64];
  // (a given norm when there are no partial sums)
  const double total = n_partial ? whole_norm(partial, n_partial, lds) : (double)norm[0];
  if (n_partial && blockIdx.x == 0 && threadIdx.x == 0) norm[0] = (float)total;
  const float factor = clip_factor(total, max_norm, eps);
  walk(d, n, chunks, !NT, [&](const GradDesc& g, int64_t v0, int64_t end) {
    if (factor == 1.f && g.in == g.out) return;
    if (whole_chunk(g, v0)) {
      if (g.dtype == ORTH_BF16)
        clip_whole<ORTH_BF16, NT>(g, v0, factor);
      else
        clip_whole<ORTH_F32, NT>(g, v0, factor);
      return;
    }
    for (int64_t v = v0 + threadIdx.x; v < end; v += kThreads) {
      const Place p = place(g, v);
      float x[8] = {};
      load_some(g, p.row * g.ld_in + p.col, p.n, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] *= factor;
      store_some(g, p.row * g.ld_out + p.col, p.n, x);
    }
  });
}

template <bool NT>
__global__ __launch_bounds__(kThreads) void grad_norm_kernel(const GradDesc* d, int n, int64_t chunks,
                                                             double* partial) {
  norm_part<NT>(d, n, chunks, partial);
}
template <bool NT>
__global__ __launch_bounds__(kThreads) void grad_norm_inline_kernel(const GradTable t, int n, int64_t chunks,
                                                                    double* partial) {
  norm_part<NT>(t, n, chunks, partial);
}
template <bool NT>
__global__ __launch_bounds__(kThreads) void grad_clip_kernel(const GradDesc* d, int n, int64_t chunks,
                                                             const double* partial, int n_partial, float* norm,
                                                             float max_norm, float eps) {
  clip_part<NT>(d, n, chunks, partial, n_partial, norm, max_norm, eps);
}
template <bool NT>
__global__ __launch_bounds__(kThreads) void grad_clip_inline_kernel(const GradTable t, int n, int64_t chunks,
                                                                    const double* partial, int n_partial, float* norm,
                                                                    float max_norm, float eps) {
  clip_part<NT>(t, n, chunks, partial, n_partial, norm, max_norm, eps);
}
// A short list in one launch: one workgroup holds every value in registers
// between the norm and the products.  (42 tensors of 48 or 192 values: 12.4
// us a call with two launches, 9.6 this way.)
struct SmallIndex {
  int32_t first[kInline + 1];   // vectors before each tensor, and in all
};
__global__ __launch_bounds__(kSmallThreads) void grad_small_kernel(const GradTable t, const SmallIndex ix, int n,
                                                                   float* norm, int clip, float max_norm, float eps) {
  __shared__ int first[kInline + 1];
  __shared__ GradDesc desc[kInline];
  __shared__ double lds[kSmallThreads / 64];
  const int tid = threadIdx.x, total = ix.first[n];
  if (tid <= n) first[tid] = ix.first[tid];
  for (int i = tid; i < n * (int)(sizeof(GradDesc) / 8); i += kSmallThreads)
    reinterpret_cast<uint64_t*>(desc)[i] = reinterpret_cast<const uint64_t*>(t.d)[i];
  __syncthreads();
  auto find = [&](int v) {
    int lo = 0, hi = n;   // first[lo] <= v < first[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      (first[mid] <= v ? lo : hi) = mid;
    }
    return lo;
  };
  float x[kSmallPer][8];
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < kSmallPer; ++i) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[i][e] = 0.f;
    const int v = i * kSmallThreads + tid;
    if (v < total) {
      const int k = find(v);
      const Place p = place(desc[k], v - first[k]);
      load_some(desc[k], p.row * desc[k].ld_in + p.col, p.n, x[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < kSmallPer; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fma((double)x[i][e], (double)x[i][e], sum);
  sum = wave_sum(sum);
  if ((tid & 63) == 0) lds[tid >> 6] = sum;
  __syncthreads();
  sum = 0.0;
  for (int w = 0; w < kSmallThreads / 64; ++w) sum += lds[w];
  const double whole = sqrt(sum);
  if (tid == 0) norm[0] = (float)whole;
  if (!clip) return;
  const float factor = clip_factor(whole, max_norm, eps);
#pragma unroll
  for (int i = 0; i < kSmallPer; ++i) {
    const int v = i * kSmallThreads + tid;
    if (v < total) {
      const int k = find(v);
      const GradDesc& g = desc[k];
      if (factor == 1.f && g.in == g.out) continue;
      const Place p = place(g, v - first[k]);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i][e] *= factor;
      store_some(g, p.row * g.ld_out + p.col, p.n, x[i]);
    }
  }
}

__global__ __launch_bounds__(kThreads) void grad_norm_join_kernel(const double* partial, int n_partial, float* norm) {
  __shared__ double lds[kThreads / 64];
  const double total = whole_norm(partial, n_partial, lds);
  if (threadIdx.x == 0) norm[0] = (float)total;
}

int invalid(const char* msg) { return report_error(ORTH_EINVAL, msg); }

// A tensor's rows as one run of bytes, with the gaps between them, and whether it
// has none.
struct Run {
  uintptr_t at, end;
  bool flat;
};
Run run_of(const void* p, const orth_grad& g, int64_t ld) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p), es = g.dtype == ORTH_BF16 ? 2 : 4;
  return {at, at + ((uintptr_t)(g.rows - 1) * (uintptr_t)ld + (uintptr_t)g.cols) * es, g.rows == 1 || ld == g.cols};
}
// Whether a gradient and its output share bytes without being the same.  Rows
// of one stride share none if they lie side by side in it.
bool shares(const orth_grad& g) {
  if (g.grad == g.out) return false;
  const Run a = run_of(g.grad, g, g.ld_grad), b = run_of(g.out, g, g.ld_out);
  if (a.at >= b.end || b.at >= a.end) return false;
  if (g.ld_grad != g.ld_out || g.rows == 1) return true;
  const uintptr_t es = g.dtype == ORTH_BF16 ? 2 : 4, ld = (uintptr_t)g.ld_out * es, cols = (uintptr_t)g.cols * es;
  const uintptr_t d = (a.at < b.at ? b.at - a.at : a.at - b.at) % ld;
  return d < cols || d + cols > ld;
}

int validate(const orth_grad* g, int32_t n, bool outs) {
  if (n < 0) return invalid("n must be >= 0");
  if (n > 0 && !g) return invalid("grads is NULL");
  for (int i = 0; i < n; ++i) {
    if (g[i].rows < 0 || g[i].cols < 0) return invalid("rows and cols must be >= 0");
    if (g[i].dtype != ORTH_F32 && g[i].dtype != ORTH_BF16) return invalid("unknown dtype");
    if (g[i].rows == 0 || g[i].cols == 0) continue;
    if (!g[i].grad || (outs && !g[i].out)) return invalid("NULL data pointer");
    if (g[i].ld_grad < g[i].cols || (outs && g[i].ld_out < g[i].cols))
      return invalid("leading dimension below the columns");
    if (outs && g[i].grad == g[i].out && g[i].ld_grad != g[i].ld_out)
      return invalid("in place needs equal leading dimensions");
    // (as in the row-grouped products: past any memory)
    if ((double)g[i].rows * (double)g[i].ld_grad > 0x1p48 || (outs && (double)g[i].rows * (double)g[i].ld_out > 0x1p48))
      return invalid("leading dimension too large");
    if (outs && shares(g[i])) return invalid("an output must be its gradient or apart from it");
  }
  if (outs) {
    std::vector<Run> to;
    for (int i = 0; i < n; ++i)
      if (g[i].rows && g[i].cols) to.push_back(run_of(g[i].out, g[i], g[i].ld_out));
    std::sort(to.begin(), to.end(), [](const Run& a, const Run& b) { return a.at < b.at; });
    // (runs with gaps may lie in each other's)
    uintptr_t flat_end = 0;
    for (size_t i = 0; i < to.size(); ++i) {
      if (i > 0 && to[i].at == to[i - 1].at) return invalid("two outputs are the same");
      if (!to[i].flat) continue;
      if (to[i].at < flat_end) return invalid("two outputs overlap");
      flat_end = to[i].end;
    }
  }
  return ORTH_OK;
}

struct Plan {
  std::vector<GradDesc> d;   // tensors that are not empty
  int64_t chunks = 0, bytes = 0, vectors = 0;
  int blocks = 1;
};
Plan make_plan(const orth_grad* g, int32_t n, bool outs) {
  Plan P;
  for (int i = 0; i < n; ++i) {
    if (!g[i].rows || !g[i].cols) continue;
    GradDesc d{g[i].grad, outs ? g[i].out : nullptr, g[i].ld_grad, g[i].ld_out, g[i].cols, P.chunks, g[i].rows, g[i].dtype, 0};
    const bool flat = g[i].rows == 1 || (d.ld_in == d.cols && (!d.out || d.ld_out == d.cols));
    if (flat) {
      d.cols *= d.rows;
      d.rows = 1;
    }
    P.chunks += (d.rows * row_vectors(d.cols, d.dtype) + kChunk - 1) / kChunk;
    d.last = P.chunks;
    P.vectors += d.rows * row_vectors(d.cols, d.dtype);
    P.bytes += (int64_t)g[i].rows * g[i].cols * (g[i].dtype == ORTH_BF16 ? 2 : 4);
    P.d.push_back(d);
  }
  P.blocks = (int)std::min<int64_t>(kBlocks, std::max<int64_t>(1, P.chunks));
  return P;
}
// (the table of a list that does not fit the kernel arguments, then the
// partial sums)
size_t table_bytes(int32_t n) { return n > kInline ? ((size_t)n * sizeof(GradDesc) + 255) / 256 * 256 : 0; }
size_t workspace_bytes_of(int32_t n) { return table_bytes(n) + kBlocks * sizeof(double); }

int hip_failed(const char* entry, hipError_t e) {
  char buf[256];
  snprintf(buf, sizeof buf, "%s: %s", entry, hipGetErrorString(e));
  return report_error(ORTH_EHIP, buf);
}

// The body of both entry points: the norm into norm[0], and (clip) the
// outputs.
int run(const orth_grad* g, int32_t n, const orth_clip_opts* o, float* norm, void* workspace, size_t workspace_bytes,
        hipStream_t s, const char* entry) {
  int rc = validate(g, n, o != nullptr);
  if (rc) return rc;
  if (!norm) return invalid("norm is NULL");
  if (!workspace) return report_error(ORTH_EWORKSPACE, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(workspace) % 256)
    return report_error(ORTH_EWORKSPACE, "workspace must be 256-byte aligned");
  if (workspace_bytes < workspace_bytes_of(n)) return report_error(ORTH_EWORKSPACE, "workspace too small");
  const Plan P = make_plan(g, n, o != nullptr);
  const int nd = (int)P.d.size();
  const bool table = nd > kInline;
  const GradDesc* dev = static_cast<const GradDesc*>(workspace);
  double* partial = reinterpret_cast<double*>(static_cast<unsigned char*>(workspace) + table_bytes(n));
  GradTable t{};
  if (table) {
    rc = upload_table(P.d.data(), P.d.size() * sizeof(GradDesc), workspace, s);
    if (rc) return rc;
  } else {
    std::copy(P.d.begin(), P.d.end(), t.d);
    for (int i = 0; i < kInline; ++i)
      t.last[i] = i + 1 < nd ? (int32_t)std::min<int64_t>(P.d[i].last, INT32_MAX) : INT32_MAX;
  }
  const dim3 grid(P.blocks), block(kThreads);
  const bool measure = !o || !o->norm_given;
  const bool nt = P.bytes > kCached;
  if (measure && !table && P.vectors <= kSmallThreads * kSmallPer) {
    SmallIndex ix{};
    for (int i = 0; i < nd; ++i)
      ix.first[i + 1] = ix.first[i] + (int)(t.d[i].rows * row_vectors(t.d[i].cols, t.d[i].dtype));
    const char* name = o ? "grad_clip" : "grad_norm";
    timing_begin(name, s);
    hipLaunchKernelGGL(grad_small_kernel, dim3(1), dim3(kSmallThreads), 0, s, t, ix, nd, norm, o ? 1 : 0,
                       o ? o->max_norm : 0.f, o ? o->eps : 0.f);
    const hipError_t e = hipGetLastError();
    timing_end(name, s);
    return e == hipSuccess ? (int)ORTH_OK : hip_failed(entry, e);
  }
  hipError_t e = hipSuccess;
  if (measure) {
    timing_begin("grad_norm", s);
    if (table)
      hipLaunchKernelGGL(nt ? grad_norm_kernel<true> : grad_norm_kernel<false>, grid, block, 0, s, dev, nd, P.chunks,
                         partial);
    else
      hipLaunchKernelGGL(nt ? grad_norm_inline_kernel<true> : grad_norm_inline_kernel<false>, grid, block, 0, s, t, nd,
                         P.chunks, partial);
    e = hipGetLastError();
    timing_end("grad_norm", s);
  }
  if (e == hipSuccess && !o) {
    timing_begin("grad_norm_join", s);
    hipLaunchKernelGGL(grad_norm_join_kernel, dim3(1), block, 0, s, partial, P.blocks, norm);
    e = hipGetLastError();
    timing_end("grad_norm_join", s);
  } else if (e == hipSuccess) {
    const int np = measure ? P.blocks : 0;
    timing_begin("grad_clip", s);
    if (table)
      hipLaunchKernelGGL(nt ? grad_clip_kernel<true> : grad_clip_kernel<false>, grid, block, 0, s, dev, nd, P.chunks,
                         partial, np, norm, o->max_norm, o->eps);
    else
      hipLaunchKernelGGL(nt ? grad_clip_inline_kernel<true> : grad_clip_inline_kernel<false>, grid, block, 0, s, t, nd,
                         P.chunks, partial, np, norm, o->max_norm, o->eps);
    e = hipGetLastError();
    timing_end("grad_clip", s);
  }
  return e == hipSuccess ? (int)ORTH_OK : hip_failed(entry, e);
}

// no C++ exception leaves the C ABI
template <typename F>
int guarded(F&& f) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return report_error(ORTH_EHIP, "out of host memory");
  }
}

}  // namespace

}  // namespace orth

using namespace orth;

extern "C" {

int orth_grad_norm_workspace_size(const orth_grad* grads, int32_t n, size_t* bytes) {
  if (!bytes) return invalid("bytes is NULL");
  return guarded([&] {
    const int rc = validate(grads, n, false);
    if (rc) return rc;
    *bytes = workspace_bytes_of(n);
    return (int)ORTH_OK;
  });
}

int orth_grad_norm_batched(const orth_grad* grads, int32_t n, float* norm, void* workspace, size_t workspace_bytes,
                           void* stream) {
  return guarded([&] {
    return run(grads, n, nullptr, norm, workspace, workspace_bytes, static_cast<hipStream_t>(stream),
               "orth_grad_norm_batched");
  });
}

int orth_grad_clip_batched(const orth_grad* grads, int32_t n, const orth_clip_opts* opts, float* norm, void* workspace,
                           size_t workspace_bytes, void* stream) {
  if (!opts) return invalid("opts is NULL");
  if (!(opts->max_norm >= 0.f) || !std::isfinite(opts->max_norm)) return invalid("max_norm must be finite and >= 0");
  if (!(opts->eps >= 0.f) || !std::isfinite(opts->eps)) return invalid("eps must be finite and >= 0");
  if (opts->norm_given != 0 && opts->norm_given != 1) return invalid("norm_given must be 0 or 1");
  return guarded([&] {
    return run(grads, n, opts, norm, workspace, workspace_bytes, static_cast<hipStream_t>(stream),
               "orth_grad_clip_batched");
  });
}

}  // extern "C"
