// Products grouped along K with few rows per group (rows.h has the
// descriptor): the gradient of a matrix from a handful of rows, bound by
// writing it.  A wave takes 32 rows of C and 128 columns, straight from memory
// into MFMA fragments and from the accumulators back: lane l of its four 32 x
// 32 tiles holds columns 4 l to 4 l + 3, so that loads and stores take whole
// lines (with pairs of columns, 128 bytes a row: 16 matrices of 4096^2 from 8
// rows each, bf16 161 us, this way 117 = 4.6 TB/s, fp32 303 and 199 = 5.4 TB/s).
// bf16 operands run on the 32x32x16 MFMA, fp32 ones on the fp32 32x32x2, exact
// products at a rate that is no limit for so few k's.
#include "rows.h"

namespace orth {

typedef orth_f32x16 f32x16;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

namespace {

// Blocks of 32 rows of C that a wave takes in turn, with up to 16 k's of B in
// registers: where that leaves work for all units.  Measured (us, 1 / 4), 16
// matrices of 4096^2, 8 rows each: bf16 148 / 117, fp32 241 / 199; one of 50000 x
// 2048 (6256 workgroups of one block): bf16 37 / 47, fp32
// 98 / 81.
int outer_rb(const RowsProd& p, int dtype) {
  const int64_t blocks = (int64_t)((p.N + 127) / 128) * ((p.M + 127) / 128) * p.groups;
  return blocks >= (dtype == ORTH_BF16 ? 8192 : 4096) ? 4 : 1;
}

// The values of 16 k's, zeros from kend on: lane (r, h) loads those of k = k0 +
// 8 h + 0 .. 7 and its four columns of B, the first `left` of which exist, and
// makes the fragments of four 32 x 32 tiles from them.
template <int DT>
struct FewB;
template <>
struct FewB<ORTH_BF16> {
  uint32_t w[8][2];
  __device__ __forceinline__ void load(const void* at, int64_t ld, int k, int kend, int left) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint16_t* q = static_cast<const uint16_t*>(at) + e * ld;
      w[e][0] = w[e][1] = 0;
      if (k + e < kend) {
        if (left >= 4) {
          const orth_u32x2_a2 u = *(const ORTH_GLOBAL orth_u32x2_a2*)q;
          w[e][0] = u.x;
          w[e][1] = u.y;
        } else {
          if (left > 0) w[e][0] = gld_u16(q, 0);
          if (left > 1) w[e][0] |= (uint32_t)gld_u16(q, 1) << 16;
          if (left > 2) w[e][1] = gld_u16(q, 2);
        }
      }
    }
  }
  __device__ __forceinline__ bf16x8 frag(int t) const {
    uint32_t c[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t x = w[2 * e][t / 2], y = w[2 * e + 1][t / 2];
      c[e] = t & 1 ? x >> 16 | (y & 0xffff0000u) : (x & 0xffffu) | y << 16;
    }
    return __builtin_bit_cast(bf16x8, make_uint4(c[0], c[1], c[2], c[3]));
  }
};
template <>
struct FewB<ORTH_F32> {
  orth_f32x4 v[8];
  __device__ __forceinline__ void load(const void* at, int64_t ld, int k, int kend, int left) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float* q = static_cast<const float*>(at) + e * ld;
      v[e] = orth_f32x4{};
      if (k + e < kend) {
        if (left >= 4) {
          v[e] = *(const ORTH_GLOBAL orth_f32x4_a4*)q;
        } else {
#pragma unroll
          for (int t = 0; t < 3; ++t)
            if (left > t) v[e][t] = gld_f32(q, t);
        }
      }
    }
  }
};
// The same of one column (step: elements between k's) of A.
template <int DT>
struct FewA;
template <>
struct FewA<ORTH_BF16> {
  uint4 v;
  __device__ __forceinline__ void load(const void* at, int64_t step, int k, int kend) {
    uint32_t w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      w[e] = 0;
      if (k + e < kend) w[e] = gld_u16(static_cast<const uint16_t*>(at) + e * step, 0);
    }
    v = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
  }
};
template <>
struct FewA<ORTH_F32> {
  float v[8];
  __device__ __forceinline__ void load(const void* at, int64_t step, int k, int kend) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = 0.f;
      if (k + e < kend) v[e] = gld_f32(static_cast<const float*>(at) + e * step, 0);
    }
  }
};
// n: k's of the first half wave (the others are zeros in both halves)
__device__ __forceinline__ void few_mma(f32x16 (&acc)[4], const FewA<ORTH_BF16>& a, const FewB<ORTH_BF16>& b, int) {
#pragma unroll
  for (int t = 0; t < 4; ++t)
    acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a.v), b.frag(t), acc[t], 0, 0, 0);
}
__device__ __forceinline__ void few_mma(f32x16 (&acc)[4], const FewA<ORTH_F32>& a, const FewB<ORTH_F32>& b, int n) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (e >= n) break;
#pragma unroll
    for (int t = 0; t < 4; ++t) acc[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[e], b.v[e][t], acc[t], 0, 0, 0);
  }
}

template <int DT, int RB>
__global__ __launch_bounds__(256, RB == 1 ? 3 : 2) void rows_outer_kernel(const RowsProd p) {
  constexpr int ES = DT == ORTH_BF16 ? 2 : 4;
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (rows_joined(p.join, tid)) return;
  const int strips = (p.N + 127) / 128;
  int i0 = (int)(blockIdx.x / strips) * (RB * 128) + wave * 32;
  const int j = (int)(blockIdx.x % strips) * 128 + 4 * r;
  const int left = p.N - j;   // columns that exist, from this lane's first on
  const int g = blockIdx.y;
  const GroupRange range = group_range(p, g, lane);
  const char* A = static_cast<const char*>(p.A) + (range.start + 8 * h) * p.lda * ES;
  const char* B = static_cast<const char*>(p.B) + ((range.start + 8 * h) * p.ldb + j) * ES;
  const int rows = range.end - range.start;
  FewA<DT> a;
  FewB<DT> b;
  a.load(A + (int64_t)min(i0 + r, p.M - 1) * ES, p.lda, 8 * h, rows);
  b.load(B, p.ldb, 8 * h, rows, left);
#pragma unroll 1
  for (int q = 0; q < RB && i0 < p.M; ++q, i0 += 128) {
    f32x16 acc[4] = {};
    few_mma(acc, a, b, min(8, rows));
    for (int k = 16; k < rows; k += 16) {
      a.load(A + ((int64_t)k * p.lda + min(i0 + r, p.M - 1)) * ES, p.lda, k + 8 * h, rows);
      b.load(B + (int64_t)k * p.ldb * ES, p.ldb, k + 8 * h, rows, left);
      few_mma(acc, a, b, min(8, rows - k));
    }
    if (q + 1 < RB) {
      a.load(A + (int64_t)min(i0 + 128 + r, p.M - 1) * ES, p.lda, 8 * h, rows);
      if (rows > 16) b.load(B, p.ldb, 8 * h, rows, left);
    }
    const int64_t base = (p.offsets ? g * p.gc : 0) + j;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int row = i0 + 8 * (v >> 2) + 4 * h + (v & 3);
      if (row < p.M)
        rows_store4(p.C, base + (int64_t)row * p.ldc, p.c_dtype, make_float4(acc[0][v], acc[1][v], acc[2][v], acc[3][v]), left);
    }
  }
}

template <int DT>
void run(const RowsProd& p, hipStream_t s) {
  const dim3 grid((unsigned)rows_outer_blocks(p, DT), p.groups);
  if (outer_rb(p, DT) == 4)
    hipLaunchKernelGGL((rows_outer_kernel<DT, 4>), grid, dim3(256), 0, s, p);
  else
    hipLaunchKernelGGL((rows_outer_kernel<DT, 1>), grid, dim3(256), 0, s, p);
}

}  // namespace

int64_t rows_outer_blocks(const RowsProd& p, int dtype) {
  const int edge = 128 * outer_rb(p, dtype);
  return (int64_t)((p.N + 127) / 128) * ((p.M + edge - 1) / edge) + rows_join_blocks(p.join);
}

hipError_t launch_rows_outer(const RowsProd& p, int dtype, const char* name, hipStream_t s) {
  timing_begin(name, s);
  if (dtype == ORTH_BF16)
    run<ORTH_BF16>(p, s);
  else
    run<ORTH_F32>(p, s);
  const hipError_t e = hipGetLastError();
  timing_end(name, s);
  return e;
}

}  // namespace orth
