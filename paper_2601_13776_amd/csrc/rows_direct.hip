// Row-grouped products whose tiles are too few to fill the chip, or whose
// groups hold few rows: a workgroup of 8 or 4 waves computes one 32 x 32 tile,
// the waves taking the chunks of k in turn (no barrier in the loop), and their
// sums are joined in LDS.
// Long k besides is cut into slices, one workgroup each, whose sums a second
// kernel joins (rows_join).
//
// bf16 operands run on v_mfma_f32_32x32x16_bf16, fp32 ones on the same as
// three bfloat16 pieces (rows_f32.hip; on fp32 MFMA 512 x 1024 x 1024 takes 19 us
// for 16, 64 rows over 64 matrices of 2048^2 220 for 197).
//
// Bound by latency where tiles are few (8 tokens over 8 matrices of 1024^2 6.0
// us on the device), by reading the matrices where they are many (64 tokens, one
// to each of 64 matrices of 4096^2 in bf16: 342 us = 6.3 TB/s; of 2048^2 in fp32:
// 197 us = 5.5 TB/s, with 9 rows and 128000 rows of B 4.1 TB/s: the splitting).
#include "rows.h"

namespace orth {

typedef orth_f32x16 f32x16;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

namespace {

__device__ __forceinline__ f32x16 mma(uint4 a, uint4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                 0);
}

// One lane's row of an operand: `at` its k 0, `ks` elements between k's (1:
// row-major).  load: the 8 values from k on (zeros from `kend` on), as they
// are stored.
template <int DT, bool KM>
struct Lane {
  static constexpr int NR = DT == ORTH_BF16 ? 1 : 2;   // 16-byte registers of 8 values
  const char* at;
  int64_t ld;
  static constexpr int ES = DT == ORTH_BF16 ? 2 : 4;
  __device__ __forceinline__ void load(int k, uint4 (&v)[NR]) const {
    if constexpr (!KM) {
      const char* q = at + (int64_t)k * ES;
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const orth_u32x4_a2 w = *(const ORTH_GLOBAL orth_u32x4_a2*)(q + 16 * i);
        v[i] = make_uint4(w.x, w.y, w.z, w.w);
      }
    } else {
      const char* q = at + (int64_t)k * ld * ES;
      uint32_t w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = DT == ORTH_BF16 ? (uint32_t)gld_u16(q + e * ld * ES, 0) : gld_u32(q + e * ld * ES, 0);
      pack(w, v);
    }
  }
  __device__ __forceinline__ void load_end(int k, int kend, uint4 (&v)[NR]) const {
    const int64_t step = (KM ? ld : 1) * ES;
    const char* q = at + k * step;
    uint32_t w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      w[e] = 0;
      if (k + e < kend) w[e] = DT == ORTH_BF16 ? (uint32_t)gld_u16(q + e * step, 0) : gld_u32(q + e * step, 0);
    }
    pack(w, v);
  }
  static __device__ __forceinline__ void pack(const uint32_t (&w)[8], uint4 (&v)[NR]) {
    if constexpr (DT == ORTH_BF16) {
      v[0] = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
    } else {
      v[0] = make_uint4(w[0], w[1], w[2], w[3]);
      v[NR - 1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
  }
};

__device__ __forceinline__ void split8(const uint4 (&v)[2], uint4 (&p)[3]) {
  uint32_t w[4][3];
  const uint32_t x[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
#pragma unroll
  for (int j = 0; j < 4; ++j)
    split2_bf16(__uint_as_float(x[2 * j]), __uint_as_float(x[2 * j + 1]), w[j][0], w[j][1], w[j][2]);
#pragma unroll
  for (int i = 0; i < 3; ++i) p[i] = make_uint4(w[0][i], w[1][i], w[2][i], w[3][i]);
}

// ROWS_DZ: rows of A into the copy (p.twice: two rows each), zeros for those
// without a target, eight rows a workgroup.  16 bytes from any alignment to an
// aligned place.
constexpr int kCopyRows = 8;
template <int DT>
__device__ __forceinline__ void copy_rows(const RowsProd& p, int block, int tid, int threads) {
  constexpr int ES = DT == ORTH_BF16 ? 2 : 4, L = 16 / ES;
  const int per = p.ld_copy / L;   // (ld_copy is a multiple of 8)
  for (int q = 0; q < kCopyRows; ++q) {
    const int64_t i = (int64_t)block * kCopyRows + q;
    if (i >= p.rows) return;
    const int64_t t = ((const ORTH_GLOBAL int64_t*)p.targets)[i];
    const bool has = t >= 0 && t < p.classes;
    for (int c = tid * L; c < per * L; c += threads * L) {
      const char* from = static_cast<const char*>(p.A) + (i * p.lda + c) * ES;
      orth_u32x4 v{};
      if (has && c + L <= p.K) {
        const orth_u32x4_a2 w = *(const ORTH_GLOBAL orth_u32x4_a2*)from;
        v = orth_u32x4{w.x, w.y, w.z, w.w};
      } else if (has) {
        uint32_t w[4] = {};
#pragma unroll
        for (int e = 0; e < L; ++e)
          if (c + e < p.K) w[e * ES / 4] |= ES == 2 ? (uint32_t)gld_u16(from, e) << (e % 2 * 16) : gld_u32(from, e);
        v = orth_u32x4{w[0], w[1], w[2], w[3]};
      }
      char* to = static_cast<char*>(p.copy) + ((i << p.twice) * p.ld_copy + c) * ES;
      *(ORTH_GLOBAL orth_u32x4*)to = v;
      if (p.twice) *(ORTH_GLOBAL orth_u32x4*)(to + (int64_t)p.ld_copy * ES) = v;
    }
  }
}

template <int DT, bool BT, int EPI, int kWaves, bool NT>
__global__ __launch_bounds__(64 * kWaves, 4) void rows_direct_kernel(const RowsProd p) {
  // k's of a chunk: one 128-byte line of a row-major operand's row, each half
  // wave a half of it, 8 values a fragment
  constexpr int KC = DT == ORTH_BF16 ? 64 : 32, NF = KC / 16;
  using LA = Lane<DT, false>;
  using LB = Lane<DT, BT>;
  // the waves' sums (a padded row: 36 floats), before them the buffers that
  // turn their chunks around
  __shared__ float4 sums[BT ? kWaves : 2 * kWaves][32][9];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nt = (p.N + 31) / 32;
  if constexpr (EPI == ROWS_DZ) {
    const int copies = p.copy ? (p.rows + kCopyRows - 1) / kCopyRows : 0, tiles = (int)gridDim.x - copies;
    if ((int)blockIdx.x >= tiles) {
      copy_rows<DT>(p, blockIdx.x - tiles, tid, 64 * kWaves);
      return;
    }
  }
  const RowsTile t = rows_tile(p, 32, nt, blockIdx.x, lane);
  if (!t.any) return;
  const int64_t i0 = (int64_t)t.start + (int64_t)t.ti * 32;
  const int mrows = (int)min((int64_t)32, t.end - i0), j0 = t.tj * 32, ncols = min(32, p.N - j0);
  const int kb = (int)min((int64_t)blockIdx.y * p.kslice, (int64_t)p.K);
  const int ke = (int)min((int64_t)kb + p.kslice, (int64_t)p.K);
  constexpr int ES = LA::ES;
  const int r = lane & 31, h = lane >> 5;
  LA la;
  LB lb;
  la.ld = p.lda;
  lb.ld = p.ldb;
  la.at = static_cast<const char*>(p.A) + (i0 + min(r, mrows - 1)) * p.lda * ES;
  lb.at = static_cast<const char*>(p.B) + (t.g * p.gb + (int64_t)(j0 + min(r, ncols - 1)) * (BT ? 1 : p.ldb)) * ES;

  f32x16 acc = {}, low = {};
  auto products = [&](const uint4 (&a)[LA::NR], const uint4 (&b)[LB::NR]) {
    if constexpr (DT == ORTH_BF16) {
      acc = mma(a[0], b[0], acc);
    } else {
      uint4 x[3], y[3];
      split8(a, x);
      split8(b, y);
      low = mma(x[2], y[0], low);
      low = mma(x[0], y[2], low);
      low = mma(x[1], y[1], low);
      low = mma(x[1], y[0], low);
      low = mma(x[0], y[1], low);
      acc = mma(x[0], y[0], acc);
    }
  };
  const int whole = (ke - kb) / KC;   // whole chunks; the wave after them takes what is left
  // A row-major operand's chunk is loaded as whole 128-byte lines, eight lanes
  // a row (a lane per row would touch 32 lines an instruction: fp32 256 x 1000
  // x 2048 took 22 us, this way 16), and turned around through LDS of the
  // wave's own: 16-byte piece c of row r lies at c ^ (r & 7).  A k-major one is
  // loaded as its fragments.
  constexpr int NP = 4;   // pieces of a chunk per lane
  uint4* turn = reinterpret_cast<uint4*>(&sums[0][0][0]) + wave * (BT ? 256 : 512);
  static_assert(sizeof(sums) >= kWaves * 512 * 16 || BT, "the turning buffers take the place of the sums");
  uint4 ra[2][NP], rb[2][BT ? NF * LB::NR : NP];
  const char *pa[NP], *pb[NP];   // this lane's pieces, at k 0
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int row = i * 8 + (lane >> 3);
    pa[i] = static_cast<const char*>(p.A) + (i0 + min(row, mrows - 1)) * p.lda * ES + (lane & 7) * 16;
    pb[i] = static_cast<const char*>(p.B) + (t.g * p.gb + (int64_t)(j0 + min(row, ncols - 1)) * p.ldb) * ES + (lane & 7) * 16;
  }
  auto load = [&](int set, int c) {
    const int k = kb + c * KC;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const orth_u32x4_a2 w = *(const ORTH_GLOBAL orth_u32x4_a2*)(pa[i] + (int64_t)k * ES);
      ra[set][i] = make_uint4(w.x, w.y, w.z, w.w);
    }
    if constexpr (BT) {
#pragma unroll
      for (int f = 0; f < NF; ++f) {
        uint4 v[LB::NR];
        lb.load(k + h * (KC / 2) + 8 * f, v);
#pragma unroll
        for (int i = 0; i < LB::NR; ++i) rb[set][f * LB::NR + i] = v[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const ORTH_GLOBAL orth_u32x4_a2* q = (const ORTH_GLOBAL orth_u32x4_a2*)(pb[i] + (int64_t)k * ES);
        const orth_u32x4_a2 w = NT ? __builtin_nontemporal_load(q) : *q;
        rb[set][i] = make_uint4(w.x, w.y, w.z, w.w);
      }
    }
  };
  auto use = [&](int set) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int row = i * 8 + (lane >> 3), at = row * 8 + ((lane & 7) ^ (row & 7));
      turn[at] = ra[set][i];
      if constexpr (!BT) turn[256 + at] = rb[set][i];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      uint4 a[LA::NR], b[LB::NR];
#pragma unroll
      for (int i = 0; i < LA::NR; ++i) {
        const int at = r * 8 + ((h * 4 + f * LA::NR + i) ^ (r & 7));
        a[i] = turn[at];
        if constexpr (BT)
          b[i] = rb[set][f * LB::NR + i];
        else
          b[i] = turn[256 + at];
      }
      products(a, b);
    }
  };
  if (wave < whole) {
    load(0, wave);
    for (int c = wave; c < whole; c += 2 * kWaves) {
      // (past the last chunk the loads re-read it)
      load(1, c + kWaves < whole ? c + kWaves : c);
      use(0);
      if (c + kWaves >= whole) break;
      load(0, c + 2 * kWaves < whole ? c + 2 * kWaves : c);
      use(1);
    }
  }
  if ((ke - kb) % KC && whole % kWaves == wave) {
    const int k = kb + whole * KC + h * (KC / 2);
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      uint4 a[LA::NR], b[LB::NR];
      la.load_end(k + 8 * f, ke, a);
      lb.load_end(k + 8 * f, ke, b);
      products(a, b);
    }
  }
  __syncthreads();   // the sums take the place of the turning buffers
  if constexpr (DT == ORTH_F32) acc += low;
  auto put = [&](int w) {
#pragma unroll
    for (int q = 0; q < 16; ++q)
      reinterpret_cast<float*>(sums[w][8 * (q >> 2) + 4 * h + (q & 3)])[r] = acc[q];
  };
  put(wave);
  __syncthreads();
  // four columns of a row per thread, the first 256 threads (the first 128
  // where rows are added by pairs)
  const int row = tid >> 3, c4 = tid & 7;
  const int two = DT == ORTH_BF16 && BT ? p.pairs : 0;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](int n) {
    v = sums[0][row << two & 31][c4];
    for (int w = 1; w < n << two; ++w) {
      const float4 u = sums[w >> two][((row << two) + (w & two)) & 31][c4];
      v.x += u.x;
      v.y += u.y;
      v.z += u.z;
      v.w += u.w;
    }
  };
  if (tid < 256) add(kWaves);
  if constexpr (DT == ORTH_F32) {
    // results that the split cannot give, from the tile's fp32 MFMA products:
    // those that are not finite or too small, each by itself
    auto fails = [](float r) { return !(r * 0.f == 0.f) || small_key(r) < small_key(kSplitLo); };
    const bool bad = tid < 256 && (fails(v.x) || fails(v.y) || fails(v.z) || fails(v.w));
    if (__syncthreads_or(bad)) {
      if (wave == 0) {
        acc = f32x16{};
#pragma unroll 1
        for (int k = kb; k < ke; k += 16) {
          uint4 x[2], y[2];
          la.load_end(k + 8 * h, ke, x);
          lb.load_end(k + 8 * h, ke, y);
          const uint32_t xs[8] = {x[0].x, x[0].y, x[0].z, x[0].w, x[1].x, x[1].y, x[1].z, x[1].w};
          const uint32_t ys[8] = {y[0].x, y[0].y, y[0].z, y[0].w, y[1].x, y[1].y, y[1].z, y[1].w};
#pragma unroll
          for (int q = 0; q < 8; ++q)
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(xs[q]), __uint_as_float(ys[q]), acc, 0, 0, 0);
          if ((k - kb) % 128 == 0 && __all(all_nan(acc))) break;
        }
        put(0);
      }
      __syncthreads();
      if (bad) {
        const float4 o = v;
        add(1);
        if (!fails(o.x)) v.x = o.x;
        if (!fails(o.y)) v.y = o.y;
        if (!fails(o.z)) v.z = o.z;
        if (!fails(o.w)) v.w = o.w;
      }
    }
  }
  if (tid >= 256) return;
  if constexpr (EPI == ROWS_LSE) {
    float e[4] = {v.x, v.y, v.z, v.w};
    float top = -INFINITY;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      e[q] = c4 * 4 + q < ncols ? e[q] * p.scale : -INFINITY;
      top = fmaxf(top, e[q]);
    }
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    const float from = lse_base(top);
    float sum = 0.f;
#pragma unroll
    for (int q = 0; q < 4; ++q) sum += c4 * 4 + q < ncols ? __builtin_amdgcn_exp2f((e[q] - from) * kLog2e) : 0.f;
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) sum += __shfl_xor(sum, d, 64);
    if (row < mrows) {
      const int64_t i = i0 + row;
      if (c4 == 0) {
        gst_f32(p.part, (i * p.n_part + t.tj) * 2, top);
        gst_f32(p.part, (i * p.n_part + t.tj) * 2 + 1, sum);
      }
      const int64_t at = ((const ORTH_GLOBAL int64_t*)p.targets)[i] - p.col0 - j0 - c4 * 4;
      if (at >= 0 && at < 4 && c4 * 4 + at < ncols) gst_f32(p.ztarget, i, at == 0 ? e[0] : at == 1 ? e[1] : at == 2 ? e[2] : e[3]);
    }
  } else if (row << two < mrows) {
    const int left = (EPI == ROWS_DZ ? (p.N + 7) / 8 * 8 : p.N) - j0;
    if constexpr (EPI == ROWS_DZ) {
      const int64_t i = i0 + row, t = ((const ORTH_GLOBAL int64_t*)p.targets)[i];
      const float l = gld_f32(p.lse, i), f = gld_f32(p.grad_loss, i) * p.scale;
      float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = c4 * 4 + q;
        const float x = __builtin_amdgcn_exp2f((e[q] * p.scale - l) * kLog2e);
        // a row without a target gets zeros whatever its values are; so do
        // the columns that pad the piece to a multiple of 8
        e[q] = t >= 0 && t < p.classes && c < ncols ? f * (p.col0 + (int64_t)j0 + c == t ? x - 1.f : x) : 0.f;
      }
      v = make_float4(e[0], e[1], e[2], e[3]);
    }
    rows_finish4<EPI>(p, EPI == ROWS_SLICE ? (int)blockIdx.y : t.g, (i0 >> two) + row, j0 + c4 * 4, v, left - c4 * 4);
  }
}

__global__ __launch_bounds__(256) void rows_join_kernel(const RowsJoin p) { rows_join_block(p, blockIdx.x, threadIdx.x); }

// The same for every group of a product grouped along K: its rows' slices
// into its C (zeros for a group without rows).
__global__ __launch_bounds__(256) void rows_join_groups_kernel(const RowsProd p) {
  const int lane = threadIdx.x & 63, g = blockIdx.y;
  int first = 0, count = 0;
  if (!p.offsets) {
    count = (p.rows + p.kslice - 1) / p.kslice;
  } else {
    int carry = 0;
    for (int base = 0; base <= g; base += 64) {
      const GroupRange r = lane_range(p.offsets, p.groups, p.rows, base + lane, lane, carry);
      const int mine = (r.end - r.start + p.kslice - 1) / p.kslice, upto = wave_scan_add(mine, lane);
      if (g < base + 64) {
        count = __shfl(mine, g - base, 64);
        first += __shfl(upto, g - base, 64) - count;
      } else {
        first += __shfl(upto, 63, 64);
      }
    }
  }
  const int nq = (p.N + 3) / 4;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, i = id / nq, n = (int64_t)p.M * p.N;
  if (i >= p.M) return;
  const int j = (int)(id - i * nq) * 4, have = min(4, p.N - j);
  const float4 v = join4(make_float4(0.f, 0.f, 0.f, 0.f), p.slices + first * n + i * p.N + j, n, count, have);
  rows_store4(p.C, g * p.gc + i * p.ldc + j, p.c_dtype, v, have);
}

// Four waves where there are workgroups for many rounds (a shorter start and
// end beside the loop), with B past the caches, as each of its values is read
// once.  (64 rows over 64 matrices of 4096^2 in bf16: 389 us with eight waves
// through the caches, 367 with four, 342 with both.)
template <int DT, bool BT, int EPI>
hipError_t run(const RowsProd& p, int64_t n, int slices, hipStream_t s) {
  const int64_t copies = EPI == ROWS_DZ && p.copy ? ((int64_t)p.rows + kCopyRows - 1) / kCopyRows : 0;
  const dim3 grid((unsigned)(n + copies), slices);
  if (!BT && n * slices > 2048)
    hipLaunchKernelGGL((rows_direct_kernel<DT, BT, EPI, BT ? 8 : 4, !BT>), grid, dim3(BT ? 512 : 256), 0, s, p);
  else
    hipLaunchKernelGGL((rows_direct_kernel<DT, BT, EPI, 8, false>), grid, dim3(512), 0, s, p);
  return hipGetLastError();
}
template <int DT>
hipError_t run_dt(const RowsProd& p, int64_t n, int slices, bool bt, int epi, hipStream_t s) {
  if (!bt && epi == ROWS_STORE) return run<DT, false, ROWS_STORE>(p, n, slices, s);
  if (!bt && epi == ROWS_LSE) return run<DT, false, ROWS_LSE>(p, n, slices, s);
  if (!bt && epi == ROWS_DZ) return run<DT, false, ROWS_DZ>(p, n, slices, s);
  if (bt && epi == ROWS_STORE) return run<DT, true, ROWS_STORE>(p, n, slices, s);
  if (bt && epi == ROWS_SUM) return run<DT, true, ROWS_SUM>(p, n, slices, s);
  if (bt && epi == ROWS_SLICE) return run<DT, true, ROWS_SLICE>(p, n, slices, s);
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_rows_direct(const RowsProd& p, int dtype, bool bt, int epi, int slices, const char* name,
                              hipStream_t s) {
  const int64_t n = rows_blocks(p, false, 32);
  if (n <= 0) return hipSuccess;
  timing_begin(name, s);
  const hipError_t e = dtype == ORTH_BF16 ? run_dt<ORTH_BF16>(p, n, slices, bt, epi, s)
                                          : run_dt<ORTH_F32>(p, n, slices, bt, epi, s);
  timing_end(name, s);
  return e;
}

hipError_t launch_rows_join(const RowsJoin& p, const char* name, hipStream_t s) {
  const int64_t n = rows_join_blocks(p);
  if (n <= 0) return hipSuccess;
  timing_begin(name, s);
  hipLaunchKernelGGL(rows_join_kernel, dim3((unsigned)n), dim3(256), 0, s, p);
  const hipError_t e = hipGetLastError();
  timing_end(name, s);
  return e;
}

hipError_t launch_rows_join_groups(const RowsProd& p, const char* name, hipStream_t s) {
  const int64_t n = ((int64_t)p.M * ((p.N + 3) / 4) + 255) / 256;
  if (n <= 0) return hipSuccess;
  timing_begin(name, s);
  hipLaunchKernelGGL(rows_join_groups_kernel, dim3((unsigned)n, p.groups), dim3(256), 0, s, p);
  const hipError_t e = hipGetLastError();
  timing_end(name, s);
  return e;
}

}  // namespace orth
