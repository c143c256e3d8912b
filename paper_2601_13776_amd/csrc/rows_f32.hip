// Row-grouped products of fp32 operands (rows.h has the descriptor), as
// rows_bf16.hip for bf16 ones.  On the way into LDS each value is split into
// three bfloat16 pieces (split2_bf16: all 24 bits), and the six products that
// matter run on the 16-bit matrix cores, the leading one and the corrections
// with an fp32 accumulator each; results that the split cannot give
// (any_failed) come from fp32 MFMA.
//
// Bound by the six products and, on the vector units beside them, by the
// splitting, which every tile does again for its operands: 8192^3 150 TFLOP/s
// of fp32 products (157 is the peak of fp32 MFMA, which reaches about 120 on
// such tiles), 115 to 130 with a few hundred k's.  6838 rows of logits over 8434
// classes, 264 features: 262 us = 116 TFLOP/s.  The split's 24 bits and the
// accumulator of its own for the corrections make the sums closer than fp32
// products' (errors 2e-7 against 5e-7).
#include <algorithm>
#include <cmath>

#include "rows.h"

namespace orth {

typedef orth_f32x16 f32x16;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

namespace {

constexpr int P = 3, NP = 6;   // pieces, products (smallest first, the leading one last)
__device__ constexpr int prod_a(int q) { return q == 0 ? 2 : q == 2 || q == 3 ? 1 : 0; }
__device__ constexpr int prod_b(int q) { return q == 1 ? 2 : q == 2 || q == 4 ? 1 : 0; }
__device__ __forceinline__ f32x16 mma(uint4 a, uint4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                 0);
}
__device__ __forceinline__ void load4(const float* p, float* x) {
  const orth_f32x4_a4 v = *(const ORTH_GLOBAL orth_f32x4_a4*)p;
  x[0] = v.x;
  x[1] = v.y;
  x[2] = v.z;
  x[3] = v.w;
}

// Results that the split cannot give: those that are not finite, and those that
// are so small (but not zero) that low pieces of their operands may have fallen
// off the end of bfloat16's range.  Each is asked by itself (a lane's 16 are as
// many rows), so that a row's results do not depend on what other rows hold.
// Blocks computed again are read value by value: a head's dW takes 4 times as long,
// 1190 us for 284 at 2000 rows, 264 features, 8000 classes, where most
// probabilities are below 2^-100 but not zero in every row, logits of +-300.
__device__ __forceinline__ bool any_failed(const f32x16& v) {
  uint32_t least = ~0u;
  float nan0 = 0.f, nan1 = 0.f;
#pragma unroll
  for (int r = 0; r < 16; r += 2) {
    least = min(least, min(small_key(v[r]), small_key(v[r + 1])));
    nan0 = fmaf(v[r], 0.f, nan0);
    nan1 = fmaf(v[r + 1], 0.f, nan1);
  }
  return !(nan0 + nan1 == 0.f) || least < small_key(kSplitLo);
}
__device__ __forceinline__ void take_failed(f32x16& v, const f32x16& u) {
#pragma unroll
  for (int r = 0; r < 16; ++r) v[r] = small_key(v[r]) < small_key(kSplitLo) || !(v[r] * 0.f == 0.f) ? u[r] : v[r];
}

// One operand of a tile: `lim` of its rows exist, K values each.
struct Side {
  const float* p;   // row 0, k 0
  int64_t ld;
  int lim;
};

// The wave's 32 x 32 block at rows i0 of A and j0 of B with fp32 MFMA,
// straight from memory (16 k at a time, the lower lanes the first eight).
template <bool AT, bool BT>
__device__ __noinline__ f32x16 block_f32(Side a, Side b, int K, int i0, int j0) {
  const int lane = threadIdx.x & 63, kh = 8 * (lane >> 5);
  f32x16 acc = {};
  auto values = [&](const Side& s, bool kmajor, int row, int k, float (&x)[8]) {
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      x[q] = 0.f;
      if (row < s.lim && k + q < K)
        x[q] = gld_f32(s.p, kmajor ? (int64_t)(k + q) * s.ld + row : (int64_t)row * s.ld + k + q);
    }
  };
#pragma unroll 1
  for (int k0 = 0; k0 < K; k0 += 16) {
    float x[8], y[8];
    values(a, AT, i0 + (lane & 31), k0 + kh, x);
    values(b, BT, j0 + (lane & 31), k0 + kh, y);
#pragma unroll
    for (int q = 0; q < 8; ++q) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[q], y[q], acc, 0, 0, 0);
    if (k0 % 128 == 0 && __all(all_nan(acc))) return acc;
  }
  return acc;
}

template <int BM, bool AT, bool BT, int EPI>
__global__ __launch_bounds__(BM == 64 ? 256 : 512, 2) void rows_f32_kernel(const RowsProd p) {
  constexpr int BK = 32, CH = BK / 8;
  constexpr int WM = 2, WN = BM == 64 ? 2 : 4;          // waves
  constexpr int MI = BM / WM / 32, NI = BM / WN / 32;   // 32 x 32 blocks per wave
  constexpr bool GROUPK = AT;
  extern __shared__ __attribute__((aligned(16))) uint4 smem[];   // [stage][operand][piece][BM rows][CH chunks]
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;
  const int nt = (p.N + BM - 1) / BM;

  int g, ti, tj, K;
  int64_t i0;   // row of C where the tile starts
  Side side[2];
  if constexpr (GROUPK) {
    if constexpr (EPI == ROWS_STORE)
      if (rows_joined(p.join, tid)) return;
    const RowsKTile t = rows_ktile<EPI>(p, BM, blockIdx.x, lane);
    if (!t.any) return;
    g = EPI == ROWS_SLICE ? t.slot : t.g;
    ti = t.ti;
    tj = t.tj;
    K = t.k1 - t.k0;
    i0 = ti * BM;
    side[0] = {static_cast<const float*>(p.A) + (int64_t)t.k0 * p.lda + ti * BM, p.lda, min(BM, p.M - ti * BM)};
    side[1].p = static_cast<const float*>(p.B) + (int64_t)t.k0 * p.ldb + tj * BM;
  } else {
    const RowsTile t = rows_tile(p, BM, nt, blockIdx.x, lane);
    if (!t.any) return;
    g = t.g;
    ti = t.ti;
    tj = t.tj;
    K = p.K;
    i0 = (int64_t)t.start + (int64_t)ti * BM;
    side[0] = {static_cast<const float*>(p.A) + i0 * p.lda, p.lda, (int)min((int64_t)BM, t.end - i0)};
    side[1].p = static_cast<const float*>(p.B) + g * p.gb + (BT ? (int64_t)tj * BM : (int64_t)tj * BM * p.ldb);
    if constexpr (EPI == ROWS_SLICE) {
      const int kb = (int)min((int64_t)blockIdx.y * p.kslice, (int64_t)p.K);
      K = min(p.K - kb, p.kslice);
      side[0].p += kb;
      side[1].p += BT ? kb * p.ldb : (int64_t)kb;
      g = blockIdx.y;
    }
  }
  side[1].ld = p.ldb;
  side[1].lim = min(BM, p.N - tj * BM);

  // chunk c (8 values of k) of row r lives at c ^ swz(r): the fragment reads
  // (one row per lane) and the row-major stores are conflict free
  auto swz = [](int r) { return ((r >> 1) & 3) ^ ((r >> 3) & 1); };
  auto plane = [&](int s, int o, int q) { return smem + ((s * 2 + o) * P + q) * (BM * CH); };
  // this thread's values: row-major (row rr, k 8 rc ..), k-major (rows tr ..
  // tr + 3, k tk and tk + 1; quads past the end take the last four rows once
  // more, which may start before the tile: those rows are staged at its far
  // end, where nobody uses them)
  const int rr = tid / CH, rc = tid % CH;
  const int tk = (tid / (BM / 4)) * 2;
  int tr[2];
  const float* at[2];   // this thread's values of the next whole step
  int64_t astep[2], half[2];
#pragma unroll
  for (int o = 0; o < 2; ++o) {
    const bool tro = o ? BT : AT;
    const Side& s = side[o];
    tr[o] = min((tid % (BM / 4)) * 4, s.lim - 4);
    if (tro) {
      at[o] = s.p + (int64_t)tk * s.ld + tr[o];
      astep[o] = BK * s.ld;
      half[o] = s.ld;
    } else {
      at[o] = s.p + (int64_t)min(rr, s.lim - 1) * s.ld + rc * 8;
      astep[o] = BK;
      half[o] = 4;
    }
  }
  float raw[2][2][8];   // [register set][operand]
  auto load = [&](int set) {
#pragma unroll
    for (int o = 0; o < 2; ++o) {
      load4(at[o], raw[set][o]);
      load4(at[o] + half[o], raw[set][o] + 4);
    }
  };
  auto split_store = [&](const float (&x)[8], int s, int o) {
    uint32_t w[4][P];
    if (o ? BT : AT) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        split2_bf16(x[j], x[j + 4], w[j][0], w[j][1], w[j][2]);
        const int r = (tr[o] + j) & (BM - 1);
        const int dst = (r * CH + ((tk >> 3) ^ swz(r))) * 4 + ((tk & 7) >> 1);
#pragma unroll
        for (int i = 0; i < P; ++i) reinterpret_cast<uint32_t*>(plane(s, o, i))[dst] = w[j][i];
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) split2_bf16(x[2 * j], x[2 * j + 1], w[j][0], w[j][1], w[j][2]);
      const int dst = rr * CH + (rc ^ swz(rr));
#pragma unroll
      for (int i = 0; i < P; ++i) plane(s, o, i)[dst] = make_uint4(w[0][i], w[1][i], w[2][i], w[3][i]);
    }
  };
  auto stage = [&](int set, int s, int o) {
    split_store(raw[set][o], s, o);
  };
  // any k, any rows: zeros past the ends
  auto stage_guarded = [&](int k0, int s, int o) {
    const bool tro = o ? BT : AT;
    const Side& sd = side[o];
    uint32_t w[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int r = tro ? (tr[o] + (q & 3)) & (BM - 1) : rr, k = k0 + (tro ? tk + (q >> 2) : rc * 8 + q);
      w[q] = 0;
      if (r < sd.lim && k < K) w[q] = gld_u32(sd.p, tro ? (int64_t)k * sd.ld + r : (int64_t)r * sd.ld + k);
    }
    float x[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) x[q] = __uint_as_float(w[q]);
    split_store(x, s, o);
  };

  f32x16 acc[2][MI][NI];   // the leading products, the corrections
#pragma unroll
  for (int q = 0; q < 2; ++q)
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) acc[q][i][j] = f32x16{};
  struct Frags {
    uint4 a[MI][P], b[NI][P];
  };
  auto read_frags = [&](int buf, int kk, Frags& f) {
#pragma unroll
    for (int q = 0; q < P; ++q) {
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const int r = wm * (BM / WM) + i * 32 + (lane & 31);
        f.a[i][q] = plane(buf, 0, q)[r * CH + ((2 * kk + (lane >> 5)) ^ swz(r))];
      }
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int r = wn * (BM / WN) + j * 32 + (lane & 31);
        f.b[j][q] = plane(buf, 1, q)[r * CH + ((2 * kk + (lane >> 5)) ^ swz(r))];
      }
    }
  };
  auto mfmas = [&](const Frags& f) {
#pragma unroll
    for (int q = 0; q < NP; ++q)
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) {
          f32x16& t = acc[q < NP - 1][i][j];
          t = mma(f.a[i][prod_a(q)], f.b[j][prod_b(q)], t);
        }
  };
  Frags f0, f1;
  // whole steps, unless a k-major operand has fewer rows than a quad
  const int steps = (AT && p.M < 4) || (BT && p.N < 4) ? 0 : K / BK;
  // The pipeline.  Step t's halves lie in LDS stage t & 1.  First half: the
  // second half's fragments are read, operand B of step t + 1 is split into
  // the other stage.  Then a barrier: step t + 1 is complete and nobody
  // reads step t's stage any more.  Second half: step t + 1's first
  // fragments are read, operand A of step t + 2 is split into step t's
  // stage.  The loads of step t + 3, issued at the barrier, have a whole step
  // to land.  Past the last step the same work runs on stale values that
  // nothing uses.
  int loaded = 0;   // steps whose loads have been issued (past the last they re-read it)
  auto fetch = [&](int set) {
    if (loaded < steps) ++loaded;
    load(set);
    const bool more = loaded < steps;
    at[0] += more ? astep[0] : 0;
    at[1] += more ? astep[1] : 0;
  };
  auto body = [&](int buf) {
    read_frags(buf, 1, f1);
    stage(buf ^ 1, buf ^ 1, 1);
    mfmas(f0);
    __syncthreads();
    fetch(buf ^ 1);
    read_frags(buf ^ 1, 0, f0);
    stage(buf, buf, 0);
    mfmas(f1);
  };
  // rows past a k-major operand's end are staged by nobody: zeros, so that
  // their results do not look like failed splits
  if ((AT && side[0].lim < BM) || (BT && side[1].lim < BM)) {
    for (int i = tid; i < 4 * P * BM * CH; i += blockDim.x) smem[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
  }
  if (steps > 0) {
    fetch(0);
    fetch(1);
    stage(0, 0, 0);
    stage(0, 0, 1);
    fetch(0);
    stage(1, 1, 0);
    __syncthreads();
    read_frags(0, 0, f0);
    for (int t = 0; t < steps; t += 2) {
      body(0);
      if (t + 1 >= steps) break;
      body(1);
    }
    __syncthreads();
  }
  // what is left of K, value by value
  int st = 0;
  for (int k0 = steps * BK; k0 < K; k0 += BK, st ^= 1) {
    stage_guarded(k0, st, 0);
    stage_guarded(k0, st, 1);
    __syncthreads();
    for (int kk = 0; kk < BK / 16; ++kk) {
      read_frags(st, kk, f0);
      mfmas(f0);
    }
  }
  __syncthreads();   // the epilogue reuses LDS

  bool bad = false;
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      acc[0][i][j] += acc[1][i][j];
      bad |= any_failed(acc[0][i][j]);
    }
  if (__builtin_expect(__any(bad), 0)) {
#pragma unroll 1
    for (int n = 0; n < MI * NI; ++n) {
      const f32x16 t = block_f32<AT, BT>(side[0], side[1], K, wm * (BM / WM) + n / NI * 32,
                                         wn * (BM / WN) + n % NI * 32);
#pragma unroll
      for (int i = 0; i < MI * NI; ++i)
        if (i == n) take_failed(acc[0][i / NI][i % NI], t);
    }
  }
  constexpr int TM = BM / WM, TN = BM / WN;
  rows_epilogue<MI, NI, EPI, false>(p, g, acc[0], reinterpret_cast<float*>(smem) + wave * (64 * TN),
                             reinterpret_cast<float*>(smem) + wave * (64 * TN) + 32 * TN, i0 + wm * TM,
                             tj * BM + wn * TN, side[0].lim - wm * TM, tj * WN + wn, lane);
}

template <int BM, bool AT, bool BT, int EPI>
hipError_t run_tile(const RowsProd& p, int64_t n, hipStream_t s) {
  constexpr int lds = 2 * 2 * P * BM * 32 * 2;   // two stages of two operands
  if constexpr (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&rows_f32_kernel<BM, AT, BT, EPI>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  // (grouped along M: the slices of k along y)
  const dim3 grid((unsigned)n, !AT && EPI == ROWS_SLICE ? (p.K + p.kslice - 1) / p.kslice : 1);
  hipLaunchKernelGGL((rows_f32_kernel<BM, AT, BT, EPI>), grid, dim3(BM == 64 ? 256 : 512), lds, s, p);
  return hipGetLastError();
}
template <bool AT, bool BT, int EPI>
hipError_t run(const RowsProd& p, int64_t n, int tile, hipStream_t s) {
  return tile == 128 ? run_tile<128, AT, BT, EPI>(p, n, s) : run_tile<64, AT, BT, EPI>(p, n, s);
}

}  // namespace

// The tile edge by the rounds that its tiles take: 128-tiles halve the
// splitting per product, but one workgroup fills a compute unit (256 at once,
// 54 us of 1024 k's); 512 of edge 64 take 34 us and more of them as much more.
int rows_f32_tile(const RowsProd& p, bool at) {
  const double n128 = rows_expected(p, at, 128), n64 = rows_expected(p, at, 64);
  return 54 * std::ceil(n128 / 256) <= 34 * std::max(1.0, n64 / 512) ? 128 : 64;
}

hipError_t launch_rows_f32(const RowsProd& p, bool at, bool bt, int epi, int tile, const char* name, hipStream_t s) {
  const int64_t n = rows_launch_blocks(p, at, epi, tile);
  if (n <= 0) return hipSuccess;
  timing_begin(name, s);
  hipError_t e = hipErrorInvalidValue;
  if (!at && !bt && epi == ROWS_STORE) e = run<false, false, ROWS_STORE>(p, n, tile, s);
  if (!at && !bt && epi == ROWS_LSE) e = run<false, false, ROWS_LSE>(p, n, tile, s);
  if (!at && !bt && epi == ROWS_DZ) e = run<false, false, ROWS_DZ>(p, n, tile, s);
  if (!at && bt && epi == ROWS_STORE) e = run<false, true, ROWS_STORE>(p, n, tile, s);
  if (!at && bt && epi == ROWS_SUM) e = run<false, true, ROWS_SUM>(p, n, tile, s);
  if (!at && bt && epi == ROWS_SLICE) e = run<false, true, ROWS_SLICE>(p, n, tile, s);
  if (at && bt && epi == ROWS_STORE) e = run<true, true, ROWS_STORE>(p, n, tile, s);
  if (at && bt && epi == ROWS_SLICE) e = run<true, true, ROWS_SLICE>(p, n, tile, s);
  timing_end(name, s);
  return e;
}

}  // namespace orth
