// Row-grouped products of bf16 operands with fp32 accumulation (rows.h has
// the descriptor): C_g = A_g B_g^T with each operand row-major along k or
// k-major, so the same kernel applies a batch of matrices to their rows
// (both row-major), applies their transposes (B k-major) and forms the
// matrices' gradients (both k-major, k over a group's rows).
//
// Square tiles of 256 or 128 with four waves, 64 k's a step, through the five
// LDS buffers of mfma_bf16.h: a 256-tile reads 1 / 128 value per product, which
// the caches deliver at the matrix cores' rate, and fills a compute unit.
// Bound by the matrix cores at the clock that their power leaves (1.7 to 2.0
// GHz, pipes busy 51 to 65% of it) and, per tile, by its start and epilogue (13
// us, beside 112 of 4096 k's).  32768 rows as a router deals them over 64
// matrices of 4096^2: 1.16 ms = 948 TFLOP/s (8192^3 as one group: 1398); dW of
// 16 matrices of 2048^2 from 32768 rows: 298 us = 922 TFLOP/s; 4096 rows of
// logits over 50003 classes, 2048 features: 0.73 ms = 1150 TFLOP/s.
#include <cmath>

#include "mfma_bf16.h"
#include "rows.h"

namespace orth {

namespace {

constexpr int kThreads = 256;

// One operand's 64-deep k-step through registers, for operands and k ranges
// that the direct loads cannot take: any alignment, any end.  16-byte chunks
// as Operand stages them; what lies past the end is zero.
template <int ROWS, bool TRANS>
struct Guarded {
  static constexpr int CPR = TRANS ? ROWS / 8 : 8, N = ROWS * 8 / kThreads;
  uint4 v[N];
  // whole: every chunk in one 16-byte load.  Rows past the end re-read the
  // last one; the chunk at a k-major operand's last rows reads past them, into
  // the next k's (which has to exist), and chunks behind it the first rows:
  // nobody stores those results.
  __device__ __forceinline__ void load(const uint16_t* p, int64_t ld, int lim, int k0, int kend, int tid) {
    const bool whole = k0 + 64 <= kend && (!TRANS || (lim & 7) == 0 || (kend - k0 - 64) * ld >= 8);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int q = i * kThreads + tid, row = q / CPR;
      const int c = ((q % CPR) ^ (TRANS ? swt(row) : swz(row))) * 8;
      if (whole) {
        const uint16_t* at = p + (TRANS ? (int64_t)(k0 + row) * ld + (c < lim ? c : 0)
                                        : (int64_t)min(row, lim - 1) * ld + k0 + c);
        const orth_u32x4_a2 w = *(const ORTH_GLOBAL orth_u32x4_a2*)at;
        v[i] = make_uint4(w.x, w.y, w.z, w.w);
        continue;
      }
      const bool in = TRANS ? k0 + row < kend : row < lim;
      const int n = !in ? 0 : TRANS ? lim - c : kend - k0 - c;   // values of the chunk that exist
      const uint16_t* at = p + (TRANS ? (int64_t)(k0 + row) * ld + c : (int64_t)row * ld + k0 + c);
      if (n >= 8) {
        const orth_u32x4_a2 w = *(const ORTH_GLOBAL orth_u32x4_a2*)at;
        v[i] = make_uint4(w.x, w.y, w.z, w.w);
      } else {
        uint32_t w[8] = {};
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < n) w[e] = gld_u16(at, e);
        v[i] = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
      }
    }
  }
  __device__ __forceinline__ void store(uint16_t* lds, int tid) const {
#pragma unroll
    for (int i = 0; i < N; ++i) *reinterpret_cast<uint4*>(lds + (i * kThreads + tid) * 8) = v[i];
  }
};

// A workgroup's tile: what it computes and from where.
struct TileWork {
  const uint16_t *A, *B;
  int K, mrows, alim, blim, j0, col;   // col: number of the tile's column
  int g;
  int64_t i0;   // row of C where the tile starts
};
struct TileLds {
  uint16_t *a0, *b0, *a1, *b1, *x;
};

// DMA: whole k-steps go through the direct-to-LDS pipeline (every chunk of
// both operands 16-byte aligned, row strides up to 2^22, rows of a k-major
// operand multiples of 8); the others, and all of them without DMA, through
// registers.
template <int BM, int BN, bool AT, bool BT, int EPI, bool DMA, int BAUX>
__device__ __forceinline__ void tile_body(const RowsProd& p, const TileWork& w, const TileLds& l, int wave, int lane,
                                          int tid) {
  constexpr int WM = 2, WN = 2, BK = 64;
  using T = Tile<BM, BN, WM, WN>;
  constexpr int MI = T::MI, NI = T::NI;
  const int wm = wave / WN, wn = wave % WN;
  f32x16 acc[MI][NI];
#pragma unroll
  for (int mi = 0; mi < MI; ++mi)
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) acc[mi][ni] = f32x16{};

  const int K = w.K, kmain = DMA ? K / BK * BK : 0;
  if constexpr (DMA)
    kloop<BM, BN, WM, WN, AT, BT, false, true, BAUX>(acc, w.A, p.lda, w.B, p.ldb, 0, kmain, l.a0, l.b0, l.a1, l.b1, l.x, wave,
                                               lane, wm, wn, Prefetch(), w.alim, w.blim);
  if (kmain < K) {
    Operand<BM, T::NW, MI, AT> oa;
    Operand<BN, T::NW, NI, BT> ob;
    oa.init(w.A, p.lda, wave, lane, wm * T::TM);
    ob.init(w.B, p.ldb, wave, lane, wn * T::TN);
    // without DMA the loads run three k-steps ahead (a step's products take a
    // quarter of a load's latency); behind it there is one step at most
    constexpr int D = DMA ? 1 : 3;
    Guarded<BM, AT> ga[D];
    Guarded<BN, BT> gb[D];
    auto load = [&](int d, int k0) {
      if (k0 < K) {
        ga[d].load(w.A, p.lda, w.alim, k0, K, tid);
        gb[d].load(w.B, p.ldb, w.blim, k0, K, tid);
      }
    };
#pragma unroll
    for (int d = 0; d < D; ++d) load(d, kmain + d * BK);
    auto step = [&](int d, uint16_t* pa, uint16_t* pb, int k0) {
      ga[d].store(pa, tid);
      gb[d].store(pb, tid);
      __syncthreads();
      load(d, k0 + D * BK);
#pragma unroll
      for (int kk = 0; kk < BK / 16; ++kk) {
        bf16x8 fa[MI], fb[NI];
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) fa[mi] = oa.frag(pa, mi, kk);
#pragma unroll
        for (int ni = 0; ni < NI; ++ni) fb[ni] = ob.frag(pb, ni, kk);
#pragma unroll
        for (int mi = 0; mi < MI; ++mi)
#pragma unroll
          for (int ni = 0; ni < NI; ++ni)
            acc[mi][ni] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[mi], fb[ni], acc[mi][ni], 0, 0, 0);
      }
    };
    // two stages: a step's stage is written again only after the next step's
    // barrier, which every wave reaches past its reads
    if constexpr (DMA) {
      step(0, l.a0, l.b0, kmain);
    } else {
      for (int k0 = 0; k0 < K; k0 += 6 * BK) {
#pragma unroll
        for (int u = 0; u < 6; ++u) {
          if (k0 + u * BK >= K) break;
          step(u % 3, u & 1 ? l.a1 : l.a0, u & 1 ? l.b1 : l.b0, k0 + u * BK);
        }
      }
    }
    __syncthreads();
  }
  // the waves' staging buffers, 32 rows of TN floats each: two fit the stage
  // that a wave takes (half a 256-tile has the stages of a whole one)
  constexpr int CH = 32 * T::TN * 2;
  uint16_t* at = wave == 0 ? l.a0 : wave == 1 ? l.b0 : wave == 2 ? l.a1 : l.b1;
  float* buf = reinterpret_cast<float*>(at);
  float* buf2 = reinterpret_cast<float*>(at + CH);
  rows_epilogue<MI, NI, EPI, !AT && BT>(p, w.g, acc, buf, buf2, w.i0 + wm * T::TM, w.j0 + wn * T::TN, w.mrows - wm * T::TM,
                             w.col * WN + wn, lane);
}

// BAUX: cache policy of B's loads.  Without DMA the registers are held to what
// leaves a unit two workgroups (us, one / two: 8000 rows, 4 x 2003 x 1333 112 / 83,
// transposed 112 / 97, 1500 x 777 x 513 19.5 / 20.3).
template <int BM, bool AT, bool BT, int EPI, bool DMA, int BAUX = 0>
__global__ __launch_bounds__(kThreads, DMA ? 1 : 2) void rows_bf16_kernel(const RowsProd p) {
  constexpr int BN = BM, BK = 64;
  __shared__ __attribute__((aligned(1024))) uint16_t sA0[BM * BK];
  __shared__ __attribute__((aligned(1024))) uint16_t sB0[BN * BK];
  __shared__ __attribute__((aligned(1024))) uint16_t sA1[BM * BK];
  __shared__ __attribute__((aligned(1024))) uint16_t sB1[BN * BK];
  __shared__ __attribute__((aligned(1024))) uint16_t sX[DMA ? BM * BK : 8];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  TileWork w;
  int tj;
  if constexpr (AT) {   // grouped along K
    if constexpr (EPI == ROWS_STORE)
      if (rows_joined(p.join, tid)) return;
    const RowsKTile t = rows_ktile<EPI>(p, BM, blockIdx.x, lane);
    if (!t.any) return;
    w.g = EPI == ROWS_SLICE ? t.slot : t.g;
    tj = t.tj;
    w.K = t.k1 - t.k0;
    w.i0 = t.ti * BM;
    w.mrows = min(BM, p.M - t.ti * BM);
    w.alim = min(BM, (p.a_pad8 ? (p.M + 7) / 8 * 8 : p.M) - t.ti * BM);
    w.A = static_cast<const uint16_t*>(p.A) + (int64_t)t.k0 * p.lda + t.ti * BM;
    w.B = static_cast<const uint16_t*>(p.B) + (int64_t)t.k0 * p.ldb + tj * BN;
  } else {
    const RowsTile t = rows_tile(p, BM, (p.N + BN - 1) / BN, blockIdx.x, lane);
    if (!t.any) return;
    w.g = t.g;
    tj = t.tj;
    w.K = p.K;
    w.i0 = (int64_t)t.start + (int64_t)t.ti * BM;
    w.mrows = w.alim = (int)min((int64_t)BM, t.end - w.i0);
    w.A = static_cast<const uint16_t*>(p.A) + w.i0 * p.lda;
    w.B = static_cast<const uint16_t*>(p.B) + w.g * p.gb + (BT ? (int64_t)tj * BN : (int64_t)tj * BN * p.ldb);
    if constexpr (EPI == ROWS_SLICE) {
      const int kb = (int)min((int64_t)blockIdx.y * p.kslice, (int64_t)p.K);
      w.K = min(p.K - kb, p.kslice);
      w.A += kb;
      w.B += BT ? kb * p.ldb : (int64_t)kb;
      w.g = blockIdx.y;
    }
  }
  w.blim = min(BN, (BT && p.b_pad8 ? (p.N + 7) / 8 * 8 : p.N) - tj * BN);
  w.j0 = tj * BN;
  w.col = tj;
  const TileLds l{sA0, sB0, sA1, sB1, sX};
  // a group's last tile may be less than half full: it takes half the products
  if constexpr (BM == 256 && !AT && EPI == ROWS_STORE) {
    if (w.mrows <= 128) {
      tile_body<128, BN, AT, BT, EPI, DMA, BAUX>(p, w, l, wave, lane, tid);
      return;
    }
  }
  tile_body<BM, BN, AT, BT, EPI, DMA, BAUX>(p, w, l, wave, lane, tid);
}

template <bool AT, bool BT, int EPI>
hipError_t run(const RowsProd& p, int64_t n, int tile, bool dma, hipStream_t s) {
  // (grouped along M: the slices of k along y)
  const dim3 grid((unsigned)n, !AT && EPI == ROWS_SLICE ? (p.K + p.kslice - 1) / p.kslice : 1), block(kThreads);
  if (!dma)
    hipLaunchKernelGGL((rows_bf16_kernel<128, AT, BT, EPI, false>), grid, block, 0, s, p);
  else if (tile == 256)
    hipLaunchKernelGGL((rows_bf16_kernel<256, AT, BT, EPI, true>), grid, block, 0, s, p);
  else if (!AT && EPI != ROWS_SUM && p.rows / p.groups <= 64 && (EPI != ROWS_DZ || (int64_t)p.N * p.K > 1 << 27))
    // few rows: each of a matrix's values is read once, past the caches (8 rows
    // of logits over 131072 classes, 4096 features: 216 us through them, 205);
    // dz's product, whose matrix dx's reads next, if 256 MB cannot hold it
    hipLaunchKernelGGL((rows_bf16_kernel<128, AT, BT, EPI, true, AT || EPI == ROWS_SUM ? 0 : 2>), grid, block, 0, s, p);
  else
    hipLaunchKernelGGL((rows_bf16_kernel<128, AT, BT, EPI, true>), grid, block, 0, s, p);
  return hipGetLastError();
}

// Whether the direct-to-LDS loads can take an operand.
bool dma_ok(const void* p, int64_t ld, int64_t group, bool kmajor, bool pad8, int rows) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0 && group % 8 == 0 && ld <= (1 << 22) &&
         (!kmajor || pad8 || rows % 8 == 0);
}
}  // namespace

bool rows_bf16_dma(const RowsProd& p, bool at, bool bt) {
  return dma_ok(p.A, p.lda, 0, at, p.a_pad8, p.M) && dma_ok(p.B, p.ldb, at ? 0 : p.gb, bt, p.b_pad8, p.N);
}

// The tile edge by the rounds that its tiles take: 256 of edge 256 run at
// once (one workgroup per compute unit), 112 us of 4096 k's, 512 of edge 128,
// 72 us.
int rows_bf16_tile(const RowsProd& p, bool at, bool bt) {
  if (!rows_bf16_dma(p, at, bt)) return 128;
  const double n256 = rows_expected(p, at, 256), n128 = rows_expected(p, at, 128);
  return 112 * std::ceil(n256 / 256) <= 72 * std::ceil(n128 / 512) ? 256 : 128;
}

hipError_t launch_rows_bf16(const RowsProd& p, bool at, bool bt, int epi, int tile, const char* name, hipStream_t s) {
  const int64_t n = rows_launch_blocks(p, at, epi, tile);
  if (n <= 0) return hipSuccess;
  const bool dma = rows_bf16_dma(p, at, bt);
  if (!dma && tile != 128) return hipErrorInvalidValue;   // (rows_bf16_tile never says so)
  timing_begin(name, s);
  hipError_t e = hipErrorInvalidValue;
  if (!at && !bt && epi == ROWS_STORE) e = run<false, false, ROWS_STORE>(p, n, tile, dma, s);
  if (!at && !bt && epi == ROWS_LSE) e = run<false, false, ROWS_LSE>(p, n, tile, dma, s);
  if (!at && !bt && epi == ROWS_DZ) e = run<false, false, ROWS_DZ>(p, n, tile, dma, s);
  if (!at && bt && epi == ROWS_STORE) e = run<false, true, ROWS_STORE>(p, n, tile, dma, s);
  if (!at && bt && epi == ROWS_SUM) e = run<false, true, ROWS_SUM>(p, n, tile, dma, s);
  if (!at && bt && epi == ROWS_SLICE) e = run<false, true, ROWS_SLICE>(p, n, tile, dma, s);
  if (at && bt && epi == ROWS_STORE) e = run<true, true, ROWS_STORE>(p, n, tile, dma, s);
  if (at && bt && epi == ROWS_SLICE) e = run<true, true, ROWS_SLICE>(p, n, tile, dma, s);
  timing_end(name, s);
  return e;
}

}  // namespace orth
