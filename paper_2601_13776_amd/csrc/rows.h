// Products over rows grouped by matrix (the application of a batch of dense
// matrices, its gradients) and the products of the classification loss:
// descriptors and device pieces shared by their bf16 and fp32 kernels.
//
// A call's product is one descriptor passed by value: no table is copied, so
// the calls can be captured into a graph.  The groups' row ranges are device
// data (a router's result) that the host never sees: every wave finds its
// tile from them by itself.
#pragma once

#include "internal.h"

namespace orth {

enum RowsEpi : int32_t {
  ROWS_STORE = 0,   // C = acc
  ROWS_SUM = 1,     // fp32 sums over several products: acc (+ sum if add) -> sum, or -> C on the last
  ROWS_LSE = 2,     // running maximum and sum of exponentials of scale * acc over the tile's columns
  ROWS_SLICE = 4,   // fp32 sums of a slice of kslice k's, which rows_join adds up (grouped along M: one
                    // group, slices along the grid's y)
  ROWS_DZ = 3       // C = scale * grad_loss * (exp(scale * acc - lse) - [column is the target]), in bf16 as
                    // two pieces (c_low)
};

// Slices' sums (M x N each, one after the other) to be added up in order,
// into sum (row stride N) or, on the last of several products, into C.
struct RowsJoin {
  const float* slices;   // nullptr: nothing to join
  float* sum;
  void* C;
  int64_t ldc;
  int32_t M, N, n;           // n: slices
  int32_t add, last, c_dtype;
};

// C_g = A_g B_g^T.  Grouped along M: A and C are rows x . with group g's rows
// at [start_g, end_g), B_g = B + g gb.  Grouped along K: A (K x M) and B
// (K x N) are stored k-major, group g's k range is its rows, C_g = C + g gc.
struct RowsProd {
  const void* A;
  const void* B;
  void* C;
  int64_t lda, ldb, ldc;     // elements
  int64_t gb, gc;            // elements from one group's B (C) to the next
  const int32_t* offsets;    // groups + 1 row numbers on the device; nullptr: one group of all rows
  int32_t groups, rows;      // rows: end of the row range
  int32_t M, N, K;           // (M or K of a grouped dimension: its rows)
  int32_t c_dtype;
  int32_t kslice;            // k's of a slice (all: K or more)
  float* slices;             // ROWS_SLICE: M x N sums of every slice, one after the other (grouped along
                             // K: the slices of all groups' rows in a row)
  int32_t a_pad8, b_pad8;    // k-major operand: readable up to the next multiple of 8 past M (N)
  // the classification loss
  int32_t classes;
  float* sum;                // ROWS_SUM: M x N, row stride N
  int32_t add, last;         // ROWS_SUM
  int32_t col0;              // ROWS_LSE, ROWS_DZ: class of column 0
  float scale;
  const int64_t* targets;
  const float* lse;
  const float* grad_loss;
  float2* part;              // ROWS_LSE: (maximum, sum) per row and column block, row stride n_part
  float* ztarget;            // ROWS_LSE: the target's logit of every row that has one
  int32_t n_part;
  // work of its own that the launch takes along in workgroups behind its
  // tiles', which spares a launch (5 us each in a chain of short ones)
  void* copy;                // ROWS_DZ of the kernel without staging: A's rows, zeros for those without a
  int32_t ld_copy;           // target and up to ld_copy columns (nullptr: none)
  int32_t twice;             // ... each as rows 2 i and 2 i + 1
  RowsJoin join;             // grouped along K: an earlier launch's slices
  // A bf16 dz is held as two pieces, the rounding of the value and of what that
  // leaves (off by 2^-16 of a value at most; with one piece, off by 2^-8, the
  // gradients were 1.9e-3 off in the 2-norm where their own rounding is
  // 1.7e-3).  Row r's lie in rows 2 r and 2 r + 1, so that its products are those
  // of twice the rows: dW's k runs over both (x's rows twice each), dx's rows
  // are added by pairs.
  int32_t pairs;             // grouped along M, bf16, B k-major: 1: A's rows are such pairs, C has M / 2 rows
  int64_t c_low;             // ROWS_DZ in bf16: elements from a value's first piece to its second
};

// Group g's row range from the offsets, whatever they hold: each clamped to
// [0, rows], and to the largest before it, so that ranges never overlap.
// Every wave computes the same; `carry` is the running maximum of the groups
// before `base`.
__device__ __forceinline__ int wave_scan_max(int v, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(v, d, 64);
    if (lane >= d) v = max(v, o);
  }
  return v;
}
__device__ __forceinline__ int wave_scan_add(int v, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(v, d, 64);
    if (lane >= d) v += o;
  }
  return v;
}
struct GroupRange {
  int start, end;
};
__device__ __forceinline__ GroupRange lane_range(const int32_t* offsets, int groups, int rows, int g, int lane,
                                                 int& carry) {
  auto at = [&](int i) { return min(max((int)gld_u32(offsets, min(i, groups)), 0), rows); };
  const int a = at(g), b = at(g + 1);
  const int start = max(wave_scan_max(a, lane), carry);
  GroupRange r{start, g < groups ? max(start, b) : start};
  carry = __shfl(r.end, 63, 64);
  return r;
}
// (start, end) of group g
__device__ __forceinline__ GroupRange group_range(const RowsProd& p, int g, int lane) {
  if (!p.offsets) return GroupRange{0, p.rows};
  int carry = 0;
  for (int base = 0;; base += 64) {
    const GroupRange r = lane_range(p.offsets, p.groups, p.rows, base + lane, lane, carry);
    if (g < base + 64)
      return GroupRange{__builtin_amdgcn_readfirstlane(__shfl(r.start, g - base, 64)),
                        __builtin_amdgcn_readfirstlane(__shfl(r.end, g - base, 64))};
  }
}

// Tile `id` of a launch: `per` tiles (columns) for every BM rows of a group.
// The tiles are dealt so that each XCD (blocks go to the 8 of them in turn)
// gets a run of consecutive tiles, which share operand panels in its L2;
// within a group they go down bands of 8 row tiles.
struct RowsTile {
  int g, start, end;   // group and its rows
  int ti, tj;
  int first;           // row tiles of the groups before
  bool any;
};
__device__ __forceinline__ int xcd_run(int id, int total) {
  const int per = total >> 3, rest = total & 7, x = id & 7;
  return x * per + min(x, rest) + (id >> 3);
}
__device__ __forceinline__ void band_order(int t, int mt, int nt, int& ti, int& tj) {
  const int band = t / (8 * nt), in = t - band * 8 * nt;
  const int h = min(8, mt - band * 8);
  ti = band * 8 + in % h;
  tj = in / h;
}
__device__ __forceinline__ RowsTile rows_tile(const RowsProd& p, int bm, int nt, int id, int lane) {
  RowsTile t{0, 0, 0, 0, 0, 0, false};
  if (!p.offsets) {
    const int mt = (p.rows + bm - 1) / bm, total = mt * nt;
    if (id >= total) return t;
    t.end = p.rows;
    band_order(xcd_run(id, total), mt, nt, t.ti, t.tj);
    t.any = true;
    return t;
  }
  // (groups 64 at a time; up to 64 of them in one pass)
  int total = 0, carry = 0, mine = 0, upto = 0;
  GroupRange r{0, 0};
  for (int base = 0; base < p.groups; base += 64) {
    r = lane_range(p.offsets, p.groups, p.rows, base + lane, lane, carry);
    mine = (r.end - r.start + bm - 1) / bm;
    upto = wave_scan_add(mine, lane);
    total += __shfl(upto, 63, 64);
  }
  if (id >= total * nt) return t;
  const int run = xcd_run(id, total * nt), row = run / nt;
  int before = 0;   // row tiles of the groups before
  carry = 0;
  for (int base = 0; base < p.groups; base += 64) {
    if (p.groups > 64) {
      r = lane_range(p.offsets, p.groups, p.rows, base + lane, lane, carry);
      mine = (r.end - r.start + bm - 1) / bm;
      upto = before + wave_scan_add(mine, lane);
    }
    const unsigned long long has = __ballot(upto > row);
    if (has) {
      const int l = __ffsll(has) - 1, mt = __builtin_amdgcn_readlane(mine, l);
      t.g = base + l;
      t.start = __builtin_amdgcn_readlane(r.start, l);
      t.end = __builtin_amdgcn_readlane(r.end, l);
      t.first = __builtin_amdgcn_readlane(upto, l) - mt;
      band_order(run - t.first * nt, mt, nt, t.ti, t.tj);
      t.any = true;
      return t;
    }
    before = __shfl(upto, 63, 64);
  }
  return t;
}

// The tile of a block of a product grouped along K (edge bm): group, tile,
// its k range [k0, k1) of the rows, and where its sums go (ROWS_SLICE).
struct RowsKTile {
  int g, ti, tj, k0, k1, slot;
  bool any;
};
template <int EPI>
__device__ __forceinline__ RowsKTile rows_ktile(const RowsProd& p, int bm, int id, int lane) {
  const int mt = (p.M + bm - 1) / bm, nt = (p.N + bm - 1) / bm;
  RowsKTile k{0, 0, 0, 0, 0, 0, false};
  if constexpr (EPI == ROWS_SLICE) {
    // slices of the groups' rows as row tiles, tiles as their columns
    const RowsTile t = rows_tile(p, p.kslice, mt * nt, id, lane);
    if (!t.any) return k;
    k.g = t.g;
    band_order(t.tj, mt, nt, k.ti, k.tj);
    k.k0 = t.start + t.ti * p.kslice;
    k.k1 = k.k0 + min(t.end - k.k0, p.kslice);
    k.slot = t.first + t.ti;
  } else {
    // up to 64 groups: the tiles of those with the most rows first, dealt to
    // the XCDs in runs of 8 (a band's column), so that the longest tiles start
    // first and everywhere.  (Groups in their order and one run per XCD: 32768
    // rows over 16 matrices of 2048^2 as a router deals them, 394 us; this
    // way 320.)
    const int tiles = mt * nt;
    if (p.offsets && p.groups <= 64) {
      const int at = ((id >> 6 << 3) + (id & 7)) * 8 + (id >> 3 & 7);
      if (at >= p.groups * tiles) return k;
      int carry = 0;
      const GroupRange r = lane_range(p.offsets, p.groups, p.rows, lane, lane, carry);
      const int mine = lane < p.groups ? r.end - r.start : -1;
      int rank = 0;
      for (int g = 0; g < p.groups; ++g) {
        const int other = __builtin_amdgcn_readlane(mine, g);
        rank += other > mine || (other == mine && g < lane);
      }
      const unsigned long long mask = __ballot(lane < p.groups && rank == at / tiles);
      k.g = __ffsll(mask) - 1;
      k.k0 = __builtin_amdgcn_readlane(r.start, k.g);
      k.k1 = __builtin_amdgcn_readlane(r.end, k.g);
      band_order(at % tiles, mt, nt, k.ti, k.tj);
    } else {
      if (id >= p.groups * tiles) return k;
      const int run = xcd_run(id, p.groups * tiles);
      k.g = run / tiles;
      band_order(run % tiles, mt, nt, k.ti, k.tj);
      const GroupRange r = group_range(p, k.g, lane);
      k.k0 = r.start;
      k.k1 = r.end;
    }
  }
  k.any = true;
  return k;
}

// Orders results by size, zero behind the largest (2 |v| as bits, less 1): a
// split product below small_key(kSplitLo) may lack low pieces of its operands.
__device__ __forceinline__ uint32_t small_key(float v) { return (__float_as_uint(v) << 1) - 1; }

// 16 or 8 bytes at any 2-byte aligned address
typedef uint32_t orth_u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t orth_u32x2_a2 __attribute__((ext_vector_type(2), aligned(2)));
typedef float orth_f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));

// Four consecutive values of row i, columns j ..: C's first n of them exist.
__device__ __forceinline__ void rows_store4(void* C, int64_t at, int dtype, float4 v, int n) {
  if (n >= 4) {
    if (dtype == ORTH_BF16)
      *(ORTH_GLOBAL orth_u32x2_a2*)(static_cast<uint16_t*>(C) + at) = orth_u32x2_a2{cvt2_bf16(v.x, v.y), cvt2_bf16(v.z, v.w)};
    else
      *(ORTH_GLOBAL orth_f32x4_a4*)(static_cast<float*>(C) + at) = orth_f32x4_a4{v.x, v.y, v.z, v.w};
  } else {
    if (n > 0) store_from_f32(C, at, dtype, v.x);
    if (n > 1) store_from_f32(C, at + 1, dtype, v.y);
    if (n > 2) store_from_f32(C, at + 2, dtype, v.z);
  }
}

// Four consecutive values summed over the slices, in order, eight loads in
// flight.  (id, n: in values; the first `have` of the four exist)
__device__ __forceinline__ float4 join4(float4 v, const float* at, int64_t n, int slices, int have) {
  for (int s = 0; s < slices; s += 8) {
    float4 u[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float* q = at + min(s + k, slices - 1) * n;
      if (have == 4) {
        const orth_f32x4_a4 w = *(const ORTH_GLOBAL orth_f32x4_a4*)q;
        u[k] = make_float4(w.x, w.y, w.z, w.w);
      } else {
        u[k] = make_float4(gld_f32(q, 0), have > 1 ? gld_f32(q, 1) : 0.f, have > 2 ? gld_f32(q, 2) : 0.f, 0.f);
      }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (s + k < slices) {
        v.x += u[k].x;
        v.y += u[k].y;
        v.z += u[k].z;
        v.w += u[k].w;
      }
  }
  return v;
}

// A workgroup's part (256 threads) of the join: a thread takes four columns of
// a row.
__device__ __forceinline__ void rows_join_block(const RowsJoin& p, int64_t block, int tid) {
  const int nq = (p.N + 3) / 4;
  const int64_t id = block * 256 + tid, i = id / nq;
  if (i >= p.M) return;
  const int j = (int)(id - i * nq) * 4, have = min(4, p.N - j);
  float* sum = p.sum + i * p.N + j;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  if (p.add) v = join4(v, sum, 0, 1, have);
  v = join4(v, p.slices + i * p.N + j, (int64_t)p.M * p.N, p.n, have);
  if (p.last)
    rows_store4(p.C, i * p.ldc + j, p.c_dtype, v, have);
  else
    rows_store4(sum, 0, ORTH_F32, v, have);
}
__host__ __device__ inline int64_t rows_join_blocks(const RowsJoin& p) {
  return p.slices ? ((int64_t)p.M * ((p.N + 3) / 4) + 255) / 256 : 0;
}
// Whether this workgroup (256 threads or more, one group) does a part of the
// join that its launch takes along; then it has.
__device__ __forceinline__ bool rows_joined(const RowsJoin& p, int tid) {
  if (!p.slices) return false;
  const int64_t block = (int64_t)blockIdx.x - ((int64_t)gridDim.x - rows_join_blocks(p));
  if (block < 0) return false;
  if (tid < 256) rows_join_block(p, block, tid);
  return true;
}

// What bf16 leaves of four values (nothing of one that it makes infinite).
__device__ __forceinline__ float4 low4(float4 v) {
  const uint32_t a = cvt2_bf16(v.x, v.y), b = cvt2_bf16(v.z, v.w);
  auto rest = [](float x, uint32_t h) {
    const float r = x - __uint_as_float(h);
    return r * 0.f == 0.f ? r : 0.f;
  };
  return make_float4(rest(v.x, a << 16), rest(v.y, a & 0xffff0000u), rest(v.z, b << 16), rest(v.w, b & 0xffff0000u));
}

// One 4-column piece of a row of a finished tile: row i (of A and C), column
// j, n columns left.
template <int EPI>
__device__ __forceinline__ void rows_finish4(const RowsProd& p, int g, int64_t i, int j, float4 v, int n) {
  if (n <= 0) return;
  if constexpr (EPI == ROWS_STORE) {
    rows_store4(p.C, (p.offsets ? g * p.gc : 0) + i * p.ldc + j, p.c_dtype, v, n);
  } else if constexpr (EPI == ROWS_SUM) {
    float* s = p.sum + i * p.N + j;
    float w[4] = {v.x, v.y, v.z, v.w};
    if (p.add) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (q < n) w[q] += gld_f32(s, q);
    }
    const float4 u = make_float4(w[0], w[1], w[2], w[3]);
    if (p.last)
      rows_store4(p.C, i * p.ldc + j, p.c_dtype, u, n);
    else
      rows_store4(s, 0, ORTH_F32, u, n);
  } else if constexpr (EPI == ROWS_SLICE) {
    rows_store4(p.slices, ((int64_t)g * (p.M >> p.pairs) + i) * p.N + j, ORTH_F32, v, n);   // (g: the slice)
  } else {
    static_assert(EPI == ROWS_DZ);
    rows_store4(p.C, i * p.ldc + j, p.c_dtype, v, 4);
    if (p.c_low) rows_store4(p.C, i * p.ldc + j + p.c_low, p.c_dtype, low4(v), 4);
  }
}

// The epilogue of a wave's block, MI x NI accumulators of 32 x 32 that start
// at row ibase and column jbase: 32 rows at a time through the wave's own LDS
// buffers in turn (two of 32 rows of 32 NI floats, 16-byte pieces XOR-swizzled by the row, so
// that neither the row-major pass nor a pass of one row per lane meets bank
// conflicts), then stores along rows.  mrows: rows of the block that exist;
// block: the column block's number (ROWS_LSE).  Whole blocks, all but those
// at the edges, run without a bounds check, from addresses that are uniform
// but for a 32-bit offset.  What each row needs (ROWS_DZ) is loaded once,
// before the first chunk.  (A round of 256-tiles of logits with K = 64 took 21
// us with checks and loads per piece, 13 us this way: 4 to the first products,
// 7 of epilogue, where every tile of the round reads or writes at once.)
typedef float orth_f32x16 __attribute__((ext_vector_type(16)));
constexpr float kLog2e = 1.4426950408889634f;

// What a sum of exponentials is relative to, by its largest value: 0 for an
// infinite one, so that no difference of infinities is formed (every value -inf:
// the sum is 0, one +inf: it is inf).
__device__ __forceinline__ float lse_base(float top) { return fabsf(top) == INFINITY ? 0.f : top; }

template <int MI, int NI, int EPI, bool PAIRS>   // PAIRS: p.pairs may be set
struct RowsEpilogue {
  static constexpr int TN = NI * 32, NC = TN / 4;   // columns, 16-byte pieces of a row
  static constexpr int RQ = 64 / NC, NQ = 32 / RQ;  // rows of a pass of the wave, passes of a chunk
  static constexpr int RV = (MI + 1) / 2;           // per-row registers: row 64 v + lane
  const RowsProd& p;
  float *buf, *next;   // the chunk's buffer, the one of the chunk after it
  int64_t ibase;
  int g, jbase, mrows, block, lane;
  // ROWS_DZ (per row): the target's column in the block (-1: elsewhere, -2:
  // the row has none), lse, scale * grad_loss; ROWS_LSE: the target's column
  int tcol[RV];
  float lse[RV], gs[RV];

  __device__ __forceinline__ int at(int r, int c) const { return r * TN + (((c >> 2) ^ (r & (NC - 1))) << 2) + (c & 3); }
  __device__ __forceinline__ orth_f32x4 piece(int r, int c) const {
    return *reinterpret_cast<const orth_f32x4*>(&buf[at(r, c)]);
  }
  __device__ __forceinline__ void load_rows() {
    if constexpr (EPI == ROWS_DZ || EPI == ROWS_LSE) {
#pragma unroll
      for (int v = 0; v < RV; ++v) {
        const int r = v * 64 + lane;
        tcol[v] = -2;
        if (r < mrows && r < MI * 32) {
          const int64_t t = ((const ORTH_GLOBAL int64_t*)p.targets)[ibase + r], c = t - p.col0 - jbase;
          tcol[v] = t < 0 || t >= p.classes ? -2 : c >= 0 && c < TN ? (int)c : -1;
          if constexpr (EPI == ROWS_DZ) {
            lse[v] = gld_f32(p.lse, ibase + r);
            gs[v] = gld_f32(p.grad_loss, ibase + r) * p.scale;
          }
        }
      }
    }
  }
  __device__ __forceinline__ void stage(const orth_f32x16 (&acc)[NI]) {
    const float f = EPI == ROWS_LSE || EPI == ROWS_DZ ? p.scale : 1.f;
#pragma unroll
    for (int ni = 0; ni < NI; ++ni)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float v = acc[ni][r];
        next[at(8 * (r >> 2) + 4 * (lane >> 5) + (r & 3), ni * 32 + (lane & 31))] =
            EPI == ROWS_LSE || EPI == ROWS_DZ ? v * f : v;
      }
  }
  // The staged chunk becomes the current one (the buffers belong to this wave
  // alone).
  __device__ __forceinline__ void turn() {
    float* t = buf;
    buf = next;
    next = t;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }

  // One row per lane, a half of its columns each.
  template <bool FULL>
  __device__ __forceinline__ void lse_chunk(int mi) {
    const int r = lane & 31, c0 = (lane >> 5) * (TN / 2);
    const int left = p.N - jbase - c0;   // columns of this half row that exist
    orth_f32x4 v[NC / 2];
    float top = -INFINITY;
#pragma unroll
    for (int q = 0; q < NC / 2; ++q) {
      v[q] = piece(r, c0 + 4 * q);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (!FULL && 4 * q + k >= left) v[q][k] = -INFINITY;
        top = fmaxf(top, v[q][k]);
      }
    }
    const float from = lse_base(top);
    float sum = 0.f;
#pragma unroll
    for (int q = 0; q < NC / 2; ++q)
#pragma unroll
      for (int k = 0; k < 4; ++k) sum += __builtin_amdgcn_exp2f((v[q][k] - from) * kLog2e);
    const float otop = __shfl_xor(top, 32, 64), osum = __shfl_xor(sum, 32, 64);
    const float m = fmaxf(top, otop), to = lse_base(m);
    const float total = sum * __builtin_amdgcn_exp2f((top - to) * kLog2e) +
                        osum * __builtin_amdgcn_exp2f((otop - to) * kLog2e);
    const int tc = __shfl(tcol[mi / 2], (mi & 1) * 32 + r, 64) - c0;
    if (FULL || mi * 32 + r < mrows) {
      const int64_t i = ibase + mi * 32 + r;
      if (lane < 32) {
        gst_f32(p.part, (i * p.n_part + block) * 2, m);
        gst_f32(p.part, (i * p.n_part + block) * 2 + 1, total);
      }
      if (tc >= 0 && tc < TN / 2) gst_f32(p.ztarget, i, buf[at(r, c0 + tc)]);
    }
  }

  // dz of a piece of row r of chunk mi
  __device__ __forceinline__ float4 dz4(int mi, int r, int c, orth_f32x4 z) const {
    const int from = (mi & 1) * 32 + r, tc = __shfl(tcol[mi / 2], from, 64);
    const float l = __shfl(lse[mi / 2], from, 64), f = __shfl(gs[mi / 2], from, 64);
    float w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float e = __builtin_amdgcn_exp2f((z[k] - l) * kLog2e);
      // a row without a target gets zeros whatever its values are
      w[k] = tc == -2 ? 0.f : f * (c + k == tc ? e - 1.f : e);
    }
    return make_float4(w[0], w[1], w[2], w[3]);
  }

  // Whole blocks: four columns per lane, RQ rows (PAIR: of C) per pass.
  template <bool BF16, bool PAIR>
  __device__ __forceinline__ void write_chunk(int mi) {
    const int lr = lane / NC, lc = (lane % NC) * 4;
    constexpr int ES = BF16 ? 2 : 4;
    const int64_t row0 = (ibase + mi * 32) >> (PAIR ? 1 : 0);
    char* base;
    int64_t ld;
    if constexpr (EPI == ROWS_SLICE) {
      base = reinterpret_cast<char*>(p.slices + ((int64_t)g * (PAIR ? p.M / 2 : p.M) + row0) * p.N + jbase);
      ld = p.N;
    } else if constexpr (EPI == ROWS_SUM) {
      base = static_cast<char*>(p.C) + (row0 * p.ldc + jbase) * ES;
      ld = p.ldc;
    } else {
      base = static_cast<char*>(p.C) + ((p.offsets ? g * p.gc : 0) + row0 * p.ldc + jbase) * ES;
      ld = p.ldc;
    }
    const uint32_t off = (uint32_t)(lr * ld + lc) * ES;
#pragma unroll
    for (int q = 0; q < (PAIR ? NQ / 2 : NQ); ++q) {
      const int r = q * RQ + lr;
      const orth_f32x4 v = PAIR ? piece(2 * r, lc) + piece(2 * r + 1, lc) : piece(r, lc);
      float4 o = make_float4(v.x, v.y, v.z, v.w);
      if constexpr (EPI == ROWS_DZ) o = dz4(mi, r, lc, v);
      if constexpr (EPI == ROWS_DZ && BF16)
        rows_store4(base + ((int64_t)q * RQ * ld + p.c_low) * ES + off, 0, ORTH_BF16, low4(o), 4);
      if constexpr (EPI == ROWS_SUM) {
        if (p.add) {
          const orth_f32x4_a4 u = *(const ORTH_GLOBAL orth_f32x4_a4*)(p.sum + (row0 + r) * p.N + jbase + lc);
          o = make_float4(o.x + u.x, o.y + u.y, o.z + u.z, o.w + u.w);
        }
        if (!p.last) {
          rows_store4(p.sum, (row0 + r) * p.N + jbase + lc, ORTH_F32, o, 4);
          continue;
        }
      }
      rows_store4(base + (int64_t)q * RQ * ld * ES + off, 0, BF16 ? ORTH_BF16 : ORTH_F32, o, 4);
    }
  }
  // Blocks at the edges.
  __device__ __forceinline__ void edge_chunk(int mi) {
    const int ncols = (EPI == ROWS_DZ ? (p.N + 7) / 8 * 8 : p.N) - jbase;   // columns to write
    const int lr = lane / NC, lc = (lane % NC) * 4;
    const int two = PAIRS ? p.pairs : 0;
#pragma unroll 4
    for (int q = 0; q < NQ; ++q) {
      if (q >= NQ >> two) break;
      const int r = q * RQ + lr;
      const orth_f32x4 v = two ? piece(2 * r, lc) + piece(2 * r + 1, lc) : piece(r, lc);
      float4 o = make_float4(v.x, v.y, v.z, v.w);
      if constexpr (EPI == ROWS_DZ) {
        o = dz4(mi, r, lc, v);
        // (the columns that pad the piece to a multiple of 8 get zeros)
        const int n = p.N - jbase - lc;
        o = make_float4(n > 0 ? o.x : 0.f, n > 1 ? o.y : 0.f, n > 2 ? o.z : 0.f, n > 3 ? o.w : 0.f);
      }
      if (mi * 32 + (r << two) < mrows)
        rows_finish4<EPI>(p, g, ((ibase + mi * 32) >> two) + r, jbase + lc, o, ncols - lc);
    }
  }

  template <bool BF16>
  __device__ __forceinline__ void write(int mi) {
    if constexpr (PAIRS) {
      if (p.pairs) {
        write_chunk<BF16, true>(mi);
        return;
      }
    }
    write_chunk<BF16, false>(mi);
  }
  __device__ __forceinline__ void run(const orth_f32x16 (&acc)[MI][NI]) {
    load_rows();
    const int64_t ld = EPI == ROWS_SLICE ? p.N : p.ldc;
    if (mrows >= MI * 32 && p.N - jbase >= TN && ld <= (1 << 24)) {   // (32-bit offsets)
      // a chunk is staged while the one before it is written
      stage(acc[0]);
#pragma unroll
      for (int mi = 0; mi < MI; ++mi) {
        turn();
        if (mi + 1 < MI) stage(acc[mi + 1 < MI ? mi + 1 : mi]);
        if constexpr (EPI == ROWS_LSE)
          lse_chunk<true>(mi);
        else if (EPI != ROWS_SLICE && p.c_dtype == ORTH_BF16)
          write<true>(mi);
        else
          write<false>(mi);
      }
    } else {
#pragma unroll
      for (int mi = 0; mi < MI; ++mi) {
        if (mi * 32 >= mrows) break;
        stage(acc[mi]);
        turn();
        if constexpr (EPI == ROWS_LSE)
          lse_chunk<false>(mi);
        else
          edge_chunk(mi);
      }
    }
  }
};
template <int MI, int NI, int EPI, bool PAIRS>
__device__ __forceinline__ void rows_epilogue(const RowsProd& p, int g, const orth_f32x16 (&acc)[MI][NI], float* buf,
                                              float* buf2, int64_t ibase, int jbase, int mrows, int block, int lane) {
  if (mrows <= 0) return;
  RowsEpilogue<MI, NI, EPI, PAIRS> e{p, buf2, buf, ibase, g, jbase, mrows, block, lane, {}, {}, {}};
  e.run(acc);
}

// row tiles (slices) of all groups, at most
inline int64_t rows_parts(const RowsProd& p, int64_t edge) {
  if (!p.offsets) return ((int64_t)p.rows + edge - 1) / edge;
  const int64_t parts = p.groups < p.rows ? p.groups : p.rows;
  return (p.rows - parts) / edge + parts;
}
// Host: blocks of a launch with square tiles of edge `tile` (grouped along M:
// an upper bound, as every group ends in at most one tile that is not full),
// the tile edge for a product, the launches.  at, bt: the operand is k-major
// (at: grouped along K).
inline int64_t rows_blocks(const RowsProd& p, bool at, int tile) {
  const int64_t nt = (p.N + tile - 1) / tile;
  return at ? (int64_t)p.groups * ((p.M + tile - 1) / tile) * nt : rows_parts(p, tile) * nt;
}
// tiles to expect: the last one of a group is half full on average
inline double rows_expected(const RowsProd& p, bool at, int tile) {
  if (at || !p.offsets) return (double)rows_blocks(p, at, tile);
  return ((double)p.rows / tile + 0.5 * (p.groups < p.rows ? p.groups : p.rows)) * ((p.N + tile - 1) / tile);
}
inline int64_t rows_launch_blocks(const RowsProd& p, bool at, int epi, int tile) {
  // (rows_ktile deals whole sets of 64)
  if (at && epi != ROWS_SLICE) return (rows_blocks(p, at, tile) + 63) / 64 * 64 + rows_join_blocks(p.join);
  if (!at) return rows_blocks(p, at, tile);
  return rows_parts(p, p.kslice) * ((p.M + tile - 1) / tile) * ((p.N + tile - 1) / tile);
}
bool rows_bf16_dma(const RowsProd& p, bool at, bool bt);   // whether the operands allow direct-to-LDS loads
int rows_bf16_tile(const RowsProd& p, bool at, bool bt);
int rows_f32_tile(const RowsProd& p, bool at);
hipError_t launch_rows_direct(const RowsProd& p, int dtype, bool bt, int epi, int slices, const char* name,
                              hipStream_t s);
hipError_t launch_rows_join(const RowsJoin& p, const char* name, hipStream_t s);
// the slices of every group's rows into its C
hipError_t launch_rows_join_groups(const RowsProd& p, const char* name, hipStream_t s);
// grouped along K, few rows (at most 65535 groups)
int64_t rows_outer_blocks(const RowsProd& p, int dtype);
hipError_t launch_rows_outer(const RowsProd& p, int dtype, const char* name, hipStream_t s);
hipError_t launch_rows_bf16(const RowsProd& p, bool at, bool bt, int epi, int tile, const char* name, hipStream_t s);
hipError_t launch_rows_f32(const RowsProd& p, bool at, bool bt, int epi, int tile, const char* name, hipStream_t s);

}  // namespace orth
