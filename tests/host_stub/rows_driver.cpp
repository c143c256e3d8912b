// Drives the host code of the row-grouped products, the head's loss and the
// gradient clipping (rows*.hip, grad_clip.hip, built for the CPU) through random
// calls, with the HIP runtime replaced: a launch enqueues nothing, but the
// memory that its kernel's descriptor says it reads and writes has to lie in
// the call's tensors and in a workspace of exactly the size that was asked for,
// and what it writes apart from what it reads.  Addresses are made up and never
// followed.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <random>
#include <string>
#include <vector>

#include "../../paper_2601_13776_amd/csrc/rows.h"

using namespace orth;

// ------------------------------------------------------------ stand-ins ---
namespace {
std::map<const void*, std::string>& names() {
  static std::map<const void*, std::string> n;
  return n;
}
std::string g_what;   // the call under way
long g_launches = 0, g_calls = 0;
const char* const kKernels[] = {"rows_bf16_kernelILi256", "rows_bf16_kernelILi128", "rows_f32_kernelILi128", "rows_f32_kernelILi64",
                                "rows_direct_kernel", "rows_outer_kernel", "rows_join_kernel", "rows_join_groups_kernel",
                                "pad_rows_kernel", "xent_join_kernelILi1", "xent_join_kernelILi4", "grad_small_kernel",
                                "grad_norm_join_kernel", "grad_norm_kernel", "grad_norm_inline_kernel", "grad_clip_kernel",
                                "grad_clip_inline_kernel"};
std::map<std::string, long> g_seen;
struct Region {
  uintptr_t at, end;
  bool writable;
  const char* name;
};
std::vector<Region> g_regions;

[[noreturn]] void violation(const std::string& msg) {
  fprintf(stderr, "VIOLATION: %s: %s\n", g_what.c_str(), msg.c_str());
  exit(3);
}
struct Extent {
  uintptr_t at;
  int64_t bytes;
  const char* name;
};
struct Access {
  std::vector<Extent> reads, writes;
  void add(std::vector<Extent>& v, const void* p, int64_t bytes, const char* name) {
    if (bytes > 0) v.push_back({reinterpret_cast<uintptr_t>(p), bytes, name});
  }
  void read(const void* p, int64_t bytes, const char* name) { add(reads, p, bytes, name); }
  void write(const void* p, int64_t bytes, const char* name) { add(writes, p, bytes, name); }
  void check(const std::string& kernel) const {
    auto inside = [&](const Extent& e, bool write) {
      for (const Region& r : g_regions)
        if (e.at >= r.at && e.at + (uintptr_t)e.bytes <= r.end && (r.writable || !write)) return;
      violation(kernel + (write ? " writes " : " reads ") + e.name + " outside the call's memory");
    };
    for (const Extent& e : reads) inside(e, false);
    for (const Extent& e : writes) inside(e, true);
    for (size_t i = 0; i < writes.size(); ++i) {
      const Extent& w = writes[i];
      auto meets = [&](const Extent& e) { return w.at < e.at + (uintptr_t)e.bytes && e.at < w.at + (uintptr_t)w.bytes; };
      for (const Extent& r : reads)
        if (meets(r)) violation(kernel + " writes " + w.name + " over " + r.name + " that it reads");
      for (size_t j = 0; j < i; ++j)
        if (meets(writes[j])) violation(kernel + " writes " + w.name + " over " + writes[j].name);
    }
  }
};
void need(bool ok, const std::string& msg) {
  if (!ok) violation(msg);
}

int64_t es_of(int dtype) { return dtype == ORTH_BF16 ? 2 : 4; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

void join_access(const RowsJoin& j, Access& a) {
  if (!j.slices) return;
  const int64_t mn = (int64_t)j.M * j.N;
  a.read(j.slices, j.n * mn * 4, "slices");
  if (j.last) {
    if (j.add) a.read(j.sum, mn * 4, "sum");
    a.write(j.C, ((int64_t)(j.M - 1) * j.ldc + j.N) * es_of(j.c_dtype), "C of a join");
  } else {
    a.write(j.sum, mn * 4, "sum");
  }
}

// A product whose operands have type dt, on tiles of edge `tile`.
void product_access(const std::string& kernel, const RowsProd& p, int dt, bool at, bool bt, int epi, int tile, dim3 grid) {
  Access a;
  const int64_t es = es_of(dt), es_c = es_of(p.c_dtype);
  const int64_t m_in = at && p.a_pad8 ? ceil_div(p.M, 8) * 8 : p.M, n_in = bt && p.b_pad8 ? ceil_div(p.N, 8) * 8 : p.N;
  const int64_t k = at ? p.rows : p.K;
  const int64_t m_out = p.M >> p.pairs;
  need(p.groups >= 1 && p.M >= 0 && p.N >= 1, kernel + ": sizes");
  need(!p.pairs || (dt == ORTH_BF16 && !at && bt && p.M % 2 == 0 && !p.offsets), kernel + ": pairs");
  if (!(at ? k == 0 : p.M == 0)) {
    a.read(p.A, at ? ((k - 1) * p.lda + m_in) * es : ((int64_t)(p.M - 1) * p.lda + k) * es, "A");
    a.read(p.B, at ? ((k - 1) * p.ldb + n_in) * es
                   : ((p.offsets ? (p.groups - 1) * p.gb : 0) + (bt ? (k - 1) * p.ldb + n_in : (p.N - 1) * p.ldb + k)) * es, "B");
  }
  if (p.offsets) a.read(p.offsets, ((int64_t)p.groups + 1) * 4, "offsets");
  const int64_t c_one = at ? ((int64_t)(p.M - 1) * p.ldc + p.N) : (m_out - 1) * p.ldc + p.N;
  int64_t blocks = 0;
  if (at) {
    blocks = epi == ROWS_SLICE ? rows_parts(p, p.kslice) * ceil_div(p.M, tile) * ceil_div(p.N, tile)
                               : (int64_t)p.groups * ceil_div(p.M, tile) * ceil_div(p.N, tile);
  } else {
    blocks = rows_parts(p, tile) * ceil_div(p.N, tile);
  }
  switch (epi) {
    case ROWS_STORE:
      a.write(p.C, ((at && p.offsets ? (p.groups - 1) * p.gc : 0) + c_one) * es_c, "C");
      break;
    case ROWS_SUM:
      if (p.last) {
        a.write(p.C, c_one * es_c, "C");
        if (p.add) a.read(p.sum, m_out * p.N * 4, "sum");
      } else {
        a.write(p.sum, m_out * p.N * 4, "sum");
      }
      break;
    case ROWS_SLICE:
      need(p.kslice > 0, kernel + ": kslice");
      if (!at) need((int64_t)grid.y == ceil_div(p.K, p.kslice), kernel + ": slices along y");
      a.write(p.slices, (at ? rows_parts(p, p.kslice) * p.M : (int64_t)grid.y * m_out) * p.N * 4, "slices");
      break;
    case ROWS_LSE: {
      const int per = tile == 32 ? 1 : dt == ORTH_BF16 ? 2 : tile / 32;
      need(p.n_part == ceil_div(p.N, tile) * per, kernel + ": n_part");
      a.read(p.targets, (int64_t)p.M * 8, "targets");
      a.write(p.part, (int64_t)p.M * p.n_part * 8, "part");
      a.write(p.ztarget, (int64_t)p.M * 4, "ztarget");
      break;
    }
    case ROWS_DZ:
      need(p.col0 + p.N <= p.classes, kernel + ": classes");
      need((dt == ORTH_BF16) == (p.c_low > 0), kernel + ": dz's pieces");
      need(p.ldc >= (p.c_low ? 2 : 1) * ceil_div(p.N, 8) * 8 && (!p.c_low || p.c_low >= ceil_div(p.N, 8) * 8), kernel + ": ldc of dz");
      a.read(p.targets, (int64_t)p.M * 8, "targets");
      a.read(p.lse, (int64_t)p.M * 4, "lse");
      a.read(p.grad_loss, (int64_t)p.M * 4, "grad_loss");
      a.write(p.C, ((int64_t)(p.M - 1) * p.ldc + p.c_low + ceil_div(p.N, 8) * 8) * es, "dz");
      if (p.copy) {
        need(tile == 32 && p.ld_copy >= p.K && p.ld_copy % 8 == 0, kernel + ": copy");
        a.write(p.copy, ((int64_t)p.M << p.twice) * p.ld_copy * es, "copy");
        blocks += ceil_div(p.rows, 8);
      }
      break;
  }
  if (at) {
    join_access(p.join, a);
    blocks += rows_join_blocks(p.join);
  }
  need((int64_t)grid.x >= blocks, kernel + ": grid too small");
  need((int64_t)grid.x < (1 << 23) + (1 << 22) && grid.y <= 65535, kernel + ": grid too large");
  a.check(kernel);
}

// The integers of a mangled name's template arguments behind `name`.
std::vector<int> args_of(const std::string& s, const char* name) {
  std::vector<int> v;
  size_t i = s.find(name);
  for (i += strlen(name) + 1; i < s.size() && s[i] == 'L'; ++i) {
    v.push_back(atoi(s.c_str() + i + 2));
    i = s.find('E', i);
  }
  return v;
}
}  // namespace

extern "C" {
void** __hipRegisterFatBinary(const void*) {
  static void* h;
  return &h;
}
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned, void*, void*, void*, void*, int*) {
  names()[host] = name;
}
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
static dim3 t_grid, t_block;
static size_t t_lds;
static hipStream_t t_stream;
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t s) {
  t_grid = grid;
  t_block = block;
  t_lds = lds;
  t_stream = s;
  return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* s) {
  *grid = t_grid;
  *block = t_block;
  *lds = t_lds;
  *s = t_stream;
  return hipSuccess;
}
hipError_t hipGetLastError(void) { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "error"; }
hipError_t hipFuncSetAttribute(const void*, hipFuncAttribute, int bytes) {
  need(bytes <= 160 * 1024, "LDS past a compute unit's");
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** args, size_t, hipStream_t) {
  ++g_launches;
  const std::string& n = names()[f];
  for (const char* k : kKernels)
    if (n.find(k) != std::string::npos) {
      ++g_seen[k];
      break;
    }
  auto is = [&](const char* s) { return n.find(s) != std::string::npos; };
  need(grid.x > 0 && grid.y > 0 && (uint64_t)grid.x * block.x < (1ull << 32), n + ": grid");
  if (is("rows_bf16_kernel")) {   // <tile, at, bt, epi, dma, aux>
    const std::vector<int> t = args_of(n, "rows_bf16_kernel");
    product_access("rows_bf16_kernel", *static_cast<RowsProd*>(args[0]), ORTH_BF16, t[1], t[2], t[3], t[0], grid);
  } else if (is("rows_f32_kernel")) {   // <tile, at, bt, epi>
    const std::vector<int> t = args_of(n, "rows_f32_kernel");
    product_access("rows_f32_kernel", *static_cast<RowsProd*>(args[0]), ORTH_F32, t[1], t[2], t[3], t[0], grid);
  } else if (is("rows_direct_kernel")) {   // <type, bt, epi, waves, nt>
    const std::vector<int> t = args_of(n, "rows_direct_kernel");
    product_access("rows_direct_kernel", *static_cast<RowsProd*>(args[0]), t[0], false, t[1], t[2], 32, grid);
  } else if (is("rows_outer_kernel")) {   // <type, blocks of a wave>
    const std::vector<int> t = args_of(n, "rows_outer_kernel");
    RowsProd p = *static_cast<RowsProd*>(args[0]);
    need((int64_t)grid.y == p.groups, "rows_outer_kernel: groups");
    need((int64_t)grid.x >= ceil_div(p.N, 128) * ceil_div(p.M, 128 * t[1]) + rows_join_blocks(p.join), "rows_outer_kernel: grid");
    p.a_pad8 = p.b_pad8 = 0;   // (it reads no padding)
    product_access("rows_outer_kernel", p, t[0], true, true, ROWS_STORE, 1 << 20, dim3(p.groups * ceil_div(p.M, 1 << 20) * ceil_div(p.N, 1 << 20) + rows_join_blocks(p.join)));
  } else if (is("rows_join_groups_kernel")) {
    const RowsProd& p = *static_cast<RowsProd*>(args[0]);
    Access a;
    if (p.offsets) a.read(p.offsets, ((int64_t)p.groups + 1) * 4, "offsets");
    a.read(p.slices, rows_parts(p, p.kslice) * p.M * p.N * 4, "slices");
    a.write(p.C, ((p.offsets ? (p.groups - 1) * p.gc : 0) + (int64_t)(p.M - 1) * p.ldc + p.N) * es_of(p.c_dtype), "C");
    need((int64_t)grid.y == p.groups && (int64_t)grid.x * 256 >= (int64_t)p.M * ((p.N + 3) / 4), "rows_join_groups_kernel: grid");
    a.check("rows_join_groups_kernel");
  } else if (is("rows_join_kernel")) {
    const RowsJoin& j = *static_cast<RowsJoin*>(args[0]);
    Access a;
    join_access(j, a);
    need((int64_t)grid.x >= rows_join_blocks(j), "rows_join_kernel: grid");
    a.check("rows_join_kernel");
  } else if (is("pad_rows_kernel")) {   // (x, ld, out, ldo, rows, cols, targets, classes, twice)
    const int64_t es = is("pad_rows_kernelIt") ? 2 : 4;
    const int64_t ld = *static_cast<int64_t*>(args[1]);
    const int ldo = *static_cast<int*>(args[3]), rows = *static_cast<int*>(args[4]), cols = *static_cast<int*>(args[5]);
    const void* targets = *static_cast<void**>(args[6]);
    Access a;
    need(ldo % 8 == 0 && ldo >= cols, "pad_rows_kernel: ldo");
    a.read(*static_cast<void**>(args[0]), ((int64_t)(rows - 1) * ld + cols) * es, "x");
    if (targets) a.read(targets, (int64_t)rows * 8, "targets");
    a.write(*static_cast<void**>(args[2]), ((int64_t)rows << *static_cast<int*>(args[8])) * ldo * es, "out");
    a.check("pad_rows_kernel");
  } else if (is("xent_join_kernel")) {   // (part, n_part, ztarget, targets, rows, classes, loss, lse)
    const int64_t n_part = *static_cast<int*>(args[1]), rows = *static_cast<int*>(args[4]);
    Access a;
    a.read(*static_cast<void**>(args[0]), rows * n_part * 8, "part");
    a.read(*static_cast<void**>(args[2]), rows * 4, "ztarget");
    a.read(*static_cast<void**>(args[3]), rows * 8, "targets");
    a.write(*static_cast<void**>(args[6]), rows * 4, "loss");
    a.write(*static_cast<void**>(args[7]), rows * 4, "lse");
    a.check("xent_join_kernel");
  } else if (is("grad_small_kernel")) {   // (table, index, n, norm, ...)
    Access a;
    a.write(*static_cast<void**>(args[3]), 4, "norm");
    a.check("grad_small_kernel");
  } else if (is("grad_norm_join_kernel")) {   // (partial, n, norm)
    Access a;
    a.read(*static_cast<void**>(args[0]), (int64_t)*static_cast<int*>(args[1]) * 8, "partial");
    a.write(*static_cast<void**>(args[2]), 4, "norm");
    a.check("grad_norm_join_kernel");
  } else if (is("grad_norm_")) {   // (table, n, chunks, partial)
    Access a;
    a.write(*static_cast<void**>(args[3]), (int64_t)grid.x * 8, "partial");
    a.check("grad_norm_kernel");
  } else if (is("grad_clip_")) {   // (table, n, chunks, partial, n_partial, norm, ...)
    Access a;
    const int np = *static_cast<int*>(args[4]);
    a.read(*static_cast<void**>(args[3]), (int64_t)np * 8, "partial");
    if (np)
      a.write(*static_cast<void**>(args[5]), 4, "norm");
    else
      a.read(*static_cast<void**>(args[5]), 4, "norm");
    a.check("grad_clip_kernel");
  } else {
    violation("unknown kernel " + n);
  }
  return hipSuccess;
}
}  // extern "C"

namespace orth {
int report_error(int code, const char* msg) {
  g_what += std::string(" [") + msg + "]";
  return code;
}
void timing_begin(const char*, hipStream_t) {}
void timing_end(const char*, hipStream_t) {}
int upload_table(const void* data, size_t bytes, void* dst, hipStream_t) {
  // (every byte is read: the sanitizer sees a table that is shorter)
  volatile unsigned char sum = 0;
  for (size_t i = 0; i < bytes; ++i) sum = sum + static_cast<const unsigned char*>(data)[i];
  Access a;
  a.write(dst, (int64_t)bytes, "table");
  a.check("upload_table");
  return ORTH_OK;
}
}  // namespace orth

// ---------------------------------------------------------------- driver --
namespace {
std::mt19937_64 rng(20);
int64_t up_to(int64_t n) { return (int64_t)(rng() % (uint64_t)n); }
int size_of(int lo, int hi) {   // spread over the logarithm, some round
  const double v = lo * std::pow((double)hi / lo, (double)rng() / 1.8446744073709552e19);
  const int step = up_to(3) == 0 ? 1 : up_to(2) ? 8 : 64;
  return std::max(lo, (int)v / step * step);
}
uintptr_t g_next;
// a tensor of `bytes` at an address aligned to `align`, apart from all others
void* tensor(int64_t bytes, bool writable, const char* name, int64_t align) {
  const uintptr_t at = (g_next + 4095) / 4096 * 4096 + (uintptr_t)(align < 256 ? align * (1 + up_to(7)) : 0);
  g_next = at + (uintptr_t)bytes + 8192;
  g_regions.push_back({at, at + (uintptr_t)bytes, writable, name});
  return reinterpret_cast<void*>(at);
}
void begin(const char* fmt, ...) {
  char buf[512];
  va_list va;
  va_start(va, fmt);
  vsnprintf(buf, sizeof buf, fmt, va);
  va_end(va);
  g_what = buf;
  g_regions.clear();
  g_next = uintptr_t(1) << 44;
  ++g_calls;
}
int g_short = 0;   // bytes by which workspaces are declared too short (a planted mistake)
void* workspace(size_t bytes) {
  return bytes ? tensor((int64_t)bytes - std::min<int64_t>(g_short, (int64_t)bytes), true, "workspace", 256) : nullptr;
}
void ok(int rc) {
  if (rc != ORTH_OK) violation("refused with " + std::to_string(rc));
}

void linear_call(bool grad) {
  orth_linear_args a{};
  a.dtype = (int)up_to(2);
  a.grad_dtype = (int)up_to(2);
  a.rows = up_to(20) ? size_of(1, 20000) : 0;
  a.groups = up_to(3) ? size_of(1, 200) : 1;
  a.in_features = size_of(1, 3000);
  a.out_features = size_of(1, 3000);
  a.transposed = grad ? 0 : (int)up_to(2);
  const int64_t es = es_of(a.dtype), eg = grad ? es_of(a.grad_dtype) : es;
  const int cx = a.transposed ? a.out_features : a.in_features, cy = a.transposed ? a.in_features : a.out_features;
  a.ld_x = cx + (up_to(2) ? up_to(40) : 0);
  a.ld_y = cy + (up_to(2) ? up_to(40) : 0);
  a.ld_w = a.in_features + (up_to(2) ? up_to(40) : 0);
  a.stride_w = (int64_t)a.out_features * a.ld_w + (up_to(2) ? up_to(100) : 0);
  begin("%s dtype %d grad %d rows %d groups %d in %d out %d transposed %d ld %ld %ld %ld", grad ? "grad_weight" : "apply", a.dtype,
        a.grad_dtype, a.rows, a.groups, a.in_features, a.out_features, a.transposed, (long)a.ld_x, (long)a.ld_w, (long)a.ld_y);
  const int64_t al = up_to(2) ? 256 : es;
  a.x = tensor(((int64_t)(a.rows - 1) * a.ld_x + cx) * es * (a.rows > 0), false, "x", al);
  a.y = tensor(((int64_t)(a.rows - 1) * a.ld_y + cy) * es * (a.rows > 0), !grad, "y", al);
  a.w = tensor(((a.groups - 1) * a.stride_w + (int64_t)(a.out_features - 1) * a.ld_w + a.in_features) * eg, grad, "w", up_to(2) ? 256 : eg);
  a.offsets = a.groups > 1 || up_to(2) ? static_cast<const int32_t*>(tensor(((int64_t)a.groups + 1) * 4, false, "offsets", 4)) : nullptr;
  if (!grad) {
    ok(orth_linear_apply(&a, nullptr));
    return;
  }
  size_t n = 0;
  ok(orth_linear_grad_weight_workspace_size(&a, &n));
  ok(orth_linear_grad_weight(&a, workspace(n), n, nullptr));
}

void xent_call() {
  orth_linear_xent_args a{};
  a.dtype = (int)up_to(2);
  a.rows = up_to(30) ? size_of(1, 9000) : 0;
  a.features = size_of(1, 3000);
  a.classes = size_of(1, 60000);
  a.ld_x = a.features + (up_to(2) ? up_to(40) : 0);
  a.ld_w = a.features + (up_to(2) ? up_to(40) : 0);
  a.scale = 1.5f;
  a.piece = up_to(2) ? 0 : size_of(std::max(1, a.classes / 20), a.classes + 10);
  const int want = 1 + (int)up_to(3);
  begin("xent dtype %d rows %d features %d classes %d ld %ld %ld piece %d want %d", a.dtype, a.rows, a.features, a.classes,
        (long)a.ld_x, (long)a.ld_w, a.piece, want);
  const int64_t es = es_of(a.dtype), al = up_to(2) ? 256 : es;
  a.x = tensor(((int64_t)(a.rows - 1) * a.ld_x + a.features) * es * (a.rows > 0), false, "x", al);
  a.w = tensor(((int64_t)(a.classes - 1) * a.ld_w + a.features) * es, false, "w", up_to(2) ? 256 : es);
  a.targets = static_cast<const int64_t*>(tensor((int64_t)a.rows * 8, false, "targets", 8));
  float* loss = static_cast<float*>(tensor((int64_t)a.rows * 4, true, "loss", 4));
  float* lse = static_cast<float*>(tensor((int64_t)a.rows * 4, true, "lse", 4));
  const std::vector<Region> kept = g_regions;
  size_t n = 0;
  ok(orth_linear_xent_workspace_size(&a, &n));
  ok(orth_linear_xent(&a, loss, lse, workspace(n), n, nullptr));
  // the backward: loss and lse are inputs now, the forward's workspace is gone
  g_regions = kept;
  for (Region& r : g_regions) r.writable = false;
  const int64_t lx = a.features + up_to(20), lw = a.features + up_to(20);
  const float* gl = static_cast<const float*>(tensor((int64_t)a.rows * 4, false, "grad_loss", 4));
  void* gx = want & 1 ? tensor(((int64_t)(a.rows - 1) * lx + a.features) * es * (a.rows > 0), true, "grad_x", up_to(2) ? 256 : es) : nullptr;
  void* gw = want & 2 ? tensor(((int64_t)(a.classes - 1) * lw + a.features) * es, true, "grad_w", up_to(2) ? 256 : es) : nullptr;
  ok(orth_linear_xent_vjp_workspace_size(&a, &n));
  ok(orth_linear_xent_vjp(&a, lse, gl, gx, lx, gw, lw, workspace(n), n, nullptr));
}

void clip_call() {
  const int n = up_to(3) ? size_of(1, 60) : size_of(50, 500);
  begin("clip %d tensors", n);
  std::vector<orth_grad> g;
  for (int i = 0; i < n; ++i) {
    orth_grad d{};
    d.dtype = (int)up_to(2);
    d.rows = up_to(9) ? size_of(1, 300) : 0;
    d.cols = up_to(9) ? size_of(1, up_to(20) ? 300 : 300000) : 0;
    d.ld_grad = d.cols + (up_to(2) ? up_to(9) : 0);
    d.ld_out = up_to(2) ? d.ld_grad : d.cols + up_to(9);
    const int64_t es = es_of(d.dtype), rows = std::max(d.rows, 1);
    d.grad = tensor((rows * d.ld_grad + 1) * es, false, "grad", es);
    d.out = d.ld_out == d.ld_grad && up_to(2) ? const_cast<void*>(d.grad) : tensor((rows * d.ld_out + 1) * es, true, "out", es);
    g.push_back(d);
  }
  float* norm = static_cast<float*>(tensor(4, true, "norm", 4));
  size_t ws = 0;
  ok(orth_grad_norm_workspace_size(g.data(), n, &ws));
  void* w = workspace(ws);
  const orth_clip_opts o{1.f, 1e-6f, (int)up_to(2)};
  ok(orth_grad_norm_batched(g.data(), n, norm, w, ws, nullptr));
  ok(orth_grad_clip_batched(g.data(), n, &o, norm, w, ws, nullptr));
}
}  // namespace

int main(int argc, char** argv) {
  if (argc > 1) g_short = atoi(argv[1]);
  for (int i = 0; i < 4000; ++i) {
    linear_call(false);
    linear_call(true);
    xent_call();
    if (i % 8 == 0) clip_call();
  }
  printf("calls %ld launches %ld\n", g_calls, g_launches);
  int missing = 0;
  for (const char* k : kKernels) {
    printf("%s %ld\n", k, g_seen[k]);
    missing += g_seen[k] == 0;
  }
  return missing ? 4 : 0;
}
