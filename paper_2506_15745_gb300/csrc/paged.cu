// C ABI of the paged cache (declared in include/ipv.h): argument checks, the
// choice of kernel and of key splits, launches.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <mutex>

#include "ipv.h"
#include "paged.cuh"

namespace ipv {
void record_error(ipv_status s, const char* msg);
}

namespace {

static_assert(static_cast<int>(ipv::kBf16) == IPV_PAGES_BF16 && static_cast<int>(ipv::kU8) == IPV_PAGES_U8 &&
                  static_cast<int>(ipv::kU4) == IPV_PAGES_U4,
              "page formats");

ipv_status reject(ipv_status s, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  std::vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  ipv::record_error(s, buf);
  return s;
}

ipv_status cuda_reject(cudaError_t e, const char* what) {
  return reject(IPV_ECUDA, "%s: %s (%s)", what, cudaGetErrorName(e), cudaGetErrorString(e));
}

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

constexpr int kMaxDevices = 64;
struct DeviceSetup {
  bool done = false;
  int num_sms = 0;
};
DeviceSetup g_setup[kMaxDevices];
std::mutex g_setup_mu;

// Once per device, with that device current: kernel limits, SM count.
ipv_status setup_current_device(int* num_sms) {
  int dev = -1;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_reject(e, "cudaGetDevice");
  if (dev < 0 || dev >= kMaxDevices) return reject(IPV_EINVAL, "device ordinal %d not supported", dev);
  std::lock_guard<std::mutex> lock(g_setup_mu);
  DeviceSetup& d = g_setup[dev];
  if (!d.done) {
    if ((e = ipv::attend_rows_prepare()) != cudaSuccess)
      return cuda_reject(e, "no usable kernel image for this device (built for sm_103a)");
    if ((e = ipv::attend_tiles_prepare()) != cudaSuccess) return cuda_reject(e, "tiled attention set-up");
    if ((e = cudaDeviceGetAttribute(&d.num_sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess)
      return cuda_reject(e, "cudaDeviceGetAttribute");
    d.done = true;
  }
  *num_sms = d.num_sms;
  return IPV_OK;
}

// Checks the pool and the batch and fills the kernels' view of them.
ipv_status check(const ipv_pages* p, const ipv_batch* b, ipv::Pages* out) {
  if (!p || !b) return reject(IPV_EINVAL, "pages and batch must not be NULL");
  const int fmt = p->format;
  if (fmt != IPV_PAGES_BF16 && fmt != IPV_PAGES_U8 && fmt != IPV_PAGES_U4)
    return reject(IPV_EINVAL, "unknown page format %d", fmt);
  if (p->n_kv_heads < 1 || p->n_kv_heads > 65535) return reject(IPV_EINVAL, "n_kv_heads %d is not in 1..65535", p->n_kv_heads);
  if (p->head_dim < 1 || p->head_dim > 128) return reject(IPV_EINVAL, "head_dim %d is not in 1..128", p->head_dim);
  if (fmt == IPV_PAGES_BF16 ? p->head_dim % 8 != 0 : p->head_dim % ipv::kGroup != 0)
    return reject(IPV_EINVAL, "head_dim %d: bf16 pages need a multiple of 8, codes 64 or 128", p->head_dim);
  if (p->page_size < 1 || p->n_pages < 1 || p->n_pages > INT32_MAX)
    return reject(IPV_EINVAL, "page_size %d and n_pages %lld must be positive and below 2^31", p->page_size,
                  static_cast<long long>(p->n_pages));
  if (p->page_stride < (p->n_pages > 1) || p->head_stride < (p->n_kv_heads > 1) || p->row_stride < 1)
    return reject(IPV_EINVAL, "strides must be positive");
  for (const int64_t stride : {p->page_stride, p->head_stride, p->row_stride})
    if (stride >= (int64_t{1} << 40) / 256)  // a row has at most 256 bytes
      return reject(IPV_EINVAL, "a stride of %lld rows exceeds 2^32", static_cast<long long>(stride));
  const double last = static_cast<double>(p->n_pages - 1) * static_cast<double>(p->page_stride) +
                      static_cast<double>(p->n_kv_heads - 1) * static_cast<double>(p->head_stride) +
                      static_cast<double>(p->page_size - 1) * static_cast<double>(p->row_stride);
  if (last >= 9007199254740992.0) return reject(IPV_EINVAL, "row numbers exceed 2^53");
  if (!p->k || !p->v) return reject(IPV_EINVAL, "k and v pages must not be NULL");
  if (!aligned(p->k, 16) || !aligned(p->v, 16)) return reject(IPV_EINVAL, "pages must be 16-byte aligned");
  if (p->k == p->v) return reject(IPV_EINVAL, "k and v pages share one buffer");
  const int groups = (p->head_dim + ipv::kGroup - 1) / ipv::kGroup;
  if (fmt != IPV_PAGES_BF16) {
    if (!p->k_par || !p->v_par) return reject(IPV_EINVAL, "pages of codes need k_par and v_par");
    if (!aligned(p->k_par, 4 * groups) || !aligned(p->v_par, 4 * groups))
      return reject(IPV_EINVAL, "k_par and v_par must be %d-byte aligned", 4 * groups);
    if (p->k_par == p->v_par) return reject(IPV_EINVAL, "k_par and v_par share one buffer");
  }
  if (b->n_seqs < 0 || b->n_seqs > 65535) return reject(IPV_EINVAL, "n_seqs %d is not in 0..65535", b->n_seqs);
  if (b->max_pages < 1) return reject(IPV_EINVAL, "max_pages must be positive");
  const bool pow2 = (p->page_size & (p->page_size - 1)) == 0;
  if (b->max_pages > 1 && (!pow2 || p->page_size < 16))
    return reject(IPV_EINVAL, "page_size %d: several pages per sequence need a power of two of at least 16", p->page_size);
  if (!b->table && b->max_pages != 1) return reject(IPV_EINVAL, "without a table max_pages must be 1");
  if (b->table && (!aligned(b->table, 4) || (b->table_stride != 0 && b->table_stride < b->max_pages)))
    return reject(IPV_EINVAL, "table must be 4-byte aligned with table_stride 0 or >= max_pages");
  if (b->total_rows < 0 || b->total_rows > INT32_MAX || b->max_rows < 0 || b->max_kv < 0)
    return reject(IPV_EINVAL, "total_rows, max_rows and max_kv must not be negative, total_rows below 2^31");
  if (b->n_seqs > 0) {
    if (!b->row_start || !b->kv_len) return reject(IPV_EINVAL, "row_start and kv_len must not be NULL");
    if (!aligned(b->row_start, 4) || !aligned(b->kv_len, 4))
      return reject(IPV_EINVAL, "row_start and kv_len must be 4-byte aligned");
  }
  const int64_t rows = b->max_rows < b->total_rows ? b->max_rows : b->total_rows;
  if (rows * p->n_kv_heads * groups > INT32_MAX)
    return reject(IPV_EINVAL, "max_rows * n_kv_heads * groups exceeds 2^31 - 1");
  ipv::Pages& o = *out;
  o.fmt = fmt;
  o.heads = p->n_kv_heads;
  o.dim = p->head_dim;
  o.page_size = p->page_size;
  o.page_shift = 31;
  if (b->max_pages > 1)
    for (o.page_shift = 4; (1 << o.page_shift) < p->page_size; ++o.page_shift) {
    }
  o.n_pages = static_cast<int>(p->n_pages);
  o.max_pages = b->max_pages;
  o.page_stride = p->page_stride;
  o.head_stride = p->head_stride;
  o.row_stride = p->row_stride;
  o.row_bytes = fmt == IPV_PAGES_BF16 ? 2 * p->head_dim : fmt == IPV_PAGES_U8 ? p->head_dim : p->head_dim / 2;
  o.groups = groups;
  o.k = static_cast<char*>(p->k);
  o.v = static_cast<char*>(p->v);
  o.k_par = static_cast<uint32_t*>(p->k_par);
  o.v_par = static_cast<uint32_t*>(p->v_par);
  o.table = b->table;
  o.table_stride = b->table_stride;
  o.row_start = b->row_start;
  o.kv_len = b->kv_len;
  o.n_seqs = b->n_seqs;
  o.total_rows = b->total_rows;
  o.max_rows = static_cast<int>(rows);
  const int64_t cap = static_cast<int64_t>(b->max_pages) * p->page_size;
  o.max_kv = static_cast<int>(b->max_kv < cap ? b->max_kv : cap);
  return IPV_OK;
}

ipv_status check_packed(const void* x, const char* name, int64_t row, int64_t head) {
  if (!x) return reject(IPV_EINVAL, "%s must not be NULL", name);
  if (!aligned(x, 16)) return reject(IPV_EINVAL, "%s must be 16-byte aligned", name);
  if (row < 0 || head < 0 || row % 8 != 0 || head % 8 != 0)
    return reject(IPV_EINVAL, "%s: strides must be multiples of 8 elements, not negative", name);
  return IPV_OK;
}

// The rows kernel reads K and V once per 16 query rows, the tiled kernel once per
// 256, after widening codes and with a longer way in and out. Up to 64 rows (per
// sequence and KV head) the rows kernel is the faster one for codes (7 query heads,
// 4 KV heads, 6000 rows, 16 sequences of 4 tokens, u4: 51 against 109 us; of 9 tokens
// 84 against 110), and for bf16 where it reads little, in millions of bytes (1 sequence of
// 8 tokens over 9000 rows, 73.7: 19 against 26 us; 16 of 9 tokens over 600, 78.6: 25 against
// 19; 16 of 3 tokens over 6000, 393: 65 against 48).
constexpr int64_t kRowsMost = 64, kRowsBytes = 76000000;

constexpr float kLog2e = 1.4426950408889634f;

ipv_status check_attend(const ipv_pages* p, const ipv_batch* b, const ipv_attend_args* t, ipv::AttendArgs* a) {
  ipv_status s = check(p, b, &a->p);
  if (s != IPV_OK) return s;
  if (!t) return reject(IPV_EINVAL, "args must not be NULL");
  if (t->n_q_heads < 1 || t->n_q_heads % p->n_kv_heads != 0)
    return reject(IPV_EINVAL, "n_q_heads %d is not a multiple of n_kv_heads %d", t->n_q_heads, p->n_kv_heads);
  if (!std::isfinite(t->scale * kLog2e)) return reject(IPV_EINVAL, "scale must be finite and below 2^127");
  if (t->causal != 0 && t->causal != 1) return reject(IPV_EINVAL, "causal must be 0 or 1");
  if (t->window < 0 || t->sinks < 0) return reject(IPV_EINVAL, "window and sinks must not be negative");
  if (t->window > 0 && !t->causal) return reject(IPV_EINVAL, "a window needs causal = 1");
  if (static_cast<int64_t>(a->p.max_rows) * t->n_q_heads > INT32_MAX)
    return reject(IPV_EINVAL, "max_rows * n_q_heads exceeds 2^31 - 1");
  const int64_t rows = static_cast<int64_t>(a->p.max_rows) * (t->n_q_heads / p->n_kv_heads);
  if ((rows + 15) / 16 * a->p.n_seqs > INT32_MAX) return reject(IPV_EINVAL, "n_seqs times the query tiles of max_rows exceeds 2^31 - 1");
  if (a->p.fmt != ipv::kBf16 && rows > kRowsMost &&  // widened into the workspace
      4.0 * a->p.n_seqs * a->p.heads * a->p.max_kv * a->p.dim >= 1152921504606846976.0)
    return reject(IPV_EINVAL, "n_seqs * n_kv_heads * max_kv * head_dim: the workspace would exceed 2^60 bytes");
  a->q_heads = t->n_q_heads;
  a->share = t->n_q_heads / p->n_kv_heads;
  a->by_share = ipv::Divide(a->share);
  a->scale_log2 = t->scale * kLog2e;
  a->causal = t->causal;
  a->window = t->window;
  a->sinks = t->window ? t->sinks : 0;
  return IPV_OK;
}

// Longest that a wait inside the tiled kernel may take (ipv_attend_wait_limit).
constexpr int64_t kDefaultLimitNs = 4000000000;
std::atomic<int64_t> g_limit_ns{kDefaultLimitNs};

// Least share of a block, in steps and what a run costs beside them: below,
// joining parts costs more than the other blocks save.
constexpr int kTilesLeast = 3, kRowsLeast = 14;
// Keys up to which a block takes a row tile whole, and there is nothing to join:
// the join and its launch take about as long as a block takes for these.
constexpr int kWhole = 512;
// Where few row tiles are better off with 8 blocks each that join their parts
// through the cluster's shared memory (one kernel on some SMs) than with all SMs
// and a second kernel: up to this many keys and bytes of K, on at most two thirds of
// the device (all of it has no place for so many clusters at once). One token, 4 KV
// heads, bf16: 600 keys 7.4 against 11.3 us, 3000 8.5 against 11.4, 6272 11.5 against 11.6,
// 12000 16 against 13; 4 bits: 1500 keys 8.5 against 14.8, 6272 13.0 against 15.1.
constexpr int64_t kClusterKeys = 8192, kClusterBytes = 1 << 20;

// Which kernel takes the call, on how many blocks, and the workspace.
struct Plan {
  bool tiles = false;
  int blocks = 0;
  ipv::TileMaps maps;  // tiled kernel: made only when launching
  int64_t k16 = 0, v16 = 0, part_o = 0, part_ml = 0, part_rec = 0, bytes = 0;  // offsets in the workspace
};

int64_t round256(int64_t x) { return (x + 255) & ~int64_t{255}; }

// a: checked arguments; the plan's tile and unit go into it.
void make_plan(ipv::AttendArgs* a, int num_sms, Plan* plan) {
  const ipv::Pages& p = a->p;
  const int64_t rows = static_cast<int64_t>(p.max_rows) * a->share;
  const int64_t keys = std::min<int64_t>(p.max_kv, a->window ? int64_t{a->window} + a->sinks + 64 : p.max_kv);
  const double read = static_cast<double>((rows + 15) / 16 * p.n_seqs) * static_cast<double>(keys) * p.heads * 2 * p.row_bytes;  // bytes
  const bool waves = p.max_kv <= kWhole && (rows + 15) / 16 * p.n_seqs * p.heads > num_sms;  // of blocks that take tiles whole
  plan->tiles = rows > kRowsMost || (rows > 16 && p.fmt == ipv::kBf16 && (read > kRowsBytes || waves));
  plan->bytes = 0;
  if (plan->tiles) {
    a->tile = ipv::kTilesRows;
    a->unit = kTilesLeast;
    plan->blocks = num_sms;
    if (p.fmt != ipv::kBf16) {
      const int64_t one = round256(static_cast<int64_t>(p.n_seqs) * p.heads * p.max_kv * p.dim * 2);
      plan->k16 = 0;
      plan->v16 = one;
      plan->bytes = 2 * one;
    }
  } else {
    a->tile = ipv::attend_rows_tile(static_cast<int>(rows));
    a->unit = kRowsLeast;
    plan->blocks = num_sms * ipv::attend_rows_resident(p.fmt, p.dim, a->tile);
  }
  a->tiles = static_cast<int>((rows + a->tile - 1) / a->tile);
  a->by_tiles = ipv::Divide(a->tiles);
  // Keys that a row tile can see, at most (its windows, the sinks, their steps' ends).
  int64_t span = p.max_kv;
  if (a->window) {
    const int64_t seen = static_cast<int64_t>(a->window) + a->tile + a->sinks + 2 * (plan->tiles ? ipv::kTilesStep : ipv::kRowsStep);
    if (seen < span) span = seen;
  }
  const int64_t items = static_cast<int64_t>(a->tiles) * p.n_seqs * p.heads;
  a->cluster = 1;
  if (span <= kWhole && items <= INT32_MAX) {
    a->unit = 0;
    plan->blocks = static_cast<int>(items);
    return;
  }
  if (!plan->tiles && span <= kClusterKeys && span * p.row_bytes <= kClusterBytes &&
      items * ipv::kRowsCluster * 3 <= static_cast<int64_t>(plan->blocks) * 2) {
    a->unit = 0;
    a->cluster = ipv::kRowsCluster;
    plan->blocks = static_cast<int>(items) * ipv::kRowsCluster;
    return;
  }
  const int64_t parts = static_cast<int64_t>(plan->blocks) * 2 * a->tile;
  plan->part_o = plan->bytes;
  plan->part_ml = plan->part_o + round256(parts * p.dim * 4);
  plan->part_rec = plan->part_ml + round256(parts * 8);
  plan->bytes = plan->part_rec + round256(static_cast<int64_t>(plan->blocks) * 2 * 16);
}

// The fp16 rows that codes are widened into, as a pool of one page per sequence.
ipv::Pages widened(const ipv::Pages& p, char* k, char* v) {
  ipv::Pages w = p;
  w.fmt = ipv::kBf16;
  w.page_size = p.max_kv > 0 ? p.max_kv : 1;
  w.page_shift = 31;
  w.n_pages = p.n_seqs;
  w.max_pages = 1;
  w.row_stride = 1;
  w.head_stride = w.page_size;
  w.page_stride = static_cast<int64_t>(w.page_size) * p.heads;
  w.row_bytes = 2 * p.dim;
  w.k = k;
  w.v = v;
  w.table = nullptr;
  return w;
}

}  // namespace

extern "C" ipv_status ipv_pages_write(const ipv_pages* pages, const ipv_batch* batch, const void* k_new,
                                      const void* v_new, int64_t row_stride, int64_t head_stride, void* stream) {
  ipv::RowsArgs a{};
  ipv_status s = check(pages, batch, &a.p);
  if (s != IPV_OK) return s;
  if (a.p.n_seqs == 0 || a.p.max_rows == 0) return IPV_OK;
  s = check_packed(k_new, "k_new", row_stride, head_stride);
  if (s == IPV_OK) s = check_packed(v_new, "v_new", row_stride, head_stride);
  if (s != IPV_OK) return s;
  a.k_new = static_cast<const uint16_t*>(k_new);
  a.v_new = static_cast<const uint16_t*>(v_new);
  a.row = row_stride;
  a.head = head_stride;
  a.by_heads = ipv::Divide(a.p.heads);
  const cudaError_t e = ipv::launch_pages_write(a, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? IPV_OK : cuda_reject(e, "page write kernel");
}

extern "C" ipv_status ipv_pages_read(const ipv_pages* pages, const ipv_batch* batch, void* k_out, void* v_out,
                                     int64_t row_stride, int64_t head_stride, void* stream) {
  ipv::RowsArgs a{};
  ipv_status s = check(pages, batch, &a.p);
  if (s != IPV_OK) return s;
  if (a.p.n_seqs == 0 || a.p.max_rows == 0) return IPV_OK;
  s = check_packed(k_out, "k_out", row_stride, head_stride);
  if (s == IPV_OK) s = check_packed(v_out, "v_out", row_stride, head_stride);
  if (s != IPV_OK) return s;
  if (k_out == v_out) return reject(IPV_EINVAL, "k_out and v_out share one buffer");
  a.k_out = static_cast<uint16_t*>(k_out);
  a.v_out = static_cast<uint16_t*>(v_out);
  a.row = row_stride;
  a.head = head_stride;
  a.by_heads = ipv::Divide(a.p.heads);
  const cudaError_t e = ipv::launch_pages_read(a, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? IPV_OK : cuda_reject(e, "page read kernel");
}

extern "C" ipv_status ipv_attend_workspace(const ipv_pages* pages, const ipv_batch* batch,
                                           const ipv_attend_args* args, int64_t* bytes_out) {
  if (!bytes_out) return reject(IPV_EINVAL, "bytes_out must not be NULL");
  *bytes_out = 0;
  ipv::AttendArgs a{};
  ipv_status s = check_attend(pages, batch, args, &a);
  if (s != IPV_OK) return s;
  if (a.p.n_seqs == 0 || a.p.max_rows == 0) return IPV_OK;
  int num_sms = 0;
  if ((s = setup_current_device(&num_sms)) != IPV_OK) return s;
  Plan plan;
  make_plan(&a, num_sms, &plan);
  *bytes_out = plan.bytes;
  return IPV_OK;
}

extern "C" ipv_status ipv_attend(const ipv_pages* pages, const ipv_batch* batch, const ipv_attend_args* args,
                                 void* stream) {
  ipv::AttendArgs a{};
  ipv_status s = check_attend(pages, batch, args, &a);
  if (s != IPV_OK) return s;
  if (a.p.n_seqs == 0 || a.p.max_rows == 0) return IPV_OK;
  s = check_packed(args->q, "q", args->q_row_stride, args->q_head_stride);
  if (s == IPV_OK) s = check_packed(args->out, "out", args->out_row_stride, args->out_head_stride);
  if (s != IPV_OK) return s;
  if (args->q == args->out) return reject(IPV_EINVAL, "q and out share one buffer");
  if (args->lse && !aligned(args->lse, 4)) return reject(IPV_EINVAL, "lse must be 4-byte aligned");
  int num_sms = 0;
  if ((s = setup_current_device(&num_sms)) != IPV_OK) return s;
  Plan plan;
  make_plan(&a, num_sms, &plan);
  if (plan.bytes > 0) {
    if (!args->workspace || args->workspace_bytes < plan.bytes)
      return reject(IPV_EINVAL, "the workspace has %lld bytes, the call needs %lld",
                    static_cast<long long>(args->workspace ? args->workspace_bytes : 0),
                    static_cast<long long>(plan.bytes));
    if (!aligned(args->workspace, 256)) return reject(IPV_EINVAL, "the workspace must be 256-byte aligned");
  }
  a.q = static_cast<const uint16_t*>(args->q);
  a.out = static_cast<uint16_t*>(args->out);
  a.lse = args->lse;
  a.q_row = args->q_row_stride;
  a.q_head = args->q_head_stride;
  a.out_row = args->out_row_stride;
  a.out_head = args->out_head_stride;
  char* ws = static_cast<char*>(args->workspace);
  a.part_o = reinterpret_cast<float*>(ws + plan.part_o);
  a.part_ml = reinterpret_cast<float2*>(ws + plan.part_ml);
  a.part_rec = reinterpret_cast<int4*>(ws + plan.part_rec);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (plan.tiles) {
    const bool bf16 = a.p.fmt == ipv::kBf16;
    if (!bf16) {
      ipv::ExpandArgs x{};
      x.p = a.p;
      x.k_out = reinterpret_cast<uint16_t*>(ws + plan.k16);
      x.v_out = reinterpret_cast<uint16_t*>(ws + plan.v16);
      x.causal = a.causal;
      x.window = a.window;
      x.sinks = a.sinks;
      x.step = ipv::kTilesStep;
      if (a.p.max_kv > 0 && (e = ipv::launch_pages_expand(x, st)) != cudaSuccess) return cuda_reject(e, "code widening kernel");
      a.p = widened(a.p, ws + plan.k16, ws + plan.v16);
    }
    if (!ipv::attend_tiles_maps(a, bf16, &plan.maps)) return reject(IPV_ECUDA, "cuTensorMapEncodeTiled refused the pool");
    e = ipv::launch_attend_tiles(a, bf16, plan.maps, plan.blocks, g_limit_ns.load(), st);
  } else {
    e = ipv::launch_attend_rows(a, plan.blocks, st);
  }
  if (e != cudaSuccess) return cuda_reject(e, "attention kernel");
  return IPV_OK;
}

extern "C" ipv_status ipv_attend_error(uint32_t* err_out) {
  if (!err_out) return reject(IPV_EINVAL, "err_out must not be NULL");
  unsigned bits = 0;
  const cudaError_t e = ipv::attend_tiles_error(&bits);
  if (e != cudaSuccess) return cuda_reject(e, "reading the attention error word");
  *err_out = bits;
  return IPV_OK;
}

extern "C" ipv_status ipv_attend_wait_limit(int64_t nanoseconds) {
  if (nanoseconds < 0) return reject(IPV_EINVAL, "the limit must not be negative");
  g_limit_ns.store(nanoseconds == 0 ? kDefaultLimitNs : nanoseconds - 1);  // 1: no wait at all
  return IPV_OK;
}
