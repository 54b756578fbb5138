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
enum Kernels : int { kDense, kChosen, kChoice, kKernelSets };  // set up apart: a caller of one does not wait for the others
struct DeviceSetup {
  bool done[kKernelSets] = {};
  int num_sms = 0;
};
DeviceSetup g_setup[kMaxDevices];
std::mutex g_setup_mu;

// Once per device and set of kernels, with that device current: kernel limits, SM count.
ipv_status setup_current_device(Kernels set, int* num_sms) {
  int dev = -1;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_reject(e, "cudaGetDevice");
  if (dev < 0 || dev >= kMaxDevices) return reject(IPV_EINVAL, "device ordinal %d not supported", dev);
  std::lock_guard<std::mutex> lock(g_setup_mu);
  DeviceSetup& d = g_setup[dev];
  if (!d.done[set]) {
    const char* what = "no usable kernel image for this device (built for sm_103a)";
    if (set == kDense) {
      if ((e = ipv::attend_rows_prepare()) == cudaSuccess && (e = ipv::attend_tiles_prepare()) != cudaSuccess) what = "tiled attention set-up";
    } else {
      e = set == kChosen ? ipv::attend_chosen_prepare() : ipv::choose_prepare();
    }
    if (e != cudaSuccess) return cuda_reject(e, what);
    if ((e = cudaDeviceGetAttribute(&d.num_sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess)
      return cuda_reject(e, "cudaDeviceGetAttribute");
    d.done[set] = true;
  }
  *num_sms = d.num_sms;
  return IPV_OK;
}

// Checks the pool.
ipv_status check_pages(const ipv_pages* p) {
  if (!p) return reject(IPV_EINVAL, "pages and batch must not be NULL");
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
  return IPV_OK;
}

// The pool as the kernels see it.
void view_pages(const ipv_pages* p, ipv::Pages* out) {
  ipv::Pages& o = *out;
  o.fmt = p->format;
  o.heads = p->n_kv_heads;
  o.dim = p->head_dim;
  o.page_size = p->page_size;
  o.n_pages = static_cast<int>(p->n_pages);
  o.page_stride = p->page_stride;
  o.head_stride = p->head_stride;
  o.row_stride = p->row_stride;
  o.row_bytes = p->format == IPV_PAGES_BF16 ? 2 * p->head_dim : p->format == IPV_PAGES_U8 ? p->head_dim : p->head_dim / 2;
  o.groups = (p->head_dim + ipv::kGroup - 1) / ipv::kGroup;
  o.k = static_cast<char*>(p->k);
  o.v = static_cast<char*>(p->v);
  o.k_par = static_cast<uint32_t*>(p->k_par);
  o.v_par = static_cast<uint32_t*>(p->v_par);
}

// Checks a batch over pages of this shape (page_size, heads, groups) and adds it to the kernels' view.
ipv_status check_batch(const ipv_batch* b, ipv::Pages* out) {
  if (!b) return reject(IPV_EINVAL, "pages and batch must not be NULL");
  const int page_size = out->page_size, heads = out->heads, groups = out->groups;
  if (b->n_seqs < 0 || b->n_seqs > 65535) return reject(IPV_EINVAL, "n_seqs %d is not in 0..65535", b->n_seqs);
  if (b->max_pages < 1) return reject(IPV_EINVAL, "max_pages must be positive");
  const bool pow2 = (page_size & (page_size - 1)) == 0;
  if (b->max_pages > 1 && (!pow2 || page_size < 16))
    return reject(IPV_EINVAL, "page_size %d: several pages per sequence need a power of two of at least 16", page_size);
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
  if (rows * heads * groups > INT32_MAX)
    return reject(IPV_EINVAL, "max_rows * n_kv_heads * groups exceeds 2^31 - 1");
  ipv::Pages& o = *out;
  o.page_shift = 31;
  if (b->max_pages > 1)
    for (o.page_shift = 4; (1 << o.page_shift) < page_size; ++o.page_shift) {
    }
  o.max_pages = b->max_pages;
  o.table = b->table;
  o.table_stride = b->table_stride;
  o.row_start = b->row_start;
  o.kv_len = b->kv_len;
  o.n_seqs = b->n_seqs;
  o.total_rows = b->total_rows;
  o.max_rows = static_cast<int>(rows);
  const int64_t cap = static_cast<int64_t>(b->max_pages) * page_size;
  o.max_kv = static_cast<int>(b->max_kv < cap ? b->max_kv : cap);
  return IPV_OK;
}

// Checks the pool and the batch and fills the kernels' view of them.
ipv_status check(const ipv_pages* p, const ipv_batch* b, ipv::Pages* out) {
  if (!p || !b) return reject(IPV_EINVAL, "pages and batch must not be NULL");
  const ipv_status s = check_pages(p);
  if (s != IPV_OK) return s;
  view_pages(p, out);
  return check_batch(b, out);
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

// chosen: NULL unless the call is for chosen pages.
ipv_status check_attend(const ipv_pages* p, const ipv_batch* b, const ipv_attend_args* t, const ipv_chosen* chosen, ipv::AttendArgs* a) {
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
  if (chosen) {
    if (!t->causal || t->window > 0 || t->sinks > 0) return reject(IPV_EINVAL, "chosen pages need causal = 1, window = 0 and sinks = 0");
    if (chosen->n_chosen < 1) return reject(IPV_EINVAL, "n_chosen must be positive");
    if (chosen->row_stride < 0 || chosen->head_stride < 0) return reject(IPV_EINVAL, "chosen: strides must not be negative");
    if (a->p.max_kv > 1 << 30) return reject(IPV_EINVAL, "chosen pages: max_kv exceeds 2^30");
    const int share = t->n_q_heads / p->n_kv_heads, tile = ipv::attend_rows_tile(share);
    if (static_cast<int64_t>(a->p.max_rows) * ((share + tile - 1) / tile) * a->p.n_seqs > INT32_MAX)
      return reject(IPV_EINVAL, "n_seqs times the query tiles of max_rows exceeds 2^31 - 1");
    a->chosen = chosen->pages;
    a->chosen_row = chosen->row_stride;
    a->chosen_head = chosen->head_stride;
    a->n_chosen = chosen->n_chosen;
  } else if (a->p.fmt != ipv::kBf16 && rows > kRowsMost &&  // widened into the workspace
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

// Chosen pages: blocks take row tiles and heads whole and in turn where that keeps them busy for this many tenths of their
// rounds: nothing to join, and the blocks that run at the same time are near one another in the cache (and in L2). Lists of
// 2048 keys, 8 KV heads, single tokens, in turn against shared out: bf16, 80 tokens (7 tenths) 100 us against 110, 100 tokens 121
// against 133; 8 bits 75 against 78 and 86 against 91; 4 bits 57 against 62 and 66 against 71. With 72 tokens (6 tenths) shares
// take 100, 72 and 57 us, no more than two rounds do.
constexpr int kInTurnTenths = 7;
// With less than a round, 4 or 2 blocks take a tile each as a cluster where they all have room at once, or one where two have
// not: no parts to write, no second kernel. 4 bits: 8 streams 13.0 us against 17.2 shared out, 24 streams 24.8 against 28.4 (two
// blocks each), 32 streams 27.2 against 32.8 (one); bf16: 4 streams 10.6 against 12.4, 12 streams 21.4 against 25.1 (one).

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
  if (a->n_chosen > 0) {
    plan->tiles = false;
    a->tile = ipv::attend_rows_tile(a->share);
    a->unit = kRowsLeast;
    plan->blocks = num_sms * ipv::attend_chosen_resident(p.fmt, p.dim, a->tile);
  } else if (plan->tiles) {
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
  a->per_row = (a->share + a->tile - 1) / a->tile;  // chosen pages only, as by_per_row
  a->by_per_row = ipv::Divide(a->per_row);
  a->tiles = a->n_chosen > 0 ? p.max_rows * a->per_row : static_cast<int>((rows + a->tile - 1) / a->tile);
  a->by_tiles = ipv::Divide(a->tiles);
  // Keys that a row tile can see, at most (its windows, the sinks, their steps' ends).
  int64_t span = p.max_kv;
  if (a->n_chosen > 0) {
    const int64_t pages = (span + p.page_size - 1) / p.page_size;
    if (pages > 1) span = std::min(pages, static_cast<int64_t>(a->n_chosen)) * p.page_size;
  } else if (a->window) {
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
  if (a->n_chosen > 0) {
    const int64_t rounds = (items + plan->blocks - 1) / plan->blocks;
    if (rounds > 1 && items * 10 >= rounds * plan->blocks * kInTurnTenths) {
      a->unit = ipv::kInTurn;
      return;
    }
    int c = 4;
    while (c > 1 && items * c > plan->blocks) c /= 2;
    if (items * c <= plan->blocks && (c == 1 || (span <= kClusterKeys && span * p.row_bytes <= kClusterBytes))) {
      a->unit = 0;
      a->cluster = c;
      plan->blocks = static_cast<int>(items) * c;
      return;
    }
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

namespace {

ipv_status attend_workspace(const ipv_pages* pages, const ipv_batch* batch, const ipv_attend_args* args, const ipv_chosen* chosen,
                            int64_t* bytes_out) {
  if (!bytes_out) return reject(IPV_EINVAL, "bytes_out must not be NULL");
  *bytes_out = 0;
  ipv::AttendArgs a{};
  ipv_status s = check_attend(pages, batch, args, chosen, &a);
  if (s != IPV_OK) return s;
  if (a.p.n_seqs == 0 || a.p.max_rows == 0) return IPV_OK;
  int num_sms = 0;
  if ((s = setup_current_device(chosen ? kChosen : kDense, &num_sms)) != IPV_OK) return s;
  Plan plan;
  make_plan(&a, num_sms, &plan);
  *bytes_out = plan.bytes;
  return IPV_OK;
}

ipv_status attend(const ipv_pages* pages, const ipv_batch* batch, const ipv_attend_args* args, const ipv_chosen* chosen, void* stream) {
  ipv::AttendArgs a{};
  ipv_status s = check_attend(pages, batch, args, chosen, &a);
  if (s != IPV_OK) return s;
  if (a.p.n_seqs == 0 || a.p.max_rows == 0) return IPV_OK;
  s = check_packed(args->q, "q", args->q_row_stride, args->q_head_stride);
  if (s == IPV_OK) s = check_packed(args->out, "out", args->out_row_stride, args->out_head_stride);
  if (s != IPV_OK) return s;
  if (args->q == args->out) return reject(IPV_EINVAL, "q and out share one buffer");
  if (args->lse && !aligned(args->lse, 4)) return reject(IPV_EINVAL, "lse must be 4-byte aligned");
  if (chosen && (!chosen->pages || !aligned(chosen->pages, 4)))
    return reject(IPV_EINVAL, "the chosen pages must not be NULL, and 4-byte aligned");
  int num_sms = 0;
  if ((s = setup_current_device(chosen ? kChosen : kDense, &num_sms)) != IPV_OK) return s;
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
    e = chosen ? ipv::launch_attend_chosen(a, plan.blocks, st) : ipv::launch_attend_rows(a, plan.blocks, st);
  }
  if (e != cudaSuccess) return cuda_reject(e, "attention kernel");
  return IPV_OK;
}

}  // namespace

extern "C" ipv_status ipv_attend_workspace(const ipv_pages* pages, const ipv_batch* batch,
                                           const ipv_attend_args* args, int64_t* bytes_out) {
  return attend_workspace(pages, batch, args, nullptr, bytes_out);
}

extern "C" ipv_status ipv_attend(const ipv_pages* pages, const ipv_batch* batch, const ipv_attend_args* args,
                                 void* stream) {
  return attend(pages, batch, args, nullptr, stream);
}

extern "C" ipv_status ipv_attend_chosen_workspace(const ipv_pages* pages, const ipv_batch* batch, const ipv_attend_args* args,
                                                  const ipv_chosen* chosen, int64_t* bytes_out) {
  if (!chosen) return reject(IPV_EINVAL, "chosen must not be NULL");
  return attend_workspace(pages, batch, args, chosen, bytes_out);
}

extern "C" ipv_status ipv_attend_chosen(const ipv_pages* pages, const ipv_batch* batch, const ipv_attend_args* args,
                                        const ipv_chosen* chosen, void* stream) {
  if (!chosen) return reject(IPV_EINVAL, "chosen must not be NULL");
  return attend(pages, batch, args, chosen, stream);
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

// Rows up to which 4 warps take one: as many blocks of 4 warps as 152 SMs hold of 6 each. 2 warps up to three times as many, then
// one: fewer look-ups per head. 28 + 4 heads with norms, 4, 2 and 1 warps: bf16, 128 channels in halves, 784 rows 7.1, 6.8, 8.4 us (a
// call is the host's 6.7), 1568 rows 8.0, 7.2, 11.1, 2352 rows 11.3, 11.1, 12.0, 3136 rows 16.1, 13.8, 14.0; into 8 bits 7.2, 8.7, 12.8
// at 784 rows, 11.0, 9.5, 14.5 at 1568, 21.0, 16.8, 16.2 at 3136; 64 channels as bf16. It is the rule of these instances: interleaved
// pairs and partial halves of 128 channels have 4 blocks per SM, and would be up to 1.4 times faster with fewer warps between
// 784 and 2352 rows (bits 8, interleaved: 784 rows 9.1, 7.0, 9.6; 1568 rows 13.0, 11.9, 10.4; 3136 rows 25.2, 19.4, 19.9).
constexpr int64_t kRotateWave = 152 * 6;

extern "C" ipv_status ipv_pages_write_rotated(const ipv_pages* pages, const ipv_batch* batch, const ipv_rotary* rotary,
                                              const ipv_rotate_args* t, void* stream) {
  ipv::RotateArgs a{};
  ipv_status s = check(pages, batch, &a.p);
  if (s != IPV_OK) return s;
  if (!rotary || !t) return reject(IPV_EINVAL, "rotary and args must not be NULL");
  if (rotary->rot_dim < 16 || rotary->rot_dim % 16 != 0 || rotary->rot_dim > a.p.dim)
    return reject(IPV_EINVAL, "rot_dim %d is not a multiple of 16 up to head_dim %d", rotary->rot_dim, a.p.dim);
  if (rotary->n_positions < 1 || rotary->n_positions > INT32_MAX) return reject(IPV_EINVAL, "n_positions must be positive and below 2^31");
  if (rotary->interleaved != 0 && rotary->interleaved != 1) return reject(IPV_EINVAL, "interleaved must be 0 or 1");
  if (rotary->n_axes < 1 || rotary->n_axes > 4) return reject(IPV_EINVAL, "n_axes %d is not in 1..4", rotary->n_axes);
  int64_t end = 0;
  for (int i = 0; i < rotary->n_axes; ++i) {
    if (rotary->sections[i] < 8 || rotary->sections[i] % 8 != 0)
      return reject(IPV_EINVAL, "sections must be positive multiples of 8");
    end += rotary->sections[i];
    if (i < 3) a.ends[i] = static_cast<int>(std::min<int64_t>(end, INT32_MAX));
  }
  if (end != rotary->rot_dim / 2) return reject(IPV_EINVAL, "the sections' sum is not rot_dim / 2");
  for (int i = rotary->n_axes - 1; i < 3; ++i) a.ends[i] = INT32_MAX;  // the last axis has no end
  if (t->n_q_heads < 1 || t->n_q_heads > 65535) return reject(IPV_EINVAL, "n_q_heads %d is not in 1..65535", t->n_q_heads);
  if (!std::isfinite(t->eps) || t->eps < 0.0f) return reject(IPV_EINVAL, "eps must be finite and not negative");
  if (!aligned(t->q_weight, 16) || !aligned(t->k_weight, 16)) return reject(IPV_EINVAL, "weights must be 16-byte aligned");
  if (a.p.n_seqs == 0 || a.p.max_rows == 0) return IPV_OK;
  s = check_packed(t->q, "q", t->q_row_stride, t->q_head_stride);
  if (s == IPV_OK) s = check_packed(t->q_out, "q_out", t->out_row_stride, t->out_head_stride);
  if (s == IPV_OK) s = check_packed(t->k_new, "k_new", t->row_stride, t->head_stride);
  if (s == IPV_OK) s = check_packed(t->v_new, "v_new", t->row_stride, t->head_stride);
  if (s != IPV_OK) return s;
  if (t->q == t->q_out && (t->q_row_stride != t->out_row_stride || t->q_head_stride != t->out_head_stride))
    return reject(IPV_EINVAL, "q_out may be q only with q's strides");
  if (!rotary->table || !aligned(rotary->table, 16)) return reject(IPV_EINVAL, "the rotary table must not be NULL, and 16-byte aligned");
  if (!t->positions || !aligned(t->positions, 4)) return reject(IPV_EINVAL, "positions must not be NULL, and 4-byte aligned");
  if (t->positions_stride < 0 || (rotary->n_axes > 1 && t->positions_stride != 0 && t->positions_stride < batch->total_rows))
    return reject(IPV_EINVAL, "positions_stride is neither 0 nor at least total_rows");
  a.q = static_cast<const uint16_t*>(t->q);
  a.q_out = static_cast<uint16_t*>(t->q_out);
  a.k_new = static_cast<const uint16_t*>(t->k_new);
  a.v_new = static_cast<const uint16_t*>(t->v_new);
  a.q_row = t->q_row_stride;
  a.q_head = t->q_head_stride;
  a.out_row = t->out_row_stride;
  a.out_head = t->out_head_stride;
  a.row = t->row_stride;
  a.head = t->head_stride;
  a.q_heads = t->n_q_heads;
  a.turns = rotary->table;
  a.n_positions = rotary->n_positions;
  a.rot = rotary->rot_dim;
  a.neighbours = rotary->interleaved != 0;
  a.positions = t->positions;
  a.positions_stride = t->positions_stride;
  a.q_weight = static_cast<const uint16_t*>(t->q_weight);
  a.k_weight = static_cast<const uint16_t*>(t->k_weight);
  a.eps = t->eps;
  a.by_dim = 1.0f / static_cast<float>(a.p.dim);
  a.row_warps_shift = a.p.total_rows <= kRotateWave ? 2 : a.p.total_rows <= 3 * kRotateWave ? 1 : 0;
  const cudaError_t e = ipv::launch_rotate(a, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? IPV_OK : cuda_reject(e, "rotated write kernel");
}

extern "C" ipv_status ipv_pages_copy(const ipv_pages* pages, const int32_t* from, const int32_t* to, int64_t n, void* stream) {
  const ipv_status s = check_pages(pages);
  if (s != IPV_OK) return s;
  if (n < 0) return reject(IPV_EINVAL, "n must not be negative");
  if (n == 0) return IPV_OK;
  if (!from || !to || !aligned(from, 4) || !aligned(to, 4)) return reject(IPV_EINVAL, "from and to must not be NULL, and 4-byte aligned");
  if (from == to) return reject(IPV_EINVAL, "from and to share one buffer");
  ipv::CopyArgs a{};
  view_pages(pages, &a.p);
  a.from = from;
  a.to = to;
  a.row_chunks = a.p.row_bytes / 16;
  const int64_t chunks = static_cast<int64_t>(a.p.heads) * a.p.page_size * a.row_chunks;
  if (chunks > INT32_MAX - ipv::pages_copy_part()) return reject(IPV_EINVAL, "a page has 2^31 16-byte pieces or more");
  a.chunks = static_cast<int>(chunks);
  a.parts = static_cast<int>((chunks + ipv::pages_copy_part() - 1) / ipv::pages_copy_part());
  if (n > INT32_MAX / a.parts) return reject(IPV_EINVAL, "n times a page's parts exceeds 2^31 - 1");
  a.by_row = ipv::Divide(a.row_chunks);
  a.by_page = ipv::Divide(a.p.page_size);
  a.by_parts = ipv::Divide(a.parts);
  const cudaError_t e = ipv::launch_pages_copy(a, n, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? IPV_OK : cuda_reject(e, "page copy kernel");
}

extern "C" ipv_status ipv_pages_gather(const ipv_pages* source_pages, const ipv_batch* source, const ipv_pages* pages,
                                       const ipv_batch* batch, const int32_t* kept, int64_t kept_seq_stride,
                                       int64_t kept_head_stride, void* stream) {
  ipv::MoveArgs a{};
  ipv_status s = check(source_pages, source, &a.src);
  if (s == IPV_OK) s = check(pages, batch, &a.p);
  if (s != IPV_OK) return s;
  if (a.src.fmt != a.p.fmt || a.src.heads != a.p.heads || a.src.dim != a.p.dim)
    return reject(IPV_EINVAL, "the two caches must have one format, n_kv_heads and head_dim");
  if (a.src.n_seqs != a.p.n_seqs) return reject(IPV_EINVAL, "the two batches must have the same sequences");
  if (kept && !aligned(kept, 4)) return reject(IPV_EINVAL, "kept must be 4-byte aligned");
  if (kept_seq_stride < 0 || kept_head_stride < 0) return reject(IPV_EINVAL, "kept: strides must not be negative");
  if (a.p.n_seqs == 0 || a.p.max_rows == 0) return IPV_OK;
  a.kept = kept;
  a.kept_seq = kept_seq_stride;
  a.kept_head = kept_head_stride;
  a.row_chunks = a.p.row_bytes / 16;
  const cudaError_t e = ipv::launch_pages_gather(a, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? IPV_OK : cuda_reject(e, "row gather kernel");
}

namespace {

ipv_status check_bounds(const ipv_bounds* b) {
  if (!b) return reject(IPV_EINVAL, "bounds must not be NULL");
  if (b->n_kv_heads < 1 || b->n_kv_heads > 65535) return reject(IPV_EINVAL, "n_kv_heads %d is not in 1..65535", b->n_kv_heads);
  if (b->head_dim < 8 || b->head_dim > 128 || b->head_dim % 8 != 0)
    return reject(IPV_EINVAL, "head_dim %d is not a multiple of 8 up to 128", b->head_dim);
  if (b->page_size < 1 || b->n_pages < 1 || b->n_pages > INT32_MAX)
    return reject(IPV_EINVAL, "page_size and n_pages must be positive and below 2^31");
  if (!b->codes || !b->steps || !aligned(b->codes, 16) || !aligned(b->steps, 4))
    return reject(IPV_EINVAL, "codes (16-byte aligned) and steps (4-byte aligned) must not be NULL");
  return IPV_OK;
}

int padded(int dim) { return dim <= 64 ? 64 : 128; }

constexpr int64_t kChoosePages = 32768;
constexpr int kChooseShare = 64;

}  // namespace

extern "C" ipv_status ipv_bounds_update(const ipv_bounds* bounds, const ipv_pages* pages, const ipv_batch* batch, void* stream) {
  ipv::BoundsArgs a{};
  ipv_status s = check_bounds(bounds);
  if (s == IPV_OK) s = check(pages, batch, &a.p);
  if (s != IPV_OK) return s;
  if (bounds->n_kv_heads != a.p.heads || bounds->head_dim != a.p.dim || bounds->page_size != a.p.page_size || bounds->n_pages != a.p.n_pages)
    return reject(IPV_EINVAL, "the bounds are of pages of another shape");
  if (a.p.n_seqs == 0 || a.p.max_rows == 0 || a.p.max_kv == 0) return IPV_OK;
  a.codes = static_cast<char*>(bounds->codes);
  a.steps = bounds->steps;
  a.padded = padded(a.p.dim);
  const int64_t held = (static_cast<int64_t>(a.p.max_kv) + a.p.page_size - 1) / a.p.page_size;
  const int64_t touched = (static_cast<int64_t>(a.p.max_rows) + a.p.page_size - 2) / a.p.page_size + 1;
  const cudaError_t e = ipv::launch_bounds(a, static_cast<int>(std::min(held, touched)), static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? IPV_OK : cuda_reject(e, "page bounds kernel");
}

extern "C" ipv_status ipv_bounds_choose(const ipv_bounds* bounds, const ipv_batch* batch, const ipv_choose_args* t, void* stream) {
  ipv_status s = check_bounds(bounds);
  if (s != IPV_OK) return s;
  ipv::ChooseArgs a{};
  a.p.heads = bounds->n_kv_heads;
  a.p.dim = bounds->head_dim;
  a.p.page_size = bounds->page_size;
  a.p.n_pages = static_cast<int>(bounds->n_pages);
  a.p.groups = 1;
  s = check_batch(batch, &a.p);
  if (s != IPV_OK) return s;
  if (!t) return reject(IPV_EINVAL, "args must not be NULL");
  if (t->n_q_heads < 1 || t->n_q_heads % a.p.heads != 0)
    return reject(IPV_EINVAL, "n_q_heads %d is not a multiple of n_kv_heads %d", t->n_q_heads, a.p.heads);
  a.share = t->n_q_heads / a.p.heads;
  if (a.share > kChooseShare) return reject(IPV_EINVAL, "%d query heads per KV head: the most is %d", a.share, kChooseShare);
  if (t->first < 0 || t->recent < 1 || t->n_chosen < 1 || static_cast<int64_t>(t->first) + t->recent > t->n_chosen)
    return reject(IPV_EINVAL, "n_chosen must be at least first + recent, first at least 0, recent at least 1");
  if (t->out_row_stride < 0 || t->out_head_stride < 0) return reject(IPV_EINVAL, "out: strides must not be negative");
  const int64_t pages = (static_cast<int64_t>(a.p.max_kv) + a.p.page_size - 1) / a.p.page_size;
  if (pages > kChoosePages) return reject(IPV_EINVAL, "max_kv spans %lld pages, the most is %lld", static_cast<long long>(pages),
                                          static_cast<long long>(kChoosePages));
  if (a.p.n_seqs == 0 || a.p.max_rows == 0) return IPV_OK;
  s = check_packed(t->q, "q", t->q_row_stride, t->q_head_stride);
  if (s != IPV_OK) return s;
  if (!t->out || !aligned(t->out, 4)) return reject(IPV_EINVAL, "out must not be NULL, and 4-byte aligned");
  int num_sms = 0;
  if ((s = setup_current_device(kChoice, &num_sms)) != IPV_OK) return s;
  a.codes = static_cast<const char*>(bounds->codes);
  a.steps = bounds->steps;
  a.padded = padded(a.p.dim);
  a.q = static_cast<const uint16_t*>(t->q);
  a.q_row = t->q_row_stride;
  a.q_head = t->q_head_stride;
  a.head_tiles = (a.share + 7) / 8;
  a.out = t->out;
  a.out_row = t->out_row_stride;
  a.out_head = t->out_head_stride;
  a.n = t->n_chosen;
  a.first = t->first;
  a.recent = t->recent;
  a.max_pages = static_cast<int>(pages);
  // Blocks for one list, as long as each warp keeps 16 pages: up to 4 where two blocks per SM have room for all, 8 where one has
  // (769 pages, 8 KV heads: 16 streams 9.8 us with 2 blocks each against 12.7 with 1; 4 streams 7.8 with 4 against 8.5 with 8).
  const int64_t lists = static_cast<int64_t>(a.p.max_rows) * a.p.n_seqs * a.p.heads;
  a.cluster = 1;
  while (a.cluster < 8 && pages > 16 * (ipv::kChooseThreads / 32) * a.cluster && lists * a.cluster * 2 <= num_sms * (a.cluster < 4 ? 2 : 1))
    a.cluster *= 2;
  if (static_cast<int64_t>(a.p.max_rows) * a.cluster > INT32_MAX) return reject(IPV_EINVAL, "max_rows times a cluster's blocks exceeds 2^31 - 1");
  const cudaError_t e = ipv::launch_choose(a, static_cast<int>(pages), static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? IPV_OK : cuda_reject(e, "page choice kernel");
}
