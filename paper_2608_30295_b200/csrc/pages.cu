// Pages of a cache: handing them out, sequences that continue from another one's rows, rows taken back, pages moved together.
//
// Host bookkeeping over the mirrors, and one kernel that carries its orders in its arguments (no copy from host memory that a caller would
// have to keep, nothing to wait for): 64 rows of K and V copied to a page, entries of the page table and segment descriptions set.
// Bound by the copied rows (1 KB a row, K and V, read and written) where there are many, by the launch where there are few
// (64 lists, 40 rows each copied: 5 us with cold caches; 466 pages moved, 30 MB: 7 us).  The kernels do
// not signal their dependents early: they write rows and table entries that a decode plan may know.
//
// Rows are shared, not copied, where that is possible.  A list that continues from another one (fork) reads the parent's rows in place up to the
// last multiple of 128 (its capacity is set to that) and the parent's full pages through its own table; only what follows is copied.  Of the
// lists that share a segment's rows at most one may append there (it has seg_len < seg_cap); the others' capacities are full.  A
// page that several lists read is full for all of them.  catekv_truncate keeps both true by copying what a list would otherwise go on
// writing to while another reads it.
#include <stdlib.h>
#include <string.h>

#include <algorithm>

#include "decode.cuh"

namespace catekv {

struct PageOp {  // kind | count << 3, and what the kind says
  int32_t kind, a, b, c;
};
enum PageOpKind {
  kOpSegment = 0,   // segment `count`: off = a, cap = b, len = c (c < 0: as it is)
  kOpTable = 1,     // `count` (1 or 2) table entries from index a on: b, c
  kOpCopyPool = 2,  // `count` rows from pool row a to overflow row b; table entry c names the page of b
  kOpCopyPage = 3,  // `count` rows from overflow row a to overflow row b; table entry c names the page of b
  kOpTableCopy = 4, // `count` table entries from index a on are those from index b on
  kOpTableRun = 5,  // `count` table entries from index a on are the pages b, b + 1, ...
  kOpTableClear = 6, // `count` table entries from index a on name no page any more
};
struct PageTargets {
  uint8_t *k_pool, *v_pool, *k_ovf, *v_ovf;
  int32_t* table;
  int32_t *seg_off, *seg_cap, *seg_cap2, *seg_len;
};
template <int kN>
struct PageOps {
  int32_t n_copy, n_set;  // the copies come first
  PageOp op[kN];
};
// Arguments of up to 3.6 KB, or as many as a launch takes (32 KB: 5 us more of the host's time).
constexpr int kFewBytes = 3584, kManyBytes = 31744;
constexpr int kFewOps = kFewBytes / 16, kManyOps = kManyBytes / 16;

// A block copies up to 64 rows of K and V, or 256 threads set one thing each.
template <int kN>
__global__ void __launch_bounds__(256) page_ops_kernel(const __grid_constant__ PageTargets t, const __grid_constant__ PageOps<kN> ops) {
  const int tid = threadIdx.x;
  if ((int)blockIdx.x < ops.n_copy) {
    const PageOp o = ops.op[blockIdx.x];
    const int rows = o.kind >> 3;
    const bool pool = (o.kind & 7) == kOpCopyPool;
    const int c = (tid & 15) * 16, part = (tid >> 4) & 1;  // 32 threads a row: 16 of K, 16 of V
    const uint8_t* src = (part ? (pool ? t.v_pool : t.v_ovf) : (pool ? t.k_pool : t.k_ovf)) + (int64_t)o.a * kRowBytes + c;
    uint8_t* dst = (part ? t.v_ovf : t.k_ovf) + (int64_t)o.b * kRowBytes + c;
    uint4 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = (tid >> 5) + 8 * i;
      if (r < rows) v[i] = *reinterpret_cast<const uint4*>(src + (int64_t)r * kRowBytes);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = (tid >> 5) + 8 * i;
      if (r < rows) *reinterpret_cast<uint4*>(dst + (int64_t)r * kRowBytes) = v[i];
    }
    if (tid == 0) t.table[o.c] = o.b / CATEKV_PAGE_ROWS;
    return;
  }
  const int i = ((int)blockIdx.x - ops.n_copy) * 256 + tid;
  if (i >= ops.n_set) return;
  const PageOp o = ops.op[ops.n_copy + i];
  const int n = o.kind >> 3;
  if ((o.kind & 7) == kOpSegment) {
    t.seg_off[n] = o.a;
    t.seg_cap[n] = o.b;
    if (t.seg_cap2) t.seg_cap2[n] = o.b;
    if (o.c >= 0) t.seg_len[n] = o.c;
  } else if ((o.kind & 7) == kOpTable) {
    t.table[o.a] = o.b;
    if (n > 1) t.table[o.a + 1] = o.c;
  } else {
    const int kind = o.kind & 7;
    for (int j = 0; j < n; ++j) t.table[o.a + j] = kind == kOpTableRun ? o.b + j : kind == kOpTableClear ? -1 : t.table[o.b + j];
  }
}

// Pages that move: page src[i] -> dst[i], src ascending, every dst below every src.  A block copies a page; the blocks behind those
// look every table entry up among the sources.
template <class T, int kBytes>
struct PageMoves {
  static constexpr int kRoom = kBytes / (2 * (int)sizeof(T));
  int32_t n, n_entries;
  T src[kRoom], dst[kRoom];
};
template <class T, int kBytes>
__global__ void __launch_bounds__(256) page_moves_kernel(const __grid_constant__ PageTargets t, const __grid_constant__ PageMoves<T, kBytes> m) {
  const int tid = threadIdx.x;
  if ((int)blockIdx.x < m.n) {
    constexpr int kChunks = CATEKV_PAGE_ROWS * kRowBytes / 16;  // of K, and of V
    const int64_t src = (int64_t)m.src[blockIdx.x] * kChunks, dst = (int64_t)m.dst[blockIdx.x] * kChunks;
    uint4 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = reinterpret_cast<const uint4*>(i < 4 ? t.k_ovf : t.v_ovf)[src + tid + (i & 3) * 256];
#pragma unroll
    for (int i = 0; i < 8; ++i) reinterpret_cast<uint4*>(i < 4 ? t.k_ovf : t.v_ovf)[dst + tid + (i & 3) * 256] = v[i];
    return;
  }
  const int e = ((int)blockIdx.x - m.n) * 256 + tid;
  if (e >= m.n_entries) return;
  const int page = t.table[e];
  int lo = 0, hi = m.n;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if ((int)m.src[mid] < page) lo = mid + 1;
    else hi = mid;
  }
  if (lo < m.n && (int)m.src[lo] == page) t.table[e] = (int)m.dst[lo];
}

constexpr int kDropSeqs = 512;
struct Drops {
  int32_t n[kDropSeqs];
};
__global__ void __launch_bounds__(128) truncate_kernel(int32_t* seg_len, const __grid_constant__ Drops d, int Hkv, int seg0, int n) {
  const int i = blockIdx.x * 128 + threadIdx.x;
  if (i >= n) return;
  const int drop = d.n[i / Hkv];
  if (drop > 0) seg_len[seg0 + i] = max(0, seg_len[seg0 + i] - drop);
}

// a growing array of host memory that does not throw
template <class T>
struct HostList {
  T* p = nullptr;
  size_t n = 0, room = 0;
  ~HostList() { free(p); }
  bool reserve(size_t m) {
    if (m <= room) return true;
    const size_t r = m < 2 * room ? 2 * room : (m < 64 ? 64 : m);
    T* q = (T*)realloc(p, r * sizeof(T));
    if (!q) return false;
    p = q;
    room = r;
    return true;
  }
  bool push(const T& x) {
    if (!reserve(n + 1)) return false;
    p[n++] = x;
    return true;
  }
  bool fill(size_t m, T x) {
    if (!reserve(m)) return false;
    n = m;
    for (size_t i = 0; i < m; ++i) p[i] = x;
    return true;
  }
  T& operator[](size_t i) { return p[i]; }
};

struct PageOrders {
  HostList<PageOp> copies, sets;
  // `rows` rows to the start of a page, which table entry `entry` names from now on
  bool copy_rows(bool pool, int64_t src, int page, int rows, int64_t entry) {
    return copies.push(PageOp{(pool ? kOpCopyPool : kOpCopyPage) | rows << 3, (int32_t)src, page * CATEKV_PAGE_ROWS, (int32_t)entry});
  }
  bool segment(int s, int off, int cap, int len) { return sets.push(PageOp{kOpSegment | s << 3, off, cap, len}); }
  bool entries_of(int64_t at, int64_t from, int n) {  // as the device's table has them
    return n == 0 || sets.push(PageOp{kOpTableCopy | n << 3, (int32_t)at, (int32_t)from, 0});
  }
  bool clear(int64_t at, int n) { return n <= 0 || sets.push(PageOp{kOpTableClear | n << 3, (int32_t)at, 0, 0}); }
  bool entries(int64_t at, const int32_t* v, int n) {
    int run = 1;
    while (run < n && v[run] == v[0] + run) ++run;
    if (run == n && n > 2) return sets.push(PageOp{kOpTableRun | n << 3, (int32_t)at, v[0], 0});
    for (int i = 0; i < n; i += 2)
      if (!sets.push(PageOp{kOpTable | (i + 1 < n ? 2 : 1) << 3, (int32_t)(at + i), v[i], i + 1 < n ? v[i + 1] : 0})) return false;
    return true;
  }
};
template <int kN>
static int send_batch(const PageTargets& t, const PageOp* copies, int nc, const PageOp* sets, int ns, cudaStream_t st) {
  PageOps<kN> ops;
  ops.n_copy = nc;
  ops.n_set = ns;
  memcpy(ops.op, copies, sizeof(PageOp) * (size_t)nc);
  memcpy(ops.op + nc, sets, sizeof(PageOp) * (size_t)ns);
  page_ops_kernel<kN><<<nc + (ns + 255) / 256, 256, 0, st>>>(t, ops);
  CATEKV_CUDA_TRY(cudaGetLastError());
  return CATEKV_OK;
}
static PageTargets targets(const catekv_cache* c) {
  const catekv_pages* p = c->pages;
  PageTargets t = {};
  t.k_pool = (uint8_t*)c->k_pool;
  t.v_pool = (uint8_t*)c->v_pool;
  t.k_ovf = (uint8_t*)p->k_ovf;
  t.v_ovf = (uint8_t*)p->v_ovf;
  t.table = p->table_dev;
  t.seg_off = const_cast<int32_t*>(c->seg_off_dev);
  t.seg_cap = const_cast<int32_t*>(p->seg_cap_dev);
  t.seg_cap2 = c->seg_cap_dev != p->seg_cap_dev ? const_cast<int32_t*>(c->seg_cap_dev) : nullptr;
  t.seg_len = c->seg_len_dev;
  return t;
}
static int send(const catekv_cache* c, PageOrders& o, cudaStream_t st) {
  const PageTargets t = targets(c);
  size_t ic = 0, is = 0;
  while (ic < o.copies.n || is < o.sets.n) {
    const size_t left = o.copies.n - ic + o.sets.n - is, room = left <= kFewOps ? kFewOps : kManyOps;
    const size_t nc = std::min(o.copies.n - ic, room), ns = std::min(o.sets.n - is, room - nc);
    const int rc = left <= kFewOps ? send_batch<kFewOps>(t, o.copies.p + ic, (int)nc, o.sets.p + is, (int)ns, st)
                                   : send_batch<kManyOps>(t, o.copies.p + ic, (int)nc, o.sets.p + is, (int)ns, st);
    if (rc) return rc;
    ic += nc;
    is += ns;
  }
  return CATEKV_OK;
}

// Which lists hold a page: counts [n_pages] of the table entries in force.  `skip` (or null): segments that are left out.
static int count_pages(const catekv_cache* c, const uint8_t* skip, HostList<int32_t>& count) {
  const catekv_pages* p = c->pages;
  if (!count.fill((size_t)p->n_pages, 0)) return CATEKV_ERR_WORKSPACE;
  for (int s = 0; s < c->B * c->Hkv; ++s) {
    if (p->seg_pages[s] < 0 || p->seg_pages[s] > p->max_pages) return CATEKV_ERR_INVALID_ARG;
    if (skip && skip[s]) continue;
    const int32_t* row = p->table + (size_t)s * p->max_pages;
    for (int q = 0; q < p->seg_pages[s]; ++q) {
      if (row[q] < 0 || row[q] >= p->n_pages) return CATEKV_ERR_INVALID_ARG;
      ++count[row[q]];
    }
  }
  return CATEKV_OK;
}
// next_free and released, from the tables as they are
static void settle(catekv_pages* p, const HostList<int32_t>& count) {
  int top = 0, live = 0;
  for (int q = 0; q < p->n_pages; ++q)
    if (count.p[q]) {
      top = q + 1;
      ++live;
    }
  p->next_free = top;
  p->released = top - live;
}
template <class T, int kBytes>
static int send_moves(const catekv_cache* c, const int32_t* src, const int32_t* dst, size_t n, cudaStream_t st) {
  PageMoves<T, kBytes> m;
  m.n_entries = c->B * c->Hkv * c->pages->max_pages;
  for (size_t i0 = 0; i0 < n; i0 += m.kRoom) {
    m.n = (int32_t)std::min(n - i0, (size_t)m.kRoom);
    for (int i = 0; i < m.n; ++i) {
      m.src[i] = (T)src[i0 + i];
      m.dst[i] = (T)dst[i0 + i];
    }
    page_moves_kernel<T, kBytes><<<m.n + (m.n_entries + 255) / 256, 256, 0, st>>>(targets(c), m);
    CATEKV_CUDA_TRY(cudaGetLastError());
  }
  return CATEKV_OK;
}
// Table entries behind those in force.  A list that gives pages back keeps their entries while the pages are free and were its own: it is likely to be given
// them again, and catekv_truncate then needs no order (drafted tokens).  Before a page is handed out or moved to, every such entry becomes -1, so
// that no list's row names a page of another one, which a replayed append without room, or attention under a plan made for a longer list, would follow.
// Host and device hold the same entries; they lie directly behind those in force.
static int entries_end(const catekv_pages* p, int s) {
  const int32_t* row = p->table + (size_t)s * p->max_pages;
  int q = p->seg_pages[s];
  while (q < p->max_pages && row[q] >= 0) ++q;
  return q;
}
// Orders that clear them, of all lists, from entry from(s) on; forget: the same on the host.
template <class From>
static bool clear_behind(const catekv_cache* c, PageOrders& orders, From from) {
  for (int s = 0; s < c->B * c->Hkv; ++s) {
    const int at = from(s), end = entries_end(c->pages, s);
    if (at < end && !orders.clear((int64_t)s * c->pages->max_pages + at, end - at)) return false;
  }
  return true;
}
static void forget(catekv_pages* p, int s, int at) {
  int32_t* row = p->table + (size_t)s * p->max_pages;
  for (int q = at; q < p->max_pages && (q < p->seg_pages[s] || row[q] >= 0); ++q) row[q] = -1;
}
struct FreePages {  // the lowest pages that no list held when the call began, one after the other
  const HostList<int32_t>& count;
  int at = 0;
  int take() {
    while (at < (int)count.n && count.p[at]) ++at;
    return at < (int)count.n ? at++ : -1;
  }
};
static int check_paged(const catekv_cache* c) {
  int rc = check_cache(c);
  if (rc) return rc;
  if (!c->pages || c->reserved) return CATEKV_ERR_INVALID_ARG;  // rows are looked at one by one: the lengths have to be exact
  const int64_t n = (int64_t)c->B * c->Hkv;
  if (n >= 1 << 28 || n * c->pages->max_pages > INT32_MAX || (int64_t)c->pages->n_pages * CATEKV_PAGE_ROWS > INT32_MAX) return CATEKV_ERR_UNSUPPORTED;
  for (int s = 0; s < (int)n; ++s) {
    if (c->seg_cap[s] < 0 || c->seg_cap[s] % CATEKV_SEG_ALIGN || c->seg_off[s] < 0) return CATEKV_ERR_INVALID_ARG;
    if (c->pages->seg_pages[s] < 0 || c->pages->seg_pages[s] > c->pages->max_pages) return CATEKV_ERR_INVALID_ARG;
    if (c->seg_len[s] < 0 || c->seg_len[s] > seg_capacity(c, s)) return CATEKV_ERR_INVALID_ARG;
  }
  return CATEKV_OK;
}
// The calls below change the host's tables: one that is captured would be replayed without that, and name pages again that are other lists' by then.
static int check_not_captured(cudaStream_t st) {
  cudaStreamCaptureStatus s = cudaStreamCaptureStatusNone;
  CATEKV_CUDA_TRY(cudaStreamIsCapturing(st, &s));
  return s == cudaStreamCaptureStatusNone ? CATEKV_OK : CATEKV_ERR_UNSUPPORTED;
}
static inline int div_up(int64_t a, int b) { return (int)((a + b - 1) / b); }

// Room for all_new rows in every list, or for each[b] in those of sequence b.
static int reserve(catekv_cache* cache, int32_t all_new, const int32_t* each, catekv_stream stream) {
  int rc = check_cache(cache);
  if (rc) return rc;
  if (!cache->pages || all_new < 0) return CATEKV_ERR_INVALID_ARG;
  for (int b = 0; each && b < cache->B; ++b)
    if (each[b] < 0) return CATEKV_ERR_INVALID_ARG;
  catekv_pages* p = cache->pages;
  const int n = cache->B * cache->Hkv;
  auto rows_over = [&](int s) -> int64_t { return (int64_t)cache->seg_len[s] + (each ? each[s / cache->Hkv] : all_new) - cache->seg_cap[s]; };
  // first pass: what is needed, nothing changed yet
  int64_t extra = 0;
  for (int s = 0; s < n; ++s) {
    if (p->seg_pages[s] < 0 || p->seg_pages[s] > p->max_pages) return CATEKV_ERR_INVALID_ARG;
    if (cache->seg_len[s] < 0 || cache->seg_len[s] > seg_capacity(cache, s)) return CATEKV_ERR_INVALID_ARG;
    const int64_t over = rows_over(s);
    const int64_t want = over > 0 ? (over + CATEKV_PAGE_ROWS - 1) / CATEKV_PAGE_ROWS : 0;
    if (want > p->max_pages) return CATEKV_ERR_CAPACITY;
    if (want > p->seg_pages[s]) extra += want - p->seg_pages[s];
  }
  if (extra == 0) return CATEKV_OK;
  if (extra > (int64_t)p->n_pages - p->next_free + p->released) return CATEKV_ERR_CAPACITY;
  if ((int64_t)n * p->max_pages > INT32_MAX) return CATEKV_ERR_UNSUPPORTED;
  // the lowest pages that are free: from next_free on, unless some below it have been released
  HostList<int32_t> count;
  if (p->released) {
    rc = count_pages(cache, nullptr, count);
    if (rc) return rc;
  }
  FreePages free_pages{count};
  HostList<int32_t> given;
  PageOrders orders;
  int next = p->next_free;
  for (int s = 0; s < n; ++s) {
    const int64_t over = rows_over(s);
    const int want = over > 0 ? div_up(over, CATEKV_PAGE_ROWS) : 0, have = p->seg_pages[s];
    const size_t g0 = given.n;
    for (int q = have; q < want; ++q) {
      const int page = p->released ? free_pages.take() : next++;
      if (page < 0) return CATEKV_ERR_INVALID_ARG;  // `released` does not fit the tables
      if (!given.push(page)) return CATEKV_ERR_WORKSPACE;
    }
    if (want > have && !orders.entries((int64_t)s * p->max_pages + have, given.p + g0, want - have)) return CATEKV_ERR_WORKSPACE;
  }
  auto pages_then = [&](int s) { return std::max(p->seg_pages[s], (int)std::max<int64_t>(0, (rows_over(s) + CATEKV_PAGE_ROWS - 1) / CATEKV_PAGE_ROWS)); };
  if (!clear_behind(cache, orders, pages_then)) return CATEKV_ERR_WORKSPACE;
  rc = check_not_captured((cudaStream_t)stream);
  if (!rc) rc = send(cache, orders, (cudaStream_t)stream);
  if (rc) return rc;
  for (int s = 0; s < n; ++s) forget(p, s, pages_then(s));
  size_t g = 0;
  int top = p->next_free;
  for (int s = 0; s < n; ++s) {
    const int64_t over = rows_over(s);
    const int want = over > 0 ? div_up(over, CATEKV_PAGE_ROWS) : 0;
    for (int q = p->seg_pages[s]; q < want; ++q) {
      top = std::max(top, given[g] + 1);
      p->table[(size_t)s * p->max_pages + q] = given[g++];
    }
    p->seg_pages[s] = std::max(p->seg_pages[s], want);
  }
  p->released += top - p->next_free - (int)extra;
  p->next_free = top;
  return CATEKV_OK;
}

}  // namespace catekv

using namespace catekv;

extern "C" int catekv_pages_reserve(catekv_cache* cache, int32_t n_new, catekv_stream stream) {
  CATEKV_API_RANGE();
  return reserve(cache, n_new, nullptr, stream);
}

extern "C" int catekv_pages_reserve_each(catekv_cache* cache, const int32_t* n_new, catekv_stream stream) {
  CATEKV_API_RANGE();
  return n_new ? reserve(cache, 0, n_new, stream) : CATEKV_ERR_INVALID_ARG;
}

extern "C" int catekv_fork(catekv_cache* cache, const int32_t* parent, catekv_stream stream) {
  CATEKV_API_RANGE();
  int rc = check_paged(cache);
  if (rc) return rc;
  if (!parent) return CATEKV_ERR_INVALID_ARG;
  const int B = cache->B, Hkv = cache->Hkv, n = B * Hkv;
  catekv_pages* p = cache->pages;
  HostList<uint8_t> is_parent, gone;
  if (!is_parent.fill(B, 0) || !gone.fill(n, 0)) return CATEKV_ERR_WORKSPACE;
  int replaced = 0;
  for (int b = 0; b < B; ++b) {
    if (parent[b] < 0 || parent[b] >= B) return CATEKV_ERR_INVALID_ARG;
    if (parent[b] != b) {
      is_parent[parent[b]] = 1;
      ++replaced;
    }
  }
  if (!replaced) return CATEKV_OK;
  for (int b = 0; b < B; ++b)
    for (int h = 0; h < Hkv; ++h) gone[(size_t)b * Hkv + h] = parent[b] != b && !is_parent[b];
  HostList<int32_t> count;  // pages that may not be given out: all but those of replaced sequences that nothing continues from
  rc = count_pages(cache, gone.p, count);
  if (rc) return rc;
  FreePages free_pages{count};
  struct Child {
    int32_t seg, off, cap, len, full, fresh, page[2];  // shares `full` pages, then has `fresh` ones of its own
  };
  HostList<Child> children;
  HostList<int32_t> entries;  // of children whose parent is replaced itself: its row of the tables as it was
  PageOrders orders;
  if (!children.reserve((size_t)replaced * Hkv) || !orders.copies.reserve((size_t)replaced * Hkv) || !orders.sets.reserve((size_t)replaced * Hkv * 3))
    return CATEKV_ERR_WORKSPACE;
  for (int b = 0; b < B; ++b) {
    if (parent[b] == b) continue;
    const bool moving = parent[parent[b]] != parent[b];
    for (int h = 0; h < Hkv; ++h) {
      const int s = b * Hkv + h, f = parent[b] * Hkv + h;
      const int len = cache->seg_len[f], cap = cache->seg_cap[f], off = cache->seg_off[f];
      const bool pool = len <= cap;  // nothing in pages
      const int64_t row = (int64_t)f * p->max_pages, to = (int64_t)s * p->max_pages;
      Child c = {s, off, pool ? len / CATEKV_SEG_ALIGN * CATEKV_SEG_ALIGN : cap, len, pool ? 0 : (len - cap) / CATEKV_PAGE_ROWS, 0, {0, 0}};
      const int done = c.cap + c.full * CATEKV_PAGE_ROWS;
      c.fresh = div_up(len - done, CATEKV_PAGE_ROWS);
      if (c.full + c.fresh > p->max_pages) return CATEKV_ERR_CAPACITY;
      bool ok = true;
      for (int i = 0; i < c.fresh; ++i) {
        c.page[i] = free_pages.take();
        if (c.page[i] < 0) return CATEKV_ERR_CAPACITY;
        const int r = done + i * CATEKV_PAGE_ROWS;
        ok = ok && orders.copy_rows(pool, pool ? (int64_t)off + r : (int64_t)p->table[row + c.full] * CATEKV_PAGE_ROWS, c.page[i],
                                    std::min(CATEKV_PAGE_ROWS, len - r), to + c.full + i);
      }
      ok = ok && children.push(c) && orders.segment(s, c.off, c.cap, c.len);
      if (moving) {
        ok = ok && orders.entries(to, p->table + row, c.full);
        for (int q = 0; q < c.full; ++q) ok = ok && entries.push(p->table[row + q]);
      } else {
        ok = ok && orders.entries_of(to, row, c.full);
      }
      if (!ok) return CATEKV_ERR_WORKSPACE;
    }
  }
  HostList<int32_t> pages_then;
  if (!pages_then.fill(n, 0)) return CATEKV_ERR_WORKSPACE;
  for (int s = 0; s < n; ++s) pages_then[s] = p->seg_pages[s];
  for (size_t i = 0; i < children.n; ++i) pages_then[children[i].seg] = children[i].full + children[i].fresh;
  if (!clear_behind(cache, orders, [&](int s) { return pages_then[s]; })) return CATEKV_ERR_WORKSPACE;
  cudaStream_t st = (cudaStream_t)stream;
  rc = check_not_captured(st);
  if (!rc) rc = send(cache, orders, st);
  if (rc) return rc;
  int32_t *seg_off = const_cast<int32_t*>(cache->seg_off), *seg_cap = const_cast<int32_t*>(cache->seg_cap);
  size_t at = 0;
  for (int s = 0; s < n; ++s)
    if (parent[s / Hkv] == s / Hkv) forget(p, s, p->seg_pages[s]);
  for (int s = 0; s < n; ++s)  // what replaced parents held; the others' pages are not counted
    if (parent[s / Hkv] != s / Hkv && !gone[s])
      for (int q = 0; q < p->seg_pages[s]; ++q) --count[p->table[(size_t)s * p->max_pages + q]];
  for (size_t i = 0; i < children.n; ++i) {
    const Child& c = children[i];
    const int b = c.seg / Hkv, from = parent[b] * Hkv + c.seg % Hkv;
    int32_t* row = p->table + (size_t)c.seg * p->max_pages;
    if (parent[parent[b]] != parent[b]) {
      if (c.full) memcpy(row, entries.p + at, sizeof(int32_t) * (size_t)c.full);
      at += (size_t)c.full;
    } else if (c.full) {
      memcpy(row, p->table + (size_t)from * p->max_pages, sizeof(int32_t) * (size_t)c.full);
    }
    for (int q = 0; q < c.fresh; ++q) row[c.full + q] = c.page[q];
    seg_off[c.seg] = c.off;
    seg_cap[c.seg] = c.cap;
    cache->seg_len[c.seg] = c.len;
    forget(p, c.seg, c.full + c.fresh);
    p->seg_pages[c.seg] = c.full + c.fresh;
    for (int q = 0; q < c.full + c.fresh; ++q) ++count[row[q]];
  }
  settle(p, count);
  return CATEKV_OK;
}

extern "C" int catekv_truncate(catekv_cache* cache, const int32_t* n_drop, catekv_stream stream) {
  CATEKV_API_RANGE();
  int rc = check_cache(cache);
  if (rc) return rc;
  if (!n_drop || cache->reserved) return CATEKV_ERR_INVALID_ARG;
  const int B = cache->B, Hkv = cache->Hkv, n = B * Hkv;
  catekv_pages* p = cache->pages;
  if (p) {
    rc = check_paged(cache);
    if (rc) return rc;
  }
  bool any = false;
  for (int b = 0; b < B; ++b) {
    if (n_drop[b] < 0) return CATEKV_ERR_INVALID_ARG;
    any = any || n_drop[b] > 0;
  }
  for (int s = 0; s < n; ++s)
    if (cache->seg_len[s] < 0) return CATEKV_ERR_INVALID_ARG;
  if (!any) return CATEKV_OK;

  struct Change {
    int32_t seg, cap, pages, n_entries, first, entry[2];  // new capacity and page count; table entries [first, first + n_entries) that change
    bool clear;                                           // the entries behind them are cleared at once
  };
  HostList<Change> changes;
  HostList<int32_t> count, at_start, cap;
  // Lists that read the same segment's rows (sequences that were forked), a group by offset, ascending: where a list's group begins, the largest
  // capacity of those behind the list, and by group that of those already passed (as this call leaves them).
  HostList<int64_t> by_off;
  HostList<int32_t> group, behind, passed;
  bool shared = false;
  PageOrders orders;
  if (p) {
    if (!cap.fill(n, 0)) return CATEKV_ERR_WORKSPACE;
    for (int s = 0; s < n; ++s) {
      cap[s] = cache->seg_cap[s];
      if (cap[s] > 0 && !by_off.push((int64_t)cache->seg_off[s] << 32 | s)) return CATEKV_ERR_WORKSPACE;
    }
    std::sort(by_off.p, by_off.p + by_off.n);
    for (size_t i = 1; i < by_off.n; ++i) shared = shared || by_off[i] >> 32 == by_off[i - 1] >> 32;
    if (shared) {
      if (!group.fill(n, 0) || !behind.fill(n, 0) || !passed.fill(by_off.n, 0)) return CATEKV_ERR_WORKSPACE;
      for (size_t i = 1; i < by_off.n; ++i) group[(int32_t)by_off[i]] = by_off[i] >> 32 == by_off[i - 1] >> 32 ? group[(int32_t)by_off[i - 1]] : (int32_t)i;
      for (size_t i = by_off.n; i-- > 1;)
        if (by_off[i] >> 32 == by_off[i - 1] >> 32) behind[(int32_t)by_off[i - 1]] = std::max(behind[(int32_t)by_off[i]], cap[(int32_t)by_off[i]]);
    }
    rc = count_pages(cache, nullptr, count);
    if (rc) return rc;
    if (!at_start.reserve(count.n)) return CATEKV_ERR_WORKSPACE;
    at_start.n = count.n;
    if (count.n) memcpy(at_start.p, count.p, sizeof(int32_t) * count.n);
    FreePages free_pages{at_start};  // (a page released by this call may still be the source of one of its copies)
    for (int s = 0; s < n; ++s) {
      const int drop = n_drop[s / Hkv];
      const bool member = shared && cap[s] > 0;
      if (drop == 0) {
        if (member) passed[group[s]] = std::max(passed[group[s]], cap[s]);
        continue;
      }
      const int len = std::max(0, cache->seg_len[s] - drop);
      int32_t* row = p->table + (size_t)s * p->max_pages;
      Change c = {s, cap[s], len > cap[s] ? div_up(len - cap[s], CATEKV_PAGE_ROWS) : 0, 0, 0, {0, 0}, len == 0};
      const bool read = member && len < cap[s] && std::max(passed[group[s]], behind[s]) > len;  // another list reads the segment's rows behind the new end
      const int kept = read ? 0 : c.pages;
      for (int q = kept; q < p->seg_pages[s]; ++q) {
        --count[row[q]];
        c.clear = c.clear || at_start[row[q]] > 1;  // another list's entry too: they would both be given it
      }
      if (read) {
        c.cap = len / CATEKV_SEG_ALIGN * CATEKV_SEG_ALIGN;
        c.pages = c.n_entries = div_up(len - c.cap, CATEKV_PAGE_ROWS);
        if (c.pages > p->max_pages) return CATEKV_ERR_CAPACITY;
        for (int q = 0; q < c.pages; ++q) {
          const int page = free_pages.take(), r = c.cap + q * CATEKV_PAGE_ROWS;
          if (page < 0) return CATEKV_ERR_CAPACITY;
          c.entry[q] = page;
          ++count[page];
          if (!orders.copy_rows(true, (int64_t)cache->seg_off[s] + r, page, std::min(CATEKV_PAGE_ROWS, len - r), (int64_t)s * p->max_pages + q))
            return CATEKV_ERR_WORKSPACE;
        }
        cap[s] = c.cap;
        if (!orders.segment(s, cache->seg_off[s], c.cap, -1)) return CATEKV_ERR_WORKSPACE;
      } else if (kept > 0 && (len - cap[s]) % CATEKV_PAGE_ROWS && count[row[kept - 1]] > 1) {
        const int page = free_pages.take();  // the last page is another list's too, and no longer full here
        if (page < 0) return CATEKV_ERR_CAPACITY;
        --count[row[kept - 1]];
        ++count[page];
        c.first = kept - 1;
        c.n_entries = 1;
        c.entry[0] = page;
        if (!orders.copy_rows(false, (int64_t)row[kept - 1] * CATEKV_PAGE_ROWS, page, (len - cap[s]) % CATEKV_PAGE_ROWS,
                              (int64_t)s * p->max_pages + kept - 1))
          return CATEKV_ERR_WORKSPACE;
      }
      if (member) passed[group[s]] = std::max(passed[group[s]], cap[s]);
      if (!changes.push(c)) return CATEKV_ERR_WORKSPACE;
    }
  }
  HostList<int32_t> pages_then;
  const bool hands_out = orders.copies.n > 0;
  if (p) {
    if (!pages_then.fill(n, 0)) return CATEKV_ERR_WORKSPACE;
    for (int s = 0; s < n; ++s) pages_then[s] = hands_out ? p->seg_pages[s] : p->max_pages;  // (what is given back by this call is not handed out by it)
    for (size_t i = 0; i < changes.n; ++i) {
      const Change& c = changes[i];
      if (c.clear) pages_then[c.seg] = c.pages;
      else if (hands_out) pages_then[c.seg] = std::max(c.pages, p->seg_pages[c.seg]);
    }
    if (!clear_behind(cache, orders, [&](int s) { return pages_then[s]; })) return CATEKV_ERR_WORKSPACE;
  }
  cudaStream_t st = (cudaStream_t)stream;
  rc = check_not_captured(st);
  if (rc) return rc;
  if (orders.copies.n + orders.sets.n) {
    rc = send(cache, orders, st);
    if (rc) return rc;
  }
  for (int b0 = 0; b0 < B; b0 += kDropSeqs) {
    Drops d;
    const int nb = std::min(kDropSeqs, B - b0);
    memcpy(d.n, n_drop + b0, sizeof(int32_t) * (size_t)nb);
    truncate_kernel<<<div_up((int64_t)nb * Hkv, 128), 128, 0, st>>>(cache->seg_len_dev, d, Hkv, b0 * Hkv, nb * Hkv);
    CATEKV_CUDA_TRY(cudaGetLastError());
  }
  for (int s = 0; s < n; ++s)
    if (n_drop[s / Hkv] > 0) cache->seg_len[s] = std::max(0, cache->seg_len[s] - n_drop[s / Hkv]);
  if (p) {
    int32_t* seg_cap = const_cast<int32_t*>(cache->seg_cap);
    for (int s = 0; s < n; ++s) forget(p, s, pages_then[s]);
    for (size_t i = 0; i < changes.n; ++i) {
      const Change& c = changes[i];
      int32_t* row = p->table + (size_t)c.seg * p->max_pages;
      seg_cap[c.seg] = c.cap;
      p->seg_pages[c.seg] = c.pages;
      for (int q = 0; q < c.n_entries; ++q) row[c.first + q] = c.entry[q];
    }
    settle(p, count);
  }
  return CATEKV_OK;
}

extern "C" int catekv_pages_compact(catekv_cache* cache, int32_t* n_used, catekv_stream stream) {
  CATEKV_API_RANGE();
  int rc = check_paged(cache);
  if (rc) return rc;
  const int n = cache->B * cache->Hkv;
  catekv_pages* p = cache->pages;
  HostList<int32_t> count, src, dst, to;  // to: where a page is afterwards
  rc = count_pages(cache, nullptr, count);
  if (rc) return rc;
  int live = 0;
  for (int q = 0; q < p->n_pages; ++q) live += count[q] > 0;
  if (!to.reserve((size_t)p->n_pages) || !src.reserve((size_t)live) || !dst.reserve((size_t)live)) return CATEKV_ERR_WORKSPACE;
  int hole = 0;
  for (int q = 0; q < p->n_pages; ++q) {
    to.p[q] = q;
    if (q < live || !count[q]) continue;
    while (count[hole]) ++hole;
    src.push(q);
    dst.push(hole);
    to.p[q] = hole++;
  }
  cudaStream_t st = (cudaStream_t)stream;
  if (src.n) {
    PageOrders orders;
    if (!clear_behind(cache, orders, [&](int s) { return p->seg_pages[s]; })) return CATEKV_ERR_WORKSPACE;
    rc = check_not_captured(st);
    if (!rc) rc = send(cache, orders, st);
    if (rc) return rc;
    for (int s = 0; s < n; ++s) forget(p, s, p->seg_pages[s]);
    rc = p->n_pages > 65536 ? send_moves<int32_t, kManyBytes>(cache, src.p, dst.p, src.n, st)
           : src.n * 4 > kFewBytes ? send_moves<uint16_t, kManyBytes>(cache, src.p, dst.p, src.n, st)
                                   : send_moves<uint16_t, kFewBytes>(cache, src.p, dst.p, src.n, st);
    if (rc) return rc;
    for (int s = 0; s < n; ++s) {
      int32_t* row = p->table + (size_t)s * p->max_pages;
      for (int q = 0; q < p->seg_pages[s]; ++q) row[q] = to.p[row[q]];
    }
  }
  p->next_free = live;
  p->released = 0;
  if (n_used) *n_used = live;
  return CATEKV_OK;
}
