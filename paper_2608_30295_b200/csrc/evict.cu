// Eviction by accumulated attention weight: the selection of what a list keeps, and the move of it, into another cache or
// in place.  Measured in a replayed graph: 64 lists of a batch (24 of 49 K cut to half, the others copied, 902 MB) 161 us,
// 0.87 of the copy bandwidth, of which 137 are the move and 20 the selection; four lists of 1280 cut to 1024: 8.3 us (two
// launches); the first in place 130 us (604 MB moved), three lists of 118 K of one sequence 122 us (75 into another cache).
#include <math.h>

#include <atomic>

#include <cooperative_groups.h>

#include "decode.cuh"

namespace cg = cooperative_groups;

namespace catekv {

constexpr int kEvMaxSegs = 2048;  // the masked segments travel in the kernel arguments
struct EvMask {
  uint32_t w[kEvMaxSegs / 32];
};
struct EvList {
  uint16_t seg[kEvMaxSegs];
};

struct EvParams {
  int32_t budget, sink, local;
};
struct EvSeg {       // what becomes of a segment
  int32_t n;         // rows it has
  int32_t keep_all;
  int32_t k_sel;     // rows to select among [sink, cand_end)
  int32_t cand_end;
  int32_t kept;      // rows it keeps
  int32_t reserved[3];
};
// The same on host and device.
__host__ __device__ inline EvSeg evict_decide(int n, bool masked, const EvParams& p) {
  EvSeg s = {};
  s.n = n;
  if (!masked || p.budget >= n || p.sink + p.local >= n) {
    s.keep_all = 1;
    s.cand_end = n;
    s.kept = n;
    return s;
  }
  const int rest = p.budget - p.sink - p.local;
  s.cand_end = n - p.local;
  s.k_sel = rest > 0 ? rest : 0;
  s.kept = p.sink + s.k_sel + p.local;
  return s;
}

// ------------------------------------------------------------------------------------------
// Selection
// ------------------------------------------------------------------------------------------
// A cluster of CL CTAs per masked segment (1 where the list is short), each with a share of the candidates as sortable
// patterns (a non-negative float's bits order like the float): in registers up to 8 per thread, else in shared memory.
// The pattern of the k-th largest is found from the top, 11 + 11 + 9 bits, with a histogram per step: weights spread over
// many powers of two, so the first step (exponent and three bits) already leaves a few per cent.  The CTAs look at one
// another's histograms in two looks of a warp, 32 sums of 64 bins and then the 64 bins of one, and as every step has a
// histogram of its own, with one cluster barrier.  What is above the pattern is kept, of what equals it the first in row
// order; a warp's votes over 32 consecutive candidates place them, so that the list is written in order.  A chain of
// dependent steps (loads, barriers of 1 us in a cluster): 20 us for 24 lists of 49 K, 5 us for one of 1 K.
constexpr int kEvThreads = 1024;
constexpr int kEvWarps = kEvThreads / 32;
constexpr int kEvBins = 2048;
constexpr int kEvGroup = kEvBins / 32;        // bins of a first look's sum
constexpr int kEvRegs = 8;                    // candidates of a thread held in registers
constexpr int kEvRegShare = kEvRegs * kEvThreads;
constexpr int kEvStageMax = 49152;            // candidates a CTA may stage in shared memory (192 KB)
static_assert(kEvRegs * 32 <= kEvThreads, "one thread per word of votes");
__device__ __forceinline__ int ev_shift(int pass) { return pass == 0 ? 20 : pass == 1 ? 9 : 0; }

struct EvSelectArgs {
  const int32_t* seg_off;
  const int32_t* seg_len;
  const float* weights;
  EvSeg* segs;
  int32_t* idx;
  int64_t idx_stride;
  int32_t* chk;   // the checked build's status block, else null
  int32_t stage;  // candidates a CTA's shared memory holds (longer shares are read from global memory)
  EvParams p;
  EvList list;    // a cluster each
};

__device__ __forceinline__ unsigned int ev_pattern(float x) {  // negative as 0, NaN as infinite
  return x != x ? 0x7f800000u : (x > 0.f ? __float_as_uint(x) : 0u);
}
// inclusive sum over the warp's lanes 0 .. lane
__device__ __forceinline__ unsigned int ev_scan(unsigned int v, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned int y = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += y;
  }
  return v;
}

// Two CTAs per SM (32 registers): with one, the clusters of 24 lists of 49 K take two waves (29 us against 20).
template <int CL, bool kReg>
__global__ void __launch_bounds__(kEvThreads, 2) evict_select_kernel(const __grid_constant__ EvSelectArgs a) {
  cg::cluster_group cluster = cg::this_cluster();
  const int seg = a.list.seg[blockIdx.x / CL];
  const int rank = CL > 1 ? (int)cluster.block_rank() : 0;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  __shared__ unsigned int hist[3][kEvBins];
  __shared__ unsigned int s_sum[3][32];               // sums of 64 bins over the cluster, larger ones first
  __shared__ unsigned int s_gt[kEvWarps], s_eq[kEvWarps];
  __shared__ unsigned int s_word[kEvRegs * 32];       // votes of 32 consecutive candidates: counts above / at the threshold
  __shared__ unsigned int s_sel[3];
  __shared__ unsigned int s_tot[2];                   // this CTA's counts above and at the threshold, read by its peers
  extern __shared__ __align__(16) unsigned int key[];
  pdl_launch_dependents();
  for (int i = tid; i < 3 * kEvBins; i += kEvThreads) (&hist[0][0])[i] = 0u;
  if (tid < 96) (&s_sum[0][0])[tid] = 0u;
  if (CL > 1) cluster.sync();  // clear everywhere before a peer adds to it
  pdl_wait();
  const int n_rows = a.seg_len[seg], off = a.seg_off[seg];  // (one trip to memory)
  const EvSeg s = evict_decide(n_rows, true, a.p);
  if (rank == 0 && tid == 0) a.segs[seg] = s;
  if (s.keep_all) return;  // the whole cluster
  auto cluster_sync = [&]() {
    if (CL > 1) cluster.sync(); else __syncthreads();
  };
  int32_t* idx = a.idx + (int64_t)seg * a.idx_stride;
  const int S = a.p.sink;
  if (s.k_sel > 0) {
    const int n_pool = s.cand_end - S;
    const int per = ((n_pool + CL - 1) / CL + 31) / 32 * 32;
    const int lo = min(n_pool, rank * per), n_loc = min(n_pool, lo + per) - lo;
    const float* w = a.weights + (int64_t)off + S + lo;
    const bool staged = n_loc <= a.stage;
    auto ld = [&](int i) { return staged ? key[i] : ev_pattern(w[i]); };
    unsigned int mine[kEvRegs];  // kReg: candidate e * 1024 + tid
    if (kReg) {
#pragma unroll
      for (int e = 0; e < kEvRegs; ++e) mine[e] = e * kEvThreads + tid < n_loc ? ev_pattern(w[e * kEvThreads + tid]) : 0u;
    }
    unsigned int prefix = 0u, pmask = 0u, need = (unsigned int)s.k_sel;
    __syncthreads();  // the histograms are clear
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = ev_shift(pass);
      const unsigned int dmask = pass == 2 ? 511u : 2047u;
      unsigned int* h = hist[pass];
      auto count = [&](bool in, unsigned int v) {  // by whole warps
        const bool hit = in && (v & pmask) == prefix;
        const unsigned int d = (v >> shift) & dmask, d0 = __shfl_sync(0xffffffffu, d, 0);
        if (__all_sync(0xffffffffu, hit && d == d0)) {
          if (lane == 0) atomicAdd(&h[d], 32u);  // equal weights (rows that no query has looked at): one addition
        } else if (hit) {
          atomicAdd(&h[d], 1u);
        }
      };
      if (kReg) {
#pragma unroll
        for (int e = 0; e < kEvRegs; ++e)
          if (e * kEvThreads < n_loc) count(e * kEvThreads + tid < n_loc, mine[e]);
      } else if (pass == 0) {  // the first step brings the candidates in, four loads in flight
        for (int i0 = 0; i0 < n_loc; i0 += 4 * kEvThreads) {
          unsigned int v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int i = i0 + e * kEvThreads + tid;
            v[e] = i < n_loc ? ev_pattern(w[i]) : 0u;
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int i = i0 + e * kEvThreads + tid;
            if (staged && i < n_loc) key[i] = v[e];
            count(i < n_loc, v[e]);
          }
        }
      } else {
        for (int i0 = 0; i0 < n_loc; i0 += kEvThreads) count(i0 + tid < n_loc, i0 + tid < n_loc ? ld(i0 + tid) : 0u);
      }
      __syncthreads();
      {
        const unsigned int* p = &h[(31 - warp) * kEvGroup + 2 * lane];
        const unsigned int t = __reduce_add_sync(0xffffffffu, p[0] + p[1]);
        // lane r adds it to CTA r's sum: after the barrier every CTA has the cluster's
        if (CL > 1) {
          if (lane < CL && t) atomicAdd(cluster.map_shared_rank(&s_sum[pass][warp], lane), t);
        } else if (lane == 0) {
          s_sum[pass][warp] = t;
        }
      }
      cluster_sync();  // all histograms and sums of this step complete
      if (warp == 0) {
        const unsigned int c = s_sum[pass][lane];
        unsigned int inc = ev_scan(c, lane);
        const int gsel = __ffs(__ballot_sync(0xffffffffu, need <= inc)) - 1;  // the first sum that reaches `need`
        const unsigned int before = __shfl_sync(0xffffffffu, inc - c, gsel);
        // lane l: bins 63 - 2 l and 62 - 2 l of the group
        const int b1 = (31 - gsel) * kEvGroup + kEvGroup - 1 - 2 * lane;
        unsigned int c1 = 0u, c0 = 0u;
#pragma unroll
        for (int r = 0; r < CL; ++r) {
          const uint2 x = *reinterpret_cast<const uint2*>(CL > 1 ? cluster.map_shared_rank(&h[b1 - 1], r) : &h[b1 - 1]);
          c0 += x.x;
          c1 += x.y;
        }
        inc = before + ev_scan(c0 + c1, lane);
        const unsigned int ex = inc - c0 - c1;
        if (ex < need && need <= inc) {  // one of this lane's bins holds the need-th largest
          const bool upper = need <= ex + c1;
          s_sel[0] = (unsigned int)(upper ? b1 : b1 - 1);
          s_sel[1] = need - ex - (upper ? 0u : c1);
          s_sel[2] = upper ? c1 : c0;
        }
      }
      __syncthreads();
      prefix |= s_sel[0] << shift;
      pmask |= dmask << shift;
      need = s_sel[1];
      const bool whole = s_sel[2] == need;
      if (whole) break;  // everything in the bin is kept: no need to look closer
      // (s_sel is written again behind the next step's barriers)
    }
    // kept: patterns above the prefix, and the first `need` of those with it
    const unsigned int top = prefix | (~pmask & 0x7fffffffu);  // (patterns are below 2^31)
    auto emit = [&](int c, unsigned int rnk) {  // candidate c of this share is the rnk-th kept
      int r = S + (int)rnk;
#ifdef CATEKV_CHECKED
      r = checked_clamp(r, S, s.kept - a.p.local - 1, a.chk, kKidEvict, seg);
#endif
      idx[r] = S + lo + c;
    };
    // counts before a position of the share, and of the shares before it
    unsigned int gt_before = 0u, eq_before = 0u;
    auto add_peers = [&](unsigned int all_gt, unsigned int all_eq) {
      if (CL > 1) {
        if (tid == 0) {
          s_tot[0] = all_gt;
          s_tot[1] = all_eq;
        }
        cluster_sync();
        unsigned int tg = 0u, te = 0u;
        if (lane < rank) {
          const unsigned int* t = cluster.map_shared_rank(&s_tot[0], lane);
          tg = t[0];
          te = t[1];
        }
        gt_before += __reduce_add_sync(0xffffffffu, tg);
        eq_before += __reduce_add_sync(0xffffffffu, te);
        // this thread's last look at a peer's shared memory lies behind it; it waits for the others' before it leaves
        asm volatile("barrier.cluster.arrive.relaxed;\n" ::: "memory");
      }
    };
    const unsigned int low = (1u << lane) - 1u;
    if (kReg) {
      // word e * 32 + warp: the votes of candidates e * 1024 + 32 warp ...
#pragma unroll
      for (int e = 0; e < kEvRegs; ++e) {
        unsigned int both = 0u;
        if (e * kEvThreads < n_loc) {
          const bool in = e * kEvThreads + tid < n_loc;
          const unsigned int mg = __ballot_sync(0xffffffffu, in && mine[e] > top);
          const unsigned int mq = __ballot_sync(0xffffffffu, in && (mine[e] & pmask) == prefix);
          both = (unsigned int)__popc(mg) | ((unsigned int)__popc(mq) << 16);
        }
        if (lane == 0) s_word[e * 32 + warp] = both;
      }
      __syncthreads();
      if (warp < kEvRegs) {  // exclusive sums within a warp's 32 words (both counts stay below 2^16), totals per warp
        const unsigned int v = s_word[tid], inc = ev_scan(v, lane);
        s_word[tid] = inc - v;
        if (lane == 31) {
          s_gt[warp] = inc & 0xffffu;
          s_eq[warp] = inc >> 16;
        }
      }
      __syncthreads();
      const unsigned int tg = lane < kEvRegs ? s_gt[lane] : 0u, te = lane < kEvRegs ? s_eq[lane] : 0u;
      const unsigned int ig = ev_scan(tg, lane), ie = ev_scan(te, lane);
      add_peers(__shfl_sync(0xffffffffu, ig, 31), __shfl_sync(0xffffffffu, ie, 31));
#pragma unroll
      for (int e = 0; e < kEvRegs; ++e) {
        if (e * kEvThreads >= n_loc) break;
        const bool in = e * kEvThreads + tid < n_loc;
        const bool g = in && mine[e] > top, q = in && (mine[e] & pmask) == prefix;
        const unsigned int mg = __ballot_sync(0xffffffffu, g), mq = __ballot_sync(0xffffffffu, q);
        const unsigned int word = s_word[e * 32 + warp];
        const unsigned int gb = gt_before + __shfl_sync(0xffffffffu, ig - tg, e) + (word & 0xffffu) + __popc(mg & low);
        const unsigned int eb = eq_before + __shfl_sync(0xffffffffu, ie - te, e) + (word >> 16) + __popc(mq & low);
        if (g || (q && eb < need)) emit(e * kEvThreads + tid, gb + min(eb, need));
      }
    } else {
      const int chunk = (n_loc + kEvThreads - 1) / kEvThreads * 32;  // a warp's consecutive candidates
      const int w0 = min(n_loc, warp * chunk), w1 = min(n_loc, w0 + chunk);
      unsigned int gt = 0u, eq = 0u;
      for (int i0 = w0; i0 < w1; i0 += 32) {
        const bool in = i0 + lane < w1;
        const unsigned int v = in ? ld(i0 + lane) : 0u;
        gt += __popc(__ballot_sync(0xffffffffu, in && v > top));
        eq += __popc(__ballot_sync(0xffffffffu, in && (v & pmask) == prefix));
      }
      if (lane == 0) {
        s_gt[warp] = gt;
        s_eq[warp] = eq;
      }
      __syncthreads();
      gt_before = __reduce_add_sync(0xffffffffu, lane < warp ? s_gt[lane] : 0u);
      eq_before = __reduce_add_sync(0xffffffffu, lane < warp ? s_eq[lane] : 0u);
      add_peers(__reduce_add_sync(0xffffffffu, s_gt[lane]), __reduce_add_sync(0xffffffffu, s_eq[lane]));
      for (int i0 = w0; i0 < w1; i0 += 32) {
        const bool in = i0 + lane < w1;
        const unsigned int v = in ? ld(i0 + lane) : 0u;
        const bool g = in && v > top, q = in && (v & pmask) == prefix;
        const unsigned int mg = __ballot_sync(0xffffffffu, g), mq = __ballot_sync(0xffffffffu, q);
        const unsigned int eb = eq_before + __popc(mq & low);
        if (g || (q && eb < need)) emit(i0 + lane, gt_before + __popc(mg & low) + min(eb, need));
        gt_before += __popc(mg);
        eq_before += __popc(mq);
      }
    }
    if (CL > 1) asm volatile("barrier.cluster.wait;\n" ::: "memory");
  }
  if (rank == 0) {
    for (int i = tid; i < S; i += kEvThreads) idx[i] = i;
    for (int i = tid; i < a.p.local; i += kEvThreads) idx[S + s.k_sel + i] = s.cand_end + i;
  }
}

// ------------------------------------------------------------------------------------------
// Move
// ------------------------------------------------------------------------------------------
struct EvMoveArgs {
  EvMask mask;
  const EvSeg* segs;       // of the masked segments
  const int32_t* src_len;  // of the others, which keep all rows
  const int32_t* idx;
  int64_t idx_stride;
  const uint8_t* k_src;
  const uint8_t* v_src;
  const int32_t* src_off;
  const float* w_src;
  uint8_t* k_dst;
  uint8_t* v_dst;
  const int32_t* dst_off;
  const int32_t* dst_cap;
  int32_t* dst_len;
  float* w_dst;
  int32_t* idx_out;
  int64_t idx_out_stride;  // also the most entries of a segment: a replayed call's list may be longer than the host saw it
  int32_t rows_per_cta;
  int32_t* status;
  int32_t* chk;
};

__device__ __forceinline__ EvSeg move_seg(const EvMoveArgs& a, int seg) {
  if ((a.mask.w[seg >> 5] >> (seg & 31)) & 1u) return a.segs[seg];
  return evict_decide(a.src_len[seg], false, EvParams{0, 0, 0});
}
__device__ __forceinline__ int kept_row(const EvMoveArgs& a, const EvSeg& s, int seg, int r) {
  int row = s.keep_all ? r : a.idx[(int64_t)seg * a.idx_stride + r];
#ifdef CATEKV_CHECKED
  row = checked_clamp(row, 0, s.n - 1, a.chk, kKidEvict, seg);
#endif
  return row;
}

// Into another cache; bound by the copy's bytes (137 us for 874 MB, 6.4 TB/s).  A CTA moves rows_per_cta consecutive rows
// of a destination segment in tiles of 32 (a warp a row: lanes 0-15 K, 16-31 V), three tiles ahead with cp.async; a thread
// reads back only what it requested itself, so nothing is synchronised, and the list entries are fetched one tile before
// they are needed (one tile per CTA and no pipeline: 189 us).  It rewrites rows that a decode plan may cover: it never
// signals its dependents early (see launch_pdl).
constexpr int kEvTile = 32;
constexpr int kEvMoveThreads = 256;
constexpr int kEvMoveStages = 4;
constexpr int kEvPerThread = kEvTile * 32 / kEvMoveThreads;  // rows of a thread in a tile
constexpr int kEvMoveSmem = kEvMoveStages * kEvTile * 2 * kRowBytes;
__global__ void __launch_bounds__(kEvMoveThreads) evict_gather_kernel(const __grid_constant__ EvMoveArgs a) {
  extern __shared__ __align__(16) uint8_t stage[];
  const int seg = blockIdx.y;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();
  const int r0 = blockIdx.x * a.rows_per_cta;
  const int cap = a.dst_cap[seg];
  if (r0 >= cap && r0 > 0) return;
  const EvSeg s = move_seg(a, seg);
  const int len = min(s.kept, cap);
  if (r0 == 0 && tid == 0) {
    a.dst_len[seg] = len;
    if (s.kept > cap || (a.idx_out && len > a.idx_out_stride)) raise_status(a.status, CATEKV_STATUS_CAPACITY, kKidEvict, seg, s.kept);
  }
  const int64_t so = a.src_off[seg], to = a.dst_off[seg];
  const int r1 = min(r0 + a.rows_per_cta, len);
  const uint8_t* src = (lane < 16 ? a.k_src : a.v_src) + so * kRowBytes + (lane & 15) * 16;
  uint8_t* dst = (lane < 16 ? a.k_dst : a.v_dst) + to * kRowBytes + (lane & 15) * 16;
  uint8_t* mine = stage + tid * 16;
  const uint32_t mine_addr = smem_u32(mine);
  int row[kEvPerThread];
  auto fetch_rows = [&](int t) {  // list entries of tile t
#pragma unroll
    for (int i = 0; i < kEvPerThread; ++i) {
      const int r = r0 + t * kEvTile + warp + i * (kEvMoveThreads / 32);
      row[i] = r < r1 ? kept_row(a, s, seg, r) : 0;
    }
  };
  auto request = [&](int t) {  // tile t, by the entries in `row`
    const int st = t % kEvMoveStages;
#pragma unroll
    for (int i = 0; i < kEvPerThread; ++i) {
      const int r = r0 + t * kEvTile + warp + i * (kEvMoveThreads / 32);
      if (r < r1) cp_async16(mine_addr + (st * kEvPerThread + i) * kEvMoveThreads * 16, src + (int64_t)row[i] * kRowBytes, 16);
    }
    cp_async_commit();
  };
  const int tiles = (r1 - r0 + kEvTile - 1) / kEvTile;  // <= 0 behind the list
  fetch_rows(0);
  for (int t = 0; t < kEvMoveStages - 1; ++t) {
    request(t);
    fetch_rows(t + 1);
  }
  // the rows' weights, and the list for the caller, while the first tiles arrive
  for (int r = r0 + tid; r < min(r0 + a.rows_per_cta, cap); r += kEvMoveThreads) {
    float w = 0.f;
    if (r < len) {
      const int from = kept_row(a, s, seg, r);
      w = a.w_src[so + from];
      if (a.idx_out && r < a.idx_out_stride) a.idx_out[(int64_t)seg * a.idx_out_stride + r] = from;
    }
    a.w_dst[to + r] = w;
  }
  for (int t = 0; t < tiles; ++t) {
    request(t + kEvMoveStages - 1);
    fetch_rows(t + kEvMoveStages);
    cp_async_wait<kEvMoveStages - 1>();
    const int st = t % kEvMoveStages;
#pragma unroll
    for (int i = 0; i < kEvPerThread; ++i) {
      const int r = r0 + t * kEvTile + warp + i * (kEvMoveThreads / 32);
      if (r < r1)
        *reinterpret_cast<uint4*>(dst + (int64_t)r * kRowBytes) =
            *reinterpret_cast<const uint4*>(mine + (st * kEvPerThread + i) * kEvMoveThreads * 16);
    }
  }
  cp_async_wait<0>();
}

// In place.  Kept row j comes from row idx[j] >= j, so a tile of destination rows may be written once it has been read
// itself: nothing behind it reads there, and what is requested ahead lies behind it.  That makes a segment sequential in
// its rows, so the work is split over the columns instead: a CTA moves kSlice bytes of every row of K or V, two tiles
// ahead with cp.async and one barrier per tile (the tile has been read by everybody; the writes are a thread's own).
// 64 bytes are two DRAM sectors; 32, where the segments are few, make twice the CTAs, 16 per list however long it is (the bound for one
// sequence: three lists of 118 K cut to half 122 us, their floor 28).  Large tiles pay: 24 lists of 49 K,
// selection included, take 130 us with tiles of 32 KB and three stages, 167 with 16 KB and four, 206 with 8 KB and eight
// (303 with a tile at a time through registers).
constexpr int kEvInThreads = 512;
constexpr int kEvInTileBytes = 32768;
constexpr int kEvInStages = 3;
constexpr int kEvInSmem = kEvInStages * kEvInTileBytes;
constexpr int kEvInChunks = kEvInTileBytes / (16 * kEvInThreads);  // 16-byte chunks of a thread in a tile
constexpr int kEvWRows = 8;                                        // weights of a thread in a tile
struct EvInArgs {
  EvMoveArgs m;
  int32_t n_masked;
  EvList list;
};
template <int kSlice>
__global__ void __launch_bounds__(kEvInThreads) evict_inplace_kernel(const __grid_constant__ EvInArgs g) {
  extern __shared__ __align__(16) uint8_t stage[];
  constexpr int kSlices = 2 * kRowBytes / kSlice;
  constexpr int kPer = kSlice / 16;  // chunks of a row
  constexpr int kRows = kEvInTileBytes / kSlice;
  const EvMoveArgs& a = g.m;
  const int tid = threadIdx.x;
  pdl_wait();
  if ((int)blockIdx.x >= g.n_masked * kSlices) {  // a segment's weights, length and list for the caller
    const int seg = blockIdx.x - g.n_masked * kSlices;
    const EvSeg s = move_seg(a, seg);
    const int len = s.kept;
    if (a.idx_out) {
      if (tid == 0 && len > a.idx_out_stride) raise_status(a.status, CATEKV_STATUS_CAPACITY, kKidEvict, seg, len);
      const int n_out = (int)min((int64_t)len, a.idx_out_stride);
      for (int r = tid; r < n_out; r += kEvInThreads) a.idx_out[(int64_t)seg * a.idx_out_stride + r] = kept_row(a, s, seg, r);
    }
    if (s.keep_all) return;
    float* w = a.w_dst + a.dst_off[seg];
    if (tid == 0) a.dst_len[seg] = len;
    for (int t0 = 0; t0 < len; t0 += kEvInThreads * kEvWRows) {
      float v[kEvWRows];
#pragma unroll
      for (int i = 0; i < kEvWRows; ++i) {
        const int r = t0 + tid + i * kEvInThreads;
        if (r < len) v[i] = w[kept_row(a, s, seg, r)];
      }
      __syncthreads();  // the tile has been read
#pragma unroll
      for (int i = 0; i < kEvWRows; ++i) {
        const int r = t0 + tid + i * kEvInThreads;
        if (r < len) w[r] = v[i];
      }
    }
    for (int r = len + tid; r < a.dst_cap[seg]; r += kEvInThreads) w[r] = 0.f;
    return;
  }
  const int seg = g.list.seg[blockIdx.x / kSlices], slice = blockIdx.x % kSlices;
  const EvSeg s = move_seg(a, seg);
  if (s.keep_all) return;
  const int len = s.kept;
  uint8_t* base = (slice < kSlices / 2 ? a.k_dst : a.v_dst) + (int64_t)a.dst_off[seg] * kRowBytes + (slice % (kSlices / 2)) * kSlice + (tid % kPer) * 16;
  uint8_t* mine = stage + tid * 16;
  const uint32_t mine_addr = smem_u32(mine);
  int row[kEvInChunks];
  auto dst_row = [&](int t, int i) { return t * kRows + (tid + i * kEvInThreads) / kPer; };
  auto fetch_rows = [&](int t) {
#pragma unroll
    for (int i = 0; i < kEvInChunks; ++i) {
      const int r = dst_row(t, i);
      row[i] = r < len ? kept_row(a, s, seg, r) : 0;
    }
  };
  auto request = [&](int t) {
#pragma unroll
    for (int i = 0; i < kEvInChunks; ++i)
      if (dst_row(t, i) < len)
        cp_async16(mine_addr + ((t % kEvInStages) * kEvInChunks + i) * kEvInThreads * 16, base + (int64_t)row[i] * kRowBytes, 16);
    cp_async_commit();
  };
  const int tiles = (len + kRows - 1) / kRows;
  fetch_rows(0);
  for (int t = 0; t < kEvInStages - 1; ++t) {
    request(t);
    fetch_rows(t + 1);
  }
  for (int t = 0; t < tiles; ++t) {
    request(t + kEvInStages - 1);
    fetch_rows(t + kEvInStages);
    cp_async_wait<kEvInStages - 1>();
    __syncthreads();  // the tile has been read by everybody
#pragma unroll
    for (int i = 0; i < kEvInChunks; ++i) {
      const int r = dst_row(t, i);
      if (r < len)
        *reinterpret_cast<uint4*>(base + (int64_t)r * kRowBytes) =
            *reinterpret_cast<const uint4*>(mine + ((t % kEvInStages) * kEvInChunks + i) * kEvInThreads * 16);
    }
  }
  cp_async_wait<0>();
}

struct EvWs {
  size_t off_status, off_segs, off_idx, bytes;
  int64_t stride;
};
static EvWs ev_ws_layout(int n_segs, int max_cap) {
  EvWs w;
  w.stride = (int64_t)align_up((size_t)(max_cap > 0 ? max_cap : 1), 64);
  size_t o = 0;
  w.off_status = o; o = CATEKV_STATUS_BYTES;
  w.off_segs = o; o = align_up(o + sizeof(EvSeg) * (size_t)n_segs, 256);
  w.off_idx = o; o = align_up(o + sizeof(int32_t) * (size_t)n_segs * w.stride, 256);
  w.bytes = o;
  return w;
}

template <int CL, bool kReg>
static int launch_evict_cluster(const EvSelectArgs& a, int n_masked, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(n_masked * CL);
  cfg.blockDim = dim3(kEvThreads);
  cfg.dynamicSmemBytes = kReg ? 0 : (size_t)a.stage * 4;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = CL;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = CL > 1 ? 2 : 1;
  CATEKV_CUDA_TRY(cudaLaunchKernelEx(&cfg, evict_select_kernel<CL, kReg>, a));
  return CATEKV_OK;
}

// the kernels' shared-memory limits, once per device
static int evict_attributes() {
  static std::atomic<bool> attr_set[64];
  int dev = 0;
  CATEKV_CUDA_TRY(cudaGetDevice(&dev));
  if (dev >= 0 && dev < 64 && attr_set[dev].load(std::memory_order_acquire)) return CATEKV_OK;
  const cudaFuncAttribute at = cudaFuncAttributeMaxDynamicSharedMemorySize;
  CATEKV_CUDA_TRY(cudaFuncSetAttribute(evict_select_kernel<1, false>, at, kEvStageMax * 4));
  CATEKV_CUDA_TRY(cudaFuncSetAttribute(evict_select_kernel<2, false>, at, kEvStageMax * 4));
  CATEKV_CUDA_TRY(cudaFuncSetAttribute(evict_select_kernel<4, false>, at, kEvStageMax * 4));
  CATEKV_CUDA_TRY(cudaFuncSetAttribute(evict_select_kernel<8, false>, at, kEvStageMax * 4));
  CATEKV_CUDA_TRY(cudaFuncSetAttribute(evict_gather_kernel, at, kEvMoveSmem));
  CATEKV_CUDA_TRY(cudaFuncSetAttribute(evict_inplace_kernel<32>, at, kEvInSmem));
  CATEKV_CUDA_TRY(cudaFuncSetAttribute(evict_inplace_kernel<64>, at, kEvInSmem));
  if (dev >= 0 && dev < 64) attr_set[dev].store(true, std::memory_order_release);
  return CATEKV_OK;
}

// max_pool: bound of a masked segment's candidates.  The smallest cluster whose CTAs hold their shares in registers, as
// long as all clusters are resident at once with two CTAs per SM; else fewer CTAs with longer shares in shared memory.  (Above
// about 22 K staged candidates an SM holds one such CTA: 19 to 37 lists of more than 178 K rows take two waves of clusters, which
// wait for nothing outside their own.)
static int launch_evict_select(EvSelectArgs& a, int n_masked, int max_pool, cudaStream_t stream) {
  auto share = [&](int CL) { return ((max_pool + CL - 1) / CL + 31) / 32 * 32; };
  int CL = 1;
  while (CL < 8 && share(CL) > kEvRegShare && n_masked * CL * 2 <= 2 * sm_count()) CL *= 2;
  while (CL < 8 && share(CL) > kEvStageMax) CL *= 2;
  a.stage = share(CL) <= kEvStageMax ? share(CL) : 0;
  if (share(CL) <= kEvRegShare) {
    if (CL == 8) return launch_evict_cluster<8, true>(a, n_masked, stream);
    if (CL == 4) return launch_evict_cluster<4, true>(a, n_masked, stream);
    if (CL == 2) return launch_evict_cluster<2, true>(a, n_masked, stream);
    return launch_evict_cluster<1, true>(a, n_masked, stream);
  }
  if (CL == 8) return launch_evict_cluster<8, false>(a, n_masked, stream);
  if (CL == 4) return launch_evict_cluster<4, false>(a, n_masked, stream);
  if (CL == 2) return launch_evict_cluster<2, false>(a, n_masked, stream);
  return launch_evict_cluster<1, false>(a, n_masked, stream);
}

static int check_evict(const catekv_cache* c, const uint8_t* mask, int32_t budget, int32_t sink, int32_t local) {
  int rc = check_cache(c);
  if (rc) return rc;
  if (c->pages) return CATEKV_ERR_UNSUPPORTED;
  if (!mask || budget < 0 || sink < 0 || local < 0 || (int64_t)sink + local > INT32_MAX) return CATEKV_ERR_INVALID_ARG;
  if (c->reserved) return CATEKV_ERR_INVALID_ARG;
  for (int s = 0; s < c->B * c->Hkv; ++s)
    if (c->seg_len[s] < 0 || c->seg_len[s] > c->seg_cap[s]) return CATEKV_ERR_INVALID_ARG;
  return CATEKV_OK;
}

}  // namespace catekv

using namespace catekv;

extern "C" size_t catekv_evict_workspace_bytes(int32_t B, int32_t Hkv, int32_t max_cap) {
  if (B <= 0 || Hkv <= 0 || max_cap < 0) return 0;
  return ev_ws_layout(B * Hkv, max_cap).bytes;
}

extern "C" int catekv_evict_lengths(const catekv_cache* src, const uint8_t* evict_mask, int32_t budget, int32_t sink,
                                    int32_t local, int32_t* lens_out) {
  int rc = check_evict(src, evict_mask, budget, sink, local);
  if (rc) return rc;
  if (!lens_out) return CATEKV_ERR_INVALID_ARG;
  const EvParams p = {budget, sink, local};
  for (int s = 0; s < src->B * src->Hkv; ++s) lens_out[s] = evict_decide(src->seg_len[s], evict_mask[s] != 0, p).kept;
  return CATEKV_OK;
}

extern "C" int catekv_evict(const catekv_cache* src, const float* weights, const uint8_t* evict_mask, int32_t budget,
                            int32_t sink, int32_t local, catekv_cache* dst, float* dst_weights, int32_t* idx_out,
                            int64_t idx_stride, void* ws, size_t ws_bytes, catekv_stream stream) {
  CATEKV_API_RANGE();
  int rc = check_evict(src, evict_mask, budget, sink, local);
  if (rc) return rc;
  rc = check_cache(dst);
  if (rc) return rc;
  if (dst->pages) return CATEKV_ERR_UNSUPPORTED;
  if (!weights || !dst_weights || !ws || !src->seg_cap_dev || !dst->seg_cap_dev) return CATEKV_ERR_INVALID_ARG;
  if (src->B != dst->B || src->Hkv != dst->Hkv) return CATEKV_ERR_INVALID_ARG;
  if (((uintptr_t)src->k_pool | (uintptr_t)src->v_pool | (uintptr_t)dst->k_pool | (uintptr_t)dst->v_pool | (uintptr_t)ws) & 15) return CATEKV_ERR_INVALID_ARG;
  if (((uintptr_t)weights | (uintptr_t)dst_weights | (uintptr_t)idx_out) & 3) return CATEKV_ERR_INVALID_ARG;
  const bool in_place = src == dst;
  if (in_place != (weights == dst_weights)) return CATEKV_ERR_INVALID_ARG;
  if (!in_place && (src->k_pool == dst->k_pool || src->v_pool == dst->v_pool || src->seg_len == dst->seg_len ||
                    src->seg_len_dev == dst->seg_len_dev))
    return CATEKV_ERR_INVALID_ARG;
  const int n = src->B * src->Hkv;
  if (n > kEvMaxSegs) return CATEKV_ERR_UNSUPPORTED;
  EvSelectArgs sa = {};
  EvMoveArgs ma = {};
  sa.p = EvParams{budget, sink, local};
  int max_cap = 0, max_masked = 0, max_dst_cap = 0, max_kept = 0, n_masked = 0;
  int64_t dst_rows = 0;
  for (int s = 0; s < n; ++s) {
    const int kept = evict_decide(src->seg_len[s], evict_mask[s] != 0, sa.p).kept;
    if (kept > dst->seg_cap[s]) return CATEKV_ERR_CAPACITY;
    max_kept = kept > max_kept ? kept : max_kept;
    max_cap = src->seg_cap[s] > max_cap ? src->seg_cap[s] : max_cap;
    max_dst_cap = dst->seg_cap[s] > max_dst_cap ? dst->seg_cap[s] : max_dst_cap;
    dst_rows += dst->seg_cap[s];
    if (evict_mask[s]) {
      ma.mask.w[s >> 5] |= 1u << (s & 31);
      max_masked = src->seg_cap[s] > max_masked ? src->seg_cap[s] : max_masked;
      sa.list.seg[n_masked++] = (uint16_t)s;
    }
  }
  if (idx_out && idx_stride < max_kept) return CATEKV_ERR_INVALID_ARG;
  const EvWs W = ev_ws_layout(n, max_cap);
  if (ws_bytes < W.bytes) return CATEKV_ERR_WORKSPACE;
  cudaStream_t st = (cudaStream_t)stream;
  uint8_t* w8 = (uint8_t*)ws;
  sa.seg_off = src->seg_off_dev;
  sa.seg_len = src->seg_len_dev;
  sa.weights = weights;
  sa.segs = (EvSeg*)(w8 + W.off_segs);
  sa.idx = (int32_t*)(w8 + W.off_idx);
  sa.idx_stride = W.stride;
  sa.chk = checked_status_ptr();
  rc = evict_attributes();
  if (rc) return rc;
  if (n_masked > 0) {
    rc = launch_evict_select(sa, n_masked, max_masked, st);
    if (rc) return rc;
  }
  ma.segs = sa.segs;
  ma.src_len = src->seg_len_dev;
  ma.idx = sa.idx;
  ma.idx_stride = W.stride;
  ma.k_src = (const uint8_t*)src->k_pool;
  ma.v_src = (const uint8_t*)src->v_pool;
  ma.src_off = src->seg_off_dev;
  ma.w_src = weights;
  ma.k_dst = (uint8_t*)dst->k_pool;
  ma.v_dst = (uint8_t*)dst->v_pool;
  ma.dst_off = dst->seg_off_dev;
  ma.dst_cap = dst->seg_cap_dev;
  ma.dst_len = dst->seg_len_dev;
  ma.w_dst = dst_weights;
  ma.idx_out = idx_out;
  ma.idx_out_stride = idx_stride;
  ma.status = (int32_t*)(w8 + W.off_status);
  ma.chk = checked_status_ptr();
  ma.rows_per_cta = 0;
  if (in_place) {
    EvInArgs ia;
    ia.m = ma;
    ia.n_masked = n_masked;
    ia.list = sa.list;
    if (n_masked * 8 >= sm_count())
      CATEKV_CUDA_TRY(launch_pdl(evict_inplace_kernel<64>, dim3(n_masked * 8 + n), dim3(kEvInThreads), kEvInSmem, st, ia));
    else
      CATEKV_CUDA_TRY(launch_pdl(evict_inplace_kernel<32>, dim3(n_masked * 16 + n), dim3(kEvInThreads), kEvInSmem, st, ia));
  } else {
    // two CTAs and more for every SM's three places, up to 256 rows each
    int64_t rows = dst_rows / (6 * sm_count()) / kEvTile * kEvTile;
    ma.rows_per_cta = rows < kEvTile ? kEvTile : rows > 256 ? 256 : (int)rows;
    const int gx = max_dst_cap > 0 ? (max_dst_cap + ma.rows_per_cta - 1) / ma.rows_per_cta : 1;
    CATEKV_CUDA_TRY(launch_pdl(evict_gather_kernel, dim3(gx, n), dim3(kEvMoveThreads), kEvMoveSmem, st, ma));
  }
  for (int s = 0; s < n; ++s) dst->seg_len[s] = evict_decide(src->seg_len[s], evict_mask[s] != 0, sa.p).kept;
  if (!in_place) dst->reserved = 0;
  return CATEKV_OK;
}
