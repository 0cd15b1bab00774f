// Eviction by accumulated attention weight: candidates' weights into the top-k's score rows, top-k (select.cu), and the
// move of what is kept, into another cache or in place.
#include "decode.cuh"
#include "select.cuh"

namespace catekv {

constexpr int kEvMaxSegs = 2048;  // the mask travels in the kernel arguments
struct EvMask {
  uint32_t w[kEvMaxSegs / 32];
};

struct EvParams {
  int32_t budget, sink, local;
};
// Sizes of a segment of n rows; the same on host and device.
__host__ __device__ inline SelSeg evict_decide(int n, bool masked, const EvParams& p, int seg) {
  SelSeg s = {};
  s.n = n;
  s.job = seg;
  if (!masked || p.budget >= n || p.sink + p.local >= n) {
    s.keep_all = 1;
    s.cand_end = n;
    s.len_ub = n;
    return s;
  }
  const int rest = p.budget - p.sink - p.local;
  s.cand_end = n - p.local;
  s.n_pool = s.cand_end - p.sink;
  s.k_sel = rest > 0 ? rest : 0;
  s.len_ub = p.sink + s.k_sel + p.local;
  return s;
}

struct EvPrepArgs {
  const int32_t* seg_off;
  const int32_t* seg_len;
  const float* weights;
  SelSeg* segs;
  float* P;
  int64_t p_stride;
  EvParams p;
  EvMask mask;
};

// The decision of every segment, and the weights of its candidates as the top-k wants them: non-negative patterns, NaN as infinity.
constexpr int kEvPrepRows = 2048;
__global__ void __launch_bounds__(256) evict_prep_kernel(const __grid_constant__ EvPrepArgs a) {
  const int seg = blockIdx.y;
  pdl_launch_dependents();
  pdl_wait();
  const SelSeg s = evict_decide(a.seg_len[seg], (a.mask.w[seg >> 5] >> (seg & 31)) & 1u, a.p, seg);
  if (blockIdx.x == 0 && threadIdx.x == 0) a.segs[seg] = s;
  if (s.keep_all || s.k_sel == 0) return;
  const float* w = a.weights + a.seg_off[seg] + a.p.sink;
  float* P = a.P + (int64_t)seg * a.p_stride;
  const int c0 = blockIdx.x * kEvPrepRows + threadIdx.x;
#pragma unroll
  for (int i = 0; i < kEvPrepRows / 256; ++i) {
    const int c = c0 + i * 256;
    if (c < s.n_pool) {
      const float x = w[c];
      P[c] = x != x ? INFINITY : (x > 0.f ? x : 0.f);
    }
  }
}

struct EvMoveArgs {
  const SelSeg* segs;
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
  int64_t idx_out_stride;
  int32_t* status;
  int32_t* chk;
};

__device__ __forceinline__ int kept_row(const EvMoveArgs& a, const SelSeg& s, int seg, int r) {
  int row = s.keep_all ? r : a.idx[(int64_t)seg * a.idx_stride + r];
#ifdef CATEKV_CHECKED
  row = checked_clamp(row, 0, s.n - 1, a.chk, kKidEvict, seg);
#endif
  return row;
}

// Into another cache: a block per 64 rows of a destination segment, a warp per row (lanes 0-15 K, 16-31 V); bound by the copy's bytes.  Rows
// that a decode plan may cover are rewritten: plain launch, no early signal to dependents (see launch_pdl).
constexpr int kEvRowsPerBlock = 64;
__global__ void __launch_bounds__(256) evict_gather_kernel(const EvMoveArgs a) {
  const int seg = blockIdx.y;
  const SelSeg s = a.segs[seg];
  const int cap = a.dst_cap[seg];
  const int len = min(s.len_ub, cap);
  const int r0 = blockIdx.x * kEvRowsPerBlock;
  if (r0 == 0 && threadIdx.x == 0) {
    a.dst_len[seg] = len;
    if (s.len_ub > cap) raise_status(a.status, CATEKV_STATUS_CAPACITY, kKidEvict, seg, s.len_ub);
  }
  if (r0 >= cap) return;
  const int64_t so = a.src_off[seg], to = a.dst_off[seg];
  if (threadIdx.x < kEvRowsPerBlock) {
    const int r = r0 + threadIdx.x;
    if (r < len) {
      const int row = kept_row(a, s, seg, r);
      a.w_dst[to + r] = a.w_src[so + row];
      if (a.idx_out) a.idx_out[(int64_t)seg * a.idx_out_stride + r] = row;
    } else if (r < cap) {
      a.w_dst[to + r] = 0.f;
    }
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint8_t* src = (lane < 16 ? a.k_src : a.v_src) + so * kRowBytes + (lane & 15) * 16;
  uint8_t* dst = (lane < 16 ? a.k_dst : a.v_dst) + to * kRowBytes + (lane & 15) * 16;
  uint4 v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + warp + i * 8;
    if (r < len) v[i] = __ldg(reinterpret_cast<const uint4*>(src + (int64_t)kept_row(a, s, seg, r) * kRowBytes));
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + warp + i * 8;
    if (r < len) *reinterpret_cast<uint4*>(dst + (int64_t)r * kRowBytes) = v[i];
  }
}

// In place.  Kept row j comes from row idx[j] >= j, so a tile of destination rows may be written once the tile itself has been read: nothing
// behind it reads there.  That makes a segment sequential in its rows, so the work is split over the columns instead: 16 CTAs
// per segment, each moving 32 bytes of every row (a DRAM sector; eight CTAs K, eight V), and one that moves the weights.
constexpr int kEvSlices = 2 * kRowBytes / 32 + 1;
constexpr int kEvInThreads = 256;
constexpr int kEvInRows = 4;  // rows per thread and tile
__global__ void __launch_bounds__(kEvInThreads) evict_inplace_kernel(const EvMoveArgs a) {
  const int seg = blockIdx.x / kEvSlices, slice = blockIdx.x % kEvSlices;
  const SelSeg s = a.segs[seg];
  const int len = s.len_ub;
  const int tid = threadIdx.x;
  if (slice == kEvSlices - 1) {
    if (a.idx_out)
      for (int r = tid; r < len; r += kEvInThreads) a.idx_out[(int64_t)seg * a.idx_out_stride + r] = kept_row(a, s, seg, r);
    if (s.keep_all) return;
    float* w = a.w_dst + a.dst_off[seg];
    if (tid == 0) a.dst_len[seg] = len;
    for (int t0 = 0; t0 < len; t0 += kEvInThreads * kEvInRows) {
      float v[kEvInRows];
#pragma unroll
      for (int i = 0; i < kEvInRows; ++i) {
        const int r = t0 + tid + i * kEvInThreads;
        if (r < len) v[i] = w[kept_row(a, s, seg, r)];
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kEvInRows; ++i) {
        const int r = t0 + tid + i * kEvInThreads;
        if (r < len) w[r] = v[i];
      }
      __syncthreads();
    }
    for (int r = len + tid; r < a.dst_cap[seg]; r += kEvInThreads) w[r] = 0.f;
    return;
  }
  if (s.keep_all) return;
  constexpr int kHalf = (kEvSlices - 1) / 2;
  uint8_t* base = (slice < kHalf ? a.k_dst : a.v_dst) + (int64_t)a.dst_off[seg] * kRowBytes + (slice % kHalf) * 32;
  for (int t0 = 0; t0 < len; t0 += kEvInThreads * kEvInRows) {
    uint4 v[kEvInRows][2];
    int row[kEvInRows];
#pragma unroll
    for (int i = 0; i < kEvInRows; ++i) {
      const int r = t0 + tid + i * kEvInThreads;
      row[i] = r < len ? kept_row(a, s, seg, r) : r;
      if (row[i] != r) {
        const uint4* p = reinterpret_cast<const uint4*>(base + (int64_t)row[i] * kRowBytes);
        v[i][0] = p[0];
        v[i][1] = p[1];
      }
    }
    __syncthreads();  // the tile has been read
#pragma unroll
    for (int i = 0; i < kEvInRows; ++i) {
      const int r = t0 + tid + i * kEvInThreads;
      if (row[i] != r) {
        uint4* p = reinterpret_cast<uint4*>(base + (int64_t)r * kRowBytes);
        p[0] = v[i][0];
        p[1] = v[i][1];
      }
    }
    __syncthreads();
  }
}

struct EvWs {
  size_t off_status, off_segs, off_len, off_P, off_idx, bytes;
  int64_t stride;
};
static EvWs ev_ws_layout(int n_segs, int max_cap) {
  EvWs w;
  w.stride = (int64_t)align_up((size_t)(max_cap > 0 ? max_cap : 1), 64);
  size_t o = 0;
  w.off_status = o; o = CATEKV_STATUS_BYTES;
  w.off_segs = o; o = align_up(o + sizeof(SelSeg) * (size_t)n_segs, 256);
  w.off_len = o; o = align_up(o + sizeof(int32_t) * (size_t)n_segs, 256);
  w.off_P = o; o = align_up(o + sizeof(float) * (size_t)n_segs * w.stride, 256);
  w.off_idx = o; o = align_up(o + sizeof(int32_t) * (size_t)n_segs * w.stride, 256);
  w.bytes = o;
  return w;
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
  for (int s = 0; s < src->B * src->Hkv; ++s) lens_out[s] = evict_decide(src->seg_len[s], evict_mask[s] != 0, p, s).len_ub;
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
  const bool in_place = src == dst;
  if (in_place != (weights == dst_weights)) return CATEKV_ERR_INVALID_ARG;
  if (!in_place && (src->k_pool == dst->k_pool || src->v_pool == dst->v_pool || src->seg_len == dst->seg_len ||
                    src->seg_len_dev == dst->seg_len_dev))
    return CATEKV_ERR_INVALID_ARG;
  const int n = src->B * src->Hkv;
  if (n > kEvMaxSegs) return CATEKV_ERR_UNSUPPORTED;
  EvPrepArgs pa = {};
  pa.p = EvParams{budget, sink, local};
  int max_cap = 0, max_dst_cap = 0, max_kept = 0, n_masked = 0;
  for (int s = 0; s < n; ++s) {
    const int kept = evict_decide(src->seg_len[s], evict_mask[s] != 0, pa.p, s).len_ub;
    if (kept > dst->seg_cap[s]) return CATEKV_ERR_CAPACITY;
    max_kept = kept > max_kept ? kept : max_kept;
    max_cap = src->seg_cap[s] > max_cap ? src->seg_cap[s] : max_cap;
    max_dst_cap = dst->seg_cap[s] > max_dst_cap ? dst->seg_cap[s] : max_dst_cap;
    if (evict_mask[s]) {
      pa.mask.w[s >> 5] |= 1u << (s & 31);
      ++n_masked;
    }
  }
  if (idx_out && idx_stride < max_kept) return CATEKV_ERR_INVALID_ARG;
  const EvWs W = ev_ws_layout(n, max_cap);
  if (ws_bytes < W.bytes) return CATEKV_ERR_WORKSPACE;
  cudaStream_t st = (cudaStream_t)stream;
  uint8_t* w8 = (uint8_t*)ws;
  pa.seg_off = src->seg_off_dev;
  pa.seg_len = src->seg_len_dev;
  pa.weights = weights;
  pa.segs = (SelSeg*)(w8 + W.off_segs);
  pa.P = (float*)(w8 + W.off_P);
  pa.p_stride = W.stride;
  const int gx = max_cap > 0 ? (max_cap + kEvPrepRows - 1) / kEvPrepRows : 1;
  CATEKV_CUDA_TRY(launch_pdl(evict_prep_kernel, dim3(gx, n), dim3(256), 0, st, pa));
  TopkArgs ta = {};
  ta.segs = pa.segs;
  ta.C = pa.P;
  ta.P = pa.P;
  ta.c_stride = W.stride;
  ta.idx = (int32_t*)(w8 + W.off_idx);
  ta.idx_stride = W.stride;
  ta.seg_len_dev = (int32_t*)(w8 + W.off_len);
  ta.sink = sink;
  ta.pool_mode = kPoolPrescored;
  ta.pool_param = 1;
  ta.row_is_seg = 1;
  ta.raw_scores = 1;
  rc = launch_topk(ta, n, max_cap, n_masked, st);
  if (rc) return rc;
  EvMoveArgs ma;
  ma.segs = pa.segs;
  ma.idx = ta.idx;
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
  if (in_place)
    evict_inplace_kernel<<<n * kEvSlices, kEvInThreads, 0, st>>>(ma);
  else
    evict_gather_kernel<<<dim3(max_dst_cap > 0 ? (max_dst_cap + kEvRowsPerBlock - 1) / kEvRowsPerBlock : 1, n), 256, 0, st>>>(ma);
  CATEKV_CUDA_TRY(cudaGetLastError());
  for (int s = 0; s < n; ++s) dst->seg_len[s] = evict_decide(src->seg_len[s], evict_mask[s] != 0, pa.p, s).len_ub;
  if (!in_place) dst->reserved = 0;
  return CATEKV_OK;
}
