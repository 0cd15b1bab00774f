// The 8-bit cache: quantisation of a bf16 cache, append, the host mirror.
//
// Codes.  x M / a is rounded as the real number it is, although it is computed with a reciprocal in fp32: x and a are
// bf16 numbers, so in units of powers of two x M / a is n M / d with integers n, d < 2^8, and a border T between two
// codes is an integer of at most 9 bits (int8: k + 1/2) or 5 bits (e4m3: half-way between 4-bit numbers).  If n M / d is
// not T then the two differ by at least 1 in an integer of at most 254 * 255, i.e. by 2^-16 of their size.  The
// product x * (M / a) is off by at most 2^-22; rounded to 20 significant bits it becomes T exactly where the quotient
// is T, and stays on its side of T (2^-20 + 2^-22 < 2^-16) where it is not.  The final conversion then sees what the
// exact quotient would have shown it.
#include "q8.cuh"

namespace catekv {

constexpr int kQ8Threads = 256;
constexpr int kQ8PairsPerThread = kQ8Block * (kD / 16) / kQ8Threads;  // 16 elements (32 bytes of bf16) per step and thread: 2
constexpr float kQ8Small = 7.8886090522101181e-31f;   // 2^-100: below it M / a could overflow
constexpr float kQ8SmallUp = 1.2676506002282294e30f;  // 2^100

// largest |x| pattern of two bf16 in a word, per half
__device__ __forceinline__ uint32_t absmax_step(uint32_t m, uint32_t w) { return __vmaxu2(m, w & 0x7fff7fffu); }

template <int kType>
__device__ __forceinline__ uint32_t q8_encode4(const float (&r)[4]) {
  if (kType == CATEKV_Q8_E4M3) {
    uint32_t w;
    asm("{\n .reg .b16 a, b;\n cvt.rn.satfinite.e4m3x2.f32 a, %2, %1;\n cvt.rn.satfinite.e4m3x2.f32 b, %4, %3;\n mov.b32 %0, {a, b};\n}\n"
        : "=r"(w)
        : "f"(r[0]), "f"(r[1]), "f"(r[2]), "f"(r[3]));
    return w;
  } else {
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = __float_as_uint(r[i] + 12582912.f);  // 1.5 2^23: the low byte is the rounded integer
    return __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
  }
}

// Encode one block by the whole CTA: `k`, `v` hold this thread's 16-element runs (run p = tid + i * kQ8Threads of the
// block's 512: row p / 8, elements 16 (p % 8) ...).
template <int kType>
__device__ __forceinline__ void q8_encode_block(const uint4 (&k)[kQ8PairsPerThread][2], const uint4 (&v)[kQ8PairsPerThread][2],
                                                uint8_t* k_out, uint8_t* v_out, float* k_scale, float* v_scale,
                                                uint32_t (*s_max)[2]) {
  const int tid = threadIdx.x;
  uint32_t mk = 0, mv = 0;
#pragma unroll
  for (int i = 0; i < kQ8PairsPerThread; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      mk = absmax_step(absmax_step(absmax_step(absmax_step(mk, k[i][h].x), k[i][h].y), k[i][h].z), k[i][h].w);
      mv = absmax_step(absmax_step(absmax_step(absmax_step(mv, v[i][h].x), v[i][h].y), v[i][h].z), v[i][h].w);
    }
  mk = __reduce_max_sync(0xffffffffu, max(mk & 0xffffu, mk >> 16));
  mv = __reduce_max_sync(0xffffffffu, max(mv & 0xffffu, mv >> 16));
  if ((tid & 31) == 0) {
    s_max[tid >> 5][0] = mk;
    s_max[tid >> 5][1] = mv;
  }
  __syncthreads();
  mk = mv = 0;
#pragma unroll
  for (int w = 0; w < kQ8Threads / 32; ++w) {
    mk = max(mk, s_max[w][0]);
    mv = max(mv, s_max[w][1]);
  }
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const uint32_t m = t ? mv : mk;
    const float a = __uint_as_float(m << 16);
    const bool finite = m < 0x7f80u;
    const bool small = a < kQ8Small;
    const float inv = a > 0.f && finite ? __fdiv_rn(q8_top<kType>(), small ? a * kQ8SmallUp : a) : 0.f;
    if (tid == 0) *(t ? v_scale : k_scale) = finite ? __fdiv_rn(a, q8_top<kType>()) : __uint_as_float(0x7fc00000u);
#pragma unroll
    for (int i = 0; i < kQ8PairsPerThread; ++i) {
      const uint4 x0 = t ? v[i][0] : k[i][0], x1 = t ? v[i][1] : k[i][1];
      const uint32_t w[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
      uint32_t c[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float r[4] = {__uint_as_float(w[2 * j] << 16), __uint_as_float(w[2 * j] & 0xffff0000u),
                      __uint_as_float(w[2 * j + 1] << 16), __uint_as_float(w[2 * j + 1] & 0xffff0000u)};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (!finite) r[e] = 0.f;
          if (small) r[e] *= kQ8SmallUp;
          r[e] = __uint_as_float((__float_as_uint(r[e] * inv) + 8u) & ~15u);  // to 20 significant bits
        }
        c[j] = q8_encode4<kType>(r);
      }
      *reinterpret_cast<uint4*>((t ? v_out : k_out) + (size_t)(tid + i * kQ8Threads) * 16) = make_uint4(c[0], c[1], c[2], c[3]);
    }
  }
}

struct QuantizeArgs {
  const uint8_t* k_src;
  const uint8_t* v_src;
  const int32_t* src_off;
  const int32_t* src_len;
  uint8_t* k_pool;
  uint8_t* v_pool;
  float* k_scale;
  float* v_scale;
  uint8_t* k_tail;
  uint8_t* v_tail;
  const int32_t* seg_off;
  int32_t* seg_len;
  int32_t seg0;  // the launch's first segment
};
// The capacities of a launch's segments travel in the kernel arguments (the 8-bit cache has none on the device): the device's lengths
// decide, which in a replayed graph may be longer than the host saw them.  Two sizes, as the longer one is 8 KB of arguments.
constexpr int kQ8FewSegs = 128, kQ8MostSegs = 2048;
template <int kSegs>
struct QuantizeCaps {
  int32_t cap[kSegs];
};

// One CTA per block of a segment (the last one takes the tail's rows), the block in registers between the maximum and the
// codes: one pass, bound by the copy's bytes (128K, 458 MB: 74 us in a replayed graph, 6.1 TB/s, 0.95 of the copy
// bandwidth).  The grid is as long as the host's longest list; where the device's is longer its CTAs go round again.
// It rewrites blocks that a decode plan may cover: launched without the programmatic attribute, no early
// signal to dependents (see launch_pdl).
template <int kType>
__device__ __forceinline__ void q8_quantize_block(const QuantizeArgs& a, int seg, int blk, int len, uint32_t (*s_max)[2]) {
  const int tid = threadIdx.x;
  const int full = len / kQ8Block;
  const int64_t row0 = (int64_t)a.src_off[seg] + (int64_t)blk * kQ8Block;
  const uint8_t* ks = a.k_src + row0 * kRowBytes;
  const uint8_t* vs = a.v_src + row0 * kRowBytes;
  uint4 k[kQ8PairsPerThread][2], v[kQ8PairsPerThread][2];
  const int rows = len - blk * kQ8Block;
#pragma unroll
  for (int i = 0; i < kQ8PairsPerThread; ++i) {
    const int p = tid + i * kQ8Threads;
    const bool ok = p / 8 < rows;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      k[i][h] = ok ? __ldg(reinterpret_cast<const uint4*>(ks + (size_t)p * 32) + h) : make_uint4(0, 0, 0, 0);
      v[i][h] = ok ? __ldg(reinterpret_cast<const uint4*>(vs + (size_t)p * 32) + h) : make_uint4(0, 0, 0, 0);
    }
  }
  if (blk == full) {
    const size_t base = (size_t)seg * kQ8Block * kRowBytes;
#pragma unroll
    for (int i = 0; i < kQ8PairsPerThread; ++i) {
      const int p = tid + i * kQ8Threads;
      if (p / 8 < rows)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          reinterpret_cast<uint4*>(a.k_tail + base + (size_t)p * 32)[h] = k[i][h];
          reinterpret_cast<uint4*>(a.v_tail + base + (size_t)p * 32)[h] = v[i][h];
        }
    }
    return;
  }
  const int64_t dblk = a.seg_off[seg] / kQ8Block + blk;
  q8_encode_block<kType>(k, v, a.k_pool + dblk * kQ8BlockBytes, a.v_pool + dblk * kQ8BlockBytes, a.k_scale + dblk,
                         a.v_scale + dblk, s_max);
}

template <int kType, int kSegs>
__global__ void __launch_bounds__(kQ8Threads) q8_quantize_kernel(const QuantizeArgs a, const __grid_constant__ QuantizeCaps<kSegs> caps) {
  __shared__ uint32_t s_max[kQ8Threads / 32][2];
  const int seg = a.seg0 + blockIdx.y;
  const int len = min(a.src_len[seg], caps.cap[blockIdx.y]);
  if (blockIdx.x == 0 && threadIdx.x == 0) a.seg_len[seg] = len;
  const int end = (len + kQ8Block - 1) / kQ8Block;
  for (int blk = blockIdx.x; blk < end; blk += gridDim.x) {
    if (blk != (int)blockIdx.x) __syncthreads();  // s_max has been read
    q8_quantize_block<kType>(a, seg, blk, len, s_max);
  }
}

template <int kType, int kSegs>
static cudaError_t q8_launch_quantize(QuantizeArgs a, const int32_t* seg_cap, int n, int gx, cudaStream_t st) {
  for (a.seg0 = 0; a.seg0 < n; a.seg0 += kSegs) {
    QuantizeCaps<kSegs> caps;  // (entries behind the last segment are not looked at)
    const int m = n - a.seg0 < kSegs ? n - a.seg0 : kSegs;
    for (int s = 0; s < m; ++s) caps.cap[s] = seg_cap[a.seg0 + s];
    q8_quantize_kernel<kType, kSegs><<<dim3(gx, m), kQ8Threads, 0, st>>>(a, caps);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}
template <int kType>
static cudaError_t q8_launch_quantize(const QuantizeArgs& a, const int32_t* seg_cap, int n, int gx, cudaStream_t st) {
  return n <= kQ8FewSegs ? q8_launch_quantize<kType, kQ8FewSegs>(a, seg_cap, n, gx, st)
                         : q8_launch_quantize<kType, kQ8MostSegs>(a, seg_cap, n, gx, st);
}

struct Q8AppendArgs {
  uint8_t* k_pool;
  uint8_t* v_pool;
  float* k_scale;
  float* v_scale;
  uint8_t* k_tail;
  uint8_t* v_tail;
  const int32_t* seg_off;
  int32_t* seg_len;
  const uint8_t* k_new;
  const uint8_t* v_new;
};

// One CTA per segment: the row goes to the tail; a CTA whose block it completes encodes the block (63 rows of the tail and
// the new one).  Bound by launch latency.  The block it writes lies behind every block that was complete when a plan was
// built: dependents may start early.
template <int kType>
__global__ void __launch_bounds__(kQ8Threads) q8_append_kernel(const Q8AppendArgs a) {
  __shared__ uint32_t s_max[kQ8Threads / 32][2];
  const int seg = blockIdx.x, tid = threadIdx.x;
  pdl_launch_dependents();
  pdl_wait();
  const int len = a.seg_len[seg];
  const int at = len % kQ8Block;
  __syncthreads();  // every thread has the length before it changes
  const size_t base = (size_t)seg * kQ8Block * kRowBytes;
  if (at == kQ8Block - 1) {
    uint4 k[kQ8PairsPerThread][2], v[kQ8PairsPerThread][2];
#pragma unroll
    for (int i = 0; i < kQ8PairsPerThread; ++i) {
      const int p = tid + i * kQ8Threads, r = p / 8;
      const bool fresh = r == at;
      const uint8_t* ks = fresh ? a.k_new + (size_t)seg * kRowBytes + (p % 8) * 32 : a.k_tail + base + (size_t)p * 32;
      const uint8_t* vs = fresh ? a.v_new + (size_t)seg * kRowBytes + (p % 8) * 32 : a.v_tail + base + (size_t)p * 32;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        k[i][h] = reinterpret_cast<const uint4*>(ks)[h];
        v[i][h] = reinterpret_cast<const uint4*>(vs)[h];
      }
    }
    const int64_t dblk = a.seg_off[seg] / kQ8Block + len / kQ8Block;
    q8_encode_block<kType>(k, v, a.k_pool + dblk * kQ8BlockBytes, a.v_pool + dblk * kQ8BlockBytes, a.k_scale + dblk,
                           a.v_scale + dblk, s_max);
  }
  if (tid < 32) {
    const uint8_t* src = (tid < 16 ? a.k_new : a.v_new) + (size_t)seg * kRowBytes + (tid & 15) * 16;
    uint8_t* dst = (tid < 16 ? a.k_tail : a.v_tail) + base + (size_t)at * kRowBytes + (tid & 15) * 16;
    *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(src);
  }
  if (tid == 0) a.seg_len[seg] = len + 1;
}

}  // namespace catekv

using namespace catekv;

extern "C" int catekv_q8_quantize(const catekv_cache* src, catekv_q8_cache* dst, catekv_stream stream) {
  CATEKV_API_RANGE();
  int rc = check_cache(src);
  if (rc) return rc;
  rc = check_q8_cache(dst);
  if (rc) return rc;
  if (src->pages) return CATEKV_ERR_UNSUPPORTED;
  // lengths that are upper bounds would make plans count blocks as complete that are not
  if (src->reserved) return CATEKV_ERR_INVALID_ARG;
  if (((uintptr_t)src->k_pool | (uintptr_t)src->v_pool) & 15) return CATEKV_ERR_INVALID_ARG;
  if (src->B != dst->B || src->Hkv != dst->Hkv) return CATEKV_ERR_INVALID_ARG;
  const int n = src->B * src->Hkv;
  if (n > 65535) return CATEKV_ERR_UNSUPPORTED;
  int max_len = 0;
  for (int s = 0; s < n; ++s) {
    if (src->seg_len[s] < 0 || src->seg_len[s] > src->seg_cap[s]) return CATEKV_ERR_INVALID_ARG;
    if (src->seg_len[s] > dst->seg_cap[s]) return CATEKV_ERR_CAPACITY;
    max_len = src->seg_len[s] > max_len ? src->seg_len[s] : max_len;
  }
  QuantizeArgs a;
  a.k_src = (const uint8_t*)src->k_pool;
  a.v_src = (const uint8_t*)src->v_pool;
  a.src_off = src->seg_off_dev;
  a.src_len = src->seg_len_dev;
  a.k_pool = (uint8_t*)dst->k_pool;
  a.v_pool = (uint8_t*)dst->v_pool;
  a.k_scale = dst->k_scale;
  a.v_scale = dst->v_scale;
  a.k_tail = (uint8_t*)dst->k_tail;
  a.v_tail = (uint8_t*)dst->v_tail;
  a.seg_off = dst->seg_off_dev;
  a.seg_len = dst->seg_len_dev;
  a.seg0 = 0;
  const int gx = max_len > 0 ? (max_len + kQ8Block - 1) / kQ8Block : 1;
  if (dst->dtype == CATEKV_Q8_E4M3)
    CATEKV_CUDA_TRY(q8_launch_quantize<CATEKV_Q8_E4M3>(a, dst->seg_cap, n, gx, (cudaStream_t)stream));
  else
    CATEKV_CUDA_TRY(q8_launch_quantize<CATEKV_Q8_INT8>(a, dst->seg_cap, n, gx, (cudaStream_t)stream));
  for (int s = 0; s < n; ++s) dst->seg_len[s] = src->seg_len[s];
  return CATEKV_OK;
}

extern "C" int catekv_q8_append(catekv_q8_cache* cache, const void* k_new, const void* v_new, catekv_stream stream) {
  CATEKV_API_RANGE();
  int rc = check_q8_cache(cache);
  if (rc) return rc;
  if (!k_new || !v_new || (((uintptr_t)k_new | (uintptr_t)v_new) & 15)) return CATEKV_ERR_INVALID_ARG;
  const int n = cache->B * cache->Hkv;
  for (int s = 0; s < n; ++s) {
    if (cache->seg_len[s] < 0) return CATEKV_ERR_INVALID_ARG;
    if (cache->seg_len[s] + 1 > cache->seg_cap[s]) return CATEKV_ERR_CAPACITY;
  }
  Q8AppendArgs a;
  a.k_pool = (uint8_t*)cache->k_pool;
  a.v_pool = (uint8_t*)cache->v_pool;
  a.k_scale = cache->k_scale;
  a.v_scale = cache->v_scale;
  a.k_tail = (uint8_t*)cache->k_tail;
  a.v_tail = (uint8_t*)cache->v_tail;
  a.seg_off = cache->seg_off_dev;
  a.seg_len = cache->seg_len_dev;
  a.k_new = (const uint8_t*)k_new;
  a.v_new = (const uint8_t*)v_new;
  if (cache->dtype == CATEKV_Q8_E4M3)
    CATEKV_CUDA_TRY(launch_pdl(q8_append_kernel<CATEKV_Q8_E4M3>, dim3(n), dim3(kQ8Threads), 0, (cudaStream_t)stream, a));
  else
    CATEKV_CUDA_TRY(launch_pdl(q8_append_kernel<CATEKV_Q8_INT8>, dim3(n), dim3(kQ8Threads), 0, (cudaStream_t)stream, a));
  for (int s = 0; s < n; ++s) cache->seg_len[s] += 1;
  return CATEKV_OK;
}

extern "C" int catekv_q8_cache_advance(catekv_q8_cache* cache, int32_t n_tokens) {
  int rc = check_q8_cache(cache);
  if (rc) return rc;
  if (n_tokens < 0) return CATEKV_ERR_INVALID_ARG;
  const int n = cache->B * cache->Hkv;
  for (int s = 0; s < n; ++s)
    if ((int64_t)cache->seg_len[s] + n_tokens > cache->seg_cap[s]) return CATEKV_ERR_CAPACITY;
  for (int s = 0; s < n; ++s) cache->seg_len[s] += n_tokens;
  return CATEKV_OK;
}
