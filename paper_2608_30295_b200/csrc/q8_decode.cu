// Decode attention over the 8-bit cache: split-KV partials on the tensor cores, and their merge.
//
// Bound by the stream of codes (256 bytes a row) where a CTA's share is long, by latency and MMA issue where it is short.  Measured, whole call in
// a replayed graph: 16 x 64K (1.09 GB) 158 us, 6.9 TB/s or 1.07 of the copy bandwidth; 128K x 3 heads int8 (93 MB) 18.9 us, 4.9 TB/s, of which 18.2
// remain when nothing is computed; 256K x 2 heads, G = 7 (136 MB) 27.0 us; 4K (4.5 MB) 7.5 us.
//
// The stream is a warp's own.  A CTA owns a contiguous range of the rows of all segments laid end to end (cut at block
// borders); its four warps take the range's units in turn, a unit being half a block (32 rows of codes, 8 KB of K and V)
// or 16 rows of a bf16 tail (8 KB as well).  Each warp keeps a ring of units in flight with cp.async and waits for no
// other warp before a segment's piece is merged.
//
// Codes are f16 numbers, so both products run on mma.m16n8k16 (f16) with the code converted in registers; tokens are M,
// the group's <= 8 query heads N.  Which token or which d a fragment slot stands for is free as long as both operands of
// a product agree, and is chosen so that every shared-memory access is a conflict-free 16-byte load and nothing is
// transposed in memory:
//   S = K Q^T   row g of A is token pi(g) = g ^ 4 (g & 1) of the 16; thread (g, c) takes the 16-byte chunks c and c + 4
//               of its rows, word i of chunk c + 4h is k-step 4h + i (Q's fragments are gathered to match);
//   O^T = V^T P row g of A holds d = 16 g + 2 j (+ 1 in row g + 8) of MMA j; thread (g, c) takes chunk g of tokens 2c,
//               (2c+1)^4 and these + 8 (the columns that P's transposed fragment has), and interleaves their bytes in
//               registers.
// Q enters as f16 under a power of two per head (bf16 has fewer bits than f16: exact except where an element is 2^-29 of
// the head's largest); the scale of a block multiplies its logits.  Probabilities are formed against the running maximum
// times 2^12 and split into an f16 hi + lo pair (22 bits).  The tensor cores cut their fp32 sums off instead of rounding
// them: chains are kept short (four MMAs), a unit's P V product is formed from zero and enters the accumulators by one
// rounded multiply-add each, which also applies the block's V scale (1.3e-6 -> 4e-7 against 64 bits).
#include <math.h>

#include <atomic>

#include "q8.cuh"

namespace catekv {

constexpr int kQ8Warps = 4;
constexpr int kQ8DecodeThreads = kQ8Warps * 32;
constexpr int kQ8Regs = 224;  // a thread: leaves 8 K of an SM to the combine kernel beside two CTAs
constexpr int kQ8Unit = 32;                              // rows of codes in a unit
constexpr int kQ8TailUnit = 16;                          // rows of a tail in a unit
constexpr int kQ8UnitBytes = 2 * kQ8Unit * kQ8RowBytes;  // K, then V
static_assert(kQ8UnitBytes == 2 * kQ8TailUnit * kRowBytes, "both kinds of unit fill a stage");
constexpr int kQ8SlotFloats = kMaxG * kD;                // a slot of the merge: [8 heads][128 d]
constexpr int q8_decode_smem(int stages) { return kQ8Warps * stages * kQ8UnitBytes + 2 * kQ8SlotFloats * 4; }
// Units a warp has requested or under way: three while a CTA's share is short, where the ramp counts (1.8 K rows, G = 4:
// 25 us against 26), two for long shares, where more requests than needed only disturb the order in which memory serves
// them (14 K rows, G = 4, either type: 157 us against 166; 7 K rows: 83 against 86; equal at 3.5 K).  int8 codes for more
// than four heads are converted and multiplied slowly enough for three at any length (14 K rows, G = 7: 158 us against
// 161; e4m3 there 171 against 158).
constexpr int kQ8LongShare = 4096;
// Segments of up to kQ8MergePieces pieces are merged by the CTA that delivers the last one (16 x 1K step: 14.3 us on the
// device against 15.3, 16 x 64K 157.6 against 159.0, and one launch less for the host, 2.4 us); longer ones by a combine pass
// (18 pieces, 4 x 32K: 25.9 us against 27.0 merged in the kernel; 98 would be 200 KB through one CTA).  Where a CTA's share is
// at most kQ8MergeShare rows the call takes the host longer than the device, and the launch counts for more: up to
// kQ8MergeMost pieces then (4K lists in 32: 7.7 us on the device against 6.2, the call 7.8 against 10).
constexpr int kQ8MergePieces = 16, kQ8MergeMost = 32, kQ8MergeShare = 128;
static_assert(kQ8MergeMost <= 32, "a lane per piece");
constexpr int32_t kQ8PlanTile = kQ8Unit;   // marks a plan of this kind (decode.cu's have kTile)
constexpr int kQ8SegEndCharge = 512;       // rows (128K: 23.4 us with 0, 22.5 with 128, 21.8 with 256, 21.1 with 512)
constexpr float kQ8PBits = 12.f;           // probabilities are at most 2^12 ...
constexpr float kQ8PUnit = 1.f / 4096.f;   // ... and the accumulators in units of it
static_assert(kQ8PlanTile != kTile, "the two kinds of plan must differ");

struct Q8DecodeArgs {
  const uint8_t* k_pool;
  const uint8_t* v_pool;
  const float* k_scale;
  const float* v_scale;
  const uint8_t* k_tail;
  const uint8_t* v_tail;
  const int32_t* seg_len;
  const uint16_t* q;  // [B, Hq, d]
  int32_t Hq, Hkv, G;
  float scale_log2;  // sm_scale * log2(e)
  const CtaHeader* ctas;
  const WorkItem* items;
  float* part_o;
  float* part_lse;
  void* out;
  int32_t out_fp32;
  float* lse_out;
  SegInfo* merge;  // few pieces per segment: the CTA that delivers a segment's last piece merges them (counts in SegInfo::arrived); else null
};

__device__ __forceinline__ void mma_f16_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
  return v;
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 unpack_f16(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
// 4-byte global->shared copy
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;\n" ::"r"(dst), "l"(src));
}

// A piece of a segment as a warp sees it: `full` units of codes starting at unit u0 of the pool (of which the first `live`
// are to be attended to: the others were complete when the plan was built but no longer are), then the tail's units.
struct Q8Cursor {
  int seg, slot, np, full, live, tail, units;
  int64_t u0;
};
constexpr int kUnitsPerBlock = kQ8Block / kQ8Unit;
__device__ __forceinline__ Q8Cursor q8_plan_cursor(const WorkItem& w) {
  Q8Cursor c;
  c.seg = w.seg;
  c.slot = w.slot;
  c.u0 = w.row_base / kQ8Unit;
  // t0 is a multiple of the unit, and so is t1 of an inner piece; the last piece's units are those of complete blocks
  c.np = max(0, (w.last ? w.t1 / kQ8Block * kUnitsPerBlock : w.t1 / kQ8Unit) - w.t0 / kQ8Unit);
  c.full = c.np;
  c.live = c.np;
  c.tail = 0;
  c.units = c.np;
  return c;
}
__device__ __forceinline__ void q8_live_cursor(const WorkItem& w, int len, Q8Cursor& c) {
  int end = len / kQ8Block * kUnitsPerBlock;
  if (!w.last) end = min(end, w.t1 / kQ8Unit);
  c.live = max(0, end - w.t0 / kQ8Unit);
  c.full = max(c.np, c.live);
  c.tail = w.last ? len % kQ8Block : 0;
  c.units = c.full + (c.tail + kQ8TailUnit - 1) / kQ8TailUnit;
}
// a load that stays where it is written (the compiler would move it down to its use, behind what it is to overlap with)
__device__ __forceinline__ uint4 ldg128_here(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
// the group's queries, 4 x 16 bytes of this thread's head: d = 16 (c + 4 hh) + 8 e ... in x[2 hh + e]
__device__ __forceinline__ void q8_load_q(const Q8DecodeArgs& a, int seg, int g, int c, uint4 (&x)[4]) {  // g: the head
  const int b = seg / a.Hkv, h = seg % a.Hkv;
  const uint4* p = reinterpret_cast<const uint4*>(a.q + ((int64_t)b * a.Hq + h * a.G + g) * kD);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = make_uint4(0, 0, 0, 0);
    if (g < a.G) x[i] = ldg128_here(p + 2 * (c + 4 * (i >> 1)) + (i & 1));
  }
}
// a slot's place of (head, d): rotated by the head pair, so that a warp's 16-byte accesses fall in different banks
__device__ __forceinline__ int q8_slot(int head, int d) { return head * kD + ((d + 4 * (head >> 1)) & (kD - 1)); }
__device__ __forceinline__ WorkItem q8_load_item(const WorkItem* p) {
  const int4 x = __ldg(reinterpret_cast<const int4*>(p)), y = __ldg(reinterpret_cast<const int4*>(p) + 1);
  WorkItem w;
  w.seg = x.x; w.t0 = x.y; w.t1 = x.z; w.slot = x.w;
  w.row_base = (int64_t)(((uint64_t)(uint32_t)y.y << 32) | (uint32_t)y.x);
  w.last = y.z; w.cap = y.w;
  return w;
}

// One head of a segment from its pieces (at most 32), by a warp: a lane per piece for the weights, four dimensions per lane for the sum.
__device__ __forceinline__ void q8_merge_pieces(const Q8DecodeArgs& a, int slot, int n, int b, int h, int hd, int lane) {
  const float l = lane < n ? __ldcg(a.part_lse + (size_t)(slot + lane) * kMaxG + hd) : -INFINITY;
  const float* po = a.part_o + ((size_t)slot * kMaxG + hd) * kD + 4 * lane;
  constexpr int kFly = 16;  // pieces in flight
  float4 v[kFly];
  auto load = [&](int u0) {
#pragma unroll
    for (int u = 0; u < kFly; ++u)
      v[u] = u0 + u < n ? __ldcg(reinterpret_cast<const float4*>(po + (size_t)(u0 + u) * (kMaxG * kD))) : make_float4(0.f, 0.f, 0.f, 0.f);
  };
  load(0);  // with the LSEs: one trip to memory for up to 16 pieces
  float M = l;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  const float e = M > -INFINITY ? exp2f(l - M) : 0.f;  // an empty piece (LSE -inf) weighs 0
  float W = e;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) W += __shfl_xor_sync(0xffffffffu, W, o);
  float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int u0 = 0; u0 < n; u0 += kFly) {
    if (u0 > 0) load(u0);
#pragma unroll
    for (int u = 0; u < kFly; ++u) {
      const float w = __shfl_sync(0xffffffffu, e, u0 + u);
      r.x += w * v[u].x;
      r.y += w * v[u].y;
      r.z += w * v[u].z;
      r.w += w * v[u].w;
    }
  }
  const float inv = W == 0.f ? 0.f : 1.f / W;  // (a NaN stays one)
  r = make_float4(r.x * inv, r.y * inv, r.z * inv, r.w * inv);
  const size_t at = ((size_t)b * a.Hq + (size_t)h * a.G + hd) * kD;
  if (a.out_fp32)
    reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out) + at)[lane] = r;
  else
    reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.out) + at)[lane] = make_uint2(pack_bf16(r.x, r.y), pack_bf16(r.z, r.w));
  if (a.lse_out && lane == 0)
    a.lse_out[(size_t)b * a.Hq + (size_t)h * a.G + hd] = W == 0.f ? -INFINITY : (M + log2f(W)) * 0.6931471805599453f;
}

// kPack (groups of up to four heads): columns 4..7 of the MMAs are the same heads again, their P the low halves: one MMA
// in place of two per product of V (the kernel is short of MMA issue where a CTA's share is small: 128K x 3 heads, int8,
// 21.2 -> 19.5 us; 64 x 1K x 8 heads 28 -> 23 us).  The two halves' sums meet when a piece is merged.
template <int kType, int kQ8Stages, bool kPack>
__global__ void __maxnreg__(kQ8Regs) q8_decode_partial_kernel(const Q8DecodeArgs a) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float s_scale[kQ8Warps][kQ8Stages][2];
  // The warps' maxima and sums of a piece.  Two copies, taken in turn: a warp without a unit in the next piece writes that piece's
  // while another may still be reading this one's for its last head; the barriers of the piece between order a copy's reuse.
  __shared__ float s_ml[2][2][kQ8Warps][kMaxG];
  __shared__ int s_last;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int g = lane >> 2, c = lane & 3;
  const int pi = g ^ ((g & 1) << 2);  // token of row g
  const int gq = kPack ? g & 3 : g;   // head of column g
  const bool low_half = kPack && c >= 2;
  pdl_launch_dependents();
  int item_begin, item_end;
  WorkItem w0;
  {
    // the plan was uploaded by a copy that precedes the previous kernel: it may be read before the wait
    const int4* hp = reinterpret_cast<const int4*>(a.ctas + blockIdx.x);
    const int4 h0 = __ldg(hp);
    item_begin = h0.x;
    item_end = h0.y;
    if (item_begin >= item_end) return;
    w0 = q8_load_item(reinterpret_cast<const WorkItem*>(hp + 1));
  }
  const uint32_t ring = smem_u32(smem) + warp * (kQ8Stages * kQ8UnitBytes);
  const uint32_t ring_scale = smem_u32(&s_scale[warp][0][0]);
  float* slots = reinterpret_cast<float*>(smem + kQ8Warps * kQ8Stages * kQ8UnitBytes);

  // ---- producer side of the warp: units warp, warp + 4, ... of every item, in order
  Q8Cursor pc = q8_plan_cursor(w0);
  int p_item = item_begin, p_u = warp, p_seq = 0;
  auto issue_unit = [&]() {
    const int stage = p_seq % kQ8Stages;
    const uint32_t sb = ring + stage * kQ8UnitBytes;
    if (p_u < pc.full) {
      const int64_t unit = pc.u0 + p_u;
      const int64_t off = unit * (kQ8Unit * kQ8RowBytes) + lane * 16;
      const uint8_t* kp = a.k_pool + off;
      const uint8_t* vp = a.v_pool + off;
      // rows of 128 bytes, chunk j of row r at place j ^ (r & 7)
      const int r = lane >> 3, j = lane & 7;
      const uint32_t d0 = sb + r * kQ8RowBytes + ((j ^ r) << 4), d1 = sb + (r + 4) * kQ8RowBytes + ((j ^ (r + 4)) << 4);
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        cp_async16(d0 + i * 512, kp + i * 512, 16);
        cp_async16(d1 + i * 512, kp + i * 512 + 512, 16);
      }
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        cp_async16(d0 + 4096 + i * 512, vp + i * 512, 16);
        cp_async16(d1 + 4096 + i * 512, vp + i * 512 + 512, 16);
      }
      if (lane < 2) cp_async4(ring_scale + (stage * 2 + lane) * 4, (lane ? a.v_scale : a.k_scale) + unit / kUnitsPerBlock);
    } else {
      const int r0 = (p_u - pc.full) * kQ8TailUnit;
      const int left = pc.tail - r0;
      const size_t off = ((size_t)pc.seg * kQ8Block + r0) * kRowBytes;
#pragma unroll
      for (int i = 0; i < 8; ++i) {  // rows of 256 bytes, as tile_off
        const int r = 2 * i + (lane >> 4), j = lane & 15;
        const int ok = r < left ? 16 : 0;
        const size_t o = ok ? off + (size_t)r * kRowBytes + j * 16 : 0;
        cp_async16(sb + tile_off(r, j), a.k_tail + o, ok);
        cp_async16(sb + 4096 + tile_off(r, j), a.v_tail + o, ok);
      }
    }
    ++p_seq;
    p_u += kQ8Warps;
  };
  // What the item behind the consumer's is made of, requested one item ahead: neither side waits for a chain of loads then.
  WorkItem nx;
  int nx_len = 0;
  int nx_item = item_begin;  // the item that these belong to
  auto prefetch_item = [&](int item, int seg) {  // items after a CTA's first belong to consecutive segments
    nx_item = item;
    if (item < item_end) {
      nx = q8_load_item(a.items + item);
      nx_len = *reinterpret_cast<const volatile int32_t*>(a.seg_len + seg);
    }
  };
  auto skip_done = [&]() {  // on to the next item that has a unit for this warp
    while (p_item < item_end && p_u >= pc.units) {
      p_u = warp;
      if (++p_item < item_end) {
        if (p_item == nx_item) {
          pc = q8_plan_cursor(nx);
          q8_live_cursor(nx, nx_len, pc);
        } else {
          const WorkItem w = q8_load_item(a.items + p_item);
          pc = q8_plan_cursor(w);
          q8_live_cursor(w, *reinterpret_cast<const volatile int32_t*>(a.seg_len + w.seg), pc);
        }
      }
    }
  };
  auto issue = [&]() {  // one unit, if any is left, = one commit group
    if (p_item < item_end) {
      issue_unit();
      skip_done();
    }
    cp_async_commit();
  };

  // Blocks that were complete when the plan was built are older than anything the previous kernel of the stream may still
  // be writing (an append writes behind them): the first units are requested before the wait.
  int pre = 0;
  for (; pre < kQ8Stages - 1 && p_u < pc.np; ++pre) {
    issue_unit();
    cp_async_commit();
  }
  pdl_wait();  // from here on: lengths, queries, and rows written by earlier kernels
  uint4 q4[4];
  q8_load_q(a, w0.seg, gq, c, q4);
  const int len0 = *reinterpret_cast<const volatile int32_t*>(a.seg_len + w0.seg);
  prefetch_item(item_begin + 1, w0.seg + 1);
  q8_live_cursor(w0, len0, pc);
  Q8Cursor cc = pc;
  skip_done();
  for (; pre < kQ8Stages - 1; ++pre) issue();

  int seq = 0;
  for (int item = item_begin; item < item_end; ++item) {
    if (item > item_begin) {
      cc = q8_plan_cursor(nx);
      q8_live_cursor(nx, nx_len, cc);
      prefetch_item(item + 1, cc.seg + 1);
    }
    const int b = cc.seg / a.Hkv, h = cc.seg % a.Hkv;
    // ---- the group's queries as B fragments: k-step 4 hh + i holds d = 16 (c + 4 hh) + 4 i + 0..3 of head g
    uint32_t qf[8][2];
    float f0, f1;  // logits of heads 2c, 2c + 1 = accumulators times these (times the block's scale)
    {
      uint32_t qb[8][2];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        qb[2 * i][0] = q4[i].x;
        qb[2 * i][1] = q4[i].y;
        qb[2 * i + 1][0] = q4[i].z;
        qb[2 * i + 1][1] = q4[i].w;
      }
      uint32_t mx = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) mx = __vmaxu2(__vmaxu2(mx, qb[i][0] & 0x7fff7fffu), qb[i][1] & 0x7fff7fffu);
      mx = max(mx & 0xffffu, mx >> 16);
      mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
      mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
      const int E = max((int)(mx >> 7), 15);  // exponent field of the head's largest |q|: it becomes 2^14 .. 2^15
      const float up = __int_as_float((268 - E) << 23), down = __int_as_float((E - 14) << 23);
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int r = 0; r < 2; ++r)
          qf[i][r] = pack_f16(__uint_as_float(qb[i][r] << 16) * up, __uint_as_float(qb[i][r] & 0xffff0000u) * up);
      f0 = __shfl_sync(0xffffffffu, down, 8 * c) * a.scale_log2;
      f1 = __shfl_sync(0xffffffffu, down, 8 * c + 4) * a.scale_log2;
    }
    float o[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
    // new maxima: what the sums so far are multiplied with
    auto rescale = [&](float mx0, float mx1) {
#pragma unroll
      for (int sh = 4; sh <= 16; sh <<= 1) {
        mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, sh));
        mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, sh));
      }
      const float mn0 = fmaxf(m0, mx0), mn1 = fmaxf(m1, mx1);
      if (__any_sync(0xffffffffu, mn0 > m0 || mn1 > m1)) {
        // exp2(-inf) = 0 on the first unit; a head whose logits have all been -inf (an infinite key) stays as it is
        const float al0 = mn0 > m0 ? fast_exp2(m0 - mn0) : 1.f, al1 = mn1 > m1 ? fast_exp2(m1 - mn1) : 1.f;
        l0 *= al0;
        l1 *= al1;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          o[i][0] *= al0;
          o[i][1] *= al1;
          o[i][2] *= al0;
          o[i][3] *= al1;
        }
        m0 = mn0;
        m1 = mn1;
      }
    };

    for (int u = warp; u < cc.units; u += kQ8Warps, ++seq) {
      cp_async_wait<kQ8Stages - 2>();
      __syncwarp();
      issue();  // into the stage that the previous unit has left
      const int stage = seq % kQ8Stages;
      const uint32_t kb = ring + stage * kQ8UnitBytes, vb = kb + 4096;
      if (u < cc.full) {
        if (u >= cc.live) continue;
        const float ks = s_scale[warp][stage][0], vs = s_scale[warp][stage][1] * kQ8PUnit;
        // ---- S[32 tokens x 8 heads] = K Q^T, the two halves of d apart
        float sh[2][2][4];
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const uint32_t ra = kb + (16 * t + pi) * kQ8RowBytes + (((c + 4 * hh) ^ (pi & 7)) << 4);
            const uint4 lo = lds128(ra), hi = lds128(ra + 8 * kQ8RowBytes);
#pragma unroll
            for (int i = 0; i < 4; ++i) sh[t][hh][i] = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t a0, a1, a2, a3;
              q8_to_f16<kType>(word(lo, i), a0, a2);
              q8_to_f16<kType>(word(hi, i), a1, a3);
              mma_f16_16816(sh[t][hh], a0, a1, a2, a3, qf[4 * hh + i][0], qf[4 * hh + i][1]);
            }
          }
        float s[2][4];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[t][i] = sh[t][0][i] + sh[t][1][i];
        // s[t][0], s[t][1]: token 16 t + pi(g), heads 2c, 2c + 1;  s[t][2], s[t][3]: that token + 8
        const float k0 = f0 * ks, k1 = f1 * ks;
        float x[2][4];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          x[t][0] = s[t][0] * k0;
          x[t][1] = s[t][1] * k1;
          x[t][2] = s[t][2] * k0;
          x[t][3] = s[t][3] * k1;
        }
        rescale(fmaxf(fmaxf(x[0][0], x[0][2]), fmaxf(x[1][0], x[1][2])), fmaxf(fmaxf(x[0][1], x[0][3]), fmaxf(x[1][1], x[1][3])));
        const float r0 = m0 > -INFINITY ? kQ8PBits - m0 : 0.f, r1 = m1 > -INFINITY ? kQ8PBits - m1 : 0.f;
        uint32_t bh[2][2], bl[2][2];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float p0 = fast_exp2(x[t][2 * e] + r0), p1 = fast_exp2(x[t][2 * e + 1] + r1);
            l0 += p0;
            l1 += p1;
            const uint32_t hi = pack_f16(p0, p1);
            const float2 hf = unpack_f16(hi);
            const uint32_t lo = pack_f16(p0 - hf.x, p1 - hf.y);
            bh[t][e] = movmatrix_trans(low_half ? lo : hi);
            if (!kPack) bl[t][e] = movmatrix_trans(lo);
          }
        // ---- O^T[128 d x 8 heads] += V^T P
        uint4 v[2][4];  // tokens 2c, (2c + 1) ^ 4, these + 8 of each half
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int t0 = 16 * t + 2 * c, t1 = 16 * t + ((2 * c + 1) ^ 4);
          const uint32_t ra = vb + t0 * kQ8RowBytes + ((g ^ (t0 & 7)) << 4), rb = vb + t1 * kQ8RowBytes + ((g ^ (t1 & 7)) << 4);
          v[t][0] = lds128(ra);
          v[t][1] = lds128(rb);
          v[t][2] = lds128(ra + 8 * kQ8RowBytes);
          v[t][3] = lds128(rb + 8 * kQ8RowBytes);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float y0[4] = {0.f, 0.f, 0.f, 0.f}, y1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            uint32_t x0, x1, x2, x3, z0, z1, z2, z3;  // d = 16 g + 4 i + 0..3: the first two tokens, the two + 8
            q8_to_f16<kType>(__byte_perm(word(v[t][0], i), word(v[t][1], i), 0x5140), x0, x1);
            q8_to_f16<kType>(__byte_perm(word(v[t][0], i), word(v[t][1], i), 0x7362), x2, x3);
            q8_to_f16<kType>(__byte_perm(word(v[t][2], i), word(v[t][3], i), 0x5140), z0, z1);
            q8_to_f16<kType>(__byte_perm(word(v[t][2], i), word(v[t][3], i), 0x7362), z2, z3);
            if (!kPack) {
              mma_f16_16816(y0, x0, x1, z0, z1, bl[t][0], bl[t][1]);
              mma_f16_16816(y1, x2, x3, z2, z3, bl[t][0], bl[t][1]);
            }
            mma_f16_16816(y0, x0, x1, z0, z1, bh[t][0], bh[t][1]);
            mma_f16_16816(y1, x2, x3, z2, z3, bh[t][0], bh[t][1]);
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            o[2 * i][r] = fmaf(y0[r], vs, o[2 * i][r]);
            o[2 * i + 1][r] = fmaf(y1[r], vs, o[2 * i + 1][r]);
          }
        }
      } else {
        // ---- 16 rows of the tail: bf16 on both sides, the same fragment slots (the queries are read again)
        const uint4* qp = reinterpret_cast<const uint4*>(a.q + ((int64_t)b * a.Hq + h * a.G + gq) * kD);
        const int left = cc.tail - (u - cc.full) * kQ8TailUnit;
        float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int ch = 2 * (c + 4 * hh) + e;
            const uint4 lo = lds128(kb + tile_off(pi, ch)), hi = lds128(kb + tile_off(pi + 8, ch));
            const uint32_t f[2][4] = {{lo.x, hi.x, lo.y, hi.y}, {lo.z, hi.z, lo.w, hi.w}};
            const uint4 x = gq < a.G ? qp[ch] : make_uint4(0, 0, 0, 0);
            mma_bf16_16816(s, f[0], x.x, x.y);
            mma_bf16_16816(s, f[1], x.z, x.w);
          }
        const bool v_lo = pi < left, v_hi = pi + 8 < left;
        const float x0 = v_lo ? s[0] * a.scale_log2 : -INFINITY, x1 = v_lo ? s[1] * a.scale_log2 : -INFINITY;
        const float x2 = v_hi ? s[2] * a.scale_log2 : -INFINITY, x3 = v_hi ? s[3] * a.scale_log2 : -INFINITY;
        rescale(fmaxf(x0, x2), fmaxf(x1, x3));
        const float r0 = m0 > -INFINITY ? kQ8PBits - m0 : 0.f, r1 = m1 > -INFINITY ? kQ8PBits - m1 : 0.f;
        float p0 = fast_exp2(x0 + r0), p1 = fast_exp2(x1 + r1), p2 = fast_exp2(x2 + r0), p3 = fast_exp2(x3 + r1);
        l0 += p0 + p2;
        l1 += p1 + p3;
        p0 *= kQ8PUnit;
        p1 *= kQ8PUnit;
        p2 *= kQ8PUnit;
        p3 *= kQ8PUnit;
        const float h0 = bf16_round(p0), h1 = bf16_round(p1), h2 = bf16_round(p2), h3 = bf16_round(p3);
        const float d0 = p0 - h0, d1 = p1 - h1, d2 = p2 - h2, d3 = p3 - h3;  // three bf16 parts: 24 bits
        const uint32_t hi0 = pack_bf16(h0, h1), hi1 = pack_bf16(h2, h3), lo0 = pack_bf16(d0, d1), lo1 = pack_bf16(d2, d3);
        const uint32_t bh0 = movmatrix_trans(low_half ? lo0 : hi0), bh1 = movmatrix_trans(low_half ? lo1 : hi1);
        const uint32_t bl0 = kPack ? 0u : movmatrix_trans(lo0), bl1 = kPack ? 0u : movmatrix_trans(lo1);
        const uint32_t mi0 = pack_bf16(d0 - bf16_round(d0), d1 - bf16_round(d1)), mi1 = pack_bf16(d2 - bf16_round(d2), d3 - bf16_round(d3));
        const uint32_t bm0 = movmatrix_trans(low_half ? 0u : mi0), bm1 = movmatrix_trans(low_half ? 0u : mi1);
        const int t0 = 2 * c, t1 = (2 * c + 1) ^ 4;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int ch = 2 * g + e;
          const uint4 v0 = lds128(vb + tile_off(t0, ch)), v1 = lds128(vb + tile_off(t1, ch));
          const uint4 v2 = lds128(vb + tile_off(t0 + 8, ch)), v3 = lds128(vb + tile_off(t1 + 8, ch));
#pragma unroll
          for (int i = 0; i < 4; ++i) {  // d = 16 g + 8 e + 2 i + 0, 1
            const uint32_t af[4] = {__byte_perm(word(v0, i), word(v1, i), 0x5410), __byte_perm(word(v0, i), word(v1, i), 0x7632),
                                    __byte_perm(word(v2, i), word(v3, i), 0x5410), __byte_perm(word(v2, i), word(v3, i), 0x7632)};
            mma_bf16_16816(o[4 * e + i], af, bm0, bm1);
            if (!kPack) mma_bf16_16816(o[4 * e + i], af, bl0, bl1);
            mma_bf16_16816(o[4 * e + i], af, bh0, bh1);
          }
        }
      }
    }

    // ---- end of the piece: merge the four warps (warps 0 and 1 fill a slot each, 2 and 3 add to them, everybody writes
    // a part of the sum)
    float (*s_m)[kMaxG] = s_ml[(item - item_begin) & 1][0], (*s_l)[kMaxG] = s_ml[(item - item_begin) & 1][1];
    if (item + 1 < item_end) q8_load_q(a, cc.seg + 1, gq, c, q4);  // on their way during the merge
    int si_slot = 0, si_pieces = 0;
    if (a.merge && cc.slot >= 0) {
      const int2 x = __ldg(reinterpret_cast<const int2*>(a.merge + cc.seg));
      si_slot = x.x;
      si_pieces = x.y;
    }
#pragma unroll
    for (int sh = 4; sh <= 16; sh <<= 1) {
      l0 += __shfl_xor_sync(0xffffffffu, l0, sh);
      l1 += __shfl_xor_sync(0xffffffffu, l1, sh);
    }
    if (g == 0) {
      s_m[warp][2 * c] = m0;
      s_m[warp][2 * c + 1] = m1;
      s_l[warp][2 * c] = l0;
      s_l[warp][2 * c + 1] = l1;
    }
    __syncthreads();  // (and the slots of the piece before have been read)
    float al[2];  // from this warp's maximum to the CTA's
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float M = s_m[0][2 * c + e];
#pragma unroll
      for (int w = 1; w < kQ8Warps; ++w) M = fmaxf(M, s_m[w][2 * c + e]);
      const float m = e ? m1 : m0;
      al[e] = m == M ? 1.f : fast_exp2(m - M);
    }
    float* slot = slots + (warp & 1) * kQ8SlotFloats;
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
      if ((warp >> 1) == pass) {
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int j = 0; j < 8; j += 2) {  // o[j][e], o[j][2 + e]: d = 16 g + 2 j, + 1 of head 2 c + e
            float4* p = reinterpret_cast<float4*>(slot + q8_slot(2 * c + e, 16 * g + 2 * j));
            float4 v = make_float4(o[j][e] * al[e], o[j][2 + e] * al[e], o[j + 1][e] * al[e], o[j + 1][2 + e] * al[e]);
            if (pass == 1) {
              const float4 x = *p;
              v = make_float4(v.x + x.x, v.y + x.y, v.z + x.z, v.w + x.w);
            }
            *p = v;
          }
      }
      __syncthreads();
    }
    for (int hd = warp; hd < a.G; hd += kQ8Warps) {
      float M = s_m[0][hd];
#pragma unroll
      for (int w = 1; w < kQ8Warps; ++w) M = fmaxf(M, s_m[w][hd]);
      float l = 0.f;
#pragma unroll
      for (int w = 0; w < kQ8Warps; ++w) l += s_m[w][hd] == M ? s_l[w][hd] : s_l[w][hd] * fast_exp2(s_m[w][hd] - M);
      l *= kQ8PUnit;
      const float inv = l == 0.f ? 0.f : 1.f / l;  // (a NaN stays one)
      const float lse = l == 0.f ? -INFINITY : M + log2f(l);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < (kPack ? 4 : 2); ++i) {
        const float4 x = *reinterpret_cast<const float4*>(slots + (i & 1) * kQ8SlotFloats + q8_slot(hd + 4 * (i >> 1), 4 * lane));
        v = make_float4(v.x + x.x, v.y + x.y, v.z + x.z, v.w + x.w);
      }
      v = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
      const size_t at = ((size_t)b * a.Hq + (size_t)h * a.G + hd) * kD;
      if (cc.slot >= 0)
        reinterpret_cast<float4*>(a.part_o + ((size_t)cc.slot * kMaxG + hd) * kD)[lane] = v;
      else if (a.out_fp32)
        reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out) + at)[lane] = v;
      else
        reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.out) + at)[lane] = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
      if (lane == 0) {
        // the combine pass takes an infinite LSE as the one partial that counts: a NaN (from a block with the scale NaN) reaches the output
        if (cc.slot >= 0) a.part_lse[(size_t)cc.slot * kMaxG + hd] = lse == lse ? lse : INFINITY;
        else if (a.lse_out) a.lse_out[(size_t)b * a.Hq + h * a.G + hd] = lse * 0.6931471805599453f;
      }
    }
    if (a.merge && cc.slot >= 0) {
      __threadfence();
      __syncthreads();  // this CTA's piece is written
      // the count wraps to 0 with the last piece: ready for the next call
      if (tid == 0) s_last = atomicInc(reinterpret_cast<unsigned int*>(&a.merge[cc.seg].arrived), (unsigned int)si_pieces - 1u) == (unsigned int)si_pieces - 1u;
      __syncthreads();
      if (s_last) {
        __threadfence();
        for (int hd = warp; hd < a.G; hd += kQ8Warps) q8_merge_pieces(a, si_slot, si_pieces, b, h, hd, lane);
      }
    }
  }
  cp_async_wait<0>();
}

// Combine: a CTA per (segment, head) pair and 32 of the 128 dimensions, a warp per 32 pieces, a lane per dimension.  Small
// enough (128 threads, at most 64 registers: all that two attention CTAs leave) to be resident beside two CTAs of the attention kernel:
// launched programmatically it has its plan entry and waits at the dependency when the last partial is written, and the
// next attention kernel's CTAs find room beside it (128K: 21.1 -> 20.5 us, 256K G = 7: 28.2 -> 26.7 us).
constexpr int kQ8CombineThreads = 128;
constexpr int kQ8CombineSplit = 4;
constexpr int kQ8CombinePerSm = 8;  // caps its registers
static_assert(2 * kQ8DecodeThreads * kQ8Regs + 65536 / kQ8CombinePerSm <= 65536 && kQ8CombineThreads * kQ8CombinePerSm <= 2048,
              "a combine CTA fits beside two attention CTAs");
__global__ void __launch_bounds__(kQ8CombineThreads, kQ8CombinePerSm) q8_combine_kernel(const CombineArgs a) {
  __shared__ float s_acc[kQ8CombineThreads / 32][32], s_w[kQ8CombineThreads / 32], s_m[kQ8CombineThreads / 32];
  const int seg = blockIdx.x, hd = blockIdx.y, part = blockIdx.z;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_launch_dependents();
  const SegInfo si = a.seg_info[seg];  // plan data: older than the previous kernel
  pdl_wait();
  if (si.n_pieces <= 1) return;  // written directly by the attention kernel
  const int n = si.n_pieces;
  const float* lse = a.part_lse + (size_t)si.slot_begin * kMaxG + hd;
  const float* po = a.part_o + ((size_t)si.slot_begin * kMaxG + hd) * kD + part * 32 + lane;
  float acc = 0.f, wsum = 0.f, mw = -INFINITY;
  for (int p0 = warp * 32; p0 < n; p0 += kQ8CombineThreads) {
    const float l = p0 + lane < n ? lse[(size_t)(p0 + lane) * kMaxG] : -INFINITY;
    float v[32];
#pragma unroll
    for (int u = 0; u < 32; ++u) v[u] = p0 + u < n ? po[(size_t)(p0 + u) * (kMaxG * kD)] : 0.f;
    float mx = l;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    mx = fmaxf(mx, mw);
    if (mx > -INFINITY) {  // the same in every lane
      const float sc = exp2f(mw - mx), e = exp2f(l - mx);  // 0 for an empty piece (LSE -inf) and on the first pass (mw = -inf)
      acc *= sc;
      wsum = wsum * sc + e;  // a lane's own pieces
      mw = mx;
#pragma unroll
      for (int u = 0; u < 32; ++u) acc += __shfl_sync(0xffffffffu, e, u) * v[u];
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) wsum += __shfl_xor_sync(0xffffffffu, wsum, o);
  s_acc[warp][lane] = acc;
  if (lane == 0) {
    s_w[warp] = wsum;
    s_m[warp] = mw;
  }
  __syncthreads();
  if (warp == 0) {
    float M = -INFINITY, W = 0.f, r = 0.f;
#pragma unroll
    for (int w = 0; w < kQ8CombineThreads / 32; ++w) M = fmaxf(M, s_m[w]);
#pragma unroll
    for (int w = 0; w < kQ8CombineThreads / 32; ++w) {
      const float f = s_m[w] > -INFINITY ? exp2f(s_m[w] - M) : 0.f;
      W += f * s_w[w];
      r += f * s_acc[w][lane];
    }
    r *= W == 0.f ? 0.f : 1.f / W;  // (a NaN stays one)
    const int b = seg / a.Hkv, h = seg % a.Hkv;
    const size_t at = ((size_t)b * a.Hq + (size_t)h * a.G + hd) * kD + part * 32 + lane;
    if (a.out_fp32)
      reinterpret_cast<float*>(a.out)[at] = r;
    else
      reinterpret_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16_rn(r);
    if (a.lse_out && part == 0 && lane == 0)
      a.lse_out[(size_t)b * a.Hq + h * a.G + hd] = W == 0.f ? -INFINITY : (M + log2f(W)) * 0.6931471805599453f;
  }
}

}  // namespace catekv

using namespace catekv;

// the kernels' shared-memory limits, once per device
template <int kType, int kStages, bool kPack>
static cudaError_t q8_allow_smem() {
  return cudaFuncSetAttribute(q8_decode_partial_kernel<kType, kStages, kPack>, cudaFuncAttributeMaxDynamicSharedMemorySize, q8_decode_smem(kStages));
}
static int q8_decode_attributes() {
  static std::atomic<bool> attr_set[64];
  int dev = 0;
  CATEKV_CUDA_TRY(cudaGetDevice(&dev));
  if (dev >= 0 && dev < 64 && attr_set[dev].load(std::memory_order_acquire)) return CATEKV_OK;
  CATEKV_CUDA_TRY((q8_allow_smem<CATEKV_Q8_E4M3, 2, false>()));
  CATEKV_CUDA_TRY((q8_allow_smem<CATEKV_Q8_E4M3, 2, true>()));
  CATEKV_CUDA_TRY((q8_allow_smem<CATEKV_Q8_E4M3, 3, false>()));
  CATEKV_CUDA_TRY((q8_allow_smem<CATEKV_Q8_E4M3, 3, true>()));
  CATEKV_CUDA_TRY((q8_allow_smem<CATEKV_Q8_INT8, 2, true>()));
  CATEKV_CUDA_TRY((q8_allow_smem<CATEKV_Q8_INT8, 3, false>()));
  CATEKV_CUDA_TRY((q8_allow_smem<CATEKV_Q8_INT8, 3, true>()));
  if (dev >= 0 && dev < 64) attr_set[dev].store(true, std::memory_order_release);
  return CATEKV_OK;
}
template <int kType, int kStages, bool kPack>
static cudaError_t q8_launch_partials(const Q8DecodeArgs& a, int num_ctas, cudaStream_t st) {
  return launch_pdl(q8_decode_partial_kernel<kType, kStages, kPack>, dim3(num_ctas), dim3(kQ8DecodeThreads), q8_decode_smem(kStages), st, a);
}

extern "C" int catekv_q8_decode_num_ctas(void) {
  int rc = q8_decode_attributes();
  if (rc) return rc;
  int per_sm = 0;
  CATEKV_CUDA_TRY(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, (q8_decode_partial_kernel<CATEKV_Q8_E4M3, 3, false>), kQ8DecodeThreads, q8_decode_smem(3)));
  return sm_count() * (per_sm < 1 ? 1 : per_sm);
}

extern "C" int catekv_q8_decode_plan(const catekv_q8_cache* cache, int32_t num_ctas, void* plan_host, void* plan_dev,
                                     size_t plan_bytes, catekv_stream stream) {
  CATEKV_API_RANGE();
  int rc = check_q8_cache(cache);
  if (rc) return rc;
  const int n_segs = cache->B * cache->Hkv;
  for (int s = 0; s < n_segs; ++s)
    if (cache->seg_len[s] < 0 || cache->seg_len[s] > cache->seg_cap[s]) return CATEKV_ERR_INVALID_ARG;
  const PlanSource src = {n_segs, cache->seg_len, cache->seg_off, cache->seg_cap, 0};
  return build_plan(src, num_ctas, kQ8PlanTile, kQ8Block, kQ8SegEndCharge, plan_host, plan_dev, plan_bytes, (cudaStream_t)stream);
}

extern "C" int catekv_q8_decode_attn(const catekv_q8_cache* cache, const void* q, int32_t Hq, float sm_scale, void* out,
                                     int32_t out_dtype, float* lse_out, const void* plan_host, void* plan_dev,
                                     size_t plan_bytes, void* ws, size_t ws_bytes, catekv_stream stream) {
  CATEKV_API_RANGE();
  int rc = check_q8_cache(cache);
  if (rc) return rc;
  if (!q || !out || !plan_host || !plan_dev || !ws) return CATEKV_ERR_INVALID_ARG;
  if (Hq <= 0 || Hq % cache->Hkv != 0) return CATEKV_ERR_INVALID_ARG;
  const int G = Hq / cache->Hkv;
  if (G > kMaxG) return CATEKV_ERR_UNSUPPORTED;
  if (out_dtype != CATEKV_OUT_BF16 && out_dtype != CATEKV_OUT_FP32) return CATEKV_ERR_UNSUPPORTED;
  if (!(sm_scale >= 0.f) || isinf(sm_scale)) return CATEKV_ERR_INVALID_ARG;
  if (((uintptr_t)q | (uintptr_t)out | (uintptr_t)ws) & 15) return CATEKV_ERR_INVALID_ARG;
  const PlanHeader* hdr = (const PlanHeader*)plan_host;
  const int n_segs = cache->B * cache->Hkv;
  if (plan_bytes < sizeof(PlanHeader) || hdr->magic != kPlanMagic || hdr->n_segs != n_segs || hdr->num_ctas <= 0 ||
      hdr->tile != kQ8PlanTile)
    return CATEKV_ERR_INVALID_ARG;
  const PlanLayout L = plan_layout(n_segs, hdr->num_ctas);
  if (plan_bytes < L.bytes) return CATEKV_ERR_WORKSPACE;
  size_t off_lse = 0;
  if (ws_bytes < ws_layout(n_segs, hdr->num_ctas, &off_lse)) return CATEKV_ERR_WORKSPACE;
  if (plan_outlived(plan_host, L.off_seg, cache->seg_len, n_segs)) return CATEKV_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  const uint8_t* pd = (const uint8_t*)plan_dev;
  rc = q8_decode_attributes();
  if (rc) return rc;
  Q8DecodeArgs a;
  a.k_pool = (const uint8_t*)cache->k_pool;
  a.v_pool = (const uint8_t*)cache->v_pool;
  a.k_scale = cache->k_scale;
  a.v_scale = cache->v_scale;
  a.k_tail = (const uint8_t*)cache->k_tail;
  a.v_tail = (const uint8_t*)cache->v_tail;
  a.seg_len = cache->seg_len_dev;
  a.q = (const uint16_t*)q;
  a.Hq = Hq;
  a.Hkv = cache->Hkv;
  a.G = G;
  a.scale_log2 = (sm_scale == 0.f ? 1.0f / sqrtf((float)kD) : sm_scale) * 1.4426950408889634f;
  a.ctas = (const CtaHeader*)(pd + L.off_cta);
  a.items = (const WorkItem*)(pd + L.off_items);
  a.part_o = (float*)ws;
  a.part_lse = (float*)((uint8_t*)ws + off_lse);
  a.out = out;
  a.out_fp32 = out_dtype == CATEKV_OUT_FP32;
  a.lse_out = lse_out;
  const int most = hdr->total_rows <= (int64_t)kQ8MergeShare * hdr->num_ctas ? kQ8MergeMost : kQ8MergePieces;
  a.merge = hdr->max_pieces <= most ? (SegInfo*)((uint8_t*)plan_dev + L.off_seg) : nullptr;
  const bool longs = hdr->total_rows >= (int64_t)kQ8LongShare * hdr->num_ctas, pack = G <= 4;
  const int n = hdr->num_ctas;
  if (cache->dtype == CATEKV_Q8_INT8) {
    if (!pack) CATEKV_CUDA_TRY((q8_launch_partials<CATEKV_Q8_INT8, 3, false>(a, n, st)));
    else if (longs) CATEKV_CUDA_TRY((q8_launch_partials<CATEKV_Q8_INT8, 2, true>(a, n, st)));
    else CATEKV_CUDA_TRY((q8_launch_partials<CATEKV_Q8_INT8, 3, true>(a, n, st)));
  } else if (longs) {
    if (pack) CATEKV_CUDA_TRY((q8_launch_partials<CATEKV_Q8_E4M3, 2, true>(a, n, st)));
    else CATEKV_CUDA_TRY((q8_launch_partials<CATEKV_Q8_E4M3, 2, false>(a, n, st)));
  } else {
    if (pack) CATEKV_CUDA_TRY((q8_launch_partials<CATEKV_Q8_E4M3, 3, true>(a, n, st)));
    else CATEKV_CUDA_TRY((q8_launch_partials<CATEKV_Q8_E4M3, 3, false>(a, n, st)));
  }
  if (hdr->n_slots > 0 && !a.merge) {
    CombineArgs ca;
    ca.seg_info = (const SegInfo*)(pd + L.off_seg);
    ca.part_o = a.part_o;
    ca.part_lse = a.part_lse;
    ca.out = out;
    ca.lse_out = lse_out;
    ca.Hq = Hq;
    ca.Hkv = cache->Hkv;
    ca.G = G;
    ca.out_fp32 = a.out_fp32;
    CATEKV_CUDA_TRY(launch_pdl(q8_combine_kernel, dim3(n_segs, G, kQ8CombineSplit), dim3(kQ8CombineThreads), 0, st, ca));
  }
  return CATEKV_OK;
}
