// Attention of a chunk of new tokens over the hybrid cache: query i of the n tokens that sequence b has just had appended
// sees the rows j < len - n + i + 1 of every list of the sequence (its own pools, then its overflow pages),
//   out = softmax(sm_scale q K^T) V,   lse = log sum exp(sm_scale q K^T).
//
// One pass over K and V with a running reference and sum per query row.  The query rows of a (sequence, KV head) are its
// tokens' heads, row r = token * G + head, so that a K tile is read once for the whole group; a block of them is 128 rows (an M = 128 tile) or,
// where K and V are more than L2 holds, 256 (two, template kQ2).  chunk_attn_kernel is persistent,
// one CTA per SM: the 128-key tiles of all blocks of all lists, laid end to end, are cut into equal shares, from the device's lengths
// (a captured call follows lists that grow).  A block that several CTAs share leaves partial results, which
// chunk_combine_kernel merges in the order of the keys.
//
// A tile is worked on in two steps of 64 keys.  Per step: S = Q K^T (tcgen05.mma, both operands in shared memory); a softmax thread owns a
// query row: it reads it (tcgen05.ld), raises its reference when the step's maximum exceeds it by more than 2^8 (the accumulator is then
// scaled in tensor memory: rare after the first tiles) and writes P = exp2(logit - reference) over S in kParts bf16 numbers, each the
// rounded rest of those before it; O += P V takes P from tensor memory and V as the MN-major operand as TMA left it.  Every M tile has softmax
// warps of its own, an accumulator, and two slots of S / P, so that S of the next step is formed while the softmax is at this one.
// (Steps of 128 keys have room for one slot only beside two accumulators: softmax and products of an M tile took turns, 4100
// cycles a tile for two M tiles and P in one part, 3400 with steps of 64, where the products need 2050; S with 64 keys reads its Q operand twice as often.)  One M tile with
// bf16 results (kSplit) has four slots and softmax warps for either step of a tile: S is formed two tiles ahead, as few rows are a chain of waits otherwise.
//
// Bounds and measures (B200, single runs).  Full blocks: the products, three for the formula's two; 4096 tokens over 8 lists of 16 K rows, G = 4, in 1220 to
// 1300 us with either form (950 to 1020 TFLOP/s of the formula's two products, half as much again in all); 4096 tokens alone in 173 to 186 us; two M tiles, 512 tokens over 3 lists of 117 K
// rows, in 417 us.  Few rows: K and V once through DRAM; 4 tokens of 16 x 32 K rows in 311 to 346 us, 6.2 to 6.9 TB/s; a token over 8 lists of 128 rows in 7.9 us, which are waits one behind the other (schedule 1 us, loads 1, S, softmax and product 2.5,
// results 0.7, the merge's launch).  fp32 results: three products for one, and the softmax's conversions; 333 tokens of 7 heads a group over
// 2 lists of 65 K rows in 280 to 316 us.
//
// Precision.  kParts = 2 (bf16 results): P with 17 significant bits in every form, so that the result's own rounding is what is seen of it (with P in one bf16
// number, 2^-9, 512 tokens over 117 K rows take 341 us for 417, and the error of results in the norm is 2.3e-3 for 1.65e-3; which form runs
// goes by the other sequences of the batch too).  Where the block has at most 64 rows they may lie in the M tile twice (kDup, kParts = 1): the copies' softmax comes out
// the same, their warps write the second part, one instruction multiplies both, and the results are added at the end.  3 (fp32 results): all of fp32's.  The tensor cores add with truncation, and what that loses
// goes by the accumulator's size and the number of instructions.  For fp32 results the parts behind the first therefore have an accumulator of their
// own, 2^-9 as large, and both are added, with rounding, to a sum in the thread's registers every kFlush tiles, where the products start from zero
// (relative error of 64K rows: 5e-6 with one accumulator and a flush every 16 tiles).  That takes one M tile, whatever the number of rows.
//
// The product with V stops at the 16 keys that hold the last row that a query of the block sees; of these, rows behind it are zeroed in shared
// memory (what lies behind a list may be NaN, and 0 * NaN is not 0); an infinity or a NaN in a new row, which later tokens see and earlier ones do not, is taken
// out there too and added to the rows that see it at the end.
//
// Warps: those of the softmax; then one each for the query block and the logits' instructions, the K and V tiles by TMA into a ring each, the V
// tiles that need a look, and the products' instructions.  Every wait is bounded; a CTA whose wait runs out frees its tensor memory, records
// CATEKV_STATUS_WAIT_EXPIRED and returns.
#include <math.h>

#include <atomic>

#include "decode.cuh"
#include "score.cuh"
#include "tc.cuh"

namespace catekv {

constexpr int kChMaxSeqs = 512;  // sequences of a call: their counts travel in the kernel's arguments
constexpr int kChMaxCtas = 256;
constexpr int kChTileBytes = 128 * 256;  // a [128 x 128] bf16 tile
constexpr int kChTmemCols = 512;         // slots of S / P in columns 0-255, the M tiles' accumulators at 256 and 384
constexpr float kChTau = 8.f;
constexpr int kChBarriers = 52;
constexpr int kLowStride = 36;  // floats: rows of 32 columns handed over in shared memory
template <bool kQ2, int kFlush, bool kDup>
struct ChunkShape {
  static constexpr bool kSplit = !kQ2 && !kFlush;   // one M tile, bf16 results: the steps of a tile have softmax warps of their own
  static constexpr int kTiles = kQ2 ? 2 : 1;        // M tiles
  static constexpr int kStagesK = kFlush ? 3 : 2, kStagesV = 3;  // of the two rings
  static constexpr int kSoft = kQ2 || kSplit ? 8 : 4;  // softmax warps
  static constexpr int kWarps = kSoft + 4, kThreads = kWarps * 32;
  // Slot of step h of a tile: 2 x + h for M tile x; kSplit: four slots, 2 (tile mod 2) + h, so that S is formed two tiles ahead.
  static constexpr int kSlotCols = kFlush ? 128 : 64;
  static constexpr int kLead = kSplit ? 2 : 1;      // K tiles loaded ahead of the V tile: K_0 .. K_{lead-1}, V_0, K_lead, V_1, ...
  static constexpr size_t kSmem = 1024 + (size_t)(kTiles + kStagesK + kStagesV) * kChTileBytes + kChBarriers * 8 + 64 + (kSplit ? 4 * 128 * sizeof(float) : 0) +
                                  (kDup ? 2 * 64 * kLowStride * sizeof(float) : 0);
  static_assert(kSmem <= 226 * 1024, "chunk_attn_kernel: one CTA's shared memory");
};
// Tiles that a block is charged (ChunkArgs::charge), with one M tile and with two.  One M tile: 64 x 300 rows of 8 heads, 4 tokens, 31.8 us with 3, 34.7
// with 2, 34.2 with 4; two: 64 tokens of 16 x 2500 rows of 8 heads 81.8 us with 2, 89.2 with 3, 86.4 with 1.
constexpr int kChCharge = 3, kChChargeTwo = 2;
constexpr int64_t kChL2Rows = (int64_t)120e6 / (2 * kRowBytes);  // rows whose K and V fill L2 (126 MB)

struct ChunkSeqs {  // host counts of every sequence
  int32_t n_new[kChMaxSeqs];
  int32_t start[kChMaxSeqs];
};
struct ChunkArgs {
  const int32_t* seg_off;
  const int32_t* seg_len;
  const int32_t* seg_cap;
  const uint16_t* v_pool;
  const uint16_t* v_ovf;
  const int32_t* table;  // null: no pages
  int32_t max_pages, n_pages;
  int32_t n_segs, Hkv, G, Hq;
  int32_t TB;  // tokens of a query block
  int32_t TQ;  // tokens of a load
  int32_t R;   // rows of a tile of part_o and part_ml
  int32_t charge;  // tiles that a block is charged beyond its own when the shares are cut: its queries, a pipeline that fills and drains, its results
  float scale_log2;
  void* out;
  float* lse;
  int32_t out_fp32;
  // Partial results, two tiles [32 d / 4][R rows] (float4: a warp's rows lie side by side) for every M tile of a CTA: of its first block, and
  // of its last.  part_ml: reference (log2 domain) and sum of the rows.
  float4* part_o;
  float2* part_ml;
  int32_t* desc;   // [CTAs][8]
  int32_t* status;
  int32_t* checked;
  uint32_t spin_limit;
  int32_t idle_producer;
};

struct ChunkSeg {  // one list as the schedule sees it
  int32_t len, n_new, n_blk, off, cap, start, head;  // start: the sequence's first token; head: the list's first query head
};
__device__ __forceinline__ void ch_set_len(const ChunkArgs& a, ChunkSeg& g, int s) {
  g.len = min(max(a.seg_len[s], 0), g.cap + CATEKV_PAGE_ROWS * a.max_pages);
}
__device__ __forceinline__ ChunkSeg ch_seg(const ChunkArgs& a, const ChunkSeqs& sq, int s, bool with_len) {
  const int b = s / a.Hkv;
  ChunkSeg g = {0, sq.n_new[b], 0, 0, 0, sq.start[b], (s - b * a.Hkv) * a.G};
  g.n_blk = (g.n_new + a.TB - 1) / a.TB;
  if (g.n_blk) {
    g.off = a.seg_off[s];
    g.cap = a.seg_cap[s];
    if (with_len) ch_set_len(a, g, s);
  }
  return g;
}
// key tiles of a block (at least one, so that rows that see nothing get their output)
__device__ __forceinline__ int ch_tiles(const ChunkArgs& a, const ChunkSeg& g, int blk) {
  const int seen = g.len - g.n_new + min(g.n_new, a.TB * (blk + 1));
  return max(1, (seen + kKeyTile - 1) / kKeyTile);
}

// a position among a block's units (the charge, then its tiles) -> its tile
__device__ __forceinline__ int ch_tile_at(const ChunkArgs& a, int p) { return max(0, p - a.charge); }

struct ChunkItem {
  int32_t seg, blk, t0, t1, nt;  // tiles [t0, t1) of the block's nt
  ChunkSeg g;
};
// The items of a CTA, one after the other; every role walks them by itself.
struct ChunkWalk {
  int32_t left, seg, blk, p;  // units left; the next block and the position in it
  ChunkSeg g;
  __device__ __forceinline__ bool next(const ChunkArgs& a, const ChunkSeqs& sq, ChunkItem& it) {
    if (left <= 0) return false;
    while (blk >= g.n_blk) {
      if (++seg >= a.n_segs) return false;
      g = ch_seg(a, sq, seg, true);
      blk = 0;
    }
    it.seg = seg;
    it.blk = blk;
    it.nt = ch_tiles(a, g, blk);
    const int end = min(it.nt + a.charge, p + left);
    it.t0 = ch_tile_at(a, p);
    it.t1 = ch_tile_at(a, end);
    it.g = g;
    left -= end - p;
    p = 0;
    ++blk;
    return it.t1 > it.t0;  // (a share that ends inside a block's charge ends there)
  }
};

// One lane of a converged warp issues for all of it.  The warp that feeds the tensor cores runs converged, so that descriptors, addresses and counters
// live in uniform registers: with one lane on a branch of its own every tcgen05.mma moved its operands there first, 70 cycles an
// instruction, and the products were bound by that.
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ int uni(int x) { return __shfl_sync(0xffffffffu, x, 0); }
// Every wait of the kernel: the warp goes on, or leaves, as a whole (its lanes may see a wait run out at different times, and what follows are
// collectives of the warp).
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, uint32_t limit) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, limit));
}

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
               : "memory");
}
// 32 bytes of this thread's row; `whole`: the address is a multiple of 32, and one store writes a sector
__device__ __forceinline__ void st_row32(void* p, const uint32_t (&w)[8], bool whole) {
  if (whole) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};\n" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]),
                 "r"(w[6]), "r"(w[7])
                 : "memory");
  } else {
    reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
    reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
}
template <int kN>
__device__ __forceinline__ float ch_max(const float* x) {
  float m0 = fmax3(x[0], x[1], x[2]), m1 = fmax3(x[3], x[4], x[5]), m2 = fmax3(x[6], x[7], x[8]), m3 = fmax3(x[9], x[10], x[11]);
#pragma unroll
  for (int c = 12; c < kN - 4; c += 8) {
    m0 = fmax3(m0, x[c], x[c + 1]);
    m1 = fmax3(m1, x[c + 2], x[c + 3]);
    m2 = fmax3(m2, x[c + 4], x[c + 5]);
    m3 = fmax3(m3, x[c + 6], x[c + 7]);
  }
  m0 = fmax3(m0, x[kN - 4], x[kN - 3]);
  m1 = fmax3(m1, x[kN - 2], x[kN - 1]);
  return fmaxf(fmaxf(m0, m1), fmaxf(m2, m3));
}
// two fp32 numbers at a time
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;\n" : "=l"(reinterpret_cast<uint64_t&>(d)) : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)), "l"(reinterpret_cast<uint64_t&>(c)));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("add.rn.f32x2 %0, %1, %2;\n" : "=l"(reinterpret_cast<uint64_t&>(d)) : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
  return d;
}
__device__ __forceinline__ void tmem_st8u(uint32_t taddr, const uint32_t (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};\n"
               :
               : "r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
// kN logits -> probabilities of kN keys in kParts bf16 numbers, kN / 2 columns each, `step` columns from part to part; returns their sum.
// kLastOnly: the last of the parts alone, at step 0.
template <int kN, int kParts, bool kLastOnly = false>
__device__ __forceinline__ float ch_probs(const float* x, float scale, float neg_ref, uint32_t to, uint32_t step) {
  float2 s0 = make_float2(0.f, 0.f), s1 = s0;
  uint32_t w[kParts][kN / 2];
#pragma unroll
  for (int c = 0; c < kN; c += 2) {
    float2 p = fma2(make_float2(x[c], x[c + 1]), make_float2(scale, scale), make_float2(neg_ref, neg_ref));
    p.x = fast_exp2(p.x);
    p.y = fast_exp2(p.y);
    if (c & 2) s1 = add2(s1, p);
    else s0 = add2(s0, p);
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
      w[k][c / 2] = pack_bf16(p.x, p.y);
      if (k + 1 < kParts)  // what is left of it (exact)
        p = fma2(make_float2(__uint_as_float(w[k][c / 2] << 16), __uint_as_float(w[k][c / 2] & 0xffff0000u)), make_float2(-1.f, -1.f), p);
    }
  }
#pragma unroll
  for (int k = kLastOnly ? kParts - 1 : 0; k < kParts; ++k) {
    if constexpr (kN == 32) tmem_st16u(to + k * step, w[k]);
    else tmem_st8u(to + k * step, w[k]);
  }
  s0 = add2(s0, s1);
  return s0.x + s0.y;
}

// rows of a V tile that the product takes, where `seen` rows from its first on are seen (at least one step, so that the accumulator is written)
__device__ __forceinline__ int ch_v_rows(int seen) { return min(max((seen + 15) & ~15, 16), kKeyTile); }
// pool row of row r of a list, or of its overflow pages (page < 0: not there)
__device__ __forceinline__ int ch_page(const ChunkArgs& a, int seg, int o) {
  const int p = o >> 6;
  const int pg = (a.table && p < a.max_pages) ? a.table[(int64_t)seg * a.max_pages + p] : -1;
#ifdef CATEKV_CHECKED
  if (pg < 0 || pg >= a.n_pages) raise_status(a.checked, CATEKV_STATUS_INDEX_RANGE, kKidChunk, seg, pg);
#endif
  return pg < a.n_pages ? pg : -1;
}

template <bool kQ2, int kParts, int kFlush, bool kDup>
__global__ void __launch_bounds__(ChunkShape<kQ2, kFlush, kDup>::kThreads, 1)
    chunk_attn_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                      const __grid_constant__ CUtensorMap ko_map, const __grid_constant__ CUtensorMap vo_map,
                      const __grid_constant__ CUtensorMap q_map, const __grid_constant__ ChunkArgs a,
                      const __grid_constant__ ChunkSeqs sq) {
  using Sh = ChunkShape<kQ2, kFlush, kDup>;
  constexpr int kStagesK = Sh::kStagesK, kStagesV = Sh::kStagesV, kTiles = Sh::kTiles, kLead = Sh::kLead, kSoft = Sh::kSoft, kWarps = Sh::kWarps;
  constexpr int kQBytes = kTiles * kChTileBytes, kQBlock = kQBytes / 2;
  constexpr bool kSplit = Sh::kSplit;
  static_assert(kParts * 32 <= Sh::kSlotCols, "P fits its slot");
  // tile number n (of the CTA): the slot of M tile x and step h, and the parity of its barriers
  auto slot_of = [](uint32_t n, int x, int h) { return kSplit ? (int)(2 * (n & 1)) + h : 2 * x + h; };
  auto phase_of = [](uint32_t n) { return (kSplit ? n >> 1 : n) & 1; };
  extern __shared__ uint8_t smem_raw[];
  __shared__ int s_scan[kWarps], s_first[10];
  const int tid = threadIdx.x, warp = uni(tid >> 5), lane = tid & 31;
  const uint32_t s_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (s_base - smem_u32(smem_raw));
  const uint32_t s_q = s_base, s_k = s_base + kQBytes, s_v = s_k + kStagesK * kChTileBytes;
  uint64_t* s_bar = reinterpret_cast<uint64_t*>(smem + kQBytes + (kStagesK + kStagesV) * kChTileBytes);
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(s_bar + kChBarriers);
  volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem + 1);
  int* s_odd = reinterpret_cast<int*>(s_tmem + 4);  // [4]: first new row with an infinity or a NaN in V, of the last blocks that had V tiles looked at
  float* s_ref = reinterpret_cast<float*>(s_tmem + 16);  // kSplit: [step][row] the rows' references, then their sums
  float* s_low = s_ref + 4 * 128;  // kDup: [step][64 rows][kLowStride]
  const uint32_t bar0 = smem_u32(s_bar);
  auto B = [&](int i) { return bar0 + 8u * (uint32_t)i; };
  constexpr int kFullK = 0, kEmptyK = kFullK + kStagesK, kFullV = kEmptyK + kStagesK, kEmptyV = kFullV + kStagesV, kFixed = kEmptyV + kStagesV,
                kDoneS = kFixed + kStagesV, kPReady = kDoneS + 4, kDonePV = kPReady + 4, kDoneO = kDonePV + 4, kQFull = kDoneO + 2, kQEmpty = kQFull + 1,
                kDec = kQEmpty + 1, kXch = kDec + 4, kLowFull = kXch + 4, kLowEmpty = kLowFull + 4;
  static_assert(kLowEmpty + 4 <= kChBarriers, "barrier table");

  pdl_launch_dependents();
  if (tid == 0) {
    *s_abort = 0;
#pragma unroll
    for (int i = 0; i < kChBarriers; ++i) {
      const int count = (i >= kPReady && i < kPReady + 4) ? 4 : (i >= kXch && i < kXch + 4) || (i >= kEmptyV && i < kEmptyV + kStagesV) ? 2 : 1;
      asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(B(i)), "r"(count));
    }
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  }
  if (warp == kSoft) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(s_tmem)), "r"(kChTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
  }
  if (tid == kSoft * 32 + 32) {
    const CUtensorMap* maps[5] = {&k_map, &v_map, &q_map, &ko_map, &vo_map};
#pragma unroll
    for (int i = 0; i < 5; ++i) asm volatile("prefetch.tensormap [%0];\n" ::"l"(maps[i]) : "memory");
  }
  // Rows of the block without a query are zeros, and so are their S and P: the tensor cores draw less for them, and calls back to back run at
  // the power limit (4 tokens of 16 x 32K rows for 0.3 s: 385 us a call with whatever lay there, 355 with zeros; a single call 346).
  for (int i = tid; i < kQBytes / 16; i += Sh::kThreads) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0u, 0u, 0u, 0u);
  fence_async_smem();
  // The list of this thread: all but its length is there before the kernels ahead have finished.
  ChunkSeg mine = {0, 0, 0, 0, 0, 0, 0};
  if (tid < a.n_segs) mine = ch_seg(a, sq, tid, false);
  pdl_wait();

  // ---- this CTA's share of the tiles of all blocks
  int total = 0, u0 = 0, u1 = 0;
  {
    auto cost_of = [&](const ChunkSeg& g) {
      int c = 0;
      for (int j = 0; j < g.n_blk; ++j) c += ch_tiles(a, g, j) + a.charge;
      return c;
    };
    if (mine.n_blk) ch_set_len(a, mine, tid);
    const int cost0 = cost_of(mine);
    const bool one_pass = a.n_segs <= Sh::kThreads;
    int inc = cost0;  // of the lists up to this thread's, within the warp
    if (!one_pass)
      for (int s = tid + Sh::kThreads; s < a.n_segs; s += Sh::kThreads) inc += cost_of(ch_seg(a, sq, s, true));
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    if (lane == 31) s_scan[warp] = inc;
    if (tid == 0) {
      s_first[0] = a.n_segs;           // no tile: nothing to do
      a.desc[blockIdx.x * 8 + 2] = 0;  // (no cut at the start of a share, unless there is one)
    }
    __syncthreads();
    int before = 0;  // of the warps before this one
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      before += w < warp ? s_scan[w] : 0;
      total += s_scan[w];
    }
    const int C = gridDim.x, c = blockIdx.x, q = total / C, r = total - q * C;
    u0 = c * q + min(c, r);
    u1 = u0 + q + (c < r ? 1 : 0);
    int passed = 0;  // of the lists of earlier rounds
    for (int s0 = 0; s0 < a.n_segs; s0 += Sh::kThreads) {
      const int s = s0 + tid;
      int cost = cost0;
      if (!one_pass) {
        __syncthreads();
        if (s0 > 0) mine = s < a.n_segs ? ch_seg(a, sq, s, true) : ChunkSeg{0, 0, 0, 0, 0, 0, 0};
        cost = s0 > 0 ? cost_of(mine) : cost0;
        inc = cost;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, inc, o);
          if (lane >= o) inc += y;
        }
        if (lane == 31) s_scan[warp] = inc;
        __syncthreads();
        before = passed;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          before += w < warp ? s_scan[w] : 0;
          passed += s_scan[w];
        }
      }
      const int ex = before + inc - cost;
      if (u1 > u0 && u0 >= ex && u0 < ex + cost) {
        int p = u0 - ex, j = 0, nt = ch_tiles(a, mine, 0);
        while (p >= nt + a.charge) {
          p -= nt + a.charge;
          nt = ch_tiles(a, mine, ++j);
        }
        s_first[0] = s;
        s_first[1] = j;
        s_first[2] = p;
        s_first[3] = mine.len;
        s_first[4] = mine.n_new;
        s_first[5] = mine.n_blk;
        s_first[6] = mine.off;
        s_first[7] = mine.cap;
        s_first[8] = mine.start;
        s_first[9] = mine.head;
        int4* d = reinterpret_cast<int4*>(a.desc + c * 8);
        d[0] = make_int4(s, j, p, nt);
        d[1] = make_int4(mine.n_new, total, 0, 0);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *s_tmem;
  ChunkWalk walk;
  walk.left = u1 - u0;
  walk.seg = s_first[0];
  walk.blk = s_first[1];
  walk.p = s_first[2];
  walk.g = ChunkSeg{s_first[3], s_first[4], s_first[5], s_first[6], s_first[7], s_first[8], s_first[9]};
  ChunkItem it;

  if (warp >= kSoft) {
  if (warp == kSoft + 1) {
    // ================= K and V tiles, in the order of their use
    // The entries of the page table are fetched 32 at a time, a lane each (one by one, a trip to memory for every tile, they were slower than the products).
    if (!a.idle_producer) {
      uint32_t n_k = 0, n_v = 0;
      bool ok = true;
      while (ok && walk.next(a, sq, it)) {
        const int n = it.t1 - it.t0;
        const int off = it.g.off, cap = it.g.cap;
        int window = -64, entry = -1;  // lane i holds the list's page window + i
        auto load = [&](const CUtensorMap* pool, const CUtensorMap* ovf, uint32_t dst, uint32_t bar, int t) {
          const int r0 = t * kKeyTile;
          if (r0 < cap) {
            if (lane == 0) {
              mbar_expect_tx(bar, kChTileBytes);
              tma_load_2d(dst, pool, 0, off + r0, bar);
              tma_load_2d(dst + kKBlockBytes, pool, 64, off + r0, bar);
            }
          } else {
            const int p = (r0 - cap) >> 6;
            if (p < window || p + 1 >= window + 32) {  // V tiles before come after this K tile
              window = max(p - 2 * kLead, 0);
              entry = cap + (window + lane) * 64 < it.g.len ? ch_page(a, it.seg, (window + lane) * 64) : -1;
            }
            const int pg0 = __shfl_sync(0xffffffffu, entry, p - window), pg1 = __shfl_sync(0xffffffffu, entry, p + 1 - window);
            if (lane == 0) {
              mbar_expect_tx(bar, (pg0 >= 0 ? kChTileBytes / 2 : 0) + (pg1 >= 0 ? kChTileBytes / 2 : 0));
              if (pg0 >= 0) {
                tma_load_2d(dst, ovf, 0, pg0 * 64, bar);
                tma_load_2d(dst + kKBlockBytes, ovf, 64, pg0 * 64, bar);
              }
              if (pg1 >= 0) {
                tma_load_2d(dst + 64 * 128, ovf, 0, pg1 * 64, bar);
                tma_load_2d(dst + kKBlockBytes + 64 * 128, ovf, 64, pg1 * 64, bar);
              }
            }
          }
          __syncwarp();
        };
        for (int t = -kLead; ok && t < n; ++t) {
          if (t >= 0) {
            const int st = n_v % kStagesV;
            if (n_v >= kStagesV && !(ok = warp_wait(B(kEmptyV + st), ((n_v / kStagesV) - 1) & 1, s_abort, a.spin_limit))) break;
            ++n_v;
            load(&v_map, &vo_map, s_v + st * kChTileBytes, B(kFullV + st), it.t0 + t);
          }
          if (t + kLead < n) {
            const int st = n_k % kStagesK;
            if (n_k >= kStagesK && !(ok = warp_wait(B(kEmptyK + st), ((n_k / kStagesK) - 1) & 1, s_abort, a.spin_limit))) break;
            ++n_k;
            load(&k_map, &ko_map, s_k + st * kChTileBytes, B(kFullK + st), it.t0 + t + kLead);
          }
        }
      }
    }
    __syncwarp();
  } else if (warp == kSoft + 3) {
    // ================= products with V (the whole warp, converged)
    if (!a.idle_producer) {
      const uint32_t idesc = umma_idesc_bf16_bmn(128, 128), tm = (uint32_t)uni((int)tmem);
      const uint64_t dv0 = umma_desc_sw128_mn(s_v, kKBlockBytes);
      uint32_t n_t = 0, fixed = 0;  // tiles; one bit per stage, the parity of its next look
      bool ok = true;
      while (ok && walk.next(a, sq, it)) {
        const int t0 = uni(it.t0), n = uni(it.t1) - t0;
        const int first = uni(it.g.len - it.g.n_new + it.blk * a.TB + 1);
        const int last = uni(it.g.len - it.g.n_new + min(it.g.n_new, a.TB * (it.blk + 1)));
        for (int t = 0; ok && t < n; ++t, ++n_t) {
          const bool look = (t0 + t + 1) * kKeyTile > first, fresh = kFlush ? t % max(kFlush, 1) == 0 : t == 0;
          const int st = n_t % kStagesV, rows = ch_v_rows(last - (t0 + t) * kKeyTile);
          ok = warp_wait(B(kFullV + st), (n_t / kStagesV) & 1, s_abort, a.spin_limit);
          if (ok && look) {
            ok = warp_wait(B(kFixed + st), (fixed >> st) & 1, s_abort, a.spin_limit);
            fixed ^= 1u << st;
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int x = 0; x < kTiles; ++x) {
              const int slot = slot_of(n_t, x, h);
              if (!ok || !(ok = warp_wait(B(kPReady + slot), phase_of(n_t), s_abort, a.spin_limit))) break;
              tc_fence_after();
              const uint64_t dv = dv0 + (uint64_t)(st * (kChTileBytes >> 4) + h * (64 * 128 >> 4));
              const uint32_t d = tm + 256 + x * 128, p = tm + slot * Sh::kSlotCols;
              const bool begin = fresh && h == 0;
              if (elect_one()) {
#pragma unroll
                for (int part = 0; part < kParts; ++part)
#pragma unroll
                  for (int kk = 0; kk < 4; ++kk)
                    if (64 * h + 16 * kk < rows)
                      umma_bf16_ta(kFlush && part ? d + 128 : d, p + part * 32 + kk * 8, dv + (uint64_t)(kk * 128), idesc,
                                   kk || part > (kFlush ? 1 : 0) ? 1u : (begin ? 0u : 1u));
                if (h == 1 && t + 1 == n) umma_commit(B(kDoneO + x));  // (the one that is waited for comes first)
                umma_commit(B(kDonePV + slot));
                if (h == 1 && x == kTiles - 1) umma_commit(B(kEmptyV + st));
              }
            }
          }
        }
      }
    }
    __syncwarp();
  } else if (warp == kSoft + 2) {
    // ================= V tiles with rows that some query of the block does not see
    uint32_t n_v = 0, n_item = 0;
    bool ok = !a.idle_producer;
    while (ok && walk.next(a, sq, it)) {
      const int n = it.t1 - it.t0;
      const int first = it.g.len - it.g.n_new + it.blk * a.TB + 1;                       // rows that every query sees
      const int last = it.g.len - it.g.n_new + min(it.g.n_new, a.TB * (it.blk + 1));     // rows that the last one sees
      bool fresh = true;
      // Every tile is waited for in its order, and its place in the ring is free when this warp has passed it too: a warp that skipped a tile, or fell two
      // uses of a place behind, could take another phase for its own.
      for (int t = 0; ok && t < n; ++t, ++n_v) {
        const int r0 = (it.t0 + t) * kKeyTile, st = n_v % kStagesV;
        if (!(ok = warp_wait(B(kFullV + st), (n_v / kStagesV) & 1, s_abort, a.spin_limit))) break;
        if (r0 + kKeyTile <= first) {
          if (lane == 0) mbar_arrive(B(kEmptyV + st));
          continue;
        }
        if (fresh) {
          // four flags in turn: this block's V tile is in the ring, so the results of the block four before it are out
          if (lane == 0) s_odd[n_item & 3] = 0x7fffffff;
          __syncwarp();
          fresh = false;
        }
        uint8_t* tile = smem + kQBytes + (kStagesK + st) * kChTileBytes;
        auto chunk = [&](int r) { return reinterpret_cast<uint4*>(tile + sw128_off(r, lane & 15, 128)); };  // 16 lanes a row
        int odd = 0x7fffffff;
        const int lo = max(first - r0, 0), hi = min(last - r0, kKeyTile);
        for (int rb = lo; rb < hi; rb += 16) {
          uint4 v[8];
          uint32_t ones = 0;  // sign bits of halves whose exponent is all ones
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int r = rb + 2 * i + (lane >> 4);
            v[i] = r < hi ? *chunk(r) : make_uint4(0u, 0u, 0u, 0u);
          }
#pragma unroll
          for (int i = 0; i < 8; ++i)
            ones |= ((v[i].x & 0x7f807f80u) + 0x00800080u) | ((v[i].y & 0x7f807f80u) + 0x00800080u) | ((v[i].z & 0x7f807f80u) + 0x00800080u) |
                    ((v[i].w & 0x7f807f80u) + 0x00800080u);
          if (!__any_sync(0xffffffffu, (ones & 0x80008000u) != 0)) continue;
          for (int i = 0; i < 8; ++i) {
            const int r = rb + 2 * i + (lane >> 4);
            if (r >= hi) break;
            uint4 y = *chunk(r);
            uint32_t* w = reinterpret_cast<uint32_t*>(&y);
            bool bad = false;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              if ((w[k] & 0x7f80u) == 0x7f80u) bad = true, w[k] &= 0xffff0000u;
              if ((w[k] & 0x7f800000u) == 0x7f800000u) bad = true, w[k] &= 0x0000ffffu;
            }
            if (bad) {
              *chunk(r) = y;
              odd = min(odd, r0 + r);
            }
          }
          __syncwarp();
        }
        const int end = ch_v_rows(last - r0);
        for (int r = max(last - r0, 0) + (lane >> 4); r < end; r += 2) *chunk(r) = make_uint4(0u, 0u, 0u, 0u);
        if (odd != 0x7fffffff) atomicMin(&s_odd[n_item & 3], odd);
        fence_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(B(kFixed + st));
          mbar_arrive(B(kEmptyV + st));
        }
      }
      n_item += fresh ? 0 : 1;
    }
    __syncwarp();
  } else if (warp == kSoft) {
    // ================= the query block of every item, and its logits (the whole warp, converged)
    // Logits and products are issued by a warp each: while one looks at its barriers the other keeps the tensor pipe fed.
    if (!a.idle_producer) {
      const uint32_t idesc = umma_idesc_bf16(128, 64), tm = (uint32_t)uni((int)tmem);
      const uint64_t dq0 = umma_desc_sw128(s_q), dk0 = umma_desc_sw128(s_k);
      uint32_t n_item = 0, n_t = 0;
      int q_rows = 0;  // rows of the query block that are not zeros
      bool ok = true;
      while (ok && walk.next(a, sq, it)) {
        const int n = uni(it.t1 - it.t0);
        if (n_item >= 1 && !(ok = warp_wait(B(kQEmpty), (n_item - 1) & 1, s_abort, a.spin_limit))) break;
        const int loads = (min(it.g.n_new - it.blk * a.TB, a.TB) + a.TQ - 1) / a.TQ, rows = loads * a.TQ * a.G;
        for (int r = rows + (lane >> 3); r < q_rows; r += 4) {  // rows that the block before had
          *reinterpret_cast<uint4*>(smem + r * 128 + (lane & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
          *reinterpret_cast<uint4*>(smem + kQBlock + r * 128 + (lane & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
          if constexpr (kDup) {
            *reinterpret_cast<uint4*>(smem + (64 + r) * 128 + (lane & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
            *reinterpret_cast<uint4*>(smem + kQBlock + (64 + r) * 128 + (lane & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
        }
        if (rows < q_rows) fence_async_smem();
        q_rows = rows;
        if (lane == 0) mbar_expect_tx(B(kQFull), (kDup ? 512 : 256) * rows);
        __syncwarp();
        if (lane < loads) {  // (at most eight)
          const uint32_t dst = s_q + lane * a.TQ * a.G * 128;
          const int token = it.g.start + it.blk * a.TB + lane * a.TQ;
          tma_load_3d(dst, &q_map, 0, it.g.head, token, B(kQFull));
          tma_load_3d(dst + kQBlock, &q_map, 64, it.g.head, token, B(kQFull));
          if constexpr (kDup) {
            tma_load_3d(dst + 64 * 128, &q_map, 0, it.g.head, token, B(kQFull));
            tma_load_3d(dst + kQBlock + 64 * 128, &q_map, 64, it.g.head, token, B(kQFull));
          }
        }
        __syncwarp();
        ok = warp_wait(B(kQFull), n_item & 1, s_abort, a.spin_limit);
        ++n_item;
        for (int t = 0; ok && t < n; ++t, ++n_t) {
          const int st = n_t % kStagesK;
          ok = warp_wait(B(kFullK + st), (n_t / kStagesK) & 1, s_abort, a.spin_limit);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int x = 0; x < kTiles; ++x) {
              const int slot = slot_of(n_t, x, h);
              // the slot's last P has been taken
              if (ok && n_t >= (kSplit ? 2 : 1)) ok = warp_wait(B(kDonePV + slot), phase_of(n_t) ^ 1, s_abort, a.spin_limit);
              if (!ok) break;
              tc_fence_after();
              const uint64_t dq = dq0 + (uint64_t)(x * (128 * 128 >> 4)), dk = dk0 + (uint64_t)(st * (kChTileBytes >> 4) + h * (64 * 128 >> 4));
              const uint32_t d = tm + slot * Sh::kSlotCols;
              if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < 8; ++kk)
                  umma_bf16(d, dq + (uint64_t)((kk >> 2) * (kQBlock >> 4) + (kk & 3) * 2),
                            dk + (uint64_t)((kk >> 2) * (kKBlockBytes >> 4) + (kk & 3) * 2), idesc, kk ? 1u : 0u);
                umma_commit(B(kDoneS + slot));
                if (h == 1 && x == kTiles - 1) {
                  umma_commit(B(kEmptyK + st));
                  if (t + 1 == n) umma_commit(B(kQEmpty));
                }
              }
            }
          }
        }
      }
    }
    __syncwarp();
    }
  } else {
    // ================= softmax; a thread owns a row of its warps' M tile, or (kSplit) the row's share of one step of every tile
    const int g = kSplit ? warp >> 2 : 0, x = kQ2 ? warp >> 2 : 0, quarter = warp & 3;
    const int lane_row = quarter * 32 + lane;
    const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
    const uint32_t acc = tmem + lane_base + 256 + x * 128;
    const int row = kDup ? lane_row & 63 : x * 128 + lane_row;  // row of the block
    const bool low = kDup && quarter >= 2;  // of the copies, whose warps write the low parts
    const int tok = row / a.G;
    float* const s_l = s_ref + 256;
    uint32_t n_s = 0, n_o = 0, n_odd = 0, n_dec = 0, n_x = 0, n_low = 0;
    bool alive = true, first_item = true;
    while (alive && walk.next(a, sq, it)) {
      const int n = it.t1 - it.t0;
      const int first = it.g.len - it.g.n_new + it.blk * a.TB + 1;
      const int token = it.blk * a.TB + tok;
      const bool valid = tok < a.TB && token < it.g.n_new;
      const int sees = it.g.len - it.g.n_new + token + 1;  // rows that this thread's query sees
      const bool idle = !__any_sync(0xffffffffu, valid);   // no row of the warp is a query: it only keeps the barriers going
      const int tile = (blockIdx.x * 2 + (first_item ? 0 : 1)) * kTiles + x;  // of partial results
      first_item = false;
      float ref = valid ? -INFINITY : INFINITY, l = 0.f, sum_ref = -INFINITY;  // (no query: every P is 0)
      float sum[kFlush ? 128 : 1];
      for (int i = 0; alive && i < n; ++i, ++n_s) {
        const bool fresh = kFlush ? i % max(kFlush, 1) == 0 : i == 0;
#pragma unroll 1
        for (int h = kSplit ? g : 0; h < (kSplit ? g + 1 : 2); ++h) {
          const int s_slot = slot_of(n_s, x, h);
          if (!(alive = warp_wait(B(kDoneS + s_slot), phase_of(n_s), s_abort, a.spin_limit))) break;
          if (idle) {
            __syncwarp();
            if (lane == 0) mbar_arrive(B(kPReady + s_slot));
            continue;
          }
          tc_fence_after();
          const uint32_t slot = tmem + lane_base + s_slot * Sh::kSlotCols;
          // the products of the step before (whose slot's earlier phases are behind us: its own S has been read)
          const uint32_t n_b = h == 0 ? n_s - 1 : n_s;
          auto wait_products = [&]() { return warp_wait(B(kDonePV + slot_of(n_b, x, h ^ 1)), phase_of(n_b), s_abort, a.spin_limit); };
          const int k0 = (it.t0 + i) * kKeyTile + 64 * h;
          float y[64];
          tmem_ld64(slot, y);
          tmem_wait_ld64(y);
          if (k0 + 64 > first) {
            const int lim = sees - k0;
#pragma unroll
            for (int c = 0; c < 64; ++c) y[c] = c < lim ? y[c] : -INFINITY;
          }
          const float mx = ch_max<64>(y) * a.scale_log2;
          float ref_o = ref;  // the accumulator's reference
          if (kSplit) {
            // The two steps' threads of a row share its reference: each decides after the other has decided for the step before.  Only that is serial.
            if (n_dec + g > 0 && !(alive = warp_wait(B(kDec + quarter), (n_dec + g - 1) & 1, s_abort, a.spin_limit))) break;
            ref_o = i + g > 0 ? s_ref[(g ^ 1) * 128 + lane_row] : ref;
          }
          const bool grow = mx > ref_o + kChTau;  // also the first step with a visible key
          const float ref_n = grow ? mx : ref_o;
          if (kSplit) {
            s_ref[g * 128 + lane_row] = ref_n;
            __syncwarp();
            if (lane == 0) mbar_arrive(B(kDec + quarter));
          }
          if (__any_sync(0xffffffffu, ref_n > ref)) {
            if (ref_n > ref) l = ref > -INFINITY ? l * fast_exp2(ref - ref_n) : l;
            const float f = grow && ref_o > -INFINITY ? fast_exp2(ref_o - ref_n) : 1.f;
            if ((h == 1 || !fresh) && __any_sync(0xffffffffu, f != 1.f)) {  // the accumulator follows, behind the products of the step before
              if (!(alive = wait_products())) break;
              tc_fence_after();
#pragma unroll 1
              for (int c0 = 0; c0 < (kFlush ? 256 : 128); c0 += 32) {
                float o[32];
                tmem_ld32(acc + c0, o);
                tmem_wait_ld32(o);
#pragma unroll
                for (int c = 0; c < 32; ++c) o[c] *= f;
                tmem_st32(acc + c0, o);
              }
            }
            ref = ref_n;
          }
          const float neg = ref > -INFINITY ? -ref : 0.f;  // nothing seen yet: every P is exp2(-inf) = 0
          if (kFlush) {
#pragma unroll
            for (int c = 0; c < 64; c += 16) l += ch_probs<16, kParts>(y + c, a.scale_log2, neg, slot + c / 2, 32);
          } else if (low) {
            l += ch_probs<32, 2, true>(y, a.scale_log2, neg, slot, 0);
            l += ch_probs<32, 2, true>(y + 32, a.scale_log2, neg, slot + 16, 0);
          } else {
            l += ch_probs<32, kParts>(y, a.scale_log2, neg, slot, 32);
            l += ch_probs<32, kParts>(y + 32, a.scale_log2, neg, slot + 16, 32);
          }
          if (kFlush && h == 0 && fresh && i > 0) {  // what the tensor cores have added up since the last time
            if (!(alive = wait_products())) break;
            tc_fence_after();
            const float f = sum_ref > -INFINITY ? fast_exp2(sum_ref - ref_o) : 0.f;
#pragma unroll
            for (int c0 = 0; c0 < 128; c0 += 16) {
              float o[16], o1[16];
              tmem_ld16(acc + c0, o);
              tmem_ld16(acc + 128 + c0, o1);
              tmem_wait_ld16(o);
              tmem_wait_ld16(o1);
#pragma unroll
              for (int c = 0; c < 16; ++c)
                if constexpr (kFlush > 0) sum[c0 + c] = i > kFlush ? fmaf(sum[c0 + c], f, o[c] + o1[c]) : o[c] + o1[c];
            }
            sum_ref = ref_o;
          }
          tmem_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(B(kPReady + s_slot));
        }
        n_dec += idle ? 0 : 2;
      }
      if (!alive) break;
      if (kSplit) {  // the row's sums of both steps, relative to the last decision (the second step's)
        if (!idle) {
          if (!(alive = warp_wait(B(kDec + quarter), (n_dec - 1) & 1, s_abort, a.spin_limit))) break;
          const float ref_end = s_ref[128 + lane_row];
          if (ref_end > ref) {
            l = ref > -INFINITY ? l * fast_exp2(ref - ref_end) : l;
            ref = ref_end;
          }
        }
        s_l[g * 128 + lane_row] = l;
        __syncwarp();
        if (lane == 0) mbar_arrive(B(kXch + quarter));
        if (!(alive = warp_wait(B(kXch + quarter), n_x & 1, s_abort, a.spin_limit))) break;
        ++n_x;
        l = s_l[lane_row] + s_l[128 + lane_row];
      }
      if (!(alive = warp_wait(B(kDoneO + x), n_o & 1, s_abort, a.spin_limit))) break;
      ++n_o;
      tc_fence_after();
      // ---- the item's result: the whole block, or a piece of it (kSplit: each step's threads write half of d)
      const bool looked = it.t1 * kKeyTile > first;
      const int odd = looked ? s_odd[n_odd & 3] : 0x7fffffff;
      n_odd += looked ? 1 : 0;
      const bool whole = n == it.nt, summed = kFlush && n > kFlush;
      const int64_t orow = (int64_t)(it.g.start + token) * a.Hq + it.g.head + (row - tok * a.G);
      const float fs = sum_ref > -INFINITY ? fast_exp2(sum_ref - ref) : 0.f;
      float4* const part = a.part_o + (int64_t)tile * (32 * a.R) + lane_row;
      const float inv = whole ? (l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l)) : 1.f;  // a NaN stays one
      if (!idle) {
#pragma unroll(kFlush ? 4 : 1)
        for (int cc = 0; cc < (kSplit ? 64 : 128); cc += 32) {
          const int c0 = g * 64 + cc;
          float o[32];
          tmem_ld32(acc + c0, o);
          tmem_wait_ld32(o);
          if constexpr (kFlush > 0) {
            float o1[32];
            tmem_ld32(acc + 128 + c0, o1);
            tmem_wait_ld32(o1);
#pragma unroll
            for (int c = 0; c < 32; ++c) o[c] = summed ? fmaf(sum[cc + c], fs, o[c] + o1[c]) : o[c] + o1[c];
          }
          if constexpr (kDup) {  // the low parts' products, from the copy's warp
            float4* const z = reinterpret_cast<float4*>(s_low + (g * 64 + row) * kLowStride);
            const uint32_t pair = g * 2 + (quarter & 1);
            if (low) {
              if (n_low > 0 && !(alive = warp_wait(B(kLowEmpty + pair), (n_low - 1) & 1, s_abort, a.spin_limit))) break;
#pragma unroll
              for (int c = 0; c < 8; ++c) z[c] = make_float4(o[4 * c], o[4 * c + 1], o[4 * c + 2], o[4 * c + 3]);
            } else {
              if (!(alive = warp_wait(B(kLowFull + pair), n_low & 1, s_abort, a.spin_limit))) break;
#pragma unroll
              for (int c = 0; c < 8; ++c) {
                const float4 w = z[c];
                o[4 * c] += w.x, o[4 * c + 1] += w.y, o[4 * c + 2] += w.z, o[4 * c + 3] += w.w;
              }
            }
            ++n_low;
            __syncwarp();
            if (lane == 0) mbar_arrive(B((low ? kLowFull : kLowEmpty) + pair));
            if (low) continue;
          }
          if (odd < sees && valid) {  // infinities and NaN that were taken out of the V tiles
            const int off = it.g.off, cap = it.g.cap;
            for (int j = max(odd, it.t0 * kKeyTile); j < min(sees, it.t1 * kKeyTile); ++j) {
              const uint16_t* v = a.v_pool + (int64_t)(off + j) * kD;
              if (j >= cap) {
                const int pg = ch_page(a, it.seg, j - cap);
                if (pg < 0) continue;
                v = a.v_ovf + ((int64_t)pg * 64 + ((j - cap) & 63)) * kD;
              }
#pragma unroll
              for (int c = 0; c < 32; ++c) {
                const uint32_t w = (uint32_t)v[c0 + c] << 16;
                if ((w & 0x7f800000u) == 0x7f800000u) o[c] += __uint_as_float(w);
              }
            }
          }
          if (valid) {
            if (!whole) {
#pragma unroll
              for (int c = 0; c < 8; ++c) part[(c0 / 4 + c) * a.R] = make_float4(o[4 * c], o[4 * c + 1], o[4 * c + 2], o[4 * c + 3]);
            } else {
              uint8_t* dst = reinterpret_cast<uint8_t*>(a.out) + (orow * kD + c0) * (kFlush ? 4 : 2);
              const bool sector = (reinterpret_cast<uintptr_t>(a.out) & 31) == 0;
#pragma unroll
              for (int c = 0; c < 32; c += kFlush ? 8 : 16) {
                uint32_t w[8];
#pragma unroll
                for (int k = 0; k < 8; ++k)
                  w[k] = kFlush ? __float_as_uint(o[c + k] * inv) : pack_bf16(o[(c + 2 * k) & 31] * inv, o[(c + 2 * k + 1) & 31] * inv);
                st_row32(dst + c * (kFlush ? 4 : 2), w, sector);
              }
            }
          }
        }
        if (!alive) break;
        if (valid && g == 0 && !low) {
          if (!whole) a.part_ml[(int64_t)tile * a.R + lane_row] = make_float2(ref, l);
          else if (a.lse) a.lse[orow] = l == 0.f ? -INFINITY : (ref + log2f(l)) * 0.6931471805599453f;
        }
      }
      tc_fence_before();
      if (kSplit) {  // the other step's threads have read the accumulator too: the next block's products may overwrite it
        __syncwarp();
        if (lane == 0) mbar_arrive(B(kXch + quarter));
        if (!(alive = warp_wait(B(kXch + quarter), n_x & 1, s_abort, a.spin_limit))) break;
        ++n_x;
      }
    }
  }

  // ---- release tensor memory (after an abort: first give copies that may still be in flight time to land)
  if (*s_abort)
    for (int i = 0; i < 200; ++i) __nanosleep(1000);
  tc_fence_before();
  __syncthreads();
  if (warp == kSoft) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(kChTmemCols) : "memory");
  if (*s_abort && tid == 0) raise_status(a.status, CATEKV_STATUS_WAIT_EXPIRED, kKidChunk, walk.seg, (int)blockIdx.x);
}

// Merge the pieces of the blocks that several CTAs share, in the order of the keys: CTA c's descriptor says whether its share
// begins inside a block; the first such CTA of a block has it merged.  A thread block takes kRows rows, a thread kVec float4 of a row; what threads are
// left share out the pieces (few rows of one long list come in up to 148), and the groups' sums are merged in their order.  Bound by its trips
// to memory: descriptors, pieces; so references are not looked through first, the sums follow them piece by piece (24 blocks of 126 rows in 7 pieces:
// 7.1 us; 147 blocks of 128 rows in 2 pieces 10 us; one list of 60 K rows in 148 pieces 9.3 us).
struct ChunkSum {
  float m, l;  // reference (log2 domain), sum
  // the weights of what is there and of what comes; a part that sees no key has nothing to add, or the NaN that it has met
  __device__ __forceinline__ float2 add(float m2, float l2) {
    float f = 1.f, w = l2 == 0.f ? 0.f : 1.f;
    if (m2 > -INFINITY) {
      const float top = fmaxf(m, m2);
      f = m > -INFINITY ? fast_exp2(m - top) : 1.f;
      w = fast_exp2(m2 - top);
      m = top;
    }
    l = fmaf(w, l2, l * f);
    return make_float2(f, w);
  }
};
__device__ __forceinline__ void ch_blend(float4& acc, const float4& v, float2 fw) {
  acc.x = fmaf(fw.y, v.x, acc.x * fw.x);
  acc.y = fmaf(fw.y, v.y, acc.y * fw.x);
  acc.z = fmaf(fw.y, v.z, acc.z * fw.x);
  acc.w = fmaf(fw.y, v.w, acc.w * fw.x);
}
template <int kRows, int kThreads, int kVec>
__global__ void __launch_bounds__(kThreads) chunk_combine_kernel(const __grid_constant__ ChunkArgs a, const __grid_constant__ ChunkSeqs sq,
                                                                          int C, int two) {
  constexpr int kCols = 32 / kVec, kGroups = kThreads / (kRows * kCols), kAtOnce = 4;
  __shared__ float4 s_o[kGroups][kRows][33];
  __shared__ float2 s_ml[kGroups][kRows];
  pdl_launch_dependents();
  pdl_wait();
  // the blockIdx.x-th CTA that has a block merged (launched for all CTAs, most thread blocks would find nothing to do, at 5 ns each)
  __shared__ int s_flags[kThreads / 32], s_pick;
  __shared__ int4 s_desc[2];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  {
    const int c = threadIdx.x;
    bool merges = false;
    int4 d0, d1;
    if (c > 0 && c < C) {
      d0 = reinterpret_cast<const int4*>(a.desc)[c * 2];
      d1 = reinterpret_cast<const int4*>(a.desc)[c * 2 + 1];
      const int total = d1.y, q = total / C, r = total - q * C;
      const int ub = c * q + min(c, r) - d0.z;
      merges = ch_tile_at(a, d0.z) > 0 && ch_tile_at(a, (c - 1) * q + min(c - 1, r) - ub) == 0;  // (no earlier CTA begins inside the block)
    }
    const uint32_t flags = __ballot_sync(0xffffffffu, merges);
    if (lane == 0) s_flags[warp] = __popc(flags);
    __syncthreads();
    int rank = __popc(flags & ((1u << lane) - 1)), all = 0;
#pragma unroll
    for (int w = 0; w < (kThreads < kChMaxCtas ? kThreads : kChMaxCtas) / 32; ++w) {
      rank += w < warp ? s_flags[w] : 0;
      all += s_flags[w];
    }
    if ((int)blockIdx.x >= all) return;
    if (merges && rank == (int)blockIdx.x) {
      s_pick = c;
      s_desc[0] = d0;
      s_desc[1] = d1;
    }
    __syncthreads();
  }
  const int c = s_pick;
  const int4 d0 = s_desc[0], d1 = s_desc[1];
  const int seg = d0.x, blk = d0.y, nt = d0.w, n_new = d1.x, total = d1.y;
  const int q = total / C, r = total % C;
  auto begin = [&](int i) { return i * q + min(i, r); };
  const int ub = begin(c) - d0.z, ue = ub + nt + a.charge;  // the block's units
  // the CTAs that begin before its end: begin(k) < ue
  int c_end = q ? (ue > r * (q + 1) ? r + (ue - r * (q + 1) + q - 1) / q : (ue + q) / (q + 1)) : min(ue, C);
  c_end = min(c_end, C);
  const int head = begin(c - 1) < ub ? 1 : 0;  // the first piece: the last block of CTA c - 1, or its only one
  const int b = seg / a.Hkv, h = seg - b * a.Hkv;
  const int row0 = blockIdx.y * kRows, x = row0 >> 7;  // row of the block; its M tile
  if (blk * a.TB + row0 / a.G >= n_new) return;
  auto tile = [&](int k) {
    const int i = k == c - 1 ? head : 0;
    return (int64_t)(two ? (k * 2 + i) * 2 + x : k * 2 + i);
  };
  const int i_row = threadIdx.x % kRows, c4 = threadIdx.x / kRows % kCols, group = threadIdx.x / (kRows * kCols);
  const int row = row0 + i_row, in_tile = row & 127, n = c_end - (c - 1);
  const bool valid = row / a.G < a.TB && blk * a.TB + row / a.G < n_new;
  ChunkSum sum = {-INFINITY, 0.f};
  float4 acc[kVec];
#pragma unroll
  for (int j = 0; j < kVec; ++j) acc[j] = make_float4(0.f, 0.f, 0.f, 0.f);
  if (valid) {
    const int k_hi = c - 1 + n * (group + 1) / kGroups;
    for (int k0 = c - 1 + n * group / kGroups; k0 < k_hi; k0 += kAtOnce) {
      float2 ml[kAtOnce];
      float4 v[kAtOnce][kVec];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u)
        if (k0 + u < k_hi) {
          const int64_t t = tile(k0 + u);
          ml[u] = a.part_ml[t * a.R + in_tile];
#pragma unroll
          for (int j = 0; j < kVec; ++j) v[u][j] = a.part_o[t * (32 * a.R) + (c4 + j * kCols) * a.R + in_tile];
        }
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u)
        if (k0 + u < k_hi) {
          const float2 fw = sum.add(ml[u].x, ml[u].y);
#pragma unroll
          for (int j = 0; j < kVec; ++j) ch_blend(acc[j], v[u][j], fw);
        }
    }
  }
#pragma unroll
  for (int j = 0; j < kVec; ++j) s_o[group][i_row][c4 + j * kCols] = acc[j];
  if (c4 == 0) s_ml[group][i_row] = make_float2(sum.m, sum.l);
  __syncthreads();
  // a warp a row now: its lanes write it side by side
  for (int i = warp; i < kRows; i += kThreads / 32) {
    const int tok = (row0 + i) / a.G;
    if (tok >= a.TB || blk * a.TB + tok >= n_new) continue;
    float4 v = s_o[0][i][lane];
    sum = ChunkSum{s_ml[0][i].x, s_ml[0][i].y};
#pragma unroll 4
    for (int g = 1; g < kGroups; ++g) ch_blend(v, s_o[g][i][lane], sum.add(s_ml[g][i].x, s_ml[g][i].y));
    const float inv = sum.l > 0.f ? 1.f / sum.l : (sum.l == 0.f ? 0.f : sum.l);
    const int64_t orow = (int64_t)(sq.start[b] + blk * a.TB + tok) * a.Hq + h * a.G + (row0 + i) % a.G;
    if (a.out_fp32) {
      reinterpret_cast<float4*>(a.out)[orow * 32 + lane] = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
    } else {
      uint2 pk;
      pk.x = pack_bf16(v.x * inv, v.y * inv);
      pk.y = pack_bf16(v.z * inv, v.w * inv);
      reinterpret_cast<uint2*>(a.out)[orow * 32 + lane] = pk;
    }
    if (lane == 0 && a.lse) a.lse[orow] = sum.l == 0.f ? -INFINITY : (sum.m + log2f(sum.l)) * 0.6931471805599453f;
  }
}
template <int kRows, int kThreads, int kVec>
static cudaError_t launch_combine(const ChunkArgs& a, const ChunkSeqs& sq, int blocks, int ctas, bool two, cudaStream_t st) {
  static_assert(kThreads >= kChMaxCtas, "a thread looks at a CTA");
  return launch_pdl(chunk_combine_kernel<kRows, kThreads, kVec>, dim3(blocks, ((two ? 256 : a.R) + kRows - 1) / kRows), dim3(kThreads), 0, st, a, sq,
                    ctas, two ? 1 : 0);
}

// ---- append: the chunk's rows behind the end of every list.  A warp copies a row (lanes 0-15 K, 16-31 V), eight in flight.  Bound by the copy: 4096
// tokens of 4 sequences and 8 heads, 67 MB written, in 17 us, part of it still in L2; a few tokens: one launch, 2 to 3 us.
struct AppendArgs {
  uint8_t* k_pool;
  uint8_t* v_pool;
  const int32_t* seg_off;
  int32_t* seg_len;
  const int32_t* seg_cap;
  PageArgs pg;
  int32_t n_pages, Hkv;
  const uint8_t* k_new;
  const uint8_t* v_new;
  int64_t stride_t, stride_h;  // bytes
  int32_t* checked;
};
constexpr int kApRows = 64;  // rows of a block
// rows that fit: the capacity and the pages that the table names
__device__ __forceinline__ uint8_t* ap_row(const AppendArgs& a, int seg, int r, bool v) {
  const int cap = a.seg_cap[seg];
  if (r < cap) return (v ? a.v_pool : a.k_pool) + ((int64_t)a.seg_off[seg] + r) * kRowBytes;
  const int o = r - cap, p = o >> 6;
  if (!a.pg.table || p >= a.pg.max_pages) return nullptr;
  const int pg = a.pg.table[(int64_t)seg * a.pg.max_pages + p];
#ifdef CATEKV_CHECKED
  if (pg >= a.n_pages) raise_status(a.checked, CATEKV_STATUS_INDEX_RANGE, kKidChunk, seg, pg);  // (-1: where the list's room ends)
#endif
  if (pg < 0 || pg >= a.n_pages) return nullptr;
  return (v ? a.pg.v_ovf : a.pg.k_ovf) + ((int64_t)pg * 64 + (o & 63)) * kRowBytes;
}
// How many of n rows behind the list's len fit: all of them, unless a replayed call has found the list full.
__device__ __forceinline__ int ap_fitting(const AppendArgs& a, int seg, int len, int n) {
  while (n > 0 && !ap_row(a, seg, len + n - 1, false)) n = max(0, a.seg_cap[seg] + (len + n - 1 - a.seg_cap[seg]) / 64 * 64 - len);
  return n;
}
// One block takes kApRows rows of a list.  kAlone: every list's rows fit one block, which also counts them in.  The kernel does not signal its dependents
// early: rows that were taken back (catekv_truncate) and come anew may be rows that a decode plan knows, which attention under it requests at its start.
template <bool kAlone>
__global__ void __launch_bounds__(256) append_chunk_kernel(const __grid_constant__ AppendArgs a, const __grid_constant__ ChunkSeqs sq) {
  const int seg = blockIdx.x, b = seg / a.Hkv, h = seg - b * a.Hkv;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = (lane & 15) * 16;
  const int n = sq.n_new[b], r0 = blockIdx.y * kApRows;
  if (r0 >= n) return;
  pdl_wait();
  const int len = a.seg_len[seg];
  const uint8_t* src = (lane < 16 ? a.k_new : a.v_new) + (int64_t)(sq.start[b]) * a.stride_t + h * a.stride_h + c;
  uint4 v[kApRows / 8];
#pragma unroll
  for (int i = 0; i < kApRows / 8; ++i) {
    const int r = r0 + warp + 8 * i;
    if (r < n) v[i] = __ldg(reinterpret_cast<const uint4*>(src + r * a.stride_t));
  }
#pragma unroll
  for (int i = 0; i < kApRows / 8; ++i) {
    const int r = r0 + warp + 8 * i;
    if (r >= n) break;
    uint8_t* dst = ap_row(a, seg, len + r, lane >= 16);
    if (dst) *reinterpret_cast<uint4*>(dst + c) = v[i];
  }
  if (kAlone) {
    __syncthreads();
    if (threadIdx.x == 0) {
      a.seg_len[seg] = len + ap_fitting(a, seg, len, n);
    }
  }
}
__global__ void __launch_bounds__(128) append_count_kernel(const __grid_constant__ AppendArgs a, const __grid_constant__ ChunkSeqs sq, int n_segs) {
  pdl_launch_dependents();
  pdl_wait();
  const int seg = blockIdx.x * 128 + threadIdx.x;
  if (seg >= n_segs) return;
  const int n = sq.n_new[seg / a.Hkv], len = a.seg_len[seg];
  if (n) a.seg_len[seg] = len + ap_fitting(a, seg, len, n);
}

// ---- host
static int take_chunk(const catekv_cache* c, const catekv_chunk* ch, ChunkSeqs* sq, int* max_new, int64_t* sum) {
  if (!ch || !ch->n_new || ch->B != c->B || ch->n_tokens < 0) return CATEKV_ERR_INVALID_ARG;
  if (ch->B > kChMaxSeqs) return CATEKV_ERR_UNSUPPORTED;
  int64_t at = 0;
  *max_new = 0;
  *sum = 0;
  bool ascending = true;
  int64_t end = 0;
  for (int b = 0; b < ch->B; ++b) {
    const int n = ch->n_new[b];
    if (n < 0) return CATEKV_ERR_INVALID_ARG;
    if (ch->start) at = ch->start[b];
    if (at < 0 || at + n > ch->n_tokens) return CATEKV_ERR_INVALID_ARG;
    sq->n_new[b] = n;
    sq->start[b] = (int32_t)at;
    if (n) {
      ascending = ascending && at >= end;
      end = at + n;
    }
    at += n;
    *sum += n;
    *max_new = n > *max_new ? n : *max_new;
  }
  if (!ascending)  // in another order: no token belongs to two sequences
    for (int b = 0; b < ch->B; ++b)
      for (int i = 0; i < b; ++i)
        if (sq->n_new[b] && sq->n_new[i] && sq->start[b] < sq->start[i] + sq->n_new[i] && sq->start[i] < sq->start[b] + sq->n_new[b])
          return CATEKV_ERR_INVALID_ARG;
  return CATEKV_OK;
}
static const int32_t* caps_on_device(const catekv_cache* c) { return c->pages ? c->pages->seg_cap_dev : c->seg_cap_dev; }

struct ChunkWs {
  size_t off_desc, off_ml, off_o, bytes;
  int R;
};
// one M tile where no sequence has more rows than it holds
static bool ch_two_tiles(int G, int max_new) { return (int64_t)G * max_new > 128; }
static ChunkWs chunk_ws_layout(int G, int max_new) {
  ChunkWs w;
  const int64_t rows = (int64_t)G * max_new;
  w.R = rows < 128 ? (int)rows : 128;
  const size_t tiles = (ch_two_tiles(G, max_new) ? 4 : 2) * (size_t)sm_count();
  size_t o = CATEKV_STATUS_BYTES;
  w.off_desc = o; o = align_up(o + (size_t)sm_count() * 8 * sizeof(int32_t), 256);
  w.off_ml = o; o = align_up(o + tiles * w.R * sizeof(float2), 256);
  w.off_o = o; o = align_up(o + tiles * w.R * (size_t)kD * sizeof(float), 256);
  w.bytes = o;
  return w;
}
static int make_pool_map(const void* p, int64_t rows, int box_rows, CUtensorMap* map) {
  EncodeTiledFn enc = encode_tiled_fn();
  if (!enc) return CATEKV_ERR_CUDA;
  if ((uintptr_t)p & 15) return CATEKV_ERR_INVALID_ARG;
  const cuuint64_t dims[2] = {(cuuint64_t)kD, (cuuint64_t)(rows > 0 ? rows : 1)};
  const cuuint64_t strides[1] = {kRowBytes};
  const cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
  const cuuint32_t estr[2] = {1, 1};
  const CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? CATEKV_OK : CATEKV_ERR_UNSUPPORTED;
}
static int make_q_map(const void* q, int n_tokens, int Hq, int G, int TB, int64_t st, int64_t sh, CUtensorMap* map) {
  EncodeTiledFn enc = encode_tiled_fn();
  if (!enc) return CATEKV_ERR_CUDA;
  const cuuint64_t dims[3] = {(cuuint64_t)kD, (cuuint64_t)Hq, (cuuint64_t)n_tokens};
  const cuuint64_t strides[2] = {(cuuint64_t)(Hq > 1 ? sh * 2 : kRowBytes), (cuuint64_t)(n_tokens > 1 ? st * 2 : kRowBytes)};
  const cuuint32_t box[3] = {64, (cuuint32_t)G, (cuuint32_t)TB};
  const cuuint32_t estr[3] = {1, 1, 1};
  const CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(q), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? CATEKV_OK : CATEKV_ERR_UNSUPPORTED;
}

template <bool kQ2, int kParts, int kFlush, bool kDup>
static int launch_chunk(int ctas, const CUtensorMap* m, const ChunkArgs& a, const ChunkSeqs& sq, cudaStream_t st) {
  static std::atomic<bool> attr_set[64];
  int dev = 0;
  CATEKV_CUDA_TRY(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64 || !attr_set[dev].load(std::memory_order_acquire)) {
    CATEKV_CUDA_TRY(cudaFuncSetAttribute(chunk_attn_kernel<kQ2, kParts, kFlush, kDup>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)ChunkShape<kQ2, kFlush, kDup>::kSmem));
    if (dev >= 0 && dev < 64) attr_set[dev].store(true, std::memory_order_release);
  }
  CATEKV_CUDA_TRY(launch_pdl(chunk_attn_kernel<kQ2, kParts, kFlush, kDup>, dim3(ctas), dim3(ChunkShape<kQ2, kFlush, kDup>::kThreads), ChunkShape<kQ2, kFlush, kDup>::kSmem, st, m[0], m[1], m[2], m[3], m[4],
                             a, sq));
  return CATEKV_OK;
}
}  // namespace catekv

using namespace catekv;

extern "C" int catekv_append_chunk(catekv_cache* cache, const catekv_chunk* chunk, const void* k_new, const void* v_new, int64_t stride_t,
                                   int64_t stride_h, catekv_stream stream) {
  CATEKV_API_RANGE();
  int rc = check_cache(cache);
  if (rc) return rc;
  ChunkSeqs sq;
  int max_new = 0;
  int64_t sum = 0;
  rc = take_chunk(cache, chunk, &sq, &max_new, &sum);
  if (rc) return rc;
  const int n_segs = cache->B * cache->Hkv;
  for (int s = 0; s < n_segs; ++s) {
    const int n = sq.n_new[s / cache->Hkv];
    if (cache->seg_len[s] < 0) return CATEKV_ERR_INVALID_ARG;
    if (n && (int64_t)cache->seg_len[s] + n > seg_capacity(cache, s)) return CATEKV_ERR_CAPACITY;
  }
  if (!caps_on_device(cache)) return CATEKV_ERR_INVALID_ARG;
  if (sum == 0) return CATEKV_OK;
  if (!k_new || !v_new || (((uintptr_t)k_new | (uintptr_t)v_new) & 15)) return CATEKV_ERR_INVALID_ARG;
  if (stride_t % 8 || stride_h % 8 || (stride_t < kD && chunk->n_tokens > 1) || (stride_h < kD && cache->Hkv > 1)) return CATEKV_ERR_UNSUPPORTED;
  const int blocks = (max_new + kApRows - 1) / kApRows;
  if (blocks > 65535) return CATEKV_ERR_UNSUPPORTED;
  AppendArgs a = {};
  a.k_pool = (uint8_t*)cache->k_pool;
  a.v_pool = (uint8_t*)cache->v_pool;
  a.seg_off = cache->seg_off_dev;
  a.seg_len = cache->seg_len_dev;
  a.seg_cap = caps_on_device(cache);
  a.pg = page_args(cache);
  a.n_pages = cache->pages ? cache->pages->n_pages : 0;
  a.Hkv = cache->Hkv;
  a.k_new = (const uint8_t*)k_new;
  a.v_new = (const uint8_t*)v_new;
  a.stride_t = stride_t * 2;
  a.stride_h = stride_h * 2;
  a.checked = checked_status_ptr();
  cudaStream_t st = (cudaStream_t)stream;
  if (blocks == 1) {
    CATEKV_CUDA_TRY(launch_pdl(append_chunk_kernel<true>, dim3(n_segs), dim3(256), 0, st, a, sq));
  } else {
    CATEKV_CUDA_TRY(launch_pdl(append_chunk_kernel<false>, dim3(n_segs, blocks), dim3(256), 0, st, a, sq));
    CATEKV_CUDA_TRY(launch_pdl(append_count_kernel, dim3((n_segs + 127) / 128), dim3(128), 0, st, a, sq, n_segs));
  }
  for (int s = 0; s < n_segs; ++s) cache->seg_len[s] += sq.n_new[s / cache->Hkv];
  return CATEKV_OK;
}

extern "C" size_t catekv_chunk_attn_workspace_bytes(int32_t Hq, int32_t Hkv, int32_t max_new) {
  if (Hq <= 0 || Hkv <= 0 || Hq % Hkv || Hq / Hkv > kMaxG || max_new < 0) return 0;
  return chunk_ws_layout(Hq / Hkv, max_new > 0 ? max_new : 1).bytes;
}

extern "C" int catekv_chunk_attn(const catekv_cache* cache, const catekv_chunk* chunk, const void* q, int64_t q_stride_t, int64_t q_stride_h,
                                 int32_t Hq, float sm_scale, void* out, int32_t out_dtype, float* lse_out, void* ws, size_t ws_bytes,
                                 catekv_stream stream) {
  CATEKV_API_RANGE();
  int rc = check_cache(cache);
  if (rc) return rc;
  ChunkSeqs sq;
  int max_new = 0;
  int64_t sum = 0;
  rc = take_chunk(cache, chunk, &sq, &max_new, &sum);
  if (rc) return rc;
  if (Hq <= 0 || Hq % cache->Hkv || !(sm_scale >= 0.f && sm_scale <= 2.0e38f) || !caps_on_device(cache)) return CATEKV_ERR_INVALID_ARG;
  const int G = Hq / cache->Hkv;
  if (G > kMaxG || (out_dtype != CATEKV_OUT_BF16 && out_dtype != CATEKV_OUT_FP32)) return CATEKV_ERR_UNSUPPORTED;
  const int n_segs = cache->B * cache->Hkv;
  int64_t units_of[2] = {0, 0}, blocks_of[2] = {0, 0};  // tiles and blocks with one M tile, with two
  int64_t most = 0;  // what the schedule could count up to, if a replayed call found the lists full, with all the pages that they may be given by then
  const int64_t page_rows = cache->pages ? (int64_t)CATEKV_PAGE_ROWS * (cache->pages->max_pages < cache->pages->n_pages ? cache->pages->max_pages : cache->pages->n_pages) : 0;
  int64_t rows = 0;  // of the lists that have queries
  for (int s = 0; s < n_segs; ++s) {
    const int n = sq.n_new[s / cache->Hkv], len = cache->seg_len[s];
    if (cache->seg_cap[s] < 0 || cache->seg_cap[s] % CATEKV_SEG_ALIGN || cache->seg_off[s] < 0) return CATEKV_ERR_INVALID_ARG;
    if (len < n || len > seg_capacity(cache, s)) return CATEKV_ERR_INVALID_ARG;  // the chunk's rows are the list's last ones
    if (n) rows += len;
    for (int w = 0; w < 2; ++w) {
      const int TB = (w ? 256 : 128) / G;
      blocks_of[w] += (n + TB - 1) / TB;
      if (w == 0) most += (int64_t)((n + TB - 1) / TB) * ((cache->seg_cap[s] + page_rows) / kKeyTile + 1 + kChCharge);
      for (int j = 0; j < n; j += TB) units_of[w] += (len - n + (n < j + TB ? n : j + TB) + kKeyTile - 1) / kKeyTile;
    }
  }
  // Two M tiles read K and V half as often.  Where L2 holds them that is no gain, and one M tile, whose steps have warps of their own, is faster (512 tokens over
  // 8 x 16 K rows 155 us with one, 165 with two; 4096 alone 179 and 185; 8 x 100 tokens over 2000 rows 63 and 71); where it does not, the second reading
  // comes from DRAM (512 tokens over 8 x 32 K rows 340 and 308, 8 x 48 K 532 and 463, 3 x 117 K 466 and 417).  Unless so many sequences have a few tokens only
  // that the blocks would be half empty (over 8 x 65 K rows each: 512 tokens beside two single ones, 0.56 of the tiles, 790 and 771; beside four, 0.6, 897
  // and 904; 512 beside 31 over 8 x 8000 rows 229 and 371).
  const bool two = out_dtype == CATEKV_OUT_BF16 && rows > kChL2Rows && units_of[1] * 5 < units_of[0] * 3;
  const int TB = (two ? 256 : 128) / G;
  const int box = 32 % G == 0 ? 32 / G : TB, TQ = max_new < box ? max_new : box;  // loads of 32 rows, where tokens come to that
  const int64_t units = units_of[two], blocks = blocks_of[two];
  if (sum == 0) return CATEKV_OK;
  if (most > 0x7fffffff) return CATEKV_ERR_UNSUPPORTED;  // (a minute's work: such a chunk is brought in by parts)
  if (!q || !out || !ws || (((uintptr_t)q | (uintptr_t)out | (uintptr_t)ws) & 15) || ((uintptr_t)lse_out & 3)) return CATEKV_ERR_INVALID_ARG;
  if ((Hq > 1 && (q_stride_h < kD || q_stride_h % 8)) || (chunk->n_tokens > 1 && (q_stride_t < kD || q_stride_t % 8))) return CATEKV_ERR_UNSUPPORTED;
  const ChunkWs W = chunk_ws_layout(G, max_new);
  if (ws_bytes < W.bytes) return CATEKV_ERR_WORKSPACE;
  CUtensorMap m[5];
  rc = make_pool_map(cache->k_pool, cache->total_rows, kKeyTile, &m[0]);
  if (!rc) rc = make_pool_map(cache->v_pool, cache->total_rows, kKeyTile, &m[1]);
  const catekv_pages* pg = cache->pages;
  if (!rc) rc = make_pool_map(pg ? pg->k_ovf : cache->k_pool, pg ? (int64_t)pg->n_pages * CATEKV_PAGE_ROWS : cache->total_rows, CATEKV_PAGE_ROWS, &m[2]);
  if (!rc) rc = make_pool_map(pg ? pg->v_ovf : cache->v_pool, pg ? (int64_t)pg->n_pages * CATEKV_PAGE_ROWS : cache->total_rows, CATEKV_PAGE_ROWS, &m[3]);
  if (!rc) rc = make_q_map(q, chunk->n_tokens, Hq, G, TQ, q_stride_t, q_stride_h, &m[4]);
  if (rc) return rc;
  uint8_t* w8 = (uint8_t*)ws;
  ChunkArgs a = {};
  a.seg_off = cache->seg_off_dev;
  a.seg_len = cache->seg_len_dev;
  a.seg_cap = caps_on_device(cache);
  a.v_pool = (const uint16_t*)cache->v_pool;
  if (pg) {
    a.v_ovf = (const uint16_t*)pg->v_ovf;
    a.table = pg->table_dev;
    a.max_pages = pg->max_pages;
    a.n_pages = pg->n_pages;
  }
  a.n_segs = n_segs;
  a.Hkv = cache->Hkv;
  a.G = G;
  a.Hq = Hq;
  a.TB = TB;
  a.TQ = TQ;
  a.R = W.R;
  a.charge = two ? kChChargeTwo : kChCharge;
  a.scale_log2 = (sm_scale == 0.f ? 1.f / sqrtf((float)kD) : sm_scale) * 1.4426950408889634f;
  a.out = out;
  a.lse = lse_out;
  a.out_fp32 = out_dtype == CATEKV_OUT_FP32;
  a.desc = (int32_t*)(w8 + W.off_desc);
  a.part_ml = (float2*)(w8 + W.off_ml);
  a.part_o = (float4*)(w8 + W.off_o);
  a.status = (int32_t*)w8;
  a.checked = checked_status_ptr();
  a.spin_limit = kSpinLimit;
  if (score_take_expire_launch()) {
    a.spin_limit = 512;
    a.idle_producer = 1;
  }
  // As many shares as there are tiles, up to one a CTA; short lists stay whole (a merge costs 2 us, a further tile 0.8, in fp32 1.2: a token over 8 lists of
  // 200 rows 7.8 against 10.1 us, 4 x 500 rows of 8 heads 10.4 against 11.7; but 8 lists of 600 rows 11 whole, 10.3 cut, and in fp32 of 500 rows 16.7 and 14.2).
  const int64_t shares = units <= (a.out_fp32 ? 3 : 4) * blocks ? blocks : units;
  const int most_ctas = sm_count() < kChMaxCtas ? sm_count() : kChMaxCtas, ctas = (int)(shares < most_ctas ? shares : most_ctas);
  // Low parts of P in rows of their own, where at most half of the M tile's rows are queries and the stream is long: half the products, and at the power
  // limit that is time (4 tokens of 16 x 32 K rows back to back 400 us without, 367 with; a token over 8 x 32 K rows, 14 tiles a CTA, 31.1 and 30.5; 4 tokens of
  // 16 x 1 K rows, 7 tiles, 19.4 and 20.3: results are handed from warp to warp).
  const bool dup = (int64_t)G * max_new <= 64 && units >= 12 * (int64_t)sm_count();
  cudaStream_t st = (cudaStream_t)stream;
  rc = a.out_fp32 ? launch_chunk<false, 3, 3, false>(ctas, m, a, sq, st)
       : two      ? launch_chunk<true, 2, 0, false>(ctas, m, a, sq, st)
       : dup      ? launch_chunk<false, 1, 0, true>(ctas, m, a, sq, st)
                  : launch_chunk<false, 2, 0, false>(ctas, m, a, sq, st);
  if (rc) return rc;
  if (ctas == 1) return CATEKV_OK;
  const int merged = (int)(blocks < ctas - 1 ? blocks : ctas - 1);  // blocks that may be cut
  // Threads to share out the pieces where a block of queries is cut into many (one list of 60 K rows, 149 pieces: 9.3 us with one row a thread block, 11
  // with 4, 20 with 8; 8 lists of 2 K, 19 pieces of 4 rows: 5.5 with 4, 7.9 with 32), more rows where it is into few (3 lists of 118 K and 512
  // tokens, 7 pieces of 256 rows: 8.6 us with 32, 13.7 with 8; 32 lists of 16 K, 5 pieces of 16 rows: 6.8 and 5.5).
  const int pieces = ctas / merged + 1;
  const cudaError_t e = pieces > 96   ? launch_combine<1, 1024, 1>(a, sq, merged, ctas, two, st)
                        : pieces > 12 ? launch_combine<4, 1024, 1>(a, sq, merged, ctas, two, st)
                        : a.R <= 16   ? launch_combine<8, 512, 1>(a, sq, merged, ctas, two, st)
                                      : launch_combine<32, 256, 4>(a, sq, merged, ctas, two, st);
  CATEKV_CUDA_TRY(e);
  return CATEKV_OK;
}
