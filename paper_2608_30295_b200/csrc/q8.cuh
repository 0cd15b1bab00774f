// Shared by the sources of the 8-bit cache: host checks, the two code types on the device.
#pragma once

#include <cuda_fp16.h>

#include "decode.cuh"

namespace catekv {

constexpr int kQ8Block = CATEKV_Q8_BLOCK;      // rows of a block: one scale each for K and V
constexpr int kQ8RowBytes = kD;                // one row of codes
constexpr int kQ8BlockBytes = kQ8Block * kQ8RowBytes;

// every pointer, the types, and that the segments lie block-aligned inside the pools
static int check_q8_cache(const catekv_q8_cache* c) {
  if (!c) return CATEKV_ERR_INVALID_ARG;
  if (c->B <= 0 || c->Hkv <= 0 || c->total_rows < 0) return CATEKV_ERR_INVALID_ARG;
  if (c->d != kD) return CATEKV_ERR_UNSUPPORTED;
  if (c->dtype != CATEKV_Q8_E4M3 && c->dtype != CATEKV_Q8_INT8) return CATEKV_ERR_UNSUPPORTED;
  if (!c->k_pool || !c->v_pool || !c->k_scale || !c->v_scale || !c->k_tail || !c->v_tail || !c->seg_off_dev ||
      !c->seg_len_dev || !c->seg_off || !c->seg_cap || !c->seg_len)
    return CATEKV_ERR_INVALID_ARG;
  if (((uintptr_t)c->k_pool | (uintptr_t)c->v_pool | (uintptr_t)c->k_tail | (uintptr_t)c->v_tail) & 15) return CATEKV_ERR_INVALID_ARG;
  const int n = c->B * c->Hkv;
  for (int s = 0; s < n; ++s) {
    if (c->seg_off[s] < 0 || c->seg_off[s] % kQ8Block || c->seg_cap[s] < 0) return CATEKV_ERR_INVALID_ARG;
    // a segment's last block is written whole
    if ((int64_t)c->seg_off[s] + ((int64_t)c->seg_cap[s] + kQ8Block - 1) / kQ8Block * kQ8Block > c->total_rows) return CATEKV_ERR_INVALID_ARG;
  }
  return CATEKV_OK;
}

template <int kType>
__device__ __forceinline__ float q8_top() {
  return kType == CATEKV_Q8_E4M3 ? 448.f : 127.f;
}

// Four codes of a word as two f16 pairs (every code of either type is an f16 number).
template <int kType>
__device__ __forceinline__ void q8_to_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if (kType == CATEKV_Q8_E4M3) {
    asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.rn.f16x2.e4m3x2 %0, a;\n cvt.rn.f16x2.e4m3x2 %1, b;\n}\n"
        : "=r"(lo), "=r"(hi)
        : "r"(w));
  } else {
    // code + 128 as the low mantissa bits of 1024 (f16 spacing 1 there), then 1152 off: exact
    const uint32_t u = w ^ 0x80808080u;
    const __half2 off = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));
    uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
    __half2 x = __hsub2(*reinterpret_cast<__half2*>(&a), off), y = __hsub2(*reinterpret_cast<__half2*>(&b), off);
    lo = *reinterpret_cast<uint32_t*>(&x);
    hi = *reinterpret_cast<uint32_t*>(&y);
  }
}

}  // namespace catekv
