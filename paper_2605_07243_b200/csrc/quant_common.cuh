// Shared pieces of the calls over an 8-bit KV cache: addressing, e4m3 conversions, checks.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"

namespace sb {

// Row of the flat [rows][n_kv_heads][head_dim] code array that holds position j of sequence b.  A page id outside the
// pool is read as page 0, so that no access leaves the pool.
__device__ inline long long quant_row(const sb_quant_cache& kv, int b, int j) {
  if (kv.page_size == 0) return (long long)b * kv.kv_capacity + j;
  const int shift = 31 - __clz(kv.page_size);  // a power of two
  const int lp = j >> shift;
  int page = kv.page_table[(long long)b * kv.max_pages + lp];
  if (page < 0 || page >= kv.num_pages) page = 0;
  return ((long long)page << shift) + (j & (kv.page_size - 1));
}
__host__ __device__ inline long long quant_rows_total(const sb_quant_cache& kv) {
  return kv.page_size == 0 ? (long long)kv.batch * kv.kv_capacity : (long long)kv.num_pages * kv.page_size;
}

// Two floats -> two e4m3 codes (nearest, ties to even), the first in the low byte.
__device__ inline uint16_t e4m3x2_of(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// Two e4m3 codes -> two fp16 values (exact: every e4m3 value is an fp16 value).
__device__ inline uint32_t half2_of_e4m3x2(uint16_t c) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(c));
  return r;
}
__device__ inline float2 float2_of_e4m3x2(uint16_t c) {
  const uint32_t h = half2_of_e4m3x2(c);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// Two fp16 values -> e4m3 codes of the nearest values and of what is left (the difference is exact in fp16 for inputs of 8 significant bits).
__device__ inline void split_e4m3(uint32_t h, uint16_t& hi, uint16_t& lo) {
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(hi) : "r"(h));
  const uint32_t near = half2_of_e4m3x2(hi);
  const __half2 rest = __hsub2(*reinterpret_cast<const __half2*>(&h), *reinterpret_cast<const __half2*>(&near));
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(lo) : "r"(*reinterpret_cast<const uint32_t*>(&rest)));
}

inline sb_status check_quant_cache(const sb_quant_cache* kv) {
  if (!kv || kv->batch < 1 || kv->n_kv_heads < 1 || !kv->k_codes || !kv->v_codes || !kv->k_scale || !kv->v_scale ||
      kv->n_layers < 1 || kv->codes_layer_stride < 0 || kv->codes_layer_stride % 16 != 0 || kv->scale_layer_stride < 0)
    return SB_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(kv->k_codes) & 15) || (reinterpret_cast<uintptr_t>(kv->v_codes) & 15) ||
      (reinterpret_cast<uintptr_t>(kv->k_scale) & 3) || (reinterpret_cast<uintptr_t>(kv->v_scale) & 3))
    return SB_ERR_INVALID_ARG;
  if (kv->head_dim != 64 && kv->head_dim != 128) return SB_ERR_UNSUPPORTED;
  const int sb = kv->scale_block;
  if (sb != 16 && sb != 32 && sb != 64 && sb != 128) return SB_ERR_UNSUPPORTED;
  if (kv->page_size < 0) return SB_ERR_INVALID_ARG;
  if (kv->page_size > 0) {
    if (kv->page_size < 16 || (kv->page_size & (kv->page_size - 1)) || kv->page_size % sb != 0) return SB_ERR_UNSUPPORTED;
    if (!kv->page_table || kv->max_pages < 1 || kv->num_pages < 1) return SB_ERR_INVALID_ARG;
    if ((long long)kv->max_pages * kv->page_size > 0x7fffffffLL - 256) return SB_ERR_UNSUPPORTED;  // positions are int32
  } else {
    if (kv->kv_capacity < 1) return SB_ERR_INVALID_ARG;
    if (kv->kv_capacity % sb != 0 || kv->kv_capacity > 0x7fffffffLL - 256) return SB_ERR_UNSUPPORTED;
  }
  return SB_OK;
}

}  // namespace sb
