// What the kernels on the paged K/V cache share: which page holds a row, and
// the 8-bit codes of a page.
#pragma once
#include <type_traits>

#include "device_common.h"
#include "vla.h"

constexpr int type_bytes(int type) { return type == VLA_KV_F32 ? 4 : type == VLA_KV_BF16 ? 2 : 1; }

// Page of row j of request b, or -1: outside the page table, or not in the pool.
VLA_DEV int page_of(const PageArgs& p, int b, long long j) {
  if (j < 0) return -1;
  const long long i = j >> p.lg;
  if (i >= p.max_pages) return -1;
  const int pid = p.table[(size_t)b * p.max_pages + i];
  return pid >= 0 && pid < p.n_pages ? pid : -1;
}

// Four codes of a dword: value of code e, and the codes of four values.
template <int TYPE>
VLA_DEV float code_f(uint32_t w, int e) {
  if constexpr (TYPE == VLA_KV_I8) {
    return (float)(int)(int8_t)(w >> (8 * e));
  } else {
    switch (e) {
      case 0: return __builtin_amdgcn_cvt_f32_fp8((int)w, 0);
      case 1: return __builtin_amdgcn_cvt_f32_fp8((int)w, 1);
      case 2: return __builtin_amdgcn_cvt_f32_fp8((int)w, 2);
      default: return __builtin_amdgcn_cvt_f32_fp8((int)w, 3);
    }
  }
}
template <int TYPE>
VLA_DEV uint32_t pack_codes(const float* y) {
  if constexpr (TYPE == VLA_KV_I8) {
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) w |= ((uint32_t)(int)rintf(y[e]) & 0xFFu) << (8 * e);
    return w;
  } else {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
    return (uint32_t)w;
  }
}
