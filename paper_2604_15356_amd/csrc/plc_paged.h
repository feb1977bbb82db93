// What the paged cache's kernels share: the checked description of a pool, as kernels take it.
#pragma once

#include "plc_device.h"

namespace plc {

struct PoolView {
  uint16_t *k, *v;
  int64_t page_s, layer_s, head_s, row_s;
  int32_t P, L, H, d8, shift;  // a page has 1 << shift rows of d8 pieces of 16 bytes
  int32_t S, M;
  int32_t *table, *lens, *refs;
  __device__ __forceinline__ bool page_ok(int32_t page) const { return (uint32_t)page < (uint32_t)P; }
};

inline bool aligned(const void *ptr, uintptr_t a) { return ptr && reinterpret_cast<uintptr_t>(ptr) % a == 0; }

// (Within a page rows are addressed with 32 bits; everything beyond it with 64.)
inline bool pages_valid(const plc_pages *p) {
  if (!p || !aligned(p->k, 16) || !aligned(p->v, 16) || !aligned(p->table, 4) || !aligned(p->lens, 4) || !aligned(p->refs, 4))
    return false;
  if (p->P < 1 || p->L < 1 || p->H < 1 || p->S < 1 || p->S > 1024 || p->M < 1 || p->d < 8 || p->d % 8) return false;
  if (p->B < 16 || p->B > 1024 || (p->B & (p->B - 1)) || (int64_t)p->M * p->B > (int64_t)1 << 30) return false;
  if ((int64_t)p->L * p->H > INT32_MAX / (2 * (int64_t)p->d)) return false;
  for (int i = 0; i < 4; ++i)
    if (p->stride[i] < 0 || p->stride[i] % 8) return false;
  return p->stride[3] >= p->d && p->stride[3] * p->B < (int64_t)1 << 30;
}

inline PoolView pool_view(const plc_pages *p) {
  PoolView v;
  v.k = static_cast<uint16_t *>(p->k), v.v = static_cast<uint16_t *>(p->v);
  v.page_s = p->stride[0], v.layer_s = p->stride[1], v.head_s = p->stride[2], v.row_s = p->stride[3];
  v.P = p->P, v.L = p->L, v.H = p->H, v.d8 = p->d / 8, v.shift = __builtin_ctz((unsigned)p->B);
  v.S = p->S, v.M = p->M;
  v.table = p->table, v.lens = p->lens, v.refs = p->refs;
  return v;
}

}  // namespace plc
