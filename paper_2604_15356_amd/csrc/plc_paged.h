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

// What calls that take rows are told of them (plc_rows), as kernels take it.
struct RowsView {
  uint16_t *k, *v;
  int64_t rows, sess_s, layer_s, head_s, row_s;
  int32_t layer, layers, packed, per_block;
};

inline bool rows_valid(const plc_pages *pages, const plc_rows *rows) {
  if (!rows || rows->layer < 0 || rows->layers < 1 || rows->layer > pages->L - rows->layers || rows->rows < 0 ||
      rows->rows > INT32_MAX || (rows->packed != 0 && rows->packed != 1))
    return false;
  for (int i = 0; i < 4; ++i)
    if ((i > 0 || !rows->packed) && (rows->stride[i] < 0 || rows->stride[i] % 8)) return false;
  return true;
}

inline RowsView rows_view(const plc_rows *rows, void *k, void *v, int32_t per_block) {
  RowsView r;
  r.k = static_cast<uint16_t *>(k), r.v = static_cast<uint16_t *>(v);
  r.rows = rows->rows;
  r.sess_s = rows->stride[0], r.layer_s = rows->stride[1], r.head_s = rows->stride[2], r.row_s = rows->stride[3];
  r.layer = rows->layer, r.layers = rows->layers, r.packed = rows->packed, r.per_block = per_block;
  return r;
}

// What positions have received (plc_weights), as kernels take it.
struct WeightsView {
  float *w;
  int64_t sess_s, layer_s, head_s, width;
};

// Whether runs of `extent` elements lie apart from each other, of which there are count[i] at a stride[i]: from the smallest stride
// to the largest each reaches past what the ones before it span.
template <int kDims>
inline bool lie_apart(const int64_t (&count)[kDims], const int64_t *stride, int64_t extent) {
  __int128 span = extent;
  bool done[kDims] = {};
  for (int step = 0; step < kDims; ++step) {
    int next = -1;
    for (int i = 0; i < kDims; ++i)
      if (!done[i] && (next < 0 || stride[i] < stride[next])) next = count[i] > 1 ? i : next;
    if (next < 0) return true;
    if (stride[next] < span) return false;
    span += (__int128)(count[next] - 1) * stride[next];
    done[next] = true;
  }
  return true;
}

// (Sessions, layers and heads each have weights of their own: workgroups rewrite them side by side.)
inline bool weights_valid(const plc_pages *p, const plc_weights *w) {
  if (!w || !aligned(w->w, 16) || w->width < 1 || w->width % 4) return false;
  for (int i = 0; i < 3; ++i)
    if (w->stride[i] % 4 || w->stride[i] < 0) return false;
  return lie_apart<3>({p->S, p->L, p->H}, w->stride, w->width);
}

inline WeightsView weights_view(const plc_weights *w) {
  return {w->w, w->stride[0], w->stride[1], w->stride[2], w->width};
}

// Whether the offsets of a call (in LDS) are what plc.h says, as one workgroup finds; the others rely on what they read alone.
template <int kThreads>
__device__ __forceinline__ void check_offsets(const PoolView &p, const RowsView &r, const int32_t *o, uint32_t *status) {
  bool bad = o[0] != 0 || (r.packed && o[p.S] > r.rows);
  for (int32_t s = threadIdx.x; s < p.S; s += kThreads) bad = bad || o[s + 1] < o[s];
  if (bad) raise(status, PLC_ERR_INVALID);
}

// Row x of a call: the session s it belongs to, its number i there, and where it lies in the buffer and in the pool, in elements
// from the first layer's and head's.  pool < 0: nowhere.
struct RowPlace {
  int64_t pool, buf, i;
  int32_t s;
};
template <bool kStore>
__device__ __forceinline__ RowPlace place_row(const PoolView &p, const RowsView &r, const int32_t *o, int64_t x, uint32_t *status) {
  RowPlace at = {-1, 0, 0, 0};
  bool here;
  if (r.packed) {
    int32_t lo = 0, hi = p.S - 1;  // the last session that begins at x or before
    while (lo < hi) {
      const int32_t mid = (lo + hi + 1) >> 1;
      if (o[mid] <= x) lo = mid;
      else hi = mid - 1;
    }
    at.s = lo;
    at.i = x - o[lo];
    here = x < r.rows && at.i >= 0 && x < o[lo + 1];
    at.buf = x * r.row_s;
  } else {
    at.s = (int32_t)min(x / r.rows, (int64_t)p.S);
    at.i = x - at.s * r.rows;
    here = at.s < p.S && at.i < (int64_t)o[min(at.s, p.S - 1) + 1] - o[min(at.s, p.S - 1)];
    at.buf = at.s * r.sess_s + at.i * r.row_s;
  }
  if (here) {
    const int64_t t = (int64_t)o[at.s + 1] - o[at.s], len = p.lens[at.s];
    const int64_t pos = len - t + at.i;
    if (t > len || len > ((int64_t)p.M << p.shift) || (!r.packed && t > r.rows)) {
      raise(status, PLC_ERR_INVALID);
    } else {
      const int32_t page = p.table[(int64_t)at.s * p.M + (pos >> p.shift)];
      if (p.page_ok(page) && (!kStore || p.refs[page] == 1)) at.pool = page * p.page_s + (pos & ((1 << p.shift) - 1)) * p.row_s;
      else raise(status, PLC_ERR_INVALID);
    }
  }
  return at;
}

__device__ __forceinline__ int32_t pages_of(int64_t rows, int shift) { return (int32_t)((rows + (1 << shift) - 1) >> shift); }

// A workgroup shortens a session, and gives back the pages behind its new length.
template <int kThreads>
__device__ __forceinline__ void trim_session(const PoolView &p, int32_t s, int64_t now, uint32_t *status) {
  const int64_t was = p.lens[s];
  if (was < 0 || was > ((int64_t)p.M << p.shift) || now < 0 || now > was) {
    if (threadIdx.x == 0) raise(status, PLC_ERR_INVALID);
    return;
  }
  for (int32_t j = pages_of(now, p.shift) + (int32_t)threadIdx.x; j < pages_of(was, p.shift); j += kThreads) {
    int32_t *const entry = &p.table[(int64_t)s * p.M + j];
    const int32_t page = *entry;
    *entry = -1;
    if (p.page_ok(page)) atomicSub(&p.refs[page], 1);
    else raise(status, PLC_ERR_INVALID);
  }
  __syncthreads();  // everybody has read the old length
  if (threadIdx.x == 0) p.lens[s] = (int32_t)now;
}

}  // namespace plc
