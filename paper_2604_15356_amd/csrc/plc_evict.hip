// Eviction from the paged cache: in every layer and head by itself the positions that have received most stay, and move
// together; see include/plc.h.
//
// Three kernels, one behind the other, because a session's table, length and counts may not change while others look at them:
//   select_kernel   a workgroup for each session, layer and head: whether the session can be shortened at all, which positions
//                   stay (a radix selection over the weights as ordered 32-bit keys, 11, 11 and 10 bits), their numbers in
//                   order, their weights moved together;
//   move_kernel     their rows moved together, K and V and 128-byte columns of them by workgroups of their own;
//   shorten_kernel  lengths, pages.
// Rows move in place and in order: the row of number j comes from position kept[j] >= j, so that a workgroup that reads the rows
// of some numbers before it writes any of them needs to look at no other order: what later numbers read lies behind it.
//
// What bounds it: HBM for the rows, read once and written once.
#include "plc_device.h"
#include "plc_paged.h"

namespace plc {
namespace {

struct EvictArgs {
  PoolView p;
  WeightsView w;
  const int32_t *keep;
  int32_t *kept, *now;  // now[S]: positions that a session is shortened to; kUnchanged; kRefused
  int32_t first, last, W, max_len;
  int32_t pieces, columns;  // 16-byte pieces of a column of rows, columns of a row
  uint32_t *status;
};
constexpr int32_t kUnchanged = -1, kRefused = -2;

// Weights in the order of whole numbers; a NaN above all.
__device__ __forceinline__ uint32_t key_of(float w) {
  const uint32_t u = __builtin_bit_cast(uint32_t, w + 0.0f);  // (-0 is 0)
  return w != w ? 0xffffffffu : u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}

constexpr int kBins = 2048;

// Exclusive prefix sum over a workgroup.  `smem`: a word for each wavefront and one more.
template <int kThreads>
__device__ __forceinline__ uint32_t scan(uint32_t v, uint32_t *smem, uint32_t *total) {
  constexpr int kWaves = kThreads / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t inc = wave_inclusive_scan(v);
  __syncthreads();
  if (lane == 63) smem[wave] = inc;
  __syncthreads();
  uint32_t base = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const uint32_t s = smem[w];
    base += w < wave ? s : 0;
    all += s;
  }
  *total = all;
  return base + inc - v;
}

template <int kThreads>
__global__ __launch_bounds__(kThreads) void select_kernel(EvictArgs a) {
  __shared__ uint32_t bins[kBins];
  __shared__ uint32_t smem[kThreads / 64 + 1];
  __shared__ uint32_t found[2];
  const PoolView &p = a.p;
  const int32_t s = (int32_t)blockIdx.y, lh = (int32_t)blockIdx.x, heads = p.L * p.H;
  const int64_t len = p.lens[s], keep = a.keep[s], now = min(len, keep);
  bool ok = len >= 0 && len <= a.max_len && len <= ((int64_t)p.M << p.shift) && len <= a.w.width && keep >= 0 && now <= a.W &&
            (now == len || now >= (int64_t)a.first + a.last);
  if (ok && now < len) {
    // the pages in use, and those that are written among them
    for (int32_t j = threadIdx.x; j < pages_of(len, p.shift); j += kThreads) {
      const int32_t page = p.table[(int64_t)s * p.M + j];
      const bool written = j >= a.first >> p.shift && j < pages_of(now, p.shift);
      ok = ok && p.page_ok(page) && (!written || p.refs[page] == 1);
    }
  }
  ok = __syncthreads_and(ok);
  if (lh == 0 && threadIdx.x == 0) {
    a.now[s] = !ok ? kRefused : now == len ? kUnchanged : (int32_t)now;
    if (!ok) raise(a.status, PLC_ERR_INVALID);
  }
  if (!ok) return;
  int32_t *const kept = a.kept + ((int64_t)s * heads + lh) * a.W;
  if (now == len) {
    for (int32_t j = threadIdx.x; j < now; j += kThreads) kept[j] = j;
    return;
  }
  float *const w = a.w.w + s * a.w.sess_s + (lh / p.H) * a.w.layer_s + (lh % p.H) * a.w.head_s;
  const int32_t n = (int32_t)len, lo = a.first, hi = n - a.last;  // positions lo .. hi-1 are chosen from
  uint32_t want = (uint32_t)now - (uint32_t)(a.first + a.last);   // of them stay (fewer than there are)

  // The key of the last one that stays, digit by digit: of the keys that begin as it does, `want` are still to be found.
  uint32_t prefix = 0;
#pragma unroll 1
  for (int digit = 0; digit < 3 && want > 0; ++digit) {
    const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit == 2 ? 10 : 11;
    for (int i = threadIdx.x; i < kBins; i += kThreads) bins[i] = 0;
    __syncthreads();
    for (int32_t i = (lo & ~3) + 4 * (int32_t)threadIdx.x; i < hi; i += 4 * kThreads) {
      const float4 v = *reinterpret_cast<const float4 *>(w + i);  // (a width's last piece is whole: checked on the host)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t key = key_of(e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w);
        if (i + e >= lo && i + e < hi && (digit == 0 || key >> (shift + bits) == prefix))
          atomicAdd(&bins[key >> shift & ((1u << bits) - 1)], 1u);
      }
    }
    __syncthreads();
    // the digits from the largest down: the first behind which there are `want`
    constexpr int kEach = kBins / kThreads;
    uint32_t mine = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) mine += bins[kBins - 1 - (kEach * (int)threadIdx.x + e)];
    uint32_t total, before = scan<kThreads>(mine, smem, &total);
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int bin = kBins - 1 - (kEach * (int)threadIdx.x + e);
      if (before < want && before + bins[bin] >= want) found[0] = (uint32_t)bin, found[1] = want - before;
      before += bins[bin];
    }
    __syncthreads();
    prefix = prefix << bits | found[0];
    want = found[1];
    __syncthreads();
  }
  const bool some = now > (int64_t)a.first + a.last;  // else nobody but the first and the last
  // Keys above `prefix` stay, and of those equal to it the first `want`.
  uint32_t above = 0, equal = 0;  // so far
  for (int32_t i0 = 0; i0 < n; i0 += 4 * kThreads) {
    const int32_t i = i0 + 4 * (int32_t)threadIdx.x;
    float v[4] = {};
    uint32_t up = 0, same = 0;
    if (i < n) {
      const float4 x = *reinterpret_cast<const float4 *>(w + i);
      v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t key = key_of(v[e]);
        const bool mid = i + e >= lo && i + e < hi, in = i + e < n;
        up |= (uint32_t)(in && (!mid || (some && key > prefix))) << e;
        same |= (uint32_t)(in && mid && some && key == prefix) << e;
      }
    }
    uint32_t total;
    const uint32_t before = scan<kThreads>((uint32_t)__builtin_popcount(up) | (uint32_t)__builtin_popcount(same) << 16, smem, &total);
    uint32_t g = above + (before & 0xffffu), q = equal + (before >> 16);
    // (everybody has read the weights of this round: what is written lies at or before them)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool is_same = same >> e & 1u, stays = (up >> e & 1u) || (is_same && q < want);
      if (stays) {
        const uint32_t j = g + min(q, want);
        kept[j] = i + e;
        if ((int32_t)j != i + e) w[j] = v[e];
      }
      g += up >> e & 1u;
      q += is_same;
    }
    above += total & 0xffffu, equal += total >> 16;
  }
}

// A lane takes 16 bytes of a row, several rows at a time; all of the workgroup's loads of a round before its first store.
constexpr int kMoveBatch = 8;
__global__ __launch_bounds__(kBlock) void move_kernel(EvictArgs a) {
  const PoolView &p = a.p;
  const int32_t s = (int32_t)blockIdx.y, now = a.now[s];
  if (now < 0) return;
  const int32_t heads = p.L * p.H, unit = (int32_t)blockIdx.x;
  const int32_t column = unit % a.columns, of_v = unit / a.columns & 1, lh = unit / (2 * a.columns);
  const int32_t at_once = kBlock / a.pieces, row = (int32_t)threadIdx.x / a.pieces, c = column * a.pieces + (int32_t)threadIdx.x % a.pieces;
  const bool here = row < at_once && c < p.d8;
  uint16_t *const base = (of_v ? p.v : p.k) + (lh / p.H) * p.layer_s + (lh % p.H) * p.head_s + (int64_t)min(c, p.d8 - 1) * 8;
  const int32_t *const kept = a.kept + ((int64_t)s * heads + lh) * a.W, *const table = p.table + (int64_t)s * p.M;
  const int32_t mask = (1 << p.shift) - 1;
  const int32_t round = kMoveBatch * at_once, last = now - 1;
  int32_t from[kMoveBatch], from_page[kMoveBatch], to_page[kMoveBatch];
  const auto fetch = [&](int32_t j0) {  // (rows behind the end are read as the last one, and not written)
#pragma unroll
    for (int u = 0; u < kMoveBatch; ++u) from[u] = kept[min(j0 + u * at_once + row, last)];
  };
  const auto fetch_pages = [&](int32_t j0) {
#pragma unroll
    for (int u = 0; u < kMoveBatch; ++u) {
      from_page[u] = table[from[u] >> p.shift];
      to_page[u] = table[min(j0 + u * at_once + row, last) >> p.shift];
    }
  };
  int32_t j0 = a.first;
  while (j0 + round <= now && kept[j0 + round - 1] == j0 + round - 1) j0 += round;  // nothing has gone before these
  if (j0 >= now) return;
  fetch(j0);
  fetch_pages(j0);
  for (; j0 < now; j0 += round) {
    uint4 v[kMoveBatch];
    uint16_t *to[kMoveBatch];
    bool moves[kMoveBatch];
#pragma unroll
    for (int u = 0; u < kMoveBatch; ++u) {
      const int32_t j = j0 + u * at_once + row;
      v[u] = *reinterpret_cast<const uint4 *>(base + from_page[u] * p.page_s + (from[u] & mask) * p.row_s);
      to[u] = base + to_page[u] * p.page_s + (j & mask) * p.row_s;
      moves[u] = here && j < now && from[u] != j;
    }
    if (j0 + round < now) {
      fetch(j0 + round);
      fetch_pages(j0 + round);
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kMoveBatch; ++u)
      if (moves[u]) *reinterpret_cast<uint4 *>(to[u]) = v[u];
  }
}

__global__ __launch_bounds__(kBlock) void shorten_kernel(EvictArgs a) {
  const int32_t s = (int32_t)blockIdx.x, now = a.now[s];
  if (now >= 0) trim_session<kBlock>(a.p, s, now, a.status);
}

}  // namespace
}  // namespace plc

using namespace plc;

extern "C" int plc_pages_evict(const plc_pages *pages, const int32_t *keep, int32_t first, int32_t last,
                               const plc_weights *weights, int32_t *kept, int32_t W, int32_t max_len, void *ws, size_t ws_bytes,
                               uint32_t *status, void *stream) {
  if (!pages_valid(pages) || !weights_valid(pages, weights) || !aligned(keep, 4) || first < 0 || last < 0 || W < 0 ||
      (W > 0 && !aligned(kept, 4)) || max_len < 0 || max_len > 1 << 30 || !aligned(ws, 256) ||
      ws_bytes < plc_pages_workspace_bytes(pages) || !status)
    return PLC_ERR_INVALID;
  EvictArgs a = {};
  a.p = pool_view(pages);
  a.w = weights_view(weights);
  a.keep = keep, a.kept = kept, a.now = static_cast<int32_t *>(ws);
  a.first = first, a.last = last, a.W = W, a.max_len = max_len;
  a.pieces = a.p.d8 % 8 == 0 ? 8 : a.p.d8 < kBlock ? a.p.d8 : kBlock;
  a.columns = (a.p.d8 + a.pieces - 1) / a.pieces;
  a.status = status;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const int64_t heads = (int64_t)a.p.L * a.p.H;
  if (heads >= 1 << 22 || heads * pages->d >= 1 << 29) return PLC_ERR_INVALID;  // (lanes of a launch < 2^32)
  const dim3 grid((unsigned)heads, (unsigned)a.p.S);
  if (max_len <= 4096) hipLaunchKernelGGL(select_kernel<256>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(select_kernel<1024>, grid, dim3(1024), 0, st, a);
  hipLaunchKernelGGL(move_kernel, dim3((unsigned)(heads * 2 * a.columns), (unsigned)a.p.S), dim3(kBlock), 0, st, a);
  hipLaunchKernelGGL(shorten_kernel, dim3((unsigned)a.p.S), dim3(kBlock), 0, st, a);
  return launch_status();
}
