// Eviction from the paged cache: in every layer and head by itself the positions that have received most stay, and move
// together; see include/plc.h.
//
// Kernels one behind the other, because a session's table, length and counts may not change while others look at them:
//   select_kernel   a workgroup for each session, layer and head: whether the session can be shortened at all, which positions
//                   stay (a radix selection over the weights as ordered 32-bit keys, 11, 11 and 10 bits), their numbers in
//                   order, their weights moved together, and their rows;
//   move_kernel     the rows, where there are few heads;
//   shorten_kernel  lengths, pages.
// Rows move in place and in order: the row of number j comes from position kept[j] >= j, so that a workgroup that reads the rows
// of some numbers before it writes any of them needs to look at no other order: what later numbers read lies behind it.
//
// What bounds it: HBM for the rows, read once and written once (4 sessions of 2048 positions halved in 32 layers of 8 heads, 128
// components: 1.09 GB in 232 us, 4.7 TB/s; a copy of such a size 5.4), which wait while all workgroups choose (14 us of it); for few the steps of
// the choice, one behind the other (7 us for 512 positions, before their rows move).
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

constexpr int64_t kLittle = 4096;  // pieces of 16 bytes of a head's K
constexpr int kBins = 2048;
// A bin's place: the wavefront that adds them up, 32 in a row to a lane, so reads from all banks.
__device__ __forceinline__ uint32_t place_of(uint32_t bin) { return (bin & (kBins / 64 - 1)) * 64 + bin / (kBins / 64); }
constexpr int64_t kCached = (int64_t)96 << 20;  // bytes moved, in and out, beyond which rows go past the caches

// A lane takes 16 bytes of a row (in one column of K's rows, or V's), several rows at a time; all of the workgroup's loads of a round before
// its first store, and the next round's addresses while they are under way.  kStream: past the caches, in and out.
constexpr int kMoveBatch = 8;
template <int kThreads, bool kStream>
__device__ __forceinline__ void move_rows(const EvictArgs &a, int32_t s, int32_t lh, int32_t of_v, int32_t column, int32_t now) {
  const PoolView &p = a.p;
  const int32_t at_once = kThreads / a.pieces, row = (int32_t)threadIdx.x / a.pieces, c = column * a.pieces + (int32_t)threadIdx.x % a.pieces;
  const bool here = row < at_once && c < p.d8;
  uint16_t *const base = (of_v ? p.v : p.k) + (lh / p.H) * p.layer_s + (lh % p.H) * p.head_s + (int64_t)min(c, p.d8 - 1) * 8;
  const int32_t *const kept = a.kept + ((int64_t)s * p.L * p.H + lh) * a.W, *const table = p.table + (int64_t)s * p.M;
  const int32_t mask = (1 << p.shift) - 1, round = kMoveBatch * at_once, last = now - 1;
  int32_t from[kMoveBatch], next[kMoveBatch], from_page[kMoveBatch], to_page[kMoveBatch];
  const auto fetch = [&](int32_t j0) {  // (rows behind the end are read as the last one, and not written)
#pragma unroll
    for (int u = 0; u < kMoveBatch; ++u) next[u] = kept[min(j0 + u * at_once + row, last)];
  };
  const auto fetch_pages = [&](int32_t j0) {
#pragma unroll
    for (int u = 0; u < kMoveBatch; ++u) {
      from[u] = next[u];
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
    u32x4 v[kMoveBatch];
    uint16_t *to[kMoveBatch];
    bool moves[kMoveBatch];
    if (j0 + round < now) fetch(j0 + round);
#pragma unroll
    for (int u = 0; u < kMoveBatch; ++u) {
      const int32_t j = j0 + u * at_once + row;
      const auto *const at = reinterpret_cast<const u32x4 *>(base + from_page[u] * p.page_s + (from[u] & mask) * p.row_s);
      v[u] = kStream ? __builtin_nontemporal_load(at) : *at;
      to[u] = base + to_page[u] * p.page_s + (j & mask) * p.row_s;
      moves[u] = here && j < now && from[u] != j;
    }
    if (j0 + round < now) fetch_pages(j0 + round);
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kMoveBatch; ++u)
      if (moves[u]) {
        if (kStream) __builtin_nontemporal_store(v[u], reinterpret_cast<u32x4 *>(to[u]));
        else *reinterpret_cast<u32x4 *>(to[u]) = v[u];
      }
  }
}

// Runs of four positions that a thread holds, at a distance of the workgroup's: 16 positions for each thread are looked at without
// being read again.
constexpr int kRuns = 4;
template <int kThreads>
struct Held {
  static constexpr int32_t kRound = 4 * kThreads, kAll = kRuns * kRound;
  uint32_t key[kRuns][4];
  float w[kRuns][4];
  __device__ __forceinline__ void load(const float *weights, int32_t i0, int32_t n) {
#pragma unroll
    for (int c = 0; c < kRuns; ++c) {
      const int32_t i = i0 + c * kRound + 4 * (int32_t)threadIdx.x;
      float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (i < n) v = *reinterpret_cast<const float4 *>(weights + i);  // (a width's last run is whole: checked on the host)
      w[c][0] = v.x, w[c][1] = v.y, w[c][2] = v.z, w[c][3] = v.w;
    }
#pragma unroll
    for (int c = 0; c < kRuns; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) key[c][e] = key_of(w[c][e]);
  }
};

// kMove: what moves with the choice; 0: the rows stay for kernels of their own; 1, 2: here, 2 past the caches.
template <int kThreads, int kMove>
__global__ __launch_bounds__(kThreads) void select_kernel(EvictArgs a) {
  constexpr int kWaves = kThreads / 64;
  using Block = Held<kThreads>;
  __shared__ __attribute__((aligned(16))) uint32_t bins[2][kBins];
  __shared__ uint32_t meet[kRuns][kWaves];
  __shared__ uint32_t found[3];
  const PoolView &p = a.p;
  const int32_t s = (int32_t)blockIdx.y, lh = (int32_t)blockIdx.x, heads = p.L * p.H;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t len = p.lens[s], keep = a.keep[s], now = min(len, keep);
  bool ok = len >= 0 && len <= a.max_len && len <= ((int64_t)p.M << p.shift) && len <= a.w.width && keep >= 0 && now <= a.W &&
            (now == len || now >= (int64_t)a.first + a.last);
  float *const w = a.w.w + s * a.w.sess_s + (lh / p.H) * a.w.layer_s + (lh % p.H) * a.w.head_s;
  const bool shorter = ok && now < len;
  Block held;
  if (shorter) held.load(w, 0, (int32_t)len);
  for (int i = 4 * threadIdx.x; i < kBins; i += 4 * kThreads) *reinterpret_cast<uint4 *>(&bins[0][i]) = make_uint4(0u, 0u, 0u, 0u);
  if (shorter) {
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
  const int32_t n = (int32_t)len, lo = a.first, hi = n - a.last;  // positions lo .. hi-1 are chosen from
  uint32_t want = (uint32_t)now - (uint32_t)(a.first + a.last);   // of them stay (fewer than there are)
  const bool some = want > 0;                                     // else nobody but the first and the last

  // The key of the last one that stays, digit by digit: of the keys that begin as it does, `want` are still to be found.
  uint32_t prefix = 0;
#pragma unroll 1
  for (int digit = 0; digit < 3 && some; ++digit) {
    const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit == 2 ? 10 : 11;
    uint32_t *const count = bins[digit & 1];
    for (int32_t i0 = 0; i0 < hi; i0 += Block::kAll) {
      if (n > Block::kAll) held.load(w, i0, n);
#pragma unroll
      for (int c = 0; c < kRuns; ++c) {
        if (i0 + c * Block::kRound >= hi) break;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int32_t i = i0 + c * Block::kRound + 4 * (int32_t)threadIdx.x + e;
          const uint32_t key = held.key[c][e];
          if (i >= lo && i < hi && (digit == 0 || key >> (shift + bits) == prefix)) atomicAdd(&count[place_of(key >> shift & ((1u << bits) - 1))], 1u);
        }
      }
    }
    __syncthreads();
    if (wave == 0) {  // the digits from the largest down, 32 to a lane: the one behind which there are `want`
      uint32_t mine = 0;
#pragma unroll 8
      for (int e = 0; e < kBins / 64; ++e) mine += count[e * 64 + 63 - lane];
      uint32_t upto = wave_inclusive_scan(mine);
      const int owner = __builtin_ctzll(__ballot(upto >= want));  // (all of them are more)
      uint32_t before = owner > 0 ? (uint32_t)__builtin_amdgcn_readlane((int)upto, owner - 1) : 0u;
      const uint32_t one = lane < kBins / 64 ? count[(kBins / 64 - 1 - lane) * 64 + 63 - owner] : 0u;
      upto = before + wave_inclusive_scan(one);
      const int nth = __builtin_ctzll(__ballot(upto >= want));
      if (nth > 0) before = (uint32_t)__builtin_amdgcn_readlane((int)upto, nth - 1);
      const uint32_t with = (uint32_t)__builtin_amdgcn_readlane((int)upto, nth);
      if (lane == 0) found[0] = (uint32_t)(kBins - 1 - owner * (kBins / 64) - nth), found[1] = want - before, found[2] = with == want;
    } else if (digit < 2) {  // the next digit's
      for (int i = 4 * (threadIdx.x - 64); i < kBins; i += 4 * (kThreads - 64))
        *reinterpret_cast<uint4 *>(&bins[(digit & 1) ^ 1][i]) = make_uint4(0u, 0u, 0u, 0u);
    }
    __syncthreads();
    prefix = prefix << bits | found[0];
    want = found[1];
    if (found[2]) {  // all that begin so stay: what follows does not matter
      prefix = (prefix << shift) - 1;  // (not of zero: then all positions would stay)
      want = 0;
      break;
    }
  }
  // Keys above `prefix` stay, and of those equal to it the first `want`.
  uint32_t above = 0, equal = 0;  // so far
  for (int32_t i0 = 0; i0 < n; i0 += Block::kAll) {
    if (n > Block::kAll) held.load(w, i0, n);
    uint32_t up[kRuns], same[kRuns], counts[kRuns], upto[kRuns];
#pragma unroll
    for (int c = 0; c < kRuns; ++c) {
      if (i0 + c * Block::kRound >= n) break;
      up[c] = same[c] = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int32_t i = i0 + c * Block::kRound + 4 * (int32_t)threadIdx.x + e;
        const uint32_t key = held.key[c][e];
        const bool mid = i >= lo && i < hi;
        up[c] |= (uint32_t)(i < n && (!mid || (some && key > prefix))) << e;
        same[c] |= (uint32_t)(mid && some && key == prefix) << e;
      }
      counts[c] = (uint32_t)__builtin_popcount(up[c]) | (uint32_t)__builtin_popcount(same[c]) << 16;
      upto[c] = wave_inclusive_scan(counts[c]);
      if (lane == 63) meet[c][wave] = upto[c];
    }
    __syncthreads();
    // (everybody has read the weights of these runs: what is written lies at or before them)
#pragma unroll
    for (int c = 0; c < kRuns; ++c) {
      if (i0 + c * Block::kRound >= n) break;
      uint32_t before = 0, total = 0;
#pragma unroll
      for (int v = 0; v < kWaves; ++v) {
        const uint32_t x = meet[c][v];
        before += v < wave ? x : 0;
        total += x;
      }
      before += upto[c] - counts[c];
      uint32_t g = above + (before & 0xffffu), q = equal + (before >> 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int32_t i = i0 + c * Block::kRound + 4 * (int32_t)threadIdx.x + e;
        const bool is_same = same[c] >> e & 1u;
        if ((up[c] >> e & 1u) || (is_same && q < want)) {
          const uint32_t j = g + min(q, want);
          kept[j] = i;
          if ((int32_t)j != i) w[j] = held.w[c][e];
        }
        g += up[c] >> e & 1u;
        q += is_same;
      }
      above += total & 0xffffu, equal += total >> 16;
    }
    __syncthreads();  // `meet` is written again; and all of `kept` is there
  }
  if constexpr (kMove != 0)
    for (int32_t i = 0; i < 2 * a.columns; ++i) move_rows<kThreads, kMove == 2>(a, s, lh, i / a.columns, i % a.columns, (int32_t)now);
}

// The rows of a session, layer and head where they are moved by workgroups of their own: K and V, and 128-byte columns of them.
template <bool kStream>
__global__ __launch_bounds__(kBlock) void move_kernel(EvictArgs a) {
  const int32_t s = (int32_t)blockIdx.y, now = a.now[s], unit = (int32_t)blockIdx.x;
  if (now >= 0) move_rows<kBlock, kStream>(a, s, unit / (2 * a.columns), unit / a.columns & 1, unit % a.columns, now);
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
  a.status = status;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const int64_t heads = (int64_t)a.p.L * a.p.H;
  if (heads >= 1 << 22 || heads * pages->d >= 1 << 29) return PLC_ERR_INVALID;  // (lanes of a launch < 2^32)
  const dim3 grid((unsigned)heads, (unsigned)a.p.S);
  // Where there are sessions and heads enough for all compute units, or little that may have to be moved (W rows: the host knows no more), a workgroup
  // moves what it has chosen, whole rows at a time; else K and V and their lines of 128 bytes have workgroups of their own.  (32 layers and 8 heads, 128 components, halved: 64 sessions of 200
  // positions 337 against 389 us, a session of 8000 228 against 235; of 8 layers, 4 sessions of 2000 65 against 70; of 4, 53 against 42.  Little:
  // in a graph, 8 heads of 64 components, 64 rows that stay 14.3 against 14.8 us, 512 18.5 against 17.7, 768 22.4 against 20.1; the launch that is saved
  // takes 3.3 of the host's.)
  const int64_t rows = heads * a.p.S;
  const bool together = rows >= kComputeUnits || (int64_t)W * a.p.d8 <= kLittle;
  const bool past = (double)rows * W * a.p.d8 * 64 > (double)kCached;  // of both halves, in and out
  a.pieces = a.p.d8 > kBlock ? kBlock : !together && a.p.d8 % 8 == 0 ? 8 : a.p.d8;
  a.columns = (a.p.d8 + a.pieces - 1) / a.pieces;
  // Four wavefronts up to the 4096 positions that they hold in registers, 16 beyond (a pass with a head's rows, us, of 256 and of 1024 threads: one head,
  // 1000 positions 17.0 and 18.0, 4096 28.8 and 27.5, 6000 40.5 and 35.5, 32,000 151 and 129; 1024 heads of 64 components, 500 positions 44 and 73,
  // 1000 71 and 88, 4000 245 and 244, 8000 483 and 464).
  const auto chosen = max_len <= 4096 ? (!together ? &select_kernel<256, 0> : past ? &select_kernel<256, 2> : &select_kernel<256, 1>)
                                      : (!together ? &select_kernel<1024, 0> : past ? &select_kernel<1024, 2> : &select_kernel<1024, 1>);
  hipLaunchKernelGGL(chosen, grid, dim3(max_len <= 4096 ? 256 : 1024), 0, st, a);
  if (!together)
    hipLaunchKernelGGL(past ? &move_kernel<true> : &move_kernel<false>, dim3((unsigned)(heads * 2 * a.columns), (unsigned)a.p.S),
                       dim3(kBlock), 0, st, a);
  hipLaunchKernelGGL(shorten_kernel, dim3((unsigned)a.p.S), dim3(kBlock), 0, st, a);
  return launch_status();
}
