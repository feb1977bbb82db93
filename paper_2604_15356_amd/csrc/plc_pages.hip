// The paged cache's own calls: sharing, growing, shortening and moving pages, rows in and out.  See include/plc.h for
// what each does.
//
// The bookkeeping (table, lengths, reference counts) is small, a few hundred KB at most, and is done by one workgroup or by
// one per session; what moves rows is spread over the chip, 16 bytes per lane, with the addresses of a block's rows
// worked out once.  Nothing here computes on the elements: the bound is HBM for the large moves, and for the small ones the
// number of launches and the two or three dependent loads (offsets, table, data) of each.  Measured: 1.07 GB of rows into
// pages (4096 positions of 32 layers, 8 heads, in and out) 191 us, 5.6 TB/s; 302 MB of pages compacted 54 us, 5.6 TB/s; 35 MB of
// rows of odd lengths out of pages 7.2 us; forking 64 sessions 3.6 us, room for their next tokens 6.6 us and the copies of their
// shared tails 3.8 us; a kernel that finds nothing to do 1.3 us.  A launch costs the host 3.3 us, so that small steps wait for it.
#include "plc_device.h"
#include "plc_paged.h"

namespace plc {
namespace {

constexpr int kManager = 1024;  // threads of the one workgroup that hands out pages; as many sessions at most

// ---- 16 bytes at a time ------------------------------------------------------------------------------------------------

// 16 bytes of a row.  Past the caches (kStream) where more is stored than they hold: 1.07 GB in and out 195 us, through them
// 208 us, 134 MB 24.9 against 28.8 us; but 67 MB, there from the call before, 14.2 against 12.3 us.  Rows that are loaded gain
// nothing by it (537 MB 114 against 110 us), and the encoder reads them next.
template <bool kStream>
__device__ __forceinline__ uint4 get16(const uint16_t *p) {
  return kStream ? load16_stream(p) : *reinterpret_cast<const uint4 *>(p);
}
template <bool kStream>
__device__ __forceinline__ void put16(uint16_t *p, uint4 v) {
  if (kStream) store16_stream(p, v);
  else *reinterpret_cast<uint4 *>(p) = v;
}

// The first `rows` rows of a page's heads slab, slab + step, ... (of both halves) from one page to another.
template <bool kStream, int kThreads>
__device__ __forceinline__ void copy_slabs(const PoolView &p, int64_t from, int64_t to, int32_t rows, int32_t slab0,
                                           int32_t slab1) {
  const int32_t items = rows * p.d8;
  const bool dense = p.row_s == (int64_t)p.d8 * 8;
  for (int32_t i = threadIdx.x; i < items; i += kThreads) {
    const int64_t in_slab = dense ? (int64_t)i * 8 : (i / p.d8) * p.row_s + (int64_t)(i % p.d8) * 8;
    for (int32_t slab = slab0; slab < slab1; slab += 4) {
      uint4 k[4], v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int32_t lh = min(slab + u, slab1 - 1);
        const int64_t at = from * p.page_s + (lh / p.H) * p.layer_s + (lh % p.H) * p.head_s + in_slab;
        k[u] = get16<kStream>(p.k + at);
        v[u] = get16<kStream>(p.v + at);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int32_t lh = slab + u;
        if (lh < slab1) {
          const int64_t at = to * p.page_s + (lh / p.H) * p.layer_s + (lh % p.H) * p.head_s + in_slab;
          put16<kStream>(p.k + at, k[u]);
          put16<kStream>(p.v + at, v[u]);
        }
      }
    }
  }
}

// ---- bookkeeping ------------------------------------------------------------------------------------------------------

// Exclusive prefix sum over the 1024 threads of a workgroup.  `smem`: 17 words.
__device__ __forceinline__ uint32_t manager_scan(uint32_t v, uint32_t *smem, uint32_t *total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t inc = wave_inclusive_scan(v);
  __syncthreads();
  if (lane == 63) smem[wave] = inc;
  __syncthreads();
  if (wave == 0) {
    const uint32_t w = lane < kManager / 64 ? smem[lane] : 0;
    const uint32_t s = wave_inclusive_scan(w);
    if (lane < kManager / 64) smem[lane] = s - w;
    if (lane == kManager / 64 - 1) smem[kManager / 64] = s;
  }
  __syncthreads();
  *total = smem[kManager / 64];
  return smem[wave] + inc - v;
}

// Which of the eight pages from p0 on are in use.
constexpr int kScanWords = 8, kScanRound = kManager * kScanWords;
__device__ __forceinline__ uint32_t used_bits(const PoolView &p, int64_t p0) {
  uint32_t bits = 0;
#pragma unroll
  for (int j = 0; j < kScanWords; ++j)
    if (p0 + j < p.P && p.refs[p0 + j] != 0) bits |= 1u << j;
  return bits;
}

// Walks the pages [first, last) in order, eight to a thread and round (one load each, so that a round of 8192 pages is one trip
// to memory, and `ready`, the first round's, can be asked for long before): visit(page, rank) for every page that is in use
// (or is not), `rank` counting them from 0.  Stops once `enough` are found.  Returns how many there were up to there.
template <class Visit>
__device__ __forceinline__ uint32_t scan_pages(const PoolView &p, int32_t first, int32_t last, bool in_use, uint32_t ready,
                                               uint32_t enough, uint32_t *smem, const Visit &visit) {
  uint32_t found = 0;
  for (int64_t base = first / kScanRound * kScanRound; base < last && found < enough; base += kScanRound) {
    const int64_t p0 = base + (int64_t)threadIdx.x * kScanWords;
    const uint32_t used = base == 0 ? ready : used_bits(p, p0);
    const int lo = (int)max((int64_t)0, min((int64_t)kScanWords, first - p0)), hi = (int)max((int64_t)0, min((int64_t)kScanWords, last - p0));
    uint32_t mine = (in_use ? used : ~used) & ((1u << hi) - 1) & ~((1u << lo) - 1), total;
    uint32_t rank = found + manager_scan((uint32_t)__builtin_popcount(mine), smem, &total);
    for (; mine; mine &= mine - 1) visit((int32_t)(p0 + __builtin_ctz(mine)), rank++);
    found += total;
  }
  return found;
}

__device__ __forceinline__ int32_t pages_of(int64_t rows, int shift) { return (int32_t)((rows + (1 << shift) - 1) >> shift); }

// One workgroup takes a strip of 16 entries of all sessions: it reads them all before it writes any, so the table is
// permuted in place.  An entry tells by itself whether there is a page behind it, so that no workgroup needs the lengths
// that another is rewriting.  Counts change by atomics on integers, in any order.
constexpr int kStrip = 16;
__global__ __launch_bounds__(kBlock) void fork_kernel(PoolView p, const int32_t *__restrict__ src, uint32_t *status) {
  extern __shared__ int32_t fork_lds[];  // [S, kStrip], [S]
  int32_t *const from = fork_lds + p.S * kStrip;
  const int32_t j0 = (int32_t)blockIdx.x * kStrip, width = min(kStrip, p.M - j0);
  for (int32_t s = threadIdx.x; s < p.S; s += kBlock) {
    int32_t f = src[s];
    if (f < -1 || f >= p.S) {
      raise(status, PLC_ERR_INVALID);
      f = s;
    }
    from[s] = f;
  }
  for (int32_t i = threadIdx.x; i < p.S * kStrip; i += kBlock) {
    const int32_t s = i / kStrip, j = i % kStrip;
    fork_lds[i] = j < width ? p.table[(int64_t)s * p.M + j0 + j] : -1;
  }
  __syncthreads();
  for (int32_t i = threadIdx.x; i < p.S * kStrip; i += kBlock) {
    const int32_t s = i / kStrip, j = i % kStrip, f = from[s];
    if (j >= width || f == s) continue;
    const int32_t was = fork_lds[i], now = f < 0 ? -1 : fork_lds[f * kStrip + j];
    if (was == now) continue;
    p.table[(int64_t)s * p.M + j0 + j] = now;
    if (p.page_ok(now)) atomicAdd(&p.refs[now], 1);
    if (p.page_ok(was)) atomicSub(&p.refs[was], 1);
    if ((now != -1 && !p.page_ok(now)) || (was != -1 && !p.page_ok(was))) raise(status, PLC_ERR_INVALID);
  }
  if (blockIdx.x == 0) {
    __syncthreads();
    for (int32_t s = threadIdx.x; s < p.S; s += kBlock) fork_lds[s] = p.lens[s];
    __syncthreads();
    for (int32_t s = threadIdx.x; s < p.S; s += kBlock)
      if (from[s] != s) p.lens[s] = from[s] < 0 ? 0 : fork_lds[from[s]];
  }
}

// Pages for the sessions' new positions, a thread per session: the list of tail pages to copy, and the pages taken, in order.
// kCopies: the tails are so small that this workgroup copies them too, a launch less (the step of 4 beams with pages of 32 KB
// that calls it: 19.4 against 22.2 us).
struct CopyList {
  uint32_t count, pad[3];
  int32_t from[kManager], to[kManager], rows[kManager];
};
template <bool kCopies>
__global__ __launch_bounds__(kManager) void extend_kernel(PoolView p, const int32_t *__restrict__ grow,
                                                          CopyList *__restrict__ copies, int32_t *__restrict__ taken,
                                                          uint32_t *status) {
  __shared__ uint32_t smem[kManager / 64 + 1];
  __shared__ __attribute__((aligned(16))) int32_t tails[kManager];
  __shared__ int32_t first_of[kManager];
  __shared__ uint32_t start_of[kManager];
  __shared__ uint32_t refused;
  const int32_t s = threadIdx.x;
  const uint32_t ready = used_bits(p, (int64_t)s * kScanWords);
  if (s == 0) refused = 0;
  __syncthreads();
  int64_t len = 0, g = 0;
  if (s < p.S) {
    len = p.lens[s];
    g = grow[s];
    if (len < 0 || len > ((int64_t)p.M << p.shift) || g < 0) {
      atomicMax(&refused, PLC_ERR_INVALID);
      len = g = 0;
    } else if (len + g > ((int64_t)p.M << p.shift)) {
      atomicMax(&refused, PLC_ERR_CAPACITY);
      g = 0;
    }
  }
  const int32_t slot = (int32_t)(len >> p.shift), rows = (int32_t)(len & ((1 << p.shift) - 1));
  const bool begun = rows > 0 && g > 0;
  int32_t tail = begun ? p.table[(int64_t)s * p.M + slot] : -1;
  int32_t held = 0;
  if (begun) {
    if (p.page_ok(tail)) {
      held = p.refs[tail];
    } else {
      atomicMax(&refused, PLC_ERR_INVALID);
      tail = -1;
    }
  }
  tails[s] = tail;
  __syncthreads();
  if (refused) {  // uniform: nobody writes it any more
    if (s == 0) {
      copies->count = 0;
      raise(status, refused);
    }
    return;
  }
  // The sessions that leave a shared page in this call leave it in order of their numbers; who finds itself the last
  // holder keeps it.
  bool copy = false;
  if (held > 1) {
    int32_t before = 0;
    for (int32_t o = 0; o < s; o += 4) {
      const int4 t = *reinterpret_cast<const int4 *>(tails + o);
      before += (t.x == tail) + (o + 1 < s && t.y == tail) + (o + 2 < s && t.z == tail) + (o + 3 < s && t.w == tail);
    }
    copy = held - before > 1;
  }
  const int32_t first = copy ? slot : pages_of(len, p.shift);
  const uint32_t need = (uint32_t)(pages_of(len + g, p.shift) - first);
  // A session may ask for 2^26 pages, all of them together for more than 32 bits count: the second sum takes the needs'
  // multiples of 2^21 along, above the copies.  Unless those alone are more than the pool has, the first sum is below
  // P + 1024 * 2^21 < 2^32, and exact.
  uint32_t total, sums;
  const uint32_t start = manager_scan(need, smem, &total);
  const uint32_t nth = manager_scan((need >> 21) << 11 | (copy ? 1u : 0u), smem, &sums) & 2047u;
  const uint32_t n_copies = sums & 2047u;
  if ((uint64_t)(sums >> 11) << 21 > (uint64_t)p.P) {
    if (s == 0) {
      copies->count = 0;
      raise(status, PLC_ERR_CAPACITY);
    }
    return;
  }
  start_of[s] = start;
  first_of[s] = first;
  __syncthreads();
  const uint32_t found = scan_pages(p, 0, p.P, false, ready, total, smem, [&](int32_t page, uint32_t rank) {
    if (rank < total) taken[rank] = page;
  });
  __syncthreads();
  if (found < total) {
    if (s == 0) {
      copies->count = 0;
      raise(status, PLC_ERR_CAPACITY);
    }
    return;
  }
  if (s == 0) copies->count = n_copies;
  for (uint32_t r = threadIdx.x; r < total; r += kManager) {
    int32_t lo = 0, hi = kManager - 1;  // the last session that starts at r or before: the one that r belongs to
    while (lo < hi) {
      const int32_t mid = (lo + hi + 1) >> 1;
      if (start_of[mid] <= r) lo = mid;
      else hi = mid - 1;
    }
    const int32_t page = taken[r];
    p.table[(int64_t)lo * p.M + first_of[lo] + (int32_t)(r - start_of[lo])] = page;
    p.refs[page] = 1;
  }
  if (copy) {
    copies->from[nth] = tail;
    copies->to[nth] = taken[start];
    copies->rows[nth] = rows;
    atomicSub(&p.refs[tail], 1);
  }
  if (g > 0) p.lens[s] = (int32_t)(len + g);
  if (kCopies) {
    __syncthreads();
    for (uint32_t i = 0; i < n_copies; ++i)
      copy_slabs<false, kManager>(p, copies->from[i], copies->to[i], copies->rows[i], 0, p.L * p.H);
  }
}

// One workgroup per session gives back the pages behind its new length.
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

__global__ __launch_bounds__(kBlock) void trim_kernel(PoolView p, const int32_t *__restrict__ new_lens, uint32_t *status) {
  trim_session<kBlock>(p, (int32_t)blockIdx.x, new_lens[blockIdx.x], status);
}

// The nodes of a session's tree that are kept: checked, as the kernels of plc_pages_accept need them.
struct Accepted {
  int32_t t, m, first;  // nodes, accepted ones, the first of them in `path`
  int64_t ctx;          // positions in front of the tree
  bool ok;
};
__device__ __forceinline__ Accepted accepted_of(const PoolView &p, int32_t s, const int32_t *off, const int32_t *path_off,
                                                int64_t path_len) {
  Accepted a;
  const int64_t len = p.lens[s], t = (int64_t)off[s + 1] - off[s], m = (int64_t)path_off[s + 1] - path_off[s];
  a.ok = len >= 0 && len <= ((int64_t)p.M << p.shift) && t >= 0 && t <= len && m >= 0 && m <= t && path_off[s] >= 0 &&
         path_off[s + 1] <= path_len;
  a.t = (int32_t)t, a.m = (int32_t)m, a.first = path_off[s], a.ctx = len - t;
  return a;
}

// Whether all of a session's path can be followed: its nodes ascend, the rows are on pages, and those that are written are
// its own.  Asked by a whole workgroup, at a time when nobody gives pages back.
template <int kThreads>
__device__ __forceinline__ bool path_ok(const PoolView &p, int32_t s, const Accepted &a, const int32_t *path) {
  bool ok = true;
  for (int32_t r = threadIdx.x; r < a.m; r += kThreads) {
    const int32_t node = path[a.first + r];
    if (node < r || node >= a.t || (r > 0 && node <= path[a.first + r - 1])) {
      ok = false;
    } else if (node != r) {
      const int64_t pf = a.ctx + node, pt = a.ctx + r;
      const int32_t page_f = p.table[(int64_t)s * p.M + (pf >> p.shift)], page_t = p.table[(int64_t)s * p.M + (pt >> p.shift)];
      ok = ok && p.page_ok(page_f) && p.page_ok(page_t) && p.refs[page_t] == 1;
    }
  }
  return __syncthreads_and(ok);
}

// The accepted sessions' new lengths.  A session whose path cannot be followed keeps its length, and all else that it has; of
// several sessions one could give back a page while another looks whether it is its own, so that the pages follow after this.
__global__ __launch_bounds__(kBlock) void accept_lens_kernel(PoolView p, const int32_t *__restrict__ off,
                                                             const int32_t *__restrict__ path, int64_t path_len,
                                                             const int32_t *__restrict__ path_off, uint32_t *status) {
  const int32_t s = (int32_t)blockIdx.x;
  const Accepted a = accepted_of(p, s, off, path_off, path_len);
  const bool ok = a.ok && path_ok<kBlock>(p, s, a, path);
  if (threadIdx.x != 0) return;
  if (ok) p.lens[s] = (int32_t)(a.ctx + a.m);
  else raise(status, PLC_ERR_INVALID);
}

// Gives back what pages a session still has behind its length, up to where its tree may have ended.
__global__ __launch_bounds__(kBlock) void accept_release_kernel(PoolView p, const int32_t *__restrict__ off, uint32_t *status) {
  const int32_t s = (int32_t)blockIdx.x;
  const int64_t most = (int64_t)p.M << p.shift, len = p.lens[s], t = (int64_t)off[s + 1] - off[s];
  if (len < 0 || len > most || t < 0) return;  // (the kernel before says so)
  const int32_t end = pages_of(min(len + t, most), p.shift);
  for (int32_t j = pages_of(len, p.shift) + (int32_t)threadIdx.x; j < end; j += kBlock) {
    int32_t *const entry = &p.table[(int64_t)s * p.M + j];
    const int32_t page = *entry;
    if (page == -1) continue;
    *entry = -1;
    if (p.page_ok(page)) atomicSub(&p.refs[page], 1);
    else raise(status, PLC_ERR_INVALID);
  }
}

// Pages in use at or above U (the number in use) go to the free ones below it: both in lists, and where page p went.
struct MoveList {
  uint32_t count, used, pad[2];
};
__global__ __launch_bounds__(kManager) void compact_kernel(PoolView p, MoveList *__restrict__ moves,
                                                           int32_t *__restrict__ holes, int32_t *__restrict__ movers,
                                                           int32_t *__restrict__ home, uint32_t *__restrict__ used_out) {
  __shared__ uint32_t smem[kManager / 64 + 1];
  const uint32_t all = 0xffffffffu, ready = used_bits(p, (int64_t)threadIdx.x * kScanWords);
  const uint32_t used = scan_pages(p, 0, p.P, true, ready, all, smem, [](int32_t, uint32_t) {});
  for (int32_t page = (int32_t)used + (int32_t)threadIdx.x; page < p.P; page += kManager) home[page] = -1;
  const uint32_t n = scan_pages(p, (int32_t)used, p.P, true, ready, all, smem,
                                [&](int32_t page, uint32_t rank) { movers[rank] = page; });
  scan_pages(p, 0, (int32_t)used, false, ready, n, smem, [&](int32_t page, uint32_t rank) { holes[rank] = page; });
  __syncthreads();
  for (uint32_t r = threadIdx.x; r < n; r += kManager) {
    const int32_t from = movers[r], to = holes[r];
    home[from] = to;
    p.refs[to] = p.refs[from];
    p.refs[from] = 0;
  }
  if (threadIdx.x == 0) {
    moves->count = n;
    moves->used = used;
    if (used_out) *used_out = used;
  }
}

// ---- rows ---------------------------------------------------------------------------------------------------------------

constexpr int kSlabs = 4;  // heads of a page that a workgroup copies at a time

__global__ __launch_bounds__(kBlock) void copy_tails_kernel(PoolView p, const CopyList *__restrict__ copies) {
  const uint32_t i = blockIdx.y;
  if (i >= copies->count) return;
  const int32_t slab = (int32_t)blockIdx.x * kSlabs, slabs = p.L * p.H;
  copy_slabs<false, kBlock>(p, copies->from[i], copies->to[i], copies->rows[i], slab, min(slab + kSlabs, slabs));
}

// The first `table_blocks` workgroups rewrite the tables, the others copy pages.
__global__ __launch_bounds__(kBlock) void move_pages_kernel(PoolView p, const MoveList *__restrict__ moves,
                                                            const int32_t *__restrict__ holes,
                                                            const int32_t *__restrict__ movers,
                                                            const int32_t *__restrict__ home, int32_t table_blocks,
                                                            uint32_t *status) {
  const uint32_t count = moves->count;
  if ((int32_t)blockIdx.x < table_blocks) {
    const int32_t used = (int32_t)moves->used;
    const int64_t entries = (int64_t)p.S * p.M;
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < entries; i += (int64_t)table_blocks * kBlock) {
      const int32_t page = p.table[i];
      if (page == -1) continue;
      if (p.page_ok(page) && page < used) continue;
      const int32_t to = p.page_ok(page) ? home[page] : -1;
      if (to >= 0) p.table[i] = to;
      else raise(status, PLC_ERR_INVALID);  // no page, or one that is counted as free
    }
    return;
  }
  const int32_t slabs = p.L * p.H, per_page = (slabs + kSlabs - 1) / kSlabs;
  const int64_t units = (int64_t)count * per_page;
  for (int64_t u = (int32_t)blockIdx.x - table_blocks; u < units; u += (int32_t)gridDim.x - table_blocks) {
    const int32_t i = (int32_t)(u / per_page), slab = (int32_t)(u % per_page) * kSlabs;
    copy_slabs<true, kBlock>(p, movers[i], holes[i], 1 << p.shift, slab, min(slab + kSlabs, slabs));
  }
}

// Rows of accepted nodes, along a path that can be followed, to the front of the tree.  A lane owns 16 bytes of a head's row and goes through the path in
// order, several nodes at a time, all of their loads before the first of their stores: a row goes only to places whose own
// node has been read (path[r] >= r, ascending).
constexpr int kPathRound = 64, kPathBatch = 8;
struct PathPlaces {
  int64_t from[kPathRound], to[kPathRound];
};
template <int kThreads>
__device__ __forceinline__ void accept_rows(const PoolView &p, int32_t s, const Accepted &a, const int32_t *path, int32_t i,
                                            PathPlaces *places) {
  const int32_t columns = 2 * p.L * p.H * p.d8;
  const int32_t c = i % p.d8, lh = i / p.d8 % (p.L * p.H);
  uint16_t *const base = (i < columns / 2 ? p.k : p.v) + (lh / p.H) * p.layer_s + (lh % p.H) * p.head_s + (int64_t)c * 8;
  for (int32_t r0 = 0; r0 < a.m; r0 += kPathRound) {
    __syncthreads();
    if (threadIdx.x < kPathRound) {
      const int32_t r = r0 + threadIdx.x;
      int64_t f = -1, t = -1;
      if (r < a.m) {
        const int32_t node = path[a.first + r];
        if (node != r) {
          const int64_t pf = a.ctx + node, pt = a.ctx + r, mask = (1 << p.shift) - 1;
          f = p.table[(int64_t)s * p.M + (pf >> p.shift)] * p.page_s + (pf & mask) * p.row_s;
          t = p.table[(int64_t)s * p.M + (pt >> p.shift)] * p.page_s + (pt & mask) * p.row_s;
        }
      }
      places->from[threadIdx.x] = f;
      places->to[threadIdx.x] = t;
    }
    __syncthreads();
    if (i < columns) {
      for (int32_t b = 0; b < min(kPathRound, a.m - r0); b += kPathBatch) {
        uint4 row[kPathBatch];
#pragma unroll
        for (int u = 0; u < kPathBatch; ++u)
          if (places->from[b + u] >= 0) row[u] = get16<false>(base + places->from[b + u]);
#pragma unroll
        for (int u = 0; u < kPathBatch; ++u)
          if (places->from[b + u] >= 0) put16<false>(base + places->to[b + u], row[u]);
      }
    }
  }
}

__global__ __launch_bounds__(kBlock) void accept_rows_kernel(PoolView p, const int32_t *__restrict__ off,
                                                             const int32_t *__restrict__ path, int64_t path_len,
                                                             const int32_t *__restrict__ path_off) {
  __shared__ PathPlaces places;
  const int32_t s = (int32_t)blockIdx.y;
  const Accepted a = accepted_of(p, s, off, path_off, path_len);
  if (!a.ok || !path_ok<kBlock>(p, s, a, path)) return;  // the next kernel says so
  accept_rows<kBlock>(p, s, a, path, (int32_t)blockIdx.x * kBlock + (int32_t)threadIdx.x, &places);
}

// All at once, for a single session of rows so short that one workgroup has them: two launches less.
__global__ __launch_bounds__(kManager) void accept_kernel(PoolView p, const int32_t *__restrict__ off,
                                                          const int32_t *__restrict__ path, int64_t path_len,
                                                          const int32_t *__restrict__ path_off, uint32_t *status) {
  __shared__ PathPlaces places;
  const Accepted a = accepted_of(p, 0, off, path_off, path_len);
  if (!a.ok || !path_ok<kManager>(p, 0, a, path)) {
    if (threadIdx.x == 0) raise(status, PLC_ERR_INVALID);
    return;
  }
  for (int32_t i = 0; i < 2 * p.L * p.H * p.d8; i += kManager) accept_rows<kManager>(p, 0, a, path, i + (int32_t)threadIdx.x, &places);
  __syncthreads();
  trim_session<kManager>(p, 0, a.ctx + a.m, status);
}

// Rows between a caller's buffer and pages.  A workgroup takes a block of consecutive rows, as many as give each thread 16
// bytes of one head, works out where they are, and goes through runs of heads: one, up to the 65,535 that a grid is wide.
constexpr int kHeadRun = 4;
struct RowsView {
  uint16_t *k, *v;
  int64_t rows, sess_s, layer_s, head_s, row_s;
  int32_t layer, layers, packed, per_block;
};
template <bool kStore, bool kStream>
__global__ __launch_bounds__(kBlock) void rows_kernel(PoolView p, RowsView r, const int32_t *__restrict__ off,
                                                      uint32_t *status) {
  extern __shared__ int64_t rows_lds[];  // [per_block] in the pool, [per_block] in the buffer, then off i32 [S + 1]
  int64_t *const in_pool = rows_lds, *const in_buf = rows_lds + r.per_block;
  int32_t *const o = reinterpret_cast<int32_t *>(rows_lds + 2 * r.per_block);
  for (int32_t s = threadIdx.x; s <= p.S; s += kBlock) o[s] = off[s];
  __syncthreads();
  const int64_t x0 = (int64_t)blockIdx.x * r.per_block;
  if (blockIdx.x == 0 && blockIdx.y == 0) {
    bool bad = o[0] != 0 || (r.packed && o[p.S] > r.rows);
    for (int32_t s = threadIdx.x; s < p.S; s += kBlock) bad = bad || o[s + 1] < o[s];
    if (bad) raise(status, PLC_ERR_INVALID);
  }
  for (int32_t b = threadIdx.x; b < r.per_block; b += kBlock) {
    const int64_t x = x0 + b;
    int64_t pool = -1, buf = 0;
    int32_t s = 0;
    int64_t i = 0;
    bool here;
    if (r.packed) {
      int32_t lo = 0, hi = p.S - 1;  // the last session that begins at x or before
      while (lo < hi) {
        const int32_t mid = (lo + hi + 1) >> 1;
        if (o[mid] <= x) lo = mid;
        else hi = mid - 1;
      }
      s = lo;
      i = x - o[s];
      here = x < r.rows && i >= 0 && x < o[s + 1];
      buf = x * r.row_s;
    } else {
      s = (int32_t)min(x / r.rows, (int64_t)p.S);
      i = x - s * r.rows;
      here = s < p.S && i < (int64_t)o[min(s, p.S - 1) + 1] - o[min(s, p.S - 1)];
      buf = s * r.sess_s + i * r.row_s;
    }
    if (here) {
      const int64_t t = (int64_t)o[s + 1] - o[s], len = p.lens[s];
      const int64_t pos = len - t + i;
      if (t > len || len > ((int64_t)p.M << p.shift) || (!r.packed && t > r.rows)) {
        raise(status, PLC_ERR_INVALID);
      } else {
        const int32_t page = p.table[(int64_t)s * p.M + (pos >> p.shift)];
        if (p.page_ok(page) && (!kStore || p.refs[page] == 1)) pool = page * p.page_s + (pos & ((1 << p.shift) - 1)) * p.row_s;
        else raise(status, PLC_ERR_INVALID);
      }
    }
    in_pool[b] = pool;
    in_buf[b] = buf;
  }
  __syncthreads();
  const int32_t heads = r.layers * p.H, items = r.per_block * p.d8;
  for (int32_t i = threadIdx.x; i < items; i += kBlock) {
    const int32_t b = i / p.d8, c = i - b * p.d8;
    if (in_pool[b] < 0) continue;
    const int64_t pool = in_pool[b] + r.layer * p.layer_s + (int64_t)c * 8, buf = in_buf[b] + (int64_t)c * 8;
    for (int32_t lh = (int32_t)blockIdx.y * kHeadRun; lh < heads; lh += (int32_t)gridDim.y * kHeadRun) {
      uint4 k[4], v[4];
      int64_t to[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int32_t e = min(lh + u, heads - 1), l = e / p.H, h = e - l * p.H;
        const int64_t at_pool = pool + l * p.layer_s + h * p.head_s, at_buf = buf + l * r.layer_s + h * r.head_s;
        k[u] = get16<kStream>((kStore ? r.k : p.k) + (kStore ? at_buf : at_pool));
        v[u] = get16<kStream>((kStore ? r.v : p.v) + (kStore ? at_buf : at_pool));
        to[u] = kStore ? at_pool : at_buf;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (lh + u < heads) {
          put16<kStream>((kStore ? p.k : r.k) + to[u], k[u]);
          put16<kStream>((kStore ? p.v : r.v) + to[u], v[u]);
        }
      }
    }
  }
}

// ---- host side ------------------------------------------------------------------------------------------------------------

constexpr int64_t kFewBytes = 256 << 10;  // that one workgroup may copy
constexpr int64_t kCached = (int64_t)96 << 20;  // bytes moved, in and out

size_t copy_list_bytes() { return align_up(sizeof(CopyList), 256); }
size_t workspace_bytes(const plc_pages *pages) {
  const size_t extend = copy_list_bytes() + 4 * (size_t)pages->P, compact = 256 + 12 * (size_t)pages->P;
  return align_up(extend > compact ? extend : compact, 256);
}

int move_rows(bool store, const plc_pages *pages, const plc_rows *rows, const int32_t *off, void *k, void *v,
              uint32_t *status, hipStream_t st) {
  if (!pages_valid(pages) || !rows || !aligned(off, 4) || !status) return PLC_ERR_INVALID;
  if (rows->layer < 0 || rows->layers < 1 || rows->layer > pages->L - rows->layers || rows->rows < 0 ||
      rows->rows > INT32_MAX || (rows->packed != 0 && rows->packed != 1))
    return PLC_ERR_INVALID;
  for (int i = 0; i < 4; ++i)
    if ((i > 0 || !rows->packed) && (rows->stride[i] < 0 || rows->stride[i] % 8)) return PLC_ERR_INVALID;
  if (rows->rows == 0) return PLC_OK;  // (an empty buffer may have no address)
  if (!aligned(k, 16) || !aligned(v, 16)) return PLC_ERR_INVALID;
  const PoolView p = pool_view(pages);
  RowsView r;
  r.k = static_cast<uint16_t *>(k), r.v = static_cast<uint16_t *>(v);
  r.rows = rows->rows;
  r.sess_s = rows->stride[0], r.layer_s = rows->stride[1], r.head_s = rows->stride[2], r.row_s = rows->stride[3];
  r.layer = rows->layer, r.layers = rows->layers, r.packed = rows->packed;
  r.per_block = p.d8 >= kBlock ? 1 : kBlock / p.d8;
  const int64_t total = rows->packed ? rows->rows : rows->rows * pages->S;
  const int64_t bx = (total + r.per_block - 1) / r.per_block, heads = (int64_t)r.layers * p.H,
                by = (heads + kHeadRun - 1) / kHeadRun;
  if (bx > INT32_MAX) return PLC_ERR_INVALID;
  const size_t lds = 16 * (size_t)r.per_block + 4 * (size_t)(p.S + 1);
  const dim3 grid((unsigned)bx, (unsigned)(by < 65535 ? by : 65535));
  const bool stream = (double)total * heads * p.d8 * 64 > (double)kCached;  // of both halves, in and out
  const auto kernel = !store ? &rows_kernel<false, false> : stream ? &rows_kernel<true, true> : &rows_kernel<true, false>;
  hipLaunchKernelGGL(kernel, grid, dim3(kBlock), lds, st, p, r, off, status);
  return launch_status();
}

}  // namespace
}  // namespace plc

using namespace plc;

extern "C" size_t plc_pages_workspace_bytes(const plc_pages *pages) { return pages_valid(pages) ? workspace_bytes(pages) : 0; }

extern "C" int plc_pages_fork(const plc_pages *pages, const int32_t *src, uint32_t *status, void *stream) {
  if (!pages_valid(pages) || !aligned(src, 4) || !status) return PLC_ERR_INVALID;
  const PoolView p = pool_view(pages);
  const size_t lds = 4 * (size_t)p.S * (kStrip + 1);
  if (lds > 64 * 1024)
    (void)hipFuncSetAttribute(reinterpret_cast<const void *>(&fork_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  hipLaunchKernelGGL(fork_kernel, dim3((unsigned)((p.M + kStrip - 1) / kStrip)), dim3(kBlock), lds,
                     static_cast<hipStream_t>(stream), p, src, status);
  return launch_status();
}

extern "C" int plc_pages_extend(const plc_pages *pages, const int32_t *grow, void *ws, size_t ws_bytes, uint32_t *status,
                                void *stream) {
  if (!pages_valid(pages) || !aligned(grow, 4) || !aligned(ws, 256) || ws_bytes < workspace_bytes(pages) || !status)
    return PLC_ERR_INVALID;
  const PoolView p = pool_view(pages);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  CopyList *const copies = static_cast<CopyList *>(ws);
  int32_t *const taken = reinterpret_cast<int32_t *>(static_cast<char *>(ws) + copy_list_bytes());
  const int64_t tails = (int64_t)p.S * p.L * p.H << p.shift;  // rows, of 16 d8 bytes in each half
  if (tails * p.d8 * 32 <= kFewBytes) {
    hipLaunchKernelGGL(extend_kernel<true>, dim3(1), dim3(kManager), 0, st, p, grow, copies, taken, status);
    return launch_status();
  }
  hipLaunchKernelGGL(extend_kernel<false>, dim3(1), dim3(kManager), 0, st, p, grow, copies, taken, status);
  hipLaunchKernelGGL(copy_tails_kernel, dim3((unsigned)((p.L * p.H + kSlabs - 1) / kSlabs), (unsigned)p.S), dim3(kBlock), 0, st,
                     p, copies);
  return launch_status();
}

extern "C" int plc_pages_trim(const plc_pages *pages, const int32_t *new_lens, uint32_t *status, void *stream) {
  if (!pages_valid(pages) || !aligned(new_lens, 4) || !status) return PLC_ERR_INVALID;
  hipLaunchKernelGGL(trim_kernel, dim3((unsigned)pages->S), dim3(kBlock), 0, static_cast<hipStream_t>(stream),
                     pool_view(pages), new_lens, status);
  return launch_status();
}

extern "C" int plc_pages_accept(const plc_pages *pages, const int32_t *off, const int32_t *path, int64_t path_len,
                                const int32_t *path_off, uint32_t *status, void *stream) {
  if (!pages_valid(pages) || !aligned(off, 4) || path_len < 0 || (path_len > 0 && !aligned(path, 4)) ||
      !aligned(path_off, 4) || !status)
    return PLC_ERR_INVALID;
  const PoolView p = pool_view(pages);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const int64_t columns = (int64_t)2 * p.L * p.H * p.d8;
  if (p.S == 1 && columns <= 2 * kManager) {
    hipLaunchKernelGGL(accept_kernel, dim3(1), dim3(kManager), 0, st, p, off, path, path_len, path_off, status);
    return launch_status();
  }
  if (path_len > 0)
    hipLaunchKernelGGL(accept_rows_kernel, dim3((unsigned)((columns + kBlock - 1) / kBlock), (unsigned)p.S), dim3(kBlock), 0,
                       st, p, off, path, path_len, path_off);
  hipLaunchKernelGGL(accept_lens_kernel, dim3((unsigned)p.S), dim3(kBlock), 0, st, p, off, path, path_len, path_off, status);
  hipLaunchKernelGGL(accept_release_kernel, dim3((unsigned)p.S), dim3(kBlock), 0, st, p, off, status);
  return launch_status();
}

extern "C" int plc_pages_compact(const plc_pages *pages, uint32_t *used, void *ws, size_t ws_bytes, uint32_t *status,
                                 void *stream) {
  if (!pages_valid(pages) || !aligned(ws, 256) || ws_bytes < workspace_bytes(pages) || !status) return PLC_ERR_INVALID;
  const PoolView p = pool_view(pages);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  MoveList *const moves = static_cast<MoveList *>(ws);
  int32_t *const holes = reinterpret_cast<int32_t *>(static_cast<char *>(ws) + 256), *const movers = holes + p.P,
                 *const home = movers + p.P;
  hipLaunchKernelGGL(compact_kernel, dim3(1), dim3(kManager), 0, st, p, moves, holes, movers, home, used);
  const int64_t entries = (int64_t)p.S * p.M, units = (int64_t)p.P / 2 * ((p.L * p.H + kSlabs - 1) / kSlabs);
  const int32_t table_blocks = (int32_t)(entries < 64 * kBlock ? (entries + kBlock - 1) / kBlock : 64);
  const int32_t copy_blocks = (int32_t)(units < 8 * kComputeUnits ? (units > 0 ? units : 1) : 8 * kComputeUnits);
  hipLaunchKernelGGL(move_pages_kernel, dim3((unsigned)(table_blocks + copy_blocks)), dim3(kBlock), 0, st, p, moves, holes,
                     movers, home, table_blocks, status);
  return launch_status();
}

extern "C" int plc_pages_store(const plc_pages *pages, const plc_rows *rows, const int32_t *off, const void *k, const void *v,
                               uint32_t *status, void *stream) {
  return move_rows(true, pages, rows, off, const_cast<void *>(k), const_cast<void *>(v), status,
                   static_cast<hipStream_t>(stream));
}

extern "C" int plc_pages_load(const plc_pages *pages, const plc_rows *rows, const int32_t *off, void *k, void *v,
                              uint32_t *status, void *stream) {
  return move_rows(false, pages, rows, off, k, v, status, static_cast<hipStream_t>(stream));
}
