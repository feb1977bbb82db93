// Attention of a session's last positions over its pages; see include/plc.h for the formula.
//
// The rows of a KV head are the nodes times the G query heads that read it.  A wavefront keeps 32 of them in its columns:
//   S^T [positions, rows] = K [positions, d] * Q^T [d, rows]       v_mfma 32x32x16, K from LDS, Q in registers
//   O^T [d, rows]        += V^T [d, positions] * P^T [positions, rows]
// so that the maximum, the sum and the scale of a row are a lane's own (its two halves hold the positions between them), and
// the accumulators of S^T, exponentiated and rounded, are the operand P^T of the second product as they stand: with the
// accumulators' positions 8 a + 4 h + b (lane half h, a, b = 0..3) taken as the order of the product's inner index, V^T has
// to come in that same order, which two transposing LDS reads of 4 positions x 16 components give.
//
// Inside a workgroup the wavefronts form RG groups of 32 rows that share what is loaded, and PG groups that take turns with
// the positions: a step of one token with few rows has up to four wavefronts on positions of their own and no barrier, a
// large tree has four times 32 rows on the same positions (launch_attend has the rule).
//
// The work is a line of chunks: session after session, in each its tiles of rows and heads, in each of those its positions,
// cut where they are long, or where there are few rows and heads to fill the chip with (attend_plan has the rule).
// Workgroups take the chunks in turn; what a cut has split is joined by a second kernel.
//
// What bounds it: few rows, HBM (64 sessions of one token, 8 heads, 4 query heads each, all of 4096 positions: 1.07 GB in
// 188 us, 5.7 TB/s; with lengths evenly up to 4096 547 MB in 114 us, 4.8 TB/s, the longest one ends last).  Many rows, the turns
// of the matrix cores and the vector units (64 nodes, 32,768 positions: 34 GFLOP in 60 us with the joining, 0.57 PFLOP/s; the
// matrix cores are busy 0.34 of the kernel's 52 us, vector instructions are issued in 0.40, a third of their time the wavefronts
// wait at barriers and for LDS; a chain of 2048 nodes after 8192 positions 504 us, 0.68 PFLOP/s).  Short contexts, the 4 us
// from a workgroup's start to its first products (offsets, table, pages, one after the other) and 4 to 5 us of its end.
#include <atomic>
#include <type_traits>

#include "plc_device.h"
#include "plc_paged.h"

namespace plc {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef short short8v __attribute__((ext_vector_type(8)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;
typedef const __attribute__((address_space(4))) int32_t const_int;  // read through the scalar cache: not written meanwhile

constexpr float kLowest = -__FLT_MAX__;  // stands for "nothing seen yet" in the running maximum (base-2 logarithms)
constexpr float kFar = 0x1p20f;       // maxima from which on scores are rounded before the maximum is subtracted
constexpr float kSlack = 8.0f;        // the maximum that weights are relative to may lag by so much: 2^8 in a weight
constexpr float kLn2 = 0.69314718055994530942f, kLog2e = 1.44269504088896340736f;
constexpr int kMaskWords = PLC_TREE_NODES / 64;
constexpr int kLineWords = 1024 + 1;  // where each session begins on it

struct AttendArgs {
  PoolView p;
  int32_t layer, G, max_nodes, max_len;
  int32_t tile_rows;  // rows of a tile
  int32_t chunk;      // positions of a chunk; 0: the work at hand in equal parts, one for each compute unit
  int64_t N, q_node, q_head, out_node, out_head;
  const uint16_t *q;
  uint16_t *out;
  float *lse;
  const int32_t *off, *parents;
  float scale2;   // scale * log2(e)
  float *part_o;  // [chunk][tile_rows][d]
  float *part_ml; // [chunk][tile_rows][2]: maximum (base 2), sum
  uint32_t *status;
};

// A session as its part of the line: none where what is said of it cannot be (status tells), or it has no nodes.
struct SessionView {
  int32_t n0, t, len, row_tiles;  // first node, nodes, positions, tiles of rows
  // chunks of one tile and head
  __device__ __forceinline__ uint32_t chunks(uint32_t chunk) const { return row_tiles ? ((uint32_t)len + chunk - 1) / chunk : 0u; }
};
__device__ __forceinline__ SessionView session_of(const AttendArgs &a, int s, bool *bad) {
  if (s >= a.p.S) return {};
  const int32_t n0 = a.off[s], n1 = a.off[s + 1], len = a.p.lens[s];
  SessionView v = {n0, n1 - n0, len, 0};
  if (v.t == 0) return v;
  if (v.t < 0 || n0 < 0 || n1 > a.N || v.t > a.max_nodes || len < v.t || len > a.max_len ||
      len > ((int64_t)a.p.M << a.p.shift)) {
    *bad = true;
    return v;
  }
  v.row_tiles = (v.t * a.G + a.tile_rows - 1) / a.tile_rows;
  return v;
}

// Where each session begins on the line, which ends at `total` (below 2^31: checked on the host).  Up to 64 sessions every
// wavefront holds for itself, a lane each; more are written down in LDS, line[S] being the total.
constexpr uint32_t kUnit = 128;  // a chunk's positions are a multiple
struct Line {
  uint32_t begin, total, chunk;
  SessionView v;
};
__device__ __forceinline__ Line draw_line(const AttendArgs &a, uint32_t *line, bool *bad) {
  const int lane = threadIdx.x & 63;
  const auto last_of = [](uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)x, 63); };
  const SessionView v0 = session_of(a, lane, bad);
  uint32_t chunk = (uint32_t)a.chunk;
  if (chunk == 0) {  // (fewer than 256 tiles and heads, of less than 2^23 units each)
    const auto weight = [&](const SessionView &v) { return (uint32_t)v.row_tiles * (uint32_t)a.p.H; };
    const auto length = [](const SessionView &v) { return ((uint32_t)v.len + kUnit - 1) / kUnit; };
    uint32_t n = wave_sum(weight(v0) * length(v0));
    for (int s0 = 64; s0 < a.p.S; s0 += 64) {
      const SessionView v = session_of(a, s0 + lane, bad);
      n += wave_sum(weight(v) * length(v));
    }
    uint32_t units = max(1u, (n + kComputeUnits - 1) / kComputeUnits);
    // No more long chunks than compute units: the ones left over would be a round of their own.  A tile and head's last chunk
    // is shorter than the others, so that the first length leaves too many; a few steps come close enough, with quotients that
    // need not be exact.  (20 sessions of 24,323 positions, 8 heads: 341 against 433 us.  Of short chunks it makes no difference:
    // 5 sessions of up to 4095 positions with trees of 27 nodes 30.3 and 30.5 us.  Beyond 64 sessions, of which a wavefront has
    // not all in its registers, the first length is taken.)
    if (units > 3 && a.p.S <= 64) {
#pragma unroll 1
      for (int step = 0; step < 4; ++step) {
        n = wave_sum(weight(v0) * (uint32_t)__builtin_ceilf((float)length(v0) * __builtin_amdgcn_rcpf((float)units)));
        if (n <= kComputeUnits) break;
        units = max(units + 1, (units * (n / 4) + kComputeUnits / 4 - 1) / (kComputeUnits / 4));
      }
    }
    chunk = units * kUnit;
  }
  Line mine = {0u, 0u, chunk, v0};
  uint32_t at = 0;
  for (int s0 = 0; s0 < a.p.S; s0 += 64) {
    const int s = s0 + lane;
    const SessionView v = s0 == 0 ? v0 : session_of(a, s, bad);
    const uint32_t n = (uint32_t)v.row_tiles * v.chunks(chunk) * (uint32_t)a.p.H, upto = wave_inclusive_scan(n);
    mine.begin = at + upto - n;
    if (a.p.S > 64 && threadIdx.x < 64 && s < a.p.S) line[s] = mine.begin;
    at += last_of(upto);
  }
  if (a.p.S > 64) {
    if (threadIdx.x == 0) line[a.p.S] = at;
    __syncthreads();
  }
  mine.total = at;
  return mine;
}

template <class T>
__device__ __forceinline__ float16v mfma(short8v a, short8v b, float16v c) {
  if constexpr (std::is_same<T, _Float16>::value)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

template <class T>
__device__ __forceinline__ uint16_t round16(float x) {
  return __builtin_bit_cast(uint16_t, (T)x);
}

template <class T>
__device__ __forceinline__ bool special(uint16_t x) {  // infinity or NaN
  constexpr uint16_t e = std::is_same<T, _Float16>::value ? 0x7c00 : 0x7f80;
  return (x & e) == e;
}

// Adds weighted sums of values, times a weight that is above zero even where it has come out as zero: an infinity stays one.
__device__ __forceinline__ void add_weighed(float4v &to, float weight, float4v sums) {
  if (weight != 0.0f) {
    to += weight * sums;
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) to[k] += fabsf(sums[k]) == __builtin_inff() ? sums[k] : 0.0f;
  }
}

// A row's two halves: the value of the lower and of the upper 32 lanes, in both.
struct Halves {
  float lo, hi;
};
__device__ __forceinline__ Halves halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  return {__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1])};
}

// LDS layout of a stage: 32 positions' rows of DP components; the 16-byte piece c of row r stands in place c ^ turn(r).
// Both kinds of reads then spread over all banks: 16 consecutive rows' same piece (K), and 4 pieces of 4 + 4 rows (V).
template <int DP>
__device__ __forceinline__ int turn(int r) {
  return DP == 64 ? ((r >> 1) & 1) << 2 | ((r >> 2) & 3) : (r & 3) << 2 | ((r >> 2) & 3);
}
template <int DP>
__device__ __forceinline__ int place(int r, int c) {
  return r * (DP * 2) + ((c ^ turn<DP>(r)) << 4);
}

template <int DP_, int RG_, int PG_, int NT_>
struct AttendShape {
  static constexpr int DP = DP_, RG = RG_, PG = PG_, NT = NT_;
  static constexpr int kThreads = 64 * RG * PG, kRows = 32 * RG;
  static constexpr int kTile = 32 * NT;               // positions of a stage
  static constexpr int kHalf = kTile * DP * 2;        // bytes of a stage's K, and of its V
  static constexpr int kStage = 2 * kHalf, kBuffers = 2;
  static constexpr int kOutRow = DP + 4;              // floats of a row where partial results meet
  static constexpr size_t kMeet = PG > 1 ? (size_t)PG * kRows * (kOutRow + 2) * 4 : 0;
  static constexpr size_t kStages = (size_t)PG * kBuffers * kStage;
  static constexpr size_t kMain = kStages > kMeet ? kStages : kMeet;
  static constexpr size_t kLds = kMain + (size_t)kRows * kMaskWords * 8 + PLC_TREE_NODES * 4 + kLineWords * 4 + 2 * RG * PG * 4;
  static_assert(kLds <= 160 * 1024, "LDS of a compute unit");
  static constexpr int kWavesPerSimd = DP <= 128 ? 2 : 1;
};

// A pointer that is the same in all lanes, in scalar registers.
__device__ __forceinline__ const char *scalar_ptr(const char *ptr) {
  const uint64_t x = (uint64_t)(uintptr_t)ptr;
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32));
  return reinterpret_cast<const char *>((uintptr_t)((uint64_t)hi << 32 | lo));
}

// Waits until at most N of this wavefront's loads are outstanding.
template <int N>
__device__ __forceinline__ void wait_loads() {
  static_assert(N >= 0 && N < 64, "vmcnt has six bits");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
  asm volatile("" ::: "memory");
}

// A step of the second product takes 16 positions, of which it reads N pairs of transposed pieces of V; two steps' reads go
// out together (kApart: bytes between them).  A transposing read gives 16 lanes the 4 x 16 block that they address 8 bytes
// each of, a column to a lane (checked on the device).  Assembly, with its wait: the compiler takes the builtin for a reader
// of whatever the loads in flight write, and would wait for all of them.
template <int kOffset, int kApart, int N>
__device__ __forceinline__ void read_transposed(const uint32_t (&at)[N][2], short8v (&v)[2][N]) {
#if defined(__HIP_DEVICE_COMPILE__)
  short4v r[2][N][2];
  if constexpr (N == 2) {
    asm volatile(
        "ds_read_b64_tr_b16 %0, %8 offset:%12\n\tds_read_b64_tr_b16 %1, %9 offset:%12\n\t"
        "ds_read_b64_tr_b16 %2, %10 offset:%12\n\tds_read_b64_tr_b16 %3, %11 offset:%12\n\t"
        "ds_read_b64_tr_b16 %4, %8 offset:%13\n\tds_read_b64_tr_b16 %5, %9 offset:%13\n\t"
        "ds_read_b64_tr_b16 %6, %10 offset:%13\n\tds_read_b64_tr_b16 %7, %11 offset:%13\n\ts_waitcnt lgkmcnt(0)"
        : "=&v"(r[0][0][0]), "=&v"(r[0][0][1]), "=&v"(r[0][1][0]), "=&v"(r[0][1][1]), "=&v"(r[1][0][0]), "=&v"(r[1][0][1]),
          "=&v"(r[1][1][0]), "=&v"(r[1][1][1])
        : "v"(at[0][0]), "v"(at[0][1]), "v"(at[1][0]), "v"(at[1][1]), "n"(kOffset), "n"(kOffset + kApart));
  } else {
    static_assert(N % 4 == 0, "two or a multiple of four");
#pragma unroll
    for (int m = 0; m < N; m += 4)
      asm volatile(
          "ds_read_b64_tr_b16 %0, %16 offset:%24\n\tds_read_b64_tr_b16 %1, %17 offset:%24\n\t"
          "ds_read_b64_tr_b16 %2, %18 offset:%24\n\tds_read_b64_tr_b16 %3, %19 offset:%24\n\t"
          "ds_read_b64_tr_b16 %4, %20 offset:%24\n\tds_read_b64_tr_b16 %5, %21 offset:%24\n\t"
          "ds_read_b64_tr_b16 %6, %22 offset:%24\n\tds_read_b64_tr_b16 %7, %23 offset:%24\n\t"
          "ds_read_b64_tr_b16 %8, %16 offset:%25\n\tds_read_b64_tr_b16 %9, %17 offset:%25\n\t"
          "ds_read_b64_tr_b16 %10, %18 offset:%25\n\tds_read_b64_tr_b16 %11, %19 offset:%25\n\t"
          "ds_read_b64_tr_b16 %12, %20 offset:%25\n\tds_read_b64_tr_b16 %13, %21 offset:%25\n\t"
          "ds_read_b64_tr_b16 %14, %22 offset:%25\n\tds_read_b64_tr_b16 %15, %23 offset:%25\n\ts_waitcnt lgkmcnt(0)"
          : "=&v"(r[0][m][0]), "=&v"(r[0][m][1]), "=&v"(r[0][m + 1][0]), "=&v"(r[0][m + 1][1]), "=&v"(r[0][m + 2][0]),
            "=&v"(r[0][m + 2][1]), "=&v"(r[0][m + 3][0]), "=&v"(r[0][m + 3][1]), "=&v"(r[1][m][0]), "=&v"(r[1][m][1]),
            "=&v"(r[1][m + 1][0]), "=&v"(r[1][m + 1][1]), "=&v"(r[1][m + 2][0]), "=&v"(r[1][m + 2][1]), "=&v"(r[1][m + 3][0]),
            "=&v"(r[1][m + 3][1])
          : "v"(at[m][0]), "v"(at[m][1]), "v"(at[m + 1][0]), "v"(at[m + 1][1]), "v"(at[m + 2][0]), "v"(at[m + 2][1]),
            "v"(at[m + 3][0]), "v"(at[m + 3][1]), "n"(kOffset), "n"(kOffset + kApart));
  }
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int m = 0; m < N; ++m) v[u][m] = __builtin_shufflevector(r[u][m][0], r[u][m][1], 0, 1, 2, 3, 4, 5, 6, 7);
#else
  (void)at, (void)v;
#endif
}

// The workgroup's barrier, and no wait for loads that are still to come.
__device__ __forceinline__ void join_round() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((15 << 0) | (7 << 4) | (0 << 8) | (3 << 14));  // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <class T, class Shape, bool kExact>
__global__ __launch_bounds__(Shape::kThreads, Shape::kWavesPerSimd) void attend_kernel(AttendArgs a) {
  constexpr int DP = Shape::DP, RG = Shape::RG, PG = Shape::PG, NT = Shape::NT;
  constexpr int KS = DP / 16, MD = DP / 32;
  // What weights are relative to lies this far below the maximum it was taken from: fp16 holds weights from 2^-14 on with all of
  // its bits, down from 2^7 that is 2^-21 of the largest, and the largest, 2^7 2^8, in its range.
  constexpr float kLift = std::is_same<T, _Float16>::value ? 7.0f : 0.0f;
  extern __shared__ __attribute__((aligned(1024))) char attend_lds[];
  lds_char *const lds = (lds_char *)attend_lds;
  uint64_t *const masks = reinterpret_cast<uint64_t *>(attend_lds + Shape::kMain);  // [kRows][kMaskWords]
  int32_t *const up = reinterpret_cast<int32_t *>(masks + Shape::kRows * kMaskWords);
  const PoolView &p = a.p;
  const int lane_id = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), rg = wave % RG, pg = wave / RG;
  uint32_t *const line = reinterpret_cast<uint32_t *>(up + PLC_TREE_NODES);
  uint32_t *const said = line + kLineWords;  // [2][wavefronts]: what each found in its chunk, in turn in two places
  Line mine;
  {
    bool bad = false;
    mine = draw_line(a, line, &bad);
    unsigned id = blockIdx.x;
    asm("" : "+s"(id));  // (or the compiler takes the number, zero here, through a lane from then on, and all that follows from it)
    if (bad && id == 0) raise(a.status, PLC_ERR_INVALID);
  }
  const auto scalar = [](uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); };
  const uint32_t total = scalar(mine.total), chunk = scalar(mine.chunk);
  bool bad_page = false;
  constexpr uint32_t kAgain = 1, kBroken = 2;

  int turns = 0;
  bool again = false;  // the chunk is gone through a second time, with what few rows need and all would wait for
  for (uint32_t at = blockIdx.x; at < total; at += again ? 0 : gridDim.x, turns ^= 1) {
  // (what follows from the lane is worked out again for every chunk, and again behind its positions: kept in registers
  // throughout it would not leave room for two wavefronts a SIMD)
  int lane = lane_id;
  asm volatile("" : "+v"(lane));
  int half = lane >> 5, col = lane & 31;
  // the session that `at` lies in: the last that begins there or before
  int s, n0, t, len;
  uint32_t s_begin;
  if (p.S <= 64) {
    s = __builtin_popcountll(__ballot(lane < p.S && mine.begin <= at)) - 1;
    s_begin = (uint32_t)__builtin_amdgcn_readlane((int)mine.begin, s);
    n0 = __builtin_amdgcn_readlane(mine.v.n0, s), t = __builtin_amdgcn_readlane(mine.v.t, s), len = __builtin_amdgcn_readlane(mine.v.len, s);
  } else {
    s = -1;
    for (int s0 = 0; s0 < p.S; s0 += 64)
      s += __builtin_popcountll(__ballot(s0 + lane < p.S && line[min(s0 + lane, p.S)] <= at));
    s_begin = scalar(line[s]);
    const const_int *const off = (const const_int *)a.off;
    n0 = off[s], t = off[s + 1] - n0, len = ((const const_int *)p.lens)[s];
  }
  const uint32_t chunks = scalar(((uint32_t)len + chunk - 1) / chunk);
  const uint32_t pair = scalar((at - s_begin) / chunks), nth = at - s_begin - pair * chunks;
  const int row_tile = (int)scalar(pair / (uint32_t)p.H), h = (int)pair - row_tile * p.H;
  const bool whole = chunks == 1;

  const int R = t * a.G, r0 = row_tile * Shape::kRows;
  const int first = (int)(nth * chunk), ctx = len - t;
  const bool chain = a.parents == nullptr;
  int last = (int)min((uint32_t)(len - first), chunk) + first;
  if (chain) last = min(last, ctx + (int)scalar((uint32_t)(min(R, r0 + Shape::kRows) - 1) / (uint32_t)a.G) + 1);  // what the tile's last node sees

  // this lane's row
  int row = r0 + rg * 32 + col;
  bool live = row < R;
  int node = (live ? row : R - 1) / a.G, head = h * a.G + (live ? row : R - 1) % a.G;
  const int node0 = r0 / a.G;  // of the tile

  bool broken = false;  // a page or a parent is none: the chunk's rows are left alone

  // ancestors of the tile's nodes, where the chunk reaches into the tree
  if (!chain && last > ctx) {
    for (int i = threadIdx.x; i < t; i += Shape::kThreads) {
      int u = a.parents[n0 + i];
      if (u < -1 || u >= i) {
        raise(a.status, PLC_ERR_INVALID);
        broken = true;
        u = -1;
      }
      up[i] = u;
    }
    __syncthreads();
    const int nodes = (min(R, r0 + Shape::kRows) - 1) / a.G - node0 + 1;
    for (int i = threadIdx.x; i < nodes; i += Shape::kThreads) {
      uint64_t m[kMaskWords] = {};
      for (int u = node0 + i; u >= 0; u = up[u]) {  // numbers fall on the way up: this ends
#pragma unroll
        for (int w = 0; w < kMaskWords; ++w)
          if (u >> 6 == w) m[w] |= 1ull << (u & 63);
      }
#pragma unroll
      for (int w = 0; w < kMaskWords; ++w) masks[i * kMaskWords + w] = m[w];
    }
    __syncthreads();
  }
  // Which of the 32 positions from `pos` on this lane's node sees.
  auto sees = [&](int pos) -> uint32_t {
    const int at = pos - ctx;  // > -32
    uint32_t w;
    if (chain) {
      const int n = node + 1 - at;
      w = n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1;
    } else {
      const uint64_t *const m = masks + (node - node0) * kMaskWords;
      if (at < 0) {
        w = ((1u << -at) - 1) | ((uint32_t)m[0] << -at);
      } else {
        const int i = at >> 6, sh = at & 63;
        const uint64_t lo = i < kMaskWords ? m[i] : 0, hi = i + 1 < kMaskWords ? m[i + 1] : 0;
        w = (uint32_t)(lo >> sh) | (sh ? (uint32_t)(hi << (64 - sh)) : 0u);
      }
    }
    return w;
  };

  short8v qf[KS];
  {
    const uint16_t *const src = a.q + (n0 + node) * a.q_node + head * a.q_head + 8 * half;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      short8v v = {};
      if (live && (kExact || 16 * ks + 8 * half < 8 * p.d8)) v = *reinterpret_cast<const short8v *>(src + 16 * ks);
      qf[ks] = v;
    }
  }

  // ---- loads: this wavefront's share of its positions group's stages
  constexpr int kLanesPerRow = DP / 8, kRowsPerLoad = 64 / kLanesPerRow, kLoads16 = 16 / kRowsPerLoad;
  constexpr int kRuns = 2 * NT;                        // runs of 16 positions, which never cross a page
  static_assert(kRuns % RG == 0 || RG % kRuns == 0, "runs go round");
  constexpr int kPieces = RG <= kRuns ? 1 : RG / kRuns;  // wavefronts that share a run
  constexpr int kMine = RG <= kRuns ? kRuns / RG : 1;    // runs of a wavefront
  constexpr int kRunLoads = kLoads16 / kPieces;
  static_assert(kRunLoads >= 1 && kLoads16 % kPieces == 0, "whole loads");
  constexpr int kStageLoads = 2 * kMine * kRunLoads;
  const int run0 = RG <= kRuns ? rg * kMine : rg / kPieces, load0 = RG <= kRuns ? 0 : (rg % kPieces) * kRunLoads;
  uint32_t lane_at[kRunLoads];  // bytes from the first of a run's rows
  bool wanted[kRunLoads];
#pragma unroll
  for (int j = 0; j < kRunLoads; ++j) {
    const int r = (load0 + j) * kRowsPerLoad + lane / kLanesPerRow, c = (lane % kLanesPerRow) ^ turn<DP>(r);
    lane_at[j] = 2 * (uint32_t)(r * (int)p.row_s + c * 8);
    wanted[j] = kExact || c < p.d8;
  }
  const int64_t head_at = a.layer * p.layer_s + h * p.head_s;
  // The chunk's table entries, 64 at a time, a lane each: a page's number is then a readlane away, where a load of it
  // in front of each stage's loads would keep them waiting.
  const int32_t *const table = p.table + (int64_t)s * p.M;
  const int last_slot = (len - 1) >> p.shift, row_mask = (1 << p.shift) - 1;
  int slot0;
  int32_t entries;
  auto fetch_entries = [&](int slot) {
    slot0 = slot;
    entries = table[min(slot0 + lane, last_slot)];
    asm volatile("" : "+v"(entries));  // waited for here: where it is used, the loads under way would be taken along
  };
  fetch_entries(first >> p.shift);
  auto page_at = [&](int pos) {  // (past the session's end any of its pages will do: no weight goes there)
    const int slot = min(pos >> p.shift, last_slot);
    if (slot >= slot0 + 64) fetch_entries(slot);
    const int32_t page = __builtin_amdgcn_readlane(entries, slot - slot0);
    if (!p.page_ok(page)) broken = bad_page = true;
    return p.page_ok(page) ? page : 0;
  };
  auto request = [&](int pos, int buf) {
#pragma unroll
    for (int m = 0; m < kMine; ++m) {
      const int run = run0 + m, at = pos + 16 * run;
      const int64_t from = page_at(at) * p.page_s + head_at + (at & row_mask) * p.row_s;
      const char *from_k = reinterpret_cast<const char *>(p.k + from), *from_v = reinterpret_cast<const char *>(p.v + from);
      // (in scalars, and not to be folded into a pointer per lane and load that lives through the loop)
      from_k = scalar_ptr(from_k), from_v = scalar_ptr(from_v);
      const int to = (pg * Shape::kBuffers + buf) * Shape::kStage + run * (16 * DP * 2);
#pragma unroll
      for (int j = 0; j < kRunLoads; ++j) {
#if defined(__HIP_DEVICE_COMPILE__)  // the host pass of the compiler does not know the device's load-to-LDS builtin
        uint32_t mine = lane_at[j];
        asm("" : "+v"(mine));  // 32 bits, next to a scalar base: one address register a lane
        if (wanted[j]) {
          __builtin_amdgcn_global_load_lds(from_k + mine, lds + to + (load0 + j) * 1024, 16, 0, 0);
          __builtin_amdgcn_global_load_lds(from_v + mine, lds + to + Shape::kHalf + (load0 + j) * 1024, 16, 0, 0);
        }
#else
        (void)from_k, (void)from_v, (void)to, (void)lds, (void)lane_at, (void)wanted;
#endif
      }
    }
  };

  if (!kExact) {  // pieces behind the last component are never loaded: zeros, in K for the product with Q's
    for (int i = threadIdx.x * 16; i < (int)Shape::kStages; i += Shape::kThreads * 16)
      *reinterpret_cast<uint4 *>(attend_lds + i) = make_uint4(0u, 0u, 0u, 0u);
    __syncthreads();
  }

  // LDS addresses of this lane's fragments: K rows col, pieces 2 ks + half; V positions 4 half + lane % 16 / 4 (+ 8) of a
  // run of 16, components 32 m + 16 (lane / 16 % 2) + 4 (lane % 4)
  int k_at[KS];
  uint32_t v_at[MD][2];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) k_at[ks] = place<DP>(col, 2 * ks + half);
#pragma unroll
  for (int m = 0; m < MD; ++m)
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const int i = lane & 15;
      v_at[m][w] = (uint32_t)(uintptr_t)lds +
                   place<DP>(8 * w + 4 * half + (i >> 2), 4 * m + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1)) + (i & 1) * 8;
    }

  float16v o[MD];
#pragma unroll
  for (int m = 0; m < MD; ++m)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[m][i] = 0.0f;
  float top = kLowest, sum = 0.0f;
  bool set_aside = false;  // infinities or NaN of V, in a place that not every row sees

  const int span = last - first;
  const int rounds = span > 0 ? (span + PG * Shape::kTile - 1) / (PG * Shape::kTile) : 0;
  auto pos_of = [&](int it) { return first + (it * PG + pg) * Shape::kTile; };
  if (rounds > 0 && pos_of(0) < last) request(pos_of(0), 0);
  // Q has come before the loop begins: waited for inside it, it would take the loads under way along
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[ks]));
  for (int it = 0; it < rounds; ++it) {
    const int pos = pos_of(it);
    const bool here = pos < last, more = it + 1 < rounds && pos_of(it + 1) < last;
    if constexpr (RG > 1) {  // everybody's share of this stage has come, and everybody is done with the one before
      wait_loads<0>();
      join_round();
      if (more) request(pos_of(it + 1), (it + 1) & 1);
    } else if (more) {  // two stages under way while the older one is waited for
      request(pos_of(it + 1), (it + 1) & 1);
      wait_loads<kStageLoads>();
    } else {
      wait_loads<0>();
    }
    if (here) {
      const lds_char *const ks_lds = lds + (pg * Shape::kBuffers + (it & 1)) * Shape::kStage, *const vs_lds = ks_lds + Shape::kHalf;
      float16v sc[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[n][i] = 0.0f;
      // K's fragments four products ahead; fences keep the order
      short8v kf[2][4];
      auto read_k = [&](int g) {
#pragma unroll
        for (int i = 4 * g; i < 4 * g + 4; ++i)
          kf[g & 1][i & 3] = *(const __attribute__((address_space(3))) short8v *)(ks_lds + i % NT * (32 * DP * 2) + k_at[i / NT]);
      };
      read_k(0);
#pragma unroll
      for (int g = 0; g < KS * NT / 4; ++g) {
        if (g + 1 < KS * NT / 4) read_k(g + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 4 * g; i < 4 * g + 4; ++i) sc[i % NT] = mfma<T>(kf[g & 1][i & 3], qf[i / NT], sc[i % NT]);
        __builtin_amdgcn_sched_barrier(0);
      }
      const bool edge = pos + Shape::kTile > ctx;  // positions that not every row sees, or that are none
      if (edge) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const uint32_t w = pos + 32 * n + 32 > ctx ? sees(pos + 32 * n) >> (4 * half) : ~0u;  // the bits of its half's accumulators in front
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (!(w >> (8 * (i >> 2) + (i & 3)) & 1u)) sc[n][i] = -__builtin_inff();
        }
      }
      float most = sc[0][0];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) most = fmaxf(most, sc[n][i]);
      const Halves both = halves(most);
      most = fmaxf(both.lo, both.hi) * a.scale2;
      if (__ballot(most > top + (kSlack + kLift)) != 0) {
        const float now = most > top + (kSlack + kLift) ? most - kLift : top;  // (by a row's own scores: the others must not show in its roundings)
        const float keep = __builtin_amdgcn_exp2f(top - now);
        top = now;
        sum *= keep;
#pragma unroll
        for (int m = 0; m < MD; ++m)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[m][i] *= keep;
      }
      // A fused product less the maximum keeps what the maximum's own rounding has lost: a common factor of a row's weights, next
      // to one up to kFar (2^(2^-4)), and without bounds beyond it.
      float by = a.scale2;
      if (again && fabsf(top) > kFar) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 16; ++i) sc[n][i] *= a.scale2;
        by = 1.0f;
      }
      // The weights, rounded to the type of V, for a matrix product of 16-bit values: half a step each, as the result is rounded
      // once more at its end.  (In 32 bits the product would take two such products.)  Their sum takes them unrounded, a stage's
      // by themselves first: many small ones would lose their last bits to a large sum one by one.
      short8v pf[NT][2];
      float part_sum = 0.0f;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[n][i], by, -top));
          part_sum += w;
          pf[n][i >> 3][i & 7] = (short)round16<T>(w);
        }
      sum += part_sum;
      uint32_t odd[NT];  // positions of the tree, or behind the end, that hold an infinity or a NaN
#pragma unroll
      for (int n = 0; n < NT; ++n) odd[n] = 0;
      if (edge) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          bool found = false;
#pragma unroll 1
          for (int c = 0; c < DP / 16; ++c) {
            const short8v v = *(const __attribute__((address_space(3))) short8v *)(vs_lds + n * (32 * DP * 2) +
                                                                                   place<DP>(col, c * 2 + half));
#pragma unroll
            for (int e = 0; e < 8; ++e) found = found || special<T>((uint16_t)v[e]);
          }
          const uint64_t b = __ballot(found && pos + 32 * n + col >= ctx);
          odd[n] = (uint32_t)b | (uint32_t)(b >> 32);
        }
      }
      const uint32_t vs_at = (uint32_t)((pg * Shape::kBuffers + (it & 1)) * Shape::kStage + Shape::kHalf);
      uint32_t v_here[MD][2];
#pragma unroll
      for (int m = 0; m < MD; ++m) v_here[m][0] = v_at[m][0] + vs_at, v_here[m][1] = v_at[m][1] + vs_at;
      auto weigh = [&](auto nu) {  // 32 positions' products with their weights
        constexpr int n = decltype(nu)::value;
        short8v vf[2][MD];
        read_transposed<n * (32 * DP * 2), 16 * DP * 2>(v_here, vf);
        if (odd[n]) {  // a weight of zero must not meet them: they are added by hand in the end
          set_aside = true;
          const uint32_t mine = odd[n] >> (4 * half);
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int m = 0; m < MD; ++m)
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if ((mine >> (16 * u + 8 * (e >> 2) + (e & 3)) & 1u) && special<T>((uint16_t)vf[u][m][e])) vf[u][m][e] = 0;
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int m = 0; m < MD; ++m) o[m] = mfma<T>(vf[u][m], pf[n][u], o[m]);
      };
      weigh(std::integral_constant<int, 0>());
      if constexpr (NT == 2) weigh(std::integral_constant<int, 1>());
    }
  }
  // Infinities and NaN among the values.  A weight that was rounded to zero has made a NaN of an infinity, and so has a maximum
  // that leapt; the formula's weights are above zero.  So where a sum is not finite, or some were set aside, it is looked up once
  // more what there is of them among the positions that a row sees: that, added up, is the sum.  (The question costs 0.1 us for a
  // single token of a short session, 0.7 for five sessions' trees.)
  {
    float zeros[4] = {};
#pragma unroll
    for (int m = 0; m < MD; ++m)
#pragma unroll
      for (int i = 0; i < 16; ++i) zeros[i & 3] = __builtin_fmaf(o[m][i], 0.0f, zeros[i & 3]);
    const int from = __ballot((zeros[0] + zeros[1]) + (zeros[2] + zeros[3]) != 0.0f) ? first : set_aside ? max(first, ctx) : last;
    if (from < last) {
      uint32_t known[MD] = {};  // sums that consist of such values
      fetch_entries(first >> p.shift);
      for (int it = 0; it < rounds; ++it)
        for (int r0 = 0; r0 < Shape::kTile; r0 += kRowsPerLoad) {
          const int pos = pos_of(it) + r0, my_pos = pos + lane / kLanesPerRow, piece = lane % kLanesPerRow;
          if (pos + kRowsPerLoad <= from || pos >= last) continue;
          const int64_t at_page = page_at(pos) * p.page_s + head_at + (my_pos & row_mask) * p.row_s;
          short8v v = {};
          if (my_pos >= from && my_pos < last && piece < p.d8) v = *reinterpret_cast<const short8v *>(p.v + at_page + piece * 8);
          bool found = false;
#pragma unroll
          for (int e = 0; e < 8; ++e) found = found || special<T>((uint16_t)v[e]);
          for (uint64_t rest = __ballot(found); rest; rest &= rest - 1) {
            const int owner = __builtin_ctzll(rest), at_pos = pos + owner / kLanesPerRow, c = owner % kLanesPerRow, base = at_pos & ~31;
            const uint32_t w = base + 32 > ctx ? sees(base) : ~0u;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint16_t lo = (uint16_t)__builtin_amdgcn_readlane((uint16_t)v[e], owner);
              const uint16_t hi = (uint16_t)__builtin_amdgcn_readlane((uint16_t)v[e + 4], owner), bits = half ? hi : lo;
              if ((w >> (at_pos & 31) & 1u) && special<T>(bits)) {
#pragma unroll
                for (int m = 0; m < MD; ++m)
#pragma unroll
                  for (int b = 0; b < 4; ++b)
                    if (4 * m + b == c) {
                      const float x = (float)__builtin_bit_cast(T, bits);
                      o[m][4 * b + e] = known[m] >> (4 * b + e) & 1u ? o[m][4 * b + e] + x : x;
                      known[m] |= 1u << (4 * b + e);
                    }
              }
            }
          }
        }
    }
  }
  {
    const bool wants = fabsf(top) > kFar && top != kLowest;
    const uint32_t mine = (!again && __ballot(wants) ? kAgain : 0) | (__ballot(broken) ? kBroken : 0);
    if (lane == 0) said[turns * (RG * PG) + wave] = mine;
    __syncthreads();  // everybody is done with the stages and the masks
    // (Nobody writes in this place again before everybody has come to the barrier of the next turn, and so has read it.)
    uint32_t all = 0;
#pragma unroll
    for (int w = 0; w < RG * PG; ++w) all |= said[turns * (RG * PG) + w];
    all = scalar(all);
    again = all & kAgain;
    if (again) continue;
    broken = all & kBroken;
    if (whole && broken) continue;
  }
  {
    const Halves both = halves(sum);
    sum = both.lo + both.hi;
  }
  lane = lane_id;
  asm volatile("" : "+v"(lane));
  half = lane >> 5, col = lane & 31;
  row = r0 + rg * 32 + col;
  live = row < R;
  node = (live ? row : R - 1) / a.G, head = h * a.G + (live ? row : R - 1) % a.G;
  const int64_t out_row = (int64_t)(n0 + node) * (p.H * a.G) + head;

  const int64_t part = (int64_t)at * Shape::kRows + rg * 32 + col;
  float *const part_o = a.part_o + part * (8 * p.d8), *const part_ml = a.part_ml + part * 2;
  uint16_t *const out = a.out + (n0 + node) * a.out_node + head * a.out_head;
  if (PG == 1) {
    if (live) {
      const float scale = whole ? (sum == 0.0f ? 0.0f : 1.0f / sum) : 1.0f;
#pragma unroll
      for (int m = 0; m < MD; ++m)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const int e = 32 * m + 8 * b + 4 * half;
          if (!kExact && e >= 8 * p.d8) continue;
          float4v v = {o[m][4 * b], o[m][4 * b + 1], o[m][4 * b + 2], o[m][4 * b + 3]};
          if (whole) {
            ushort4 w = make_ushort4(round16<T>(v[0] * scale), round16<T>(v[1] * scale), round16<T>(v[2] * scale),
                                     round16<T>(v[3] * scale));
            if (sum == 0.0f) w = make_ushort4(0, 0, 0, 0);
            *reinterpret_cast<ushort4 *>(out + e) = w;
          } else {
            *reinterpret_cast<float4v *>(part_o + e) = v;
          }
        }
      if (half == 0) {
        if (whole) {
          if (a.lse) a.lse[out_row] = sum == 0.0f ? -__builtin_inff() : (top + __builtin_amdgcn_logf(sum)) * kLn2;
        } else {
          part_ml[0] = broken ? __builtin_nanf("") : top;
          part_ml[1] = sum;
        }
      }
    }
    continue;
  }

  // the positions groups meet: their sums, relative to the largest maximum, row by row
  float *const meet = reinterpret_cast<float *>(attend_lds);            // [PG][kRows][kOutRow]
  float *const meet_ml = meet + PG * Shape::kRows * Shape::kOutRow;     // [PG][kRows][2]
  {
    const int r = pg * Shape::kRows + rg * 32 + col;
#pragma unroll
    for (int m = 0; m < MD; ++m)
#pragma unroll
      for (int b = 0; b < 4; ++b)
        *reinterpret_cast<float4v *>(meet + r * Shape::kOutRow + 32 * m + 8 * b + 4 * half) =
            float4v{o[m][4 * b], o[m][4 * b + 1], o[m][4 * b + 2], o[m][4 * b + 3]};
    if (half == 0) {
      meet_ml[2 * r] = top;
      meet_ml[2 * r + 1] = sum;
    }
  }
  __syncthreads();
  constexpr int kPieces4 = DP / 4;
  for (int i = threadIdx.x; i < min(Shape::kRows, R - r0) * kPieces4; i += Shape::kThreads) {
    const int r = i / kPieces4, e = i % kPieces4 * 4;
    if (!kExact && e >= 8 * p.d8) continue;
    float peak = kLowest, sums = 0.0f;
    float4v v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int g = 0; g < PG; ++g) peak = fmaxf(peak, meet_ml[2 * (g * Shape::kRows + r)]);
#pragma unroll
    for (int g = 0; g < PG; ++g) {
      const float w = __builtin_amdgcn_exp2f(meet_ml[2 * (g * Shape::kRows + r)] - peak);
      const float n = meet_ml[2 * (g * Shape::kRows + r) + 1];
      if (n != 0.0f) {  // (a group that has seen nothing has weight zero, not zero times what it holds)
        sums += w * n;
        add_weighed(v, w, *reinterpret_cast<const float4v *>(meet + (g * Shape::kRows + r) * Shape::kOutRow + e));
      }
    }
    const int my_node = (r0 + r) / a.G, my_head = h * a.G + (r0 + r) % a.G;
    const int64_t to = (int64_t)(n0 + my_node) * (p.H * a.G) + my_head;
    if (whole) {
      const float scale = sums == 0.0f ? 0.0f : 1.0f / sums;
      *reinterpret_cast<ushort4 *>(a.out + (n0 + my_node) * a.out_node + my_head * a.out_head + e) =
          make_ushort4(round16<T>(v[0] * scale), round16<T>(v[1] * scale), round16<T>(v[2] * scale), round16<T>(v[3] * scale));
      if (e == 0 && a.lse) a.lse[to] = sums == 0.0f ? -__builtin_inff() : (peak + __builtin_amdgcn_logf(sums)) * kLn2;
    } else {
      const int64_t mine = (int64_t)at * Shape::kRows + r;
      *reinterpret_cast<float4v *>(a.part_o + mine * (8 * p.d8) + e) = v;
      if (e == 0) {
        a.part_ml[2 * mine] = broken ? __builtin_nanf("") : peak;
        a.part_ml[2 * mine + 1] = sums;
      }
    }
  }
  __syncthreads();  // the next chunk loads where they met
  }
  if (bad_page && lane_id == 0) raise(a.status, PLC_ERR_INVALID);
}

// Joins the chunks of rows whose positions were cut: four components to a lane, and kGroups groups of lanes that go through
// the parts in turn, each with a maximum of its own, so that all loads of a batch are under way at once.
constexpr int kJoinBatch = 8;
template <class T, int kGroups>
__global__ __launch_bounds__(kBlock) void join_kernel(AttendArgs a) {
  __shared__ uint32_t line[kLineWords];
  __shared__ float4v meet_o[kBlock];
  __shared__ float2 meet_ml[kBlock];
  constexpr int kLanes = kBlock / kGroups;
  const PoolView &p = a.p;
  bool bad = false;
  const Line mine = draw_line(a, line, &bad);
  const int s = (int)blockIdx.y;
  const uint32_t s_begin = p.S <= 64 ? (uint32_t)__builtin_amdgcn_readlane((int)mine.begin, s) : line[s];
  const SessionView v = session_of(a, s, &bad);
  const int row_tile = (int)blockIdx.x / p.H, h = (int)blockIdx.x % p.H;
  if (row_tile >= v.row_tiles) return;
  const int parts = (int)v.chunks(mine.chunk);
  if (parts <= 1) return;
  const int64_t part0 = (int64_t)s_begin + (int64_t)blockIdx.x * parts;
  const int pieces = 2 * p.d8, i = (int)blockIdx.z * kLanes + (int)threadIdx.x % kLanes, group = (int)threadIdx.x / kLanes;
  const int r = i / pieces, e = i % pieces * 4, row = row_tile * a.tile_rows + r;
  const bool here = r < a.tile_rows && row < v.t * a.G;
  float peak = kLowest, sums = 0.0f;
  bool broken = false;  // a part's maximum that is a NaN: the row is left alone
  float4v o = {0.0f, 0.0f, 0.0f, 0.0f};
  // (a part that has seen nothing has weight zero, not zero times what it holds)
  auto add = [&](float2 m, float4v x, float now) {
    const float w = __builtin_amdgcn_exp2f(m.x - now);
    const bool any = m.y != 0.0f;
    if (any) {
      sums += w * m.y;
      add_weighed(o, w, x);
    }
  };
  if (here) {
    for (int c = group; c < parts; c += kGroups * kJoinBatch) {
      float2 m[kJoinBatch];
      float4v x[kJoinBatch];
#pragma unroll
      for (int u = 0; u < kJoinBatch; ++u) {
        const int64_t part = (part0 + min(c + u * kGroups, parts - 1)) * a.tile_rows + r;
        m[u] = *reinterpret_cast<const float2 *>(a.part_ml + 2 * part);
        x[u] = *reinterpret_cast<const float4v *>(a.part_o + part * (8 * p.d8) + e);
        broken = broken || m[u].x != m[u].x;
        if (c + u * kGroups >= parts) m[u] = make_float2(kLowest, 0.0f);
      }
      float now = peak;
#pragma unroll
      for (int u = 0; u < kJoinBatch; ++u) now = fmaxf(now, m[u].x);
      const float keep = __builtin_amdgcn_exp2f(peak - now);
      peak = now;
      sums *= keep;
      const float4v before = o;
      o = float4v{0.0f, 0.0f, 0.0f, 0.0f};
      add_weighed(o, keep, before);
#pragma unroll
      for (int u = 0; u < kJoinBatch; ++u) add(m[u], x[u], now);
    }
  }
  meet_o[threadIdx.x] = o;
  meet_ml[threadIdx.x] = make_float2(broken ? __builtin_nanf("") : peak, sums);
  __syncthreads();
  if (group != 0 || !here) return;
#pragma unroll
  for (int g = 0; g < kGroups; ++g) broken = broken || meet_ml[threadIdx.x + g * kLanes].x != meet_ml[threadIdx.x + g * kLanes].x;
  if (broken) return;
#pragma unroll
  for (int g = 1; g < kGroups; ++g) peak = fmaxf(peak, meet_ml[threadIdx.x + g * kLanes].x);
  sums = 0.0f;
  o = float4v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int g = 0; g < kGroups; ++g) add(meet_ml[threadIdx.x + g * kLanes], meet_o[threadIdx.x + g * kLanes], peak);
  const int node = v.n0 + row / a.G, head = h * a.G + row % a.G;
  const float scale = sums == 0.0f ? 0.0f : 1.0f / sums;
  *reinterpret_cast<ushort4 *>(a.out + node * a.out_node + head * a.out_head + e) =
      make_ushort4(round16<T>(o[0] * scale), round16<T>(o[1] * scale), round16<T>(o[2] * scale), round16<T>(o[3] * scale));
  if (e == 0 && a.lse)
    a.lse[(int64_t)node * (p.H * a.G) + head] = sums == 0.0f ? -__builtin_inff() : (peak + __builtin_amdgcn_logf(sums)) * kLn2;
}

// ---- host side ------------------------------------------------------------------------------------------------------------

struct AttendPlan {
  int rows;                        // of a tile
  int32_t chunk;                   // positions; 0: set by the work at hand
  int64_t row_tiles, parts, line;  // tiles of a session, chunks of a tile and head (as far as is known here), chunks of all: at most
};

constexpr int64_t kMostGroups = 2048;  // workgroups: bounds from the host may be far above what there is to do
constexpr int kLongest = 8192;         // positions of a chunk
constexpr int64_t kPartRows = 131072;  // rows of partial results, at most, that long contexts of many sessions are cut for

AttendPlan attend_plan(const plc_pages *p, int32_t G, int32_t max_nodes, int32_t max_len) {
  AttendPlan plan;
  const int64_t rows = (int64_t)max_nodes * G;
  plan.rows = rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
  plan.row_tiles = (rows + plan.rows - 1) / plan.rows;
  const int64_t pairs = plan.row_tiles * p->H * p->S;
  // A chunk is a workgroup's work, and a workgroup's LDS a compute unit's.  Whole positions of a tile of rows and head need no
  // joining (a launch, 5 us), and where there is one for every compute unit nothing is gained by cutting them: 64 sessions x 8
  // heads of up to 4000 positions 108 us, cut in two 121 us.  Fewer are cut into as many chunks as there are compute units, of
  // a length that the kernels find from the sessions' own.  Short ones are quicker done by one workgroup: 8 heads of 4 rows, 600
  // positions 11.6 against 12.2 us, 800 positions 13.4 against 12.2; of 64 rows, 300 positions 15.1 against 16.1, 500 positions
  // 19.2 against 17.3; of 128 rows 21.4 against 21.0 and 25.9 against 20.8.  With more than half as many tiles and heads as compute
  // units (160), contexts of equal lengths are better whole (2400 positions 33.7 against 36.6 us), but the host does not know
  // them equal: evenly up to 1600 21.0 against 21.4, up to 2400 27.1 against 26.4.
  const int64_t enough = plan.rows == 32 ? 768 : 384;
  if (max_len > (2 * pairs > kComputeUnits ? 1536 : enough) && pairs < kComputeUnits) {
    plan.chunk = 0;
    plan.parts = (kComputeUnits + pairs - 1) / pairs;
    plan.line = kComputeUnits + pairs;  // a tile and head's last chunk may be short
    return plan;
  }
  int64_t chunk = max_len;
  if (max_len > enough) {
    const int64_t most = kPartRows / plan.rows / pairs;  // parts
    chunk = chunk > kLongest ? kLongest : chunk;
    if (most < 2) chunk = max_len;
    else if (chunk * most < max_len) chunk = (max_len + most - 1) / most;
  }
  plan.chunk = (int32_t)(chunk > INT32_MAX - (int64_t)kUnit ? INT32_MAX - (int64_t)kUnit + 1 : (chunk + kUnit - 1) / kUnit * kUnit);
  plan.parts = (max_len + (int64_t)plan.chunk - 1) / plan.chunk;
  plan.line = pairs > INT32_MAX ? INT64_MAX : pairs * plan.parts;
  return plan;
}

bool attend_valid(const plc_pages *p, int32_t G, int64_t N, int32_t max_nodes, int32_t max_len) {
  return pages_valid(p) && p->d <= 256 && G >= 1 && N >= 0 && N <= INT32_MAX && max_nodes >= 1 && max_len >= 1 &&
         (int64_t)p->H * G <= 65536 && (int64_t)max_nodes * G <= INT32_MAX / 256 && p->stride[3] * 32 < (int64_t)1 << 30;
}

size_t attend_bytes(const plc_pages *p, const AttendPlan &plan) {
  if (plan.parts <= 1) return 256;
  return align_up((size_t)plan.line * plan.rows * (p->d + 2) * sizeof(float), 256);
}

template <class T, class Shape>
void launch_attend(const AttendArgs &a, const AttendPlan &plan, hipStream_t st) {
  const bool exact = 8 * a.p.d8 == Shape::DP;
  const auto kernel = exact ? &attend_kernel<T, Shape, true> : &attend_kernel<T, Shape, false>;
  static std::atomic<uint64_t> sized{0};  // devices that know of the kernels' LDS: to tell them costs a call's host time over again
  int device = 0;
  (void)hipGetDevice(&device);
  const uint64_t bit = device < 64 ? 1ull << device : 0;
  if (!(sized.load(std::memory_order_relaxed) & bit)) {
    for (const auto f : {&attend_kernel<T, Shape, false>, &attend_kernel<T, Shape, true>})
      (void)hipFuncSetAttribute(reinterpret_cast<const void *>(f), hipFuncAttributeMaxDynamicSharedMemorySize, (int)Shape::kLds);
    sized.fetch_or(bit, std::memory_order_relaxed);
  }
  hipLaunchKernelGGL(kernel, dim3((unsigned)(plan.line < kMostGroups ? plan.line : kMostGroups)), dim3(Shape::kThreads), Shape::kLds, st, a);
}

template <class T, int DP>
void launch_attend(const AttendArgs &a, const AttendPlan &plan, hipStream_t st) {
  // A workgroup that fills a compute unit's LDS leaves fewer partial results, and more of it is under way for one tile and
  // head (64 sessions of 8 heads, up to 4096 positions: 112 against 120 us).  Where there are several tiles and heads for each
  // compute unit, two workgroups of half the size hide each other's beginnings and ends: 20 sessions of 64 heads and 243
  // positions 37 against 48 us, 64 sessions of 16 heads with trees of up to 27 nodes over up to 500 positions 56 against 81 us.
  const bool many = plan.line >= 4 * kComputeUnits;
  if constexpr (DP <= 128) {
    if (plan.rows == 32 && many) launch_attend<T, AttendShape<DP, 1, 2, 1>>(a, plan, st);
    else if (plan.rows == 32) launch_attend<T, AttendShape<DP, 1, 4, 1>>(a, plan, st);
    else if (plan.rows == 64 && many) launch_attend<T, AttendShape<DP, 2, 2, 1>>(a, plan, st);
    else if (plan.rows == 64) launch_attend<T, AttendShape<DP, 2, 4, 1>>(a, plan, st);
    else if (many) launch_attend<T, AttendShape<DP, 4, 1, 2>>(a, plan, st);
    else launch_attend<T, AttendShape<DP, 4, 2, 2>>(a, plan, st);
  } else {
    if (plan.rows == 32 && many) launch_attend<T, AttendShape<DP, 1, 1, 1>>(a, plan, st);
    else if (plan.rows == 32) launch_attend<T, AttendShape<DP, 1, 2, 1>>(a, plan, st);
    else if (plan.rows == 64 && many) launch_attend<T, AttendShape<DP, 2, 1, 1>>(a, plan, st);
    else if (plan.rows == 64) launch_attend<T, AttendShape<DP, 2, 2, 1>>(a, plan, st);
    else launch_attend<T, AttendShape<DP, 4, 1, 1>>(a, plan, st);
  }
}

template <class T>
int attend(const AttendArgs &a, const AttendPlan &plan, hipStream_t st) {
  const int d = 8 * a.p.d8;
  if (d <= 64) launch_attend<T, 64>(a, plan, st);
  else if (d <= 128) launch_attend<T, 128>(a, plan, st);
  else launch_attend<T, 256>(a, plan, st);
  if (plan.parts > 1) {
    const int64_t joined = (int64_t)a.max_nodes * a.G < plan.rows ? (int64_t)a.max_nodes * a.G : plan.rows;  // rows of a tile
    const int groups = plan.parts > 4 * kJoinBatch ? 16 : plan.parts > kJoinBatch ? 4 : 1;
    const auto join = groups == 16 ? &join_kernel<T, 16> : groups == 4 ? &join_kernel<T, 4> : &join_kernel<T, 1>;
    hipLaunchKernelGGL(join, dim3((unsigned)(plan.row_tiles * a.p.H), (unsigned)a.p.S,
                                  (unsigned)((joined * 2 * a.p.d8 * groups + kBlock - 1) / kBlock)),
                       dim3(kBlock), 0, st, a);
  }
  return launch_status();
}

}  // namespace
}  // namespace plc

using namespace plc;

extern "C" size_t plc_attend_workspace_bytes(const plc_pages *pages, int32_t G, int64_t N, int32_t max_nodes, int32_t max_len) {
  if (!attend_valid(pages, G, N, max_nodes, max_len)) return 0;
  const AttendPlan plan = attend_plan(pages, G, max_nodes, max_len);
  return plan.line > INT32_MAX ? 0 : attend_bytes(pages, plan);
}

extern "C" int plc_attend(const plc_pages *pages, int32_t layer, int32_t type, const void *q, const int64_t *q_stride,
                          int32_t G, int64_t N, const int32_t *off, const int32_t *parents, int32_t max_nodes,
                          int32_t max_len, float scale, void *out, const int64_t *out_stride, float *lse, void *ws,
                          size_t ws_bytes, uint32_t *status, void *stream) {
  if (!attend_valid(pages, G, N, max_nodes, max_len) || layer < 0 || layer >= pages->L || !q_stride || !out_stride ||
      !aligned(off, 4) || (parents && (!aligned(parents, 4) || max_nodes > PLC_TREE_NODES)) || (lse && !aligned(lse, 4)) ||
      !status || !(scale > 0.0f) || !(scale < __builtin_inff()) || (type != PLC_FP16 && type != PLC_BF16))
    return PLC_ERR_INVALID;
  for (int i = 0; i < 2; ++i)
    if (q_stride[i] < 0 || q_stride[i] % 8 || out_stride[i] < 0 || out_stride[i] % 8) return PLC_ERR_INVALID;
  if (N == 0) return PLC_OK;
  const AttendPlan plan = attend_plan(pages, G, max_nodes, max_len);
  if (plan.line > INT32_MAX || !aligned(q, 16) || !aligned(out, 16) || !aligned(ws, 256) ||
      ws_bytes < attend_bytes(pages, plan))
    return PLC_ERR_INVALID;
  AttendArgs a;
  a.p = pool_view(pages);
  a.layer = layer, a.G = G, a.max_nodes = max_nodes, a.max_len = max_len;
  a.tile_rows = plan.rows, a.chunk = plan.chunk;
  a.N = N, a.q_node = q_stride[0], a.q_head = q_stride[1], a.out_node = out_stride[0], a.out_head = out_stride[1];
  a.q = static_cast<const uint16_t *>(q), a.out = static_cast<uint16_t *>(out), a.lse = lse;
  a.off = off, a.parents = parents, a.scale2 = scale * kLog2e;
  a.part_ml = static_cast<float *>(ws);
  a.part_o = a.part_ml + (plan.parts > 1 ? (size_t)plan.line * plan.rows * 2 : 0);
  a.status = status;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return type == PLC_FP16 ? attend<_Float16>(a, plan, st) : attend<__bf16>(a, plan, st);
}
