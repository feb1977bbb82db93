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
// Positions are cut into chunks, one workgroup each, joined by a second kernel where a session has more than one.  Inside a
// workgroup the wavefronts form RG groups of 32 rows that share what is loaded, and PG groups that take turns with the
// positions: a step of one token with few rows has a wavefront per 32 positions and no barrier, a large tree has four times
// 32 rows on the same positions.
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

constexpr float kLowest = -1.0e30f;   // stands for "nothing seen yet" in the running maximum (base-2 logarithms)
constexpr float kSlack = 8.0f;        // the maximum that weights are relative to may lag by so much: 2^8 in a weight
constexpr float kLn2 = 0.69314718055994530942f, kLog2e = 1.44269504088896340736f;
constexpr int kMaskWords = PLC_TREE_NODES / 64;

struct AttendArgs {
  PoolView p;
  int32_t layer, G, max_nodes, max_len, chunk;  // positions of a chunk
  int64_t N, q_node, q_head, out_node, out_head;
  const uint16_t *q;
  uint16_t *out;
  float *lse;
  const int32_t *off, *parents;
  float scale2;   // scale * log2(e)
  float *part_o;  // [chunk][N H G][d]
  float *part_ml; // [chunk][N H G][2]: maximum (base 2), sum
  uint32_t *status;
};

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
  static constexpr size_t kLds = kMain + (size_t)kRows * kMaskWords * 8 + PLC_TREE_NODES * 4;
  static_assert(kLds <= 160 * 1024, "LDS of a compute unit");
};

// Waits until at most N of this wavefront's loads are outstanding.
template <int N>
__device__ __forceinline__ void wait_loads() {
  static_assert(N >= 0 && N < 64, "vmcnt has six bits");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
  asm volatile("" ::: "memory");
}

// One step of the second product reads MD pairs of transposed pieces of V.  A transposing read gives 16 lanes the 4 x 16
// block that they address 8 bytes each of, a column to a lane (checked on the device).  Assembly, with its wait: the
// compiler takes the builtin for a reader of whatever the loads in flight write, and would wait for all of them.
template <int N>
__device__ __forceinline__ void read_transposed(const uint32_t (&at)[N][2], int base, short8v (&v)[N]) {
#if defined(__HIP_DEVICE_COMPILE__)
  short4v r[N][2];
#pragma unroll
  for (int m = 0; m < N; m += 2) {
    // (a wait of its own for each four: the products of the first can start while the last are read)
    asm volatile(
        "ds_read_b64_tr_b16 %0, %4\n\tds_read_b64_tr_b16 %1, %5\n\tds_read_b64_tr_b16 %2, %6\n\t"
        "ds_read_b64_tr_b16 %3, %7\n\ts_waitcnt lgkmcnt(0)"
        : "=&v"(r[m][0]), "=&v"(r[m][1]), "=&v"(r[m + 1][0]), "=&v"(r[m + 1][1])
        : "v"(at[m][0] + base), "v"(at[m][1] + base), "v"(at[m + 1][0] + base), "v"(at[m + 1][1] + base));
  }
#pragma unroll
  for (int m = 0; m < N; ++m) v[m] = __builtin_shufflevector(r[m][0], r[m][1], 0, 1, 2, 3, 4, 5, 6, 7);
#else
  (void)at, (void)base, (void)v;
#endif
}

template <class T, class Shape, bool kExact>
__global__ __launch_bounds__(Shape::kThreads) void attend_kernel(AttendArgs a) {
  constexpr int DP = Shape::DP, RG = Shape::RG, PG = Shape::PG, NT = Shape::NT;
  constexpr int KS = DP / 16, MD = DP / 32;
  extern __shared__ __attribute__((aligned(1024))) char attend_lds[];
  lds_char *const lds = (lds_char *)attend_lds;
  uint64_t *const masks = reinterpret_cast<uint64_t *>(attend_lds + Shape::kMain);  // [kRows][kMaskWords]
  int32_t *const up = reinterpret_cast<int32_t *>(masks + Shape::kRows * kMaskWords);
  const PoolView &p = a.p;
  const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), rg = wave % RG, pg = wave / RG;
  const int s = (int)blockIdx.z, chunk = (int)blockIdx.y;
  const int h = (int)blockIdx.x % p.H, row_tile = (int)blockIdx.x / p.H;

  const const_int *const off = (const const_int *)a.off;
  const int n0 = off[s], t = off[s + 1] - n0, len = ((const const_int *)p.lens)[s];
  if (t == 0) return;
  if (t < 0 || n0 < 0 || (int64_t)n0 + t > a.N || t > a.max_nodes || len < t || len > a.max_len ||
      len > ((int64_t)p.M << p.shift)) {
    if (threadIdx.x == 0 && chunk == 0 && blockIdx.x == 0) raise(a.status, PLC_ERR_INVALID);
    return;
  }
  const int R = t * a.G, r0 = row_tile * Shape::kRows;
  const int first = chunk * a.chunk;
  if (r0 >= R || first >= len) return;
  const int ctx = len - t;
  const bool chain = a.parents == nullptr;
  int last = min(len, first + a.chunk);
  if (chain) last = min(last, ctx + (min(R, r0 + Shape::kRows) - 1) / a.G + 1);  // what the tile's last node sees
  const bool whole = len <= a.chunk;  // the session's only chunk

  // this lane's row
  const int row = r0 + rg * 32 + col;
  const bool live = row < R;
  const int node = (live ? row : R - 1) / a.G, head = h * a.G + (live ? row : R - 1) % a.G;
  const int node0 = r0 / a.G;  // of the tile
  const int64_t out_row = (int64_t)(n0 + node) * (p.H * a.G) + head;

  // ancestors of the tile's nodes, where the chunk reaches into the tree
  if (!chain && last > ctx) {
    for (int i = threadIdx.x; i < t; i += Shape::kThreads) {
      int u = a.parents[n0 + i];
      if (u < -1 || u >= i) {
        raise(a.status, PLC_ERR_INVALID);
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
  // Which of the 32 positions from `pos` on this lane's node sees, the bits of its half's accumulators in front.
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
    return w >> (4 * half);
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
  constexpr int kUnits = 2 * NT;                       // runs of 16 positions, which never cross a page
  static_assert(kUnits % RG == 0 || RG % kUnits == 0, "units go round");
  constexpr int kPieces = RG <= kUnits ? 1 : RG / kUnits;  // wavefronts that share a unit
  constexpr int kMine = RG <= kUnits ? kUnits / RG : 1;    // units of a wavefront
  constexpr int kUnitLoads = kLoads16 / kPieces;
  static_assert(kUnitLoads >= 1 && kLoads16 % kPieces == 0, "whole loads");
  constexpr int kStageLoads = 2 * kMine * kUnitLoads;
  const int unit0 = RG <= kUnits ? rg * kMine : rg / kPieces, load0 = RG <= kUnits ? 0 : (rg % kPieces) * kUnitLoads;
  uint32_t lane_at[kUnitLoads];  // bytes from the first of a unit's rows
  bool wanted[kUnitLoads];
#pragma unroll
  for (int j = 0; j < kUnitLoads; ++j) {
    const int r = (load0 + j) * kRowsPerLoad + lane / kLanesPerRow, c = (lane % kLanesPerRow) ^ turn<DP>(r);
    lane_at[j] = 2 * (uint32_t)(r * (int)p.row_s + c * 8);
    wanted[j] = kExact || c < p.d8;
  }
  const int64_t head_at = a.layer * p.layer_s + h * p.head_s;
  const const_int *const table = (const const_int *)p.table + (int64_t)s * p.M;
  const int last_slot = (len - 1) >> p.shift, row_mask = (1 << p.shift) - 1;
  bool bad_page = false;
  auto page_at = [&](int pos) {  // (past the session's end any of its pages will do: no weight goes there)
    const int32_t page = table[min(pos >> p.shift, last_slot)];
    if (!p.page_ok(page)) bad_page = true;
    return p.page_ok(page) ? page : 0;
  };
  auto request = [&](int pos, int buf) {
#pragma unroll
    for (int m = 0; m < kMine; ++m) {
      const int unit = unit0 + m, at = pos + 16 * unit;
      const int64_t from = page_at(at) * p.page_s + head_at + (at & row_mask) * p.row_s;
      const char *const from_k = reinterpret_cast<const char *>(p.k + from), *const from_v = reinterpret_cast<const char *>(p.v + from);
      const int to = (pg * Shape::kBuffers + buf) * Shape::kStage + unit * (16 * DP * 2);
#pragma unroll
      for (int j = 0; j < kUnitLoads; ++j) {
#if defined(__HIP_DEVICE_COMPILE__)  // the host pass of the compiler does not know the device's load-to-LDS builtin
        if (wanted[j]) {
          __builtin_amdgcn_global_load_lds(from_k + lane_at[j], lds + to + (load0 + j) * 1024, 16, 0, 0);
          __builtin_amdgcn_global_load_lds(from_v + lane_at[j], lds + to + Shape::kHalf + (load0 + j) * 1024, 16, 0, 0);
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

  const int span = last - first;
  const int rounds = span > 0 ? (span + PG * Shape::kTile - 1) / (PG * Shape::kTile) : 0;
  auto pos_of = [&](int it) { return first + (it * PG + pg) * Shape::kTile; };
  if (rounds > 0 && pos_of(0) < last) request(pos_of(0), 0);
  for (int it = 0; it < rounds; ++it) {
    const int pos = pos_of(it);
    const bool mine = pos < last, more = it + 1 < rounds && pos_of(it + 1) < last;
    if (more) {
      request(pos_of(it + 1), (it + 1) & 1);
      wait_loads<kStageLoads>();
    } else {
      wait_loads<0>();
    }
    if (RG > 1) __syncthreads();
    if (mine) {
      const lds_char *const ks_lds = lds + (pg * Shape::kBuffers + (it & 1)) * Shape::kStage, *const vs_lds = ks_lds + Shape::kHalf;
      float16v sc[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[n][i] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const short8v kf = *(const __attribute__((address_space(3))) short8v *)(ks_lds + n * (32 * DP * 2) + k_at[ks]);
          sc[n] = mfma<T>(kf, qf[ks], sc[n]);
        }
      }
      const bool edge = pos + Shape::kTile > ctx;  // positions that not every row sees, or that are none
      if (edge) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const uint32_t w = pos + 32 * n + 32 > ctx ? sees(pos + 32 * n) : ~0u;
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
      if (__ballot(most > top + kSlack) != 0) {
        const float now = fmaxf(top, most), keep = __builtin_amdgcn_exp2f(top - now);
        top = now;
        sum *= keep;
#pragma unroll
        for (int m = 0; m < MD; ++m)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[m][i] *= keep;
      }
      short8v pf[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[n][i], a.scale2, -top));
          sum += w;
          sc[n][i] = w;
          pf[n][i >> 3][i & 7] = (short)round16<T>(w);
        }
      uint32_t odd[NT];  // positions of the tree, or behind the end, that hold an infinity or a NaN
#pragma unroll
      for (int n = 0; n < NT; ++n) odd[n] = 0;
      if (edge) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          bool found = false;
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
      const int vs_at = (pg * Shape::kBuffers + (it & 1)) * Shape::kStage + Shape::kHalf;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          short8v vf[MD];
          read_transposed(v_at, vs_at + n * (32 * DP * 2) + u * (16 * DP * 2), vf);
          if (odd[n]) {  // a weight of zero must not meet them: they are added by hand where the weight is not zero
#pragma unroll
            for (int m = 0; m < MD; ++m)
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (special<T>((uint16_t)vf[m][e])) vf[m][e] = 0;
          }
#pragma unroll
          for (int m = 0; m < MD; ++m) o[m] = mfma<T>(vf[m], pf[n][u], o[m]);
        }
#pragma unroll
      for (int n = 0; n < NT; ++n)
        for (uint32_t rest = odd[n]; rest; rest &= rest - 1) {
          const int r = __builtin_ctz(rest);
          float w = 0.0f;
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if ((r & 3) == (i & 3) && r >> 3 == i >> 2) w = sc[n][i];
          w = __shfl(w, col + 32 * ((r >> 2) & 1));
          if (w > 0.0f) {
#pragma unroll
            for (int m = 0; m < MD; ++m)
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const int e = 32 * m + 8 * (i >> 2) + 4 * half + (i & 3);
                const uint16_t bits = *(const __attribute__((address_space(3))) uint16_t *)(vs_lds + n * (32 * DP * 2) +
                                                                                            place<DP>(r, e >> 3) + (e & 7) * 2);
                if (special<T>(bits)) o[m][i] += w * (float)__builtin_bit_cast(T, bits);
              }
          }
        }
    }
    // The buffer is loaded into again in the next round.
    if (RG > 1) __syncthreads();
  }
  if (bad_page && lane == 0) raise(a.status, PLC_ERR_INVALID);
  {
    const Halves both = halves(sum);
    sum = both.lo + both.hi;
  }

  float *const part_o = a.part_o + ((int64_t)chunk * a.N * (p.H * a.G) + out_row) * (8 * p.d8);
  float *const part_ml = a.part_ml + ((int64_t)chunk * a.N * (p.H * a.G) + out_row) * 2;
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
          part_ml[0] = top;
          part_ml[1] = sum;
        }
      }
    }
    return;
  }

  // the positions groups meet: their sums, relative to the largest maximum, row by row
  __syncthreads();
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
    float peak = kLowest, total = 0.0f;
    float4v v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int g = 0; g < PG; ++g) peak = fmaxf(peak, meet_ml[2 * (g * Shape::kRows + r)]);
#pragma unroll
    for (int g = 0; g < PG; ++g) {
      const float w = __builtin_amdgcn_exp2f(meet_ml[2 * (g * Shape::kRows + r)] - peak);
      const float n = meet_ml[2 * (g * Shape::kRows + r) + 1];
      if (n != 0.0f) {  // (a group that has seen nothing has weight zero, not zero times what it holds)
        total += w * n;
        v += w * *reinterpret_cast<const float4v *>(meet + (g * Shape::kRows + r) * Shape::kOutRow + e);
      }
    }
    const int my_node = (r0 + r) / a.G, my_head = h * a.G + (r0 + r) % a.G;
    const int64_t to = (int64_t)(n0 + my_node) * (p.H * a.G) + my_head;
    if (whole) {
      const float scale = total == 0.0f ? 0.0f : 1.0f / total;
      *reinterpret_cast<ushort4 *>(a.out + (n0 + my_node) * a.out_node + my_head * a.out_head + e) =
          make_ushort4(round16<T>(v[0] * scale), round16<T>(v[1] * scale), round16<T>(v[2] * scale), round16<T>(v[3] * scale));
      if (e == 0 && a.lse) a.lse[to] = total == 0.0f ? -__builtin_inff() : (peak + __builtin_amdgcn_logf(total)) * kLn2;
    } else {
      const int64_t at = (int64_t)chunk * a.N * (p.H * a.G) + to;
      *reinterpret_cast<float4v *>(a.part_o + at * (8 * p.d8) + e) = v;
      if (e == 0) {
        a.part_ml[2 * at] = peak;
        a.part_ml[2 * at + 1] = total;
      }
    }
  }
}

// Joins the chunks of sessions that have several: four components to a lane.
template <class T>
__global__ __launch_bounds__(kBlock) void join_kernel(AttendArgs a) {
  const PoolView &p = a.p;
  const int s = (int)blockIdx.y;
  const int n0 = a.off[s], t = a.off[s + 1] - n0, len = p.lens[s];
  if (t <= 0 || n0 < 0 || (int64_t)n0 + t > a.N || t > a.max_nodes || len < t || len > a.max_len || len <= a.chunk ||
      len > ((int64_t)p.M << p.shift))
    return;
  const int heads = p.H * a.G, pieces = 2 * p.d8;
  const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
  if (i >= (int64_t)t * heads * pieces) return;
  const int e = (int)(i % pieces) * 4, x = (int)(i / pieces);
  const int node = n0 + x / heads, head = x % heads;
  const int64_t row = (int64_t)node * heads + head, step = a.N * heads;
  const int chunks = (len + a.chunk - 1) / a.chunk;
  float peak = kLowest;
  for (int c = 0; c < chunks; ++c) peak = fmaxf(peak, a.part_ml[2 * (c * step + row)]);
  float total = 0.0f;
  float4v v = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int c = 0; c < chunks; ++c) {
    const float2 ml = *reinterpret_cast<const float2 *>(a.part_ml + 2 * (c * step + row));
    if (ml.y != 0.0f) {
      const float w = __builtin_amdgcn_exp2f(ml.x - peak);
      total += w * ml.y;
      v += w * *reinterpret_cast<const float4v *>(a.part_o + (c * step + row) * (8 * p.d8) + e);
    }
  }
  const float scale = total == 0.0f ? 0.0f : 1.0f / total;
  *reinterpret_cast<ushort4 *>(a.out + node * a.out_node + head * a.out_head + e) =
      make_ushort4(round16<T>(v[0] * scale), round16<T>(v[1] * scale), round16<T>(v[2] * scale), round16<T>(v[3] * scale));
  if (e == 0 && a.lse) a.lse[row] = total == 0.0f ? -__builtin_inff() : (peak + __builtin_amdgcn_logf(total)) * kLn2;
}

// ---- host side ------------------------------------------------------------------------------------------------------------

struct AttendPlan {
  int rows, step;  // rows of a workgroup; positions that one round of it takes
  int64_t row_tiles, chunks;
  int32_t chunk;
};

AttendPlan attend_plan(const plc_pages *p, int32_t G, int32_t max_nodes, int32_t max_len) {
  AttendPlan plan;
  const int64_t rows = (int64_t)max_nodes * G;
  const bool wide = p->d > 128;
  plan.rows = rows <= 32 ? 32 : rows <= 64 || wide ? 64 : 128;
  plan.step = plan.rows == 32 ? (wide ? 64 : 128) : plan.rows == 64 ? (wide ? 32 : 64) : 64;
  plan.row_tiles = (rows + plan.rows - 1) / plan.rows;
  const int64_t groups = (int64_t)p->S * p->H * plan.row_tiles;
  int64_t chunks = (8 * kComputeUnits + groups - 1) / groups;
  const int64_t most = (max_len + 255) / 256;
  if (chunks > most) chunks = most;
  int64_t chunk = (max_len + chunks - 1) / chunks;
  chunk = (chunk + plan.step - 1) / plan.step * plan.step;
  plan.chunk = (int32_t)(chunk < INT32_MAX ? chunk : INT32_MAX / plan.step * plan.step);
  plan.chunks = (max_len + (int64_t)plan.chunk - 1) / plan.chunk;
  return plan;
}

bool attend_valid(const plc_pages *p, int32_t G, int64_t N, int32_t max_nodes, int32_t max_len) {
  return pages_valid(p) && p->d <= 256 && G >= 1 && N >= 0 && N <= INT32_MAX && max_nodes >= 1 && max_len >= 1 &&
         (int64_t)p->H * G <= 65536 && (int64_t)max_nodes * G <= INT32_MAX / 256 && p->stride[3] * 32 < (int64_t)1 << 30;
}

size_t attend_bytes(const plc_pages *p, int32_t G, int64_t N, const AttendPlan &plan) {
  if (plan.chunks <= 1) return 256;
  return align_up((size_t)plan.chunks * (size_t)N * p->H * G * (p->d + 2) * sizeof(float), 256);
}

template <class T, class Shape>
void launch_attend(const AttendArgs &a, dim3 grid, hipStream_t st) {
  const bool exact = 8 * a.p.d8 == Shape::DP;
  const auto kernel = exact ? &attend_kernel<T, Shape, true> : &attend_kernel<T, Shape, false>;
  (void)hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)Shape::kLds);
  hipLaunchKernelGGL(kernel, grid, dim3(Shape::kThreads), Shape::kLds, st, a);
}

template <class T, int DP>
void launch_attend(const AttendArgs &a, const AttendPlan &plan, dim3 grid, hipStream_t st) {
  if constexpr (DP <= 128) {
    if (plan.rows == 32) launch_attend<T, AttendShape<DP, 1, 4, 1>>(a, grid, st);
    else if (plan.rows == 64) launch_attend<T, AttendShape<DP, 2, 2, 1>>(a, grid, st);
    else launch_attend<T, AttendShape<DP, 4, 1, 2>>(a, grid, st);
  } else {
    if (plan.rows == 32) launch_attend<T, AttendShape<DP, 1, 2, 1>>(a, grid, st);
    else launch_attend<T, AttendShape<DP, 2, 1, 1>>(a, grid, st);
  }
}

template <class T>
int attend(const AttendArgs &a, const AttendPlan &plan, hipStream_t st) {
  const dim3 grid((unsigned)(plan.row_tiles * a.p.H), (unsigned)plan.chunks, (unsigned)a.p.S);
  const int d = 8 * a.p.d8;
  if (d <= 64) launch_attend<T, 64>(a, plan, grid, st);
  else if (d <= 128) launch_attend<T, 128>(a, plan, grid, st);
  else launch_attend<T, 256>(a, plan, grid, st);
  if (plan.chunks > 1) {
    const int64_t lanes = (int64_t)a.max_nodes * a.p.H * a.G * 2 * a.p.d8;
    hipLaunchKernelGGL(join_kernel<T>, dim3((unsigned)((lanes + kBlock - 1) / kBlock), (unsigned)a.p.S), dim3(kBlock), 0, st, a);
  }
  return launch_status();
}

}  // namespace
}  // namespace plc

using namespace plc;

extern "C" size_t plc_attend_workspace_bytes(const plc_pages *pages, int32_t G, int64_t N, int32_t max_nodes, int32_t max_len) {
  if (!attend_valid(pages, G, N, max_nodes, max_len)) return 0;
  return attend_bytes(pages, G, N, attend_plan(pages, G, max_nodes, max_len));
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
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(ws, 256) || ws_bytes < attend_bytes(pages, G, N, plan))
    return PLC_ERR_INVALID;
  if (plan.row_tiles * pages->H > INT32_MAX || plan.chunks > 65535) return PLC_ERR_INVALID;
  AttendArgs a;
  a.p = pool_view(pages);
  a.layer = layer, a.G = G, a.max_nodes = max_nodes, a.max_len = max_len, a.chunk = plan.chunk;
  a.N = N, a.q_node = q_stride[0], a.q_head = q_stride[1], a.out_node = out_stride[0], a.out_head = out_stride[1];
  a.q = static_cast<const uint16_t *>(q), a.out = static_cast<uint16_t *>(out), a.lse = lse;
  a.off = off, a.parents = parents, a.scale2 = scale * kLog2e;
  a.part_ml = static_cast<float *>(ws);
  a.part_o = a.part_ml + (plan.chunks > 1 ? (size_t)plan.chunks * N * pages->H * G * 2 : 0);
  a.status = status;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return type == PLC_FP16 ? attend<_Float16>(a, plan, st) : attend<__bf16>(a, plan, st);
}
