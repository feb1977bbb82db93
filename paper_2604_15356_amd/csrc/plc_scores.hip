// What logits say of tokens: log-sum-exp, entropy, the log-probability of a given token and the k largest logits, in one pass over
// a row; see include/plc.h.
//
// A thread goes through the row's 16-byte pieces in steps of the workgroup and keeps a running maximum m, Z = sum 2^a and
// T = sum a 2^a, a = c x - c m with c = scale * log2(e): then lse = ln 2 (c m + log2 Z) and the entropy is ln 2 (log2 Z - T / Z).
// c m is rounded once, and the same number is taken from every c x by a fused product, so that its rounding drops out: below 2^24 it
// is half a unit at most, and no weight is above sqrt 2.  Beyond that it would take weights out of range (at -1e10, a mask's value, it is
// hundreds), so a maximum starts at -2^24: what lies far below weighs nothing, and where the whole row's lies beyond
// it on either side, the row is gone through again with a = c (x - its largest).
//
// The k largest: call what each of 64 fours of threads has seen a group.  The group with the k-th largest maximum bounds the k
// largest from below: at least k logits are as large.  What is not below it goes into a list in LDS: a thread looks its pieces through
// where they are all in its registers still; else it reads the piece that holds its maximum again, or all that it has seen, where
// the largest of its other pieces, which it has kept too, is not below the bound.  The list is ranked by counting.  Where it
// has no room for all (many large logits with few threads), the row is gone through again and the list shortened on the way.
// Keys are 64 bits, the logit as an ordered whole number over the token's complement: no two are equal, so that the
// result does not depend on the order they came in.
//
// What bounds it: HBM for many rows (4096 rows of 50,016 bf16 logits, 410 MB, k = 8: 83 us, 4.9 TB/s; k = 0 78 us, k = 32 85), a
// workgroup for each; for few the host's time, and behind that the steps of one workgroup, one behind the other (a row of 50,016, k = 4: 9.3
// us).  Long rows, where they are few, are cut into parts that a second kernel joins.  (A workgroup of 1024 threads for a row 12.2 us; the
// bound from 256 maxima 95 us for the 4096 rows; all that the threads with such maxima have seen read again 111 us for k = 32, where its scattered
// lines are as many as the row's; a bound from the first 8192 logits, and each piece looked at against it, 150.)
#include <type_traits>

#include "plc_device.h"

namespace plc {
namespace {

constexpr float kLn2 = 0.69314718055994530942f, kLog2e = 1.44269504088896340736f;
constexpr float kNothing = -0x1p24f;  // c m before anything was seen; from +-it on fp32 has no fractions, and the row is gone through again
constexpr float kGone = -200.0f;      // 2^kGone is zero
constexpr int kGroups = 64, kMostK = 32, kMostParts = 32;
constexpr int64_t kPartRows = 512;  // workgroups that rows are cut into parts for
constexpr int64_t kLongRow = 8192;  // pieces of a row that is

struct ScoreArgs {
  const char *logits;
  int64_t row_bytes, N;
  int32_t V, k, parts;
  float scale, scale2;
  const int32_t *tokens;
  float *logprob, *entropy, *lse;
  int32_t *ids;
  float *top_logprobs, *probs;
  int32_t *chosen;
  char *ws;
  uint32_t *status;
};

// Of a row, or of a part: the largest logit; Z and T of a = c (x - base) - shift.  base is zero but where the largest c x is 2^24 or more, or
// -2^24 or less.
struct Stats {
  float best, base, shift, z, t;
};
struct Part {
  Stats stats;
  uint32_t pad[3];
};

__device__ __forceinline__ uint64_t key_of(float x, uint32_t low) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);  // (-0 is 0)
  return (uint64_t)(u ^ (u >> 31 ? 0xffffffffu : 0x80000000u)) << 32 | low;
}
__device__ __forceinline__ float logit_of(uint64_t key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __builtin_bit_cast(float, u ^ (u >> 31 ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ int32_t token_of(uint64_t key) { return (int32_t)(0xffffffffu - (uint32_t)key); }

template <class T>
struct Logits {
  static constexpr int E = 16 / sizeof(T);  // of a piece
  const T *row;
  int32_t V, mis, pieces;  // logits between the 16-byte boundary below the row and its first
  __device__ __forceinline__ Logits(const ScoreArgs &a, int64_t x) {
    row = reinterpret_cast<const T *>(a.logits + x * a.row_bytes);
    V = a.V;
    mis = (int32_t)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    pieces = (mis + V + E - 1) / E;
  }
  // First and last token of a piece, which may lie outside of the row.
  __device__ __forceinline__ int32_t first_of(int32_t piece) const { return piece * E - mis; }
  __device__ __forceinline__ uint4 load(int32_t piece) const {
    typedef T T8 __attribute__((ext_vector_type(E)));
    const int32_t j = first_of(piece);
    if (j >= 0 && j + E <= V) return *reinterpret_cast<const uint4 *>(row + j);
    T8 v;
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = j + e >= 0 && j + e < V ? row[j + e] : (T)-__builtin_inff();
    return __builtin_bit_cast(uint4, v);
  }
  __device__ __forceinline__ uint4 whole(int32_t piece) const { return *reinterpret_cast<const uint4 *>(row + first_of(piece)); }
  static __device__ __forceinline__ void unpack(uint4 raw, float (&x)[E]) {
    typedef T T8 __attribute__((ext_vector_type(E)));
    const T8 v = __builtin_bit_cast(T8, raw);
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = (float)v[e];
  }
};

// Maximum and sum over the 64 lanes of a wavefront, the same in every lane: through the lanes' own registers, as wave_inclusive_scan.
template <int kControl, int kRows>
__device__ __forceinline__ float from_lane(float v, float otherwise) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, otherwise), __builtin_bit_cast(int, v), kControl, kRows, 0xf, false));
}
template <class Join>
__device__ __forceinline__ float wave_join(float v, float nothing, Join join) {
  v = join(v, from_lane<0x111, 0xf>(v, nothing));  // row_shr:1
  v = join(v, from_lane<0x112, 0xf>(v, nothing));  // row_shr:2
  v = join(v, from_lane<0x114, 0xf>(v, nothing));  // row_shr:4
  v = join(v, from_lane<0x118, 0xf>(v, nothing));  // row_shr:8
  v = join(v, from_lane<0x142, 0xa>(v, nothing));  // row_bcast:15 into rows 1 and 3
  v = join(v, from_lane<0x143, 0xc>(v, nothing));  // row_bcast:31 into rows 2 and 3
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
__device__ __forceinline__ float wave_max(float v) {
  return wave_join(v, -__builtin_inff(), [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float wave_add(float v) {
  return wave_join(v, 0.0f, [](float a, float b) { return a + b; });
}

// Brings sums from one reference to another, `d` below it.
__device__ __forceinline__ void rebase(float d, float *z, float *t) {
  d = fmaxf(d, kGone);
  const float f = __builtin_amdgcn_exp2f(d);
  *t = (*t + *z * d) * f;
  *z *= f;
}

// Candidates, and what is known of the k-th largest of all.
template <int kCap>
struct List {
  uint64_t keys[kCap], top[kMostK], bound;
  uint32_t count;
};

// Ranks the list: its k largest in order in `top` (zero where there are fewer), and unless it is the last time to its front.
template <bool kLast, int kCap>
__device__ __forceinline__ void rank(List<kCap> &list, int32_t k) {
  const uint32_t n = list.count;
  if (n < (uint32_t)k) {
    if (threadIdx.x < kMostK) list.top[threadIdx.x] = 0;
    __syncthreads();
  }
  for (uint32_t i = threadIdx.x; i < n; i += kBlock) {
    const uint64_t mine = list.keys[i];
    uint32_t above = 0;
#pragma unroll 8
    for (uint32_t j = 0; j < n; ++j) above += list.keys[j] > mine;
    if (above < (uint32_t)k) list.top[above] = mine;
  }
  __syncthreads();
  if (kLast) return;
  if (threadIdx.x < (uint32_t)k) list.keys[threadIdx.x] = list.top[threadIdx.x];
  if (threadIdx.x == 0) {
    list.count = min(n, (uint32_t)k);
    if (n >= (uint32_t)k) list.bound = list.top[k - 1];
  }
  __syncthreads();
}

// The results of a row, by a whole workgroup.
template <class T>
__device__ __forceinline__ void finish(const ScoreArgs &a, int64_t x, const Stats &s, const uint64_t *top, int32_t *found) {
  const bool bad = !(s.z > 0.0f) || !(fabsf(s.best) < __builtin_inff());
  const int32_t token = a.tokens ? a.tokens[x] : -1;
  const bool known = token >= 0 && token < a.V;
  if (threadIdx.x == 0) *found = -1;
  __syncthreads();
  const float log_z = __builtin_amdgcn_logf(s.z), nan = __builtin_nanf("");
  // (halved until the end: c x may be out of range where its natural logarithm is not)
  const auto logprob = [&](float y) { return (__builtin_fmaf(y - s.base, 0.5f * a.scale2, -0.5f * s.shift) - 0.5f * log_z) * (2.0f * kLn2); };
  if (threadIdx.x < (uint32_t)a.k) {
    const uint64_t key = top[threadIdx.x];
    const int32_t id = bad ? -1 : token_of(key);
    const float lp = bad ? nan : logprob(logit_of(key));
    const int64_t at = x * a.k + threadIdx.x;
    if (a.ids) a.ids[at] = id;
    if (a.top_logprobs) a.top_logprobs[at] = lp;
    if (a.probs) a.probs[at] = bad ? nan : __builtin_amdgcn_exp2f(lp * kLog2e);
    if (known && id == token) *found = (int32_t)threadIdx.x;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    if (bad || (a.tokens && !known && token != -1)) raise(a.status, PLC_ERR_INVALID);
    if (a.lse) a.lse[x] = bad ? nan : __builtin_fmaf(s.base, a.scale, (s.shift + log_z) * kLn2);
    if (a.entropy) a.entropy[x] = bad ? nan : fmaxf(0.0f, (log_z - s.t / s.z) * kLn2);
    if (a.tokens && a.logprob) {
      float lp = token == -1 ? 0.0f : nan;
      if (known) lp = logprob((float)reinterpret_cast<const T *>(a.logits + x * a.row_bytes)[token]);
      a.logprob[x] = bad ? nan : lp;
    }
    if (a.tokens && a.chosen) a.chosen[x] = bad ? -1 : *found;
  }
}

template <class T>
struct ScoreShape {
  static constexpr int E = Logits<T>::E, kLimit = 256, kCap = kBlock * E + kLimit;  // of the list: shortened at; room
  static constexpr int kUnroll = 4, kRound = kBlock * kUnroll;  // pieces under way of a thread, of a workgroup
};

// A row, or a part of one, to a workgroup.
template <class T>
__global__ __launch_bounds__(kBlock) void score_kernel(ScoreArgs a) {
  using Shape = ScoreShape<T>;
  constexpr int E = Shape::E, kUnroll = Shape::kUnroll, kRound = Shape::kRound, kWaves = kBlock / 64, kOf = kBlock / kGroups;
  __shared__ List<Shape::kCap> list;
  __shared__ float meet[3][kWaves];
  __shared__ __attribute__((aligned(16))) uint64_t group_key[kGroups];
  __shared__ int32_t holders[kMostK * kOf], n_holders;
  __shared__ int32_t found;
  const int64_t x = blockIdx.x / (uint32_t)a.parts;
  const int32_t part = (int32_t)(blockIdx.x - (uint32_t)x * (uint32_t)a.parts);
  const Logits<T> row(a, x);
  const int32_t each = (row.pieces + a.parts - 1) / a.parts;
  const int32_t q0 = min(row.pieces, part * each), q1 = min(row.pieces, q0 + each);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  constexpr uint32_t kInf = sizeof(T) == 4 ? 0xff800000u : std::is_same<T, _Float16>::value ? 0xfc00fc00u : 0xff80ff80u;  // minus infinity
  if (threadIdx.x == 0) list.count = 0, list.bound = 0, n_holders = 0;

  // A piece's logits that may be among the k largest, to the list; not those that it has no room for, which its length tells.
  const auto take = [&](uint4 piece, int32_t j, uint64_t bound, float least) {
    float v[E];
    Logits<T>::unpack(piece, v);
    const int32_t first = row.first_of(j);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (!(v[e] >= least)) continue;
      const uint64_t key = key_of(v[e], 0xffffffffu - (uint32_t)(first + e));
      if (key < bound || first + e < 0 || first + e >= a.V) continue;
      const uint32_t at = atomicAdd(&list.count, 1u);
      if (at < (uint32_t)Shape::kCap) list.keys[at] = key;
    }
  };

  // this thread's largest logit, the first piece that holds it, and the largest of the other pieces
  float best = -__builtin_inff(), second = -__builtin_inff(), shift = kNothing, z = 0.0f, t = 0.0f;
  int32_t best_piece = q0 + (int32_t)threadIdx.x < q1 ? q0 + (int32_t)threadIdx.x : -1;
  uint4 raw[kUnroll];
  const bool ragged = row.mis != 0 || row.first_of(row.pieces) != row.V;  // its first or its last piece is not all its own
  for (int32_t r0 = q0; r0 < q1; r0 += kRound) {
    const int32_t j0 = r0 + (int32_t)threadIdx.x;
    if (r0 + kRound <= q1 && !(ragged && (r0 == 0 || r0 + kRound >= row.pieces))) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) raw[u] = row.whole(j0 + u * kBlock);
    } else {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) raw[u] = j0 + u * kBlock < q1 ? row.load(j0 + u * kBlock) : make_uint4(kInf, kInf, kInf, kInf);
    }
    const float before = best;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      float v[E];
      Logits<T>::unpack(raw[u], v);
      float most = v[0];
#pragma unroll
      for (int e = 1; e < E; ++e) most = fmaxf(most, v[e]);
      best_piece = most > best ? j0 + u * kBlock : best_piece;
      second = fmaxf(second, fminf(most, best));
      best = fmaxf(most, best);
    }
    if (best > before) {
      const float now = best * a.scale2;
      if (now > shift) {
        rebase(shift - now, &z, &t);
        shift = now;
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      float v[E], zs = 0.0f, ts = 0.0f;
      Logits<T>::unpack(raw[u], v);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float y = __builtin_fmaf(v[e], a.scale2, -shift), w = __builtin_amdgcn_exp2f(y);
        zs += w;
        ts = __builtin_fmaf(w, fmaxf(y, kGone), ts);  // (a weight of zero must not meet minus infinity)
      }
      z += zs, t += ts;
    }
  }

  // the workgroup's
  Stats s = {};
  const uint64_t mine = best_piece < 0 ? 0 : key_of(best, 0xffffffffu - (uint32_t)(row.first_of(best_piece) + E - 1));
  {
    uint64_t key = mine;
#pragma unroll
    for (int d = 1; d < kOf; d <<= 1) {
      const uint64_t other = (uint64_t)__shfl_xor((unsigned long long)key, d);
      key = other > key ? other : key;
    }
    if (threadIdx.x % kOf == 0) group_key[threadIdx.x / kOf] = key;
    const float m = wave_max(best);
    if (lane == 0) meet[0][wave] = m;
    __syncthreads();
    s.best = meet[0][0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) s.best = fmaxf(s.best, meet[0][w]);
    s.shift = s.best * a.scale2;
    const bool finite = fabsf(s.best) < __builtin_inff();
    if (finite && !(fabsf(s.shift) < -kNothing)) {  // once more, from the largest
      s.base = s.best, s.shift = 0.0f;
      z = t = 0.0f;
      for (int32_t j = q0 + (int32_t)threadIdx.x; j < q1; j += kBlock) {
        float v[E];
        Logits<T>::unpack(row.load(j), v);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float y = (v[e] - s.base) * a.scale2, w = __builtin_amdgcn_exp2f(y);
          z += w;
          t = __builtin_fmaf(w, fmaxf(y, kGone), t);
        }
      }
    } else if (finite) {
      rebase(shift - s.shift, &z, &t);
    }
    z = wave_add(z), t = wave_add(t);
    if (lane == 0) meet[1][wave] = z, meet[2][wave] = t;
  }
  if (a.k > 0) {
    {  // the group with the k-th largest maximum: kOf threads compare one with all
      const uint64_t key = group_key[threadIdx.x / kOf];
      const int g0 = (int)threadIdx.x % kOf * (kGroups / kOf);
      int32_t above = 0;
#pragma unroll
      for (int i = 0; i < kGroups / kOf; ++i) above += group_key[g0 + i] > key;
#pragma unroll
      for (int d = 1; d < kOf; d <<= 1) above += __shfl_xor(above, d);
      if (threadIdx.x % kOf == 0 && above == a.k - 1 && key != 0) list.bound = key;  // (no two are equal, but of groups without a piece)
    }
    __syncthreads();
    const uint64_t bound = list.bound;
    const float least = bound ? logit_of(bound) : -__builtin_inff();
    const bool holds = mine >= bound && mine != 0;
    const int32_t rounds = (q1 - q0 + kBlock - 1) / kBlock;
    if (q1 - q0 <= kRound) {  // a thread's pieces are all in its registers
      if (holds) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          const int32_t j = q0 + (int32_t)threadIdx.x + u * kBlock;
          if (j < q1) take(raw[u], j, bound, least);
        }
      }
    } else {
      if (holds) {
        if (second < least) take(row.load(best_piece), best_piece, bound, least);
        else holders[atomicAdd(&n_holders, 1)] = (int32_t)threadIdx.x;  // (in any order: so is the list)
      }
      __syncthreads();
      for (int32_t i = (int32_t)threadIdx.x; i < n_holders * rounds; i += kBlock * kUnroll) {
        int32_t j[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          const int32_t item = i + u * kBlock, h = item / rounds;
          j[u] = item < n_holders * rounds ? q0 + holders[h] + (item - h * rounds) * kBlock : q1;
          if (j[u] < q1) raw[u] = row.load(j[u]);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
          if (j[u] < q1) take(raw[u], j[u], bound, least);
      }
    }
  }
  __syncthreads();
  const bool too_many = a.k > 0 && list.count > (uint32_t)Shape::kCap;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) s.z += meet[1][w], s.t += meet[2][w];
  if (too_many) {  // all pieces again, and the list shortened, and with it the bound raised, where it grows long
    if (threadIdx.x == 0) list.count = 0;
    __syncthreads();
    for (int32_t r0 = q0; r0 < q1; r0 += kBlock) {
      const int32_t j = r0 + (int32_t)threadIdx.x;
      const uint64_t bound = list.bound;
      if (j < q1) take(row.load(j), j, bound, bound ? logit_of(bound) : -__builtin_inff());
      __syncthreads();  // (nobody adds to the list before everybody has read how long it is)
      const bool full = list.count > Shape::kLimit;
      __syncthreads();
      if (full) rank<false>(list, a.k);
    }
  }
  if (a.k > 0) rank<true>(list, a.k);
  if (a.parts == 1) {
    finish<T>(a, x, s, list.top, &found);
    return;
  }
  char *const to = a.ws + (int64_t)blockIdx.x * (sizeof(Part) + 8 * a.k);
  if (threadIdx.x == 0) *reinterpret_cast<Stats *>(to) = s;
  if (threadIdx.x < (uint32_t)a.k) reinterpret_cast<uint64_t *>(to + sizeof(Part))[threadIdx.x] = list.top[threadIdx.x];
}

// Joins the parts of a row.
template <class T>
__global__ __launch_bounds__(kBlock) void score_join_kernel(ScoreArgs a) {
  __shared__ List<kMostParts * kMostK> list;
  __shared__ Stats joined;
  __shared__ int32_t found;
  const int64_t x = blockIdx.x;
  const size_t bytes = sizeof(Part) + 8 * a.k;
  const char *const from = a.ws + x * a.parts * (int64_t)bytes;
  if (threadIdx.x < 64) {
    const bool here = (int)threadIdx.x < a.parts;
    Stats s = {-__builtin_inff(), 0.0f, 0.0f, 0.0f, 0.0f};
    if (here) s = *reinterpret_cast<const Stats *>(from + threadIdx.x * bytes);
    const float best = wave_max(s.best);
    const int owner = __builtin_ctzll(__ballot(s.best == best) | 1ull << 63);
    Stats all = {best, __shfl(s.base, owner), __shfl(s.shift, owner), 0.0f, 0.0f};
    if (here && s.best > -__builtin_inff() && best < __builtin_inff())
      rebase(__builtin_fmaf(s.base - all.base, a.scale2, s.shift - all.shift), &s.z, &s.t);
    all.z = wave_add(s.z), all.t = wave_add(s.t);
    if (threadIdx.x == 0) {
      joined = all;
      list.count = (uint32_t)(a.parts * a.k), list.bound = 0;
    }
  }
  for (int32_t i = threadIdx.x; i < a.parts * a.k; i += kBlock)
    list.keys[i] = reinterpret_cast<const uint64_t *>(from + i / a.k * bytes + sizeof(Part))[i % a.k];
  __syncthreads();
  if (a.k > 0) rank<true>(list, a.k);
  const Stats s = joined;
  finish<T>(a, x, s, list.top, &found);
}

template <class T>
int scores(ScoreArgs a, hipStream_t st) {
  // A workgroup has a row of 50,016 16-bit logits in 9.4 us; in parts and with the joining 8.9, but a launch costs the host 3.3 more.  Of 131,072
  // 15.6 against 10.2, of 300,000 30 against 12.7.  With more rows than half the compute units the chip is full as it is (300 rows of
  // 50,016 in 32 bits: 16.7 against 19.1).
  const int64_t pieces = ((int64_t)a.V * sizeof(T) + 15) / 16;
  int64_t parts = 1;
  if (2 * a.N <= kComputeUnits && pieces > kLongRow) {
    parts = (kPartRows + a.N - 1) / a.N;
    const int64_t most = (pieces + ScoreShape<T>::kRound - 1) / ScoreShape<T>::kRound;
    parts = parts > most ? most : parts;
    parts = parts > kMostParts ? kMostParts : parts;
  }
  a.parts = (int32_t)parts;
  hipLaunchKernelGGL(score_kernel<T>, dim3((unsigned)(a.N * a.parts)), dim3(kBlock), 0, st, a);
  if (a.parts > 1) hipLaunchKernelGGL(score_join_kernel<T>, dim3((unsigned)a.N), dim3(kBlock), 0, st, a);
  return launch_status();
}

bool shape_ok(int32_t V, int32_t k) { return V >= 1 && V <= 1 << 30 && k >= 0 && k <= kMostK && k <= V; }
size_t workspace_bytes(int32_t k) { return align_up((size_t)(2 * kPartRows) * (sizeof(Part) + 8 * (size_t)k), 256); }

}  // namespace
}  // namespace plc

using namespace plc;

extern "C" size_t plc_score_workspace_bytes(int32_t V, int32_t k) { return shape_ok(V, k) ? workspace_bytes(k) : 0; }

extern "C" int plc_score_tokens(int32_t type, const void *logits, int64_t row_stride, int64_t N, int32_t V, float scale,
                                const int32_t *tokens, int32_t k, float *logprob, float *entropy, float *lse, int32_t *ids,
                                float *top_logprobs, float *probs, int32_t *chosen, void *ws, size_t ws_bytes, uint32_t *status,
                                void *stream) {
  const auto fine = [](const void *p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; };  // (or null)
  if ((type != PLC_FP16 && type != PLC_BF16 && type != PLC_FP32) || row_stride < 0 || N < 0 || N >= 1 << 24 || !shape_ok(V, k) ||
      !(scale > 0.0f) || !(scale * kLog2e < __builtin_inff()) || !fine(tokens) || !fine(logprob) || !fine(entropy) || !fine(lse) ||
      !fine(ids) || !fine(top_logprobs) || !fine(probs) || !fine(chosen) || ((logprob || chosen) && !tokens) ||
      ((ids || top_logprobs || probs || chosen) && k == 0) || !status || reinterpret_cast<uintptr_t>(ws) % 256 || !ws ||
      ws_bytes < workspace_bytes(k))
    return PLC_ERR_INVALID;
  if (N == 0) return PLC_OK;
  const int size = type == PLC_FP32 ? 4 : 2;
  if (!logits || reinterpret_cast<uintptr_t>(logits) % size) return PLC_ERR_INVALID;
  ScoreArgs a = {};
  a.logits = static_cast<const char *>(logits), a.row_bytes = row_stride * size, a.N = N;
  a.V = V, a.k = k, a.scale = scale, a.scale2 = scale * kLog2e;
  a.tokens = tokens, a.logprob = logprob, a.entropy = entropy, a.lse = lse;
  a.ids = ids, a.top_logprobs = top_logprobs, a.probs = probs, a.chosen = chosen;
  a.ws = static_cast<char *>(ws), a.status = status;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return type == PLC_FP16 ? scores<_Float16>(a, st) : type == PLC_BF16 ? scores<__bf16>(a, st) : scores<float>(a, st);
}
