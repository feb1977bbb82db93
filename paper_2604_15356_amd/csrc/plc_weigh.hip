// What positions receive of attention: for each position of a session and KV head the sum of the weights that the rows of a call
// give it, from the rows' log-sum-exp; see include/plc.h for the formula.
//
// A wavefront keeps 32 positions in its columns and takes the rows 32 at a time:
//   S [rows, positions] = Q [rows, d] * K^T [d, positions]       v_mfma 32x32x16
// so that a lane's 16 accumulators are rows of one position: their weights exp2(scale' S - lse') are added up in the lane itself,
// row by row in a fixed order, and only the two halves of a position meet at the end.  K is read once, straight into the operand's
// registers (a lane holds 16 bytes of its position's row at a time); nothing of the scores leaves the registers.
//
// What bounds it: few rows, HBM (64 sessions' tokens, 8 heads of 4, 128 components: after 4096 positions each 537 MB in 116 us, 4.6 TB/s; after
// up to 4096 273 MB in 64 us; staged through LDS the first took 113, past the caches 164).  Many rows, the turns of the matrix cores and the
// vector units: 32 x 32 scores of 128 components take 256 cycles of products, and some 64 vector instructions, 16 of them exponentials.  8
// sessions of 512 tokens after 8192 positions 334 us, 0.84 PFLOP/s, where the matrix cores are busy 0.39 of the time and vector instructions
// are issued 0.55; one such session 60 us, 0.58 PFLOP/s: its 544 workgroups are 2.1 for each compute unit, where some have 3.
// Stages of rows two or three ahead (61 and 80 us), two groups of wavefronts that take turns with the rows (70), 64 positions to a wavefront
// (83), 64 rows' scores at once where all rows see all positions (62), products among the exponentials of those before (59) and workgroups
// of 64 or 96 positions (152, 69) do not change that.
#include <atomic>
#include <type_traits>

#include "plc_device.h"
#include "plc_paged.h"

namespace plc {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short short8v __attribute__((ext_vector_type(8)));
typedef float float16v __attribute__((ext_vector_type(16)));

typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) float lds_float;
typedef float float4v __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kSpanOfGroup = 32 * (kBlock / 64);  // positions of a workgroup, 32 of each wavefront
constexpr int64_t kMostGroups = 1 << 16;  // workgroups: bounds from the host may be far above what there is to do

struct WeighArgs {
  PoolView p;
  WeightsView w;
  int32_t layer, G, max_nodes, max_len;
  int64_t N, q_node, q_head;
  const uint16_t *q;
  const float *lse;
  const int32_t *off;
  float scale2, decay;  // scale * log2(e)
  int32_t pairs;        // sessions and heads
  uint32_t *status;
};

template <class T>
__device__ __forceinline__ float16v mfma(short8v a, short8v b, float16v c) {
  if constexpr (std::is_same<T, _Float16>::value)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// A session's part in a call: none where what is said of it cannot be (status tells), or it has no nodes.
struct SessionView {
  int32_t n0, t, len;
  bool ok;
};
__device__ __forceinline__ SessionView session_of(const WeighArgs &a, int s, bool tell) {
  const int32_t n0 = a.off[s], n1 = a.off[s + 1], len = a.p.lens[s];
  SessionView v = {n0, n1 - n0, len, false};
  if (n1 == n0) return v;
  v.ok = n0 >= 0 && n1 > n0 && n1 <= a.N && v.t <= a.max_nodes && len >= v.t && len <= a.max_len &&
         len <= ((int64_t)a.p.M << a.p.shift) && len <= a.w.width;
  if (!v.ok && tell && threadIdx.x == 0) raise(a.status, PLC_ERR_INVALID);
  return v;
}

__device__ __forceinline__ void put_weight(const WeighArgs &a, float *at, bool old, float before, float sum) {
  *at = old && a.decay != 0.0f ? __builtin_fmaf(a.decay, before, sum) : sum;
}

// LDS layout of a stage of rows: rows of DP components; the 16-byte piece c of row r stands in place c ^ turn(r), so that 16 consecutive
// rows' same piece spread over all banks.
template <int DP>
__device__ __forceinline__ int turn(int r) {
  return DP == 64 ? r >> 1 & 7 : r & 15;
}
template <int DP>
__device__ __forceinline__ int place(int r, int c) {
  return r * (DP * 2) + ((c ^ turn<DP>(r)) << 4);
}

// Up to 32 rows: they stay in registers, and the positions stream by, kTiles times 32 for each wavefront, the next ones' rows of K on their way
// while one is worked on.
template <class T, int DP, int kTiles>
__global__ __launch_bounds__(kBlock, DP <= 128 ? 2 : 1) void weigh_few_kernel(WeighArgs a) {
  constexpr int KS = DP / 16;
  const PoolView &p = a.p;
  const int pair = (int)(blockIdx.x % (uint32_t)a.pairs), s = pair / p.H, h = pair - s * p.H;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, col = lane & 31;
  const SessionView v = session_of(a, s, pair % p.H == 0 && blockIdx.x < (uint32_t)a.pairs);
  if (!v.ok) return;
  const int32_t ctx = v.len - v.t, R = v.t * a.G;
  const int32_t *const table = p.table + (int64_t)s * p.M;
  const uint16_t *const keys = p.k + a.layer * p.layer_s + h * p.head_s + 8 * half;
  float *const weights = a.w.w + s * a.w.sess_s + a.layer * a.w.layer_s + h * a.w.head_s;
  const int32_t row_mask = (1 << p.shift) - 1;

  short8v qf[KS];
  float lse2[16];
  {
    const int32_t r = min(col, R - 1);
    const uint16_t *const q = a.q + (v.n0 + r / a.G) * a.q_node + (h * a.G + r % a.G) * a.q_head + 8 * half;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qf[ks] = short8v{};
      if (16 * ks + 8 * half < 8 * p.d8) qf[ks] = *reinterpret_cast<const short8v *>(q + 16 * ks);
    }
    // a lane's log-sum-exp, from which the rows' are handed out
    const float mine = a.lse[(int64_t)(v.n0 + r / a.G) * (p.H * a.G) + h * a.G + r % a.G] * kLog2e;
#pragma unroll
    for (int i = 0; i < 16; ++i) lse2[i] = __shfl(mine, 8 * (i >> 2) + 4 * half + (i & 3));
  }

  const int32_t span = kTiles * 32 * (kBlock / 64), step = (int32_t)(gridDim.x / (uint32_t)a.pairs);
  for (int32_t chunk = (int32_t)(blockIdx.x / (uint32_t)a.pairs); (int64_t)chunk * span < v.len; chunk += step) {
    const int32_t first = chunk * span + wave * kTiles * 32;
    if (first >= v.len) continue;
    int32_t page[kTiles];
#pragma unroll
    for (int n = 0; n < kTiles; ++n) page[n] = table[min(first + 32 * n + col, v.len - 1) >> p.shift];
    short8v kf[2][KS];
    float before[2];
    const auto request = [&](int n) {
      const int32_t at = min(first + 32 * n + col, v.len - 1);
      const uint16_t *const k = keys + (p.page_ok(page[n]) ? page[n] : 0) * p.page_s + (at & row_mask) * p.row_s;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        kf[n & 1][ks] = short8v{};
        if (16 * ks + 8 * half < 8 * p.d8) kf[n & 1][ks] = *reinterpret_cast<const short8v *>(k + 16 * ks);
      }
      before[n & 1] = a.decay != 0.0f ? weights[at] : 0.0f;
    };
    request(0);
#pragma unroll
    for (int n = 0; n < kTiles; ++n) {
      if (first + 32 * n >= v.len) break;
      if (n + 1 < kTiles) request(n + 1);
      float16v sc;
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] = 0.0f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) sc = mfma<T>(qf[ks], kf[n & 1][ks], sc);
      const int32_t pos = first + 32 * n + col, my_first = max(0, pos - ctx) * a.G;  // the first row that sees it
      float part[2] = {0.0f, 0.0f};  // (in the order that the kernel of many rows has: a session's bits are its own, whatever bounds the call has)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        if (8 * g < R) {
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const int r = 8 * g + 4 * half + b;
            const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[4 * g + b], a.scale2, -lse2[4 * g + b]));
            part[b & 1] += r < R && r >= my_first ? w : 0.0f;
          }
        }
      }
      float sum = part[0] + part[1];
      sum += __shfl_xor(sum, 32);
      if (pos < v.len && half == 0) {
        if (p.page_ok(page[n])) put_weight(a, weights + pos, pos < ctx, before[n & 1], sum);
        else raise(a.status, PLC_ERR_INVALID);
      }
    }
  }
}

// More rows: four wavefronts keep 32 positions each in registers, and the rows come by in stages of 64 that they share, the next one on
// its way to LDS while one is worked on.
template <int DP_>
struct ManyShape {
  static constexpr int DP = DP_, kRows = 64, kSpan = kSpanOfGroup;
  static constexpr int kStage = kRows * DP * 2, kPerRow = DP / 8, kLoads = kRows * kPerRow / kBlock, kApart = kBlock / kPerRow;
  static constexpr size_t kLds = 2 * (size_t)(kStage + kRows * 4);
};

// Four wavefronts a SIMD, though at 128 components 8 to 10 registers are kept in scratch for it, outside of the loops: 8 sessions, 8 heads of 4, 512
// nodes after 8192 positions 334 us, with three 340; 5 sessions of up to 27 nodes and 4095 positions 12.0 and 12.6; as good as the same: one session of
// 512 nodes after 8192 (61 and 60.5 us), 2048 after 8192 (222), 16 sessions, 8 heads of 8, 16 nodes after 3000 (30.7).
template <class T, int DP, bool kExact>
__global__ __launch_bounds__(kBlock, DP <= 128 ? 4 : 2) void weigh_many_kernel(WeighArgs a) {
  using Shape = ManyShape<DP>;
  constexpr int KS = DP / 16, kRows = Shape::kRows, kSpan = Shape::kSpan, kStage = Shape::kStage, kLoads = Shape::kLoads,
                kApart = Shape::kApart, kPerRow = Shape::kPerRow;
  // two stages, then [2][kRows] of the rows' log-sum-exp.  (Through pointers to LDS: the compiler takes others for readers of what
  // the loads in flight write, and would wait for those.)
  extern __shared__ __attribute__((aligned(1024))) char weigh_lds[];
  lds_char *const lds = (lds_char *)weigh_lds;
  const PoolView &p = a.p;
  const int pair = (int)(blockIdx.x % (uint32_t)a.pairs), s = pair / p.H, h = pair - s * p.H;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, col = lane & 31;
  const SessionView v = session_of(a, s, pair % p.H == 0 && blockIdx.x < (uint32_t)a.pairs);
  if (!v.ok) return;
  const int32_t ctx = v.len - v.t;
  const int32_t *const table = p.table + (int64_t)s * p.M;
  const uint16_t *const keys = p.k + a.layer * p.layer_s + h * p.head_s + 8 * half;
  float *const weights = a.w.w + s * a.w.sess_s + a.layer * a.w.layer_s + h * a.w.head_s;
  const int32_t row_mask = (1 << p.shift) - 1;
  const uint16_t *const queries = a.q + v.n0 * a.q_node + (int64_t)h * a.G * a.q_head;
  const float *const lse = a.lse + (int64_t)v.n0 * (p.H * a.G) + h * a.G;

  if (!kExact) {  // pieces behind the last component are never loaded: zeros
    for (int i = threadIdx.x * 16; i < 2 * kStage; i += kBlock * 16) *reinterpret_cast<uint4 *>(weigh_lds + i) = make_uint4(0u, 0u, 0u, 0u);
    __syncthreads();
  }
  // A stage is `nodes` whole nodes, or where a node has more heads than a stage has rows `heads` of one: its row r is node r / heads, head
  // r % heads, at a distance from the stage's first that stays, so that the way from stage to stage is a scalar.  Rows behind
  // those are filled with one of them, and weigh nothing: their log-sum-exp is infinite.
  const int32_t parts = (a.G + kRows - 1) / kRows, heads = (a.G + parts - 1) / parts, nodes = max(1, kRows / a.G);
  const int32_t stages = (v.t + nodes - 1) / nodes * parts;
  struct Stage {
    int32_t node0, head0;
  };
  const auto begin_of = [&](int32_t stage) {
    if (parts == 1) return Stage{stage * nodes, 0};
    return Stage{stage / parts, stage % parts * heads};
  };
  int32_t my_node[kLoads], my_head[kLoads];
  int64_t my_at[kLoads];
#pragma unroll
  for (int j = 0; j < kLoads; ++j) {
    const int row = (int)threadIdx.x / kPerRow + j * kApart, c = ((int)threadIdx.x % kPerRow) ^ turn<DP>(row), r = min(row, nodes * heads - 1);
    my_node[j] = r / heads, my_head[j] = r - my_node[j] * heads;
    my_at[j] = my_node[j] * a.q_node + my_head[j] * a.q_head + c * 8;
  }
  const int32_t lse_row = min((int)threadIdx.x, nodes * heads - 1), lse_node = lse_row / heads, lse_head = lse_row - lse_node * heads;
  const int64_t lse_at = (int64_t)lse_node * (p.H * a.G) + lse_head;
  int q_at[KS];  // of a stage: this lane's fragments (the turns of 32 rows repeat)
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) q_at[ks] = place<DP>(col, 2 * ks + half);
  float next_lse = 0.0f;
  const auto request = [&](Stage st, int buf) {
    const bool full = st.node0 + nodes <= v.t && st.head0 + heads <= a.G;
    const uint16_t *const base = queries + st.node0 * a.q_node + st.head0 * a.q_head;
    // (every lane loads one, and first: a wait for it must not be one for the stage)
    int64_t at_lse = lse_at;
    if (!full) at_lse = (int64_t)min(lse_node, v.t - 1 - st.node0) * (p.H * a.G) + min(lse_head, a.G - 1 - st.head0);
    next_lse = lse[(int64_t)st.node0 * (p.H * a.G) + st.head0 + at_lse];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int row = (int)threadIdx.x / kPerRow + j * kApart, c = ((int)threadIdx.x % kPerRow) ^ turn<DP>(row);
      int64_t at = my_at[j];
      if (!full) at = min(my_node[j], v.t - 1 - st.node0) * a.q_node + min(my_head[j], a.G - 1 - st.head0) * a.q_head + c * 8;
#if defined(__HIP_DEVICE_COMPILE__)  // the host pass of the compiler does not know the device's load-to-LDS builtin
      if (kExact || c < p.d8) __builtin_amdgcn_global_load_lds(base + at, lds + buf * kStage + (j * kBlock + wave * 64) * 16, 16, 0, 0);
#else
      (void)at, (void)c, (void)base, (void)lds, (void)buf;
#endif
    }
  };

  const int32_t step = (int32_t)(gridDim.x / (uint32_t)a.pairs);
  for (int32_t chunk = (int32_t)(blockIdx.x / (uint32_t)a.pairs); (int64_t)chunk * kSpan < v.len; chunk += step) {
    const int32_t first = chunk * kSpan + wave * 32, pos = first + col;
    // nodes before that at the workgroup's first position see none of them
    int32_t stage = max(0, chunk * kSpan - ctx) / nodes * parts;
    Stage here = begin_of(stage);
    request(here, 0);
    short8v kf[KS];
    bool page_ok;
    {
      const int32_t at = min(pos, v.len - 1), page = table[at >> p.shift];
      page_ok = p.page_ok(page);
      const uint16_t *const k = keys + (page_ok ? page : 0) * p.page_s + (at & row_mask) * p.row_s;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        kf[ks] = short8v{};
        if (kExact || 16 * ks + 8 * half < 8 * p.d8) kf[ks] = *reinterpret_cast<const short8v *>(k + 16 * ks);
      }
    }
    // K has come before the loop begins: waited for inside it, it would take the loads under way along
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(kf[ks]));
    float sum = 0.0f;
    for (int buf = 0; stage < stages; ++stage, buf ^= 1) {
      // rows of this stage that are some, and those in front that do not see all of the wavefront's positions
      const int32_t node0 = here.node0, some = min(nodes, v.t - node0) * min(heads, a.G - here.head0);
      const int32_t blind = max(0, first + 31 - ctx - node0) * heads;
      lds_char *const stage_lse = lds + 2 * kStage + buf * kRows * 4;
      if (threadIdx.x < kRows) *(lds_float *)(stage_lse + 4 * threadIdx.x) = (int)threadIdx.x < some ? next_lse * kLog2e : __builtin_inff();
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (the compiler does not wait for loads to LDS at a barrier)
      __syncthreads();  // this stage has come, and everybody is done with the one before
      here = begin_of(stage + 1);
      if (stage + 1 < stages) request(here, buf ^ 1);
#pragma unroll
      for (int m = 0; m < kRows / 32; ++m) {
        if (32 * m >= some) break;
        float16v sc;
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = 0.0f;
        // Q's fragments four products ahead; fences keep the order
        short8v qf[2][4];
        const auto read_q = [&](int g) {
#pragma unroll
          for (int ks = 4 * g; ks < 4 * g + 4; ++ks)
            qf[g & 1][ks & 3] = *(const __attribute__((address_space(3))) short8v *)(lds + buf * kStage + 32 * m * (DP * 2) + q_at[ks]);
        };
        read_q(0);
#pragma unroll
        for (int g = 0; g < KS / 4; ++g) {
          if (g + 1 < KS / 4) read_q(g + 1);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int ks = 4 * g; ks < 4 * g + 4; ++ks) sc = mfma<T>(qf[g & 1][ks & 3], kf[ks], sc);
          __builtin_amdgcn_sched_barrier(0);
        }
        float lse2[16];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float4v x = *(const __attribute__((address_space(3))) float4v *)(stage_lse + 4 * (32 * m + 8 * g + 4 * half));
#pragma unroll
          for (int b = 0; b < 4; ++b) lse2[4 * g + b] = x[b];
        }
        float part[2] = {0.0f, 0.0f};  // a tile's rows by themselves first: a long sum loses less
        if (blind <= 32 * m) {
#pragma unroll
          for (int i = 0; i < 16; ++i) part[i & 1] += __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i], a.scale2, -lse2[i]));
        } else {
          // a bit for each row that is one and sees this lane's position: from `lo` on, below `hi`
          const int lo = min(max(max(0, pos - ctx - node0) * heads - 32 * m, 0), 32), hi = min(some - 32 * m, 32);
          const uint32_t sees = (uint32_t)(((1ull << hi) - 1) & ~((1ull << lo) - 1)) >> (4 * half);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i], a.scale2, -lse2[i]));
            part[i & 1] += sees >> (8 * (i >> 2) + (i & 3)) & 1u ? w : 0.0f;
          }
        }
        sum += part[0] + part[1];
      }
    }
    sum += __shfl_xor(sum, 32);
    if (pos < v.len && half == 0) {
      if (page_ok) put_weight(a, weights + pos, pos < ctx, a.decay != 0.0f ? weights[pos] : 0.0f, sum);
      else raise(a.status, PLC_ERR_INVALID);
    }
    __syncthreads();  // the next chunk's first stage goes where others may still read
  }
}

int64_t groups_of(const WeighArgs &a, int64_t span) {
  const int64_t chunks = (a.max_len + span - 1) / span, most = (kMostGroups + a.pairs - 1) / a.pairs;
  return a.pairs * (chunks < most ? chunks : most);
}

template <class T, int DP, int kTiles>
void launch_few(const WeighArgs &a, hipStream_t st) {
  hipLaunchKernelGGL((weigh_few_kernel<T, DP, kTiles>), dim3((unsigned)groups_of(a, kTiles * kSpanOfGroup)), dim3(kBlock), 0, st, a);
}

template <class T, int DP, bool kExact>
void launch_many(const WeighArgs &a, hipStream_t st) {
  constexpr size_t lds = ManyShape<DP>::kLds;
  static std::atomic<uint64_t> told{0};
  allow_lds(&weigh_many_kernel<T, DP, kExact>, lds, &told);
  hipLaunchKernelGGL((weigh_many_kernel<T, DP, kExact>), dim3((unsigned)groups_of(a, kSpanOfGroup)), dim3(kBlock), lds, st, a);
}

// Four tiles a wavefront where there are that many: 64 sessions, 8 heads of 4, one token after up to 4096 positions 78 us, with one tile 93, two 85,
// eight 79; 20 sessions of 24,323 positions 214, 244, 232 and 212.
template <class T, int DP>
void weigh(const WeighArgs &a, hipStream_t st) {
  const int64_t tiles = (int64_t)a.pairs * ((a.max_len + 31) / 32);
  if ((int64_t)a.max_nodes * a.G > 32) {
    if (8 * a.p.d8 == DP) launch_many<T, DP, true>(a, st);
    else launch_many<T, DP, false>(a, st);
  } else if (tiles >= 64 * kComputeUnits) {
    launch_few<T, DP, DP <= 128 ? 4 : 2>(a, st);
  } else {
    launch_few<T, DP, 1>(a, st);
  }
}

template <class T>
int weigh(const WeighArgs &a, hipStream_t st) {
  const int d = 8 * a.p.d8;
  if (d <= 64) weigh<T, 64>(a, st);
  else if (d <= 128) weigh<T, 128>(a, st);
  else weigh<T, 256>(a, st);
  return launch_status();
}

}  // namespace
}  // namespace plc

using namespace plc;

extern "C" int plc_attend_weights(const plc_pages *pages, int32_t layer, int32_t type, const void *q, const int64_t *q_stride,
                                  int32_t G, int64_t N, const int32_t *off, int32_t max_nodes, int32_t max_len, float scale,
                                  const float *lse, float decay, const plc_weights *weights, uint32_t *status, void *stream) {
  if (!pages_valid(pages) || pages->d > 256 || layer < 0 || layer >= pages->L || (type != PLC_FP16 && type != PLC_BF16) ||
      !q_stride || q_stride[0] < 0 || q_stride[0] % 8 || q_stride[1] < 0 || q_stride[1] % 8 || G < 1 || N < 0 || N > INT32_MAX ||
      (int64_t)pages->H * G > 65536 || max_nodes < 1 || (int64_t)max_nodes * G > INT32_MAX / 256 || max_len < 1 ||
      !aligned(off, 4) || !(scale > 0.0f) || !(scale * kLog2e < __builtin_inff()) || !(decay >= 0.0f) || !(decay <= 1.0f) ||
      !weights_valid(pages, weights) || !status)
    return PLC_ERR_INVALID;
  if ((int64_t)pages->S * pages->H >= 1 << 23) return PLC_ERR_INVALID;  // (lanes of a launch < 2^32)
  if (N == 0) return PLC_OK;
  if (!aligned(q, 16) || !aligned(lse, 4)) return PLC_ERR_INVALID;
  WeighArgs a = {};
  a.p = pool_view(pages);
  a.w = weights_view(weights);
  a.layer = layer, a.G = G, a.max_nodes = max_nodes;
  const int64_t most = (int64_t)pages->M * pages->B;  // (no session has more, whatever the caller bounds it by)
  a.max_len = max_len < most ? max_len : (int32_t)most;
  a.N = N, a.q_node = q_stride[0], a.q_head = q_stride[1];
  a.q = static_cast<const uint16_t *>(q), a.lse = lse, a.off = off;
  a.scale2 = scale * kLog2e, a.decay = decay;
  a.pairs = pages->S * pages->H;
  a.status = status;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return type == PLC_FP16 ? weigh<_Float16>(a, st) : weigh<__bf16>(a, st);
}
