// What positions receive of attention: for each position of a session and KV head the sum of the weights that the rows of a call
// give it, from the rows' log-sum-exp; see include/plc.h for the formula.
//
// A wavefront keeps 32 positions in its columns and takes the rows 32 at a time:
//   S [rows, positions] = Q [rows, d] * K^T [d, positions]       v_mfma 32x32x16
// so that a lane's 16 accumulators are rows of one position: their weights exp2(scale' S - lse') are added up in the lane itself,
// row by row in a fixed order, and only the two halves of a position meet at the end.  K is read once, straight into the operand's
// registers (a lane holds 16 bytes of its position's row at a time); nothing of the scores leaves the registers.
#include <type_traits>

#include "plc_device.h"
#include "plc_paged.h"

namespace plc {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short short8v __attribute__((ext_vector_type(8)));
typedef float float16v __attribute__((ext_vector_type(16)));

typedef __attribute__((address_space(3))) char lds_char;

constexpr float kLog2e = 1.44269504088896340736f;
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
      float sum = 0.0f;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        if (8 * g < R) {
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const int r = 8 * g + 4 * half + b;
            const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[4 * g + b], a.scale2, -lse2[4 * g + b]));
            sum += r < R && r >= my_first ? w : 0.0f;
          }
        }
      }
      sum += __shfl_xor(sum, 32);
      if (pos < v.len && half == 0) {
        if (p.page_ok(page[n])) put_weight(a, weights + pos, pos < ctx, before[n & 1], sum);
        else raise(a.status, PLC_ERR_INVALID);
      }
    }
  }
}

// LDS layout of a stage: kStageRows rows of DP components; the 16-byte piece c of row r stands in place c ^ turn(r), so that 16
// consecutive rows' same piece spread over all banks.
constexpr int kStageRows = 64;
template <int DP>
__device__ __forceinline__ int turn(int r) {
  return DP == 64 ? r >> 1 & 7 : r & 15;
}
template <int DP>
__device__ __forceinline__ int place(int r, int c) {
  return r * (DP * 2) + ((c ^ turn<DP>(r)) << 4);
}

// More rows: the positions stay in registers, 32 NT for each of four wavefronts, and the rows come by in stages of 64 that all of
// them share.
template <class T, int DP, int NT, bool kExact>
__global__ __launch_bounds__(kBlock, DP <= 128 ? 2 : 1) void weigh_many_kernel(WeighArgs a) {
  constexpr int KS = DP / 16, kSpan = 32 * NT * (kBlock / 64), kStage = kStageRows * DP * 2;
  __shared__ __attribute__((aligned(1024))) char stages[2 * kStage];
  __shared__ __attribute__((aligned(16))) float lses[2][kStageRows];
  lds_char *const lds = (lds_char *)stages;
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
  const uint16_t *const queries = a.q + v.n0 * a.q_node + (int64_t)h * a.G * a.q_head;
  const float *const lse = a.lse + (int64_t)v.n0 * (p.H * a.G) + h * a.G;

  // this thread's pieces of a stage
  constexpr int kPerRow = DP / 8, kLoads = kStageRows * kPerRow / kBlock, kApart = kStageRows / kLoads;  // rows between its loads
  const int my_row = (int)threadIdx.x / kPerRow;
  if (!kExact) {  // pieces behind the last component are never loaded: zeros
    for (int i = threadIdx.x * 16; i < 2 * kStage; i += kBlock * 16) *reinterpret_cast<uint4 *>(stages + i) = make_uint4(0u, 0u, 0u, 0u);
    __syncthreads();
  }
  const auto request = [&](int32_t r0, int buf) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int row = my_row + j * kApart, c = ((int)threadIdx.x % kPerRow) ^ turn<DP>(row);
      const int32_t r = min(r0 + row, R - 1), node = r / a.G, g = r - node * a.G;
      const uint16_t *const from = queries + node * a.q_node + g * a.q_head + c * 8;
      lds_char *const to = lds + buf * kStage + (j * kBlock + wave * 64) * 16;
#if defined(__HIP_DEVICE_COMPILE__)  // the host pass of the compiler does not know the device's load-to-LDS builtin
      if (kExact || c < p.d8) __builtin_amdgcn_global_load_lds(from, to, 16, 0, 0);
#else
      (void)from, (void)to;
#endif
    }
  };
  const auto lse_of = [&](int32_t r0) {
    const int32_t r = min(r0 + ((int)threadIdx.x & (kStageRows - 1)), R - 1), node = r / a.G;
    return lse[(int64_t)node * (p.H * a.G) + r - node * a.G] * kLog2e;
  };

  const int32_t step = (int32_t)(gridDim.x / (uint32_t)a.pairs);
  for (int32_t chunk = (int32_t)(blockIdx.x / (uint32_t)a.pairs); (int64_t)chunk * kSpan < v.len; chunk += step) {
    const int32_t first = chunk * kSpan + wave * 32 * NT;
    // rows before those of the node at the workgroup's first position see none of them
    const int32_t row0 = max(0, chunk * kSpan - ctx) * a.G / kStageRows * kStageRows;
    request(row0, 0);
    float next_lse = lse_of(row0);
    short8v kf[NT][KS];
    bool page_ok[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int32_t at = min(first + 32 * n + col, v.len - 1), page = table[at >> p.shift];
      page_ok[n] = p.page_ok(page);
      const uint16_t *const k = keys + (page_ok[n] ? page : 0) * p.page_s + (at & row_mask) * p.row_s;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        kf[n][ks] = short8v{};
        if (kExact || 16 * ks + 8 * half < 8 * p.d8) kf[n][ks] = *reinterpret_cast<const short8v *>(k + 16 * ks);
      }
    }
    float sums[NT] = {};
    int buf = 0;
    for (int32_t r0 = row0; r0 < R; r0 += kStageRows, buf ^= 1) {
      if (threadIdx.x < kStageRows) lses[buf][threadIdx.x] = next_lse;
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (the compiler does not wait for loads to LDS at a barrier)
      __syncthreads();  // this stage has come, and everybody is done with the one before
      if (r0 + kStageRows < R) {
        request(r0 + kStageRows, buf ^ 1);
        next_lse = lse_of(r0 + kStageRows);
      }
#pragma unroll
      for (int m = 0; m < kStageRows / 32; ++m) {
        float16v sc[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 16; ++i) sc[n][i] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const short8v qf = *(const __attribute__((address_space(3))) short8v *)(lds + buf * kStage + place<DP>(32 * m + col, 2 * ks + half));
#pragma unroll
          for (int n = 0; n < NT; ++n) sc[n] = mfma<T>(qf, kf[n][ks], sc[n]);
        }
        float lse2[16];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float4 x = *reinterpret_cast<const float4 *>(&lses[buf][32 * m + 8 * g + 4 * half]);
          lse2[4 * g] = x.x, lse2[4 * g + 1] = x.y, lse2[4 * g + 2] = x.z, lse2[4 * g + 3] = x.w;
        }
        const int32_t r1 = r0 + 32 * m;
        // all of these rows are some, and see all of the wavefront's positions
        const bool whole = r1 + 32 <= R && (int64_t)(first + 32 * NT - 1 - ctx) * a.G <= r1;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float part[2] = {0.0f, 0.0f};  // a tile's rows by themselves first: a long sum loses less
          if (whole) {
#pragma unroll
            for (int i = 0; i < 16; ++i) part[i & 1] += __builtin_amdgcn_exp2f(__builtin_fmaf(sc[n][i], a.scale2, -lse2[i]));
          } else {
            const int64_t my_first = (int64_t)max(0, first + 32 * n + col - ctx) * a.G;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int32_t r = r1 + 8 * (i >> 2) + 4 * half + (i & 3);
              const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[n][i], a.scale2, -lse2[i]));
              part[i & 1] += r < R && r >= my_first ? w : 0.0f;
            }
          }
          sums[n] += part[0] + part[1];
        }
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float sum = sums[n] + __shfl_xor(sums[n], 32);
      const int32_t pos = first + 32 * n + col;
      if (pos < v.len && half == 0) {
        if (page_ok[n]) put_weight(a, weights + pos, pos < ctx, a.decay != 0.0f ? weights[pos] : 0.0f, sum);
        else raise(a.status, PLC_ERR_INVALID);
      }
    }
    __syncthreads();  // the next chunk's first stage goes where others may still read
  }
}

template <class K>
void launch_weigh(const K &kernel, WeighArgs a, int64_t span, hipStream_t st) {
  const int64_t chunks = (a.max_len + span - 1) / span, most = (kMostGroups + a.pairs - 1) / a.pairs;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(a.pairs * (chunks < most ? chunks : most))), dim3(kBlock), 0, st, a);
}

template <class T, int DP>
void weigh(const WeighArgs &a, hipStream_t st) {
  const int64_t tiles = (int64_t)a.pairs * ((a.max_len + 31) / 32);
  constexpr int kMany = DP <= 128 ? 4 : 2;
  if ((int64_t)a.max_nodes * a.G <= 32) {
    if (tiles >= 16 * 1024) launch_weigh(&weigh_few_kernel<T, DP, kMany>, a, 32 * 4 * kMany, st);
    else launch_weigh(&weigh_few_kernel<T, DP, 1>, a, 32 * 4, st);
    return;
  }
  const bool exact = 8 * a.p.d8 == DP;
  constexpr int NT = DP <= 128 ? 2 : 1;
  if (DP <= 128 && tiles >= 8 * 1024) {
    if (exact) launch_weigh(&weigh_many_kernel<T, DP, NT, true>, a, 128 * NT, st);
    else launch_weigh(&weigh_many_kernel<T, DP, NT, false>, a, 128 * NT, st);
  } else {
    if (exact) launch_weigh(&weigh_many_kernel<T, DP, 1, true>, a, 128, st);
    else launch_weigh(&weigh_many_kernel<T, DP, 1, false>, a, 128, st);
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
      !aligned(off, 4) || !(scale > 0.0f) || !(scale < __builtin_inff()) || !(decay >= 0.0f) || !(decay <= 1.0f) ||
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
