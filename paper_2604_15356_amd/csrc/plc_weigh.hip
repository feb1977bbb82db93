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

constexpr float kLog2e = 1.44269504088896340736f;

struct WeighArgs {
  PoolView p;
  WeightsView w;
  int32_t layer, G, max_nodes, max_len;
  int64_t N, q_node, q_head;
  const uint16_t *q;
  const float *lse;
  const int32_t *off;
  float scale2, decay;  // scale * log2(e)
  uint32_t *status;
};

template <class T>
__device__ __forceinline__ float16v mfma(short8v a, short8v b, float16v c) {
  if constexpr (std::is_same<T, _Float16>::value)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

template <class T, int DP>
__global__ __launch_bounds__(kBlock) void weigh_kernel(WeighArgs a) {
  constexpr int KS = DP / 16;
  const PoolView &p = a.p;
  const int s = (int)blockIdx.z, h = (int)blockIdx.y;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, col = lane & 31;
  const int32_t n0 = a.off[s], n1 = a.off[s + 1], len = p.lens[s];
  const int64_t t = (int64_t)n1 - n0;
  if (t == 0) return;
  if (t < 0 || n0 < 0 || n1 > a.N || t > a.max_nodes || len < t || len > a.max_len || len > ((int64_t)p.M << p.shift) || len > a.w.width) {
    if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) raise(a.status, PLC_ERR_INVALID);
    return;
  }
  const int32_t ctx = len - (int32_t)t, R = (int32_t)t * a.G;
  const int32_t first = ((int32_t)blockIdx.x * (kBlock / 64) + wave) * 32, pos = first + col;
  if (first >= len) return;
  const bool in = pos < len;

  short8v kf[KS];
  bool page_ok;
  {
    const int32_t at = min(pos, len - 1), page = p.table[(int64_t)s * p.M + (at >> p.shift)];
    page_ok = p.page_ok(page);
    if (!page_ok) raise(a.status, PLC_ERR_INVALID);
    const uint16_t *const k = p.k + (page_ok ? page : 0) * p.page_s + a.layer * p.layer_s + h * p.head_s +
                              (at & ((1 << p.shift) - 1)) * p.row_s + 8 * half;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      short8v v = {};
      if (16 * ks + 8 * half < 8 * p.d8) v = *reinterpret_cast<const short8v *>(k + 16 * ks);
      kf[ks] = v;
    }
  }
  float sum = 0.0f;
  const int32_t row0 = max(0, first - ctx) * a.G / 32 * 32;  // no row before it sees any of these positions
  const int32_t my_first = max(0, pos - ctx) * a.G;          // the first that sees this lane's
  for (int32_t r0 = row0; r0 < R; r0 += 32) {
    float16v sc;
#pragma unroll
    for (int i = 0; i < 16; ++i) sc[i] = 0.0f;
    {
      const int32_t r = min(r0 + col, R - 1);
      const uint16_t *const q = a.q + (n0 + r / a.G) * a.q_node + (h * a.G + r % a.G) * a.q_head + 8 * half;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        short8v v = {};
        if (16 * ks + 8 * half < 8 * p.d8) v = *reinterpret_cast<const short8v *>(q + 16 * ks);
        sc = mfma<T>(v, kf[ks], sc);
      }
    }
    float part = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int32_t r = r0 + 8 * (i >> 2) + 4 * half + (i & 3), rr = min(r, R - 1);
      const float lse = a.lse[(int64_t)(n0 + rr / a.G) * (p.H * a.G) + h * a.G + rr % a.G] * kLog2e;
      const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i], a.scale2, -lse));
      part += r < R && r >= my_first ? w : 0.0f;
    }
    sum += part;
  }
  sum += __shfl_xor(sum, 32);
  if (half == 0 && in && page_ok) {
    float *const w = a.w.w + s * a.w.sess_s + a.layer * a.w.layer_s + h * a.w.head_s + pos;
    *w = pos < ctx && a.decay != 0.0f ? __builtin_fmaf(a.decay, *w, sum) : sum;
  }
}

template <class T>
int weigh(const WeighArgs &a, hipStream_t st) {
  const dim3 grid((unsigned)(((int64_t)a.max_len + 127) / 128), (unsigned)a.p.H, (unsigned)a.p.S);
  const int d = 8 * a.p.d8;
  const auto kernel = d <= 64 ? &weigh_kernel<T, 64> : d <= 128 ? &weigh_kernel<T, 128> : &weigh_kernel<T, 256>;
  hipLaunchKernelGGL(kernel, grid, dim3(kBlock), 0, st, a);
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
  a.status = status;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return type == PLC_FP16 ? weigh<_Float16>(a, st) : weigh<__bf16>(a, st);
}
