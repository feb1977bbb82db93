// Rotary positions: rows of a buffer turned to their positions, and the store into pages that turns keys on their way and the
// queries beside them; see include/plc.h for the formula.
//
// A lane owns 16 components of a row (8 pairs), and takes them through many heads: the cosines and sines of its pairs are
// worked out once, by itself, and stay in registers.  With halves that are whole pieces of 16 bytes its components are one piece of
// each half, interleaved they are two pieces side by side; halves of other widths go by what they are aligned to, 8, 4 or 2 bytes.
//
// The angle in turns, times 2^64, is a whole number; times the position it wraps around exactly as the angle does, so that
// its upper 32 bits are the fraction of a turn to 2^-32 for any position, where fp32 products of position and frequency are off by
// 0.06 rad at a million.  Cosine and sine of what is left within an eighth of a turn are sums of their power series.
//
// What bounds it: HBM where there is much (4096 rows of 32 layers and 8 heads, 128 components, 1.07 GB in and out, 197 us, 5.4 TB/s; the
// store that does not rotate 188); in the caches the angles, some 20 instructions for each of a thread's 8 pairs (2048 tokens, 50 MB,
// 13.5 us); for few rows the host's time (a token's 12 heads: 5.7 us of one launch after the other).
#include <cmath>
#include <type_traits>

#include "plc_device.h"
#include "plc_paged.h"

namespace plc {
namespace {

struct Turning {
  const uint64_t *turns;
  int32_t r, interleaved;
  float magnitude, sign;  // sign -1: back
};

struct RotateArgs {
  Turning by;
  PoolView p;
  RowsView r;
  const int32_t *off, *base, *rel;  // of a store; without, rel holds the rows' positions
  int32_t heads, d8;                // query heads
  const uint16_t *q;
  uint16_t *q_out;
  int64_t q_node, q_head, out_node, out_head;
  int32_t lanes, block_rows, slots;  // lanes of a row, rows of a workgroup, heads side by side in it
  uint32_t *status;
};

// cos and sin of 2 pi f / 2^32.
__device__ __forceinline__ void turn_by(uint32_t f, float *c, float *s) {
  const uint32_t quarter = (f + 0x20000000u) >> 30;
  const float t = (float)(int32_t)(f - (quarter << 30)) * 1.4629180792671596e-9f;  // 2 pi / 2^32: |t| <= pi / 4
  const float z = t * t;
  // the power series up to t^9 and t^10; what follows is below 2^-29 and 2^-33
  float sn = __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6);
  sn = __builtin_fmaf(t * z, sn, t);
  float cs = __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, -1.0f / 3628800, 1.0f / 40320), -1.0f / 720), 1.0f / 24), -0.5f);
  cs = __builtin_fmaf(z, cs, 1.0f);
  const float a = quarter & 1 ? sn : cs, b = quarter & 1 ? cs : sn;
  *c = (quarter + 1) & 2 ? -a : a;
  *s = quarter & 2 ? -b : b;
}

// How a lane's components lie in a row: two runs of up to 8, and the pairs that they make (none: they pass).
struct Lane {
  int32_t at[2], n[2], first, count;
};

// A run of n components, in pieces of kWide, which they are a multiple of and aligned as; past the caches (kStream).
template <int kWide, bool kStream>
__device__ __forceinline__ uint4 get_run(const uint16_t *from, int32_t n) {
  if constexpr (kWide == 8) {
    if (n == 0) return make_uint4(0u, 0u, 0u, 0u);
    return kStream ? load16_stream(from) : *reinterpret_cast<const uint4 *>(from);
  } else {
    typedef uint16_t Piece __attribute__((ext_vector_type(kWide)));
    typedef uint16_t Eight __attribute__((ext_vector_type(8)));
    Eight v = {};
#pragma unroll
    for (int c = 0; c < 8; c += kWide)
      if (c < n) {
        const Piece x = *reinterpret_cast<const Piece *>(from + c);
#pragma unroll
        for (int e = 0; e < kWide; ++e) v[c + e] = x[e];
      }
    return __builtin_bit_cast(uint4, v);
  }
}
template <int kWide, bool kStream>
__device__ __forceinline__ void put_run(uint16_t *to, int32_t n, uint4 run) {
  if constexpr (kWide == 8) {
    if (n == 0) return;
    if (kStream) store16_stream(to, run);
    else *reinterpret_cast<uint4 *>(to) = run;
  } else {
    typedef uint16_t Piece __attribute__((ext_vector_type(kWide)));
    typedef uint16_t Eight __attribute__((ext_vector_type(8)));
    const Eight v = __builtin_bit_cast(Eight, run);
#pragma unroll
    for (int c = 0; c < 8; c += kWide)
      if (c < n) {
        Piece x;
#pragma unroll
        for (int e = 0; e < kWide; ++e) x[e] = v[c + e];
        *reinterpret_cast<Piece *>(to + c) = x;
      }
  }
}

// kWide: components that lie aligned together, in halves too (8: interleaved, or halves of whole 16-byte pieces).  kStream: stores past the
// caches, and with 2 loads too.
template <class T, bool kStore, int kWide, int kStream>
__global__ __launch_bounds__(kBlock) void rotate_kernel(RotateArgs a) {
  extern __shared__ int64_t rotate_lds[];  // of a store: [block_rows] in the pool, in the buffer, position; then off i32 [S + 1]
  const PoolView &p = a.p;
  const int64_t x0 = (int64_t)blockIdx.x * a.block_rows;
  if constexpr (kStore) {
    int64_t *const in_pool = rotate_lds, *const in_buf = in_pool + a.block_rows, *const positions = in_buf + a.block_rows;
    int32_t *const o = reinterpret_cast<int32_t *>(positions + a.block_rows);
    for (int32_t s = threadIdx.x; s <= p.S; s += kBlock) o[s] = a.off[s];
    __syncthreads();
    if (blockIdx.x == 0 && blockIdx.y == 0) check_offsets<kBlock>(p, a.r, o, a.status);
    for (int32_t b = threadIdx.x; b < a.block_rows; b += kBlock) {
      const int64_t x = x0 + b;
      const RowPlace at = place_row<true>(p, a.r, o, x, a.status);
      int64_t pos = 0;
      if (at.pool >= 0) {
        pos = a.base ? a.base[at.s] : p.lens[at.s] - (o[at.s + 1] - o[at.s]);
        pos += a.rel ? a.rel[x] : at.i;
      }
      in_pool[b] = at.pool;
      in_buf[b] = at.buf;
      positions[b] = pos;
    }
    __syncthreads();
  }
  const int32_t unit = (int32_t)threadIdx.x / a.lanes, j = (int32_t)threadIdx.x - unit * a.lanes;
  const int32_t slot = unit / a.block_rows, b = unit - slot * a.block_rows;
  if (slot >= a.slots) return;
  const int64_t x = x0 + b;
  int64_t pool = 0, buf = 0, pos;
  if constexpr (kStore) {
    pool = rotate_lds[b], buf = rotate_lds[a.block_rows + b], pos = rotate_lds[2 * a.block_rows + b];
    if (pool < 0) return;
    pool += a.r.layer * p.layer_s;
  } else {
    if (x >= a.r.rows) return;
    pos = a.rel[x];
  }

  const int32_t half = a.by.r / 2, d = 8 * a.d8, turning = (half + 7) / 8;  // lanes with pairs
  Lane lane;
  if (kWide == 8 && a.by.interleaved) {
    lane = {{16 * j, 16 * j + 8}, {8, min(8, d - 16 * j - 8)}, 8 * j, max(0, min(8, half - 8 * j))};
  } else if (j < turning) {
    const int32_t n = min(8, half - 8 * j);
    lane = {{8 * j, 8 * j + half}, {n, n}, 8 * j, n};
  } else {
    const int32_t e = a.by.r + 16 * (j - turning);
    lane = {{e, e + 8}, {min(8, d - e), max(0, min(8, d - e - 8))}, 0, 0};
  }
  float cs[8], sn[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    cs[i] = 1.0f, sn[i] = 0.0f;
    if (i < lane.count) {
      turn_by((uint32_t)(((uint64_t)pos * a.by.turns[lane.first + i]) >> 32), &cs[i], &sn[i]);
      cs[i] *= a.by.magnitude, sn[i] *= a.by.sign * a.by.magnitude;
    }
  }

  const int32_t keys = kStore ? a.r.layers * p.H : 0, all = 2 * keys + a.heads;
  const auto place = [&](int32_t e, const uint16_t **from, uint16_t **to) {
    if (kStore && e < 2 * keys) {
      const int32_t lh = e < keys ? e : e - keys, l = lh / p.H, h = lh - l * p.H;
      *from = (e < keys ? a.r.k : a.r.v) + buf + l * a.r.layer_s + h * a.r.head_s;
      *to = (e < keys ? p.k : p.v) + pool + l * p.layer_s + h * p.head_s;
    } else {
      const int32_t h = e - 2 * keys;
      *from = a.q + x * a.q_node + h * a.q_head;
      *to = a.q_out + x * a.out_node + h * a.out_head;
    }
  };
  const auto turned = [&](int32_t e) { return e < keys || e >= 2 * keys; };
  const int32_t e0 = (int32_t)blockIdx.y * a.slots + slot, step = (int32_t)gridDim.y * a.slots;

  typedef T T8 __attribute__((ext_vector_type(8)));
  constexpr int kBatch = 4;
  for (int32_t e = e0; e < all; e += kBatch * step) {
    uint4 in[kBatch][2];
    uint16_t *to[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const uint16_t *from;
      place(min(e + u * step, all - 1), &from, &to[u]);
      in[u][0] = get_run<kWide, kStream == 2>(from + lane.at[0], lane.n[0]);
      in[u][1] = get_run<kWide, kStream == 2>(from + lane.at[1], lane.n[1]);
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int32_t mine = e + u * step;
      if (mine >= all) break;
      if (turned(mine) && lane.count > 0) {
        const T8 v0 = __builtin_bit_cast(T8, in[u][0]), v1 = __builtin_bit_cast(T8, in[u][1]);
        T8 w0 = v0, w1 = v1;
        if (kWide == 8 && a.by.interleaved) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float xa = (float)v0[2 * i], ya = (float)v0[2 * i + 1], xb = (float)v1[2 * i], yb = (float)v1[2 * i + 1];
            if (i < lane.count) {
              w0[2 * i] = (T)__builtin_fmaf(xa, cs[i], -(ya * sn[i]));
              w0[2 * i + 1] = (T)__builtin_fmaf(ya, cs[i], xa * sn[i]);
            }
            if (i + 4 < lane.count) {
              w1[2 * i] = (T)__builtin_fmaf(xb, cs[i + 4], -(yb * sn[i + 4]));
              w1[2 * i + 1] = (T)__builtin_fmaf(yb, cs[i + 4], xb * sn[i + 4]);
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float xa = (float)v0[i], ya = (float)v1[i];
            w0[i] = (T)__builtin_fmaf(xa, cs[i], -(ya * sn[i]));
            w1[i] = (T)__builtin_fmaf(ya, cs[i], xa * sn[i]);
          }
        }
        in[u][0] = __builtin_bit_cast(uint4, w0), in[u][1] = __builtin_bit_cast(uint4, w1);
      }
      put_run<kWide, kStream != 0>(to[u] + lane.at[0], lane.n[0], in[u][0]);
      put_run<kWide, kStream != 0>(to[u] + lane.at[1], lane.n[1], in[u][1]);
    }
  }
}

// ---- host side ------------------------------------------------------------------------------------------------------------

constexpr int64_t kCached = (int64_t)96 << 20;         // bytes moved, in and out, beyond which stores go past the caches
constexpr int64_t kLoadedCached = (int64_t)512 << 20;  // beyond which loads do too: what is read may still lie in the last-level cache

bool rotary_valid(const plc_rotary *rot, int32_t d) {
  return rot && aligned(rot->turns, 8) && rot->r >= 2 && rot->r % 2 == 0 && rot->r <= d && d >= 8 && d % 8 == 0 && d <= 2048 &&
         (rot->interleaved == 0 || rot->interleaved == 1) && rot->magnitude > 0.0f && rot->magnitude < __builtin_inff() &&
         1.0f / rot->magnitude > 0.0f && 1.0f / rot->magnitude < __builtin_inff();
}

bool strides_ok(const int64_t *stride) {
  return stride && stride[0] >= 0 && stride[0] % 8 == 0 && stride[1] >= 0 && stride[1] % 8 == 0;
}

// (Rows that are written may not lie on each other.)
bool strides_out_ok(const int64_t *stride, int64_t rows, int64_t heads, int32_t d) {
  return strides_ok(stride) && lie_apart<2>({rows, heads}, stride, d);
}

// Four heads to a thread, which its angles are for, while there are two workgroups for each compute unit, else fewer: 2048 tokens with 48
// heads of keys, values and queries 13.5 us, with up to 8 the same, with one or two at a time 17; 4096 rows of 512 heads 197 us, of
// up to 8 heads 204, of 16 216.
template <class T, bool kStore, int kWide>
int launch_rotate(RotateArgs a, int64_t rows, int64_t heads, hipStream_t st) {
  const int32_t half = a.by.r / 2, d = 8 * a.d8;
  a.lanes = kWide == 8 ? (d + 15) / 16 : (half + 7) / 8 + (d - a.by.r + 15) / 16;
  const int32_t units = kBlock / a.lanes;
  a.block_rows = units;
  while (a.block_rows > 1 && a.block_rows / 2 >= rows) a.block_rows /= 2;
  a.slots = units / a.block_rows;
  const int64_t bx = (rows + a.block_rows - 1) / a.block_rows;
  if (bx >= 1 << 24) return PLC_ERR_INVALID;  // (lanes of a launch < 2^32)
  int64_t each = 4, by;  // heads of a thread
  while (true) {
    by = (heads + each * a.slots - 1) / (each * a.slots);
    if (each == 1 || bx * by >= 2 * kComputeUnits) break;
    each /= 2;
  }
  by = by > 65535 ? 65535 : by;
  const double bytes = (double)rows * heads * d * 4;
  const auto kernel = kWide != 8 || bytes <= (double)kCached ? &rotate_kernel<T, kStore, kWide, 0>
                      : bytes <= (double)kLoadedCached       ? &rotate_kernel<T, kStore, kWide, kWide == 8 ? 1 : 0>
                                                             : &rotate_kernel<T, kStore, kWide, kWide == 8 ? 2 : 0>;
  const size_t lds = kStore ? 24 * (size_t)a.block_rows + 4 * (size_t)(a.p.S + 1) : 0;
  hipLaunchKernelGGL(kernel, dim3((unsigned)bx, (unsigned)by), dim3(kBlock), lds, st, a);
  return launch_status();
}

template <class T, bool kStore>
int rotate(const RotateArgs &a, int64_t rows, int64_t heads, hipStream_t st) {
  const int32_t half = a.by.r / 2;
  if (a.by.interleaved || half % 8 == 0) return launch_rotate<T, kStore, 8>(a, rows, heads, st);
  if (half % 4 == 0) return launch_rotate<T, kStore, 4>(a, rows, heads, st);
  if (half % 2 == 0) return launch_rotate<T, kStore, 2>(a, rows, heads, st);
  return launch_rotate<T, kStore, 1>(a, rows, heads, st);
}

template <bool kStore>
int rotate(const RotateArgs &a, int32_t type, int64_t rows, int64_t heads, hipStream_t st) {
  return type == PLC_FP16 ? rotate<_Float16, kStore>(a, rows, heads, st) : rotate<__bf16, kStore>(a, rows, heads, st);
}

constexpr long double kTwoPi = 6.283185307179586476925286766559005768L;

}  // namespace
}  // namespace plc

using namespace plc;

extern "C" int plc_rotary_frequencies(const plc_rotary_spec *spec, double *theta) {
  if (!spec || !theta || spec->r < 2 || spec->r % 2 || spec->r > 2048 || spec->scaling < PLC_ROTARY_PLAIN ||
      spec->scaling > PLC_ROTARY_RAMP || !(spec->base > 0.0) || !std::isfinite(spec->base))
    return PLC_ERR_INVALID;
  const int32_t kind = spec->scaling, r = spec->r;
  if (kind != PLC_ROTARY_PLAIN && (!(spec->factor > 0.0) || !std::isfinite(spec->factor))) return PLC_ERR_INVALID;
  const bool by_turns = kind == PLC_ROTARY_PARTS || kind == PLC_ROTARY_RAMP;
  if (by_turns && (!(spec->low > 0.0) || !(spec->high > spec->low) || !std::isfinite(spec->high) || spec->trained < 1))
    return PLC_ERR_INVALID;
  if (kind == PLC_ROTARY_RAMP && !(spec->base > 1.0)) return PLC_ERR_INVALID;
  long double base = spec->base;
  if (kind == PLC_ROTARY_STRETCHED && r > 2) base *= powl(spec->factor, (long double)r / (r - 2));
  long double ramp0 = 0.0L, ramp1 = 0.0L;
  if (kind == PLC_ROTARY_RAMP) {
    const auto at = [&](double turns) { return r * logl(spec->trained / (kTwoPi * turns)) / (2.0L * logl(base)); };
    ramp0 = fmaxl(floorl(at(spec->high)), 0.0L), ramp1 = fminl(ceill(at(spec->low)), r - 1.0L);
  }
  for (int32_t i = 0; i < r / 2; ++i) {
    long double t = powl(base, -2.0L * i / r);
    if (kind == PLC_ROTARY_LINEAR) {
      t /= spec->factor;
    } else if (by_turns) {
      long double g = kind == PLC_ROTARY_PARTS ? (spec->trained * t / kTwoPi - spec->low) / ((long double)spec->high - spec->low)
                                               : 1.0L - (i - ramp0) / fmaxl(ramp1 - ramp0, 0.001L);
      g = fminl(fmaxl(g, 0.0L), 1.0L);
      t = g * t + (1.0L - g) * t / spec->factor;
    }
    theta[i] = (double)t;
  }
  return PLC_OK;
}

extern "C" int plc_rotary_turns(const double *theta, int32_t pairs, uint64_t *turns) {
  if (!theta || !turns || pairs < 1) return PLC_ERR_INVALID;
  for (int32_t i = 0; i < pairs; ++i)
    if (!std::isfinite(theta[i])) return PLC_ERR_INVALID;
  for (int32_t i = 0; i < pairs; ++i) {
    long double t = theta[i] / kTwoPi;
    t = rintl((t - floorl(t)) * 0x1p64L);
    turns[i] = t >= 0x1p64L ? 0 : (uint64_t)t;
  }
  return PLC_OK;
}

extern "C" int plc_rotate(const plc_rotary *rotary, int32_t type, const void *x, const int64_t *x_stride, int64_t rows,
                          int32_t heads, int32_t d, const int32_t *positions, int32_t inverse, void *out,
                          const int64_t *out_stride, void *stream) {
  if (!rotary_valid(rotary, d) || (type != PLC_FP16 && type != PLC_BF16) || !strides_ok(x_stride) || !strides_out_ok(out_stride, rows, heads, d) ||
      rows < 0 || rows > INT32_MAX || heads < 1 || (int64_t)heads * d > INT32_MAX || (inverse != 0 && inverse != 1))
    return PLC_ERR_INVALID;
  if (x == out && (x_stride[0] != out_stride[0] || x_stride[1] != out_stride[1])) return PLC_ERR_INVALID;
  if (rows == 0) return PLC_OK;
  if (!aligned(x, 16) || !aligned(out, 16) || !aligned(positions, 4)) return PLC_ERR_INVALID;
  RotateArgs a = {};
  a.by = {rotary->turns, rotary->r, rotary->interleaved, inverse ? 1.0f / rotary->magnitude : rotary->magnitude, inverse ? -1.0f : 1.0f};
  a.r.rows = rows;
  a.rel = positions;
  a.heads = heads, a.d8 = d / 8;
  a.q = static_cast<const uint16_t *>(x), a.q_out = static_cast<uint16_t *>(out);
  a.q_node = x_stride[0], a.q_head = x_stride[1], a.out_node = out_stride[0], a.out_head = out_stride[1];
  return rotate<false>(a, type, rows, heads, static_cast<hipStream_t>(stream));
}

extern "C" int plc_rotate_store(const plc_pages *pages, const plc_rows *rows, const plc_rotary *rotary, int32_t type,
                                const int32_t *off, const int32_t *base, const int32_t *rel, const void *k, const void *v,
                                const void *q, const int64_t *q_stride, int32_t G, void *q_out, const int64_t *q_out_stride,
                                uint32_t *status, void *stream) {
  if (!pages_valid(pages) || !rows_valid(pages, rows) || !rotary_valid(rotary, pages->d) || (type != PLC_FP16 && type != PLC_BF16) ||
      !aligned(off, 4) || (base && !aligned(base, 4)) || (rel && !aligned(rel, 4)) || !status ||
      (int64_t)rows->layers * pages->H >= 1 << 29)
    return PLC_ERR_INVALID;
  if ((q == nullptr) != (q_out == nullptr)) return PLC_ERR_INVALID;
  if (q && (!rows->packed || !strides_ok(q_stride) || G < 1 || !strides_out_ok(q_out_stride, rows->rows, (int64_t)pages->H * G, pages->d) || (int64_t)pages->H * G >= 1 << 29 ||
            (q == q_out && (q_stride[0] != q_out_stride[0] || q_stride[1] != q_out_stride[1]))))
    return PLC_ERR_INVALID;
  if (rows->rows == 0) return PLC_OK;
  if (!aligned(k, 16) || !aligned(v, 16) || (q && (!aligned(q, 16) || !aligned(q_out, 16)))) return PLC_ERR_INVALID;
  RotateArgs a = {};
  a.by = {rotary->turns, rotary->r, rotary->interleaved, rotary->magnitude, 1.0f};
  a.p = pool_view(pages);
  a.r = rows_view(rows, const_cast<void *>(k), const_cast<void *>(v), 0);
  a.off = off, a.base = base, a.rel = rel;
  a.d8 = a.p.d8;
  if (q) {
    a.heads = pages->H * G;
    a.q = static_cast<const uint16_t *>(q), a.q_out = static_cast<uint16_t *>(q_out);
    a.q_node = q_stride[0], a.q_head = q_stride[1], a.out_node = q_out_stride[0], a.out_head = q_out_stride[1];
  }
  a.status = status;
  const int64_t total = rows->packed ? rows->rows : rows->rows * pages->S;
  return rotate<true>(a, type, total, 2 * (int64_t)rows->layers * pages->H + a.heads, static_cast<hipStream_t>(stream));
}
