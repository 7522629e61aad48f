// Rotary positions of queries and keys, with the rotated keys and the values
// written to their cache slots.
//
// Pair i of a head (elements x, y) at position t turns by the angle t theta_i:
//   x' = r (x cos - y sin), y' = r (y cos + x sin),  r the caller's magnitude.
// Angles of far positions need more than a float's 24 bits (at t = 10^6 a float
// product is off by up to 0.03 rad), so theta_i comes as a fixed-point fraction of a
// turn, T_i = theta_i / (2 pi) 2^64: t T_i mod 2^64 is the exact phase of T_i's
// multiple, and full turns fall away without a division.
//
// 8 lanes hold a head's 128 elements, lane c the pairs 8c .. 8c + 7 (half layout:
// elements 8c.. and rotary_dim / 2 + 8c..; pair layout: 16c .. 16c + 15), so that a
// lane's cosines and sines serve every head that its wave turns.  The kernel is bound
// by HBM: q in and out, k and v in, their cache rows out.  16384 tokens of 64 + 2 x 8 heads
// into an 8-bit pool, not in a cache, take 128 us (638 MB, 5.0 TB/s; a plain copy reaches
// 5.2), 64 tokens of 32 + 2 x 8 heads 4.4 us (a launch).
#include <algorithm>

#include "common.h"
#include "rope.h"

namespace ekv {
namespace {

constexpr int kWaves = 4;

// m cos and m sin of 2 pi p 2^-64, rounded once as a rule (0.30 units in the last place rms,
// where one rounding has 0.29; 2.5 at most, for phases of a few 2^-32): the nearest
// quarter turn taken off exactly, the rest as x + e (a product and what it rounded away),
// then the Taylor polynomials on [-pi/4, pi/4] (to x^10 and x^9: truncated below 2e-9),
// their small terms added to x and to 1 - x^2 / 2 at the end, and what that addition
// rounds away carried through the product with m.  Products are fused where it says so
// and nowhere else: one that is added fused and subtracted rounded would count what it
// rounds away twice (that, and m on a rounded sum, left 16 to 42 % more 16-bit outputs
// that are not the nearest; 64 tokens 4.3 us then, 4.4 now).
__device__ __forceinline__ void cos_sin(uint64_t p, float m, float& c, float& s) {
#pragma clang fp contract(off)
  constexpr double kUnit = 1.46291807926715968e-9;   // 2 pi / 2^32
  constexpr float kHigh = (float)kUnit, kLow = (float)(kUnit - (double)kHigh);
  const uint32_t quarter = ((uint32_t)(p >> 32) + 0x20000000u) >> 30;
  const int32_t rest = (int32_t)((uint32_t)(p >> 32) - (quarter << 30));   // (|rest| <= 2^29)
  const float r = (float)rest, below = fmaf((float)(uint32_t)p, 0x1p-32f, (float)(rest - (int32_t)r));
  const float x = r * kHigh;
  const float e = fmaf(r, kHigh, -x) + fmaf(r, kLow, below * kHigh);
  const float z = x * x;
  const float odd = x * z * fmaf(z, fmaf(z, fmaf(z, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6);
  const float even = z * z * fmaf(z, fmaf(z, fmaf(z, -1.0f / 3628800, 1.0f / 40320), -1.0f / 720), 1.0f / 24);
  const float half = 0.5f * z, top = fmaf(-0.5f, z, 1.0f);
  const float small_s = fmaf(e, top, odd), small_c = ((1.0f - top) - half) + fmaf(-x, e, fmaf(-0.5f, fmaf(x, x, -z), even));
  const float sum_s = x + small_s, sum_c = top + small_c;
  const float sn = fmaf(m, sum_s, m * (small_s - (sum_s - x)));
  const float cs = fmaf(m, sum_c, m * (small_c - (sum_c - top)));
  const bool swap = quarter & 1;
  c = swap ? sn : cs;
  s = swap ? cs : sn;
  if ((quarter + 1) & 2) c = -c;
  if (quarter & 2) s = -s;
}

// 8 floats -> 8 words of T (to nearest) or, for an 8-bit pool, 8 E5M2 bytes (to nearest, straight from 32 bits)
template <typename T>
__device__ __forceinline__ u32x4 words8(const float (&x)[8]) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float back;
    w[i] = (uint32_t)Mma<T>::round(x[2 * i], &back) | ((uint32_t)Mma<T>::round(x[2 * i + 1], &back) << 16);
  }
  return w;
}
__device__ __forceinline__ u32x2 bytes8(const float (&x)[8]) {
  u32x2 w;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int d = __builtin_amdgcn_cvt_pk_bf8_f32(x[4 * i], x[4 * i + 1], 0, false);
    w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(x[4 * i + 2], x[4 * i + 3], d, true);
  }
  return w;
}
template <typename T>
__device__ __forceinline__ void floats8(u32x4 w, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = Mma<T>::widen((uint16_t)w[i]);
    x[2 * i + 1] = Mma<T>::widen((uint16_t)(w[i] >> 16));
  }
}

// ONCE: inputs are read past the caches
template <typename T, bool F8, bool ONCE>
__global__ __launch_bounds__(64 * kWaves) void rope_kernel(RopeArgs a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 7;
  const int rows = a.num_q_heads + 2 * a.num_kv_heads;   // rows of a token: query heads, key heads, value heads
  const unsigned parts = (unsigned)(rows + a.rows_per_wave - 1) / a.rows_per_wave, item = blockIdx.x * kWaves + wave;
  const int token = item / parts, row0 = (item - token * parts) * a.rows_per_wave;
  if (token >= a.n) return;
  const int row_end = min(rows, row0 + a.rows_per_wave);

  const int slot = a.slots[token];
  const int64_t position = a.positions[token];
  const int turned = a.rotary_dim / 16;                            // lanes whose pairs turn
  // this lane's two 8-element chunks of a head
  const int chunk0 = a.pairs ? 2 * c : (c < turned ? c : 2 * turned + 2 * (c - turned));
  const int chunk1 = a.pairs ? 2 * c + 1 : (c < turned ? turned + c : chunk0 + 1);
  const int values0 = a.num_q_heads + a.num_kv_heads;              // the first value head
  auto load = [&](int r, u32x4& w0, u32x4& w1) {
    const uint16_t* src = r < a.num_q_heads ? a.q + token * a.q_stride + (size_t)r * kHeadDim
                          : r < values0     ? a.k + token * a.k_stride + (size_t)(r - a.num_q_heads) * kHeadDim
                                            : a.v + token * a.v_stride + (size_t)(r - values0) * kHeadDim;
    const u32x4 *p0 = reinterpret_cast<const u32x4*>(src + 8 * chunk0), *p1 = reinterpret_cast<const u32x4*>(src + 8 * chunk1);
    if constexpr (ONCE) {
      w0 = __builtin_nontemporal_load(p0);
      w1 = __builtin_nontemporal_load(p1);
    } else {
      w0 = *p0;
      w1 = *p1;
    }
  };
  // (the first row's values are on their way while the angles are worked out, the next row's while one is turned)
  int r = row0 + (lane >> 3);
  u32x4 next0{0u, 0u, 0u, 0u}, next1{0u, 0u, 0u, 0u};
  if (r < row_end) load(r, next0, next1);

  const bool in_pool = slot >= 0 && slot / kPage < a.num_blocks;   // (outside the pool: the cache is left as it is)
  float cs[8], sn[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    cs[i] = 1.0f;
    sn[i] = 0.0f;
    if (c < turned) cos_sin((uint64_t)position * a.turns[8 * c + i], a.magnitude, cs[i], sn[i]);
  }

#pragma unroll 1
  for (; r < row_end; r += 8) {
    u32x4 w0 = next0, w1 = next1;
    if (r + 8 < row_end) load(r + 8, next0, next1);
    const int kind = r < a.num_q_heads ? 0 : (r < values0 ? 1 : 2);   // query, key, value
    if (kind != 0 && !in_pool) continue;
    float x[8], y[8];
    if (kind != 2 && c < turned) {
      floats8<T>(w0, x);
      floats8<T>(w1, y);
      if (a.pairs) {   // elements 16 c + 2 i, + 1
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x0 = x[2 * i], x1 = x[2 * i + 1], y0 = y[2 * i], y1 = y[2 * i + 1];
          x[2 * i] = x0 * cs[i] - x1 * sn[i];
          x[2 * i + 1] = x1 * cs[i] + x0 * sn[i];
          y[2 * i] = y0 * cs[4 + i] - y1 * sn[4 + i];
          y[2 * i + 1] = y1 * cs[4 + i] + y0 * sn[4 + i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x0 = x[i], y0 = y[i];
          x[i] = x0 * cs[i] - y0 * sn[i];
          y[i] = y0 * cs[i] + x0 * sn[i];
        }
      }
      w0 = words8<T>(x);
      w1 = words8<T>(y);
    } else if (F8) {
      floats8<T>(w0, x);
      floats8<T>(w1, y);
    }
    if (kind == 0) {
      uint16_t* dst = a.q_out + token * a.out_stride + (size_t)r * kHeadDim;
      *reinterpret_cast<u32x4*>(dst + 8 * chunk0) = w0;
      *reinterpret_cast<u32x4*>(dst + 8 * chunk1) = w1;
    } else {
      const int head = r - (kind == 1 ? a.num_q_heads : values0);
      const size_t at = (((size_t)(slot / kPage) * 2 + (kind - 1)) * a.num_kv_heads + head) * kTileWords + (slot % kPage) * kHeadDim;
      if constexpr (F8) {
        uint8_t* dst = static_cast<uint8_t*>(a.pool) + at;
        *reinterpret_cast<u32x2*>(dst + 8 * chunk0) = bytes8(x);
        *reinterpret_cast<u32x2*>(dst + 8 * chunk1) = bytes8(y);
      } else {
        uint16_t* dst = static_cast<uint16_t*>(a.pool) + at;
        *reinterpret_cast<u32x4*>(dst + 8 * chunk0) = w0;
        *reinterpret_cast<u32x4*>(dst + 8 * chunk1) = w1;
      }
    }
  }
}

template <typename T, bool F8>
void launch_typed(const RopeArgs& a, dim3 grid, dim3 block, bool once, hipStream_t st) {
  if (once) hipLaunchKernelGGL((rope_kernel<T, F8, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((rope_kernel<T, F8, false>), grid, block, 0, st, a);
}

}  // namespace

hipError_t launch_rope(const RopeArgs& a, int dtype, hipStream_t st) {
  if (a.n == 0) return hipSuccess;
  RopeArgs b = a;
  const int rows = a.num_q_heads + 2 * a.num_kv_heads;
  // A wave works the angles out once for its rows, 8 at a time: as many rows as leave 2048
  // waves (8 a CU).  Measured with 48 rows a token, us at 8 / 16 / 24 / 48 rows a wave:
  // 64 tokens 4.4 / 4.8 / 5.3 / 6.7, 512 tokens 6.1 / 5.7 / 6.1 / 7.4, 1024 tokens
  // 9.2 / 7.5 / 7.0 / 7.9, 8192 tokens 52.1 / 41.2 / 38.5 / 37.6.
  const int64_t share = ((int64_t)a.n * rows + 2047) / 2048;
  b.rows_per_wave = (int)std::min<int64_t>((share + 7) / 8 * 8, rows);
  const int64_t waves = (int64_t)a.n * ((rows + b.rows_per_wave - 1) / b.rows_per_wave);   // (at most 2048 + a.n)
  // Inputs of 32 MB and more are read past the caches, which the outputs, read next, then
  // have to themselves: a copy that makes q, k and v, this kernel and a copy of its queries
  // take 105.5 us for 8192 tokens of 48 rows (111.3 with plain loads), 58.5 (59.9) for
  // 4096; 1337 tokens (16 MB) alone, their inputs still cached, 11.9 (9.7).  Stores past the
  // caches make this kernel 5 % faster and what reads its outputs slower by more.
  const bool once = (int64_t)a.n * rows * kHeadDim * 2 >= (32 << 20);
  const dim3 grid((unsigned)((waves + kWaves - 1) / kWaves)), block(64 * kWaves);
  switch (dtype) {
    case 0: launch_typed<Bf16, false>(b, grid, block, once, st); break;
    case 1: launch_typed<Fp16, false>(b, grid, block, once, st); break;
    case 3: launch_typed<Fp16, true>(b, grid, block, once, st); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace ekv
