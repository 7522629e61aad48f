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
// into an 8-bit pool, not in a cache, take 126 us (638 MB, 5.0 TB/s; a plain copy reaches
// 5.2), 64 tokens of 32 + 2 x 8 heads 3.4 us (a launch).  A wave's lane works out one pair's angle
// and passes it on through LDS (each of a head's 8 lanes for itself, all of them eight times over: 128 and 4.4 us,
// 2048 tokens with norms 11.9 where they are 9.6 now).
//
// Heads may be levelled first (the norms of queries and keys): x / sqrt(mean(x^2) + eps) (offset +
// weight) in the same registers, the squares summed over the 8 lanes, so that a norm adds no byte but
// its weights.  16384 tokens of 64 + 2 x 8 heads into an 8-bit pool take 126 us with norms as without;
// 8192 of 32 + 2 x 8 into a 16-bit one 38.1 (35.6 without: its vector work, 350 instructions a
// wave and 8 rows, is not all hidden behind its loads and stores), 64 4.0.
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
// that are not the nearest; 64 tokens 4.3 us then, 4.4 with it).
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
typedef float f32x2 __attribute__((ext_vector_type(2)));
template <typename T> struct Pair;
template <> struct Pair<Bf16> { typedef __bf16 two __attribute__((ext_vector_type(2))); };
template <> struct Pair<Fp16> { typedef _Float16 two __attribute__((ext_vector_type(2))); };
template <typename T>
__device__ __forceinline__ u32x4 words8(const float (&x)[8]) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x[2 * i], x[2 * i + 1]}), typename Pair<T>::two));
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

// Sum over the 8 lanes that hold a head (each pair, each four, then the other four, mirrored).
__device__ __forceinline__ float sum8(float x) {
  x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0xB1, 0xf, 0xf, true));    // quad_perm 1,0,3,2
  x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x4E, 0xf, 0xf, true));    // quad_perm 2,3,0,1
  x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x141, 0xf, 0xf, true));   // row_half_mirror
  return x;
}
__device__ __forceinline__ float squares(const float (&x)[8], const float (&y)[8]) {
  float s = 0.0f, t = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    s = fmaf(x[i], x[i], s);
    t = fmaf(y[i], y[i], t);
  }
  return sum8(s + t);
}

// A head's elements times 1 / sqrt(mean of their squares + eps) and the weights.  Squares
// are summed in 32 bits; where that overflows (bf16 values beyond 10^18), over elements
// 2^-70 as large, whose squares are far above any eps that was not lost before.
__device__ __forceinline__ void level(const RopeArgs& a, float (&x)[8], float (&y)[8], const float (&u)[8], const float (&v)[8]) {
  constexpr float kDown = 0x1p-70f;
  float sum = squares(x, y), eps = a.eps;
  if (!(sum < __builtin_inff())) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] *= kDown;
      y[i] *= kDown;
    }
    sum = squares(x, y);
    eps = 0.0f;
  }
  const float f = __builtin_amdgcn_rsqf(fmaf(sum, 1.0f / kHeadDim, eps));
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[i] = x[i] * f * u[i];   // (x f is at most the root of 128)
    y[i] = y[i] * f * v[i];
  }
}

// Norms: none; by weights that all heads share (or none), kept in registers; by weights read for each row.
enum Norm { kNoNorm, kShared, kPerHead };

// ONCE: inputs are read past the caches
template <typename T, bool F8, bool ONCE, int NORM>
__global__ __launch_bounds__(64 * kWaves) void rope_kernel(RopeArgs a) {
  __shared__ float2 turns[kWaves][64];
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
  // Weights of this lane's elements: as loaded (row r's head's; 0 for all heads'), and plus the offset, or 1.
  auto load_weights = [&](const uint16_t* src, int head, int stride, u32x4& w0, u32x4& w1) {
    if (!src) return;
    w0 = *reinterpret_cast<const u32x4*>(src + head * stride + 8 * chunk0);
    w1 = *reinterpret_cast<const u32x4*>(src + head * stride + 8 * chunk1);
  };
  auto weights = [&](const uint16_t* src, u32x4 w0, u32x4 w1, float (&u)[8], float (&v)[8]) {
    floats8<T>(w0, u);
    floats8<T>(w1, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      u[i] = src ? u[i] + a.offset : 1.0f;
      v[i] = src ? v[i] + a.offset : 1.0f;
    }
  };
  auto load_head_weights = [&](int r, u32x4& w0, u32x4& w1) {
    if (r < a.num_q_heads) load_weights(a.q_weight, r, a.q_weight_stride, w0, w1);
    else if (r < values0) load_weights(a.k_weight, r - a.num_q_heads, a.k_weight_stride, w0, w1);
  };
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
  u32x4 weight0{0u, 0u, 0u, 0u}, weight1{0u, 0u, 0u, 0u}, k_weight0{0u, 0u, 0u, 0u}, k_weight1{0u, 0u, 0u, 0u};
  if (r < row_end) {
    load(r, next0, next1);
    if constexpr (NORM == kPerHead) load_head_weights(r, weight0, weight1);
  }
  if constexpr (NORM == kShared) {
    load_weights(a.q_weight, 0, 0, weight0, weight1);
    load_weights(a.k_weight, 0, 0, k_weight0, k_weight1);
  }

  const bool in_pool = slot >= 0 && slot / kPage < a.num_blocks;   // (outside the pool: the cache is left as it is)
  // Lane i works pair i out, for the 8 lanes that hold it, one of each head.
  float2 turn = make_float2(1.0f, 0.0f);
  if (lane < 8 * turned) cos_sin((uint64_t)position * a.turns[lane], a.magnitude, turn.x, turn.y);
  turns[wave][lane] = turn;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (of one wave: its LDS accesses stay in order)
  __builtin_amdgcn_wave_barrier();
  float cs[8], sn[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    cs[i] = turns[wave][8 * c + i].x;
    sn[i] = turns[wave][8 * c + i].y;
  }

  float qu[8], qv[8], ku[8], kv[8];
  if constexpr (NORM == kShared) {
    weights(a.q_weight, weight0, weight1, qu, qv);
    weights(a.k_weight, k_weight0, k_weight1, ku, kv);
  }

#pragma unroll 1
  for (; r < row_end; r += 8) {
    u32x4 w0 = next0, w1 = next1;
    const u32x4 u0 = weight0, u1 = weight1;
    if (r + 8 < row_end) {
      load(r + 8, next0, next1);
      if constexpr (NORM == kPerHead) load_head_weights(r + 8, weight0, weight1);
    }
    const int kind = r < a.num_q_heads ? 0 : (r < values0 ? 1 : 2);   // query, key, value
    if (kind != 0 && !in_pool) continue;
    float x[8], y[8];
    if (kind != 2 && (NORM != kNoNorm || c < turned)) {
      floats8<T>(w0, x);
      floats8<T>(w1, y);
      if constexpr (NORM != kNoNorm) {
        float u[8], v[8];
        if constexpr (NORM == kShared) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            u[i] = kind == 0 ? qu[i] : ku[i];
            v[i] = kind == 0 ? qv[i] : kv[i];
          }
        } else {
          weights(kind == 0 ? a.q_weight : a.k_weight, u0, u1, u, v);
        }
        level(a, x, y, u, v);
      }
      if (NORM != kNoNorm && c >= turned) {
        // (levelled, not turned)
      } else if (a.pairs) {   // elements 16 c + 2 i, + 1 (which product is fused is said, not left to the compiler)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x0 = x[2 * i], x1 = x[2 * i + 1], y0 = y[2 * i], y1 = y[2 * i + 1];
          x[2 * i] = fmaf(x0, cs[i], -(x1 * sn[i]));
          x[2 * i + 1] = fmaf(x0, sn[i], x1 * cs[i]);
          y[2 * i] = fmaf(y0, cs[4 + i], -(y1 * sn[4 + i]));
          y[2 * i + 1] = fmaf(y0, sn[4 + i], y1 * cs[4 + i]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x0 = x[i], y0 = y[i];
          x[i] = fmaf(x0, cs[i], -(y0 * sn[i]));
          y[i] = fmaf(y0, cs[i], x0 * sn[i]);
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

template <typename T, bool F8, int NORM>
void launch_once(const RopeArgs& a, dim3 grid, dim3 block, bool once, hipStream_t st) {
  if (once) hipLaunchKernelGGL((rope_kernel<T, F8, true, NORM>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((rope_kernel<T, F8, false, NORM>), grid, block, 0, st, a);
}
template <typename T, bool F8>
void launch_typed(const RopeArgs& a, dim3 grid, dim3 block, bool once, hipStream_t st) {
  if (!a.norm) launch_once<T, F8, kNoNorm>(a, grid, block, once, st);
  // (shared weights are worth keeping from 16 rows a wave on: 1024 tokens of 32 / 8 heads 7.2 us, read a row 7.4, 2048 9.5 and
  // 9.9, 8192 36.4 and 37.8; with 8 rows a wave, 512 tokens, 5.1 and 4.8)
  else if (a.q_weight_stride == 0 && a.k_weight_stride == 0 && a.rows_per_wave > 8) launch_once<T, F8, kShared>(a, grid, block, once, st);
  else launch_once<T, F8, kPerHead>(a, grid, block, once, st);
}

}  // namespace

hipError_t launch_rope(const RopeArgs& a, int dtype, hipStream_t st) {
  if (a.n == 0) return hipSuccess;
  RopeArgs b = a;
  const int rows = a.num_q_heads + 2 * a.num_kv_heads;
  // A wave works the angles out once for its rows, 8 at a time: as many rows as leave 4096
  // waves (16 a CU).  Measured with 48 rows a token, us at 1024 / 2048 / 4096 / 8192 waves:
  // 64 tokens 2.9 at any (8 rows a wave), 512 tokens 4.6 / 4.3 / 4.0 / 3.9, 1024 tokens
  // 7.0 / 6.4 / 6.1 / 6.3, 2048 9.7 / 9.7 / 9.0 / 9.1, 8192 36.1 / 35.7 / 35.6 / 35.5.
  const int64_t share = ((int64_t)a.n * rows + 4095) / 4096;
  b.rows_per_wave = (int)std::min<int64_t>((share + 7) / 8 * 8, rows);
  const int64_t waves = (int64_t)a.n * ((rows + b.rows_per_wave - 1) / b.rows_per_wave);   // (at most 4096 + a.n)
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
