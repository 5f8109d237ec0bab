// Shared by the cache operators (rotary.cu, cache.cu, cache_attention*.cu): rows of either type, e4m3 codes, block scales, rotation
// angles, and the host's checks of lantern_cache and lantern_rotation.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "lantern.h"
#include "lantern_device.cuh"

namespace lantern {

constexpr float kCodeMax = 448.0f;     // largest e4m3 value
constexpr int kLeastExponent = -100;   // of a block's scale: a block of zeros has 2^-100
constexpr int kMaxHeadDim = 128;
constexpr int kMaxTreeRows = 1025;     // as lantern_verify: at most 1024 drafts

struct RowStride {
  int64_t b, r, h;
};

// ---- eight consecutive components -----------------------------------------------------------------------------------------
__device__ __forceinline__ void bf16x2_widen(uint32_t w, float& lo, float& hi) {
  lo = __uint_as_float(w << 16);
  hi = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ uint32_t bf16x2_round(float lo, float hi) {   // to nearest even
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <bool BF16>
struct Row;
template <>
struct Row<true> {
  using T = __nv_bfloat16;
  static __device__ __forceinline__ float get(const T* p) { return __bfloat162float(*p); }
  static __device__ __forceinline__ void put(T* p, float v) { *p = __float2bfloat16_rn(v); }
  static __device__ __forceinline__ void get8(const T* p, float (&v)[8]) {   // 16-byte aligned
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    bf16x2_widen(x.x, v[0], v[1]), bf16x2_widen(x.y, v[2], v[3]), bf16x2_widen(x.z, v[4], v[5]), bf16x2_widen(x.w, v[6], v[7]);
  }
  static __device__ __forceinline__ void put8(T* p, const float (&v)[8]) {
    *reinterpret_cast<uint4*>(p) =
        make_uint4(bf16x2_round(v[0], v[1]), bf16x2_round(v[2], v[3]), bf16x2_round(v[4], v[5]), bf16x2_round(v[6], v[7]));
  }
};
template <>
struct Row<false> {
  using T = float;
  static __device__ __forceinline__ float get(const T* p) { return *p; }
  static __device__ __forceinline__ void put(T* p, float v) { *p = v; }
  static __device__ __forceinline__ void get8(const T* p, float (&v)[8]) {
    const float4 x = *reinterpret_cast<const float4*>(p), y = *reinterpret_cast<const float4*>(p + 4);
    v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w, v[4] = y.x, v[5] = y.y, v[6] = y.z, v[7] = y.w;
  }
  static __device__ __forceinline__ void put8(T* p, const float (&v)[8]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
  }
};

// ---- e4m3 codes ---------------------------------------------------------------------------------------------------------
// To nearest even; values beyond 448 do not occur under a block's scale, NaN becomes the NaN code 0x7f.
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  return static_cast<uint32_t>(lo) | (static_cast<uint32_t>(hi) << 16);
}
// two codes -> two halves (exact)
__device__ __forceinline__ uint32_t decode2(uint16_t codes) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(codes));
  return r;
}
__device__ __forceinline__ void decode4(uint32_t codes, float (&v)[4]) {
  const uint32_t lo = decode2(static_cast<uint16_t>(codes & 0xffffu)), hi = decode2(static_cast<uint16_t>(codes >> 16));
  const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo)), b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
  v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y;
}

// ---- block scales -------------------------------------------------------------------------------------------------------
// The least power of two 2^e, e >= -100, with amax <= 448 * 2^e (448 = 0.875 * 2^9); amax finite and >= 0.
__device__ __forceinline__ float scale_for(float amax) {
  const uint32_t bits = __float_as_uint(amax);
  int e = static_cast<int>(bits >> 23) - 135 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);   // amax = 1.m * 2^(E - 127); 448 = 1.75 * 2^8
  e = max(e, kLeastExponent);                                                              // (a subnormal amax has e < -100)
  return __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
}
// x / scale: a multiplication where the scale is a power of two, as append leaves them
struct Divider {
  float scale, inverse;
  bool exact;
  __device__ __forceinline__ float operator()(float x) const { return exact ? x * inverse : __fdiv_rn(x, scale); }
};
__device__ __forceinline__ Divider divider(float s) { return {s, __frcp_rn(s), (__float_as_uint(s) & 0x7fffffu) == 0}; }
__device__ __forceinline__ bool usable_scale(float s) { return s > 0.0f && s < __int_as_float(0x7f800000); }

// ---- rotation -----------------------------------------------------------------------------------------------------------
struct Rotation {
  const float* inv_freq;      // NULL: no rotation
  const int32_t* positions;   // [axes, B, R]
  int64_t plane;              // B * R
  int pairs, interleaved;
  int ends[LANTERN_MAX_AXES];   // running sums of the sections; axes that are not used end at `pairs`
};
// The turns that one position stands for, as a 64-bit fraction (whole turns dropped): of a position's multiple of it, modulo one turn, an integer product
// is exact, however far the position.  The product with 1 / (2 pi) has that number in two doubles and its own rounding beside it, so that the fraction is
// good to its last bit and 2^31 positions to 2^-33 of a turn.
__device__ __forceinline__ uint64_t turn_step(const Rotation& R, int j) {
  constexpr double kTurns = 0.15915494309189535, kTurnsRest = -9.839338337591243e-18, kOne = 18446744073709551616.0;
  const double f = static_cast<double>(__ldg(R.inv_freq + j)), turns = f * kTurns, rest = __fma_rn(f, kTurnsRest, __fma_rn(f, kTurns, -turns));
  return static_cast<uint64_t>(__double2ll_rn((turns - rint(turns)) * kOne)) + static_cast<uint64_t>(__double2ll_rn((rest - rint(rest)) * kOne));
}
// cos and sin of a position's angle, which lies within half a turn; what rounding it to single precision leaves (at most 2^-25 half turns) turns the
// result once more.
__device__ __forceinline__ float2 turn_by(uint64_t step, int position) {
  const uint64_t angle = step * static_cast<uint64_t>(static_cast<int64_t>(position));
  const int halves = static_cast<int>(static_cast<uint32_t>(angle >> 32));   // in 2^-31 half turns
  const float near = static_cast<float>(halves);
  const float rest = __fmaf_rn(static_cast<float>(static_cast<int>(static_cast<int64_t>(halves) - static_cast<int64_t>(near))), 4294967296.0f,
                               static_cast<float>(static_cast<uint32_t>(angle))) * (3.14159265f * 1.0842021724855044e-19f);   // (2^-63)
  float s, c;
  sincospif(near * 4.656612873077393e-10f, &s, &c);   // (2^-31)
  return make_float2(__fmaf_rn(-s, rest, c), __fmaf_rn(c, rest, s));
}
__device__ __forceinline__ int position_of(const Rotation& R, int64_t token, int j) {
  const int axis = (j >= R.ends[0]) + (j >= R.ends[1]) + (j >= R.ends[2]);
  return __ldg(R.positions + axis * R.plane + token);
}
__device__ __forceinline__ float2 turn(const Rotation& R, int64_t token, int j) { return turn_by(turn_step(R, j), position_of(R, token, j)); }

// The two components of a turned pair, each with one fused rounding and one of the product: with the angles above, every kernel and path gives the same bits.
__device__ __forceinline__ float turned_low(float a, float b, float2 cs) { return __fmaf_rn(a, cs.x, -__fmul_rn(b, cs.y)); }
__device__ __forceinline__ float turned_high(float a, float b, float2 cs) { return __fmaf_rn(b, cs.x, __fmul_rn(a, cs.y)); }

// ---- host checks --------------------------------------------------------------------------------------------------------
static inline lantern_status check_cache(const lantern_cache* c, const int32_t* table, int width, int B) {
  if (!c || !c->k_code || !c->v_code || !c->k_scale || !c->v_scale || (!table && B != 0)) return LANTERN_E_NULL;
  const int S = c->page_tokens;
  if (S != 16 && S != 32 && S != 64 && S != 128) return LANTERN_E_SHAPE;
  if (c->head_dim < 16 || c->head_dim > kMaxHeadDim || c->head_dim % 16 != 0 || c->pages < 1 || c->heads < 1 || width < 1) return LANTERN_E_SHAPE;
  if (static_cast<int64_t>(c->pages) * c->heads > INT32_MAX / S || width > (1 << 30) / S) return LANTERN_E_SHAPE;
  if ((reinterpret_cast<uintptr_t>(c->k_code) & 15) || (reinterpret_cast<uintptr_t>(c->v_code) & 15)) return LANTERN_E_ALIGN;
  return LANTERN_OK;
}
static inline lantern_status make_rotation(const lantern_rotation* r, int B, int R, int D, Rotation* out) {
  if (!r->inv_freq || (!r->positions && B != 0 && R != 0)) return LANTERN_E_NULL;
  if (r->axes < 1 || r->axes > LANTERN_MAX_AXES) return LANTERN_E_SHAPE;
  out->inv_freq = r->inv_freq;
  out->positions = r->positions;
  out->plane = static_cast<int64_t>(B) * R;
  out->interleaved = r->interleaved != 0;
  int sum = 0;
  for (int a = 0; a < LANTERN_MAX_AXES; ++a) {
    if (a < r->axes) {
      if (r->section[a] < 0 || r->section[a] > D) return LANTERN_E_SHAPE;
      sum += r->section[a];
    }
    out->ends[a] = sum;
  }
  if (sum < 1 || 2 * sum > D) return LANTERN_E_SHAPE;
  for (int a = r->axes - 1; a < LANTERN_MAX_AXES; ++a) out->ends[a] = sum;
  out->pairs = sum;
  return LANTERN_OK;
}
static inline bool aligned16(const void* p, const int64_t (&stride)[3], int size) {   // every row of every head starts on 16 bytes
  const int64_t unit = 16 / size;
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && stride[0] % unit == 0 && stride[1] % unit == 0 && stride[2] % unit == 0;
}

}  // namespace lantern
