// Rotary positions with several axes.  Pair (a, b) -> (a cos - b sin, a sin + b cos); the gradient is the same with -sin.
//
// A CTA takes a few rows (tokens), forms the cosines and sines of its rows' pairs once -- heads share them -- in shared memory and turns
// all heads.  Bound by HBM: every component is read and written once (8 x 1021 rows of 32 heads of 128 fp32 components: 45 us, 5.9 TB/s; one
// tree's queries, 61 rows of 2 sequences: a launch).
#include "cache_common.cuh"

namespace lantern {

constexpr int RT = 256;

struct RotaryParams {
  const void* x;
  void* out;
  RowStride xs, os;
  Rotation rot;
  int R, H, D;
  int64_t rows;        // B * R
  int per_cta;         // rows per CTA
  float sign;
  bool in_place;
};

// One unit: VEC components.  Pairs of halves: the VEC components from j on and the VEC from j + P on; interleaved: VEC in a row.
template <bool BF16, int VEC>
__device__ __forceinline__ void load_unit(const typename Row<BF16>::T* p, float (&v)[VEC]) {
  if constexpr (VEC == 8) {
    Row<BF16>::get8(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = Row<BF16>::get(p + i);
  }
}
template <bool BF16, int VEC>
__device__ __forceinline__ void store_unit(typename Row<BF16>::T* p, const float (&v)[VEC]) {
  if constexpr (VEC == 8) {
    Row<BF16>::put8(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) Row<BF16>::put(p + i, v[i]);
  }
}

template <bool BF16, int VEC, bool INTERLEAVED>
__global__ void __launch_bounds__(RT) lantern_rotary_kernel(RotaryParams P) {
  using T = typename Row<BF16>::T;
  extern __shared__ float2 cs[];   // [rows of the CTA][pairs]
  const int pairs = P.rot.pairs;
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * P.per_cta;
  const int rows = static_cast<int>(P.rows - row0 < P.per_cta ? P.rows - row0 : P.per_cta);
  for (int i = threadIdx.x; i < rows * pairs; i += RT) {
    const int t = i / pairs;
    float2 v = turn(P.rot, row0 + t, i - t * pairs);
    v.y *= P.sign;
    cs[i] = v;
  }
  __syncthreads();
  const T* x = static_cast<const T*>(P.x);
  T* out = static_cast<T*>(P.out);
  const int turned = INTERLEAVED ? 2 * pairs / VEC : pairs / VEC;              // units of turned components in a head
  const int units = turned + (P.in_place ? 0 : (P.D - 2 * pairs) / VEC);       // and of those that are only copied
  const int per_row = P.H * units;
  for (int i = threadIdx.x; i < rows * per_row; i += RT) {
    const int t = i / per_row, rest = i - t * per_row, h = rest / units, u = rest - h * units;
    const int64_t row = row0 + t, b = row / P.R, r = row - b * P.R;
    const T* px = x + b * P.xs.b + r * P.xs.r + h * P.xs.h;
    T* po = out + b * P.os.b + r * P.os.r + h * P.os.h;
    const float2* c = cs + t * pairs;
    if (u >= turned) {
      const int d = 2 * pairs + (u - turned) * VEC;
      float v[VEC];
      load_unit<BF16, VEC>(px + d, v);
      store_unit<BF16, VEC>(po + d, v);
    } else if constexpr (INTERLEAVED) {
      const int d = u * VEC;
      float v[VEC];
      load_unit<BF16, VEC>(px + d, v);
#pragma unroll
      for (int e = 0; e < VEC; e += 2) {
        const float2 w = c[(d + e) >> 1];
        const float a = v[e], bb = v[e + 1];
        v[e] = turned_low(a, bb, w);
        v[e + 1] = turned_high(a, bb, w);
      }
      store_unit<BF16, VEC>(po + d, v);
    } else {
      const int j = u * VEC;
      float v[VEC], w[VEC];
      load_unit<BF16, VEC>(px + j, v);
      load_unit<BF16, VEC>(px + j + pairs, w);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float2 q = c[j + e];
        const float a = v[e], bb = w[e];
        v[e] = turned_low(a, bb, q);
        w[e] = turned_high(a, bb, q);
      }
      store_unit<BF16, VEC>(po + j, v);
      store_unit<BF16, VEC>(po + j + pairs, w);
    }
  }
}

template <bool BF16, int VEC, bool INTERLEAVED>
static cudaError_t launch_rotary(RotaryParams& P, cudaStream_t st) {
  // rows per CTA: about four units per thread, and no more angles than one per thread and a few rounds
  const int64_t per_row = static_cast<int64_t>(P.H) * P.D / VEC;
  int64_t per = per_row ? (4 * RT + per_row - 1) / per_row : 1;
  const int64_t most = 4 * RT / P.rot.pairs;
  if (per > most) per = most;
  if (per < 1) per = 1;
  P.per_cta = static_cast<int>(per);
  const int64_t grid = (P.rows + per - 1) / per;
  lantern_rotary_kernel<BF16, VEC, INTERLEAVED>
      <<<static_cast<unsigned>(grid), RT, static_cast<size_t>(per) * P.rot.pairs * sizeof(float2), st>>>(P);
  return cudaGetLastError();
}

}  // namespace lantern

using namespace lantern;

extern "C" lantern_status lantern_rotary(const void* x, void* out, int dtype, int B, int R, int H, int D, const int64_t x_stride[3],
                                         const int64_t out_stride[3], const lantern_rotation* rotation, int inverse, void* cuda_stream) {
  if (dtype != LANTERN_F32 && dtype != LANTERN_BF16) return LANTERN_E_PARAM;
  if (B < 0 || R < 0 || H < 0 || D < 2 || D > 512 || D % 2) return LANTERN_E_SHAPE;
  if (!rotation || !x_stride || !out_stride) return LANTERN_E_NULL;
  RotaryParams P;
  const lantern_status bad = make_rotation(rotation, B, R, D, &P.rot);
  if (bad != LANTERN_OK) return bad;
  P.rows = static_cast<int64_t>(B) * R;
  if (P.rows > INT32_MAX || static_cast<int64_t>(H) * D > INT32_MAX / 2) return LANTERN_E_SHAPE;
  if (P.rows == 0 || H == 0) return LANTERN_OK;
  if (!x || !out) return LANTERN_E_NULL;
  if ((B > 1 && out_stride[0] == 0) || (R > 1 && out_stride[1] == 0) || (H > 1 && out_stride[2] == 0)) return LANTERN_E_PARAM;   // (one row for several)
  P.x = x;
  P.out = out;
  P.xs = {x_stride[0], x_stride[1], x_stride[2]};
  P.os = {out_stride[0], out_stride[1], out_stride[2]};
  P.R = R;
  P.H = H;
  P.D = D;
  P.sign = inverse ? -1.0f : 1.0f;
  P.in_place = x == out;
  const bool bf = dtype == LANTERN_BF16, inter = rotation->interleaved != 0;
  const int size = bf ? 2 : 4;
  if (reinterpret_cast<uintptr_t>(x) % size || reinterpret_cast<uintptr_t>(out) % size) return LANTERN_E_ALIGN;
  const int64_t xs[3] = {P.xs.b, P.xs.r, P.xs.h}, os[3] = {P.os.b, P.os.r, P.os.h};
  // eight components at a time where every unit starts on 16 bytes
  const bool wide = aligned16(x, xs, size) && aligned16(out, os, size) && D % 8 == 0 && (inter ? P.rot.pairs % 4 == 0 : P.rot.pairs % 8 == 0);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e;
  if (inter) {
    if (wide) e = bf ? launch_rotary<true, 8, true>(P, st) : launch_rotary<false, 8, true>(P, st);
    else e = bf ? launch_rotary<true, 2, true>(P, st) : launch_rotary<false, 2, true>(P, st);
  } else {
    if (wide) e = bf ? launch_rotary<true, 8, false>(P, st) : launch_rotary<false, 8, false>(P, st);
    else e = bf ? launch_rotary<true, 1, false>(P, st) : launch_rotary<false, 1, false>(P, st);
  }
  return e == cudaSuccess ? LANTERN_OK : LANTERN_E_CUDA;
}
