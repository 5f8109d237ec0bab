// Attention of a step's rows to the paged 8-bit cache.
//
//   out = sum_c p_c v_c / sum_c p_c,   p_c = 2^(x_c - max x),   x_c = scale log2(e) k_scale (q . k_c)
//
// over the tokens a row sees, in one pass with a running maximum and sum.  A CTA takes the rows of one sequence and cache head (all
// heads of the group: they share the codes) and a part of the tokens; a producer warp copies 64 tokens of codes per stage into
// shared memory, four warps multiply.  Codes become halves in registers (every e4m3 value is one), so do the queries after
// a power of two of their own (8 bits of a bf16 query fit; an fp32 query goes in as two halves, 22 bits), and products are
// m16n8k16 with fp32 accumulators.
#include "cache_attention.cuh"

namespace lantern {

constexpr int CT = 160;   // four warps and the producer
constexpr int kStages = 4;

__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t half2_of(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t half2_rest(float lo, float hi, uint32_t rounded) {   // what the rounding left
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&rounded));
  return half2_of(lo - f.x, hi - f.y);
}
__device__ __forceinline__ uint32_t without_nan(uint32_t codes) { return codes & ~__vcmpeq4(codes & 0x7f7f7f7fu, 0x7f7f7f7fu); }

constexpr int kTile = 64;

struct AttendShared : StageShared<kTile, kStages> {
  float ml[4][16][2];
};

// ROWS = 16: the four warps take 16 tokens of a stage each, for the same 16 rows.  ROWS = 64: each takes 16 rows and all tokens.
template <int ROWS, int DP, bool BF16>
__global__ void __launch_bounds__(CT) lantern_attention_kernel(AttendParams P, const __grid_constant__ CUtensorMap kmap,
                                                               const __grid_constant__ CUtensorMap vmap) {
  using T = typename Row<BF16>::T;
  constexpr int TERMS = BF16 ? 1 : 2;         // halves that a query or probability goes in as
  constexpr int KS = DP / 16, NT = DP / 8;    // steps of the scores' products, column tiles of the output
  constexpr int EL = DP / 4;                  // components of a row that a lane holds, side by side
  constexpr int kStageBytes = 2 * kTile * DP;
  constexpr bool WIDE = ROWS == 64;
  extern __shared__ __align__(1024) uint8_t smem[];
  AttendShared& S = *reinterpret_cast<AttendShared*>(smem + kStages * kStageBytes);
  uint32_t* bits = reinterpret_cast<uint32_t*>(smem + kStages * kStageBytes + sizeof(AttendShared));
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t unit = blockIdx.x / P.splits;
  const Unit u = unit_of(P, ROWS, kTile, unit, static_cast<int>(blockIdx.x - unit * P.splits));
  grid_dependents_launch();
  if (!u.rows || u.split >= u.parts) return;
  const int words = (P.R + 31) >> 5, first_row = u.m0 / P.G;
  if (tid == 0) {
    S.fault = u.fault;
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&S.full[i], 1);
      mbar_init(&S.empty[i], 4);
    }
    fence_mbar_init();
  }
  __syncthreads();
  if (P.parents && !u.fault) {
    ancestor_bits(P, u, (ROWS + P.G - 1) / P.G + 1, words, reinterpret_cast<int32_t*>(bits + ((ROWS + P.G - 1) / P.G + 1) * words), bits, &S.fault, tid, CT);
    __syncthreads();
  }
  const int stop = S.fault ? u.lo : u.hi;   // uniform: nothing is read where the unit is at fault already
  __syncthreads();                          // (the producer may add to it from here on)

  if (warp == 4) {   // ---- producer ----
    produce<kTile, DP, kStages>(P, u, stop, smem, S, &kmap, &vmap, lane);
    __syncthreads();
    return;
  }

  // ---- rows ----
  const int g = lane >> 2, t = lane & 3;
  const int m_warp = u.m0 + (WIDE ? warp * 16 : 0);
  uint32_t qa[KS][TERMS][4];
  float factor[2];
  int row_of[2];   // step row; behind the last: not there
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int m = m_warp + g + 8 * half, r = m / P.G;
    const bool there = r < u.n;
    row_of[half] = there ? r : -1;
    float v[EL];
    const T* p = static_cast<const T*>(P.q) + u.b * P.qs.b + r * P.qs.r + (static_cast<int64_t>(u.h) * P.G + (m - r * P.G)) * P.qs.h;
    float most = 0.0f;
    bool odd = false;
#pragma unroll
    for (int e = 0; e < EL; e += 8) {
      float x[8];
      const int d = t * EL + e;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = 0.0f;
      if (there && d < P.D) {
        if (P.vec) {
          Row<BF16>::get8(p + d, x);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = Row<BF16>::get(p + d + i);
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        odd |= !(fabsf(x[i]) < __int_as_float(0x7f800000));
        most = fmaxf(most, fabsf(x[i]));
        v[e + i] = x[i];
      }
    }
    most = fmaxf(most, __shfl_xor_sync(kFull, most, 1));
    most = fmaxf(most, __shfl_xor_sync(kFull, most, 2));
    odd = __shfl_xor_sync(kFull, odd, 1) | odd;
    odd = __shfl_xor_sync(kFull, odd, 2) | odd;
    // largest component to [2^14, 2^15): the halves of its neighbours lose nothing above 2^-24 of 2^-15 of it
    const int E = static_cast<int>(__float_as_uint(most) >> 23);
    const int up = min(268 - E, 254);   // biased exponent of the multiplier
    const float mult = most == 0.0f || odd ? 0.0f : __uint_as_float(static_cast<uint32_t>(up) << 23);
    factor[half] = odd ? __int_as_float(0x7fffffff) : ldexpf(P.scale_log2, 127 - up);
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int pair = 0; pair < 2; ++pair) {
        const float lo = odd ? 0.0f : v[4 * s + 2 * pair] * mult, hi = odd ? 0.0f : v[4 * s + 2 * pair + 1] * mult;
        const uint32_t w = half2_of(lo, hi);
        qa[s][0][2 * pair + half] = w;
        if constexpr (TERMS == 2) qa[s][1][2 * pair + half] = half2_rest(lo, hi, w);
      }
  }

  float o[NT][4];
#pragma unroll
  for (int i = 0; i < NT; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
  float ref[2] = {-INFINITY, -INFINITY}, sum[2] = {0.0f, 0.0f};   // sum: this lane's columns
  float vref = 0.0f;
  const int warp_last = WIDE ? min(u.n - 1, (m_warp + 15) / P.G) : 0x3fffffff;   // last step row of this warp

  auto step = [&](const uint8_t* keys, const uint8_t* values, int token0, int sb, float ks, float vs) {
    const bool edge = token0 < u.begin || token0 + 16 > u.len + (P.parents ? 0 : first_row + 1);   // some row may not see all of the 16
    float c[2][4];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      c[j][0] = c[j][1] = c[j][2] = c[j][3] = 0.0f;
      const int token = sb * 16 + 8 * j + g;
      uint32_t w[KS];
#pragma unroll
      for (int i = 0; i < KS / 4; ++i) {
        const uint4 x = *reinterpret_cast<const uint4*>(keys + chunk_at<DP>(token, t * (KS / 4) + i));
        w[4 * i] = x.x, w[4 * i + 1] = x.y, w[4 * i + 2] = x.z, w[4 * i + 3] = x.w;
      }
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const uint32_t b0 = decode2(static_cast<uint16_t>(w[s] & 0xffffu)), b1 = decode2(static_cast<uint16_t>(w[s] >> 16));
#pragma unroll
        for (int q = 0; q < TERMS; ++q) mma16816(c[j], qa[s][q], b0, b1);
      }
    }
    uint32_t bad = 0;   // tokens of the 16 with a NaN among their values (looked for where a token may be hidden from a row)
    if (edge) {
      const int token = lane >> 1;
      bool mine = false;
#pragma unroll
      for (int i = 0; i < DP / 32; ++i) {
        const uint4 x = *reinterpret_cast<const uint4*>(values + chunk_at<DP>(sb * 16 + token, (lane & 1) * (DP / 32) + i));
        mine |= ((__vcmpeq4(x.x & 0x7f7f7f7fu, 0x7f7f7f7fu) | __vcmpeq4(x.y & 0x7f7f7f7fu, 0x7f7f7f7fu)) |
                 (__vcmpeq4(x.z & 0x7f7f7f7fu, 0x7f7f7f7fu) | __vcmpeq4(x.w & 0x7f7f7f7fu, 0x7f7f7f7fu))) != 0;
      }
      bad = __ballot_sync(kFull, mine);
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const float f = factor[half] * ks;
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float x = c[j][2 * half + e] * f;
          if (edge) {
            const int at = 8 * j + 2 * t + e, token = token0 + at, r = row_of[half], ahead = token - u.len;
            bool see = r >= 0 && token >= u.begin && token < u.end;
            if (see && ahead >= 0)
              see = P.parents ? (bits[(r - first_row) * words + (ahead >> 5)] >> (ahead & 31)) & 1u : ahead <= r;
            x = see ? x : -INFINITY;
            if (see && (bad >> (2 * at)) & 3u) x = __int_as_float(0x7fffffff);
          }
          c[j][2 * half + e] = x;
        }
    }
    float most[2];
    bool grow = vs > vref * 32.0f;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      float m = fmaxf(fmaxf(c[0][2 * half], c[0][2 * half + 1]), fmaxf(c[1][2 * half], c[1][2 * half + 1]));
      m = fmaxf(m, __shfl_xor_sync(kFull, m, 1));
      m = fmaxf(m, __shfl_xor_sync(kFull, m, 2));
      most[half] = m;
      grow |= m > ref[half] + 8.0f;
    }
    // The maximum that the numerators refer to follows the running maximum only when it has fallen behind by 2^8 (the reference scale of the
    // values: 2^5), so that the accumulators are rarely touched; a numerator stays below 2^8 * 2^5, a half's largest value is 2^16.
    if (__any_sync(kFull, grow)) {
      const float v_new = fmaxf(vref, vs), v_ratio = v_new > 0.0f ? vref / v_new : 0.0f;
      float w[2];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const float m = fmaxf(ref[half], most[half]);
        const float k = ref[half] == -INFINITY ? 0.0f : ex2_approx(ref[half] - m);
        ref[half] = m;
        sum[half] *= k;
        w[half] = k * v_ratio;
      }
      vref = v_new;
#pragma unroll
      for (int i = 0; i < NT; ++i) o[i][0] *= w[0], o[i][1] *= w[0], o[i][2] *= w[1], o[i][3] *= w[1];
    }
    const float vr = vref > 0.0f ? vs / vref : 0.0f;   // (a scale of zero: a block of zeros)
    uint32_t pa[TERMS][4];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const float base = ref[half] == -INFINITY ? 0.0f : ref[half];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float p0 = ex2_approx(c[j][2 * half] - base), p1 = ex2_approx(c[j][2 * half + 1] - base);
        sum[half] += p0 + p1;
        p0 *= vr, p1 *= vr;
        const uint32_t w = half2_of(p0, p1);
        pa[0][2 * j + half] = w;
        if constexpr (TERMS == 2) pa[1][2 * j + half] = half2_rest(p0, p1, w);
      }
    }
    const int v0 = sb * 16 + 2 * t;
    constexpr int VW = DP / 32;   // words of values per token that a lane takes: DP / 8 components from g * DP / 8 on
    uint32_t x[4][VW];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int token = v0 + (i & 1) + (i >> 1) * 8;
      if constexpr (DP == 128) {
        const uint4 y = *reinterpret_cast<const uint4*>(values + chunk_at<DP>(token, g));
        x[i][0] = y.x, x[i][1] = y.y, x[i][2] = y.z, x[i][3] = y.w;
      } else {
        const uint2 y = *reinterpret_cast<const uint2*>(values + chunk_at<DP>(token, g >> 1) + (g & 1) * 8);
        x[i][0] = y.x, x[i][1] = y.y;
      }
    }
    if (bad) {   // (uniform)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int w = 0; w < VW; ++w) x[i][w] = without_nan(x[i][w]);
    }
#pragma unroll
    for (int w = 0; w < VW; ++w) {
      const uint32_t a = __byte_perm(x[0][w], x[1][w], 0x5140), b = __byte_perm(x[0][w], x[1][w], 0x7362);
      const uint32_t d = __byte_perm(x[2][w], x[3][w], 0x5140), e = __byte_perm(x[2][w], x[3][w], 0x7362);
      const uint32_t first[4] = {a & 0xffffu, a >> 16, b & 0xffffu, b >> 16}, second[4] = {d & 0xffffu, d >> 16, e & 0xffffu, e >> 16};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t b0 = decode2(static_cast<uint16_t>(first[i])), b1 = decode2(static_cast<uint16_t>(second[i]));
#pragma unroll
        for (int q = 0; q < TERMS; ++q) mma16816(o[4 * w + i], pa[q], b0, b1);
      }
    }
  };

  int it = 0;
  for (int tile = u.lo; tile < stop; ++tile, ++it) {
    const int stage = it % kStages;
    if (!__all_sync(kFull, await(&S.full[stage], (it / kStages) & 1))) {
      if (lane == 0) atomicOr(&S.fault, LANTERN_ST_INTERNAL);
      break;
    }
    const uint8_t* keys = smem + stage * kStageBytes;
#pragma unroll 1
    for (int sb = WIDE ? 0 : warp; sb < (WIDE ? 4 : warp + 1); ++sb) {
      const int token0 = (u.tile0 + tile) * kTile + sb * 16;
      if (token0 >= u.end || token0 + 16 <= u.begin || token0 > u.len + warp_last) continue;
      step(keys, keys + kTile * DP, token0, sb, S.scale[stage][0][sb], S.scale[stage][1][sb]);
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(&S.empty[stage]);
  }
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    sum[half] += __shfl_xor_sync(kFull, sum[half], 1);
    sum[half] += __shfl_xor_sync(kFull, sum[half], 2);
  }
  __syncthreads();   // the producer is through as well: faults are known, stages are free
  const int fault = S.fault;
  if (fault && tid == 0 && P.status) atomicOr(P.status + u.b, fault);

  float L[2], w[2];   // sum and the factor of this warp's accumulators, relative to the unit's maximum
  if constexpr (WIDE) {
#pragma unroll
    for (int half = 0; half < 2; ++half) L[half] = sum[half], w[half] = vref;
  } else {
    if (t == 0)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        S.ml[warp][g + 8 * half][0] = ref[half];
        S.ml[warp][g + 8 * half][1] = sum[half];
      }
    asm volatile("bar.sync 1, 128;" ::: "memory");
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      float M = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i) M = fmaxf(M, S.ml[i][g + 8 * half][0]);
      const float base = M == -INFINITY ? 0.0f : M;
      L[half] = 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) L[half] += S.ml[i][g + 8 * half][1] * ex2_approx(S.ml[i][g + 8 * half][0] - base);
      w[half] = vref * ex2_approx(ref[half] - base);
      ref[half] = M;
    }
    // the four warps' accumulators meet in shared memory: [warp][row][DP + 4]
    float* buf = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int i = 0; i < NT; i += 4)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          *reinterpret_cast<float4*>(buf + (warp * 16 + g + 8 * half) * (DP + 4) + t * EL + e * NT + i) =
              make_float4(o[i][2 * half + e] * w[half], o[i + 1][2 * half + e] * w[half], o[i + 2][2 * half + e] * w[half], o[i + 3][2 * half + e] * w[half]);
    asm volatile("bar.sync 1, 128;" ::: "memory");
    // warp i writes components [i DP/4, (i+1) DP/4) of every row: its lanes keep rows g, g + 8 and DP / 16 components from t DP/16 on
  }
  const bool whole = u.parts == 1;
  const int64_t part = (unit * P.splits + u.split) * ROWS;
  constexpr int OUT = WIDE ? EL : EL / 4;   // components per lane and row
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int row = (WIDE ? warp * 16 : 0) + g + 8 * half, r = row_of[half];
    if (r < 0) continue;
    const int d0 = WIDE ? t * EL : warp * EL + t * OUT;
    float v[OUT];
    if constexpr (WIDE) {
#pragma unroll
      for (int i = 0; i < NT; ++i) v[i] = o[i][2 * half] * w[half], v[NT + i] = o[i][2 * half + 1] * w[half];
    } else {
      const float* buf = reinterpret_cast<const float*>(smem);
#pragma unroll
      for (int i = 0; i < OUT; ++i) {
        v[i] = 0.0f;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[i] += buf[(k * 16 + row) * (DP + 4) + d0 + i];
      }
    }
    if (whole) {
      const float inv = fault ? __int_as_float(0x7fffffff) : (L[half] == 0.0f ? 0.0f : 1.0f / L[half]);
      const int m = u.m0 + row;
      T* out = static_cast<T*>(P.out) + ((static_cast<int64_t>(u.b) * P.R + r) * P.q_heads + u.h * P.G + (m - r * P.G)) * P.D;
#pragma unroll
      for (int i = 0; i < OUT; i += 4)
        if (d0 + i < P.D) {
          if constexpr (BF16) *reinterpret_cast<uint2*>(out + d0 + i) = make_uint2(bf16x2_round(v[i] * inv, v[i + 1] * inv), bf16x2_round(v[i + 2] * inv, v[i + 3] * inv));
          else *reinterpret_cast<float4*>(out + d0 + i) = make_float4(v[i] * inv, v[i + 1] * inv, v[i + 2] * inv, v[i + 3] * inv);
        }
    } else {
#pragma unroll
      for (int i = 0; i < OUT; i += 4)
        if (d0 + i < P.D) *reinterpret_cast<float4*>(P.parts + (part + row) * DP + d0 + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
      if (d0 == 0) P.part_ml[part + row] = make_float2(ref[half], fault ? __int_as_float(0x7fffffff) : L[half]);
    }
  }
}

// ---- host ---------------------------------------------------------------------------------------------------------------

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static EncodeFn encode_fn() {
  static const EncodeFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeFn>(p);
  }();
  return fn;
}
lantern_status code_map(CUtensorMap* map, const void* code, const lantern_cache* c, int DP, int tokens) {
  const EncodeFn fn = encode_fn();
  if (!fn) return LANTERN_E_CUDA;
  const cuuint64_t rows = static_cast<cuuint64_t>(c->heads) * c->page_tokens, D = c->head_dim;
  const cuuint64_t dims[3] = {D, rows, static_cast<cuuint64_t>(c->pages)}, strides[2] = {D, D * rows};
  const cuuint32_t box[3] = {static_cast<cuuint32_t>(DP), static_cast<cuuint32_t>(tokens), 1}, step[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(code), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
            DP == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? LANTERN_OK
             : LANTERN_E_CUDA;
}

static Division divide(int B, int R, int q_heads, const lantern_cache* c, int width) {
  Division d;
  const int64_t G = q_heads / c->heads, M = G * R;
  d.DP = c->head_dim <= 64 ? 64 : 128;
  d.rows = M <= 16 ? 16 : M <= 64 ? 64 : 128;
  d.tile = d.rows > 16 && d.DP == 128 ? 128 : kTile;
  d.row_tiles = static_cast<int>((M + d.rows - 1) / d.rows);
  d.units = static_cast<int64_t>(B) * c->heads * d.row_tiles;
  const int64_t slots = 148 * 2, tiles = (static_cast<int64_t>(width) * c->page_tokens + d.tile - 1) / d.tile;
  d.least = 2;
  int64_t splits = d.units >= slots ? 1 : (2 * slots + d.units - 1) / (d.units > 0 ? d.units : 1);
  if (splits > tiles / d.least) splits = tiles / d.least;
  d.splits = static_cast<int>(splits < 1 ? 1 : splits > 128 ? 128 : splits);
  return d;
}
static size_t parts_bytes(const Division& d) {
  return d.splits == 1 ? 0 : static_cast<size_t>(d.units) * d.splits * d.rows * (d.DP * sizeof(float) + sizeof(float2));
}
static lantern_status check_attention(int dtype, int B, int R, int q_heads, const lantern_cache* c, int width, bool tree) {
  if (dtype != LANTERN_F32 && dtype != LANTERN_BF16) return LANTERN_E_PARAM;
  if (B < 0 || R < 0 || q_heads < 1 || q_heads % c->heads != 0 || (tree && R > kMaxTreeRows)) return LANTERN_E_SHAPE;
  if (static_cast<int64_t>(R) * (q_heads / c->heads) > INT32_MAX / 2 || static_cast<int64_t>(B) * R > INT32_MAX) return LANTERN_E_SHAPE;
  const Division d = divide(B, R, q_heads, c, width);
  if (d.units * (d.splits > 16 ? d.splits : 16) > INT32_MAX) return LANTERN_E_SHAPE;
  return LANTERN_OK;
}

template <int ROWS, int DP, bool BF16>
static cudaError_t launch_attention(const AttendParams& P, const CUtensorMap& k, const CUtensorMap& v, const Division& d, cudaStream_t st) {
  constexpr size_t kFixed = kStages * 2 * kTile * DP + sizeof(AttendShared);
  const size_t words = (P.R + 31) / 32, rows = (ROWS + P.G - 1) / P.G + 1;
  const size_t smem = kFixed + (P.parents ? (rows * words + P.R) * 4 : 0);
  static DeviceFlags ready;
  cudaError_t e = allow_shared_memory(lantern_attention_kernel<ROWS, DP, BF16>, kFixed + ((ROWS + 1) * 33 + kMaxTreeRows) * 4, ready);
  if (e != cudaSuccess) return e;
  lantern_attention_kernel<ROWS, DP, BF16><<<static_cast<unsigned>(d.units * d.splits), CT, smem, st>>>(P, k, v);
  if ((e = cudaGetLastError()) != cudaSuccess || d.splits == 1) return e;
  return launch_join<DP, BF16>(P, d, st);
}

}  // namespace lantern

using namespace lantern;

extern "C" size_t lantern_cache_attention_workspace_bytes(int dtype, int B, int R, int q_heads, const lantern_cache* cache, int table_width) {
  if (!cache || check_cache(cache, nullptr, table_width, 0) != LANTERN_OK) return 0;
  if (check_attention(dtype, B, R, q_heads, cache, table_width, false) != LANTERN_OK || B == 0 || R == 0) return 0;
  return parts_bytes(divide(B, R, q_heads, cache, table_width));
}

extern "C" lantern_status lantern_cache_attention(const void* q, void* out, int dtype, int B, int R, int q_heads, const int64_t q_stride[3],
                                                  const lantern_cache* cache, const int32_t* table, int table_width, const int32_t* lengths,
                                                  const int32_t* counts, const int32_t* starts, const int32_t* tree_parents, float scale,
                                                  int32_t* status, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  lantern_status bad = check_cache(cache, table, table_width, B);
  if (bad != LANTERN_OK) return bad;
  if ((bad = check_attention(dtype, B, R, q_heads, cache, table_width, tree_parents != nullptr)) != LANTERN_OK) return bad;
  if (!isfinite(scale)) return LANTERN_E_PARAM;
  if (B == 0 || R == 0) return LANTERN_OK;
  if (!q || !out || !q_stride || !lengths) return LANTERN_E_NULL;
  const bool bf = dtype == LANTERN_BF16;
  const int size = bf ? 2 : 4;
  if (reinterpret_cast<uintptr_t>(q) % size || (reinterpret_cast<uintptr_t>(out) & 15)) return LANTERN_E_ALIGN;
  const Division d = divide(B, R, q_heads, cache, table_width);
  const size_t need = parts_bytes(d);
  if (need && (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 255))) return LANTERN_E_WORKSPACE;
  AttendParams P;
  P.q = q;
  P.out = out;
  P.qs = {q_stride[0], q_stride[1], q_stride[2]};
  P.k_scale = cache->k_scale;
  P.v_scale = cache->v_scale;
  P.table = table;
  P.lengths = lengths;
  P.counts = counts;
  P.starts = starts;
  P.parents = R > 1 ? tree_parents : nullptr;   // (a single row is its own root)
  P.status = status;
  P.parts = static_cast<float*>(workspace);
  P.part_ml = reinterpret_cast<float2*>(P.parts + static_cast<size_t>(d.units) * d.splits * d.rows * d.DP);
  P.B = B;
  P.R = R;
  P.q_heads = q_heads;
  P.heads = cache->heads;
  P.G = q_heads / cache->heads;
  P.S = cache->page_tokens;
  P.D = cache->head_dim;
  P.width = table_width;
  P.pages = cache->pages;
  P.row_tiles = d.row_tiles;
  P.splits = d.splits;
  P.least = d.least;
  const int64_t qs[3] = {q_stride[0], q_stride[1], q_stride[2]};
  P.vec = aligned16(q, qs, size);
  P.scale_log2 = scale * 1.44269504088896340736f;
  CUtensorMap km, vm;
  const int tokens = P.S < d.tile ? P.S : d.tile;
  if ((bad = code_map(&km, cache->k_code, cache, d.DP, tokens)) != LANTERN_OK || (bad = code_map(&vm, cache->v_code, cache, d.DP, tokens)) != LANTERN_OK) return bad;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e;
  if (d.rows > 16) e = launch_attention_wide(P, km, vm, d, bf, st);
  else if (d.DP == 64) e = bf ? launch_attention<16, 64, true>(P, km, vm, d, st) : launch_attention<16, 64, false>(P, km, vm, d, st);
  else e = bf ? launch_attention<16, 128, true>(P, km, vm, d, st) : launch_attention<16, 128, false>(P, km, vm, d, st);
  return e == cudaSuccess ? LANTERN_OK : LANTERN_E_CUDA;
}
