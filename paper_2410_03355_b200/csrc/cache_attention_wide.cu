// Attention of many rows (draft trees, chunks of prompts, grouped heads) to the paged 8-bit cache, on the fifth-generation tensor cores.
//
//   out = sum_c p_c v_c / sum_c p_c,   p_c = 2^(x_c - max x),   x_c = scale log2(e) k_scale (q . k_c)
//
// A CTA takes 128 rows of one sequence and cache head and a part of the tokens:
//   - a producer warp copies a tile of codes per stage (TMA, block by block through the table);
//   - four warps turn codes into halves (every e4m3 value is one) in the layout that the products read, values times their scale over the part's
//     largest (a power of two: exact);
//   - one thread issues scores = queries . keys and output += probabilities . values, 128 rows wide, queries and probabilities out of tensor
//     memory, one tile of scores ahead of the softmax;
//   - four warps, a thread per row, take the scores from tensor memory, keep the row's running maximum and sum and put the probabilities
//     in the scores' place as halves.
// Queries go in as halves after a power of two of their own (8 bits of a bf16 query fit); fp32 queries and probabilities as two halves each
// (22 bits), in products of their own.  Accumulators are fp32.
// With at most 64 rows the second half of the 128 holds the same rows again and takes the second half of every tile's tokens (a part of its
// own, joined at the end), so that all four warps have work.
#include "cache_attention.cuh"

namespace lantern {

namespace {

constexpr int kThreads = 320;   // softmax warps 0..3, converting warps 4..7, producer 8, products 9

template <int DP>
struct Shape {
  static constexpr int kTile = DP == 64 ? 64 : 128;
  static constexpr int kStages = DP == 64 ? 3 : 2;
  static constexpr int kColumns = DP == 64 ? 256 : 512;                  // of tensor memory; two CTAs per SM with 256
  static constexpr int kScores = 0, kOutput = 2 * kTile, kQuery = kOutput + DP;   // columns: two tiles of scores, the output, queries
  static constexpr int kRaw = 2 * kTile * DP, kHalves = kTile * DP * 2;   // bytes of a stage; of one tile of keys or of values as halves
  static constexpr int kBytes = kStages * kRaw + 4 * kHalves;
};

template <int DP>
struct WideShared : StageShared<Shape<DP>::kTile, Shape<DP>::kStages> {
  uint64_t keys_full[2], keys_free[2], values_full[2], values_free[2], scores_full[2], probs_full[2], query_full;
  float key_scale[4][Shape<DP>::kTile / 16];
  uint32_t bad[4][4];     // tokens with a NaN among their values, by converting warp
  float2 ml[64];
  uint32_t tmem;
  int vmax;               // largest value scale of the part, as the bits of a float
};

// ---- tensor memory and products -----------------------------------------------------------------------------------------
__device__ __forceinline__ void tmem_ld32(uint32_t (&r)[32], uint32_t at) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, "
      "%22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
      "tcgen05.wait::ld.sync.aligned;"   // (in one statement: nothing may use the registers in between)
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
        "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]),
        "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(at)
      : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t at, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, "
      "%22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(at),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
      "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]),
      "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(at), "r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]),
      "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Descriptor of 64 components by n tokens of halves, 128-byte rows swizzled: rows of 8 tokens are 1024 bytes apart, runs of 64 components `run` bytes.
__device__ __forceinline__ uint64_t halves_at(uint32_t address, uint32_t run) {
  return static_cast<uint64_t>((address >> 4) & 0x3fffu) | (static_cast<uint64_t>((run >> 4) & 0x3fffu) << 16) | (static_cast<uint64_t>(1024 >> 4) << 32) |
         (1ull << 46) | (2ull << 61);
}
// 128 rows by `columns`, halves, fp32 accumulators; the second operand with its rows along the product's axis (keys) or across it (values)
__host__ __device__ constexpr uint32_t product(int columns, bool across) {
  return (1u << 4) | (across ? 1u << 16 : 0u) | (static_cast<uint32_t>(columns >> 3) << 17) | ((128u >> 4) << 24);
}
__device__ __forceinline__ void multiply(uint32_t d, uint32_t a, uint64_t b, uint32_t form, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(form), "r"(static_cast<uint32_t>(add))
      : "memory");
}
__device__ __forceinline__ void commit(uint64_t* bar) {   // arrives when the products issued so far are done
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
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
__device__ __forceinline__ bool has_nan(uint4 x) {
  return ((__vcmpeq4(x.x & 0x7f7f7f7fu, 0x7f7f7f7fu) | __vcmpeq4(x.y & 0x7f7f7f7fu, 0x7f7f7f7fu)) |
          (__vcmpeq4(x.z & 0x7f7f7f7fu, 0x7f7f7f7fu) | __vcmpeq4(x.w & 0x7f7f7f7fu, 0x7f7f7f7fu))) != 0;
}
__device__ __forceinline__ uint32_t times(uint32_t halves, __half2 ratio) {
  const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&halves), ratio);
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }

template <int DP, bool BF16>
__global__ void __launch_bounds__(kThreads, DP == 64 ? 2 : 1) lantern_attention_wide_kernel(AttendParams P, int unit_rows, const __grid_constant__ CUtensorMap kmap,
                                                                                         const __grid_constant__ CUtensorMap vmap) {
  using T = typename Row<BF16>::T;
  using C = Shape<DP>;
  constexpr int TILE = C::kTile, STAGES = C::kStages;
  constexpr int TERMS = BF16 ? 1 : 2;
  constexpr int RUN = TILE * 128;   // bytes of 64 components of a tile of halves
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t* halves = smem + STAGES * C::kRaw;   // [2][keys, values]
  WideShared<DP>& S = *reinterpret_cast<WideShared<DP>*>(smem + C::kBytes);
  uint32_t* bits = reinterpret_cast<uint32_t*>(smem + C::kBytes + sizeof(WideShared<DP>));
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t unit = blockIdx.x / P.splits;
  const Unit u = unit_of(P, unit_rows, TILE, unit, static_cast<int>(blockIdx.x - unit * P.splits));
  grid_dependents_launch();
  if (!u.rows || u.split >= u.parts) return;
  const int words = (P.R + 31) >> 5, first_row = u.m0 / P.G, table_rows = (unit_rows + P.G - 1) / P.G + 1;
  if (tid == 0) {
    S.fault = u.fault;
    S.vmax = 0;
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(&S.full[i], 1);
      mbar_init(&S.empty[i], 4);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&S.keys_full[i], 4);
      mbar_init(&S.keys_free[i], 1);
      mbar_init(&S.values_full[i], 4);
      mbar_init(&S.values_free[i], 1);
      mbar_init(&S.scores_full[i], 2);
      mbar_init(&S.probs_full[i], 4);
    }
    mbar_init(&S.query_full, 4);
    fence_mbar_init();
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&S.tmem)), "r"(C::kColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const uint32_t tmem = S.tmem;
  if (P.parents && !u.fault) {
    ancestor_bits(P, u, table_rows, words, reinterpret_cast<int32_t*>(bits + table_rows * words), bits, &S.fault, tid, kThreads);
    __syncthreads();
  }
  const int stop = S.fault ? u.lo : u.hi;   // uniform: nothing is read where the unit is at fault already
  {   // the largest value scale of the part
    const int sub = min(P.S, TILE), boxes = (stop - u.lo) * (TILE / sub);
    float most = 0.0f;
    for (int i = tid; i < boxes; i += kThreads) {
      const int64_t token = static_cast<int64_t>(u.tile0 + u.lo) * TILE + static_cast<int64_t>(i) * sub;
      if (token < u.end && token + sub > u.begin) {
        const int page = __ldg(P.table + static_cast<int64_t>(u.b) * P.width + token / P.S);
        if (page >= 0 && page < P.pages) most = fmaxf(most, __ldg(P.v_scale + static_cast<int64_t>(page) * P.heads + u.h));
      }
    }
    __syncthreads();   // (the producer may add to the faults from here on)
    if (most > 0.0f) atomicMax(&S.vmax, __float_as_int(most));
  }
  __syncthreads();
  const float vref = __int_as_float(S.vmax);
  const int tiles = stop - u.lo;

  if (warp == 8) {   // ---- producer ----
    produce<TILE, DP, STAGES>(P, u, stop, smem, S, &kmap, &vmap, lane);
  } else if (warp == 9) {   // ---- products ----
    if (lane == 0 && tiles > 0) {
      bool ok = await(&S.query_full, 0);
      tmem_fence_after();
      const uint32_t base = smem_addr(halves);
      auto scores = [&](int i) {
        const int k = i & 1;
        ok = ok && await(&S.keys_full[k], (i >> 1) & 1);
        tmem_fence_after();
#pragma unroll
        for (int s = 0; s < DP / 16; ++s)
#pragma unroll
          for (int q = 0; q < TERMS; ++q)
            multiply(tmem + C::kScores + k * TILE, tmem + C::kQuery + q * (DP / 2) + s * 8,
                     halves_at(base + k * 2 * C::kHalves + (s >> 2) * RUN + (s & 3) * 32, RUN), product(TILE, false), s + q > 0);
        commit(&S.scores_full[k]);
        commit(&S.keys_free[k]);
        mbar_arrive(&S.scores_full[k]);   // (what the converting warps wrote beside the keys is ordered by this arrival)
      };
      scores(0);
      for (int i = 0; i < tiles && ok; ++i) {
        const int k = i & 1;
        if (i + 1 < tiles) scores(i + 1);
        ok = ok && await(&S.probs_full[k], (i >> 1) & 1) && await(&S.values_full[k], (i >> 1) & 1);
        tmem_fence_after();
#pragma unroll
        for (int s = 0; s < TILE / 16; ++s)
#pragma unroll
          for (int q = 0; q < TERMS; ++q)
            multiply(tmem + C::kOutput, tmem + C::kScores + k * TILE + (s >> 1) * 32 + (s & 1) * 8 + q * 16,
                     halves_at(base + (k * 2 + 1) * C::kHalves + s * 2048, RUN), product(DP, true), i > 0 || s + q > 0);
        commit(&S.values_free[k]);
      }
      if (!ok) atomicOr(&S.fault, LANTERN_ST_INTERNAL);
    }
    __syncwarp();
  } else if (warp >= 4) {   // ---- codes to halves ----
    // a thread per token, two where a tile has 64 of them: 16 components at a time
    constexpr int SHARE = 128 / TILE, CHUNKS = DP / 16 / SHARE;
    const int who = tid - 128, token = who % TILE, share = who / TILE, w = warp - 4;
    bool ok = true;
    for (int i = 0; i < tiles && ok; ++i) {
      const int k = i & 1, stage = i % STAGES, round = i >> 1, at = i & 3;
      ok = await(&S.full[stage], (i / STAGES) & 1);
      const int token0 = (u.tile0 + u.lo + i) * TILE;
      const bool edge = token0 < u.begin || token0 + TILE > u.len + (P.parents ? 0 : first_row + 1);
      const uint8_t* raw = smem + stage * C::kRaw;
      if (share == 0 && (token & 15) == 0) S.key_scale[at][token >> 4] = S.scale[stage][0][token >> 4];
      const float vs = S.scale[stage][1][token >> 4];
      const __half2 ratio = __float2half2_rn(vref > 0.0f ? vs / vref : 0.0f);
      bool nan = false;
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        if (i >= 2) ok = ok && await(which ? &S.values_free[k] : &S.keys_free[k], (round - 1) & 1);
        uint8_t* out = halves + (k * 2 + which) * C::kHalves;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
          const int chunk = share * CHUNKS + c;
          uint4 x = *reinterpret_cast<const uint4*>(raw + which * TILE * DP + chunk_at<DP>(token, chunk));
          if (which == 1 && edge) {   // where a token may be hidden from a row its NaN must not reach the row through a zero probability
            nan |= has_nan(x);
            x.x = without_nan(x.x), x.y = without_nan(x.y), x.z = without_nan(x.z), x.w = without_nan(x.w);
          }
          const uint32_t in[4] = {x.x, x.y, x.z, x.w};
          uint32_t h[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            h[2 * e] = decode2(static_cast<uint16_t>(in[e] & 0xffffu));
            h[2 * e + 1] = decode2(static_cast<uint16_t>(in[e] >> 16));
          }
          if (which == 1)
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] = times(h[e], ratio);
          uint8_t* row = out + (chunk >> 2) * RUN + token * 128;
          const int p = (chunk & 3) * 2;
          *reinterpret_cast<uint4*>(row + (((p) ^ (token & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
          *reinterpret_cast<uint4*>(row + (((p + 1) ^ (token & 7)) << 4)) = make_uint4(h[4], h[5], h[6], h[7]);
        }
        if (which == 1) {
          const uint32_t found = __ballot_sync(kFull, nan);
          if (lane == 0) S.bad[at][w] = found;
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(which ? &S.values_full[k] : &S.keys_full[k]);
      }
      if (lane == 0) mbar_arrive(&S.empty[stage]);
      ok = __all_sync(kFull, ok);
    }
    if (!ok && lane == 0) atomicOr(&S.fault, LANTERN_ST_INTERNAL);
  }

  // ---- softmax: a thread per row ----
  float ref = -INFINITY, sum = 0.0f;
  const bool twice = unit_rows == 64;
  const int row = twice ? tid & 63 : tid & 127, group = twice ? (tid >> 6) & 1 : 0;
  const int m = u.m0 + row, r = m / P.G;
  const bool there = r < u.n;
  const uint32_t lanes = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
  if (warp < 4 && tiles > 0) {
    const T* p = static_cast<const T*>(P.q) + u.b * P.qs.b + r * P.qs.r + (static_cast<int64_t>(u.h) * P.G + (m - r * P.G)) * P.qs.h;
    float most = 0.0f, factor;
    bool odd = false;
    auto components = [&](int d, float (&x)[8]) {
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
    };
#pragma unroll 4
    for (int d = 0; d < DP; d += 8) {
      float x[8];
      components(d, x);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        odd |= !(fabsf(x[i]) < __int_as_float(0x7f800000));
        most = fmaxf(most, fabsf(x[i]));
      }
    }
    // largest component to [2^14, 2^15); the scale's sign goes with the query, so that factors are positive
    const int up = min(268 - static_cast<int>(__float_as_uint(most) >> 23), 254);   // biased exponent of the multiplier
    float mult = most == 0.0f || odd || P.scale_log2 == 0.0f ? 0.0f : __uint_as_float(static_cast<uint32_t>(up) << 23);
    if (P.scale_log2 < 0.0f) mult = -mult;
    factor = odd ? __int_as_float(0x7fffffff) : ldexpf(fabsf(P.scale_log2), 127 - up);
#pragma unroll
    for (int d0 = 0; d0 < DP; d0 += 32) {
      uint32_t h[16], l[16];
#pragma unroll
      for (int e = 0; e < 32; e += 8) {
        float x[8];
        components(d0 + e, x);
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          const float a = odd ? 0.0f : x[i] * mult, b = odd ? 0.0f : x[i + 1] * mult;
          h[(e + i) / 2] = half2_of(a, b);
          l[(e + i) / 2] = half2_rest(a, b, h[(e + i) / 2]);
        }
      }
      tmem_st16(lanes + C::kQuery + d0 / 2, h);
      if constexpr (TERMS == 2) tmem_st16(lanes + C::kQuery + DP / 2 + d0 / 2, l);
    }
    tmem_st_wait();
    tmem_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(&S.query_full);

    constexpr int CH = TILE / 32;   // runs of 32 tokens
    const int c0 = group * (CH / 2), c1 = twice ? c0 + CH / 2 : CH;   // those of this thread
    const uint32_t* mine = bits + (there ? r - first_row : 0) * words;
    bool ok = true;
    for (int i = 0; i < tiles && ok; ++i) {
      const int k = i & 1;
      ok = await(&S.scores_full[k], (i >> 1) & 1);
      __syncwarp();
      const int token0 = (u.tile0 + u.lo + i) * TILE;
      const bool edge = token0 < u.begin || token0 + TILE > u.len + (P.parents ? 0 : first_row + 1);
      uint32_t see[CH], nan[CH];
      if (edge) {
        ok = ok && await(&S.values_full[k], (i >> 1) & 1);
        __syncwarp();
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          const int a = token0 + 32 * c, ahead = a - u.len;
          nan[c] = TILE == 64 ? S.bad[i & 3][c] | S.bad[i & 3][c + 2] : S.bad[i & 3][c];
          uint32_t v = low_bits(-ahead + (P.parents ? 0 : r + 1));
          if (P.parents) {
            if (ahead >= 0) {
              const int w = ahead >> 5;
              const uint32_t lo = w < words ? mine[w] : 0u, hi = w + 1 < words ? mine[w + 1] : 0u;
              v |= __funnelshift_r(lo, hi, ahead & 31);
            } else if (ahead > -32) {
              v |= mine[0] << -ahead;
            }
          }
          v &= ~low_bits(u.begin - a);
          see[c] = there ? v : 0u;
        }
      }
      tmem_fence_after();
      float f[2 * CH];
#pragma unroll
      for (int c = 0; c < 2 * CH; ++c) {
        f[c] = factor * S.key_scale[i & 3][c];
        if (f[c] < 1.17549435e-38f) f[c] = 1.17549435e-38f;   // (not zero: a hidden token stays at minus infinity)
      }
      const uint32_t scores = lanes + C::kScores + k * TILE;
      float top = -INFINITY;
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        if (c < c0 || c >= c1) continue;
        uint32_t x[32];
        tmem_ld32(x, scores + 32 * c);
        if (edge) {
#pragma unroll
          for (int e = 0; e < 32; ++e) x[e] = (see[c] >> e) & 1u ? x[e] : 0xff800000u;
        }
        float a = -INFINITY, b = -INFINITY;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          a = fmaxf(a, __uint_as_float(x[e]));
          b = fmaxf(b, __uint_as_float(x[16 + e]));
        }
        top = fmaxf(top, fmaxf(a * f[2 * c], b * f[2 * c + 1]));
      }
      // The maximum that the probabilities refer to follows the running maximum only when it has fallen behind by 2^8 (a half holds 2^16), so
      // that the accumulators are rarely touched.
      if (__any_sync(kFull, top > ref + 8.0f)) {
        const float to = fmaxf(ref, top), w = ref == -INFINITY ? 0.0f : ex2_approx(ref - to);
        ref = to;
        sum *= w;
        if (i > 0) {
          ok = ok && await(&S.values_free[(i - 1) & 1], ((i - 1) >> 1) & 1);
          __syncwarp();
          tmem_fence_after();
#pragma unroll
          for (int c = 0; c < DP / 32; ++c) {
            uint32_t x[32];
            tmem_ld32(x, lanes + C::kOutput + 32 * c);
#pragma unroll
            for (int e = 0; e < 32; ++e) x[e] = __float_as_uint(__uint_as_float(x[e]) * w);
            tmem_st32(lanes + C::kOutput + 32 * c, x);
          }
        }
      }
      const float base = ref == -INFINITY ? 0.0f : ref;
      float part = 0.0f;
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        uint32_t h[16], l[16];
        if (c < c0 || c >= c1) {
#pragma unroll
          for (int e = 0; e < 16; ++e) h[e] = l[e] = 0u;
        } else {
          uint32_t x[32];
          tmem_ld32(x, scores + 32 * c);
          if (edge) {
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              x[e] = (see[c] >> e) & 1u ? x[e] : 0xff800000u;
              if ((see[c] & nan[c]) >> e & 1u) x[e] = 0x7fffffffu;
            }
          }
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const float ff = f[2 * c + (e >> 4)];
            const float a = ex2_approx(__fmaf_rn(__uint_as_float(x[e]), ff, -base)), b = ex2_approx(__fmaf_rn(__uint_as_float(x[e + 1]), ff, -base));
            part += a + b;
            h[e / 2] = half2_of(a, b);
            if constexpr (TERMS == 2) l[e / 2] = half2_rest(a, b, h[e / 2]);
          }
        }
        tmem_st16(scores + 32 * c, h);
        if constexpr (TERMS == 2) tmem_st16(scores + 32 * c + 16, l);
      }
      sum += part;
      tmem_st_wait();
      tmem_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&S.probs_full[k]);
      ok = __all_sync(kFull, ok);
    }
    ok = ok && await(&S.values_free[(tiles - 1) & 1], ((tiles - 1) >> 1) & 1);
    __syncwarp();
    tmem_fence_after();
    if (!ok && lane == 0) atomicOr(&S.fault, LANTERN_ST_INTERNAL);
  }
  tmem_fence_before();
  __syncthreads();   // everybody is through: faults are known, shared memory is free
  tmem_fence_after();
  const int fault = S.fault;
  if (fault && tid == 0 && P.status) atomicOr(P.status + u.b, fault);

  if (warp < 4) {
    const bool whole = u.parts == 1;
    float mine = 1.0f, theirs = 0.0f;   // weights of this half's accumulators and of the other's
    float L = sum;
    float* buf = reinterpret_cast<float*>(smem);   // [64][DP + 4]: the second half's accumulators
    if (twice) {
      if (group == 1) {
        S.ml[row] = make_float2(ref, sum);
#pragma unroll
        for (int c = 0; c < DP / 32; ++c) {
          uint32_t x[32];
          if (tiles > 0) tmem_ld32(x, lanes + C::kOutput + 32 * c);
#pragma unroll
          for (int e = 0; e < 32; e += 4)
            *reinterpret_cast<float4*>(buf + row * (DP + 4) + 32 * c + e) =
                tiles > 0 ? make_float4(__uint_as_float(x[e]), __uint_as_float(x[e + 1]), __uint_as_float(x[e + 2]), __uint_as_float(x[e + 3]))
                          : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
      }
      asm volatile("bar.sync 1, 128;" ::: "memory");
      const float2 other = S.ml[row];
      const float M = fmaxf(ref, other.x), base = M == -INFINITY ? 0.0f : M;
      mine = ex2_approx(ref - base), theirs = ex2_approx(other.x - base);
      L = sum * mine + other.y * theirs;
      ref = M;
    }
    if (group == 0) {
      const float inv = fault ? __int_as_float(0x7fffffff) : (L == 0.0f ? 0.0f : 1.0f / L);
      const float scale = whole ? vref * inv : vref;
      const int64_t part = (unit * P.splits + u.split) * unit_rows + row;
      T* out = static_cast<T*>(P.out) + ((static_cast<int64_t>(u.b) * P.R + r) * P.q_heads + u.h * P.G + (m - r * P.G)) * P.D;
      float* to = P.parts + part * DP;
#pragma unroll
      for (int c = 0; c < DP / 32; ++c) {
        uint32_t x[32];
        if (tiles > 0) tmem_ld32(x, lanes + C::kOutput + 32 * c);
#pragma unroll
        for (int e = 0; e < 32; e += 8) {
          float v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            v[i] = tiles > 0 ? __uint_as_float(x[e + i]) * mine : 0.0f;
            if (twice) v[i] += buf[row * (DP + 4) + 32 * c + e + i] * theirs;
            v[i] = fault ? __int_as_float(0x7fffffff) : v[i] * scale;
          }
          const int d = 32 * c + e;
          if (there && d < P.D) {
            if (whole) {
              Row<BF16>::put8(out + d, v);
            } else {
              *reinterpret_cast<float4*>(to + d) = make_float4(v[0], v[1], v[2], v[3]);
              *reinterpret_cast<float4*>(to + d + 4) = make_float4(v[4], v[5], v[6], v[7]);
            }
          }
        }
      }
      if (there && !whole) P.part_ml[part] = make_float2(ref, fault ? __int_as_float(0x7fffffff) : L);
    }
  }
  tmem_fence_before();
  __syncthreads();
  if (warp == 9) {
    tmem_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::kColumns) : "memory");
  }
}

template <int DP, bool BF16>
cudaError_t launch(const AttendParams& P, const CUtensorMap& k, const CUtensorMap& v, const Division& d, cudaStream_t st) {
  constexpr size_t kFixed = Shape<DP>::kBytes + sizeof(WideShared<DP>);
  const size_t words = (P.R + 31) / 32, rows = (d.rows + P.G - 1) / P.G + 1;
  const size_t smem = kFixed + (P.parents ? (rows * words + P.R) * 4 : 0);
  static DeviceFlags ready;
  cudaError_t e = allow_shared_memory(lantern_attention_wide_kernel<DP, BF16>, kFixed + (129 * 33 + kMaxTreeRows) * 4, ready);
  if (e != cudaSuccess) return e;
  lantern_attention_wide_kernel<DP, BF16><<<static_cast<unsigned>(d.units * d.splits), kThreads, smem, st>>>(P, d.rows, k, v);
  if ((e = cudaGetLastError()) != cudaSuccess || d.splits == 1) return e;
  return launch_join<DP, BF16>(P, d, st);
}

}  // namespace

cudaError_t launch_attention_wide(const AttendParams& P, const CUtensorMap& k, const CUtensorMap& v, const Division& d, bool bf16, cudaStream_t st) {
  if (d.DP == 64) return bf16 ? launch<64, true>(P, k, v, d, st) : launch<64, false>(P, k, v, d, st);
  return bf16 ? launch<128, true>(P, k, v, d, st) : launch<128, false>(P, k, v, d, st);
}

}  // namespace lantern
