// Attention of up to 16 rows of a sequence and cache head (single tokens, short chains) to the paged 8-bit cache.
//
//   out = sum_c p_c v_c / sum_c p_c,   p_c = 2^(x_c - max x),   x_c = scale log2(e) k_scale (q . k_c)
//
// Bound by the codes' way from HBM: with few rows there are a handful of operations per byte, and what is left to do is to keep enough bytes
// under way and enough warps ready.  So every warp goes its own way: it copies 32 tokens at a time (TMA, block by block through the table) into
// stages of its own, four warps taking turns in the tokens of a part, and joins the others at the end only.
//
// Tokens stand where products are 16 wide and rows where they are 8 wide (scores^T = K Q^T, output^T = V^T P^T, m16n8k16, halves, fp32
// accumulators): up to 8 rows waste nothing of it.  Codes become halves in registers straight from shared memory (every e4m3 value is one; a
// lane's components of a token are 16 bytes side by side, a permutation of the products' inner axis), queries are halves after a power of two
// of their own (8 bits of a bf16 query fit; an fp32 query goes in as two halves, 22 bits, and so do its probabilities).
//
// 128 single tokens, 32 heads over 8, contexts of 500 to 4100 tokens of 128 components: 116 us, 5.2 TB/s; with rows where products are 16 wide, a
// producer warp and barriers between four warps 193.
#include "cache_attention.cuh"

namespace lantern {

namespace {

constexpr int kThreads = 128, kWarps = 4, kTile = 32;
template <int DP>
constexpr int kStagesOf = DP == 64 ? 4 : 2;

template <int ROWS>
struct FewShared {
  uint64_t full[kWarps][4];
  float scale[kWarps][8][2][2];   // of every 16 tokens, keys and values, of a warp's last eight tiles
  float2 ml[kWarps][ROWS];
  int fault;
};

__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {   // of 8 by 8 halves
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ uint32_t low2(uint32_t w) { return decode2(static_cast<uint16_t>(w & 0xffffu)); }
__device__ __forceinline__ uint32_t high2(uint32_t w) { return decode2(static_cast<uint16_t>(w >> 16)); }

// NQ: eights of rows.
template <int NQ, int DP, bool BF16>
__global__ void __launch_bounds__(kThreads, NQ == 1 && BF16 ? 3 : 2) lantern_attention_few_kernel(AttendParams P, const __grid_constant__ CUtensorMap kmap,
                                                                                               const __grid_constant__ CUtensorMap vmap) {
  using T = typename Row<BF16>::T;
  constexpr int ROWS = 16, TERMS = BF16 ? 1 : 2, STAGES = kStagesOf<DP>;
  constexpr int KS = DP / 16, MT = DP / 16;   // steps of the scores' products, row tiles of the output
  constexpr int EL = DP / 4;                  // components of a row that a lane holds for the scores, side by side
  constexpr int VL = DP / 8;                  // components of a token's values that a lane holds, side by side: 16 or 8
  constexpr int kStageBytes = 2 * kTile * DP;
  extern __shared__ __align__(1024) uint8_t smem[];
  FewShared<ROWS>& S = *reinterpret_cast<FewShared<ROWS>*>(smem + kWarps * STAGES * kStageBytes);
  uint32_t* bits = reinterpret_cast<uint32_t*>(smem + kWarps * STAGES * kStageBytes + sizeof(FewShared<ROWS>));
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const uint32_t unit = blockIdx.x / static_cast<uint32_t>(P.splits);
  const Unit u = unit_of(P, ROWS, kTile, unit, static_cast<int>(blockIdx.x - unit * P.splits), unit_in(P, unit));
  grid_dependents_launch();
  if (!u.rows || u.split >= u.parts) return;
  uint8_t* stages = smem + warp * STAGES * kStageBytes;
  uint64_t* full = S.full[warp];
  if (tid == 0) S.fault = u.fault;
  if (lane == 0) {
    for (int i = 0; i < STAGES; ++i) mbar_init(&full[i], 1);
    fence_mbar_init();
  }
  __syncwarp();

  // ---- this warp's tiles of codes: every fourth of the part's; a lane per box, looked up for as many tiles as there are lanes, a batch ahead ----
  const int sub = min(P.S, kTile), subs = kTile / sub, batch = 32 / subs;   // tokens of a box, boxes of a tile, tiles of a batch
  const int my_tile = lane / subs, my_sub = (lane - my_tile * subs) * sub;
  const int tiles = u.hi > u.lo + warp ? (u.hi - u.lo - warp + kWarps - 1) / kWarps : 0;
  int found = 0;   // faults of the table
  Box box, next = look_up<kTile>(P, u, u.lo + warp + kWarps * my_tile, my_sub, u.hi, found);
  auto ask = [&](int i) {   // tile i into its stage, which this warp has read
    const int in_batch = i & (batch - 1), stage = i % STAGES;
    if (in_batch == 0) {
      box = next;
      if (i + batch < tiles) next = look_up<kTile>(P, u, u.lo + warp + kWarps * (i + batch + my_tile), my_sub, u.hi, found);
    }
    const bool turn = my_tile == in_batch, mine = turn && box.mine;
    const int token0 = (u.tile0 + u.lo + warp + kWarps * i) * kTile;
    const int copies = __popc(__ballot_sync(kFull, mine));   // (at least one: every tile has a token that some row sees)
    if (lane == 0) mbar_expect_tx(&full[stage], copies * 2 * sub * DP);
    __syncwarp();
    if (mine && !withheld<kTile>(P, token0)) {
      uint8_t* at = stages + stage * kStageBytes + my_sub * DP;
      const int row = u.h * P.S + (token0 + my_sub) % P.S;
      tma_load(at, &kmap, row, box.page, &full[stage]);
      tma_load(at + kTile * DP, &vmap, row, box.page, &full[stage]);
    }
    if (turn)
      for (int e = 0; e < sub / 16; ++e) {
        S.scale[warp][i & 7][0][my_sub / 16 + e] = box.ks;
        S.scale[warp][i & 7][1][my_sub / 16 + e] = box.vs;
      }
  };
  for (int i = 0; i < min(tiles, STAGES); ++i) ask(i);

  // ---- queries: row 8 q + g, this lane's components from t EL on ----
  uint32_t query[NQ][KS][TERMS][2];
  float factor[NQ][2];   // of the rows 8 q + 2 t, 8 q + 2 t + 1, which this lane has scores of
  int row_of[NQ][2];     // their step rows; -1: not there
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    const int m = 8 * q + g, r = m / P.G;
    const bool there = r < u.n;
    const T* p = static_cast<const T*>(P.q) + u.b * P.qs.b + r * P.qs.r + (static_cast<int64_t>(u.h) * P.G + (m - r * P.G)) * P.qs.h + t * EL;
    float v[EL], most = 0.0f;
    int odd = 0;
    if (P.vec) {
#pragma unroll
      for (int e = 0; e < EL; e += 8) {
        float x[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        if (there && t * EL + e < P.D) Row<BF16>::get8(p + e, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[e + i] = x[i];
      }
    } else {
#pragma unroll
      for (int e = 0; e < EL; ++e) v[e] = there && t * EL + e < P.D ? Row<BF16>::get(p + e) : 0.0f;
    }
#pragma unroll
    for (int e = 0; e < EL; ++e) {
      odd |= !(fabsf(v[e]) < __int_as_float(0x7f800000));
      most = fmaxf(most, fabsf(v[e]));
    }
    most = fmaxf(most, __shfl_xor_sync(kFull, most, 1));
    most = fmaxf(most, __shfl_xor_sync(kFull, most, 2));
    odd |= __shfl_xor_sync(kFull, odd, 1);
    odd |= __shfl_xor_sync(kFull, odd, 2);
    const QueryPower power = query_power(P, most, odd);
    const float mult = power.mult, f = power.factor;
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float a = odd ? 0.0f : v[4 * s + 2 * k] * mult, b = odd ? 0.0f : v[4 * s + 2 * k + 1] * mult;
        query[q][s][0][k] = half2_of(a, b);
        if constexpr (TERMS == 2) query[q][s][1][k] = half2_rest(a, b, query[q][s][0][k]);
      }
#pragma unroll
    for (int e = 0; e < 2; ++e) {   // row 2 t + e is held by the lanes of group 2 t + e
      factor[q][e] = __shfl_sync(kFull, f, 4 * (2 * t + e));
      const int mr = 8 * q + 2 * t + e, rr = mr / P.G;
      row_of[q][e] = rr < u.n ? rr : -1;
    }
  }
  if (P.parents && !u.fault) {
    const int32_t* parents = P.parents + static_cast<int64_t>(u.b) * (P.R - 1);
    int32_t* nodes = reinterpret_cast<int32_t*>(bits + ROWS);   // (a unit is all rows there are, 16 at most: a word of bits each)
    __syncthreads();   // (the fault word is there)
    if (tid < u.n - 1) {
      const int p = __ldg(parents + tid);
      nodes[tid] = p;
      if (p < -1 || p >= tid) atomicOr(&S.fault, LANTERN_ST_BAD_PARENT);
    }
    __syncthreads();
    if (tid < u.n) {
      uint32_t mine = 0u;
      if (!(S.fault & LANTERN_ST_BAD_PARENT)) {
        for (int r = tid; r > 0; r = nodes[r - 1] + 1) mine |= 1u << r;
        mine |= 1u;
      }
      bits[tid] = mine;
    }
    __syncthreads();
  }

  float o[NQ][MT][4];   // components (VL g + 2 i, VL g + 2 i + 1) of rows 8 q + 2 t and + 1: [0], [1] the first component, [2], [3] the second
#pragma unroll
  for (int q = 0; q < NQ; ++q)
#pragma unroll
    for (int i = 0; i < MT; ++i) o[q][i][0] = o[q][i][1] = o[q][i][2] = o[q][i][3] = 0.0f;
  float ref[NQ][2], sum[NQ][2], vref = 0.0f, v_over = 0.0f;   // largest value scale met (roughly) and its reciprocal; sum: this lane's tokens
#pragma unroll
  for (int q = 0; q < NQ; ++q)
#pragma unroll
    for (int e = 0; e < 2; ++e) ref[q][e] = -INFINITY, sum[q][e] = 0.0f;
  bool ok = true;

  for (int i = 0; i < tiles; ++i) {
    const int stage = i % STAGES;
    ok = __all_sync(kFull, await(P, &full[stage], (i / STAGES) & 1));
    if (!ok) {   // nothing may be under way into the stages when they are used for something else, or when the CTA ends
      for (int k = i; k < min(i + STAGES, tiles); ++k) await(P, &full[k % STAGES], (k / STAGES) & 1);
      break;
    }
    const uint8_t *keys = stages + stage * kStageBytes, *values = keys + kTile * DP;
    const int token0 = (u.tile0 + u.lo + warp + kWarps * i) * kTile;
    const bool edge = token0 < u.begin || token0 + kTile > u.len + (P.parents ? 0 : 1);   // some row may not see all of the tile
    const float ks[2] = {S.scale[warp][i & 7][0][0], S.scale[warp][i & 7][0][1]}, vs[2] = {S.scale[warp][i & 7][1][0], S.scale[warp][i & 7][1][1]};

    float c[2][NQ][4];   // 16 tokens each: [0], [1] token g, rows 2 t and 2 t + 1; [2], [3] token g + 8
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
      for (int q = 0; q < NQ; ++q) c[k][q][0] = c[k][q][1] = c[k][q][2] = c[k][q][3] = 0.0f;
      uint32_t w[2][KS];
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int e = 0; e < KS / 4; ++e) {
          const uint4 x = *reinterpret_cast<const uint4*>(keys + chunk_at<DP>(16 * k + 8 * r + g, t * (KS / 4) + e));
          w[r][4 * e] = x.x, w[r][4 * e + 1] = x.y, w[r][4 * e + 2] = x.z, w[r][4 * e + 3] = x.w;
        }
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const uint32_t a0 = low2(w[0][s]), a1 = low2(w[1][s]), a2 = high2(w[0][s]), a3 = high2(w[1][s]);
#pragma unroll
        for (int q = 0; q < NQ; ++q)
#pragma unroll
          for (int n = 0; n < TERMS; ++n) mma16816(c[k][q], a0, a1, a2, a3, query[q][s][n][0], query[q][s][n][1]);
      }
    }
    uint32_t bad = 0;   // tokens with a NaN among their values (looked for where a token may be hidden from a row)
    if (edge) {
      bool mine = false;
#pragma unroll
      for (int e = 0; e < DP / 16; ++e) mine |= has_nan(*reinterpret_cast<const uint4*>(values + chunk_at<DP>(lane, e)));
      bad = __ballot_sync(kFull, mine);
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int q = 0; q < NQ; ++q)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int at = 16 * k + 8 * (e >> 1) + g, token = token0 + at, r = row_of[q][e & 1], ahead = token - u.len;
            bool see = r >= 0 && token >= u.begin && token < u.end;
            if (see && ahead >= 0) see = P.parents ? (bits[r] >> ahead) & 1u : ahead <= r;
            if (!see) c[k][q][e] = -INFINITY;
            else if ((bad >> at) & 1u) c[k][q][e] = __int_as_float(0x7fffffff);
          }
    }
    float f[NQ][2][2];   // of a row and 16 tokens
    const float v_most = fmaxf(vs[0], vs[1]);
    bool grow = v_most > vref * kScaleLag;
    float most[NQ][2];
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          f[q][e][k] = factor[q][e] * ks[k];
          if (edge && f[q][e][k] < 1.17549435e-38f) f[q][e][k] = 1.17549435e-38f;   // (not zero: a hidden token stays at minus infinity)
        }
        float m = fmaxf(fmaxf(c[0][q][e], c[0][q][2 + e]) * f[q][e][0], fmaxf(c[1][q][e], c[1][q][2 + e]) * f[q][e][1]);
        m = fmaxf(m, __shfl_xor_sync(kFull, m, 4));
        m = fmaxf(m, __shfl_xor_sync(kFull, m, 8));
        m = fmaxf(m, __shfl_xor_sync(kFull, m, 16));
        most[q][e] = m;
        grow |= m > ref[q][e] + kLag;
      }
    if (__any_sync(kFull, grow)) {
      const float v_new = fmaxf(vref, v_most), v_ratio = v_new > 0.0f ? vref / v_new : 0.0f;
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        float w[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float m = fmaxf(ref[q][e], most[q][e]), k = ref[q][e] == -INFINITY ? 0.0f : ex2_approx(ref[q][e] - m);
          ref[q][e] = m;
          sum[q][e] *= k;
          w[e] = k * v_ratio;
        }
#pragma unroll
        for (int n = 0; n < MT; ++n) o[q][n][0] *= w[0], o[q][n][1] *= w[1], o[q][n][2] *= w[0], o[q][n][3] *= w[1];
      }
      vref = v_new;
      v_over = v_new > 0.0f ? __frcp_rn(v_new) : 0.0f;   // (a scale of zero: a block of zeros)
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {   // 16 tokens
      const float vr = vs[k] * v_over * kLift;
      uint32_t p[NQ][TERMS][2];
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        const float b0 = ref[q][0] == -INFINITY ? 0.0f : ref[q][0], b1 = ref[q][1] == -INFINITY ? 0.0f : ref[q][1];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float x = ex2_approx(__fmaf_rn(c[k][q][2 * r], f[q][0][k], -b0)), y = ex2_approx(__fmaf_rn(c[k][q][2 * r + 1], f[q][1][k], -b1));
          sum[q][0] += x, sum[q][1] += y;
          x *= vr, y *= vr;
          const uint32_t h = half2_of(x, y);
          p[q][0][r] = transposed(h);
          if constexpr (TERMS == 2) p[q][1][r] = transposed(half2_rest(x, y, h));
        }
      }
      // values of tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9: components VL g ... side by side
      constexpr int VW = VL / 4;
      uint32_t x[4][VW];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int token = 16 * k + 2 * t + (e & 1) + 8 * (e >> 1);
        if constexpr (DP == 128) {
          const uint4 y = *reinterpret_cast<const uint4*>(values + chunk_at<DP>(token, g));
          x[e][0] = y.x, x[e][1] = y.y, x[e][2] = y.z, x[e][3] = y.w;
        } else {
          const uint2 y = *reinterpret_cast<const uint2*>(values + chunk_at<DP>(token, g >> 1) + (g & 1) * 8);
          x[e][0] = y.x, x[e][1] = y.y;
        }
      }
      if (bad) {   // (uniform)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int n = 0; n < VW; ++n) x[e][n] = without_nan(x[e][n]);
      }
#pragma unroll
      for (int n = 0; n < VW; ++n) {   // four components: two tiles of (first, second) components
        const uint32_t a = __byte_perm(x[0][n], x[1][n], 0x5140), b = __byte_perm(x[0][n], x[1][n], 0x7362);
        const uint32_t d = __byte_perm(x[2][n], x[3][n], 0x5140), e = __byte_perm(x[2][n], x[3][n], 0x7362);
        const uint32_t a0 = low2(a), a1 = high2(a), a2 = low2(d), a3 = high2(d), e0 = low2(b), e1 = high2(b), e2 = low2(e), e3 = high2(e);
#pragma unroll
        for (int q = 0; q < NQ; ++q)
#pragma unroll
          for (int m = 0; m < TERMS; ++m) {
            mma16816(o[q][2 * n], a0, a1, a2, a3, p[q][m][0], p[q][m][1]);
            mma16816(o[q][2 * n + 1], e0, e1, e2, e3, p[q][m][0], p[q][m][1]);
          }
      }
    }
    __syncwarp();
    if (i + STAGES < tiles) ask(i + STAGES);
  }
#pragma unroll
  for (int q = 0; q < NQ; ++q)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      sum[q][e] += __shfl_xor_sync(kFull, sum[q][e], 4);
      sum[q][e] += __shfl_xor_sync(kFull, sum[q][e], 8);
      sum[q][e] += __shfl_xor_sync(kFull, sum[q][e], 16);
      if (g == 0) S.ml[warp][8 * q + 2 * t + e] = make_float2(ref[q][e], sum[q][e]);
    }
  if (!ok) found |= LANTERN_ST_INTERNAL;
  __syncthreads();   // all stages are read, the fault word is there
  if (found) atomicOr(&S.fault, found);

  // ---- the four warps' accumulators meet in shared memory: [warp][row][DP + 4] ----
  float* buf = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int q = 0; q < NQ; ++q)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int row = 8 * q + 2 * t + e;
      float M = -INFINITY;
#pragma unroll
      for (int k = 0; k < kWarps; ++k) M = fmaxf(M, S.ml[k][row].x);
      const float w = vref * (1.0f / kLift) * ex2_approx(ref[q][e] - (M == -INFINITY ? 0.0f : M));
#pragma unroll
      for (int n = 0; n < MT; n += 2)
        *reinterpret_cast<float4*>(buf + (warp * 8 * NQ + row) * (DP + 4) + VL * g + 2 * n) =
            make_float4(o[q][n][e] * w, o[q][n][2 + e] * w, o[q][n + 1][e] * w, o[q][n + 1][2 + e] * w);
    }
  __syncthreads();
  const int fault = S.fault;
  if (fault && tid == 0 && P.status) atomicOr(P.status + u.b, fault);
  const bool whole = u.parts == 1;
  const int64_t part = static_cast<int64_t>(blockIdx.x) * ROWS;
  const int per_row = P.D >> 2, rows = min(8 * NQ, u.n * P.G);
  for (int i = tid; i < rows * per_row; i += kThreads) {
    const int row = i / per_row, d = (i - row * per_row) * 4, r = row / P.G;
    float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    float M = -INFINITY, L = 0.0f;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) {
      const float4 y = *reinterpret_cast<const float4*>(buf + (k * 8 * NQ + row) * (DP + 4) + d);
      x.x += y.x, x.y += y.y, x.z += y.z, x.w += y.w;
      M = fmaxf(M, S.ml[k][row].x);
    }
    const float base = M == -INFINITY ? 0.0f : M;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) L += S.ml[k][row].y * ex2_approx(S.ml[k][row].x - base);
    if (whole) {
      const float inv = fault ? __int_as_float(0x7fffffff) : L == 0.0f ? 0.0f : 1.0f / L;
      T* out = static_cast<T*>(P.out) + ((static_cast<int64_t>(u.b) * P.R + r) * P.q_heads + u.h * P.G + (row - r * P.G)) * P.D + d;
      if constexpr (BF16) *reinterpret_cast<uint2*>(out) = make_uint2(bf16x2_round(x.x * inv, x.y * inv), bf16x2_round(x.z * inv, x.w * inv));
      else *reinterpret_cast<float4*>(out) = make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
    } else {
      *reinterpret_cast<float4*>(P.parts + (part + row) * DP + d) = x;
      if (d == 0) P.part_ml[part + row] = make_float2(M, fault ? __int_as_float(0x7fffffff) : L);
    }
  }
}

template <int NQ, int DP, bool BF16>
cudaError_t launch(const AttendParams& P, const CUtensorMap& k, const CUtensorMap& v, const Division& d, cudaStream_t st) {
  constexpr size_t kFixed = kWarps * kStagesOf<DP> * 2 * kTile * DP + sizeof(FewShared<16>);
  static_assert(kWarps * 8 * NQ * (DP + 4) * sizeof(float) <= kWarps * kStagesOf<DP> * 2 * kTile * DP, "accumulators");
  const size_t smem = kFixed + (P.parents ? 2 * 16 * 4 : 0);   // (a word of bits and a parent for each row)
  static DeviceFlags ready;
  cudaError_t e = allow_shared_memory(lantern_attention_few_kernel<NQ, DP, BF16>, kFixed + 2 * 16 * 4, ready);
  if (e != cudaSuccess) return e;
  lantern_attention_few_kernel<NQ, DP, BF16><<<static_cast<unsigned>(d.units * d.splits), kThreads, smem, st>>>(P, k, v);
  if ((e = cudaGetLastError()) != cudaSuccess || d.splits == 1) return e;
  return launch_join<DP, BF16>(P, d, st);
}

}  // namespace

cudaError_t launch_attention_few(const AttendParams& P, const CUtensorMap& k, const CUtensorMap& v, const Division& d, bool bf16, cudaStream_t st) {
  if (static_cast<int64_t>(P.R) * P.G <= 8) {
    if (d.DP == 64) return bf16 ? launch<1, 64, true>(P, k, v, d, st) : launch<1, 64, false>(P, k, v, d, st);
    return bf16 ? launch<1, 128, true>(P, k, v, d, st) : launch<1, 128, false>(P, k, v, d, st);
  }
  if (d.DP == 64) return bf16 ? launch<2, 64, true>(P, k, v, d, st) : launch<2, 64, false>(P, k, v, d, st);
  return bf16 ? launch<2, 128, true>(P, k, v, d, st) : launch<2, 128, false>(P, k, v, d, st);
}

}  // namespace lantern
