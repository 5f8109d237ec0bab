// Attention of 17 to 64 bf16 rows of a sequence and cache head (a draft tree, say) to the paged 8-bit cache.
//
//   out = sum_c p_c v_c / sum_c p_c,   p_c = 2^(x_c - max x),   x_c = scale log2(e) k_scale (q . k_c)
//
// A CTA of four warps takes the 64 rows and a part of the tokens, in tiles of 64 (32 with 128 components).  The first warp asks for tiles of codes (TMA,
// block by block through the table) two ahead; all four turn a tile's codes into halves (every e4m3 value is one), a quarter of the tokens
// each and one tile ahead, and multiply 16 rows each by all of its tokens: m16n8k16 products of halves with fp32 accumulators, operands by
// ldmatrix, scores and probabilities in registers.  Queries go in as halves after a power of two of their own (their 8 bits fit).
//
// What costs is neither memory nor the tensor cores alone: ldmatrix (every warp reads the whole tile) and the products keep shared memory and the
// tensor pipe half busy each, and a warp's chain from scores to output does the rest.  256 trees of 61 rows, 20 heads of 64 components over 650
// tokens: 363 us (1.4 TB/s of codes); codes turned into halves by every warp for itself 505; 32 rows a warp 472 (registers).
// Where contexts can be long the tcgen05 path takes the same rows (cache_attention_wide.cu; both sides of the line are measured at `divide`).
#include "cache_attention.cuh"

namespace lantern {

namespace {

constexpr int kThreads = 128;
constexpr int kRows = 64, kStages = 2;

template <int DP>
constexpr int kTileOf = DP == 64 ? 64 : 32;   // (registers)

struct MidShared {
  uint64_t full[kStages];
  alignas(16) float scale[4][2][4];   // of every 16 tokens, keys and values, of the last four tiles
  uint32_t bad[2][4];                 // tokens with a NaN among their values, of each warp's quarter
  int fault;
};

__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void load4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void load4_across(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
// byte offset of 16 bytes of a token's halves: `unit` counts them along the row, 128-byte runs swizzled
template <int DP>
__device__ __forceinline__ int half_at(int token, int unit) {
  return DP == 64 ? token * 128 + ((unit ^ (token & 7)) << 4) : token * 256 + (((unit & 8) | ((unit ^ token) & 7)) << 4);
}

template <int DP>
__global__ void __launch_bounds__(kThreads, DP == 64 ? 3 : 2) lantern_attention_mid_kernel(AttendParams P, const __grid_constant__ CUtensorMap kmap,
                                                                                       const __grid_constant__ CUtensorMap vmap) {
  using T = __nv_bfloat16;
  constexpr int KS = DP / 16, NT = DP / 8;             // steps of the scores' products, column tiles of the output
  constexpr int kTile = kTileOf<DP>, ST = kTile / 8, SG = kTile / 16;   // tokens of a tile, score tiles, groups of 16 tokens
  constexpr int QUARTER = kTile / 4;                                   // tokens that a warp converts
  constexpr int kRaw = 2 * kTile * DP, kHalves = kTile * DP * 2;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t* halves = smem + kStages * kRaw;   // [2][keys, values]
  MidShared& S = *reinterpret_cast<MidShared*>(halves + 4 * kHalves);
  uint32_t* bits = reinterpret_cast<uint32_t*>(halves + 4 * kHalves + sizeof(MidShared));
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t unit = blockIdx.x / static_cast<uint32_t>(P.splits);
  const Unit u = unit_of(P, kRows, kTile, unit, static_cast<int>(blockIdx.x - unit * P.splits), unit_in(P, unit));
  grid_dependents_launch();
  if (!u.rows || u.split >= u.parts) return;
  // ---- queries and the tree's parents: asked for before anything waits ----
  const int g = lane >> 2, t = lane & 3;
  int row_of[2];   // step row; -1: not there
  uint32_t raw[2][KS][2];   // pairs of components 16 s + 2 t and 8 further
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int m = warp * 16 + g + 8 * half, r = m / P.G;   // (a unit is all rows there are: its first is row 0)
    row_of[half] = r < u.n ? r : -1;
    const T* p = static_cast<const T*>(P.q) + u.b * P.qs.b + r * P.qs.r + (static_cast<int64_t>(u.h) * P.G + (m - r * P.G)) * P.qs.h;
    if (P.vec) {
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int d = 16 * s + 8 * k + 2 * t;
          raw[half][s][k] = r < u.n && d < P.D ? __ldg(reinterpret_cast<const uint32_t*>(p + d)) : 0u;
        }
    } else {
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int d = 16 * s + 8 * k + 2 * t;
          raw[half][s][k] = r < u.n && d < P.D ? static_cast<uint32_t>(__ldg(reinterpret_cast<const uint16_t*>(p + d))) |
                                                     (static_cast<uint32_t>(__ldg(reinterpret_cast<const uint16_t*>(p + d + 1))) << 16)
                                               : 0u;
        }
    }
  }
  const int32_t* parents = P.parents && !u.fault ? P.parents + static_cast<int64_t>(u.b) * (P.R - 1) : nullptr;
  const int parent = parents && tid < u.n - 1 ? __ldg(parents + tid) : -1;
  const int words = (P.R + 31) >> 5;   // (1 or 2)
  if (tid == 0) {
    S.fault = u.fault;
    for (int i = 0; i < kStages; ++i) mbar_init(&S.full[i], 1);
    fence_mbar_init();
  }
  __syncthreads();

  // ---- tiles of codes, by the first warp: a lane per box; the table and the scales are looked up for as many tiles as there are lanes, a batch ahead ----
  const int sub = min(P.S, kTile), subs = kTile / sub, batch = 32 / subs;   // tokens of a box, boxes of a tile, tiles of a batch
  const int my_tile = lane / subs, my_sub = (lane - my_tile * subs) * sub;
  const int tiles = u.hi - u.lo;
  int found = 0;   // faults of the table
  Box box{0, 0, 1.0f, 0.0f}, next = box;
  if (warp == 0) next = look_up<kTile>(P, u, u.lo + my_tile, my_sub, u.hi, found);
  auto ask = [&](int i) {   // tile i into its stage, which nobody reads any more
    const int in_batch = i % batch, stage = i % kStages;
    if (in_batch == 0) {
      box = next;
      next = look_up<kTile>(P, u, u.lo + i + batch + my_tile, my_sub, u.hi, found);
    }
    const bool turn = my_tile == in_batch, mine = turn && box.mine;
    const int copies = __popc(__ballot_sync(kFull, mine));   // (at least one: every tile has a token that some row sees)
    if (lane == 0) mbar_expect_tx(&S.full[stage], copies * 2 * sub * DP);
    __syncwarp();
    const int token0 = (u.tile0 + u.lo + i) * kTile;
    if (mine && !withheld<kTile>(P, token0)) {
      uint8_t* at = smem + (stage * 2 * kTile + my_sub) * DP;
      const int row = u.h * P.S + (token0 + my_sub) % P.S;
      tma_load(at, &kmap, row, box.page, &S.full[stage]);
      tma_load(at + kTile * DP, &vmap, row, box.page, &S.full[stage]);
    }
    if (turn)   // (read behind a barrier of the block, not behind the copies)
      for (int e = 0; e < sub / 16; ++e) {
        S.scale[i & 3][0][my_sub / 16 + e] = box.ks;
        S.scale[i & 3][1][my_sub / 16 + e] = box.vs;
      }
  };
  if (warp == 0)
    for (int i = 0; i < min(tiles, kStages); ++i) ask(i);

  // ---- queries: halves ----
  uint32_t q[KS][4];
  float factor[2];
  {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      float most = 0.0f;
      int odd = 0;
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float a, b;
          bf16x2_widen(raw[half][s][k], a, b);
          odd |= !(fabsf(a) < __int_as_float(0x7f800000)) | !(fabsf(b) < __int_as_float(0x7f800000));
          most = fmaxf(most, fmaxf(fabsf(a), fabsf(b)));
        }
      most = fmaxf(most, __shfl_xor_sync(kFull, most, 1));
      most = fmaxf(most, __shfl_xor_sync(kFull, most, 2));
      odd |= __shfl_xor_sync(kFull, odd, 1);
      odd |= __shfl_xor_sync(kFull, odd, 2);
      const QueryPower power = query_power(P, most, odd);
      const float mult = power.mult;
      factor[half] = power.factor;
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float a, b;
          bf16x2_widen(raw[half][s][k], a, b);
          q[s][2 * k + half] = odd ? 0u : half2_of(a * mult, b * mult);
        }
    }
  }
  if (parents) {
    int32_t* nodes = reinterpret_cast<int32_t*>(bits + P.R * words);
    if (tid < u.n - 1) {
      nodes[tid] = parent;
      if (parent < -1 || parent >= tid) atomicOr(&S.fault, LANTERN_ST_BAD_PARENT);
    }
    if (tid < P.R * words) bits[tid] = 0;
    __syncthreads();
    if (tid < u.n && !(S.fault & LANTERN_ST_BAD_PARENT)) {
      uint32_t* mine = bits + tid * words;
      for (int r = tid; r > 0; r = nodes[r - 1] + 1) mine[r >> 5] |= 1u << (r & 31);
      mine[0] |= 1u;
    }
  }

  float o[NT][4];
#pragma unroll
  for (int i = 0; i < NT; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
  float ref[2] = {-INFINITY, -INFINITY}, sum[2] = {0.0f, 0.0f};   // sum: this lane's columns
  float vref = 0.0f, v_over = 0.0f;   // largest value scale met (roughly) and its reciprocal
  const uint32_t base = smem_addr(halves);
  bool ok = true;
  int converted = 0;   // tiles that this warp has waited for

  // Offsets of a lane's 16 bytes: of its token's codes (chunk lane / QUARTER; the j-th of its chunks lies at an exclusive or with j << kCodeStep), of the
  // halves that they become (j << kHalfStep, second half 16), and of its ldmatrix rows (keys: step s at s << 5; values: column tiles n, n + 1 at n << 4).  Whole groups of eight
  // tokens leave the swizzle as it is: they are added.
  constexpr int kRowBytes = 2 * DP, kCodeStep = DP == 64 ? 5 : 6, kHalfStep = DP == 64 ? 6 : 7;
  const int mine = warp * QUARTER + lane % QUARTER;
  const int code_from = chunk_at<DP>(mine, lane / QUARTER), half_to = half_at<DP>(mine, 2 * (lane / QUARTER));
  const int key_from = half_at<DP>((lane & 7) + ((lane >> 4) & 1) * 8, (lane >> 3) & 1), value_from = half_at<DP>((lane & 7) + ((lane >> 3) & 1) * 8, lane >> 4);

  auto edge_of = [&](int i) {
    const int token0 = (u.tile0 + u.lo + i) * kTile;
    return token0 < u.begin || token0 + kTile > u.len + (P.parents ? 0 : 1);   // some row may not see all of the tile
  };
  // this warp's quarter of tile i as halves
  auto convert = [&](int i) {
    const int stage = i % kStages, k = i & 1;
    ok = ok && __all_sync(kFull, await(P, &S.full[stage], (i / kStages) & 1));
    converted += ok;
    const uint8_t* raw = smem + stage * kRaw;
    uint8_t* to = halves + 2 * k * kHalves;
    const bool edge = edge_of(i);
    bool nan = false;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {   // (a quarter's codes are 64 times 16 bytes)
        uint4 x = *reinterpret_cast<const uint4*>(raw + which * kTile * DP + (code_from ^ (j << kCodeStep)));
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
        *reinterpret_cast<uint4*>(to + which * kHalves + (half_to ^ (j << kHalfStep))) = make_uint4(h[0], h[1], h[2], h[3]);
        *reinterpret_cast<uint4*>(to + which * kHalves + (half_to ^ (j << kHalfStep) ^ 16)) = make_uint4(h[4], h[5], h[6], h[7]);
      }
    }
    if (edge) {
      uint32_t hit = __ballot_sync(kFull, nan);
      hit |= hit >> 16;
      if (QUARTER == 8) hit |= hit >> 8;
      if (lane == 0) S.bad[k][warp] = hit & ((1u << QUARTER) - 1u);
    }
  };

  // this warp's rows and tile i
  auto step = [&](int i, const float (&ks)[SG], const float (&vs)[SG]) {
    const uint32_t keys = base + 2 * (i & 1) * kHalves + key_from, values = base + (2 * (i & 1) + 1) * kHalves + value_from;
    const bool edge = edge_of(i);
    float c[ST][4];
#pragma unroll
    for (int j = 0; j < ST; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) c[j][e] = 0.0f;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const uint32_t at = keys ^ (s << 5);
#pragma unroll
      for (int j = 0; j < ST; j += 2) {
        uint32_t b[4];
        load4(b, at + j * 8 * kRowBytes);
        mma16816(c[j], q[s], b[0], b[1]);
        mma16816(c[j + 1], q[s], b[2], b[3]);
      }
    }
    if (edge) {
      const int token0 = (u.tile0 + u.lo + i) * kTile;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int r = row_of[half];
        const uint32_t* seen = bits + (r < 0 ? 0 : r) * words;
#pragma unroll
        for (int w = 0; w < kTile / 32; ++w) {
          const int a = token0 + 32 * w, ahead = a - u.len;
          uint32_t see = low_bits(-ahead + (P.parents ? 0 : r + 1));
          if (P.parents) {
            if (ahead >= 0) {
              const int k = ahead >> 5;
              see |= __funnelshift_r(k < words ? seen[k] : 0u, k + 1 < words ? seen[k + 1] : 0u, ahead & 31);
            } else if (ahead > -32) {
              see |= seen[0] << -ahead;
            }
          }
          see &= ~low_bits(u.begin - a);
          if (r < 0) see = 0;
          const uint32_t* of = S.bad[i & 1];
          const uint32_t bad = see & (QUARTER == 16 ? of[2 * w] | (of[2 * w + 1] << 16) : of[0] | (of[1] << 8) | (of[2] << 16) | (of[3] << 24));
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float& x = c[4 * w + j][2 * half + e];
              const int bit = 8 * j + 2 * t + e;
              if (!((see >> bit) & 1u)) x = -INFINITY;
              if ((bad >> bit) & 1u) x = __int_as_float(0x7fffffff);
            }
        }
      }
    }
    float f[2][SG], most[2], v_most = vs[0];
#pragma unroll
    for (int k = 1; k < SG; ++k) v_most = fmaxf(v_most, vs[k]);
    bool grow = v_most > vref * kScaleLag;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      float m = -INFINITY;
#pragma unroll
      for (int k = 0; k < SG; ++k) {
        f[half][k] = factor[half] * ks[k];
        if (edge && f[half][k] < 1.17549435e-38f) f[half][k] = 1.17549435e-38f;   // (not zero: a hidden token stays at minus infinity)
        const float a = max3(max3(c[2 * k][2 * half], c[2 * k][2 * half + 1], c[2 * k + 1][2 * half]), c[2 * k + 1][2 * half + 1], -INFINITY);
        m = fmaxf(m, a * f[half][k]);
      }
      most[half] = m;   // of this lane's tokens
      grow |= m > ref[half] + kLag;
    }
    // (the lanes' maxima are put together only when the reference moves)
    if (__any_sync(kFull, grow)) {
      const float v_new = fmaxf(vref, v_most), v_ratio = v_new > 0.0f ? vref / v_new : 0.0f;
      float w[2];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        float m = fmaxf(most[half], __shfl_xor_sync(kFull, most[half], 1));
        m = fmaxf(ref[half], fmaxf(m, __shfl_xor_sync(kFull, m, 2)));
        const float k = ref[half] == -INFINITY ? 0.0f : ex2_approx(ref[half] - m);
        ref[half] = m;
        sum[half] *= k;
        w[half] = k * v_ratio;
      }
      vref = v_new;
      v_over = v_new > 0.0f ? __frcp_rn(v_new) : 0.0f;   // (a scale of zero: a block of zeros)
#pragma unroll
      for (int n = 0; n < NT; ++n) o[n][0] *= w[0], o[n][1] *= w[0], o[n][2] *= w[1], o[n][3] *= w[1];
    }
    const float back[2] = {ref[0] == -INFINITY ? 0.0f : -ref[0], ref[1] == -INFINITY ? 0.0f : -ref[1]};
    uint64_t part[2] = {pack2(0.0f, 0.0f), pack2(0.0f, 0.0f)};
#pragma unroll
    for (int k = 0; k < SG; ++k) {   // 16 tokens
      uint32_t p[4];
      const float vr = vs[k] * v_over * kLift;
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float a, b;
          unpack2(fma2(pack2(c[2 * k + j][2 * half], c[2 * k + j][2 * half + 1]), pack2(f[half][k], f[half][k]), pack2(back[half], back[half])), a, b);
          a = ex2_approx(a), b = ex2_approx(b);
          part[half] = add2(part[half], pack2(a, b));
          unpack2(mul2(pack2(a, b), pack2(vr, vr)), a, b);
          p[2 * j + half] = half2_of(a, b);
        }
#pragma unroll
      for (int n = 0; n < NT; n += 2) {
        uint32_t b[4];
        load4_across(b, (values ^ (n << 4)) + 16 * k * kRowBytes);
        mma16816(o[n], p, b[0], b[1]);
        mma16816(o[n + 1], p, b[2], b[3]);
      }
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      float a, b;
      unpack2(part[half], a, b);
      sum[half] += a + b;
    }
  };

  if (tiles > 0) convert(0);
  __syncthreads();
  for (int i = 0; i < tiles; ++i) {
    if (warp == 0 && ok && i + kStages < tiles) ask(i + kStages);   // (into the stage that tile i has been taken from)
    if (i + 1 < tiles) convert(i + 1);
    float ks[SG], vs[SG];
#pragma unroll
    for (int k = 0; k < SG; ++k) ks[k] = S.scale[i & 3][0][k], vs[k] = S.scale[i & 3][1][k];
    step(i, ks, vs);
    __syncthreads();   // the next tile's halves are there, this one's are read
  }
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    sum[half] += __shfl_xor_sync(kFull, sum[half], 1);
    sum[half] += __shfl_xor_sync(kFull, sum[half], 2);
  }
  if (!ok) {
    found |= LANTERN_ST_INTERNAL;
    if (warp == 0)   // nothing may be under way when the CTA ends: tiles up to kStages behind the last that came have been asked for
      for (int i = converted; i < min(converted + kStages, tiles); ++i) await(P, &S.full[i % kStages], (i / kStages) & 1);
  }
  if (found) atomicOr(&S.fault, found);
  __syncthreads();
  const int fault = S.fault;
  if (fault && tid == 0 && P.status) atomicOr(P.status + u.b, fault);
  const bool whole = u.parts == 1;
  const int64_t part = static_cast<int64_t>(blockIdx.x) * kRows;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int row = warp * 16 + g + 8 * half, r = row_of[half];
    if (r < 0) continue;
    T* out = static_cast<T*>(P.out) + ((static_cast<int64_t>(u.b) * P.R + r) * P.q_heads + u.h * P.G + (row - r * P.G)) * P.D;
    float* to = P.parts + (part + row) * DP;
    const float own = vref * (1.0f / kLift);
    const float scale = fault ? __int_as_float(0x7fffffff) : whole ? (sum[half] == 0.0f ? 0.0f : own / sum[half]) : own;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int d = 8 * n + 2 * t;
      if (d < P.D) {
        const float a = o[n][2 * half] * scale, b = o[n][2 * half + 1] * scale;
        if (whole) *reinterpret_cast<uint32_t*>(out + d) = bf16x2_round(a, b);
        else *reinterpret_cast<float2*>(to + d) = make_float2(a, b);
      }
    }
    if (!whole && t == 0) P.part_ml[part + row] = make_float2(ref[half], fault ? __int_as_float(0x7fffffff) : sum[half]);
  }
}

template <int DP>
cudaError_t launch(const AttendParams& P, const CUtensorMap& k, const CUtensorMap& v, const Division& d, cudaStream_t st) {
  constexpr size_t kFixed = (kStages * 2 + 8) * kTileOf<DP> * DP + sizeof(MidShared);
  const size_t smem = kFixed + (P.parents ? (P.R * ((P.R + 31) / 32) + P.R) * 4 : 0);
  static DeviceFlags ready;
  cudaError_t e = allow_shared_memory(lantern_attention_mid_kernel<DP>, kFixed + (kRows * 2 + kRows) * 4, ready);   // (at most 64 rows)
  if (e != cudaSuccess) return e;
  lantern_attention_mid_kernel<DP><<<static_cast<unsigned>(d.units * d.splits), kThreads, smem, st>>>(P, k, v);
  if ((e = cudaGetLastError()) != cudaSuccess || d.splits == 1) return e;
  return launch_join<DP, true>(P, d, st);
}

}  // namespace

cudaError_t launch_attention_mid(const AttendParams& P, const CUtensorMap& k, const CUtensorMap& v, const Division& d, cudaStream_t st) {
  return d.DP == 64 ? launch<64>(P, k, v, d, st) : launch<128>(P, k, v, d, st);
}

}  // namespace lantern
