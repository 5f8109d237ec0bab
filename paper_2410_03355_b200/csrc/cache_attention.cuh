// What the attention kernels share: the call's parameters, what a unit of work covers, tensor maps of the codes, and the joining of parts.
#pragma once

#include <cuda.h>

#include "cache_common.cuh"

namespace lantern {

// Numerators go into the products as halves, whose bits end at 2^-24, and a row's small ones count: many of them may be all that a row has besides a token
// without a value.  So they are lifted towards a half's largest value, 2^16.  They refer to a maximum that follows the running one only when it
// has fallen behind by 2^kLag, so that accumulators are rarely touched, and come with their value's scale over a largest one that may
// have fallen behind by kScaleLag (few, mid), or with that scale's digits (wide, fp32): at most 2^4 * 2 * 2^10.  What is 2^-24 of the row's largest is still a normal half, what is lost is 2^-35 of
// it.  A lag of 2^2 with 2^12 costs 0.5 % of 256 trees (mid) and 3.5 % of 16 trees of 8 heads a group (wide) more than these; 2^8, 2^5 and no lift 2 % less
// and the same.
constexpr float kLift = 1024.0f, kLag = 4.0f, kScaleLag = 2.0f;

struct AttendParams {
  const void* q;
  void* out;
  RowStride qs;
  const float* k_scale;
  const float* v_scale;
  const int32_t* table;
  const int32_t* lengths;
  const int32_t* counts;
  const int32_t* starts;
  const int32_t* parents;
  int32_t* status;
  float* parts;       // [unit][split][rows of a unit][DP] numerators, relative to 2^maximum
  float2* part_ml;    // [unit][split][rows of a unit] maximum (base 2), sum
  int B, R, q_heads, heads, G, S, D, width, pages;
  int row_tiles;      // units per sequence and cache head
  uint32_t items;     // units * splits
  int splits;         // parts that a unit's tokens are divided into, at most
  int least;          // tiles per part, at least
  int vec;            // query rows may be read 16 bytes at a time
  float scale_log2;   // scale * log2(e)
  uint32_t tries;     // limit of a wait for a copy
  int withhold;       // self-test only: the copies of the tile that holds this token are never issued (-1: none)
};
// The copies of a tile of TILE tokens from token0 on are withheld.
template <int TILE>
__device__ __forceinline__ bool withheld(const AttendParams& P, int token0) {
  return static_cast<uint32_t>(P.withhold - token0) < static_cast<uint32_t>(TILE);
}

// What rows [m0, m0 + ROWS) of one sequence and cache head (row m: step row m / G, head m % G) have to read.
struct Unit {
  int b, h, m0, split;
  int len, n;            // cached tokens, rows of the step (what the checks leave of them)
  int begin, end;        // tokens [begin, end) that some row of the unit may see
  int tile0, lo, hi;     // first tile of the unit; tiles [lo, hi) of it are this part's
  int parts;             // parts with work
  int fault;
  bool rows;             // there are rows to answer
};
// What a unit's sequence says of it (read ahead of time where a unit follows another).
struct UnitIn {
  int len, n, begin;
};
__device__ __forceinline__ int sequence_of(const AttendParams& P, uint32_t unit) {
  return static_cast<int>(unit / (static_cast<uint32_t>(P.row_tiles) * static_cast<uint32_t>(P.heads)));
}
__device__ __forceinline__ UnitIn unit_in(const AttendParams& P, uint32_t unit) {
  const int b = sequence_of(P, unit);
  return {__ldg(P.lengths + b), P.counts ? __ldg(P.counts + b) : P.R, P.starts ? max(__ldg(P.starts + b), 0) : 0};
}
// (rows of a unit, tokens of a stage)
__device__ __forceinline__ Unit unit_of(const AttendParams& P, int ROWS, int TILE, uint32_t unit, int split, const UnitIn& in) {
  Unit u;
  u.split = split;
  const uint32_t bh = unit / static_cast<uint32_t>(P.row_tiles);
  const int mt = static_cast<int>(unit - bh * P.row_tiles);
  u.b = static_cast<int>(bh / static_cast<uint32_t>(P.heads));
  u.h = static_cast<int>(bh) - u.b * P.heads;
  u.m0 = mt * ROWS;
  u.len = in.len;
  u.n = in.n;
  u.begin = in.begin;
  u.fault = 0;
  if (u.len < 0 || u.n < 0 || u.n > P.R || static_cast<int64_t>(u.len) + u.n > static_cast<int64_t>(P.width) * P.S) {
    u.fault = LANTERN_ST_BAD_LENGTH;
    if (u.n < 0 || u.n > P.R) u.n = P.R;
    u.len = 0;
  }
  const int first = u.m0 / P.G, last = min(u.n - 1, (u.m0 + ROWS - 1) / P.G);
  u.rows = first < u.n;
  u.end = u.fault ? u.begin : u.len + last + 1;   // (an ancestor has a smaller row: trees and chains alike)
  u.tile0 = u.begin / TILE;
  const int tiles = u.end > u.begin ? (u.end + TILE - 1) / TILE - u.tile0 : 0;
  const int per = max((tiles + P.splits - 1) / P.splits, P.least);
  u.parts = max(1, (tiles + per - 1) / per);
  u.lo = split * per;
  u.hi = min(tiles, u.lo + per);
  return u;
}

// Joins the parts of a unit: a warp per row, a lane per four components; the weights of up to 32 parts are formed at once, a lane each.
constexpr int kSms = 148;
constexpr int kJoinThreads = 128;
template <int DP, bool BF16>
__global__ void __launch_bounds__(kJoinThreads) lantern_join_kernel(AttendParams P, int ROWS, int TILE) {
  using T = typename Row<BF16>::T;
  constexpr int kPerCta = kJoinThreads / 32;
  const int lane = threadIdx.x & 31;
  const uint32_t unit = blockIdx.x / (ROWS / kPerCta);
  const int row = static_cast<int>(blockIdx.x % (ROWS / kPerCta)) * kPerCta + (threadIdx.x >> 5);
  const Unit u = unit_of(P, ROWS, TILE, unit, 0, unit_in(P, unit));
  grid_dependency_wait();
  if (!u.rows || u.parts == 1 || row >= u.n * P.G - u.m0) return;
  const int64_t base = static_cast<int64_t>(unit) * P.splits;
  float M = -INFINITY;
  bool odd = false;
  for (int s = lane; s < u.parts; s += 32) {
    const float2 ml = P.part_ml[(base + s) * ROWS + row];
    M = fmaxf(M, ml.x);
    odd |= ml.y != ml.y;
  }
  M = warp_max(M);
  odd = __any_sync(kFull, odd);
  const float sub = M == -INFINITY ? 0.0f : M;
  float L = 0.0f;
  float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  const int d = lane * 4;
  for (int s0 = 0; s0 < u.parts; s0 += 32) {
    float w = 0.0f;
    if (s0 + lane < u.parts) {
      const float2 ml = P.part_ml[(base + s0 + lane) * ROWS + row];
      w = ex2_approx(ml.x - sub);
      L += ml.y * w;
    }
    const int n = min(32, u.parts - s0);
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
      const float wi = __shfl_sync(kFull, w, i);
      if (d < P.D) {
        const float4 o = *reinterpret_cast<const float4*>(P.parts + ((base + s0 + i) * ROWS + row) * DP + d);
        acc.x += o.x * wi, acc.y += o.y * wi, acc.z += o.z * wi, acc.w += o.w * wi;
      }
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) L += __shfl_xor_sync(kFull, L, o);
  const float inv = odd ? __int_as_float(0x7fffffff) : (L == 0.0f ? 0.0f : 1.0f / L);   // (nothing seen: zeros)
  if (d >= P.D) return;
  const int m = u.m0 + row, r = m / P.G;
  T* out = static_cast<T*>(P.out) + ((static_cast<int64_t>(u.b) * P.R + r) * P.q_heads + u.h * P.G + (m - r * P.G)) * P.D + d;
  const float v[4] = {acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv};
  if constexpr (BF16) *reinterpret_cast<uint2*>(out) = make_uint2(bf16x2_round(v[0], v[1]), bf16x2_round(v[2], v[3]));
  else *reinterpret_cast<float4*>(out) = make_float4(v[0], v[1], v[2], v[3]);
}

__device__ __forceinline__ void tma_load(void* dst, const CUtensorMap* map, int row, int page, uint64_t* bar) {   // x = 0: rows start on 16 bytes
  asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(smem_addr(dst)),
               "l"(map), "r"(0), "r"(row), "r"(page), "r"(smem_addr(bar))
               : "memory");
}

// Bounded wait for a phase without a suspension hint: with one, a thread that has to wait sleeps, and a tile's few waits in a row cost more
// than its products.
constexpr uint32_t kTries = 1u << 19;
__device__ __forceinline__ bool await(const AttendParams& P, uint64_t* bar, uint32_t parity) {
  const uint32_t a = smem_addr(bar);
  for (uint32_t i = 0; i < P.tries; ++i) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(a), "r"(parity)
        : "memory");
    if (ok) return true;
  }
  return false;
}

// ---- halves, NaN codes, bits ----
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
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }

// A query row's halves are its components times `mult`, which takes the largest of them (`most`) to [2^14, 2^15) and has the scale's sign, so that `factor`,
// what the products come back with, is positive.  odd: a component is not finite.
struct QueryPower {
  float mult, factor;
};
__device__ __forceinline__ QueryPower query_power(const AttendParams& P, float most, bool odd) {
  const int up = min(268 - static_cast<int>(__float_as_uint(most) >> 23), 254);   // biased exponent of the multiplier
  float mult = most == 0.0f || odd || P.scale_log2 == 0.0f ? 0.0f : __uint_as_float(static_cast<uint32_t>(up) << 23);
  if (P.scale_log2 < 0.0f) mult = -mult;
  return {mult, odd ? __int_as_float(0x7fffffff) : ldexpf(fabsf(P.scale_log2), 127 - up)};
}

// byte offset of a 16-byte chunk of a token's codes within a stage's keys or values, as the swizzled copy leaves it
template <int DP>
__device__ __forceinline__ int chunk_at(int token, int chunk) {
  return DP == 128 ? token * 128 + ((chunk ^ (token & 7)) << 4) : token * 64 + ((chunk ^ ((token >> 1) & 3)) << 4);
}
// One lane's box of a stage: where its tokens are, and their scales.
struct Box {
  int page, mine;   // mine: some row sees one of its tokens
  float ks, vs;
};
template <int TILE>
__device__ __forceinline__ Box look_up(const AttendParams& P, const Unit& u, int tile, int sub, int stop, int& fault) {
  Box x{0, 0, 1.0f, 0.0f};
  const int64_t token = static_cast<int64_t>(u.tile0 + tile) * TILE + sub;
  x.mine = tile < stop && token < u.end && token + min(P.S, TILE) > u.begin;
  if (x.mine) {
    x.page = __ldg(P.table + static_cast<int64_t>(u.b) * P.width + token / P.S);
    if (x.page < 0 || x.page >= P.pages) {
      fault |= LANTERN_ST_BAD_BLOCK;
      x.page = 0;
    }
    const int64_t block = static_cast<int64_t>(x.page) * P.heads + u.h;
    x.ks = __ldg(P.k_scale + block), x.vs = __ldg(P.v_scale + block);
  }
  return x;
}
// Host: what lantern_debug_wait_test has set for this thread (verify.cu); `tries` stays where that is nothing.
void wait_test(uint32_t* tries, int* withhold);

// Host: how a call's rows and tokens are divided.
struct Division {
  enum { kFew, kMid, kWide } kernel;
  int rows, tile, DP;    // rows per unit; tokens per stage; padded components
  int row_tiles, splits, least;
  int64_t units;
};

template <int DP, bool BF16>
static cudaError_t launch_join(const AttendParams& P, const Division& d, cudaStream_t st) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(d.units * (d.rows * 32 / kJoinThreads)));
  cfg.blockDim = dim3(kJoinThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, lantern_join_kernel<DP, BF16>, P, d.rows, d.tile);
}

// Up to 16 rows of a sequence and cache head (cache_attention_few.cu).
cudaError_t launch_attention_few(const AttendParams& P, const CUtensorMap& k, const CUtensorMap& v, const Division& d, bool bf16, cudaStream_t st);
// bf16 queries, up to 64 rows of a sequence and cache head (cache_attention_mid.cu).
cudaError_t launch_attention_mid(const AttendParams& P, const CUtensorMap& k, const CUtensorMap& v, const Division& d, cudaStream_t st);
// More than 16 rows of a sequence and cache head (cache_attention_wide.cu).
cudaError_t launch_attention_wide(const AttendParams& P, const CUtensorMap& k, const CUtensorMap& v, const Division& d, bool bf16, cudaStream_t st);

// Host: the codes as [page][head * slot][component], boxes of `tokens` rows of DP bytes (components behind D read as zero codes).
lantern_status code_map(CUtensorMap* map, const void* code, const lantern_cache* c, int DP, int tokens);

}  // namespace lantern
