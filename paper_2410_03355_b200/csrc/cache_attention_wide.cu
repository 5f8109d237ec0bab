// Attention of many rows (draft trees, chunks of prompts, grouped heads) to the paged 8-bit cache, on the fifth-generation tensor cores.
//
//   out = sum_c p_c v_c / sum_c p_c,   p_c = 2^(x_c - max x),   x_c = scale log2(e) k_scale (q . k_c)
//
// A CTA takes 128 rows of one sequence and cache head and a part of the tokens:
//   - a producer warp copies a tile of codes per stage (TMA, block by block through the table);
//   - four warps turn codes into halves (every e4m3 value is one) in the layout that the products read, values times their scale over the part's
//     largest and times 2^7, which is the room that a half leaves above 448 -- exact where scales are powers of two, as append leaves them; where a caller's are
//     not, rounded to a half's 11 bits with bf16, while with fp32 only the power of two goes with the value and the scale's digits go with the probabilities;
//   - one thread issues scores = queries . keys and output += probabilities . values, 128 rows wide, queries and probabilities out of tensor
//     memory, one tile of scores ahead of the softmax;
//   - four warps, a thread per row, take the scores from tensor memory, keep the row's running maximum and sum and put the probabilities
//     in the scores' place as halves.
// Queries go in as halves after a power of two of their own (8 bits of a bf16 query fit); fp32 queries and probabilities as two halves each
// (22 bits), in products of their own.  Accumulators are fp32.
// With at most 64 rows the second half of the 128 holds the same rows again and takes the second half of every tile's tokens (a part of its
// own, joined at the end), so that all four warps have work.
// CTAs are persistent: the producer goes on to the next unit while the softmax warps finish one, since a short unit's start and end take as long as
// its tiles.  What the other roles need to know of a tile travels with it.
//
// Bound by the softmax warps, one per scheduler and CTA, and by the instruction cache, which five roles' code shares: with all runs of tokens unrolled
// 16 trees of 61 rows, 8 heads a group of 128 components over 1200 tokens took 102 us, in loops 73 (268 TFLOP/s).  At most 64
// fp32 rows (one sequence of 32 over 100 000 tokens, 128 components: 61 us and 9 for the join) also keep the tensor pipe 46 % busy: their products are of 128
// rows and two terms, a quarter of which counts.
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

enum { kFirst = 1, kLast = 2, kEnd = 4, kEdge = 8 };   // of a tile: of its unit; there are no more; some row may not see all of its tokens

constexpr float kValueLift = 128.0f;
constexpr int kJoinRow = 68;   // (rows 16 bytes apart in the banks)
constexpr int kSlots = 8;   // units that can be under way: one per tile in the stages, in the halves and in the scores, at most
template <int DP>
struct WideShared {
  static constexpr int kTile = Shape<DP>::kTile, kStages = Shape<DP>::kStages;
  uint64_t full[kStages], empty[kStages];
  uint64_t keys_full[2], keys_free[2], values_full[2], values_free[2], scores_full[2], probs_full[2], query_full, given_up;
  float scale[kStages][2][kTile / 16];   // of every 16 tokens: keys; values, over the largest of the part, lifted
  int flags[kStages];                    // of a stage's tile
  float key_scale[4][kTile / 16];        // of the tiles whose scores are under way
  float lift[4][kTile / 16];             // fp32: kLift times the digits (1 to 2) of the value scale
  int tile_flags[4];
  uint32_t bad[4][4];                    // tokens with a NaN among their values, by converting warp
  float vref[kSlots];
  int fault[kSlots];                     // of a unit, found by the producer
  float2 ml[64];
  alignas(16) uint32_t tmem;   // (what follows in shared memory starts on 16 bytes)
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

__device__ __forceinline__ uint32_t times(uint32_t halves, __half2 ratio) {
  const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&halves), ratio);
  return *reinterpret_cast<const uint32_t*>(&r);
}
// x is a power of two (zero, or what is not finite, as it is) times its digits, 1 to 2
__device__ __forceinline__ float power_of(float x) {
  const uint32_t b = __float_as_uint(x);
  return (b & 0x7f800000u) == 0x7f800000u ? x : __uint_as_float(b & 0xff800000u);
}
__device__ __forceinline__ float digits_of(float x) { return __uint_as_float((__float_as_uint(x) & 0x7fffffu) | 0x3f800000u); }

__device__ __forceinline__ void rows_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }   // of the softmax warps
__device__ __forceinline__ bool rows_any(bool x) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(r)
               : "r"(static_cast<uint32_t>(x))
               : "memory");
  return r != 0;
}

template <int DP, bool BF16, bool TWICE>   // TWICE: at most 64 rows, see above
__global__ void __launch_bounds__(kThreads, DP == 64 ? 2 : 1) lantern_attention_wide_kernel(AttendParams P, const __grid_constant__ CUtensorMap kmap,
                                                                                         const __grid_constant__ CUtensorMap vmap) {
  using T = typename Row<BF16>::T;
  using C = Shape<DP>;
  constexpr int TILE = C::kTile, STAGES = C::kStages;
  constexpr int TERMS = BF16 ? 1 : 2, ROWS = TWICE ? 64 : 128;
  // Numerators are lifted with the argument of exp2, the sum with them (bf16: the argument's rounding is then 2^-21), or by a product (fp32).
  constexpr float kRaise = BF16 ? 10.0f : 0.0f, kSumLift = BF16 ? kLift : 1.0f;
  static_assert(kLift == 1024.0f, "2^10");
  constexpr int RUN = TILE * 128;   // bytes of 64 components of a tile of halves
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t* halves = smem + STAGES * C::kRaw;   // [2][keys, values]
  WideShared<DP>& S = *reinterpret_cast<WideShared<DP>*>(smem + C::kBytes);
  float(*join)[kJoinRow] = reinterpret_cast<float(*)[kJoinRow]>(smem + C::kBytes + sizeof(WideShared<DP>));   // TWICE: 64 components of the second half's accumulators
  uint32_t* bits = reinterpret_cast<uint32_t*>(join + (TWICE ? 64 : 0));   // [rows][words], then the nodes of a tree
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  grid_dependents_launch();
  if (tid == 0) {
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
    mbar_init(&S.given_up, 1);
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

  // The items of this CTA, one after the other: `u` is the present one's unit, `v` the next one's that has rows (and, if `tokens`, tokens) of its own.
  // What the sequences say of an item is read an item earlier.
  struct Walk {
    uint32_t item, after;
    Unit u, v;
    UnitIn ahead;
  };
  auto inputs = [&](uint32_t item) { return unit_in(P, min(item, P.items - 1) / static_cast<uint32_t>(P.splits)); };
  auto unit_at = [&](uint32_t item, const UnitIn& in) {
    const uint32_t unit = item / static_cast<uint32_t>(P.splits);
    return unit_of(P, ROWS, TILE, unit, static_cast<int>(item - unit * P.splits), in);
  };
  auto next_item = [&](Walk& w, bool tokens) {   // looks for `after`, from w.after on, whose inputs are in w.ahead
    while (w.after < P.items) {
      w.v = unit_at(w.after, w.ahead);
      const bool good = w.v.rows && w.v.split < w.v.parts && (!tokens || w.v.lo < w.v.hi);
      w.ahead = inputs(w.after + gridDim.x);
      if (good) break;
      w.after += gridDim.x;
    }
  };
  auto first_item = [&](Walk& w, bool tokens) {
    w.after = blockIdx.x;
    w.ahead = inputs(w.after);
    next_item(w, tokens);
  };
  auto advance = [&](Walk& w, bool tokens) {   // the next item becomes the present one
    w.item = w.after;
    w.u = w.v;
    w.after = min(w.item, P.items - 1) + gridDim.x;
    next_item(w, tokens);
  };

  if (warp == 8) {   // ---- producer: a lane per box of a stage; what it needs of the table is looked up a batch of stages, or a unit, ahead ----
    const int sub = min(P.S, TILE), subs = TILE / sub, batch = 32 / subs;   // tokens of a box, boxes of a stage, stages of a batch
    const int my_stage = lane / subs, my_sub = (lane - my_stage * subs) * sub;
    int n = 0, slot = 0;   // tiles, units so far
    bool ok = true;
    Walk w;
    int late = 0;   // faults of the unit whose boxes have been looked up
    Box next;
    first_item(w, true);
    if (w.after < P.items) next = look_up<TILE>(P, w.v, w.v.lo + my_stage, my_sub, w.v.hi, late);
    while (w.after < P.items && ok) {
      advance(w, true);
      const Unit &u = w.u, &v = w.v;
      const int tiles = u.hi - u.lo;
      float most = next.mine ? next.vs : 0.0f;
      for (int i = batch; i < tiles; i += batch) {   // (parts of more tiles than one batch)
        int seen = 0;
        const Box x = look_up<TILE>(P, u, u.lo + i + my_stage, my_sub, u.hi, seen);
        if (x.mine) most = fmaxf(most, x.vs);
      }
      most = warp_max(most);
      if (!BF16) most = fmaxf(power_of(most), 1.17549435e-38f);   // (so that quotients are exact)
      if (lane == 0) S.vref[slot & (kSlots - 1)] = most;
      const int first_row = u.m0 / P.G;
      int fault = late;
      Box x = next;
      for (int i = 0; i < tiles; ++i, ++n) {
        const int in_batch = i % batch;
        if (in_batch == 0) {
          x = next;
          late = 0;
          if (i + batch < tiles) next = look_up<TILE>(P, u, u.lo + i + batch + my_stage, my_sub, u.hi, late);
          else if (w.after < P.items) next = look_up<TILE>(P, v, v.lo + my_stage, my_sub, v.hi, late);
          if (i + batch < tiles) fault |= late;
        }
        const int stage = n % STAGES;
        ok = n < STAGES || await(P, &S.empty[stage], ((n / STAGES) - 1) & 1);
        ok = __all_sync(kFull, ok);
        if (!ok) break;
        const bool turn = my_stage == in_batch, mine = turn && x.mine;
        if (turn)
          for (int e = 0; e < sub / 16; ++e) {
            S.scale[stage][0][my_sub / 16 + e] = x.ks;
            S.scale[stage][1][my_sub / 16 + e] = most > 0.0f ? x.vs / most * kValueLift : 0.0f;
          }
        const int token0 = (u.tile0 + u.lo + i) * TILE;
        const int any_fault = __reduce_or_sync(kFull, fault);
        const int copies = __popc(__ballot_sync(kFull, mine));   // (at least one: every tile has a token that some row sees)
        if (lane == 0) {
          const bool edge = token0 < u.begin || token0 + TILE > u.len + (P.parents ? 0 : first_row + 1);
          S.flags[stage] = (i == 0 ? kFirst : 0) | (i == tiles - 1 ? kLast : 0) | (edge ? kEdge : 0);
          S.fault[slot & (kSlots - 1)] = any_fault;
          mbar_expect_tx(&S.full[stage], copies * 2 * sub * DP);
        }
        __syncwarp();
        if (mine && !withheld<TILE>(P, token0)) {
          uint8_t* at = smem + (stage * 2 * TILE + my_sub) * DP;
          const int row = u.h * P.S + (token0 + my_sub) % P.S;
          tma_load(at, &kmap, row, x.page, &S.full[stage]);
          tma_load(at + TILE * DP, &vmap, row, x.page, &S.full[stage]);
        }
      }
      ++slot;
    }
    // no more: a stage without copies says so; and nothing may be in flight when the CTA ends
    if (ok) {
      const int stage = n % STAGES;
      ok = n < STAGES || await(P, &S.empty[stage], ((n / STAGES) - 1) & 1);
      ok = __all_sync(kFull, ok);
      if (ok && lane == 0) {
        S.flags[stage] = kEnd;
        mbar_arrive(&S.full[stage]);
      }
    }
    // (the tile that was in the last stage before has been read: its barrier has gone on)
    for (int i = max(0, n - STAGES + (ok ? 1 : 0)); i < n; ++i) await(P, &S.full[i % STAGES], (i / STAGES) & 1);
    __syncwarp();
  } else if (warp == 9) {   // ---- products ----
    if (lane == 0) {
      const uint32_t base = smem_addr(halves);
      bool ok = true;
      int units = 0;
      auto flags_of = [&](int n) {   // waits for the tile's keys
        ok = ok && await(P, &S.keys_full[n & 1], (n >> 1) & 1);
        return ok ? S.tile_flags[n & 3] : static_cast<int>(kEnd);
      };
      auto scores = [&](int n, int flags) {
        const int k = n & 1;
        if (flags & kFirst) {
          ok = ok && await(P, &S.query_full, units & 1);
          ++units;
        }
        tmem_fence_after();
#pragma unroll
        for (int q = TERMS - 1; q >= 0; --q)   // (the small terms first: every addition to the large ones costs a rounding)
#pragma unroll
          for (int s = 0; s < DP / 16; ++s)
            multiply(tmem + C::kScores + k * TILE, tmem + C::kQuery + q * (DP / 2) + s * 8,
                     halves_at(base + k * 2 * C::kHalves + (s >> 2) * RUN + (s & 3) * 32, RUN), product(TILE, false), s > 0 || q < TERMS - 1);
        commit(&S.scores_full[k]);
        commit(&S.keys_free[k]);
        mbar_arrive(&S.scores_full[k]);   // (what the converting warps wrote beside the keys is ordered by this arrival)
      };
      int flags = flags_of(0);
      if (!(flags & kEnd)) scores(0, flags);
      for (int n = 0; ok && !(flags & kEnd); ++n) {
        const int k = n & 1, coming = flags_of(n + 1);
        // the next tile's scores go ahead of this one's output, unless they have to wait for the next unit's queries
        if (!(coming & (kEnd | kFirst))) scores(n + 1, coming);
        ok = ok && await(P, &S.probs_full[k], (n >> 1) & 1) && await(P, &S.values_full[k], (n >> 1) & 1);
        tmem_fence_after();
#pragma unroll
        for (int s = 0; s < TILE / 16; ++s)
#pragma unroll
          for (int q = 0; q < TERMS; ++q)
            multiply(tmem + C::kOutput, tmem + C::kScores + k * TILE + (s >> 1) * 32 + (s & 1) * 8 + q * 16,
                     halves_at(base + (k * 2 + 1) * C::kHalves + s * 2048, RUN), product(DP, true), !(flags & kFirst) || s + q > 0);
        commit(&S.values_free[k]);
        if (coming & kFirst) scores(n + 1, coming);
        flags = coming;
      }
      if (!ok) {   // (a wait ran out, and nobody waits for what has been issued: it ends before the tensor memory is given back)
        commit(&S.given_up);
        await(P, &S.given_up, 0);
      }
    }
    __syncwarp();
  } else if (warp >= 4 && warp < 8) {   // ---- codes to halves ----
    // a thread per token, two where a tile has 64 of them: 16 components at a time
    constexpr int SHARE = 128 / TILE, CHUNKS = DP / 16 / SHARE;
    const int who = tid - 128, token = who % TILE, share = who / TILE, w = warp - 4;
    // of the thread's first 16 codes and of the halves that they become (the others: an exclusive or away)
    const int code_from = chunk_at<DP>(token, share * CHUNKS), half_to = token * 128 + (((share * CHUNKS * 2) ^ (token & 7)) << 4);
    bool ok = true;
    for (int n = 0; ok; ++n) {
      const int k = n & 1, stage = n % STAGES, at = n & 3;
      ok = await(P, &S.full[stage], (n / STAGES) & 1);
      ok = __all_sync(kFull, ok);
      if (!ok) break;
      const int flags = S.flags[stage];
      if (tid == 128) S.tile_flags[at] = flags;
      if (flags & kEnd) {
        __syncwarp();
        if (lane == 0) mbar_arrive(&S.keys_full[k]);
        break;
      }
      const bool edge = flags & kEdge;
      const uint8_t* raw = smem + stage * C::kRaw;
      if (share == 0 && (token & 15) == 0) S.key_scale[at][token >> 4] = S.scale[stage][0][token >> 4];
      const float factor = S.scale[stage][1][token >> 4];
      const __half2 ratio = __float2half2_rn(BF16 ? factor : power_of(factor));
      if (!BF16 && share == 0 && (token & 15) == 0) S.lift[at][token >> 4] = kLift * digits_of(factor);
      bool nan = false;
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        if (n >= 2) ok = ok && await(P, which ? &S.values_free[k] : &S.keys_free[k], ((n >> 1) - 1) & 1);
        uint8_t* out = halves + (k * 2 + which) * C::kHalves;
#pragma unroll 2
        for (int c = 0; c < CHUNKS; ++c) {
          uint4 x = *reinterpret_cast<const uint4*>(raw + which * TILE * DP + (code_from ^ (c << 4)));
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
          uint8_t* row = out + (c >> 2) * RUN;
          *reinterpret_cast<uint4*>(row + (half_to ^ ((c & 3) << 5))) = make_uint4(h[0], h[1], h[2], h[3]);
          *reinterpret_cast<uint4*>(row + (half_to ^ ((c & 3) << 5) ^ 16)) = make_uint4(h[4], h[5], h[6], h[7]);
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
  } else if (warp < 4) {   // ---- softmax: a thread per row ----
    const int row = TWICE ? tid & 63 : tid, group = TWICE ? tid >> 6 : 0;
    const uint32_t lanes = tmem + (static_cast<uint32_t>(warp * 32) << 16);
    constexpr int CH = TILE / 32;   // runs of 32 tokens
    constexpr bool KEEP = TWICE;
    constexpr int MINE = TWICE ? CH / 2 : CH;   // those of this thread, from c0 on
    const int c0 = group * (CH / 2);
    const int words = (P.R + 31) >> 5;
    uint32_t* seen = bits + row * words;   // step rows that this thread's row sees
    int32_t* nodes = reinterpret_cast<int32_t*>(bits + ROWS * words);
    bool ok = true;
    int n = 0, slot = 0;   // tiles, units so far
    float factor = 0.0f;

    auto query_row = [&](const Unit& u, int r, int m) {
      return static_cast<const T*>(P.q) + u.b * P.qs.b + r * P.qs.r + (static_cast<int64_t>(u.h) * P.G + (m - r * P.G)) * P.qs.h;
    };
    auto prefetch_queries = [&](const Unit& u) {   // into L1, a unit ahead
      const int m = u.m0 + row, r = m / P.G;
      const char* p = reinterpret_cast<const char*>(query_row(u, r, m));
      if (r < u.n)
        for (int i = 0; i < P.D * static_cast<int>(sizeof(T)); i += 128) asm volatile("prefetch.global.L1 [%0];" ::"l"(p + i));
    };
    // The unit's queries as halves into tensor memory (no product reads the last unit's any more).
    auto put_queries = [&](const Unit& u) {
      const int m = u.m0 + row, r = m / P.G;
      const bool there = r < u.n;
      const T* p = query_row(u, r, m);
      constexpr int PER = 16 / sizeof(T), RUNS = DP * sizeof(T) / 128;   // components of 16 bytes; runs of 128 bytes
      uint4 raw[8];
      auto fetch = [&](int run) {   // 128 bytes of the row, all loads under way together
        if (P.vec) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            raw[i] = there && (run * 8 + i) * PER < P.D ? __ldg(reinterpret_cast<const uint4*>(p) + run * 8 + i) : make_uint4(0, 0, 0, 0);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            T t[PER];
#pragma unroll
            for (int e = 0; e < PER; ++e) {
              const int d = (run * 8 + i) * PER + e;
              t[e] = there && d < P.D ? p[d] : static_cast<T>(0.0f);
            }
            raw[i] = *reinterpret_cast<const uint4*>(t);
          }
        }
      };
      auto pair = [&](uint32_t w0, uint32_t w1, float& a, float& b) {   // two components
        if constexpr (BF16) bf16x2_widen(w0, a, b);
        else a = __uint_as_float(w0), b = __uint_as_float(w1);
      };
      float most = 0.0f;
      bool odd = false;
#pragma unroll 1
      for (int run = 0; run < RUNS; ++run) {
        fetch(run);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
          for (int e = 0; e < 4; e += BF16 ? 1 : 2) {
            float a, b;
            pair(w[e], w[BF16 ? e : e + 1], a, b);
            odd |= !(fabsf(a) < __int_as_float(0x7f800000)) | !(fabsf(b) < __int_as_float(0x7f800000));
            most = fmaxf(most, fmaxf(fabsf(a), fabsf(b)));
          }
        }
      }
      const QueryPower power = query_power(P, most, odd);
      const float mult = power.mult;
      factor = power.factor;
#pragma unroll 1
      for (int run = 0; run < RUNS; ++run) {
        if (RUNS > 1) fetch(run);
        constexpr int WORDS = 64 / sizeof(T);   // of halves in a run: 32 or 16
        uint32_t h[WORDS], l[WORDS];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
          for (int e = 0; e < 4; e += BF16 ? 1 : 2) {
            float a, b;
            pair(w[e], w[BF16 ? e : e + 1], a, b);
            a = odd ? 0.0f : a * mult, b = odd ? 0.0f : b * mult;
            const int at = i * (BF16 ? 4 : 2) + (BF16 ? e : e / 2);
            h[at] = half2_of(a, b);
            if constexpr (TERMS == 2) l[at] = half2_rest(a, b, h[at]);
          }
        }
        __syncwarp();
        if constexpr (BF16) {
          tmem_st32(lanes + C::kQuery + run * 32, h);
        } else {
          tmem_st16(lanes + C::kQuery + run * 16, h);
          tmem_st16(lanes + C::kQuery + DP / 2 + run * 16, l);
        }
      }
      tmem_st_wait();
      tmem_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&S.query_full);
    };
    // Which step rows this thread's row sees, as bits; true if a parent of the sequence is out of range.  `mine`: the parent of node tid.
    auto parent_of = [&](const Unit& u) { return tid < u.n - 1 ? __ldg(P.parents + static_cast<int64_t>(u.b) * (P.R - 1) + tid) : -1; };
    auto put_ancestors = [&](const Unit& u, int mine) {
      bool bad = false;
      rows_sync();   // (nobody walks the last unit's nodes any more)
      for (int i = tid; i < u.n - 1; i += 128) {
        const int p = i < 128 ? mine : __ldg(P.parents + static_cast<int64_t>(u.b) * (P.R - 1) + i);
        nodes[i] = p;
        bad |= p < -1 || p >= i;
      }
      const bool fault = rows_any(bad);
      int r = (u.m0 + row) / P.G;
      const bool there = r < u.n && !fault;
      if (group == 0) {   // (of two threads with the same row the first)
        if (words <= 2) {
          uint64_t x = there ? 1u : 0u;
          if (there)
            for (; r > 0; r = nodes[r - 1] + 1) x |= 1ull << r;
          seen[0] = static_cast<uint32_t>(x);
          if (words == 2) seen[1] = static_cast<uint32_t>(x >> 32);
        } else {
          for (int w = 0; w < words; ++w) seen[w] = 0;
          if (there) {
            for (; r > 0; r = nodes[r - 1] + 1) seen[r >> 5] |= 1u << (r & 31);
            seen[0] |= 1u;
          }
        }
      }
      if (TWICE) rows_sync();
      return fault;
    };

    Walk w;
    int parent = -1;
    first_item(w, false);
    if (w.after < P.items) {
      if (P.parents) parent = parent_of(w.v);
      if (w.v.lo < w.v.hi) put_queries(w.v);
    }
    while (w.after < P.items) {
      advance(w, false);
      const Unit &u = w.u, &v = w.v;
      const uint32_t item = w.item;
      const bool more = w.after < P.items;
      const int tiles = u.hi - u.lo;
      const int m = u.m0 + row, r = m / P.G;
      const bool there = r < u.n;
      int fault = u.fault;
      if (P.parents && !fault && put_ancestors(u, parent)) fault |= LANTERN_ST_BAD_PARENT;
      if (more) {
        if (P.parents) parent = parent_of(v);
        prefetch_queries(v);
      }
      const float f0 = factor;
      float ref = -INFINITY, sum = 0.0f;
      for (int i = 0; i < tiles && ok; ++i, ++n) {
        const int k = n & 1;
        ok = await(P, &S.scores_full[k], (n >> 1) & 1);
        const int token0 = (u.tile0 + u.lo + i) * TILE;
        const bool edge = S.tile_flags[n & 3] & kEdge;
        if (edge) ok = ok && await(P, &S.values_full[k], (n >> 1) & 1);
        __syncwarp();
        tmem_fence_after();
        auto factors = [&](int j, float& fa, float& fb) {   // of the two sixteens of run j of this thread's
          fa = f0 * S.key_scale[n & 3][2 * (c0 + j)], fb = f0 * S.key_scale[n & 3][2 * (c0 + j) + 1];
          if (fa < 1.17549435e-38f) fa = 1.17549435e-38f;   // (not zero: a hidden token stays at minus infinity)
          if (fb < 1.17549435e-38f) fb = 1.17549435e-38f;
        };
        auto visible = [&](int j, uint32_t& see, uint32_t& nan) {   // tokens of run j that the row sees, and those of them with a NaN among their values
          const int c = c0 + j, a = token0 + 32 * c, ahead = a - u.len;
          see = low_bits(-ahead + (P.parents ? 0 : r + 1));
          if (P.parents) {
            if (ahead >= 0) {
              const int w = ahead >> 5;
              const uint32_t lo = w < words ? seen[w] : 0u, hi = w + 1 < words ? seen[w + 1] : 0u;
              see |= __funnelshift_r(lo, hi, ahead & 31);
            } else if (ahead > -32) {
              see |= seen[0] << -ahead;
            }
          }
          see &= ~low_bits(u.begin - a);
          if (!there) see = 0u;
          nan = see & (TILE == 64 ? S.bad[n & 3][c] | S.bad[n & 3][c + 2] : S.bad[n & 3][c]);
        };
        const uint32_t scores = lanes + C::kScores + k * TILE;
        float top = -INFINITY;
        uint32_t x[KEEP ? MINE : 1][32];   // the scores, if there are registers for them
        auto get = [&](int j, uint32_t (&y)[32]) {   // run j of this thread's, hidden tokens at minus infinity
          tmem_ld32(y, scores + 32 * (c0 + j));
          if (edge) {
            uint32_t see, nan;
            visible(j, see, nan);
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              y[e] = (see >> e) & 1u ? y[e] : 0xff800000u;
              if ((nan >> e) & 1u) y[e] = 0x7fffffffu;
            }
          }
        };
        constexpr int UNROLL = KEEP ? MINE : 1;   // (code that does not fit the instruction cache costs more than a loop)
#pragma unroll UNROLL
        for (int j = 0; j < MINE; ++j) {
          uint32_t(&y)[32] = x[KEEP ? j : 0];
          get(j, y);
          float a[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, fa, fb;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            a[0] = fmaxf(a[0], __uint_as_float(y[e])), a[1] = fmaxf(a[1], __uint_as_float(y[8 + e]));
            a[2] = fmaxf(a[2], __uint_as_float(y[16 + e])), a[3] = fmaxf(a[3], __uint_as_float(y[24 + e]));
          }
          factors(j, fa, fb);
          top = fmaxf(top, fmaxf(fmaxf(a[0], a[1]) * fa, fmaxf(a[2], a[3]) * fb));
        }
        if (__any_sync(kFull, top > ref + kLag)) {   // (the probabilities' reference)
          const float to = fmaxf(ref, top), w = ref == -INFINITY ? 0.0f : ex2_approx(ref - to);
          ref = to;
          sum *= w;
          if (i > 0) {
            ok = ok && await(P, &S.values_free[(n - 1) & 1], ((n - 1) >> 1) & 1);
            __syncwarp();
            tmem_fence_after();
#pragma unroll 1
            for (int c = 0; c < DP / 32; ++c) {
              uint32_t x[32];
              tmem_ld32(x, lanes + C::kOutput + 32 * c);
#pragma unroll
              for (int e = 0; e < 32; ++e) x[e] = __float_as_uint(__uint_as_float(x[e]) * w);
              tmem_st32(lanes + C::kOutput + 32 * c, x);
            }
          }
        }
        const float base = ref == -INFINITY ? 0.0f : ref - kRaise;
        uint64_t part[2] = {pack2(0.0f, 0.0f), pack2(0.0f, 0.0f)};
        const uint64_t back = pack2(-base, -base);
#pragma unroll UNROLL
        for (int j = 0; j < MINE; ++j) {
          uint32_t(&y)[32] = x[KEEP ? j : 0];
          if (!KEEP) get(j, y);
          uint32_t h[16], l[16];
          float fa, fb;
          factors(j, fa, fb);
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const float ff = e < 16 ? fa : fb;
            float a, b;
            unpack2(fma2(pack2(__uint_as_float(y[e]), __uint_as_float(y[e + 1])), pack2(ff, ff), back), a, b);
            a = ex2_approx(a), b = ex2_approx(b);
            part[(e >> 1) & 1] = add2(part[(e >> 1) & 1], pack2(a, b));
            if constexpr (!BF16) {
              const float up = S.lift[n & 3][2 * (c0 + j) + (e < 16 ? 0 : 1)];
              unpack2(mul2(pack2(a, b), pack2(up, up)), a, b);
            }
            h[e / 2] = half2_of(a, b);
            if constexpr (TERMS == 2) l[e / 2] = half2_rest(a, b, h[e / 2]);
          }
          tmem_st16(scores + 32 * (c0 + j), h);
          if constexpr (TERMS == 2) tmem_st16(scores + 32 * (c0 + j) + 16, l);
        }
        if constexpr (TWICE) {   // the other half's tokens count for nothing in these rows
          uint32_t zero[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) zero[e] = 0u;
#pragma unroll
          for (int j = 0; j < MINE; ++j) {
            tmem_st16(scores + 32 * (CH / 2 - c0 + j), zero);
            if constexpr (TERMS == 2) tmem_st16(scores + 32 * (CH / 2 - c0 + j) + 16, zero);
          }
        }
        float even, odd;
        unpack2(add2(part[0], part[1]), even, odd);
        sum += even + odd;
        tmem_st_wait();
        tmem_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&S.probs_full[k]);
        ok = __all_sync(kFull, ok);
      }
      if (more && v.lo < v.hi && ok) put_queries(v);   // the next unit's scores can begin
      if (tiles > 0) {
        ok = ok && await(P, &S.values_free[(n - 1) & 1], ((n - 1) >> 1) & 1);
        __syncwarp();
        tmem_fence_after();
        if (ok) fault |= S.fault[slot & (kSlots - 1)];
      }
      if (!ok) fault |= LANTERN_ST_INTERNAL;
      if (fault && tid == 0 && P.status) atomicOr(P.status + u.b, fault);
      const float vref = tiles > 0 ? S.vref[slot & (kSlots - 1)] * (1.0f / (kLift * kValueLift)) : 0.0f;
      const bool whole = u.parts == 1;
      float mine = 1.0f, theirs = 0.0f;   // weights of this half's accumulators and of the other's
      float L = sum;
      const int64_t part = static_cast<int64_t>(item) * ROWS + row;
      T* out = static_cast<T*>(P.out) + ((static_cast<int64_t>(u.b) * P.R + r) * P.q_heads + u.h * P.G + (m - r * P.G)) * P.D;
      float* to = P.parts + part * DP;
      float scale = 0.0f;
      // What the last unit's rows still read: with tiles the wait for values_free says that they are done (it takes every warp's probabilities).
      if (TWICE && tiles == 0) rows_sync();
      if (TWICE && group == 1) S.ml[row] = make_float2(ref, sum);
#pragma unroll
      for (int d0 = 0; d0 < DP; d0 += 64) {   // (a thread that waits for products of the next unit is not ahead of one that still reads here)
        uint32_t y[2][32];
        __syncwarp();
        if (tiles > 0) {
          tmem_ld32(y[0], lanes + C::kOutput + d0);
          tmem_ld32(y[1], lanes + C::kOutput + d0 + 32);
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) y[0][e] = y[1][e] = 0u;
        }
        if constexpr (TWICE) {
          if (d0 > 0) rows_sync();
          if (group == 1)
#pragma unroll
            for (int e = 0; e < 64; e += 4)
              *reinterpret_cast<uint4*>(&join[row][e]) = make_uint4(y[e >> 5][e & 31], y[e >> 5][(e & 31) + 1], y[e >> 5][(e & 31) + 2], y[e >> 5][(e & 31) + 3]);
          rows_sync();
        }
        if (d0 == 0) {
          if (TWICE) {
            const float2 other = S.ml[row];
            const float M = fmaxf(ref, other.x), base = M == -INFINITY ? 0.0f : M;
            mine = ex2_approx(ref - base), theirs = ex2_approx(other.x - base);
            L = sum * mine + other.y * theirs;
            ref = M;
          }
          L *= 1.0f / kSumLift;
          scale = whole ? (L == 0.0f ? 0.0f : vref / L) : vref;
        }
        if (group == 0 && there) {
#pragma unroll
          for (int e = 0; e < 64; e += 8) {
            const int d = d0 + e;
            float x[8], other[8];
            if constexpr (TWICE) Row<false>::get8(&join[row][e], other);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              x[i] = __uint_as_float(y[(e + i) >> 5][(e + i) & 31]);
              if (TWICE) x[i] = x[i] * mine + other[i] * theirs;
              x[i] = fault ? __int_as_float(0x7fffffff) : x[i] * scale;
            }
            if (d < P.D) {
              if (whole) {
                Row<BF16>::put8(out + d, x);
              } else {
                *reinterpret_cast<float4*>(to + d) = make_float4(x[0], x[1], x[2], x[3]);
                *reinterpret_cast<float4*>(to + d + 4) = make_float4(x[4], x[5], x[6], x[7]);
              }
            }
          }
        }
      }
      if (group == 0 && there && !whole) P.part_ml[part] = make_float2(ref, fault ? __int_as_float(0x7fffffff) : L);
      if (tiles > 0) ++slot;
    }
  }
  tmem_fence_before();
  __syncthreads();
  if (warp == 9) {
    tmem_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::kColumns) : "memory");
  }
}

template <int DP, bool BF16, bool TWICE>
cudaError_t launch(const AttendParams& P, const CUtensorMap& k, const CUtensorMap& v, const Division& d, cudaStream_t st) {
  constexpr size_t kFixed = Shape<DP>::kBytes + sizeof(WideShared<DP>) + (TWICE ? 64 * kJoinRow * sizeof(float) : 0);
  constexpr size_t kMost = kFixed + ((TWICE ? 64 : 128) * 33 + kMaxTreeRows) * 4;
  static_assert(kMost <= 227 * 1024, "shared memory");
  const size_t smem = kFixed + (P.parents ? (static_cast<size_t>(TWICE ? 64 : 128) * ((P.R + 31) / 32) + P.R) * 4 : 0);
  static DeviceFlags ready;
  cudaError_t e = allow_shared_memory(lantern_attention_wide_kernel<DP, BF16, TWICE>, kMost, ready);
  if (e != cudaSuccess) return e;
  const int64_t items = d.units * d.splits, slots = static_cast<int64_t>(kSms) * (DP == 64 ? 2 : 1);
  lantern_attention_wide_kernel<DP, BF16, TWICE><<<static_cast<unsigned>(items < slots ? items : slots), kThreads, smem, st>>>(P, k, v);
  if ((e = cudaGetLastError()) != cudaSuccess || d.splits == 1) return e;
  return launch_join<DP, BF16>(P, d, st);
}

}  // namespace

cudaError_t launch_attention_wide(const AttendParams& P, const CUtensorMap& k, const CUtensorMap& v, const Division& d, bool bf16, cudaStream_t st) {
  if (d.rows == 64) {
    if (d.DP == 64) return bf16 ? launch<64, true, true>(P, k, v, d, st) : launch<64, false, true>(P, k, v, d, st);
    return bf16 ? launch<128, true, true>(P, k, v, d, st) : launch<128, false, true>(P, k, v, d, st);
  }
  if (d.DP == 64) return bf16 ? launch<64, true, false>(P, k, v, d, st) : launch<64, false, false>(P, k, v, d, st);
  return bf16 ? launch<128, true, false>(P, k, v, d, st) : launch<128, false, false>(P, k, v, d, st);
}

}  // namespace lantern
