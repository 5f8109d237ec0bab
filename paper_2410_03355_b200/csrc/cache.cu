// The paged 8-bit cache of keys and values: appending rows (keys rotated on the way), keeping an accepted path, reading back.
//
// A block (page, head) has one scale for its keys and one for its values.  Scales are powers of two, so that taking a larger one moves the
// codes' exponents and loses nothing but bits that fall below the smallest normal code.
#include "cache_common.cuh"

namespace lantern {

struct CacheView {
  uint8_t* code[2];    // keys, values
  float* scale[2];
  const int32_t* table;
  int pages, heads, S, D, width;
  __device__ __forceinline__ int64_t block(int page, int head) const { return static_cast<int64_t>(page) * heads + head; }
  __device__ __forceinline__ uint8_t* row(int which, int page, int head, int slot) const {
    return code[which] + ((block(page, head) * S) + slot) * D;
  }
};
static CacheView view_of(const lantern_cache* c, const int32_t* table, int width) {
  return {{static_cast<uint8_t*>(c->k_code), static_cast<uint8_t*>(c->v_code)}, {c->k_scale, c->v_scale}, table,
          c->pages, c->heads, c->page_tokens, c->head_dim, width};
}

__device__ __forceinline__ uint2 recode8(uint2 codes, float ratio) {   // codes * ratio, ratio <= 1
  float a[4], b[4];
  decode4(codes.x, a), decode4(codes.y, b);
  return make_uint2(encode4(a[0] * ratio, a[1] * ratio, a[2] * ratio, a[3] * ratio), encode4(b[0] * ratio, b[1] * ratio, b[2] * ratio, b[3] * ratio));
}

// ---- append -------------------------------------------------------------------------------------------------------------

struct AppendParams {
  CacheView c;
  const void* x[2];
  RowStride xs[2];
  Rotation rot;
  const int32_t* lengths;
  const int32_t* counts;
  int32_t* status;
  int B, R;
  int vec;             // rows may be read eight components at a time
  int heads_per_cta;
};

// What of block j (the j-th that the sequence's rows touch) is new: slots [low, high), the first of them row `row`; held slots ahead of them.
struct Span {
  int page, low, high, row, fault;
};
__device__ __forceinline__ Span append_span(const AppendParams& P, int b, int j) {
  Span s{0, 0, 0, 0, 0};
  const int len = __ldg(P.lengths + b), n = P.counts ? __ldg(P.counts + b) : P.R;
  if (len < 0 || n < 0 || n > P.R || static_cast<int64_t>(len) + n > static_cast<int64_t>(P.c.width) * P.c.S) {
    s.fault = LANTERN_ST_BAD_LENGTH;
    return s;
  }
  const int S = P.c.S, block = len / S + j;
  const int64_t first = static_cast<int64_t>(block) * S;
  if (first >= static_cast<int64_t>(len) + n) return s;   // (nothing: low == high)
  const int page = __ldg(P.c.table + static_cast<int64_t>(b) * P.c.width + block);
  if (page < 0 || page >= P.c.pages) {
    s.fault = LANTERN_ST_BAD_BLOCK;
    return s;
  }
  s.page = page;
  s.low = j == 0 ? len - static_cast<int>(first) : 0;
  const int64_t left = static_cast<int64_t>(len) + n - first;
  s.high = left < S ? static_cast<int>(left) : S;
  s.row = j == 0 ? 0 : static_cast<int>(first - len);
  return s;
}

// Eight components as they lie in memory.
template <bool BF16>
struct Raw {
  uint4 w[BF16 ? 1 : 2];
};
template <bool BF16>
__device__ __forceinline__ Raw<BF16> raw8(const typename Row<BF16>::T* p) {
  Raw<BF16> r;
#pragma unroll
  for (int i = 0; i < (BF16 ? 1 : 2); ++i) r.w[i] = __ldg(reinterpret_cast<const uint4*>(p) + i);
  return r;
}
template <bool BF16>
__device__ __forceinline__ void widen8(const Raw<BF16>& r, float (&v)[8]) {
  if constexpr (BF16) {
    bf16x2_widen(r.w[0].x, v[0], v[1]), bf16x2_widen(r.w[0].y, v[2], v[3]), bf16x2_widen(r.w[0].z, v[4], v[5]), bf16x2_widen(r.w[0].w, v[6], v[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      v[4 * i] = __uint_as_float(r.w[i].x), v[4 * i + 1] = __uint_as_float(r.w[i].y), v[4 * i + 2] = __uint_as_float(r.w[i].z), v[4 * i + 3] = __uint_as_float(r.w[i].w);
  }
}
// A row of the table of cosines and sines has its pairs two by two (16 bytes), exchanged among eights so that neighbours, which read eight pairs (or
// four) each, find different banks.  Rows are padded to eights.
__device__ __forceinline__ int eights(int pairs) { return (pairs + 7) & ~7; }
__device__ __forceinline__ int place_of(int pair) { return pair ^ (((pair >> 4) & 3) << 1); }
__device__ __forceinline__ float4 two_angles(const float2* table, int pair) { return *reinterpret_cast<const float4*>(table + place_of(pair)); }   // pair even
// Eight keys turned: v their components from d on, o their partners' in the other half (if not interleaved).
__device__ __forceinline__ void turn8(const Rotation& rot, int d, const float2* table, float (&v)[8], const float (&o)[8]) {
  const int pairs = rot.pairs;
  if (d >= 2 * pairs) return;
  if (rot.interleaved) {
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      const float4 ww = two_angles(table, (d + i) >> 1);
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        if (d + i + e < 2 * pairs) {
          const float2 w = e ? make_float2(ww.z, ww.w) : make_float2(ww.x, ww.y);
          const float a = v[i + e], b = v[i + e + 1];
          v[i + e] = turned_low(a, b, w);
          v[i + e + 1] = turned_high(a, b, w);
        }
      }
    }
  } else {
    const bool lower = d < pairs;
    const int j = lower ? d : d - pairs;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float4 ww = two_angles(table, j + i);
      const float2 w0 = make_float2(ww.x, ww.y), w1 = make_float2(ww.z, ww.w);
      v[i] = lower ? turned_low(v[i], o[i], w0) : turned_high(o[i], v[i], w0);
      v[i + 1] = lower ? turned_low(v[i + 1], o[i + 1], w1) : turned_high(o[i + 1], v[i + 1], w1);
    }
  }
}

// Components [d, d + 8) of a row of keys (turned) or values.  table: cosines and sines of the row's pairs, NULL = not rotated.
template <bool BF16>
__device__ __forceinline__ void new_values(const AppendParams& P, const typename Row<BF16>::T* p, int d, const float2* table, float (&v)[8]) {
  if (P.vec) {
    Row<BF16>::get8(p + d, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = Row<BF16>::get(p + d + i);
  }
  if (!table) return;
  const int pairs = P.rot.pairs;
  if (d >= 2 * pairs) return;
  if (P.rot.interleaved) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      if (d + i < 2 * pairs) {
        const float2 w = table[place_of((d + i) >> 1)];
        const float a = v[i], b = v[i + 1];
        v[i] = turned_low(a, b, w);
        v[i + 1] = turned_high(a, b, w);
      }
    }
  } else if (P.vec && pairs % 8 == 0) {   // the eight lie in one half, their partners in the other
    float o[8];
    const bool lower = d < pairs;
    const int j = lower ? d : d - pairs;
    Row<BF16>::get8(p + (lower ? d + pairs : d - pairs), o);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 w = table[place_of(j + i)];
      v[i] = lower ? turned_low(v[i], o[i], w) : turned_high(o[i], v[i], w);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (d + i < 2 * pairs) {
        const bool lower = d + i < pairs;
        const int j = lower ? d + i : d + i - pairs;
        const float2 w = table[place_of(j)];
        const float o = Row<BF16>::get(p + (lower ? d + i + pairs : j));
        v[i] = lower ? turned_low(v[i], o, w) : turned_high(o, v[i], w);
      }
    }
  }
}
// Largest finite magnitude; `odd` is set if one of them is not finite, which then becomes NaN.  (As integers, magnitudes order like floats and
// everything that is not finite comes last.)
__device__ __forceinline__ float magnitude(float (&v)[8], int& odd) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
  if (m >= 0x7f800000u) {
    odd = 1;
    m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t x = __float_as_uint(v[i]) & 0x7fffffffu;
      if (x < 0x7f800000u) m = max(m, x);
      else v[i] = __int_as_float(0x7fffffff);
    }
  }
  return __uint_as_float(m);
}
// eight values' codes under a scale
__device__ __forceinline__ uint2 encode8(const float (&v)[8], const Divider& over) {
  if (over.exact) {
    const float k = over.inverse;
    return make_uint2(encode4(v[0] * k, v[1] * k, v[2] * k, v[3] * k), encode4(v[4] * k, v[5] * k, v[6] * k, v[7] * k));
  }
  return make_uint2(encode4(over(v[0]), over(v[1]), over(v[2]), over(v[3])), encode4(over(v[4]), over(v[5]), over(v[6]), over(v[7])));
}
// the scale that the block gets
__device__ __forceinline__ float new_scale(float amax, float old, bool held, int& odd) {
  const float need = scale_for(amax);
  if (!held) return need;
  if (!usable_scale(old)) {
    odd = 1;
    return need;
  }
  return fmaxf(need, old);
}

// A CTA per touched block, run of heads and kind (keys or values): a block's angles are formed once for the heads of the run, then every head goes through
// registers, U units of eight components per thread: maximum over the block, scale, codes.  Bound by the latency of a head's reads, the
// maximum and the writes one after the other, and (keys) by the angles' arithmetic (32 prompts of 0 to 1024 rows, 8 heads of 128: 58 us for 100 MB;
// of rows that L2 holds 48, 33 without rotation, 53 with the angles in their order, eight threads to a bank; with angles formed in double precision and a read at a time 81;
// both kinds in one CTA 69; the next head's reads under way ahead of this one's maximum: fp32 blocks of 32 tokens 74 -> 82 with the read, for registers).
template <bool BF16, int AT, int U>   // AT threads
__global__ void __launch_bounds__(AT, (U == 1 ? 5 : U == 2 ? 4 : 2) * 256 / AT) lantern_append_kernel(AppendParams P) {
  using T = typename Row<BF16>::T;
  extern __shared__ __align__(16) float2 angles[];   // [new slots][eights of pairs]
  __shared__ float most[2][AT / 32];
  __shared__ uint64_t steps[kMaxHeadDim / 2];
  const int b = blockIdx.z, j = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int which = blockIdx.x & 1, h0 = (blockIdx.x >> 1) * P.heads_per_cta, h1 = min(h0 + P.heads_per_cta, P.c.heads);
  const Span s = append_span(P, b, j);
  if (s.fault && tid == 0 && P.status) atomicOr(P.status + b, s.fault);
  const int n = s.high - s.low;
  if (s.fault || n <= 0) return;
  const bool turns = P.rot.inv_freq != nullptr && which == 0;
  const int pairs = turns ? P.rot.pairs : 1;
  if (turns) {
    for (int i = tid; i < pairs; i += AT) steps[i] = turn_step(P.rot, i);
    __syncthreads();
    const int at_once = AT / pairs, t0 = tid / pairs, k = tid - t0 * pairs;   // (at most 64 pairs)
    const uint64_t step = steps[k];
    if (t0 < at_once)
#pragma unroll 2
      for (int t = t0; t < n; t += at_once) angles[t * eights(pairs) + place_of(k)] = turn_by(step, position_of(P.rot, static_cast<int64_t>(b) * P.R + s.row + t, k));
  }
  // A thread keeps its eight components d.. of a row and goes through rows t0, t0 + at_once, ...
  const int D = P.c.D, per_row = D >> 3, at_once = AT / per_row, t0 = tid / per_row, d = (tid - t0 * per_row) * 8;
  const bool works = t0 < at_once;
  const bool partners = turns && !P.rot.interleaved;
  const int partner = d < pairs ? pairs : d < 2 * pairs ? -pairs : 0;   // where the other half of the pairs is
  int odd = 0, turn_of = 0;
  for (int h = h0; h < h1; ++h) {
    {
      const T* x = static_cast<const T*>(P.x[which]) + b * P.xs[which].b + h * P.xs[which].h;
      float v[U][8], m = 0.0f;
      if (P.vec && (!partners || pairs % 8 == 0)) {   // all reads of the head are under way before the first is used
        Raw<BF16> own[U], other[U];
        const T* p = x + s.row * P.xs[which].r + d;
        const int64_t stride = P.xs[which].r;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int t = min(t0 + u * at_once, n - 1);
          own[u] = raw8<BF16>(p + t * stride);
          if (partners) other[u] = raw8<BF16>(p + t * stride + partner);
        }
        if (turn_of == 0) __syncthreads();   // the angles are there
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int t = t0 + u * at_once;
          if (works && t < n) {
            widen8<BF16>(own[u], v[u]);
            if (turns) {
              float o[8];
              if (partners) widen8<BF16>(other[u], o);
              turn8(P.rot, d, angles + t * eights(pairs), v[u], o);
            }
            m = fmaxf(m, magnitude(v[u], odd));
          }
        }
      } else {
        if (turn_of == 0) __syncthreads();
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int t = t0 + u * at_once;
          if (works && t < n) {
            new_values<BF16>(P, x + (s.row + t) * P.xs[which].r, d, turns ? angles + t * eights(pairs) : nullptr, v[u]);
            m = fmaxf(m, magnitude(v[u], odd));
          }
        }
      }
      m = warp_max(m);
      float* mine = most[turn_of & 1];
      if (lane == 0) mine[warp] = m;
      const int64_t block = P.c.block(s.page, h);
      const float old = P.c.scale[which][block];
      __syncthreads();   // (also: everybody has read the scale; the other buffer's readers are through)
#pragma unroll
      for (int w = 0; w < AT / 32; ++w) m = fmaxf(m, mine[w]);
      const float scale = new_scale(m, old, s.low > 0, odd);
      const Divider over = divider(scale);
      uint8_t* to = P.c.row(which, s.page, h, s.low) + d;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int t = t0 + u * at_once;
        if (works && t < n) *reinterpret_cast<uint2*>(to + t * D) = encode8(v[u], over);
      }
      if (s.low > 0 && scale != old) {   // what the block holds is coded anew
        const float ratio = usable_scale(old) ? old / scale : 0.0f;
        uint2* held = reinterpret_cast<uint2*>(P.c.row(which, s.page, h, 0));
        for (int i = tid; i < s.low * per_row; i += AT) held[i] = recode8(held[i], ratio);
      }
      if (tid == 0 && scale != old) P.c.scale[which][block] = scale;
      ++turn_of;
    }
  }
  if (odd && P.status) atomicOr(P.status + b, LANTERN_ST_NONFINITE);
}

// Few rows a sequence: a warp per touched block, head and kind.  The rows are read twice (the second time from L1); angles are formed by the
// lane that needs them.  Bound by latency: 128 sequences of one row, 8 heads of 128: 6.6 us, most of it the launch, where the blocks' scales stay; 14.5 where all
// grow and 32 held tokens of a block on average are coded anew, 8 bytes a lane at a time (21 with blocks of 128 tokens).
constexpr int FT = 128;
template <bool BF16>
__global__ void __launch_bounds__(FT) lantern_append_few_kernel(AppendParams P) {
  using T = typename Row<BF16>::T;
  __shared__ __align__(16) float2 angles[FT / 32][kMaxHeadDim / 2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int item = blockIdx.x * (FT / 32) + warp;   // (head, kind)
  const int b = blockIdx.z, j = blockIdx.y;
  if (item >= 2 * P.c.heads) return;
  const int which = item & 1, h = item >> 1;
  const Span s = append_span(P, b, j);
  if (s.fault && item == 0 && lane == 0 && P.status) atomicOr(P.status + b, s.fault);
  const int n = s.high - s.low;
  if (s.fault || n <= 0) return;
  const int D = P.c.D, per_row = D >> 3;
  const bool rotate = P.rot.inv_freq != nullptr && which == 0;
  uint64_t step[kMaxHeadDim / 64];   // of the pairs that this lane turns
#pragma unroll
  for (int e = 0; e < kMaxHeadDim / 64; ++e) step[e] = rotate && lane + 32 * e < P.rot.pairs ? turn_step(P.rot, lane + 32 * e) : 0;
  const T* x = static_cast<const T*>(P.x[which]) + b * P.xs[which].b + h * P.xs[which].h;
  const int64_t block = P.c.block(s.page, h);
  const float old = P.c.scale[which][block];
  int odd = 0;
  float m = 0.0f, v[8];
  auto values = [&](int t) {   // row t's eight components of this lane (per_row <= 16 lanes take part)
    const T* p = x + (s.row + t) * P.xs[which].r;
    if (rotate) {
      __syncwarp();
#pragma unroll
      for (int e = 0; e < kMaxHeadDim / 64; ++e) {
        const int i = lane + 32 * e;
        if (i < P.rot.pairs) angles[warp][place_of(i)] = turn_by(step[e], position_of(P.rot, static_cast<int64_t>(b) * P.R + s.row + t, i));
      }
      __syncwarp();
    }
    if (lane < per_row) new_values<BF16>(P, p, lane * 8, rotate ? angles[warp] : nullptr, v);
    return lane < per_row ? magnitude(v, odd) : 0.0f;
  };
  for (int t = 0; t < n; ++t) m = fmaxf(m, values(t));
  m = warp_max(m);
  const float scale = new_scale(m, old, s.low > 0, odd);
  const Divider over = divider(scale);
  for (int t = n - 1; t >= 0; --t) {
    if (t != n - 1) values(t);   // (the last row's are still there)
    if (lane < per_row)
      *reinterpret_cast<uint2*>(P.c.row(which, s.page, h, s.low + t) + lane * 8) = encode8(v, over);
  }
  if (s.low > 0 && scale != old) {
    const float ratio = usable_scale(old) ? old / scale : 0.0f;
    uint2* held = reinterpret_cast<uint2*>(P.c.row(which, s.page, h, 0));
    for (int i = lane; i < s.low * per_row; i += 32) held[i] = recode8(held[i], ratio);
  }
  if (lane == 0 && scale != old) P.c.scale[which][block] = scale;
  if (odd && P.status) atomicOr(P.status + b, LANTERN_ST_NONFINITE);
}

template <bool BF16, int AT, int U>
static cudaError_t launch_append(const AppendParams& P, dim3 grid, size_t smem, cudaStream_t st) {
  static DeviceFlags ready;
  const cudaError_t e = allow_shared_memory(lantern_append_kernel<BF16, AT, U>, 128 * (kMaxHeadDim / 2) * sizeof(float2), ready);
  if (e != cudaSuccess) return e;
  lantern_append_kernel<BF16, AT, U><<<grid, AT, smem, st>>>(P);
  return cudaGetLastError();
}

// ---- keep ---------------------------------------------------------------------------------------------------------------

struct KeepParams {
  CacheView c;
  const int32_t* lengths;
  const int32_t* accept_len;
  const int32_t* path;
  int32_t* out_lengths;
  int32_t* status;
  int N;
};

// A warp per sequence, head and kind.  Targets ascend and no target lies behind its source (a path is increasing), so that going through the
// targets in order, block by block, never overwrites a source that is still needed.  Bound by latency: accepted path, table, scale, code one after the
// other (256 trees, 20 heads: 16 us with nothing in L2).
constexpr int KT = 128;
__global__ void __launch_bounds__(KT) lantern_keep_kernel(KeepParams P) {
  const int lane = threadIdx.x & 31;
  const int item = blockIdx.x * (KT / 32) + (threadIdx.x >> 5), b = blockIdx.y;
  if (item >= 2 * P.c.heads) return;
  const int which = item & 1, h = item >> 1, S = P.c.S, D = P.c.D, N = P.N;
  const int32_t* path = P.path + static_cast<int64_t>(b) * N;
  const int32_t* table = P.c.table + static_cast<int64_t>(b) * P.c.width;
  const int len = __ldg(P.lengths + b), n = __ldg(P.accept_len + b);
  int fault = 0, moved = 0;   // moved: some token of the path moves
  if (len < 0) fault |= LANTERN_ST_BAD_LENGTH;
  if (n < 0 || n > N) fault |= LANTERN_ST_BAD_PATH;
  if (!fault) {
    const int64_t room = static_cast<int64_t>(P.c.width) * S;
    if (static_cast<int64_t>(len) + 1 + n > room) fault |= LANTERN_ST_BAD_LENGTH;
    for (int i = lane; i < n; i += 32) {
      const int at = __ldg(path + i), before = i ? __ldg(path + i - 1) : -1;
      if (at <= before || at < 0 || at >= N) {
        fault |= LANTERN_ST_BAD_PATH;
      } else if (at != i) {
        moved = 1;
        const int64_t from = static_cast<int64_t>(len) + 1 + at, to = static_cast<int64_t>(len) + 1 + i;
        if (from >= room || to >= room) {
          fault |= LANTERN_ST_BAD_LENGTH;
        } else if (static_cast<unsigned>(__ldg(table + from / S)) >= static_cast<unsigned>(P.c.pages) ||
                   static_cast<unsigned>(__ldg(table + to / S)) >= static_cast<unsigned>(P.c.pages)) {
          fault |= LANTERN_ST_BAD_BLOCK;
        }
      }
    }
  }
  fault = __reduce_or_sync(kFull, fault);
  moved = __any_sync(kFull, moved);
  if (item == 0 && lane == 0) {
    P.out_lengths[b] = fault ? len : len + 1 + n;
    if (fault && P.status) atomicOr(P.status + b, fault);
  }
  if (fault || !moved) return;
  const int first = len + 1, vecs = D >> 4;   // 16 bytes of a row per lane, 32 / vecs rows at a time
  const int rows = 32 / vecs, sub = lane / vecs, at = lane - sub * vecs;
  for (int j0 = 0; j0 < n;) {   // targets [j0, j1) of one block
    const int block = (first + j0) / S, j1 = min(n, (block + 1) * S - first);
    const int page = __ldg(table + block);
    float* own = P.c.scale[which] + P.c.block(page, h);
    float most = 0.0f;
    int moves = 0;
    for (int j = j0 + lane; j < j1; j += 32) {
      const int from = __ldg(path + j);
      moves |= from != j;
      if (from != j) most = fmaxf(most, P.c.scale[which][P.c.block(__ldg(table + (first + from) / S), h)]);
    }
    most = warp_max(most);
    if (__any_sync(kFull, moves)) {
      const float old = *own, scale = fmaxf(old, most);
      __syncwarp();
      if (scale != old) {
        const float ratio = old / scale;
        uint2* held = reinterpret_cast<uint2*>(P.c.row(which, page, h, 0));
        for (int i = lane; i < S * D / 8; i += 32) held[i] = recode8(held[i], ratio);
        if (lane == 0) *own = scale;
        __syncwarp();
      }
      for (int j = j0; j < j1; j += rows) {
        const int mine = j + sub;
        const int from = sub < rows && mine < j1 ? __ldg(path + mine) : mine;
        uint4 c = make_uint4(0, 0, 0, 0);
        if (from != mine) {
          const int token = first + from, source = __ldg(table + token / S);
          c = *reinterpret_cast<const uint4*>(P.c.row(which, source, h, token % S) + at * 16);
          const float theirs = source == page ? scale : P.c.scale[which][P.c.block(source, h)];
          if (theirs != scale) {
            const float ratio = theirs / scale;
            const uint2 lo = recode8(make_uint2(c.x, c.y), ratio), hi = recode8(make_uint2(c.z, c.w), ratio);
            c = make_uint4(lo.x, lo.y, hi.x, hi.y);
          }
        }
        __syncwarp();   // the sources of these rows are read before a row is written
        if (from != mine) *reinterpret_cast<uint4*>(P.c.row(which, page, h, (first + mine) % S) + at * 16) = c;
        __syncwarp();
      }
    }
    j0 = j1;
  }
}

// ---- read ---------------------------------------------------------------------------------------------------------------

struct ReadParams {
  CacheView c;
  const int32_t* first;
  const int32_t* counts;
  int32_t* status;
  void* out[2];
  int B, R;
  int units;   // of a sequence: R * heads * D / 16
};

// A thread per 16 components of a row, keys and values.  Bound by HBM: one byte in, two or four out (32 contexts of 4000 tokens, 8 heads of 128,
// bf16: 146 us, 5.4 TB/s; 8 components a thread and two rows 154, 16 and two rows 158).
constexpr int DT = 256;
template <bool BF16>
__global__ void __launch_bounds__(DT) lantern_read_kernel(ReadParams P) {
  using T = typename Row<BF16>::T;
  const int i = blockIdx.x * DT + threadIdx.x;
  if (i >= P.units) return;
  const int vecs = P.c.D >> 4, per_row = P.c.heads * vecs;
  const int r = i / per_row, rest = i - r * per_row, h = rest / vecs, d = (rest - h * vecs) * 16;
  for (int b = blockIdx.y; b < P.B; b += gridDim.y) {
  const int first = __ldg(P.first + b), n = P.counts ? __ldg(P.counts + b) : P.R;
  int fault = 0, page = 0;
  const int64_t token = static_cast<int64_t>(first) + r;
  if (first < 0 || n < 0 || n > P.R || static_cast<int64_t>(first) + n > static_cast<int64_t>(P.c.width) * P.c.S) {
    fault = LANTERN_ST_BAD_LENGTH;
  } else if (r >= n) {
    continue;
  } else {
    page = __ldg(P.c.table + static_cast<int64_t>(b) * P.c.width + token / P.c.S);
    if (page < 0 || page >= P.c.pages) fault = LANTERN_ST_BAD_BLOCK;
  }
  if (fault && rest == 0 && P.status) atomicOr(P.status + b, fault);
  uint4 c[2];
  float scale[2];
#pragma unroll
  for (int which = 0; which < 2; ++which) {   // (both reads under way before either is used)
    c[which] = fault ? make_uint4(0x7f7f7f7f, 0x7f7f7f7f, 0x7f7f7f7f, 0x7f7f7f7f)
                     : *reinterpret_cast<const uint4*>(P.c.row(which, page, h, static_cast<int>(token % P.c.S)) + d);
    scale[which] = fault ? 1.0f : P.c.scale[which][P.c.block(page, h)];
  }
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float v[16];
    const uint32_t w[4] = {c[which].x, c[which].y, c[which].z, c[which].w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float x[4];
      decode4(w[q], x);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * q + e] = x[e] * scale[which];
    }
    T* out = static_cast<T*>(P.out[which]) + (static_cast<int64_t>(b) * P.units + i) * 16;
    const float lo[8] = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]}, hi[8] = {v[8], v[9], v[10], v[11], v[12], v[13], v[14], v[15]};
    Row<BF16>::put8(out, lo);
    Row<BF16>::put8(out + 8, hi);
  }
  }
}

}  // namespace lantern

using namespace lantern;

extern "C" lantern_status lantern_cache_append(const void* k, const void* v, int dtype, int B, int R, const int64_t k_stride[3],
                                               const int64_t v_stride[3], const lantern_cache* cache, const int32_t* table, int table_width,
                                               const int32_t* lengths, const int32_t* counts, const lantern_rotation* rotation, int32_t* status,
                                               void* cuda_stream) {
  if (dtype != LANTERN_F32 && dtype != LANTERN_BF16) return LANTERN_E_PARAM;
  lantern_status bad = check_cache(cache, table, table_width, B);
  if (bad != LANTERN_OK) return bad;
  if (B < 0 || B > 65535 || R < 0) return LANTERN_E_SHAPE;
  AppendParams P;
  P.rot.inv_freq = nullptr;
  if (rotation && (bad = make_rotation(rotation, B, R, cache->head_dim, &P.rot)) != LANTERN_OK) return bad;
  if (B == 0 || R == 0) return LANTERN_OK;
  if (!k || !v || !k_stride || !v_stride || !lengths) return LANTERN_E_NULL;
  const int S = cache->page_tokens, D = cache->head_dim, H = cache->heads, size = dtype == LANTERN_BF16 ? 2 : 4;
  if (reinterpret_cast<uintptr_t>(k) % size || reinterpret_cast<uintptr_t>(v) % size) return LANTERN_E_ALIGN;
  const int64_t touched = R == 1 ? 1 : (static_cast<int64_t>(R) + S - 2) / S + 1;   // blocks that R rows can touch
  if (touched > 65535) return LANTERN_E_SHAPE;
  P.c = view_of(cache, table, table_width);
  P.x[0] = k;
  P.x[1] = v;
  P.xs[0] = {k_stride[0], k_stride[1], k_stride[2]};
  P.xs[1] = {v_stride[0], v_stride[1], v_stride[2]};
  P.lengths = lengths;
  P.counts = counts;
  P.status = status;
  P.B = B;
  P.R = R;
  const int64_t ks[3] = {k_stride[0], k_stride[1], k_stride[2]}, vs[3] = {v_stride[0], v_stride[1], v_stride[2]};
  P.vec = aligned16(k, ks, size) && aligned16(v, vs, size);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const bool bf = dtype == LANTERN_BF16;
  cudaError_t e;
  // Up to 4 rows a warp per block, head and kind, else a CTA per block and run of heads (8 heads of 128, with the read: 128 sequences of 1 row 17 us, by CTAs
  // 32; of 4 rows 24 and 31; of 5 26 and 31, of 8 31 and 33, of 16 47 and 37.  2 sequences of 1 row 9.3 and 10.3, of 4 13.7 and 10.8, of 8 20 and 10.8).
  if (R <= 4) {
    const dim3 grid((2 * H + FT / 32 - 1) / (FT / 32), static_cast<unsigned>(touched), B);
    if (bf) lantern_append_few_kernel<true><<<grid, FT, 0, st>>>(P);
    else lantern_append_few_kernel<false><<<grid, FT, 0, st>>>(P);
    e = cudaGetLastError();
  } else {
    // Heads share a block's angles: as many per CTA as leave eight CTAs per SM, four at most.
    const int64_t per = static_cast<int64_t>(B) * touched * 2 * H / (8 * 148), most = H < 4 ? H : 4;
    P.heads_per_cta = static_cast<int>(per < 1 ? 1 : per > most ? most : per);
    const dim3 grid(2 * ((H + P.heads_per_cta - 1) / P.heads_per_cta), static_cast<unsigned>(touched), B);
    const size_t smem = rotation ? static_cast<size_t>(S) * ((P.rot.pairs + 7) & ~7) * sizeof(float2) : 0;
    // Units of eight components for each of 256 threads: at most 8.  Where they take so many registers that a CTA leaves no room for others, 512 threads
    // (with the read, fp32 blocks of 64 tokens of 128: 85 -> 82 us, bf16 ones of 128: 103 -> 91; bf16 of 64: 75 and 76).
    const int u = (S + 256 / (D / 8) - 1) / (256 / (D / 8));
    if (u <= 1) e = bf ? launch_append<true, 256, 1>(P, grid, smem, st) : launch_append<false, 256, 1>(P, grid, smem, st);
    else if (u <= 2) e = bf ? launch_append<true, 256, 2>(P, grid, smem, st) : launch_append<false, 256, 2>(P, grid, smem, st);
    else if (u <= 4) e = bf ? launch_append<true, 256, 4>(P, grid, smem, st) : launch_append<false, 512, 2>(P, grid, smem, st);
    else e = bf ? launch_append<true, 512, 4>(P, grid, smem, st) : launch_append<false, 512, 4>(P, grid, smem, st);
  }
  return e == cudaSuccess ? LANTERN_OK : LANTERN_E_CUDA;
}

extern "C" lantern_status lantern_cache_keep(const lantern_cache* cache, const int32_t* table, int table_width, const int32_t* lengths,
                                             const int32_t* accept_len, const int32_t* accept_path, int B, int N, int32_t* out_lengths,
                                             int32_t* status, void* cuda_stream) {
  const lantern_status bad = check_cache(cache, table, table_width, B);
  if (bad != LANTERN_OK) return bad;
  if (B < 0 || B > 65535 || N < 0 || N > 1024) return LANTERN_E_SHAPE;
  if (B == 0) return LANTERN_OK;
  if (!lengths || !accept_len || !out_lengths || (N > 0 && !accept_path)) return LANTERN_E_NULL;
  // (every warp of a sequence reads these, and one of them writes the new length)
  const auto overlaps = [&](const int32_t* p, int64_t n) { return p && out_lengths < p + n && p < out_lengths + B; };
  if (overlaps(lengths, B) || overlaps(accept_len, B) || overlaps(accept_path, static_cast<int64_t>(B) * N)) return LANTERN_E_PARAM;
  KeepParams P{view_of(cache, table, table_width), lengths, accept_len, accept_path, out_lengths, status, N};
  const dim3 grid((2 * cache->heads + KT / 32 - 1) / (KT / 32), B);
  lantern_keep_kernel<<<grid, KT, 0, static_cast<cudaStream_t>(cuda_stream)>>>(P);
  return cudaGetLastError() == cudaSuccess ? LANTERN_OK : LANTERN_E_CUDA;
}

extern "C" lantern_status lantern_cache_read(const lantern_cache* cache, const int32_t* table, int table_width, const int32_t* first,
                                             const int32_t* counts, int B, int R, int dtype, void* out_k, void* out_v, int32_t* status,
                                             void* cuda_stream) {
  if (dtype != LANTERN_F32 && dtype != LANTERN_BF16) return LANTERN_E_PARAM;
  const lantern_status bad = check_cache(cache, table, table_width, B);
  if (bad != LANTERN_OK) return bad;
  if (B < 0 || R < 0 || static_cast<int64_t>(B) * R > INT32_MAX) return LANTERN_E_SHAPE;
  if (B == 0 || R == 0) return LANTERN_OK;
  if (!first || !out_k || !out_v) return LANTERN_E_NULL;
  if ((reinterpret_cast<uintptr_t>(out_k) & 15) || (reinterpret_cast<uintptr_t>(out_v) & 15)) return LANTERN_E_ALIGN;
  const int64_t units = static_cast<int64_t>(R) * cache->heads * (cache->head_dim / 16);
  if (units > INT32_MAX - DT) return LANTERN_E_SHAPE;
  ReadParams P{view_of(cache, table, table_width), first, counts, status, {out_k, out_v}, B, R, static_cast<int>(units)};
  const dim3 grid(static_cast<unsigned>((units + DT - 1) / DT), B < 65535 ? B : 65535);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (dtype == LANTERN_BF16) lantern_read_kernel<true><<<grid, DT, 0, st>>>(P);
  else lantern_read_kernel<false><<<grid, DT, 0, st>>>(P);
  return cudaGetLastError() == cudaSuccess ? LANTERN_OK : LANTERN_E_CUDA;
}
