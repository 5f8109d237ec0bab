// Attention of a step's rows to the paged 8-bit cache: the call.  The kernels are in cache_attention_few.cu, _mid.cu and _wide.cu, by the number of
// rows of a sequence and cache head.
#include "cache_attention.cuh"

namespace lantern {

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

// Which kernel takes a call, and how its rows and tokens are divided.
//   Up to 16 rows: `few` (128 single tokens of 4 heads a group over 2300 tokens: 116 us; as 64 rows mostly empty, 193).
//   Up to 64 bf16 rows: `mid` where contexts are short, `wide` where they can be long enough for its units' longer start and end (trees of 61 rows, 20
//   heads.  64 components: 64 trees over 140 tokens mid 49 us, wide 57; 256 over 640 363 and 363; 64 over 1120 155 and 143, over 2250 292 and 228.  128
//   components: 64 over 140 89 and 107, over 340 133 and 129, over 640 196 and 169.  Where units are few `wide` is ahead on short contexts too: 2 trees
//   over 140 tokens 15 and 13.5, 16 over 640 57 and 42).  A call knows no lengths: `room` is what the table can hold, about twice these averages where
//   tables are cut to the contexts.  A wider table is taken for longer contexts: nothing for 256 trees over 640 tokens, and 9 to 11 us for one token, whose
//   call then has a join that finds one part.
//   More rows, and fp32 ones from 17 on: `wide` (16 trees of 61 rows, 8 heads a group, 1200 tokens: 73 us, in 64 rows at a time as mid takes them 135).
static Division divide(int dtype, int B, int R, int q_heads, const lantern_cache* c, int width) {
  Division d;
  const int64_t G = q_heads / c->heads, M = G * R, room = static_cast<int64_t>(width) * c->page_tokens;
  d.DP = c->head_dim <= 64 ? 64 : 128;
  d.rows = M <= 16 ? 16 : M <= 64 ? 64 : 128;
  d.kernel = d.rows == 16 ? Division::kFew : d.rows == 64 && dtype == LANTERN_BF16 && room < (d.DP == 64 ? 2048 : 1024) ? Division::kMid : Division::kWide;
  d.tile = d.kernel == Division::kFew ? 32 : d.DP == 64 ? 64 : d.kernel == Division::kMid ? 32 : 128;   // (as the kernels have it)
  d.row_tiles = static_cast<int>((M + d.rows - 1) / d.rows);
  d.units = static_cast<int64_t>(B) * c->heads * d.row_tiles;
  // A unit is divided where there are fewer units than places for CTAs on the GPU: into as many parts as fill the places once where CTAs are
  // persistent (`wide`: a part's start and end cost as much as several tiles), else twice; a part has 512 tokens at least, so that a short
  // context is one launch.
  const int64_t tiles = (room + d.tile - 1) / d.tile, units = d.units > 0 ? d.units : 1;
  const int64_t places = kSms * (d.kernel == Division::kWide ? (d.DP == 64 ? 2 : 1) : d.kernel == Division::kFew || d.DP == 64 ? 3 : 2);
  d.least = 512 / d.tile;
  int64_t splits = units >= places ? 1 : d.kernel == Division::kWide ? places / units : (2 * places + units - 1) / units;
  const int64_t most = (tiles + d.least - 1) / d.least;
  if (splits > most) splits = most;
  d.splits = static_cast<int>(splits < 1 ? 1 : splits > 512 ? 512 : splits);
  return d;
}
static size_t parts_bytes(const Division& d) {
  return d.splits == 1 ? 0 : static_cast<size_t>(d.units) * d.splits * d.rows * (d.DP * sizeof(float) + sizeof(float2));
}
static lantern_status check_attention(int dtype, int B, int R, int q_heads, const lantern_cache* c, int width, bool tree) {
  if (dtype != LANTERN_F32 && dtype != LANTERN_BF16) return LANTERN_E_PARAM;
  if (B < 0 || R < 0 || q_heads < 1 || q_heads % c->heads != 0 || (tree && R > kMaxTreeRows)) return LANTERN_E_SHAPE;
  if (static_cast<int64_t>(R) * (q_heads / c->heads) > INT32_MAX / 2 || static_cast<int64_t>(B) * R > INT32_MAX) return LANTERN_E_SHAPE;
  const Division d = divide(dtype, B, R, q_heads, c, width);
  if (d.units * (d.splits > 16 ? d.splits : 16) > INT32_MAX) return LANTERN_E_SHAPE;
  return LANTERN_OK;
}

}  // namespace lantern

using namespace lantern;

extern "C" size_t lantern_cache_attention_workspace_bytes(int dtype, int B, int R, int q_heads, const lantern_cache* cache, int table_width) {
  if (!cache || check_cache(cache, nullptr, table_width, 0) != LANTERN_OK) return 0;
  if (check_attention(dtype, B, R, q_heads, cache, table_width, false) != LANTERN_OK || B == 0 || R == 0) return 0;
  return parts_bytes(divide(dtype, B, R, q_heads, cache, table_width));
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
  if (q == out) return LANTERN_E_PARAM;
  const bool bf = dtype == LANTERN_BF16;
  const int size = bf ? 2 : 4;
  if (reinterpret_cast<uintptr_t>(q) % size || (reinterpret_cast<uintptr_t>(out) & 15)) return LANTERN_E_ALIGN;
  const Division d = divide(dtype, B, R, q_heads, cache, table_width);
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
  P.items = static_cast<uint32_t>(d.units * d.splits);
  P.splits = d.splits;
  P.least = d.least;
  const int64_t qs[3] = {q_stride[0], q_stride[1], q_stride[2]};
  P.vec = aligned16(q, qs, size);
  P.scale_log2 = scale * 1.44269504088896340736f;
  P.tries = kTries;
  wait_test(&P.tries, &P.withhold);
  CUtensorMap km, vm;
  const int tokens = P.S < d.tile ? P.S : d.tile;
  if ((bad = code_map(&km, cache->k_code, cache, d.DP, tokens)) != LANTERN_OK || (bad = code_map(&vm, cache->v_code, cache, d.DP, tokens)) != LANTERN_OK) return bad;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e;
  if (d.kernel == Division::kFew) e = launch_attention_few(P, km, vm, d, bf, st);
  else if (d.kernel == Division::kMid) e = launch_attention_mid(P, km, vm, d, st);
  else e = launch_attention_wide(P, km, vm, d, bf, st);
  return e == cudaSuccess ? LANTERN_OK : LANTERN_E_CUDA;
}
