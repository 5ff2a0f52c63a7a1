// Token embedding: the lookup with scaling, and its gradient by sorted tokens.
//
//   k_lookup       out[t] = s table[id_t]
//   k_rank         stable order of the tokens by id, and what the gradient's output holds where no token is (zeros, or "no row")
//   k_tile_sum     sums over runs of equal ids inside tiles of the sorted order
//   k_join_tiles   runs that cross tiles
//
// Sums run over the tokens of an id in their order in the batch, with borders that the sorted order alone fixes: no atomics, the same bits
// every time.
#include "fullrank.h"

#include <algorithm>
#include <cmath>

namespace lordo {

constexpr int TILE = 32;              // sorted tokens of a workgroup of k_tile_sum

struct Ids {
  const void* p;
  int32_t wide;                       // int64, else int32
  int32_t vocab;
  int64_t pad_id;
};
// What a token is sorted by: its id, or `vocab` (behind all others) where it takes no part.
__device__ __forceinline__ int32_t token_key(const Ids& ids, int64_t t) {
  const int64_t id = ids.wide ? reinterpret_cast<const int64_t*>(ids.p)[t] : (int64_t)reinterpret_cast<const int32_t*>(ids.p)[t];
  return id < 0 || id >= ids.vocab || id == ids.pad_id ? ids.vocab : (int32_t)id;
}

template <bool IN_BF, bool OUT_BF>
__global__ __launch_bounds__(256) void k_lookup(const void* table, Ids ids, int64_t tokens, int64_t cols, int lanes_log2, float scale, void* out) {
  const int lanes = 1 << lanes_log2;                                   // threads of a row
  const int64_t t = (int64_t)blockIdx.x * (256 >> lanes_log2) + (threadIdx.x >> lanes_log2);
  if (t >= tokens) return;
  const int32_t id = token_key(ids, t);
  const int64_t from = (int64_t)id * cols, to = t * cols;
  for (int64_t c = (int64_t)(threadIdx.x & (lanes - 1)) * 4; c < cols; c += (int64_t)lanes * 4) {
    const int cnt = cols - c >= 4 ? 4 : (int)(cols - c);
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    if (cnt == 4) {
      if (id < ids.vocab) load_quad<IN_BF, false>(table, from + c, x);
      for (int e = 0; e < 4; ++e) x[e] *= scale;
      store_quad<OUT_BF, false>(out, to + c, x);
    } else {
      for (int e = 0; e < cnt; ++e) store_element<OUT_BF>(out, to + c + e, id < ids.vocab ? load_element<IN_BF>(table, from + c + e) * scale : 0.f);
    }
  }
}

// rank of token i = tokens with a smaller key + tokens before it with the same key.  A workgroup ranks 64 tokens, its sixteen waves a sixteenth
// of the batch each.  The workgroups behind them fill `fill` (bytes) with `value`.
struct Sorted { int32_t *key, *pos; };
__global__ __launch_bounds__(1024) void k_rank(Ids ids, int32_t tokens, Sorted out, int rank_blocks, void* fill, int64_t fill_bytes, uint32_t value) {
  if ((int)blockIdx.x >= rank_blocks) {
    char* p = reinterpret_cast<char*>(fill);
    const int64_t lead = std::min<int64_t>(fill_bytes, (int64_t)(-(intptr_t)p & 15)), whole = (fill_bytes - lead) / 16, tail = fill_bytes - lead - whole * 16;
    const int64_t first = (int64_t)((int)blockIdx.x - rank_blocks) * 1024 + threadIdx.x, stride = (int64_t)((int)gridDim.x - rank_blocks) * 1024;
    const u32x4a x = {value, value, value, value};
    for (int64_t i = first; i < whole; i += stride) __builtin_nontemporal_store(x, reinterpret_cast<u32x4a*>(p + lead) + i);
    if (first < lead / 2) reinterpret_cast<uint16_t*>(p)[first] = (uint16_t)value;             // (both halves of `value` are alike)
    if (first < tail / 2) reinterpret_cast<uint16_t*>(p + lead + whole * 16)[first] = (uint16_t)value;
    return;
  }
  __shared__ int32_t part[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int32_t i = (int32_t)blockIdx.x * 64 + lane, mine = i < tokens ? token_key(ids, i) : 0;
  const int32_t tiles = (tokens + 63) / 64, each = (tiles + 15) / 16, last = std::min(tiles, (wave + 1) * each);
  int32_t rank = 0;
  for (int32_t b = wave * each; b < last; ++b) {
    const int32_t j = b * 64 + lane;
    const int32_t key = j < tokens ? token_key(ids, j) : INT32_MAX;
    const int32_t limit = b < (int32_t)blockIdx.x ? mine + 1 : mine;      // equal keys count if they come before
#pragma unroll 16
    for (int l = 0; l < 64; ++l) rank += __builtin_amdgcn_readlane(key, l) < limit;
    if (b == (int32_t)blockIdx.x)
      for (int l = 0; l < 64; ++l) rank += __builtin_amdgcn_readlane(key, l) == mine && l < lane;
  }
  part[wave][lane] = rank;
  __syncthreads();
  if (wave == 0 && i < tokens) {
    rank = 0;
    for (int k = 0; k < 16; ++k) rank += part[k][lane];
    out.key[rank] = mine;
    out.pos[rank] = i;
  }
}

struct GradOut {
  void* dst;                          // vocab x cols, or rows in the order of the first of their tokens
  int32_t* index;                     // rows: row of dst of an id, behind it the id of a row of dst (null: dense)
  float* part;                        // two partial rows a tile: of the run it goes on with, and of the one that goes on behind it
  float scale;
  int32_t add;
};

// ADD and the type of the output are uniform: a branch a row is nothing beside its loads.
template <bool OUT_BF>
__device__ __forceinline__ void put_row(const GradOut& o, int64_t row, int64_t cols, int64_t c, int cnt, float (&x)[4]) {
  for (int e = 0; e < 4; ++e) x[e] *= o.scale;
  const int64_t at = row * cols + c;
  if (cnt == 4) {
    if (o.add) {
      float old[4];
      load_quad<OUT_BF, false>(o.dst, at, old);
      for (int e = 0; e < 4; ++e) x[e] += old[e];
    }
    store_quad<OUT_BF, false>(o.dst, at, x);
  } else {
    for (int e = 0; e < cnt; ++e) store_element<OUT_BF>(o.dst, at + e, o.add ? x[e] + load_element<OUT_BF>(o.dst, at + e) : x[e]);
  }
}

// A workgroup sums TILE sorted tokens over 1024 columns, a thread four of them.  A run of one id that lies inside the tile goes to the output; one that
// came in or goes on leaves a partial row.
template <bool IN_BF, bool OUT_BF>
__global__ __launch_bounds__(256) void k_tile_sum(const void* dy, Sorted in, int32_t tokens, int32_t vocab, int64_t cols, GradOut o) {
  const int32_t tile = (int32_t)blockIdx.x, first = tile * TILE, end = std::min(first + TILE, tokens);
  const int64_t c = (int64_t)blockIdx.y * 1024 + threadIdx.x * 4;
  const int cnt = cols - c >= 4 ? 4 : cols > c ? (int)(cols - c) : 0;
  const bool from_before = first > 0 && in.key[first - 1] == in.key[first];
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  int32_t start = first;
  for (int32_t s = first; s < end; ++s) {
    const int32_t key = in.key[s];
    if (key == vocab) break;                          // the rest takes no part
    const int64_t from = (int64_t)in.pos[s] * cols + c;
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    if (cnt == 4) load_quad<IN_BF, false>(dy, from, x);
    else
      for (int e = 0; e < cnt; ++e) x[e] = load_element<IN_BF>(dy, from + e);
    for (int e = 0; e < 4; ++e) sum[e] += x[e];
    const bool more = s + 1 < tokens && in.key[s + 1] == key;
    if (more && s + 1 < end) continue;
    const bool came = start == first && from_before;
    if (!came && o.index && blockIdx.y == 0 && threadIdx.x == 0) {
      o.index[key] = start;
      o.index[vocab + start] = key;
    }
    if (!came && !more) {
      put_row<OUT_BF>(o, o.index ? start : key, cols, c, cnt, sum);
    } else {
      float* p = o.part + ((int64_t)tile * 2 + (came ? 0 : 1)) * cols + c;
      for (int e = 0; e < cnt; ++e) p[e] = sum[e];
    }
    for (int e = 0; e < 4; ++e) sum[e] = 0.f;
    start = s + 1;
  }
}

// The run that begins in tile k and goes on: its partial rows in order.
template <bool OUT_BF>
__global__ __launch_bounds__(256) void k_join_tiles(Sorted in, int32_t tokens, int32_t vocab, int64_t cols, GradOut o) {
  const int32_t tile = (int32_t)blockIdx.x, first = tile * TILE, next = first + TILE;
  if (next >= tokens) return;
  const int32_t key = in.key[next];
  if (key == vocab || in.key[next - 1] != key) return;
  if (in.key[first] == key && first > 0 && in.key[first - 1] == key) return;      // it began before
  const int64_t c = (int64_t)blockIdx.y * 1024 + threadIdx.x * 4;
  const int cnt = cols - c >= 4 ? 4 : cols > c ? (int)(cols - c) : 0;
  int32_t start = next - 1;
  while (start > first && in.key[start - 1] == key) --start;
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  const float* p = o.part + ((int64_t)tile * 2 + 1) * cols + c;
  for (int e = 0; e < cnt; ++e) sum[e] = p[e];
  for (int32_t k = tile + 1; k * TILE < tokens && in.key[k * TILE] == key; ++k) {
    p = o.part + (int64_t)k * 2 * cols + c;
    for (int e = 0; e < cnt; ++e) sum[e] += p[e];
  }
  put_row<OUT_BF>(o, o.index ? start : key, cols, c, cnt, sum);
}

}  // namespace lordo

using namespace lordo;

namespace {

bool float_type(int32_t t) { return t == LORDO_F32 || t == LORDO_BF16; }
bool float_aligned(const void* p, int32_t t) { return (reinterpret_cast<uintptr_t>(p) & (t == LORDO_F32 ? 3 : 1)) == 0; }
bool good_ids(const void* ids, int32_t dtype, int64_t tokens) {
  if ((dtype != LORDO_I32 && dtype != LORDO_I64) || tokens < 0 || tokens > LORDO_MAX_TOKENS) return false;
  return tokens == 0 || (ids && (reinterpret_cast<uintptr_t>(ids) & (dtype == LORDO_I64 ? 7 : 3)) == 0);
}
bool good_table(int64_t vocab, int64_t cols) { return vocab > 0 && vocab <= LORDO_MAX_VOCAB && cols > 0 && cols <= LORDO_MAX_EMBED_COLS; }
int64_t up256(int64_t x) { return (x + 255) & ~int64_t(255); }

struct GradPlan { int64_t key, pos, part, bytes; };
GradPlan plan_gradient(int64_t tokens, int64_t cols) {
  GradPlan p;
  p.key = 0;
  p.pos = up256(4 * tokens);
  p.part = p.pos + up256(4 * tokens);
  p.bytes = p.part + up256((tokens + TILE - 1) / TILE * 2 * cols * 4);
  return p;
}

int embed_gradient(Ids ids, int64_t tokens, const void* dy, int32_t dy_dtype, int64_t cols, float scale, void* dst, int32_t dst_dtype, int32_t* index, bool add,
                   char* ws, hipStream_t s) {
  const GradPlan p = plan_gradient(tokens, cols);
  const Sorted sorted{reinterpret_cast<int32_t*>(ws + p.key), reinterpret_cast<int32_t*>(ws + p.pos)};
  const GradOut o{dst, index, reinterpret_cast<float*>(ws + p.part), scale, add ? 1 : 0};
  // where no token is: zeros in a dense gradient that is overwritten, no row for an id and no id for a row
  void* fill = index ? index : add ? nullptr : dst;
  const int64_t fill_bytes = index ? 4 * (ids.vocab + tokens) : add ? 0 : (int64_t)ids.vocab * cols * (dst_dtype == LORDO_F32 ? 4 : 2);
  const int rank_blocks = (int)((tokens + 63) / 64), fill_blocks = (int)std::min<int64_t>((fill_bytes + 65535) / 65536, 2048);
  if (rank_blocks + fill_blocks == 0) return LORDO_OK;
  hipLaunchKernelGGL(k_rank, dim3((unsigned)(rank_blocks + fill_blocks)), dim3(1024), 0, s, ids, (int32_t)tokens, sorted, rank_blocks, fill, fill_bytes,
                     index ? 0xffffffffu : 0u);
  int rc = launched("k_rank");
  if (rc != LORDO_OK || tokens == 0) return rc;
  const dim3 grid((unsigned)((tokens + TILE - 1) / TILE), (unsigned)((cols + 1023) / 1024)), block(256);
  const bool in_bf = dy_dtype == LORDO_BF16, out_bf = dst_dtype == LORDO_BF16;
  const int32_t n = (int32_t)tokens, vocab = ids.vocab;
  if (in_bf && out_bf) hipLaunchKernelGGL((k_tile_sum<true, true>), grid, block, 0, s, dy, sorted, n, vocab, cols, o);
  else if (in_bf) hipLaunchKernelGGL((k_tile_sum<true, false>), grid, block, 0, s, dy, sorted, n, vocab, cols, o);
  else if (out_bf) hipLaunchKernelGGL((k_tile_sum<false, true>), grid, block, 0, s, dy, sorted, n, vocab, cols, o);
  else hipLaunchKernelGGL((k_tile_sum<false, false>), grid, block, 0, s, dy, sorted, n, vocab, cols, o);
  rc = launched("k_tile_sum");
  if (rc != LORDO_OK) return rc;
  if (out_bf) hipLaunchKernelGGL((k_join_tiles<true>), grid, block, 0, s, sorted, n, vocab, cols, o);
  else hipLaunchKernelGGL((k_join_tiles<false>), grid, block, 0, s, sorted, n, vocab, cols, o);
  return launched("k_join_tiles");
}

}  // namespace

extern "C" {

int lordo_embed_lookup(const void* table, int32_t table_dtype, int64_t vocab, int64_t cols, const void* ids, int32_t ids_dtype, int64_t tokens,
                       double scale, void* out, int32_t out_dtype, void* stream) {
  if (!good_table(vocab, cols) || !good_ids(ids, ids_dtype, tokens) || !float_type(table_dtype) || !float_type(out_dtype) || !std::isfinite(scale))
    return LORDO_EINVAL;
  if (tokens == 0) return LORDO_OK;
  if (!table || !out || !float_aligned(table, table_dtype) || !float_aligned(out, out_dtype)) return LORDO_EINVAL;
  const Ids id{ids, ids_dtype == LORDO_I64, (int32_t)vocab, -1};
  int lanes_log2 = 0;
  while (lanes_log2 < 8 && (int64_t(4) << lanes_log2) < cols) ++lanes_log2;
  const int64_t per_block = 256 >> lanes_log2;
  const dim3 grid((unsigned)((tokens + per_block - 1) / per_block)), block(256);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const float f = (float)scale;
  const bool in_bf = table_dtype == LORDO_BF16, out_bf = out_dtype == LORDO_BF16;
  if (in_bf && out_bf) hipLaunchKernelGGL((k_lookup<true, true>), grid, block, 0, s, table, id, tokens, cols, lanes_log2, f, out);
  else if (in_bf) hipLaunchKernelGGL((k_lookup<true, false>), grid, block, 0, s, table, id, tokens, cols, lanes_log2, f, out);
  else if (out_bf) hipLaunchKernelGGL((k_lookup<false, true>), grid, block, 0, s, table, id, tokens, cols, lanes_log2, f, out);
  else hipLaunchKernelGGL((k_lookup<false, false>), grid, block, 0, s, table, id, tokens, cols, lanes_log2, f, out);
  return launched("k_lookup");
}

int lordo_embed_workspace_bytes(int64_t tokens, int64_t vocab, int64_t cols, size_t* out_bytes) {
  if (!out_bytes || !good_table(vocab, cols) || tokens < 0 || tokens > LORDO_MAX_TOKENS) return LORDO_EINVAL;
  *out_bytes = (size_t)plan_gradient(tokens, cols).bytes;
  return LORDO_OK;
}

int lordo_embed_gradient(const void* ids, int32_t ids_dtype, int64_t tokens, const void* dy, int32_t dy_dtype, int64_t vocab, int64_t cols, double scale,
                         int64_t pad_id, int32_t accumulate, void* dw, int32_t dw_dtype, void* workspace, size_t workspace_bytes, void* stream) {
  if (!good_table(vocab, cols) || !good_ids(ids, ids_dtype, tokens) || !float_type(dy_dtype) || !float_type(dw_dtype) || !std::isfinite(scale))
    return LORDO_EINVAL;
  if ((accumulate != 0 && accumulate != 1) || !dw || !float_aligned(dw, dw_dtype)) return LORDO_EINVAL;
  if (tokens > 0 && (!dy || !float_aligned(dy, dy_dtype) || !workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0)) return LORDO_EINVAL;
  if (workspace_bytes < (size_t)plan_gradient(tokens, cols).bytes) return LORDO_ENOMEM;
  return embed_gradient(Ids{ids, ids_dtype == LORDO_I64, (int32_t)vocab, pad_id}, tokens, dy, dy_dtype, cols, (float)scale, dw, dw_dtype, nullptr,
                        accumulate != 0, reinterpret_cast<char*>(workspace), reinterpret_cast<hipStream_t>(stream));
}

int lordo_embed_gradient_rows(const void* ids, int32_t ids_dtype, int64_t tokens, const void* dy, int32_t dy_dtype, int64_t vocab, int64_t cols, double scale,
                              int64_t pad_id, void* rows, int32_t rows_dtype, int32_t* index, void* workspace, size_t workspace_bytes, void* stream) {
  if (!good_table(vocab, cols) || !good_ids(ids, ids_dtype, tokens) || !float_type(dy_dtype) || !float_type(rows_dtype) || !std::isfinite(scale))
    return LORDO_EINVAL;
  if (!index || (reinterpret_cast<uintptr_t>(index) & 3) != 0) return LORDO_EINVAL;
  if (tokens > 0 && (!rows || !float_aligned(rows, rows_dtype) || !dy || !float_aligned(dy, dy_dtype) || !workspace ||
                     (reinterpret_cast<uintptr_t>(workspace) & 255) != 0))
    return LORDO_EINVAL;
  if (workspace_bytes < (size_t)plan_gradient(tokens, cols).bytes) return LORDO_ENOMEM;
  return embed_gradient(Ids{ids, ids_dtype == LORDO_I64, (int32_t)vocab, pad_id}, tokens, dy, dy_dtype, cols, (float)scale, rows, rows_dtype, index, false,
                        reinterpret_cast<char*>(workspace), reinterpret_cast<hipStream_t>(stream));
}

}  // extern "C"
