// Token embedding: the lookup with scaling, and its gradient by sorted tokens.
//
//   k_lookup              out[t] = s table[id_t]
//   k_rank                stable order of up to 8192 tokens by id, one launch; or
//   k_count, k_place      the digits of the id from the lowest on, two launches a digit
//   k_tile_sum            sums over runs of equal ids, tile by tile of the sorted order
//   k_join_tiles          runs longer than two tiles
//
// The first launch also writes what the output holds where no token is.  Sums run over the tokens of an id in their order in the batch, with borders
// that the sorted order alone fixes: no atomics on values, the same bits every time.
#include "fullrank.h"

#include <algorithm>
#include <cmath>

namespace lordo {

constexpr int MOST_TILE = 32;         // most sorted tokens of a workgroup of k_tile_sum: a wave holds two tiles of them, one a lane
constexpr int RANK_TOKENS = 8192;     // most tokens of k_rank
constexpr int RANK_ROW = 32;          // tokens that a workgroup of it ranks
constexpr int PLACE_CHUNK = 2048;     // tokens that a workgroup of k_place has in registers
constexpr int PLACE_BLOCKS = 256;     // most workgroups of a digit
constexpr int MAX_BINS = 512;
constexpr int64_t LOOKUP_TOKENS = 1 << 23;   // most tokens of a launch of k_lookup: a launch has less than 2^32 threads, and long rows are a workgroup each

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

// A thread copies eight columns of a row.  NARROW: rows shorter than that, a thread an element.
// Memory: 32768 tokens, an eighth of them padding, of a 32000 x 2048 fp32 table to bf16 48 us: 134 MB written and 235 read, two thirds of that from the caches.
// Four columns a thread took 58.  Four rows a thread, all requested before the first is written, took 49, and were 0 to 25 % slower from 512 to 32768
// workgroups of one row, tables of both types, 64 to 4096 columns: so many workgroups keep enough in flight.
template <bool IN_BF, bool OUT_BF, bool NARROW>
__global__ __launch_bounds__(256) void k_lookup(const void* table, Ids ids, int64_t tokens, int64_t cols, int lanes_log2, float scale, void* out) {
  constexpr int VEC = NARROW ? 1 : 8;
  const int lanes = 1 << lanes_log2, per = 256 >> lanes_log2;          // threads of a row, rows of a workgroup
  const int64_t c0 = ((int64_t)blockIdx.y * lanes + (threadIdx.x & (lanes - 1))) * VEC;
  const int64_t row = (int64_t)blockIdx.x * per + (threadIdx.x >> lanes_log2);
  if (c0 >= cols || row >= tokens) return;
  const int64_t c = std::min(c0, cols - VEC);                          // the last piece of a row ends where the row does
  const int32_t id = token_key(ids, row);
  Piece<IN_BF, VEC> x;
  x.clear();
  if (id < ids.vocab) x.load(table, (int64_t)id * cols + c);
  float y[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) y[e] = x.value(e) * scale;
  put_piece<OUT_BF, VEC>(out, row * cols + c, y, (int)(c0 - c));
}

struct Sorted { int32_t *key, *pos; };

// What an output holds before any token is added: `bytes` of it, halves of `value` (both alike), by the workgroups that a launch has to spare.
struct Fill {
  void* p;
  int64_t bytes;
  uint32_t value;
};
__device__ __forceinline__ void fill_share(const Fill& f, int64_t first, int64_t stride) {
  char* p = reinterpret_cast<char*>(f.p);
  const int64_t lead = std::min<int64_t>(f.bytes, (int64_t)(-(intptr_t)p & 15)), whole = (f.bytes - lead) / 16, tail = f.bytes - lead - whole * 16;
  const u32x4a x = {f.value, f.value, f.value, f.value};
  for (int64_t i = first; i < whole; i += stride) __builtin_nontemporal_store(x, reinterpret_cast<u32x4a*>(p + lead) + i);
  if (first < lead / 2) reinterpret_cast<uint16_t*>(p)[first] = (uint16_t)f.value;
  if (first < tail / 2) reinterpret_cast<uint16_t*>(p + lead + whole * 16)[first] = (uint16_t)f.value;
}

// Order of up to 8192 tokens in one launch.  Key and position in one 32-bit number are all different, so the place of a token is how many numbers are
// smaller: all pairs are compared, two instructions a pair, with the other side read from LDS, four numbers a (broadcast) read.  A workgroup places 32 tokens: the two
// halves of a wave compare them with different numbers, its sixteen waves with a 32nd of the batch each half.  8192 tokens are 256 workgroups, one a compute unit.
// 4095 tokens 5.7 us, 8192 9.8, of which 3 are comparisons; the two digits that 64k tokens need take 27 without what they fill, so comparing ends at 8192.
__global__ __launch_bounds__(1024) void k_rank(Ids ids, int32_t tokens, int pos_bits, Sorted out, int rank_blocks, Fill fill) {
  if ((int)blockIdx.x >= rank_blocks) {
    fill_share(fill, (int64_t)((int)blockIdx.x - rank_blocks) * 1024 + threadIdx.x, (int64_t)((int)gridDim.x - rank_blocks) * 1024);
    return;
  }
  __shared__ uint32_t number[RANK_TOKENS];
  __shared__ int32_t part[32][RANK_ROW];
  const int half = threadIdx.x >> 5, lane = threadIdx.x & 31;           // 32 halves of waves
  const int32_t each = (tokens + 127) / 128 * 4;                        // numbers of a half, whole quads
  for (int32_t j = threadIdx.x; j < each * 32; j += 1024)
    number[j] = j < tokens ? (uint32_t)token_key(ids, j) << pos_bits | (uint32_t)j : 0xffffffffu;
  __syncthreads();
  const int32_t i = (int32_t)blockIdx.x * RANK_ROW + lane;
  const uint32_t mine = i < tokens ? number[i] : 0;
  int32_t rank = 0;
  const uint4* q = reinterpret_cast<const uint4*>(number + half * each);
#pragma unroll 4
  for (int32_t k = 0; k < each / 4; ++k) {
    const uint4 x = q[k];
    rank += x.x < mine;
    rank += x.y < mine;
    rank += x.z < mine;
    rank += x.w < mine;
  }
  part[half][lane] = rank;
  __syncthreads();
  if (half == 0 && i < tokens) {
    rank = 0;
    for (int k = 0; k < 32; ++k) rank += part[k][lane];
    out.key[rank] = (int32_t)(mine >> pos_bits);
    out.pos[rank] = i;
  }
}

// More tokens: by the digits of the key, the lowest first, stable.  A workgroup has `block` consecutive tokens; k_count leaves how many of each digit it
// holds, k_place adds up what is before it (smaller digits anywhere, its own in earlier workgroups) and moves its tokens there.
// Latency: 65536 tokens with ids of 15 bits 5 + 8 us a digit (comparing all pairs: 639 us), or 13 to 15 a launch with a quarter of 262 MB of zeros each, which hide
// it (all zeros in the first launch: 52 + 12 + 5 + 11).
struct Digit { int32_t tokens, block, blocks, shift, bits; };

template <bool FIRST>
__global__ __launch_bounds__(256) void k_count(Ids ids, Sorted in, Digit d, int32_t* count, Fill fill) {
  if ((int)blockIdx.x >= d.blocks) {
    fill_share(fill, (int64_t)((int)blockIdx.x - d.blocks) * 256 + threadIdx.x, (int64_t)((int)gridDim.x - d.blocks) * 256);
    return;
  }
  __shared__ int32_t bins[MAX_BINS];
  for (int k = threadIdx.x; k < MAX_BINS; k += 256) bins[k] = 0;
  __syncthreads();
  const int32_t first = (int32_t)blockIdx.x * d.block, end = std::min(first + d.block, d.tokens), mask = (1 << d.bits) - 1;
  for (int32_t j = first + (int32_t)threadIdx.x; j < end; j += 256) {
    const int32_t key = FIRST ? token_key(ids, j) : in.key[j];
    atomicAdd(&bins[(key >> d.shift) & mask], 1);
  }
  __syncthreads();
  for (int k = threadIdx.x; k < (1 << d.bits); k += 256) count[(int64_t)blockIdx.x << d.bits | k] = bins[k];
}

template <bool FIRST>
__global__ __launch_bounds__(1024) void k_place(Ids ids, Sorted in, Sorted out, Digit d, const int32_t* count, Fill fill) {
  if ((int)blockIdx.x >= d.blocks) {
    fill_share(fill, (int64_t)((int)blockIdx.x - d.blocks) * 1024 + threadIdx.x, (int64_t)((int)gridDim.x - d.blocks) * 1024);
    return;
  }
  constexpr int ROUNDS = PLACE_CHUNK / 1024;
  __shared__ int32_t base[MAX_BINS], bins[16][MAX_BINS], sums[8];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, digits = 1 << d.bits, mask = digits - 1;
  const int32_t first = (int32_t)blockIdx.x * d.block, end = std::min(first + d.block, d.tokens);
  // A share of the workgroups' counts for every thread: of digit k of a group of MAX_BINS threads, every second workgroup.  bins[0 ... 3] hold the sums.
  {
    const int k = threadIdx.x & (MAX_BINS - 1), group = threadIdx.x / MAX_BINS;
    int32_t total = 0, before = 0;
    if (k < digits) {
#pragma unroll 16
      for (int b = group; b < d.blocks; b += 1024 / MAX_BINS) {
        const int32_t c = count[(int64_t)b << d.bits | k];
        total += c;
        before += b < (int)blockIdx.x ? c : 0;
      }
    }
    bins[group][k] = total;
    bins[2 + group][k] = before;
  }
  __syncthreads();
  {
    const int k = threadIdx.x;
    int32_t total = 0, before = 0, run = 0;
    if (k < MAX_BINS) {
      total = bins[0][k] + bins[1][k];
      before = bins[2][k] + bins[3][k];
      run = total;
      for (int m = 1; m < 64; m <<= 1) {
        const int32_t o = __shfl_up(run, m);
        if (lane >= m) run += o;
      }
      if (lane == 63) sums[wave] = run;
    }
    __syncthreads();
    if (k < MAX_BINS) {
      run -= total;
      for (int w = 0; w < wave; ++w) run += sums[w];
      base[k] = run + before;
    }
  }
  for (int32_t at = first; at < end; at += PLACE_CHUNK) {
    int32_t key[ROUNDS], pos[ROUNDS], rank[ROUNDS];
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      const int32_t j = at + (wave * ROUNDS + r) * 64 + lane;
      key[r] = j < end ? (FIRST ? token_key(ids, j) : in.key[j]) : -1;
      pos[r] = FIRST || j >= end ? j : in.pos[j];
    }
    __syncthreads();
    for (int k = threadIdx.x; k < 16 * MAX_BINS; k += 1024) (&bins[0][0])[k] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      const int digit = (key[r] >> d.shift) & mask;
      uint64_t same = __ballot(key[r] >= 0);
      for (int b = 0; b < d.bits; ++b) {
        const uint64_t set = __ballot((digit >> b) & 1);
        same &= (digit >> b) & 1 ? set : ~set;
      }
      const int lead = same ? __ffsll((unsigned long long)same) - 1 : lane;
      int32_t old = 0;
      if (lane == lead && key[r] >= 0) old = atomicAdd(&bins[wave][digit], (int32_t)__popcll(same));
      rank[r] = __shfl(old, lead) + __popcll(same & ((1ull << lane) - 1));
    }
    __syncthreads();
    if ((int)threadIdx.x < digits) {                  // counts of the waves -> where each wave's tokens of the digit begin
      int32_t run = base[threadIdx.x];
#pragma unroll
      for (int w = 0; w < 16; ++w) {
        const int32_t c = bins[w][threadIdx.x];
        bins[w][threadIdx.x] = run;
        run += c;
      }
      base[threadIdx.x] = run;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      if (key[r] < 0) continue;
      const int32_t to = bins[wave][(key[r] >> d.shift) & mask] + rank[r];
      out.key[to] = key[r];
      out.pos[to] = pos[r];
    }
  }
}

struct GradOut {
  void* dst;                          // vocab x cols, or rows in the order of the first of their tokens
  int32_t* index;                     // rows: row of dst of an id, behind it the id of a row of dst (null: dense)
  float* part;                        // two partial rows a tile: of the run it goes on with, and of the one that goes on behind it
  float scale;
  int32_t add;
};

// A workgroup sums the runs of one id that begin in its tile of sorted tokens, a thread sixteen bytes of columns.  A run that ends in the next tile is summed here to its
// end, so a tile works on at most two tiles of tokens and only longer runs leave partial rows: one of the tile they begin in (slot 1), one
// of each tile they go on in (slot 0).  Every wave holds ids and positions of both tiles, a lane one; rows are requested eight at a time, with
// them what the output holds where the sums are added to it.  NARROW: rows shorter than a piece, a thread an element.
// HBM: 57344 of 65536 rows of 2048 bf16 summed to 13000 of fp32: 63 us, 5.5 TB/s (one row in flight: 142 us); 8192 rows of 4096 fp32 to 3500: 32 us.
// 4095 rows of 1023 bf16 added: 7.8 us, latency (what the output holds requested at the end of each run: 47 us).
template <bool IN_BF, bool OUT_BF, bool ADD, bool NARROW>
__global__ __launch_bounds__(256) void k_tile_sum(const void* dy, Sorted in, int32_t tokens, int32_t tile_tokens, int32_t vocab, int64_t cols, GradOut o) {
  constexpr int VEC = NARROW ? 1 : IN_BF ? 8 : 4, AHEAD = 8;
  const int32_t tile = (int32_t)blockIdx.x, first = tile * tile_tokens;
  const int lane = threadIdx.x & 63;
  const int32_t at = first + lane;
  const int32_t key = lane < 2 * tile_tokens && at < tokens ? in.key[at] : vocab, pos = at < tokens ? in.pos[at] : 0;
  const int32_t before = first > 0 ? in.key[first - 1] : -1;                           // of the tile before: its last id,
  const int32_t earlier = first > tile_tokens ? in.key[first - tile_tokens - 1] : -1;  // and the last one before it
  const int32_t after = first + 2 * tile_tokens < tokens ? in.key[first + 2 * tile_tokens] : vocab;
  const int there = __popcll(__ballot(key != vocab));                                  // (tokens that take no part are at the end)
  if (there == 0) return;
  const int32_t next = __shfl_down(key, 1);
  const uint64_t ends = __ballot(lane < 2 * tile_tokens && key != (lane == 2 * tile_tokens - 1 ? after : next));
  const int32_t head = __builtin_amdgcn_readfirstlane(key);
  const bool came = head == before;
  const int head_end = ends ? __ffsll((unsigned long long)ends) - 1 : 64;
  const bool came_far = came && (head == earlier || head_end >= tile_tokens);          // longer than the tile before may finish
  const int begin = came && !came_far ? head_end + 1 : 0;
  int limit = tile_tokens;
  if (!(came_far && head_end >= tile_tokens - 1)) {
    const uint64_t later = ends >> (tile_tokens - 1);                                  // (bit 0: a run ends with the tile)
    if (later) limit = tile_tokens + __ffsll((unsigned long long)later) - 1;
  }
  limit = std::min(limit, there);
  const int64_t c0 = ((int64_t)blockIdx.y * blockDim.x + threadIdx.x) * VEC;
  if (c0 - lane * VEC >= cols) return;                 // a whole wave: every lane of the others stays, for what it holds of the two tiles
  const int64_t c = std::min(c0, cols - VEC);          // the last piece of a row ends where the row does
  const int skip = (int)std::min<int64_t>(c0 - c, VEC);
  float sum[VEC] = {};
  int start = begin;
  for (int s = begin; s < limit; s += AHEAD) {
    Piece<IN_BF, VEC> x[AHEAD];
    Piece<OUT_BF, VEC> old[ADD ? AHEAD : 1];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int l = std::min(s + k, limit - 1);
      x[k].load(dy, (int64_t)__builtin_amdgcn_readlane(pos, l) * cols + c);
      if constexpr (ADD) old[k].load(o.dst, (int64_t)__builtin_amdgcn_readlane(key, l) * cols + c);
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (s + k >= limit) break;
#pragma unroll
      for (int e = 0; e < VEC; ++e) sum[e] += x[k].value(e);
      const bool done = (ends >> (s + k)) & 1;
      if (!done && s + k + 1 < limit) continue;
      const bool part = came_far && start == 0;
      const int32_t id = __builtin_amdgcn_readlane(key, s + k);
      if (!part && o.index && c0 == 0) {
        o.index[id] = first + start;
        o.index[vocab + first + start] = id;
      }
      if (part || !done) {
        put_piece<false, VEC>(o.part, ((int64_t)tile * 2 + (part ? 0 : 1)) * cols + c, sum, skip);
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          sum[e] *= o.scale;
          if constexpr (ADD) sum[e] += old[k].value(e);
        }
        put_piece<OUT_BF, VEC>(o.dst, (int64_t)(o.index ? first + start : id) * cols + c, sum, skip);
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) sum[e] = 0.f;
      start = s + k + 1;
    }
  }
}

// Runs longer than two tiles: the partial rows of each in order.  A workgroup looks at one tile, 1024 columns of it; its four groups of four waves take consecutive
// shares of the tiles that a run goes on in.
// Latency of three dependent loads and the launch: 6 to 10 us (65536 tokens; 46 with sixteen tiles a workgroup and one request in flight).
template <bool OUT_BF>
__global__ __launch_bounds__(1024) void k_join_tiles(Sorted in, int32_t tokens, int32_t tile_tokens, int32_t vocab, int64_t cols, GradOut o) {
  const int32_t tile = (int32_t)blockIdx.x, first = tile * tile_tokens, tiles = (tokens + tile_tokens - 1) / tile_tokens;
  // its last run goes on over the whole next tile (which is not the last: the grid ends two tiles before the end) and began in this one
  const int32_t id = in.key[first + tile_tokens - 1], beyond = in.key[first + 2 * tile_tokens], before = first > 0 ? in.key[first - 1] : -1;
  if (id == vocab || beyond != id || before == id) return;
  __shared__ float sums[4][1024];
  const int lane = threadIdx.x & 63, group = threadIdx.x >> 8, column = (threadIdx.x & 255) * 4;
  const int64_t c = (int64_t)blockIdx.y * 1024 + column;
  const int cnt = cols - c >= 4 ? 4 : cols > c ? (int)(cols - c) : 0;
  const int32_t own = lane < tile_tokens ? in.key[first + lane] : id;
  float old[4] = {0.f, 0.f, 0.f, 0.f};                 // what the output holds, requested with what follows
  if (o.add && group == 0) {
    if (cnt == 4) load_quad<OUT_BF, false>(o.dst, (int64_t)id * cols + c, old);
    else
      for (int e = 0; e < cnt; ++e) old[e] = load_element<OUT_BF>(o.dst, (int64_t)id * cols + c + e);
  }
  int32_t last = tile + 2;                             // last tile that begins with the run
  for (bool more = true; more;) {
    const int32_t k = last + 1 + lane;
    const uint64_t same = __ballot(k < tiles && in.key[std::min(k, tiles - 1) * tile_tokens] == id);
    last += same == ~0ull ? 64 : __ffsll((unsigned long long)~same) - 1;
    more = same == ~0ull;
  }
  const uint64_t other = __ballot(own != id);
  const int start = other ? 64 - __clzll((long long)other) : 0;
  const int32_t each = (last - tile + 3) / 4, from = tile + 1 + group * each, to = std::min(from + each, last + 1);
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  const float* const p = o.part + c;
  if (group == 0)
    for (int e = 0; e < cnt; ++e) sum[e] = p[((int64_t)tile * 2 + 1) * cols + e];
  if (cnt == 4) {
    for (int32_t k = from; k < to; k += 8) {
      float x[8][4];
#pragma unroll
      for (int q = 0; q < 8; ++q) load_quad<false, false>(p, (int64_t)std::min(k + q, to - 1) * 2 * cols, x[q]);
#pragma unroll
      for (int q = 0; q < 8; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += k + q < to ? x[q][e] : 0.f;
    }
  } else {
    for (int32_t k = from; k < to; ++k)
      for (int e = 0; e < cnt; ++e) sum[e] += p[(int64_t)k * 2 * cols + e];
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) sums[group][column + e] = sum[e];
  __syncthreads();
  if (group != 0 || cnt == 0) return;
  const int64_t at = (int64_t)(o.index ? first + start : id) * cols + c;
#pragma unroll
  for (int e = 0; e < 4; ++e) sum[e] = (((sum[e] + sums[1][column + e]) + sums[2][column + e]) + sums[3][column + e]) * o.scale + old[e];
  if (cnt < 4)
    for (int e = 0; e < cnt; ++e) store_element<OUT_BF>(o.dst, at + e, sum[e]);
  else
    store_quad<OUT_BF, false>(o.dst, at, sum);
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

template <bool IN_BF, bool OUT_BF>
void launch_lookup_as(const void* table, Ids ids, int64_t tokens, int64_t cols, float scale, void* out, hipStream_t s) {
  const bool narrow = cols < 8;
  const int64_t pieces = narrow ? cols : (cols + 7) / 8;
  int lanes_log2 = 0;
  while (lanes_log2 < 8 && (int64_t(1) << lanes_log2) < pieces) ++lanes_log2;
  const int64_t per = 256 >> lanes_log2, columns = (pieces + (int64_t(1) << lanes_log2) - 1) >> lanes_log2;
  for (int64_t at = 0; at < tokens; at += LOOKUP_TOKENS) {
    const int64_t n = std::min(tokens - at, LOOKUP_TOKENS);
    Ids part = ids;
    part.p = reinterpret_cast<const char*>(ids.p) + at * (ids.wide ? 8 : 4);
    void* const to = reinterpret_cast<char*>(out) + at * cols * (OUT_BF ? 2 : 4);
    const dim3 grid((unsigned)((n + per - 1) / per), (unsigned)columns), block(256);
    if (narrow) hipLaunchKernelGGL((k_lookup<IN_BF, OUT_BF, true>), grid, block, 0, s, table, part, n, cols, lanes_log2, scale, to);
    else hipLaunchKernelGGL((k_lookup<IN_BF, OUT_BF, false>), grid, block, 0, s, table, part, n, cols, lanes_log2, scale, to);
  }
}
void launch_lookup(const void* table, bool in_bf, Ids ids, int64_t tokens, int64_t cols, float scale, void* out, bool out_bf, hipStream_t s) {
  if (in_bf && out_bf) launch_lookup_as<true, true>(table, ids, tokens, cols, scale, out, s);
  else if (in_bf) launch_lookup_as<true, false>(table, ids, tokens, cols, scale, out, s);
  else if (out_bf) launch_lookup_as<false, true>(table, ids, tokens, cols, scale, out, s);
  else launch_lookup_as<false, false>(table, ids, tokens, cols, scale, out, s);
}

// Threads of a row of k_tile_sum, and tokens of its tiles: as many as leave 4096 waves (four a SIMD), 8 to 32.  Within 6 % of the best of 8, 16 and 32 for 2048 to 65536
// tokens of 64 to 4096 columns; the whole gradient by rows in us, tiles of 8, 16 and 32: 2048 x 512 bf16 12.5, 14.4, 18.6 (8); 8192 x 2048 30.1, 28.5, 31.1 (8 taken),
// fp32 34.1, 32.3, 33.1 (16); 65536 x 2048 bf16 160, 138, 126 (32).
struct GradShape { int64_t pieces; unsigned threads; int tile; bool narrow; };
GradShape gradient_shape(int64_t tokens, int64_t cols, bool in_bf) {
  GradShape g;
  const int vec = in_bf ? 8 : 4;
  g.narrow = cols < vec;
  g.pieces = g.narrow ? cols : (cols + vec - 1) / vec;
  g.threads = (unsigned)std::min<int64_t>(256, (g.pieces + 63) / 64 * 64);
  const int64_t waves = (g.pieces + 63) / 64;
  g.tile = MOST_TILE;
  while (g.tile > 8 && (tokens + g.tile - 1) / g.tile * waves < 4096) g.tile /= 2;
  return g;
}

struct GradPlan { int64_t key[2], pos[2], count, part, bytes; };
GradPlan plan_gradient(int64_t tokens, int64_t cols) {
  GradPlan p;
  const int64_t list = up256(4 * tokens);
  const int tile = std::min(gradient_shape(tokens, cols, false).tile, gradient_shape(tokens, cols, true).tile);
  int64_t at = 0;
  for (int k = 0; k < 2; ++k) { p.key[k] = at; p.pos[k] = at + list; at += 2 * list; }
  p.count = at;
  p.part = p.count + 4 * PLACE_BLOCKS * MAX_BINS;
  p.bytes = p.part + up256((tokens + tile - 1) / tile * 2 * cols * 4);
  return p;
}

template <bool IN_BF, bool OUT_BF>
void launch_tile_sum(const GradShape& g, bool add, dim3 grid, hipStream_t s, const void* dy, Sorted in, int32_t n, int32_t vocab, int64_t cols, const GradOut& o) {
  const dim3 block(g.threads);
  if (add && g.narrow) hipLaunchKernelGGL((k_tile_sum<IN_BF, OUT_BF, true, true>), grid, block, 0, s, dy, in, n, g.tile, vocab, cols, o);
  else if (add) hipLaunchKernelGGL((k_tile_sum<IN_BF, OUT_BF, true, false>), grid, block, 0, s, dy, in, n, g.tile, vocab, cols, o);
  else if (g.narrow) hipLaunchKernelGGL((k_tile_sum<IN_BF, OUT_BF, false, true>), grid, block, 0, s, dy, in, n, g.tile, vocab, cols, o);
  else hipLaunchKernelGGL((k_tile_sum<IN_BF, OUT_BF, false, false>), grid, block, 0, s, dy, in, n, g.tile, vocab, cols, o);
}

int embed_gradient(Ids ids, int64_t tokens, const void* dy, int32_t dy_dtype, int64_t cols, float scale, void* dst, int32_t dst_dtype, int32_t* index, bool add,
                   char* ws, hipStream_t s) {
  const GradPlan p = plan_gradient(tokens, cols);
  Sorted sorted[2];
  for (int k = 0; k < 2; ++k) sorted[k] = Sorted{reinterpret_cast<int32_t*>(ws + p.key[k]), reinterpret_cast<int32_t*>(ws + p.pos[k])};
  const GradOut o{dst, index, reinterpret_cast<float*>(ws + p.part), scale, add ? 1 : 0};
  // where no token is: zeros in a dense gradient that is overwritten, no row for an id and no id for a row
  Fill fill{index ? index : dst, index ? 4 * (ids.vocab + tokens) : add ? 0 : (int64_t)ids.vocab * cols * (dst_dtype == LORDO_F32 ? 4 : 2), index ? 0xffffffffu : 0u};
  const int fill_blocks = (int)std::min<int64_t>((fill.bytes + 65535) / 65536, 2048);
  int key_bits = 1, pos_bits = 1;
  while ((ids.vocab >> key_bits) != 0) ++key_bits;
  while (((tokens - 1) >> pos_bits) > 0) ++pos_bits;
  const int32_t n = (int32_t)tokens, vocab = ids.vocab;
  int last = 0, rc = LORDO_OK;
  if (tokens == 0 || (tokens <= RANK_TOKENS && key_bits + pos_bits <= 32)) {
    const int rank_blocks = (n + RANK_ROW - 1) / RANK_ROW;
    if (rank_blocks + fill_blocks == 0) return LORDO_OK;
    hipLaunchKernelGGL(k_rank, dim3((unsigned)(rank_blocks + fill_blocks)), dim3(1024), 0, s, ids, n, pos_bits, sorted[0], rank_blocks, fill);
    rc = launched("k_rank");
    if (rc != LORDO_OK || tokens == 0) return rc;
  } else {
    int32_t* const count = reinterpret_cast<int32_t*>(ws + p.count);
    Digit d;
    d.tokens = n;
    d.block = (int32_t)((tokens + (int64_t)PLACE_BLOCKS * PLACE_CHUNK - 1) / ((int64_t)PLACE_BLOCKS * PLACE_CHUNK)) * PLACE_CHUNK;
    d.blocks = (n + d.block - 1) / d.block;
    const int digits = (key_bits + 8) / 9;
    d.bits = (key_bits + digits - 1) / digits;
    // every launch fills a share, while its own few workgroups wait for memory
    const int64_t piece = 65536 * 2 * digits, share = (fill.bytes + piece - 1) / piece * 65536;
    auto next_fill = [&] {
      Fill f = fill;
      f.bytes = std::min(share, fill.bytes);
      fill.p = reinterpret_cast<char*>(fill.p) + f.bytes;
      fill.bytes -= f.bytes;
      return f;
    };
    auto grid_of = [&](const Fill& f, int threads) {
      return dim3((unsigned)(d.blocks + std::min<int64_t>((f.bytes + 65535) / 65536, 2048 * (1024 / threads))));
    };
    for (int k = 0; k < digits && rc == LORDO_OK; ++k) {
      d.shift = k * d.bits;
      const Sorted &from = sorted[(k + 1) & 1], &to = sorted[k & 1];
      Fill f = next_fill();
      if (k == 0) hipLaunchKernelGGL(k_count<true>, grid_of(f, 256), dim3(256), 0, s, ids, from, d, count, f);
      else hipLaunchKernelGGL(k_count<false>, grid_of(f, 256), dim3(256), 0, s, ids, from, d, count, f);
      f = next_fill();
      if (k == 0) hipLaunchKernelGGL(k_place<true>, grid_of(f, 1024), dim3(1024), 0, s, ids, from, to, d, count, f);
      else hipLaunchKernelGGL(k_place<false>, grid_of(f, 1024), dim3(1024), 0, s, ids, from, to, d, count, f);
      rc = launched("k_place");
      last = k & 1;
    }
    if (rc != LORDO_OK) return rc;
  }
  const Sorted in = sorted[last];
  const bool in_bf = dy_dtype == LORDO_BF16, out_bf = dst_dtype == LORDO_BF16;
  const GradShape g = gradient_shape(tokens, cols, in_bf);
  const unsigned tiles = (unsigned)((tokens + g.tile - 1) / g.tile);
  const dim3 grid(tiles, (unsigned)((g.pieces + g.threads - 1) / g.threads));
  if (in_bf && out_bf) launch_tile_sum<true, true>(g, add, grid, s, dy, in, n, vocab, cols, o);
  else if (in_bf) launch_tile_sum<true, false>(g, add, grid, s, dy, in, n, vocab, cols, o);
  else if (out_bf) launch_tile_sum<false, true>(g, add, grid, s, dy, in, n, vocab, cols, o);
  else launch_tile_sum<false, false>(g, add, grid, s, dy, in, n, vocab, cols, o);
  rc = launched("k_tile_sum");
  if (rc != LORDO_OK || tiles < 3) return rc;          // (no run is longer than two tiles)
  const dim3 join(tiles - 2, (unsigned)((cols + 1023) / 1024));
  if (out_bf) hipLaunchKernelGGL((k_join_tiles<true>), join, dim3(1024), 0, s, in, n, g.tile, vocab, cols, o);
  else hipLaunchKernelGGL((k_join_tiles<false>), join, dim3(1024), 0, s, in, n, g.tile, vocab, cols, o);
  return launched("k_join_tiles");
}

}  // namespace

extern "C" {

int lordo_embed_lookup(const void* table, int32_t table_dtype, int64_t vocab, int64_t cols, const void* ids, int32_t ids_dtype, int64_t tokens,
                       double scale, void* out, int32_t out_dtype, void* stream) {
  if (!good_table(vocab, cols) || !good_ids(ids, ids_dtype, tokens) || !float_type(table_dtype) || !float_type(out_dtype) || !finite_in_fp32(scale))
    return LORDO_EINVAL;
  if (tokens == 0) return LORDO_OK;
  if (!table || !out || !float_aligned(table, table_dtype) || !float_aligned(out, out_dtype)) return LORDO_EINVAL;
  const Ids id{ids, ids_dtype == LORDO_I64, (int32_t)vocab, -1};
  launch_lookup(table, table_dtype == LORDO_BF16, id, tokens, cols, (float)scale, out, out_dtype == LORDO_BF16, reinterpret_cast<hipStream_t>(stream));
  return launched("k_lookup");
}

int lordo_embed_workspace_bytes(int64_t tokens, int64_t vocab, int64_t cols, size_t* out_bytes) {
  if (!out_bytes || !good_table(vocab, cols) || tokens < 0 || tokens > LORDO_MAX_TOKENS) return LORDO_EINVAL;
  *out_bytes = (size_t)plan_gradient(tokens, cols).bytes;
  return LORDO_OK;
}

int lordo_embed_gradient(const void* ids, int32_t ids_dtype, int64_t tokens, const void* dy, int32_t dy_dtype, int64_t vocab, int64_t cols, double scale,
                         int64_t pad_id, int32_t accumulate, void* dw, int32_t dw_dtype, void* workspace, size_t workspace_bytes, void* stream) {
  if (!good_table(vocab, cols) || !good_ids(ids, ids_dtype, tokens) || !float_type(dy_dtype) || !float_type(dw_dtype) || !finite_in_fp32(scale))
    return LORDO_EINVAL;
  if ((accumulate != 0 && accumulate != 1) || !dw || !float_aligned(dw, dw_dtype)) return LORDO_EINVAL;
  if (tokens > 0 && (!dy || !float_aligned(dy, dy_dtype) || !workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0)) return LORDO_EINVAL;
  if (workspace_bytes < (size_t)plan_gradient(tokens, cols).bytes) return LORDO_ENOMEM;
  return embed_gradient(Ids{ids, ids_dtype == LORDO_I64, (int32_t)vocab, pad_id}, tokens, dy, dy_dtype, cols, (float)scale, dw, dw_dtype, nullptr,
                        accumulate != 0, reinterpret_cast<char*>(workspace), reinterpret_cast<hipStream_t>(stream));
}

int lordo_embed_gradient_rows(const void* ids, int32_t ids_dtype, int64_t tokens, const void* dy, int32_t dy_dtype, int64_t vocab, int64_t cols, double scale,
                              int64_t pad_id, void* rows, int32_t rows_dtype, int32_t* index, void* workspace, size_t workspace_bytes, void* stream) {
  if (!good_table(vocab, cols) || !good_ids(ids, ids_dtype, tokens) || !float_type(dy_dtype) || !float_type(rows_dtype) || !finite_in_fp32(scale))
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
