// Attention of a batch's query rows over the paged cache:
//
//   o = sum_j softmax_j(scale q . k_j) v_j,  lse = log sum_j exp(scale q . k_j)
//
// over the tokens of the row's prefix run (all of them) and of its own run (up
// to the row's own place, or all).
//
// A tile is 16 or 128 consecutive (row, head) pairs of one segment and one key
// head: a segment is a sequence's rows, over its own run, or the rows of all
// the sequences of a group, over the group's prefix, which is so read once for
// all of them.  Pair x of a segment is row x / r, head x % r of the key head's r
// query heads, so grouped heads share every key and value that is read.  Keys
// are cut into chunks; a workgroup takes a tile, a key head and a chunk, and
// keeps the running maximum m, the sum l of 2^(s - m) and the values weighted by
// 2^(s - m) (scores s in powers of two).  A row with a single part is done; the
// others' parts go to the workspace and combine_kernel joins them:
//   o = sum_p 2^(m_p - M) o_p / sum_p 2^(m_p - M) l_p,  M = max_p m_p.
//
// A sequence's pairs to a key head decide what its rows run in:
//   up to 16          thin tiles (memory-bound: the waves split the keys); in a batch of
//                     few and short ones wide_kernel's, with twice the waves, the prefix
//                     beside the own run, and no parts
//   more              tall tiles (the waves split the pairs)
//   more than kFuse   tall tiles that take the prefix's keys first and then its own:
//                     such a sequence fills tiles by itself, so sharing the prefix's
//                     reads saves nothing and parts would only be written and read.
// Where that is less work, all sequences of a batch take their prefixes so (ALONE).
//
// Scores, maxima, sums and outputs are float32.  A probability is rounded to the cache's type
// where it meets its value: the bfloat16 matrix instructions take both operands so, and a second
// product for the rest would be half as much work again in the tall tiles, which the matrix cores'
// power bounds.  The thin tiles round alike, so that a row has one accuracy whatever batch it is
// in.  The sum l takes the probabilities unrounded.  Against 64 bits the bfloat16 cases are off by
// 2.0e-3 to 2.3e-3 of the output (root mean square), of which 1.65e-3 is the output's own rounding.
#include <float.h>

#include <algorithm>
#include <type_traits>

#include "sp_internal.h"
#include "cache_rows.h"
#include "lds_dma.h"

namespace sp {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) bf16x4_t* ltr_t;
typedef __attribute__((address_space(3))) char* lds_t;

constexpr int kThin = 16, kTall = 128;     // pairs of a tile
constexpr int kFuse = 64;                  // pairs of a sequence past which it takes its prefix by itself
constexpr int kWaves = 4;
constexpr int kWide = 8;                   // of a wide workgroup
constexpr int kMaxParts = 1024;
constexpr int kThinStep = 16 * kWaves;     // keys that the waves of a thin tile take together
constexpr int kTallStep = 64;
// Running maxima start here: a masked score (-inf) then weighs 2^-inf = 0 also
// where a row has seen nothing yet.
constexpr float kLowest = -FLT_MAX;
constexpr float kRescale = 8.0f;           // log2 of the largest unscaled probability

// The kernel's arguments where they lie, read again from there: code after a long loop
// that reads them through this keeps no scalar registers for them over the loop.
__device__ __forceinline__ const AttendArgs& arguments() {
  auto p = (const __attribute__((address_space(4))) AttendArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const AttendArgs*)p;
}

// LDS that lanes of one wave exchange: its accesses are in order by themselves, the
// compiler's are by this.
__device__ __forceinline__ void lds_exchanged() { asm volatile("" ::: "memory"); }

// 16 bytes of a type.
template <typename T>
struct Chunk;
template <>
struct Chunk<__bf16> {
  static constexpr int N = 8;
  typedef bf16x8_t vec;
};
template <>
struct Chunk<float> {
  static constexpr int N = 4;
  typedef f32x4_t vec;
};

// The 64-bit number that lane `from` holds, in scalar registers.
__device__ __forceinline__ int64_t lane_value(uint32_t lo, uint32_t hi, int from) {
  const uint32_t l = __builtin_amdgcn_readlane(lo, from), h = __builtin_amdgcn_readlane(hi, from);
  return (int64_t)((uint64_t)h << 32 | l);
}

// ---------------------------------------------------------------- tiles

struct Tile {
  int64_t row0;           // the segment's first row
  int pairs;              // rows of the segment times r
  int x0;                 // the tile's first pair
  int seg;                // sequence or group
  int n;                  // rows of the segment
  int len;                // tokens of its run
  const int32_t* table;   // its pages
  int group, before;      // (tall tiles of a sequence) its group, -1 without one, and the tokens of the prefix
};

__device__ __forceinline__ int ratio(const AttendArgs& a) { return a.shape.q_heads / a.shape.kv_heads; }

// Group g's rows: those from its first sequence's to the next group's.
__device__ __forceinline__ int group_rows(const AttendArgs& a, int g, int64_t& first, int64_t& n) {
  const int s0 = a.grp_off[g], s1 = a.grp_off[g + 1];
  if (s0 < 0 || s1 < s0 || s1 > a.runs.count) return SP_DEV_BAD_OFFSETS;
  first = first_row(a.rows, s0);
  n = first_row(a.rows, s1) - first;
  return first < 0 || n < 0 || first + n > a.rows.rows ? SP_DEV_BAD_OFFSETS : SP_DEV_OK;
}

// Tile `index` of TILE pairs among all segments' tiles.  Segment i's tiles are
// numbered from floor(first row r / TILE) + i on, which leaves each segment as many
// numbers as it has tiles or one more, needs no sum over the segments, and bounds the
// grid by rows r / TILE + segments.  False: the number is nobody's.
template <int TILE>
__device__ __forceinline__ bool find_tile(const AttendArgs& a, bool prefix, int index, Tile& t) {
  const int r = ratio(a);
  const int count = prefix ? a.prefix.count : a.runs.count;
  auto start = [&](int i) {
    const int s = prefix ? min(max(a.grp_off[i], 0), a.runs.count) : i;
    return first_row(a.rows, s) * r / TILE + i;
  };
  t.seg = wave_find_last(count, (int64_t)index, start);
  int64_t n;
  if (prefix) {
    if (group_rows(a, t.seg, t.row0, n) != SP_DEV_OK) return false;
  } else {
    int rows;
    if (rows_of(a.rows, t.seg, t.row0, rows) != SP_DEV_OK) return false;
    n = rows;
  }
  const int64_t x0 = ((int64_t)index - (t.row0 * r / TILE + t.seg)) * TILE;
  if (x0 < 0 || x0 >= n * r) return false;
  t.n = (int)n;
  t.pairs = (int)(n * r);
  t.x0 = (int)x0;
  const CacheRuns& runs = prefix ? a.prefix : a.runs;
  t.table = runs.table + (int64_t)t.seg * runs.width;
  return tokens_of(runs, t.seg, t.len) == SP_DEV_OK;
}

// The group of sequence s: -1 without one.
__device__ __forceinline__ int group_of(const AttendArgs& a, int s) {
  if (a.prefix.count == 0) return -1;
  const int g = wave_find_last(a.prefix.count, s, [&](int i) { return a.grp_off[i]; });
  return s < a.grp_off[g] || s >= a.grp_off[g + 1] ? -1 : g;
}

// The tokens of its prefix.  (`len` is the prefixes' entry: loaded ahead of its use)
__device__ __forceinline__ int prefix_tokens(const AttendArgs& a, int g, int len) {
  return g < 0 || len < 0 || len > a.prefix.max_len ? 0 : len;
}

__device__ __forceinline__ void find_prefix(const AttendArgs& a, Tile& t) {
  t.group = group_of(a, t.seg);
  t.before = prefix_tokens(a, t.group, t.group < 0 ? 0 : a.prefix.len[t.group]);
}

// The same for tall tiles of up to 64 segments, a lane to each: the segments with the most
// keys come first, and of a segment the tiles with the most, so that the launch ends with
// small work.  (64 prompts on prefixes of 894 to 2264 tokens, 28 heads on 4: in the order
// of the batch 154 us, in this one 137.)
constexpr int kSorted = 64;
// LDS: kSorted entries of `table`, the wave's own.
template <bool ALONE>
__device__ __forceinline__ bool find_sorted_tile(const AttendArgs& a, bool prefix, int index, Tile& t, uint2* table) {
  const int lane = threadIdx.x & 63, r = ratio(a), G = a.prefix.count;
  const CacheRuns& runs = prefix ? a.prefix : a.runs;
  const bool grouped = !prefix && G > 0 && G <= 64;          // a lane to a group
  int64_t row0 = 0, n = 0;
  int len = 0, tiles = 0, off = INT_MAX, end = 0, tokens = 0, group = -1;
  if (lane < runs.count) {
    int rows = 0;
    bool ok;
    if (prefix) {
      ok = group_rows(a, lane, row0, n) == SP_DEV_OK;
    } else {
      ok = rows_of(a.rows, lane, row0, rows) == SP_DEV_OK && (int64_t)rows * r > kThin;    // (others are thin tiles)
      n = rows;
    }
    ok = tokens_of(runs, lane, len) == SP_DEV_OK && ok;
    if (ok) tiles = (int)((n * r + kTall - 1) / kTall);
  }
  if (grouped) {
    if (lane < G) {
      off = a.grp_off[lane];
      end = a.grp_off[lane + 1];
      tokens = a.prefix.len[lane];
    }
    int* const offsets = reinterpret_cast<int*>(table);
    offsets[lane] = off;
    lds_exchanged();
    for (int k = 0; k < G; k += 8)
#pragma unroll
      for (int i = 0; i < 8; ++i) group += offsets[k + i] <= lane;
    lds_exchanged();
    end = __shfl(end, max(group, 0));
    tokens = __shfl(tokens, max(group, 0));
    if (lane >= end) group = -1;
    tokens = prefix_tokens(a, group, tokens);
  }
  // order: keys, then the place in the batch
  const uint32_t keys = (uint32_t)len + (grouped && (ALONE || n * r > kFuse) ? (uint32_t)tokens : 0);
  const uint32_t order = min(keys, (1u << 26) - 1) << 6 | (63 - lane);
  table[lane] = make_uint2(order, (uint32_t)tiles);
  lds_exchanged();
  int start = 0;
#pragma unroll 1
  for (int k = 0; k < runs.count; k += 16)           // (the lanes past the last segment have no tiles)
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const uint4 v = *reinterpret_cast<const uint4*>(table + k + i);
      start += (v.x > order ? v.y : 0) + (v.z > order ? v.w : 0);
    }
  const uint64_t mine = __ballot(index >= start && index < start + tiles);
  if (mine == 0) return false;
  t.seg = __builtin_ctzll(mine);
  t.row0 = lane_value((uint32_t)row0, (uint32_t)(row0 >> 32), t.seg);
  t.n = __builtin_amdgcn_readlane((int)n, t.seg);
  t.len = __builtin_amdgcn_readlane(len, t.seg);
  t.pairs = t.n * r;
  t.x0 = (__builtin_amdgcn_readlane(start, t.seg) + __builtin_amdgcn_readlane(tiles, t.seg) - 1 - index) * kTall;
  t.table = runs.table + (int64_t)t.seg * runs.width;
  t.group = __builtin_amdgcn_readlane(group, t.seg);
  t.before = __builtin_amdgcn_readlane(tokens, t.seg);
  if (!prefix && G > 64) find_prefix(a, t);
  return true;
}

// Errors of the batch's entries, wherever they are; by one workgroup of a launch.
__device__ __forceinline__ void report_entries(const AttendArgs& a, bool prefix) {
  const int count = prefix ? a.prefix.count : a.runs.count;
  for (int i = threadIdx.x; i < count; i += blockDim.x) {
    int64_t f, m;
    int n, len;
    int code = prefix ? group_rows(a, i, f, m) : rows_of(a.rows, i, f, n);
    if (code == SP_DEV_OK) code = tokens_of(prefix ? a.prefix : a.runs, i, len);
    if (code != SP_DEV_OK) set_device_error(a.err, code);
  }
}

// Tokens of the segment's run that its row `row` sees.
__device__ __forceinline__ int sees(const AttendArgs& a, const Tile& t, bool prefix, int row) {
  if (prefix || a.all) return t.len;
  const int64_t v = (int64_t)t.len - t.n + row + 1;
  return v < 0 ? 0 : (int)v;
}

__device__ __forceinline__ const int32_t* pages_of(const AttendArgs& a, bool prefix, int i) {
  return prefix ? a.prefix.table + (int64_t)i * a.prefix.width : a.runs.table + (int64_t)i * a.runs.width;
}

__device__ __forceinline__ int ceil_div(int x, int y) { return (x + y - 1) / y; }

__device__ __forceinline__ int checked_page(const AttendArgs& a, int page) {
  if ((uint32_t)page < (uint32_t)a.shape.pages) return page;
  set_device_error(a.err, SP_DEV_BAD_PAGE);
  return 0;
}

// Where the keys from `key` on lie in the key array (the values: in the value array).
template <int ROW>
__device__ __forceinline__ int64_t place_of(const AttendArgs& a, int page, int h, int key) {
  const int shift = a.shape.page_shift;
  return (((int64_t)page * a.shape.kv_heads + h << shift) + (key & ((1 << shift) - 1))) * ROW;
}

// Places of the 16-key blocks that a wave takes, one every `stride` keys from `first` on:
// lane j holds that of block 64 (i / 64) + j, and the page of the block 64 further on.
// The pages' loads need no length (prime can go ahead of the loads of the batch's
// entries): entries past the run's tokens are read, within the table, and not used.
template <int ROW>
struct Places {
  const int32_t* table;
  int first, stride, width;
  uint32_t lo, hi;
  int ahead;
  __device__ __forceinline__ int entry(const AttendArgs& a, int i) const {
    const int64_t at = (first + (int64_t)stride * (i + (int)(threadIdx.x & 63))) >> a.shape.page_shift;
    return at < width ? table[at] : 0;
  }
  __device__ __forceinline__ void prime(const AttendArgs& a, const CacheRuns& runs, int run, int key, int step) {
    table = runs.table + (int64_t)run * runs.width;
    width = runs.width;
    first = key;
    stride = step;
    ahead = entry(a, 0);
  }
  // of block i, asked for in order
  __device__ __forceinline__ int64_t of(const AttendArgs& a, int len, int h, int i) {
    if ((i & 63) == 0) {
      const int64_t key = first + (int64_t)stride * (i + (int)(threadIdx.x & 63));
      const int64_t at = place_of<ROW>(a, checked_page(a, key < len ? ahead : 0), h, (int)key);
      lo = (uint32_t)at;
      hi = (uint32_t)(at >> 32);
      ahead = entry(a, i + 64);
    }
    return lane_value(lo, hi, i & 63);
  }
};

// ---- where a pair's result goes

struct Out {
  int64_t pair;           // row q_heads + head; -1: nowhere
  bool done;              // the only part: into O; else a part, at
  float* o;
  float2* ml;
};

// Sequences of up to this many pairs are short: their parts lie by sequence.
__device__ __forceinline__ bool is_short(const AttendArgs& a, int pairs) { return pairs <= a.plan.short_pairs; }

// Where the parts of row i of sequence s, row `row` of the batch, begin: by row where all
// sequences are short (its sequence need not be known then), else by sequence (the rows of
// the long ones would leave large gaps).
__device__ __forceinline__ int64_t short_base(const AttendArgs& a, int64_t row, int s, int i) {
  return (a.plan.by_row ? row : (int64_t)s * a.plan.short_rows + i) * a.shape.q_heads;
}

// Pair x of sequence t.seg and key head h: the place of its result over chunk `chunk` of
// the `own` chunks of its own keys, with `pre` parts of its prefix beside them.  First
// chunk: the row's parts, for combine_kernel.
__device__ __forceinline__ Out own_place(const AttendArgs& a, const Tile& t, int h, int x, int chunk, int own, int pre) {
  Out u;
  u.pair = -1;
  u.done = pre == 0 && own <= 1;                     // (a row that sees nothing: zeros, by its first chunk)
  const int r = ratio(a), i = x / r, head = h * r + (x - i * r);
  const int64_t row = t.row0 + i;
  if (chunk == 0 && h == 0 && x == i * r) a.row_parts[row] = make_int2(u.done ? 0 : own, pre);
  if (chunk >= own && !(u.done && chunk == 0)) return u;
  u.pair = row * a.shape.q_heads + head;
  int64_t at;
  if (is_short(a, t.pairs)) {
    at = (short_base(a, row, t.seg, i) + head) * a.plan.short_parts + chunk;
    u.o = a.short_o;
    u.ml = reinterpret_cast<float2*>(a.short_ml);
  } else {
    at = u.pair * a.plan.tall_parts + chunk;
    u.o = a.tall_o;
    u.ml = reinterpret_cast<float2*>(a.tall_ml);
  }
  u.o += at * a.shape.head_dim;
  u.ml += at;
  return u;
}

// The same for pair x of group t.seg over a chunk of the group's prefix.  Nowhere: a padded
// slice's rows past its count, and the rows of a sequence that takes the prefix by itself.
__device__ __forceinline__ Out prefix_place(const AttendArgs& a, const Tile& t, int h, int x, int chunk) {
  Out u;
  u.pair = -1;
  u.done = false;
  const int r = ratio(a), j = x / r, head = h * r + (x - j * r);
  const int64_t row = t.row0 + j;
  int s = 0, i = 0;
  if (a.rows.padded) {
    s = (int)(row / a.rows.rows_per_seq);
    i = (int)(row - (int64_t)s * a.rows.rows_per_seq);
    const int n = a.rows.info[s];
    if (i >= n || n > a.rows.max_rows || (int64_t)n * r > a.plan.short_pairs) return u;
  } else if (!a.plan.by_row) {                       // info[s] <= row < info[s + 1]
    s = a.grp_off[t.seg];
    for (int hi = a.grp_off[t.seg + 1]; hi - s > 1;) {
      const int mid = (s + hi) >> 1;
      if (a.rows.info[mid] <= row) s = mid;
      else hi = mid;
    }
    const int first = a.rows.info[s], n = a.rows.info[s + 1] - first;
    i = (int)(row - first);
    if (i < 0 || i >= n || n > a.rows.max_rows || (int64_t)n * r > a.plan.short_pairs) return u;
  }
  u.pair = row * a.shape.q_heads + head;
  const int64_t at = (short_base(a, row, s, i) + head) * a.plan.prefix_parts + chunk;
  u.o = a.prefix_o + at * a.shape.head_dim;
  u.ml = reinterpret_cast<float2*>(a.prefix_ml) + at;
  return u;
}

__device__ __forceinline__ float lse_of(float m, float l) {
  return l > 0.0f || l != l ? (m + __log2f(l)) * 0.6931471805599453f : -INFINITY;
}

__device__ __forceinline__ void store_ml(const AttendArgs& a, const Out& u, float m, float l) {
  if (!u.done) *u.ml = make_float2(m, l);
  else if (a.lse) a.lse[u.pair] = lse_of(m, l);
}

// ---------------------------------------------------------------- operands

__device__ __forceinline__ float half_max(float v) {      // of this lane and the lane 32 away
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float quad_max(float v) {      // of the four lanes 16 apart
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return half_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float quad_sum(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return half_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// A head's rows in LDS: ROW bytes each, 16-byte chunks swizzled so that a pass of a
// fragment read touches every bank once: K (a chunk of each of 16 or 32 rows) by the
// row, V (64 bytes of each of four rows) by the row on 64-byte pieces.
template <int D>
struct Geo {
  static constexpr int ROW = 2 * D, CHUNKS = ROW / 16, LOAD_ROWS = 1024 / ROW;   // rows of a load
  static constexpr int LOADS = 16 / LOAD_ROWS;                                    // loads of 16 keys
  __device__ static __forceinline__ int kswz(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }
  __device__ static __forceinline__ int vswz(int r) { return D == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2; }
};

// The loads of 16 keys (of one page) into LDS rows of K or of V: an instruction fills
// 1 KB, lane i lands on chunk i % CHUNKS of row i / CHUNKS and fetches the chunk that
// the swizzle puts there.  Keys past a run's end are loaded too (a page is whole), their
// scores masked and their values cleared (clear_rows).
template <int D>
struct Loader {
  using G = Geo<D>;
  uint32_t ko[G::LOADS], vo;
  __device__ __forceinline__ void init() {
    const int lane = threadIdx.x & 63, ch = lane % G::CHUNKS, lr = lane / G::CHUNKS;
#pragma unroll
    for (int g = 0; g < G::LOADS; ++g)
      ko[g] = g * 1024 + lr * G::ROW + ((ch ^ G::kswz(G::LOAD_ROWS * g + lr)) << 4);
    vo = lr * G::ROW + ((ch ^ G::vswz(lr)) << 4);
  }
  // load g of the 16 keys (values) from src, the same in all lanes
  __device__ __forceinline__ void keys(const char* src, uint32_t dst, int g) const { lds_dma16(src, ko[g], dst + g * 1024); }
  __device__ __forceinline__ void values(const char* src, uint32_t dst, int g) const {
    lds_dma16(src + g * 1024, vo, dst + g * 1024);
  }
};

// Zeros into rows `from` .. 15 of 16 rows.
template <int D>
__device__ __forceinline__ void clear_rows(char* rows, int from) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int c = 0; c < 16 * Geo<D>::CHUNKS; c += 64)
    if (c + lane >= from * Geo<D>::CHUNKS) *reinterpret_cast<uint4*>(rows + (c + lane) * 16) = make_uint4(0, 0, 0, 0);
}

// In a tile, a key that some pairs see and others do not is weighed with 0 for those,
// which is NaN where its value is infinite or NaN.  A wave with such a key whose outputs are
// not all finite begins again here, key by key, each pair over the keys that it sees alone
// (a hundred times slower, and never needed by sound data).  Lane l holds pair l % PAIRS;
// with p = l / PAIRS of P lanes a pair and E elements in 16 bytes, elements E (P s + p) + 0
// .. E - 1 of its query in q[s] and 4 (P g + p) + 0 .. 3 of its output in elements 4 g + 0
// .. 3 of o, whose vectors have W.
template <typename T, int D, int PAIRS, int W, typename O>
struct KeyByKey {
  using vec = typename Chunk<T>::vec;
  typedef T vec4 __attribute__((ext_vector_type(4)));
  static constexpr int P = 64 / PAIRS, E = Chunk<T>::N;
  O& o;
  float &m, &l;
  __device__ __forceinline__ KeyByKey(O& out, float& max, float& sum) : o(out), m(max), l(sum) {
#pragma unroll
    for (int e = 0; e < D / P; ++e) o[e / W][e % W] = 0.0f;
    m = kLowest;
    l = 0.0f;
  }
  __device__ __forceinline__ void add(const AttendArgs& a, const int32_t* table, int head, const vec (&q)[D / (E * P)],
                                      int from, int to, int lim) {
    const int p = (threadIdx.x & 63) / PAIRS;
#pragma unroll 1
    for (int key = from; key < to; ++key) {
      const int64_t at =
          place_of<D * (int)sizeof(T)>(a, checked_page(a, table[key >> a.shape.page_shift]), head, key);
      const char* K = static_cast<const char*>(a.k_cache) + at;
      const char* V = static_cast<const char*>(a.v_cache) + at;
      float dot = 0.0f;
#pragma unroll
      for (int s = 0; s < D / (E * P); ++s) {
        const vec k = *reinterpret_cast<const vec*>(K + 16 * (P * s + p));
#pragma unroll
        for (int j = 0; j < E; ++j) dot = fmaf((float)q[s][j], (float)k[j], dot);
      }
      const float st = P == 2 ? half_sum(dot) : quad_sum(dot);
      if (key < lim) {
        const float mn = fmaxf(m, st * a.c2), f = __builtin_amdgcn_exp2f(m - mn);
        float e = fmaf(st, a.c2, -mn);               // (as in the tiles)
        if (sizeof(T) == 4 && st > kLowest) e = fmaf(st, a.c2_low, e);
        const float w = __builtin_amdgcn_exp2f(e);
        m = mn;
        l = fmaf(l, f, w);
        const float wt = (float)(T)w;                // (as in the tiles)
#pragma unroll
        for (int g = 0; g < D / (4 * P); ++g) {
          const vec4 v = *reinterpret_cast<const vec4*>(V + sizeof(vec4) * (P * g + p));
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int i = 4 * g + k;
            o[i / W][i % W] = fmaf(wt, (float)v[k], o[i / W][i % W] * f);
          }
        }
      }
    }
  }
};

// ---------------------------------------------------------------- the thin tiles

// 16 pairs.  The keys of one head go to all four waves, each every fourth block of 16, and
// the waves' results are joined through LDS; or (spread) each wave takes a head of its own.
// Scores S^T = K Q^T and O^T += V^T P as in the tall tiles, with 16 x 16 matrices: lane l
// holds pair l % 16, scores of keys 4 (l / 16) + i, output elements 16 t + 4 (l / 16) + i.
//
// Bound by memory.  Two blocks are in registers or on their way there, K and V in whole
// 1 KB loads; through LDS they come into the operands' layouts.  Where they are read once,
// they are not kept in the caches (STREAM): 128 single tokens of 256 to 8192 keys, 28 heads
// on 4, 192 us (5.6 TB/s), with ordinary loads 202, and three blocks ahead 195; float32
// prompts, whose tiles read the same keys, lose by it: 32 of 200 rows over 1000 keys, 16
// heads of 64, 375 us and 333 with ordinary loads.  Key heads are innermost here too: 128
// tokens of 32 heads on 8 prefixes 133 us, with heads outermost 175.
template <typename T, int D, int WAVES>
struct ThinShape {
  static constexpr int ROW = D * (int)sizeof(T), CHUNKS = ROW / 16, LOAD_ROWS = 1024 / ROW, LOADS = 16 / LOAD_ROWS;
  // LDS rows: bfloat16 as in the tall tiles; float32 padded by 16 bytes, so that 16 rows'
  // chunks (K), and four rows' runs of 16 elements (V), touch every bank once
  static constexpr int LDS_ROW = sizeof(T) == 2 ? ROW : ROW + 16;
  static constexpr int BLOCK = 16 * LDS_ROW;                    // 16 keys of K or V
  static constexpr int PART_ROW = D + 4;
  static constexpr int DEPTH = 2;
  static constexpr int BLOCKS = 2 * WAVES * BLOCK, PARTS = WAVES * kThin * (PART_ROW + 2) * 4;
  static constexpr int LDS = BLOCKS > PARTS ? BLOCKS : PARTS;   // the blocks, then the waves' results
};

template <bool STREAM>
__device__ __forceinline__ u32x4_t fetch(const char* p) {
  if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
  else return *reinterpret_cast<const u32x4_t*>(p);
}

template <typename T, int D, bool STREAM, int WAVES, bool ALONE>
__device__ __forceinline__ void thin_tile(const AttendArgs& a, char* smem, bool prefix, const Tile& t,
                                          Places<D * (int)sizeof(T)>& places, int h, int chunk, int g, bool spread) {
  using SH = ThinShape<T, D, WAVES>;
  using vec = typename Chunk<T>::vec;
  constexpr int E = Chunk<T>::N, QS = D / (4 * E);               // query vectors of a lane
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ql = lane & 15, quad = lane >> 4, r = ratio(a);
  const int chunk_keys = prefix ? a.plan.chunk_prefix : a.plan.chunk_thin;
  const int prefix_len = prefix || g < 0 ? 0 : a.prefix.len[g];    // (used later)
  // a tile that takes the prefix too, with its first keys
  const bool both = ALONE && chunk == 0 && g >= 0;
  Places<D * (int)sizeof(T)> before = places;
  const int step = places.stride, own_first = places.first, prefix_first = spread ? 0 : 16 * wave;
  if (both) before.prime(a, a.prefix, g, prefix_first, step);
  // the last pair's limit is the tile's
  const int tile_end = sees(a, t, prefix, (min(t.x0 + kThin, t.pairs) - 1) / r);
  const int k0 = chunk * chunk_keys;
  if (k0 >= tile_end && (prefix || chunk > 0)) return;
  const int k1 = min(tile_end, k0 + chunk_keys);

  const int x = t.x0 + ql;
  const bool live = x < t.pairs;
  const int row = live ? x / r : 0;
  const T* qsrc = static_cast<const T*>(a.Q) + (t.row0 + row) * a.ldq + (h * r + (x - row * r)) * D + E * quad;
  vec q[QS];
#pragma unroll
  for (int s = 0; s < QS; ++s) {
    u32x4_t u = {0, 0, 0, 0};
    if (live) u = *reinterpret_cast<const u32x4_t*>(qsrc + 4 * E * s);
    q[s] = __builtin_bit_cast(vec, u);
  }
  const int own_lim = live ? sees(a, t, prefix, row) : 0, own_lim0 = sees(a, t, prefix, t.x0 / r);

  const char* const Kc = static_cast<const char*>(a.k_cache);
  const char* const Vc = static_cast<const char*>(a.v_cache);
  struct Block {
    u32x4_t k[SH::LOADS], v[SH::LOADS];
  };
  f32x4_t o[D / 16];
#pragma unroll
  for (int e = 0; e < D / 16; ++e) o[e] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  float m = kLowest, l = 0.0f;
  const float c2 = a.c2, c2_low = a.c2_low;
  // LDS addresses: K, then V; a lane writes chunk ch of row lr of each load
  typedef __attribute__((address_space(3))) u32x4_t* l16_t;
  typedef __attribute__((address_space(3))) float* l4_t;
  const uint32_t K = (uint32_t)(uintptr_t)(lds_t)smem + wave * 2 * SH::BLOCK, V = K + SH::BLOCK;
  const int lr = lane / SH::CHUNKS, ch = lane % SH::CHUNKS, vr = (lane >> 2) & 3;
  uint32_t kdst, ksrc, vdst, vsrc;
  if constexpr (sizeof(T) == 2) {
    // Row LOAD_ROWS c + lr of K has chunk ch at ch ^ kswz of the row, in which c and lr set
    // bits apart.  V^T's read: 16 lanes read four keys x 16 columns, lane i receives
    // column i of the four keys.
    using G = Geo<D>;
    kdst = K + lr * SH::ROW + ((ch ^ G::kswz(lr)) << 4);
    ksrc = K + ql * SH::ROW + ((quad ^ G::kswz(ql)) << 4);
    vdst = V + lr * SH::ROW + ((ch ^ G::vswz(lr)) << 4);
    vsrc = V + (4 * quad + vr) * SH::ROW + (G::vswz(vr) << 4) + (lane & 3) * 8;
  } else {
    kdst = K + lr * SH::LDS_ROW + ch * 16;
    ksrc = K + ql * SH::LDS_ROW + quad * 16;
    vdst = V + lr * SH::LDS_ROW + ch * 16;
    vsrc = V + 4 * quad * SH::LDS_ROW + ql * 4;
  }
  // keys of the tile's own run, then of the prefix
  for (int run = 0; run < (both ? 2 : 1); ++run) {
    const bool pre = run == 1;
    const int len = pre ? prefix_tokens(a, g, prefix_len) : t.len;
    const int to = pre ? len : k1, lim = pre ? len : own_lim, lim0 = pre ? len : own_lim0;
    if (pre) places = before;
    // block i of the wave: 16 keys from first + step i on
    const int first = pre ? prefix_first : own_first;
    const int blocks = to > first ? (to - first + step - 1) / step : 0;
    // No load is left out (the waits count them): past the last block all lanes load one place.
    auto load = [&](Block& b, int i) {
      const int64_t at = places.of(a, len, h, i);
      const uint32_t mine = i < blocks ? lane * 16 : 0, next = i < blocks ? 1024 : 0;
#pragma unroll
      for (int c = 0; c < SH::LOADS; ++c) b.k[c] = fetch<STREAM>(Kc + at + c * next + mine);
#pragma unroll
      for (int c = 0; c < SH::LOADS; ++c) b.v[c] = fetch<STREAM>(Vc + at + c * next + mine);
    };
    auto use = [&](Block& b, int i) {
      const int kb = first + step * i;
      f32x4_t st = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < SH::LOADS; ++c) {
        const uint32_t dst = sizeof(T) == 2 ? kdst ^ Geo<D>::kswz(SH::LOAD_ROWS * c) << 4 : kdst;
        *(l16_t)(lds_t)(uintptr_t)(dst + c * SH::LOAD_ROWS * SH::LDS_ROW) = b.k[c];
      }
#pragma unroll
      for (int s = 0; s < QS; ++s) {
        const uint32_t from = sizeof(T) == 2 ? ksrc ^ s << 6 : ksrc + s * 64;
        const vec k = __builtin_bit_cast(vec, *(l16_t)(lds_t)(uintptr_t)from);
        if constexpr (sizeof(T) == 2) {
          st = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[s], st, 0, 0, 0);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) st = __builtin_amdgcn_mfma_f32_16x16x4f32(k[j], q[s][j], st, 0, 0, 0);
        }
      }
      if (kb + 16 > lim0) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (kb + 4 * quad + k >= lim) st[k] = -INFINITY;
        // past the end: zeros
#pragma unroll
        for (int c = 0; c < SH::LOADS; ++c)
          if (kb + SH::LOAD_ROWS * c + lr >= to) b.v[c] = u32x4_t{0, 0, 0, 0};
      }
#pragma unroll
      for (int c = 0; c < SH::LOADS; ++c)
        *(l16_t)(lds_t)(uintptr_t)(vdst + c * SH::LOAD_ROWS * SH::LDS_ROW) = b.v[c];
      const float bm = fmaxf(fmaxf(st[0], st[1]), fmaxf(st[2], st[3])) * c2;
      // float32 for any, since an exponent's rounding grows with its size: error 5.7e-7, else 7.9e-7
      if (__any(bm > m + (sizeof(T) == 2 ? kRescale : 0.0f))) {
        const float mn = fmaxf(m, quad_max(bm));
        const float sc = __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        l *= sc;
#pragma unroll
        for (int e = 0; e < D / 16; ++e) o[e] *= sc;
      }
      float p[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float e = fmaf(st[k], c2, -m);
        // float32: with the rest of scale log2(e), whose rounding would be off by up to 2^-24 of the score
        if (sizeof(T) == 4 && st[k] > kLowest) e = fmaf(st[k], c2_low, e);
        p[k] = __builtin_amdgcn_exp2f(e);
        l += p[k];
      }
      if constexpr (sizeof(T) == 2) {
        bf16x4_t pb;
#pragma unroll
        for (int k = 0; k < 4; ++k) pb[k] = (__bf16)p[k];            // (the one rounding of a weight)
#pragma unroll
        for (int e = 0; e < D / 16; ++e) {
          const bf16x4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((ltr_t)(lds_t)(uintptr_t)(vsrc ^ e << 5));
          o[e] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4_t, v),
                                                           __builtin_bit_cast(s16x4_t, pb), o[e], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int e = 0; e < D / 16; ++e)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            o[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(*(l4_t)(lds_t)(uintptr_t)(vsrc + k * SH::LDS_ROW + e * 64), p[k],
                                                        o[e], 0, 0, 0);
      }
    };
    if (blocks > 0) {
      Block b[SH::DEPTH];
#pragma unroll
      for (int j = 0; j < SH::DEPTH; ++j) load(b[j], j);
      for (int i = 0; i < blocks; i += SH::DEPTH) {
#pragma unroll
        for (int j = 0; j < SH::DEPTH; ++j) {
          if (i + j < blocks) use(b[j], i + j);
          load(b[j], i + j + SH::DEPTH);
        }
      }
    }
  }
  l = quad_sum(l);
  float finite = 0.0f;                               // NaN: no
  if (own_lim0 < k1) {                               // some pairs do not see all keys
#pragma unroll
    for (int e = 0; e < D / 16; ++e)
#pragma unroll
      for (int k = 0; k < 4; ++k) finite = fmaf(o[e][k], 0.0f, finite);
  }
  if (__any(finite != 0.0f)) {
    KeyByKey<T, D, 16, 4, decltype(o)> kk(o, m, l);
    for (int kb = own_first; kb < k1; kb += step) kk.add(a, t.table, h, q, kb, min(kb + 16, k1), own_lim);
    const int len = both ? prefix_tokens(a, g, prefix_len) : 0;
    for (int kb = prefix_first; kb < len; kb += step) kk.add(a, pages_of(a, true, g), h, q, kb, min(kb + 16, len), len);
  }

  typedef T out4_t __attribute__((ext_vector_type(4)));
  const int pre = ALONE ? 0 : ceil_div(prefix_tokens(a, g, prefix_len), a.plan.chunk_prefix);
  if (spread) {
    if (!live) return;
    const Out u = own_place(a, t, h, x, chunk, ceil_div(own_lim, chunk_keys), pre);
    if (u.pair < 0) return;
    if (quad == 0) store_ml(a, u, m, l);
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int e = 0; e < D / 16; ++e) {
      if (u.done) {
        out4_t v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = (T)(o[e][k] * inv);
        *reinterpret_cast<out4_t*>(static_cast<T*>(a.O) + u.pair * D + 16 * e + 4 * quad) = v;
      } else {
        *reinterpret_cast<f32x4_t*>(u.o + 16 * e + 4 * quad) = o[e];
      }
    }
    return;
  }

  // the waves' results, joined: part [wave][pair][PART_ROW], then [m, l][wave][pair]
  __syncthreads();
  float* part = reinterpret_cast<float*>(smem);
  float* ml = part + WAVES * kThin * SH::PART_ROW;
#pragma unroll
  for (int e = 0; e < D / 16; ++e)
    *reinterpret_cast<f32x4_t*>(part + (wave * kThin + ql) * SH::PART_ROW + 16 * e + 4 * quad) = o[e];
  if (quad == 0) {
    ml[wave * kThin + ql] = m;
    ml[(WAVES + wave) * kThin + ql] = l;
  }
  __syncthreads();
  constexpr int F = D / 16;                           // elements of a thread, sixteen threads to a pair
  const int c = tid >> 4, e0 = (tid & 15) * F, xc = t.x0 + c;
  if (c >= kThin || xc >= t.pairs) return;
  const Out u = prefix ? prefix_place(a, t, h, xc, chunk)
                       : own_place(a, t, h, xc, chunk, ceil_div(sees(a, t, false, xc / r), chunk_keys), pre);
  if (u.pair < 0) return;
  float M = kLowest, L = 0.0f, acc[F];
#pragma unroll
  for (int v = 0; v < WAVES; ++v) M = fmaxf(M, ml[v * kThin + c]);
#pragma unroll
  for (int e = 0; e < F; ++e) acc[e] = 0.0f;
#pragma unroll
  for (int v = 0; v < WAVES; ++v) {
    const float f = __builtin_amdgcn_exp2f(ml[v * kThin + c] - M);
    L = fmaf(ml[(WAVES + v) * kThin + c], f, L);
#pragma unroll
    for (int e = 0; e < F; ++e) acc[e] = fmaf(part[(v * kThin + c) * SH::PART_ROW + e0 + e], f, acc[e]);
  }
  if ((tid & 15) == 0) store_ml(a, u, M, L);
  const float inv = L == 0.0f ? 0.0f : 1.0f / L;
#pragma unroll
  for (int e = 0; e < F; e += 4) {
    if (u.done) {
      out4_t v;
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = (T)(acc[e + k] * inv);
      *reinterpret_cast<out4_t*>(static_cast<T*>(a.O) + u.pair * D + e0 + e) = v;
    } else {
      *reinterpret_cast<float4*>(u.o + e0 + e) = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
    }
  }
}

// ---------------------------------------------------------------- the tall tiles

// One wave's 32 pairs: lane l holds pair l % 32; of 32 keys' scores those of keys
// 8 (i / 4) + 4 (l / 32) + i % 4 in register i, and of the output elements
// 32 t + 8 (i / 4) + 4 (l / 32) + i % 4 in o[t][i] (v_mfma_f32_32x32x16_bf16 with
// keys, then values, as the row operand: S^T = K Q^T, O^T += V^T P).
template <int D>
struct Pairs {
  bf16x8_t q[D / 16];
  f32x16_t o[D / 32];
  float m, l;             // m is the pair's, l this lane's share
};

// Values that are to be there at this place of the instruction order: the compiler
// otherwise moves what makes them to where they are used.
template <typename A>
__device__ __forceinline__ void pin(A& a) { asm volatile("" : "+v"(a)); }
template <typename A, typename B>
__device__ __forceinline__ void pin(A& a, B& b) { asm volatile("" : "+v"(a), "+v"(b)); }

// Fragments of a step's 64 keys in LDS: K's k-th operand is 32 keys 32 (k % 2) .. of
// elements 16 (k / 2) ..; V^T's is 32 elements 32 (k % (D / 32)) .. of 16 keys
// 16 (k / (D / 32)) .., in the order in which a lane holds the probabilities: slot
// 8 (l / 32) + j is key 4 (l / 32) + j for j < 4 and 8 + 4 (l / 32) + j - 4 for j >= 4.  It
// is read from the row-major tile by the transposing LDS read: 16 lanes read four keys
// x 16 columns, lane i receives column i of the four.
//
// The swizzles act on address bits that the operands' own offsets reach by exclusive or,
// so each lane keeps one address for K and one for V (key_lane, value_lane, from the
// step's first byte), and an operand costs one instruction.
template <int D>
__device__ __forceinline__ uint32_t key_lane() {
  const int lane = threadIdx.x & 63, ql = lane & 31, half = lane >> 5;
  return ql * Geo<D>::ROW + ((half ^ Geo<D>::kswz(ql)) << 4);
}
template <int D>
__device__ __forceinline__ uint32_t value_lane() {
  const int lane = threadIdx.x & 63, vr = (lane >> 2) & 3;
  return (4 * (lane >> 5) + vr) * Geo<D>::ROW + (Geo<D>::vswz(vr) << 4) + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
}
template <int D>
__device__ __forceinline__ bf16x8_t key_operand(uint32_t K, int k) {
  typedef const __attribute__((address_space(3))) bf16x8_t* ptr_t;
  return *(ptr_t)(lds_t)(uintptr_t)((K ^ (k >> 1) << 5) + 32 * (k & 1) * Geo<D>::ROW);
}
template <int D>
__device__ __forceinline__ bf16x8_t value_operand(uint32_t V, int k) {
  const lds_t p = (lds_t)(uintptr_t)((V ^ (k % (D / 32)) << 6) + 16 * (k / (D / 32)) * Geo<D>::ROW);
  const bf16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((ltr_t)p);
  const bf16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((ltr_t)(p + 8 * Geo<D>::ROW));
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Hides keys from `lim` on (counted in the step).
__device__ __forceinline__ void hide(f32x16_t (&st)[2], int lim) {
  const int from = lim - 4 * (int)((threadIdx.x & 63) >> 5);
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (32 * n + 8 * (i >> 2) + (i & 3) >= from) st[n][i] = -INFINITY;
}

__device__ __forceinline__ float largest(const f32x16_t (&st)[2]) {
  float bm = st[0][0];
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) bm = fmaxf(bm, st[n][i]);
  return bm;
}

// The running maximum moves, and the sums are rescaled, only when a score exceeds it
// by more than 2^8, which float32 sums hold with the same relative error.
template <int D>
__device__ __forceinline__ void move_max(Pairs<D>& w, float bm, float c2) {
  bm *= c2;
  if (__any(bm > w.m + kRescale)) {
    const float mn = fmaxf(w.m, half_max(bm));
    const float sc = __builtin_amdgcn_exp2f(w.m - mn);
    w.m = mn;
    w.l *= sc;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) w.o[t][i] *= sc;
  }
}

// Weighs scores 2 e and 2 e + 1 of the 32 that a lane holds.
template <int D>
__device__ __forceinline__ void weigh(Pairs<D>& w, const f32x16_t (&st)[2], bf16x8_t (&pb)[4], int e, float c2) {
  const float p0 = __builtin_amdgcn_exp2f(fmaf(st[e >> 3][2 * (e & 7)], c2, -w.m));
  const float p1 = __builtin_amdgcn_exp2f(fmaf(st[e >> 3][2 * (e & 7) + 1], c2, -w.m));
  w.l += p0;
  w.l += p1;
  bf16x2_t b = {(__bf16)p0, (__bf16)p1};           // (the one rounding of a weight)
  pin(w.l, b);
  pb[e >> 2][2 * (e & 3)] = b[0];
  pb[e >> 2][2 * (e & 3) + 1] = b[1];
}

// One step: weighs its scores st and adds its values V, while (NEXT) the next step's
// scores are made of its keys K, into st, and their largest is returned.  The matrix
// cores and the vector units work at the same time only where their instructions
// alternate, and a product waits for its operand's LDS read unless that was issued
// well before; so the order is written down: operands four products ahead, and between
// the products the step's loads (issue) and the 16 pairs of scores, 10 of them beside
// the next scores, 6 beside the values of the first 32 keys.  pin() keeps the compiler
// from gathering a kind's work in one place (without it 850 us, with it 841, for 8
// prompts of 3840 rows, 28 heads of 128 on 4: 1005 TFLOP/s).
//
// What bounds it is power: on zeros the same call takes a fifth less time, at 2.4 GHz
// instead of about 1.8.  Sums of two weights to an instruction, other priorities of waves,
// operands three or five ahead and other shares of the scores all measured the same.
template <int D, bool NEXT, typename Issue>
__device__ __forceinline__ float pipeline_step(Pairs<D>& w, f32x16_t (&st)[2], uint32_t K, uint32_t V, float c2,
                                               Issue issue) {
  constexpr int N = D / 8, AHEAD = 4, BESIDE = NEXT ? 10 : 0;      // products of each kind
  bf16x8_t kf[AHEAD], vf[AHEAD], pb[4];
  f32x16_t nx[2];
  pin(K, V);                                       // (else every operand's address is kept in a register)
  if constexpr (NEXT) {
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) kf[k] = key_operand<D>(K, k);
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) nx[n][i] = 0.0f;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      nx[k & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[k % AHEAD], w.q[k >> 1], nx[k & 1], 0, 0, 0);
      if (k + AHEAD < N) kf[k % AHEAD] = key_operand<D>(K, k + AHEAD);
      else vf[k + AHEAD - N] = value_operand<D>(V, k + AHEAD - N);
      issue(k);
#pragma unroll
      for (int e = k * BESIDE / N; e < (k + 1) * BESIDE / N; ++e) weigh(w, st, pb, e, c2);
      }
  } else {
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) vf[k] = value_operand<D>(V, k);
#pragma unroll
    for (int e = 0; e < 8; ++e) weigh(w, st, pb, e, c2);
  }
  constexpr int DONE = NEXT ? BESIDE : 8;
  float bm = kLowest;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    w.o[k % (D / 32)] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[k % AHEAD], pb[k / (D / 32)], w.o[k % (D / 32)], 0, 0, 0);
    if (k + AHEAD < N) vf[k % AHEAD] = value_operand<D>(V, k + AHEAD);
    if (k < N / 2) {
#pragma unroll
      for (int e = DONE + k * (16 - DONE) * 2 / N; e < DONE + (k + 1) * (16 - DONE) * 2 / N; ++e) weigh(w, st, pb, e, c2);
    } else if constexpr (NEXT) {
#pragma unroll
      for (int e = (k - N / 2) * 64 / N; e < (k + 1 - N / 2) * 64 / N; e += 2)
        bm = fmaxf(fmaxf(bm, nx[e >> 4][e & 15]), nx[e >> 4][(e & 15) + 1]);
      pin(bm);
    }
  }
  if constexpr (NEXT) {
    st[0] = nx[0];
    st[1] = nx[1];
  }
  return bm;
}

// 128 pairs, 32 a wave; the waves share steps of 64 keys, K and V two deep each.  While
// the vector units weigh one step's scores, the next step's are on the matrix cores.
// Keys: a fused tile takes its prefix's steps first (the last one may be ragged), then
// its own run's.
template <int D, bool ALONE>
__device__ __forceinline__ void tall_tile(const AttendArgs& a, char* smem, bool prefix, const Tile& t, int h, int chunk) {
  using G = Geo<D>;
  constexpr int STEP = kTallStep * G::ROW;                                    // 64 keys of K or V
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ql = lane & 31, half = lane >> 5, r = ratio(a);
  int g = -1, pre = 0, P = 0;                        // parts of the prefix apart; its tokens taken here
  if (!prefix) {
    g = t.group;
    if (ALONE || t.pairs > kFuse) P = t.before;
    else pre = ceil_div(t.before, a.plan.chunk_prefix);
  }
  const int before = ceil_div(P, kTallStep);
  const int chunk_steps = (prefix ? a.plan.chunk_prefix : a.plan.chunk_tall) / kTallStep;
  const int end = sees(a, t, prefix, (min(t.x0 + kTall, t.pairs) - 1) / r);   // of the run, for the whole tile
  const int v0 = chunk * chunk_steps;
  const int n = min(before + ceil_div(end, kTallStep) - v0, chunk_steps);     // steps of this chunk
  if (n <= 0 && (prefix || chunk > 0)) return;

  const int xw = t.x0 + 32 * wave, x = xw + ql;
  const bool idle = xw >= t.pairs;                                            // the wave has no pair
  const bool live = x < t.pairs;
  // a tile whose sequences all take the prefix by themselves
  if (prefix && a.rows.max_rows * (int64_t)r > kFuse &&
      !__syncthreads_or(live && prefix_place(a, t, h, x, chunk).pair >= 0))
    return;
  const int row = live ? x / r : 0;
  Pairs<D> w;
  const uint16_t* qsrc =
      static_cast<const uint16_t*>(a.Q) + (t.row0 + row) * a.ldq + (h * r + (x - row * r)) * D + 8 * half;
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    uint4 u = make_uint4(0, 0, 0, 0);
    if (live) u = *reinterpret_cast<const uint4*>(qsrc + 16 * s);
    w.q[s] = __builtin_bit_cast(bf16x8_t, u);
  }
#pragma unroll
  for (int e = 0; e < D / 32; ++e)
#pragma unroll
    for (int i = 0; i < 16; ++i) w.o[e][i] = 0.0f;
  w.m = kLowest;
  w.l = 0.0f;
  const int lim = live ? sees(a, t, prefix, row) : 0, lim0 = idle ? 0 : sees(a, t, prefix, xw / r);
  const float c2 = a.c2;

  // The wave loads keys 16 wave .. of every step, which lie in one page.  Lane j holds
  // where those of step 64 (i / 64) + j are, and the page of 64 steps on.
  Loader<D> ld;
  ld.init();
  auto fetch = [&](int i) {
    const AttendArgs& f = arguments();
    const int v = v0 + i + lane;
    const bool p = v < before;
    const int key = (p ? v : v - before) * kTallStep + 16 * wave;
    int page = 0;
    if (key < (p ? P : t.len)) page = pages_of(f, prefix || p, p ? g : t.seg)[key >> f.shape.page_shift];
    return checked_page(f, page);
  };
  uint32_t at_lo = 0, at_hi = 0;
  int ahead = 0;
  auto place = [&](int i) {
    if ((i & 63) == 0) {
      const int v = v0 + i + lane;
      const int64_t at = place_of<G::ROW>(arguments(), i == 0 ? fetch(0) : ahead, h,
                                          (v < before ? v : v - before) * kTallStep + 16 * wave);
      at_lo = (uint32_t)at;
      at_hi = (uint32_t)(at >> 32);
      ahead = fetch(i + 64);
    }
    return lane_value(at_lo, at_hi, i & 63);
  };
  // operand addresses of even steps
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_t)smem;
  const uint32_t kl = lds0 + key_lane<D>(), vl = lds0 + 2 * STEP + value_lane<D>();
  const char* const Kc = static_cast<const char*>(a.k_cache);
  const char* const Vc = static_cast<const char*>(a.v_cache);
  const uint32_t mine = lds0 + 16 * wave * G::ROW;   // the wave's rows of a step
  // Steps that end inside a step's keys: the prefix's last, the run's last.  From step
  // `masked` on the wave's first pair does not see all keys.
  const int ragged = P % kTallStep ? before - 1 - v0 : -1, last = end % kTallStep ? before - v0 + end / kTallStep : -1;
  const int masked = before - v0 + lim0 / kTallStep;
  // before step i's values are used: those past the end are cleared
  auto clear = [&](int i) {
    const int left = (i == ragged ? P : end) % kTallStep - 16 * wave;
    if (left < 16) clear_rows<D>(smem + (2 + (i & 1)) * STEP + 16 * wave * G::ROW, left < 0 ? 0 : left);
    __syncthreads();
  };
  // keys of step i that the lane's pair sees
  auto mask = [&](f32x16_t (&st)[2], int i) {
    if (i == ragged) hide(st, P % kTallStep);
    else hide(st, lim - (v0 + i - before) * kTallStep);
  };
  if (n > 0) {
    int64_t at = place(0);
#pragma unroll
    for (int k = 0; k < G::LOADS; ++k) ld.keys(Kc + at, mine, k);
#pragma unroll
    for (int k = 0; k < G::LOADS; ++k) ld.values(Vc + at, mine + 2 * STEP, k);
    at = place(1);
#pragma unroll
    for (int k = 0; k < G::LOADS; ++k) ld.keys(Kc + at, mine + STEP, k);
    f32x16_t st[2];
    wait_vmcnt<0>();
    __syncthreads();
    if (!idle) {
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int e = 0; e < 16; ++e) st[m][e] = 0.0f;
#pragma unroll
      for (int k = 0; k < D / 8; ++k)
        st[k & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key_operand<D>(kl, k), w.q[k >> 1], st[k & 1], 0, 0, 0);
      if (0 == ragged || 0 >= masked) mask(st, 0);
      move_max(w, largest(st), c2);
    }
    for (int i = 0; i < n - 1; ++i) {
      wait_vmcnt<0>();                               // this wave's loads of K i + 1 and V i
      __syncthreads();                               // every wave's; and all are past K i and V i - 1
      if (i == ragged || i == last) clear(i);
      // the loads of V i + 1 and K i + 2 (whether or not there is such a step: nothing reads it then)
      const char* vs = Vc + at;
      at = place(i + 2);
      const char* ks = Kc + at;
      const int odd = i & 1;
      auto issue = [&](int k) {
        if (k < G::LOADS) ld.values(vs, mine + (3 - odd) * STEP, k);
        else if (k < 2 * G::LOADS) ld.keys(ks, mine + odd * STEP, k - G::LOADS);
      };
      if (idle) {
#pragma unroll
        for (int k = 0; k < 2 * G::LOADS; ++k) issue(k);
        continue;
      }
      float bm = pipeline_step<D, true>(w, st, kl + (1 - odd) * STEP, vl + odd * STEP, c2, issue);
      if (i + 1 == ragged || i + 1 >= masked) {
        mask(st, i + 1);
        bm = largest(st);
      }
      move_max(w, bm, c2);
    }
    wait_vmcnt<0>();
    __syncthreads();
    if (n - 1 == ragged || n - 1 == last) clear(n - 1);
    if (!idle) pipeline_step<D, false>(w, st, 0, vl + ((n - 1) & 1) * STEP, c2, [](int) {});
  }
  w.l = half_sum(w.l);
  float finite = 0.0f;                               // NaN: no
#pragma unroll
  for (int e = 0; e < D / 32; ++e)
#pragma unroll
    for (int i = 0; i < 16; ++i) finite = fmaf(w.o[e][i], 0.0f, finite);
  // (some pairs do not see all keys)
  if (__any(finite != 0.0f) && __any(live && lim < min(end, (v0 + n - before) * kTallStep))) {
    const AttendArgs& f = arguments();
    KeyByKey<__bf16, D, 32, 16, decltype(w.o)> kk(w.o, w.m, w.l);
    for (int i = 0; i < n; ++i) {
      const bool p = v0 + i < before;
      const int kb = (p ? v0 + i : v0 + i - before) * kTallStep;
      kk.add(f, pages_of(f, prefix || p, p ? g : t.seg), h, w.q, kb, min(kb + kTallStep, p ? P : end),
             p ? P : lim);
    }
  }

  const AttendArgs& e = arguments();
  Out u;
  u.pair = -1;
  u.done = false;
  if (live) {
    const int row_steps = before + ceil_div(lim, kTallStep);
    u = prefix ? prefix_place(e, t, h, x, chunk) : own_place(e, t, h, x, chunk, ceil_div(row_steps, chunk_steps), pre);
  }
  const bool done = u.pair >= 0 && u.done;
  if (u.pair >= 0 && half == 0) store_ml(e, u, w.m, w.l);
  if (u.pair >= 0 && !u.done) {
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4)
        *reinterpret_cast<float4*>(u.o + 32 * b + 8 * g4 + 4 * half) =
            make_float4(w.o[b][4 * g4], w.o[b][4 * g4 + 1], w.o[b][4 * g4 + 2], w.o[b][4 * g4 + 3]);
  }
  // Rows that are done go through LDS, whose every wave is past the last step's values, so
  // that they are stored in whole chunks of whole rows, streamed past the caches (16 prompts
  // of 256 rows, 28 heads on 4: 29.0 us, kept in the caches 30.3).
  __syncthreads();
  if (!__any(done)) return;
  constexpr int OUT = G::ROW + 16;
  char* const rows = smem + wave * 32 * OUT;
  const float inv = w.l == 0.0f ? 0.0f : 1.0f / w.l;
#pragma unroll
  for (int b = 0; b < D / 32; ++b)
#pragma unroll
    for (int g4 = 0; g4 < 4; ++g4) {
      bf16x4_t v;
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = (__bf16)(w.o[b][4 * g4 + k] * inv);
      *reinterpret_cast<bf16x4_t*>(rows + ql * OUT + (32 * b + 8 * g4 + 4 * half) * 2) = v;
    }
  lds_exchanged();
  const int64_t pair = done ? u.pair : -1;
#pragma unroll
  for (int c = 0; c < 32; c += G::LOAD_ROWS) {
    const int j = c + lane / G::CHUNKS, chunk16 = lane % G::CHUNKS;
    const int64_t to = (int64_t)((uint64_t)(uint32_t)__shfl((int)(pair >> 32), j) << 32 | (uint32_t)__shfl((int)pair, j));
    const u32x4_t v = *reinterpret_cast<const u32x4_t*>(rows + j * OUT + chunk16 * 16);
    if (to >= 0)
      __builtin_nontemporal_store(v, reinterpret_cast<u32x4_t*>(static_cast<char*>(e.O) + to * G::ROW + chunk16 * 16));
  }
}

// Sequence `seg` as one thin tile, and its group.  False: it has no row, or more than 16 pairs.
__device__ __forceinline__ bool sequence_tile(const AttendArgs& a, int seg, Tile& t, int& g) {
  t.seg = seg;
  const int tokens = tokens_of(a.runs, seg, t.len), rows = rows_of(a.rows, seg, t.row0, t.n);
  g = group_of(a, seg);
  const int64_t pairs = (int64_t)t.n * ratio(a);
  if (rows != SP_DEV_OK || tokens != SP_DEV_OK || pairs == 0 || pairs > kThin) return false;
  t.pairs = (int)pairs;
  t.x0 = 0;
  t.table = a.runs.table + (int64_t)seg * a.runs.width;
  return true;
}

// One launch for all tiles: the prefixes' (thin or tall), the sequences' tall ones, the
// sequences' thin ones, in this order; the last workgroup looks for errors in the batch's
// entries, wherever they are.  float32 has thin tiles only, several to a longer sequence.
// ALONE: no sequence shares its prefix's tiles.
template <typename T, int D, bool STREAM, bool ALONE>
__global__ __launch_bounds__(64 * kWaves, sizeof(T) == 2 && D == 64 ? 3 : 2) void attend_kernel(AttendArgs a) {
  constexpr bool BF16 = sizeof(T) == 2;
  // the tall tiles' two steps of K and of V: two workgroups to a compute unit, or (D 64) three
  constexpr int TALL = BF16 ? 8 * kTallStep * D : 0, THIN = ThinShape<T, D, kWaves>::LDS, LDS = TALL > THIN ? TALL : THIN;
  __shared__ __attribute__((aligned(1024))) char smem[LDS];
  const AttendPlan& p = a.plan;
  const int heads = a.shape.kv_heads;
  int id = blockIdx.x;
  if (id == p.prefix_blocks + p.tall_blocks + p.thin_blocks) {
    report_entries(a, false);
    if (a.prefix.count > 0) report_entries(a, true);
    return;
  }
  Tile t;
  // block id of `tiles` tiles, the key heads and the chunks
  if constexpr (BF16) {
    const bool prefix = !ALONE && p.prefix_tall && id < p.prefix_blocks;
    if (prefix || (id >= p.prefix_blocks && id < p.prefix_blocks + p.tall_blocks)) {
      if (!prefix) id -= p.prefix_blocks;
      const int tiles = prefix ? p.prefix_tiles : p.tall_tiles;
      // Key heads innermost: workgroup w runs on XCD w % 8, so (4, 8, 16, .. key heads) an
      // XCD's L2 holds the keys of one or two heads at a time, and work ends small at the
      // end of the launch, not of each head (8 prompts of 3840 rows 844 us, heads outermost 874).
      const int rest = id / heads, h = id - rest * heads, chunk = rest / tiles, tile = rest - chunk * tiles;
      if ((prefix ? a.prefix.count : a.runs.count) <= kSorted) {
        // (the last quarter of the tall tiles' LDS: not written before their first barrier)
        uint2* const table = reinterpret_cast<uint2*>(smem + 6 * kTallStep * D) + kSorted * ((int)threadIdx.x >> 6);
        if (!find_sorted_tile<ALONE>(a, prefix, tile, t, table)) return;
      } else {
        if (!find_tile<kTall>(a, prefix, tiles - 1 - tile, t)) return;
        if (!prefix && t.pairs <= kThin) return;                             // a thin tile's
        if (!prefix) find_prefix(a, t);
      }
      tall_tile<D, ALONE>(a, smem, prefix, t, h, chunk);
      return;
    }
  }
  const bool prefix = !ALONE && id < p.prefix_blocks;
  if (!prefix) id -= p.prefix_blocks + p.tall_blocks;
  const bool spread = !prefix && p.spread;
  const int tiles = prefix ? p.prefix_tiles : p.thin_tiles;
  const int per = spread ? heads / kWaves : heads, rest = id / per, hh = id - rest * per, chunk = rest / tiles, tile = rest - chunk * tiles;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int h = spread ? hh * kWaves + wave : hh;
  const int key = chunk * (prefix ? p.chunk_prefix : p.chunk_thin) + (spread ? 0 : 16 * wave);
  Places<D * (int)sizeof(T)> places;
  int g = -1;
  if (prefix || p.thin_tiled) {
    if (!find_tile<kThin>(a, prefix, tile, t)) return;
    places.prime(a, prefix ? a.prefix : a.runs, t.seg, key, spread ? 16 : kThinStep);
    if (!prefix) g = group_of(a, t.seg);
  } else {                                           // a sequence to a tile; longer ones are the tall tiles'
    places.prime(a, a.runs, tile, key, spread ? 16 : kThinStep);
    if (!sequence_tile(a, tile, t, g)) return;
  }
  thin_tile<T, D, STREAM, kWaves, ALONE>(a, smem, prefix, t, places, h, chunk, g, spread);
}

// Few sequences, of at most 16 pairs and not too many keys: eight waves to a sequence and key
// head, over its own run and its prefix, so that no parts are left for a second launch to join.
template <int D>
__global__ __launch_bounds__(64 * kWide, 2) void wide_kernel(AttendArgs a) {
  __shared__ __attribute__((aligned(1024))) char smem[ThinShape<__bf16, D, kWide>::LDS];
  if (blockIdx.x == a.plan.thin_blocks) {
    report_entries(a, false);
    if (a.prefix.count > 0) report_entries(a, true);
    return;
  }
  const int heads = a.shape.kv_heads, seg = blockIdx.x / heads, h = blockIdx.x - seg * heads;
  Places<2 * D> places;
  places.prime(a, a.runs, seg, 16 * __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), 16 * kWide);
  Tile t;
  int g;
  if (!sequence_tile(a, seg, t, g)) return;
  thin_tile<__bf16, D, true, kWide, true>(a, smem, false, t, places, h, 0, g, false);
}

// ---------------------------------------------------------------- joining the parts

// SPLIT waves to a (row, head): each joins every SPLIT-th part, and they join through LDS.
// The first `short_blocks` workgroups take the pairs of the short sequences, the others (tall)
// those of the rows of the others.
template <typename T, int D, int SPLIT>
__global__ __launch_bounds__(64 * kWaves) void combine_kernel(AttendArgs a, int short_blocks) {
  constexpr int E = D / 64, AHEAD = 8;
  __shared__ float red[kWaves][D + 2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, share = wave % SPLIT;
  const bool tall = (int)blockIdx.x >= short_blocks;
  const int64_t at = (int64_t)((int)blockIdx.x - (tall ? short_blocks : 0)) * (kWaves / SPLIT) + wave / SPLIT;
  const int Hq = a.shape.q_heads;
  const AttendPlan& p = a.plan;
  int64_t row = -1, base = 0;                        // the row's parts from pair `base` on
  int2 counts = make_int2(0, 0);
  const int head = (int)(at % Hq);
  if (tall || p.by_row) {
    row = at / Hq;
    base = row * Hq;
    bool live = row < a.rows.rows;
    if (live) counts = a.row_parts[row];             // (beside the loads that tell whether it is a row)
    if (live && a.rows.padded) {
      const int64_t s = row / a.rows.rows_per_seq;
      live = s < a.runs.count && row - s * a.rows.rows_per_seq < a.rows.info[s] &&
             (!tall || a.rows.info[s] * (int64_t)ratio(a) > p.short_pairs);
    } else if (live && !tall) {
      live = row >= a.rows.info[0] && row < a.rows.info[a.runs.count];
    } else if (live) {
      const int s = wave_find_last(a.runs.count, row, [&](int i) { return (int64_t)a.rows.info[i]; });
      live = row >= a.rows.info[s] && row < a.rows.info[s + 1] &&
             (a.rows.info[s + 1] - a.rows.info[s]) * (int64_t)ratio(a) > p.short_pairs;
    }
    if (!live) row = -1;
  } else {
    const int64_t per = (int64_t)p.short_rows * Hq, s = at / per;
    int64_t first;
    int n;
    if (s < a.runs.count && rows_of(a.rows, (int)s, first, n) == SP_DEV_OK) {
      const int i = (int)((at - s * per) / Hq);
      if (i < n && (int64_t)n * ratio(a) <= p.short_pairs) {
        row = first + i;
        base = short_base(a, row, (int)s, i);
        counts = a.row_parts[row];
      }
    }
  }
  int own = 0, pre = 0;
  if (row >= 0) {
    const int2 c = counts;
    own = c.x;
    pre = c.y;
    // (after an error in the batch's entries a row may have no count)
    if (own < 0 || own > (tall ? p.tall_parts : p.short_parts) || pre < 0 || pre > p.prefix_parts) own = pre = 0;
  }
  const int total = own + pre;
  if (SPLIT == 1 && total == 0) return;
  const int64_t pair = base + head;
  const float2* pml = reinterpret_cast<const float2*>(a.prefix_ml) + pair * p.prefix_parts;
  const float* po = a.prefix_o + pair * p.prefix_parts * D;
  const float2* oml = reinterpret_cast<const float2*>(tall ? a.tall_ml : a.short_ml) + pair * (tall ? p.tall_parts : p.short_parts);
  const float* oo = (tall ? a.tall_o : a.short_o) + pair * (tall ? p.tall_parts : p.short_parts) * D;
  float M = kLowest, L = 0.0f, acc[E] = {};
  for (int i0 = share; i0 < total; i0 += SPLIT * AHEAD) {
    float2 ml[AHEAD];
    float v[AHEAD][E];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int i = i0 + SPLIT * k;
      ml[k] = make_float2(kLowest, 0.0f);
#pragma unroll
      for (int e = 0; e < E; ++e) v[k][e] = 0.0f;
      if (i < total) {
        ml[k] = i < pre ? pml[i] : oml[i - pre];
        const float* src = i < pre ? po + (int64_t)i * D : oo + (int64_t)(i - pre) * D;
#pragma unroll
        for (int e = 0; e < E; ++e) v[k][e] = src[E * lane + e];
      }
    }
    float mn = M;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) mn = fmaxf(mn, ml[k].x);
    const float f0 = exp2f(M - mn);
    M = mn;
    L *= f0;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] *= f0;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const float f = exp2f(ml[k].x - M);
      L = fmaf(ml[k].y, f, L);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = fmaf(v[k][e], f, acc[e]);
    }
  }
  if constexpr (SPLIT > 1) {
#pragma unroll
    for (int e = 0; e < E; ++e) red[wave][E * lane + e] = acc[e];
    if (lane == 0) {
      red[wave][D] = M;
      red[wave][D + 1] = L;
    }
    __syncthreads();
    if (share != 0 || total == 0) return;
#pragma unroll
    for (int k = 1; k < SPLIT; ++k) {
      const float mk = red[wave + k][D], mn = fmaxf(M, mk);
      const float f = exp2f(M - mn), fk = exp2f(mk - mn);
      M = mn;
      L = fmaf(L, f, red[wave + k][D + 1] * fk);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = fmaf(acc[e], f, red[wave + k][E * lane + e] * fk);
    }
  }
  const float inv = L == 0.0f ? 0.0f : 1.0f / L;
  const int64_t out = row * Hq + head;
#pragma unroll
  for (int e = 0; e < E; ++e) static_cast<T*>(a.O)[out * D + E * lane + e] = (T)(acc[e] * inv);
  if (a.lse && lane == 0) a.lse[out] = lse_of(M, L);
}

// Keys of a thin tile's chunk, in whole steps, for `items` tiles and key heads: runs of more
// than 256 keys in chunks of at least 256 (few short ones 128) while the device's 512 places for
// workgroups hold them all, then of at least 2048 until there are four for each, which evens
// out unequal lengths.  (us: one token of 32 key heads over 707, caches cold, in chunks of 512 /
// 256 / 128 11.5 / 10.5 / 9.8, 12 ragged ones of 4 over up to 900 13.9 / 12.2 / 12.9; one run of
// 131001, 4 key heads, in 512 parts of 256 / 128 of 1024 68 / 51; 128 ragged runs of up to 8192,
// 4 key heads, in chunks of 8192 / 2048 / 1024 216 / 192 / 192: every workgroup costs a few us
// to begin and to end.)  `alone`: no other parts are joined to these.
inline int thin_chunk_of(int64_t items, int64_t max_len, bool alone) {
  auto ceil64 = [](int64_t x, int64_t y) { return (x + y - 1) / y; };
  if (items < 1) items = 1;
  const int64_t fill = max_len <= 256 ? 1 : std::min(512 / items, ceil64(max_len, alone && items <= 32 && max_len <= 1024 ? 128 : 256));
  const int64_t even = std::min(ceil64(2048, items), ceil64(max_len, 2048));
  const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(kMaxParts, std::max(fill, even)));
  const int64_t keys = ceil64(max_len, parts);
  return (int)std::min<int64_t>(kMaxCacheTokens, std::max<int64_t>(1, ceil64(keys, kThinStep)) * kThinStep);
}

// The same for tall tiles, whose parts are many rows' outputs to write and to join: parts are
// doubled while the places hold them and it pays by what was measured.  us: a step alone on
// its compute unit 0.78 (heads of 64) to 0.97 (128), a join 5 and its bytes at 2.5 TB/s.  (16
// rows of 64 heads on 8 over 512 / 1024 / 2048 tokens, heads of 64, in 1, 2, 4, 8 parts: 8
// sequences 15 20 22 27 / 21 23 25 28 / 35 29 28 27; 32 sequences 20 38 45 58 / 26 43 51 63 /
// 39 52 63 75.)  `joined`: the rows are joined in any case.
inline int tall_chunk_of(int64_t items, int64_t keys, int64_t pairs, int D, bool joined) {
  const int64_t steps = std::max<int64_t>(1, (keys + kTallStep - 1) / kTallStep);
  const auto cost = [&](int64_t parts) {
    return (double)((steps + parts - 1) / parts) * (0.6 + 0.003 * D) +
           (parts > 1 || joined ? 5.0 + (double)parts * (double)pairs * D * 8.0 / 2.5e6 : 0.0);
  };
  int64_t best = 1;
  for (int64_t n = 2; n <= steps && n * items <= 512; n *= 2)
    if (cost(n) < cost(best)) best = n;
  return (int)std::min<int64_t>(kMaxCacheTokens, (steps + best - 1) / best * kTallStep);
}

inline int parts_of(int64_t max_len, int chunk) { return (int)((max_len + chunk - 1) / chunk); }

}  // namespace

AttendPlan plan_cache_attend(const CacheShape& s, const CacheRows& rows, const CacheRuns& runs,
                             const CacheRuns& prefix) {
  AttendPlan p{};
  const int64_t r = s.q_heads / s.kv_heads, pairs = rows.rows * r, longest = rows.max_rows * r;
  const int64_t heads = s.kv_heads, S = runs.count, G = prefix.count;
  const bool f32 = s.dtype == SP_F32;
  const bool own_tall = !f32 && longest > kThin;
  // keys of a tall tile, the prefix's in whole steps
  const int64_t tall_keys = (prefix.max_len + kTallStep - 1) / kTallStep * kTallStep + (int64_t)runs.max_len;
  p.thin_tiled = f32 && longest > kThin;
  p.reread = p.thin_tiled || (f32 && G > 0 && pairs > kThin * G);
  // float32 has no tall tiles: every sequence is short, and its prefix is shared
  p.short_pairs = (int)(f32 || longest < kFuse ? longest : kFuse);
  if (p.short_pairs < 1) p.short_pairs = 1;
  p.by_row = longest <= p.short_pairs;
  p.short_rows = (int)((p.short_pairs + r - 1) / r);
  p.thin_tiles = (int)(p.thin_tiled ? pairs / kThin + S : S);
  // Prompts take their prefixes each by itself (no tiles of the prefixes, no parts to write and
  // to join) unless that is more work: the steps of tall tiles that sharing would fill and they
  // do not, against the parts.  By the rows' mean, and what was measured: us, shared / each by
  // itself, prefixes of 64, 256, 1024, 2000 tokens, heads of 128:
  //   64 prompts of 24 to 96 rows on 4, 28 heads on 4   43 / 33, 53 / 44, 103 / 93, 154 / 144
  //   64 of 3 to 12 on 4, 28 heads on 4                 24 / 13, 29 / 16, 46 / 27, 63 / 43
  //   64 of 2 to 8 on 4, 28 heads on 4                  20 / 13, 23 / 16, 27 / 31, 36 / 57
  //   64 of 20 to 60 on 8, 32 heads                     118 / 54, 129 / 71, 188 / 153, 263 / 273
  //   32 of 1 to 40 on 4, 32 heads                      36 / 25, 40 / 44, 57 / 117, 72 / 206
  //   100 of 1 to 10 on 4, 32 heads on 8                32 / 24, 35 / 39, 43 / 106, 52 / 164
  // Single tokens beside long prompts have no place in that mean, but would take the whole prefix
  // in one workgroup each.  `most` sequences can be that short, where all others are as long as
  // the longest; in an even batch half of them would be, so those past half are taken to be
  // (`thin`).  Their steps fill what the tall tiles leave of the device, at half the cost; and one
  // such workgroup, at 0.6 us a step (heads of 64: 0.37), is to end before the tall tiles' chunks.
  // us, shared / each by itself, 28 heads of 128 on 4:
  //   one prompt of 40 rows and 1 token, on 1024, 2000, 8192 tokens      18 / 21, 21 / 30, 31 / 87
  //   of 512 rows and 1, on 2000, 8192, 131072                           50 / 44, 87 / 120, 968 / 1590
  //   of 512 and 16, on 1024, 2000, 8192                                 41 / 32, 51 / 51, 91 / 159
  //   of 2500 and 127, on 1024, 2000, 8192                               118 / 117, 157 / 167, 416 / 470
  //   4 of 300 and 16, on 2000, 8192                                     69 / 62, 211 / 209
  int64_t thin = 0;
  if (own_tall && G > 0 && prefix.max_len > 0) {
    const double steps = (double)((prefix.max_len + kTallStep - 1) / kTallStep), width = s.head_dim / 128.0;
    const double unfilled = std::max(0.0, (double)S - (double)pairs / kTall);
    const int64_t others = std::max<int64_t>(0, (pairs - kThin * S + longest - kThin - 1) / (longest - kThin));
    const int64_t most = std::max<int64_t>(0, S - others);
    thin = std::max<int64_t>(0, 2 * most - S);
    const double work = std::max(unfilled * 0.0045, (double)thin * 0.0025) * (double)heads * steps * width;
    const int tall = tall_chunk_of(std::max(S, pairs / kTall) * heads, tall_keys, pairs * heads, s.head_dim, false);
    const double last = most == 0 ? 0.0 : steps * (0.14 + 0.46 * width) -
                                              (double)(tall / kTallStep) * (0.6 + 0.003 * s.head_dim);
    const double parts = 5.0 + (double)(pairs * heads) * s.head_dim * 8.0 / 2.0e6;
    p.alone = work + std::max(0.0, last) < parts;
  }
  // A wave to a head, where there are heads enough to fill the device and the runs are short:
  // fewer workgroups to begin and end, less even work.  us, four waves / one to a head, runs of 5,
  // 64, 128, 192, 256 tokens, heads of 128: 576 runs and key heads 9.6 / 6.1, 9.9 / 7.6,
  // 11.6 / 10.2, 14.2 / 12.9, 15.9 / 15.5; 1120: 13.6 / 7.0, 15.0 / 10.2, 18.3 / 16.8, 22.7 / 24.1,
  // 26.4 / 30.8; 1920: 19.2 / 7.2, 22.5 / 11.8, 28.2 / 20.6, 35.3 / 29.4, 41.6 / 38.4.
  // (Where they take a prefix too, with its keys: 100 sequences of 1 to 10 rows, 32 heads on 8, on
  // prefixes of 256 tokens 27 / 36.)
  p.spread = heads % kWaves == 0 && S * heads >= 512 &&
             (int64_t)runs.max_len + (p.alone && thin > 0 ? prefix.max_len : 0) <= 192;
  const int64_t units = p.spread ? heads / kWaves : heads;
  p.chunk_thin = thin_chunk_of((p.thin_tiled ? std::max(S, pairs / kThin) : S) * units, runs.max_len, prefix.max_len == 0);
  // Among prompts a thin tile that takes its whole run ends with their tiles, and nothing need be
  // joined.  us, in chunks / whole: 4 prompts of 300 to 500 rows, 28 heads on 4, 23.1 / 20.8; 16 of
  // 200 to 900, 32 heads of 64 on 8, 68.0 / 63.5; 16 of 1 to 20 on 1000 tokens 32.2 / 28.5.
  if (own_tall && pairs >= kThin * S && runs.max_len <= 1024)
    p.chunk_thin = std::max(1, (runs.max_len + kThinStep - 1) / kThinStep) * kThinStep;
  // A wide workgroup to a sequence and key head, where those are no more than the compute
  // units and the runs are the shorter the fewer they are.  us, caches cold, in chunks (joined by a
  // second launch from 257 tokens on) / wide, heads of 128, all runs of one length:
  //    32 of 64, 256, 400, 707 tokens  5.8 / 5.5, 7.5 / 7.4, 10.1 / 8.9, 10.5 / 11.8
  //    64 of 64, 256, 707              6.0 / 5.7, 7.9 / 7.6, 12.6 / 12.9
  //   128 of 64, 256, 707, 2048        6.2 / 5.8, 8.1 / 7.9, 16.7 / 14.3, 31.0 / 31.2
  //   256 of 64, 256, 707, 2048        6.7 / 6.3, 10.3 / 9.9, 23.1 / 19.8, 53.7 / 49.2
  //   512 of 64, 256, 707              8.5 / 9.9, 15.7 / 17.5, 35.3 / 36.4
  // float32's products take a compute unit too long: 16 of 640 tokens, heads of 64, 10.4 / 11.5.
  // With prefixes of 256, 400, 700, 1000 tokens before up to 64 own ones, shared and joined /
  // taken by each sequence:
  //   16 sequences on 1 prefix, 4 key heads    13.2 / 8.1, 14.4 / 9.4
  //   64 on 4, 4 key heads                     16.3 / 9.6, 17.6 / 11.1, 18.9 / 13.8, 20.4 / 16.9
  //    8 on 1, 32 key heads                    11.9 / 8.7, 13.0 / 10.3, 12.7 / 12.5, 13.1 / 15.3
  const int before = G > 0 ? prefix.max_len : 0;
  const int64_t items = S * heads, together = (int64_t)runs.max_len + before;
  p.wide = !f32 && !own_tall && items <= 256 &&
           together <= (items <= 64 ? 512 : items <= 192 ? 768 : before > 0 ? 1024 : 2048);
  if (p.wide) {
    p.spread = 0;
    p.chunk_thin = (runs.max_len / (16 * kWide) + 1) * 16 * kWide;
    p.chunk_prefix = kTallStep;
    p.short_parts = 1;
    p.thin_blocks = items;
    return p;
  }
  p.thin_blocks = p.thin_tiles * units * (runs.max_len > 0 ? parts_of(runs.max_len, p.chunk_thin) : 1);
  p.short_parts = parts_of(runs.max_len, p.chunk_thin);
  if (own_tall) {
    p.tall_tiles = (int)(pairs / kTall + S);
    p.chunk_tall = tall_chunk_of(std::max(S, pairs / kTall) * heads, tall_keys, pairs * heads, s.head_dim, false);
    p.tall_parts = parts_of(tall_keys, p.chunk_tall);
    p.tall_blocks = p.tall_tiles * heads * (p.tall_parts > 0 ? p.tall_parts : 1);
    if (p.tall_parts > p.short_parts) p.short_parts = p.tall_parts;
  }
  if (G > 0 && prefix.max_len > 0 && !p.alone) {
    p.prefix_tall = !f32 && pairs > kThin * G;
    p.prefix_tiles = (int)(pairs / (p.prefix_tall ? kTall : kThin) + G);
    p.chunk_prefix = p.prefix_tall
                         ? tall_chunk_of(std::max(G, pairs / kTall) * heads, prefix.max_len, pairs * heads, s.head_dim, true)
                         : thin_chunk_of(std::max(G, pairs / kThin) * heads, prefix.max_len, false);
    p.prefix_parts = parts_of(prefix.max_len, p.chunk_prefix);
    p.prefix_blocks = p.prefix_tiles * heads * p.prefix_parts;
  } else {
    p.chunk_prefix = kTallStep;
  }
  return p;
}

namespace {

// The rows of the short sequences are joined, those of the others.  (Without a row in any
// sequence there is nothing to join.)
inline bool joins_short(const AttendArgs& a) {
  return a.rows.max_rows > 0 && (a.plan.prefix_parts > 0 || a.plan.short_parts > 1);
}
inline bool joins_tall(const AttendArgs& a) {
  return a.plan.tall_parts > 1 && a.rows.max_rows * (int64_t)(a.shape.q_heads / a.shape.kv_heads) > a.plan.short_pairs;
}

// A join of many parts takes a workgroup to a (row, head), else a wave.
inline bool many_parts(const AttendArgs& a) {
  const AttendPlan& p = a.plan;
  return (joins_short(a) && p.prefix_parts + p.short_parts > 16) || (joins_tall(a) && p.tall_parts > 16);
}
inline int64_t join_blocks(const AttendArgs& a, int64_t pairs) {
  return many_parts(a) ? pairs : (pairs + kWaves - 1) / kWaves;
}
inline int64_t short_join_blocks(const AttendArgs& a) { return joins_short(a) ? join_blocks(a, short_slots(a)) : 0; }
inline int64_t tall_join_blocks(const AttendArgs& a) {
  return joins_tall(a) ? join_blocks(a, a.rows.rows * a.shape.q_heads) : 0;
}

template <typename T, int D>
void launch_attend(const AttendArgs& a, hipStream_t stream) {
  const AttendPlan& p = a.plan;
  const dim3 grid((unsigned)(p.prefix_blocks + p.tall_blocks + p.thin_blocks + 1)), block(64 * kWaves);
  if (p.wide) hipLaunchKernelGGL((wide_kernel<D>), grid, dim3(64 * kWide), 0, stream, a);
  else if (p.alone) hipLaunchKernelGGL((attend_kernel<__bf16, D, true, true>), grid, block, 0, stream, a);
  else if (std::is_same<T, float>::value && p.reread)
    hipLaunchKernelGGL((attend_kernel<float, D, false, false>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((attend_kernel<T, D, true, false>), grid, block, 0, stream, a);
  const int64_t first = short_join_blocks(a), second = tall_join_blocks(a);
  if (first + second == 0) return;
  const dim3 joins((unsigned)(first + second));
  if (many_parts(a)) hipLaunchKernelGGL((combine_kernel<T, D, kWaves>), joins, block, 0, stream, a, (int)first);
  else hipLaunchKernelGGL((combine_kernel<T, D, 1>), joins, block, 0, stream, a, (int)first);
}

}  // namespace

bool cache_attend_fits(const AttendArgs& a) {
  constexpr int64_t most = (1 << 24) - 1;            // workgroups of 256: a launch has fewer than 2^32 threads
  const AttendPlan& p = a.plan;
  return p.prefix_blocks + p.tall_blocks + p.thin_blocks < most &&
         short_join_blocks(a) + tall_join_blocks(a) <= most;
}

hipError_t launch_cache_attend(const AttendArgs& a, hipStream_t stream) {
  if (a.rows.rows == 0 || a.runs.count == 0) return hipSuccess;
  const bool wide = a.shape.head_dim == 128;
  if (a.shape.dtype == SP_F32) wide ? launch_attend<float, 128>(a, stream) : launch_attend<float, 64>(a, stream);
  else wide ? launch_attend<__bf16, 128>(a, stream) : launch_attend<__bf16, 64>(a, stream);
  return hipGetLastError();
}

}  // namespace sp
