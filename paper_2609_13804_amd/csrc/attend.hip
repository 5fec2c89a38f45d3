// Attention of a batch's query rows over the paged cache:
//
//   o = sum_j softmax_j(scale q . k_j) v_j,  lse = log sum_j exp(scale q . k_j)
//
// over the tokens of the row's prefix run (all of them) and of its own run (up
// to the row's own place, or all).
//
// A tile is 32 or 128 consecutive (row, head) pairs of one segment and one key
// head: a segment is a sequence's rows, over its own run, or the rows of all
// the sequences of a group, over the group's prefix, which is so read once for
// all of them.  Pair x of a segment is row x / r, head x % r of the key head's r
// query heads, so grouped heads share every key and value that is read.  Keys
// are cut into chunks; a workgroup takes a tile, a key head and a chunk, and
// keeps the running maximum m, the sum l of 2^(s - m) and the values weighted by
// 2^(s - m) (scores s in powers of two).  A row with a single part is done; the
// others' parts go to the workspace and combine_kernel joins them:
//   o = sum_p 2^(m_p - M) o_p / sum_p 2^(m_p - M) l_p,  M = max_p m_p.
#include <float.h>

#include "sp_internal.h"
#include "cache_rows.h"
#include "lds_dma.h"

namespace sp {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) bf16x4_t* ltr_t;

constexpr int kThin = 32, kTall = 128;     // pairs of a tile
constexpr int kThinF32 = 16;
constexpr int kWaves = 4;
constexpr int kThinStep = 32 * kWaves;     // keys that the waves of a thin tile take together
constexpr int kTallStep = 64;
// Running maxima start here: a masked score (-inf) then weighs 2^-inf = 0 also
// where a row has seen nothing yet.
constexpr float kLowest = -FLT_MAX;
constexpr float kRescale = 8.0f;           // log2 of the largest unscaled probability

// what lanes past the last key load
__device__ __align__(16) const uint32_t zeros16[4] = {0, 0, 0, 0};

// ---------------------------------------------------------------- tiles

struct Tile {
  int64_t row0;           // the segment's first row
  int pairs;              // rows of the segment times r
  int x0;                 // the tile's first pair
  int seg;                // sequence or group
  int n;                  // rows of the segment
  int len;                // tokens of its run
  const int32_t* table;   // its pages
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
    const int s = prefix ? min(max(a.grp_off[i], 0), a.runs.count - 1) : i;
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

// Tokens that pair x sees of the segment's run.
__device__ __forceinline__ int sees(const AttendArgs& a, const Tile& t, bool prefix, int row) {
  if (prefix || a.all) return t.len;
  const int64_t v = (int64_t)t.len - t.n + row + 1;
  return v < 0 ? 0 : (int)v;
}

// Parts of a row's prefix: 0 without one.
__device__ __forceinline__ int prefix_parts(const AttendArgs& a, int s) {
  if (a.prefix.count == 0) return 0;
  const int g = wave_find_last(a.prefix.count, s, [&](int i) { return a.grp_off[i]; });
  int len;
  if (s < a.grp_off[g] || s >= a.grp_off[g + 1] || tokens_of(a.prefix, g, len) != SP_DEV_OK) return 0;
  return (len + a.plan.chunk_prefix - 1) / a.plan.chunk_prefix;
}

// A run's pages by block of 16 tokens, 64 blocks at a time in a wave's lanes.
struct Pages {
  const int32_t* table;
  int shift, count, blocks;    // log2 of blocks of a page; pages of the cache; blocks of the run
  __device__ __forceinline__ int load(int block0, int32_t* err) const {
    const int b = block0 + (int)(threadIdx.x & 63);
    int p = 0;
    if (b < blocks) p = table[b >> shift];
    if ((uint32_t)p >= (uint32_t)count) {
      set_device_error(err, SP_DEV_BAD_PAGE);
      p = 0;
    }
    return p;
  }
};

// ---------------------------------------------------------------- bfloat16

__device__ __forceinline__ float half_max(float v) {      // of this lane and the lane 32 away
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A head's rows in LDS: ROW bytes each, 16-byte chunks swizzled so that a pass of a
// fragment read touches every bank once: K (32 rows, a chunk of each) by the row,
// V (four rows, 64 bytes of each) by the row on 64-byte pieces.
template <int D>
struct Geo {
  static constexpr int ROW = 2 * D, CHUNKS = ROW / 16, LOAD_ROWS = 1024 / ROW;   // rows of a load
  static constexpr int BLOCK = 32 * ROW;                                          // 32 keys
  static constexpr int LOADS = BLOCK / 1024;
  __device__ static __forceinline__ int kswz(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }
  __device__ static __forceinline__ int vswz(int r) { return D == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2; }
};

// One wave's 32 pairs: lane l holds pair l % 32; of 32 keys' scores those of keys
// 8 (i / 4) + 4 (l / 32) + i % 4 in register i, and of the output elements
// 32 t + 8 (i / 4) + 4 (l / 32) + i % 4 in o[t][i] (v_mfma_f32_32x32x16_bf16 with
// keys, then values, as the row operand).
template <int D>
struct Pairs {
  bf16x8_t q[D / 16];
  f32x16_t o[D / 32];
  float m, l;             // m is the pair's, l this lane's share
  int lim;                // tokens that the pair sees
  int lim0;               // and the first pair of the wave
};

template <int D>
__device__ __forceinline__ void init_pairs(Pairs<D>& w) {
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) w.o[t][i] = 0.0f;
  w.m = kLowest;
  w.l = 0.0f;
}

// Loads the wave's queries; x is this lane's pair.  Pairs past the segment are zero.
template <int D>
__device__ __forceinline__ void load_queries(const AttendArgs& a, const Tile& t, bool prefix, int h, int x,
                                             int x_first, Pairs<D>& w) {
  const int half = (threadIdx.x & 63) >> 5, r = ratio(a);
  const bool live = x < t.pairs;
  const int row = live ? x / r : 0, sub = x - row * r;
  const uint16_t* src = static_cast<const uint16_t*>(a.Q) + (t.row0 + row) * a.ldq + (h * r + sub) * D;
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    uint4 u = make_uint4(0, 0, 0, 0);
    if (live) u = *reinterpret_cast<const uint4*>(src + 16 * s + 8 * half);
    w.q[s] = __builtin_bit_cast(bf16x8_t, u);
  }
  w.lim = live ? sees(a, t, prefix, row) : 0;
  w.lim0 = x_first < t.pairs ? sees(a, t, prefix, x_first / r) : 0;
}

template <int D>
__device__ __forceinline__ bf16x4_t read_vt(const char* V, int t, int row0) {
  const int lane = threadIdx.x & 63, vr = (lane >> 2) & 3, row = row0 + 4 * (lane >> 5) + vr;
  const int piece = 4 * t ^ Geo<D>::vswz(vr);             // (row0 + 4 half is a multiple of 4)
  return __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
      (ltr_t)(V + row * Geo<D>::ROW + piece * 16 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8));
}

// 32 NB keys from key kb on, in the LDS tiles K and V, whose rows hold zeros from key
// `loaded` on.  values() returns once V is there.
template <int D, int NB, typename Wait>
__device__ __forceinline__ void step(Pairs<D>& w, const char* K, const char* V, int kb, int loaded,
                                     float c2, Wait values) {
  using G = Geo<D>;
  const int lane = threadIdx.x & 63, ql = lane & 31, half = lane >> 5;
  f32x16_t st[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) st[n][i] = 0.0f;
#pragma unroll
  for (int s = 0; s < D / 16; ++s)
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const uint4 u = *reinterpret_cast<const uint4*>(K + n * G::BLOCK + ql * G::ROW +
                                                      (((2 * s + half) ^ G::kswz(ql)) << 4));
      st[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, u), w.q[s], st[n], 0, 0, 0);
    }
  const bool masked = kb + 32 * NB > w.lim0;
  if (masked) {
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (kb + 32 * n + 8 * (i >> 2) + 4 * half + (i & 3) >= w.lim) st[n][i] = -INFINITY;
  }
  float bm = st[0][0];
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) bm = fmaxf(bm, st[n][i]);
  const float mx = half_max(bm) * c2;
  if (__any(mx > w.m + kRescale)) {
    const float mn = fmaxf(w.m, mx);
    const float sc = __builtin_amdgcn_exp2f(w.m - mn);
    w.m = mn;
    w.l *= sc;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) w.o[t][i] *= sc;
  }
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      st[n][i] = __builtin_amdgcn_exp2f(fmaf(st[n][i], c2, -w.m));
      w.l += st[n][i];
    }
  values();
  // Keys that some pairs see and others do not: a product would weigh them with 0
  // for the others, which is NaN where the value is infinite or NaN.  Such tiles
  // (never in sound data) go key by key.
  if (masked && min(kb + 32 * NB, loaded) > w.lim0) {
    uint32_t bad = 0;
#pragma unroll
    for (int c = 0; c < NB * G::LOADS; ++c) {
      const uint4 u = *reinterpret_cast<const uint4*>(V + c * 1024 + lane * 16);
      const uint32_t v[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int k = 0; k < 4; ++k)
        bad |= (uint32_t)((v[k] & 0x7f800000u) == 0x7f800000u) | (uint32_t)((v[k] & 0x7f80u) == 0x7f80u);
    }
    if (__any(bad)) {
      for (int n = 0; n < NB; ++n)
        for (int i = 0; i < 16; ++i) {
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const float p = (float)(__bf16)__shfl(st[0][0], ql + 32 * hf, 64);
            const int key = 32 * n + 8 * (i >> 2) + 4 * hf + (i & 3);
            if (kb + key < w.lim) {
#pragma unroll
              for (int t = 0; t < D / 32; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                  const bf16x4_t v = *reinterpret_cast<const bf16x4_t*>(
                      V + key * G::ROW + (((4 * t + g) ^ G::vswz(key)) << 4) + 8 * half);
#pragma unroll
                  for (int k = 0; k < 4; ++k) w.o[t][4 * g + k] = fmaf(p, (float)v[k], w.o[t][4 * g + k]);
                }
            }
          }
          // the next key's probability into st[0][0]: registers have no index
#pragma unroll
          for (int k = 0; k < 16 * NB - 1; ++k) st[k >> 4][k & 15] = st[(k + 1) >> 4][(k + 1) & 15];
        }
      return;
    }
  }
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    bf16x8_t pb[2];
#pragma unroll
    for (int i = 0; i < 16; ++i) pb[i >> 3][i & 7] = (__bf16)st[n][i];
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int t = 0; t < D / 32; ++t) {
        const bf16x4_t lo = read_vt<D>(V, t, 32 * n + 16 * g), hi = read_vt<D>(V, t, 32 * n + 16 * g + 8);
        const bf16x8_t v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        w.o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pb[g], w.o[t], 0, 0, 0);
      }
  }
}

// An address that is the same in all lanes, in scalar registers.
__device__ __forceinline__ const char* uniform(const char* p) {
  const uint64_t u = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)u);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(u >> 32));
  return reinterpret_cast<const char*>(((uint64_t)hi << 32) | lo);
}

// Loads LOAD_ROWS keys from key0 on (one page) into rows row0 .. of a tile of K and of V: an
// instruction fills 1 KB, lane i lands on chunk i % CHUNKS of row i / CHUNKS and
// fetches the chunk that the swizzle puts there.  Keys from `end` on are zeros.
template <int D>
__device__ __forceinline__ void load_group(const char* Kc, const char* Vc, int64_t head_page, int page_mask,
                                           int key0, int row0, int end, char* K, char* V) {
  using G = Geo<D>;
  const int lane = threadIdx.x & 63, lr = lane / G::CHUNKS, ch = lane % G::CHUNKS;
  const int64_t at = (head_page * (page_mask + 1) + (key0 & page_mask)) * G::ROW;   // uniform
  const uint32_t ko = lr * G::ROW + ((ch ^ G::kswz(row0 + lr)) << 4);
  const uint32_t vo = lr * G::ROW + ((ch ^ G::vswz(lr)) << 4);
  if (key0 + G::LOAD_ROWS <= end) {
    lds_dma16(uniform(Kc + at), ko, K + row0 * G::ROW);
    lds_dma16(uniform(Vc + at), vo, V + row0 * G::ROW);
  } else {
    const bool in = key0 + lr < end;
    lds_dma16(in ? (const void*)(Kc + at + ko) : (const void*)zeros16, K + row0 * G::ROW);
    lds_dma16(in ? (const void*)(Vc + at + vo) : (const void*)zeros16, V + row0 * G::ROW);
  }
}

// ---- where a pair's result goes

struct Out {
  int64_t row;            // -1: nowhere
  int head;
  bool done;              // the only part: into O; else a part
  int part, parts;
};

// The pair's place and whether this part is its only one (own: parts of its
// prefix pp).  First chunk: the row's count of parts, for combine_kernel.
__device__ __forceinline__ Out place_of(const AttendArgs& a, const Tile& t, bool prefix, int h, int x, int chunk_keys,
                                        int chunk, int pp) {
  Out u;
  const int r = ratio(a);
  u.parts = a.plan.prefix_parts + a.plan.own_parts;
  u.row = -1;
  u.done = false;
  u.part = prefix ? chunk : a.plan.prefix_parts + chunk;
  u.head = 0;
  if (x >= t.pairs) return u;
  const int i = x / r;
  const int64_t row = t.row0 + i;
  u.head = h * r + (x - i * r);
  if (prefix) {
    // a padded slice's rows past its count
    if (a.rows.padded && (int)(row % a.rows.rows_per_seq) >= a.rows.info[row / a.rows.rows_per_seq]) return u;
    u.row = row;
    return u;
  }
  const int own = (sees(a, t, false, i) + chunk_keys - 1) / chunk_keys;
  if (chunk == 0 && h == 0 && x == i * r) a.row_parts[row] = pp == 0 && own <= 1 ? 0 : (own | pp << 16);
  u.done = pp == 0 && own <= 1;                      // (a row that sees nothing: zeros, by its first chunk)
  if (chunk < own || (u.done && chunk == 0)) u.row = row;
  return u;
}

__device__ __forceinline__ float lse_of(float m, float l) {
  return l > 0.0f || l != l ? (m + __log2f(l)) * 0.6931471805599453f : -INFINITY;
}

__device__ __forceinline__ void store_ml(const AttendArgs& a, const Out& u, float m, float l) {
  const int64_t pair = u.row * a.shape.q_heads + u.head;
  if (u.done) {
    if (a.lse) a.lse[pair] = lse_of(m, l);
  } else {
    reinterpret_cast<float2*>(a.part_ml)[pair * u.parts + u.part] = make_float2(m, l);
  }
}

// ---------------------------------------------------------------- the thin tiles

// 32 pairs; each of four waves takes every fourth block of 32 keys, through a ring
// of its own in LDS (no barrier until the end), and the waves' results are
// joined through LDS.
template <int D>
struct ThinShape {
  static constexpr int STAGES = D == 128 ? 2 : 4;
  static constexpr int RING = STAGES * 2 * Geo<D>::BLOCK;
  static constexpr int PART_ROW = D + 4;
  static constexpr int PARTS = kWaves * 32 * (PART_ROW + 2) * 4;
  static constexpr int LDS = kWaves * RING > PARTS ? kWaves * RING : PARTS;
};

template <int D>
__global__ __launch_bounds__(64 * kWaves, 1) void thin_kernel(AttendArgs a, int prefix, int tiled) {
  using G = Geo<D>;
  using SH = ThinShape<D>;
  __shared__ __attribute__((aligned(1024))) char smem[SH::LDS];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), ql = lane & 31;
  const int h = blockIdx.y, chunk = blockIdx.z;
  if (blockIdx.x == 0 && h == 0 && chunk == 0) report_entries(a, prefix);
  Tile t;
  if (tiled) {
    if (!find_tile<kThin>(a, prefix, blockIdx.x, t)) return;
  } else {                                           // a sequence to a tile; longer ones are the tall tiles'
    t.seg = blockIdx.x;
    if (rows_of(a.rows, t.seg, t.row0, t.n) != SP_DEV_OK) return;
    const int64_t pairs = (int64_t)t.n * ratio(a);
    if (pairs == 0 || pairs > kThin || tokens_of(a.runs, t.seg, t.len) != SP_DEV_OK) return;
    t.pairs = (int)pairs;
    t.x0 = 0;
    t.table = a.runs.table + (int64_t)t.seg * a.runs.width;
  }
  const int chunk_keys = prefix ? a.plan.chunk_prefix : a.plan.chunk_thin;
  const int pp = prefix ? 0 : prefix_parts(a, t.seg);
  // the last pair's limit is the tile's
  const int last = min(t.x0 + kThin, t.pairs) - 1;
  const int tile_end = sees(a, t, prefix, last / ratio(a));
  const int k0 = chunk * chunk_keys;
  if (k0 >= tile_end && (prefix || chunk > 0)) return;
  const int k1 = min(tile_end, k0 + chunk_keys);

  Pairs<D> w;
  init_pairs(w);
  load_queries<D>(a, t, prefix, h, t.x0 + ql, t.x0, w);

  const int page_mask = (1 << a.shape.page_shift) - 1;
  const Pages pages{t.table, a.shape.page_shift - 4, a.shape.pages, (t.len + 15) >> 4};
  const char* Kc = static_cast<const char*>(a.k_cache);
  const char* Vc = static_cast<const char*>(a.v_cache);
  char* ring = smem + wave * SH::RING;
  // block i of the wave: keys k0 + 32 (wave + 4 i); its two 16-key pages in lane i % 64's registers
  const int blocks = k1 - k0 > 32 * wave ? (k1 - k0 - 32 * wave + kThinStep - 1) / kThinStep : 0;
  int pg[2] = {0, 0};
  auto fetch_pages = [&](int i0) {
    const int b = (k0 >> 4) + 2 * (wave + kWaves * (i0 + lane));
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      int p = 0;
      if (b + e < pages.blocks) p = pages.table[(b + e) >> pages.shift];
      if ((uint32_t)p >= (uint32_t)pages.count) {
        set_device_error(a.err, SP_DEV_BAD_PAGE);
        p = 0;
      }
      pg[e] = p;
    }
  };
  auto issue = [&](int i) {
    if ((i & 63) == 0) fetch_pages(i);
    const int kb = k0 + 32 * (wave + kWaves * i);
    char* K = ring + (i % SH::STAGES) * 2 * G::BLOCK;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int64_t head_page = (int64_t)__builtin_amdgcn_readlane(pg[e], i & 63) * a.shape.kv_heads + h;
#pragma unroll
      for (int g = 0; g < G::LOADS / 2; ++g) {
        const int row0 = 16 * e + G::LOAD_ROWS * g;
        load_group<D>(Kc, Vc, head_page, page_mask, kb + row0, row0, k1, K, K + G::BLOCK);
      }
    }
  };
#pragma unroll
  for (int i = 0; i < SH::STAGES - 1; ++i)
    if (i < blocks) issue(i);
  for (int i = 0; i < blocks; ++i) {
    if (i + SH::STAGES - 1 < blocks) {
      wait_lgkm0();                                  // the reads of the buffer that is filled next
      issue(i + SH::STAGES - 1);
      wait_vmcnt<(SH::STAGES - 1) * 2 * G::LOADS>();
    } else {
      wait_vmcnt<0>();
    }
    // (the wait alone does not keep the compiler from moving reads of LDS over it)
    asm volatile("" ::: "memory");
    const char* K = ring + (i % SH::STAGES) * 2 * G::BLOCK;
    step<D, 1>(w, K, K + G::BLOCK, k0 + 32 * (wave + kWaves * i), k1, a.c2, [] {});
  }
  w.l = half_sum(w.l);

  // the waves' results, joined: part [wave][pair][PART_ROW], then [m, l][wave][pair]
  __syncthreads();
  float* part = reinterpret_cast<float*>(smem);
  float* ml = part + kWaves * 32 * SH::PART_ROW;
  const int half = lane >> 5;
#pragma unroll
  for (int e = 0; e < D / 32; ++e)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<float4*>(part + (wave * 32 + ql) * SH::PART_ROW + 32 * e + 8 * g + 4 * half) =
          make_float4(w.o[e][4 * g], w.o[e][4 * g + 1], w.o[e][4 * g + 2], w.o[e][4 * g + 3]);
  if (half == 0) {
    ml[wave * 32 + ql] = w.m;
    ml[(kWaves + wave) * 32 + ql] = w.l;
  }
  __syncthreads();
  constexpr int E = D / 8;                            // elements of a thread, eight threads to a pair
  const int c = tid >> 3, e0 = (tid & 7) * E;
  const Out u = place_of(a, t, prefix, h, t.x0 + c, chunk_keys, chunk, pp);
  if (u.row < 0) return;
  float M = kLowest, L = 0.0f, acc[E];
#pragma unroll
  for (int v = 0; v < kWaves; ++v) M = fmaxf(M, ml[v * 32 + c]);
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.0f;
#pragma unroll
  for (int v = 0; v < kWaves; ++v) {
    const float f = __builtin_amdgcn_exp2f(ml[v * 32 + c] - M);
    L = fmaf(ml[(kWaves + v) * 32 + c], f, L);
#pragma unroll
    for (int e = 0; e < E; e += 4) {
      const float4 x = *reinterpret_cast<const float4*>(part + (v * 32 + c) * SH::PART_ROW + e0 + e);
      acc[e] = fmaf(x.x, f, acc[e]);
      acc[e + 1] = fmaf(x.y, f, acc[e + 1]);
      acc[e + 2] = fmaf(x.z, f, acc[e + 2]);
      acc[e + 3] = fmaf(x.w, f, acc[e + 3]);
    }
  }
  if ((tid & 7) == 0) store_ml(a, u, M, L);
  const int64_t pair = u.row * a.shape.q_heads + u.head;
  if (u.done) {
    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
    __bf16* dst = static_cast<__bf16*>(a.O) + pair * D + e0;
#pragma unroll
    for (int e = 0; e < E; e += 8) {
      bf16x8_t v;
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = (__bf16)(acc[e + k] * inv);
      *reinterpret_cast<bf16x8_t*>(dst + e) = v;
    }
  } else {
    float* dst = a.part_o + (pair * u.parts + u.part) * D + e0;
#pragma unroll
    for (int e = 0; e < E; e += 4)
      *reinterpret_cast<float4*>(dst + e) = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
  }
}

// ---------------------------------------------------------------- the tall tiles

// 128 pairs, 32 a wave; the waves share tiles of 64 keys, two deep.
template <int D>
__global__ __launch_bounds__(64 * kWaves, 2) void tall_kernel(AttendArgs a, int prefix) {
  using G = Geo<D>;
  __shared__ __attribute__((aligned(1024))) char smem[2 * 4 * G::BLOCK];     // [buffer][K, V][64 keys]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), ql = lane & 31, half = lane >> 5;
  const int h = blockIdx.y, chunk = blockIdx.z;
  if (blockIdx.x == 0 && h == 0 && chunk == 0 && prefix) report_entries(a, prefix);
  Tile t;
  if (!find_tile<kTall>(a, prefix, blockIdx.x, t)) return;
  if (!prefix && t.pairs <= kThin) return;                                   // a thin tile's
  const int chunk_keys = prefix ? a.plan.chunk_prefix : a.plan.chunk_tall;
  const int pp = prefix ? 0 : prefix_parts(a, t.seg);
  const int r = ratio(a);
  const int tile_end = sees(a, t, prefix, (min(t.x0 + kTall, t.pairs) - 1) / r);
  const int k0 = chunk * chunk_keys;
  if (k0 >= tile_end && (prefix || chunk > 0)) return;
  const int k1 = min(tile_end, k0 + chunk_keys);

  const int xw = t.x0 + 32 * wave, x = xw + ql;
  Pairs<D> w;
  init_pairs(w);
  load_queries<D>(a, t, prefix, h, x, xw, w);
  // keys that this wave needs: none without a pair
  const int wave_end = xw >= t.pairs ? 0 : min(k1, sees(a, t, prefix, (min(xw + 32, t.pairs) - 1) / r));

  const int page_mask = (1 << a.shape.page_shift) - 1;
  const Pages pages{t.table, a.shape.page_shift - 4, a.shape.pages, (t.len + 15) >> 4};
  const char* Kc = static_cast<const char*>(a.k_cache);
  const char* Vc = static_cast<const char*>(a.v_cache);
  const int tiles = k1 > k0 ? (k1 - k0 + kTallStep - 1) / kTallStep : 0;
  int pg = 0;                                        // lane l: the page of block 64 (i / 16) + l of the chunk
  auto issue = [&](int i) {
    if ((i & 15) == 0) pg = pages.load((k0 >> 4) + 4 * i, a.err);
    const int kb = k0 + kTallStep * i;
    char* K = smem + (i & 1) * 4 * G::BLOCK;
#pragma unroll
    for (int j = 0; j < 2 * G::LOADS / kWaves; ++j) {
      const int row0 = (wave + kWaves * j) * G::LOAD_ROWS;
      const int64_t head_page =
          (int64_t)__builtin_amdgcn_readlane(pg, 4 * (i & 15) + (row0 >> 4)) * a.shape.kv_heads + h;
      load_group<D>(Kc, Vc, head_page, page_mask, kb + row0, row0, k1, K, K + 2 * G::BLOCK);
    }
  };
  if (tiles > 0) issue(0);
  for (int i = 0; i < tiles; ++i) {
    wait_vmcnt<0>();                                 // this wave's loads of tile i
    __syncthreads();                                 // every wave's; and all are past tile i - 1
    if (i + 1 < tiles) issue(i + 1);
    const int kb = k0 + kTallStep * i;
    const char* K = smem + (i & 1) * 4 * G::BLOCK;
    if (kb < wave_end) step<D, 2>(w, K, K + 2 * G::BLOCK, kb, k1, a.c2, [] {});
  }
  w.l = half_sum(w.l);

  const Out u = place_of(a, t, prefix, h, x, chunk_keys, chunk, pp);
  if (u.row < 0) return;
  if (half == 0) store_ml(a, u, w.m, w.l);
  const int64_t pair = u.row * a.shape.q_heads + u.head;
  const float inv = w.l == 0.0f ? 0.0f : 1.0f / w.l;
  __bf16* out = static_cast<__bf16*>(a.O) + pair * D;
  float* dst = a.part_o + (pair * u.parts + u.part) * D;
#pragma unroll
  for (int e = 0; e < D / 32; ++e)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int c = 32 * e + 8 * g + 4 * half;
      if (u.done) {
        bf16x4_t v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = (__bf16)(w.o[e][4 * g + k] * inv);
        *reinterpret_cast<bf16x4_t*>(out + c) = v;
      } else {
        *reinterpret_cast<float4*>(dst + c) =
            make_float4(w.o[e][4 * g], w.o[e][4 * g + 1], w.o[e][4 * g + 2], w.o[e][4 * g + 3]);
      }
    }
}

// ---------------------------------------------------------------- float32

// 16 pairs; each of four waves takes every fourth block of 16 keys (one page),
// straight from memory into the operands' registers:
//   S^T = K Q^T (v_mfma_f32_16x16x4_f32): lane l holds key l % 16 and, of each 16
//   elements of a row, the four from 4 (l / 16) on, one to each of four products;
//   scores of keys 4 (l / 16) + i of pair l % 16;
//   O^T += V^T P: lane l holds element l % 16 of each 16 of the keys 4 (l / 16) + i.
template <int D>
__global__ __launch_bounds__(64 * kWaves) void attend_f32_kernel(AttendArgs a, int prefix) {
  constexpr int PART_ROW = D + 4;
  __shared__ __attribute__((aligned(16))) float smem[kWaves * 16 * (PART_ROW + 2)];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), ql = lane & 15, quad = lane >> 4;
  const int h = blockIdx.y, chunk = blockIdx.z;
  if (blockIdx.x == 0 && h == 0 && chunk == 0) report_entries(a, prefix);
  Tile t;
  if (!find_tile<kThinF32>(a, prefix, blockIdx.x, t)) return;
  const int chunk_keys = prefix ? a.plan.chunk_prefix : a.plan.chunk_thin;
  const int pp = prefix ? 0 : prefix_parts(a, t.seg);
  const int r = ratio(a);
  const int tile_end = sees(a, t, prefix, (min(t.x0 + kThinF32, t.pairs) - 1) / r);
  const int k0 = chunk * chunk_keys;
  if (k0 >= tile_end && (prefix || chunk > 0)) return;
  const int k1 = min(tile_end, k0 + chunk_keys);

  const int x = t.x0 + ql;
  const bool live = x < t.pairs;
  const int row = live ? x / r : 0;
  const float* qsrc = static_cast<const float*>(a.Q) + (t.row0 + row) * a.ldq + (h * r + (x - row * r)) * D + 4 * quad;
  f32x4_t q[D / 16];
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    q[s] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    if (live) q[s] = *reinterpret_cast<const f32x4_t*>(qsrc + 16 * s);
  }
  const int lim = live ? sees(a, t, prefix, row) : 0;
  const int lim0 = sees(a, t, prefix, t.x0 / r);

  f32x4_t o[D / 16];
#pragma unroll
  for (int e = 0; e < D / 16; ++e) o[e] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  float m = kLowest, l = 0.0f;
  const int page_mask = (1 << a.shape.page_shift) - 1;
  const Pages pages{t.table, a.shape.page_shift - 4, a.shape.pages, (t.len + 15) >> 4};
  const int blocks = k1 - k0 > 16 * wave ? (k1 - k0 - 16 * wave + 16 * kWaves - 1) / (16 * kWaves) : 0;
  int pg = 0;                                        // lane l: the page of block i - i % 16 + l / 4 of wave l % 4
  for (int i = 0; i < blocks; ++i) {
    if ((i & 15) == 0) pg = pages.load((k0 >> 4) + 4 * i, a.err);
    const int kb = k0 + 16 * (wave + kWaves * i);
    const int64_t head_page =
        (int64_t)__builtin_amdgcn_readlane(pg, 4 * (i & 15) + wave) * a.shape.kv_heads + h;
    const int64_t at = (head_page * (page_mask + 1) + (kb & page_mask)) * D;
    const float* K = static_cast<const float*>(a.k_cache) + at;
    const float* V = static_cast<const float*>(a.v_cache) + at;
    const int in = k1 - kb;                          // keys of the block
    f32x4_t k[D / 16];
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      k[s] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
      if (ql < in) k[s] = *reinterpret_cast<const f32x4_t*>(K + ql * D + 16 * s + 4 * quad);
    }
    float v[D / 16][4];
#pragma unroll
    for (int e = 0; e < D / 16; ++e)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        v[e][g] = 0.0f;
        if (4 * quad + g < in) v[e][g] = V[(4 * quad + g) * D + 16 * e + ql];
      }
    f32x4_t st = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
#pragma unroll
      for (int g = 0; g < 4; ++g) st = __builtin_amdgcn_mfma_f32_16x16x4f32(k[s][g], q[s][g], st, 0, 0, 0);
    const bool masked = kb + 16 > lim0;
    if (masked) {
#pragma unroll
      for (int g = 0; g < 4; ++g)
        if (kb + 4 * quad + g >= lim) st[g] = -INFINITY;
    }
    float bm = fmaxf(fmaxf(st[0], st[1]), fmaxf(st[2], st[3]));
    bm = fmaxf(bm, __shfl_xor(bm, 16, 64));
    bm = fmaxf(bm, __shfl_xor(bm, 32, 64));
    const float mn = fmaxf(m, bm * a.c2);
    const float sc = exp2f(m - mn);
    m = mn;
    l *= sc;
#pragma unroll
    for (int e = 0; e < D / 16; ++e) o[e] *= sc;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      st[g] = exp2f(fmaf(st[g], a.c2, -m));
      l += st[g];
    }
    if (masked && min(kb + 16, k1) > lim0) {         // as in the bfloat16 step
      bool bad = false;
#pragma unroll
      for (int e = 0; e < D / 16; ++e)
#pragma unroll
        for (int g = 0; g < 4; ++g) bad |= !(fabsf(v[e][g]) <= FLT_MAX);
      if (__any(bad)) {
        for (int g = 0; g < 4; ++g) {
          for (int qd = 0; qd < 4; ++qd) {
            const float p = __shfl(st[0], ql + 16 * qd, 64);
            const int key = 4 * qd + g;
            if (kb + key < lim) {
#pragma unroll
              for (int e = 0; e < D / 16; ++e)
                o[e] += p * *reinterpret_cast<const f32x4_t*>(V + key * D + 16 * e + 4 * quad);
            }
          }
          st[0] = st[1];
          st[1] = st[2];
          st[2] = st[3];
        }
        continue;
      }
    }
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
      for (int e = 0; e < D / 16; ++e) o[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e][g], st[g], o[e], 0, 0, 0);
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);

  float* ml = smem + kWaves * 16 * PART_ROW;         // part [wave][pair][PART_ROW], then [m, l][wave][pair]
#pragma unroll
  for (int e = 0; e < D / 16; ++e)
    *reinterpret_cast<f32x4_t*>(smem + (wave * 16 + ql) * PART_ROW + 16 * e + 4 * quad) = o[e];
  if (quad == 0) {
    ml[wave * 16 + ql] = m;
    ml[(kWaves + wave) * 16 + ql] = l;
  }
  __syncthreads();
  constexpr int E = D / 16;                          // sixteen threads to a pair
  const int c = tid >> 4, e0 = (tid & 15) * E;
  const Out u = place_of(a, t, prefix, h, t.x0 + c, chunk_keys, chunk, pp);
  if (u.row < 0) return;
  float M = kLowest, L = 0.0f, acc[E];
#pragma unroll
  for (int y = 0; y < kWaves; ++y) M = fmaxf(M, ml[y * 16 + c]);
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.0f;
#pragma unroll
  for (int y = 0; y < kWaves; ++y) {
    const float f = exp2f(ml[y * 16 + c] - M);
    L = fmaf(ml[(kWaves + y) * 16 + c], f, L);
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = fmaf(smem[(y * 16 + c) * PART_ROW + e0 + e], f, acc[e]);
  }
  if ((tid & 15) == 0) store_ml(a, u, M, L);
  const int64_t pair = u.row * a.shape.q_heads + u.head;
  const float inv = !u.done ? 1.0f : L == 0.0f ? 0.0f : 1.0f / L;
  float* dst = u.done ? static_cast<float*>(a.O) + pair * D : a.part_o + (pair * u.parts + u.part) * D;
#pragma unroll
  for (int e = 0; e < E; e += 4)
    *reinterpret_cast<float4*>(dst + e0 + e) =
        make_float4(acc[e] * inv, acc[e + 1] * inv, acc[e + 2] * inv, acc[e + 3] * inv);
}

// ---------------------------------------------------------------- joining the parts

// One wave to a (row, head): the parts' maxima and sums, then their outputs.
template <typename T, int D>
__global__ __launch_bounds__(64 * kWaves) void combine_kernel(AttendArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t pair = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  const int64_t row = pair / a.shape.q_heads;
  if (row >= a.rows.rows) return;
  // rows of no sequence have no count of parts
  if (a.rows.padded) {
    const int64_t s = a.rows.rows_per_seq > 0 ? row / a.rows.rows_per_seq : a.runs.count;
    if (s >= a.runs.count || row - s * a.rows.rows_per_seq >= a.rows.info[s]) return;
  } else if (row < a.rows.info[0] || row >= a.rows.info[a.runs.count]) {
    return;
  }
  const int code = a.row_parts[row], own = code & 0xffff, pre = code >> 16;
  if (code == 0 || own > a.plan.own_parts || pre > a.plan.prefix_parts) return;
  const int parts = a.plan.prefix_parts + a.plan.own_parts;
  const float2* ml = reinterpret_cast<const float2*>(a.part_ml) + pair * parts;
  const float* po = a.part_o + pair * parts * D;
  auto slot = [&](int i) { return i < pre ? i : a.plan.prefix_parts + i - pre; };
  float M = kLowest;
  for (int i = lane; i < pre + own; i += 64) M = fmaxf(M, ml[slot(i)].x);
  for (int s = 32; s >= 1; s >>= 1) M = fmaxf(M, __shfl_xor(M, s, 64));
  constexpr int E = D / 64;
  float L = 0.0f, acc[E] = {};
  for (int i = 0; i < pre + own; ++i) {
    const int p = slot(i);
    const float f = exp2f(ml[p].x - M);
    L = fmaf(ml[p].y, f, L);
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = fmaf(po[(int64_t)p * D + E * lane + e], f, acc[e]);
  }
  const float inv = L == 0.0f ? 0.0f : 1.0f / L;
#pragma unroll
  for (int e = 0; e < E; ++e) static_cast<T*>(a.O)[pair * D + E * lane + e] = (T)(acc[e] * inv);
  if (a.lse && lane == 0) a.lse[pair] = lse_of(M, L);
}

// Keys of a chunk: enough chunks that `tiles` tiles and key heads give the device
// about `target` workgroups, of at least `least` keys each, in whole steps.
inline int chunk_of(int64_t tiles, int max_len, int64_t target, int least, int step) {
  int64_t parts = (target + tiles - 1) / tiles;
  const int64_t most = (max_len + least - 1) / least;
  if (parts > most) parts = most;
  if (parts > 1024) parts = 1024;
  if (parts < 1) parts = 1;
  const int64_t keys = (max_len + parts - 1) / parts;
  return (int)((keys + step - 1) / step * step) + (keys == 0 ? step : 0);
}

inline int parts_of(int max_len, int chunk) { return (max_len + chunk - 1) / chunk; }

}  // namespace

AttendPlan plan_cache_attend(const CacheShape& s, const CacheRows& rows, const CacheRuns& runs,
                             const CacheRuns& prefix) {
  AttendPlan p{};
  const int64_t r = s.q_heads / s.kv_heads, pairs = rows.rows * r;
  const int64_t S = runs.count > 0 ? runs.count : 1, G = prefix.count > 0 ? prefix.count : 1;
  const bool f32 = s.dtype == SP_F32;
  p.prefix_tall = !f32 && prefix.count > 0 && pairs > (int64_t)kThin * G;
  p.own_tall = !f32 && rows.max_rows * r > kThin;
  const int thin = f32 ? kThinF32 : kThin, thin_step = f32 ? 16 * kWaves : kThinStep;
  const int64_t heads = s.kv_heads;
  p.chunk_thin = chunk_of((f32 ? pairs / thin + S : S) * heads, runs.max_len, 512, 256, thin_step);
  p.chunk_tall = chunk_of((pairs / kTall + S) * heads, runs.max_len, 512, 512, kTallStep);
  const int tile = p.prefix_tall ? kTall : thin;
  p.chunk_prefix = chunk_of((pairs / tile + G) * heads, prefix.max_len, 512, p.prefix_tall ? 512 : 256,
                            p.prefix_tall ? kTallStep : thin_step);
  p.prefix_parts = prefix.count > 0 ? parts_of(prefix.max_len, p.chunk_prefix) : 0;
  p.own_parts = parts_of(runs.max_len, p.chunk_thin);
  if (p.own_tall && parts_of(runs.max_len, p.chunk_tall) > p.own_parts)
    p.own_parts = parts_of(runs.max_len, p.chunk_tall);
  return p;
}

namespace {

template <int D>
void launch_tiles(const AttendArgs& a, hipStream_t stream) {
  const AttendPlan& p = a.plan;
  const int64_t r = a.shape.q_heads / a.shape.kv_heads, pairs = a.rows.rows * r;
  const unsigned heads = (unsigned)a.shape.kv_heads, S = (unsigned)a.runs.count, G = (unsigned)a.prefix.count;
  auto chunks = [](int max_len, int chunk) { return (unsigned)(max_len > 0 ? parts_of(max_len, chunk) : 1); };
  const dim3 block(64 * kWaves);
  if (a.shape.dtype == SP_F32) {
    if (p.prefix_parts > 0)
      hipLaunchKernelGGL(attend_f32_kernel<D>, dim3((unsigned)(pairs / kThinF32) + G, heads, p.prefix_parts), block,
                         0, stream, a, 1);
    hipLaunchKernelGGL(attend_f32_kernel<D>,
                       dim3((unsigned)(pairs / kThinF32) + S, heads, chunks(a.runs.max_len, p.chunk_thin)), block, 0,
                       stream, a, 0);
    return;
  }
  if (p.prefix_parts > 0) {
    if (p.prefix_tall)
      hipLaunchKernelGGL(tall_kernel<D>, dim3((unsigned)(pairs / kTall) + G, heads, p.prefix_parts), block, 0, stream,
                         a, 1);
    else
      hipLaunchKernelGGL(thin_kernel<D>, dim3((unsigned)(pairs / kThin) + G, heads, p.prefix_parts), block, 0, stream,
                         a, 1, 1);
  }
  if (p.own_tall)
    hipLaunchKernelGGL(tall_kernel<D>,
                       dim3((unsigned)(pairs / kTall) + S, heads, chunks(a.runs.max_len, p.chunk_tall)), block, 0,
                       stream, a, 0);
  hipLaunchKernelGGL(thin_kernel<D>, dim3(S, heads, chunks(a.runs.max_len, p.chunk_thin)), block, 0, stream, a, 0, 0);
}

template <typename T>
void launch_combine(const AttendArgs& a, hipStream_t stream) {
  const int64_t pairs = a.rows.rows * a.shape.q_heads;
  const dim3 grid((unsigned)((pairs + kWaves - 1) / kWaves)), block(64 * kWaves);
  if (a.shape.head_dim == 128) hipLaunchKernelGGL((combine_kernel<T, 128>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((combine_kernel<T, 64>), grid, block, 0, stream, a);
}

}  // namespace

hipError_t launch_cache_attend(const AttendArgs& a, hipStream_t stream) {
  if (a.rows.rows == 0 || a.runs.count == 0) return hipSuccess;
  if (a.shape.head_dim == 128) launch_tiles<128>(a, stream);
  else launch_tiles<64>(a, stream);
  if (a.plan.prefix_parts > 0 || a.plan.own_parts > 1) {
    if (a.shape.dtype == SP_F32) launch_combine<float>(a, stream);
    else launch_combine<__bf16>(a, stream);
  }
  return hipGetLastError();
}

}  // namespace sp
