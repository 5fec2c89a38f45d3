// Appending a batch's keys and values to a paged cache, the keys (and the
// queries, on their way to the attention) rotated by position:
//
//   slot p = len[s] - n_s + i of run s for row i of sequence s;
//   k[p]_(x, x') = (x c - x' s, x' c + x s),  (c, s) = cos_sin[pos[axis(j)][row]][j];
//   v[p] = v.
//
// Bound by memory: every element is read once and written once.  A lane holds
// the two 16-byte chunks of a head whose elements pair up (halves: chunk j and
// its partner half a rotation away; interleaved: chunks 2j and 2j + 1), and the
// cosines and sines of their pairs, which it keeps for all the heads of its row
// that it passes over.  Few rows are bound by the chain of loads from a row to its
// sequence, length, page and angles; the row's own loads go ahead of it.  Stores are
// streamed past the caches: 54070 rows of 28 + 8 heads of 128 (997 MB) 172 us (5.8
// TB/s), with ordinary stores 188; 3400 rows 11.7 and 14.7 us.
#include "sp_internal.h"
#include "cache_rows.h"

namespace sp {
namespace {

constexpr int kAppendWaves = 4;
constexpr int kPasses = 4;            // passes whose loads are in flight together

template <typename T>
struct Chunk;                         // 16 bytes
template <>
struct Chunk<__bf16> {
  static constexpr int N = 8;
  typedef __bf16 vec __attribute__((ext_vector_type(8)));
};
template <>
struct Chunk<float> {
  static constexpr int N = 4;
  typedef float vec __attribute__((ext_vector_type(4)));
};

template <typename T, int D>
__global__ __launch_bounds__(64 * kAppendWaves) void append_kernel(AppendArgs a) {
  using C = Chunk<T>;
  using vec = typename C::vec;
  constexpr int N = C::N, LANES = D / (2 * N), HEADS = 64 / LANES;   // lanes of a head, heads of a pass
  const int tid = threadIdx.x, lane = tid & 63;
  const int S = a.runs.count;
  if (blockIdx.x == gridDim.x - 1) {  // every sequence's entries, whether or not a row leads to them
    for (int s = tid; s < S; s += 64 * kAppendWaves) {
      int64_t f;
      int n, L;
      int code = rows_of(a.rows, s, f, n);
      if (code == SP_DEV_OK) code = tokens_of(a.runs, s, L);
      if (code == SP_DEV_OK && L < n) code = SP_DEV_BAD_OFFSETS;
      if (code != SP_DEV_OK) set_device_error(a.err, code);
    }
    return;
  }
  const int64_t wave = __builtin_amdgcn_readfirstlane((int)blockIdx.x * kAppendWaves + (tid >> 6));
  const int64_t row = wave / a.splits;
  const int split = (int)(wave - row * a.splits);
  if (row >= a.rows.rows) return;
  // this lane's chunks of a head
  const int j = lane % LANES, hsub = lane / LANES;
  const int turning = a.cos_sin ? a.rot_dim / (2 * N) : 0;          // lanes of a head that rotate
  const bool turns = j < turning;
  const int c0 = turns && !a.interleaved ? j : 2 * j;               // (turning lanes halve the rotation)
  const int c1 = turns && !a.interleaved ? j + turning : 2 * j + 1;
  const int Hq = a.Q ? a.shape.q_heads : 0, Hk = a.shape.kv_heads, H = Hq + 2 * Hk;
  const int h_end = min(H, (split + 1) * a.per_wave * HEADS);
  vec x0[kPasses], x1[kPasses];
  auto load = [&](int h0) {
#pragma unroll
    for (int u = 0; u < kPasses; ++u) {
      const int h = h0 + u * HEADS + hsub;
      if (h >= h_end) break;
      const T* src = h < Hq ? static_cast<const T*>(a.Q) + row * a.ldq + h * D
                     : h < Hq + Hk ? static_cast<const T*>(a.K) + row * a.ldk + (h - Hq) * D
                                   : static_cast<const T*>(a.V) + row * a.ldv + (h - Hq - Hk) * D;
      x0[u] = reinterpret_cast<const vec*>(src)[c0];
      x1[u] = reinterpret_cast<const vec*>(src)[c1];
    }
  };
  const int h_first = split * a.per_wave * HEADS;
  load(h_first);                      // on its way while the row's place is found

  // the row's sequence and slot
  int s;
  if (a.rows.padded) {
    if (a.rows.rows_per_seq == 0) return;
    const int64_t q = row / a.rows.rows_per_seq;
    if (q >= S) return;
    s = (int)q;
  } else {
    s = wave_find_last(S, row, [&](int i) { return (int64_t)a.rows.info[i]; });
  }
  int64_t first;
  int n, len;
  if (rows_of(a.rows, s, first, n) != SP_DEV_OK || row < first || row >= first + n) return;
  if (tokens_of(a.runs, s, len) != SP_DEV_OK || len < n) return;
  const int slot = len - n + (int)(row - first);
  const int page = a.runs.table[(int64_t)s * a.runs.width + (slot >> a.shape.page_shift)];
  if ((uint32_t)page >= (uint32_t)a.shape.pages) {
    if (lane == 0) set_device_error(a.err, SP_DEV_BAD_PAGE);
    return;
  }
  const int place = slot & ((1 << a.shape.page_shift) - 1);

  // the pairs' cosines and sines
  float cs[N], sn[N];
  if (a.cos_sin) {
    int at[3];
    at[0] = a.pos ? a.pos[row] : slot;
    at[1] = a.axes > 1 ? a.pos[a.rows.rows + row] : at[0];
    at[2] = a.axes > 2 ? a.pos[2 * a.rows.rows + row] : at[0];
#pragma unroll
    for (int x = 0; x < 3; ++x)
      if ((uint32_t)at[x] >= (uint32_t)a.positions) {               // uniform: the row is left out
        if (lane == 0) set_device_error(a.err, SP_DEV_BAD_POSITION);
        return;
      }
    if (turns) {
      const int pairs = a.rot_dim / 2;
      if (a.axes == 1) {
#pragma unroll
        for (int k = 0; k < N; k += 2) {
          const float4 u = *reinterpret_cast<const float4*>(a.cos_sin + 2 * ((int64_t)at[0] * pairs + N * j + k));
          cs[k] = u.x;
          sn[k] = u.y;
          cs[k + 1] = u.z;
          sn[k + 1] = u.w;
        }
      } else {
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const int p = N * j + k;
          const int64_t where = p < a.sec1 ? at[0] : p < a.sec2 ? at[1] : at[2];
          const float2 u = reinterpret_cast<const float2*>(a.cos_sin)[where * pairs + p];
          cs[k] = u.x;
          sn[k] = u.y;
        }
      }
    }
  }

  const int64_t page0 = ((int64_t)page * Hk << a.shape.page_shift) + place;   // in rows of D: head 0's
  for (int h0 = h_first; h0 < h_end; h0 += kPasses * HEADS) {
    if (h0 > h_first) load(h0);       // (Q_out may be Q: head by head the same lane's)
#pragma unroll
    for (int u = 0; u < kPasses; ++u) {
      const int h = h0 + u * HEADS + hsub;
      if (h >= h_end) break;
      if (turns && h < Hq + Hk) {
        if (a.interleaved) {
#pragma unroll
          for (int k = 0; k < N / 2; ++k) {
            const float p = (float)x0[u][2 * k], q = (float)x0[u][2 * k + 1];
            x0[u][2 * k] = (T)fmaf(p, cs[k], -(q * sn[k]));
            x0[u][2 * k + 1] = (T)fmaf(q, cs[k], p * sn[k]);
            const float r = (float)x1[u][2 * k], t = (float)x1[u][2 * k + 1];
            x1[u][2 * k] = (T)fmaf(r, cs[N / 2 + k], -(t * sn[N / 2 + k]));
            x1[u][2 * k + 1] = (T)fmaf(t, cs[N / 2 + k], r * sn[N / 2 + k]);
          }
        } else {
#pragma unroll
          for (int k = 0; k < N; ++k) {
            const float p = (float)x0[u][k], q = (float)x1[u][k];
            x0[u][k] = (T)fmaf(p, cs[k], -(q * sn[k]));
            x1[u][k] = (T)fmaf(q, cs[k], p * sn[k]);
          }
        }
      }
      T* dst;
      if (h < Hq) {
        dst = static_cast<T*>(a.Q_out) + (row * Hq + h) * D;
      } else {
        const int g = h - Hq < Hk ? h - Hq : h - Hq - Hk;
        dst = static_cast<T*>(h - Hq < Hk ? a.k_cache : a.v_cache) +
              (page0 + ((int64_t)g << a.shape.page_shift)) * D;
      }
      __builtin_nontemporal_store(x0[u], reinterpret_cast<vec*>(dst) + c0);
      __builtin_nontemporal_store(x1[u], reinterpret_cast<vec*>(dst) + c1);
    }
  }
}

template <typename T, int D>
void launch_append(AppendArgs& a, hipStream_t stream) {
  constexpr int HEADS = 64 / (D / (2 * Chunk<T>::N));
  const int H = (a.Q ? a.shape.q_heads : 0) + 2 * a.shape.kv_heads;
  const int passes = (H + HEADS - 1) / HEADS;
  // Few rows: a wave to every pass, so that a call's latency is one pass's.
  a.per_wave = 1;
  while (a.per_wave < passes && a.rows.rows * (passes / a.per_wave) > 4096) a.per_wave *= 2;
  a.splits = (passes + a.per_wave - 1) / a.per_wave;
  const int64_t waves = a.rows.rows * a.splits;
  hipLaunchKernelGGL((append_kernel<T, D>), dim3((unsigned)((waves + kAppendWaves - 1) / kAppendWaves + 1)),
                     dim3(64 * kAppendWaves), 0, stream, a);
}

}  // namespace

hipError_t launch_cache_append(AppendArgs a, hipStream_t stream) {
  if (a.rows.rows == 0 || a.runs.count == 0) return hipSuccess;
  const bool wide = a.shape.head_dim == 128;
  if (a.shape.dtype == SP_F32)
    wide ? launch_append<float, 128>(a, stream) : launch_append<float, 64>(a, stream);
  else
    wide ? launch_append<__bf16, 128>(a, stream) : launch_append<__bf16, 64>(a, stream);
  return hipGetLastError();
}

}  // namespace sp
