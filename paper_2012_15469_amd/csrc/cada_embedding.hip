// Embedding lookup with scaling, and its gradient by sorted tokens (cada_ops.h).
//
// The gradient sums, for each row of the table, the rows of dy whose token it is.  Positions are first sorted by token, equal ones in their own order, so that sums have
// one order and no float is added by an atomic: each workgroup owns a range of tokens, goes over all of them and puts down the positions of those in its range (k_sort).  The
// sorted positions are then taken in chunks of one length, however often a token occurs: a token's run that lies in one chunk is written to the table, the parts of one that
// crosses a chunk's border are joined by k_join.  Table rows without a token are cleared next to that.
#include <algorithm>

#include "cada_ops_internal.h"

namespace cada {
namespace {

struct Lookup {
  const void *tokens, *w;
  void *y;
  int64_t rows, vocab, ignore, ldw, ldy;
  int32_t width, token_bytes, lanes;
  float scale;
};

__device__ __forceinline__ int64_t token_at(const void *tokens, int bytes, int64_t i) {
  return bytes == 8 ? static_cast<const int64_t *>(tokens)[i] : (int64_t)static_cast<const int32_t *>(tokens)[i];
}

// Columns that a lane takes: pieces of 16 bytes, the last of which begins early enough to end with the row (its first columns are another lane's too, which writes the same).
// Rows of less than a piece go element by element.
template <typename T> __device__ __forceinline__ int first_column(int piece, int width) {
  constexpr int E = Elem<T>::kPer16;
  return max(0, min(piece * E, width - E));
}
template <typename T> __device__ __forceinline__ u32x4v load_piece(const T *p, int width) { return width >= Elem<T>::kPer16 ? load16(p) : load16_n(p, width); }
template <typename T> __device__ __forceinline__ void store_piece(T *p, int width, const float (&f)[Elem<T>::kPer16]) {
  if (width >= Elem<T>::kPer16) {
    store16(p, pack<T>(f));
  } else {
#pragma unroll
    for (int e = 0; e < Elem<T>::kPer16; ++e) if (e < width) p[e] = from_f32<T>(f[e]);
  }
}

// 2^lanes threads along a row, the others of 256 on further rows, four rows of a thread on their way at once.  Bound by memory: 32768 tokens with frequencies as in text, 2048 of 50001 in bf16, 33 us,
// 134 MB written at 4.1 TB/s and as much read, rows that occur often from caches.
constexpr int kLookupRows = 4;
template <typename T>
__global__ __launch_bounds__(256) void k_lookup(const Lookup a) {
  constexpr int E = Elem<T>::kPer16, U = kLookupRows;
  const int high = 256 >> a.lanes, piece = ((int)blockIdx.y << a.lanes) + (threadIdx.x & ((1 << a.lanes) - 1));
  if (piece * E >= a.width) return;
  const int c = first_column<T>(piece, a.width);
  for (int64_t r0 = (int64_t)blockIdx.x * high * U + (threadIdx.x >> a.lanes); r0 < a.rows; r0 += (int64_t)gridDim.x * high * U) {
    int64_t t[U];
    u32x4v raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) t[u] = token_at(a.tokens, a.token_bytes, min(r0 + u * high, a.rows - 1));
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool known = t[u] != a.ignore && t[u] >= 0 && t[u] < a.vocab;
      raw[u] = load_piece(static_cast<const T *>(a.w) + (known ? t[u] : 0) * a.ldw + c, a.width);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t r = r0 + u * high;
      if (r >= a.rows) break;
      const bool known = t[u] >= 0 && t[u] < a.vocab;
      float f[E];
      unpack<T>(raw[u], f);
#pragma unroll
      for (int e = 0; e < E; ++e) f[e] = t[u] == a.ignore ? 0.f : known ? f[e] * a.scale : __builtin_nanf("");
      store_piece(static_cast<T *>(a.y) + r * a.ldy + c, a.width, f);
    }
  }
}

// ---- gradient ----

struct Scatter {
  const void *tokens, *dy;
  void *dw;
  int32_t *start, *order, *key;        // [vocab + 1]; [rows] each, sorted
  float *part;                         // [chunks][2][width]: of the run that comes from the chunk before, and of the one that goes on in the next
  int64_t rows, lddy, lddw;
  uint32_t ignore32;                   // the ignored token, or one that is none
  int32_t vocab, width, token_bytes, lanes, join_lanes, range, chunk;      // range: tokens of a workgroup of k_sort; chunk: sorted positions of one of k_sums
  uint32_t chunk_blocks;
  float scale;
};

// A workgroup's tokens are [first, first + range).  Each of its sixteen wavefronts goes over a sixteenth of the positions and lists those of its tokens;
// smaller tokens outside the range are only counted.  It counts each of its tokens, and, when all have counted, puts their positions down behind those of the
// smaller tokens and of the wavefronts before it.  A wavefront whose list is full (tokens that are mostly of one range) goes over the positions behind those of
// its list again.  Every workgroup reads all tokens (from L2), so what counts is the operations per token: they are 32-bit numbers, of which those that add
// nothing are the largest, and 64 of them are skipped together where none is in the range.  Equal tokens of a batch are counted together, not by an atomic each
// (64 additions to one place in LDS are 64 turns).  32768 tokens of 50001: 13 us (37 with 64-bit comparisons and no lists); 100000 tokens of 27 values, with
// frequencies as in text, 30 (74 with lists of 1024, all of whose tokens were read again); 131072 of 30000 35.  The whole gradient of 80000 tokens of 27,
// evenly, in rows of 64 bf16 30 us; all of them one, which is one workgroup's list, 83.
constexpr int kSortThreads = 1024, kSortWaves = 16, kFewRange = 2048;
constexpr uint32_t kNoToken = ~0u;
template <typename W> __device__ __forceinline__ uint32_t token32(const W *tokens, uint32_t i, uint32_t ignore) {
  uint32_t k;
  if constexpr (sizeof(W) == 8) {
    const uint2 x = reinterpret_cast<const uint2 *>(tokens)[i];
    k = x.y ? kNoToken : x.x;
  } else {
    k = reinterpret_cast<const uint32_t *>(tokens)[i];
  }
  return k == ignore ? kNoToken : k;
}
template <typename W, int RANGE>
__global__ __launch_bounds__(kSortThreads) void k_sort(const Scatter a) {
  constexpr int U = 8;        // batches of 64 on their way at once
  constexpr int kList = RANGE <= 256 ? 2048 : RANGE <= 512 ? 1024 : 256, kKeyBits = 11;        // entries: position from the wavefront's first << kKeyBits | token from the range's first
  __shared__ int32_t count[kSortWaves][RANGE];
  __shared__ uint32_t list[kSortWaves][kList];
  __shared__ int32_t wave_sum[2][kSortWaves];
  static_assert(RANGE <= 1 << kKeyBits, "");
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const uint64_t lower = (1ull << lane) - 1;
  const uint32_t first = blockIdx.x * (uint32_t)a.range, range = min((uint32_t)a.range, (uint32_t)a.vocab - first);
  // (a wavefront's positions, from its first on: at most 2^26)
  const int64_t per = (a.rows + kSortWaves * 64 - 1) / (kSortWaves * 64) * 64, from = wave * per;
  const int mine = (int)max((int64_t)0, min(a.rows - from, per));
  const W *tokens = static_cast<const W *>(a.tokens) + from;
  for (int i = t; i < kSortWaves * RANGE; i += kSortThreads) (&count[0][0])[i] = 0;
  auto batches = [&](int i0, auto each) __attribute__((always_inline)) {        // each(position of the batch's first token, a lane's token), from the batch at i0 on
    for (; i0 + 64 * U <= mine; i0 += 64 * U) {
      uint32_t k[U];
#pragma unroll
      for (int u = 0; u < U; ++u) k[u] = token32(tokens, (uint32_t)(i0 + 64 * u + lane), a.ignore32);
#pragma unroll
      for (int u = 0; u < U; ++u) each(i0 + 64 * u, k[u]);
    }
    if (i0 < mine) {
      uint32_t k[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + 64 * u + lane;
        k[u] = token32(tokens, (uint32_t)min(i, mine - 1), a.ignore32);
        k[u] = i < mine ? k[u] : kNoToken;
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i0 + 64 * u < mine) each(i0 + 64 * u, k[u]);
    }
  };
  // (how many are of the range, of which so many are listed, all of those before position `rest`)
  int32_t below = 0, found = per <= 1 << (32 - kKeyBits) ? 0 : kList + 1, listed = 0, rest = 0;
  batches(0, [&](int i, uint32_t k) __attribute__((always_inline)) {
    below += __popcll(__ballot(k < first));
    const uint64_t in = __ballot(k - first < range);
    if (in) {
      const int32_t at = found;
      found += __popcll(in);
      if (found <= kList) {
        if (k - first < range) list[wave][at + __popcll(in & lower)] = (uint32_t)(i + lane) << kKeyBits | (k - first);
        listed = found;
        rest = i + 64;
      }
    }
  });
  if (found <= kList) rest = mine;
  // Calls each(position, token from the range's first or -1, the lanes that have the same one) for batches of mine.  Equal tokens are found by a ballot for
  // each of their bits, and a batch makes one trip to LDS, however many tokens it has.
  const int bits = 32 - __builtin_clz(max(range, 2u) - 1);
  auto tokens_of_mine = [&](auto each) __attribute__((always_inline)) {
    auto batch = [&](int i, int32_t k) __attribute__((always_inline)) {
      uint64_t same = __ballot(k >= 0);
      if (!same) return;
      for (int b = 0; b < bits; ++b) {
        const bool one = k >> b & 1;
        const uint64_t ones = __ballot(one);
        same &= one ? ones : ~ones;
      }
      each(i, k, same);
    };
    for (int e = 0; e < listed; e += 64) {
      const uint32_t x = list[wave][min(e + lane, kList - 1)];
      batch((int)(x >> kKeyBits), e + lane < listed ? (int32_t)(x & ((1u << kKeyBits) - 1)) : -1);
    }
    if (rest < mine) batches(rest, [&](int i, uint32_t k) __attribute__((always_inline)) { batch(i + lane, k - first < range ? (int32_t)(k - first) : -1); });
  };
  volatile int32_t *places = count[wave];
  __syncthreads();
  tokens_of_mine([&](int, int32_t k, uint64_t same) __attribute__((always_inline)) {
    if (k >= 0 && (same & lower) == 0) __hip_atomic_fetch_add(&count[wave][k], (int32_t)__popcll(same), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  });
  if (lane == 0) wave_sum[0][wave] = below;
  __syncthreads();
  below = 0;
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) below += wave_sum[0][w];
  // exclusive sums over the range's tokens, in turns of a token per thread
  int32_t base = below;
  for (int k0 = 0; k0 < RANGE; k0 += kSortThreads) {
    const int k = k0 + t;
    int32_t total = 0;
    if (k < RANGE) {
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) total += count[w][k];
    }
    int32_t sum = total;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int32_t other = __shfl_up(sum, o, 64);
      if (lane >= o) sum += other;
    }
    __syncthreads();
    if (lane == 63) wave_sum[1][wave] = sum;
    __syncthreads();
    int32_t before = base, all = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      before += w < wave ? wave_sum[1][w] : 0;
      all += wave_sum[1][w];
    }
    int32_t at = before + sum - total;
    if ((uint32_t)k < range) a.start[first + k] = at;
    if (k < RANGE) {
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) {
        const int32_t n = count[w][k];
        count[w][k] = at;
        at += n;
      }
    }
    base += all;
  }
  if (t == 0 && first + range == (uint32_t)a.vocab) a.start[a.vocab] = base;
  __syncthreads();
  tokens_of_mine([&](int i, int32_t k, uint64_t same) __attribute__((always_inline)) {
    if (k >= 0) {
      const int32_t base = places[k], at = base + __popcll(same & lower);
      a.order[at] = (int32_t)(from + i);
      a.key[at] = (int32_t)first + k;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      if ((same & lower) == 0) places[k] = base + (int32_t)__popcll(same);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  });
}

// Sums of a chunk of sorted positions, in their order: 2^lanes threads along a row, one piece each (blockIdx.y: which of a wide row's), eight rows on their way; and zeros for
// the table's rows that have none, by the workgroups behind the chunks'.  Bound by memory: 32768 x 2048 of 50001 in bf16, 339 MB in 74 us, 4.6 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void k_sums(const Scatter a) {
  constexpr int E = Elem<T>::kPer16, U = 8;
  const int high = 256 >> a.lanes, group = threadIdx.x >> a.lanes, piece = ((int)blockIdx.y << a.lanes) + (threadIdx.x & ((1 << a.lanes) - 1));
  if (piece * E >= a.width) return;
  const int col = first_column<T>(piece, a.width);
  T *dw = static_cast<T *>(a.dw) + col;
  if (blockIdx.x >= a.chunk_blocks) {
    const float zero[E] = {};
    const int64_t stride = (int64_t)(gridDim.x - a.chunk_blocks) * high;
#pragma unroll 4
    for (int64_t v = (int64_t)(blockIdx.x - a.chunk_blocks) * high + group; v < a.vocab; v += stride)
      if (a.start[v] == a.start[v + 1]) store_piece(dw + v * a.lddw, a.width, zero);
    return;
  }
  const int64_t c = (int64_t)blockIdx.x * high + group, n = a.start[a.vocab], lo = c * a.chunk, hi = min(n, lo + a.chunk);
  if (lo >= n) return;
  float acc[E] = {};
  int32_t now = a.key[lo];
  bool from_before = lo > 0 && a.key[lo - 1] == now;
  auto flush = [&](bool goes_on) __attribute__((always_inline)) {
    if (!from_before && !goes_on) {
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] *= a.scale;
      store_piece(dw + (int64_t)now * a.lddw, a.width, acc);
    } else {
      float *to = a.part + (2 * c + (from_before ? 0 : 1)) * a.width + col;
#pragma unroll
      for (int e = 0; e < E; ++e) if (e < a.width) to[e] = acc[e];
    }
  };
  for (int64_t j = lo; j < hi; j += U) {
    int32_t k[U], at[U];
    u32x4v raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = min(j + u, hi - 1);
      k[u] = a.key[i];
      at[u] = a.order[i];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = load_piece(static_cast<const T *>(a.dy) + (int64_t)at[u] * a.lddy + col, a.width);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (j + u >= hi) break;
      if (k[u] != now) {
        flush(false);
        from_before = false;
        now = k[u];
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = 0.f;
      }
      float f[E];
      unpack<T>(raw[u], f);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += f[e];
    }
  }
  flush(hi < n && a.key[hi] == now);
}

// Runs that cross borders: a wavefront at each border, which has something to do if it is its run's first.  It adds the run's parts up by itself, four columns
// per lane and 2^join_lanes lanes along a part, or leaves a run of many parts to its whole workgroup: a workgroup's sixteen borders are at most one such run's
// first (40735 tokens of 3527 with frequencies as in text, rows of 400 bf16, the longest run in hundreds of parts: 9.9 us, and 41 with a workgroup of four
// wavefronts at each border; 32768 of 50001 x 2048 7.0 and 13).  Bound by the trips to memory of a run's search and its parts.  No sum's order goes by time.
constexpr int kJoinWaves = 16, kLongRun = kJoinWaves + 1;        // a run of more parts crosses more borders than a workgroup has
template <typename T>
__global__ __launch_bounds__(64 * kJoinWaves) void k_join(const Scatter a) {
  __shared__ v4s sums[kJoinWaves][64];
  __shared__ int32_t long_token, long_parts;
  __shared__ int64_t long_border;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int along = 1 << a.join_lanes, turns = 64 >> a.join_lanes, turn = lane >> a.join_lanes, in_row = lane & (along - 1);
  const int64_t columns = (int64_t)gridDim.y * along * 4;
  // the sum of parts first, first + step, ...; then of the wavefront's turns
  auto sum_parts = [&](int64_t border, int32_t parts, int first, int step, int64_t c) __attribute__((always_inline)) {
    v4s s = {0.f, 0.f, 0.f, 0.f};
    if (c < a.width) {
#pragma unroll 8
      for (int i = first; i < parts; i += step) {        // of chunk border - 1 what goes on, of the others what comes from before
        const u32x4v x = load16_n(a.part + (2 * (border - 1 + i) + (i == 0 ? 1 : 0)) * a.width + c, a.width - c);
        s += __builtin_bit_cast(v4s, x);
      }
    }
    for (int o = along; o < 64; o <<= 1)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] += __shfl_xor(s[e], o, 64);
    return s;
  };
  if (t == 0) long_parts = 0;
  const int64_t b = (int64_t)blockIdx.x * kJoinWaves + wave + 1, at = b * a.chunk, i = min(at, a.rows - 1);
  const int32_t n = a.start[a.vocab], v = a.key[i], before = a.key[i - 1];        // (asked for together; behind the last position they are what was there)
  int32_t parts = 0;
  if (at < n && before == v) {
    const int32_t start = a.start[v], end = a.start[v + 1];
    if (start >= at - a.chunk) parts = (int32_t)((end - 1) / a.chunk - b + 2);
  }
  __syncthreads();
  if (parts > kLongRun) {
    if (lane == 0) {
      long_token = v;
      long_border = b;
      long_parts = parts;
    }
  } else if (parts > 0) {
    for (int64_t c0 = (int64_t)blockIdx.y * along * 4; c0 < a.width; c0 += columns) {
      const int64_t c = c0 + in_row * 4;
      const v4s s = sum_parts(b, parts, turn, turns, c);
      if (turn == 0) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (c + e < a.width) static_cast<T *>(a.dw)[(int64_t)v * a.lddw + c + e] = from_f32<T>(s[e] * a.scale);
      }
    }
  }
  __syncthreads();
  if (long_parts == 0) return;
  for (int64_t c0 = (int64_t)blockIdx.y * along * 4; c0 < a.width; c0 += columns) {
    const v4s s = sum_parts(long_border, long_parts, wave * turns + turn, kJoinWaves * turns, c0 + in_row * 4);
    if (turn == 0) sums[wave][in_row] = s;
    __syncthreads();
    if (t < along * 4 && c0 + t < a.width) {
      float x = sums[0][t >> 2][t & 3];
#pragma unroll
      for (int w = 1; w < kJoinWaves; ++w) x += sums[w][t >> 2][t & 3];
      static_cast<T *>(a.dw)[(int64_t)long_token * a.lddw + c0 + t] = from_f32<T>(x * a.scale);
    }
    __syncthreads();
  }
}

// Few positions, one per thread: a workgroup finds those of its range of tokens and sorts them in LDS (by counting, for each, the smaller ones).  2^lanes
// threads go along a row; the others of 1024 take other tokens' rows, or, of a token that occurs more than sixteen times, every so many sixteen of them, whose
// sums are joined in the groups' order.  One launch for three (us, that of the three in brackets: 400 tokens of 1001 x 301 float32 6.7 (12.2), with a token's
// frequency as in text 7.1 (14.1), all one token 25 (13); of 50001 x 1024 bf16 16.6 (23.2); 400 of 2 x 2048 bf16 21 (12)).
constexpr int kFewPositions = 512, kFewThreads = 1024;
template <typename T, typename W>
__global__ __launch_bounds__(kFewThreads) void k_few(const Scatter a) {
  constexpr int E = Elem<T>::kPer16, U = 16, kPosBits = 9, kWaves = kFewThreads / 64;
  __shared__ uint32_t listed[kFewPositions];
  __shared__ uint16_t position[kFewPositions], token[kFewPositions], long_at[kFewPositions / U], long_size[kFewPositions / U];
  __shared__ uint8_t size[kFewPositions], any[kFewRange];        // size: of the run that begins there, 0: none, or a long one
  __shared__ float sums[kFewThreads * E];
  __shared__ int waves[kWaves], n_long;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, rows = (int)a.rows;
  const uint32_t first = blockIdx.x * (uint32_t)a.range, range = min((uint32_t)a.range, (uint32_t)a.vocab - first);
  const uint32_t k = t < rows ? token32(static_cast<const W *>(a.tokens), (uint32_t)t, a.ignore32) : kNoToken;
  const bool in = k - first < range;
  const uint64_t mask = __ballot(in);
  if (lane == 0) waves[wave] = __popcll(mask);
  if (t < kFewPositions) size[t] = 0;
  if (t == 0) n_long = 0;
  for (int i = t; i < (int)range; i += kFewThreads) any[i] = 0;
  __syncthreads();
  int before = 0, n = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    before += w < wave ? waves[w] : 0;
    n += waves[w];
  }
  const uint32_t mine = (k - first) << kPosBits | t;
  if (in) {
    listed[before + __popcll(mask & ((1ull << lane) - 1))] = mine;
    any[k - first] = 1;
  }
  __syncthreads();
  if (in) {
    int at = 0, smaller_tokens = 0, equal = 0;
    for (int i = 0; i < n; ++i) {
      const uint32_t x = listed[i];
      at += x < mine;
      smaller_tokens += x >> kPosBits < k - first;
      equal += x >> kPosBits == k - first;
    }
    position[at] = (uint16_t)t;
    token[at] = (uint16_t)(k - first);
    if (at == smaller_tokens) {        // (its first)
      if (equal > U) {
        const int r = atomicAdd(&n_long, 1);        // (in which order they are worked on changes no sum)
        long_at[r] = (uint16_t)at;
        long_size[r] = (uint16_t)equal;
      } else {
        size[at] = (uint8_t)equal;
      }
    }
  }
  __syncthreads();
  const int high = kFewThreads >> a.lanes, group = t >> a.lanes, piece = ((int)blockIdx.y << a.lanes) + (t & ((1 << a.lanes) - 1));
  const bool here = piece * E < a.width;
  const int col = first_column<T>(piece, a.width);
  T *dw = static_cast<T *>(a.dw) + (int64_t)first * a.lddw + col;
  const T *dy = static_cast<const T *>(a.dy) + col;
  // up to sixteen rows from sorted position i on
  auto add = [&](float (&acc)[E], int i, int rows_here) __attribute__((always_inline)) {
    u32x4v raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      raw[u] = u32x4v{0, 0, 0, 0};
      if (u < rows_here) raw[u] = load_piece(dy + position[i + u] * a.lddy, a.width);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float f[E];
      unpack<T>(raw[u], f);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += f[e];
    }
  };
  if (here) {
    const float zero[E] = {};
    for (uint32_t v = group; v < range; v += high)
      if (!any[v]) store_piece(dw + v * a.lddw, a.width, zero);
    for (int i = group; i < n; i += high) {
      if (size[i] == 0) continue;
      float acc[E] = {};
      add(acc, i, size[i]);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] *= a.scale;
      store_piece(dw + token[i] * a.lddw, a.width, acc);
    }
  }
  for (int r = 0; r < n_long; ++r) {
    const int at = long_at[r], count = long_size[r];
    float acc[E] = {};
    if (here)
      for (int i = group * U; i < count; i += high * U) add(acc, at + i, min(U, count - i));
    __syncthreads();
#pragma unroll
    for (int e = 0; e < E; ++e) sums[e * kFewThreads + t] = acc[e];
    __syncthreads();
    if (here && group == 0) {
      for (int g = 1; g < high; ++g) {
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] += sums[e * kFewThreads + (g << a.lanes) + t];
      }
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] *= a.scale;
      store_piece(dw + token[at] * a.lddw, a.width, acc);
    }
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_clear(T *p, int64_t ld, int64_t rows, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * n; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / n;
    p[r * ld + (i - r * n)] = from_f32<T>(0.f);
  }
}

// ---- host ----
constexpr int64_t kMostVocab = 1 << 24, kMostRows = 1 << 30;

bool check_shape(int64_t rows, int64_t vocab, int64_t width, int type, int token_bytes, double scale) {
  if (rows < 0 || rows > kMostRows) { set_error("rows must be in [0, 2^30] (got %lld)", (long long)rows); return false; }
  if (vocab < 1 || vocab > kMostVocab) { set_error("vocab must be in [1, 2^24] (got %lld)", (long long)vocab); return false; }
  if (width < 1 || width > CADA_MAX_WIDTH) { set_error("width must be in [1, %d] (got %lld)", CADA_MAX_WIDTH, (long long)width); return false; }
  if (type != CADA_F32 && type != CADA_BF16) { set_error("type must be CADA_F32 or CADA_BF16 (got %d)", type); return false; }
  if (token_bytes != 4 && token_bytes != 8) { set_error("token_bytes must be 4 or 8 (got %d)", token_bytes); return false; }
  if (!((float)scale - (float)scale == 0.f)) { set_error("scale must be finite in float32"); return false; }
  return true;
}
bool check_tokens(const void *tokens, int bytes) {
  if (!tokens) { set_error("tokens is NULL"); return false; }
  if (reinterpret_cast<uintptr_t>(tokens) % bytes != 0) { set_error("tokens is not aligned to its elements"); return false; }
  return true;
}
// Threads along a row, as a power of two up to a workgroup.
int lanes_for(int64_t width, int per16) {
  int lanes = 0;
  while (lanes < 8 && ((int64_t)per16 << lanes) < width) ++lanes;
  return lanes;
}
unsigned slices(int64_t width, int per16, int lanes) { return (unsigned)ceil_div(width, (int64_t)per16 << lanes); }

struct ScatterPlan { bool few; int32_t range, chunk; int64_t chunks; size_t off_order, off_key, off_part, bytes; };
ScatterPlan plan_scatter(const cada_embedding_grad *a) {
  ScatterPlan p{};
  if (a->rows == 0) return p;
  p.few = a->rows <= std::min<int64_t>(kFewPositions, 128 * a->vocab);        // (long runs go through one workgroup)
  if (p.few) {        // (no more workgroups than find their tokens and clear their rows at once)
    p.range = (int32_t)std::min<int64_t>(kFewRange, ceil_div(a->vocab, 1024));
    return p;
  }
  // a workgroup's range of tokens: one for each CU, and no more than its counts have room for
  p.range = (int32_t)std::min<int64_t>(2048, ceil_div(a->vocab, 256));
  // chunks for a million lanes, where that leaves some rows to each and no run in too many parts
  const int64_t lanes = std::min<int64_t>(ceil_div(a->width, 16 / (int)type_bytes(a->type)), 1024);
  p.chunk = 8;
  while (p.chunk < 128 && (int64_t)p.chunk << 18 < a->rows * lanes) p.chunk *= 2;
  while (p.chunk < 128 && (int64_t)p.chunk << 13 < a->rows) p.chunk *= 2;
  p.chunks = ceil_div(a->rows, p.chunk);
  p.off_order = ops_align((size_t)(a->vocab + 1) * 4);
  p.off_key = p.off_order + ops_align((size_t)a->rows * 4);
  p.off_part = p.off_key + ops_align((size_t)a->rows * 4);
  p.bytes = p.off_part + (p.chunks > 1 ? ops_align((size_t)p.chunks * 2 * a->width * 4) : 0);
  return p;
}

template <typename T>
int lookup(const cada_embedding *a) {
  constexpr int E = Elem<T>::kPer16;
  Lookup l{};
  l.tokens = a->tokens; l.w = a->w; l.y = a->y; l.rows = a->rows; l.vocab = a->vocab; l.ignore = a->ignore_index; l.ldw = a->ldw; l.ldy = a->ldy;
  l.width = (int32_t)a->width; l.token_bytes = a->token_bytes; l.lanes = lanes_for(a->width, E); l.scale = (float)a->scale;
  const int64_t high = 256 >> l.lanes;
  const dim3 grid((unsigned)std::min<int64_t>(ceil_div(a->rows, high * kLookupRows), 1 << 20), slices(a->width, E, l.lanes));
  k_lookup<T><<<grid, 256, 0, static_cast<hipStream_t>(a->stream)>>>(l);
  return ops_launched("embedding");
}

template <typename T>
int scatter(const cada_embedding_grad *a, const ScatterPlan &p) {
  constexpr int E = Elem<T>::kPer16;
  hipStream_t st = static_cast<hipStream_t>(a->stream);
  if (a->rows == 0) {
    k_clear<T><<<(unsigned)std::min<int64_t>(ceil_div(a->vocab * a->width, 256), 1 << 16), 256, 0, st>>>(static_cast<T *>(a->dw), a->lddw, a->vocab, a->width);
    return ops_launched("embedding clear");
  }
  char *ws = static_cast<char *>(a->workspace);
  Scatter s{};
  s.tokens = a->tokens; s.dy = a->dy; s.dw = a->dw; s.rows = a->rows; s.ignore32 = a->ignore_index >= 0 && a->ignore_index < a->vocab ? (uint32_t)a->ignore_index : kNoToken; s.lddy = a->lddy; s.lddw = a->lddw;
  s.start = reinterpret_cast<int32_t *>(ws); s.order = reinterpret_cast<int32_t *>(ws + p.off_order); s.key = reinterpret_cast<int32_t *>(ws + p.off_key); s.part = reinterpret_cast<float *>(ws + p.off_part);
  s.vocab = (int32_t)a->vocab; s.width = (int32_t)a->width; s.token_bytes = a->token_bytes; s.lanes = lanes_for(a->width, E); s.join_lanes = std::min(6, lanes_for(a->width, 4)); s.range = p.range; s.chunk = p.chunk;
  s.scale = (float)a->scale;
  const unsigned groups = (unsigned)ceil_div(a->vocab, p.range);
  if (p.few) {
    const dim3 grid(groups, slices(a->width, E, s.lanes));
    if (a->token_bytes == 8) k_few<T, int64_t><<<grid, kFewThreads, 0, st>>>(s);
    else k_few<T, int32_t><<<grid, kFewThreads, 0, st>>>(s);
    return ops_launched("embedding gradient");
  }
  auto sort = [&](auto token) {
    typedef decltype(token) W;
    if (p.range <= 256) k_sort<W, 256><<<groups, kSortThreads, 0, st>>>(s);
    else if (p.range <= 512) k_sort<W, 512><<<groups, kSortThreads, 0, st>>>(s);
    else k_sort<W, 2048><<<groups, kSortThreads, 0, st>>>(s);
  };
  if (a->token_bytes == 8) sort((int64_t)0);
  else sort((int32_t)0);
  if (int rc = ops_launched("embedding sort")) return rc;
  const int64_t high = 256 >> s.lanes;
  s.chunk_blocks = (uint32_t)ceil_div(p.chunks, high);
  const unsigned fill = (unsigned)std::min<int64_t>(ceil_div(a->vocab, high * 4), 4096), across = slices(a->width, E, s.lanes);
  k_sums<T><<<dim3(s.chunk_blocks + fill, across), 256, 0, st>>>(s);
  if (int rc = ops_launched("embedding gradient")) return rc;
  if (p.chunks == 1) return CADA_OK;
  k_join<T><<<dim3((unsigned)ceil_div(p.chunks - 1, kJoinWaves), (unsigned)std::min<int64_t>(ceil_div(a->width, (int64_t)4 << s.join_lanes), 1024)), 64 * kJoinWaves, 0, st>>>(s);
  return ops_launched("embedding join");
}

}  // namespace
}  // namespace cada

using namespace cada;

extern "C" {

int cada_embedding_forward(const cada_embedding *a) {
  if (!a) { set_error("the arguments are NULL"); return CADA_EINVAL; }
  if (!check_shape(a->rows, a->vocab, a->width, a->type, a->token_bytes, a->scale)) return CADA_EINVAL;
  if (a->rows == 0) return CADA_OK;
  if (!check_tokens(a->tokens, a->token_bytes) || !ops_check_table("w", a->w, a->ldw, a->width, a->type) || !ops_check_table("y", a->y, a->ldy, a->width, a->type)) return CADA_EINVAL;
  const size_t elem = type_bytes(a->type);
  const Span y = span("y", a->y, a->rows, a->ldy, a->width, elem);
  if (!ops_apart(y, span("w", a->w, a->vocab, a->ldw, a->width, elem)) || !ops_apart(y, span("tokens", a->tokens, (size_t)a->rows * a->token_bytes))) return CADA_EINVAL;
  return a->type == CADA_BF16 ? lookup<bf16>(a) : lookup<float>(a);
}

int cada_embedding_backward_workspace(cada_embedding_grad *a) {
  if (!a) { set_error("the arguments are NULL"); return CADA_EINVAL; }
  if (!check_shape(a->rows, a->vocab, a->width, a->type, a->token_bytes, a->scale)) return CADA_EINVAL;
  a->workspace_bytes = plan_scatter(a).bytes;
  return CADA_OK;
}

int cada_embedding_backward(const cada_embedding_grad *a) {
  if (!a) { set_error("the arguments are NULL"); return CADA_EINVAL; }
  if (!check_shape(a->rows, a->vocab, a->width, a->type, a->token_bytes, a->scale)) return CADA_EINVAL;
  if (a->rows > 0 && (!check_tokens(a->tokens, a->token_bytes) || !ops_check_table("dy", a->dy, a->lddy, a->width, a->type))) return CADA_EINVAL;
  if (!ops_check_table("dw", a->dw, a->lddw, a->width, a->type)) return CADA_EINVAL;
  const ScatterPlan p = plan_scatter(a);
  if (int rc = ops_check_workspace(a->workspace, a->workspace_bytes, p.bytes)) return rc;
  const size_t elem = type_bytes(a->type);
  const Span dw = span("dw", a->dw, a->vocab, a->lddw, a->width, elem), dy = span("dy", a->rows ? a->dy : nullptr, a->rows, a->lddy, a->width, elem);
  const Span tokens = span("tokens", a->tokens, (size_t)a->rows * a->token_bytes), workspace = span("workspace", a->workspace, p.bytes);
  if (!ops_apart(dw, dy) || !ops_apart(dw, tokens) || !ops_apart(workspace, dw) || !ops_apart(workspace, dy) || !ops_apart(workspace, tokens)) return CADA_EINVAL;
  return a->type == CADA_BF16 ? scatter<bf16>(a, p) : scatter<float>(a, p);
}

}  // extern "C"
