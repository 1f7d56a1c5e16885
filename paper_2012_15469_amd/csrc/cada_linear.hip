// A layer's product with bias, activation and residual, and its gradients (cada_ops.h).
//
// Three products of two tables: y = x w (contraction over x's columns), dx = dz w^T (over dz's columns) and dw = x^T dz (over
// the rows of both).  A table is read either along the contraction ("kc": consecutive elements are consecutive
// contraction indices) or across it ("oc").  One tile kernel serves all of them: a workgroup of four or eight wavefronts takes a tile of
// BM x BN outputs and walks the contraction in steps of 128 bytes per row, the next one to three steps of both operands on their way into a ring in
// LDS while the matrix instructions (32x32x16 bf16, 32x32x2 f32; float32 accumulators) take this one.
#include <algorithm>
#include <cmath>
#include <cstdio>

#include "cada_linear_plan.h"
#include "cada_ops_internal.h"

namespace cada {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <typename T> constexpr int kStep = kStepBytes / (int)sizeof(T);

// What a finished sum goes through on its way out.
struct Epilogue {
  const void *bias, *residual;
  void *pre, *out;
  int64_t ldr, ldpre, ldo;
  int act;
};

// One product C[M, N] = sum_k A(m, k) B(k, n).
struct Product {
  const void *a, *b;
  int64_t lda, ldb, M, K;
  int64_t a_cols, b_cols;    // oc tables: columns that lie in memory (>= M, N), whole pieces where they are read directly
  int64_t k_per_split;       // a multiple of the step
  int32_t N, tiles_m, tiles_n, splits;
  float *partial;            // [splits][M][N up to whole groups of eight] where splits > 1: the sums are joined by k_join
  Epilogue epi;
  // small gradients: the operand that is the signal is read as dy, and dz = dy * act'(pre) is formed on its way into LDS
  const void *pre;
  int64_t ldpre;
  int32_t act;
  void *db;                  // column sums of dz (or null), by the tiles of the first rows; their parts where the contraction is split
  float *db_part;            // [splits][N]
};

// ---- operands in LDS ----
//
// A tile step of an operand is kStepBytes x (BM or BN) bytes, moved in pieces of 16 bytes; piece q lies at byte 16 q, and thread t
// of 256 moves the pieces 256 i + t, so that a wavefront fills consecutive kilobytes (what the LDS-direct load asks for).
//   kc: [outer][8 pieces]; row r keeps its pieces in the order p ^ (r / 2 % 8): a fragment read takes the same piece of 32 consecutive
//       rows, two of which lie 256 bytes apart as the 64 banks do, and in this order 16 consecutive rows cover the banks once.
//   oc: [k][outer]; bf16 rows keep their 32-byte chunks in the order c ^ swizzle(r): a transposing read takes 32 bytes of each of four
//       consecutive rows, which without it lie in the same banks.
template <typename T, bool KC, int BO, int TH> struct Side {
  static constexpr int E = Elem<T>::kPer16;
  static constexpr int kPieces = BO * 8 / TH;                   // per thread
  static constexpr int kRow16 = KC ? 8 : BO / E;                // pieces per row in LDS
  static constexpr int kBytes = kStepBytes * BO;
  __device__ static __forceinline__ int swizzle(int krow) { return sizeof(T) == 4 || BO < 64 ? 0 : BO >= 128 ? (krow & 3) << 1 : krow & 2; }
  // row of LDS and source piece in it of thread t's i-th piece
  __device__ static __forceinline__ void place(int i, int t, int &row, int &piece) {
    const int q = i * TH + t;
    row = q / kRow16;
    const int pos = q % kRow16;
    if constexpr (KC) piece = pos ^ ((row >> 1) & 7);
    else piece = pos ^ (swizzle(row) << 1);
  }
};

// The general way: through registers, any alignment, whatever lies outside [0, left) x [.., k_end) zero.  A piece is always one load and no branch (a branch
// per piece makes the compiler wait for one piece before it asks for the next): behind a row's end it reads the next row, and past the
// table's last element (`end`) the 16 bytes before that, so a table holds 16 bytes at least.  What does not belong to the row is masked, and what was read
// from before its place is shifted there, when the piece is put into LDS, a step or two later.
template <typename T, bool KC, int BO, int TH>
__device__ __forceinline__ void piece_offsets(uint32_t (&off)[BO * 8 / TH], int64_t ld, int t) {
  typedef Side<T, KC, BO, TH> S;
#pragma unroll
  for (int i = 0; i < S::kPieces; ++i) {
    int row, piece;
    S::place(i, t, row, piece);
    off[i] = (uint32_t)(((int64_t)row * ld + piece * S::E) * (int64_t)sizeof(T));
  }
}
template <typename T, int N>
__device__ __forceinline__ void fetch(u32x4v (&reg)[N], const T *src, const uint32_t (&off)[N], const T *end) {
  const T *last = end - Elem<T>::kPer16, *base = src < last ? src : last;
  const uint32_t most = (uint32_t)min((int64_t)0xFFFFFFF0, (last - base) * (int64_t)sizeof(T));
#pragma unroll
  for (int i = 0; i < N; ++i) reg[i] = load16(reinterpret_cast<const T *>(reinterpret_cast<const unsigned char *>(base) + min(off[i], most)));
}
template <typename T, bool KC, int BO, int TH>
__device__ __forceinline__ void mask(u32x4v (&reg)[BO * 8 / TH], const T *src, int64_t ld, const T *end, int left, int k_left, int t) {
  typedef Side<T, KC, BO, TH> S;
  if (left >= BO && k_left >= kStep<T>) return;
#pragma unroll
  for (int i = 0; i < S::kPieces; ++i) {
    int row, piece;
    S::place(i, t, row, piece);
    const int along = (KC ? row < left : row < k_left) ? (KC ? k_left : left) - piece * S::E : 0;        // elements of the piece that exist
    const int64_t over = src + (int64_t)row * ld + piece * S::E + S::E - end;
    if (along > 0 && over > 0) {
      const int bits = (int)over * 8 * (int)sizeof(T);        // < 128, as the piece's first element exists
      uint64_t lo = (uint64_t)reg[i][1] << 32 | reg[i][0], hi = (uint64_t)reg[i][3] << 32 | reg[i][2];
      if (bits >= 64) { lo = hi >> (bits - 64); hi = 0; }
      else { lo = lo >> bits | hi << (64 - bits); hi >>= bits; }
      reg[i] = u32x4v{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
    }
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      if constexpr (S::E == 8) reg[i][d] &= along >= 2 * d + 2 ? 0xFFFFFFFFu : along == 2 * d + 1 ? 0xFFFFu : 0u;
      else reg[i][d] = along > d ? reg[i][d] : 0u;
    }
  }
}
// The same for a whole step that no piece leaves the table in: rows (kc) or columns (oc) beyond the table, which are the same ones in every step.
template <typename T, bool KC, int BO, int TH> struct Edge {
  typedef Side<T, KC, BO, TH> S;
  uint32_t keep[KC ? S::kPieces : 4];
  __device__ __forceinline__ Edge(int left, int t) {
    int row, piece;
    if constexpr (KC) {
#pragma unroll
      for (int i = 0; i < S::kPieces; ++i) {
        S::place(i, t, row, piece);
        keep[i] = row < left ? 0xFFFFFFFFu : 0u;
      }
    } else {
      S::place(0, t, row, piece);        // (a thread's pieces are the same columns of different rows)
      const int along = left - piece * S::E;
#pragma unroll
      for (int d = 0; d < 4; ++d) keep[d] = S::E == 8 ? (along >= 2 * d + 2 ? 0xFFFFFFFFu : along == 2 * d + 1 ? 0xFFFFu : 0u) : along > d ? 0xFFFFFFFFu : 0u;
    }
  }
  __device__ __forceinline__ void cut(u32x4v (&reg)[S::kPieces]) const {
#pragma unroll
    for (int i = 0; i < S::kPieces; ++i)
#pragma unroll
      for (int d = 0; d < 4; ++d) reg[i][d] &= keep[KC ? i : d];
  }
};
// dz = dy * act'(pre) in place of dy, and its sums per element of a piece (the pieces of a thread of an oc table are the same columns of different rows).
template <typename T, int N>
__device__ __forceinline__ void signal(u32x4v (&dy)[N], const u32x4v (&pre)[N], int act, float (&sum)[Elem<T>::kPer16]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float f[Elem<T>::kPer16], z[Elem<T>::kPer16];
    unpack<T>(dy[i], f);
    if (act != CADA_ACT_NONE) {
      unpack<T>(pre[i], z);
#pragma unroll
      for (int e = 0; e < Elem<T>::kPer16; ++e) f[e] *= activation_slope<T>(z[e], act);
      dy[i] = pack<T>(f);
    }
#pragma unroll
    for (int e = 0; e < Elem<T>::kPer16; ++e) sum[e] += f[e];
  }
}
template <int N, int TH>
__device__ __forceinline__ void put(unsigned char *lds, const u32x4v (&reg)[N], int t) {
#pragma unroll
  for (int i = 0; i < N; ++i) *reinterpret_cast<u32x4v *>(lds + (i * TH + t) * 16) = reg[i];
}

// The direct way: LDS-direct loads of a whole step.  Every row starts on a 16-byte boundary, and pieces lie in memory whole or not at
// all (kc: a step's are all there); one that does not is read from the last row or piece that does and enters outputs that nobody stores.
template <typename T, bool KC, int BO, int TH>
__device__ __forceinline__ void direct_offsets(uint32_t (&off)[BO * 8 / TH], int64_t ld, int64_t left, int t) {
  typedef Side<T, KC, BO, TH> S;
#pragma unroll
  for (int i = 0; i < S::kPieces; ++i) {
    int row, piece;
    S::place(i, t, row, piece);
    const int64_t at = KC ? min((int64_t)row, left - 1) * ld + piece * S::E : (int64_t)row * ld + min((int64_t)piece * S::E, left - S::E);
    off[i] = (uint32_t)(at * (int64_t)sizeof(T));
  }
}
// One kilobyte per wavefront: 16 bytes per lane to consecutive places.  (In assembly: for the builtin the compiler waits for the loads before
// the next read of LDS, whatever it reads, and the loop is as slow as their latency; here the wait is the one at the step's end.)
__device__ __forceinline__ void direct_kilobyte(uint32_t lds, const void *base, uint32_t off) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(__builtin_amdgcn_readfirstlane(lds)) : "memory", "m0");
}
// The same pointer in scalar registers (it is the same in every lane, which the compiler cannot always see).
template <typename P> __device__ __forceinline__ const P *uniform(const P *p) {
  const uint64_t x = reinterpret_cast<uint64_t>(p);
  return reinterpret_cast<const P *>((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x) | (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(x >> 32)) << 32);
}
template <int N, int TH>
__device__ __forceinline__ void direct(const unsigned char *lds, const void *src, const uint32_t (&off)[N], int wave) {
  const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const unsigned char *)lds + wave * 1024;
  const void *base = uniform(static_cast<const unsigned char *>(src));
#pragma unroll
  for (int i = 0; i < N; ++i) direct_kilobyte(at + i * (TH * 16), base, off[i]);
}
// What this wavefront has asked for, but for the last N loads, has arrived, in registers and in LDS; then so for the others.
template <int N> __device__ __forceinline__ void landed() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory"); }

// ---- fragments ----
// Sub-step ks of four: lane l holds outer index l % 32; bf16: 8 contraction indices from 16 ks + 8 (l / 32) on; float32: 4 from 8 ks + 4 (l / 32) on, one
// for each of four matrix instructions (both operands in the same order, so the sum is complete).
template <bool KC, int BO>
__device__ __forceinline__ bf16x8 fragment(const unsigned char *lds, int outer, int ks, int lane, bf16) {
  if constexpr (KC) {
    const int row = outer + (lane & 31), piece = ks * 2 + (lane >> 5);
    return *reinterpret_cast<const bf16x8 *>(lds + row * kStepBytes + ((piece ^ ((row >> 1) & 7)) << 4));
  } else {
    // ds_read_b64_tr_b16 works on groups of 16 lanes: source lane s of a group passes the address of four consecutive units of row s / 4, and lane
    // l receives unit l of rows 0..3.  The groups are (units 0-15 | 16-31) x (rows 0-7 | 8-15 of the sub-step), two reads of four rows each.
    const int krow = ks * 16 + ((lane >> 5) << 3) + ((lane & 15) >> 2), chunk = (outer >> 4) + ((lane >> 4) & 1);
    const unsigned char *at = lds + krow * (BO * 2) + ((chunk ^ Side<bf16, false, BO, 256>::swizzle(krow)) << 5) + ((lane & 3) << 3);
    typedef __attribute__((address_space(3))) i16x4 *lds_p;
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_p)(at)), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_p)(at + 4 * BO * 2));
    return __builtin_bit_cast(bf16x8, (i16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
}
template <bool KC, int BO>
__device__ __forceinline__ v4s fragment(const unsigned char *lds, int outer, int ks, int lane, float) {
  if constexpr (KC) {
    const int row = outer + (lane & 31), piece = ks * 2 + (lane >> 5);
    return *reinterpret_cast<const v4s *>(lds + row * kStepBytes + ((piece ^ ((row >> 1) & 7)) << 4));
  } else {
    const float *at = reinterpret_cast<const float *>(lds) + (ks * 8 + ((lane >> 5) << 2)) * BO + outer + (lane & 31);
    return v4s{at[0], at[BO], at[2 * BO], at[3 * BO]};
  }
}
__device__ __forceinline__ f32x16 multiply(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 multiply(v4s a, v4s b, f32x16 c) {
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
  return c;
}

// Eight consecutive columns n .. of row m of a finished sum; `left` of them exist.
template <typename T>
__device__ __forceinline__ void finish8(const Epilogue &e, int64_t m, int n, int64_t left, float (&f)[8]) {
  if (left <= 0) return;
  float o[8];
  if (e.bias) {
    load8_n(static_cast<const T *>(e.bias) + n, left, o);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] += o[i];
  }
  if (e.pre) store8_n(static_cast<T *>(e.pre) + m * e.ldpre + n, left, f);
  if (e.act != CADA_ACT_NONE) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = activation<T>(f[i], e.act);
  }
  if (e.residual) {
    load8_n(static_cast<const T *>(e.residual) + m * e.ldr + n, left, o);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] += o[i];
  }
  store8_n(static_cast<T *>(e.out) + m * e.ldo + n, left, f);
}

// WY x WX wavefronts share the tile; with KW = 4 four wavefronts each take the whole (32 x 32) tile and one of the four sub-steps of every step, and their sums are joined
// on the way out: short steps for few outputs.
enum { NO_SIGNAL = 0, A_SIGNAL = 1, B_SIGNAL = 2 };
template <typename T, int BM, int BN, int WY, int WX, bool AKC, bool BKC, bool DIRECT, int STAGES, int KW = 1, int SIGNAL = NO_SIGNAL>
__device__ __forceinline__ void tile_product(const Product &p, uint32_t tile, unsigned char *lds) {
  constexpr int TH = 64 * WY * WX * KW, NK = 4 / KW;
  typedef Side<T, AKC, BM, TH> SA;
  typedef Side<T, BKC, BN, TH> SB;
  constexpr int WM = BM / WY, WN = BN / WX, FM = WM / 32, FN = WN / 32, kHalf = SA::kBytes + SB::kBytes, BK = kStep<T>;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int place = wave % (WY * WX), kw = wave / (WY * WX), wm = place / WX * WM, wn = place % WX * WN;
  // Tiles in bands of eight rows of tiles, columns slowest in a band: the tiles that run together share operands.
  const uint32_t per_split = (uint32_t)p.tiles_m * p.tiles_n, band_tiles = 8u * p.tiles_n;
  const uint32_t split = tile / per_split, r = tile - split * per_split, band = r / band_tiles, in_band = r - band * band_tiles;
  const uint32_t rows_here = min(8u, (uint32_t)p.tiles_m - band * 8), col = in_band / rows_here;
  const int64_t m0 = (int64_t)(band * 8 + in_band - col * rows_here) * BM, m_left = p.M - m0;
  const int n0 = (int)col * BN;
  const int64_t n_left = p.N - n0, k0 = split * p.k_per_split, k1 = min(p.K, k0 + p.k_per_split);
  const T *a = static_cast<const T *>(p.a) + (AKC ? m0 * p.lda + k0 : k0 * p.lda + m0);
  const T *b = static_cast<const T *>(p.b) + (BKC ? n0 * p.ldb + k0 : k0 * p.ldb + n0);
  // (one past the tables' last elements)
  const T *a_end = static_cast<const T *>(p.a) + (AKC ? (p.M - 1) * p.lda + p.K : (p.K - 1) * p.lda + p.M);
  const T *b_end = static_cast<const T *>(p.b) + (BKC ? ((int64_t)p.N - 1) * p.ldb + p.K : (p.K - 1) * p.ldb + p.N);
  const int64_t a_step = AKC ? BK : BK * p.lda, b_step = BKC ? BK : BK * p.ldb;
  const int steps = (int)((k1 - k0 + BK - 1) / BK), whole = (int)((k1 - k0) / BK);

  uint32_t oa[SA::kPieces], ob[SB::kPieces], op[SIGNAL == A_SIGNAL ? SA::kPieces : SIGNAL == B_SIGNAL ? SB::kPieces : 1];
  if constexpr (DIRECT) {
    direct_offsets<T, AKC, BM, TH>(oa, p.lda, AKC ? m_left : p.a_cols - m0, t);
    direct_offsets<T, BKC, BN, TH>(ob, p.ldb, BKC ? n_left : p.b_cols - n0, t);
  } else {
    piece_offsets<T, AKC, BM, TH>(oa, p.lda, t);
    piece_offsets<T, BKC, BN, TH>(ob, p.ldb, t);
  }
  // The way through registers: asked for early, put into LDS where the step before has been read.
  struct Pieces { u32x4v a[SA::kPieces], b[SB::kPieces], pre[SIGNAL == A_SIGNAL ? SA::kPieces : SIGNAL == B_SIGNAL ? SB::kPieces : 1]; };
  float column_sum[Elem<T>::kPer16] = {};
  const int m_in = (int)min(m_left, (int64_t)BM), n_in = (int)min(n_left, (int64_t)BN);
  auto k_in = [&](int s) __attribute__((always_inline)) { return (int)min(k1 - k0 - (int64_t)s * BK, (int64_t)BK); };
  // (without an activation there is no pre: the signal itself is read again, and not used, rather than a branch among the loads)
  const bool no_act = SIGNAL == NO_SIGNAL || p.act == CADA_ACT_NONE;
  const int64_t ldpre = no_act ? (SIGNAL == A_SIGNAL ? p.lda : p.ldb) : p.ldpre;
  const T *pre = static_cast<const T *>(no_act ? (SIGNAL == A_SIGNAL ? p.a : p.b) : p.pre), *pre_end = pre;
  if constexpr (SIGNAL != NO_SIGNAL) {
    pre_end += SIGNAL == A_SIGNAL ? (p.M - 1) * ldpre + p.K : (p.K - 1) * ldpre + p.N;
    pre += SIGNAL == A_SIGNAL ? m0 * ldpre + k0 : k0 * ldpre + n0;
  }
  const int64_t pre_step = SIGNAL == A_SIGNAL ? BK : BK * ldpre;
  if constexpr (SIGNAL == A_SIGNAL) piece_offsets<T, AKC, BM, TH>(op, ldpre, t);
  if constexpr (SIGNAL == B_SIGNAL) piece_offsets<T, BKC, BN, TH>(op, ldpre, t);
  auto ask = [&](Pieces &r, int s) __attribute__((always_inline)) {
    fetch(r.a, a + s * a_step, oa, a_end);
    fetch(r.b, b + s * b_step, ob, b_end);
    if constexpr (SIGNAL != NO_SIGNAL) fetch(r.pre, pre + s * pre_step, op, pre_end);
  };
  // Rows of a table that is read across the contraction whose pieces may pass the table's last element, where fetch takes the 16 bytes before that and only mask() shifts them to their
  // place: the last one, and as many as a piece of a narrow table reaches over.  Tables read along the contraction meet their ends in its last step.
  const int64_t whole_piece = SB::E;
  const int narrowest = (int)min(min(AKC ? whole_piece : p.lda, BKC ? whole_piece : p.ldb), min(SIGNAL == B_SIGNAL ? ldpre : whole_piece, whole_piece));
  const int64_t k_inner = p.K - (SB::E - 2 + narrowest) / narrowest;
  const Edge<T, AKC, BM, TH> a_edge(m_in, t);
  const Edge<T, BKC, BN, TH> b_edge(n_in, t);
  auto put_step = [&](Pieces &r, int s, unsigned char *dst) __attribute__((always_inline)) {
    const int k = k_in(s);
    if (DIRECT || k0 + (int64_t)(s + 1) * BK > k_inner) {        // (the contraction's last step, which may end inside, and steps that read up to the tables' ends)
      mask<T, AKC, BM, TH>(r.a, a + s * a_step, p.lda, a_end, m_in, k, t);
      mask<T, BKC, BN, TH>(r.b, b + s * b_step, p.ldb, b_end, n_in, k, t);
      if constexpr (SIGNAL == A_SIGNAL) mask<T, AKC, BM, TH>(r.pre, pre + s * pre_step, ldpre, pre_end, m_in, k, t);
      if constexpr (SIGNAL == B_SIGNAL) mask<T, BKC, BN, TH>(r.pre, pre + s * pre_step, ldpre, pre_end, n_in, k, t);
    } else {
      if (m_in < BM) {
        a_edge.cut(r.a);
        if constexpr (SIGNAL == A_SIGNAL) a_edge.cut(r.pre);
      }
      if (n_in < BN) {
        b_edge.cut(r.b);
        if constexpr (SIGNAL == B_SIGNAL) b_edge.cut(r.pre);
      }
    }
    if constexpr (SIGNAL == A_SIGNAL) signal<T>(r.a, r.pre, p.act, column_sum);
    if constexpr (SIGNAL == B_SIGNAL) signal<T>(r.b, r.pre, p.act, column_sum);
    put<SA::kPieces, TH>(dst, r.a, t);
    put<SB::kPieces, TH>(dst + SA::kBytes, r.b, t);
  };
  auto load_step = [&](int s, unsigned char *dst) __attribute__((always_inline)) {
    direct<SA::kPieces, TH>(dst, a + s * a_step, oa, wave);
    direct<SB::kPieces, TH>(dst + SA::kBytes, b + s * b_step, ob, wave);
  };

  f32x16 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;

  typedef decltype(fragment<AKC, BM>(lds, 0, 0, 0, T())) Frag;
  auto read_fragments = [&](Frag (&fa)[FM], Frag (&fb)[FN], const unsigned char *src, int ks) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < FM; ++i) fa[i] = fragment<AKC, BM>(src, wm + 32 * i, ks * KW + kw, lane, T());
#pragma unroll
    for (int j = 0; j < FN; ++j) fb[j] = fragment<BKC, BN>(src + SA::kBytes, wn + 32 * j, ks * KW + kw, lane, T());
  };
  // (lane: row l % 32 of the tile, four consecutive columns at a time)
  auto multiply_all = [&](const Frag (&fa)[FM], const Frag (&fb)[FN]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = multiply(fb[j], fa[i], acc[i][j]);
  };
  Frag fa[2][FM], fb[2][FN];
  Pieces reg[2];
  auto whole_step = [&](const unsigned char *src) __attribute__((always_inline)) {
    read_fragments(fa[0], fb[0], src, 0);
#pragma unroll
    for (int ks = 0; ks < NK; ++ks) {
      if (ks < NK - 1) read_fragments(fa[(ks + 1) & 1], fb[(ks + 1) & 1], src, ks + 1);
      __builtin_amdgcn_sched_barrier(0);
      multiply_all(fa[ks & 1], fb[ks & 1]);
    }
  };
  // The last sub-step of a step, when the next step can be read: its first fragments on their way, then the products.
  auto last_of_step = [&](const unsigned char *there) __attribute__((always_inline)) {
    constexpr int next = NK == 1 ? 1 : 0;
    read_fragments(fa[next], fb[next], there, 0);
    __builtin_amdgcn_sched_barrier(0);
    multiply_all(fa[(NK - 1) & 1], fb[(NK - 1) & 1]);
    if constexpr (NK == 1) {
      fa[0][0] = fa[1][0];
      fb[0][0] = fb[1][0];
    }
  };
  if constexpr (DIRECT) {
    // Whole steps; what is left of the contraction comes through registers behind them, asked for first where the tile leaves registers for it.
    constexpr bool kEarly = BM < 256;
    auto ask_tail = [&]() __attribute__((always_inline)) {
      uint32_t ta[SA::kPieces], tb[SB::kPieces];
      piece_offsets<T, AKC, BM, TH>(ta, p.lda, t);
      piece_offsets<T, BKC, BN, TH>(tb, p.ldb, t);
      fetch(reg[0].a, a + whole * a_step, ta, a_end);
      fetch(reg[0].b, b + whole * b_step, tb, b_end);
    };
    if (whole > 0) {
      constexpr int P = SA::kPieces + SB::kPieces;
#pragma unroll
      for (int q = 0; q < STAGES; ++q) {
        if (q < whole) load_step(q, lds + q * kHalf);
        if (q == 0 && kEarly && whole < steps) ask_tail();
      }
      if (whole >= STAGES) landed<(STAGES - 1) * P>();
      else landed<0>();
      read_fragments(fa[0], fb[0], lds, 0);
      for (int s = 0; s < whole; ++s) {
        unsigned char *here = lds + (s & (STAGES - 1)) * kHalf, *there = lds + ((s + 1) & (STAGES - 1)) * kHalf;
#pragma unroll
        for (int ks = 0; ks < NK - 1; ++ks) {
          read_fragments(fa[(ks + 1) & 1], fb[(ks + 1) & 1], here, ks + 1);
          __builtin_amdgcn_sched_barrier(0);        // (the reads of the next sub-step go out before this one's products, not between them)
          multiply_all(fa[ks & 1], fb[ks & 1]);
        }
        // the next step is there, and everybody has read this one
        if (STAGES > 2 && s + STAGES - 1 < whole) landed<(STAGES - 2) * P>();
        else landed<0>();
        if (s + STAGES < whole) load_step(s + STAGES, here);
        last_of_step(there);        // (past the last step: fragments that nobody uses)
      }
    }
    if (whole < steps) {
      if (!kEarly || whole == 0) ask_tail();
      __syncthreads();
      put_step(reg[0], whole, lds);
      __syncthreads();
      whole_step(lds);
    }
  } else {
    // Two steps ahead in registers (asked for also where there is no such step: the loads are in bounds, and a branch around them would be waited at); the next
    // step is put into LDS between this one's products.
    ask(reg[0], 0);
    if (steps > 1) ask(reg[1], 1);
    put_step(reg[0], 0, lds);
    lds_sync();
    read_fragments(fa[0], fb[0], lds, 0);
    auto one = [&](Pieces &next, Pieces &after, int s) __attribute__((always_inline)) {
      unsigned char *here = lds + (s & 1) * kHalf, *there = lds + ((s + 1) & 1) * kHalf;
      if (steps > 1) ask(after, s + 2);
#pragma unroll
      for (int ks = 0; ks < NK - 1; ++ks) {
        read_fragments(fa[(ks + 1) & 1], fb[(ks + 1) & 1], here, ks + 1);
        __builtin_amdgcn_sched_barrier(0);
        multiply_all(fa[ks & 1], fb[ks & 1]);
        if (ks == 1 && s + 1 < steps) put_step(next, s + 1, there);
      }
      if (NK == 1 && s + 1 < steps) put_step(next, s + 1, there);
      lds_sync();
      last_of_step(there);
    };
    for (int s = 0; s < steps; s += 2) {
      one(reg[1], reg[0], s);
      if (s + 1 < steps) one(reg[0], reg[1], s + 1);
    }
  }
  __syncthreads();

  if constexpr (SIGNAL == B_SIGNAL) {
    if (p.db && m0 == 0) {
      // threads t % (pieces of a row) hold the same columns (a thread's piece is that of its first row: rows of its others differ by multiples of four)
      constexpr int E = Elem<T>::kPer16, kRow16 = SB::kRow16, kLanes = TH / kRow16;
      static_assert(TH / kRow16 % 4 == 0 && kLanes * BN * 4 <= 2 * kHalf, "");
      float *part = reinterpret_cast<float *>(lds);
      int row, piece;
      SB::place(0, t, row, piece);
#pragma unroll
      for (int e = 0; e < E; ++e) part[t / kRow16 * BN + piece * E + e] = column_sum[e];
      __syncthreads();
      if (t < BN && n0 + t < p.N) {
        float x = 0.f;
        for (int i = 0; i < kLanes; ++i) x += part[i * BN + t];
        if (p.splits > 1) p.db_part[(int64_t)split * p.N + n0 + t] = x;
        else static_cast<T *>(p.db)[n0 + t] = from_f32<T>(x);
      }
      __syncthreads();
    }
  }

  if constexpr (KW > 1) {
    // The wavefronts' sums side by side in LDS; four lanes for each row join them.
    static_assert(FM == 1 && FN == 1 && BM == 32 && BN == 32 && KW == 4, "");
    constexpr int kLd = BN + 4;
    float *sums = reinterpret_cast<float *>(lds), *mine = sums + kw * BM * kLd + (lane & 31) * kLd + 4 * (lane >> 5);
#pragma unroll
    for (int q = 0; q < 4; ++q) *reinterpret_cast<v4s *>(mine + 8 * q) = v4s{acc[0][0][4 * q], acc[0][0][4 * q + 1], acc[0][0][4 * q + 2], acc[0][0][4 * q + 3]};
    __syncthreads();
    if (t < BM * 4 && m0 + t / 4 < p.M) {
      const float *src = sums + t / 4 * kLd + (t & 3) * 8;
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = (src[e] + src[BM * kLd + e]) + (src[2 * BM * kLd + e] + src[3 * BM * kLd + e]);
      const int64_t m = m0 + t / 4, left = (int64_t)p.N - n0 - (t & 3) * 8;
      const int n = n0 + (t & 3) * 8;
      if (p.splits > 1) store8_n(p.partial + ((int64_t)split * p.M + m) * eights(p.N) + n, left > 0 ? 8 : 0, f);
      else finish8<T>(p.epi, m, n, left, f);
    }
    return;
  }

  // Out through LDS, 32 rows of the wavefront's tile at a time, so that memory is met in eight consecutive columns per lane.  (One copy of the code
  // behind it: with one for every group of rows a 256 x 256 tile spent 8 us fetching instructions.)
  constexpr int kLd = WN + 4, kLanes = WN / 8, kRows = 64 / kLanes;
  static_assert(KW > 1 || WY * WX * 32 * kLd * 4 <= 2 * kHalf, "the wavefronts' strips fit the operands' LDS");
  float *strip = reinterpret_cast<float *>(lds) + wave * 32 * kLd;
  const int n = n0 + wn + lane % kLanes * 8;
  const int64_t left = (int64_t)p.N - n;
#pragma unroll 1
  for (int i = 0; i < FM; ++i) {
#pragma unroll
    for (int ii = 0; ii < FM; ++ii) {
      if (ii == i) {
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            *reinterpret_cast<v4s *>(strip + (lane & 31) * kLd + 32 * j + 8 * q + 4 * (lane >> 5)) = v4s{acc[ii][j][4 * q], acc[ii][j][4 * q + 1], acc[ii][j][4 * q + 2], acc[ii][j][4 * q + 3]};
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 2
    for (int row = lane / kLanes; row < 32; row += kRows) {
      const int64_t m = m0 + wm + 32 * i + row;
      const float *src = strip + row * kLd + lane % kLanes * 8;
      const v4s x = *reinterpret_cast<const v4s *>(src), y = *reinterpret_cast<const v4s *>(src + 4);
      float f[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
      if (m < p.M) {
        if (p.splits > 1) store8_n(p.partial + ((int64_t)split * p.M + m) * eights(p.N) + n, left > 0 ? 8 : 0, f);
        else finish8<T>(p.epi, m, n, left, f);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// Tiles of a launch, dealt to the eight XCDs in consecutive eighths (each has an L2 of its own).  `first`: workgroups of an XCD that have other tiles.
__device__ __forceinline__ uint32_t tile_of_block(uint32_t total, uint32_t first = 0) {
  const uint32_t per = (total + 7) / 8, i = (blockIdx.x >> 3) - first, t = (blockIdx.x & 7) * per + i;
  return i < per && t < total ? t : ~0u;
}

// LDS of a tile: the ring of steps, or what the four wavefronts of KW = 4 leave there.
constexpr int tile_lds(int bm, int bn, int stages, int kw) { return kw > 1 && stages * kStepBytes * (bm + bn) < kw * bm * (bn + 4) * 4 ? kw * bm * (bn + 4) * 4 : stages * kStepBytes * (bm + bn); }

template <typename T, int BM, int BN, int WY, int WX, bool DIRECT, int STAGES, int KW = 1>
__global__ __launch_bounds__(64 * WY * WX * KW) void k_forward(const Product p) {
  __shared__ __align__(16) unsigned char lds[tile_lds(BM, BN, STAGES, KW)];
  const uint32_t tile = tile_of_block((uint32_t)p.tiles_m * p.tiles_n * p.splits);
  if (tile != ~0u) tile_product<T, BM, BN, WY, WX, true, false, DIRECT, STAGES, KW>(p, tile, lds);
}

// One or two rows (a single sample answered): a read of the weights.  A workgroup takes C columns, a lane eight of them, and 1024 or 512 weight rows at a time, asked
// for together with x, which waits in LDS; a column's lanes exchange halves of their sums until each has one, and the wavefronts' sums are added in their order
// (1 x 784 x 512 bf16 4.9 us; with sums of all values over all lanes, and weights asked for behind x, 5.6).  One launch, unless the contraction is split.  What bounds
// it: a launch and two trips to memory, one of them the kernel's own (1 x 1024 x 4096 bf16 4.7 us, from memory 7.4; 8192 x 16384 53.2 us, 5.0 TB/s; float32 4.8, 9.9 and
// 100.6 us, 5.3 TB/s; 4096 x 1024 in two launches, from memory, bf16 11.0 us, float32 13.8).
constexpr int kFewThreads = 1024;
template <typename T, int C>
__global__ __launch_bounds__(kFewThreads) void k_few_rows(const Product p) {
  constexpr int R = kFewRows, E = Elem<T>::kPer16, kVecs = 8 / E;        // kVecs: loads of eight columns
  constexpr int kLanes = C / 8, kApart = kFewThreads / kLanes, U = 8 / kVecs, kFewStep = U * kApart;
  __shared__ float xs[R][kFewStep], part[16][R][C];
  const int t = threadIdx.x, lane = t & 63, cg = t % kLanes, kl = t / kLanes, n0 = blockIdx.x * C, n = n0 + cg * 8;
  const int64_t left = (int64_t)p.N - n, k_end = min(p.K, (blockIdx.y + 1) * p.k_per_split);
  const T *w = static_cast<const T *>(p.b) + n, *x = static_cast<const T *>(p.a);
  float acc[R][8] = {};
  for (int64_t k0 = blockIdx.y * p.k_per_split; k0 < k_end; k0 += kFewStep) {
    const int here = (int)min((int64_t)kFewStep, k_end - k0);
    float xv[R];
#pragma unroll
    for (int r = 0; r < R; ++r) xv[r] = r < p.M && t < here ? to_f32(x[r * p.lda + k0 + t]) : 0.f;
    u32x4v raw[U][kVecs];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int v = 0; v < kVecs; ++v) raw[u][v] = load16_n(w + (k0 + kl + u * kApart) * p.ldb + v * E, kl + u * kApart < here ? left - v * E : 0);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) if (t < kFewStep) xs[r][t] = xv[r];
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (kl + u * kApart >= here) break;
#pragma unroll
      for (int r = 0; r < R; ++r) xv[r] = xs[r][kl + u * kApart];
#pragma unroll
      for (int v = 0; v < kVecs; ++v) {
        float f[E];
        unpack<T>(raw[u][v], f);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int e = 0; e < E; ++e) acc[r][v * E + e] = fmaf(xv[r], f[e], acc[r][v * E + e]);
      }
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
#pragma unroll
    for (int o = kLanes; o < 8; o *= 2)
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[r][e] += __shfl_xor(acc[r][e], o, 64);
#pragma unroll
    for (int h = 4; h > 0; h /= 2) {        // lanes 8 h apart: the upper one goes on with the upper half
      const bool upper = lane & 8 * h;
#pragma unroll
      for (int e = 0; e < h; ++e) {
        const float mine = upper ? acc[r][e + h] : acc[r][e], other = upper ? acc[r][e] : acc[r][e + h];
        acc[r][e] = mine + __shfl_xor(other, 8 * h, 64);
      }
    }
    if ((lane & 7) < kLanes) part[t >> 6][r][cg * 8 + (lane >> 5) * 4 + (lane >> 4 & 1) * 2 + (lane >> 3 & 1)] = acc[r][0];
  }
  __syncthreads();
  if (t < R * C) {
    float v = part[0][t / C][t % C];
#pragma unroll
    for (int i = 1; i < 16; ++i) v += part[i][t / C][t % C];
    part[0][t / C][t % C] = v;
  }
  __syncthreads();
  const int m = t / kLanes;
  if (m >= R || m >= p.M) return;
  float f[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = part[0][m][cg * 8 + e];
  if (p.splits > 1) store8_n(p.partial + ((int64_t)blockIdx.y * p.M + m) * eights(p.N) + n, left > 0 ? 8 : 0, f);
  else finish8<T>(p.epi, m, n, left, f);
}

// dx and dw in one launch (either may have no tiles), the one with the longer contraction first: its tiles would be the launch's tail.
struct Turn { uint32_t tile; bool dw; };
__device__ __forceinline__ Turn backward_tile(const Product &dx, const Product &dw) {
  const uint32_t n_dw = (uint32_t)dw.tiles_m * dw.tiles_n * dw.splits, n_dx = (uint32_t)dx.tiles_m * dx.tiles_n * dx.splits;
  const bool dw_first = dw.k_per_split >= dx.k_per_split;
  const uint32_t n_first = dw_first ? n_dw : n_dx, n_second = dw_first ? n_dx : n_dw, first = (n_first + 7) / 8;
  const bool in_first = (blockIdx.x >> 3) < first;
  return Turn{in_first ? tile_of_block(n_first) : tile_of_block(n_second, first), in_first == dw_first};
}
template <typename T, int BM, int BN, int WY, int WX, bool DIRECT, int STAGES, int KW = 1>
__global__ __launch_bounds__(64 * WY * WX * KW) void k_backward(const Product dx, const Product dw) {
  __shared__ __align__(16) unsigned char lds[tile_lds(BM, BN, STAGES, KW)];
  const Turn turn = backward_tile(dx, dw);
  if (turn.tile == ~0u) return;
  if (turn.dw) tile_product<T, BM, BN, WY, WX, false, false, DIRECT, STAGES, KW>(dw, turn.tile, lds);
  else tile_product<T, BM, BN, WY, WX, true, true, DIRECT, STAGES, KW>(dx, turn.tile, lds);
}

// The same for small gradients: any alignment, and dz formed on the way (dy's and pre's rows in the place of dz's).
template <typename T, int E, int W, int KW>
__global__ __launch_bounds__(256) void k_backward_small(const Product dx, const Product dw) {
  __shared__ __align__(16) unsigned char lds[tile_lds(E, E, 2, KW)];
  const Turn turn = backward_tile(dx, dw);
  if (turn.tile == ~0u) return;
  if (turn.dw) tile_product<T, E, E, W, W, false, false, false, 2, KW, B_SIGNAL>(dw, turn.tile, lds);
  else tile_product<T, E, E, W, W, true, true, false, 2, KW, A_SIGNAL>(dx, turn.tile, lds);
}

// Tables of less than 16 bytes (the contraction has few terms, or there are few outputs in a row or column), and rows so far apart that a tile's
// do not lie within 4 GB: a thread per output.
template <typename T, bool AKC, bool BKC, int SIGNAL>
__global__ __launch_bounds__(256) void k_by_element(const Product p) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < p.M * p.N; i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / p.N, n = i - m * p.N;
    float sum = 0.f, column = 0.f;
    for (int64_t k = 0; k < p.K; ++k) {
      float a = to_f32(static_cast<const T *>(p.a)[AKC ? m * p.lda + k : k * p.lda + m]), b = to_f32(static_cast<const T *>(p.b)[BKC ? n * p.ldb + k : k * p.ldb + n]);
      if constexpr (SIGNAL != NO_SIGNAL) {
        float &dz = SIGNAL == A_SIGNAL ? a : b;
        if (p.act != CADA_ACT_NONE) dz *= activation_slope<T>(to_f32(static_cast<const T *>(p.pre)[SIGNAL == A_SIGNAL ? m * p.ldpre + k : k * p.ldpre + n]), p.act);
        column += dz;
        dz = to_f32(from_f32<T>(dz));
      }
      sum = fmaf(a, b, sum);
    }
    float f[8] = {sum};
    finish8<T>(p.epi, m, (int)n, 1, f);
    if (SIGNAL == B_SIGNAL && p.db && m == 0) static_cast<T *>(p.db)[n] = from_f32<T>(column);
  }
}

// Joins the sums of a split contraction, in the order of the splits, and finishes them; eight columns per thread.
struct Join {
  Product p[2];
  int64_t groups[2];         // M * ceil(N / 8), 0 where there is nothing to join
  const float *db_part;      // [db_parts][N of the second product] or null
  void *db;
  int db_parts, db_n;
  unsigned db_block;         // the first workgroup of the column sums
};
template <typename T>
__global__ __launch_bounds__(256) void k_join(const Join j) {
  int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (blockIdx.x < j.db_block && g < j.groups[i]) {
      const Product &p = j.p[i];
      const int per = (p.N + 7) / 8;
      const int64_t m = g / per;
      const int n = (int)(g - m * per) * 8;
      const int64_t left = (int64_t)p.N - n, apart = p.M * per * 8 / 4;        // (four floats apart)
      const v4s *src = reinterpret_cast<const v4s *>(p.partial + (m * per * 8 + n));
      v4s lo = src[0], hi = src[1];
      for (int s = 1; s < p.splits; s += 8) {        // eight parts on their way at once
        v4s l[8], h[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const v4s *at = src + (int64_t)min(s + u, p.splits - 1) * apart;
          l[u] = at[0];
          h[u] = at[1];
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          if (s + u < p.splits) { lo += l[u]; hi += h[u]; }
        }
      }
      float f[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      finish8<T>(p.epi, m, n, left, f);
      return;
    }
    g -= j.groups[i];
  }
  if (blockIdx.x < j.db_block) return;
  if (!j.db_part) return;
  // Column sums of dz: a workgroup of its own takes 32 columns, eight lanes of each every eighth part.
  __shared__ float part[8][32];
  const int c = (int)(blockIdx.x - j.db_block) * 32 + (threadIdx.x & 31), lane = threadIdx.x >> 5;
  float s = 0.f;
  if (c < j.db_n) {
#pragma unroll 8
    for (int i = lane; i < j.db_parts; i += 8) s += j.db_part[(int64_t)i * j.db_n + c];
  }
  part[lane][threadIdx.x & 31] = s;
  __syncthreads();
  if (lane == 0 && c < j.db_n) {
#pragma unroll
    for (int i = 1; i < 8; ++i) s += part[i][threadIdx.x];
    static_cast<T *>(j.db)[c] = from_f32<T>(s);
  }
}

// dz = dy * act'(pre), written in the operands' type with rows on 16-byte boundaries, and its column sums per block of rows.  A workgroup is 2^lanes threads
// of eight columns each, as many as the columns need up to 32, by as many rows at a time.  Of bf16 tables dz is rounded to bf16, which the matrix
// instructions' operands are (the way that forms it on its way into LDS rounds it alike): dx and dw are 2.3e-3 from 64 bits, relative in the 2-norm, where the rounding of the outputs alone leaves
// 1.7e-3; two bf16 parts of dz would be twice the products.  The column sums are of dz before that.
struct Signal {
  const void *dy, *pre;
  int64_t lddy, ldpre, rows, rows_per_block;
  int32_t n, act, lanes;
  void *dz;                  // or null
  int64_t lddz;
  float *db_part;            // [blocks of rows][n] or null
};
template <typename T>
__global__ __launch_bounds__(256) void k_signal(const Signal a) {
  __shared__ float part[256 * 9];
  const int t = threadIdx.x, width = 1 << a.lanes, cx = t & (width - 1), ry = t >> a.lanes, high = 256 >> a.lanes;
  const int n = (blockIdx.x * width + cx) * 8;
  const int64_t left = (int64_t)a.n - n, r0 = (int64_t)blockIdx.y * a.rows_per_block, r1 = min(a.rows, r0 + a.rows_per_block);
  float sum[8] = {};
  if (left > 0) {
    for (int64_t r = r0 + ry; r < r1; r += high) {
      float f[8], z[8];
      load8_n(static_cast<const T *>(a.dy) + r * a.lddy + n, left, f);
      if (a.act != CADA_ACT_NONE) {
        load8_n(static_cast<const T *>(a.pre) + r * a.ldpre + n, left, z);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] *= activation_slope<T>(z[i], a.act);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] += f[i];
      if (a.dz) store8_n(static_cast<T *>(a.dz) + r * a.lddz + n, 8, f);        // (a whole group always: the rows have room for it, and the fill is zero)
    }
  }
  if (!a.db_part) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) part[t * 9 + i] = sum[i];
  __syncthreads();
  const int c = blockIdx.x * width * 8 + t;
  if (t < width * 8 && c < a.n) {
    float s = 0.f;
    for (int i = 0; i < high; ++i) s += part[((i << a.lanes) + (t >> 3)) * 9 + (t & 7)];
    a.db_part[(int64_t)blockIdx.y * a.n + c] = s;
  }
}

// Tables whose rows start on no 16-byte boundary, copied to rows that do (filled up with zeros), for products large enough to be worth it.
struct Pack { const void *src; void *dst; int64_t ld, rows, cols, ldd; };
struct Packs { Pack p[2]; int64_t pieces[2]; };
template <typename T>
__global__ __launch_bounds__(256) void k_pack(const Packs a) {
  constexpr int E = Elem<T>::kPer16;
  for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < a.pieces[0] + a.pieces[1]; at += (int64_t)gridDim.x * 256) {
    const int q = at < a.pieces[0] ? 0 : 1;
    const int64_t i = at - (q ? a.pieces[0] : 0);
    const Pack &p = a.p[q];
    const int64_t per = p.ldd / E, row = i / per, col = (i - row * per) * E;
    *reinterpret_cast<u32x4v *>(static_cast<T *>(p.dst) + row * p.ldd + col) = load16_n(static_cast<const T *>(p.src) + row * p.ld + col, p.cols - col);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_zero(T *p, int64_t ld, int64_t rows, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * n; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / n;
    p[r * ld + (i - r * n)] = from_f32<T>(0.f);
  }
}

// ---- host ----

// Workgroups of 256 threads for so many items, which the kernel's loop takes on from there.
unsigned many(int64_t items) { return (unsigned)std::min<int64_t>(ceil_div(items, 256), 1 << 20); }
template <typename T>
int launch_pack(Packs &a, hipStream_t st) {
  int64_t total = 0;
  for (int i = 0; i < 2; ++i) {
    a.pieces[i] = a.p[i].src ? a.p[i].rows * (a.p[i].ldd / Elem<T>::kPer16) : 0;
    total += a.pieces[i];
  }
  if (total == 0) return CADA_OK;
  k_pack<T><<<many(total), 256, 0, st>>>(a);
  return ops_launched("linear pack");
}
void lay(Product *p, const Cut &c, const void *a, int64_t lda, const void *b, int64_t ldb, int64_t M, int64_t N, int64_t K, float *partial) {
  p->a_cols = M; p->b_cols = N;
  p->a = a; p->lda = lda; p->b = b; p->ldb = ldb; p->M = M; p->N = (int32_t)N; p->K = K;
  p->tiles_m = (int32_t)ceil_div(M, c.tile); p->tiles_n = (int32_t)ceil_div(N, c.tile);
  p->splits = c.splits; p->k_per_split = c.k_per_split; p->partial = c.splits > 1 ? partial : nullptr;
}
int64_t tiles_of(const Product &p) { return (int64_t)p.tiles_m * p.tiles_n * p.splits; }

bool check_shape(int64_t rows, int64_t in, int64_t out, int type, int act) {
  if (rows < 0 || rows > (int64_t)1 << 40) { set_error("rows must be in [0, 2^40] (got %lld)", (long long)rows); return false; }
  if (in < 1 || in > CADA_MAX_WIDTH || out < 1 || out > CADA_MAX_WIDTH) { set_error("in and out must be in [1, %d] (got %lld, %lld)", CADA_MAX_WIDTH, (long long)in, (long long)out); return false; }
  if (type != CADA_F32 && type != CADA_BF16) { set_error("type must be CADA_F32 or CADA_BF16 (got %d)", type); return false; }
  if (act < CADA_ACT_NONE || act > CADA_ACT_SILU) { set_error("act must be one of CADA_ACT_* (got %d)", act); return false; }
  const int64_t t = std::max({ceil_div(rows, 64) * ceil_div(out, 64), ceil_div(rows, 64) * ceil_div(in, 64), ceil_div(in, 64) * ceil_div(out, 64)});
  if (t > kMostTiles) { set_error("more than %lld tiles of 64 x 64 outputs", (long long)kMostTiles); return false; }
  return true;
}
bool check_table(const char *name, const void *p, int64_t ld, int64_t cols, int type) {
  if (!p) { set_error("%s is NULL", name); return false; }
  if (ld < cols) { set_error("the row length of %s (%lld) is less than its %lld columns", name, (long long)ld, (long long)cols); return false; }
  if (reinterpret_cast<uintptr_t>(p) % type_bytes(type) != 0) { set_error("%s is not aligned to its elements", name); return false; }
  return true;
}

// ---- forward ----

// Four steps on their way where LDS has room for them (few tiles: long contractions come from memory, 64 x 64 x 4096 with one tile per CU 32 -> 18.5 us); two, and more
// workgroups on a CU, where there are many tiles (64 x 64 x 1024 with four per CU 17 -> 15.5 us).
bool deep(int tile, int64_t tiles) { return tiles <= (tile <= 64 ? 2 : 1) * kCUs; }

template <typename T, int E, int WY, int WX, int KW>
void forward_tiles(const Product &p, bool dir, hipStream_t st) {
  const unsigned grid = (unsigned)(ceil_div(tiles_of(p), 8) * 8);
  if constexpr (E <= 64) {
    if (!dir) { k_forward<T, E, E, WY, WX, false, 2, KW><<<grid, 64 * WY * WX * KW, 0, st>>>(p); return; }
  }
  if constexpr (E < 256) {
    if (deep(E, tiles_of(p))) { k_forward<T, E, E, WY, WX, true, 4, KW><<<grid, 64 * WY * WX * KW, 0, st>>>(p); return; }
  }
  k_forward<T, E, E, WY, WX, true, 2, KW><<<grid, 64 * WY * WX * KW, 0, st>>>(p);
}

template <typename T>
int launch_join(Join &j, hipStream_t st) {
  int64_t total = 0;
  for (int i = 0; i < 2; ++i) {
    j.groups[i] = j.p[i].splits > 1 ? j.p[i].M * ceil_div(j.p[i].N, 8) : 0;
    total += j.groups[i];
  }
  j.db_block = (unsigned)ceil_div(total, 256);
  const unsigned grid = j.db_block + (j.db_part ? (unsigned)ceil_div(j.db_n, 32) : 0);
  if (grid == 0) return CADA_OK;
  k_join<T><<<grid, 256, 0, st>>>(j);
  return ops_launched("linear join");
}

template <typename T>
int forward(const cada_linear *a, const ForwardPlan &f) {
  hipStream_t st = static_cast<hipStream_t>(a->stream);
  Product p{};
  lay(&p, f.cut, a->x, a->ldx, a->w, a->ldw, a->rows, a->out, a->in, static_cast<float *>(a->workspace));
  if (f.pack_x || f.pack_w) {
    Packs k{};
    char *ws = static_cast<char *>(a->workspace);
    if (f.pack_x) {
      k.p[0] = Pack{a->x, ws + f.off_x, a->ldx, a->rows, a->in, packed_ld(a->in)};
      p.a = k.p[0].dst; p.lda = k.p[0].ldd;
    }
    if (f.pack_w) {
      k.p[1] = Pack{a->w, ws + f.off_w, a->ldw, a->in, a->out, packed_ld(a->out)};
      p.b = k.p[1].dst; p.ldb = p.b_cols = k.p[1].ldd;
    }
    if (int rc = launch_pack<T>(k, st)) return rc;
  }
  p.epi = Epilogue{a->bias, a->residual, a->pre, a->y, a->ldr, a->ldpre, a->ldy, a->act};
  if (f.few) {
    const int columns = few_columns(sizeof(T), a->out);
    const dim3 grid((unsigned)ceil_div(a->out, columns), p.splits);
    if (columns == 64) k_few_rows<T, 64><<<grid, kFewThreads, 0, st>>>(p);
    else if constexpr (sizeof(T) == 4) k_few_rows<T, 32><<<grid, kFewThreads, 0, st>>>(p);
  } else if (f.by_element) {
    k_by_element<T, true, false, NO_SIGNAL><<<many(a->rows * a->out), 256, 0, st>>>(p);
  } else if (f.cut.tile == 32) {
    forward_tiles<T, 32, 1, 1, 4>(p, f.direct, st);
  } else if (f.cut.tile == 64) {
    forward_tiles<T, 64, 2, 2, 1>(p, f.direct, st);
  } else if constexpr (sizeof(T) == 2) {
    if (f.cut.tile == 128) forward_tiles<T, 128, 2, 4, 1>(p, f.direct, st);
    if (f.cut.tile == 256) forward_tiles<T, 256, 2, 4, 1>(p, f.direct, st);
  }
  if (int rc = ops_launched("linear")) return rc;
  if (p.splits == 1) return CADA_OK;
  Join j{};
  j.p[0] = p;
  return launch_join<T>(j, st);
}

// ---- backward ----

template <typename T>
int zero_table(void *p, int64_t ld, int64_t rows, int64_t n, hipStream_t st) {
  k_zero<T><<<(unsigned)std::min<int64_t>(ceil_div(rows * n, 256), 4096), 256, 0, st>>>(static_cast<T *>(p), ld, rows, n);
  return ops_launched("linear clear");
}

template <typename T, int E, int WY, int WX, int KW>
void backward_tiles(const Product &dx, const Product &dw, bool dir, hipStream_t st) {
  const unsigned grid = (unsigned)((ceil_div(tiles_of(dx), 8) + ceil_div(tiles_of(dw), 8)) * 8);
  if constexpr (E <= 64) {
    if (!dir) { k_backward<T, E, E, WY, WX, false, 2, KW><<<grid, 64 * WY * WX * KW, 0, st>>>(dx, dw); return; }
  }
  if constexpr (E < 256) {
    if (deep(E, tiles_of(dx) + tiles_of(dw))) { k_backward<T, E, E, WY, WX, true, 4, KW><<<grid, 64 * WY * WX * KW, 0, st>>>(dx, dw); return; }
  }
  k_backward<T, E, E, WY, WX, true, 2, KW><<<grid, 64 * WY * WX * KW, 0, st>>>(dx, dw);
}

template <typename T>
int backward(const cada_linear_grad *a, const BackwardPlan &b) {
  hipStream_t st = static_cast<hipStream_t>(a->stream);
  if (a->rows == 0) {
    if (a->dw) if (int rc = zero_table<T>(a->dw, a->lddw, a->in, a->out, st)) return rc;
    if (a->db) return zero_table<T>(a->db, a->out, 1, a->out, st);
    return CADA_OK;
  }
  char *ws = static_cast<char *>(a->workspace);
  float *db_part = reinterpret_cast<float *>(ws + b.off_db);
  const bool db_by_products = b.small || (b.by_element && a->dw);
  if (b.own_dz || (a->db && !db_by_products)) {
    Signal s{};
    s.dy = a->dy; s.lddy = a->lddy; s.pre = a->pre; s.ldpre = a->ldpre; s.rows = a->rows; s.rows_per_block = b.rows_per_block; s.n = (int32_t)a->out; s.act = a->act; s.lanes = b.signal_lanes;
    s.dz = b.own_dz ? ws : nullptr; s.lddz = b.lddz;
    s.db_part = a->db ? db_part : nullptr;
    k_signal<T><<<dim3((unsigned)b.signal_columns, (unsigned)b.row_blocks), 256, 0, st>>>(s);
    if (int rc = ops_launched("linear signal")) return rc;
  }
  const void *dz = b.own_dz ? ws : a->dy;
  const int64_t lddz = b.own_dz ? b.lddz : a->lddy;
  Product dx{}, dw{};
  if (a->dx) {
    lay(&dx, b.dx, dz, lddz, a->w, a->ldw, a->rows, a->in, a->out, reinterpret_cast<float *>(ws + b.off_dx));
    dx.epi.out = a->dx; dx.epi.ldo = a->lddx;
    dx.pre = a->pre; dx.ldpre = a->ldpre; dx.act = a->act;
  }
  if (a->dw) {
    lay(&dw, b.dw, a->x, a->ldx, dz, lddz, a->in, a->out, a->rows, reinterpret_cast<float *>(ws + b.off_dw));
    if (b.own_dz) dw.b_cols = b.lddz;      // (dz's rows in the workspace are filled with zeros up to whole pieces)
    dw.epi.out = a->dw; dw.epi.ldo = a->lddw;
    dw.pre = a->pre; dw.ldpre = a->ldpre; dw.act = a->act;
    if (db_by_products) { dw.db = a->db; dw.db_part = db_part; }
  }
  if (b.pack_x || b.pack_w) {
    Packs k{};
    if (b.pack_x) {
      k.p[0] = Pack{a->x, ws + b.off_x, a->ldx, a->rows, a->in, packed_ld(a->in)};
      dw.a = k.p[0].dst; dw.lda = dw.a_cols = k.p[0].ldd;
    }
    if (b.pack_w) {
      k.p[1] = Pack{a->w, ws + b.off_w, a->ldw, a->in, a->out, packed_ld(a->out)};
      dx.b = k.p[1].dst; dx.ldb = k.p[1].ldd;
    }
    if (int rc = launch_pack<T>(k, st)) return rc;
  }
  if (a->dx || a->dw) {
    const int tile = a->dx ? b.dx.tile : b.dw.tile;
    const unsigned grid = (unsigned)((ceil_div(tiles_of(dx), 8) + ceil_div(tiles_of(dw), 8)) * 8);
    if (b.by_element) {
      if (a->dx) k_by_element<T, true, true, A_SIGNAL><<<many(a->rows * a->in), 256, 0, st>>>(dx);
      if (a->dw) k_by_element<T, false, false, B_SIGNAL><<<many(a->in * a->out), 256, 0, st>>>(dw);
    } else if (b.small && tile == 32) {
      k_backward_small<T, 32, 1, 4><<<grid, 256, 0, st>>>(dx, dw);
    } else if (b.small) {
      k_backward_small<T, 64, 2, 1><<<grid, 256, 0, st>>>(dx, dw);
    } else if (tile == 32) {
      backward_tiles<T, 32, 1, 1, 4>(dx, dw, b.direct, st);
    } else if (tile == 64) {
      backward_tiles<T, 64, 2, 2, 1>(dx, dw, b.direct, st);
    } else if constexpr (sizeof(T) == 2) {
      if (tile == 128) backward_tiles<T, 128, 2, 4, 1>(dx, dw, b.direct, st);
      if (tile == 256) backward_tiles<T, 256, 2, 4, 1>(dx, dw, b.direct, st);
    }
    if (int rc = ops_launched("linear gradients")) return rc;
  }
  Join j{};
  j.p[0] = dx; j.p[1] = dw;
  if (a->db && (!db_by_products || b.dw.splits > 1)) { j.db_part = db_part; j.db = a->db; j.db_parts = (int)b.row_blocks; j.db_n = (int)a->out; }
  return launch_join<T>(j, st);
}

}  // namespace

bool ops_apart(const Span &out, const Span &other) {
  if (!out.at || !other.at) return true;
  const uintptr_t a = reinterpret_cast<uintptr_t>(out.at), b = reinterpret_cast<uintptr_t>(other.at);
  if (a + ((out.rows - 1) * out.ld + out.cols) <= b || b + ((other.rows - 1) * other.ld + other.cols) <= a) return true;
  // (both lie in rows of one length: a single row in those of the other)
  if (out.rows == 1 || other.rows == 1 || out.ld == other.ld) {
    const int64_t row = out.rows > 1 ? out.ld : other.ld, between = ((int64_t)(b - a) % row + row) % row;      // from out's column to the other's in a row of both
    if (between >= out.cols && between + other.cols <= row) return true;
  }
  set_error("%s and %s share memory", out.name, other.name);
  return false;
}
bool ops_apart(Range *ranges, size_t n) {
  std::sort(ranges, ranges + n, [](const Range &x, const Range &y) { return x.at != y.at ? reinterpret_cast<uintptr_t>(x.at) < reinterpret_cast<uintptr_t>(y.at) : x.index < y.index; });
  auto end = [](const Range &r) { return reinterpret_cast<uintptr_t>(r.at) + r.bytes; };
  const Range *last = nullptr, *last_written = nullptr;      // of those that begin no later, the ones that end last
  for (const Range *r = ranges; r < ranges + n; ++r) {
    if (!r->at || r->bytes == 0) continue;
    const Range *other = r->written ? last : last_written;
    if (other && end(*other) > reinterpret_cast<uintptr_t>(r->at)) {
      char text[2][64];
      for (int i = 0; i < 2; ++i) {
        const Range &x = i == 0 ? *other : *r;
        if (x.index >= 0) snprintf(text[i], sizeof(text[i]), "%s %d", x.name, x.index);
        else snprintf(text[i], sizeof(text[i]), "%s", x.name);
      }
      set_error("%s and %s share memory", text[0], text[1]);
      return false;
    }
    if (!last || end(*r) > end(*last)) last = r;
    if (r->written && (!last_written || end(*r) > end(*last_written))) last_written = r;
  }
  return true;
}
int ops_check_workspace(const void *ws, size_t given, size_t need) {
  if (need == 0) return CADA_OK;
  if (!ws) { set_error("workspace is NULL"); return CADA_EWORKSPACE; }
  if (reinterpret_cast<uintptr_t>(ws) % kOpsAlign != 0) { set_error("workspace must be %zu-byte aligned", kOpsAlign); return CADA_EWORKSPACE; }
  if (given < need) { set_error("workspace too small: %zu bytes given, %zu needed", given, need); return CADA_EWORKSPACE; }
  return CADA_OK;
}
int ops_launched(const char *what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return CADA_OK;
  set_error("%s: %s", what, hipGetErrorString(e));
  return CADA_EHIP;
}

}  // namespace cada

using namespace cada;

extern "C" {

int cada_linear_forward_workspace(cada_linear *a) {
  if (!a) { set_error("the arguments are NULL"); return CADA_EINVAL; }
  if (!check_shape(a->rows, a->in, a->out, a->type, a->act)) return CADA_EINVAL;
  a->workspace_bytes = plan_forward(a).bytes;
  return CADA_OK;
}

int cada_linear_forward(const cada_linear *a) {
  if (!a) { set_error("the arguments are NULL"); return CADA_EINVAL; }
  if (!check_shape(a->rows, a->in, a->out, a->type, a->act)) return CADA_EINVAL;
  if (a->rows == 0) return CADA_OK;
  if (!check_table("x", a->x, a->ldx, a->in, a->type) || !check_table("w", a->w, a->ldw, a->out, a->type) || !check_table("y", a->y, a->ldy, a->out, a->type)) return CADA_EINVAL;
  if (a->bias && !check_table("bias", a->bias, a->out, a->out, a->type)) return CADA_EINVAL;
  if (a->residual && !check_table("residual", a->residual, a->ldr, a->out, a->type)) return CADA_EINVAL;
  if (a->pre && !check_table("pre", a->pre, a->ldpre, a->out, a->type)) return CADA_EINVAL;
  const ForwardPlan f = plan_forward(a);
  if (int rc = ops_check_workspace(a->workspace, a->workspace_bytes, f.bytes)) return rc;
  const size_t elem = type_bytes(a->type);
  const Span y = span("y", a->y, a->rows, a->ldy, a->out, elem), pre = span("pre", a->pre, a->rows, a->ldpre, a->out, elem), residual = span("residual", a->residual, a->rows, a->ldr, a->out, elem);
  const Span ins[] = {span("x", a->x, a->rows, a->ldx, a->in, elem), span("w", a->w, a->in, a->ldw, a->out, elem), span("bias", a->bias, 1, a->out, a->out, elem)};
  for (const Span &in : ins)
    if (!ops_apart(y, in) || !ops_apart(pre, in)) return CADA_EINVAL;
  const bool in_place = a->residual == a->y && (a->ldr == a->ldy || a->rows == 1);
  if (!ops_apart(y, pre) || !ops_apart(pre, residual) || (!in_place && !ops_apart(y, residual))) return CADA_EINVAL;
  const Span workspace = span("workspace", a->workspace, f.bytes);
  for (const Span &other : {ins[0], ins[1], ins[2], y, pre, residual})
    if (!ops_apart(workspace, other)) return CADA_EINVAL;
  return a->type == CADA_BF16 ? forward<bf16>(a, f) : forward<float>(a, f);
}

int cada_linear_backward_workspace(cada_linear_grad *a) {
  if (!a) { set_error("the arguments are NULL"); return CADA_EINVAL; }
  if (!check_shape(a->rows, a->in, a->out, a->type, a->act)) return CADA_EINVAL;
  a->workspace_bytes = plan_backward(a).bytes;
  return CADA_OK;
}

int cada_linear_backward(const cada_linear_grad *a) {
  if (!a) { set_error("the arguments are NULL"); return CADA_EINVAL; }
  if (!check_shape(a->rows, a->in, a->out, a->type, a->act)) return CADA_EINVAL;
  if (a->rows > 0) {
    if ((a->dx || a->dw || a->db) && !check_table("dy", a->dy, a->lddy, a->out, a->type)) return CADA_EINVAL;
    if ((a->dx || a->dw || a->db) && a->act != CADA_ACT_NONE && !check_table("pre", a->pre, a->ldpre, a->out, a->type)) return CADA_EINVAL;
    if (a->dx && (!check_table("w", a->w, a->ldw, a->out, a->type) || !check_table("dx", a->dx, a->lddx, a->in, a->type))) return CADA_EINVAL;
    if (a->dw && !check_table("x", a->x, a->ldx, a->in, a->type)) return CADA_EINVAL;
  }
  if (a->dw && !check_table("dw", a->dw, a->lddw, a->out, a->type)) return CADA_EINVAL;
  if (a->db && !check_table("db", a->db, a->out, a->out, a->type)) return CADA_EINVAL;
  const BackwardPlan b = plan_backward(a);
  if (int rc = ops_check_workspace(a->workspace, a->workspace_bytes, b.bytes)) return rc;
  const size_t elem = type_bytes(a->type);
  const Span outs[] = {span("dx", a->rows ? a->dx : nullptr, a->rows, a->lddx, a->in, elem), span("dw", a->dw, a->in, a->lddw, a->out, elem), span("db", a->db, 1, a->out, a->out, elem)};
  const Span ins[] = {span("dy", a->dy, a->rows, a->lddy, a->out, elem), span("x", a->dw ? a->x : nullptr, a->rows, a->ldx, a->in, elem), span("w", a->dx ? a->w : nullptr, a->in, a->ldw, a->out, elem),
                      span("pre", a->act != CADA_ACT_NONE ? a->pre : nullptr, a->rows, a->ldpre, a->out, elem)};
  for (int i = 0; i < 3; ++i) {
    for (const Span &in : ins)
      if (a->rows && !ops_apart(outs[i], in)) return CADA_EINVAL;
    for (int j = 0; j < i; ++j)
      if (!ops_apart(outs[i], outs[j])) return CADA_EINVAL;
  }
  const Span workspace = span("workspace", a->workspace, b.bytes);        // (none without rows)
  for (const Span &other : {ins[0], ins[1], ins[2], ins[3], outs[0], outs[1], outs[2]})
    if (!ops_apart(workspace, other)) return CADA_EINVAL;
  return a->type == CADA_BF16 ? backward<bf16>(a, b) : backward<float>(a, b);
}

}  // extern "C"
