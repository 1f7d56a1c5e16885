// The tile kernel that a layer's products (cada_linear.hip) and a last layer's loss (cada_linear_xent.hip) are made of, and the launches that the second takes from the first.
#pragma once

#include "cada_linear_plan.h"
#include "cada_ops_internal.h"

namespace cada {

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
  float *partial;            // [splits][M][N up to whole groups of eight], or null: sums that k_join joins and finishes (splits > 1, or a contraction that goes on in another launch)
  Epilogue epi;
  // small gradients: the operand that is the signal is read as dy, and dz = dy * act'(pre) is formed on its way into LDS
  const void *pre;
  int64_t ldpre;
  int32_t act;
  void *db;                  // column sums of dz (or null), by the tiles of the first rows; their parts where the contraction is split
  float *db_part;            // [splits][N]
  // PIECES: a factor of finished sums, in device memory, and whether unfinished ones are added to what is in `partial` already.  (Behind all that a layer's
  // products read: with the two before the epilogue and in it, 1 x 1024 x 4096 bf16 6.14 us instead of 6.00, 15499 x 2097 x 16 23.15 instead of 22.96.)
  const float *factor;
  int32_t add;
};

// Joins the sums of a split contraction, in the order of the splits, and finishes them; eight columns per thread.
struct Join {
  Product p[2];
  int64_t groups[2];         // M * ceil(N / 8), 0 where there is nothing to join
  const float *db_part;      // [db_parts][N of the second product] or null
  void *db;
  const float *db_factor;    // PIECES: of the column sums, in device memory
  int db_parts, db_n;
  unsigned db_block;         // the first workgroup of the column sums
};
// Tables whose rows start on no 16-byte boundary, copied to rows that do (filled up with zeros), for products large enough to be worth it.
struct Pack { const void *src; void *dst; int64_t ld, rows, cols, ldd; };
struct Packs { Pack p[2]; int64_t pieces[2]; };

// Products, joins and copies of a type (CADA_F32 or CADA_BF16), for other files than cada_linear.hip; products and joins with PIECES.
int linear_sums(int type, int tile, bool direct, const Product &p, hipStream_t st);        // a forward product whose sums go to p.partial
int linear_products(int type, int tile, bool direct, const Product &dx, const Product &dw, hipStream_t st);
int linear_join(int type, Join &j, hipStream_t st);

// Workgroups of 256 threads for so many items, which the kernel's loop takes on from there.
inline unsigned many(int64_t items) { return (unsigned)std::min<int64_t>(ceil_div(items, 256), 1 << 20); }
inline void lay(Product *p, const Cut &c, const void *a, int64_t lda, const void *b, int64_t ldb, int64_t M, int64_t N, int64_t K, float *partial) {
  p->a_cols = M; p->b_cols = N;
  p->a = a; p->lda = lda; p->b = b; p->ldb = ldb; p->M = M; p->N = (int32_t)N; p->K = K;
  p->tiles_m = (int32_t)ceil_div(M, c.tile); p->tiles_n = (int32_t)ceil_div(N, c.tile);
  p->splits = c.splits; p->k_per_split = c.k_per_split; p->partial = c.splits > 1 ? partial : nullptr;
}
inline int64_t tiles_of(const Product &p) { return (int64_t)p.tiles_m * p.tiles_n * p.splits; }

// Four steps on their way where LDS has room for them (few tiles: long contractions come from memory, 64 x 64 x 4096 with one tile per CU 32 -> 18.5 us); two, and more
// workgroups on a CU, where there are many tiles (64 x 64 x 1024 with four per CU 17 -> 15.5 us).
inline bool deep(int tile, int64_t tiles) { return tiles <= (tile <= 64 ? 2 : 1) * kCUs; }

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <typename T> constexpr int kStep = kStepBytes / (int)sizeof(T);

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
template <typename T, bool PIECES = false>
__device__ __forceinline__ void finish8(const Product &p, int64_t m, int n, int64_t left, float (&f)[8]) {
  if (left <= 0) return;
  const Epilogue &e = p.epi;
  float o[8];
  if constexpr (PIECES) {
    const float factor = *p.factor;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] *= factor;
  }
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

// Eight columns of an unfinished sum.
template <bool PIECES> __device__ __forceinline__ void put_part(const Product &p, uint32_t split, int64_t m, int n, int64_t left, float (&f)[8]) {
  if (left <= 0) return;
  float *to = p.partial + ((int64_t)split * p.M + m) * eights(p.N) + n;
  if (PIECES && p.add) {
    float o[8];
    load8_n(to, 8, o);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] += o[e];
  }
  store8_n(to, 8, f);
}

// What becomes of a tile's sums: a layer's output, here (PIECES: of a contraction that comes in several launches, with a factor that is in device memory); a
// last layer's loss has its own (cada_linear_xent.hip), which take the sums where the matrix instructions leave them, sums(), and where wavefronts share a
// tile's contraction and join their sums in LDS, eight columns of a row per lane, row().
template <bool PIECES = false> struct ToTable {
  static constexpr bool kOwn = false;
  __device__ __forceinline__ void begin(const Product &, int64_t, int, int) const {}
  template <typename T> __device__ __forceinline__ void row(const Product &p, uint32_t split, int64_t m, int n, int64_t left, float (&f)[8]) const {
    if (p.partial) put_part<PIECES>(p, split, m, n, left, f);
    else finish8<T, PIECES>(p, m, n, left, f);
  }
};

// WY x WX wavefronts share the tile; with KW = 4 four wavefronts each take the whole (32 x 32) tile and one of the four sub-steps of every step, and their sums are joined
// on the way out: short steps for few outputs.
enum { NO_SIGNAL = 0, A_SIGNAL = 1, B_SIGNAL = 2 };
template <typename T, int BM, int BN, int WY, int WX, bool AKC, bool BKC, bool DIRECT, int STAGES, int KW = 1, int SIGNAL = NO_SIGNAL, typename OUT = ToTable<>>
__device__ __forceinline__ void tile_product(const Product &p, uint32_t tile, unsigned char *lds, OUT out = OUT()) {
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
  out.begin(p, m0, n0, t);
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
    if (t < BM * 4 && (OUT::kOwn || m0 + t / 4 < p.M)) {
      const float *src = sums + t / 4 * kLd + (t & 3) * 8;
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = (src[e] + src[BM * kLd + e]) + (src[2 * BM * kLd + e] + src[3 * BM * kLd + e]);
      const int64_t m = m0 + t / 4, left = (int64_t)p.N - n0 - (t & 3) * 8;
      const int n = n0 + (t & 3) * 8;
      if constexpr (OUT::kOwn) out.template row<T>(p, m0, n0, t, f);
      else out.template row<T>(p, split, m, n, left, f);
    }
    return;
  }
  if constexpr (OUT::kOwn) {
    out.template sums<T, FM, FN>(p, acc, m0, n0, wm, wn, lane, lds + wave * (2 * kHalf / (WY * WX)));
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
    for (int turn = 0; turn < 32 / kRows; ++turn) {
      const int row = lane / kLanes + turn * kRows;
      const int64_t m = m0 + wm + 32 * i + row;
      const float *src = strip + row * kLd + lane % kLanes * 8;
      const v4s x = *reinterpret_cast<const v4s *>(src), y = *reinterpret_cast<const v4s *>(src + 4);
      float f[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
      if constexpr (!OUT::kOwn) {
        if (m < p.M) out.template row<T>(p, split, m, n, left, f);
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

}  // namespace
}  // namespace cada
