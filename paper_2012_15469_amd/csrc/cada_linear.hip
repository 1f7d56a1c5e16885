// A layer's product with bias, activation and residual, and its gradients (cada_ops.h).
//
// Three products of two tables: y = x w (contraction over x's columns), dx = dz w^T (over dz's columns) and dw = x^T dz (over
// the rows of both).  A table is read either along the contraction ("kc": consecutive elements are consecutive
// contraction indices) or across it ("oc").  One tile kernel serves all of them: a workgroup of four wavefronts (2 x 2) takes a tile of
// BM x BN outputs and walks the contraction in steps of 128 bytes per row, both operands' next step on its way into the other half
// of LDS while the matrix instructions (32x32x16 bf16, 32x32x2 f32; float32 accumulators) take this one.
#include <algorithm>

#include "cada_ops_internal.h"

namespace cada {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kStepBytes = 128;      // of a row per step of the contraction: 64 bf16 or 32 float32
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
  float *partial;            // [splits][M][N] where splits > 1: the sums are joined by k_join
  Epilogue epi;
};

// ---- operands in LDS ----
//
// A tile step of an operand is kStepBytes x (BM or BN) bytes, moved in pieces of 16 bytes; piece q lies at byte 16 q, and thread t
// of 256 moves the pieces 256 i + t, so that a wavefront fills consecutive kilobytes (what the LDS-direct load asks for).
//   kc: [outer][8 pieces]; row r keeps its pieces in the order p ^ (r % 8): a fragment read takes the same piece of 32 consecutive
//       rows, and 8 of them in this order cover the banks once.
//   oc: [k][outer]; bf16 rows keep their 32-byte chunks in the order c ^ swizzle(r): a transposing read takes 32 bytes of each of four
//       consecutive rows, which without it lie in the same banks.
template <typename T, bool KC, int BO> struct Side {
  static constexpr int E = Elem<T>::kPer16;
  static constexpr int kPieces = BO / 32;                       // per thread
  static constexpr int kRow16 = KC ? 8 : BO / E;                // pieces per row in LDS
  static constexpr int kBytes = kStepBytes * BO;
  __device__ static __forceinline__ int swizzle(int krow) { return sizeof(T) == 4 ? 0 : BO >= 128 ? (krow & 3) << 1 : krow & 2; }
  // row of LDS and source piece in it of thread t's i-th piece
  __device__ static __forceinline__ void place(int i, int t, int &row, int &piece) {
    const int q = i * 256 + t;
    row = q / kRow16;
    const int pos = q % kRow16;
    if constexpr (KC) piece = pos ^ (row & 7);
    else piece = pos ^ (swizzle(row) << 1);
  }
};

// The general way: through registers, any alignment, whatever lies outside [0, left) x [.., k_end) zero.
template <typename T, bool KC, int BO>
__device__ __forceinline__ void fetch(u32x4v (&reg)[BO / 32], const T *src, int64_t ld, int64_t left, int64_t k_left, int t) {
  typedef Side<T, KC, BO> S;
#pragma unroll
  for (int i = 0; i < S::kPieces; ++i) {
    int row, piece;
    S::place(i, t, row, piece);
    const int64_t along = KC ? k_left - piece * S::E : left - piece * S::E;        // elements from the piece's first to the row's end
    const bool row_in = KC ? row < left : row < k_left;
    reg[i] = load16_n(src + (int64_t)row * ld + piece * S::E, row_in ? along : 0);
  }
}
template <typename T, bool KC, int BO>
__device__ __forceinline__ void put(unsigned char *lds, const u32x4v (&reg)[BO / 32], int t) {
#pragma unroll
  for (int i = 0; i < BO / 32; ++i) *reinterpret_cast<u32x4v *>(lds + (i * 256 + t) * 16) = reg[i];
}

// The direct way: LDS-direct loads of a whole step.  Every row starts on a 16-byte boundary, and pieces lie in memory whole or not at
// all (kc: a step's are all there); one that does not is read from the last row or piece that does and enters outputs that nobody stores.
template <typename T, bool KC, int BO>
__device__ __forceinline__ void direct_offsets(uint32_t (&off)[BO / 32], int64_t ld, int64_t left, int t) {
  typedef Side<T, KC, BO> S;
#pragma unroll
  for (int i = 0; i < S::kPieces; ++i) {
    int row, piece;
    S::place(i, t, row, piece);
    const int64_t at = KC ? min((int64_t)row, left - 1) * ld + piece * S::E : (int64_t)row * ld + min((int64_t)piece * S::E, left - S::E);
    off[i] = (uint32_t)(at * (int64_t)sizeof(T));
  }
}
// (one kilobyte per wavefront: 16 bytes per lane to consecutive places)
__device__ __forceinline__ void direct_kilobyte(unsigned char *lds, const unsigned char *src) {
  __builtin_amdgcn_global_load_lds(src, (__attribute__((address_space(3))) void *)lds, 16, 0, 0);
}
template <int N>
__device__ __forceinline__ void direct(unsigned char *lds, const void *src, const uint32_t (&off)[N], int wave) {
#pragma unroll
  for (int i = 0; i < N; ++i) direct_kilobyte(lds + (i * 4 + wave) * 1024, static_cast<const unsigned char *>(src) + off[i]);
}

// ---- fragments ----
// Sub-step ks of four: lane l holds outer index l % 32; bf16: 8 contraction indices from 16 ks + 8 (l / 32) on; float32: 4 from 8 ks + 4 (l / 32) on, one
// for each of four matrix instructions (both operands in the same order, so the sum is complete).
template <bool KC, int BO>
__device__ __forceinline__ bf16x8 fragment(const unsigned char *lds, int outer, int ks, int lane, bf16) {
  if constexpr (KC) {
    const int row = outer + (lane & 31), piece = ks * 2 + (lane >> 5);
    return *reinterpret_cast<const bf16x8 *>(lds + row * kStepBytes + ((piece ^ (row & 7)) << 4));
  } else {
    // ds_read_b64_tr_b16 works on groups of 16 lanes: source lane s of a group passes the address of four consecutive units of row s / 4, and lane
    // l receives unit l of rows 0..3.  The groups are (units 0-15 | 16-31) x (rows 0-7 | 8-15 of the sub-step), two reads of four rows each.
    const int krow = ks * 16 + ((lane >> 5) << 3) + ((lane & 15) >> 2), chunk = (outer >> 4) + ((lane >> 4) & 1);
    const unsigned char *at = lds + krow * (BO * 2) + ((chunk ^ Side<bf16, false, BO>::swizzle(krow)) << 5) + ((lane & 3) << 3);
    typedef __attribute__((address_space(3))) i16x4 *lds_p;
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_p)(at)), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_p)(at + 4 * BO * 2));
    return __builtin_bit_cast(bf16x8, (i16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
}
template <bool KC, int BO>
__device__ __forceinline__ v4s fragment(const unsigned char *lds, int outer, int ks, int lane, float) {
  if constexpr (KC) {
    const int row = outer + (lane & 31), piece = ks * 2 + (lane >> 5);
    return *reinterpret_cast<const v4s *>(lds + row * kStepBytes + ((piece ^ (row & 7)) << 4));
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
    for (int i = 0; i < 8; ++i) f[i] = activation(f[i], e.act);
  }
  if (e.residual) {
    load8_n(static_cast<const T *>(e.residual) + m * e.ldr + n, left, o);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] += o[i];
  }
  store8_n(static_cast<T *>(e.out) + m * e.ldo + n, left, f);
}

template <typename T, int BM, int BN, bool AKC, bool BKC, bool DIRECT>
__device__ __forceinline__ void tile_product(const Product &p, int64_t tile, unsigned char *lds) {
  typedef Side<T, AKC, BM> SA;
  typedef Side<T, BKC, BN> SB;
  constexpr int WM = BM / 2, WN = BN / 2, FM = WM / 32, FN = WN / 32, kHalf = SA::kBytes + SB::kBytes, BK = kStep<T>;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), wm = (wave >> 1) * WM, wn = (wave & 1) * WN;
  // Tiles in bands of eight rows of tiles, columns slowest in a band: the tiles that run together share operands.
  const int64_t per_split = (int64_t)p.tiles_m * p.tiles_n;
  const int split = (int)(tile / per_split);
  const int64_t r = tile - split * per_split, band = r / (8 * (int64_t)p.tiles_n);
  const int in_band = (int)(r - band * 8 * p.tiles_n), rows_here = (int)min((int64_t)8, p.tiles_m - band * 8);
  const int64_t m0 = (band * 8 + in_band % rows_here) * BM, m_left = p.M - m0;
  const int n0 = in_band / rows_here * BN;
  const int64_t n_left = p.N - n0, k0 = split * p.k_per_split, k1 = min(p.K, k0 + p.k_per_split);
  const T *a = static_cast<const T *>(p.a) + (AKC ? m0 * p.lda + k0 : k0 * p.lda + m0);
  const T *b = static_cast<const T *>(p.b) + (BKC ? n0 * p.ldb + k0 : k0 * p.ldb + n0);
  const int64_t a_step = AKC ? BK : BK * p.lda, b_step = BKC ? BK : BK * p.ldb;
  const int steps = (int)((k1 - k0 + BK - 1) / BK), whole = (int)((k1 - k0) / BK);

  uint32_t oa[DIRECT ? SA::kPieces : 1], ob[DIRECT ? SB::kPieces : 1];
  if constexpr (DIRECT) {
    direct_offsets<T, AKC, BM>(oa, p.lda, AKC ? m_left : p.a_cols - m0, t);
    direct_offsets<T, BKC, BN>(ob, p.ldb, BKC ? n_left : p.b_cols - n0, t);
  }
  auto through_registers = [&](int s, unsigned char *dst) __attribute__((always_inline)) {
    u32x4v ra[SA::kPieces], rb[SB::kPieces];
    fetch<T, AKC, BM>(ra, a + s * a_step, p.lda, m_left, k1 - k0 - (int64_t)s * BK, t);
    fetch<T, BKC, BN>(rb, b + s * b_step, p.ldb, n_left, k1 - k0 - (int64_t)s * BK, t);
    put<T, AKC, BM>(dst, ra, t);
    put<T, BKC, BN>(dst + SA::kBytes, rb, t);
  };
  auto load_step = [&](int s, unsigned char *dst) __attribute__((always_inline)) {
    if constexpr (DIRECT) {
      if (s < whole) {
        direct(dst, a + s * a_step, oa, wave);
        direct(dst + SA::kBytes, b + s * b_step, ob, wave);
        return;
      }
    }
    through_registers(s, dst);
  };

  f32x16 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;

  load_step(0, lds);
  __syncthreads();
  for (int s = 0; s < steps; ++s) {
    unsigned char *here = lds + (s & 1) * kHalf;
    if (s + 1 < steps) load_step(s + 1, lds + ((s + 1) & 1) * kHalf);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      decltype(fragment<AKC, BM>(here, 0, 0, 0, T())) fa[FM], fb[FN];
#pragma unroll
      for (int i = 0; i < FM; ++i) fa[i] = fragment<AKC, BM>(here, wm + 32 * i, ks, lane, T());
#pragma unroll
      for (int j = 0; j < FN; ++j) fb[j] = fragment<BKC, BN>(here + SA::kBytes, wn + 32 * j, ks, lane, T());
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = multiply(fb[j], fa[i], acc[i][j]);        // lane: row l % 32 of the tile, four consecutive columns at a time
    }
    __syncthreads();
  }

  // Out through LDS, 32 rows of the wavefront's tile at a time, so that memory is met in eight consecutive columns per lane.
  constexpr int kLd = WN + 4, kLanes = WN / 8, kRows = 64 / kLanes;
  static_assert(4 * 32 * kLd * 4 <= 2 * kHalf, "the wavefronts' strips fit the operands' LDS");
  float *strip = reinterpret_cast<float *>(lds) + wave * 32 * kLd;
#pragma unroll
  for (int i = 0; i < FM; ++i) {
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<v4s *>(strip + (lane & 31) * kLd + 32 * j + 8 * q + 4 * (lane >> 5)) = v4s{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int rr = 0; rr < 32; rr += kRows) {
      const int row = rr + lane / kLanes, col = lane % kLanes * 8;
      const int64_t m = m0 + wm + 32 * i + row;
      const int n = n0 + wn + col;
      const float *src = strip + row * kLd + col;
      const v4s x = *reinterpret_cast<const v4s *>(src), y = *reinterpret_cast<const v4s *>(src + 4);
      float f[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
      if (m < p.M) {
        if (p.splits > 1) store8_n(p.partial + ((int64_t)split * p.M + m) * p.N + n, (int64_t)p.N - n, f);
        else finish8<T>(p.epi, m, n, (int64_t)p.N - n, f);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// Tiles of a launch, dealt to the eight XCDs in consecutive eighths (each has an L2 of its own).
__device__ __forceinline__ int64_t tile_of_block(int64_t total) {
  const int64_t per = (total + 7) / 8, t = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  return (blockIdx.x >> 3) < per && t < total ? t : -1;
}

template <typename T, int BM, int BN, bool DIRECT>
__global__ __launch_bounds__(256) void k_forward(const Product p) {
  __shared__ __align__(16) unsigned char lds[2 * kStepBytes * (BM + BN)];
  const int64_t tile = tile_of_block((int64_t)p.tiles_m * p.tiles_n * p.splits);
  if (tile >= 0) tile_product<T, BM, BN, true, false, DIRECT>(p, tile, lds);
}

// dx and dw in one launch (either may have no tiles).
template <typename T, int BM, int BN, bool DIRECT>
__global__ __launch_bounds__(256) void k_backward(const Product dx, const Product dw) {
  __shared__ __align__(16) unsigned char lds[2 * kStepBytes * (BM + BN)];
  const int64_t n_dw = (int64_t)dw.tiles_m * dw.tiles_n * dw.splits, n_dx = (int64_t)dx.tiles_m * dx.tiles_n * dx.splits;
  const int64_t tile = tile_of_block(n_dw + n_dx);
  if (tile < 0) return;
  if (tile < n_dw) tile_product<T, BM, BN, false, false, DIRECT>(dw, tile, lds);
  else tile_product<T, BM, BN, true, true, DIRECT>(dx, tile - n_dw, lds);
}

// Joins the sums of a split contraction, in the order of the splits, and finishes them; eight columns per thread.
struct Join {
  Product p[2];
  int64_t groups[2];         // M * ceil(N / 8), 0 where there is nothing to join
  const float *db_part;      // [db_parts][N of the second product] or null
  void *db;
  int db_parts, db_n;
};
template <typename T>
__global__ __launch_bounds__(256) void k_join(const Join j) {
  int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (g < j.groups[i]) {
      const Product &p = j.p[i];
      const int per = (p.N + 7) / 8;
      const int64_t m = g / per;
      const int n = (int)(g - m * per) * 8;
      const float *src = p.partial + m * p.N + n;
      const int64_t left = (int64_t)p.N - n;
      float f[8], o[8];
      load8_n(src, left, f);
      for (int s = 1; s < p.splits; ++s) {
        load8_n(src + (int64_t)s * p.M * p.N, left, o);
#pragma unroll
        for (int q = 0; q < 8; ++q) f[q] += o[q];
      }
      finish8<T>(p.epi, m, n, left, f);
      return;
    }
    g -= j.groups[i];
  }
  if (j.db_part && g < j.db_n) {
    float s = 0.f;
    for (int i = 0; i < j.db_parts; ++i) s += j.db_part[(int64_t)i * j.db_n + g];
    static_cast<T *>(j.db)[g] = from_f32<T>(s);
  }
}

// dz = dy * act'(pre), written in the operands' type with rows on 16-byte boundaries, and its column sums per block of rows.  A workgroup takes 256 columns:
// 32 lanes of eight columns each by eight rows at a time.
struct Signal {
  const void *dy, *pre;
  int64_t lddy, ldpre, rows, rows_per_block;
  int32_t n, act;
  void *dz;                  // or null
  int64_t lddz;
  float *db_part;            // [blocks of rows][n] or null
};
template <typename T>
__global__ __launch_bounds__(256) void k_signal(const Signal a) {
  __shared__ float part[8][32][9];
  const int t = threadIdx.x, cx = t & 31, ry = t >> 5;
  const int n = (blockIdx.x * 32 + cx) * 8;
  const int64_t left = (int64_t)a.n - n, r0 = (int64_t)blockIdx.y * a.rows_per_block, r1 = min(a.rows, r0 + a.rows_per_block);
  float sum[8] = {};
  if (left > 0) {
    for (int64_t r = r0 + ry; r < r1; r += 8) {
      float f[8], z[8];
      load8_n(static_cast<const T *>(a.dy) + r * a.lddy + n, left, f);
      if (a.act != CADA_ACT_NONE) {
        load8_n(static_cast<const T *>(a.pre) + r * a.ldpre + n, left, z);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] *= activation_slope(z[i], a.act);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] += f[i];
      if (a.dz) store8_n(static_cast<T *>(a.dz) + r * a.lddz + n, 8, f);        // (a whole group always: the rows have room for it, and the fill is zero)
    }
  }
  if (!a.db_part) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) part[ry][cx][i] = sum[i];
  __syncthreads();
  const int c = blockIdx.x * 256 + t;
  if (c < a.n) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += part[i][t >> 3][t & 7];
    a.db_part[(int64_t)blockIdx.y * a.n + c] = s;
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

constexpr int kCUs = 256;

// How a product is cut: the tile's edge, and into how many parts its contraction.
struct Cut { int tile, splits; int64_t k_per_split; };
Cut cut(int64_t M, int64_t N, int64_t K, int step) {
  Cut c;
  const int64_t big = ceil_div(M, 128) * ceil_div(N, 128);
  c.tile = big >= kCUs ? 128 : 64;
  const int64_t tiles = ceil_div(M, c.tile) * ceil_div(N, c.tile), steps = ceil_div(K, step);
  int64_t splits = 1;
  if (tiles < kCUs) splits = std::max<int64_t>(1, std::min({2 * kCUs / tiles, steps / 4, (int64_t)32}));
  const int64_t per = ceil_div(steps, splits);
  c.k_per_split = per * step;
  c.splits = (int)std::max<int64_t>(1, ceil_div(steps, per));
  return c;
}
size_t partial_bytes(const Cut &c, int64_t M, int64_t N) { return c.splits > 1 ? ops_align((size_t)c.splits * M * N * 4) : 0; }

void lay(Product *p, const Cut &c, const void *a, int64_t lda, const void *b, int64_t ldb, int64_t M, int64_t N, int64_t K, float *partial) {
  p->a_cols = M; p->b_cols = N;
  p->a = a; p->lda = lda; p->b = b; p->ldb = ldb; p->M = M; p->N = (int32_t)N; p->K = K;
  p->tiles_m = (int32_t)ceil_div(M, c.tile); p->tiles_n = (int32_t)ceil_div(N, c.tile);
  p->splits = c.splits; p->k_per_split = c.k_per_split; p->partial = c.splits > 1 ? partial : nullptr;
}
int64_t tiles_of(const Product &p) { return (int64_t)p.tiles_m * p.tiles_n * p.splits; }

// Whether a table can be read by LDS-direct loads: rows on 16-byte boundaries, offsets of a tile in 32 bits, and, read across the contraction, whole pieces.
bool direct_kc(const void *p, int64_t ld, size_t elem) { return aligned16(p, ld, elem) && 128 * ld * (int64_t)elem < (int64_t)1 << 31; }
bool direct_oc(const void *p, int64_t ld, int64_t cols, size_t elem) { return direct_kc(p, ld, elem) && cols % (int64_t)(16 / elem) == 0; }

bool check_shape(int64_t rows, int64_t in, int64_t out, int type, int act) {
  if (rows < 0 || rows > (int64_t)1 << 40) { set_error("rows must be in [0, 2^40] (got %lld)", (long long)rows); return false; }
  if (in < 1 || in > CADA_MAX_WIDTH || out < 1 || out > CADA_MAX_WIDTH) { set_error("in and out must be in [1, %d] (got %lld, %lld)", CADA_MAX_WIDTH, (long long)in, (long long)out); return false; }
  if (type != CADA_F32 && type != CADA_BF16) { set_error("type must be CADA_F32 or CADA_BF16 (got %d)", type); return false; }
  if (act < CADA_ACT_NONE || act > CADA_ACT_SILU) { set_error("act must be one of CADA_ACT_* (got %d)", act); return false; }
  const int64_t t = std::max({ceil_div(rows, 64) * ceil_div(out, 64), ceil_div(rows, 64) * ceil_div(in, 64), ceil_div(in, 64) * ceil_div(out, 64)});
  if (t > (int64_t)1 << 28) { set_error("more than 2^28 tiles of 64 x 64 outputs"); return false; }
  return true;
}
bool check_table(const char *name, const void *p, int64_t ld, int64_t cols, int type) {
  if (!p) { set_error("%s is NULL", name); return false; }
  if (ld < cols) { set_error("the row length of %s (%lld) is less than its %lld columns", name, (long long)ld, (long long)cols); return false; }
  if (reinterpret_cast<uintptr_t>(p) % type_bytes(type) != 0) { set_error("%s is not aligned to its elements", name); return false; }
  return true;
}

template <typename T>
int launch_forward(const Product &p, int tile, bool dir, hipStream_t st) {
  const unsigned grid = (unsigned)(ceil_div(tiles_of(p), 8) * 8);
  if (tile == 128) {
    if (dir) k_forward<T, 128, 128, true><<<grid, 256, 0, st>>>(p);
    else k_forward<T, 128, 128, false><<<grid, 256, 0, st>>>(p);
  } else {
    if (dir) k_forward<T, 64, 64, true><<<grid, 256, 0, st>>>(p);
    else k_forward<T, 64, 64, false><<<grid, 256, 0, st>>>(p);
  }
  return ops_launched("linear");
}
template <typename T>
int launch_backward(const Product &dx, const Product &dw, int tile, bool dir, hipStream_t st) {
  const unsigned grid = (unsigned)(ceil_div(tiles_of(dx) + tiles_of(dw), 8) * 8);
  if (tile == 128) {
    if (dir) k_backward<T, 128, 128, true><<<grid, 256, 0, st>>>(dx, dw);
    else k_backward<T, 128, 128, false><<<grid, 256, 0, st>>>(dx, dw);
  } else {
    if (dir) k_backward<T, 64, 64, true><<<grid, 256, 0, st>>>(dx, dw);
    else k_backward<T, 64, 64, false><<<grid, 256, 0, st>>>(dx, dw);
  }
  return ops_launched("linear gradients");
}
template <typename T>
int launch_join(Join &j, hipStream_t st) {
  int64_t total = j.db_part ? j.db_n : 0;
  for (int i = 0; i < 2; ++i) {
    j.groups[i] = j.p[i].splits > 1 ? j.p[i].M * ceil_div(j.p[i].N, 8) : 0;
    total += j.groups[i];
  }
  if (total == 0) return CADA_OK;
  k_join<T><<<(unsigned)ceil_div(total, 256), 256, 0, st>>>(j);
  return ops_launched("linear join");
}

struct BackwardPlan {
  Cut dx, dw;
  int64_t lddz, rows_per_block, row_blocks;
  size_t off_db, off_dx, off_dw, bytes;
};
BackwardPlan plan_backward(int64_t rows, int64_t in, int64_t out, int type) {
  BackwardPlan b;
  const size_t elem = type_bytes(type);
  const int step = kStepBytes / (int)elem;
  b.dx = cut(rows, in, out, step);
  b.dw = cut(in, out, rows, step);
  if (b.dx.tile != b.dw.tile) {      // one launch, one tile
    b.dx.tile = b.dw.tile = 64;
  }
  b.lddz = ceil_div(out, 8) * 8;
  b.rows_per_block = std::max<int64_t>(32, ceil_div(ceil_div(rows, 64), 8) * 8);
  b.row_blocks = ceil_div(rows, b.rows_per_block);
  size_t off = ops_align((size_t)rows * b.lddz * elem);
  b.off_db = off; off += ops_align((size_t)b.row_blocks * out * 4);
  b.off_dx = off; off += partial_bytes(b.dx, rows, in);
  b.off_dw = off; off += partial_bytes(b.dw, in, out);
  b.bytes = off;
  return b;
}

template <typename T>
int zero_table(void *p, int64_t ld, int64_t rows, int64_t n, hipStream_t st) {
  k_zero<T><<<(unsigned)std::min<int64_t>(ceil_div(rows * n, 256), 4096), 256, 0, st>>>(static_cast<T *>(p), ld, rows, n);
  return ops_launched("linear clear");
}

template <typename T>
int backward(const cada_linear_grad *a) {
  hipStream_t st = static_cast<hipStream_t>(a->stream);
  if (a->rows == 0) {
    if (a->dw) if (int rc = zero_table<T>(a->dw, a->lddw, a->in, a->out, st)) return rc;
    if (a->db) return zero_table<T>(a->db, a->out, 1, a->out, st);
    return CADA_OK;
  }
  const BackwardPlan b = plan_backward(a->rows, a->in, a->out, a->type);
  char *ws = static_cast<char *>(a->workspace);
  // dz in the workspace, unless dy itself will do
  const bool products = a->dx || a->dw;
  const bool own_dz = products && (a->act != CADA_ACT_NONE || !direct_oc(a->dy, a->lddy, a->out, sizeof(T)));
  if (own_dz || a->db) {
    Signal s{};
    s.dy = a->dy; s.lddy = a->lddy; s.pre = a->pre; s.ldpre = a->ldpre; s.rows = a->rows; s.rows_per_block = b.rows_per_block; s.n = (int32_t)a->out; s.act = a->act;
    s.dz = own_dz ? ws : nullptr; s.lddz = b.lddz;
    s.db_part = a->db ? reinterpret_cast<float *>(ws + b.off_db) : nullptr;
    k_signal<T><<<dim3((unsigned)ceil_div(a->out, 256), (unsigned)b.row_blocks), 256, 0, st>>>(s);
    if (int rc = ops_launched("linear signal")) return rc;
  }
  const void *dz = own_dz ? ws : a->dy;
  // (dz's rows in the workspace are filled with zeros up to whole pieces)
  const int64_t lddz = own_dz ? b.lddz : a->lddy;
  Product dx{}, dw{};
  bool dir = true;
  if (a->dx) {
    lay(&dx, b.dx, dz, lddz, a->w, a->ldw, a->rows, a->in, a->out, reinterpret_cast<float *>(ws + b.off_dx));
    dx.epi = Epilogue{nullptr, nullptr, nullptr, a->dx, 0, 0, a->lddx, CADA_ACT_NONE};
    dir = dir && direct_kc(a->w, a->ldw, sizeof(T)) && direct_kc(dz, lddz, sizeof(T));
  }
  if (a->dw) {
    lay(&dw, b.dw, a->x, a->ldx, dz, lddz, a->in, a->out, a->rows, reinterpret_cast<float *>(ws + b.off_dw));
    dw.epi = Epilogue{nullptr, nullptr, nullptr, a->dw, 0, 0, a->lddw, CADA_ACT_NONE};
    dw.b_cols = own_dz ? b.lddz : a->out;
    dir = dir && direct_oc(a->x, a->ldx, a->in, sizeof(T)) && direct_oc(dz, lddz, dw.b_cols, sizeof(T));
  }
  if (products) if (int rc = launch_backward<T>(dx, dw, a->dx ? b.dx.tile : b.dw.tile, dir, st)) return rc;
  Join j{};
  j.p[0] = dx; j.p[1] = dw;
  if (a->db) { j.db_part = reinterpret_cast<float *>(ws + b.off_db); j.db = a->db; j.db_parts = (int)b.row_blocks; j.db_n = (int)a->out; }
  return launch_join<T>(j, st);
}

template <typename T>
int forward(const cada_linear *a) {
  hipStream_t st = static_cast<hipStream_t>(a->stream);
  const Cut c = cut(a->rows, a->out, a->in, kStep<T>);
  Product p{};
  lay(&p, c, a->x, a->ldx, a->w, a->ldw, a->rows, a->out, a->in, static_cast<float *>(a->workspace));
  p.epi = Epilogue{a->bias, a->residual, a->pre, a->y, a->ldr, a->ldpre, a->ldy, a->act};
  const bool dir = direct_kc(a->x, a->ldx, sizeof(T)) && direct_oc(a->w, a->ldw, a->out, sizeof(T));
  if (int rc = launch_forward<T>(p, c.tile, dir, st)) return rc;
  Join j{};
  j.p[0] = p;
  return launch_join<T>(j, st);
}

size_t forward_workspace(const cada_linear *a) {
  if (a->rows == 0) return 0;
  return partial_bytes(cut(a->rows, a->out, a->in, kStepBytes / (int)type_bytes(a->type)), a->rows, a->out);
}
size_t backward_workspace(const cada_linear_grad *a) { return a->rows == 0 ? 0 : plan_backward(a->rows, a->in, a->out, a->type).bytes; }

}  // namespace

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
  a->workspace_bytes = forward_workspace(a);
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
  if (int rc = ops_check_workspace(a->workspace, a->workspace_bytes, forward_workspace(a))) return rc;
  return a->type == CADA_BF16 ? forward<bf16>(a) : forward<float>(a);
}

int cada_linear_backward_workspace(cada_linear_grad *a) {
  if (!a) { set_error("the arguments are NULL"); return CADA_EINVAL; }
  if (!check_shape(a->rows, a->in, a->out, a->type, a->act)) return CADA_EINVAL;
  a->workspace_bytes = backward_workspace(a);
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
    if (int rc = ops_check_workspace(a->workspace, a->workspace_bytes, backward_workspace(a))) return rc;
  }
  if (a->dw && !check_table("dw", a->dw, a->lddw, a->out, a->type)) return CADA_EINVAL;
  if (a->db && !check_table("db", a->db, a->out, a->out, a->type)) return CADA_EINVAL;
  return a->type == CADA_BF16 ? backward<bf16>(a) : backward<float>(a);
}

}  // extern "C"
