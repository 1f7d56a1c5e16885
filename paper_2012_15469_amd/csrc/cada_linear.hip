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

#include "cada_linear_tiles.h"

namespace cada {
namespace {

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
  else finish8<T>(p, m, n, left, f);
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
template <typename T, int BM, int BN, int WY, int WX, bool DIRECT, int STAGES, int KW, bool PIECES>
__global__ __launch_bounds__(64 * WY * WX * KW) void k_backward(const Product dx, const Product dw) {
  __shared__ __align__(16) unsigned char lds[tile_lds(BM, BN, STAGES, KW)];
  const Turn turn = backward_tile(dx, dw);
  if (turn.tile == ~0u) return;
  if (turn.dw) tile_product<T, BM, BN, WY, WX, false, false, DIRECT, STAGES, KW, NO_SIGNAL>(dw, turn.tile, lds, ToTable<PIECES>());
  else tile_product<T, BM, BN, WY, WX, true, true, DIRECT, STAGES, KW, NO_SIGNAL>(dx, turn.tile, lds, ToTable<PIECES>());
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
    finish8<T>(p, m, (int)n, 1, f);
    if (SIGNAL == B_SIGNAL && p.db && m == 0) static_cast<T *>(p.db)[n] = from_f32<T>(column);
  }
}

template <typename T, bool PIECES>
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
      finish8<T, PIECES>(p, m, n, left, f);
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
    static_cast<T *>(j.db)[c] = from_f32<T>(PIECES ? s * *j.db_factor : s);
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
bool check_shape(int64_t rows, int64_t in, int64_t out, int type, int act) {
  if (rows < 0 || rows > (int64_t)1 << 40) { set_error("rows must be in [0, 2^40] (got %lld)", (long long)rows); return false; }
  if (in < 1 || in > CADA_MAX_WIDTH || out < 1 || out > CADA_MAX_WIDTH) { set_error("in and out must be in [1, %d] (got %lld, %lld)", CADA_MAX_WIDTH, (long long)in, (long long)out); return false; }
  if (type != CADA_F32 && type != CADA_BF16) { set_error("type must be CADA_F32 or CADA_BF16 (got %d)", type); return false; }
  if (act < CADA_ACT_NONE || act > CADA_ACT_SILU) { set_error("act must be one of CADA_ACT_* (got %d)", act); return false; }
  const int64_t t = std::max({ceil_div(rows, 64) * ceil_div(out, 64), ceil_div(rows, 64) * ceil_div(in, 64), ceil_div(in, 64) * ceil_div(out, 64)});
  if (t > kMostTiles) { set_error("more than %lld tiles of 64 x 64 outputs", (long long)kMostTiles); return false; }
  return true;
}
// ---- forward ----

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
void forward_tiles_of(int tile, bool direct, const Product &p, hipStream_t st) {
  if (tile == 32) forward_tiles<T, 32, 1, 1, 4>(p, direct, st);
  if (tile == 64) forward_tiles<T, 64, 2, 2, 1>(p, direct, st);
  if constexpr (sizeof(T) == 2) {
    if (tile == 128) forward_tiles<T, 128, 2, 4, 1>(p, direct, st);
    if (tile == 256) forward_tiles<T, 256, 2, 4, 1>(p, direct, st);
  }
}

template <typename T, bool PIECES>
int launch_join(Join &j, hipStream_t st) {
  int64_t total = 0;
  for (int i = 0; i < 2; ++i) {
    j.groups[i] = j.p[i].partial ? j.p[i].M * ceil_div(j.p[i].N, 8) : 0;
    total += j.groups[i];
  }
  j.db_block = (unsigned)ceil_div(total, 256);
  const unsigned grid = j.db_block + (j.db_part ? (unsigned)ceil_div(j.db_n, 32) : 0);
  if (grid == 0) return CADA_OK;
  k_join<T, PIECES><<<grid, 256, 0, st>>>(j);
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
  } else {
    forward_tiles_of<T>(f.cut.tile, f.direct, p, st);
  }
  if (int rc = ops_launched("linear")) return rc;
  if (p.splits == 1) return CADA_OK;
  Join j{};
  j.p[0] = p;
  return launch_join<T, false>(j, st);
}

// ---- backward ----

template <typename T>
int zero_table(void *p, int64_t ld, int64_t rows, int64_t n, hipStream_t st) {
  k_zero<T><<<(unsigned)std::min<int64_t>(ceil_div(rows * n, 256), 4096), 256, 0, st>>>(static_cast<T *>(p), ld, rows, n);
  return ops_launched("linear clear");
}

template <typename T, int E, int WY, int WX, int KW, bool PIECES>
void backward_tiles(const Product &dx, const Product &dw, bool dir, hipStream_t st) {
  const unsigned grid = (unsigned)((ceil_div(tiles_of(dx), 8) + ceil_div(tiles_of(dw), 8)) * 8);
  if constexpr (E <= 64) {
    if (!dir) { k_backward<T, E, E, WY, WX, false, 2, KW, PIECES><<<grid, 64 * WY * WX * KW, 0, st>>>(dx, dw); return; }
  }
  if constexpr (E < 256) {
    if (deep(E, tiles_of(dx) + tiles_of(dw))) { k_backward<T, E, E, WY, WX, true, 4, KW, PIECES><<<grid, 64 * WY * WX * KW, 0, st>>>(dx, dw); return; }
  }
  k_backward<T, E, E, WY, WX, true, 2, KW, PIECES><<<grid, 64 * WY * WX * KW, 0, st>>>(dx, dw);
}

template <typename T, bool PIECES>
int products(int tile, bool direct, const Product &dx, const Product &dw, hipStream_t st) {
  if (tile == 32) backward_tiles<T, 32, 1, 1, 4, PIECES>(dx, dw, direct, st);
  if (tile == 64) backward_tiles<T, 64, 2, 2, 1, PIECES>(dx, dw, direct, st);
  if constexpr (sizeof(T) == 2) {
    if (tile == 128) backward_tiles<T, 128, 2, 4, 1, PIECES>(dx, dw, direct, st);
    if (tile == 256) backward_tiles<T, 256, 2, 4, 1, PIECES>(dx, dw, direct, st);
  }
  return ops_launched("linear gradients");
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
    } else if (int rc = products<T, false>(tile, b.direct, dx, dw, st)) {
      return rc;
    }
    if (int rc = ops_launched("linear gradients")) return rc;
  }
  Join j{};
  j.p[0] = dx; j.p[1] = dw;
  if (a->db && (!db_by_products || b.dw.splits > 1)) { j.db_part = db_part; j.db = a->db; j.db_parts = (int)b.row_blocks; j.db_n = (int)a->out; }
  return launch_join<T, false>(j, st);
}

}  // namespace

int linear_sums(int type, int tile, bool direct, const Product &p, hipStream_t st) {
  if (type == CADA_BF16) forward_tiles_of<bf16>(tile, direct, p, st);
  else forward_tiles_of<float>(tile, direct, p, st);
  return ops_launched("linear");
}
int linear_products(int type, int tile, bool direct, const Product &dx, const Product &dw, hipStream_t st) { return type == CADA_BF16 ? products<bf16, true>(tile, direct, dx, dw, st) : products<float, true>(tile, direct, dx, dw, st); }
int linear_join(int type, Join &j, hipStream_t st) { return type == CADA_BF16 ? launch_join<bf16, true>(j, st) : launch_join<float, true>(j, st); }

bool ops_check_table(const char *name, const void *p, int64_t ld, int64_t cols, int type) {
  if (!p) { set_error("%s is NULL", name); return false; }
  if (ld < cols) { set_error("the row length of %s (%lld) is less than its %lld columns", name, (long long)ld, (long long)cols); return false; }
  if (reinterpret_cast<uintptr_t>(p) % type_bytes(type) != 0) { set_error("%s is not aligned to its elements", name); return false; }
  return true;
}
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
  if (!ops_check_table("x", a->x, a->ldx, a->in, a->type) || !ops_check_table("w", a->w, a->ldw, a->out, a->type) || !ops_check_table("y", a->y, a->ldy, a->out, a->type)) return CADA_EINVAL;
  if (a->bias && !ops_check_table("bias", a->bias, a->out, a->out, a->type)) return CADA_EINVAL;
  if (a->residual && !ops_check_table("residual", a->residual, a->ldr, a->out, a->type)) return CADA_EINVAL;
  if (a->pre && !ops_check_table("pre", a->pre, a->ldpre, a->out, a->type)) return CADA_EINVAL;
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
    if ((a->dx || a->dw || a->db) && !ops_check_table("dy", a->dy, a->lddy, a->out, a->type)) return CADA_EINVAL;
    if ((a->dx || a->dw || a->db) && a->act != CADA_ACT_NONE && !ops_check_table("pre", a->pre, a->ldpre, a->out, a->type)) return CADA_EINVAL;
    if (a->dx && (!ops_check_table("w", a->w, a->ldw, a->out, a->type) || !ops_check_table("dx", a->dx, a->lddx, a->in, a->type))) return CADA_EINVAL;
    if (a->dw && !ops_check_table("x", a->x, a->ldx, a->in, a->type)) return CADA_EINVAL;
  }
  if (a->dw && !ops_check_table("dw", a->dw, a->lddw, a->out, a->type)) return CADA_EINVAL;
  if (a->db && !ops_check_table("db", a->db, a->out, a->out, a->type)) return CADA_EINVAL;
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
