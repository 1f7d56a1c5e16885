// Layer norm over the rows of a table, forward and backward (cada_ops.h).
//
// A group of 4 to 512 lanes takes a row, by its length, and keeps it in registers as it was read: the mean, then the squared distances from it (two passes over
// registers; a sum of squares would cancel), then the row out.  A workgroup goes on to further rows with the weights in registers, and asks for the next row before it
// works on this one.  The gradient's sums over the rows stay in the lanes that have those columns, one part per workgroup is written, and a second launch adds the parts
// up in their order.  Bound by memory: a row is read once and written once.  Rows beyond what a workgroup holds are read again, and their column sums are a kernel of their own.
// Forward, 16384 x 4096 bf16: 50 us, 5.4 TB/s (one row 2.7 us: the launch); backward with a residual: 102 to 108 us, 5.0 to 5.3 TB/s, and 5 us for the join.
#include <algorithm>

#include "cada_ops_internal.h"

namespace cada {
namespace {

struct Norm {
  const void *x, *weight, *bias;
  void *y;
  float *mean, *rstd;
  int64_t rows, ldx, ldy;
  int32_t width;
  float eps;
};
struct NormGrad {
  const void *dy, *x, *weight, *residual;
  const float *mean, *rstd;
  void *dx, *dw, *db;
  float *part;               // [2][parts][width]: of dw, of db
  int64_t rows, lddy, ldx, ldr, lddx;
  int32_t width, parts;
  int64_t rows_per_part;     // of the wide rows' column sums
};

template <int LANES> constexpr int kThreads = LANES <= 64 ? 256 : LANES;
template <int LANES> constexpr int kRowsAtOnce = kThreads<LANES> / LANES;

// Sums of N values over the LANES lanes of a row's group; every lane gets them.  `part` is not read by an earlier call that some wavefront may still be in: callers take two in turn.
template <int LANES, int N> __device__ __forceinline__ void group_sum(float (&x)[N], float (*part)[N]) {
  constexpr int W = LANES < 64 ? LANES : 64;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) x[i] += __shfl_xor(x[i], o, 64);
  if constexpr (LANES > 64) {
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) part[threadIdx.x >> 6][i] = x[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = part[0][i];
#pragma unroll
      for (int w = 1; w < LANES / 64; ++w) x[i] += part[w][i];
    }
  }
}

// A row in pieces of 16 bytes, which the lanes take in turn, and the few columns behind the last whole piece, one per lane.  What does not exist is zero.
template <typename T, int LANES, int V> struct Pieces {
  static constexpr int E = Elem<T>::kPer16;
  u32x4v raw[V];
  float behind;
  __device__ __forceinline__ void load(const T *p, int width, int lane) {
    const int whole = width / E * E;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * LANES + lane) * E;
      raw[v] = u32x4v{0, 0, 0, 0};
      if (c < whole) raw[v] = load16(p + c);
    }
    behind = lane < width - whole ? to_f32(p[whole + lane]) : 0.f;
  }
  // (The empty asm keeps the compiler from holding the row as float32 from one use to the next: twice the registers of bf16 pieces, which spill.)
  __device__ __forceinline__ void get(int v, float (&f)[E]) {
    asm volatile("" : "+v"(raw[v]));
    unpack<T>(raw[v], f);
  }
};

template <typename T, int LANES, int V>
__global__ __launch_bounds__(kThreads<LANES>, LANES >= 512 ? 2 : 4) void k_norm(const Norm a) {
  constexpr int E = Elem<T>::kPer16, kAtOnce = kRowsAtOnce<LANES>;
  __shared__ float part[2][LANES > 64 ? LANES / 64 : 1][1];
  const int lane = threadIdx.x % LANES, whole = a.width / E * E;
  static_assert(LANES >= E, "one column per lane behind the last piece");
  const T *x = static_cast<const T *>(a.x);
  T *y = static_cast<T *>(a.y);
  const float share = 1.f / (float)a.width;
  const int64_t stride = (int64_t)gridDim.x * kAtOnce, last = a.rows - 1;
  int64_t r = (int64_t)blockIdx.x * kAtOnce + threadIdx.x / LANES;
  Pieces<T, LANES, V> row, next, weight, bias;
  row.load(x + min(r, last) * a.ldx, a.width, lane);
  if (a.weight) weight.load(static_cast<const T *>(a.weight), a.width, lane);
  if (a.bias) bias.load(static_cast<const T *>(a.bias), a.width, lane);
  // (a workgroup's groups go on together: the sums of long rows meet at barriers)
  for (int64_t r0 = (int64_t)blockIdx.x * kAtOnce; r0 < a.rows; r0 += stride, r += stride) {
    const bool here = r < a.rows, more = r0 + stride < a.rows;
    if (more) next.load(x + min(r + stride, last) * a.ldx, a.width, lane);
    float f[E], mean[1] = {row.behind}, var[1] = {0.f};
#pragma unroll
    for (int v = 0; v < V; ++v) {
      row.get(v, f);
#pragma unroll
      for (int e = 0; e < E; ++e) mean[0] += f[e];
    }
    group_sum<LANES>(mean, part[0]);
    mean[0] *= share;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      row.get(v, f);
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) s = fmaf(f[e] - mean[0], f[e] - mean[0], s);
      var[0] += (v * LANES + lane) * E < whole ? s : 0.f;
    }
    const float d = row.behind - mean[0];
    var[0] += lane < a.width - whole ? d * d : 0.f;
    group_sum<LANES>(var, part[1]);
    const float rstd = 1.f / sqrtf(fmaf(var[0], share, a.eps));
    if (here) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int c = (v * LANES + lane) * E;
        float g[E];
        row.get(v, f);
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = (f[e] - mean[0]) * rstd;
        if (a.weight) {
          weight.get(v, g);
#pragma unroll
          for (int e = 0; e < E; ++e) f[e] *= g[e];
        }
        if (a.bias) {
          bias.get(v, g);
#pragma unroll
          for (int e = 0; e < E; ++e) f[e] += g[e];
        }
        if (c < whole) store16(y + r * a.ldy + c, pack<T>(f));
      }
      if (lane < a.width - whole) y[r * a.ldy + whole + lane] = from_f32<T>(d * rstd * (a.weight ? weight.behind : 1.f) + (a.bias ? bias.behind : 0.f));
      if (lane == 0 && a.mean) a.mean[r] = mean[0];
      if (lane == 0 && a.rstd) a.rstd[r] = rstd;
    }
    if (more) row = next;
  }
}

// Rows that no group's registers hold: a workgroup reads a row three times, the second and third from caches (4096 x 40000 bf16: 189 us, 3.5 TB/s of the row in and out).
template <typename T>
__global__ __launch_bounds__(1024) void k_norm_wide(const Norm a) {
  __shared__ float part[2][16][1];
  const float share = 1.f / (float)a.width;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T *x = static_cast<const T *>(a.x) + r * a.ldx;
    T *y = static_cast<T *>(a.y) + r * a.ldy;
    float mean[1] = {0.f}, var[1] = {0.f}, f[8], g[8];
    for (int c = threadIdx.x * 8; c < a.width; c += 8192) {
      load8_n(x + c, a.width - c, f);
#pragma unroll
      for (int e = 0; e < 8; ++e) mean[0] += f[e];
    }
    group_sum<1024>(mean, part[0]);
    mean[0] *= share;
    for (int c = threadIdx.x * 8; c < a.width; c += 8192) {
      load8_n(x + c, a.width - c, f);
#pragma unroll
      for (int e = 0; e < 8; ++e) var[0] += c + e < a.width ? (f[e] - mean[0]) * (f[e] - mean[0]) : 0.f;
    }
    group_sum<1024>(var, part[1]);
    const float rstd = 1.f / sqrtf(fmaf(var[0], share, a.eps));
    for (int c = threadIdx.x * 8; c < a.width; c += 8192) {
      load8_n(x + c, a.width - c, f);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = (f[e] - mean[0]) * rstd;
      if (a.weight) {
        load8_n(static_cast<const T *>(a.weight) + c, a.width - c, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] *= g[e];
      }
      if (a.bias) {
        load8_n(static_cast<const T *>(a.bias) + c, a.width - c, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] += g[e];
      }
      store8_n(y + c, a.width - c, f);
    }
    if (threadIdx.x == 0 && a.mean) a.mean[r] = mean[0];
    if (threadIdx.x == 0 && a.rstd) a.rstd[r] = rstd;
  }
}

// dx of the rows, and the sums of dw and db over a workgroup's rows: these cross no lanes until a workgroup ends, only the two sums of dx do, for each row
// (2400 x 617 float32: 8.8 us in two turns of 300 workgroups; 2048 rows in one turn of 512 6.6, a single row 3.7).
template <typename T, int LANES, int V>
__global__ __launch_bounds__(kThreads<LANES>, 2) void k_norm_grad(const NormGrad a) {
  constexpr int E = Elem<T>::kPer16, kAtOnce = kRowsAtOnce<LANES>, kCols = LANES * V * E;
  constexpr bool kAhead = V * E <= 16;        // (registers for a second row)
  constexpr bool kHeld = V < 8;              // (and for the weights and what is added, which are read where they are used otherwise: 8000 x 16000 float32 920 us with both held, 640 without)
  __shared__ float part[2][LANES > 64 ? LANES / 64 : 1][2];
  __shared__ float sums[LANES <= 64 ? kAtOnce * kCols : 1];
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES, whole = a.width / E * E;
  const T *dy = static_cast<const T *>(a.dy), *x = static_cast<const T *>(a.x), *res = static_cast<const T *>(a.residual);
  T *dx = static_cast<T *>(a.dx);
  const float share = 1.f / (float)a.width;
  const int64_t stride = (int64_t)gridDim.x * kAtOnce, last = a.rows - 1;
  int64_t r = (int64_t)blockIdx.x * kAtOnce + group;
  struct Row { Pieces<T, LANES, V> x, dy, res; float mean, rstd; } row, next;
  Pieces<T, LANES, V> weight;
  auto load = [&](Row &to, int64_t at) __attribute__((always_inline)) {
    at = min(at, last);
    to.x.load(x + at * a.ldx, a.width, lane);
    to.dy.load(dy + at * a.lddy, a.width, lane);
    if (kHeld && res) to.res.load(res + at * a.ldr, a.width, lane);
    to.mean = a.mean[at];
    to.rstd = a.rstd[at];
  };
  load(row, r);
  const T *w = static_cast<const T *>(a.weight);
  weight.behind = 1.f;
  if (kHeld && w) weight.load(w, a.width, lane);
  else if (w && lane < a.width - whole) weight.behind = to_f32(w[whole + lane]);
  // a piece of the weights
  auto weights = [&](int v, float (&f)[E]) __attribute__((always_inline)) {
    if constexpr (kHeld) return weight.get(v, f);
    const int c = (v * LANES + lane) * E;
    unpack<T>(c < whole ? load16(w + c) : u32x4v{0, 0, 0, 0}, f);
  };
  float dw[V][E] = {}, db[V][E] = {}, dw_behind = 0.f, db_behind = 0.f;
  int turn = 0;
  for (int64_t r0 = (int64_t)blockIdx.x * kAtOnce; r0 < a.rows; r0 += stride, r += stride, turn ^= 1) {
    const bool here = r < a.rows, more = r0 + stride < a.rows;
    if (kAhead && more) load(next, r + stride);
    const float mean = row.mean, rstd = row.rstd;
    // sums of g = dy * weight and of g u, u = (x - mean) rstd, over the row
    float s[2] = {0.f, 0.f}, f[E], u[E], g[E];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      row.dy.get(v, f);
      row.x.get(v, u);
      if (w) weights(v, g);
      // (a column that does not exist holds zero: its u, which may pass float32 where no column's of the row does, is nothing)
      const float rstd_here = (v * LANES + lane) * E < whole ? rstd : 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        u[e] = (u[e] - mean) * rstd_here;
        if (here) {
          dw[v][e] = fmaf(f[e], u[e], dw[v][e]);
          db[v][e] += f[e];
        }
        if (w) f[e] *= g[e];
        s[0] += f[e];
        s[1] = fmaf(f[e], u[e], s[1]);
      }
      if constexpr (!kAhead) __builtin_amdgcn_sched_barrier(0);        // (piece by piece: interleaved, they spill)
    }
    const float u_behind = (row.x.behind - mean) * (lane < a.width - whole ? rstd : 0.f), g_behind = row.dy.behind * (w ? weight.behind : 1.f);
    if (here) {
      dw_behind = fmaf(row.dy.behind, u_behind, dw_behind);
      db_behind += row.dy.behind;
    }
    s[0] += g_behind;
    s[1] = fmaf(g_behind, u_behind, s[1]);
    if (a.dx) {
      group_sum<LANES>(s, part[turn]);
      const float mean_g = s[0] * share, mean_gu = s[1] * share;
      if (here) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int c = (v * LANES + lane) * E;
          row.dy.get(v, f);
          row.x.get(v, u);
          if (w) {
            weights(v, g);
#pragma unroll
            for (int e = 0; e < E; ++e) f[e] *= g[e];
          }
#pragma unroll
          for (int e = 0; e < E; ++e) f[e] = rstd * (f[e] - mean_g - (u[e] - mean) * rstd * mean_gu);
          if (res) {
            if constexpr (kHeld) row.res.get(v, g);
            else unpack<T>(c < whole ? load16(res + r * a.ldr + c) : u32x4v{0, 0, 0, 0}, g);
#pragma unroll
            for (int e = 0; e < E; ++e) f[e] += g[e];
          }
          if (c < whole) store16(dx + r * a.lddx + c, pack<T>(f));
          if constexpr (!kAhead) __builtin_amdgcn_sched_barrier(0);
        }
        if (lane < a.width - whole) dx[r * a.lddx + whole + lane] = from_f32<T>(rstd * (g_behind - mean_g - u_behind * mean_gu) + (!res ? 0.f : kHeld ? row.res.behind : to_f32(res[r * a.ldr + whole + lane])));
      }
    }
    if (more) {
      if (kAhead) row = next;
      else load(row, r + stride);
    }
  }
  if (!a.dw && !a.db) return;
  const bool alone = gridDim.x == 1;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    T *out = static_cast<T *>(which == 0 ? a.dw : a.db);
    if (!out) continue;
    float *to = a.part + ((int64_t)which * a.parts + blockIdx.x) * a.width;
    if constexpr (LANES <= 64) {
      // the groups' sums of a column, in the groups' order
      __syncthreads();
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int c = (v * LANES + lane) * E;
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (c < whole) sums[group * kCols + c + e] = which == 0 ? dw[v][e] : db[v][e];
      }
      if (lane < a.width - whole) sums[group * kCols + whole + lane] = which == 0 ? dw_behind : db_behind;
      __syncthreads();
      for (int c = threadIdx.x; c < a.width; c += 256) {
        float t = sums[c];
        for (int i = 1; i < kAtOnce; ++i) t += sums[i * kCols + c];
        if (alone) out[c] = from_f32<T>(t);
        else to[c] = t;
      }
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int c = (v * LANES + lane) * E;
        if (c >= whole) continue;
        const float (&t)[E] = which == 0 ? dw[v] : db[v];
        if (alone) {
          store16(out + c, pack<T>(t));
        } else {
#pragma unroll
          for (int e = 0; e < E; e += 4) store16(to + c + e, pack<float>({t[e], t[e + 1], t[e + 2], t[e + 3]}));
        }
      }
      if (lane < a.width - whole) {
        const float t = which == 0 ? dw_behind : db_behind;
        if (alone) out[whole + lane] = from_f32<T>(t);
        else to[whole + lane] = t;
      }
    }
  }
}

// Wide rows: the column sums over a part of the rows, eight columns per thread (before dx is written, which may lie where dy does); then dx (4096 x 20000 float32: 76 and 201 us, 8.6 TB/s for tables
// that the caches hold in part, and 4.9).
template <typename T>
__global__ __launch_bounds__(256) void k_norm_grad_columns(const NormGrad a) {
  const int c = ((int)blockIdx.x * 256 + threadIdx.x) * 8, left = a.width - c;
  if (left <= 0) return;
  const int64_t r0 = (int64_t)blockIdx.y * a.rows_per_part, r1 = min(a.rows, r0 + a.rows_per_part);
  float dw[8] = {}, db[8] = {};
#pragma unroll 4
  for (int64_t r = r0; r < r1; ++r) {
    float f[8], u[8];
    load8_n(static_cast<const T *>(a.dy) + r * a.lddy + c, left, f);
    load8_n(static_cast<const T *>(a.x) + r * a.ldx + c, left, u);
    const float mean = a.mean[r], rstd = a.rstd[r];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      dw[e] = fmaf(f[e], (u[e] - mean) * rstd, dw[e]);
      db[e] += f[e];
    }
  }
  if (a.dw) store8_n(a.part + (int64_t)blockIdx.y * a.width + c, left, dw);
  if (a.db) store8_n(a.part + ((int64_t)a.parts + blockIdx.y) * a.width + c, left, db);
}
template <typename T>
__global__ __launch_bounds__(1024) void k_norm_grad_wide(const NormGrad a) {
  __shared__ float part[2][16][2];
  const float share = 1.f / (float)a.width;
  int turn = 0;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x, turn ^= 1) {
    const T *dy = static_cast<const T *>(a.dy) + r * a.lddy, *x = static_cast<const T *>(a.x) + r * a.ldx, *res = static_cast<const T *>(a.residual);
    T *dx = static_cast<T *>(a.dx) + r * a.lddx;
    const float mean = a.mean[r], rstd = a.rstd[r];
    float s[2] = {0.f, 0.f}, f[8], u[8], g[8];
    auto at = [&](int c) __attribute__((always_inline)) {        // f = dy * weight, u
      load8_n(dy + c, a.width - c, f);
      load8_n(x + c, a.width - c, u);
      if (a.weight) {
        load8_n(static_cast<const T *>(a.weight) + c, a.width - c, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] *= g[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) u[e] = (u[e] - mean) * rstd;
    };
    for (int c = threadIdx.x * 8; c < a.width; c += 8192) {
      at(c);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s[0] += f[e];
        s[1] = fmaf(f[e], c + e < a.width ? u[e] : 0.f, s[1]);
      }
    }
    group_sum<1024>(s, part[turn]);
    for (int c = threadIdx.x * 8; c < a.width; c += 8192) {
      at(c);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = rstd * (f[e] - s[0] * share - u[e] * (s[1] * share));
      if (res) {
        load8_n(res + r * a.ldr + c, a.width - c, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] += g[e];
      }
      store8_n(dx + c, a.width - c, f);
    }
  }
}

// The parts of the column sums, in their order: a workgroup takes 32 columns, LANES lanes of each every LANES-th part (32 where there are few columns: 617
// columns of 300 parts 4.9 -> 4.0 us; 16000 of 256 with 8 lanes 6.8 us, with 32 11).
template <typename T, int LANES>
__global__ __launch_bounds__(32 * LANES) void k_norm_join(const NormGrad a) {
  __shared__ float part[LANES][33];
  T *out = static_cast<T *>(blockIdx.y == 0 ? a.dw : a.db);
  if (!out) return;
  const int column = threadIdx.x & 31, lane = threadIdx.x >> 5, c = (int)blockIdx.x * 32 + column;
  const float *src = a.part + (int64_t)blockIdx.y * a.parts * a.width + c;
  float s = 0.f;
  if (c < a.width) {
#pragma unroll 8
    for (int i = lane; i < a.parts; i += LANES) s += src[(int64_t)i * a.width];
  }
  part[lane][column] = s;
  __syncthreads();
  // (a column's sums to LANES neighbouring lanes)
  const int mine = threadIdx.x / LANES;
  s = part[threadIdx.x % LANES][mine];
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if (threadIdx.x % LANES == 0 && (int)blockIdx.x * 32 + mine < a.width) out[blockIdx.x * 32 + mine] = from_f32<T>(s);
}
template <typename T>
__global__ __launch_bounds__(256) void k_norm_clear(T *dw, T *db, int width) {
  const int c = (int)blockIdx.x * 256 + threadIdx.x;
  if (c < width && dw) dw[c] = from_f32<T>(0.f);
  if (c < width && db) db[c] = from_f32<T>(0.f);
}

// ---- host ----
constexpr int64_t kCUs = 256;
struct NormShape { int lanes, pieces; };        // pieces 0: wide
NormShape norm_shape(int64_t width, int per16) {
  const int64_t n = ceil_div(width, per16);
  if (n <= per16) return {per16, 1};
  if (n <= 16) return {16, 1};
  if (n <= 32) return {32, 1};
  if (n <= 64) return {64, 1};
  if (n <= 128) return {64, 2};
  if (n <= 256) return {64, 4};
  if (n <= 512) return {256, 2};
  if (n <= 1024) return {256, 4};
  if (n <= 2048) return {512, 4};
  if (n <= 4096) return {512, 8};
  return {1024, 0};
}
// The gradient's lanes hold the sums of their columns besides the rows: sixteen columns each, or 24 or 32 for rows that take a workgroup of 512; rows beyond
// 16384 are wide.  (Workgroups of 1024, whose lanes have half the registers, spill: 8000 x 16000 bf16 514 us.  24 columns do not, 28 and 32 of float32 do:
// 12206 x 8864 float32 248 us with 24, 434 with 32; 8000 x 12000 with a residual 293 and 510, bf16 156 and 169.  24 with the next row asked for ahead, and for
// that the weights where they are used, 319, 388, 214.)
NormShape norm_grad_shape(int64_t width, int per16) {
  const int64_t n = ceil_div(width, per16);
  const int most = 16 / per16;
  if (n <= per16) return {per16, 1};
  if (n <= 16) return {16, 1};
  if (n <= 32) return {32, 1};
  for (int lanes = 64; lanes <= 512; lanes *= 2)
    for (int pieces = 1; pieces <= most; pieces *= 2)
      if (n <= lanes * pieces && (lanes == 64 || pieces == most)) return {lanes, pieces};
  if (n <= 768 * most) return {512, most + most / 2};
  return n <= 1024 * most ? NormShape{512, 2 * most} : NormShape{1024, 0};
}
int64_t rows_at_once(const NormShape &s) { return s.lanes <= 64 ? 256 / s.lanes : 1; }

template <int L, int V> struct ShapeOf { static constexpr int lanes = L, pieces = V; };
template <typename S, typename F> void by_shape(const NormShape &s, F f, S shape) { if (s.lanes == S::lanes && s.pieces == S::pieces) f(shape); }
template <typename F, typename... S> void by_shape(const NormShape &s, F f, S... shapes) { (by_shape(s, f, shapes), ...); }

template <typename T>
int forward(const Norm &n, hipStream_t st) {
  constexpr int E = Elem<T>::kPer16;
  const NormShape s = norm_shape(n.width, E);
  if (s.pieces == 0) {
    k_norm_wide<T><<<(unsigned)std::min(n.rows, 2 * kCUs), 1024, 0, st>>>(n);
  } else {
    const unsigned grid = (unsigned)std::min(ceil_div(n.rows, rows_at_once(s)), (s.lanes <= 256 ? 8 : 4) * kCUs);
    by_shape(s, [&](auto shape) { k_norm<T, shape.lanes, shape.pieces><<<grid, kThreads<shape.lanes>, 0, st>>>(n); }, ShapeOf<E, 1>(), ShapeOf<16, 1>(), ShapeOf<32, 1>(), ShapeOf<64, 1>(), ShapeOf<64, 2>(),
             ShapeOf<64, 4>(), ShapeOf<256, 2>(), ShapeOf<256, 4>(), ShapeOf<512, 4>(), ShapeOf<512, 8>());
  }
  return ops_launched("layer norm");
}

// Workgroups of the gradient, each of which leaves a part of the column sums.
struct NormGradPlan { NormShape shape; int64_t parts, rows_per_part; size_t bytes; };
NormGradPlan plan_grad(const cada_norm_grad *a) {
  NormGradPlan p{};
  p.shape = norm_grad_shape(a->width, 16 / (int)type_bytes(a->type));
  if (a->rows == 0) return p;
  if (p.shape.pieces == 0) {
    const int64_t columns = ceil_div(a->width, 2048);
    p.rows_per_part = std::max<int64_t>(16, ceil_div(a->rows, ceil_div(4 * kCUs, columns)));
    p.parts = ceil_div(a->rows, p.rows_per_part);
  } else {
    // (as many turns of rows for each, and no more parts than that takes)
    const int64_t turns = ceil_div(a->rows, rows_at_once(p.shape));
    p.parts = ceil_div(turns, ceil_div(turns, (p.shape.lanes <= 256 ? 2 : 1) * kCUs));
  }
  if ((a->dw || a->db) && (p.parts > 1 || p.shape.pieces == 0)) p.bytes = ops_align((size_t)2 * p.parts * a->width * 4);
  return p;
}
template <typename T>
int backward(const cada_norm_grad *a, const NormGradPlan &p) {
  hipStream_t st = static_cast<hipStream_t>(a->stream);
  NormGrad n{};
  n.dy = a->dy; n.x = a->x; n.weight = a->weight; n.residual = a->dx ? a->residual : nullptr; n.mean = a->mean; n.rstd = a->rstd;
  n.dx = a->dx; n.dw = a->dw; n.db = a->db; n.part = static_cast<float *>(a->workspace);
  n.rows = a->rows; n.lddy = a->lddy; n.ldx = a->ldx; n.ldr = a->ldr; n.lddx = a->lddx;
  n.width = (int32_t)a->width; n.parts = (int32_t)p.parts; n.rows_per_part = p.rows_per_part;
  const bool sums = a->dw || a->db;
  if (a->rows == 0) {
    if (!sums) return CADA_OK;
    k_norm_clear<T><<<(unsigned)ceil_div(a->width, 256), 256, 0, st>>>(static_cast<T *>(a->dw), static_cast<T *>(a->db), n.width);
    return ops_launched("layer norm clear");
  }
  if (p.shape.pieces == 0) {
    if (sums) k_norm_grad_columns<T><<<dim3((unsigned)ceil_div(a->width, 2048), (unsigned)p.parts), 256, 0, st>>>(n);
    if (a->dx) k_norm_grad_wide<T><<<(unsigned)std::min(a->rows, 2 * kCUs), 1024, 0, st>>>(n);
  } else if (sums || a->dx) {
    constexpr int E = Elem<T>::kPer16, most = 16 / E;
    by_shape(p.shape, [&](auto shape) {
      if constexpr (shape.pieces <= most || shape.lanes == 512) k_norm_grad<T, shape.lanes, shape.pieces><<<(unsigned)p.parts, kThreads<shape.lanes>, 0, st>>>(n);
    }, ShapeOf<E, 1>(), ShapeOf<16, 1>(), ShapeOf<32, 1>(), ShapeOf<64, 1>(), ShapeOf<64, 2>(), ShapeOf<64, 4>(), ShapeOf<128, most>(), ShapeOf<256, most>(), ShapeOf<512, most>(), ShapeOf<512, most + most / 2>(), ShapeOf<512, 2 * most>());
  }
  if (int rc = ops_launched("layer norm gradients")) return rc;
  if (p.bytes == 0) return CADA_OK;
  const dim3 grid((unsigned)ceil_div(a->width, 32), 2);
  if (a->width <= 4096) k_norm_join<T, 32><<<grid, 1024, 0, st>>>(n);
  else k_norm_join<T, 8><<<grid, 256, 0, st>>>(n);
  return ops_launched("layer norm join");
}

bool check_shape(int64_t rows, int64_t width, int type) {
  if (rows < 0 || rows > (int64_t)1 << 40) { set_error("rows must be in [0, 2^40] (got %lld)", (long long)rows); return false; }
  if (width < 1 || width > CADA_MAX_WIDTH) { set_error("width must be in [1, %d] (got %lld)", CADA_MAX_WIDTH, (long long)width); return false; }
  if (type != CADA_F32 && type != CADA_BF16) { set_error("type must be CADA_F32 or CADA_BF16 (got %d)", type); return false; }
  return true;
}

}  // namespace
}  // namespace cada

using namespace cada;

extern "C" {

int cada_layer_norm_forward(const cada_norm *a) {
  if (!a) { set_error("the arguments are NULL"); return CADA_EINVAL; }
  if (!check_shape(a->rows, a->width, a->type)) return CADA_EINVAL;
  if (!(a->eps > 0.0) || (float)a->eps == 0.f || !((float)a->eps < __builtin_inff())) { set_error("eps must be positive and finite in float32"); return CADA_EINVAL; }
  if (a->rows == 0) return CADA_OK;
  if (!ops_check_table("x", a->x, a->ldx, a->width, a->type) || !ops_check_table("y", a->y, a->ldy, a->width, a->type)) return CADA_EINVAL;
  if (a->weight && !ops_check_table("weight", a->weight, a->width, a->width, a->type)) return CADA_EINVAL;
  if (a->bias && !ops_check_table("bias", a->bias, a->width, a->width, a->type)) return CADA_EINVAL;
  if (!ops_check_table("mean", a->mean ? a->mean : a->y, 1, 1, a->mean ? CADA_F32 : a->type) || !ops_check_table("rstd", a->rstd ? a->rstd : a->y, 1, 1, a->rstd ? CADA_F32 : a->type)) return CADA_EINVAL;
  const size_t elem = type_bytes(a->type);
  const Span x = span("x", a->x, a->rows, a->ldx, a->width, elem), y = span("y", a->y, a->rows, a->ldy, a->width, elem);
  const Span mean = span("mean", a->mean, (size_t)a->rows * 4), rstd = span("rstd", a->rstd, (size_t)a->rows * 4);
  const Span ins[] = {x, span("weight", a->weight, 1, a->width, a->width, elem), span("bias", a->bias, 1, a->width, a->width, elem)};
  const bool in_place = a->x == a->y && (a->ldx == a->ldy || a->rows == 1);
  for (const Span &in : ins)
    if ((!(&in == ins && in_place) && !ops_apart(y, in)) || !ops_apart(mean, in) || !ops_apart(rstd, in)) return CADA_EINVAL;
  if (!ops_apart(y, mean) || !ops_apart(y, rstd) || !ops_apart(mean, rstd)) return CADA_EINVAL;
  Norm n{};
  n.x = a->x; n.weight = a->weight; n.bias = a->bias; n.y = a->y; n.mean = a->mean; n.rstd = a->rstd;
  n.rows = a->rows; n.ldx = a->ldx; n.ldy = a->ldy; n.width = (int32_t)a->width; n.eps = (float)a->eps;
  hipStream_t st = static_cast<hipStream_t>(a->stream);
  return a->type == CADA_BF16 ? forward<bf16>(n, st) : forward<float>(n, st);
}

int cada_layer_norm_backward_workspace(cada_norm_grad *a) {
  if (!a) { set_error("the arguments are NULL"); return CADA_EINVAL; }
  if (!check_shape(a->rows, a->width, a->type)) return CADA_EINVAL;
  a->workspace_bytes = plan_grad(a).bytes;
  return CADA_OK;
}

int cada_layer_norm_backward(const cada_norm_grad *a) {
  if (!a) { set_error("the arguments are NULL"); return CADA_EINVAL; }
  if (!check_shape(a->rows, a->width, a->type)) return CADA_EINVAL;
  if (a->rows > 0 && (a->dx || a->dw || a->db)) {
    if (!ops_check_table("dy", a->dy, a->lddy, a->width, a->type) || !ops_check_table("x", a->x, a->ldx, a->width, a->type)) return CADA_EINVAL;
    if (!ops_check_table("mean", a->mean, 1, 1, CADA_F32) || !ops_check_table("rstd", a->rstd, 1, 1, CADA_F32)) return CADA_EINVAL;
    if (a->weight && !ops_check_table("weight", a->weight, a->width, a->width, a->type)) return CADA_EINVAL;
    if (a->dx && a->residual && !ops_check_table("residual", a->residual, a->ldr, a->width, a->type)) return CADA_EINVAL;
    if (a->dx && !ops_check_table("dx", a->dx, a->lddx, a->width, a->type)) return CADA_EINVAL;
  }
  if (a->dw && !ops_check_table("dw", a->dw, a->width, a->width, a->type)) return CADA_EINVAL;
  if (a->db && !ops_check_table("db", a->db, a->width, a->width, a->type)) return CADA_EINVAL;
  const NormGradPlan p = plan_grad(a);
  if (int rc = ops_check_workspace(a->workspace, a->workspace_bytes, p.bytes)) return rc;
  const size_t elem = type_bytes(a->type);
  const bool any = a->rows > 0;
  const Span outs[] = {span("dx", any ? a->dx : nullptr, a->rows, a->lddx, a->width, elem), span("dw", a->dw, 1, a->width, a->width, elem), span("db", a->db, 1, a->width, a->width, elem),
                       span("workspace", a->workspace, p.bytes)};
  const Span ins[] = {span("dy", any ? a->dy : nullptr, a->rows, a->lddy, a->width, elem), span("x", any ? a->x : nullptr, a->rows, a->ldx, a->width, elem),
                      span("residual", any && a->dx ? a->residual : nullptr, a->rows, a->ldr, a->width, elem), span("weight", any ? a->weight : nullptr, 1, a->width, a->width, elem),
                      span("mean", a->mean, (size_t)a->rows * 4), span("rstd", a->rstd, (size_t)a->rows * 4)};
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < 6; ++j) {
      const bool in_place = i == 0 && (j == 0 || j == 2) && a->dx == ins[j].at && (a->rows == 1 || a->lddx == (j == 0 ? a->lddy : a->ldr));
      if (!in_place && !ops_apart(outs[i], ins[j])) return CADA_EINVAL;
    }
    for (int j = 0; j < i; ++j)
      if (!ops_apart(outs[i], outs[j])) return CADA_EINVAL;
  }
  return a->type == CADA_BF16 ? backward<bf16>(a, p) : backward<float>(a, p);
}

}  // extern "C"
