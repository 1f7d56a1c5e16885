// The softmax cross-entropy of a last layer's product, with its gradients, without the logits in memory (cada_ops.h).
//
// The logits' tiles (cada_linear_tiles.h) end in statistics: of each row, and of each strip of 32 or 64 columns, the largest logit and the sum of the
// exponentials of the distances to it.  A row's strips are then joined, as one goes along, to the row's largest and its sum, which is its loss.  For the
// gradients the logits are formed again in pieces of the classes; their tiles end in softmax - target (but for a factor) in the operands' type, from which the
// products of a layer's gradients are taken while it is in the caches: dw is finished piece by piece, dx is added up in float32.  That is four products where
// keeping the logits would take three, and memory for one piece instead of all.  Logits that are not more than a piece are kept in float32: for a pass over
// whole rows (k_kept_rows), or, of long rows, left behind by the statistics (k_left_signal).
#include <algorithm>

#include "cada_linear_tiles.h"

namespace cada {
namespace {

// distance: the sum of (z - top) share over the classes that are left (smoothing), left: their number.  With share = 1 / classes such sums, and joins of
// them, overflow nowhere that z - top does not: a mask of the type's lowest value at any number of classes leaves a loss of some 1e37.
struct Stat { float top, sum, distance, left; };
struct RowInfo { float base, f_total, f_each; int32_t label; };      // base infinite (exponentials are zero), f_total 0, label < 0: a row without gradient
struct Loss {
  const void *labels, *bias;
  LossHead *head;
  float *stats;              // [chunks][rows][stat_floats]
  RowInfo *info;
  float *z_label, *loss, *mean;
  void *signal;              // [rows, piece] or null
  float *db_part;            // [strips][piece] or null
  int64_t rows, ignore, ldz, chunks;
  int32_t classes, label_bytes, first;      // first: the piece's first class
  const float *kept, *kept_bias;            // kept logits without their bias, in `splits` parts; the biases in float32, -inf behind the last class
  int32_t splits;
  float *left;               // [rows][classes up to whole groups of eight]: where statistics leave the logits, with their bias, or null
  int64_t left_rows;
  int32_t lanes;             // rows of a workgroup of k_rows, as a power of two
  float smoothing, keep, scale, share;      // keep = 1 - smoothing, rounded once
};

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kInf = __builtin_inff();

__device__ __forceinline__ int64_t label_at(const void *labels, int bytes, int64_t r) {
  return bytes == 8 ? static_cast<const int64_t *>(labels)[r] : (int64_t)static_cast<const int32_t *>(labels)[r];
}
__device__ __forceinline__ bool counts(const Loss &q, int64_t label) { return label != q.ignore && label >= 0 && label < q.classes; }

// exp(z - base) is the hardware's exp2 of the rounded difference times log2(e): off by |z - base| 2^-23 and an ulp or two, relative.  The difference comes
// first, so that a mask of the type's lowest value (or a row of nothing else) overflows nowhere.
__device__ __forceinline__ float power(float z, float base) { return __builtin_amdgcn_exp2f((z - base) * kLog2e); }

// The biases of a tile's columns in LDS: -inf for a column that does not exist, so that it is a class that is ruled out (what the matrix instructions made of it is something of the table's).
template <typename T> __device__ __forceinline__ void put_bias(const Loss &q, const Product &p, int n0, int t, int columns, float *to) {
  if (t >= columns) return;
  const int n = n0 + t;
  to[t] = n >= p.N ? -kInf : q.bias ? to_f32(static_cast<const T *>(q.bias)[q.first + n]) : 0.f;
}

// A tile's logits into statistics.  A lane has FN x 16 logits of a row, and the lane 32 further the row's others.
// Bound by the vector unit: an addition, a comparison, two operations and an exponential (four times an operation's time) per logit.
template <typename T, int BM, int BN, bool LEFT> struct ToStatistics {
  static constexpr bool kOwn = true;
  const Loss &q;
  int32_t *label;            // [BM], in LDS
  float *bias;               // [BN], in LDS
  __device__ __forceinline__ ToStatistics(const Loss &loss, int32_t *l, float *b) : q(loss), label(l), bias(b) {}
  __device__ __forceinline__ void begin(const Product &p, int64_t m0, int n0, int t) {
    put_bias<T>(q, p, n0, t, BN, bias);
    if (t >= BM) return;
    const int64_t l = m0 + t < p.M ? label_at(q.labels, q.label_bytes, m0 + t) : -1;
    label[t] = counts(q, l) ? (int32_t)l : -1;
  }
  __device__ __forceinline__ void put(int64_t m, int64_t strip, const Stat &s) const {
    const int64_t to = strip * q.rows + m;
    if (q.smoothing != 0.f) reinterpret_cast<Stat *>(q.stats)[to] = s;
    else reinterpret_cast<float2 *>(q.stats)[to] = float2{s.top, s.sum};
  }
  template <typename, int FM, int FN> __device__ __forceinline__ void sums(const Product &p, f32x16 (&z)[FM][FN], int64_t m0, int n0, int wm, int wn, int lane, unsigned char *) {
    const int half = lane >> 5;
    Stat s[FM];
#pragma unroll
    for (int i = 0; i < FM; ++i) s[i] = Stat{-kInf, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const v4s b = *reinterpret_cast<const v4s *>(bias + wn + 32 * j + 8 * r + 4 * half);
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            z[i][j][4 * r + e] += b[e];
            s[i].top = fmaxf(s[i].top, z[i][j][4 * r + e]);
          }
        if (FM >= 4) __builtin_amdgcn_sched_barrier(0);
        if constexpr (LEFT) {
          const int n = n0 + wn + 32 * j + 8 * r + 4 * half, columns = (q.classes + 7) / 8 * 8;
#pragma unroll
          for (int i = 0; i < FM; ++i) {
            const int64_t m = m0 + wm + 32 * i + (lane & 31);
            if (m < p.M && n < columns) *reinterpret_cast<v4s *>(q.left + m * columns + n) = v4s{z[i][j][4 * r], z[i][j][4 * r + 1], z[i][j][4 * r + 2], z[i][j][4 * r + 3]};
          }
        }
      }
    float base[FM];
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      s[i].top = fmaxf(s[i].top, __shfl_xor(s[i].top, 32, 64));
      // (a strip of nothing but -inf and NaN: its exponentials are taken against 0, so that only a NaN makes the sum NaN)
      base[i] = s[i].top == -kInf ? 0.f : s[i].top;
    }
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[i].sum += power(z[i][j][r], base[i]);
          if (FM >= 4 && r % 8 == 7) __builtin_amdgcn_sched_barrier(0);        // (few at a time: interleaved, they spill)
        }
    if (q.smoothing != 0.f) {
      float left = 0.f;
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const v4s b = *reinterpret_cast<const v4s *>(bias + wn + 32 * j + 8 * r + 4 * half);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool in = b[e] != -kInf;
            left += in ? 1.f : 0.f;
#pragma unroll
            for (int i = 0; i < FM; ++i) s[i].distance = fmaf(in ? z[i][j][4 * r + e] - base[i] : 0.f, q.share, s[i].distance);
          }
          if (FM >= 4) __builtin_amdgcn_sched_barrier(0);
        }
      left += __shfl_xor(left, 32, 64);
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        s[i].distance += __shfl_xor(s[i].distance, 32, 64);
        s[i].left = left;
      }
    }
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      s[i].sum += __shfl_xor(s[i].sum, 32, 64);
      const int row = wm + 32 * i + (lane & 31);
      const int64_t m = m0 + row;
      const int at = label[row] - (n0 + wn);
      const bool mine = at >= 0 && at < 32 * FN && (at >> 2 & 1) == half;
      if (__ballot(mine)) {
        float zl = 0.f;
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) zl = at == 32 * j + (r >> 2) * 8 + 4 * half + (r & 3) ? z[i][j][r] : zl;
        if (mine) q.z_label[m] = zl;
      }
      if (half == 0 && m < p.M) put(m, (n0 + wn) / (32 * FN), s[i]);
    }
  }
  // The same of eight columns of a row per lane, four lanes to a row.
  template <typename> __device__ __forceinline__ void row(const Product &p, int64_t m0, int n0, int t, float (&z)[8]) {
    const int64_t m = m0 + t / 4;
    const int c = (t & 3) * 8;
    Stat s = {-kInf, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      z[e] += bias[c + e];
      s.top = fmaxf(s.top, z[e]);
    }
    s.top = fmaxf(s.top, __shfl_xor(s.top, 1, 64));
    s.top = fmaxf(s.top, __shfl_xor(s.top, 2, 64));
    const float base = s.top == -kInf ? 0.f : s.top;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool in = bias[c + e] != -kInf;
      s.sum += power(z[e], base);
      s.left += in ? 1.f : 0.f;
      s.distance = fmaf(in ? z[e] - base : 0.f, q.share, s.distance);
    }
    float *parts[3] = {&s.sum, &s.left, &s.distance};
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      *parts[i] += __shfl_xor(*parts[i], 1, 64);
      *parts[i] += __shfl_xor(*parts[i], 2, 64);
    }
    if (m >= p.M) return;
    if constexpr (LEFT) {
      if (n0 + c < p.N) {
        v4s *to = reinterpret_cast<v4s *>(q.left + m * ((q.classes + 7) / 8 * 8) + n0 + c);
        to[0] = v4s{z[0], z[1], z[2], z[3]};
        to[1] = v4s{z[4], z[5], z[6], z[7]};
      }
    }
    const int at = label[t / 4] - (n0 + c);
    if (at >= 0 && at < 8) {
      float zl = z[0];
#pragma unroll
      for (int e = 1; e < 8; ++e) zl = at == e ? z[e] : zl;
      q.z_label[m] = zl;
    }
    if ((t & 3) == 0) put(m, n0 / 32, s);
  }
};

// A tile's logits into the signal (softmax - target) / (1 - smoothing), and its column sums over a strip of rows.  What is left of the gradient's factor, (1 - smoothing) scale / count, is
// taken to the products' float32 sums: a bf16 signal is rounded, and with that factor in it the label's -(1 - p) of every row would be rounded the same way wherever p is small, up to 2^-8 off
// (1 / 100 rows), while -1 + p / (1 - smoothing) is next to a value that bf16 has (100, 96 and 300 rows:
// dx and dw 1.75e-3, 1.77e-3 and 1.70e-3 from 64 bits, relative in the 2-norm; with the factor in the signal 2.2e-3, 2.9e-3 and 2.5e-3; rounding the outputs alone is 1.66e-3).
// Rows without gradient have a sum of infinity (and x = 0), classes that are ruled out a logit of -inf.
template <typename T, int BM> struct ToSignal {
  static constexpr bool kOwn = true;
  const Loss &q;
  RowInfo *info;             // [BM], in LDS
  float *bias;               // [BM], in LDS
  __device__ __forceinline__ ToSignal(const Loss &loss, RowInfo *r, float *b) : q(loss), info(r), bias(b) {}
  __device__ __forceinline__ void begin(const Product &p, int64_t m0, int n0, int t) {
    put_bias<T>(q, p, n0, t, BM, bias);
    if (t >= BM) return;
    const RowInfo &r = q.info[min(m0 + t, p.M - 1)];
    const bool in = m0 + t < p.M;
    info[t].base = in ? r.base : kInf;
    info[t].f_total = in ? r.f_total : 0.f;
    info[t].f_each = in ? r.f_each : 0.f;
    info[t].label = in ? r.label : -1;
  }
  __device__ __forceinline__ float signal(float z, bool in, const RowInfo &r) const {
    const float p = power(z, r.base) * r.f_total;
    return q.smoothing != 0.f ? p - (in ? r.f_each : 0.f) : p;
  }
  template <typename, int FM, int FN> __device__ __forceinline__ void sums(const Product &p, f32x16 (&z)[FM][FN], int64_t m0, int n0, int wm, int wn, int lane, unsigned char *lds) {
    constexpr int WN = 32 * FN, kLd = WN + 16 / sizeof(T), kLanes = WN / 8, kRows = 64 / kLanes;
    const int half = lane >> 5;
    float column[FN][16];
    RowInfo info_of[FM];
#pragma unroll
    for (int i = 0; i < FM; ++i) info_of[i] = info[wm + 32 * i + (lane & 31)];
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const v4s b = *reinterpret_cast<const v4s *>(bias + wn + 32 * j + 8 * r + 4 * half);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool in = b[e] != -kInf;
          column[j][4 * r + e] = 0.f;
#pragma unroll
          for (int i = 0; i < FM; ++i) {
            z[i][j][4 * r + e] = signal(z[i][j][4 * r + e] + b[e], in, info_of[i]);
            column[j][4 * r + e] += z[i][j][4 * r + e];
          }
        }
      }
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int at = info_of[i].label < 0 ? -1 : info_of[i].label - q.first - (n0 + wn);
      if (__ballot(at >= 0 && at < WN)) {
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float one = at == 32 * j + (r >> 2) * 8 + 4 * half + (r & 3) ? 1.f : 0.f;
            z[i][j][r] -= one;
            column[j][r] -= one;
          }
      }
    }
    if (q.signal) {
      // through LDS, 32 rows at a time, in the table's type, to eight consecutive columns per lane
      T *strip = reinterpret_cast<T *>(lds);
      const int n = n0 + wn + lane % kLanes * 8;
#pragma unroll
      for (int i = 0; i < FM; ++i) {
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            T *to = strip + (lane & 31) * kLd + 32 * j + 8 * r + 4 * half;
            const f32x16 &f = z[i][j];
            if constexpr (sizeof(T) == 2) *reinterpret_cast<uint64_t *>(to) = (uint64_t)f2bf_pk(f[4 * r + 2], f[4 * r + 3]) << 32 | f2bf_pk(f[4 * r], f[4 * r + 1]);
            else *reinterpret_cast<v4s *>(to) = v4s{f[4 * r], f[4 * r + 1], f[4 * r + 2], f[4 * r + 3]};
          }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int turn = 0; turn < 32 / kRows; ++turn) {
          const int row = lane / kLanes + turn * kRows;
          const int64_t m = m0 + wm + 32 * i + row;
          const T *from = strip + row * kLd + lane % kLanes * 8;
          u32x4v x[sizeof(T) / 2];
#pragma unroll
          for (int k = 0; k < (int)sizeof(T) / 2; ++k) x[k] = reinterpret_cast<const u32x4v *>(from)[k];
          if (m < p.M && n < p.N) {        // (eight columns whole: the signal's rows have room for it)
            T *to = static_cast<T *>(q.signal) + m * q.ldz + n;
#pragma unroll
            for (int k = 0; k < (int)sizeof(T) / 2; ++k) reinterpret_cast<u32x4v *>(to)[k] = x[k];
          }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
    }
    if (!q.db_part) return;
    // A column's 32 lanes (rows) exchange halves of their sums until each has one column's, of which FN = 1 leaves two lanes with the same.
    float *all = &column[0][0];
    int mine = 0;
#pragma unroll
    for (int h = 8 * FN; h > 0; h /= 2) {
      const bool upper = lane & h;
      mine += upper ? h : 0;
#pragma unroll
      for (int e = 0; e < h; ++e) {
        const float keep = upper ? all[e + h] : all[e], other = upper ? all[e] : all[e + h];
        all[e] = keep + __shfl_xor(other, h, 64);
      }
    }
    if constexpr (FN == 1) all[0] += __shfl_xor(all[0], 16, 64);
    const int n = n0 + wn + 32 * (mine >> 4) + 8 * (mine >> 2 & 3) + 4 * half + (mine & 3);
    if ((FN == 2 || (lane & 16) == 0) && n < p.N) q.db_part[((m0 + wm) / (32 * FM)) * p.N + n] = all[0];
  }
  template <typename> __device__ __forceinline__ void row(const Product &p, int64_t m0, int n0, int t, float (&z)[8]) {
    const int64_t m = m0 + t / 4;
    const int c = (t & 3) * 8, n = n0 + c;
    const RowInfo r = info[t / 4];
    const int at = r.label < 0 ? -1 : r.label - q.first - n;
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = signal(z[e] + bias[c + e], bias[c + e] != -kInf, r) - (at == e ? 1.f : 0.f);
    if (q.signal && m < p.M && n < p.N) store8_n(static_cast<T *>(q.signal) + m * q.ldz + n, 8, z);
    if (!q.db_part) return;
#pragma unroll
    for (int h = 4; h > 0; h /= 2) {        // lanes 8 h apart: the upper one goes on with the upper half
      const bool upper = t & 8 * h;
#pragma unroll
      for (int e = 0; e < h; ++e) {
        const float keep = upper ? z[e + h] : z[e], other = upper ? z[e] : z[e + h];
        z[e] = keep + __shfl_xor(other, 8 * h, 64);
      }
    }
    z[0] += __shfl_xor(z[0], 4, 64);
    const int column = n + (t >> 5 & 1) * 4 + (t >> 4 & 1) * 2 + (t >> 3 & 1);
    if ((t & 4) == 0 && column < p.N) q.db_part[(m0 / BM * 2 + (t >> 6)) * p.N + column] = z[0];
  }
};

__device__ __forceinline__ void clear_counters(LossHead *head) {        // (by a launch before the one that counts)
  if (threadIdx.x < kCounters) head->done[threadIdx.x * kLineWords] = 0;
  if (threadIdx.x == 0) head->full[0] = 0;
}
// The workgroups' losses and numbers of rows that count, whose last one to come adds them up in the workgroups' order: `sum` and `used` are thread 0's.
__device__ __forceinline__ void add_up(const Loss &q, double sum, int64_t used) {
  __shared__ bool last;
  const int t = threadIdx.x;
  if (t == 0) {
    // (few workgroups count themselves in the one place, 12 ns each and one trip less)
    const bool few = gridDim.x <= 256;
    const uint32_t c = blockIdx.x % kCounters, of_mine = (gridDim.x - c + kCounters - 1) / kCounters, counters = few ? gridDim.x : kCounters;
    __hip_atomic_store(&q.head->loss[blockIdx.x], sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(&q.head->used[blockIdx.x], used, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // (they are where the last workgroup reads them before this one is counted)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    last = (few || __hip_atomic_fetch_add(&q.head->done[c * kLineWords], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == of_mine - 1) &&
           __hip_atomic_fetch_add(&q.head->full[0], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == counters - 1;
  }
  __syncthreads();
  if (!last || t >= 64) return;
  sum = 0.0;
  used = 0;
#pragma unroll 4
  for (int i = t; i < (int)gridDim.x; i += 64) {
    sum += __hip_atomic_load(&q.head->loss[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    used += __hip_atomic_load(&q.head->used[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  sum = wave_sum_f64(sum);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) used += __shfl_xor(used, o, 64);
  if (t == 0) {
    const int64_t count = max(used, (int64_t)1);
    if (q.mean) *q.mean = (float)(sum / (double)count);
    q.head->factor = q.keep * q.scale / (float)count;
  }
}
// A row's loss from its statistics and its label's logit (log(sum exp z) - keep z_y - smoothing mean_left z, with the largest taken out of all three).
__device__ __forceinline__ float loss_of(const Loss &q, const Stat &s, float base, float z_label, bool used, bool known) {
  float l = logf(s.sum) - q.keep * (z_label - base);
  if (q.smoothing != 0.f) l -= q.smoothing * s.distance * ((float)q.classes / s.left);
  if (s.top == -kInf && s.sum == 0.f) l = kInf;
  if (!known) l = __builtin_nanf("");
  return used ? l : 0.f;
}

// The logits, formed a first time for the rows' statistics: bound by the matrix instructions where there are many rows (8192 x 4096 x 65536 bf16 3360 us,
// 1.31 PFLOP/s; 4096 x 1024 x 50001 424 us, 0.99: 12.25 rounds of tiles of 256 x 256, one to a CU, take 13), by the weights where there are few
// (64 x 1024 x 50001, whose odd rows go through registers: 25 us, 4.1 TB/s).
template <typename T, int BM, int BN, int WY, int WX, bool DIRECT, int STAGES, int KW, bool LEFT>
__global__ __launch_bounds__(64 * WY * WX * KW) void k_statistics(const Product p, const Loss q) {
  __shared__ __align__(16) unsigned char lds[tile_lds(BM, BN, STAGES, KW)];
  __shared__ int32_t label[BM];
  __shared__ __align__(16) float bias[BN];
  if (blockIdx.x == 0) clear_counters(q.head);
  const uint32_t tile = tile_of_block((uint32_t)p.tiles_m * p.tiles_n);
  if (tile != ~0u) tile_product<T, BM, BN, WY, WX, true, false, DIRECT, STAGES, KW, NO_SIGNAL>(p, tile, lds, ToStatistics<T, BM, BN, LEFT>(q, label, bias));
}
// The logits of a piece, formed again for its signal (the largest case above: eight pieces of 442 us, 1.24 PFLOP/s; the other: three of 169, whose 4.1 rounds take 5).
template <typename T, int BM, int WY, int WX, bool DIRECT, int STAGES, int KW = 1>
__global__ __launch_bounds__(64 * WY * WX * KW) void k_signal(const Product p, const Loss q) {
  __shared__ __align__(16) unsigned char lds[tile_lds(BM, BM, STAGES, KW)];
  __shared__ RowInfo info[BM];
  __shared__ __align__(16) float bias[BM];
  const uint32_t tile = tile_of_block((uint32_t)p.tiles_m * p.tiles_n);
  if (tile != ~0u) tile_product<T, BM, BM, WY, WX, true, false, DIRECT, STAGES, KW, NO_SIGNAL>(p, tile, lds, ToSignal<T, BM>(q, info, bias));
}

// Joins statistics `b` to `a`: both against the larger of the two largest.
template <bool SMOOTH> __device__ __forceinline__ void join(Stat &a, const Stat &b, float share) {
  if (b.top == -kInf) {        // no class left there, or NaN
    a.sum += b.sum;
    a.left += b.left;
    a.distance += b.distance;
    return;
  }
  if (a.top == -kInf) {
    a = Stat{b.top, b.sum + a.sum, b.distance + a.distance, b.left + a.left};
    return;
  }
  const float top = fmaxf(a.top, b.top);
  a.sum = a.sum * __builtin_amdgcn_exp2f((a.top - top) * kLog2e) + b.sum * __builtin_amdgcn_exp2f((b.top - top) * kLog2e);
  if constexpr (SMOOTH) {
    a.distance = fmaf(a.left * share, a.top - top, a.distance) + fmaf(b.left * share, b.top - top, b.distance);
    a.left += b.left;
  }
  a.top = top;
}

// 2^lanes rows by the other threads of 1024 over their strips; a row's strips are joined in one order.  The last workgroup adds the losses up, in the workgroups' order.  (64 rows
// of 1564 strips 9 us, 8192 of 1024 28: the launch, a workgroup's strips, and the wait for the last one's sum.  Labels and their logits asked for before the strips: the same.)
template <bool SMOOTH>
__global__ __launch_bounds__(1024) void k_rows(const Loss q) {
  __shared__ Stat part[16][64];
  __shared__ float losses[64];
  __shared__ uint8_t used_rows[64];
  const int here = 1 << q.lanes, t = threadIdx.x, row = t & (here - 1), lane = t >> q.lanes, high = 1024 >> q.lanes;
  double sum = 0.0;
  int64_t used_sum = 0;
  for (int64_t r0 = (int64_t)blockIdx.x * here; r0 < q.rows; r0 += (int64_t)gridDim.x * here) {
    const int64_t r = r0 + row, at = min(r, q.rows - 1);
    Stat s = {-kInf, 0.f, 0.f, 0.f};
    if constexpr (SMOOTH) {
#pragma unroll 4
      for (int64_t c = lane; c < q.chunks; c += high) join<true>(s, reinterpret_cast<const Stat *>(q.stats)[c * q.rows + at], q.share);
    } else {
#pragma unroll 8
      for (int64_t c = lane; c < q.chunks; c += high) {
        const float2 x = reinterpret_cast<const float2 *>(q.stats)[c * q.rows + at];
        join<false>(s, Stat{x.x, x.y, 0.f, 0.f}, q.share);
      }
    }
    // a row's lanes of a wavefront, then its wavefronts, in their order
    for (int o = here; o < 64; o <<= 1) {
      Stat other = {__shfl_xor(s.top, o, 64), __shfl_xor(s.sum, o, 64), 0.f, 0.f};
      if constexpr (SMOOTH) {
        other.distance = __shfl_xor(s.distance, o, 64);
        other.left = __shfl_xor(s.left, o, 64);
      }
      if (t & o) {        // (in one order for both)
        join<SMOOTH>(other, s, q.share);
        s = other;
      } else {
        join<SMOOTH>(s, other, q.share);
      }
    }
    if ((t & 63) < here) part[t >> 6][row] = s;
    for (int h = 8; h > 0; h >>= 1) {
      __syncthreads();
      if (lane < h) {
        s = part[lane][row];
        join<SMOOTH>(s, part[lane + h][row], q.share);
        part[lane][row] = s;
      }
    }
    if (lane == 0) {
      losses[row] = 0.f;
      used_rows[row] = 0;
    }
    if (lane == 0 && r < q.rows) {
      const int64_t label = label_at(q.labels, q.label_bytes, r);
      const bool used = label != q.ignore, known = counts(q, label), none = s.top == -kInf && s.sum == 0.f;
      const float base = s.top == -kInf ? 0.f : s.top;
      const float l = loss_of(q, s, base, known ? q.z_label[r] : 0.f, used, known);
      losses[row] = l;
      used_rows[row] = used;
      if (q.loss) q.loss[r] = l;
      q.info[r] = known && used && !none ? RowInfo{base, 1.f / (s.sum * q.keep), SMOOTH ? q.smoothing / (s.left * q.keep) : 0.f, (int32_t)label} : RowInfo{kInf, 0.f, 0.f, -1};
    }
    __syncthreads();
    if (t == 0) {
      for (int i = 0; i < here; ++i) {
        sum += (double)losses[i];
        used_sum += used_rows[i];
      }
    }
    __syncthreads();
  }
  add_up(q, sum, used_sum);
}

// Kept logits: a group of LANES lanes takes a row, V pieces of four classes per lane, which stay in registers from the statistics to the signal.  A workgroup goes on to further rows and adds up, in
// registers too, its part of the signal's column sums.  The logits are read once (in all their parts), the signal is written once.
template <int LANES, int N> __device__ __forceinline__ void group_join(float (&x)[N], float (*part)[N], bool largest) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const float y = __shfl_xor(x[i], o, 64);
      x[i] = largest ? fmaxf(x[i], y) : x[i] + y;
    }
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
      for (int w = 1; w < LANES / 64; ++w) x[i] = largest ? fmaxf(x[i], part[w][i]) : x[i] + part[w][i];
    }
  }
}
// (8192 x 1000 to bf16 22 us, 2.2 TB/s; 1000 x 16000 47 us, 2.0; 120 x 1001 to float32 8: the wait between a row's read, its sums and its signal.)
template <typename T, int LANES, int V>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void k_kept_rows(const Loss q) {
  constexpr int kGroups = LANES < 256 ? 256 / LANES : 1;
  __shared__ float part_top[LANES / 64][1], part_sum[LANES / 64][3];
  __shared__ double group_loss[kGroups];
  __shared__ int64_t group_used[kGroups];
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES, columns = (q.classes + 7) / 8 * 8;
  v4s z[V], column[V];
#pragma unroll
  for (int v = 0; v < V; ++v) column[v] = v4s{0.f, 0.f, 0.f, 0.f};
  double losses = 0.0;
  int64_t used_rows = 0;
  const int64_t stride = (int64_t)gridDim.x * kGroups;
  v4s next[V];        // the next row's first part, on its way while this row is worked on
  int64_t next_label;
  auto ask = [&](int64_t at) __attribute__((always_inline)) {
    at = min(at, q.rows - 1);
    next_label = label_at(q.labels, q.label_bytes, at);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * LANES + lane) * 4;
      next[v] = v4s{-kInf, -kInf, -kInf, -kInf};
      if (c < columns) next[v] = *reinterpret_cast<const v4s *>(q.kept + at * columns + c);
    }
  };
  ask((int64_t)blockIdx.x * kGroups + group);
  for (int64_t r0 = (int64_t)blockIdx.x * kGroups; r0 < q.rows; r0 += stride) {
    const int64_t r = min(r0 + group, q.rows - 1);
    const bool here = r0 + group < q.rows;
    const float *from = q.kept + r * columns;
    const int64_t label = next_label;
#pragma unroll
    for (int v = 0; v < V; ++v) z[v] = next[v];
    if (r0 + stride < q.rows) ask(r0 + stride + group);
    const bool used = label != q.ignore, known = counts(q, label);
    float top[1] = {-kInf}, z_label = 0.f;
    if (known) {
      for (int i = 0; i < q.splits; ++i) z_label += from[i * q.rows * columns + label];
      z_label += q.kept_bias[label];
    }
    for (int i = 1; i < q.splits; ++i) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int c = (v * LANES + lane) * 4;
        if (c < columns) z[v] += *reinterpret_cast<const v4s *>(from + i * q.rows * columns + c);
      }
    }
    float s[3] = {0.f, 0.f, 0.f};        // sum, left, distance
    uint32_t in = 0;        // which of the lane's classes are not ruled out
    static_assert(4 * V <= 32, "");
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * LANES + lane) * 4;
      const v4s b = *reinterpret_cast<const v4s *>(q.kept_bias + min(c, columns - 4));
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool left = c + e < q.classes && b[e] != -kInf;
        in |= left ? 1u << (4 * v + e) : 0u;
        z[v][e] = c + e < q.classes ? z[v][e] + b[e] : -kInf;        // (what lies behind the last class is no sum of anything)
        top[0] = fmaxf(top[0], z[v][e]);
      }
    }
    group_join<LANES>(top, part_top, true);
    const float base = top[0] == -kInf ? 0.f : top[0];
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[0] += power(z[v][e], base);
        if (q.smoothing != 0.f) {
          const bool left = in >> (4 * v + e) & 1;
          s[1] += left ? 1.f : 0.f;
          s[2] = fmaf(left ? z[v][e] - base : 0.f, q.share, s[2]);
        }
      }
    group_join<LANES>(s, part_sum, false);
    const Stat stat = {top[0], s[0], s[2], s[1]};
    if (lane == 0 && here) {
      const float l = loss_of(q, stat, base, z_label, used, known);
      if (q.loss) q.loss[r] = l;
      losses += (double)l;
      used_rows += used;
    }
    if (!here) continue;        // (no barrier until the next row's: a workgroup's groups go on together)
    const bool flat = !used || !known || (top[0] == -kInf && s[0] == 0.f);
    const float f_total = flat ? 0.f : 1.f / (s[0] * q.keep), f_each = flat || q.smoothing == 0.f ? 0.f : q.smoothing / (s[1] * q.keep), from_top = flat ? kInf : base;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * LANES + lane) * 4;
      if (c >= columns) continue;
      v4s g;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        g[e] = power(z[v][e], from_top) * f_total - (in >> (4 * v + e) & 1 ? f_each : 0.f);
        if (flat) g[e] = 0.f;        // (whatever the logits are)
        else if (label == c + e) g[e] -= 1.f;
      }
      column[v] += g;
      if (q.signal) {
        T *to = static_cast<T *>(q.signal) + r * q.ldz + c;
        if constexpr (sizeof(T) == 2) *reinterpret_cast<uint64_t *>(to) = (uint64_t)f2bf_pk(g[2], g[3]) << 32 | f2bf_pk(g[0], g[1]);
        else *reinterpret_cast<v4s *>(to) = g;
      }
    }
  }
  if (q.db_part) {
    float *to = q.db_part + (int64_t)blockIdx.x * q.classes;
    if constexpr (kGroups > 1) {        // (the groups' sums in their order)
      __shared__ v4s sums[kGroups][V * LANES];
#pragma unroll
      for (int v = 0; v < V; ++v) sums[group][v * LANES + lane] = column[v];
      __syncthreads();
      for (int c = threadIdx.x; c < q.classes; c += 256) {
        float x = 0.f;
        for (int i = 0; i < kGroups; ++i) x += sums[i][c >> 2][c & 3];
        to[c] = x;
      }
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int c = (v * LANES + lane) * 4 + e;
          if (c < q.classes) to[c] = column[v][e];
        }
    }
  }
  if (lane == 0) {
    group_loss[group] = losses;
    group_used[group] = used_rows;
  }
  __syncthreads();
  losses = 0.0;
  used_rows = 0;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kGroups; ++i) {
      losses += group_loss[i];
      used_rows += group_used[i];
    }
  }
  add_up(q, losses, used_rows);
}

// Logits that the statistics left behind into the signal, eight classes of a row per lane, and its column sums over a workgroup's rows (300 x 32000 float32 13.6 us, 5.6 TB/s).
template <typename T>
__global__ __launch_bounds__(256) void k_left_signal(const Loss q) {
  const int c = ((int)blockIdx.x * 256 + threadIdx.x) * 8, columns = (q.classes + 7) / 8 * 8;
  static_assert(kLeftColumns == 256 * 8, "");
  if (c >= columns) return;
  const int64_t r0 = (int64_t)blockIdx.y * q.left_rows, r1 = min(q.rows, r0 + q.left_rows);
  float bias[8], column[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) bias[e] = column[e] = 0.f;
  if (q.bias) load8_n(static_cast<const T *>(q.bias) + c, q.classes - c, bias);
#pragma unroll 4
  for (int64_t r = r0; r < r1; ++r) {
    const RowInfo &row = q.info[r];
    const float base = row.base, f_total = row.f_total, f_each = row.f_each;
    const int at = row.label < 0 ? -1 : row.label - c;
    float z[8];
    load8_n(q.left + r * columns + c, 8, z);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float g = power(z[e], base) * f_total;
      if (q.smoothing != 0.f) g -= bias[e] != -kInf ? f_each : 0.f;
      g -= at == e ? 1.f : 0.f;
      z[e] = row.label < 0 || c + e >= q.classes ? 0.f : g;
      column[e] += z[e];
    }
    if (q.signal) store8_n(static_cast<T *>(q.signal) + r * q.ldz + c, 8, z);
  }
  if (q.db_part) store8_n(q.db_part + (int64_t)blockIdx.y * q.classes + c, q.classes - c, column);
}

// dw of up to R rows: a lane keeps a piece of 16 bytes of the signal's rows, times the factor, and goes down dw's rows, x's values for which wait in LDS.  Bound by the writes of dw where
// rows are few (6 rows, 3104 x 35488 float32: 441 MB in 63 us, 7.0 TB/s; 16 rows, 1024 x 35488 bf16: 73 MB in 29 us, 2.5).
struct Outer {
  const void *x, *signal;
  void *dw;
  const float *factor;
  int64_t ldx, ldz, lddw;
  int32_t rows, in, columns, per;      // per: rows of dw of a workgroup
  uint32_t across;                     // workgroups along a row
};
constexpr int kOuterPer = 64;
template <typename T, int R>
__global__ __launch_bounds__(256) void k_outer(const Outer a) {
  constexpr int E = Elem<T>::kPer16;
  __shared__ __align__(16) float xs[kOuterPer][R];
  const uint32_t down = blockIdx.x / a.across;
  const int c = (int)(blockIdx.x - down * a.across) * 256 * E + threadIdx.x * E, k0 = (int)down * a.per, here = min(a.per, a.in - k0);
  for (int i = threadIdx.x; i < here * R; i += 256) {
    const int r = i / here, k = i - r * here;
    xs[k][r] = r < a.rows ? to_f32(static_cast<const T *>(a.x)[r * a.ldx + k0 + k]) : 0.f;
  }
  const float factor = *a.factor;
  float g[R][E];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    u32x4v raw = {0, 0, 0, 0};
    if (r < a.rows && c < a.columns) raw = *reinterpret_cast<const u32x4v *>(static_cast<const T *>(a.signal) + r * a.ldz + c);      // (whole: the signal's rows have room for it)
    unpack<T>(raw, g[r]);
#pragma unroll
    for (int e = 0; e < E; ++e) g[r][e] *= factor;
  }
  __syncthreads();
  if (c >= a.columns) return;
  T *to = static_cast<T *>(a.dw) + (int64_t)k0 * a.lddw + c;
  const int left = a.columns - c;
#pragma unroll 2
  for (int k = 0; k < here; ++k, to += a.lddw) {
    float f[E] = {};
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int e = 0; e < E; ++e) f[e] = fmaf(xs[k][r], g[r][e], f[e]);
    if (left >= E) {
      store16(to, pack<T>(f));
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) if (e < left) to[e] = from_f32<T>(f[e]);
    }
  }
}

// Copies in rows on 16-byte boundaries: of x, with zeros for rows that do not count, and of w, each where there is one to make; and of the biases in float32 for kept logits.  Bound by memory (x of
// 4096 x 1024 and w of 1024 x 50001 bf16: 222 MB in 50 us, 4.4 TB/s).
template <typename T>
__global__ __launch_bounds__(256) void k_copy(const Loss q, const Packs a, float *bias) {
  constexpr int E = Elem<T>::kPer16;
  if (blockIdx.x == 0) clear_counters(q.head);
  const int64_t biases = bias ? (q.classes + 7) / 8 * 8 : 0;
  for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < a.pieces[0] + a.pieces[1] + biases; at += (int64_t)gridDim.x * 256) {
    if (at >= a.pieces[0] + a.pieces[1]) {
      const int64_t n = at - a.pieces[0] - a.pieces[1];
      bias[n] = n >= q.classes ? -kInf : q.bias ? to_f32(static_cast<const T *>(q.bias)[n]) : 0.f;
      continue;
    }
    const int which = at < a.pieces[0] ? 0 : 1;
    const Pack &p = a.p[which];
    const int64_t i = at - (which ? a.pieces[0] : 0), per = p.ldd / E, row = i / per, col = (i - row * per) * E;
    u32x4v x = load16_n(static_cast<const T *>(p.src) + row * p.ld + col, p.cols - col);
    if (which == 0 && !counts(q, label_at(q.labels, q.label_bytes, row))) x = u32x4v{0, 0, 0, 0};
    *reinterpret_cast<u32x4v *>(static_cast<T *>(p.dst) + row * p.ldd + col) = x;
  }
}
__global__ void k_no_rows(float *mean) { *mean = 0.f; }

// ---- host ----

template <typename T, int E, int WY, int WX, int KW>
void tiles(const Product &p, const Loss &q, bool statistics, bool direct, hipStream_t st) {
  const unsigned grid = (unsigned)(ceil_div(tiles_of(p), 8) * 8), threads = 64 * WY * WX * KW;
  auto launch = [&](auto dir, auto stages) {
    if (statistics && q.left) k_statistics<T, E, E, WY, WX, dir(), stages(), KW, true><<<grid, threads, 0, st>>>(p, q);
    else if (statistics) k_statistics<T, E, E, WY, WX, dir(), stages(), KW, false><<<grid, threads, 0, st>>>(p, q);
    else k_signal<T, E, WY, WX, dir(), stages(), KW><<<grid, threads, 0, st>>>(p, q);
  };
  if constexpr (E <= 64) {
    if (!direct) return launch(std::false_type(), std::integral_constant<int, 2>());
  }
  if constexpr (E < 256) {
    if (deep(E, tiles_of(p))) return launch(std::true_type(), std::integral_constant<int, 4>());
  }
  launch(std::true_type(), std::integral_constant<int, 2>());
}
// Statistics of up to 64 rows of bf16: tiles twice as wide (LossPlan::wide says when).
int wide_statistics(Product p, const Loss &q, bool direct, hipStream_t st) {
  p.tiles_n = (int32_t)ceil_div(p.N, kWideColumns);
  const unsigned grid = (unsigned)(ceil_div(tiles_of(p), 8) * 8);
  if (direct) k_statistics<bf16, 64, kWideColumns, 1, 4, true, 2, 1, false><<<grid, 256, 0, st>>>(p, q);
  else k_statistics<bf16, 64, kWideColumns, 1, 4, false, 2, 1, false><<<grid, 256, 0, st>>>(p, q);
  return ops_launched("linear cross-entropy");
}
template <typename T>
int logits(const Product &p, const Loss &q, int tile, bool statistics, bool direct, hipStream_t st) {
  if (tile == 32) tiles<T, 32, 1, 1, 4>(p, q, statistics, direct, st);
  if (tile == 64) tiles<T, 64, 2, 2, 1>(p, q, statistics, direct, st);
  if constexpr (sizeof(T) == 2) {
    if (tile == 128) tiles<T, 128, 2, 4, 1>(p, q, statistics, direct, st);
    if (tile == 256) tiles<T, 256, 2, 4, 1>(p, q, statistics, direct, st);
  }
  return ops_launched("linear cross-entropy");
}

template <typename T>
int kept_rows(const Loss &q, hipStream_t st) {
  const KeptShape s = kept_shape(q.rows, q.classes);
  const unsigned grid = (unsigned)std::min(ceil_div(q.rows, std::max(1, 256 / s.lanes)), s.groups), threads = (unsigned)std::max(256, s.lanes);
  if (s.lanes == 64 && s.pieces == 1) k_kept_rows<T, 64, 1><<<grid, threads, 0, st>>>(q);
  if (s.lanes == 64 && s.pieces == 4) k_kept_rows<T, 64, 4><<<grid, threads, 0, st>>>(q);
  if (s.lanes == 256 && s.pieces == 1) k_kept_rows<T, 256, 1><<<grid, threads, 0, st>>>(q);
  if (s.lanes == 256 && s.pieces == 4) k_kept_rows<T, 256, 4><<<grid, threads, 0, st>>>(q);
  if (s.lanes == 512 && s.pieces == 8) k_kept_rows<T, 512, 8><<<grid, threads, 0, st>>>(q);
  return ops_launched("linear cross-entropy rows");
}

template <typename T>
int loss(const cada_linear_xent *a, const LossPlan &f) {
  hipStream_t st = static_cast<hipStream_t>(a->stream);
  char *ws = static_cast<char *>(a->workspace);
  Loss q{};
  q.labels = a->labels; q.bias = a->bias; q.head = reinterpret_cast<LossHead *>(ws);
  q.stats = reinterpret_cast<float *>(ws + f.off_stats); q.info = reinterpret_cast<RowInfo *>(ws + f.off_info); q.z_label = reinterpret_cast<float *>(ws + f.off_label);
  q.loss = a->loss ? a->loss : reinterpret_cast<float *>(ws + f.off_loss); q.mean = a->mean;
  q.rows = a->rows; q.ignore = a->ignore_index; q.chunks = f.chunks; q.classes = (int32_t)a->classes; q.label_bytes = a->label_bytes;
  q.smoothing = (float)a->smoothing; q.keep = (float)(1.0 - a->smoothing); q.scale = (float)a->scale; q.share = (float)(1.0 / (double)a->classes);
  const T *x = static_cast<const T *>(a->x), *w = static_cast<const T *>(a->w);
  int64_t ldx = a->ldx, ldw = a->ldw, x_cols = a->in, w_cols = a->classes;
  Packs k{};
  if (f.copy_x) {
    k.p[0] = Pack{a->x, ws + f.off_x, a->ldx, a->rows, a->in, packed_ld(a->in)};
    k.pieces[0] = a->rows * (k.p[0].ldd / Elem<T>::kPer16);
    x = static_cast<const T *>(k.p[0].dst); ldx = x_cols = k.p[0].ldd;
  }
  if (f.copy_w) {
    k.p[1] = Pack{a->w, ws + f.off_w, a->ldw, a->in, a->classes, packed_ld(a->classes)};
    k.pieces[1] = a->in * (k.p[1].ldd / Elem<T>::kPer16);
    w = static_cast<const T *>(k.p[1].dst); ldw = w_cols = k.p[1].ldd;
  }
  float *bias = f.kept ? reinterpret_cast<float *>(ws + f.off_bias) : nullptr;
  if (f.copy_x || f.copy_w) {
    k_copy<T><<<many(k.pieces[0] + k.pieces[1] + (bias ? eights(a->classes) : 0)), 256, 0, st>>>(q, k, bias);
    if (int rc = ops_launched("linear cross-entropy copy")) return rc;
  }
  Product z{};
  lay(&z, f.logits, x, ldx, w, ldw, a->rows, a->classes, a->in, nullptr);
  z.b_cols = w_cols;
  if (f.kept) {
    z.partial = reinterpret_cast<float *>(ws + f.off_stats);
    q.kept = z.partial; q.kept_bias = bias; q.splits = f.logits.splits; q.signal = f.grads ? ws + f.off_signal : nullptr; q.ldz = f.ldz;
    q.db_part = a->db ? reinterpret_cast<float *>(ws + f.off_db) : nullptr;
    if (int rc = linear_sums(a->type, f.logits.tile, f.direct, z, st)) return rc;
    if (int rc = kept_rows<T>(q, st)) return rc;
  } else {
    q.left = f.left ? reinterpret_cast<float *>(ws + f.off_left) : nullptr;
    q.left_rows = f.left_rows;
    if (int rc = f.wide ? wide_statistics(z, q, f.direct, st) : logits<T>(z, q, f.logits.tile, true, f.direct, st)) return rc;
    while (q.lanes < 6 && ((int64_t)kLossGroups << q.lanes) < a->rows) ++q.lanes;
    const unsigned groups = (unsigned)std::min<int64_t>(ceil_div(a->rows, 1 << q.lanes), kLossGroups);
    if (q.smoothing != 0.f) k_rows<true><<<groups, 1024, 0, st>>>(q);
    else k_rows<false><<<groups, 1024, 0, st>>>(q);
    if (int rc = ops_launched("linear cross-entropy rows")) return rc;
  }
  if (!f.signal) return CADA_OK;
  void *signal = f.grads ? ws + f.off_signal : nullptr;
  for (int64_t i = 0; i < f.pieces; ++i) {
    const int64_t first = i * f.piece, here = std::min(f.piece, a->classes - first);
    q.first = (int32_t)first; q.signal = signal; q.ldz = f.ldz; q.db_part = a->db ? reinterpret_cast<float *>(ws + f.off_db) : nullptr;
    if (f.left) {
      k_left_signal<T><<<dim3((unsigned)ceil_div(a->classes, kLeftColumns), (unsigned)f.strips), 256, 0, st>>>(q);
      if (int rc = ops_launched("linear cross-entropy signal")) return rc;
    } else if (!f.kept) {
      lay(&z, f.piece_logits, x, ldx, w + first, ldw, a->rows, here, a->in, nullptr);
      z.b_cols = w_cols - first;
      if (int rc = logits<T>(z, q, f.piece_logits.tile, false, f.direct, st)) return rc;
    }
    Product dx{}, dw{};
    Join j{};
    if (a->dx) {
      Cut c = f.dx;
      c.splits = (int)std::min<int64_t>(c.splits, ceil_div(here, c.k_per_split));        // (the last piece may have less)
      lay(&dx, c, signal, f.ldz, w + first, ldw, a->rows, a->in, here, nullptr);
      if (f.pieces > 1 || f.dx.splits > 1) dx.partial = reinterpret_cast<float *>(ws + f.off_dx);
      dx.add = i > 0;
      dx.epi.out = a->dx; dx.epi.ldo = a->lddx; dx.factor = &q.head->factor;
    }
    if (f.outer) {
      Outer o{};
      o.x = x; o.signal = signal; o.dw = static_cast<T *>(a->dw) + first; o.factor = &q.head->factor; o.ldx = ldx; o.ldz = f.ldz; o.lddw = a->lddw;
      o.rows = (int32_t)a->rows; o.in = (int32_t)a->in; o.columns = (int32_t)here;
      o.across = (uint32_t)ceil_div(here, 256 * Elem<T>::kPer16);
      o.per = (int32_t)std::clamp<int64_t>(ceil_div(a->in * o.across, 16 * kCUs), 4, kOuterPer);
      const unsigned grid = o.across * (unsigned)ceil_div(a->in, o.per);
      if (a->rows <= 4) k_outer<T, 4><<<grid, 256, 0, st>>>(o);
      else if (a->rows <= 8) k_outer<T, 8><<<grid, 256, 0, st>>>(o);
      else k_outer<T, 16><<<grid, 256, 0, st>>>(o);
      if (int rc = ops_launched("linear cross-entropy outer product")) return rc;
    } else if (a->dw) {
      lay(&dw, f.dw, x, ldx, signal, f.ldz, a->in, here, a->rows, reinterpret_cast<float *>(ws + f.off_dw));
      dw.a_cols = x_cols; dw.b_cols = eights(here);
      dw.epi.out = static_cast<T *>(a->dw) + first; dw.epi.ldo = a->lddw; dw.factor = &q.head->factor;
    }
    if (a->dx || (a->dw && !f.outer)) {
      if (int rc = linear_products(a->type, a->dx ? f.dx.tile : f.dw.tile, f.direct, dx, dw, st)) return rc;
    }
    if (i == f.pieces - 1) {
      j.p[0] = dx;
      j.p[0].splits = f.dx.splits;
    }
    j.p[1] = dw;
    if (a->db) { j.db_part = q.db_part; j.db_factor = &q.head->factor; j.db = static_cast<T *>(a->db) + first; j.db_parts = (int)f.strips; j.db_n = (int)here; }
    if (int rc = linear_join(a->type, j, st)) return rc;
  }
  return CADA_OK;
}

bool check(const cada_linear_xent *a) {
  if (!a) { set_error("the arguments are NULL"); return false; }
  if (a->rows < 0 || a->rows > (int64_t)1 << 30) { set_error("rows must be in [0, 2^30] (got %lld)", (long long)a->rows); return false; }
  if (a->in < 1 || a->in > CADA_MAX_WIDTH || a->classes < 1 || a->classes > CADA_MAX_WIDTH) { set_error("in and classes must be in [1, %d] (got %lld, %lld)", CADA_MAX_WIDTH, (long long)a->in, (long long)a->classes); return false; }
  if (a->type != CADA_F32 && a->type != CADA_BF16) { set_error("type must be CADA_F32 or CADA_BF16 (got %d)", a->type); return false; }
  if (a->label_bytes != 4 && a->label_bytes != 8) { set_error("label_bytes must be 4 or 8 (got %d)", a->label_bytes); return false; }
  if (!(a->smoothing >= 0.0 && a->smoothing < 1.0)) { set_error("smoothing must be in [0, 1)"); return false; }
  const int64_t t = std::max({ceil_div(a->rows, 64) * ceil_div(a->classes, 64), ceil_div(a->rows, 64) * ceil_div(a->in, 64), ceil_div(a->in, 64) * ceil_div(a->classes, 64)});
  if (t > kMostTiles) { set_error("more than %lld tiles of 64 x 64 outputs", (long long)kMostTiles); return false; }
  return true;
}

}  // namespace
}  // namespace cada

using namespace cada;

extern "C" {

int cada_linear_xent_workspace(cada_linear_xent *a) {
  if (!check(a)) return CADA_EINVAL;
  a->workspace_bytes = plan_loss(a).bytes;
  return CADA_OK;
}

int cada_linear_cross_entropy(const cada_linear_xent *a) {
  if (!check(a)) return CADA_EINVAL;
  const bool any = a->rows > 0;
  if (any) {
    if (!ops_check_table("x", a->x, a->ldx, a->in, a->type) || !ops_check_table("w", a->w, a->ldw, a->classes, a->type)) return CADA_EINVAL;
    if (a->bias && !ops_check_table("bias", a->bias, a->classes, a->classes, a->type)) return CADA_EINVAL;
    if (!a->labels) { set_error("labels is NULL"); return CADA_EINVAL; }
    if (reinterpret_cast<uintptr_t>(a->labels) % a->label_bytes != 0) { set_error("labels is not aligned to its elements"); return CADA_EINVAL; }
    if (a->dx && !ops_check_table("dx", a->dx, a->lddx, a->in, a->type)) return CADA_EINVAL;
  }
  if (a->dw && !ops_check_table("dw", a->dw, a->lddw, a->classes, a->type)) return CADA_EINVAL;
  if (a->db && !ops_check_table("db", a->db, a->classes, a->classes, a->type)) return CADA_EINVAL;
  if ((a->mean && !ops_check_table("mean", a->mean, 1, 1, CADA_F32)) || (a->loss && !ops_check_table("loss", a->loss, 1, 1, CADA_F32))) return CADA_EINVAL;
  const LossPlan f = plan_loss(a);
  if (int rc = ops_check_workspace(a->workspace, a->workspace_bytes, f.bytes)) return rc;
  const size_t elem = type_bytes(a->type);
  const Span outs[] = {span("dx", any ? a->dx : nullptr, a->rows, a->lddx, a->in, elem), span("dw", a->dw, a->in, a->lddw, a->classes, elem), span("db", a->db, 1, a->classes, a->classes, elem),
                       span("loss", a->loss, (size_t)a->rows * 4), span("mean", a->mean, 4), span("workspace", a->workspace, f.bytes)};
  const Span ins[] = {span("x", any ? a->x : nullptr, a->rows, a->ldx, a->in, elem), span("w", any ? a->w : nullptr, a->in, a->ldw, a->classes, elem), span("bias", any ? a->bias : nullptr, 1, a->classes, a->classes, elem),
                      span("labels", a->labels, (size_t)a->rows * a->label_bytes)};
  for (int i = 0; i < 6; ++i) {
    for (const Span &in : ins)
      if (!ops_apart(outs[i], in)) return CADA_EINVAL;
    for (int j = 0; j < i; ++j)
      if (!ops_apart(outs[i], outs[j])) return CADA_EINVAL;
  }
  if (!any) {
    if (a->mean) {
      k_no_rows<<<1, 1, 0, static_cast<hipStream_t>(a->stream)>>>(a->mean);
      if (int rc = ops_launched("linear cross-entropy")) return rc;
    }
    cada_linear_grad g{};
    g.in = a->in; g.out = a->classes; g.type = a->type; g.dw = a->dw; g.lddw = a->lddw; g.db = a->db; g.stream = a->stream;
    return cada_linear_backward(&g);        // (clears both)
  }
  return a->type == CADA_BF16 ? loss<bf16>(a, f) : loss<float>(a, f);
}

}  // extern "C"
