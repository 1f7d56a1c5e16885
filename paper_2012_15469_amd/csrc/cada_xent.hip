// Softmax cross-entropy over any number of classes, with its gradient (cada_ops.h).
//
// A row's logits are read once and stay in registers, as they were read, between the statistics and the gradient: max, then sum of exp(z - max) with the
// classes that are left and their logits' mean (smoothing), then softmax - target.  A group of 4 to 1024 lanes takes a row, by its length; rows beyond what
// 1024 lanes hold (131072 bf16, 65536 float32) are read again.  Two launches: the rows that count, which every gradient is divided by, and the rows, the last
// workgroup of which adds the losses up in the rows' order; rows that fit one workgroup are counted there, in one launch.
#include <algorithm>

#include "cada_ops_internal.h"

namespace cada {
namespace {

// Rows that are not ignored, and workgroups whose losses are written: counted in kCounters places of a line each, and those that are full in one more (one
// counter for all takes 12 ns per workgroup: 205 us for 16384).
constexpr uint32_t kCounters = 64, kLineWords = 32;
struct Head { int64_t count; uint32_t pad[kLineWords - 2]; uint32_t full[kLineWords]; uint32_t done[kCounters * kLineWords]; };
struct Xent {
  const void *logits, *labels;
  void *grad;
  float *loss, *mean;
  Head *head;
  int64_t rows, ldz, ldg, ignore;
  int32_t classes, label_bytes;
  float smoothing, keep, scale;      // keep = 1 - smoothing, rounded once
};

__device__ __forceinline__ int64_t label_at(const void *labels, int bytes, int64_t r) {
  return bytes == 8 ? static_cast<const int64_t *>(labels)[r] : (int64_t)static_cast<const int32_t *>(labels)[r];
}

__global__ __launch_bounds__(1024) void k_count(const void *labels, int bytes, int64_t rows, int64_t ignore, Head *head, float *mean) {
  __shared__ int64_t part[16];
  int64_t n = 0;
#pragma unroll 4
  for (int64_t r = threadIdx.x; r < rows; r += 1024) n += label_at(labels, bytes, r) != ignore;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x < kCounters) head->done[threadIdx.x * kLineWords] = 0;
  if (threadIdx.x == 0) {
    head->full[0] = 0;
    n = 0;
    for (int i = 0; i < 16; ++i) n += part[i];
    head->count = n;
    if (rows == 0 && mean) *mean = 0.f;
  }
}

// Over the LANES lanes of a row's group; every lane gets the result.
template <int LANES, typename OP>
__device__ __forceinline__ float group_reduce(float x, float *part, OP op) {
  constexpr int W = LANES < 64 ? LANES : 64;
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) x = op(x, __shfl_xor(x, o, 64));
  if constexpr (LANES > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    x = part[0];
#pragma unroll
    for (int i = 1; i < LANES / 64; ++i) x = op(x, part[i]);
  }
  return x;
}

// Exponentials of either type are the hardware's exp2 of the difference times log2(e), both rounded to float32: off by about (z - top) 2^-23 and an ulp or two, relative, where a
// library's exponential would be off by an ulp.  Small probabilities take the larger errors, so that sums and gradients are off by less than float32's own sums leave
// (ten classes: 5e-8 from 64 bits, relative in the 2-norm).
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kInf = __builtin_inff();

// A row in pieces of 16 bytes, which the lanes take in turn, and the few classes behind the last whole piece, one per lane.  Pieces and classes that do not exist are -inf.
template <typename T> constexpr uint32_t kInfBits = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;

// LANES lanes for a row, V pieces each; V = 0: as many as it takes, read again for each use.
template <typename T, int LANES, int V, bool SMOOTH>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES, LANES >= 512 ? 4 : 2) void k_rows(const Xent a) {
  constexpr int kRows = LANES < 256 ? 256 / LANES : 1, E = Elem<T>::kPer16;
  __shared__ float part[16];
  __shared__ bool last;
  const int lane = threadIdx.x % LANES;
  const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES;
  const bool here = row < a.rows;
  const int64_t r = here ? row : a.rows - 1;
  const T *z = static_cast<const T *>(a.logits) + r * a.ldz;
  T *g = a.grad ? static_cast<T *>(a.grad) + r * a.ldg : nullptr;
  static_assert(LANES >= E, "one class per lane behind the last piece");
  const int whole = a.classes / E * E;
  u32x4v raw[V > 0 ? V : 1];
  if constexpr (V > 0) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * LANES + lane) * E;
      raw[v] = u32x4v{kInfBits<T>, kInfBits<T>, kInfBits<T>, kInfBits<T>};
      if (c < whole) raw[v] = load16(z + c);
    }
  }
  const float behind = lane < a.classes - whole ? to_f32(z[whole + lane]) : -kInf;
  const int64_t label = label_at(a.labels, a.label_bytes, r);
  const bool used = label != a.ignore, known = label >= 0 && label < a.classes;
  const float zy = used && known ? to_f32(z[label]) : 0.f;      // (read before the gradient may overwrite it)
  // (a launch of one workgroup counts its rows itself, and no other kernel runs)
  const bool alone = gridDim.x == 1;
  int64_t count;
  if (alone) {
    const float n = group_reduce<(LANES < 256 ? 256 : LANES)>(here && lane == 0 && used ? 1.f : 0.f, part, [](float x, float y) { return x + y; });
    count = (int64_t)n;
  } else {
    count = a.head->count;
  }
  const float inv = a.scale / (float)max(count, (int64_t)1);

  // Calls f(class of the first, logits) for each piece of this lane.  (The empty asm keeps the compiler from holding all pieces as float32 from one
  // use to the next, which is twice the registers and spills.)
  auto pieces = [&](auto f) __attribute__((always_inline)) {
    float x[E];
    if constexpr (V > 0) {
      int first = lane * E;
      asm volatile("" : "+v"(first));        // (nor which pieces exist, in scalar registers)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        asm volatile("" : "+v"(raw[v]));
        unpack<T>(raw[v], x);
        f(v * LANES * E + first, x);
        if constexpr (V >= 16) __builtin_amdgcn_sched_barrier(0);        // (piece by piece: interleaved, the comparisons' results spill)
      }
    } else {
      for (int c = lane * E; c < whole; c += LANES * E) {
        unpack<T>(load16(z + c), x);
        f(c, x);
      }
    }
  };
  float top = -kInf;
  pieces([&](int, const float (&x)[E]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < E; ++i) top = fmaxf(top, x[i]);
  });
  top = fmaxf(top, behind);
  top = group_reduce<LANES>(top, part, [](float x, float y) { return fmaxf(x, y); });      // (a NaN, which this drops, is in the sum below)
  // Differences to the largest first, so that a mask of the type's lowest value (or a row of nothing else) overflows nowhere.  A row of nothing but -inf and
  // NaN has top = -inf; its exponentials are taken against 0, so that those of -inf are 0 and only a NaN makes the sum NaN.
  const float base = top == -kInf ? 0.f : top, share = 1.f / (float)a.classes;
  constexpr bool kBallot = LANES >= 64;        // a wavefront's lanes have one row: the classes left are counted by the scalar unit
  uint32_t wave_left = 0;
  float total = 0.f, left = 0.f, mean_left = 0.f;        // mean_left: first the sum of (z - top) / classes, which cannot overflow
  auto statistics = [&](float x) __attribute__((always_inline)) {
    const float d = x - base;
    total += __builtin_amdgcn_exp2f(d * kLog2e);
    if constexpr (SMOOTH) {
      const bool in = x != -kInf;
      if constexpr (kBallot) wave_left += (uint32_t)__popcll(__ballot(in));
      else left += in ? 1.f : 0.f;
      mean_left = fmaf(in ? d : 0.f, share, mean_left);
    }
  };
  pieces([&](int, const float (&x)[E]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < E; ++i) statistics(x[i]);
  });
  statistics(behind);
  auto plus = [](float x, float y) { return x + y; };
  total = group_reduce<LANES>(total, part, plus);
  const bool none = top == -kInf && total == 0.f;        // no class left
  if constexpr (SMOOTH) {
    if constexpr (kBallot) left = lane % 64 == 0 ? (float)wave_left : 0.f;
    left = group_reduce<LANES>(left, part, plus);
    mean_left = group_reduce<LANES>(mean_left, part, plus) * ((float)a.classes / left);
  }
  if (here && lane == 0 && a.loss) {
    // log(sum exp z) - keep z_y - smoothing mean_left z, with top taken out of all three
    float l = logf(total) - a.keep * (zy - base) - (SMOOTH ? a.smoothing * mean_left : 0.f);
    if (none) l = kInf;
    if (!known) l = __builtin_nanf("");
    // (to where every XCD sees it, for the last workgroup)
    __hip_atomic_store(a.loss + r, used ? l : 0.f, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  if (g) {
    const bool flat = !used || !known || none;      // no gradient
    const float f_total = inv / total, f_keep = a.keep * inv, f_each = SMOOTH ? a.smoothing / left * inv : 0.f;
    auto gradient = [&](float x) __attribute__((always_inline)) {
      float p = __builtin_amdgcn_exp2f((x - base) * kLog2e) * f_total;
      if constexpr (SMOOTH) p -= x != -kInf ? f_each : 0.f;
      return p;
    };
    pieces([&](int c, float (&x)[E]) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < E; ++i) x[i] = gradient(x[i]);
      if (label >= c && label < c + E) {
#pragma unroll
        for (int i = 0; i < E; ++i) if (label == c + i) x[i] -= f_keep;
      }
      if (flat) {
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = 0.f;
      }
      if (here && c < whole) store16(g + c, pack<T>(x));
    });
    if (here && lane < a.classes - whole) g[whole + lane] = from_f32<T>(flat ? 0.f : gradient(behind) - (label == whole + lane ? f_keep : 0.f));
  }
  if (!a.mean) return;
  // The losses that this workgroup wrote are where the last one reads them before it counts itself (no fence: it would write back the gradient's lines).
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0 && alone) last = true;
  if (threadIdx.x == 0 && !alone) {
    const uint32_t c = blockIdx.x % kCounters, of_mine = (gridDim.x - c + kCounters - 1) / kCounters, counters = min(gridDim.x, kCounters);
    last = __hip_atomic_fetch_add(&a.head->done[c * kLineWords], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == of_mine - 1 &&
           __hip_atomic_fetch_add(&a.head->full[0], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == counters - 1;
  }
  __syncthreads();
  if (!last) return;
  constexpr int TH = LANES < 256 ? 256 : LANES;
  __shared__ double sums[TH / 64];
  double s = 0.0;
#pragma unroll 8
  for (int64_t i = threadIdx.x; i < a.rows; i += TH) s += (double)__hip_atomic_load(a.loss + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  s = wave_sum_f64(s);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0;
    for (int i = 0; i < TH / 64; ++i) s += sums[i];
    *a.mean = (float)(s / (double)max(count, (int64_t)1));
  }
}

int rows_together(int lanes) { return lanes < 256 ? 256 / lanes : 1; }      // of a workgroup
template <typename T, int LANES, int V>
void launch_rows(const Xent &x, hipStream_t st) {
  const unsigned grid = (unsigned)ceil_div(x.rows, rows_together(LANES)), threads = LANES < 256 ? 256 : LANES;
  if (x.smoothing != 0.f) k_rows<T, LANES, V, true><<<grid, threads, 0, st>>>(x);
  else k_rows<T, LANES, V, false><<<grid, threads, 0, st>>>(x);
}
// Lanes and pieces by the row's length: few lanes for a few classes, so that a wavefront holds several rows; beyond that as many as keep a lane's pieces in at
// most 64 registers, so that two workgroups of 512 fit a CU and one reads while the other computes.
int lanes_for(int64_t classes, int per16) {
  const int64_t n = ceil_div(classes, per16);
  return n <= per16 ? per16 : n <= 16 ? 16 : n <= 256 ? 64 : n <= 2048 ? 256 : n <= 8192 ? 512 : 1024;
}
template <typename T>
int rows(const Xent &x, hipStream_t st) {
  const int64_t n = ceil_div(x.classes, Elem<T>::kPer16);
  switch (lanes_for(x.classes, Elem<T>::kPer16)) {
    case Elem<T>::kPer16: launch_rows<T, Elem<T>::kPer16, 1>(x, st); break;
    case 16: launch_rows<T, 16, 1>(x, st); break;
    case 64: if (n <= 64) launch_rows<T, 64, 1>(x, st); else launch_rows<T, 64, 4>(x, st); break;
    case 256: if (n <= 1024) launch_rows<T, 256, 4>(x, st); else launch_rows<T, 256, 8>(x, st); break;
    case 512: if (n <= 4096) launch_rows<T, 512, 8>(x, st); else launch_rows<T, 512, 16>(x, st); break;
    default: if (n <= 16384) launch_rows<T, 1024, 16>(x, st); else launch_rows<T, 1024, 0>(x, st);
  }
  return ops_launched("cross-entropy");
}

bool check(const cada_xent *a) {
  if (!a) { set_error("the arguments are NULL"); return false; }
  if (a->rows < 0 || a->rows > (int64_t)1 << 30) { set_error("rows must be in [0, 2^30] (got %lld)", (long long)a->rows); return false; }
  if (a->classes < 1 || a->classes > 0x7fffffff - (1 << 20)) { set_error("classes must be in [1, 2^31 - 2^20) (got %lld)", (long long)a->classes); return false; }
  if (a->type != CADA_F32 && a->type != CADA_BF16) { set_error("type must be CADA_F32 or CADA_BF16 (got %d)", a->type); return false; }
  return true;
}

bool one_workgroup(const cada_xent *a) { return a->rows > 0 && a->rows <= rows_together(lanes_for(a->classes, 16 / (int)type_bytes(a->type))); }
size_t workspace(const cada_xent *a) { return (one_workgroup(a) ? 0 : ops_align(sizeof(Head))) + (a->mean && !a->loss ? ops_align((size_t)a->rows * 4) : 0); }

}  // namespace
}  // namespace cada

using namespace cada;

extern "C" {

int cada_xent_workspace(cada_xent *a) {
  if (!check(a)) return CADA_EINVAL;
  a->workspace_bytes = workspace(a);
  return CADA_OK;
}

int cada_cross_entropy(const cada_xent *a) {
  if (!check(a)) return CADA_EINVAL;
  if (a->label_bytes != 4 && a->label_bytes != 8) { set_error("label_bytes must be 4 or 8 (got %d)", a->label_bytes); return CADA_EINVAL; }
  if (!(a->smoothing >= 0.0 && a->smoothing < 1.0)) { set_error("smoothing must be in [0, 1)"); return CADA_EINVAL; }
  if (a->rows > 0) {
    if (!a->logits || !a->labels) { set_error("logits and labels must be device pointers"); return CADA_EINVAL; }
    if (a->ldz < a->classes || (a->grad && a->ldg < a->classes)) { set_error("the row length of logits or grad is less than the %lld classes", (long long)a->classes); return CADA_EINVAL; }
    if (a->grad == a->logits && a->rows > 1 && a->ldg != a->ldz) { set_error("grad in the place of logits must have their row length"); return CADA_EINVAL; }
    if (reinterpret_cast<uintptr_t>(a->logits) % type_bytes(a->type) != 0 || reinterpret_cast<uintptr_t>(a->grad) % type_bytes(a->type) != 0 ||
        reinterpret_cast<uintptr_t>(a->labels) % a->label_bytes != 0) { set_error("logits, grad or labels are not aligned to their elements"); return CADA_EINVAL; }
  }
  const int lanes = lanes_for(a->classes, 16 / (int)type_bytes(a->type));
  if (ceil_div(a->rows, rows_together(lanes)) * std::max(lanes, 256) >= (int64_t)1 << 32) { set_error("%lld rows of %lld classes are more than one launch takes", (long long)a->rows, (long long)a->classes); return CADA_EINVAL; }
  if (int rc = ops_check_workspace(a->workspace, a->workspace_bytes, workspace(a))) return rc;
  const size_t elem = type_bytes(a->type);
  const bool any = a->rows > 0;
  const Span logits = span("logits", any ? a->logits : nullptr, a->rows, a->ldz, a->classes, elem), labels = span("labels", a->labels, (size_t)a->rows * a->label_bytes);
  const Span outs[] = {span("grad", any ? a->grad : nullptr, a->rows, a->ldg, a->classes, elem), span("loss", a->loss, (size_t)a->rows * sizeof(float)), span("mean", a->mean, sizeof(float)),
                       span("workspace", a->workspace, workspace(a))};
  for (int i = 0; i < 4; ++i) {
    if ((!(i == 0 && a->grad == a->logits) && !ops_apart(outs[i], logits)) || !ops_apart(outs[i], labels)) return CADA_EINVAL;
    for (int j = 0; j < i; ++j)
      if (!ops_apart(outs[i], outs[j])) return CADA_EINVAL;
  }
  hipStream_t st = static_cast<hipStream_t>(a->stream);
  Head *head = static_cast<Head *>(a->workspace);
  Xent x{};
  x.logits = a->logits; x.labels = a->labels; x.grad = a->grad;
  x.loss = a->loss ? a->loss : a->mean ? reinterpret_cast<float *>(static_cast<char *>(a->workspace) + (one_workgroup(a) ? 0 : ops_align(sizeof(Head)))) : nullptr;
  x.mean = a->mean; x.head = head; x.rows = a->rows; x.ldz = a->ldz; x.ldg = a->ldg; x.ignore = a->ignore_index;
  x.classes = (int32_t)a->classes; x.label_bytes = a->label_bytes;
  x.smoothing = (float)a->smoothing; x.keep = (float)(1.0 - a->smoothing); x.scale = (float)a->scale;
  if (!one_workgroup(a)) {
    k_count<<<1, 1024, 0, st>>>(a->labels, a->label_bytes, a->rows, a->ignore_index, head, a->mean);
    if (int rc = ops_launched("cross-entropy count")) return rc;
  }
  if (a->rows == 0) return CADA_OK;
  return a->type == CADA_BF16 ? rows<bf16>(x, st) : rows<float>(x, st);
}

}  // extern "C"
