// Softmax cross-entropy over any number of classes, with its gradient (cada_ops.h).
//
// A row's logits are read once and stay in registers between the statistics and the gradient: max, then sum of exp(z - max) with the
// classes that are left and their logits' sum (smoothing), then softmax - target.  A group of 16, 64, 256 or 1024 lanes takes a row, by its length;
// rows beyond what 1024 lanes hold are read again for the gradient.
#include <algorithm>

#include "cada_ops_internal.h"

namespace cada {
namespace {

struct Xent {
  const void *logits, *labels;
  void *grad;
  float *loss;
  const int64_t *count;       // rows that are not ignored
  int64_t rows, ldz, ldg, ignore;
  int32_t classes, label_bytes;
  float smoothing, keep, scale;      // keep = 1 - smoothing, rounded once
};

__device__ __forceinline__ int64_t label_at(const void *labels, int bytes, int64_t r) {
  return bytes == 8 ? static_cast<const int64_t *>(labels)[r] : (int64_t)static_cast<const int32_t *>(labels)[r];
}

__global__ __launch_bounds__(1024) void k_count(const void *labels, int bytes, int64_t rows, int64_t ignore, int64_t *count) {
  __shared__ int64_t part[16];
  int64_t n = 0;
  for (int64_t r = threadIdx.x; r < rows; r += 1024) n += label_at(labels, bytes, r) != ignore;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x == 0) {
    n = 0;
    for (int i = 0; i < 16; ++i) n += part[i];
    *count = n;
  }
}

__global__ __launch_bounds__(1024) void k_mean(const float *loss, int64_t rows, const int64_t *count, float *mean) {
  __shared__ double part[16];
  double s = 0.0;
  for (int64_t r = threadIdx.x; r < rows; r += 1024) s += (double)loss[r];
  s = wave_sum_f64(s);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0;
    for (int i = 0; i < 16; ++i) s += part[i];
    *mean = (float)(s / (double)max(*count, (int64_t)1));
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

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kInf = __builtin_inff();

// Eight logits of a row from class c on; classes beyond the last are -inf.
template <typename T>
__device__ __forceinline__ void logits8(const T *z, int c, int classes, float (&f)[8]) {
  load8_n(z + c, classes - c, f);
#pragma unroll
  for (int i = 0; i < 8; ++i) if (c + i >= classes) f[i] = -kInf;
}

template <typename T, int LANES, int V>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void k_rows(const Xent a) {
  constexpr int kRows = LANES < 256 ? 256 / LANES : 1;
  __shared__ float part[16];
  const int lane = threadIdx.x % LANES;
  const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES;
  const bool here = row < a.rows;
  const int64_t r = here ? row : a.rows - 1;
  const T *z = static_cast<const T *>(a.logits) + r * a.ldz;
  T *g = a.grad ? static_cast<T *>(a.grad) + r * a.ldg : nullptr;
  const int64_t label = label_at(a.labels, a.label_bytes, r);
  const bool used = label != a.ignore, known = label >= 0 && label < a.classes;
  const float zy = used && known ? to_f32(z[label]) : 0.f;      // (read before the gradient may overwrite it)
  const float inv = a.scale / (float)max(*a.count, (int64_t)1);

  float f[V > 0 ? V : 1][8];
  float top = -kInf;
  auto bigger = [](float x, float y) { return fmaxf(x, y); };      // (a NaN is in the sum below)
  auto plus = [](float x, float y) { return x + y; };
  if constexpr (V > 0) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      logits8(z, (v * LANES + lane) * 8, a.classes, f[v]);
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, f[v][i]);
    }
  } else {
    for (int c = lane * 8; c < a.classes; c += LANES * 8) {
      logits8(z, c, a.classes, f[0]);
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, f[0][i]);
    }
  }
  top = group_reduce<LANES>(top, part, bigger);
  // Differences to the largest first, so that a mask of the type's lowest value (or a row of nothing else) overflows nowhere.  A row with
  // nothing left has top = -inf; its exponentials are taken against 0, so that they are 0 and not NaN.
  const bool none = top == -kInf;
  const float base = none ? 0.f : top, share = 1.f / (float)a.classes;
  float total = 0.f, left = 0.f, mean_left = 0.f;        // mean_left: first the sum of (z - top) / classes, which cannot overflow
  auto statistics = [&](const float (&x)[8]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float d = x[i] - base;
      total += __builtin_amdgcn_exp2f(d * kLog2e);
      left += x[i] != -kInf ? 1.f : 0.f;
      mean_left = fmaf(x[i] != -kInf ? d : 0.f, share, mean_left);
    }
  };
  if constexpr (V > 0) {
#pragma unroll
    for (int v = 0; v < V; ++v) statistics(f[v]);
  } else {
    for (int c = lane * 8; c < a.classes; c += LANES * 8) { logits8(z, c, a.classes, f[0]); statistics(f[0]); }
  }
  total = group_reduce<LANES>(total, part, plus);
  if (a.smoothing != 0.f) {
    left = group_reduce<LANES>(left, part, plus);
    mean_left = group_reduce<LANES>(mean_left, part, plus) * ((float)a.classes / left);
  }
  if (here && lane == 0 && a.loss) {
    // log(sum exp z) - keep z_y - smoothing mean_left z, with top taken out of all three
    float l = logf(total) - a.keep * (zy - base) - (a.smoothing != 0.f ? a.smoothing * mean_left : 0.f);
    if (none) l = kInf;
    if (!known) l = __builtin_nanf("");
    a.loss[r] = used ? l : 0.f;
  }
  if (!g) return;
  const bool flat = !used || !known || none;      // no gradient
  const float f_total = flat ? 0.f : inv / total, f_keep = a.keep * inv, f_each = a.smoothing != 0.f ? a.smoothing / left * inv : 0.f;
  auto gradient = [&](int c, float (&x)[8]) __attribute__((always_inline)) {
    if (c >= a.classes) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float p = __builtin_amdgcn_exp2f((x[i] - base) * kLog2e) * f_total;
      if (x[i] != -kInf) p -= f_each;
      if (label == c + i) p -= f_keep;
      x[i] = flat ? 0.f : p;
    }
    if (here) store8_n(g + c, a.classes - c, x);
  };
  if constexpr (V > 0) {
#pragma unroll
    for (int v = 0; v < V; ++v) gradient((v * LANES + lane) * 8, f[v]);
  } else {
    for (int c = lane * 8; c < a.classes; c += LANES * 8) { logits8(z, c, a.classes, f[0]); gradient(c, f[0]); }
  }
}

template <typename T, int LANES, int V>
void launch_rows(const Xent &x, hipStream_t st) {
  constexpr int kRows = LANES < 256 ? 256 / LANES : 1;
  k_rows<T, LANES, V><<<(unsigned)ceil_div(x.rows, kRows), LANES < 256 ? 256 : LANES, 0, st>>>(x);
}
template <typename T>
int rows(const Xent &x, hipStream_t st) {
  const int c = x.classes;
  if (c <= 16 * 8) launch_rows<T, 16, 1>(x, st);
  else if (c <= 64 * 8) launch_rows<T, 64, 1>(x, st);
  else if (c <= 64 * 32) launch_rows<T, 64, 4>(x, st);
  else if (c <= 256 * 32) launch_rows<T, 256, 4>(x, st);
  else if (c <= 1024 * 32) launch_rows<T, 1024, 4>(x, st);
  else launch_rows<T, 1024, 0>(x, st);
  return ops_launched("cross-entropy");
}

bool check(const cada_xent *a) {
  if (!a) { set_error("the arguments are NULL"); return false; }
  if (a->rows < 0 || a->rows > (int64_t)1 << 30) { set_error("rows must be in [0, 2^30] (got %lld)", (long long)a->rows); return false; }
  return true;
}

size_t workspace(const cada_xent *a) { return kOpsAlign + (a->mean && !a->loss ? ops_align((size_t)a->rows * 4) : 0); }

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
  if (a->classes < 1 || a->classes > 0x7fffffff - (1 << 20)) { set_error("classes must be in [1, 2^31 - 2^20) (got %lld)", (long long)a->classes); return CADA_EINVAL; }
  if (a->type != CADA_F32 && a->type != CADA_BF16) { set_error("type must be CADA_F32 or CADA_BF16 (got %d)", a->type); return CADA_EINVAL; }
  if (a->label_bytes != 4 && a->label_bytes != 8) { set_error("label_bytes must be 4 or 8 (got %d)", a->label_bytes); return CADA_EINVAL; }
  if (!(a->smoothing >= 0.0 && a->smoothing < 1.0)) { set_error("smoothing must be in [0, 1)"); return CADA_EINVAL; }
  if (a->rows > 0) {
    if (!a->logits || !a->labels) { set_error("logits and labels must be device pointers"); return CADA_EINVAL; }
    if (a->ldz < a->classes || (a->grad && a->ldg < a->classes)) { set_error("the row length of logits or grad is less than the %lld classes", (long long)a->classes); return CADA_EINVAL; }
    if (a->grad == a->logits && a->ldg != a->ldz) { set_error("grad in the place of logits must have their row length"); return CADA_EINVAL; }
    if (reinterpret_cast<uintptr_t>(a->logits) % type_bytes(a->type) != 0 || reinterpret_cast<uintptr_t>(a->grad) % type_bytes(a->type) != 0 ||
        reinterpret_cast<uintptr_t>(a->labels) % a->label_bytes != 0) { set_error("logits, grad or labels are not aligned to their elements"); return CADA_EINVAL; }
  }
  if (int rc = ops_check_workspace(a->workspace, a->workspace_bytes, workspace(a))) return rc;
  hipStream_t st = static_cast<hipStream_t>(a->stream);
  int64_t *count = static_cast<int64_t *>(a->workspace);
  Xent x{};
  x.logits = a->logits; x.labels = a->labels; x.grad = a->grad;
  x.loss = a->loss ? a->loss : a->mean ? reinterpret_cast<float *>(static_cast<char *>(a->workspace) + kOpsAlign) : nullptr;
  x.count = count; x.rows = a->rows; x.ldz = a->ldz; x.ldg = a->ldg; x.ignore = a->ignore_index;
  x.classes = (int32_t)a->classes; x.label_bytes = a->label_bytes;
  x.smoothing = (float)a->smoothing; x.keep = (float)(1.0 - a->smoothing); x.scale = (float)a->scale;
  k_count<<<1, 1024, 0, st>>>(a->labels, a->label_bytes, a->rows, a->ignore_index, count);
  if (int rc = ops_launched("cross-entropy count")) return rc;
  if (a->rows > 0) if (int rc = a->type == CADA_BF16 ? rows<bf16>(x, st) : rows<float>(x, st)) return rc;
  if (a->mean) {
    k_mean<<<1, 1024, 0, st>>>(x.loss, a->rows, count, a->mean);
    return ops_launched("cross-entropy mean");
  }
  return CADA_OK;
}

}  // extern "C"
