// The AdamW step over many tensors in one launch, moments in 32 or in 8 bits (cada_ops.h).
//
// The plan in the caller's workspace is a table of tensors and a table that says which tensor each chunk of kChunk elements
// belongs to; a workgroup takes one chunk, eight consecutive elements per thread, so that 32 lanes hold one block of moments.
// Bound by memory: every element is read and written once.  Each operation is rounded by itself (no contraction), as the header says, so that
// codes do not depend on how a compiler joins operations.
#include <cmath>
#include <exception>
#include <new>
#include <vector>

#include "cada_ops_internal.h"

namespace cada {
namespace {

constexpr int kChunk = 2048, kNormBlocks = 512;
constexpr float kMomentMax = 127.f * 127.f, kRootMax = 255.f * 255.f, kScaleMin = 1e-30f;

struct Tensor {
  void *param;
  const void *grad;
  uint16_t *copy;
  int64_t n, moments;        // elements; where its moments start
  double decay;
  int32_t types;             // bit 0: param is bf16, bit 1: grad is bf16
};
struct ChunkAt { int32_t tensor, index; };

struct Step {
  const Tensor *tensors;
  const ChunkAt *chunks;
  void *m, *v;
  float *m_scale, *v_scale;
  const float *grad_scale;   // or null
  const double *norm_part;   // [kNormBlocks], or null (no clipping)
  float *norm;
  double lr;
  float beta1, beta2, omb1, omb2, eps, step_size, root, max_norm;
};

static_assert(kNormBlocks == 512, "a step's workgroup adds them up, two per thread");

template <typename T> __device__ __forceinline__ void load8_as(const void *p, int64_t at, int64_t left, float (&f)[8]) { load8_n(static_cast<const T *>(p) + at, left, f); }

// Sum of the squares of all gradients, in double: one part per workgroup, in a fixed order.  Each quarter of a workgroup takes a chunk at a time.  Its wavefronts look 64 chunks
// up at once, one per lane, and then have nothing to wait for but the data, four chunks of which are on their way together (with a chunk's place in the table, its tensor
// and its data asked for one after the other: 59M bf16 gradients 57 us, now 38; a plain read of them takes as long).
__global__ __launch_bounds__(1024) void k_norm(const Tensor *tensors, const ChunkAt *chunks, int64_t n_chunks, double *part) {
  __shared__ double red[16];
  constexpr int U = 4;
  double s = 0.0;
  const int lane = threadIdx.x & 63;
  const int64_t stride = (int64_t)gridDim.x * 4, e = (threadIdx.x & 255) * 8;
  for (int64_t c = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 8); c < n_chunks; c += 64 * stride) {
    const ChunkAt at = chunks[min(c + lane * stride, n_chunks - 1)];
    const Tensor *t = tensors + at.tensor;
    const int types = t->types;
    const int64_t first = (int64_t)at.index * kChunk, size = t->n - first;      // elements from the chunk's first to the tensor's end
    const uint64_t grad = reinterpret_cast<uint64_t>(t->grad) + first * (types & 2 ? 2 : 4);
    const int here = (int)min((int64_t)64, (n_chunks - c + stride - 1) / stride);
    for (int i = 0; i < here; i += U) {
      u32x4v raw[U][2];
      bool half[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int l = min(i + u, here - 1);
        const uint64_t p = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(grad >> 32), l) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)grad, l);
        const int64_t left = i + u < here ? (int64_t)__builtin_amdgcn_readlane((int)min(size, (int64_t)kChunk), l) - e : 0;
        half[u] = __builtin_amdgcn_readlane(types, l) & 2;
        raw[u][1] = u32x4v{0, 0, 0, 0};
        if (half[u]) {
          raw[u][0] = load16_n(reinterpret_cast<const bf16 *>(p) + e, left);
        } else {
          raw[u][0] = load16_n(reinterpret_cast<const float *>(p) + e, left);
          raw[u][1] = load16_n(reinterpret_cast<const float *>(p) + e + 4, left - 4);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float f[8];
        if (half[u]) {
          unpack<bf16>(raw[u][0], f);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) { f[j] = __uint_as_float(raw[u][0][j]); f[4 + j] = __uint_as_float(raw[u][1][j]); }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) s = fma((double)f[j], (double)f[j], s);
      }
    }
  }
  s = wave_sum_f64(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0;
    for (int i = 0; i < 16; ++i) s += red[i];
    part[blockIdx.x] = s;
  }
}

// Largest bit pattern of non-negative values over the 32 lanes of a half wavefront (NaN above infinity above all others, so that neither is lost).
__device__ __forceinline__ float half_max(float x) {
  uint32_t u = __float_as_uint(x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) u = max(u, (uint32_t)__shfl_xor((int)u, o, 64));
  return __uint_as_float(u);
}

__device__ __forceinline__ float finite_or_nan(float x) { return x < __builtin_inff() ? x : __builtin_nanf(""); }

template <int BITS>
__global__ __launch_bounds__(256) void k_adamw(const Step a) {
#pragma clang fp contract(off)
  __shared__ double red[4];
  const ChunkAt at = a.chunks[blockIdx.x];
  const Tensor t = a.tensors[at.tensor];
  const int64_t e = (int64_t)at.index * kChunk + threadIdx.x * 8, left = t.n - e;
  float factor = a.grad_scale ? *a.grad_scale : 1.f;
  float g[8], p[8], m[8], v[8], r[8];
  if (t.types & 2) load8_as<bf16>(t.grad, e, left, g); else load8_as<float>(t.grad, e, left, g);
  if (t.types & 1) load8_as<bf16>(t.param, e, left, p); else load8_as<float>(t.param, e, left, p);
  const int64_t me = t.moments + e;
  // (the moments' part of a tensor is filled up to whole blocks, not to whole chunks)
  const bool in = e < (t.n + CADA_MOMENT_BLOCK - 1) / CADA_MOMENT_BLOCK * CADA_MOMENT_BLOCK;
  if (in) {
    if constexpr (BITS == 32) {
      const v4s *pm = reinterpret_cast<const v4s *>(static_cast<float *>(a.m) + me), *pv = reinterpret_cast<const v4s *>(static_cast<float *>(a.v) + me);
      const v4s m0 = pm[0], m1 = pm[1], v0 = pv[0], v1 = pv[1];
#pragma unroll
      for (int i = 0; i < 4; ++i) { m[i] = m0[i]; m[4 + i] = m1[i]; v[i] = v0[i]; v[4 + i] = v1[i]; }
    } else {
      const uint64_t qm = *reinterpret_cast<const uint64_t *>(static_cast<int8_t *>(a.m) + me), qv = *reinterpret_cast<const uint64_t *>(static_cast<uint8_t *>(a.v) + me);
      const float sm = a.m_scale[me / CADA_MOMENT_BLOCK] * (1.f / kMomentMax), sv = a.v_scale[me / CADA_MOMENT_BLOCK] * (1.f / kRootMax);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float q = (float)(int8_t)(qm >> (8 * i)), c = (float)(uint8_t)(qv >> (8 * i));
        m[i] = (q * fabsf(q)) * sm;
        const float root = (c * c) * sv;
        v[i] = root * root;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) m[i] = v[i] = 0.f;
  }
  if (a.norm_part) {
    double s = wave_sum_f64(a.norm_part[threadIdx.x] + a.norm_part[256 + threadIdx.x]);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    s = (red[0] + red[1]) + (red[2] + red[3]);
    const float norm = (float)(sqrt(s) * fabs((double)factor));
    const float ratio = a.max_norm / norm;
    factor *= ratio > 1.f ? 1.f : ratio;      // (NaN stays)
    if (a.norm && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = norm;
  }
  const float decay = (float)(a.lr * t.decay);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float gf = g[i] * factor;
    m[i] = m[i] * a.beta1 + gf * a.omb1;
    v[i] = v[i] * a.beta2 + (gf * a.omb2) * gf;
    r[i] = sqrtf(v[i]);
    p[i] = (p[i] - p[i] * decay) - (m[i] * a.step_size) / (r[i] * a.root + a.eps);
  }
  if (left < 8) {        // (the fill's gradients are zero, but a factor that is not finite would make them NaN)
#pragma unroll
    for (int i = 0; i < 8; ++i) if (i >= left) m[i] = v[i] = r[i] = 0.f;
  }
  if (t.types & 1) store8_n(static_cast<bf16 *>(t.param) + e, left, p); else store8_n(static_cast<float *>(t.param) + e, left, p);
  if (t.copy) store8_n(reinterpret_cast<bf16 *>(t.copy) + e, left, p);
  if constexpr (BITS == 32) {
    if (in) {
      v4s *pm = reinterpret_cast<v4s *>(static_cast<float *>(a.m) + me), *pv = reinterpret_cast<v4s *>(static_cast<float *>(a.v) + me);
      pm[0] = v4s{m[0], m[1], m[2], m[3]}; pm[1] = v4s{m[4], m[5], m[6], m[7]};
      pv[0] = v4s{v[0], v[1], v[2], v[3]}; pv[1] = v4s{v[4], v[5], v[6], v[7]};
    }
  } else {
    float sm = 0.f, sv = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      sm = __uint_as_float(max(__float_as_uint(sm), __float_as_uint(fabsf(m[i]))));
      sv = __uint_as_float(max(__float_as_uint(sv), __float_as_uint(fabsf(r[i]))));
    }
    // (a block with an infinity becomes NaN: codes of infinity are zero or infinite, and sqrt(v) would go on dividing by it)
    sm = finite_or_nan(half_max(sm));
    sv = finite_or_nan(half_max(sv));
    const float im = sm >= kScaleMin ? kMomentMax / sm : 0.f, iv = sv >= kScaleMin ? kRootMax / sv : 0.f;
    uint64_t qm = 0, qv = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int q = (int)fminf(rintf(sqrtf(fabsf(m[i]) * im)), 127.f);
      int c = (int)fminf(rintf(sqrtf(r[i] * iv)), 255.f);
      if (r[i] > 0.f) c = max(c, 1);
      qm |= (uint64_t)(uint8_t)(int8_t)(m[i] < 0.f ? -q : q) << (8 * i);
      qv |= (uint64_t)(uint8_t)c << (8 * i);
    }
    if (in) {
      *reinterpret_cast<uint64_t *>(static_cast<int8_t *>(a.m) + me) = qm;
      *reinterpret_cast<uint64_t *>(static_cast<uint8_t *>(a.v) + me) = qv;
      if ((threadIdx.x & 31) == 0) {
        a.m_scale[me / CADA_MOMENT_BLOCK] = sm;
        a.v_scale[me / CADA_MOMENT_BLOCK] = sv;
      }
    }
  }
}

// The moments as values; eight elements per thread.
template <int BITS>
__global__ __launch_bounds__(256) void k_moments(const void *m, const void *v, const float *m_scale, const float *v_scale, float *m_out, float *v_out, int64_t n) {
#pragma clang fp contract(off)
  const int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (e >= n) return;
  if constexpr (BITS == 8) {
    const uint64_t qm = *reinterpret_cast<const uint64_t *>(static_cast<const int8_t *>(m) + e), qv = *reinterpret_cast<const uint64_t *>(static_cast<const uint8_t *>(v) + e);
    const float sm = m_scale[e / CADA_MOMENT_BLOCK] * (1.f / kMomentMax), sv = v_scale[e / CADA_MOMENT_BLOCK] * (1.f / kRootMax);
    float fm[8], fv[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float q = (float)(int8_t)(qm >> (8 * i)), c = (float)(uint8_t)(qv >> (8 * i));
      fm[i] = (q * fabsf(q)) * sm;
      const float root = (c * c) * sv;
      fv[i] = root * root;
    }
    if (m_out) store8_n(m_out + e, 8, fm);
    if (v_out) store8_n(v_out + e, 8, fv);
  } else {
    float f[8];
    if (m_out) { load8_n(static_cast<const float *>(m) + e, 8, f); store8_n(m_out + e, 8, f); }
    if (v_out) { load8_n(static_cast<const float *>(v) + e, 8, f); store8_n(v_out + e, 8, f); }
  }
}

struct Plan {
  Step step;
  hipStream_t stream;
  double beta1, beta2;
  int64_t n_chunks, elements;
  double *norm_part;
  int bits;
  std::vector<char> host;      // the tables, as copied to the workspace
};

// Elements of the moments, chunks; false and an error text if the sizes are invalid.
bool sizes(const cada_adamw_config *cfg, int64_t *elements, int64_t *chunks) {
  if (!cfg) { set_error("cfg is NULL"); return false; }
  if (!cfg->tensors || cfg->n_tensors < 1 || cfg->n_tensors > 1 << 20) { set_error("there must be 1 to 2^20 tensors (got %d)", cfg->n_tensors); return false; }
  int64_t e = 0, c = 0;
  for (int i = 0; i < cfg->n_tensors; ++i) {
    const int64_t n = cfg->tensors[i].n;
    if (n < 0 || n > (int64_t)1 << 34) { set_error("tensor %d: n must be in [0, 2^34] (got %lld)", i, (long long)n); return false; }
    e += ceil_div(n, CADA_MOMENT_BLOCK) * CADA_MOMENT_BLOCK;
    c += ceil_div(n, kChunk);
    if (c > (int64_t)1 << 23) { set_error("more than 2^34 elements in all"); return false; }
  }
  *elements = e;
  *chunks = c;
  return true;
}
struct Layout { size_t tensors, chunks, norm, bytes; };
Layout layout(int32_t n_tensors, int64_t chunks) {
  Layout l;
  l.tensors = 0;
  l.chunks = ops_align((size_t)n_tensors * sizeof(Tensor));
  l.norm = l.chunks + ops_align((size_t)chunks * sizeof(ChunkAt));
  l.bytes = l.norm + ops_align(kNormBlocks * sizeof(double));
  return l;
}
int check_config(const cada_adamw_config *cfg, int64_t *elements, int64_t *chunks) {
  if (!sizes(cfg, elements, chunks)) return CADA_EINVAL;
  if (cfg->moment_bits != CADA_MOMENTS_32 && cfg->moment_bits != CADA_MOMENTS_8) { set_error("moment_bits must be one of CADA_MOMENTS_* (got %d)", cfg->moment_bits); return CADA_EINVAL; }
  if (!(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0 && cfg->beta2 >= 0.0 && cfg->beta2 < 1.0)) { set_error("beta1, beta2 must be in [0, 1)"); return CADA_EINVAL; }
  if (!(cfg->eps >= 0.0)) { set_error("eps must be >= 0"); return CADA_EINVAL; }
  if (!(cfg->max_norm >= 0.0)) { set_error("max_norm must be >= 0"); return CADA_EINVAL; }
  for (int i = 0; i < cfg->n_tensors; ++i) {
    const cada_adamw_tensor &t = cfg->tensors[i];
    if ((t.param_type != CADA_F32 && t.param_type != CADA_BF16) || (t.grad_type != CADA_F32 && t.grad_type != CADA_BF16)) { set_error("tensor %d: types must be CADA_F32 or CADA_BF16", i); return CADA_EINVAL; }
    if (t.n > 0 && (!t.param || !t.grad)) { set_error("tensor %d: param and grad must be device pointers", i); return CADA_EINVAL; }
    if (reinterpret_cast<uintptr_t>(t.param) % type_bytes(t.param_type) != 0 || reinterpret_cast<uintptr_t>(t.grad) % type_bytes(t.grad_type) != 0 ||
        reinterpret_cast<uintptr_t>(t.copy) % 2 != 0) { set_error("tensor %d: param, grad or copy is not aligned to its elements", i); return CADA_EINVAL; }
    if (!(std::isfinite(t.weight_decay))) { set_error("tensor %d: weight_decay must be finite", i); return CADA_EINVAL; }
  }
  if (*elements > 0) {
    if (!cfg->m || !cfg->v) { set_error("m and v must be device pointers"); return CADA_EINVAL; }
    if (reinterpret_cast<uintptr_t>(cfg->m) % 16 != 0 || reinterpret_cast<uintptr_t>(cfg->v) % 16 != 0) { set_error("m and v must be 16-byte aligned"); return CADA_EINVAL; }
    if (cfg->moment_bits == CADA_MOMENTS_8 && (!cfg->m_scale || !cfg->v_scale)) { set_error("8-bit moments need m_scale and v_scale"); return CADA_EINVAL; }
  }
  return CADA_OK;
}

// Whether parameters, copies, moments, norm and workspace, which a step writes, share memory with nothing: workgroups meet them in no order.
bool apart(const cada_adamw_config *cfg, int64_t elements, size_t workspace_bytes) {
  std::vector<Range> r;
  r.reserve((size_t)cfg->n_tensors * 3 + 6);
  for (int i = 0; i < cfg->n_tensors; ++i) {
    const cada_adamw_tensor &t = cfg->tensors[i];
    r.push_back(Range{"param", i, t.param, (size_t)t.n * type_bytes(t.param_type), true});
    r.push_back(Range{"grad", i, t.grad, (size_t)t.n * type_bytes(t.grad_type), false});
    r.push_back(Range{"copy", i, t.copy, (size_t)t.n * 2, true});
  }
  const bool eight = cfg->moment_bits == CADA_MOMENTS_8;
  const size_t size = (size_t)elements * (eight ? 1 : 4), scales = eight ? (size_t)elements / CADA_MOMENT_BLOCK * 4 : 0;
  r.push_back(Range{"m", -1, cfg->m, size, true});
  r.push_back(Range{"v", -1, cfg->v, size, true});
  r.push_back(Range{"m_scale", -1, cfg->m_scale, scales, true});
  r.push_back(Range{"v_scale", -1, cfg->v_scale, scales, true});
  r.push_back(Range{"norm", -1, cfg->norm, cfg->max_norm > 0.0 ? sizeof(float) : 0, true});
  r.push_back(Range{"workspace", -1, cfg->workspace, workspace_bytes, true});
  return ops_apart(r.data(), r.size());
}

}  // namespace
}  // namespace cada

using namespace cada;

struct cada_adamw { cada::Plan p; };

extern "C" {

int64_t cada_adamw_moment_elements(const cada_adamw_config *cfg) {
  int64_t e, c;
  return sizes(cfg, &e, &c) ? e : -1;
}

int cada_adamw_workspace(cada_adamw_config *cfg) {
  int64_t e, c;
  if (!sizes(cfg, &e, &c)) return CADA_EINVAL;
  cfg->workspace_bytes = layout(cfg->n_tensors, c).bytes;
  return CADA_OK;
}

int cada_adamw_init(const cada_adamw_config *cfg, cada_adamw **out) {
  if (!out) { set_error("out is NULL"); return CADA_EINVAL; }
  *out = nullptr;
  int64_t elements, chunks;
  if (int rc = check_config(cfg, &elements, &chunks)) return rc;
  const Layout l = layout(cfg->n_tensors, chunks);
  if (int rc = ops_check_workspace(cfg->workspace, cfg->workspace_bytes, l.bytes)) return rc;
  cada_adamw *h = nullptr;
  try {
    if (!apart(cfg, elements, l.bytes)) return CADA_EINVAL;
    h = new cada_adamw();
    Plan &p = h->p;
    p.host.resize(l.norm);
    Tensor *t = reinterpret_cast<Tensor *>(p.host.data());
    ChunkAt *c = reinterpret_cast<ChunkAt *>(p.host.data() + l.chunks);
    int64_t moments = 0;
    for (int i = 0; i < cfg->n_tensors; ++i) {
      const cada_adamw_tensor &x = cfg->tensors[i];
      t[i] = Tensor{x.param, x.grad, static_cast<uint16_t *>(x.copy), x.n, moments, x.weight_decay, (x.param_type == CADA_BF16 ? 1 : 0) | (x.grad_type == CADA_BF16 ? 2 : 0)};
      moments += ceil_div(x.n, CADA_MOMENT_BLOCK) * CADA_MOMENT_BLOCK;
      for (int64_t k = 0; k < ceil_div(x.n, kChunk); ++k) *c++ = ChunkAt{i, (int32_t)k};
    }
    p.stream = static_cast<hipStream_t>(cfg->stream);
    p.beta1 = cfg->beta1; p.beta2 = cfg->beta2;
    p.n_chunks = chunks; p.elements = elements; p.bits = cfg->moment_bits;
    char *ws = static_cast<char *>(cfg->workspace);
    p.norm_part = reinterpret_cast<double *>(ws + l.norm);
    Step &s = p.step;
    s = Step{};
    s.tensors = reinterpret_cast<const Tensor *>(ws); s.chunks = reinterpret_cast<const ChunkAt *>(ws + l.chunks);
    s.m = cfg->m; s.v = cfg->v; s.m_scale = cfg->m_scale; s.v_scale = cfg->v_scale;
    s.norm_part = cfg->max_norm > 0.0 ? p.norm_part : nullptr; s.norm = cfg->norm; s.max_norm = (float)cfg->max_norm;
    s.beta1 = (float)cfg->beta1; s.beta2 = (float)cfg->beta2; s.omb1 = (float)(1.0 - cfg->beta1); s.omb2 = (float)(1.0 - cfg->beta2); s.eps = (float)cfg->eps;
    const hipError_t e = hipMemcpyAsync(ws, p.host.data(), p.host.size(), hipMemcpyHostToDevice, p.stream);
    if (e != hipSuccess) { set_error("hipMemcpyAsync: %s", hipGetErrorString(e)); delete h; return CADA_EHIP; }
  } catch (const std::exception &) {      // (memory, or a size that no vector has)
    delete h;
    set_error("out of host memory");
    return CADA_EINVAL;
  }
  *out = h;
  return CADA_OK;
}

int cada_adamw_step(cada_adamw *plan, int64_t t, double lr, const float *grad_scale) {
  if (!plan) { set_error("plan is NULL"); return CADA_EINVAL; }
  if (t < 1) { set_error("t must be >= 1 (got %lld)", (long long)t); return CADA_EINVAL; }
  if (!std::isfinite(lr)) { set_error("lr must be finite"); return CADA_EINVAL; }
  Plan &p = plan->p;
  if (p.n_chunks == 0) return CADA_OK;
  Step s = p.step;
  s.grad_scale = grad_scale;
  s.lr = lr;
  s.step_size = (float)(lr / (1.0 - std::pow(p.beta1, (double)t)));
  s.root = (float)(1.0 / std::sqrt(1.0 - std::pow(p.beta2, (double)t)));
  if (s.norm_part) {
    k_norm<<<kNormBlocks, 1024, 0, p.stream>>>(s.tensors, s.chunks, p.n_chunks, p.norm_part);
    if (int rc = ops_launched("adamw norm")) return rc;
  }
  if (p.bits == 32) k_adamw<32><<<(unsigned)p.n_chunks, 256, 0, p.stream>>>(s);
  else k_adamw<8><<<(unsigned)p.n_chunks, 256, 0, p.stream>>>(s);
  return ops_launched("adamw");
}

int cada_adamw_moments(cada_adamw *plan, float *m, float *v) {
  if (!plan) { set_error("plan is NULL"); return CADA_EINVAL; }
  const Plan &p = plan->p;
  if (p.elements == 0 || (!m && !v)) return CADA_OK;
  const size_t values = (size_t)p.elements * sizeof(float), held = p.bits == 32 ? values : (size_t)p.elements, scales = p.bits == 32 ? 0 : values / CADA_MOMENT_BLOCK;
  Range r[] = {{"the values of m", -1, m, values, true}, {"the values of v", -1, v, values, true}, {"m", -1, p.step.m, held, false}, {"v", -1, p.step.v, held, false},
               {"m_scale", -1, p.step.m_scale, scales, false}, {"v_scale", -1, p.step.v_scale, scales, false}, {"workspace", -1, p.step.tensors, p.host.size(), false}};
  if (!ops_apart(r, sizeof(r) / sizeof(r[0]))) return CADA_EINVAL;
  const unsigned grid = (unsigned)ceil_div(p.elements, 2048);
  if (p.bits == 32) k_moments<32><<<grid, 256, 0, p.stream>>>(p.step.m, p.step.v, nullptr, nullptr, m, v, p.elements);
  else k_moments<8><<<grid, 256, 0, p.stream>>>(p.step.m, p.step.v, p.step.m_scale, p.step.v_scale, m, v, p.elements);
  return ops_launched("adamw moments");
}

void cada_adamw_destroy(cada_adamw *plan) { delete plan; }

}  // extern "C"
