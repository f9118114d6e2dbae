// Global norm of all gradients, their clipping and the AdamW step, over a list of tensors in one launch each.
//
//   norm = sqrt(sum over all tensors of g^2),  s = min(1, max_norm / (norm + 1e-6))
//   clip:   out = s g
//   AdamW:  m' = b1 m + (1 - b1) s g,  v' = b2 v + (1 - b2) (s g)^2,
//           p' = p (1 - lr decay) - lr m' / (1 - b1^t) / (sqrt(v' / (1 - b2^t)) + eps)
//
// A tensor list is laid out once in the caller's memory: all tensors cut into chunks of at most kChunk elements, 64 bytes of
// addresses each, so that a launch walks over chunks whatever the number and the sizes of the tensors.  All three calls are
// bound by memory.
#include "common.h"
#include "bf16_mfma.h"
#include <math.h>

namespace {

constexpr int kChunk = 4096;                 // elements per chunk
constexpr int kThreads = 256;
constexpr int kUnits = kChunk / (4 * kThreads);
constexpr int kMaxParts = 2048;              // workgroups of the norm, one partial sum each
constexpr int kRecords = 48;                 // tensors per launch of the layout kernel (its arguments hold them)
constexpr uint32_t kBuilt = 0x56445431u;

struct Chunk {
  void* grad;
  void* clip;
  float* param;
  float* m;
  float* v;
  bf16_t* weight;
  int count;
  float decay;
  int flags;
  int pad;
};
static_assert(sizeof(Chunk) == 64, "");
enum { kGradBf16 = 1, kClipBf16 = 2 };

// Head of the table: counters of finished workgroups (zero between launches), then the norm's partial sums, then the chunks.
struct Head {
  uint32_t norm_done, step_done;
  uint32_t pad[62];
  double part[kMaxParts];
};

struct Record {
  void *grad, *clip;
  float *param, *m, *v;
  bf16_t* weight;
  long long numel;
  int first, flags;
  float decay;
};
struct Records {
  Record r[kRecords];
};
static_assert(sizeof(Records) <= 3800, "kernel arguments");

__global__ __launch_bounds__(256) void list_kernel(Records a, Head* head, Chunk* chunks, int clear) {
  if (clear && blockIdx.x == 0 && threadIdx.x == 0) {
    head->norm_done = 0;
    head->step_done = 0;
  }
  const Record r = a.r[blockIdx.x];
  const long long n = (r.numel + kChunk - 1) / kChunk;
  for (long long i = threadIdx.x; i < n; i += blockDim.x) {
    const long long at = i * kChunk;
    Chunk c;
    c.grad = (char*)r.grad + at * (r.flags & kGradBf16 ? 2 : 4);
    c.clip = r.clip ? (char*)r.clip + at * (r.flags & kClipBf16 ? 2 : 4) : nullptr;
    c.param = r.param ? r.param + at : nullptr;
    c.m = r.m ? r.m + at : nullptr;
    c.v = r.v ? r.v + at : nullptr;
    c.weight = r.weight ? r.weight + at : nullptr;
    c.count = (int)min((long long)kChunk, r.numel - at);
    c.decay = r.decay;
    c.flags = r.flags;
    c.pad = 0;
    chunks[r.first + i] = c;
  }
}

// Four neighbouring elements; tensors need no more than element alignment.
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2u __attribute__((ext_vector_type(2), aligned(2)));
__device__ inline void load4(const float* p, int left, float (&v)[4]) {
  if (left >= 4) {
    const f32x4u t = *reinterpret_cast<const f32x4u*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = t[e];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = e < left ? p[e] : 0.f;
  }
}
__device__ inline void load4(const bf16_t* p, int left, float (&v)[4]) {
  if (left >= 4) {
    const u32x2u t = *reinterpret_cast<const u32x2u*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(e & 1 ? t[e >> 1] & 0xffff0000u : t[e >> 1] << 16);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = e < left ? bf2f(p[e]) : 0.f;
  }
}
__device__ inline void store4(float* p, int left, const float (&v)[4]) {
  if (left >= 4) {
    *reinterpret_cast<f32x4u*>(p) = f32x4u{v[0], v[1], v[2], v[3]};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) p[e] = v[e];
  }
}
__device__ inline void store4(bf16_t* p, int left, const float (&v)[4]) {
  if (left >= 4) {
    *reinterpret_cast<u32x2u*>(p) = u32x2u{pack2(v[0], v[1]), pack2(v[2], v[3])};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) p[e] = f2bf(v[e]);
  }
}
__device__ inline void load_grads(const Chunk& c, float (&g)[kUnits][4]) {
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const int at = (u * kThreads + threadIdx.x) * 4;
    if (c.flags & kGradBf16) load4((const bf16_t*)c.grad + at, c.count - at, g[u]);
    else load4((const float*)c.grad + at, c.count - at, g[u]);
  }
}

__device__ inline double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
// sum over the workgroup, the same in all of its threads
__device__ inline double block_sum(double v, double* red) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) v += red[w];
  __syncthreads();
  return v;
}

// Squares are formed and added in 64 bits: no gradient is too large or too small for its square, and the sum keeps every digit the
// result has.  The workgroup that finishes last adds the partial sums in their order, so the result does not depend on which it was.
__global__ __launch_bounds__(kThreads) void grad_norm_kernel(Head* head, const Chunk* __restrict__ chunks, int n, float* norm) {
  __shared__ double red[kThreads / 64];
  __shared__ bool last;
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const Chunk c = chunks[i];
    float g[kUnits][4];
    load_grads(c, g);
#pragma unroll
    for (int u = 0; u < kUnits; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const double x = (double)g[u][e];
        s[e] = fma(x, x, s[e]);
      }
  }
  const double mine = block_sum((s[0] + s[1]) + (s[2] + s[3]), red);
  if (threadIdx.x == 0) {
    __hip_atomic_store(&head->part[blockIdx.x], mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    last = __hip_atomic_fetch_add(&head->norm_done, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  double t = 0.0;
  for (int i = threadIdx.x; i < (int)gridDim.x; i += kThreads)
    t += __hip_atomic_load(&head->part[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  t = block_sum(t, red);
  if (threadIdx.x == 0) {
    *norm = (float)sqrt(t);
    __hip_atomic_store(&head->norm_done, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

// Factor of the gradients; false when the norm is not finite.
__device__ inline bool clip_factor(const float* norm, float max_norm, float& s) {
  s = 1.f;
  if (!norm) return true;
  const float v = *norm;
  if (!(v - v == 0.f)) return false;
  if (max_norm > 0.f) s = fminf(1.f, max_norm / (v + 1e-6f));
  return true;
}

__global__ __launch_bounds__(kThreads) void clip_kernel(const Chunk* __restrict__ chunks, int n, const float* norm, float max_norm, int32_t* status) {
  float s;
  if (!clip_factor(norm, max_norm, s)) {
    if (status && blockIdx.x == 0 && threadIdx.x == 0) *status = 1;
    return;
  }
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const Chunk c = chunks[i];
    void* out = c.clip ? c.clip : c.grad;
    if (out == c.grad && s == 1.f) continue;          // in place and short enough: nothing changes
    const bool bf16 = c.flags & (c.clip ? kClipBf16 : kGradBf16);
    float g[kUnits][4];
    load_grads(c, g);
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int at = (u * kThreads + threadIdx.x) * 4;
#pragma unroll
      for (int e = 0; e < 4; ++e) g[u][e] *= s;
      if (bf16) store4((bf16_t*)out + at, c.count - at, g[u]);
      else store4((float*)out + at, c.count - at, g[u]);
    }
  }
}

struct Adam {
  float lr, b1, c1, b2, c2, eps;       // c = 1 - b
  float rate, root;                    // lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
  double log_b1, log_b2;
  float max_norm;
  const float* norm;
  const float* lr_dev;
  int64_t* step_dev;
  int advance;
  int32_t* status;
};

__global__ __launch_bounds__(kThreads) void adamw_kernel(Head* head, const Chunk* __restrict__ chunks, int n, Adam a) {
  float s;
  if (!clip_factor(a.norm, a.max_norm, s)) {
    if (a.status && blockIdx.x == 0 && threadIdx.x == 0) *a.status = 1;
    return;
  }
  int64_t t = 0;
  if (a.step_dev) {                    // (the host has filled `rate` and `root` in otherwise)
    t = *a.step_dev + 1;
    a.lr = *a.lr_dev;
    a.rate = (float)((double)a.lr / -expm1((double)t * a.log_b1));
    a.root = (float)(1.0 / sqrt(-expm1((double)t * a.log_b2)));
  }
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const Chunk c = chunks[i];
    float g[kUnits][4], p[kUnits][4], m[kUnits][4], v[kUnits][4];
    load_grads(c, g);
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int at = (u * kThreads + threadIdx.x) * 4, left = c.count - at;
      load4(c.param + at, left, p[u]);
      load4(c.m + at, left, m[u]);
      load4(c.v + at, left, v[u]);
    }
    const float keep = 1.f - a.lr * c.decay;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int at = (u * kThreads + threadIdx.x) * 4, left = c.count - at;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = s * g[u][e];
        m[u][e] = fmaf(a.b1, m[u][e], a.c1 * x);
        v[u][e] = fmaf(a.b2, v[u][e], a.c2 * x * x);
        p[u][e] = fmaf(-a.rate, m[u][e] / fmaf(sqrtf(v[u][e]), a.root, a.eps), keep * p[u][e]);
      }
      store4(c.param + at, left, p[u]);
      store4(c.m + at, left, m[u]);
      store4(c.v + at, left, v[u]);
      if (c.weight) store4(c.weight + at, left, p[u]);
    }
  }
  if (a.step_dev && a.advance) {       // whoever finishes last: all others have read the counter
    __syncthreads();
    if (threadIdx.x == 0 &&
        __hip_atomic_fetch_add(&head->step_done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1) {
      *a.step_dev = t;
      __hip_atomic_store(&head->step_done, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
}

// ---------------------------------------------------------------- host side
Head* head_of(const vardrop_tensor_list* l) { return (Head*)l->table; }
Chunk* chunks_of(const vardrop_tensor_list* l) { return (Chunk*)((char*)l->table + sizeof(Head)); }
enum { kHasParams = 1 };

int check_list(const vardrop_ctx* ctx, const vardrop_tensor_list* l) {
  if (!ctx || !l || l->built != kBuilt || !l->table || l->chunks < 0) return VARDROP_EINVAL;
  return VARDROP_OK;
}

unsigned blocks_for(const vardrop_tensor_list* l, int most) { return (unsigned)(l->chunks < 1 ? 1 : l->chunks < most ? l->chunks : most); }

int adamw(vardrop_ctx* ctx, const vardrop_tensor_list* l, Adam a, double beta1, double beta2, double eps, int64_t step, void* stream) {
  const int rc = check_list(ctx, l);
  if (rc) return rc;
  if (l->tensors > 0 && !(l->has & kHasParams)) return VARDROP_EINVAL;
  if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps > 0.0) || !(eps - eps == 0.0)) return VARDROP_EINVAL;
  if (!(a.max_norm >= 0.f) || (a.max_norm > 0.f && !a.norm)) return VARDROP_EINVAL;
  a.b1 = (float)beta1;
  a.c1 = (float)(1.0 - beta1);
  a.b2 = (float)beta2;
  a.c2 = (float)(1.0 - beta2);
  a.eps = (float)eps;
  a.log_b1 = log(beta1);
  a.log_b2 = log(beta2);
  if (!a.step_dev) {
    a.rate = (float)((double)a.lr / -expm1((double)step * a.log_b1));
    a.root = (float)(1.0 / sqrt(-expm1((double)step * a.log_b2)));
  }
  hipStream_t s = (hipStream_t)stream;
  VdTimer timer(ctx, VARDROP_K_ADAMW, s);
  VD_KERNEL(ctx, adamw_kernel, dim3(blocks_for(l, 8 * ctx->num_cus)), dim3(kThreads), 0, s, head_of(l), chunks_of(l), l->chunks, a);
  VD_LAUNCH_CHECK(ctx);
  return VARDROP_OK;
}

}  // namespace

extern "C" size_t vardrop_tensor_list_bytes(int tensors, const int64_t* numel_host) {
  if (tensors < 0 || (tensors > 0 && !numel_host)) return 0;
  long long chunks = 0;
  for (int i = 0; i < tensors; ++i) {
    if (numel_host[i] < 0 || numel_host[i] > (1ll << 40)) return 0;
    chunks += (numel_host[i] + kChunk - 1) / kChunk;
  }
  if (chunks >= (1ll << 31)) return 0;
  return vd_align_up(sizeof(Head) + (size_t)chunks * sizeof(Chunk), 256);
}

extern "C" int vardrop_tensor_list_build(vardrop_ctx* ctx, int tensors, const int64_t* numel_host, void* const* grad_host,
                                         const int32_t* grad_dtype_host, void* const* clip_host, const int32_t* clip_dtype_host,
                                         float* const* param_host, float* const* m_host, float* const* v_host,
                                         void* const* weight_host, const float* decay_host, void* table, size_t table_bytes,
                                         vardrop_tensor_list* list_host, void* stream) {
  if (!ctx || tensors < 0 || !list_host || (tensors > 0 && (!numel_host || !grad_host))) return VARDROP_EINVAL;
  const bool params = param_host || m_host || v_host;
  if (params && !(param_host && m_host && v_host)) return VARDROP_EINVAL;
  if (!params && (weight_host || decay_host)) return VARDROP_EINVAL;
  const size_t need = vardrop_tensor_list_bytes(tensors, numel_host);
  if (need == 0) return VARDROP_EINVAL;
  auto known = [](const int32_t* t, int i) { return !t || t[i] == VARDROP_F32 || t[i] == VARDROP_BF16; };
  for (int i = 0; i < tensors; ++i) {
    if (!known(grad_dtype_host, i) || (clip_host && !known(clip_dtype_host, i))) return VARDROP_EINVAL;
    if (decay_host && !(decay_host[i] - decay_host[i] == 0.f)) return VARDROP_EINVAL;
    if (numel_host[i] == 0) continue;
    const size_t ga = grad_dtype_host && grad_dtype_host[i] == VARDROP_BF16 ? 2 : 4;
    const size_t ca = clip_dtype_host && clip_dtype_host[i] == VARDROP_BF16 ? 2 : 4;
    if (!grad_host[i] || !vd_aligned(grad_host[i], ga)) return VARDROP_EINVAL;
    if (clip_host && (!clip_host[i] || !vd_aligned(clip_host[i], ca))) return VARDROP_EINVAL;
    if (params && (!param_host[i] || !m_host[i] || !v_host[i] || !vd_aligned(param_host[i], 4) || !vd_aligned(m_host[i], 4) ||
                   !vd_aligned(v_host[i], 4)))
      return VARDROP_EINVAL;
    if (weight_host && !vd_aligned(weight_host[i], 2)) return VARDROP_EINVAL;
  }
  if (!table || !vd_aligned(table, 256) || table_bytes < need) return VARDROP_EWORKSPACE;
  vardrop_tensor_list l = {};
  l.table = table;
  l.table_bytes = table_bytes;
  l.tensors = tensors;
  l.has = params ? kHasParams : 0;
  l.built = kBuilt;
  hipStream_t s = (hipStream_t)stream;
  int done = 0;
  bool clear = true;
  while (done < tensors || clear) {
    Records a = {};
    int k = 0;
    for (; k < kRecords && done < tensors; ++done) {
      if (numel_host[done] == 0) continue;
      Record& r = a.r[k++];
      r.grad = grad_host[done];
      r.clip = clip_host ? clip_host[done] : nullptr;
      r.param = params ? param_host[done] : nullptr;
      r.m = params ? m_host[done] : nullptr;
      r.v = params ? v_host[done] : nullptr;
      r.weight = weight_host ? (bf16_t*)weight_host[done] : nullptr;
      r.numel = numel_host[done];
      r.first = l.chunks;
      r.decay = decay_host ? decay_host[done] : 0.f;
      r.flags = (grad_dtype_host && grad_dtype_host[done] == VARDROP_BF16 ? kGradBf16 : 0) |
                (clip_host && clip_dtype_host && clip_dtype_host[done] == VARDROP_BF16 ? kClipBf16 : 0);
      l.chunks += (int)((r.numel + kChunk - 1) / kChunk);
      l.numel += r.numel;
    }
    if (k == 0 && !clear) break;
    hipLaunchKernelGGL(list_kernel, dim3(k ? k : 1), dim3(256), 0, s, a, head_of(&l), chunks_of(&l), clear ? 1 : 0);
    VD_LAUNCH_CHECK(ctx);
    clear = false;
  }
  *list_host = l;
  return VARDROP_OK;
}

extern "C" int vardrop_grad_norm(vardrop_ctx* ctx, const vardrop_tensor_list* list, float* norm, void* stream) {
  const int rc = check_list(ctx, list);
  if (rc) return rc;
  if (!norm) return VARDROP_EINVAL;
  hipStream_t s = (hipStream_t)stream;
  VdTimer timer(ctx, VARDROP_K_GRAD_NORM, s);
  VD_KERNEL(ctx, grad_norm_kernel, dim3(blocks_for(list, kMaxParts)), dim3(kThreads), 0, s, head_of(list), chunks_of(list),
            list->chunks, norm);
  VD_LAUNCH_CHECK(ctx);
  return VARDROP_OK;
}

extern "C" int vardrop_clip_grads(vardrop_ctx* ctx, const vardrop_tensor_list* list, const float* norm, float max_norm,
                                  int32_t* status, void* stream) {
  const int rc = check_list(ctx, list);
  if (rc) return rc;
  if (!norm || !(max_norm > 0.f)) return VARDROP_EINVAL;
  if (list->chunks == 0) return VARDROP_OK;
  hipStream_t s = (hipStream_t)stream;
  VdTimer timer(ctx, VARDROP_K_CLIP, s);
  VD_KERNEL(ctx, clip_kernel, dim3(blocks_for(list, 8 * ctx->num_cus)), dim3(kThreads), 0, s, chunks_of(list), list->chunks, norm,
            max_norm, status);
  VD_LAUNCH_CHECK(ctx);
  return VARDROP_OK;
}

extern "C" int vardrop_adamw(vardrop_ctx* ctx, const vardrop_tensor_list* list, double lr, double beta1, double beta2, double eps,
                             int64_t step, const float* norm, float max_norm, int32_t* status, void* stream) {
  if (step < 1 || !(lr >= 0.0) || !(lr - lr == 0.0)) return VARDROP_EINVAL;
  Adam a = {};
  a.lr = (float)lr;
  a.max_norm = max_norm;
  a.norm = norm;
  a.status = status;
  return adamw(ctx, list, a, beta1, beta2, eps, step, stream);
}

extern "C" int vardrop_adamw_dev(vardrop_ctx* ctx, const vardrop_tensor_list* list, const float* lr_dev, double beta1, double beta2,
                                 double eps, int64_t* step_dev, int advance, const float* norm, float max_norm, int32_t* status,
                                 void* stream) {
  if (!lr_dev || !step_dev || !vd_aligned(step_dev, 8)) return VARDROP_EINVAL;
  Adam a = {};
  a.lr_dev = lr_dev;
  a.step_dev = step_dev;
  a.advance = advance ? 1 : 0;
  a.max_norm = max_norm;
  a.norm = norm;
  a.status = status;
  return adamw(ctx, list, a, beta1, beta2, eps, 0, stream);
}
