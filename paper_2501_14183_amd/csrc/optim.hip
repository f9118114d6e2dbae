// Global norm of all gradients, their clipping and the AdamW step, over a list of tensors in one launch each.
//
//   norm = sqrt(sum over all tensors of g^2),  s = min(1, max_norm / (norm + 1e-6))
//   clip:   out = s g
//   AdamW:  m' = b1 m + (1 - b1) s g,  v' = b2 v + (1 - b2) (s g)^2,
//           p' = p (1 - lr decay) - lr m' / (1 - b1^t) / (sqrt(v' / (1 - b2^t)) + eps)
//
// A tensor list is laid out once in the caller's memory: all tensors cut into chunks, 64 bytes of
// addresses each, so that a launch walks over chunks whatever the number and the sizes of the tensors.  All three calls are
// bound by memory.
#include "common.h"
#include "bf16_mfma.h"
#include <math.h>

namespace {

constexpr int kThreads = 256;                // of the norm and of clipping
constexpr int kAdamThreads = 512;            // 57 million weights 242 us, with 256 threads of sixteen elements each 250; 1.1 million 10.4, 9.8
constexpr int kMaxParts = 2048;              // workgroups of the norm, one partial sum each
constexpr int kRecords = 48;                 // tensors per launch of the layout kernel (its arguments hold them)
constexpr uint32_t kBuilt = 0x56445431u;

constexpr int kChunk = 4096;                 // elements of a chunk

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

// Counters of finished workgroups, zero between launches.  Increments of one address follow each other at about 12 ns, so
// workgroups share a counter in groups and the last of a group counts for all at the top (a line of memory each).
constexpr int kGroups = 64, kGroupLeast = 32;
struct Tickets {
  uint32_t group[kGroups][32];
  uint32_t top[32];
};
// Head of the table; the chunks follow.
struct Head {
  Tickets norm, step;
  uint64_t part[kMaxParts];          // of doubles
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
  if (clear && blockIdx.x == 0)
    for (int i = threadIdx.x; i < (int)(2 * sizeof(Tickets) / 4); i += blockDim.x) ((uint32_t*)head)[i] = 0;
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

// Four neighbouring elements of a tensor; tensors need no more than element alignment.  (The addresses come from the table: the
// address space has to be named, or the compiler takes them for addresses that may be LDS.)
template <typename T> using gptr = __attribute__((address_space(1))) T*;
template <typename T> struct Four;
template <> struct Four<float> {
  typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
  __device__ static float get(const vec& t, int e) { return t[e]; }
  __device__ static vec put(const float (&v)[4]) { return vec{v[0], v[1], v[2], v[3]}; }
  __device__ static float one(float t) { return t; }
  __device__ static float round(float t) { return t; }
};
template <> struct Four<bf16_t> {
  typedef uint32_t vec __attribute__((ext_vector_type(2), aligned(2)));
  __device__ static float get(const vec& t, int e) { return __uint_as_float(e & 1 ? t[e >> 1] & 0xffff0000u : t[e >> 1] << 16); }
  __device__ static vec put(const float (&v)[4]) { return vec{pack2(v[0], v[1]), pack2(v[2], v[3])}; }
  __device__ static float one(bf16_t t) { return bf2f(t); }
  __device__ static bf16_t round(float t) { return f2bf(t); }
};
// kOnce: data that no kernel reads again soon, not kept in the caches.
template <typename T, bool kOnce = false> __device__ inline typename Four<T>::vec load4(const void* p, int at) {
  const auto q = (gptr<const typename Four<T>::vec>)((gptr<const T>)(const T*)p + at);
  return kOnce ? __builtin_nontemporal_load(q) : *q;
}
template <typename T, bool kOnce = false> __device__ inline void store4(void* p, int at, const float (&v)[4]) {
  const auto q = (gptr<typename Four<T>::vec>)((gptr<T>)(T*)p + at);
  if (kOnce) __builtin_nontemporal_store(Four<T>::put(v), q);
  else *q = Four<T>::put(v);
}
template <typename T> __device__ inline float load1(const void* p, int at) { return Four<T>::one(((gptr<const T>)(const T*)p)[at]); }
template <typename T> __device__ inline void store1(void* p, int at, float v) { ((gptr<T>)(T*)p)[at] = Four<T>::round(v); }

// A chunk of `count` elements among T threads: thread t has the fours at 4 (u T + t), u < kChunk / (4 T), as far as they are
// whole ones, and the first three threads one each of the elements behind the last whole four.
template <int T> struct Places {
  int count;
  __device__ explicit Places(int n) : count(n) {}
  __device__ int at(int u) const { return (u * T + threadIdx.x) * 4; }
  __device__ bool whole(int u) const { return at(u) + 4 <= count; }
  __device__ int rest() const { return (count & ~3) + threadIdx.x; }
  __device__ bool has_rest() const { return rest() < count; }
};

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

// True in the one workgroup of the grid that comes last.  By one thread, which has waited for what the
// others' reads and writes before this call have to be done with.
__device__ inline bool comes_last(Tickets* t) {
  auto count = [](uint32_t* p) { return __hip_atomic_fetch_add(p, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
  auto reset = [](uint32_t* p) { __hip_atomic_store(p, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
  const uint32_t size = max((uint32_t)kGroupLeast, (gridDim.x + kGroups - 1) / kGroups);
  const uint32_t group = blockIdx.x / size, groups = (gridDim.x + size - 1) / size;
  if (count(t->group[group]) != min(size, gridDim.x - group * size) - 1) return false;
  reset(t->group[group]);
  if (count(t->top) != groups - 1) return false;
  reset(t->top);
  return true;
}

// Bound by memory: 57 million fp32 gradients 41.6 us alone (5.5 TB/s), 61 between two steps of AdamW, whose writes go to memory
// meanwhile; 1.1 million 5.0 us, most of it launch, one round of loads, counting and the last sum.
// Squares are formed and added in 64 bits: no gradient is too large or too small for its square, and the sum keeps every digit the
// result has.  The workgroup that finishes last adds the partial sums in their order, so the result does not depend on which it was.
__global__ __launch_bounds__(kThreads) void grad_norm_kernel(Head* head, const Chunk* __restrict__ chunks, int n, float* norm) {
  __shared__ double red[kThreads / 64];
  __shared__ bool last;
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  auto add = [&](float v, int e) { s[e] = fma((double)v, (double)v, s[e]); };
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const Chunk c = chunks[i];
    const Places<kThreads> at(c.count);
    constexpr int U = kChunk / (4 * kThreads);
    auto sum = [&](auto type) {
      typedef decltype(type) T;
      typename Four<T>::vec g[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        g[u] = typename Four<T>::vec{};
        if (at.whole(u)) g[u] = load4<T>(c.grad, at.at(u));
      }
      float one = 0.f;
      if (at.has_rest()) one = load1<T>(c.grad, at.rest());
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) add(Four<T>::get(g[u], e), e);
      add(one, 0);
    };
    if (c.flags & kGradBf16) sum(bf16_t{});
    else sum(float{});
  }
  const double mine = block_sum((s[0] + s[1]) + (s[2] + s[3]), red);
  if (threadIdx.x == 0) {
    // The sum is exchanged, not stored: when the old value is back the new one is where every die sees it, so it can be
    // counted without a release, which would write this die's L2 back (10.5 million gradients: 58 us instead of 32).
    const uint64_t old = __hip_atomic_exchange(&head->part[blockIdx.x], __builtin_bit_cast(uint64_t, mine), __ATOMIC_RELAXED,
                                               __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("" ::"v"((uint32_t)old) : "memory");
    last = comes_last(&head->norm);
  }
  __syncthreads();
  if (!last) return;
  uint64_t part[kMaxParts / kThreads];               // all asked for before the first is added
#pragma unroll
  for (int k = 0; k < kMaxParts / kThreads; ++k) {
    const int i = min(k * kThreads + (int)threadIdx.x, (int)gridDim.x - 1);
    part[k] = __hip_atomic_load(&head->part[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  double t = 0.0;
#pragma unroll
  for (int k = 0; k < kMaxParts / kThreads; ++k)
    t += k * kThreads + (int)threadIdx.x < (int)gridDim.x ? __builtin_bit_cast(double, part[k]) : 0.0;
  t = block_sum(t, red);
  if (threadIdx.x == 0) *norm = (float)sqrt(t);
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

// 10.5 million fp32 gradients into others 11.4 us (7.4 TB/s, they are still in the memory-side cache); 1.1 million into bf16 3.3 us.
__global__ __launch_bounds__(kThreads) void clip_kernel(const Chunk* __restrict__ chunks, int n, const float* norm, float max_norm, int32_t* status) {
  float s;
  const bool sound = clip_factor(norm, max_norm, s);
  if (!sound) {                                       // the formula without its minimum, which would take 1 for NaN
    if (status && blockIdx.x == 0 && threadIdx.x == 0) *status = 1;
    s = max_norm / *norm;
  }
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const Chunk c = chunks[i];
    void* out = c.clip ? c.clip : c.grad;
    if (out == c.grad && (s == 1.f || !sound)) continue;          // in place: nothing changes, or nothing may
    const Places<kThreads> at(c.count);
    constexpr int U = kChunk / (4 * kThreads);
    auto scale = [&](auto from, auto to) {
      typedef decltype(from) T;
      typedef decltype(to) R;
      typename Four<T>::vec g[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (at.whole(u)) g[u] = load4<T>(c.grad, at.at(u));
      float one = 0.f;
      if (at.has_rest()) one = load1<T>(c.grad, at.rest());
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = s * Four<T>::get(g[u], e);
        if (at.whole(u)) store4<R>(out, at.at(u), v);
      }
      if (at.has_rest()) store1<R>(out, at.rest(), s * one);
    };
    const bool from = c.flags & kGradBf16, to = c.flags & (c.clip ? kClipBf16 : kGradBf16);
    if (from) to ? scale(bf16_t{}, bf16_t{}) : scale(bf16_t{}, float{});
    else to ? scale(float{}, bf16_t{}) : scale(float{}, float{});
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

// 57 million weights with fp32 gradients and bf16 copies 242 us (7.1 TB/s of 30 bytes each); 5 million with bf16 gradients 21.6 us (6.1 TB/s);
// 1.1 million 10 us: one round of loads, arithmetic and stores, and the write-back of 16 MB at the kernel's end.  Chunks of 1024
// elements for small lists: 10.0 us there, 15.1 instead of 11.3 for clipping.
template <bool kOnce>
__global__ __launch_bounds__(kAdamThreads) void adamw_kernel(Head* head, const Chunk* __restrict__ chunks, int n, Adam a) {
  float s = 1.f;
  int64_t t = 0;
  bool ready = false, sound = true;
  // What the whole step shares, asked for when the first chunk is on its way.
  auto prepare = [&]() {
    ready = true;
    sound = clip_factor(a.norm, a.max_norm, s);
    if (a.step_dev) {                  // (the host has filled `rate` and `root` in otherwise, and refused what is not sound)
      t = *a.step_dev + 1;
      a.lr = *a.lr_dev;
      a.rate = (float)((double)a.lr / -expm1((double)t * a.log_b1));
      a.root = (float)(1.0 / sqrt(-expm1((double)t * a.log_b2)));
      sound = sound && t >= 1 && a.lr >= 0.f && a.rate - a.rate == 0.f;
    }
    if (!sound && a.status && blockIdx.x == 0 && threadIdx.x == 0) *a.status = 1;
  };
  for (int i = blockIdx.x; i < n && sound; i += gridDim.x) {
    const Chunk c = chunks[i];
    const Places<kAdamThreads> at(c.count);
    constexpr int U = kChunk / (4 * kAdamThreads);
    float shrink = 0.f;                // lr decay
    auto move = [&](float g, float& p, float& m, float& v) {
      const float x = s * g;
      m = fmaf(a.b1, m, a.c1 * x);
      v = fmaf(a.b2, v, a.c2 * x * x);
      // (the decay as a difference: 1 - lr decay itself would lose the digits of lr decay that lie below 2^-24)
      p = fmaf(-a.rate, m / fmaf(sqrtf(v), a.root, a.eps), fmaf(-shrink, p, p));
    };
    auto update = [&](auto type) {
      typedef decltype(type) T;
      typename Four<T>::vec g[U];
      Four<float>::vec p[U], m[U], v[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (at.whole(u)) {
          g[u] = load4<T, kOnce>(c.grad, at.at(u));
          p[u] = load4<float, kOnce>(c.param, at.at(u));
          m[u] = load4<float, kOnce>(c.m, at.at(u));
          v[u] = load4<float, kOnce>(c.v, at.at(u));
        }
      if (!ready) prepare();
      if (!sound) return;
      shrink = a.lr * c.decay;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (at.whole(u)) {
          float np[4], nm[4], nv[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            np[e] = p[u][e];
            nm[e] = m[u][e];
            nv[e] = v[u][e];
            move(Four<T>::get(g[u], e), np[e], nm[e], nv[e]);
          }
          store4<float, kOnce>(c.param, at.at(u), np);
          store4<float, kOnce>(c.m, at.at(u), nm);
          store4<float, kOnce>(c.v, at.at(u), nv);
          if (c.weight) store4<bf16_t>(c.weight, at.at(u), np);
        }
      if (at.has_rest()) {
        const int k = at.rest();
        float p1 = load1<float>(c.param, k), m1 = load1<float>(c.m, k), v1 = load1<float>(c.v, k);
        move(load1<T>(c.grad, k), p1, m1, v1);
        store1<float>(c.param, k, p1);
        store1<float>(c.m, k, m1);
        store1<float>(c.v, k, v1);
        if (c.weight) store1<bf16_t>(c.weight, k, p1);
      }
    };
    if (c.flags & kGradBf16) update(bf16_t{});
    else update(float{});
  }
  if (a.step_dev && a.advance) {       // whoever finishes last: all others have read the counter
    if (!ready) prepare();             // (a list without elements)
    __syncthreads();
    if (sound && threadIdx.x == 0 && comes_last(&head->step)) *a.step_dev = t;
  }
}

// ---------------------------------------------------------------- host side
Head* head_of(const vardrop_tensor_list* l) { return (Head*)l->table; }
Chunk* chunks_of(const vardrop_tensor_list* l) { return (Chunk*)((char*)l->table + sizeof(Head)); }
enum { kHasParams = 1 };

// Weights and moments are next read a step later.  A large model's have left the caches by then, and what they pushed out on their
// way is written back in the next kernels' time: they pass the caches by.  Norm and step with fp32 gradients, kept -> passed by, us,
// three lists in turn (one list over and over): 4.3 million weights 26.3 -> 29.2 (26.3 -> 27.6), 5.3 36.3 -> 35.5 (31.6 -> 34.1), 6.4 46.5 -> 39.9
// (37.2 -> 38.6), 8.5 63.6 -> 52.8 (47.8 -> 52.4), 12.7 89.5 -> 76.4 (68.4 -> 76.5), 25.3 168 -> 138 (162 -> 137), 57 378 -> 314 (378 -> 303).
constexpr int64_t kOnceAbove = 6000000;

int check_list(const vardrop_ctx* ctx, const vardrop_tensor_list* l) {
  if (!ctx || !l || l->built != kBuilt || !l->table || l->chunks < 0) return VARDROP_EINVAL;
  return VARDROP_OK;
}

// Workgroups of a launch: one for every chunk (57 million weights, 256 threads: 250 us, with 2048 workgroups that take several chunks each 263); of
// the norm, as many as are resident together at most, each leaves a partial sum.
unsigned blocks_for(const vardrop_tensor_list* l, int most = 1 << 20) { return (unsigned)(l->chunks < 1 ? 1 : l->chunks < most ? l->chunks : most); }

int adamw(vardrop_ctx* ctx, const vardrop_tensor_list* l, Adam a, double beta1, double beta2, double eps, int64_t step, void* stream) {
  const int rc = check_list(ctx, l);
  if (rc) return rc;
  if (l->tensors > 0 && !(l->has & kHasParams)) return VARDROP_EINVAL;
  if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0)) return VARDROP_EINVAL;
  if (!(a.max_norm >= 0.f) || (a.max_norm > 0.f && !a.norm)) return VARDROP_EINVAL;
  a.b1 = (float)beta1;
  a.c1 = (float)(1.0 - beta1);
  a.b2 = (float)beta2;
  a.c2 = (float)(1.0 - beta2);
  a.eps = (float)eps;
  if (!(a.eps > 0.f) || !(a.eps - a.eps == 0.f)) return VARDROP_EINVAL;      // (it is used in fp32: no 0 / 0 for a weight without moments)
  a.log_b1 = log(beta1);
  a.log_b2 = log(beta2);
  if (!a.step_dev) {
    a.rate = (float)((double)a.lr / -expm1((double)step * a.log_b1));
    a.root = (float)(1.0 / sqrt(-expm1((double)step * a.log_b2)));
    if (!(a.rate - a.rate == 0.f)) return VARDROP_EINVAL;       // (a.lr is at most that)
  }
  hipStream_t s = (hipStream_t)stream;
  VdTimer timer(ctx, VARDROP_K_ADAMW, s);
  const dim3 grid(blocks_for(l)), block(kAdamThreads);
  if (l->numel > kOnceAbove) VD_KERNEL(ctx, adamw_kernel<true>, grid, block, 0, s, head_of(l), chunks_of(l), l->chunks, a);
  else VD_KERNEL(ctx, adamw_kernel<false>, grid, block, 0, s, head_of(l), chunks_of(l), l->chunks, a);
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
  for (int i = 0; i < tensors; ++i) l.numel += numel_host[i];
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
  VD_KERNEL(ctx, clip_kernel, dim3(blocks_for(list)), dim3(kThreads), 0, s, chunks_of(list), list->chunks, norm,
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
