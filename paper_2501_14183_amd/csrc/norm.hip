// Norms before and after a block, fused with the block's gate and the residual scale: what stands between two blocks of
// the backbone (Sec. 4.1) that the attention of this library is one of.
//
//   u = post(f),  r = alpha x + beta g * u,  h = pre(r)          post, pre: LayerNorm, RMSNorm or nothing, over d
//
// with g one row for all tokens, one for each window, or ones.  With hat(v) = (v - mean) rstd (mean = 0 for RMSNorm) and
// <.> the mean over d (the first of the two only for LayerNorm), the gradients are
//
//   D  = dr + rstd (w dh - <w dh> - hat(r) <w dh hat(r)>),  dx = alpha D
//   df = rstd' (q - <q> - hat(f) <q hat(f)>),  q = beta g wp D
//   db = T0 = sum dh,  dw = T1 = sum dh hat(r)                                  sums over the tokens
//   S0 = sum D,  S1 = sum D hat(f) over the tokens of one gate row:
//   dg = beta (wp S1 + bp S0),  dwp = beta sum g S1,  dbp = beta sum g S0       (sum over the gate rows)
//
// so that four column sums give all five vector gradients.  Every row is read once and written once; both directions are bound
// by memory.
#include "common.h"
#include "bf16_mfma.h"
#include <initializer_list>

namespace {

constexpr int kVec = 4;                  // neighbouring elements of a row that a lane holds per chunk
constexpr int kMaxD = 8192;

// A row of d elements belongs to LPR lanes with CH chunks each: element ((c * LPR + lane) * kVec + e).  Rows need no
// alignment: global loads and stores take any element-aligned address.
template <typename T> struct Unit;
template <> struct Unit<float> {
  typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
  float v[4];
  __device__ float get(int e) const { return v[e]; }
  __device__ void load(const float* p) {
    const vec t = *reinterpret_cast<const vec*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = t[e];
  }
  __device__ void load1(const float* p, int e) { v[e] = p[e]; }
  __device__ void zero() { v[0] = v[1] = v[2] = v[3] = 0.f; }
  __device__ static void store(float* p, const float (&t)[4]) { *reinterpret_cast<vec*>(p) = vec{t[0], t[1], t[2], t[3]}; }
  __device__ static void store1(float* p, float t) { *p = t; }
};
template <> struct Unit<bf16_t> {
  typedef uint32_t vec __attribute__((ext_vector_type(2), aligned(2)));
  uint32_t v[2];
  __device__ float get(int e) const { return __uint_as_float(e & 1 ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16); }
  __device__ void load(const bf16_t* p) {
    const vec t = *reinterpret_cast<const vec*>(p);
    v[0] = t.x;
    v[1] = t.y;
  }
  __device__ void load1(const bf16_t* p, int e) { v[e >> 1] |= (uint32_t)p[e] << (16 * (e & 1)); }
  __device__ void zero() { v[0] = v[1] = 0; }
  __device__ static void store(bf16_t* p, const float (&t)[4]) { *reinterpret_cast<vec*>(p) = vec{pack2(t[0], t[1]), pack2(t[2], t[3])}; }
  __device__ static void store1(bf16_t* p, float t) { *p = f2bf(t); }
};

// the chunk that begins at element `at` of a row of d; elements past its end are zero
template <typename T> __device__ inline Unit<T> load_unit(const T* row, int at, int d) {
  Unit<T> u;
  if (at + kVec <= d) {
    u.load(row + at);
  } else {
    u.zero();
    for (int e = 0; e < kVec; ++e)
      if (at + e < d) u.load1(row + at, e);
  }
  return u;
}
template <typename T> __device__ inline void store_unit(T* row, int at, int d, const float (&t)[4]) {
  if (at + kVec <= d) {
    Unit<T>::store(row + at, t);
  } else {
#pragma unroll
    for (int e = 0; e < kVec; ++e)
      if (at + e < d) Unit<T>::store1(row + at + e, t[e]);
  }
}
// a vector of parameters; `none` stands for an absent one, 0 for elements past the end
template <typename T> __device__ inline void load_param(const T* p, int at, int d, float none, float (&out)[4]) {
  if (!p) {
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = at + e < d ? none : 0.f;
    return;
  }
  const Unit<T> u = load_unit(p, at, d);
#pragma unroll
  for (int e = 0; e < 4; ++e) out[e] = u.get(e);
}

template <int CTRL> __device__ inline float dpp_add(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
// Sum over the LPR lanes of a row, the same in all of them.  Rows of several wavefronts meet in `red` (two sets in turn, so that
// one barrier a sum is enough).
template <int LPR, int N>
__device__ inline void row_sum(float (&v)[N], float (*red)[N], int& turn) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = dpp_add<0xB1>(v[i]);          // lane ^ 1
    v[i] = dpp_add<0x4E>(v[i]);          // lane ^ 2
    v[i] = dpp_add<0x141>(v[i]);         // the other four of eight
    v[i] = dpp_add<0x140>(v[i]);         // the other eight of sixteen
    if (LPR >= 32) {
      const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[i]), __float_as_uint(v[i]), false, false);
      v[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if (LPR >= 64) {
      const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[i]), __float_as_uint(v[i]), false, false);
      v[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
  }
  if (LPR > 64) {
    constexpr int W = LPR / 64;
    float (*set)[N] = red + turn * W;
    turn ^= 1;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) set[threadIdx.x >> 6][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) s += set[w][i];
      v[i] = s;
    }
  }
}

struct NormArgs {
  const void *x, *f;                       // forward
  const void *dr, *dh, *r_in;              // backward (and f)
  const void *w, *b, *wp, *bp, *gate;
  void *r, *h;                             // forward
  void *dx, *df;                           // backward
  float* stats;                            // [rows][4]: mean and rstd of post, mean and rstd of pre
  float* part;                             // backward: [segments * pieces][4][d] of T0, T1, S0, S1
  int B, n, d, gates, pre, post, pieces;
  float alpha, beta, eps;
  const int32_t* n_dev;
  int32_t* status;
};

template <int LPR> constexpr int threads_of() { return LPR > 256 ? LPR : 256; }

// One row per group of LPR lanes.  The statistics are taken from fp32 values before r is rounded, deviations about the mean.
template <typename TR, typename TB, int LPR, int CH>
__global__ __launch_bounds__(threads_of<LPR>()) void block_norm_fwd_kernel(NormArgs a) {
  constexpr int T = threads_of<LPR>();
  __shared__ float red[LPR > 64 ? 2 * LPR / 64 : 1][1];
  int n;
  if (!vd_count(a.n_dev, a.n, n, a.status)) return;
  const long long rows = (long long)a.B * n;
  const int lane = threadIdx.x % LPR, d = a.d;
  const float inv_d = 1.f / (float)d;
  int turn = 0;
  for (long long row = (long long)blockIdx.x * (T / LPR) + threadIdx.x / LPR; row < rows; row += (long long)gridDim.x * (T / LPR)) {
    const long long off = row * d;
    const TB* gate = a.gate ? (const TB*)a.gate + (a.gates > 1 ? (long long)((uint32_t)row / (uint32_t)n) * d : 0) : nullptr;

    Unit<TR> xr[CH];
    Unit<TB> fr[CH];
  #pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int at = (c * LPR + lane) * kVec;
      xr[c] = load_unit((const TR*)a.x + off, at, d);
      if (a.f) fr[c] = load_unit((const TB*)a.f + off, at, d);
    }
    float v[CH][4];
    float mean_p = 0.f, rstd_p = 1.f, mean = 0.f, rstd = 1.f;
    auto moments = [&](int kind, float& m, float& k) {
      m = 0.f;
      k = 1.f;
      if (kind == VARDROP_NORM_NONE) return;
      if (kind == VARDROP_NORM_LAYER) {
        float s[1] = {0.f};
  #pragma unroll
        for (int c = 0; c < CH; ++c)
  #pragma unroll
          for (int e = 0; e < 4; ++e) s[0] += v[c][e];
        row_sum<LPR>(s, red, turn);
        m = s[0] * inv_d;
      }
      float q[1] = {0.f};
  #pragma unroll
      for (int c = 0; c < CH; ++c)
  #pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float t = (c * LPR + lane) * kVec + e < d ? v[c][e] - m : 0.f;
          q[0] = fmaf(t, t, q[0]);
        }
      row_sum<LPR>(q, red, turn);
      k = 1.f / sqrtf(q[0] * inv_d + a.eps);
    };
    if (a.f) {
  #pragma unroll
      for (int c = 0; c < CH; ++c)
  #pragma unroll
        for (int e = 0; e < 4; ++e) v[c][e] = fr[c].get(e);
      moments(a.post, mean_p, rstd_p);
  #pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int at = (c * LPR + lane) * kVec;
        float wp[4], bp[4], g[4];
        load_param((const TB*)a.wp, at, d, 1.f, wp);
        load_param((const TB*)a.bp, at, d, 0.f, bp);
        load_param(gate, at, d, 1.f, g);
  #pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float u = fmaf((v[c][e] - mean_p) * rstd_p, wp[e], bp[e]);
          v[c][e] = fmaf(a.beta * g[e], u, a.alpha * xr[c].get(e));
        }
      }
    } else {
  #pragma unroll
      for (int c = 0; c < CH; ++c)
  #pragma unroll
        for (int e = 0; e < 4; ++e) v[c][e] = a.alpha * xr[c].get(e);
    }
    if (a.r)
  #pragma unroll
      for (int c = 0; c < CH; ++c) store_unit((TR*)a.r + off, (c * LPR + lane) * kVec, d, v[c]);
    moments(a.pre, mean, rstd);
    if (a.h) {
  #pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int at = (c * LPR + lane) * kVec;
        float w[4], b[4], o[4];
        load_param((const TB*)a.w, at, d, 1.f, w);
        load_param((const TB*)a.b, at, d, 0.f, b);
  #pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = fmaf((v[c][e] - mean) * rstd, w[e], b[e]);
        store_unit((TB*)a.h + off, at, d, o);
      }
    }
    if (a.stats && lane == 0) *reinterpret_cast<float4*>(a.stats + 4 * row) = make_float4(mean_p, rstd_p, mean, rstd);
  }
}

// Rows of one segment (the tokens of a gate row) in `pieces` ranges, one workgroup each; its groups walk the range in
// turn and keep their column sums in registers, the next row on its way while this one is worked on.
template <typename TR, typename TB, int LPR, int CH>
__global__ __launch_bounds__(threads_of<LPR>()) void block_norm_bwd_kernel(NormArgs a) {
  constexpr int T = threads_of<LPR>(), G = T / LPR;
  __shared__ float red[LPR > 64 ? 2 * LPR / 64 : 1][2];
  __shared__ float sums[G > 1 ? G : 1][G > 1 ? LPR * CH * 4 : 1];
  int n;
  if (!vd_count(a.n_dev, a.n, n, a.status)) return;
  const int segment = blockIdx.x / a.pieces, piece = blockIdx.x - segment * a.pieces, d = a.d;
  const long long seg_rows = a.gates > 1 ? n : (long long)a.B * n;
  const long long chunk = (seg_rows + a.pieces - 1) / a.pieces;
  const long long first = segment * seg_rows;
  const long long r0 = first + min(seg_rows, piece * chunk), r1 = first + min(seg_rows, (piece + 1) * chunk);
  const int group = threadIdx.x / LPR, lane = threadIdx.x % LPR;
  const float inv_d = 1.f / (float)d;
  const bool branch = a.df != nullptr || a.f != nullptr;
  const float pre_mean = a.pre == VARDROP_NORM_LAYER ? inv_d : 0.f, post_mean = a.post == VARDROP_NORM_LAYER ? inv_d : 0.f;
  int turn = 0;

  float w[CH][4], gq[CH][4];               // weight of pre; beta g wp
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int at = (c * LPR + lane) * kVec;
    load_param((const TB*)a.w, at, d, 1.f, w[c]);
    float wp[4], g[4];
    load_param((const TB*)a.wp, at, d, 1.f, wp);
    load_param(a.gate ? (const TB*)a.gate + (long long)segment * d : nullptr, at, d, 1.f, g);
#pragma unroll
    for (int e = 0; e < 4; ++e) gq[c][e] = a.beta * g[e] * wp[e];
  }
  float t0[CH][4] = {}, t1[CH][4] = {}, s0[CH][4] = {}, s1[CH][4] = {};

  Unit<TR> dr[CH], r[CH];
  Unit<TB> dh[CH], f[CH];
  float4 st = make_float4(0.f, 1.f, 0.f, 1.f);
  auto fetch = [&](long long row) {
    const long long off = row * d;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int at = (c * LPR + lane) * kVec;
      if (a.dr) dr[c] = load_unit((const TR*)a.dr + off, at, d);
      if (a.dh) {
        dh[c] = load_unit((const TB*)a.dh + off, at, d);
        r[c] = load_unit((const TR*)a.r_in + off, at, d);
      }
      if (a.f) f[c] = load_unit((const TB*)a.f + off, at, d);
    }
    if (a.stats) st = *reinterpret_cast<const float4*>(a.stats + 4 * row);
  };
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    dr[c].zero();
    r[c].zero();
    dh[c].zero();
    f[c].zero();
  }
  long long row = r0 + group;
  // (rows of several wavefronts: one group, so that all threads meet at the barriers)
  if (row < r1) fetch(row);
  for (; row < r1; row += G) {
    const long long off = row * d;
    const float mean_p = st.x, rstd_p = st.y, mean = st.z, rstd = st.w;
    float D[CH][4], fh[CH][4];
    {
      float hat[CH][4], t[CH][4], s[2] = {0.f, 0.f};
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool in = (c * LPR + lane) * kVec + e < d;      // (past the end all of these are zero)
          const float g = dh[c].get(e);
          D[c][e] = dr[c].get(e);
          fh[c][e] = in ? (f[c].get(e) - mean_p) * rstd_p : 0.f;
          hat[c][e] = in ? (r[c].get(e) - mean) * rstd : 0.f;
          t[c][e] = w[c][e] * g;
          s[0] += t[c][e];
          s[1] = fmaf(t[c][e], hat[c][e], s[1]);
          t0[c][e] += g;
          t1[c][e] = fmaf(g, hat[c][e], t1[c][e]);
        }
      if (row + G < r1) fetch(row + G);
      if (a.dh) {
        row_sum<LPR>(s, red, turn);
        const float m0 = s[0] * pre_mean, m1 = s[1] * inv_d;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) D[c][e] = fmaf(rstd, t[c][e] - m0 - hat[c][e] * m1, D[c][e]);
      }
    }
    if (a.dx)
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        float o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = a.alpha * D[c][e];
        store_unit((TR*)a.dx + off, (c * LPR + lane) * kVec, d, o);
      }
    if (branch) {
      float q[2] = {0.f, 0.f};
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s0[c][e] += D[c][e];
          s1[c][e] = fmaf(D[c][e], fh[c][e], s1[c][e]);
          D[c][e] = (c * LPR + lane) * kVec + e < d ? D[c][e] * gq[c][e] : 0.f;
          q[0] += D[c][e];
          q[1] = fmaf(D[c][e], fh[c][e], q[1]);
        }
      if (a.post != VARDROP_NORM_NONE) row_sum<LPR>(q, red, turn);
      const float m0 = a.post == VARDROP_NORM_NONE ? 0.f : q[0] * post_mean, m1 = a.post == VARDROP_NORM_NONE ? 0.f : q[1] * inv_d;
      if (a.df)
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          float o[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = rstd_p * (D[c][e] - m0 - fh[c][e] * m1);
          store_unit((TB*)a.df + off, (c * LPR + lane) * kVec, d, o);
        }
    }
  }
  // column sums of the groups, in their order
  float* part = a.part + (long long)blockIdx.x * 4 * d;
  auto flush = [&](float (&v)[CH][4], float* out) {
    if (G == 1) {
#pragma unroll
      for (int c = 0; c < CH; ++c) store_unit(out, (c * LPR + lane) * kVec, d, v[c]);
      return;
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) sums[group][(c * LPR + lane) * kVec + e] = v[c][e];
    __syncthreads();
    for (int i = threadIdx.x; i < d; i += T) {
      float s = 0.f;
#pragma unroll
      for (int g = 0; g < G; ++g) s += sums[g][i];
      out[i] = s;
    }
  };
  if (!a.part) return;
  flush(t0, part);
  flush(t1, part + d);
  flush(s0, part + 2 * d);
  flush(s1, part + 3 * d);
}

// The vector gradients from the pieces' column sums.  A workgroup takes 64 columns; blockIdx.y 0: db, dw; 1: dbp, dwp (every
// piece weighted with its gate row); 2 + g: gate row g.
template <typename TB>
__global__ __launch_bounds__(1024) void block_norm_vectors_kernel(NormArgs a, float* dw, float* db, float* dwp, float* dbp,
                                                                  float* dgate, int segments) {
  __shared__ float red[16][64][2];
  int n;
  if (!vd_count(a.n_dev, a.n, n)) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, what = blockIdx.y, d = a.d;
  const int col = blockIdx.x * 64 + lane, c = min(col, d - 1);
  int p0 = 0, p1 = segments * a.pieces;
  if (what >= 2 && a.gates > 1) {
    p0 = (what - 2) * a.pieces;
    p1 = p0 + a.pieces;
  }
  const bool weighted = what == 1 && a.gates > 1;
  const float* src = a.part + (what == 0 ? 0 : 2 * d) + c;
  float s0 = 0.f, s1 = 0.f;
  for (int p = p0 + wave; p < p1; p += 16 * 8) {
    float v0[8], v1[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float* q = src + (long long)min(p + 16 * i, p1 - 1) * 4 * d;
      v0[i] = q[0];
      v1[i] = q[d];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int at = p + 16 * i;
      if (at >= p1) break;
      float g = 1.f;
      if (weighted) {
        const TB* row = (const TB*)a.gate + (long long)(at / a.pieces) * d + c;
        Unit<TB> u;
        u.zero();
        u.load1(row, 0);
        g = u.get(0);
      }
      s0 = fmaf(g, v0[i], s0);
      s1 = fmaf(g, v1[i], s1);
    }
  }
  red[wave][lane][0] = s0;
  red[wave][lane][1] = s1;
  __syncthreads();
  if (wave != 0 || col >= d) return;
  s0 = s1 = 0.f;
#pragma unroll
  for (int w = 0; w < 16; ++w) {
    s0 += red[w][lane][0];
    s1 += red[w][lane][1];
  }
  auto param = [&](const void* p, float none) {
    if (!p) return none;
    Unit<TB> u;
    u.zero();
    u.load1((const TB*)p + col, 0);
    return u.get(0);
  };
  if (what == 0) {
    if (db) db[col] = s0;
    if (dw) dw[col] = s1;
  } else if (what == 1) {
    const float k = a.beta * (a.gates == 1 ? param(a.gate, 1.f) : 1.f);
    if (dbp) dbp[col] = k * s0;
    if (dwp) dwp[col] = k * s1;
  } else {
    dgate[(long long)(what - 2) * d + col] = a.beta * fmaf(param(a.wp, 1.f), s1, param(a.bp, 0.f) * s0);
  }
}

// ---------------------------------------------------------------- host side
struct Shape {
  int lanes, chunks;
};
// Lanes and chunks of a row of d elements: as many lanes as hold it with one chunk each, up to a wavefront; then up to four chunks;
// then several wavefronts.
Shape shape_of(int d) {
  if (d <= 64) return {16, 1};
  if (d <= 128) return {32, 1};
  if (d <= 1024) return {64, vd_ceil_div(d, 256)};
  if (d <= 4096) return {256, d <= 2048 ? 2 : 4};
  return {512, 4};
}
#define VD_NORM_SHAPES(X) X(16, 1) X(32, 1) X(64, 1) X(64, 2) X(64, 3) X(64, 4) X(256, 2) X(256, 4) X(512, 4)

// Workgroups per segment of the backward.
int pieces_of(int B, int n, int d, int gates) {
  const int segments = gates > 1 ? gates : 1;
  const Shape s = shape_of(d);
  const int groups = (s.lanes > 256 ? s.lanes : 256) / s.lanes;
  const long long rows = gates > 1 ? n : (long long)B * n;
  long long p = vd_ceil_div(768, segments);
  const long long most = (rows + groups - 1) / groups;
  if (p > most) p = most;
  return p < 1 ? 1 : (int)p;
}

// Workgroups of the forward: one turn for every row up to half a million of them (a launch holds fewer than 2^32 threads).
unsigned blocks_of(long long rows, int groups) {
  const long long b = (rows + groups - 1) / groups;
  return (unsigned)(b < (1 << 19) ? b : (1 << 19));
}

template <bool kBackward, typename TR, typename TB>
int launch(vardrop_ctx* ctx, const NormArgs& a, long long groups_of_rows, hipStream_t s) {
  const Shape sh = shape_of(a.d);
  VdTimer timer(ctx, kBackward ? VARDROP_K_BLOCK_NORM_BWD : VARDROP_K_BLOCK_NORM_FWD, s);
#define VD_CASE(L, C)                                                                                              \
  if (sh.lanes == L && sh.chunks == C) {                                                                           \
    constexpr int T = threads_of<L>();                                                                             \
    if (kBackward) VD_KERNEL(ctx, (block_norm_bwd_kernel<TR, TB, L, C>), dim3((unsigned)groups_of_rows), dim3(T), 0, s, a); \
    else VD_KERNEL(ctx, (block_norm_fwd_kernel<TR, TB, L, C>), dim3(blocks_of(groups_of_rows, T / L)), dim3(T), 0, s, a); \
  }
  VD_NORM_SHAPES(VD_CASE)
#undef VD_CASE
  VD_LAUNCH_CHECK(ctx);
  return VARDROP_OK;
}

template <bool kBackward>
int launch_types(vardrop_ctx* ctx, const NormArgs& a, int res_dtype, int dtype, long long count, hipStream_t s) {
  if (dtype == VARDROP_F32) return launch<kBackward, float, float>(ctx, a, count, s);
  if (res_dtype == VARDROP_F32) return launch<kBackward, float, bf16_t>(ctx, a, count, s);
  return launch<kBackward, bf16_t, bf16_t>(ctx, a, count, s);
}

bool is_kind(int k) { return k == VARDROP_NORM_NONE || k == VARDROP_NORM_LAYER || k == VARDROP_NORM_RMS; }
bool is_finite(float v) { return v - v == 0.f; }
// Element alignment of the tensors of one type (null pointers count as aligned).
template <typename... P> bool aligned_to(int dtype, P... p) {
  uintptr_t all = 0;
  for (const void* q : {(const void*)p...}) all |= (uintptr_t)q;
  return all % (dtype == VARDROP_F32 ? 4 : 2) == 0;
}

int check(vardrop_ctx* ctx, int B, int n, int d, int res_dtype, int dtype, int post, const void* wp, const void* bp,
          const void* gate, int gates, float alpha, float beta, int pre, const void* w, const void* b) {
  if (!ctx || B < 0 || n < 0 || d < 1) return VARDROP_EINVAL;
  if ((dtype != VARDROP_F32 && dtype != VARDROP_BF16) || (res_dtype != VARDROP_F32 && res_dtype != VARDROP_BF16)) return VARDROP_EINVAL;
  if (!is_kind(pre) || !is_kind(post)) return VARDROP_EINVAL;
  if ((pre == VARDROP_NORM_NONE && (w || b)) || (post == VARDROP_NORM_NONE && (wp || bp))) return VARDROP_EINVAL;
  if (gate ? (gates != 1 && gates != B) : gates != 0) return VARDROP_EINVAL;
  if (!is_finite(alpha) || !is_finite(beta)) return VARDROP_EINVAL;
  if (dtype == VARDROP_F32 && res_dtype != VARDROP_F32) return VARDROP_EUNSUPPORTED;
  if (d > kMaxD || (long long)B * n >= (1ll << 31) || gates > 65000) return VARDROP_EUNSUPPORTED;
  return VARDROP_OK;
}

int forward(vardrop_ctx* ctx, const void* x, const void* f, int B, int n, int d, int res_dtype, int dtype, int post,
            const void* wp, const void* bp, const void* gate, int gates, float alpha, float beta, int pre, const void* w,
            const void* b, float eps, void* r, void* h, float* stats, void* stream, VdDevCount dn) {
  const int rc = check(ctx, B, n, d, res_dtype, dtype, post, wp, bp, gate, gates, alpha, beta, pre, w, b);
  if (rc) return rc;
  if (!(eps > 0.f) || !is_finite(eps)) return VARDROP_EINVAL;
  if ((long long)B * n == 0) return VARDROP_OK;          // (pointers to nothing may be null)
  if (!f && (post != VARDROP_NORM_NONE || gate)) return VARDROP_EINVAL;
  if ((h != nullptr) != (pre != VARDROP_NORM_NONE)) return VARDROP_EINVAL;
  if (!r && !h) return VARDROP_EINVAL;
  if (!x || !vd_aligned(stats, 16) || !aligned_to(res_dtype, x, r) || !aligned_to(dtype, f, h, w, b, wp, bp, gate)) return VARDROP_EINVAL;
  NormArgs a = {};
  a.x = x; a.f = f; a.w = w; a.b = b; a.wp = wp; a.bp = bp; a.gate = gate; a.r = r; a.h = h; a.stats = stats;
  a.B = B; a.n = n; a.d = d; a.gates = gates; a.pre = pre; a.post = post;
  a.alpha = alpha; a.beta = beta; a.eps = eps;
  a.n_dev = dn.dev; a.status = dn.status;
  return launch_types<false>(ctx, a, res_dtype, dtype, (long long)B * n, (hipStream_t)stream);
}

int backward(vardrop_ctx* ctx, const void* dr, const void* dh, const void* r, const void* f, const float* stats, int B, int n,
             int d, int res_dtype, int dtype, int post, const void* wp, const void* bp, const void* gate, int gates, float alpha,
             float beta, int pre, const void* w, void* dx, void* df, float* dw, float* db, float* dwp, float* dbp, float* dgate,
             void* ws, size_t ws_bytes, void* stream, VdDevCount dn) {
  const int rc = check(ctx, B, n, d, res_dtype, dtype, post, wp, bp, gate, gates, alpha, beta, pre, w, nullptr);
  if (rc) return rc;
  const bool normed = pre != VARDROP_NORM_NONE || post != VARDROP_NORM_NONE;
  if ((long long)B * n > 0) {
    if (!dr && !dh) return VARDROP_EINVAL;
    if ((dh != nullptr) != (pre != VARDROP_NORM_NONE) || (dh && !r)) return VARDROP_EINVAL;
    if (!f && (post != VARDROP_NORM_NONE || gate || dgate)) return VARDROP_EINVAL;
    if (normed && !stats) return VARDROP_EINVAL;
  }
  if ((pre == VARDROP_NORM_NONE && (dw || db)) || (post == VARDROP_NORM_NONE && (dwp || dbp)) || (dgate && !gate)) return VARDROP_EINVAL;
  if (!vd_aligned(stats, 16) || !aligned_to(res_dtype, dr, r, dx) || !aligned_to(dtype, dh, f, df, w, wp, bp, gate) ||
      !aligned_to(VARDROP_F32, dw, db, dwp, dbp, dgate))
    return VARDROP_EINVAL;
  const bool vectors = dw || db || dwp || dbp || dgate;
  if ((long long)B * n == 0 && !vectors) return VARDROP_OK;
  const size_t need = vardrop_block_norm_workspace_bytes(B, n, d, gates);
  if (vectors && (!ws || !vd_aligned(ws, 256) || ws_bytes < need)) return VARDROP_EWORKSPACE;
  NormArgs a = {};
  a.dr = dr; a.dh = dh; a.r_in = r; a.f = f; a.w = w; a.wp = wp; a.bp = bp; a.gate = gate; a.dx = dx; a.df = df;
  a.stats = normed ? const_cast<float*>(stats) : nullptr;
  a.part = vectors ? (float*)ws : nullptr;
  a.B = B; a.n = n; a.d = d; a.gates = gates; a.pre = pre; a.post = post;
  a.alpha = alpha; a.beta = beta;
  a.n_dev = dn.dev; a.status = dn.status;
  a.pieces = pieces_of(B, n, d, gates);
  const int segments = gates > 1 ? gates : 1;
  hipStream_t s = (hipStream_t)stream;
  const int rb = launch_types<true>(ctx, a, res_dtype, dtype, (long long)segments * a.pieces, s);
  if (rb || !vectors) return rb;
  const dim3 grid((unsigned)vd_ceil_div(d, 64), (unsigned)(dgate ? 2 + gates : (dwp || dbp) ? 2 : 1));
  VdTimer timer(ctx, VARDROP_K_BLOCK_NORM_VECTORS, s);
  if (dtype == VARDROP_F32) VD_KERNEL(ctx, block_norm_vectors_kernel<float>, grid, dim3(1024), 0, s, a, dw, db, dwp, dbp, dgate, segments);
  else VD_KERNEL(ctx, block_norm_vectors_kernel<bf16_t>, grid, dim3(1024), 0, s, a, dw, db, dwp, dbp, dgate, segments);
  VD_LAUNCH_CHECK(ctx);
  return VARDROP_OK;
}

}  // namespace

extern "C" size_t vardrop_block_norm_workspace_bytes(int B, int n, int d, int gates) {
  if (B < 0 || n < 0 || d < 1 || d > kMaxD || gates < 0 || gates > 65000 || (gates > 1 && gates != B)) return 0;
  const size_t segments = gates > 1 ? gates : 1;
  return vd_align_up(segments * pieces_of(B, n, d, gates) * 4 * (size_t)d * sizeof(float), 256);
}

extern "C" int vardrop_block_norm_fwd(vardrop_ctx* ctx, const void* x, const void* f, int B, int n, int d, int res_dtype,
                                      int dtype, int post, const void* wp, const void* bp, const void* gate, int gates,
                                      float alpha, float beta, int pre, const void* w, const void* b, float eps,
                                      void* r, void* h, float* stats, void* stream) {
  return forward(ctx, x, f, B, n, d, res_dtype, dtype, post, wp, bp, gate, gates, alpha, beta, pre, w, b, eps, r, h, stats,
                 stream, {nullptr, nullptr});
}

extern "C" int vardrop_block_norm_fwd_dev(vardrop_ctx* ctx, const void* x, const void* f, int B, const int32_t* n_dev, int n_max,
                                          int32_t* status, int d, int res_dtype, int dtype, int post, const void* wp,
                                          const void* bp, const void* gate, int gates, float alpha, float beta, int pre,
                                          const void* w, const void* b, float eps, void* r, void* h, float* stats, void* stream) {
  if (!n_dev || n_max < 1) return VARDROP_EINVAL;
  return forward(ctx, x, f, B, n_max, d, res_dtype, dtype, post, wp, bp, gate, gates, alpha, beta, pre, w, b, eps, r, h, stats,
                 stream, {n_dev, status});
}

extern "C" int vardrop_block_norm_bwd(vardrop_ctx* ctx, const void* dr, const void* dh, const void* r, const void* f,
                                      const float* stats, int B, int n, int d, int res_dtype, int dtype, int post,
                                      const void* wp, const void* bp, const void* gate, int gates, float alpha, float beta,
                                      int pre, const void* w, void* dx, void* df, float* dw, float* db, float* dwp, float* dbp,
                                      float* dgate, void* ws, size_t ws_bytes, void* stream) {
  return backward(ctx, dr, dh, r, f, stats, B, n, d, res_dtype, dtype, post, wp, bp, gate, gates, alpha, beta, pre, w, dx, df,
                  dw, db, dwp, dbp, dgate, ws, ws_bytes, stream, {nullptr, nullptr});
}

extern "C" int vardrop_block_norm_bwd_dev(vardrop_ctx* ctx, const void* dr, const void* dh, const void* r, const void* f,
                                          const float* stats, int B, const int32_t* n_dev, int n_max, int32_t* status, int d,
                                          int res_dtype, int dtype, int post, const void* wp, const void* bp, const void* gate,
                                          int gates, float alpha, float beta, int pre, const void* w, void* dx, void* df,
                                          float* dw, float* db, float* dwp, float* dbp, float* dgate, void* ws, size_t ws_bytes,
                                          void* stream) {
  if (!n_dev || n_max < 1) return VARDROP_EINVAL;
  return backward(ctx, dr, dh, r, f, stats, B, n_max, d, res_dtype, dtype, post, wp, bp, gate, gates, alpha, beta, pre, w, dx,
                  df, dw, db, dwp, dbp, dgate, ws, ws_bytes, stream, {n_dev, status});
}
