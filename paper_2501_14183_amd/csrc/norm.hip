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
#include <type_traits>

namespace {

constexpr int kVec = 4;                  // neighbouring elements of a row that a lane holds per chunk
constexpr int kMaxD = 8192;

// A row of d elements belongs to LPR lanes with CH chunks each: element ((c * LPR + lane) * kVec + e).  All chunks but the last
// are whole; how the last one ends (End) is part of a kernel's type: d is a multiple of what the lanes hold; of kVec only; not of
// kVec; less than kVec.
enum End { kWhole, kCut, kRagged, kTiny };

// All tensors are reached through buffer descriptors that begin at the wavefront's row: what is not there (a tensor that was
// not given, lanes past the end of a row, rows past the last) lies outside a descriptor's range, where loads give zero and
// stores are dropped.  So a row's loads and stores stand without branches, and the wait for the loads of the next row need
// not wait for the stores of this one: with branches the compiler cannot count the stores behind the loads (backward of 39 062 x 640
// bf16 93 us instead of 66).  Rows need element alignment only.
typedef __amdgpu_buffer_rsrc_t Window;
constexpr int kRange = 1 << 28, kOutside = 1 << 28;      // bytes; elements, of two bytes or more
template <typename T> __device__ inline Window window(const void* tensor, long long first) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)((const T*)tensor + first), 0, tensor ? kRange : 0, 0x00020000);
}

typedef uint32_t raw4 __attribute__((ext_vector_type(4)));
typedef uint32_t raw2 __attribute__((ext_vector_type(2)));
template <typename T> struct Unit;
template <> struct Unit<float> {
  raw4 v;
  __device__ float get(int e) const { return __uint_as_float(v[e]); }
  __device__ void load(Window w, int at) { v = __builtin_amdgcn_raw_buffer_load_b128(w, at * 4, 0, 0); }
  __device__ void load1(Window w, int at, int e) { v[e] = __builtin_amdgcn_raw_buffer_load_b32(w, at * 4, 0, 0); }
  __device__ void fill(float f) { v = __float_as_uint(f); }
  // the elements from the k-th on, k < 4, zeros behind them
  __device__ void drop(int k) {
    if (k & 1) v = raw4{v[1], v[2], v[3], 0};
    if (k & 2) v = raw4{v[2], v[3], 0, 0};
  }
  template <int kCache> __device__ static void store(Window w, int at, const float (&t)[4]) {
    __builtin_amdgcn_raw_buffer_store_b128(raw4{__float_as_uint(t[0]), __float_as_uint(t[1]), __float_as_uint(t[2]), __float_as_uint(t[3])}, w, at * 4, 0, kCache);
  }
  __device__ static void store1(Window w, int at, float t) { __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(t), w, at * 4, 0, 0); }
};
template <> struct Unit<bf16_t> {
  raw2 v;
  __device__ float get(int e) const { return __uint_as_float(e & 1 ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16); }
  __device__ void load(Window w, int at) { v = __builtin_amdgcn_raw_buffer_load_b64(w, at * 2, 0, 0); }
  __device__ void load1(Window w, int at, int e) {
    const uint32_t t = __builtin_amdgcn_raw_buffer_load_b16(w, at * 2, 0, 0);
    v[e >> 1] = e & 1 ? v[e >> 1] | t << 16 : t;
  }
  __device__ void fill(float f) { v = f2bf(f) * 0x10001u; }
  __device__ void drop(int k) {
    const uint64_t t = ((uint64_t)v[1] << 32 | v[0]) >> (16 * k);
    v = raw2{(uint32_t)t, (uint32_t)(t >> 32)};
  }
  template <int kCache> __device__ static void store(Window w, int at, const float (&t)[4]) {
    __builtin_amdgcn_raw_buffer_store_b64(raw2{pack2(t[0], t[1]), pack2(t[2], t[3])}, w, at * 2, 0, kCache);
  }
  __device__ static void store1(Window w, int at, float t) { __builtin_amdgcn_raw_buffer_store_b16(f2bf(t), w, at * 2, 0, 0); }
};

// Where a lane's chunk lies in a window whose rows are d apart: `sub` rows behind the window's first, nowhere unless `active`.
template <End kEnd> struct Spot {
  int at, d, base;
  bool active;
  __device__ Spot(int at_, int d_, int sub, bool active_) : at(at_), d(d_), base(sub * d_), active(active_) {}
  __device__ int one(int e) const { return active && at + e < d ? base + at + e : kOutside; }
  template <typename T> __device__ void load(Unit<T>& u, Window w) const {
    if constexpr (kEnd == kTiny) {
#pragma unroll
      for (int e = 0; e < kVec; ++e) u.load1(w, one(e), e);
    } else {
      // (a ragged chunk is cut from the last four elements of the row, see trim)
      const int from = kEnd == kRagged ? min(at, d - kVec) : at;
      u.load(w, active && (kEnd == kWhole || at < d) ? base + from : kOutside);
    }
  }
  // after the wait: brings a loaded chunk into place
  template <typename T> __device__ void trim(Unit<T>& u) const {
    if constexpr (kEnd == kRagged) u.drop(at < d ? max(0, at - (d - kVec)) : 0);
  }
  // past: no copy is left in the caches (see kPastCaches)
  template <typename T, bool kPast = false> __device__ void store(Window w, const float (&t)[4]) const {
    constexpr int kNontemporal = 2;
    if constexpr (kEnd != kTiny) {
      const int to = active && (kEnd == kWhole || at + kVec <= d) ? base + at : kOutside;
      Unit<T>::template store<kPast ? kNontemporal : 0>(w, to, t);
    }
    if constexpr (kEnd == kRagged || kEnd == kTiny) {
#pragma unroll
      for (int e = 0; e < kVec - 1; ++e) Unit<T>::store1(w, at + kVec > d ? one(e) : kOutside, t[e]);
    }
  }
  __device__ bool has(int e) const { return kEnd == kWhole || at + e < d; }
};

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
  bool past;                               // forward: h is written past the caches
  float alpha, beta, eps;
  const int32_t* n_dev;
  int32_t* status;
};

template <int LPR> constexpr int threads_of() { return LPR > 256 ? LPR : 256; }

// Calls body(c, spot) for every chunk.
template <int LPR, int CH, End kEnd, typename F> __device__ inline void for_chunks(int d, int sub, bool active, F body) {
  const int lane = threadIdx.x % LPR;
#pragma unroll
  for (int c = 0; c < CH - 1; ++c) body(c, Spot<kWhole>((c * LPR + lane) * kVec, d, sub, active));
  body(CH - 1, Spot<kEnd>(((CH - 1) * LPR + lane) * kVec, d, sub, active));
}
// A wavefront's first group of lanes, the same in all its lanes, and a lane's group behind that.
template <int LPR> __device__ inline int first_group() {
  return LPR <= 64 ? __builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64)) * (64 / LPR) : 0;
}
template <int LPR> __device__ inline int sub_group() { return LPR < 64 ? (int)(threadIdx.x % 64) / LPR : 0; }

// A row has LPR lanes of 4 to 16 elements each (shape_of); a group of lanes takes one row or several, the next one on its way
// while this one is worked on.  Everything a row needs is asked for at once.  27 584 rows of 512 with a fp32 residual, norms on both sides and a
// gate for each window 27-28 us (6.1 TB/s; 46 with each vector asked for when it was needed), 2080 rows of 512 bf16 4.6 us (launch and one round
// of loads).  The statistics are taken from fp32 values before r is rounded, deviations about the mean.
template <typename TR, typename TB, int LPR, int CH, End kEnd>
__global__ __launch_bounds__(threads_of<LPR>()) void block_norm_fwd_kernel(NormArgs a) {
  constexpr int T = threads_of<LPR>();
  __shared__ float red[LPR > 64 ? 2 * LPR / 64 : 1][1];
  int n;
  if (!vd_count(a.n_dev, a.n, n, a.status)) return;
  const long long rows = (long long)a.B * n;
  const int d = a.d, sub = sub_group<LPR>();
  const float inv_d = 1.f / (float)d;
  int turn = 0;
  Unit<TB> wp[CH], bp[CH], w[CH], b[CH];
  {
    const Window wwp = window<TB>(a.wp, 0), wbp = window<TB>(a.bp, 0), ww = window<TB>(a.w, 0), wb = window<TB>(a.b, 0);
    for_chunks<LPR, CH, kEnd>(d, 0, true, [&](int c, auto at) {
      at.load(wp[c], wwp);
      at.load(bp[c], wbp);
      at.load(w[c], ww);
      at.load(b[c], wb);
    });
  }
  Unit<TR> x[CH];
  Unit<TB> f[CH], g[CH];
  auto fetch = [&](long long row) {
    const bool active = LPR >= 64 || row + sub < rows;
    const Window wx = window<TR>(a.x, row * d), wf = window<TB>(a.f, row * d);
    for_chunks<LPR, CH, kEnd>(d, sub, active, [&](int c, auto at) {
      at.load(x[c], wx);
      at.load(f[c], wf);
    });
    int gate = 0, sub_gate = 0;
    if (a.gates > 1) {
      gate = (int)((uint32_t)row / (uint32_t)n);
      if (LPR < 64) sub_gate = (int)((uint32_t)(row + sub) / (uint32_t)n) - gate;
    }
    const Window wg = window<TB>(a.gate, (long long)gate * d);
    for_chunks<LPR, CH, kEnd>(d, sub_gate, active, [&](int c, auto at) { at.load(g[c], wg); });
  };
  const long long stride = (long long)gridDim.x * (T / LPR);
  long long row = (long long)blockIdx.x * (T / LPR) + first_group<LPR>();
  if (row < rows) fetch(row);
  for_chunks<LPR, CH, kEnd>(d, 0, true, [&](int c, auto at) {
    at.trim(wp[c]);
    at.trim(bp[c]);
    at.trim(w[c]);
    at.trim(b[c]);
    if (!a.wp) wp[c].fill(1.f);
    if (!a.w) w[c].fill(1.f);
  });
  for (; row < rows; row += stride) {
    const bool active = LPR >= 64 || row + sub < rows;
    float v[CH][4], res[CH][4], scale[CH][4];       // f; alpha x; beta g
    for_chunks<LPR, CH, kEnd>(d, sub, active, [&](int c, auto at) {
      at.trim(x[c]);
      at.trim(f[c]);
      at.trim(g[c]);
      if (!a.gate) g[c].fill(1.f);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[c][e] = f[c].get(e);
        res[c][e] = a.alpha * x[c].get(e);
        scale[c][e] = a.beta * g[c].get(e);
      }
    });
    if (row + stride < rows) fetch(row + stride);
    float mean_p = 0.f, rstd_p = 1.f, mean = 0.f, rstd = 1.f;
    auto moments = [&](int kind, float& m, float& k) {
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
      for_chunks<LPR, CH, kEnd>(d, sub, active, [&](int c, auto at) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float t = at.has(e) ? v[c][e] - m : 0.f;
          q[0] = fmaf(t, t, q[0]);
        }
      });
      row_sum<LPR>(q, red, turn);
      k = 1.f / sqrtf(q[0] * inv_d + a.eps);
    };
    moments(a.post, mean_p, rstd_p);
    for_chunks<LPR, CH, kEnd>(d, sub, active, [&](int c, auto at) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float u = fmaf((v[c][e] - mean_p) * rstd_p, wp[c].get(e), bp[c].get(e));
        v[c][e] = at.has(e) ? fmaf(scale[c][e], u, res[c][e]) : 0.f;
      }
    });
    const Window wr = window<TR>(a.r, row * d), wh = window<TB>(a.h, row * d);
    for_chunks<LPR, CH, kEnd>(d, sub, active, [&](int c, auto at) { at.template store<TR, true>(wr, v[c]); });
    moments(a.pre, mean, rstd);
    for_chunks<LPR, CH, kEnd>(d, sub, active, [&](int c, auto at) {
      float o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = fmaf((v[c][e] - mean) * rstd, w[c].get(e), b[c].get(e));
      if (a.past) at.template store<TB, true>(wh, o);
      else at.template store<TB>(wh, o);
    });
    if (a.stats && active && threadIdx.x % LPR == 0)
      *reinterpret_cast<float4*>(a.stats + 4 * (row + sub)) = make_float4(mean_p, rstd_p, mean, rstd);
  }
}

// Rows of one segment (the tokens of a gate row) in `pieces` ranges, one workgroup each; its groups walk the range in
// turn and keep their column sums in registers, the next row on its way while this one is worked on.  65 536 rows of 768 bf16, everything on, 121 us:
// 5.0 TB/s, as a large copy, but less than the 7.1 that the update of the weights reaches, so that memory is not all that bounds it; two
// wavefronts a SIMD are what its 172 registers leave.  2784 of 512 7.8 us, 2002 of 2048 fp32 18.4 us.  The instances of fp32 blocks beyond 6144
// channels, and of bf16 blocks with a fp32 residual whose rows do not fill 512 lanes of 16, keep 4 to 21 registers of a lane in scratch memory.
template <typename TR, typename TB, int LPR, int CH, End kEnd>
__global__ __launch_bounds__(threads_of<LPR>()) void block_norm_bwd_kernel(NormArgs a) {
  constexpr int T = threads_of<LPR>(), G = T / LPR;
  __shared__ float red[LPR > 64 ? 2 * LPR / 64 : 1][2];
  __shared__ float sums[G > 1 ? 4 : 1][G > 1 ? G : 1][G > 1 ? LPR * CH * 4 : 1];
  int n;
  if (!vd_count(a.n_dev, a.n, n, a.status)) return;
  const int segment = blockIdx.x / a.pieces, piece = blockIdx.x - segment * a.pieces, d = a.d;
  const long long seg_rows = a.gates > 1 ? n : (long long)a.B * n;
  const long long chunk = (seg_rows + a.pieces - 1) / a.pieces;
  const long long first = segment * seg_rows;
  const long long r0 = first + min(seg_rows, piece * chunk), r1 = first + min(seg_rows, (piece + 1) * chunk);
  const int sub = sub_group<LPR>();
  const float inv_d = 1.f / (float)d;
  int turn = 0;

  Unit<TR> dr[CH], r[CH];
  Unit<TB> dh[CH], f[CH];
  raw4 st;
  auto fetch = [&](long long row) {
    const bool active = LPR >= 64 || row + sub < r1;
    const Window wdr = window<TR>(a.dr, row * d), wr = window<TR>(a.r_in, row * d), wdh = window<TB>(a.dh, row * d),
                 wf = window<TB>(a.f, row * d), ws = window<float>(a.stats, row * 4);
    st = __builtin_amdgcn_raw_buffer_load_b128(ws, active ? 16 * sub : kOutside, 0, 0);
    for_chunks<LPR, CH, kEnd>(d, sub, active, [&](int c, auto at) {
      at.load(dr[c], wdr);
      at.load(dh[c], wdh);
      at.load(r[c], wr);
      at.load(f[c], wf);
    });
  };
  float w[CH][4], gq[CH][4];               // weight of pre; beta g wp
  long long row = r0 + first_group<LPR>();
  {
    const Window ww = window<TB>(a.w, 0), wwp = window<TB>(a.wp, 0), wg = window<TB>(a.gate, a.gates > 1 ? (long long)segment * d : 0);
    Unit<TB> uw[CH], up[CH], ug[CH];
    for_chunks<LPR, CH, kEnd>(d, 0, true, [&](int c, auto at) {
      at.load(uw[c], ww);
      at.load(up[c], wwp);
      at.load(ug[c], wg);
    });
    if (row < r1) fetch(row);
    for_chunks<LPR, CH, kEnd>(d, 0, true, [&](int c, auto at) {
      at.trim(uw[c]);
      at.trim(up[c]);
      at.trim(ug[c]);
      if (!a.w) uw[c].fill(1.f);
      if (!a.wp) up[c].fill(1.f);
      if (!a.gate) ug[c].fill(1.f);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        w[c][e] = uw[c].get(e);
        gq[c][e] = at.has(e) ? a.beta * ug[c].get(e) * up[c].get(e) : 0.f;
      }
    });
  }
  float t0[CH][4] = {}, t1[CH][4] = {}, s0[CH][4] = {}, s1[CH][4] = {};
  for (; row < r1; row += G) {
    const bool active = LPR >= 64 || row + sub < r1;
    const bool there = a.stats != nullptr;
    const float mean_p = __uint_as_float(st[0]), rstd_p = there ? __uint_as_float(st[1]) : 1.f, mean = __uint_as_float(st[2]),
                rstd = __uint_as_float(st[3]);
    float D[CH][4], fh[CH][4];
    {
      float hat[CH][4], t[CH][4], s[2] = {0.f, 0.f};
      for_chunks<LPR, CH, kEnd>(d, sub, active, [&](int c, auto at) {
        at.trim(dr[c]);
        at.trim(dh[c]);
        at.trim(r[c]);
        at.trim(f[c]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {            // (past the end all of these are zero)
          const float g = dh[c].get(e);
          D[c][e] = dr[c].get(e);
          fh[c][e] = at.has(e) ? (f[c].get(e) - mean_p) * rstd_p : 0.f;
          hat[c][e] = at.has(e) ? (r[c].get(e) - mean) * rstd : 0.f;
          t[c][e] = w[c][e] * g;
          s[0] += t[c][e];
          s[1] = fmaf(t[c][e], hat[c][e], s[1]);
          t0[c][e] += g;
          t1[c][e] = fmaf(g, hat[c][e], t1[c][e]);
        }
      });
      if (row + G < r1) fetch(row + G);
      if (a.dh) {
        row_sum<LPR>(s, red, turn);
        const float m0 = a.pre == VARDROP_NORM_LAYER ? s[0] * inv_d : 0.f, m1 = s[1] * inv_d;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) D[c][e] = fmaf(rstd, t[c][e] - m0 - hat[c][e] * m1, D[c][e]);
      }
    }
    const Window wdx = window<TR>(a.dx, row * d), wdf = window<TB>(a.df, row * d);
    float q[2] = {0.f, 0.f};
    for_chunks<LPR, CH, kEnd>(d, sub, active, [&](int c, auto at) {
      float o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        o[e] = a.alpha * D[c][e];
        s0[c][e] += D[c][e];
        s1[c][e] = fmaf(D[c][e], fh[c][e], s1[c][e]);
        D[c][e] = at.has(e) ? D[c][e] * gq[c][e] : 0.f;
        q[0] += D[c][e];
        q[1] = fmaf(D[c][e], fh[c][e], q[1]);
      }
      at.template store<TR, true>(wdx, o);
    });
    // Without the norm, beta g D as it is: 0 in the place of a sum would make NaN of the elements beside one that is not finite.
    if (a.post != VARDROP_NORM_NONE) {
      row_sum<LPR>(q, red, turn);
      const float m0 = a.post == VARDROP_NORM_LAYER ? q[0] * inv_d : 0.f, m1 = q[1] * inv_d;
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) D[c][e] = rstd_p * (D[c][e] - m0 - fh[c][e] * m1);
    }
    for_chunks<LPR, CH, kEnd>(d, sub, active, [&](int c, auto at) { at.template store<TB>(wdf, D[c]); });
  }
  if (!a.part) return;
  // column sums of the groups, in their order
  float* part = a.part + (long long)blockIdx.x * 4 * d;
  auto leave = [&](int which, float (&v)[CH][4]) {
    if (G == 1) {
      const Window wp = window<float>(part, (long long)which * d);
      for_chunks<LPR, CH, kEnd>(d, 0, true, [&](int c, auto at) { at.template store<float>(wp, v[c]); });
    } else {
#pragma unroll
      for (int c = 0; c < CH; ++c)
        *reinterpret_cast<float4*>(&sums[which][threadIdx.x / LPR][(c * LPR + threadIdx.x % LPR) * kVec]) =
            make_float4(v[c][0], v[c][1], v[c][2], v[c][3]);
    }
  };
  leave(0, t0);
  leave(1, t1);
  leave(2, s0);
  leave(3, s1);
  if (G == 1) return;
  __syncthreads();
  for (int i = threadIdx.x; i < 4 * d; i += T) {
    const int which = i / d, col = i - which * d;
    float s = 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g) s += sums[which][g][col];
    part[i] = s;
  }
}

// The vector gradients from the pieces' column sums.  A workgroup takes 16 columns (64 bytes of a sum) and 64 pieces at a time, so
// that it has all it reads under way in one round (6.2-7.3 us for 512 pieces of 768 columns and eight gate rows, 18.6 with 64 columns a workgroup
// and three rounds and more; 4.2 us is the least; the sums are read from memory twice, by different dies); blockIdx.y 0: db, dw; 1: dbp, dwp (every piece weighted with its
// gate row) and the gradient of a single gate row; 2 + g: gate row g of several.
constexpr int kVectorCols = 16;
__device__ inline float to_float(float v) { return v; }
__device__ inline float to_float(bf16_t v) { return bf2f(v); }
template <typename TB>
__global__ __launch_bounds__(1024) void block_norm_vectors_kernel(NormArgs a, float* dw, float* db, float* dwp, float* dbp,
                                                                  float* dgate, int segments) {
  constexpr int R = 1024 / kVectorCols, N = 8;     // pieces side by side; rounds in flight
  __shared__ float red[2][R][kVectorCols + 1];
  const int j = threadIdx.x % kVectorCols, k = threadIdx.x / kVectorCols, what = blockIdx.y, d = a.d;
  const bool one_gate = what == 1 && a.gates == 1 && dgate;
  if ((what == 0 && !dw && !db) || (what == 1 && !dwp && !dbp && !one_gate)) return;
  int n;
  if (!vd_count(a.n_dev, a.n, n)) return;
  const int col = blockIdx.x * kVectorCols + j, c = min(col, d - 1);
  int p0 = 0, p1 = segments * a.pieces;
  if (what >= 2) {
    p0 = (what - 2) * a.pieces;
    p1 = p0 + a.pieces;
  }
  const bool weighted = what == 1 && a.gates > 1;
  const float* src = a.part + (what == 0 ? 0 : 2 * d) + c;
  auto param = [&](const void* p, long long at, float none) {
    return p ? to_float(((const TB*)p)[at]) : none;
  };
  // what the results are multiplied with is asked for before the sums
  const float gate = what == 1 && a.gates == 1 ? param(a.gate, c, 1.f) : 1.f;
  const float wp = what >= 1 ? param(a.wp, c, 1.f) : 1.f, bp = what >= 1 ? param(a.bp, c, 0.f) : 0.f;
  float s0 = 0.f, s1 = 0.f;
  for (int p = p0 + k; p < p1; p += N * R) {
    float v0[N], v1[N], g[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = min(p + i * R, p1 - 1);
      v0[i] = src[(long long)at * 4 * d];
      v1[i] = src[(long long)at * 4 * d + d];
      g[i] = weighted ? param(a.gate, (long long)(at / a.pieces) * d + c, 1.f) : 1.f;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float t = p + i * R < p1 ? g[i] : 0.f;
      s0 = p + i * R < p1 ? fmaf(t, v0[i], s0) : s0;
      s1 = p + i * R < p1 ? fmaf(t, v1[i], s1) : s1;
    }
  }
  // 64 sums of a column: sixteen threads take four each, then one adds those
  red[0][k][j] = s0;
  red[1][k][j] = s1;
  __syncthreads();
  if (k < 16) {
#pragma unroll
    for (int i = 1; i < R / 16; ++i) {
      s0 += red[0][k + 16 * i][j];
      s1 += red[1][k + 16 * i][j];
    }
    red[0][k][j] = s0;
    red[1][k][j] = s1;
  }
  __syncthreads();
  if (k != 0 || col >= d) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) {
    s0 += red[0][i][j];
    s1 += red[1][i][j];
  }
  if (what == 0) {
    if (db) db[col] = s0;
    if (dw) dw[col] = s1;
  } else if (what == 1) {
    const float f = a.beta * gate;
    if (dbp) dbp[col] = f * s0;
    if (dwp) dwp[col] = f * s1;
  }
  // (no product with a bias that is not there: 0 times an infinite S0 is NaN)
  if (what >= 2 || one_gate) dgate[(long long)(what >= 2 ? what - 2 : 0) * d + col] = a.beta * (a.bp ? fmaf(wp, s1, bp * s0) : wp * s1);
}

// ---------------------------------------------------------------- host side
struct Shape {
  int lanes, chunks;
  End end;
};
// Lanes and chunks of a row of d elements: as many lanes as hold it with one chunk each, up to a wavefront; then up to four chunks;
// then several wavefronts.  All chunks but the last are whole.
Shape shape_of(int d) {
  const int lanes = d <= 64 ? 16 : d <= 128 ? 32 : d <= 1024 ? 64 : d <= 4096 ? 256 : 512;
  const int chunks = vd_ceil_div(d, lanes * kVec);
  return {lanes, chunks, d < kVec ? kTiny : d % kVec ? kRagged : d == lanes * kVec * chunks ? kWhole : kCut};
}
#define VD_NORM_SHAPES(X) \
  X(16, 1) X(32, 1) X(64, 1) X(64, 2) X(64, 3) X(64, 4) X(256, 2) X(256, 3) X(256, 4) X(512, 3) X(512, 4)

// Ranges of rows per segment: 512 over all segments, 256 for rows wider than 1024, whose column sums (32 d bytes a range, written and read
// again) weigh more; rounded up in every segment (five gate rows have 515), and no more than one for eight rows or two for every group of
// lanes (9 rows have two).  512 are two workgroups a compute unit where registers allow them: fp32 of 769 to 1024 and of 3073 to 4096
// channels, and ragged widths of these with a fp32 residual alone, have one.  Both launches with 256 / 512 / 1024 ranges, us: 390 625 x 64 bf16 84 /
// 65 / 68, 97 656 x 256 82 / 64 / 69, 77 881 x 321 86 / 78 / 79, 48 828 x 512 64.1 / 65.9 / 67.7, 39 062 x 640 69.7 / 67.2 / 67.2 (with eight gate rows
// 67.9 / 73.4 / 69.6), 24 414 x 1024 67.6 / 68.0 / 69.2, fp32 126 / 125 / 127; 12 207 x 2048 67.6 / 70.2 / 77.7, 6103 x 4096 70.5 / 78.2 / 84.4, fp32
// 131 / 136 / 141.  Few rows: 6016 x 512 15.0 / 15.8 / 17.6; 2784 x 512 with 128 / 256 / 348 ranges 13.7 / 11.7 / 12.2, x 1024 17.6 / 15.6 / 16.7, fp32
// 19.3 / 19.0 / 22.0; 2002 x 2048 fp32 with 64 / 128 / 252 39.9 / 27.9 / 24.7.
int pieces_of(int B, int n, int d, int gates) {
  const int segments = gates > 1 ? gates : 1;
  const Shape s = shape_of(d);
  const int groups = (s.lanes > 256 ? s.lanes : 256) / s.lanes;
  const long long rows = gates > 1 ? n : (long long)B * n;
  const int least = 2 * groups > 8 ? 2 * groups : 8;
  const long long most = (rows + least - 1) / least;
  long long p = vd_ceil_div(d > 1024 ? 256 : 512, segments);
  if (p > most) p = most;
  return p < 1 ? 1 : (int)p;
}

// Workgroups of the forward: 4096 at most, all with the same number of turns but for the last ones; a wavefront with several rows asks for
// the vectors once and has the next row on its way.  One row for every group of lanes -> up to 1024, 2048, 4096 workgroups, us: 390 625 x 64 bf16
// 55.4 -> 43.5, 46.7, 41.3; 97 656 x 256 50.1 -> 45.3, 42.8, 40.9; 48 828 x 512 45.7 -> 39.7, 40.1, 38.3; 12 207 x 2048 45.9 -> 39.7, 41.1, 39.5.
unsigned blocks_of(long long rows, int groups) {
  const long long b = (rows + groups - 1) / groups, turns = (b + 4095) / 4096;
  return (unsigned)((b + turns - 1) / turns);
}

template <bool kBackward, typename TR, typename TB>
int launch(vardrop_ctx* ctx, const NormArgs& a, long long groups_of_rows, hipStream_t s) {
  const Shape sh = shape_of(a.d);
  VdTimer timer(ctx, kBackward ? VARDROP_K_BLOCK_NORM_BWD : VARDROP_K_BLOCK_NORM_FWD, s);
#define VD_CASE_END(L, C, F)                                                                                       \
  if (sh.lanes == L && sh.chunks == C && sh.end == F) {                                                            \
    constexpr int T = threads_of<L>();                                                                             \
    if (kBackward) VD_KERNEL(ctx, (block_norm_bwd_kernel<TR, TB, L, C, F>), dim3((unsigned)groups_of_rows), dim3(T), 0, s, a); \
    else VD_KERNEL(ctx, (block_norm_fwd_kernel<TR, TB, L, C, F>), dim3(blocks_of(groups_of_rows, T / L)), dim3(T), 0, s, a); \
  }
#define VD_CASE(L, C) VD_CASE_END(L, C, kWhole) VD_CASE_END(L, C, kCut) VD_CASE_END(L, C, kRagged)
  VD_NORM_SHAPES(VD_CASE)
  VD_CASE_END(16, 1, kTiny)
#undef VD_CASE
#undef VD_CASE_END
  VD_LAUNCH_CHECK(ctx);
  return VARDROP_OK;
}

template <bool kBackward>
int launch_types(vardrop_ctx* ctx, const NormArgs& a, int res_dtype, int dtype, long long count, hipStream_t s) {
  if (dtype == VARDROP_F32) return launch<kBackward, float, float>(ctx, a, count, s);
  if (res_dtype == VARDROP_F32) return launch<kBackward, float, bf16_t>(ctx, a, count, s);
  return launch<kBackward, bf16_t, bf16_t>(ctx, a, count, s);
}

// What is read again only after the block between (r, dx) is written past the caches: as dirty lines of the L2s it is written back
// at the kernel's end, when nothing else runs.  h and df are what the next kernel reads; h goes past from this size on.  us, all
// kept -> r and dx past -> all past: forward of 27 584 x 512 (fp32 residual, 28 MB of h) 35.0 -> 33.6 -> 30.7, backward of 2002 x 2048 fp32 27.3 -> 24.5
// -> 22.8, of 65 536 x 768 131.3 -> 130.1 -> 129.6; norm, attention and back, 32 x 862 tokens of 512 545 each, 8 x 2000 of 768 778 -> 778 -> 780, 32 x 87
// of 512 66.3 -> 65.6 -> 65.6, but 32 x 321 of 512 (10.5 MB) 193 -> 194 -> 198.
constexpr long long kPastCaches = 16 << 20;
bool is_past(int B, int n, int d, int dtype) { return (long long)B * n * d * (dtype == VARDROP_F32 ? 4 : 2) >= kPastCaches; }

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
  a.past = is_past(B, n, d, dtype);
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
  // (f is read wherever it is given, also where neither a post norm nor a gate's gradient needs it: a sixth of the bytes there)
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
  const dim3 grid((unsigned)vd_ceil_div(d, kVectorCols), (unsigned)(dgate && gates > 1 ? 2 + gates : (dgate || dwp || dbp) ? 2 : 1));
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
