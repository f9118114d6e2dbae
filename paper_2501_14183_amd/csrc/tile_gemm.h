// Matrix products whose results are worked on before they are stored: the feed-forward block (ffn.hip) and the 8-bit integer
// products (int8.hip).
//
//   C = A B, tiles of BM x 128, four wavefronts of (BM / 2) x 64 each; fp32 (bf16 operands) or int32 (8-bit operands) sums.
//
// Both operands are copied straight into LDS, two or three stages deep, one barrier a stage; every wavefront copies its share and
// computes.  A stage is 128 bytes of k for an operand that is contiguous along k ([M][K], [N][K]), 64 k-rows for a bf16
// operand that is contiguous the other way ([K][M], [K][N]; read through the transposing LDS read).  In bytes both types are
// the same kernel: v_mfma_f32_32x32x16_bf16 and v_mfma_i32_32x32x32_i8 take 16 bytes of k a lane.
// What lies outside a matrix (rows past M or N, k past K where K is a count of tokens) lies outside the range of its buffer
// descriptor, whose loads give zero: there are no masks, and memory behind a tensor is not read.
// The sums go through LDS once, by which each lane gets eight neighbouring columns of a row: what is done to a row there (Epi)
// needs no other layout, its stores are whole lines, and its columns' constants are loaded once a tile.
#ifndef VARDROP_TILE_GEMM_H
#define VARDROP_TILE_GEMM_H
#include "bf16_mfma.h"

namespace {

typedef int intx16 __attribute__((ext_vector_type(16)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

struct TileArgs {
  const void *A, *B;
  long long lda, ldb;          // bytes from one row to the next
  int M, N, K;                 // elements; K of a k-contiguous operand is whole stages
  int slices;                  // > 1: cut along k, one workgroup a slice
  // device-side token count (see vd_count): M (n_role 0) or K (n_role 1) is n_mul * n
  const int32_t* n_dev;
  int32_t* status;
  int n_max, n_mul, n_role;
};

constexpr int kTileThreads = 256, kTileN = 128, kTilePitch = 64 * 4 + 16;

template <int BM, int NS>
constexpr int tile_lds() {
  constexpr int ring = NS * (BM + kTileN) * 128, out = 4 * 32 * kTilePitch;
  return ring > out ? ring : out;
}

// Descriptor of the memory from p on, `bytes` long (none: every load gives zero).
__device__ inline copy_src tile_source(const void* p, long long bytes) {
  const long long most = 0xfffffff0ll;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)(uint32_t)(bytes < 0 ? 0 : (bytes > most ? most : bytes)), 0x00020000);
}
// (keeps uses of an LDS read behind the wait before this)
__device__ inline void tie(Frag& f) { asm volatile("" : "+v"(f.q)); }

__device__ inline uint32_t sum_bits(float v) { return __float_as_uint(v); }
__device__ inline uint32_t sum_bits(int v) { return (uint32_t)v; }
template <bool I8> struct TileSum { typedef floatx16 type; };
template <> struct TileSum<true> { typedef intx16 type; };
__device__ inline floatx16 tile_mfma(const Frag& a, const Frag& b, floatx16 c) { return mfma(a, b, c); }
__device__ inline intx16 tile_mfma(const Frag& a, const Frag& b, intx16 c) {
  return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(intx4, a.q), __builtin_bit_cast(intx4, b.q), c, 0, 0, 0);
}

// AKC, BKC: operand contiguous along k.  Epi: `columns(n, live)` once, then `row(slice, m, live, v)` with eight sums of row m for
// every row of the tile; `live` is false outside the result, lanes of one row and block of 32 columns come together.
template <bool I8, bool AKC, bool BKC, int BM, int NS, typename Epi>
__global__ __launch_bounds__(kTileThreads, 2) void tile_gemm_kernel(TileArgs g, typename Epi::Args args) {
  static_assert(!I8 || (AKC && BKC), "8-bit operands are contiguous along k");
  typedef typename TileSum<I8>::type Sum;
  constexpr int BN = kTileN, MI = BM / 64, A_BYTES = BM * 128, STAGE = A_BYTES + BN * 128;
  constexpr int IA = A_BYTES / 4096, IB = BN * 128 / 4096, LPS = IA + IB;        // 1 KB copies per wavefront and stage
  constexpr int OPK = (AKC ? MI : 2 * MI) + (BKC ? 2 : 4);                       // LDS reads per step
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  int M = g.M, K = g.K;
  if (g.n_dev) {
    int n;
    if (!vd_count(g.n_dev, g.n_max, n, g.status)) return;
    if (g.n_role == 0) M = g.n_mul * n;
    else K = g.n_mul * n;
  }
  const int gx = (g.N + BN - 1) / BN, gy = (M + BM - 1) / BM, total = gx * gy * g.slices;
  if ((int)blockIdx.x >= total) return;                 // (a grid sized for the bound of a device-side count)
  // tiles in the order n fastest, then m, then slice: a die's range shares its rows of A
  const int t = xcd_contiguous(blockIdx.x, total);
  const int n0 = t % gx * BN, m0 = t / gx % gy * BM, slice = t / (gx * gy);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, half = lane >> 5;
  const int wm = wave >> 1, wn = wave & 1;
  // this slice's stages
  constexpr int ES = I8 ? 1 : 2, KU = 128 / ES;         // bytes of an element, k of a stage
  const int stages = (K + KU - 1) / KU, per = (stages + g.slices - 1) / g.slices, s0 = min(stages, slice * per);
  const int nk = min(stages, s0 + per) - s0;

  // ---- sources: descriptors from the tile's first byte of the slice to the end of the matrix
  const unsigned char* pa = (const unsigned char*)g.A + (AKC ? m0 * g.lda + s0 * 128ll : (long long)s0 * KU * g.lda + m0 * 2ll);
  const unsigned char* pb = (const unsigned char*)g.B + (BKC ? n0 * g.ldb + s0 * 128ll : (long long)s0 * KU * g.ldb + n0 * 2ll);
  const long long ea = AKC ? (M - m0 - 1) * g.lda + (long long)K * ES - s0 * 128ll : (K - s0 * KU - 1) * g.lda + (M - m0) * 2ll;
  const long long eb = BKC ? (g.N - n0 - 1) * g.ldb + (long long)K * ES - s0 * 128ll : (K - s0 * KU - 1) * g.ldb + (g.N - n0) * 2ll;
  const copy_src srcA = tile_source(pa, nk > 0 ? ea : 0), srcB = tile_source(pb, nk > 0 ? eb : 0);
  uint32_t offA[IA], offB[IB];
#pragma unroll
  for (int u = 0; u < IA; ++u) {
    if constexpr (AKC) {
      const int row = (u * 4 + wave) * 8 + (lane >> 3);
      offA[u] = (uint32_t)row * (uint32_t)g.lda + (((lane & 7) ^ swz_kc<64>(row)) * 16);
    } else {
      constexpr int CH = BM / 8;
      const int krow = (u * 4 + wave) * (64 / CH) + lane / CH;
      offA[u] = (uint32_t)krow * (uint32_t)g.lda + ((lane % CH) ^ swz_nc<BM>(krow)) * 16;
    }
  }
#pragma unroll
  for (int u = 0; u < IB; ++u) {
    if constexpr (BKC) {
      const int row = (u * 4 + wave) * 8 + (lane >> 3);
      offB[u] = (uint32_t)row * (uint32_t)g.ldb + (((lane & 7) ^ swz_kc<64>(row)) * 16);
    } else {
      constexpr int CH = BN / 8;
      const int krow = (u * 4 + wave) * (64 / CH) + lane / CH;
      offB[u] = (uint32_t)krow * (uint32_t)g.ldb + ((lane % CH) ^ swz_nc<BN>(krow)) * 16;
    }
  }
  const uint32_t stepA = AKC ? 128u : 64u * (uint32_t)g.lda, stepB = BKC ? 128u : 64u * (uint32_t)g.ldb;
  auto issue = [&](int k, int buf) {
    unsigned char* sp = smem + buf * STAGE + wave * 1024;
#pragma unroll
    for (int u = 0; u < IA; ++u) dma16_buf(srcA, offA[u], k * stepA, sp + u * 4096);
#pragma unroll
    for (int u = 0; u < IB; ++u) dma16_buf(srcB, offB[u], k * stepB, sp + A_BYTES + u * 4096);
  };
  // ---- fragment addresses (LDS bytes relative to a stage): one for every step of a k-contiguous operand (blocks of 32 rows are a
  // fixed distance apart), one for every block of the other kind (steps are)
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
  uint32_t addrA[AKC ? 4 : MI], addrB[BKC ? 4 : 2];
  const int krow = 8 * half + ((lane & 15) >> 2), mn = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  if constexpr (AKC) {
    const int ra = wm * (BM / 2) + col;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) addrA[ks] = lds0 + ra * 128 + (((2 * ks + half) ^ swz_kc<64>(ra)) * 16);
  } else {
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int c = wm * (BM / 2) + i * 32 + mn;
      addrA[i] = lds0 + krow * (BM * 2) + (((c >> 3) ^ swz_nc<BM>(krow)) * 16) + ((c >> 2) & 1) * 8;
    }
  }
  if constexpr (BKC) {
    const int rb = wn * 64 + col;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) addrB[ks] = lds0 + A_BYTES + rb * 128 + (((2 * ks + half) ^ swz_kc<64>(rb)) * 16);
  } else {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int c = wn * 64 + j * 32 + mn;
      addrB[j] = lds0 + A_BYTES + krow * (BN * 2) + (((c >> 3) ^ swz_nc<BN>(krow)) * 16) + ((c >> 2) & 1) * 8;
    }
  }
  Sum acc[MI][2];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;

#pragma unroll
  for (int s = 0; s < NS - 1; ++s)
    if (s < nk) issue(s, s);
  for (int t0 = 0; t0 < nk; t0 += NS) {
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const int k = t0 + s;
      if (k < nk) {
        // stage k has landed once at most NS - 2 younger ones are in flight
        if (NS == 3 && k + 1 < nk) wait_vm<LPS>(); else wait_vm<0>();
        __builtin_amdgcn_s_barrier();       // everyone has seen stage k land and is done with stage k - 1, whose buffer is next
        if (k + NS - 1 < nk) issue(k + NS - 1, (s + NS - 1) % NS);
        const uint32_t so = s * STAGE;
        Frag fa[2][MI], fb[2][2];
#define VD_TILE_READ(KS_, SET)                                                                      \
  {                                                                                                 \
    if constexpr (AKC) {                                                                            \
      const uint32_t p = addrA[AKC ? (KS_) : 0] + so;                                               \
      lds_read16_at<0>(fa[SET][0].q, p);                                                            \
      if constexpr (MI > 1) lds_read16_at<4096>(fa[SET][MI > 1 ? 1 : 0].q, p);                      \
    } else {                                                                                        \
      _Pragma("unroll") for (int i = 0; i < MI; ++i) {                                              \
        lds_read8_tr<(KS_) * 16 * BM * 2>(fa[SET][i].d[0], addrA[i] + so);                          \
        lds_read8_tr<(KS_) * 16 * BM * 2 + 4 * BM * 2>(fa[SET][i].d[1], addrA[i] + so);             \
      }                                                                                             \
    }                                                                                               \
    if constexpr (BKC) {                                                                            \
      const uint32_t p = addrB[BKC ? (KS_) : 0] + so;                                               \
      lds_read16_at<0>(fb[SET][0].q, p);                                                            \
      lds_read16_at<4096>(fb[SET][1].q, p);                                                         \
    } else {                                                                                        \
      _Pragma("unroll") for (int j = 0; j < 2; ++j) {                                               \
        lds_read8_tr<(KS_) * 16 * BN * 2>(fb[SET][j].d[0], addrB[j] + so);                          \
        lds_read8_tr<(KS_) * 16 * BN * 2 + 4 * BN * 2>(fb[SET][j].d[1], addrB[j] + so);             \
      }                                                                                             \
    }                                                                                               \
  }
#define VD_TILE_MFMA(SET, PENDING)                                                                  \
  {                                                                                                 \
    wait_lds_count<PENDING>();                                                                      \
    _Pragma("unroll") for (int i = 0; i < MI; ++i) tie(fa[SET][i]);                                 \
    tie(fb[SET][0]);                                                                                \
    tie(fb[SET][1]);                                                                                \
    _Pragma("unroll") for (int i = 0; i < MI; ++i)                                                  \
      _Pragma("unroll") for (int j = 0; j < 2; ++j) acc[i][j] = tile_mfma(fb[SET][j], fa[SET][i], acc[i][j]); \
    __builtin_amdgcn_sched_barrier(0);                                                              \
  }
        VD_TILE_READ(0, 0)
        VD_TILE_READ(1, 1)
        VD_TILE_MFMA(0, OPK)
        VD_TILE_READ(2, 0)
        VD_TILE_MFMA(1, OPK)
        VD_TILE_READ(3, 1)
        VD_TILE_MFMA(0, OPK)
        VD_TILE_MFMA(1, 0)
#undef VD_TILE_READ
#undef VD_TILE_MFMA
      }
    }
  }
  // ---- 32 rows x 64 columns of a wavefront at a time through its own part of LDS.  acc[i][j] element 4 q + e is row i * 32 + col,
  // column j * 32 + 8 q + 4 half + e; back comes row (lane >> 3) + 8 u, columns 8 (lane & 7) ..
  __syncthreads();                          // every wavefront is done reading the last stage
  unsigned char* own = smem + wave * (32 * kTilePitch);
  const int n = n0 + wn * 64 + 8 * (lane & 7);
  Epi epi{args};
  epi.columns(n, g.N);
#pragma unroll
  for (int i = 0; i < MI; ++i) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        u32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = sum_bits(acc[i][j][4 * q + e]);
        *reinterpret_cast<u32x4*>(own + col * kTilePitch + (j * 32 + 8 * q + 4 * half) * 4) = v;
      }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int row = 8 * u + (lane >> 3), m = m0 + wm * (BM / 2) + i * 32 + row;
      const u32x4 lo = *reinterpret_cast<const u32x4*>(own + row * kTilePitch + (lane & 7) * 32);
      const u32x4 hi = *reinterpret_cast<const u32x4*>(own + row * kTilePitch + (lane & 7) * 32 + 16);
      float v[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (I8) {
          v[e] = (float)(int)lo[e];
          v[4 + e] = (float)(int)hi[e];
        } else {
          v[e] = __uint_as_float(lo[e]);
          v[4 + e] = __uint_as_float(hi[e]);
        }
      }
      epi.row(slice, m, n, m < M && n < g.N, v);
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
  }
}

template <bool I8, bool AKC, bool BKC, int BM, int NS, typename Epi>
int launch_tile_gemm(vardrop_ctx* ctx, int kid, const TileArgs& g, const typename Epi::Args& epi, hipStream_t s) {
  constexpr int lds = tile_lds<BM, NS>();
  const void* fn = (const void*)tile_gemm_kernel<I8, AKC, BKC, BM, NS, Epi>;
  static int configured_device = -1;        // (a setting of a function on a device)
  if (lds > 65536 && configured_device != ctx->device) {
    VD_HIP(ctx, hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    configured_device = ctx->device;
  }
  const long long grid = (long long)vd_ceil_div(g.N, kTileN) * vd_ceil_div(g.M, BM) * g.slices;
  if (grid >= (1ll << 31)) return VARDROP_EUNSUPPORTED;
  if (grid == 0) return VARDROP_OK;
  {
    VdTimer timer(ctx, kid, s);
    VD_KERNEL(ctx, (tile_gemm_kernel<I8, AKC, BKC, BM, NS, Epi>), dim3((unsigned)grid), dim3(kTileThreads), lds, s, g, epi);
  }
  VD_LAUNCH_CHECK(ctx);
  return VARDROP_OK;
}

}  // namespace
#endif  // VARDROP_TILE_GEMM_H
