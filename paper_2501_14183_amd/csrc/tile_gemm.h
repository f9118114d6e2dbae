// Matrix products whose results are worked on before they are stored: the feed-forward block (ffn.hip) and the 8-bit integer
// products (int8.hip).
//
//   C = A B in tiles of a shape (TileShape); fp32 sums of bf16 operands, int32 sums of 8-bit ones.
//
// Both operands are copied straight into LDS, two to four stages deep, one barrier a stage; every wavefront copies its share and
// multiplies 32 x 32 blocks.  A stage is 64 or 128 bytes of k for an operand that is contiguous along k ([M][K], [N][K]), as many k-rows
// as these bytes hold of bf16 for one that is contiguous the other way ([K][M], [K][N]; read through the transposing LDS read).  In bytes
// both types are the same kernel: v_mfma_f32_32x32x16_bf16 and v_mfma_i32_32x32x32_i8 take 16 bytes of k a lane.
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
  long long planeA, planeB;    // bytes from one part of an operand to the next (Epi::kPartsA, kPartsB)
  int slices;                  // > 1: cut along k, one workgroup a slice
  // device-side token count (see vd_count): M (n_role 0) or K (n_role 1) is n_mul * n
  const int32_t* n_dev;
  int32_t* status;
  int n_max, n_mul, n_role;
};

// Shape of a tile and its workgroup: BM x BN, WR x WC wavefronts, BKB bytes of k a stage (of a k-contiguous operand), NS stages, room for
// PLANES parts of either operand in each.
template <int BM_, int BN_, int WR_, int WC_, int BKB_, int NS_, int PLANES = 1>
struct TileShape {
  static constexpr int BM = BM_, BN = BN_, WR = WR_, WC = WC_, BKB = BKB_, NS = NS_;
  static constexpr int WAVES = WR * WC, THREADS = WAVES * 64;
  static constexpr int MI = BM / WR / 32, NJ = BN / WC / 32;       // 32 x 32 blocks of a wavefront
  static constexpr int PITCH = NJ * 128 + 16;                      // LDS row of 32 x (32 NJ) sums
  static constexpr int A_BYTES = BM * BKB, B_BYTES = BN * BKB, STAGE = PLANES * (A_BYTES + B_BYTES);
  static constexpr int ring = NS * STAGE, out = WAVES * 32 * PITCH, lds = ring > out ? ring : out;
  static constexpr int per_cu = (160 << 10) / lds;                 // workgroups of a compute unit
  static constexpr int simd = per_cu * WAVES / 4 > 0 ? per_cu * WAVES / 4 : 1;
};

typedef TileShape<64, 64, 2, 2, 128, 4> Tile64;
typedef TileShape<128, 128, 2, 2, 128, 2> Tile128;
typedef TileShape<256, 128, 4, 2, 64, 3> TileWide;
typedef TileShape<256, 256, 2, 4, 128, 2> Tile256;
typedef TileShape<64, 64, 2, 2, 64, 3, 3> Parts64;
typedef TileShape<128, 128, 2, 4, 64, 3, 3> Parts128;

// ---- which tile.  What a tile of BM x BN over K (of 2 bytes) costs beside others of its kind, in products of 32 x 32 x 1 of a
// chip whose every place is taken; its start and end cost as much as kEnds of K.
constexpr double kEnds = 250;
struct ShapeCost {
  int BM, BN, places;          // places: workgroups that are resident together on 256 compute units
  double rate;                 // of the largest tile's
};
// Products whose rows are worked on take 256 x 128 as their largest, two workgroups a compute unit: while one is at its end the other
// multiplies.  us, 256 x 256 -> 256 x 128: activation 240 -> 192 (65 536 x 768 x 1536), 103 -> 88 (27 584 x 512 x 2048), its gradient 233 -> 223 and 110 -> 97;
// but dx 137 -> 161 and 53 -> 69.  8-bit products, 128 x 128 -> 256 x 128: 81 -> 72 (27 584 x 512 x 2048), 34.5 -> 28.2 (65 536 x 128 x 768).
// Few rows take 64 x 64, four stages deep: us, 64 x 128 in three -> 64 x 64 in four: activation 8.0 -> 7.3 (2784 x 512 x 512), 7.4 -> 5.8 (300 x 512 x
// 2048), dx there 6.2 -> 5.9 and 12.8 -> 9.5.
constexpr ShapeCost kShapes[3] = {{64, 64, 512, 0.5}, {128, 128, 512, 0.85}, {256, 256, 256, 1.0}};
// Operands in parts: 128 x 128 is the largest whose parts fit three deep.  us, 64 x 64 -> 128 x 128: activation 9.3 -> 18.6 (999 x 321 x 449), 19.7 -> 24.8 (4000 x 512 x
// 512), 26.4 -> 24.5 (6000 x 512 x 512), 56.7 -> 52.0 (12 000 x 256 x 1024).
constexpr ShapeCost kPartShapes[2] = {{64, 64, 512, 0.6}, {128, 128, 256, 1.0}};
constexpr ShapeCost kRowShapes[3] = {{64, 64, 512, 0.5}, {128, 128, 512, 0.93}, {256, 128, 512, 1.0}};
inline double tile_time(const ShapeCost& c, double K) { return c.BM * c.BN / 1024.0 * (K + kEnds) * c.places / 512.0 / c.rate; }
inline long long tiles_of(const ShapeCost& c, long long M, int N) { return (M + c.BM - 1) / c.BM * vd_ceil_div(N, c.BN); }
template <int SHAPES>
inline int product_shape(const ShapeCost (&shapes)[SHAPES], long long T, int N, int K) {
  int best = 0;
  double least = 0;
  for (int i = 0; i < SHAPES; ++i) {
    // (workgroups end at different times: the last round is seldom a whole one longer)
    const double rounds = (double)tiles_of(shapes[i], T, N) / shapes[i].places;
    const double t = (rounds <= 1 ? 1 : rounds + 0.3) * tile_time(shapes[i], K);
    if (i == 0 || t < least) {
      least = t;
      best = i;
    }
  }
  return best;
}
// a call of CALL for the tile of kShapes, or with WIDE = TileWide of kRowShapes
#define VD_BY_SHAPE(SHAPE, CALL, WIDE) ((SHAPE) == 0 ? CALL(Tile64) : (SHAPE) == 1 ? CALL(Tile128) : CALL(WIDE))
#define VD_BY_PARTS(SHAPE, CALL) ((SHAPE) == 0 ? CALL(Parts64) : CALL(Parts128))

// Descriptor of the memory from p on, `bytes` long (none: every load gives zero).
__device__ inline copy_src tile_source(const void* p, long long bytes) {
  const long long most = 0xfffffff0ll;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)(uint32_t)(bytes < 0 ? 0 : (bytes > most ? most : bytes)), 0x00020000);
}
template <int N> struct Int { static constexpr int value = N; };
// waits until at most min(younger, A) * LPS of this wavefront's copies are in flight
template <int A, int LPS>
__device__ __forceinline__ void wait_stages(int younger) {
  if constexpr (A <= 0) {
    wait_vm<0>();
  } else {
    if (younger >= A) wait_vm<A * LPS>();
    else wait_stages<A - 1, LPS>(younger);
  }
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

// sum of the eight bf16 numbers of a fragment
__device__ inline float eight_sum(const Frag& f) {
  float lo = 0.f, hi = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    lo += __uint_as_float(f.w[e] << 16);
    hi += __uint_as_float(f.w[e] & 0xffff0000u);
  }
  return lo + hi;
}

// The end of a tile: 32 rows x 32 NJ columns of a wavefront at a time through its own part of LDS (`smem`: 32 PITCH bytes a wavefront).
// acc[i][j] element 4 q + e is row i * 32 + lane % 32, column j * 32 + 8 q + 4 (lane / 32) + e; back come eight columns a lane, the lanes of
// a row beside each other.
template <typename S, typename Epi, typename Sum>
__device__ __forceinline__ void tile_finish(const Sum (&acc)[S::MI][S::NJ], unsigned char* smem, Epi& epi, int slice, int M, int N, int m0, int n0) {
  constexpr int MI = S::MI, NJ = S::NJ, LPR = NJ * 4, RPS = 64 / LPR;     // lanes of a row, rows of a step
  constexpr bool I8 = __is_same(Sum, intx16);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, half = lane >> 5;
  const int wm = wave / S::WC, wn = wave % S::WC;
  unsigned char* own = smem + wave * (32 * S::PITCH);
  const int n = n0 + wn * (NJ * 32) + 8 * (lane % LPR);
  auto row_of = [&](int i, int u) { return m0 + wm * (MI * 32) + i * 32 + RPS * u + lane / LPR; };
  if constexpr (Epi::kFetch) {
    // what the rows need from memory is on its way while the sums go through LDS
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int u = 0; u < 32 / RPS; ++u) epi.fetch(i * (32 / RPS) + u, row_of(i, u), n, row_of(i, u) < M && n < N);
  }
  epi.columns(n, N);
#pragma unroll
  for (int i = 0; i < MI; ++i) {
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        u32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = sum_bits(acc[i][j][4 * q + e]);
        *reinterpret_cast<u32x4*>(own + col * S::PITCH + (j * 32 + 8 * q + 4 * half) * 4) = v;
      }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int u = 0; u < 32 / RPS; ++u) {
      const int row = RPS * u + lane / LPR, m = row_of(i, u);
      const u32x4 lo = *reinterpret_cast<const u32x4*>(own + row * S::PITCH + (lane % LPR) * 32);
      const u32x4 hi = *reinterpret_cast<const u32x4*>(own + row * S::PITCH + (lane % LPR) * 32 + 16);
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
      epi.row(slice, i * (32 / RPS) + u, m, n, m < M && n < N, v);
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
  }
  if constexpr (Epi::kRowSums != 0) {
    if (!epi.a.sums) return;
    // lanes of the same columns, then the wavefronts above each other
#pragma unroll
    for (int u = LPR; u < 64; u <<= 1)
#pragma unroll
      for (int e = 0; e < 8; ++e) epi.total[e] += __shfl_xor(epi.total[e], u, 64);
    float* all = reinterpret_cast<float*>(smem);
    __syncthreads();
    if (lane < LPR) {
#pragma unroll
      for (int e = 0; e < 8; ++e) all[wm * S::BN + n - n0 + e] = epi.total[e];
    }
    __syncthreads();
    for (int t = threadIdx.x; t < S::BN; t += S::THREADS) {
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < S::WR; ++w) sum += all[w * S::BN + t];
      if (n0 + t < N) epi.a.sums[(long long)(m0 / S::BM) * N + n0 + t] = sum;
    }
  }
}

// AKC, BKC: operand contiguous along k.  Epi: `columns(n, N)` once, then `row(slice, k, m, n, live, v)` with eight sums of row m from
// column n on, for every row of the tile (k counts a wavefront's); `live` is false outside the result, lanes of one row and block of 32 columns come together.
// Epi::kSums (B not k-contiguous): column sums of B, from the fragments that are multiplied.  The tiles above each other share the stages
// among them and their wavefronts above each other the steps, so that none is held up; what one has goes to `sums(piece, n, live, v)`,
// tile_pieces() of them for a column.
// Epi::kRowSums: what `row` adds up over the rows in total[8] goes to a.sums [tiles above each other][N].
// Epi::kPartsA, kPartsB (bf16 operands that stand for fp32 numbers): 3 and 3, both operands in three parts hi + mid + lo, each the nearest
// bf16 number to what the ones before leave; 1 and 3, A in one part; 1 and 1, plain.  A stage holds all parts of its k.  Every product of
// two parts is exact, and of the nine those are added up, the small ones of a step first, that are not below 2^-24 of the whole:
// hi lo, mid mid, lo hi, hi mid, mid hi, hi hi.  (One pair of parts after the other, over all of k, copies and reads each part twice and meets
// six times the barriers: products of 2002 x 512 x 1024 backward 104 us, and not 73; 27 584 x 512 x 2048 in 256 x 256 tiles 1458 and 1453.)
// t: the tile, n fastest, then m, then slice.
template <bool I8, bool AKC, bool BKC, typename S, typename Epi>
__device__ __forceinline__ void tile_gemm(const TileArgs& g, const typename Epi::Args& args, int M, int K, int t) {
  static_assert(!I8 || (AKC && BKC), "8-bit operands are contiguous along k");
  typedef typename TileSum<I8>::type Sum;
  constexpr int BM = S::BM, BN = S::BN, MI = S::MI, NJ = S::NJ, NS = S::NS, A_BYTES = S::A_BYTES, B_BYTES = S::B_BYTES, W = S::WAVES;
  constexpr int PA = Epi::kPartsA, PB = Epi::kPartsB, STAGE = PA * A_BYTES + PB * B_BYTES;
  static_assert(STAGE <= S::STAGE && (PA == 1 || PA == PB), "room for the parts");
  constexpr int BK = S::BKB / 2, KS = S::BKB / 32;                               // k-rows of a stage, steps of a stage
  constexpr int IA = A_BYTES / (1024 * W), IB = B_BYTES / (1024 * W), LPS = PA * IA + PB * IB;   // 1 KB copies per wavefront, part and stage
  constexpr int OPK = PA * (AKC ? MI : 2 * MI) + PB * (BKC ? NJ : 2 * NJ);       // LDS reads per step
  constexpr int OPEN = OPK < 15 ? OPK : 15;                                       // (as many as the counter counts)
  constexpr int CHK = S::BKB / 16, CHA = AKC ? CHK : BM / 8, CHB = BKC ? CHK : BN / 8;    // 16-byte chunks of an LDS row
  static_assert(IA * 1024 * W == A_BYTES && IB * 1024 * W == B_BYTES, "whole copies");
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int gx = (g.N + BN - 1) / BN, gy = (M + BM - 1) / BM;
  const int n0 = t % gx * BN, m0 = t / gx % gy * BM, slice = t / (gx * gy);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, half = lane >> 5;
  const int wm = wave / S::WC, wn = wave % S::WC;
  // this slice's stages
  constexpr int ES = I8 ? 1 : 2, KU = S::BKB / ES;      // bytes of an element, k of a stage
  const int stages = (K + KU - 1) / KU, per = (stages + g.slices - 1) / g.slices, s0 = min(stages, slice * per);
  const int nk = min(stages, s0 + per) - s0;

  // ---- sources: descriptors from the tile's first byte of the slice to the end of the matrix
  const unsigned char* pa = (const unsigned char*)g.A + (AKC ? m0 * g.lda + (long long)s0 * S::BKB : (long long)s0 * KU * g.lda + m0 * 2ll);
  const unsigned char* pb = (const unsigned char*)g.B + (BKC ? n0 * g.ldb + (long long)s0 * S::BKB : (long long)s0 * KU * g.ldb + n0 * 2ll);
  const long long ea = AKC ? (M - m0 - 1) * g.lda + (long long)K * ES - (long long)s0 * S::BKB : (K - s0 * KU - 1) * g.lda + (M - m0) * 2ll;
  const long long eb = BKC ? (g.N - n0 - 1) * g.ldb + (long long)K * ES - (long long)s0 * S::BKB : (K - s0 * KU - 1) * g.ldb + (g.N - n0) * 2ll;
  copy_src srcA[PA], srcB[PB];
#pragma unroll
  for (int p = 0; p < PA; ++p) srcA[p] = tile_source(pa + p * g.planeA, nk > 0 ? ea : 0);
#pragma unroll
  for (int p = 0; p < PB; ++p) srcB[p] = tile_source(pb + p * g.planeB, nk > 0 ? eb : 0);
  uint32_t offA[IA], offB[IB];
#pragma unroll
  for (int u = 0; u < IA; ++u) {
    const int row = (u * W + wave) * (64 / CHA) + lane / CHA;
    const int c = (lane % CHA) ^ (AKC ? swz_kc<BK>(row) : swz_nc<BM>(row));
    offA[u] = (uint32_t)row * (uint32_t)g.lda + c * 16;
  }
#pragma unroll
  for (int u = 0; u < IB; ++u) {
    const int row = (u * W + wave) * (64 / CHB) + lane / CHB;
    const int c = (lane % CHB) ^ (BKC ? swz_kc<BK>(row) : swz_nc<BN>(row));
    offB[u] = (uint32_t)row * (uint32_t)g.ldb + c * 16;
  }
  const uint32_t stepA = AKC ? (uint32_t)S::BKB : BK * (uint32_t)g.lda, stepB = BKC ? (uint32_t)S::BKB : BK * (uint32_t)g.ldb;
  auto issue = [&](int stage, int buf) {
    unsigned char* sp = smem + buf * STAGE + wave * 1024;
#pragma unroll
    for (int p = 0; p < PA; ++p)
#pragma unroll
      for (int u = 0; u < IA; ++u) dma16_buf(srcA[p], offA[u], stage * stepA, sp + p * A_BYTES + u * W * 1024);
#pragma unroll
    for (int p = 0; p < PB; ++p)
#pragma unroll
      for (int u = 0; u < IB; ++u) dma16_buf(srcB[p], offB[u], stage * stepB, sp + PA * A_BYTES + p * B_BYTES + u * W * 1024);
  };
  // ---- fragment addresses (LDS bytes relative to a stage): one for every step of a k-contiguous operand (blocks of 32 rows are a
  // fixed distance apart), one for every block of the other kind (steps are)
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
  uint32_t addrA[AKC ? KS : MI], addrB[BKC ? KS : NJ];
  const int krow = 8 * half + ((lane & 15) >> 2), mn = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  if constexpr (AKC) {
    const int ra = wm * (MI * 32) + col;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) addrA[ks] = lds0 + ra * S::BKB + (((2 * ks + half) ^ swz_kc<BK>(ra)) * 16);
  } else {
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int c = wm * (MI * 32) + i * 32 + mn;
      addrA[i] = lds0 + krow * (BM * 2) + (((c >> 3) ^ swz_nc<BM>(krow)) * 16) + ((c >> 2) & 1) * 8;
    }
  }
  if constexpr (BKC) {
    const int rb = wn * (NJ * 32) + col;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) addrB[ks] = lds0 + PA * A_BYTES + rb * S::BKB + (((2 * ks + half) ^ swz_kc<BK>(rb)) * 16);
  } else {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int c = wn * (NJ * 32) + j * 32 + mn;
      addrB[j] = lds0 + PA * A_BYTES + krow * (BN * 2) + (((c >> 3) ^ swz_nc<BN>(krow)) * 16) + ((c >> 2) & 1) * 8;
    }
  }
  Sum acc[MI][NJ];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;

  float csum[NJ];
  int next_sum = m0 / BM;
#pragma unroll
  for (int j = 0; j < NJ; ++j) csum[j] = 0.f;
#pragma unroll
  for (int s = 0; s < NS - 1; ++s)
    if (s < nk) issue(s, s);
  for (int t0 = 0; t0 < nk; t0 += NS) {
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const int k = t0 + s;
      if (k < nk) {
        wait_stages<NS - 2, LPS>(nk - 1 - k);     // stage k has landed once at most NS - 2 younger ones are in flight
        __builtin_amdgcn_s_barrier();             // everyone has seen it land and is done with stage k - 1, whose buffer is next
        if (k + NS - 1 < nk) issue(k + NS - 1, (s + NS - 1) % NS);
        const uint32_t so = s * STAGE;
        Frag fa[2][PA][MI], fb[2][PB][NJ];
        auto read_part = [&](auto step, auto part, int set) {
          constexpr int ks = decltype(step)::value, p = decltype(part)::value;
          if constexpr (p < PA) {
            Frag(&f)[MI] = fa[set][p < PA ? p : 0];
            if constexpr (AKC) {
              const uint32_t at = addrA[AKC ? ks : 0] + so;
              lds_read16_at<p * A_BYTES>(f[0].q, at);
              if constexpr (MI > 1) lds_read16_at<p * A_BYTES + 32 * S::BKB>(f[MI > 1 ? 1 : 0].q, at);
              if constexpr (MI > 2) lds_read16_at<p * A_BYTES + 64 * S::BKB>(f[MI > 2 ? 2 : 0].q, at);
              if constexpr (MI > 3) lds_read16_at<p * A_BYTES + 96 * S::BKB>(f[MI > 3 ? 3 : 0].q, at);
            } else {
#pragma unroll
              for (int i = 0; i < MI; ++i) {
                lds_read8_tr<p * A_BYTES + ks * 16 * BM * 2>(f[i].d[0], addrA[i] + so);
                lds_read8_tr<p * A_BYTES + ks * 16 * BM * 2 + 4 * BM * 2>(f[i].d[1], addrA[i] + so);
              }
            }
          }
          if constexpr (p < PB) {
            Frag(&f)[NJ] = fb[set][p < PB ? p : 0];
            if constexpr (BKC) {
              const uint32_t at = addrB[BKC ? ks : 0] + so;
              lds_read16_at<p * B_BYTES>(f[0].q, at);
              if constexpr (NJ > 1) lds_read16_at<p * B_BYTES + 32 * S::BKB>(f[NJ > 1 ? 1 : 0].q, at);
            } else {
#pragma unroll
              for (int j = 0; j < NJ; ++j) {
                lds_read8_tr<p * B_BYTES + ks * 16 * BN * 2>(f[j].d[0], addrB[j] + so);
                lds_read8_tr<p * B_BYTES + ks * 16 * BN * 2 + 4 * BN * 2>(f[j].d[1], addrB[j] + so);
              }
            }
          }
        };
        auto read = [&](auto step, int set) {
          read_part(step, Int<0>{}, set);
          read_part(step, Int<1>{}, set);
          read_part(step, Int<2>{}, set);
        };
        const bool summing = Epi::kSums && k == next_sum;
        if (summing) next_sum += gy;
        auto multiply = [&](auto pending, int set, int ks) {
          wait_lds_count<decltype(pending)::value>();
#pragma unroll
          for (int p = 0; p < PA; ++p)
#pragma unroll
            for (int i = 0; i < MI; ++i) tie(fa[set][p][i]);
#pragma unroll
          for (int p = 0; p < PB; ++p)
#pragma unroll
            for (int j = 0; j < NJ; ++j) tie(fb[set][p][j]);
          // pairs of parts whose places add up to 2, 1, 0
#pragma unroll
          for (int both = PB - 1; both >= 0; --both)
#pragma unroll
            for (int p = 0; p <= both && p < PA; ++p)
#pragma unroll
              for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NJ; ++j) acc[i][j] = tile_mfma(fb[set][both - p][j], fa[set][p][i], acc[i][j]);
          if constexpr (Epi::kSums) {
            if (summing && ks % S::WR == wm) {
#pragma unroll
              for (int p = PB - 1; p >= 0; --p)
#pragma unroll
                for (int j = 0; j < NJ; ++j) csum[j] += eight_sum(fb[set][p][j]);
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        };
        read(Int<0>{}, 0);
        read(Int<1>{}, 1);
        multiply(Int<OPEN>{}, 0, 0);
        if constexpr (KS == 4) {
          read(Int<2>{}, 0);
          multiply(Int<OPEN>{}, 1, 1);
          read(Int<3>{}, 1);
          multiply(Int<OPEN>{}, 0, 2);
        }
        multiply(Int<0>{}, 1, KS - 1);
      }
    }
  }
  __syncthreads();                                // every wavefront is done reading the last stage
  Epi epi{args};
  if constexpr (Epi::kSums) {
    static_assert(KS % S::WR == 0, "steps for every row of wavefronts");
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const float sum = csum[j] + __shfl_xor(csum[j], 32, 64);
      const int n = n0 + wn * (NJ * 32) + j * 32 + col;
      epi.sums((slice * gy + m0 / BM) * S::WR + wm, n, lane < 32 && n < g.N, sum);
    }
  }
  tile_finish<S, Epi>(acc, smem, epi, slice, M, g.N, m0, n0);
}

// products of two parts that one of fp32 numbers takes
template <typename Epi> constexpr int tile_pairs() { return Epi::kPartsA > 1 ? 6 : Epi::kPartsB; }
// A product's dimensions with a device-side count resolved; false: the count is invalid.
__device__ __forceinline__ bool tile_dims(const TileArgs& g, int& M, int& K) {
  M = g.M;
  K = g.K;
  if (!g.n_dev) return true;
  int n;
  if (!vd_count(g.n_dev, g.n_max, n, g.status)) return false;
  (g.n_role == 0 ? M : K) = g.n_mul * n;
  return true;
}
template <typename S>
inline int tile_pieces(const TileArgs& g) { return g.slices * ((g.M + S::BM - 1) / S::BM) * S::WR; }
template <typename S>
__host__ __device__ inline long long tile_count(const TileArgs& g, int M) {
  return (long long)((g.N + S::BN - 1) / S::BN) * ((M + S::BM - 1) / S::BM) * g.slices;
}

template <bool I8, bool AKC, bool BKC, typename S, typename Epi>
__global__ __launch_bounds__(S::THREADS, S::simd) void tile_gemm_kernel(TileArgs g, typename Epi::Args args) {
  int M, K;
  if (!tile_dims(g, M, K)) return;
  const int total = (int)tile_count<S>(g, M);
  if ((int)blockIdx.x >= total) return;           // (a grid sized for the bound of a device-side count)
  // a die's range of the tiles shares its rows of A
  tile_gemm<I8, AKC, BKC, S, Epi>(g, args, M, K, xcd_contiguous(blockIdx.x, total));
}

// Raises the dynamic LDS limit of a kernel on the context's device, which need not be the current one; `configured` remembers the device.
inline int tile_allow_lds(vardrop_ctx* ctx, const void* fn, int lds, int& configured) {
  if (lds <= 65536 || configured == ctx->device) return VARDROP_OK;
  int current = ctx->device;
  VD_HIP(ctx, hipGetDevice(&current));
  if (current != ctx->device) VD_HIP(ctx, hipSetDevice(ctx->device));
  const hipError_t e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (current != ctx->device) (void)hipSetDevice(current);
  VD_HIP(ctx, e);
  configured = ctx->device;
  return VARDROP_OK;
}

template <bool I8, bool AKC, bool BKC, typename S, typename Epi>
int launch_tile_gemm(vardrop_ctx* ctx, int kid, const TileArgs& g, const typename Epi::Args& epi, hipStream_t s) {
  static int configured = -1;
  const int rc = tile_allow_lds(ctx, (const void*)tile_gemm_kernel<I8, AKC, BKC, S, Epi>, S::lds, configured);
  if (rc) return rc;
  const long long grid = tile_count<S>(g, g.M);
  if (grid >= (1ll << 31)) return VARDROP_EUNSUPPORTED;
  if (grid == 0) return VARDROP_OK;
  {
    VdTimer timer(ctx, kid, s);
    VD_KERNEL(ctx, (tile_gemm_kernel<I8, AKC, BKC, S, Epi>), dim3((unsigned)grid), dim3(S::THREADS), S::lds, s, g, epi);
  }
  VD_LAUNCH_CHECK(ctx);
  return VARDROP_OK;
}

}  // namespace
#endif  // VARDROP_TILE_GEMM_H
