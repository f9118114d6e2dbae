// Activations in 8 bits (format: pack8.h): pack and unpack.
//
// Bound by memory: 2 or 4 bytes an element one way, 33/32 the other.  27 584 x 512 in bf16: pack 9.7 us (4.4 TB/s), unpack 8.0 (5.3).
#include "pack8.h"

namespace {

struct PackArgs {
  const void* x;             // what is packed
  void* values;              // what is unpacked
  uint8_t* codes;
  uint8_t* exps;
  int B, n, d;
  const int32_t* n_dev;
  int32_t* status;
};

__device__ inline bool pack_rows(const PackArgs& p, long long& rows) {
  int n;
  if (!vd_count(p.n_dev, p.n, n, p.status)) return false;
  rows = (long long)p.B * n;
  return true;
}

// Whole blocks (d a multiple of 32): the tensor is one line of groups of eight, a lane each; four lanes are a block.
template <typename T, int U>
__global__ __launch_bounds__(256) void pack8_kernel(PackArgs p) {
  long long rows;
  if (!pack_rows(p, rows)) return;
  const long long groups = rows * (p.d >> 3);
  const T* x = (const T*)p.x;
  for (long long at = (long long)blockIdx.x * (256 * U); at < groups; at += (long long)gridDim.x * (256 * U)) {
    float v[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long i = at + u * 256 + threadIdx.x;
      if (i < groups) load_eight(x + i * 8, v[u]);
      else
#pragma unroll
        for (int j = 0; j < 8; ++j) v[u][j] = 0.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long i = at + u * 256 + threadIdx.x;
      const bool live = i < groups;              // (a block's four lanes agree: groups is a multiple of four)
      uint32_t e;
      const u32x2 c = pack_eight(v[u], e);
      if (live) *reinterpret_cast<u32x2*>(p.codes + i * 8) = c;
      // four exponents of sixteen lanes leave as one word
      const uint32_t word = e | ((uint32_t)__builtin_amdgcn_mov_dpp((int)e, 0x104, 0xf, 0xf, true) << 8) |
                            ((uint32_t)__builtin_amdgcn_mov_dpp((int)e, 0x108, 0xf, 0xf, true) << 16) |
                            ((uint32_t)__builtin_amdgcn_mov_dpp((int)e, 0x10c, 0xf, 0xf, true) << 24);
      if ((i | 15) < groups) {
        if ((threadIdx.x & 15) == 0) *reinterpret_cast<uint32_t*>(p.exps + (i >> 2)) = word;
      } else if (live && (threadIdx.x & 3) == 0) {
        p.exps[i >> 2] = (uint8_t)e;
      }
    }
  }
}

// Any width and alignment: half a wavefront a block, a lane a channel.  The tensor above by elements: 26.8 and 20.0 us; 65 536 x 321 in fp32 38 and
// 30 (2.8 and 3.6 TB/s): a load, five steps of a maximum and a store of one byte for every element.  (Eight elements a lane, their stores 8 to 32
// bytes apart: pack 28 -> 18 in bf16 and 26 -> 28 in fp32, unpack 20 -> 21 and 20 -> 37.)
__device__ inline long long block_row(long long b, int nb, long long blocks) {
  return blocks <= 0x7fffffff ? (long long)((uint32_t)b / (uint32_t)nb) : b / nb;         // (in 32 bits a third of the work)
}
template <typename T>
__global__ __launch_bounds__(256) void pack8_any_kernel(PackArgs p) {
  long long rows;
  if (!pack_rows(p, rows)) return;
  constexpr int U = 4;
  const int nb = pack_blocks(p.d), l = threadIdx.x & 31;
  const long long blocks = rows * nb;
  for (long long at = (long long)blockIdx.x * (8 * U); at < blocks; at += (long long)gridDim.x * (8 * U)) {
    float v[U];
    long long row[U];
    int c[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long b = at + u * 8 + (threadIdx.x >> 5);
      row[u] = block_row(b, nb, blocks);
      c[u] = (int)(b - row[u] * nb) * kPackBlock + l;
      v[u] = b < blocks && c[u] < p.d ? to_float(((const T*)p.x)[row[u] * p.d + c[u]]) : 0.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long b = at + u * 8 + (threadIdx.x >> 5);
      const bool live = b < blocks && c[u] < p.d;
      float top = __builtin_fabsf(v[u]);
      top = most_of(top, __uint_as_float(__builtin_amdgcn_mov_dpp((int)__float_as_uint(top), 0xb1, 0xf, 0xf, true)));      // lanes ^ 1
      top = most_of(top, __uint_as_float(__builtin_amdgcn_mov_dpp((int)__float_as_uint(top), 0x4e, 0xf, 0xf, true)));      // lanes ^ 2
      top = most_of(top, __uint_as_float(__builtin_amdgcn_mov_dpp((int)__float_as_uint(top), 0x141, 0xf, 0xf, true)));     // the other four of eight
      top = most_of(top, __uint_as_float(__builtin_amdgcn_mov_dpp((int)__float_as_uint(top), 0x140, 0xf, 0xf, true)));     // the other eight of sixteen
      top = most_of(top, __shfl_xor(top, 16, 64));
      const uint32_t e = pack_exponent(__float_as_uint(top));
      if (live) p.codes[row[u] * p.d + c[u]] = (uint8_t)pack_code(e >= 248u ? pack_limit(v[u]) : v[u], pack_up(e));
      if (live && l == 0) p.exps[b] = (uint8_t)e;
    }
  }
}

template <typename T, int U>
__global__ __launch_bounds__(256) void unpack8_kernel(PackArgs p) {
  long long rows;
  if (!pack_rows(p, rows)) return;
  const long long groups = rows * (p.d >> 3);
  for (long long at = (long long)blockIdx.x * (256 * U); at < groups; at += (long long)gridDim.x * (256 * U)) {
    u32x2 c[U];
    uint32_t e[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long i = at + u * 256 + threadIdx.x;
      if (i < groups) {
        c[u] = *reinterpret_cast<const u32x2*>(p.codes + i * 8);
        e[u] = p.exps[i >> 2];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long i = at + u * 256 + threadIdx.x;
      if (i < groups) {
        float v[8];
        unpack_eight(c[u], e[u], v);
        store_eight((T*)p.values + i * 8, v);
      }
    }
  }
}

template <typename T>
__global__ __launch_bounds__(256) void unpack8_any_kernel(PackArgs p) {
  long long rows;
  if (!pack_rows(p, rows)) return;
  constexpr int U = 4;
  const int nb = pack_blocks(p.d), l = threadIdx.x & 31;
  const long long blocks = rows * nb;
  for (long long at = (long long)blockIdx.x * (8 * U); at < blocks; at += (long long)gridDim.x * (8 * U)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long b = at + u * 8 + (threadIdx.x >> 5), row = block_row(b, nb, blocks);
      const int c = (int)(b - row * nb) * kPackBlock + l;
      if (b >= blocks || c >= p.d) continue;
      const long long i = row * p.d + c;
      from_float((T*)p.values + i, (float)(int8_t)p.codes[i] * pack_step(p.exps[b]));
    }
  }
}

unsigned pack_grid(long long items, int per_block) {
  const long long b = (items + per_block - 1) / per_block;
  return (unsigned)(b > 4096 ? 4096 : b);
}

template <typename T>
int launch_pack(vardrop_ctx* ctx, const PackArgs& p, long long rows, hipStream_t s) {
  VdTimer timer(ctx, VARDROP_K_PACK8, s);
  if (p.d % kPackBlock == 0 && vd_aligned(p.x, 16)) VD_KERNEL(ctx, (pack8_kernel<T, 4>), dim3(pack_grid(rows * (p.d / 8), 1024)), dim3(256), 0, s, p);
  else VD_KERNEL(ctx, pack8_any_kernel<T>, dim3(pack_grid(rows * pack_blocks(p.d), 32)), dim3(256), 0, s, p);
  VD_LAUNCH_CHECK(ctx);
  return VARDROP_OK;
}
template <typename T>
int launch_unpack(vardrop_ctx* ctx, const PackArgs& p, long long rows, hipStream_t s) {
  VdTimer timer(ctx, VARDROP_K_UNPACK8, s);
  if (p.d % kPackBlock == 0 && vd_aligned(p.values, 16)) VD_KERNEL(ctx, (unpack8_kernel<T, 4>), dim3(pack_grid(rows * (p.d / 8), 1024)), dim3(256), 0, s, p);
  else VD_KERNEL(ctx, unpack8_any_kernel<T>, dim3(pack_grid(rows * pack_blocks(p.d), 32)), dim3(256), 0, s, p);
  VD_LAUNCH_CHECK(ctx);
  return VARDROP_OK;
}

int check_pack(vardrop_ctx* ctx, int B, int n, int d, int dtype, const void* x, const void* saved) {
  if (!ctx || B < 0 || n < 0 || d < 1 || (dtype != VARDROP_F32 && dtype != VARDROP_BF16)) return VARDROP_EINVAL;
  if ((long long)B * n >= (1ll << 31) || d > (1 << 20)) return VARDROP_EUNSUPPORTED;
  if ((long long)B * n == 0) return VARDROP_OK;
  if (!x || !vd_aligned(x, dtype == VARDROP_F32 ? 4 : 2)) return VARDROP_EINVAL;
  if (!saved || !vd_aligned(saved, 256)) return VARDROP_EWORKSPACE;
  return VARDROP_OK;
}
PackArgs pack_args(const void* x, void* values, const void* saved, int B, int n, int d, VdDevCount dn) {
  uint8_t* codes = (uint8_t*)const_cast<void*>(saved);
  return {x, values, codes, codes + pack_exponents_at((long long)B * n, d), B, n, d, dn.dev, dn.status};
}
int pack(vardrop_ctx* ctx, const void* x, int B, int n, int d, int dtype, void* saved, hipStream_t s, VdDevCount dn) {
  const int rc = check_pack(ctx, B, n, d, dtype, x, saved);
  if (rc || (long long)B * n == 0) return rc;
  const PackArgs p = pack_args(x, nullptr, saved, B, n, d, dn);
  return dtype == VARDROP_BF16 ? launch_pack<bf16_t>(ctx, p, (long long)B * n, s) : launch_pack<float>(ctx, p, (long long)B * n, s);
}
int unpack(vardrop_ctx* ctx, const void* saved, int B, int n, int d, int dtype, void* x, hipStream_t s, VdDevCount dn) {
  const int rc = check_pack(ctx, B, n, d, dtype, x, saved);
  if (rc || (long long)B * n == 0) return rc;
  const PackArgs p = pack_args(nullptr, x, saved, B, n, d, dn);
  return dtype == VARDROP_BF16 ? launch_unpack<bf16_t>(ctx, p, (long long)B * n, s) : launch_unpack<float>(ctx, p, (long long)B * n, s);
}

}  // namespace

extern "C" size_t vardrop_pack8_bytes(int B, int n, int d) {
  if (B < 0 || n < 0 || d < 1 || (long long)B * n >= (1ll << 31) || d > (1 << 20)) return 0;
  return pack_bytes((long long)B * n, d);
}
extern "C" int vardrop_pack8(vardrop_ctx* ctx, const void* x, int B, int n, int d, int dtype, void* saved, void* stream) {
  return pack(ctx, x, B, n, d, dtype, saved, (hipStream_t)stream, {nullptr, nullptr});
}
extern "C" int vardrop_unpack8(vardrop_ctx* ctx, const void* saved, int B, int n, int d, int dtype, void* x, void* stream) {
  return unpack(ctx, saved, B, n, d, dtype, x, (hipStream_t)stream, {nullptr, nullptr});
}
extern "C" int vardrop_pack8_dev(vardrop_ctx* ctx, const void* x, int B, const int32_t* n_dev, int n_max, int32_t* status, int d, int dtype,
                                 void* saved, void* stream) {
  if (!n_dev || n_max < 1) return VARDROP_EINVAL;
  return pack(ctx, x, B, n_max, d, dtype, saved, (hipStream_t)stream, {n_dev, status});
}
extern "C" int vardrop_unpack8_dev(vardrop_ctx* ctx, const void* saved, int B, const int32_t* n_dev, int n_max, int32_t* status, int d, int dtype,
                                   void* x, void* stream) {
  if (!n_dev || n_max < 1) return VARDROP_EINVAL;
  return unpack(ctx, saved, B, n_max, d, dtype, x, (hipStream_t)stream, {n_dev, status});
}
