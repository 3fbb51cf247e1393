// Rows of a paged latent cache in eight bits (MLA_CACHE_E4M3), and what its kernels share.
//
// A page is page_size rows of [r_kv latents in e4m3 | positional values in bf16], then page_size powers of
// two (fp32), padded to 16 bytes.  The rows are multiples of 64 bytes at the widths that attention serves
// (192, 320 and 640 bytes), so that a tile of them is copied and read in whole 16-byte pieces of whole lines;
// with its power inside a row they would not be.  One power a row is enough: e4m3 has an exponent of its own,
// so a latent keeps its three bits of fraction down to 2^-14 of the row's largest, which finer powers
// (for every 32 latents, say) would gain for smaller ones only.  A power of two makes a latent's value exact in
// bf16, and its e4m3 value exact in fp16: attention multiplies the e4m3 values and brings the power in by the
// row, in the logit and in the weight.
#pragma once
#include "common.h"

namespace mla {

constexpr int E4M3_MIN_EXP = -80, E4M3_MAX_EXP = 120;  // of the rows' powers

struct E4m3Page {
  int page_size, rkv, row_bytes;  // row_bytes: without the power
  int64_t bytes;
  E4m3Page() = default;
  __host__ __device__ E4m3Page(int page_size_, int rkv_, int pe)
      : page_size(page_size_), rkv(rkv_), row_bytes(rkv_ + 2 * pe),
        bytes(((int64_t)page_size_ * (rkv_ + 2 * (int64_t)pe + 4) + 15) & ~(int64_t)15) {}
  __device__ __forceinline__ char* row(void* pool, int page, int r) const {
    return (char*)pool + page * bytes + (int64_t)r * row_bytes;
  }
  __device__ __forceinline__ float* power(void* pool, int page, int r) const {
    return (float*)((char*)pool + page * bytes + (int64_t)page_size * row_bytes) + r;
  }
};

// The exponent of a row's power from the bits of its largest finite magnitude (fp32): the least e with
// top <= 448 2^e = 1.75 2^(e + 8).
__device__ __forceinline__ int e4m3_exponent(uint32_t top) {
  const int e = (int)(top >> 23) - 135 + ((top & 0x7fffffu) > 0x600000u);
  return min(max(e, E4M3_MIN_EXP), E4M3_MAX_EXP);
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

// 8 bf16 values times 2^-e, as e4m3 (nearest, halves to even; NaN for what is not finite)
__device__ __forceinline__ u32x2 to_e4m3(u32x4 v, float scale) {
  float f[8];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint32_t lo = v[q] << 16, hi = v[q] & 0xffff0000u;
    f[2 * q] = (lo & 0x7f800000u) == 0x7f800000u ? NAN : __uint_as_float(lo) * scale;
    f[2 * q + 1] = (hi & 0x7f800000u) == 0x7f800000u ? NAN : __uint_as_float(hi) * scale;
  }
  u32x2 o;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * q], f[4 * q + 1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * q + 2], f[4 * q + 3], w, true);
    o[q] = (uint32_t)w;
  }
  return o;
}

// 8 e4m3 values times a power of two, as bf16 (exact but past bf16's ends)
__device__ __forceinline__ u32x4 from_e4m3(u32x2 v, float power) {
  u32x4 o;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[q], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[q], true);
    o[2 * q] = pack2bf(a[0] * power, a[1] * power);
    o[2 * q + 1] = pack2bf(b[0] * power, b[1] * power);
  }
  return o;
}

// The sequence of packed row i: the largest b with offsets[b] <= i (offsets[0] <= i).
__device__ __forceinline__ int sequence_of(const int32_t* offsets, int B, int i) {
  int lo = 0, hi = B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (offsets[mid] <= i) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

}  // namespace mla
