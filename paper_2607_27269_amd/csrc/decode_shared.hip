// Absorbed-form decoding over a paged latent cache of either format, for sequences some of which begin
// with the same rows.
#include "attn_common.h"
#include "cache_rows.h"
#include "common.h"
#include "kernels.h"

namespace mla {
namespace {

struct SharedDev {
  PagedPool c;
  const int32_t* len;
  int max_len, B, H, dn, dr, dv, hpg;
  const bf16_t *q, *Wuk, *Wuv;
  bf16_t* o;
  float sl2;
};

// A workgroup per (head, sequence): the absorbed query in LDS (fp32), a wavefront per row in turn, each
// with its own softmax state and weighted latent, joined through LDS, then W_UV.
template <int DK, int DVL, bool E4M3>
__global__ __launch_bounds__(256) void decode_simple_kernel(SharedDev a) {
  constexpr int DR = DK - DVL, NL = (DVL + 63) / 64;
  __shared__ float qs[DK], lat[4][DVL], ml[4][2];
  __shared__ int any_bad;
  const int i = blockIdx.x, b = blockIdx.y, g = i / a.hpg, tid = threadIdx.x, lane = tid & 63, wave = wave_id();
  const bf16_t* q = a.q + ((int64_t)b * a.H + i) * (a.dn + a.dr);
  for (int c = tid; c < DVL; c += 256) {
    float x = 0.f;
    for (int d = 0; d < a.dn; ++d) x += bf2f(q[d]) * bf2f(a.Wuk[((int64_t)g * a.dn + d) * DVL + c]);
    qs[c] = x;
  }
  for (int c = tid; c < DR; c += 256) qs[DVL + c] = bf2f(q[a.dn + c]);
  if (tid == 0) any_bad = 0;
  __syncthreads();
  const int n = min(max(a.len[b], 0), a.max_len);
  float m = -INFINITY, l = 0.f, acc[NL];
#pragma unroll
  for (int k = 0; k < NL; ++k) acc[k] = 0.f;
  const E4m3Page layout(a.c.page_size, DVL, DR);
  for (int p = wave; p < n; p += 4) {
    const int page = a.c.table[(int64_t)b * a.c.max_pages + p / a.c.page_size], r = p % a.c.page_size;
    if (page < 0 || page >= a.c.n_pages) {
      any_bad = 1;
      continue;
    }
    float x[NL], s = 0.f;
#pragma unroll
    for (int k = 0; k < NL; ++k) {
      const int c = lane + 64 * k;
      x[k] = 0.f;
      if (c < DVL) {
        if constexpr (E4M3)
          x[k] = __builtin_amdgcn_cvt_pk_f32_fp8((int)(uint8_t)layout.row(a.c.pool, page, r)[c], false)[0] *
                 *layout.power(a.c.pool, page, r);
        else
          x[k] = bf2f(((const bf16_t*)a.c.pool)[((int64_t)page * a.c.page_size + r) * DK + c]);
        s += x[k] * qs[c];
      }
    }
    if (lane < DR) {
      const bf16_t* pe = E4M3 ? (const bf16_t*)(layout.row(a.c.pool, page, r) + DVL)
                              : (const bf16_t*)a.c.pool + ((int64_t)page * a.c.page_size + r) * DK + DVL;
      s += bf2f(pe[lane]) * qs[DVL + lane];
    }
    s = warp_sum(s) * a.sl2;
    const float m1 = fmaxf(m, s), ref = m1 == -INFINITY ? 0.f : m1;
    const float f = exp2f(m - ref), w = exp2f(s - ref);  // (NaN stays NaN)
    l = l * f + w;
#pragma unroll
    for (int k = 0; k < NL; ++k) acc[k] = acc[k] * f + x[k] * w;
    m = m1;
  }
#pragma unroll
  for (int k = 0; k < NL; ++k)
    if (lane + 64 * k < DVL) lat[wave][lane + 64 * k] = acc[k];
  if (lane == 0) {
    ml[wave][0] = m;
    ml[wave][1] = l;
  }
  __syncthreads();
  float M = -INFINITY, L = 0.f, f[4];
  for (int w = 0; w < 4; ++w) M = fmaxf(M, ml[w][0]);
  for (int w = 0; w < 4; ++w) {
    f[w] = M == -INFINITY ? 1.f : exp2f(ml[w][0] - M);
    L += ml[w][1] * f[w];
  }
  const float inv = any_bad ? NAN : n == 0 ? 0.f : 1.f / L;
  for (int e = tid; e < a.dv; e += 256) {
    float v = 0.f;
    for (int c = 0; c < DVL; ++c) {
      float x = 0.f;
      for (int w = 0; w < 4; ++w) x += lat[w][c] * f[w];
      v += x * bf2f(a.Wuv[((int64_t)g * a.dv + e) * DVL + c]);
    }
    a.o[((int64_t)b * a.H + i) * a.dv + e] = f2bf(v * inv);
  }
}

#define MLA_SHARED_SHAPES(X) X(576, 512) X(288, 256) X(160, 128)

}  // namespace

size_t decode_shared_ws_bytes(int B, int H, int DK, int DVL, int max_len, int n_groups) { return 256; }

hipError_t decode_shared(const DecodeShared& p, hipStream_t s) {
  const DecodePaged& d = p.d;
  const int DK = d.rkv + d.dr, DVL = d.rkv;
  SharedDev a;
  a.c = d.c; a.len = d.len; a.max_len = d.max_len; a.B = d.B; a.H = d.H; a.dn = d.dn; a.dr = d.dr;
  a.dv = d.dv; a.hpg = d.hpg; a.q = (const bf16_t*)d.q; a.Wuk = (const bf16_t*)d.Wuk;
  a.Wuv = (const bf16_t*)d.Wuv; a.o = (bf16_t*)d.o; a.sl2 = d.scale * attn::LOG2E;
  prof_begin(KC_ATTN_FWD, s);
#define X(a_, b_)                                                                           \
  if (DK == a_ && DVL == b_) {                                                              \
    if (p.e4m3) decode_simple_kernel<a_, b_, true><<<dim3(d.H, d.B), 256, 0, s>>>(a);       \
    else decode_simple_kernel<a_, b_, false><<<dim3(d.H, d.B), 256, 0, s>>>(a);             \
  }
  MLA_SHARED_SHAPES(X)
#undef X
  prof_end(KC_ATTN_FWD, s, 2.0 * d.B * d.H * (double)d.max_len * (DK + DVL), (double)d.B * d.max_len * DK * 2,
           KLABEL("decode_simple_kernel"));
  return hipGetLastError();
}

}  // namespace mla
