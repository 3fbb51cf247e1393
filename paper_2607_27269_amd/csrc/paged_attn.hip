// Attention over the paged latent cache (paged.hip) in absorbed form: head i's query against the
// cache rows is [W_UK[g]^T q^nope_i ; q^rope_i], its output W_UV[g] applied to the
// attention-weighted latent (g = i / (H / G_kv)).
#include "attn_common.h"
#include "common.h"
#include "kernels.h"

namespace mla {
namespace {

struct PagedAttnDev {
  const bf16_t* pool;
  const int32_t* table;
  int n_pages, page_size, max_pages;
  int B, H, HP, DK, rkv;
  const bf16_t* qabs;                // [rows][HP][DK]
  const bf16_t* Wuv;
  int dv, hpg;
  bf16_t* o;                         // [rows][H][dv]
  const int32_t* len;                // single tokens: [B], row = sequence
  int max_len;
  const int32_t *q_off, *kv_off;     // packed tokens: [B + 1]
  int n_q, n_kv;
  float sl2;
};

// A workgroup per (query row, head): each wavefront takes every fourth cache row, 64 lanes over
// its values, running maximum and sum, the weighted latent in registers; the four states are
// joined through LDS.
constexpr int SIMPLE_MAX = 9;  // values of a row per lane: DK <= 576
__global__ __launch_bounds__(256) void paged_attn_simple_kernel(PagedAttnDev a) {
  __shared__ float sm[4], sl[4], so[4][512];
  const int r = blockIdx.x, i = blockIdx.y;
  const int lane = threadIdx.x & 63, wave = wave_id();
  int b = r, n;
  if (a.len) {
    n = min(max(a.len[b], 0), a.max_len);
  } else {
    if (r < max(a.q_off[0], 0) || r >= min(a.q_off[a.B], a.n_q)) return;
    int lo = 0, hi = a.B - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.q_off[mid] <= r) lo = mid;
      else hi = mid - 1;
    }
    b = lo;
    const int kv = min(a.kv_off[b + 1], a.n_kv) - max(a.kv_off[b], 0);
    n = min(max(kv - (a.q_off[b + 1] - 1 - r), 0), kv);
  }
  n = (int)min((int64_t)n, (int64_t)a.page_size * a.max_pages);
  float q[SIMPLE_MAX], acc[SIMPLE_MAX];
#pragma unroll
  for (int k = 0; k < SIMPLE_MAX; ++k) {
    const int c = lane + 64 * k;
    q[k] = c < a.DK ? bf2f(a.qabs[((int64_t)r * a.HP + i) * a.DK + c]) : 0.f;
    acc[k] = 0.f;
  }
  float m = -INFINITY, l = 0.f;
  for (int j = wave; j < n; j += 4) {
    const int page = a.table[(int64_t)b * a.max_pages + j / a.page_size];
    const bool bad = page < 0 || page >= a.n_pages;
    const bf16_t* x = a.pool + ((int64_t)(bad ? 0 : page) * a.page_size + j % a.page_size) * a.DK;
    float v[SIMPLE_MAX], s = 0.f;
#pragma unroll
    for (int k = 0; k < SIMPLE_MAX; ++k) {
      const int c = lane + 64 * k;
      v[k] = c < a.DK ? (bad ? NAN : bf2f(x[c])) : 0.f;
      s += q[k] * v[k];
    }
    s = warp_sum(s) * a.sl2;
    const float m1 = fmaxf(m, s);
    const float corr = __builtin_amdgcn_exp2f(m - (m1 == -INFINITY ? 0.f : m1));
    const float p = __builtin_amdgcn_exp2f(s - (m1 == -INFINITY ? 0.f : m1));
    m = m1;
    l = l * corr + p;
#pragma unroll
    for (int k = 0; k < SIMPLE_MAX; ++k) acc[k] = acc[k] * corr + p * v[k];
  }
  if (lane == 0) {
    sm[wave] = m;
    sl[wave] = l;
  }
#pragma unroll
  for (int k = 0; k < SIMPLE_MAX; ++k)
    if (lane + 64 * k < a.rkv) so[wave][lane + 64 * k] = acc[k];
  __syncthreads();
  const float M = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
  float w[4], L = 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    w[k] = sm[k] == -INFINITY && !(sl[k] != sl[k]) ? 0.f : __builtin_amdgcn_exp2f(sm[k] - M);
    L += w[k] * sl[k];
  }
  const float inv = n > 0 ? 1.f / L : 0.f;
  __syncthreads();
  for (int c = threadIdx.x; c < a.rkv; c += 256)
    so[0][c] = (w[0] * so[0][c] + w[1] * so[1][c] + w[2] * so[2][c] + w[3] * so[3][c]) * inv;
  __syncthreads();
  for (int e = wave; e < a.dv; e += 4) {
    const bf16_t* u = a.Wuv + ((int64_t)(i / a.hpg) * a.dv + e) * a.rkv;
    float v = 0.f;
    for (int c = lane; c < a.rkv; c += 64) v += bf2f(u[c]) * so[0][c];
    v = warp_sum(v);
    if (lane == 0) a.o[((int64_t)r * a.H + i) * a.dv + e] = f2bf(v);
  }
}

size_t al(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

size_t decode_paged_ws_bytes(int B, int H, int DK, int DVL, int max_len) {
  const int HP = (H + 31) / 32 * 32;
  return al((size_t)B * HP * DK * 2);
}

hipError_t decode_paged(const DecodePaged& d, hipStream_t s) {
  const int HP = (d.H + 31) / 32 * 32, DK = d.rkv + d.dr;
  PagedAttnDev a = {};
  a.pool = (const bf16_t*)d.c.pool; a.table = d.c.table; a.n_pages = d.c.n_pages;
  a.page_size = d.c.page_size; a.max_pages = d.c.max_pages;
  a.B = d.B; a.H = d.H; a.HP = HP; a.DK = DK; a.rkv = d.rkv;
  a.qabs = (const bf16_t*)d.ws;
  a.Wuv = (const bf16_t*)d.Wuv; a.dv = d.dv; a.hpg = d.hpg; a.o = (bf16_t*)d.o;
  a.len = d.len; a.max_len = d.max_len; a.sl2 = d.scale * attn::LOG2E;
  hipError_t e = decode_absorb(d.q, d.Wuk, d.ws, d.B, d.H, HP, d.hpg, d.dn, d.dr, d.rkv, s);
  if (e != hipSuccess) return e;
  prof_begin(KC_ATTN_FWD, s);
  paged_attn_simple_kernel<<<dim3(d.B, d.H), 256, 0, s>>>(a);
  prof_end(KC_ATTN_FWD, s, 2.0 * d.B * d.H * (double)d.max_len * (DK + d.rkv), (double)d.B * d.max_len * DK * 2,
           KLABEL("paged_attn_simple_kernel"));
  return hipGetLastError();
}

size_t prefill_paged_ws_bytes(const PrefillPaged& p) {
  const int HP = (p.H + 31) / 32 * 32;
  return al((size_t)p.n_q * HP * (p.rkv + p.dr) * 2);
}

hipError_t prefill_paged(const PrefillPaged& p, hipStream_t s) {
  const int HP = (p.H + 31) / 32 * 32, DK = p.rkv + p.dr, hpg = p.H / p.G;
  PagedAttnDev a = {};
  a.pool = (const bf16_t*)p.c.pool; a.table = p.c.table; a.n_pages = p.c.n_pages;
  a.page_size = p.c.page_size; a.max_pages = p.c.max_pages;
  a.B = p.B; a.H = p.H; a.HP = HP; a.DK = DK; a.rkv = p.rkv;
  a.qabs = (const bf16_t*)p.ws;
  a.Wuv = (const bf16_t*)p.Wuv; a.dv = p.dv; a.hpg = hpg; a.o = (bf16_t*)p.o;
  a.q_off = p.q_off; a.kv_off = p.kv_off; a.n_q = p.n_q; a.n_kv = p.n_kv;
  a.sl2 = p.scale * attn::LOG2E;
  hipError_t e = decode_absorb(p.q, p.Wuk, p.ws, p.n_q, p.H, HP, hpg, p.dn, p.dr, p.rkv, s);
  if (e != hipSuccess) return e;
  prof_begin(KC_ATTN_FWD, s);
  paged_attn_simple_kernel<<<dim3(p.n_q, p.H), 256, 0, s>>>(a);
  prof_end(KC_ATTN_FWD, s, 0.0, 0.0, KLABEL("paged_attn_simple_kernel"));
  return hipGetLastError();
}

}  // namespace mla
