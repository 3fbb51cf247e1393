// What the absorbed-form decoding kernels over paged caches share (paged_attn.hip, decode_shared.hip):
// the cut of a list of tiles, matrix products pinned to their registers, the merge of softmax states.
#pragma once
#include "common.h"
#include "kernels.h"

namespace mla {
namespace {

constexpr int PD_KT = 32;         // rows per tile
constexpr int PD_WAVES = 4;
constexpr float PD_SLACK = 8.f;   // log2 units the running reference maximum may lag
constexpr int PD_CUS = 256;
// Tiles that a wavefront sums before its state is put down and the next begins.  An fp32 sum of n values of one size is off by
// up to n 2^-25 of itself, in one direction where they are equal: of 4096 tiles 2^-12 (a weighted latent, two additions
// a tile) and 2^-13 (the weights, first a tile's).  (Of one sequence of 2^31 - 1 rows alike, 65536 tiles a wavefront and each
// weight added by itself, 0.7 %; of three behind as many shared rows 5 %.)  States are joined up to a thousand times: 2^-15 more.
constexpr int PD_RUN = 4096;

__device__ __forceinline__ int tiles_of(int n) { return (int)(((uint32_t)n + PD_KT - 1) / PD_KT); }  // (n up to 2^31 - 1)
// The list's cut: tiles per workgroup (at least one for each wavefront), and the part of
// workgroup w and of its wavefronts.
struct ListCut {
  int total, share;
  __device__ __forceinline__ ListCut(int tiles, int nwg) : total(tiles), share(max(PD_WAVES, (tiles + nwg - 1) / nwg)) {}
  __device__ __forceinline__ int lo(int w) const { return (int)min((int64_t)w * share, (int64_t)total); }
  __device__ __forceinline__ int hi(int w) const { return min(lo(w) + share, total); }
  __device__ __forceinline__ int per_wave(int w) const { return (hi(w) - lo(w) + PD_WAVES - 1) / PD_WAVES; }
};

// Matrix products with their accumulators where they are wanted: the weighted latents fill the 256
// accumulation registers, the tile's logits are in vector registers.  (The compiler puts every
// product's result on one side, and moved 256 values out and in around each tile for the few that
// are rescaled.)  The waits are those that the compiler keeps around products it knows: two
// states after the vector ALU wrote an operand, and the product's passes (19 states at most)
// before the vector ALU reads a result.  The compiler does not know that latency: that it puts no move or
// spill of an accumulator there (the kernel of 576-wide rows spills 4 vector and 22 scalar registers) is
// checked on the built code by tests/test_matrix_waits.py.
__device__ __forceinline__ void mfma_v_first(f32x16& d, bf16x8 x, bf16x8 y) {
  asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(d) : "v"(x), "v"(y));
}
__device__ __forceinline__ void mfma_v_next(f32x16& d, bf16x8 x, bf16x8 y) {
  asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(d) : "v"(x), "v"(y));
}
__device__ __forceinline__ void mfma_v_done(f32x16& d) { asm volatile("s_nop 15\n\ts_nop 7" : "+v"(d)); }
__device__ __forceinline__ void mfma_a(f32x16& d, bf16x8 x, bf16x8 y) {
  asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(d) : "v"(x), "v"(y));
}
template <int N>
__device__ __forceinline__ void mfma_a_done(f32x16 (&d)[N]) {
  asm volatile("s_nop 15\n\ts_nop 7" : "+a"(d[0]));
#pragma unroll
  for (int c = 1; c < N; ++c) asm volatile("" : "+a"(d[c]));
}
// v *= f on accumulation registers
__device__ __forceinline__ void acc_scale(f32x16& v, float f) {
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    float x = v[e], t;
    asm volatile("v_accvgpr_read_b32 %1, %0\n\tv_mul_f32 %1, %1, %2\n\tv_accvgpr_write_b32 %0, %1"
                 : "+a"(x), "=&v"(t)
                 : "v"(f));
    v[e] = x;
  }
}

// elements 4 g .. of accumulation registers, which stay where they are
__device__ __forceinline__ f32x4 acc_read4(const f32x16& v, int g) {
  f32x4 o;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float x = v[4 * g + k];
    float t;
    asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(t) : "a"(x));
    o[k] = t;
  }
  return o;
}

// 2^d, d <= 0, the factor of a state whose reference moves up by -d.  A sum of weights may be as large as 2^126 where its rows'
// powers of two are small (decode_shared.hip), and what 2^d, which fp32 holds down to 2^-126, makes of it still count:
// half of d at a time.  (Past d = -252 a sum is below 2^-126, the weighted latents past -126.)  POWERS: whether there are such.
template <bool POWERS>
struct StateFactor {
  float f;
  __device__ __forceinline__ explicit StateFactor(float d) : f(__builtin_amdgcn_exp2f(POWERS ? 0.5f * d : d)) {}
  __device__ __forceinline__ float value() const { return POWERS ? f * f : f; }
  __device__ __forceinline__ float sum(float l) const { return POWERS ? l * f * f : l * f; }
};

// 1 KB from a uniform address plus the lanes' offsets to the LDS byte address `lds`
__device__ __forceinline__ void copy_s(uint64_t sbase, uint32_t voff, uint32_t lds) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(voff), "s"(sbase), "{m0}"(lds) : "memory");
}

// The states of a (sequence, head) joined, then W_UV on the matrix cores: lat[d] = sum_s o_s[d]
// 2^(m_s - M) / sum_s l_s 2^(m_s - M), o[e] = sum_d W_UV[g][e][d] lat[d].  A workgroup owns HB heads
// of a KV group and RB sequences, the columns of the product.  W_UV of the group is copied to LDS,
// asked for before anything else (read from memory as the matrix operand its rows' 16-byte pieces
// cost 64 address cycles a KB, 3.4 us for 128 KB; copied 0.9); DVL / 4 threads, four latents each,
// take a column's states (or every so-many-th of them), eight in flight.  States in the list's
// order.  The latent enters the product as the sum of two bf16 values, so that it is not rounded
// between the softmax and W_UV.  Bound by latency: the list's places, the states, the product.
constexpr int PF_THREADS = 1024;

// Where the states of the sequence with tiles [t0, t1) are: n of them, the first n0 in the slots
// of its first workgroup (one if that is joined), one for each workgroup inside (or one for each of its
// wavefronts, if their shares are longer than PD_RUN), the last in those of its last workgroup.
struct States {
  int n = 0, n0 = 0, mid = 0, step = PD_WAVES, at0 = 0, at_mid = 0, at1 = 0;
  States() = default;
  __device__ __forceinline__ States(const ListCut& cut, int b, int t0, int t1) {
    if (t1 <= t0) return;
    const int w0 = t0 / cut.share, w1 = (t1 - 1) / cut.share;
    int v;
    n0 = part(cut, w0, t0, t1, v);
    at0 = PD_WAVES * w0 + v + b;
    n = n0;
    if (w1 > w0) {
      mid = w1 - w0 - 1;
      if (cut.per_wave(w0 + 1) > PD_RUN && mid > 0) {
        mid *= PD_WAVES;
        step = 1;
      }
      at_mid = PD_WAVES * (w0 + 1) + b;
      n += mid + part(cut, w1, t0, t1, v);
      at1 = PD_WAVES * w1 + v + b;
    }
  }
  __device__ __forceinline__ static int part(const ListCut& cut, int w, int t0, int t1, int& v) {
    const int lo = cut.lo(w), hi = cut.hi(w), per = cut.per_wave(w);
    v = 0;
    if (t0 <= lo && hi <= t1 && per <= PD_RUN) return 1;  // joined
    v = (max(t0, lo) - lo) / per;
    return (min(t1, hi) - 1 - lo) / per - v + 1;
  }
  __device__ __forceinline__ int slot(int k) const {
    if (k < n0) return at0 + k;
    k -= n0;
    if (k < mid) return at_mid + step * k;
    return at1 + k - mid;
  }
};

// Where the states are: of the paged decoding, in slots of HP heads.
struct ListWhere {
  static constexpr bool POWERS = false;
  const int32_t* tile_off;
  int B, HP, nwg;
  __device__ __forceinline__ States states(int b, int head) const {
    return States(ListCut(tile_off[B], nwg), b, tile_off[b], tile_off[b + 1]);
  }
  __device__ __forceinline__ int64_t row(const States& st, int k, int head) const {
    return (int64_t)st.slot(k) * HP + head;
  }
};

template <int DVL, int DV, int HB, int RB, class Where>
__global__ __launch_bounds__(PF_THREADS) void paged_finish_kernel(const float* __restrict__ part_o,
                                                                  const float* __restrict__ part_ml, Where where,
                                                                  const bf16_t* __restrict__ Wuv,
                                                                  bf16_t* __restrict__ o, int B, int H, int hpg) {
  constexpr int NCG = DVL / 4, NCOL = HB * RB, NSLOT = PF_THREADS / NCG / NCOL, U = 8;
  constexpr int CHW = DVL / 8, NCPW = DV * CHW / 64, NW = PF_THREADS / 64, LDL = DVL + 8;
  constexpr int RED = NSLOT > 1 ? NCOL * NSLOT * DVL * 4 : 16, LAT = 2 * NCOL * LDL * 2;
  static_assert(NSLOT >= 1 && NCPW % NW == 0 && NCOL <= 16 && CHW >= 16, "finish shape");
  __shared__ __attribute__((aligned(1024))) bf16_t Ws[DV * DVL];  // chunk c of row e at c ^ (e % 16)
  __shared__ __attribute__((aligned(16))) char red_mem[RED];
  __shared__ __attribute__((aligned(16))) char lat_mem[LAT];
  __shared__ float sm[NCOL][NSLOT], sl[NCOL][NSLOT];
  float(*red)[DVL] = (float(*)[DVL])red_mem;                  // [NCOL * NSLOT]
  bf16_t* lat = (bf16_t*)lat_mem;                             // [2][NCOL][LDL]: rounded, and what that lost
  const int i0 = HB * blockIdx.x, b0 = RB * blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_id();
  const bf16_t* Wg = Wuv + (int64_t)(i0 / hpg) * DV * DVL;
#pragma unroll
  for (int k0 = 0; k0 < NCPW / NW; ++k0) {
    const int k = k0 * NW + wave, idx = 64 * k + lane, e = idx / CHW, c = (idx % CHW) ^ (e & 15);
    dma16(Wg + e * DVL + 8 * c, Ws + 512 * k);
  }
  // this thread's column: head i0 + h, sequence b0 + r
  const int cg = tid % NCG, grp = tid / NCG, col = grp / NSLOT, slot = grp % NSLOT;
  const int h = col % HB, b = b0 + col / HB;
  decltype(where.states(0, 0)) st;
  if (b < B) st = where.states(b, i0 + h);
  float M = -INFINITY, L = 0.f;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = slot; k0 < st.n; k0 += U * NSLOT) {
    f32x4 x[U];
    f32x2 ml[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + u * NSLOT;
      ml[u] = f32x2{-INFINITY, 0.f};
      x[u] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (k < st.n) {
        const int64_t rw = where.row(st, k, i0 + h);
        x[u] = *(const f32x4*)(part_o + rw * DVL + 4 * cg);
        ml[u] = *(const f32x2*)(part_ml + 2 * rw);
      }
    }
    float m1 = M;
#pragma unroll
    for (int u = 0; u < U; ++u) m1 = fmaxf(m1, ml[u][0]);
    const float ref = m1 == -INFINITY ? 0.f : m1;
    const StateFactor<Where::POWERS> c(M - ref);
    v *= c.value();
    L = c.sum(L);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const StateFactor<Where::POWERS> w(ml[u][0] - ref);
      v += x[u] * w.value();
      L += w.sum(ml[u][1]);
    }
    M = m1;
  }
  if (NSLOT > 1) {
    *(f32x4*)&red[grp][4 * cg] = v;
    if (cg == 0) {
      sm[col][slot] = M;
      sl[col][slot] = L;
    }
    __syncthreads();
  }
  if (slot == 0) {
    if (NSLOT > 1) {  // the column's slots, in order
      float ref = -INFINITY;
#pragma unroll
      for (int k = 0; k < NSLOT; ++k) ref = fmaxf(ref, sm[col][k]);
      if (ref == -INFINITY) ref = 0.f;
      v = f32x4{0.f, 0.f, 0.f, 0.f};
      L = 0.f;
#pragma unroll
      for (int k = 0; k < NSLOT; ++k) {
        const StateFactor<Where::POWERS> f(sm[col][k] - ref);
        v += *(const f32x4*)&red[grp + k][4 * cg] * f.value();
        L += f.sum(sl[col][k]);
      }
    }
    v *= L == 0.f ? 0.f : 1.f / L;  // (NaN stays NaN)
    const u32x2 hi = {pack2bf(v[0], v[1]), pack2bf(v[2], v[3])};
    *(u32x2*)(lat + col * LDL + 4 * cg) = hi;
    *(u32x2*)(lat + (NCOL + col) * LDL + 4 * cg) =
        u32x2{pack2bf(v[0] - __uint_as_float(hi[0] << 16), v[1] - __uint_as_float(hi[0] & 0xffff0000u)),
              pack2bf(v[2] - __uint_as_float(hi[1] << 16), v[3] - __uint_as_float(hi[1] & 0xffff0000u))};
  }
  wait_vm<0>();  // W_UV
  __syncthreads();
  if (wave >= DV / 16) return;
  // W_UV rows 16 wave + lane % 16 as the A operand, column lane % 16 of the latents as the B operand
  const int n = lane & 15, q = lane >> 4, e = 16 * wave + n;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int kk = 0; kk < DVL / 32; ++kk) {
    const bf16x8 wf = *(const bf16x8*)(Ws + e * DVL + 8 * ((4 * kk + q) ^ (e & 15)));
#pragma unroll
    for (int p = 0; p < 2; ++p)
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
          wf, *(const bf16x8*)(lat + (p * NCOL + min(n, NCOL - 1)) * LDL + 32 * kk + 8 * q), acc, 0, 0, 0);
  }
  if (n >= NCOL || b0 + n / HB >= B) return;
  bf16_t* op = o + ((int64_t)(b0 + n / HB) * H + i0 + n % HB) * DV + 16 * wave + 4 * q;
#pragma unroll
  for (int k = 0; k < 4; ++k) op[k] = f2bf(acc[k]);  // (o may have any alignment)
}

// One column a workgroup while that is one round on the CUs, else eight that share W_UV (four heads of two
// sequences, or one of eight where a group's heads are no multiple of four): 64 columns of many states
// 9.7 us by one, 38 by eight; 2048 columns 36 us by one, 8.2 by eight.
template <int DVL, int DV, class Where>
void decode_finish_v(const DecodePaged& d, const float* part_o, const float* part_ml, const Where& w, hipStream_t s) {
#define FIN(hb_, rb_)                                                                                        \
  paged_finish_kernel<DVL, DV, hb_, rb_><<<dim3(d.H / hb_, (d.B + rb_ - 1) / rb_), PF_THREADS, 0, s>>>(      \
      part_o, part_ml, w, (const bf16_t*)d.Wuv, (bf16_t*)d.o, d.B, d.H, d.hpg)
  if ((int64_t)d.B * d.H <= PD_CUS) FIN(1, 1);
  else if (d.hpg % 4 == 0) FIN(4, 2);
  else FIN(1, 8);
#undef FIN
}
template <int DVL, class Where>
void decode_finish(const DecodePaged& d, const float* part_o, const float* part_ml, const Where& w, hipStream_t s) {
  if (d.dv == 128) decode_finish_v<DVL, 128>(d, part_o, part_ml, w, s);
  else decode_finish_v<DVL, 64>(d, part_o, part_ml, w, s);
}

}  // namespace
}  // namespace mla
