// The absorbed queries of decoding (decode.hip, decode_shared.hip).
#pragma once
#include "common.h"

namespace mla {

// The absorbed queries of the heads of group g: row r = (b, j) of the
// B hpg rows is head i = g hpg + j of sequence b; qabs[b][i][c] = sum_d q[b][i][d] W_UK[g][d][c]
// for c < rkv, then the rotary part copied.  A workgroup (two wavefronts) makes 32 rows x 64
// columns; W_UK's 64 columns are staged in LDS as they lie ([d][c]) and read transposed
// (MFMA row = c), the query rows come straight from memory (MFMA column = row), so that a
// lane ends with 4 consecutive c of its row: 8-byte stores.  Bound by latency (W_UK is 1 MB at
// H = 32, r_kv = 512; one round of small workgroups), fp32 accumulation.  Measured with the
// rotary copy: 64 sequences 26 -> 7.1 us, one sequence 13.6 -> 4.1 us (a vector-ALU product and
// a copy launch before).
// Ws: ABS_LDS elements of LDS.
// ABS_FRAG: qabs in the order in which the paged decoding reads it, [b][block of 32 heads][16-wide step
// kk][half][head][8]: a matrix operand is 1 KB in one piece there.
// ABS_F16: fp16 for the decoding over an eight-bit cache, as [b][block of heads][step][half][head][8]: step 2 i + e
// of half h holds latents 32 i + 16 h + 8 e + 0..7.  32 latents of a head are brought to [2^8, 2^9) by a power of
// two, whose exponent is written to exps [b][block of heads][head][rkv / 32]; the rotary part is written in bf16, as by
// ABS_FRAG.  ABS_BOTH: ABS_FRAG and ABS_F16.
constexpr int ABS_LD = 96;  // LDS row stride: 4 rows of a transposing read on distinct banks
constexpr int ABS_DN = 192;
constexpr int ABS_LDS = ABS_DN * ABS_LD;  // elements of LDS, 16-byte aligned
enum AbsorbOut { ABS_ROWS, ABS_FRAG, ABS_F16, ABS_BOTH };
constexpr int ABS_MIN_EXP = -126, ABS_MAX_EXP = 120;
template <AbsorbOut OUT>
__device__ __forceinline__ void absorb_block(const bf16_t* __restrict__ q, const bf16_t* __restrict__ Wuk,
                                             bf16_t* __restrict__ qabs, bf16_t* __restrict__ qabs16,
                                             int8_t* __restrict__ exps, bf16_t* Ws, int B, int H, int HP, int hpg, int dn, int dr, int rkv, int bx, int by, int g) {
  const int c0 = 64 * bx, r0 = 32 * by;
  const int DK = rkv + dr, dq = dn + dr, tid = threadIdx.x;
  const int lane = tid & 63, wave = wave_id(), half = lane >> 5, col = lane & 31;
  const int dnp = (dn + 15) & ~15;  // d rounded up to the K step, zero filled
  const bf16_t* Wg = Wuk + (int64_t)g * dn * rkv + c0;
  const bool aligned = (uintptr_t)Wuk % 16 == 0;  // uniform
  constexpr int PIECES = ABS_DN * 8 / 128;
  u32x4 staged[PIECES];  // all asked for at once (a piece at a time took its round trip each: 8.8 us for 7.1)
  if (aligned) {
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
      const int e = tid + 128 * k, d = e >> 3, c = 8 * (e & 7);
      staged[k] = u32x4{0u, 0u, 0u, 0u};
      if (d < dn) staged[k] = *(const u32x4*)(Wg + (int64_t)d * rkv + c);
    }
  } else {
    for (int e = tid; e < dnp * 64; e += 128) {
      const int d = e >> 6, c = e & 63;
      Ws[d * ABS_LD + c] = d < dn ? Wg[(int64_t)d * rkv + c] : (bf16_t)0;
    }
  }
  const int rows = B * hpg, rr = r0 + col, rc = min(rr, rows - 1);
  const int64_t bi = (int64_t)(rc / hpg) * H + g * hpg + rc % hpg;           // row of q
  const int64_t qi = (int64_t)(rc / hpg) * HP + g * hpg + rc % hpg;          // row of qabs
  const bf16_t* qp = q + bi * dq + 8 * half;
  bf16x8 qf[ABS_DN / 16];  // this lane's row, asked for before the staging's barrier
#pragma unroll
  for (int kk = 0; kk < ABS_DN / 16; ++kk) {
    u32x4 w = {0u, 0u, 0u, 0u};
    if (16 * kk + 8 * half < dn) w = *(const u32x4*)(qp + 16 * kk);
    qf[kk] = __builtin_bit_cast(bf16x8, w);
  }
  if (aligned) {
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
      const int e = tid + 128 * k;
      if (e < dnp * 8) *(u32x4*)(Ws + (e >> 3) * ABS_LD + 8 * (e & 7)) = staged[k];
    }
  }
  // where 8 aligned elements c .. of row rc go
  const int head = g * hpg + rc % hpg;
  const int64_t fi = ((int64_t)(rc / hpg) * (HP / 32) + head / 32) * (DK / 16) * 512 + head % 32 * 8;
  auto place = [&](int c) {
    return OUT != ABS_ROWS ? qabs + fi + (c >> 4) * 512 + (c >> 3 & 1) * 256 : qabs + qi * DK + c;
  };
  if (bx == 0 && wave == 0 && rr < rows)  // rotary part: dr elements, half a row per lane
    for (int c = 8 * half; c < dr; c += 16)
      *(u32x4*)place(rkv + c) = *(const u32x4*)(q + bi * dq + dn + c);
  __syncthreads();
  f32x16 acc;
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[e] = 0.f;
#pragma unroll
  for (int kk = 0; kk < ABS_DN / 16; ++kk)
    if (16 * kk < dnp)  // uniform
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          lds_operand_tr(Ws, ABS_LD, 32 * wave, 16 * kk + 8 * half, 16 * kk + 8 * half + 4), qf[kk], acc,
          0, 0, 0);
  if constexpr (OUT == ABS_F16 || OUT == ABS_BOTH) {
    float top = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) top = fmaxf(top, fabsf(acc[e]));
    top = pair_max32(top);  // (the lane pair has the row's 32 latents of this wavefront)
    const int t = min(max((int)(__float_as_uint(top) >> 23) - 135, ABS_MIN_EXP), ABS_MAX_EXP), i = c0 / 32 + wave;
    const float down = __uint_as_float((uint32_t)(127 - t) << 23);
    if (rr >= rows) return;
    if (half == 0) exps[qi * (rkv / 32) + i] = (int8_t)t;
    bf16_t* to = qabs16 + ((int64_t)(rc / hpg) * (HP / 32) + head / 32) * rkv * 32 + head % 32 * 8;
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4)
      *(u32x2*)(to + (2 * i + (e4 & 1)) * 512 + (e4 >> 1) * 256 + 4 * half) =
          u32x2{pack2h(acc[4 * e4] * down, acc[4 * e4 + 1] * down), pack2h(acc[4 * e4 + 2] * down, acc[4 * e4 + 3] * down)};
    if constexpr (OUT == ABS_F16) return;
  }
  if (rr >= rows) return;
#pragma unroll
  for (int e4 = 0; e4 < 4; ++e4)
    *(u32x2*)(place(c0 + 32 * wave + 8 * e4) + 4 * half) = u32x2{pack2bf(acc[4 * e4], acc[4 * e4 + 1]), pack2bf(acc[4 * e4 + 2], acc[4 * e4 + 3])};
}

}  // namespace mla
