// Attention over the paged latent cache (paged.hip): single tokens in absorbed form (head i's query
// against the cache rows is [W_UK[g]^T q^nope_i ; q^rope_i], its output W_UV[g] applied to the
// attention-weighted latent, g = i / (H / G_kv)), packed prompts with keys and values written out.
#include "attn_common.h"
#include "common.h"
#include "kernels.h"

namespace mla {
namespace {

size_t al(size_t x) { return (x + 255) & ~(size_t)255; }

// ---- decoding -------------------------------------------------------------------------
// With one positional key all heads attend to the same row, so decoding is multi-query
// attention over rows of DK = r_kv + d_rope whose first DVL = r_kv values are the values too:
// every cache row is read once for all heads, 60 operations a byte at 32 heads, and the rows'
// stream bounds the kernel.
//
// * The rows of all sequences, in tiles of 32, form one list; a workgroup (one a CU) takes an
//   equal share of it, whatever the lengths, and each of its four wavefronts a quarter of the
//   share, a run of tiles that may cross from sequence to sequence.
// * A wavefront works on its run by itself: its own LDS buffer, its own softmax state (running
//   maximum and sum of each head, the weighted latents of all heads in 256 registers), no barrier
//   and no exchange.  While one wavefront waits for its copies the others multiply: about three of
//   the four 36 KB tiles of a CU are in flight at any time.
// * Where a wavefront leaves a sequence it stores the state to slot (wavefront + sequence), which
//   nobody else has: along the list one of the two grows from state to state.  Where the whole
//   share lies in one sequence the four states are joined through LDS first and only one is stored
//   (with long sequences a quarter of the traffic).
// * S^T = K Q^T has the row in the MFMA row and the head in its column, so a lane owns one head's
//   state, and the accumulator of S^T is, after the exponential, the B operand of O^T = V^T P^T
//   (the order of the rows inside a K step is the same on both sides).  V^T comes from the same
//   LDS tile by transposing reads.
//
// 64 sequences of 4096 rows of 576 values, 32 heads: 65 us, 4.7 TB/s; 2 of 100001 rows 48 us; 109683 rows
// of 41 sequences of 1 to 16001 rows 41 us, a few tiles a wavefront and a state stored for each sequence
// that it meets.  64 sequences that give each of the 1024 wavefronts 1, 2, 4, 8, 16 or 32 tiles: 20, 26, 35,
// 64, 120 and 222 us, so 5 to 7 us a tile, and about 15 us for the list, the first copies and the states (8 of
// them still seen beside many tiles).  With a workgroup or a few those take less: one sequence of 32 to 300
// rows 11 to 12 us, 8 to 9 with rows of 288 values.
//
// Precision: the absorbed queries are bf16 operands, and their rounding is what the output loses beside its
// own (2.3e-3 of the norm against 1.65e-3); probabilities and weighted latents are held as two bf16 values each,
// sums and states in fp32.
constexpr int PD_KT = 32;         // rows per tile
constexpr int PD_WAVES = 4;
constexpr float PD_SLACK = 8.f;   // log2 units the running reference maximum may lag
constexpr int PD_CUS = 256;

struct PagedDecodeDev {
  const bf16_t* pool;
  const int32_t* table;
  int n_pages, page_size, max_pages;
  const int32_t* len;
  int max_len, B, H, HP;
  const bf16_t* qabs;  // [B][HP / 32][DK / 16][64 lanes][8]: matrix operands
  float* part_o;       // [slot][HP][DVL], not normalised
  float* part_ml;      // [slot][HP][2]: reference maximum (log2), sum
  int32_t* tile_off;   // [B + 1]: first tile of each sequence in the list
  float sl2;
};

__device__ __forceinline__ int decode_len(const PagedDecodeDev& a, int b) {
  return min(max(a.len[b], 0), a.max_len);
}
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

// A tile in LDS: 32 rows of CHR 16-byte chunks, not padded; chunk c of row r lies at c ^ swz(r), which
// spreads both read patterns over the banks: 16 bytes of 16 consecutive rows (S^T, no conflicts), and
// the transposing reads' 32 bytes of four consecutive rows (V^T; the rows that share banks differ
// in chunk bit 1; two conflict cycles a read are left, 1.0e6 beside 4.1e6 active LDS cycles in 64 x 4096
// rows).  Without padding a copy's lanes meet the same chunks again after PERIOD copies (ROWS rows), so
// that the lanes' source offsets are a few registers and a copy of rows that lie together costs no
// arithmetic.
template <int DK>
struct Tile {
  static constexpr int CHR = DK / 8;
  static constexpr bool WIDE = DK / 2 % 64 == 32;  // two rows span the banks; else four
  static constexpr int ROWS = WIDE ? 8 : 16;
  static constexpr int PERIOD = ROWS * CHR / 64;
  static constexpr int HALF_COPIES = 16 * CHR / 64;  // copies of 16 rows
  static constexpr int ELEMS = PD_KT * DK;
  static_assert(DK / 2 % 64 == 32 || DK / 2 % 64 == 16, "row stride in banks");
  static_assert(CHR % (WIDE ? 8 : 4) == 0 && ROWS * CHR % 64 == 0, "whole copies");
  __device__ __forceinline__ static constexpr int swz(int r) {
    return WIDE ? (r >> 1 & 1) << 1 | (r >> 2 & 1) << 2 | (r >> 3 & 1) : r >> 2 & 3;
  }
};

// 1 KB from a uniform address plus the lanes' offsets to the LDS byte address `lds`
__device__ __forceinline__ void copy_s(uint64_t sbase, uint32_t voff, uint32_t lds) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(voff), "s"(sbase), "{m0}"(lds) : "memory");
}

template <int DK, int DVL, int OCC>
__global__ __launch_bounds__(64 * PD_WAVES, OCC) void paged_decode_kernel(PagedDecodeDev a) {
  using TL = Tile<DK>;
  constexpr int CHR = TL::CHR;
  constexpr int NKK = DK / 16, NC = DVL / 32;
  static_assert(DK % 16 == 0 && NC % 4 == 0, "decode shape");
  static_assert(NC / 2 * 2048 <= TL::ELEMS, "half of every state fits the tiles");
  constexpr int PF = 5, PV = 3;  // operand reads in flight ahead of the products of S, and of P V
  __shared__ __attribute__((aligned(1024))) bf16_t tiles[PD_WAVES][TL::ELEMS];
  __shared__ float ml[PD_WAVES][2][32];
  __shared__ int wave_sum[PD_WAVES], plan_b[PD_WAVES], plan_at[PD_WAVES];

  const int tid = threadIdx.x, lane = tid & 63, wave = wave_id();
  const int half = lane >> 5, col = lane & 31;
  const int wg = blockIdx.x, h0 = 32 * blockIdx.y;

  // the list: each thread counts the tiles of a run of sequences, a scan gives their places
  const int run = (a.B + 64 * PD_WAVES - 1) / (64 * PD_WAVES);
  const int b_lo = min(tid * run, a.B), b_hi = min(b_lo + run, a.B);
  int mine = 0;
  for (int b = b_lo; b < b_hi; ++b) mine += tiles_of(decode_len(a, b));
  int upto = mine;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int v = __shfl_up(upto, d, 64);
    if (lane >= d) upto += v;
  }
  if (lane == 63) wave_sum[wave] = upto;
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int w = 0; w < PD_WAVES; ++w) {
    if (w < wave) upto += wave_sum[w];
    total += wave_sum[w];
  }
  const ListCut cut(total, gridDim.x);
  const int t_lo = cut.lo(wg), t_hi = cut.hi(wg), per = cut.per_wave(wg);
  // the sequence of each wavefront's first tile
  const bool first = wg == 0 && blockIdx.y == 0;
  int at = upto - mine;
  if (first || (at < t_hi && at + mine > t_lo)) {
    for (int b = b_lo; b < b_hi; ++b) {
      const int n = tiles_of(decode_len(a, b));
      if (first) a.tile_off[b] = at;
#pragma unroll
      for (int w = 0; w < PD_WAVES; ++w) {
        const int t = t_lo + w * per;
        if (t < t_hi && at <= t && t < at + n) {
          plan_b[w] = b;
          plan_at[w] = at;
        }
      }
      at += n;
    }
  }
  if (first && tid == 0) a.tile_off[a.B] = total;
  __syncthreads();
  if (t_lo >= t_hi) return;

  int T = t_lo + wave * per;                       // this wavefront's run: tiles [T, T_end)
  const int T_end = min(T + per, t_hi);
  int b = 0, seq0 = 0, n = 0, nt = 0;              // the current sequence: first tile, rows, tiles
  if (T < T_end) {
    b = __builtin_amdgcn_readfirstlane(plan_b[wave]);
    seq0 = __builtin_amdgcn_readfirstlane(plan_at[wave]);
    n = __builtin_amdgcn_readfirstlane(decode_len(a, b));
    nt = tiles_of(n);
  }
  // whether the share lies in one sequence (the same in every wavefront)
  const int b_first = __builtin_amdgcn_readfirstlane(plan_b[0]);
  const bool joined = t_hi <= __builtin_amdgcn_readfirstlane(plan_at[0]) + tiles_of(__builtin_amdgcn_readfirstlane(decode_len(a, b_first)));

  const uint64_t heads = __ballot(h0 + col < a.H);  // (columns without a head move no reference)
  bf16_t* kt = tiles[wave];
  const uint32_t kt_lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)kt);

  // lane offsets: the copies' sources within ROWS rows; the operands in the tile
  uint32_t voff[TL::PERIOD];
#pragma unroll
  for (int k = 0; k < TL::PERIOD; ++k) {
    const int r = (64 * k + lane) / CHR, pc = (64 * k + lane) % CHR;
    voff[k] = 16u * (uint32_t)(r * CHR + (pc ^ TL::swz(r)));
  }
  const bf16_t* kb[4];  // row col, chunk 2 kk + half for kk % 4 = 0..3
#pragma unroll
  for (int j = 0; j < 4; ++j) kb[j] = kt + col * DK + 8 * ((2 * j + half) ^ TL::swz(col));
  // rows 4 half + (lane % 16) / 4 (+ 8), latents 16 ((lane / 16) % 2) + 4 (lane % 4) (+ 32)
  const bf16_t* vb[2][2];
#pragma unroll
  for (int h8 = 0; h8 < 2; ++h8)
#pragma unroll
    for (int odd = 0; odd < 2; ++odd) {
      const int r = 8 * h8 + 4 * half + ((lane & 15) >> 2);
      const int d = 32 * odd + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
      vb[h8][odd] = kt + r * DK + 8 * ((d >> 3) ^ TL::swz(r)) + (d & 7);
    }

  // row `col` of tile t (of its sequence) of sequence bb with nn rows (the last row again past the
  // end, which gets no weight): its page's table entry, and its address
  auto entry = [&](int bb, int t, int nn) {
    const int p = min(t * PD_KT + col, nn - 1);
    return a.table[(int64_t)bb * a.max_pages + p / a.page_size];
  };
  auto address = [&](int t, int nn, int page, bool& bad) {
    const int p = min(t * PD_KT + col, nn - 1);
    const bool out = page < 0 || page >= a.n_pages;
    bad = __ballot(out) != 0;
    return (uint64_t)(uintptr_t)(a.pool + ((int64_t)(out ? 0 : page) * a.page_size + p % a.page_size) * DK);
  };
  auto row_address = [&](uint64_t at, int r) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)at, r) |
           (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(at >> 32), r) << 32;
  };
  // rows 16 g .. 16 g + 15 of a tile whose 16 rows lie together
  auto issue_half = [&](int g, uint64_t at) __attribute__((always_inline)) {
    uint64_t base = row_address(at, 16 * g);
    asm volatile("s_nop 4" : "+s"(base));  // (vector ALU to scalar register to memory operation)
    uint32_t lds = kt_lds;  // opaque: its sums with constants are cheaper made again than kept
    asm volatile("" : "+s"(lds));
#pragma unroll
    for (int k = 0; k < TL::HALF_COPIES; ++k) {
      const int q = k / TL::PERIOD;
      uint32_t v = voff[k % TL::PERIOD];
      if (TL::WIDE && (q & 1)) asm volatile("v_xor_b32 %0, 16, %0" : "+v"(v));  // (again, not kept)
      copy_s(base + (uint64_t)(q * TL::ROWS * DK * 2), v, lds + 2 * (16 * g * DK + 512 * k));
    }
  };
  // any tile: copy k fills chunks 64 k .. 64 k + 63, of rows known at compile time
  auto issue_rows = [&](uint64_t at) __attribute__((always_inline)) {
    int ln = lane;  // opaque: the lanes' chunk numbers are cheaper made again than kept in registers
    asm volatile("" : "+v"(ln));
#pragma unroll
    for (int k = 0; k < 2 * TL::HALF_COPIES; ++k) {
      const int r0 = 64 * k / CHR, skip = 64 * k % CHR;
      uint64_t src = 0;
      int c = 0;
#pragma unroll
      for (int r = 0; r * CHR < skip + 64; ++r) {  // the rows that 64 chunks touch
        const uint64_t base = row_address(at, r0 + r);
        const int pc = ln + skip - r * CHR;
        if (r == 0 || pc >= 0) {
          src = base;
          c = pc ^ TL::swz(r0 + r);
        }
      }
      dma16((const bf16_t*)(uintptr_t)(src + 16u * (uint32_t)c), kt + 512 * k);
      __builtin_amdgcn_sched_barrier(0);  // (or every row's address waits in scalar registers)
    }
  };
  // whether 16-row halves of whole tiles lie together
  const bool whole16 = a.page_size % 16 == 0;

  bool bad = false, any_bad = false;
  bf16x8 qf[NKK];  // this lane's head as B operand fragments (k = 16 kk + 8 half + 0..7)
  auto load_q = [&](int bb) __attribute__((always_inline)) {
    const bf16_t* qsrc = a.qabs + ((int64_t)bb * a.HP + h0) * DK + 8 * lane;
#pragma unroll
    for (int kk = 0; kk < NKK; ++kk) qf[kk] = *(const bf16x8*)(qsrc + 512 * kk);
  };
  if (T < T_end) issue_rows(address(T - seq0, n, entry(b, T - seq0, n), bad));
  else if (!joined) return;

  do {  // a sequence's part of the run
    const int seg_end = min(T_end, seq0 + nt);
    int b2 = b, n2 = n, seq2 = seq0;  // the sequence after it
    const int seg_begin = T;
    any_bad = false;
    if (T < seg_end) load_q(b);
    f32x16 acc[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[c][e] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;

    for (; T < seg_end; ++T) {
      any_bad |= bad;
      const int t = T - seq0;
      // the tile after this one: the next of the sequence, or the first of the next that has rows
      int page = 0;
      if (T + 1 < T_end) {
        if (T + 1 == seg_end) {
          seq2 += nt;
          do n2 = __builtin_amdgcn_readfirstlane(decode_len(a, ++b2));
          while (n2 == 0);
        }
        page = entry(b2, T + 1 - seq2, n2);
      }
      wait_vm<0>();
      // S^T, the operand reads PF ahead of the products (pinned: the compiler would read each operand
      // right before its product and wait for it)
      f32x16 s;
      {
        bf16x8 kf[PF];
        auto kread = [&](int kk) { return *(const bf16x8*)(kb[kk % 4] + 64 * (kk / 4)); };
#pragma unroll
        for (int j = 0; j < PF; ++j) kf[j] = kread(j);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kk = 0; kk < NKK; ++kk) {
          if (kk == 0) mfma_v_first(s, kf[0], qf[0]);
          else mfma_v_next(s, kf[kk % PF], qf[kk]);
          if (kk + PF < NKK) kf[kk % PF] = kread(kk + PF);
          __builtin_amdgcn_sched_barrier(0);
        }
        mfma_v_done(s);
      }
      // V^T operand of step j = NC u + c: latents 32 c .., rows 16 u + {4 half.., 8 + 4 half..}
      auto vread = [&](int j) {
        const int c = j % NC, at = 16 * (j / NC) * DK + 64 * (c / 2);
        const u32x2 lo = lds_read_tr4(vb[0][c & 1] + at), hi = lds_read_tr4(vb[1][c & 1] + at);
        return __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
      };
      bf16x8 vf[PV];
#pragma unroll
      for (int j = 0; j < PV; ++j) vf[j] = vread(j);
      // rows past the end (the last tile only; a real branch): no weight
      if (t * PD_KT > n - PD_KT) {
        asm volatile("");
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (t * PD_KT + 8 * (e >> 2) + 4 * half + (e & 3) >= n) s[e] = -INFINITY;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[e]);
      mx = pair_max32(mx) * a.sl2;
      // the reference moves only when a tile's maximum exceeds it by more than PD_SLACK (P <= 2^8)
      if ((__ballot(mx > m_run + PD_SLACK) & heads) != 0) {
        const float m_new = fmaxf(m_run, mx);
        const float corr = __builtin_amdgcn_exp2f(m_run - (m_new == -INFINITY ? 0.f : m_new));
        m_run = m_new;
        l_run *= corr;
        if (T != seg_begin) {  // (nothing is there yet at the first tile)
#pragma unroll
          for (int c = 0; c < NC; ++c) acc_scale(acc[c], corr);
        }
      }
      const float m_use = m_run == -INFINITY ? 0.f : m_run;
      // P as two bf16 operands, rounded and what that lost: a rounding of P alone would add as much
      // error as that of the output, and the second products hide behind the copies
      bf16x8 pf[2], pl[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        u32x4 w, w2;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * u + 2 * q], a.sl2, -m_use));
          const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * u + 2 * q + 1], a.sl2, -m_use));
          l_run += p0 + p1;
          w[q] = pack2bf(p0, p1);
          w2[q] = pack2bf(p0 - __uint_as_float(w[q] << 16), p1 - __uint_as_float(w[q] & 0xffff0000u));
        }
        pf[u] = __builtin_bit_cast(bf16x8, w);
        pl[u] = __builtin_bit_cast(bf16x8, w2);
      }
      __builtin_amdgcn_sched_barrier(0);
      // the next tile's first 16 rows are asked for as soon as those of this one have been read (LDS
      // reads return in order: that of step NC is there), the others behind the last read
      const bool more = T + 1 < T_end;
      uint64_t at = 0;
      bool together = false;
      if (more) {
        at = address(T + 1 - seq2, n2, page, bad);
        together = whole16 && (T + 1 - seq2) * PD_KT <= n2 - PD_KT;
      }
#pragma unroll
      for (int j = 0; j < 2 * NC; ++j) {
        mfma_a(acc[j % NC], vf[j % PV], pf[j / NC]);
        mfma_a(acc[j % NC], vf[j % PV], pl[j / NC]);
        if (j + PV < 2 * NC) vf[j % PV] = vread(j + PV);
        __builtin_amdgcn_sched_barrier(0);
        if (j == NC) {
          mfma_a_done(acc);  // (no branch, where the compiler may move registers, before the products' waits)
          if (together) issue_half(0, at);
        }
      }
      mfma_a_done(acc);
      // every read of the tile has returned before the next copies may overwrite it
      asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
      if (more) {
        if (together) issue_half(1, at);
        else issue_rows(at);
      }
    }

    if (!joined) {  // leaving the sequence: its state
      const float l = any_bad ? NAN : pair_sum32(l_run);  // (a row on no page)
      if (h0 + col < a.H) {
        const int64_t row = ((int64_t)PD_WAVES * wg + wave + b) * a.HP + h0 + col;
        // lane (head col, half) holds latents 32 c + 8 g + 4 half + 0..3
        float* po = a.part_o + row * DVL + 4 * half;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            *(f32x4*)(po + 32 * c + 8 * g) =
                f32x4{acc[c][4 * g], acc[c][4 * g + 1], acc[c][4 * g + 2], acc[c][4 * g + 3]};
        if (half == 0) {
          a.part_ml[2 * row] = m_run;
          a.part_ml[2 * row + 1] = l;
        }
      }
      b = b2;
      n = n2;
      seq0 = seq2;
      nt = tiles_of(n);
      continue;
    }

    // the four states of one sequence: one reference and sum, then the latents, half of them at a time
    // through LDS: every wavefront writes its half, then sums a quarter of it
    const float l = any_bad ? NAN : pair_sum32(l_run);
    if (half == 0) {
      ml[wave][0][col] = m_run;
      ml[wave][1][col] = l;
    }
    float* buf = (float*)tiles[0];
    constexpr int NH = NC / 2;
    float M = -INFINITY, L = 0.f, f[PD_WAVES];
    const int64_t row = ((int64_t)PD_WAVES * wg + b_first) * a.HP + h0 + col;
    float* po = a.part_o + row * DVL + 4 * half;
#pragma unroll
    for (int ph = 0; ph < 2; ++ph) {
      __syncthreads();  // (every wavefront is done with its tile, or with the first half)
      if (ph == 0) {
#pragma unroll
        for (int w = 0; w < PD_WAVES; ++w) M = fmaxf(M, ml[w][0][col]);
#pragma unroll
        for (int w = 0; w < PD_WAVES; ++w) {
          const float mw = ml[w][0][col];
          f[w] = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw - M);
          L += ml[w][1][col] * f[w];
        }
      }
#pragma unroll
      for (int c = 0; c < NH; ++c)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x16& v = acc[ph * NH + c];
          *(f32x4*)(buf + (((wave * NH + c) * 4 + g) * 64 + lane) * 4) = f32x4{v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]};
        }
      __syncthreads();
#pragma unroll
      for (int c0 = 0; c0 < NH; c0 += PD_WAVES) {
        const int c = c0 + wave;
        if (c < NH) {
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < PD_WAVES; ++w) v += *(const f32x4*)(buf + (((w * NH + c) * 4 + g) * 64 + lane) * 4) * f[w];
            if (h0 + col < a.H) *(f32x4*)(po + 32 * (ph * NH + c) + 8 * g) = v;
          }
        }
      }
    }
    if (wave == 0 && half == 0 && h0 + col < a.H) {
      a.part_ml[2 * row] = M;
      a.part_ml[2 * row + 1] = L;
    }
  } while (!joined && T < T_end);
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
// of its first workgroup (one if that is joined), one for each workgroup inside, the last in those
// of its last workgroup.
struct States {
  int n = 0, n0 = 0, mid = 0, at0 = 0, at_mid = 0, at1 = 0;
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
      at_mid = PD_WAVES * (w0 + 1) + b;
      n += mid + part(cut, w1, t0, t1, v);
      at1 = PD_WAVES * w1 + v + b;
    }
  }
  __device__ __forceinline__ static int part(const ListCut& cut, int w, int t0, int t1, int& v) {
    const int lo = cut.lo(w), hi = cut.hi(w), per = cut.per_wave(w);
    v = 0;
    if (t0 <= lo && hi <= t1) return 1;  // joined
    v = (max(t0, lo) - lo) / per;
    return (min(t1, hi) - 1 - lo) / per - v + 1;
  }
  __device__ __forceinline__ int slot(int k) const {
    if (k < n0) return at0 + k;
    k -= n0;
    if (k < mid) return at_mid + PD_WAVES * k;
    return at1 + k - mid;
  }
};

template <int DVL, int DV, int HB, int RB>
__global__ __launch_bounds__(PF_THREADS) void paged_finish_kernel(const float* __restrict__ part_o,
                                                                  const float* __restrict__ part_ml,
                                                                  const int32_t* __restrict__ tile_off,
                                                                  const bf16_t* __restrict__ Wuv,
                                                                  bf16_t* __restrict__ o, int B, int H, int HP,
                                                                  int nwg, int hpg) {
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
  const ListCut cut(tile_off[B], nwg);
  States st;
  if (b < B) st = States(cut, b, tile_off[b], tile_off[b + 1]);
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
        const int64_t rw = (int64_t)st.slot(k) * HP + i0 + h;
        x[u] = *(const f32x4*)(part_o + rw * DVL + 4 * cg);
        ml[u] = *(const f32x2*)(part_ml + 2 * rw);
      }
    }
    float m1 = M;
#pragma unroll
    for (int u = 0; u < U; ++u) m1 = fmaxf(m1, ml[u][0]);
    const float ref = m1 == -INFINITY ? 0.f : m1, c = __builtin_amdgcn_exp2f(M - ref);
    v *= c;
    L *= c;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float w = __builtin_amdgcn_exp2f(ml[u][0] - ref);
      v += x[u] * w;
      L += ml[u][1] * w;
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
        const float f = __builtin_amdgcn_exp2f(sm[col][k] - ref);
        v += *(const f32x4*)&red[grp + k][4 * cg] * f;
        L += sl[col][k] * f;
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

// Workgroups over the list, for each block of 32 heads: one a CU in all, and no more than have a
// tile for each wavefront at the largest lengths.
int decode_workgroups(int B, int H, int max_len) {
  const int hb = (H + 31) / 32;
  const int64_t tiles = (int64_t)B * ((max_len + (int64_t)PD_KT - 1) / PD_KT);
  const int64_t most = PD_CUS / hb > 1 ? PD_CUS / hb : 1;
  const int64_t n = (tiles + PD_WAVES - 1) / PD_WAVES;
  return (int)(n < most ? n : most);
}

struct DecodeLayout {
  size_t qabs, part_o, part_ml, tile_off, bytes;
};
DecodeLayout decode_layout(int B, int H, int DK, int DVL, int nwg) {
  const size_t HP = (H + 31) / 32 * 32, slots = (size_t)PD_WAVES * nwg + B;
  DecodeLayout l;
  l.qabs = 0;
  l.part_o = l.qabs + al(B * HP * DK * 2);
  l.part_ml = l.part_o + al(slots * HP * DVL * 4);
  l.tile_off = l.part_ml + al(slots * HP * 2 * 4);
  l.bytes = l.tile_off + al(((size_t)B + 1) * 4);
  return l;
}

// (DK, DVL, workgroups a CU: what LDS and registers hold)
#define MLA_PAGED_SHAPES(X) X(576, 512, 1) X(288, 256, 1) X(160, 128, 2)

}  // namespace

size_t decode_paged_ws_bytes(int B, int H, int DK, int DVL, int max_len) {
  return decode_layout(B, H, DK, DVL, decode_workgroups(B, H, max_len)).bytes;
}

hipError_t decode_paged(const DecodePaged& d, hipStream_t s) {
  const int HP = (d.H + 31) / 32 * 32, DK = d.rkv + d.dr, DVL = d.rkv;
  const int nwg = decode_workgroups(d.B, d.H, d.max_len);
  const DecodeLayout l = decode_layout(d.B, d.H, DK, DVL, nwg);
  char* ws = (char*)d.ws;
  PagedDecodeDev a;
  a.pool = (const bf16_t*)d.c.pool; a.table = d.c.table; a.n_pages = d.c.n_pages;
  a.page_size = d.c.page_size; a.max_pages = d.c.max_pages; a.len = d.len; a.max_len = d.max_len;
  a.B = d.B; a.H = d.H; a.HP = HP; a.qabs = (const bf16_t*)(ws + l.qabs);
  a.part_o = (float*)(ws + l.part_o); a.part_ml = (float*)(ws + l.part_ml);
  a.tile_off = (int32_t*)(ws + l.tile_off); a.sl2 = d.scale * attn::LOG2E;
  hipError_t e = decode_absorb(d.q, d.Wuk, ws + l.qabs, d.B, d.H, HP, d.hpg, d.dn, d.dr, d.rkv, true, s);
  if (e != hipSuccess) return e;
  // algorithmic work at full lengths
  prof_begin(KC_ATTN_FWD, s);
#define X(a_, b_, c_) \
  if (DK == a_ && DVL == b_) paged_decode_kernel<a_, b_, c_><<<dim3(nwg, HP / 32), 64 * PD_WAVES, 0, s>>>(a);
  MLA_PAGED_SHAPES(X)
#undef X
  prof_end(KC_ATTN_FWD, s, 2.0 * d.B * d.H * (double)d.max_len * (DK + DVL), (double)d.B * d.max_len * DK * 2,
           KLABEL("paged_decode_kernel"));
  prof_begin(KC_ELEM, s);
  // One column a workgroup while that is one round on the CUs, else eight that share W_UV (four heads of two
  // sequences, or one of eight where a group's heads are no multiple of four): 64 columns of many states
  // 9.7 us by one, 38 by eight; 2048 columns 36 us by one, 8.2 by eight.
  const bool few = (int64_t)d.B * d.H <= PD_CUS, heads4 = d.hpg % 4 == 0;
#define FIN(b_, v_, hb_, rb_)                                                                             \
  paged_finish_kernel<b_, v_, hb_, rb_><<<dim3(d.H / hb_, (d.B + rb_ - 1) / rb_), PF_THREADS, 0, s>>>(    \
      a.part_o, a.part_ml, a.tile_off, (const bf16_t*)d.Wuv, (bf16_t*)d.o, d.B, d.H, HP, nwg, d.hpg)
#define FINV(b_, v_)           \
  if (few) FIN(b_, v_, 1, 1);  \
  else if (heads4) FIN(b_, v_, 4, 2); \
  else FIN(b_, v_, 1, 8)
#define X(a_, b_, c_)          \
  if (DK == a_ && DVL == b_) { \
    if (d.dv == 128) {         \
      FINV(b_, 128);           \
    } else {                   \
      FINV(b_, 64);            \
    }                          \
  }
  MLA_PAGED_SHAPES(X)
#undef X
#undef FINV
#undef FIN
  prof_end(KC_ELEM, s, 2.0 * d.B * d.H * d.dv * d.rkv, ((double)nwg + d.B) * d.H * (DVL + 2) * 4,
           KLABEL("paged_finish_kernel"));
  return hipGetLastError();
}

// ---- prefill --------------------------------------------------------------------------
// With many queries per cached row the keys W_UK c and values W_UV c are written out once (as for
// the contiguous cache) and the attention runs on heads of d_nope + d_rope and d_k: gather, one
// grouped product, attention over the packed sequences.  Keys are bf16, whose rounding is most of what the
// output loses beside its own (2.2e-3 of the norm against 1.65e-3), values and probabilities fp16 (3e-5).
namespace {

// The cached rows of all sequences behind one another, and what the products need; a wavefront per row.
//
// Values are expanded to fp16, whose 11 bits make their rounding an eighth of bf16's, in a range that
// fits by scaling with powers of two: row n of the latents by 2^-e[n], e a multiple of 16 in [-64, 64] (0
// where the row's largest value lies in [2^-8, 2^8), which it is brought to), row d of W_UV to a largest
// value in [1/8, 1/4) (v_scale[d] undoes it).  A scaled value is then below rkv 2^8 / 4 <= 2^15, and
// typically above 2^-9, in fp16's normal range.  Both scalings are exact in bf16 but for values that
// vanish beside a row's largest (2^-100).
//
// Masked keys get P = 0, which keeps a row out of a product only if its values are finite.  So a row
// that is not finite, has a latent of 2^72 or more or lies on no page becomes zeros with a NaN positional
// key: its values and non-positional key are 0 and its logits NaN, for exactly the queries that see it.
// Rows of no sequence become zeros.  Bound by memory (14083 rows of 576 values 10.9 us, 4.4 TB/s) and, for
// few rows, by three dependent loads (77 rows 3.4 us).
constexpr int GATHER_EXP = 64;  // largest |e|
constexpr int GATHER_TOP = 127 + GATHER_EXP + 8;  // exponent field of the first latent too large
struct GatherDev {
  PagedPool c;
  const int32_t* kv_off;
  int B, n_kv, rkv, nv;
  const bf16_t* Wuv;
  bf16_t* rows;      // [n_kv][width]
  bf16_t* lat;       // [n_kv][width], scaled latents (rows as far apart as the rows': products of alike operands)
  float* key_exp;    // [n_kv]: e
  bf16_t* W;         // [nv][rkv], scaled
  float* v_scale;    // [nv]
};
// the largest exponent field among a lane's 8 values
__device__ __forceinline__ uint32_t top_exponent(u32x4 v) {
  uint32_t top = 0u;
#pragma unroll
  for (int q = 0; q < 4; ++q) top = max(top, max(v[q] << 16 & 0x7f800000u, v[q] & 0x7f800000u));
  return top >> 23;
}
__device__ __forceinline__ int wave_max(int x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x = max(x, __shfl_xor(x, d, 64));
  return x;
}
// 8 values times 2^k (|k| <= 127; in two steps, as 2^-127 is no normal number)
__device__ __forceinline__ u32x4 scaled(u32x4 v, int k) {
  const float f = __uint_as_float((uint32_t)(127 + k / 2) << 23), f2 = __uint_as_float((uint32_t)(127 + k - k / 2) << 23);
  u32x4 o;
#pragma unroll
  for (int q = 0; q < 4; ++q)
    o[q] = pack2bf(__uint_as_float(v[q] << 16) * f * f2, __uint_as_float(v[q] & 0xffff0000u) * f * f2);
  return o;
}
__global__ __launch_bounds__(256) void gather_rows_kernel(GatherDev a) {
  const int row = 4 * blockIdx.x + wave_id(), lane = threadIdx.x & 63;
  const PagedPool& c = a.c;
  const bool in_lat = 8 * lane < a.rkv;
  const u32x4 zero = {0u, 0u, 0u, 0u};
  const int rows4 = (a.n_kv + 3) / 4 * 4;
  if (row >= rows4) {  // a row of W_UV
    const int e = row - rows4;
    if (e >= a.nv) return;
    u32x4 w = zero;
    if (in_lat) w = *(const u32x4*)(a.Wuv + (int64_t)e * a.rkv + 8 * lane);
    const int k = max(min(wave_max((int)top_exponent(w)) - 127, 124), -100) + 3;
    if (in_lat) *(u32x4*)(a.W + (int64_t)e * a.rkv + 8 * lane) = scaled(w, -k);
    if (lane == 0) a.v_scale[e] = __uint_as_float((uint32_t)(127 + k) << 23);
    return;
  }
  if (row >= a.n_kv) return;
  const int dr = c.width - a.rkv;
  bf16_t* dst = a.rows + (int64_t)row * c.width;
  u32x4 lat = zero, pe = zero;
  const bool in_pe = 8 * lane < dr;
  int top = 0;
  if (row >= a.kv_off[0] && row < a.kv_off[a.B]) {  // (uniform)
    int lo = 0, hi = a.B - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.kv_off[mid] <= row) lo = mid;
      else hi = mid - 1;
    }
    const int p = row - a.kv_off[lo], pg = p / c.page_size;
    const int page = p >= 0 && pg < c.max_pages ? c.table[(int64_t)lo * c.max_pages + pg] : -1;
    bool any = page < 0 || page >= c.n_pages;
    if (!any) {
      const bf16_t* src = (const bf16_t*)c.pool + ((int64_t)page * c.page_size + p % c.page_size) * c.width;
      if (in_lat) lat = *(const u32x4*)(src + 8 * lane);
      if (in_pe) pe = *(const u32x4*)(src + a.rkv + 8 * lane);
      top = wave_max((int)top_exponent(lat));
      any = __ballot(top >= GATHER_TOP || top_exponent(pe) == 255u) != 0;
    }
    if (any) {
      lat = zero;
      top = 0;
      pe = u32x4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
    }
  }
  const int e = top == 0 ? 0 : max((top - 127 + 8) >> 4 << 4, -GATHER_EXP);
  if (in_lat) {
    *(u32x4*)(dst + 8 * lane) = lat;
    *(u32x4*)(a.lat + (int64_t)row * c.width + 8 * lane) = scaled(lat, -e);
  }
  if (in_pe) *(u32x4*)(dst + a.rkv + 8 * lane) = pe;
  if (lane == 0) a.key_exp[row] = (float)e;
}

struct PrefillLayout {
  size_t rows, lat, key_exp, W, v_scale, keys, vals, split, split_elems, bytes;
};
Gemm expand(const PrefillPaged& p, const void* rows, const void* W, int n, void* out, DType t) {
  Gemm g;
  g.M = p.n_kv; g.N = n; g.K = p.rkv;
  g.A = rows; g.lda = p.rkv + p.dr; g.a_kmajor = true;
  g.B = W; g.ldb = p.rkv; g.b_kmajor = true;
  g.C = out; g.ldc = n; g.in_t = DT_BF16; g.c_t = t; g.alpha = 1.f; g.beta = 0.f;
  return g;
}
AttnPacked packed_attention(const PrefillPaged& p, const PrefillLayout& l, char* ws) {
  const void *rows = ws + l.rows, *keys = ws + l.keys, *vals = ws + l.vals;
  AttnPacked a;
  a.key_exp = (const float*)(ws + l.key_exp); a.v_scale = (const float*)(ws + l.v_scale);
  const int W = p.rkv + p.dr, dqk = p.dn + p.dr, hpg = p.H / p.G;
  const bf16_t* kpe = (const bf16_t*)rows + p.rkv;
  a.B = p.B; a.H = p.H; a.dqk = dqk; a.dv = p.dv;
  a.dnope = p.dn > 0 ? p.dn : dqk;  // (no non-positional keys: the positional key is the whole key)
  a.Q = HeadView{p.q, (int64_t)p.H * dqk, dqk, 1};
  a.Ka = p.dn > 0 ? HeadView{keys, (int64_t)p.G * p.dn, p.dn, hpg} : HeadView{kpe, W, 0, p.H};
  a.Kb = HeadView{kpe, W, 0, p.H};
  a.V = HeadView{vals, (int64_t)p.G * p.dv, p.dv, hpg};
  a.O = p.o; a.o_tok = (int64_t)p.H * p.dv; a.scale = p.scale;
  a.q_off = p.q_off; a.kv_off = p.kv_off; a.n_q = p.n_q; a.n_kv = p.n_kv;
  a.ws = ws + l.split;  // (the products' partials are done with)
  return a;
}
PrefillLayout prefill_layout(const PrefillPaged& p) {
  PrefillLayout l;
  l.rows = 0;
  l.lat = l.rows + al((size_t)p.n_kv * (p.rkv + p.dr) * 2);
  l.key_exp = l.lat + al((size_t)p.n_kv * (p.rkv + p.dr) * 2);
  l.W = l.key_exp + al((size_t)p.n_kv * 4);
  l.v_scale = l.W + al((size_t)p.G * p.dv * p.rkv * 2);
  l.keys = l.v_scale + al((size_t)p.G * p.dv * 4);
  l.vals = l.keys + al((size_t)p.n_kv * p.G * p.dn * 2);
  l.split_elems = 0;  // partials of the products
  if (p.n_kv > 0) {
    if (p.dn > 0) l.split_elems = gemm_scratch_elems(expand(p, nullptr, nullptr, p.G * p.dn, nullptr, DT_BF16));
    const size_t v = gemm_scratch_elems(expand(p, nullptr, nullptr, p.G * p.dv, nullptr, DT_F16));
    if (v > l.split_elems) l.split_elems = v;
  }
  l.split = l.vals + al((size_t)p.n_kv * p.G * p.dv * 2);
  const size_t parts = attn_packed_ws_bytes(packed_attention(p, l, nullptr));
  l.bytes = l.split + al(l.split_elems * 4 > parts ? l.split_elems * 4 : parts);
  return l;
}

}  // namespace

size_t prefill_paged_ws_bytes(const PrefillPaged& p) {
  const size_t n = prefill_layout(p).bytes;
  return n > 256 ? n : 256;
}

hipError_t prefill_paged(const PrefillPaged& p, hipStream_t s) {
  const PrefillLayout l = prefill_layout(p);
  char* ws = (char*)p.ws;
  const int W = p.rkv + p.dr, nk = p.G * p.dn, nv = p.G * p.dv;
  prof_begin(KC_ELEM, s);
  GatherDev g;
  g.c = p.c; g.kv_off = p.kv_off; g.B = p.B; g.n_kv = p.n_kv; g.rkv = p.rkv; g.nv = nv;
  g.Wuv = (const bf16_t*)p.Wuv; g.rows = (bf16_t*)(ws + l.rows); g.lat = (bf16_t*)(ws + l.lat);
  g.key_exp = (float*)(ws + l.key_exp); g.W = (bf16_t*)(ws + l.W); g.v_scale = (float*)(ws + l.v_scale);
  gather_rows_kernel<<<(p.n_kv + 3) / 4 + (nv + 3) / 4, 256, 0, s>>>(g);
  prof_end(KC_ELEM, s, 0.0, ((double)p.n_kv * (2 * W + p.rkv) + 2.0 * nv * p.rkv) * 2, KLABEL("gather_rows_kernel"));
  if (p.n_kv > 0) {
    Gemm up[2];
    int n = 0;
    if (p.dn > 0) up[n++] = expand(p, ws + l.rows, p.Wuk, nk, ws + l.keys, DT_BF16);
    up[n++] = expand(p, ws + l.lat, ws + l.W, nv, ws + l.vals, DT_F16);
    const hipError_t e = gemm_group(up, n, (float*)(ws + l.split), l.split_elems, s);
    if (e != hipSuccess) return e;
  }
  return attn_fwd_packed(packed_attention(p, l, ws), s);
}

}  // namespace mla
