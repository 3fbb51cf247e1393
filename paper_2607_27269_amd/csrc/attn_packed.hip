// Causal softmax attention over packed sequences of different lengths on gfx950 matrix cores (bf16
// operands, fp32 softmax): prompts that arrived together, or new tokens after cached ones.
//
// A workgroup (8 wavefronts) owns 256 (query, head) pairs of one sequence: HG heads that share their
// keys and values times 256 / HG queries; a wavefront has 32 queries of one head.  The queries of a
// sequence stand at the last positions of its keys: query t sees keys 0 .. t + diag, diag = keys -
// queries (negative where there are fewer keys: the first queries see none and give 0).
//
// Query tiles are numbered without a scan over the lengths: sequence b owns the numbers from
// q_off[b] / BQH + b, at least as many as it has tiles, and the few others are empty.
//
// Keys and values stream through three LDS stages of 64 keys.  S^T = K Q^T has the key in the MFMA row
// and the query in its column, so a lane owns a query's state and the exponential of its accumulator
// is the B operand of O^T = V^T P^T as it lies (V^T by transposing LDS reads).  The loop goes by 32
// keys: the products of the next 32 keys' logits are issued between the exponentials of the present
// ones, each operand read PK ahead of its product.  That order is pinned, chunk by chunk: left to
// itself the compiler reads an operand right before its product and waits for LDS each time.  The
// reference maximum moves only when a block exceeds it by 2^8.
//
// 5505 tokens of 6 sequences, 32 heads of 192 and 128: 125 us, 660 TFLOP/s of the causal pairs; 463 tokens
// after 13620 cached ones, heads of 128 and 64: 44 us, and 7.4 to join 5 parts.  With a workgroup on every CU
// (2048 queries of 32 heads, up to 65536 rows before them) a tile of 64 keys takes 2.4 to 2.9 us at widths
// 192 and 128, 1.85 at 128 and 64.  No unit is busy all the time: in the first call the matrix cores 36 %, the
// vector ALU 33 %, LDS 25 % and 7 % more in bank conflicts.  The rest are waits in the chain from logits to
// probabilities to products, which two wavefronts a SIMD do not cover.
//
// The values and the probabilities are fp16 operands: with bf16 ones their two roundings were most of
// the output's squared error (2.9e-3 of its norm; 2.0 to 2.2e-3 now), at the same rate.  fp16 has the range for it because each
// row of values is scaled by a power of two 2^-e[n] and each column by another.  The row's goes into the
// exponent: with x' = x + e[n], P' = 2^(x' - m) is the weight of the scaled row, m the reference maximum
// of x'.  P' is at most 2^(PA_SLACK + PA_UP), and what fp16 cannot hold lies 2^-(24 + PA_UP) below a row's
// largest.  The sum's terms are 2^(x - m), by an exponential of their own: P' 2^-e[n] would be 0 for rows of
// small latents under a reference that rows of large ones set, where P' is below fp32's range and the term is
// not.  As |e| <= 64, the row at the reference keeps the sum above 2^(PA_UP - 64), and no term exceeds
// 2^(PA_UP + PA_SLACK + 64); the reference may move by more than 2^126 at once, so the sum is scaled by two
// factors.  Keys whose e are all 0 (any cache with latents of ordinary size) take a loop without them: 125 us
// against 144 in the first call above.
//
// Few queries over many keys leave CUs idle: the keys are then cut into nsplit parts per query tile,
// each with a result of its own (fp32), and a second launch joins them.
#include "attn_common.h"
#include "mfma.h"

namespace mla {
namespace attn {
namespace {

constexpr int PA_WAVES = 8;
constexpr int PA_BQ = 32 * PA_WAVES;
constexpr float PA_SLACK = 8.f;  // log2 units the running reference maximum may lag
constexpr float PA_UP = 7.f;     // P' = 2^PA_UP at the reference

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

struct PackedDev {
  int B, H, dnope;
  float sl2;  // softmax scale * log2(e)
  const bf16_t* Q; int64_t q_tok; int q_head;
  const bf16_t* Ka; int64_t ka_tok; int ka_head; int ka_div;
  const bf16_t* Kb; int64_t kb_tok; int kb_head; int kb_div;
  const bf16_t* V; int64_t v_tok; int v_head; int v_div;  // (fp16: copied as 16-bit values)
  const float *key_exp, *v_scale;  // e of each key, the factor of each column of values
  float bias;  // 1 / sl2
  bf16_t* O; int64_t o_tok;
  const int32_t *q_off, *kv_off;
  int n_q, n_kv, nqb, nsplit;
  float* part_o;   // [nsplit][n_q][H][DV], not normalised
  float* part_ml;  // [nsplit][n_q][H][2]: reference maximum (log2), sum
};

// A tile of 64 rows in LDS, not padded: 16-byte chunk c of row r lies at c ^ swz(r), which spreads what one
// read takes over the banks.  Keys: 16 bytes of 16 consecutive rows.  Values: the transposing reads' 32 bytes
// of four consecutive rows (pairs of chunks stay pairs); each of them still counts two conflict cycles (4.2e6
// beside 15.0e6 active LDS cycles in 5505 tokens), the keys' reads none.
template <int D>
struct KeySwz {
  static constexpr int BANKS = D / 2 % 64;  // row stride
  static_assert(BANKS % 16 == 0 && (BANKS != 0 || D % 128 == 0), "row stride in banks");
  // chunk bits that it changes
  static constexpr int BITS = BANKS == 0 ? 4 : BANKS == 32 ? 3 : 2;
  static_assert(D / 8 % (1 << BITS) == 0, "chunks stay in their row");
  __device__ __forceinline__ static int swz(int r) { return BANKS == 0 ? r & 15 : BANKS == 32 ? r >> 1 & 7 : r >> 2 & 3; }
};
template <int D>
struct ValueSwz {
  static_assert(D == 64 || D == 128, "row stride in banks");
  __device__ __forceinline__ static int swz(int r) { return D == 128 ? (r & 3) << 1 : (r >> 1 & 1) << 1; }
};

// x 2^d, d <= 0, by two factors: one alone is 0 below 2^-126, the product may not be
__device__ __forceinline__ float scaled_down(float x, float d) {
  return x * __builtin_amdgcn_exp2f(fmaxf(d, -126.f)) * __builtin_amdgcn_exp2f(fminf(d + 126.f, 0.f));
}

// 64 values of 4 bytes from the lanes' addresses to consecutive LDS words
__device__ __forceinline__ void dma4(const float* src, float* lds) {
  const uint32_t l = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)lds);
  asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(src), "{m0}"(l) : "memory");
}

// A tile's copies by one wavefront: each lane's source, which moves on by 64 rows a tile.
template <int D, class SWZ>
struct RowStream {
  static constexpr int CHR = D / 8, NBLK = BKV * CHR / 64, PER = (NBLK + PA_WAVES - 1) / PA_WAVES;
  static constexpr int ELEMS = BKV * D;
  const bf16_t* p[PER];
  int step[PER];  // bytes from row to row
  int row[PER];

  // element (r, c) of the sequence at src(c) + r * tok(c)
  template <class S, class K>
  __device__ __forceinline__ void init(S src, K tok, int64_t row0) {
    const int lane = threadIdx.x & 63, wave = wave_id();
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int idx = min(wave + k * PA_WAVES, NBLK - 1) * 64 + lane;
      row[k] = idx / CHR;
      const int c = 8 * ((idx % CHR) ^ SWZ::swz(row[k]));
      const int64_t t = tok(c);
      p[k] = src(c) + (row0 + row[k]) * t;
      step[k] = (int)(2 * t);
    }
  }
  // the next tile, whose first row is j0, into LDS; rows past `last` repeat it (finite values that get
  // no weight)
  __device__ __forceinline__ void next(bf16_t* lds, int j0, int last) {
    const int wave = wave_id();
    const bool whole = j0 + BKV - 1 <= last;  // (uniform)
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int b = wave + k * PA_WAVES;
      const char* src = (const char*)p[k];
      if (!whole) {
        asm volatile("");
        src -= (int64_t)max(j0 + row[k] - last, 0) * step[k];
      }
      if (NBLK % PA_WAVES == 0 || b < NBLK) dma16((const bf16_t*)src, lds + b * 512);
      p[k] = (const bf16_t*)((const char*)p[k] + (int64_t)BKV * step[k]);
    }
  }
};

template <int DQK, int DV, int HG, bool SPLIT>
__global__ __launch_bounds__(64 * PA_WAVES) void attn_packed_kernel(PackedDev a) {
  using KW = KeySwz<DQK>;
  using KS = RowStream<DQK, KW>;
  using VS = RowStream<DV, ValueSwz<DV>>;
  constexpr int NST = 3, STAGE = KS::ELEMS + VS::ELEMS;
  constexpr int NKK = DQK / 16, NC = DV / 32, BQH = PA_BQ / HG;
  constexpr int PK = 4, PV = 4;  // operand reads in flight ahead of the products
  __shared__ __attribute__((aligned(1024))) bf16_t smem[NST * STAGE];
  __shared__ __attribute__((aligned(256))) float kexp[NST][BKV];  // e

  const int pid = xcd_remap(blockIdx.x, gridDim.x);
  const int z = SPLIT ? pid % a.nsplit : 0, tile = SPLIT ? pid / a.nsplit : pid;
  const int qb = a.nqb - 1 - tile % a.nqb, i0 = tile / a.nqb * HG;
  auto q_at = [&](int b) { return min(max(a.q_off[b], 0), a.n_q); };
  auto k_at = [&](int b) { return min(max(a.kv_off[b], 0), a.n_kv); };
  int b = 0;
  for (int hi = a.B - 1; b < hi;) {  // the last sequence whose numbers start at qb or before
    const int mid = (b + hi + 1) >> 1;
    if (q_at(mid) / BQH + mid <= qb) b = mid;
    else hi = mid - 1;
  }
  const int qs = q_at(b), ks = k_at(b);
  const int Tq = max(q_at(b + 1) - qs, 0), Tk = max(k_at(b + 1) - ks, 0), diag = Tk - Tq;
  const int q0 = (qb - (qs / BQH + b)) * BQH;
  if (q0 < 0 || q0 >= Tq) return;

  const int lane = threadIdx.x & 63, wave = wave_id();
  const int half = lane >> 5, col = lane & 31;
  const int i = i0 + wave % HG;           // this wavefront's head
  const int qw0 = q0 + (wave / HG) * 32;  // and its first query
  const int my_q = qw0 + col;
  const int64_t row = (int64_t)qs + my_q;  // of Q and O

  const int kend = min(Tk, q0 + BQH + diag);
  const int nkb = kend > 0 ? (kend + BKV - 1) / BKV : 0;
  const int per = SPLIT ? (nkb + a.nsplit - 1) / a.nsplit : nkb;
  const int kb0 = z * per, kb1 = min(nkb, kb0 + per);
  // tiles that this wavefront sees: [kb0, nvis)
  const int nvis = min(kb1, ((qw0 + 31 + diag) >> 6) + 1);
  static_assert(BKV == 64, "the shift above");

  f32x16 acc[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[c][e] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;

  if (kb0 < kb1) {
    // this lane's query as B operand fragments (d = 16 kk + 8 half + 0..7)
    bf16x8 qf[NKK];
    {
      const bf16_t* qp = a.Q + (qs + (int64_t)min(my_q, Tq - 1)) * a.q_tok + (int64_t)i * a.q_head + 8 * half;
#pragma unroll
      for (int kk = 0; kk < NKK; ++kk) qf[kk] = *(const bf16x8*)(qp + 16 * kk);
    }
    KS kst;
    VS vst;
    {
      const bf16_t* ka = a.Ka + (int64_t)(i0 / a.ka_div) * a.ka_head;
      const bf16_t* kb = a.Kb + (int64_t)(i0 / a.kb_div) * a.kb_head - a.dnope;
      const bf16_t* vb = a.V + (int64_t)(i0 / a.v_div) * a.v_head;
      const int64_t r0 = (int64_t)ks + (int64_t)BKV * kb0;
      kst.init([&](int c) { return (c < a.dnope ? ka : kb) + c; },
               [&](int c) { return c < a.dnope ? a.ka_tok : a.kb_tok; }, r0);
      vst.init([&](int c) { return vb + c; }, [&](int) { return a.v_tok; }, r0);
    }
    auto issue = [&](int kb) __attribute__((always_inline)) {
      bf16_t* st = smem + (kb - kb0) % NST * STAGE;
      kst.next(st, kb * BKV, Tk - 1);
      vst.next(st + KS::ELEMS, kb * BKV, Tk - 1);
      if (wave == 0) dma4(a.key_exp + ks + min(kb * BKV + lane, Tk - 1), kexp[(kb - kb0) % NST]);
    };
    issue(kb0);
    if (kb0 + 1 < kb1) issue(kb0 + 1);
    // whether a key has an e other than 0
    bool any = false;
    for (int r0 = kb0 * BKV; r0 < min(kb1 * BKV, Tk); r0 += 8 * 64 * PA_WAVES) {
      float e[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) e[u] = a.key_exp[ks + min(r0 + 64 * PA_WAVES * u + (int)threadIdx.x, Tk - 1)];
#pragma unroll
      for (int u = 0; u < 8; ++u) any |= e[u] != 0.f;
    }
    wait_all();
    any = __syncthreads_or(any);
    // (in registers from here on: or the compiler's waits for them would also wait for copies)
#pragma unroll
    for (int kk = 0; kk < NKK; ++kk) asm volatile("" : "+v"(qf[kk]));

    // operand offsets in a stage.  Keys: row col (+ 32), chunk 2 kk + half, one offset for each value of
    // the changed bits.  Values: rows 4 half + (lane % 16) / 4 (+ 8, 16 ..: the same change), values
    // 16 ((lane / 16) % 2) + 4 (lane % 4) (+ 32 c: one offset for even and for odd c).
    constexpr int NKB = (1 << KW::BITS) / 2;
    int kofs[NKB], vofs[2];
#pragma unroll
    for (int j = 0; j < NKB; ++j) kofs[j] = col * DQK + 8 * ((2 * j + half) ^ KW::swz(col));
#pragma unroll
    for (int odd = 0; odd < 2; ++odd) {
      const int r = 4 * half + ((lane & 15) >> 2), d = 32 * odd + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
      vofs[odd] = r * DV + 8 * ((d >> 3) ^ ValueSwz<DV>::swz(r)) + (d & 7);
    }
    auto kread = [&](const bf16_t* kt, int kk) {
      return *(const bf16x8*)(kt + kofs[kk % NKB] + 16 * NKB * (kk / NKB));
    };

    // e of keys 8 g + 4 half + 0..3 (+ 32 h) of a stage
    auto eread = [&](int st, int h, int g) { return *(const f32x4*)&kexp[st][32 * h + 8 * g + 4 * half]; };
    // a logit accumulator starts at e / sl2
    auto start = [&](f32x16& s, int st, int h, auto any) __attribute__((always_inline)) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        f32x4 e = {0.f, 0.f, 0.f, 0.f};
        if (any) e = eread(st, h, g) * a.bias;
#pragma unroll
        for (int q = 0; q < 4; ++q) s[4 * g + q] = e[q];
      }
    };
    // the logits s of keys j0 .. j0 + 31: masked, and the reference moved if they need it
    auto settle = [&](f32x16& s, int j0, auto any) __attribute__((always_inline)) {
      if (j0 + 31 > qw0 + diag) {
        asm volatile("");  // (a real branch)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (j0 + 8 * (e >> 2) + 4 * half + (e & 3) > my_q + diag) s[e] = -INFINITY;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[e]);
      mx = pair_max32(mx) * a.sl2;
      if (__ballot(mx > m_run + PA_SLACK) != 0) {
        const float m_new = fmaxf(m_run, mx);
        const float d = m_run - (m_new == -INFINITY ? 0.f : m_new), corr = __builtin_amdgcn_exp2f(d);
        m_run = m_new;
        l_run = any ? scaled_down(l_run, d) : l_run * corr;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[c][e] *= corr;
      }
    };
    // half h of stage st: its settled logits sc become P and enter O, the logits of the 32 keys at kn
    // (the half behind it, in stage st_n) become sn meanwhile
    auto step = [&](const bf16_t* kn, const bf16_t* vs, f32x16& sc, f32x16& sn, int st, int h, int st_n, auto any) __attribute__((always_inline)) {
      const float m_use = (m_run == -INFINITY ? 0.f : m_run) - PA_UP;
      auto vread = [&](int j) {  // step j = NC u + c: keys 16 u .., values 32 c ..
        const bf16_t* q = vs + vofs[j % NC % 2] + 16 * (j / NC) * DV + 64 * (j % NC / 2);
        const u32x2 lo = lds_read_tr4(q), hi = lds_read_tr4(q + 8 * DV);
        return __builtin_bit_cast(f16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
      };
      bf16x8 kf[PK];
      f16x8 vf[PV];
      f32x4 ke[4];
#pragma unroll
      for (int j = 0; j < PK; ++j) kf[j] = kread(kn, j);
      start(sn, st_n, 1 - h, any);
#pragma unroll
      for (int g = 0; g < 4; ++g)
        if (any) ke[g] = eread(st, h, g);
      u32x4 w[2];
      float l0 = 0.f, l1 = 0.f;
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int kk = 0; kk < NKK; ++kk) {
        sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[kk % PK], qf[kk], sn, 0, 0, 0);
        if (kk + PK < NKK) kf[kk % PK] = kread(kn, kk + PK);
        else if (kk + PK - NKK < PV) vf[kk + PK - NKK] = vread(kk + PK - NKK);
#pragma unroll
        for (int e2 = 8 * kk / NKK; e2 < 8 * (kk + 1) / NKK; ++e2) {  // a share of the 8 pairs
          const float t0 = __builtin_fmaf(sc[2 * e2], a.sl2, -m_use), t1 = __builtin_fmaf(sc[2 * e2 + 1], a.sl2, -m_use);
          const float p0 = __builtin_amdgcn_exp2f(t0), p1 = __builtin_amdgcn_exp2f(t1);
          l0 += any ? __builtin_amdgcn_exp2f(t0 - ke[e2 / 2][2 * e2 % 4]) : p0;
          l1 += any ? __builtin_amdgcn_exp2f(t1 - ke[e2 / 2][2 * e2 % 4 + 1]) : p1;
          w[e2 / 4][e2 % 4] = pack2h(p0, p1);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      l_run += l0 + l1;
      const f16x8 pf[2] = {__builtin_bit_cast(f16x8, w[0]), __builtin_bit_cast(f16x8, w[1])};
#pragma unroll
      for (int j = 0; j < 2 * NC; ++j) {
        acc[j % NC] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[j % PV], pf[j / NC], acc[j % NC], 0, 0, 0);
        if (j + PV < 2 * NC) vf[j % PV] = vread(j + PV);
        __builtin_amdgcn_sched_barrier(0);
      }
    };

    f32x16 sa, sb;
    auto run = [&](auto scaled) __attribute__((always_inline)) {
      if (kb0 < nvis) {
        start(sa, 0, 0, scaled);
#pragma unroll
        for (int kk = 0; kk < NKK; ++kk)
          sa = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kread(smem, kk), qf[kk], sa, 0, 0, 0);
        settle(sa, kb0 * BKV, scaled);
      }
      for (int kb = kb0; kb < kb1; ++kb) {
        if (kb + 2 < kb1) issue(kb + 2);
        if (kb < nvis) {  // (uniform in the wavefront)
          // stage offsets pass through readfirstlane: opaque to the loop optimiser, which would keep one
          // induction variable per LDS read
          const int st = (kb - kb0) % NST, st_n = (kb + 1 - kb0) % NST;
          const int cur = __builtin_amdgcn_readfirstlane(st * STAGE), nxt = __builtin_amdgcn_readfirstlane(st_n * STAGE);
          const bf16_t* vs = smem + cur + KS::ELEMS;
          step(smem + cur + 32 * DQK, vs, sa, sb, st, 0, st, scaled);
          if (kb * BKV + 32 <= qw0 + 31 + diag) {  // the second half is not all behind the diagonal
            settle(sb, kb * BKV + 32, scaled);
            // (past the last tile the next logits come from a stale stage and are not used)
            step(smem + nxt, vs + 32 * DV, sb, sa, st, 1, st_n, scaled);
            if (kb + 1 < nvis) settle(sa, (kb + 1) * BKV, scaled);
          }
        }
        // tile kb + 2 has landed and nobody reads tile kb's stage any more
        wait_all();
        __syncthreads();
      }
    };
    if (any) run(std::true_type{});
    else run(std::false_type{});
  }

  // lane holds query my_q, d = 32 c + 8 g + 4 half + 0..3
  const float l = pair_sum32(l_run);
  if (my_q >= Tq) return;
  if (SPLIT) {
    const int64_t at = ((int64_t)z * a.n_q + row) * a.H + i;
    if (half == 0) {
      a.part_ml[2 * at] = m_run;
      a.part_ml[2 * at + 1] = l;
    }
    if (kb0 >= kb1) return;  // (an empty part has no weight: its values are not read)
    float* po = a.part_o + at * DV + 4 * half;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *(f32x4*)(po + 32 * c + 8 * g) =
            f32x4{acc[c][4 * g], acc[c][4 * g + 1], acc[c][4 * g + 2], acc[c][4 * g + 3]};
  } else {
    const float* vsc = a.v_scale + (int64_t)(i / a.v_div) * a.v_head + 4 * half;
    const float inv = l == 0.f ? 0.f : 1.f / l;  // (l = 0: a query that sees no key)
    bf16_t* op = a.O + row * a.o_tok + (int64_t)i * DV + 4 * half;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 v = f32x4{acc[c][4 * g], acc[c][4 * g + 1], acc[c][4 * g + 2], acc[c][4 * g + 3]} * inv *
                        *(const f32x4*)(vsc + 32 * c + 8 * g);
        *(u32x2*)(op + 32 * c + 8 * g) = u32x2{pack2bf(v[0], v[1]), pack2bf(v[2], v[3])};
      }
  }
}

// The parts of every (query, head) joined in order; a thread has four values.  Parts without weight
// (no key seen: reference -infinity, sum 0) are not read.  References may lie more than 2^126 apart (a part
// of small latents beside one of large ones).
__global__ __launch_bounds__(256) void attn_packed_join_kernel(PackedDev a, int dv) {
  const int64_t e = 4 * ((int64_t)blockIdx.x * 256 + threadIdx.x), at = e / dv;
  const int64_t row = at / a.H;
  if (row >= a.n_q || row < a.q_off[0] || row >= a.q_off[a.B]) return;
  const int i = (int)(at % a.H), d = (int)(e % dv);
  const int64_t stride = (int64_t)a.n_q * a.H;
  float M = -INFINITY;
  for (int z = 0; z < a.nsplit; ++z) M = fmaxf(M, a.part_ml[2 * (at + z * stride)]);
  float L = 0.f;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  for (int z = 0; z < a.nsplit; ++z) {
    const f32x2 ml = *(const f32x2*)(a.part_ml + 2 * (at + z * stride));
    if (ml[0] == -INFINITY && ml[1] == 0.f) continue;
    const float down = ml[0] - (M == -INFINITY ? 0.f : M);
    L += scaled_down(ml[1], down);
    v += *(const f32x4*)(a.part_o + (at + z * stride) * dv + d) * __builtin_amdgcn_exp2f(down);
  }
  v *= (L == 0.f ? 0.f : 1.f / L) * *(const f32x4*)(a.v_scale + (int64_t)(i / a.v_div) * a.v_head + d);
  *(u32x2*)(a.O + row * a.o_tok + (int64_t)i * dv + d) = u32x2{pack2bf(v[0], v[1]), pack2bf(v[2], v[3])};
}

// Four heads per workgroup when they share every key / value source, else one: a quarter of the copies for
// the same products, 123 us against 171 with one (5505 tokens, 32 heads in 8 groups).
int heads_per_group(const AttnPacked& a) {
  return a.H % 4 == 0 && a.Ka.div % 4 == 0 && a.V.div % 4 == 0 && (a.dnope == a.dqk || a.Kb.div % 4 == 0) ? 4 : 1;
}
// query tile numbers of all sequences
int tile_numbers(const AttnPacked& a) { return a.n_q / (PA_BQ / heads_per_group(a)) + a.B; }
// Parts of the keys: where the tiles do not fill the CUs once, as many as fill them twice, each of
// four or more key tiles of an average sequence.  463 queries of 8 sequences after 13620 rows: 76 us
// uncut, 41 and 7 to join in parts; 5505 tokens of 6 sequences, 736 tiles, are not cut.  The rule knows the
// average sequence only: four new tokens of each of 64 sequences, one of 100000 rows and the others of 300,
// are not cut, and the whole call takes 3.4 ms where as many rows spread evenly take 0.68.
int parts_of(const AttnPacked& a) {
  const int64_t tiles = (int64_t)tile_numbers(a) * (a.H / heads_per_group(a));
  if (tiles >= 256) return 1;
  const int64_t fill = (512 + tiles - 1) / tiles, most = a.n_kv / ((int64_t)a.B * BKV * 4);
  const int64_t n = fill < most ? fill : most;
  return (int)(n < 1 ? 1 : n < 16 ? n : 16);
}

template <int DQK, int DV, int HG>
void launch(const PackedDev& d, hipStream_t s) {
  const unsigned grid = (unsigned)(d.H / HG * d.nqb * d.nsplit);
  if (d.nsplit > 1) attn_packed_kernel<DQK, DV, HG, true><<<grid, 64 * PA_WAVES, 0, s>>>(d);
  else attn_packed_kernel<DQK, DV, HG, false><<<grid, 64 * PA_WAVES, 0, s>>>(d);
}

}  // namespace
}  // namespace attn

// Enough for the parts of every call of no more queries, keys and sequences.  Fewer keys or more sequences
// never mean more parts; more queries do mean fewer, at each further query tile: so one sequence, all the
// keys, and of the query counts up to n_q the last before each further tile.
size_t attn_packed_ws_bytes(const AttnPacked& a) {
  AttnPacked c = a;
  c.B = 1;
  const int bqh = attn::PA_BQ / attn::heads_per_group(a);
  size_t rows = 0;
  for (int64_t end = bqh - 1;; end += bqh) {
    c.n_q = (int)(end < a.n_q ? end : a.n_q);
    const int n = attn::parts_of(c);
    if (n > 1 && (size_t)n * c.n_q > rows) rows = (size_t)n * c.n_q;
    if (n <= 1 || c.n_q == a.n_q) break;
  }
  return rows * a.H * (a.dv + 2) * 4;
}

hipError_t attn_fwd_packed(const AttnPacked& a, hipStream_t s) {
  if (!attn_mfma_supported(a.dqk, a.dv)) return hipErrorInvalidValue;
  if (a.n_q == 0) return hipSuccess;
  attn::PackedDev d;
  d.B = a.B; d.H = a.H; d.dnope = a.dnope; d.sl2 = a.scale * attn::LOG2E;
  d.Q = (const bf16_t*)a.Q.p; d.q_tok = a.Q.tok; d.q_head = (int)a.Q.head;
  d.Ka = (const bf16_t*)a.Ka.p; d.ka_tok = a.Ka.tok; d.ka_head = (int)a.Ka.head; d.ka_div = a.Ka.div;
  d.Kb = (const bf16_t*)a.Kb.p; d.kb_tok = a.Kb.tok; d.kb_head = (int)a.Kb.head; d.kb_div = a.Kb.div;
  d.key_exp = a.key_exp; d.v_scale = a.v_scale; d.bias = 1.f / d.sl2;
  d.V = (const bf16_t*)a.V.p; d.v_tok = a.V.tok; d.v_head = (int)a.V.head; d.v_div = a.V.div;
  d.O = (bf16_t*)a.O; d.o_tok = a.o_tok;
  d.q_off = a.q_off; d.kv_off = a.kv_off; d.n_q = a.n_q; d.n_kv = a.n_kv;
  d.nqb = attn::tile_numbers(a); d.nsplit = attn::parts_of(a);
  d.part_o = (float*)a.ws;
  d.part_ml = d.part_o + (size_t)d.nsplit * a.n_q * a.H * a.dv;
  const int hg = attn::heads_per_group(a);
  // (the lengths are on the device: the pairs are not counted)
  prof_begin(KC_ATTN_FWD, s);
#define X(a_, b_)                                            \
  if (a.dqk == a_ && a.dv == b_) {                           \
    if (hg == 4) attn::launch<a_, b_, 4>(d, s);              \
    else attn::launch<a_, b_, 1>(d, s);                      \
  }
  MLA_MFMA_SHAPES(X)
#undef X
  prof_end(KC_ATTN_FWD, s, 0.0, ((double)a.n_q + a.n_kv) * a.H * (a.dqk + a.dv) * 2,
           a.dqk == 192 ? KLABEL("attn_packed_kernel<192,128>") : KLABEL("attn_packed_kernel"));
  if (d.nsplit > 1) {
    prof_begin(KC_ELEM, s);
    const int64_t n = (int64_t)a.n_q * a.H * a.dv / 4;
    attn::attn_packed_join_kernel<<<(unsigned)((n + 255) / 256), 256, 0, s>>>(d, a.dv);
    prof_end(KC_ELEM, s, 0.0, (double)n * 4 * (4.0 * d.nsplit + 2), KLABEL("attn_packed_join_kernel"));
  }
  return hipGetLastError();
}

}  // namespace mla
