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

// ---- decoding -------------------------------------------------------------------------
// With one positional key all heads attend to the same row, so decoding is multi-query
// attention over rows of DK = r_kv + d_rope whose first DVL = r_kv values are the values too:
// every cache row is read once for all heads, 60 operations a byte at 32 heads, and the rows'
// stream bounds the kernel.
//
// * The rows of all sequences, in tiles of 32, form one list; a workgroup takes an equal share
//   of it, whatever the lengths (one workgroup a CU).  The part of a sequence in a workgroup's
//   share is a segment; its partial result goes to slot (workgroup + sequence), which no other
//   segment has: along the list one of the two grows from segment to segment.
// * Within a segment every wavefront takes every fourth tile by itself: its own LDS buffer, its
//   own softmax state (running maximum and sum of each head, the weighted latents of all heads in
//   256 registers), no barrier and no exchange until the segment ends.  While one wavefront waits
//   for its copies the others multiply: about three of the four 37 KB tiles of a CU are in flight
//   at any time.
// * S^T = K Q^T has the row in the MFMA row and the head in its column, so a lane owns one head's
//   state, and the accumulator of S^T is, after the exponential, the B operand of O^T = V^T P^T
//   (the order of the rows inside a K step is the same on both sides).  V^T comes from the same
//   LDS tile by transposing reads.
// * The four states of a segment are joined through LDS in two exchanges of halves.
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
  const bf16_t* qabs;  // [B][HP][DK]
  float* part_o;       // [slot][HP][DVL], not normalised
  float* part_ml;      // [slot][HP][2]: reference maximum (log2), sum
  int32_t* tile_off;   // [B + 1]: first tile of each sequence in the list
  float sl2;
};

__device__ __forceinline__ int decode_len(const PagedDecodeDev& a, int b) {
  return min(max(a.len[b], 0), a.max_len);
}
__device__ __forceinline__ int tiles_of(int n) { return (n + PD_KT - 1) / PD_KT; }
// Tiles per workgroup: at least one for each wavefront.
__device__ __forceinline__ int share_of(int tiles, int nwg) { return max(PD_WAVES, (tiles + nwg - 1) / nwg); }

// Matrix products with their accumulators where they are wanted: the weighted latents fill the 256
// accumulation registers, the tile's logits are in vector registers.  (The compiler puts every
// product's result on one side, and moved 256 values out and in around each tile for the few that
// are rescaled.)  The waits are those that the compiler keeps around products it knows: two
// states after the vector ALU wrote an operand, and the product's passes (19 states at most)
// before the vector ALU reads a result.
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
// v *= f, v[4 g ..] += y on accumulation registers
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
__device__ __forceinline__ void acc_add(f32x16& v, int g, f32x4 y) {
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    float x = v[4 * g + r], t;
    asm volatile("v_accvgpr_read_b32 %1, %0\n\tv_add_f32 %1, %1, %2\n\tv_accvgpr_write_b32 %0, %1"
                 : "+a"(x), "=&v"(t)
                 : "v"(y[r]));
    v[4 * g + r] = x;
  }
}

template <int DK, int DVL>
__global__ __launch_bounds__(64 * PD_WAVES, 1) void paged_decode_kernel(PagedDecodeDev a) {
  constexpr int LD = attn::ld_of(DK);          // padded rows: conflict-free operand reads
  constexpr int CH = LD / 8, DCH = DK / 8;     // 16-byte chunks of a row, with and without padding
  constexpr int NCP = (PD_KT * CH + 63) / 64;  // copies (of 64 chunks) of a tile
  constexpr int NKK = DK / 16, NC = DVL / 32;
  static_assert(DK % 16 == 0 && NC % 4 == 0 && CH >= 64 / 4, "decode shape");
  static_assert(2 * NC * 4096 <= PD_WAVES * NCP * 1024, "two states fit the tiles");
  __shared__ __attribute__((aligned(1024))) bf16_t tiles[PD_WAVES][NCP * 512];
  __shared__ float ml[PD_WAVES][2][32];
  __shared__ int scan[64 * PD_WAVES], plan[2];

  const int tid = threadIdx.x, lane = tid & 63, wave = wave_id();
  const int half = lane >> 5, col = lane & 31;
  const int wg = blockIdx.x, nwg = gridDim.x, h0 = 32 * blockIdx.y;

  // the list: each thread counts the tiles of a run of sequences, a scan gives their places
  const int run = (a.B + 64 * PD_WAVES - 1) / (64 * PD_WAVES);
  const int b_lo = min(tid * run, a.B), b_hi = min(b_lo + run, a.B);
  int mine = 0;
  for (int b = b_lo; b < b_hi; ++b) mine += tiles_of(decode_len(a, b));
  scan[tid] = mine;
  __syncthreads();
  for (int d = 1; d < 64 * PD_WAVES; d *= 2) {
    const int v = tid >= d ? scan[tid - d] : 0;
    __syncthreads();
    scan[tid] += v;
    __syncthreads();
  }
  const int total = scan[64 * PD_WAVES - 1];
  const int share = share_of(total, nwg);
  const int t_lo = min((int64_t)wg * share, (int64_t)total), t_hi = min(t_lo + share, total);
  {
    int at = scan[tid] - mine;
    const bool first = wg == 0 && blockIdx.y == 0;
    if (first || (at <= t_lo && t_lo < at + mine)) {
      for (int b = b_lo; b < b_hi; ++b) {
        const int n = tiles_of(decode_len(a, b));
        if (first) a.tile_off[b] = at;
        if (at <= t_lo && t_lo < at + n) {
          plan[0] = b;
          plan[1] = at;
        }
        at += n;
      }
      if (first && tid == 64 * PD_WAVES - 1) a.tile_off[a.B] = total;
    }
  }
  __syncthreads();
  if (t_lo >= t_hi) return;
  int b = __builtin_amdgcn_readfirstlane(plan[0]);
  int seq0 = __builtin_amdgcn_readfirstlane(plan[1]);  // first tile of sequence b in the list

  const uint64_t heads = __ballot(h0 + col < a.H);  // (columns without a head move no reference)
  bf16_t* kt = tiles[wave];

  // row `lane` of tile t of sequence b (the last row again past the end, which gets no weight):
  // its page's table entry, and its address
  auto entry = [&](int t, int n) {
    const int p = min(t * PD_KT + col, n - 1);
    return a.table[(int64_t)b * a.max_pages + p / a.page_size];
  };
  auto issue = [&](int t, int n, int page, bool& bad) {
    const int p = min(t * PD_KT + col, n - 1);
    const bool out = page < 0 || page >= a.n_pages;
    bad = __ballot(out) != 0;
    const uint64_t at = (uint64_t)(uintptr_t)(a.pool + ((int64_t)(out ? 0 : page) * a.page_size + p % a.page_size) * DK);
    const uint32_t lo = (uint32_t)at, hi = (uint32_t)(at >> 32);
    int ln = lane;  // opaque: the lanes' chunk numbers are cheaper made again than kept in 74 registers
    asm volatile("" : "+v"(ln));
    // copy k fills chunks 64 k .. 64 k + 63 of the padded tile: rows r0 and r0 + 1 (one row's
    // padding lies between them and takes any chunk), both known at compile time
#pragma unroll
    for (int k = 0; k < NCP; ++k) {
      constexpr int LAST = PD_KT - 1;
      const int r0 = 64 * k / CH, skip = 64 * k % CH;
      uint64_t src = 0;
      int c = ln + skip;
#pragma unroll
      for (int r = 0; r <= 64 / CH + 1; ++r) {  // the rows that 64 chunks can touch
        if (r > 0 && r * CH >= skip + 64) break;
        const int rr = r0 + r < LAST ? r0 + r : LAST;
        const uint64_t base = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)lo, rr) |
                              (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)hi, rr) << 32;
        const int cc = ln + skip - r * CH;
        if (r == 0 || cc >= 0) {
          src = base;
          c = cc;
        }
      }
      if (c >= DCH) c = 0;
      dma16((const bf16_t*)(uintptr_t)(src + 16u * (uint32_t)c), kt + 512 * k);
      __builtin_amdgcn_sched_barrier(0);  // (or every row's address waits in scalar registers)
    }
  };

  for (int t0 = t_lo; t0 < t_hi;) {
    const int n = __builtin_amdgcn_readfirstlane(decode_len(a, b));
    const int nt = tiles_of(n);
    if (nt == 0) {
      ++b;
      continue;
    }
    const int first = t0 - seq0, last = min(t_hi - seq0, nt);  // tiles [first, last) of sequence b
    const int slot = wg + b;

    int t = first + wave;
    bool bad = false, any_bad = false;
    if (t < last) issue(t, n, entry(t, n), bad);
    bf16x8 qf[NKK];  // this lane's head as B operand fragments (k = 16 kk + 8 half + 0..7)
    {
      const bf16_t* qsrc = a.qabs + ((int64_t)b * a.HP + h0 + col) * DK + 8 * half;
#pragma unroll
      for (int kk = 0; kk < NKK; ++kk) qf[kk] = *(const bf16x8*)(qsrc + 16 * kk);
    }
    f32x16 acc[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[c][e] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;

    for (; t < last; t += PD_WAVES) {
      any_bad |= bad;
      const int next = t + PD_WAVES;
      int page = 0;
      if (next < last) page = entry(next, n);
      wait_vm<0>();
      f32x16 s;
      mfma_v_first(s, *(const bf16x8*)(kt + col * LD + 8 * half), qf[0]);
#pragma unroll
      for (int kk = 1; kk < NKK; ++kk)
        mfma_v_next(s, *(const bf16x8*)(kt + col * LD + 16 * kk + 8 * half), qf[kk]);
      mfma_v_done(s);
      // rows past the end (the last tile only; a real branch): no weight
      if ((t + 1) * PD_KT > n) {
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
#pragma unroll
        for (int c = 0; c < NC; ++c) acc_scale(acc[c], corr);
      }
      const float m_use = m_run == -INFINITY ? 0.f : m_run;
      bf16x8 pf[2];  // P rounded to bf16, the matrix cores' operand
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        u32x4 w;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * u + 2 * q], a.sl2, -m_use));
          const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * u + 2 * q + 1], a.sl2, -m_use));
          l_run += p0 + p1;
          w[q] = pack2bf(p0, p1);
        }
        pf[u] = __builtin_bit_cast(bf16x8, w);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int klo = 16 * u + 4 * half;
#pragma unroll
        for (int c = 0; c < NC; ++c) mfma_a(acc[c], lds_operand_tr(kt, LD, 32 * c, klo, klo + 8), pf[u]);
      }
      mfma_a_done(acc);
      // every read of the tile has returned before the next copies may overwrite it
      asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
      if (next < last) issue(next, n, page, bad);
    }

    // join the wavefronts' states: one reference and sum, then the latents
    float l = pair_sum32(l_run);
    if (any_bad) l = NAN;  // a row on no page
    if (half == 0) {
      ml[wave][0][col] = m_run;
      ml[wave][1][col] = l;
    }
    __syncthreads();  // (and every wavefront is done with its tile)
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int w = 0; w < PD_WAVES; ++w) M = fmaxf(M, ml[w][0][col]);
#pragma unroll
    for (int w = 0; w < PD_WAVES; ++w) {
      const float mw = ml[w][0][col];
      L += ml[w][1][col] * (mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw - M));
    }
    const float f = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - M);
    // wavefronts 2 and 3 hand theirs to 0 and 1, then 1 to 0
    float* buf = (float*)tiles[0];
    // (always inlined: a reference to the registers would put them in memory)
    auto put = [&](float* p) __attribute__((always_inline)) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *(f32x4*)(p + ((c * 4 + g) * 64 + lane) * 4) =
              f32x4{acc[c][4 * g], acc[c][4 * g + 1], acc[c][4 * g + 2], acc[c][4 * g + 3]};
    };
    auto add = [&](const float* p) __attribute__((always_inline)) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int g = 0; g < 4; ++g) acc_add(acc[c], g, *(const f32x4*)(p + ((c * 4 + g) * 64 + lane) * 4));
    };
#pragma unroll
    for (int c = 0; c < NC; ++c) acc_scale(acc[c], f);
    constexpr int STATE = NC * 1024;  // floats of a wavefront's state
    if (wave >= 2) put(buf + (wave - 2) * STATE);
    __syncthreads();
    if (wave < 2) add(buf + wave * STATE);
    __syncthreads();
    if (wave == 1) put(buf);
    __syncthreads();
    if (wave == 0) {
      add(buf);
      // lane (head col, half) holds latents 32 c + 8 g + 4 half + 0..3
      if (h0 + col < a.H) {
        const int64_t row = (int64_t)slot * a.HP + h0 + col;
        float* po = a.part_o + row * DVL + 4 * half;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            *(f32x4*)(po + 32 * c + 8 * g) =
                f32x4{acc[c][4 * g], acc[c][4 * g + 1], acc[c][4 * g + 2], acc[c][4 * g + 3]};
        if (half == 0) {
          a.part_ml[2 * row] = M;
          a.part_ml[2 * row + 1] = L;
        }
      }
    }
    t0 = seq0 + last;
    if (t0 < t_hi) __syncthreads();  // the buffers take tiles again
    seq0 += nt;
    ++b;
  }
}

// The segments of a (sequence, head) joined, then W_UV on the matrix cores: lat[d] = sum_s o_s[d]
// 2^(m_s - M) / sum_s l_s 2^(m_s - M), rounded to bf16, o[e] = sum_d W_UV[g][e][d] lat[d].  A
// workgroup owns a head and PF_RB sequences; its wavefronts ask for their W_UV rows first, so that
// the merge hides them.  Segments in the list's order.  Bound by latency.
constexpr int PF_RB = 8;
template <int DVL, int DV>
__global__ __launch_bounds__(256) void paged_finish_kernel(const float* __restrict__ part_o,
                                                           const float* __restrict__ part_ml,
                                                           const int32_t* __restrict__ tile_off,
                                                           const bf16_t* __restrict__ Wuv,
                                                           bf16_t* __restrict__ o, int B, int H, int HP,
                                                           int nwg, int hpg) {
  constexpr int NCG = DVL / 4, NSLOT = 256 / NCG, NK = DVL / 32, NT = DV / 64, LDL = DVL + 8;
  __shared__ float red[PF_RB][NSLOT][DVL];
  __shared__ __attribute__((aligned(16))) bf16_t lat[PF_RB * LDL];
  __shared__ float sM[PF_RB], sInv[PF_RB];
  __shared__ int s0[PF_RB], sn[PF_RB];
  const int i = blockIdx.x, b0 = PF_RB * blockIdx.y, nb = min(PF_RB, B - b0);
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_id();
  bf16x8 wf[NT][NK];  // W_UV rows 16 (NT wave + t) + lane % 16, k = 32 kk + 8 (lane / 16) + 0..7
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const bf16_t* wp = Wuv + ((int64_t)(i / hpg) * DV + 16 * (NT * wave + t) + (lane & 15)) * DVL + 8 * (lane >> 4);
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) wf[t][kk] = *(const bf16x8*)(wp + 32 * kk);
  }
  const int share = share_of(tile_off[B], nwg);
  // maxima and sums: a wavefront per sequence and round, a lane takes every 64th segment
  for (int bb = wave; bb < PF_RB; bb += 4) {
    int slot = 0, ns = 0;
    if (bb < nb) {
      const int t0 = tile_off[b0 + bb], t1 = tile_off[b0 + bb + 1];
      if (t1 > t0) {
        slot = t0 / share + b0 + bb;
        ns = (t1 - 1) / share - t0 / share + 1;
      }
    }
    float M = -INFINITY, L = 0.f;
    for (int sp = lane; sp < ns; sp += 64) {
      const f32x2 x = *(const f32x2*)(part_ml + 2 * ((int64_t)(slot + sp) * HP + i));
      const float m1 = fmaxf(M, x[0]);
      const float ref = m1 == -INFINITY ? 0.f : m1;
      L = L * __builtin_amdgcn_exp2f(M - ref) + x[1] * __builtin_amdgcn_exp2f(x[0] - ref);
      M = m1;
    }
    const float Mw = warp_max(M);
    const float Lw = warp_sum(M == -INFINITY ? L : L * __builtin_amdgcn_exp2f(M - Mw));
    if (lane == 0) {
      s0[bb] = slot;
      sn[bb] = ns;
      sM[bb] = Mw == -INFINITY ? 0.f : Mw;
      sInv[bb] = Lw == 0.f ? 0.f : 1.f / Lw;  // (NaN stays NaN)
    }
  }
  __syncthreads();
  const int cg = tid % NCG, sl = tid / NCG;
  for (int bb = 0; bb < nb; ++bb) {
    const int ns = sn[bb];
    const float M = sM[bb];
    const int64_t row0 = (int64_t)s0[bb] * HP + i;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int sp = sl; sp < ns; sp += 8 * NSLOT) {
      f32x4 x[8];
      float m[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int64_t rw = row0 + (int64_t)HP * min(sp + u * NSLOT, ns - 1);
        x[u] = *(const f32x4*)(part_o + rw * DVL + 4 * cg);
        m[u] = part_ml[2 * rw];
      }
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (sp + u * NSLOT < ns) v += x[u] * __builtin_amdgcn_exp2f(m[u] - M);
    }
    *(f32x4*)&red[bb][sl][4 * cg] = v;
  }
  __syncthreads();
  for (int e = tid; e < nb * NCG; e += 256) {
    const int bb = e / NCG, c = 4 * (e % NCG);
    f32x4 v = *(const f32x4*)&red[bb][0][c];
#pragma unroll
    for (int k = 1; k < NSLOT; ++k) v += *(const f32x4*)&red[bb][k][c];
    v *= sInv[bb];
    if (sn[bb] == 0) v = f32x4{0.f, 0.f, 0.f, 0.f};
    *(u32x2*)(lat + bb * LDL + c) = u32x2{pack2bf(v[0], v[1]), pack2bf(v[2], v[3])};
  }
  __syncthreads();
  const int n = lane & 15;  // MFMA column: sequence b0 + n
  const bf16_t* lp = lat + min(n, nb - 1) * LDL + 8 * (lane >> 4);
  f32x4 acc[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int kk = 0; kk < NK; ++kk) {
    const bf16x8 lf = *(const bf16x8*)(lp + 32 * kk);
#pragma unroll
    for (int t = 0; t < NT; ++t)
      acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[t][kk], lf, acc[t], 0, 0, 0);
  }
  if (n >= nb) return;
#pragma unroll
  for (int t = 0; t < NT; ++t) {  // rows 4 (lane / 16) + 0..3 of each 16-row tile
    bf16_t* op = o + ((int64_t)(b0 + n) * H + i) * DV + 16 * (NT * wave + t) + 4 * (lane >> 4);
#pragma unroll
    for (int k = 0; k < 4; ++k) op[k] = f2bf(acc[t][k]);
  }
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
  const size_t HP = (H + 31) / 32 * 32, slots = (size_t)nwg + B;
  DecodeLayout l;
  l.qabs = 0;
  l.part_o = l.qabs + al(B * HP * DK * 2);
  l.part_ml = l.part_o + al(slots * HP * DVL * 4);
  l.tile_off = l.part_ml + al(slots * HP * 2 * 4);
  l.bytes = l.tile_off + al(((size_t)B + 1) * 4);
  return l;
}

#define MLA_PAGED_SHAPES(X) X(576, 512) X(288, 256) X(160, 128)

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
  hipError_t e = decode_absorb(d.q, d.Wuk, ws + l.qabs, d.B, d.H, HP, d.hpg, d.dn, d.dr, d.rkv, s);
  if (e != hipSuccess) return e;
  // algorithmic work at full lengths
  prof_begin(KC_ATTN_FWD, s);
#define X(a_, b_) \
  if (DK == a_ && DVL == b_) paged_decode_kernel<a_, b_><<<dim3(nwg, HP / 32), 64 * PD_WAVES, 0, s>>>(a);
  MLA_PAGED_SHAPES(X)
#undef X
  prof_end(KC_ATTN_FWD, s, 2.0 * d.B * d.H * (double)d.max_len * (DK + DVL), (double)d.B * d.max_len * DK * 2,
           KLABEL("paged_decode_kernel"));
  prof_begin(KC_ELEM, s);
  const dim3 grid(d.H, (d.B + PF_RB - 1) / PF_RB);
#define X(a_, b_)                                                                                        \
  if (DK == a_ && DVL == b_) {                                                                           \
    if (d.dv == 128)                                                                                     \
      paged_finish_kernel<b_, 128><<<grid, 256, 0, s>>>(a.part_o, a.part_ml, a.tile_off,                 \
                                                        (const bf16_t*)d.Wuv, (bf16_t*)d.o, d.B, d.H, HP, \
                                                        nwg, d.hpg);                                     \
    else                                                                                                 \
      paged_finish_kernel<b_, 64><<<grid, 256, 0, s>>>(a.part_o, a.part_ml, a.tile_off,                  \
                                                       (const bf16_t*)d.Wuv, (bf16_t*)d.o, d.B, d.H, HP, \
                                                       nwg, d.hpg);                                      \
  }
  MLA_PAGED_SHAPES(X)
#undef X
  prof_end(KC_ELEM, s, 2.0 * d.B * d.H * d.dv * d.rkv, ((double)nwg + d.B) * d.H * (DVL + 2) * 4,
           KLABEL("paged_finish_kernel"));
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
