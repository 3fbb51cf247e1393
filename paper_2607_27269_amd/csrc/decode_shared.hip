// Absorbed-form decoding over a paged latent cache of either format, for sequences some of which begin
// with the same rows.
#include <type_traits>

#include "absorb.h"
#include "attn_common.h"
#include "cache_rows.h"
#include "common.h"
#include "decode_parts.h"
#include "kernels.h"

namespace mla {
namespace {

size_t al(size_t x) { return (x + 255) & ~(size_t)255; }

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// Attention is that of paged_attn.hip: a block of 32 heads of a sequence (32 queries) is one column block
// of the matrix products, its state belongs to a wavefront, tiles have 32 rows.  Here the rows of
// a sequence may begin with ones that its group shares, and there are two lists of tiles:
//
// * own rows: the tiles of all query blocks behind what they share.  A wavefront works on a run of tiles of its
//   own; the four of a workgroup are in the same block's rows and join their states, or, where there are too many
//   blocks or tiles for that, the list is cut into equal runs as in paged_attn.hip;
// * shared rows: a group's query blocks in fours ("quads"), for each quad the tiles of the shared rows.
//   A workgroup takes a run of these items; its four wavefronts have a query block each and one tile in
//   LDS for all of them, which is then read from memory once for four blocks and once from the
//   caches for the group's other quads.  For large groups the tiles are images that the launch before has
//   made: in fp16 with a power of two a row, in the order in which LDS holds them.
//
// Behind PD_RUN tiles of a run or a piece the state is put down, joined to that in its slot, and the next begins at zero.
//
// The workgroups are divided between the lists by their tiles.  A tile of one block's own rows and
// an item of four blocks cost a workgroup about the same: the first waits for its copy (64 sequences of the 8B layer
// behind 8192 shared rows, 400 of their own, bf16, without images: 70 us; with own tiles counted as 3/4, 2/3, 1/2:
// 71, 76, 87; with images 62, as 3/4 70, as 4/3 and 3/2 62).
//
// Three launches: the absorbed queries with the plan, the attention, the merge with W_UV.  Measured: whole calls, beside
// them the launches as the profiler shows them (with it attached all are longer, so that they add up to more), what the
// rows' bytes (at a large copy's 5.2 TB/s) or the operations (at a large product's 1444 TFLOP/s) need alone, and decoding
// each sequence for itself:
//   e4m3, 64 sequences to 4096 rows, 32 heads of 512 + 64   64 us (7.0, 50, 9.0;   33)
//   e4m3, 41 ragged ones to 16001                           44    (5.6, 30, 10.7;  14)
//   e4m3, one of 300, 14 heads of 256 + 32                  17    (4.5, 10, 3.9;   0)
//   bf16, 64 behind 8192 shared rows                        86    (12, 64, 17.0;   26; apart 87)
//   e4m3, 45 in 7 groups behind 20000                       89    (7.9, 73, 17.8;  23; apart 71)
//   bf16, 4 behind 1000, 14 heads                           20    (6.4, 10, 4.3;   0;  apart 17)
struct LatentDev {
  const char* pool;
  const int32_t* table;
  int n_pages, page_size, max_pages;
  uint32_t div_mul;       // p / page_size = (2 p div_mul >> 32) >> div_shift for p below 2^31
  int div_shift;
  int64_t page_bytes;
  const int32_t* len;
  int max_len, B, H, HB;  // HB: blocks of 32 heads
  const bf16_t* qabs;     // [B HB][DK / 16][64 lanes][8], bf16; not the latents of an e4m3 cache
  const bf16_t* qabs16;   // the latents in fp16 (absorb.h; [B HB][DVL / 16][64 lanes][8]): of an e4m3 cache, or for images
  const int8_t* qexp;     // [B HB][32][DVL / 32], exponents of their powers of two
  char* images;           // [n_groups][image_tiles] tiles of the shared rows, as LDS holds them, in fp16
  float* image_powers;    // [n_groups][image_tiles][32]
  int image_tiles;
  float* part_o;          // [slot][32][DVL], not normalised
  float* part_ml;         // [slot][32][2]: reference (log2), sum
  float sl2;
  int nwg;
  // the lists, made by the plan (one workgroup of the launch before)
  int n_groups, max_pieces;
  const int32_t* group_off;
  const int32_t* shared_len;
  int32_t* head;          // [4]: pieces of the shared rows, workgroups for them, tiles of own rows, and of a
                          // wavefront at most where each workgroup is in one block's (else 0)
  int32_t* start;         // [B]: rows that the sequence shares, a multiple of PD_KT
  int32_t* tile_off;      // [B HB + 1]: first tile of each block's own rows
  int32_t* wg_off;        // [B HB + 1]: first workgroup of each block's own rows, if each is in one block's
  int32_t* member;        // [B]: the sequence's group if it has shared rows, else -1
  int32_t* group;         // [n_groups][GROUP_INTS]
  int32_t* lens;          // [B]: lengths, within [0, max_len]
  int32_t* scratch;       // [5 n_groups + 1]
};

__device__ __forceinline__ int len_of(const LatentDev& a, int b) { return min(max(a.len[b], 0), a.max_len); }

// A group in the plan: its first piece, quads, pieces of each quad, tiles, first block, blocks, and the sequence (one
// that has rows) whose page table the shared rows are read through.  Piece p of quad q is
// number first + p quads + q: workgroups with neighbouring numbers read the same rows for different quads.
constexpr int GROUP_INTS = 7;
enum { G_FIRST, G_QUADS, G_PIECES, G_TILES, G_X0, G_BLOCKS, G_SEQ };

// How many workgroups the shared rows get, where they have `shared` tiles of quads and the own rows `own` tiles.
__device__ __forceinline__ int shared_workgroups(int nwg, int64_t shared, int64_t own) {
  if (shared == 0) return 0;
  if (own == 0) return nwg;
  return (int)min(max((nwg * shared + (shared + own) / 2) / (shared + own), (int64_t)1), (int64_t)nwg - 1);
}

__device__ __forceinline__ int page_of(const LatentDev& a, int p) {
  return (int)(__umulhi(2u * (uint32_t)p, a.div_mul) >> a.div_shift);
}

// ---- the plan -------------------------------------------------------------------------
// Sums over the threads before this one, and over all (NT threads), of N values at once.
template <int NT, int N>
__device__ __forceinline__ void scan_before(int (&v)[N], int (&total)[N]) {
  __shared__ int sums[N][NT / 64];
  const int lane = threadIdx.x & 63, wave = wave_id();
  int upto[N];
#pragma unroll
  for (int k = 0; k < N; ++k) upto[k] = v[k];
#pragma unroll
  for (int d = 1; d < 64; d *= 2)
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int o = __shfl_up(upto[k], d, 64);
      if (lane >= d) upto[k] += o;
    }
  __syncthreads();
  if (lane == 63)
#pragma unroll
    for (int k = 0; k < N; ++k) sums[k][wave] = upto[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) {
    v[k] = upto[k] - v[k];
    total[k] = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
      if (w < wave) v[k] += sums[k][w];
      total[k] += sums[k][w];
    }
  }
}
template <int NT>
__device__ __forceinline__ int scan_before(int mine, int& total) {
  int v[1] = {mine}, t[1];
  scan_before<NT>(v, t);
  total = t[0];
  return v[0];
}

__device__ __forceinline__ int agent_load(const int32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// One workgroup of NT threads.  Group offsets that decrease give a plan of no meaning whose indexes
// are in range.  Bound by latency: what is looked at again lies in LDS for up to 512 sequences and 256 groups
// (from memory each look took its round trip: 5.5 us of this launch for one sequence, 4.4 from LDS; 8.4 and 5.9
// for a group of four).
template <int NT>
__device__ void make_plan(const LatentDev& a, int rkv, int32_t* lds) {
  const int tid = threadIdx.x, G = a.n_groups;
  constexpr int LDS_G = 256, LDS_B = 512;
  static_assert((5 * LDS_G + 1 + 3 * LDS_B) * 4 <= ABS_LDS * 2, "in the LDS of the absorbed queries");
  int32_t *group_lds = lds, *seq_lds = lds + 5 * LDS_G + 1;
  const bool g_lds = G <= LDS_G, b_lds = a.B <= LDS_B;
  int32_t* tmp = g_lds ? group_lds : a.scratch;
  // per group: the shared rows that all its sequences have, how many have rows, and the first that has; its tiles, its first
  // sequence
  int32_t *group_min = tmp, *group_cnt = tmp + G, *group_seq = tmp + 2 * G, *group_tiles = tmp + 3 * G, *group_off = tmp + 4 * G;
  int32_t *lens = b_lds ? seq_lds : a.lens, *member = b_lds ? seq_lds + LDS_B : a.member;
  int32_t* start = b_lds ? seq_lds + 2 * LDS_B : a.start;
  for (int g = tid; g <= G && G > 0; g += NT) {
    group_off[g] = a.group_off[g];
    if (g == G) break;
    __hip_atomic_store(group_min + g, min(max(a.shared_len[g], 0), a.max_len), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(group_cnt + g, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(group_seq + g, a.B, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  for (int b = tid; b < a.B; b += NT) lens[b] = len_of(a, b);
  __syncthreads();
  for (int b = tid; b < a.B; b += NT) {
    int g = -1;
    const int n = lens[b];
    if (G > 0 && n > 0) {
      g = sequence_of(group_off, G, b);
      if (b < group_off[g] || b >= group_off[g + 1]) g = -1;
    }
    member[b] = g;
    if (g >= 0) {
      atomicMin(group_min + g, n);
      atomicAdd(group_cnt + g, 1);
      atomicMin(group_seq + g, b);
    }
  }
  __syncthreads();
  const int run = (G + NT - 1) / NT, g_lo = min(tid * run, G), g_hi = min(g_lo + run, G);
  auto first_of = [&](int g) { return min(max(group_off[g], 0), a.B); };
  auto blocks_of = [&](int g) { return max(first_of(g + 1) - first_of(g), 0) * a.HB; };
  auto quads_of = [&](int g) { return (blocks_of(g) + 3) / 4; };
  int both[2] = {0, 0}, totals[2];  // quads, and their tiles
  for (int g = g_lo; g < g_hi; ++g) {
    // (two blocks gain nothing: 32 pairs of the 8B layer behind 16384 rows of bf16 212 us apart and 226 shared, of
    // e4m3 138 and 193; 2 x 3 sequences behind 131072 164 and 125, 100 and 106; with 64 heads 16 pairs behind 16384
    // 160 and 134, 127 and 115)
    const int t = agent_load(group_cnt + g) * (int64_t)a.HB >= 3 ? agent_load(group_min + g) / PD_KT : 0;
    group_tiles[g] = t;
    if (t > 0) {
      both[0] += quads_of(g);
      both[1] += quads_of(g) * t;
    }
  }
  scan_before<NT>(both, totals);
  const int total_q = totals[0], total_i = totals[1];
  // own rows
  const int runb = (a.B + NT - 1) / NT, b_lo = min(tid * runb, a.B), b_hi = min(b_lo + runb, a.B);
  int mine = 0, total;
  for (int b = b_lo; b < b_hi; ++b) {
    const int g = member[b], n = lens[b], t = g >= 0 ? group_tiles[g] : 0;
    a.start[b] = start[b] = min(t * PD_KT, n);
    a.member[b] = t == 0 ? -1 : g;
    mine += tiles_of(n - start[b]) * a.HB;
  }
  int at = scan_before<NT>(mine, total);
  for (int b = b_lo; b < b_hi; ++b) {
    const int n = tiles_of(lens[b] - start[b]);
    for (int h = 0; h < a.HB; ++h, at += n) a.tile_off[b * a.HB + h] = at;
  }
  // Own rows, each workgroup in one block's: the least number of tiles a wavefront for which there are enough
  // workgroups, if that is not much more than equal runs need.  Equal runs cross blocks: every wavefront
  // then writes a state, or two, where here the workgroup writes one (of 512 values 64 KB, which the merge reads
  // again), and loads a block's queries more often.  Whole calls over e4m3 rows, equal runs / this, us: 512 values: 41
  // sequences of 1024 rows 39 / 31, of 4096 53 / 45, 250 of 2048 143 / 114, 200 of 4096 (24 tiles a wavefront / 32)
  // 175 / 154, 250 of 8192 (59 / 64) 316 / 273; 256 values: 250 of 512 35 / 30, 100 of 4096 (13 / 16) 44 / 46, 200
  // of 4096 (24 / 32) 71 / 79.
  const int n_s = shared_workgroups(a.nwg, total_i, total), n_p = max(a.nwg - n_s, 1);
  const int least = (ListCut(total, n_p).share + PD_WAVES - 1) / PD_WAVES, more = rkv >= 512 ? least / 3 + 2 : 1;
  constexpr int TRIES = 6;
  auto tried = [&](int k) { return least + more * k / (TRIES - 1); };
  int wanted[TRIES] = {}, sums[TRIES], per_wave = 0, wgs = 0;
  for (int b = b_lo; b < b_hi; ++b) {
    const int n = tiles_of(lens[b] - start[b]);
#pragma unroll
    for (int k = 0; k < TRIES; ++k) wanted[k] += (n + PD_WAVES * tried(k) - 1) / (PD_WAVES * tried(k)) * a.HB;
  }
  scan_before<NT>(wanted, sums);
#pragma unroll
  for (int k = TRIES - 1; k >= 0; --k)
    if (sums[k] <= n_p && tried(k) <= PD_RUN) {  // (longer runs take equal shares, and put states down on their way)
      per_wave = tried(k);
      wgs = wanted[k];
    }
  if (per_wave > 0) {
    for (int b = b_lo; b < b_hi; ++b) {
      const int n = (tiles_of(lens[b] - start[b]) + PD_WAVES * per_wave - 1) / (PD_WAVES * per_wave);
      for (int h = 0; h < a.HB; ++h, wgs += n) a.wg_off[b * a.HB + h] = wgs;
    }
    if (b_lo < a.B && b_hi == a.B) a.wg_off[a.B * a.HB] = wgs;
  }
  // The shared rows' workgroups take a piece each: the least number of tiles a piece for which there are enough of
  // them (with more quads than workgroups a quad is a piece).
  auto pieces_at = [&](int t) {
    int n = 0, sum;
    for (int g = g_lo; g < g_hi; ++g) n += quads_of(g) * ((group_tiles[g] + t - 1) / t);
    scan_before<NT>(n, sum);
    return sum;
  };
  int lo = 1, hi = total_i;  // (as many tiles as there are: a quad is a piece)
  if (total_q < n_s) {
    lo = (total_i + n_s - 1) / n_s;
    hi = (total_i + n_s - total_q - 1) / (n_s - total_q);  // (enough: a quad's last piece is all that is rounded up)
    while (lo < hi) {
      const int mid = lo + (hi - lo) / 2;
      if (pieces_at(mid) <= n_s) hi = mid;
      else lo = mid + 1;
    }
  }
  hi = max(hi, 1);
  int count = 0, pieces;
  for (int g = g_lo; g < g_hi; ++g) count += quads_of(g) * ((group_tiles[g] + hi - 1) / hi);
  int first = scan_before<NT>(count, pieces);
  for (int g = g_lo; g < g_hi; ++g) {
    const int of = (group_tiles[g] + hi - 1) / hi;
    const int64_t end = first + (int64_t)quads_of(g) * of;
    int32_t* d = a.group + GROUP_INTS * g;
    d[G_FIRST] = first;
    d[G_QUADS] = quads_of(g);
    d[G_PIECES] = first < 0 || end > a.max_pieces ? 0 : of;  // (0: of decreasing offsets, no slots)
    d[G_TILES] = group_tiles[g];
    d[G_X0] = first_of(g) * a.HB;
    d[G_BLOCKS] = blocks_of(g);
    d[G_SEQ] = agent_load(group_seq + g);
    first = (int)min(end, (int64_t)a.max_pieces);
  }
  if (tid == 0) {
    a.tile_off[a.B * a.HB] = total;
    a.head[0] = min(pieces, a.max_pieces);
    a.head[1] = n_s;
    a.head[2] = total;
    a.head[3] = per_wave;
  }
}

// ---- attention ------------------------------------------------------------------------
// The products here have no wait for operands: these come from LDS, or were converted a product before
// (tests/test_latent_waits.py looks at the built code).
#define MLA_PRODUCTS(T, op)                                                                                       \
  __device__ __forceinline__ void pv_first(f32x16& d, T x, T y) {                                                 \
    asm volatile("v_mfma_f32_32x32x16_" op " %0, %1, %2, 0" : "=&v"(d) : "v"(x), "v"(y));                         \
  }                                                                                                               \
  __device__ __forceinline__ void pv_next(f32x16& d, T x, T y) {                                                  \
    asm volatile("v_mfma_f32_32x32x16_" op " %0, %1, %2, %0" : "+v"(d) : "v"(x), "v"(y));                         \
  }                                                                                                               \
  __device__ __forceinline__ void pa_next(f32x16& d, T x, T y) {                                                  \
    asm volatile("v_mfma_f32_32x32x16_" op " %0, %1, %2, %0" : "+a"(d) : "v"(x), "v"(y));                         \
  }
MLA_PRODUCTS(bf16x8, "bf16")
MLA_PRODUCTS(f16x8, "f16")
#undef MLA_PRODUCTS
// operands of coming products, written by the vector ALU here at the latest: two wait states
template <class T>
__device__ __forceinline__ void operand_written(T& x) { asm volatile("s_nop 1" : "+v"(x)); }
// 8 e4m3 values as fp16 (exact)
__device__ __forceinline__ f16x8 e4m3_to_f16(uint32_t lo, uint32_t hi) {
  u32x4 w;
  w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, 1.f, false));
  w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, 1.f, true));
  w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, 1.f, false));
  w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, 1.f, true));
  return __builtin_bit_cast(f16x8, w);
}
// LDS transposing read of bytes: in each group of 16 lanes, lane r gives the address of 8 bytes; lane j receives
// byte j % 8 of what lanes j / 8, j / 8 + 2, .. gave.
__device__ __forceinline__ u32x2 lds_read_tr8(const char* p) {
  typedef int i32x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2*)p));
}
// 4 bytes a lane from the lanes' addresses to the LDS byte address `lds`
__device__ __forceinline__ void dma4(const void* src, uint32_t lds) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(src), "{m0}"(lds) : "memory");
}

// A tile in LDS: 32 rows of CHR 16-byte chunks without padding, chunk c of row r at c ^ swz(r)
// (paged_attn.hip).  S^T reads 16 bytes of 16 consecutive rows, which take different banks; the transposing
// reads 16 bytes of rows {0..3, 8..11} (+ 4) at two neighbouring chunks (bf16: 32 bytes of four rows).  In
// eight bits the rows of those that share banks differ in bits 1 and 3 where two rows span the banks (640
// bytes), which go to chunk bits 1 and 2.
template <int DK, int DVL, bool E4M3>
struct LatentTile {
  static constexpr int RB = E4M3 ? DVL + 2 * (DK - DVL) : 2 * DK;  // bytes of a row
  static constexpr int CHR = RB / 16;
  static constexpr bool WIDE = RB % 256 == 128;
  static constexpr int ROWS = WIDE ? 8 : 16;
  static constexpr int PERIOD = ROWS * CHR / 64;
  static constexpr int HALF_COPIES = 16 * CHR / 64;
  static constexpr int BYTES = PD_KT * RB;
  static_assert(RB % 64 == 0 && CHR % (WIDE ? 8 : 4) == 0 && ROWS * CHR % 64 == 0, "whole copies");
  __device__ __forceinline__ static constexpr int swz(int r) {
    if (!WIDE) return r >> 2 & 3;
    return E4M3 ? (r >> 1 & 1) << 1 | (r >> 3 & 1) << 2 | (r >> 2 & 1) : (r >> 1 & 1) << 1 | (r >> 2 & 1) << 2 | (r >> 3 & 1);
  }
  static constexpr int XOR8 = 16 * (E4M3 ? 4 : 1);  // what 8 rows further do to an offset (WIDE)
};

// The absorbed queries (absorb.h), one workgroup, the first, for the plan, and the images of the shared rows' tiles.
constexpr int PREP_THREADS = 128;
// Tile t of group g as LDS holds it (LatentTile of 16 bits), the latents in fp16: what its members with rows all
// have, read through the first of them (the plan uses as much of it as it finds).  Sixteen lanes a row.  Bound by
// latency (lengths, page numbers, rows): 8192 rows of 1152 bytes make the launch 13 us, without images 8.5.
template <int DK, int DVL, bool E4M3>
__device__ __forceinline__ void image_tile(const LatentDev& a, int g, int t) {
  using FT = LatentTile<DK, DVL, false>;
  constexpr int NQ = DVL / 128, RB = LatentTile<DK, DVL, E4M3>::RB;
  __shared__ int least, first;
  const int tid = threadIdx.x, l = tid & 15;
  const int lo = max(a.group_off[g], 0), hi = min(a.group_off[g + 1], a.B), shared = min(max(a.shared_len[g], 0), a.max_len);
  if (tid == 0) {
    least = shared;
    first = a.B;
  }
  __syncthreads();
  for (int b = lo + tid; b < hi; b += PREP_THREADS) {
    const int n = len_of(a, b);
    if (n > 0) {
      atomicMin(&least, n);
      atomicMin(&first, b);
    }
  }
  __syncthreads();
  if (first >= a.B || t >= least / PD_KT) return;
  char* image = a.images + ((int64_t)g * a.image_tiles + t) * FT::BYTES;
  // (everything is asked for before anything is used: a row after the other took a round trip each)
  constexpr int ROWS = PD_KT / 8;
  const char* from[ROWS];
  bool bad[ROWS];
  float power[ROWS];
  u32x4 v[ROWS][NQ], pe[ROWS];
  int page[ROWS];
#pragma unroll
  for (int k = 0; k < ROWS; ++k) page[k] = a.table[(int64_t)first * a.max_pages + page_of(a, t * PD_KT + 8 * k + (tid >> 4))];
#pragma unroll
  for (int k = 0; k < ROWS; ++k) {
    const int p = t * PD_KT + 8 * k + (tid >> 4), row = p - page_of(a, p) * a.page_size;
    bad[k] = page[k] < 0 || page[k] >= a.n_pages;
    const char* at = a.pool + (bad[k] ? 0 : page[k]) * a.page_bytes;
    from[k] = at + (int64_t)row * RB;
    if constexpr (E4M3) power[k] = *(const float*)(at + (int64_t)a.page_size * RB + 4 * (int64_t)row);
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      if constexpr (E4M3) {
        const u32x2 w = *(const u32x2*)(from[k] + 8 * (16 * q + l));
        v[k][q] = u32x4{w[0], w[1], 0u, 0u};
      } else {
        v[k][q] = *(const u32x4*)(from[k] + 16 * (16 * q + l));
      }
    }
    if (l < (DK - DVL) / 8) pe[k] = *(const u32x4*)(from[k] + (E4M3 ? DVL : 2 * DVL) + 16 * l);
  }
#pragma unroll
  for (int k = 0; k < ROWS; ++k) {
    const int r = 8 * k + (tid >> 4);
    if constexpr (E4M3) {
#pragma unroll
      for (int q = 0; q < NQ; ++q) v[k][q] = __builtin_bit_cast(u32x4, e4m3_to_f16(v[k][q][0], v[k][q][1]));
    } else {
      u16x2 top = {0, 0};
#pragma unroll
      for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, v[k][q][e] & 0x7fff7fffu));
      int m = max((int)top[0], (int)top[1]);
#pragma unroll
      for (int d = 8; d > 0; d >>= 1) m = max(m, __shfl_xor(m, d, 64));
      const int e2 = min(max((m >> 7) - 141, E4M3_MIN_EXP), E4M3_MAX_EXP);  // (bits 7 .. 14: the exponent)
      const float down = power_of_two(-e2);
      power[k] = power_of_two(e2);
#pragma unroll
      for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          v[k][q][e] = pack2h(__uint_as_float(v[k][q][e] << 16) * down, __uint_as_float(v[k][q][e] & 0xffff0000u) * down);
    }
#pragma unroll
    for (int q = 0; q < NQ; ++q) *(u32x4*)(image + r * FT::RB + 16 * ((16 * q + l) ^ FT::swz(r))) = v[k][q];
    if (l < (DK - DVL) / 8) *(u32x4*)(image + r * FT::RB + 16 * ((DVL / 8 + l) ^ FT::swz(r))) = pe[k];
    // (a row on no page: NaN for whoever sees it)
    if (l == 0) a.image_powers[((int64_t)g * a.image_tiles + t) * PD_KT + r] = bad[k] ? NAN : power[k];
  }
}
// DK 0: no images.
template <bool E4M3, int DK, int DVL>
__global__ __launch_bounds__(PREP_THREADS) void latent_prepare_kernel(LatentDev a, const bf16_t* q, const bf16_t* Wuk,
                                                                      int hpg, int dn, int dr, int rkv) {
  __shared__ __attribute__((aligned(16))) bf16_t lds[ABS_LDS];
  if (blockIdx.x == 0) {
    make_plan<PREP_THREADS>(a, rkv, (int32_t*)lds);
    return;
  }
  int k = blockIdx.x - 1;
  if constexpr (DK > 0) {  // (the images first: they take longer)
    if (k < a.n_groups * a.image_tiles) {
      image_tile<DK, DVL, E4M3>(a, k / a.image_tiles, k % a.image_tiles);
      return;
    }
    k -= a.n_groups * a.image_tiles;
  }
  const int nx = rkv / 64, ny = (a.B * hpg + 31) / 32;
  constexpr AbsorbOut OUT = E4M3 ? ABS_F16 : DK == 0 ? ABS_FRAG : ABS_BOTH;
  absorb_block<OUT>(q, Wuk, (bf16_t*)a.qabs, (bf16_t*)a.qabs16, (int8_t*)a.qexp, lds, a.B, a.H, 32 * a.HB, hpg, dn, dr,
                    rkv, k % nx, k / nx % ny, k / nx / ny);
}

// How a tile's latents enter the products.
// * AS_BF16 (a bf16 cache): as they are, with bf16 queries and the weights as two bf16 operands.
// * AS_E8 (an e4m3 cache): the e4m3 values, made fp16 as they are read.
// * AS_F16 (images of shared rows): fp16, made by the launch before of e4m3 values, or of bf16 values divided by a
//   power of two of the row (its largest to [2^14, 2^15)): exact down to 2^-31 of the row's largest.
// In the last two a latent is c times its row's power 2^e.  The products take c: logits are multiplied by 2^e
// (before the positional part is added), and a row's weight in the weighted latents is
// p 2^e = 2^(x + e - m) with x the logit in log2 units and m the running maximum of x + e over the rows.  So weights
// are at most 2^(SLACK + BIAS) < 2^16 and fp16 holds them with 11 bits down to 2^-22 of the largest (their
// rounding is an eighth of bf16's, and one operand does where bf16 takes two).  The sum of the p = 2^(x - m) is in
// fp32, whose range holds them down to 2^-14 of the largest even beside the largest power, 2^120, and up to 2^88 each
// for rows of the smallest, 2^-80.  What a reference that moves multiplies the sum by may be as small as 2^-200 (rows
// of zeros, then some of 2^120) while the product counts: StateFactor.
// Absorbed queries are fp16 too, each head's brought to [2^8, 2^9) by a power of two; the rotary part is bf16
// and divided by the same power, so that the logit is multiplied by it last.
enum LatentAs { AS_BF16, AS_E8, AS_F16 };
template <int V>
using As = std::integral_constant<int, V>;
constexpr float E8_SLACK = 7.f, E8_BIAS = 8.f;

// As AS_BF16 the absorbed queries are bf16 (as in the paged decoding): their rounding, 2^-9 of each, is most of the
// error, 2.7e-3 to 3.3e-3 of the output's norm where the output's own rounding is 1.7e-3; with fp16 queries, as AS_E8
// and AS_F16, it is 1.7e-3 in all.
//
// What bounds it.  Own rows: the stream of the rows (in eight bits 20 KB a wavefront and tile, 3.4 TB/s over the
// kernel) behind a fixed 9 us (launch, plan, queries, first tile), then the states.  Shared rows: a tile costs a
// workgroup 3.2 us in bf16, of which its products take about half (100 of 32 cycles a wavefront at the 1.5 to 1.9 GHz
// that such a loop runs at), 2 us of an image (68 products, and no addresses to make); the softmax and the copies
// run between the products, and the reads of four wavefronts keep LDS as busy as S^T's products the matrix cores.
// Ahead of that 9 us as above; behind it the states, 64 KB a block and piece (12 us for 56 MB; the merge reads
// them again, 16 us).
// Tried for the shared rows and not kept: tiles made fp16 by each workgroup, once for its wavefronts: 78 us for 70 in
// bf16, 71 for 72 in e4m3, LDS being read and written once more a tile; operands read further ahead (PF 7, PV 6
// to 8), no change.  (With P V after its own tile's softmax, and pieces that crossed quads, 77.)
template <int DK, int DVL, bool E4M3, int OCC, bool IMAGES>
__global__ __launch_bounds__(64 * PD_WAVES, OCC) void latent_decode_kernel(LatentDev a) {
  using TL = LatentTile<DK, DVL, E4M3>;
  using FT = LatentTile<DK, DVL, false>;  // of images
  constexpr int OWN = E4M3 ? AS_E8 : AS_BF16, SHARED = IMAGES ? AS_F16 : OWN;
  constexpr int RB = TL::RB, CHR = TL::CHR, DR = DK - DVL;
  constexpr int NL = DVL / 16, NR = DR / 16, NC = DVL / 32;
  constexpr int PF = 5;  // operand reads in flight ahead of the products of S
  static_assert(DVL % 128 == 0 && DR % 16 == 0, "decode shape");
  // In eight bits a wavefront has two tiles, all of the LDS at 576 values; what is small lies in a second tile: of
  // wavefront 0 (the plan, before the copies) and of the wavefront itself (reference and sum, after its tiles).
  constexpr int NBUF = E4M3 ? 2 : 1, SMALL = NBUF * PD_WAVES * TL::BYTES - (E4M3 ? PD_WAVES * TL::BYTES : 0);
  // (the plan's, the offsets of the shared rows' copies, each wavefront's page table entries and powers of four tiles)
  constexpr int TABLE = 64 + TL::PERIOD * 256 + PD_WAVES * (E4M3 ? 2048 : 1024);
  constexpr int ALL = NBUF * PD_WAVES * TL::BYTES + (E4M3 ? 0 : 1024 + TABLE);
  // (images: four tiles, the plan's, each wavefront's powers of four tiles)
  constexpr int IMAGE_ALL = IMAGES ? 4 * FT::BYTES + 64 + PD_WAVES * 1024 : 0;
  __shared__ __attribute__((aligned(1024))) char tiles[ALL > IMAGE_ALL ? ALL : IMAGE_ALL];
  auto ml = [&](int w) { return (float*)(tiles + SMALL + w * (E4M3 ? TL::BYTES : 256)); };  // [2][32]

  const int tid = threadIdx.x, lane = tid & 63, wave = wave_id();
  const int half = lane >> 5, col = lane & 31;
  const int total_p = a.head[2], VB = a.B * a.HB;
  const int n_s = __builtin_amdgcn_readfirstlane(a.head[1]);
  const bool on_shared = (int)blockIdx.x < n_s;
  const int wg = on_shared ? xcd_remap(blockIdx.x, n_s) : (int)blockIdx.x - n_s;
  int* plan_x = (int*)(tiles + (IMAGES && on_shared ? 4 * FT::BYTES : SMALL + (E4M3 ? 0 : 1024)));  // [PD_WAVES], then plan_at
  int* plan_at = plan_x + PD_WAVES;

  // ---- what both lists use ----
  // lane offsets in a tile: S^T's operand (chunk 2 i + half of row col, i % 4 = 0..3), V^T's
  int kb[4], vb[4];
  auto offsets = [&](auto as) __attribute__((always_inline)) {
    using T = typename std::conditional<as() == AS_E8, TL, FT>::type;
#pragma unroll
    for (int j = 0; j < 4; ++j) kb[j] = col * T::RB + 16 * ((2 * j + half) ^ T::swz(col));
    if constexpr (as() == AS_E8) {  // rows 4 half + 0..3, 8 + 4 half + 0..3, latents 16 ((lane / 16) % 2) + 8 (lane % 2) (+ 32 j)
      const int i = (lane & 15) >> 1, r = 4 * half + (i & 3) + 8 * (i >> 2);
#pragma unroll
      for (int j = 0; j < 4; ++j) vb[j] = r * T::RB + 16 * ((2 * j + (lane >> 4 & 1)) ^ T::swz(r)) + 8 * (lane & 1);
    } else {  // [8 more rows][32 latents further]: rows 4 half + (lane % 16) / 4, latents 16 ((lane / 16) % 2) + 4 (lane % 4)
#pragma unroll
      for (int h8 = 0; h8 < 2; ++h8)
#pragma unroll
        for (int odd = 0; odd < 2; ++odd) {
          const int r = 8 * h8 + 4 * half + ((lane & 15) >> 2);
          const int d = 32 * odd + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
          vb[2 * h8 + odd] = r * T::RB + 16 * ((d >> 3) ^ T::swz(r)) + 2 * (d & 7);
        }
    }
  };
  // the row at position p of sequence b (the last of the tile's again past the end, which gets no weight)
  auto entry = [&](int b, int p) { return a.table[(int64_t)b * a.max_pages + page_of(a, p)]; };
  auto address = [&](int p, int page, bool& bad, uint64_t& power) {
    const bool out = page < 0 || page >= a.n_pages;
    bad = __ballot(out) != 0;
    const uint64_t base = (uint64_t)(uintptr_t)a.pool + (uint64_t)((out ? 0 : page) * a.page_bytes);
    const int r = p - page_of(a, p) * a.page_size;
    if constexpr (E4M3) power = base + (uint64_t)((int64_t)a.page_size * RB + 4 * (int64_t)r);
    return base + (uint64_t)((int64_t)r * RB);
  };
  auto row_address = [&](uint64_t at, int r) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)at, r) |
           (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(at >> 32), r) << 32;
  };
  const bool whole16 = a.page_size % 16 == 0;  // 16-row halves of whole tiles lie together

  auto pin = [](f32x16(&d)[NC]) __attribute__((always_inline)) {  // stays in the accumulation registers here
#pragma unroll
    for (int c = 0; c < NC; ++c) asm volatile("" : "+a"(d[c]));
  };

  // ---- a wavefront's state: 32 queries ----
  u32x4 qf[NL];          // this lane's head as B operand fragments, bf16 or fp16
  bf16x8 qr[NR];
  float sl2 = a.sl2;     // logits to log2 units (eight bits: times what the fragments were divided by)
  f32x16 acc[NC];
  float m_run, l_run, l_tile;  // (l_tile: the sum of a tile's weights, in order of e)
  bool any_bad;
  auto begin = [&](auto as, int x) __attribute__((always_inline)) {
    const bf16_t* src = a.qabs + (int64_t)x * 32 * DK + 8 * lane;
#pragma unroll
    for (int s = 0; s < NR; ++s) qr[s] = *(const bf16x8*)(src + 512 * (NL + s));
    if constexpr (as() == AS_BF16) {
#pragma unroll
      for (int s = 0; s < NL; ++s) qf[s] = *(const u32x4*)(src + 512 * s);
    } else {
      // stored step 2 i + e of half h has latents 32 i + 16 h + 8 e .., which are what one LDS read of e4m3 values
      // gives; of fp16 values step k of half h takes latents 16 k + 8 h ..
      const bf16_t* src16 = a.qabs16 + (int64_t)x * 32 * DVL;
#pragma unroll
      for (int s = 0; s < NL; ++s)
        qf[s] = *(const u32x4*)(as() == AS_E8 ? src16 + 512 * s + 8 * lane
                                              : src16 + 512 * (s / 2 * 2 + half) + 256 * (s % 2) + 8 * col);
      // one power for the head's queries
      const int8_t* e = a.qexp + ((int64_t)x * 32 + col) * NC;
      int t[NC], top = ABS_MIN_EXP;
#pragma unroll
      for (int i = 0; i < NC; i += 4) {
        const uint32_t w = *(const uint32_t*)(e + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          t[i + k] = (int)(w << (24 - 8 * k)) >> 24;
          top = max(top, t[i + k]);
        }
      }
      // the positional part is divided by it: logits of that part alone hold up to 2^31 beside small absorbed queries,
      // and beside none (or all below 2^-104, which count as zeros) up to fp32's range
      top = top < -112 ? 0 : max(top, -96);
      sl2 = a.sl2 * power_of_two(top);
      const float down = power_of_two(-top);
#pragma unroll
      for (int s = 0; s < NR; ++s) {
        const u32x4 v = __builtin_bit_cast(u32x4, qr[s]);
        u32x4 w;
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = pack2bf(__uint_as_float(v[k] << 16) * down, __uint_as_float(v[k] & 0xffff0000u) * down);
        qr[s] = __builtin_bit_cast(bf16x8, w);
      }
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const _Float16 f = (_Float16)power_of_two(min(max(t[i] - top, -30), 0));  // (below 2^-24: zero)
#pragma unroll
        for (int s = 2 * i; s < 2 * i + 2; ++s) {
          f16x8 v = __builtin_bit_cast(f16x8, qf[s]);
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] *= f;
          qf[s] = __builtin_bit_cast(u32x4, v);
        }
      }
    }
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[c][e] = 0.f;
    m_run = -INFINITY;
    l_run = 0.f;
    any_bad = false;
  };
  // S^T of the tile at kt.  AS_E8, AS_F16: the rows' powers are in it; pw takes those of the rows of s
  // (8 (e / 4) + 4 half + e % 4) from powers(e), the address of four of them, once the tile's last read is asked for.
  auto logits = [&](auto as, const char* kt, f32x16& s, float (&pw)[16], auto powers) __attribute__((always_inline)) {
    auto take_powers = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const f32x4 v4 = *powers(e);
#pragma unroll
        for (int k = 0; k < 4; ++k) pw[e + k] = v4[k];
      }
    };
    auto kread = [&](int i) { return *(const u32x4*)(kt + kb[i % 4] + 128 * (i / 4)); };
    u32x4 raw[PF];  // (pinned: the compiler would read each operand right before its product and wait for it)
#pragma unroll
    for (int j = 0; j < PF; ++j) raw[j] = kread(j);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (as() == AS_E8) {
      f16x8 k0 = e4m3_to_f16(raw[0][0], raw[0][1]), k1 = e4m3_to_f16(raw[0][2], raw[0][3]);
      asm volatile("" : "+v"(k0));
      operand_written(k1);
#pragma unroll
      for (int i = 0; i < NL / 2; ++i) {
        const u32x4 v = raw[(i + 1) % PF];
        if (i == 0) pv_first(s, k0, __builtin_bit_cast(f16x8, qf[0]));
        else pv_next(s, k0, __builtin_bit_cast(f16x8, qf[2 * i]));
        if (i + 1 < NL / 2) {
          k0 = e4m3_to_f16(v[0], v[1]);
          operand_written(k0);
        }
        __builtin_amdgcn_sched_barrier(0);
        pv_next(s, k1, __builtin_bit_cast(f16x8, qf[2 * i + 1]));
        if (i + 1 < NL / 2) {
          k1 = e4m3_to_f16(v[2], v[3]);
          operand_written(k1);
        }
        if (i + PF < NL / 2 + NR) raw[i % PF] = kread(i + PF);
        if (i == NL / 2 - 2) take_powers();
        __builtin_amdgcn_sched_barrier(0);
      }
      mfma_v_done(s);
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] *= pw[e];
      operand_written(s);
#pragma unroll
      for (int j = 0; j < NR; ++j) {
        pv_next(s, __builtin_bit_cast(bf16x8, raw[(NL / 2 + j) % PF]), qr[j]);
      }
      static_assert(NR <= PF - 1, "the positional part is read before the powers are");
    } else if constexpr (as() == AS_F16) {
#pragma unroll
      for (int kk = 0; kk < NL; ++kk) {
        const f16x8 k = __builtin_bit_cast(f16x8, raw[kk % PF]);
        if (kk == 0) pv_first(s, k, __builtin_bit_cast(f16x8, qf[0]));
        else pv_next(s, k, __builtin_bit_cast(f16x8, qf[kk]));
        if (kk + PF < NL + NR) raw[kk % PF] = kread(kk + PF);
        if (kk == NL - 3) take_powers();
        __builtin_amdgcn_sched_barrier(0);
      }
      mfma_v_done(s);
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] *= pw[e];
      operand_written(s);
#pragma unroll
      for (int j = 0; j < NR; ++j) pv_next(s, __builtin_bit_cast(bf16x8, raw[(NL + j) % PF]), qr[j]);
    } else {
#pragma unroll
      for (int kk = 0; kk < NL + NR; ++kk) {
        const bf16x8 k = __builtin_bit_cast(bf16x8, raw[kk % PF]);
        if (kk == 0) pv_first(s, k, __builtin_bit_cast(bf16x8, qf[0]));
        else pv_next(s, k, kk < NL ? __builtin_bit_cast(bf16x8, qf[kk % NL]) : qr[kk - NL < 0 ? 0 : kk - NL]);
        if (kk + PF < NL + NR) raw[kk % PF] = kread(kk + PF);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    mfma_v_done(s);
  };
  // V^T operand of step j = NC u + c: latents 32 c .., rows 16 u + {4 half.., 8 + 4 half..}
  auto vread = [&](auto as, const char* kt, int j) {
    const int c = j % NC, u = j / NC;
    if constexpr (as() == AS_E8) {
      return lds_read_tr8(kt + vb[c % 4] + 128 * (c / 4) + 16 * RB * u);
    } else {
      const char* p = kt + 16 * FT::RB * u + 128 * (c / 2);
      const u32x2 lo = lds_read_tr4((const bf16_t*)(p + vb[c & 1])), hi = lds_read_tr4((const bf16_t*)(p + vb[2 + (c & 1)]));
      return u32x4{lo[0], lo[1], hi[0], hi[1]};
    }
  };
  // A tile's weights as matrix operands: fp16, or two bf16 values each (rounded, and what that lost: a rounding of
  // P alone would add as much error as that of the output)
  struct Weights {
    u32x4 hi[2], lo[2];
  };
  // P V of the tile at kt; step(j) is called behind the products of step j.  Operands are read PV steps ahead and
  // converted one.
  auto weighted = [&](auto as, const char* kt, const Weights& w, auto step) __attribute__((always_inline)) {
    constexpr int PV = as() == AS_E8 ? 5 : 3;
    decltype(vread(as, kt, 0)) vf[PV];
#pragma unroll
    for (int j = 0; j < PV; ++j) vf[j] = vread(as, kt, j);
    f16x8 v;
    if constexpr (as() == AS_E8) {
      v = e4m3_to_f16(vf[0][0], vf[0][1]);
      operand_written(v);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = 0; j < 2 * NC; ++j) {
      if constexpr (as() == AS_E8) {
        pa_next(acc[j % NC], v, __builtin_bit_cast(f16x8, w.hi[j / NC]));
        if (j + PV < 2 * NC) vf[j % PV] = vread(as, kt, j + PV);
        if (j + 1 < 2 * NC) {
          v = e4m3_to_f16(vf[(j + 1) % PV][0], vf[(j + 1) % PV][1]);
          operand_written(v);
        }
      } else {
        if constexpr (as() == AS_F16) {
          pa_next(acc[j % NC], __builtin_bit_cast(f16x8, vf[j % PV]), __builtin_bit_cast(f16x8, w.hi[j / NC]));
        } else {
          pa_next(acc[j % NC], __builtin_bit_cast(bf16x8, vf[j % PV]), __builtin_bit_cast(bf16x8, w.hi[j / NC]));
          pa_next(acc[j % NC], __builtin_bit_cast(bf16x8, vf[j % PV]), __builtin_bit_cast(bf16x8, w.lo[j / NC]));
        }
        if (j + PV < 2 * NC) vf[j % PV] = vread(as, kt, j + PV);
      }
      step(j);
      __builtin_amdgcn_sched_barrier(0);
    }
    mfma_a_done(acc);
    // every read of the tile has returned before copies may overwrite it
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
  };
  // The softmax of a tile in steps that can be spread over the products of another: the references first (they move only
  // when the tile's maximum exceeds one by more than the slack; returns whether the weighted latents are
  // to be multiplied by corr), then 16 exponentials, then 8 pairs of operands.  With powers a weight must stay below
  // 2^16, so that logits are rounded to log2 units once: a fused product, not rounded, may exceed a large maximum's
  // rounded one by 2^7 and more.
  auto softmax_refs = [&](auto as, f32x16& s, const float (&pw)[16], uint64_t heads, float& corr) __attribute__((always_inline)) {
#pragma clang fp contract(off)
    float my = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; ++e) {  // (a power's exponent from its bits; that of a row never written counts as -80)
      if constexpr (as() != AS_BF16) s[e] *= sl2;
      my = fmaxf(my, as() == AS_BF16 ? s[e]
                                     : __builtin_fmaf((float)max(__float_as_uint(pw[e]), (uint32_t)(127 + E4M3_MIN_EXP) << 23),
                                                      0x1p-23f, s[e]));
    }
    my = pair_max32(my);
    if constexpr (as() != AS_BF16) my -= 127.f;
    else my *= sl2;
    const bool move = (__ballot(my > m_run + (as() != AS_BF16 ? E8_SLACK : PD_SLACK)) & heads) != 0;
    // (no branch: products may be under way)
    const float m_new = move ? fmaxf(m_run, my) : m_run, d = m_run - (m_new == -INFINITY ? 0.f : m_new);
    const StateFactor<as() != AS_BF16> f(d);
    corr = f.value();
    l_run = f.sum(l_run);
    m_run = m_new;
    return move;
  };
  auto softmax_exp = [&](auto as, f32x16& s, const float (&pw)[16], int e) __attribute__((always_inline)) {
    const float ref = (m_run == -INFINITY ? 0.f : m_run) - (as() != AS_BF16 ? E8_BIAS : 0.f);
    s[e] = __builtin_amdgcn_exp2f(as() == AS_BF16 ? __builtin_fmaf(s[e], sl2, -ref) : s[e] - ref);
    l_tile = e == 0 ? s[0] : l_tile + s[e];
    if (e == 15) l_run += l_tile;
    if constexpr (as() != AS_BF16) s[e] *= pw[e];
  };
  auto softmax_pack = [&](auto as, f32x16& s, int q) __attribute__((always_inline)) {  // (in place: weights() takes them)
    const float p0 = s[2 * q], p1 = s[2 * q + 1];
    if constexpr (as() != AS_BF16) {
      s[2 * q] = __uint_as_float(pack2h(p0, p1));
    } else {
      const uint32_t h = pack2bf(p0, p1);
      s[2 * q] = __uint_as_float(h);
      s[2 * q + 1] = __uint_as_float(pack2bf(p0 - __uint_as_float(h << 16), p1 - __uint_as_float(h & 0xffff0000u)));
    }
  };
  auto weights = [&](auto as, const f32x16& s) __attribute__((always_inline)) {
    Weights w;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      w.hi[q / 4][q % 4] = __float_as_uint(s[2 * q]);
      w.lo[q / 4][q % 4] = __float_as_uint(s[2 * q + 1]);
    }
    if constexpr (as() == AS_BF16) asm volatile("" : "+v"(w.lo[0]), "+v"(w.lo[1]));
    asm volatile("" : "+v"(w.hi[0]));
    operand_written(w.hi[1]);
    return w;
  };
  auto rescale = [&](float corr) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < NC; ++c) acc_scale(acc[c], corr);
  };
  // One tile at kt, of which `left` rows count; power: of row col (eight bits).  `heads`: the columns with a head.
  // `early` is called when the reads of the first 16 rows (and of all keys) have returned.
  auto tile = [&](char* kt, float power, int left, uint64_t heads, bool first, auto early) __attribute__((always_inline)) {
    constexpr As<OWN> as;
    f32x16 s;
    float pw[16];
    // (the powers pass through the tile's first positional values, which have been read by then: 16 of them a row)
    auto powers = [&](int e) {
      if (e == 0) *(float*)(kt + (col >> 4) * RB + DVL + 4 * (col & 15)) = power;
      const int r = 2 * e + 4 * half;
      return (const f32x4*)(kt + (e >> 3) * RB + DVL + 4 * (r & 15));
    };
    logits(as, kt, s, pw, powers);
    if (left < PD_KT) {  // rows past the end: no weight (a real branch)
      asm volatile("");
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (8 * (e >> 2) + 4 * half + (e & 3) >= left) s[e] = -INFINITY;
    }
    float corr;
    if (softmax_refs(as, s, pw, heads, corr) && !first) rescale(corr);  // (nothing is there yet at the first tile)
#pragma unroll
    for (int e = 0; e < 16; ++e) softmax_exp(as, s, pw, e);
#pragma unroll
    for (int q = 0; q < 8; ++q) softmax_pack(as, s, q);
    const Weights w = weights(as, s);
    weighted(as, kt, w, [&](int j) __attribute__((always_inline)) {
      if (j == NC) {
        mfma_a_done(acc);  // (no branch, where the compiler may move registers, before the products' waits)
        early();
      }
    });
  };
  // the reference and sum of the state, as a merge of states takes them
  auto reference = [&](auto as) { return as() != AS_BF16 ? m_run - E8_BIAS : m_run; };
  auto sum = [&] {
    return any_bad ? NAN : pair_sum32(l_run);  // (a row on no page)
  };
  // first: whether the slot has no state yet; else this one is joined to it
  auto store = [&](auto as, int64_t slot, bool has_head, bool first) __attribute__((always_inline)) {
    float l = sum(), m = reference(as);
    if (!has_head) return;
    const int64_t row = slot * 32 + col;
    float* po = a.part_o + row * DVL + 4 * half;  // lane (head col, half) holds latents 32 c + 8 g + 4 half + 0..3
    if (first) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *(f32x4*)(po + 32 * c + 8 * g) = f32x4{acc[c][4 * g], acc[c][4 * g + 1], acc[c][4 * g + 2], acc[c][4 * g + 3]};
    } else {
      const float m0 = a.part_ml[2 * row], l0 = a.part_ml[2 * row + 1], top = fmaxf(m, m0), ref = top == -INFINITY ? 0.f : top;
      const StateFactor<as() != AS_BF16> f(m - ref), f0(m0 - ref);
      l = f.sum(l) + f0.sum(l0);
      m = top;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          f32x4* at = (f32x4*)(po + 32 * c + 8 * g);
          *at = acc_read4(acc[c], g) * f.value() + *at * f0.value();  // (or the compiler moves and spills accumulators)
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (half == 0) {
      a.part_ml[2 * row] = m;
      a.part_ml[2 * row + 1] = l;
    }
  };

  if (on_shared) {
    // ---- shared rows: pieces of four query blocks ----
    constexpr As<SHARED> as;
    offsets(as);
    // This wavefront's part of a tile's copies: 8 rows (WIDE) or half of 16, its lanes' source offsets in a table in LDS.
    int* table = plan_x + 16;  // row (times 4) << 16 | bytes from its start
    for (int u = tid; !IMAGES && u < 64 * TL::PERIOD; u += 64 * PD_WAVES) {
      const int r = u / CHR, pc = u % CHR;
      table[u] = r << 18 | 16 * (pc ^ TL::swz(r));
    }
    constexpr int NJ = TL::WIDE ? TL::PERIOD : (TL::PERIOD + 1) / 2;
    const int row0 = TL::WIDE ? 8 * wave : 16 * (wave >> 1), flip = TL::WIDE && (wave & 1) ? TL::XOR8 : 0;
    auto copy_of = [&](int j) { return TL::WIDE ? j : min(2 * j + (wave & 1), TL::PERIOD - 1); };
    const uint32_t tiles_lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)tiles) + row0 * RB;
    // copy j of a tile whose row col is at `at`, in three parts (each waits for the LDS reads of the one before)
    struct Copy {
      int from;
      uint32_t lo, hi;
    };
    auto copy_offset = [&](Copy& c, int j) __attribute__((always_inline)) {
      c.from = (table[64 * copy_of(j) + lane] ^ flip) + (row0 << 18);
    };
    auto copy_row = [&](Copy& c, uint64_t at) __attribute__((always_inline)) {
      c.lo = (uint32_t)__builtin_amdgcn_ds_bpermute(c.from >> 16, (int)(uint32_t)at);
      c.hi = (uint32_t)__builtin_amdgcn_ds_bpermute(c.from >> 16, (int)(uint32_t)(at >> 32));
    };
    auto copy_issue = [&](const Copy& c, int j, int buf) __attribute__((always_inline)) {
      const uint64_t src = ((uint64_t)c.hi << 32 | c.lo) + (uint32_t)(c.from & 0xffff);
      const uint32_t dst = __builtin_amdgcn_readfirstlane(tiles_lds + buf * TL::BYTES) + 1024 * copy_of(j);
      asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(src), "{m0}"(dst) : "memory");
    };
    const int* ahead = table + 64 * TL::PERIOD + wave * (E4M3 ? 512 : 256);
    const uint32_t ahead_lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)ahead);
    const int pieces = __builtin_amdgcn_readfirstlane(a.head[0]);
    for (int piece = wg, done = 0; piece < pieces;) {  // (done: tiles of the piece that are behind a state)
      if (tid == 0) plan_x[0] = -1;
      __syncthreads();
      for (int g = tid; g < a.n_groups; g += 64 * PD_WAVES) {
        const int32_t* d = a.group + GROUP_INTS * g;
        if (d[G_FIRST] <= piece && piece < d[G_FIRST] + d[G_QUADS] * d[G_PIECES]) plan_x[0] = g;
      }
      __syncthreads();
      const int g = __builtin_amdgcn_readfirstlane(plan_x[0]);
      if (g < 0) {
        piece += n_s;
        continue;
      }
      const int32_t* d = a.group + GROUP_INTS * g;
      const int quads = __builtin_amdgcn_readfirstlane(d[G_QUADS]), of = __builtin_amdgcn_readfirstlane(d[G_PIECES]);
      const int nt = __builtin_amdgcn_readfirstlane(d[G_TILES]), k = piece - __builtin_amdgcn_readfirstlane(d[G_FIRST]);
      const int q = k % quads, pp = k / quads;
      const int x0 = __builtin_amdgcn_readfirstlane(d[G_X0]) + 4 * q, nx = min(__builtin_amdgcn_readfirstlane(d[G_BLOCKS]) - 4 * q, 4);
      int i = (int)((int64_t)nt * pp / of) + done;
      const int i_hi = (int)((int64_t)nt * (pp + 1) / of), q_hi = min(i + PD_RUN, i_hi);
      // (a wavefront without a block works on the last one's, and stores nothing)
      const int b0 = __builtin_amdgcn_readfirstlane(d[G_SEQ]), x = x0 + min(wave, nx - 1);
      const int h0 = 32 * (x % a.HB);
      const uint64_t heads = __ballot(h0 + col < a.H);
      // Tile i: P V while the softmax of the next tile runs between the products.  Copies are asked for three tiles
      // ahead (four buffers; spread(step of P V, tile) does it between the products), without a register that the
      // compiler would wait for: a wait names how many operations of the later tiles may be under way.
      auto pipeline = [&](auto ops, auto powers_of, auto before, auto spread) __attribute__((always_inline)) {
        constexpr int BYTES = IMAGES ? FT::BYTES : TL::BYTES;
        auto buffer = [&](int j) { return tiles + (j & 3) * BYTES; };
        __syncthreads();
        f32x16 s;
        float pw[16], corr;
        logits(as, buffer(i), s, pw, powers_of(i));
        softmax_refs(as, s, pw, heads, corr);
        bool move = false;  // (nothing is there yet at the first tile)
#pragma unroll
        for (int e = 0; e < 16; ++e) softmax_exp(as, s, pw, e);
#pragma unroll
        for (int q = 0; q < 8; ++q) softmax_pack(as, s, q);
        Weights w = weights(as, s);
        pin(acc);
        for (; i + 1 < q_hi; ++i) {
          pin(acc);
          wait_vm<decltype(ops)::value>();  // (the tile after the next one's may be under way)
          __syncthreads();
          before(i + 3);
          logits(as, buffer(i + 1), s, pw, powers_of(i + 1));
          if (move) rescale(corr);
          constexpr int K = 16 / NC;  // exponentials a step
          weighted(as, buffer(i), w, [&](int j) __attribute__((always_inline)) {
            if (j == 0) move = softmax_refs(as, s, pw, heads, corr);
#pragma unroll
            for (int k = 0; k < K; ++k) {
              const int e = (j - 1) * K + k;
              if (e >= 0 && e < 16) softmax_exp(as, s, pw, e);
              if (e >= 16 && e < 24) softmax_pack(as, s, e - 16);
            }
            spread(j, i + 3);
          });
          w = weights(as, s);
        }
        pin(acc);
        if (move) rescale(corr);
        weighted(as, buffer(i), w, [](int) {});
        wait_vm<0>();  // (copies past the end)
      };
      constexpr int ST = 2 * NC;  // steps of P V
      bool bad = false;
      if constexpr (IMAGES) {
        // 1 KB after the other, in fours for the wavefronts; the tile's powers for each wavefront
        constexpr int CH = FT::BYTES / 1024, NI = (CH + PD_WAVES - 1) / PD_WAVES;
        const uint64_t image = (uint64_t)(uintptr_t)a.images + (uint64_t)g * a.image_tiles * FT::BYTES;
        const float* powers = a.image_powers + (int64_t)g * a.image_tiles * PD_KT;
        const float* ring = (const float*)(plan_x + 16) + 256 * wave;
        const uint32_t ring_lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)ring);
        const uint32_t base_lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)tiles);
        auto copy = [&](int j, int c) __attribute__((always_inline)) {  // (the last tile's again past the end)
          const int at = __builtin_amdgcn_readfirstlane(min(j, q_hi - 1)), k = min(PD_WAVES * c + wave, CH - 1);
          copy_s(image + (uint64_t)at * FT::BYTES + 1024 * k, 16 * lane,
                 __builtin_amdgcn_readfirstlane(base_lds + (j & 3) * FT::BYTES + 1024 * k));
        };
        auto copy_powers = [&](int j) __attribute__((always_inline)) {
          dma4(powers + min(j, q_hi - 1) * (int64_t)PD_KT + col, __builtin_amdgcn_readfirstlane(ring_lds + 256 * (j & 3)));
        };
        auto copy_all = [&](int j) __attribute__((always_inline)) {
          copy_powers(j);
#pragma unroll
          for (int c = 0; c < NI; ++c) copy(j, c);
        };
        __syncthreads();  // (the buffers are free)
        copy_all(i);
        begin(as, x);
        wait_vm<0>();
        copy_all(i + 1);
        copy_all(i + 2);
        pipeline(As<NI + 1>(), [&](int j) { return [=](int e) { return (const f32x4*)(ring + 64 * (j & 3) + 2 * e + 4 * half); }; },
                 [](int) {},
                 [&](int j, int next) __attribute__((always_inline)) {
                   if (j == 1) copy_powers(next);
#pragma unroll
                   for (int c = 0; c < NI; ++c)
                     if (j == 1 + c * (ST - 1) / NI) copy(next, c);
                 });
      } else {
        // the page table's entries two tiles before the copies
        auto ask = [&](int j) __attribute__((always_inline)) {  // (the last tile's entries again past the end)
          dma4(a.table + (int64_t)b0 * a.max_pages + page_of(a, min(j, q_hi - 1) * PD_KT + col), ahead_lds + 256 * (j & 3));
        };
        auto locate = [&](int j, int page) __attribute__((always_inline)) {  // tile j's rows (the last tile's again past the end)
          uint64_t power_at = 0;
          bool out;
          const uint64_t at = address(min(j, q_hi - 1) * PD_KT + col, page, out, power_at);
          bad |= out;
          if constexpr (E4M3) dma4((const void*)(uintptr_t)power_at, ahead_lds + 1024 + 256 * (j & 3));
          return at;
        };
        using Ops = As<NJ + (E4M3 ? 2 : 1)>;  // of a tile: its copies, its powers, table entries
        auto copy = [&](int j, int page) __attribute__((always_inline)) {
          const uint64_t at = locate(j, page);
#pragma unroll
          for (int c = 0; c < NJ; ++c) {
            Copy k;
            copy_offset(k, c);
            copy_row(k, at);
            copy_issue(k, c, j & 3);
          }
        };
        auto powers_of = [&](int j) { return [=](int e) { return (const f32x4*)(ahead + 256 + 64 * (j & 3) + 2 * e + 4 * half); }; };
        const int page0 = entry(b0, i * PD_KT + col), page1 = entry(b0, min(i + 1, q_hi - 1) * PD_KT + col),
                  page2 = entry(b0, min(i + 2, q_hi - 1) * PD_KT + col);
        __syncthreads();  // (the buffers are free)
        copy(i, page0);
        begin(as, x);
        wait_vm<0>();
        copy(i + 1, page1);
        ask(i + 3);
        copy(i + 2, page2);
        ask(i + 4);
        Copy c[NJ];
        int page = 0;
        uint64_t at = 0;
        pipeline(Ops(), powers_of, [&](int next) __attribute__((always_inline)) { page = ahead[64 * (next & 3) + lane]; },
                 [&](int j, int next) __attribute__((always_inline)) {
                   if (j == 1) at = locate(next, page);
                   if (j == 2) ask(next + 2);
#pragma unroll
                   for (int k = 0; k < NJ; ++k) {
                     // (an LDS read's result is asked for some steps behind it)
                     constexpr int LAG = ST >= 32 ? 3 : 1;
                     const int when = 2 + 2 * LAG + k * (ST - 2 - 2 * LAG) / NJ;
                     if (j == when - 2 * LAG) copy_offset(c[k], k);
                     if (j == when - LAG) copy_row(c[k], at);
                     if (j == when) copy_issue(c[k], k, next & 3);
                   }
                 });
      }
      any_bad = bad;
      store(as, (int64_t)4 * piece + wave, wave < nx && h0 + col < a.H, done == 0);
      done += PD_RUN;
      if (q_hi == i_hi) {
        piece += n_s;
        done = 0;
      }
    }
    return;
  }

  // ---- own rows: a run of tiles a wavefront ----
  offsets(As<OWN>());
  const bool in_one = __builtin_amdgcn_readfirstlane(a.head[3]) > 0;
  const int64_t slot0 = (int64_t)4 * a.max_pieces;  // (behind the shared rows')
  int t_lo, t_hi, per;
  if (in_one) {
    if (wg >= __builtin_amdgcn_readfirstlane(a.wg_off[VB])) return;
    for (int x = tid; x < VB; x += 64 * PD_WAVES) {
      const int lo = a.wg_off[x], hi = a.wg_off[x + 1];
      if (lo <= wg && wg < hi) {
        const int at = a.tile_off[x], n = a.tile_off[x + 1] - at;
#pragma unroll
        for (int w = 0; w < PD_WAVES; ++w) {
          plan_x[w] = x;
          plan_at[w] = at;
        }
        plan_at[PD_WAVES] = at + (int)((int64_t)n * (wg - lo) / (hi - lo));
        plan_at[PD_WAVES + 1] = at + (int)((int64_t)n * (wg + 1 - lo) / (hi - lo));
      }
    }
    __syncthreads();
    t_lo = __builtin_amdgcn_readfirstlane(plan_at[PD_WAVES]);
    t_hi = __builtin_amdgcn_readfirstlane(plan_at[PD_WAVES + 1]);
    per = (t_hi - t_lo + PD_WAVES - 1) / PD_WAVES;
  } else {
    const ListCut cut(total_p, a.nwg - n_s);
    t_lo = cut.lo(wg), t_hi = cut.hi(wg), per = cut.per_wave(wg);
    if (t_lo >= t_hi) return;
    for (int x = tid; x < VB; x += 64 * PD_WAVES) {
      const int lo = a.tile_off[x], hi = a.tile_off[x + 1];
#pragma unroll
      for (int w = 0; w < PD_WAVES; ++w) {
        const int t = t_lo + w * per;
        if (t < t_hi && lo <= t && t < hi) {
          plan_x[w] = x;
          plan_at[w] = lo;
        }
      }
    }
    __syncthreads();
  }
  const int t_first = t_lo + wave * per;
  int T = t_first;                                 // this wavefront's run: tiles [T, T_end)
  const int T_end = min(T + per, t_hi);
  int x = 0, b = 0, seq0 = 0, s0 = 0, n = 0, nt = 0;  // the current block: first tile, first row, rows, tiles
  auto sequence = [&](int xx, int& bb, int& ss, int& nn) {
    bb = xx / a.HB;
    ss = __builtin_amdgcn_readfirstlane(a.start[bb]);
    nn = __builtin_amdgcn_readfirstlane(len_of(a, bb));
  };
  if (T < T_end) {
    x = __builtin_amdgcn_readfirstlane(plan_x[wave]);
    seq0 = __builtin_amdgcn_readfirstlane(plan_at[wave]);
    sequence(x, b, s0, n);
    nt = tiles_of(n - s0);
  }
  // whether the share lies in one block's rows (the same in every wavefront)
  const int x_first = __builtin_amdgcn_readfirstlane(plan_x[0]);
  const bool joined = per <= PD_RUN && t_hi <= __builtin_amdgcn_readfirstlane(a.tile_off[x_first + 1]);

  char* kt = tiles + wave * TL::BYTES;
  const uint32_t kt_lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)kt);
  uint32_t voff[TL::PERIOD];  // the copies' sources within ROWS rows
#pragma unroll
  for (int k = 0; k < TL::PERIOD; ++k) {
    const int r = (64 * k + lane) / CHR, pc = (64 * k + lane) % CHR;
    voff[k] = 16u * (uint32_t)(r * CHR + (pc ^ TL::swz(r)));
  }
  // rows 16 g .. 16 g + 15 of a tile whose 16 rows lie together
  auto issue_half = [&](int g, uint64_t at, uint32_t kt_lds) __attribute__((always_inline)) {
    uint64_t base = row_address(at, 16 * g);
    asm volatile("s_nop 4" : "+s"(base));  // (vector ALU to scalar register to memory operation)
    uint32_t lds = kt_lds;  // opaque: its sums with constants are cheaper made again than kept
    asm volatile("" : "+s"(lds));
#pragma unroll
    for (int k = 0; k < TL::HALF_COPIES; ++k) {
      const int q = k / TL::PERIOD;
      uint32_t v = voff[k % TL::PERIOD];
      if (TL::WIDE && (q & 1)) asm volatile("v_xor_b32 %0, %1, %0" : "+v"(v) : "n"(TL::XOR8));  // (again, not kept)
      copy_s(base + (uint64_t)(q * TL::ROWS * RB), v, lds + 16 * g * RB + 1024 * k);
    }
  };
  // any tile: copy k fills chunks 64 k .. 64 k + 63, of rows known at compile time
  auto issue_rows = [&](uint64_t at, char* kt) __attribute__((always_inline)) {
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
      dma16((const bf16_t*)(uintptr_t)(src + 16u * (uint32_t)c), (bf16_t*)(kt + 1024 * k));
      __builtin_amdgcn_sched_barrier(0);  // (or every row's address waits in scalar registers)
    }
  };
  // position of row col of tile t of a block with rows [ss, nn)
  auto position = [&](int ss, int nn, int t) { return min(ss + t * PD_KT + col, nn - 1); };

  bool bad = false;
  float power = 1.f;
  if constexpr (E4M3) __syncthreads();  // (the plan has been read: copies may overwrite it)
  if (T < T_end) {
    const int p = position(s0, n, T - seq0);
    uint64_t power_at = 0;
    const uint64_t at = address(p, entry(b, p), bad, power_at);
    if constexpr (E4M3) power = *(const float*)(uintptr_t)power_at;
    issue_rows(at, kt);
  } else if (!joined) {
    return;
  }

  do {  // a block's part of the run, PD_RUN tiles of it at most
    const int block_end = seq0 + nt, seg_end = min(min(T_end, block_end), T + PD_RUN);
    int x2 = x, b2 = b, s2 = s0, n2 = n, seq2 = seq0;  // the block after it
    const int seg_begin = T, h0 = 32 * (x % a.HB);
    const uint64_t heads = __ballot(h0 + col < a.H);  // (columns without a head move no reference)
    begin(As<OWN>(), x);  // (a wavefront without tiles, in a joined share, has an empty state)
    for (; T < seg_end; ++T) {
      any_bad |= bad;
      const int t = T - seq0, left = n - s0 - t * PD_KT;
      // the tile after this one: the next of the block, or the first of the next that has rows
      int page = 0, p2 = 0;
      const bool more = T + 1 < T_end;
      if (more) {
        if (T + 1 == block_end) {
          seq2 += nt;
          do sequence(++x2, b2, s2, n2);
          while (n2 - s2 == 0);
        }
        p2 = position(s2, n2, T + 1 - seq2);
        page = entry(b2, p2);
      }
      const bool together = more && whole16 && (T + 1 - seq2) * PD_KT <= n2 - s2 - PD_KT;
      wait_vm<0>();
      if constexpr (E4M3) {
        // the other buffer takes the next tile, asked for before this one is worked on
        float power_next = 1.f;
        asm volatile("" : "+v"(page), "+v"(power));  // (loaded: no wait for them behind the copies)
        const int now = __builtin_amdgcn_readfirstlane((T - t_first) & 1), next = (now ^ 1) * PD_WAVES * TL::BYTES;
        if (more) {
          uint64_t power_at = 0;
          const uint64_t at = address(p2, page, bad, power_at);
          if (together) {
            issue_half(0, at, kt_lds + next);
            issue_half(1, at, kt_lds + next);
          } else {
            issue_rows(at, kt + next);
          }
          power_next = *(const float*)(uintptr_t)power_at;
        }
        tile(kt + now * PD_WAVES * TL::BYTES, power, left, heads, T == seg_begin, [] {});
        power = power_next;
      } else {
        uint64_t at = 0;
        tile(kt, 1.f, left, heads, T == seg_begin, [&]() __attribute__((always_inline)) {
          // the next tile's first 16 rows are asked for as soon as those of this one have been read (LDS
          // reads return in order), the others behind the last read
          if (more) {
            uint64_t unused;
            at = address(p2, page, bad, unused);
            if (together) issue_half(0, at, kt_lds);
          }
        });
        if (more) {
          if (together) issue_half(1, at, kt_lds);
          else issue_rows(at, kt);
        }
      }
    }

    if (!joined) {  // leaving the block: its state
      store(As<OWN>(), slot0 + (int64_t)PD_WAVES * wg + wave + x, h0 + col < a.H, seg_begin == max(seq0, t_first));
      x = x2;
      b = b2;
      s0 = s2;
      n = n2;
      seq0 = seq2;
      nt = tiles_of(n - s0);
      continue;
    }

    // the four states of one block: one reference and sum, then the latents, a part of them at a time
    // through LDS: every wavefront writes its part, then sums a quarter of it
    constexpr int PH = E4M3 ? 4 : 2, NH = NC / PH;
    static_assert(PD_WAVES * NH * 4096 <= PD_WAVES * TL::BYTES, "a part of every state fits the (first) tiles");
    const float l = sum(), ref = reference(As<OWN>());
    if (half == 0) {
      ml(wave)[col] = ref;
      ml(wave)[32 + col] = l;
    }
    float* buf = (float*)tiles;
    float M = -INFINITY, L = 0.f, f[PD_WAVES];
    const int hj = 32 * (x_first % a.HB);
    const int64_t row = (slot0 + (in_one ? (int64_t)wg : (int64_t)PD_WAVES * wg + x_first)) * 32 + col;
    float* po = a.part_o + row * DVL + 4 * half;
#pragma unroll
    for (int ph = 0; ph < PH; ++ph) {
      __syncthreads();  // (every wavefront is done with its tile, or with the part before)
      if (ph == 0) {
#pragma unroll
        for (int w = 0; w < PD_WAVES; ++w) M = fmaxf(M, ml(w)[col]);
#pragma unroll
        for (int w = 0; w < PD_WAVES; ++w) {
          const float mw = ml(w)[col];
          const StateFactor<E4M3> of(mw == -INFINITY ? mw : mw - M);
          f[w] = of.value();
          L += of.sum(ml(w)[32 + col]);
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
            if (hj + col < a.H) *(f32x4*)(po + 32 * (ph * NH + c) + 8 * g) = v;
          }
        }
      }
    }
    if (wave == 0 && half == 0 && hj + col < a.H) {
      a.part_ml[2 * row] = M;
      a.part_ml[2 * row + 1] = L;
    }
  } while (!joined && T < T_end);
}

// ---- the merge ------------------------------------------------------------------------
// Where the states of a (sequence, head) are: those of its own rows, then those of the shared ones.
struct LatentStates {
  States own;
  int n = 0, first = 0, step = 0;  // of the shared rows' states: the first slot, and from piece to piece
};
template <bool POWERS_>
struct LatentWhere {
  static constexpr bool POWERS = POWERS_;
  const int32_t *head, *tile_off, *wg_off, *member, *group;
  int HB, nwg, max_pieces;
  __device__ __forceinline__ LatentStates states(int b, int h) const {
    const int x = b * HB + h / 32;
    LatentStates s;
    if (head[3] > 0) {
      s.own.at0 = wg_off[x];
      s.own.n = s.own.n0 = wg_off[x + 1] - s.own.at0;
    } else {
      s.own = States(ListCut(head[2], max(nwg - head[1], 1)), x, tile_off[x], tile_off[x + 1]);
    }
    s.n = s.own.n;
    const int g = member[b];
    if (g >= 0) {
      const int32_t* d = group + GROUP_INTS * g;
      const int j = x - d[G_X0];
      s.n += d[G_PIECES];
      s.first = 4 * (d[G_FIRST] + j / 4) + j % 4;
      s.step = 4 * d[G_QUADS];
    }
    return s;
  }
  __device__ __forceinline__ int64_t row(const LatentStates& s, int k, int h) const {
    const int64_t slot = k < s.own.n ? 4 * (int64_t)max_pieces + s.own.slot(k) : s.first + (int64_t)s.step * (k - s.own.n);
    return slot * 32 + h % 32;
  }
};

struct SharedLayout {
  size_t qabs, qabs16, qexp, part_o, part_ml, plan, images, image_powers, bytes;
  int max_pieces, nwg, image_tiles;  // (0: without images)
};
// Images of the shared rows' tiles, at most 256 MiB of them, for groups of 16 blocks of heads and more on the
// average.  Whole calls without and with them, us (groups x sequences, shared rows each; 64 of their own), the 8B
// layer: bf16 8 x 8, 4096 rows 62 / 67; 1 x 8, 16384 53 / 54; 1 x 16, 4096 51 / 49; 4 x 16, 4096 61 / 62; 1 x 32, 16384 82 / 77;
// 4 x 32, 4096 93 / 88; 1 x 64, 16384 125 / 113; 1 x 256, 8192 272 / 232; e4m3 8 x 8, 4096 60 / 62; 4 x 16, 4096
// 60 / 59; 1 x 64, 16384 115 / 103; 1 x 256, 8192 245 / 209; the 0.5B one, 1 x 64, 1024 30 / 32, 16384 74 / 71.
// The workspace has room for as many tiles as the largest number of such groups has, so that it grows with
// sequences, rows and groups.
constexpr int IMAGE_BLOCKS = 16;
constexpr size_t IMAGE_BYTES = (size_t)256 << 20;
SharedLayout shared_layout(int B, int H, int DK, int DVL, int max_len, int n_groups) {
  const size_t HB = (H + 31) / 32, VB = B * HB;
  SharedLayout l;
  const int64_t tiles = (int64_t)VB * ((max_len + (int64_t)PD_KT - 1) / PD_KT);
  l.nwg = (int)(tiles < 2 ? 2 : tiles < PD_CUS ? tiles : PD_CUS);
  // a piece a workgroup, or a quad a piece (the plan stays below both)
  l.max_pieces = n_groups == 0 ? 0 : (int)(VB / 4 + n_groups > (size_t)l.nwg ? VB / 4 + n_groups : l.nwg);
  const size_t slots = 4 * ((size_t)l.nwg + l.max_pieces) + VB;
  const size_t tile = PD_KT * (2 * (size_t)DK + 4), row_tiles = (max_len + (size_t)PD_KT - 1) / PD_KT;
  const size_t room = n_groups == 0 ? 0 : std::min(IMAGE_BYTES / tile, VB / IMAGE_BLOCKS * row_tiles);
  l.image_tiles = n_groups > 0 && (size_t)n_groups * IMAGE_BLOCKS <= VB && n_groups * row_tiles <= room ? (int)row_tiles : 0;
  l.qabs = 0;
  l.qabs16 = l.qabs + al(VB * 32 * DK * 2);
  l.qexp = l.qabs16 + al(VB * 32 * DVL * 2);
  l.part_o = l.qexp + al(VB * 32 * (DVL / 32));
  l.part_ml = l.part_o + al(slots * 32 * DVL * 4);
  l.plan = l.part_ml + al(slots * 32 * 2 * 4);
  l.images = l.plan + al((8 + 3 * (size_t)B + 2 * (VB + 1) + (GROUP_INTS + 5) * (size_t)n_groups + 1) * 4);
  l.image_powers = l.images + al(room * PD_KT * 2 * DK);
  l.bytes = l.image_powers + al(room * PD_KT * 4);
  return l;
}

// (DK, DVL, workgroups a CU: what LDS and registers hold)
#define MLA_SHARED_SHAPES(X) X(576, 512, 1) X(288, 256, 1) X(160, 128, 2)

}  // namespace

size_t decode_shared_ws_bytes(int B, int H, int DK, int DVL, int max_len, int n_groups) {
  return shared_layout(B, H, DK, DVL, max_len, n_groups).bytes;
}

hipError_t decode_shared(const DecodeShared& p, hipStream_t s) {
  const DecodePaged& d = p.d;
  const int DK = d.rkv + d.dr, DVL = d.rkv, HB = (d.H + 31) / 32, VB = d.B * HB;
  if (d.dn > ABS_DN || d.rkv % 64) return hipErrorInvalidValue;
  const SharedLayout l = shared_layout(d.B, d.H, DK, DVL, d.max_len, p.n_groups);
  char* ws = (char*)d.ws;
  LatentDev a;
  a.pool = (const char*)d.c.pool; a.table = d.c.table; a.n_pages = d.c.n_pages; a.page_size = d.c.page_size;
  a.max_pages = d.c.max_pages;
  // with 2^(shift - 1) < page_size <= 2^shift: 2^(31 + shift) / page_size rounded up, off by less than 1 / page_size
  // in a quotient
  a.div_shift = 0;
  while (((int64_t)1 << a.div_shift) < d.c.page_size) ++a.div_shift;
  a.div_mul = (uint32_t)((((uint64_t)1 << (31 + a.div_shift)) + d.c.page_size - 1) / d.c.page_size);
  a.page_bytes = p.e4m3 ? E4m3Page(d.c.page_size, d.rkv, d.dr).bytes : (int64_t)d.c.page_size * DK * 2;
  a.len = d.len; a.max_len = d.max_len; a.B = d.B; a.H = d.H; a.HB = HB;
  a.qabs = (const bf16_t*)(ws + l.qabs); a.qabs16 = (const bf16_t*)(ws + l.qabs16);
  a.qexp = (const int8_t*)(ws + l.qexp); a.part_o = (float*)(ws + l.part_o); a.part_ml = (float*)(ws + l.part_ml);
  a.sl2 = d.scale * attn::LOG2E; a.nwg = l.nwg;
  a.n_groups = p.n_groups; a.max_pieces = l.max_pieces; a.group_off = p.group_off; a.shared_len = p.shared_len;
  int32_t* at = (int32_t*)(ws + l.plan);
  a.head = at; at += 8;
  a.start = at; at += d.B;
  a.member = at; at += d.B;
  a.lens = at; at += d.B;
  a.tile_off = at; at += VB + 1;
  a.wg_off = at; at += VB + 1;
  a.group = at; at += GROUP_INTS * p.n_groups;
  a.scratch = at;
  a.images = ws + l.images; a.image_powers = (float*)(ws + l.image_powers); a.image_tiles = l.image_tiles;
  const bool images = l.image_tiles > 0;
  prof_begin(KC_ELEM, s);
  const int64_t grid = 1 + (int64_t)p.n_groups * l.image_tiles +
                       (int64_t)(d.rkv / 64) * ((d.B * (int64_t)d.hpg + 31) / 32) * (d.H / d.hpg);
#define PREP(e_, a_, b_)                                                                                      \
  latent_prepare_kernel<e_, a_, b_><<<(unsigned)grid, PREP_THREADS, 0, s>>>(a, (const bf16_t*)d.q, (const bf16_t*)d.Wuk, \
                                                                           d.hpg, d.dn, d.dr, d.rkv)
  if (!images && p.e4m3) PREP(true, 0, 0);
  else if (!images) PREP(false, 0, 0);
#define X(a_, b_, c_)                              \
  else if (DK == a_ && DVL == b_) {                \
    if (p.e4m3) PREP(true, a_, b_);                \
    else PREP(false, a_, b_);                      \
  }
  MLA_SHARED_SHAPES(X)
#undef X
#undef PREP
  // work at full lengths (the device alone knows the others): images of all rows that there is room for, and
  // every row read for each sequence
  const double row_bytes = p.e4m3 ? d.rkv + 2 * d.dr + 4 : DK * 2;
  prof_end(KC_ELEM, s, 2.0 * d.B * d.H * d.dn * d.rkv,
           (double)d.B * d.H * (d.rkv + d.dr + d.dn + d.dr) * 2 +
               (double)p.n_groups * l.image_tiles * PD_KT * (row_bytes + DK * 2 + 4),
           KLABEL("latent_prepare_kernel"));
  prof_begin(KC_ATTN_FWD, s);
#define X(a_, b_, c_)                                                                      \
  if (DK == a_ && DVL == b_) {                                                             \
    constexpr int C_ = c_;                                                                 \
    auto run = [&](auto e, auto i) {                                                       \
      latent_decode_kernel<a_, b_, e(), C_, i()><<<l.nwg, 64 * PD_WAVES, 0, s>>>(a);       \
    };                                                                                     \
    if (p.e4m3 && images) run(std::true_type(), std::true_type());                         \
    else if (p.e4m3) run(std::true_type(), std::false_type());                             \
    else if (images) run(std::false_type(), std::true_type());                             \
    else run(std::false_type(), std::false_type());                                        \
  }
  MLA_SHARED_SHAPES(X)
#undef X
  prof_end(KC_ATTN_FWD, s, 2.0 * d.B * d.H * (double)d.max_len * (DK + DVL),
           (double)d.B * d.max_len * row_bytes, KLABEL("latent_decode_kernel"));
  prof_begin(KC_ELEM, s);
  auto where = [&](auto powers) {
    return LatentWhere<powers()>{a.head, a.tile_off, a.wg_off, a.member, a.group, HB, l.nwg, l.max_pieces};
  };
#define X(a_, b_, c_)                                                                                  \
  if (DK == a_ && DVL == b_) {                                                                         \
    if (p.e4m3 || images) decode_finish<b_>(d, a.part_o, a.part_ml, where(std::true_type()), s);       \
    else decode_finish<b_>(d, a.part_o, a.part_ml, where(std::false_type()), s);                       \
  }
  MLA_SHARED_SHAPES(X)
#undef X
  prof_end(KC_ELEM, s, 2.0 * d.B * d.H * d.dv * d.rkv, ((double)l.nwg + d.B) * d.H * (DVL + 2) * 4,
           KLABEL("paged_finish_kernel"));
  return hipGetLastError();
}

}  // namespace mla
