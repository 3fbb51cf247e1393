// Sequences of different lengths behind one another: their query tiles, and the order in which the
// tiles are worked on.
#pragma once
#include "common.h"

namespace mla {

// Sequence b has the queries q_off[b] .. q_off[b + 1] - 1 and the keys kv_off[b] .. (device [B + 1]
// each, clamped to n_q and n_kv), its queries at the last positions of its keys.  Tiles of `bq`
// queries are numbered without a scan over the lengths: sequence b owns the numbers from
// q_off[b] / bq + b, at least as many as it has tiles, and the few others are empty.
struct PackedSeqs {
  const int32_t *q_off, *kv_off;
  int B, n_q, n_kv, bq;

  struct Tile {
    int qs, ks, Tq, Tk;  // the sequence's first query and key row, its queries and keys
    int q0;              // first query of the tile (empty: not within 0 .. Tq - 1)
    __device__ __forceinline__ bool empty() const { return q0 < 0 || q0 >= Tq; }
    // keys that the tile's last query can see
    __device__ __forceinline__ int keys(int bq) const { return max(min(Tk, q0 + bq + Tk - Tq), 0); }
  };
  __device__ __forceinline__ int q_at(int b) const { return min(max(q_off[b], 0), n_q); }
  __device__ __forceinline__ int k_at(int b) const { return min(max(kv_off[b], 0), n_kv); }
  __device__ __forceinline__ Tile tile(int number) const {
    int b = 0;
    for (int hi = B - 1; b < hi;) {  // the last sequence whose numbers start here or before
      const int mid = (b + hi + 1) >> 1;
      if (q_at(mid) / bq + mid <= number) b = mid;
      else hi = mid - 1;
    }
    const int qs = q_at(b), ks = k_at(b);
    return Tile{qs, ks, max(q_at(b + 1) - qs, 0), max(k_at(b + 1) - ks, 0), (number - (qs / bq + b)) * bq};
  }
};

// The tiles 0 .. n - 1, those with the most keys first (in ORDER_BUCKETS classes), so that no long
// tile starts last, each as the five numbers that a workgroup needs of it (found by a search over
// the offsets, its loads one after the other: 3 us and more where every workgroup does it itself).
// One workgroup of 256 threads, a counting sort; the order within a class is not fixed, and no
// result depends on it.  At most ORDER_MAX tiles of ORDER_SEQS sequences.
constexpr int ORDER_MAX = 4096, ORDER_SEQS = 1024, ORDER_BUCKETS = 1024;
constexpr int ORDER_INTS = 8;  // of an entry: qs, ks, Tq, Tk, q0 (and three not used)
__device__ __forceinline__ void order_tiles(const PackedSeqs& in, int n, int32_t* order) {
  __shared__ int count[ORDER_BUCKETS], top, wave_sum[4];
  __shared__ int keys[ORDER_MAX];
  __shared__ int32_t off[2][ORDER_SEQS + 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int i = tid; i < ORDER_BUCKETS; i += 256) count[i] = 0;
  for (int i = tid; i <= in.B; i += 256) {
    off[0][i] = in.q_off[i];
    off[1][i] = in.kv_off[i];
  }
  if (tid == 0) top = 1;
  __syncthreads();
  const PackedSeqs q{off[0], off[1], in.B, in.n_q, in.n_kv, in.bq};
  int mine = 0;
  for (int i = tid; i < n; i += 256) {
    const PackedSeqs::Tile t = q.tile(i);
    keys[i] = t.empty() ? 0 : t.keys(q.bq);
    mine = max(mine, keys[i]);
  }
  atomicMax(&top, mine);
  __syncthreads();
  auto bucket = [&](int i) { return ORDER_BUCKETS - 1 - (int)((int64_t)keys[i] * (ORDER_BUCKETS - 1) / top); };
  for (int i = tid; i < n; i += 256) atomicAdd(&count[bucket(i)], 1);
  __syncthreads();
  int c[ORDER_BUCKETS / 256], sum = 0;  // the classes' first places
#pragma unroll
  for (int k = 0; k < ORDER_BUCKETS / 256; ++k) {
    c[k] = sum;
    sum += count[ORDER_BUCKETS / 256 * tid + k];
  }
  int upto = sum;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int v = __shfl_up(upto, d, 64);
    if (lane >= d) upto += v;
  }
  if (lane == 63) wave_sum[wave] = upto;
  __syncthreads();
  for (int w = 0; w < wave; ++w) upto += wave_sum[w];
#pragma unroll
  for (int k = 0; k < ORDER_BUCKETS / 256; ++k) count[ORDER_BUCKETS / 256 * tid + k] = upto - sum + c[k];
  __syncthreads();
  for (int i = tid; i < n; i += 256) {
    const PackedSeqs::Tile t = q.tile(i);
    int32_t* o = order + ORDER_INTS * atomicAdd(&count[bucket(i)], 1);
    o[0] = t.qs;
    o[1] = t.ks;
    o[2] = t.Tq;
    o[3] = t.Tk;
    o[4] = t.q0;
  }
}
__device__ __forceinline__ PackedSeqs::Tile ordered_tile(const int32_t* order, int nth) {
  const int32_t* o = order + (int64_t)ORDER_INTS * nth;
  return PackedSeqs::Tile{o[0], o[1], o[2], o[3], o[4]};
}

}  // namespace mla
