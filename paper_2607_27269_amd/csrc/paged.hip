// The paged latent cache: new tokens written into it, and pages copied.
//
// Position p of sequence b lies in row p % page_size of page table[b][p / page_size] of the
// pool, and the row is [c^KV | R_p k^PE] (Eq. 5's cache).  Row addresses are 64-bit: a pool of
// 288 GB holds 2.7e8 rows of 1152 bytes.
#include "common.h"
#include "kernels.h"

namespace mla {
namespace {

// ---- append ---------------------------------------------------------------------------
struct AppendDev {
  char* pool;
  const int32_t* table;
  int n_pages, page_size, max_pages, width;
  int B, H, dn, dr, rkv, Gr;
  const void* rows;
  const void* q;
  void* q_out;
  const int32_t* offsets;
  const int32_t* start;
  const float* inv_freq;
};

// Four elements of the storage type: 8 bytes (bf16) or 16 (fp32).  A rotary block's halves
// are multiples of four elements, not of eight.
template <typename T> struct Vec4;
template <> struct Vec4<bf16_t> {
  typedef u32x2 V;
  static __device__ __forceinline__ f32x4 up(V v) {
    return f32x4{__uint_as_float(v[0] << 16), __uint_as_float(v[0] & 0xffff0000u),
                 __uint_as_float(v[1] << 16), __uint_as_float(v[1] & 0xffff0000u)};
  }
  static __device__ __forceinline__ V down(f32x4 f) { return V{pack2bf(f[0], f[1]), pack2bf(f[2], f[3])}; }
};
template <> struct Vec4<float> {
  typedef f32x4 V;
  static __device__ __forceinline__ f32x4 up(V v) { return v; }
  static __device__ __forceinline__ V down(f32x4 f) { return f; }
};

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

// A workgroup per packed row.  Angles p inv_freq in fp64 turns (one product and one subtraction
// of whole turns, so a position far into a long cache keeps its fraction), sine and cosine of
// the fraction in fp32; they are shared by the row's heads through LDS.  Bound by memory: every
// value is read once and written once: 10981 rows of 6720 values (bf16) 52 us, 5.6 TB/s, where a copy of
// 1 GiB reaches 5.2; a few rows 4.8 us, a launch.
template <typename T>
__global__ __launch_bounds__(256) void cache_append_kernel(AppendDev a) {
  using V = typename Vec4<T>::V;
  extern __shared__ __attribute__((aligned(16))) float trig[];  // [Gr][dr / 2] cosines, then the sines
  const int row = blockIdx.x, tid = threadIdx.x;
  const int np = a.dr / 2, nang = a.Gr * np;
  if (row < a.offsets[0] || row >= a.offsets[a.B]) return;  // (uniform)
  const int b = sequence_of(a.offsets, a.B, row);
  const int64_t p = (int64_t)a.start[b] + (row - a.offsets[b]);
  for (int k = tid; k < nang; k += 256) {
    double turns = (double)p * (double)a.inv_freq[k] * 0.15915494309189533577;  // 1 / (2 pi)
    turns -= rint(turns);
    float s, c;
    sincospif(2.f * (float)turns, &s, &c);
    trig[k] = c;
    trig[nang + k] = s;
  }
  __syncthreads();
  // four pairs (d, d + np) of a rotary block at x -> y
  auto rotate = [&](const T* x, T* y, int g, int d) {
    const f32x4 c = *(const f32x4*)(trig + g * np + d), s = *(const f32x4*)(trig + nang + g * np + d);
    const f32x4 lo = Vec4<T>::up(*(const V*)(x + d)), hi = Vec4<T>::up(*(const V*)(x + np + d));
    *(V*)(y + d) = Vec4<T>::down(lo * c - hi * s);
    *(V*)(y + np + d) = Vec4<T>::down(lo * s + hi * c);
  };
  if (a.rows) {
    const int64_t pg = p / a.page_size;
    int page = -1;
    if (p >= 0 && pg < a.max_pages) page = a.table[(int64_t)b * a.max_pages + pg];
    if (page >= 0 && page < a.n_pages) {
      const T* x = (const T*)a.rows + (int64_t)row * a.width;
      T* y = (T*)a.pool + ((int64_t)page * a.page_size + (p - pg * a.page_size)) * a.width;
      for (int u = tid; u < a.rkv / 4; u += 256) *(V*)(y + 4 * u) = *(const V*)(x + 4 * u);
      for (int u = tid; u < nang / 4; u += 256) {
        const int g = 4 * u / np, d = 4 * u % np;
        rotate(x + a.rkv + g * a.dr, y + a.rkv + g * a.dr, g, d);
      }
    }
  }
  if (a.q) {
    const int dq = a.dn + a.dr, hpr = a.H / a.Gr;
    const T* x = (const T*)a.q + (int64_t)row * a.H * dq;
    T* y = (T*)a.q_out + (int64_t)row * a.H * dq;
    if (x != y) {
      const int per = a.dn / 4;
      for (int u = tid; u < a.H * per; u += 256) {
        const int e = u / per * dq + 4 * (u % per);
        *(V*)(y + e) = *(const V*)(x + e);
      }
    }
    const int per = np / 4;
    for (int u = tid; u < a.H * per; u += 256) {
      const int i = u / per;
      rotate(x + i * dq + a.dn, y + i * dq + a.dn, i / hpr, 4 * (u % per));
    }
  }
}

// ---- page copies ----------------------------------------------------------------------
// The pairs travel in the launch's arguments: nothing to allocate, upload or keep alive.
constexpr int COPY_PAIRS = 448;  // 3584 of the 4096 bytes that arguments may take
struct CopyDev {
  char* pool;
  int64_t layer_stride, page_bytes;
  int32_t pairs[2 * COPY_PAIRS];
};

// Grid (blocks of a page, pairs, layers); bound by memory: 257 pages of 16 layers, 303 MB, 110 us (5.5
// TB/s read and written, some of the reads from the last-level cache), one page of 16 layers 2.4 us (the call
// 8.6 to 9.4, append's small ones 7.2: a likely cause is the 3.6 KB of arguments, which few pairs carry too).
constexpr int COPY_BLOCK = 256 * 16;
__global__ __launch_bounds__(256) void copy_pages_kernel(CopyDev a) {
  const int64_t at = (int64_t)blockIdx.x * COPY_BLOCK + 16 * threadIdx.x;
  if (at >= a.page_bytes) return;
  char* layer = a.pool + blockIdx.z * a.layer_stride;
  const int64_t src = a.pairs[2 * blockIdx.y], dst = a.pairs[2 * blockIdx.y + 1];
  *(u32x4*)(layer + dst * a.page_bytes + at) = *(const u32x4*)(layer + src * a.page_bytes + at);
}

}  // namespace

hipError_t cache_append(const CacheAppend& c, hipStream_t s) {
  if (c.n_rows == 0 || (!c.rows && !c.q)) return hipSuccess;
  AppendDev a;
  a.pool = (char*)c.c.pool; a.table = c.c.table; a.n_pages = c.c.n_pages;
  a.page_size = c.c.page_size; a.max_pages = c.c.max_pages; a.width = c.c.width;
  a.B = c.B; a.H = c.H; a.dn = c.dn; a.dr = c.dr; a.rkv = c.rkv; a.Gr = c.Gr;
  a.rows = c.rows; a.q = c.q; a.q_out = c.q_out;
  a.offsets = c.offsets; a.start = c.start; a.inv_freq = c.inv_freq;
  const size_t lds = (size_t)c.Gr * c.dr * 4;
  prof_begin(KC_ELEM, s);
  if (c.t == DT_BF16)
    cache_append_kernel<bf16_t><<<c.n_rows, 256, lds, s>>>(a);
  else
    cache_append_kernel<float><<<c.n_rows, 256, lds, s>>>(a);
  const double width = (c.rows ? c.c.width : 0) + (c.q ? (double)c.H * (c.dn + c.dr) : 0.0);
  prof_end(KC_ELEM, s, 0.0, 2.0 * c.n_rows * width * dsize(c.t), KLABEL("cache_append_kernel"));
  return hipGetLastError();
}

hipError_t cache_copy_pages(void* pool, int n_layers, int64_t layer_stride, int64_t page_bytes,
                            const int32_t* pairs, int n_pairs, hipStream_t s) {
  CopyDev a;
  a.pool = (char*)pool;
  a.layer_stride = layer_stride;
  a.page_bytes = page_bytes;
  for (int64_t i0 = 0; i0 < n_pairs; i0 += COPY_PAIRS) {
    const int n = n_pairs - i0 < COPY_PAIRS ? (int)(n_pairs - i0) : COPY_PAIRS;
    for (int i = 0; i < 2 * n; ++i) a.pairs[i] = pairs[2 * i0 + i];
    prof_begin(KC_ELEM, s);
    copy_pages_kernel<<<dim3((unsigned)((page_bytes + COPY_BLOCK - 1) / COPY_BLOCK), n, n_layers), 256, 0,
                        s>>>(a);
    prof_end(KC_ELEM, s, 0.0, 2.0 * n * n_layers * page_bytes, KLABEL("copy_pages_kernel"));
  }
  return hipGetLastError();
}

}  // namespace mla
