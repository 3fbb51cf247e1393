// The paged latent cache: new tokens written into it, and pages copied.
//
// Position p of sequence b lies in row p % page_size of page table[b][p / page_size] of the
// pool, and the row is [c^KV | R_p k^PE] (Eq. 5's cache).  Row addresses are 64-bit: a pool of
// 288 GB holds 2.7e8 rows of 1152 bytes.
#include "cache_rows.h"
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

// A workgroup per packed row.  Angles p inv_freq in fp64 turns (one product and one subtraction
// of whole turns, so a position far into a long cache keeps its fraction), sine and cosine of
// the fraction in fp32; they are shared by the row's heads through LDS.  Bound by memory: every
// value is read once and written once: 10981 rows of 6720 values (bf16) 52 us, 5.6 TB/s, where a copy of
// 1 GiB reaches 5.2; a few rows 4.8 us, a launch.
// E4M3: the first wavefront takes the row's latents, 8 a lane, whose largest gives their power of two (cache_rows.h):
// 18217 rows of 576 values and 32 heads of queries 92 us, 5.2 TB/s, as a copy; one row 3.4 us.
template <typename T, bool E4M3>
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
      const int r = (int)(p - pg * a.page_size);
      T* pe;
      if constexpr (E4M3) {
        const E4m3Page layout(a.page_size, a.rkv, a.Gr * a.dr);
        char* y = layout.row(a.pool, page, r);
        pe = (T*)(y + a.rkv);
        if (tid < 64) {
          uint32_t top = 0u;
          for (int c = 8 * tid; c < a.rkv; c += 512) {
            const u32x4 v = *(const u32x4*)(x + c);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t lo = v[k] << 16 & 0x7fffffffu, hi = v[k] & 0x7fff0000u;
              top = max(top, max(lo < 0x7f800000u ? lo : 0u, hi < 0x7f800000u ? hi : 0u));
            }
          }
#pragma unroll
          for (int d = 32; d > 0; d >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d, 64));
          const int e = e4m3_exponent(top);
          for (int c = 8 * tid; c < a.rkv; c += 512) *(u32x2*)(y + c) = to_e4m3(*(const u32x4*)(x + c), power_of_two(-e));
          if (tid == 0) *layout.power(a.pool, page, r) = power_of_two(e);
        }
      } else {
        T* y = (T*)a.pool + ((int64_t)page * a.page_size + r) * a.width;
        pe = y + a.rkv;
        for (int u = tid; u < a.rkv / 4; u += 256) *(V*)(y + 4 * u) = *(const V*)(x + 4 * u);
      }
      for (int u = tid; u < nang / 4; u += 256) {
        const int g = 4 * u / np, d = 4 * u % np;
        rotate(x + a.rkv + g * a.dr, pe + g * a.dr, g, d);
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

// ---- reading rows back ----------------------------------------------------------------
struct ReadDev {
  PagedPool c;
  int B, rkv, pe, n_rows;
  char* rows;
  const int32_t* offsets;
  const int32_t* start;
};

// A wavefront per packed row, 16 bytes a lane; a value is read and written once.  Bound by memory: 44000 rows of e4m3
// to bf16 (79 MB in all) 18.8 us, 4.2 TB/s; 513 rows of bf16 2.9 us, a launch and two dependent loads.
template <typename T, bool E4M3>
__global__ __launch_bounds__(256) void cache_read_kernel(ReadDev a) {
  const int row = 4 * blockIdx.x + wave_id(), lane = threadIdx.x & 63;
  const PagedPool& c = a.c;
  if (row >= a.n_rows || row < a.offsets[0] || row >= a.offsets[a.B]) return;
  const int b = sequence_of(a.offsets, a.B, row);
  const int64_t p = (int64_t)a.start[b] + (row - a.offsets[b]), pg = p < 0 ? -1 : p / c.page_size;
  int page = -1;
  if (pg >= 0 && pg < c.max_pages) page = c.table[(int64_t)b * c.max_pages + pg];
  const int r = (int)(p - pg * c.page_size);
  constexpr int PER = 16 / sizeof(T);  // values of 16 bytes
  T* y = (T*)a.rows + (int64_t)row * c.width;
  if (page < 0 || page >= c.n_pages) {
    const uint32_t nan = sizeof(T) == 4 ? 0x7fc00000u : 0x7fc07fc0u;
    for (int d = PER * lane; d < c.width; d += 64 * PER) *(u32x4*)(y + d) = u32x4{nan, nan, nan, nan};
    return;
  }
  if constexpr (E4M3) {
    const E4m3Page layout(c.page_size, a.rkv, a.pe);
    const char* x = layout.row(c.pool, page, r);
    const float power = *layout.power(c.pool, page, r);
    for (int d = 8 * lane; d < a.rkv; d += 512) *(u32x4*)(y + d) = from_e4m3(*(const u32x2*)(x + d), power);
    for (int d = 8 * lane; d < a.pe; d += 512) {  // (8-byte loads: rows are multiples of 8 bytes)
      const u32x2 *v = (const u32x2*)(x + a.rkv + 2 * d), lo = v[0], hi = v[1];
      *(u32x4*)(y + a.rkv + d) = u32x4{lo[0], lo[1], hi[0], hi[1]};
    }
  } else {
    const T* x = (const T*)c.pool + ((int64_t)page * c.page_size + r) * c.width;
    for (int d = PER * lane; d < c.width; d += 64 * PER) *(u32x4*)(y + d) = *(const u32x4*)(x + d);
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
  if (c.e4m3)
    cache_append_kernel<bf16_t, true><<<c.n_rows, 256, lds, s>>>(a);
  else if (c.t == DT_BF16)
    cache_append_kernel<bf16_t, false><<<c.n_rows, 256, lds, s>>>(a);
  else
    cache_append_kernel<float, false><<<c.n_rows, 256, lds, s>>>(a);
  const double width = (c.rows ? c.c.width : 0) + (c.q ? (double)c.H * (c.dn + c.dr) : 0.0);
  prof_end(KC_ELEM, s, 0.0,
           2.0 * c.n_rows * width * dsize(c.t) - (c.e4m3 && c.rows ? (double)c.n_rows * (c.rkv - 4) : 0.0),
           c.e4m3 ? KLABEL("cache_append_kernel<e4m3>") : KLABEL("cache_append_kernel"));
  return hipGetLastError();
}

hipError_t cache_read(const CacheRead& c, hipStream_t s) {
  if (c.n_rows == 0) return hipSuccess;
  ReadDev a;
  a.c = c.c; a.B = c.B; a.rkv = c.rkv; a.pe = c.c.width - c.rkv; a.n_rows = c.n_rows;
  a.rows = (char*)c.rows; a.offsets = c.offsets; a.start = c.start;
  const int grid = (c.n_rows + 3) / 4;
  prof_begin(KC_ELEM, s);
  if (c.e4m3)
    cache_read_kernel<bf16_t, true><<<grid, 256, 0, s>>>(a);
  else if (c.t == DT_BF16)
    cache_read_kernel<bf16_t, false><<<grid, 256, 0, s>>>(a);
  else
    cache_read_kernel<float, false><<<grid, 256, 0, s>>>(a);
  prof_end(KC_ELEM, s, 0.0,
           2.0 * c.n_rows * c.c.width * dsize(c.t) - (c.e4m3 ? (double)c.n_rows * (c.rkv - 4) : 0.0),
           KLABEL("cache_read_kernel"));
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
