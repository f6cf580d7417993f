// A paged cache of keys and values: rows written as they are or in 8 bits, and read back.
//
//   8 bits: scale = max |x| / 127 over a row of one head, code = x / scale to the nearest whole number
//
// Memory bound: 2 rows of d entries in, 2 of d codes and two scales out, or the other way.  A wavefront takes four rows of one head: 16 lanes
// a row, 8 channels a lane; the row's largest entry is four exchanges between lanes.  8 192 rows of 8 heads of 128 from and to bf16: written in
// 13.5 to 15 us (3.6 TB/s; with a division an entry 19 to 21), read in 9 to 10.5 (5 TB/s); places are scattered, 128 bytes of codes each.  (The 100 MB
// of these passes are still near when the next one comes: half of what writing reads comes from an L2.)  Written and read as they are: 23.6 us of
// 16-bit types, 51 of floats, 5.7 and 5.2 TB/s of both together.
#include "../../include/sparse_attention.h"

#include "mma_common.hpp"

#include <math.h>

namespace sc {

void note_hip_error(int32_t code);

struct KvParams {
  const void* in[2];
  void* out[2];
  int64_t stride[2];               // of the rows outside the cache, entries
  const int64_t* slots;
  const void* pages_in[2];
  void* pages[2];
  const float* scales_in[2];
  float* scales[2];
  int64_t rows, places;            // places: pages * page_rows
  int32_t kv_heads, d, shift, entries;
};

constexpr int kKvLanes = 16, kKvChannels = 8;      // lanes of a row of one head, and their channels

// The lane's 8 channels of a row, zeros beyond d.
template <typename T, bool VEC> __device__ __forceinline__ void kv_load(const T* row, int c, int d, float (&x)[kKvChannels]) {
  constexpr int V = 16 / (int)sizeof(T);
#pragma unroll
  for (int g = 0; g < kKvChannels / V; ++g) {
    T e[V];
    if constexpr (VEC) {
      v4i w = {0, 0, 0, 0};
      if (c + g * V < d) w = *reinterpret_cast<const v4i*>(row + c + g * V);
      __builtin_memcpy(e, &w, 16);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) e[i] = c + g * V + i < d ? row[c + g * V + i] : T(0);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) x[g * V + i] = (float)e[i];
  }
}
template <typename T, bool VEC> __device__ __forceinline__ void kv_store(T* row, int c, int d, const float (&x)[kKvChannels]) {
  constexpr int V = 16 / (int)sizeof(T);
#pragma unroll
  for (int g = 0; g < kKvChannels / V; ++g) {
    T e[V];
#pragma unroll
    for (int i = 0; i < V; ++i) e[i] = (T)x[g * V + i];
    if constexpr (VEC) {
      v4i w;
      __builtin_memcpy(&w, e, 16);
      if (c + g * V < d) *reinterpret_cast<v4i*>(row + c + g * V) = w;
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (c + g * V + i < d) row[c + g * V + i] = e[i];
    }
  }
}

// One share: a row and head.  Place of it in the cache, or -1.
__device__ __forceinline__ int64_t kv_place(const KvParams& p, int64_t row, int head) {
  const int64_t slot = p.slots[row];
  if (slot < 0 || slot >= p.places) return -1;
  return (((slot >> p.shift) * p.kv_heads + head) << p.shift) + (slot & ((1 << p.shift) - 1));
}

template <typename T, bool BITS8, bool VEC> __global__ __launch_bounds__(256) void kv_write_kernel(const KvParams p) {
  const int64_t share = ((int64_t)blockIdx.x * 256 + threadIdx.x) / kKvLanes, row = share / p.kv_heads;
  const int head = (int)(share - row * p.kv_heads), c = (threadIdx.x % kKvLanes) * kKvChannels;
  if (row >= p.rows) return;
  const int64_t at = kv_place(p, row, head);
  if (at < 0) return;
  float x[2][kKvChannels];
#pragma unroll
  for (int k = 0; k < 2; ++k)
    kv_load<T, VEC>(static_cast<const T*>(p.in[k]) + row * p.stride[k] + (int64_t)head * p.d, c, p.d, x[k]);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if constexpr (BITS8) {
      // the largest size as a whole number: NaN is above infinity, and both above every number
      unsigned most = 0;
#pragma unroll
      for (int i = 0; i < kKvChannels; ++i) most = max(most, __builtin_bit_cast(unsigned, x[k][i]) & 0x7fffffffu);
#pragma unroll
      for (int s = 1; s < kKvLanes; s <<= 1) most = max(most, (unsigned)__shfl_xor((int)most, s));
      const bool finite = most < 0x7f800000u;
      const float scale = finite ? fmaxf(__fdiv_rn(__builtin_bit_cast(float, most), 127.0f), 0x1p-126f) : __builtin_nanf("");
      // x / scale by a product may lie on the other side of a half: what is left of x is exact there, and decides
      const float per = finite ? __fdiv_rn(1.0f, scale) : 0.0f, half = 0.5f * scale;
      float code[kKvChannels], left[kKvChannels], most_left = 0.0f;
#pragma unroll
      for (int i = 0; i < kKvChannels; ++i) {
        code[i] = finite ? rintf(x[k][i] * per) : 0.0f;
        left[i] = __builtin_fmaf(-code[i], scale, x[k][i]);
        most_left = fmaxf(most_left, fabsf(left[i]));
      }
      if (most_left >= half) {
#pragma unroll
        for (int i = 0; i < kKvChannels; ++i) {
          const bool odd = (int)code[i] & 1;
          if (left[i] > half || (left[i] == half && odd)) code[i] += 1.0f;
          else if (left[i] < -half || (left[i] == -half && odd)) code[i] -= 1.0f;
        }
      }
      uint64_t codes = 0;
#pragma unroll
      for (int i = 0; i < kKvChannels; ++i) codes |= (uint64_t)(uint8_t)(int8_t)(int)code[i] << (8 * i);
      if (c < p.entries) *reinterpret_cast<uint64_t*>(static_cast<int8_t*>(p.pages[k]) + at * p.entries + c) = codes;
      if (c == 0) p.scales[k][at] = scale;
    } else {
      kv_store<T, true>(static_cast<T*>(p.pages[k]) + at * p.entries, c, p.entries, x[k]);
    }
  }
}

template <typename T, bool BITS8, bool VEC> __global__ __launch_bounds__(256) void kv_read_kernel(const KvParams p) {
  const int64_t share = ((int64_t)blockIdx.x * 256 + threadIdx.x) / kKvLanes, row = share / p.kv_heads;
  const int head = (int)(share - row * p.kv_heads), c = (threadIdx.x % kKvLanes) * kKvChannels;
  if (row >= p.rows) return;
  const int64_t at = kv_place(p, row, head);
  float x[2][kKvChannels];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if constexpr (BITS8) {
      uint64_t codes = 0;
      float scale = 0.0f;
      if (at >= 0 && c < p.entries) {
        codes = *reinterpret_cast<const uint64_t*>(static_cast<const int8_t*>(p.pages_in[k]) + at * p.entries + c);
        scale = p.scales_in[k][at];
      }
#pragma unroll
      for (int i = 0; i < kKvChannels; ++i) x[k][i] = (float)(int8_t)(codes >> (8 * i)) * scale;
    } else {
      kv_load<T, true>(static_cast<const T*>(p.pages_in[k]) + at * p.entries, c, at >= 0 ? p.entries : 0, x[k]);
    }
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) kv_store<T, VEC>(static_cast<T*>(p.out[k]) + row * p.stride[k] + (int64_t)head * p.d, c, p.d, x[k]);
}

template <typename T> static hipError_t kv_launch(const KvParams& p, bool write, bool bits8, bool vec, hipStream_t s) {
  const int64_t blocks = (p.rows * p.kv_heads * kKvLanes + 255) / 256;
  auto kernel = write ? (bits8 ? (vec ? kv_write_kernel<T, true, true> : kv_write_kernel<T, true, false>)
                               : (vec ? kv_write_kernel<T, false, true> : kv_write_kernel<T, false, false>))
                      : (bits8 ? (vec ? kv_read_kernel<T, true, true> : kv_read_kernel<T, true, false>)
                               : (vec ? kv_read_kernel<T, false, true> : kv_read_kernel<T, false, false>));
  kernel<<<dim3((unsigned)blocks), dim3(256), 0, s>>>(p);
  return hipGetLastError();
}

int32_t kv_entries(const sc_kv_desc* d) {
  const int per = 16 / (d->bits == 8 ? 1 : d->dtype == SC_F32 ? 4 : 2);
  return (d->d + per - 1) / per * per;
}
sc_status check_kv(const sc_kv_desc* d) {
  if (!d) return SC_ERR_NULL;
  if (d->dtype != SC_F32 && d->dtype != SC_F16 && d->dtype != SC_BF16) return SC_ERR_UNSUPPORTED;
  if (d->bits != 0 && d->bits != 8) return SC_ERR_UNSUPPORTED;
  if (d->kv_heads < 1 || d->kv_heads > (1 << 20) || d->d < 1 || d->pages < 1 || d->page_rows < 1 || d->page_rows > 65536 || (d->page_rows & (d->page_rows - 1)))
    return SC_ERR_BAD_SHAPE;
  if ((int64_t)d->pages * d->page_rows > 0x7fffffff / d->kv_heads) return SC_ERR_BAD_SHAPE;
  if (d->d > 128) return SC_ERR_UNSUPPORTED;
  return SC_OK;
}

// the checks that write and read share; vec: the rows outside the cache are whole 16-byte groups
static sc_status kv_check_call(const sc_kv_desc* d, int64_t rows, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                               const int64_t* slots, const void* k_pages, const void* v_pages, const float* k_scales,
                               const float* v_scales, bool* vec, KvParams* p) {
  const sc_status st = check_kv(d);
  if (st != SC_OK) return st;
  const int64_t width = (int64_t)d->kv_heads * d->d;
  if (rows < 0 || rows > 0x7fffffff || rows * d->kv_heads >= (1 << 28) - 16) return SC_ERR_BAD_SHAPE;      // a launch has fewer than 2^32 lanes
  if (k_stride < width || v_stride < width || k_stride > ((int64_t)1 << 40) || v_stride > ((int64_t)1 << 40)) return SC_ERR_BAD_SHAPE;
  if (rows > 0 && (!k || !v || !slots)) return SC_ERR_NULL;
  if (!k_pages || !v_pages || (d->bits == 8 && (!k_scales || !v_scales))) return SC_ERR_NULL;
  const int eb = d->dtype == SC_F32 ? 4 : 2;
  if (((uintptr_t)k | (uintptr_t)v) % eb || (uintptr_t)slots % 8) return SC_ERR_ALIGN;
  if (((uintptr_t)k_pages | (uintptr_t)v_pages | (uintptr_t)k_scales | (uintptr_t)v_scales) & 15) return SC_ERR_ALIGN;
  *vec = d->d * eb % 16 == 0 && (k_stride * eb | v_stride * eb | (int64_t)(uintptr_t)k | (int64_t)(uintptr_t)v) % 16 == 0;
  *p = {};
  p->stride[0] = k_stride;
  p->stride[1] = v_stride;
  p->slots = slots;
  p->rows = rows;
  p->places = (int64_t)d->pages * d->page_rows;
  p->kv_heads = d->kv_heads;
  p->d = d->d;
  p->shift = __builtin_ctz(d->page_rows);
  p->entries = kv_entries(d);
  return SC_OK;
}

static sc_status kv_call(const sc_kv_desc* d, const KvParams& p, bool write, bool vec, void* hip_stream) {
  if (p.rows == 0) return SC_OK;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const hipError_t e = d->dtype == SC_BF16  ? kv_launch<__bf16>(p, write, d->bits == 8, vec, s)
                       : d->dtype == SC_F16 ? kv_launch<_Float16>(p, write, d->bits == 8, vec, s)
                                            : kv_launch<float>(p, write, d->bits == 8, vec, s);
  if (e != hipSuccess) { note_hip_error((int32_t)e); return SC_ERR_HIP; }
  return SC_OK;
}

}  // namespace sc

extern "C" {

sc_status sparse_kv_row_entries(const sc_kv_desc* desc, int32_t* entries) {
  if (!entries) return SC_ERR_NULL;
  *entries = 0;
  const sc_status st = sc::check_kv(desc);
  if (st == SC_OK) *entries = sc::kv_entries(desc);
  return st;
}

sc_status sparse_kv_write(const sc_kv_desc* desc, int64_t rows, const void* k_dev, int64_t k_stride, const void* v_dev, int64_t v_stride,
                          const int64_t* slots_dev, void* k_pages_dev, void* v_pages_dev, float* k_scales_dev, float* v_scales_dev,
                          void* hip_stream) {
  sc::KvParams p;
  bool vec;
  const sc_status st = sc::kv_check_call(desc, rows, k_dev, k_stride, v_dev, v_stride, slots_dev, k_pages_dev, v_pages_dev, k_scales_dev,
                                         v_scales_dev, &vec, &p);
  if (st != SC_OK) return st;
  p.in[0] = k_dev;
  p.in[1] = v_dev;
  p.pages[0] = k_pages_dev;
  p.pages[1] = v_pages_dev;
  p.scales[0] = k_scales_dev;
  p.scales[1] = v_scales_dev;
  return sc::kv_call(desc, p, true, vec, hip_stream);
}

sc_status sparse_kv_read(const sc_kv_desc* desc, int64_t rows, const int64_t* slots_dev, const void* k_pages_dev, const void* v_pages_dev,
                         const float* k_scales_dev, const float* v_scales_dev, void* k_dev, int64_t k_stride, void* v_dev,
                         int64_t v_stride, void* hip_stream) {
  sc::KvParams p;
  bool vec;
  const sc_status st = sc::kv_check_call(desc, rows, k_dev, k_stride, v_dev, v_stride, slots_dev, k_pages_dev, v_pages_dev, k_scales_dev,
                                         v_scales_dev, &vec, &p);
  if (st != SC_OK) return st;
  p.out[0] = k_dev;
  p.out[1] = v_dev;
  p.pages_in[0] = k_pages_dev;
  p.pages_in[1] = v_pages_dev;
  p.scales_in[0] = k_scales_dev;
  p.scales_in[1] = v_scales_dev;
  return sc::kv_call(desc, p, false, vec, hip_stream);
}

}  // extern "C"
