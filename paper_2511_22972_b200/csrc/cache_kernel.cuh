// Paged key/value cache: where a position lies, how a row is held, and the kernels that write and read rows.
//
// A row is the head_dim values of one token, head and tensor.  BF16 holds them as they are.  E4M3 holds codes c and one scale
// byte s, value = c * 2^(s - 127): with a power of two as scale the only rounding is that of a value to its code, and every value that
// is held is a bf16 number (four significant bits, exponent far inside the range), so reading back is exact.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace fly {
namespace cache {

constexpr uint32_t kFlagNotWritten = 32u;  // row_flags bit 5
constexpr int kScaleBias = 127;
constexpr int kScaleMin = 7;               // 2^-120: what is held stays exact in bf16
constexpr int kScaleNan = 255;

struct View {
  uint8_t* k_pages;
  uint8_t* v_pages;
  uint8_t* k_scales;
  uint8_t* v_scales;
  int64_t page_stride, token_stride, head_stride;  // elements
  const int32_t* table;
  int64_t table_stride;
  const int32_t* lengths;
  int num_pages, page_shift, kv_heads, head_dim;
  int capacity;  // max_pages * page_size
};

struct Rows {
  uint8_t* data;  // bf16
  int64_t batch_stride, token_stride, head_stride;  // elements
};

// Positions that sequence b held before the chunk, -1: the value is out of range and the sequence has none.
__device__ __forceinline__ int length_of(const View& c, int b) {
  const int L = c.lengths[b];
  return L < 0 || L > c.capacity ? -1 : L;
}
__device__ __forceinline__ int count_of(const int32_t* counts, int b, int n) {
  if (!counts) return n;
  const int m = counts[b];
  return m < 0 || m > n ? 0 : m;
}
// Page of position pos of sequence b, -1 if there is none.
__device__ __forceinline__ int page_of(const View& c, int b, int pos) {
  if (pos < 0 || pos >= c.capacity) return -1;
  const int page = c.table[(int64_t)b * c.table_stride + (pos >> c.page_shift)];
  return page < 0 || page >= c.num_pages ? -1 : page;
}
__device__ __forceinline__ int64_t row_at(const View& c, int page, int slot, int head) {
  return (int64_t)page * c.page_stride + (int64_t)slot * c.token_stride + (int64_t)head * c.head_stride;
}
__device__ __forceinline__ int64_t scale_at(const View& c, int page, int slot, int head) {
  return (((int64_t)page * c.kv_heads + head) << c.page_shift) + slot;
}

// Scale byte of a row whose largest magnitude has these bits (bf16, sign cleared): the smallest s >= 7 with amax <= 448 * 2^(s - 127).
// amax = 1.f * 2^(x - 127) and 448 = 1.75 * 2^8.
__device__ __forceinline__ int scale_of(uint32_t amax) {
  if (amax >= 0x7f80u) return kScaleNan;
  const int s = (int)(amax >> 7) - 8 + ((amax & 0x7fu) > 0x60u ? 1 : 0);
  return s < kScaleMin ? kScaleMin : s;
}
// 2^(s - 127); NaN for 255.
__device__ __forceinline__ float scale_value(int s) {
  return __uint_as_float(s == kScaleNan ? 0x7fc00000u : s == 0 ? 0x00400000u : (uint32_t)s << 23);
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t pack_e4m3(float x0, float x1, float x2, float x3) {
  uint16_t a, b;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(a) : "f"(x1), "f"(x0));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(b) : "f"(x3), "f"(x2));
  return (uint32_t)a | ((uint32_t)b << 16);
}
// Two codes as fp32 (every code is an fp16 number).
__device__ __forceinline__ void unpack_e4m3(uint16_t w, float& lo, float& hi) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(w));
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(lo), "=f"(hi) : "r"(h));
}
// Four codes as two pairs of bf16, scaled.
__device__ __forceinline__ uint2 values_e4m3(uint32_t codes, float scale) {
  float a, b, c, d;
  unpack_e4m3((uint16_t)codes, a, b);
  unpack_e4m3((uint16_t)(codes >> 16), c, d);
  return make_uint2(pack_bf16(a * scale, b * scale), pack_bf16(c * scale, d * scale));
}

// Sixteen codes as eight pairs of bf16, scaled, for where conversions are what there is to do.  Placed into a bf16's bits (sign, then exponent and
// mantissa four places lower) a code reads as its value times 2^-120, subnormal codes as subnormal bf16; one multiplication by
// 2^(s - 7) puts both right.  Not so for scales above 134 and for code 0x7f (NaN, which append never writes): plain4_e4m3 says whether
// 4 x 16 codes are without, and any16_e4m3 takes all.
__device__ __forceinline__ bool plain4_e4m3(const uint4 (&c)[4], const int (&s)[4]) {
  uint32_t nan = 0u;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    nan |= ((c[i].x & 0x7f7f7f7fu) + 0x01010101u) | ((c[i].y & 0x7f7f7f7fu) + 0x01010101u) | ((c[i].z & 0x7f7f7f7fu) + 0x01010101u) |
           ((c[i].w & 0x7f7f7f7fu) + 0x01010101u);
  return (nan & 0x80808080u) == 0u && max(max(s[0], s[1]), max(s[2], s[3])) <= 134;
}
__device__ __forceinline__ void plain16_e4m3(const uint4& codes, int s, uint32_t (&w)[8]) {
  const uint32_t c[4] = {codes.x, codes.y, codes.z, codes.w}, f = (uint32_t)(s + 120) * 0x00800080u;  // 2^(s - 7) twice
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint32_t h = __byte_perm(c[i], 0u, k ? 0x3424 : 0x1404);  // two codes in the upper bytes
      const uint32_t v = (h & 0x80008000u) | ((h >> 4) & 0x07f007f0u);
      asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(w[2 * i + k]) : "r"(v), "r"(f));
    }
  }
}
__device__ __forceinline__ void any16_e4m3(const uint4& codes, int s, uint32_t (&w)[8]) {
  const uint32_t c[4] = {codes.x, codes.y, codes.z, codes.w};
  const float scale = scale_value(s);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint2 v = values_e4m3(c[i], scale);
    w[2 * i] = v.x;
    w[2 * i + 1] = v.y;
  }
}

// Eight consecutive bf16.  wide: the address is a whole number of 16 bytes.
__device__ __forceinline__ uint4 load8(const uint8_t* p, bool wide) {
  if (wide) return *reinterpret_cast<const uint4*>(p);
  const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = (uint32_t)h[2 * i] | ((uint32_t)h[2 * i + 1] << 16);
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(uint8_t* p, uint4 v, bool wide) {
  if (wide) {
    *reinterpret_cast<uint4*>(p) = v;
    return;
  }
  uint16_t* h = reinterpret_cast<uint16_t*>(p);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    h[2 * i] = (uint16_t)w[i];
    h[2 * i + 1] = (uint16_t)(w[i] >> 16);
  }
}
__device__ __forceinline__ uint32_t amax2(uint32_t a, uint32_t b) {  // of two pairs of 16-bit magnitudes
  return __vmaxu2(a & 0x7fff7fffu, b & 0x7fff7fffu);
}

constexpr int kThreads = 256;

// One group of D / 8 lanes per (sequence, token, head), eight values of the key and eight of the value per lane.
template <int D, bool E4M3>
__global__ void __launch_bounds__(kThreads) append_kernel(const View c, const Rows k, const Rows v, int B, int n, const int32_t* counts,
                                                          uint32_t* row_flags, int wide) {
  constexpr int kLanes = D / 8;
  asm volatile("griddepcontrol.wait;" ::: "memory");  // the kernel before may have written any of the inputs
  asm volatile("griddepcontrol.launch_dependents;");
  const int lane = (int)threadIdx.x % kLanes;
  const int64_t row = (int64_t)blockIdx.x * (kThreads / kLanes) + threadIdx.x / kLanes;
  if (row >= (int64_t)n * c.kv_heads) return;  // (whole groups)
  const int i = (int)(row / c.kv_heads), head = (int)(row - (int64_t)i * c.kv_heads);
  for (int b = (int)blockIdx.y; b < B; b += (int)gridDim.y) {
    if (i >= count_of(counts, b, n)) continue;
    const int L = length_of(c, b);
    const int64_t pos = (int64_t)L + i;
    const int page = L < 0 || pos >= c.capacity ? -1 : page_of(c, b, (int)pos);
    if (row_flags && lane == 0 && head == 0) row_flags[(int64_t)b * n + i] = page < 0 ? kFlagNotWritten : 0u;
    if (page < 0) continue;
    const int slot = (int)pos & ((1 << c.page_shift) - 1);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const Rows& src = t ? v : k;
      const uint4 x = load8(src.data + 2 * ((int64_t)b * src.batch_stride + (int64_t)i * src.token_stride + (int64_t)head * src.head_stride + lane * 8),
                            (wide >> t) & 1);
      uint8_t* pages = t ? c.v_pages : c.k_pages;
      const int64_t at = row_at(c, page, slot, head) + lane * 8;
      if (!E4M3) {
        *reinterpret_cast<uint4*>(pages + 2 * at) = x;
        continue;
      }
      const uint32_t m2 = __vmaxu2(amax2(x.x, x.y), amax2(x.z, x.w));
      uint32_t m = max(m2 & 0xffffu, m2 >> 16);
      const unsigned group = (kLanes == 32 ? 0xffffffffu : ((1u << kLanes) - 1u) << ((threadIdx.x & 31) / kLanes * kLanes));
      m = __reduce_max_sync(group, m);
      const int s = scale_of(m);
      const float inv = __uint_as_float((uint32_t)(254 - s) << 23);
      uint2 codes = make_uint2(0u, 0u);
      if (s != kScaleNan)
        codes = make_uint2(pack_e4m3(bf16_lo(x.x) * inv, bf16_hi(x.x) * inv, bf16_lo(x.y) * inv, bf16_hi(x.y) * inv),
                           pack_e4m3(bf16_lo(x.z) * inv, bf16_hi(x.z) * inv, bf16_lo(x.w) * inv, bf16_hi(x.w) * inv));
      *reinterpret_cast<uint2*>(pages + at) = codes;
      if (lane == 0) (t ? c.v_scales : c.k_scales)[scale_at(c, page, slot, head)] = (uint8_t)s;
    }
  }
}

template <int D, bool E4M3>
__global__ void __launch_bounds__(kThreads) read_kernel(const View c, const Rows k, const Rows v, int B, int n, const int32_t* starts, int wide) {
  constexpr int kLanes = D / 8;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  const int lane = (int)threadIdx.x % kLanes;
  const int64_t row = (int64_t)blockIdx.x * (kThreads / kLanes) + threadIdx.x / kLanes;
  if (row >= (int64_t)n * c.kv_heads) return;
  const int i = (int)(row / c.kv_heads), head = (int)(row - (int64_t)i * c.kv_heads);
  for (int b = (int)blockIdx.y; b < B; b += (int)gridDim.y) {
    const int64_t pos = (starts ? (int64_t)starts[b] : 0) + i;
    if (pos < 0 || pos >= length_of(c, b)) continue;
    const int page = page_of(c, b, (int)pos);
    if (page < 0) continue;
    const int slot = (int)pos & ((1 << c.page_shift) - 1);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint8_t* pages = t ? c.v_pages : c.k_pages;
      const int64_t at = row_at(c, page, slot, head) + lane * 8;
      uint4 x;
      if (E4M3) {
        const uint2 codes = *reinterpret_cast<const uint2*>(pages + at);
        const float scale = scale_value((t ? c.v_scales : c.k_scales)[scale_at(c, page, slot, head)]);
        const uint2 a = values_e4m3(codes.x, scale), d = values_e4m3(codes.y, scale);
        x = make_uint4(a.x, a.y, d.x, d.y);
      } else {
        x = *reinterpret_cast<const uint4*>(pages + 2 * at);
      }
      const Rows& dst = t ? v : k;
      store8(dst.data + 2 * ((int64_t)b * dst.batch_stride + (int64_t)i * dst.token_stride + (int64_t)head * dst.head_stride + lane * 8), x,
             (wide >> t) & 1);
    }
  }
}

}  // namespace cache
}  // namespace fly
