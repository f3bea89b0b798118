// Paged key/value cache: where a position lies, how a row is held, and the kernels that write and read rows.
//
// A row is the head_dim values of one token, head and tensor.  BF16 holds them as they are.  E4M3 holds codes c and one scale
// byte s, value = c * 2^(s - 127): with a power of two as scale the only rounding is that of a value to its code, and every value that
// is held is a bf16 number, so reading back is exact: it has four significant bits, is a multiple of 2^-129 (the smallest code at the
// smallest scale; bf16 goes down to 2^-133) and below 2^128.  The last takes care: with the largest scale, 2^120, code 256 would
// stand for 2^128, so magnitudes from 248 * 2^120 on are held as 240 * 2^120, the nearest value that there is.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace fly {
namespace cache {

constexpr uint32_t kFlagNotWritten = 32u;  // row_flags bit 5
constexpr int kScaleMin = 7;               // 2^-120: what is held stays exact in bf16
constexpr int kScaleTop = 247;             // of the largest bf16 numbers: codes from 256 on are not finite
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
// Four codes of up to 256, of which 256 (0x78) becomes 240 (0x77).
__device__ __forceinline__ uint32_t below_256(uint32_t w) { return w - (__vcmpeq4(w & 0x7f7f7f7fu, 0x78787878u) & 0x01010101u); }
// Two codes as fp32 (every code is an fp16 number).
__device__ __forceinline__ void unpack_e4m3(uint16_t w, float& lo, float& hi) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(w));
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(lo), "=f"(hi) : "r"(h));
}
// Four bf16 times inv as four e4m3 codes, and what is left of them as four e5m2 codes.
__device__ __forceinline__ void split_e4m3_e5m2(uint32_t a, uint32_t b, float inv, uint32_t& hi, uint32_t& lo) {
  const float x[4] = {bf16_lo(a) * inv, bf16_hi(a) * inv, bf16_lo(b) * inv, bf16_hi(b) * inv};
  hi = pack_e4m3(x[0], x[1], x[2], x[3]);
  float y[4];
  unpack_e4m3((uint16_t)hi, y[0], y[1]);
  unpack_e4m3((uint16_t)(hi >> 16), y[2], y[3]);
  uint16_t u, v;
  asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(u) : "f"(x[1] - y[1]), "f"(x[0] - y[0]));
  asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(v) : "f"(x[3] - y[3]), "f"(x[2] - y[2]));
  lo = (uint32_t)u | ((uint32_t)v << 16);
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
// 2^(s - 7) puts both right.  Not so for scales above 134 and for code 0x7f (NaN, which append never writes): plain_e4m3 says whether
// N x 16 codes are without, and any16_e4m3 takes all.
template <int N>
__device__ __forceinline__ bool plain_e4m3(const uint4 (&c)[N], const int (&s)[N]) {
  uint32_t nan = 0u;  // (a byte 0x7f or 0xff changes its upper bit when one is added; others only by the carry of one of these)
  int top = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    nan |= ((c[i].x + 0x01010101u) ^ c[i].x) | ((c[i].y + 0x01010101u) ^ c[i].y) | ((c[i].z + 0x01010101u) ^ c[i].z) | ((c[i].w + 0x01010101u) ^ c[i].w);
    top = max(top, s[i]);
  }
  return (nan & 0x80808080u) == 0u && top <= 134;
}
__device__ __forceinline__ void plain16_e4m3(const uint4& codes, int s, uint32_t (&w)[8]) {
  const uint32_t c[4] = {codes.x, codes.y, codes.z, codes.w}, f = (uint32_t)(s + 120) * 0x00800080u;  // 2^(s - 7) twice
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint32_t h = __byte_perm(c[i], 0u, k ? 0x4342 : 0x4140);  // two codes in the lower bytes
      const uint32_t v = (h & 0x00800080u) * 0xf0u + h * 16u;        // four places up, the sign (2^7, now 2^11) to 2^15: two of the four on the FMA pipe
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

// Threads of a block, and rows of a lane group read together so that their loads are in flight together.  us, rows at a time: append 3 x 4099
// tokens of 8 heads x 128 to e4m3 1: 15.7 = 4.8 TB/s (blocks of 256 threads 16.8), 2: 19.7; read 8 x 4 - 16 k tokens of 8 heads x 128 from e4m3
// 1: 102.4, 2: 101.9, 4: 96.1 = 5.1 TB/s (blocks of 128 threads 98.9), 8: 103.
constexpr int kAppendThreads = 128, kReadThreads = 256, kReadRows = 4;

// A group of D / 16 lanes per (sequence, token, head), sixteen values of the key and sixteen of the value per lane.  What bounds these kernels is
// bytes, or for small calls the chain length -> page -> row.
template <int D, bool E4M3>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(const View c, const Rows k, const Rows v, int B, int n, const int32_t* counts,
                                                          uint32_t* row_flags, int wide) {
  constexpr int kLanes = D / 16, kGroups = kAppendThreads / kLanes;
  asm volatile("griddepcontrol.wait;" ::: "memory");  // the kernel before may have written any of the inputs
  asm volatile("griddepcontrol.launch_dependents;");
  const int lane = (int)threadIdx.x % kLanes;
  const uint32_t row = blockIdx.x * kGroups + threadIdx.x / kLanes, rows = (uint32_t)n * (uint32_t)c.kv_heads;
  const int token = (int)(row / (uint32_t)c.kv_heads), head = (int)(row - (uint32_t)token * (uint32_t)c.kv_heads);
  const unsigned group = ((1u << kLanes) - 1u) << ((threadIdx.x & 31) / kLanes * kLanes);
  for (int b = (int)blockIdx.y; b < B; b += (int)gridDim.y) {
    const int count = count_of(counts, b, n), L = length_of(c, b);
    if (row >= rows || token >= count) continue;  // (whole groups)
    const int page = L < 0 || (int64_t)L + token >= c.capacity ? -1 : page_of(c, b, L + token);
    uint4 x[2][2];  // (the rows need no page)
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const Rows& src = t ? v : k;
      const uint8_t* from = src.data + 2 * ((int64_t)b * src.batch_stride + (int64_t)token * src.token_stride + (int64_t)head * src.head_stride + lane * 16);
      x[t][0] = load8(from, (wide >> t) & 1);
      x[t][1] = load8(from + 16, (wide >> t) & 1);
    }
    if (row_flags && lane == 0 && head == 0) row_flags[(int64_t)b * n + token] = page < 0 ? kFlagNotWritten : 0u;
    if (page < 0) continue;
    const int slot = (L + token) & ((1 << c.page_shift) - 1);
    const int64_t at = row_at(c, page, slot, head) + lane * 16;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      uint8_t* pages = t ? c.v_pages : c.k_pages;
      const uint4 y = x[t][0], z = x[t][1];
      if (!E4M3) {
        *reinterpret_cast<uint4*>(pages + 2 * at) = y;
        *reinterpret_cast<uint4*>(pages + 2 * at + 16) = z;
        continue;
      }
      const uint32_t m2 = __vmaxu2(__vmaxu2(amax2(y.x, y.y), amax2(y.z, y.w)), __vmaxu2(amax2(z.x, z.y), amax2(z.z, z.w)));
      uint32_t m = max(m2 & 0xffffu, m2 >> 16);
      m = __reduce_max_sync(group, m);
      const int s = scale_of(m);
      const float inv = __uint_as_float((uint32_t)(254 - s) << 23);
      uint4 codes = make_uint4(0u, 0u, 0u, 0u);
      if (s != kScaleNan)
        codes = make_uint4(pack_e4m3(bf16_lo(y.x) * inv, bf16_hi(y.x) * inv, bf16_lo(y.y) * inv, bf16_hi(y.y) * inv),
                           pack_e4m3(bf16_lo(y.z) * inv, bf16_hi(y.z) * inv, bf16_lo(y.w) * inv, bf16_hi(y.w) * inv),
                           pack_e4m3(bf16_lo(z.x) * inv, bf16_hi(z.x) * inv, bf16_lo(z.y) * inv, bf16_hi(z.y) * inv),
                           pack_e4m3(bf16_lo(z.z) * inv, bf16_hi(z.z) * inv, bf16_lo(z.w) * inv, bf16_hi(z.w) * inv));
      if (s == kScaleTop) codes = make_uint4(below_256(codes.x), below_256(codes.y), below_256(codes.z), below_256(codes.w));
      *reinterpret_cast<uint4*>(pages + at) = codes;
      if (lane == 0) (t ? c.v_scales : c.k_scales)[scale_at(c, page, slot, head)] = (uint8_t)s;
    }
  }
}

// The same groups; a lane's sixteen values come as codes or as they are.
template <int D, bool E4M3, int ROWS>
__global__ void __launch_bounds__(kReadThreads) read_kernel(const View c, const Rows k, const Rows v, int B, int n, const int32_t* starts, int wide) {
  constexpr int kLanes = D / 16, kGroups = kReadThreads / kLanes;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  const int lane = (int)threadIdx.x % kLanes;
  const uint32_t row0 = blockIdx.x * (kGroups * ROWS) + threadIdx.x / kLanes, rows = (uint32_t)n * (uint32_t)c.kv_heads;
  for (int b = (int)blockIdx.y; b < B; b += (int)gridDim.y) {
    const int64_t start = starts ? (int64_t)starts[b] : 0;
    const int L = length_of(c, b);
    int page[ROWS], token[ROWS], head[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const uint32_t row = row0 + r * kGroups;
      token[r] = (int)(row / (uint32_t)c.kv_heads);
      head[r] = (int)(row - (uint32_t)token[r] * (uint32_t)c.kv_heads);
      const int64_t pos = start + token[r];
      page[r] = row < rows && pos >= 0 && pos < L ? page_of(c, b, (int)pos) : -1;
    }
    uint4 x[ROWS][2][2];
    int s[ROWS][2];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (page[r] < 0) continue;
      const int slot = (int)(start + token[r]) & ((1 << c.page_shift) - 1);
      const int64_t at = row_at(c, page[r], slot, head[r]) + lane * 16;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint8_t* pages = t ? c.v_pages : c.k_pages;
        if (E4M3) {
          x[r][t][0] = *reinterpret_cast<const uint4*>(pages + at);
          s[r][t] = (t ? c.v_scales : c.k_scales)[scale_at(c, page[r], slot, head[r])];
        } else {
          x[r][t][0] = *reinterpret_cast<const uint4*>(pages + 2 * at);
          x[r][t][1] = *reinterpret_cast<const uint4*>(pages + 2 * at + 16);
        }
      }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (page[r] < 0) continue;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (E4M3) {
          uint32_t w[8];
          any16_e4m3(x[r][t][0], s[r][t], w);
          x[r][t][0] = make_uint4(w[0], w[1], w[2], w[3]);
          x[r][t][1] = make_uint4(w[4], w[5], w[6], w[7]);
        }
        const Rows& dst = t ? v : k;
        uint8_t* to = dst.data + 2 * ((int64_t)b * dst.batch_stride + (int64_t)token[r] * dst.token_stride + (int64_t)head[r] * dst.head_stride + lane * 16);
        store8(to, x[r][t][0], (wide >> t) & 1);
        store8(to + 16, x[r][t][1], (wide >> t) & 1);
      }
    }
  }
}

}  // namespace cache
}  // namespace fly
