// Attention of a chunk of new tokens over a paged cache.
//
// A warp per (sequence, token, query head).  Positions are taken one at a time with the running maximum and sum of the softmax:
// with m the largest score so far, l = sum e^{s - m} and o = sum e^{s - m} v, a new score s moves m to max(m, s) and scales l
// and o by e^{m_old - m}.  A lane holds D / 32 of the head's values.
#pragma once
#include "cache_kernel.cuh"
#include "fly_common.cuh"

namespace fly {
namespace attn {

struct Params {
  cache::View c;
  cache::Rows q, out;
  float* lse;
  const int32_t* counts;
  int B, n, heads, group;  // group: query heads per key/value head
  int window, sinks;       // window 0: none
  float scale;             // log2(e) * the softmax's scale
};

constexpr int kThreads = 128;

template <int D, bool E4M3>
__global__ void __launch_bounds__(kThreads) attention_kernel(const Params p) {
  constexpr int kVals = D / 32;  // 2 or 4 per lane
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  const int lane = (int)threadIdx.x & 31;
  const int64_t item = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  if (item >= (int64_t)p.B * p.n * p.heads) return;
  const int h = (int)(item % p.heads), i = (int)(item / p.heads % p.n), b = (int)(item / p.heads / p.n);
  if (i >= cache::count_of(p.counts, b, p.n)) return;
  const int kvh = h / p.group;
  const int L = cache::length_of(p.c, b);
  const int hi = L < 0 ? 0 : min(L + i, p.c.capacity - 1) + 1;
  const int lo = p.window > 0 ? max(0, L + i - p.window + 1) : 0;
  auto load = [&](const uint8_t* pages, const uint8_t* scales, int page, int slot, float (&x)[kVals]) {
    const int64_t at = cache::row_at(p.c, page, slot, kvh) + lane * kVals;
    if (E4M3) {
      const float scale = cache::scale_value(scales[cache::scale_at(p.c, page, slot, kvh)]);
#pragma unroll
      for (int j = 0; j < kVals; j += 2) {
        cache::unpack_e4m3(*reinterpret_cast<const uint16_t*>(pages + at + j), x[j], x[j + 1]);
        x[j] *= scale;
        x[j + 1] *= scale;
      }
    } else {
#pragma unroll
      for (int j = 0; j < kVals; j += 2) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(pages + 2 * (at + j));
        x[j] = cache::bf16_lo(w);
        x[j + 1] = cache::bf16_hi(w);
      }
    }
  };
  float q[kVals], o[kVals];
  const uint8_t* qp = p.q.data + 2 * ((int64_t)b * p.q.batch_stride + (int64_t)i * p.q.token_stride + (int64_t)h * p.q.head_stride + lane * kVals);
#pragma unroll
  for (int j = 0; j < kVals; j += 2) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(qp + 2 * j);
    q[j] = cache::bf16_lo(w);
    q[j + 1] = cache::bf16_hi(w);
    o[j] = o[j + 1] = 0.f;
  }
  float m = -INFINITY, l = 0.f;
  for (int pos = p.sinks > 0 ? 0 : lo; pos < hi; ++pos) {
    if (pos >= p.sinks && pos < lo) { pos = lo - 1; continue; }
    const int page = cache::page_of(p.c, b, pos);
    if (page < 0) continue;
    const int slot = pos & ((1 << p.c.page_shift) - 1);
    float k[kVals], v[kVals];
    load(p.c.k_pages, p.c.k_scales, page, slot, k);
    load(p.c.v_pages, p.c.v_scales, page, slot, v);
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < kVals; ++j) s = fmaf(q[j], k[j], s);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    s *= p.scale;
    const float mn = fmaxf(m, s);
    const float ref = mn == -INFINITY ? 0.f : mn;
    const float w = exp2f(s - ref), a = exp2f(m - ref);
    m = mn;
    l = fmaf(l, a, w);
#pragma unroll
    for (int j = 0; j < kVals; ++j) o[j] = fmaf(o[j], a, w == 0.f ? 0.f : w * v[j]);
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  uint8_t* op = p.out.data + 2 * ((int64_t)b * p.out.batch_stride + (int64_t)i * p.out.token_stride + (int64_t)h * p.out.head_stride + lane * kVals);
#pragma unroll
  for (int j = 0; j < kVals; j += 2) *reinterpret_cast<uint32_t*>(op + 2 * j) = cache::pack_bf16(o[j] * inv, o[j + 1] * inv);
  if (p.lse && lane == 0) p.lse[item] = l == 0.f ? -INFINITY : kLn2 * (m + log2f(l));
}

}  // namespace attn
}  // namespace fly
