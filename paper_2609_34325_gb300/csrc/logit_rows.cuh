// Rows of logits (bf16, fp16 or fp32, at any alignment) as the kernels over them read
// them: 16-byte granules, and the sums of a softmax and its entropy from them.
//
// With m the largest logit, d_j = z_j - m and e_j = e^{k d_j} for a factor k (one over the
// temperature; given as `scale` = k log2 e, so that one multiplication leads to the base-2
// exponential), a part of a row is (m, s = sum e_j, t = sum e_j d_j).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "dora_ptx.cuh"
#include "granule.cuh"
#include "update_ptx.cuh"

namespace dora {
namespace policy {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

constexpr float kFloor = -1e30f;          // e^kFloor is 0: keeps 0 * inf out of e d

// A row's granules.  [whole_lo, whole_hi): those that lie wholly in its first n
// elements; [0, some_hi): those that hold some of them.
template <typename T>
struct RowPtr {
  static constexpr int kE = Granule<T>::kElems;
  const T* z;                             // the row's first element
  int mis;                                // elements of its first granule before it
  int whole_lo, whole_hi, some_hi;
  __device__ __forceinline__ RowPtr(const T* p, int n)
      : z(p), mis(static_cast<int>((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T))) {
    whole_lo = mis > 0 ? 1 : 0;
    whole_hi = (n + mis) / kE;
    some_hi = (n + mis + kE - 1) / kE;
  }
  __device__ __forceinline__ bool whole(int i) const { return i >= whole_lo && i < whole_hi; }
  __device__ __forceinline__ int granules(int classes) const {
    return (classes + mis + kE - 1) / kE;
  }
  __device__ __forceinline__ const uint4* at(int i) const {
    return reinterpret_cast<const uint4*>(z - mis) + i;
  }
  // The granules of a row that starts like this one.
  __device__ __forceinline__ uint4* as_granules(T* to) const {
    return reinterpret_cast<uint4*>(to - mis);
  }
  // Granule i of the row by its elements, those outside [0, n) as -inf.
  __device__ __forceinline__ uint4 load_part(int i, int n) const {
    const int c = i * kE - mis;
    float v[kE];
#pragma unroll
    for (int e = 0; e < kE; ++e)
      v[e] = c + e >= 0 && c + e < n ? to_float(z[c + e]) : -INFINITY;
    return Granule<T>::pack(v);           // exact: the values come from T
  }
  // Granule i of the row, -inf where it has no legal logits.
  __device__ __forceinline__ uint4 load(int i, int n) const {
    if (whole(i)) return *at(i);
    if (i < some_hi) return load_part(i, n);
    constexpr uint32_t kNone = Granule<T>::kNegInfWord;
    return make_uint4(kNone, kNone, kNone, kNone);
  }
  // The same of a granule that is at hand.
  __device__ __forceinline__ uint4 only_row(uint4 q, int i, int n) const {
    const int c = i * kE - mis;
    float v[kE];
    Granule<T>::unpack(q, v);
#pragma unroll
    for (int e = 0; e < kE; ++e)
      if (c + e < 0 || c + e >= n) v[e] = -INFINITY;
    return Granule<T>::pack(v);
  }
  // Granule i into the row at `to` of `classes` elements, 0 from n on.
  __device__ __forceinline__ void store_part(T* to, bool aligned, int i, int n, int classes,
                                             uint4 q) const {
    const int c = i * kE - mis;
    float v[kE];
    Granule<T>::unpack(q, v);
#pragma unroll
    for (int e = 0; e < kE; ++e)
      if (c + e >= n) v[e] = 0.f;
    if (aligned && c >= 0 && c + kE <= classes) {
      *reinterpret_cast<uint4*>(to + c) = Granule<T>::pack(v);   // exact: values of T
    } else {
#pragma unroll
      for (int e = 0; e < kE; ++e)
        if (c + e >= 0 && c + e < classes) from_float(v[e], to + c + e);
    }
  }
};

// The elements of a granule less m: 16-bit ones by mixed additions, without a
// conversion before.
template <typename T>
__device__ __forceinline__ void differences(uint4 q, float minus_m, float* d);
template <>
__device__ __forceinline__ void differences<float>(uint4 q, float minus_m, float* d) {
  Granule<float>::unpack(q, d);
#pragma unroll
  for (int e = 0; e < 4; e += 2)
    f2_unpack(f2_add(f2_pack(d[e], d[e + 1]), f2_pack(minus_m, minus_m)), d[e], d[e + 1]);
}
template <>
__device__ __forceinline__ void differences<__nv_bfloat16>(uint4 q, float minus_m, float* d) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    asm("{\n\t.reg .b16 lo, hi;\n\t"
        "mov.b32 {lo, hi}, %2;\n\t"
        "add.f32.bf16 %0, lo, %3;\n\t"
        "add.f32.bf16 %1, hi, %3;\n\t}"
        : "=f"(d[2 * e]), "=f"(d[2 * e + 1])
        : "r"(w[e]), "f"(minus_m));
}
template <>
__device__ __forceinline__ void differences<__half>(uint4 q, float minus_m, float* d) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    asm("{\n\t.reg .b16 lo, hi;\n\t"
        "mov.b32 {lo, hi}, %2;\n\t"
        "add.f32.f16 %0, lo, %3;\n\t"
        "add.f32.f16 %1, hi, %3;\n\t}"
        : "=f"(d[2 * e]), "=f"(d[2 * e + 1])
        : "r"(w[e]), "f"(minus_m));
}

// e^{k d} of two differences.
__device__ __forceinline__ uint64_t exps_of(float d0, float d1, float scale = kLog2e) {
  float x0, x1;
  f2_unpack(f2_mul(f2_pack(d0, d1), f2_pack(scale, scale)), x0, x1);
  return f2_pack(ex2(x0), ex2(x1));
}

// An m of -inf (nothing but -inf so far) counts as 0: its terms are 0 and not NaN.
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }

__device__ __forceinline__ float warp_max(float v, int lanes) {
  for (int off = lanes / 2; off > 0; off >>= 1)
    v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, off));
  return v;
}
__device__ __forceinline__ float warp_sum(float v, int lanes) {
  for (int off = lanes / 2; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
  return v;
}

// (m, s, t) of a part of a row, and the action's logit where it is known.
// Stored 16 bytes at once, also into other CTAs' shared memory: aligned to them.
struct alignas(16) Part {
  float m, s, t, za;
};
static_assert(sizeof(Part) == 16 && alignof(Part) == 16, "one 16-byte store");

// Adds a part to sums whose largest logit is m.
__device__ __forceinline__ void add_part(const Part& h, float m, float* s, float* t,
                                         float scale = kLog2e) {
  if (h.m == -INFINITY && h.s == 0.f) return;             // a NaN sum is taken along
  const float d = h.m - m, x = ex2(d * scale);
  *s = fmaf(h.s, x, *s);
  *t = fmaf(fmaf(h.s, fmaxf(d, kFloor), h.t), x, *t);
}

// A thread's running sums, in pairs: what it has is brought to the new largest logit,
// then the new granules are added.
struct RowSum {
  float m;
  uint64_t s, t;
  __device__ __forceinline__ void clear() {
    m = -INFINITY;
    s = t = 0;
  }
  template <typename T, int kN>
  __device__ __forceinline__ void add(const uint4 (&q)[kN], float scale = kLog2e) {
    constexpr int kE = Granule<T>::kElems;
    float top = m;
#pragma unroll
    for (int u = 0; u < kN; ++u) top = fmaxf(top, Granule<T>::largest(q[u]));
    const float base = base_of(top), d0 = fmaxf(m - base, kFloor), x0 = ex2(d0 * scale);
    const uint64_t x = f2_pack(x0, x0);
    t = f2_mul(f2_fma(s, f2_pack(d0, d0), t), x);
    s = f2_mul(s, x);
    m = top;
#pragma unroll
    for (int u = 0; u < kN; ++u) {
      float d[kE];
      differences<T>(q[u], -base, d);
#pragma unroll
      for (int e = 0; e < kE; e += 2) {
        const uint64_t p = exps_of(d[e], d[e + 1], scale);
        s = f2_add(s, p);
        t = f2_fma(p, f2_pack(fmaxf(d[e], kFloor), fmaxf(d[e + 1], kFloor)), t);
      }
    }
  }
  // The sums of `lanes` lanes, in all of them.
  __device__ __forceinline__ Part over(int lanes, float scale = kLog2e) const {
    float s0, s1, t0, t1;
    f2_unpack(s, s0, s1);
    f2_unpack(t, t0, t1);
    const float top = warp_max(m, lanes);
    const float d = fmaxf(m - base_of(top), kFloor), x = ex2(d * scale);
    const float sum = s0 + s1;
    return {top, warp_sum(sum * x, lanes), warp_sum(fmaf(sum, d, t0 + t1) * x, lanes), 0.f};
  }
};

__device__ __forceinline__ bool same_alignment(const void* a, const void* b) {
  return ((reinterpret_cast<uintptr_t>(a) ^ reinterpret_cast<uintptr_t>(b)) & 15u) == 0;
}

// The row's sums from its kParts parts, in every lane of a warp.
template <int kParts>
__device__ __forceinline__ Part join_parts(const Part* slots, float scale = kLog2e) {
  constexpr int kPer = (kParts + 31) / 32;
  const int lane = threadIdx.x & 31;
  Part h[kPer];
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int at = lane + 32 * i;
    h[i] = at < kParts ? slots[at] : Part{-INFINITY, 0.f, 0.f, 0.f};
    m = fmaxf(m, h[i].m);
  }
  m = warp_max(m, 32);
  float s = 0.f, t = 0.f;
#pragma unroll
  for (int i = 0; i < kPer; ++i) add_part(h[i], m, &s, &t, scale);
  return Part{m, warp_sum(s, 32), warp_sum(t, 32), slots[0].za};
}

// A part into the place `slot` of CTA `cta` of the cluster.
__device__ __forceinline__ void store_part_remote(const Part& x, Part* slot, uint32_t cta) {
  asm volatile(
      "{\n\t.reg .b32 ra;\n\t"
      "mapa.shared::cluster.u32 ra, %0, %1;\n\t"
      "st.shared::cluster.v4.f32 [ra], {%2, %3, %4, %5};\n\t}" ::"r"(smem_u32(slot)),
      "r"(cta), "f"(x.m), "f"(x.s), "f"(x.t), "f"(x.za)
      : "memory");
}

}  // namespace policy
}  // namespace dora
