// Clipped policy losses with their gradients (the PPO update of App. D.2: ratio
// clipped at 1 +- eps), for the two kinds of action that the actor takes:
//   categorical actions      logits of the legal actions (App. A.2: infeasible
//                            budgets are masked before the softmax) to the loss,
//                            its KL and entropy terms and d loss / d logits;
//   ordered removals         Plackett-Luce sequences (App. A.3), selector scores
//                            to the loss and d loss / d scores.
//
// An action of log-probability l under the policy, q when it was taken, q_ref
// under a reference policy, with advantage A and weight w:
//   rho  = exp(l - q),   x = q_ref - l,
//   loss = w [ -min(rho A, clip(rho, 1 - e_lo, 1 + e_hi) A)
//              + beta (exp x - 1 - x) - c H ],
//   g    = d loss / d l = w [ -rho A 1(rho A <= clip(rho) A) + beta (1 - exp x) ]
// (exp x - 1 - x >= 0 is the estimate of KL(pi || pi_ref) from one action).
//
// What bounds them: the categorical loss reads the logits and writes the gradient once
// each.  2048 rows of 32000 bf16 logits, a seventh of them idle, 46 us, 5.2 TB/s (a copy
// 6.8); 4095 x 50001 fp16 163, 4.9; 1024 x 131072 fp32 196, 5.5; 16384 x 2000 bf16 33,
// 4.0; a rollout's 256 x 96 fp32 5, of which the totals are 2.  About a dozen
// instructions an element, two of them exponentials, on warps that wait for one another
// at every row: issue slots are 58% busy where memory is at 75%.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <atomic>

#include "dora.h"
#include "dora_ptx.cuh"
#include "granule.cuh"
#include "token_ops.cuh"
#include "update_ptx.cuh"

namespace dora {
namespace policy {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kTerms = 6;                 // sums over the rows, in the order of `totals`
constexpr int kMaxCtas = 152 * 16;        // partial sums that the workspace holds
constexpr int kThreads = 256;
constexpr int kMaxVisual = 2048;          // visual tokens per image held in shared memory

// A sum as a pair of fp32 values, the second what the first lost (Knuth's two-sum).
// Six fp32 additions where fp64 has one: fp64 sums over the rows took the kernel on
// short rows four times as long as the rows (65536 x 96 fp32: 17 us without, 61 with).
struct Pair {
  float v, lost;
  __device__ __forceinline__ void add(float x) {
    const float t = v + x, b = t - v;
    lost += (v - (t - b)) + (x - b);
    v = t;
  }
  __device__ __forceinline__ void add(Pair o) {
    add(o.v);
    lost += o.lost;
  }
  // What an infinite sum lost is inf - inf.
  __device__ __forceinline__ float rest() const { return isinf(v) ? 0.f : lost; }
  __device__ __forceinline__ float value() const { return v + rest(); }
};
__device__ __forceinline__ Pair shfl_xor(Pair p, int off) {
  return {__shfl_xor_sync(0xffffffffu, p.v, off), __shfl_xor_sync(0xffffffffu, p.lost, off)};
}

struct Workspace {
  unsigned ticket;                        // CTAs done; zero between calls
  unsigned pad[63];
  Pair partial[kMaxCtas][kTerms];
};

// What both losses take per action, and the terms' coefficients.
struct Actions {
  const float* old_logp;
  const float* ref_logp;                  // nullable
  const float* advantages;
  const float* weights;                   // nullable: 1
  float clip_low, clip_high, kl_coef, entropy_coef;
  float* logp;
  float* row_loss;                        // nullable
  float* totals;                          // nullable
  Workspace* ws;                          // used with totals
};

// The terms that a row adds to the totals: loss, policy term, KL, entropy, clipped
// weight, weight.  They are counted by six lanes, each its own.
struct Terms {
  float v[kTerms];
  __device__ __forceinline__ float of(int lane) const {
    float x = v[0];
#pragma unroll
    for (int i = 1; i < kTerms; ++i) x = lane == i ? v[i] : x;
    return lane < kTerms ? x : 0.f;
  }
};
__device__ __forceinline__ Terms all_terms(float x) { return {{x, x, x, x, x, x}}; }

// One row's loss from l - q, x = q_ref - l and the entropy h; returns g.  A NaN
// ratio is left to spread (comparisons, no fmin).  A term of coefficient 0 is not
// multiplied by it: e^x passes fp32's range where x does 88.
__device__ __forceinline__ float row_terms(const Actions& p, float log_ratio, float x, float adv,
                                           float w, float h, Terms* terms) {
  const float ratio = expf(log_ratio);
  const float lo = 1.f - p.clip_low, hi = 1.f + p.clip_high;
  const float cut = (ratio < lo ? lo : (ratio > hi ? hi : ratio)) * adv;
  // an advantage of 0 has no policy term, also where the ratio passes fp32's range
  const float plain = adv == 0.f && ratio == INFINITY ? 0.f : ratio * adv;
  const bool inside = !(plain > cut);
  const float surrogate = -(inside ? plain : cut);
  float g = inside ? -plain : 0.f, kl = 0.f;
  if (p.ref_logp != nullptr) {
    const float em1 = expm1f(x);
    kl = em1 == INFINITY ? em1 : em1 - x;                 // x too is where l is -inf
    if (p.kl_coef != 0.f) g = fmaf(-p.kl_coef, em1, g);
  }
  float row = surrogate;
  if (p.kl_coef != 0.f) row = fmaf(p.kl_coef, kl, row);
  if (p.entropy_coef != 0.f) row = fmaf(-p.entropy_coef, h, row);
  *terms = Terms{{w * row, w * surrogate, w * kl, w * h, inside ? 0.f : w, w}};
  return g * w;
}

// Two terms of a CTA that is done.
__device__ __forceinline__ float4 load_terms(const Workspace* ws, int cta, int i) {
  return __ldcg(reinterpret_cast<const float4*>(ws->partial[cta]) + i);
}

// The totals.  Lanes i < kTerms of a CTA's first warp hold its sum of term i.  It goes
// to the CTA's place in the workspace; the CTA that is last adds all of them in the
// order of the CTAs, so that the totals do not depend on which one that is, and leaves
// the ticket at zero for the next call.
template <int kWarps>
__device__ __forceinline__ void finish_totals(const Actions& p, Pair sum) {
  if (p.totals == nullptr) return;
  if (gridDim.x == 1) {
    if (threadIdx.x < kTerms) p.totals[threadIdx.x] = sum.value();
    return;
  }
  __shared__ bool last;
  Workspace* ws = p.ws;
  if (threadIdx.x < 32) {
    if (threadIdx.x < kTerms) ws->partial[blockIdx.x][threadIdx.x] = sum;
    __syncwarp();
    if (threadIdx.x == 0) last = take_ticket(&ws->ticket) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  constexpr int kLoads = 3, kBatch = 3;   // a CTA's terms are three 16-byte loads
  static_assert(kTerms == 2 * kLoads, "two pairs a load");
  constexpr int threads = kWarps * 32;
  const int lane = threadIdx.x & 31, ctas = gridDim.x;
  Pair t[kTerms];
#pragma unroll
  for (int i = 0; i < kTerms; ++i) t[i] = Pair{0.f, 0.f};
  for (int first = threadIdx.x; first < ctas; first += kBatch * threads) {
    float4 x[kBatch][kLoads];             // all on their way before the first is added
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        x[u][i] = first + u * threads < ctas ? load_terms(ws, first + u * threads, i)
                                             : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        t[2 * i].add(Pair{x[u][i].x, x[u][i].y});
        t[2 * i + 1].add(Pair{x[u][i].z, x[u][i].w});
      }
  }
  __shared__ Pair warps[kWarps][kTerms];
#pragma unroll
  for (int i = 0; i < kTerms; ++i) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) t[i].add(shfl_xor(t[i], off));
    if (lane == 0) warps[threadIdx.x >> 5][i] = t[i];
  }
  __syncthreads();
  if (threadIdx.x < kTerms) {
    Pair all = warps[0][threadIdx.x];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) all.add(warps[w][threadIdx.x]);
    p.totals[threadIdx.x] = all.value();
  }
  if (threadIdx.x == 0) ws->ticket = 0;
}

// ---------------------------------------------------------------------------
// Categorical actions.  A row is read once, as 16-byte granules, by a group of lanes,
// a CTA or a cluster of CTAs; from there come its sums and its gradient.  With m the
// largest logit, d_j = z_j - m and e_j = e^{d_j} (the difference first: the largest has
// e = 1 to the last bit, and an action that is certain log-probability and gradient 0):
//   s = sum e_j,  t = sum e_j d_j,
//   l = (z_a - m) - ln s,  H = ln s - t / s,  p_j = e_j / s,
//   d loss / d z_j = g (1(j = a) - p_j) + w c_H p_j (log p_j + H)
//                  = e_j (a + b d_j) + g 1(j = a).
// Rows start at any alignment: granules are aligned in memory, `mis` elements of
// the first belong to what lies before the row, and a granule that is not wholly
// inside is loaded and stored by its elements.
// ---------------------------------------------------------------------------
template <typename T>
struct Rows {
  const T* logits;
  T* grad;                                // nullable; may be logits
  int64_t ld;
  int rows, classes;
  const int32_t* legal;                   // nullable: classes
  const int32_t* actions;
  float* entropy;                         // nullable
  int32_t* status;
};

// A row's action, weight and legal logits as they are loaded, a row or two ahead:
// nothing is made of them before their row's turn, so that no warp waits for them.
struct RowAhead {
  int action, n;
  float w;
};
template <typename T>
__device__ __forceinline__ RowAhead row_ahead(const Rows<T>& r, const Actions& p, int row) {
  RowAhead a = {-1, 0, 1.f};
  if (row < r.rows) {
    a.action = r.actions[row];
    a.n = r.legal != nullptr ? r.legal[row] : r.classes;
    if (p.weights != nullptr) a.w = p.weights[row];
  }
  return a;
}

// Whether a row takes part, and how many of its logits are legal (-1: not valid).
struct RowUse {
  int action, n;
  bool takes;
};
template <typename T>
__device__ __forceinline__ RowUse row_use(const Rows<T>& r, const RowAhead& a) {
  const bool valid = a.n >= 0 && a.n <= r.classes && a.action < a.n;
  return {a.action, valid ? a.n : -1, a.action >= 0 && a.w != 0.f};
}
__device__ __forceinline__ bool computed(const RowUse& u) { return u.takes && u.n > 0; }

// The other scalars of a row that takes part.
struct RowIn {
  float w, old_logp, adv, ref;
};
__device__ __forceinline__ RowIn row_in(const Actions& p, int row, int rows) {
  if (row >= rows) return {0.f, 0.f, 0.f, 0.f};
  return {p.weights != nullptr ? p.weights[row] : 1.f, p.old_logp[row], p.advantages[row],
          p.ref_logp != nullptr ? p.ref_logp[row] : 0.f};
}

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

// e^d of two differences.
__device__ __forceinline__ uint64_t exps_of(float d0, float d1) {
  float x0, x1;
  f2_unpack(f2_mul(f2_pack(d0, d1), f2_pack(kLog2e, kLog2e)), x0, x1);
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
__device__ __forceinline__ void add_part(const Part& h, float m, float* s, float* t) {
  if (h.m == -INFINITY && h.s == 0.f) return;             // a NaN sum is taken along
  const float d = h.m - m, x = ex2(d * kLog2e);
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
  __device__ __forceinline__ void add(const uint4 (&q)[kN]) {
    constexpr int kE = Granule<T>::kElems;
    float top = m;
#pragma unroll
    for (int u = 0; u < kN; ++u) top = fmaxf(top, Granule<T>::largest(q[u]));
    const float base = base_of(top), d0 = fmaxf(m - base, kFloor), x0 = ex2(d0 * kLog2e);
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
        const uint64_t p = exps_of(d[e], d[e + 1]);
        s = f2_add(s, p);
        t = f2_fma(p, f2_pack(fmaxf(d[e], kFloor), fmaxf(d[e + 1], kFloor)), t);
      }
    }
  }
  // The sums of `lanes` lanes, in all of them.
  __device__ __forceinline__ Part over(int lanes) const {
    float s0, s1, t0, t1;
    f2_unpack(s, s0, s1);
    f2_unpack(t, t0, t1);
    const float top = warp_max(m, lanes);
    const float d = fmaxf(m - base_of(top), kFloor), x = ex2(d * kLog2e);
    const float sum = s0 + s1;
    return {top, warp_sum(sum * x, lanes), warp_sum(fmaf(sum, d, t0 + t1) * x, lanes), 0.f};
  }
};

// What the gradient of a row needs.
struct RowGrad {
  float m, a, b, at_action;               // e^{z - m} (a + b (z - m)); the action's own
};

template <typename T, bool kEntropy>
__device__ __forceinline__ uint4 grad_granule(uint4 q, const RowGrad& k) {
  constexpr int kE = Granule<T>::kElems;
  float d[kE];
  differences<T>(q, -k.m, d);
  const uint64_t a = f2_pack(k.a, k.a), b = f2_pack(k.b, k.b);
#pragma unroll
  for (int e = 0; e < kE; e += 2) {
    const uint64_t p = exps_of(d[e], d[e + 1]);
    const uint64_t f =
        kEntropy ? f2_fma(f2_pack(fmaxf(d[e], kFloor), fmaxf(d[e + 1], kFloor)), b, a) : a;
    f2_unpack(f2_mul(p, f), d[e], d[e + 1]);
  }
  return Granule<T>::pack(d);
}
template <typename T>
__device__ __forceinline__ uint4 grad_granule(uint4 q, const RowGrad& k) {
  return k.b == 0.f ? grad_granule<T, false>(q, k) : grad_granule<T, true>(q, k);
}

// The row's outputs, its terms and what its gradient needs, from the row's sums and
// the action's logit; `leader` writes.
template <typename T>
__device__ __forceinline__ RowGrad finish_row(const Rows<T>& r, const Actions& p, const RowIn& in,
                                              int row, float za, const Part& x, bool leader,
                                              Terms* terms) {
  const float ls = logf(x.s), inv = 1.f / x.s, h = fmaf(-x.t, inv, ls);
  const float da = za - x.m, lp = da - ls;
  const float g = row_terms(p, lp - in.old_logp, in.ref - lp, in.adv, in.w, h, terms);
  if (leader) {
    p.logp[row] = lp;
    if (r.entropy != nullptr) r.entropy[row] = h;
    if (p.row_loss != nullptr) p.row_loss[row] = terms->v[0];
  }
  const float cw = in.w * p.entropy_coef;
  const float a = (cw * (h - ls) - g) * inv, b = cw * inv;
  return RowGrad{x.m, a, b, fmaf(ex2(da * kLog2e), fmaf(b, fmaxf(da, kFloor), a), g)};
}

template <typename T>
__device__ __forceinline__ void write_row(const Rows<T>& r, const Actions& p, int row,
                                          float fill) {
  p.logp[row] = fill;
  if (r.entropy != nullptr) r.entropy[row] = fill;
  if (p.row_loss != nullptr) p.row_loss[row] = fill;
}
// The outputs of a row that takes no part (0) or is not valid (NaN).
template <typename T>
__device__ __forceinline__ void fill_row(const Rows<T>& r, const Actions& p, int row, float fill) {
  if (fill != 0.f) record_status(r.status, DORA_ERR_DEVICE_BAD_COUNT);
  write_row(r, p, row, fill);
}

template <typename T>
__device__ __forceinline__ void fill_granule(const RowPtr<T>& z, T* dz, bool aligned, int i,
                                             int classes, float fill) {
  float v[Granule<T>::kElems];
#pragma unroll
  for (int e = 0; e < Granule<T>::kElems; ++e) v[e] = fill;
  z.store_part(dz, aligned, i, classes, classes, Granule<T>::pack(v));
}

__device__ __forceinline__ bool same_alignment(const void* a, const void* b) {
  return ((reinterpret_cast<uintptr_t>(a) ^ reinterpret_cast<uintptr_t>(b)) & 15u) == 0;
}

// Short rows: kLanes lanes of a warp hold one, kHeld granules each (65536 x 96 fp32 14 us,
// 3.6 TB/s; 16384 x 1000 bf16 16, 4.0; 16384 x 2000 33, 4.0; 8192 x 4096 38, 3.5): no
// barrier, and what a row costs besides its elements is paid by one warp.
template <typename T, int kLanes, int kHeld>
__global__ void __launch_bounds__(kThreads) policy_warp_kernel(Rows<T> r, Actions p) {
  constexpr int kRowsPerCta = kThreads / kLanes;
  pdl_wait();
  const int lane = threadIdx.x % kLanes;
  const int step = gridDim.x * kRowsPerCta;
  Pair sum = {0.f, 0.f};
  // the loop is the same for all groups of a warp: shuffles need every lane
  const int first = blockIdx.x * kRowsPerCta + (threadIdx.x / 32) * (32 / kLanes);
  int row = first + (threadIdx.x % 32) / kLanes;
  RowAhead next = row_ahead(r, p, row);
  for (int base = first; base < r.rows; base += step, row += step) {
    const RowUse use = row_use(r, next);
    const bool exists = row < r.rows, live = computed(use);
    const int n = live ? use.n : 0;
    const RowPtr<T> z(r.logits + (exists ? row : 0) * r.ld, n);
    uint4 q[kHeld];
#pragma unroll
    for (int u = 0; u < kHeld; ++u) q[u] = z.load(lane + u * kLanes, n);
    RowIn in = {0.f, 0.f, 0.f, 0.f};
    float za = 0.f;
    if (live) {
      in = row_in(p, row, r.rows);
      za = to_float(z.z[use.action]);
    }
    next = row_ahead(r, p, row + step);
    RowSum x;
    x.clear();
    constexpr int kStep = kHeld < 4 ? kHeld : 4;
#pragma unroll
    for (int u = 0; u < kHeld; u += kStep) {
      uint4 some[kStep];
#pragma unroll
      for (int v = 0; v < kStep; ++v) some[v] = q[u + v];
      // legal logits may end long before the classes do
      if (kHeld <= 4 || lane + u * kLanes < z.some_hi) x.add<T>(some);
    }
    const Part part = x.over(kLanes);
    __syncwarp();                         // every lane has read its logits: grad may be logits
    if (exists) {
      T* dz = r.grad != nullptr ? r.grad + row * r.ld : nullptr;
      const bool aligned = dz != nullptr && same_alignment(dz, z.z);
      const int end = z.granules(r.classes);
      if (live) {
        Terms terms;
        const RowGrad k = finish_row(r, p, in, row, za, part, lane == 0, &terms);
        sum.add(terms.of(lane));
        if (dz != nullptr) {
#pragma unroll
          for (int u = 0; u < kHeld; ++u) {
            const int i = lane + u * kLanes;
            if (i >= end) continue;
            const uint4 v = grad_granule<T>(q[u], k);
            if (aligned && z.whole(i)) *(z.as_granules(dz) + i) = v;
            else z.store_part(dz, aligned, i, n, r.classes, v);
          }
          // the lane that has stored the action's granule
          if (((use.action + z.mis) / z.kE) % kLanes == lane)
            from_float(k.at_action, dz + use.action);
        }
      } else {
        const float fill = use.takes ? NAN : 0.f;
        if (lane == 0) fill_row(r, p, row, fill);
        sum.add(all_terms(fill).of(lane));
        if (dz != nullptr)
          for (int i = lane; i < end; i += kLanes) fill_granule(z, dz, aligned, i, r.classes, fill);
      }
    }
  }
  if (p.totals == nullptr) return;
  // lane i of every group holds its term i: groups of a warp, then warps
  __shared__ Pair all[kThreads / 32][kTerms];
#pragma unroll
  for (int off = 16; off >= kLanes; off >>= 1) sum.add(shfl_xor(sum, off));
  if ((threadIdx.x & 31) < kTerms) all[threadIdx.x >> 5][threadIdx.x & 31] = sum;
  __syncthreads();
  if (threadIdx.x < kTerms)
#pragma unroll
    for (int k = 1; k < kThreads / 32; ++k) sum.add(all[k][threadIdx.x]);
  finish_totals<kThreads / 32>(p, sum);
}

// The row's sums from its kParts parts, in every lane of a warp.
template <int kParts>
__device__ __forceinline__ Part join_parts(const Part* slots) {
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
  for (int i = 0; i < kPer; ++i) add_part(h[i], m, &s, &t);
  return Part{m, warp_sum(s, 32), warp_sum(t, 32), slots[0].za};
}

// Middling rows: a CTA holds one, kHeld granules a thread, and as many CTAs share an SM
// as registers allow, so that one's loads cover another's barrier (8192 x 6000 bf16
// 46 us, 4.3 TB/s; 4096 x 8000 fp32 45, 5.8).
template <typename T, int kBlock, int kHeld>
__global__ void __launch_bounds__(kBlock, 1024 / kBlock)
    policy_cta_kernel(Rows<T> r, Actions p) {
  constexpr int kWarps = kBlock / 32, kStep = 4;
  static_assert(kHeld % kStep == 0, "granules are added four at a time");
  __shared__ Part slots[2][kWarps];
  pdl_wait();
  const int me = threadIdx.x, warp = me >> 5;
  int parity = 0;
  Pair sum = {0.f, 0.f};
  int row = blockIdx.x;
  RowAhead next = row_ahead(r, p, row);
  for (; row < r.rows; row += gridDim.x) {
    const RowUse use = row_use(r, next);
    const RowPtr<T> z(r.logits + row * r.ld, use.n);
    T* dz = r.grad != nullptr ? r.grad + row * r.ld : nullptr;
    const bool aligned = dz != nullptr && same_alignment(dz, z.z);
    const int n = use.n, end = z.granules(r.classes);
    if (computed(use)) {
      uint4 q[kHeld];
#pragma unroll
      for (int u = 0; u < kHeld; ++u) q[u] = z.load(me + u * kBlock, n);
      const RowIn in = row_in(p, row, r.rows);
      const float za = to_float(z.z[use.action]);
      next = row_ahead(r, p, row + gridDim.x);
      RowSum x;
      x.clear();
#pragma unroll
      for (int u = 0; u < kHeld; u += kStep) {
        const uint4 some[kStep] = {q[u], q[u + 1], q[u + 2], q[u + 3]};
        if (me + u * kBlock < z.some_hi) x.add<T>(some);
      }
      Part part = x.over(32);
      if ((me & 31) == 0) slots[parity][warp] = part;
      // after this barrier every logit of the row has been read: grad may be logits;
      // places alternate, so that a warp that is a row ahead writes where nobody reads
      __syncthreads();
      part = join_parts<kWarps>(slots[parity]);
      parity ^= 1;
      Terms terms;
      const RowGrad k = finish_row(r, p, in, row, za, part, me == 0, &terms);
      sum.add(terms.of(me));
      if (dz == nullptr) continue;
#pragma unroll
      for (int u = 0; u < kHeld; ++u) {
        const int i = me + u * kBlock;
        if (i >= end) continue;
        if (aligned && z.whole(i)) *(z.as_granules(dz) + i) = grad_granule<T>(q[u], k);
        else z.store_part(dz, aligned, i, n, r.classes, grad_granule<T>(q[u], k));
      }
      // the thread that has stored the action's granule
      if (((use.action + z.mis) / z.kE) % kBlock == me) from_float(k.at_action, dz + use.action);
    } else {
      next = row_ahead(r, p, row + gridDim.x);
      const float fill = use.takes ? NAN : 0.f;
      if (me == 0) fill_row(r, p, row, fill);
      sum.add(all_terms(fill).of(me));
      if (dz != nullptr)
        for (int i = me; i < end; i += kBlock) fill_granule(z, dz, aligned, i, r.classes, fill);
    }
  }
  finish_totals<kWarps>(p, sum);
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

// Longer rows: kCtas CTAs (a cluster when there are several) hold one, an equal part
// each, in a ring of kStages stages of shared memory (more, where they fit, changed
// nothing).  Four kinds of warps, so that a row's steps, which wait for one another,
// run beside those of the rows before and after it:
//   warp 2            fills the stages: one bulk copy of a row's whole granules;
//   kSumWarps         sum their granules and leave the parts to warp 0 or 1;
//   warps 0 and 1     take every other row each: join the CTA's parts, send the CTA's
//                     own to every CTA of the cluster, join those, finish the row's
//                     scalars and hand the gradient's coefficients to
//   kGradWarps        which write the gradient and free the stage.
// (One kind of warp that sums row i and then writes the gradient of row i - 1 took
// 48 us for 2048 x 32000 bf16 and 179 for 4096 x 50000 fp16: a row costs a warp about a
// microsecond besides its granules, of which nothing was hidden.)
// Between CTAs only the joining warps speak: an arrival that others may read behind
// waits for all that its thread has stored, and other warps have gradients on their way.
// Within a CTA two places for the parts are enough: a warp leaves those of row i + 2
// once those of row i are taken.  The cluster's need four, two a joining warp: a warp
// that has row i + 2 does not know whether the other CTAs have read row i, only that
// they have sent it; one that has row i + 4 has had row i + 2 from every CTA's own warp,
// which sends it when it is done with row i.
//
// A wait is bounded.  Where one runs out, its warp is out of step with the others and
// with the other CTAs, which may take one row's parts for another's.  The rows carry on
// as they are, at a wait's first look each, and at the end all of the cluster's become
// NaN, so that no call without a status word takes them for results.
template <typename T, int kSumWarps, int kGradWarps, int kStage, int kCtas>
__global__ void __launch_bounds__((3 + kSumWarps + kGradWarps) * 32, 1)
    policy_ring_kernel(Rows<T> r, Actions p) {
  constexpr int kStages = 3, kPlaces = 4;
  extern __shared__ __align__(128) uint4 ring[];
  __shared__ Part slots[2][kSumWarps], ctas[kPlaces][kCtas];
  __shared__ RowGrad grads[2];
  __shared__ uint64_t full[kStages], empty[kStages], summed[2], joined[kPlaces], ready[2], taken[2];
  __shared__ int abort;
  const int rank = kCtas > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int step = gridDim.x / kCtas, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    abort = 0;
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], kGradWarps);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&summed[s], kSumWarps);
      mbar_init(&ready[s], 1);
      mbar_init(&taken[s], kGradWarps);
    }
    for (int s = 0; s < kPlaces; ++s) mbar_init(&joined[s], kCtas);
    fence_barrier_init();
  }
  if (kCtas > 1) cluster_sync();          // the others' barriers are there to be written
  else __syncthreads();
  pdl_wait();

  // The copied granules [from, to) of this CTA's [lo, hi): all that hold some of the
  // row's legal logits, and with them a few of its neighbours' (looked at by nobody),
  // but nothing before the first row's or past the last one's logits.
  const T* last = r.logits + (r.rows - 1) * r.ld + r.classes;
  auto copied = [&](const RowPtr<T>& z, int row, int lo, int hi, int* from, int* to) {
    *from = max(lo, row == 0 ? z.whole_lo : 0);
    *to = min(hi, z.z - z.mis + z.some_hi * z.kE <= last ? z.some_hi : z.whole_hi);
  };
  // granules [lo, hi) of a row are this CTA's
  auto bounds = [&](const RowPtr<T>& z, int* lo, int* hi) {
    const int all = z.granules(r.classes), per = (all + kCtas - 1) / kCtas;
    *lo = min(rank * per, all);
    *hi = min(*lo + per, all);
  };
  auto wait = [&](uint64_t* bar, int phase) {
    if (!mbar_wait(bar, phase & 1, &abort)) record_status(r.status, DORA_ERR_TIMEOUT);
  };
  // Whether the row's first granule (it starts inside it), or its last with legal logits
  // (they end inside it), is this CTA's: thread 0 and thread 1 of a kind see to them.
  auto is_part = [](const RowPtr<T>& z, int me, int lo, int hi) {
    if (me == 0) return lo == 0 && z.whole_lo > 0;
    return z.whole_hi < z.some_hi && z.whole_hi >= max(lo, z.whole_lo) && z.whole_hi < hi;
  };
  auto part_of = [&](const RowPtr<T>& z, int row, int lo, int hi, int i, int n,
                     const uint4* held) {
    int from, to;
    copied(z, row, lo, hi, &from, &to);
    return i >= from && i < to ? z.only_row(held[i], i, n) : z.load_part(i, n);
  };
  Pair sum = {0.f, 0.f};
  int row = blockIdx.x / kCtas;
  int stage = 0, lap = 0, count = 0;      // of the rows that are computed
  auto advance = [&]() {
    ++count;
    if (++stage == kStages) {
      stage = 0;
      ++lap;
    }
  };
  RowAhead next = row_ahead(r, p, row);

  if (warp == 2) {
    if (lane == 0) {
      for (; row < r.rows; row += step) {
        const RowUse use = row_use(r, next);
        next = row_ahead(r, p, row + step);
        if (!computed(use)) continue;
        const RowPtr<T> z(r.logits + row * r.ld, use.n);
        int lo, hi, from, to;
        bounds(z, &lo, &hi);
        copied(z, row, lo, hi, &from, &to);
        if (lap > 0) wait(&empty[stage], lap - 1);
        // warps that have given up waiting for a stage leave it too: no copy then, whose
        // bytes would count for a phase that is not theirs
        if (abort) break;
#ifdef DORA_TEST_WITHHOLD_ROW_LOAD
        // timeout-path test library only: the first CTA's second row is never copied nor
        // its bytes expected, so that the waits for it run out with no copy in flight
        if (blockIdx.x == 0 && count == 1) {
          advance();
          continue;
        }
#endif
        if (to > from) {
          mbar_arrive_expect_tx(&full[stage], (to - from) * 16);
          bulk_load(ring + stage * kStage + (from - lo), z.at(from), (to - from) * 16,
                    &full[stage]);
        } else {
          mbar_arrive(&full[stage]);
        }
        advance();
      }
      for (int s = 0; s < kStages; ++s)   // no copy may land after the CTA is gone
        mbar_wait_limited(&full[s], (s < stage ? lap : lap - 1) & 1, kWaitLimitNs / 8);
    }
  } else if (warp < 2) {
    const bool leader = rank == 0 && lane == 0;
    RowIn in = row_in(p, row, r.rows);
    for (; row < r.rows; row += step) {
      const RowUse use = row_use(r, next);
      next = row_ahead(r, p, row + step);
      const RowIn next_in = row_in(p, row + step, r.rows);
      if (computed(use)) {
        const int slot = count & 1, phase = count >> 1;
        if (slot == warp) {
          wait(&summed[slot], phase);
          __syncwarp();
          Part x = join_parts<kSumWarps>(slots[slot]);
          if (kCtas > 1) {
            const int place = count % kPlaces;
            if (lane < kCtas) {
              store_part_remote(x, &ctas[place][rank], lane);
              mbar_arrive_remote(&joined[place], lane);
            }
            if (!mbar_wait_cluster(&joined[place], count / kPlaces & 1, &abort))
              record_status(r.status, DORA_ERR_TIMEOUT);
            __syncwarp();
            x = join_parts<kCtas>(ctas[place]);
          }
          Terms terms;
          const RowGrad k = finish_row(r, p, in, row, x.za, x, leader, &terms);
          // the coefficients before the last ones have been taken
          if (count >= 2) wait(&taken[slot], phase - 1);
          __syncwarp();
          if (lane == 0) {
            grads[slot] = k;
            mbar_arrive(&ready[slot]);
          }
          if (rank == 0) sum.add(terms.of(lane));
        }
        ++count;
      } else if (warp == 0) {
        const float fill = use.takes ? NAN : 0.f;
        if (leader) fill_row(r, p, row, fill);
        if (rank == 0) sum.add(all_terms(fill).of(lane));
      }
      in = next_in;
    }
  } else if (warp < 3 + kSumWarps) {
    constexpr int kSum = kSumWarps * 32;
    const int me = threadIdx.x - 96;
    // The action's logit goes with the first warp's part: read before any CTA can write
    // the row's gradient, which may lie over its logits.  It and the row's scalars are
    // on their way a row and two rows ahead.
    auto action_logit = [&](int at, const RowUse& u) {
      T z;
      from_float(0.f, &z);
      if (warp == 3 && computed(u)) z = r.logits[at * r.ld + u.action];
      return z;
    };
    RowUse use = row_use(r, next);
    next = row_ahead(r, p, row + step);
    T za = action_logit(row, use);
    for (; row < r.rows; row += step) {
      const RowUse next_use = row_use(r, next);
      next = row_ahead(r, p, row + 2 * step);
      const T next_za = action_logit(row + step, next_use);
      if (computed(use)) {
        const RowPtr<T> z(r.logits + row * r.ld, use.n);
        int lo, hi;
        bounds(z, &lo, &hi);
        const int n = use.n, from = max(lo, z.whole_lo), to = min(hi, z.whole_hi);
        const uint4* held = ring + stage * kStage - lo;
        RowSum x;
        x.clear();
        wait(&full[stage], lap);
        int i = from + me;
        for (; i + 3 * kSum < to; i += 4 * kSum) {
          const uint4 q[4] = {held[i], held[i + kSum], held[i + 2 * kSum], held[i + 3 * kSum]};
          x.add<T>(q);
        }
        for (; i < to; i += kSum) {
          const uint4 q[1] = {held[i]};
          x.add<T>(q);
        }
        if (me < 2 && is_part(z, me, lo, hi)) {
          i = me == 0 ? 0 : z.whole_hi;
          const uint4 q[1] = {part_of(z, row, lo, hi, i, n, held)};
          x.add<T>(q);
        }
        Part part = x.over(32);
        part.za = to_float(za);
        const int slot = count & 1;
        if (count >= 2) wait(&ready[slot], (count >> 1) - 1);   // the last ones are taken
        if (lane == 0) {
          slots[slot][warp - 3] = part;
          mbar_arrive(&summed[slot]);
        }
        advance();
      }
      use = next_use;
      za = next_za;
    }
  } else {
    constexpr int kGrad = kGradWarps * 32;
    const int me = threadIdx.x - 96 - kSumWarps * 32;
    for (; row < r.rows; row += step) {
      const RowUse use = row_use(r, next);
      next = row_ahead(r, p, row + step);
      const RowPtr<T> z(r.logits + row * r.ld, use.n);
      T* dz = r.grad != nullptr ? r.grad + row * r.ld : nullptr;
      const bool aligned = dz != nullptr && same_alignment(dz, z.z);
      int lo, hi;
      bounds(z, &lo, &hi);
      if (computed(use)) {
        const int n = use.n, from = max(lo, z.whole_lo), to = min(hi, z.whole_hi);
        const uint4* held = ring + stage * kStage - lo;
        wait(&full[stage], lap);
        wait(&ready[count & 1], count >> 1);
        const RowGrad k = grads[count & 1];
        __syncwarp();
        if (lane == 0) mbar_arrive(&taken[count & 1]);
        if (dz != nullptr) {
          int i = from + me;
          if (aligned) {
            uint4* out = z.as_granules(dz);
            if (k.b == 0.f) {
#pragma unroll 2
              for (; i < to; i += kGrad) out[i] = grad_granule<T, false>(held[i], k);
            } else {
#pragma unroll 2
              for (; i < to; i += kGrad) out[i] = grad_granule<T, true>(held[i], k);
            }
          } else {
            for (; i < to; i += kGrad)
              z.store_part(dz, false, i, n, r.classes, grad_granule<T>(held[i], k));
          }
          // the granules that are not whole, and those past the legal logits
          i = me == 0 ? 0 : z.whole_hi;
          if (me < 2 && is_part(z, me, lo, hi))
            z.store_part(dz, aligned, i, n, r.classes,
                         grad_granule<T>(part_of(z, row, lo, hi, i, n, held), k));
          for (i = max(lo, z.some_hi) + me; i < hi; i += kGrad)
            fill_granule(z, dz, aligned, i, r.classes, 0.f);
          // the thread that has stored the action's granule
          const int ia = (use.action + z.mis) / z.kE;
          const int owner = ia < z.whole_lo ? 0 : ia < z.whole_hi ? (ia - from) % kGrad : 1;
          if (ia >= lo && ia < hi && owner == me) from_float(k.at_action, dz + use.action);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&empty[stage]);
        advance();
      } else if (dz != nullptr) {
        const float fill = use.takes ? NAN : 0.f;
        for (int i = lo + me; i < hi; i += kGrad)
          fill_granule(z, dz, aligned, i, r.classes, fill);
      }
    }
  }
  __shared__ Pair odd[kTerms];            // of warp 1's rows
  if (warp == 1 && lane < kTerms) odd[lane] = sum;
  __syncthreads();
  if (kCtas > 1) {
    if (abort != 0 && threadIdx.x < kCtas) store_remote(1, &abort, threadIdx.x);
    __syncwarp();
    cluster_sync();                       // nobody leaves while parts may be on their way to it
  }
  if (threadIdx.x < kTerms) sum.add(odd[threadIdx.x]);
  if (abort != 0) {
    for (row = blockIdx.x / kCtas; row < r.rows; row += step) {
      const RowUse use = row_use(r, row_ahead(r, p, row));
      if (!computed(use)) continue;
      const RowPtr<T> z(r.logits + row * r.ld, use.n);
      T* dz = r.grad != nullptr ? r.grad + row * r.ld : nullptr;
      int lo, hi;
      bounds(z, &lo, &hi);
      if (rank == 0 && threadIdx.x == 0) write_row(r, p, row, NAN);
      if (dz != nullptr)
        for (int i = lo + static_cast<int>(threadIdx.x); i < hi; i += blockDim.x)
          fill_granule(z, dz, same_alignment(dz, z.z), i, r.classes, NAN);
    }
    if (rank == 0) sum.add(all_terms(NAN).of(threadIdx.x));
  }
  finish_totals<3 + kSumWarps + kGradWarps>(p, sum);
}

// Rows longer than eight CTAs' rings: eight CTAs a row without one, which read it a
// second time (from L2, where the clusters' rows fit) for its gradient: 128 x 400000
// bf16, a seventh of them idle, 58 us, 3.0 TB/s of the two passes that it needs (26 at
// a copy's rate).
constexpr int kLongBlock = 512, kLongCtas = 8, kLongStep = 4;

template <typename T>
__global__ void __launch_bounds__(kLongBlock, 2) policy_long_kernel(Rows<T> r, Actions p) {
  constexpr int kWarps = kLongBlock / 32, kStride = kLongBlock * kLongCtas;
  __shared__ Part slots[2][kWarps * kLongCtas];
  cluster_sync();                         // the others' shared memory is there to be written
  pdl_wait();
  const int rank = static_cast<int>(cluster_ctarank());
  const int step = gridDim.x / kLongCtas;
  const int g0 = rank * kLongBlock + threadIdx.x;
  const bool leader = rank == 0 && threadIdx.x == 0;
  int parity = 0;
  Pair sum = {0.f, 0.f};
  for (int row = blockIdx.x / kLongCtas; row < r.rows; row += step) {
    const RowUse use = row_use(r, row_ahead(r, p, row));
    const RowPtr<T> z(r.logits + row * r.ld, use.n);
    T* dz = r.grad != nullptr ? r.grad + row * r.ld : nullptr;
    const bool aligned = dz != nullptr && same_alignment(dz, z.z);
    const int end = z.granules(r.classes);
    if (computed(use)) {
      const int n = use.n;
      const RowIn in = row_in(p, row, r.rows);
      const float za = to_float(z.z[use.action]);
      RowSum x;
      x.clear();
      for (int i = g0; i < end; i += kStride * kLongStep) {
        uint4 q[kLongStep];
#pragma unroll
        for (int u = 0; u < kLongStep; ++u) q[u] = z.load(i + u * kStride, n);
        x.add<T>(q);
      }
      Part part = x.over(32);
      // every warp's part goes to every CTA; places alternate from row to row, so that a
      // warp that is a row ahead writes where nobody reads
      if ((threadIdx.x & 31) < kLongCtas)
        store_part_remote(part, slots[parity] + rank * kWarps + (threadIdx.x >> 5),
                          threadIdx.x & 31);
      // after this barrier every logit of the row has been read: grad may be logits
      cluster_sync();
      part = join_parts<kWarps * kLongCtas>(slots[parity]);
      parity ^= 1;
      Terms terms;
      const RowGrad k = finish_row(r, p, in, row, za, part, leader, &terms);
      if (rank == 0) sum.add(terms.of(threadIdx.x));
      if (dz != nullptr) {
        for (int i = g0; i < end; i += kStride) {
          if (aligned && z.whole(i))
            *(z.as_granules(dz) + i) = grad_granule<T>(*z.at(i), k);
          else
            z.store_part(dz, aligned, i, n, r.classes,
                         grad_granule<T>(z.whole(i) ? *z.at(i) : z.load_part(i, n), k));
        }
        // the thread that has stored the action's granule
        if (((use.action + z.mis) / z.kE) % kStride == g0)
          from_float(k.at_action, dz + use.action);
      }
    } else {
      const float fill = use.takes ? NAN : 0.f;
      if (leader) fill_row(r, p, row, fill);
      if (rank == 0) sum.add(all_terms(fill).of(threadIdx.x));
      if (dz != nullptr)
        for (int i = g0; i < end; i += kStride) fill_granule(z, dz, aligned, i, r.classes, fill);
    }
  }
  finish_totals<kWarps>(p, sum);
}

// ---------------------------------------------------------------------------
// Ordered removals.  With M the image's largest score, e_j = e^{s_j - M}, and
//   S_t = sum of e over the tokens not removed before step t   (suffix sums)
//   Q_t = sum_{u <= t} 1 / S_u                                 (prefix sums)
//   l = sum_t (s_{i_t} - M) - ln S_t,
//   d l / d s_j = 1(j removed) - e_j Q_{u_j}, u_j its step, k for a token that stays:
// both scans only add, and cost one exponential a token.  Scores that lie further
// apart than kRange would underflow: such an image's sums are kept as pairs (m, s) for
// s e^m, each with a maximum of its own, at two exponentials an addition.
//
// One CTA an image, a thread an equal run of steps.  An image takes the time of its
// chain (boundaries, scores, order, two scans, five barriers), so the CTAs are small,
// and the grid is what is resident at once, seven CTAs an SM by their shared memory: 256
// images of 197 tokens, up to 60 removed, 6 us, 1024 of 577, up to 120 removed, 10, of
// which the totals are 2 and 4; 1200 of 577 12.2 (13.1 with a grid of eight an SM).
// ---------------------------------------------------------------------------
constexpr int kSeqThreads = 128, kSeqWarps = kSeqThreads / 32, kSeqPerSm = 7;
constexpr float kRange = 80.f;            // e^-kRange and its reciprocal are far from fp32's ends

struct Scaled {                           // s e^m
  float m, s;
};
__device__ __forceinline__ Scaled plus(Scaled a, Scaled b) {
  if (a.s == 0.f) return b;
  if (b.s == 0.f) return a;
  const float m = fmaxf(a.m, b.m);
  return {m, a.s * expf(a.m - m) + b.s * expf(b.m - m)};
}
__device__ __forceinline__ float plus(float a, float b) { return a + b; }
__device__ __forceinline__ float zero(float) { return 0.f; }
__device__ __forceinline__ Scaled zero(Scaled) { return {-INFINITY, 0.f}; }
__device__ __forceinline__ float from_lane(float v, int lane) {
  return __shfl_sync(0xffffffffu, v, lane);
}
__device__ __forceinline__ Scaled from_lane(Scaled v, int lane) {
  return {__shfl_sync(0xffffffffu, v.m, lane), __shfl_sync(0xffffffffu, v.s, lane)};
}
// For d = s - M: e^d, a sum's reciprocal, d less a sum's logarithm, e^d times a sum.
__device__ __forceinline__ float term_of(float d, float) { return expf(d); }
__device__ __forceinline__ Scaled term_of(float d, Scaled) {
  return {d, d == -INFINITY ? 0.f : 1.f};   // not 1 e^-inf: two of them would meet at inf - inf
}
__device__ __forceinline__ float inverse(float v) { return 1.f / v; }
__device__ __forceinline__ Scaled inverse(Scaled v) { return {-v.m, 1.f / v.s}; }
__device__ __forceinline__ float log_of(float d, float v) { return d - logf(v); }
__device__ __forceinline__ float log_of(float d, Scaled v) { return (d - v.m) - logf(v.s); }
__device__ __forceinline__ float times_exp(float d, float v) { return expf(d) * v; }
__device__ __forceinline__ float times_exp(float d, Scaled v) { return expf(d + v.m) * v.s; }

// Sum of the lanes before (kForward) or after each lane of the warp; `all` the warp's.
template <bool kForward, typename V>
__device__ __forceinline__ V warp_scan(V v, V* all) {
  const int lane = threadIdx.x & 31;
  V inc = v;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const V o = from_lane(inc, kForward ? lane - off : lane + off);
    if (kForward ? lane >= off : lane + off < 32) inc = plus(o, inc);
  }
  *all = from_lane(inc, kForward ? 31 : 0);
  const V before = from_lane(inc, kForward ? lane - 1 : lane + 1);
  return lane == (kForward ? 0 : 31) ? zero(v) : before;
}

struct Sequences {
  const float* scores;
  float* grad;                            // nullable
  const int32_t* cu;
  int batch, t_cap;
  const int32_t* k;
  const int32_t* order;
  int k_cap;
  int32_t* status;
};

struct SequenceShared {
  float s[kMaxVisual];                    // s_j - M
  unsigned short step[kMaxVisual];        // 1 + the step that removes j, 0 if kept
  Scaled sums[kMaxVisual];                // S_t, then Q_t (fp32: the first half)
  Scaled part[3][kSeqWarps];
  Pair lp[kSeqWarps];
  float hi[kSeqWarps], lo[kSeqWarps];
  int bad;
};
// Of an SM's 228 KB; a CTA takes another 1 KB, and less than that for its totals.
static_assert(kSeqPerSm * (sizeof(SequenceShared) + 2048) <= 228 * 1024, "resident at once");

// An image's log-probability (in every thread); Q_t in h->sums.
template <typename V>
__device__ __forceinline__ Pair sequence_sums(SequenceShared* h, const int32_t* seq, int n, int k) {
  V* sums = reinterpret_cast<V*>(h->sums);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int per = (k + kSeqThreads - 1) / kSeqThreads;
  const int c0 = min(static_cast<int>(threadIdx.x) * per, k), c1 = min(c0 + per, k);
  const V none = zero(V());
  V rest = none, own = none, all;
  for (int j = threadIdx.x; j < n; j += kSeqThreads)
    if (h->step[j] == 0) rest = plus(rest, term_of(h->s[j], V()));
  for (int t = c0; t < c1; ++t) own = plus(own, term_of(h->s[seq[t]], V()));
  warp_scan<true>(rest, &all);
  V* part = reinterpret_cast<V*>(h->part);
  if (lane == 0) part[warp] = all;
  V acc = warp_scan<false>(own, &all);
  if (lane == 0) part[kSeqWarps + warp] = all;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kSeqWarps; ++w) {
    acc = plus(acc, part[w]);
    if (w > warp) acc = plus(acc, part[kSeqWarps + w]);
  }
  Pair lp = {0.f, 0.f};
  V inv = none;
  for (int t = c1 - 1; t >= c0; --t) {
    const float d = h->s[seq[t]];
    acc = plus(acc, term_of(d, V()));
    sums[t] = acc;
    lp.add(log_of(d, acc));
    inv = plus(inv, inverse(acc));
  }
  V up = warp_scan<true>(inv, &all);
  if (lane == 0) part[2 * kSeqWarps + warp] = all;
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) lp.add(shfl_xor(lp, off));
  if (lane == 0) h->lp[warp] = lp;
  __syncthreads();
  lp = h->lp[0];
#pragma unroll
  for (int w = 0; w < kSeqWarps; ++w) {
    if (w > 0) lp.add(h->lp[w]);
    if (w < warp) up = plus(up, part[2 * kSeqWarps + w]);
  }
  for (int t = c0; t < c1; ++t) {
    up = plus(up, inverse(sums[t]));
    sums[t] = up;
  }
  __syncthreads();
  return lp;
}

template <typename V>
__device__ __forceinline__ void sequence_grad(const SequenceShared& h, float* grad, int n, int k,
                                              float g) {
  const V* sums = reinterpret_cast<const V*>(h.sums);
  if (threadIdx.x == 0) grad[0] = 0.f;                                      // CLS
  for (int j = threadIdx.x; j < n; j += kSeqThreads) {
    const int u = h.step[j];
    grad[1 + j] = g * ((u > 0 ? 1.f : 0.f) - times_exp(h.s[j], sums[(u > 0 ? u : k) - 1]));
  }
}

__global__ void __launch_bounds__(kSeqThreads, kSeqPerSm)
    pl_policy_loss_kernel(Sequences q, Actions p) {
  __shared__ SequenceShared h;
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Pair sum = {0.f, 0.f};
  for (int img = blockIdx.x; img < q.batch; img += gridDim.x) {
    const int lo = q.cu[img], hi = q.cu[img + 1];
    int n = hi - lo - 1, k = q.k[img];
    const RowIn in = row_in(p, img, q.batch);
    const bool inside = lo >= 0 && hi >= lo && hi <= q.t_cap;
    __syncthreads();                      // the image before is done with shared memory
    if (threadIdx.x == 0) h.bad = 0;
    if (!inside || n > kMaxVisual) {
      if (threadIdx.x == 0) record_status(q.status, DORA_ERR_DEVICE_SEQLEN);
      n = 0;
    }
    n = n < 0 ? 0 : n;
    if (k < 0 || k > n || k > q.k_cap) {
      if (threadIdx.x == 0) record_status(q.status, DORA_ERR_DEVICE_BAD_COUNT);
      k = k < 0 ? 0 : (k > n ? n : k);
      k = k > q.k_cap ? q.k_cap : k;
    }
    const bool takes = k > 0 && in.w != 0.f;
    const int32_t* seq = q.order + static_cast<size_t>(img) * q.k_cap;
    float top = -INFINITY, low = INFINITY;
    if (takes)
      for (int j = threadIdx.x; j < n; j += kSeqThreads) {
        const float s = q.scores[lo + 1 + j];
        h.s[j] = s;
        h.step[j] = 0;
        top = fmaxf(top, s);
        low = fminf(low, s);
      }
    top = warp_max(top, 32);
    low = -warp_max(-low, 32);
    if (lane == 0) {
      h.hi[warp] = top;
      h.lo[warp] = low;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kSeqWarps; ++w) {
      top = fmaxf(top, h.hi[w]);
      low = fminf(low, h.lo[w]);
    }
    if (takes) {
      for (int j = threadIdx.x; j < n; j += kSeqThreads) h.s[j] -= top;
      for (int t = threadIdx.x; t < k; t += kSeqThreads) {
        const int j = seq[t];
        if (j < 0 || j >= n ||
            atomicCAS(&h.step[j], static_cast<unsigned short>(0),
                      static_cast<unsigned short>(t + 1)) != 0)
          h.bad = 1;                      // out of range, or twice
      }
    }
    __syncthreads();
    if (!takes || h.bad) {
      const float fill = takes ? NAN : 0.f;
      if (threadIdx.x == 0) {
        if (takes) record_status(q.status, DORA_ERR_DEVICE_BAD_COUNT);
        p.logp[img] = fill;
        if (p.row_loss != nullptr) p.row_loss[img] = fill;
      }
      sum.add(all_terms(fill).of(threadIdx.x));
      if (q.grad != nullptr && inside)
        for (int r = lo + threadIdx.x; r < hi; r += kSeqThreads) q.grad[r] = fill;
      continue;
    }
    const bool narrow = top - low <= kRange;              // false for infinities
    const Pair lp = narrow ? sequence_sums<float>(&h, seq, n, k)
                           : sequence_sums<Scaled>(&h, seq, n, k);
    // l - q from the pair: the ratio of a long sequence keeps its digits
    const float x = p.ref_logp != nullptr ? (in.ref - lp.v) - lp.rest() : 0.f;
    Terms terms;
    const float g = row_terms(p, (lp.v - in.old_logp) + lp.rest(), x, in.adv, in.w, 0.f, &terms);
    sum.add(terms.of(threadIdx.x));
    if (threadIdx.x == 0) {
      p.logp[img] = lp.value();
      if (p.row_loss != nullptr) p.row_loss[img] = terms.v[0];
    }
    if (q.grad == nullptr) continue;
    if (narrow) sequence_grad<float>(h, q.grad + lo, n, k, g);
    else sequence_grad<Scaled>(h, q.grad + lo, n, k, g);
  }
  finish_totals<kSeqWarps>(p, sum);
}

}  // namespace policy
}  // namespace dora

using namespace dora;

namespace {
int device_or_error() {
  const int dev = checked_device();
  if (dev == -1) return DORA_ERR_CUDA;
  if (dev < 0) return DORA_ERR_UNSUPPORTED;
  return DORA_OK;
}
int launched(cudaError_t e) { return e == cudaSuccess ? DORA_OK : DORA_ERR_CUDA; }
constexpr int kMaxDevices = 64;

// The pointers are looked at when there are rows at all: an empty batch has none.
int check_actions(const policy::Actions& p, int rows, size_t workspace_bytes) {
  if (rows > 0 && (p.old_logp == nullptr || p.advantages == nullptr || p.logp == nullptr))
    return DORA_ERR_INVALID_ARG;
  if (!(p.clip_low >= 0.f && p.clip_low <= 1.f) || !(p.clip_high >= 0.f) ||
      !isfinite(p.clip_high) || !isfinite(p.kl_coef) || !isfinite(p.entropy_coef))
    return DORA_ERR_INVALID_ARG;
  if (rows > 0 && p.ref_logp == nullptr && p.kl_coef != 0.f) return DORA_ERR_INVALID_ARG;
  if (p.totals != nullptr &&
      (p.ws == nullptr || (reinterpret_cast<uintptr_t>(p.ws) & 255u) != 0 ||
       workspace_bytes < sizeof(policy::Workspace)))
    return DORA_ERR_INVALID_ARG;
  return DORA_OK;
}

int grid_for(int rows, int per_sm) {
  const int most = num_sms() * per_sm;
  const int ctas = rows < most ? rows : most;
  return ctas < policy::kMaxCtas ? ctas : policy::kMaxCtas;
}

template <typename T>
using RowsKernel = void (*)(policy::Rows<T>, policy::Actions);

// A dependent launch of `teams` clusters of `ctas` CTAs.
template <typename T>
int launch_rows(RowsKernel<T> kern, int teams, int block, int ctas, size_t smem,
                cudaStream_t stream, const policy::Rows<T>& r, const policy::Actions& p) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(teams * ctas);
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (ctas > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = ctas;
    attr[n].val.clusterDim.y = 1;
    attr[n++].val.clusterDim.z = 1;
  }
  if (pdl_enabled()) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  return launched(cudaLaunchKernelEx(&cfg, kern, r, p));
}

// How many clusters of this kernel the device holds at once; asked once a device.
// A cluster's CTAs come from one group of SMs, so that these are fewer than the SMs
// divided by the CTAs, and a grid of more would run the rest after the others' end.
template <typename T>
int resident_clusters(RowsKernel<T> kern, int block, int ctas, size_t smem,
                      std::atomic<int>* cache) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return 0;
  int n = cache[dev].load(std::memory_order_relaxed);
  if (n > 0) return n;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ctas;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess || n < 1) return 0;
  cache[dev].store(n, std::memory_order_relaxed);
  return n;
}

// One CTA an SM; the grid is what is resident at once.
template <typename T, int kSumWarps, int kGradWarps, int kStage, int kCtas>
int launch_ring(cudaStream_t stream, const policy::Rows<T>& r, const policy::Actions& p) {
  const RowsKernel<T> kern =
      policy::policy_ring_kernel<T, kSumWarps, kGradWarps, kStage, kCtas>;
  constexpr size_t smem = static_cast<size_t>(3) * kStage * 16;
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             static_cast<int>(smem));
  if (e != cudaSuccess) return launched(e);
  static std::atomic<int> cache[kMaxDevices];
  constexpr int kThreads = (3 + kSumWarps + kGradWarps) * 32;
  const int most = kCtas == 1 ? num_sms()
                              : resident_clusters<T>(kern, kThreads, kCtas, smem, cache);
  if (most < 1) return DORA_ERR_CUDA;
  return launch_rows<T>(kern, r.rows < most ? r.rows : most, kThreads, kCtas, smem, stream, r, p);
}

template <typename T>
int launch_policy(const void* logits, void* grad, int64_t ld, int rows, int classes,
                  const int32_t* legal, const int32_t* actions, float* entropy, int32_t* status,
                  const policy::Actions& p, cudaStream_t stream) {
  const policy::Rows<T> r = {static_cast<const T*>(logits), static_cast<T*>(grad), ld, rows,
                             classes, legal, actions, entropy, status};
  constexpr int kE = Granule<T>::kElems;
  // granules that a row can touch: one more where rows may start inside one
  const bool aligned = (reinterpret_cast<uintptr_t>(logits) & 15u) == 0 && ld % kE == 0;
  const int64_t need = (static_cast<int64_t>(classes) + (aligned ? 0 : kE - 1) + kE - 1) / kE;
  // The fewest lanes that hold a row: what a row costs besides its granules is paid per
  // warp (16384 x 2000 bf16: a warp a row 32 us, a CTA 79).
  const int sms = num_sms();
  if (need <= 32) {
    const int ctas = grid_for((rows + 31) / 32, 8);
    return need <= 8 ? launch_rows<T>(policy::policy_warp_kernel<T, 8, 1>, ctas, 256, 1, 0, stream,
                                      r, p)
                     : launch_rows<T>(policy::policy_warp_kernel<T, 8, 4>, ctas, 256, 1, 0, stream,
                                      r, p);
  }
  const int eights = grid_for((rows + 7) / 8, 8);
  if (need <= 128)
    return launch_rows<T>(policy::policy_warp_kernel<T, 32, 4>, eights, 256, 1, 0, stream, r, p);
  // From here on few rows get more lanes each, as long as all have their place at once
  // (256 x 4000 bf16: a CTA a row 6.2 us, a warp 8.5).
  if (need <= 512 && rows > 8 * sms)
    return need <= 256 ? launch_rows<T>(policy::policy_warp_kernel<T, 32, 8>, eights, 256, 1, 0,
                                        stream, r, p)
                       : launch_rows<T>(policy::policy_warp_kernel<T, 32, 16>, eights, 256, 1, 0,
                                        stream, r, p);
  if (need <= 1024)
    return launch_rows<T>(policy::policy_cta_kernel<T, 128, 8>, grid_for(rows, 8), 128, 1, 0,
                          stream, r, p);
  if (need > 4096 * 8) {
    static std::atomic<int> cache[kMaxDevices];
    const int most = resident_clusters<T>(policy::policy_long_kernel<T>, policy::kLongBlock,
                                          policy::kLongCtas, 0, cache);
    if (most < 1) return DORA_ERR_CUDA;
    return launch_rows<T>(policy::policy_long_kernel<T>, rows < most ? rows : most,
                          policy::kLongBlock, policy::kLongCtas, 0, stream, r, p);
  }
  int ctas = 1;
  while (need > 4096 * ctas) ctas *= 2;
  while (ctas < 8 && rows * ctas * 2 <= sms) ctas *= 2;
  if (ctas == 1 && need <= 2048)
    return launch_rows<T>(policy::policy_cta_kernel<T, 256, 8>, grid_for(rows, 4), 256, 1, 0,
                          stream, r, p);
  switch (ctas) {
    case 1: return launch_ring<T, 8, 8, 4096, 1>(stream, r, p);
    case 2: return launch_ring<T, 8, 8, 4096, 2>(stream, r, p);
    case 4: return launch_ring<T, 8, 8, 4096, 4>(stream, r, p);
    default: return launch_ring<T, 8, 8, 4096, 8>(stream, r, p);
  }
}
}  // namespace

extern "C" {

size_t dora_policy_workspace_size(void) { return (sizeof(policy::Workspace) + 255) / 256 * 256; }

int dora_policy_loss(const void* logits, int32_t dtype, int32_t rows, int32_t classes, int64_t ld,
                     const int32_t* legal, const int32_t* actions, const float* old_logp,
                     const float* ref_logp, const float* advantages, const float* weights,
                     float clip_low, float clip_high, float kl_coef, float entropy_coef,
                     float* logp, float* entropy, float* row_loss, void* grad, float* totals,
                     void* workspace, size_t workspace_bytes, int32_t* status,
                     dora_stream_t stream_) {
  // rows and granules are counted in 32 bits, with room for a step past the last
  if (rows < 0 || rows > (1 << 30) || classes < 1 || classes > (1 << 30) || ld < classes ||
      dtype < DORA_BF16 || dtype > DORA_F32)
    return DORA_ERR_INVALID_ARG;
  if (rows > 0 && (logits == nullptr || actions == nullptr)) return DORA_ERR_INVALID_ARG;
  const uintptr_t size_mask = dtype == DORA_F32 ? 3u : 1u;
  if ((reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(grad)) & size_mask)
    return DORA_ERR_INVALID_ARG;
  const policy::Actions p = {old_logp, ref_logp, advantages, weights, clip_low, clip_high, kl_coef,
                             entropy_coef, logp, row_loss, totals,
                             static_cast<policy::Workspace*>(workspace)};
  int e = check_actions(p, rows, workspace_bytes);
  if (e != DORA_OK) return e;
  e = device_or_error();
  if (e != DORA_OK) return e;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  if (rows == 0)
    return totals == nullptr
               ? DORA_OK
               : launched(cudaMemsetAsync(totals, 0, policy::kTerms * sizeof(float), stream));
  switch (dtype) {
    case DORA_BF16:
      return launch_policy<__nv_bfloat16>(logits, grad, ld, rows, classes, legal, actions, entropy,
                                          status, p, stream);
    case DORA_F16:
      return launch_policy<__half>(logits, grad, ld, rows, classes, legal, actions, entropy,
                                   status, p, stream);
    default:
      return launch_policy<float>(logits, grad, ld, rows, classes, legal, actions, entropy, status,
                                  p, stream);
  }
}

int dora_pl_policy_loss(const float* scores, const int32_t* cu, int32_t batch, int32_t t_cap,
                        const int32_t* k, const int32_t* order, int32_t k_cap,
                        const float* old_logp, const float* ref_logp, const float* advantages,
                        const float* weights, float clip_low, float clip_high, float kl_coef,
                        float* logp, float* row_loss, float* grad, float* totals, void* workspace,
                        size_t workspace_bytes, int32_t* status, dora_stream_t stream_) {
  if (batch < 0 || batch > (1 << 24) || t_cap < 0 || k_cap < 1 || k_cap > policy::kMaxVisual)
    return DORA_ERR_INVALID_ARG;
  if (batch > 0 && (scores == nullptr || cu == nullptr || k == nullptr || order == nullptr))
    return DORA_ERR_INVALID_ARG;
  const policy::Actions p = {old_logp, ref_logp, advantages, weights, clip_low, clip_high, kl_coef,
                             0.f, logp, row_loss, totals,
                             static_cast<policy::Workspace*>(workspace)};
  int e = check_actions(p, batch, workspace_bytes);
  if (e != DORA_OK) return e;
  e = device_or_error();
  if (e != DORA_OK) return e;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  if (batch == 0)
    return totals == nullptr
               ? DORA_OK
               : launched(cudaMemsetAsync(totals, 0, policy::kTerms * sizeof(float), stream));
  const policy::Sequences q = {scores, grad, cu, batch, t_cap, k, order, k_cap, status};
  return launched(launch_pdl(policy::pl_policy_loss_kernel,
                             dim3(grid_for(batch, policy::kSeqPerSm)), dim3(policy::kSeqThreads),
                             0, stream, q, p));
}

}  // extern "C"
