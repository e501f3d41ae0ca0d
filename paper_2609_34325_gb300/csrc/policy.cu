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
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "dora.h"
#include "dora_ptx.cuh"
#include "granule.cuh"
#include "token_ops.cuh"

namespace dora {
namespace policy {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kTerms = 6;                 // sums over the rows, in the order of `totals`
constexpr int kMaxCtas = 152 * 16;        // partial sums that the workspace holds
constexpr int kThreads = 256;
constexpr int kMaxVisual = 2048;          // visual tokens per image held in shared memory
constexpr int kPerThread = kMaxVisual / kThreads;

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
};
__device__ __forceinline__ Pair shfl_xor(Pair p, int off) {
  return {__shfl_xor_sync(0xffffffffu, p.v, off), __shfl_xor_sync(0xffffffffu, p.lost, off)};
}

struct Workspace {
  unsigned ticket;                        // CTAs done; zero between calls
  unsigned pad[63];
  Pair partial[kTerms][kMaxCtas];
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

// Sums over a thread's rows: loss, policy term, KL, entropy, clipped weight, weight.
struct Sums {
  Pair v[kTerms];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < kTerms; ++i) v[i] = Pair{0.f, 0.f};
  }
  __device__ __forceinline__ void add(int i, float x) { v[i].add(x); }
};

// One row's loss from l - q, x = q_ref - l and the entropy h; returns g.  A NaN
// ratio is left to spread (comparisons, no fmin).  `sums` of the one thread that
// counts the row, null for the others.
__device__ __forceinline__ float row_terms(const Actions& p, float log_ratio, float x, float adv,
                                           float w, float h, float* loss, Sums* sums) {
  const float ratio = expf(log_ratio);
  const float lo = 1.f - p.clip_low, hi = 1.f + p.clip_high;
  const float cut = (ratio < lo ? lo : (ratio > hi ? hi : ratio)) * adv;
  const float plain = ratio * adv;
  const bool inside = !(plain > cut);
  const float surrogate = -(inside ? plain : cut);
  float g = inside ? -plain : 0.f, kl = 0.f;
  if (p.ref_logp != nullptr) {
    const float em1 = expm1f(x);
    kl = em1 - x;
    g = fmaf(-p.kl_coef, em1, g);
  }
  float row = fmaf(p.kl_coef, kl, surrogate);
  if (p.entropy_coef != 0.f) row = fmaf(-p.entropy_coef, h, row);
  row *= w;
  *loss = row;
  if (sums == nullptr) return g * w;
  sums->add(0, row);
  sums->add(1, w * surrogate);
  sums->add(2, w * kl);
  sums->add(3, w * h);
  sums->add(4, inside ? 0.f : w);
  sums->add(5, w);
  return g * w;
}

// The CTA's sums (held by thread 0) go to its place in the workspace; the CTA that
// is last adds all of them in the order of the CTAs, so that the totals do not
// depend on which one that is, and leaves the ticket at zero for the next call.
__device__ __forceinline__ void finish_totals(const Actions& p, const Sums& sums) {
  if (p.totals == nullptr) return;
  if (gridDim.x == 1) {
    if (threadIdx.x == 0)
#pragma unroll
      for (int i = 0; i < kTerms; ++i) p.totals[i] = sums.v[i].v + sums.v[i].lost;
    return;
  }
  __shared__ bool last;
  Workspace* ws = p.ws;
  if (threadIdx.x == 0) {
#pragma unroll
    for (int i = 0; i < kTerms; ++i) ws->partial[i][blockIdx.x] = sums.v[i];
    __threadfence();
    last = atomicAdd(&ws->ticket, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  for (int i = threadIdx.x >> 5; i < kTerms; i += warps) {
    Pair t = {0.f, 0.f};
    for (int c = lane; c < static_cast<int>(gridDim.x); c += 32) {
      const float2 x = __ldcg(reinterpret_cast<const float2*>(&ws->partial[i][c]));
      t.add(Pair{x.x, x.y});
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) t.add(shfl_xor(t, off));
    if (lane == 0) p.totals[i] = t.v + t.lost;
  }
  if (threadIdx.x == 0) ws->ticket = 0;
}

template <typename F>
__device__ __forceinline__ F block_sum(F v, F* scratch) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
  __syncthreads();
  v = scratch[0];
#pragma unroll
  for (int w = 1; w < kThreads / 32; ++w) v += scratch[w];
  return v;
}

// ---------------------------------------------------------------------------
// Categorical actions.  A row is read once into registers, as 16-byte granules,
// by the lanes of a warp, a CTA or a cluster of CTAs; from there come its maximum
// m, its sums s = sum e^{z - m} and t = sum e^{z - m} (z - m), and the gradient:
//   p_j = e^{z_j - m} / s,  H = log s - t / s,
//   d loss / d z_j = g (1(j = a) - p_j) + w c p_j (log p_j + H).
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

// A row's scalars, loaded while the row before is worked on.
struct RowIn {
  int action, n;
  float w, old_logp, adv, ref;
};

template <typename T>
__device__ __forceinline__ RowIn row_in(const Rows<T>& r, const Actions& p, int row) {
  RowIn in = {-1, 0, 0.f, 0.f, 0.f, 0.f};
  if (row < r.rows) {
    in.action = r.actions[row];
    in.w = p.weights != nullptr ? p.weights[row] : 1.f;
    in.n = r.legal != nullptr ? r.legal[row] : r.classes;
    in.old_logp = p.old_logp[row];
    in.adv = p.advantages[row];
    in.ref = p.ref_logp != nullptr ? p.ref_logp[row] : 0.f;
  }
  return in;
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// e^d for a difference d <= 0 of logits.
__device__ __forceinline__ float exp_of(float d) { return ex2(d * kLog2e); }

constexpr float kFloor = -200.f;          // below it e^d is 0: keeps 0 * inf out of e^d * d

template <typename T>
struct RowPtr {
  static constexpr int kE = Granule<T>::kElems;
  const T* z;                             // the row's first element
  int mis;                                // elements of its first granule before it
  __device__ __forceinline__ explicit RowPtr(const T* p)
      : z(p), mis(static_cast<int>((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T))) {}

  // Granule i of the row, elements outside [0, n) as -inf.
  __device__ __forceinline__ uint4 load(int i, int n) const {
    const int c = i * kE - mis;
    if (c >= 0 && c + kE <= n) return *reinterpret_cast<const uint4*>(z + c);
    constexpr uint32_t kNone = Granule<T>::kNegInfWord;
    uint4 q = make_uint4(kNone, kNone, kNone, kNone);
    if (c < n) {
      float v[kE];
      Granule<T>::unpack(q, v);
#pragma unroll
      for (int e = 0; e < kE; ++e)
        if (c + e >= 0 && c + e < n) v[e] = to_float(z[c + e]);
      q = Granule<T>::pack(v);            // exact: the values come from T
    }
    return q;
  }
  // kHeld granules from i on, kStep apart.
  template <int kHeld, int kStep>
  __device__ __forceinline__ void load_all(int i, int n, uint4* q) const {
    const int c = i * kE - mis;
    if (c >= 0 && c + ((kHeld - 1) * kStep + 1) * kE <= n) {
      const uint4* g = reinterpret_cast<const uint4*>(z + c);
#pragma unroll
      for (int u = 0; u < kHeld; ++u) q[u] = g[u * kStep];
    } else {
#pragma unroll
      for (int u = 0; u < kHeld; ++u) q[u] = load(i + u * kStep, n);
    }
  }
  // Values of granule i into the row at `to` of `classes` elements, 0 from n on.
  __device__ __forceinline__ void store(T* to, bool aligned, int i, int n, int classes,
                                        float* v) const {
    const int c = i * kE - mis;
    if (c >= classes) return;
#pragma unroll
    for (int e = 0; e < kE; ++e)
      if (c + e >= n) v[e] = 0.f;
    if (aligned && c >= 0 && c + kE <= classes) {
      *reinterpret_cast<uint4*>(to + c) = Granule<T>::pack(v);
    } else {
#pragma unroll
      for (int e = 0; e < kE; ++e)
        if (c + e >= 0 && c + e < classes) from_float(v[e], to + c + e);
    }
  }
};

// Sums of e^{z - m} and e^{z - m} (z - m) over one granule.  An m of -inf (nothing
// but -inf so far) counts as 0, so that its terms are 0 and not NaN.
template <typename T>
__device__ __forceinline__ void add_exps(uint4 q, float m, float* s, float* t) {
  constexpr int kE = Granule<T>::kElems;
  float v[kE];
  Granule<T>::unpack(q, v);
#pragma unroll
  for (int e = 0; e < kE; ++e) {
    const float d = v[e] - m, x = exp_of(d);
    *s += x;
    *t = fmaf(x, fmaxf(d, kFloor), *t);
  }
}
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }

// What the gradient of a row needs.
struct RowGrad {
  float m, a, b, g;                       // d loss / d z = e^{z - m} (a + b (z - m)) + g 1(j = a)
  int granule, element;                   // of the action
};

template <typename T>
__device__ __forceinline__ void grad_granule(uint4 q, const RowGrad& k, int i, float* v) {
  constexpr int kE = Granule<T>::kElems;
  Granule<T>::unpack(q, v);
  if (k.b == 0.f) {
#pragma unroll
    for (int e = 0; e < kE; ++e) v[e] = exp_of(v[e] - k.m) * k.a;
  } else {
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      const float d = v[e] - k.m;
      v[e] = exp_of(d) * fmaf(k.b, fmaxf(d, kFloor), k.a);
    }
  }
  if (i == k.granule) {
#pragma unroll
    for (int e = 0; e < kE; ++e)
      if (e == k.element) v[e] += k.g;
  }
}

// The row's outputs and what its gradient needs, from m, s, t and the action's logit;
// `leader` writes and counts.
template <typename T>
__device__ __forceinline__ RowGrad finish_row(const Rows<T>& r, const Actions& p, const RowIn& in,
                                              int row, float za, float m, float s, float t,
                                              int mis, bool leader, Sums* sums) {
  constexpr int kE = Granule<T>::kElems;
  const float ls = logf(s), inv = 1.f / s, h = ls - t * inv;
  const float lp = (za - m) - ls;
  float loss;
  const float g = row_terms(p, lp - in.old_logp, in.ref - lp, in.adv, in.w, h, &loss,
                            leader ? sums : nullptr);
  if (leader) {
    p.logp[row] = lp;
    if (r.entropy != nullptr) r.entropy[row] = h;
    if (p.row_loss != nullptr) p.row_loss[row] = loss;
  }
  const float cw = in.w * p.entropy_coef;
  return RowGrad{m, (cw * (h - ls) - g) * inv, cw * inv, g, (in.action + mis) / kE,
                 (in.action + mis) % kE};
}

// A row that takes no part (0) or is not valid (NaN).
template <typename T>
__device__ __forceinline__ void fill_row(const Rows<T>& r, const Actions& p, int row, float fill,
                                         Sums* sums) {
  if (fill != 0.f) {
    record_status(r.status, DORA_ERR_DEVICE_BAD_COUNT);
    for (int i = 0; i < kTerms; ++i) sums->add(i, fill);
  }
  p.logp[row] = fill;
  if (r.entropy != nullptr) r.entropy[row] = fill;
  if (p.row_loss != nullptr) p.row_loss[row] = fill;
}

__device__ __forceinline__ bool same_alignment(const void* a, const void* b) {
  return ((reinterpret_cast<uintptr_t>(a) ^ reinterpret_cast<uintptr_t>(b)) & 15u) == 0;
}

// Thread 0 gets the sums of all threads that are a multiple of kStride (the others'
// are zero).
template <int kStride>
__device__ __forceinline__ void gather_sums(const Actions& p, Sums* sums) {
  if (p.totals == nullptr) return;
  __shared__ Pair all[kTerms][kThreads / 32];
#pragma unroll
  for (int i = 0; i < kTerms; ++i) {
    Pair t = sums->v[i];
#pragma unroll
    for (int off = 16; off >= kStride; off >>= 1) t.add(shfl_xor(t, off));
    if ((threadIdx.x & 31) == 0) all[i][threadIdx.x >> 5] = t;
  }
  __syncthreads();
  if (threadIdx.x < 32) {                 // lane: warp (low bits) of terms 0..3, then of 4, 5
    static_assert(kThreads / 32 == 8 && kTerms == 6, "eight warps in groups of eight lanes");
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int i = 4 * half + (threadIdx.x >> 3);
      Pair t = i < kTerms ? all[i][threadIdx.x & 7] : Pair{0.f, 0.f};
#pragma unroll
      for (int off = 4; off > 0; off >>= 1) t.add(shfl_xor(t, off));
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const Pair o = {__shfl_sync(0xffffffffu, t.v, 8 * k),
                        __shfl_sync(0xffffffffu, t.lost, 8 * k)};
        if (4 * half + k < kTerms) sums->v[4 * half + k] = o;
      }
    }
  }
}

// Short rows: kLanes lanes of a warp hold one, kHeld granules each.
template <typename T, int kLanes, int kHeld>
__global__ void __launch_bounds__(kThreads) policy_warp_kernel(Rows<T> r, Actions p) {
  constexpr int kRowsPerCta = kThreads / kLanes;
  pdl_wait();
  const int lane = threadIdx.x % kLanes;
  const int step = gridDim.x * kRowsPerCta;
  Sums sums;
  sums.clear();
  // the loop is the same for all groups of a warp: shuffles need every lane
  const int first = blockIdx.x * kRowsPerCta + (threadIdx.x / 32) * (32 / kLanes);
  int row = first + (threadIdx.x % 32) / kLanes;
  RowIn in = row_in(r, p, row);
  for (int base = first; base < r.rows; base += step, row += step) {
    const bool exists = row < r.rows;
    const bool takes = exists && in.action >= 0 && in.w != 0.f;
    const bool bad = takes && (in.n < 0 || in.n > r.classes || in.action >= in.n);
    const int n = takes && !bad ? in.n : 0;
    const RowPtr<T> z(r.logits + (exists ? row : 0) * r.ld);
    const float za = n > 0 ? to_float(z.z[in.action]) : 0.f;
    uint4 q[kHeld];
    z.template load_all<kHeld, kLanes>(lane, n, q);
    const RowIn next = row_in(r, p, row + step);
    float m = -INFINITY, s = 0.f, t = 0.f;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) m = fmaxf(m, Granule<T>::largest(q[i]));
#pragma unroll
    for (int off = kLanes / 2; off > 0; off >>= 1)
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
#pragma unroll
    for (int i = 0; i < kHeld; ++i) add_exps<T>(q[i], m, &s, &t);
#pragma unroll
    for (int off = kLanes / 2; off > 0; off >>= 1) {
      s += __shfl_xor_sync(0xffffffffu, s, off);
      t += __shfl_xor_sync(0xffffffffu, t, off);
    }
    __syncwarp();                         // every lane has read its logits: grad may be logits
    if (exists) {
      T* dz = r.grad != nullptr ? r.grad + row * r.ld : nullptr;
      const bool aligned = dz != nullptr && same_alignment(dz, z.z);
      if (n > 0) {
        const RowGrad k = finish_row(r, p, in, row, za, m, s, t, z.mis, lane == 0, &sums);
        if (dz != nullptr)
#pragma unroll
          for (int i = 0; i < kHeld; ++i) {
            float v[Granule<T>::kElems];
            grad_granule<T>(q[i], k, lane + i * kLanes, v);
            z.store(dz, aligned, lane + i * kLanes, n, r.classes, v);
          }
      } else {
        const float fill = bad ? NAN : 0.f;
        if (lane == 0) fill_row(r, p, row, fill, &sums);
        if (dz != nullptr)
#pragma unroll
          for (int i = 0; i < kHeld; ++i) {
            float v[Granule<T>::kElems];
#pragma unroll
            for (int e = 0; e < Granule<T>::kElems; ++e) v[e] = fill;
            z.store(dz, aligned, lane + i * kLanes, r.classes, r.classes, v);
          }
      }
    }
    in = next;
  }
  gather_sums<kLanes>(p, &sums);
  finish_totals(p, sums);
}

// (m, s, t) of a part of a row; parts are brought to a common m exactly as often as
// they are joined.
struct Part {
  float m, s, t, pad;
};

// Every warp's part goes to every CTA of the cluster, and every warp joins them all:
// one barrier a row.  `slots` alternate from row to row, so that a warp that is a
// row ahead writes where nobody reads.
template <int kWarps, int kCtas>
__device__ __forceinline__ Part join_parts(Part mine, Part* slots) {
  constexpr int kParts = kWarps * kCtas;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (kCtas == 1) {
    if (lane == 0) slots[warp] = mine;
    __syncthreads();
  } else {
    if (lane < kCtas) {
      const uint32_t local = smem_u32(slots + cluster_ctarank() * kWarps + warp);
      asm volatile(
          "{\n\t.reg .b32 ra;\n\t"
          "mapa.shared::cluster.u32 ra, %0, %1;\n\t"
          "st.shared::cluster.v4.f32 [ra], {%2, %3, %4, %5};\n\t}" ::"r"(local),
          "r"(lane), "f"(mine.m), "f"(mine.s), "f"(mine.t), "f"(0.f)
          : "memory");
    }
    cluster_sync();
  }
  constexpr int kPer = (kParts + 31) / 32;
  Part h[kPer];
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int at = lane + 32 * i;
    h[i] = at < kParts ? slots[at] : Part{-INFINITY, 0.f, 0.f, 0.f};
    m = fmaxf(m, h[i].m);
  }
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
  float s = 0.f, t = 0.f;
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    if (h[i].m != -INFINITY || h[i].s != 0.f) {             // a NaN sum is taken along
      const float d = h[i].m - m, x = exp_of(d);
      s = fmaf(h[i].s, x, s);
      t = fmaf(fmaf(h[i].s, fmaxf(d, kFloor), h[i].t), x, t);
    }
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    s += __shfl_xor_sync(0xffffffffu, s, off);
    t += __shfl_xor_sync(0xffffffffu, t, off);
  }
  return Part{m, s, t, 0.f};
}

// Longer rows: kCtas CTAs (a cluster when there are several) hold one.
template <typename T, int kBlock, int kHeld, int kCtas>
__global__ void __launch_bounds__(kBlock, kHeld > 4 ? 2 : (kBlock > 128 ? 3 : 10))
    policy_block_kernel(Rows<T> r, Actions p) {
  constexpr int kWarps = kBlock / 32;
  __shared__ Sums sums;                   // thread 0's: registers are for the row
  __shared__ Part slots[2][kWarps * kCtas];
  pdl_wait();
  const int rank = kCtas > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int step = gridDim.x / kCtas;
  const int g0 = rank * kBlock * kHeld + threadIdx.x;
  const bool leader = rank == 0 && threadIdx.x == 0;
  int parity = 0;
  if (threadIdx.x == 0) sums.clear();
  int row = blockIdx.x / kCtas;
  RowIn in = row_in(r, p, row);
  for (; row < r.rows; row += step) {
    const RowIn next = row_in(r, p, row + step);
    const bool takes = in.action >= 0 && in.w != 0.f;
    const bool bad = takes && (in.n < 0 || in.n > r.classes || in.action >= in.n);
    const RowPtr<T> z(r.logits + row * r.ld);
    T* dz = r.grad != nullptr ? r.grad + row * r.ld : nullptr;
    const bool aligned = dz != nullptr && same_alignment(dz, z.z);
    if (takes && !bad) {
      const float za = to_float(z.z[in.action]);
      uint4 q[kHeld];
      z.template load_all<kHeld, kBlock>(g0, in.n, q);
      Part part = {-INFINITY, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kHeld; ++i) part.m = fmaxf(part.m, Granule<T>::largest(q[i]));
#pragma unroll
      for (int off = 16; off > 0; off >>= 1)
        part.m = fmaxf(part.m, __shfl_xor_sync(0xffffffffu, part.m, off));
#pragma unroll
      for (int i = 0; i < kHeld; ++i) add_exps<T>(q[i], base_of(part.m), &part.s, &part.t);
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) {
        part.s += __shfl_xor_sync(0xffffffffu, part.s, off);
        part.t += __shfl_xor_sync(0xffffffffu, part.t, off);
      }
      // after its barrier every logit of the row has been read: grad may be logits
      part = join_parts<kWarps, kCtas>(part, slots[parity]);
      parity ^= 1;
      const RowGrad k =
          finish_row(r, p, in, row, za, part.m, part.s, part.t, z.mis, leader, &sums);
      if (dz != nullptr) {
        const int c = g0 * Granule<T>::kElems - z.mis;
        if (aligned && c >= 0 && c + ((kHeld - 1) * kBlock + 1) * Granule<T>::kElems <= in.n) {
          uint4* to = reinterpret_cast<uint4*>(dz + c);
#pragma unroll
          for (int i = 0; i < kHeld; ++i) {
            float v[Granule<T>::kElems];
            grad_granule<T>(q[i], k, g0 + i * kBlock, v);
            to[i * kBlock] = Granule<T>::pack(v);
          }
        } else {
#pragma unroll
          for (int i = 0; i < kHeld; ++i) {
            float v[Granule<T>::kElems];
            grad_granule<T>(q[i], k, g0 + i * kBlock, v);
            z.store(dz, aligned, g0 + i * kBlock, in.n, r.classes, v);
          }
        }
      }
    } else {
      const float fill = bad ? NAN : 0.f;
      if (leader) fill_row(r, p, row, fill, &sums);
      if (dz != nullptr)
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
          float v[Granule<T>::kElems];
#pragma unroll
          for (int e = 0; e < Granule<T>::kElems; ++e) v[e] = fill;
          z.store(dz, aligned, g0 + i * kBlock, r.classes, r.classes, v);
        }
    }
    in = next;
  }
  finish_totals(p, sums);
}

// Rows longer than the registers of a cluster: the same, but the row is read a second
// time (from L2, where the clusters' rows fit) for its gradient.
constexpr int kLongBlock = 512, kLongCtas = 8, kLongStep = 4;

template <typename T>
__global__ void __launch_bounds__(kLongBlock, 2) policy_long_kernel(Rows<T> r, Actions p) {
  constexpr int kWarps = kLongBlock / 32, kStride = kLongBlock * kLongCtas;
  __shared__ Part slots[2][kWarps * kLongCtas];
  __shared__ Sums sums;
  pdl_wait();
  const int rank = static_cast<int>(cluster_ctarank());
  const int step = gridDim.x / kLongCtas;
  const int g0 = rank * kLongBlock + threadIdx.x;
  const bool leader = rank == 0 && threadIdx.x == 0;
  int parity = 0;
  if (threadIdx.x == 0) sums.clear();
  for (int row = blockIdx.x / kLongCtas; row < r.rows; row += step) {
    const RowIn in = row_in(r, p, row);
    const bool takes = in.action >= 0 && in.w != 0.f;
    const bool bad = takes && (in.n < 0 || in.n > r.classes || in.action >= in.n);
    const RowPtr<T> z(r.logits + row * r.ld);
    T* dz = r.grad != nullptr ? r.grad + row * r.ld : nullptr;
    const bool aligned = dz != nullptr && same_alignment(dz, z.z);
    const int granules = (r.classes + z.mis + Granule<T>::kElems - 1) / Granule<T>::kElems;
    if (takes && !bad) {
      const float za = to_float(z.z[in.action]);
      Part part = {-INFINITY, 0.f, 0.f, 0.f};
      for (int i = g0; i < granules; i += kStride * kLongStep) {
        uint4 q[kLongStep];
        z.template load_all<kLongStep, kStride>(i, in.n, q);
        float m = part.m;
#pragma unroll
        for (int u = 0; u < kLongStep; ++u) m = fmaxf(m, Granule<T>::largest(q[u]));
        if (m > part.m && part.s != 0.f) {
          const float d = part.m - m, x = exp_of(d);
          part.t = fmaf(part.s, fmaxf(d, kFloor), part.t) * x;
          part.s *= x;
        }
        part.m = m;
#pragma unroll
        for (int u = 0; u < kLongStep; ++u) add_exps<T>(q[u], base_of(m), &part.s, &part.t);
      }
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) {
        const Part o = {__shfl_xor_sync(0xffffffffu, part.m, off),
                        __shfl_xor_sync(0xffffffffu, part.s, off),
                        __shfl_xor_sync(0xffffffffu, part.t, off), 0.f};
        const float m = fmaxf(part.m, o.m), c = base_of(m);
        const float da = part.m - c, db = o.m - c, xa = exp_of(da), xb = exp_of(db);
        part.t = fmaf(part.s, fmaxf(da, kFloor), part.t) * xa +
                 fmaf(o.s, fmaxf(db, kFloor), o.t) * xb;
        part.s = part.s * xa + o.s * xb;
        part.m = m;
      }
      part = join_parts<kWarps, kLongCtas>(part, slots[parity]);
      parity ^= 1;
      const RowGrad k =
          finish_row(r, p, in, row, za, part.m, part.s, part.t, z.mis, leader, &sums);
      if (dz != nullptr)
        for (int i = g0; i < granules; i += kStride) {
          float v[Granule<T>::kElems];
          grad_granule<T>(z.load(i, in.n), k, i, v);
          z.store(dz, aligned, i, in.n, r.classes, v);
        }
    } else {
      const float fill = bad ? NAN : 0.f;
      if (leader) fill_row(r, p, row, fill, &sums);
      if (dz != nullptr)
        for (int i = g0; i < granules; i += kStride) {
          float v[Granule<T>::kElems];
#pragma unroll
          for (int e = 0; e < Granule<T>::kElems; ++e) v[e] = fill;
          z.store(dz, aligned, i, r.classes, r.classes, v);
        }
    }
  }
  finish_totals(p, sums);
}

// ---------------------------------------------------------------------------
// Ordered removals.  (m, s) stands for m + log s; sums of exponentials are only
// ever added, so that nothing cancels whatever the range of the scores.
// ---------------------------------------------------------------------------
struct Lse {
  float m, s;
};
__device__ __forceinline__ Lse lse_merge(Lse a, Lse b) {
  if (a.s == 0.f) return b;
  if (b.s == 0.f) return a;
  const float m = fmaxf(a.m, b.m);
  return {m, a.s * expf(a.m - m) + b.s * expf(b.m - m)};
}

// Inclusive scan over the block's threads of one pair each, from thread 0 on
// (forward) or from the last one back; returns the exclusive value (what the
// threads before, or after, hold together).
template <bool kForward>
__device__ __forceinline__ Lse block_scan(Lse v, Lse* scratch) {
  constexpr int kWarps = kThreads / 32;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Lse inc = v;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const Lse o = kForward ? Lse{__shfl_up_sync(0xffffffffu, inc.m, off),
                                 __shfl_up_sync(0xffffffffu, inc.s, off)}
                           : Lse{__shfl_down_sync(0xffffffffu, inc.m, off),
                                 __shfl_down_sync(0xffffffffu, inc.s, off)};
    if (kForward ? lane >= off : lane + off < 32) inc = lse_merge(o, inc);
  }
  __syncthreads();
  if (lane == (kForward ? 31 : 0)) scratch[warp] = inc;
  Lse before = kForward ? Lse{__shfl_up_sync(0xffffffffu, inc.m, 1),
                              __shfl_up_sync(0xffffffffu, inc.s, 1)}
                        : Lse{__shfl_down_sync(0xffffffffu, inc.m, 1),
                              __shfl_down_sync(0xffffffffu, inc.s, 1)};
  if (lane == (kForward ? 0 : 31)) before = Lse{-INFINITY, 0.f};
  __syncthreads();
  for (int i = 0; i < kWarps; ++i)
    if (kForward ? i < warp : i > warp) before = lse_merge(before, scratch[i]);
  return before;
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

__global__ void __launch_bounds__(kThreads) pl_policy_loss_kernel(Sequences q, Actions p) {
  __shared__ float s[kMaxVisual];
  __shared__ int32_t pos[kMaxVisual];     // 1 + the step that removes j, 0 if kept
  __shared__ Lse upto[kMaxVisual];        // sum over u <= t of exp(-L_u)
  __shared__ Lse part[kThreads / 32];
  __shared__ double dpart[kThreads / 32];
  __shared__ int bad;
  pdl_wait();
  Sums sums;
  sums.clear();
  for (int img = blockIdx.x; img < q.batch; img += gridDim.x) {
    const int lo = q.cu[img], hi = q.cu[img + 1];
    int n = hi - lo - 1, k = q.k[img];
    const float w = p.weights != nullptr ? p.weights[img] : 1.f;
    const bool inside = lo >= 0 && hi >= lo && hi <= q.t_cap;
    __syncthreads();                      // the image before is done with shared memory
    if (threadIdx.x == 0) bad = 0;
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
    const bool takes = k > 0 && w != 0.f;
    const int32_t* seq = q.order + static_cast<size_t>(img) * q.k_cap;
    for (int j = threadIdx.x; j < n; j += kThreads) {
      s[j] = takes ? q.scores[lo + 1 + j] : 0.f;
      pos[j] = 0;
    }
    __syncthreads();
    if (takes)
      for (int t = threadIdx.x; t < k; t += kThreads) {
        const int j = seq[t];
        if (j < 0 || j >= n || atomicCAS(&pos[j], 0, t + 1) != 0) bad = 1;   // range, repeats
      }
    __syncthreads();
    if (!takes || bad) {
      const float fill = takes ? NAN : 0.f;
      if (threadIdx.x == 0) {
        if (takes) record_status(q.status, DORA_ERR_DEVICE_BAD_COUNT);
        p.logp[img] = fill;
        if (p.row_loss != nullptr) p.row_loss[img] = fill;
        for (int i = 0; i < kTerms; ++i) sums.add(i, fill);
      }
      if (q.grad != nullptr && inside)
        for (int r = lo + threadIdx.x; r < hi; r += kThreads) q.grad[r] = fill;
      continue;
    }
    // what is never removed
    Lse rest = {-INFINITY, 0.f};
    for (int j = threadIdx.x; j < n; j += kThreads)
      if (pos[j] == 0) rest = lse_merge(rest, Lse{s[j], 1.f});
#pragma unroll
    for (int off = 16; off > 0; off >>= 1)
      rest = lse_merge(rest, Lse{__shfl_xor_sync(0xffffffffu, rest.m, off),
                                 __shfl_xor_sync(0xffffffffu, rest.s, off)});
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = rest;
    __syncthreads();
    rest = part[0];
    for (int i = 1; i < kThreads / 32; ++i) rest = lse_merge(rest, part[i]);
    // thread i holds steps [c0, c1); L_t from the back
    const int chunk = (k + kThreads - 1) / kThreads;
    const int c0 = min(static_cast<int>(threadIdx.x) * chunk, k), c1 = min(c0 + chunk, k);
    float v[kPerThread];
    Lse left[kPerThread];
    Lse own = {-INFINITY, 0.f};
#pragma unroll
    for (int i = kPerThread - 1; i >= 0; --i)
      if (c0 + i < c1) {
        v[i] = s[seq[c0 + i]];
        own = lse_merge(own, Lse{v[i], 1.f});
      }
    Lse acc = lse_merge(rest, block_scan<false>(own, part));
    double lp = 0.;
    Lse inv = {-INFINITY, 0.f};           // sum of exp(-L_t) over the thread's steps
#pragma unroll
    for (int i = kPerThread - 1; i >= 0; --i)
      if (c0 + i < c1) {
        acc = lse_merge(acc, Lse{v[i], 1.f});
        left[i] = acc;
        lp += (v[i] - acc.m) - logf(acc.s);
        inv = lse_merge(inv, Lse{-acc.m, 1.f / acc.s});
      }
    if (q.grad != nullptr) {
      Lse up = block_scan<true>(inv, part);
#pragma unroll
      for (int i = 0; i < kPerThread; ++i)
        if (c0 + i < c1) {
          up = lse_merge(up, Lse{-left[i].m, 1.f / left[i].s});
          upto[c0 + i] = up;
        }
    }
    lp = block_sum(lp, dpart);            // its barriers publish `upto`
    const float x = p.ref_logp != nullptr ? static_cast<float>(p.ref_logp[img] - lp) : 0.f;
    float loss;
    const float g = row_terms(p, static_cast<float>(lp - p.old_logp[img]), x, p.advantages[img], w,
                              0.f, &loss, threadIdx.x == 0 ? &sums : nullptr);
    if (threadIdx.x == 0) {
      p.logp[img] = static_cast<float>(lp);
      if (p.row_loss != nullptr) p.row_loss[img] = loss;
    }
    if (q.grad == nullptr) continue;
    if (threadIdx.x == 0) q.grad[lo] = 0.f;                                 // CLS
    for (int j = threadIdx.x; j < n; j += kThreads) {
      const int u = pos[j];
      const Lse a = upto[u > 0 ? u - 1 : k - 1];
      q.grad[lo + 1 + j] = g * ((u > 0 ? 1.f : 0.f) - a.s * expf(s[j] + a.m));
    }
  }
  finish_totals(p, sums);
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

// A dependent launch of clusters of `ctas` CTAs.
template <typename T>
int launch_rows(void (*kern)(policy::Rows<T>, policy::Actions), int grid, int block, int ctas,
                cudaStream_t stream, const policy::Rows<T>& r, const policy::Actions& p) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(block);
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

template <typename T, int kHeld>
int launch_blocks(int ctas, cudaStream_t stream, const policy::Rows<T>& r,
                  const policy::Actions& p) {
  const int clusters = grid_for(r.rows, kHeld > 4 ? 2 : 3);   // CTAs that an SM holds
  const int grid = ctas * (clusters * ctas > num_sms() * (kHeld > 4 ? 2 : 3)
                               ? num_sms() * (kHeld > 4 ? 2 : 3) / ctas
                               : clusters);
  switch (ctas) {
    case 1: return launch_rows(policy::policy_block_kernel<T, 512, kHeld, 1>, grid, 512, 1, stream, r, p);
    case 2: return launch_rows(policy::policy_block_kernel<T, 512, kHeld, 2>, grid, 512, 2, stream, r, p);
    case 4: return launch_rows(policy::policy_block_kernel<T, 512, kHeld, 4>, grid, 512, 4, stream, r, p);
    default: return launch_rows(policy::policy_block_kernel<T, 512, kHeld, 8>, grid, 512, 8, stream, r, p);
  }
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
  if (need <= 8)
    return launch_rows(policy::policy_warp_kernel<T, 8, 1>, grid_for((rows + 31) / 32, 8), 256, 1,
                       stream, r, p);
  if (need <= 32)
    return launch_rows(policy::policy_warp_kernel<T, 8, 4>, grid_for((rows + 31) / 32, 8), 256, 1,
                       stream, r, p);
  if (need <= 128)
    return launch_rows(policy::policy_warp_kernel<T, 32, 4>, grid_for((rows + 7) / 8, 8), 256, 1,
                       stream, r, p);
  if (need <= 512)
    return launch_rows(policy::policy_block_kernel<T, 128, 4, 1>, grid_for(rows, 12), 128, 1,
                       stream, r, p);
  if (need > 512 * 8 * 8)
    return launch_rows(policy::policy_long_kernel<T>,
                       policy::kLongCtas * grid_for(rows, 1) > num_sms() * 2
                           ? num_sms() * 2 / policy::kLongCtas * policy::kLongCtas
                           : policy::kLongCtas * rows,
                       policy::kLongBlock, policy::kLongCtas, stream, r, p);
  int ctas = 1;
  while (need > 512 * 8 * ctas) ctas *= 2;
  while (ctas < 8 && rows * ctas * 2 <= num_sms()) ctas *= 2;   // few rows: more SMs a row
  return need <= 512 * 4 * ctas ? launch_blocks<T, 4>(ctas, stream, r, p)
                                : launch_blocks<T, 8>(ctas, stream, r, p);
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
  if (rows < 0 || classes < 1 || ld < classes || dtype < DORA_BF16 || dtype > DORA_F32)
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
  return launched(launch_pdl(policy::pl_policy_loss_kernel, dim3(grid_for(batch, 6)),
                             dim3(policy::kThreads), 0, stream, q, p));
}

}  // extern "C"
