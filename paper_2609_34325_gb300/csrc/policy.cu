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

struct Workspace {
  unsigned ticket;                        // CTAs done; zero between calls
  unsigned pad[63];
  double partial[kMaxCtas][kTerms];
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
  double v[kTerms] = {0., 0., 0., 0., 0., 0.};
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
  sums->v[0] += row;
  sums->v[1] += static_cast<double>(w) * surrogate;
  sums->v[2] += static_cast<double>(w) * kl;
  sums->v[3] += static_cast<double>(w) * h;
  sums->v[4] += inside ? 0.f : w;
  sums->v[5] += w;
  return g * w;
}

// The CTA's sums (held by thread 0) go to its place in the workspace; the CTA that
// is last adds all of them in the order of the CTAs, so that the totals do not
// depend on which one that is, and leaves the ticket at zero for the next call.
__device__ __forceinline__ void finish_totals(const Actions& p, const Sums& sums) {
  if (p.totals == nullptr) return;
  __shared__ bool last;
  Workspace* ws = p.ws;
  if (threadIdx.x == 0) {
#pragma unroll
    for (int i = 0; i < kTerms; ++i) ws->partial[blockIdx.x][i] = sums.v[i];
    __threadfence();
    last = atomicAdd(&ws->ticket, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  for (int i = threadIdx.x >> 5; i < kTerms; i += warps) {
    double t = 0.;
    for (int c = lane; c < static_cast<int>(gridDim.x); c += 32)
      t += __ldcg(&ws->partial[c][i]);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) t += __shfl_xor_sync(0xffffffffu, t, off);
    if (lane == 0) p.totals[i] = static_cast<float>(t);
  }
  if (threadIdx.x == 0) ws->ticket = 0;
}

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void from_float(float v, float* to) { *to = v; }
__device__ __forceinline__ void from_float(float v, __half* to) { *to = __float2half_rn(v); }
__device__ __forceinline__ void from_float(float v, __nv_bfloat16* to) {
  *to = __float2bfloat16_rn(v);
}

__device__ __forceinline__ float block_max(float v, float* scratch) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, off));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
  __syncthreads();
  v = scratch[0];
#pragma unroll
  for (int w = 1; w < kThreads / 32; ++w) v = fmaxf(v, scratch[w]);
  return v;
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
// Categorical actions: one CTA walks the rows; a row is read for its maximum,
// for its sums s = sum e^{z - m} and t = sum e^{z - m} (z - m), and for the
// gradient:  p_j = e^{z_j - m} / s,  H = log s - t / s,
//   d loss / d z_j = g (1(j = a) - p_j) + w c p_j (log p_j + H).
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

template <typename T>
__global__ void __launch_bounds__(kThreads) policy_loss_kernel(Rows<T> r, Actions p) {
  __shared__ float scratch[kThreads / 32];
  pdl_wait();
  Sums sums;
  for (int row = blockIdx.x; row < r.rows; row += gridDim.x) {
    const T* z = r.logits + row * r.ld;
    T* dz = r.grad != nullptr ? r.grad + row * r.ld : nullptr;
    const int action = r.actions[row];
    const float w = p.weights != nullptr ? p.weights[row] : 1.f;
    const int n = r.legal != nullptr ? r.legal[row] : r.classes;
    const bool takes = action >= 0 && w != 0.f;
    const bool bad = takes && (n < 0 || n > r.classes || action >= n);
    if (!takes || bad) {
      const float fill = bad ? NAN : 0.f;
      if (threadIdx.x == 0) {
        if (bad) record_status(r.status, DORA_ERR_DEVICE_BAD_COUNT);
        p.logp[row] = fill;
        if (r.entropy != nullptr) r.entropy[row] = fill;
        if (p.row_loss != nullptr) p.row_loss[row] = fill;
        for (int i = 0; i < kTerms; ++i) sums.v[i] += fill;
      }
      if (dz != nullptr)
        for (int j = threadIdx.x; j < r.classes; j += kThreads) from_float(fill, dz + j);
      continue;
    }
    float m = -INFINITY;
    for (int j = threadIdx.x; j < n; j += kThreads) m = fmaxf(m, to_float(z[j]));
    m = block_max(m, scratch);
    float s = 0.f, t = 0.f;
    for (int j = threadIdx.x; j < n; j += kThreads) {
      const float d = to_float(z[j]) - m;
      const float e = expf(d);
      s += e;
      t = fmaf(e, fmaxf(d, -200.f), t);   // e = 0 at -inf: no 0 * inf
    }
    s = block_sum(s, scratch);
    t = block_sum(t, scratch);
    const float za = to_float(z[action]);
    const float ls = logf(s), h = ls - t / s;
    const float lp = (za - m) - ls;
    const float x = p.ref_logp != nullptr ? p.ref_logp[row] - lp : 0.f;
    float loss;
    const float g = row_terms(p, lp - p.old_logp[row], x, p.advantages[row], w, h, &loss,
                              threadIdx.x == 0 ? &sums : nullptr);
    if (threadIdx.x == 0) {
      p.logp[row] = lp;
      if (r.entropy != nullptr) r.entropy[row] = h;
      if (p.row_loss != nullptr) p.row_loss[row] = loss;
    }
    if (dz == nullptr) continue;
    __syncthreads();                      // the action's logit is read before it is overwritten
    const float cw = w * p.entropy_coef, a = (cw * (h - ls) - g) / s, b = cw / s;
    for (int j = threadIdx.x; j < r.classes; j += kThreads) {
      float v = 0.f;
      if (j < n) {
        const float d = to_float(z[j]) - m;
        v = expf(d) * fmaf(b, fmaxf(d, -200.f), a);
        if (j == action) v += g;
      }
      from_float(v, dz + j);
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
        for (int i = 0; i < kTerms; ++i) sums.v[i] += fill;
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

template <typename T>
int launch_policy(const void* logits, void* grad, int64_t ld, int rows, int classes,
                  const int32_t* legal, const int32_t* actions, float* entropy, int32_t* status,
                  const policy::Actions& p, cudaStream_t stream) {
  policy::Rows<T> r = {static_cast<const T*>(logits), static_cast<T*>(grad), ld, rows, classes,
                       legal, actions, entropy, status};
  return launched(launch_pdl(policy::policy_loss_kernel<T>, dim3(grid_for(rows, 8)),
                             dim3(policy::kThreads), 0, stream, r, p));
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
