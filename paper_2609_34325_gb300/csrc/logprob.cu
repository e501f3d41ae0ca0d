// What a rollout takes down of its actions, and the gradient of that: log-probabilities
// of given tokens under softmax(z / T), the entropy, and the most probable alternatives
// (App. A.3's rollouts keep the first of them for the clipped loss).
//
// With m the largest legal logit, d_j = z_j - m, s = sum_j e^{d_j / T} and
// t = sum_j e^{d_j / T} d_j:
//   l = (z_a - m) / T - ln s,   H = ln s - t / (T s),   p_j = e^{d_j / T - ln s};
// and from dl = d loss / d l and dH = d loss / d H, with (m, ln s, H) of the forward:
//   d loss / d z_j = [dl (1(j = a) - p_j) - dH p_j (ln p_j + H)] / T
//                  = p_j (A + B d_j) + 1(j = a) dl / T,
//   A = (-dl - dH (H - ln s)) / T,   B = -dH / T^2.
// Both are bound by memory: the forward reads the legal logits once, the gradient reads
// them once and writes as many.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "dora.h"
#include "dora_ptx.cuh"
#include "granule.cuh"
#include "logit_rows.cuh"
#include "token_ops.cuh"
#include "update_ptx.cuh"

namespace dora {
namespace logprob {

using policy::Part;
using policy::RowPtr;
using policy::RowSum;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxTop = 32;
constexpr int kCandidates = 256;

// A batch of rows; T is their type.
template <typename T>
struct Batch {
  const T* logits;
  int64_t ld;
  int rows, classes;
  const int32_t* legal;                   // nullable: classes
  const int32_t* tokens;                  // nullable: rows without tokens, all take part
  float inv_t;
  int32_t* status;
};

// Whether a row is computed, has no part (its outputs are 0) or is not valid (NaN).
enum RowKind { kNone, kInvalid, kComputed };
struct RowUse {
  RowKind kind;
  int token, n;                           // token -1: the row has none
};
template <typename T>
__device__ __forceinline__ RowUse row_use(const Batch<T>& b, int row) {
  const int token = b.tokens != nullptr ? b.tokens[row] : -1;
  const int n = b.legal != nullptr ? b.legal[row] : b.classes;
  if (b.tokens != nullptr && token < 0) return {kNone, -1, 0};
  if (n < 0 || n > b.classes || token >= n) {
    if (b.tokens == nullptr && n == 0) return {kNone, -1, 0};
    return {kInvalid, -1, 0};
  }
  return {n > 0 ? kComputed : kNone, token, n};
}

struct Outputs {
  float* logp;                            // nullable where there are no tokens
  float* entropy;                         // nullable
  float* norm;                            // nullable, [rows, 2]: m and ln s
  int top;                                // alternatives wanted
  float* top_logp;                        // [rows, top]
  int32_t* top_tokens;
};

// The scalars of a row; returns ln s.
__device__ __forceinline__ float write_row(const Outputs& o, int row, const Part& x, float za,
                                           bool has_token, float inv_t, bool leader) {
  const float ls = logf(x.s);
  if (leader) {
    if (o.logp != nullptr) o.logp[row] = has_token ? fmaf(za - x.m, inv_t, -ls) : 0.f;
    if (o.entropy != nullptr) o.entropy[row] = fmaf(-x.t / x.s, inv_t, ls);
    if (o.norm != nullptr) {
      const bool fine = isfinite(ls);     // not where all logits are -inf, or one is NaN or +inf
      o.norm[2 * static_cast<int64_t>(row)] = fine ? x.m : NAN;
      o.norm[2 * static_cast<int64_t>(row) + 1] = fine ? ls : NAN;
    }
  }
  return ls;
}
// The outputs of a row that has no part (0) or is not valid (NaN), by `lanes` lanes.
__device__ __forceinline__ void fill_row(const Outputs& o, int row, float fill, int lane,
                                         int lanes, int32_t* status) {
  if (lane == 0) {
    if (fill != 0.f) record_status(status, DORA_ERR_DEVICE_BAD_COUNT);
    if (o.logp != nullptr) o.logp[row] = fill;
    if (o.entropy != nullptr) o.entropy[row] = fill;
    if (o.norm != nullptr)
      o.norm[2 * static_cast<int64_t>(row)] = o.norm[2 * static_cast<int64_t>(row) + 1] = fill;
  }
  for (int i = lane; i < o.top; i += lanes) {
    o.top_logp[static_cast<int64_t>(row) * o.top + i] = fill == 0.f ? -INFINITY : fill;
    o.top_tokens[static_cast<int64_t>(row) * o.top + i] = -1;
  }
}

// ---------------------------------------------------------------------------
// The alternatives: the `top` largest logits above -inf, equal ones by index.  Every
// thread knows the largest logit m_i of its granules from the softmax' sums.  With
// tau at or below the top-th largest m_i, all that is wanted is at or above tau, and only
// threads with m_i >= tau (a few more than `top`) own any of it: their granules are read
// again, a warp each.  What is at or above tau is put in order by counting, for each, those
// before it.  Where too much is (many equal logits), the order is found by one look at the
// row for each alternative.
// ---------------------------------------------------------------------------

// Ordered like the values (-0 as 0), for comparisons of integers.
__device__ __forceinline__ int ordered(float v) {
  const int bits = __float_as_int(v + 0.f);
  return bits ^ ((bits >> 31) & 0x7FFFFFFF);
}
__device__ __forceinline__ float unordered(int o) {
  return __int_as_float(o ^ ((o >> 31) & 0x7FFFFFFF));
}
// Larger for what comes first: the value, then the lower index.
__device__ __forceinline__ uint64_t key_of(float v, int index) {
  return (static_cast<uint64_t>(static_cast<uint32_t>(ordered(v)) ^ 0x80000000u) << 32) |
         (0xFFFFFFFFu - static_cast<uint32_t>(index));
}
__device__ __forceinline__ float value_of(uint64_t key) {
  return unordered(static_cast<int>(static_cast<uint32_t>(key >> 32) ^ 0x80000000u));
}
__device__ __forceinline__ int index_of(uint64_t key) {
  return static_cast<int>(0xFFFFFFFFu - static_cast<uint32_t>(key));
}

// A value such that at least `top` of a warp's kPer values a lane are at or above it, not
// many more if the values differ; -inf where there are not as many above -inf.
template <int kPer>
__device__ __forceinline__ float threshold(const float (&m)[kPer], int top) {
  int o[kPer], most = ordered(-INFINITY);
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    o[i] = ordered(m[i]);
    most = max(most, o[i]);
  }
  int lo = ordered(-INFINITY), hi = __reduce_max_sync(0xffffffffu, most);
  const int enough = top + top / 4 + 2;
  // at or above lo: enough; the search ends there, or where the two meet
  while (lo < hi) {
    const int mid = lo + static_cast<int>((static_cast<unsigned>(hi) - lo + 1) >> 1);
    int c = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) c += o[i] >= mid;
    c = __reduce_add_sync(0xffffffffu, c);
    if (c >= top) {
      lo = mid;
      if (c <= enough) break;
    } else {
      hi = mid - 1;
    }
  }
  return unordered(lo);
}

// A CTA a row, its granules dealt out to the threads in turn.
template <typename T>
__global__ void __launch_bounds__(kThreads, 4) logprob_cta_kernel(Batch<T> b, Outputs o) {
  constexpr int kE = Granule<T>::kElems, kU = 4;
  __shared__ Part slots[kWarps];
  __shared__ float maxima[kThreads], tau_at;
  __shared__ int owners[kThreads], n_owners, n_candidates;
  __shared__ uint64_t candidates[kCandidates], best[kWarps];
  pdl_wait();
  const int me = threadIdx.x, warp = me >> 5, lane = me & 31;
  const float scale = b.inv_t * policy::kLog2e;
  for (int row = blockIdx.x; row < b.rows; row += gridDim.x) {
    const RowUse use = row_use(b, row);
    if (use.kind != kComputed) {
      fill_row(o, row, use.kind == kNone ? 0.f : NAN, me, kThreads, b.status);
      continue;
    }
    const int n = use.n;
    const RowPtr<T> z(b.logits + row * b.ld, n);
    float za = 0.f;
    if (me == 0 && use.token >= 0) za = to_float(z.z[use.token]);
    RowSum x;
    x.clear();
    for (int i = me; i < z.some_hi; i += kU * kThreads) {
      uint4 q[kU];
#pragma unroll
      for (int u = 0; u < kU; ++u) q[u] = z.load(i + u * kThreads, n);
      x.add<T>(q, scale);
    }
    Part part = x.over(32, scale);
    if (lane == 0) slots[warp] = part;
    maxima[me] = x.m;
    if (me == 0) n_owners = n_candidates = 0;
    __syncthreads();
    part = policy::join_parts<kWarps>(slots, scale);
    const float ls = write_row(o, row, part, za, use.token >= 0, b.inv_t, me == 0);
    if (o.top > 0) {
      const int64_t at = static_cast<int64_t>(row) * o.top;
      if (!isfinite(ls)) {                // a row that is not finite has no order
        for (int i = me; i < o.top; i += kThreads) {
          o.top_logp[at + i] = NAN;
          o.top_tokens[at + i] = -1;
        }
      } else {
        if (warp == 0) {
          float m[kWarps];
#pragma unroll
          for (int i = 0; i < kWarps; ++i) m[i] = maxima[lane + 32 * i];
          const float t = threshold<kWarps>(m, o.top);
          if (lane == 0) tau_at = t;
        }
        __syncthreads();
        const float tau = tau_at;
        if (x.m >= tau && x.m > -INFINITY) owners[atomicAdd(&n_owners, 1)] = me;
        __syncthreads();
        const int own = n_owners;
        for (int w = warp; w < own; w += kWarps)
          for (int i = owners[w] + lane * kThreads; i < z.some_hi; i += 32 * kThreads) {
            float v[kE];
            Granule<T>::unpack(z.load(i, n), v);
#pragma unroll
            for (int e = 0; e < kE; ++e)
              if (v[e] >= tau && v[e] > -INFINITY) {
                const int c = atomicAdd(&n_candidates, 1);
                if (c < kCandidates) candidates[c] = key_of(v[e], i * kE - z.mis + e);
              }
          }
        __syncthreads();
        const int found = n_candidates;
        if (found <= kCandidates) {
          if (me < found) {
            const uint64_t key = candidates[me];
            int before = 0;
            for (int c = 0; c < found; ++c) before += candidates[c] > key;
            if (before < o.top) {
              o.top_logp[at + before] = fmaf(value_of(key) - part.m, b.inv_t, -ls);
              o.top_tokens[at + before] = index_of(key);
            }
          }
          if (me >= found && me < o.top) {
            o.top_logp[at + me] = -INFINITY;
            o.top_tokens[at + me] = -1;
          }
        } else {
          uint64_t last = ~0ull;
          for (int rank = 0; rank < o.top; ++rank) {
            uint64_t mine = 0;
            for (int i = me; i < z.some_hi; i += kThreads) {
              float v[kE];
              Granule<T>::unpack(z.load(i, n), v);
#pragma unroll
              for (int e = 0; e < kE; ++e) {
                const uint64_t key = v[e] > -INFINITY ? key_of(v[e], i * kE - z.mis + e) : 0;
                if (key < last && key > mine) mine = key;
              }
            }
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) {
              const uint64_t other = __shfl_xor_sync(0xffffffffu, mine, off);
              mine = other > mine ? other : mine;
            }
            if (lane == 0) best[warp] = mine;
            __syncthreads();
            mine = best[0];
#pragma unroll
            for (int w = 1; w < kWarps; ++w) mine = best[w] > mine ? best[w] : mine;
            __syncthreads();
            if (me == 0) {
              o.top_logp[at + rank] =
                  mine != 0 ? fmaf(value_of(mine) - part.m, b.inv_t, -ls) : -INFINITY;
              o.top_tokens[at + rank] = mine != 0 ? index_of(mine) : -1;
            }
            last = mine;
          }
        }
      }
    }
    __syncthreads();                      // the shared places are free for the next row
  }
}

// ---------------------------------------------------------------------------
// The gradient: one look at every granule, nothing to wait for.
// ---------------------------------------------------------------------------
template <typename T>
struct GradIn {
  const float* norm;                      // [rows, 2]
  const float* entropy;                   // nullable, with dentropy
  const float* dlogp;                     // nullable
  const float* dentropy;                  // nullable
  T* grad;
};

struct RowGrad {
  float m, shift, a, b, at_token;         // e^{scale d - shift} (a + b d) (+ at_token)
};

template <typename T>
__device__ __forceinline__ RowGrad row_grad(const Batch<T>& b, const GradIn<T>& g, int row) {
  const float2 norm = reinterpret_cast<const float2*>(g.norm)[row];
  const float dl = g.dlogp != nullptr ? g.dlogp[row] : 0.f;
  float a = -dl, dh = 0.f;
  if (g.dentropy != nullptr) {
    dh = g.dentropy[row];
    a = fmaf(-dh, g.entropy[row] - norm.y, a);
  }
  return {norm.x, norm.y * policy::kLog2e, a * b.inv_t, -dh * b.inv_t * b.inv_t, dl * b.inv_t};
}

template <typename T>
__device__ __forceinline__ uint4 grad_granule(uint4 q, const RowGrad& k, float scale, int token) {
  constexpr int kE = Granule<T>::kElems;
  float d[kE];
  policy::differences<T>(q, -k.m, d);
#pragma unroll
  for (int e = 0; e < kE; ++e) {
    const float p = policy::ex2(fmaf(d[e], scale, -k.shift));
    float v = p * fmaf(k.b, fmaxf(d[e], policy::kFloor), k.a);
    if (e == token) v += k.at_token;
    d[e] = v;
  }
  return Granule<T>::pack(d);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) logprob_grad_kernel(Batch<T> b, GradIn<T> g) {
  constexpr int kE = Granule<T>::kElems;
  pdl_wait();
  const int me = threadIdx.x;
  const float scale = b.inv_t * policy::kLog2e;
  for (int row = blockIdx.x; row < b.rows; row += gridDim.x) {
    const RowUse use = row_use(b, row);
    const int n = use.kind == kComputed ? use.n : 0;
    const RowPtr<T> z(b.logits + row * b.ld, n);
    T* dz = g.grad + row * b.ld;
    const bool aligned = policy::same_alignment(dz, z.z);
    const int end = z.granules(b.classes);
    if (use.kind != kComputed) {
      if (use.kind == kInvalid && me == 0) record_status(b.status, DORA_ERR_DEVICE_BAD_COUNT);
      float v[kE];
#pragma unroll
      for (int e = 0; e < kE; ++e) v[e] = use.kind == kInvalid ? NAN : 0.f;
      const uint4 q = Granule<T>::pack(v);
      for (int i = me; i < end; i += kThreads)
        z.store_part(dz, aligned, i, b.classes, b.classes, q);
      continue;
    }
    const RowGrad k = row_grad(b, g, row);
    const int at = use.token + z.mis;     // of the token among the granules' elements
    for (int i = me; i < end; i += kThreads) {
      const int token = use.token >= 0 ? at - i * kE : -1;
      const uint4 v = grad_granule<T>(z.load(i, n), k, scale, token);
      if (aligned && z.whole(i)) *(z.as_granules(dz) + i) = v;
      else z.store_part(dz, aligned, i, n, b.classes, v);
    }
  }
}

}  // namespace logprob
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

// The checks that both entry points make.
bool valid_batch(const void* logits, int32_t dtype, int32_t rows, int32_t classes, int64_t ld,
                 float temperature) {
  // rows and granules are counted in 32 bits, with room for a step past the last
  if (rows < 0 || rows > (1 << 30) || classes < 1 || classes > (1 << 30) || ld < classes ||
      dtype < DORA_BF16 || dtype > DORA_F32)
    return false;
  if (!(temperature > 0.f) || !isfinite(temperature) || !isfinite(1.f / temperature)) return false;
  return rows == 0 || (logits != nullptr && (reinterpret_cast<uintptr_t>(logits) &
                                             (dtype == DORA_F32 ? 3u : 1u)) == 0);
}

int grid_for(int rows, int per_sm) {
  const int most = num_sms() * per_sm;
  return rows < most ? rows : most;
}

template <typename T>
logprob::Batch<T> batch_of(const void* logits, int32_t rows, int32_t classes, int64_t ld,
                           const int32_t* legal, const int32_t* tokens, float temperature,
                           int32_t* status) {
  return {static_cast<const T*>(logits), ld, rows, classes, legal, tokens, 1.f / temperature,
          status};
}

template <typename T>
int launch_logprob(const logprob::Batch<T>& b, const logprob::Outputs& o, cudaStream_t stream) {
  return launched(launch_pdl(logprob::logprob_cta_kernel<T>, dim3(grid_for(b.rows, 4)),
                             dim3(logprob::kThreads), 0, stream, b, o));
}

template <typename T>
int launch_grad(const logprob::Batch<T>& b, const logprob::GradIn<T>& g, cudaStream_t stream) {
  return launched(launch_pdl(logprob::logprob_grad_kernel<T>, dim3(grid_for(b.rows, 8)),
                             dim3(logprob::kThreads), 0, stream, b, g));
}
}  // namespace

extern "C" {

int dora_token_logprob(const void* logits, int32_t dtype, int32_t rows, int32_t classes,
                       int64_t ld, const int32_t* legal, const int32_t* tokens,
                       float temperature, int32_t top, float* logp, float* entropy, float* norm,
                       float* top_logp, int32_t* top_tokens, int32_t* status,
                       dora_stream_t stream_) {
  if (!valid_batch(logits, dtype, rows, classes, ld, temperature) || top < 0 ||
      top > logprob::kMaxTop)
    return DORA_ERR_INVALID_ARG;
  if (rows > 0 && ((tokens == nullptr) != (logp == nullptr) ||
                   (top > 0 && (top_logp == nullptr || top_tokens == nullptr))))
    return DORA_ERR_INVALID_ARG;
  const int e = device_or_error();
  if (e != DORA_OK || rows == 0) return e;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  const logprob::Outputs o = {logp, entropy, norm, top, top_logp, top_tokens};
  if (dtype == DORA_BF16)
    return launch_logprob(batch_of<__nv_bfloat16>(logits, rows, classes, ld, legal, tokens,
                                                  temperature, status), o, stream);
  if (dtype == DORA_F16)
    return launch_logprob(batch_of<__half>(logits, rows, classes, ld, legal, tokens, temperature,
                                           status), o, stream);
  return launch_logprob(batch_of<float>(logits, rows, classes, ld, legal, tokens, temperature,
                                        status), o, stream);
}

int dora_token_logprob_grad(const void* logits, int32_t dtype, int32_t rows, int32_t classes,
                            int64_t ld, const int32_t* legal, const int32_t* tokens,
                            float temperature, const float* norm, const float* entropy,
                            const float* dlogp, const float* dentropy, void* grad,
                            int32_t* status, dora_stream_t stream_) {
  if (!valid_batch(logits, dtype, rows, classes, ld, temperature)) return DORA_ERR_INVALID_ARG;
  if (rows > 0 && (norm == nullptr || (reinterpret_cast<uintptr_t>(norm) & 7u) != 0 ||
                   grad == nullptr || (dlogp == nullptr && dentropy == nullptr) ||
                   (dlogp != nullptr && tokens == nullptr) ||
                   (dentropy != nullptr && entropy == nullptr) ||
                   (reinterpret_cast<uintptr_t>(grad) & (dtype == DORA_F32 ? 3u : 1u)) != 0))
    return DORA_ERR_INVALID_ARG;
  const int e = device_or_error();
  if (e != DORA_OK || rows == 0) return e;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  if (dtype == DORA_BF16)
    return launch_grad(batch_of<__nv_bfloat16>(logits, rows, classes, ld, legal, tokens,
                                               temperature, status),
                       logprob::GradIn<__nv_bfloat16>{norm, entropy, dlogp, dentropy,
                                                      static_cast<__nv_bfloat16*>(grad)}, stream);
  if (dtype == DORA_F16)
    return launch_grad(batch_of<__half>(logits, rows, classes, ld, legal, tokens, temperature,
                                        status),
                       logprob::GradIn<__half>{norm, entropy, dlogp, dentropy,
                                               static_cast<__half*>(grad)}, stream);
  return launch_grad(batch_of<float>(logits, rows, classes, ld, legal, tokens, temperature,
                                     status),
                     logprob::GradIn<float>{norm, entropy, dlogp, dentropy,
                                            static_cast<float*>(grad)}, stream);
}

}  // extern "C"
