// What a rollout takes down of its actions, and the gradient of that: log-probabilities
// of given tokens under softmax(z / T), the entropy, and the most probable alternatives
// (App. A.3's rollouts keep the first of them for the clipped loss).
//
// With m the largest legal logit, d_j = z_j - m, s = sum_j e^{d_j / T} and
// t = sum_j e^{d_j / T} d_j:
//   l = (z_a - m) / T - ln s,   H = ln s - t / (T s),   p_j = e^{d_j / T - ln s};
// and from dl = d loss / d l and dH = d loss / d H, with (m, ln s, H) of the forward:
//   d loss / d z_j = [dl (1(j = a) - p_j) - dH p_j (ln p_j + H)] / T
//                  = p_j (A + B d_j / T) + 1(j = a) dl / T,
//   A = (-dl - dH (H - ln s)) / T,   B = -dH / T.
// The forward reads the legal logits once, the gradient reads them once and writes as many.
// Measured, against what that takes of memory: 2048 x 32000 bf16 with 8 alternatives (15% of the
// rows idle) 33 us of 16, its gradient 43 of 36; 4095 x 50001 fp16 with 5 81 of 57 and 133 of
// 118; fp32, all rows at work, 47 of 39 and 133 of 121.  The gradient is memory's.  The forward
// starts and ends its rows together, all being resident at once, and the ends find the
// alternatives: without them 2048 rows take 26 us, 9728 99 of 92 (with 8 121).
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

// A key into CTA `cta` of the cluster.
__device__ __forceinline__ void store_key_remote(uint64_t v, uint64_t* to, uint32_t cta) {
  asm volatile(
      "{\n\t.reg .b32 ra;\n\t"
      "mapa.shared::cluster.u32 ra, %0, %1;\n\t"
      "st.shared::cluster.u64 [ra], %2;\n\t}" ::"r"(smem_u32(to)),
      "r"(cta), "l"(v)
      : "memory");
}

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

// (z - m) / T - ln s.  By halves: two finite logits may be further apart than 32 bits hold.
__device__ __forceinline__ float log_prob(float z, float m, float inv_t, float ls) {
  return fmaf(0.5f * z - 0.5f * m, 2.f * inv_t, -ls);
}

// The scalars of a row; returns ln s.
__device__ __forceinline__ float write_row(const Outputs& o, int row, const Part& x, float za,
                                           bool has_token, float inv_t, bool leader) {
  const float ls = logf(x.s);
  if (leader) {
    if (o.logp != nullptr) o.logp[row] = has_token ? log_prob(za, x.m, inv_t, ls) : 0.f;
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
// thread knows the largest logit m_i of its granules from the softmax' sums, and leaves the
// largest of every few of them.  With tau at or below the top-th largest m_i, all that is
// wanted is at or above tau, and lies in the few granules whose largest logit is: they are read
// again.  (All granules of the threads with m_i >= tau, instead: 8 alternatives of 2048 x 32000
// bf16 took 6.7 us beside the sums' 28.)  What is at or above tau is put in order by counting,
// for each, those before it.  Where too much is (many equal logits), the order is
// found by one look at the row for each alternative.
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
  int o[kPer], most = ordered(-INFINITY), least = 0x7FFFFFFF;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    o[i] = ordered(m[i]);
    most = max(most, o[i]);
    least = min(least, o[i]);
  }
  // all are at or above the least one
  int lo = top <= 32 * kPer ? __reduce_min_sync(0xffffffffu, least) : ordered(-INFINITY);
  int hi = __reduce_max_sync(0xffffffffu, most);
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

// Puts the found keys in order, `mine` of them for each of `lanes` lanes, and writes the row's
// alternatives; equal keys there are none.
__device__ __forceinline__ void write_top(const Outputs& o, int64_t at, const uint64_t* keys,
                                          int found, int lane, int lanes, float m, float inv_t,
                                          float ls) {
  for (int i = lane; i < found; i += lanes) {
    const uint64_t key = keys[i];
    int before = 0;
    for (int c = 0; c < found; ++c) before += keys[c] > key;
    if (before < o.top) {
      o.top_logp[at + before] = log_prob(value_of(key), m, inv_t, ls);
      o.top_tokens[at + before] = index_of(key);
    }
  }
  for (int i = found + lane; i < o.top; i += lanes) {
    o.top_logp[at + i] = -INFINITY;
    o.top_tokens[at + i] = -1;
  }
}
// A row that is not finite has no order.
__device__ __forceinline__ void write_no_top(const Outputs& o, int64_t at, int lane, int lanes) {
  for (int i = lane; i < o.top; i += lanes) {
    o.top_logp[at + i] = NAN;
    o.top_tokens[at + i] = -1;
  }
}
__device__ __forceinline__ uint64_t warp_largest(uint64_t key) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    const uint64_t other = __shfl_xor_sync(0xffffffffu, key, off);
    key = other > key ? other : key;
  }
  return key;
}
// The keys of granule i that are at or above tau, to `keep`.
template <typename T, typename F>
__device__ __forceinline__ void for_candidates(uint4 q, int first, float tau, F keep) {
  constexpr int kE = Granule<T>::kElems;
  if (!(Granule<T>::largest(q) >= tau)) return;   // most have none
  float v[kE];
  Granule<T>::unpack(q, v);
#pragma unroll
  for (int e = 0; e < kE; ++e)
    if (v[e] >= tau && v[e] > -INFINITY) keep(key_of(v[e], first + e));
}
// The largest key of granule i below `last`, or `best`.
template <typename T>
__device__ __forceinline__ uint64_t largest_below(uint4 q, int first, uint64_t last,
                                                  uint64_t best) {
  for_candidates<T>(q, first, -INFINITY, [&](uint64_t key) {
    if (key < last && key > best) best = key;
  });
  return best;
}

// Short rows: a warp holds one, kHeld granules a lane; no barrier.  256 rows of 96 fp32 logits
// take 9 us in a call, the host's time.
template <typename T, int kHeld>
__global__ void __launch_bounds__(kThreads) logprob_warp_kernel(Batch<T> b, Outputs o) {
  constexpr int kE = Granule<T>::kElems, kKeys = 128;
  __shared__ uint64_t all_keys[kWarps][kKeys];
  __shared__ int n_keys[kWarps];
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint64_t* keys = all_keys[warp];
  const float scale = b.inv_t * policy::kLog2e;
  const int step = gridDim.x * kWarps;
  for (int row = blockIdx.x * kWarps + warp; row < b.rows; row += step) {
    const RowUse use = row_use(b, row);
    if (use.kind != kComputed) {
      fill_row(o, row, use.kind == kNone ? 0.f : NAN, lane, 32, b.status);
      continue;
    }
    const int n = use.n;
    const RowPtr<T> z(b.logits + row * b.ld, n);
    uint4 q[kHeld];
#pragma unroll
    for (int u = 0; u < kHeld; ++u) q[u] = z.load(lane + 32 * u, n);
    float za = 0.f;
    if (use.token >= 0) za = to_float(z.z[use.token]);
    RowSum x;
    x.clear();
    constexpr int kStep = kHeld < 4 ? kHeld : 4;
#pragma unroll
    for (int u = 0; u < kHeld; u += kStep) {
      uint4 some[kStep];
#pragma unroll
      for (int v = 0; v < kStep; ++v) some[v] = q[u + v];
      if (kHeld <= 4 || 32 * u < z.some_hi) x.add<T>(some, scale);
    }
    const Part part = x.over(32, scale);
    const float ls = write_row(o, row, part, za, use.token >= 0, b.inv_t, lane == 0);
    if (o.top == 0) continue;
    const int64_t at = static_cast<int64_t>(row) * o.top;
    if (!isfinite(ls)) {
      write_no_top(o, at, lane, 32);
      continue;
    }
    const float mine[1] = {x.m};
    const float tau = threshold<1>(mine, o.top);
    if (lane == 0) n_keys[warp] = 0;
    __syncwarp();
    // few lanes have any: read again, so that the others' registers are not held
    if (x.m >= tau && x.m > -INFINITY)
#pragma unroll 1
      for (int i = lane; i < z.some_hi; i += 32)
        for_candidates<T>(z.load(i, n), i * kE - z.mis, tau, [&](uint64_t key) {
          const int c = atomicAdd(&n_keys[warp], 1);
          if (c < kKeys) keys[c] = key;
        });
    __syncwarp();
    int found = n_keys[warp];
    if (found > kKeys) {                  // many equal logits: one by one
      uint64_t last = ~0ull;
      __syncwarp();
      for (found = 0; found < o.top; ++found) {
        uint64_t best = 0;
#pragma unroll 1
        for (int i = lane; i < z.some_hi; i += 32)
          best = largest_below<T>(z.load(i, n), i * kE - z.mis, last, best);
        last = warp_largest(best);
        if (last == 0) break;
        if (lane == 0) keys[found] = last;
      }
      __syncwarp();
    }
    write_top(o, at, keys, found, lane, 32, part.m, b.inv_t, ls);
    __syncwarp();
  }
}

// Longer rows: a CTA for each, or a cluster of kCtas, an equal part of its granules each, dealt
// out to the threads in turn; the next granules are on their way while some are added.
template <typename T, int kBlock, int kCtas>
__global__ void __launch_bounds__(kBlock, 1024 / kBlock)
    logprob_cta_kernel(Batch<T> b, Outputs o) {
  constexpr int kE = Granule<T>::kElems, kW = kBlock / 32, kU = 4;
  constexpr int kKeys = kCtas > 1 ? 64 : 256;   // of a CTA
  constexpr int kSlots = 16, kHits = 2 * kKeys;
  __shared__ Part slots[kW], parts[kCtas];
  __shared__ float maxima[kBlock], tau_at, some[kSlots][kBlock];
  __shared__ int hits[kHits], n_hits, n_keys, found_in[kCtas];
  __shared__ uint64_t keys[kCtas * kKeys], best[kW];
  const int me = threadIdx.x, warp = me >> 5, lane = me & 31;
  const int rank = kCtas > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const float scale = b.inv_t * policy::kLog2e;
  const int row = blockIdx.x / kCtas;
  if (me == 0) n_hits = n_keys = 0;
  if (kCtas > 1) cluster_sync();          // the others are there to be written to
  pdl_wait();
  const RowUse use = row_use(b, row);
  if (use.kind != kComputed) {
    if (rank == 0) fill_row(o, row, use.kind == kNone ? 0.f : NAN, me, kBlock, b.status);
    return;
  }
  const int n = use.n;
  const RowPtr<T> z(b.logits + row * b.ld, n);
  const int each = (z.some_hi + kCtas - 1) / kCtas;
  const int lo = rank * each, hi = min(lo + each, z.some_hi);
  const auto load = [&](int i) { return z.load(i < hi ? i : z.some_hi, n); };
  uint4 q[kU];
#pragma unroll
  for (int u = 0; u < kU; ++u) q[u] = load(lo + me + u * kBlock);
  float za = 0.f;
  if (me == 0 && use.token >= 0) za = to_float(z.z[use.token]);
  RowSum x;
  x.clear();
  // the largest logit of every kU << shift of a thread's granules to a slot of its own
  int shift = 0, batch = 0;
  while (((each + kU * kBlock - 1) / (kU * kBlock) - 1) >> shift >= kSlots) ++shift;
  float largest = -INFINITY;
  for (int i = lo + me; i < hi; i += kU * kBlock, ++batch) {
    uint4 next[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) next[u] = load(i + (kU + u) * kBlock);
    x.add<T>(q, scale);
    if (o.top > 0) {
#pragma unroll
      for (int u = 0; u < kU; ++u) largest = fmaxf(largest, Granule<T>::largest(q[u]));
      some[batch >> shift][me] = largest;
      if (((batch + 1) & ((1 << shift) - 1)) == 0) largest = -INFINITY;
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) q[u] = next[u];
  }
  Part part = x.over(32, scale);
  if (lane == 0) slots[warp] = part;
  maxima[me] = x.m;
  __syncthreads();
  part = policy::join_parts<kW>(slots, scale);
  if (kCtas > 1) {
    if (me < kCtas) policy::store_part_remote(part, &parts[rank], me);
  }
  const int64_t at = static_cast<int64_t>(row) * o.top;
  if (o.top > 0) {
    if (warp == 0) {
      float m[kW];
#pragma unroll
      for (int i = 0; i < kW; ++i) m[i] = maxima[lane + 32 * i];
      const float t = threshold<kW>(m, o.top);
      if (lane == 0) tau_at = t;
    }
    __syncthreads();
    const float tau = tau_at;
    if (x.m >= tau && x.m > -INFINITY)
      for (int k = 0; k << shift < batch; ++k)
        if (some[k][me] >= tau) {
          const int h = atomicAdd(&n_hits, 1);
          if (h < kHits) hits[h] = k * kBlock + me;
        }
    __syncthreads();
    const int n_hit = n_hits, log = 2 + shift;   // granules of a hit
    static_assert(kU == 4, "two bits of an index into them");
    if (n_hit <= kHits)
      for (int w = me; w < n_hit << log; w += kBlock) {
        const int hit = hits[w >> log], in = w & ((1 << log) - 1);
        const int i = lo + hit % kBlock + ((hit / kBlock << log) + in) * kBlock;
        if (i < hi)
          for_candidates<T>(z.load(i, n), i * kE - z.mis, tau, [&](uint64_t key) {
            const int c = atomicAdd(&n_keys, 1);
            if (c < kKeys) keys[rank * kKeys + c] = key;
          });
      }
    __syncthreads();
    int found = n_keys;
    if (found > kKeys || n_hit > kHits) {   // many equal logits: one by one
      uint64_t last = ~0ull;
      __syncthreads();
      for (found = 0; found < o.top; ++found) {
        uint64_t mine = 0;
        for (int i = lo + me; i < hi; i += kBlock)
          mine = largest_below<T>(z.load(i, n), i * kE - z.mis, last, mine);
        mine = warp_largest(mine);
        if (lane == 0) best[warp] = mine;
        __syncthreads();
        last = best[0];
#pragma unroll
        for (int w = 1; w < kW; ++w) last = best[w] > last ? best[w] : last;
        __syncthreads();
        if (last == 0) break;
        if (me == 0) keys[rank * kKeys + found] = last;
      }
      __syncthreads();
    }
    if (kCtas > 1) {                    // to the first CTA
      if (rank != 0)
        for (int i = me; i < found; i += kBlock)
          store_key_remote(keys[rank * kKeys + i], &keys[rank * kKeys + i], 0);
      if (me == 0) store_remote(found, &found_in[rank], 0);
    } else if (me == 0) {
      found_in[0] = found;
    }
  }
  if (kCtas > 1) cluster_sync();        // the parts and the keys have arrived
  else if (o.top > 0) __syncthreads();
  if (rank == 0) {
    if (kCtas > 1) part = policy::join_parts<kCtas>(parts, scale);
    const float ls = write_row(o, row, part, za, use.token >= 0, b.inv_t, me == 0);
    if (o.top > 0) {
      if (!isfinite(ls)) {
        write_no_top(o, at, me, kBlock);
      } else {
        int found = found_in[0];
        if (kCtas > 1) {                // close the gaps between the CTAs' keys
          found = 0;
          for (int c = 0; c < kCtas; ++c) {
            const int some = found_in[c];
            uint64_t key = 0;
            if (me < some) key = keys[c * kKeys + me];
            __syncthreads();
            if (me < some) keys[found + me] = key;
            found += some;
          }
          __syncthreads();
        }
        write_top(o, at, keys, found, me, kBlock, part.m, b.inv_t, ls);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// The gradient: one look at every granule, nothing to wait for; memory (6.0 TB/s of a copy's 6.8).
// ---------------------------------------------------------------------------
constexpr float kLn2 = 0.6931471805599453f;
// At or below this power of two, whatever the row (its shift is 0 or more), p is 0, and so are
// p a and p b y, with no infinity to make a NaN of them.
constexpr float kLeast = -512.f;

template <typename T>
struct GradIn {
  const float* norm;                      // [rows, 2]
  const float* entropy;                   // nullable, with dentropy
  const float* dlogp;                     // nullable
  const float* dentropy;                  // nullable
  T* grad;
};

struct RowGrad {
  float m, shift, a, b, at_token;         // 2^{y - shift} (a + b y) (+ at_token), y = scale d
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
  return {norm.x, norm.y * policy::kLog2e, a * b.inv_t, -dh * b.inv_t * kLn2, dl * b.inv_t};
}

template <typename T>
__device__ __forceinline__ uint4 grad_granule(uint4 q, const RowGrad& k, float scale, int token) {
  constexpr int kE = Granule<T>::kElems;
  float d[kE];
  policy::differences<T>(q, -k.m, d);
#pragma unroll
  for (int e = 0; e < kE; ++e) {
    const float y = fmaxf(d[e] * scale, kLeast);
    float v = policy::ex2(y - k.shift) * fmaf(k.b, y, k.a);
    if (e == token) v += k.at_token;
    d[e] = v;
  }
  return Granule<T>::pack(d);
}

// A row, or kUnit granules of one: kU granules for each of kLanes lanes, all loaded before the
// first is computed.  Rows of up to 128 granules are a warp's; longer ones are cut, and the units
// dealt out in turn.
constexpr int kUnit = 4 * kThreads;

template <typename T, int kLanes, int kU>
__global__ void __launch_bounds__(kThreads, 4)
    logprob_grad_kernel(Batch<T> b, GradIn<T> g, int64_t units, int a_row) {
  constexpr int kE = Granule<T>::kElems, kTeams = kThreads / kLanes;
  pdl_wait();
  const int me = threadIdx.x % kLanes;
  const float scale = b.inv_t * policy::kLog2e;
  const int64_t step = static_cast<int64_t>(gridDim.x) * kTeams;
  for (int64_t unit = static_cast<int64_t>(blockIdx.x) * kTeams + threadIdx.x / kLanes;
       unit < units; unit += step) {
    const int row = a_row == 1 ? static_cast<int>(unit) : static_cast<int>(unit / a_row);
    const int first = a_row == 1 ? 0 : static_cast<int>(unit - static_cast<int64_t>(row) * a_row) *
                                           (kU * kLanes);
    const RowUse use = row_use(b, row);
    const bool live = use.kind == kComputed;
    const int n = live ? use.n : 0;
    const RowPtr<T> z(b.logits + row * b.ld, n);
    uint4 q[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) q[u] = z.load(first + me + u * kLanes, n);
    T* dz = g.grad + row * b.ld;
    const bool aligned = policy::same_alignment(dz, z.z);
    const int end = z.granules(b.classes);
    if (live) {
      const RowGrad k = row_grad(b, g, row);
      const int at = use.token + z.mis;   // of the token among the granules' elements
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int i = first + me + u * kLanes;
        if (i >= end) continue;
        const uint4 v = grad_granule<T>(q[u], k, scale, use.token >= 0 ? at - i * kE : -1);
        if (aligned && z.whole(i)) *(z.as_granules(dz) + i) = v;
        else z.store_part(dz, aligned, i, n, b.classes, v);
      }
    } else {
      if (use.kind == kInvalid && me == 0 && first == 0)
        record_status(b.status, DORA_ERR_DEVICE_BAD_COUNT);
      float v[kE];
#pragma unroll
      for (int e = 0; e < kE; ++e) v[e] = use.kind == kInvalid ? NAN : 0.f;
      const uint4 fill = Granule<T>::pack(v);
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int i = first + me + u * kLanes;
        if (i < end) z.store_part(dz, aligned, i, b.classes, b.classes, fill);
      }
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
  // Below 1e18 a difference at policy::kFloor, which stands for all larger ones, has an
  // exponential of 0; above 1e-18 one over the temperature leaves room for the gradients.
  if (!(temperature >= 1e-18f && temperature <= 1e18f)) return false;
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

template <typename T, int kBlock, int kCtas>
int launch_rows(const logprob::Batch<T>& b, const logprob::Outputs& o, int teams,
                cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (kCtas > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = kCtas;
    attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
    ++n;
  }
  if (pdl_enabled()) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  cfg.gridDim = dim3(teams * kCtas);
  cfg.blockDim = dim3(kBlock);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = n;
  return launched(cudaLaunchKernelEx(&cfg, logprob::logprob_cta_kernel<T, kBlock, kCtas>, b, o));
}

template <typename T>
int launch_logprob(const logprob::Batch<T>& b, const logprob::Outputs& o, cudaStream_t stream) {
  // granules that a row may touch
  const int64_t need = (b.classes + 2 * Granule<T>::kElems - 2) / Granule<T>::kElems;
  const int sms = num_sms(), eights = grid_for((b.rows + 7) / 8, 8);
  const auto warps = [&](auto kern) {
    return launched(launch_pdl(kern, dim3(eights), dim3(logprob::kThreads), 0, stream, b, o));
  };
  if (need <= 32) return warps(logprob::logprob_warp_kernel<T, 1>);
  if (need <= 128) return warps(logprob::logprob_warp_kernel<T, 4>);
  if (need <= 256 && b.rows > 8 * sms) return warps(logprob::logprob_warp_kernel<T, 8>);
  // A CTA a row, the smaller the more rows there are: rows are put in order behind barriers, and
  // of many small CTAs others are adding meanwhile (2048 x 32000 bf16, 8 alternatives: 64
  // threads 32.3 us, 128 33.2, 256 39.5; 4095 x 50001 fp16 80.6, 85.1, 96.7).  Few rows get
  // several CTAs.
  if (b.rows >= 8 * sms) return launch_rows<T, 64, 1>(b, o, b.rows, stream);
  if (b.rows >= 4 * sms) return launch_rows<T, 128, 1>(b, o, b.rows, stream);
  int ctas = 1;
  while (ctas < 8 && b.rows * ctas <= sms && need > 512 * ctas) ctas *= 2;
  switch (ctas) {
    case 1: return launch_rows<T, 256, 1>(b, o, b.rows, stream);
    case 2: return launch_rows<T, 256, 2>(b, o, b.rows, stream);
    case 4: return launch_rows<T, 256, 4>(b, o, b.rows, stream);
    default: return launch_rows<T, 256, 8>(b, o, b.rows, stream);
  }
}

template <typename T>
int launch_grad(const logprob::Batch<T>& b, const logprob::GradIn<T>& g, cudaStream_t stream) {
  const int64_t need = (b.classes + 2 * Granule<T>::kElems - 2) / Granule<T>::kElems;
  const int64_t most = num_sms() * 8;
  const auto run = [&](auto kern, int64_t units, int a_row, int teams) {
    const int64_t ctas = (units + teams - 1) / teams;
    return launched(launch_pdl(kern, dim3(static_cast<unsigned>(ctas < most ? ctas : most)),
                               dim3(logprob::kThreads), 0, stream, b, g, units, a_row));
  };
  if (need <= 32) return run(logprob::logprob_grad_kernel<T, 32, 1>, b.rows, 1, 8);
  if (need <= 128) return run(logprob::logprob_grad_kernel<T, 32, 4>, b.rows, 1, 8);
  const int64_t a_row = (need + logprob::kUnit - 1) / logprob::kUnit;
  return run(logprob::logprob_grad_kernel<T, 256, 4>, b.rows * a_row, static_cast<int>(a_row), 1);
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
