// The end of a policy update, over all tensors of a parameter list in one launch
// each: the global gradient norm, clipping by it, and an Adam step (App. D.2,
// Table 4) that takes the clipping factor as it reads the gradients.
//
// The list lives on the device: one entry per tensor, and the tensors cut into
// units of kUnit elements that are dealt out evenly as spans of consecutive
// units, whatever the tensors' sizes.  A CTA walks its span, piece by piece.  To
// begin a tensor costs a CTA about as long as kBegin units take (its entry, then its
// first values: two round trips to memory), and counts as that many: a hundred
// vectors in a row would otherwise be one CTA's, while the others wait for it (norm of
// 86 M parameters, the vectors last: 75 us without, 39 with 6 units, 32 with 12).  A
// list with no more units than spans has a unit a span, and nothing to count.
//
// All three are bound by memory: 86 M fp32 gradients are normed in 54 us (6.4 TB/s; a
// copy 6.8) and clipped in 162 (three passes, 6.4 TB/s); an Adam step on 86 M fp32
// weights, bf16 gradients and bf16 copies takes 384 after a norm of 32 (6.2 TB/s).  Lists
// of a few hundred KB take the time of their chain (launch, span, values, sums, ticket):
// 5 us for the norm, 8 with clipping, 10 for norm and step.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "dora.h"
#include "dora_ptx.cuh"
#include "granule.cuh"
#include "token_ops.cuh"
#include "update_ptx.cuh"

namespace dora {
namespace optim {

constexpr int kThreads = 256;
constexpr int kUnit = 2048;               // elements
constexpr int kBegin = 12;                // units, in lists of more than kMaxSpans
constexpr int kCtasPerSm = 4;             // resident, by their registers
constexpr int kMaxSpans = 152 * kCtasPerSm;   // a span a CTA, all at once
constexpr int kFill = 48;                 // entries written by one launch, passed by value

struct Entry {
  const void* grad;
  void* clipped;                          // null: in place
  void* param;
  float *m, *v;
  uint16_t* copy;                         // nullable, bf16
  int64_t n;
  int64_t first_unit;                     // of its elements; `begin` units before belong to it
  int32_t begin;
  int32_t grad_type, param_type, pad;
};

// Units [unit, unit_end) of the whole list, from tensor `tensor` to `last_tensor`,
// with those tensors' entries, so that a CTA reads where to begin in one load.
struct Span {
  int64_t unit, unit_end;
  int32_t tensor, last_tensor;
  Entry first, last;
};

// A CTA's sum of squares: fp32, and what did not fit its range in 64 bits.
struct Partial {
  float sum;
  int has_wide;                           // fp64 comparisons are as slow as the sums
  double wide;
};

struct Header {
  unsigned ticket;                        // CTAs done; zero between calls
  unsigned pad[63];
  Partial partial[kMaxSpans];
};

struct List {
  Header* header;
  Entry* entries;
  Span* spans;
  int count, n_spans;
};

struct FillArgs {
  Entry e[kFill];
};

__global__ void fill_entries_kernel(Header* header, Entry* entries, int first, int count,
                                    FillArgs args) {
  pdl_wait();
  if (first == 0 && threadIdx.x == 0) header->ticket = 0;
  if (threadIdx.x < count) entries[first + threadIdx.x] = args.e[threadIdx.x];
}

// The last tensor that starts at or before a unit (the one that holds it: tensors
// without elements start where the next one does).
__device__ __forceinline__ int tensor_of(const List& list, int64_t unit) {
  int lo = 0, hi = list.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (list.entries[mid].first_unit - list.entries[mid].begin <= unit) lo = mid; else hi = mid - 1;
  }
  return lo;
}

__global__ void fill_spans_kernel(List list, int64_t units) {
  pdl_wait();
  const int b = blockIdx.x * blockDim.x + threadIdx.x;
  if (b >= list.n_spans) return;
  Span s;
  s.unit = units * b / list.n_spans;
  s.unit_end = units * (b + 1) / list.n_spans;
  s.tensor = tensor_of(list, s.unit);
  s.last_tensor = s.unit_end > s.unit ? tensor_of(list, s.unit_end - 1) : s.tensor;
  s.first = list.entries[s.tensor];
  s.last = list.entries[s.last_tensor];
  list.spans[b] = s;
}

// f(entry, first element, elements) for every piece of the span, from its first to
// its last tensor, or the other way round.  The entry stays in memory, and a piece
// has at most kPiece elements, counted in 32 bits: both leave registers to the data.
constexpr int kPiece = 1 << 28;

template <bool kForward, typename F>
__device__ __forceinline__ void for_pieces(const List& list, int span, F f) {
  const Span* s = list.spans + span;
  const int64_t unit = s->unit, end = s->unit_end;
  if (unit >= end) return;
  int tensor = kForward ? s->tensor : s->last_tensor;
  const int stop = kForward ? s->last_tensor : s->tensor;
  const Entry* e = kForward ? &s->first : &s->last;
  while (true) {
    const int64_t n = e->n, first_unit = e->first_unit;
    int64_t from = unit > first_unit ? (unit - first_unit) * kUnit : 0;
    int64_t to = (end - first_unit) * kUnit;
    to = to < n ? to : n;
    while (to > from) {
      const int some = to - from < kPiece ? static_cast<int>(to - from) : kPiece;
      f(*e, kForward ? from : to - some, some);
      if (kForward) from += some; else to -= some;
    }
    if (tensor == stop) return;
    tensor += kForward ? 1 : -1;
    e = list.entries + tensor;
  }
}

// A tensor's type is looked at where its values are unpacked or packed, not by a
// loop for each type: the loads in flight are the same for all, and one loop leaves
// them their registers (three types times three in Adam's took 255, or spilled).
__device__ __forceinline__ int size_of(int type) { return type == DORA_F32 ? 4 : 2; }
__device__ __forceinline__ const char* at_elem(const void* p, int type, int64_t i) {
  return static_cast<const char*>(p) + i * size_of(type);
}
__device__ __forceinline__ char* at_elem(void* p, int type, int64_t i) {
  return static_cast<char*>(p) + i * size_of(type);
}
__device__ __forceinline__ float load_one(const void* p, int type, int i) {
  if (type == DORA_F32) return static_cast<const float*>(p)[i];
  if (type == DORA_BF16) return to_float(static_cast<const __nv_bfloat16*>(p)[i]);
  return to_float(static_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ void store_one(float v, void* p, int type, int i) {
  if (type == DORA_F32) static_cast<float*>(p)[i] = v;
  else if (type == DORA_BF16) from_float(v, static_cast<__nv_bfloat16*>(p) + i);
  else from_float(v, static_cast<__half*>(p) + i);
}

// Elements before the first 16-byte boundary (at most n).
__device__ __forceinline__ int head_of(const void* p, int type, int n) {
  const int h = static_cast<int>((16u - (reinterpret_cast<uintptr_t>(p) & 15u)) & 15u) /
                size_of(type);
  return h < n ? h : n;
}

// ---------------------------------------------------------------------------
// Norm.  Squares are summed in 32 bits over the elements that a thread has at
// hand at once; a thread carries the sums on in a pair of fp32 values, the second
// what the first lost (Knuth's two-sum: six additions where an fp64 one takes the
// warp 16 cycles or more).  A CTA's threads are joined by a tree of fp32 additions
// (of positive values: a few 2^-24 of the sum, half of that on the norm), the CTAs
// in pairs again.  A sum out of the middle of the range (gradients above about 1e11
// or below 1e-16) is taken again, and joined, in 64 bits.
// ---------------------------------------------------------------------------
constexpr float kSquaresLow = 1e-30f, kSquaresHigh = 1e25f;

struct SumOfSquares {
  float sum, lost;
  int has_wide;
  double wide;
  __device__ __forceinline__ bool add(float x) {         // false: out of range
    if (!(x > kSquaresLow && x < kSquaresHigh)) return false;
    const float t = sum + x, b = t - sum;
    lost += (sum - (t - b)) + (x - b);
    sum = t;
    return true;
  }
  __device__ __forceinline__ void add_wide(double x) {
    has_wide = 1;
    wide += x;
  }
  __device__ __forceinline__ void add_one(float v) {
    if (!add(v * v) && v != 0.f) add_wide(static_cast<double>(v) * v);
  }
};

template <typename T>
__device__ __forceinline__ void add_squares(uint4 q, float* a, float* b) {
  float v[Granule<T>::kElems];
  Granule<T>::unpack(q, v);
#pragma unroll
  for (int k = 0; k < Granule<T>::kElems; k += 2) {
    *a = fmaf(v[k], v[k], *a);
    *b = fmaf(v[k + 1], v[k + 1], *b);
  }
}

template <typename T>
__device__ __forceinline__ double wide_squares(uint4 q) {
  float v[Granule<T>::kElems];
  Granule<T>::unpack(q, v);
  double t = 0.;
#pragma unroll
  for (int k = 0; k < Granule<T>::kElems; ++k) t += static_cast<double>(v[k]) * v[k];
  return t;
}

// A second pass over the values begins at the spans' ends (below).  So that L2 still has
// them, what lies more than kKeep bytes before a piece's end is read to be evicted first
// (clip of 344 MB fp32 168 us, 162 with it; 600 MB bf16 292 and 284; shorter lists, and
// a step after the norm, are as fast).
constexpr int kKeep = 150 << 10;          // of 608 spans: 91 MB

__device__ __forceinline__ uint64_t evict_first() {
  uint64_t policy;
  asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
  return policy;
}
__device__ __forceinline__ uint64_t evict_normal() {
  uint64_t policy;
  asm("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));
  return policy;
}
__device__ __forceinline__ uint4 load_as(const uint4* p, uint64_t policy) {
  uint4 q;
  asm volatile("ld.global.L2::cache_hint.v4.u32 {%0, %1, %2, %3}, [%4], %5;"
               : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w)
               : "l"(p), "l"(policy)
               : "memory");
  return q;
}

__device__ __forceinline__ void piece_squares(const void* p, int type, int n, SumOfSquares* acc) {
  constexpr int kInFlight = 8;
  const int elems = 16 / size_of(type);
  const int head = head_of(p, type, n);
  const int granules = (n - head) / elems, tail = head + granules * elems;
  if (threadIdx.x < head) acc->add_one(load_one(p, type, threadIdx.x));
  if (tail + threadIdx.x < n) acc->add_one(load_one(p, type, tail + threadIdx.x));
  const uint4* g = reinterpret_cast<const uint4*>(at_elem(p, type, head));
  const uint64_t once = evict_first(), again = evict_normal();
  for (int i = threadIdx.x; i < granules; i += kInFlight * kThreads) {
    const uint64_t policy = granules - i > kKeep / 16 ? once : again;
    uint4 q[kInFlight];
#pragma unroll
    for (int u = 0; u < kInFlight; ++u)
      q[u] = i + u * kThreads < granules ? load_as(g + i + u * kThreads, policy)
                                           : make_uint4(0, 0, 0, 0);
    float a = 0.f, b = 0.f;
    if (type == DORA_F32) {
#pragma unroll
      for (int u = 0; u < kInFlight; ++u) add_squares<float>(q[u], &a, &b);
    } else if (type == DORA_BF16) {
#pragma unroll
      for (int u = 0; u < kInFlight; ++u) add_squares<__nv_bfloat16>(q[u], &a, &b);
    } else {
#pragma unroll
      for (int u = 0; u < kInFlight; ++u) add_squares<__half>(q[u], &a, &b);
    }
    if (!acc->add(a + b)) {
#pragma unroll
      for (int u = 0; u < kInFlight; ++u)
        if ((q[u].x | q[u].y | q[u].z | q[u].w) != 0)
          acc->add_wide(type == DORA_F32    ? wide_squares<float>(q[u])
                        : type == DORA_BF16 ? wide_squares<__nv_bfloat16>(q[u])
                                            : wide_squares<__half>(q[u]));
    }
  }
}

// The sum over the block of what its threads summed, in thread 0.  fp32 in a tree: a
// few roundings of values in the middle of the range; 64 bits, slow here, only for
// what left it.
__device__ __forceinline__ Partial block_sum(const SumOfSquares& mine, Partial* scratch) {
  float f = mine.sum + mine.lost;
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) f += __shfl_xor_sync(0xffffffffu, f, off);
  const int has_wide = __any_sync(0xffffffffu, mine.has_wide);
  double wide = 0.;
  if (has_wide) {
    wide = mine.wide;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) wide += __shfl_xor_sync(0xffffffffu, wide, off);
  }
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = Partial{f, has_wide, wide};
  __syncthreads();
  Partial all = scratch[0];
  if (threadIdx.x == 0)
#pragma unroll
    for (int w = 1; w < kThreads / 32; ++w) {
      all.sum += scratch[w].sum;
      if (scratch[w].has_wide) {
        all.has_wide = 1;
        all.wide += scratch[w].wide;
      }
    }
  return all;
}

// out[0] = the norm, out[1] = min(1, max_norm / norm), 1 for a norm that is not finite.
__device__ __forceinline__ void write_norm(const Partial& all, float max_norm, float* out) {
  float norm = sqrtf(all.sum);
  if (all.has_wide) norm = static_cast<float>(sqrt(all.wide + all.sum));
  out[0] = norm;
  out[1] = isfinite(norm) && norm > max_norm ? max_norm / norm : 1.f;
}

// The CTA that is last adds the spans' sums in their order.
__global__ void __launch_bounds__(kThreads, kCtasPerSm)
    grad_norm_kernel(List list, float max_norm, float* __restrict__ out) {
  __shared__ Partial scratch[kThreads / 32];
  __shared__ bool last;
  pdl_wait();
  SumOfSquares mine = {0.f, 0.f, 0, 0.};
  for_pieces<true>(list, blockIdx.x, [&](const Entry& e, int64_t from, int n) {
    piece_squares(at_elem(e.grad, e.grad_type, from), e.grad_type, n, &mine);
  });
  const Partial cta = block_sum(mine, scratch);
  if (gridDim.x == 1) {
    if (threadIdx.x == 0) write_norm(cta, max_norm, out);
    return;
  }
  if (threadIdx.x == 0) {
    list.header->partial[blockIdx.x] = cta;
    last = take_ticket(&list.header->ticket) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  constexpr int kLoads = (kMaxSpans + kThreads - 1) / kThreads;
  int4 x[kLoads];                         // all on their way before the first is added
#pragma unroll
  for (int u = 0; u < kLoads; ++u) {
    const int b = threadIdx.x + u * kThreads;
    x[u] = b < static_cast<int>(gridDim.x)
               ? __ldcg(reinterpret_cast<const int4*>(&list.header->partial[b]))
               : make_int4(0, 0, 0, 0);
  }
  mine = SumOfSquares{0.f, 0.f, 0, 0.};
#pragma unroll
  for (int u = 0; u < kLoads; ++u) {
    const float f = __int_as_float(x[u].x);
    if (!mine.add(f) && f != 0.f) mine.add_wide(f);
    if (x[u].y) mine.add_wide(__hiloint2double(x[u].w, x[u].z));
  }
  const Partial all = block_sum(mine, scratch);
  if (threadIdx.x == 0) {
    write_norm(all, max_norm, out);
    list.header->ticket = 0;
  }
}

// ---------------------------------------------------------------------------
// Clipping.  A norm that is not finite leaves the gradients as they are.  Spans
// are walked from their ends, which the norm has read last and L2 may still hold
// (67 MB of fp32 28.7 us, 32.3 from the beginnings; 344 MB 162, of which
// three passes at the copy rate are 152).
// ---------------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ uint4 scaled(uint4 q, float f) {
  float v[Granule<T>::kElems];
  Granule<T>::unpack(q, v);
#pragma unroll
  for (int k = 0; k < Granule<T>::kElems; ++k) v[k] *= f;
  return Granule<T>::pack(v);
}

__device__ __forceinline__ void piece_scale(const void* p, void* y, int type, int n, float f) {
  constexpr int kInFlight = 8;
  if ((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(y)) & 15u) {
    for (int i = threadIdx.x; i < n; i += kThreads) store_one(load_one(p, type, i) * f, y, type, i);
    return;
  }
  const int elems = 16 / size_of(type);
  const int head = head_of(p, type, n);
  const int granules = (n - head) / elems, tail = head + granules * elems;
  if (threadIdx.x < head)
    store_one(load_one(p, type, threadIdx.x) * f, y, type, threadIdx.x);
  if (tail + threadIdx.x < n)
    store_one(load_one(p, type, tail + threadIdx.x) * f, y, type, tail + threadIdx.x);
  const uint4* g = reinterpret_cast<const uint4*>(at_elem(p, type, head));
  uint4* o = reinterpret_cast<uint4*>(at_elem(y, type, head));
  for (int i = granules - 1 - static_cast<int>(threadIdx.x); i >= 0; i -= kInFlight * kThreads) {
    uint4 q[kInFlight];
#pragma unroll
    for (int u = 0; u < kInFlight; ++u)
      if (i >= u * kThreads) q[u] = g[i - u * kThreads];
#pragma unroll
    for (int u = 0; u < kInFlight; ++u)
      if (i >= u * kThreads)
        o[i - u * kThreads] = type == DORA_F32    ? scaled<float>(q[u], f)
                              : type == DORA_BF16 ? scaled<__nv_bfloat16>(q[u], f)
                                                  : scaled<__half>(q[u], f);
  }
}

__global__ void __launch_bounds__(kThreads, kCtasPerSm)
    scale_grads_kernel(List list, const float* __restrict__ norm) {
  pdl_wait();
  const float f = isfinite(norm[0]) ? norm[1] : 1.f;
  for_pieces<false>(list, blockIdx.x, [&](const Entry& e, int64_t from, int n) {
    void* to = e.clipped != nullptr ? e.clipped : const_cast<void*>(e.grad);
    if (to == e.grad && f == 1.f) return;
    piece_scale(at_elem(e.grad, e.grad_type, from), at_elem(to, e.grad_type, from), e.grad_type, n,
                f);
  });
}

// ---------------------------------------------------------------------------
// Adam.  The powers beta^t are carried in 64 bits from step to step by the CTA
// that is last, so that a captured step counts on when it is replayed.
// ---------------------------------------------------------------------------
struct AdamState {
  int64_t step;                           // steps taken
  double power1, power2;                  // beta1^step, beta2^step
  unsigned ticket;
  unsigned pad[9];
};
static_assert(sizeof(AdamState) == 64, "the state's size is part of the interface");

struct AdamArgs {
  AdamState* state;
  const float* clip;                      // nullable: norm and factor
  double beta1, beta2;
  float b1, omb1, b2, omb2;               // beta, 1 - beta
  float lr, keep, eps;                    // keep = 1 - lr decay
};

struct AdamStep {
  float f, step_size, root_scale;         // factor, lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
};

__device__ __forceinline__ void adam_one(const AdamArgs& a, const AdamStep& s, float g, float* p,
                                         float* m, float* v) {
  const float d = g * s.f;
  *m = fmaf(a.b1, *m, a.omb1 * d);
  *v = fmaf(a.b2, *v, a.omb2 * (d * d));
  *p = fmaf(*p, a.keep, -(s.step_size * *m) / fmaf(sqrtf(*v), s.root_scale, a.eps));
}

// Four elements at an address that is a multiple of their size: 16 bytes of fp32, 8
// (in x and y) of the others.
__device__ __forceinline__ uint4 load_quad(const void* p, int type, int i) {
  if (type == DORA_F32) return static_cast<const uint4*>(p)[i];
  const uint2 q = static_cast<const uint2*>(p)[i];
  return make_uint4(q.x, q.y, 0u, 0u);
}
template <typename T>
__device__ __forceinline__ void unpack_half_granule(uint4 q, float* v) {
  float w[Granule<T>::kElems];
  Granule<T>::unpack(q, w);
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = w[k];
}
__device__ __forceinline__ void unpack_quad(uint4 q, int type, float* v) {
  if (type == DORA_F32) Granule<float>::unpack(q, v);
  else if (type == DORA_BF16) unpack_half_granule<__nv_bfloat16>(q, v);
  else unpack_half_granule<__half>(q, v);
}
template <typename T>
__device__ __forceinline__ uint2 pack_half_granule(const float* v) {
  return make_uint2(Granule<T>::pair(v[0], v[1]), Granule<T>::pair(v[2], v[3]));
}
__device__ __forceinline__ void store_quad(const float* v, void* p, int type, int i) {
  if (type == DORA_F32) static_cast<uint4*>(p)[i] = Granule<float>::pack(v);
  else static_cast<uint2*>(p)[i] = type == DORA_BF16 ? pack_half_granule<__nv_bfloat16>(v)
                                                     : pack_half_granule<__half>(v);
}
__device__ __forceinline__ bool has_quads(const void* p, int type) {
  return (reinterpret_cast<uintptr_t>(p) & (4 * size_of(type) - 1)) == 0;
}

__device__ __forceinline__ void piece_adam(const AdamArgs& a, const AdamStep& s, const Entry& e,
                                           int64_t from, int n) {
  constexpr int kInFlight = 2;
  const int gt = e.grad_type, pt = e.param_type;
  const void* g = at_elem(e.grad, gt, from);
  void* p = at_elem(e.param, pt, from);
  float *m = e.m + from, *v = e.v + from;
  uint16_t* c = e.copy != nullptr ? e.copy + from : nullptr;
  // Whole quads where the buffers agree on where they lie: those of one flat buffer each,
  // or of the framework's allocator, do, whatever the tensors' sizes.
  const int misplaced = static_cast<int>(reinterpret_cast<uintptr_t>(p) / size_of(pt) & 3u);
  const int head = min(n, (4 - misplaced) & 3);
  int first = 0, done = 0;
  if (has_quads(at_elem(g, gt, head), gt) && has_quads(m + head, DORA_F32) &&
      has_quads(v + head, DORA_F32) && (c == nullptr || has_quads(c + head, DORA_BF16))) {
    first = head;
    const int quads = (n - head) / 4;
    done = head + quads * 4;
    const void* gq = at_elem(g, gt, head);
    void* pq = at_elem(p, pt, head);
    float *mq = m + head, *vq = v + head;
    uint16_t* cq = c != nullptr ? c + head : nullptr;
    for (int i = quads - 1 - static_cast<int>(threadIdx.x); i >= 0; i -= kInFlight * kThreads) {
      uint4 qp[kInFlight], qg[kInFlight], qm[kInFlight], qv[kInFlight];
#pragma unroll
      for (int u = 0; u < kInFlight; ++u)
        if (i >= u * kThreads) {
          qg[u] = load_quad(gq, gt, i - u * kThreads);
          qp[u] = load_quad(pq, pt, i - u * kThreads);
          qm[u] = load_quad(mq, DORA_F32, i - u * kThreads);
          qv[u] = load_quad(vq, DORA_F32, i - u * kThreads);
        }
#pragma unroll
      for (int u = 0; u < kInFlight; ++u)
        if (i >= u * kThreads) {
          float fp[4], fg[4], fm[4], fv[4];
          unpack_quad(qp[u], pt, fp);
          unpack_quad(qg[u], gt, fg);
          unpack_quad(qm[u], DORA_F32, fm);
          unpack_quad(qv[u], DORA_F32, fv);
#pragma unroll
          for (int k = 0; k < 4; ++k) adam_one(a, s, fg[k], fp + k, fm + k, fv + k);
          store_quad(fp, pq, pt, i - u * kThreads);
          store_quad(fm, mq, DORA_F32, i - u * kThreads);
          store_quad(fv, vq, DORA_F32, i - u * kThreads);
          if (cq != nullptr) store_quad(fp, cq, DORA_BF16, i - u * kThreads);
        }
    }
  }
  // the rest by elements: the head, then what is past the quads (all of it where the
  // buffers do not agree)
  for (int k = threadIdx.x; k < first + n - done; k += kThreads) {
    const int i = k < first ? k : k - first + done;
    float pi = load_one(p, pt, i), mi = m[i], vi = v[i];
    adam_one(a, s, load_one(g, gt, i), &pi, &mi, &vi);
    store_one(pi, p, pt, i);
    m[i] = mi;
    v[i] = vi;
    if (c != nullptr) store_one(pi, c, DORA_BF16, i);
  }
}

__global__ void __launch_bounds__(kThreads, kCtasPerSm) adam_step_kernel(List list, AdamArgs a) {
  pdl_wait();
  const AdamState st = *a.state;
  AdamStep s = {1.f, 0.f, 0.f};
  bool skip = false;
  if (a.clip != nullptr) {
    skip = !isfinite(a.clip[0]);
    s.f = a.clip[1];
  }
  // fp64 for one thread: for all of them it would take the CTA longer than a small tensor
  __shared__ float scales[2];
  double p1 = 0., p2 = 0.;
  if (threadIdx.x == 0) {
    p1 = (st.step > 0 ? st.power1 : 1.) * a.beta1;
    p2 = (st.step > 0 ? st.power2 : 1.) * a.beta2;
    scales[0] = a.lr / static_cast<float>(1. - p1);
    scales[1] = 1.f / sqrtf(static_cast<float>(1. - p2));
  }
  __syncthreads();
  s.step_size = scales[0];
  s.root_scale = scales[1];
  if (!skip)
    for_pieces<false>(list, blockIdx.x, [&](const Entry& e, int64_t from, int n) {
      piece_adam(a, s, e, from, n);
    });
  __syncthreads();                        // every thread of the CTA has read the state
  if (threadIdx.x == 0) {
    if (take_ticket(&a.state->ticket) == gridDim.x - 1) {
      if (!skip) {
        a.state->step = st.step + 1;
        a.state->power1 = p1;
        a.state->power2 = p2;
      }
      a.state->ticket = 0;
    }
  }
}

__global__ void adam_init_kernel(AdamState* state, int64_t step, double power1, double power2) {
  pdl_wait();
  *state = AdamState{step, power1, power2, 0u, {}};
}

}  // namespace optim
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

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

bool aligned_to(const void* p, int32_t dtype) {
  return (reinterpret_cast<uintptr_t>(p) & (dtype == DORA_F32 ? 3u : 1u)) == 0;
}

bool known_type(int32_t t) { return t >= DORA_BF16 && t <= DORA_F32; }

int64_t units_of(int64_t n) { return (n + optim::kUnit - 1) / optim::kUnit; }

// The units that a tensor's begin counts for in a list of so many, and all of them.
struct Layout {
  int begin, spans;
  int64_t units;
};
Layout layout_of(int64_t units, int64_t tensors) {
  if (units <= optim::kMaxSpans) return {0, units > 0 ? static_cast<int>(units) : 1, units};
  return {optim::kBegin, optim::kMaxSpans, units + tensors * optim::kBegin};
}

// Checks the tensors and counts their units, elements and those that are not empty;
// false when one is not valid.
bool count_units(const dora_param* params, int32_t count, Layout* out, int64_t* elements,
                 bool* has_params) {
  int64_t units = 0, tensors = 0;
  *elements = 0;
  *has_params = true;
  for (int32_t i = 0; i < count; ++i) {
    const dora_param& t = params[i];
    if (t.n < 0 || t.n > (int64_t{1} << 40) || !known_type(t.grad_dtype)) return false;
    if (t.n > 0 && (t.grad == nullptr || !aligned_to(t.grad, t.grad_dtype) ||
                    !aligned_to(t.clipped, t.grad_dtype)))
      return false;
    const int given = (t.param != nullptr) + (t.exp_avg != nullptr) + (t.exp_avg_sq != nullptr);
    if (t.n > 0 && given != 0 && given != 3) return false;
    if (t.n > 0 && given == 0) *has_params = false;
    if (given == 3 && (!known_type(t.param_dtype) || !aligned_to(t.param, t.param_dtype) ||
                       !aligned_to(t.exp_avg, DORA_F32) || !aligned_to(t.exp_avg_sq, DORA_F32) ||
                       !aligned_to(t.copy, DORA_BF16)))
      return false;
    units += units_of(t.n);
    tensors += t.n > 0;
    *elements += t.n;
  }
  *out = layout_of(units, tensors);
  return true;
}

optim::List layout(void* data, int count, int spans) {
  char* p = static_cast<char*>(data);
  optim::List l;
  l.header = reinterpret_cast<optim::Header*>(p);
  p += round256(sizeof(optim::Header));
  l.entries = reinterpret_cast<optim::Entry*>(p);
  p += round256(static_cast<size_t>(count) * sizeof(optim::Entry));
  l.spans = reinterpret_cast<optim::Span*>(p);
  l.count = count;
  l.n_spans = spans;
  return l;
}

bool valid_list(const dora_param_list* list) {
  return list != nullptr && list->data != nullptr && list->count >= 1 && list->spans >= 1 &&
         list->spans <= optim::kMaxSpans;
}
}  // namespace

extern "C" {

size_t dora_param_list_size(const dora_param* params, int32_t count) {
  if (params == nullptr || count < 1) return 0;
  int64_t elements;
  bool has_params;
  Layout plan;
  if (!count_units(params, count, &plan, &elements, &has_params)) return 0;
  return round256(sizeof(optim::Header)) +
         round256(static_cast<size_t>(count) * sizeof(optim::Entry)) +
         round256(static_cast<size_t>(plan.spans) * sizeof(optim::Span));
}

int dora_param_list_prepare(const dora_param* params, int32_t count, void* data, size_t bytes,
                            dora_param_list* list, dora_stream_t stream_) {
  if (params == nullptr || count < 1 || data == nullptr || list == nullptr ||
      (reinterpret_cast<uintptr_t>(data) & 255u) != 0)
    return DORA_ERR_INVALID_ARG;
  int64_t elements;
  bool has_params;
  Layout plan;
  if (!count_units(params, count, &plan, &elements, &has_params) ||
      bytes < dora_param_list_size(params, count))
    return DORA_ERR_INVALID_ARG;
  const int e = device_or_error();
  if (e != DORA_OK) return e;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  const optim::List l = layout(data, count, plan.spans);
  int64_t unit = 0;
  for (int32_t first = 0; first < count; first += optim::kFill) {
    const int some = count - first < optim::kFill ? count - first : optim::kFill;
    optim::FillArgs args = {};
    for (int i = 0; i < some; ++i) {
      const dora_param& t = params[first + i];
      const int begin = t.n > 0 ? plan.begin : 0;
      args.e[i] = optim::Entry{t.grad, t.clipped, t.param, t.exp_avg, t.exp_avg_sq, t.copy, t.n,
                               unit + begin, begin, t.grad_dtype, t.param_dtype, 0};
      unit += begin + units_of(t.n);
    }
    const int rc = launched(launch_pdl(optim::fill_entries_kernel, dim3(1), dim3(optim::kFill), 0,
                                       stream, l.header, l.entries, first, some, args));
    if (rc != DORA_OK) return rc;
  }
  const int rc = launched(launch_pdl(optim::fill_spans_kernel, dim3((l.n_spans + 127) / 128),
                                     dim3(128), 0, stream, l, plan.units));
  if (rc != DORA_OK) return rc;
  *list = dora_param_list{data, elements, count, l.n_spans, has_params ? 1 : 0};
  return DORA_OK;
}

int dora_grad_norm(const dora_param_list* list, float max_norm, float* norm,
                   dora_stream_t stream) {
  if (!valid_list(list) || norm == nullptr || !(max_norm >= 0.f)) return DORA_ERR_INVALID_ARG;
  const int e = device_or_error();
  if (e != DORA_OK) return e;
  const optim::List l = layout(list->data, list->count, list->spans);
  return launched(launch_pdl(optim::grad_norm_kernel, dim3(l.n_spans), dim3(optim::kThreads), 0,
                             reinterpret_cast<cudaStream_t>(stream), l, max_norm, norm));
}

int dora_clip_grads(const dora_param_list* list, float max_norm, float* norm,
                    dora_stream_t stream) {
  const int e = dora_grad_norm(list, max_norm, norm, stream);
  if (e != DORA_OK) return e;
  const optim::List l = layout(list->data, list->count, list->spans);
  return launched(launch_pdl(optim::scale_grads_kernel, dim3(l.n_spans), dim3(optim::kThreads), 0,
                             reinterpret_cast<cudaStream_t>(stream), l, norm));
}

size_t dora_adam_state_size(void) { return sizeof(optim::AdamState); }

int dora_adam_init(void* state, int64_t step, double beta1, double beta2, dora_stream_t stream) {
  if (state == nullptr || (reinterpret_cast<uintptr_t>(state) & 15u) != 0 || step < 0 ||
      !(beta1 >= 0. && beta1 < 1.) || !(beta2 >= 0. && beta2 < 1.))
    return DORA_ERR_INVALID_ARG;
  const int e = device_or_error();
  if (e != DORA_OK) return e;
  return launched(launch_pdl(optim::adam_init_kernel, dim3(1), dim3(1), 0,
                             reinterpret_cast<cudaStream_t>(stream),
                             static_cast<optim::AdamState*>(state), step,
                             pow(beta1, static_cast<double>(step)),
                             pow(beta2, static_cast<double>(step))));
}

int dora_adam_step(const dora_param_list* list, void* state, double lr, double beta1, double beta2,
                   double eps, double weight_decay, const float* clip, dora_stream_t stream) {
  if (!valid_list(list) || list->has_params == 0 || state == nullptr ||
      (reinterpret_cast<uintptr_t>(state) & 15u) != 0)
    return DORA_ERR_INVALID_ARG;
  if (!isfinite(lr) || !(beta1 >= 0. && beta1 < 1.) || !(beta2 >= 0. && beta2 < 1.) ||
      !(eps >= 0.) || !isfinite(eps) || !(weight_decay >= 0.) || !isfinite(weight_decay))
    return DORA_ERR_INVALID_ARG;
  const int e = device_or_error();
  if (e != DORA_OK) return e;
  const optim::List l = layout(list->data, list->count, list->spans);
  const optim::AdamArgs a = {static_cast<optim::AdamState*>(state),
                             clip,
                             beta1,
                             beta2,
                             static_cast<float>(beta1),
                             static_cast<float>(1. - beta1),
                             static_cast<float>(beta2),
                             static_cast<float>(1. - beta2),
                             static_cast<float>(lr),
                             static_cast<float>(1. - lr * weight_decay),
                             static_cast<float>(eps)};
  return launched(launch_pdl(optim::adam_step_kernel, dim3(l.n_spans), dim3(optim::kThreads), 0,
                             reinterpret_cast<cudaStream_t>(stream), l, a));
}

}  // extern "C"
