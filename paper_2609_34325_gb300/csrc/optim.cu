// The end of a policy update, over all tensors of a parameter list in one launch
// each: the global gradient norm, clipping by it, and an Adam step (App. D.2,
// Table 4) that takes the clipping factor as it reads the gradients.
//
// The list lives on the device: one entry per tensor, and the tensors cut into
// units of kUnit elements that are dealt out evenly as spans of consecutive
// units, whatever the tensors' sizes.  A CTA walks its spans, piece by piece.
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
namespace optim {

constexpr int kThreads = 256;
constexpr int kUnit = 1024;               // elements
constexpr int kMaxSpans = 152 * 8;
constexpr int kFill = 48;                 // entries written by one launch, passed by value

struct Entry {
  const void* grad;
  void* clipped;                          // null: in place
  void* param;
  float *m, *v;
  uint16_t* copy;                         // nullable, bf16
  int64_t n;
  int64_t first_unit;
  int32_t grad_type, param_type;
};

// Units [unit, unit_end) of the whole list, starting in tensor `tensor`.
struct Span {
  int64_t unit, unit_end;
  int32_t tensor, pad;
  Entry first;                            // the entry of that tensor
};

struct Header {
  unsigned ticket;                        // CTAs done; zero between calls
  unsigned pad[63];
  double partial[kMaxSpans];
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

__device__ __forceinline__ int64_t units_of(int64_t n) { return (n + kUnit - 1) / kUnit; }

__global__ void fill_spans_kernel(List list, int64_t units) {
  pdl_wait();
  const int b = blockIdx.x * blockDim.x + threadIdx.x;
  if (b >= list.n_spans) return;
  Span s;
  s.unit = units * b / list.n_spans;
  s.unit_end = units * (b + 1) / list.n_spans;
  int lo = 0, hi = list.count - 1;        // the last tensor that starts at or before the unit
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (list.entries[mid].first_unit <= s.unit) lo = mid; else hi = mid - 1;
  }
  s.tensor = lo;
  s.pad = 0;
  s.first = list.entries[lo];
  list.spans[b] = s;
}

// f(entry, first element, elements) for every piece of the span.
template <typename F>
__device__ __forceinline__ void for_pieces(const List& list, int span, F f) {
  const Span& s = list.spans[span];
  int64_t unit = s.unit;
  const int64_t end = s.unit_end;
  if (unit >= end) return;
  int tensor = s.tensor;
  Entry e = s.first;
  while (true) {
    const int64_t from = (unit - e.first_unit) * kUnit;
    const int64_t last = (end - e.first_unit) * kUnit;
    const int64_t to = last < e.n ? last : e.n;
    if (to > from) f(e, from, to - from);
    unit = e.first_unit + units_of(e.n);
    if (unit >= end || ++tensor >= list.count) return;
    e = list.entries[tensor];
  }
}

// Elements before the first 16-byte boundary (at most n).
template <typename T>
__device__ __forceinline__ int64_t head_of(const T* p, int64_t n) {
  const int64_t h = ((16u - (reinterpret_cast<uintptr_t>(p) & 15u)) & 15u) / sizeof(T);
  return h < n ? h : n;
}

// ---------------------------------------------------------------------------
// Norm.  Squares are summed in 32 bits over the elements that a thread has at
// hand at once and carried on in 64, so the result does not depend on the list's
// length; a 32-bit sum that left the middle of its range (gradients above about
// 1e18 or below 1e-18) is taken again in 64 bits.
// ---------------------------------------------------------------------------
constexpr float kSquaresLow = 1e-30f, kSquaresHigh = 1e37f;

template <int N>
__device__ __forceinline__ double squares(const float (&v)[N]) {
  float a = 0.f, b = 0.f;
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    a = fmaf(v[i], v[i], a);
    if (i + 1 < N) b = fmaf(v[i + 1], v[i + 1], b);
  }
  a += b;
  if (a > kSquaresLow && a < kSquaresHigh) return a;
  double t = 0.;
#pragma unroll
  for (int i = 0; i < N; ++i) t += static_cast<double>(v[i]) * v[i];
  return t;
}

template <typename T>
__device__ __forceinline__ double piece_squares(const T* p, int64_t n) {
  constexpr int kE = Granule<T>::kElems, kInFlight = 4;
  double acc = 0.;
  const int64_t head = head_of(p, n);
  const int64_t granules = (n - head) / kE, tail = head + granules * kE;
  if (threadIdx.x < head) {
    const float v[1] = {to_float(p[threadIdx.x])};
    acc += squares(v);
  }
  if (tail + threadIdx.x < n) {
    const float v[1] = {to_float(p[tail + threadIdx.x])};
    acc += squares(v);
  }
  const uint4* g = reinterpret_cast<const uint4*>(p + head);
  for (int64_t i = threadIdx.x; i < granules; i += kInFlight * kThreads) {
    uint4 q[kInFlight];
#pragma unroll
    for (int u = 0; u < kInFlight; ++u)
      q[u] = i + u * kThreads < granules ? __ldg(g + i + u * kThreads) : make_uint4(0, 0, 0, 0);
    uint32_t any = 0;
    float v[kInFlight * kE];
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
      any |= q[u].x | q[u].y | q[u].z | q[u].w;
      Granule<T>::unpack(q[u], v + u * kE);
    }
    if (any != 0) acc += squares(v);
  }
  return acc;
}

__device__ __forceinline__ double block_sum(double v, double* scratch) {
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

// out[0] = the norm, out[1] = min(1, max_norm / norm), 1 for a norm that is not finite; the CTA that is last adds
// the spans' sums in their order.
__global__ void __launch_bounds__(kThreads)
    grad_norm_kernel(List list, float max_norm, float* __restrict__ out) {
  __shared__ double scratch[kThreads / 32];
  __shared__ bool last;
  pdl_wait();
  double acc = 0.;
  for_pieces(list, blockIdx.x, [&](const Entry& e, int64_t from, int64_t n) {
    if (e.grad_type == DORA_F32)
      acc += piece_squares(static_cast<const float*>(e.grad) + from, n);
    else if (e.grad_type == DORA_BF16)
      acc += piece_squares(static_cast<const __nv_bfloat16*>(e.grad) + from, n);
    else
      acc += piece_squares(static_cast<const __half*>(e.grad) + from, n);
  });
  acc = block_sum(acc, scratch);
  if (threadIdx.x == 0) {
    list.header->partial[blockIdx.x] = acc;
    __threadfence();
    last = atomicAdd(&list.header->ticket, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  double t = 0.;
  for (int b = threadIdx.x; b < static_cast<int>(gridDim.x); b += kThreads)
    t += __ldcg(&list.header->partial[b]);
  t = block_sum(t, scratch);
  if (threadIdx.x == 0) {
    const float norm = static_cast<float>(sqrt(t));
    out[0] = norm;
    out[1] = isfinite(norm) && norm > max_norm ? static_cast<float>(max_norm / sqrt(t)) : 1.f;
    list.header->ticket = 0;
  }
}

// ---------------------------------------------------------------------------
// Clipping.  A norm that is not finite leaves the gradients as they are.
// ---------------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ void piece_scale(const T* p, T* y, int64_t n, float f) {
  constexpr int kE = Granule<T>::kElems, kInFlight = 4;
  if ((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(y)) & 15u) {
    for (int64_t i = threadIdx.x; i < n; i += kThreads) from_float(to_float(p[i]) * f, y + i);
    return;
  }
  const int64_t head = head_of(p, n);
  const int64_t granules = (n - head) / kE, tail = head + granules * kE;
  if (threadIdx.x < head) from_float(to_float(p[threadIdx.x]) * f, y + threadIdx.x);
  if (tail + threadIdx.x < n)
    from_float(to_float(p[tail + threadIdx.x]) * f, y + tail + threadIdx.x);
  const uint4* g = reinterpret_cast<const uint4*>(p + head);
  uint4* o = reinterpret_cast<uint4*>(y + head);
  for (int64_t i = threadIdx.x; i < granules; i += kInFlight * kThreads) {
    uint4 q[kInFlight];
#pragma unroll
    for (int u = 0; u < kInFlight; ++u)
      if (i + u * kThreads < granules) q[u] = g[i + u * kThreads];
#pragma unroll
    for (int u = 0; u < kInFlight; ++u)
      if (i + u * kThreads < granules) {
        float v[kE];
        Granule<T>::unpack(q[u], v);
#pragma unroll
        for (int k = 0; k < kE; ++k) v[k] *= f;
        o[i + u * kThreads] = Granule<T>::pack(v);
      }
  }
}

__global__ void __launch_bounds__(kThreads)
    scale_grads_kernel(List list, const float* __restrict__ norm) {
  pdl_wait();
  const float f = isfinite(norm[0]) ? norm[1] : 1.f;
  for_pieces(list, blockIdx.x, [&](const Entry& e, int64_t from, int64_t n) {
    void* to = e.clipped != nullptr ? e.clipped : const_cast<void*>(e.grad);
    if (to == e.grad && f == 1.f) return;
    if (e.grad_type == DORA_F32)
      piece_scale(static_cast<const float*>(e.grad) + from, static_cast<float*>(to) + from, n, f);
    else if (e.grad_type == DORA_BF16)
      piece_scale(static_cast<const __nv_bfloat16*>(e.grad) + from,
                  static_cast<__nv_bfloat16*>(to) + from, n, f);
    else
      piece_scale(static_cast<const __half*>(e.grad) + from, static_cast<__half*>(to) + from, n,
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

// Four elements of T at an address that is a multiple of their size.
template <typename T>
struct Quad {                             // bf16, fp16
  uint2 q;
  __device__ __forceinline__ void load(const T* p) { q = *reinterpret_cast<const uint2*>(p); }
  __device__ __forceinline__ void unpack(float* v) const {
    float w[8];
    Granule<T>::unpack(make_uint4(q.x, q.y, 0u, 0u), w);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = w[k];
  }
  static __device__ __forceinline__ void store(const float* v, T* p) {
    *reinterpret_cast<uint2*>(p) =
        make_uint2(Granule<T>::pair(v[0], v[1]), Granule<T>::pair(v[2], v[3]));
  }
};
template <>
struct Quad<float> {
  uint4 q;
  __device__ __forceinline__ void load(const float* p) { q = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void unpack(float* v) const { Granule<float>::unpack(q, v); }
  static __device__ __forceinline__ void store(const float* v, float* p) {
    *reinterpret_cast<uint4*>(p) = Granule<float>::pack(v);
  }
};
template <typename T>
__device__ __forceinline__ bool quads(const T* p) {
  return (reinterpret_cast<uintptr_t>(p) & (4 * sizeof(T) - 1)) == 0;
}

template <typename P, typename G>
__device__ __forceinline__ void piece_adam(const AdamArgs& a, const AdamStep& s, const Entry& e,
                                           int64_t from, int64_t n) {
  constexpr int kInFlight = 2;
  P* p = static_cast<P*>(e.param) + from;
  const G* g = static_cast<const G*>(e.grad) + from;
  float *m = e.m + from, *v = e.v + from;
  __nv_bfloat16* c =
      e.copy != nullptr ? reinterpret_cast<__nv_bfloat16*>(e.copy) + from : nullptr;
  int64_t done = 0;
  if (quads(p) && quads(g) && quads(m) && quads(v) && (c == nullptr || quads(c))) {
    const int64_t groups = n / 4;
    done = groups * 4;
    for (int64_t i = threadIdx.x; i < groups; i += kInFlight * kThreads) {
      Quad<P> qp[kInFlight];
      Quad<G> qg[kInFlight];
      Quad<float> qm[kInFlight], qv[kInFlight];
#pragma unroll
      for (int u = 0; u < kInFlight; ++u) {
        const int64_t at = 4 * (i + u * kThreads);
        if (at < done) {
          qg[u].load(g + at);
          qp[u].load(p + at);
          qm[u].load(m + at);
          qv[u].load(v + at);
        }
      }
#pragma unroll
      for (int u = 0; u < kInFlight; ++u) {
        const int64_t at = 4 * (i + u * kThreads);
        if (at < done) {
          float fp[4], fg[4], fm[4], fv[4];
          qp[u].unpack(fp);
          qg[u].unpack(fg);
          qm[u].unpack(fm);
          qv[u].unpack(fv);
#pragma unroll
          for (int k = 0; k < 4; ++k) adam_one(a, s, fg[k], fp + k, fm + k, fv + k);
          Quad<P>::store(fp, p + at);
          Quad<float>::store(fm, m + at);
          Quad<float>::store(fv, v + at);
          if (c != nullptr) Quad<__nv_bfloat16>::store(fp, c + at);
        }
      }
    }
  }
  for (int64_t i = done + threadIdx.x; i < n; i += kThreads) {
    float pi = to_float(p[i]), mi = m[i], vi = v[i];
    adam_one(a, s, to_float(g[i]), &pi, &mi, &vi);
    from_float(pi, p + i);
    m[i] = mi;
    v[i] = vi;
    if (c != nullptr) from_float(pi, c + i);
  }
}

template <typename P>
__device__ __forceinline__ void piece_adam_of(const AdamArgs& a, const AdamStep& s, const Entry& e,
                                              int64_t from, int64_t n) {
  if (e.grad_type == DORA_F32) piece_adam<P, float>(a, s, e, from, n);
  else if (e.grad_type == DORA_BF16) piece_adam<P, __nv_bfloat16>(a, s, e, from, n);
  else piece_adam<P, __half>(a, s, e, from, n);
}

__global__ void __launch_bounds__(kThreads) adam_step_kernel(List list, AdamArgs a) {
  pdl_wait();
  const AdamState st = *a.state;
  AdamStep s = {1.f, 0.f, 0.f};
  bool skip = false;
  if (a.clip != nullptr) {
    skip = !isfinite(a.clip[0]);
    s.f = a.clip[1];
  }
  const double p1 = (st.step > 0 ? st.power1 : 1.) * a.beta1;
  const double p2 = (st.step > 0 ? st.power2 : 1.) * a.beta2;
  s.step_size = a.lr / static_cast<float>(1. - p1);
  s.root_scale = 1.f / sqrtf(static_cast<float>(1. - p2));
  if (!skip)
    for_pieces(list, blockIdx.x, [&](const Entry& e, int64_t from, int64_t n) {
      if (e.param_type == DORA_F32) piece_adam_of<float>(a, s, e, from, n);
      else if (e.param_type == DORA_BF16) piece_adam_of<__nv_bfloat16>(a, s, e, from, n);
      else piece_adam_of<__half>(a, s, e, from, n);
    });
  __syncthreads();                        // every thread of the CTA has read the state
  if (threadIdx.x == 0) {
    __threadfence();
    if (atomicAdd(&a.state->ticket, 1u) == gridDim.x - 1) {
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

// Checks the tensors and counts their units; -1 when one is not valid.
int64_t count_units(const dora_param* params, int32_t count, int64_t* elements, bool* has_params) {
  int64_t units = 0;
  *elements = 0;
  *has_params = true;
  for (int32_t i = 0; i < count; ++i) {
    const dora_param& t = params[i];
    if (t.n < 0 || t.n > (int64_t{1} << 40) || !known_type(t.grad_dtype)) return -1;
    if (t.n > 0 && (t.grad == nullptr || !aligned_to(t.grad, t.grad_dtype) ||
                    !aligned_to(t.clipped, t.grad_dtype)))
      return -1;
    const int given = (t.param != nullptr) + (t.exp_avg != nullptr) + (t.exp_avg_sq != nullptr);
    if (t.n > 0 && given != 0 && given != 3) return -1;
    if (t.n > 0 && given == 0) *has_params = false;
    if (given == 3 && (!known_type(t.param_dtype) || !aligned_to(t.param, t.param_dtype) ||
                       !aligned_to(t.exp_avg, DORA_F32) || !aligned_to(t.exp_avg_sq, DORA_F32) ||
                       !aligned_to(t.copy, DORA_BF16)))
      return -1;
    units += (t.n + optim::kUnit - 1) / optim::kUnit;
    *elements += t.n;
  }
  return units;
}

int spans_for(int64_t units) {
  if (units < 1) return 1;
  return units < optim::kMaxSpans ? static_cast<int>(units) : optim::kMaxSpans;
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
  const int64_t units = count_units(params, count, &elements, &has_params);
  if (units < 0) return 0;
  return round256(sizeof(optim::Header)) +
         round256(static_cast<size_t>(count) * sizeof(optim::Entry)) +
         round256(static_cast<size_t>(spans_for(units)) * sizeof(optim::Span));
}

int dora_param_list_prepare(const dora_param* params, int32_t count, void* data, size_t bytes,
                            dora_param_list* list, dora_stream_t stream_) {
  if (params == nullptr || count < 1 || data == nullptr || list == nullptr ||
      (reinterpret_cast<uintptr_t>(data) & 255u) != 0)
    return DORA_ERR_INVALID_ARG;
  int64_t elements;
  bool has_params;
  const int64_t units = count_units(params, count, &elements, &has_params);
  if (units < 0 || bytes < dora_param_list_size(params, count)) return DORA_ERR_INVALID_ARG;
  const int e = device_or_error();
  if (e != DORA_OK) return e;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  const optim::List l = layout(data, count, spans_for(units));
  int64_t first_unit = 0;
  for (int32_t first = 0; first < count; first += optim::kFill) {
    const int some = count - first < optim::kFill ? count - first : optim::kFill;
    optim::FillArgs args = {};
    for (int i = 0; i < some; ++i) {
      const dora_param& t = params[first + i];
      args.e[i] = optim::Entry{t.grad, t.clipped, t.param, t.exp_avg, t.exp_avg_sq, t.copy, t.n,
                               first_unit, t.grad_dtype, t.param_dtype};
      first_unit += (t.n + optim::kUnit - 1) / optim::kUnit;
    }
    const int rc = launched(launch_pdl(optim::fill_entries_kernel, dim3(1), dim3(optim::kFill), 0,
                                       stream, l.header, l.entries, first, some, args));
    if (rc != DORA_OK) return rc;
  }
  const int rc = launched(launch_pdl(optim::fill_spans_kernel, dim3((l.n_spans + 127) / 128),
                                     dim3(128), 0, stream, l, units));
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
