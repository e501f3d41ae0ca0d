// Orthogonalised updates: Newton-Schulz iterations over a list of matrices, alone and as
// the end of a Muon step (momentum, orthogonalisation, weights).
//
// With X the update U (or U^T, so that X is m x n with m <= n) over its Frobenius norm,
//   A = X X^T,   X <- a X + (b A + c A^2) X
// brings every singular value near 1 (the quintic of coefficients a, b, c below, whose
// values stay below 1.21).  Three products an iteration on the tensor cores, the two
// symmetric ones by half: 3 m^2 n + m^3 operations.
//
// Precision.  The products take fp16 operands (11 bits; with bf16's 8 the result is 1 to
// 20% off) and add in fp32.  Two things keep the rounding small where it counts: X itself is carried
// as hi + lo, two fp16 values of 22 bits, of which only hi goes into the products; and
// the diagonals of A and of B = b A + c A^2, which hold most of both once the singular
// values are near 1, stay out of the products, in fp32.  With A = D + F and B = E + G (D, E
// diagonal, F, G without one):
//   A^2 = D^2 + D F + F D + F F,    B X = E X + G X_hi,
//   E = b D + c (D^2 + diag(F F)),  G = b F + c (D F + F D + F F) off the diagonal,
//   X <- (a + E) X + G X_hi,
// so that what is rounded is multiplied by the small G rather than by B, whose product with
// X nearly cancels against a X.  The result is 2e-4 to 1.2e-3 off the iteration in 64 bits
// (relative 2-norm), half the rounding of a bf16 output.
//
// Layout.  X hi, X lo, F and G are kept in tiles of 128 x 64 fp16 values (16 KB, rows of 128
// bytes), padded with zeros: whatever the matrices' sizes, one tensor map describes all
// of them.  A tile is an operand either way: K-major (rows of X for X X^T) or MN-major (rows
// of X as the K of G X).
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include "dora.h"
#include "dora_ptx.cuh"
#include "granule.cuh"
#include "token_ops.cuh"
#include "update_ptx.cuh"

namespace dora {
namespace ortho {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kScale = 256.f;           // of X, F and G in fp16: their values are below 4
constexpr float kLoScale = 2048.f;        // of lo, on top of it
constexpr int kMaxSteps = 32;
constexpr int kTileRows = 128, kTileCols = 64;
constexpr int kTileBytes = kTileRows * kTileCols * 2;
constexpr int kChunk = 4096;              // elements of a matrix that a CTA takes at once
constexpr int kRowThreads = 256, kRowCtas = 4;
constexpr int kMaxShort = 16384, kMaxLong = 1 << 24;

struct Squares;

struct Entry {
  const void* grad;
  void* param;
  float* momentum;
  uint16_t *copy, *out;                   // bf16
  int32_t rows, cols, grad_type, param_type;
  float scale;
  int32_t m, n, tall;                     // X is m x n; tall: X = U^T
  int32_t mb, nb;                         // blocks of 128 rows, of 128 columns; X, F and G
                                          // have an even number of the first
  int64_t x[2], lo, f, g;                 // first tiles of X hi (two, in turn), X lo, F, G
  float *d, *e;                           // the diagonals of A and B
  Squares* partial;                       // of its chunks
  float2* norm;                           // one over the norm of u 2^-k, and 2^-k
  unsigned* ticket;                       // chunks done; zero between calls
  int32_t chunks, pad;
  // first of its chunks, of its tiles of X and of its output tiles among the list's
  int64_t first_chunk, first_x, first_sym, first_all;
};

struct Header {
  int abort;                              // a bounded wait of this call has run out
  int pad[63];
};

// One piece of work: block row and block column of a matrix, and its columns.
struct Tile {
  int32_t matrix, i, j, width;
};

struct List {
  Header* header;
  Entry* entries;
  int32_t* chunk_of;                      // matrix of every chunk
  Tile *x, *sym, *all;
  char* tiles;
  int count;
  int n_chunks, n_x, n_sym, n_all;
};

constexpr int kFill = 16;                 // entries written by one launch, passed by value
struct FillArgs {
  Entry e[kFill];
};

__global__ void fill_entries_kernel(List list, int first, int count, FillArgs args) {
  pdl_wait();
  if (first == 0 && threadIdx.x == 0) list.header->abort = 0;
  if (threadIdx.x < count) {
    list.entries[first + threadIdx.x] = args.e[threadIdx.x];
    *args.e[threadIdx.x].ticket = 0;
  }
}

template <typename F>
__device__ __forceinline__ int matrix_of(const List& list, int64_t at, F first) {
  int lo = 0, hi = list.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first(list.entries[mid]) <= at) lo = mid; else hi = mid - 1;
  }
  return lo;
}

__global__ void fill_tiles_kernel(List list) {
  pdl_wait();
  const int t = blockIdx.x * blockDim.x + threadIdx.x;
  if (t < list.n_chunks)
    list.chunk_of[t] = matrix_of(list, t, [](const Entry& e) { return e.first_chunk; });
  if (t < list.n_x) {
    const int q = matrix_of(list, t, [](const Entry& e) { return e.first_x; });
    const int at = static_cast<int>(t - list.entries[q].first_x), w = 2 * list.entries[q].nb;
    list.x[t] = Tile{q, at / w, at % w, 0};
  }
  if (t < list.n_all) {
    const int q = matrix_of(list, t, [](const Entry& e) { return e.first_all; });
    const int at = static_cast<int>(t - list.entries[q].first_all), nb = list.entries[q].nb;
    const int w = (nb + 1) / 2, j = at % w;
    list.all[t] = Tile{q, at / w, j, 2 * j + 1 < nb ? 256 : 128};
  }
  if (t < list.n_sym) {
    const int q = matrix_of(list, t, [](const Entry& e) { return e.first_sym; });
    const int mb = list.entries[q].mb;
    int at = static_cast<int>(t - list.entries[q].first_sym), i = 0, left = (mb + 1) / 2;
    while (at >= left) {
      at -= left--;
      ++i;
    }
    list.sym[t] = Tile{q, i, i + at, 2 * (i + at) + 1 < mb ? 256 : 128};
  }
}

__device__ __forceinline__ int size_of(int type) { return type == DORA_F32 ? 4 : 2; }
__device__ __forceinline__ float load_one(const void* p, int type, int64_t i) {
  if (type == DORA_F32) return static_cast<const float*>(p)[i];
  if (type == DORA_BF16) return to_float(static_cast<const __nv_bfloat16*>(p)[i]);
  return to_float(static_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ void store_one(float v, void* p, int type, int64_t i) {
  if (type == DORA_F32) static_cast<float*>(p)[i] = v;
  else if (type == DORA_BF16) from_float(v, static_cast<__nv_bfloat16*>(p) + i);
  else from_float(v, static_cast<__half*>(p) + i);
}

// Four elements from the k-th, zeros past the last: 16 bytes of fp32, 8 (in x and y) of the
// others, at once where `quads` says that they are aligned to that.
__device__ __forceinline__ bool in_quads(const void* p, int type) {
  return (reinterpret_cast<uintptr_t>(p) & (4 * size_of(type) - 1)) == 0;
}
__device__ __forceinline__ uint4 whole_quad(const void* p, int type, int64_t k) {
  if (type == DORA_F32) return *reinterpret_cast<const uint4*>(static_cast<const float*>(p) + k);
  const uint2 q = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + k);
  return make_uint4(q.x, q.y, 0u, 0u);
}
__device__ __forceinline__ uint4 load_quad(const void* p, int type, int64_t k, int64_t total,
                                           bool quads) {
  if (quads && k + 4 <= total) return whole_quad(p, type, k);
  uint32_t w[4] = {0u, 0u, 0u, 0u};
  if (type == DORA_F32) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (k + j < total) w[j] = static_cast<const uint32_t*>(p)[k + j];
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (k + j < total)
        w[j >> 1] |= static_cast<uint32_t>(static_cast<const uint16_t*>(p)[k + j]) << (16 * (j & 1));
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void unpack_quad(uint4 q, int type, float* v) {
  float w[8];
  if (type == DORA_F32) Granule<float>::unpack(q, w);
  else if (type == DORA_BF16) Granule<__nv_bfloat16>::unpack(q, w);
  else Granule<__half>::unpack(q, w);
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = w[j];
}

// What all kernels of a call take.
struct Args {
  const float* clip;                      // nullable: norm and factor
  int muon;                               // 0: U is the gradient itself
  int nesterov;
  float mu, omu;                          // momentum, 1 - momentum
  float lr, keep;                         // keep = 1 - lr decay
  int32_t* status;
};

// A step is skipped where the norm of the gradients is not finite.
__device__ __forceinline__ bool skipped(const Args& a) {
  return a.clip != nullptr && !isfinite(a.clip[0]);
}
__device__ __forceinline__ float factor(const Args& a) {
  return a.clip != nullptr ? a.clip[1] : 1.f;
}
// The update from a clipped gradient and the new momentum.
__device__ __forceinline__ float update_of(const Args& a, float d, float m) {
  if (!a.muon) return d;
  return a.nesterov ? fmaf(a.mu, m, a.omu * d) : m;
}

// ---------------------------------------------------------------------------
// Momentum, and the update's norm.  A CTA takes a run of chunks, a matrix's one after the
// other.  A thread sums its squares in fp32; where that leaves the middle of the range, it sums
// those of u 2^-k, with k the exponent of its largest |u|, so that no finite update
// overflows or vanishes.  The chunks are joined in their order by the CTA that is last
// of the matrix.
// ---------------------------------------------------------------------------
// A sum of squares of values times 2^-k.
struct Squares {
  float sum;
  int k;
  __device__ __forceinline__ void add(Squares o) {
    if (o.k == k) {
      sum += o.sum;
    } else if (o.sum != 0.f) {
      const int most = k > o.k ? k : o.k;
      sum = ldexpf(sum, 2 * (k - most)) + ldexpf(o.sum, 2 * (o.k - most));
      k = most;
    }
  }
};
__device__ __forceinline__ Squares warp_squares(Squares s) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1)
    s.add(Squares{__shfl_xor_sync(0xffffffffu, s.sum, off),
                  __shfl_xor_sync(0xffffffffu, s.k, off)});
  return s;
}
// Over the block, in thread 0.
__device__ __forceinline__ Squares block_squares(Squares s, Squares* scratch) {
  s = warp_squares(s);
  __syncthreads();                        // the places are free
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0)
#pragma unroll
    for (int w = 1; w < kRowThreads / 32; ++w) s.add(scratch[w]);
  return s;
}

template <int kN>
__device__ __forceinline__ Squares squares_of(const float (&u)[kN]) {
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < kN; ++i) sum = fmaf(u[i], u[i], sum);
  if (sum > 1e-25f && sum < 1e30f) return {sum, 0};
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < kN; ++i) top = fmaxf(top, fabsf(u[i]));
  int k = static_cast<int>(__float_as_uint(top) >> 23) - 127;
  k = k < -126 ? -126 : (k > 126 ? 126 : k);
  const float scale = __uint_as_float(static_cast<uint32_t>(127 - k) << 23);   // 2^-k
  sum = 0.f;
#pragma unroll
  for (int i = 0; i < kN; ++i) sum = fmaf(u[i] * scale, u[i] * scale, sum);
  return {sum, k};
}

__global__ void __launch_bounds__(kRowThreads, kRowCtas) momentum_kernel(List list, Args a) {
  constexpr int kPer = kChunk / kRowThreads;
  __shared__ Squares scratch[kRowThreads / 32];
  __shared__ bool last;
  pdl_wait();
  if (skipped(a)) return;
  const float f = factor(a);
  if (blockIdx.x == 0 && threadIdx.x == 0) list.header->abort = 0;
  int c = static_cast<int>(static_cast<int64_t>(list.n_chunks) * blockIdx.x / gridDim.x);
  const int end = static_cast<int>(static_cast<int64_t>(list.n_chunks) * (blockIdx.x + 1) /
                                   gridDim.x);
  const Entry* at = list.entries + (c < end ? list.chunk_of[c] : 0);
  for (; c < end; ++c) {
    if (c - at->first_chunk >= at->chunks) ++at;
    const Entry& e = *at;
    const int64_t total = static_cast<int64_t>(e.m) * e.n;
    const int64_t from = static_cast<int64_t>(c - e.first_chunk) * kChunk;
    // quads of elements, all on their way before the first is looked at
    const bool quads = in_quads(e.grad, e.grad_type) && (!a.muon || in_quads(e.momentum, DORA_F32));
    uint4 qg[kPer / 4], qm[kPer / 4];
    if (quads && from + kChunk <= total) {
#pragma unroll
      for (int i = 0; i < kPer / 4; ++i) {
        const int64_t k = from + 4 * (threadIdx.x + i * kRowThreads);
        qg[i] = whole_quad(e.grad, e.grad_type, k);
        qm[i] = a.muon ? whole_quad(e.momentum, DORA_F32, k) : make_uint4(0, 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kPer / 4; ++i) {
        const int64_t k = from + 4 * (threadIdx.x + i * kRowThreads);
        qg[i] = load_quad(e.grad, e.grad_type, k, total, quads);
        qm[i] = a.muon ? load_quad(e.momentum, DORA_F32, k, total, quads) : make_uint4(0, 0, 0, 0);
      }
    }
    float u[kPer];
#pragma unroll
    for (int i = 0; i < kPer / 4; ++i) {
      const int64_t k = from + 4 * (threadIdx.x + i * kRowThreads);
      float d[4], m[4];
      unpack_quad(qg[i], e.grad_type, d);
      Granule<float>::unpack(qm[i], m);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        d[j] *= f;
        if (a.muon) m[j] = fmaf(a.mu, m[j], a.omu * d[j]);
        u[4 * i + j] = update_of(a, d[j], m[j]);
      }
      if (!a.muon) continue;
      if (quads && k + 4 <= total) {
        *reinterpret_cast<uint4*>(e.momentum + k) = Granule<float>::pack(m);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (k + j < total) e.momentum[k + j] = m[j];
      }
    }
    const Squares sum = block_squares(squares_of(u), scratch);
    if (threadIdx.x == 0) {
      e.partial[c - e.first_chunk] = sum;
      last = take_ticket(e.ticket) == static_cast<unsigned>(e.chunks) - 1;
    }
    __syncthreads();
    if (!last) continue;
    Squares all = {0.f, -126};
    for (int i = threadIdx.x; i < e.chunks; i += kRowThreads) {
      const int2 p = __ldcg(reinterpret_cast<const int2*>(&e.partial[i]));
      all.add(Squares{__int_as_float(p.x), p.y});
    }
    all = block_squares(all, scratch);
    if (threadIdx.x == 0) {
      // a matrix of zeros stays one; one that is not finite becomes NaN
      *e.norm = make_float2(
          all.sum == 0.f ? 0.f : (isfinite(all.sum) ? 1.f / sqrtf(all.sum) : NAN),
          __uint_as_float(static_cast<uint32_t>(127 - all.k) << 23));
      *e.ticket = 0;
    }
  }
}

// ---------------------------------------------------------------------------
// Tiles.  Element (r, c) of a tile lies at this offset.
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t tile_offset(int r, int c) {
  return static_cast<uint32_t>(r * 128 + c * 2);
}
__device__ __forceinline__ char* tile_at(const List& list, int64_t tile) {
  return list.tiles + tile * kTileBytes;
}
__device__ __forceinline__ uint32_t pair_of(float a, float b) {
  return Granule<__half>::pair(a, b);
}

// Eight values `step` apart, zeros from the some-th on.
template <typename T>
__device__ __forceinline__ void load_eight(const T* p, int64_t step, int some, float* v) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = i < some ? to_float(p[i * step]) : 0.f;
}

// hi and lo of eight values that are scaled already.
__device__ __forceinline__ void split(const float* v, uint4* hi, uint4* lo) {
  float rest[8], back[8];
  *hi = Granule<__half>::pack(v);
  Granule<__half>::unpack(*hi, back);
#pragma unroll
  for (int i = 0; i < 8; ++i) rest[i] = (v[i] - back[i]) * kLoScale;
  *lo = Granule<__half>::pack(rest);
}

// The normalised update into its tiles; a CTA takes a run of them.
__global__ void __launch_bounds__(kRowThreads, kRowCtas) normalise_kernel(List list, Args a) {
  pdl_wait();
  if (skipped(a)) return;
  const float f = factor(a);
  int t = static_cast<int>(static_cast<int64_t>(list.n_x) * blockIdx.x / gridDim.x);
  const int end = static_cast<int>(static_cast<int64_t>(list.n_x) * (blockIdx.x + 1) / gridDim.x);
  if (t >= end) return;
  const Tile first = list.x[t];
  int matrix = first.matrix, ti = first.i, tj = first.j;
  for (; t < end; ++t) {
    const Entry& e = list.entries[matrix];
    const float2 norm = *e.norm;
    const int64_t at = static_cast<int64_t>(ti) * (2 * e.nb) + tj;
    char* hi = tile_at(list, e.x[0] + at);
    char* lo = tile_at(list, e.lo + at);
    const bool quads = !e.tall && (e.n & 7) == 0 && in_quads(e.grad, e.grad_type) &&
                       (!a.muon || in_quads(e.momentum, DORA_F32));
    constexpr int kItems = kTileRows * 8 / kRowThreads, kSome = 2;
    // pieces of eight columns, the lanes along what is contiguous in the matrix
    for (int w0 = 0; w0 < kItems; w0 += kSome) {
      float d[kSome][8], m[kSome][8];
#pragma unroll
      for (int y = 0; y < kSome; ++y) {
        const int w = threadIdx.x + (w0 + y) * kRowThreads;
        const int r = e.tall ? w % kTileRows : w / 8, piece = e.tall ? w / kTileRows : w % 8;
        const int row = ti * kTileRows + r, col = tj * kTileCols + piece * 8;
        const int some = row < e.m ? e.n - col : 0;     // columns that there are
        const int64_t step = e.tall ? e.m : 1;
        const int64_t k = e.tall ? static_cast<int64_t>(col) * e.m + row
                                 : static_cast<int64_t>(row) * e.n + col;
        if (quads && some >= 8) {
#pragma unroll
          for (int i = 0; i < 8; i += 4) {
            unpack_quad(whole_quad(e.grad, e.grad_type, k + i), e.grad_type, d[y] + i);
            if (a.muon) Granule<float>::unpack(whole_quad(e.momentum, DORA_F32, k + i), m[y] + i);
          }
        } else if (e.grad_type == DORA_F32) {
          load_eight(static_cast<const float*>(e.grad) + k, step, some, d[y]);
        } else if (e.grad_type == DORA_BF16) {
          load_eight(static_cast<const __nv_bfloat16*>(e.grad) + k, step, some, d[y]);
        } else {
          load_eight(static_cast<const __half*>(e.grad) + k, step, some, d[y]);
        }
        if (a.muon && !(quads && some >= 8)) load_eight(e.momentum + k, step, some, m[y]);
      }
#pragma unroll
      for (int y = 0; y < kSome; ++y) {
        const int w = threadIdx.x + (w0 + y) * kRowThreads;
        const int r = e.tall ? w % kTileRows : w / 8, piece = e.tall ? w / kTileRows : w % 8;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
          v[i] = update_of(a, d[y][i] * f, a.muon ? m[y][i] : 0.f) * norm.y * norm.x * kScale;
        uint4 h, l;
        split(v, &h, &l);
        const uint32_t to = tile_offset(r, piece * 8);
        *reinterpret_cast<uint4*>(hi + to) = h;
        *reinterpret_cast<uint4*>(lo + to) = l;
      }
    }
    if (++tj == 2 * e.nb) {
      tj = 0;
      if (++ti == 2 * ((e.mb + 1) / 2)) {
        ti = 0;
        ++matrix;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// The products.  Persistent CTAs in pairs take output tiles of 256 rows and 256 or 128
// columns: one MMA spans the pair, each CTA holding its 128 rows of the left operand and half
// of the right one, so that a stage is 32 KB for each.  In a CTA one warp copies operands into
// a ring of stages, one issues the MMAs (in the first CTA) into one of two accumulators, and
// eight finish the other one, 32 x 32 values at a time: what they read besides (F; X hi and lo)
// comes by copies of its own into three places a warp, two of them ahead, and is written
// over there and copied out.
// ---------------------------------------------------------------------------
enum Phase { kGram, kSquare, kApply, kLast };

constexpr int kStages = 4;
constexpr int kBlock = 128;               // rows of a CTA's part of an output tile
constexpr int kWide = 256;                // columns of one
constexpr int kK = 64;                    // of a stage
constexpr int kEpiWarps = 8;
constexpr int kThreads = 64 + 32 * kEpiWarps;
constexpr int kHalfTile = kTileBytes / 2; // 64 rows
constexpr int kPlaces = 3;
constexpr int kPiece = 32 * 32;           // values that a warp finishes at once
constexpr uint16_t kPairMask = 0x3;

struct Smem {
  uint8_t a[kStages][kTileBytes];
  uint8_t b[kStages][kTileBytes];
  uint16_t piece[kEpiWarps][kPlaces][2][kPiece];
  uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2], drain;
  uint64_t piece_full[kEpiWarps][kPlaces];
  uint32_t tmem;
  int abort, issued, consumed;
};
static_assert(sizeof(Smem) <= 227 * 1024, "shared memory");

// The maps of all tiles: whole ones, their halves of 64 rows, and 32 x 32 values.
struct Maps {
  CUtensorMap tile, half, piece;
};

__host__ __device__ constexpr uint32_t idesc_f16(int m, int n, bool b_mn_major) {
  return (1u << 4) | ((b_mn_major ? 1u : 0u) << 16) | (static_cast<uint32_t>(n >> 3) << 17) |
         (static_cast<uint32_t>(m >> 4) << 24);
}

// 16-byte part `p` of lane's row of a piece (rows of 64 bytes, as a copy swizzles them).
__device__ __forceinline__ uint4* piece_at(uint16_t* piece, int row, int p) {
  return reinterpret_cast<uint4*>(reinterpret_cast<char*>(piece) + row * 64 +
                                  ((p ^ ((row >> 1) & 3)) << 4));
}
__device__ __forceinline__ uint16_t* value_in(uint16_t* piece, int row, int c) {
  return reinterpret_cast<uint16_t*>(piece_at(piece, row, c >> 3)) + (c & 7);
}

// 32 values `pitch` apart: the first `some` of x, times f, are written there, or the weights
// there are updated by them, which leaves the new weights in x.
template <typename T>
__device__ __forceinline__ void store_rows(const float (&x)[32], T* p, int64_t pitch, int some,
                                           float f) {
#pragma unroll
  for (int i = 0; i < 32; ++i)
    if (i < some) from_float(x[i] * f, p + i * pitch);
}
template <typename T>
__device__ __forceinline__ void update_rows(float (&x)[32], T* p, int64_t pitch, int some,
                                            float keep, float step) {
  T old[32];                              // all on their way before the first is used
#pragma unroll
  for (int i = 0; i < 32; ++i)
    if (i < some) old[i] = p[i * pitch];
#pragma unroll
  for (int i = 0; i < 32; ++i)
    if (i < some) {
      x[i] = fmaf(to_float(old[i]), keep, step * x[i]);
      from_float(x[i], p + i * pitch);
    }
}

// A warp's part of an output tile.
struct Part {
  int row, col;                           // first row, first column in the matrix
  int pieces;
};

template <Phase kPhase>
__global__ void __launch_bounds__(kThreads, 1)
    product_kernel(const __grid_constant__ Maps maps, List list, Args a, int from) {
  extern __shared__ __align__(1024) uint8_t raw[];
  pdl_trigger();
  Smem& s = *reinterpret_cast<Smem*>(raw);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = static_cast<int>(cluster_ctarank()), cid = blockIdx.x >> 1;
  const int n_clusters = gridDim.x >> 1;
  constexpr bool kSym = kPhase == kGram || kPhase == kSquare;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&s.full[i], 1);
      mbar_init(&s.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s.acc_full[i], 1);
      mbar_init(&s.acc_empty[i], 2 * kEpiWarps);
    }
    for (int w = 0; w < kEpiWarps; ++w)
      for (int i = 0; i < kPlaces; ++i) mbar_init(&s.piece_full[w][i], 1);
    mbar_init(&s.drain, 1);
    s.abort = s.issued = s.consumed = 0;
    fence_barrier_init();
    tma_prefetch_desc(&maps.tile);
    tma_prefetch_desc(&maps.half);
    tma_prefetch_desc(&maps.piece);
  }
  if (warp == 1) tmem_alloc_pair(&s.tmem, 2 * kWide);
  tc_fence_before();
  cluster_sync();
  tc_fence_after();
  pdl_wait();
  const Tile* tiles = kSym ? list.sym : list.all;
  const int n_tiles = skipped(a) || list.header->abort ? 0 : (kSym ? list.n_sym : list.n_all);
  const uint32_t tmem = s.tmem;
  volatile int* abort = &s.abort;
  // stages of a tile: the K of its product over 64
  auto steps = [&](const Entry& e) { return ((kPhase == kGram ? e.n : e.m) + kK - 1) / kK; };

  if (warp == 0) {
    if (elect_one()) {
      int it = 0;
      bool ok = true;
      for (int w = cid; ok && w < n_tiles; w += n_clusters) {
        const Tile t = tiles[w];
        const Entry& e = list.entries[t.matrix];
        const int n = steps(e), row_tiles = kPhase == kGram ? 2 * e.nb : 2 * e.mb;
        const int64_t left = kPhase == kGram ? e.x[from] : (kPhase == kSquare ? e.f : e.g);
        const bool wide = t.width == kWide;
        const int32_t ya =
            static_cast<int32_t>((left + static_cast<int64_t>(2 * t.i + rank) * row_tiles) * kTileRows);
        // symmetric: rows of the left operand, 128 or 64 for each CTA; else 64 rows of X, two
        // column tiles or one for each CTA
        int32_t yb;
        if (kSym)
          yb = static_cast<int32_t>(
                   (left + static_cast<int64_t>(2 * t.j + (wide ? rank : 0)) * row_tiles) *
                   kTileRows) +
               (wide ? 0 : rank * 64);
        else
          yb = static_cast<int32_t>((e.x[from] + 4 * t.j + (wide ? 2 * rank : rank)) * kTileRows);
        for (int k = 0; k < n; ++k, ++it) {
          const int st = it % kStages;
          if (!mbar_wait(&s.empty[st], ((it / kStages) & 1) ^ 1, abort)) {
            ok = false;
            break;
          }
          // the bytes of both CTAs are counted on the first one's barrier
          if (rank == 0)
            mbar_arrive_expect_tx(&s.full[st], 2 * (kTileBytes + (wide ? kTileBytes : kHalfTile)));
          tma_load_2d_pair(s.a[st], &maps.tile, &s.full[st], 0, 0, ya + k * kTileRows);
          if (kSym) {
            tma_load_2d_pair(s.b[st], wide ? &maps.tile : &maps.half, &s.full[st], 0, 0,
                             yb + k * kTileRows);
          } else {
            const int32_t y = yb + (k >> 1) * 2 * e.nb * kTileRows + (k & 1) * 64;
            tma_load_2d_pair(s.b[st], &maps.half, &s.full[st], 0, 0, y);
            if (wide)
              tma_load_2d_pair(s.b[st] + kHalfTile, &maps.half, &s.full[st], 0, 0, y + kTileRows);
          }
        }
      }
      s.issued = it;
    }
  } else if (warp == 1) {
    if (elect_one() && rank == 0) {
      int it = 0, ti = 0;
      bool ok = true;
      for (int w = cid; ok && w < n_tiles; w += n_clusters, ++ti) {
        const Tile t = tiles[w];
        const int n = steps(list.entries[t.matrix]);
        const uint32_t idesc = idesc_f16(2 * kBlock, t.width, !kSym);
        const int acc = ti & 1;
        if (!mbar_wait(&s.acc_empty[acc], ((ti >> 1) & 1) ^ 1, abort)) break;
        tc_fence_after();
        const uint32_t d = tmem + static_cast<uint32_t>(acc * kWide);
        for (int k = 0; k < n; ++k, ++it) {
          const int st = it % kStages;
          if (!mbar_wait(&s.full[st], (it / kStages) & 1, abort)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint64_t ad = sdesc_sw128(smem_u32(s.a[st]), 16, 1024);
          const uint64_t bd = kSym ? sdesc_sw128(smem_u32(s.b[st]), 16, 1024)
                                   : sdesc_sw128(smem_u32(s.b[st]), kHalfTile, 1024);
#pragma unroll
          for (int q = 0; q < kK / 16; ++q)   // 16 of K: 32 bytes of a row, or 16 rows
            mma_bf16_ss_pair(d, ad + 2 * q, bd + (kSym ? 2 : 128) * q, idesc,
                             (k | q) != 0 ? 1u : 0u);
          mma_commit_pair(&s.empty[st], kPairMask);
        }
        if (ok) mma_commit_pair(&s.acc_full[acc], kPairMask);
      }
      s.consumed = it;
      mma_commit_pair(&s.drain, 0x1);
      mbar_wait_limited(&s.drain, 0, kWaitLimitNs);
    }
  } else {
    const int ew = warp - 2, q = warp & 3, half = ew >> 2;
    constexpr bool kReads = kPhase != kGram;
    auto part_of = [&](const Tile& t) {
      return Part{(2 * t.i + rank) * kBlock + q * 32, t.j * kWide + half * (t.width >> 1),
                  t.width >> 6};
    };
    // map row of the piece at (row, col) of a matrix whose tiles begin at `first`, row_tiles a
    // block row; its map column is col & 32
    auto piece_row = [&](int64_t first, int row_tiles, int row, int col) {
      return static_cast<int32_t>((first + static_cast<int64_t>(row >> 7) * row_tiles + (col >> 6)) *
                                      kTileRows + (row & 127));
    };
    // The copies run two pieces ahead, over the ends of tiles.
    int ahead_w = cid, ahead_c = 0, loads = 0;
    auto load_next = [&]() {
      if (!kReads || ahead_w >= n_tiles) return;
      const Tile t = tiles[ahead_w];
      const Entry& e = list.entries[t.matrix];
      const Part p = part_of(t);
      const int place = loads % kPlaces, col = p.col + 32 * ahead_c;
      if (lane == 0) {
        uint64_t* bar = &s.piece_full[ew][place];
        if (kPhase == kSquare) {
          mbar_arrive_expect_tx(bar, kPiece * 2);
          tma_load_2d(s.piece[ew][place][0], &maps.piece, bar, col & 32,
                      piece_row(e.f, 2 * e.mb, p.row, col));
        } else {
          mbar_arrive_expect_tx(bar, 2 * kPiece * 2);
          tma_load_2d(s.piece[ew][place][0], &maps.piece, bar, col & 32,
                      piece_row(e.x[from], 2 * e.nb, p.row, col));
          tma_load_2d(s.piece[ew][place][1], &maps.piece, bar, col & 32,
                      piece_row(e.lo, 2 * e.nb, p.row, col));
        }
      }
      ++loads;
      if (++ahead_c == p.pieces) {
        ahead_c = 0;
        ahead_w += n_clusters;
      }
    };
    load_next();
    load_next();
    int ti = 0, done = 0;
    bool ok = true;
    for (int w = cid; ok && w < n_tiles; w += n_clusters, ++ti) {
      const Tile t = tiles[w];
      const Entry& e = list.entries[t.matrix];
      const Part p = part_of(t);
      const int row = p.row + lane, acc = ti & 1;
      const bool mirrored = kSym && t.i != t.j && p.row < e.mb * kBlock;
      float di = 0.f, ae = 0.f;
      if (kPhase == kSquare) di = e.d[row];
      if (!kSym) ae = kA + e.e[row];
      if (!mbar_wait_warp(&s.acc_full[acc], (ti >> 1) & 1, abort)) break;
      tc_fence_after();
      for (int c = 0; c < p.pieces; ++c, ++done) {
        const int col = p.col + 32 * c, place = done % kPlaces;
        uint16_t *one = s.piece[ew][place][0], *two = s.piece[ew][place][1];
        float dj = 0.f;
        if (kPhase == kSquare) dj = e.d[col + lane];
        uint32_t v[32];
        tmem_ld32(tmem + (static_cast<uint32_t>(q * 32) << 16) + acc * kWide + (col - t.j * kWide),
                  v);
        if (kReads) {
          if (!mbar_wait_warp(&s.piece_full[ew][place], (done / kPlaces) & 1, abort)) {
            tmem_ld_wait();
            ok = false;
            break;
          }
        } else {                          // the copy out of this place has read it
          if (lane == 0) bulk_wait_group_read1();
          __syncwarp();
        }
        tmem_ld_wait();
        if (c == p.pieces - 1) {          // this warp is done with the accumulator
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_remote(&s.acc_empty[acc], 0);
        }
        if constexpr (kSym) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            float x[8];
            if constexpr (kPhase == kGram) {
#pragma unroll
              for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(v[8 * k + i]) * (1.f / kScale);
              if (row >= col && row < col + 32) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                  if (row == col + 8 * k + i) {
                    e.d[row] = x[i] * (1.f / kScale);
                    x[i] = 0.f;
                  }
              }
            } else {
              float off[8];
              Granule<__half>::unpack(*piece_at(one, lane, k), off);
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const float ff = __uint_as_float(v[8 * k + i]) * (1.f / kScale);   // scaled once
                const float d2 = di + __shfl_sync(0xffffffffu, dj, 8 * k + i);
                x[i] = fmaf(kC, fmaf(d2, off[i], ff), kB * off[i]);
                if (row == col + 8 * k + i) {
                  e.e[row] = fmaf(kC, fmaf(di, di, ff * (1.f / kScale)), kB * di);
                  x[i] = 0.f;
                }
              }
            }
            const uint4 h = Granule<__half>::pack(x);
            *piece_at(one, lane, k) = h;
            if (mirrored) {
              const uint32_t words[4] = {h.x, h.y, h.z, h.w};
#pragma unroll
              for (int i = 0; i < 8; ++i)
                *value_in(two, 8 * k + i, lane) =
                    static_cast<uint16_t>(words[i >> 1] >> (16 * (i & 1)));
            }
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            const int64_t to = kPhase == kGram ? e.f : e.g;
            tma_store_2d(&maps.piece, one, col & 32, piece_row(to, 2 * e.mb, p.row, col));
            if (mirrored)
              tma_store_2d(&maps.piece, two, p.row & 32, piece_row(to, 2 * e.mb, col, p.row));
            bulk_commit_group();
          }
        } else {
          float x[32];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            float h[8], l[8];
            Granule<__half>::unpack(*piece_at(one, lane, k), h);
            Granule<__half>::unpack(*piece_at(two, lane, k), l);
#pragma unroll
            for (int i = 0; i < 8; ++i)
              x[8 * k + i] = fmaf(ae, fmaf(l[i], 1.f / kLoScale, h[i]),
                                  __uint_as_float(v[8 * k + i]) * (1.f / kScale));
          }
          if constexpr (kPhase == kApply) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              uint4 h, l;
              split(x + 8 * k, &h, &l);
              *piece_at(one, lane, k) = h;
              *piece_at(two, lane, k) = l;
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
              tma_store_2d(&maps.piece, one, col & 32,
                           piece_row(e.x[from ^ 1], 2 * e.nb, p.row, col));
              tma_store_2d(&maps.piece, two, col & 32, piece_row(e.lo, 2 * e.nb, p.row, col));
              bulk_commit_group();
            }
          } else {
            // 32 x 32 values to the weights: lanes along what is contiguous there, which for
            // a wide matrix are columns (the values change places in shared memory)
            if (!e.tall) {
              float* swap = reinterpret_cast<float*>(one);
              __syncwarp();               // every lane has read its part of the piece
#pragma unroll
              for (int i = 0; i < 32; ++i) swap[lane * 32 + ((i + lane) & 31)] = x[i];
              __syncwarp();
#pragma unroll
              for (int i = 0; i < 32; ++i) x[i] = swap[i * 32 + ((lane + i) & 31)];
              __syncwarp();
              fence_proxy_async_smem();
            }
            const int outer = e.tall ? col : p.row, inner = (e.tall ? p.row : col) + lane;
            const int outers = e.tall ? e.n : e.m, inners = e.tall ? e.m : e.n;
            if (inner < inners) {
              const int64_t at = static_cast<int64_t>(outer) * inners + inner;
              const int some = outers - outer < 32 ? outers - outer : 32;
              if (!a.muon) {
                store_rows(x, reinterpret_cast<__nv_bfloat16*>(e.out) + at, inners, some,
                           1.f / kScale);
              } else {
                const float step = -(a.lr * e.scale) * (1.f / kScale);
                if (e.param_type == DORA_F32)
                  update_rows(x, static_cast<float*>(e.param) + at, inners, some, a.keep, step);
                else if (e.param_type == DORA_BF16)
                  update_rows(x, static_cast<__nv_bfloat16*>(e.param) + at, inners, some, a.keep,
                              step);
                else
                  update_rows(x, static_cast<__half*>(e.param) + at, inners, some, a.keep, step);
                if (e.copy != nullptr)
                  store_rows(x, reinterpret_cast<__nv_bfloat16*>(e.copy) + at, inners, some, 1.f);
              }
            }
            __syncwarp();
          }
        }
        if (kReads) {
          // the place two pieces on was copied out one piece ago
          if (kPhase != kLast && lane == 0) bulk_wait_group_read1();
          __syncwarp();
          load_next();
        }
      }
    }
    if (lane == 0) {
      bulk_wait_group0();                 // copies are done before the CTA ends
      // after an abort: those that nobody waited for
      for (; kReads && done < loads; ++done)
        mbar_wait_limited(&s.piece_full[ew][done % kPlaces], (done / kPlaces) & 1,
                          100ull * 1000 * 1000);
    }
    __syncwarp();
  }

  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (*abort) {
    if (threadIdx.x == 0) {
      list.header->abort = 1;
      record_status(a.status, DORA_ERR_TIMEOUT);
      if (rank == 0)                      // loads that were issued but never consumed land first
        for (int it = s.consumed; it < s.issued; ++it)
          mbar_wait_limited(&s.full[it % kStages], (it / kStages) & 1, 100ull * 1000 * 1000);
    }
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, 2 * kWide);
  }
  cluster_sync();                         // no CTA leaves while its peer may still signal it
}

}  // namespace ortho
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

int64_t round256(int64_t n) { return (n + 255) / 256 * 256; }

bool aligned_to(const void* p, int32_t dtype) {
  return (reinterpret_cast<uintptr_t>(p) & (dtype == DORA_F32 ? 3u : 1u)) == 0;
}
bool known_type(int32_t t) { return t >= DORA_BF16 && t <= DORA_F32; }

// Sizes of a matrix, and of all of them.
struct Shape {
  int32_t m, n, mb, nb;
  int64_t chunks, x_tiles, f_tiles, sym, all, diag;   // diag: blocks of 128 of a diagonal
};
Shape shape_of(const dora_matrix& t) {
  Shape s;
  s.m = t.rows < t.cols ? t.rows : t.cols;
  s.n = t.rows < t.cols ? t.cols : t.rows;
  s.mb = (s.m + 127) / 128;
  s.nb = (s.n + 127) / 128;
  s.chunks = (static_cast<int64_t>(s.m) * s.n + ortho::kChunk - 1) / ortho::kChunk;
  const int64_t pairs = (s.mb + 1) / 2;
  s.x_tiles = pairs * 2 * 2 * s.nb;
  s.f_tiles = pairs * 2 * 2 * s.mb;
  s.sym = pairs * (pairs + 1) / 2;
  s.all = pairs * ((s.nb + 1) / 2);
  s.diag = pairs * 2;
  return s;
}
struct Sizes {
  int64_t chunks = 0, x_tiles = 0, sym = 0, all = 0, tiles = 0, diag = 0;
  bool has_params = true, has_outs = true;
};

bool count_all(const dora_matrix* ms, int32_t count, Sizes* out) {
  Sizes z;
  for (int32_t i = 0; i < count; ++i) {
    const dora_matrix& t = ms[i];
    if (t.rows < 1 || t.cols < 1 || t.grad == nullptr || !known_type(t.grad_dtype) ||
        !aligned_to(t.grad, t.grad_dtype) || !isfinite(t.scale))
      return false;
    if ((t.param == nullptr) != (t.momentum == nullptr) ||
        (t.copy != nullptr && t.param == nullptr))
      return false;
    if (t.param != nullptr && (!known_type(t.param_dtype) || !aligned_to(t.param, t.param_dtype)))
      return false;
    if (!aligned_to(t.momentum, DORA_F32) || !aligned_to(t.copy, DORA_BF16) ||
        !aligned_to(t.out, DORA_BF16))
      return false;
    const Shape s = shape_of(t);
    if (s.m > ortho::kMaxShort || s.n > ortho::kMaxLong) return false;
    z.chunks += s.chunks;
    z.x_tiles += s.x_tiles;
    z.sym += s.sym;
    z.all += s.all;
    z.tiles += 3 * s.x_tiles + 2 * s.f_tiles;
    z.diag += s.diag;
    if (t.param == nullptr) z.has_params = false;
    if (t.out == nullptr) z.has_outs = false;
    // counted in 32 bits, the tiles' rows among them
    if (z.tiles > (1 << 23) || z.chunks > (1 << 30)) return false;
  }
  *out = z;
  return true;
}

struct Places {
  int64_t entries, chunk_of, x, sym, all, partial, norm, ticket, diag, tiles, end;
};
Places places_of(const Sizes& z, int64_t count) {
  Places p;
  p.entries = round256(sizeof(ortho::Header));
  p.chunk_of = p.entries + round256(count * sizeof(ortho::Entry));
  p.x = p.chunk_of + round256(z.chunks * 4);
  p.sym = p.x + round256(z.x_tiles * sizeof(ortho::Tile));
  p.all = p.sym + round256(z.sym * sizeof(ortho::Tile));
  p.partial = p.all + round256(z.all * sizeof(ortho::Tile));
  p.norm = p.partial + round256(z.chunks * 8);
  p.ticket = p.norm + round256(count * 8);
  p.diag = p.ticket + round256(count * 4);
  p.tiles = p.diag + z.diag * 2 * 512;
  p.end = p.tiles + z.tiles * ortho::kTileBytes;
  return p;
}

ortho::List list_of(const dora_matrix_list& l) {
  const Sizes z = {l.chunks, l.x_tiles, l.symmetric, l.outputs, l.tiles, l.diagonals};
  const Places p = places_of(z, l.count);
  char* at = static_cast<char*>(l.data);
  ortho::List o;
  o.header = reinterpret_cast<ortho::Header*>(at);
  o.entries = reinterpret_cast<ortho::Entry*>(at + p.entries);
  o.chunk_of = reinterpret_cast<int32_t*>(at + p.chunk_of);
  o.x = reinterpret_cast<ortho::Tile*>(at + p.x);
  o.sym = reinterpret_cast<ortho::Tile*>(at + p.sym);
  o.all = reinterpret_cast<ortho::Tile*>(at + p.all);
  o.tiles = at + p.tiles;
  o.count = l.count;
  o.n_chunks = static_cast<int>(z.chunks);
  o.n_x = static_cast<int>(z.x_tiles);
  o.n_sym = static_cast<int>(z.sym);
  o.n_all = static_cast<int>(z.all);
  return o;
}

bool valid_list(const dora_matrix_list* l) {
  return l != nullptr && l->data != nullptr && l->count >= 1 && l->chunks >= 1 && l->tiles >= 1;
}

template <ortho::Phase kPhase>
int launch_product(const ortho::Maps& maps, const ortho::List& l, const ortho::Args& a, int from,
                   cudaStream_t stream) {
  constexpr int smem = sizeof(ortho::Smem);
  auto kern = ortho::product_kernel<kPhase>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return launched(e);
  const int tiles = kPhase == ortho::kGram || kPhase == ortho::kSquare ? l.n_sym : l.n_all;
  const int pairs = num_sms() / 2;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3(2 * (tiles < pairs ? tiles : pairs));
  cfg.blockDim = dim3(ortho::kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = pdl_enabled() ? 2 : 1;
  return launched(cudaLaunchKernelEx(&cfg, kern, maps, l, a, from));
}

int run(const dora_matrix_list* list, int32_t steps, const ortho::Args& a, cudaStream_t stream) {
  const int dev = device_or_error();
  if (dev != DORA_OK) return dev;
  const ortho::List l = list_of(*list);
  ortho::Maps maps;
  static_assert(sizeof(maps) == sizeof(list->map), "the maps' size is part of the interface");
  memcpy(&maps, list->map, sizeof(maps));
  const int most = num_sms() * ortho::kRowCtas;
  int e = launched(launch_pdl(ortho::momentum_kernel, dim3(l.n_chunks < most ? l.n_chunks : most),
                              dim3(ortho::kRowThreads), 0, stream, l, a));
  if (e == DORA_OK)
    e = launched(launch_pdl(ortho::normalise_kernel, dim3(l.n_x < most ? l.n_x : most),
                            dim3(ortho::kRowThreads), 0, stream, l, a));
  for (int s = 0; s < steps && e == DORA_OK; ++s) {
    e = launch_product<ortho::kGram>(maps, l, a, s & 1, stream);
    if (e == DORA_OK) e = launch_product<ortho::kSquare>(maps, l, a, s & 1, stream);
    if (e == DORA_OK)
      e = s + 1 < steps ? launch_product<ortho::kApply>(maps, l, a, s & 1, stream)
                        : launch_product<ortho::kLast>(maps, l, a, s & 1, stream);
  }
  return e;
}
}  // namespace

extern "C" {

size_t dora_matrix_list_size(const dora_matrix* matrices, int32_t count) {
  Sizes z;
  if (matrices == nullptr || count < 1 || !count_all(matrices, count, &z)) return 0;
  return static_cast<size_t>(places_of(z, count).end);
}

int dora_matrix_list_prepare(const dora_matrix* matrices, int32_t count, void* data, size_t bytes,
                             dora_matrix_list* list, dora_stream_t stream_) {
  Sizes z;
  if (matrices == nullptr || count < 1 || data == nullptr || list == nullptr ||
      (reinterpret_cast<uintptr_t>(data) & 255u) != 0 || !count_all(matrices, count, &z) ||
      bytes < static_cast<size_t>(places_of(z, count).end))
    return DORA_ERR_INVALID_ARG;
  const int dev = device_or_error();
  if (dev != DORA_OK) return dev;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  const Places p = places_of(z, count);
  char* at = static_cast<char*>(data);
  dora_matrix_list l = {};
  l.data = data;
  l.chunks = z.chunks;
  l.x_tiles = z.x_tiles;
  l.symmetric = z.sym;
  l.outputs = z.all;
  l.tiles = z.tiles;
  l.diagonals = z.diag;
  l.count = count;
  l.has_params = z.has_params;
  l.has_outs = z.has_outs;
  // all tiles as one tall matrix of 64 columns
  ortho::Maps maps;
  const uint64_t rows = static_cast<uint64_t>(z.tiles) * ortho::kTileRows;
  if (encode_tmap_2d_bf16(&maps.tile, at + p.tiles, 64, rows, 128, 64, 128) != 0 ||
      encode_tmap_2d_bf16(&maps.half, at + p.tiles, 64, rows, 128, 64, 64) != 0 ||
      encode_tmap_2d_bf16(&maps.piece, at + p.tiles, 64, rows, 128, 32, 32, 64) != 0)
    return DORA_ERR_CUDA;
  memcpy(l.map, &maps, sizeof(maps));
  const ortho::List o = list_of(l);
  int64_t tile = 0, chunk = 0, x = 0, sym = 0, all = 0, diag = 0;
  for (int32_t first = 0; first < count; first += ortho::kFill) {
    const int some = count - first < ortho::kFill ? count - first : ortho::kFill;
    ortho::FillArgs args = {};
    for (int i = 0; i < some; ++i) {
      const dora_matrix& t = matrices[first + i];
      const Shape s = shape_of(t);
      ortho::Entry& e = args.e[i];
      e.grad = t.grad;
      e.param = t.param;
      e.momentum = t.momentum;
      e.copy = t.copy;
      e.out = t.out;
      e.rows = t.rows;
      e.cols = t.cols;
      e.grad_type = t.grad_dtype;
      e.param_type = t.param_dtype;
      e.scale = t.scale;
      e.m = s.m;
      e.n = s.n;
      e.tall = t.rows > t.cols;
      e.mb = s.mb;
      e.nb = s.nb;
      e.x[0] = tile;
      e.x[1] = tile + s.x_tiles;
      e.lo = tile + 2 * s.x_tiles;
      e.f = tile + 3 * s.x_tiles;
      e.g = e.f + s.f_tiles;
      tile = e.g + s.f_tiles;
      e.d = reinterpret_cast<float*>(at + p.diag) + diag * 256;
      e.e = e.d + s.diag * 128;
      diag += s.diag;
      e.partial = reinterpret_cast<ortho::Squares*>(at + p.partial) + chunk;
      e.norm = reinterpret_cast<float2*>(at + p.norm) + first + i;
      e.ticket = reinterpret_cast<unsigned*>(at + p.ticket) + first + i;
      e.chunks = static_cast<int32_t>(s.chunks);
      e.first_chunk = chunk;
      e.first_x = x;
      e.first_sym = sym;
      e.first_all = all;
      chunk += s.chunks;
      x += s.x_tiles;
      sym += s.sym;
      all += s.all;
    }
    const int rc = launched(launch_pdl(ortho::fill_entries_kernel, dim3(1), dim3(32), 0, stream, o,
                                       first, some, args));
    if (rc != DORA_OK) return rc;
  }
  int64_t most = z.chunks > z.x_tiles ? z.chunks : z.x_tiles;
  if (z.sym > most) most = z.sym;
  const int rc = launched(launch_pdl(ortho::fill_tiles_kernel,
                                     dim3(static_cast<unsigned>((most + 127) / 128)), dim3(128), 0,
                                     stream, o));
  if (rc != DORA_OK) return rc;
  *list = l;
  return DORA_OK;
}

int dora_orthogonalize(const dora_matrix_list* list, int32_t steps, int32_t* status,
                       dora_stream_t stream) {
  if (!valid_list(list) || !list->has_outs || steps < 1 || steps > ortho::kMaxSteps)
    return DORA_ERR_INVALID_ARG;
  ortho::Args a = {};
  a.status = status;
  return run(list, steps, a, reinterpret_cast<cudaStream_t>(stream));
}

int dora_muon_step(const dora_matrix_list* list, double lr, double momentum, int32_t nesterov,
                   double weight_decay, int32_t steps, const float* clip, int32_t* status,
                   dora_stream_t stream) {
  if (!valid_list(list) || !list->has_params || steps < 1 || steps > ortho::kMaxSteps ||
      !isfinite(lr) || !(momentum >= 0. && momentum < 1.) || !(weight_decay >= 0.) ||
      !isfinite(weight_decay))
    return DORA_ERR_INVALID_ARG;
  ortho::Args a = {};
  a.clip = clip;
  a.muon = 1;
  a.nesterov = nesterov != 0;
  a.mu = static_cast<float>(momentum);
  a.omu = static_cast<float>(1. - momentum);
  a.lr = static_cast<float>(lr);
  a.keep = static_cast<float>(1. - lr * weight_decay);
  a.status = status;
  return run(list, steps, a, reinterpret_cast<cudaStream_t>(stream));
}

}  // extern "C"
