// Orthogonalised updates: Newton-Schulz iterations over a list of matrices, alone and as
// the end of a Muon step (momentum, orthogonalisation, weights).
//
// With X the update U (or U^T, so that X is m x n with m <= n) over its Frobenius norm,
//   A = X X^T,   X <- a X + (b A + c A^2) X
// brings every singular value near 1 (the quintic that K. Jordan et al. published with Muon, 2024,
// of coefficients a, b, c below, whose values stay below 1.21).  Three products an iteration on
// the tensor cores, the two symmetric ones by half: 3 m^2 n + m^3 operations.
//
// Precision.  What lies beside the directions that hold most of a matrix is raised by 3.4 an
// iteration, and every error there with it, up to 140 times in five: products of fp16 operands
// (11 bits) were up to 3e-2 off where few directions or few rows hold a gradient.  Therefore
// every operand is hi + lo, two fp16 values of 22 bits, of which the products take hi hi, hi lo
// and lo hi, added in fp32.  (Taking lo of X alone would leave up to 3e-3 where two rows are not
// zero: the roundings of few values do not average out.)  The diagonals of A and of
// B = b A + c A^2, which hold most of both once the singular values are near 1, stay out of the
// products, in fp32.  With A = D + F and B = E + G (D, E diagonal, F, G without one):
//   A^2 = D^2 + D F + F D + F F,    B X = E X + G X,
//   E = b D + c (D^2 + diag(F F)),  G = b F + c (D F + F D + F F) off the diagonal,
//   X <- (a + E) X + G X.
// (lo has no factor of its own: with X times 2^15, its smallest step is 1e-9 of a normalised
// update's average.)  Measured against the iteration in 64 bits (relative 2-norm): matrices of
// noise 1e-6 to 2e-5 (64 x 512 to 4096 x 4096), one direction over 1e-3 of noise 5e-5 to 2.3e-4
// (64 x 512 to 1024 x 1024), 6.6e-4 (4096 x 4096); the iteration in fp32 4e-6, 2.2e-4, 4.3e-4.
// What is left of it is how the tensor cores add: cut off, not rounded, so that long sums are
// too small, 7e-4 off for a side of 65536.
//
// Layout.  X, F and G are kept in tiles of 128 x 64 fp16 values (16 KB, rows of 128
// bytes): whatever the matrices' sizes, a few tensor maps describe all of them.  The first block
// of rows past a matrix' end is filled up with zeros; the second of a last pair is not
// defined, and nothing that is kept is made of it.  A tile is an operand either way: K-major
// (rows of X for X X^T) or MN-major (rows of X as the K of G X).
// X's halves, hi and lo, take turns in three slots (slot_tile).  F and G are symmetric: hi lies
// above the diagonal, the mirror image of lo below it, in as much memory as one of them takes.
// With T the matrix that is stored, F = T + T^T, in the blocks of the diagonal too; elsewhere one
// of the two terms is hi, the other lo.
//
// Measured (five iterations with momentum and weights): 96 matrices of 1024 x 1024 and 48 of
// 4096 x 1024, bf16 gradients and copies, fp32 weights: 13.1 ms, of which the two passes
// before the products 0.92; at three times their 5.4e12 operations the products run at 1.3
// PFLOP/s of 1.94.  72 of 384 x 384 to 1536 x 384 0.77 ms, four of 4096 x 1024 and its transpose
// 1.0, the actor's twelve small ones 85, with momentum and weights 88 us.  (Operands of 11 bits:
// 6.8, 0.50, 0.42 ms, 67 and 70 us.)
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>

#include "dora.h"
#include "dora_ptx.cuh"
#include "granule.cuh"
#include "token_ops.cuh"
#include "update_ptx.cuh"

namespace dora {
namespace ortho {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
// Factors of X and F in fp16, whose values stay below 1.21 and 1.5; G has none.
constexpr float kXScale = 32768.f, kFScale = 256.f;
constexpr int kMaxSteps = 32;
// Elements of a group of matrices, about.  A larger group hides the waits between a matrix'
// phases, a smaller one keeps X in L2; 96 of 1024 x 1024 and 48 of 4096 x 1024: 6 M elements
// 32.3 ms, 18 M 15.7, 32 M 13.5, 48 M 13.1, 128 M 13.1.
constexpr int64_t kGroup = 64 << 20;
constexpr int kTileRows = 128, kTileCols = 64;
constexpr int kTileBytes = kTileRows * kTileCols * 2;
constexpr int kChunk = 4096;              // elements of a matrix that a CTA takes at once
constexpr int kRowThreads = 256, kRowCtas = 4, kMomentumCtas = 3;
// Largest sides.  A's sums of n products are added 16 at a time into 32 bits, three times over,
// each time cut off rather than rounded, which makes A too small by up to 3 n 2^-28 of itself:
// with the longest n the result is 2.6e-3 off for it (130 x 2^18, noise).  A phase of the largest
// matrix, 2.1e14 operations, takes 0.2 s at the large list's rate; a wait's limit is 1 s.
constexpr int kMaxShort = 16384, kMaxLong = 262144;

struct Squares;

struct Entry {
  const void* grad;
  void* param;
  float* momentum;
  uint16_t *copy, *out;                   // bf16
  int32_t grad_type, param_type;
  float scale;
  int32_t m, n, tall;                     // X is m x n; tall: X = U^T
  int32_t quads;                          // what is written is aligned to four values, row by row
  int32_t mb, nb;                         // blocks of 128 rows, of 128 columns; X, F and G
                                          // have an even number of the first
  int64_t x, slot, f, g;                  // first tiles of X's three slots, tiles of each, F, G
  float *d, *e;                           // the diagonals of A and B
  Squares* partial;                       // of its chunks
  float2* norm;                           // one over the norm of u 2^-k, and 2^-k
  unsigned* ticket;                       // chunks done; zero between calls
  unsigned* done;                         // CTAs' parts of its tiles that are done, in this call
  int32_t chunks;
  int32_t n_sym, n_all;                   // its tiles of A and B, and of half of X
  int32_t sym_width, all_width;           // their columns
  int32_t parts;                          // of a small matrix: CTAs
  // first of its chunks, of its tiles of X and of its output tiles among the list's
  int64_t first_chunk, first_x, first_sym, first_all;
};

struct Header {
  int abort;                              // a bounded wait of this call has run out
  unsigned ticket;                        // tiles taken in this call
  int n_groups;
  int pad[61];
};

// The tiles of a group of matrices.
struct Group {
  int sym0, sym1, all0, all1;
};

// One piece of work: a pair of block rows (or one) of a matrix, its first column, of A and B in
// blocks, of a half of X in tiles, and its columns.
struct Tile {
  int32_t matrix, i, j, width;
};

struct List {
  Header* header;
  Entry* entries;                         // `count` of them, then the small matrices'
  int32_t* chunk_of;                      // matrix of every chunk
  Tile *x, *sym, *all;
  Group* groups;
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
    if (args.e[threadIdx.x].ticket != nullptr) *args.e[threadIdx.x].ticket = 0;
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
    const Entry& e = list.entries[q];
    const int at = static_cast<int>(t - e.first_all), each = e.all_width / kTileCols;
    const int w = (e.nb + each - 1) / each, j = at % w * each;
    list.all[t] = Tile{q, at / w, j, (j + each <= e.nb ? each : e.nb - j) * kTileCols};
  }
  if (t < list.n_sym) {
    const int q = matrix_of(list, t, [](const Entry& e) { return e.first_sym; });
    const Entry& e = list.entries[q];
    const int each = e.sym_width / 128;
    int at = static_cast<int>(t - e.first_sym), i = 0, left = (e.mb + each - 1) / each;
    while (at >= left) {
      at -= left;
      ++i;
      left = (e.mb - 2 * i + each - 1) / each;
    }
    const int j = 2 * i + at * each;
    list.sym[t] = Tile{q, i, j, j + each <= e.mb ? e.sym_width : 128};
  }
  if (t == 0 && list.count > 0) {         // whole matrices until a group is large enough
    int n = 0;
    int64_t size = 0;
    Group g = {0, 0, 0, 0};
    for (int q = 0; q < list.count; ++q) {
      const Entry& e = list.entries[q];
      g.sym1 += e.n_sym;
      g.all1 += e.n_all;
      size += static_cast<int64_t>(e.m) * e.n;
      if (size >= kGroup || q == list.count - 1) {
        list.groups[n++] = g;
        g.sym0 = g.sym1;
        g.all0 = g.all1;
        size = 0;
      }
    }
    list.header->n_groups = n;
  }
}

__device__ __forceinline__ int size_of(int type) { return type == DORA_F32 ? 4 : 2; }

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
        w[j >> 1] |= static_cast<uint32_t>(static_cast<const uint16_t*>(p)[k + j])
                     << (16 * (j & 1));
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

__device__ __forceinline__ void store_quad(const float* v, void* p, int type, int64_t k) {
  if (type == DORA_F32)
    *reinterpret_cast<uint4*>(static_cast<float*>(p) + k) = Granule<float>::pack(v);
  else
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p) + k) =
        type == DORA_BF16 ? make_uint2(Granule<__nv_bfloat16>::pair(v[0], v[1]),
                                       Granule<__nv_bfloat16>::pair(v[2], v[3]))
                          : make_uint2(Granule<__half>::pair(v[0], v[1]),
                                       Granule<__half>::pair(v[2], v[3]));
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
// Momentum, and the update's norm: memory (201 M elements of bf16 gradients 452 us, 4.5 TB/s).
// The loads of a chunk are all on their way while the one before is joined behind a barrier, and
// a CTA says once a matrix what it has done (for every chunk, with its fence: 584 us; three CTAs
// an SM, whose registers are enough, 452, four 492).  A CTA takes a run of chunks, a matrix's one
// after the other.  A thread sums its squares in fp32; where that leaves the middle of the range,
// it sums those of u 2^-k,
// with k the exponent of its largest |u|, so that no finite update
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

__global__ void __launch_bounds__(kRowThreads, kMomentumCtas) momentum_kernel(List list, Args a) {
  constexpr int kPer = kChunk / kRowThreads;
  __shared__ Squares scratch[kRowThreads / 32];
  __shared__ bool last;
  pdl_wait();
  if (skipped(a)) return;
  const float f = factor(a);
  if (blockIdx.x == 0) {                  // what the products count
    if (threadIdx.x == 0) {
      list.header->abort = 0;
      list.header->ticket = 0;
    }
    for (int i = threadIdx.x; i < list.count; i += kRowThreads) *list.entries[i].done = 0;
  }
  int c = static_cast<int>(static_cast<int64_t>(list.n_chunks) * blockIdx.x / gridDim.x);
  const int end = static_cast<int>(static_cast<int64_t>(list.n_chunks) * (blockIdx.x + 1) /
                                   gridDim.x);
  const Entry* at = list.entries + (c < end ? list.chunk_of[c] : 0);
  uint4 qg[kPer / 4], qm[kPer / 4];
  // quads of a chunk's elements, all on their way before the first is looked at
  auto quads_of = [&](const Entry& e) {
    return in_quads(e.grad, e.grad_type) && (!a.muon || in_quads(e.momentum, DORA_F32));
  };
  auto elements = [&](const Entry& e, int64_t from) {
    const int64_t left = static_cast<int64_t>(e.m) * e.n - from;
    return left < kChunk ? static_cast<int>(left) : kChunk;
  };
  auto load = [&](const Entry& e, int chunk) {
    const int64_t from = static_cast<int64_t>(chunk - e.first_chunk) * kChunk;
    const int some = elements(e, from);
    const bool quads = quads_of(e);
    const char* g = static_cast<const char*>(e.grad) + from * size_of(e.grad_type);
    const float* m = e.momentum + from;
    if (quads && some == kChunk) {
#pragma unroll
      for (int i = 0; i < kPer / 4; ++i) {
        const int k = 4 * (threadIdx.x + i * kRowThreads);
        qg[i] = whole_quad(g, e.grad_type, k);
        qm[i] = a.muon ? whole_quad(m, DORA_F32, k) : make_uint4(0, 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kPer / 4; ++i) {
        const int k = 4 * (threadIdx.x + i * kRowThreads);
        qg[i] = load_quad(g, e.grad_type, k, some, quads);
        qm[i] = a.muon ? load_quad(m, DORA_F32, k, some, quads) : make_uint4(0, 0, 0, 0);
      }
    }
  };
  unsigned chunks = 0;                    // of the matrix, by this CTA
  if (c < end) load(*at, c);
  for (; c < end; ++c) {
    const Entry& e = *at;
    const int64_t from = static_cast<int64_t>(c - e.first_chunk) * kChunk;
    const int some = elements(e, from);
    const bool quads = quads_of(e);
    float* momentum = e.momentum + from;
    float u[kPer];
#pragma unroll
    for (int i = 0; i < kPer / 4; ++i) {
      const int k = 4 * (threadIdx.x + i * kRowThreads);
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
      if (quads && k + 4 <= some) {
        *reinterpret_cast<uint4*>(momentum + k) = Granule<float>::pack(m);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (k + j < some) momentum[k + j] = m[j];
      }
    }
    Squares sum = squares_of(u);
    // the next chunk's are on their way while this one's squares are joined
    const bool more = c + 1 < end && c + 1 - e.first_chunk < e.chunks;
    if (c + 1 - e.first_chunk >= e.chunks) ++at;
    if (c + 1 < end) load(*at, c + 1);
    sum = block_squares(sum, scratch);
    if (threadIdx.x == 0) e.partial[c - e.first_chunk] = sum;
    ++chunks;
    if (more) continue;
    // the matrix' last chunk here: one fence and one count for all of them
    if (threadIdx.x == 0)
      last = take_tickets(e.ticket, chunks) == static_cast<unsigned>(e.chunks) - chunks;
    chunks = 0;
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
// X lies in two halves of nb columns of tiles, each hi, then lo, in two of three slots.  An
// iteration writes the new left half to the third and the new right one over the old left one, so
// that `turn` iterations (mod 3) later the left half is in slot -turn, the right one in the next.
// What an iteration writes lies where the next one looks for it.
__device__ __forceinline__ int64_t slot_tile(const Entry& e, int turn, int half) {
  const int at = half - turn;
  return e.x + (at < 0 ? at + 3 : at) * e.slot;
}
// Tile of hi (part 0) or lo (1) of a block row and a column of tiles.
__device__ __forceinline__ int64_t x_tile(const Entry& e, int turn, int row, int col, int part) {
  const int half = col >= e.nb ? 1 : 0;
  return slot_tile(e, turn, half) + part * (e.slot / 2) + static_cast<int64_t>(row) * e.nb + col -
         half * e.nb;
}

// The gradient and the momentum of eight columns from `col` of a row of X, as they are loaded:
// nothing is made of them before all loads of a thread are on their way.  What is not there is 0.
struct Eight {
  uint32_t g[8], m[8];
};
__device__ __forceinline__ bool aligned16(const void* p) {
  return (reinterpret_cast<uintptr_t>(p) & 15u) == 0;
}
// Whether eight columns are 16-byte loads.
__device__ __forceinline__ bool in_eights(const Entry& e, const Args& a) {
  return !e.tall && (e.n & 7) == 0 && aligned16(e.grad) && (!a.muon || aligned16(e.momentum));
}
__device__ __forceinline__ void put(uint32_t* w, uint4 q) {
  w[0] = q.x;
  w[1] = q.y;
  w[2] = q.z;
  w[3] = q.w;
}
__device__ __forceinline__ Eight load_eight(const Entry& e, const Args& a, bool eights, int row,
                                            int col) {
  Eight x;
  const int some = row < e.m ? e.n - col : 0;
  const int64_t step = e.tall ? e.m : 1;
  const int64_t k = e.tall ? static_cast<int64_t>(col) * e.m + row
                           : static_cast<int64_t>(row) * e.n + col;
  if (eights && some > 0) {               // a multiple of eight columns: all of them
    const uint4* g = reinterpret_cast<const uint4*>(static_cast<const char*>(e.grad) +
                                                    k * size_of(e.grad_type));
    put(x.g, g[0]);
    if (e.grad_type == DORA_F32) put(x.g + 4, g[1]);
    if (a.muon) {
      put(x.m, reinterpret_cast<const uint4*>(e.momentum + k)[0]);
      put(x.m + 4, reinterpret_cast<const uint4*>(e.momentum + k)[1]);
    }
    return x;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) x.g[i] = x.m[i] = 0u;
  if (e.grad_type == DORA_F32) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < some) x.g[i] = static_cast<const uint32_t*>(e.grad)[k + i * step];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < some) x.g[i] = static_cast<const uint16_t*>(e.grad)[k + i * step];
  }
  if (a.muon)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < some) x.m[i] = reinterpret_cast<const uint32_t*>(e.momentum)[k + i * step];
  return x;
}
// Their values; `packed`: 16-bit ones lie two in a word.
__device__ __forceinline__ void values_of(const Entry& e, const Eight& x, bool packed, float* d,
                                          float* m) {
  if (e.grad_type == DORA_F32) {
#pragma unroll
    for (int i = 0; i < 8; ++i) d[i] = __uint_as_float(x.g[i]);
  } else {
    const uint4 q = packed ? make_uint4(x.g[0], x.g[1], x.g[2], x.g[3])
                           : make_uint4(x.g[0] | x.g[1] << 16, x.g[2] | x.g[3] << 16,
                                        x.g[4] | x.g[5] << 16, x.g[6] | x.g[7] << 16);
    if (e.grad_type == DORA_BF16) Granule<__nv_bfloat16>::unpack(q, d);
    else Granule<__half>::unpack(q, d);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) m[i] = __uint_as_float(x.m[i]);
}

// hi and lo of eight values that are scaled already.
__device__ __forceinline__ void split(const float* v, uint4* hi, uint4* lo) {
  float rest[8], back[8];
  *hi = Granule<__half>::pack(v);
  Granule<__half>::unpack(*hi, back);
#pragma unroll
  for (int i = 0; i < 8; ++i) rest[i] = v[i] - back[i];
  *lo = Granule<__half>::pack(rest);
}

// Eight rows of a column of X, contiguous where X is the transpose.
__device__ __forceinline__ Eight load_down(const Entry& e, const Args& a, int row, int col) {
  Eight x = {};
  if (row >= e.m || col >= e.n) return x;   // a multiple of eight rows: all of them
  const int64_t k = static_cast<int64_t>(col) * e.m + row;
  const uint4* g = reinterpret_cast<const uint4*>(static_cast<const char*>(e.grad) +
                                                  k * size_of(e.grad_type));
  put(x.g, g[0]);
  if (e.grad_type == DORA_F32) put(x.g + 4, g[1]);
  if (a.muon) {
    put(x.m, reinterpret_cast<const uint4*>(e.momentum + k)[0]);
    put(x.m + 4, reinterpret_cast<const uint4*>(e.momentum + k)[1]);
  }
  return x;
}

// The normalised update into its tiles, two that lie side by side at a time; a CTA takes a run of
// them.  Memory (201 M elements 463 us, 4.3 TB/s): the norm must be known first, so that gradient
// and momentum are read a second time (the update in a buffer of its own, instead, would be
// written and read).  Where X is the transpose, eight of its rows are loaded at once and change
// places in shared memory (one by one, and a tile at a time: 572 us).
__global__ void __launch_bounds__(kRowThreads, kRowCtas) normalise_kernel(List list, Args a) {
  __shared__ __align__(16) uint16_t turned[2][kTileRows * kTileCols];   // hi, lo
  pdl_wait();
  if (skipped(a)) return;
  const float f = factor(a);
  const int pairs = list.n_x / 2;
  int t = static_cast<int>(static_cast<int64_t>(pairs) * blockIdx.x / gridDim.x);
  const int end = static_cast<int>(static_cast<int64_t>(pairs) * (blockIdx.x + 1) / gridDim.x);
  if (t >= end) return;
  const Tile first = list.x[2 * t];
  int matrix = first.matrix, ti = first.i, tj = first.j;
  for (; t < end; ++t) {
    const Entry& e = list.entries[matrix];
    const float2 norm = *e.norm;
    // of the tile and of the one beside it
    const auto hi = [&](int side) { return tile_at(list, x_tile(e, 0, ti, tj + side, 0)); };
    const auto lo = [&](char* p) { return p + e.slot / 2 * kTileBytes; };
    constexpr int kSome = 2;              // eights of a thread on their way at once
    // hi and lo of eight values
    auto finish = [&](const Eight& x, bool packed, uint4* h, uint4* l) {
      float d[8], m[8], v[8];
      values_of(e, x, packed, d, m);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        v[i] = update_of(a, d[i] * f, a.muon ? m[i] : 0.f) * norm.y * norm.x * kXScale;
      split(v, h, l);
    };
    if (e.tall && (e.m & 7) == 0 && aligned16(e.grad) && (!a.muon || aligned16(e.momentum))) {
      const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll 1
      for (int side = 0; side < 2; ++side) {
        // a warp takes 64 rows of four columns; 16-byte parts of a row change places with its
        // eights of rows
        auto place = [&](int y, int* r, int* c) {
          const int w = warp + y * (kRowThreads / 32);
          *r = 64 * (w & 1) + 8 * (lane & 7);
          *c = 4 * (w >> 1) + (lane >> 3);
        };
#pragma unroll 1
        for (int y0 = 0; y0 < 4; y0 += kSome) {
          Eight x[kSome];
#pragma unroll
          for (int y = 0; y < kSome; ++y) {
            int r, c;
            place(y0 + y, &r, &c);
            x[y] = load_down(e, a, ti * kTileRows + r, (tj + side) * kTileCols + c);
          }
#pragma unroll
          for (int y = 0; y < kSome; ++y) {
            int r, c;
            place(y0 + y, &r, &c);
            uint4 h, l;
            finish(x[y], true, &h, &l);
            const uint32_t hs[4] = {h.x, h.y, h.z, h.w}, ls[4] = {l.x, l.y, l.z, l.w};
            const int to = r * kTileCols + (((c >> 3) ^ ((r >> 3) & 7)) << 3) + (c & 7);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              turned[0][to + i * kTileCols] = static_cast<uint16_t>(hs[i >> 1] >> (16 * (i & 1)));
              turned[1][to + i * kTileCols] = static_cast<uint16_t>(ls[i >> 1] >> (16 * (i & 1)));
            }
          }
        }
        __syncthreads();
#pragma unroll
        for (int y = 0; y < kTileRows * 8 / kRowThreads; ++y) {
          const int w = threadIdx.x + y * kRowThreads, r = w >> 3, k = w & 7;
          const int from = r * kTileCols + ((k ^ ((r >> 3) & 7)) << 3);
          char* to = hi(side) + tile_offset(r, 8 * k);
          *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(&turned[0][from]);
          *reinterpret_cast<uint4*>(lo(to)) = *reinterpret_cast<const uint4*>(&turned[1][from]);
        }
        __syncthreads();
      }
    } else {
      const bool eights = in_eights(e, a);
      // pieces of eight columns, the lanes along what is contiguous in the matrix
      auto place = [&](int y, int* r, int* piece) {
        const int w = threadIdx.x + y * kRowThreads;
        *r = e.tall ? w % kTileRows : w / 16;
        *piece = e.tall ? w / kTileRows : w % 16;
      };
#pragma unroll 1
      for (int y0 = 0; y0 < kTileRows * 16 / kRowThreads; y0 += kSome) {
        Eight x[kSome];
#pragma unroll
        for (int y = 0; y < kSome; ++y) {
          int r, piece;
          place(y0 + y, &r, &piece);
          x[y] = load_eight(e, a, eights, ti * kTileRows + r, tj * kTileCols + piece * 8);
        }
#pragma unroll
        for (int y = 0; y < kSome; ++y) {
          int r, piece;
          place(y0 + y, &r, &piece);
          // a row or columns past the end were loaded one by one
          const bool packed = eights && ti * kTileRows + r < e.m &&
                              tj * kTileCols + piece * 8 < e.n;
          uint4 h, l;
          finish(x[y], packed, &h, &l);
          char* to = hi(piece >> 3) + tile_offset(r, piece % 8 * 8);
          *reinterpret_cast<uint4*>(to) = h;
          *reinterpret_cast<uint4*>(lo(to)) = l;
        }
      }
    }
    tj += 2;
    if (tj == 2 * e.nb) {
      tj = 0;
      if (++ti == 2 * ((e.mb + 1) / 2)) {
        ti = 0;
        ++matrix;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// The products, all iterations of all matrices in one launch.  The work is a list of
// output tiles (256 rows, 256 or 128 columns) in an order in which each depends on
// earlier ones only: the matrices in groups, of a group one phase of all its
// matrices after the other.  CTA pairs take the tiles as they get done with others
// (a counter), and a tile waits until its matrix has finished the phase before (a counter
// a matrix).  Whoever holds a tile runs, and the earliest unfinished one waits for
// nobody, so that there is always progress, however many CTAs are resident.
//
// One MMA spans a pair, each CTA holding its 128 rows of the left operand and half of the right
// one.  64 of K take two stages of 32 KB in each: hi of both operands, or F and G as they lie, then
// lo, or their mirror images, MN-major; of the four products of their parts lo lo is left out, but
// where a part is hi and lo at once (K in a block of the diagonal).  In a CTA one warp copies
// operands into a ring of stages, one issues the MMAs (in the first CTA) into one of two
// accumulators, and eight finish the other one, 32 x 32 values at a time: what they read besides
// (F; X hi and lo) a warp copies ahead of them, into three places for each, where it is written
// over, and from where another one copies it out and reports the tile.  The second CTA's idle MMA
// warp fetches the tiles.
//
// What bounds it: with many stages of K a tile, the tensor cores' three products and the
// operands' way from L2, 128 KB for 64 of K and a pair; with few, the epilogues and X's traffic;
// with few tiles, the chain of phases.
// ---------------------------------------------------------------------------
enum Phase { kGram, kSquare, kApply, kLast };

constexpr int kStages = 4;                // 5 (two places): large list 12.8 ms instead of 13.1,
                                          // four large matrices 1.00 instead of 0.99
constexpr int kBlock = 128;               // rows of a CTA's part of an output tile
constexpr int kWide = 256;                // columns of one
constexpr int kK = 64;                    // of a stage
constexpr int kEpiWarps = 8;
constexpr int kThreads = 128 + 32 * kEpiWarps;
constexpr int kHalfTile = kTileBytes / 2; // 64 rows
constexpr int kPlaces = 3;
constexpr int kPiece = 32 * 32;           // values that a warp finishes at once
constexpr int kRing = 4;                  // tiles fetched ahead (384-wide blocks' list, four large
                                          // matrices: 2 782 and 919 us, 3 758 and 975, 4 769 and
                                          // 991, 6 789 and 975)
constexpr int kTileArrivals = 2;           // at a matrix' counter: one a CTA
constexpr uint16_t kPairMask = 0x3;

// A tile as the roles of a pair receive it, with its matrix' entry: waiting for other CTAs
// empties the L1 cache, and every look at the list would go to L2.
struct Task {
  int matrix, i, j, width, phase, turn, need, half;
  Entry e;
};
constexpr int kTaskWords = sizeof(Task) / 4;

struct Smem {
  uint8_t a[kStages][kTileBytes];
  uint8_t b[kStages][kTileBytes];
  uint16_t piece[kPlaces][2][2][4][kPiece];   // of each half of the columns, four warps' rows
  float dj[kPlaces][2][32];               // of the diagonal of A
  uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2], drain;
  uint64_t piece_full[2][kPlaces], piece_done[2][kPlaces], piece_empty[2][kPlaces];
  uint64_t task_full[kRing], task_empty[kRing];
  Task task[kRing];
  uint32_t tmem;
  int abort, issued, consumed;
};
static_assert(sizeof(Smem) <= 227 * 1024, "shared memory");

// The maps of all tiles: whole ones, their halves of 64 rows, 32 columns of 128 and of 32 rows.
struct Maps {
  CUtensorMap tile, half, column, piece;
};

__host__ __device__ constexpr uint32_t idesc_f16(int m, int n, bool b_mn_major,
                                                 bool a_mn_major = false) {
  return (1u << 4) | ((a_mn_major ? 1u : 0u) << 15) | ((b_mn_major ? 1u : 0u) << 16) |
         (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(m >> 4) << 24);
}

// 16-byte part `p` of lane's row of a piece (rows of 64 bytes, as a copy swizzles them).
__device__ __forceinline__ uint4* piece_at(uint16_t* piece, int row, int p) {
  return reinterpret_cast<uint4*>(reinterpret_cast<char*>(piece) + row * 64 +
                                  ((p ^ ((row >> 1) & 3)) << 4));
}
__device__ __forceinline__ uint16_t* value_in(uint16_t* piece, int row, int c) {
  return reinterpret_cast<uint16_t*>(piece_at(piece, row, c >> 3)) + (c & 7);
}

// Between CTAs: what a warp wrote, by copies or by itself, is there for whoever has seen
// the counter that it adds to afterwards.
__device__ __forceinline__ void fence_proxy_async_all() {
  asm volatile("fence.proxy.async;" ::: "memory");
}
__device__ __forceinline__ void signal(unsigned* done) {
  asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(done) : "memory");
}
__device__ __forceinline__ unsigned load_acquire(const unsigned* p) {
  unsigned v;
  asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ unsigned load_relaxed(const unsigned* p) {
  unsigned v;
  asm volatile("ld.relaxed.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
// Wait until at most one bulk group of this thread has not completed.
__device__ __forceinline__ void bulk_wait_group1() {
  asm volatile("cp.async.bulk.wait_group 1;" ::: "memory");
}
// Waits until `need` arrivals were counted; the limit runs anew with each that comes.
__device__ __forceinline__ bool wait_done(const unsigned* done, unsigned need, volatile int* abort,
                                          const Header* header) {
  unsigned v = load_relaxed(done);
  if (v < need) {
    uint64_t t0 = globaltimer_ns();
    while (true) {
      const unsigned now = load_relaxed(done);
      if (now >= need) break;
      if (*abort) return false;
      if (now != v) {
        v = now;
        t0 = globaltimer_ns();
      } else if (globaltimer_ns() - t0 > kWaitLimitNs || __ldcg(&header->abort) != 0) {
        *abort = 1;
        return false;
      }
      __nanosleep(32);
    }
  }
  (void)load_acquire(done);
  fence_proxy_async_all();
  return true;
}

// The weights of a CTA's part of an output tile to L2, a line a lane.
__device__ __forceinline__ void prefetch_weights(const Entry& e, int block, int col, int width,
                                                 int lane) {
  const int inners = e.tall ? e.m : e.n, outers = e.tall ? e.n : e.m;
  const int inner = e.tall ? block * kBlock : col, outer = e.tall ? col : block * kBlock;
  const int inner_end = min(inner + (e.tall ? kBlock : width), inners);
  const int outer_end = min(outer + (e.tall ? width : kBlock), outers);
  const int step = 128 / size_of(e.param_type);
  for (int o = outer + lane; o < outer_end; o += 32)
    for (int i = inner; i < inner_end; i += step)
      asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const char*>(e.param) +
                                                    (static_cast<int64_t>(o) * inners + i) *
                                                        size_of(e.param_type)));
}

// The pieces of a warp's half of a tile, 32 columns each; none in the second of a pair of block
// rows where the matrix ends with the first: what lies there is not defined, and no other row is
// made of it.
__device__ __forceinline__ int pieces_of(const Task& t, int block) {
  return block < t.e.mb ? t.width >> 6 : 0;
}
// A tile's first column, of A and B or of X.
__device__ __forceinline__ int first_column(const Task& t) {
  return t.phase < kApply ? t.j * kBlock : (t.j + t.half * t.e.nb) * kTileCols;
}

// Two values of a 16-byte part, as a pair of fp32.
__device__ __forceinline__ uint64_t halves(uint32_t w) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
  return f2_pack(f.x, f.y);
}
__device__ __forceinline__ uint32_t to_halves(uint64_t v) {
  float lo, hi;
  f2_unpack(v, lo, hi);
  return Granule<__half>::pair(lo, hi);
}
__device__ __forceinline__ uint64_t twice(float v) { return f2_pack(v, v); }

__device__ __forceinline__ float half_value(uint16_t w) {
  return __half2float(__ushort_as_half(w));
}
__device__ __forceinline__ uint16_t half_bits(float v) {
  return __half_as_ushort(__float2half_rn(v));
}
// Where a 32 x 32 piece of F or G lies: above the diagonal, on it, or below, where it is made of
// its mirror image.
enum Place { kAbove, kOn, kBelow };
__device__ __forceinline__ Place place_of(int row0, int col) {
  return col > row0 ? kAbove : (col == row0 ? kOn : kBelow);
}

// One value a lane in each of `some` rows: keep times the weight at p (none: 0) plus value(row),
// to p and, rounded, to copy; kAtOnce weights are loaded at a time (a small matrix' 32 rows at
// once: 2 us of the actor's step less; the product kernel has no registers for more than 16).
template <int kAtOnce, typename T, typename F>
__device__ __forceinline__ void write_rows(T* p, __nv_bfloat16* copy, int64_t pitch, int some,
                                           float keep, F value) {
  for (int i0 = 0; i0 < some; i0 += kAtOnce) {
    T old[kAtOnce];                       // all on their way before the first is used
    if (p != nullptr)
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i)
        if (i0 + i < some) old[i] = p[(i0 + i) * pitch];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i)
      if (i0 + i < some) {
        float w = value(i0 + i);
        if (p != nullptr) {
          w = fmaf(to_float(old[i]), keep, w);
          from_float(w, p + (i0 + i) * pitch);
        }
        if (copy != nullptr) from_float(w, copy + (i0 + i) * pitch);
      }
  }
}

// 32 x 32 values in rows of 128 bytes, 16 rows in `low`, 16 in `high`; their 16-byte parts change
// places with the row.
__device__ __forceinline__ float4* swapped_part(uint16_t* low, uint16_t* high, int i, int k) {
  return reinterpret_cast<float4*>(i < 16 ? low : high) + (i & 15) * 8 + (k ^ (i & 7));
}
// Those of them that exist to the weights (or out), a value a lane: where sizes or alignment do
// not allow four.
template <int kAtOnce>
__device__ __forceinline__ void finish_ragged(void* param, int param_type, __nv_bfloat16* copy,
                                           int64_t pitch, int some, float keep, float step,
                                           uint16_t* low, uint16_t* high) {
  const int lane = threadIdx.x & 31;
  const auto value = [&](int i) {
    return reinterpret_cast<const float*>(swapped_part(low, high, i, lane >> 2))[lane & 3] * step;
  };
  if (param == nullptr || param_type == DORA_F32)
    write_rows<kAtOnce>(static_cast<float*>(param), copy, pitch, some, keep, value);
  else if (param_type == DORA_BF16)
    write_rows<kAtOnce>(static_cast<__nv_bfloat16*>(param), copy, pitch, some, keep, value);
  else
    write_rows<kAtOnce>(static_cast<__half*>(param), copy, pitch, some, keep, value);
}

// 32 x 32 new values of X (scaled; a row a lane) to where the caller wants them, lanes along
// what is contiguous there: four values each, where sizes and alignment allow, after they have
// changed places in shared memory, 16 rows in `low`, 16 in `high`.  kRagged: they may not allow it
// (a kernel of its own: with both ways in one the other spills).
template <bool kRagged, int kAtOnce = 16>
__device__ __forceinline__ void finish_last(const Entry& e, const Args& a, int row0, int col0,
                                            int lane, float (&x)[32], uint16_t* low,
                                            uint16_t* high) {
  const int outer = e.tall ? col0 : row0, inner = e.tall ? row0 : col0;
  const int outers = e.tall ? e.n : e.m, inners = e.tall ? e.m : e.n;
  const int some = outers - outer < 32 ? outers - outer : 32;
  auto part = [&](int i, int k) { return swapped_part(low, high, i, k); };
  __syncwarp();                           // every lane has read its part of the piece
  if (e.tall) {
#pragma unroll
    for (int i = 0; i < 32; ++i) reinterpret_cast<float*>(part(i, lane >> 2))[lane & 3] = x[i];
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      *part(lane, k) = make_float4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
  }
  __syncwarp();
  const float step = a.muon ? -(a.lr * e.scale) * (1.f / kXScale) : 1.f / kXScale;
  if (!kRagged || e.quads) {
    const int k = lane & 7, i0 = lane >> 3;
    if (inner + 4 * k >= inners) return;
    const int64_t at = static_cast<int64_t>(outer + i0) * inners + inner + 4 * k;
    const int64_t next = 4 * static_cast<int64_t>(inners);
    uint4 old[8];                         // all on their way before the first is used
    if (a.muon)
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (i0 + 4 * u < some) old[u] = whole_quad(e.param, e.param_type, at + u * next);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (i0 + 4 * u >= some) continue;
      const float4 y = *part(i0 + 4 * u, k);
      float w[4] = {y.x * step, y.y * step, y.z * step, y.w * step};
      if (a.muon) {
        float v[4];
        unpack_quad(old[u], e.param_type, v);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = fmaf(v[j], a.keep, w[j]);
        store_quad(w, e.param, e.param_type, at + u * next);
        if (e.copy != nullptr) store_quad(w, e.copy, DORA_BF16, at + u * next);
      } else {
        store_quad(w, e.out, DORA_BF16, at + u * next);
      }
    }
  } else if (inner + lane < inners) {
    const int64_t at = static_cast<int64_t>(outer) * inners + inner + lane;
    void* param = a.muon ? const_cast<char*>(static_cast<const char*>(e.param)) +
                               at * size_of(e.param_type)
                         : nullptr;
    __nv_bfloat16* copy = reinterpret_cast<__nv_bfloat16*>(a.muon ? e.copy : e.out);
    if (copy != nullptr) copy += at;
    finish_ragged<kAtOnce>(param, e.param_type, copy, inners, some, a.keep, step, low, high);
  }
}

// What finishes 32 x 32 values of an accumulator, v, whose other inputs lie in `one`, `two`
// and, the diagonal over its columns, `dj`.  `reload` brings the next values to v, as soon as
// these have been used.  Of F and G, `one` is hi, `two` the mirror image of lo; on the diagonal
// `one` is both, hi above it and lo below.
template <Phase kPhase, bool kRagged, typename F>
__device__ __forceinline__ void finish_piece(const Entry& e, const Args& a, int row0, int col,
                                             int lane, float own, const float* dj,
                                             const uint32_t (&v)[32], uint16_t* one,
                                             uint16_t* two, F reload) {
  const int row = row0 + lane;
  if constexpr (kPhase == kGram || kPhase == kSquare) {
    const Place place = place_of(row0, col);
    constexpr float kFactor =
        kPhase == kGram ? kFScale / (kXScale * kXScale) : kC / (kFScale * kFScale);
    // c F F + (b + c (d_i + d_j)) f
    const float base = fmaf(kC, own, kB) * (1.f / kFScale);
    if (place == kAbove) {
      uint32_t high[16], low[16];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint4 f = kPhase == kSquare ? *piece_at(one, lane, k) : make_uint4(0, 0, 0, 0);
        const uint32_t fs[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int c = 8 * k + 2 * i;
          uint64_t x = f2_mul(f2_pack(__uint_as_float(v[c]), __uint_as_float(v[c + 1])),
                              twice(kFactor));
          if (kPhase == kSquare) {
            const uint64_t rest = f2_pack(half_value(*value_in(two, c, lane)),
                                          half_value(*value_in(two, c + 1, lane)));
            const float2 d = *reinterpret_cast<const float2*>(dj + c);
            x = f2_fma(f2_add(halves(fs[i]), rest),
                       f2_fma(f2_pack(d.x, d.y), twice(kC / kFScale), twice(base)), x);
          }
          high[4 * k + i] = to_halves(x);
          low[4 * k + i] = to_halves(f2_fma(halves(high[4 * k + i]), twice(-1.f), x));
        }
      }
      reload();
#pragma unroll
      for (int k = 0; k < 4; ++k)
        *piece_at(one, lane, k) = make_uint4(high[4 * k], high[4 * k + 1], high[4 * k + 2],
                                             high[4 * k + 3]);
#pragma unroll
      for (int c = 0; c < 32; ++c)
        *value_in(two, c, lane) = static_cast<uint16_t>(low[c >> 1] >> (16 * (c & 1)));
    } else if (place == kOn) {
      // a lane reads and writes its own row's values behind the diagonal and their mirror images
#pragma unroll
      for (int c = 0; c < 32; ++c) {
        float x = __uint_as_float(v[c]) * kFactor;
        if (c == lane) {
          if (kPhase == kGram) e.d[row] = x * (1.f / kFScale);
          else e.e[row] = fmaf(fmaf(kC, own, kB), own, x);
          *value_in(one, lane, lane) = 0;
        } else if (c > lane) {
          uint16_t *high = value_in(one, lane, c), *low = value_in(one, c, lane);
          if (kPhase == kSquare)
            x = fmaf(half_value(*high) + half_value(*low), fmaf(dj[c], kC / kFScale, base), x);
          *high = half_bits(x);
          *low = half_bits(x - half_value(*high));
        }
      }
      reload();
    } else {
      reload();
    }
  } else {
    float x[kPhase == kLast ? 32 : 1];
    uint32_t nh[kPhase == kApply ? 16 : 1], nl[kPhase == kApply ? 16 : 1];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint4 h = *piece_at(one, lane, k), l = *piece_at(two, lane, k);
      const uint32_t hs[4] = {h.x, h.y, h.z, h.w}, ls[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = 8 * k + 2 * i;
        // (a + E) X + G X_hi
        const uint64_t y = f2_fma(twice(own), f2_add(halves(hs[i]), halves(ls[i])),
                                  f2_pack(__uint_as_float(v[c]), __uint_as_float(v[c + 1])));
        if constexpr (kPhase == kApply) {
          nh[4 * k + i] = to_halves(y);
          nl[4 * k + i] = to_halves(f2_fma(halves(nh[4 * k + i]), twice(-1.f), y));
        } else {
          f2_unpack(y, x[c], x[c + 1]);
        }
      }
    }
    reload();
    if constexpr (kPhase == kApply) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        *piece_at(one, lane, k) = make_uint4(nh[4 * k], nh[4 * k + 1], nh[4 * k + 2],
                                             nh[4 * k + 3]);
        *piece_at(two, lane, k) = make_uint4(nl[4 * k], nl[4 * k + 1], nl[4 * k + 2],
                                             nl[4 * k + 3]);
      }
    } else {
      finish_last<kRagged>(e, a, row0, col, lane, x, one, two);
    }
  }
}

template <bool kRagged>
__global__ void __launch_bounds__(kThreads, 1)
    product_kernel(const __grid_constant__ Maps maps, List list, Args a, int steps) {
  extern __shared__ __align__(1024) uint8_t raw[];
  Smem& s = *reinterpret_cast<Smem*>(raw);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = static_cast<int>(cluster_ctarank());
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&s.full[i], 1);
      mbar_init(&s.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s.acc_full[i], 1);
      mbar_init(&s.acc_empty[i], 2 * kEpiWarps);
    }
    for (int h = 0; h < 2; ++h)
      for (int i = 0; i < kPlaces; ++i) {
        mbar_init(&s.piece_full[h][i], 1);
        mbar_init(&s.piece_done[h][i], kEpiWarps / 2);
        mbar_init(&s.piece_empty[h][i], 1);
      }
    for (int i = 0; i < kRing; ++i) {
      mbar_init(&s.task_full[i], 1);
      mbar_init(&s.task_empty[i], 2 * (3 + kEpiWarps) + 1);
    }
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
  pdl_trigger();                          // all that came before the call is complete: small_kernel
  const bool none = skipped(a);
  const uint32_t tmem = s.tmem;
  volatile int* abort = &s.abort;
  // stages of a tile: the K of its product over 64
  auto stages_of = [&](const Entry& e, const Task& t) {
    return ((t.phase == kGram ? e.n : e.m) + kK - 1) / kK;
  };
  // The n-th task, null when there are no more; its place is used again once all roles are
  // done with it.
  auto task = [&](int n) -> const Task* {
    const int i = n % kRing;
    if (none || !mbar_wait_cluster(&s.task_full[i], (n / kRing) & 1, abort)) return nullptr;
    return s.task[i].matrix >= 0 ? &s.task[i] : nullptr;
  };
  auto task_done = [&](int n) { mbar_arrive_remote(&s.task_empty[n % kRing], 1); };

  if (warp == 0) {
    if (elect_one()) {
      int it = 0;
      bool ok = true;
      bool known = false;                 // that what the task needs is there
      const Task* at;
      for (int n = 0; ok && (at = task(n)) != nullptr; ++n) {
        const Task& t = *at;
        const Entry& e = t.e;
        if (!known && !wait_done(e.done, t.need, abort, list.header)) break;
        known = false;
        const bool gram = t.phase == kGram, apply = t.phase >= kApply;
        const int count = stages_of(e, t), mb = e.mb, nb = e.nb, block = 2 * t.i + rank;
        const bool wide = t.width > 128;
        const int64_t fg = apply ? e.g : e.f;
        // columns of tiles of the right operand that this CTA holds (MN-major); those past a
        // tile's end are the last one's again, and not looked at
        const int first = t.j + (wide ? 2 * rank : rank), last = t.j + (t.width >> 6) - 1;
        const int c0 = min(first, last), c1 = min(first + 1, last);
        // two stages for 64 of K: hi of X, or F and G as they lie, then lo of X, or their mirror
        // image
        for (int k = 0; ok && k < count; ++k)
          for (int part = 0; part < 2; ++part, ++it) {
            const int st = it % kStages;
            // a look at the next task while the stages are full anyway
            if (part == 1 && k == count - 1 && 2 * k >= kStages &&
                mbar_test(&s.task_full[(n + 1) % kRing], ((n + 1) / kRing) & 1)) {
              const Task* next = task(n + 1);
              if (next != nullptr &&
                  load_acquire(next->e.done) >= static_cast<unsigned>(next->need)) {
                fence_proxy_async_all();
                known = true;
              }
            }
            if (!mbar_wait(&s.empty[st], ((it / kStages) & 1) ^ 1, abort)) {
              ok = false;
              break;
            }
#ifdef DORA_TEST_WITHHOLD_TILE_LOAD
            // timeout-path test library only: the first pair never loads its first stage nor
            // expects its bytes, so that the wait for it runs out with no copy of it in flight
            if (blockIdx.x < 2 && it == 0) continue;
#endif
            // the bytes of both CTAs are counted on the first one's barrier
            if (rank == 0)
              mbar_arrive_expect_tx(&s.full[st],
                                    2 * (kTileBytes + (wide ? kTileBytes : kHalfTile)));
            const auto load = [&](const CUtensorMap* map, void* to, int64_t tile, int row) {
              tma_load_2d_pair(to, map, &s.full[st], 0, 0,
                               static_cast<int32_t>(tile * kTileRows) + row);
            };
            uint8_t *sa = s.a[st], *sb = s.b[st];
            const int kb = k >> 1, kr = (k & 1) * 64;   // block row of 64 of K, and row in it
            if (gram) {
              load(&maps.tile, sa, x_tile(e, t.turn, block, k, part), 0);
              if (wide) load(&maps.tile, sb, x_tile(e, t.turn, t.j + rank, k, part), 0);
              else load(&maps.half, sb, x_tile(e, t.turn, t.j, k, part), 64 * rank);
              continue;
            }
            const auto straight = [&](int row) {          // 64 columns of a block row
              return fg + static_cast<int64_t>(row) * (2 * mb) + k;
            };
            const auto turned = [&](int col) {            // 64 rows of a column of tiles
              return fg + static_cast<int64_t>(kb) * (2 * mb) + col;
            };
            if (part == 0) {
              load(&maps.tile, sa, straight(block), 0);
            } else {
              load(&maps.half, sa, turned(2 * block), kr);
              load(&maps.half, sa + kHalfTile, turned(2 * block + 1), kr);
            }
            if (apply) {
              const int64_t x = slot_tile(e, t.turn, t.half) + part * (e.slot / 2) +
                                static_cast<int64_t>(kb) * nb;
              load(&maps.half, sb, x + c0, kr);
              if (wide) load(&maps.half, sb + kHalfTile, x + c1, kr);
            } else if (part == 0) {
              if (wide) load(&maps.tile, sb, straight(t.j + rank), 0);
              else load(&maps.half, sb, straight(t.j), 64 * rank);
            } else {
              const int c = 2 * t.j + (wide ? 2 * rank : rank);
              load(&maps.half, sb, turned(c), kr);
              if (wide) load(&maps.half, sb + kHalfTile, turned(c + 1), kr);
            }
          }
        task_done(n);
      }
      s.issued = it;
    }
  } else if (warp == 1 && rank == 0) {
    if (elect_one()) {
      int it = 0;
      bool ok = true;
      const Task* at;
      for (int n = 0; ok && (at = task(n)) != nullptr; ++n) {
        const int count = stages_of(at->e, *at), phase = at->phase;
        const int i = at->i, j = at->j, wide = at->width > 128 ? 1 : 0;
        task_done(n);
        const bool gram = phase == kGram, apply = phase >= kApply;
        const int acc = n & 1;
        if (!mbar_wait(&s.acc_empty[acc], ((n >> 1) & 1) ^ 1, abort)) break;
        tc_fence_after();
        const uint32_t d = tmem + static_cast<uint32_t>(acc * kWide);
        uint32_t more = 0;                // 0: the tile's first MMA, which adds to nothing
        // Part p of the left operand times part q of the right one: K-major, but F and G's mirror
        // images and the right operand of G X are MN-major.
        const auto product = [&](int p, int q, int st) {
          const bool a_mn = !gram && p == 1, b_mn = apply || (!gram && q == 1);
          const int sa = p == 0 ? st : (st + 1) % kStages, sb = q == 0 ? st : (st + 1) % kStages;
          const uint64_t ad = sdesc_sw128(smem_u32(s.a[sa]), a_mn ? kHalfTile : 16, 1024);
          const uint64_t bd = sdesc_sw128(smem_u32(s.b[sb]), b_mn ? kHalfTile : 16, 1024);
          // 16 of K further on: 32 bytes of a row, or 16 rows
          const uint64_t step_a = a_mn ? 128 : 2, step_b = b_mn ? 128 : 2;
          const uint32_t idesc = idesc_f16(2 * kBlock, wide ? 256 : 128, b_mn, a_mn);
#pragma unroll
          for (int c = 0; c < kK / 16; ++c) {
            mma_bf16_ss_pair(d, ad + step_a * c, bd + step_b * c, idesc, more);
            more = 1;
          }
        };
        for (int k = 0; k < count; ++k, it += 2) {
          // which parts are lo: their product is left out.  F and G's first part is hi behind the
          // diagonal's blocks, lo before them, and both in them.
          const int kb = k >> 1;
          const int low_a = gram ? 1 : (kb >> 1 < i ? 0 : (kb >> 1 > i ? 1 : 2));
          const int low_b = gram || apply ? 1 : (kb < j ? 0 : (kb > j + wide ? 1 : 2));
          const auto wanted = [&](int p, int q) { return p != low_a || q != low_b; };
          const int st = it % kStages;
          if (!mbar_wait(&s.full[st], (it / kStages) & 1, abort)) {
            ok = false;
            break;
          }
          tc_fence_after();
          if (wanted(0, 0)) product(0, 0, st);
          const int st1 = (it + 1) % kStages;
          if (!mbar_wait(&s.full[st1], ((it + 1) / kStages) & 1, abort)) {
            ++it;
            ok = false;
            break;
          }
          tc_fence_after();
          if (wanted(1, 0)) product(1, 0, st);
          if (wanted(0, 1)) product(0, 1, st);
          if (wanted(1, 1)) product(1, 1, st);
          mma_commit_pair(&s.empty[st], kPairMask);
          mma_commit_pair(&s.empty[st1], kPairMask);
        }
        if (ok) mma_commit_pair(&s.acc_full[acc], kPairMask);
      }
      s.consumed = it;
      mma_commit_pair(&s.drain, 0x1);
      mbar_wait_limited(&s.drain, 0, kWaitLimitNs);
    }
  } else if (warp == 1) {
    // tiles for the pair, a few ahead
    if (!none) {
      const int n_groups = list.header->n_groups;
      int g = 0;
      unsigned base = 0;
      for (int n = 0;; ++n) {
        const int i = n % kRing;
        if (!__all_sync(0xffffffffu,
                        mbar_wait_cluster(&s.task_empty[i], ((n / kRing) & 1) ^ 1, abort)))
          break;
        unsigned w = 0;
        if (lane == 0) w = atomicAdd(&list.header->ticket, 1u);
        w = __shfl_sync(0xffffffffu, w, 0);
        Tile x = {-1, 0, 0, 0};
        int phase = 0, step = 0, half = 0;
        unsigned before = 0;
        for (; g < n_groups; ++g) {
          const Group q = list.groups[g];
          const unsigned sym = q.sym1 - q.sym0, all = q.all1 - q.all0, each = 2 * (sym + all);
          if (w - base >= each * steps) {
            base += each * steps;
            continue;
          }
          step = static_cast<int>((w - base) / each);
          const unsigned r = (w - base) % each;
          half = r >= 2 * sym + all;
          x = r < 2 * sym ? list.sym[q.sym0 + (r < sym ? r : r - sym)]
                          : list.all[q.all0 + (r - 2 * sym - (half ? all : 0))];
          phase = r < sym ? kGram : (r < 2 * sym ? kSquare : (step + 1 < steps ? kApply : kLast));
          break;
        }
        if (__ldcg(&list.header->abort) != 0) x.matrix = -1;
        x.matrix = __shfl_sync(0xffffffffu, x.matrix, 0);
        // the entry by words, a few a lane
        const Entry* e = list.entries + (x.matrix < 0 ? 0 : x.matrix);
        // the right half is written over the left one, where it is written
        before = phase == kGram ? 0u : (phase == kSquare ? e->n_sym : 2u * e->n_sym);
        if (phase == kApply && half) before += e->n_all;
        const int need =
            static_cast<int>(kTileArrivals * (2u * step * (e->n_sym + e->n_all) + before));
        const int head[8] = {x.matrix, x.i, x.j, x.width, phase, step % 3, need, half};
        int* to = reinterpret_cast<int*>(&s.task[i]);
        for (int cta = 0; cta < 2; ++cta) {
          if (lane == 0)
#pragma unroll
            for (int k = 0; k < 8; ++k) store_remote(head[k], to + k, cta);
          for (int k = lane; k < kTaskWords - 8; k += 32)
            store_remote(reinterpret_cast<const int*>(e)[k], to + 8 + k, cta);
          __syncwarp();
          if (lane == 0) mbar_arrive_remote(&s.task_full[i], cta);
        }
        if (x.matrix < 0) break;
      }
    }
  } else if (warp == 2 + kEpiWarps) {
    // The inputs of the pieces, in the order in which they are finished: 32 columns of the
    // CTA's 128 rows at a time, for each half of the tile's columns.  What the last phase
    // reads besides, the weights, is brought to L2.
    int loads = 0;                        // pieces of every warp
    bool ok = true;
    for (int n = 0; ok; ++n) {
      const Task* at = task(n);
      if (!__all_sync(0xffffffffu, at != nullptr)) break;
      const Entry& e = at->e;
      const int phase = at->phase, half = at->width >> 1;
      const int block = 2 * at->i + rank, pieces = pieces_of(*at, block);
      const int first_col = first_column(*at);
      const int64_t x = slot_tile(e, at->turn, at->half) +
                        static_cast<int64_t>(block) * e.nb - at->half * e.nb;
      bool there = true;
      if (lane == 0) there = wait_done(e.done, at->need, abort, list.header);
      if (!__all_sync(0xffffffffu, there)) break;
      if (phase == kLast && e.param != nullptr)
        prefetch_weights(e, block, first_col, at->width, lane);
      for (int c = 0; ok && c < pieces; ++c, ++loads) {
        const int i = loads % kPlaces;
        for (int h = 0; ok && h < 2; ++h) {
          ok = mbar_wait_warp(&s.piece_empty[h][i], ((loads / kPlaces) & 1) ^ 1, abort);
          if (!ok || !elect_one()) continue;
          const int col = first_col + h * half + 32 * c, block_col = col >> 7;
          uint64_t* bar = &s.piece_full[h][i];
          // nothing to read: the place is free
          if (phase == kGram || (phase == kSquare && block_col < block)) {
            mbar_arrive(bar);
            continue;
          }
          mbar_arrive_expect_tx(bar, 8 * kPiece * 2 + (phase == kSquare ? 128 : 0));
          if (phase == kSquare) {
            const int64_t f = e.f + static_cast<int64_t>(block) * (2 * e.mb) + (col >> 6);
            bulk_load(s.dj[i][h], e.d + col, 128, bar);
            tma_load_2d(s.piece[i][0][h], &maps.column, bar, col & 32,
                        static_cast<int32_t>(f * kTileRows));
            const int64_t image = e.f + static_cast<int64_t>(block_col) * (2 * e.mb) + 2 * block;
            for (int w = 0; w < 4; ++w)
              tma_load_2d(s.piece[i][1][h][w], &maps.piece, bar, (w & 1) * 32,
                          static_cast<int32_t>((image + (w >> 1)) * kTileRows + (col & 127)));
          } else {
            for (int part = 0; part < 2; ++part)
              tma_load_2d(s.piece[i][part][h], &maps.column, bar, col & 32,
                          static_cast<int32_t>((x + part * (e.slot / 2) + (col >> 6)) *
                                               kTileRows));
          }
        }
        __syncwarp();
      }
      __syncwarp();
      if (lane == 0) task_done(n);
    }
    // after an abort too: what was issued lands before the CTA ends
    if (lane == 0)
      for (int k = loads - kPlaces; *abort && k <= loads; ++k)
        for (int h = 0; k >= 0 && h < 2; ++h)
          mbar_wait_limited(&s.piece_full[h][k % kPlaces], (k / kPlaces) & 1, 10ull * 1000 * 1000);
  } else if (warp == 3 + kEpiWarps) {
    // What the pieces became, out of their places: half a tile's columns, the CTA's rows.
    if (elect_one()) {
      unsigned* unsaid = nullptr;         // counter of a tile that is not reported
      uint64_t* place = nullptr;          // of the copies before the newest
      int done = 0;
      bool ok = true;
      // a tile is reported once its copies are complete: all but the newest, or all
      auto report = [&](bool newest_too) {
        if (newest_too) bulk_wait_group0(); else bulk_wait_group1();
        fence_proxy_async_all();
        signal(unsaid);
        unsaid = nullptr;
      };
      for (int n = 0; ok; ++n) {
        // no waiting with a report to make: others may wait for it
        if (unsaid != nullptr && !mbar_test(&s.task_full[n % kRing], (n / kRing) & 1)) report(true);
        const Task* at = task(n);
        if (at == nullptr) break;
        const Entry& e = at->e;
        const int phase = at->phase, half = at->width >> 1;
        const int block = 2 * at->i + rank, first_col = first_column(*at);
        const int pieces = pieces_of(*at, block);
        if (pieces == 0) {
          // Nothing to copy, but no report before the matrix' phase has begun: it would be
          // counted for the one before.
          if (unsaid != nullptr) report(true);
          if (!wait_done(e.done, at->need, abort, list.header)) break;
        }
        const int row_tiles = 2 * e.mb;
        const int64_t to = phase == kGram ? e.f : e.g;
        // X as it lies an iteration later
        const int64_t x = slot_tile(e, at->turn == 2 ? 0 : at->turn + 1, at->half) +
                          static_cast<int64_t>(block) * e.nb - at->half * e.nb;
        for (int c = 0; ok && c < pieces; ++c, ++done) {
          const int i = done % kPlaces;
          for (int h = 0; h < 2; ++h) {
            if (unsaid != nullptr && !mbar_test(&s.piece_done[h][i], (done / kPlaces) & 1))
              report(true);
            ok = mbar_wait(&s.piece_done[h][i], (done / kPlaces) & 1, abort);
            if (!ok) break;
            const int col = first_col + h * half + 32 * c, block_col = col >> 7;
            if (phase == kApply) {
              for (int part = 0; part < 2; ++part)
                tma_store_2d(&maps.column, s.piece[i][part][h], col & 32,
                             static_cast<int32_t>((x + part * (e.slot / 2) + (col >> 6)) *
                                                  kTileRows));
            } else if (phase < kApply && block_col >= block) {
              // hi, four warps' rows at once but in the diagonal's blocks, and 32 columns of the
              // mirror image of lo each
              const int64_t tile = to + static_cast<int64_t>(block) * row_tiles + (col >> 6);
              const int64_t image = to + static_cast<int64_t>(block_col) * row_tiles + 2 * block;
              const int above = block_col > block ? 4 : (col & 127) >> 5;
              if (above == 4)
                tma_store_2d(&maps.column, s.piece[i][0][h], col & 32,
                             static_cast<int32_t>(tile * kTileRows));
              else
                for (int w = 0; w <= above; ++w)
                  tma_store_2d(&maps.piece, s.piece[i][0][h][w], col & 32,
                               static_cast<int32_t>(tile * kTileRows + 32 * w));
              for (int w = 0; w < above; ++w)
                tma_store_2d(&maps.piece, s.piece[i][1][h][w], (w & 1) * 32,
                             static_cast<int32_t>((image + (w >> 1)) * kTileRows + (col & 127)));
            }
            bulk_commit_group();          // also without any: one for every place
            bulk_wait_group_read1();
            if (place != nullptr) mbar_arrive(place);
            place = &s.piece_empty[h][i];
            if (unsaid != nullptr) report(false);
          }
        }
        unsaid = e.done;
        task_done(n);
      }
      if (unsaid != nullptr && ok && !*abort) report(true);
      bulk_wait_group0();                 // copies are done before the CTA ends
    }
  } else {
    const int q = warp & 3, half = (warp - 2) >> 2;
    int done = 0;
    bool ok = true;
    for (int n = 0; ok; ++n) {
      const int slot = n % kRing, acc = n & 1;
      if (none || !__all_sync(0xffffffffu,
                              mbar_wait_cluster(&s.task_full[slot], (n / kRing) & 1, abort)))
        break;
      const Task& t = s.task[slot];
      if (t.matrix < 0) break;
      const Entry& e = t.e;
      const int phase = t.phase, pieces = pieces_of(t, 2 * t.i + rank);
      const int row0 = (2 * t.i + rank) * kBlock + q * 32;
      const int col0 = first_column(t) + half * (t.width >> 1);
      if (!mbar_wait_warp(&s.acc_full[acc], (n >> 1) & 1, abort)) break;
      tc_fence_after();
      const uint32_t from = tmem + (static_cast<uint32_t>(q * 32) << 16) + acc * kWide +
                            half * (t.width >> 1);
      uint32_t v[32];
      if (pieces > 0) {
        tmem_ld32(from, v);
      } else {                            // nothing of the accumulator is wanted
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_remote(&s.acc_empty[acc], 0);
      }
      float own = 0.f;                    // of the lane's row: d, or a + e
      if (phase == kSquare) own = __ldcg(&e.d[row0 + lane]);
      if (phase >= kApply) own = kA + __ldcg(&e.e[row0 + lane]);
      for (int c = 0; c < pieces; ++c, ++done) {
        const int col = col0 + 32 * c, place = done % kPlaces;
        uint16_t *one = s.piece[place][0][half][q], *two = s.piece[place][1][half][q];
        const bool there = mbar_wait_warp(&s.piece_full[half][place], (done / kPlaces) & 1, abort);
        tmem_ld_wait();
        if (!there) {
          ok = false;
          break;
        }
        const float* dj = s.dj[place][half];
        auto reload = [&] {
          if (c + 1 < pieces) {
            tmem_ld32(from + 32 * (c + 1), v);
          } else {                        // this warp is done with the accumulator
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_remote(&s.acc_empty[acc], 0);
          }
        };
        if (phase == kGram)
          finish_piece<kGram, kRagged>(e, a, row0, col, lane, own, dj, v, one, two, reload);
        else if (phase == kSquare)
          finish_piece<kSquare, kRagged>(e, a, row0, col, lane, own, dj, v, one, two, reload);
        else if (phase == kApply)
          finish_piece<kApply, kRagged>(e, a, row0, col, lane, own, dj, v, one, two, reload);
        else
          finish_piece<kLast, kRagged>(e, a, row0, col, lane, own, dj, v, one, two, reload);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s.piece_done[half][place]);
      }
      __syncwarp();
      if (lane == 0) task_done(n);
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
      // Loads that were issued but never consumed land first.  Those of the second CTA are counted
      // by the first, which need not have asked for as many: time for them instead.
      if (rank == 0)
        for (int it = s.consumed; it < s.issued; ++it)
          mbar_wait_limited(&s.full[it % kStages], (it / kStages) & 1, 10ull * 1000 * 1000);
      const uint64_t t0 = globaltimer_ns();
      while (globaltimer_ns() - t0 < 1000ull * 1000) __nanosleep(1000);
    }
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, 2 * kWide);
  }
  cluster_sync();                         // no CTA leaves while its peer may still signal it
}

// ---------------------------------------------------------------------------
// Small matrices (m <= 128, n <= 2048): a whole step in one launch.  A CTA, or a cluster of 2, 4
// or 8, holds one, 256 columns of X each, in shared memory; A, B and what they are made of are
// 128 x 128.  Where there are several CTAs each adds up its rows of X X^T over all of them and
// sends every one its rows of F.  What bounds it is the chain of three products an iteration,
// each with its reading of tensor memory; the first pass and the last take as long as one or two.
//
// All operands are hi + lo here too.  The actor's twelve matrices take 85 us (a step 88).
//
// In a list of both kinds it runs beside the products, on the SMs that they leave (`beside`): it
// needs nothing of theirs, and they start it when all work before the call is complete.  One CTA
// waits for them at its end, so that whatever follows waits for both.
// ---------------------------------------------------------------------------
constexpr int kSmallRows = 128, kSmallTiles = 4, kMaxParts = 8;
constexpr int kSmallThreads = 256;

struct SmallSmem {
  uint8_t hi[kSmallTiles][kTileBytes], lo[kSmallTiles][kTileBytes];
  uint8_t f[4][kTileBytes];               // F, then G in its place: hi of 64 columns each, then lo
  uint8_t extra[2][kTileBytes];
  float d[kSmallRows], e[kSmallRows];
  Squares sums[kMaxParts], scratch[kSmallThreads / 32];
  uint64_t done, drain;                   // the MMAs of a product; all, after an abort
  uint32_t tmem;
  int abort, bad[kMaxParts];
};
static_assert(sizeof(SmallSmem) <= 227 * 1024, "shared memory");

// 16-byte part k of row r of a tile, where the tensor cores look for it.
__device__ __forceinline__ uint4* tile_part(uint8_t* tile, int r, int k) {
  return reinterpret_cast<uint4*>(tile + r * 128 + ((k ^ (r & 7)) << 4));
}
// Part k of row r of a matrix of fp32 values of `cols` columns, 64 or 128.
__device__ __forceinline__ uint4* wide_part(uint8_t* matrix, int cols, int r, int k) {
  return reinterpret_cast<uint4*>(matrix + r * cols * 4 + ((k ^ (r & (cols / 4 - 1))) << 4));
}
__device__ __forceinline__ uint4 load_remote(const uint4* from, uint32_t cta) {
  uint4 q;
  asm volatile(
      "{\n\t.reg .b32 ra;\n\t"
      "mapa.shared::cluster.u32 ra, %4, %5;\n\t"
      "ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [ra];\n\t}"
      : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w)
      : "r"(smem_u32(from)), "r"(cta)
      : "memory");
  return q;
}
__device__ __forceinline__ void store_remote_part(uint4 q, uint4* to, uint32_t cta) {
  asm volatile(
      "{\n\t.reg .b32 ra;\n\t"
      "mapa.shared::cluster.u32 ra, %0, %1;\n\t"
      "st.shared::cluster.v4.u32 [ra], {%2, %3, %4, %5};\n\t}" ::"r"(smem_u32(to)),
      "r"(cta), "r"(q.x), "r"(q.y), "r"(q.z), "r"(q.w)
      : "memory");
}

// The matrix of a CTA, or its part of one.
__device__ __forceinline__ void small_matrix(const Entry& e, const Args& a, int steps, int rank,
                                             SmallSmem& s) {
  const int me = threadIdx.x, warp = me >> 5, lane = me & 31, parts = e.parts;
  if (me == 0) {
    mbar_init(&s.done, 1);
    mbar_init(&s.drain, 1);
    s.abort = 0;
    fence_barrier_init();
  }
  if (warp == 0) tmem_alloc(&s.tmem, 512);
  tc_fence_before();
  // all CTAs of the matrix: also that the others are there
  auto sync = [&]() {
    if (parts > 1) cluster_sync();
    else __syncthreads();
  };
  sync();
  tc_fence_after();
  const uint32_t tmem = s.tmem;
  volatile int* abort = &s.abort;
  const int all = (e.n + 63) / 64, each = (all + parts - 1) / parts;
  const int tile0 = rank * each, tiles = max(0, min(each, all - tile0)), col0 = 64 * tile0;
  const int halves = (e.m + 63) / 64;     // of the products over m
  const int wide = 64 * halves;           // rows and columns of A that are looked at
  // a CTA's part of A, for the others: beside F where it is small, else in F's place, so that all
  // have read it before F is written
  uint8_t* part_of_a = halves == 1 ? s.extra[0] : s.f[0];
  const float f = factor(a);
  const bool eights = in_eights(e, a);

  // momentum and the update's norm, then the normalised update; between them the update lies
  // in its tiles' places as fp32, 64 rows of a tile in each
  auto raw_at = [&](int r, int k, int i) {    // values 4 i .. of part k of row r
    uint8_t* tile = r < 64 ? s.hi[k >> 3] : s.lo[k >> 3];
    return reinterpret_cast<uint4*>(tile + (r & 63) * 256 + (((2 * (k & 7) + i) ^ (r & 7)) << 4));
  };
  Squares sum = {0.f, -126};
  if (parts > 1) {                        // F has no more than the matrix' rows and columns
    uint4* zero = reinterpret_cast<uint4*>(s.f[0]);
    for (int i = me; i < 4 * kTileBytes / 16; i += kSmallThreads) zero[i] = make_uint4(0, 0, 0, 0);
    if (me < kSmallRows) s.d[me] = 0.f;
  }
  if (eights) {
    constexpr int kSome = 4;
    for (int w0 = me; w0 < kSmallRows * 8 * tiles; w0 += kSome * kSmallThreads) {
      Eight x[kSome];
#pragma unroll
      for (int y = 0; y < kSome; ++y) {   // the count is a multiple of what all threads take
        const int w = w0 + y * kSmallThreads;
        x[y] = load_eight(e, a, true, w / (8 * tiles), col0 + w % (8 * tiles) * 8);
      }
#pragma unroll
      for (int y = 0; y < kSome; ++y) {
        const int w = w0 + y * kSmallThreads, r = w / (8 * tiles), k = w % (8 * tiles);
        const bool there = r < e.m && col0 + 8 * k < e.n;
        float d[8], m[8], u[8];
        values_of(e, x[y], there, d, m);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          d[i] *= f;
          if (a.muon) m[i] = fmaf(a.mu, m[i], a.omu * d[i]);
          u[i] = update_of(a, d[i], m[i]);
        }
        if (a.muon && there) {
          const int64_t at = static_cast<int64_t>(r) * e.n + col0 + 8 * k;
          store_quad(m, e.momentum, DORA_F32, at);
          store_quad(m + 4, e.momentum, DORA_F32, at + 4);
        }
        sum.add(squares_of(u));
        *raw_at(r, k, 0) = Granule<float>::pack(u);
        *raw_at(r, k, 1) = Granule<float>::pack(u + 4);
      }
    }
  } else {
    // by elements, lanes along what is contiguous; then zeros where there are none
    const int cols = max(0, min(64 * tiles, e.n - col0)), count = e.m * cols;
    const int inner = max(1, e.tall ? e.m : cols);
    const int step_i = kSmallThreads % inner, step_o = kSmallThreads / inner;
    constexpr int kSome = 16;
    int i = me % inner, o = me / inner;   // of this thread's next element, without divisions
    for (int w0 = me; w0 < count; w0 += kSome * kSmallThreads) {
      uint32_t raw_d[kSome], raw_m[kSome];   // as they are loaded
      float d[kSome];
      int at[kSome], to[kSome];           // where, of at most 128 x 2048; row and column
#pragma unroll
      for (int y = 0; y < kSome; ++y) {
        at[y] = e.tall ? (col0 + o) * e.m + i : o * e.n + col0 + i;
        to[y] = e.tall ? i << 16 | o : o << 16 | i;
        raw_d[y] = raw_m[y] = 0u;
        if (w0 + y * kSmallThreads < count) {
          raw_d[y] = e.grad_type == DORA_F32 ? static_cast<const uint32_t*>(e.grad)[at[y]]
                                             : static_cast<const uint16_t*>(e.grad)[at[y]];
          if (a.muon) raw_m[y] = reinterpret_cast<const uint32_t*>(e.momentum)[at[y]];
        }
        i += step_i;
        o += step_o;
        if (i >= inner) {
          i -= inner;
          ++o;
        }
      }
#pragma unroll
      for (int y = 0; y < kSome; ++y) {
        float one[4];
        unpack_quad(make_uint4(raw_d[y], 0u, 0u, 0u), e.grad_type, one);
        d[y] = one[0] * f;
        if (w0 + y * kSmallThreads >= count) continue;
        float m = __uint_as_float(raw_m[y]);
        if (a.muon) {
          m = fmaf(a.mu, m, a.omu * d[y]);
          e.momentum[at[y]] = m;
        }
        d[y] = update_of(a, d[y], m);
        const int r = to[y] >> 16, c = to[y] & 0xFFFF;
        reinterpret_cast<float*>(raw_at(r, c >> 3, (c >> 2) & 1))[c & 3] = d[y];
      }
      sum.add(squares_of(d));
    }
    // whole parts of eight where the matrix has no row or column; the rest by elements
    for (int w = me; w < kSmallRows * 8 * tiles; w += kSmallThreads) {
      const int r = w / (8 * tiles), k = w % (8 * tiles);
      if (r < e.m && 8 * k + 8 <= cols) continue;
      for (int c = 8 * k; c < 8 * k + 8; ++c)
        if (r >= e.m || c >= cols)
          reinterpret_cast<float*>(raw_at(r, k, (c >> 2) & 1))[c & 3] = 0.f;
    }
    __syncthreads();                      // an element is another thread's from here on
  }
  sum = block_squares(sum, s.scratch);
  if (me == 0)
    for (int c = 0; c < parts; ++c) {
      if (parts > 1) {
        store_remote(__float_as_int(sum.sum), reinterpret_cast<int*>(&s.sums[rank].sum), c);
        store_remote(sum.k, &s.sums[rank].k, c);
      } else {
        s.sums[0] = sum;
      }
    }
  sync();
  sum = s.sums[0];
  for (int c = 1; c < parts; ++c) sum.add(s.sums[c]);
  const float inv = (sum.sum == 0.f ? 0.f : (isfinite(sum.sum) ? 1.f / sqrtf(sum.sum) : NAN)),
              near1 = __uint_as_float(static_cast<uint32_t>(127 - sum.k) << 23);
  for (int t = 0; t < tiles; ++t) {
    constexpr int kMine = kSmallRows * 8 / kSmallThreads;
    uint4 h[kMine], l[kMine];
#pragma unroll
    for (int y = 0; y < kMine; ++y) {
      const int w = me + y * kSmallThreads, r = w >> 3, k = 8 * t + (w & 7);
      float v[8];
      Granule<float>::unpack(*raw_at(r, k, 0), v);
      Granule<float>::unpack(*raw_at(r, k, 1), v + 4);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = v[i] * near1 * inv * kXScale;
      split(v, &h[y], &l[y]);
    }
    __syncthreads();                      // the tile's values have been read
#pragma unroll
    for (int y = 0; y < kMine; ++y) {
      const int w = me + y * kSmallThreads, r = w >> 3, k = w & 7;
      *tile_part(s.hi[t], r, k) = h[y];
      *tile_part(s.lo[t], r, k) = l[y];
    }
  }

  const int q = warp & 3, half = warp >> 2, row = q * 32 + lane;
  const uint32_t lanes = static_cast<uint32_t>(q * 32) << 16;
  const bool has_rows = q * 32 < wide, has_part = has_rows && half < halves;
  int products = 0;
  // What the threads wrote to shared memory is there for the tensor cores; one thread issues the
  // MMAs of a product, all wait for it.
  auto product = [&](auto issue) {
    fence_proxy_async_smem();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0 && elect_one()) {
      issue();
#ifdef DORA_TEST_WITHHOLD_TILE_LOAD
      // timeout-path test library only: the first CTA never says that its first product is done
      if (blockIdx.x != 0 || products != 0)
#endif
      mma_commit(&s.done);
    }
    __syncwarp();
    mbar_wait_warp(&s.done, products++ & 1, abort);
    tc_fence_after();
  };
  for (int step = 0; step < steps; ++step) {
    product([&] {
      for (int t = 0; t < tiles; ++t) {
        const uint64_t x = sdesc_sw128(smem_u32(s.hi[t]), 16, 1024);
        const uint64_t y = sdesc_sw128(smem_u32(s.lo[t]), 16, 1024);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          constexpr uint32_t idesc = idesc_f16(128, 128, false);
          mma_bf16_ss(tmem, x + 2 * k, x + 2 * k, idesc, (t | k) != 0);
          mma_bf16_ss(tmem, x + 2 * k, y + 2 * k, idesc, 1u);
          mma_bf16_ss(tmem, y + 2 * k, x + 2 * k, idesc, 1u);
        }
      }
    });
    // F and d, from A
    auto keep = [&](int r, int k, float (&x)[8], auto store) {   // part k of row r, scaled
      if ((r >> 3) == k) {
        float own = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i == (r & 7)) {
            own = x[i] * (1.f / kFScale);
            x[i] = 0.f;
          }
        store(own, true, x);
      } else {
        store(0.f, false, x);
      }
    };
    if (has_part)
#pragma unroll
      for (int c = 0; c < 2; ++c) {       // 32 columns at a time
        uint32_t v[32];
        tmem_ld32(tmem + lanes + 64 * half + 32 * c, v);
        tmem_ld_wait();
        if (tiles == 0)
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = 0u;
        if (parts > 1) {
#pragma unroll
          for (int k = 0; k < 8; ++k)
            *wide_part(part_of_a, wide, row, 16 * half + 8 * c + k) =
                make_uint4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
              x[i] = __uint_as_float(v[8 * k + i]) * (kFScale / (kXScale * kXScale));
            keep(row, 8 * half + 4 * c + k, x, [&](float own, bool diagonal, const float* y) {
              if (diagonal) s.d[row] = own;
              uint4 h, l;
              split(y, &h, &l);
              *tile_part(s.f[half], row, 4 * c + k) = h;
              *tile_part(s.f[2 + half], row, 4 * c + k) = l;
            });
          }
        }
      }
    if (parts > 1) {
      cluster_sync();                     // all parts of A are there
      // an equal share of the rows and columns that there are (in F's place: of all) for each,
      // eight columns at a time; a thread adds up to 64 values, all on their way before the first
      // is added
      const int log = parts == 2 ? 1 : (parts == 4 ? 2 : 3);
      const int eighths = halves == 1 ? (e.m + 7) / 8 : wide / 8, groups = 8 * eighths * eighths;
      const int share = (groups + parts - 1) >> log, end = min((rank + 1) * share, groups);
      const int group = rank * share + me;
      uint4 in[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {      // of the i-th pair: eight columns, a part of A
        const int pair = i >> 1, g = group + (pair >> log) * kSmallThreads;
        in[i] = g < end ? load_remote(wide_part(part_of_a, wide, g / eighths,
                                                2 * (g % eighths) + (i & 1)), pair & (parts - 1))
                        : make_uint4(0, 0, 0, 0);
      }
      if (halves == 2) cluster_sync();    // all have read them
      float x[8];
#pragma unroll
      for (int pair = 0; pair < 8; ++pair) {
        float y[8];
        Granule<float>::unpack(in[2 * pair], y);
        Granule<float>::unpack(in[2 * pair + 1], y + 4);
        const int p = pair & (parts - 1);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = p == 0 ? y[i] : x[i] + y[i];
        const int g = group + (pair >> log) * kSmallThreads;
        if (p != parts - 1 || g >= end) continue;
        const int r = g / eighths, c8 = g % eighths;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= kFScale / (kXScale * kXScale);
        keep(r, c8, x, [&](float own, bool diagonal, const float* y) {
          uint4 h, l;
          split(y, &h, &l);
          for (int c = 0; c < parts; ++c) {
            if (diagonal) store_remote(__float_as_int(own), reinterpret_cast<int*>(&s.d[r]), c);
            store_remote_part(h, tile_part(s.f[c8 >> 3], r, c8 & 7), c);
            store_remote_part(l, tile_part(s.f[2 + (c8 >> 3)], r, c8 & 7), c);
          }
        });
      }
      cluster_sync();                     // all of F
    }
    product([&] {
      for (int t = 0; t < halves; ++t) {
        const uint64_t x = sdesc_sw128(smem_u32(s.f[t]), 16, 1024);
        const uint64_t y = sdesc_sw128(smem_u32(s.f[2 + t]), 16, 1024);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          constexpr uint32_t idesc = idesc_f16(128, 128, false);
          mma_bf16_ss(tmem + 128, x + 2 * k, x + 2 * k, idesc, (t | k) != 0);
          mma_bf16_ss(tmem + 128, x + 2 * k, y + 2 * k, idesc, 1u);
          mma_bf16_ss(tmem + 128, y + 2 * k, x + 2 * k, idesc, 1u);
        }
      }
    });
    const float di = s.d[row], base = fmaf(kC, di, kB) * (1.f / kFScale);
    if (has_part)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        uint32_t v[32];
        tmem_ld32(tmem + 128 + lanes + 64 * half + 32 * c, v);
        tmem_ld_wait();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int col = 64 * half + 32 * c + 8 * k;
          uint4 *hi = tile_part(s.f[half], row, 4 * c + k),
                *lo = tile_part(s.f[2 + half], row, 4 * c + k);
          float x[8], h[8], l[8];
          Granule<__half>::unpack(*hi, h);
          Granule<__half>::unpack(*lo, l);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float ff = __uint_as_float(v[8 * k + i]) * (kC / (kFScale * kFScale));
            x[i] = fmaf(h[i] + l[i], fmaf(s.d[col + i], kC / kFScale, base), ff);
            if (row == col + i) {
              s.e[row] = fmaf(fmaf(kC, di, kB), di, ff);
              x[i] = 0.f;
            }
          }
          split(x, hi, lo);               // G, in F's place
        }
      }
    product([&] {
      if (tiles == 0) return;
      const uint32_t idesc = idesc_f16(128, 64 * tiles, true);
      for (int t = 0; t < halves; ++t) {
        const uint64_t x = sdesc_sw128(smem_u32(s.f[t]), 16, 1024);
        const uint64_t y = sdesc_sw128(smem_u32(s.hi[0]) + t * kHalfTile, kTileBytes, 1024);
        const uint64_t xl = sdesc_sw128(smem_u32(s.f[2 + t]), 16, 1024);
        const uint64_t yl = sdesc_sw128(smem_u32(s.lo[0]) + t * kHalfTile, kTileBytes, 1024);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          mma_bf16_ss(tmem + 256, x + 2 * k, y + 128 * k, idesc, (t | k) != 0);
          mma_bf16_ss(tmem + 256, x + 2 * k, yl + 128 * k, idesc, 1u);
          mma_bf16_ss(tmem + 256, xl + 2 * k, y + 128 * k, idesc, 1u);
        }
      }
    });
    const bool last = step + 1 == steps;
    if (last) {
      // where a wait has run out in any of the CTAs the matrix stays as it is
      if (me < parts) {
        if (parts > 1) store_remote(*abort, &s.bad[rank], me);
        else s.bad[0] = *abort;
      }
      sync();
      int bad = 0;
      for (int c = 0; c < parts; ++c) bad |= s.bad[c];
      if (bad) {
        if (me == 0) record_status(a.status, DORA_ERR_TIMEOUT);
        break;
      }
    }
    const float own = kA + s.e[row];
    for (int p = half; has_rows && p < 2 * tiles; p += 2) {
      uint32_t v[32];
      tmem_ld32(tmem + 256 + lanes + 32 * p, v);
      tmem_ld_wait();
      float x[32];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint4 *hi = tile_part(s.hi[p >> 1], row, 4 * (p & 1) + k),
              *lo = tile_part(s.lo[p >> 1], row, 4 * (p & 1) + k);
        float h[8], l[8];
        Granule<__half>::unpack(*hi, h);
        Granule<__half>::unpack(*lo, l);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          x[8 * k + i] = fmaf(own, h[i] + l[i], __uint_as_float(v[8 * k + i]));
        if (!last) split(x + 8 * k, hi, lo);
      }
      if (last) {
        uint16_t* scratch = reinterpret_cast<uint16_t*>(s.extra[0]) + warp * 2 * kPiece;
        finish_last<true, 32>(e, a, q * 32, col0 + 32 * p, lane, x, scratch, scratch + kPiece);
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (*abort && warp == 0) {              // MMAs that were not waited for end first
    if (elect_one()) {
      mma_commit(&s.drain);
      mbar_wait_limited(&s.drain, 0, kWaitLimitNs);
    }
    __syncwarp();
  }
  if (warp == 0) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

__global__ void __launch_bounds__(kSmallThreads, 1)
    small_kernel(List list, Args a, int steps, int cluster, bool beside) {
  extern __shared__ __align__(1024) uint8_t raw[];
  SmallSmem& s = *reinterpret_cast<SmallSmem*>(raw);
  const int rank = cluster > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  if (!beside) pdl_wait();
  const Entry e = list.entries[list.count + blockIdx.x / cluster];   // read once
  // those of a cluster that have no part leave, and are not waited for
  if (!skipped(a) && rank < e.parts) small_matrix(e, a, steps, rank, s);
  if (beside && blockIdx.x == 0) pdl_wait();   // for the products
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
bool in_quads(const void* p, int32_t dtype) {
  return (reinterpret_cast<uintptr_t>(p) & (dtype == DORA_F32 ? 15u : 7u)) == 0;
}
bool written_in_quads(const dora_matrix& t) {
  return (t.cols & 3) == 0 && in_quads(t.param, t.param_dtype) && in_quads(t.copy, DORA_BF16) &&
         in_quads(t.out, DORA_BF16);
}
bool known_type(int32_t t) { return t >= DORA_BF16 && t <= DORA_F32; }

// Sizes of a matrix, and of all of them.
struct Shape {
  int32_t m, n, mb, nb;
  int64_t chunks, x_tiles, f_tiles, diag;   // diag: blocks of 128 of a diagonal
  int64_t sym[2], all[2];
  int32_t parts;                          // of a small matrix: CTAs; 0: it is not small
};
Shape shape_of(const dora_matrix& t) {
  Shape s;
  s.m = t.rows < t.cols ? t.rows : t.cols;
  s.n = t.rows < t.cols ? t.cols : t.rows;
  s.mb = (s.m + 127) / 128;
  s.nb = (s.n + 127) / 128;
  s.parts = 0;
  if (s.m <= ortho::kSmallRows && s.n <= 64 * ortho::kSmallTiles * ortho::kMaxParts) {
    s.chunks = s.x_tiles = s.f_tiles = s.diag = 0;
    s.sym[0] = s.sym[1] = s.all[0] = s.all[1] = 0;
    s.parts = 1;
    while ((s.n + 63) / 64 > s.parts * ortho::kSmallTiles) s.parts *= 2;
    return s;
  }
  s.chunks = (static_cast<int64_t>(s.m) * s.n + ortho::kChunk - 1) / ortho::kChunk;
  const int64_t pairs = (s.mb + 1) / 2;
  s.x_tiles = pairs * 2 * 2 * s.nb;
  s.f_tiles = pairs * 2 * 2 * s.mb;
  s.diag = pairs * 2;
  // of 256 columns, and of 128; of X in each of its halves
  s.sym[0] = pairs * (pairs + 1) / 2;
  s.all[0] = pairs * ((s.nb + 3) / 4);
  s.sym[1] = pairs * s.mb - pairs * (pairs - 1);
  s.all[1] = pairs * ((s.nb + 1) / 2);
  return s;
}
// A list of fewer wide tiles than pairs of SMs is cut into narrow ones: four matrices of
// 4096 x 1024 and its transpose 0.99 ms, with wide ones 1.04; lists of more are slower with narrow
// ones (384-wide blocks 886 us for 769, the large list 16.3 ms for 13.1).
constexpr int64_t kFewTiles = 76;
struct Sizes {
  int64_t chunks = 0, x_tiles = 0, sym = 0, all = 0, tiles = 0, diag = 0;
  int narrow_sym = 0, narrow_all = 0;     // 1: tiles of 128 columns
  int32_t large = 0, parts = 1;           // matrices that are not small; most CTAs of a small one
  bool has_params = true, has_outs = true, ragged = false;   // ragged: among the large ones
};

// A buffer of a list: [from, to), written by the calls or only read.
struct Extent {
  uintptr_t from, to;
  bool written;
};
// Whether a buffer that is written overlaps any other.
bool overlapping(const dora_matrix* ms, int32_t count) {
  Extent* all = static_cast<Extent*>(malloc(sizeof(Extent) * 5 * static_cast<size_t>(count)));
  if (all == nullptr) return true;
  size_t n = 0;
  for (int32_t i = 0; i < count; ++i) {
    const dora_matrix& t = ms[i];
    const uint64_t elements = static_cast<uint64_t>(t.rows) * static_cast<uint64_t>(t.cols);
    const auto add = [&](const void* p, int32_t dtype, bool written) {
      const uintptr_t at = reinterpret_cast<uintptr_t>(p);
      if (p != nullptr) all[n++] = {at, at + elements * (dtype == DORA_F32 ? 4 : 2), written};
    };
    add(t.grad, t.grad_dtype, false);
    add(t.param, t.param_dtype, true);
    add(t.momentum, DORA_F32, true);
    add(t.copy, DORA_BF16, true);
    add(t.out, DORA_BF16, true);
  }
  std::sort(all, all + n, [](const Extent& a, const Extent& b) { return a.from < b.from; });
  uintptr_t read_to = 0, written_to = 0;  // ends of the buffers so far
  bool overlap = false;
  for (size_t i = 0; i < n; ++i) {
    overlap |= all[i].from < written_to || (all[i].written && all[i].from < read_to);
    uintptr_t& to = all[i].written ? written_to : read_to;
    if (all[i].to > to) to = all[i].to;
  }
  free(all);
  return overlap;
}

bool count_all(const dora_matrix* ms, int32_t count, Sizes* out) {
  Sizes z;
  int64_t sym[2] = {0, 0}, all[2] = {0, 0};
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
    for (int k = 0; k < 2; ++k) {
      sym[k] += s.sym[k];
      all[k] += s.all[k];
    }
    z.tiles += 3 * s.x_tiles + 2 * s.f_tiles;
    z.diag += s.diag;
    z.large += s.parts == 0;
    z.ragged |= s.parts == 0 && !written_in_quads(t);
    if (s.parts > z.parts) z.parts = s.parts;
    if (t.param == nullptr) z.has_params = false;
    if (t.out == nullptr) z.has_outs = false;
    // counted in 32 bits, the tiles' rows among them
    if (z.tiles > (1 << 23) || z.chunks > (1 << 30)) return false;
  }
  if (overlapping(ms, count)) return false;
  // Narrow tiles where wide ones would leave pairs of SMs without any.
  z.narrow_sym = sym[0] < kFewTiles;
  z.narrow_all = all[0] < kFewTiles;
  z.sym = sym[z.narrow_sym];
  z.all = all[z.narrow_all];
  *out = z;
  return true;
}

struct Places {
  int64_t entries, chunk_of, x, sym, all, groups, partial, norm, ticket, done, diag, tiles, end;
};
Places places_of(const Sizes& z, int64_t count) {
  Places p;
  p.entries = round256(sizeof(ortho::Header));
  p.chunk_of = p.entries + round256(count * sizeof(ortho::Entry));
  p.x = p.chunk_of + round256(z.chunks * 4);
  p.sym = p.x + round256(z.x_tiles * sizeof(ortho::Tile));
  p.all = p.sym + round256(z.sym * sizeof(ortho::Tile));
  p.groups = p.all + round256(z.all * sizeof(ortho::Tile));
  p.partial = p.groups + round256(count * sizeof(ortho::Group));
  p.norm = p.partial + round256(z.chunks * 8);
  p.ticket = p.norm + round256(count * 8);
  p.done = p.ticket + round256(count * 4);
  p.diag = p.done + round256(count * 4);
  p.tiles = p.diag + z.diag * 2 * 512;
  p.end = p.tiles + (z.tiles > 0 ? z.tiles : 1) * ortho::kTileBytes;
  return p;
}

ortho::List list_of(const dora_matrix_list& l) {
  Sizes z;
  z.chunks = l.chunks;
  z.x_tiles = l.x_tiles;
  z.sym = l.symmetric;
  z.all = l.outputs;
  z.tiles = l.tiles;
  z.diag = l.diagonals;
  const Places p = places_of(z, l.count);
  char* at = static_cast<char*>(l.data);
  ortho::List o;
  o.header = reinterpret_cast<ortho::Header*>(at);
  o.entries = reinterpret_cast<ortho::Entry*>(at + p.entries);
  o.chunk_of = reinterpret_cast<int32_t*>(at + p.chunk_of);
  o.x = reinterpret_cast<ortho::Tile*>(at + p.x);
  o.sym = reinterpret_cast<ortho::Tile*>(at + p.sym);
  o.all = reinterpret_cast<ortho::Tile*>(at + p.all);
  o.groups = reinterpret_cast<ortho::Group*>(at + p.groups);
  o.tiles = at + p.tiles;
  o.count = l.large;
  o.n_chunks = static_cast<int>(z.chunks);
  o.n_x = static_cast<int>(z.x_tiles);
  o.n_sym = static_cast<int>(z.sym);
  o.n_all = static_cast<int>(z.all);
  return o;
}

bool valid_list(const dora_matrix_list* l) {
  return l != nullptr && l->data != nullptr && l->count >= 1 && l->large >= 0 &&
         l->large <= l->count && l->parts >= 1 && l->parts <= ortho::kMaxParts;
}

int launch_products(const ortho::Maps& maps, const ortho::List& l, const ortho::Args& a, int steps,
                    bool ragged, cudaStream_t stream) {
  constexpr int smem = sizeof(ortho::Smem);
  const auto kern = ragged ? ortho::product_kernel<true> : ortho::product_kernel<false>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return launched(e);
  const int tiles = l.n_sym > 2 * l.n_all ? l.n_sym : 2 * l.n_all, pairs = num_sms() / 2;
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
  return launched(cudaLaunchKernelEx(&cfg, kern, maps, l, a, steps));
}

int launch_small(const ortho::List& l, const ortho::Args& a, int steps, int matrices, int parts,
                 bool beside, cudaStream_t stream) {
  constexpr int smem = sizeof(ortho::SmallSmem);
  const cudaError_t e = cudaFuncSetAttribute(
      ortho::small_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return launched(e);
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (parts > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = parts;
    attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
    ++n;
  }
  if (pdl_enabled()) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  cfg.gridDim = dim3(matrices * parts);
  cfg.blockDim = dim3(ortho::kSmallThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = n;
  return launched(cudaLaunchKernelEx(&cfg, ortho::small_kernel, l, a, steps, parts, beside));
}

int run(const dora_matrix_list* list, int32_t steps, const ortho::Args& a, cudaStream_t stream) {
  const int dev = device_or_error();
  if (dev != DORA_OK) return dev;
  const ortho::List l = list_of(*list);
  ortho::Maps maps;
  static_assert(sizeof(maps) == sizeof(list->map), "the maps' size is part of the interface");
  memcpy(&maps, list->map, sizeof(maps));
  const int most = num_sms() * ortho::kRowCtas, some = num_sms() * ortho::kMomentumCtas;
  int e = DORA_OK;
  if (l.count > 0) {
    e = launched(launch_pdl(ortho::momentum_kernel, dim3(l.n_chunks < some ? l.n_chunks : some),
                            dim3(ortho::kRowThreads), 0, stream, l, a));
    if (e == DORA_OK)
      e = launched(launch_pdl(ortho::normalise_kernel, dim3(l.n_x / 2 < most ? l.n_x / 2 : most),
                              dim3(ortho::kRowThreads), 0, stream, l, a));
    if (e == DORA_OK) e = launch_products(maps, l, a, steps, list->ragged != 0, stream);
  }
  if (e == DORA_OK && list->count > list->large)
    e = launch_small(l, a, steps, list->count - list->large, list->parts, l.count > 0, stream);
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
  l.large = z.large;
  l.parts = z.parts;
  l.ragged = z.ragged;
  l.has_params = z.has_params;
  l.has_outs = z.has_outs;
  // all tiles as one tall matrix of 64 columns
  ortho::Maps maps;
  const uint64_t rows = static_cast<uint64_t>(z.tiles > 0 ? z.tiles : 1) * ortho::kTileRows;
  if (encode_tmap_2d_bf16(&maps.tile, at + p.tiles, 64, rows, 128, 64, 128) != 0 ||
      encode_tmap_2d_bf16(&maps.half, at + p.tiles, 64, rows, 128, 64, 64) != 0 ||
      encode_tmap_2d_bf16(&maps.column, at + p.tiles, 64, rows, 128, 32, 128, 64) != 0 ||
      encode_tmap_2d_bf16(&maps.piece, at + p.tiles, 64, rows, 128, 32, 32, 64) != 0)
    return DORA_ERR_CUDA;
  memcpy(l.map, &maps, sizeof(maps));
  const ortho::List o = list_of(l);
  int64_t tile = 0, chunk = 0, x = 0, sym = 0, all = 0, diag = 0;
  // the small ones after the others
  int32_t at_small[2] = {0, 0};           // next of either kind among the caller's
  const auto next = [&](bool small) -> const dora_matrix& {
    int32_t& i = at_small[small];
    while ((shape_of(matrices[i]).parts > 0) != small) ++i;
    return matrices[i++];
  };
  for (int32_t first = 0; first < count; first += ortho::kFill) {
    const int some = count - first < ortho::kFill ? count - first : ortho::kFill;
    ortho::FillArgs args = {};
    for (int i = 0; i < some; ++i) {
      const dora_matrix& t = next(first + i >= z.large);
      const Shape s = shape_of(t);
      ortho::Entry& e = args.e[i];
      e.grad = t.grad;
      e.param = t.param;
      e.momentum = t.momentum;
      e.copy = t.copy;
      e.out = t.out;
      e.grad_type = t.grad_dtype;
      e.param_type = t.param_dtype;
      e.scale = t.scale;
      e.m = s.m;
      e.n = s.n;
      e.tall = t.rows > t.cols;
      e.quads = written_in_quads(t);
      e.mb = s.mb;
      e.nb = s.nb;
      e.x = tile;
      e.slot = s.x_tiles;
      e.f = tile + 3 * s.x_tiles;
      e.g = e.f + s.f_tiles;
      tile = e.g + s.f_tiles;
      e.d = reinterpret_cast<float*>(at + p.diag) + diag * 256;
      e.e = e.d + s.diag * 128;
      diag += s.diag;
      e.partial = reinterpret_cast<ortho::Squares*>(at + p.partial) + chunk;
      e.norm = reinterpret_cast<float2*>(at + p.norm) + first + i;
      e.ticket = s.parts > 0 ? nullptr : reinterpret_cast<unsigned*>(at + p.ticket) + first + i;
      e.parts = s.parts;
      e.done = reinterpret_cast<unsigned*>(at + p.done) + first + i;
      e.chunks = static_cast<int32_t>(s.chunks);
      e.n_sym = static_cast<int32_t>(s.sym[z.narrow_sym]);
      e.n_all = static_cast<int32_t>(s.all[z.narrow_all]);
      e.sym_width = z.narrow_sym ? 128 : 256;
      e.all_width = z.narrow_all ? 128 : 256;
      e.first_chunk = chunk;
      e.first_x = x;
      e.first_sym = sym;
      e.first_all = all;
      chunk += s.chunks;
      x += s.x_tiles;
      sym += e.n_sym;
      all += e.n_all;
    }
    const int rc = launched(launch_pdl(ortho::fill_entries_kernel, dim3(1), dim3(32), 0, stream, o,
                                       first, some, args));
    if (rc != DORA_OK) return rc;
  }
  int64_t most = z.chunks > z.x_tiles ? z.chunks : z.x_tiles;
  if (z.sym > most) most = z.sym;
  if (z.all > most) most = z.all;
  if (most == 0) most = 1;
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
      !isfinite(static_cast<float>(lr)) || !(momentum >= 0. && momentum < 1.) ||
      !(weight_decay >= 0.) || !isfinite(static_cast<float>(1. - lr * weight_decay)))
    return DORA_ERR_INVALID_ARG;          // the kernels take them in 32 bits
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
