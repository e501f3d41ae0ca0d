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
constexpr int kChunk = 8192;              // elements of a matrix that a CTA takes at once
constexpr int kRowThreads = 256;
constexpr int kMaxShort = 16384, kMaxLong = 1 << 24;

struct Entry {
  const void* grad;
  void* param;
  float* momentum;
  uint16_t *copy, *out;                   // bf16
  int32_t rows, cols, grad_type, param_type;
  float scale;
  int32_t m, n, tall;                     // X is m x n; tall: X = U^T
  int32_t mb, nb;                         // blocks of 128 rows, of 128 columns
  int64_t x[2], lo, f, g;                 // first tiles of X hi (two, in turn), X lo, F, G
  float *d, *e;                           // the diagonals of A and B [128 mb]
  float2* partial;                        // of its chunks: sum of squares and exponent
  float2* norm;                           // one over the norm of u 2^-k, and 2^-k's exponent
  unsigned* ticket;                       // chunks done; zero between calls
  int32_t chunks, pad;
  // first of its chunks, of its tiles of X and of its output tiles among the list's
  int64_t first_chunk, first_x, first_sym, first_all;
};

struct Header {
  int abort;                              // a bounded wait of this call has run out
  int pad[63];
};

// One piece of work: block row and block column of a matrix.
struct Tile {
  int32_t matrix, i, j, pad;
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
    const int at = static_cast<int>(t - list.entries[q].first_all), w = list.entries[q].nb;
    list.all[t] = Tile{q, at / w, at % w, 0};
  }
  if (t < list.n_sym) {
    const int q = matrix_of(list, t, [](const Entry& e) { return e.first_sym; });
    int at = static_cast<int>(t - list.entries[q].first_sym), i = 0, left = list.entries[q].mb;
    while (at >= left) {
      at -= left--;
      ++i;
    }
    list.sym[t] = Tile{q, i, i + at, 0};
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
// Momentum, and the update's norm.  Squares are summed of u 2^-k with k the exponent of the
// chunk's largest |u|, so that no finite update overflows or vanishes; the chunks are joined
// in their order by the CTA that is last of the matrix.
// ---------------------------------------------------------------------------
__device__ __forceinline__ float block_reduce(float v, bool largest, float* scratch) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    const float o = __shfl_xor_sync(0xffffffffu, v, off);
    v = largest ? fmaxf(v, o) : v + o;
  }
  __syncthreads();                        // the places are free
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
  __syncthreads();
  v = scratch[0];
#pragma unroll
  for (int w = 1; w < kRowThreads / 32; ++w) v = largest ? fmaxf(v, scratch[w]) : v + scratch[w];
  return v;
}

// The exponent by which values up to `top` are brought near 1.
__device__ __forceinline__ int exponent_of(float top) {
  const int e = static_cast<int>(__float_as_uint(top) >> 23) - 127;   // top >= 0
  return e < -126 ? -126 : (e > 127 ? 127 : e);
}

__global__ void __launch_bounds__(kRowThreads) momentum_kernel(List list, Args a) {
  constexpr int kPer = kChunk / kRowThreads;
  __shared__ float scratch[kRowThreads / 32];
  __shared__ bool last;
  pdl_wait();
  if (skipped(a)) return;
  const float f = factor(a);
  if (blockIdx.x == 0 && threadIdx.x == 0) list.header->abort = 0;
  for (int c = blockIdx.x; c < list.n_chunks; c += gridDim.x) {
    const Entry& e = list.entries[list.chunk_of[c]];
    const int at = static_cast<int>(c - e.first_chunk);
    const int64_t total = static_cast<int64_t>(e.rows) * e.cols;
    const int64_t from = static_cast<int64_t>(at) * kChunk;
    float u[kPer], top = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int64_t k = from + threadIdx.x + i * kRowThreads;
      u[i] = 0.f;
      if (k < total) {
        const float d = load_one(e.grad, e.grad_type, k) * f;
        float m = 0.f;
        if (a.muon) {
          m = fmaf(a.mu, e.momentum[k], a.omu * d);
          e.momentum[k] = m;
        }
        u[i] = update_of(a, d, m);
        top = fmaxf(top, fabsf(u[i]));
      }
    }
    const int k = exponent_of(block_reduce(top, true, scratch));
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const float v = ldexpf(u[i], -k);
      sum = fmaf(v, v, sum);
    }
    sum = block_reduce(sum, false, scratch);
    if (threadIdx.x == 0) {
      e.partial[at] = make_float2(sum, static_cast<float>(k));
      last = take_ticket(e.ticket) == static_cast<unsigned>(e.chunks) - 1;
    }
    __syncthreads();
    if (!last) continue;
    float most = -126.f;
    for (int i = threadIdx.x; i < e.chunks; i += kRowThreads)
      most = fmaxf(most, __ldcg(&e.partial[i]).y);
    most = block_reduce(most, true, scratch);
    float all = 0.f;
    for (int i = threadIdx.x; i < e.chunks; i += kRowThreads) {
      const float2 p = __ldcg(&e.partial[i]);
      all += ldexpf(p.x, 2 * static_cast<int>(p.y - most));
    }
    all = block_reduce(all, false, scratch);
    if (threadIdx.x == 0) {
      // a matrix of zeros stays one; one that is not finite becomes NaN
      *e.norm = make_float2(all == 0.f ? 0.f : (isfinite(all) ? rsqrtf(all) : NAN), -most);
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

// hi and lo of eight values that are scaled already.
__device__ __forceinline__ void split(const float* v, uint4* hi, uint4* lo) {
  float rest[8], back[8];
  *hi = Granule<__half>::pack(v);
  Granule<__half>::unpack(*hi, back);
#pragma unroll
  for (int i = 0; i < 8; ++i) rest[i] = (v[i] - back[i]) * kLoScale;
  *lo = Granule<__half>::pack(rest);
}

// The normalised update into its tiles, a tile a CTA.
__global__ void __launch_bounds__(kRowThreads) normalise_kernel(List list, Args a) {
  pdl_wait();
  if (skipped(a)) return;
  const float f = factor(a);
  for (int t = blockIdx.x; t < list.n_x; t += gridDim.x) {
    const Tile tile = list.x[t];
    const Entry& e = list.entries[tile.matrix];
    const float2 norm = *e.norm;
    const int64_t at = static_cast<int64_t>(tile.i) * (2 * e.nb) + tile.j;
    char* hi = tile_at(list, e.x[0] + at);
    char* lo = tile_at(list, e.lo + at);
    for (int w = threadIdx.x; w < kTileRows * 8; w += kRowThreads) {
      // the lanes along what is contiguous in the matrix
      const int r = e.tall ? w % kTileRows : w / 8, piece = e.tall ? w / kTileRows : w % 8;
      const int row = tile.i * kTileRows + r, col = tile.j * kTileCols + piece * 8;
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[i] = 0.f;
        if (row < e.m && col + i < e.n) {
          const int64_t k = e.tall ? static_cast<int64_t>(col + i) * e.m + row
                                   : static_cast<int64_t>(row) * e.n + col + i;
          const float d = load_one(e.grad, e.grad_type, k) * f;
          const float u = update_of(a, d, a.muon ? e.momentum[k] : 0.f);
          v[i] = ldexpf(u, static_cast<int>(norm.y)) * norm.x * kScale;
        }
      }
      uint4 h, l;
      split(v, &h, &l);
      const uint32_t to = tile_offset(r, piece * 8);
      *reinterpret_cast<uint4*>(hi + to) = h;
      *reinterpret_cast<uint4*>(lo + to) = l;
    }
  }
}

// ---------------------------------------------------------------------------
// The products.  One persistent CTA an SM takes output tiles of 128 x 128: one warp copies
// operands into a ring of stages, one issues the MMAs into one of two accumulators, four
// read the other one and write what comes of it.
// ---------------------------------------------------------------------------
enum Phase { kGram, kSquare, kApply, kLast };

constexpr int kStages = 6;
constexpr int kBlock = 128;               // of an output tile
constexpr int kK = 64;                    // of a stage
constexpr int kThreads = 192;
constexpr int kHalfTile = kTileBytes / 2; // 64 rows: what one copy brings

struct Smem {
  uint8_t a[kStages][kTileBytes];
  uint8_t b[kStages][kTileBytes];
  uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2], drain;
  uint32_t tmem;
  int abort, issued, consumed;
};

__host__ __device__ constexpr uint32_t idesc_f16(int m, int n, bool b_mn_major) {
  return (1u << 4) | ((b_mn_major ? 1u : 0u) << 16) | (static_cast<uint32_t>(n >> 3) << 17) |
         (static_cast<uint32_t>(m >> 4) << 24);
}

// A row of 32 fp32 values of the accumulator at hand, with its place in the matrix.
template <Phase kPhase>
__device__ __forceinline__ void finish_row(const List& list, const Entry& e, const Args& a,
                                           const Tile& t, int from, int r, int c,
                                           const uint32_t (&acc)[32]) {
  const int row = t.i * kBlock + r, col = t.j * kBlock + c;   // c: the first of 32 columns
  if (kPhase == kGram || kPhase == kSquare) {
    const int64_t first = kPhase == kGram ? e.f : e.g;
    char* to = tile_at(list, first + static_cast<int64_t>(t.i) * 2 * e.mb + 2 * t.j + (c >> 6));
    char* mirror = tile_at(list, first + static_cast<int64_t>(t.j) * 2 * e.mb + 2 * t.i + (r >> 6));
    const char* f = kPhase == kSquare
                        ? tile_at(list, e.f + static_cast<int64_t>(t.i) * 2 * e.mb + 2 * t.j +
                                            (c >> 6))
                        : nullptr;
    const float di = kPhase == kSquare ? e.d[row] : 0.f;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      float v[8];
      if constexpr (kPhase == kGram) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x = __uint_as_float(acc[8 * p + i]);
          if (row == col + 8 * p + i) e.d[row] = x * (1.f / (kScale * kScale));
          v[i] = row == col + 8 * p + i ? 0.f : x * (1.f / kScale);
        }
      } else {
        float off[8];
        Granule<__half>::unpack(
            *reinterpret_cast<const uint4*>(f + tile_offset(r, (c & 63) + 8 * p)), off);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float ff = __uint_as_float(acc[8 * p + i]) * (1.f / kScale);   // scaled once
          const float dj = e.d[col + 8 * p + i];
          v[i] = fmaf(kC, fmaf(di + dj, off[i], ff), kB * off[i]);
          if (row == col + 8 * p + i) {
            e.e[row] = fmaf(kC, fmaf(di, di, ff * (1.f / kScale)), kB * di);
            v[i] = 0.f;
          }
        }
      }
      const uint4 q = Granule<__half>::pack(v);
      *reinterpret_cast<uint4*>(to + tile_offset(r, (c & 63) + 8 * p)) = q;
      if (t.i != t.j) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 8; ++i)
          *reinterpret_cast<uint16_t*>(mirror + tile_offset(c + 8 * p + i, r & 63)) =
              static_cast<uint16_t>(w[i >> 1] >> (16 * (i & 1)));
      }
    }
    return;
  }
  const int64_t at = static_cast<int64_t>(t.i) * (2 * e.nb) + 2 * t.j + (c >> 6);
  const char* hi = tile_at(list, e.x[from] + at);
  char* lo = tile_at(list, e.lo + at);
  char* to = tile_at(list, e.x[from ^ 1] + at);
  const float ae = kA + e.e[row];
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const uint32_t o = tile_offset(r, (c & 63) + 8 * p);
    float h[8], l[8], v[8];
    Granule<__half>::unpack(*reinterpret_cast<const uint4*>(hi + o), h);
    Granule<__half>::unpack(*reinterpret_cast<const uint4*>(lo + o), l);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      v[i] = fmaf(ae, fmaf(l[i], 1.f / kLoScale, h[i]),
                  __uint_as_float(acc[8 * p + i]) * (1.f / kScale));
    if constexpr (kPhase == kApply) {
      uint4 vh, vl;
      split(v, &vh, &vl);
      *reinterpret_cast<uint4*>(to + o) = vh;
      *reinterpret_cast<uint4*>(lo + o) = vl;
    } else if (row < e.m) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int cc = col + 8 * p + i;
        if (cc >= e.n) continue;
        const int64_t k = e.tall ? static_cast<int64_t>(cc) * e.m + row
                                 : static_cast<int64_t>(row) * e.n + cc;
        const float x = v[i] * (1.f / kScale);
        if (!a.muon) {
          store_one(x, e.out, DORA_BF16, k);
        } else {
          const float w = fmaf(load_one(e.param, e.param_type, k), a.keep, -(a.lr * e.scale) * x);
          store_one(w, e.param, e.param_type, k);
          if (e.copy != nullptr) store_one(w, e.copy, DORA_BF16, k);
        }
      }
    }
  }
}

template <Phase kPhase>
__global__ void __launch_bounds__(kThreads, 1)
    product_kernel(const __grid_constant__ CUtensorMap map, List list, Args a, int from) {
  extern __shared__ __align__(1024) uint8_t raw[];
  pdl_trigger();
  Smem& s = *reinterpret_cast<Smem*>(raw);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr bool kSym = kPhase == kGram || kPhase == kSquare;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&s.full[i], 1);
      mbar_init(&s.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s.acc_full[i], 1);
      mbar_init(&s.acc_empty[i], 4);
    }
    mbar_init(&s.drain, 1);
    s.abort = s.issued = s.consumed = 0;
    fence_barrier_init();
    tma_prefetch_desc(&map);
  }
  if (warp == 1) tmem_alloc(&s.tmem, 2 * kBlock);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_wait();
  const Tile* tiles = kSym ? list.sym : list.all;
  const int n_tiles = skipped(a) || list.header->abort ? 0 : (kSym ? list.n_sym : list.n_all);
  const uint32_t tmem = s.tmem;
  volatile int* abort = &s.abort;
  // stages of a tile: the K of its product over 64
  auto steps = [&](const Entry& e) { return kPhase == kGram ? 2 * e.nb : 2 * e.mb; };

  if (warp == 0) {
    if (elect_one()) {
      int it = 0;
      bool ok = true;
      for (int w = blockIdx.x; ok && w < n_tiles; w += gridDim.x) {
        const Tile t = tiles[w];
        const Entry& e = list.entries[t.matrix];
        const int n = steps(e), wide = kPhase == kGram ? 2 * e.nb : 2 * e.mb;
        const int64_t first_a = kPhase == kGram ? e.x[from] : (kPhase == kSquare ? e.f : e.g);
        const int64_t row_a = first_a + static_cast<int64_t>(t.i) * wide;
        for (int k = 0; k < n; ++k, ++it) {
          const int st = it % kStages;
          if (!mbar_wait(&s.empty[st], ((it / kStages) & 1) ^ 1, abort)) {
            ok = false;
            break;
          }
          mbar_arrive_expect_tx(&s.full[st], 2 * kTileBytes);
          const int32_t ya = static_cast<int32_t>((row_a + k) * kTileRows);
          tma_load_2d(s.a[st], &map, &s.full[st], 0, ya);
          tma_load_2d(s.a[st] + kHalfTile, &map, &s.full[st], 0, ya + 64);
          int32_t yb, yb2;
          if (kSym) {
            yb = static_cast<int32_t>((first_a + static_cast<int64_t>(t.j) * wide + k) * kTileRows);
            yb2 = yb + 64;
          } else {                        // 64 rows of X, of two tiles side by side
            yb = static_cast<int32_t>(
                (e.x[from] + static_cast<int64_t>(k >> 1) * 2 * e.nb + 2 * t.j) * kTileRows +
                (k & 1) * 64);
            yb2 = yb + kTileRows;
          }
          tma_load_2d(s.b[st], &map, &s.full[st], 0, yb);
          tma_load_2d(s.b[st] + kHalfTile, &map, &s.full[st], 0, yb2);
        }
      }
      s.issued = it;
    }
  } else if (warp == 1) {
    if (elect_one()) {
      constexpr uint32_t idesc = idesc_f16(kBlock, kBlock, !kSym);
      int it = 0, ti = 0;
      bool ok = true;
      for (int w = blockIdx.x; ok && w < n_tiles; w += gridDim.x, ++ti) {
        const int n = steps(list.entries[tiles[w].matrix]);
        const int acc = ti & 1;
        if (!mbar_wait(&s.acc_empty[acc], ((ti >> 1) & 1) ^ 1, abort)) break;
        tc_fence_after();
        const uint32_t d = tmem + static_cast<uint32_t>(acc * kBlock);
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
            mma_bf16_ss(d, ad + 2 * q, bd + (kSym ? 2 : 128) * q, idesc, (k | q) != 0 ? 1u : 0u);
          mma_commit(&s.empty[st]);
        }
        if (ok) mma_commit(&s.acc_full[acc]);
      }
      s.consumed = it;
      mma_commit(&s.drain);
      mbar_wait_limited(&s.drain, 0, kWaitLimitNs);
    }
  } else {
    const int q = warp & 3, r = q * 32 + lane;
    int ti = 0;
    for (int w = blockIdx.x; w < n_tiles; w += gridDim.x, ++ti) {
      const Tile t = tiles[w];
      const Entry& e = list.entries[t.matrix];
      const int acc = ti & 1;
      if (!mbar_wait_warp(&s.acc_full[acc], (ti >> 1) & 1, abort)) break;
      tc_fence_after();
      for (int c = 0; c < kBlock; c += 32) {
        uint32_t v[32];
        tmem_ld32(tmem + (static_cast<uint32_t>(q * 32) << 16) + acc * kBlock + c, v);
        tmem_ld_wait();
        finish_row<kPhase>(list, e, a, t, from, r, c, v);
      }
      warp_arrive(&s.acc_empty[acc]);
    }
  }

  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (*abort) {
    if (threadIdx.x == 0) {
      list.header->abort = 1;
      record_status(a.status, DORA_ERR_TIMEOUT);
      // loads that were issued but never consumed land first
      for (int it = s.consumed; it < s.issued; ++it)
        mbar_wait_limited(&s.full[it % kStages], (it / kStages) & 1, 100ull * 1000 * 1000);
    }
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 2 * kBlock);
  }
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
  int64_t chunks, x_tiles, f_tiles, sym, all;
};
Shape shape_of(const dora_matrix& t) {
  Shape s;
  s.m = t.rows < t.cols ? t.rows : t.cols;
  s.n = t.rows < t.cols ? t.cols : t.rows;
  s.mb = (s.m + 127) / 128;
  s.nb = (s.n + 127) / 128;
  s.chunks = (static_cast<int64_t>(s.m) * s.n + ortho::kChunk - 1) / ortho::kChunk;
  s.x_tiles = static_cast<int64_t>(s.mb) * 2 * s.nb;
  s.f_tiles = static_cast<int64_t>(s.mb) * 2 * s.mb;
  s.sym = static_cast<int64_t>(s.mb) * (s.mb + 1) / 2;
  s.all = static_cast<int64_t>(s.mb) * s.nb;
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
    z.diag += s.mb;
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
int launch_product(const CUtensorMap& map, const ortho::List& l, const ortho::Args& a, int from,
                   cudaStream_t stream) {
  constexpr int smem = sizeof(ortho::Smem);
  const cudaError_t e = cudaFuncSetAttribute(ortho::product_kernel<kPhase>,
                                             cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return launched(e);
  const int tiles = kPhase == ortho::kGram || kPhase == ortho::kSquare ? l.n_sym : l.n_all;
  return launched(launch_pdl(ortho::product_kernel<kPhase>,
                             dim3(tiles < num_sms() ? tiles : num_sms()), dim3(ortho::kThreads),
                             smem, stream, map, l, a, from));
}

int run(const dora_matrix_list* list, int32_t steps, const ortho::Args& a, cudaStream_t stream) {
  const int dev = device_or_error();
  if (dev != DORA_OK) return dev;
  const ortho::List l = list_of(*list);
  CUtensorMap map;
  memcpy(&map, list->map, sizeof(map));
  const int most = num_sms() * 4;
  int e = launched(launch_pdl(ortho::momentum_kernel, dim3(l.n_chunks < most ? l.n_chunks : most),
                              dim3(ortho::kRowThreads), 0, stream, l, a));
  if (e == DORA_OK)
    e = launched(launch_pdl(ortho::normalise_kernel, dim3(l.n_x < most ? l.n_x : most),
                            dim3(ortho::kRowThreads), 0, stream, l, a));
  for (int s = 0; s < steps && e == DORA_OK; ++s) {
    e = launch_product<ortho::kGram>(map, l, a, s & 1, stream);
    if (e == DORA_OK) e = launch_product<ortho::kSquare>(map, l, a, s & 1, stream);
    if (e == DORA_OK)
      e = s + 1 < steps ? launch_product<ortho::kApply>(map, l, a, s & 1, stream)
                        : launch_product<ortho::kLast>(map, l, a, s & 1, stream);
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
  CUtensorMap map;
  // all tiles as one tall matrix of 64 columns
  if (encode_tmap_2d_bf16(&map, at + p.tiles, ortho::kTileCols,
                          static_cast<uint64_t>(z.tiles) * ortho::kTileRows, 128,
                          ortho::kTileCols, 64) != 0)
    return DORA_ERR_CUDA;
  memcpy(l.map, &map, sizeof(map));
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
      e.e = e.d + s.mb * 128;
      diag += s.mb;
      e.partial = reinterpret_cast<float2*>(at + p.partial) + chunk;
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
