// Embeddings of a tree's packed tokens and their gradient.
//
// Forward x[t] = scale * table[id_t], a gather of rows.  Backward d_table[v] = scale * sum of d_x over the tokens
// with id v: the host has sorted the tokens by id, so every row of the gradient has one owner that adds its tokens' rows
// in ascending order in fp32: no atomics, and nothing is read or written twice but the partial sums of ids with more
// than 64 tokens.  Both are bound by memory.  56462 tokens of width 4096, bf16: forward 141 us for the 0.93 GB that x and
// its tokens' rows are (6.6 TB/s; rows of ids that come again are found in the caches); backward into 65536 rows 201 us, 6 of them
// for the long sums, for the 1.0 GB of d_x and d_table (5.0 TB/s; a large copy reaches 5.2).
#include "dta_vocab.h"

namespace dta {
namespace {

constexpr int kThreads = 256;

// A thread holds 16 bytes of a row: 8 bf16 or 4 fp32.
template <typename T>
struct Piece;
template <>
struct Piece<float> {
  static constexpr int kN = 4;
  typedef float raw __attribute__((ext_vector_type(4)));
  __device__ static void widen(const raw& r, float* f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = r[e];
  }
  __device__ static raw narrow(const float* f) {
    raw r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = f[e];
    return r;
  }
};
template <>
struct Piece<__bf16> {
  static constexpr int kN = 8;
  typedef __bf16 raw __attribute__((ext_vector_type(8)));
  __device__ static void widen(const raw& r, float* f) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (float)r[e];
  }
  __device__ static raw narrow(const float* f) {
    raw r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (__bf16)f[e];
    return r;
  }
};

// Results that the memory-side cache (256 MB) cannot keep for the pass that reads them next are stored past it: they would drive
// out what the call still reads and, dirty, be written out under the next pass' reads.  By itself a call is faster that way at
// almost any size, but the pass behind it then finds nothing in the cache; what counts is both together.  us of both, by plain
// stores and past the cache, and in brackets of the call alone (bf16, width 2560, three sets of tensors in turn; fp32 is alike):
//   x of            112 MB 89, 94 (54, 31); 200 MB 150, 160 (91, 52); 300 MB 242, 232 (131, 76); 500 MB 391, 369 (208, 125)
//   a table from 90 MB of d_x: 180 MB 120, 137 (72, 65); 250 MB 157, 176 (94, 80); 330 MB 216, 221 (113, 96);
//                   420 MB 281, 268 (133, 113); 600 MB 380, 366 (170, 148); 1300 MB 753, 748 (291, 284)
//   from 8 MB:      250 MB 131, 154; 330 MB 192, 197; 420 MB 245, 243; 850 MB 478, 479;  from 350 MB: 261, 266; 312, 313; 379, 369; 630, 602
// The sign goes by the result's size, whatever d_x or the table beside it takes.  A table's pass behind begins while the call's
// other reads still fill the cache: it crosses later.
constexpr int64_t kStreamRows = (int64_t)256 << 20, kStreamTable = (int64_t)384 << 20;   // bytes of the result

template <bool STREAM, typename R>   // (a type's choice: two branches are made one plain store)
__device__ __forceinline__ void put_raw(R* p, const R& x) {
  if (STREAM) __builtin_nontemporal_store(x, p);
  else *p = x;
}

// How a block of 256 threads lies over rows of `pieces` 16-byte pieces: 2^shift threads side by side on a row (256, or
// the power of two that covers a shorter row), 256 >> shift rows.
int row_shift(int pieces) {
  int s = 3;
  while (s < 8 && (1 << s) < pieces) ++s;
  return s;
}

template <typename T, bool STREAM>
__global__ void __launch_bounds__(kThreads)
embed_fwd_kernel(const T* __restrict__ table, const int32_t* __restrict__ id, T* __restrict__ x, int64_t n_rows, int pieces,
                 int shift, int col_blocks, float scale) {
  typedef typename Piece<T>::raw raw;
  const int64_t rb = blockIdx.x / col_blocks;
  const int piece = (int)(blockIdx.x % col_blocks) * kThreads + (int)(threadIdx.x & ((1 << shift) - 1));
  const int64_t t = (rb << (8 - shift)) + (threadIdx.x >> shift);
  if (t >= n_rows || piece >= pieces) return;
  const raw r = ((const raw*)table)[(int64_t)id[t] * pieces + piece];
  float f[Piece<T>::kN];
  Piece<T>::widen(r, f);
#pragma unroll
  for (int e = 0; e < Piece<T>::kN; ++e) f[e] *= scale;
  put_raw<STREAM>((raw*)x + t * pieces + piece, Piece<T>::narrow(f));
}

// One row of the gradient, or of the partial sums.  O: what it is written as; `add`: into an fp32 accumulator.
template <typename T, bool STREAM>
__device__ void put(void* out, int64_t row, int pieces, int piece, const float* f, bool add) {
  typedef typename Piece<T>::raw raw;
  constexpr int N = Piece<T>::kN;
  if (!add) {
    put_raw<STREAM>((raw*)out + row * pieces + piece, Piece<T>::narrow(f));
    return;
  }
  float4* acc = (float4*)out + (row * pieces + piece) * (N / 4);
#pragma unroll
  for (int q = 0; q < N / 4; ++q) {
    float4 v = acc[q];
    v.x += f[4 * q];
    v.y += f[4 * q + 1];
    v.z += f[4 * q + 2];
    v.w += f[4 * q + 3];
    acc[q] = v;
  }
}

template <typename T, bool STREAM>
__global__ void __launch_bounds__(kThreads)
embed_bwd_kernel(const T* __restrict__ d_x, const EmbedPart* __restrict__ part, int n_parts, const int32_t* __restrict__ order,
                 const uint32_t* __restrict__ present, int vocab, void* __restrict__ d_table, float* __restrict__ partial,
                 int pieces, int shift, int col_blocks, int64_t part_blocks, float scale, bool add) {
  typedef typename Piece<T>::raw raw;
  constexpr int N = Piece<T>::kN;
  const int piece = (int)(blockIdx.x % col_blocks) * kThreads + (int)(threadIdx.x & ((1 << shift) - 1));
  if (piece >= pieces) return;
  const int64_t b = blockIdx.x / col_blocks;
  const int sub = (int)(threadIdx.x >> shift), subs = kThreads >> shift;
  if (b >= part_blocks) {   // ids that do not occur: 32 of them
    const int64_t v0 = (b - part_blocks) * 32;
    const uint32_t word = present[b - part_blocks];
    float zero[N] = {};
    for (int i = sub; i < 32; i += subs)
      if (v0 + i < vocab && !(word >> i & 1)) put_raw<STREAM>((raw*)d_table + (v0 + i) * pieces + piece, Piece<T>::narrow(zero));
    return;
  }
  const int64_t at = b * subs + sub;
  if (at >= n_parts) return;
  const EmbedPart p = part[at];
  float sum[N] = {};
  int i = p.begin;
  for (; i + 4 <= p.end; i += 4) {   // four rows in flight, added in order
    raw r[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) r[u] = ((const raw*)d_x)[(int64_t)order[i + u] * pieces + piece];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      float f[N];
      Piece<T>::widen(r[u], f);
#pragma unroll
      for (int e = 0; e < N; ++e) sum[e] += f[e];
    }
  }
  for (; i < p.end; ++i) {
    float f[N];
    Piece<T>::widen(((const raw*)d_x)[(int64_t)order[i] * pieces + piece], f);
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] += f[e];
  }
  if (p.slot >= 0) {
    float4* dst = (float4*)partial + ((int64_t)p.slot * pieces + piece) * (N / 4);
#pragma unroll
    for (int q = 0; q < N / 4; ++q) dst[q] = make_float4(sum[4 * q], sum[4 * q + 1], sum[4 * q + 2], sum[4 * q + 3]);
    return;
  }
#pragma unroll
  for (int e = 0; e < N; ++e) sum[e] *= scale;
  put<T, STREAM>(d_table, p.id, pieces, piece, sum, add);
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
embed_merge_kernel(const float* __restrict__ partial, const EmbedMerge* __restrict__ merge, int n_merges,
                   void* __restrict__ d_table, int pieces, int shift, int col_blocks, float scale, bool add) {
  constexpr int N = Piece<T>::kN;
  const int piece = (int)(blockIdx.x % col_blocks) * kThreads + (int)(threadIdx.x & ((1 << shift) - 1));
  const int64_t at = (int64_t)(blockIdx.x / col_blocks) * (kThreads >> shift) + (threadIdx.x >> shift);
  if (piece >= pieces || at >= n_merges) return;
  const EmbedMerge m = merge[at];
  float sum[N] = {};
#pragma unroll 4
  for (int i = 0; i < m.n; ++i) {
    const float4* src = (const float4*)partial + ((int64_t)(m.first + i) * pieces + piece) * (N / 4);
#pragma unroll
    for (int q = 0; q < N / 4; ++q) {
      const float4 v = src[q];
      sum[4 * q] += v.x;
      sum[4 * q + 1] += v.y;
      sum[4 * q + 2] += v.z;
      sum[4 * q + 3] += v.w;
    }
  }
#pragma unroll
  for (int e = 0; e < N; ++e) sum[e] *= scale;
  put<T, false>(d_table, m.id, pieces, piece, sum, add);
}

template <typename T>
int embed_fwd(const VocabArgs& a) {
  const int pieces = a.p.width / Piece<T>::kN, shift = row_shift(pieces), cols = (pieces + kThreads - 1) / kThreads;
  const int rows = kThreads >> shift;
  const int64_t T_ = a.tokens->n_tokens;
  clear_hip_error();
  const auto kernel = T_ * pieces * 16 >= kStreamRows ? embed_fwd_kernel<T, true> : embed_fwd_kernel<T, false>;
  launch(a, true, kernel, (size_t)((T_ + rows - 1) / rows * cols), kThreads, (const T*)a.table, a.tab.id, (T*)a.x, T_, pieces, shift,
         cols, a.p.scale);
  return launch_status("embeddings");
}

template <typename T>
int embed_bwd(const VocabArgs& a) {
  const dta_tokens* t = a.tokens;
  const int pieces = a.p.width / Piece<T>::kN, shift = row_shift(pieces), cols = (pieces + kThreads - 1) / kThreads;
  const int rows = kThreads >> shift;
  const int64_t part_blocks = (t->n_parts + rows - 1) / rows;
  const int64_t zero_blocks = a.add || t->n_distinct == t->vocab ? 0 : ((int64_t)t->vocab + 31) / 32;
  float* partial = (float*)a.workspace;
  clear_hip_error();
  const auto kernel = (int64_t)t->vocab * pieces * 16 >= kStreamTable ? embed_bwd_kernel<T, true> : embed_bwd_kernel<T, false>;
  launch(a, t->n_merges == 0, kernel, (size_t)((part_blocks + zero_blocks) * cols), kThreads, (const T*)a.d_x, a.tab.part, t->n_parts,
         a.tab.order, a.tab.present, t->vocab, a.d_table, partial, pieces, shift, cols, part_blocks, a.p.scale, a.add);
  if (t->n_merges)
    launch(a, true, embed_merge_kernel<T>, (size_t)((t->n_merges + rows - 1) / rows * cols), kThreads, partial, a.tab.merge,
           t->n_merges, a.d_table, pieces, shift, cols, a.p.scale, a.add);
  return launch_status("embedding gradient");
}

}  // namespace

size_t embed_bwd_workspace(const dta_tokens* t, const dta_vocab_params_t* p) {
  return (size_t)t->n_slots * (size_t)p->width * sizeof(float);   // (a multiple of 256: width is one of 64)
}

int launch_embed_fwd(const VocabArgs& a) { return a.p.dtype == DTA_F32 ? embed_fwd<float>(a) : embed_fwd<__bf16>(a); }
int launch_embed_bwd(const VocabArgs& a) { return a.p.dtype == DTA_F32 ? embed_bwd<float>(a) : embed_bwd<__bf16>(a); }

}  // namespace dta
