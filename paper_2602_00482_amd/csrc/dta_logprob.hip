// Log-probabilities of a tree's tokens under a softmax over the vocabulary, and their gradient.
//
//   z = scale * H W^T          H: hidden states of the rows before a scored token, W: the output matrix
//   lse = ln sum exp z,  logp = z[id] - lse
//   dz = d_logp at the ids - c exp(z - lse),   dH = scale dz W,   dW = scale dz^T H
//
// All of it is matrix products; what is around them happens in their epilogues, so the logits never leave the chip in
// the forward pass, and in the backward pass dz exists for a block of the vocabulary at a time.
//
// What bounds it: from about 200 rows on the matrix instructions, with fewer the way of W from memory.  Measured, bf16
// unless said otherwise (rows x ids x width; a large library product of such sizes does 1.49 PFLOP/s, a large copy 5.2 TB/s; GPUs of
// the kind differ by 5 % under the power limit):
//   logits and their statistics   18.4K x 50021 x 2048 2.7 to 2.85 ms, 1.33 to 1.40 PFLOP/s; 18.4K x 65536 x 4096 6.6 to 7.0 ms, 1.42 to 1.49
//   logits again and dz           the latter 6.8 to 7.1 ms;  dH 7.1 to 7.4 ms;  dW 7.1 to 7.5 ms: 1.45 to 1.32
//   33 x 131072 x 4096            181 us, W at 5.9 TB/s
//   fp32 in three parts           4.6K x 32000 x 1024 1.2 to 1.36 ms: 1.33 to 1.50 PFLOP/s of the bf16 instruction
#include <algorithm>
#include <type_traits>

#include "dta_mfma.h"
#include "dta_vocab.h"

namespace dta {
namespace {

// ---- operands -----------------------------------------------------------------------
// The products are C[n][m] = sum_k A[m][k] B[n][k], with the accumulators' rows along m: a lane of the matrix instruction
// (n = l % 16, g = l / 16) then holds 4 consecutive m of one n, which is the order results are stored in
// (m: vocabulary for z and dz, width for dH and dW), and a softmax row (n) is a lane.
//   z  [row][v]:      A = W           B = H        k = width
//   dH [row][width]:  A = W^T         B = dz       k = vocabulary
//   dW [v][width]:    A = H^T         B = dz^T     k = rows
// Operands of the first product and dz in the second lie with k along memory ("row operand"), the others with m or n along
// memory ("column operand", read through the transposing LDS read).

struct Bf16 {
  typedef __bf16 type, out;
  typedef bf16x8 frag;                 // A or B operand of one step
  static constexpr int kStep = 64;     // k of one step of the walk: 128 bytes
  static constexpr int kPlanes = 1;
};
struct F32 {
  typedef float type, out;
  typedef f32x4 frag;
  static constexpr int kStep = 32;
  static constexpr int kPlanes = 1;
};
// fp32 numbers as sums of three bf16 numbers, 24 bits, in three planes; a product is six of the bf16 instruction's, the
// smallest first.  The three left out are together up to 2^-24 of it.  The bf16 instruction does six products in
// 6 / 16 of the time that the fp32 one takes for one.
struct Parts {
  typedef __bf16 type;
  typedef float out;
  typedef bf16x8 frag;
  static constexpr int kStep = 64;
  static constexpr int kPlanes = 3;
};
template <typename E>
constexpr int kPairs = E::kPlanes == 3 ? 6 : 1;
constexpr uint32_t kPairA = 0x052, kPairB = 0x118;   // planes of the pairs, 2 bits each: 20 02 11 10 01 00

__device__ __forceinline__ f32x4 multiply(bf16x8 a, bf16x8 b, f32x4 c) { return mfma16(a, b, c); }
// (element j of both operands is k = 4 * g + j of the 16: which k a lane group holds is free as long as both agree)
__device__ __forceinline__ f32x4 multiply(f32x4 a, f32x4 b, f32x4 c) {
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
  return c;
}

struct Operand {
  const char* base;
  int64_t pitch;          // bytes between rows
  const int32_t* rows;    // row numbers, or null: rows in order (row operands only)
  int32_t n;              // rows there are; those after the last are read as the last
  int32_t cols;           // column operands: columns there are; those after the last are read as the first
  int64_t plane;          // bytes between planes
  bool twice;             // row operands: every 16 rows are there twice

  __device__ __forceinline__ int64_t row(int64_t r) const {
    if (r >= n) r = n - 1;
    return rows ? rows[r] : twice ? (r >> 4) * 32 + (r & 15) : r;
  }
};

// Starts the copy of 16 bytes per lane, base + offset (base uniform), to consecutive LDS (1 KB at lds_addr, uniform).  Inline
// assembly: for the builtin the compiler drains every load in flight before the next LDS read.  With the walk's position in
// the scalar base a copy takes no vector instruction.
__device__ __forceinline__ void copy16(uint32_t lds_addr, const char* base, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(offset), "s"(base), "s"(lds_addr) : "memory");
}

// A pointer that is the same in every lane, as a scalar.  (readfirstlane returns a signed int: widened through uint32_t.)
__device__ __forceinline__ const char* uniform(const char* p) {
  const uint64_t x = (uint64_t)(uintptr_t)p;
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(x >> 32));
  return (const char*)(uintptr_t)((uint64_t)hi << 32 | lo);
}

// 1024 times the wave's number, once and for all in a scalar register: worked out again before each copy it would hold up
// the wave, and with it the matrix instructions behind it.
__device__ __forceinline__ uint32_t wave_place() {
  uint32_t w = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) * 1024;
  asm volatile("" : "+s"(w));
  return w;
}

// A tile of a row operand: ROWS rows of 128 bytes.  A copy's lanes land in consecutive LDS, 8 rows per wave, so rows cannot be
// padded; instead a row's eight 16-byte pieces are exchanged by row (piece ^ (row / 2) % 8), which spreads the 16 rows
// that one pass of a 16-byte read touches over all 64 banks.
template <int ROWS, int WAVES>
struct RowTile {
  static constexpr int kCopies = ROWS / 8 / WAVES;
  static_assert(kCopies * 8 * WAVES == ROWS, "every wave copies the same number of row groups");
  const char* base;
  uint32_t off[kCopies];   // from the tile's first row (32 bits: the launchers see to it where rows are gathered)
  uint32_t wave;           // this wave's place in LDS

  __device__ __forceinline__ void init(const Operand& op, int64_t row0, int64_t k_bytes) {
    const int w = threadIdx.x >> 6, l = threadIdx.x & 63;
    const int64_t first = op.row(row0);
    base = uniform(op.base + first * op.pitch + k_bytes);
    wave = wave_place();
#pragma unroll
    for (int j = 0; j < kCopies; ++j) {
      const int r = 8 * (w + WAVES * j) + (l >> 3);
      off[j] = (uint32_t)((op.row(row0 + r) - first) * op.pitch) + (((l & 7) ^ ((r >> 1) & 7)) << 4);
    }
  }
  __device__ __forceinline__ void copy(int j, uint32_t lds) { copy16(lds + wave + WAVES * j * 1024, base, off[j]); }
  __device__ __forceinline__ void advance() { base += 128; }

  // Where a lane reads block `row0` (of 16 rows) of the tile: half kk (of two) of the step.  Lane (n, g) holds row n, piece
  // 4 kk + g; the next block is 2048 bytes on.
  __device__ __forceinline__ static uint32_t lane(int row0, int kk) {
    const int n = threadIdx.x & 15, g = (threadIdx.x >> 4) & 3;
    return (row0 + n) * 128 + (((4 * kk + g) ^ ((n >> 1) & 7)) << 4);
  }
};

// A tile of a column operand: 128 / sizeof(T) rows (k) of COLS columns.  Pieces are exchanged by row so that the four rows of
// one pass of a transposing read (bf16: also the next group's four) lie in different banks.
template <typename E, int COLS, int WAVES>
struct ColTile {
  static constexpr int kSize = sizeof(typename E::type);
  static constexpr int kRowBytes = COLS * kSize, kPieces = kRowBytes / 16, kRowsPerCopy = 64 / kPieces;
  static constexpr int kCopies = E::kStep / kRowsPerCopy / WAVES;
  static_assert(kCopies * kRowsPerCopy * WAVES == E::kStep, "every wave copies the same number of rows");
  const char* base;
  uint32_t off[kCopies], pitch, wave;
  int64_t left;            // rows from here on

  __device__ __forceinline__ static int swizzle(int k) {
    return kSize == 2 ? 2 * ((k & 3) + 4 * ((k >> 3) & 1)) : 4 * ((k >> 2) & 3);
  }
  __device__ __forceinline__ static int row_in_tile(int j) {
    return ((int)(threadIdx.x >> 6) + WAVES * j) * kRowsPerCopy + (int)(threadIdx.x & 63) / kPieces;
  }
  __device__ __forceinline__ void init(const Operand& op, int64_t col0, int64_t row0) {
    base = uniform(op.base + row0 * op.pitch);
    wave = wave_place();
    pitch = (uint32_t)op.pitch;
    left = op.n - row0;
#pragma unroll
    for (int j = 0; j < kCopies; ++j) {
      const int piece = ((int)(threadIdx.x & 63) % kPieces) ^ swizzle(row_in_tile(j));
      int64_t col = col0 + piece * (16 / kSize);
      if (col >= op.cols) col = 0;
      off[j] = (uint32_t)(col * kSize) + (uint32_t)row_in_tile(j) * pitch;
    }
  }
  __device__ __forceinline__ void copy(int j, uint32_t lds) {
    uint32_t o = off[j];
    if (left < E::kStep) {   // the walk's last step (uniform branch)
      const int r = row_in_tile(j);
      if (r >= left) o -= (uint32_t)(r - (int)left + 1) * pitch;
    }
    copy16(lds + wave + WAVES * j * 1024, base, o);
  }
  __device__ __forceinline__ void advance() {
    base += (int64_t)E::kStep * pitch;
    left -= E::kStep;
  }

  // Where a lane reads the block of 16 columns from col0, first half of the step; the other half is kStep / 2 rows on.
  __device__ __forceinline__ static uint32_t lane(int col0) {
    const int n = threadIdx.x & 15, g = (threadIdx.x >> 4) & 3;
    if constexpr (kSize == 2) {
      const int f = 2 * ((n >> 2) + 4 * (g & 1));
      return (8 * g + (n >> 2)) * kRowBytes + (((col0 / 8 + ((n & 3) >> 1)) ^ f) << 4) + 8 * (n & 1);
    } else {
      return 4 * g * kRowBytes + (((col0 / 4 + (n >> 2)) ^ (4 * g)) << 4) + 4 * (n & 3);
    }
  }
  __device__ __forceinline__ static typename E::frag read(const char* p) {
    if constexpr (kSize == 2) {
      union {
        struct { s16x4 a, b; } s;
        bf16x8 v;
      } u;
      u.s.a = lds_read_tr4((const uint16_t*)p);
      u.s.b = lds_read_tr4((const uint16_t*)(p + 4 * kRowBytes));
      return u.v;
    } else {
      f32x4 v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = *(const float*)(p + j * kRowBytes);
      return v;
    }
  }
};

// ---- the product of one tile ----------------------------------------------------------
// A block of WM x WN waves computes BM (m) x BN (n); a wave BM / WM x BN / WN.
template <int BM_, int BN_, int WM_, int WN_, int STAGES_>
struct Form {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, kStages = STAGES_;
  static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves;
  static constexpr int TM = BM / WM / 16, TN = BN / WN / 16;   // 16 x 16 blocks of a wave
  static constexpr int kStageBytes = (BM + BN) * 128;
  static constexpr int kLds = kStages * kStageBytes;
};

template <int N>
__device__ __forceinline__ void wait_copies() {   // until at most N of this wave's are in flight
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void block_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// The copies of one walk, and where a wave's lanes read their operands.
template <typename E, typename F, bool COL, bool BCOL>   // column operands: A, B
struct Walk {
  typedef RowTile<F::BM, F::kWaves> RowA;
  typedef ColTile<E, F::BM, F::kWaves> ColA;
  typedef RowTile<F::BN, F::kWaves> RowB;
  typedef ColTile<E, F::BN, F::kWaves> ColB;
  RowA ra;
  ColA ca;
  RowB rb;
  ColB cb;
  static constexpr int kA = COL ? ColA::kCopies : RowA::kCopies;
  static constexpr int kB = BCOL ? ColB::kCopies : RowB::kCopies, kCount = kA + kB;

  // planes: the walk goes over the same steps once for each pair
  const char *a0, *b0;
  int64_t a_plane, b_plane, a_left, b_left;
  int per_pair, a_in_pair, b_in_pair, a_pair, b_pair;

  __device__ __forceinline__ void init(const Operand& A, const Operand& B, int64_t m0, int64_t n0, int64_t step, int64_t steps) {
    if constexpr (COL) ca.init(A, m0, step * E::kStep);
    else ra.init(A, m0, step * 128);
    if constexpr (BCOL) cb.init(B, n0, step * E::kStep);
    else rb.init(B, n0, step * 128);
    if constexpr (E::kPlanes > 1) {
      a0 = COL ? ca.base : ra.base;
      b0 = BCOL ? cb.base : rb.base;
      a_plane = A.plane;
      b_plane = B.plane;
      a_left = COL ? ca.left : 0;
      b_left = BCOL ? cb.left : 0;
      per_pair = (int)steps;
      a_pair = b_pair = 0;
      begin_pair_a();
      begin_pair_b();
    }
  }
  __device__ __forceinline__ void begin_pair_a() {
    const char* const a = a0 + (int64_t)((kPairA >> 2 * a_pair++) & 3) * a_plane;
    if constexpr (COL) {
      ca.base = a;
      ca.left = a_left;
    } else {
      ra.base = a;
    }
    a_in_pair = per_pair;
  }
  __device__ __forceinline__ void begin_pair_b() {
    const char* const b = b0 + (int64_t)((kPairB >> 2 * b_pair++) & 3) * b_plane;
    if constexpr (BCOL) {
      cb.base = b;
      cb.left = b_left;
    } else {
      rb.base = b;
    }
    b_in_pair = per_pair;
  }
  // copy j of a step's kA (kB) to the stage at lds; steps in order, advance_a (advance_b) after a step's last
  __device__ __forceinline__ void copy_a(int j, uint32_t lds) {
    if constexpr (COL) ca.copy(j, lds);
    else ra.copy(j, lds);
    if (j == kA - 1) {
      if constexpr (COL) ca.advance();
      else ra.advance();
      if constexpr (E::kPlanes > 1)
        if (--a_in_pair == 0) begin_pair_a();
    }
  }
  __device__ __forceinline__ void copy_b(int j, uint32_t lds) {
    if constexpr (BCOL) cb.copy(j, lds + F::BM * 128);
    else rb.copy(j, lds + F::BM * 128);
    if (j == kB - 1) {
      if constexpr (BCOL) cb.advance();
      else rb.advance();
      if constexpr (E::kPlanes > 1)
        if (--b_in_pair == 0) begin_pair_b();
    }
  }
  __device__ __forceinline__ void copy_step(uint32_t lds) {
#pragma unroll
    for (int j = 0; j < kA; ++j) copy_a(j, lds);
#pragma unroll
    for (int j = 0; j < kB; ++j) copy_b(j, lds);
  }

  static constexpr int kABases = COL ? F::TM : 2, kBBases = BCOL ? F::TN : 2;
  struct Lanes {           // offsets into LDS
    uint32_t a[kABases], b[kBBases];
    __device__ __forceinline__ void init(uint32_t stage, int wm, int wn) {
      const int m = wm * (F::BM / F::WM), n = wn * (F::BN / F::WN);
#pragma unroll
      for (int i = 0; i < kABases; ++i) a[i] = stage + (COL ? ColA::lane(m + 16 * i) : RowA::lane(m, i));
#pragma unroll
      for (int j = 0; j < kBBases; ++j) b[j] = stage + F::BM * 128 + (BCOL ? ColB::lane(n + 16 * j) : RowB::lane(n, j));
    }
    __device__ __forceinline__ void other_stage() {   // of two
      static_assert(F::kStages > 2 || (F::kStageBytes & (F::kStageBytes - 1)) == 0, "a bit of the offset");
#pragma unroll
      for (int i = 0; i < kABases; ++i) a[i] ^= F::kStageBytes;
#pragma unroll
      for (int j = 0; j < kBBases; ++j) b[j] ^= F::kStageBytes;
    }
    __device__ __forceinline__ typename E::frag read_a(const char* lds, int i, int kk) const {
      if constexpr (COL) return ColA::read(lds + a[i] + kk * (E::kStep / 2) * ColA::kRowBytes);
      else return *(const typename E::frag*)(lds + a[kk] + i * 2048);
    }
    __device__ __forceinline__ typename E::frag read_b(const char* lds, int j, int kk) const {
      if constexpr (BCOL) return ColB::read(lds + b[j] + kk * (E::kStep / 2) * ColB::kRowBytes);
      else return *(const typename E::frag*)(lds + b[kk] + j * 2048);
    }
  };
};

// acc[i][j] += the product over steps [step_begin, step_end) of the tile at (m0, n0)
template <typename E, typename F, bool COL, bool BCOL>
__device__ __forceinline__ void product(const Operand& A, const Operand& B, int64_t m0, int64_t n0, int64_t step_begin,
                                        int64_t step_end, char* lds, f32x4 (&acc)[F::TM][F::TN]) {
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = w % F::WM, wn = w / F::WM;
  const uint32_t lds_addr = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)lds;
  typedef Walk<E, F, COL, BCOL> W;
  W walk;
  walk.init(A, B, m0, n0, step_begin, step_end - step_begin);
  const int steps = (int)(step_end - step_begin) * kPairs<E>;
  if constexpr (F::kStages > 2) {
    // Bound by the copies: as many stages in flight as there are.
    constexpr int kAhead = F::kStages - 1;
#pragma unroll
    for (int s = 0; s < kAhead; ++s)
      if (s < steps) walk.copy_step(lds_addr + s * F::kStageBytes);
    int stage = 0;
    for (int step = 0; step < steps; ++step) {
      // this step's copies are in (those started after it may not be), and every wave has left the stage they go to next: its
      // reads of it have ended (as the compiler places the products they have anyway; here it does not rest on that)
      if (step + kAhead - 1 < steps) wait_copies<(kAhead - 1) * W::kCount>();
      else wait_copies<0>();
      __builtin_amdgcn_s_waitcnt(0xC07F);
      block_barrier();
      if (step + kAhead < steps) walk.copy_step(lds_addr + (stage == 0 ? F::kStages - 1 : stage - 1) * F::kStageBytes);
      typename W::Lanes at;
      at.init(stage * F::kStageBytes, wm, wn);
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        typename E::frag fb[F::TN], fa[F::TM];
#pragma unroll
        for (int j = 0; j < F::TN; ++j) fb[j] = at.read_b(lds, j, kk);
#pragma unroll
        for (int i = 0; i < F::TM; ++i) fa[i] = at.read_a(lds, i, kk);
#pragma unroll
        for (int i = 0; i < F::TM; ++i)
#pragma unroll
          for (int j = 0; j < F::TN; ++j) acc[i][j] = multiply(fa[i], fb[j], acc[i][j]);
      }
      stage = stage + 1 == F::kStages ? 0 : stage + 1;
    }
  } else {
    // Bound by the products.  A step is a chain of groups (half kk, block row i) of TN products each, whose A operand was
    // read three groups before; the B operands are read in the first groups, so that B's half of the stage is free
    // (kFreeB) long before the step ends.  The wave goes over to the next stage two groups before the end, when the last
    // operands of this one are in registers: barriers and reads lie under products.  The copies of the step after
    // the next go into what is free, one every few groups: eight at a time hold the wave up, since all waves of the CU
    // issue theirs at the same place.
    constexpr int G = 2 * F::TM, kSwitch = G - 2, kReadB = F::TM > 4 ? 4 : 2, kFreeB = F::TM > 4 ? 6 : 3;
    constexpr int kEachA = (G / 2 + W::kA - 1) / W::kA > 2 ? 2 : (G / 2 + W::kA - 1) / W::kA;   // groups between A's copies
    constexpr int kFirstA = 2 / kEachA;                                                        // of them before the step ends
    constexpr int kReads = COL && sizeof(typename E::type) == 2 ? 2 : 1;   // LDS reads of an A operand, at least
    static_assert(G % 4 == 0 && G >= 8, "a ring of four A operands");
    static_assert(kFirstA < W::kA && (W::kA - kFirstA - 1) * kEachA < kFreeB, "A's copies come before B's");
    typename E::frag fa[4], fb[2][F::TN];
    typename W::Lanes at;
    at.init(0, wm, wn);
    walk.copy_step(lds_addr);
    if (steps > 1) {
#pragma unroll
      for (int j = 0; j < W::kB; ++j) walk.copy_b(j, lds_addr + F::kStageBytes);
#pragma unroll
      for (int j = 0; j < kFirstA; ++j) walk.copy_a(j, lds_addr + F::kStageBytes);
      wait_copies<W::kB + kFirstA>();
    } else {
      wait_copies<0>();
    }
    block_barrier();
#pragma unroll
    for (int j = 0; j < F::TN; ++j) fb[0][j] = at.read_b(lds, j, 0);
#pragma unroll
    for (int t = 0; t < 3; ++t) fa[t] = at.read_a(lds, t, 0);
    uint32_t stage = lds_addr;   // the stage that is read
    // kLast: one of the last two steps, which have fewer copies to start (tests and branches cost as much as the copies)
    const auto one_step = [&](auto kLast, int left) {
      const bool two_more = !decltype(kLast)::value || left > 2, one_more = !decltype(kLast)::value || left > 1;
#pragma unroll
      for (int t = 0; t < G; ++t) {
        const auto products = [&] {
#pragma unroll
          for (int j = 0; j < F::TN; ++j)
            acc[t % F::TM][j] = multiply(fa[t & 3], fb[t / F::TM][j], acc[t % F::TM][j]);
        };
        if (t == 0) {   // (first, since the compiler waits here for every read that is on its way)
          products();
          __builtin_amdgcn_sched_barrier(0);
        }
        if (t + 3 < G) fa[(t + 3) & 3] = at.read_a(lds, (t + 3) % F::TM, (t + 3) / F::TM);
#pragma unroll
        for (int j = 0; j < F::TN; ++j)
          if (t == j * kReadB / F::TN) fb[1][j] = at.read_b(lds, j, 1);
        // A's copies of the next step, the rest
#pragma unroll
        for (int j = kFirstA; j < W::kA; ++j)
          if (t == (j - kFirstA) * kEachA && one_more) walk.copy_a(j, lds_addr + ((stage - lds_addr) ^ F::kStageBytes));
        if (t == kFreeB) {   // (the operands of A read since may be on their way)
          __builtin_amdgcn_s_waitcnt(0xC07F | (kReads * (kFreeB - kReadB) << 8));
          block_barrier();
        }
        // B's of the step after the next
#pragma unroll
        for (int j = 0; j < W::kB; ++j)
          if (t == kFreeB + j * (kSwitch - kFreeB) / W::kB && two_more) walk.copy_b(j, stage);
        if (t == kSwitch) {
          // the next stage's copies are in (those of B after them need not be), this stage's operands too
          if (two_more) __builtin_amdgcn_s_waitcnt(0x0070 | (W::kB & 15) | ((W::kB >> 4) << 14));
          else __builtin_amdgcn_s_waitcnt(0x0070);
          block_barrier();
          at.other_stage();
        }
#pragma unroll
        for (int j = 0; j < kFirstA; ++j)
          if (t == kSwitch + j * kEachA && two_more) walk.copy_a(j, stage);
        // (after the last step: reads of no account)
#pragma unroll
        for (int j = 0; j < F::TN; ++j)
          if (t == kSwitch + j * 2 / F::TN) fb[0][j] = at.read_b(lds, j, 0);
        if (t == kSwitch) fa[0] = at.read_a(lds, 0, 0);
        if (t == kSwitch + 1) {
          fa[1] = at.read_a(lds, 1, 0);
          fa[2] = at.read_a(lds, 2, 0);
        }
        if (t > 0) products();
        __builtin_amdgcn_sched_barrier(0);
      }
      stage = lds_addr + ((stage - lds_addr) ^ F::kStageBytes);
    };
    int left = steps;
    for (; left > 2; --left) one_step(std::false_type(), left);
    for (; left > 0; --left) one_step(std::true_type(), left);
  }
  block_barrier();   // the stages may be used for something else
}

// Which tile a block works on.  Block b runs on XCD b % 8; each XCD gets a contiguous run of tiles, in which `across`
// n-tiles are taken side by side for every m-tile, so that the blocks that share an L2 also share operands.
// Four across: one is 5 % slower on 18.4K x 50021 x 2048, two 0 to 2 %, eight and sixteen 3 %.
// (In 32 bits: a 64-bit division takes a block the time of a step.)
__device__ __forceinline__ void tile_of_block(unsigned m_tiles, unsigned n_tiles, unsigned across, int* mt, int* nt) {
  const unsigned b = blockIdx.x, xcd = b & 7, q = gridDim.x >> 3, r = gridDim.x & 7;
  const unsigned t = xcd * q + (xcd < r ? xcd : r) + (b >> 3);
  const unsigned per = across * m_tiles, group = t / per, in = t - group * per;
  const unsigned left = n_tiles - group * across, wide = left < across ? left : across;
  *mt = (int)(in / wide);
  *nt = (int)(group * across + in % wide);
}

// ---- logits ---------------------------------------------------------------------------

// What a logit is kept in between the product and the exponential: fp32 mode natural units (z = scale * acc, one rounding);
// bf16 mode units of exp2 (acc * (scale * log2 e), which saves a multiplication per exponential; the factor's own rounding
// moves every logit by the same 2^-24 of itself, logp's two terms alike).
template <typename E>
struct Unit {
  static constexpr float kPerNat = 1.f, kNat = 1.f, kExp2 = kLog2e;   // units per nat, nats per unit, exp2 per unit
};
template <>
struct Unit<Bf16> {
  static constexpr float kPerNat = kLog2e, kNat = kLn2, kExp2 = 1.f;
};

struct LogitArgs {
  Operand w, h;              // w: from the first id of the block of the vocabulary on
  int v0, n_vocab;           // that id, ids in the block
  int n_rows, steps;
  int m_tiles, n_tiles, across;
  float scale;
  const int32_t *edge_ptr, *only, *edge_token, *edge_id;
  // forward
  float2* partial;           // [row][partial_pitch] (maximum, sum of exp(z - maximum)) of each m-tile
  int64_t partial_pitch;
  int first_tile;            // of this block of the vocabulary
  float* logp;               // z[id] of the scored tokens, for now
  // backward
  const float *coef, *lse;   // [rows padded] c, lse
  char* dz;                  // [rows][dz_pitch] elements; two parts: 16 rows of one, the same 16 of the other, and so on
  int64_t dz_pitch;
  int64_t dz_plane;          // Parts: bytes between planes
  int dz_parts;
  const int* gate;           // the launch is meant only if *gate == want (null: always)
  int want;
};

// The scored tokens after `row` whose ids lie in [lo, lo + count): calls f(edge, id - lo) for each.  `only`: the row's entry of
// that table, read before the product: almost every row comes before one token, whose id then decides without another read.
template <typename Fn>
__device__ __forceinline__ void edges_in(const LogitArgs& a, int row, int only, int lo, int count, Fn f) {
  if (only >= 0) {
    if ((unsigned)(only - lo) < (unsigned)count) f(a.edge_ptr[row], only - lo);
  } else if (only == -2) {
    int e = a.edge_ptr[row];
    const int end = a.edge_ptr[row + 1];
    int top = end;
    while (e < top) {   // first edge with id >= lo
      const int mid = (e + top) >> 1;
      if (a.edge_id[mid] < lo) e = mid + 1;
      else top = mid;
    }
    for (; e < end; ++e) {
      const int at = a.edge_id[e] - lo;
      if (at >= count) break;
      f(e, at);
    }
  }
}

// The logits of a tile, down to a maximum and a sum of exp per row, and those of scored ids: bound by the matrix instructions.
// A step of a 256 x 256 tile copies 64 KB for 8.4 MFLOP, which at full rate is 12 TB/s out of the L2s; 128 x 128 copies twice
// as much per product, but two such blocks are on a CU and one's epilogue lies under the other's products (step and block
// times: choose() below).
template <typename E, typename F>
__global__ void __launch_bounds__(F::kThreads)
logits_fwd_kernel(LogitArgs a) {
  if (a.gate && *a.gate != a.want) return;
  __shared__ __attribute__((aligned(1024))) char lds[F::kLds];
  int mt, nt;
  tile_of_block(a.m_tiles, a.n_tiles, a.across, &mt, &nt);
  const int m0 = mt * F::BM, n0 = nt * F::BN;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = w % F::WM, wn = w / F::WM;
  const int n = threadIdx.x & 15, g = (threadIdx.x >> 4) & 3;
  const int wave_m = m0 + wm * (F::BM / F::WM), wave_n = n0 + wn * (F::BN / F::WN);
  int only[F::TN];
#pragma unroll
  for (int j = 0; j < F::TN; ++j) only[j] = wave_n + 16 * j + n < a.n_rows ? a.only[wave_n + 16 * j + n] : -1;
  f32x4 acc[F::TM][F::TN] = {};
  product<E, F, false, false>(a.w, a.h, m0, n0, 0, a.steps, lds, acc);

  float2* const joint = (float2*)lds;   // [WM][BN]
  constexpr float kExp2 = Unit<E>::kExp2;
  const float to_unit = a.scale * Unit<E>::kPerNat;
  const bool padded = wave_m + F::BM / F::WM > a.n_vocab;
#pragma unroll
  for (int j = 0; j < F::TN; ++j) {
    const int row = wave_n + 16 * j + n;
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < F::TM; ++i)
#pragma unroll
      for (int v = 0; v < 4; ++v) acc[i][j][v] *= to_unit;
    if (padded)
#pragma unroll
      for (int i = 0; i < F::TM; ++i)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          if (wave_m + 16 * i + 4 * g + v >= a.n_vocab) acc[i][j][v] = -INFINITY;
#pragma unroll
    for (int i = 0; i < F::TM; ++i)
#pragma unroll
      for (int v = 0; v < 4; ++v) top = fmaxf(top, acc[i][j][v]);
    edges_in(a, row, only[j], a.v0 + wave_m, F::BM / F::WM, [&](int e, int at) {
      if (((at >> 2) & 3) != g) return;
      float z = 0.f;
#pragma unroll
      for (int i = 0; i < F::TM; ++i)
#pragma unroll
        for (int v = 0; v < 4; ++v) z = at == 16 * i + 4 * g + v ? acc[i][j][v] : z;
      a.logp[a.edge_token[e]] = z * Unit<E>::kNat;
    });
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    float sum = 0.f;
    if (__builtin_amdgcn_ballot_w64(!(fabsf(top) < INFINITY))) {
      // an infinite maximum: equal infinities count as exp 0, not exp NaN (added in the order of the other branch, so that the
      // wave's other rows come out as without it)
#pragma unroll
      for (int i = 0; i < F::TM; ++i) {
        float e[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) e[v] = __builtin_amdgcn_exp2f((acc[i][j][v] == top ? 0.f : acc[i][j][v] - top) * kExp2);
        sum += (e[0] + e[1]) + (e[2] + e[3]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < F::TM; ++i) {   // (four exponentials, then their sum: an addition right behind its exponential waits)
        float e[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) e[v] = __builtin_amdgcn_exp2f((acc[i][j][v] - top) * kExp2);
        sum += (e[0] + e[1]) + (e[2] + e[3]);
      }
    }
    if (wave_m >= a.n_vocab) sum = 0.f;   // nothing but padding
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (g == 0) joint[wm * F::BN + wn * (F::BN / F::WN) + 16 * j + n] = make_float2(top, sum);
  }
  __syncthreads();
  for (int r = threadIdx.x; r < F::BN; r += F::kThreads) {
    if (n0 + r >= a.n_rows) continue;
    float top = joint[r].x, sum = 0.f;
#pragma unroll
    for (int q = 1; q < F::WM; ++q) top = fmaxf(top, joint[q * F::BN + r].x);
#pragma unroll
    for (int q = 0; q < F::WM; ++q) {
      const float2 p = joint[q * F::BN + r];
      sum += p.y * __builtin_amdgcn_exp2f((p.x == top ? 0.f : p.x - top) * kExp2);
    }
    a.partial[(int64_t)(n0 + r) * a.partial_pitch + a.first_tile + mt] = make_float2(top, sum);
  }
}

// lse of every row from its tiles' maxima and sums, one wave per row of the tree; then the scored tokens after it.  Bound by
// latency with few rows (5 us), by reading them with many (18.4K rows of 196 tiles: 18 us).
__global__ void __launch_bounds__(256)
lse_kernel(const float2* __restrict__ partial, int64_t pitch, int tiles, TokenTables tab, int64_t n_tokens,
           float* __restrict__ logp, float* __restrict__ lse, float nat, float exp2_unit, const int* gate, int want) {
  if (gate && *gate != want) return;
  const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int l = threadIdx.x & 63;
  if (t >= n_tokens) return;
  if (l == 0 && tab.before[t] < 0) logp[t] = 0.f;
  const int r = tab.slot[t];
  if (r < 0) {
    if (l == 0) lse[t] = 0.f;
    return;
  }
  const float2* p = partial + (int64_t)r * pitch;
  // (each lane keeps a running maximum, then the lanes' are joined; equal infinities: exp 0, not exp NaN)
  float top = -INFINITY, sum = 0.f;
  const auto join = [&](float other, float its) {
    const float both = fmaxf(top, other);
    sum = sum * __builtin_amdgcn_exp2f((top == both ? 0.f : top - both) * exp2_unit) +
          its * __builtin_amdgcn_exp2f((other == both ? 0.f : other - both) * exp2_unit);
    top = both;
  };
#pragma unroll 4
  for (int i = l; i < tiles; i += 64) join(p[i].x, p[i].y);
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) join(__shfl_xor(top, s), __shfl_xor(sum, s));
  const float of_row = top * nat + logf(sum);
  if (l == 0) lse[t] = of_row;
  for (int e = tab.edge_ptr[r] + l; e < tab.edge_ptr[r + 1]; e += 64) logp[tab.edge_token[e]] -= of_row;
}

// ---- gradient -------------------------------------------------------------------------

// The rows before scored tokens, gathered (zeros up to the padding), with their lse and c; where dz has two parts every 16 rows
// are there twice, as dz has them.  Bound by memory: 18.4K rows of width 4096 47 us, 6.4 TB/s.
template <typename T>
__global__ void __launch_bounds__(256)
gather_kernel(const T* __restrict__ hidden, T* __restrict__ rows, int pieces, int n_rows, int k_rows, int parts, TokenTables tab,
              const float* __restrict__ lse, const float* __restrict__ d_logp, float* __restrict__ lse_rows,
              float* __restrict__ coef, const int* gate, int want) {
  if (gate && *gate != want) return;
  for (int b = blockIdx.x; b < k_rows; b += gridDim.x) {
    const int r = parts == 1 ? b : (b >> 5) * 16 + (b & 15);
    const bool there = r < n_rows;
    const int64_t t = there ? tab.row[r] : 0;
    const float4* src = (const float4*)hidden + t * pieces;
    float4* dst = (float4*)rows + (int64_t)b * pieces;
    for (int i = threadIdx.x; i < pieces; i += 256) dst[i] = there ? src[i] : make_float4(0.f, 0.f, 0.f, 0.f);
    if (lse_rows && (parts == 1 || !(b & 16)) && threadIdx.x < 64) {
      float c = 0.f;
      if (there)
        for (int e = tab.edge_ptr[r] + (int)threadIdx.x; e < tab.edge_ptr[r + 1]; e += 64) c += d_logp[tab.edge_token[e]];
#pragma unroll
      for (int s = 1; s < 64; s <<= 1) c += __shfl_xor(c, s);
      if (threadIdx.x == 0) {
        coef[r] = c;
        lse_rows[r] = there ? lse[t] : 0.f;
      }
    }
  }
}

// fp32 rows as planes: src rows [0, n_rows) (of `row`, if given) to out [plane][out_rows][width], zeros after the last; for the
// gradient's hidden states also lse and c, as above.  *big becomes 1 where a number is 2^40 or more in magnitude, infinite
// or NaN (products of its planes would overflow, with either sign): the fp32 instruction then does the call.
// Bound by memory: 36.6K rows of width 1024 in two launches 61 us for 375 MB.
__global__ void __launch_bounds__(256)
split_kernel(const float* __restrict__ src, const int32_t* __restrict__ row, int n_rows, int out_rows, char* __restrict__ out, int64_t plane,
             int width, int* __restrict__ big, TokenTables tab, const float* __restrict__ lse, const float* __restrict__ d_logp,
             float scale, float* __restrict__ lse_rows, float* __restrict__ coef) {
  bool beyond = false;
  for (int64_t r = blockIdx.x; r < out_rows; r += gridDim.x) {
    const bool there = r < n_rows;
    const int64_t t = there ? (row ? row[r] : r) : 0;
    for (int i = threadIdx.x * 4; i < width; i += 1024) {
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
      if (there) x = *(const f32x4*)(src + t * width + i);
#pragma unroll
      for (int v = 0; v < 4; ++v) beyond |= !(fabsf(x[v]) < 0x1p40f);
      if (out)
#pragma unroll
        for (int q = 0; q < 3; ++q) {
          bf16x4 b;
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            b[v] = (__bf16)x[v];
            x[v] -= (float)b[v];
          }
          *(bf16x4*)(out + q * plane + (r * width + i) * 2) = b;
        }
    }
    if (coef && threadIdx.x < 64) {
      float c = 0.f;
      if (there)
        for (int e = tab.edge_ptr[r] + (int)threadIdx.x; e < tab.edge_ptr[r + 1]; e += 64) {
          c += d_logp[tab.edge_token[e]];
          beyond |= !(fabsf(d_logp[tab.edge_token[e]] * scale) < 0x1p40f);
        }
#pragma unroll
      for (int s = 1; s < 64; s <<= 1) c += __shfl_xor(c, s);
      beyond |= !(fabsf(c * scale) < 0x1p40f);
      if (threadIdx.x == 0) {
        coef[r] = c;
        lse_rows[r] = there ? lse[t] : 0.f;
      }
    }
  }
  if (beyond) *big = 1;
}

__global__ void clear_kernel(int* p) { *p = 0; }

// 4 consecutive values as T, or what rounding left of them (part 1)
__device__ __forceinline__ void put4(char* p, const f32x4& x, __bf16) {
  bf16x4 r;
#pragma unroll
  for (int v = 0; v < 4; ++v) r[v] = (__bf16)x[v];
  *(bf16x4*)p = r;
}
__device__ __forceinline__ void put4(char* p, const f32x4& x, float) { *(f32x4*)p = x; }

template <typename E, typename F>
struct DzTile {   // dz of a tile in LDS, [BN rows][BM ids], rows padded against bank conflicts
  typedef typename E::type T;
  static constexpr int kPitch = F::BM + 16 / (int)sizeof(T);
  static constexpr int kBytes = F::BN * kPitch * (int)sizeof(T);
};

// dz of a tile: the logits again, their exponentials, d_logp at the ids.  Through LDS on its way out, so that stores are whole
// rows of the tile; d_logp is added there, where a lane finds the element of an id.  Bound by the matrix instructions; a tile's
// epilogue takes about 9 us of the 100 that a tile of width 4096 does.
template <typename E, typename F>
__global__ void __launch_bounds__(F::kThreads)
logits_bwd_kernel(LogitArgs a, const float* __restrict__ d_logp) {
  if (a.gate && *a.gate != a.want) return;
  typedef typename E::type T;
  typedef DzTile<E, F> D;
  __shared__ __attribute__((aligned(1024))) char lds[F::kLds > D::kBytes ? F::kLds : D::kBytes];
  int mt, nt;
  tile_of_block(a.m_tiles, a.n_tiles, a.across, &mt, &nt);
  const int m0 = mt * F::BM, n0 = nt * F::BN;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = w % F::WM, wn = w / F::WM;
  const int n = threadIdx.x & 15, g = (threadIdx.x >> 4) & 3;
  const int wave_m = m0 + wm * (F::BM / F::WM), wave_n = n0 + wn * (F::BN / F::WN);
  int only[F::TN];
  float coef[F::TN], lse[F::TN];
#pragma unroll
  for (int j = 0; j < F::TN; ++j) {
    const int row = wave_n + 16 * j + n;
    const bool there = row < a.n_rows;
    only[j] = there ? a.only[row] : -1;
    coef[j] = there ? -a.coef[row] * a.scale : 0.f;
    lse[j] = there ? a.lse[row] * Unit<E>::kPerNat : 0.f;
  }
  f32x4 acc[F::TM][F::TN] = {};
  if (n0 < a.n_rows) product<E, F, false, false>(a.w, a.h, m0, n0, 0, a.steps, lds, acc);   // (else zeros to be written)

  const float to_unit = a.scale * Unit<E>::kPerNat;
  const bool padded = wave_m + F::BM / F::WM > a.n_vocab || wave_n + F::BN / F::WN > a.n_rows;
#pragma unroll
  for (int j = 0; j < F::TN; ++j) {
    const int row = wave_n + 16 * j + n;
    const bool there = row < a.n_rows;
    const float c = coef[j], l = lse[j];
#pragma unroll
    for (int i = 0; i < F::TM; ++i)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        // (fp32: the product's rounding is that of the forward pass)
        const float x = sizeof(typename E::out) == 2 ? fmaf(acc[i][j][v], to_unit, -l) : acc[i][j][v] * to_unit - l;
        acc[i][j][v] = c * __builtin_amdgcn_exp2f(x * Unit<E>::kExp2);
      }
    if (padded)
#pragma unroll
      for (int i = 0; i < F::TM; ++i)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          if (!(there && wave_m + 16 * i + 4 * g + v < a.n_vocab)) acc[i][j][v] = 0.f;
    edges_in(a, row, only[j], a.v0 + wave_m, F::BM / F::WM, [&](int e, int at) {
      if (((at >> 2) & 3) != g) return;
      const float d = d_logp[a.edge_token[e]] * a.scale;
#pragma unroll
      for (int i = 0; i < F::TM; ++i)
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[i][j][v] += at == 16 * i + 4 * g + v ? d : 0.f;
    });
  }
  for (int part = 0; part < a.dz_parts; ++part) {
    if (part) __syncthreads();
    T* const tile = (T*)lds;
#pragma unroll
    for (int j = 0; j < F::TN; ++j)
#pragma unroll
      for (int i = 0; i < F::TM; ++i) {
        T* const at = tile + (wave_n - n0 + 16 * j + n) * D::kPitch + wave_m - m0 + 16 * i + 4 * g;
        put4((char*)at, acc[i][j], T());
        if (sizeof(T) == 2 && part + 1 < a.dz_parts)
#pragma unroll
          for (int v = 0; v < 4; ++v) acc[i][j][v] -= (float)(__bf16)acc[i][j][v];
      }
    __syncthreads();
    constexpr int kE = 16 / sizeof(T);   // elements of a 16-byte store
    char* const out = a.dz + (E::kPlanes == 3 ? part * a.dz_plane : 0);
    for (int q = threadIdx.x; q < F::BN * F::BM / kE; q += F::kThreads) {
      const int r = q / (F::BM / kE), c = q % (F::BM / kE) * kE;
      const int row = a.dz_parts == 1 || E::kPlanes == 3 ? n0 + r : ((n0 + r) >> 4) * 32 + part * 16 + (r & 15);
      *(float4*)(out + ((int64_t)row * a.dz_pitch + m0 + c) * sizeof(T)) = *(const float4*)(tile + r * D::kPitch + c);
    }
  }
}

// 16 rows of a wave's results as bf16 through LDS of its own (pieces of 16 bytes exchanged by row, against bank conflicts): stores of
// whole 128 bytes, and no wave waits for another.
template <typename F>
struct Staging16 {
  static_assert(F::TM == 4, "64 columns");
  static constexpr int kPitch = 128, kWave = 16 * kPitch, kStores = 2;
  // blocks acc[.][j] to out[row ..][m ..]; `whole`: all of it is there
  __device__ __forceinline__ static void store(char* own, const f32x4 (&acc)[F::TM][F::TN], int j, char* out, int64_t pitch,
                                               int64_t row, int64_t rows, int64_t m, int64_t cols, bool whole) {
    const int l = threadIdx.x & 63, n = l & 15, g = l >> 4;
#pragma unroll
    for (int i = 0; i < F::TM; ++i) put4(own + n * kPitch + (((2 * i + (g >> 1)) ^ (n & 7)) << 4) + 8 * (g & 1), acc[i][j], __bf16());
    asm volatile("" ::: "memory");   // (one wave's LDS operations are done in order)
#pragma unroll
    for (int u = 0; u < kStores; ++u) {
      const int r = (l >> 3) + 8 * u, c = l & 7;
      const float4 x = *(const float4*)(own + r * kPitch + 16 * (c ^ (r & 7)));
      float4* const to = (float4*)(out + (row + r) * pitch + (m + 8 * c) * 2);
      if (whole) *to = x;
      else if (row + r < rows && m + 8 * c < cols) *to = x;
    }
    asm volatile("" ::: "memory");
  }
};

struct GradArgs {
  Operand a, b;
  const int* gate;         // as in LogitArgs
  int want;
  int n_parts;             // parts of dz along n, 16 rows of each in turn: their products are added at the end
  int steps;
  int splits;
  int m_tiles, n_tiles, across;
  int n_rows;              // rows of the result there are
  int width;               // m there are
  float* partial;          // [split][n][width] fp32: sums over a split's steps (`add`: added to what is there)
  int64_t partial_stride;  // elements between splits
  void* out;               // [n][width]; null: partial sums
  bool add;                // out is fp32 and added to
};

// C[n][m] of A^T B: dH, or dW (BCOL; rows of `out` in the order of n).  Bound by the matrix instructions, dH of few rows by W's way
// from memory (105 rows x 131072 x 2048: 173 us).  Where tiles alone would leave CUs idle the contraction is split, and sums
// of splits are added in order by the kernel below.
template <typename E, typename F, bool BCOL>
__global__ void __launch_bounds__(F::kThreads)
grad_kernel(GradArgs a) {
  if (a.gate && *a.gate != a.want) return;
  typedef typename E::out T;
  typedef DzTile<E, F> D;
  constexpr bool kThroughLds = sizeof(T) == 2;
  __shared__ __attribute__((aligned(1024))) char lds[kThroughLds && D::kBytes > F::kLds ? D::kBytes : F::kLds];
  int mt, nt;
  tile_of_block(a.m_tiles, a.n_tiles * a.splits, a.across, &mt, &nt);
  const int split = nt / a.n_tiles;
  nt -= split * a.n_tiles;
  const int m0 = mt * F::BM, n0 = nt * F::BN;
  const int each = a.steps / a.splits, more = a.steps % a.splits;   // steps of a split; the first `more` have one more
  const int s0 = split * each + min(split, more), s1 = s0 + each + (split < more);
  f32x4 acc[F::TM][F::TN] = {};
  if (s1 > s0) product<E, F, true, BCOL>(a.a, a.b, m0, n0, s0, s1, lds, acc);

  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = w % F::WM, wn = w / F::WM;
  const int n = threadIdx.x & 15, g = (threadIdx.x >> 4) & 3;
  const int wave_m = m0 + wm * (F::BM / F::WM), wave_n = n0 + wn * (F::BN / F::WN);
  if (kThroughLds && a.out && !a.add) {
    // 4 bf16 per lane and row would be stores of 32 bytes: whole rows of the tile instead, through LDS
    T* const tile = (T*)lds;
#pragma unroll
    for (int j = 0; j < F::TN; ++j)
#pragma unroll
      for (int i = 0; i < F::TM; ++i)
        put4((char*)(tile + (wave_n - n0 + 16 * j + n) * D::kPitch + wave_m - m0 + 16 * i + 4 * g), acc[i][j], T());
    __syncthreads();
    for (int q = threadIdx.x; q < F::BN * F::BM / 8; q += F::kThreads) {
      const int r = q / (F::BM / 8), c = q % (F::BM / 8) * 8;
      if (n0 + r < a.n_rows && m0 + c < a.width)
        *(float4*)((T*)a.out + (int64_t)(n0 + r) * a.width + m0 + c) = *(const float4*)(tile + r * D::kPitch + c);
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < F::TN; ++j) {
    int64_t row = wave_n + 16 * j + n;
    if (a.n_parts == 2) {
      if (j & 1) continue;
      row = (wave_n + 16 * j) / 2 + n;
    }
    if (row >= a.n_rows) continue;
#pragma unroll
    for (int i = 0; i < F::TM; ++i) {
      const int64_t m = wave_m + 16 * i + 4 * g;
      if (m >= a.width) continue;
      f32x4 x = acc[i][j];
      if (a.n_parts == 2 && j + 1 < F::TN) x += acc[i][j + 1];
      if (!a.out) {
        f32x4* const p = (f32x4*)(a.partial + split * a.partial_stride + row * a.width + m);
        if (a.add) x += *p;
        *p = x;
      } else if (a.add) {
        f32x4* const p = (f32x4*)((float*)a.out + row * a.width + m);
        *p += x;
      } else {
        put4((char*)a.out + (row * a.width + m) * sizeof(T), x, T());
      }
    }
  }
}

// dW of few rows (bf16, dz in two parts, ROWS = 64 or 128 rows padded): bound by storing it.  As tiles of a product a block would
// spend most of its time beginning and ending (256 x 256: 15 us, of which four steps); here a block keeps dz of its 128 ids
// in registers and walks over the width, 128 columns of H at a time in a ring of four buffers, so that copies, products
// and stores of different columns overlap.  Both parts meet the same rows of H: a matrix instruction's k is 16 rows of
// one part and the same 16 of the other, as dz has them, and its upper lanes read the lower ones' rows of H again.
// us, this and as tiles: 30 rows x 131072 ids x 2048 103 and 167 (the stores alone 104), 100 rows 164 to 182 and 228, 100 x 32000 x
// 4096 83 and 100, 128 x 50176 x 1024 48 and 48, 20 x 1000 x 64 4 and 7.  More than 64 rows: one block a CU (a ring of two
// buffers makes room for two, which then have 128 registers a lane and spill 33: 242).
struct OuterArgs {
  const char* rows;    // H, every 16 rows twice
  const char* dz;
  int64_t dz_pitch;    // bytes
  int n_ids, width;
  int m_blocks;        // blocks side by side along the width
  void* out;           // [id][width]
  bool add;            // fp32, added to
};

template <int ROWS>
__global__ void __launch_bounds__(512, ROWS == 64 ? 4 : 2)   // 64 rows: two blocks a CU, to the byte of its LDS
outer_kernel(OuterArgs a) {
  typedef Form<128, 128, 2, 4, 2> F;                 // a wave: 64 columns x 32 ids
  typedef Staging16<F> S;
  constexpr int kBuffer = ROWS * 256, kCopies = ROWS / 32, kStores = F::TN * S::kStores, kK = ROWS / 16;
  __shared__ __attribute__((aligned(1024))) char lds[4 * kBuffer];
  __shared__ __attribute__((aligned(16))) char staging[8 * S::kWave];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = w % F::WM, wn = w / F::WM;
  const int l = threadIdx.x & 63, n = l & 15, g = l >> 4;
  const int n0 = (int)blockIdx.x / a.m_blocks * 128, mb = (int)blockIdx.x % a.m_blocks;
  const int all = (a.width + 127) / 128, c0 = all * mb / a.m_blocks, c1 = all * (mb + 1) / a.m_blocks;
  const uint32_t lds_addr = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)lds;
  const uint32_t wave = wave_place();
  const int64_t pitch = (int64_t)a.width * 2;
  // a copy covers 4 rows of 256 bytes, pieces exchanged as in column operands
  uint32_t off[kCopies];
  int piece[kCopies];
#pragma unroll
  for (int j = 0; j < kCopies; ++j) {
    const int r = 4 * (w + 8 * j) + (l >> 4);
    piece[j] = (l & 15) ^ (2 * ((r & 3) + 4 * ((r >> 3) & 1)));
    off[j] = (uint32_t)(((r >> 4) * 32 + (r & 15)) * pitch) + piece[j] * 16;
  }
  const char* base = uniform(a.rows + (int64_t)c0 * 256);
  int copied = c0;   // chunks whose copies have been started
  const auto copy_chunk = [&] {
    const bool half = copied * 128 + 64 >= a.width;   // 64 columns left: those beyond are read again from these
#pragma unroll
    for (int j = 0; j < kCopies; ++j)
      copy16(lds_addr + (uint32_t)((copied - c0) & 3) * kBuffer + wave + 8 * j * 1024, base, off[j] - (half && piece[j] >= 8 ? 128 : 0));
    base += 256;
    ++copied;
  };
  if (c0 >= c1) return;
  // dz of the block's ids through the upper two buffers into registers, the first two chunks into the lower ones
#pragma unroll
  for (int j = 0; j < 2 * kCopies; ++j) {
    const int r = 4 * (w + 8 * j) + (l >> 4);
    copy16(lds_addr + 2 * kBuffer + wave + 8 * j * 1024, a.dz + (int64_t)n0 * 2,
           (uint32_t)(r * a.dz_pitch) + (((l & 15) ^ (2 * ((r & 3) + 4 * ((r >> 3) & 1)))) << 4));
  }
  copy_chunk();
  if (copied < c1) copy_chunk();
  wait_copies<0>();
  block_barrier();
  typedef ColTile<Bf16, 128, 8> Col;
  bf16x8 fb[kK][F::TN];
#pragma unroll
  for (int j = 0; j < F::TN; ++j) {
    const char* const at = lds + 2 * kBuffer + Col::lane(wn * 32 + 16 * j);
#pragma unroll
    for (int k = 0; k < kK; ++k) fb[k][j] = Col::read(at + k * 32 * 256);
  }
  uint32_t la[F::TM];
#pragma unroll
  for (int i = 0; i < F::TM; ++i) {
    const int f = 2 * ((n >> 2) + 4 * (g & 1)), col = wm * 64 + 16 * i;
    la[i] = (8 * (g & 1) + (n >> 2)) * 256 + (((col / 8 + ((n & 3) >> 1)) ^ f) << 4) + 8 * (n & 1);
  }
  __builtin_amdgcn_s_waitcnt(0xC07F);   // (dz is in registers before anything is copied over it)
  block_barrier();
  if (copied < c1) copy_chunk();
  if (copied < c1) copy_chunk();
  const bool whole = n0 + 128 <= a.n_ids && !a.add;
  for (int c = c0; c < c1; ++c) {
    // chunk c is in (the copies and stores after it need not have ended; where their number is not known, all are waited for)
    if (whole && c >= c0 + 4 && c + 3 < c1) wait_copies<2 * kCopies + 3 * kStores>();
    else if (c > c0) wait_copies<0>();
    block_barrier();
    if (c > c0 && copied < c1) copy_chunk();   // over chunk c - 1, which every wave has left
    f32x4 acc[F::TM][F::TN] = {};
    const char* const buffer = lds + ((c - c0) & 3) * kBuffer;
#pragma unroll
    for (int k = 0; k < kK; ++k) {
      bf16x8 fa[F::TM];
#pragma unroll
      for (int i = 0; i < F::TM; ++i) fa[i] = Col::read(buffer + la[i] + k * 16 * 256);
#pragma unroll
      for (int i = 0; i < F::TM; ++i)
#pragma unroll
        for (int j = 0; j < F::TN; ++j) acc[i][j] = mfma16(fa[i], fb[k][j], acc[i][j]);
    }
#pragma unroll
    for (int j = 0; j < F::TN; ++j) {
      const int64_t row = n0 + wn * 32 + 16 * j, m = c * 128 + wm * 64;
      if (!a.add) {
        S::store(staging + w * S::kWave, acc, j, (char*)a.out, pitch, row, a.n_ids, m, a.width, whole && (c + 1) * 128 <= a.width);
      } else if (row + n < a.n_ids && m < a.width) {
#pragma unroll
        for (int i = 0; i < F::TM; ++i) {
          f32x4* const p = (f32x4*)((float*)a.out + (row + n) * a.width + m + 16 * i + 4 * g);
          *p += acc[i][j];
        }
      }
    }
  }
}

// Adds the partial sums of the splits, in order, and puts them where they belong: rows of the tree by `slot` (rows without
// one: zeros), or rows in order (slot null).  Bound by memory: 18.4K rows of width 4096 in one part 125 us.
template <typename T>
__global__ void __launch_bounds__(256)
sum_kernel(const float* __restrict__ partial, int splits, int64_t stride, const int32_t* __restrict__ slot, int64_t n_rows,
           int quads, void* __restrict__ out, bool add, const int* gate, int want) {
  if (gate && *gate != want) return;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n_rows * quads) return;
  const int64_t t = i / quads;
  const int q = (int)(i - t * quads);
  const int64_t r = slot ? slot[t] : t;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  if (r >= 0) {
    const float* at = partial + (r * quads + q) * 4;
    int s = 0;
    for (; s + 8 <= splits; s += 8, at += 8 * stride) {   // eight reads in flight, added in order
      f32x4 y[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) y[u] = *(const f32x4*)(at + u * stride);
#pragma unroll
      for (int u = 0; u < 8; ++u) x += y[u];
    }
    for (; s < splits; ++s, at += stride) x += *(const f32x4*)at;
  }
  if (add) {
    f32x4* const p = (f32x4*)out + i;
    *p += x;
  } else {
    put4((char*)out + i * 4 * sizeof(T), x, T());
  }
}

// ---- launches -------------------------------------------------------------------------

typedef Form<128, 32, 4, 1, 3> Few;       // 4 waves, two blocks per CU; up to 64 rows: bound by the way of A into LDS
typedef Form<128, 64, 4, 1, 3> Thin;
typedef Form<256, 128, 4, 2, 3> Wide;     // 8 waves, one block per CU; up to 128 rows, like these
typedef Form<128, 128, 2, 2, 2> Medium;   // 4 waves, two blocks per CU: bound by the products
typedef Form<256, 256, 2, 4, 2> Large;    // 8 waves, one block per CU

inline size_t round256(size_t x) { return (x + 255) / 256 * 256; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

enum { kFew, kThin, kWide, kMedium, kLarge, kForms };
const int kTileM[kForms] = {Few::BM, Thin::BM, Wide::BM, Medium::BM, Large::BM}, kTileN[kForms] = {Few::BN, Thin::BN, Wide::BN, Medium::BN, Large::BN};
const int kSlots[kForms] = {512, 512, 256, 512, 256};   // blocks the chip holds

// Which form computes a product of n x m over `steps`, in how many splits of the steps: the least estimated time, of
//  - rounds of as many blocks as the chip holds, a block taking step_us for a step and block_us besides;
//  - A's way from memory, at the rate that a form with so many copies in flight reaches (blocks side by side share it, not
//    quite all);
//  - the partial sums of splits, written and read.
// The constants are measured on products that fill the chip.  Rows x ids x width in us, the form it takes and the next:
// logits 30 x 131072 x 2048 Few 108, Thin 112; 100 x 131072 x 2048 Thin 128, Wide 132, Medium 180; dH of 30 rows Thin 103,
// Few 135; of 100 Wide 155, Medium 179.
enum Kind { kBf16, kF32, kParts };
struct Choice {
  int form, splits;
  double time;
};
Choice choose(Kind kind, int64_t n, int64_t m, int64_t steps, bool may_split, int least = kFew) {
  static const double step_us[2][kForms] = {{0.6, 0.65, 0.96, 1.05, 1.42}, {1.1, 2.1, 4.2, 4.2, 0}};
  static const double block_us[kForms] = {4, 4, 6, 6, 9}, read_tb[kForms] = {4.9, 4.9, 4.4, 3.0, 2.4};
  const int64_t pairs = kind == kParts ? 6 : 1;
  Choice best{0, 1, 1e300};
  for (int f = least; f < kForms; ++f) {
    const double us = step_us[kind == kF32][f];
    if (us == 0) continue;
    const int64_t n_tiles = ceil_div(n, kTileN[f]), m_tiles = ceil_div(m, kTileM[f]);
    const double from_memory = (double)(steps * pairs) * 128 * (double)(m_tiles * kTileM[f]) * (1 + 0.1 * (double)std::min<int64_t>(n_tiles - 1, 8));
    for (int64_t s = 1; s <= (may_split ? 64 : 1) && (s == 1 || steps * pairs / s >= 4); ++s) {
      const double rounds = (double)ceil_div(n_tiles * m_tiles * s, kSlots[f]);
      const double time = std::max(rounds * ((double)(ceil_div(steps, s) * pairs) * us + block_us[f]), from_memory / (read_tb[f] * 1e6)) +
                          (s > 1 ? 8 + (double)s * (double)n * (double)m * 8 / 5e6 : 0);
      if (time < best.time) best = Choice{f, (int)s, time};
    }
  }
  return best;
}

// What a call's sizes decide, for one way of multiplying.
struct Plan {
  Kind kind;
  int64_t R, padded, V, D;   // rows, rows padded to kRowPad, vocabulary, width
  int64_t k_rows;            // rows as the contraction of dW sees them: padded to 64, once for each part of dz (bf16)
  int size;                  // of an element as it is multiplied
  int planes;
  bool pack;                 // the forward gathers its rows: they may lie further apart than a copy's 32-bit offsets reach
  int64_t block, blocks;     // ids of a block of the vocabulary, and how many blocks
  Choice z;                  // logits
  int64_t tiles;             // m-tiles of all blocks
  // backward
  int parts;                 // of dz along rows (bf16)
  Choice h, w;               // dH, and dW where dz is in one part
  // workspace
  size_t at_big, at_lse, at_coef, at_rows, at_planes_h, at_planes_w, at_partial, at_dz, at_h, at_w, bytes;
};

// The narrowest form that the logits of a forward call and dH take: numbers in parts are for calls of many rows, and of 9 10^7
// sizes of the one and 4 10^6 of the other none would take Few.  (The logits of a gradient do: 754 rows x 2529 x 5632 567 us,
// and 626 on the fp32 instruction, which is next.)
constexpr int least_form(int planes) { return planes == 3 ? kThin : kFew; }

// block: 0, or what the blocks of the vocabulary have to be
Plan plan_for(Kind kind, const dta_tokens* t, const dta_vocab_params_t* p, bool backward, int64_t block) {
  Plan s{};
  s.kind = kind;
  s.R = t->n_rows();
  s.padded = t->rows_padded();
  s.V = t->vocab;
  s.D = p->width;
  s.size = kind == kF32 ? 4 : 2;
  s.planes = kind == kParts ? 3 : 1;
  s.pack = !backward && kind != kParts && t->n_tokens * s.D * s.size > (int64_t)UINT32_MAX;
  s.parts = backward && kind == kBf16 && s.R <= 128 ? 2 : 1;
  s.k_rows = s.parts * ceil_div(s.R, 64) * 64;
  const int64_t groups = ceil_div(s.V, 256);   // of ids
  int64_t most = groups;
  // a launch has fewer than 2^32 threads, and the form with the smallest tiles 16 logits a thread
  most = std::min(most, std::max<int64_t>(1, ((int64_t)1 << 36) / s.padded / 256));
  // dz of a block takes up to 2 GiB, and so do the planes of its part of the matrix
  if (backward) most = std::min(most, std::max<int64_t>(1, ((int64_t)1 << 31) / (s.parts * s.padded * s.size * s.planes) / 256));
  if (kind == kParts) most = std::min(most, std::max<int64_t>(1, ((int64_t)1 << 31) / (6 * s.D) / 256));
  s.block = block ? block : ceil_div(groups, ceil_div(groups, most)) * 256;
  s.blocks = ceil_div(s.V, s.block);
  const int64_t width_steps = s.D * s.size / 128;
  const int64_t ids = s.blocks == 1 ? s.V : s.block;
  const int least = least_form(s.planes);
  s.z = choose(kind, backward ? ceil_div(s.R, 64) * 64 : s.R, ids, width_steps, false, backward ? kFew : least);   // (dz is padded to 64 rows)
  s.tiles = ceil_div(s.V, kTileM[s.z.form]);
  if (backward) {
    s.h = choose(kind, s.parts * s.R, s.D, ceil_div(ids * s.size, 128), true, least);
    if (s.parts == 1) s.w = choose(kind, ids, s.D, s.k_rows * s.size / 128, true, kind == kF32 ? kThin : kWide);   // (dz by columns: rows of 256 bytes and more)
  }
  return s;
}

// The way of multiplying a call's numbers (s), and for numbers in planes the way to be taken where some are too large (*f32).
Plan plan(const dta_tokens* t, const dta_vocab_params_t* p, bool backward, Plan* f32) {
  if (!t->n_rows()) return Plan{};
  Plan s = plan_for(p->dtype == DTA_BF16 ? kBf16 : kF32, t, p, backward, 0);
  bool two = false;
  if (s.kind == kF32) {
    // planes: made of all numbers (10 bytes each written and read), and a few more launches
    const Plan q = plan_for(kParts, t, p, backward, 0);
    const double made = (double)(s.V + s.R) * (double)s.D * 10 / 4.5e6 + (backward ? 40 : 25) + (q.blocks > 1 ? (double)s.V * (double)s.D * 4 / 4.5e6 : 0);
    const auto total = [](const Plan& x) { return (double)x.blocks * (x.z.time + x.h.time + x.w.time); };
    if (total(q) + made < total(s)) {
      *f32 = plan_for(kF32, t, p, backward, q.block);
      s = q;
      two = true;
    }
  }
  size_t at = 0;
  const auto take = [&](int64_t n) {
    const size_t begin = at;
    at += round256((size_t)n);
    return begin;
  };
  const auto larger = [&](int64_t mine, int64_t of_f32) { return two ? std::max(mine, of_f32) : mine; };
  const Plan& o = *f32;
  if (two) {
    s.at_big = take(4);
    s.at_planes_h = take(6 * s.k_rows * s.D);
    s.at_planes_w = take(6 * s.block * s.D);
  }
  if (!backward) {
    if (s.pack || o.pack) s.at_rows = take(s.k_rows * s.D * (int64_t)elem_size(*p));
    s.at_partial = take(larger(s.R * s.tiles, o.R * o.tiles) * (int64_t)sizeof(float2));
  } else {
    const int own = (int)elem_size(*p);
    s.at_lse = take(s.padded * 4);
    s.at_coef = take(s.padded * 4);
    s.at_rows = take(std::max(s.padded, s.k_rows) * s.D * own);
    s.at_dz = take(larger(s.planes * s.parts * s.padded * s.block * s.size, o.padded * o.block * 4));
    s.at_h = take(larger(s.h.splits, o.h.splits) * s.R * s.D * 4);
    const auto w_sums = [](const Plan& x) { return x.w.splits > 1 ? x.w.splits * x.block * x.D * 4 : (int64_t)0; };
    s.at_w = take(larger(w_sums(s), w_sums(o)));
  }
  s.bytes = at;
  if (two) {   // (the same workspace)
    Plan g = *f32;
    *f32 = s;
    f32->kind = kF32;
    f32->size = 4;
    f32->planes = 1;
    f32->pack = g.pack;
    f32->z = g.z;
    f32->h = g.h;
    f32->w = g.w;
    f32->tiles = g.tiles;
  }
  return s;
}

// Calls f(form) with the form's type, LEAST or a wider one.
template <typename E, int LEAST, typename Fn>
void with_form(int form, Fn f) {
  if constexpr (LEAST == kFew)
    if (form == kFew) f(Few());
  if (form == kThin) f(Thin());
  if (form == kWide) f(Wide());
  if (form == kMedium) f(Medium());
  if constexpr (sizeof(typename E::type) == 2)
    if (form == kLarge) f(Large());
}

// Whether a launch is meant, as the device finds out: *flag == want.
struct Gate {
  const int* flag = nullptr;
  int want = 0;
};

LogitArgs logit_args(const VocabArgs& a, const Plan& s, int64_t v0, int64_t n, const Gate& gate) {
  LogitArgs l{};
  l.w = Operand{(const char*)a.weight + v0 * s.D * s.size, s.D * s.size, nullptr, (int32_t)n, 0, 0, false};
  if (s.kind == kParts) l.w = Operand{a.workspace + s.at_planes_w, s.D * 2, nullptr, (int32_t)n, 0, s.block * s.D * 2, false};
  l.v0 = (int)v0;
  l.n_vocab = (int)n;
  l.n_rows = (int)s.R;
  l.steps = (int)(s.D * s.size / 128);
  l.m_tiles = (int)ceil_div(n, kTileM[s.z.form]);
  l.n_tiles = (int)ceil_div(s.R, kTileN[s.z.form]);
  l.across = 4;
  l.scale = a.p.scale;
  l.edge_ptr = a.tab.edge_ptr;
  l.only = a.tab.only;
  l.edge_token = a.tab.edge_token;
  l.edge_id = a.tab.edge_id;
  l.gate = gate.flag;
  l.want = gate.want;
  return l;
}

// Blocks of a launch that has one for every row, of 256 threads each: fewer than 2^32 threads, the rest in further rounds.
size_t row_blocks(int64_t rows) { return (size_t)std::min<int64_t>(rows, 1 << 23); }

// Planes of the hidden rows; where the vocabulary comes in blocks, a look over the whole matrix, so that all of them are
// multiplied the same way.
void split_rows(const VocabArgs& a, const Plan& s, bool backward) {
  int* const big = (int*)(a.workspace + s.at_big);
  float* const none = nullptr;
  launch(a, false, clear_kernel, 1, 1, big);
  launch(a, false, split_kernel, row_blocks(s.k_rows), 256, (const float*)a.hidden, a.tab.row, s.R, s.k_rows, a.workspace + s.at_planes_h,
         s.k_rows * s.D * 2, (int)s.D, big, a.tab, a.lse_in, a.d_logp, a.p.scale, backward ? (float*)(a.workspace + s.at_lse) : none,
         backward ? (float*)(a.workspace + s.at_coef) : none);
  if (s.blocks > 1)
    launch(a, false, split_kernel, row_blocks(s.V), 256, (const float*)a.weight, (const int32_t*)nullptr, s.V, s.V, (char*)nullptr, (int64_t)0,
           (int)s.D, big, a.tab, (const float*)nullptr, (const float*)nullptr, 0.f, none, none);
}
// Planes of a block of the matrix.
void split_matrix(const VocabArgs& a, const Plan& s, int64_t v0, int64_t n) {
  float* const none = nullptr;
  launch(a, false, split_kernel, row_blocks(n), 256, (const float*)a.weight + v0 * s.D, (const int32_t*)nullptr, n, n,
         a.workspace + s.at_planes_w, s.block * s.D * 2, (int)s.D, (int*)(a.workspace + s.at_big), a.tab, (const float*)nullptr,
         (const float*)nullptr, 0.f, none, none);
}

template <typename E>
void fwd_block(const VocabArgs& a, const Plan& s, int64_t b, const Gate& gate) {
  const int64_t v0 = b * s.block, n = std::min(s.block, s.V - v0);
  LogitArgs l = logit_args(a, s, v0, n, gate);
  l.h = Operand{(const char*)a.hidden, s.D * s.size, a.tab.row, (int32_t)s.R, 0, 0, false};
  if (s.pack) l.h = Operand{a.workspace + s.at_rows, s.D * s.size, nullptr, (int32_t)s.R, 0, 0, false};
  if (s.kind == kParts) l.h = Operand{a.workspace + s.at_planes_h, s.D * 2, nullptr, (int32_t)s.R, 0, s.k_rows * s.D * 2, false};
  l.partial = (float2*)(a.workspace + s.at_partial);
  l.partial_pitch = s.tiles;
  l.first_tile = (int)(v0 / kTileM[s.z.form]);
  l.logp = a.logp;
  with_form<E, least_form(E::kPlanes)>(s.z.form, [&](auto f) {
    typedef decltype(f) F;
    launch(a, false, logits_fwd_kernel<E, F>, (size_t)l.m_tiles * l.n_tiles, F::kThreads, l);
  });
}

template <typename E>
void lse_of_rows(const VocabArgs& a, const Plan& s, const Gate& gate, bool last) {
  launch(a, last, lse_kernel, (size_t)ceil_div(a.tokens->n_tokens, 4), 256, (const float2*)(a.workspace + s.at_partial), s.tiles,
         (int)s.tiles, a.tab, a.tokens->n_tokens, a.logp, a.lse, Unit<E>::kNat, Unit<E>::kExp2, gate.flag, gate.want);
}

// The rows themselves, gathered, for one-plane products; with lse and c (`sums`).
template <typename T>
void gather_rows(const VocabArgs& a, const Plan& s, const Gate& gate, bool sums) {
  launch(a, false, gather_kernel<T>, row_blocks(s.k_rows), 256, (const T*)a.hidden, (T*)(a.workspace + s.at_rows),
         (int)(s.D * sizeof(T) / 16), s.R, s.k_rows, s.parts, a.tab, a.lse_in, a.d_logp, sums ? (float*)(a.workspace + s.at_lse) : nullptr,
         (float*)(a.workspace + s.at_coef), gate.flag, gate.want);
}

int logprob_fwd(const VocabArgs& a) {
  Plan f32{};
  const Plan s = plan(a.tokens, &a.p, false, &f32);
  clear_hip_error();
  if (a.p.dtype == DTA_BF16) {
    if (s.pack) gather_rows<__bf16>(a, s, Gate(), false);
    for (int64_t b = 0; b < s.blocks; ++b) fwd_block<Bf16>(a, s, b, Gate());   // (none without rows)
    lse_of_rows<Bf16>(a, s, Gate(), true);
  } else if (s.kind != kParts) {
    if (s.pack) gather_rows<float>(a, s, Gate(), false);
    for (int64_t b = 0; b < s.blocks; ++b) fwd_block<F32>(a, s, b, Gate());
    lse_of_rows<F32>(a, s, Gate(), true);
  } else {
    const Gate parts{(const int*)(a.workspace + s.at_big), 0}, big{parts.flag, 1};
    split_rows(a, s, false);
    for (int64_t b = 0; b < s.blocks; ++b) {
      split_matrix(a, s, b * s.block, std::min(s.block, s.V - b * s.block));
      if (b == 0 && f32.pack) gather_rows<float>(a, f32, big, false);
      fwd_block<Parts>(a, s, b, parts);
      fwd_block<F32>(a, f32, b, big);
    }
    lse_of_rows<Parts>(a, s, parts, false);
    lse_of_rows<F32>(a, f32, big, true);
  }
  return launch_status("log-probabilities");
}

template <typename T>
void sum_rows(const VocabArgs& a, const float* partial, int splits, int64_t stride, const int32_t* slot, int64_t n, void* out,
              bool add, const Gate& gate, bool last) {
  const int quads = a.p.width / 4;
  launch(a, last, sum_kernel<T>, (size_t)ceil_div(n * quads, 256), 256, partial, splits, stride, slot, n, quads, out, add, gate.flag,
         gate.want);
}

template <typename E>
void bwd_block(const VocabArgs& a, const Plan& s, int64_t b, const Gate& gate, bool last_launch) {
  typedef typename E::out Out;
  const int64_t row_bytes = s.D * s.size, v0 = b * s.block, n = std::min(s.block, s.V - v0);
  const bool last_block = b + 1 == s.blocks, planes = s.kind == kParts;
  float *const h_sum = (float*)(a.workspace + s.at_h), *const w_sum = (float*)(a.workspace + s.at_w);
  char* const dz = a.workspace + s.at_dz;
  const char* const rows = a.workspace + (planes ? s.at_planes_h : s.at_rows);
  const int64_t rows_plane = s.k_rows * row_bytes, dz_plane = s.padded * s.block * s.size;

  LogitArgs l = logit_args(a, s, v0, n, gate);
  l.m_tiles = (int)(ceil_div(n, 256) * 256 / kTileM[s.z.form]);   // (dz is padded to 256 ids with zeros)
  l.h = Operand{rows, row_bytes, nullptr, (int32_t)s.R, 0, rows_plane, s.parts == 2};
  l.n_tiles = (int)ceil_div(s.k_rows / s.parts, kTileN[s.z.form]);   // (... and to 64 rows)
  l.coef = (const float*)(a.workspace + s.at_coef);
  l.lse = (const float*)(a.workspace + s.at_lse);
  l.dz = dz;
  l.dz_pitch = s.block;
  l.dz_plane = dz_plane;
  l.dz_parts = planes ? 3 : s.parts;
  with_form<E, kFew>(s.z.form, [&](auto f) {
    typedef decltype(f) F;
    launch(a, false, logits_bwd_kernel<E, F>, (size_t)l.m_tiles * l.n_tiles, F::kThreads, l, a.d_logp);
  });
  const auto run = [&](auto weight, GradArgs& g, const Choice& c, int64_t n_wide, bool last) {
    constexpr bool kWeight = decltype(weight)::value;
    g.splits = c.splits;
    g.m_tiles = (int)ceil_div(s.D, kTileM[c.form]);
    g.n_tiles = (int)ceil_div(n_wide, kTileN[c.form]);
    g.width = (int)s.D;
    g.across = 4;
    g.gate = gate.flag;
    g.want = gate.want;
    with_form<E, least_form(E::kPlanes)>(c.form, [&](auto f) {
      typedef decltype(f) F;
      if constexpr (!kWeight || F::BN * sizeof(typename E::type) >= 256)
        launch(a, last, grad_kernel<E, F, kWeight>, (size_t)g.m_tiles * g.n_tiles * g.splits, F::kThreads, g);
    });
  };
  if (a.d_hidden) {
    GradArgs g{};
    g.a = Operand{l.w.base, row_bytes, nullptr, (int32_t)n, (int32_t)s.D, l.w.plane, false};
    g.b = Operand{dz, s.block * s.size, nullptr, (int32_t)(s.parts * s.padded), 0, dz_plane, false};
    g.n_parts = s.parts;
    g.steps = (int)ceil_div(n * s.size, 128);
    g.n_rows = (int)s.R;
    g.partial = h_sum;
    g.partial_stride = s.R * s.D;
    g.add = b > 0;
    run(std::false_type(), g, s.h, s.parts * (s.parts == 1 ? s.R : ceil_div(s.R, 16) * 16), false);
    if (last_block)
      sum_rows<Out>(a, h_sum, s.h.splits, s.R * s.D, a.tab.slot, a.tokens->n_tokens, a.d_hidden, false, gate, last_launch && !a.d_weight);
  }
  if (a.d_weight && s.parts == 2) {
    // enough blocks for every CU, each with four chunks of columns at least
    const int64_t along = ceil_div(n, 128), chunks = ceil_div(s.D, 128);
    OuterArgs o{rows, dz, s.block * 2, (int)n, (int)s.D, 1, (char*)a.d_weight + v0 * s.D * (a.add ? 4 : 2), a.add};
    o.m_blocks = (int)std::max<int64_t>(1, std::min(ceil_div(2 * kNumCUs, along), chunks / 4));
    const size_t grid = (size_t)(along * o.m_blocks);
    if (s.k_rows == 128) launch(a, last_launch, outer_kernel<64>, grid, 512, o);
    else launch(a, last_launch, outer_kernel<128>, grid, 512, o);
  } else if (a.d_weight) {
    GradArgs g{};
    g.a = Operand{rows, row_bytes, nullptr, (int32_t)s.k_rows, (int32_t)s.D, rows_plane, false};
    g.b = Operand{dz, s.block * s.size, nullptr, (int32_t)s.k_rows, (int32_t)s.block, dz_plane, false};
    g.n_parts = 1;
    g.steps = (int)(s.k_rows * s.size / 128);
    g.n_rows = (int)n;
    char* const out = (char*)a.d_weight + v0 * s.D * (a.add ? 4 : (int)sizeof(Out));
    if (s.w.splits == 1) {
      g.out = out;
      g.add = a.add;
      run(std::true_type(), g, s.w, n, last_launch);
    } else {
      g.partial = w_sum;
      g.partial_stride = s.block * s.D;
      run(std::true_type(), g, s.w, n, false);
      sum_rows<Out>(a, w_sum, s.w.splits, s.block * s.D, nullptr, n, out, a.add, gate, last_launch);
    }
  }
}

int logprob_bwd(const VocabArgs& a) {
  const char* const what = "gradient of log-probabilities";
  clear_hip_error();
  if (!a.tokens->n_rows()) {   // no row before a scored token: zeros
    const bool weight = a.d_weight && !a.add;
    const auto zero = [&](void* out, int64_t rows, bool last) {
      if (a.p.dtype == DTA_BF16) sum_rows<__bf16>(a, nullptr, 0, 0, nullptr, rows, out, false, Gate(), last);
      else sum_rows<float>(a, nullptr, 0, 0, nullptr, rows, out, false, Gate(), last);
    };
    if (a.d_hidden) zero(a.d_hidden, a.tokens->n_tokens, !weight);
    if (weight) zero(a.d_weight, a.tokens->vocab, true);
    return launch_status(what);
  }
  Plan f32{};
  const Plan s = plan(a.tokens, &a.p, true, &f32);
  if (s.kind == kBf16) {
    gather_rows<__bf16>(a, s, Gate(), true);
    for (int64_t b = 0; b < s.blocks; ++b) bwd_block<Bf16>(a, s, b, Gate(), b + 1 == s.blocks);
  } else if (s.kind == kF32) {
    gather_rows<float>(a, s, Gate(), true);
    for (int64_t b = 0; b < s.blocks; ++b) bwd_block<F32>(a, s, b, Gate(), b + 1 == s.blocks);
  } else {
    const Gate parts{(const int*)(a.workspace + s.at_big), 0}, big{parts.flag, 1};
    split_rows(a, s, true);
    for (int64_t b = 0; b < s.blocks; ++b) {
      split_matrix(a, s, b * s.block, std::min(s.block, s.V - b * s.block));
      if (b == 0) gather_rows<float>(a, f32, big, false);
      bwd_block<Parts>(a, s, b, parts, false);
      bwd_block<F32>(a, f32, b, big, b + 1 == s.blocks);
    }
  }
  return launch_status(what);
}

size_t workspace(const dta_tokens* t, const dta_vocab_params_t* p, bool backward) {
  Plan f32{};
  return plan(t, p, backward, &f32).bytes;
}

}  // namespace

size_t logprob_fwd_workspace(const dta_tokens* t, const dta_vocab_params_t* p) { return workspace(t, p, false); }
size_t logprob_bwd_workspace(const dta_tokens* t, const dta_vocab_params_t* p) { return workspace(t, p, true); }
int launch_logprob_fwd(const VocabArgs& a) { return logprob_fwd(a); }
int launch_logprob_bwd(const VocabArgs& a) { return logprob_bwd(a); }

}  // namespace dta
