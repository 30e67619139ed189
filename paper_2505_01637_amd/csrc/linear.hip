// The Matmul with bias, activation, dropout and residual in its epilogue, and the row passes of its gradient
// (operators.h): kernels and launches.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "operators.h"

namespace mrl {
namespace {

constexpr int kStep = 128;                 // bytes of a step along k: 64 bf16 or 32 f32
constexpr uint32_t kLaunch = 1u << 22;     // workgroups of a launch

// ---- tiles in shared memory
//
// A step holds 128 bytes along k of every row (column) of the tile, as chunks of 16 bytes.  KC: the operand's neighbours along k
// are adjacent, a line of the tile is a row of A (column of B), 8 chunks.  Otherwise a line is one k with the W rows.
// A chunk's place in its line is its number xor swizzle(line): without it the lines that one instruction reads lie in the same
// banks.
template <class T, bool KC, bool IS_B, int W>
struct Tile {
  static constexpr int E = 16 / sizeof(T);                           // elements of a chunk
  static constexpr int kSteps = kStep / sizeof(T);                          // k of a step
  static constexpr int kLineBytes = KC ? kStep : W * (int)sizeof(T);
  static constexpr int kChunks = kLineBytes / 16;                    // of a line
  __device__ static __forceinline__ uint32_t swizzle(uint32_t line) {
    if (sizeof(T) == 2) {
      if (KC) return IS_B ? (line & 3) | (line >> 1 & 4) : line & 7;
      if (W < 64) return 0;
      if (W == 64) return (line & 2) << 1 | (line >> 2 & 2);
      return (line & 3) << 2 | (line >> 2 & 2);
    }
    if (KC) return line >> 1 & 7;
    return W < 64 ? line & 4 : (line & 4) << 1;
  }
  __device__ static __forceinline__ uint32_t at(uint32_t line, uint32_t chunk) { return line * kLineBytes + ((chunk ^ swizzle(line)) << 4); }
};

// A wave's operand for MFMA blocks of 16 x 16: rows (columns) `base` + 32 per pair of blocks.  q = lane % 16 names the row of a
// block, g = lane / 16 a quarter of the instruction's k.  The rows of a block are chosen so that a lane ends up with eight
// neighbouring columns of the result, and so that f32 reads take two blocks' rows at once:
//   bf16, A:  block i, q -> 16 i + q
//   bf16, B:  block i, q -> 32 (i / 2) + 8 (q / 4) + 4 (i % 2) + q % 4
//   f32:      block i, q -> 32 (i / 2) + 2 q + i % 2
template <class T, bool IS_B>
__device__ __forceinline__ uint32_t row_of(uint32_t i, uint32_t q) {
  if (sizeof(T) == 4) return 32 * (i >> 1) + 2 * q + (i & 1);
  return IS_B ? 32 * (i >> 1) + 8 * (q >> 2) + 4 * (i & 1) + (q & 3) : 16 * i + q;
}

typedef __attribute__((address_space(3))) const char* lds_ptr;
typedef short s16x4 __attribute__((ext_vector_type(4)));

// bf16: block i's operand of the half step kk (32 k): a lane has k = 32 kk + 8 g .. + 7.
template <bool KC, bool IS_B, int W>
__device__ __forceinline__ bf16x8 read_block(lds_ptr tile, uint32_t base, uint32_t i, uint32_t kk, uint32_t q, uint32_t g) {
  using Tl = Tile<bf16, KC, IS_B, W>;
  if (KC) {
    const uint32_t line = base + row_of<bf16, IS_B>(i, q);
    return *(const __attribute__((address_space(3))) bf16x8*)(tile + Tl::at(line, kk * 4 + g));
  }
  // a transposing read: sixteen lanes give four lines of four times four neighbours and get a column of four k each
  const uint32_t row = base + row_of<bf16, IS_B>(i, 4 * (q & 3));
  union { s16x4 h[2]; bf16x8 v; } u;
#pragma unroll
  for (uint32_t h = 0; h < 2; h++) {
    const uint32_t line = kk * 32 + 8 * g + 4 * h + (q >> 2);
    u.h[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(tile + Tl::at(line, row >> 3) + (row & 7) * 2));
  }
  return u.v;
}
// f32: blocks i and i + 1 (i even) of the half step kk (16 k): element j is k = 16 kk + 4 g + j.
template <bool KC, bool IS_B, int W>
__device__ __forceinline__ void read_pair(lds_ptr tile, uint32_t base, uint32_t i, uint32_t kk, uint32_t q, uint32_t g, f32x4& v0, f32x4& v1) {
  using Tl = Tile<float, KC, IS_B, W>;
  const uint32_t row = base + row_of<float, IS_B>(i, q);
  if (KC) {
    v0 = *(const __attribute__((address_space(3))) f32x4*)(tile + Tl::at(row, kk * 4 + g));
    v1 = *(const __attribute__((address_space(3))) f32x4*)(tile + Tl::at(row + 1, kk * 4 + g));
  } else {
#pragma unroll
    for (uint32_t j = 0; j < 4; j++) {
      const uint32_t line = kk * 16 + 4 * g + j;
      const f32x2 t = *(const __attribute__((address_space(3))) f32x2*)(tile + Tl::at(line, row >> 2) + (row & 3) * 4);
      v0[j] = t[0];
      v1[j] = t[1];
    }
  }
}

// What a lane holds of N blocks for a half step.
template <class T> struct Operand { using Type = bf16x8; };
template <> struct Operand<float> { using Type = f32x4; };

template <class T, bool KC, bool IS_B, int W, int N>
__device__ __forceinline__ void read_blocks(lds_ptr tile, uint32_t base, uint32_t first, uint32_t kk, uint32_t q, uint32_t g, typename Operand<T>::Type (&v)[N]) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = read_block<KC, IS_B, W>(tile, base, first + i, kk, q, g);
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 2) read_pair<KC, IS_B, W>(tile, base, first + i, kk, q, g, v[i], v[i + 1]);
  }
}

// acc[first + i][j] += the products of A's block i and B's block j over a half step, one of kParts parts.  The products are taken as B^T A^T: in the
// MFMA result a lane has one column and four neighbouring rows, which are then one row of the result and neighbouring columns.
template <class T, int NM> constexpr int kParts = sizeof(T) == 2 ? NM : 4;
template <int NM, int BN, int BM>
__device__ __forceinline__ void multiply(const bf16x8 (&a)[NM], const bf16x8 (&b)[BN], uint32_t first, int part, f32x4 (&acc)[BM][BN]) {
#pragma unroll
  for (int j = 0; j < BN; j++) acc[first + part][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j], a[part], acc[first + part][j], 0, 0, 0);
}
template <int NM, int BN, int BM>
__device__ __forceinline__ void multiply(const f32x4 (&a)[NM], const f32x4 (&b)[BN], uint32_t first, int part, f32x4 (&acc)[BM][BN]) {
#pragma unroll
  for (int i = 0; i < NM; i++)
#pragma unroll
    for (int j = 0; j < BN; j++) acc[first + i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(b[j][part], a[i][part], acc[first + i][j], 0, 0, 0);
}

// The part of a tile that a thread brings from global memory through registers, from any address.
//
// WIDE: every line has at least a chunk's elements.  Then every chunk is one load of 16 bytes whatever the edge: a chunk that ends past its line
// is read from the line's last 16 bytes, a line that is not there at the last one, and both are put right (shifted, zeroed) on the way
// to shared memory, so that no load waits for a branch.  Otherwise element by element.
template <class T, bool KC, bool IS_B, int W, int THREADS, bool WIDE>
struct Stage {
  using Tl = Tile<T, KC, IS_B, W>;
  static constexpr int N = W * 8 / THREADS, E = Tl::E;
  u32x4 r[N];
  uint32_t ks;                     // k that are left where r was read
  int64_t offset[N];               // bytes from a whole step's first element (worked out once: a 64-bit product per load and step costs more than the load)
  __device__ static __forceinline__ uint32_t line(int i, uint32_t t) { return (t + i * THREADS) / Tl::kChunks; }
  __device__ static __forceinline__ int32_t at(int i, uint32_t t) { return (t + i * THREADS) % Tl::kChunks * E; }
  __device__ static __forceinline__ int64_t place(int i, uint32_t t, int64_t ld, uint32_t rows, uint32_t left) {
    const uint32_t lines = KC ? rows : left, width = KC ? left : rows;
    return ((int64_t)min(line(i, t), lines - 1) * ld + min(at(i, t), (int32_t)min(width, 1u << 30) - E)) * (int64_t)sizeof(T);
  }
  __device__ __forceinline__ void init(int64_t ld, uint32_t rows, uint32_t t) {
    if constexpr (WIDE)
#pragma unroll
      for (int i = 0; i < N; i++) offset[i] = place(i, t, ld, rows, Tl::kSteps);
  }

  // src: the tile's first row (column) at k = k0; rows and left: how many rows (columns) and k there are from there on
  __device__ __forceinline__ void load(const T* src, int64_t ld, uint32_t rows, uint32_t left, uint32_t t) {
    ks = left;
    if constexpr (WIDE) {
      if (left >= (uint32_t)Tl::kSteps) {
#pragma unroll
        for (int i = 0; i < N; i++) __builtin_memcpy(&r[i], (const char*)src + offset[i], 16);
      } else {
#pragma unroll
        for (int i = 0; i < N; i++) __builtin_memcpy(&r[i], (const char*)src + place(i, t, ld, rows, left), 16);
      }
      return;
    }
    const uint32_t lines = KC ? rows : left, width = KC ? left : rows;
#pragma unroll
    for (int i = 0; i < N; i++) {
      const uint32_t l = line(i, t);
      const T* p = src + (int64_t)l * ld;
      T v[E];
#pragma unroll
      for (int e = 0; e < E; e++) v[e] = l < lines && (uint32_t)at(i, t) + e < width ? p[at(i, t) + e] : (T)0.0f;
      __builtin_memcpy(&r[i], v, 16);
    }
  }
  __device__ __forceinline__ void store(char* tile, uint32_t rows, uint32_t t) {
    if (WIDE && (ks < (uint32_t)Tl::kSteps || (!KC && rows < W))) {
      const uint32_t width = KC ? ks : rows;
#pragma unroll
      for (int i = 0; i < N; i++) {
        // (behind the end of the sum zeros; rows and columns that are not there may hold anything, as nothing of them is stored)
        const int32_t past = max(at(i, t) + E - (int32_t)min(width, 1u << 30), 0);
        const bool none = past >= E || (!KC && line(i, t) >= ks);
        const uint32_t s = past * 8 * sizeof(T) & 127;
        const uint64_t lo = (uint64_t)r[i][1] << 32 | r[i][0], hi = (uint64_t)r[i][3] << 32 | r[i][2];
        const uint64_t l = s >= 64 ? hi >> (s - 64) : s ? lo >> s | hi << (64 - s) : lo, h = s >= 64 ? 0 : hi >> s;
        r[i] = none ? u32x4{0, 0, 0, 0} : u32x4{(uint32_t)l, (uint32_t)(l >> 32), (uint32_t)h, (uint32_t)(h >> 32)};
      }
    }
#pragma unroll
    for (int i = 0; i < N; i++) *(u32x4*)(tile + Tl::at(line(i, t), (uint32_t)at(i, t) / E)) = r[i];
  }
};

// Where a workgroup's tile lies.
struct Place { uint32_t tm, tn, split, batch; };
// Workgroups go to the eight dies in turn, each with an L2 of its own: a die gets a stretch of consecutive tiles, and
// consecutive tiles are kGroup rows of tiles high, so that the tiles that are worked on at once share rows and columns there.
constexpr uint32_t kDies = 8, kGroup = 8;
__device__ __forceinline__ Place place(uint32_t first, uint32_t tiles_m, uint32_t tiles_n, uint32_t splits) {
  const uint32_t i = blockIdx.x, die = i % kDies, each = gridDim.x / kDies, rest = gridDim.x % kDies;
  uint32_t id = first + die * each + min(die, rest) + i / kDies;
  const uint32_t tiles = tiles_m * tiles_n, outer = id / tiles;
  id -= outer * tiles;
  Place at;
  at.split = outer % splits;
  at.batch = outer / splits;
  const uint32_t band = id / (kGroup * tiles_n), top = band * kGroup, high = min(kGroup, tiles_m - top);
  id -= band * kGroup * tiles_n;
  at.tm = top + id % high;
  at.tn = id / high;
  return at;
}

// Four neighbouring columns of a pair of blocks' results, the first (x = 0) or last of the eight that a lane has.
template <class T>
__device__ __forceinline__ f32x4 chunk_of(const f32x4& lo, const f32x4& hi, int x) {
  return sizeof(T) == 2 ? (x ? hi : lo) : f32x4{lo[2 * x], hi[2 * x], lo[2 * x + 1], hi[2 * x + 1]};
}

// Eight sums: the epilogue, or where others share them into the workspace.
__device__ __forceinline__ void put8(const Product& p, const Place& at, uint32_t splits, uint32_t m, uint32_t n, const float (&bias)[8], float (&v)[8], float* partial) {
  if (splits > 1) {
    float* out = partial + (((uint64_t)at.split * p.batches + at.batch) * p.M + m) * ((p.N + 7) & ~7u) + n;
#pragma unroll
    for (int x = 0; x < 2; x++) *(f32x4*)(out + 4 * x) = f32x4{v[4 * x], v[4 * x + 1], v[4 * x + 2], v[4 * x + 3]};
  } else {
    finish8(p.e, at.batch, p.M, m, n, p.N - n, bias, v);
  }
}

// A wave's results: a lane has row row_of(i, q) and, of the pair of blocks 2 j, 2 j + 1, the eight columns from 32 j + 8 g on.  They go
// through shared memory that is the wave's own, PASS blocks of 16 rows at a time, so that a row's results are stored side by side (lines of
// 128 bytes and more) and the epilogue is a short loop: unrolled over the registers it is as long as the instruction cache.  The 16-byte chunks of a
// row lie at their number xor the row's, against bank conflicts.
template <class T, int PASS, int BM, int BN>
__device__ __forceinline__ void write_out(const Product& p, const Place& at, uint32_t splits, uint32_t m0, uint32_t n0, uint32_t lane,
                                          const f32x4 (&acc)[BM][BN], char* mine, float* __restrict__ partial) {
  constexpr uint32_t CHUNKS = BN * 4, GROUPS = BN * 2, ROWS = 64 / GROUPS;      // chunks and groups of 8 columns of a row; rows at a time
  const uint32_t q = lane & 15, g = lane >> 4;
  const uint32_t c = lane % GROUPS, n = n0 + c * 8;
  float bias[8];
  bias8(p.e, n, n < p.N ? p.N - n : 0, bias);
#pragma unroll
  for (int h = 0; h < BM; h += PASS) {
#pragma unroll
    for (int i = 0; i < PASS; i++) {
      const uint32_t r = 16 * i + q;
#pragma unroll
      for (int j = 0; j < BN / 2; j++)
#pragma unroll
        for (int x = 0; x < 2; x++)
          *(f32x4*)(mine + (r * CHUNKS + ((8 * j + 2 * g + x) ^ (r & (CHUNKS - 1)))) * 16) = chunk_of<T>(acc[h + i][2 * j], acc[h + i][2 * j + 1], x);
    }
    asm volatile("" ::: "memory");         // (a wave's accesses to shared memory are done in their order)
    if (n < p.N) {
#pragma unroll 2
      for (uint32_t r = lane / GROUPS; r < 16 * PASS; r += ROWS) {
        const uint32_t m = m0 + row_of<T, false>(h + (r >> 4), r & 15);
        if (m >= p.M) continue;
        float v[8];
#pragma unroll
        for (int x = 0; x < 2; x++) {
          const f32x4 t = *(const f32x4*)(mine + (r * CHUNKS + ((2 * c + x) ^ (r & (CHUNKS - 1)))) * 16);
#pragma unroll
          for (int e = 0; e < 4; e++) v[4 * x + e] = t[e];
        }
        put8(p, at, splits, m, n, bias, v, partial);
      }
    }
    asm volatile("" ::: "memory");
  }
}

// One tile of TM x TN, WAVES_M x WAVES_N waves, over a stretch of the steps along k: operands of any stride and alignment.
template <class T, bool AKC, bool BKC, int TM, int TN, int WAVES_M, int WAVES_N, bool WIDE>
__global__ __launch_bounds__(64 * WAVES_M * WAVES_N) void product_kernel(const Product p, uint32_t steps, uint32_t per_split, uint32_t splits,
                                                                         uint32_t first, float* __restrict__ partial) {
  constexpr int THREADS = 64 * WAVES_M * WAVES_N, WM = TM / WAVES_M, WN = TN / WAVES_N, BM = WM / 16, BN = WN / 16;
  constexpr uint32_t KS = kStep / sizeof(T);
  __shared__ __attribute__((aligned(16))) char lds[2][(TM + TN) * kStep];

  const Place at = place(first, (p.M + TM - 1) / TM, (p.N + TN - 1) / TN, splits);
  const uint32_t m0 = at.tm * TM, n0 = at.tn * TN;
  const uint32_t t = threadIdx.x, lane = t & 63, wave = t >> 6, q = lane & 15, g = lane >> 4;
  const uint32_t wm = wave / WAVES_N * WM, wn = wave % WAVES_N * WN;
  const uint32_t begin = at.split * per_split, end = min(begin + per_split, steps);

  // the next step to load
  const uint32_t seg_steps = (p.K + KS - 1) / KS;
  uint32_t seg = begin < end ? begin / seg_steps : 0, k = (begin - seg * seg_steps) * KS;
  const T* a = (const T*)p.a + (int64_t)at.batch * p.batch_a + (AKC ? (int64_t)m0 * p.lda : (int64_t)m0);
  const T* b = (const T*)p.b + (int64_t)at.batch * p.batch_b + (BKC ? (int64_t)n0 * p.ldb : (int64_t)n0);
  Stage<T, AKC, false, TM, THREADS, WIDE> sa;
  Stage<T, BKC, true, TN, THREADS, WIDE> sb;
  sa.init(p.lda, p.M - m0, t);
  sb.init(p.ldb, p.N - n0, t);
  const auto load = [&] {
    sa.load(a + (int64_t)seg * p.seg_a + (AKC ? (int64_t)k : (int64_t)k * p.lda), p.lda, p.M - m0, p.K - k, t);
    sb.load(b + (int64_t)seg * p.seg_b + (BKC ? (int64_t)k : (int64_t)k * p.ldb), p.ldb, p.N - n0, p.K - k, t);
    k += KS;
    if (k >= p.K) { k = 0; seg++; }
  };
  const auto store = [&](char* stage) {
    sa.store(stage, p.M - m0, t);
    sb.store(stage + TM * kStep, p.N - n0, t);
  };

  f32x4 acc[BM][BN];
#pragma unroll
  for (int i = 0; i < BM; i++)
#pragma unroll
    for (int j = 0; j < BN; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  if (begin < end) {
    load();
    store(lds[0]);
  }
  __syncthreads();
  for (uint32_t step = begin; step < end; step++) {
    const uint32_t cur = (step - begin) & 1;
    if (step + 1 < end) load();
    const lds_ptr ta = (lds_ptr)lds[cur], tb = ta + TM * kStep;
#pragma unroll
    for (uint32_t kk = 0; kk < 2; kk++) {
      typename Operand<T>::Type fa[BM], fb[BN];
      read_blocks<T, AKC, false, TM>(ta, wm, 0, kk, q, g, fa);
      read_blocks<T, BKC, true, TN>(tb, wn, 0, kk, q, g, fb);
#pragma unroll
      for (int part = 0; part < kParts<T, BM>; part++) multiply(fa, fb, 0, part, acc);
    }
    if (step + 1 < end) store(lds[cur ^ 1]);
    __syncthreads();
  }
  write_out<T, BM, BM, BN>(p, at, splits, m0 + wm, n0 + wn, lane, acc, &lds[0][0] + wave * (WM * WN * 4), partial);
}

// ---- operands whose lines start at multiples of 16 bytes
//
// Loads go from memory to shared memory past the registers (a wave's load writes 1024 bytes in a row, a lane 16 of them, so the swizzle
// is applied to the address that a lane reads), through a buffer descriptor whose range check gives 0 for what lies behind the operand.

// Waits until at most LEFT of the wave's loads are under way and its reads of shared memory are done, then for the other waves.
template <int LEFT>
__device__ __forceinline__ void arrive() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory"); }

// (The load is written out because the compiler, which cannot tell the stages apart, would wait for every load under way before any
// read of shared memory.  It has no output register; its address registers are read as it is issued.)
__device__ __forceinline__ void load_to_lds(uint32_t lds, uint32_t offset, u32x4 buffer) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(offset), "s"(buffer) : "memory");
}

constexpr uint32_t kOutside = 0x80000000u;        // beyond any buffer's range

template <class T, bool KC, bool IS_B, int W, int THREADS>
struct Feed {
  using Tl = Tile<T, KC, IS_B, W>;
  static constexpr int N = W * 8 / THREADS;       // loads of a thread and step
  uint32_t offset[N];                             // bytes from the tile's first element of a step
  __device__ __forceinline__ void init(int64_t ld, uint32_t t) {
#pragma unroll
    for (int i = 0; i < N; i++) {
      const uint32_t c = t + i * THREADS, line = c / Tl::kChunks, chunk = c % Tl::kChunks ^ Tl::swizzle(line);
      offset[i] = line * (uint32_t)ld * (uint32_t)sizeof(T) + chunk * 16;
    }
  }
  // Descriptor of what lies behind the tile's first element of a step; left: bytes to the operand's end.
  __device__ static __forceinline__ u32x4 buffer(const char* from, int64_t left) {
    const uint64_t base = (uint64_t)from;
    const uint32_t low = (uint32_t)left, range = (uint32_t)(left >> 32) | low >> 31 ? kOutside : low;      // (scalar units have no 64-bit minimum)
    return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)base), (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(base >> 32) & 0xFFFFu),
                 (uint32_t)__builtin_amdgcn_readfirstlane(range), 0x27000u};
  }
  // The thread's i-th load of a step; ks: k that are left in the segment; lds: where the wave's first load goes.
  __device__ __forceinline__ void load(int i, const u32x4& buffer, uint32_t ks, uint32_t lds, uint32_t t) const {
    uint32_t at = offset[i];
    if (KC && ks < Tl::kSteps) {                  // chunks past the end of the sum would be the next line's
      const uint32_t c = t + i * THREADS, line = c / Tl::kChunks, chunk = c % Tl::kChunks ^ Tl::swizzle(line);
      if (chunk * Tl::E >= ks) at = kOutside;
    }
    load_to_lds(lds + i * THREADS * 16, at, buffer);
  }
};

// One tile of TM x TN, WAVES_M x WAVES_N waves, STAGES steps in shared memory.
//
// A wave of the 256 tile has 128 x 64 of it: 24 KB read from shared memory for 64 MFMA of a step, 192 KB and 64 KB written by all eight
// waves in 2048 cycles of products.  8192-cube in bf16 805 us, 1360 TFLOP/s: 577 us without loads and reads of shared memory, 650 without the loads, 770
// without the reads, 755 with every step's operands in L2; so what bounds it is the way of the operands to shared memory, then their
// reads.  2048-cube in f32 (128 x 128, eight waves) 135 us, of which the products take 117 at the clock it runs at.
template <class T, bool AKC, bool BKC, int TM, int TN, int WAVES_M, int WAVES_N, int STAGES>
__global__ __launch_bounds__(64 * WAVES_M * WAVES_N, 2) void fast_kernel(const Product p, uint32_t steps, uint32_t per_split, uint32_t splits,
                                                                      uint32_t first, float* __restrict__ partial) {
  constexpr int THREADS = 64 * WAVES_M * WAVES_N, WM = TM / WAVES_M, WN = TN / WAVES_N, BM = WM / 16, BN = WN / 16;
  constexpr int PASS = BM > 4 ? BM / 2 : BM;
  constexpr uint32_t KS = kStep / sizeof(T), STAGE = (TM + TN) * kStep, OUT = 16 * PASS * WN * 4;
  __shared__ __attribute__((aligned(1024))) char lds[STAGES * STAGE];
  static_assert(WAVES_M * WAVES_N * OUT <= sizeof lds, "the results go where the stages were");

  const Place at = place(first, (p.M + TM - 1) / TM, (p.N + TN - 1) / TN, splits);
  const uint32_t m0 = at.tm * TM, n0 = at.tn * TN;
  const uint32_t t = threadIdx.x, lane = t & 63, q = lane & 15, g = lane >> 4;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const uint32_t wm = wave / WAVES_N * WM, wn = wave % WAVES_N * WN;

  Feed<T, AKC, false, TM, THREADS> fa;
  Feed<T, BKC, true, TN, THREADS> fb;
  fa.init(p.lda, t);
  fb.init(p.ldb, t);
  constexpr int LOADS = decltype(fa)::N + decltype(fb)::N;
  const uint32_t seg_steps = (p.K + KS - 1) / KS;
  const int64_t step_a = (AKC ? (int64_t)KS : KS * p.lda) * sizeof(T), step_b = (BKC ? (int64_t)KS : KS * p.ldb) * sizeof(T);

  const uint32_t from = at.split * per_split, end = min(from + per_split, steps), n = end > from ? end - from : 0;

  // the next step to load: where it starts in either operand, the bytes that are left behind that, the k
  const uint32_t seg = n ? from / seg_steps : 0, step0 = from - seg * seg_steps;
  uint32_t k = step0 * KS, loaded = 0;
  const char* sa = (const char*)((const T*)p.a + (int64_t)at.batch * p.batch_a + (int64_t)seg * p.seg_a + (AKC ? (int64_t)m0 * p.lda : (int64_t)m0)) + step0 * step_a;
  const char* sb = (const char*)((const T*)p.b + (int64_t)at.batch * p.batch_b + (int64_t)seg * p.seg_b + (BKC ? (int64_t)n0 * p.ldb : (int64_t)n0)) + step0 * step_b;
  int64_t left_a = (AKC ? ((int64_t)(p.M - m0) - 1) * p.lda + p.wa : ((int64_t)p.K - 1) * p.lda + (p.wa - m0)) * (int64_t)sizeof(T) - step0 * step_a;
  int64_t left_b = (BKC ? ((int64_t)(p.N - n0) - 1) * p.ldb + p.wb : ((int64_t)p.K - 1) * p.ldb + (p.wb - n0)) * (int64_t)sizeof(T) - step0 * step_b;
  // (behind the last step the buffers have no bytes: zeros are written that nothing uses, and every step has the same loads under way)
  u32x4 buf_a, buf_b;
  uint32_t to, ks;
  const auto aim = [&](uint32_t stage) {          // at the next step, to be put into `stage`
    const bool more = loaded++ < n;
    to = (uint32_t)(uintptr_t)(lds_ptr)lds + stage * STAGE + wave * 1024;
    ks = p.K - k;
    buf_a = fa.buffer(sa, more ? left_a : 0);
    buf_b = fb.buffer(sb, more ? left_b : 0);
    if (!more) return;
    k += KS;
    sa += step_a;
    sb += step_b;
    left_a -= step_a;
    left_b -= step_b;
    if (k >= p.K) {                               // the next segment
      k = 0;
      sa += p.seg_a * (int64_t)sizeof(T) - seg_steps * step_a;
      sb += p.seg_b * (int64_t)sizeof(T) - seg_steps * step_b;
      left_a += seg_steps * step_a;
      left_b += seg_steps * step_b;
    }
  };
  const auto load = [&](int i) {
    if (i < fa.N) fa.load(i, buf_a, ks, to, t);
    else fb.load(i - fa.N, buf_b, ks, to + TM * kStep, t);
  };
  f32x4 acc[BM][BN];
#pragma unroll
  for (int i = 0; i < BM; i++)
#pragma unroll
    for (int j = 0; j < BN; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  // A step is two half steps of one or two phases, of NM blocks of rows each.  A phase first reads the operands of the next one, then
  // multiplies, so that the reads' latency lies under the products.  Before the last phase everything of the step has been read and
  // the next step's tile must be there: the one barrier of a step; behind it this step's place is free for the step STAGES ahead.  Its
  // loads go out one by one between the products from there on: all at once they fill the queue to memory, and the wave stands still
  // before its products until the queue has room (8192-cube 850 us, spread 820).
  constexpr int NM = BM > 4 ? BM / 2 : BM, PHASES = 2 * BM / NM, PARTS = kParts<T, NM>;
  constexpr bool SPREAD = BM > 4;
  static_assert(LOADS <= PHASES * PARTS, "one load at most beside a part of the products");
  typename Operand<T>::Type oa[2][NM], ob[2][BN];
  if (n) {
#pragma unroll
    for (int s = 0; s < STAGES; s++) {
      aim(s);
#pragma unroll
      for (int i = 0; i < LOADS; i++) load(i);
    }
    arrive<(STAGES - 1) * LOADS>();
    read_blocks<T, AKC, false, TM>((lds_ptr)lds, wm, 0, 0, q, g, oa[0]);
    read_blocks<T, BKC, true, TN>((lds_ptr)lds + TM * kStep, wn, 0, 0, q, g, ob[0]);
    uint32_t cur = 0;
    for (uint32_t s = 0; s < n; s++) {
      const uint32_t next = cur + 1 == STAGES ? 0 : cur + 1;
#pragma unroll
      for (int ph = 0; ph < PHASES; ph++) {
        const int then = (ph + 1) % PHASES, kk = then / (PHASES / 2), m = then % (PHASES / 2) * NM;
        if (ph == PHASES - 1) {
          arrive<(STAGES - 2) * LOADS>();
          aim(cur);
#pragma unroll
          for (int i = 0; i < (SPREAD ? 0 : LOADS); i++) load(i);
        }
        const lds_ptr stage = (lds_ptr)lds + (ph == PHASES - 1 ? next : cur) * STAGE;
        read_blocks<T, AKC, false, TM>(stage, wm, m, kk, q, g, oa[then & 1]);
        if (m == 0) read_blocks<T, BKC, true, TN>(stage + TM * kStep, wn, 0, kk, q, g, ob[kk]);
#pragma unroll
        for (int part = 0; part < PARTS; part++) {
          multiply(oa[ph & 1], ob[ph / (PHASES / 2)], ph % (PHASES / 2) * NM, part, acc);
          // (in the first step, before its barrier, the last stage's loads again: the same bytes to the same place)
          if (SPREAD && then * PARTS + part < LOADS) {
            load(then * PARTS + part);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      cur = next;
    }
    arrive<0>();                  // nothing is under way to shared memory when it is given up
  }
  write_out<T, PASS, BM, BN>(p, at, splits, m0 + wm, n0 + wn, lane, acc, lds + wave * OUT, partial);
}

// The sums of a workgroup's waves over one tile of few rows and 64 columns, added in their order: each wave's in shared memory of its own, `each`
// bytes apart, rows of 64 with the 16-byte chunks of a row at their number xor the row's.
// bias: of the eight columns that the thread stores, asked for before the sums are made.
template <class T, int WAVES, int BM>
__device__ __forceinline__ void add_waves(const Product& p, const Place& at, uint32_t splits, uint32_t m0, uint32_t n0, uint32_t t, const float (&bias)[8],
                                          const f32x4 (&acc)[BM][4], char* lds, uint32_t each, float* __restrict__ partial) {
  static_assert(BM * 16 * 8 <= 64 * WAVES, "eight columns a thread");
  const uint32_t q = t & 15, g = t >> 4 & 3;
  char* const mine = lds + (t >> 6) * each;
#pragma unroll
  for (int i = 0; i < BM; i++) {
    const uint32_t r = row_of<T, false>(i, q);
#pragma unroll
    for (int j = 0; j < 2; j++)
#pragma unroll
      for (int x = 0; x < 2; x++) *(f32x4*)(mine + (r * 16 + ((8 * j + 2 * g + x) ^ (r & 15))) * 16) = chunk_of<T>(acc[i][2 * j], acc[i][2 * j + 1], x);
  }
  __syncthreads();
  const uint32_t r = t / 8, c = t % 8, m = m0 + r, col = n0 + c * 8;
  if (r >= BM * 16 || m >= p.M || col >= p.N) return;
  float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int w = 0; w < WAVES; w++)
#pragma unroll
    for (int x = 0; x < 2; x++) {
      const f32x4 y = *(const f32x4*)(lds + w * each + (r * 16 + ((2 * c + x) ^ (r & 15))) * 16);
#pragma unroll
      for (int e = 0; e < 4; e++) v[4 * x + e] += y[e];
    }
  put8(p, at, splits, m, col, bias, v, partial);
}

// Few rows: the sum is split among the waves of a workgroup, each with a ring of STAGES steps of its own in shared memory and no barrier
// until their sums are added up.  A tile of 16 rows (f32: 32, as its operands are read two blocks at a time) and 64 columns; wave w takes the
// steps w, w + WAVES, ...  Bound by the read of the columns: 1 x 2048 x 16384 in bf16 keeps 96 KB under way on every compute unit.
template <class T, bool AKC, bool BKC, int WAVES, int STAGES>
__global__ __launch_bounds__(64 * WAVES) void rows_kernel(const Product p, uint32_t steps, uint32_t per_split, uint32_t splits, uint32_t first,
                                                          float* __restrict__ partial) {
  constexpr int TM = sizeof(T) == 2 ? 16 : 32, TN = 64, BM = TM / 16, BN = TN / 16;
  constexpr uint32_t KS = kStep / sizeof(T), STAGE = (TM + TN) * kStep;
  __shared__ __attribute__((aligned(1024))) char lds[WAVES][STAGES * STAGE];

  const Place at = place(first, (p.M + TM - 1) / TM, (p.N + TN - 1) / TN, splits);
  const uint32_t m0 = at.tm * TM, n0 = at.tn * TN;
  const uint32_t t = threadIdx.x, lane = t & 63, q = lane & 15, g = lane >> 4;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(t >> 6);

  float bias[8];
  bias8(p.e, n0 + t % 8 * 8, n0 + t % 8 * 8 < p.N ? p.N - (n0 + t % 8 * 8) : 0, bias);
  Feed<T, AKC, false, TM, 64> fa;
  Feed<T, BKC, true, TN, 64> fb;
  fa.init(p.lda, lane);
  fb.init(p.ldb, lane);
  constexpr int LOADS = decltype(fa)::N + decltype(fb)::N;

  const uint32_t seg_steps = (p.K + KS - 1) / KS;
  const uint32_t begin = at.split * per_split, end = min(begin + per_split, steps);
  uint32_t step = begin + wave;                   // the next one to load
  const uint32_t n = end > step ? (end - step + WAVES - 1) / WAVES : 0;
  const char *a0 = (const char*)((const T*)p.a + (int64_t)at.batch * p.batch_a + (AKC ? (int64_t)m0 * p.lda : (int64_t)m0));
  const char *b0 = (const char*)((const T*)p.b + (int64_t)at.batch * p.batch_b + (BKC ? (int64_t)n0 * p.ldb : (int64_t)n0));
  const int64_t size_a = (AKC ? ((int64_t)(p.M - m0) - 1) * p.lda + p.wa : ((int64_t)p.K - 1) * p.lda + (p.wa - m0)) * (int64_t)sizeof(T);
  const int64_t size_b = (BKC ? ((int64_t)(p.N - n0) - 1) * p.ldb + p.wb : ((int64_t)p.K - 1) * p.ldb + (p.wb - n0)) * (int64_t)sizeof(T);
  char* const ring = lds[wave];
  const auto load = [&](uint32_t stage) {
    const uint32_t to = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_ptr)ring + stage * STAGE);
    const bool more = step < end;
    const uint32_t seg = more ? step / seg_steps : 0, k = more ? (step - seg * seg_steps) * KS : 0;
    const int64_t off_a = (AKC ? (int64_t)k : (int64_t)k * p.lda) * (int64_t)sizeof(T), off_b = (BKC ? (int64_t)k : (int64_t)k * p.ldb) * (int64_t)sizeof(T);
    const u32x4 buf_a = fa.buffer(a0 + (int64_t)seg * p.seg_a * (int64_t)sizeof(T) + off_a, more ? size_a - off_a : 0);
    const u32x4 buf_b = fb.buffer(b0 + (int64_t)seg * p.seg_b * (int64_t)sizeof(T) + off_b, more ? size_b - off_b : 0);
#pragma unroll
    for (int i = 0; i < fa.N; i++) fa.load(i, buf_a, p.K - k, to, lane);
#pragma unroll
    for (int i = 0; i < fb.N; i++) fb.load(i, buf_b, p.K - k, to + TM * kStep, lane);
    step += WAVES;
  };

  f32x4 acc[BM][BN];
#pragma unroll
  for (int i = 0; i < BM; i++)
#pragma unroll
    for (int j = 0; j < BN; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  if (n) {
#pragma unroll
    for (int s = 0; s < STAGES; s++) load(s);
    uint32_t cur = 0;
    for (uint32_t s = 0; s < n; s++) {
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"((STAGES - 1) * LOADS) : "memory");
      const lds_ptr tile = (lds_ptr)ring + cur * STAGE;
      typename Operand<T>::Type oa[2][BM], ob[2][BN];
#pragma unroll
      for (uint32_t kk = 0; kk < 2; kk++) {
        read_blocks<T, AKC, false, TM>(tile, 0, 0, kk, q, g, oa[kk]);
        read_blocks<T, BKC, true, TN>(tile + TM * kStep, 0, 0, kk, q, g, ob[kk]);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // read before the place is loaded again
      load(cur);
#pragma unroll
      for (int kk = 0; kk < 2; kk++)
#pragma unroll
        for (int part = 0; part < kParts<T, BM>; part++) multiply(oa[kk], ob[kk], 0, part, acc);
      cur = cur + 1 == STAGES ? 0 : cur + 1;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }

  add_waves<T, WAVES>(p, at, splits, m0, n0, t, bias, acc, &lds[0][0], sizeof lds[0], partial);
}

// The same for operands of any alignment: through registers, the next step's loads under way while this one is multiplied.
template <class T, bool AKC, bool BKC, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void rows_wide_kernel(const Product p, uint32_t steps, uint32_t per_split, uint32_t splits, uint32_t first,
                                                               float* __restrict__ partial) {
  constexpr int TM = sizeof(T) == 2 ? 16 : 32, TN = 64, BM = TM / 16, BN = TN / 16;
  constexpr uint32_t KS = kStep / sizeof(T);
  __shared__ __attribute__((aligned(16))) char lds[WAVES][(TM + TN) * kStep];

  const Place at = place(first, (p.M + TM - 1) / TM, (p.N + TN - 1) / TN, splits);
  const uint32_t m0 = at.tm * TM, n0 = at.tn * TN;
  const uint32_t t = threadIdx.x, lane = t & 63, q = lane & 15, g = lane >> 4;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(t >> 6);

  const uint32_t seg_steps = (p.K + KS - 1) / KS;
  const uint32_t begin = at.split * per_split, end = min(begin + per_split, steps);
  const T* a = (const T*)p.a + (int64_t)at.batch * p.batch_a + (AKC ? (int64_t)m0 * p.lda : (int64_t)m0);
  const T* b = (const T*)p.b + (int64_t)at.batch * p.batch_b + (BKC ? (int64_t)n0 * p.ldb : (int64_t)n0);
  float bias[8];
  bias8(p.e, n0 + t % 8 * 8, n0 + t % 8 * 8 < p.N ? p.N - (n0 + t % 8 * 8) : 0, bias);
  Stage<T, AKC, false, TM, 64, true> sa;
  Stage<T, BKC, true, TN, 64, true> sb;
  sa.init(p.lda, p.M - m0, lane);
  sb.init(p.ldb, p.N - n0, lane);
  const auto load = [&](uint32_t step) {
    const uint32_t seg = step / seg_steps, k = (step - seg * seg_steps) * KS;
    sa.load(a + (int64_t)seg * p.seg_a + (AKC ? (int64_t)k : (int64_t)k * p.lda), p.lda, p.M - m0, p.K - k, lane);
    sb.load(b + (int64_t)seg * p.seg_b + (BKC ? (int64_t)k : (int64_t)k * p.ldb), p.ldb, p.N - n0, p.K - k, lane);
  };

  f32x4 acc[BM][BN];
#pragma unroll
  for (int i = 0; i < BM; i++)
#pragma unroll
    for (int j = 0; j < BN; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  char* const mine = lds[wave];
  if (begin + wave < end) load(begin + wave);
  for (uint32_t step = begin + wave; step < end; step += WAVES) {
    asm volatile("" ::: "memory");         // (a wave's accesses to shared memory are done in their order)
    sa.store(mine, p.M - m0, lane);
    sb.store(mine + TM * kStep, p.N - n0, lane);
    asm volatile("" ::: "memory");
    if (step + WAVES < end) load(step + WAVES);
#pragma unroll
    for (uint32_t kk = 0; kk < 2; kk++) {
      typename Operand<T>::Type oa[BM], ob[BN];
      read_blocks<T, AKC, false, TM>((lds_ptr)mine, 0, 0, kk, q, g, oa);
      read_blocks<T, BKC, true, TN>((lds_ptr)mine + TM * kStep, 0, 0, kk, q, g, ob);
#pragma unroll
      for (int part = 0; part < kParts<T, BM>; part++) multiply(oa, ob, 0, part, acc);
    }
  }
  asm volatile("" ::: "memory");
  add_waves<T, WAVES>(p, at, splits, m0, n0, t, bias, acc, &lds[0][0], sizeof lds[0], partial);
}

// What is left to do when a call's products and rows are through, in one launch: the sums over splits of up to two products with their
// epilogues, and the column sums of dz.  All are added in an order that sizes, types and alignments alone decide.
struct Rest {
  Product p[2];
  uint32_t splits[2];              // 1: nothing to join
  const float* partial[2];
  uint64_t blocks[2];
  const float* sums;               // the row blocks' column sums, nullptr: none
  uint32_t row_blocks, N, dbias_bf16, bias_blocks;
  void* dbias;
};

// Eight columns a thread.
__device__ __forceinline__ void join(const Product& p, uint32_t splits, const float* __restrict__ partial, uint64_t id) {
  const uint32_t groups = (p.N + 7) / 8;
  const uint64_t rows = (uint64_t)p.batches * p.M, row = id / groups;
  if (row >= rows) return;
  const uint32_t n = (uint32_t)(id - row * groups) * 8;
  const float* in = partial + row * (groups * 8) + n;
  float bias[8], v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
  bias8(p.e, n, p.N - n, bias);
#pragma unroll 4
  for (uint32_t s = 0; s < splits; s++) {
    const f32x4 x = *(const f32x4*)in, y = *(const f32x4*)(in + 4);
#pragma unroll
    for (int e = 0; e < 4; e++) { v[e] += x[e]; v[4 + e] += y[e]; }
    in += rows * (groups * 8);
  }
  const uint32_t batch = (uint32_t)(row / p.M);
  finish8(p.e, batch, p.M, (uint32_t)(row - (uint64_t)batch * p.M), n, p.N - n, bias, v);
}

__global__ __launch_bounds__(256) void rest_kernel(const Rest r, uint64_t first) {
  __shared__ float sums[8][32];
  uint64_t block = first + blockIdx.x;
  if (block < r.bias_blocks) {     // 32 columns, eight rows of sums at a time
    const uint32_t c = threadIdx.x & 31, l = threadIdx.x >> 5, n = (uint32_t)block * 32 + c;
    float s = 0.0f;
    if (n < r.N) {
#pragma unroll 8
      for (uint32_t i = l; i < r.row_blocks; i += 8) s += r.sums[(uint64_t)i * r.N + n];
    }
    sums[l][c] = s;
    __syncthreads();
    if (l || n >= r.N) return;
    for (int i = 1; i < 8; i++) s += sums[i][c];
    if (r.dbias_bf16) ((bf16*)r.dbias)[n] = (bf16)s;
    else ((float*)r.dbias)[n] = s;
    return;
  }
  block -= r.bias_blocks;
  if (block < r.blocks[0]) join(r.p[0], r.splits[0], r.partial[0], block * 256 + threadIdx.x);
  else join(r.p[1], r.splits[1], r.partial[1], (block - r.blocks[0]) * 256 + threadIdx.x);
}

// ---- rows

// Rows of a workgroup of grad_rows_kernel: 8 to 32, fewer where there would not be a thousand workgroups (1000 x 777 in f32: 64 rows
// 21 us, 8 rows 7 us; 4096 x 16384 in bf16 with ReLU and the sums: 128 rows 136 us, 64 rows 122, 32 rows 115, 16 rows 115 and more partial sums to read).
// Up to 64 rows are one block: its sums are dbias, and no launch follows to add them up.
uint32_t grad_rows(uint64_t rows, uint32_t N) {
  const uint64_t blocks_n = (N + 255) / 256;
  if (rows <= 64) return 64;
  uint32_t each = 32;
  while (each > 8 && (rows + each - 1) / each * blocks_n < 1024) each /= 2;
  return each;
}

// dz, and for dbias the column sums of the workgroup's rows before dz is rounded.  A workgroup: 256 columns, eight a thread, eight
// rows at a time; grid: column blocks x row blocks.
__global__ __launch_bounds__(256) void grad_rows_kernel(const GradRows p, uint32_t each, uint32_t first, float* __restrict__ partial) {
  __shared__ float sums[8][256];
  const uint32_t blocks_n = (p.N + 255) / 256, id = first + blockIdx.x, bn = id % blocks_n, br = id / blocks_n;
  const uint32_t c = threadIdx.x & 31, r = threadIdx.x >> 5, n = bn * 256 + c * 8, rows = p.batches * p.M;
  float sum[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
  if (n < p.N) {
    const uint32_t valid = p.N - n;
    for (uint32_t i = 0; i < each / 8; i++) {
      const uint64_t at = (uint64_t)br * each + i * 8 + r;
      if (at >= rows) break;
      const uint32_t row = (uint32_t)at, batch = row / p.M, m = row - batch * p.M;
      float v[8];
      load8(p.grad.data, p.grad.bf16, (int64_t)batch * p.grad.batch + (int64_t)m * p.grad.ld + n, valid, v);
      if (p.pre.data) {
        float z[8];
        load8(p.pre.data, p.pre.bf16, (int64_t)batch * p.pre.batch + (int64_t)m * p.pre.ld + n, valid, z);
        slope8(p.activation, z, v);
      }
      if (p.drop.drop) drop8(p.drop, row, n, v);       // (last: a dropped element is 0 whatever its z was)
#pragma unroll
      for (int e = 0; e < 8; e++) sum[e] += v[e];
      if (p.dz.data) store8(p.dz.data, p.dz.bf16, (int64_t)batch * p.dz.batch + (int64_t)m * p.dz.ld + n, 8, v);     // (zeros up to a multiple of 8)
    }
  }
  if (!p.dbias) return;
#pragma unroll
  for (int e = 0; e < 8; e++) sums[r][c * 8 + e] = sum[e];
  __syncthreads();
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; i++) s += sums[i][threadIdx.x];
  const uint32_t at = bn * 256 + threadIdx.x;
  if (at >= p.N) return;
  if (partial) partial[(uint64_t)br * p.N + at] = s;
  else if (p.dbias_bf16) ((bf16*)p.dbias)[at] = (bf16)s;
  else ((float*)p.dbias)[at] = s;
}

__global__ __launch_bounds__(256) void drop_kernel(const DropRows p, uint64_t first) {
  const uint32_t groups = (p.N + 7) / 8;
  const uint64_t id = first + (uint64_t)blockIdx.x * 256 + threadIdx.x, row = id / groups;
  if (row >= p.M) return;
  const uint32_t n = (uint32_t)(id - row * groups) * 8, valid = p.N - n;
  float v[8];
  load8(p.x.data, p.x.bf16, (int64_t)row * p.x.ld + n, valid, v);
  if (p.drop.drop) drop8(p.drop, (uint32_t)row, n, v);
  if (p.residual.data) {
    float r[8];
    load8(p.residual.data, p.residual.bf16, (int64_t)row * p.residual.ld + n, valid, r);
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] += r[e];
  }
  store8(p.out.data, p.out.bf16, (int64_t)row * p.out.ld + n, valid, v);
}

// Work of `blocks` workgroups in launches of at most kLaunch: f(first, count)
template <class F>
hipError_t in_launches(uint64_t blocks, F&& f) {
  for (uint64_t at = 0; at < blocks; at += kLaunch) {
    f(at, (uint32_t)std::min<uint64_t>(kLaunch, blocks - at));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class T, bool AKC, bool BKC>
hipError_t launch_tiles(const Product& p, const ProductPlan& plan, float* partial, hipStream_t st) {
  return in_launches(plan.blocks, [&](uint64_t first, uint32_t n) {
    const auto go = [&](auto kernel, uint32_t threads) { kernel<<<n, threads, 0, st>>>(p, plan.steps, plan.per_split, plan.splits, (uint32_t)first, partial); };
    switch (plan.kernel) {
      case kFast256: return go(fast_kernel<T, AKC, BKC, 256, 256, 2, 4, 2>, 512);
      case kFast256x128: return go(fast_kernel<T, AKC, BKC, 256, 128, 4, 2, 3>, 512);
      case kFast128: return go(fast_kernel<T, AKC, BKC, 128, 128, 2, 4, 2>, 512);
      case kFast128Alone: return go(fast_kernel<T, AKC, BKC, 128, 128, 2, 4, 4>, 512);
      case kFast64: return go(fast_kernel<T, AKC, BKC, 64, 64, 2, 2, 4>, 256);
      case kRows: return go(rows_kernel<T, AKC, BKC, 4, 3>, 256);
      case kRowsWide: return go(rows_wide_kernel<T, AKC, BKC, 8>, 512);
      case kWide128: return go(product_kernel<T, AKC, BKC, 128, 128, 2, 2, true>, 256);
      case kWide64: return go(product_kernel<T, AKC, BKC, 64, 64, 2, 2, true>, 256);
      case kAny64: return go(product_kernel<T, AKC, BKC, 64, 64, 2, 2, false>, 256);
    }
  });
}
template <class T>
hipError_t launch_layout(const Product& p, const ProductPlan& plan, float* partial, hipStream_t st) {
  if (p.a_kc) return p.b_kc ? launch_tiles<T, true, true>(p, plan, partial, st) : launch_tiles<T, true, false>(p, plan, partial, st);
  return p.b_kc ? launch_tiles<T, false, true>(p, plan, partial, st) : launch_tiles<T, false, false>(p, plan, partial, st);
}

// What operands allow.  kAligned: every line that is read starts at a multiple of 16 bytes, ends at one, and follows the one before, and
// offsets within a tile fit 31 bits.  kWide: every line holds 16 bytes at least, of the elements that the sum is over or the tile has (Stage moves a
// load that ends past those back by as much, and zeros that follow a shorter line do not keep it from starting before the line).
enum Access { kAligned, kWide, kAny };
bool aligned(const void* data, int64_t ld, int64_t batch, int64_t seg, int64_t width, int64_t e) {
  return (uintptr_t)data % 16 == 0 && ld % e == 0 && batch % e == 0 && seg % e == 0 && width % e == 0 && ld >= width && ld < (int64_t)1 << 21;
}

// Matrices of `lines` lines of `width` elements, copied to lines of `pitch` elements (a multiple of 16 bytes), zeros behind the width.
struct Copy {
  const void* from;
  void* to;
  int64_t ld, step;                // from a line to the next, from a matrix to the next
  uint32_t matrices, lines, width, pitch;
  uint64_t chunks() const { return (uint64_t)matrices * lines * pitch; }        // (times the elements of a chunk)
};

// 16 bytes a thread, first of a's copy, then of b's.
template <class T>
__global__ __launch_bounds__(256) void copy_kernel(const Copy a, const Copy b, uint64_t chunks_a, uint64_t chunks, uint64_t first) {
  constexpr uint32_t E = 16 / sizeof(T);
  uint64_t id = (first + blockIdx.x) * 256 + threadIdx.x;
  if (id >= chunks) return;
  const Copy& c = id < chunks_a ? a : b;
  if (id >= chunks_a) id -= chunks_a;
  const uint32_t per = c.pitch / E;
  const uint64_t line = id / per, matrix = line / c.lines;
  const uint32_t at = (uint32_t)(id - line * per) * E;
  const T* from = (const T*)c.from + (int64_t)matrix * c.step + (int64_t)(line - matrix * c.lines) * c.ld + at;
  T v[E];
  if (at + E <= c.width) {
    __builtin_memcpy(v, from, 16);
  } else {
#pragma unroll
    for (uint32_t e = 0; e < E; e++) v[e] = at + e < c.width ? from[e] : (T)0.0f;
  }
  *(u32x4*)((T*)c.to + line * c.pitch + at) = *(const u32x4*)v;
}

// The copy of an operand: as many matrices as it has, lines along the other index than its own.
Copy copy_of(const void* from, uint32_t kc, int64_t ld, int64_t batch, int64_t seg, uint32_t width, const Product& p, uint32_t others) {
  const uint32_t e = p.bf16 ? 8 : 4;
  const bool batched = p.batches > 1 && batch, segmented = p.segs > 1 && seg;       // (never both)
  return Copy{from, nullptr, ld, batched ? batch : seg, batched ? p.batches : segmented ? p.segs : 1, kc ? others : p.K, width, (width + e - 1) / e * e};
}
Copy copy_a(const Product& p) { return copy_of(p.a, p.a_kc, p.lda, p.batch_a, p.seg_a, p.a_kc ? p.K : p.M, p, p.M); }
Copy copy_b(const Product& p) { return copy_of(p.b, p.b_kc, p.ldb, p.batch_b, p.seg_b, p.b_kc ? p.K : p.N, p, p.N); }

}  // namespace

// How long a kernel takes, in us: a round of workgroups on the 256 compute units, one each or two at once, is `fixed` and a
// step's time for each step along k.  What the rule takes, from products whose tiles are one whole round, 2048 and 8192 long along k:
//                           step bf16 (one, two)   step f32 (one, two)
//   256 x 256                    1.52     -          7.33     -
//   256 x 128                    0.87     -          3.81     -
//   128 x 128, 4 stages          0.50     -          1.99     -        (2 stages alone: 0.56; four fill the shared memory)
//   128 x 128, 2 stages            -     0.93          -     3.78
//   64 x 64                      0.25    0.37        0.62    1.07
//   few rows                     0.12    0.24        0.27    0.54
//   few rows, any alignment      0.11    0.42        0.20    0.70
//   128 x 128, any alignment     1.25    1.70        2.50    4.80
//   64 x 64, any alignment       0.80    0.86        0.72    1.15
//   64 x 64, narrow lines        2.0     3.0         2.0     3.0      (round numbers, see below)
// The same products back to back in a graph, from odd elements on where any alignment is allowed, take 1.53, 0.93, 0.56 (two: 1.01), 0.28 (0.40), 0.13 (0.24),
// 0.21 (0.40), 0.96 (1.33), 0.69 (0.66) and 2.1 (3.4) in bf16, 7.3, 3.8, 2.0 (3.8), 0.61 (1.05), 0.30 (0.58), 0.33 (0.64), 2.3 (4.2), 0.81 (1.26) and 1.1 (1.9) in f32.
// Narrow lines (a line holds less than 16 bytes, so loads go element by element) were not measured when the rule was made, and f32 is priced too high: with the
// measured times one narrow f32 product in seven would not be copied, or be split, and 40 such products took the same time on geometric mean, 0.7 to 1.5 of it
// each.  `fixed` is set, not measured: with a launch and the results' stores a round takes 15, 9, 7, 5, 4, 4, 9, 2 and 2 beside its steps in bf16, 18, 14, 10, 6, 6, 8, 10, 5
// and 10 in f32, so it holds 2 to 6 less, which all kernels have in common.
// So a large tile does more per time (16 units of 64 x 64 in 1.52 against 1 in 0.25) and a small one leaves fewer compute units
// without work.  Where the tiles are few, workgroups share a tile's sum and a second launch adds up: its time, and the partial sums
// written and read at 4.5 TB/s (bf16: 1 x 16384 x 2048 17 us split and 31 whole, 4096 x 16384 x 1024 131 and 165).  Operands that are
// not aligned may be copied first, at the same rates (bf16: 4750 x 2297 x 4096 121 us copied and 158 through registers, 7 x 2047 x 1001 15 and 11).
struct Kernel { uint32_t id, tm, tn; Access access; float fixed, one[2], two[2]; };
constexpr Kernel kKernels[] = {
    {kFast256, 256, 256, kAligned, 11, {1.52f, 7.33f}, {0, 0}},
    {kFast256x128, 256, 128, kAligned, 6, {0.87f, 3.81f}, {0, 0}},
    {kFast128, 128, 128, kAligned, 4, {0.50f, 1.99f}, {0.93f, 3.78f}},
    {kFast64, 64, 64, kAligned, 2, {0.25f, 0.62f}, {0.37f, 1.07f}},
    {kRows, 0, 64, kAligned, 3, {0.12f, 0.27f}, {0.24f, 0.54f}},
    {kRowsWide, 0, 64, kWide, 3, {0.11f, 0.20f}, {0.42f, 0.70f}},
    {kWide128, 128, 128, kWide, 4, {1.25f, 2.50f}, {1.70f, 4.80f}},
    {kWide64, 64, 64, kWide, 2, {0.80f, 0.72f}, {0.86f, 1.15f}},
    {kAny64, 64, 64, kAny, 2, {2.0f, 2.0f}, {3.0f, 3.0f}},
};
constexpr float kLaunch1 = 6, kBytes = 4.5e6f;                     // a further launch, us; bytes a us

ProductPlan plan_product(const Product& p) {
  ProductPlan plan{};
  const uint32_t size = p.bf16 ? 2 : 4, ks = kStep / size, f32 = !p.bf16;
  const uint32_t e = 16 / size;
  const bool a = aligned(p.a, p.lda, p.batches > 1 ? p.batch_a : 0, p.segs > 1 ? p.seg_a : 0, p.wa, e);
  const bool b = aligned(p.b, p.ldb, p.batches > 1 ? p.batch_b : 0, p.segs > 1 ? p.seg_b : 0, p.wb, e);
  const Access both = a && b ? kAligned : (p.a_kc ? p.K : p.M) >= e && (p.b_kc ? p.K : p.N) >= e ? kWide : kAny;
  plan.steps = (p.K + ks - 1) / ks * p.segs;
  const float out = (float)p.batches * p.M * p.N * 4;
  // operands that are not aligned may be copied so that they are
  const Copy ca = copy_a(p), cb = copy_b(p);
  const uint64_t bytes_a = a ? 0 : (ca.chunks() * size + 255) / 256 * 256, bytes_b = b ? 0 : (cb.chunks() * size + 255) / 256 * 256;
  const bool copies = both != kAligned && ca.pitch < 1u << 21 && cb.pitch < 1u << 21;
  float best = 0;
  for (const Kernel& k : kKernels) {
    const bool copied = k.access == kAligned && both != kAligned;
    if (copied ? !copies : k.access != both) continue;
    const uint32_t tm = k.tm ? k.tm : f32 ? 32 : 16;
    const uint64_t tiles = (uint64_t)((p.M + tm - 1) / tm) * ((p.N + k.tn - 1) / k.tn) * p.batches;
    for (uint32_t splits = 1; splits <= 64; splits = splits == 1 ? 2 : splits & splits - 1 ? splits / 3 * 4 : splits / 2 * 3) {
      const uint32_t per = (plan.steps + splits - 1) / splits;
      if (splits > 1 && (per < 4 || tiles * splits > 1024)) break;
      const float one = k.fixed + per * k.one[f32], two = k.two[0] ? k.fixed + per * k.two[f32] : 2 * one;
      const uint64_t blocks = tiles * splits, rounds = blocks / 512, rest = blocks % 512;
      float t = rounds * two + (rest > 256 ? two : rest ? one : 0);
      if (splits > 1) t += kLaunch1 + (splits + 1) * out / kBytes;
      if (copied) t += kLaunch1 + 2 * (bytes_a + bytes_b) / kBytes;
      if (best && t >= best) continue;
      best = t;
      plan.kernel = k.id == kFast128 && blocks <= 256 ? kFast128Alone : k.id;
      plan.per_split = per;
      plan.splits = per ? (plan.steps + per - 1) / per : 1;
      plan.blocks = tiles * plan.splits;
      plan.copy_a_bytes = copied ? bytes_a : 0;
      plan.copy_b_bytes = copied ? bytes_b : 0;
    }
  }
  plan.partial_bytes = plan.splits > 1 ? (uint64_t)plan.splits * p.batches * p.M * ((p.N + 7) / 8 * 8) * 4 : 0;
  return plan;
}

hipError_t launch_product(const Product& given, const ProductPlan& plan, void* workspace, hipStream_t st) {
  Product p = given;
  if (plan.blocks && plan.copy_a_bytes + plan.copy_b_bytes) {
    Copy a = copy_a(p), b = copy_b(p);
    a.to = workspace;
    b.to = (char*)workspace + plan.copy_a_bytes;
    const uint32_t e = p.bf16 ? 8 : 4;
    const uint64_t chunks_a = plan.copy_a_bytes ? a.chunks() / e : 0, chunks = chunks_a + (plan.copy_b_bytes ? b.chunks() / e : 0);
    const hipError_t err = in_launches((chunks + 255) / 256, [&](uint64_t first, uint32_t n) {
      if (p.bf16) copy_kernel<bf16><<<n, 256, 0, st>>>(a, b, chunks_a, chunks, first);
      else copy_kernel<float><<<n, 256, 0, st>>>(a, b, chunks_a, chunks, first);
    });
    if (err != hipSuccess) return err;
    if (plan.copy_a_bytes) {
      p.a = a.to;
      p.lda = p.wa = a.pitch;
      if (p.batch_a) p.batch_a = (int64_t)a.lines * a.pitch;
      if (p.seg_a) p.seg_a = (int64_t)a.lines * a.pitch;
    }
    if (plan.copy_b_bytes) {
      p.b = b.to;
      p.ldb = p.wb = b.pitch;
      if (p.batch_b) p.batch_b = (int64_t)b.lines * b.pitch;
      if (p.seg_b) p.seg_b = (int64_t)b.lines * b.pitch;
    }
  }
  float* const partial = plan.partial(workspace);
  return p.bf16 ? launch_layout<bf16>(p, plan, partial, st) : launch_layout<float>(p, plan, partial, st);
}

hipError_t launch_rest(const Product* const p[2], const ProductPlan* const plan[2], const float* const partial[2], const GradRows* rows, const float* sums, hipStream_t st) {
  Rest r{};
  uint64_t blocks = 0;
  for (int i = 0; i < 2; i++) {
    if (!p[i] || plan[i]->splits < 2) continue;
    r.p[i] = *p[i];
    r.splits[i] = plan[i]->splits;
    r.partial[i] = partial[i];
    r.blocks[i] = ((uint64_t)p[i]->batches * p[i]->M * ((p[i]->N + 7) / 8) + 255) / 256;
    blocks += r.blocks[i];
  }
  const uint64_t n = rows ? (uint64_t)rows->batches * rows->M : 0;
  const uint32_t each = rows ? grad_rows(n, rows->N) : 0;
  if (rows && rows->dbias && n > each) {
    r.sums = sums;
    r.row_blocks = (uint32_t)((n + each - 1) / each);
    r.N = rows->N;
    r.dbias = rows->dbias;
    r.dbias_bf16 = rows->dbias_bf16;
    r.bias_blocks = (rows->N + 31) / 32;
    blocks += r.bias_blocks;
  }
  return in_launches(blocks, [&](uint64_t first, uint32_t n) { rest_kernel<<<n, 256, 0, st>>>(r, first); });
}

uint64_t grad_rows_bytes(uint32_t batches, uint32_t M, uint32_t N, bool dbias) {
  const uint64_t rows = (uint64_t)batches * M;
  const uint32_t each = grad_rows(rows, N);
  return dbias && rows > each ? (rows + each - 1) / each * N * 4 : 0;
}

hipError_t launch_grad_rows(const GradRows& g, float* partial, hipStream_t st) {
  if (!g.N) return hipSuccess;
  const uint64_t rows = (uint64_t)g.batches * g.M;
  const uint32_t each = grad_rows(rows, g.N);
  const uint64_t row_blocks = rows ? (rows + each - 1) / each : 1;       // (of no rows: dbias is 0)
  return in_launches(row_blocks * ((g.N + 255) / 256), [&](uint64_t first, uint32_t n) {
    grad_rows_kernel<<<n, 256, 0, st>>>(g, each, (uint32_t)first, rows > each ? partial : nullptr);
  });
}

hipError_t launch_drop(const DropRows& d, hipStream_t st) {
  if (!d.M || !d.N) return hipSuccess;
  const uint64_t items = (uint64_t)d.M * ((d.N + 7) / 8);
  return in_launches((items + 255) / 256, [&](uint64_t first, uint32_t n) { drop_kernel<<<n, 256, 0, st>>>(d, first * 256); });
}

}  // namespace mrl
