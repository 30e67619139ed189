// Internal: what the kernels of products share (linear.hip): tiles in shared memory, the way there, the
// order in which workgroups take tiles, and the way of results through the epilogue.
#pragma once
#include <algorithm>

#include "operators.h"

namespace mrl {
namespace {

constexpr int kStep = 128;                 // bytes of a step along k: 64 bf16 or 32 f32
constexpr uint32_t kLaunch = 1u << 22;     // workgroups of a launch, of up to 512 threads: it has fewer than 2^32

// Work of `blocks` workgroups in launches of at most `most`: f(first, count)
template <class F>
hipError_t in_launches(uint64_t blocks, F&& f, uint32_t most = kLaunch) {
  for (uint64_t at = 0; at < blocks; at += most) {
    f(at, (uint32_t)std::min<uint64_t>(most, blocks - at));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// 16 bytes, and eight neighbouring elements, past the caches.
__device__ __forceinline__ void store16_past(void* to, const void* from) {
  typedef uint32_t words __attribute__((ext_vector_type(4), aligned(2)));
  words w;
  __builtin_memcpy(&w, from, 16);
  __builtin_nontemporal_store(w, (words*)to);
}
// Bytes that are there of 16, given the elements of 2^shift bytes that are left of the row: up to 2^31 of them, whose bytes 32 bits do not hold.
constexpr __host__ __device__ uint32_t bytes_there(uint32_t left, uint32_t shift) { return (left < 16u >> shift ? left : 16u >> shift) << shift; }
static_assert(bytes_there(1u << 30, 2) == 16 && bytes_there((1u << 30) + 3, 2) == 16 && bytes_there(0x7FFFFFFF, 1) == 16 && bytes_there(3, 2) == 12 && bytes_there(7, 1) == 14 &&
              bytes_there(0, 1) == 0, "");
template <class T>
__device__ __forceinline__ void store8_past(T* p, const float (&v)[8]) {
  T t[8];
#pragma unroll
  for (int e = 0; e < 8; e++) t[e] = (T)v[e];
#pragma unroll
  for (uint32_t i = 0; i < sizeof t / 16; i++) store16_past((char*)p + 16 * i, (const char*)t + 16 * i);
}
// Whether the results of layer_norm and of products go there, by their bytes: 11 to 32 MB, which would all lie in the dies' caches at the end and be written back before the next
// launch, and 256 MB and more, which the cache at the memory does not hold; between the two the reader loses more than is gained.  Past and not, alone, and with mx_quantize of the
// results behind it, in us, operands from memory (those that are in a cache gain a little more):
//   layer_norm, rows of 2048 in bf16:  6 MB  5.7  6.0  10.8 11.3;  11 MB 8.8 9.2  14.8 16.8;  16 MB 11.0 11.6  18.4 18.4;  24 MB 13.9 14.6  22.1 23.0;  32 MB 17.2 17.4  26.8 25.9;
//                                      64 MB 29.4 27.5  46.3 42.1;  128 MB 48 47  85 73;  256 MB 111 109  177 171;  320 MB 140 140  221 222
//   mx_linear, k = 512, 4096 columns:  6 MB  7.1  7.3  12.5 12.9;  11 MB 8.6 9.2  15.8 17.0;  16 MB  9.0 10.3  19.9 22.1;  24 MB 12.3 13.5  25.1 25.3;  32 MB 13.9 15.3  28.2 27.3;
//                                      64 MB 28.5 25.9  45.2 41.9;  128 MB 45 41  76 67;  256 MB 81.5 77.0  145 146;  320 MB 96 96  172 200
// So at 32 MB a reader loses 3 %, about what the writer gains, and the gain does not end at 11 MB.  8192 x 2048 x 16384 (256 MB, several tiles a workgroup) 210 and 242, 297 and 306.
constexpr uint64_t kCaches = 32ull << 20, kBeyond = 256ull << 20;
__device__ __forceinline__ bool goes_past(uint64_t bytes) { return (bytes >= kCaches / 3 && bytes <= kCaches) || bytes >= kBeyond; }

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

// ---- workgroups and results

// Where a workgroup's tile lies.
struct Place { uint32_t tm, tn, split, batch; };
// Workgroups go to the eight dies in turn, each with an L2 of its own: a die gets a stretch of consecutive tiles, and
// consecutive tiles are kGroup rows of tiles high, so that the tiles that are worked on at once share rows and columns there.
constexpr uint32_t kDies = 8, kGroup = 8;
__device__ __forceinline__ Place place_of(uint32_t id, uint32_t tiles_m, uint32_t tiles_n, uint32_t splits) {
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
// A workgroup's stretch of `tiles`: those of its die from `id` to before `end`, of which it takes every `every`-th.
struct Stretch {
  uint32_t id, end, every;
  __device__ __forceinline__ Stretch(uint32_t first, uint32_t tiles) {
    const uint32_t die = blockIdx.x % kDies, each = tiles / kDies, rest = tiles % kDies;
    id = first + die * each + min(die, rest);
    end = id + each + (die < rest);
    id += blockIdx.x / kDies;
    every = gridDim.x / kDies + (die < gridDim.x % kDies);       // the workgroups of the die
  }
};
__device__ __forceinline__ Place place(uint32_t first, uint32_t tiles_m, uint32_t tiles_n, uint32_t splits) {
  return place_of(Stretch(first, gridDim.x).id, tiles_m, tiles_n, splits);
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

}  // namespace
}  // namespace mrl
