// Microscaled 4-bit floating point (operators.h): values to blocks of 32 along k and back, and the product of
// operands in such blocks, whose scales the matrix instructions apply.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "tiles.h"

namespace mrl {
namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x8 __attribute__((ext_vector_type(8)));

// The scale byte of a block whose largest magnitude is `most`, as bits of an f32 (finite): floor(log2) - 2, biased.  A magnitude below 2^-126
// has no exponent of its own there, and the byte of any below 2^-124 is 0.
__device__ __forceinline__ uint32_t scale_of(uint32_t most) { return max((int32_t)(most >> 23) - 2, 0); }
__device__ __forceinline__ float power_of(uint32_t scale) { return __uint_as_float(scale ? scale << 23 : 1u << 22); }       // 2^(scale - 127)

// Eight values' codes, divided by the scale, rounded to the nearest (ties to the even code) and kept within 6 by the conversion.
__device__ __forceinline__ uint32_t codes8(const float (&v)[8], float power) {
  uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, v[0], v[1], power, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], power, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], power, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], power, 3);
}

// Where the scale of a line of a group of 64 and of block g of a step lies in their 256 bytes.
__device__ __forceinline__ uint32_t scale_at(uint32_t line, uint32_t g) {
  return ((g * 16 + (line >> 3 & 3) * 4 + (line & 3)) << 2) + (line >> 5) * 2 + (line >> 2 & 1);
}

// What a workgroup quantises or reads back: 64 lines by a step of 128 values.  Lanes take eight neighbouring values of a line, sixteen lanes a line.
struct Tile64 {
  uint32_t s, group, batch;                // step, group of lines, batch
  uint64_t scales;                         // where the tile's 256 bytes of scales lie
  __device__ __forceinline__ Tile64(const MxRows& p, uint64_t id, bool shared) {
    const uint32_t steps = mx_steps(p.k), groups = (p.lines + 63) / 64;
    const uint64_t outer = id / steps;
    s = (uint32_t)(id - outer * steps);
    batch = (uint32_t)(outer / groups);
    group = (uint32_t)(outer - (uint64_t)batch * groups);
    scales = (((uint64_t)(shared ? 0 : batch) * groups + group) * steps + s) * 256;
  }
};
// The codes of a line's step.
__device__ __forceinline__ uint8_t* codes_of(const MxRows& p, uint32_t batch, uint32_t line, uint32_t s) {
  const uint32_t steps = mx_steps(p.k);
  return p.codes + (((uint64_t)batch * p.lines + line) * steps + s) * 64;
}

// The largest of four lanes'.
__device__ __forceinline__ uint32_t max4(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true));        // lanes 1, 0, 3, 2
  return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, true));     // lanes 2, 3, 0, 1
}

// Eight neighbouring values of a line of K, K at least 8, without a branch that a load would wait for: a chunk that ends past the line is read from the line's
// last eight and moved down, zeros behind it.
template <class T> struct Eight {
  T t[8];
  __device__ __forceinline__ void load(const T* line, uint32_t k, uint32_t K) { __builtin_memcpy(t, line + min(k, K - 8), sizeof t); }
  __device__ __forceinline__ void values(uint32_t k, uint32_t K, float (&v)[8]) const {
    const uint32_t past = k + 8 > K ? k + 8 - K : 0;
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = (float)t[e];
    if (K % 8) {
#pragma unroll
      for (int by = 1; by < 8; by *= 2)
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = past & by ? (e + by < 8 ? v[e + by] : 0.0f) : v[e];
    }
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = past >= 8 ? 0.0f : v[e];
  }
};

// Lines whose neighbours along k are adjacent: four lanes share a block.
template <class T>
__global__ __launch_bounds__(256) void mx_quantize_kernel(const MxRows p, uint64_t first) {
  __shared__ __attribute__((aligned(4))) uint8_t scales[256];
  const Tile64 at(p, first + blockIdx.x, false);
  const uint32_t c = threadIdx.x & 15, l0 = threadIdx.x >> 4, k = at.s * 128 + c * 8;
  const T* const x = (const T*)p.x.data + (int64_t)at.batch * p.x.batch;
  float v[4][8];
  if (p.k >= 8) {
    Eight<T> t[4];
#pragma unroll
    for (uint32_t i = 0; i < 4; i++) t[i].load(x + (int64_t)min(at.group * 64 + i * 16 + l0, p.lines - 1) * p.x.ld, k, p.k);
#pragma unroll
    for (uint32_t i = 0; i < 4; i++) t[i].values(at.group * 64 + i * 16 + l0 < p.lines ? k : p.k, p.k, v[i]);
  } else {
#pragma unroll
    for (uint32_t i = 0; i < 4; i++) {
      const uint32_t line = at.group * 64 + i * 16 + l0;
      load8(x + (int64_t)line * p.x.ld + k, line < p.lines && k < p.k ? p.k - k : 0, v[i]);
    }
  }
#pragma unroll
  for (uint32_t i = 0; i < 4; i++) {
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 8; e++) most = max(most, __float_as_uint(v[i][e]) & 0x7FFFFFFFu);
    most = max4(most);
    const bool finite = most < 0x7F800000u;
    const uint32_t scale = finite ? scale_of(most) : 255, l = i * 16 + l0, line = at.group * 64 + l;
    if ((c & 3) == 0) scales[scale_at(l, c >> 2)] = (uint8_t)scale;
    const uint32_t codes = finite ? codes8(v[i], power_of(scale)) : 0;
    if (line < p.lines) *(uint32_t*)(codes_of(p, at.batch, line, at.s) + c * 4) = codes;
  }
  __syncthreads();
  if (threadIdx.x < 64) *(uint32_t*)(p.scales + at.scales + threadIdx.x * 4) = *(const uint32_t*)(scales + threadIdx.x * 4);
}

// Lines that are adjacent (a matrix k x lines that is row-major): the tile comes row by row, 16 bytes a lane, and goes through shared memory, from
// which a thread takes a block; so do the codes, so that a line's 64 bytes are stored side by side.
template <class T>
__global__ __launch_bounds__(256) void mx_quantize_across_kernel(const MxRows p, uint64_t first) {
  constexpr uint32_t E = 16 / sizeof(T), PER = 64 / E, ROWS = 256 / PER;     // elements of a load, loads of a row of 64 lines, rows at a time
  __shared__ __attribute__((aligned(16))) T tile[128][64];
  __shared__ __attribute__((aligned(16))) u32x4 codes[64][5];                // (a place more a line, against bank conflicts)
  __shared__ __attribute__((aligned(4))) uint8_t scales[256];
  const Tile64 at(p, first + blockIdx.x, false);
  const uint32_t k0 = at.s * 128, line0 = at.group * 64, c = threadIdx.x % PER * E, r0 = threadIdx.x / PER;
  const T* const x = (const T*)p.x.data + (int64_t)at.batch * p.x.batch + line0 + c;
  const uint32_t there = line0 + c < p.lines ? p.lines - line0 - c : 0;
  u32x4 v[128 / ROWS];
#pragma unroll
  for (uint32_t i = 0; i < 128 / ROWS; i++) {
    const uint32_t k = k0 + i * ROWS + r0;
    const T* const from = x + (int64_t)k * p.x.ld;
    const uint32_t valid = k < p.k ? there : 0;
    if (valid >= E) {
      __builtin_memcpy(&v[i], from, 16);
    } else {
      T t[E];
#pragma unroll
      for (uint32_t e = 0; e < E; e++) t[e] = e < valid ? from[e] : (T)0.0f;
      __builtin_memcpy(&v[i], t, 16);
    }
  }
#pragma unroll
  for (uint32_t i = 0; i < 128 / ROWS; i++) *(u32x4*)&tile[i * ROWS + r0][c] = v[i];
  __syncthreads();
  const uint32_t l = threadIdx.x & 63, g = threadIdx.x >> 6;
  float w[4][8];
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 32; i++) {
    w[i / 8][i % 8] = (float)tile[g * 32 + i][l];
    most = max(most, __float_as_uint(w[i / 8][i % 8]) & 0x7FFFFFFFu);
  }
  const bool finite = most < 0x7F800000u;
  const uint32_t scale = finite ? scale_of(most) : 255;
  scales[scale_at(l, g)] = (uint8_t)scale;
  u32x4 q = {0, 0, 0, 0};
  if (finite) {
#pragma unroll
    for (int i = 0; i < 4; i++) q[i] = codes8(w[i], power_of(scale));
  }
  codes[l][g] = q;
  __syncthreads();
  const uint32_t line = threadIdx.x >> 2, part = threadIdx.x & 3;
  if (line0 + line < p.lines) *(u32x4*)(codes_of(p, at.batch, line0 + line, at.s) + part * 16) = codes[line][part];
  if (threadIdx.x < 64) *(uint32_t*)(p.scales + at.scales + threadIdx.x * 4) = *(const uint32_t*)(scales + threadIdx.x * 4);
}

// Blocks to values: 16 bytes of values a lane, so that a wave stores 1024 side by side (in f32 32 bytes a lane, in two halves, 49 us for 2048 x 16384).
template <class T>
__global__ __launch_bounds__(256) void mx_dequantize_kernel(const MxRows p, uint64_t first) {
  constexpr uint32_t E = 16 / sizeof(T), LANES = 128 / E, N = 64 * LANES / 256;        // values of a lane, lanes of a line, lines of a thread
  const Tile64 at(p, first + blockIdx.x, p.shared);
  const uint32_t c = threadIdx.x % LANES, l0 = threadIdx.x / LANES, k = at.s * 128 + c * E;
  if (k >= p.k) return;
  uint32_t codes[N], scale[N];
#pragma unroll
  for (uint32_t i = 0; i < N; i++) {
    const uint32_t line = min(at.group * 64 + i * (256 / LANES) + l0, p.lines - 1);
    const uint8_t* const from = codes_of(p, p.shared ? 0 : at.batch, line, at.s) + c * (E / 2);
    codes[i] = E == 8 ? *(const uint32_t*)from : *(const uint16_t*)from;
    scale[i] = p.scales[at.scales + scale_at(line & 63, c / (32 / E))];
  }
  T* const x = (T*)p.x.data + (int64_t)at.batch * p.x.batch + k;
  const bool past = (uint64_t)p.batches * p.lines * p.k * sizeof(T) >= kBeyond;        // (up to 32 MB it makes no difference here)
#pragma unroll
  for (uint32_t i = 0; i < N; i++) {
    const uint32_t line = at.group * 64 + i * (256 / LANES) + l0;
    if (line >= p.lines) break;
    const float power = power_of(scale[i]);
    f32x2 t[E / 2];
    t[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[i], power, 0);
    t[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[i], power, 1);
    if constexpr (E == 8) {
      t[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[i], power, 2);
      t[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[i], power, 3);
    }
    T v[E];
#pragma unroll
    for (uint32_t e = 0; e < E; e++) v[e] = (T)(scale[i] == 255 ? __uint_as_float(0x7FC00000u) : t[e / 2][e % 2]);
    T* const to = x + (int64_t)line * p.x.ld;
    if (p.k - k >= E) {
      if (past) store16_past(to, v);
      else __builtin_memcpy(to, v, 16);
    } else {
#pragma unroll
      for (uint32_t e = 0; e < E; e++)
        if (e < p.k - k) to[e] = v[e];
    }
  }
}

// acc += a's block of 16 lines times b's over 128 values; sa and sb hold four blocks' scales, byte by byte.
template <int OA, int OB>
__device__ __forceinline__ f32x4 multiply(const i32x4& a, const i32x4& b, uint32_t sa, uint32_t sb, const f32x4& acc) {
  const i32x8 x = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, y = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(y, x, acc, 4, 4, OB, (int)sb, OA, (int)sa);       // (4: both operands are 4-bit floating point)
}

// The same with places that are known once loops are unrolled.
__device__ __forceinline__ f32x4 multiply(const bf16x8& a, const bf16x8& b, uint32_t sa, uint32_t sb, int oa, int ob, const f32x4& acc) {
  const i32x4 x = __builtin_bit_cast(i32x4, a), y = __builtin_bit_cast(i32x4, b);
  switch (oa * 4 + ob) {
    case 0: return multiply<0, 0>(x, y, sa, sb, acc);
    case 1: return multiply<0, 1>(x, y, sa, sb, acc);
    case 2: return multiply<0, 2>(x, y, sa, sb, acc);
    case 3: return multiply<0, 3>(x, y, sa, sb, acc);
    case 4: return multiply<1, 0>(x, y, sa, sb, acc);
    case 5: return multiply<1, 1>(x, y, sa, sb, acc);
    case 6: return multiply<1, 2>(x, y, sa, sb, acc);
    case 7: return multiply<1, 3>(x, y, sa, sb, acc);
    case 8: return multiply<2, 0>(x, y, sa, sb, acc);
    case 9: return multiply<2, 1>(x, y, sa, sb, acc);
    case 10: return multiply<2, 2>(x, y, sa, sb, acc);
    case 11: return multiply<2, 3>(x, y, sa, sb, acc);
    case 12: return multiply<3, 0>(x, y, sa, sb, acc);
    case 13: return multiply<3, 1>(x, y, sa, sb, acc);
    case 14: return multiply<3, 2>(x, y, sa, sb, acc);
    default: return multiply<3, 3>(x, y, sa, sb, acc);
  }
}

// 256 bytes from memory to shared memory, four a lane.
__device__ __forceinline__ void load4_to_lds(uint32_t lds, uint32_t offset, u32x4 buffer) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(offset), "s"(buffer) : "memory");
}

// A step is 256 values, 128 bytes of codes a line, so tiles lie in shared memory and get there as those of two-byte operands do; a half step is one
// instruction's 128 values.  Both operands' lines are in the order that the products of linear.hip have for B, which is the one that scales are stored in.
constexpr uint32_t kUnits = 64;            // of four values, in a step

// The scales of a tile of `groups` groups of 64 lines: 256 bytes for a group and half step.
struct Scales {
  u32x4 buffer;
  __device__ __forceinline__ Scales(const uint8_t* scales, uint32_t line, uint32_t lines, uint32_t pitch, uint32_t groups) {
    const uint64_t base = (uint64_t)(scales + (uint64_t)(line / 64) * pitch);
    buffer = u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)base), (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(base >> 32) & 0xFFFFu),
                   (uint32_t)__builtin_amdgcn_readfirstlane(min(groups, (lines + 63) / 64 - line / 64) * pitch), 0x27000u};
  }
};
constexpr uint32_t kNoHalf = 0x400000;     // beyond any half step
// The 256 bytes of a group and a step's first half step (odd = 0) or second (1), as a wave loads them.  A half step that is not there has scales of 0
// (2^-127): the byte that happens to follow could be a NaN's.  (Worked out without a branch: with one the loop's products were moved behind its barrier, and a step of
// 256 x 256 x 256 took 1.88 us instead of 1.70.)
struct Slot {
  uint32_t offset, odd, halves;
  __device__ __forceinline__ void init(uint32_t pitch, uint32_t group, uint32_t half, uint32_t lane) {
    odd = half;
    halves = pitch / 256;
    offset = group * pitch + lane * 4;
  }
  __device__ __forceinline__ void load(uint32_t half, uint32_t lds, u32x4 buffer) const { load4_to_lds(lds, half + odd < halves ? offset + (half + odd) * 256 : kOutside, buffer); }
};

// A wave's scales of W of a tile's lines from `first` on, for a half step: four blocks a word.
template <int W>
__device__ __forceinline__ void read_scales(lds_ptr slots, uint32_t first, uint32_t kk, uint32_t lane, uint32_t (&s)[(W + 63) / 64]) {
#pragma unroll
  for (uint32_t i = 0; i < (W + 63) / 64; i++) s[i] = *(const __attribute__((address_space(3))) uint32_t*)(slots + ((first / 64 + i) * 2 + kk) * 256 + lane * 4);
  if (W < 64) s[0] >>= first % 64 / 16 * 8;
}

// A wave's results.  A lane has row row_of(i, q) and, of the pair of blocks 2 j, 2 j + 1, the eight columns from 32 j + 8 g on; they are finished in its registers
// and go 16 rows of 128 bytes at a time through shared memory that is the wave's own (16-byte chunks, at their number xor the row's, against bank conflicts), so
// that neighbouring lanes store neighbouring bytes.  As sums, before the epilogue (write_out of tiles.h), 4096 x 16384 x 2048 with a residual took 85 us instead of 75, 8192 x 2048 x 16384 177
// instead of 171; with halves changed between lanes eight apart instead, whole lines but in another order of lanes, rows that start at odd elements take an eighth longer.
constexpr uint32_t kOut = 16 * 128;
template <int BM, int BN>
__device__ __forceinline__ void store_results(const Product& p, const Place& at, uint32_t splits, uint32_t m0, uint32_t n0, uint32_t lane, const f32x4 (&acc)[BM][BN],
                                              char* mine, float* __restrict__ partial) {
  constexpr int PAIRS = BN / 2;
  const Epilogue& e = p.e;
  const uint32_t q = lane & 15, g = lane >> 4, n = n0 + 8 * g;
  const uint32_t pitch = (p.N + 7) & ~7u;
  const RowsOf out = splits > 1 ? RowsOf{partial + (uint64_t)at.split * p.batches * p.M * pitch, pitch, (int64_t)p.M * pitch, 0} : e.out;
  const bool ends = splits == 1, residual = ends && e.residual.data, past = ends && goes_past((uint64_t)p.batches * p.M * p.N << (out.bf16 ? 1 : 2));
  const uint32_t activation = ends ? e.activation : 0, out_shift = out.bf16 ? 1 : 2, width = ends ? p.N : pitch;
  const auto valid = [&](uint32_t column) { return column < width ? width - column : 0; };
  float bias[PAIRS][8];
#pragma unroll
  for (int j = 0; j < PAIRS; j++) {
    if (ends) bias8(e, n + 32 * j, valid(n + 32 * j), bias[j]);
    else
#pragma unroll
      for (int k = 0; k < 8; k++) bias[j][k] = 0.0f;
  }
  const char* from = (const char*)e.residual.data + (((int64_t)at.batch * e.residual.batch + (int64_t)m0 * e.residual.ld + n) << (e.residual.bf16 ? 1 : 2));
  char* to = (char*)out.data + (((int64_t)at.batch * out.batch + (int64_t)m0 * out.ld + n0) << out_shift);
  const auto store = [&](uint32_t row, uint32_t column, const uint32_t (&w)[4]) {       // 16 bytes
    const uint32_t left = bytes_there(valid(n0 + column), out_shift);
    if (m0 + row >= p.M) return;
    char* here = to + (((int64_t)row * out.ld + column) << out_shift);
    if (left >= 16) {
      if (past) store16_past(here, w);
      else __builtin_memcpy(here, w, 16);
    } else {
#pragma unroll
      for (uint32_t k = 0; k < 4; k++) {
        if (4 * k + 4 <= left) __builtin_memcpy(here + 4 * k, &w[k], 4);
        else if (4 * k + 2 <= left) __builtin_memcpy(here + 4 * k, &w[k], 2);
      }
    }
  };
#pragma unroll
  for (int i = 0; i < BM; i++) {
    const uint32_t row = row_of<bf16, true>(i, q);
    float v[PAIRS][8];
#pragma unroll
    for (int j = 0; j < PAIRS; j++)
#pragma unroll
      for (int k = 0; k < 8; k++) v[j][k] = acc[i][2 * j + k / 4][k % 4] + bias[j][k];
    const auto activate = [&](uint32_t act) {
#pragma unroll
      for (int j = 0; j < PAIRS; j++) activate8(act, v[j]);
    };
    if (activation == kActRelu) activate(kActRelu);
    else if (activation == kActGelu) activate(kActGelu);
    else if (activation == kActSilu) activate(kActSilu);
    if (residual && m0 + row < p.M) {
      float y[PAIRS][8];
#pragma unroll
      for (int j = 0; j < PAIRS; j++) load8(from, e.residual.bf16, (int64_t)row * e.residual.ld + 32 * j, valid(n + 32 * j), y[j]);
#pragma unroll
      for (int j = 0; j < PAIRS; j++)
#pragma unroll
        for (int k = 0; k < 8; k++) v[j][k] += y[j][k];
    }
    // 16 rows of eight chunks of 16 bytes (four, where the wave has no more columns), and of those what a lane stores
    const auto put = [&](uint32_t chunk, const uint32_t (&w)[4]) { __builtin_memcpy(mine + (q * 8 + (chunk ^ (q & 7))) * 16, w, 16); };
    const auto go = [&](uint32_t column, uint32_t chunks) {
      asm volatile("" ::: "memory");
#pragma unroll
      for (uint32_t h = 0; h < 2; h++) {
        if (h * 64 >= 16 * chunks) break;
        const uint32_t r = (lane + h * 64) / chunks, c = lane % chunks;
        uint32_t w[4];
        __builtin_memcpy(w, mine + (r * 8 + (c ^ (r & 7))) * 16, 16);
        store(row_of<bf16, true>(i, r), column + c * (out.bf16 ? 8 : 4), w);
      }
      asm volatile("" ::: "memory");
    };
    if (out.bf16) {
#pragma unroll
      for (int j = 0; j < PAIRS; j++) {
        bf16 t[8];
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 8; k++) t[k] = (bf16)v[j][k];
        __builtin_memcpy(w, t, 16);
        put(j % 2 * 4 + g, w);
        if (j % 2 || PAIRS == 1) go(32 * (j & ~1), PAIRS == 1 ? 4 : 8);
      }
    } else {
#pragma unroll
      for (int j = 0; j < PAIRS; j++) {
        uint32_t w[2][4];
        __builtin_memcpy(w, v[j], 32);
        put(2 * g, w[0]);
        put(2 * g + 1, w[1]);
        go(32 * j, 8);
      }
    }
    __builtin_amdgcn_sched_barrier(0);     // (or the next rows' values are worked out first, and kept)
  }
}

// The arguments lie in memory.  All their lines are asked for at once here: as the compiler has it, a few at a time where they are used, several trips there follow each
// other (8192 x 2048 x 16384 197 us instead of 195, 4096^3 0.7 us more).
__device__ __forceinline__ void ask_for(const MxProduct& x) {
  constexpr int LINES = (sizeof(MxProduct) + 63) / 64;
  uint32_t w[6];
  static_assert(LINES == 6, "a word of each line");
#pragma unroll
  for (int i = 0; i < LINES; i++) __builtin_memcpy(&w[i], (const char*)&x + i * 64, 4);
  asm volatile("" ::"s"(w[0]), "s"(w[1]), "s"(w[2]), "s"(w[3]), "s"(w[4]), "s"(w[5]));
  __builtin_amdgcn_sched_barrier(0);
}

// What store_results needs of a product in the arguments' memory.
typedef const __attribute__((address_space(4))) Product& product_ref;
__device__ __forceinline__ Product results_of(product_ref p) {
  const auto rows = [](const __attribute__((address_space(4))) RowsOf& r) { return RowsOf{r.data, r.ld, r.batch, r.bf16}; };
  Product by{};
  by.batches = p.batches;
  by.M = p.M;
  by.N = p.N;
  by.e.out = rows(p.e.out);
  by.e.residual = rows(p.e.residual);
  by.e.bias = p.e.bias;
  by.e.bias_bf16 = p.e.bias_bf16;
  by.e.activation = p.e.activation;
  return by;
}

// Tiles of TM x TN, WAVES_M x WAVES_N waves, STAGES steps in shared memory: the loop of linear.hip's fast_kernel.  A wave of the 256 tile has 128 x 64.  Where there are
// more tiles than run at once, a workgroup has several (two stages: only then every wait of the loop is for all loads under way, results among them): the last steps of a
// tile load the first ones of the next, and its results leave meanwhile.
//
// 8192-cube 252 us, 4360 TFLOP/s, where the matrix units sustain 7600 on operands like these: they are busy 54 % of its cycles, at 1.9 GHz, shared memory 25 %.  8192 x 2048 x 16384 with GELU
// from blocks, one behind the other, 202 us: 162 without the activation (an exponential and a reciprocal are a quarter of the rate), 115 without results, whose 268 MB are 52 us of memory's
// time; a call that puts lhs into blocks before it takes 197 to 203 in all, and 8 % more with a workgroup a tile.  4096 x 16384 x 2048 with f32 results and a residual 77 us, 65 without results.  Half steps twice as many ahead (64 bytes of a line at a time) took 274 us for the cube where this took 247; the second of two smaller workgroups a
// compute unit started half a tile later, or lines asked for steps before, changed nothing or cost time.
template <int TM, int TN, int WAVES_M, int WAVES_N, int STAGES>
__global__ __launch_bounds__(64 * WAVES_M * WAVES_N, 2) void mx_tile_kernel(const MxProduct x, uint32_t steps, uint32_t per_split, uint32_t splits, uint32_t first,
                                                                         uint32_t tiles) {
  constexpr int WAVES = WAVES_M * WAVES_N, THREADS = 64 * WAVES, WM = TM / WAVES_M, WN = TN / WAVES_N, BM = WM / 16, BN = WN / 16;
  constexpr int GA = TM / 64, GB = TN / 64, SLOTS = 2 * (GA + GB), EACH = (SLOTS + WAVES - 1) / WAVES;       // 256 bytes of scales; and how many a wave loads
  constexpr uint32_t CODES = (TM + TN) * kStep, STAGE = CODES + EACH * WAVES * 256;
  constexpr bool MORE = STAGES == 2;       // a workgroup may have several tiles
  __shared__ __attribute__((aligned(1024))) char lds[STAGES * STAGE + (MORE ? WAVES * kOut : 0)];
  const Product& p = x.p;

  ask_for(x);
  const uint32_t tiles_m = (p.M + TM - 1) / TM, tiles_n = (p.N + TN - 1) / TN;
  Stretch mine(first, tiles);
  Place at = place_of(mine.id, tiles_m, tiles_n, splits);
  const uint32_t t = threadIdx.x, lane = t & 63, q = lane & 15, g = lane >> 4;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const uint32_t wm = wave / WAVES_N * WM, wn = wave % WAVES_N * WN;

  Feed<bf16, true, true, TM, THREADS> fa;
  Feed<bf16, true, true, TN, THREADS> fb;
  fa.init(p.lda, t);
  fb.init(p.ldb, t);
  const uint32_t from = at.split * per_split, end = min(from + per_split, steps), n = end > from ? end - from : 0;
  const uint32_t pitch = p.K / 32 * 256;   // bytes of scales from 64 lines to the next
  Slot slots[EACH];                // first A's groups, two half steps each, then B's
  static_assert(2 * GA % EACH == 0, "a wave has slots of one operand");
#pragma unroll
  for (int i = 0; i < EACH; i++) {
    const uint32_t slot = wave * EACH + i, group = slot / 2;
    slots[i].init(pitch, group < GA ? group : group - GA, slot < SLOTS ? slot & 1 : kNoHalf, lane);
  }
  // the step to load next and the one that its tile ends before, where that starts in either operand, the bytes that are left behind that, the scales
  uint32_t step, till;
  const char *ca, *cb;
  int64_t left_a, left_b;
  u32x4 scales;
  const auto begin = [&](const Place& at) {
    const uint32_t m0 = at.tm * TM, n0 = at.tn * TN;
    step = from;
    till = end;
    ca = (const char*)p.a + ((int64_t)at.batch * p.batch_a + (int64_t)m0 * p.lda + (int64_t)from * kUnits) * 2;
    cb = (const char*)p.b + ((int64_t)at.batch * p.batch_b + (int64_t)n0 * p.ldb + (int64_t)from * kUnits) * 2;
    left_a = ((int64_t)(p.M - m0) * p.lda - (int64_t)from * kUnits) * 2;
    left_b = ((int64_t)(p.N - n0) * p.ldb - (int64_t)from * kUnits) * 2;
    const bool of_a = wave * EACH < 2 * GA;
    scales = Scales((of_a ? x.scales_a : x.scales_b) + (int64_t)at.batch * (of_a ? x.scales_batch_a : x.scales_batch_b), of_a ? m0 : n0, of_a ? p.M : p.N, pitch, of_a ? GA : GB).buffer;
  };
  begin(at);
  constexpr int NA = decltype(fa)::N, NB = decltype(fb)::N, LOADS = NA + NB + EACH;

  // (behind the last step the buffers have no bytes: zeros are written that nothing uses, and every step has the same loads under way)
  u32x4 buf_a, buf_b, buf_s;
  uint32_t to, half;
  const auto aim = [&](uint32_t stage) {          // at the next step, to be put into `stage`
    const bool more = step < till;
    to = (uint32_t)(uintptr_t)(lds_ptr)lds + stage * STAGE;
    half = more ? step * 2 : kNoHalf;
    buf_a = fa.buffer(ca, more ? left_a : 0);
    buf_b = fb.buffer(cb, more ? left_b : 0);
    buf_s = scales;                // (the last loads of a step may go out when the next tile has begun)
    const uint32_t on = more ? kStep : 0;
    step += more;
    ca += on;
    cb += on;
    left_a -= on;
    left_b -= on;
  };
  const auto load = [&](int i) {
    // (Of a last half step that is not there the next line's codes come.  They are finite and their scales 2^-127 each, so that their products are less than half of any
    // sum's last bit, which is 2^-149 at least.  Left out by a comparison and two selections a load, 8192^3 took 254 us instead of 252, 4096 x 16384 x 2048 71.6 instead of 69.5.)
    if (i < NA) load_to_lds(to + wave * 1024 + i * THREADS * 16, fa.offset[i], buf_a);
    else if (i < NA + NB) load_to_lds(to + TM * kStep + wave * 1024 + (i - NA) * THREADS * 16, fb.offset[i - NA], buf_b);
    else slots[i - NA - NB].load(half, to + CODES + (wave * EACH + (i - NA - NB)) * 256, buf_s);
  };
  constexpr int NM = BM > 4 ? BM / 2 : BM, PHASES = 2 * BM / NM;
  // (4096 x 16384 x 2048 by tiles of 256 x 128 83 us with a step's loads all at once, 77 spread)
  constexpr bool SPREAD = LOADS <= PHASES * NM;      // one beside a part of the products
  bf16x8 oa[2][NM], ob[2][BN];
  uint32_t ka[2][(WM + 63) / 64], kb[2][(WN + 63) / 64];
  const auto read_a = [&](lds_ptr stage, int m, int kk, bf16x8 (&o)[NM]) { read_blocks<bf16, true, true, TM>(stage, wm, m, kk, q, g, o); };
  const auto read_b = [&](lds_ptr stage, int kk) {        // and the scales of the half step
    read_blocks<bf16, true, true, TN>(stage + TM * kStep, wn, 0, kk, q, g, ob[kk]);
    read_scales<WM>(stage + CODES, wm, kk, lane, ka[kk]);
    read_scales<WN>(stage + CODES + 2 * GA * 256, wn, kk, lane, kb[kk]);
  };
  if (n) {
#pragma unroll
    for (int s = 0; s < STAGES; s++) {
      aim(s);
#pragma unroll
      for (int i = 0; i < LOADS; i++) load(i);
    }
    arrive<(STAGES - 1) * LOADS>();
  }
  uint32_t cur = 0;
  for (;;) {
    const bool more = MORE && mine.id + mine.every < mine.end;
    f32x4 acc[BM][BN];
#pragma unroll
    for (int i = 0; i < BM; i++)
#pragma unroll
      for (int j = 0; j < BN; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (n) {
      read_a((lds_ptr)lds + cur * STAGE, 0, 0, oa[0]);
      read_b((lds_ptr)lds + cur * STAGE, 0);
    }
    // (the last steps load the next tile's first ones.  Which tile that is is found between two runs of one loop: selected inside it, 8192^3 took 309 us instead of 257)
    const uint32_t early = n - min(n, (uint32_t)STAGES);
    Place behind = at;
#pragma unroll 1
    for (uint32_t last = 0; last < (MORE ? 2 : 1); last++) {
      for (uint32_t s = MORE ? last ? n - early : early : n; s; s--) {
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
          read_a(stage, m, kk, oa[then & 1]);
          if (m == 0) read_b(stage, kk);
          if (WM >= 64 && WN >= 64) __builtin_amdgcn_sched_barrier(0);      // (the scales of fewer lines are shifted, which would be waited for here)
          __builtin_amdgcn_s_setprio(1);        // (a wave with products goes first; without, 8192^3 takes 1 % longer)
#pragma unroll
          for (int part = 0; part < NM; part++) {
            const int i = ph % (PHASES / 2) * NM + part, k = ph / (PHASES / 2);
#pragma unroll
            for (int j = 0; j < BN; j++) acc[i][j] = multiply(oa[ph & 1][part], ob[k][j], ka[k][i / 4], kb[k][j / 4], i % 4, j % 4, acc[i][j]);
            // (in the first step, before its barrier, the last stage's loads again: the same bytes to the same place)
            if (SPREAD && then * NM + part < LOADS) {
              load(then * NM + part);
              __builtin_amdgcn_sched_barrier(0);
            }
          }
          __builtin_amdgcn_s_setprio(0);
          __builtin_amdgcn_sched_barrier(0);
        }
        cur = next;
      }
      if (MORE && !last) {
        mine.id += mine.every;
        till = from;
        if (more) begin(behind = place_of(mine.id, tiles_m, tiles_n, splits));
      }
    }
    if (!MORE && n) arrive<0>();    // nothing is under way to shared memory where the results go
    // the arguments and the lane are asked for anew: what is worked out of them for the results would be kept in registers beside the products, and a scalar load that
    // could still be under way makes every wait for a read of shared memory one for all of them
    auto again = (const __attribute__((address_space(4))) MxProduct*)__builtin_amdgcn_kernarg_segment_ptr();
    uint32_t own = lane;
    asm volatile("" : "+s"(again), "+v"(own));
    store_results(results_of(again->p), at, splits, at.tm * TM + wm, at.tn * TN + wn, own, acc, lds + (MORE ? STAGES * STAGE : 0) + wave * kOut, again->partial);
    if (!more) break;
    at = behind;
  }
  if (MORE) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // nor when it is given up
}

// lhs of a product of few rows that the workgroup puts into blocks itself, in shared memory: `rows` lines of `per` steps, then a byte of scale for each half step,
// quarter of it and line.  It has kOwnChunks chunks of eight values at most: more take longer than a launch that puts lhs into blocks once for all (us, here and there: of 1024 chunks
// 6.1 and 7.6, 2048 7.2 and 7.6, 4096 9.5 and 7.7 for 4, 8 and 16 x 2048 x 16384; 9.8 and 11.9, 11.0 and 11.8, 13.4 and 11.8 for 1, 2 and 4 x 8192 x 8192).
constexpr uint32_t kOwnChunks = 2048;
__host__ __device__ constexpr uint32_t own_pitch(uint32_t per) { return per * kStep + 64; }       // (64 more, against bank conflicts)
__host__ __device__ constexpr uint32_t own_bytes(uint32_t rows, uint32_t per) { return rows * own_pitch(per) + per * 2 * 64; }
constexpr uint32_t kOwnLhs = own_bytes(1, kOwnChunks / 32);       // (the most that rows * per * 32 chunks take, of one to sixteen rows)
static_assert(own_bytes(16, kOwnChunks / 512) <= kOwnLhs, "of more rows it is less");

// Eight values a thread, four threads a block, BATCH times before the first is used.  (x.k is at least 8.)
template <class T>
__device__ __forceinline__ void own_blocks(const MxRows& x, uint32_t batch, uint32_t m0, uint32_t rows, uint32_t step0, uint32_t per, char* codes, uint8_t* scales) {
  constexpr uint32_t BATCH = 4;
  const uint32_t line = per * 32, items = rows * line, k0 = step0 * 256;         // chunks of eight of a line
  const T* const from = (const T*)x.x.data + (int64_t)batch * x.x.batch + (int64_t)m0 * x.x.ld;
  for (uint32_t first = threadIdx.x; first < items; first += BATCH * blockDim.x) {
    Eight<T> t[BATCH];
#pragma unroll
    for (uint32_t b = 0; b < BATCH; b++) {
      const uint32_t i = min(first + b * blockDim.x, items - 1), r = i / line;
      t[b].load(from + (int64_t)r * x.x.ld, k0 + (i - r * line) * 8, x.k);
    }
#pragma unroll
    for (uint32_t b = 0; b < BATCH; b++) {
      const uint32_t i = first + b * blockDim.x, r = i / line, c = i - r * line;
      if (i >= items) continue;    // (four lanes of a block at once)
      float v[8];
      t[b].values(k0 + c * 8, x.k, v);
      uint32_t most = 0;
#pragma unroll
      for (int e = 0; e < 8; e++) most = max(most, __float_as_uint(v[e]) & 0x7FFFFFFFu);
      most = max4(most);
      const bool finite = most < 0x7F800000u;
      const uint32_t scale = finite ? scale_of(most) : 255;
      *(uint32_t*)(codes + r * own_pitch(per) + c * 4) = finite ? codes8(v, power_of(scale)) : 0;
      if (c % 4 == 0) scales[c / 4 * 16 + r] = (uint8_t)scale;
    }
  }
}

// Few rows: the loop of linear.hip's rows_kernel, the sum split among the waves of a workgroup, each with a ring of its own.  A tile of 16 rows, in their own
// order (so their scales are bytes here and there of the group's), and 64 columns.  OWN: lhs is a matrix of T, which the workgroup puts into blocks while its first
// steps of rhs are under way (1 x 2048 x 16384 5.4 us; from blocks 5.0, and 4 for the launch that makes them).
template <int WAVES, int STAGES, class T, bool OWN>
__global__ __launch_bounds__(64 * WAVES) void mx_rows_kernel(const MxProduct x, uint32_t steps, uint32_t per_split, uint32_t splits, uint32_t first, float* __restrict__ partial) {
  constexpr int TM = 16, TN = 64, BN = TN / 16;
  constexpr uint32_t A = OWN ? 0 : TM * kStep, CODES = A + TN * kStep, SA = OWN ? 0 : 512, STAGE = CODES + SA + 512;
  __shared__ __attribute__((aligned(1024))) char lds[WAVES][STAGES * STAGE];
  __shared__ __attribute__((aligned(16))) char own[OWN ? kOwnLhs : 16];
  const Product& p = x.p;

  const Place at = place(first, (p.M + TM - 1) / TM, (p.N + TN - 1) / TN, splits);
  const uint32_t m0 = at.tm * TM, n0 = at.tn * TN;
  const uint32_t t = threadIdx.x, lane = t & 63, q = lane & 15, g = lane >> 4;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(t >> 6);

  float bias[8];
  bias8(p.e, n0 + t % 8 * 8, n0 + t % 8 * 8 < p.N ? p.N - (n0 + t % 8 * 8) : 0, bias);
  Feed<bf16, true, false, TM, 64> fa;
  Feed<bf16, true, true, TN, 64> fb;
  fb.init(p.ldb, lane);
  const uint32_t pitch = p.K / 32 * 256;
  const Scales scales_a(x.scales_a + (int64_t)at.batch * x.scales_batch_a, m0, p.M, pitch, 1), scales_b(x.scales_b + (int64_t)at.batch * x.scales_batch_b, n0, p.N, pitch, 1);
  Slot sa[2], sb[2];
  if (!OWN) fa.init(p.lda, lane);
#pragma unroll
  for (uint32_t kk = 0; kk < 2; kk++) {
    if (!OWN) sa[kk].init(pitch, 0, kk, lane);
    sb[kk].init(pitch, 0, kk, lane);
  }
  constexpr int LOADS = decltype(fb)::N + 2 + (OWN ? 0 : decltype(fa)::N + 2);

  const uint32_t begin = at.split * per_split, end = min(begin + per_split, steps);
  uint32_t step = begin + wave;                   // the next one to load
  const uint32_t n = end > step ? (end - step + WAVES - 1) / WAVES : 0;
  const char* const ca = (const char*)p.a + ((int64_t)at.batch * p.batch_a + (int64_t)m0 * p.lda) * 2;
  const char* const cb = (const char*)p.b + ((int64_t)at.batch * p.batch_b + (int64_t)n0 * p.ldb) * 2;
  const int64_t size_a = (int64_t)(p.M - m0) * p.lda * 2, size_b = (int64_t)(p.N - n0) * p.ldb * 2;
  char* const ring = lds[wave];
  const auto load = [&](uint32_t stage) {
    const uint32_t to = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_ptr)ring + stage * STAGE);
    const bool more = step < end;
    const uint32_t s = more ? step : 0, half = more ? step * 2 : kNoHalf;
    const u32x4 buf_b = fb.buffer(cb + (int64_t)s * kStep, more ? size_b - (int64_t)s * kStep : 0);
#pragma unroll
    for (int i = 0; i < fb.N; i++) fb.load(i, buf_b, p.K - s * kUnits, to + A, lane);
#pragma unroll
    for (uint32_t kk = 0; kk < 2; kk++) sb[kk].load(half, to + CODES + SA + kk * 256, scales_b.buffer);
    if (!OWN) {
      const u32x4 buf_a = fa.buffer(ca + (int64_t)s * kStep, more ? size_a - (int64_t)s * kStep : 0);
#pragma unroll
      for (int i = 0; i < fa.N; i++) fa.load(i, buf_a, p.K - s * kUnits, to, lane);
#pragma unroll
      for (uint32_t kk = 0; kk < 2; kk++) sa[kk].load(half, to + CODES + kk * 256, scales_a.buffer);
    }
    step += WAVES;
  };

  f32x4 acc[1][BN];
#pragma unroll
  for (int j = 0; j < BN; j++) acc[0][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const uint32_t rows = min(p.M - m0, (uint32_t)TM), per = end > begin ? end - begin : 0;
  const uint32_t mine = OWN ? g * 16 + min(q, rows - 1) : scale_at(m0 % 64 + q, g);        // where the lane's scales of a half step lie
  uint8_t* const own_scales = (uint8_t*)own + rows * own_pitch(per);

  if (n) {
#pragma unroll
    for (int s = 0; s < STAGES; s++) load(s);
  }
  if (OWN && per) own_blocks<T>(x.lhs, at.batch, m0, rows, begin, per, own, own_scales);
  if (OWN) __syncthreads();
  if (n) {
    uint32_t cur = 0, at_own = wave;              // the step of the workgroup's
    for (uint32_t s = 0; s < n; s++, at_own += WAVES) {
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"((STAGES - 1) * LOADS) : "memory");
      const lds_ptr tile = (lds_ptr)ring + cur * STAGE;
      bf16x8 oa[2][1], ob[2][BN];
      uint32_t ka[2], kb[2][1];
#pragma unroll
      for (uint32_t kk = 0; kk < 2; kk++) {
        if (OWN) {
          oa[kk][0] = *(const bf16x8*)(own + min(q, rows - 1) * own_pitch(per) + at_own * kStep + kk * 64 + g * 16);
          ka[kk] = own_scales[(at_own * 2 + kk) * 64 + mine];
        } else {
          read_blocks<bf16, true, false, TM>(tile, 0, 0, kk, q, g, oa[kk]);
          ka[kk] = *(const __attribute__((address_space(3))) uint8_t*)(tile + CODES + kk * 256 + mine);
        }
        read_blocks<bf16, true, true, TN>(tile + A, 0, 0, kk, q, g, ob[kk]);
        read_scales<TN>(tile + CODES + SA, 0, kk, lane, kb[kk]);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // read before the place is loaded again
      load(cur);
#pragma unroll
      for (int kk = 0; kk < 2; kk++)
#pragma unroll
        for (int j = 0; j < BN; j++) acc[0][j] = multiply(oa[kk][0], ob[kk][j], ka[kk], kb[kk][0], 0, j, acc[0][j]);
      cur = cur + 1 == STAGES ? 0 : cur + 1;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }
  add_waves<bf16, WAVES>(p, at, splits, m0, n0, t, bias, acc, &lds[0][0], sizeof lds[0], partial);
}

}  // namespace

hipError_t launch_mx_quantize(const MxRows& p, hipStream_t st) {
  return in_launches((uint64_t)p.batches * ((p.lines + 63ull) / 64) * mx_steps(p.k), [&](uint64_t first, uint32_t n) {
    if (p.kc && p.x.bf16) mx_quantize_kernel<bf16><<<n, 256, 0, st>>>(p, first);
    else if (p.kc) mx_quantize_kernel<float><<<n, 256, 0, st>>>(p, first);
    else if (p.x.bf16) mx_quantize_across_kernel<bf16><<<n, 256, 0, st>>>(p, first);
    else mx_quantize_across_kernel<float><<<n, 256, 0, st>>>(p, first);
  });
}

hipError_t launch_mx_dequantize(const MxRows& p, hipStream_t st) {
  return in_launches((uint64_t)p.batches * ((p.lines + 63ull) / 64) * mx_steps(p.k), [&](uint64_t first, uint32_t n) {
    if (p.x.bf16) mx_dequantize_kernel<bf16><<<n, 256, 0, st>>>(p, first);
    else mx_dequantize_kernel<float><<<n, 256, 0, st>>>(p, first);
  });
}

// How long a kernel takes, in us, as linear.hip's rule has it: a round of workgroups on the 256 compute units, one each or two at once, is `fixed`
// and a step's time for each step along k.  Measured on products whose tiles are one whole round (or two at once), 2048 and 16384 long along k, replayed in a graph.  (On another card a step takes 3 to 8 % less throughout: 1.65, 0.97, 0.64 and 1.10, 0.36 and 0.50.)
struct Kernel { uint32_t id, tm, tn; float fixed, one, two; };
constexpr Kernel kKernels[] = {
    {kFast256, 256, 256, 12, 1.70f, 0},       {kFast256x128, 256, 128, 10.5f, 1.045f, 0}, {kFast128, 128, 128, 8, 0.666f, 1.13f},
    {kFast64, 64, 64, 4.4f, 0.388f, 0.545f},  {kRows, 16, 64, 2.5f, 0, 0},
};
constexpr float kLaunch1 = 3, kQuantize = 2, kBytes = 4.5e6f;      // a further launch, one for lhs's blocks, us; bytes a us
// Few rows: one workgroup at once, whose step takes 0.15 us until the columns' tiles and splits are so many that memory's 6.5 TB/s bound it (0.33 us for 256); lhs's blocks
// take it 0.8 us for each 1024 chunks of eight values.  (1 x 16384 x 2048 alone, in 4 and 8 splits 12.0, 8.7 and 8.3 us; 16 x 4096 x 4096 alone, in 2 and 4 14.5, 12.1 and 9.6.)
float rows_time(uint64_t blocks, uint64_t columns, uint32_t per, uint32_t rows, bool own) {
  const float step = std::max(0.15f, 0.0013f * std::min<uint64_t>(columns, 256));
  return 1 + (float)((blocks + 255) / 256) * (2.5f + per * step + (own ? 0.8f * ((rows * per * 32 + 1023) / 1024) : 0));
}
bool fits_own(uint32_t rows, uint32_t per) { return (uint64_t)std::min(rows, 16u) * per * 32 <= kOwnChunks; }

// By the sizes alone: the kernel and the splits are the order of the sums, which is to be the same for a lhs in blocks as for one that the call puts into them.  So both
// are priced as a row-major matrix is.  (One size in eighty would be split otherwise from blocks: 3 x 5250 x 768 takes 7.1 us so and would take 6.3, 2 x 16129 x 4087 12.2 and 13.8.)
ProductPlan plan_mx(const MxProduct& x) {
  const Product& p = x.p;
  ProductPlan plan{};
  plan.steps = (p.K + kUnits - 1) / kUnits;
  const float out = (float)p.batches * p.M * p.N * 4;
  float best = 0;
  for (const Kernel& k : kKernels) {
    const uint64_t columns = (uint64_t)((p.N + k.tn - 1) / k.tn) * p.batches, tiles = (uint64_t)((p.M + k.tm - 1) / k.tm) * columns;
    for (uint32_t splits = 1; splits <= 64; splits = splits == 1 ? 2 : splits & splits - 1 ? splits / 3 * 4 : splits / 2 * 3) {
      const uint32_t per = (plan.steps + splits - 1) / splits;
      if (splits > 1 && (per < 4 || tiles * splits > 1024)) break;
      const uint64_t blocks = tiles * splits, rounds = blocks / 512, rest = blocks % 512;
      const bool own = k.id == kRows && fits_own(p.M, per);
      const float one = k.fixed + per * k.one, two = k.two ? k.fixed + per * k.two : 2 * one;
      float t = k.id == kRows ? rows_time(blocks, columns * splits, per, std::min(p.M, 16u), own) : rounds * two + (rest > 256 ? two : rest ? one : 0);
      if (splits > 1) t += kLaunch1 + (splits + 1) * out / kBytes;
      if (!own) t += kQuantize;
      if (best && t >= best) continue;
      best = t;
      plan.kernel = k.id == kFast128 && blocks <= 256 ? kFast128Alone : k.id;
      plan.per_split = per;
      plan.splits = per ? (plan.steps + per - 1) / per : 1;
      plan.blocks = tiles * plan.splits;
    }
  }
  plan.partial_bytes = plan.splits > 1 ? (uint64_t)plan.splits * p.batches * p.M * ((p.N + 7) / 8 * 8) * 4 : 0;
  return plan;
}

bool mx_takes_rows(const MxProduct& x, const ProductPlan& plan, const MxRows& lhs) { return plan.kernel == kRows && lhs.kc && lhs.k >= 8 && fits_own(x.p.M, plan.per_split); }

hipError_t launch_mx(const MxProduct& x, const ProductPlan& plan, float* partial, hipStream_t st) {
  MxProduct by = x;
  by.partial = partial;
  const auto tiles = [&](auto kernel, uint32_t threads, uint32_t at_once) {
    const auto go = [&](uint64_t first, uint32_t n, uint32_t tiles) { kernel<<<n, threads, 0, st>>>(by, plan.steps, plan.per_split, plan.splits, (uint32_t)first, tiles); };
    if (!at_once || plan.splits > 1 || plan.steps < 2 || plan.blocks <= at_once) return in_launches(plan.blocks, [&](uint64_t first, uint32_t n) { go(first, n, n); });
    go(0, at_once, (uint32_t)plan.blocks);
    return hipGetLastError();
  };
  const auto rows = [&](auto kernel) {
    return in_launches(plan.blocks, [&](uint64_t first, uint32_t n) { kernel<<<n, 256, 0, st>>>(x, plan.steps, plan.per_split, plan.splits, (uint32_t)first, partial); });
  };
  switch (plan.kernel) {
    case kFast256: return tiles(mx_tile_kernel<256, 256, 2, 4, 2>, 512, 256);
    case kFast256x128: return tiles(mx_tile_kernel<256, 128, 4, 2, 3>, 512, 0);
    case kFast128: return tiles(mx_tile_kernel<128, 128, 2, 2, 2>, 256, 512);
    case kFast128Alone: return tiles(mx_tile_kernel<128, 128, 2, 4, 4>, 512, 0);
    case kFast64: return tiles(mx_tile_kernel<64, 64, 2, 2, 4>, 256, 0);
    default:
      if (!x.lhs.x.data) return rows(mx_rows_kernel<4, 3, bf16, false>);
      return x.lhs.x.bf16 ? rows(mx_rows_kernel<4, 3, bf16, true>) : rows(mx_rows_kernel<4, 3, float, true>);
  }
}

}  // namespace mrl
