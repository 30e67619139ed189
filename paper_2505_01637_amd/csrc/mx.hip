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

// A block a thread: 64 lines by a step of 128 values a workgroup.
__global__ __launch_bounds__(256) void mx_quantize_kernel(const MxRows p, uint64_t first) {
  const uint32_t steps = mx_steps(p.k), groups = (p.lines + 63) / 64;
  const uint64_t id = first + blockIdx.x;
  const uint32_t s = (uint32_t)(id % steps), group = (uint32_t)(id / steps % groups), batch = (uint32_t)(id / steps / groups);
  const uint32_t l = threadIdx.x & 63, g = threadIdx.x >> 6, line = group * 64 + l, k0 = s * 128 + g * 32;
  float v[32];
  uint32_t most = 0;
#pragma unroll
  for (int e = 0; e < 32; e++) {
    const uint32_t k = k0 + e;
    v[e] = 0.0f;
    if (line < p.lines && k < p.k) {
      const int64_t at = (int64_t)batch * p.x.batch + (p.kc ? (int64_t)line * p.x.ld + k : (int64_t)k * p.x.ld + line);
      v[e] = p.x.bf16 ? (float)((const bf16*)p.x.data)[at] : ((const float*)p.x.data)[at];
    }
    most = max(most, __float_as_uint(v[e]) & 0x7FFFFFFFu);
  }
  const bool finite = most < 0x7F800000u;
  const uint32_t scale = finite ? scale_of(most) : 255;
  p.scales[(((uint64_t)batch * groups + group) * steps + s) * 256 + scale_at(l, g)] = (uint8_t)scale;
  if (line >= p.lines) return;
  u32x4 c = {0, 0, 0, 0};
  if (finite) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const float x[8] = {v[8 * i], v[8 * i + 1], v[8 * i + 2], v[8 * i + 3], v[8 * i + 4], v[8 * i + 5], v[8 * i + 6], v[8 * i + 7]};
      c[i] = codes8(x, power_of(scale));
    }
  }
  *(u32x4*)(p.codes + (((uint64_t)batch * p.lines + line) * steps + s) * 64 + g * 16) = c;
}

// Eight values a thread.
__global__ __launch_bounds__(256) void mx_dequantize_kernel(const MxRows p, uint64_t first) {
  const uint32_t per = (p.k + 7) / 8, steps = mx_steps(p.k), groups = (p.lines + 63) / 64;
  const uint64_t id = (first + blockIdx.x) * 256 + threadIdx.x, row = id / per;
  if (row >= (uint64_t)p.batches * p.lines) return;
  const uint32_t at = (uint32_t)(id - row * per), batch = (uint32_t)(row / p.lines), line = (uint32_t)(row - (uint64_t)batch * p.lines);
  const uint32_t from = p.shared ? 0 : batch, s = at / 16, g = at / 4 % 4;
  const uint32_t c = *(const uint32_t*)(p.codes + (((uint64_t)from * p.lines + line) * steps) * 64 + at * 4);
  const uint32_t scale = p.scales[(((uint64_t)from * groups + line / 64) * steps + s) * 256 + scale_at(line & 63, g)];
  const float power = scale == 255 ? __uint_as_float(0x7FC00000u) : power_of(scale);
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; e++) {
    const uint32_t code = c >> 4 * e & 15, m = code & 7;
    // magnitudes below 1 are 0 and 0.5; the others have an exponent of two bits above one of mantissa
    const float a = m < 2 ? 0.5f * (float)m : __uint_as_float((126 + (m >> 1)) << 23 | (m & 1) << 22);
    v[e] = (code & 8 ? -a : a) * power;
  }
  store8(p.x.data, p.x.bf16, (int64_t)batch * p.x.batch + (int64_t)line * p.x.ld + at * 8, p.k - at * 8, v);
}

// acc += a's block of 16 lines times b's over 128 values; sa and sb hold four blocks' scales, byte by byte.
template <int OA, int OB>
__device__ __forceinline__ f32x4 multiply(const i32x4& a, const i32x4& b, uint32_t sa, uint32_t sb, const f32x4& acc) {
  const i32x8 x = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, y = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(y, x, acc, 4, 4, OB, (int)sb, OA, (int)sa);       // (4: both operands are 4-bit floating point)
}

// A tile of 64 x 64, a quarter a wave, operands straight from memory.
__global__ __launch_bounds__(256) void mx_kernel(const MxProduct x, uint32_t first) {
  const Product& p = x.p;
  __shared__ __attribute__((aligned(16))) char lds[4][32 * 32 * 4];
  const Place at = place(first, (p.M + 63) / 64, (p.N + 63) / 64, 1);
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, q = lane & 15, g = lane >> 4;
  const uint32_t m0 = at.tm * 64 + wave / 2 * 32, n0 = at.tn * 64 + wave % 2 * 32, steps = p.K / 32;
  const uint8_t* const sa = x.scales_a + (int64_t)at.batch * x.scales_batch_a + (uint64_t)at.tm * steps * 256 + lane * 4;
  const uint8_t* const sb = x.scales_b + (int64_t)at.batch * x.scales_batch_b + (uint64_t)at.tn * steps * 256 + lane * 4;
  const char *a[2], *b[2];
#pragma unroll
  for (int i = 0; i < 2; i++) {
    a[i] = (const char*)p.a + ((int64_t)at.batch * p.batch_a + (int64_t)min(m0 + row_of<bf16, true>(i, q), p.M - 1) * p.lda) * 2 + g * 16;
    b[i] = (const char*)p.b + ((int64_t)at.batch * p.batch_b + (int64_t)min(n0 + row_of<bf16, true>(i, q), p.N - 1) * p.ldb) * 2 + g * 16;
  }
  f32x4 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; i++)
#pragma unroll
    for (int j = 0; j < 2; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (uint32_t s = 0; s < steps; s++) {
    const uint32_t ka = *(const uint32_t*)(sa + (uint64_t)s * 256) >> wave / 2 * 16, kb = *(const uint32_t*)(sb + (uint64_t)s * 256) >> wave % 2 * 16;
    i32x4 va[2], vb[2];
#pragma unroll
    for (int i = 0; i < 2; i++) {
      va[i] = *(const i32x4*)(a[i] + (uint64_t)s * 64);
      vb[i] = *(const i32x4*)(b[i] + (uint64_t)s * 64);
    }
    acc[0][0] = multiply<0, 0>(va[0], vb[0], ka, kb, acc[0][0]);
    acc[0][1] = multiply<0, 1>(va[0], vb[1], ka, kb, acc[0][1]);
    acc[1][0] = multiply<1, 0>(va[1], vb[0], ka, kb, acc[1][0]);
    acc[1][1] = multiply<1, 1>(va[1], vb[1], ka, kb, acc[1][1]);
  }
  write_out<bf16, 2, 2, 2, true>(p, at, 1, m0, n0, lane, acc, lds[wave], nullptr);
}

}  // namespace

hipError_t launch_mx_quantize(const MxRows& p, hipStream_t st) {
  return in_launches((uint64_t)p.batches * ((p.lines + 63ull) / 64) * mx_steps(p.k), [&](uint64_t first, uint32_t n) { mx_quantize_kernel<<<n, 256, 0, st>>>(p, first); });
}

hipError_t launch_mx_dequantize(const MxRows& p, hipStream_t st) {
  const uint64_t items = (uint64_t)p.batches * p.lines * ((p.k + 7ull) / 8);
  return in_launches((items + 255) / 256, [&](uint64_t first, uint32_t n) { mx_dequantize_kernel<<<n, 256, 0, st>>>(p, first); });
}

ProductPlan plan_mx(const MxProduct& x) {
  ProductPlan plan{};
  plan.splits = 1;
  plan.blocks = (uint64_t)x.p.batches * ((x.p.M + 63) / 64) * ((x.p.N + 63) / 64);
  return plan;
}

hipError_t launch_mx(const MxProduct& x, const ProductPlan& plan, float*, hipStream_t st) {
  return in_launches(plan.blocks, [&](uint64_t first, uint32_t n) { mx_kernel<<<n, 256, 0, st>>>(x, (uint32_t)first); });
}

}  // namespace mrl
