// Layer normalisation of rows and its gradients (operators.h): kernels and launches.
//
//   mean = S x / n,  var = S (x - mean)^2 / n,  r = 1 / sqrt(var + eps),  h = (x - mean) r,  out = h w + b
//   g = grad w,  dx = residual + r (g - S g / n - h S(g h) / n),  dw = S_rows grad h,  db = S_rows grad
#include <hip/hip_runtime.h>

#include <algorithm>

#include "tiles.h"

namespace mrl {
namespace {

constexpr uint32_t kThreads = 256;

// The sums of two values over the workgroup, in every thread.  Their order is that of the threads.
__device__ __forceinline__ f32x2 sum_block(f32x2 v) {
  __shared__ f32x2 sums[kThreads / 64];
#pragma unroll
  for (int i = 32; i; i >>= 1) {
    v[0] += __shfl_xor(v[0], i);
    v[1] += __shfl_xor(v[1], i);
  }
  __syncthreads();                 // (the sums of the call before have been read)
  if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = v;
  __syncthreads();
  v = sums[0];
#pragma unroll
  for (uint32_t w = 1; w < kThreads / 64; w++) {
    v[0] += sums[w][0];
    v[1] += sums[w][1];
  }
  return v;
}

__device__ __forceinline__ int64_t start(const RowsOf& x, uint32_t row, uint32_t M) {
  const uint32_t batch = row / M;
  return (int64_t)batch * x.batch + (int64_t)(row - batch * M) * x.ld;
}

// A row a workgroup, eight elements a thread at a time, three passes over it.
__global__ __launch_bounds__(kThreads) void norm_kernel(const NormRows p, uint32_t first) {
  const uint32_t row = first + blockIdx.x;
  const int64_t x = start(p.x, row, p.M), out = start(p.out, row, p.M);
  const float N = (float)p.N;
  float v[8];
  f32x2 s = {0.0f, 0.0f};
  for (uint64_t n = threadIdx.x * 8; n < p.N; n += kThreads * 8) {
    load8(p.x.data, p.x.bf16, x + n, p.N - n, v);
#pragma unroll
    for (int e = 0; e < 8; e++) s[0] += v[e];
  }
  const float about = sum_block(s)[0] / N;
  // the sum of what is left puts the mean right: where it is far from 0, its own sum has lost that much
  s = f32x2{0.0f, 0.0f};
  for (uint64_t n = threadIdx.x * 8; n < p.N; n += kThreads * 8) {
    const uint32_t valid = p.N - n;
    load8(p.x.data, p.x.bf16, x + n, valid, v);
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const float d = (uint32_t)e < valid ? v[e] - about : 0.0f;
      s[0] += d;
      s[1] += d * d;
    }
  }
  s = sum_block(s);
  const float rest = s[0] / N, var = s[1] / N - rest * rest, r = 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + p.eps);       // (NaN stays)
  if (p.stats && threadIdx.x == 0) {
    p.stats[2 * (uint64_t)row] = about + rest;
    p.stats[2 * (uint64_t)row + 1] = r;
  }
  for (uint64_t n = threadIdx.x * 8; n < p.N; n += kThreads * 8) {
    const uint32_t valid = p.N - n;
    float w[8];
    load8(p.x.data, p.x.bf16, x + n, valid, v);
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = (v[e] - about - rest) * r;
    if (p.weight) {
      load8(p.weight, p.weight_bf16, n, valid, w);
#pragma unroll
      for (int e = 0; e < 8; e++) v[e] *= w[e];
    }
    if (p.bias) {
      load8(p.bias, p.bias_bf16, n, valid, w);
#pragma unroll
      for (int e = 0; e < 8; e++) v[e] += w[e];
    }
    store8(p.out.data, p.out.bf16, out + n, valid, v);
  }
}

// dx, a row a workgroup: two passes over it.
__global__ __launch_bounds__(kThreads) void norm_grad_kernel(const NormGrad p, uint32_t first) {
  const uint32_t row = first + blockIdx.x;
  const int64_t x = start(p.x, row, p.M), grad = start(p.grad, row, p.M), dx = start(p.dx, row, p.M);
  const float mean = p.stats[2 * (uint64_t)row], r = p.stats[2 * (uint64_t)row + 1];
  float v[8], g[8], w[8];
  const auto load = [&](uint64_t n) {              // h and g
    const uint32_t valid = p.N - n;
    load8(p.x.data, p.x.bf16, x + n, valid, v);
    load8(p.grad.data, p.grad.bf16, grad + n, valid, g);
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = (v[e] - mean) * r;
    if (p.weight) {
      load8(p.weight, p.weight_bf16, n, valid, w);
#pragma unroll
      for (int e = 0; e < 8; e++) g[e] *= w[e];
    }
  };
  f32x2 s = {0.0f, 0.0f};
  for (uint64_t n = threadIdx.x * 8; n < p.N; n += kThreads * 8) {
    load(n);
#pragma unroll
    for (int e = 0; e < 8; e++) {
      if ((uint64_t)e + n >= p.N) continue;
      s[0] += g[e];
      s[1] += g[e] * v[e];
    }
  }
  s = sum_block(s);
  const float a = s[0] / (float)p.N, b = s[1] / (float)p.N;
  for (uint64_t n = threadIdx.x * 8; n < p.N; n += kThreads * 8) {
    load(n);
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = r * (g[e] - a - v[e] * b);
    if (p.residual.data) {
      load8(p.residual.data, p.residual.bf16, start(p.residual, row, p.M) + n, p.N - n, g);
#pragma unroll
      for (int e = 0; e < 8; e++) v[e] += g[e];
    }
    store8(p.dx.data, p.dx.bf16, dx + n, p.N - n, v);
  }
}

// dw and db: a column a thread.
__global__ __launch_bounds__(kThreads) void norm_columns_kernel(const NormGrad p) {
  const uint32_t n = blockIdx.x * kThreads + threadIdx.x, rows = p.batches * p.M;
  if (n >= p.N) return;
  float dw = 0.0f, db = 0.0f;
  for (uint32_t row = 0; row < rows; row++) {
    const int64_t at = start(p.grad, row, p.M) + n;
    const float g = p.grad.bf16 ? (float)((const bf16*)p.grad.data)[at] : ((const float*)p.grad.data)[at];
    db += g;
    if (!p.dweight) continue;
    const int64_t to = start(p.x, row, p.M) + n;
    const float x = p.x.bf16 ? (float)((const bf16*)p.x.data)[to] : ((const float*)p.x.data)[to];
    dw += g * ((x - p.stats[2 * (uint64_t)row]) * p.stats[2 * (uint64_t)row + 1]);
  }
  if (p.dweight && p.dweight_bf16) ((bf16*)p.dweight)[n] = (bf16)dw;
  else if (p.dweight) ((float*)p.dweight)[n] = dw;
  if (p.dbias && p.dbias_bf16) ((bf16*)p.dbias)[n] = (bf16)db;
  else if (p.dbias) ((float*)p.dbias)[n] = db;
}

}  // namespace

hipError_t launch_norm(const NormRows& p, hipStream_t st) {
  if (!p.N) return hipSuccess;
  return in_launches((uint64_t)p.batches * p.M, [&](uint64_t first, uint32_t n) { norm_kernel<<<n, kThreads, 0, st>>>(p, (uint32_t)first); });
}

uint64_t norm_grad_bytes(const NormGrad&) { return 0; }

hipError_t launch_norm_grad(const NormGrad& p, float*, hipStream_t st) {
  if (!p.N) return hipSuccess;
  hipError_t e = hipSuccess;
  if (p.dx.data) e = in_launches((uint64_t)p.batches * p.M, [&](uint64_t first, uint32_t n) { norm_grad_kernel<<<n, kThreads, 0, st>>>(p, (uint32_t)first); });
  if (e == hipSuccess && (p.dweight || p.dbias)) {
    norm_columns_kernel<<<(p.N + kThreads - 1) / kThreads, kThreads, 0, st>>>(p);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace mrl
