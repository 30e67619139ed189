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

// ---- gradients of rows that a workgroup keeps in registers

template <int CTRL>
__device__ __forceinline__ float moved(float x) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xF, 0xF, true)); }
// The sum over a wave, in every lane: within rows of sixteen lanes by moves, the four rows' after that.
__device__ __forceinline__ float sum_wave(float x) {
  x += moved<0xB1>(x);             // lanes 1, 0, 3, 2
  x += moved<0x4E>(x);             // lanes 2, 3, 0, 1
  x += moved<0x141>(x);            // mirrored in eight
  x += moved<0x140>(x);            // and in sixteen
  const int v = __float_as_int(x);
  return (__int_as_float(__builtin_amdgcn_readlane(v, 0)) + __int_as_float(__builtin_amdgcn_readlane(v, 16))) +
         (__int_as_float(__builtin_amdgcn_readlane(v, 32)) + __int_as_float(__builtin_amdgcn_readlane(v, 48)));
}

// Eight neighbouring elements as they are stored.
template <class T> struct Raw { T v[8]; };
template <class T>
__device__ __forceinline__ Raw<T> load_raw(const T* p, uint32_t valid) {
  Raw<T> r;
  if (valid >= 8) {
    __builtin_memcpy(r.v, p, sizeof r.v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; e++) r.v[e] = (uint32_t)e < valid ? p[e] : (T)0.0f;
  }
  return r;
}

constexpr uint32_t kRowThreads = 512;      // of a workgroup that keeps rows
constexpr uint32_t kKeep = 4;              // times 8 elements a thread has of a row at most: 16384 elements

// `waves` waves a row, R times eight elements a thread; the workgroup's groups of waves take its `each` rows in turn and keep the columns' sums, which they add
// in their order at the end.  partial: the workgroups' sums (2 x N each: dw, db), nullptr where there is one workgroup.
// Memory bounds it, so the next row's loads go out before this row's sums are made (where there is room: not four times f32).
template <class TX, class TG, int R>
__global__ __launch_bounds__(kRowThreads) void norm_grad_rows_kernel(const NormGrad p, uint32_t waves, uint32_t each, uint32_t first, float* __restrict__ partial) {
  constexpr bool AHEAD = R * (sizeof(TX) + sizeof(TG)) < 32;
  __shared__ f32x2 sums[2][kRowThreads / 64];
  __shared__ float columns[2][R == 1 ? kRowThreads / 2 * 8 : 8];         // (more than one group only where a row has half of the threads or fewer)
  const uint32_t block = first + blockIdx.x, rows = p.batches * p.M;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = wave / waves, groups = blockDim.x / 64 / waves;
  const uint32_t t = threadIdx.x - group * waves * 64, pitch = waves * 512;
  const uint64_t begin = (uint64_t)block * each;
  const uint32_t end = (uint32_t)min(begin + each, (uint64_t)rows);
  const bool wants = p.dweight || p.dbias;

  float w[R][8], dw[R][8], db[R][8];
#pragma unroll
  for (int i = 0; i < R; i++) {
    const uint32_t n = i * pitch + t * 8, valid = n < p.N ? p.N - n : 0;
#pragma unroll
    for (int e = 0; e < 8; e++) { w[i][e] = 1.0f; dw[i][e] = db[i][e] = 0.0f; }
    if (p.weight) load8(p.weight, p.weight_bf16, n, valid, w[i]);
  }
  Raw<TX> x[R], x1[R];
  Raw<TG> g[R], g1[R];
  float mean, r, mean1 = 0.0f, r1 = 0.0f;
  const auto load = [&](uint32_t row, Raw<TX> (&x)[R], Raw<TG> (&g)[R], float& mean, float& r) {
    if (row >= end) return;
    const int64_t at_x = start(p.x, row, p.M), at_g = start(p.grad, row, p.M);
    mean = p.stats[2 * (uint64_t)row];
    r = p.stats[2 * (uint64_t)row + 1];
#pragma unroll
    for (int i = 0; i < R; i++) {
      const uint32_t n = i * pitch + t * 8, valid = n < p.N ? p.N - n : 0;
      x[i] = load_raw((const TX*)p.x.data + at_x + n, valid);
      g[i] = load_raw((const TG*)p.grad.data + at_g + n, valid);
    }
  };
  if (AHEAD) load((uint32_t)begin + group, x1, g1, mean1, r1);
  uint32_t turn = 0;
  for (uint32_t row0 = (uint32_t)begin; row0 < end; row0 += groups, turn ^= 1) {
    const uint32_t row = row0 + group;
    if (AHEAD) {
#pragma unroll
      for (int i = 0; i < R; i++) { x[i] = x1[i]; g[i] = g1[i]; }
      mean = mean1;
      r = r1;
      load(row + groups, x1, g1, mean1, r1);
    } else {
      load(row, x, g, mean, r);
    }
    float s0 = 0.0f, s1 = 0.0f;
    if (row < end) {
#pragma unroll
      for (int i = 0; i < R; i++)
#pragma unroll
        for (int e = 0; e < 8; e++) {
          const uint32_t n = i * pitch + t * 8 + e;
          const float grad = (float)g[i].v[e], h = ((float)x[i].v[e] - mean) * r, gw = grad * w[i][e];
          if (n < p.N) {           // (behind the row's end: a NaN of its statistics would come in)
            s0 += gw;
            s1 += gw * h;
            dw[i][e] += grad * h;
            db[i][e] += grad;
          }
        }
    }
    if (!p.dx.data) continue;
    s0 = sum_wave(s0);
    s1 = sum_wave(s1);
    if (waves > 1) {
      if (threadIdx.x % 64 == 0) sums[turn][wave] = f32x2{s0, s1};
      __syncthreads();             // (and the other half is free: what was read there was read before this)
      s0 = s1 = 0.0f;
      for (uint32_t i = 0; i < waves; i++) {
        const f32x2 s = sums[turn][group * waves + i];
        s0 += s[0];
        s1 += s[1];
      }
    }
    if (row >= end) continue;
    const float a = s0 / (float)p.N, b = s1 / (float)p.N;
    const int64_t dx = start(p.dx, row, p.M), residual = p.residual.data ? start(p.residual, row, p.M) : 0;
#pragma unroll
    for (int i = 0; i < R; i++) {
      const uint32_t n = i * pitch + t * 8;
      if (n >= p.N) continue;
      float v[8], z[8];
      if (p.residual.data) load8(p.residual.data, p.residual.bf16, residual + n, p.N - n, z);
#pragma unroll
      for (int e = 0; e < 8; e++) v[e] = r * ((float)g[i].v[e] * w[i][e] - a - ((float)x[i].v[e] - mean) * r * b);
      if (p.residual.data) {
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] += z[e];
      }
      store8(p.dx.data, p.dx.bf16, dx + n, p.N - n, v);
    }
  }
  if (!wants) return;
  for (uint32_t k = 1; k < groups; k++) {          // the other groups' sums to the first, one after the other
    __syncthreads();
    if (group == k) {
#pragma unroll
      for (int e = 0; e < 8; e++) { columns[0][t * 8 + e] = dw[0][e]; columns[1][t * 8 + e] = db[0][e]; }
    }
    __syncthreads();
    if (group == 0) {
#pragma unroll
      for (int e = 0; e < 8; e++) { dw[0][e] += columns[0][t * 8 + e]; db[0][e] += columns[1][t * 8 + e]; }
    }
  }
  if (group) return;
#pragma unroll
  for (int i = 0; i < R; i++) {
    const uint32_t n = i * pitch + t * 8, valid = n < p.N ? p.N - n : 0;
    if (!valid) continue;
    if (partial) {
      float* const to = partial + (uint64_t)block * 2 * p.N + n;
      store8(to, valid, dw[i]);
      store8(to + p.N, valid, db[i]);
    } else {
      if (p.dweight) store8(p.dweight, p.dweight_bf16, n, valid, dw[i]);
      if (p.dbias) store8(p.dbias, p.dbias_bf16, n, valid, db[i]);
    }
  }
}

// The sums over columns alone, for rows too long for registers: 256 columns, eight a thread, `each` rows, eight at a time.
__global__ __launch_bounds__(256) void norm_columns_kernel(const NormGrad p, uint32_t each, uint32_t first, float* __restrict__ partial) {
  __shared__ float sums[2][8][256];
  const uint32_t blocks_n = (p.N + 255) / 256, id = first + blockIdx.x, bn = id % blocks_n, br = id / blocks_n;
  const uint32_t c = threadIdx.x & 31, l = threadIdx.x >> 5, n = bn * 256 + c * 8, rows = p.batches * p.M;
  float dw[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f}, db[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
  if (n < p.N) {
    for (uint32_t i = l; i < each; i += 8) {
      const uint64_t at = (uint64_t)br * each + i;
      if (at >= rows) break;
      const uint32_t row = (uint32_t)at;
      float x[8], g[8];
      load8(p.grad.data, p.grad.bf16, start(p.grad, row, p.M) + n, p.N - n, g);
#pragma unroll
      for (int e = 0; e < 8; e++) db[e] += g[e];
      if (!p.dweight) continue;
      load8(p.x.data, p.x.bf16, start(p.x, row, p.M) + n, p.N - n, x);
      const float mean = p.stats[2 * at], r = p.stats[2 * at + 1];
#pragma unroll
      for (int e = 0; e < 8; e++) dw[e] += g[e] * ((x[e] - mean) * r);
    }
  }
#pragma unroll
  for (int e = 0; e < 8; e++) { sums[0][l][c * 8 + e] = dw[e]; sums[1][l][c * 8 + e] = db[e]; }
  __syncthreads();
  const uint32_t at = bn * 256 + threadIdx.x;
  if (at >= p.N) return;
  float s[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < 8; i++) { s[0] += sums[0][i][threadIdx.x]; s[1] += sums[1][i][threadIdx.x]; }
  if (partial) {
    partial[(uint64_t)br * 2 * p.N + at] = s[0];
    partial[((uint64_t)br * 2 + 1) * p.N + at] = s[1];
    return;
  }
  if (p.dweight && p.dweight_bf16) ((bf16*)p.dweight)[at] = (bf16)s[0];
  else if (p.dweight) ((float*)p.dweight)[at] = s[0];
  if (p.dbias && p.dbias_bf16) ((bf16*)p.dbias)[at] = (bf16)s[1];
  else if (p.dbias) ((float*)p.dbias)[at] = s[1];
}

// dw and db from `blocks` workgroups' sums: 32 columns of the two side by side, 32 workgroups' at a time.
__global__ __launch_bounds__(1024) void norm_sums_kernel(const NormGrad p, uint32_t blocks, const float* __restrict__ partial) {
  __shared__ float sums[32][33];
  const uint32_t c = threadIdx.x & 31, l = threadIdx.x >> 5;
  const uint64_t at = (uint64_t)blockIdx.x * 32 + c;
  float s = 0.0f;
  if (at < 2ull * p.N) {
#pragma unroll 8
    for (uint32_t i = l; i < blocks; i += 32) s += partial[(uint64_t)i * 2 * p.N + at];
  }
  sums[l][c] = s;
  __syncthreads();
  if (l || at >= 2ull * p.N) return;
  for (int i = 1; i < 32; i++) s += sums[i][c];
  const uint32_t n = (uint32_t)(at < p.N ? at : at - p.N), is_bf16 = at < p.N ? p.dweight_bf16 : p.dbias_bf16;
  void* const to = at < p.N ? p.dweight : p.dbias;
  if (!to) return;
  if (is_bf16) ((bf16*)to)[n] = (bf16)s;
  else ((float*)to)[n] = s;
}

// How a gradient is launched, by its sizes alone (and whether column sums are wanted).
struct GradPlan {
  uint32_t keep, waves, groups;            // R and the waves of a row (0: too long to be kept), rows at a time of a workgroup
  uint32_t each, blocks;                   // rows of a workgroup (of a block of rows), how many of them
};
GradPlan plan_grad(const NormGrad& p) {
  const uint64_t rows = (uint64_t)p.batches * p.M;
  const bool sums = p.dweight || p.dbias;
  GradPlan g{};
  constexpr uint32_t most = kRowThreads * 8;
  if (p.N <= most * kKeep) {
    g.keep = p.N <= most ? 1 : p.N <= 2 * most ? 2 : 4;
    g.waves = (p.N + 512 * g.keep - 1) / (512 * g.keep);
    g.groups = kRowThreads / 64 / g.waves;
    const uint64_t want = sums ? 512 : 4096;                   // workgroups
    g.each = (uint32_t)((rows + want * g.groups - 1) / (want * g.groups)) * g.groups;
    if (rows <= 4 * g.groups) g.each = 4 * g.groups;           // (few rows: no second launch)
  } else {
    const uint64_t blocks_n = (p.N + 255) / 256;
    g.each = 64;
    while (g.each < rows && (rows + g.each - 1) / g.each * blocks_n > 4096) g.each *= 2;
  }
  if (!g.each) g.each = 8;
  g.blocks = rows ? (uint32_t)((rows + g.each - 1) / g.each) : 1;           // (of no rows the sums are 0)
  return g;
}

template <class TX, class TG>
hipError_t launch_rows(const NormGrad& p, const GradPlan& g, float* partial, hipStream_t st) {
  return in_launches(g.blocks, [&](uint64_t first, uint32_t n) {
    const auto go = [&](auto kernel) { kernel<<<n, g.groups * g.waves * 64, 0, st>>>(p, g.waves, g.each, (uint32_t)first, g.blocks > 1 ? partial : nullptr); };
    switch (g.keep) {
      case 1: return go(norm_grad_rows_kernel<TX, TG, 1>);
      case 2: return go(norm_grad_rows_kernel<TX, TG, 2>);
      default: return go(norm_grad_rows_kernel<TX, TG, 4>);
    }
  });
}

}  // namespace

hipError_t launch_norm(const NormRows& p, hipStream_t st) {
  if (!p.N) return hipSuccess;
  return in_launches((uint64_t)p.batches * p.M, [&](uint64_t first, uint32_t n) { norm_kernel<<<n, kThreads, 0, st>>>(p, (uint32_t)first); });
}

uint64_t norm_grad_bytes(const NormGrad& p) {
  if (!p.dweight && !p.dbias) return 0;
  const GradPlan g = plan_grad(p);
  return g.blocks > 1 ? (uint64_t)g.blocks * 2 * p.N * 4 : 0;
}

hipError_t launch_norm_grad(const NormGrad& p, float* partial, hipStream_t st) {
  const bool sums = p.dweight || p.dbias;
  if (!p.N || (!sums && !p.dx.data)) return hipSuccess;
  const GradPlan g = plan_grad(p);
  hipError_t e = hipSuccess;
  if (g.keep) {
    if (p.x.bf16) e = p.grad.bf16 ? launch_rows<bf16, bf16>(p, g, partial, st) : launch_rows<bf16, float>(p, g, partial, st);
    else e = p.grad.bf16 ? launch_rows<float, bf16>(p, g, partial, st) : launch_rows<float, float>(p, g, partial, st);
  } else {
    // (the sums first: d_x may be x or grad itself)
    if (sums) e = in_launches((uint64_t)g.blocks * ((p.N + 255) / 256), [&](uint64_t first, uint32_t n) {
      norm_columns_kernel<<<n, 256, 0, st>>>(p, g.each, (uint32_t)first, g.blocks > 1 ? partial : nullptr);
    });
    if (e == hipSuccess && p.dx.data)
      e = in_launches((uint64_t)p.batches * p.M, [&](uint64_t first, uint32_t n) { norm_grad_kernel<<<n, kThreads, 0, st>>>(p, (uint32_t)first); });
  }
  if (e == hipSuccess && sums && g.blocks > 1) {
    norm_sums_kernel<<<(uint32_t)((2ull * p.N + 31) / 32), 1024, 0, st>>>(p, g.blocks, partial);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace mrl
